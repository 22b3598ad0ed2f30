"""GPU tests of rotary positions and of the paged 8-bit cache against the float64 definitions of oracle/serving_ref.py.

Tolerances count roundings: half a step of bf16 is 2^-8 relative, of a half 2^-11, of fp32 2^-24."""
import math

import numpy as np
import pytest

from oracle import serving_ref as R
from paper_2602_21788_b200 import build, fcp

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

BF16, HALF, F32 = 2.0 ** -8, 2.0 ** -11, 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build()
    torch.cuda.set_device(0)


def dev(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a)).to(dtype).cuda()


def bf16(rng, *shape, scale=1.0):
    return torch.as_tensor(rng.standard_normal(shape) * scale).to(torch.bfloat16)


def f64(t):
    return t.detach().double().cpu().numpy()


def stream():
    return torch.cuda.current_stream().cuda_stream


# ---------------------------------------------------------------------------------------------------------
# Rotary positions
# ---------------------------------------------------------------------------------------------------------
def check_rope(got, x, positions, freqs, rotary, layout, magnitude, backward=False):
    x = f64(x)
    want = R.rope(x, positions, freqs, rotary, layout, magnitude, backward)
    pair = np.abs(x).max(axis=-1, keepdims=True) * 2 * magnitude        # bounds |x| + |y| of any pair
    # the angle is exact to 2^-24 of a half turn, sine and cosine to a few 2^-24, then two products and a sum in fp32
    assert np.all(np.abs(f64(got) - want) <= BF16 * np.abs(want) + 24 * F32 * pair + 1e-40)
    assert np.array_equal(f64(got)[..., rotary:], x[..., rotary:])


@pytest.mark.parametrize("head_dim,rotary", [(64, 64), (64, 32), (64, 2), (64, 30), (128, 128), (128, 64), (128, 126), (128, 16), (128, 48)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("backward", [False, True])
def test_rope_packed_batch(head_dim, rotary, layout, backward):
    rng = np.random.default_rng(head_dim + rotary)
    off = np.cumsum([0, 1, 0, 37, 5, 0, 300, 2])
    T, hq, hkv = int(off[-1]), 6, 2
    table = fcp.RopeTable(head_dim, rotary, layout, base=10000.0, scaling="yarn", factor=4.0, original_length=2048.0)
    freqs, m = R.rope_frequencies(rotary, 10000.0, "yarn", 4.0, 2048.0), R.rope_magnitude("yarn", 4.0)
    q, k = bf16(rng, T, hq, head_dim).cuda(), bf16(rng, T, hkv, head_dim).cuda()
    q_out, k_out = torch.full_like(q, 7), torch.full_like(k, 7)
    call = fcp.fcp_rope_bwd if backward else fcp.fcp_rope_fwd
    call(table, q, k, q_out, k_out, row_offset=dev(off), stream=stream())
    pos = np.concatenate([np.arange(b - a) for a, b in zip(off, off[1:])])
    check_rope(q_out, q, pos, freqs, rotary, layout, m, backward)
    check_rope(k_out, k, pos, freqs, rotary, layout, m, backward)
    # positions of sequences that go on, in place, on slices of wider rows
    length = np.diff(off) + np.asarray([100000, 5, 0, 2 ** 31 - 400, 3, 1, 70000])
    wide = torch.full((T, hq + 2 * hkv, head_dim), 3.0, dtype=torch.bfloat16, device="cuda")
    wide[:, :hq], wide[:, hq:hq + hkv] = q, k
    call(table, wide[:, :hq], wide[:, hq:hq + hkv], wide[:, :hq], wide[:, hq:hq + hkv], row_offset=dev(off), length=dev(length), stream=stream())
    far = np.concatenate([np.arange(b - a) + int(n) - (b - a) for a, b, n in zip(off, off[1:], length)])
    check_rope(wide[:, :hq], q, far, freqs, rotary, layout, m, backward)
    check_rope(wide[:, hq:hq + hkv], k, far, freqs, rotary, layout, m, backward)
    assert bool((wide[:, hq + hkv:] == 3).all())
    # given positions, negative ones among them; one tensor alone; rows at an address that allows no wide access
    pos = rng.integers(-2 ** 31, 2 ** 31, T)
    buf = torch.zeros(T * hkv * head_dim + 1, dtype=torch.bfloat16, device="cuda")
    odd = buf[1:].view(T, hkv, head_dim)
    call(table, None, k, None, odd, positions=dev(pos), stream=stream())
    check_rope(odd, k, pos, freqs, rotary, layout, m, backward)
    call(table, q, None, q_out, None, positions=dev(pos), stream=stream())
    check_rope(q_out, q, pos, freqs, rotary, layout, m, backward)


@pytest.mark.parametrize("T", [1, 3, 591, 592, 593, 2000])
def test_rope_rows_behind_the_batch_stay(T):
    rng = np.random.default_rng(T)
    q = bf16(rng, T + 3, 2, 64).cuda()
    table, out = fcp.RopeTable(64), torch.full((T + 3, 2, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    first = min(2, T - 1)
    fcp.fcp_rope_fwd(table, q, None, out, None, row_offset=dev([first, T]), stream=stream())
    assert bool((out[T:] == 5).all()) and bool((out[:first] == 5).all())
    check_rope(out[first:T], q[first:T], np.arange(T - first), R.rope_frequencies(64, 10000.0), 64, "half", 1.0)


def test_rope_many_sequences_and_offsets_that_make_no_sense():
    rng = np.random.default_rng(5)
    n = rng.integers(0, 3, 70001)
    off = np.concatenate([[0], np.cumsum(n)])
    T = int(off[-1])
    q = bf16(rng, T, 1, 64).cuda()
    table, out = fcp.RopeTable(64), torch.empty_like(q)
    fcp.fcp_rope_fwd(table, q, None, out, None, row_offset=dev(off), stream=stream())
    pos = np.concatenate([np.arange(i) for i in n])
    check_rope(out, q, pos, R.rope_frequencies(64, 10000.0), 64, "half", 1.0)
    # falling or far offsets: whatever comes out, the call ends and stays inside its tensors
    for bad in ([5, 3, 1, 0], [-2 ** 31, 2 ** 31 - 1, -5, 7], [2 ** 31 - 1] * 4):
        guard = torch.full((T + 64, 1, 64), 9.0, dtype=torch.bfloat16, device="cuda")
        fcp.fcp_rope_fwd(table, q, None, guard[:T], None, row_offset=dev(bad), stream=stream())
        torch.cuda.synchronize()
        assert bool((guard[T:] == 9).all())


def test_rope_gradient_is_that_of_the_forward_call():
    rng = np.random.default_rng(6)
    T, rotary = 40, 32
    table = fcp.RopeTable(64, rotary, "interleaved", scaling="linear", factor=2.0)
    pos = dev(rng.integers(0, 500, T))
    x, g = bf16(rng, T, 2, 64).cuda(), bf16(rng, T, 2, 64).cuda()
    y, dx = torch.empty_like(x), torch.empty_like(x)
    fcp.fcp_rope_fwd(table, x, None, y, None, positions=pos, stream=stream())
    fcp.fcp_rope_bwd(table, g, None, dx, None, positions=pos, stream=stream())
    # the map is linear: <dx, e> is the difference <g, rope(x + e) - rope(x)> in float64
    f, p = R.rope_frequencies(rotary, 10000.0, "linear", 2.0), pos.cpu().numpy()
    for _ in range(8):
        e = rng.standard_normal((T, 2, 64))
        rise = (f64(g) * (R.rope(f64(x) + e, p, f, rotary, "interleaved") - R.rope(f64(x), p, f, rotary, "interleaved"))).sum()
        assert abs((f64(dx) * e).sum() - rise) <= 2 * BF16 * np.abs(f64(dx) * e).sum() + 1e-9
    # forward and backward undo each other to two roundings
    fcp.fcp_rope_bwd(table, y, None, y, None, positions=pos, stream=stream())
    assert np.all(np.abs(f64(y) - f64(x)) <= 4 * BF16 * np.abs(f64(x)).max(axis=-1, keepdims=True))


# ---------------------------------------------------------------------------------------------------------
# The cache
# ---------------------------------------------------------------------------------------------------------
class World:
    """A cache on the device and the same in float64, with a pool of pages in random order."""

    def __init__(self, seed, kind, page, hkv, d, lengths, weight=True, spare=4, width=None):
        self.rng = rng = np.random.default_rng(seed)
        self.kind, self.page, self.hkv, self.d = kind, page, hkv, d
        need = [-(-n // page) for n in lengths]
        self.width = max([width or 1] + need)
        self.n_pages = sum(need) + spare
        self.order = rng.permutation(self.n_pages)
        self.table = np.full((len(lengths), self.width), -1)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = self.order[at:at + n]
            at += n
        self.free = self.order[at:]
        self.length = np.asarray(lengths)
        shape = (self.n_pages, hkv, page, d)
        self.codes = {n: rng.integers(0, 256, shape).astype(np.uint8) for n in "kv"}       # every code, NaN too
        self.scale = {n: (2.0 ** rng.integers(-9, -2, shape[:2])).astype(np.float32) for n in "kv"}
        self.weight = rng.random(shape[:3]).astype(np.float32) if weight else None

    def fill(self, spread=1.0):
        """Finite values where tokens are; the rest of the pages holds anything."""
        for b, n in enumerate(self.length):
            for j in range(-(-n // self.page)):
                p, m = self.table[b, j], min(self.page, n - j * self.page)
                for name in "kv":
                    x = self.rng.standard_normal((self.hkv, m, self.d)) * spread
                    top = np.abs(x).max(axis=(1, 2))
                    s = 2.0 ** np.ceil(np.log2(top / R.TOP[self.kind]))
                    x = torch.as_tensor(x / s[:, None, None])
                    c = x.float().to(torch.float8_e4m3fn).view(torch.uint8) if self.kind == "e4m3" else x.round().to(torch.int8).view(torch.uint8)
                    self.codes[name][p, :, :m] = c.numpy()
                    self.scale[name][p] = s
        return self

    def up(self):
        self.k, self.v = (torch.as_tensor(self.codes[n]).cuda() for n in "kv")
        self.ks, self.vs = (torch.as_tensor(self.scale[n]).cuda() for n in "kv")
        self.w = None if self.weight is None else torch.as_tensor(self.weight).cuda()
        self.status = torch.zeros(4, dtype=torch.int32, device="cuda")
        self.cache = fcp.Cache(self.k, self.v, self.ks, self.vs, self.status, weight=self.w, kind=self.kind)
        return self

    def batch(self, new, rows=None, max_new=None, length=None):
        self.off = np.concatenate([[0], np.cumsum(new)])
        rows = int(self.off[-1]) if rows is None else rows
        return fcp.CacheBatch(dev(self.table), dev(self.length if length is None else length), dev(self.off), rows=rows,
                              max_new=int(max(list(new) + [0])) if max_new is None else max_new)

    def state(self):
        return dict(k=R.code_values(self.kind, self.codes["k"]), v=R.code_values(self.kind, self.codes["v"]),
                    k_scale=self.scale["k"].astype(np.float64), v_scale=self.scale["v"].astype(np.float64),
                    weight=None if self.weight is None else self.weight.astype(np.float64))

    def now(self):
        k, v = self.k.view(torch.uint8).cpu().numpy(), self.v.view(torch.uint8).cpu().numpy()
        return dict(k=R.code_values(self.kind, k), v=R.code_values(self.kind, v), k_scale=f64(self.ks), v_scale=f64(self.vs),
                    weight=None if self.w is None else f64(self.w))


def same(a, b):
    for n in a:
        assert (a[n] is None) == (b[n] is None)
        if a[n] is not None:
            assert np.array_equal(a[n], b[n], equal_nan=True), n


CASES = [("e4m3", 16, 2, 64), ("int8", 16, 1, 128), ("e4m3", 32, 3, 128), ("int8", 64, 2, 64), ("e4m3", 128, 2, 128), ("int8", 128, 2, 128),
         ("e4m3", 128, 1, 64)]


@pytest.mark.parametrize("kind,page,hkv,d", CASES)
@pytest.mark.parametrize("new", [[1], [1, 1, 1, 0, 1], [0, 0], [5, 0, 130, 1, 63], [300, 17, 1]])
def test_append_bit_for_bit(kind, page, hkv, d, new):
    rng = np.random.default_rng(len(new))
    before = [int(rng.integers(0, 3 * page)) if b % 3 else [0, page, page - 1, 2 * page + 1][b % 4] for b in range(len(new))]
    w = World(11, kind, page, hkv, d, [a + n for a, n in zip(before, new)])
    # a clean start: stale NaN codes may lie in pages, but the earlier tokens are values
    for n in "kv":
        w.codes[n] = np.where((w.codes[n] & 127) == 127, 3, w.codes[n]).astype(np.uint8) if kind == "e4m3" else np.where(w.codes[n] == 128, 3, w.codes[n]).astype(np.uint8)
    w.up()
    rows = int(np.sum(new))
    # sizes from far below to far above what the pages hold
    k = (bf16(w.rng, rows + 2, hkv, d) * torch.as_tensor(2.0 ** w.rng.integers(-12, 6, (rows + 2, hkv, 1)))).to(torch.bfloat16)
    v = bf16(w.rng, rows + 2, hkv, d)
    batch = w.batch(new, rows=rows + 2, max_new=max(new))
    state = w.state()
    fcp.fcp_cache_append(w.cache, batch, k.cuda(), v.cuda(), stream=stream())
    R.append(kind, state, w.table, w.length, w.off, f64(k), f64(v))
    same(w.now(), state)
    fcp.fcp_cache_append(w.cache, batch, k.cuda(), v.cuda(), stream=stream())           # again: nothing changes
    same(w.now(), state)
    assert w.cache.device_status().tolist() == [0, 0, 0, 0]


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_append_of_unusual_values(kind):
    w = World(12, kind, 16, 1, 64, [16, 20, 16, 3, 7, 2])
    w.up()
    new = [16, 4, 16, 3, 1, 2]
    x = torch.zeros(sum(new), 1, 64)
    x[0:16] = torch.tensor([float("inf"), -float("inf"), float("nan"), 3e38]).repeat(16)
    x[16:20] = 0.0
    x[20:36] = 1e-38
    x[36:39] = float("nan")
    x[39] = -448 * 2.0 ** 20
    x[40:42, 0, 0] = 127 * 2.0 ** -130            # a subnormal bf16
    x = x.to(torch.bfloat16)
    state = w.state()
    for n in "kv":
        state[n][w.table[1][1]], w.codes[n][w.table[1][1]] = 0, 0                       # its earlier tokens
        state[n][w.table[4][0]], w.codes[n][w.table[4][0]] = 1.0, 0x38 if kind == "e4m3" else 1
    w.up()
    batch = w.batch(new)
    fcp.fcp_cache_append(w.cache, batch, x.cuda(), x.cuda(), stream=stream())
    R.append(kind, state, w.table, w.length, w.off, f64(x), f64(x))
    same(w.now(), state)


def test_append_scales_that_are_no_powers_of_two():
    w = World(13, "int8", 32, 2, 64, [40, 9])
    for n in "kv":
        w.scale[n] = w.rng.random(w.scale[n].shape).astype(np.float32)
        w.codes[n] = np.where(w.codes[n] == 128, 0, w.codes[n]).astype(np.uint8)
    w.up()
    x = bf16(w.rng, 5, 2, 64, scale=20)
    state = w.state()
    fcp.fcp_cache_append(w.cache, w.batch([4, 1]), x.cuda(), x.cuda(), stream=stream())
    R.append("int8", state, w.table, w.length, w.off, f64(x), f64(x))
    now = w.now()
    assert np.array_equal(now["k_scale"], state["k_scale"])
    # x / scale is rounded to fp32 before it is rounded to a code: at most one code apart, and only next to a border
    for n in "kv":
        assert np.abs(now[n] - state[n]).max() <= 1 and (now[n] != state[n]).mean() < 1e-3


def goes_by_copies(w, new, hq):
    """Whether a call with these new tokens asks for room for bf16 copies of all keys and values, besides the partial results."""
    rows = max(new) * hq // w.hkv
    tile = next((t for t in (8, 16, 32) if rows <= t), 128)
    partial, copies = 2 * 148 * tile * (w.d + 1) * 4, len(new) * w.width * w.page * w.hkv * w.d * 4
    return fcp.fcp_cache_attn_workspace_bytes(w.cache, w.batch(new), hq) >= partial + copies


def check_attn(w, state, r, o, lse, rows, weight=HALF, lost=0.0):
    """Against the definition: the rounding of the weights (to halves 2^-11; in calls that go by copies to bf16, 2^-8), of o to bf16 (2^-8), and the fp32 sums of the scores (D products of size at most `size` in all, each sum truncated at 2^-23)."""
    off = w.off
    for name, x in (("o", o), ("lse", lse)):
        assert x.shape[0] >= rows
    score = w.d * 2 * F32 * r["size"] + 2.0 ** -20
    got, got_lse = f64(o)[:rows], f64(lse)[:rows]
    dead = ~np.isfinite(r["lse"])
    assert np.array_equal(dead, got_lse == -np.inf)
    assert np.all(got[dead] == 0)
    live = ~dead
    assert np.all(np.abs(got_lse[live] - r["lse"][live]) <= (score + 4 * F32 * np.abs(np.where(live, r["lse"], 0)))[live])
    bound = BF16 * np.abs(r["o"]) + (weight + 2 * score[..., None]) * r["spread"] * (1 + BF16) + lost + 1e-30
    assert np.all(np.abs(got - r["o"]) <= bound), np.max(np.abs(got - r["o"]) / bound)
    assert off[-1] == rows


def attend(w, new, hq, accumulate=False, scale=0.0, spare=2, stride_heads=0, max_new=None):
    rows = int(np.sum(new))
    q = bf16(w.rng, rows + spare, hq + stride_heads, w.d)[:, :hq]
    batch = w.batch(new, rows=rows + spare, max_new=max_new)
    o = torch.full((rows + spare, hq, w.d), 3.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((rows + spare, hq), 5.0, device="cuda")
    n = fcp.fcp_cache_attn_workspace_bytes(w.cache, batch, hq)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    q_dev = torch.zeros(rows + spare, hq + stride_heads, w.d, dtype=torch.bfloat16, device="cuda")
    q_dev[:, :hq] = q.cuda()
    fcp.fcp_cache_attn(w.cache, batch, q_dev[:, :hq], o, lse, ws, n, scale=scale, accumulate=accumulate, stream=stream())
    torch.cuda.synchronize()
    assert bool((o[rows:] == 3).all()) and bool((lse[rows:] == 5).all())
    return q, o, lse, rows


@pytest.mark.parametrize("kind,page,hkv,d", CASES)
@pytest.mark.parametrize("group,new,before", [
    (1, [1], [0]), (1, [1, 1, 1], [15, 16, 127]), (4, [1, 0, 1, 1], [700, 5, 128, 1290]), (8, [2, 2], [300, 0]),
    (5, [4, 1, 3], [1000, 64, 3]), (3, [20, 1], [250, 900]), (8, [17, 40, 2], [130, 0, 5]),
])
def test_attention_over_the_cache(kind, page, hkv, d, group, new, before):
    w = World(21, kind, page, hkv, d, [a + n for a, n in zip(before, new)]).fill().up()
    q, o, lse, rows = attend(w, new, hkv * group, stride_heads=1)
    r = R.attention(w.state(), w.table, w.length, w.off, f64(q)[:rows])
    check_attn(w, None, r, o, lse, rows, weight=BF16 if goes_by_copies(w, new, hkv * group) else HALF)
    assert w.cache.device_status().tolist() == [0, 0, 0, 0]


@pytest.mark.parametrize("kind,page,hkv,d", [("e4m3", 16, 2, 64), ("int8", 32, 2, 128), ("e4m3", 128, 1, 128)])
@pytest.mark.parametrize("group,new,before", [(1, [1, 1], [5, 700]), (4, [3, 0, 1], [500, 9, 0]), (8, [5, 30], [1100, 2])])
def test_weights_that_attention_leaves(kind, page, hkv, d, group, new, before):
    w = World(22, kind, page, hkv, d, [a + n for a, n in zip(before, new)]).fill().up()
    state, was = w.state(), w.now()["weight"]
    q, o, lse, rows = attend(w, new, hkv * group, accumulate=True)
    r = R.attention(state, w.table, w.length, w.off, f64(q)[:rows])
    check_attn(w, None, r, o, lse, rows)
    want, tol = was.copy(), F32 * 4 * np.abs(was) + 1e-30
    score = w.d * 2 * F32 * r["size"].max() + 2.0 ** -20
    for b, t in enumerate(w.length):
        for p in range(t):
            page_id, slot = w.table[b][p // page], p % page
            want[page_id, :, slot] += r["weights"][b][:, p]
            tol[page_id, :, slot] += r["weights"][b][:, p] * (3 * score + 64 * F32)
    now = w.now()["weight"]
    assert np.all(np.abs(now - want) <= tol)                      # places without tokens stay as they were
    # the same call on the same start gives the same bits
    w2 = World(22, kind, page, hkv, d, [a + n for a, n in zip(before, new)]).fill().up()
    attend(w2, new, hkv * group, accumulate=True)
    assert np.array_equal(w2.now()["weight"], now)


def test_long_ragged_batch_is_split_and_joined():
    lengths = [20011, 1, 130, 0, 4097, 33, 700]
    w = World(23, "e4m3", 16, 2, 128, lengths).fill().up()
    new = [1, 1, 1, 0, 1, 1, 1]
    q, o, lse, rows = attend(w, new, 8)
    r = R.attention(w.state(), w.table, w.length, w.off, f64(q)[:rows])
    check_attn(w, None, r, o, lse, rows)
    a, b = o.clone(), lse.clone()
    w.rng = np.random.default_rng(99)
    q1, o1, lse1, _ = attend(w, new, 8)
    w.rng = np.random.default_rng(99)
    q2, o2, lse2, _ = attend(w, new, 8)
    assert torch.equal(o1, o2) and torch.equal(lse1, lse2) and not torch.equal(o1, a)


@pytest.mark.parametrize("kind,page,d", [("e4m3", 16, 64), ("int8", 16, 128), ("e4m3", 32, 128), ("int8", 64, 64), ("e4m3", 128, 128), ("int8", 128, 128)])
@pytest.mark.parametrize("hkv,group,new,before", [(8, 8, [300], [0]), (8, 8, [257, 0, 1], [70, 300, 5]), (8, 6, [300, 40, 257], [129, 0, 300])])
def test_attention_of_long_chunks(kind, page, d, hkv, group, new, before):
    w = World(71, kind, page, hkv, d, [a + n for a, n in zip(before, new)]).fill().up()
    assert goes_by_copies(w, new, hkv * group)
    q, o, lse, rows = attend(w, new, hkv * group, stride_heads=1, accumulate=True)
    r = R.attention(w.state(), w.table, w.length, w.off, f64(q)[:rows])
    check_attn(w, None, r, o, lse, rows, weight=BF16)
    assert w.cache.device_status().tolist() == [0, 0, 0, 0]
    assert math.isclose(float(w.w.double().sum()) - float(w.weight.astype(np.float64).sum()), rows * hkv * group, rel_tol=1e-4)
    w.rng = np.random.default_rng(5)
    q1, o1, lse1, _ = attend(w, new, hkv * group)
    w.rng = np.random.default_rng(5)
    q2, o2, lse2, _ = attend(w, new, hkv * group)
    assert torch.equal(o1, o2) and torch.equal(lse1, lse2)


@pytest.mark.parametrize("kind,page,hkv,d", CASES)
@pytest.mark.parametrize("group,new,before", [(1, [33, 0, 128], [0, 40, 500]), (4, [9, 1, 31, 0], [1500, 3, 130, 64]), (2, [200], [500]), (8, [16, 16, 1], [127, 5, 2000])])
def test_many_rows_without_copies(kind, page, hkv, d, group, new, before):
    """More than 32 rows per KV head, up to and beyond a tile of 128, few enough in all that no copies are made."""
    w = World(74, kind, page, hkv, d, [a + n for a, n in zip(before, new)]).fill().up()
    assert not goes_by_copies(w, new, hkv * group)
    q, o, lse, rows = attend(w, new, hkv * group, accumulate=True)
    r = R.attention(w.state(), w.table, w.length, w.off, f64(q)[:rows])
    check_attn(w, None, r, o, lse, rows)


def test_chunk_of_a_wide_table_is_captured_and_replayed():
    """Lengths of a captured chunk change; the table is far wider than the sequences."""
    w = World(72, "e4m3", 32, 8, 64, [500, 400], width=64).fill().up()
    hq, rows = 32, 300
    length, off = dev([0, 0]), dev([0, 0, 0])
    q = torch.zeros(rows, hq, 64, dtype=torch.bfloat16, device="cuda")
    o, lse = torch.zeros_like(q), torch.zeros(rows, hq, device="cuda")
    batch = fcp.CacheBatch(dev(w.table), length, off, rows=rows, max_new=260)
    assert goes_by_copies(w, [260, 40], hq)
    n = fcp.fcp_cache_attn_workspace_bytes(w.cache, batch, hq)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    step = lambda: fcp.fcp_cache_attn(w.cache, batch, q, o, lse, ws, n, stream=stream())
    with torch.cuda.stream(torch.cuda.Stream()):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lengths, new in [([500, 400], [130, 170]), ([260, 0], [260, 0]), ([3, 399], [3, 1])]:
        xq = bf16(w.rng, rows, hq, 64)
        q.copy_(xq), o.fill_(3.0)
        w.off = np.concatenate([[0], np.cumsum(new)])
        length.copy_(dev(lengths)), off.copy_(dev(w.off))
        graph.replay()
        torch.cuda.synchronize()
        m = int(w.off[-1])
        r = R.attention(w.state(), w.table, lengths, w.off, f64(xq)[:m])
        check_attn(w, None, r, o[:m], lse[:m], m, weight=BF16)
        assert bool((o[m:] == 3).all())


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_chunks_with_sequences_that_need_care(kind):
    """In one call with ordinary sequences: a NaN among the new values, more rows than tokens, a page that does not exist, lengths
    that make no sense."""
    new, hkv, group = [140, 150, 133, 20, 200], 4, 8
    w = World(73, kind, 16, hkv, 64, [300, 90, 200, 100, 260]).fill()
    if kind == "e4m3":
        w.codes["v"][w.table[0][290 // 16], 1, 290 % 16, 7] = 0xff
    good = w.state()
    table = w.table.copy()
    w.table[2, 1] = w.n_pages + 5
    w.up()
    assert goes_by_copies(w, new, hkv * group)
    w.length[4] = 10 ** 6
    q, o, lse, rows = attend(w, new, hkv * group, spare=0)
    w.length[4] = 260
    off = w.off
    with np.errstate(invalid="ignore"):
        r = R.attention(good, table, w.length, off, f64(q)[:rows])
    got, got_lse = f64(o), f64(lse)
    st = w.cache.device_status().tolist()
    assert st[0] == fcp.FCP_ERR_INVALID_ARG and st[1:3] in ([fcp.FCP_CACHE_BAD_LENGTH, 4], [fcp.FCP_CACHE_BAD_PAGE, 2])
    assert np.all(got[off[4]:] == 3) and np.all(got_lse[off[4]:] == 5)
    # sequence 2 without its tokens 16..31
    for j in (0, 70, 132):
        for head in range(hkv * group):
            k = R.gather(good, "k", np.asarray(table[2][:13], dtype=np.int64), 200, head // group)
            seen = [p for p in range(200 - 133 + j + 1) if not 16 <= p < 32]
            s = k[seen] @ f64(q)[off[2] + j, head] / 8
            assert abs(got_lse[off[2] + j, head] - np.log(np.exp(s).sum())) < 1e-3
    for b in (0, 1, 3):
        for row in range(off[b], off[b + 1]):
            bad = np.isnan(r["o"][row])
            assert np.array_equal(np.isnan(got[row]), bad), (b, row)
            ok = ~bad
            assert np.all(np.abs(got[row] - r["o"][row])[ok] <= (2 * BF16 * np.abs(r["o"][row]) + 2 * BF16 * r["spread"][row])[ok])
    assert np.isneginf(got_lse[off[1]:off[1] + 60]).all() and np.all(got[off[1]:off[1] + 60] == 0)


def test_many_sequences():
    rng = np.random.default_rng(3)
    lengths = rng.integers(0, 40, 700)
    lengths[::7] = 0
    w = World(24, "int8", 16, 1, 64, lengths).fill().up()
    new = np.minimum(lengths, 1)
    new[5::70] = 0
    q, o, lse, rows = attend(w, new, 2)
    r = R.attention(w.state(), w.table, w.length, w.off, f64(q)[:rows])
    check_attn(w, None, r, o, lse, rows)


def test_rows_that_see_nothing():
    w = World(25, "e4m3", 16, 2, 64, [0, 3, 0]).fill().up()
    q, o, lse, rows = attend(w, [2, 5, 1], 4, accumulate=True)    # more new rows than tokens: the first ones are no tokens
    r = R.attention(w.state(), w.table, w.length, w.off, f64(q)[:rows])
    assert np.isneginf(r["lse"]).sum() == 4 * 5
    check_attn(w, None, r, o, lse, rows)
    added = f64(w.w) - w.weight
    assert np.isfinite(added).all() and math.isclose(added.sum(), 4 * 3, rel_tol=1e-5)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_tiles_of_rows_that_see_nothing_or_differ_in_size(kind):
    """40 rows and more: more new rows than tokens, no tokens at all, queries and scales of very different size; the same bits again."""
    w = World(29, kind, 16, 1, 64, [0, 13, 300]).fill()
    for i, p in enumerate(w.table[2]):
        if p >= 0:
            w.scale["v"][p] *= 2.0 ** (-40 + 4 * (i % 20))
            w.scale["k"][p] *= 2.0 ** -(i % 5)
    w.up()
    new, rows = [40, 50, 45], 135
    q = bf16(w.rng, rows, 1, 64)
    q[::7] *= 2.0 ** -130
    q[3::7] *= 2.0 ** 6
    q[5::7] = 0
    batch = w.batch(new)
    assert not goes_by_copies(w, new, 1)
    n = fcp.fcp_cache_attn_workspace_bytes(w.cache, batch, 1)
    both = []
    for _ in range(2):
        o, lse = torch.empty(rows, 1, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(rows, 1, device="cuda")
        ws = torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255)
        fcp.fcp_cache_attn(w.cache, batch, q.cuda(), o, lse, ws, n, scale=2.0 ** -4, stream=stream())
        both.append((o, lse))
    r = R.attention(w.state(), w.table, w.length, w.off, f64(q), scale=2.0 ** -4)
    assert np.isneginf(r["lse"]).sum() == 40 + 37
    # A half rounds below 2^-14 in steps of 2^-24, an error of 2^-25, and the row's largest product of a weight and its value scale is
    # held as 2^8 or more: every code is off by at most 2^-33 of that product.
    lost = np.zeros((rows, 1, 64))
    state = w.state()
    for b in (1, 2):
        t = w.length[b]
        pages = np.asarray(w.table[b][:-(-t // 16)])
        k, code = R.gather(state, "k", pages, t, 0), state["v"][pages, 0].reshape(-1, 64)[:t]
        scale = np.repeat(state["v_scale"][pages, 0], 16)[:t]
        for j in range(max(0, new[b] - t), new[b]):
            row, seen = w.off[b] + j, t - new[b] + j + 1
            s = k[:seen] @ f64(q)[row, 0] * 2.0 ** -4
            lost[row, 0] = 2.0 ** -33 * (np.exp(s - r["lse"][row, 0]) * scale[:seen]).max() * np.abs(code[:seen]).sum(axis=0)
    check_attn(w, None, r, o, lse, rows, lost=lost)
    assert all(torch.equal(a, b) for a, b in zip(*both))


@pytest.mark.parametrize("new", [1, 6, 12, 40])
def test_nan_values_behind_and_among_the_new_tokens(new):
    """What no row may see must not reach it: stale NaN codes behind the length, and a NaN key or value of a later new token."""
    w = World(26, "e4m3", 16, 1, 128, [117 + new, 64 + new]).fill()
    place = lambda b, p: (w.table[b][p // 16], 0, p % 16)
    at = 117 + max(new - 3, 0)
    w.codes["v"][place(0, at)][::5] = 0x7f
    w.codes["k"][place(1, 64 + new - 1)][3] = 0xff
    w.up()
    q, o, lse, rows = attend(w, [new, new], 2)
    with np.errstate(invalid="ignore"):
        r = R.attention(w.state(), w.table, w.length, w.off, f64(q)[:rows])
    first = at - 117                                              # row of sequence 0 that first sees the NaN value
    got = f64(o)[:rows]
    assert np.isnan(got[first:new, :, ::5]).all()
    assert np.isnan(got[2 * new - 1]).all() and np.isnan(f64(lse)[2 * new - 1]).all()
    rest = np.ones(got.shape, bool)
    rest[first:new, :, ::5] = False
    rest[2 * new - 1] = False
    assert not np.isnan(got[rest]).any()
    assert np.all(np.abs(got - r["o"])[rest] <= (BF16 * np.abs(r["o"]) + 2 * HALF * np.nan_to_num(r["spread"], nan=1.0) + 1e-3 * np.nan_to_num(r["spread"], nan=1.0))[rest])


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_scales_of_very_different_size(kind):
    w = World(27, kind, 16, 1, 64, [400]).fill()
    for i, p in enumerate(w.table[0]):
        w.scale["v"][p] *= 2.0 ** (-40 + 4 * (i % 20))
        w.scale["k"][p] *= 2.0 ** -(i % 5)
    w.up()
    q, o, lse, rows = attend(w, [1], 3)
    r = R.attention(w.state(), w.table, w.length, w.off, f64(q)[:rows])
    check_attn(w, None, r, o, lse, rows)


def test_queries_of_unusual_size():
    w = World(28, "int8", 16, 1, 64, [50, 50, 50, 50]).fill().up()
    rows = 4
    q = bf16(w.rng, rows, 1, 64)
    q[0] *= 2.0 ** -130
    q[1] *= 2.0 ** 12
    q[2] = 0
    q[3, 0, 0] = 2.0 ** 9                                         # one large column, the others 2^-20 and less of it
    q[3, 0, 1:] *= 2.0 ** -12
    batch = w.batch([1] * 4)
    o, lse = torch.empty(4, 1, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(4, 1, device="cuda")
    n = fcp.fcp_cache_attn_workspace_bytes(w.cache, batch, 1)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    fcp.fcp_cache_attn(w.cache, batch, q.cuda(), o, lse, ws, n, scale=2.0 ** -6, stream=stream())
    r = R.attention(w.state(), w.table, w.length, w.off, f64(q), scale=2.0 ** -6)
    check_attn(w, None, r, o, lse, rows)


def test_what_the_kernels_refuse():
    """Pages that do not exist, scales out of range, lengths and rows that make no sense: absent, with a status; the rest is right."""
    w = World(31, "e4m3", 16, 2, 64, [100, 64, 33, 20, 10]).fill()
    good = World(31, "e4m3", 16, 2, 64, [100, 64, 33, 20, 10]).fill()

    def attn(length, off, rows=6, max_new=2):
        batch = fcp.CacheBatch(dev(w.table), dev(length), dev(off), rows=rows, max_new=max_new)
        o = torch.full((rows, 4, 64), 3.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((rows, 4), 5.0, device="cuda")
        n = fcp.fcp_cache_attn_workspace_bytes(w.cache, batch, 4)
        fcp.fcp_cache_attn(w.cache, batch, q, o, lse, torch.empty(n, dtype=torch.uint8, device="cuda"), n, accumulate=True, stream=stream())
        return f64(o), f64(lse)
    q = bf16(w.rng, 6, 4, 64).cuda()
    ref = R.attention(good.state(), good.table, good.length, [0, 1, 2, 3, 4, 5], f64(q))
    bad_rows = lambda got, rows: [i for i in rows if not np.allclose(got[1][i], ref["lse"][i], atol=1e-4)]
    for length, off, code, seq, untouched in [
        ([100, 64, 33, -1, 10], [0, 1, 2, 3, 4, 5], fcp.FCP_CACHE_BAD_LENGTH, 3, [3]),
        ([100, 10 ** 6, 33, 20, 10], [0, 1, 2, 3, 4, 5], fcp.FCP_CACHE_BAD_LENGTH, 1, [1]),
        ([100, 64, 33, 20, 10], [0, 1, 2, 3, 4, 7], fcp.FCP_CACHE_BAD_ROWS, 4, [4, 5]),
    ]:
        w.up()
        got = attn(length, off)
        assert w.cache.device_status().tolist()[:3] == [fcp.FCP_ERR_INVALID_ARG, code, seq]
        assert np.all(got[0][untouched] == 3) and np.all(got[1][untouched] == 5)
        assert bad_rows(got, [i for i in range(5) if i not in untouched]) == []
    w.up()
    got = attn([100, 64, 33, 20, 10], [5, 4, 4, 4, 4, 4])                               # falling offsets, then nothing
    assert w.cache.device_status().tolist()[:3] == [fcp.FCP_ERR_INVALID_ARG, fcp.FCP_CACHE_BAD_ROWS, 0]
    assert np.all(got[0] == 3)
    for page in (-1, w.n_pages, 2 ** 31 - 1, -2 ** 31):
        for name, bad in (("page", page), ("scale", 0.0), ("scale", float("nan")), ("scale", -1.0), ("scale", 1e38)):
            if name == "scale" and page != -1:
                continue
            keep, w.scale["k"] = w.table.copy(), w.scale["k"].copy()
            if name == "page":
                w.table[0, 2] = bad
            else:
                w.scale["v"], saved = w.scale["v"].copy(), w.scale["v"].copy()
                w.scale["v"][w.table[0, 2], :] = bad
            w.up()
            before = f64(w.w)
            got = attn([100, 64, 33, 20, 10], [0, 1, 2, 3, 4, 5])
            assert w.cache.device_status().tolist()[:3] == [fcp.FCP_ERR_INVALID_ARG, fcp.FCP_CACHE_BAD_PAGE if name == "page" else fcp.FCP_CACHE_BAD_SCALE, 0]
            assert bad_rows(got, [1, 2, 3, 4]) == []
            # sequence 0 without its tokens 32..47
            pages = [keep[0][i] for i in range(7) if i != 2]
            k = np.stack([R.gather(good.state(), "k", pages, 84, h) for h in range(2)])
            s = np.einsum("hd,htd->ht", f64(q)[0], np.repeat(k, 2, 0)) / 8
            assert np.allclose(got[1][0], np.log(np.exp(s).sum(-1)), atol=1e-4)
            assert np.array_equal(f64(w.w)[keep[0][2]], before[keep[0][2]])
            w.table[:] = keep
            if name == "scale":
                w.scale["v"] = saved
    # append and evict: nothing is written through a page that does not exist
    keep = w.table.copy()
    w.table[1, 3] = w.n_pages
    w.up()
    k = bf16(w.rng, 5, 2, 64).cuda()
    was = w.now()
    fcp.fcp_cache_append(w.cache, fcp.CacheBatch(dev(w.table), dev(w.length), dev([0, 1, 2, 3, 4, 5]), rows=5, max_new=1), k, k, stream=stream())
    assert w.cache.device_status().tolist()[:3] == [fcp.FCP_ERR_INVALID_ARG, fcp.FCP_CACHE_BAD_PAGE, 1]
    now = w.now()
    touched = {int(keep[b][(n - 1) // 16]) for b, n in enumerate(w.length) if b != 1}
    for p in range(w.n_pages):
        if p not in touched:
            assert np.array_equal(now["k"][p], was["k"][p], equal_nan=True) and np.array_equal(now["k_scale"][p], was["k_scale"][p])
    w.up()
    dst = dev([[-1], [int(w.free[0])]])
    new_length, kept = torch.empty(2, dtype=torch.int32, device="cuda"), torch.empty(2, 2, 12, dtype=torch.int32, device="cuda")
    fcp.fcp_cache_evict(w.cache, fcp.CacheBatch(dev(w.table[:2]), dev([100, -4])), 4, 4, 4, dst, new_length, kept, stream=stream())
    assert w.cache.device_status().tolist()[0] == fcp.FCP_ERR_INVALID_ARG
    assert new_length.tolist() == [12, 0] and bool((kept[1] == -1).all())
    same(w.now(), was)


def test_wide_offsets():
    """A pool of more than 2^32 bytes: the last pages are read and written where they are."""
    page, hkv, d, n_pages = 128, 1, 128, 300000
    k = torch.zeros((n_pages, hkv, page, d), dtype=torch.uint8, device="cuda")
    v = torch.zeros_like(k)
    ks, vs = torch.ones(n_pages, hkv, device="cuda"), torch.ones(n_pages, hkv, device="cuda")
    status, w = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.ones(n_pages, hkv, page, device="cuda")
    cache = fcp.Cache(k, v, ks, vs, status, weight=w, kind="e4m3")
    rng = np.random.default_rng(1)
    table = np.asarray([[n_pages - 1, 0, n_pages - 2]])
    x, y = bf16(rng, 300, 1, d), bf16(rng, 300, 1, d)
    batch = fcp.CacheBatch(dev(table), dev([300]), dev([0, 300]), rows=300)
    fcp.fcp_cache_append(cache, batch, x.cuda(), y.cuda(), stream=stream())
    state = dict(k=np.zeros((3, 1, page, d)), v=np.zeros((3, 1, page, d)), k_scale=np.ones((3, 1)), v_scale=np.ones((3, 1)))
    R.append("e4m3", state, [[0, 1, 2]], [300], [0, 300], f64(x), f64(y))
    at = torch.as_tensor(table[0]).cuda()
    assert np.array_equal(R.code_values("e4m3", k[at].cpu().numpy()), state["k"]) and np.array_equal(f64(vs[at]), state["v_scale"])
    q, o, lse = bf16(rng, 1, 2, d), torch.empty(1, 2, d, dtype=torch.bfloat16, device="cuda"), torch.empty(1, 2, device="cuda")
    step = fcp.CacheBatch(dev(table), dev([300]), dev([0, 1]), rows=1)
    n = fcp.fcp_cache_attn_workspace_bytes(cache, step, 2)
    fcp.fcp_cache_attn(cache, step, q.cuda(), o, lse, torch.empty(n, dtype=torch.uint8, device="cuda"), n, accumulate=True, stream=stream())
    r = R.attention(state, [[0, 1, 2]], [300], [0, 1], f64(q))
    assert np.allclose(f64(lse), r["lse"], atol=1e-4) and np.abs(f64(o) - r["o"]).max() < 0.02
    assert math.isclose(float(w.double().sum()), n_pages * page - 300 + 2, rel_tol=1e-9)      # append zeroed 300 weights, attention added 2
    dst = dev([[n_pages - 3]])
    new_length, kept = torch.empty(1, dtype=torch.int32, device="cuda"), torch.empty(1, 1, 40, dtype=torch.int32, device="cuda")
    fcp.fcp_cache_evict(cache, step, 4, 30, 6, dst, new_length, kept, stream=stream())
    assert torch.equal(k[n_pages - 3, 0, :4], k[n_pages - 1, 0, :4]) and torch.equal(v[n_pages - 3, 0, 34:40].cpu(), v[n_pages - 2, 0, 38:44].cpu())


@pytest.mark.parametrize("kind,page,hkv,d", CASES)
@pytest.mark.parametrize("sink,heavy,recent", [(4, 20, 10), (0, 37, 0), (0, 1, 0), (130, 0, 3), (1, 200, 64), (0, 0, 16)])
def test_eviction(kind, page, hkv, d, sink, heavy, recent):
    keep = sink + heavy + recent
    lengths = [keep + 1, 1000, keep, 0, 1, 333, 1500]
    need = -(-keep // page)
    w = World(41, kind, page, hkv, d, lengths, spare=len(lengths) * need + 1).fill()
    w.weight = np.where(w.rng.random(w.weight.shape) < 0.5, np.round(w.weight * 8) / 8, w.weight).astype(np.float32)       # many equal ones
    w.weight[w.table[1][0], 0, :5] = [np.nan, np.inf, -1.0, -np.inf, -0.0]
    w.weight[w.table[5][0]] = 0
    w.up()
    dst = w.free[:len(lengths) * need].reshape(len(lengths), need)
    new_length = torch.full((len(lengths),), -7, dtype=torch.int32, device="cuda")
    kept = torch.full((len(lengths), hkv, keep), -7, dtype=torch.int32, device="cuda")
    state = w.state()
    fcp.fcp_cache_evict(w.cache, fcp.CacheBatch(dev(w.table), dev(w.length)), sink, heavy, recent, dev(dst), new_length, kept, stream=stream())
    want_kept, want_length = R.evict(kind, state, w.table, w.length, sink, heavy, recent, dst)
    assert new_length.tolist() == want_length.tolist()
    assert np.array_equal(kept.cpu().numpy(), want_kept)
    same(w.now(), state)
    assert w.cache.device_status().tolist() == [0, 0, 0, 0]


@pytest.mark.parametrize("length", [49152 + 60, 49152 + 61, 90001])
def test_eviction_from_a_long_sequence(length):
    """Around as many candidates as fit shared memory, and beyond; weights that share their upper bits."""
    w = World(42, "int8", 128, 1, 64, [length], spare=120)
    w.weight = (1.0 + np.round(w.rng.random(w.weight.shape) * 5000) * 2.0 ** -23).astype(np.float32)
    w.codes = {n: np.where(c == 128, 0, c).astype(np.uint8) for n, c in w.codes.items()}
    w.up()
    dst = w.free[:118][None]
    new_length, kept = torch.empty(1, dtype=torch.int32, device="cuda"), torch.empty(1, 1, 15000, dtype=torch.int32, device="cuda")
    fcp.fcp_cache_evict(w.cache, fcp.CacheBatch(dev(w.table), dev(w.length)), 10, 14940, 50, dev(dst), new_length, kept, stream=stream())
    pos = R.choose(w.weight[w.table[0], 0].reshape(-1)[:length].tolist(), 10, 14940, 50)
    assert np.array_equal(kept.cpu().numpy()[0, 0], pos)
    src = torch.as_tensor(w.table[0][pos // 128] * 128 + pos % 128).cuda()
    to = torch.as_tensor(dst[0][np.arange(15000) // 128] * 128 + np.arange(15000) % 128).cuda()
    assert torch.equal(w.w.view(-1)[to], w.w.view(-1)[src])


# ---------------------------------------------------------------------------------------------------------
# Streams, graphs, and the calls as they are used together
# ---------------------------------------------------------------------------------------------------------
def test_captured_step_is_replayed_with_new_contents():
    """A decode step (rotary, append, attention) captured once, with row and length buffers larger than the batch it sees."""
    w = World(51, "e4m3", 16, 2, 64, [60, 30, 17, 5], width=8).fill().up()
    B, hq, table = 4, 4, fcp.RopeTable(64, 32, "interleaved")
    length, off = dev([0] * B), dev([0] * (B + 1))
    q, k, v = (torch.zeros(B, h, 64, dtype=torch.bfloat16, device="cuda") for h in (hq, 2, 2))
    o, lse = torch.zeros(B, hq, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, hq, device="cuda")
    batch = fcp.CacheBatch(dev(w.table), length, off, rows=B, max_new=1)
    n = fcp.fcp_cache_attn_workspace_bytes(w.cache, batch, hq)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")

    def step():
        s = stream()
        fcp.fcp_rope_fwd(table, q, k, q, k, row_offset=off, length=length, stream=s)
        fcp.fcp_cache_append(w.cache, batch, k, v, stream=s)
        fcp.fcp_cache_attn(w.cache, batch, q, o, lse, ws, n, accumulate=True, stream=s)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()                                                    # lengths of zero: nothing happens
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    f = R.rope_frequencies(32, 10000.0)
    for lengths in ([60, 30, 17, 5], [60, 0, 17, 1], [1, 30, 0, 0]):
        new = [int(x > 0) for x in lengths]
        rows = sum(new)
        xq, xk, xv = (bf16(w.rng, B, h, 64) for h in (hq, 2, 2))
        q.copy_(xq), k.copy_(xk), v.copy_(xv), o.fill_(3.0)
        length.copy_(dev(lengths)), off.copy_(dev(np.concatenate([[0], np.cumsum(new)])))
        state = w.now()
        graph.replay()
        torch.cuda.synchronize()
        pos = [x - 1 for x in lengths if x]
        check_rope(q[:rows], xq[:rows].cuda(), pos, f, 32, "interleaved", 1.0)
        R.append("e4m3", state, w.table, lengths, off.cpu().numpy(), f64(k), f64(v))
        now = w.now()
        for name in ("k", "v", "k_scale", "v_scale"):
            assert np.array_equal(now[name], state[name], equal_nan=True)
        w.off = off.cpu().numpy()
        r = R.attention(state, w.table, lengths, w.off, f64(q)[:rows])
        check_attn(w, None, r, o[:rows], lse[:rows], rows)
        assert bool((o[rows:] == 3).all())
    assert w.cache.device_status().tolist() == [0, 0, 0, 0]


def test_calls_on_two_streams():
    """Two batches on two caches at once, each with its own workspace."""
    worlds = [World(52 + i, "int8", 64, 2, 128, [3000, 500]).fill().up() for i in range(2)]
    want, got, streams = [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for w in worlds:
        w.q = bf16(w.rng, 2, 8, 128).cuda()
        w.b = w.batch([1, 1])
        w.n = fcp.fcp_cache_attn_workspace_bytes(w.cache, w.b, 8)
        w.ws = torch.empty(w.n, dtype=torch.uint8, device="cuda")
        o, lse = torch.empty(2, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(2, 8, device="cuda")
        fcp.fcp_cache_attn(w.cache, w.b, w.q, o, lse, w.ws, w.n, stream=stream())
        want.append((o, lse))
    torch.cuda.synchronize()
    for i in range(20):
        for w, s in zip(worlds, streams):
            o, lse = torch.empty(2, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(2, 8, device="cuda")
            s.wait_stream(torch.cuda.current_stream())
            fcp.fcp_cache_attn(w.cache, w.b, w.q, o, lse, w.ws, w.n, stream=s.cuda_stream)
            got.append((o, lse))
    torch.cuda.synchronize()
    for i, (o, lse) in enumerate(got):
        assert torch.equal(o, want[i % 2][0]) and torch.equal(lse, want[i % 2][1])


def test_a_cache_in_host_memory_is_refused():
    z = lambda *s, t: torch.zeros(s, dtype=t)
    cache = fcp.Cache(z(2, 1, 16, 64, t=torch.int8), z(2, 1, 16, 64, t=torch.int8), z(2, 1, t=torch.float32), z(2, 1, t=torch.float32), z(4, t=torch.int32))
    x = torch.zeros(1, 1, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(fcp.FcpError) as e:
        fcp.fcp_cache_append(cache, fcp.CacheBatch(dev([[0]]), dev([1]), dev([0, 1]), rows=1), x, x, stream=stream())
    assert e.value.status == fcp.FCP_ERR_INVALID_ARG


@pytest.mark.parametrize("kind,d", [("e4m3", 128), ("int8", 64)])
def test_prompt_then_tokens_then_eviction(kind, d):
    """As a model would use them: the prompt through rotary, the packed attention of this library and the cache; tokens one by one;
    eviction; tokens again on the new pages."""
    hq, hkv, page, prompts, steps = 4, 2, 16, [200, 33], 6
    w = World(61, kind, page, hkv, d, [p + steps for p in prompts], spare=20)
    w.weight[:] = 0
    w.up()
    table = fcp.RopeTable(d, d, base=10000.0, scaling="wavelength", factor=4.0, original_length=128.0)
    freqs = R.rope_frequencies(d, 10000.0, "wavelength", 4.0, 128.0)
    rows = sum(prompts)
    q, k, v = (bf16(w.rng, rows, h, d).cuda() for h in (hq, hkv, hkv))
    off = dev(np.concatenate([[0], np.cumsum(prompts)]))
    fcp.fcp_rope_fwd(table, q, k, q, k, row_offset=off, stream=stream())
    plan = fcp.Plan(prompts, [1, 1], hq, hkv, d).upload()
    o, lse = torch.empty_like(q), torch.empty(rows, hq, device="cuda")
    fcp.fcp_attn_fwd_fused(plan, q, k, v, o, lse, stream=stream())
    pages, length = dev(w.table), dev(prompts)
    batch = fcp.CacheBatch(pages, length, off, rows=rows, max_new=max(prompts))
    fcp.fcp_cache_append(w.cache, batch, k, v, stream=stream())
    o8, lse8 = torch.empty_like(q), torch.empty(rows, hq, device="cuda")
    n = fcp.fcp_cache_attn_workspace_bytes(w.cache, batch, hq)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    fcp.fcp_cache_attn(w.cache, batch, q, o8, lse8, ws, n, accumulate=True, stream=stream())
    # the cache's keys are off by half a step of e4m3 (2^-4) or of int8 under a power-of-two scale (2^-7 of the page's largest)
    step = 2.0 ** -4 if kind == "e4m3" else 2.0 ** -7 * 6
    assert (o8.float() - o.float()).norm() <= 2 * step * o.float().norm() and (lse8 - lse).abs().max() < 12 * step

    def tokens(pages, lengths, times):
        lengths = list(lengths)
        for _ in range(times):
            positions = dev([p + done[0] for p in prompts])
            done[0] += 1
            lengths = [x + 1 for x in lengths]
            step_batch = fcp.CacheBatch(pages, dev(lengths), dev([0, 1, 2]), rows=2, max_new=1)
            q1, k1, v1 = (bf16(w.rng, 2, h, d).cuda() for h in (hq, hkv, hkv))
            raw = k1.clone()
            fcp.fcp_rope_fwd(table, q1, k1, q1, k1, positions=positions, stream=stream())
            check_rope(k1, raw, positions.cpu().numpy(), freqs, d, "half", 1.0)
            fcp.fcp_cache_append(w.cache, step_batch, k1, v1, stream=stream())
            o1, lse1 = torch.empty(2, hq, d, dtype=torch.bfloat16, device="cuda"), torch.empty(2, hq, device="cuda")
            state = w.now()
            m = fcp.fcp_cache_attn_workspace_bytes(w.cache, step_batch, hq)
            fcp.fcp_cache_attn(w.cache, step_batch, q1, o1, lse1, torch.empty(m, dtype=torch.uint8, device="cuda"), m, accumulate=True, stream=stream())
            w.off = np.asarray([0, 1, 2])
            r = R.attention(state, pages.cpu().numpy(), lengths, w.off, f64(q1))
            check_attn(w, None, r, o1, lse1, 2)
            assert math.isclose(float(w.w.double().sum() - state["weight"].sum()), 2 * hq, rel_tol=1e-5)
        return lengths
    done = [0]
    lengths = tokens(pages, prompts, 3)
    state = w.now()
    dst = np.full((2, 6), -1)
    dst[0], dst[1] = w.free[:6], w.free[6:12]
    new_length, kept = torch.empty(2, dtype=torch.int32, device="cuda"), torch.empty(2, hkv, 80, dtype=torch.int32, device="cuda")
    fcp.fcp_cache_evict(w.cache, fcp.CacheBatch(pages, dev(lengths)), 4, 60, 16, dev(dst), new_length, kept, stream=stream())
    want_kept, want_length = R.evict(kind, state, w.table, lengths, 4, 60, 16, dst)
    assert np.array_equal(kept.cpu().numpy(), want_kept) and new_length.tolist() == want_length.tolist() == [80, 36]
    same(w.now(), state)
    tokens(dev(dst), new_length.tolist(), 3)
    assert w.cache.device_status().tolist() == [0, 0, 0, 0]


# ---------------------------------------------------------------------------------------------------------
# Values and scales at the ends of their range
# ---------------------------------------------------------------------------------------------------------
def unit_code(kind):
    """The code of 1."""
    return 0x38 if kind == "e4m3" else 1


def shared_batch(w, B):
    """B sequences of one new token each, all on the pages of the first one."""
    table = np.repeat(w.table[:1], B, axis=0)
    return fcp.CacheBatch(dev(table), dev([int(w.length[0])] * B), dev(np.arange(B + 1)), rows=B, max_new=1)


def attend_batch(w, batch, q, hq, scale=0.0, accumulate=False):
    o, lse = torch.full((batch.rows, hq, w.d), 3.0, dtype=torch.bfloat16, device="cuda"), torch.full((batch.rows, hq), 5.0, device="cuda")
    n = fcp.fcp_cache_attn_workspace_bytes(w.cache, batch, hq)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    fcp.fcp_cache_attn(w.cache, batch, q.cuda(), o, lse, ws, n, scale=scale, accumulate=accumulate, stream=stream())
    torch.cuda.synchronize()
    return o, lse


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("hq", [1, 10, 25, 40])
@pytest.mark.parametrize("B", [1, 74, 148])
def test_zero_values_and_scores_that_rise(kind, hq, B):
    """A KV head whose values are all zero has pages of the smallest scale, 2^-100.  The first keys of every block's share have score 0,
    the others 4.6875: the sum of the weights over the value scales has to stay finite.  Alone, two blocks a sequence, one block a sequence."""
    T = 320 * 128
    w = World(81, kind, 128, 1, 64, [T], spare=0)
    low = np.zeros(T, bool)
    low[:256] = low[159 * 128:161 * 128] = True
    k = np.zeros((T, 64), np.uint8)
    k[~low, 0] = unit_code(kind)
    for i, p in enumerate(w.table[0]):
        w.codes["k"][p, 0], w.codes["v"][p, 0] = k[i * 128:(i + 1) * 128], 0
    w.scale["k"][:], w.scale["v"][:], w.weight[:] = 1.0, 2.0 ** -100, 0.0
    w.up()
    q = torch.zeros(B, hq, 64, dtype=torch.bfloat16)
    q[..., 0] = 37.5                                              # times 1/8
    o, lse = attend_batch(w, shared_batch(w, B), q, hq, accumulate=True)
    s = np.where(low, 0.0, 4.6875)
    want = 4.6875 + math.log(np.exp(s - 4.6875).sum())
    # a thread adds at most T / 32 weights, one rounding each; the join of threads, warps and blocks a few hundred roundings more;
    # scores are exact but for their place in log2 units (2^-23 of at most 16)
    tol = (T / 32 + 300) * F32 + 16 * 2.0 ** -22
    assert np.abs(f64(lse) - want).max() <= tol
    assert bool((o == 0).all())
    weight = f64(w.w)[w.table[0], 0].reshape(-1)
    assert np.all(np.abs(weight / (B * hq * np.exp(s - want)) - 1) <= 2 * tol + (B + 64) * F32)


@pytest.mark.parametrize("kind,page,d", [("e4m3", 16, 64), ("int8", 16, 128), ("int8", 128, 64), ("e4m3", 128, 128)])
@pytest.mark.parametrize("new,hq", [(1, 3), (3, 4), (5, 5), (1, 40)])
@pytest.mark.parametrize("top", [-100, -77, -3])
def test_value_scales_down_to_the_smallest(kind, page, d, new, hq, top):
    """Pages whose value scales, powers of two and others, lie between 2^-100 and 2^top."""
    w = World(82, kind, page, 1, d, [2000, 5000]).fill()
    exponent = np.minimum(-100 + w.rng.integers(0, 28, w.n_pages), top)
    exponent[::9] = top
    w.scale["v"][:, 0] = 2.0 ** exponent * np.where((exponent > -100) & (w.rng.random(w.n_pages) < 0.5), w.rng.uniform(0.75, 1.0, w.n_pages), 1.0)
    w.up()
    q, o, lse, rows = attend(w, [new, new], hq, spare=0)
    state = w.state()
    r = R.attention(state, w.table, w.length, w.off, f64(q))
    # as in test_tiles_of_rows_that_see_nothing_or_differ_in_size, with scales below 2^-80 counted as up to 2^-79: every code is off by
    # at most 2^-33 of the row's largest product of a weight and such a scale
    lost = np.zeros((rows, hq, d))
    for b in range(2):
        t = w.length[b]
        pages = np.asarray(w.table[b][:-(-t // page)])
        k, code = R.gather(state, "k", pages, t, 0), state["v"][pages, 0].reshape(-1, d)[:t]
        scale = np.maximum(np.repeat(state["v_scale"][pages, 0], page)[:t], 2.0 ** -79)
        for j in range(new):
            row, seen = w.off[b] + j, t - new + j + 1
            for h in range(hq):
                s = k[:seen] @ f64(q)[row, h] / math.sqrt(d)
                lost[row, h] = 2.0 ** -33 * (np.exp(s - r["lse"][row, h]) * scale[:seen]).max() * np.abs(code[:seen]).sum(axis=0)
    score = d * 2 * F32 * r["size"] + 2.0 ** -20
    assert np.all(np.abs(f64(lse) - r["lse"]) <= score + 4 * F32 * np.abs(r["lse"]))
    bound = BF16 * np.abs(r["o"]) + (HALF + 2 * score[..., None]) * r["spread"] * (1 + BF16) + lost
    assert np.all(np.abs(f64(o) - r["o"]) <= bound), np.max(np.abs(f64(o) - r["o"]) / bound)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("hq", [1, 10, 25, 40])
def test_a_huge_value_that_weighs_little(kind, hq):
    """One block's share of a sequence holds keys of small score, the largest of them with a value as an infinity is stored: that block's
    result is beyond fp32, the whole one is not."""
    T, at = 320 * 128, 200 * 128 + 40
    w = World(83, kind, 128, 1, 64, [T], spare=0)
    unit, s = unit_code(kind), np.zeros(T)
    s[at - 1000:at + 1000], s[at] = -40.0, -30.0
    k, v = np.zeros((T, 64), np.uint8), np.zeros((T, 64), np.uint8)
    k[s == -40, 0] = k[at, 1] = unit
    v[:] = unit
    v[at] = 0x7e if kind == "e4m3" else 127
    top = R.TOP[kind] * 2.0 ** (120 if kind == "e4m3" else 122)
    for i, p in enumerate(w.table[0]):
        w.codes["k"][p, 0], w.codes["v"][p, 0] = k[i * 128:(i + 1) * 128], v[i * 128:(i + 1) * 128]
    w.scale["k"][:], w.scale["v"][:] = 1.0, 1.0
    page = w.table[0][at // 128]
    w.scale["v"][page] = top / R.TOP[kind]
    keep = w.codes["v"][page, 0, at % 128].copy()
    w.codes["v"][page, 0], w.codes["v"][page, 0, at % 128] = 0, keep
    w.up()
    q = torch.zeros(1, hq, 64, dtype=torch.bfloat16)
    q[..., 0], q[..., 1] = -320.0, -240.0                         # times 1/8
    o, lse = attend_batch(w, shared_batch(w, 1), q, hq)
    z = np.exp(s).sum()
    value = np.exp(-30.0) * top / z                               # what the other values add is below 2^-60 of it
    assert np.abs(f64(lse) - math.log(z)).max() <= (T / 32 + 300) * F32 + 2.0 ** -20
    assert np.all(np.abs(f64(o) - value) <= (BF16 + HALF + 2.0 ** -12) * value)


@pytest.mark.parametrize("kind,page,d", [("e4m3", 16, 64), ("int8", 16, 128), ("int8", 128, 64), ("e4m3", 128, 128)])
@pytest.mark.parametrize("new,hq", [(1, 3), (3, 4), (5, 5), (1, 40)])
@pytest.mark.parametrize("exponents", [[-9], [-100, -9], [-9, 120], [-100, -60, -35, -9, 20, 60, 120]])
def test_value_scales_far_apart(kind, page, d, new, hq, exponents):
    """Probabilities count in full however small their value scale is beside the others': pages of zeros, ordinary ones, and those of
    values that were infinite."""
    w = World(85, kind, page, 1, d, [3, 700, 9000]).fill()
    w.scale["v"][:, 0] = 2.0 ** np.asarray(exponents)[w.rng.integers(0, len(exponents), w.n_pages)]
    w.up()
    q, o, lse, rows = attend(w, [min(new, 3), new, new], hq, spare=0)
    state = w.state()
    r = R.attention(state, w.table, w.length, w.off, f64(q))
    lost = np.zeros((rows, hq, d))                                # as in test_tiles_of_rows_that_see_nothing_or_differ_in_size
    for b, n in enumerate(np.diff(w.off)):
        t = w.length[b]
        pages = np.asarray(w.table[b][:-(-t // page)])
        k, code = R.gather(state, "k", pages, t, 0), state["v"][pages, 0].reshape(-1, d)[:t]
        scale = np.repeat(state["v_scale"][pages, 0], page)[:t]
        for j in range(n):
            row, seen = w.off[b] + j, t - n + j + 1
            for h in range(hq):
                s = k[:seen] @ f64(q)[row, h] / math.sqrt(d)
                lost[row, h] = 2.0 ** -33 * (np.exp(s - r["lse"][row, h]) * scale[:seen]).max() * np.abs(code[:seen]).sum(axis=0)
    # a score stands in log2 units beside the log2 of its value scale: an fp32 below 2^8, half a step 2^-17, and so does the reference
    score = d * 2 * F32 * r["size"] + (2.0 ** -20 if exponents == [-9] else 2.0 ** -16)
    assert np.all(np.abs(f64(lse) - r["lse"]) <= score + 4 * F32 * np.abs(r["lse"]))
    bound = BF16 * np.abs(r["o"]) + (HALF + 2 * score[..., None]) * r["spread"] * (1 + BF16) + lost
    fits = np.abs(r["o"]) + bound < 3.38e38                       # beyond what a bf16 holds an infinity stands for the number
    assert np.all((np.abs(f64(o) - r["o"]) <= bound)[fits]) and not np.isnan(f64(o)).any()


@pytest.mark.parametrize("kind,page,d", [("e4m3", 16, 64), ("int8", 128, 128)])
@pytest.mark.parametrize("new,hq", [(1, 3), (3, 4), (5, 5), (1, 40)])
@pytest.mark.parametrize("exponent", [24, 60, 110])
def test_scores_far_beyond_the_exponentials(kind, page, d, new, hq, exponent):
    """Scores of 2^24 to 2^116: the key with the largest takes all, and nothing overflows."""
    w = World(86, kind, page, 1, d, [3, 700, 9000]).fill()
    w.scale["k"] *= np.float32(2.0 ** exponent)
    w.up()
    q, o, lse, rows = attend(w, [min(new, 3), new, new], hq, spare=0)
    state = w.state()
    r = R.attention(state, w.table, w.length, w.off, f64(q))
    score = d * 2 * F32 * r["size"]
    assert np.all(np.abs(f64(lse) - r["lse"]) <= score + 4 * F32 * np.abs(r["lse"]) + 1)
    # one key: its weight and the sum are the same number but for two roundings of an exponential
    clear, got = 0, f64(o)
    for b, n in enumerate(np.diff(w.off)):
        t = w.length[b]
        pages = np.asarray(w.table[b][:-(-t // page)])
        k, v = R.gather(state, "k", pages, t, 0), R.gather(state, "v", pages, t, 0)
        for j in range(n):
            row, seen = w.off[b] + j, t - n + j + 1
            for h in range(hq):
                s = k[:seen] @ f64(q)[row, h] / math.sqrt(d)
                at, gap = s.argmax(), np.diff(np.sort(s)[-2:]) if seen > 1 else np.inf
                if gap > 2 * score[row, h] + 100:
                    clear += 1
                    assert np.all(np.abs(got[row, h] - v[at]) <= (BF16 + HALF + 2.0 ** -18) * np.abs(v[at]) + 1e-30)
    assert clear > 0.9 * rows * hq and not np.isnan(got).any()


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128])
def test_chunks_with_values_beyond_bf16(kind, d):
    """Keys and values that were infinite or next to the largest bf16 stand in the cache as numbers beyond bf16; in calls that go by
    copies they reach the rows that see them, and no others."""
    new, before, hkv, group = [200, 150, 300, 133], [100, 0, 37, 300], 4, 8
    w = World(84, kind, 16, hkv, d, [a + n for a, n in zip(before, new)]).fill().up()
    hq, rows = hkv * group, sum(new)
    assert goes_by_copies(w, new, hq)
    batch = w.batch(new)
    k, v, q = bf16(w.rng, rows, hkv, d), bf16(w.rng, rows, hkv, d), bf16(w.rng, rows, hq, d)
    at = {0: 150, 1: 120, 2: 290}                                 # of each sequence's new tokens
    v[w.off[0] + at[0], 1, 5], v[w.off[0] + at[0], 2, 6] = math.inf, -math.inf
    v[w.off[1] + at[1], :, 3] = 3.3e38
    k[w.off[2] + at[2], 0, 2] = math.inf
    k[w.off[2] + at[2], 3, 0] = 1e30
    fcp.fcp_cache_append(w.cache, batch, k.cuda(), v.cuda(), stream=stream())
    o, lse = attend_batch(w, batch, q, hq)
    r = R.attention(w.now(), w.table, w.length, w.off, f64(q))
    got, got_lse = f64(o), f64(lse)
    score = d * 2 * F32 * r["size"] + 2.0 ** -20
    # scores are fp32 in units of log 2: 448 * 2^120 times a query above 3 is 6.0e38 * 3 / 8 * 1.44 = 3.3e38 or more, and fp32 ends at
    # 3.4e38; what such a row gets is not defined
    held = r["size"] * math.log2(math.e) < 3.4e38
    assert held.mean() > 0.99
    assert not np.isnan(got[held]).any() and not np.isnan(got_lse[held]).any()
    assert np.all((np.abs(got_lse - r["lse"]) <= score + 4 * F32 * np.abs(r["lse"]))[held])
    bound = BF16 * np.abs(r["o"]) + (BF16 + 2 * score[..., None]) * r["spread"] * (1 + BF16) + 1e-30
    # a number beyond bf16, 448 * 2^120 or 127 * 2^122 at most, counts as the largest bf16, 2^128: 1 / 1.99 of it or more; a sum may be infinite
    great = r["spread"] > 1e30
    assert np.all((np.abs(got - r["o"]) <= bound)[held[..., None] & ~great])
    assert np.all((np.sign(got) == np.sign(r["o"]))[great]) and np.all((np.abs(got) >= 0.49 * np.abs(r["o"]) - bound)[great])
    for b, j in at.items():                                       # the rows in front of it know nothing of it
        assert not great[w.off[b]:w.off[b] + j].any() and held[w.off[b]:w.off[b] + j].all()
    assert great[w.off[0] + at[0]:w.off[1]].any() and great[w.off[1] + at[1]:w.off[2]].any()


@pytest.mark.parametrize("page,rows,off", [(64, 240, [17, 187, 31, 80, 161, 236, 239]), (16, 160, [29, 30, 59, 124, 82, 141]), (128, 341, [46, 54, 282, 68, 149, 161, 173, 289]),
                                           (16, 55, [8, 24, 28, 32, 41, 3, 45, 48]), (32, 190, [19, 61, 72, 5, 93, 119, 186]), (16, 40, [0, 20, 41])])
def test_append_reports_offsets_that_fall(page, rows, off):
    """Whichever sequences the search for a page's sequence finds: the bad one is reported, and only pages of the batch are written."""
    B = len(off) - 1
    w = World(87, "int8", page, 2, 64, [400] * B).up()
    was = w.now()
    k = bf16(w.rng, rows, 2, 64).cuda()
    fcp.fcp_cache_append(w.cache, fcp.CacheBatch(dev(w.table), dev(w.length), dev(off), rows=rows), k, k, stream=stream())
    bad = [b for b in range(B) if off[b + 1] < off[b] or off[b + 1] > rows]
    st = w.cache.device_status().tolist()
    assert st[:2] == [fcp.FCP_ERR_INVALID_ARG, fcp.FCP_CACHE_BAD_ROWS] and st[2] in bad
    now = w.now()
    good = [b for b in range(B) if b not in bad]
    touched = {int(w.table[b][p // page]) for b in good for p in range(400 - (off[b + 1] - off[b]), 400)}
    for p in range(w.n_pages):
        if p not in touched:
            assert np.array_equal(now["k"][p], was["k"][p], equal_nan=True) and np.array_equal(now["v_scale"][p], was["v_scale"][p])


def check_weights(w, was, new, hq, r):
    """Every weight against the definition: a score's fp32 error three times (score, and the log-sum-exp's own), and the sum over rows."""
    want, tol = was.copy(), F32 * 4 * np.abs(was) + 1e-30
    score = w.d * 2 * F32 * r["size"].max() + 2.0 ** -20
    for b, t in enumerate(w.length):
        rows = new[b] * hq // w.hkv
        for p in range(t):
            page_id, slot = w.table[b][p // w.page], p % w.page
            want[page_id, :, slot] += r["weights"][b][:, p]
            tol[page_id, :, slot] += r["weights"][b][:, p] * (3 * score + (64 + rows / 4) * F32)
    now = w.now()["weight"]
    assert np.all(np.abs(now - want) <= tol), np.max(np.abs(now - want) / tol)


@pytest.mark.parametrize("kind,page,d", [("e4m3", 16, 64), ("int8", 16, 128), ("int8", 64, 64), ("e4m3", 128, 128)])
@pytest.mark.parametrize("hkv,group,new,before", [(8, 8, [300], [0]), (8, 8, [257, 0, 1], [70, 300, 5]), (8, 6, [300, 40, 257], [129, 0, 300])])
def test_weights_that_long_chunks_leave(kind, page, d, hkv, group, new, before):
    w = World(88, kind, page, hkv, d, [a + n for a, n in zip(before, new)]).fill().up()
    assert goes_by_copies(w, new, hkv * group)
    state, was = w.state(), w.now()["weight"]
    q, o, lse, rows = attend(w, new, hkv * group, accumulate=True)
    r = R.attention(state, w.table, w.length, w.off, f64(q)[:rows])
    check_weights(w, was, new, hkv * group, r)


@pytest.mark.parametrize("kind,page,hkv,d", [("e4m3", 16, 2, 64), ("int8", 128, 2, 128)])
@pytest.mark.parametrize("group,new,before", [(1, [33, 0, 128], [0, 40, 500]), (4, [9, 1, 31, 0], [1500, 3, 130, 64]), (2, [200], [500]), (8, [16, 16, 1], [127, 5, 2000])])
def test_weights_that_many_rows_leave(kind, page, hkv, d, group, new, before):
    w = World(89, kind, page, hkv, d, [a + n for a, n in zip(before, new)]).fill().up()
    assert not goes_by_copies(w, new, hkv * group)
    state, was = w.state(), w.now()["weight"]
    q, o, lse, rows = attend(w, new, hkv * group, accumulate=True)
    r = R.attention(state, w.table, w.length, w.off, f64(q)[:rows])
    check_weights(w, was, new, hkv * group, r)


def test_weights_of_a_chunk_with_sequences_that_need_care():
    """Tokens on a page that does not exist get none; a sequence with more rows than tokens leaves those of its tokens."""
    new, hkv, group = [140, 150, 133], 4, 8
    w = World(90, "int8", 16, hkv, 64, [300, 90, 200]).fill()
    good, table = w.state(), w.table.copy()
    w.table[2, 1] = w.n_pages + 5
    w.up()
    assert goes_by_copies(w, new, hkv * group)
    was = w.now()["weight"]
    q, o, lse, rows = attend(w, new, hkv * group, accumulate=True, spare=0)
    r = R.attention(good, table, w.length, w.off, f64(q))
    added = w.now()["weight"] - was
    sums = added[table[0][:19]].sum(axis=(0, 2)), added[table[1][:6]].sum(axis=(0, 2)), added[table[2][:13]].sum(axis=(0, 2))
    for got, n in zip(sums, (140, 90, 133)):
        assert np.allclose(got, n * group, rtol=1e-4)
    assert np.all(added[table[2][1]] == 0)
    score = 64 * 2 * F32 * r["size"].max() + 2.0 ** -20
    for b in (0, 1):
        for p in range(w.length[b]):
            want = r["weights"][b][:, p]
            got = added[table[b][p // 16], :, p % 16]
            assert np.all(np.abs(got - want) <= want * (3 * score + 400 * F32) + 8 * F32)


@pytest.mark.parametrize("d", [64, 128])
def test_chunks_with_nan_keys_among_the_new_tokens(d):
    """By copies: a NaN key of a new token reaches the rows that see it and no others, and no other sequence; stale NaN codes behind the length none."""
    new, hkv, group = [200, 150, 133], 4, 8
    w = World(91, "e4m3", 16, hkv, d, [300, 150, 200]).fill()
    w.codes["k"][w.table[0][230 // 16], 1, 230 % 16, 3] = 0x7f
    w.codes["k"][w.table[1][149 // 16], 2, 149 % 16, 0] = 0xff
    w.up()
    assert goes_by_copies(w, new, hkv * group)
    q, o, lse, rows = attend(w, new, hkv * group, spare=0)
    with np.errstate(invalid="ignore"):
        r = R.attention(w.state(), w.table, w.length, w.off, f64(q))
    got, got_lse = f64(o), f64(lse)
    bad = np.isnan(r["lse"])
    assert bad[130:200, 8:16].all() and bad[349, 16:24].all() and bad.sum() == 70 * 8 + 8
    assert np.array_equal(np.isnan(got_lse), bad) and np.isnan(got[bad]).all()
    score = d * 2 * F32 * np.nan_to_num(r["size"]) + 2.0 ** -20
    bound = BF16 * np.abs(r["o"]) + (BF16 + 2 * score[..., None]) * r["spread"] * (1 + BF16) + 1e-30
    assert np.all((np.abs(got - r["o"]) <= bound)[~bad])
