"""The operators around attention: rotary positions, and a cache of keys and values in 8 bits with the attention that
reads it and the eviction that keeps it small.

  rope     fcp_rope_fwd / fcp_rope_bwd     rotates queries and keys by their positions
  append   fcp_cache_append                new keys and values into pages of one byte per value, a scale per page and head
  attn     fcp_cache_attn                  the newest tokens of each sequence over all its cached ones; with `weights` each
                                           cached token's share is added to its page
  evict    fcp_cache_evict                 first, newest and heaviest tokens of each head into new pages

A case is plain values.  Lengths follow from the case alone, tensors from the seed.  `own` chooses between the plain
forms below (elementary operations, 32 bits) and the framework's calls.
"""
import math

import numpy as np
import torch

own = False

E4M3_MAX, INT8_MAX = 448.0, 127.0
SMALLEST_SCALE = 2.0 ** -100


def listed():
    return [
        # one new token in each of 64 running sequences, far positions, frequencies blended by wavelength
        dict(name="rope_decode_64", op="rope", mix="ones", seqs=64, tokens=64, hq=32, hkv=8, head_dim=128, rotary_dim=128,
             layout="half", scaling="wavelength", base=500000.0, factor=8.0, original=8192.0, cached=131072, fused=False,
             backward=False, lengths=1),
        # the ordinary training batch: 64K packed tokens of a 32/8-head layer, positions restart with every sequence
        dict(name="rope_train_64k", op="rope", mix="lognormal", seqs=0, tokens=65536, hq=32, hkv=8, head_dim=128,
             rotary_dim=128, layout="half", scaling="none", base=500000.0, factor=1.0, original=8192.0, cached=0, fused=False,
             backward=False, lengths=7),
        # backward of a small model's layer: half of the head rotates, interleaved, odd lengths that go on behind 100K
        # cached tokens, gradients are slices of one buffer of the fused projection
        dict(name="rope_backward_16k_d64", op="rope", mix="lognormal", seqs=0, tokens=16411, hq=12, hkv=4, head_dim=64,
             rotary_dim=32, layout="interleaved", scaling="yarn", base=10000.0, factor=32.0, original=4096.0, cached=100003,
             fused=True, backward=True, lengths=4),
        # one new token in each of 128 running sequences
        dict(name="append_decode_128", op="append", mix="ones", seqs=128, tokens=128, hkv=8, head_dim=128, page=16,
             kind="e4m3", cached=8192, fused=False, lengths=2),
        # the prompts of a 64K-token batch, some behind tokens that are cached already
        dict(name="append_prompt_64k", op="append", mix="lognormal", seqs=0, tokens=65536, hkv=8, head_dim=128, page=64,
             kind="int8", cached=2000, fused=True, lengths=7),
        # the smallest call: one token of one short sequence of a small model
        dict(name="attn_one_short", op="attn", seqs=1, new=1, lo=700, hi=700, hq=4, hkv=4, head_dim=64, page=16, kind="e4m3",
             weights=False, lengths=1),
        # 64 running sequences of all lengths up to 8K, one token each
        dict(name="attn_decode_64x8k", op="attn", seqs=64, new=1, lo=300, hi=8192, hq=32, hkv=8, head_dim=128, page=16,
             kind="e4m3", weights=False, lengths=3),
        # one token behind a 384K-token document
        dict(name="attn_decode_384k", op="attn", seqs=1, new=1, lo=393216, hi=393216, hq=64, hkv=8, head_dim=128, page=64,
             kind="e4m3", weights=False, lengths=1),
        # five drafted tokens to verify in each of 16 long sequences, weights kept for the eviction
        dict(name="attn_verify_16x32k", op="attn", seqs=16, new=5, lo=4097, hi=32768, hq=40, hkv=8, head_dim=128, page=32,
             kind="int8", weights=True, lengths=5),
        # a chunk of 512 prompt tokens behind 6K to 12K cached ones
        dict(name="attn_chunk_4x512", op="attn", seqs=4, new=512, lo=6001, hi=12288, hq=32, hkv=8, head_dim=128, page=128,
             kind="int8", weights=False, lengths=6),
        # eight sequences of up to 8K tokens cut to 2K, no grouped heads
        dict(name="evict_8x8k", op="evict", seqs=8, lo=1025, hi=8192, hkv=32, head_dim=128, page=16, kind="int8", sink=4,
             heavy=1500, recent=544, lengths=8),
        # two 128K documents cut to 16K
        dict(name="evict_2x128k", op="evict", seqs=2, lo=120000, hi=131072, hkv=8, head_dim=128, page=64, kind="e4m3", sink=16,
             heavy=12273, recent=4095, lengths=9),
    ]


def draw(rng):
    """One more case of the ranges above."""
    def log_int(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    hq, hkv, head_dim = rng.choice([(4, 4, 64), (12, 4, 64), (16, 2, 64), (8, 8, 128), (32, 8, 128), (28, 4, 128),
                                    (40, 8, 128), (64, 8, 128), (32, 32, 128)])
    lengths = rng.randrange(1, 1 << 30)
    page, kind = rng.choice([16, 32, 64, 128]), rng.choice(["e4m3", "int8"])
    op = rng.choice(["rope", "append", "attn", "attn", "evict"])
    if op == "rope":
        decode = rng.random() < 0.3
        tokens = log_int(1, 512) if decode else log_int(512, 65536)
        rotary = rng.choice([head_dim, head_dim, head_dim // 2, 2 * rng.randint(1, head_dim // 2)])
        return dict(op=op, mix="ones" if decode else "lognormal", seqs=tokens if decode else 0, tokens=tokens, hq=hq, hkv=hkv,
                    head_dim=head_dim, rotary_dim=max(4, rotary), layout=rng.choice(["half", "interleaved"]),
                    scaling=rng.choice(["none", "linear", "ntk", "yarn", "wavelength"]), base=rng.choice([10000.0, 500000.0]),
                    factor=rng.choice([2.0, 8.0, 32.0]), original=rng.choice([4096.0, 8192.0]),
                    cached=log_int(1, 1000000) if rng.random() < 0.5 else 0, fused=rng.random() < 0.5,
                    backward=rng.random() < 0.5, lengths=lengths)
    if op == "append":
        decode = rng.random() < 0.5
        tokens = log_int(1, 512) if decode else log_int(256, 65536)
        return dict(op=op, mix="ones" if decode else "lognormal", seqs=tokens if decode else 0, tokens=tokens, hkv=hkv,
                    head_dim=head_dim, page=page, kind=kind, cached=log_int(1, 4096), fused=rng.random() < 0.5, lengths=lengths)
    if op == "attn":
        seqs, new = rng.choice([(log_int(1, 96), 1), (log_int(1, 32), rng.randint(2, 16)), (log_int(1, 4), log_int(17, 600))])
        most = int(min(131072, 450000 / seqs, 1.5e9 / (hq * new * seqs), 1e8 / (new * seqs)))
        hi = max(new + 1, log_int(64, max(65, most)))
        return dict(op=op, seqs=seqs, new=new, lo=max(1, hi // rng.choice([1, 3, 20])), hi=hi, hq=hq, hkv=hkv, head_dim=head_dim,
                    page=page, kind=kind, weights=rng.random() < 0.4, lengths=lengths)
    seqs = log_int(1, 16)
    hi = log_int(200, min(131072, 250000 // seqs))
    keep = max(3, int(hi * rng.uniform(0.05, 0.6)))
    recent = int(keep * rng.uniform(0, 0.5))
    sink = min(keep - recent, rng.choice([0, 1, 4, 16]))
    return dict(op=op, seqs=seqs, lo=max(1, hi // rng.choice([1, 2, 10])), hi=hi, hkv=min(hkv, 8) if hi > 16384 else hkv,
                head_dim=head_dim, page=page, kind=kind, sink=sink, heavy=keep - recent - sink, recent=recent, lengths=lengths)


# ---------------------------------------------------------------------------------------------------------
# Layout of a case: new tokens and total lengths of its sequences (host arrays, from the case alone)
# ---------------------------------------------------------------------------------------------------------
def lengths_of(case):
    rng = np.random.Generator(np.random.PCG64([case["lengths"], 0xCAC4E]))
    if case["op"] in ("attn", "evict"):
        n = case["seqs"]
        total = np.rint(np.exp(rng.uniform(math.log(case["lo"]), math.log(case["hi"]), n))).astype(np.int64)
        total[rng.integers(n)] = case["hi"]
        new = np.full(n, case.get("new", 0), np.int64)
        return np.minimum(new, total), total
    if case["mix"] == "ones":
        new = np.ones(case["seqs"], np.int64)
    else:
        parts, left = [], case["tokens"]
        while left > 0:
            parts.append(min(left, int(np.clip(round(float(rng.lognormal(math.log(1500.0), 1.0))), 1, 32768))))
            left -= parts[-1]
        new = np.asarray(parts, np.int64)
    before = rng.integers(0, case["cached"] + 1, len(new)) if case["cached"] else np.zeros(len(new), np.int64)
    return new, new + before


def frequencies(case):
    """Radians per token of each pair, and the magnitude of the rotation."""
    r, base, s, original = case["rotary_dim"], case["base"], case["factor"], case["original"]
    i = np.arange(r // 2, dtype=np.float64)
    scaling = case["scaling"]
    if scaling == "ntk" and r > 2:
        base = base * s ** (r / (r - 2.0))
    f = base ** (-2.0 * i / r)
    if scaling == "linear":
        return f / s, 1.0
    if scaling == "yarn":          # dimensions that turn more than 32 times in the original length stay, below once are stretched
        def dim(turns):
            return r * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))
        low, high = max(math.floor(dim(32.0)), 0), min(math.ceil(dim(1.0)), r - 1)
        ramp = np.clip((i - low) / max(high - low, 1e-3), 0.0, 1.0)
        return f / s * ramp + f * (1 - ramp), 0.1 * math.log(s) + 1.0
    if scaling == "wavelength":    # wavelengths below a quarter of the original length stay, above it are stretched
        turns = original * f / (2 * math.pi)
        smooth = np.clip((turns - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        return f * smooth + f / s * (1 - smooth), 1.0
    return f, 1.0


# ---------------------------------------------------------------------------------------------------------
# What a program has in hand
# ---------------------------------------------------------------------------------------------------------
def _i32(a):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32, device="cuda")


def _rows(case, gen, tokens, heads, fused_with=0, scale=None):
    """bf16 rows [tokens][heads][head_dim]; `fused_with`: a slice of a buffer with that many more heads."""
    d = case["head_dim"]
    x = torch.randn((tokens, heads + fused_with, d), dtype=torch.float32, device="cuda", generator=gen)
    if scale is not None:
        x *= scale.repeat_interleave((heads + fused_with) // scale.numel() + 1)[: heads + fused_with, None]
    return x.to(torch.bfloat16)[:, fused_with:]


def _cache(case, gen, pages):
    """A filled cache: values about N(0, 1) times a magnitude of the head, quantised page by page."""
    shape = (pages, case["hkv"], case["page"], case["head_dim"])
    e4m3 = case["kind"] == "e4m3"
    top = E4M3_MAX if e4m3 else INT8_MAX
    out = []
    for _ in range(2):
        magnitude = torch.exp(torch.randn((1, case["hkv"], 1, 1), device="cuda", generator=gen))
        codes = torch.empty(shape, dtype=torch.float8_e4m3fn if e4m3 else torch.int8, device="cuda")
        scales = torch.empty(shape[:2], dtype=torch.float32, device="cuda")
        step = max(1, (1 << 27) // (shape[1] * shape[2] * shape[3]))
        for at in range(0, pages, step):
            n = min(step, pages - at)
            x = torch.randn((n, *shape[1:]), device="cuda", generator=gen) * magnitude
            s = torch.ldexp(torch.ones((), device="cuda"), torch.ceil(torch.log2(x.abs().amax((2, 3)) / top)).int())
            x /= s[:, :, None, None]
            codes[at:at + n] = x.clamp_(-top, top).to(codes.dtype) if e4m3 else x.round_().clamp_(-top, top).to(codes.dtype)
            scales[at:at + n] = s
        out += [codes, scales]
    return out


def prepare(case, seed):
    new, total = lengths_of(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    offset = np.concatenate([[0], np.cumsum(new)])
    rows, d = int(offset[-1]), case["head_dim"]
    st = dict(case=case, new=new, total=total, rows=rows, row_offset=_i32(offset), length=_i32(total), kept_for_calls={})
    if case["op"] == "rope":
        if case["fused"]:         # slices of the projection's output
            qkv = _rows(case, gen, rows, case["hq"] + 2 * case["hkv"])
            st["q"], st["k"] = qkv[:, :case["hq"]], qkv[:, case["hq"]:case["hq"] + case["hkv"]]
        else:
            st["q"], st["k"] = _rows(case, gen, rows, case["hq"]), _rows(case, gen, rows, case["hkv"])
        st["q_out"] = torch.empty((rows, case["hq"], d), dtype=torch.bfloat16, device="cuda")
        st["k_out"] = torch.empty((rows, case["hkv"], d), dtype=torch.bfloat16, device="cuda")
        return st
    page = case["page"]
    n_pages = -(-total // page)
    width, pool = int(n_pages.max()), int(n_pages.sum()) + 3
    keep = case.get("sink", 0) + case.get("heavy", 0) + case.get("recent", 0)
    moved = np.minimum(total, keep) if case["op"] == "evict" else np.zeros(len(total), np.int64)
    dst_pages = -(-moved // page)
    pool += int(dst_pages.sum())
    order = torch.randperm(pool, device="cuda", generator=gen).to(torch.int32)      # pages lie anywhere
    def table(counts, at, w):
        first = np.concatenate([[0], np.cumsum(counts)])[:-1]
        index = np.minimum(at + first[:, None] + np.arange(w)[None], pool - 1)
        return torch.where(torch.as_tensor(np.arange(w)[None] < counts[:, None], device="cuda"),
                           order[torch.as_tensor(index, device="cuda")], 0).contiguous()
    st["page_table"] = table(n_pages, 0, width)
    st["k_cache"], st["k_scale"], st["v_cache"], st["v_scale"] = _cache(case, gen, pool)
    st["status"] = torch.zeros(4, dtype=torch.int32, device="cuda")
    st["weight"] = None
    if case["op"] == "append":
        # a new token is now and then larger than what its page has seen
        magnitude = torch.exp(torch.randn((case["hkv"],), device="cuda", generator=gen))
        extra = case["hkv"] if case["fused"] else 0
        st["k"] = _rows(case, gen, rows, case["hkv"], extra, magnitude)
        st["v"] = _rows(case, gen, rows, case["hkv"], extra, magnitude)
    elif case["op"] == "attn":
        st["q"] = _rows(case, gen, rows, case["hq"])
        st["o"] = torch.empty((rows, case["hq"], d), dtype=torch.bfloat16, device="cuda")
        st["lse"] = torch.empty((rows, case["hq"]), dtype=torch.float32, device="cuda")
        if case["weights"]:
            st["weight"] = torch.rand((pool, case["hkv"], page), device="cuda", generator=gen)
    else:
        # weights as attention leaves them: few heavy tokens, many light ones, some equal
        x = torch.randn((pool, case["hkv"], page), device="cuda", generator=gen)
        st["weight"] = torch.where(x > 1.5, torch.exp(2 * x), torch.round(torch.exp(x) * 4096) / 4096)
        st["dst_table"] = table(dst_pages, int(n_pages.sum()), max(1, int(dst_pages.max())))
        st["new_length"] = torch.empty(len(total), dtype=torch.int32, device="cuda")
        st["kept"] = torch.empty((len(total), case["hkv"], keep), dtype=torch.int32, device="cuda")
    return st


# ---------------------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------------------
def run(st):
    if own:
        return _calls(st)
    return {"rope": _plain_rope, "append": _plain_append, "attn": _plain_attn, "evict": _plain_evict}[st["case"]["op"]](st)


def _calls(st):
    """The framework's calls; tables and handles are made once, as a program keeps them."""
    from paper_2602_21788_b200 import fcp
    case, kept = st["case"], st["kept_for_calls"]
    op = case["op"]
    stream = torch.cuda.current_stream().cuda_stream
    if op == "rope":
        if not kept:
            kept["table"] = fcp.RopeTable(case["head_dim"], case["rotary_dim"], layout=case["layout"], base=case["base"],
                                          scaling=case["scaling"], factor=case["factor"], original_length=case["original"])
        call = fcp.fcp_rope_bwd if case["backward"] else fcp.fcp_rope_fwd
        call(kept["table"], st["q"], st["k"], st["q_out"], st["k_out"], row_offset=st["row_offset"],
             length=st["length"] if case["cached"] else None, stream=stream)
        return [st["q_out"], st["k_out"]]
    if not kept:
        kept["cache"] = fcp.Cache(st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"], st["status"], weight=st["weight"])
        kept["batch"] = fcp.CacheBatch(st["page_table"], st["length"], st["row_offset"], rows=st["rows"],
                                       max_new=int(st["new"].max()))
        if op == "attn":
            n = fcp.fcp_cache_attn_workspace_bytes(kept["cache"], kept["batch"], case["hq"])
            kept["workspace"], kept["bytes"] = torch.empty(n, dtype=torch.uint8, device="cuda"), n
    cache, batch = kept["cache"], kept["batch"]
    if op == "append":
        fcp.fcp_cache_append(cache, batch, st["k"], st["v"], stream=stream)
        return [st["k_cache"], st["k_scale"], st["v_cache"], st["v_scale"]]
    if op == "attn":
        fcp.fcp_cache_attn(cache, batch, st["q"], st["o"], st["lse"], kept["workspace"], kept["bytes"],
                           accumulate=case["weights"], stream=stream)
        return [st["o"], st["lse"]] + ([st["weight"]] if case["weights"] else [])
    fcp.fcp_cache_evict(cache, batch, case["sink"], case["heavy"], case["recent"], st["dst_table"], st["new_length"], st["kept"],
                        stream=stream)
    return [st["kept"], st["new_length"], st["k_cache"], st["k_scale"], st["v_cache"], st["v_scale"], st["weight"]]


def _token_rows(st):
    """Sequence and position of every new token."""
    off = st["row_offset"].long()
    t = torch.arange(st["rows"], device="cuda")
    b = torch.searchsorted(off, t, right=True) - 1
    return b, t - off[b], st["length"].long()[b] - (off[b + 1] - off[b]) + t - off[b]


def _plain_rope(st):
    case = st["case"]
    _, j, position = _token_rows(st)
    position = position if case["cached"] else j
    f, magnitude = frequencies(case)
    angle = position.double()[:, None] * torch.as_tensor(f, device="cuda")[None]
    cos, sin = (torch.cos(angle) * magnitude).float()[:, None], (torch.sin(angle) * magnitude).float()[:, None]
    if case["backward"]:
        sin = -sin
    r = case["rotary_dim"]

    def turned(x):
        x = x.float()
        y = x.clone()
        if case["layout"] == "half":
            a, b = x[..., :r // 2], x[..., r // 2:r]
            y[..., :r // 2], y[..., r // 2:r] = a * cos - b * sin, b * cos + a * sin
        else:
            a, b = x[..., 0:r:2], x[..., 1:r:2]
            y[..., 0:r:2], y[..., 1:r:2] = a * cos - b * sin, b * cos + a * sin
        return y.to(torch.bfloat16)
    return [turned(st["q"]), turned(st["k"])]


def _to_codes(x, like):
    """Values over their scale -> codes, to the nearest, ties to even."""
    return x.to(like.dtype) if like.dtype == torch.float8_e4m3fn else x.round().to(like.dtype)


def _put(codes, index, values):
    """codes[index] = values, through the bytes (indexed stores know no 8-bit floats)."""
    codes.view(torch.uint8)[index] = values.view(torch.uint8)


def _plain_append(st):
    page = st["case"]["page"]
    b, _, position = _token_rows(st)
    owner = st["page_table"].long()[b, position // page]
    slot = position % page
    start = st["length"].long() - (st["row_offset"][1:] - st["row_offset"][:-1]).long()
    filled = start % page                                     # tokens that the first page touched holds already
    has = filled > 0
    first = st["page_table"].long()[torch.arange(len(start), device="cuda"), torch.clamp(start // page, max=st["page_table"].shape[1] - 1)]
    first, filled = first[has], filled[has]
    earlier = (torch.arange(page, device="cuda")[None] < filled[:, None])[:, None, :, None]
    for name in ("k", "v"):
        x, codes, scale = st[name].float(), st[name + "_cache"], st[name + "_scale"]
        top = E4M3_MAX if codes.dtype == torch.float8_e4m3fn else INT8_MAX
        largest = torch.zeros_like(scale).index_reduce_(0, owner, x.abs().amax(-1), "amax")
        # largest / top = mantissa * 2^exponent, mantissa in [0.5, 1); by a tensor, because division by a number multiplies by its inverse
        mantissa, exponent = torch.frexp(largest / torch.full_like(largest, top))
        fresh = torch.ldexp(torch.ones_like(largest), torch.where(mantissa == 0.5, exponent - 1, exponent))
        fresh = torch.where(largest > 0, fresh, 0.0).clamp(min=SMALLEST_SCALE)
        old = scale[first]
        fresh[first] = torch.maximum(old, fresh[first])
        shrunk = _to_codes(codes.view(codes.dtype)[first].float() * (old / fresh[first])[:, :, None, None], codes)
        at_first = torch.where(earlier, shrunk.view(torch.uint8), codes.view(torch.uint8)[first])
        codes.view(torch.uint8)[first] = at_first
        scale[owner] = fresh[owner]
        _put(codes, (owner, slice(None), slot), _to_codes(x / fresh[owner][:, :, None], codes))
    return [st["k_cache"], st["k_scale"], st["v_cache"], st["v_scale"]]


def _gathered(codes, scale, table):
    """Cached values [B][hkv][width * page][head_dim] in 32 bits."""
    x = codes[table].float() * scale[table][..., None, None]
    n, w, h, p, d = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(n, h, w * p, d)


def _plain_attn(st):
    case = st["case"]
    hq, hkv, d = case["hq"], case["hkv"], case["head_dim"]
    g, n, most = hq // hkv, len(st["total"]), int(st["new"].max())
    table, length = st["page_table"].long(), st["length"].long()
    b, j, _ = _token_rows(st)
    q = torch.zeros((n, most, hq, d), device="cuda")
    q[b, j] = st["q"].float()
    q = q.view(n, most, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(n, hkv, most * g, d)
    key = torch.arange(table.shape[1] * case["page"], device="cuda")
    fresh = (st["row_offset"][1:] - st["row_offset"][:-1]).long()
    last = (length - fresh)[:, None] + torch.arange(most, device="cuda")[None]            # last position that a new token sees
    seen = (key[None, None] <= last[:, :, None]) & (key[None, None] < length[:, None, None])
    seen = seen.repeat_interleave(g, 1)[:, None]
    s = torch.matmul(q, _gathered(st["k_cache"], st["k_scale"], table).transpose(2, 3)) * (1.0 / math.sqrt(d))
    s = torch.where(seen, s, -torch.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), 0.0, m)
    p = torch.exp(s - m)
    del s
    z = p.sum(-1, keepdim=True)
    v = _gathered(st["v_cache"], st["v_scale"], table)
    v = torch.where((key[None] < length[:, None])[:, None, :, None], v, 0.0)
    p /= torch.where(z > 0, z, 1.0)
    o = torch.matmul(p, v)
    lse = (m + torch.log(z))[..., 0]

    def packed(x):
        x = x.view(n, hkv, most, g, -1).permute(0, 2, 1, 3, 4).reshape(n, most, hq, -1)
        return x[b, j]
    out = [packed(o).to(torch.bfloat16), packed(lse[..., None])[..., 0].contiguous()]
    if case["weights"]:
        p = torch.where((torch.arange(most, device="cuda")[None] < fresh[:, None]).repeat_interleave(g, 1)[:, None, :, None], p, 0.0)
        share = p.sum(2).view(n, hkv, -1, case["page"]).transpose(1, 2)
        st["weight"].index_add_(0, table.reshape(-1), share.reshape(-1, hkv, case["page"]))
        out.append(st["weight"])
    return out


def _plain_evict(st):
    case, page = st["case"], st["case"]["page"]
    sink, heavy, recent = case["sink"], case["heavy"], case["recent"]
    keep = sink + heavy + recent
    table, length = st["page_table"].long(), st["length"].long()
    n, h = len(length), case["hkv"]
    w = st["weight"][table].permute(0, 2, 1, 3).reshape(n, h, -1)
    at = torch.arange(w.shape[-1], device="cuda")
    fixed = (at[None] < sink) | (at[None] >= length[:, None] - recent) | (length[:, None] <= keep)
    w = torch.where(fixed[:, None], torch.inf, w)
    w = torch.where((at[None] < length[:, None])[:, None], w, -torch.inf)
    first = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :keep]
    if first.shape[-1] < keep:
        first = torch.nn.functional.pad(first, (0, keep - first.shape[-1]), value=int(at[-1]) + 1)
    new_length = torch.clamp(length, max=keep)
    rank = torch.arange(keep, device="cuda")
    valid = (rank[None] < new_length[:, None])[:, None].expand(n, h, keep)
    kept = torch.sort(torch.where(valid, first, 1 << 40), dim=-1).values
    st["kept"].copy_(torch.where(valid, kept, -1))
    st["new_length"].copy_(new_length)
    b, hh, r = torch.nonzero(valid, as_tuple=True)
    src = kept[b, hh, r]
    src_page, src_slot = table[b, src // page], src % page
    dst_page, dst_slot = st["dst_table"].long()[b, r // page], r % page
    for name in ("k", "v"):
        codes, scale = st[name + "_cache"], st[name + "_scale"]
        from_scale = scale[src_page, hh]
        blocks = torch.zeros(scale.numel(), device="cuda")
        blocks.index_reduce_(0, dst_page * h + hh, from_scale, "amax")
        to_scale = blocks[dst_page * h + hh]
        moved = codes[src_page, hh, src_slot].float() * (from_scale / to_scale)[:, None]
        _put(codes, (dst_page, hh, dst_slot), _to_codes(moved, codes))
        scale[dst_page, hh] = to_scale
    st["weight"][dst_page, hh, dst_slot] = st["weight"][src_page, hh, src_slot]
    return [st["kept"], st["new_length"], st["k_cache"], st["k_scale"], st["v_cache"], st["v_scale"], st["weight"]]


# ---------------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------------------------
def work(case):
    new, total = lengths_of(case)
    rows, d = int(new.sum()), case["head_dim"]
    if case["op"] == "rope":
        values = rows * (case["hq"] + case["hkv"]) * d
        return {"bytes": 4 * values, "flops": 3 * values * case["rotary_dim"] // d}
    h, page = case["hkv"], case["page"]
    if case["op"] == "append":
        return {"bytes": 2 * rows * h * d * 3 + 8 * h * int((-(-new // page)).sum()), "flops": 4 * rows * h * d}
    if case["op"] == "attn":
        pairs = int(sum(n * t - n * (n - 1) // 2 for n, t in zip(new.tolist(), total.tolist())))
        cached = int(total.sum())
        moved = 2 * cached * h * d + 8 * h * int((-(-total // page)).sum()) + rows * case["hq"] * (4 * d + 4)
        return {"bytes": moved + (8 * cached * h if case["weights"] else 0), "flops": 4 * pairs * case["hq"] * d}
    keep = case["sink"] + case["heavy"] + case["recent"]
    moved = int(np.minimum(total, keep).sum())
    return {"bytes": h * (4 * int(total.sum()) + moved * (4 * d + 8)), "flops": 2 * h * moved * d}


# ---------------------------------------------------------------------------------------------------------
# The definitions in 64 bits, one sequence after the other
# ---------------------------------------------------------------------------------------------------------
def _nearest(x, kind):
    """Nearest code value of each entry, ties to even."""
    if kind == "int8":
        return torch.round(x)
    exponent = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -40))).clamp(min=-6.0)
    step = torch.exp2(exponent - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    st = prepare(case, seed)
    return {"rope": _exact_rope, "append": _exact_append, "attn": _exact_attn, "evict": _exact_evict}[case["op"]](case, st)


def _exact_rope(case, st):
    f, magnitude = frequencies(case)
    f = torch.as_tensor(f, device="cuda")
    r, out = case["rotary_dim"], []
    starts = np.concatenate([[0], np.cumsum(st["new"])])
    position = np.concatenate([np.arange(n) + (t - n if case["cached"] else 0) for n, t in zip(st["new"], st["total"])])
    assert len(position) == starts[-1]
    turn = torch.polar(torch.full((), magnitude, dtype=torch.float64, device="cuda"),
                       torch.as_tensor(position, dtype=torch.float64, device="cuda")[:, None] * f)
    turn = turn.conj() if case["backward"] else turn
    for name in ("q", "k"):
        y = st[name].double()
        part = y[..., :r].clone()
        pair = part.unflatten(-1, (2, r // 2)).transpose(-1, -2) if case["layout"] == "half" else part.unflatten(-1, (r // 2, 2))
        z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn[:, None])
        y[..., :r] = (z.transpose(-1, -2) if case["layout"] == "half" else z).flatten(-2)
        out.append(y)
    return out


def _exact_append(case, st):
    page, kind = case["page"], case["kind"]
    top = E4M3_MAX if kind == "e4m3" else INT8_MAX
    table = st["page_table"].cpu().numpy()
    powers = torch.as_tensor(2.0 ** np.arange(-100, 128), device="cuda")
    out = []
    starts = np.concatenate([[0], np.cumsum(st["new"])])
    # every page touched: its rows in x, the place of the first of them, and how much it held
    jobs = []
    for b, (n, t) in enumerate(zip(st["new"].tolist(), st["total"].tolist())):
        for p in range((t - n) // page, (t - 1) // page + 1):
            lo, hi = max(t - n, p * page), min(t, (p + 1) * page)
            jobs.append((table[b, p], starts[b] + lo - (t - n), lo - p * page, hi - lo))
    jobs = np.asarray(jobs, np.int64).reshape(-1, 4)
    pages, at, held, count = (torch.as_tensor(jobs[:, i], device="cuda") for i in range(4))
    slots = torch.arange(page, device="cuda")[None]
    is_new = (slots >= held[:, None]) & (slots < (held + count)[:, None])
    row = torch.where(is_new, at[:, None] + slots - held[:, None], 0)
    for name in ("k", "v"):
        codes, scale = st[name + "_cache"].double(), st[name + "_scale"].double()
        for i in range(0, len(pages), 4096):       # a few thousand pages at a time
            pg, fresh = pages[i:i + 4096], is_new[i:i + 4096][..., None, None]
            x = st[name].double()[row[i:i + 4096]] * fresh                  # [pages][slot][head][dim]
            size = x.abs().amax((1, 3))
            new_scale = powers[torch.searchsorted(top * powers, size)]           # the smallest that covers it
            has = (held[i:i + 4096] > 0)[:, None]
            new_scale = torch.where(has, torch.maximum(new_scale, scale[pg]), new_scale)
            cur = codes[pg].transpose(1, 2)
            old = _nearest(cur * (scale[pg] / new_scale)[:, None, :, None], kind)
            before = (slots < held[i:i + 4096, None])[..., None, None]
            codes[pg] = torch.where(fresh, _nearest(x / new_scale[:, None, :, None], kind),
                                    torch.where(before, old, cur)).transpose(1, 2)
            scale[pg] = new_scale
        out += [codes if kind == "e4m3" else codes.to(torch.int8), scale]
    return out


def _exact_attn(case, st):
    hq, hkv, d, page = case["hq"], case["hkv"], case["head_dim"], case["page"]
    g = hq // hkv
    o = torch.zeros((st["rows"], hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((st["rows"], hq), -math.inf, dtype=torch.float64, device="cuda")
    weight = st["weight"].double() if case["weights"] else None
    row = 0
    for b, (n, t) in enumerate(zip(st["new"].tolist(), st["total"].tolist())):
        pages = st["page_table"][b, :-(-t // page)].long()
        seen = torch.arange(t, device="cuda")[None] <= torch.arange(t - n, t, device="cuda")[:, None]
        for h in range(hkv):
            k = (st["k_cache"][pages, h].double() * st["k_scale"][pages, h].double()[:, None, None]).reshape(-1, d)[:t]
            v = (st["v_cache"][pages, h].double() * st["v_scale"][pages, h].double()[:, None, None]).reshape(-1, d)[:t]
            s = torch.einsum("jgd,td->jgt", st["q"][row:row + n, h * g:(h + 1) * g].double(), k) / math.sqrt(d)
            s.masked_fill_(~seen[:, None], -math.inf)
            lse[row:row + n, h * g:(h + 1) * g] = torch.logsumexp(s, -1)
            p = torch.softmax(s, -1)
            o[row:row + n, h * g:(h + 1) * g] = torch.einsum("jgt,td->jgd", p, v)
            if weight is not None:
                position = torch.arange(t, device="cuda")
                weight[pages[position // page], h, position % page] += p.sum((0, 1))
        row += n
    return [o, lse] + ([weight] if weight is not None else [])


def _exact_evict(case, st):
    page, kind = case["page"], case["kind"]
    sink, heavy, recent = case["sink"], case["heavy"], case["recent"]
    keep = sink + heavy + recent
    table, dst = st["page_table"].cpu().numpy().astype(np.int64), st["dst_table"].cpu().numpy().astype(np.int64)
    weight = st["weight"].cpu().numpy()
    codes = {n: st[n + "_cache"].double() for n in ("k", "v")}
    scale = {n: st[n + "_scale"].double() for n in ("k", "v")}
    new_weight = st["weight"].double()
    kept = np.full((len(table), case["hkv"], keep), -1, np.int32)
    for b, t in enumerate(st["total"].tolist()):
        for h in range(case["hkv"]):
            w = weight[table[b, :-(-t // page)], h].reshape(-1)[:t]
            if t <= keep:
                chosen = np.arange(t)
            else:
                middle = w[sink:t - recent].astype(np.float64)
                best = sink + np.lexsort((np.arange(len(middle)), -middle))[:heavy]
                chosen = np.sort(np.concatenate([np.arange(sink), best, np.arange(t - recent, t)]))
            kept[b, h, :len(chosen)] = chosen
            src = torch.as_tensor(table[b, chosen // page], device="cuda"), torch.as_tensor(chosen % page, device="cuda")
            r = np.arange(len(chosen))
            to = torch.as_tensor(dst[b, r // page], device="cuda"), torch.as_tensor(r % page, device="cuda")
            blocks = -(-len(chosen) // page)
            for n in ("k", "v"):
                s = scale[n][src[0], h]
                each = torch.zeros(blocks * page, dtype=torch.float64, device="cuda")
                each[:len(chosen)] = s
                top = each.view(blocks, page).amax(1)
                codes[n][to[0], h, to[1]] = _nearest(codes[n][src[0], h, src[1]] * (s / top[torch.as_tensor(r // page, device="cuda")])[:, None], kind)
                scale[n][torch.as_tensor(dst[b, :blocks], device="cuda"), h] = top
            new_weight[to[0], h, to[1]] = new_weight[src[0], h, src[1]]
    new_length = np.minimum(st["total"], keep).astype(np.int32)
    out = []
    for n in ("k", "v"):
        out += [codes[n] if kind == "e4m3" else codes[n].to(torch.int8), scale[n]]
    return [torch.as_tensor(kept), torch.as_tensor(new_length), *out, new_weight]
