"""Host-side checks of rotary positions and of the paged cache: frequencies, refusals (none of which needs a GPU), index
arithmetic of the kernels compiled for the host, and pins of the definitions the GPU tests compare with."""
import ctypes as C
import math
import os
import re
import subprocess

import numpy as np
import pytest

from oracle import serving_ref as R
from paper_2602_21788_b200 import build, fcp

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2602_21788_b200", "csrc")


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


# ------------------------------------------------------------------------------------------ rotary table
@pytest.mark.parametrize("rotary", [4, 32, 64, 126, 128])
@pytest.mark.parametrize("scaling,more", [
    ("none", {}), ("linear", dict(factor=4.0)), ("ntk", dict(factor=8.0)),
    ("yarn", dict(factor=32.0, original_length=4096.0)), ("yarn", dict(factor=2.0, original_length=64.0, low=2.0, high=9.0)),
    ("wavelength", dict(factor=8.0, original_length=8192.0)), ("wavelength", dict(factor=3.0, original_length=100.0, low=0.5, high=3.0)),
])
def test_frequencies_of_every_scaling(rotary, scaling, more):
    t = fcp.RopeTable(128, rotary, base=500000.0, scaling=scaling, **more)
    want = R.rope_frequencies(rotary, 500000.0, scaling, **more)
    # 64-bit fractions of a turn: relative 2^-52 of the formula's own double arithmetic (a few operations), absolute 2^-64 turns
    assert np.allclose(t.frequencies(), want, rtol=64 * 2.0 ** -53, atol=2 * math.pi * 2.0 ** -63)
    assert t.struct.magnitude == np.float32(R.rope_magnitude(scaling, more.get("factor", 1.0)))


def test_magnitude_is_taken_if_given():
    assert fcp.RopeTable(64, scaling="yarn", factor=4.0, original_length=1.0, magnitude=1.5).struct.magnitude == 1.5


@pytest.mark.parametrize("args,status", [
    (dict(head_dim=96), fcp.FCP_ERR_UNSUPPORTED), (dict(head_dim=64, rotary_dim=66), fcp.FCP_ERR_INVALID_ARG),
    (dict(head_dim=64, rotary_dim=7), fcp.FCP_ERR_INVALID_ARG), (dict(head_dim=64, rotary_dim=0), fcp.FCP_ERR_INVALID_ARG),
    (dict(head_dim=64, layout=2), fcp.FCP_ERR_INVALID_ARG), (dict(head_dim=64, scaling=9), fcp.FCP_ERR_INVALID_ARG),
    (dict(head_dim=64, base=1.0), fcp.FCP_ERR_INVALID_ARG), (dict(head_dim=64, base=math.nan), fcp.FCP_ERR_INVALID_ARG),
    (dict(head_dim=64, scaling="linear", factor=0.5), fcp.FCP_ERR_INVALID_ARG),
    (dict(head_dim=64, rotary_dim=2, scaling="ntk", factor=2.0), fcp.FCP_ERR_INVALID_ARG),
    (dict(head_dim=64, scaling="yarn", factor=2.0), fcp.FCP_ERR_INVALID_ARG),
    (dict(head_dim=64, scaling="wavelength", factor=2.0, original_length=10.0, low=4.0, high=4.0), fcp.FCP_ERR_INVALID_ARG),
    (dict(head_dim=64, scaling="wavelength", factor=math.inf, original_length=10.0), fcp.FCP_ERR_INVALID_ARG),
])
def test_tables_that_are_refused(args, status):
    with pytest.raises(fcp.FcpError) as e:
        fcp.RopeTable(**args)
    assert e.value.status == status
    with pytest.raises(ValueError):
        fcp.RopeTable(64, layout="diagonal")


def test_rope_calls_that_are_refused():
    L, t = fcp.lib(), fcp.RopeTable(64)
    x = np.zeros(4096, np.uint16)
    p = x.ctypes.data
    base = dict(T=4, q=p, qs=0, hq=2, k=p, ks=0, hkv=1, qo=p, qos=0, ko=p, kos=0, pos=p, off=None, length=None, B=0)

    def call(table=t.ref, f=L.fcp_rope_fwd, **more):
        return f(table, *{**base, **more}.values(), None)
    bad = [dict(table=None), dict(T=-1), dict(T=1 << 31), dict(q=None), dict(ko=None), dict(hq=-1), dict(pos=None), dict(B=-1), dict(qs=64),
           dict(kos=63), dict(q=p + 1), dict(hq=65536)]
    for f in (L.fcp_rope_fwd, L.fcp_rope_bwd):
        for more in bad:
            assert call(f=f, **more) == fcp.FCP_ERR_INVALID_ARG, more
            assert fcp.lib().fcp_last_error_message()
        for nothing in (dict(T=0), dict(T=0, q=None, k=None, qo=None, ko=None, pos=None), dict(hq=0, hkv=0), dict(pos=None, off=p, B=0)):       # nothing to do: no GPU is asked for
            assert call(f=f, **nothing) == fcp.FCP_OK
    blank = fcp.FcpRopeTable()
    assert call(table=C.byref(blank)) == fcp.FCP_ERR_INVALID_ARG
    a, b = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(4, 1, 64, dtype=torch.bfloat16)
    off = torch.zeros(2, dtype=torch.int32)
    for args in [(a.float(), b, a, b), (a, b, b, b), (a, b[:3], a, b[:3]), (a.transpose(0, 1), b, a, b), (a[..., :32], b, a[..., :32], b)]:
        with pytest.raises(ValueError):
            fcp.fcp_rope_fwd(t, *args, row_offset=off)
    with pytest.raises(ValueError):
        fcp.fcp_rope_fwd(t, a, b, a, b, positions=torch.zeros(4, dtype=torch.int64))


# ------------------------------------------------------------------------------------------ cache refusals
def _config(**more):
    buf = np.zeros(1 << 12, np.uint8)
    p = buf.ctypes.data // 256 * 256 + 256
    c = dict(k=p, v=p, k_scale=p, v_scale=p, weight=p, status=p, n_pages=4, page_tokens=16, hkv=2, head_dim=64, kind=0, **{})
    c.update(more)
    return buf, fcp.FcpCacheConfig(*c.values())


@pytest.mark.parametrize("more,status", [
    (dict(k=None), -1), (dict(v=None), -1), (dict(k_scale=None), -1), (dict(v_scale=None), -1), (dict(status=None), -1),
    (dict(n_pages=0), -1), (dict(hkv=0), -1), (dict(head_dim=80), -3), (dict(page_tokens=48), -3), (dict(page_tokens=8), -3),
    (dict(kind=2), -1), (dict(kind=-1), -1), (dict(n_pages=1 << 26), -1), (dict(n_pages=(1 << 31) - 1), -1), (dict(k=0x1008), -1),
    (dict(k_scale=0x1002), -1), (dict(weight=0x1001), -1),
])
def test_descriptions_that_are_refused(more, status):
    buf, c = _config(**more)
    h = C.c_void_p(1)
    assert fcp.lib().fcp_cache_create(C.byref(c), C.byref(h)) == status
    assert not h.value


def test_largest_pool_and_null_arguments():
    L = fcp.lib()
    buf, c = _config(n_pages=(1 << 26) - 1)                  # 2^26 - 1 pages of 2 heads and 16 tokens: 2^31 - 32 rows
    h = C.c_void_p()
    assert L.fcp_cache_create(C.byref(c), C.byref(h)) == fcp.FCP_OK and h.value
    assert L.fcp_cache_destroy(h) == fcp.FCP_OK and L.fcp_cache_destroy(None) == fcp.FCP_OK
    assert L.fcp_cache_create(None, C.byref(h)) == fcp.FCP_ERR_INVALID_ARG
    assert L.fcp_cache_create(C.byref(c), None) == fcp.FCP_ERR_INVALID_ARG
    assert L.fcp_cache_device_status(None, None) == fcp.FCP_ERR_INVALID_ARG


def test_cache_calls_that_are_refused():
    L = fcp.lib()
    buf, c = _config()
    buf2, c2 = _config(weight=None)
    h, h2 = C.c_void_p(), C.c_void_p()
    assert L.fcp_cache_create(C.byref(c), C.byref(h)) == 0 and L.fcp_cache_create(C.byref(c2), C.byref(h2)) == 0
    p = c.k
    good = dict(B=2, rows=4, max_new=2, table_width=3, page_table=p, length=p, row_offset=p)
    n = C.c_int64()

    def batch(**more):
        return C.byref(fcp.FcpCacheBatch(*{**good, **more}.values()))

    def append(b=batch(), hh=h, k=p, ks=0, v=p, vs=0):
        return L.fcp_cache_append(hh, b, k, ks, v, vs, None)

    def attn(b=batch(), hh=h, q=p, qs=0, hq=4, scale=0.0, o=p, lse=p, acc=0, ws=p, wsb=1 << 40):
        return L.fcp_cache_attn(hh, b, q, qs, hq, scale, o, lse, acc, ws, wsb, None)

    def evict(b=batch(), hh=h, sink=1, heavy=2, recent=3, dst=p, width=1, new=p, kept=p):
        return L.fcp_cache_evict(hh, b, sink, heavy, recent, dst, width, new, kept, None)
    for call in (append, attn, evict):
        assert call(hh=None) == -1 and call(b=None) == -1
        for more in (dict(B=-1), dict(table_width=0), dict(table_width=1 << 27), dict(table_width=(1 << 27) - 15), dict(page_table=None), dict(length=None)):
            assert call(b=batch(**more)) == -1, more
        assert call(b=batch(B=0)) == 0
    for call in (append, attn):
        for more in (dict(rows=-1), dict(max_new=-1), dict(max_new=5), dict(row_offset=None), dict(rows=(1 << 31) - 2, max_new=1)):
            assert call(b=batch(**more)) == -1, more
        assert call(b=batch(rows=0, max_new=0)) == 0 and call(b=batch(max_new=0)) == 0
    for more in (dict(k=None), dict(v=None), dict(k=p + 8), dict(ks=127), dict(vs=132), dict(ks=64)):
        assert append(**more) == -1, more
    for more in (dict(q=None), dict(q=p + 2), dict(qs=255), dict(qs=260), dict(o=None), dict(lse=None), dict(o=p + 2), dict(lse=p + 2),
                 dict(hq=0), dict(hq=-2), dict(scale=math.nan), dict(scale=math.inf), dict(hh=h2, acc=1)):
        assert attn(**more) == -1, more
    assert attn(hq=3) == fcp.FCP_ERR_UNSUPPORTED
    assert L.fcp_cache_attn_workspace_bytes(h, batch(), 4, C.byref(n)) == 0 and n.value > 0
    assert attn(wsb=n.value - 1) == attn(ws=None) == attn(ws=p + 64) == fcp.FCP_ERR_WORKSPACE
    assert L.fcp_cache_attn_workspace_bytes(h, batch(), 4, None) == -1
    assert L.fcp_cache_attn_workspace_bytes(h, batch(), 5, C.byref(n)) == fcp.FCP_ERR_UNSUPPORTED
    for more in (dict(hh=h2), dict(sink=-1), dict(heavy=-1), dict(recent=-1), dict(sink=0, heavy=0, recent=0), dict(width=0), dict(recent=14),
                 dict(dst=None), dict(new=None), dict(kept=None), dict(heavy=(1 << 31) - 1, recent=(1 << 31) - 1)):
        assert evict(**more) == -1, more
    assert evict(b=batch(B=65536)) == fcp.FCP_ERR_UNSUPPORTED
    assert L.fcp_cache_destroy(h) == 0 and L.fcp_cache_destroy(h2) == 0


def test_binding_checks_shapes():
    z = lambda *s, t=torch.float32: torch.zeros(s, dtype=t)
    k, sc, st = z(3, 2, 16, 64, t=torch.int8), z(3, 2), z(4, t=torch.int32)
    cache = fcp.Cache(k, k.clone(), sc, sc.clone(), st)
    for args in [(k, k[:2], sc, sc, st), (k, k, sc[:2], sc, st), (k, k, sc, sc, st[:3]), (k, k, sc.double(), sc, st), (k, k, sc, sc, st, z(3, 2, 32)),
                 (k.transpose(0, 1), k, sc, sc, st), (k.view(torch.uint8), k, sc, sc, st), (k.view(torch.float8_e5m2), k, sc, sc, st)]:
        with pytest.raises(ValueError):
            fcp.Cache(*args)
    assert fcp.Cache(k.view(torch.uint8), k, sc, sc, st, kind="e4m3").handle.value and fcp.Cache(k.view(torch.float8_e4m3fn), k, sc, sc, st).handle.value
    table, length, off = z(2, 3, t=torch.int32), z(2, t=torch.int32), z(3, t=torch.int32)
    batch = fcp.CacheBatch(table, length, off, rows=2)
    for args in [(table, length[:1], off), (table, length, off[:2]), (table.long(), length, off)]:
        with pytest.raises(ValueError):
            fcp.CacheBatch(*args, rows=2)
    x = z(2, 2, 64, t=torch.bfloat16)
    for a, b in [(x[:1], x), (x, x[:, :1]), (x.float(), x)]:
        with pytest.raises(ValueError):
            fcp.fcp_cache_append(cache, batch, a, b)
    for q, o, lse in [(x, x[:1], z(2, 2)), (x, x, z(2, 3)), (x, x.float(), z(2, 2))]:
        with pytest.raises(ValueError):
            fcp.fcp_cache_attn(cache, batch, q, o, lse, None, 0)
    with pytest.raises(ValueError):
        fcp.fcp_cache_evict(cache, batch, 1, 1, 1, table[:1], length, z(2, 2, 3, t=torch.int32))
    with pytest.raises(ValueError):
        fcp.fcp_cache_evict(cache, batch, 1, 1, 1, table, length, z(2, 2, 4, t=torch.int32))



def test_sizes_next_to_2_to_the_31_are_refused():
    """Where the kernels' 32-bit loops would pass the end: 2^31 - 8192 kept tokens are the most, 2^31 - 257 sequences of rotary calls."""
    L, t = fcp.lib(), fcp.RopeTable(64)
    buf, c = _config()
    h = C.c_void_p()
    assert L.fcp_cache_create(C.byref(c), C.byref(h)) == 0
    p = c.k
    batch = C.byref(fcp.FcpCacheBatch(0, 0, 0, 3, p, p, p))          # no sequences: what is not refused does nothing
    evict = lambda *keep: L.fcp_cache_evict(h, batch, *keep, p, 1 << 27, p, p, None)
    assert evict(4, (1 << 31) - 8192 - 20, 16) == evict((1 << 31) - 8192, 0, 0) == 0
    for keep in ((4, (1 << 31) - 8191 - 20, 16), ((1 << 31) - 8191, 0, 0), (0, 0, (1 << 31) - 1), (0, (1 << 31) - 1, 0)):
        assert evict(*keep) == fcp.FCP_ERR_INVALID_ARG, keep
    assert L.fcp_cache_destroy(h) == 0
    for f in (L.fcp_rope_fwd, L.fcp_rope_bwd):
        rope = lambda B: f(t.ref, 0, p, 0, 1, None, 0, 0, p, 0, None, 0, None, p, None, B, None)
        assert rope((1 << 31) - 257) == 0
        assert rope((1 << 31) - 256) == rope((1 << 31) - 1) == fcp.FCP_ERR_INVALID_ARG


def test_binding_refuses_types_and_rows_that_share_memory():
    """Expanded tensors (row stride 0, which the library takes for dense rows), other 2-byte and 4-byte types."""
    t = fcp.RopeTable(64)
    cache, batch, x, lse = _host_cache()
    one = torch.zeros(1, 2, 64, dtype=torch.bfloat16)
    wide = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    overlapping = torch.zeros(1000, dtype=torch.bfloat16).as_strided((2, 2, 64), (64, 64, 1))
    off = torch.tensor([0, 2], dtype=torch.int32)
    for bad in (one.expand(2, 2, 64), overlapping, x.half(), x.view(torch.int16)):
        for call in (fcp.fcp_rope_fwd, fcp.fcp_rope_bwd):
            for args in [(bad, None, x, None), (x, None, bad, None), (None, bad, None, x), (None, x, None, bad)]:
                with pytest.raises(ValueError, match="bf16|share memory"):
                    call(t, *args, row_offset=off)
        for args in [(bad, x), (x, bad)]:
            with pytest.raises(ValueError, match="bf16|share memory"):
                fcp.fcp_cache_append(cache, batch, *args)
        for q, o in [(bad, x), (x, bad)]:
            with pytest.raises(ValueError, match="bf16|share memory|contiguous"):
                fcp.fcp_cache_attn(cache, batch, q, o, lse, None, 0)
    assert fcp._heads(wide[:, :2], 64, "q")[2] == 256 and fcp._heads(one.expand(1, 2, 64), 64, "q")[2] == 128        # slices, single rows
    for bad in (lse.int(), lse.double(), lse.half()):
        with pytest.raises(ValueError, match="fp32"):
            fcp.fcp_cache_attn(cache, batch, x, x, bad, None, 0)
    with pytest.raises(ValueError, match="workspace"):
        fcp.fcp_cache_attn(cache, batch, x, x, lse, torch.zeros(10, dtype=torch.uint8), 11)
    k, v, ks, vs, status, weight = (torch.zeros(s, dtype=d) for s, d in (((3, 2, 16, 64), torch.int8), ((3, 2, 16, 64), torch.int8), ((3, 2), torch.float32),
                                    ((3, 2), torch.float32), (4, torch.int32), ((3, 2, 16), torch.float32)))
    for args in [(k, v, ks.int(), vs, status, weight), (k, v, ks, vs.int(), status, weight), (k, v, ks, vs, status.float(), weight), (k, v, ks, vs, status, weight.int())]:
        with pytest.raises(ValueError):
            fcp.Cache(*args)
    table = torch.zeros(2, 3, dtype=torch.int32)
    for bad in (table.float(), table.bool(), table.short()):
        with pytest.raises(ValueError, match="int32"):
            fcp.CacheBatch(bad, batch.tensors[1])


def _host_cache():
    """A cache, a batch of two rows and tensors of its calls, all in host memory."""
    k = torch.zeros(3, 2, 16, 64, dtype=torch.int8)
    cache = fcp.Cache(k, k.clone(), torch.ones(3, 2), torch.ones(3, 2), torch.zeros(4, dtype=torch.int32), weight=torch.zeros(3, 2, 16))
    batch = fcp.CacheBatch(torch.zeros(2, 3, dtype=torch.int32), torch.ones(2, dtype=torch.int32), torch.tensor([0, 1, 2], dtype=torch.int32), rows=2)
    return cache, batch, torch.zeros(2, 2, 64, dtype=torch.bfloat16), torch.zeros(2, 2)


class _Elsewhere:
    """A tensor of host memory that says it lies on a GPU."""

    def __init__(self, x, device):
        self.x, self.device_number = x, device

    def get_device(self):
        return self.device_number

    def __getattr__(self, name):
        return getattr(self.x, name)


def test_binding_refuses_tensors_of_other_devices():
    t, x = fcp.RopeTable(64), torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    off = torch.tensor([0, 2], dtype=torch.int32)
    for args in [(x, None, x, None), (None, x, None, x), (x, x, x, x)]:
        with pytest.raises(ValueError, match="one GPU"):
            fcp.fcp_rope_fwd(t, *args, row_offset=off)
    here = lambda y: _Elsewhere(y, 0)
    for args in [(here(x), None, x, None), (here(x), None, _Elsewhere(x, 1), None), (here(x), here(x), here(x), x)]:
        with pytest.raises(ValueError, match="one GPU"):
            fcp.fcp_rope_fwd(t, *args, row_offset=here(off))
    with pytest.raises(ValueError, match="one GPU"):
        fcp.fcp_rope_fwd(t, here(x), None, here(x), None, row_offset=off)
    cache, batch, x, lse = _host_cache()
    k, v, ks, vs, status, weight = cache.tensors
    for i in range(6):
        parts = [here(y) for y in (k, v, ks, vs, status, weight)]
        parts[i] = parts[i].x
        with pytest.raises(ValueError, match="different devices"):
            fcp.Cache(*parts, kind="int8")
    table, length, row_offset = batch.tensors
    for args in [(here(table), length, here(row_offset)), (here(table), here(length), row_offset)]:
        with pytest.raises(ValueError, match="different devices"):
            fcp.CacheBatch(*args, rows=2)
    cache.device = 0                                              # as if its pages were there
    for b in (batch, fcp.CacheBatch(_Elsewhere(table, 1), _Elsewhere(length, 1), _Elsewhere(row_offset, 1), rows=2)):
        with pytest.raises(ValueError, match="batch does not"):
            fcp.fcp_cache_append(cache, b, here(x), here(x))
    there = fcp.CacheBatch(here(table), here(length), here(row_offset), rows=2)
    for args in [(x, here(x)), (here(x), x), (here(x), _Elsewhere(x, 1))]:
        with pytest.raises(ValueError, match="one GPU"):
            fcp.fcp_cache_append(cache, there, *args)
    ws = torch.zeros(16, dtype=torch.uint8)
    for args in [(x, here(x), here(lse), here(ws)), (here(x), x, here(lse), here(ws)), (here(x), here(x), lse, here(ws)), (here(x), here(x), here(lse), ws)]:
        with pytest.raises(ValueError, match="one GPU"):
            fcp.fcp_cache_attn(cache, there, *args, 16)
    kept = torch.zeros(2, 2, 3, dtype=torch.int32)
    for args in [(table, here(length), here(kept)), (here(table), length, here(kept)), (here(table), here(length), kept)]:
        with pytest.raises(ValueError, match="one GPU"):
            fcp.fcp_cache_evict(cache, there, 1, 1, 1, *args)


# ------------------------------------------------------------------------------------------ index arithmetic
INDEX_MAIN = r"""
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "fcp_cache_index.hpp"
using namespace fcp;
static void want(bool ok, const char* what, long a, long b, long c) {
  if (!ok) { printf("%s %ld %ld %ld\n", what, a, b, c); exit(1); }
}
int main() {
  // pages: outside -> -1, inside -> the row, up to the last one below 2^31
  want(page_row(-1, 5, 3, 0, 16) == -1 && page_row(5, 5, 3, 0, 16) == -1 && page_row(2147483647, 5, 3, 0, 16) == -1 && page_row(-2147483647 - 1, 5, 3, 0, 16) == -1, "page", 0, 0, 0);
  want(page_row(4, 5, 3, 2, 16) == (4 * 3 + 2) * 16, "row", 0, 0, 0);
  want(page_row((1 << 26) - 2, (1 << 26) - 1, 2, 1, 16) == 2147483647 - 47, "last row", page_row((1 << 26) - 2, (1 << 26) - 1, 2, 1, 16), 0, 0);
  // sequences: whatever the device holds, a usable view stays inside the buffers
  const int odd[] = {-2147483647 - 1, -1, 0, 1, 7, 63, 64, 65, 2147483647};
  for (int x : odd) for (int y : odd) for (int l : odd) {
    SeqView s = seq_view(x, y, l, 64, 7, 64);
    want(s.row0 >= 0 && s.n >= 0 && (long)s.row0 + s.n <= 64 && s.n <= 7 && s.length >= 0 && s.length <= 64, "view", x, y, l);
    const bool good = x >= 0 && y >= x && y <= 64 && (long)y - x <= 7 && l >= 0 && l <= 64;
    want(good == (s.bad == 0), "bad", x, y, l);
    if (s.bad) want(s.n == 0 && s.length == 0, "absent", x, y, l);
  }
  // append: the slots of a batch touch every (sequence, page with new tokens) once, and every new token once
  srand(7);
  for (int trial = 0; trial < 4000; ++trial) {
    const int p = 16 << (rand() % 4), B = 1 + rand() % 6;
    std::vector<int> off(1, 0), len;
    for (int b = 0; b < B; ++b) {
      const int n = rand() % 4 == 0 ? 0 : rand() % (trial % 3 == 0 ? 3 : 300);
      off.push_back(off.back() + n);
      len.push_back(rand() % 8 == 0 ? n / 2 : n + rand() % 200);          // now and then more rows than tokens
    }
    const int slots = append_slot(off.back(), B, p);
    std::vector<std::vector<int>> seen(B);
    for (int b = 0; b < B; ++b) seen[b].assign(len[b] + 1, 0);
    for (int w = 0; w < slots; ++w) {
      int lo = 0, hi = B - 1;
      while (lo < hi) { const int mid = (lo + hi + 1) / 2; if (append_slot(off[mid], mid, p) <= w) lo = mid; else hi = mid - 1; }
      const SeqView s = seq_view(off[lo], off[lo + 1], len[lo], off.back(), 300, 1 << 20);
      const AppendSpan a = append_span(s, w - append_slot(s.row0, lo, p), p);
      for (int t = a.lo; t < a.hi; ++t) { want(t >= 0 && t < len[lo] && t / p == a.page, "span", t, a.page, lo); ++seen[lo][t]; }
    }
    for (int b = 0; b < B; ++b)
      for (int t = 0; t < len[b]; ++t) want(seen[b][t] == (t >= len[b] - (off[b + 1] - off[b])), "cover", b, t, seen[b][t]);
  }
  // far ends: no overflow
  SeqView far = {0, 100, 2147483647 - 16, 0};
  for (int i = 0; i < 9; ++i) { AppendSpan a = append_span(far, i, 16); want(a.hi <= far.length && a.lo >= 0, "far", i, a.lo, a.hi); }
  puts("ok");
}
"""


def test_index_arithmetic_stays_inside_the_buffers(tmp_path):
    src, exe = tmp_path / "index.cpp", tmp_path / "index"
    src.write_text(INDEX_MAIN)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined,address", "-fno-sanitize-recover=all", "-I", CSRC, str(src), "-o", str(exe)],
                   check=True, capture_output=True, text=True)
    assert subprocess.run([str(exe)], capture_output=True, text=True).stdout.strip() == "ok"


def test_codes_of_the_header_match_the_index_arithmetic():
    hdr = open(os.path.join(ROOT, "include", "fcp.h")).read()
    code = {n: int(v) for n, v in re.findall(r"#define FCP_CACHE_BAD_(\w+)\s+(\d+)", hdr)}
    assert code == dict(LENGTH=1001, ROWS=1002, PAGE=1003, SCALE=1004)
    index = open(os.path.join(CSRC, "fcp_cache_index.hpp")).read()
    assert "s.bad = 1002" in index and "s.bad = 1001" in index


@pytest.mark.parametrize("name", ["fcp_rope.cu", "fcp_cache.cuh"])
def test_every_kernel_waits_for_the_one_before_it(name):
    """Kernels become resident while the one before them still writes: each one waits in front of its first access."""
    code = re.sub(r"/\*.*?\*/|//[^\n]*", "", open(os.path.join(CSRC, name)).read(), flags=re.S)
    bodies = re.findall(r"__global__[^{;]*\)\s*\{(.*?)\n\}", code, flags=re.S)
    assert len(bodies) == {"fcp_rope.cu": 1, "fcp_cache.cuh": 8}[name]
    for body in bodies:
        wait = re.search(r"grid_(begin|wait)\(\)", body)
        assert wait and not re.search(r"\bld_|tma_load", body[:wait.start()])
    assert "__restrict__" not in code and "__ldg" not in code


# ------------------------------------------------------------------------------------------ pins of the definitions
def test_rope_definition_turns_and_its_transpose_turns_back():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((5, 2, 64))
    f = R.rope_frequencies(32, 10000.0)
    pos = [0, 1, 2, 1000, 77777]
    for layout in ("half", "interleaved"):
        y = R.rope(x, pos, f, 32, layout)
        assert np.allclose(np.linalg.norm(y, axis=-1), np.linalg.norm(x, axis=-1))
        assert np.array_equal(y[0], x[0]) and np.array_equal(y[..., 32:], x[..., 32:])
        assert np.allclose(R.rope(y, pos, f, 32, layout, backward=True), x)
        # products of a query and a key depend on the distance alone
        q, k = rng.standard_normal((1, 1, 64)), rng.standard_normal((1, 1, 64))
        dot = lambda a, b: float((R.rope(q, [a], f, 32, layout) * R.rope(k, [b], f, 32, layout)).sum())
        assert math.isclose(dot(5, 3), dot(1005, 1003), rel_tol=1e-9)
        assert np.allclose(R.rope(x, pos, f, 32, layout, magnitude=2.0)[..., :32], 2 * y[..., :32])


def test_code_definitions():
    v = R.e4m3_values()
    assert np.nanmax(v) == 448 and v[1] == 2.0 ** -9 and np.isnan(v[127]) and np.isnan(v[255])
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(t, v.astype(np.float32), equal_nan=True)
    x = np.random.default_rng(1).standard_normal(20000) * 100
    x = np.clip(x, -448, 448).astype(np.float32)
    assert np.array_equal(R.nearest("e4m3", x), torch.from_numpy(x).to(torch.float8_e4m3fn).float().numpy())
    assert R.nearest("int8", [2.5, -3.5, 200, np.inf, np.nan]).tolist() == [2, -4, 127, 127, 0]
    assert R.fresh_scale("e4m3", [448.0]) == 1 and R.fresh_scale("e4m3", [449.0]) == 2 and R.fresh_scale("int8", [127.0]) == 1
    assert R.fresh_scale("int8", []) == R.fresh_scale("e4m3", [0.0]) == 2.0 ** -100
    assert R.fresh_scale("e4m3", [np.inf]) == 2.0 ** 120 and R.fresh_scale("int8", [np.inf]) == 2.0 ** 122


def test_attention_definition_against_scipy():
    from scipy.special import logsumexp, softmax
    rng = np.random.default_rng(2)
    state = dict(k=rng.integers(-127, 128, (4, 1, 16, 64)).astype(float), v=rng.integers(-127, 128, (4, 1, 16, 64)).astype(float),
                 k_scale=rng.random((4, 1)) / 64, v_scale=rng.random((4, 1)) / 64)
    q = rng.standard_normal((2, 3, 64))
    r = R.attention(state, [[2, 0, 3]], [40], [0, 2], q)
    k, v = R.gather(state, "k", [2, 0, 3], 40, 0), R.gather(state, "v", [2, 0, 3], 40, 0)
    s = np.einsum("jhd,td->jht", q, k) / 8
    s[0, :, 39] = -np.inf
    assert np.allclose(r["lse"], logsumexp(s, -1)) and np.allclose(r["o"], softmax(s, -1) @ v)
    assert np.allclose(r["weights"][0][0], softmax(s, -1).sum((0, 1))) and math.isclose(r["weights"][0].sum(), 6.0)


def test_eviction_definition():
    w = [9, 1, 5, 5, float("nan"), 5, 0, 2, 3]
    assert R.choose(w, 1, 2, 2).tolist() == [0, 2, 3, 7, 8]
    assert R.choose(w, 0, 9, 0).tolist() == list(range(9))
    assert R.choose(w, 2, 5, 1).tolist() == [0, 1, 2, 3, 5, 6, 7, 8]
