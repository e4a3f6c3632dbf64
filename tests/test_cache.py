"""Rotary positions and the plain cache, host side: the plan of the pairs, what every entry point refuses before any launch,
and the pins of the plain fp64 statement that the GPU tests compare with.  No GPU needed."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from oracle import wave_oracle as wo
from paper_2505_02922_amd import binding as wb
from paper_2505_02922_amd import synth

ARG, SHAPE, DTYPE, WORKSPACE = 1, 2, 3, 4
FAKE = 0x10000


@pytest.mark.parametrize("rot,sections,order", [(128, [64], 0), (128, [16, 24, 24], 0), (128, [16, 24, 24], 1), (64, [5, 0, 27], 1),
                                                (96, [16, 16, 16], 2), (16, [1, 2, 3, 2], 2), (64, [0, 32], 0)])
def test_rotary_plan(rot, sections, order):
    r = wb.wave_rotary_plan(rot, 500000.0, sections, order, wb.WAVE_ROTARY_NEIGHBOURS)
    axis, freq = co.pair_plan(rot, 500000.0, sections, order)
    assert (r.rot_dim, r.n_axes, r.pairing) == (rot, len(sections), 1)
    assert list(r.axis)[:rot // 2] == axis
    assert np.allclose(list(r.inv_freq)[:rot // 2], freq, rtol=1e-14, atol=0)


def test_rotary_plan_refuses():
    for rot, base, sections, order, pairing, status in [
            (0, 1e4, [0], 0, 0, SHAPE), (24, 1e4, [12], 0, 0, SHAPE), (144, 1e4, [72], 0, 0, SHAPE),
            (64, 1e4, [31], 0, 0, SHAPE), (64, 1e4, [16, 17], 0, 0, SHAPE), (64, 1e4, [33, -1], 0, 0, ARG),
            (64, 0.0, [32], 0, 0, ARG), (64, math.inf, [32], 0, 0, ARG), (64, math.nan, [32], 0, 0, ARG),
            (64, 1e4, [], 0, 0, ARG), (64, 1e4, [8, 8, 8, 4, 4], 0, 0, ARG), (64, 1e4, [32], 3, 0, ARG),
            (64, 1e4, [32], 0, 2, ARG)]:
        with pytest.raises(wb.WaveError) as e:
            wb.wave_rotary_plan(rot, base, sections, order, pairing)
        assert e.value.status == status, (rot, base, sections, order, pairing)


def test_struct_layouts():
    assert ctypes.sizeof(wb.wave_cache) == 5 * 4 + 4 + 6 * 8
    assert ctypes.sizeof(wb.wave_rotary) == 4 * (3 + 64) + 4 + 8 * 64


def _cache(dtype=1, B=2, Hkv=2, d=128, capacity=64, base=FAKE):
    c = wb.wave_cache()
    c.dtype, c.B, c.Hkv, c.d, c.capacity = dtype, B, Hkv, d, capacity
    rows = B * Hkv * capacity
    at = base
    for name, size in (("k", rows * d * 4), ("v", rows * d * 4), ("positions", rows * 4), ("weights", rows * 4),
                       ("lengths", B * 4), ("tokens", B * 4)):
        setattr(c, name, at)
        at += (size + 4095) // 4096 * 4096
    return c


def _changed(c, **kw):
    n = wb.wave_cache()
    ctypes.memmove(ctypes.byref(n), ctypes.byref(c), ctypes.sizeof(c))
    for k, v in kw.items():
        setattr(n, k, v)
    return n


BAD_CACHES = [(dict(dtype=2), DTYPE), (dict(B=0), ARG), (dict(Hkv=0), ARG), (dict(capacity=0), ARG), (dict(d=96), SHAPE),
              (dict(B=1 << 24), SHAPE), (dict(k=0), ARG), (dict(v=0), ARG), (dict(lengths=0), ARG), (dict(k=FAKE + 8), ARG),
              (dict(v=FAKE + 4), ARG)]


def test_rotary_apply_refuses():
    r = wb.wave_rotary_plan(64, 1e4)
    L = wb.lib()
    x, y = 0x100000, 0x900000
    call = lambda x=x, coords=FAKE, r=r, dt=1, B=2, H=3, N=5, d=128, y=y: L.wave_rotary_apply(
        x, coords, ctypes.byref(r) if r is not None else None, dt, B, H, N, d, y, None)
    assert call(dt=2) == DTYPE and call(d=96) == SHAPE and call(B=0) == ARG and call(H=0) == ARG and call(N=0) == ARG
    assert call(x=None) == ARG and call(y=None) == ARG and call(coords=None) == ARG and call(r=None) == ARG
    assert call(x=x + 8) == ARG and call(y=y + 2) == ARG
    assert call(y=x + 256) == ARG                        # overlaps without being the same
    assert call(B=1 << 16, N=1 << 15) == SHAPE
    assert call(r=wb.wave_rotary_plan(128, 1e4), d=64) == SHAPE
    for change, status in ((dict(rot_dim=8), SHAPE), (dict(rot_dim=40), SHAPE), (dict(n_axes=0), ARG), (dict(n_axes=5), ARG),
                           (dict(pairing=7), ARG)):
        bad = wb.wave_rotary_plan(64, 1e4)
        for k, v in change.items():
            setattr(bad, k, v)
        assert call(r=bad) == status, change
    bad = wb.wave_rotary_plan(64, 1e4)
    bad.axis[31] = 1
    assert call(r=bad) == ARG
    bad = wb.wave_rotary_plan(64, 1e4)
    bad.inv_freq[3] = math.nan
    assert call(r=bad) == ARG


def test_append_refuses():
    L = wb.lib()
    c, r = _cache(), wb.wave_rotary_plan(64, 1e4)
    kn, vn, q, qo, lo, to = (0x4000000 + i * 0x100000 for i in range(6))

    def call(c=c, kn=kn, vn=vn, q=q, Hq=4, n=3, counts=None, r=r, coords=FAKE, qo=qo, lo=lo, to=to):
        return L.wave_cache_append(ctypes.byref(c) if c is not None else None, kn, vn, q, Hq, n, counts,
                                   ctypes.byref(r) if r is not None else None, coords, qo, lo, to, None)

    for change, status in BAD_CACHES:
        assert call(c=_changed(c, **change)) == status, change
    assert call(c=None) == ARG and call(kn=None) == ARG and call(vn=None) == ARG and call(n=0) == ARG and call(n=-1) == ARG
    assert call(kn=kn + 2) == ARG and call(q=q + 4) == ARG and call(qo=None) == ARG and call(qo=qo + 8) == ARG
    assert call(Hq=0) == ARG and call(lo=None) == ARG and call(to=None) == ARG
    assert call(n=(1 << 30) + 1) == SHAPE
    # no rotary plan: nothing to do for q, nothing to read coordinates for
    assert call(r=None, q=None) == ARG and call(r=None, coords=None) == ARG
    # positions, and text coordinates, need the token numbers
    none = _changed(c, tokens=0)
    assert call(c=none, to=None) == ARG
    none = _changed(none, positions=0)
    assert call(c=none) == ARG and call(c=none, to=None, coords=None) == ARG
    # overlaps
    assert call(qo=q + 256) == ARG and call(qo=c.k) == ARG and call(qo=c.v) == ARG and call(qo=kn) == ARG
    assert call(kn=c.k) == ARG and call(vn=c.v + 4096) == ARG and call(vn=c.k) == ARG and call(q=c.k) == ARG
    assert call(lo=c.lengths + 4) == ARG and call(lo=c.tokens) == ARG and call(to=c.lengths) == ARG and call(to=lo) == ARG
    assert call(counts=lo) == ARG


def test_coordinates_apart_from_what_is_written():
    L = wb.lib()
    c, one, two = _cache(), wb.wave_rotary_plan(64, 1e4), wb.wave_rotary_plan(64, 1e4, [16, 16])
    kn, vn, q, qo, lo, to = (0x4000000 + i * 0x100000 for i in range(6))

    def append(coords, r=one, n=1, lo=lo, to=to):
        return L.wave_cache_append(ctypes.byref(c), kn, vn, q, 4, n, None, ctypes.byref(r), coords, qo, lo, to, None)

    assert append(lo) == ARG and append(to) == ARG and append(qo) == ARG and append(qo + 2 * 4 * 128 * 2 - 4) == ARG
    assert append(c.lengths, n=3, lo=c.lengths) == ARG and append(c.lengths, r=two, lo=c.lengths) == ARG
    assert append(c.tokens + 4, to=c.tokens) == ARG and append(c.tokens, r=two, to=c.tokens) == ARG
    x, y = 0x100000, 0x900000
    apply = lambda coords, B=2, H=3, N=5, y=y: L.wave_rotary_apply(x, coords, ctypes.byref(two), 1, B, H, N, 64, y, None)
    assert apply(y) == ARG and apply(y - 4 * 2 * 2 * 5 + 4) == ARG and apply(y + 2 * 3 * 5 * 64 * 2 - 4) == ARG
    assert apply(FAKE, B=1, H=(1 << 30) + 1, N=1) == SHAPE and apply(FAKE, B=1, H=1, N=(1 << 30) + 1) == SHAPE


def test_append_refuses_to_write_what_it_reads():
    """Every array that the call reads or writes, in each of the cache's arrays (which workgroups write in no order), and
    what else it writes in one another; the call that all of them are changed from is not refused."""
    L = wb.lib()
    c, r = _cache(), wb.wave_rotary_plan(64, 1e4)
    kn, vn, q, qo, lo, to, xy, cnt = (0x4000000 + i * 0x100000 for i in range(8))

    def call(kn=kn, vn=vn, q=q, coords=xy, counts=cnt, qo=qo, lo=lo, to=to):
        return L.wave_cache_append(ctypes.byref(c), kn, vn, q, 4, 3, counts, ctypes.byref(r), coords, qo, lo, to, None)

    if not torch.cuda.is_available():     # made-up addresses: the launch has to fail
        assert call() == 6 and call(counts=None, coords=None) == 6 and call(qo=q) == 6 and call(lo=c.lengths, to=c.tokens) == 6
        assert call(counts=c.lengths) == 6 and call(coords=cnt) == 6
    ends = {"k": 2 * 2 * 64 * 128 * 2, "v": 2 * 2 * 64 * 128 * 2, "positions": 2 * 2 * 64 * 4, "weights": 2 * 2 * 64 * 4}
    for name, size in ends.items():
        at = getattr(c, name)
        for p in (at, at + size - 16):
            for arg in ("kn", "vn", "q", "coords", "counts", "qo", "lo", "to"):
                assert call(**{arg: p}) == ARG, (name, arg)
    assert call(counts=qo) == ARG and call(counts=qo + 2 * 4 * 3 * 128 * 2 - 4) == ARG and call(counts=to) == ARG
    assert call(coords=qo) == ARG and call(coords=lo) == ARG and call(coords=c.tokens, to=c.tokens) == ARG


def test_attention_refuses():
    L = wb.lib()
    c = _cache()
    need = L.wave_cache_attention_workspace(ctypes.byref(c), 4, 100, 1)
    assert need > L.wave_cache_attention_workspace(ctypes.byref(c), 4, 100, 0) > 0 and need % 256 == 0
    assert need > L.wave_cache_attention_workspace(ctypes.byref(c), 4, 0, 1)
    for Hq, P in ((3, 0), (1, 0), (18, 0), (4, -1), (4, (1 << 30) + 1)):
        assert L.wave_cache_attention_workspace(ctypes.byref(c), Hq, P, 0) == 0, (Hq, P)
    q, pk, pv, wo_, out, lse, ws = (0x4000000 + i * 0x100000 for i in range(7))

    def call(c=c, q=q, Hq=4, pk=pk, pv=pv, P=100, decay=1.0, wout=wo_, out=out, lse=lse, ws=ws, nbytes=need):
        return L.wave_cache_attention_decode(q, Hq, ctypes.byref(c) if c is not None else None, pk, pv, P, decay, wout, out,
                                             lse, ws, nbytes, None)

    for change, status in BAD_CACHES:
        assert call(c=_changed(c, **change)) == status, change
    assert call(c=None) == ARG and call(q=None) == ARG and call(q=q + 8) == ARG and call(out=None) == ARG and call(lse=None) == ARG
    assert call(Hq=3) == SHAPE and call(Hq=18) == SHAPE and call(Hq=1) == SHAPE
    assert call(P=-1) == ARG and call(pk=None) == ARG and call(pv=None) == ARG and call(pk=pk + 8) == ARG
    for decay in (-0.5, 1.5, math.nan, math.inf):
        assert call(decay=decay) == ARG
    assert call(c=_changed(c, weights=0)) == ARG        # nothing to decay
    assert call(wout=c.weights + 16) == ARG
    assert call(ws=None) == WORKSPACE and call(ws=ws + 64) == WORKSPACE and call(nbytes=need - 1) == WORKSPACE


@pytest.mark.parametrize("B,Hkv,G", [(1, 8, 4), (64, 4, 7), (3, 1, 1), (200, 2, 8)])
def test_attention_workspace_of_a_larger_cache_is_enough(B, Hkv, G):
    def need(cap, P):
        return wb.lib().wave_cache_attention_workspace(ctypes.byref(_cache(B=B, Hkv=Hkv, capacity=cap)), Hkv * G, P, 1)

    by_rows = [need(cap, 500) for cap in (1, 2, 127, 128, 129, 1000, 5000, 70000)]
    assert all(a <= b for a, b in zip(by_rows, by_rows[1:])) and by_rows[0] > 0


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,Hkv,G,cap", [(8, 8, 4, 2048), (3, 2, 4, 256), (1, 1, 1, 1), (64, 4, 7, 4352), (200, 2, 8, 100), (60, 8, 1, 700),
                                         (13, 7, 5, 90000), (1000, 8, 8, 200)])
def test_attention_workspace_of_a_longer_prefix_is_enough(dtype, d, B, Hkv, G, cap):
    c = _cache(dtype=dtype, B=B, Hkv=Hkv, d=d, capacity=cap)
    lengths = sorted(set(list(range(0, 1100, 17)) + [128 * i + j for i in range(1, 700, 3) for j in (-1, 0, 1)]
                         + [32766, 32767, 32768, 32893, 65536, 65537, 100000, 1 << 20, 1 << 30]))
    for accumulate in (0, 1):
        need = [wb.lib().wave_cache_attention_workspace(ctypes.byref(c), Hkv * G, P, accumulate) for P in lengths]
        assert all(a <= b for a, b in zip(need, need[1:])) and need[0] > 0, (accumulate, [p for p, a, b in zip(lengths, need, need[1:]) if a > b])


def test_evict_refuses():
    L = wb.lib()
    c, d = _cache(), _cache(base=0x4000000)
    need = L.wave_cache_evict_workspace(ctypes.byref(c), 32)
    assert need > 0 and need % 256 == 0 and L.wave_cache_evict_workspace(ctypes.byref(c), -1) == 0
    ws = 0x9000000
    call = lambda a=c, b=c, keep=32, sink=4, local=8, ws=ws, nbytes=need: L.wave_cache_evict(
        ctypes.byref(a) if a is not None else None, ctypes.byref(b) if b is not None else None, keep, sink, local, ws, nbytes, None)
    for change, status in BAD_CACHES:
        assert call(a=_changed(c, **change)) == status, change
        assert call(b=_changed(c, **change)) != 0, change
    for name in ("weights", "positions", "tokens"):
        assert call(a=_changed(c, **{name: 0})) == ARG and call(b=_changed(c, **{name: 0})) == ARG
    assert call(a=None) == ARG and call(b=None) == ARG
    assert call(keep=-1, sink=0, local=0) == ARG and call(sink=-1) == ARG and call(local=-1) == ARG and call(sink=25) == ARG
    assert call(keep=(1 << 31) - 1, sink=(1 << 31) - 1, local=1) == ARG
    assert call(b=_changed(d, Hkv=1)) == SHAPE and call(b=_changed(d, d=64)) == SHAPE and call(b=_changed(d, dtype=0)) == SHAPE
    assert call(b=_changed(d, capacity=31)) == SHAPE
    assert call(b=_changed(d, k=c.k)) == ARG             # k in place, v elsewhere
    assert call(b=_changed(c, k=d.k)) == ARG
    assert call(b=_changed(c, capacity=40)) == ARG       # one array at two strides
    assert call(b=_changed(d, k=c.k + 4096, v=d.v)) == ARG and call(b=_changed(d, v=c.k)) == ARG
    assert call(b=_changed(d, weights=c.weights + 4)) == ARG and call(b=_changed(d, lengths=c.tokens)) == ARG
    assert call(b=_changed(d, tokens=d.lengths)) == ARG and call(b=_changed(d, positions=d.weights)) == ARG
    assert call(ws=None) == WORKSPACE and call(ws=ws + 128) == WORKSPACE and call(nbytes=need - 1) == WORKSPACE


def test_binding_refuses_what_is_not_on_a_gpu():
    cache = wb.alloc_cache(torch.float32, 2, 1, 64, 8, device="cpu")
    x = torch.zeros(2, 1, 3, 64)
    coords = torch.zeros(1, 2, 3, dtype=torch.int32)
    rot = wb.wave_rotary_plan(64, 1e4)
    for call in (lambda: wb.wave_rotary_apply(x, coords, rot), lambda: wb.wave_cache_append(cache, x, x),
                 lambda: wb.wave_cache_attention_decode(x[:, :, 0], cache), lambda: wb.wave_cache_evict(cache, 4, 0, 0)):
        with pytest.raises((wb.WaveError, RuntimeError)):
            call()


def test_binding_refuses_shapes_and_types():
    cache = wb.alloc_cache(torch.float32, 2, 1, 64, 8, device="cpu")
    x = torch.zeros(2, 1, 3, 64)
    rot = wb.wave_rotary_plan(64, 1e4)
    for call, status in [
            (lambda: wb.wave_rotary_apply(x, torch.zeros(1, 2, 4, dtype=torch.int32), rot), SHAPE),
            (lambda: wb.wave_rotary_apply(x, torch.zeros(1, 2, 3), rot), DTYPE),
            (lambda: wb.wave_rotary_apply(x[0], torch.zeros(1, 2, 3, dtype=torch.int32), rot), SHAPE),
            (lambda: wb.wave_cache_append(cache, x[:1], x[:1]), SHAPE), (lambda: wb.wave_cache_append(cache, x, x[:, :, :2]), SHAPE),
            (lambda: wb.wave_cache_append(cache, x.bfloat16(), x.bfloat16()), DTYPE),
            (lambda: wb.wave_cache_append(cache, x, x, q=x[:, :, :1], rotary=rot), SHAPE),
            (lambda: wb.wave_cache_append(cache, x, x, coords=torch.zeros(1, 2, 3, dtype=torch.int32)), ARG),
            (lambda: wb.wave_cache_append(cache, x, x, counts=torch.zeros(2)), DTYPE),
            (lambda: wb.wave_cache_append(cache, x, x, counts=torch.zeros(3, dtype=torch.int32)), SHAPE),
            (lambda: wb.wave_cache_append(cache, x, x, lengths_out=torch.zeros(2)), DTYPE),
            (lambda: wb.wave_cache_attention_decode(x[:, :, 0, :32], cache), SHAPE),
            (lambda: wb.wave_cache_attention_decode(x[:, :, 0].bfloat16(), cache), DTYPE),
            (lambda: wb.wave_cache_attention_decode(x[:, :, 0], cache, x[0]), ARG),
            (lambda: wb.wave_cache_attention_decode(x[:, :, 0], cache, x[:, 0], x[:, 0]), SHAPE),
            (lambda: wb.wave_cache_attention_decode(x[:, :, 0], cache, weights_out=torch.zeros(2, 1, 9)), SHAPE),
            (lambda: wb.cache_from_tensors(x, x.transpose(1, 2), None, None, torch.zeros(2, dtype=torch.int32), None), SHAPE),
            (lambda: wb.cache_from_tensors(x[..., ::2], x[..., ::2], None, None, torch.zeros(2, dtype=torch.int32), None), ARG),
            (lambda: wb.cache_from_tensors(x, x, None, None, torch.zeros(2), None), DTYPE),
            (lambda: wb.cache_from_tensors(x.half(), x.half(), None, None, torch.zeros(2, dtype=torch.int32), None), DTYPE)]:
        with pytest.raises(wb.WaveError) as e:
            call()
        assert e.value.status == status


@pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: the launch has to fail")
def test_documented_sizes_reach_the_launch():
    """Sizes up to the documented limits are not refused: without a GPU the launch is what fails."""
    HIP = 6
    L = wb.lib()
    r = wb.wave_rotary_plan(64, 1e4)
    x, coords = 1 << 44, 1 << 40
    for B, H, N, d, dt in [(1 << 24, 1, 1, 64, 1), ((1 << 31) - 1, 1, 1, 64, 1), (1, 1, 1 << 30, 64, 1), (1, 1, 1 << 30, 128, 0),
                           (1, 1 << 30, 1, 64, 0), (2, 1, 1 << 29, 64, 0), ((1 << 24) - 1, 1, 1, 64, 1)]:
        assert L.wave_rotary_apply(x, coords, ctypes.byref(r), dt, B, H, N, d, x, None) == HIP, (B, H, N, d, dt)
    for B, n, Hkv, d, dt in [(1, 1 << 30, 1, 64, 1), (1, 1 << 30, 1, 128, 0), ((1 << 21) - 1, 1, 1, 64, 1), (2, (1 << 30) - 1, 1, 64, 1),
                             (1 << 18, 4096, 7, 64, 1)]:
        c = _cache(dtype=dt, B=B, Hkv=Hkv, d=d, capacity=8, base=1 << 30)
        assert L.wave_cache_append(ctypes.byref(c), x, x, None, 0, n, None, ctypes.byref(r), coords, None, c.lengths, c.tokens,
                                   None) == HIP, (B, n, Hkv, d, dt)
    c = _cache(B=1, Hkv=1, d=128, capacity=1 << 30, base=1 << 30)
    for n_keep, status in ((1 << 29, SHAPE), (1 << 28, SHAPE), ((1 << 28) - 16, SHAPE), ((1 << 28) - 17, HIP), (100, HIP), ((1 << 30) - 100, HIP)):
        ws = L.wave_cache_evict_workspace(ctypes.byref(c), n_keep)
        assert ws > 0 and L.wave_cache_evict(ctypes.byref(c), ctypes.byref(c), n_keep, 0, 0, 1 << 45, ws, None) == status, n_keep


def test_sizes_beyond_the_documented_limits():
    L = wb.lib()
    r = wb.wave_rotary_plan(64, 1e4)
    x, coords = 1 << 44, 1 << 40
    for B, H, N in [(1 << 30, 2, 1), (1 << 30, 1, 2), (1, (1 << 30) + 1, 1), (1, 1, (1 << 30) + 1)]:
        assert L.wave_rotary_apply(x, coords, ctypes.byref(r), 1, B, H, N, 64, x, None) == SHAPE, (B, H, N)
    c = _cache(B=2, Hkv=1, capacity=8, base=1 << 30)
    append = lambda n, Hq: L.wave_cache_append(ctypes.byref(c), x, x, x if Hq else None, Hq, n, None, ctypes.byref(r), coords,
                                               x if Hq else None, c.lengths, c.tokens, None)
    assert append(1 << 30, 0) == SHAPE and append((1 << 30) + 1, 0) == SHAPE and append(1, 1 << 23) == SHAPE
    for bad in (_cache(B=1 << 20, Hkv=2, capacity=8), _cache(B=1, Hkv=1, capacity=(1 << 30) + 1)):
        assert L.wave_cache_attention_workspace(ctypes.byref(bad), 2, 0, 0) == 0 and L.wave_cache_evict_workspace(ctypes.byref(bad), 4) == 0
    for B, cap, most in ((1 << 20, 1, True), ((1 << 20) - 1, 8 * 1024, True), (1 << 20, 8 * 1024, False), ((1 << 21) - 1, 1, False)):
        c = _cache(B=B, Hkv=1, capacity=cap)
        assert (L.wave_cache_attention_workspace(ctypes.byref(c), 8, 0, 0) > 0) == most, (B, cap)


# --------------------------------------------------------------------------- pins of the plain statement
def test_turn_by_hand_and_its_laws():
    axis, freq = [0, 1], [math.pi / 2, math.pi / 6]
    x = np.array([1.0, 2.0, 3.0, 4.0, 9.0])
    y = co.rotate(x, [1, 2], axis, freq, co.HALVES)     # (1, 3) a quarter, (2, 4) a sixth of a circle
    h = math.sqrt(3) / 2
    assert np.allclose(y, [-3, 2 * 0.5 - 4 * h, 1, 2 * h + 4 * 0.5, 9])
    y = co.rotate(x, [1, 2], axis, freq, co.NEIGHBOURS)
    assert np.allclose(y, [-2, 1, 3 * 0.5 - 4 * h, 3 * h + 4 * 0.5, 9])
    assert np.isclose(np.linalg.norm(y), np.linalg.norm(x))
    assert np.allclose(co.rotate(y, [-1, -2], axis, freq, co.NEIGHBOURS), x)
    assert np.allclose(co.rotate(co.rotate(x, [3, 5], axis, freq, 0), [4, -1], axis, freq, 0), co.rotate(x, [7, 4], axis, freq, 0))


def test_one_axis_is_the_synthetic_workloads_encoding():
    x = torch.randn(5, 64, generator=torch.Generator().manual_seed(3), dtype=torch.float64)
    at = torch.tensor([0, 1, 17, 4000, 1048576])
    want = synth.rope(x, at, 500000.0)
    axis, freq = co.pair_plan(64, 500000.0, [32], co.RUNS)
    for i in range(5):
        assert np.allclose(co.rotate(x[i].numpy(), [int(at[i])], axis, freq, co.HALVES), want[i].numpy(), atol=1e-9)


def test_attention_over_prefix_and_rows_is_full_attention():
    g = np.random.default_rng(5)
    q, K, V = g.standard_normal((2, 16)), g.standard_normal((9, 16)), g.standard_normal((9, 16))
    pk, pv = g.standard_normal((4, 16)), g.standard_normal((4, 16))
    old = g.random(9)
    out, lse, w = co.cache_attention(q, K, V, 6, pk, pv, old, 0.5)
    share = 0.0
    for i in range(2):
        o, l = wo.full_attention(q[i], np.concatenate([pk, K[:6]]), np.concatenate([pv, V[:6]]))
        assert np.allclose(out[i], o) and np.isclose(lse[i], l)
        zp = pk @ q[i] / 4.0
        share += 1.0 - np.exp(zp - l).sum()
    assert np.isclose((w - 0.5 * old[:6]).sum(), share)
    out, lse, w = co.cache_attention(q, K, V, 0, None, None, old, 1.0)
    assert not out.any() and np.all(lse == -np.inf) and w.size == 0


def test_eviction_by_hand():
    nan = math.nan
    #            sink      weights ...               newest
    positions = [0, 5, 2, 7, 1, 9]
    weights = [0.0, 3.0, 1.0, 1.0, 9.0, 0.0]
    assert co.evict(positions, weights, 6, 10, 4, 1, 1) == [0, 1, 4, 5]      # 2 and 3 leave, 4 and 5 close up
    assert co.evict(positions, weights, 6, 10, 4, 0, 0) == [4, 1, 2, 3]
    assert co.evict(positions, [1.0] * 6, 6, 10, 4, 0, 0) == [0, 1, 2, 3]    # equal: the lower rows stay
    assert co.evict(positions, [nan, -1.0, nan, -2.0, 0.0, nan], 6, 10, 4, 0, 0) == [0, 1, 4, 3]
    assert co.evict(positions, weights, 3, 10, 4, 0, 0) == [0, 1, 2]
    assert co.evict(positions, weights, 6, 10, 0, 0, 0) == []
