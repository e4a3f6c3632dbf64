"""Norms with rotary positions and the paged 8-bit cache, host side: what every entry point refuses before any launch, and the
pins of the plain statement that the GPU tests compare with.  No GPU needed."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from oracle import pages_oracle as po
from paper_2505_02922_amd import binding as wb

ARG, SHAPE, DTYPE, WORKSPACE, HIP = 1, 2, 3, 4, 6
FAKE = 1 << 30
OWN = ("k_tail", "v_tail", "table", "lengths", "references")


def _sizes(c):
    es = 2 if c.dtype == 1 else 4
    tail = c.B * c.Hkv * c.page * c.d * es
    codes = c.n_pages * c.Hkv * c.page * c.d
    return dict(k_codes=codes, v_codes=codes, k_scales=c.n_pages * c.Hkv * 4, v_scales=c.n_pages * c.Hkv * 4, k_tail=tail, v_tail=tail,
                table=c.B * c.max_pages * 4, lengths=c.B * 4, references=c.n_pages * 4)


def _pages(dtype=1, B=2, Hkv=2, d=128, page=64, n_pages=9, max_pages=5, base=FAKE):
    c = wb.wave_pages()
    c.dtype, c.B, c.Hkv, c.d, c.page, c.n_pages, c.max_pages = dtype, B, Hkv, d, page, n_pages, max_pages
    at = base
    for name, size in _sizes(c).items():
        setattr(c, name, at)
        at += (size + 8191) // 4096 * 4096
    return c


def _changed(c, **kw):
    n = type(c)()
    ctypes.memmove(ctypes.byref(n), ctypes.byref(c), ctypes.sizeof(c))
    for k, v in kw.items():
        setattr(n, k, v)
    return n


def _beside(c, base=FAKE + (1 << 29)):
    """Another state of the same pool."""
    o = _pages(c.dtype, c.B, c.Hkv, c.d, c.page, c.n_pages, c.max_pages, base)
    return _changed(c, **{name: getattr(o, name) for name in OWN})


def _dense(at, H, n, d=128):
    return wb.wave_rows(at, H * n * d, n * d, d)


BAD_PAGES = [(dict(dtype=2), DTYPE), (dict(B=0), ARG), (dict(Hkv=0), ARG), (dict(n_pages=0), ARG), (dict(max_pages=0), ARG),
             (dict(B=-1), ARG), (dict(d=96), SHAPE), (dict(page=16), SHAPE), (dict(page=48), SHAPE), (dict(page=256), SHAPE), (dict(page=0), SHAPE),
             (dict(B=1 << 20), SHAPE), (dict(n_pages=(1 << 28) + 1), SHAPE), (dict(max_pages=(1 << 24) + 1), SHAPE)]
BAD_BUFFERS = [(dict(k_codes=0), ARG), (dict(v_codes=0), ARG), (dict(k_scales=0), ARG), (dict(v_scales=0), ARG), (dict(k_tail=0), ARG),
               (dict(v_tail=0), ARG), (dict(table=0), ARG), (dict(lengths=0), ARG), (dict(k_codes=FAKE + 8), ARG), (dict(v_tail=FAKE + 4), ARG)]


def test_struct_layouts():
    assert ctypes.sizeof(wb.wave_pages) == 7 * 4 + 4 + 9 * 8
    assert ctypes.sizeof(wb.wave_rows) == 4 * 8 and ctypes.sizeof(wb.wave_head_norm) == 3 * 8


def test_norm_rotary_refuses():
    L = wb.lib()
    rot = wb.wave_rotary_plan(64, 1e4)
    q, k, qo, ko, xy, qw, kw = (0x4000000 + i * 0x100000 for i in range(7))
    norm = wb.wave_head_norm(qw, kw, 1e-6)
    B, N, d, Hq, Hk = 2, 5, 128, 4, 2
    Q, K = _dense(q, Hq, N), _dense(k, Hk, N)

    def call(Q=Q, Hq=Hq, K=K, Hk=Hk, norm=norm, rot=rot, xy=xy, dt=1, B=B, N=N, d=d, qo=qo, ko=ko):
        return L.wave_norm_rotary_apply(Q, Hq, K, Hk, norm, rot, xy, dt, B, N, d, qo, ko, None)

    if not torch.cuda.is_available():      # made-up addresses: the launch has to fail
        fused = wb.wave_rows(q, 8 * N * d, d, 8 * d)
        assert call() == HIP and call(Q=None, Hq=0, qo=None) == HIP and call(K=None, Hk=0, ko=None) == HIP and call(norm=None) == HIP
        assert call(rot=None, xy=None) == HIP and call(qo=q, ko=k) == HIP and call(Q=fused, K=_changed(fused, data=q + 4 * d * 2)) == HIP
        assert call(Q=wb.wave_rows(q, 0, 0, 0)) == HIP and call(norm=wb.wave_head_norm(None, kw, 0.0)) == HIP
        assert call(norm=wb.wave_head_norm(qw, qw, 0.0)) == HIP
    assert call(dt=2) == DTYPE and call(d=96) == SHAPE and call(B=0) == ARG and call(N=0) == ARG and call(Hq=0) == ARG and call(Hk=0) == ARG
    assert call(Q=None, K=None) == ARG and call(qo=None) == ARG and call(ko=None) == ARG and call(qo=qo + 8) == ARG and call(ko=ko + 2) == ARG
    assert call(xy=None) == ARG and call(rot=None) == ARG and call(rot=None, xy=None, norm=None) == ARG
    for eps in (-1.0, math.nan, math.inf):
        assert call(norm=wb.wave_head_norm(qw, kw, eps)) == ARG
    assert call(norm=wb.wave_head_norm(qw + 2, kw, 0.0)) == ARG and call(norm=wb.wave_head_norm(qw, kw + 8, 0.0)) == ARG
    for change in (dict(data=0), dict(data=q + 8), dict(stride_b=-128), dict(stride_h=-8), dict(stride_n=100), dict(stride_h=4)):
        assert call(Q=_changed(Q, **change)) == ARG, change
        assert call(K=_changed(K, **change)) == ARG, change
    assert call(Q=_changed(Q, stride_b=1 << 62)) == SHAPE
    assert call(rot=wb.wave_rotary_plan(128, 1e4), d=64) == SHAPE
    assert call(B=1 << 16, N=1 << 15) == SHAPE and call(N=(1 << 30) + 1, B=1) == SHAPE
    # what is written apart from everything else, to the last byte
    qb, kb = B * Hq * N * d * 2, B * Hk * N * d * 2
    assert call(qo=q + 256) == ARG and call(qo=k) == ARG and call(ko=q) == ARG and call(ko=qo + qb - 16) == ARG and call(qo=ko + kb - 16) == ARG
    assert call(xy=qo) == ARG and call(xy=ko + kb - 4) == ARG and call(qo=qw) == ARG and call(ko=kw - kb + 16) == ARG
    assert call(Q=_changed(Q, stride_n=2 * d), qo=q) == ARG          # in place only where the input is dense
    assert call(Q=wb.wave_rows(q, 0, 0, 0), qo=q) == ARG
    bad = wb.wave_rotary_plan(64, 1e4)
    bad.axis[3] = 2
    assert call(rot=bad) == ARG


def test_append_refuses():
    L = wb.lib()
    c, rot = _pages(), wb.wave_rotary_plan(64, 1e4)
    o = _beside(c)
    n, Hq, d = 3, 4, 128
    kn, vn, q, qo, xy, cnt, qw, kw, ws = ((1 << 32) + i * 0x100000 for i in range(9))
    norm = wb.wave_head_norm(qw, kw, 1e-6)
    need = L.wave_pages_append_workspace(c)
    assert need > 0 and need % 256 == 0

    def call(a=c, b=o, kn=_dense(kn, 2, n), vn=_dense(vn, 2, n), q=_dense(q, Hq, n), Hq=Hq, n=n, cnt=cnt, norm=norm, rot=rot, xy=xy, qo=qo,
             ws=ws, nbytes=need):
        return L.wave_pages_append(a, b, kn, vn, q, Hq, n, cnt, norm, rot, xy, qo, ws, nbytes, None)

    if not torch.cuda.is_available():
        assert call() == HIP and call(b=c) == HIP and call(q=None, qo=None) == HIP and call(cnt=None, xy=None) == HIP and call(norm=None) == HIP
        assert call(rot=None, xy=None) == HIP and call(qo=q) == HIP and call(rot=None, xy=None, norm=None, q=None) == HIP
    for change, status in BAD_PAGES + BAD_BUFFERS + [(dict(references=0), ARG)]:
        assert call(a=_changed(c, **change)) == status, change
        assert call(b=_changed(o, **change)) != 0, change
    assert call(a=None) == ARG and call(b=None) == ARG and call(kn=None) == ARG and call(vn=None) == ARG
    assert call(n=0) == ARG and call(n=-1) == ARG and call(Hq=0) == ARG and call(qo=None) == ARG and call(qo=qo + 8) == ARG
    assert call(rot=None) == ARG and call(rot=None, xy=None, norm=wb.wave_head_norm(None, kw, 0.0)) == ARG   # nothing to do for q
    assert call(n=(1 << 30) + 1) == SHAPE and call(n=1 << 30) == SHAPE and call(Hq=1 << 23) == SHAPE
    for change in (dict(data=kn + 8), dict(stride_b=-128), dict(stride_h=4), dict(data=0)):
        assert call(kn=_changed(_dense(kn, 2, n), **change)) == ARG and call(vn=_changed(_dense(vn, 2, n), **change)) == ARG, change
        assert call(q=_changed(_dense(q, 4, n), **change)) == ARG, change
    assert call(norm=wb.wave_head_norm(qw, kw, -1.0)) == ARG and call(norm=wb.wave_head_norm(qw + 4, kw, 0.0)) == ARG
    assert call(ws=None) == WORKSPACE and call(ws=ws + 64) == WORKSPACE and call(nbytes=need - 1) == WORKSPACE
    # one pool, one shape; every list its own or none
    assert call(b=_changed(o, B=1)) == SHAPE and call(b=_changed(o, max_pages=4)) == SHAPE and call(b=_changed(o, n_pages=8)) == SHAPE
    assert call(b=_changed(o, page=32)) == SHAPE and call(b=_changed(o, Hkv=1)) == SHAPE and call(b=_changed(o, dtype=0)) == SHAPE
    for name in ("k_codes", "v_codes", "k_scales", "v_scales"):
        assert call(b=_changed(o, **{name: getattr(o, name) + 4096})) == ARG, name
    for name in OWN:
        assert call(b=_changed(o, **{name: getattr(c, name)})) == ARG, name
        assert call(b=_changed(c, **{name: getattr(o, name)})) == ARG, name
    # what is written (the pool, the new state, q_out, the workspace) apart from all that is read, to the last byte
    size = _sizes(c)
    size["qo"], size["ws"] = 2 * Hq * n * d * 2, need
    kb, at = 2 * 2 * n * d * 2, {name: getattr(o, name) for name in size if name not in ("qo", "ws")}
    at["qo"], at["ws"] = qo, ws
    for name, end in size.items():
        for p in (at[name], (at[name] + end - 1) & ~15):
            assert call(kn=_dense(p, 2, n)) == ARG and call(vn=_dense(p, 2, n)) == ARG and call(cnt=p) == ARG and call(xy=p) == ARG, name
            assert call(norm=wb.wave_head_norm(p, kw, 0.0)) == ARG and call(norm=wb.wave_head_norm(qw, p, 0.0)) == ARG, name
            if name != "qo":
                assert call(q=_dense(p, Hq, n)) == ARG and call(qo=p) == ARG, name
        assert call(kn=_dense(at[name] - kb + 16, 2, n)) == ARG, name
    for name in OWN:                                                    # (and, apart, what the old state is)
        assert call(qo=getattr(c, name)) == ARG and call(b=_changed(o, table=getattr(c, name) - 16)) == ARG, name
        assert call(b=c, cnt=getattr(c, name)) == ARG and call(b=c, xy=getattr(c, name)) == ARG, name
    assert call(b=_changed(o, references=o.lengths)) == ARG and call(b=_changed(o, k_tail=o.v_tail + 256)) == ARG
    assert call(qo=kn) == ARG and call(qo=q + 256) == ARG and call(ws=c.table & ~255) == ARG


def test_append_refuses_tokens_whose_numbers_pass_31_bits():
    """Without coordinates a token's position is its number: the last row that the table has room for, and n_new - 1 behind it (the
    queries of tokens that find no room are turned too)."""
    L = wb.lib()
    c, rot = _pages(B=1, Hkv=1, d=64, page=128, n_pages=1, max_pages=1 << 23), wb.wave_rotary_plan(64, 1e4)
    kn, q, qo, xy, ws = (i << 44 for i in range(1, 6))
    once = wb.wave_rows(kn, 0, 0, 0)
    most = (1 << 31) - (c.max_pages * c.page + c.page - 1)

    def call(n, rot=rot, xy=None, q=wb.wave_rows(q, 0, 0, 0), qo=qo):
        return L.wave_pages_append(c, c, once, once, q, 1, n, None, wb.wave_head_norm(kn + (1 << 40), None, 0.0), rot, xy, qo, ws, 1 << 20, None)

    assert most < 1 << 30
    for n in (most + 1, 1 << 30):
        assert call(n) == SHAPE
    if not torch.cuda.is_available():      # made-up addresses: the launch has to fail
        assert call(most) == HIP and call(1 << 30, xy=xy) == HIP and call(1 << 30, rot=None) == HIP and call(1 << 30, q=None, qo=None) == HIP


def test_read_refuses():
    L = wb.lib()
    c = _pages()
    k, v, first, n = 1 << 32, (1 << 32) + (1 << 24), (1 << 32) + (1 << 25), 7
    call = lambda c=c, first=first, n=n, k=k, v=v: L.wave_pages_read(c, first, n, k, v, None)
    if not torch.cuda.is_available():
        assert call() == HIP and call(first=None) == HIP and call(k=None) == HIP and call(v=None) == HIP and call(c=_changed(c, references=0)) == HIP
    for change, status in BAD_PAGES + BAD_BUFFERS:
        assert call(c=_changed(c, **change)) == status, change
    assert call(c=None) == ARG and call(n=0) == ARG and call(n=-3) == ARG and call(k=None, v=None) == ARG and call(k=k + 8) == ARG and call(v=v + 4) == ARG
    assert call(n=(1 << 30) + 1) == SHAPE and call(c=_changed(c, B=16), n=1 << 30) == SHAPE
    size = _sizes(c)
    size.pop("references")
    for name, end in size.items():
        for p in (getattr(c, name), (getattr(c, name) + end - 1) & ~15):
            assert call(k=p) == ARG and call(v=p) == ARG, name
    assert call(k=v) == ARG and call(v=k + 2 * 2 * 7 * 128 * 2 - 16) == ARG and call(first=k) == ARG and call(first=v) == ARG


def test_attention_refuses():
    L = wb.lib()
    c = _pages()
    q, out, lse, ws = ((1 << 32) + i * 0x1000000 for i in range(4))
    need = L.wave_pages_attention_workspace(c, 4)
    assert need > 0 and need % 256 == 0
    for Hq in (0, 1, 3, 18, -2):
        assert L.wave_pages_attention_workspace(c, Hq) == 0

    def call(c=c, q=q, Hq=4, out=out, lse=lse, ws=ws, nbytes=need):
        return L.wave_pages_attention_decode(q, Hq, c, out, lse, ws, nbytes, None)

    if not torch.cuda.is_available():
        assert call() == HIP and call(c=_changed(c, references=0)) == HIP and call(out=out + 4) == HIP
    for change, status in BAD_PAGES + BAD_BUFFERS:
        assert call(c=_changed(c, **change)) == status, change
    assert call(c=None) == ARG and call(q=None) == ARG and call(q=q + 8) == ARG and call(out=None) == ARG and call(lse=None) == ARG
    assert call(out=out + 2) == ARG and call(lse=lse + 1) == ARG
    assert call(Hq=3) == SHAPE and call(Hq=18) == SHAPE and call(Hq=1) == SHAPE
    assert call(ws=None) == WORKSPACE and call(ws=ws + 64) == WORKSPACE and call(nbytes=need - 1) == WORKSPACE
    size = _sizes(c)
    size.pop("references")
    for name, end in size.items():
        for p in (getattr(c, name), getattr(c, name) + end - 4):
            assert call(out=p) == ARG and call(lse=p) == ARG, name
    assert call(out=q) == ARG and call(lse=q + 16) == ARG and call(lse=out) == ARG and call(out=ws) == ARG and call(q=ws) == ARG


@pytest.mark.parametrize("B,Hkv,G", [(1, 8, 4), (64, 4, 7), (3, 1, 1), (200, 2, 8)])
def test_attention_workspace_of_a_longer_table_is_enough(B, Hkv, G):
    need = [wb.lib().wave_pages_attention_workspace(_pages(B=B, Hkv=Hkv, page=page, max_pages=most), Hkv * G)
            for most, page in ((1, 32), (1, 64), (1, 128), (2, 128), (5, 64), (16, 128), (70, 32), (1000, 64), (8000, 64))]
    assert all(a <= b for a, b in zip(need, need[1:])) and need[0] > 0


def test_reorder_refuses():
    L = wb.lib()
    c = _pages()
    o = _beside(c)
    parent = 1 << 32
    call = lambda a=c, b=o, parent=parent: L.wave_pages_reorder(a, b, parent, None)
    if not torch.cuda.is_available():
        assert call() == HIP and call(b=c) == HIP and call(b=_changed(o, B=1)) == HIP
    for change, status in BAD_PAGES + BAD_BUFFERS + [(dict(references=0), ARG)]:
        assert call(a=_changed(c, **change)) == status, change
        assert call(b=_changed(o, **change)) != 0, change
    assert call(a=None) == ARG and call(b=None) == ARG and call(parent=None) == ARG
    assert call(b=_changed(c, B=1)) == SHAPE and call(b=_changed(o, max_pages=6)) == SHAPE and call(b=_changed(o, n_pages=8)) == SHAPE
    for name in ("k_codes", "v_codes", "k_scales", "v_scales"):
        assert call(b=_changed(o, **{name: getattr(o, name) + 4096})) == ARG, name
    for name in OWN:
        assert call(b=_changed(o, **{name: getattr(c, name)})) == ARG and call(b=_changed(c, **{name: getattr(o, name)})) == ARG, name
        for x, y in ((c, o), (c, c)):
            assert call(a=x, b=y, parent=getattr(y, name)) == ARG and call(a=x, b=y, parent=getattr(y, name) + _sizes(c)[name] - 4) == ARG, name
    assert call(b=_changed(o, lengths=c.lengths + 4)) == ARG and call(b=_changed(o, table=o.references)) == ARG


def test_binding_refuses():
    pages = wb.alloc_pages(torch.float32, 2, 1, 64, 32, 5, 3, device="cpu")
    x, w = torch.zeros(2, 1, 3, 64), torch.ones(64)
    xy = torch.zeros(1, 2, 3, dtype=torch.int32)
    rot = wb.wave_rotary_plan(64, 1e4)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    for call, status in [
            (lambda: wb.wave_norm_rotary_apply(None, None, w, w), SHAPE), (lambda: wb.wave_norm_rotary_apply(x[0], None, w), SHAPE),
            (lambda: wb.wave_norm_rotary_apply(x, x[:1], w), SHAPE), (lambda: wb.wave_norm_rotary_apply(x, x.bfloat16(), w), DTYPE),
            (lambda: wb.wave_norm_rotary_apply(x, x, w[:32]), SHAPE), (lambda: wb.wave_norm_rotary_apply(x, x, w.double()), DTYPE),
            (lambda: wb.wave_norm_rotary_apply(x, x, w, coords=xy), ARG), (lambda: wb.wave_norm_rotary_apply(x, x, w, coords=xy[:, :1], rotary=rot), SHAPE),
            (lambda: wb.wave_norm_rotary_apply(x, x, w, coords=xy.long(), rotary=rot), DTYPE),
            (lambda: wb.wave_norm_rotary_apply(x, x, w, q_out=x[:1]), SHAPE), (lambda: wb.wave_norm_rotary_apply(x, x, w, k_out=x.bfloat16()), DTYPE),
            (lambda: wb.wave_norm_rotary_apply(x, x, w, w), ARG),                                     # not on a GPU
            (lambda: wb.wave_pages_append(pages, x[:1], x[:1]), SHAPE), (lambda: wb.wave_pages_append(pages, x, x[:, :, :2]), SHAPE),
            (lambda: wb.wave_pages_append(pages, x.bfloat16(), x.bfloat16()), DTYPE), (lambda: wb.wave_pages_append(pages, x, x, q=x[:, :, :1], rotary=rot), SHAPE),
            (lambda: wb.wave_pages_append(pages, x, x, coords=xy), ARG), (lambda: wb.wave_pages_append(pages, x, x, counts=i32(3)), SHAPE),
            (lambda: wb.wave_pages_append(pages, x, x, counts=torch.zeros(2)), DTYPE), (lambda: wb.wave_pages_append(pages, x, x, k_weight=w[:3]), SHAPE),
            (lambda: wb.wave_pages_read(pages, -1), ARG), (lambda: wb.wave_pages_read(pages, 4, first=i32(3)), SHAPE),
            (lambda: wb.wave_pages_read(pages, 4, first=torch.zeros(2)), DTYPE), (lambda: wb.wave_pages_read(pages, 4, k_out=x), SHAPE),
            (lambda: wb.wave_pages_read(pages, 3), ARG),
            (lambda: wb.wave_pages_attention_decode(x[:, :, 0, :32], pages), SHAPE), (lambda: wb.wave_pages_attention_decode(x[:, :, 0].bfloat16(), pages), DTYPE),
            (lambda: wb.wave_pages_attention_decode(x[:, :, 0], pages, out=x), SHAPE),
            (lambda: wb.wave_pages_reorder(pages, i32(3)), SHAPE), (lambda: wb.wave_pages_reorder(pages, torch.zeros(2)), DTYPE),
            (lambda: wb.wave_pages_reorder(pages, i32(2)), ARG),
            (lambda: wb.pages_from_tensors(*[pages.t[n] for n in wb.PAGE_POOL], pages.k_tail, pages.v_tail.bfloat16(), pages.table, pages.lengths, pages.references), DTYPE),
            (lambda: wb.pages_from_tensors(*[pages.t[n] for n in wb.PAGE_POOL], pages.k_tail, pages.v_tail, pages.table.t().contiguous(), pages.lengths, pages.references), SHAPE),
            (lambda: wb.alloc_pages(torch.float16, 2, 1, 64, 32, 5, 3, device="cpu"), DTYPE)]:
        with pytest.raises(wb.WaveError) as e:
            call()
        assert e.value.status == status


# --------------------------------------------------------------------------- pins of the plain statement
def test_norm_by_hand():
    x = np.array([3.0, -4.0, 0.0, 0.0])
    assert np.allclose(po.norm(x, np.array([1.0, 2.0, 5.0, 5.0]), 0.0), [1.2, -3.2, 0, 0])          # root mean square 2.5
    assert np.allclose(po.norm(x, np.ones(4), 6.25 * 3), x / 5)
    assert np.array_equal(po.norm(x, None, 1.0), x) and not po.norm(np.zeros(4), np.ones(4), 1e-6).any()
    assert np.allclose(po.norm_rotate(x, np.ones(4), 0.0, [1], [0, 0], [math.pi / 2, 0.0], co.NEIGHBOURS), [1.6, 1.2, 0, 0])


def test_page_by_hand_and_its_bound():
    codes, scale = po.page_codes(np.array([[127.0, -63.5, 0.49], [0.5, 1.5, -126.6]]))
    assert codes.tolist() == [[127, -64, 0], [0, 2, -127]] and scale == 1.0                          # ties to even
    assert po.page_codes(np.zeros((2, 3)))[1] == 0 and not po.page_codes(np.full((2, 3), 2.0 ** -101))[0].any()
    assert po.page_codes(np.full((2, 3), 2.0 ** -100))[0].all()
    for bad in (math.nan, math.inf, -math.inf):
        codes, scale = po.page_codes(np.array([[1.0, bad]]))
        assert not codes.any() and math.isnan(scale)
    g = np.random.default_rng(1)
    for size in (1e-25, 1.0, 3e38):
        x = (g.standard_normal((32, 64)).clip(-3, 3) / 3.1 * size).astype(np.float32)
        codes, scale = po.page_codes(x)
        # half a code, and 2^-24 relative for each of: 1 / max, its products with 127 and x, scale, at up to 127 codes; a max above
        # 2^126 has a subnormal reciprocal, off by up to 2^-150 of at least 2^-128: 2^-22
        assert np.abs(codes * np.float64(scale) - x).max() <= scale * (0.5 + 127 * (4 * 2.0 ** -24 + (2.0 ** -22 if size > 2.0 ** 125 else 0)))
        assert np.abs(codes).max() == 127


def test_appends_in_any_pieces_give_the_same_pages():
    g = np.random.default_rng(2)
    k, v = g.standard_normal((2, 2, 21, 4)), g.standard_normal((2, 2, 21, 4))
    whole, parts = po.Paged(2, 4, 20, 9), po.Paged(2, 4, 20, 9)
    whole.append(k, v)
    for n0, n1 in ((0, 1), (1, 3), (3, 11), (11, 12), (12, 21)):
        parts.append(k[:, :, n0:n1], v[:, :, n0:n1])
    assert [whole.length(b) for b in (0, 1)] == [21, 21] == [parts.length(b) for b in (0, 1)]
    assert whole.pages == [[0, 1, 2, 3, 4], [5, 6, 7, 8, 9]] and parts.pages != whole.pages and sorted(sum(parts.pages, [])) == list(range(10))
    for b in (0, 1):
        for h in (0, 1):
            assert np.array_equal(whole.rows(b, h)[0], parts.rows(b, h)[0]) and np.array_equal(whole.rows(b, h)[1], parts.rows(b, h)[1])
            assert np.array_equal(whole.rows(b, h)[0][20:], k[b, h, 20:])


def test_pool_and_table_that_are_full():
    g = np.random.default_rng(3)
    x = g.standard_normal((3, 1, 30, 4))
    c = po.Paged(3, 4, 5, 3)
    c.append(x, x, [30, 7, 30])
    assert c.pages == [[0, 1, 2], [3], [4]] and [c.length(b) for b in range(3)] == [15, 7, 7]        # a table's row, then the pool
    c = c.reorder([-1, 1, 2])
    assert c.references == [0, 0, 0, 1, 1]
    c.append(x, x, [0, 1, 9])
    assert c.pages == [[], [3, 0], [4, 1, 2]] and [c.length(b) for b in range(3)] == [0, 8, 15]


def test_references_are_the_tables_entries():
    g = np.random.default_rng(4)
    c = po.Paged(4, 4, 64, 9)
    for step in range(12):
        n = int(g.integers(1, 9))
        c.append(g.standard_normal((len(c.pages), 1, n, 4)), g.standard_normal((len(c.pages), 1, n, 4)))
        c = c.reorder(g.integers(-1, len(c.pages), int(g.integers(1, 6))).tolist())
        held = sum(c.pages, [])
        assert c.references == [held.count(p) for p in range(64)]
