"""Rotary positions and the plain cache on the GPU against the plain fp64 statement, through the C ABI.

Tolerances count roundings (u = 2^-24 for fp32, half a step):
  rotary   sine and cosine are off by less than 4 u (the angle in turns is rounded once, pi u, the functions by about one
           step), the two products and their sum by 3 u more, of the pair's length: 8 u of it; then half a step of the type
  scores   a sum of d products in fp32: (d + 2) u of the sum of the products' magnitudes (delta below)
  weights  of a row: the exponential of that, 2 delta + 8 u
  output   sum of p |v| times: 2 delta, 2^-17 for a weight in two bf16 numbers (the nearest, at most half a step of 2^-7 off
           in 1 .. 2, and the nearest to that rest, at most half a step of 2^-16 off; bf16 and long shared prefixes only),
           n u for the sums of n terms, 16 u for the joining; and, as the errors of different rows have no sign in common,
           1e-5 of the norm
"""
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2505_02922_amd import binding as wb

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def _gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def _same_bits(a, b):
    v = torch.int16 if a.dtype == torch.bfloat16 else torch.int32
    return torch.equal(a.contiguous().view(v), b.contiguous().view(v))


# --------------------------------------------------------------------------- rotary
def _turned(x, coords, plan, pairing, base):
    """x [B, H, N, d] double, coords [axes, B, N] -> the turned rows and the length of every channel's pair, in numpy."""
    rot, sections, order = plan
    axis, freq = co.pair_plan(rot, base, sections, order)
    y, size = x.copy(), np.zeros_like(x)
    for i, (a, f) in enumerate(zip(axis, freq)):
        p, q = (i, i + rot // 2) if pairing == co.HALVES else (2 * i, 2 * i + 1)
        angle = coords[a].astype(np.float64)[:, None] * f
        c, s = np.cos(angle), np.sin(angle)
        y[..., p], y[..., q] = x[..., p] * c - x[..., q] * s, x[..., p] * s + x[..., q] * c
        size[..., p] = size[..., q] = np.hypot(x[..., p], x[..., q])
    return y, size


def test_vectorised_turn_is_the_plain_one():
    x = np.random.default_rng(1).standard_normal((2, 3, 4, 64))
    coords = np.random.default_rng(2).integers(0, 99, (2, 2, 4))
    y, _ = _turned(x, coords, (48, [10, 14], co.TURNS), co.NEIGHBOURS, 1e4)
    axis, freq = co.pair_plan(48, 1e4, [10, 14], co.TURNS)
    for b in range(2):
        for h in range(3):
            for n in range(4):
                assert np.allclose(y[b, h, n], co.rotate(x[b, h, n], coords[:, b, n], axis, freq, co.NEIGHBOURS))


def _near_turned(got, x, coords, plan, pairing, base, dtype, tag):
    want, size = _turned(x.double().numpy(), coords.numpy(), plan, pairing, base)
    # 2^-51 of the largest angle: fp64 angles on both sides
    far = float(np.abs(coords.numpy().astype(np.float64)).max()) * 2.0 ** -51
    bar = (8 * U + far) * size * (1 + HALF_STEP[dtype]) + np.where(size > 0, HALF_STEP[dtype] * np.abs(want), 0.0)
    err = np.abs(got.double().cpu().numpy() - want)
    assert np.all(err <= bar), (tag, float((err - bar).max()))


PLANS = [(128, 128, [64], 0, 0), (128, 128, [16, 24, 24], 1, 0), (128, 64, [16, 16], 2, 1), (64, 64, [32], 0, 1), (64, 48, [8, 9, 7], 0, 0),
         (64, 16, [1, 2, 3, 2], 1, 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,rot,sections,order,pairing", PLANS)
@pytest.mark.parametrize("B,H,N", [(1, 1, 1), (2, 3, 31), (1, 5, 33), (3, 40, 2), (1, 2, 300)])
def test_rotary(dtype, d, rot, sections, order, pairing, B, H, N):
    g = _gen(N)
    x = torch.randn(B, H, N, d, generator=g).to(TYPES[dtype])
    coords = torch.randint(0, 1 << 20, (len(sections), B, N), generator=g, dtype=torch.int32)
    coords[0, 0, 0] = -5
    r = wb.wave_rotary_plan(rot, 500000.0, sections, order, pairing)
    got = wb.wave_rotary_apply(x.cuda(), coords.cuda(), r)
    _near_turned(got, x, coords, (rot, sections, order), pairing, 500000.0, dtype, "apart")
    y = x.cuda()
    assert wb.wave_rotary_apply(y, coords.cuda(), r, out=y) is y       # in place
    assert _same_bits(y, got)
    assert _same_bits(got[..., rot:].cpu(), x[..., rot:])               # channels behind the rotated ones


def test_rotary_far_positions_and_strided_input():
    """Positions at the ends of int32, and a transposed tensor with strided coordinates."""
    g = _gen(7)
    x = torch.randn(2, 9, 4, 128, generator=g).transpose(1, 2)          # [B, H, N, d] = [2, 4, 9, 128]
    coords = torch.randint(-2 ** 31, 2 ** 31 - 1, (2, 9, 2), generator=g, dtype=torch.int64).to(torch.int32)
    coords[0, 0] = 2 ** 31 - 1
    coords[0, 1] = -2 ** 31
    coords = coords.permute(2, 0, 1)                                     # [axes, B, N]
    r = wb.wave_rotary_plan(128, 1e4, [40, 24])
    got = wb.wave_rotary_apply(x.cuda(), coords.cuda(), r)
    _near_turned(got, x, coords, (128, [40, 24], 0), 0, 1e4, "f32", "far")


def test_rotary_with_frequencies_of_its_own():
    x = torch.randn(1, 2, 5, 64, generator=_gen(8))
    coords = torch.arange(5, dtype=torch.int32)[None, None]
    r = wb.wave_rotary_plan(64, 1e4)
    for i in range(32):
        r.inv_freq[i] *= 0.125                                           # eight times the context
    got = wb.wave_rotary_apply(x.cuda(), (coords * 8).contiguous().cuda(), r)
    _near_turned(got, x, coords, (64, [32], 0), 0, 1e4, "f32", "scaled")


@pytest.mark.parametrize("d,rot,sections,order,pairing", PLANS)
def test_rotary_gradient(d, rot, sections, order, pairing):
    """The turn back (inv_freq negated) is the gradient: against differences of the formula, which is linear, in fp64."""
    g, base = _gen(9), 5e5
    B, H, N = 2, 3, 7
    x, dy = (torch.randn(B, H, N, d, generator=g) for _ in range(2))
    coords = torch.randint(0, 4096, (len(sections), B, N), generator=g, dtype=torch.int32)
    r = wb.wave_rotary_plan(rot, base, sections, order, pairing)
    for i in range(rot // 2):
        r.inv_freq[i] = -r.inv_freq[i]
    got = wb.wave_rotary_apply(dy.cuda(), coords.cuda(), r)
    plan = (rot, sections, order)
    _near_turned(got, dy, -coords, plan, pairing, base, "f32", "gradient")      # the formula's: the transposed turn
    loss = lambda x: float((_turned(x, coords.numpy(), plan, pairing, base)[0] * dy.double().numpy()).sum())
    _, size = _turned(dy.double().numpy(), coords.numpy(), plan, pairing, base)
    for b, h, n, c in ((0, 0, 0, 0), (1, 2, 6, rot - 1), (0, 1, 3, rot // 2), (1, 0, 5, d - 1), (0, 2, 1, 1)):
        step = np.zeros((B, H, N, d))
        step[b, h, n, c] = 1.0
        at = x.double().numpy()
        change = (loss(at + step) - loss(at - step)) / 2
        # 9 u of the pair's length as in _near_turned; the differences themselves are off by 2^-53 of some thousand terms
        assert abs(float(got[b, h, n, c]) - change) <= 9 * U * size[b, h, n, c] + 1e-11, (b, h, n, c)


@pytest.mark.parametrize("N", [1, 2])
def test_rotary_of_more_workgroups_than_a_launch_row(N):
    """Tokens flattened into the batch, and pairs of them: the same rows as one long sequence, which takes few workgroups."""
    B = (1 << 24) + 3
    x = torch.randn(B, 1, N, 64, device="cuda", dtype=torch.bfloat16)
    coords = torch.randint(0, 1 << 20, (1, B, N), device="cuda", dtype=torch.int32)
    r = wb.wave_rotary_plan(48, 1e4, None, 0, 1)
    want = wb.wave_rotary_apply(x.view(1, 1, B * N, 64), coords.view(1, 1, B * N), r)
    got = wb.wave_rotary_apply(x, coords, r)
    assert _same_bits(got.view(-1), want.view(-1))
    assert wb.wave_rotary_apply(x, coords, r, out=x) is x and _same_bits(x.view(-1), want.view(-1))


# --------------------------------------------------------------------------- append
def _filled_cache(dtype, B, Hkv, d, cap, lengths, seed):
    """A cache whose rows behind the lengths hold no numbers."""
    g = _gen(seed)
    k, v = torch.randn(B, Hkv, cap, d, generator=g), torch.randn(B, Hkv, cap, d, generator=g)
    w = torch.rand(B, Hkv, cap, generator=g)
    pos = torch.empty(B, Hkv, cap, dtype=torch.int32)
    for b, n in enumerate(lengths):
        n = min(max(n, 0), cap)
        k[b, :, n:], v[b, :, n:], w[b, :, n:] = math.nan, math.nan, math.nan
        for h in range(Hkv):
            pos[b, h] = torch.randperm(cap, generator=g).to(torch.int32)
            pos[b, h, :n] = torch.randperm(n, generator=g).to(torch.int32)
    cache = wb.cache_from_tensors(k.to(TYPES[dtype]).cuda(), v.to(TYPES[dtype]).cuda(), pos.cuda(), w.cuda(),
                                  torch.tensor(lengths, dtype=torch.int32).cuda(), torch.tensor([max(n, 0) for n in lengths], dtype=torch.int32).cuda())
    return cache


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,rot,sections,order,pairing", [PLANS[1], PLANS[4]])
@pytest.mark.parametrize("B,Hq,Hkv,n,lengths,counts", [
    (1, 4, 1, 1, [0], None), (3, 14, 2, 1, [5, 0, 39], None), (2, 6, 6, 33, [0, 7], None), (3, 8, 2, 17, [1, 30, 3], [17, 0, 4]),
    (2, 0, 2, 5, [38, 40], None), (4, 2, 1, 3, [-3, 99, 39, 0], [99, 3, 3, -1])])
def test_append(dtype, d, rot, sections, order, pairing, B, Hq, Hkv, n, lengths, counts):
    cap, g = 40, _gen(11)
    cache = _filled_cache(dtype, B, Hkv, d, cap, lengths, 5)
    before = {name: t.clone() for name, t in cache.t.items()}
    cast = lambda *s: torch.randn(*s, generator=g).to(TYPES[dtype])
    k, v, q = cast(B, Hkv, n, d), cast(B, Hkv, n, d), cast(B, Hq, n, d) if Hq else None
    coords = torch.randint(0, 5000, (len(sections), B, n), generator=g, dtype=torch.int32)
    r = wb.wave_rotary_plan(rot, 1e6, sections, order, pairing)
    c = None if counts is None else torch.tensor(counts, dtype=torch.int32).cuda()
    q_out = torch.full(q.shape, 7.0).to(TYPES[dtype]).cuda() if Hq else None
    got_q = wb.wave_cache_append(cache, k.cuda(), v.cuda(), q=q.cuda() if Hq else None, coords=coords.cuda(), rotary=r, counts=c, q_out=q_out)
    kt = wb.wave_rotary_apply(k.cuda(), coords.cuda(), r)
    qt = wb.wave_rotary_apply(q.cuda(), coords.cuda(), r) if Hq else None
    want = {name: t.clone() for name, t in before.items()}
    for b in range(B):
        length = min(max(lengths[b], 0), cap)
        given = n if counts is None else min(max(counts[b], 0), n)
        fit = min(given, cap - length)
        first = max(lengths[b], 0)
        want["k"][b, :, length:length + fit], want["v"][b, :, length:length + fit] = kt[b, :, :fit], v[b, :, :fit].cuda()
        want["positions"][b, :, length:length + fit] = torch.arange(first, first + fit, dtype=torch.int32).cuda()
        want["weights"][b, :, length:length + fit] = 0.0
        want["lengths"][b], want["tokens"][b] = length + fit, first + fit
        if Hq:
            assert _same_bits(got_q[b, :, :given], qt[b, :, :given])
            assert bool((got_q[b, :, given:] == 7.0).all())
    for name, t in want.items():
        assert _same_bits(cache.t[name], t), name


def test_append_forms_agree():
    """Numbers in place or apart, text coordinates given or not, q in place, no rotation, a cache without bookkeeping."""
    g = _gen(12)
    B, Hq, Hkv, n, d, cap = 3, 4, 2, 70, 64, 200
    lengths = [4, 100, 0]
    cast = lambda *s: torch.randn(*s, generator=g).cuda()
    k, v, q = cast(B, Hkv, n, d), cast(B, Hkv, n, d), cast(B, Hq, n, d)
    r = wb.wave_rotary_plan(64, 1e4, [20, 12])
    a, b = (_filled_cache("f32", B, Hkv, d, cap, lengths, 6) for _ in range(2))
    coords = (torch.tensor(lengths)[:, None] + torch.arange(n)).to(torch.int32).expand(2, B, n).cuda()
    qa = wb.wave_cache_append(a, k, v, q=q, coords=coords, rotary=r)
    lo, to = torch.full((B,), -1, dtype=torch.int32, device="cuda"), torch.full((B,), -1, dtype=torch.int32, device="cuda")
    qb = q.clone()
    assert wb.wave_cache_append(b, k, v, q=qb, rotary=r, q_out=qb, lengths_out=lo, tokens_out=to) is qb
    assert _same_bits(qa, qb) and _same_bits(a.k, b.k) and _same_bits(a.v, b.v) and _same_bits(a.positions, b.positions)
    assert torch.equal(lo, a.lengths) and torch.equal(to, a.tokens) and b.lengths.tolist() == lengths and b.tokens.tolist() == lengths
    assert lo.tolist() == [x + n for x in lengths]
    bare = wb.cache_from_tensors(torch.zeros_like(a.k), torch.zeros_like(a.v), None, None, torch.tensor(lengths, dtype=torch.int32).cuda(), None)
    assert wb.wave_cache_append(bare, k, v) is None
    for i, x in enumerate(lengths):
        assert _same_bits(bare.k[i, :, x:x + n], k[i]) and _same_bits(bare.v[i, :, x:x + n], v[i])
        assert not bare.k[i, :, :x].any() and not bare.k[i, :, x + n:].any()
    assert bare.lengths.tolist() == [x + n for x in lengths]


@pytest.mark.parametrize("Hq,Hkv", [(2, 1), (128, 16)])
@pytest.mark.parametrize("name", ["lengths", "tokens"])
def test_append_with_its_own_numbers_as_coordinates(name, Hq, Hkv):
    """One new token whose coordinate is the sequence's length, which the same call advances (one workgroup a sequence, and
    several)."""
    g, B, d = _gen(13), 3, 128
    a, b = (_filled_cache("f32", B, Hkv, d, 24, [3, 0, 17], 6) for _ in range(2))
    r = wb.wave_rotary_plan(d, 1e4)
    for _ in range(5):
        k, v, q = (torch.randn(B, h, 1, d, generator=g).cuda() for h in (Hkv, Hkv, Hq))
        qa = wb.wave_cache_append(a, k, v, q=q, rotary=r)
        qb = wb.wave_cache_append(b, k, v, q=q, rotary=r, coords=b.t[name].view(1, B, 1))
        assert _same_bits(qa, qb)
    for key, t in a.t.items():
        assert _same_bits(t, b.t[key]), key


def test_append_of_more_workgroups_than_a_launch_row():
    """Two million sequences with 129 tokens each, three workgroups a sequence, of which the first two tokens fit (33 GiB of new
    rows; keys and values are the same array)."""
    B, n, d = (1 << 21) - 1, 129, 64
    row = torch.randn(B, 1, 1, d, device="cuda", dtype=torch.bfloat16)
    new = row.expand(B, 1, n, d).contiguous()
    cache = wb.alloc_cache(torch.bfloat16, B, 1, d, 2)
    cache.tokens.copy_(torch.randint(0, 1 << 20, (B,), device="cuda", dtype=torch.int32))
    first = cache.tokens.clone()
    r = wb.wave_rotary_plan(d, 1e4)
    assert wb.wave_cache_append(cache, new, new, rotary=r) is None
    at = torch.stack([first, first + 1], 1)[None]
    want = wb.wave_rotary_apply(row.expand(B, 1, 2, d).contiguous(), at.contiguous(), r)
    assert _same_bits(cache.k, want) and _same_bits(cache.v, new[:, :, :2])
    assert bool((cache.lengths == 2).all()) and torch.equal(cache.tokens, first + 2) and torch.equal(cache.positions[:, 0], at[0])


# --------------------------------------------------------------------------- attention
def _check_attention(dtype, q, cache, lengths, pk, pv, decay, old, out, lse, w, tag=""):
    B, Hq, d = q.shape
    Hkv, cap = cache.Hkv, cache.capacity
    G, P = Hq // Hkv, 0 if pk is None else pk.shape[1]
    two_numbers = dtype == "bf16" and P >= 32768 and B * G > 64
    qn, K, V = q.double().cpu().numpy(), cache.k.double().cpu().numpy(), cache.v.double().cpu().numpy()
    pkn, pvn = (None, None) if pk is None else (pk.double().cpu().numpy(), pv.double().cpu().numpy())
    out, lse, oldn = out.double().cpu().numpy(), lse.double().cpu().numpy(), old.double().cpu().numpy()
    err2, ref2 = 0.0, 0.0
    for b in range(B):
        n = min(max(lengths[b], 0), cap)
        for h in range(Hkv):
            qg = qn[b, h * G:(h + 1) * G]
            p_k, p_v = (None, None) if pk is None else (pkn[h], pvn[h])
            o, l, ww = co.cache_attention(qg, K[b, h], V[b, h], n, p_k, p_v, oldn[b, h], decay)
            rows = K[b, h, :n] if pk is None else np.concatenate([p_k, K[b, h, :n]])
            vals = V[b, h, :n] if pk is None else np.concatenate([p_v, V[b, h, :n]])
            share = np.zeros(n)
            for g in range(G):
                go, gl = out[b, h * G + g], lse[b, h * G + g]
                if P + n == 0:
                    assert not go.any() and gl == -math.inf, tag
                    continue
                mags = np.abs(rows) @ np.abs(qg[g]) / math.sqrt(d)
                p = np.exp(rows @ qg[g] / math.sqrt(d) - l[g])
                delta = (d + 2) * U * mags
                bar = p @ (np.abs(vals) * (2 * delta[:, None] + (2.0 ** -17 if two_numbers else 0.0) + (len(p) + 16) * U)) \
                    + np.abs(o[g]) * (p @ (2 * delta) + 8 * U)
                assert np.all(np.abs(go - o[g]) <= bar + 1e-30), (tag, b, h, g, float(np.abs(go - o[g]).max()))
                assert abs(gl - l[g]) <= p @ delta + (len(p) + 16) * U + 4 * U * abs(l[g]), (tag, b, h, g, gl, l[g])
                err2 += float(((go - o[g]) ** 2).sum())
                ref2 += float((p ** 2 @ vals ** 2).sum())
                share += p[P:] * (2 * delta[P:] + p @ (2 * delta) + (len(p) + 32) * U)
            if w is not None:
                got = w[b, h].double().cpu().numpy()
                assert np.all(np.abs(got[:n] - ww) <= share + 4 * U * np.abs(ww)), (tag, b, h, float(np.abs(got[:n] - ww).max()))
    assert err2 <= (1e-5 ** 2) * max(ref2, 1e-30) or ref2 == 0, (tag, math.sqrt(err2 / ref2))


def _inputs(dtype, B, Hq, Hkv, d, cap, lengths, P, seed, peak=2.0):
    cache = _filled_cache(dtype, B, Hkv, d, cap, lengths, seed)
    g = _gen(seed + 1)
    q = (peak * torch.randn(B, Hq, d, generator=g)).to(TYPES[dtype]).cuda()
    pk, pv = (torch.randn(Hkv, P, d, generator=g).to(TYPES[dtype]).cuda() for _ in range(2)) if P else (None, None)
    return cache, q, pk, pv


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,Hq,Hkv,cap,lengths,P", [
    (1, 1, 1, 1, [1], 0), (1, 8, 1, 40, [33], 1), (2, 6, 2, 200, [0, 129], 0), (3, 7, 1, 130, [128, 1, 130], 127),
    (5, 10, 2, 70, [0, 70, 31, 32, 64], 129), (2, 24, 3, 1500, [1500, 7], 515), (9, 8, 1, 20, [0] * 9, 300),
    (2, 2, 2, 50, [-4, 90], 0), (17, 16, 4, 33, list(range(17)), 65)])
def test_attention(dtype, d, B, Hq, Hkv, cap, lengths, P):
    cache, q, pk, pv = _inputs(dtype, B, Hq, Hkv, d, cap, lengths, P, B + P)
    old = cache.weights.clone()
    out, lse = wb.wave_cache_attention_decode(q, cache, pk, pv)
    _check_attention(dtype, q, cache, lengths, pk, pv, 1.0, old, out, lse, None, "plain")
    assert _same_bits(cache.weights, old)
    for decay in (0.0, 0.75, 1.0):
        w = torch.full_like(old, -3.0)
        o2, l2 = wb.wave_cache_attention_decode(q, cache, pk, pv, decay=decay, weights_out=w)
        assert _same_bits(o2, out) and _same_bits(l2, lse)
        _check_attention(dtype, q, cache, lengths, pk, pv, decay, old, o2, l2, w, f"decay {decay}")
        for b in range(B):
            assert bool((w[b, :, min(max(lengths[b], 0), cap):] == -3.0).all())     # rows behind the length
    wb.wave_cache_attention_decode(q, cache, pk, pv, decay=1.0, weights_out=cache.weights)   # in place
    for b in range(B):
        n = min(max(lengths[b], 0), cap)
        assert _same_bits(cache.weights[b, :, :n], w[b, :, :n]) and _same_bits(cache.weights[b, :, n:], old[b, :, n:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 6, 7, 8])
def test_attention_heads_and_batches(dtype, G):
    """Every group size, batches whose query rows fill one, two, four and more tiles and more sequences than a wave has lanes."""
    for B in (1, 4, 9, 70):
        lengths = [(13 * b) % 41 for b in range(B)]
        cache, q, pk, pv = _inputs(dtype, B, 2 * G, 2, 64, 41, lengths, 260, G)
        w = torch.zeros_like(cache.weights)
        out, lse = wb.wave_cache_attention_decode(q, cache, pk, pv, weights_out=w, decay=0.0)
        _check_attention(dtype, q, cache, lengths, pk, pv, 0.0, cache.weights, out, lse, w, f"B {B}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_long(dtype):
    """Many pieces of unlike lengths, peaked and flat softmax, a prefix cut into many ranges."""
    for peak, seed in ((0.1, 3), (6.0, 4)):
        lengths = [20011, 1, 4096, 0]
        cache, q, pk, pv = _inputs(dtype, 4, 8, 2, 128, 20011, lengths, 9001, seed, peak)
        w = torch.zeros_like(cache.weights)
        out, lse = wb.wave_cache_attention_decode(q, cache, pk, pv, weights_out=w)
        _check_attention(dtype, q, cache, lengths, pk, pv, 1.0, cache.weights, out, lse, w, f"peak {peak}")


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 128)])
@pytest.mark.parametrize("B,Hq,Hkv,cap,lengths,P", [
    (30, 4, 4, 6001, [17 * b for b in range(29)] + [6001], 0),                 # one long among short ones
    (9, 8, 4, 2600, [2600 - 256 * b for b in range(9)], 1),                    # no even share of the pieces
    (70, 16, 2, 1500, [(97 * b) % 400 for b in range(69)] + [1500], 0),        # more sequences than a wave has lanes, many heads
    (300, 8, 1, 60, [b % 61 for b in range(300)], 40),
    (129, 8, 8, 300, [0] * 64 + [300] * 64 + [1], 0)])
def test_attention_ragged(dtype, d, B, Hq, Hkv, cap, lengths, P):
    cache, q, pk, pv = _inputs(dtype, B, Hq, Hkv, d, cap, lengths, P, B)
    w = torch.zeros_like(cache.weights)
    out, lse = wb.wave_cache_attention_decode(q, cache, pk, pv, weights_out=w, decay=0.5)
    _check_attention(dtype, q, cache, lengths, pk, pv, 0.5, cache.weights, out, lse, w, f"B {B}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,P", [(20, 32768), (17, 32767), (40, 33001)])
def test_attention_long_prefix_of_many_query_rows(d, B, P):
    """On both sides of the line from which the prefix's weights are two numbers; a last tile with waves that have no column."""
    lengths = [b % 5 for b in range(B)]
    cache, q, pk, pv = _inputs("bf16", B, 4, 1, d, 8, lengths, P, P, 3.0)
    w = torch.zeros_like(cache.weights)
    out, lse = wb.wave_cache_attention_decode(q, cache, pk, pv, weights_out=w)
    _check_attention("bf16", q, cache, lengths, pk, pv, 1.0, cache.weights, out, lse, w, f"P {P}")


@pytest.mark.parametrize("d,B,Hq,Hkv,P", [(128, 33, 8, 2, 1000), (128, 33, 8, 2, 13001), (64, 33, 8, 2, 13001), (64, 64, 64, 8, 13225)])
def test_attention_prefix_of_many_query_rows(d, B, Hq, Hkv, P):
    """One and two tiles of columns a wave, weights in three numbers; some of the sequences are looked at."""
    lengths = [(7 * b) % 30 for b in range(B)]
    cache, q, pk, pv = _inputs("bf16", B, Hq, Hkv, d, 600, lengths, P, P, 3.0)
    w = torch.zeros_like(cache.weights)
    out, lse = wb.wave_cache_attention_decode(q, cache, pk, pv, weights_out=w, decay=0.25)
    some = [0, B // 2, B - 1]
    pick = wb.cache_from_tensors(*(cache.t[n][some].contiguous() for n in ("k", "v", "positions", "weights", "lengths", "tokens")))
    _check_attention("bf16", q[some], pick, [lengths[b] for b in some], pk, pv, 0.25, pick.weights, out[some], lse[some], w[some])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,Hq,P", [(1, 8, 66000), (3, 2, 40001)])
def test_attention_of_many_partial_results(dtype, B, Hq, P):
    """One KV head: as many ranges of the prefix, and pieces of a long sequence, as there may be."""
    lengths = [30000, 1, 0][:B]
    cache, q, pk, pv = _inputs(dtype, B, Hq, 1, 64, 30000, lengths, P, P, 2.0)
    w = torch.zeros_like(cache.weights)
    out, lse = wb.wave_cache_attention_decode(q, cache, pk, pv, weights_out=w, decay=0.0)
    _check_attention(dtype, q, cache, lengths, pk, pv, 0.0, cache.weights, out, lse, w)


@pytest.mark.parametrize("d,c", [(64, 0.625), (128, 0.4375)])
@pytest.mark.parametrize("B,P", [(1, 32768), (16, 32768), (17, 32768), (40, 33001), (17, 4000)])
def test_attention_weights_keep_their_bits_behind_any_prefix(d, c, B, P):
    """Two rows of the prefix have all the weight, one of them nearly all of it, 2^5 .. 2^8 over the reference that the other one
    has set: a weight that lost bits shows in the output, whatever the length and the number of query rows are.  The scores are exact
    (16 bits a product, up to 128 equal ones), the weights' exponents off by 4 roundings of up to 8, 22 u of the weight, and
    the exponential by 2 u: that moves the output by 24 u p0 p1 |v1 - v0|; the products with the values, their sums, the joining
    and the quotient are 16 roundings at most."""
    g = _gen(P + B)
    cache = wb.alloc_cache(torch.bfloat16, B, 1, d, 8)
    f = (0.7 + 0.4 * torch.rand(B, 4, 1, generator=g)).bfloat16()
    k = torch.full((1, P, d), -100.0)
    k[0, 3], k[0, 100] = 0.0, c
    v = torch.randn(1, P, d, generator=g).bfloat16()
    out, lse = wb.wave_cache_attention_decode(f.expand(B, 4, d).contiguous().cuda(), cache, k.bfloat16().cuda(), v.cuda())
    z = f.double() * c * math.sqrt(d)
    p1, v0, v1 = torch.sigmoid(z), v[0, 3].double(), v[0, 100].double()
    p0 = 1 - p1
    bar = 16 * U * (p0 * v0.abs() + p1 * v1.abs()) + 24 * U * p0 * p1 * (v1 - v0).abs()
    err = (out.double().cpu() - (p0 * v0 + p1 * v1)).abs()
    assert bool((err <= bar).all()), float((err / bar).max())
    assert torch.allclose(lse.double().cpu(), torch.log1p(torch.exp(z))[..., 0], rtol=0, atol=64 * U)


@pytest.mark.parametrize("B", [2, 8, 20])
def test_attention_values_that_are_not_finite_show_in_their_channel(B):
    """An infinite value in the last prefix row, and in the last own row: its channel is not finite (a weight is a sum of bf16
    numbers of which some may be zero or negative, so infinity times it may be no number: never a finite one), the others are
    as without it, although the rows that fill up the last step are copies of the last row; 8, 32 and 80 query rows."""
    cache, q, pk, pv = _inputs("bf16", B, 4, 1, 128, 8, [5] * B, 77, 3, 0.5)
    good, _ = wb.wave_cache_attention_decode(q, cache, pk, pv)
    pv[0, 76, 5] = math.inf
    cache.v[0, 0, 4, 9] = -math.inf
    out, _ = wb.wave_cache_attention_decode(q, cache, pk, pv)
    assert not torch.isfinite(out[..., 5]).any() and not torch.isfinite(out[0, :, 9]).any()
    keep = [c for c in range(128) if c not in (5, 9)]
    assert _same_bits(out[..., keep], good[..., keep]) and _same_bits(out[1:, :, 9], good[1:, :, 9])


def test_attention_with_the_workspace_of_the_longest_prefix():
    """One workspace, asked for once, for prefixes of fewer rows (which are cut into more ranges) and of none."""
    cache, q, pk, pv = _inputs("bf16", 8, 32, 8, 128, 2048, [7 * b for b in range(8)], 8255, 4)
    ws = wb.workspace(wb.wave_cache_attention_workspace(cache, 32, 8255, True))
    for P in (8255, 8128, 1000, 129, 1, 0):
        k, v = (x[:, :P].contiguous() if P else None for x in (pk, pv))
        out, lse = wb.wave_cache_attention_decode(q, cache, k, v, ws=ws)
        own = wb.wave_cache_attention_decode(q, cache, k, v)
        assert _same_bits(out, own[0]) and _same_bits(lse, own[1]), P


@pytest.mark.parametrize("B,Hq,Hkv,cap", [(3, 8, 2, 20), (3, 8, 2, 700), (64, 32, 4, 700)])
def test_attention_into_outputs_that_lie_on_floats(B, Hq, Hkv, cap):
    """Outputs a float behind a 16-byte line: one launch, a workgroup and a wave a head in the joining."""
    lengths = [(5 * b) % (cap + 1) for b in range(B)]
    cache, q, pk, pv = _inputs("bf16", B, Hq, Hkv, 64, cap, lengths, 100, 6)
    want = wb.wave_cache_attention_decode(q, cache, pk, pv, weights_out=torch.zeros_like(cache.weights), decay=0.0)
    w0 = torch.full_like(cache.weights, -3.0)
    wb.wave_cache_attention_decode(q, cache, pk, pv, weights_out=w0, decay=0.0)
    for shift in (1, 2, 3):
        room = lambda *shape: torch.full((math.prod(shape) + 4,), -3.0, device="cuda")[shift:shift + math.prod(shape)].view(*shape)
        out, lse, w = room(B, Hq, 64), room(B, Hq), room(*cache.weights.shape)
        assert out.data_ptr() % 16 == 4 * shift
        wb.wave_cache_attention_decode(q, cache, pk, pv, weights_out=w, decay=0.0, out=out, lse=lse)
        assert _same_bits(out, want[0]) and _same_bits(lse, want[1]) and _same_bits(w, w0), shift


def test_attention_without_rows_anywhere():
    cache, q, _, _ = _inputs("bf16", 3, 4, 2, 128, 16, [0, 0, 0], 0, 5)
    w = torch.full_like(cache.weights, 2.0)
    out, lse = wb.wave_cache_attention_decode(q, cache, weights_out=w)
    assert not out.any() and bool((lse == -math.inf).all()) and bool((w == 2.0).all())
    empty = torch.zeros(2, 0, 128, dtype=torch.bfloat16, device="cuda")
    out, lse = wb.wave_cache_attention_decode(q, cache, empty, empty)
    assert not out.any() and bool((lse == -math.inf).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_extreme_scores(dtype):
    """Rising scores (the reference has to follow), one dominant row, and infinite and undefined scores: they show up, in
    their own head alone."""
    B, Hq, Hkv, d, n = 1, 4, 1, 128, 700
    cache, q, _, _ = _inputs(dtype, B, Hq, Hkv, d, n, [n], 0, 9, 1.0)
    cache.k[0, 0] = (torch.arange(n)[:, None] / n * 4 * torch.ones(d)).to(cache.dtype).cuda()    # scores rise row by row
    cache.k[0, 0, 650] *= 8
    q[0, 0] = 1.0
    q[0, 1] = -1.0
    w = torch.zeros_like(cache.weights)
    out, lse = wb.wave_cache_attention_decode(q, cache, weights_out=w, decay=0.0)
    _check_attention(dtype, q, cache, [n], None, None, 0.0, cache.weights, out, lse, w, "rising")
    good = out.clone()
    q[0, 2, 5] = math.nan
    o2, l2 = wb.wave_cache_attention_decode(q, cache)
    assert bool(torch.isnan(o2[0, 2]).all()) and bool(torch.isnan(l2[0, 2]))
    for h in (0, 1, 3):
        assert _same_bits(o2[0, h], good[0, h])
    q[0, 2, 5] = math.inf
    o2, l2 = wb.wave_cache_attention_decode(q, cache)
    assert bool(torch.isnan(o2[0, 2]).all()) and _same_bits(o2[0, 3], good[0, 3])
    # scores of -infinity: those rows have no weight; a head that has nothing else counts as having no rows
    q[0, 2] = -1.0
    cache.k[0, 0, :650] = math.inf
    o2, l2 = wb.wave_cache_attention_decode(q, cache)
    K, V = cache.k[0, 0, 650:].double().cpu().numpy(), cache.v[0, 0, 650:].double().cpu().numpy()
    o, l, _ = co.attend(q[0, 2].double().cpu().numpy(), K, V)
    assert np.allclose(o2[0, 2].cpu().numpy(), o, atol=1e-4) and abs(float(l2[0, 2]) - l) < 1e-3
    cache.k[0, 0] = math.inf
    o2, l2 = wb.wave_cache_attention_decode(q, cache)
    assert not o2[0, 2].any() and float(l2[0, 2]) == -math.inf


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,Hq,Hkv,lengths,P", [
    (1, 1, 1, [1], 0), (1, 8, 1, [33], 1), (2, 6, 2, [0, 129], 0), (3, 7, 1, [128, 1, 700], 127), (5, 10, 2, [0, 70, 31, 32, 64], 129),
    (9, 8, 1, [0] * 9, 300), (2, 2, 2, [-4, 900], 0), (17, 16, 4, list(range(17)), 65)])
def test_attention_with_room_for_many_rows(dtype, d, B, Hq, Hkv, lengths, P):
    """Room for 700 rows a unit: cut into pieces and joined, whatever is in use."""
    test_attention(dtype, d, B, Hq, Hkv, 700, lengths, P)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 6, 7, 8])
def test_attention_heads_and_room(dtype, G):
    for B, cap in ((4, 700), (9, 250), (70, 700), (70, 120)):
        lengths = [(13 * b) % 41 for b in range(B)]
        cache, q, pk, pv = _inputs(dtype, B, 2 * G, 2, 64, cap, lengths, 6, G)
        w = torch.zeros_like(cache.weights)
        out, lse = wb.wave_cache_attention_decode(q, cache, pk, pv, weights_out=w, decay=0.0)
        _check_attention(dtype, q, cache, lengths, pk, pv, 0.0, cache.weights, out, lse, w, f"B {B} cap {cap}")


@pytest.mark.parametrize("cap", [50, 700])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_of_scores_that_are_no_numbers(dtype, cap):
    """In a short cache and in one of pieces: a head whose scores are not numbers says so, one whose scores are all -infinity
    counts as without rows, its weights too, and the other heads are as they were."""
    n, d = 50, 128
    cache, q, pk, pv = _inputs(dtype, 1, 4, 1, d, cap, [n], 40, 9, 1.0)
    cache.k[0, 0, :n] = cache.k[0, 0, :n].abs() + 0.125
    q[0, 3] = -1.0
    good, glse = wb.wave_cache_attention_decode(q, cache)
    both, blse = wb.wave_cache_attention_decode(q, cache, pk, pv)
    q[0, 1, 5] = math.nan
    for k, v, want in ((None, None, good), (pk, pv, both)):
        w = torch.zeros_like(cache.weights)
        out, lse = wb.wave_cache_attention_decode(q, cache, k, v, weights_out=w)
        assert bool(torch.isnan(out[0, 1]).all()) and bool(torch.isnan(lse[0, 1])) and bool(torch.isnan(w[0, 0, :n]).all())
        assert _same_bits(out[0, [0, 2, 3]], want[0, [0, 2, 3]])
    q[0, 1] = -1.0
    cache.k[0, 0, :n] = math.inf
    w = torch.zeros_like(cache.weights)
    out, lse = wb.wave_cache_attention_decode(q[:, [1, 3, 1, 3]].contiguous(), cache, weights_out=w)
    assert not out.any() and bool((lse == -math.inf).all()) and _same_bits(w[0, 0, :n], cache.weights[0, 0, :n])
    out, lse = wb.wave_cache_attention_decode(q[:, [1, 3, 1, 3]].contiguous(), cache, pk, pv, weights_out=w)
    alone, alse = wb.wave_cache_attention_decode(q[:, [1, 3, 1, 3]].contiguous(), wb.alloc_cache(cache.dtype, 1, 1, d, cap), pk, pv)
    # The same sums of 40 weights, with other waves' nothing between them: up to 40 + 16 roundings each, of values up to 5.
    assert torch.allclose(out, alone, rtol=0, atol=2 * 56 * 5 * U) and torch.allclose(lse, alse, rtol=0, atol=2 * 56 * U)
    assert _same_bits(w[0, 0, :n], cache.weights[0, 0, :n])        # (decay 1: the old weights and nothing)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_prompt_appended_to_its_own_cache_is_the_prefix(dtype):
    """A one-sequence cache with as much room as the prompt has rows is the prefix as it lies; part of a larger one (a view that
    the call copies) gives the same bits."""
    P, B, Hq, Hkv, d = 203, 3, 8, 2, 64
    cache, q, _, _ = _inputs(dtype, B, Hq, Hkv, d, 40, [40, 0, 9], 0, 12)
    k, v = (torch.randn(1, Hkv, P, d, generator=_gen(s)).to(TYPES[dtype]).cuda() for s in (1, 2))
    rot = wb.wave_rotary_plan(d, 1e4)
    tight, roomy = wb.alloc_cache(TYPES[dtype], 1, Hkv, d, P), wb.alloc_cache(TYPES[dtype], 1, Hkv, d, P + 50)
    for prompt in (tight, roomy):
        wb.wave_cache_append(prompt, k, v, rotary=rot)
    assert tight.k[0].is_contiguous() and not roomy.k[0, :, :P].is_contiguous()
    out, lse = wb.wave_cache_attention_decode(q, cache, tight.k[0], tight.v[0])
    _check_attention(dtype, q, cache, [40, 0, 9], tight.k[0], tight.v[0], 1.0, cache.weights, out, lse, None)
    o2, l2 = wb.wave_cache_attention_decode(q, cache, roomy.k[0, :, :P], roomy.v[0, :, :P])
    assert _same_bits(out, o2) and _same_bits(lse, l2)


def test_attention_equals_full_attention_decode():
    g = _gen(21)
    K, V = (torch.randn(2, 2, 1000, 128, generator=g).bfloat16().cuda() for _ in range(2))
    q = torch.randn(2, 8, 128, generator=g).bfloat16().cuda()
    o1, l1 = wb.wave_full_attention_decode(q, K, V)
    cache = wb.cache_from_tensors(K, V, None, None, torch.full((2,), 1000, dtype=torch.int32, device="cuda"), None)
    o2, l2 = wb.wave_cache_attention_decode(q, cache)
    # both against the exact value by less than 2^-18 and the sums' roundings
    assert float((o1 - o2).abs().max()) < 2e-5 and float((l1 - l2).abs().max()) < 2e-5
    # the same rows as prefix of the first and rows of the second half
    half = wb.cache_from_tensors(K[:1, :, 400:].contiguous(), V[:1, :, 400:].contiguous(), None, None,
                                 torch.full((1,), 600, dtype=torch.int32, device="cuda"), None)
    o3, l3 = wb.wave_cache_attention_decode(q[:1], half, K[0, :, :400].contiguous(), V[0, :, :400].contiguous())
    assert float((o1[:1] - o3).abs().max()) < 2e-5 and float((l1[:1] - l3).abs().max()) < 2e-5


def test_prefix_through_its_index_and_own_rows_join_by_their_normalisers():
    """Keys of a shared prompt rotated in place, indexed, attended with every cluster retrieved, and joined with the own rows'
    attention by log-sum-exp: the same as the prefix and the own rows in one call."""
    g = _gen(71)
    P, B, Hq, Hkv, d = 1100, 1, 8, 2, 128
    rot = wb.wave_rotary_plan(d, 500000.0, [24, 20, 20], wb.WAVE_ROTARY_TURNS)
    K, V = (torch.randn(B, Hkv, P, d, generator=g).bfloat16().cuda() for _ in range(2))
    at = torch.arange(P, dtype=torch.int32).expand(3, B, P).contiguous().cuda()
    wb.wave_rotary_apply(K, at, rot, out=K)
    ix = wb.wave_index_build(K, V, 4, 64, 512, 32, 3, 0)
    cache = wb.alloc_cache(torch.bfloat16, B, Hkv, d, 64)
    k, v = (torch.randn(B, Hkv, 33, d, generator=g).bfloat16().cuda() for _ in range(2))
    q = torch.randn(B, Hq, 33, d, generator=g).bfloat16().cuda()
    cache.tokens.fill_(P)                                              # the conversation goes on behind the prompt
    qr = wb.wave_cache_append(cache, k, v, q=q, rotary=rot)[:, :, 32].contiguous()
    o1, l1, _ = wb.wave_attention_decode(qr, ix, ix.m)
    o2, l2 = wb.wave_cache_attention_decode(qr, cache)
    both = torch.logaddexp(l1, l2)
    joined = o1 * torch.exp(l1 - both)[..., None] + o2 * torch.exp(l2 - both)[..., None]
    o3, l3 = wb.wave_cache_attention_decode(qr, cache, K[0], V[0])
    assert float((joined - o3).abs().max()) < 2e-5 and float((both - l3).abs().max()) < 2e-5


# --------------------------------------------------------------------------- eviction
def _check_evict(cache, before, lengths, n_keep, n_sink, n_local, to, dst_before):
    B, Hkv, cap = cache.B, cache.Hkv, cache.capacity
    pos, wts = before["positions"].cpu().numpy(), before["weights"].cpu().numpy()
    tokens = before["tokens"].tolist()
    want = {name: t.clone() for name, t in dst_before.items()}
    for b in range(B):
        n = min(max(lengths[b], 0), cap)
        rows = None
        for h in range(Hkv):
            rows = co.evict(pos[b, h].tolist(), wts[b, h].tolist(), n, tokens[b], n_keep, n_sink, n_local)
            at = torch.tensor(rows, dtype=torch.long, device="cuda")
            for name in ("k", "v", "positions", "weights"):
                want[name][b, h, :len(rows)] = before[name][b, h][at]
        want["lengths"][b], want["tokens"][b] = min(n, n_keep), tokens[b]
    for name, t in want.items():
        assert _same_bits(to.t[name], t), name


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("f32", 128), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("B,Hkv,cap,lengths,n_keep,n_sink,n_local", [
    (1, 1, 1, [1], 0, 0, 0), (1, 2, 9, [9], 4, 1, 2), (3, 2, 70, [70, 0, 33], 32, 4, 8), (2, 1, 3000, [2999, 3000], 2998, 4, 100),
    (2, 2, 5000, [4097, 5000], 1025, 0, 1025), (2, 1, 300, [300, 200], 400, 2, 2), (3, 1, 64, [-5, 99, 64], 63, 0, 0),
    (1, 2, 2100, [2100], 1, 1, 0)])
@pytest.mark.parametrize("ties", [False, True])
def test_evict(dtype, d, B, Hkv, cap, lengths, n_keep, n_sink, n_local, ties):
    def fresh():
        c = _filled_cache(dtype, B, Hkv, d, cap, lengths, cap)
        if ties:   # few values, both zeros, negative and infinite ones, and no numbers
            few = torch.tensor([0.0, -0.0, 0.5, 0.5, 1.0, -1.0, math.inf, -math.inf, math.nan])
            c.weights.copy_(few[torch.randint(0, 9, tuple(c.weights.shape), generator=_gen(cap))])
        return c
    cache = fresh()
    before = {name: t.clone() for name, t in cache.t.items()}
    assert wb.wave_cache_evict(cache, n_keep, n_sink, n_local) is cache               # in place
    _check_evict(cache, before, lengths, n_keep, n_sink, n_local, cache, before)
    cache = fresh()                                                                       # into a cache that just holds them
    room = max(min(n_keep, cap), 1)
    to = wb.alloc_cache(TYPES[dtype], B, Hkv, d, room)
    for t in to.t.values():
        t.fill_(3)
    dst = {name: t.clone() for name, t in to.t.items()}
    assert wb.wave_cache_evict(cache, n_keep, n_sink, n_local, to=to) is to
    _check_evict(cache, before, lengths, n_keep, n_sink, n_local, to, dst)
    for name, t in cache.t.items():
        assert _same_bits(t, before[name]), name                                          # the old one is as it was
    mixed = wb.cache_from_tensors(cache.k, cache.v, torch.full_like(cache.positions, -9), cache.weights, torch.zeros_like(cache.lengths),
                                  cache.tokens)                                            # some arrays in place, some not
    dst = {name: t.clone() for name, t in mixed.t.items()}
    wb.wave_cache_evict(cache, n_keep, n_sink, n_local, to=mixed)
    _check_evict(cache, before, lengths, n_keep, n_sink, n_local, mixed, dst)


@pytest.mark.parametrize("keys", list(range(1, 17)))
def test_evict_every_number_of_keys_a_thread(keys):
    """Rooms at both ends of each: the last row with a key of its own, and one row less."""
    for cap in (1024 * (keys - 1) + 1, 1024 * keys):
        lengths = [cap, cap - 1, cap // 2]
        cache = _filled_cache("bf16", 3, 1, 64, cap, lengths, keys)
        before = {name: t.clone() for name, t in cache.t.items()}
        n_keep = max(cap * 2 // 3, 1)
        wb.wave_cache_evict(cache, n_keep, min(1, n_keep), 0)
        _check_evict(cache, before, lengths, n_keep, min(1, n_keep), 0, cache, before)


def test_evict_long():
    cache = _filled_cache("bf16", 1, 2, 64, 131000, [130999], 3)
    before = {name: t.clone() for name, t in cache.t.items()}
    wb.wave_cache_evict(cache, 16385, 4, 1024)
    _check_evict(cache, before, [130999], 16385, 4, 1024, cache, before)


@pytest.mark.parametrize("n_keep,n_sink,n_local", [(0, 0, 0), (1, 0, 1), (8192, 4, 100), (8193, 4, 4000), (16000, 0, 0), (19999, 1, 1)])
@pytest.mark.parametrize("ties", [False, True])
def test_evict_caches_of_more_rows_than_a_workgroup_holds(n_keep, n_sink, n_local, ties):
    """In place and apart; full, half full, short and empty sequences in the same call."""
    lengths = [20001, 9000, 0, 16385]
    cache = _filled_cache("bf16", 4, 1, 64, 20001, lengths, n_keep)
    if ties:
        few = torch.tensor([0.0, -0.0, 0.25, 0.25, math.nan])
        cache.weights.copy_(few[torch.randint(0, 5, tuple(cache.weights.shape), generator=_gen(1))])
    before = {name: t.clone() for name, t in cache.t.items()}
    to = wb.alloc_cache(torch.bfloat16, 4, 1, 64, max(n_keep, 1) + 3)
    dst = {name: t.clone() for name, t in to.t.items()}
    wb.wave_cache_evict(cache, n_keep, n_sink, n_local, to=to)
    _check_evict(cache, before, lengths, n_keep, n_sink, n_local, to, dst)
    mixed = wb.cache_from_tensors(cache.k, cache.v, torch.full_like(cache.positions, -9), torch.zeros_like(cache.weights),
                                  cache.lengths, torch.zeros_like(cache.tokens))
    dst = {name: t.clone() for name, t in mixed.t.items()}
    wb.wave_cache_evict(cache, n_keep, n_sink, n_local, to=mixed)
    _check_evict(cache, before, lengths, n_keep, n_sink, n_local, mixed, dst)


# --------------------------------------------------------------------------- together


def _decode_loop(dtype, steps, run):
    """`run(step, q, k, v)` for every token; returns the last outputs."""
    g = _gen(31)
    outs = []
    for i in range(steps):
        q, k, v = (torch.randn(2, h, 1, 64, generator=g).to(TYPES[dtype]).cuda() for h in (4, 2, 2))
        outs.append(run(i, q, k, v))
    return outs


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_conversation(dtype):
    """Prompt, decode steps with accumulated weights behind a shared prefix, eviction whenever the cache is full: the GPU's
    own stored rows and weights against the plain statement of every step."""
    B, Hq, Hkv, d, cap, keep = 2, 4, 2, 64, 48, 24
    cache = wb.alloc_cache(TYPES[dtype], B, Hkv, d, cap)
    g = _gen(32)
    pk, pv = (torch.randn(Hkv, 77, d, generator=g).to(TYPES[dtype]).cuda() for _ in range(2))
    rot = wb.wave_rotary_plan(64, 1e4, [16, 16], wb.WAVE_ROTARY_TURNS)
    prompt_k, prompt_v = (torch.randn(B, Hkv, 30, d, generator=g).to(TYPES[dtype]).cuda() for _ in range(2))
    counts = torch.tensor([30, 11], dtype=torch.int32, device="cuda")
    wb.wave_cache_append(cache, prompt_k, prompt_v, rotary=rot, counts=counts)
    lengths, tokens = [30, 11], [30, 11]
    assert cache.lengths.tolist() == lengths

    def step(i, q, k, v):
        qr = wb.wave_cache_append(cache, k, v, q=q, rotary=rot)
        for b in range(B):
            lengths[b] += 1
            tokens[b] += 1
            assert cache.positions[b, :, lengths[b] - 1].tolist() == [tokens[b] - 1] * Hkv
        old = cache.weights.clone()
        out, lse = wb.wave_cache_attention_decode(qr[:, :, 0], cache, pk, pv, decay=0.9, weights_out=cache.weights)
        _check_attention(dtype, qr[:, :, 0], cache, lengths, pk, pv, 0.9, old, out, lse, cache.weights, f"step {i}")
        if max(lengths) == cap:
            before = {name: t.clone() for name, t in cache.t.items()}
            wb.wave_cache_evict(cache, keep, 2, 8)
            _check_evict(cache, before, lengths, keep, 2, 8, cache, before)
            for b in range(B):
                lengths[b] = min(lengths[b], keep)
        assert cache.lengths.tolist() == lengths and cache.tokens.tolist() == tokens
        return out

    _decode_loop(dtype, 60, step)
    # what every unit still holds: its first and its newest tokens among it
    for b in range(B):
        for h in range(Hkv):
            held = set(cache.positions[b, h, :lengths[b]].tolist())
            assert {0, 1} <= held and set(range(tokens[b] - (8 if lengths[b] >= keep else 1), tokens[b])) <= held and len(held) == lengths[b]


def test_captured_steps_replay():
    """A captured decode step (append, attention with weights, eviction) replayed with work of its own between the replays,
    against the same steps run eagerly; another captured graph shares the workspace."""
    dtype, B, Hq, Hkv, d, cap, keep = "bf16", 2, 8, 2, 128, 64, 60
    rot = wb.wave_rotary_plan(128, 1e4)
    g = _gen(41)
    pk, pv = (torch.randn(Hkv, 130, d, generator=g).bfloat16().cuda() for _ in range(2))
    tokens = [[torch.randn(B, h, 1, d, generator=g).bfloat16().cuda() for h in (Hq, Hkv, Hkv)] for _ in range(8)]
    lengths = [60, 3]

    def make():
        c = _filled_cache(dtype, B, Hkv, d, cap, lengths, 8)
        ws = wb.workspace(max(wb.wave_cache_attention_workspace(c, Hq, 130, True), wb.wave_cache_evict_workspace(c, keep)))
        bufs = dict(q=tokens[0][0].clone(), k=tokens[0][1].clone(), v=tokens[0][2].clone(), q_out=torch.empty_like(tokens[0][0]),
                    out=torch.empty(B, Hq, d, device="cuda"), lse=torch.empty(B, Hq, device="cuda"))
        return c, ws, bufs

    def step(c, ws, x):
        wb.wave_cache_append(c, x["k"], x["v"], q=x["q"], rotary=rot, q_out=x["q_out"])
        wb.wave_cache_attention_decode(x["q_out"].view(B, Hq, d), c, pk, pv, decay=0.95, weights_out=c.weights, out=x["out"],
                                       lse=x["lse"], ws=ws)
        wb.wave_cache_evict(c, keep, 4, 8, ws=ws)

    ce, we, be = make()
    cg, wg, bg = make()
    ch, _, bh = make()
    step(*make())                                      # first launches outside the capture
    torch.cuda.synchronize()
    saved = {n: t.clone() for n, t in cg.t.items()}
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(cg, wg, bg)
    with torch.cuda.graph(other):
        step(ch, wg, bh)
    for n, t in saved.items():
        cg.t[n].copy_(t)
    for i, (q, k, v) in enumerate(tokens):
        for x in (be, bg, bh):
            x["q"].copy_(q), x["k"].copy_(k), x["v"].copy_(v)
        step(ce, we, be)
        torch.cuda.synchronize()
        graph.replay()
        other.replay()
        torch.cuda.synchronize()
        for x, c in ((bg, cg), (bh, ch)):
            assert _same_bits(be["out"], x["out"]) and _same_bits(be["lse"], x["lse"]) and _same_bits(be["q_out"], x["q_out"]), i
            for n in ce.t:
                assert _same_bits(ce.t[n], c.t[n]), (i, n)


def test_two_streams_and_repeated_calls_give_the_same_bits():
    lengths = [700, 31, 0]
    cache, q, pk, pv = _inputs("bf16", 3, 14, 2, 128, 700, lengths, 400, 51)
    first = wb.wave_cache_attention_decode(q, cache, pk, pv, weights_out=torch.zeros_like(cache.weights))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [wb.workspace(wb.wave_cache_attention_workspace(cache, 14, 400, True)) for _ in streams]
    ww = [torch.zeros_like(cache.weights) for _ in streams]
    outs = []
    torch.cuda.synchronize()
    for _ in range(3):
        for s, w, x in zip(streams, ws, ww):
            with torch.cuda.stream(s):
                outs.append(wb.wave_cache_attention_decode(q, cache, pk, pv, weights_out=x, ws=w))
    torch.cuda.synchronize()
    for out, lse in outs:
        assert _same_bits(out, first[0]) and _same_bits(lse, first[1])
    assert _same_bits(ww[0], ww[1])


def test_offsets_beyond_32_bits():
    """A cache whose last unit starts more than 4 GiB into its arrays."""
    B, Hkv, d, cap, n = 1, 2, 128, 17_000_000, 300
    k, v = (torch.zeros(B, Hkv, cap, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache = wb.cache_from_tensors(k, v, torch.full((B, Hkv, cap), -1, dtype=torch.int32, device="cuda"),
                                  torch.zeros(B, Hkv, cap, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda"),
                                  torch.zeros(B, dtype=torch.int32, device="cuda"))
    g = _gen(61)
    kn, vn = (torch.randn(B, Hkv, n, d, generator=g).bfloat16().cuda() for _ in range(2))
    q = torch.randn(B, 4, d, generator=g).bfloat16().cuda()
    wb.wave_cache_append(cache, kn, vn)
    small = wb.alloc_cache(torch.bfloat16, B, Hkv, d, 700)   # (room for more than one launch takes: the same order of sums)
    wb.wave_cache_append(small, kn, vn)
    for c in (cache, small):
        c.out = wb.wave_cache_attention_decode(q, c, weights_out=c.weights)
        wb.wave_cache_evict(c, 100, 1, 10)
    assert _same_bits(cache.out[0], small.out[0]) and _same_bits(cache.out[1], small.out[1])
    for name in ("k", "v", "positions", "weights"):
        assert _same_bits(cache.t[name][:, :, :n], small.t[name][:, :, :n]), name
    # rows at the far end of the last unit
    cache.lengths.fill_(cap - 1)
    wb.wave_cache_append(cache, kn, vn)
    assert cache.lengths.tolist() == [cap] and _same_bits(cache.k[0, 1, cap - 1], kn[0, 1, 0])
