"""Operators of the paged 8-bit cache and of the norms before it, as cases that can be timed and compared.

  norm     `wave_norm_rotary_apply`: queries and keys normed for each head and turned by their positions, read where they lie
  append   `wave_pages_append`: new tokens' rows collected until a page is complete, which is held in 8 bits with a scale for
           each page and head; then `wave_pages_read` of the rows around them, as an index that is built from them reads them
  read     `wave_pages_read`: rows of a paged cache back in the storage type
  attend   `wave_pages_attention_decode`: one token's attention over a paged cache
  reorder  `wave_pages_reorder`: sequences copied, forked and freed by sharing and counting pages

`run` has two forms of each: elementary torch operations in 32 bits (`own = False`), and the calls that a program makes of
`paper_2505_02922_amd.binding` (`own = True`).  `exact` is the definition in 64 bits.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}

# One transformer layer of the workloads the benchmark names; a case replaces what differs.
_LLAMA = dict(dtype="bf16", Hq=32, Hkv=8, d=128)
_QWEN = dict(dtype="bf16", Hq=28, Hkv=4, d=128)
_TINY = dict(dtype="f32", Hq=8, Hkv=2, d=64)

_EPS = 1e-6
_LEAST = 2.0 ** -100  # a page of smaller values than this reads as zeros


def listed():
    return [
        # Every decode step of a large batch, queries and keys as the fused projection leaves them.
        dict(_QWEN, name="norm_bf16_token_b64", op="norm", B=64, n=1, fused=True, rot=128, base=1000000.0, sections="64", halves=True, far=65536),
        # Two prompts before their index is built.
        dict(_LLAMA, name="norm_bf16_16k_b2", op="norm", B=2, n=16381, fused=True, rot=128, base=500000.0, sections="64", halves=True, far=16381),
        # A decode step of a large batch: a token for each sequence, and about one sequence in 64 completes a page.
        dict(_QWEN, name="append_bf16_token_b64", op="append", B=64, n=1, page=64, short=700, long=4351, shared=0, ragged=False, fused=True, norm=True,
             rot=128, base=1000000.0, sections="64", halves=True),
        # The prompts of four chats with images (three axes), padded to the longest, into empty caches.
        dict(_LLAMA, name="append_bf16_prompt_b4_3axes", op="append", B=4, n=8191, page=64, short=0, long=0, shared=0, ragged=True, fused=False,
             norm=False, rot=128, base=500000.0, sections="16,24,24", halves=True),
        # A few short fp32 sequences read back: the smallest call.
        dict(_TINY, name="read_f32_300_b3", op="read", B=3, page=32, short=100, long=300, shared=0, n=300),
        # A prompt of 120K tokens read back before its index is built.
        dict(_LLAMA, name="read_bf16_120k_b1", op="read", B=1, page=128, short=122877, long=122877, shared=0, n=122880),
        # A few short fp32 sequences: the smallest call.
        dict(_TINY, name="attend_f32_200_b3", op="attend", B=3, page=32, short=1, long=200, shared=0),
        # A single chat of 4K tokens: the interactive step.
        dict(_LLAMA, name="attend_bf16_4k_b1", op="attend", B=1, page=64, short=4093, long=4093, shared=0),
        # A large batch on a model with seven queries per KV head; all sequences begin with the same 1K tokens.
        dict(_QWEN, name="attend_bf16_4k_b64", op="attend", B=64, page=64, short=700, long=4351, shared=16),
        # Eight long sequences of unlike lengths.
        dict(_LLAMA, name="attend_bf16_64k_b8", op="attend", B=8, page=64, short=3001, long=65536, shared=0),
        # A beam search's step: eight beams of one short sequence.
        dict(_TINY, name="reorder_f32_beams_b8", op="reorder", B=8, to=8, page=32, short=200, long=200, shared=6),
        # A large batch of samples that begin alike; some leave, some are forked.
        dict(_LLAMA, name="reorder_bf16_8k_b256", op="reorder", B=256, to=256, page=128, short=700, long=8191, shared=4),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def plan(d):
        rot = rng.choice([r for r in (32, 64, 96, 128) if r <= d])
        axes = rng.randint(1, 3)
        cuts = sorted(rng.sample(range(1, rot // 2), axes - 1))
        sections = ",".join(str(b - a) for a, b in zip([0] + cuts, cuts + [rot // 2]))
        return dict(rot=rot, base=rng.choice([10000.0, 500000.0, 1000000.0]), sections=sections, halves=rng.random() < 0.7)

    Hkv = rng.choice([1, 2, 4, 8])
    case = dict(dtype="bf16" if rng.random() < 0.7 else "f32", Hkv=Hkv, Hq=Hkv * rng.randint(1, 8), d=rng.choice([64, 128, 128]))
    case["op"] = op = rng.choice(["norm", "append", "read", "attend", "attend", "reorder"])
    case["B"] = B = log(1, 256 if op == "reorder" else 64)
    if op == "norm":
        n = log(1, max(2, (1 << 20) // (B * case["Hq"])))
        return dict(case, n=n, fused=rng.random() < 0.5, far=log(n + 1, 1 << 20), **plan(case["d"]))
    case["page"] = rng.choice([32, 64, 128])
    if op == "append":
        n = 1 if rng.random() < 0.5 else log(2, max(3, 16384 // B))
        long = log(1, 4000)
        return dict(case, n=n, short=rng.randint(0, long), long=long, shared=0, ragged=n > 1 and rng.random() < 0.5, fused=rng.random() < 0.5,
                    norm=rng.random() < 0.5, **plan(case["d"]))
    long = log(1, max(2, min(65536, (300000 if op == "read" else 1000000) // (B * Hkv))))
    short = rng.randint(0 if op == "reorder" else 1, long)
    case.update(short=short, long=long, shared=rng.choice([0, rng.randint(0, short // case["page"])]))
    if op == "read":
        return dict(case, n=log(1, long))
    if op == "reorder":
        return dict(case, to=log(1, 256))
    return case


# ---------------------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------------------
def _spread(lo, hi, B):
    """B lengths from lo to hi, the longest first, the others in no order."""
    step = next(k for k in (7, 11, 13) if B % k)
    return [hi - (hi - lo) * ((b * step) % B) // max(B - 1, 1) for b in range(B)]


def _lengths(case):
    return _spread(case["short"], case["long"], case["B"])


def _counts(case):
    return _spread((case["n"] + 1) // 2, case["n"], case["B"]) if case["ragged"] else [case["n"]] * case["B"]


def _turns(case):
    """fp32 rows go into the pages as they are (normed and turned by a call before)."""
    return case["op"] == "norm" or case["dtype"] == "bf16"


def _sections(case):
    return [int(pairs) for pairs in case["sections"].split(",")]


def _pair_plan(case):
    """Axis and frequency (radians a position) of every turned pair."""
    pairs = case["rot"] // 2
    axis = [a for a, s in enumerate(_sections(case)) for _ in range(s)]
    return axis, [case["base"] ** (-i / pairs) for i in range(pairs)]


def _means(case, g):
    return torch.randn(case["Hkv"], 64, case["d"], generator=g, device="cuda")


def _key_rows(h, g, means, lead):
    """Clusterable keys of head h [*lead, d]: a component's mean and noise."""
    x = means[h][torch.randint(0, 64, lead, generator=g, device="cuda")]
    return x + 0.25 * torch.randn(x.shape, generator=g, device="cuda")


def _projection(case, s, g):
    """New queries, keys and values [B, heads, n, d]: dense, or views of what one projection gives ([B, n, heads, d])."""
    B, Hq, Hkv, n, d = case["B"], case["Hq"], case["Hkv"], case["n"], case["d"]
    heads = Hq + 2 * Hkv
    x = torch.empty(B, n, heads, d, dtype=_TYPES[case["dtype"]], device="cuda")
    x = x if case["fused"] else x.view(B, heads, n, d).transpose(1, 2)
    means = _means(case, g)
    for h in range(heads):
        is_k = Hq <= h < Hq + Hkv
        x[:, :, h] = _key_rows(h - Hq, g, means, (B, n)) if is_k else torch.randn(B, n, d, generator=g, device="cuda")
    x = x.transpose(1, 2)
    parts = x.split([Hq, Hkv, Hkv], dim=1)
    s["q_new"], s["k_new"], s["v_new"] = parts if case["fused"] else [p.contiguous() for p in parts]


def _positions(case, s, g, first):
    """Coordinates [axes, B, n]: text on every axis alike, with grids of images in between where there are several axes; the plan of the
    turns; the norms' weights."""
    B, n, axes = case["B"], case["n"], len(_sections(case))
    at = first[:, None] + torch.arange(n, device="cuda")[None, :]
    coords = at.expand(axes, B, n).clone()
    if axes > 1:
        cell = torch.arange(n, device="cuda") % 1024
        image = (torch.arange(n, device="cuda") // 1024) % 2 == 1
        start = at - cell
        coords[0] = torch.where(image, start, coords[0])
        coords[1] = torch.where(image, start + cell // 32, coords[1])
        if axes > 2:
            coords[2] = torch.where(image, start + cell % 32, coords[2])
    s["coords"] = coords.to(torch.int32).contiguous()
    axis, freq = _pair_plan(case)
    s["axis"] = torch.tensor(axis, device="cuda")
    s["freq"] = torch.tensor(freq, dtype=torch.float64, device="cuda")
    normed = case["op"] == "norm" or case["norm"]
    for name in ("q_weight", "k_weight"):
        w = 1.0 + 0.2 * torch.randn(case["d"], generator=g, device="cuda")
        s[name] = w.to(_TYPES[case["dtype"]]) if normed else None
    if own:
        from paper_2505_02922_amd import binding as wb
        s["rotary"] = wb.wave_rotary_plan(case["rot"], case["base"], _sections(case), wb.WAVE_ROTARY_RUNS,
                                          wb.WAVE_ROTARY_HALVES if case["halves"] else wb.WAVE_ROTARY_NEIGHBOURS)


def _paged(case, s, g, rows, spare):
    """A paged cache as a serving loop holds it after a while: sequences' pages lie anywhere in the pool, the first `shared` pages of
    every sequence are the same, `spare` more tokens of every sequence find room.  rows: pages and tails hold rows that are read."""
    B, Hkv, d, T = case["B"], case["Hkv"], case["d"], case["page"]
    lengths = _lengths(case)
    whole = [n // T for n in lengths]
    room = [(n + spare) // T for n in lengths]
    most, shared = max(1, max(room)), case["shared"]
    pool = sum(room) + 1 + shared
    s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    column = torch.arange(most, device="cuda")[None, :]
    held = column < torch.tensor(whole, device="cuda")[:, None]
    place = torch.randperm(pool, generator=g, device="cuda")
    alone = held & (column >= shared)
    rank = (alone.flatten().cumsum(0).view(B, most) - 1 + shared).clamp(min=0)
    at = torch.where(alone, rank, column.expand(B, most).clamp(max=pool - 1))
    s["table"] = torch.where(held, place[at], -1).to(torch.int32)
    s["references"] = torch.zeros(pool + 1, dtype=torch.int32, device="cuda")
    s["references"] = s["references"].scatter_add(0, torch.where(held, place[at], pool).flatten(), held.flatten().to(torch.int32))[:pool].contiguous()
    s["k_codes"], s["v_codes"] = (torch.zeros(pool, Hkv, T, d, dtype=torch.int8, device="cuda") for _ in range(2))
    s["k_scales"], s["v_scales"] = (torch.zeros(pool, Hkv, device="cuda") for _ in range(2))
    s["k_tail"], s["v_tail"] = (torch.zeros(B, Hkv, T, d, dtype=_TYPES[case["dtype"]], device="cuda") for _ in range(2))
    means = _means(case, g)
    for h in range(Hkv):
        for name in ("k", "v"):
            make = (lambda lead: _key_rows(h, g, means, lead)) if name == "k" else (lambda lead: torch.randn(lead + (d,), generator=g, device="cuda"))
            s[name + "_tail"][:, h] = make((B, T))
            if rows:
                x = make((pool, T))
                top = x.abs().amax((1, 2))
                s[name + "_codes"][:, h] = torch.round(x * (127.0 / top)[:, None, None]).clamp(-127, 127).to(torch.int8)
                s[name + "_scales"][:, h] = top / 127.0
    s["means"] = means
    if own:
        from paper_2505_02922_amd import binding as wb
        s["pages"] = wb.pages_from_tensors(*(s[n] for n in _POOL + _OWN))


_POOL = ("k_codes", "v_codes", "k_scales", "v_scales")
_OWN = ("k_tail", "v_tail", "table", "lengths", "references")


def _beside(case, s, B):
    """Where the state after a call goes: arrays of its own beside the old state's (which stays good), pages in the same pool."""
    Hkv, d, T = case["Hkv"], case["d"], case["page"]
    s["to_k_tail"], s["to_v_tail"] = (torch.zeros(B, Hkv, T, d, dtype=_TYPES[case["dtype"]], device="cuda") for _ in range(2))
    s["to_table"] = torch.full((B, s["table"].shape[1]), -1, dtype=torch.int32, device="cuda")
    s["to_lengths"] = torch.zeros(B, dtype=torch.int32, device="cuda")
    s["to_references"] = torch.zeros_like(s["references"])
    if own:
        from paper_2505_02922_amd import binding as wb
        s["to"] = wb.pages_from_tensors(*(s[n] for n in _POOL), *(s["to_" + n] for n in _OWN))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, B, Hq, Hkv, d, op = _TYPES[case["dtype"]], case["B"], case["Hq"], case["Hkv"], case["d"], case["op"]
    s = {"case": case}
    if op == "norm":
        _projection(case, s, g)
        _positions(case, s, g, torch.randint(0, case["far"] - case["n"] + 1, (B,), generator=g, device="cuda"))
        s["q_out"], s["k_out"] = (torch.empty(B, h, case["n"], d, dtype=dt, device="cuda") for h in (Hq, Hkv))
        return s
    _paged(case, s, g, op in ("read", "attend"), case["n"] if op == "append" else 0)
    if op == "append":
        _projection(case, s, g)
        if _turns(case):
            _positions(case, s, g, s["lengths"].long())
            s["q_out"] = torch.zeros(B, Hq, case["n"], d, dtype=dt, device="cuda")
        s["counts"] = torch.tensor(_counts(case), dtype=torch.int32, device="cuda") if case["ragged"] else None
        _beside(case, s, B)
        s["first"] = s["lengths"] // case["page"] * case["page"]  # the first row of the page that the first new token goes into
    if op == "read":
        s["first"] = torch.tensor([max(n - case["n"], 0) // 2 for n in _lengths(case)], dtype=torch.int32, device="cuda")
    if op in ("append", "read"):
        n = _window(case)
        s["k_read"], s["v_read"] = (torch.zeros(B, Hkv, n, d, dtype=dt, device="cuda") for _ in range(2))
    if op == "attend":
        aim = s["means"][torch.arange(Hkv, device="cuda")[None, :, None], torch.randint(0, 64, (B, Hkv, Hq // Hkv), generator=g, device="cuda")]
        s["q"] = (aim + 0.5 * torch.randn(B, Hkv, Hq // Hkv, d, generator=g, device="cuda")).reshape(B, Hq, d).to(dt)
        s["out"], s["lse"] = torch.empty(B, Hq, d, device="cuda"), torch.empty(B, Hq, device="cuda")
    if op == "reorder":
        # one in eight ends, the others go on from a sequence that may be another's too
        parent = torch.randint(0, B, (case["to"],), generator=g, device="cuda")
        s["parent"] = torch.where(torch.rand(case["to"], generator=g, device="cuda") < 0.125, -1, parent).to(torch.int32)
        _beside(case, s, case["to"])
    if own and op in ("append", "attend"):  # the workspace that a serving loop keeps
        from paper_2505_02922_amd import binding as wb
        s["ws"] = wb.workspace(wb.wave_pages_append_workspace(s["pages"]) if op == "append" else wb.wave_pages_attention_workspace(s["pages"], Hq))
    return s


def _window(case):
    """Rows that are read: after an append the new tokens and what is in the page that the first of them goes into."""
    return case["n"] + case["page"] - 1 if case["op"] == "append" else case["n"]


# ---------------------------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if own:
        from paper_2505_02922_amd import binding as wb
        if case["op"] == "norm":
            return list(wb.wave_norm_rotary_apply(s["q_new"], s["k_new"], s["q_weight"], s["k_weight"], _EPS, coords=s["coords"], rotary=s["rotary"],
                                                  q_out=s["q_out"], k_out=s["k_out"]))
        if case["op"] == "append":
            if _turns(case):
                wb.wave_pages_append(s["pages"], s["k_new"], s["v_new"], q=s["q_new"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=_EPS,
                                     coords=s["coords"], rotary=s["rotary"], counts=s["counts"], q_out=s["q_out"], to=s["to"], ws=s["ws"])
            else:
                wb.wave_pages_append(s["pages"], s["k_new"], s["v_new"], counts=s["counts"], to=s["to"], ws=s["ws"])
            wb.wave_pages_read(s["to"], _window(case), first=s["first"], k_out=s["k_read"], v_out=s["v_read"])
            return [s["to_" + n] for n in _OWN] + [s["k_read"], s["v_read"]] + ([s["q_out"]] if _turns(case) else [])
        if case["op"] == "read":
            return list(wb.wave_pages_read(s["pages"], case["n"], first=s["first"], k_out=s["k_read"], v_out=s["v_read"]))
        if case["op"] == "attend":
            return list(wb.wave_pages_attention_decode(s["q"], s["pages"], out=s["out"], lse=s["lse"], ws=s["ws"]))
        wb.wave_pages_reorder(s["pages"], s["parent"], s["to"])
        return [s["to_" + n] for n in _OWN]
    return {"norm": _plain_norm, "append": _plain_append, "read": _plain_read, "attend": _plain_attend, "reorder": _plain_reorder}[case["op"]](s)


def _normed_and_turned(x, weight, s):
    """x [B, H, n, d], rounded once."""
    case, f = s["case"], x.float()
    if weight is not None:
        f = f * torch.rsqrt(f.square().mean(-1, keepdim=True) + _EPS) * weight.float()
    rot = case["rot"]
    angle = s["coords"][s["axis"]].permute(1, 2, 0).double() * s["freq"]  # [B, n, pairs]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if case["halves"]:
        a, b = f[..., :rot // 2], f[..., rot // 2:rot]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos, f[..., rot:]], -1)
    else:
        a, b = f[..., 0:rot:2], f[..., 1:rot:2]
        y = torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), f[..., rot:]], -1)
    return y.to(x.dtype)


def _plain_norm(s):
    return [_normed_and_turned(s["q_new"], s["q_weight"], s), _normed_and_turned(s["k_new"], s["k_weight"], s)]


def _window_rows(s, k, v, first_row, length):
    """The window [B, Hkv, n, d] of rows k, v [B, Hkv, rows, d], which begin with row first_row [B] of their sequences."""
    case = s["case"]
    t = torch.arange(_window(case), device="cuda")[None, :] + s["first"][:, None]
    live = (t < length[:, None])[:, None, :, None]
    at = (t - first_row[:, None]).clamp(0, k.shape[2] - 1)[:, None, :, None].expand(*s["k_read"].shape)
    return [torch.where(live, k.gather(2, at), s["k_read"]), torch.where(live, v.gather(2, at), s["v_read"])]


def _plain_append(s):
    case = s["case"]
    B, Hkv, d, n, T = case["B"], case["Hkv"], case["d"], case["n"], case["page"]
    outputs = []
    k, v = s["k_new"], s["v_new"]
    old = s["lengths"].long()
    count = torch.full_like(old, n) if s["counts"] is None else s["counts"].long()  # (the pool and the tables have room for all)
    if _turns(case):
        k = _normed_and_turned(k, s["k_weight"], s)
        q = _normed_and_turned(s["q_new"], s["q_weight"], s)
        outputs = [torch.where((torch.arange(n, device="cuda")[None, :] < count[:, None])[:, None, :, None], q, s["q_out"])]
    new = old + count
    # all rows of the pages that the new tokens touch
    touched = (T - 1 + n - 1) // T + 1
    page0, first = old // T, old // T * T
    at = torch.arange(touched * T, device="cuda")[None, :] + first[:, None]
    before = (at < old[:, None])[:, None, :, None]
    pick = (at - old[:, None]).clamp(0, n - 1)[:, None, :, None].expand(B, Hkv, touched * T, d)
    place = torch.arange(touched * T, device="cuda").clamp(max=T - 1)
    rows = [torch.where(before, tail[:, :, place], x.gather(2, pick)) for tail, x in ((s["k_tail"], k), (s["v_tail"], v))]
    # the complete ones take the lowest free pages, in the order of the sequences
    need = new // T - page0
    u = torch.arange(touched, device="cuda")[None, :]
    complete = u < need[:, None]
    pool = s["references"].shape[0]
    number = torch.arange(pool, device="cuda")
    free = torch.where(s["references"] <= 0, number, pool).sort().values
    ids = free[((need.cumsum(0) - need)[:, None] + u).clamp(max=pool - 1)]
    taken = torch.zeros(pool + 1, dtype=torch.bool, device="cuda").scatter(0, torch.where(complete, ids, pool).flatten(), True)[:pool]
    references = torch.where(taken, 1, s["references"])
    column = torch.arange(s["table"].shape[1], device="cuda")[None, :]
    mine = (column >= page0[:, None]) & (column < (page0 + need)[:, None])
    table = torch.where(mine, ids.gather(1, (column - page0[:, None]).clamp(0, touched - 1)).to(torch.int32), s["table"])
    values, tails = [], []
    rest = torch.arange(T, device="cuda")[None, :] + (need * T)[:, None]
    for name, x in zip(("k", "v"), rows):
        paged = x.float().view(B, Hkv, touched, T, d)
        top = paged.abs().amax((3, 4))
        codes = torch.round(paged * (127.0 / top.clamp(min=_LEAST))[..., None, None]).clamp(-127, 127)
        scale = torch.where(top < _LEAST, 0.0, top / 127.0)
        s[name + "_codes"][ids[complete]] = codes.to(torch.int8).transpose(1, 2)[complete]
        s[name + "_scales"][ids[complete]] = scale.transpose(1, 2)[complete]
        held = torch.where(complete[:, None, :, None, None], (codes * scale[..., None, None]).to(x.dtype), x.view(B, Hkv, touched, T, d))
        values.append(held.view(B, Hkv, touched * T, d))
        kept = x.gather(2, rest.clamp(max=touched * T - 1)[:, None, :, None].expand(B, Hkv, T, d))
        tails.append(torch.where((torch.arange(T, device="cuda")[None, :] < (new % T)[:, None])[:, None, :, None], kept, s["to_%s_tail" % name]))
    return tails + [table, new.to(torch.int32), references.to(torch.int32)] + _window_rows(s, *values, first, new) + outputs


def _values(s, name):
    """The rows of all pages of every sequence, in 32 bits: [B, Hkv, pages * T, d]."""
    case = s["case"]
    at = s["table"].long().clamp(min=0)
    x = s[name + "_codes"][at].float() * s[name + "_scales"][at][..., None, None]  # [B, pages, Hkv, T, d]
    return x.transpose(1, 2).reshape(case["B"], case["Hkv"], -1, case["d"])


def _plain_read(s):
    length, T = s["lengths"].long(), s["case"]["page"]
    N = s["table"].shape[1] * T
    t = torch.arange(N + T, device="cuda")[None, :]
    paged = t < (length // T * T)[:, None]
    at = torch.where(paged, t, N + t % T)[:, None, :, None].expand(s["case"]["B"], s["case"]["Hkv"], N + T, s["case"]["d"])
    k, v = (torch.cat([_values(s, x).to(s[x + "_tail"].dtype), s[x + "_tail"]], 2).gather(2, at) for x in ("k", "v"))
    return _window_rows(s, k, v, torch.zeros_like(length), length)


def _plain_attend(s):
    case = s["case"]
    B, Hkv, G, d, T = case["B"], case["Hkv"], case["Hq"] // case["Hkv"], case["d"], case["page"]
    length = s["lengths"].long()[:, None]
    k, v = (torch.cat([_values(s, x), s[x + "_tail"].float()], 2) for x in ("k", "v"))
    N = k.shape[2] - T
    t = torch.arange(N + T, device="cuda")[None, :]
    live = torch.where(t < N, t < length // T * T, t - N < length % T)[:, None]  # [B, 1, N + T]
    q = s["q"].float().reshape(B, Hkv, G, d)
    z = torch.matmul(k, q.transpose(-1, -2).contiguous()) / math.sqrt(d)  # [B, Hkv, N + T, G]
    z = torch.where(live[..., None], z, -math.inf)
    top = z.amax(2, keepdim=True)
    e = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(2, keepdim=True)
    p = torch.where(total > 0, e / total, 0.0).transpose(-1, -2).contiguous()
    out = torch.matmul(p, torch.where(live[..., None], v, 0.0))
    return [out.reshape(B, case["Hq"], d), (top + torch.log(total)).reshape(B, case["Hq"])]


def _plain_reorder(s):
    T, B = s["case"]["page"], s["case"]["B"]
    parent = s["parent"].long()
    lives = (parent >= 0) & (parent < B)
    source = parent.clamp(0, B - 1)
    length = torch.where(lives, s["lengths"].long()[source], 0)
    tails = [torch.where((torch.arange(T, device="cuda")[None, :] < (length % T)[:, None])[:, None, :, None], s[x][source], s["to_" + x])
             for x in ("k_tail", "v_tail")]
    column = torch.arange(s["table"].shape[1], device="cuda")[None, :]
    held = column < (length // T)[:, None]
    table = torch.where(held, s["table"][source], s["to_table"])
    before = column < (s["lengths"].long() // T)[:, None]
    pool = s["references"].shape[0]
    references = torch.cat([s["references"], s["references"].new_zeros(1)])
    for uses, entries, sign in ((held, table, 1), (before, s["table"], -1)):
        references = references.scatter_add(0, torch.where(uses, entries.long(), pool).flatten(), sign * uses.flatten().to(torch.int32))
    return tails + [table, length.to(torch.int32), references[:pool]]


# ---------------------------------------------------------------------------------------------------------------
# What a pass cannot do without, and its result in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    B, Hkv, Hq, d, op = case["B"], case["Hkv"], case["Hq"], case["d"], case["op"]
    if op == "norm":
        n = B * case["n"]
        return {"bytes": 2 * n * (Hq + Hkv) * d * es + 4 * n * len(_sections(case)), "flops": n * (Hq + Hkv) * (4 * d + 3 * case["rot"])}
    T, rows = case["page"], _lengths(case)
    row = 2 * Hkv * d  # keys and values of a token
    if op == "append":
        total, flops = 8 * B, 0
        for n, c in zip(rows, _counts(case)):
            old, new = n % T, (n + c) % T
            whole = (n + c) // T - n // T
            # new rows in; codes of the complete pages and the rows behind them out; rows that were there are read, the state's own lists too
            total += c * row * es + whole * (row * T + 8 * Hkv + 4) + (new + old) * row * es + 4 * 2 * (n // T) + 4 * whole
            seen = min(c + old, _window(case))  # read back
            total += seen * row * es + min(whole * T, seen) * row + max(seen - whole * T, 0) * row * es
            flops += 4 * (c + old) * row
            if _turns(case):
                total += 2 * c * Hq * d * es + 4 * c * len(_sections(case))
                flops += 3 * c * (Hq + Hkv) * case["rot"] + (4 * c * (Hq + Hkv) * d if case["norm"] else 0)
        return {"bytes": total, "flops": flops}
    if op == "read":
        total, flops = 8 * B, 0
        for n in rows:
            first = max(n - case["n"], 0) // 2
            seen = min(n - first, case["n"])
            paged = max(min(first + seen, n // T * T) - first, 0)
            total += seen * row * es + paged * row + (seen - paged) * row * es + (8 * Hkv + 4) * (-(-paged // T))
            flops += paged * row
        return {"bytes": total, "flops": flops}
    if op == "attend":
        whole = [n // T for n in rows]
        apart = sum(whole) - (B - 1) * case["shared"]
        return {"bytes": apart * (row * T + 8 * Hkv) + 4 * sum(whole) + sum(n % T for n in rows) * row * es + B * Hq * (d * (es + 4) + 4),
                "flops": 4 * Hq * sum(rows) * d}
    # (a mean: which sequences go on is the seed's)
    kept = 0.875 * case["to"] / B
    return {"bytes": int(sum(kept * (2 * (n % T) * row * es + 8 * (n // T)) + 4 * (n // T) for n in rows)) + 8 * (sum(n // T for n in rows) + B),
            "flops": 0}


def _exact_rows(x, weight, s, case):
    y, rot = x.double(), case["rot"]
    if weight is not None:
        y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / case["d"] + _EPS) * weight.double()
    z = y.clone()
    for i, (a, f) in enumerate(zip(*_pair_plan(case))):
        one, two = (i, i + rot // 2) if case["halves"] else (2 * i, 2 * i + 1)
        angle = s["coords"][a].double()[:, None] * f
        z[..., one] = y[..., one] * torch.cos(angle) - y[..., two] * torch.sin(angle)
        z[..., two] = y[..., two] * torch.cos(angle) + y[..., one] * torch.sin(angle)
    return z


def _exact_sequence(s, b, h, name):
    """A sequence's rows of one head, page by page."""
    T, n = s["case"]["page"], _lengths(s["case"])[b]
    at = s["table"][b, :n // T].long()
    pages = s[name + "_codes"][at, h].double() * s[name + "_scales"][at, h].double()[:, None, None]
    return torch.cat([pages.reshape(-1, s["case"]["d"]), s[name + "_tail"][b, h, :n % T].double()])


def exact(case, seed):
    s = prepare(case, seed)
    B, Hq, Hkv, d, op = case["B"], case["Hq"], case["Hkv"], case["d"], case["op"]
    if op == "norm":
        return [_exact_rows(s["q_new"], s["q_weight"], s, case), _exact_rows(s["k_new"], s["k_weight"], s, case)]
    lengths, T = _lengths(case), case["page"]
    if op == "read":
        out = [s["k_read"].double(), s["v_read"].double()]
        for b, n in enumerate(lengths):
            first = int(s["first"][b])
            last = min(n, first + case["n"])
            for h in range(Hkv):
                for o, name in zip(out, ("k", "v")):
                    o[b, h, :last - first] = _exact_sequence(s, b, h, name)[first:last]
        return out
    if op == "append":
        k, v = s["k_new"].double(), s["v_new"].double()
        if _turns(case):
            q, k = _exact_rows(s["q_new"], s["q_weight"], s, case), _exact_rows(k, s["k_weight"], s, case)
        tails = [s["to_k_tail"].double(), s["to_v_tail"].double()]
        read = [s["k_read"].double(), s["v_read"].double()]
        Q = s["q_out"].double() if _turns(case) else None
        for b, (n, c) in enumerate(zip(lengths, _counts(case))):
            if Q is not None:
                Q[b, :, :c] = q[b, :, :c]
            for i, (name, x) in enumerate((("k", k), ("v", v))):
                # rows are of the storage type before they are held in 8 bits
                x = torch.cat([s[name + "_tail"][b, :, :n % T], x[b, :, :c].to(_TYPES[case["dtype"]])], 1).double()
                whole = x.shape[1] // T
                paged = x[:, :whole * T].view(Hkv, whole, T, d)
                step = paged.abs().amax((2, 3), keepdim=True) / 127
                held = (torch.round(paged / step.clamp(min=1e-300)) * step).reshape(Hkv, whole * T, d)
                tails[i][b, :, :x.shape[1] - whole * T] = x[:, whole * T:]
                rows = torch.cat([held, x[:, whole * T:]], 1)[:, :_window(case)]
                read[i][b, :, :rows.shape[1]] = rows
        return tails + [None, None, None] + read + ([Q] if Q is not None else [])
    if op == "attend":
        G = Hq // Hkv
        out, lse = torch.zeros(B, Hq, d, dtype=torch.float64, device="cuda"), torch.zeros(B, Hq, dtype=torch.float64, device="cuda")
        for b in range(B):
            for h in range(Hkv):
                z = s["q"][b, h * G:(h + 1) * G].double() @ _exact_sequence(s, b, h, "k").T / math.sqrt(d)
                total = torch.logsumexp(z, -1)
                out[b, h * G:(h + 1) * G] = torch.exp(z - total[:, None]) @ _exact_sequence(s, b, h, "v")
                lse[b, h * G:(h + 1) * G] = total
        return [out, lse]
    tails = [s["to_k_tail"].double(), s["to_v_tail"].double()]
    for b, p in enumerate(s["parent"].tolist()):
        if 0 <= p < B:
            for to, name in zip(tails, ("k", "v")):
                to[b, :, :lengths[p] % T] = s[name + "_tail"][p, :, :lengths[p] % T].double()
    return tails + [None, None, None]
