"""Operators of the plain key/value cache, as cases that can be timed and compared: each pass is one call.

  rotary   `wave_rotary_apply`: rotary positions with one or several axes on a tensor of heads
  append   `wave_cache_append`: new tokens' keys and queries rotated, keys and values written behind each
           sequence's rows
  attend   `wave_cache_attention_decode`: one token's attention over a shared prefix and a sequence's own rows,
           with the weights that the own rows received added up
  evict    `wave_cache_evict`: the rows with the least accumulated weight leave, the rest close up

`run` has two forms of each: elementary torch operations in 32 bits (`own = False`), and the calls that a
program makes of `paper_2505_02922_amd.binding` (`own = True`).  `exact` is the definition in 64 bits.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}

# One transformer layer of the workloads the benchmark names; a case replaces what differs.
_LLAMA = dict(dtype="bf16", Hq=32, Hkv=8, d=128)
_QWEN = dict(dtype="bf16", Hq=28, Hkv=4, d=128)
_TINY = dict(dtype="f32", Hq=1, Hkv=1, d=64)

# Which pairs follow which axis: runs of pairs, pairs dealt out in turn, or runs with frequencies of their own.
RUNS, TURNS, LADDERS = 0, 1, 2


def listed():
    return [
        # The keys of a short fp32 sequence, text positions: nothing but a launch.
        dict(_TINY, name="rotary_f32_4k_b1", op="rotary", B=1, H=1, N=4096, rot=64, base=500000.0, sections="32",
             order=RUNS, halves=True, far=4096),
        # The query heads of a prompt of images and text before its index is built, positions along time, height
        # and width, far out.
        dict(_LLAMA, name="rotary_bf16_32k_b2_3axes", op="rotary", B=2, H=32, N=32749, rot=128, base=500000.0,
             sections="16,24,24", order=TURNS, halves=True, far=1048576),
        # Every decode step of a large batch: one token for each sequence.
        dict(_QWEN, name="append_bf16_token_b64", op="append", B=64, n=1, capacity=4352, short=1000, long=4351, ragged=False,
             rot=128, base=1000000.0, sections="64", order=RUNS, halves=True),
        # The prompts of four chats, padded to the longest, with images (three axes), into empty caches.
        dict(_LLAMA, name="append_bf16_prompt_b4_3axes", op="append", B=4, n=8191, capacity=9216, short=0, long=0, ragged=True,
             rot=128, base=500000.0, sections="16,24,24", order=RUNS, halves=True),
        # A few fp32 sequences behind a short shared prompt: the smallest call.
        dict(_TINY, name="prefix_f32_1k_b3", op="attend", B=3, Hq=8, Hkv=2, P=1021, capacity=256, short=1, long=200,
             decay=1.0, count=False),
        # Thirty-two chats behind one system prompt and documents of 32K tokens.
        dict(_LLAMA, name="prefix_bf16_32k_b32", op="attend", B=32, P=32768, capacity=1024, short=5, long=1021, decay=1.0, count=False),
        # A large batch on a model with seven queries per KV head, a 64K prefix, own rows kept at a budget: weights
        # are added up with a decay.
        dict(_QWEN, name="prefix_bf16_64k_b64_weights", op="attend", B=64, P=65519, capacity=4352, short=700, long=4352,
             decay=0.99, count=True),
        # A single short chat without a prefix: the interactive step.
        dict(_LLAMA, name="attend_bf16_1k_b1_weights", op="attend", B=1, P=0, capacity=2048, short=1000, long=1000, decay=1.0, count=True),
        # Eight long sequences of unlike lengths without a prefix.
        dict(_LLAMA, name="attend_bf16_64k_b8_weights", op="attend", B=8, P=0, capacity=65536, short=3001, long=65536, decay=1.0, count=True),
        # One row leaves each head's cache after every token.
        dict(_LLAMA, name="evict_bf16_one_b16", op="evict", B=16, capacity=2304, short=2049, long=2049, n_keep=2048, n_sink=4,
             n_local=256, apart=False),
        # A large batch's caches halve whenever they are full.
        dict(_QWEN, name="evict_bf16_half_b64", op="evict", B=64, capacity=4352, short=4100, long=4352, n_keep=2048, n_sink=4,
             n_local=1024, apart=False),
        # Two prompts of about 120K rows shrink to a cache of 16K rows of its own.
        dict(_LLAMA, name="evict_bf16_120k_b2", op="evict", B=2, capacity=122880, short=100003, long=122880, n_keep=16384, n_sink=4,
             n_local=1024, apart=True),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def plan(d):
        rot = rng.choice([r for r in (32, 64, 96, 128) if r <= d])
        axes = rng.randint(1, 3)
        cuts = sorted(rng.sample(range(1, rot // 2), axes - 1))
        sections = ",".join(str(b - a) for a, b in zip([0] + cuts, cuts + [rot // 2]))
        return dict(rot=rot, base=rng.choice([10000.0, 500000.0, 1000000.0]), sections=sections,
                    order=rng.choice([RUNS, TURNS, LADDERS]), halves=rng.random() < 0.7)

    Hkv = rng.choice([1, 2, 4, 8])
    case = dict(dtype="bf16" if rng.random() < 0.7 else "f32", Hkv=Hkv, Hq=Hkv * rng.randint(1, 8), d=rng.choice([64, 128, 128]))
    op = rng.choice(["rotary", "append", "attend", "attend", "evict"])
    B = log(1, 64)
    if op == "rotary":
        H = rng.randint(1, 32)
        N = log(1, max(2, (1 << 20) // (B * H)))
        return dict(case, op=op, B=B, H=H, N=N, far=log(N + 1, 1 << 20), **plan(case["d"]))
    if op == "append":
        n = 1 if rng.random() < 0.5 else log(2, max(3, 16384 // B))
        long = log(1, 4000)
        return dict(case, op=op, B=B, n=n, capacity=long + n + rng.randint(0, 300), short=rng.randint(0, long), long=long,
                    ragged=n > 1 and rng.random() < 0.5, **plan(case["d"]))
    if op == "attend":
        P = 0 if rng.random() < 0.3 else log(1, min(40000, 100000000 // (B * case["Hq"])))
        long = log(1, max(2, min(65536, 1000000 // (B * Hkv))))
        return dict(case, op=op, B=B, P=P, capacity=long + rng.randint(0, 100), short=rng.randint(0 if P else 1, long), long=long,
                    decay=rng.choice([1.0, 0.99, 0.5]), count=rng.random() < 0.6)
    long = log(16, max(17, min(122880, 1000000 // (B * Hkv))))
    n_keep = rng.randint(1, long)
    n_sink = rng.randint(0, min(4, n_keep))
    return dict(case, op=op, B=B, capacity=long + rng.randint(0, 100), short=rng.randint(1, long), long=long, n_keep=n_keep,
                n_sink=n_sink, n_local=rng.randint(0, (n_keep - n_sink) // 2), apart=rng.random() < 0.3)


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


def _sections(case):
    return [int(pairs) for pairs in case["sections"].split(",")]


def _pair_plan(case):
    """Axis and frequency (radians a position) of every rotated pair."""
    pairs, sections = case["rot"] // 2, _sections(case)
    if case["order"] == TURNS:
        left, axis = list(sections), []
        while len(axis) < pairs:
            for a in range(len(sections)):
                if left[a]:
                    left[a] -= 1
                    axis.append(a)
    else:
        axis = [a for a, s in enumerate(sections) for _ in range(s)]
    if case["order"] == LADDERS:
        freq = [case["base"] ** (-i / s) for s in sections for i in range(s)]
    else:
        freq = [case["base"] ** (-i / pairs) for i in range(pairs)]
    return axis, freq


def _means(case, g):
    return torch.randn(case["Hkv"], 64, case["d"], generator=g, device="cuda")


def _keys(case, g, means, lead, n):
    """Clusterable keys [*lead, Hkv, n, d]: a component's mean and noise."""
    dt = _TYPES[case["dtype"]]
    K = torch.empty(lead + (case["Hkv"], n, case["d"]), dtype=dt, device="cuda")
    for h in range(case["Hkv"]):
        comp = torch.randint(0, 64, lead + (n,), generator=g, device="cuda")
        x = means[h][comp]
        K[..., h, :, :] = x + 0.25 * torch.randn(x.shape, generator=g, device="cuda")
    return K


def _values(case, g, lead, n):
    V = torch.empty(lead + (case["Hkv"], n, case["d"]), dtype=_TYPES[case["dtype"]], device="cuda")
    for h in range(case["Hkv"]):
        V[..., h, :, :] = torch.randn(lead + (n, case["d"]), generator=g, device="cuda")
    return V


def _rotation(case, s):
    axis, freq = _pair_plan(case)
    s["axis"] = torch.tensor(axis, device="cuda")
    s["freq"] = torch.tensor(freq, dtype=torch.float64, device="cuda")
    if own:
        from paper_2505_02922_amd import binding as wb
        s["rotary"] = wb.wave_rotary_plan(case["rot"], case["base"], _sections(case), case["order"], 0 if case["halves"] else 1)


def _coordinates(case, g, first, n, far):
    """Positions [axes, B, n]: text on every axis alike, with grids of images in between where there are several axes."""
    B, axes = case["B"], len(_sections(case))
    at = first[:, None] + torch.arange(n, device="cuda")[None, :] + (max(far - n, 0) // 2)
    coords = at.expand(axes, B, n).clone()
    if axes > 1:
        cell = torch.arange(n, device="cuda") % 1024
        image = (torch.arange(n, device="cuda") // 1024) % 2 == 1
        start = at - cell
        coords[0] = torch.where(image, start, coords[0])
        coords[1] = torch.where(image, start + cell // 32, coords[1])
        if axes > 2:
            coords[2] = torch.where(image, start + cell % 32, coords[2])
    return coords.to(torch.int32).contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, B, Hkv, d = _TYPES[case["dtype"]], case["B"], case["Hkv"], case["d"]
    s = {"case": case}
    if case["op"] == "rotary":
        s["x"] = torch.empty(B, case["H"], case["N"], d, dtype=dt, device="cuda")
        for b in range(B):
            s["x"][b] = torch.randn(case["H"], case["N"], d, generator=g, device="cuda")
        first = torch.randint(0, max(case["far"] // 2, 1), (B,), generator=g, device="cuda")
        s["coords"] = _coordinates(case, g, first, case["N"], case["far"])
        s["out"] = torch.empty_like(s["x"])
        _rotation(case, s)
        return s
    cap = case["capacity"]
    s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
    s["tokens"] = s["lengths"] + torch.randint(0, 1000, (B,), generator=g, device="cuda", dtype=torch.int32)
    live = torch.arange(cap, device="cuda")[None, :] < s["lengths"][:, None]
    if case["op"] == "append":
        n = case["n"]
        s["k"], s["v"] = (torch.zeros(B, Hkv, cap, d, dtype=dt, device="cuda") for _ in range(2))
        s["positions"] = torch.full((B, Hkv, cap), -1, dtype=torch.int32, device="cuda")
        s["weights"] = torch.rand(B, Hkv, cap, generator=g, device="cuda")
        s["q_new"] = torch.randn(B, case["Hq"], n, d, generator=g, device="cuda").to(dt)
        s["k_new"] = _keys(case, g, _means(case, g), (B,), n)
        s["v_new"] = _values(case, g, (B,), n)
        s["coords"] = _coordinates(case, g, s["tokens"].long(), n, n)
        s["counts"] = torch.tensor(_counts(case), dtype=torch.int32, device="cuda") if case["ragged"] else None
        s["q_out"] = torch.zeros_like(s["q_new"])
        s["lengths_out"], s["tokens_out"] = torch.empty_like(s["lengths"]), torch.empty_like(s["tokens"])
        _rotation(case, s)
    else:
        means = _means(case, g)
        s["k"], s["v"] = _keys(case, g, means, (B,), cap), _values(case, g, (B,), cap)
        # Positions: the rows came in no order, as after earlier evictions (own to each head); the last ones are the newest.
        order = torch.rand(B, Hkv, cap, generator=g, device="cuda")
        order = torch.where(live[:, None], order, 2.0).argsort(-1).argsort(-1)
        newest = s["tokens"][:, None, None] - s["lengths"][:, None, None]
        s["positions"] = torch.where(live[:, None], order + newest, -1).to(torch.int32).contiguous()
        # Accumulated weights: a few rows hold most of the weight, some never got any.
        w = torch.exp(2.0 * torch.randn(B, Hkv, cap, generator=g, device="cuda") - 4.0)
        s["weights"] = torch.where(torch.rand(B, Hkv, cap, generator=g, device="cuda") < 0.02, 0.0, w)
    if case["op"] == "attend":
        G, P = case["Hq"] // Hkv, case["P"]
        comp = torch.randint(0, 64, (B, Hkv, G), generator=g, device="cuda")
        aim = means[torch.arange(Hkv, device="cuda")[None, :, None], comp]
        s["q"] = (aim + 0.5 * torch.randn(B, Hkv, G, d, generator=g, device="cuda")).reshape(B, case["Hq"], d).to(dt)
        s["prefix_k"], s["prefix_v"] = (_keys(case, g, means, (), P), _values(case, g, (), P)) if P else (None, None)
        s["out"] = torch.empty(B, case["Hq"], d, device="cuda")
        s["lse"] = torch.empty(B, case["Hq"], device="cuda")
        s["weights_out"] = torch.zeros_like(s["weights"]) if case["count"] else None
    if case["op"] == "evict":
        rows = min(case["n_keep"], cap)
        s["to_k"] = torch.zeros(B, Hkv, rows, d, dtype=dt, device="cuda") if case["apart"] else s["k"]
        s["to_v"] = torch.zeros_like(s["to_k"]) if case["apart"] else s["v"]
        small = (B, Hkv, rows if case["apart"] else cap)
        s["to_positions"] = torch.full(small, -1, dtype=torch.int32, device="cuda")
        s["to_weights"] = torch.zeros(small, device="cuda")
        s["to_lengths"], s["to_tokens"] = torch.empty_like(s["lengths"]), torch.empty_like(s["tokens"])
    if own:  # the handles and the workspace that a serving loop keeps
        from paper_2505_02922_amd import binding as wb
        s["cache"] = wb.cache_from_tensors(s["k"], s["v"], s["positions"], s["weights"], s["lengths"], s["tokens"])
        if case["op"] == "attend":
            s["ws"] = wb.workspace(wb.wave_cache_attention_workspace(s["cache"], case["Hq"], case["P"], case["count"]))
        if case["op"] == "evict":
            s["to"] = wb.cache_from_tensors(s["to_k"], s["to_v"], s["to_positions"], s["to_weights"], s["to_lengths"], s["to_tokens"])
            s["ws"] = wb.workspace(wb.wave_cache_evict_workspace(s["cache"], case["n_keep"]))
    return s


# ---------------------------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if own:
        from paper_2505_02922_amd import binding as wb
        if case["op"] == "rotary":
            return [wb.wave_rotary_apply(s["x"], s["coords"], s["rotary"], out=s["out"])]
        if case["op"] == "append":
            wb.wave_cache_append(s["cache"], s["k_new"], s["v_new"], q=s["q_new"], coords=s["coords"], rotary=s["rotary"],
                                 counts=s["counts"], q_out=s["q_out"], lengths_out=s["lengths_out"], tokens_out=s["tokens_out"])
            return [s[n] for n in ("q_out", "k", "v", "positions", "weights", "lengths_out", "tokens_out")]
        if case["op"] == "attend":
            wb.wave_cache_attention_decode(s["q"], s["cache"], s["prefix_k"], s["prefix_v"], decay=case["decay"],
                                           weights_out=s["weights_out"], out=s["out"], lse=s["lse"], ws=s["ws"])
            return [s["out"], s["lse"]] + ([s["weights_out"]] if case["count"] else [])
        wb.wave_cache_evict(s["cache"], case["n_keep"], case["n_sink"], case["n_local"], to=s["to"], ws=s["ws"])
        return [s["to_" + n] for n in ("k", "v", "positions", "weights", "lengths", "tokens")]
    return {"rotary": _plain_rotary, "append": _plain_append, "attend": _plain_attend, "evict": _plain_evict}[case["op"]](s)


def _turned(x, s):
    """x [B, H, n, d] rotated by the state's coordinates, rounded once."""
    case, d = s["case"], x.shape[-1]
    rot = case["rot"]
    angle = s["coords"][s["axis"]].permute(1, 2, 0).double() * s["freq"]  # [B, n, pairs]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    f = x.float()
    if case["halves"]:
        a, b = f[..., :rot // 2], f[..., rot // 2:rot]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos, f[..., rot:]], -1)
    else:
        a, b = f[..., 0:rot:2], f[..., 1:rot:2]
        y = torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), f[..., rot:]], -1)
    return y.to(x.dtype)


def _plain_rotary(s):
    return [_turned(s["x"], s)]


def _plain_append(s):
    case = s["case"]
    B, n, cap = case["B"], case["n"], case["capacity"]
    q, k = _turned(s["q_new"], s), _turned(s["k_new"], s)
    lengths, tokens = s["lengths"].long(), s["tokens"].long()
    if s["counts"] is None and n == 1:
        b = torch.arange(B, device="cuda")
        s["k"][b, :, lengths], s["v"][b, :, lengths] = k[:, :, 0], s["v_new"][:, :, 0]
        s["positions"][b, :, lengths] = s["tokens"][:, None].expand(B, case["Hkv"])
        s["weights"][b, :, lengths] = 0.0
        return [q, s["k"], s["v"], s["positions"], s["weights"], s["lengths"] + 1, s["tokens"] + 1]
    counts = torch.full_like(lengths, n) if s["counts"] is None else s["counts"].long()
    t = torch.arange(cap, device="cuda")[None, :] - lengths[:, None]
    new = (t >= 0) & (t < counts[:, None])
    at = t.clamp(0, n - 1)[:, None, :, None].expand(B, case["Hkv"], cap, case["d"])
    s["k"].copy_(torch.where(new[:, None, :, None], k.gather(2, at), s["k"]))
    s["v"].copy_(torch.where(new[:, None, :, None], s["v_new"].gather(2, at), s["v"]))
    s["positions"].copy_(torch.where(new[:, None], (tokens[:, None] + t)[:, None].to(torch.int32), s["positions"]))
    s["weights"].copy_(torch.where(new[:, None], 0.0, s["weights"]))
    held = torch.arange(n, device="cuda")[None, :] < counts[:, None]
    q = torch.where(held[:, None, :, None], q, s["q_out"])
    fit = torch.minimum(counts, cap - lengths).to(torch.int32)
    return [q, s["k"], s["v"], s["positions"], s["weights"], s["lengths"] + fit, s["tokens"] + fit]


def _plain_attend(s):
    case = s["case"]
    B, Hkv, G, d, P, cap = case["B"], case["Hkv"], case["Hq"] // case["Hkv"], case["d"], case["P"], case["capacity"]
    live = (torch.arange(cap, device="cuda")[None, :] < s["lengths"][:, None])[:, None, None]  # [B, 1, 1, cap]
    q = s["q"].float().reshape(B, Hkv, G, d)
    z = torch.matmul(q, s["k"].float().transpose(-1, -2)) / math.sqrt(d)
    z = torch.where(live, z, -math.inf)
    if P:
        shared = q.transpose(0, 1).reshape(Hkv, B * G, d)
        zp = torch.matmul(shared, s["prefix_k"].float().transpose(-1, -2)) / math.sqrt(d)
        z = torch.cat([zp.reshape(Hkv, B, G, P).transpose(0, 1), z], -1)
    top = z.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(z - top)
    total = e.sum(-1, keepdim=True)
    p = torch.where(total > 0, e / total, 0.0)
    v = torch.where(live[:, :, 0, :, None], s["v"].float(), 0.0)
    out = torch.matmul(p[..., P:], v)
    if P:
        pp = p[..., :P].transpose(0, 1).reshape(Hkv, B * G, P)
        out = out + torch.matmul(pp, s["prefix_v"].float()).reshape(Hkv, B, G, d).transpose(0, 1)
    outputs = [out.reshape(B, case["Hq"], d), (top + torch.log(total)).reshape(B, case["Hq"])]
    if case["count"]:
        w = case["decay"] * s["weights"] + p[..., P:].sum(2)
        outputs.append(torch.where(live[:, :, 0], w, s["weights_out"]))
    return outputs


def _plain_evict(s):
    case = s["case"]
    cap = case["capacity"]
    row = torch.arange(cap, device="cuda").expand(case["B"], case["Hkv"], cap)
    length, tokens = s["lengths"].long()[:, None, None], s["tokens"].long()[:, None, None]
    after = length.clamp(max=case["n_keep"])
    held = (s["positions"] < case["n_sink"]) | (s["positions"] >= tokens - case["n_local"])
    key = torch.where(held, math.inf, s["weights"])
    key = torch.where(row < length, key, -math.inf)
    best = torch.sort(key, dim=-1, descending=True, stable=True).indices
    kept = torch.zeros_like(row, dtype=torch.bool).scatter(-1, best, row < after)
    hole, mover = ~kept & (row < after), kept & (row >= after)
    # the i-th mover's row at entry i, then every hole reads the entry of its own rank
    ranked = torch.zeros(case["B"], case["Hkv"], cap + 1, dtype=torch.long, device="cuda")
    ranked = ranked.scatter(-1, torch.where(mover, mover.long().cumsum(-1) - 1, cap), row)
    source = torch.where(hole, ranked.gather(-1, (hole.long().cumsum(-1) - 1).clamp(min=0)), row)
    rows = s["to_k"].shape[2]
    fill = (row < after)[..., :rows]
    source = source[..., :rows]
    outputs = []
    for name in ("k", "v"):
        moved = s[name].gather(2, source[..., None].expand(*source.shape, case["d"]))
        outputs.append(torch.where(fill[..., None], moved, s["to_" + name]))
    rows = s["to_weights"].shape[2]
    for name in ("positions", "weights"):
        outputs.append(torch.where(fill, s[name].gather(2, source), s["to_" + name]))
    return outputs + [s["lengths"].clamp(max=case["n_keep"]), s["tokens"].clone()]


# ---------------------------------------------------------------------------------------------------------------
# What a pass cannot do without, and its result in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    B, Hkv, Hq, d = case["B"], case["Hkv"], case["Hq"], case["d"]
    if case["op"] == "rotary":
        n = B * case["N"]
        return {"bytes": 2 * n * case["H"] * d * es + 4 * n * len(_sections(case)), "flops": 3 * n * case["H"] * case["rot"]}
    if case["op"] == "append":
        n = sum(_counts(case))
        return {"bytes": n * (2 * (Hq + 2 * Hkv) * d * es + 4 * len(_sections(case)) + 8 * Hkv) + 16 * B, "flops": 3 * n * (Hq + Hkv) * case["rot"]}
    rows = _lengths(case)
    if case["op"] == "attend":
        seen = sum(rows) + B * case["P"]
        return {"bytes": 2 * Hkv * (case["P"] + sum(rows)) * d * es + B * Hq * (d * (es + 4) + 4) + (8 * Hkv * sum(rows) if case["count"] else 0),
                "flops": 4 * Hq * seen * d}
    total = 16 * B
    for n in rows:
        keep = min(n, case["n_keep"])
        # rows written: all that stay where there is a new place for them, else the holes below the budget
        moved = keep if case["apart"] else keep * (n - keep) / n
        total += Hkv * (8 * n + 8 * keep + 4 * moved * d * es)
    return {"bytes": int(total), "flops": 0}


def _exact_rotation(x, s, case):
    axis, freq = _pair_plan(case)
    y, rot = x.double(), case["rot"]
    for i, (a, f) in enumerate(zip(axis, freq)):
        one, two = (i, i + rot // 2) if case["halves"] else (2 * i, 2 * i + 1)
        angle = s["coords"][a].double()[:, None] * f
        u, w = x[..., one].double(), x[..., two].double()
        y[..., one] = u * torch.cos(angle) - w * torch.sin(angle)
        y[..., two] = w * torch.cos(angle) + u * torch.sin(angle)
    return y


def exact(case, seed):
    s = prepare(case, seed)
    B, Hkv, d = case["B"], case["Hkv"], case["d"]
    if case["op"] == "rotary":
        return [_exact_rotation(s["x"], s, case)]
    lengths = _lengths(case)
    if case["op"] == "append":
        q, k = _exact_rotation(s["q_new"], s, case), _exact_rotation(s["k_new"], s, case)
        K, V, Q = s["k"].double(), s["v"].double(), s["q_out"].double()
        for b, (n, c) in enumerate(zip(lengths, _counts(case))):
            Q[b, :, :c] = q[b, :, :c]
            c = min(c, case["capacity"] - n)
            K[b, :, n:n + c], V[b, :, n:n + c] = k[b, :, :c], s["v_new"][b, :, :c].double()
        return [Q, K, V, None, None, None, None]
    if case["op"] == "attend":
        G, P = case["Hq"] // Hkv, case["P"]
        out, lse = torch.empty(B, case["Hq"], d, dtype=torch.float64, device="cuda"), torch.empty(B, case["Hq"], dtype=torch.float64, device="cuda")
        w = s["weights_out"].double() if case["count"] else None
        for h in range(Hkv):
            pk, pv = (s["prefix_k"][h].double(), s["prefix_v"][h].double()) if P else (None, None)
            for b, n in enumerate(lengths):
                kk, vv = s["k"][b, h, :n].double(), s["v"][b, h, :n].double()
                if P:
                    kk, vv = torch.cat([pk, kk]), torch.cat([pv, vv])
                z = s["q"][b, h * G:(h + 1) * G].double() @ kk.T / math.sqrt(d)
                total = torch.logsumexp(z, -1)
                p = torch.exp(z - total[:, None])
                out[b, h * G:(h + 1) * G], lse[b, h * G:(h + 1) * G] = p @ vv, total
                if case["count"]:
                    w[b, h, :n] = case["decay"] * s["weights"][b, h, :n].double() + p[:, P:].sum(0)
        return [out, lse] + ([w] if case["count"] else [])
    return None
