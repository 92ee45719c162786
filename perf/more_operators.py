"""A cache of bounded length, as timed cases: rotation, windows, accumulated weights, eviction.

Six kinds of pass, one attention layer each, through the public binding:

  rotate       the newest tokens' query and key heads are normed and turned by their positions; keys and values go into the cache
               (`lfps_rotate_append`).
  window       causal attention of the newest tokens over a sliding window and the first rows (`lfps_window_attn`).
  window_step  the same of one decode step (`lfps_window_attn_decode`).
  mass         the attention weights that the newest tokens give every row, added up (`lfps_attn_mass`).
  mass_step    one decode step's full attention, which adds its weights up too (`lfps_full_attn_mass_decode`).
  evict        every KV head keeps its first rows, its newest and those of the largest accumulated weight, moved to the front
               (`lfps_evict`), in place or into other blocks.

A case says the shapes: B requests; each brings T_lo..T_hi new tokens behind P_lo..P_hi rows that the cache holds (steps and
evict: P_lo..P_hi rows in all); Hq query heads over Hkv KV heads of 128 channels; the cache format (f32 / bf16 / f16 / fp8kv =
FP8 keys and values beside bf16 queries) and layout (page = rows per block, 0 = contiguous); lens_seed, from which the lengths
inside the ranges come.
"""
import random

import torch

own = False

D = 128
DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "fp8kv": torch.bfloat16}
EPS = 1e-6

BASE = {"kind": "rotate", "B": 1, "T_lo": 1, "T_hi": 1, "P_lo": 0, "P_hi": 0, "Hq": 32, "Hkv": 8, "dtype": "bf16", "page": 0,
        "lens_seed": 1,
        # rotate: channels turned, axes of a position, pairing, norms, type of the queries handed on, distance of the first position
        "rot": 128, "axes": 1, "interleaved": False, "norm": True, "q_f32": False, "pos_off": 0,
        # window, evict: rows behind a token that it sees (its own among them), first rows that stay, newest rows that stay
        "window": 0, "sink": 0, "recent": 0,
        # mass: what is left of earlier weights; evict: per cent of its rows that a request may keep, and where they go
        "decay": 1.0, "keep_lo": 0, "keep_hi": 0, "in_place": True}


def _case(name, **kw):
    return dict(BASE, name=name, **kw)


def listed():
    return [
        # One token of every request of a decoding batch, into FP8 pages; queries in 32 bits, as the decode steps take them.
        _case("rotate_b32_1_fp8kv_paged", B=32, P_lo=100, P_hi=9000, dtype="fp8kv", page=16, q_f32=True),
        # A packed batch of prompts with pictures in them: positions of three axes.
        _case("rotate_b8_ragged_3axes_bf16_paged", B=8, T_lo=1000, T_hi=6000, P_hi=300, axes=3, page=16, lens_seed=6),
        # Two long chunks far into their contexts, half of the channels turned, neighbouring channels paired, no norms.
        _case("rotate_b2_partial_f16", B=2, T_lo=5000, T_hi=8191, rot=64, interleaved=True, norm=False, dtype="f16", pos_off=1000003, lens_seed=4),
        # Five drafted tokens of one request in a layer with a window of a thousand rows: latency.
        _case("window_b1_5_of_4k_paged", kind="window", T_lo=5, T_hi=5, P_lo=4099, P_hi=4099, window=1024, sink=4, page=16),
        # One long prompt in such a layer.
        _case("window_b1_16k_w1024_bf16", kind="window", T_lo=16384, T_hi=16384, window=1024, sink=4),
        # Chunks of ragged prompts behind rows that are cached, an odd window, fp16.
        _case("window_b6_ragged_f16_paged", kind="window", B=6, T_lo=100, T_hi=4000, P_hi=4000, Hq=16, dtype="f16", page=64, window=517, sink=37,
              lens_seed=7),
        # A decoding batch over long contexts, serving cache.
        _case("window_step_b32_w4096_fp8kv_paged", kind="window_step", B=32, P_lo=3000, P_hi=20000, window=4096, sink=4, dtype="fp8kv", page=16,
              lens_seed=5),
        # The last tokens of a long prompt say which of its rows matter.
        _case("mass_b1_32_of_32k_bf16", kind="mass", T_lo=32, T_hi=32, P_lo=32736, P_hi=32736),
        # Every token of a prompt of some length says so, over FP8 pages.
        _case("mass_b2_8k_fp8kv_paged", kind="mass", B=2, T_lo=3500, T_hi=8192, dtype="fp8kv", page=16, decay=0.95, lens_seed=3),
        # A decode step of a batch that keeps accounts.
        _case("mass_step_b16_32k_bf16_paged", kind="mass_step", B=16, P_lo=2000, P_hi=32768, page=16, lens_seed=9),
        # One long context is cut to a quarter, in place.
        _case("evict_b1_32k_bf16", kind="evict", P_lo=32768, P_hi=32768, keep_lo=25, keep_hi=25, sink=4, recent=512),
        # A batch is cut to about half, into other pages.
        _case("evict_b32_ragged_fp8kv_paged", kind="evict", B=32, P_lo=300, P_hi=9000, keep_lo=30, keep_hi=110, sink=4, recent=200, dtype="fp8kv",
              page=16, in_place=False, lens_seed=8),
    ]


def _spread(rng, lo, hi):
    """A whole number in [lo, hi], over the logarithm."""
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    """A case of the listed ranges that costs no more than the largest listed one."""
    while True:
        kind = rng.choice(["rotate", "rotate", "window", "window", "window_step", "mass", "mass_step", "evict"])
        hkv = rng.choice([1, 2, 4, 8, 8])
        c = dict(BASE, kind=kind, Hkv=hkv, Hq=hkv * rng.choice([1, 2, 4, 4]), lens_seed=rng.randrange(1 << 30),
                 dtype=rng.choice(["bf16", "bf16", "f16", "fp8kv", "f32"]), page=rng.choice([0, 16, 64, 256]))
        c["B"] = _spread(rng, 1, 32)
        if kind in ("rotate", "window", "mass"):
            c["T_hi"] = _spread(rng, 1, 8192 if kind == "rotate" else 16384)
            c["T_lo"] = _spread(rng, 1, c["T_hi"])
            c["P_hi"] = _spread(rng, 1, 32768) if rng.random() < 0.6 else 0
            c["P_lo"] = c["P_hi"] // 3
        else:
            c["P_hi"] = _spread(rng, 300, 32768)
            c["P_lo"] = c["P_hi"] // 4
        if kind == "rotate":
            c.update(rot=16 * rng.randint(1, 8), axes=rng.choice([1, 1, 3]), interleaved=rng.random() < 0.3, norm=rng.random() < 0.7,
                     q_f32=rng.random() < 0.3, pos_off=_spread(rng, 1, 2000000))
        if kind in ("window", "window_step"):
            c.update(window=_spread(rng, 1, 8192), sink=rng.choice([0, 1, 4, _spread(rng, 1, 300)]))
        if kind == "mass":
            c["decay"] = rng.choice([1.0, 0.95, 0.5])
        if kind == "evict":
            c.update(keep_lo=rng.randint(1, 60), keep_hi=rng.randint(60, 110), sink=rng.choice([0, 4, 64]), recent=_spread(rng, 1, 1000),
                     in_place=rng.random() < 0.5)
        w = work(c)
        rows = c["B"] * (c["T_hi"] + c["P_hi"]) * hkv
        padded = c["B"] * c["T_hi"] * (c["T_hi"] + c["P_hi"]) * c["Hq"] if kind in ("window", "mass") else 0
        if w["flops"] <= 2.7e11 and padded <= 8.5e9 and w["bytes"] <= 2.0e9 and rows <= 4_200_000 and \
                (c["dtype"] != "f32" or w["flops"] <= 1.0e11):
            return c


# ---------------------------------------------------------------- shapes and work

def _lens(case):
    """Per request: new tokens, rows held before them."""
    r = random.Random(case["lens_seed"])
    new = [r.randint(case["T_lo"], case["T_hi"]) for _ in range(case["B"])]
    if case["kind"] in ("window_step", "mass_step", "evict"):
        new = [0] * case["B"]
    return new, [r.randint(case["P_lo"], case["P_hi"]) for _ in range(case["B"])]


def _budgets(case):
    r = random.Random(case["lens_seed"] + 1)
    return [max(1, h * r.randint(case["keep_lo"], case["keep_hi"]) // 100) for h in _lens(case)[1]]


def _seen_of_step(case, n):
    return min(n, case["window"] + case["sink"])


def _seen(case, t, h):
    """Pairs of t new tokens behind h rows and rows that these see; rows that any of them sees."""
    n = t + h
    if case["kind"] == "mass":
        return t * h + t * (t + 1) // 2, n
    w, s = case["window"], case["sink"]
    edge = max(0, h + 1 - w)                                          # the first token's window begins there
    return sum(min(p + 1, w) + min(s, max(0, p + 1 - w)) for p in range(h, n)), n - edge + min(s, edge)


def work(case):
    new, held = _lens(case)
    kind, f32 = case["kind"], case["dtype"] == "f32"
    row = 2 * case["Hkv"] * D * {"f32": 4, "fp8kv": 1}.get(case["dtype"], 2)
    token = D * (4 if f32 else 2)
    Hq, Hkv, B = case["Hq"], case["Hkv"], case["B"]
    if kind == "rotate":
        each = (Hq + 2 * Hkv) * token + Hq * D * (4 if case["q_f32"] or f32 else 2) + row + 4 * case["axes"]
        return {"bytes": sum(new) * each, "flops": 10 * sum(new) * (Hq + Hkv) * D}
    if kind == "window":
        both = [_seen(case, t, h) for t, h in zip(new, held)]
        return {"bytes": 2 * sum(new) * Hq * token + sum(x[1] for x in both) * row, "flops": 4 * D * Hq * sum(x[0] for x in both)}
    if kind == "window_step":
        rows = sum(_seen_of_step(case, n) for n in held)
        return {"bytes": rows * row + 2 * B * Hq * D * 4, "flops": 4 * D * Hq * rows}
    if kind == "mass":
        both = [_seen(case, t, h) for t, h in zip(new, held)]
        return {"bytes": sum(new) * Hq * token + sum(x[1] for x in both) * (row // 2 + 4 * Hkv) + sum(held) * 4 * Hkv,
                "flops": 2 * D * Hq * sum(x[0] for x in both)}
    if kind == "mass_step":
        return {"bytes": sum(held) * (row + 8 * Hkv) + 2 * B * Hq * D * 4, "flops": 4 * D * Hq * sum(held)}
    kept = [min(h, m) for h, m in zip(held, _budgets(case))]
    moved = [max(0, m - case["sink"]) if case["in_place"] and m < h else (0 if case["in_place"] else m) for h, m in zip(held, kept)]
    return {"bytes": 4 * Hkv * (sum(held) + 2 * sum(kept)) + 2 * sum(moved) * row, "flops": 0}


# ---------------------------------------------------------------- inputs

def _cache_dtype(case):
    return torch.float8_e4m3fn if case["dtype"] == "fp8kv" else DTYPES[case["dtype"]]


def _to_cache(x, dt):
    return x.clamp(-448.0, 448.0).to(dt) if dt == torch.float8_e4m3fn else x.to(dt)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, device=DEV, generator=gen)  # noqa: E731
    B, Hq, Hkv, page, kind = case["B"], case["Hq"], case["Hkv"], case["page"], case["kind"]
    dt, cdt = DTYPES[case["dtype"]], _cache_dtype(case)
    new, held = _lens(case)
    s = {"case": case}
    lens = [t + h for t, h in zip(new, held)]
    s["lens"], s["cap"], s["T"] = _ints(lens), max(1, max(lens)), sum(new)
    # Queries lean towards a direction of their KV head, and so do the first four rows' keys (attention sinks).
    lean = normal(Hkv, 1, D)

    def tables(spare):
        per = -(-s["cap"] // page)
        n_blocks = B * per + spare
        return torch.randperm(n_blocks, device=DEV, generator=gen)[:B * per].view(B, per).to(torch.int32).contiguous(), (n_blocks, Hkv, page, D)

    if page:
        s["table"], shape = tables(7)
    else:
        shape = (B, Hkv, s["cap"], D)
    if kind == "rotate":
        s["K"], s["V"] = (torch.zeros(shape, device=DEV).to(cdt) for _ in range(2))
    else:
        k = normal(*shape)
        if page:
            first = torch.zeros((shape[0], 1, page, 1), device=DEV)
            first[s["table"][:, 0].long(), :, :min(4, page)] = 1.0
        else:
            first = torch.zeros((B, 1, s["cap"], 1), device=DEV)
            first[:, :, :4] = 1.0
        k += 0.8 * first * lean
        s["K"], s["V"] = _to_cache(k, cdt), _to_cache(normal(*shape), cdt)
        del k
    at = [0]
    for t in new:
        at.append(at[-1] + t)
    s["cu"], s["at"], s["T_max"] = _ints(at), at, max(new)
    if kind in ("rotate", "window", "mass"):
        qkv = normal(s["T"], Hq + 2 * Hkv, D)
        if kind == "rotate":
            qkv *= 0.1 + 3.0 * torch.rand((s["T"], Hq + 2 * Hkv, 1), device=DEV, generator=gen)      # heads of unlike size, as a projection leaves them
            if case["dtype"] == "fp8kv":
                qkv[:, Hq + Hkv:] *= 1.0 + 200.0 * (torch.rand((s["T"], Hkv, 1), device=DEV, generator=gen) < 0.01)      # outlier rows: FP8 saturates
        else:
            qkv[:, :Hq] = 0.8 * qkv[:, :Hq] + 0.6 * lean.view(1, Hkv, 1, D).expand(s["T"], Hkv, Hq // Hkv, D).reshape(s["T"], Hq, D)
        s["qkv"] = qkv.to(dt)                         # the layer's fused projection; q, k and v are slices of it
        del qkv
        s["q"], s["k_new"], s["v_new"] = s["qkv"].split([Hq, Hkv, Hkv], dim=1)
    if kind in ("window_step", "mass_step"):
        s["q"] = 0.8 * normal(B, Hq, D) + 0.6 * lean.expand(Hkv, Hq // Hkv, D).reshape(1, Hq, D)
        s["out"] = torch.zeros((B, Hq, D), device=DEV)
    if kind == "window":
        s["out"] = torch.zeros((s["T"], Hq, D), dtype=dt, device=DEV)
    if kind == "rotate":
        half = case["rot"] // 2
        s["q_out"] = torch.zeros((s["T"], Hq, D), dtype=torch.float32 if case["q_f32"] else dt, device=DEV)
        s["q_weight"], s["k_weight"] = (1.0 + 0.2 * normal(D) if case["norm"] else None for _ in range(2))
        s["inv_freq"] = torch.tensor([1e6 ** (-i / half) for i in range(half)], device=DEV)
        place = torch.cat([torch.arange(h, h + t) for t, h in zip(new, held)]) + case["pos_off"]
        if case["axes"] == 1:
            s["positions"], s["pair_axis"] = place.to(torch.int32).to(DEV).view(1, -1), None
        else:                                         # pictures of 16 x 16 patches: one time, rows, columns
            base = place - place % 256
            s["positions"] = torch.stack([base, base + place % 256 // 16, base + place % 16]).to(torch.int32).to(DEV)
            s["pair_axis"] = _ints([0 if 4 * i < half else (1 if 8 * i < 5 * half else 2) for i in range(half)])
    if kind in ("mass", "mass_step", "evict"):
        mass = torch.exp(2.0 * normal(B, Hkv, s["cap"]) - 4.0)
        mass[:, :, :4] += 100.0
        mass *= torch.rand(mass.shape, device=DEV, generator=gen) > 0.05           # rows that nobody has looked at: ties
        s["mass"] = mass
        s["held"] = _ints([n - 1 for n in lens] if kind == "mass_step" else held)
    if kind == "evict":
        s["budget"] = _ints(_budgets(case))
        s["mass_out"], s["lens_out"] = torch.zeros_like(s["mass"]), torch.zeros_like(s["lens"])
        s["kept"] = torch.zeros((B, Hkv, s["cap"]), dtype=torch.int32, device=DEV)
        s["K_to"], s["V_to"], s["table_to"] = s["K"], s["V"], s.get("table")
        if not case["in_place"]:
            if page:
                s["table_to"], shape = tables(3)
            s["K_to"], s["V_to"] = (torch.zeros(shape, device=DEV).to(cdt) for _ in range(2))
    if own:
        from paper_2506_15704_amd.binding import Lfps
        ctx = Lfps(batch=B, n_q_heads=Hq, n_kv_heads=Hkv, kv_dtype="bf16" if case["dtype"] == "fp8kv" else case["dtype"],
                   max_seq_len=s["cap"], max_k=1, radius=1, k_fp8=case["dtype"] == "fp8kv", v_fp8=case["dtype"] == "fp8kv")
        s["ctx"] = ctx
        s["kv"] = ctx.paged_kv_view(s["K"], s["V"], s["table"], s["lens"]) if page else ctx.kv_view(s["K"], s["V"], s["lens"])
        if kind == "rotate":
            s["rotary"] = ctx.rotary(inv_freq=s["inv_freq"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS,
                                     pair_axis=s["pair_axis"], n_axes=case["axes"], interleaved=case["interleaved"])
        if kind == "evict" and not case["in_place"]:
            s["to"] = (ctx.paged_kv_view(s["K_to"], s["V_to"], s["table_to"], s["lens_out"]) if page
                       else ctx.kv_view(s["K_to"], s["V_to"], s["lens_out"]))
    return s


# ---------------------------------------------------------------- the pass

def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        ctx = s["ctx"]
        if kind == "rotate":
            ctx.lfps_rotate_append(s["rotary"], s["q"], s["k_new"], s["v_new"], s["positions"], s["cu"], s["kv"], s["q_out"])
        elif kind == "window":
            ctx.lfps_window_attn(s["q"], s["cu"], s["kv"], case["window"], case["sink"], s["out"])
        elif kind == "window_step":
            ctx.lfps_window_attn_decode(s["q"], s["kv"], case["window"], case["sink"], s["out"])
        elif kind == "mass":
            ctx.lfps_attn_mass(s["q"], s["cu"], s["kv"], s["mass"], held=s["held"], decay=case["decay"])
        elif kind == "mass_step":
            ctx.lfps_full_attn_mass_decode(s["q"], s["kv"], s["mass"], s["out"], held=s["held"], decay=case["decay"])
        else:
            ctx.lfps_evict(s["kv"], s["mass"], s["budget"], case["sink"], case["recent"], s["mass_out"], s["kept"], s["lens_out"], to=s.get("to"))
    else:
        {"rotate": _rotate, "window": _window, "window_step": _window_step, "mass": _mass, "mass_step": _mass_step, "evict": _evict}[kind](s)
    if kind == "rotate":
        return {"q": s["q_out"], "K": s["K"], "V": s["V"]}
    if kind in ("window", "window_step"):
        return s["out"]
    if kind == "mass":
        return s["mass"]
    if kind == "mass_step":
        return {"out": s["out"], "mass": s["mass"]}
    return {"K": s["K_to"], "V": s["V_to"], "mass": s["mass_out"], "kept": s["kept"], "lens": s["lens_out"]}


def _bytes(x):
    return x.view(torch.uint8) if x.element_size() == 1 else x


def _tokens(s):
    """Of every packed token: its request, its place among that one's new ones, its row."""
    cu = s["cu"].long()
    t = torch.arange(s["T"], device=DEV)
    b = torch.searchsorted(cu[1:], t, right=True)
    return b, t - cu[b], s["lens"].long()[b] - (cu[b + 1] - t)


def _place(s, b, row, table="table"):
    page = s["case"]["page"]
    return (s[table].long()[b, row // page], row % page) if page else (b, row)


def _rotate(s):
    case = s["case"]
    half, R = case["rot"] // 2, case["rot"]
    b, _, row = _tokens(s)
    pos = s["positions"].double()
    of_pair = pos[s["pair_axis"].long()] if s["pair_axis"] is not None else pos.expand(half, -1)
    angle = (of_pair * s["inv_freq"].double().view(-1, 1)).t()               # [T, half]
    cos, sin = angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)
    first, second = (slice(0, R, 2), slice(1, R, 2)) if case["interleaved"] else (slice(0, half), slice(half, R))

    def turned(x, weight):
        y = x.float()
        if weight is not None:
            y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * weight
        z = y.clone()
        z[..., first] = y[..., first] * cos - y[..., second] * sin
        z[..., second] = y[..., second] * cos + y[..., first] * sin
        return z

    s["q_out"].copy_(turned(s["q"], s["q_weight"]))
    block, at = _place(s, b, row)
    _bytes(s["K"])[block, :, at] = _bytes(_to_cache(turned(s["k_new"], s["k_weight"]), s["K"].dtype))
    _bytes(s["V"])[block, :, at] = _bytes(_to_cache(s["v_new"].float(), s["V"].dtype))


def _rows(s, name, i):
    """Rows i [B, N] of the requests' K or V, [B, Hkv, N, D] fp32."""
    b = torch.arange(i.shape[0], device=DEV).view(-1, 1).expand_as(i)
    block, at = _place(s, b, i)
    x = _bytes(s[name])[block, :, at]                   # [B, N, Hkv, D]
    x = x.view(s[name].dtype) if x.dtype == torch.uint8 else x
    return x.float().transpose(1, 2).contiguous()


def _all_rows(s, name):
    return _rows(s, name, torch.arange(s["cap"], device=DEV).expand(s["case"]["B"], -1))


def _weights(q, k, seen):
    """softmax(q k^T / sqrt(D)) where seen, [B, Hkv, G, M, N], for q [B, Hkv, G, M, D], k [B, Hkv, N, D]; no row: zeros."""
    B, H, G, M, _ = q.shape
    x = torch.matmul(q.reshape(B, H, G * M, D), k.transpose(2, 3)).view(B, H, G, M, -1)
    x *= D ** -0.5
    x.masked_fill_(~seen, float("-inf"))
    x -= x.amax(-1, keepdim=True).clamp_min(-1e30)
    x.exp_()
    x /= x.sum(-1, keepdim=True).clamp_min(1e-38)
    return x


def _spread_queries(s):
    """The packed queries as [B, Hkv, G, T_max, D], and the rows of their tokens [B, T_max] (-1: no token)."""
    case = s["case"]
    b, at, row = _tokens(s)
    q = torch.zeros((case["B"], s["T_max"], case["Hq"], D), device=DEV)
    q[b, at] = s["q"].float()
    p = torch.full((case["B"], s["T_max"]), -1, dtype=torch.long, device=DEV)
    p[b, at] = row
    return q.view(case["B"], s["T_max"], case["Hkv"], -1, D).permute(0, 2, 3, 1, 4).contiguous(), p, b, at


def _window(s):
    case = s["case"]
    q, p, b, at = _spread_queries(s)
    j, p = torch.arange(s["cap"], device=DEV), p.view(case["B"], 1, 1, -1, 1)
    w = _weights(q, _all_rows(s, "K"), (j <= p) & ((j > p - case["window"]) | (j < case["sink"])))
    B, H, G, M, N = w.shape
    o = torch.matmul(w.view(B, H, G * M, N), _all_rows(s, "V")).view(B, H * G, M, D)
    s["out"].copy_(o.transpose(1, 2)[b, at])


def _step(s, i, seen):
    """One decode step over rows i of which those in `seen` count: weights [B, Hkv, G, N] and the output."""
    case = s["case"]
    q = s["q"].view(case["B"], case["Hkv"], -1, 1, D)
    w = _weights(q, _rows(s, "K", i), seen.view(case["B"], 1, 1, 1, -1)).squeeze(3)
    s["out"].copy_(torch.matmul(w, _rows(s, "V", i)).view(case["B"], case["Hq"], D))
    return w


def _window_step(s):
    case = s["case"]
    n = s["lens"].long().view(-1, 1)
    first = torch.arange(case["sink"], device=DEV).expand(case["B"], -1)
    newest = n - case["window"] + torch.arange(case["window"], device=DEV)
    i = torch.cat([first, newest], 1)
    seen = torch.cat([first < n - case["window"], newest >= 0], 1)
    _step(s, i.clamp_min(0).minimum(n - 1), seen)


def _add_up(s, new):
    """mass = (what is held, decayed) + new [B, Hkv, N], in the rows that there are."""
    j, m = torch.arange(s["cap"], device=DEV), s["mass"]
    old = torch.where(j < s["held"].view(-1, 1, 1), m * s["case"]["decay"], 0.0)
    m.copy_(torch.where(j < s["lens"].view(-1, 1, 1), old + new, m))


def _mass(s):
    q, p, _, _ = _spread_queries(s)
    j = torch.arange(s["cap"], device=DEV)
    _add_up(s, _weights(q, _all_rows(s, "K"), j <= p.view(p.shape[0], 1, 1, -1, 1)).sum((2, 3)))


def _mass_step(s):
    i = torch.arange(s["cap"], device=DEV).expand(s["case"]["B"], -1)
    _add_up(s, _step(s, i, i < s["lens"].view(-1, 1)).sum(2))


def _evict(s):
    case = s["case"]
    n, m = s["lens"].long().view(-1, 1, 1), s["budget"].long().view(-1, 1, 1)
    m = torch.minimum(n, m)
    j = torch.arange(s["cap"], device=DEV)
    sinks = m.clamp_max(case["sink"])
    recent = (m - sinks).clamp_max(case["recent"])
    rank = torch.where(j < sinks, float("inf"), s["mass"])
    rank = torch.where((j >= n - recent) & (j < n), float("inf"), rank)
    rank = torch.where(j < n, rank, float("-inf"))
    order = torch.argsort(rank, dim=-1, descending=True, stable=True)          # ties to the lower row
    inside = j < m
    kept = torch.where(inside, order, s["cap"]).sort(-1).values                # the first m of the order, as rows in order
    s["kept"].copy_(torch.where(inside, kept, s["kept"]))
    s["mass_out"].copy_(torch.where(inside, s["mass"].gather(2, kept.clamp_max(s["cap"] - 1)), s["mass_out"]))
    s["lens_out"].copy_(m.view(-1))
    b, g, i = inside.expand(kept.shape).nonzero(as_tuple=True)
    block, at = _place(s, b, kept[b, g, i])
    block_to, at_to = _place(s, b, i, "table_to")
    k, v = _bytes(s["K"])[block, g, at], _bytes(s["V"])[block, g, at]
    _bytes(s["K_to"])[block_to, g, at_to] = k
    _bytes(s["V_to"])[block_to, g, at_to] = v


# ---------------------------------------------------------------- in 64 bits, from the definitions

def exact(case, seed):
    """Rotation, attention and weights in float64, request by request.  Moves of rows and whole numbers have no such value."""
    kind = case["kind"]
    if kind == "evict" or work(case)["flops"] > 1.0e12:
        return None
    s = prepare(case, seed)
    new, held = _lens(case)
    Hq, Hkv, G, page = case["Hq"], case["Hkv"], case["Hq"] // case["Hkv"], case["page"]

    def values(x):
        return x.to(torch.float32).double()

    def where(b, lo, hi):
        i = torch.arange(lo, hi, device=DEV)
        return (s["table"][b].long()[i // page], i % page) if page else (torch.full_like(i, b), i)

    if kind == "rotate":
        K, V = values(s["K"]), values(s["V"])
        q_out = torch.zeros((s["T"], Hq, D), dtype=torch.float64, device=DEV)
        half = case["rot"] // 2
        axis = s["pair_axis"].tolist() if s["pair_axis"] is not None else [0] * half
        pairs = [(2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half) for i in range(half)]

        def turned(x, weight):
            x = values(x)
            if weight is not None:
                x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / D + EPS) * weight.double()
            z = x.clone()
            for i, (a, c) in enumerate(pairs):
                angle = (s["positions"][axis[i]].double() * s["inv_freq"][i].double()).view(-1, 1)
                z[:, :, a] = x[:, :, a] * angle.cos() - x[:, :, c] * angle.sin()
                z[:, :, c] = x[:, :, a] * angle.sin() + x[:, :, c] * angle.cos()
            return z

        q_out[:] = turned(s["q"], s["q_weight"])
        k, v = turned(s["k_new"], s["k_weight"]), values(s["v_new"])
        if case["dtype"] == "fp8kv":
            k, v = k.clamp(-448.0, 448.0), v.clamp(-448.0, 448.0)
        for b in range(case["B"]):
            block, at = where(b, held[b], held[b] + new[b])
            K[block, :, at], V[block, :, at] = k[s["at"][b]:s["at"][b + 1]], v[s["at"][b]:s["at"][b + 1]]
        return {"q": q_out, "K": K, "V": V}

    def rows(x, b, g, n):
        block, at = where(b, 0, n)
        raw = _bytes(x)[block, g, at]
        return values(raw.view(x.dtype) if raw.dtype == torch.uint8 else raw)

    steps = kind in ("window_step", "mass_step")
    out = torch.zeros((case["B"] if steps else s["T"], Hq, D), dtype=torch.float64, device=DEV)
    mass = s["mass"].double() if kind in ("mass", "mass_step") else None
    for b in range(case["B"]):
        n = new[b] + held[b]
        t0, t1 = (b, b + 1) if steps else (s["at"][b], s["at"][b + 1])
        row = torch.arange(n - (t1 - t0), n, device=DEV)
        for g in range(Hkv):
            k, v = rows(s["K"], b, g, n), rows(s["V"], b, g, n)
            total = torch.zeros(n, dtype=torch.float64, device=DEV)
            for h in range(g * G, g * G + G):
                for lo in range(0, t1 - t0, 4096):
                    x = values(s["q"][t0:t1, h][lo:lo + 4096]) @ k.T.contiguous() / D ** 0.5
                    p, j = row[lo:lo + 4096].view(-1, 1), torch.arange(n, device=DEV)
                    hidden = j > p
                    if case["window"]:
                        hidden = hidden | ((j <= p - case["window"]) & (j >= case["sink"]))
                    w = torch.softmax(x.masked_fill(hidden, float("-inf")), 1)
                    total += w.sum(0)
                    if kind != "mass":
                        out[t0 + lo:t0 + lo + x.shape[0], h] = w @ v
            if mass is not None:
                keep = int(s["held"][b])
                total[:keep] += case["decay"] * mass[b, g, :keep]
                mass[b, g, :n] = total
    if kind == "mass":
        return mass
    return {"out": out, "mass": mass} if kind == "mass_step" else out
