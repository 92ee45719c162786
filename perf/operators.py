"""Prompts, forks and pages over the KV cache, as timed cases.

Four kinds of pass, one attention layer each, through the public binding:

  append   the newest K and V rows of every request, as slices of a fused projection, into the cache (`lfps_append`).
  prompt   causal attention of every request's newest tokens over its cache (`lfps_prompt_attn`): whole prompts, chunks of
           long ones behind rows that are in the cache already, a few drafted tokens.
  prefix   one decode step's full attention where groups of requests share their first rows (`lfps_prefix_attn_decode`).
  fork     requests continue others, grow or end: new block tables, copies of shared half-filled blocks
           (`lfps_pages_update`, `lfps_pages_copy`).
  compact  the live blocks of a pool move to its front (`lfps_pages_compact`, `lfps_pages_copy`).

A case says the shapes: B requests; each brings T_lo..T_hi new tokens behind P_lo..P_hi rows that the cache holds (prefix:
S_lo..S_hi rows of its own behind a shared prefix of P_lo..P_hi rows, `group` requests to a group); Hq query heads over Hkv KV
heads of 128 channels; the cache format (f32 / bf16 / f16 / fp8kv = FP8 keys and values beside bf16 queries) and layout
(page = rows per block, 0 = contiguous); lens_seed, from which the lengths inside the ranges come.
"""
import random

import torch

own = False

D = 128
DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "fp8kv": torch.bfloat16}

BASE = {"kind": "prompt", "B": 1, "T_lo": 1, "T_hi": 1, "P_lo": 0, "P_hi": 0, "S_lo": 0, "S_hi": 0, "group": 1, "Hq": 32,
        "Hkv": 8, "dtype": "bf16", "page": 0, "lens_seed": 1, "blocks": 0, "live": 0.0}


def _case(name, **kw):
    return dict(BASE, name=name, **kw)


def listed():
    return [
        # Five drafted tokens of one request over an ordinary context: few rows, latency counts.
        _case("prompt_b1_5_of_4k_paged", T_lo=5, T_hi=5, P_lo=4099, P_hi=4099, page=16),
        # A batch of prompts of unlike lengths, as they arrive, packed; fp16 cache, two heads per group.
        _case("prompt_b8_ragged_f16_paged", B=8, T_lo=61, T_hi=4096, Hq=16, Hkv=8, dtype="f16", page=64, lens_seed=7),
        # One long prompt into an empty cache.
        _case("prompt_b1_16k_bf16", T_lo=16384, T_hi=16384),
        # The last chunk of a longer prompt, over the FP8 pages that the earlier chunks left.
        _case("prompt_b1_8k_of_32k_fp8kv_paged", T_lo=8192, T_hi=8192, P_lo=24576, P_hi=24576, dtype="fp8kv", page=16),
        # Two short prompts over an fp32 cache.
        _case("prompt_b2_odd_f32", B=2, T_lo=701, T_hi=1333, dtype="f32", lens_seed=3),
        # Four continuations of one short prompt.
        _case("prefix_b4_2k_bf16", kind="prefix", B=4, group=4, P_lo=2049, P_hi=2049, S_lo=3, S_hi=60, lens_seed=2),
        # Eight requests to each of four system prompts, serving cache.
        _case("prefix_b32_8k_fp8kv_paged", kind="prefix", B=32, group=8, P_lo=8000, P_hi=12000, S_lo=100, S_hi=2000,
              dtype="fp8kv", page=16, lens_seed=5),
        # One long document, sixty-four questions.
        _case("prefix_b64_32k_bf16_paged", kind="prefix", B=64, group=64, P_lo=32768, P_hi=32768, S_lo=1, S_hi=900, page=64,
              lens_seed=4),
        # One token each of a decoding batch, into FP8 pages: the call that every decode step begins with.
        _case("append_b32_1_fp8kv_paged", kind="append", B=32, P_lo=1, P_hi=30, dtype="fp8kv", page=16),
        # A long packed batch of prompts, out of the fused projection.
        _case("append_b8_ragged_bf16_paged", kind="append", B=8, T_lo=1000, T_hi=6000, P_lo=0, P_hi=300, page=16, lens_seed=6),
        # Sampling of several continuations: a few parents are forked into most slots, some slots end, all grow by a token.
        _case("fork_b64_16k_paged", kind="fork", B=64, P_lo=500, P_hi=16384, page=16, blocks=65536, lens_seed=8),
        # A pool after a day of requests that came and went: a third of its blocks live, scattered.
        _case("compact_b64_paged", kind="compact", B=64, P_lo=2000, P_hi=9000, page=16, blocks=65536, lens_seed=9),
    ]


def _spread(rng, lo, hi):
    """A whole number in [lo, hi], over the logarithm."""
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    """A case of the listed ranges that costs no more than the largest listed one."""
    while True:
        kind = rng.choice(["prompt", "prompt", "prompt", "prefix", "prefix", "append", "fork", "compact"])
        hkv = rng.choice([1, 2, 4, 8, 8])
        c = dict(BASE, kind=kind, Hkv=hkv, Hq=hkv * rng.choice([1, 2, 4, 4]), lens_seed=rng.randrange(1 << 30),
                 dtype=rng.choice(["bf16", "bf16", "f16", "fp8kv", "f32"]), page=rng.choice([0, 16, 64, 256]))
        if kind == "prompt":
            c["B"] = _spread(rng, 1, 32)
            c["T_hi"] = _spread(rng, 1, 16384)
            c["T_lo"] = _spread(rng, 1, c["T_hi"])
            c["P_hi"] = _spread(rng, 1, 32768) if rng.random() < 0.5 else 0
            c["P_lo"] = c["P_hi"] // 3
        elif kind == "prefix":
            c["group"] = _spread(rng, 2, 64)
            c["B"] = c["group"] * rng.choice([1, 1, 2, 4])
            c["P_hi"] = _spread(rng, 200, 32768)
            c["P_lo"] = c["P_hi"] // 2
            c["S_hi"] = _spread(rng, 1, 2000)
        elif kind == "append":
            c["B"] = _spread(rng, 1, 64)
            c["T_hi"] = _spread(rng, 1, 6000)
            c["T_lo"] = _spread(rng, 1, c["T_hi"])
            c["P_hi"] = _spread(rng, 1, 300)
        else:
            c["B"] = _spread(rng, 2, 64)
            c["page"] = rng.choice([16, 64])
            c["P_hi"] = _spread(rng, 100, 16384)
            c["P_lo"] = c["P_hi"] // 4
            c["blocks"] = 2 * c["B"] * (-(-(c["P_hi"] + 64) // c["page"])) + rng.randrange(1, 1000)
        w = work(c)
        rows = c["B"] * (c["T_hi"] + c["P_hi"] + c["S_hi"])
        padded = c["B"] * c["T_hi"] * (c["T_hi"] + c["P_hi"]) * (c["Hq"] // hkv)
        if w["flops"] <= 2.0e12 and padded <= 8.0e9 and w["bytes"] <= 2.0e9 and rows * c["Hkv"] <= 20_000_000 and \
                c["blocks"] * c["page"] * c["Hkv"] <= 12_000_000 and (c["dtype"] != "f32" or w["flops"] <= 2.0e11):
            return c


# ---------------------------------------------------------------- shapes and work

def _lens(case):
    """Per request (new tokens, rows held before them); prefix: (own rows, shared rows)."""
    r = random.Random(case["lens_seed"])
    B = case["B"]
    if case["kind"] == "prefix":
        shared = [r.randint(case["P_lo"], case["P_hi"]) for _ in range(B // case["group"])]
        return [r.randint(case["S_lo"], case["S_hi"]) for _ in range(B)], [shared[b // case["group"]] for b in range(B)]
    new = [r.randint(case["T_lo"], case["T_hi"]) for _ in range(B)]
    return new, [r.randint(case["P_lo"], case["P_hi"]) for _ in range(B)]


def _forks(case):
    """fork: each slot's parent (-1: the slot ends) and its new length."""
    r = random.Random(case["lens_seed"] + 1)
    _, held = _lens(case)
    few = [r.randrange(case["B"]) for _ in range(max(1, case["B"] // 8))]
    parent = [-1 if r.random() < 0.1 else (r.choice(few) if r.random() < 0.7 else b) for b in range(case["B"])]
    return parent, [0 if p < 0 else held[p] + 1 for p in parent]


def _row_bytes(case):
    return D * {"f32": 4, "fp8kv": 1}.get(case["dtype"], 2)


def work(case):
    new, held = _lens(case)
    row, q_row = 2 * case["Hkv"] * _row_bytes(case), case["Hq"] * D * (4 if case["dtype"] == "f32" else 2)
    if case["kind"] == "append":
        rows = sum(new)
        return {"bytes": rows * (row + 2 * case["Hkv"] * D * (4 if case["dtype"] == "f32" else 2)), "flops": 0}
    if case["kind"] == "prompt":
        seen = sum(t * h + t * (t + 1) // 2 for t, h in zip(new, held))
        return {"bytes": 2 * sum(new) * q_row + sum(t + h for t, h in zip(new, held)) * row, "flops": 4 * D * case["Hq"] * seen}
    if case["kind"] == "prefix":
        rows = sum(held[::case["group"]]) + sum(new)
        return {"bytes": rows * row + 2 * case["B"] * case["Hq"] * D * 4, "flops": 4 * D * case["Hq"] * (sum(new) + sum(held))}
    entries = sum(-(-h // case["page"]) for h in held)
    if case["kind"] == "fork":
        parent, _ = _forks(case)
        copied = sum(held[p] % case["page"] for p in parent if p >= 0)
        return {"bytes": 8 * entries + 2 * copied * row, "flops": 0}
    live = entries                       # at most this many; those past the front move
    moved = max(0, live - live * live // case["blocks"])
    return {"bytes": 8 * entries + 4 * case["blocks"] + 2 * moved * case["page"] * row, "flops": 0}


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
    s["lens"] = _ints([h if kind in ("fork", "compact") else t + h for t, h in zip(new, held)])
    cap = max(1, max(held) + (64 if kind in ("fork", "compact") else max(new)))
    s["cap"] = cap
    # Queries lean towards a direction of their KV head, and so do the first four rows' keys (attention sinks).
    lean = normal(Hkv, 1, D)
    if page:
        per = -(-cap // page)
        n_blocks = case["blocks"] or B * per + 7
        places = torch.randperm(n_blocks, device=DEV, generator=gen)[:B * per].view(B, per)
        s["table"] = places.to(torch.int32).contiguous()
        shape = (n_blocks, Hkv, page, D)
    else:
        shape = (B, Hkv, cap, D)
    if kind in ("prompt", "prefix"):
        k = normal(*shape)
        if page:
            first = torch.zeros((shape[0], 1, page, 1), device=DEV)
            first[places[:, 0].long(), :, :min(4, page)] = 1.0
        else:
            first = torch.zeros((B, 1, cap, 1), device=DEV)
            first[:, :, :4] = 1.0
        k += 0.8 * first * lean
        s["K"], s["V"] = _to_cache(k, cdt), _to_cache(normal(*shape), cdt)
        del k
    elif kind == "append":
        s["K"], s["V"] = (torch.zeros(shape, device=DEV).to(cdt) for _ in range(2))
    else:
        s["K"], s["V"] = (torch.randn(shape, device=DEV, generator=gen, dtype=torch.bfloat16 if cdt.itemsize == 1 else cdt).to(cdt)
                          for _ in range(2))
    if kind in ("prompt", "append"):
        T = sum(new)
        at = [0]
        for t in new:
            at.append(at[-1] + t)
        s["cu"] = _ints(at)
        s["at"], s["T_max"] = at, max(new)
        qkv = normal(T, Hq + 2 * Hkv, D)
        qkv[:, :Hq] = 0.8 * qkv[:, :Hq] + 0.6 * lean.view(1, Hkv, 1, D).expand(T, Hkv, Hq // Hkv, D).reshape(T, Hq, D)
        if kind == "append":
            qkv[:, Hq:] *= 1.0 + 200.0 * (torch.rand((T, 2 * Hkv, 1), device=DEV, generator=gen) < 0.01)   # outlier rows: FP8 saturates
        s["qkv"] = qkv.to(dt)                         # the layer's fused projection; q, k and v are slices of it
        del qkv
        s["q"], s["k_new"], s["v_new"] = s["qkv"].split([Hq, Hkv, Hkv], dim=1)
        if kind == "prompt":
            s["out"] = torch.zeros((T, Hq, D), dtype=dt, device=DEV)
    if kind == "prefix":
        n_groups = B // case["group"]
        s["q"] = 0.8 * normal(B, Hq, D) + 0.6 * lean.expand(Hkv, Hq // Hkv, D).reshape(1, Hq, D)
        s["group_start"] = _ints([case["group"] * g for g in range(n_groups + 1)])
        s["prefix_len"] = _ints(held[::case["group"]])
        s["out"] = torch.zeros((B, Hq, D), device=DEV)
        if page:                                      # the members' tables name the first member's blocks as far as these are full
            full = s["prefix_len"].repeat_interleave(case["group"]).view(B, 1) // page
            j = torch.arange(s["table"].shape[1], device=DEV)
            lead = (torch.arange(B, device=DEV) // case["group"]) * case["group"]
            s["table"] = torch.where(j < full, s["table"][lead], s["table"]).contiguous()
    if kind in ("fork", "compact"):
        s["table_out"] = torch.zeros_like(s["table"])
    if kind == "fork":
        parent, lens = _forks(case)
        s["parent"], s["new_lens"] = _ints(parent), _ints(lens)
        s["lens_out"], s["copies"] = torch.zeros_like(s["lens"]), torch.zeros((B, 3), dtype=torch.int32, device=DEV)
    if kind == "compact":
        n = s["K"].shape[0]
        s["map"], s["n_live"] = _ints([0]).expand(n).contiguous(), _ints([0])
        s["copies"] = torch.zeros((n // 2, 3), dtype=torch.int32, device=DEV)
    if own:
        from paper_2506_15704_amd.binding import Lfps
        ctx = Lfps(batch=B, n_q_heads=Hq, n_kv_heads=Hkv, kv_dtype="bf16" if case["dtype"] == "fp8kv" else case["dtype"],
                   max_seq_len=cap, max_k=1, radius=1, k_fp8=case["dtype"] == "fp8kv", v_fp8=case["dtype"] == "fp8kv")
        s["ctx"] = ctx
        s["kv"] = ctx.paged_kv_view(s["K"], s["V"], s["table"], s["lens"]) if page else ctx.kv_view(s["K"], s["V"], s["lens"])
        if kind in ("fork", "compact"):
            s["work"] = ctx.pages_workspace(s["K"].shape[0])
    return s


# ---------------------------------------------------------------- the pass

def run(s):
    kind = s["case"]["kind"]
    if own:
        ctx = s["ctx"]
        if kind == "append":
            ctx.lfps_append(s["k_new"], s["v_new"], s["cu"], s["kv"])
        elif kind == "prompt":
            ctx.lfps_prompt_attn(s["q"], s["cu"], s["kv"], s["out"])
        elif kind == "prefix":
            ctx.lfps_prefix_attn_decode(s["q"], s["kv"], s["group_start"], s["prefix_len"], s["out"])
        elif kind == "fork":
            ctx.lfps_pages_update(s["kv"], s["parent"], s["new_lens"], s["table_out"], s["lens_out"], s["copies"], s["work"])
            ctx.lfps_pages_copy(s["kv"], s["copies"])
        else:
            ctx.lfps_pages_compact(s["kv"], s["table_out"], s["copies"], s["map"], s["n_live"], s["work"])
            ctx.lfps_pages_copy(s["kv"], s["copies"])
    else:
        {"append": _append, "prompt": _prompt, "prefix": _prefix, "fork": _fork, "compact": _compact}[kind](s)
    if kind == "append":
        return {"K": s["K"], "V": s["V"]}
    if kind in ("prompt", "prefix"):
        return s["out"]
    if kind == "fork":
        return {"K": s["K"], "V": s["V"], "table": s["table_out"], "lens": s["lens_out"], "copies": s["copies"]}
    return {"K": s["K"], "V": s["V"], "table": s["table_out"], "copies": s["copies"], "map": s["map"], "n_live": s["n_live"]}


def _bytes(x):
    return x.view(torch.uint8) if x.element_size() == 1 else x


def _append(s):
    case, cu = s["case"], s["cu"].long()
    T = s["k_new"].shape[0]
    t = torch.arange(T, device=DEV)
    b = torch.searchsorted(cu[1:], t, right=True)
    pos = s["lens"].long()[b] - (cu[b + 1] - t)
    page = case["page"]
    block, row = (s["table"].long()[b, pos // page], pos % page) if page else (b, pos)
    for cache, new in (("K", "k_new"), ("V", "v_new")):
        x = s[new].float()
        _bytes(s[cache])[block, :, row] = _bytes(_to_cache(x, s[cache].dtype))


def _rows(s, name, lead=None, shared=None):
    """Every request's rows of K or V in order, [B, Hkv, cap, D] fp32 (rows below `shared` those of request `lead`)."""
    x, page = s[name], s["case"]["page"]
    B = s["case"]["B"]
    i = torch.arange(s["cap"], device=DEV).expand(B, -1)
    b = torch.arange(B, device=DEV).view(B, 1).expand_as(i)
    if lead is not None:
        b = torch.where(i < shared.view(B, 1), lead.view(B, 1), b)
    block, row = (s["table"].long()[b, i // page], i % page) if page else (b, i)
    x = _bytes(x)[block, :, row]                       # [B, cap, Hkv, D]
    x = x.view(s[name].dtype) if x.dtype == torch.uint8 else x
    return x.float().transpose(1, 2).contiguous()


def _attend(q, k, v, seen):
    """softmax(q k^T / sqrt(D)) v over the first `seen` rows: q [B, G, M, D], k, v [B, N, D], seen [B, M]; no row: zeros."""
    B, G, M, _ = q.shape
    x = torch.matmul(q.reshape(B, G * M, D), k.transpose(1, 2)).view(B, G, M, -1) * D ** -0.5
    hidden = torch.arange(k.shape[1], device=DEV) >= seen.view(B, 1, M, 1)
    x.masked_fill_(hidden, float("-inf"))
    x -= x.amax(-1, keepdim=True).clamp_min(-1e30)
    x.exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(B, G * M, -1), v).view(B, G, M, D)
    return torch.where(total > 0, o / total.clamp_min(1e-38), torch.zeros_like(o))


def _prompt(s):
    case, cu = s["case"], s["cu"].long()
    Hkv, G, T = case["Hkv"], case["Hq"] // case["Hkv"], s["q"].shape[0]
    t = torch.arange(T, device=DEV)
    b = torch.searchsorted(cu[1:], t, right=True)
    at = t - cu[b]                                                   # place of a token among its request's new ones
    seen = torch.zeros((case["B"], s["T_max"]), dtype=torch.long, device=DEV)
    seen[b, at] = s["lens"].long()[b] - (cu[b + 1] - t) + 1
    k, v = _rows(s, "K"), _rows(s, "V")
    q = torch.zeros((case["B"], s["T_max"], case["Hq"], D), device=DEV)
    q[b, at] = s["q"].float()
    q = q.view(case["B"], s["T_max"], Hkv, G, D).permute(2, 0, 3, 1, 4).contiguous()
    for g in range(Hkv):                                             # one KV head at a time: the scores are large
        o = _attend(q[g], k[:, g], v[:, g], seen)                    # [B, G, T_max, D]
        s["out"][:, g * G:(g + 1) * G] = o.permute(0, 2, 1, 3)[b, at].to(s["out"].dtype)


def _prefix(s):
    case = s["case"]
    B, Hkv, G = case["B"], case["Hkv"], case["Hq"] // case["Hkv"]
    lead = torch.arange(B, device=DEV) // case["group"] * case["group"]
    shared = s["prefix_len"].long().repeat_interleave(case["group"])
    k, v = _rows(s, "K", lead, shared), _rows(s, "V", lead, shared)
    o = _attend(s["q"].view(B * Hkv, 1, G, D), k.view(B * Hkv, -1, D), v.view(B * Hkv, -1, D),
                s["lens"].long().repeat_interleave(Hkv).view(-1, 1).expand(-1, G))
    s["out"].copy_(o.view(B, case["Hq"], D))


def _live(s):
    page = s["case"]["page"]
    table = s["table"].long()
    used = torch.arange(table.shape[1], device=DEV) < -(-s["lens"].long() // page).view(-1, 1)
    n = s["K"].shape[0]
    mark = torch.zeros(n + 1, dtype=torch.bool, device=DEV)
    mark[torch.where(used, table, n)] = True
    return mark[:n], used, table


def _fork(s):
    """(The pools of these cases always have the blocks that are asked for.)"""
    page = s["case"]["page"]
    live, _, table = _live(s)
    B, per = table.shape
    n = live.numel()
    slot, j = torch.arange(B, device=DEV), torch.arange(per, device=DEV)
    parent = s["parent"].long()
    ends = parent < 0
    p = parent.clamp_min(0)
    length = torch.where(ends, 0, s["new_lens"].long())
    kept_rows = torch.minimum(torch.where(ends, 0, s["lens"].long()[p]), length)
    kept, wanted = -(-kept_rows // page), -(-length // page)
    entries = torch.where(j < kept.view(-1, 1), table[p], n)          # n: none
    writes = (length > kept_rows) & (kept_rows % page != 0)           # into a block that holds rows already
    tail = torch.where(writes, entries[slot, (kept - 1).clamp_min(0)], n)
    one = torch.ones((), dtype=torch.long, device=DEV)
    holders = torch.zeros(n + 1, dtype=torch.long, device=DEV).index_add_(0, entries.flatten(), one.expand(B * per))
    writers = torch.zeros(n + 1, dtype=torch.long, device=DEV).index_add_(0, tail, one.expand(B))
    first = torch.full((n + 1,), B, device=DEV).scatter_reduce_(0, tail, slot, "amin")
    copy = writes & ((holders[tail] > writers[tail]) | (first[tail] != slot))
    need = copy.long() + wanted - kept
    start = need.cumsum(0) - need
    free = torch.argsort(live.to(torch.int8), stable=True)            # the free blocks in order, then the others
    fresh = start.view(-1, 1) + copy.long().view(-1, 1) + (j - kept.view(-1, 1))
    out = torch.where((j >= kept.view(-1, 1)) & (j < wanted.view(-1, 1)), free[fresh.clamp(0, n - 1)], entries)
    mine = free[start.clamp(0, n - 1)]
    out = torch.where(copy.view(-1, 1) & (j == (kept - 1).view(-1, 1)), mine.view(-1, 1), out)
    s["table_out"].copy_(torch.where(out == n, -1, out))
    s["lens_out"].copy_(length)
    rows = kept_rows % page
    minus = torch.full_like(tail, -1)
    s["copies"].copy_(torch.stack([torch.where(copy, tail, minus), torch.where(copy, mine, minus), torch.where(copy, rows, 0)], 1))
    # rows of a block's head that are copied: the others of the destination stay as they are
    r = torch.arange(page, device=DEV)
    src, dst = torch.where(copy, tail, 0), torch.where(copy, mine, 0)
    take = (copy.view(-1, 1) & (r < rows.view(-1, 1))).nonzero()
    for name in ("K", "V"):
        x = _bytes(s[name])
        x[dst[take[:, 0]], :, take[:, 1]] = x[src[take[:, 0]], :, take[:, 1]]


def _compact(s):
    live, used, table = _live(s)
    n = live.numel()
    total = live.sum()
    ids = torch.arange(n, device=DEV)
    hole, mover = ~live & (ids < total), live & (ids >= total)
    to = torch.argsort((~hole).to(torch.int8), stable=True)           # the holes in order, then the others
    rank = mover.long().cumsum(0) - 1
    new = torch.where(mover, to[rank.clamp_min(0)], torch.where(live, ids, -1))
    s["map"].copy_(new)
    s["n_live"].copy_(total.view(1))
    s["table_out"].copy_(torch.where(used, new[table.clamp(0, n - 1)], -1))
    moves = s["copies"].shape[0]
    src = torch.argsort((~mover).to(torch.int8), stable=True)[:moves]
    there = torch.arange(moves, device=DEV) < mover.sum()
    s["copies"].copy_(torch.stack([torch.where(there, src, -1), torch.where(there, to[:moves], -1),
                                   torch.where(there, s["case"]["page"], 0)], 1))
    i = there.nonzero().view(-1)
    for name in ("K", "V"):
        x = _bytes(s[name])
        x[to[i]] = x[src[i]]


# ---------------------------------------------------------------- in 64 bits, from the definitions

def exact(case, seed):
    """Attention: every query on its own rows in float64.  Moves of rows and whole numbers have no such value."""
    if case["kind"] not in ("prompt", "prefix") or work(case)["flops"] > 6.0e12:
        return None
    s = prepare(case, seed)
    new, held = _lens(case)
    Hkv, G, page = case["Hkv"], case["Hq"] // case["Hkv"], case["page"]

    def rows(x, b, lo, hi):
        if not page:
            return x[b, :, lo:hi].to(torch.float32).double()
        i = torch.arange(lo, hi, device=DEV)
        block = s["table"][b].long()[i // page]
        raw = _bytes(x)[block, :, i % page]
        return (raw.view(x.dtype) if raw.dtype == torch.uint8 else raw).to(torch.float32).double().transpose(0, 1)

    def softmax_sum(q, k, v, first):
        """q [M, D] whose row i sees k[:first + i // G]."""
        out = torch.zeros((q.shape[0], D), dtype=torch.float64, device=DEV)
        for lo in range(0, q.shape[0], 4096):
            x = q[lo:lo + 4096] @ k.T.contiguous() / D ** 0.5
            limit = first + torch.arange(lo, lo + x.shape[0], device=DEV) // G
            x[torch.arange(k.shape[0], device=DEV) >= limit.view(-1, 1)] = float("-inf")
            out[lo:lo + 4096] = torch.softmax(x, 1) @ v
        return out

    if case["kind"] == "prompt":
        out = torch.zeros((s["at"][-1], case["Hq"], D), dtype=torch.float64, device=DEV)
        for b in range(case["B"]):
            t0, t1, n = s["at"][b], s["at"][b + 1], new[b] + held[b]
            k, v = rows(s["K"], b, 0, n), rows(s["V"], b, 0, n)
            for g in range(Hkv):
                q = s["q"][t0:t1, g * G:(g + 1) * G].to(torch.float32).double().reshape(-1, D)
                out[t0:t1, g * G:(g + 1) * G] = softmax_sum(q, k[g], v[g], held[b] + 1).view(-1, G, D)
        return out
    out = torch.zeros((case["B"], case["Hq"], D), dtype=torch.float64, device=DEV)
    for b in range(case["B"]):
        lead, p = b // case["group"] * case["group"], held[b]
        k = torch.cat([rows(s["K"], lead, 0, p), rows(s["K"], b, p, p + new[b])], 1)
        v = torch.cat([rows(s["V"], lead, 0, p), rows(s["V"], b, p, p + new[b])], 1)
        for g in range(Hkv):
            x = s["q"][b, g * G:(g + 1) * G].double() @ k[g].T.contiguous() / D ** 0.5
            out[b, g * G:(g + 1) * G] = torch.softmax(x, 1) @ v[g]
    return out
