"""The operators of a long-context cache that is kept small, as cases to be timed and compared.

A serving program that runs out of room for the grouped-value cache has two ways out: hold each value in 4 bits, and drop
the tokens that attention no longer looks at.  Four kinds of case stand for them:

  decode   one decode step of a batch over the 4-bit cache: the new token is quantised into its page, then attention over
           all tokens (append + decode)
  chunk    a prompt or a chunk of one enters the 4-bit cache, and the rows come back widened to bf16 pages, as the chunk's
           own prefill reads them (append_chunk + widen)
  weights  the attention weight that every cached token received from the new queries, added to what it has gathered so far
  evict    the tokens with the least gathered weight leave the cache, which closes up in place

`run` is the plain form in elementary torch operations, or, where `own` is set, the library's calls.
"""
import math

import numpy as np
import torch

own = False

# head layouts: the ones the repository's tests and benchmark use (d_c = d_v everywhere)
_HEADS = {"a": (16, 4, 64, 16), "b": (32, 8, 128, 32), "c": (16, 4, 64, 24), "a0": (16, 4, 64, 0), "b0": (32, 8, 128, 0),
          "g1": (4, 1, 64, 16), "g2": (8, 2, 128, 32), "g8": (32, 8, 64, 16), "g3": (12, 3, 64, 0)}
_BASE = 10000.0


# ---------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one user, a short chat: nothing but latency
        {"name": "decode-b1-t97", "kind": "decode", "heads": "a", "B": 1, "lo": 97, "hi": 97, "page": 64},
        # a small batch at ordinary lengths, odd ones, 48-byte positional rows, larger pages
        {"name": "decode-b7-ragged-dr24", "kind": "decode", "heads": "c", "B": 7, "lo": 301, "hi": 4999, "page": 128},
        # the long-context batch of the benchmark: 1 M cached tokens
        {"name": "decode-b32-t32768", "kind": "decode", "heads": "a", "B": 32, "lo": 32768, "hi": 32768, "page": 64},
        # the ragged wide-head batch of the benchmark
        {"name": "decode-b64-ragged-wide", "kind": "decode", "heads": "b", "B": 64, "lo": 1024, "hi": 16384, "page": 64},
        # the second chunk of a few prompts, odd lengths
        {"name": "chunk-b3-q437", "kind": "chunk", "heads": "a", "B": 3, "q_lo": 211, "q_hi": 437, "ctx_lo": 77, "ctx_hi": 1030, "page": 64},
        # whole prompts of a prefill batch, wide heads
        {"name": "chunk-b8-q8192-wide", "kind": "chunk", "heads": "b", "B": 8, "q_lo": 8192, "q_hi": 8192, "ctx_lo": 0, "ctx_hi": 0, "page": 64},
        # one decode step's weights, small bf16 cache
        {"name": "weights-bf16-b4-t1000", "kind": "weights", "dtype": "bf16", "heads": "a", "B": 4, "lo": 500, "hi": 1500, "rows": 1, "page": 64},
        # one decode step's weights over the 1 M tokens, 4 bits
        {"name": "weights-q4-b32-t32768", "kind": "weights", "dtype": "q4", "heads": "a", "B": 32, "lo": 32768, "hi": 32768, "rows": 1, "page": 64},
        # the last tokens of four prompts, up to 32 each, decide what the prompts' cache keeps; e4m3, wide heads
        {"name": "weights-fp8-b4-r32-wide", "kind": "weights", "dtype": "fp8", "heads": "b", "B": 4, "lo": 5000, "hi": 8192, "rows": 32, "page": 64},
        # a few sequences over their budget by a little, bf16
        {"name": "evict-bf16-b3-t1300", "kind": "evict", "dtype": "bf16", "heads": "a", "B": 3, "lo": 1100, "hi": 1500, "keep": 1024, "sinks": 4, "recent": 128, "page": 64},
        # the 1 M token batch down to a quarter, 4 bits
        {"name": "evict-q4-b32-t32768", "kind": "evict", "dtype": "q4", "heads": "a", "B": 32, "lo": 32768, "hi": 32768, "keep": 8192, "sinks": 4, "recent": 512, "page": 64},
        # the ragged wide-head batch held to a common budget, bf16
        {"name": "evict-bf16-b64-wide", "kind": "evict", "dtype": "bf16", "heads": "b", "B": 64, "lo": 1024, "hi": 16384, "keep": 6000, "sinks": 16, "recent": 256, "page": 64},
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["decode", "decode", "chunk", "weights", "weights", "evict"])
    heads = rng.choice(["a", "a", "b", "c", "a0", "b0", "g1", "g2", "g8", "g3"])
    case = {"kind": kind, "heads": heads, "page": rng.choice([32, 64, 64, 128, 256])}
    wide = _HEADS[heads][2] * _HEADS[heads][1] // 256 or 1           # a token's size against the narrow layout's
    most = 32 * 32768 // wide                                        # tokens in all
    if kind == "chunk":
        case["B"] = log(1, 16)
        q = min(log(1, 8192), 65536 // wide // case["B"])
        case["q_lo"], case["q_hi"] = max(1, int(q * rng.uniform(0.3, 1.0))), q
        case["ctx_lo"], case["ctx_hi"] = 0, rng.choice([0, log(1, 5000)])
        return case
    B = log(1, 64)
    t = min(log(1, 40000), most // B)
    case.update(B=B, lo=max(1, int(t * rng.choice([1.0, rng.uniform(0.05, 1.0)]))), hi=t)
    if kind == "weights":
        case["rows"] = rng.choice([1, 1, 2, 8, rng.randint(2, 48)])
        H = _HEADS[heads][0]
        case["hi"] = max(1, min(case["hi"], 130_000_000 // (case["rows"] * H * B)))
        case["lo"] = min(case["lo"], case["hi"])
    if kind == "evict":
        case.update(keep=max(1, int(case["hi"] * rng.uniform(0.1, 1.1))), sinks=rng.choice([0, 1, 4, 16]), recent=rng.choice([0, 1, 64, log(1, 1000)]))
    if kind in ("weights", "evict"):
        kinds = ["q4", "bf16", "fp8"] if heads != "c" and case["page"] % 64 == 0 else ["q4", "bf16"]
        case["dtype"] = rng.choice(kinds)
    return case


def _spread(lo, hi, n):
    """n whole numbers over [lo, hi], the same for every seed; the largest is hi."""
    return [hi if i == 0 else lo + int((hi - lo) * ((i * 0.6180339887) % 1.0)) for i in range(n)]


def _row_counts(case):
    """New tokens of every sequence: a count of its own for each, the first the largest."""
    return [1 + (i * 7 + case["rows"] - 1) % case["rows"] for i in range(case["B"])]


def _row_bytes(dtype, heads):
    H, G, d_v, d_r = _HEADS[heads]
    return {"q4": G * (d_v // 2 + 4) + 2 * d_r, "bf16": 2 * (G * d_v + d_r), "fp8": G * d_v + d_r}[dtype]


def work(case):
    H, G, d_v, d_r = _HEADS[case["heads"]]
    B = case["B"]
    if case["kind"] == "chunk":
        n = sum(_spread(case["q_lo"], case["q_hi"], B))
        # f32 rows in, 4-bit rows out, and the widened rows (what was just written need not be read again)
        return {"bytes": n * (4 * (G * d_v + d_r) + _row_bytes("q4", case["heads"]) + _row_bytes("bf16", case["heads"])), "flops": 8 * n * G * d_v}
    lens = _spread(case["lo"], case["hi"], B)
    n = sum(lens)
    if case["kind"] == "decode":
        io = B * 4 * (H * (d_v + d_r) + H * d_v + H + G * d_v + d_r)
        return {"bytes": n * _row_bytes("q4", case["heads"]) + io, "flops": 2 * n * H * (2 * d_v + d_r)}
    if case["kind"] == "weights":
        rows = _row_counts(case)
        return {"bytes": n * (_row_bytes(case["dtype"], case["heads"]) + 8) + sum(rows) * 4 * H * (d_v + d_r + 1),
                "flops": 2 * sum(a * b for a, b in zip(lens, rows)) * H * (d_v + d_r)}
    kept = [min(case["keep"], t) for t in lens]
    # every weight and position is read and every slot's new ones are written; of a random set of survivors, the share
    # (len - keep) / len of the kept slots are holes, and each is filled by one row read and written
    moved = sum(k * (t - k) / t for k, t in zip(kept, lens))
    return {"bytes": 16 * n + moved * 2 * _row_bytes(case["dtype"], case["heads"]), "flops": n}


# --------------------------------------------------------------------------------------------------------------- inputs
def _paged(lens, page, gen):
    """Block table [B][max_pages] with the pages in a random order, a few pages left over; numbers of pages."""
    most = max(1, max((t + page - 1) // page for t in lens))
    pages = len(lens) * most + 3
    table = torch.randperm(pages, generator=gen, device="cuda")[: len(lens) * most].to(torch.int32).reshape(len(lens), most)
    return table.contiguous(), pages, most


def _pools(dtype, heads, pages, page, gen):
    H, G, d_v, d_r = _HEADS[heads]
    rand = lambda *shape: torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)  # noqa: E731
    if dtype == "q4":
        # what the quantiser leaves of rows ~ N(0, 1): codes bell-shaped around the middle, a step of about 5 / 15
        v = torch.empty(pages, G, page, d_v // 2, dtype=torch.uint8, device="cuda")
        for lo in range(0, pages, 4096):
            n = min(4096, pages - lo)
            c = (rand(n, G, page, d_v // 2, 2) * 3.0 + 7.5).round_().clamp_(0, 15).to(torch.uint8)
            v[lo:lo + n] = c[..., 0] | (c[..., 1] << 4)
        step = 0.33 + 0.03 * rand(pages, G, page).clamp_(-3, 3)
        sz = torch.stack([step, -7.5 * step + 0.1 * rand(pages, G, page)], dim=-1).half()
        return {"v": v, "sz": sz, "kr": rand(pages, page, d_r).bfloat16()}
    kind = {"bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}[dtype]
    v = torch.empty(pages, G, page, d_v, dtype=kind, device="cuda")
    for lo in range(0, pages, 4096):
        n = min(4096, pages - lo)
        v[lo:lo + n] = rand(n, G, page, d_v).to(kind)
    return {"v": v, "kr": rand(pages, page, d_r).to(kind)}


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    rand = lambda *shape: torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)  # noqa: E731
    H, G, d_v, d_r = _HEADS[case["heads"]]
    B, page, kind = case["B"], case["page"], case["kind"]
    s = {"case": dict(case), "scale": 1.0 / math.sqrt(d_v + d_r)}
    if kind == "chunk":
        q, ctx = _spread(case["q_lo"], case["q_hi"], B), _spread(case["ctx_lo"], case["ctx_hi"], B)
        lens = [a + b for a, b in zip(q, ctx)]
        s["table"], pages, s["most"] = _paged(lens, page, gen)
        s["pools"] = _pools("q4", case["heads"], pages, page, gen)
        s["wide_table"], wide_pages, s["wide_most"] = _paged(lens, page, gen)
        s["wide_v"] = torch.zeros(wide_pages, G, page, d_v, dtype=torch.bfloat16, device="cuda")
        s["wide_kr"] = torch.zeros(wide_pages, page, d_r, dtype=torch.bfloat16, device="cuda")
        n = sum(q)
        s["v_new"] = rand(n, G, d_v) * (1.0 + 0.5 * rand(n, G, 1).abs()) + 0.2 * rand(n, G, 1)   # rows of their own width and middle
        s["kr_new"] = rand(n, d_r)
        s["cu_q"] = _ints(np.concatenate([[0], np.cumsum(q)]).tolist())
        s["ctx"], s["lens"] = _ints(ctx), _ints(lens)
        s["first_pos"] = _ints([c + 1000 * (i % 3) for i, c in enumerate(ctx)])     # tokens evicted before: positions run ahead of slots
        s["n"], s["max_len"] = n, max(lens)
        return _hold(s) if own else s
    lens = _spread(case["lo"], case["hi"], B)
    dtype = case.get("dtype", "q4")
    s["table"], pages, s["most"] = _paged(lens, page, gen)
    s["pools"] = _pools(dtype, case["heads"], pages, page, gen)
    s["lens"], s["max_len"] = _ints(lens), max(lens)
    if kind == "decode":
        s["q"] = rand(B, H, d_v + d_r)
        s["v_new"], s["kr_new"] = rand(B, G, d_v), rand(B, d_r)
        s["slots"] = _ints([t - 1 for t in lens])
        s["pos"] = _ints([t - 1 + 700 * (i % 3) for i, t in enumerate(lens)])
    elif kind == "weights":
        rows = _row_counts(case)
        s["q"] = 1.5 * rand(sum(rows), H, d_v + d_r)
        s["cu_q"] = _ints(np.concatenate([[0], np.cumsum(rows)]).tolist())
        s["rows"] = max(rows)
        s["decay"] = 0.75
        s["stride"] = s["max_len"] + 5
        s["w_in"] = (2.0 * rand(B, s["stride"])).exp() * 1e-3
        s["w_out"] = torch.zeros_like(s["w_in"])
        q, real, see = _rows_of(s)
        s["lse"] = torch.logsumexp(_scores(s, q).masked_fill(~see, -math.inf), dim=-1)[real].contiguous()   # as attention returned it
    else:
        s["stride"] = s["max_len"] + 5
        w = (2.0 * rand(B, s["stride"])).exp()
        s["w_in"] = torch.where(torch.rand(w.shape, generator=gen, device="cuda") < 0.05, torch.zeros_like(w), w)   # 5 % never looked at: ties
        gaps = torch.randint(1, 4, w.shape, generator=gen, device="cuda")
        at = torch.arange(s["stride"], device="cuda")
        mixed = torch.where(at < s["stride"] // 2, torch.rand(w.shape, generator=gen, device="cuda"), at.float() + 1.0)
        pos = torch.cumsum(gaps, dim=1)
        s["pos_in"] = pos.gather(1, mixed.argsort(dim=1)).to(torch.int32)                  # an earlier eviction has mixed the first half
        live = at < s["lens"][:, None]
        s["next_pos"] = (torch.where(live, s["pos_in"], torch.zeros_like(s["pos_in"])).amax(dim=1) + 1).to(torch.int32)
        s["keep"] = _ints([case["keep"]] * B)
        s["w_out"] = torch.zeros_like(s["w_in"])
        s["pos_out"] = torch.zeros_like(s["pos_in"])
        s["new_lens"] = torch.zeros_like(s["lens"])
    return _hold(s) if own else s


def _hold(s):
    """What a program that uses the library keeps beside its tensors: the handle, the workspace, its calls."""
    from paper_2609_13285_b200 import binding as gb

    case, pools = s["case"], s["pools"]
    H, G, d_v, d_r = _HEADS[case["heads"]]
    B, dtype = case["B"], case.get("dtype", "q4")
    h = gb.gva_create(H=H, G=G, d_v=d_v, d_c=d_v, d_r=d_r, page_size=case["page"], cache_dtype=gb.GVA_E4M3 if dtype == "fp8" else gb.GVA_BF16)
    kr = pools["kr"] if d_r else None
    if dtype == "q4":
        cache = gb.make_q4_cache(pools["v"], pools["sz"], kr, s["table"], pools["v"].shape[0], s["most"])
    else:
        cache = gb.make_cache(pools["v"], kr, s["table"], pools["v"].shape[0], s["most"])
    q4 = "gva_q4_" if dtype == "q4" else "gva_"
    if case["kind"] == "decode":
        s["out"] = torch.empty(B, H, d_v, device="cuda")
        s["lse"] = torch.empty(B, H, device="cuda")
        ws = torch.empty(gb.gva_q4_decode_workspace_bytes(h, B, s["max_len"]), dtype=torch.uint8, device="cuda")
        s["calls"] = [gb.prepare_call("gva_q4_append", h, cache, s["v_new"], s["kr_new"] if d_r else None, s["slots"], s["pos"], B, None),
                      gb.prepare_call("gva_q4_decode", h, cache, s["q"], s["lens"], s["out"], s["lse"], ws, ws.numel(), B, s["max_len"], 0, None)]
    elif case["kind"] == "chunk":
        wide = gb.make_cache(s["wide_v"], s["wide_kr"] if d_r else None, s["wide_table"], s["wide_v"].shape[0], s["wide_most"])
        s["calls"] = [gb.prepare_call("gva_q4_append_chunk", h, cache, s["v_new"], s["kr_new"] if d_r else None, s["cu_q"], s["ctx"], s["first_pos"], B, s["n"], None),
                      gb.prepare_call("gva_q4_widen", h, cache, wide, s["ctx"], s["lens"], B, s["max_len"], None)]
    elif case["kind"] == "weights":
        s["calls"] = [gb.prepare_call(q4 + "attention_weights", h, cache, s["q"], s["lse"], s["cu_q"], s["lens"], s["decay"], s["w_in"], s["w_out"], s["stride"], B, s["rows"],
                                      s["max_len"], None)]
    else:
        ws = torch.empty(gb.gva_evict_workspace_bytes(h, B, s["max_len"]), dtype=torch.uint8, device="cuda")
        s["calls"] = [gb.prepare_call(q4 + "evict", h, cache, s["w_in"], s["pos_in"], s["lens"], s["keep"], s["next_pos"], case["sinks"], case["recent"], s["w_out"], s["pos_out"],
                                      s["new_lens"], s["stride"], ws, ws.numel(), B, s["max_len"], None)]
    return s


# ----------------------------------------------------------------------------------------------------------- plain form
def _where(table, at, page):
    """(page number, slot in it) of the slots `at` [B][n] of every sequence."""
    return table.gather(1, (at // page).clamp(max=table.shape[1] - 1).long()).long(), (at % page).long()


def _rotated(x, pos):
    """x [n][d_r] rotated at pos [n]: pairs (2 i, 2 i + 1) by pos * base^(-2 i / d_r), in 64 bits."""
    d = x.shape[-1]
    angle = pos.double()[:, None] * _BASE ** (-2.0 * torch.arange(d // 2, device=x.device, dtype=torch.float64) / max(d, 1))
    c, s, a, b = angle.cos(), angle.sin(), x[:, 0::2].double(), x[:, 1::2].double()
    return torch.stack([a * c - b * s, a * s + b * c], dim=-1).reshape(x.shape)


def _half_below(x):
    """The largest 16-bit float that is not above x."""
    h = x.half()
    over, bits = h.double() > x.double(), h.view(torch.int16)
    below = torch.where(h > 0, bits - 1, torch.where(h < 0, bits + 1, torch.full_like(bits, -32767)))
    return torch.where(over, below, bits).view(torch.float16)


def _quantised(x):
    """Rows x [..][d] in 4 bits: (codes, step, lowest).  lowest = the row's minimum rounded down to 16 bits, step = the
    smallest 16-bit float with lowest + 15 step >= the row's maximum, code = the nearest multiple (a tie goes up).  Which
    side of a border a value falls on is decided in 64 bits, where all of these are exact."""
    x = x.clamp(-65504.0, 65504.0)
    low, high = _half_below(x.amin(dim=-1)), x.amax(dim=-1).double()
    bits = ((high - low.double()) / 15.0).half().view(torch.int16)
    reach = lambda b: low.double() + 15.0 * b.view(torch.float16).double()  # noqa: E731
    bits = torch.where(reach(bits) < high, bits + 1, bits)
    smaller = (bits - 1).clamp(min=0)
    bits = torch.where(reach(smaller) >= high, smaller, bits)
    step = bits.view(torch.float16)
    s, z = step.double()[..., None], low.double()[..., None]
    code = ((x.double() - z) / torch.where(s > 0, s, torch.ones_like(s))).round()
    code = torch.where(x.double() < z + (code - 0.5) * s, code - 1, code)
    code = torch.where(x.double() >= z + (code + 0.5) * s, code + 1, code)
    code = torch.where(s > 0, code.clamp(0, 15), torch.zeros_like(code))
    return code.to(torch.uint8), step, low


def _store(s, page_of, slot_of, v_new, kr_new, pos):
    pools = s["pools"]
    code, step, low = _quantised(v_new)
    pools["v"][page_of, :, slot_of] = code[..., 0::2] | (code[..., 1::2] << 4)
    pools["sz"][page_of, :, slot_of] = torch.stack([step, low], dim=-1)
    pools["kr"][page_of, slot_of] = _rotated(kr_new, pos).to(torch.bfloat16)


def _cached(s, dtype, at):
    """Values [B][n][G][d_v] and positional keys [B][n][d_r] of the slots `at` [B][n], in 32 bits."""
    pools = s["pools"]
    pg, slot = _where(s["table"], at, s["case"]["page"])
    kr = pools["kr"].view(torch.uint8)[pg, slot].view(pools["kr"].dtype).float() if dtype == "fp8" and pools["kr"].shape[-1] else pools["kr"][pg, slot].float()
    if dtype == "q4":
        byte = pools["v"][pg, :, slot]
        code = torch.stack([byte & 15, byte >> 4], dim=-1).flatten(-2).float()
        sz = pools["sz"][pg, :, slot].float()
        return code * sz[..., :1] + sz[..., 1:], kr
    if dtype == "fp8":
        return pools["v"].view(torch.uint8)[pg, :, slot].view(torch.float8_e4m3fn).float(), kr
    return pools["v"][pg, :, slot].float(), kr


def _slots(s):
    return torch.arange(s["max_len"], device="cuda")[None, :].expand(s["lens"].shape[0], -1)


def _scores(s, q, cached=None):
    """Scaled scores [B][R][H][T] of queries q [B][R][H][d_v + d_r] against every cached token."""
    H, G, d_v, d_r = _HEADS[s["case"]["heads"]]
    v, kr = cached if cached is not None else _cached(s, s["case"].get("dtype", "q4"), _slots(s))
    B, R = q.shape[:2]
    content = torch.einsum("brgjd,btgd->brgjt", q[..., :d_v].reshape(B, R, G, H // G, d_v), v).reshape(B, R, H, -1)
    return (content + torch.einsum("brhd,btd->brht", q[..., d_v:], kr)) * s["scale"]


def _rows_of(s):
    """The queries as [B][R][H][d_q], which (b, r) are real, and which tokens each sees [B][R][1][T]."""
    cu, B, R = s["cu_q"].long(), s["lens"].shape[0], s["rows"]
    count = (cu[1:] - cu[:-1])[:, None]
    r = torch.arange(R, device="cuda")[None, :]
    real = r < count
    q = s["q"][(cu[:-1, None] + r).clamp(max=s["q"].shape[0] - 1)]
    see = _slots(s)[:, None, :] < (s["lens"].long()[:, None] - (count - 1 - r))[:, :, None]
    return q, real, (see & real[:, :, None])[:, :, None, :]


def run(state):
    s, case = state, state["case"]
    kind = case["kind"]
    if own:
        for call in s["calls"]:
            call()
        if kind == "decode":
            return {"out": s["out"], "lse": s["lse"], "cache": s["pools"]}
        if kind == "chunk":
            return {"v": s["wide_v"], "kr": s["wide_kr"], "cache": s["pools"]}
        if kind == "weights":
            return {"weights": s["w_out"]}
        return _evicted(s)
    B, page = case["B"], case["page"]
    if kind == "decode":
        pg, slot = _where(s["table"], s["slots"][:, None], page)
        _store(s, pg[:, 0], slot[:, 0], s["v_new"], s["kr_new"], s["pos"])
        v, kr = _cached(s, "q4", _slots(s))
        x = _scores(s, s["q"][:, None], (v, kr))[:, 0].masked_fill((_slots(s) >= s["lens"][:, None])[:, None, :], -math.inf)
        top = x.amax(dim=-1, keepdim=True)
        p = (x - top).exp()
        total = p.sum(dim=-1, keepdim=True)
        G = v.shape[2]
        o = torch.einsum("bgjt,btgd->bgjd", (p / total).reshape(B, G, -1, p.shape[-1]), v)
        return {"out": o.reshape(B, -1, v.shape[-1]), "lse": (top + total.log())[..., 0], "cache": s["pools"]}
    if kind == "chunk":
        q_lens = (s["cu_q"][1:] - s["cu_q"][:-1]).long()
        b = torch.repeat_interleave(torch.arange(B, device="cuda"), q_lens)
        i = torch.arange(s["n"], device="cuda") - s["cu_q"].long()[b]
        at = s["ctx"].long()[b] + i
        pg, slot = s["table"].long()[b, at // page], at % page
        _store(s, pg, slot, s["v_new"], s["kr_new"], s["first_pos"][b] + i)
        pools = s["pools"]
        byte, sz = pools["v"][pg, :, slot], pools["sz"][pg, :, slot].float()
        wide = torch.stack([byte & 15, byte >> 4], dim=-1).flatten(-2).float() * sz[..., :1] + sz[..., 1:]
        to = s["wide_table"].long()[b, at // page]
        s["wide_v"][to, :, slot] = wide.bfloat16()
        s["wide_kr"][to, slot] = pools["kr"][pg, slot]
        return {"v": s["wide_v"], "kr": s["wide_kr"], "cache": s["pools"]}
    if kind == "weights":
        q, real, see = _rows_of(s)
        lse = torch.zeros(q.shape[:3], device="cuda")
        lse[real] = s["lse"]
        p = (_scores(s, q) - lse[..., None]).exp().masked_fill(~see, 0.0).sum(dim=(1, 2))
        n = s["max_len"]
        s["w_out"][:, :n] = torch.where(_slots(s) < s["lens"][:, None], s["decay"] * s["w_in"][:, :n] + p, s["w_out"][:, :n])
        return {"weights": s["w_out"]}
    n, at = s["max_len"], _slots(s)
    live = at < s["lens"][:, None]
    w, pos = s["w_in"][:, :n], s["pos_in"][:, :n]
    safe = (pos < case["sinks"]) | (pos >= s["next_pos"][:, None] - case["recent"])
    key = torch.where(safe, math.inf, torch.nan_to_num(w, nan=-math.inf, posinf=math.inf, neginf=-math.inf)).masked_fill(~live, -math.inf)
    keep = torch.minimum(s["keep"], s["lens"])
    order = key.argsort(dim=1, descending=True, stable=True)
    kept = torch.zeros_like(live).scatter(1, order, at < keep[:, None])
    first = at < keep[:, None]
    hb, ht = (first & ~kept).nonzero(as_tuple=True)        # holes, by sequence and slot
    mb, mt = (kept & ~first).nonzero(as_tuple=True)        # as many survivors behind the new end
    new_w = torch.where(first, w, 0.0)
    new_p = torch.where(first, pos, -1)
    new_w[hb, ht], new_p[hb, ht] = w[mb, mt], pos[mb, mt]
    s["w_out"][:, :n] = torch.where(live, new_w, s["w_out"][:, :n])
    s["pos_out"][:, :n] = torch.where(live, new_p, s["pos_out"][:, :n])
    s["new_lens"].copy_(keep)
    table = s["table"].long()
    for name, pool in s["pools"].items():
        pool = pool.view(torch.uint8) if pool.element_size() == 1 else pool
        if name == "kr":
            pool[table[hb, ht // page], ht % page] = pool[table[mb, mt // page], mt % page]
        else:
            pool[table[hb, ht // page], :, ht % page] = pool[table[mb, mt // page], :, mt % page]
    return _evicted(s)


def _evicted(s):
    """The state after an eviction.  Rows are moved bit for bit, so codes are compared as they stand."""
    got = {"weights": s["w_out"], "positions": s["pos_out"], "lens": s["new_lens"]}
    for name, pool in s["pools"].items():
        got[name] = pool.view(torch.uint8) if pool.element_size() == 1 else pool
    return got


# --------------------------------------------------------------------------------------------------------------- 64 bits
def _exact_rows(x):
    """Rows x [..][d] (numpy, 64 bits) as the 4-bit cache holds them: counts the borders below each value."""
    x = np.clip(x, -65504.0, 65504.0)
    low = x.min(axis=-1).astype(np.float16)
    low = np.where(low.astype(np.float64) > x.min(axis=-1), np.nextafter(low, np.float16(-np.inf)), low)
    z, high = low.astype(np.float64), x.max(axis=-1)
    step = ((high - z) / 15.0).astype(np.float16)
    for _ in range(2):
        step = np.where(z + 15.0 * step.astype(np.float64) < high, np.nextafter(step, np.float16(np.inf)), step)
    for _ in range(2):
        less = np.nextafter(step, np.float16(0))
        step = np.where((step > 0) & (z + 15.0 * less.astype(np.float64) >= high), less, step)
    s, code = step.astype(np.float64), np.zeros(x.shape)
    for k in range(15):
        code += (x >= (z + (k + 0.5) * s)[..., None]) & (s[..., None] > 0)
    return z[..., None] + s[..., None] * code


def _exact_rope(x, pos):
    out = np.empty(x.shape)
    for i in range(x.shape[-1] // 2):
        turn = np.exp(1j * pos * _BASE ** (-2.0 * i / x.shape[-1])) * (x[:, 2 * i] + 1j * x[:, 2 * i + 1])
        out[:, 2 * i], out[:, 2 * i + 1] = turn.real, turn.imag
    return out


def _exact_cache(s, b, n):
    """Values [n][G][d_v] and positional keys [n][d_r] of sequence b, page by page, in 64 bits."""
    page, pools = s["case"]["page"], s["pools"]
    ids = s["table"][b, : (n + page - 1) // page].long()
    wide = lambda name: pools[name].view(torch.uint8)[ids].view(pools[name].dtype).double() if pools[name].numel() else pools[name][ids].double()  # noqa: E731
    if s["case"].get("dtype", "q4") == "q4":
        byte, sz = pools["v"][ids].to(torch.int32), wide("sz")
        v = torch.empty(*byte.shape[:-1], 2 * byte.shape[-1], dtype=torch.float64, device="cuda")
        v[..., 0::2], v[..., 1::2] = byte % 16, byte // 16
        v = v * sz[..., 0:1] + sz[..., 1:2]
    else:
        v = wide("v")
    v = v.transpose(1, 2).reshape(len(ids) * page, v.shape[1], v.shape[3])[:n]
    kr = wide("kr")
    return v, kr.reshape(len(ids) * page, kr.shape[-1])[:n]


def exact(case, seed):
    s = prepare(case, seed)
    H, G, d_v, d_r = _HEADS[case["heads"]]
    B = case["B"]
    scale = 1.0 / math.sqrt(d_v + d_r)
    lens = s["lens"].tolist()
    if case["kind"] == "chunk":
        v, kr = s["wide_v"].double().cpu().numpy(), s["wide_kr"].double().cpu().numpy()
        if s["v_new"].numel() > 20_000_000:
            return None
        cu, ctx, first, table = (s[k].cpu().numpy() for k in ("cu_q", "ctx", "first_pos", "wide_table"))
        rows, keys = _exact_rows(s["v_new"].double().cpu().numpy()), s["kr_new"].double().cpu().numpy()
        for b in range(B):
            i = np.arange(cu[b + 1] - cu[b])
            at = ctx[b] + i
            to = table[b, at // case["page"]]
            v[to, :, at % case["page"]] = rows[cu[b]:cu[b + 1]]
            kr[to, at % case["page"]] = _exact_rope(keys[cu[b]:cu[b + 1]], (first[b] + i).astype(np.float64))
        return {"v": torch.from_numpy(v), "kr": torch.from_numpy(kr), "cache": None}
    if case["kind"] == "decode":
        rows = torch.from_numpy(_exact_rows(s["v_new"].double().cpu().numpy())).cuda()
        keys = _exact_rope(s["kr_new"].double().cpu().numpy(), s["pos"].double().cpu().numpy())
        keys = torch.from_numpy(keys).cuda().to(torch.bfloat16).double()             # as the cache holds them
        out = torch.empty(B, H, d_v, dtype=torch.float64, device="cuda")
        lse = torch.empty(B, H, dtype=torch.float64, device="cuda")
        for b, n in enumerate(lens):
            v, kr = _exact_cache(s, b, n)
            v[n - 1], kr[n - 1] = rows[b], keys[b]
            for h in range(H):
                vg, q = v[:, h // (H // G)], s["q"][b, h].double()
                x = (vg @ q[:d_v] + kr @ q[d_v:]) * scale
                lse[b, h] = torch.logsumexp(x, 0)
                out[b, h] = vg.T @ (x - lse[b, h]).exp()
        return {"out": out, "lse": lse, "cache": None}
    if case["kind"] == "weights":
        got, cu = s["w_out"].double(), s["cu_q"].tolist()
        for b, n in enumerate(lens):
            v, kr = _exact_cache(s, b, n)
            total = s["decay"] * s["w_in"][b, :n].double()
            for r in range(cu[b], cu[b + 1]):
                m = n - (cu[b + 1] - 1 - r)
                if m > 0:
                    for g in range(G):
                        heads = slice(g * (H // G), (g + 1) * (H // G))
                        q = s["q"][r, heads].double()
                        x = (v[:m, g] @ q[:, :d_v].T + kr[:m] @ q[:, d_v:].T) * scale
                        total[:m] += (x - s["lse"][r, heads].double()).exp().sum(dim=1)
            got[b, :n] = total
        return {"weights": got}
    w, pos, nxt = s["w_in"].double().cpu().numpy(), s["pos_in"].cpu().numpy(), s["next_pos"].tolist()
    got = np.zeros(w.shape)
    for b, n in enumerate(lens):
        keep = min(case["keep"], n)
        safe = (pos[b, :n] < case["sinks"]) | (pos[b, :n] >= nxt[b] - case["recent"])
        ranked = np.lexsort((np.arange(n), -w[b, :n], ~safe))
        # those safe come first, by slot; of the others the heavier, by slot where they weigh the same
        ranked = np.concatenate([np.sort(ranked[: int(safe.sum())]), ranked[int(safe.sum()):]])
        stay = np.sort(ranked[:keep])
        got[b, stay[stay < keep]] = w[b, stay[stay < keep]]
        got[b, np.setdiff1d(np.arange(keep), stay)] = w[b, stay[stay >= keep]]
    return {"weights": torch.from_numpy(got), "positions": None, "lens": None, **{k: None for k in s["pools"]}}
