"""The operators of a serving step whose new tokens are a tree of drafts, as cases to be timed and compared.

A serving program drafts several continuations of every sequence at once, as a tree, and lets the model look at all of them
in one step.  Four kinds of case stand for that step:

  plan     pages are given out and taken back, and every new row gets its sequence, position and slot; with a tree, which of
           the other drafted tokens each one sees (assign_pages, tree_masks)
  append   the new rows are rotated to their positions and written to the pages through the slot map: keys, values and queries
           of the matched GQA cache (gqa_append), or the grouped values with their positional key (gva_append_rows)
  tree     attention of the drafted tokens over the cache: all of the context, and of the drafts their own ancestors
  commit   the drafts that the model agrees with become part of the sequence, and the cache closes up behind them

`run` is the plain form in elementary torch operations, or, where `own` is set, the library's calls.
"""
import math

import numpy as np
import torch

own = False

# head layouts (H, G, d_v, d_r): the ones the repository's tests and benchmark use (d_c = d_v everywhere)
_HEADS = {"a": (16, 4, 64, 16), "b": (32, 8, 128, 32), "c": (16, 4, 64, 24), "a0": (16, 4, 64, 0), "b0": (32, 8, 128, 0),
          "g1": (4, 1, 64, 16), "g2": (8, 2, 128, 32), "g8": (32, 8, 64, 16), "g3": (12, 3, 64, 0)}
_BASE = 10000.0


# ---------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # four chats in the middle of an answer: one token each
        {"name": "plan-b4-decode", "kind": "plan", "B": 4, "lo": 90, "hi": 2000, "new_lo": 1, "new_hi": 1, "tree": False, "done": 0, "page": 64},
        # a full batch with a tree for every sequence, a few of them done with their answers
        {"name": "plan-b256-trees", "kind": "plan", "B": 256, "lo": 100, "hi": 9000, "new_lo": 1, "new_hi": 40, "tree": True, "done": 9, "page": 64},
        # 48 prompts come in, odd lengths up to 8192 tokens: 0.2 M rows
        {"name": "plan-b48-prompts", "kind": "plan", "B": 48, "lo": 0, "hi": 0, "new_lo": 777, "new_hi": 8192, "tree": False, "done": 0, "page": 64},
        # one user's next token: e4m3 cache, narrow heads, halves of the whole head
        {"name": "append-gqa-fp8-n1", "kind": "append", "form": "gqa", "heads": "a", "dtype": "fp8", "n": 1, "far": 3000, "layout": "halves", "d_rot": 64, "scaling": "plain", "page": 64},
        # the trees of a batch over the grouped values: rows of several sequences, positions that repeat
        {"name": "append-gva-n500", "kind": "append", "form": "gva", "heads": "a", "dtype": "bf16", "n": 500, "far": 32768, "page": 64},
        # whole prompts of a prefill batch, wide heads, half of each head rotated, a context eight times the trained one
        {"name": "append-gqa-n65536-wide", "kind": "append", "form": "gqa", "heads": "b", "dtype": "bf16", "n": 65536, "far": 65536, "layout": "pairs", "d_rot": 64, "scaling": "parts", "page": 64},
        # one user, a short chat, five drafted tokens: nothing but latency
        {"name": "tree-b1-t97-n5", "kind": "tree", "heads": "a", "B": 1, "lo": 97, "hi": 97, "n_lo": 5, "n_hi": 5, "page": 64},
        # a small batch at ordinary lengths, odd ones, 48-byte positional rows, small pages
        {"name": "tree-b7-ragged-n24-dr24", "kind": "tree", "heads": "c", "B": 7, "lo": 301, "hi": 4999, "n_lo": 1, "n_hi": 24, "page": 32},
        # the long-context batch of the benchmark, 1 M cached tokens, sixteen drafts each
        {"name": "tree-b32-t32768-n16", "kind": "tree", "heads": "a", "B": 32, "lo": 32768, "hi": 32768, "n_lo": 16, "n_hi": 16, "page": 64},
        # the ragged wide-head batch of the benchmark with large trees
        {"name": "tree-b64-ragged-wide-n64", "kind": "tree", "heads": "b", "B": 64, "lo": 1024, "hi": 16384, "n_lo": 9, "n_hi": 64, "page": 64},
        # two chats with a small tree
        {"name": "commit-b2-n8", "kind": "commit", "heads": "a", "dtype": "bf16", "B": 2, "lo": 90, "hi": 1500, "n_lo": 5, "n_hi": 8, "page": 64},
        # a full batch with large trees, wide heads
        {"name": "commit-b256-n64-wide", "kind": "commit", "heads": "b", "dtype": "bf16", "B": 256, "lo": 100, "hi": 2000, "n_lo": 9, "n_hi": 64, "page": 64},
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["plan", "append", "append", "tree", "tree", "tree", "commit"])
    page = rng.choice([32, 64, 64, 128, 256])
    if kind == "plan":
        form = rng.choice(["decode", "tree", "prompt"])
        B = log(1, 1000)
        hi = log(1, 20000)
        case = {"kind": kind, "B": B, "lo": max(0, int(hi * rng.uniform(0.0, 1.0))), "hi": hi, "new_lo": 1, "new_hi": 1, "tree": form == "tree",
                "done": rng.choice([0, 0, 3, 7]), "page": page}
        if form == "tree":
            case["new_hi"] = log(1, 64)
        if form == "prompt":
            case.update(lo=0, hi=rng.choice([0, log(1, 5000)]), new_hi=min(log(1, 8192), 200_000 // B))
            case["new_lo"] = max(1, int(case["new_hi"] * rng.uniform(0.1, 1.0)))
        return case
    heads = rng.choice(["a", "a", "b", "c", "a0", "b0", "g1", "g2", "g8", "g3"])
    H, G, d_v, d_r = _HEADS[heads]
    if kind == "append":
        case = {"kind": kind, "heads": heads, "page": page, "form": rng.choice(["gqa", "gqa", "gva"]), "far": log(10, 200_000)}
        case["n"] = min(log(1, 65536), 65536 * 32 * 128 // (H * d_v))
        if case["form"] == "gqa":
            case["dtype"] = rng.choice(["bf16", "bf16", "fp8", "f32"]) if page % 64 == 0 and heads != "c" else rng.choice(["bf16", "f32"])
            case.update(layout=rng.choice(["pairs", "halves"]), d_rot=rng.choice([d_v, d_v, d_v // 2, 8 * rng.randint(1, d_v // 8)]),
                        scaling=rng.choice(["plain", "linear", "base", "parts"]))
        else:
            case["dtype"] = rng.choice(["bf16", "fp8", "f32"]) if page % 64 == 0 and heads != "c" else rng.choice(["bf16", "f32"])
        return case
    if kind == "commit":
        case = {"kind": kind, "heads": heads, "page": page, "B": log(1, 256), "n_hi": log(1, 64)}
        case["dtype"] = rng.choice(["bf16", "fp8", "f32"]) if page % 64 == 0 and heads != "c" else rng.choice(["bf16", "f32"])
        case["hi"] = min(log(1, 20000), 512_000 // case["B"])
        case["lo"] = max(0, int(case["hi"] * rng.uniform(0.1, 1.0)))
        case["n_lo"] = max(1, int(case["n_hi"] * rng.uniform(0.1, 1.0)))
        return case
    wide = d_v * G // 256 or 1                                      # a token's size against the narrow layout's
    B = log(1, 64)
    t = min(log(1, 40000), 32 * 32768 // wide // B)
    n = min(log(1, 64), max(1, 180_000_000_000 // (B * t * H * (2 * d_v + d_r))))
    return {"kind": kind, "heads": heads, "page": page, "B": B, "lo": max(0, int(t * rng.choice([1.0, rng.uniform(0.05, 1.0)]))), "hi": t,
            "n_lo": max(1, int(n * rng.choice([1.0, rng.uniform(0.1, 1.0)]))), "n_hi": n}


def _spread(lo, hi, n):
    """n whole numbers over [lo, hi], the same for every seed; the largest is hi."""
    return [hi if i == 0 else lo + int((hi - lo) * ((i * 0.6180339887) % 1.0)) for i in range(n)]


def _element(dtype):
    return {"bf16": 2, "fp8": 1, "f32": 4}[dtype]


def _plan_lens(case):
    """Tokens that every sequence has, and that it asks for (none once it is done)."""
    used = _spread(case["lo"], case["hi"], case["B"])
    new = _spread(case["new_lo"], case["new_hi"], case["B"])
    done = case["done"]
    return used, [0 if done and i % done == done - 1 else u + n for i, (u, n) in enumerate(zip(used, new))]


def work(case):
    kind = case["kind"]
    if kind == "plan":
        used, want = _plan_lens(case)
        P = case["page"]
        rows = sum(max(w - u, 0) for u, w in zip(used, want))
        pages = sum(abs((w + P - 1) // P - (u + P - 1) // P) for u, w in zip(used, want))
        words = (max(max(w - u, 0) for u, w in zip(used, want)) + 31) // 32
        return {"bytes": 4 * (7 * case["B"] + 2 * pages + 2 * rows + (rows * (2 + words) if case["tree"] else 0)), "flops": 0}
    H, G, d_v, d_r = _HEADS[case["heads"]]
    if kind == "append":
        n, e = case["n"], _element(case["dtype"])
        if case["form"] == "gva":
            return {"bytes": n * (8 + (G * d_v + d_r) * (4 + e)), "flops": 3 * n * d_r}
        return {"bytes": n * (8 + 4 * (2 * H + 2 * G) * d_v + 2 * G * d_v * e), "flops": 3 * n * (H + G) * case["d_rot"]}
    ctx, nodes = _spread(case["lo"], case["hi"], case["B"]), _spread(case["n_lo"], case["n_hi"], case["B"])
    if kind == "commit":
        # a third of the tree's rows at most move, each read and written
        moved = sum(max(0, a - f) for a, f in (_accepted(n) for n in nodes))
        return {"bytes": 16 * sum(nodes) + moved * 2 * _element(case["dtype"]) * (G * d_v + d_r), "flops": 0}
    words = (max(nodes) + 31) // 32
    seen = sum(n * (t + (n + 1) / 2) for t, n in zip(ctx, nodes))
    return {"bytes": 2 * (G * d_v + d_r) * (sum(ctx) + sum(nodes)) + sum(nodes) * (2 * H * (2 * d_v + d_r) + 4 * H + 4 * words),
            "flops": 2 * seen * H * (2 * d_v + d_r)}


# --------------------------------------------------------------------------------------------------------------- inputs
def _ints(values):
    return torch.tensor(np.asarray(values), dtype=torch.int32, device="cuda")


def _paged(lens, page, gen):
    """Block table [B][max_pages] with the pages in a random order, a few pages left over; numbers of pages."""
    most = max(1, max((t + page - 1) // page for t in lens))
    pages = len(lens) * most + 3
    table = torch.randperm(pages, generator=gen, device="cuda")[: len(lens) * most].to(torch.int32).reshape(len(lens), most)
    return table.contiguous(), pages, most


def _pool(shape, dtype, gen):
    kind = {"bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn, "f32": torch.float32}[dtype]
    pool = torch.empty(shape, dtype=kind, device="cuda")
    for lo in range(0, shape[0], 4096):
        pool[lo:lo + 4096] = torch.randn(pool[lo:lo + 4096].shape, generator=gen, device="cuda").to(kind)
    return pool


def _parents(nodes, rng):
    """Parents of the nodes of every sequence's tree, -1 for the first: the earlier a node the more children it has."""
    got = []
    for n in nodes:
        i = np.arange(n)
        got.append(np.where(i == 0, -1, np.floor(i * rng.random_sample(n) ** 1.5)))
    return np.concatenate(got).astype(np.int32) if got else np.zeros(0, np.int32)


def _accepted(n):
    """(length of the accepted path in a tree of n nodes, how much of it lies at the tree's beginning)."""
    a = 1 + (n * 7) % max(1, min(6, (n + 2) // 3))
    return a, 1 + (n * 5) % a


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    rng = np.random.RandomState(int(seed) % (1 << 31))
    rand = lambda *shape: torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)  # noqa: E731
    kind, page = case["kind"], case["page"]
    s = {"case": dict(case)}
    if kind == "plan":
        used, want = _plan_lens(case)
        B = case["B"]
        held = [(u + page - 1) // page + (1 if i % 5 == 4 else 0) for i, u in enumerate(used)]      # a page ahead, left by a larger tree
        tp = [(w + page - 1) // page for w in want]
        s["most"] = max(1, max(held + tp))
        take = sum(max(t - h, 0) for t, h in zip(tp, held))
        s["num_pages"] = sum(held) + take + 11
        order = torch.randperm(s["num_pages"], generator=gen, device="cuda").to(torch.int32)
        s["table"] = torch.full((B, s["most"]), -1, dtype=torch.int32, device="cuda")
        mine = torch.arange(s["most"], device="cuda")[None, :] < _ints(held)[:, None]
        s["table"][mine] = order[: sum(held)]
        free = order[sum(held):]
        s["first"] = int(rng.randint(s["num_pages"]))
        s["ring"] = torch.full((s["num_pages"],), -1, dtype=torch.int32, device="cuda")
        s["ring"][(s["first"] + torch.arange(len(free), device="cuda")) % s["num_pages"]] = free
        s["free"], s["free_out"] = _ints([s["first"], len(free)]), _ints([0, 0])
        s["used"], s["want"], s["held"] = _ints(used), _ints(want), _ints(held)
        s["lens"], s["pages"], s["cu_q"] = _ints([0] * B), _ints([0] * B), _ints([0] * (B + 1))
        rows = [max(w - u, 0) for u, w in zip(used, want)]
        s["rows"] = sum(rows) + 5
        s["pos"], s["slots"] = _ints(np.zeros(s["rows"])), _ints(np.zeros(s["rows"]))
        if case["tree"]:
            s["most_nodes"] = max(rows)
            s["words"] = (max(rows) + 31) // 32
            s["parents"] = _ints(np.concatenate([_parents(rows, rng), np.full(5, -1)]))
            s["mask"], s["depth_pos"] = _ints(np.zeros((s["rows"], s["words"]))), _ints(np.zeros(s["rows"]))
        return _hold(s) if own else s
    H, G, d_v, d_r = _HEADS[case["heads"]]
    if kind == "append":
        n, far = case["n"], case["far"]
        pages = (n + 40 + page - 1) // page + 3
        slots = torch.randperm(pages * page, generator=gen, device="cuda")[:n].to(torch.int32)
        s["slots"] = torch.sort(slots)[0] if n > 64 else slots      # long runs lie in order, as those of a prompt do
        s["pos"] = (far - 1 - torch.randint(0, max(1, far // 2), (n,), generator=gen, device="cuda")).to(torch.int32)
        if case["form"] == "gva":
            s["v_new"], s["kr_new"] = rand(n, G, d_v), rand(n, d_r)
            s["pools"] = {"v": _pool((pages, G, page, d_v), case["dtype"], gen), "kr": _pool((pages, page, d_r), case["dtype"], gen)}
        else:
            # one row of a packed projection: queries, keys, values
            s["qkv"] = rand(n, H + 2 * G, d_v)
            s["q_out"] = torch.empty(n, H, d_v, device="cuda")
            s["pools"] = {"k": _pool((pages, G, page, d_v), case["dtype"], gen), "v": _pool((pages, G, page, d_v), case["dtype"], gen)}
            s["rope"] = {"plain": {}, "linear": {"factor": 4.0}, "base": {"factor": 4.0},
                         "parts": {"factor": 8.0, "low": 1.0, "high": 4.0, "original_len": 8192, "magnitude": 1.2079}}[case["scaling"]]
        return _hold(s) if own else s
    ctx, nodes = _spread(case["lo"], case["hi"], case["B"]), _spread(case["n_lo"], case["n_hi"], case["B"])
    lens = [t + n for t, n in zip(ctx, nodes)]
    s["table"], pages, s["most"] = _paged(lens, page, gen)
    s["ctx"], s["cu_q"] = _ints(ctx), _ints(np.concatenate([[0], np.cumsum(nodes)]))
    s["n"], s["most_nodes"], s["max_len"] = sum(nodes), max(nodes), max(lens)
    s["pools"] = {"v": _pool((pages, G, page, d_v), case.get("dtype", "bf16"), gen), "kr": _pool((pages, page, d_r), case.get("dtype", "bf16"), gen)}
    if kind == "tree":
        s["words"] = (s["most_nodes"] + 31) // 32
        s["q"] = (1.5 * rand(s["n"], H, d_v + d_r)).bfloat16()
        s["mask"] = _masks(_ints(_parents(nodes, rng)), s["cu_q"], s["most_nodes"], s["words"])[0]
        return _hold(s) if own else s
    # the accepted path lies at the tree's beginning and then behind its own length, as in a tree kept level by level
    parents, tokens, chosen = [], [], []
    for n in nodes:
        a, f = _accepted(n)
        path = np.concatenate([np.arange(f), np.sort(rng.permutation(np.arange(a, n))[: a - f])]) if n - a >= a - f else np.arange(a)
        par = np.where(np.arange(n) == 0, -1, np.floor(np.arange(n) * rng.random_sample(n) ** 1.5)).astype(np.int64)
        par[path[1:]] = path[:-1]
        tok = 2 * rng.randint(0, 16000, n)
        cho = tok[rng.randint(0, n, n)] + 1                          # an odd token: none of those drafted
        cho[path[:-1]] = tok[path[1:]]
        for i, j in zip(path[:-1], path[1:]):                        # and no sibling in front of it says the same
            same = (par[:j] == i) & (tok[:j] == tok[j])
            tok[:j][same] += 2
        parents.append(par), tokens.append(tok), chosen.append(cho)
    s["parents"], s["tokens"], s["chosen"] = (_ints(np.concatenate(x)) for x in (parents, tokens, chosen))
    s["path"] = _ints(np.full(s["n"], -7))
    s["lens"], s["last"] = _ints([0] * case["B"]), _ints([0] * case["B"])
    return _hold(s) if own else s


def _hold(s):
    """What a program that uses the library keeps beside its tensors: the handle, the workspace, its calls."""
    from paper_2609_13285_b200 import binding as gb

    case, kind = s["case"], s["case"]["kind"]
    H, G, d_v, d_r = _HEADS[case.get("heads", "a")]
    dtype = {"bf16": gb.GVA_BF16, "fp8": gb.GVA_E4M3, "f32": gb.GVA_F32}[case.get("dtype", "bf16")]
    h = gb.gva_create(H=H, G=G, d_v=d_v, d_c=d_v, d_r=d_r, page_size=case["page"], cache_dtype=dtype)
    if kind == "plan":
        B = case["B"]
        s["calls"] = [gb.prepare_call("gva_assign_pages", h, s["used"], s["want"], s["held"], s["pages"], s["table"], s["most"], s["num_pages"], s["ring"], s["free"],
                                      s["free_out"], s["lens"], s["cu_q"], s["pos"], s["slots"], s["rows"], B, None)]
        if case["tree"]:
            s["calls"].append(gb.prepare_call("gva_tree_masks", h, s["parents"], s["cu_q"], s["used"], s["mask"], s["words"], s["depth_pos"], B, s["most_nodes"], None))
        return s
    pools = s["pools"]
    if kind == "append" and case["form"] == "gqa":
        rope = {"plain": gb.GVA_ROPE_PLAIN, "linear": gb.GVA_ROPE_LINEAR, "base": gb.GVA_ROPE_BASE, "parts": gb.GVA_ROPE_PARTS}[case["scaling"]]
        gb.gqa_set_rope(h, gb.make_rope(layout=gb.GVA_ROPE_HALVES if case["layout"] == "halves" else gb.GVA_ROPE_PAIRS, d_rot=case["d_rot"], base=_BASE, scaling=rope, **s["rope"]))
        cache = gb.make_gqa_cache(pools["k"], pools["v"], None, pools["k"].shape[0], pools["k"].shape[0])
        row = (H + 2 * G) * d_v
        q, k, v = s["qkv"][:, :H], s["qkv"][:, H:H + G], s["qkv"][:, H + G:]
        s["calls"] = [gb.prepare_call("gqa_append", h, cache, q, row, k, row, v, row, s["pos"], s["slots"], s["q_out"], case["n"], None)]
        return s
    kr = pools["kr"] if d_r else None
    if kind == "append":
        cache = gb.make_cache(pools["v"], kr, None, pools["v"].shape[0], pools["v"].shape[0])
        s["calls"] = [gb.prepare_call("gva_append_rows", h, cache, s["v_new"], s["kr_new"] if d_r else None, s["pos"], s["slots"], case["n"], None)]
        return s
    cache = gb.make_cache(pools["v"], kr, s["table"], pools["v"].shape[0], s["most"])
    B = case["B"]
    if kind == "tree":
        s["out"] = torch.empty(s["n"], H, d_v, dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.empty(s["n"], H, device="cuda")
        ws = torch.empty(gb.gva_decode_tree_workspace_bytes(h, B, s["n"], s["most_nodes"], s["max_len"]), dtype=torch.uint8, device="cuda")
        s["calls"] = [gb.prepare_call("gva_decode_tree", h, cache, s["q"], s["mask"], s["words"], s["cu_q"], s["ctx"], s["out"], s["lse"], ws, ws.numel(), B, s["n"],
                                      s["most_nodes"], s["max_len"], 0, None)]
    else:
        s["calls"] = [gb.prepare_call("gva_tree_commit", h, cache, s["parents"], s["tokens"], s["chosen"], s["cu_q"], s["ctx"], s["path"], s["lens"], s["last"], B,
                                      s["most_nodes"], None)]
    return s


# ----------------------------------------------------------------------------------------------------------- plain form
def _trees(parents, cu, most):
    """What every node sees of its own tree, itself included: [B][N][N] (the closure of `is my parent`), and which nodes are real."""
    cu = cu.long()
    i = torch.arange(most, device="cuda")
    real = i[None, :] < (cu[1:] - cu[:-1])[:, None]
    par = parents.long()[(cu[:-1, None] + i).clamp(max=max(0, parents.numel() - 1))]
    up = (par[:, :, None] == i) | torch.eye(most, dtype=torch.bool, device="cuda")
    for _ in range(max(1, most).bit_length()):                      # paths twice as long each time
        up = torch.bmm(up.float(), up.float()) > 0
    return up & real[:, :, None], real


def _masks(parents, cu, most, words):
    """Bit j of a row: it sees node j of its tree ([rows][words], 32 bits each); and its depth."""
    up, real = _trees(parents, cu, most)
    up = up[real]
    bits = torch.zeros(up.shape[0], words * 32, dtype=torch.int64, device="cuda")
    bits[:, :most] = up
    word = (bits.reshape(-1, words, 32) << torch.arange(32, device="cuda")).sum(dim=-1)
    return torch.where(word >= 1 << 31, word - (1 << 32), word).to(torch.int32), up.sum(dim=-1) - 1


def _frequencies(case, rope):
    d = case["d_rot"]
    i = torch.arange(d // 2, device="cuda", dtype=torch.float64)
    base = _BASE * rope["factor"] ** (d / (d - 2)) if case["scaling"] == "base" else _BASE
    f = base ** (-2.0 * i / d)
    if case["scaling"] == "linear":
        f = f / rope["factor"]
    if case["scaling"] == "parts":
        turns = rope["original_len"] * f / (2.0 * math.pi)
        part = ((turns - rope["low"]) / (rope["high"] - rope["low"])).clamp(0.0, 1.0)
        f = f * (part + (1.0 - part) / rope["factor"])
    return f


def _turned(x, cos, sin, halves, d):
    """Heads x [n][heads][..] with their first d elements rotated; cos, sin [n][d / 2]."""
    head, cos, sin = x[..., :d], cos[:, None], sin[:, None]
    a, b = (head[..., : d // 2], head[..., d // 2:]) if halves else (head[..., 0::2], head[..., 1::2])
    u, v = a * cos - b * sin, a * sin + b * cos
    got = torch.cat([u, v], dim=-1) if halves else torch.stack([u, v], dim=-1).flatten(-2)
    return torch.cat([got, x[..., d:]], dim=-1)


def _rotated(x, pos):
    """x [n][d_r] rotated at pos [n]: pairs (2 i, 2 i + 1) by pos * base^(-2 i / d_r), in 64 bits."""
    d = x.shape[-1]
    angle = pos.double()[:, None] * _BASE ** (-2.0 * torch.arange(d // 2, device=x.device, dtype=torch.float64) / max(d, 1))
    return _turned(x.double()[:, None], angle.cos(), angle.sin(), False, d)[:, 0]


def _put(pool, slots, rows, page):
    """rows into the slots of a pool [pages][G][page][d] or [pages][page][d]."""
    slots = slots.long()
    rows = rows.clamp(-448.0, 448.0).to(pool.dtype) if pool.dtype == torch.float8_e4m3fn else rows.to(pool.dtype)
    if pool.element_size() == 1:
        pool, rows = pool.view(torch.uint8), rows.view(torch.uint8)
    if pool.dim() == 4:
        pool[slots // page, :, slots % page] = rows
    else:
        pool[slots // page, slots % page] = rows


def _plan(s):
    P, N = s["case"]["page"], s["num_pages"]
    used, want, held = s["used"].long(), s["want"].long(), s["held"].long()
    first, count = s["free"][0].long(), s["free"][1].long()
    to, rows = (want + P - 1) // P, (want - used).clamp(min=0)
    take = (to - held).clamp(min=0)
    grows = (rows > 0) | (take > 0)
    served = ~grows | ((take.cumsum(0) <= count) & (rows.cumsum(0) <= s["rows"]))
    to, rows, take = torch.where(served, to, held), torch.where(served, rows, 0), torch.where(served, take, 0)
    give = (held - to).clamp(min=0)
    s["pages"].copy_(to)
    s["lens"].copy_(torch.where(served, want, used))
    s["cu_q"][1:] = rows.cumsum(0)
    seq = torch.arange(len(used), device="cuda")

    def each(counts):
        """(sequence, number within it, number in all) of counts[b] things of every sequence b."""
        b = torch.repeat_interleave(seq, counts)
        at = torch.arange(len(b), device="cuda")
        return b, at - (counts.cumsum(0) - counts)[b], at

    b, i, at = each(take)
    s["table"][b, held[b] + i] = s["ring"][(first + at) % N]
    b, i, at = each(give)
    s["ring"][(first + count + at) % N] = s["table"][b, to[b] + i]
    s["free_out"].copy_(torch.stack([(first + take.sum()) % N, count - take.sum() + give.sum()]))
    b, i, at = each(rows)
    pos = used[b] + i
    s["pos"][at] = pos.to(torch.int32)
    s["slots"][at] = (s["table"].long()[b, pos // P] * P + pos % P).to(torch.int32)
    return b


def run(state):
    s, case = state, state["case"]
    kind, page = case["kind"], case["page"]
    if own:
        for call in s["calls"]:
            call()
        return _outputs(s)
    if kind == "plan":
        b = _plan(s)
        if case["tree"]:
            n = len(b)
            mask, depth = _masks(s["parents"], s["cu_q"], s["most_nodes"], s["words"])
            s["mask"][:n] = mask
            s["depth_pos"][:n] = s["used"][b] + depth.to(torch.int32)
        return _outputs(s)
    H, G, d_v, d_r = _HEADS[case["heads"]]
    if kind == "append" and case["form"] == "gva":
        _put(s["pools"]["v"], s["slots"], s["v_new"], page)
        if d_r:
            _put(s["pools"]["kr"], s["slots"], _rotated(s["kr_new"], s["pos"]), page)
        return _outputs(s)
    if kind == "append":
        angle = s["pos"].double()[:, None] * _frequencies(case, s["rope"])
        m = s["rope"].get("magnitude", 1.0)
        cos, sin = (m * angle.cos()).float(), (m * angle.sin()).float()
        turned = _turned(s["qkv"][:, : H + G], cos, sin, case["layout"] == "halves", case["d_rot"])
        s["q_out"].copy_(turned[:, :H])
        _put(s["pools"]["k"], s["slots"], turned[:, H:], page)
        _put(s["pools"]["v"], s["slots"], s["qkv"][:, H + G:], page)
        return _outputs(s)
    B, table = case["B"], s["table"].long()
    cu, ctx = s["cu_q"].long(), s["ctx"].long()
    if kind == "tree":
        t = torch.arange(s["max_len"], device="cuda")
        pg = table[:, t // page]
        v = s["pools"]["v"][pg, :, t % page].float()                               # [B][T][G][d_v]
        kr = s["pools"]["kr"][pg, t % page].float()
        r = torch.arange(s["most_nodes"], device="cuda")
        count = (cu[1:] - cu[:-1])[:, None]
        real = r < count
        at = (cu[:-1, None] + r).clamp(max=s["n"] - 1)
        q = s["q"][at].float()                                                     # [B][R][H][d_v + d_r]
        R = len(r)
        x = torch.einsum("brgjd,btgd->brgjt", q[..., :d_v].reshape(B, R, G, H // G, d_v), v).reshape(B, R, H, -1)
        x = (x + torch.einsum("brhd,btd->brht", q[..., d_v:], kr)) / math.sqrt(d_v + d_r)
        i = t[None, :] - ctx[:, None]                                              # which draft a slot holds
        word = s["mask"][at].long().gather(2, (i.clamp(0, 32 * s["words"] - 1) // 32)[:, None, :].expand(-1, R, -1))
        bit = (word >> (i.clamp(min=0) % 32)[:, None, :]) & 1
        see = (i < 0)[:, None, :] | ((bit == 1) & (i < count)[:, None, :])
        x = x.masked_fill(~see[:, :, None, :], -math.inf)
        top = x.amax(dim=-1, keepdim=True)
        top = torch.where(top == -math.inf, 0.0, top)
        p = (x - top).exp()
        total = p.sum(dim=-1, keepdim=True)
        o = torch.einsum("brgjt,btgd->brgjd", (p / torch.where(total > 0, total, 1.0)).reshape(B, R, G, H // G, -1), v).reshape(B, R, H, d_v)
        return {"out": o[real].bfloat16(), "lse": (top + total.log())[..., 0][real]}
    up, real = _trees(s["parents"], s["cu_q"], s["most_nodes"])
    r = torch.arange(s["most_nodes"], device="cuda")
    at = (cu[:-1, None] + r).clamp(max=s["n"] - 1)
    par, tok, cho = (s[k].long()[at] for k in ("parents", "tokens", "chosen"))
    said = real & (par >= 0) & (tok == cho.gather(1, par.clamp(min=0)))            # the model says this token after the parent
    twin = (par[:, :, None] == par[:, None, :]) & said[:, :, None] & said[:, None, :] & (r[None, :] < r[:, None])
    good = (said & ~twin.any(dim=-1)) | ((r == 0) & real)
    taken = real & ~(up & ~good[:, None, :]).any(dim=-1)                           # every ancestor is good
    count = taken.sum(dim=1)
    path = torch.where(taken, r, s["most_nodes"]).sort(dim=1)[0]
    s["path"].copy_(torch.where(r < count[:, None], path, -1)[real])
    s["lens"].copy_(ctx + count)
    s["last"].copy_(torch.where(count > 0, cho.gather(1, path.gather(1, (count - 1).clamp(min=0)[:, None]).clamp(max=s["most_nodes"] - 1))[:, 0], -1))
    b, i = ((r < count[:, None]) & (path != r)).nonzero(as_tuple=True)
    src, dst = ctx[b] + path[b, i], ctx[b] + i
    for name, pool in s["pools"].items():
        pool = pool.view(torch.uint8) if pool.element_size() == 1 else pool
        if name == "kr":
            pool[table[b, dst // page], dst % page] = pool[table[b, src // page], src % page]
        else:
            pool[table[b, dst // page], :, dst % page] = pool[table[b, src // page], :, src % page]
    return _outputs(s)


def _outputs(s):
    kind = s["case"]["kind"]
    if kind == "plan":
        return {k: s[k] for k in ("table", "pages", "lens", "cu_q", "pos", "slots", "ring", "free_out", "mask", "depth_pos") if k in s}
    if kind == "append":
        return {"pools": s["pools"], **({"q": s["q_out"]} if "q_out" in s else {})}
    if kind == "tree":
        return {"out": s["out"], "lse": s["lse"]}
    bits = {1: torch.uint8, 2: torch.int16, 4: torch.int32}
    pools = {k: p.view(bits[p.element_size()]) for k, p in s["pools"].items()}     # rows are moved bit for bit
    return {"path": s["path"], "lens": s["lens"], "last": s["last"], "pools": pools}


# --------------------------------------------------------------------------------------------------------------- 64 bits
def _exact_append(s, case):
    H, G, d_v, d_r = _HEADS[case["heads"]]
    page, slots, pos = case["page"], s["slots"].cpu().numpy(), s["pos"].double()
    pg, at = torch.from_numpy(slots // page).long().cuda(), torch.from_numpy(slots % page).long().cuda()
    pools = {k: p.double() for k, p in s["pools"].items()}

    def turn(x, d, f, halves, m):
        """x [n][heads][..]: element by element, the angle of each pair as a complex number of size m."""
        y = x.clone()
        for i in range(d // 2):
            a, b = (i, i + d // 2) if halves else (2 * i, 2 * i + 1)
            z = torch.polar(torch.full_like(pos, m), pos * f[i])[:, None] * torch.complex(x[..., a], x[..., b])
            y[..., a], y[..., b] = z.real, z.imag
        return y

    if case["form"] == "gva":
        pools["v"][pg, :, at] = s["v_new"].double()
        if d_r:
            pools["kr"][pg, at] = turn(s["kr_new"].double()[:, None], d_r, [_BASE ** (-2.0 * i / d_r) for i in range(d_r // 2)], False, 1.0)[:, 0]
        return {"pools": pools}
    d, rope = case["d_rot"], s["rope"]
    f = []
    for i in range(d // 2):
        base = _BASE * (rope["factor"] ** (d / (d - 2.0)) if case["scaling"] == "base" else 1.0)
        x = math.exp(-2.0 * i / d * math.log(base))
        if case["scaling"] == "linear":
            x /= rope["factor"]
        if case["scaling"] == "parts":
            g = min(1.0, max(0.0, (rope["original_len"] * x / (2.0 * math.pi) - rope["low"]) / (rope["high"] - rope["low"])))
            x = x * g + x / rope["factor"] * (1.0 - g)
        f.append(x)
    x = turn(s["qkv"][:, : H + G].double(), d, f, case["layout"] == "halves", rope.get("magnitude", 1.0))
    pools["k"][pg, :, at] = x[:, H:]
    pools["v"][pg, :, at] = s["qkv"][:, H + G:].double()
    return {"pools": pools, "q": x[:, :H]}


def exact(case, seed):
    if case["kind"] in ("plan", "commit"):
        return None                                                                # whole numbers, and rows as they are
    s = prepare(case, seed)
    H, G, d_v, d_r = _HEADS[case["heads"]]
    if case["kind"] == "append":
        return _exact_append(s, case)
    page, cu, ctx = case["page"], s["cu_q"].tolist(), s["ctx"].tolist()
    bits = s["mask"].cpu().numpy().view(np.uint8)
    sees = np.unpackbits(bits.reshape(s["n"], -1), axis=1, bitorder="little").astype(bool)
    out = torch.zeros(s["n"], H, d_v, dtype=torch.float64, device="cuda")
    lse = torch.full((s["n"], H), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(case["B"]):
        lo, n = cu[b], cu[b + 1] - cu[b]
        t = ctx[b] + n
        ids = s["table"][b, : (t + page - 1) // page].long()
        v = s["pools"]["v"][ids].double().transpose(1, 2).reshape(len(ids) * page, G, d_v)[:t]
        kr = s["pools"]["kr"][ids].double().reshape(len(ids) * page, d_r)[:t]
        hide = torch.zeros(n, t, dtype=torch.bool, device="cuda")
        hide[:, ctx[b]:] = torch.from_numpy(~sees[lo:lo + n, :n]).cuda()
        for h in range(H):
            q = s["q"][lo:lo + n, h].double()
            x = (q[:, :d_v] @ v[:, h // (H // G)].T + q[:, d_v:] @ kr.T) / math.sqrt(d_v + d_r)
            x = x.masked_fill(hide, -math.inf)
            lse[lo:lo + n, h] = torch.logsumexp(x, 1)
            out[lo:lo + n, h] = torch.nan_to_num((x - lse[lo:lo + n, h, None]).exp()) @ v[:, h // (H // G)]
    return {"out": out, "lse": lse}
