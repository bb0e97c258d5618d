"""The operators of generation with drafted tokens, as measurable cases: what a program does around and inside one step.

A case names an operation and the shape it meets:

  pages    page tables, packed rows and slots of the next step from lengths and requests: pages of ended sequences, of rejected
           tokens and behind a window go back to a ring of free ones, new tokens get theirs from it
  norm     root-mean-square norm of every head of Q and K, then the rotation by position, in one pass; "backward" is the
           gradient of both, "append" the same on the way into a paged cache, at the positions of a tree of drafted tokens
  tree     depths and visible ancestors of drafted tokens from their parents, under a mask
  attend   attention of drafted tokens: of a tree's token over the cached context and its own ancestors
  keep     the accepted tokens' keys and values move to the places behind the context, in the caches of several layers

Sequence i of S has a context between "context_lo" and "context" and brings between "new_lo" and "new" tokens, spread evenly
over the logarithm by a fixed low-discrepancy sequence, so that the lengths belong to the case and the values to the seed.
Tensors are [H][T][d] views of what a projection writes, [T][H][d]; pages lie in any order in the cache.
"""
import math

import torch

own = False

_DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2}
_DEVICE = "cuda"
_EPSILON = 1e-6
_MOST_BYTES = 2.0e9
_MOST_FLOPS = 1.5e11


def _pages(name, S, context_lo, context, new_lo, new, page, window=0, n_global=0, ended=0, kept=False, padding=0):
    """ended: of so many sequences one ends; kept: the last step's tokens were drafts, part of which is kept; window 0: nothing
    is given back behind one."""
    return {"name": name, "op": "pages", "S": S, "context_lo": context_lo, "context": context, "new_lo": new_lo, "new": new, "page": page,
            "window": window, "n_global": n_global, "ended": ended, "kept": kept, "padding": padding}


def _norm(name, dtype, Hq, Hkv, T, d, channels, layout, weights, offset=0.0, backward=False):
    return {"name": name, "op": "norm", "dtype": dtype, "Hq": Hq, "Hkv": Hkv, "T": T, "d": d, "channels": channels, "layout": layout,
            "weights": weights, "offset": offset, "backward": backward}


def _append(name, dtype, Hq, Hkv, d, S, context_lo, context, new_lo, new, page, channels, layout, weights, padding=0):
    return {"name": name, "op": "append", "dtype": dtype, "Hq": Hq, "Hkv": Hkv, "d": d, "S": S, "context_lo": context_lo,
            "context": context, "new_lo": new_lo, "new": new, "page": page, "channels": channels, "layout": layout, "weights": weights,
            "offset": 0.0, "chain": 0.3, "padding": padding}


def _tree(name, S, context_lo, context, new_lo, new, window, n_global=0, chain=0.3, padding=0):
    """chain: the share of tokens that follow the one before them."""
    return {"name": name, "op": "tree", "S": S, "context_lo": context_lo, "context": context, "new_lo": new_lo, "new": new, "page": 16,
            "window": window, "n_global": n_global, "chain": chain, "padding": padding}


def _attend(name, dtype, Hq, Hkv, d, S, context_lo, context, new_lo, new, page, window, n_global=0, chain=0.3, padding=0):
    return {"name": name, "op": "attend", "dtype": dtype, "Hq": Hq, "Hkv": Hkv, "d": d, "S": S, "context_lo": context_lo,
            "context": context, "new_lo": new_lo, "new": new, "page": page, "window": window, "n_global": n_global, "chain": chain,
            "padding": padding}


def _keep(name, dtype, layers, Hkv, d, S, context_lo, context, new_lo, new, page, accepted):
    return {"name": name, "op": "keep", "dtype": dtype, "layers": layers, "Hkv": Hkv, "d": d, "S": S, "context_lo": context_lo,
            "context": context, "new_lo": new_lo, "new": new, "page": page, "accepted": accepted}


def listed():
    return [
        # the next decoding step of 64 sequences of up to 32,768 tokens: a token each
        _pages("pages_step", 64, 512, 32768, 1, 1, 16),
        # a busy server: prompts, drafts of the last step, windows that move on, one sequence of nine ends
        _pages("pages_prompts", 700, 100, 40000, 1, 2000, 16, window=4096, n_global=16, ended=9, kept=True, padding=61),
        # queries and keys of 16 drafted tokens of 16 sequences on their way into the cache
        _append("norm_append_drafts_f16", "f16", 32, 8, 128, 16, 500, 4096, 5, 16, 16, 128, "half", "same"),
        # queries and keys of a long prompt, or of a training batch
        _norm("norm_prompt_bf16", "bf16", 32, 8, 32768, 128, 128, "half", "same"),
        # their gradient in training
        _norm("norm_gradient_bf16", "bf16", 32, 8, 32768, 128, 128, "half", "f32", backward=True),
        # the gradient in full precision, an odd length, narrow heads of which half turns, weights stored as their difference from 1
        _norm("norm_gradient_f32", "f32", 8, 2, 10007, 64, 32, "interleaved", "f32", offset=1.0, backward=True),
        # wide trees of many sequences, a window narrower than the deepest of them
        _tree("tree_build", 256, 4, 20000, 16, 500, 24, n_global=16, chain=0.5, padding=5),
        # one sequence with a short draft, one head: the smallest call
        _attend("attend_tree_one_f32", "f32", 1, 1, 64, 1, 2000, 2000, 7, 7, 16, 2048),
        # a step of 64 sequences over every key, shared key heads, contexts that differ by a factor of 64
        _attend("attend_tree_step_bf16", "bf16", 32, 8, 128, 64, 512, 32768, 5, 16, 16, 65536),
        # larger trees under a window with global tokens, padding rows
        _attend("attend_tree_window_f16", "f16", 32, 4, 128, 32, 1000, 65536, 30, 200, 32, 4096, n_global=16, padding=19),
        # what one layer of a decoding step accepts
        _keep("keep_step_bf16", "bf16", 1, 8, 128, 64, 100, 4000, 16, 16, 16, 5),
        # the caches of eight layers at once, larger drafts
        _keep("keep_layers_f16", "f16", 8, 8, 128, 128, 20, 1000, 20, 100, 16, 30),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        case = _draw_any(rng)
        w = work(case)
        e, held = _SIZE.get(case.get("dtype"), 4), 0.0          # what the caches and the plain form keep at once
        if case["op"] in ("append", "attend", "keep"):
            held = 2.0 * e * case["S"] * (case["context"] + case["new"]) * case["Hkv"] * case["d"] * case.get("layers", 1)
        scores = 0.0
        if case["op"] == "attend":
            span = min(case["window"], case["context"]) + case["n_global"] + case["new"]
            scores = float(case["S"]) * span * (case["Hq"] * case["new"] + 2 * case["Hkv"] * case["d"])
        if case["op"] == "tree":
            scores = 8.0 * case["S"] * case["new"] ** 2
        if w["bytes"] <= _MOST_BYTES and w["flops"] <= (_MOST_FLOPS if case.get("dtype") != "f32" else _MOST_FLOPS / 20) \
                and held <= 6.0e9 and scores <= 6.0e9:
            return case


def _draw_any(rng):
    op = rng.choice(("pages", "norm", "norm", "append", "tree", "attend", "attend", "attend", "keep"))
    dtype = rng.choice(("f32", "f16", "bf16"))
    d = rng.choice((32, 64, 64, 128, 128, 128, 256))
    channels = rng.choice((d, d, d // 2, 16))
    layout = rng.choice(("half", "interleaved"))
    weights = rng.choice(("same", "same", "f32", "none"))
    Hkv = rng.choice((1, 2, 4, 8, 8, 16))
    Hq = Hkv * rng.choice((1, 1, 2, 3, 4, 4, 7, 8))
    page = rng.choice((1, 5, 16, 16, 24, 32, 64, 128, 256))
    padding = rng.choice((0, 0, 1, 29))
    S = _log(rng, 1, 256)
    new = _log(rng, 2, 200)
    new_lo = max(1, new // rng.choice((1, 2, 10)))
    context = _log(rng, 1, 65536)
    context_lo = max(1, context // rng.choice((1, 3, 50)))
    window = rng.choice((1 << 20, 1 << 20, _log(rng, 1, 4096)))
    n_global = rng.choice((0, 0, 1, 16, 60))
    chain = rng.choice((0.0, 0.3, 0.3, 0.8, 1.0))
    if op == "pages":
        top = _log(rng, 1, 4000)
        c = _pages("", _log(rng, 1, 1500), context_lo, context, max(1, top // rng.choice((1, 50))), top, max(page, 5),
                   rng.choice((0, 0, window)), n_global, rng.choice((0, 0, 3, 20)), rng.random() < 0.4, padding)
    elif op == "norm":
        d = rng.choice((d, d, 80, 96))
        c = _norm("", dtype, Hq, Hkv, _log(rng, 1, 40000), d, channels if channels <= d else d, layout, weights,
                  rng.choice((0.0, 0.0, 1.0)), rng.random() < 0.5)
    elif op == "append":
        c = _append("", dtype, Hq, Hkv, d, S, context_lo, context, new_lo, new, page, channels, layout, weights, padding)
    elif op == "tree":
        c = _tree("", S, context_lo, context, new_lo, new, window, n_global, chain, padding)
    elif op == "attend":
        c = _attend("", dtype, Hq, Hkv, d, S, context_lo, context, new_lo, new, page, window, n_global, chain, padding)
    else:
        c = _keep("", dtype, rng.choice((1, 1, 2, 5)), Hkv, d, S, context_lo, context, new_lo, new, page, rng.randint(1, new))
    del c["name"]
    return c


def _spread(S, lo, hi, turn):
    return [int(round(lo * (hi / lo) ** ((0.5 + i * turn) % 1.0))) if S > 1 else hi for i in range(S)]


def _lengths(case):
    """New tokens of every sequence and tokens before them."""
    return _spread(case["S"], case["new_lo"], case["new"], 0.7548776662466927), \
        _spread(case["S"], case["context_lo"], case["context"], 0.6180339887498949)


def _words(case):
    return -(-case["new"] // 32)


def _columns(case):
    return -(-(case["context"] + case["new"]) // case["page"])


def work(case):
    if case["op"] == "norm":
        e, rows, T = _SIZE[case["dtype"]], case["Hq"] + case["Hkv"], case["T"]
        times = 3 if case["backward"] else 2
        return {"bytes": float(times * rows * T * case["d"] * e + 8 * T), "flops": float(rows * T * (4 * (times - 1) * case["d"] + 3 * case["channels"]))}
    new, context = _lengths(case)
    T = sum(new)
    if case["op"] == "pages":
        return {"bytes": float(8 * case["S"] * _columns(case) + 32 * case["S"] + 16 * T), "flops": float(4 * case["S"] * _columns(case))}
    if case["op"] == "tree":
        return {"bytes": float(T * (8 + 4 * _words(case))), "flops": float(T * (2 + _words(case)))}
    e, d = _SIZE[case["dtype"]], case["d"]
    if case["op"] == "append":
        heads = case["Hq"] + case["Hkv"]
        return {"bytes": float(2 * T * d * e * (heads + case["Hkv"])), "flops": float(T * heads * (4 * d + 3 * case["channels"]))}
    if case["op"] == "keep":
        rows = sum(min(k, n) for k, n in zip(_accepted(case), new))
        return {"bytes": float(4 * case["layers"] * case["Hkv"] * d * e * rows), "flops": 0.0}
    seen = [min(case["window"], c) + min(case["n_global"], max(0, c - case["window"])) for c in context]
    return {"bytes": float(2 * T * case["Hq"] * d * e + 2 * case["Hkv"] * d * e * sum(k + n for k, n in zip(seen, new))),
            "flops": float(4 * d * case["Hq"] * sum(n * (k + 1) for k, n in zip(seen, new)))}


# ---- inputs ---------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device=_DEVICE)
    g.manual_seed(seed)
    return g


def _frequencies(channels):
    return 10000.0 ** (-torch.arange(0, channels, 2, dtype=torch.float64, device=_DEVICE) / channels)


def _new_rows(H, T, d, dtype, g):
    """[H][T][d], the heads of a token side by side."""
    return torch.randn(T, H, d, generator=g, device=_DEVICE, dtype=dtype).transpose(0, 1)


def _weight(case, dtype, g):
    if case["weights"] == "none":
        return None
    w = 1.0 - case["offset"] + 0.2 * torch.randn(case["d"], generator=g, device=_DEVICE)
    return w if case["weights"] == "f32" else w.to(dtype)


def _table(case, lengths, g, extra=3):
    """Page table of sequences of these lengths and the number of pages of the cache, some of them free; and the order of the pages."""
    columns = _columns(case)
    L = torch.tensor(lengths, device=_DEVICE).unsqueeze(1)
    needed = torch.arange(columns, device=_DEVICE).unsqueeze(0) * case["page"] < L
    count = int(needed.sum())
    order = torch.randperm(count + extra, generator=g, device=_DEVICE).to(torch.int32)
    table = torch.full((case["S"], columns), -1, dtype=torch.int32, device=_DEVICE)
    table[needed] = order[:count]
    return table, count + extra, order[count:]


def _pointers(new):
    ptr = torch.zeros(len(new) + 1, dtype=torch.int64, device=_DEVICE)
    ptr[1:] = torch.tensor(new, device=_DEVICE).cumsum(0)
    return ptr


def _parents(case, ptr, T, g):
    """For every row of the packed tensors the index, among its sequence's new tokens, of the one that it follows, -1 for the last of
    the context; and the row's own index, its sequence (S for padding)."""
    row = torch.arange(T, device=_DEVICE)
    seq = torch.searchsorted(ptr[1:].contiguous(), row, right=True)
    t = row - ptr[seq.clamp(max=case["S"] - 1)]
    u = torch.rand(T, 2, generator=g, device=_DEVICE, dtype=torch.float64)
    parent = torch.where(u[:, 0] < case["chain"], t - 1, (u[:, 1] * (t + 1)).long().clamp(max=t) - 1)
    return parent.to(torch.int32), t, seq


def _ancestors(parent, ptr, n_max):
    """Depth [S, n_max] and a table [S, n_max, n_max] of who is whose ancestor or itself: paths of twice the length, step by step."""
    S = ptr.numel() - 1
    t = torch.arange(n_max, device=_DEVICE)
    real = t < ptr.diff().unsqueeze(1)
    up = torch.where(real, parent.long()[torch.where(real, ptr[:-1, None] + t, 0)], -1)
    up = torch.cat((torch.where(up < 0, n_max, up), torch.full((S, 1), n_max, device=_DEVICE)), 1)     # index n_max: nobody
    has = torch.zeros(S, n_max + 1, n_max, dtype=torch.bool, device=_DEVICE)
    has[:, :n_max] = torch.eye(n_max, dtype=torch.bool, device=_DEVICE)
    for _ in range(max(1, (n_max - 1).bit_length())):
        has = has | torch.gather(has, 1, up.unsqueeze(-1).expand(-1, -1, n_max))
        up = torch.gather(up, 1, up)
    has = has[:, :n_max]
    return has.sum(-1) - 1, has, real


def _accepted(case):
    return _spread(case["S"], 1, case["accepted"], 0.5698402909980532)


def prepare(case, seed):
    g = _generator(seed)
    s = {"case": case}
    if case["op"] == "norm":
        dtype, T, d = _DTYPE[case["dtype"]], case["T"], case["d"]
        for name, H in (("Q", case["Hq"]), ("K", case["Hkv"])):
            s[name] = _new_rows(H, T, d, dtype, g)
            s["w" + name] = _weight(case, dtype, g)
            s["out" + name] = torch.empty_like(s[name])
            if case["backward"]:
                s["g" + name] = _new_rows(H, T, d, dtype, g)
        start = int(torch.randint(0, 100000, (1,), generator=g, device=_DEVICE))
        s["positions"] = torch.arange(start, start + T, device=_DEVICE)
        s["frequencies"] = _frequencies(case["channels"])
        if own:
            import paper_2502_01659_amd as sga
            s["rotary"] = sga.Rotary(s["frequencies"], layout=case["layout"])
            s["norm"] = {n: sga.Norm(s["w" + n], epsilon=_EPSILON, offset=case["offset"]) for n in ("Q", "K")}
            if case["backward"]:
                s["workspace"] = sga.alloc_norm_workspace(T, case["Hq"], case["Hkv"], d)
        return s
    new, context = _lengths(case)
    if case["op"] == "pages":
        return _prepare_pages(s, case, new, context, g)
    T = sum(new) + case.get("padding", 0)
    s["ptr"], s["new"] = _pointers(new), max(new)
    lengths = [n + c for n, c in zip(new, context)]
    s["length"] = torch.tensor(lengths, dtype=torch.int32, device=_DEVICE)
    s["table"], n_pages, _ = _table(case, lengths, g)
    longest = max(lengths)
    if case["op"] != "keep":
        s["parent"], s["t"], s["seq"] = _parents(case, s["ptr"], T, g)
    if case["op"] == "tree":
        s["depth"] = torch.zeros(T, dtype=torch.int32, device=_DEVICE)
        s["seen"] = torch.zeros(T, _words(case), dtype=torch.int32, device=_DEVICE)
        if own:
            s["mask"], s["batch"] = _mask(case, longest), _batch(case, s, T, n_pages)
            s["tree"] = _handle(s["depth"], s["seen"])
        return s
    dtype, d, page = _DTYPE[case["dtype"]], case["d"], case["page"]
    shape = (n_pages, case["Hkv"], page, d)
    if case["op"] == "keep":
        s["cache_k"], s["cache_v"] = (torch.randn(case["layers"], *shape, generator=g, device=_DEVICE, dtype=dtype) for _ in range(2))
        kept = [min(a, n) for a, n in zip(_accepted(case), new)]
        s["count"] = torch.tensor(kept, dtype=torch.int32, device=_DEVICE)
        most = max(kept)
        # so many different indices of a sequence's tokens, in their order
        key = torch.rand(case["S"], s["new"], generator=g, device=_DEVICE)
        key = torch.where(torch.arange(s["new"], device=_DEVICE) < s["ptr"].diff().unsqueeze(1), key, 2.0)
        first = key.argsort(1)[:, :most]
        first = torch.where(torch.arange(most, device=_DEVICE) < s["count"].unsqueeze(1), first, s["new"])
        s["path"] = first.sort(1).values.to(torch.int32).contiguous()
        if own:
            s["batch"] = _batch(case, s, T, n_pages)
        return s
    s["depths"], s["sees"], _ = _ancestors(s["parent"], s["ptr"], s["new"])
    s["Q"] = _new_rows(case["Hq"], T, d, dtype, g)
    s["out"] = torch.zeros_like(s["Q"])
    if case["op"] == "append":
        s["K"], s["V"] = (_new_rows(case["Hkv"], T, d, dtype, g) for _ in range(2))
        s["cache_k"], s["cache_v"] = (torch.zeros(shape, dtype=dtype, device=_DEVICE) for _ in range(2))
        s["frequencies"] = _frequencies(case["channels"])
        s["wQ"], s["wK"] = _weight(case, dtype, g), _weight(case, dtype, g)
    else:
        s["cache_k"], s["cache_v"] = (torch.randn(shape, generator=g, device=_DEVICE, dtype=dtype) for _ in range(2))
        s["lse"] = torch.zeros(case["Hq"], T, device=_DEVICE)
        s["scale"] = 1.0 / math.sqrt(d)
        s["sees"] &= _near(case, s)
    if own:      # the handles, the workspace and the step's tree that a program keeps for all its layers
        import paper_2502_01659_amd as sga
        s["batch"], s["mask"] = _batch(case, s, T, n_pages), _mask(case, longest)
        s["tree"] = sga.build_draft_tree(s["parent"], s["batch"], s["mask"], most=s["new"])
        if case["op"] == "append":
            s["rotary"] = sga.Rotary(s["frequencies"], layout=case["layout"])
            s["norm"] = {n: sga.Norm(s["w" + n], epsilon=_EPSILON, offset=case["offset"]) for n in ("Q", "K")}
        else:
            s["workspace"] = sga.alloc_paged_workspace(s["batch"], s["mask"], case["Hq"], case["Hkv"], d, case["dtype"], tree=s["tree"])
    return s


def _prepare_pages(s, case, new, context, g):
    """Sequences hold the last step's tokens, drafts if "kept"; the ring of free pages begins anywhere."""
    S, page = case["S"], case["page"]
    drafts = [min(c, 1 + i % 8) if case["kept"] else min(c, 1) for i, c in enumerate(context)]
    s["table"], n_pages, free = _table(case, context, g, extra=sum(-(-n // page) + 1 for n in new) * 9 // 10 + 2)
    columns = torch.arange(s["table"].shape[1], device=_DEVICE)
    s["length"] = torch.tensor(context, dtype=torch.int32, device=_DEVICE)
    s["ptr"] = _pointers(drafts)
    if case["window"]:                           # pages that an earlier step found behind the window are gone
        gone = ((columns + 2) * page + case["new"] <= (s["length"].long() - case["window"]).unsqueeze(1)) & (columns * page >= case["n_global"])
        s["table"][gone] = -1
    ask = torch.tensor(new, dtype=torch.int32, device=_DEVICE)
    if case["ended"]:
        ask[case["ended"] // 2::case["ended"]] = -1
    s["ask"] = ask
    s["kept"] = (torch.rand(S, generator=g, device=_DEVICE) * (s["ptr"].diff() + 1)).to(torch.int32) if case["kept"] else None
    T = sum(new) + case["padding"]
    s["T"], s["n_pages"] = T, n_pages
    first = int(torch.randint(0, n_pages, (1,), generator=g, device=_DEVICE))
    s["ring"] = torch.full((n_pages,), -1, dtype=torch.int32, device=_DEVICE)
    s["ring"][(first + torch.arange(free.numel(), device=_DEVICE)) % n_pages] = free
    s["state"] = torch.tensor([first, free.numel()], device=_DEVICE)
    s["positions"], s["slots"] = (torch.zeros(T, dtype=torch.int64, device=_DEVICE) for _ in range(2))
    if own:
        import paper_2502_01659_amd as sga
        s["mask"] = _mask(case, 1 << 30) if case["window"] else None
        s["batch"] = sga.PagedBatch(s["table"], s["ptr"], s["length"], T, page, n_pages)
        s["next"] = sga.PagedBatch(torch.empty_like(s["table"]), torch.empty_like(s["ptr"]), torch.empty_like(s["length"]), T, page, n_pages)
        s["pool"] = sga.PagePool(s["ring"], s["state"])
        s["next_pool"] = sga.PagePool(s["ring"], torch.empty_like(s["state"]))
        s["workspace"] = sga.alloc_pages_workspace(s["batch"])
    return s


def _mask(case, L):
    from sga_inputs import MaskSpec, KIND_SLIDING, KIND_GLOBAL_LOCAL
    kind = KIND_GLOBAL_LOCAL if case.get("n_global", 0) else KIND_SLIDING
    return MaskSpec(kind, L, window=min(case.get("window", L), L), n_global=min(case.get("n_global", 0), L))


def _batch(case, s, T, n_pages):
    import paper_2502_01659_amd as sga
    return sga.PagedBatch(s["table"], s["ptr"], s["length"], T, case["page"], n_pages)


def _handle(depth, seen):
    import paper_2502_01659_amd as sga
    return sga.DraftTree(depth, seen)


# ---- the operators --------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    return {"pages": _pages_plain, "norm": _norm_plain, "append": _append_plain, "tree": _tree_plain, "attend": _attend_plain,
            "keep": _keep_plain}[case["op"]](s, case)


def _run_own(s, case):
    import paper_2502_01659_amd as sga
    if case["op"] == "pages":
        sga.pages_advance(s["batch"], s["pool"], s["ask"], kept=s["kept"], spec=s["mask"], positions=s["positions"], slots=s["slots"],
                          out=(s["next"], s["next_pool"]), workspace=s["workspace"])
        return {"table": s["next"].page_table, "ptr": s["next"].seq_ptr, "length": s["next"].seq_len, "state": s["next_pool"].state,
                "ring": s["ring"], "positions": s["positions"], "slots": s["slots"]}
    if case["op"] == "norm" and not case["backward"]:
        Q, K = sga.norm_rotary(s["Q"], s["K"], rotary=s["rotary"], q_norm=s["norm"]["Q"], k_norm=s["norm"]["K"], positions=s["positions"],
                               Q_out=s["outQ"], K_out=s["outK"])
        return {"Q": Q, "K": K}
    if case["op"] == "norm":
        dQ, dwQ, dK, dwK = sga.norm_rotary_backward(s["Q"], s["gQ"], s["K"], s["gK"], rotary=s["rotary"], q_norm=s["norm"]["Q"],
                                                    k_norm=s["norm"]["K"], positions=s["positions"], dQ=s["outQ"], dK=s["outK"],
                                                    workspace=s["workspace"])
        return {"dQ": dQ, "dK": dK, "dwQ": dwQ, "dwK": dwK}
    if case["op"] == "append":
        sga.cache_append(s["K"], s["V"], s["cache_k"], s["cache_v"], s["batch"], rotary=s["rotary"], Q=s["Q"], Q_out=s["out"],
                         q_norm=s["norm"]["Q"], k_norm=s["norm"]["K"], tree=s["tree"])
        return {"cache_k": s["cache_k"], "cache_v": s["cache_v"], "Q": s["out"]}
    if case["op"] == "tree":
        sga.build_draft_tree(s["parent"], s["batch"], s["mask"], tree=s["tree"])
        return {"depth": s["depth"], "seen": s["seen"]}
    if case["op"] == "keep":
        sga.cache_keep(s["cache_k"], s["cache_v"], s["batch"], s["path"], s["count"])
        return {"cache_k": s["cache_k"], "cache_v": s["cache_v"]}
    O, lse = sga.attention_paged(s["Q"], s["cache_k"], s["cache_v"], s["batch"], s["mask"], s["scale"], O=s["out"], lse=s["lse"],
                                 workspace=s["workspace"], tree=s["tree"])
    return {"O": O, "lse": lse}


def _pages_plain(s, case):
    S, page, n_pages, T = case["S"], case["page"], s["n_pages"], s["T"]
    table, ask, rows = s["table"], s["ask"].long(), s["ptr"].diff()
    ended = ask < 0
    length = s["length"].long()
    if s["kept"] is not None:
        length = length - rows + torch.minimum(s["kept"].long(), rows)
    length = torch.where(ended, 0, length)
    C = table.shape[1]
    candidate = (ask > 0) & (length + ask <= C * page)
    want = torch.where(candidate, ask, 0)
    column = torch.arange(C, device=_DEVICE)
    first_new, end = (length + page - 1) // page, (length + want + page - 1) // page
    held = (table >= 0) & (table < n_pages)
    give = column >= end.unsqueeze(1)
    if case["window"]:
        give |= ((column + 1) * page <= (length - case["window"]).unsqueeze(1)) & (column * page >= case["n_global"])
    give &= held
    need = ~held & (column >= first_new.unsqueeze(1)) & (column < end.unsqueeze(1))
    needs = need.sum(1)
    pages, tokens = needs.cumsum(0), want.cumsum(0)
    first, count = s["state"][0], s["state"][1]
    granted = candidate & (tokens <= T) & ((needs == 0) | (pages <= count))
    rows_new = torch.where(granted, want, 0)
    ptr = torch.zeros_like(s["ptr"])
    ptr[1:] = rows_new.cumsum(0)
    take = need & granted.unsqueeze(1)
    place = (pages - needs).unsqueeze(1) + need.cumsum(1) - 1
    taken = s["ring"][(first + torch.where(take, place, 0)) % n_pages]
    back = table[give]
    after = torch.where(take, taken, torch.where(give, -1, table))
    s["ring"][(first + count + torch.arange(back.numel(), device=_DEVICE)) % n_pages] = back
    total = take.sum()
    state = torch.stack(((first + total) % n_pages, count - total + give.sum()))
    row = torch.arange(T, device=_DEVICE)
    seq = torch.searchsorted(ptr[1:].contiguous(), row, right=True)
    real = seq < S
    seq = seq.clamp(max=S - 1)
    position = length[seq] + row - ptr[seq]
    entry = after[seq, (position // page).clamp(max=C - 1)].long()
    slot = torch.where((entry >= 0) & (entry < n_pages), entry * page + position % page, -1)
    return {"table": after, "ptr": ptr, "length": (length + rows_new).to(torch.int32), "state": state, "ring": s["ring"],
            "positions": torch.where(real, position, 0), "slots": torch.where(real, slot, 0)}


def _turns(positions, s, sign=1.0):
    angle = positions.to(torch.float64).unsqueeze(1) * s["frequencies"]
    return angle.cos().float(), sign * angle.sin().float()


def _rotate(x, turns, case):
    """[H][T][d] in 32 bits, turned by [T][channels / 2]."""
    c, (cos, sin) = case["channels"], turns
    if case["layout"] == "half":
        a, b = x[..., :c // 2], x[..., c // 2:c]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    else:
        a, b = x[..., 0:c:2], x[..., 1:c:2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    return torch.cat((turned, x[..., c:]), -1)


def _weight32(w, case):
    return w.float() + case["offset"] if w is not None else torch.ones(case["d"], device=_DEVICE)


def _normed(x, w, case):
    x = x.float()
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + _EPSILON) * _weight32(w, case)


def _norm_plain(s, case):
    if not case["backward"]:
        turns = _turns(s["positions"], s)
        return {n: _rotate(_normed(s[n], s["w" + n], case), turns, case).to(s[n].dtype) for n in ("Q", "K")}
    turns, out = _turns(s["positions"], s, -1.0), {}
    for n in ("Q", "K"):
        x, g, w = s[n].float(), _rotate(s["g" + n].float(), turns, case), _weight32(s["w" + n], case)
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + _EPSILON)
        unit = x * r
        out["d" + n] = (r * (w * g - unit * (w * g * unit).mean(-1, keepdim=True))).to(s[n].dtype)
        out["dw" + n] = (g * unit).sum((0, 1), dtype=torch.float64).float() if s["w" + n] is not None else None
    return out


def _append_plain(s, case):
    n = s["ptr"].numel() - 1
    real = s["seq"] < n
    seq = s["seq"].clamp(max=n - 1)
    base = s["length"].long()[seq] - s["ptr"].diff()[seq]
    depth = s["depths"][seq, torch.where(real, s["t"], 0)]
    turns = _turns(base + depth, s)
    K = _rotate(_normed(s["K"], s["wK"], case), turns, case).to(s["K"].dtype)
    Q = _rotate(_normed(s["Q"], s["wQ"], case), turns, case).to(s["Q"].dtype)
    seq, slot = seq[real], (base + s["t"])[real]
    page, row = s["table"][seq, slot // case["page"]].long(), slot % case["page"]
    s["cache_k"][page, :, row] = K[:, real].transpose(0, 1)
    s["cache_v"][page, :, row] = s["V"][:, real].transpose(0, 1)
    return {"cache_k": s["cache_k"], "cache_v": s["cache_v"], "Q": torch.where(real[:, None], Q, torch.zeros_like(Q))}


def _near(case, s):
    """[S, n, n]: whether the mask lets new token i see new token j, were it its ancestor."""
    base = s["length"].long() - s["ptr"].diff()
    p = base[:, None] + s["depths"]
    i, j = p.unsqueeze(2), p.unsqueeze(1)
    return (i - j <= case["window"]) | (j < case["n_global"]) | (i < case["n_global"])


def _tree_plain(s, case):
    s["depths"], has, real = _ancestors(s["parent"], s["ptr"], s["new"])
    has &= _near(case, s)
    words = _words(case)
    bits = torch.zeros(*has.shape[:2], 32 * words, dtype=torch.int64, device=_DEVICE)
    bits[..., :has.shape[2]] = has.long()
    packed = (bits.view(*has.shape[:2], words, 32) << torch.arange(32, device=_DEVICE)).sum(-1).to(torch.int32)
    T = s["parent"].numel()
    depth, seen = torch.zeros(T, dtype=torch.int32, device=_DEVICE), torch.zeros(T, words, dtype=torch.int32, device=_DEVICE)
    row = (s["ptr"][:-1, None] + torch.arange(s["new"], device=_DEVICE))[real]
    depth[row], seen[row] = s["depths"][real].to(torch.int32), packed[real]
    return {"depth": depth, "seen": seen}


def _attend_plain(s, case):
    """All keys that a sequence's tokens can see side by side: global ones, the context's last within the window, the new ones."""
    S, Hkv, d, page, ng, n = case["S"], case["Hkv"], case["d"], case["page"], case["n_global"], s["new"]
    G, ptr = case["Hq"] // Hkv, s["ptr"]
    t = torch.arange(n, device=_DEVICE)
    real = t < ptr.diff().unsqueeze(1)
    token = torch.where(real, ptr[:-1, None] + t, 0)                               # [S, n]
    base = (s["length"].long() - ptr.diff()).unsqueeze(1)
    span = min(case["window"], case["context"])
    first = base - span
    j = torch.cat((torch.arange(ng, device=_DEVICE).expand(S, ng), first + torch.arange(span, device=_DEVICE), base + t), 1)
    usable = torch.cat((j[:, :ng] < first, j[:, ng:ng + span] >= 0, real), 1)
    i_, j_ = (base + s["depths"]).unsqueeze(2), j[:, :ng + span].unsqueeze(1)
    seen = torch.cat(((i_ - j_ <= case["window"]) | (j_ < ng) | (i_ < ng), s["sees"]), 2) & usable.unsqueeze(1)
    seen = seen[:, None, None]                                                    # [S, 1, 1, n, keys]
    j = j.clamp(min=0)
    held = torch.gather(s["table"].long(), 1, (j // page).clamp(max=s["table"].shape[1] - 1)).clamp(min=0)
    K, V = (s[name][held, :, j % page].float().transpose(1, 2) for name in ("cache_k", "cache_v"))          # [S, Hkv, keys, d]
    Q = s["Q"].float()[:, token].view(Hkv, G, S, n, d).permute(2, 0, 1, 3, 4).reshape(S, Hkv, G * n, d)
    score = (torch.matmul(Q, K.transpose(-1, -2).contiguous()) * s["scale"]).view(S, Hkv, G, n, -1)
    score = torch.where(seen, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    score.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = score.sum(-1, keepdim=True)
    mix = torch.matmul(score.view(S, Hkv, G * n, -1), V.contiguous()).view(S, Hkv, G, n, d) / torch.where(total == 0, 1.0, total)
    lse = (top + total.log()).squeeze(-1)
    O, out_lse = torch.zeros_like(s["out"]), torch.zeros_like(s["lse"])
    O[:, token[real]] = mix.permute(1, 2, 0, 3, 4).reshape(Hkv * G, S, n, d)[:, real].to(O.dtype)
    out_lse[:, token[real]] = lse.permute(1, 2, 0, 3).reshape(Hkv * G, S, n)[:, real]
    return {"O": O, "lse": out_lse}


def _keep_plain(s, case):
    page, base = case["page"], (s["length"].long() - s["ptr"].diff()).unsqueeze(1)
    k = torch.arange(s["path"].shape[1], device=_DEVICE).expand_as(s["path"])
    use = k < s["count"].unsqueeze(1)
    seq = torch.arange(case["S"], device=_DEVICE).unsqueeze(1).expand_as(k)[use]
    there, here = (base + s["path"].long())[use], (base + k)[use]
    page_from, page_to = s["table"][seq, there // page].long(), s["table"][seq, here // page].long()
    for name in ("cache_k", "cache_v"):
        s[name][:, page_to, :, here % page] = s[name][:, page_from, :, there % page]
    return {"cache_k": s["cache_k"], "cache_v": s["cache_v"]}


# ---- the definitions in 64 bits ---------------------------------------------------------------------
def _turn64(x, at, f, case, back=False):
    """Rows of x [..., T, d] (64 bits) as complex numbers, times e^(i position frequency)."""
    c = case["channels"]
    y = x.clone()
    one, two = (slice(0, c // 2), slice(c // 2, c)) if case["layout"] == "half" else (slice(0, c, 2), slice(1, c, 2))
    angle = at.double()[:, None] * f * (-1.0 if back else 1.0)
    z = torch.complex(y[..., one].contiguous(), y[..., two].contiguous()) * torch.polar(torch.ones_like(angle), angle)
    y[..., one], y[..., two] = z.real, z.imag
    return y


def _norm64(x, w, case):
    x = x.double()
    size = (torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / x.shape[-1] + _EPSILON) ** 0.5
    return x / size * ((w.double() if w is not None else 1.0) + (case["offset"] if w is not None else 0.0))


def _path_of(parent, t):
    """The indices from t up to its first ancestor."""
    path = []
    while t >= 0:
        path.append(t)
        t = parent[t]
    return path


def exact(case, seed):
    if case["op"] in ("pages", "tree"):
        return None                       # whole numbers: equal or wrong
    s = prepare(case, seed)
    if case["op"] == "norm":
        if not case["backward"]:
            return {n: _turn64(_norm64(s[n], s["w" + n], case), s["positions"], s["frequencies"], case) for n in ("Q", "K")}
        out = {}
        for n in ("Q", "K"):
            with torch.enable_grad():
                x = s[n].double().detach().requires_grad_(True)
                w = s["w" + n].double().detach().requires_grad_(True) if s["w" + n] is not None else None
                y = _norm64(x, w, case)
                g = _turn64(s["g" + n].double(), s["positions"], s["frequencies"], case, back=True)
                got = torch.autograd.grad(y, [x] + ([w] if w is not None else []), g)
            out["d" + n], out["dw" + n] = got[0], got[1] if w is not None else None
        return out
    new, context = _lengths(case)
    ptr = [0]
    for n in new:
        ptr.append(ptr[-1] + n)
    if case["op"] == "keep":
        k, v = s["cache_k"].double(), s["cache_v"].double()
        path, count = s["path"].tolist(), s["count"].tolist()
        for i, c in enumerate(context):
            for to in range(count[i]):
                a, b = c + path[i][to], c + to
                p, q = (int(s["table"][i, x // case["page"]]) for x in (a, b))
                for cache in (k, v):
                    cache[:, q, :, b % case["page"]] = cache[:, p, :, a % case["page"]].clone()
        return {"cache_k": k, "cache_v": v}
    parent = s["parent"].tolist()
    if case["op"] == "append":
        k, v, q = s["cache_k"].double(), s["cache_v"].double(), torch.zeros_like(s["out"], dtype=torch.float64)
        for i, (n, c) in enumerate(zip(new, context)):
            rows = slice(ptr[i], ptr[i + 1])
            at = torch.tensor([c + len(_path_of(parent[rows], t)) - 1 for t in range(n)], device=_DEVICE)
            slot = torch.arange(c, c + n, device=_DEVICE)
            page, row = s["table"][i][slot // case["page"]].long(), slot % case["page"]
            k[page, :, row] = _turn64(_norm64(s["K"][:, rows], s["wK"], case), at, s["frequencies"], case).transpose(0, 1)
            v[page, :, row] = s["V"][:, rows].double().transpose(0, 1)
            q[:, rows] = _turn64(_norm64(s["Q"][:, rows], s["wQ"], case), at, s["frequencies"], case)
        return {"cache_k": k, "cache_v": v, "Q": q}
    O = torch.zeros(s["out"].shape, dtype=torch.float64, device=_DEVICE)
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=_DEVICE)
    G, w, ng, Hkv = case["Hq"] // case["Hkv"], case["window"], case["n_global"], case["Hkv"]
    for i, (n, c) in enumerate(zip(new, context)):
        paths = [_path_of(parent[ptr[i]:ptr[i + 1]], t) for t in range(n)]
        low = max(0, c - w)
        if c < ng:
            low = 0
        k_at = torch.cat((torch.arange(min(ng, low), device=_DEVICE), torch.arange(low, c + n, device=_DEVICE)))
        is_new = k_at >= c
        p = torch.tensor([c + len(x) - 1 for x in paths], device=_DEVICE)
        hidden = (p[:, None] - k_at > w) & ~((p < ng)[:, None] | (k_at < ng)) | is_new
        mine = torch.ones(n, n, dtype=torch.bool)
        for t, x in enumerate(paths):
            for up, a in enumerate(x):
                mine[t, a] = up > w and not (c + len(x) - 1 - up < ng or c + len(x) - 1 < ng)
        hidden[:, is_new] = mine.to(_DEVICE)
        page, row = s["table"][i][k_at // case["page"]].long(), k_at % case["page"]
        Q = s["Q"][:, ptr[i]:ptr[i + 1]].double().reshape(Hkv, G * n, case["d"])
        K, V = (s[x][page, :, row].double().transpose(0, 1).contiguous() for x in ("cache_k", "cache_v"))
        z = torch.matmul(Q, K.transpose(1, 2).contiguous()).mul_(s["scale"]).view(Hkv, G, n, -1)
        z.masked_fill_(hidden, -math.inf)
        total = torch.logsumexp(z, -1)
        z = (z - total.unsqueeze(-1)).exp()
        O[:, ptr[i]:ptr[i + 1]] = torch.matmul(z.view(Hkv, -1, z.shape[-1]), V).view(case["Hq"], n, case["d"])
        lse[:, ptr[i]:ptr[i + 1]] = total.reshape(case["Hq"], n)
    return {"O": O, "lse": lse}
