"""The operators of serving with a paged cache, as measurable cases: what a model does with its new tokens.

A case names an operation and the shape it meets:

  rotary   rotation of Q or K by position: half and interleaved channel pairs, all or part of the
           head; "inverse" is the gradient
  append   new keys (rotated) and values written into the pages of a cache, queries rotated beside them
  attend   attention of the new tokens of every sequence over the cache, causal or not, under a
           window (window >= L: every key) with or without leading global tokens

Tensors are [H][T][d] views of what a projection writes, [T][H][d]; values are N(0, 1).  Pages lie in
any order in the cache.  Sequence i of S has a length between "context_lo" and "context" and brings
between "new_lo" and "new" tokens, spread evenly over the logarithm by a fixed low-discrepancy
sequence, so that the lengths belong to the case and the values to the seed.
"""
import math

import torch

own = False

_DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2}
_DEVICE = "cuda"
_MOST_BYTES = 4.0e9
_MOST_FLOPS = 1.2e12


def _rotary(name, dtype, H, T, d, channels, layout, inverse=False, factor=1.0, reach=131072):
    return {"name": name, "op": "rotary", "dtype": dtype, "H": H, "T": T, "d": d, "channels": channels, "layout": layout,
            "inverse": inverse, "factor": factor, "reach": reach}


def _append(name, dtype, Hq, Hkv, d, S, context_lo, context, new_lo, new, page, channels, layout, padding=0):
    return {"name": name, "op": "append", "dtype": dtype, "Hq": Hq, "Hkv": Hkv, "d": d, "S": S, "context_lo": context_lo,
            "context": context, "new_lo": new_lo, "new": new, "page": page, "channels": channels, "layout": layout,
            "padding": padding}


def _attend(name, dtype, Hq, Hkv, d, S, context_lo, context, new_lo, new, page, window, n_global=0, causal=True, padding=0):
    return {"name": name, "op": "attend", "dtype": dtype, "Hq": Hq, "Hkv": Hkv, "d": d, "S": S, "context_lo": context_lo,
            "context": context, "new_lo": new_lo, "new": new, "page": page, "window": window, "n_global": n_global,
            "causal": causal, "padding": padding}


def listed():
    return [
        # the queries of one decoding step of 16 sequences: a launch, hardly any data
        _rotary("rotary_step_f16", "f16", 32, 16, 128, 128, "half"),
        # the queries of a long prompt, stretched to eight times the trained length
        _rotary("rotary_64k_bf16", "bf16", 32, 65536, 128, 128, "half", factor=8.0),
        # the gradient of a layer that rotates half of every head, an odd length, far positions
        _rotary("rotary_gradient_f32", "f32", 8, 100003, 64, 32, "interleaved", inverse=True, reach=160_000_000),
        # one decoding step of 64 sequences: a token each goes into the cache
        _append("append_step_bf16", "bf16", 32, 8, 128, 64, 500, 16384, 1, 1, 16, 128, "half"),
        # prompts of several lengths in one packed call, half of the head rotated
        _append("append_prompts_f16", "f16", 32, 8, 128, 12, 1000, 8192, 1000, 8192, 64, 64, "interleaved", padding=37),
        # a single sequence, a narrow window, one head: the smallest call
        _attend("attend_one_f32", "f32", 1, 1, 64, 1, 4096, 4096, 1, 1, 16, 32),
        # one decoding step over every key: shared key heads, lengths that differ by a factor of 64
        _attend("attend_step_bf16", "bf16", 32, 8, 128, 64, 512, 32768, 1, 1, 16, 32768),
        # one decoding step of many sequences with a window and global tokens: pages behind the window are given back
        _attend("attend_window_step_f16", "f16", 32, 4, 128, 160, 300, 131072, 1, 1, 32, 2048, n_global=16),
        # a piece of a prompt behind what the cache holds of it
        _attend("attend_chunks_bf16", "bf16", 32, 8, 128, 8, 2048, 16384, 200, 256, 16, 16384),
        # a whole prompt under a window: 32 heads of 128 channels
        _attend("attend_prompt_f16", "f16", 32, 32, 128, 1, 32768, 32768, 32768, 32768, 64, 2048),
        # full precision, the window and global tokens of a long document, not causal, odd pages, padding rows
        _attend("attend_document_f32", "f32", 8, 8, 64, 6, 1500, 4096, 900, 4096, 24, 128, n_global=16, causal=False, padding=50),
        # single tokens and short drafts together, wide heads
        _attend("attend_drafts_d256_bf16", "bf16", 16, 2, 256, 33, 100, 20000, 1, 9, 32, 4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        case = _draw_any(rng)
        w = work(case)
        scores = 1.0
        if case["op"] == "attend":      # what the plain form keeps at once
            full = case["window"] + case["new"] >= case["context"] or (not case["causal"] and case["n_global"] > 0)
            span = case["context"] if full else 3 * case["window"] + 1024
            scores = float(case["S"]) * case["Hq"] * case["new"] * span
        if w["bytes"] <= _MOST_BYTES and w["flops"] <= (_MOST_FLOPS if case["dtype"] != "f32" else _MOST_FLOPS / 20) and scores <= 2.0e9:
            return case


def _draw_any(rng):
    op = rng.choice(("rotary", "append", "attend", "attend", "attend"))
    dtype = rng.choice(("f32", "f16", "bf16"))
    d = rng.choice((32, 64, 64, 128, 128, 128, 256))
    channels = rng.choice((d, d, d // 2, 16))
    layout = rng.choice(("half", "interleaved"))
    if op == "rotary":
        c = _rotary("", dtype, rng.choice((1, 2, 8, 16, 32, 40)), _log(rng, 1, 100000), d, channels, layout,
                    rng.random() < 0.5, rng.choice((1.0, 4.0, 8.0)), _log(rng, 1000, 1 << 30))
    else:
        Hkv = rng.choice((1, 2, 4, 8, 8, 16))
        Hq = Hkv * rng.choice((1, 1, 2, 3, 4, 4, 7, 8))
        page = rng.choice((1, 5, 16, 16, 24, 32, 64, 128, 256))
        kind = rng.choice(("step", "step", "drafts", "chunks", "prompts"))
        S = _log(rng, 1, 256 if kind in ("step", "drafts") else 16)
        new = {"step": 1, "drafts": rng.randint(2, 16), "chunks": _log(rng, 17, 1024), "prompts": _log(rng, 17, 8192)}[kind]
        new_lo = {"step": 1, "drafts": 1, "chunks": max(1, new // 3), "prompts": max(1, new // 5)}[kind]
        context = new if kind == "prompts" else max(new, _log(rng, 1, 65536))
        context_lo = new_lo if kind == "prompts" else max(1, context // rng.choice((1, 3, 50)))
        padding = rng.choice((0, 0, 1, 29))
        if op == "append":
            c = _append("", dtype, Hq, Hkv, d, S, context_lo, context, new_lo, new, page, channels, layout, padding)
        else:
            window = rng.choice((context, context, _log(rng, 1, 4096)))
            c = _attend("", dtype, Hq, Hkv, d, S, context_lo, context, new_lo, new, page, window, rng.choice((0, 0, 1, 16, 60)),
                        rng.random() < 0.8, padding)
    del c["name"]
    return c


def _spread(S, lo, hi, turn):
    return [int(round(lo * (hi / lo) ** ((0.5 + i * turn) % 1.0))) if S > 1 else hi for i in range(S)]


def _lengths(case):
    """New tokens and total length of every sequence."""
    new = _spread(case["S"], case["new_lo"], case["new"], 0.7548776662466927)
    context = _spread(case["S"], case["context_lo"], case["context"], 0.6180339887498949)
    if case["context"] == case["new"]:
        return new, new
    return new, [max(a, b) for a, b in zip(new, context)]


def _low(case, p):
    return max(0, p - case["window"])


def _edges(case, n, L):
    """(query, key) pairs of a sequence of L tokens, the last n of them new, and keys that any of them sees."""
    w, g, causal = case["window"], min(case["n_global"], L), case["causal"]
    p = torch.arange(L - n, L, dtype=torch.int64)
    lo = (p - w).clamp(min=0)
    hi = p if causal else (p + w).clamp(max=L - 1)
    glob = p < g
    last = hi if causal else torch.where(glob, torch.full_like(p, L - 1), hi)
    lo = torch.where(glob, torch.zeros_like(lo), lo)
    pairs = (last - lo + 1) + torch.minimum(lo, torch.full_like(lo, g))
    first = int(lo.min())
    return int(pairs.sum()), int(last.max()) + 1 - first + min(first, g)


def work(case):
    e, d = _SIZE[case["dtype"]], case["d"]
    if case["op"] == "rotary":
        n = case["H"] * case["T"]
        return {"bytes": float(2 * n * d * e + 8 * case["T"]), "flops": float(3 * n * case["channels"])}
    new, context = _lengths(case)
    T = sum(new)
    if case["op"] == "append":
        heads = case["Hq"] + case["Hkv"]
        return {"bytes": float(2 * T * d * e * (heads + case["Hkv"])), "flops": float(3 * T * heads * case["channels"])}
    seen = [_edges(case, n, L) for n, L in zip(new, context)]
    return {"bytes": float(2 * T * case["Hq"] * d * e + 2 * case["Hkv"] * d * e * sum(k for _, k in seen)),
            "flops": float(4 * d * case["Hq"] * sum(p for p, _ in seen))}


# ---- inputs ---------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device=_DEVICE)
    g.manual_seed(seed)
    return g


def _frequencies(case):
    """base^(-2i / channels); stretched by a factor, the low ones are divided by it and the high ones kept."""
    c = case["channels"]
    f = 10000.0 ** (-torch.arange(0, c, 2, dtype=torch.float64, device=_DEVICE) / c)
    factor = case.get("factor", 1.0)
    if factor == 1.0:
        return f, 1.0
    turns = 8192.0 * f / (2 * math.pi)
    keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
    return f * (keep + (1.0 - keep) / factor), 0.1 * math.log(factor) + 1.0


def _new_rows(H, T, d, dtype, g):
    """[H][T][d], the heads of a token side by side."""
    return torch.randn(T, H, d, generator=g, device=_DEVICE, dtype=dtype).transpose(0, 1)


def _pages(case, g):
    """Page table, lengths and the number of pages of the cache, some of them free."""
    new, context = _lengths(case)
    page = case["page"]
    columns = -(-max(context) // page)
    L = torch.tensor(context, device=_DEVICE).unsqueeze(1)
    at = torch.arange(columns, device=_DEVICE).unsqueeze(0)
    needed = at * page < L
    if case["op"] == "attend" and case["new"] == 1:      # pages wholly behind the window are given back
        needed &= ((at + 1) * page > L - 1 - case["window"]) | (at * page < case["n_global"])
    count = int(needed.sum())
    n_pages = count + 3
    order = torch.randperm(n_pages, generator=g, device=_DEVICE)[:count]
    table = torch.full((case["S"], columns), -1, dtype=torch.int32, device=_DEVICE)
    table[needed] = order.to(torch.int32)
    ptr = torch.zeros(case["S"] + 1, dtype=torch.int64, device=_DEVICE)
    ptr[1:] = torch.tensor(new, device=_DEVICE).cumsum(0)
    return table, ptr, torch.tensor(context, dtype=torch.int32, device=_DEVICE), n_pages


def prepare(case, seed):
    g = _generator(seed)
    dtype, d = _DTYPE[case["dtype"]], case["d"]
    s = {"case": case}
    if case["op"] == "rotary":
        s["X"] = _new_rows(case["H"], case["T"], d, dtype, g)
        start = int(torch.randint(0, max(1, case["reach"] - case["T"]), (1,), generator=g, device=_DEVICE))
        s["positions"] = torch.arange(start, start + case["T"], device=_DEVICE)
        s["frequencies"], s["magnitude"] = _frequencies(case)
        s["out"] = torch.empty_like(s["X"])
    else:
        new, _ = _lengths(case)
        T = sum(new) + case["padding"]
        s["table"], s["ptr"], s["length"], n_pages = _pages(case, g)
        shape = (n_pages, case["Hkv"], case["page"], d)
        s["Q"] = _new_rows(case["Hq"], T, d, dtype, g)
        s["out"] = torch.zeros_like(s["Q"])
        s["new"], s["longest"] = max(new), int(s["length"].max())
        if case["op"] == "append":
            s["K"], s["V"] = (_new_rows(case["Hkv"], T, d, dtype, g) for _ in range(2))
            s["cache_k"], s["cache_v"] = (torch.zeros(shape, dtype=dtype, device=_DEVICE) for _ in range(2))
            s["frequencies"], s["magnitude"] = _frequencies(case)
        else:
            s["cache_k"], s["cache_v"] = (torch.randn(shape, generator=g, device=_DEVICE, dtype=dtype) for _ in range(2))
            s["lse"] = torch.zeros(case["Hq"], T, device=_DEVICE)
            s["scale"] = 1.0 / math.sqrt(d)
    if own:      # the handles and the workspace that a program keeps
        import paper_2502_01659_amd as sga
        from sga_inputs import MaskSpec, KIND_SLIDING, KIND_GLOBAL_LOCAL
        if case["op"] != "attend":
            s["rotary"] = sga.Rotary(s["frequencies"], layout=case["layout"], magnitude=s["magnitude"])
        if case["op"] != "rotary":
            s["batch"] = sga.PagedBatch(s["table"], s["ptr"], s["length"], T, case["page"], n_pages)
        if case["op"] == "attend":
            kind = KIND_GLOBAL_LOCAL if case["n_global"] else KIND_SLIDING
            s["mask"] = MaskSpec(kind, s["longest"], window=case["window"], n_global=min(case["n_global"], s["longest"]))
            s["workspace"] = sga.alloc_paged_workspace(s["batch"], s["mask"], case["Hq"], case["Hkv"], d, case["dtype"])
    return s


# ---- the operators --------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    if case["op"] == "rotary":
        return {"Y": _rotate(s["X"], s["positions"], s, case, -1.0 if case["inverse"] else 1.0)}
    if case["op"] == "append":
        return _append_plain(s, case)
    return _attend_plain(s, case)


def _run_own(s, case):
    import paper_2502_01659_amd as sga
    if case["op"] == "rotary":
        return {"Y": sga.rotary(s["X"], s["rotary"], positions=s["positions"], inverse=case["inverse"], out=s["out"])}
    if case["op"] == "append":
        sga.cache_append(s["K"], s["V"], s["cache_k"], s["cache_v"], s["batch"], rotary=s["rotary"], Q=s["Q"], Q_out=s["out"])
        return {"cache_k": s["cache_k"], "cache_v": s["cache_v"], "Q": s["out"]}
    O, lse = sga.attention_paged(s["Q"], s["cache_k"], s["cache_v"], s["batch"], s["mask"], s["scale"], causal=case["causal"],
                                 O=s["out"], lse=s["lse"], workspace=s["workspace"])
    return {"O": O, "lse": lse}


def _rotate(X, positions, s, case, sign):
    """[H][T][d] rotated at positions [T], angles in 64 bits."""
    c = case["channels"]
    angle = positions.to(torch.float64).unsqueeze(1) * s["frequencies"]
    cos, sin = (s["magnitude"] * angle.cos()).float(), (sign * s["magnitude"] * angle.sin()).float()
    x = X.float()
    if case["layout"] == "half":
        a, b = x[..., :c // 2], x[..., c // 2:c]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    else:
        a, b = x[..., 0:c:2], x[..., 1:c:2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    return torch.cat((turned, x[..., c:]), -1).to(X.dtype)


def _append_plain(s, case):
    T = s["K"].shape[1]
    token = torch.arange(T, device=_DEVICE)
    seq = torch.searchsorted(s["ptr"][1:], token, right=True)
    real = seq < case["S"]
    seq = seq.clamp(max=case["S"] - 1)
    position = s["length"][seq] - s["ptr"][seq + 1] + token
    K = _rotate(s["K"], position, s, case, 1.0)
    Q = _rotate(s["Q"], position, s, case, 1.0)
    seq, position = seq[real], position[real]
    page, row = s["table"][seq, position // case["page"]].long(), position % case["page"]
    s["cache_k"][page, :, row] = K[:, real].transpose(0, 1)
    s["cache_v"][page, :, row] = s["V"][:, real].transpose(0, 1)
    return {"cache_k": s["cache_k"], "cache_v": s["cache_v"], "Q": torch.where(real[:, None], Q, torch.zeros_like(Q))}


def _attend_plain(s, case):
    """Queries in blocks of one span of keys each; one block of all where the span is the whole context."""
    S, Hkv, d, page, w, ng = case["S"], case["Hkv"], case["d"], case["page"], case["window"], case["n_global"]
    G, longest, causal = case["Hq"] // Hkv, s["longest"], case["causal"]
    B = min(s["new"], 1024)
    span = B + w + (0 if causal else w)
    if span >= longest or (ng > 0 and not causal):
        B, span = s["new"], longest
    blocks = -(-s["new"] // B)
    start, count, length = s["ptr"][:-1, None, None], s["ptr"].diff()[:, None, None], s["length"].long()[:, None, None]
    t = torch.arange(blocks * B, device=_DEVICE).view(1, blocks, B)
    real = t < count
    token = torch.where(real, start + t, 0)
    p = length - count + t                                                       # [S, blocks, B]
    first = (p[..., :1] - w).clamp(min=0) if span < longest else torch.zeros_like(p[..., :1])
    j = first + torch.arange(span, device=_DEVICE)                               # [S, blocks, span]
    own_span = torch.ones_like(j, dtype=torch.bool)
    if ng > 0 and span < longest:                                                # global keys before the span
        lead = torch.arange(ng, device=_DEVICE).expand(S, blocks, ng)
        j, own_span = torch.cat((lead, j), -1), torch.cat((lead < first, own_span), -1)
    held = torch.gather(s["table"].long(), 1, (j // page).clamp(max=s["table"].shape[1] - 1).flatten(1)).view(j.shape)
    usable = own_span & (j < length) & (held >= 0)
    i_, j_ = p.unsqueeze(-1), j.unsqueeze(-2)
    seen = ((i_ - j_).abs() <= w) | (j_ < ng) | (i_ < ng)
    if causal:
        seen &= j_ <= i_
    seen = (seen & usable.unsqueeze(-2)).unsqueeze(2).unsqueeze(3)               # [S, blocks, 1, 1, B, keys]
    K, V = (s[name][held.clamp(min=0), :, j % page].float().permute(0, 1, 3, 2, 4) for name in ("cache_k", "cache_v"))
    Q = s["Q"].float()[:, token].view(Hkv, G, S, blocks, B, d).permute(2, 3, 0, 1, 4, 5).reshape(S, blocks, Hkv, G * B, d)
    score = (torch.matmul(Q, K.transpose(-1, -2)) * s["scale"]).view(S, blocks, Hkv, G, B, -1)
    score = torch.where(seen, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    score.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = score.sum(-1, keepdim=True)
    mix = torch.matmul(score.view(S, blocks, Hkv, G * B, -1), V).view(S, blocks, Hkv, G, B, d) / torch.where(total == 0, 1.0, total)
    lse = (top + total.log()).squeeze(-1)
    O, out_lse = torch.zeros_like(s["out"]), torch.zeros_like(s["lse"])
    O[:, token[real]] = mix.permute(2, 3, 0, 1, 4, 5).reshape(Hkv * G, S, blocks, B, d)[:, real].to(O.dtype)
    out_lse[:, token[real]] = lse.permute(2, 3, 0, 1, 4).reshape(Hkv * G, S, blocks, B)[:, real]
    return {"O": O, "lse": out_lse}


# ---- the definitions in 64 bits ---------------------------------------------------------------------
def _turn64(x, at, f, m, case):
    """Rows of x [..., T, d] as complex numbers, multiplied by m e^(i position frequency)."""
    c = case["channels"]
    y = x.double().clone()
    one, two = (slice(0, c // 2), slice(c // 2, c)) if case["layout"] == "half" else (slice(0, c, 2), slice(1, c, 2))
    turn = torch.polar(torch.full_like(at.double()[:, None] * f, m), (at.double()[:, None] * f) * (-1.0 if case.get("inverse") else 1.0))
    z = torch.complex(y[..., one].contiguous(), y[..., two].contiguous()) * turn
    y[..., one], y[..., two] = z.real, z.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotary":
        return {"Y": _turn64(s["X"], s["positions"], s["frequencies"], s["magnitude"], case)}
    new, context = _lengths(case)
    if case["op"] == "append":
        k, v, q = s["cache_k"].double(), s["cache_v"].double(), torch.zeros_like(s["out"], dtype=torch.float64)
        at = 0
        for i, (n, L) in enumerate(zip(new, context)):
            where = torch.arange(L - n, L, device=_DEVICE)
            page, row = s["table"][i][where // case["page"]].long(), where % case["page"]
            rows = slice(at, at + n)
            k[page, :, row] = _turn64(s["K"][:, rows], where, s["frequencies"], s["magnitude"], case).transpose(0, 1)
            v[page, :, row] = s["V"][:, rows].double().transpose(0, 1)
            q[:, rows] = _turn64(s["Q"][:, rows], where, s["frequencies"], s["magnitude"], case)
            at += n
        return {"cache_k": k, "cache_v": v, "Q": q}
    O = torch.zeros(s["out"].shape, dtype=torch.float64, device=_DEVICE)
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=_DEVICE)
    G, w, ng, at = case["Hq"] // case["Hkv"], case["window"], case["n_global"], 0
    for i, (n, L) in enumerate(zip(new, context)):
        everything = L - n < ng and not case["causal"]
        for r0 in range(0, n, 512):
            r1 = min(n, r0 + 512)
            q_at = torch.arange(L - n + r0, L - n + r1, device=_DEVICE)
            a = 0 if everything else max(0, L - n + r0 - w)
            b = L if everything or not case["causal"] else L - n + r1
            b = b if everything else min(b, L - n + r1 + w)
            k_at = torch.cat((torch.arange(min(ng, a), device=_DEVICE), torch.arange(a, b, device=_DEVICE)))
            page, row = s["table"][i][k_at // case["page"]].long(), k_at % case["page"]
            far = (q_at[:, None] - k_at).abs() > w
            hidden = far & ~((q_at < ng)[:, None] | (k_at < ng)) | (page < 0)
            if case["causal"]:
                hidden |= k_at > q_at[:, None]
            Q = s["Q"][:, at + r0:at + r1].double().reshape(case["Hkv"], G * (r1 - r0), case["d"])
            K, V = (s[x][page.clamp(min=0), :, row].double().transpose(0, 1).contiguous() for x in ("cache_k", "cache_v"))
            z = torch.matmul(Q, K.transpose(1, 2).contiguous()).mul_(s["scale"]).view(case["Hkv"], G, r1 - r0, -1)
            z.masked_fill_(hidden, -math.inf)
            total = torch.logsumexp(z, -1)
            z = (z - torch.where(total.isinf(), 0.0, total).unsqueeze(-1)).exp()
            O[:, at + r0:at + r1] = torch.matmul(z.view(case["Hkv"], -1, z.shape[-1]), V).view(case["Hq"], r1 - r0, case["d"])
            lse[:, at + r0:at + r1] = total.reshape(case["Hq"], r1 - r0)
        at += n
    return {"O": O, "lse": lse}
