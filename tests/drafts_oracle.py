"""Plain 64-bit definitions of the operators of generation with drafted tokens (NumPy, host) and the error bars that follow from how
the kernels round.  Nothing here is shared with the library."""
import numpy as np

from serving_oracle import HALF_STEP, places, rotate
from sga_inputs import KIND_GLOBAL_LOCAL


# ---- pages ------------------------------------------------------------------------------------------
def advance(table, ptr, length, ring, state, ask, kept, n_tokens, page, n_pages, spec=None):
    """One step, sequence by sequence: (table, ptr, length, ring, state, positions, slots), the last two None for rows of no sequence."""
    table, ring = table.copy(), ring.copy()
    S, C = table.shape
    first, count = int(state[0]) % n_pages, min(max(int(state[1]), 0), n_pages)
    is_page = lambda e: 0 <= e < n_pages
    tokens = pages = taken = 0
    back, new_ptr, new_length, positions, slots = [], [0], [], [None] * n_tokens, [None] * n_tokens
    for s in range(S):
        l = max(int(length[s]), 0)
        if kept is not None:
            rows = min(max(int(ptr[s + 1] - ptr[s]), 0), l)
            l = l - rows + min(max(int(kept[s]), 0), rows)
        a = int(ask[s])
        if a < 0:
            l = 0
        want = a if a > 0 and l + a <= C * page else 0
        begin, end = -(-l // page), -(-(l + want) // page)
        need = [c for c in range(begin, min(end, C)) if not is_page(table[s, c])]
        tokens += want
        pages += len(need)
        granted = want > 0 and tokens <= n_tokens and (not need or pages <= count)
        for c in range(C):
            if not is_page(table[s, c]):
                continue
            behind = spec is not None and (c + 1) * page <= l - spec.window and c * page >= (spec.n_global if spec.kind == KIND_GLOBAL_LOCAL else 0)
            if a < 0 or c >= end or behind:
                back.append(int(table[s, c]))
                table[s, c] = -1
        if granted:
            for c in need:
                table[s, c] = ring[(first + taken) % n_pages]
                taken += 1
            for t in range(want):
                p = l + t
                e = int(table[s, p // page])
                positions[new_ptr[-1] + t], slots[new_ptr[-1] + t] = p, e * page + p % page if is_page(e) else -1
        new_ptr.append(new_ptr[-1] + (want if granted else 0))
        new_length.append(l + (want if granted else 0))
    for i, p in enumerate(back):
        if count + i < n_pages:
            ring[(first + count + i) % n_pages] = p
    state = [(first + taken) % n_pages, min(count + len(back), n_pages) - taken]
    return table, np.array(new_ptr), np.array(new_length), ring, np.array(state), positions, slots


# ---- norms ------------------------------------------------------------------------------------------
def norm(x, weight, epsilon, offset):
    """x float64 [..., d] -> (normed, its inverse size r [..., 1])."""
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + epsilon)
    return x * r * (weight + offset if weight is not None else 1.0), r


def norm_rotate(x, positions, freqs, layout, magnitude, weight, epsilon, offset, normed=True):
    """(y, size of every channel's pair)."""
    n = norm(x, weight, epsilon, offset)[0] if normed else x
    return rotate(n, positions, freqs, layout, magnitude) if freqs is not None else (n, np.abs(n))


def norm_bar(y, size, dtype):
    """The sum of squares: up to 16 additions a lane and 6 across, half of which r feels, the mean, epsilon and the root: 2^-20.  Weights
    and the two products: three half steps.  The rotation: 2^-21 of the pair's size.  All below 2^-19 of it; then one rounding (fp16: or
    half its smallest step)."""
    return size * 2.0 ** -19 + np.abs(y) * HALF_STEP[dtype] + (2.0 ** -25 if dtype == "f16" else 1e-37)


def norm_gradient(x, g, positions, freqs, layout, magnitude, weight, epsilon, offset, normed=True):
    """(dx, dw, sizes of dx's terms, sizes of dw's terms)."""
    t, t_size = rotate(g, positions, freqs, layout, magnitude, inverse=True) if freqs is not None else (g, np.abs(g))
    if not normed:
        return t, None, t_size, None
    w = weight + offset if weight is not None else np.ones(x.shape[-1])
    _, r = norm(x, None, epsilon, 0.0)
    n = x * r
    dx = r * (w * t - n * (w * t * n).mean(-1, keepdims=True))
    size = r * (np.abs(w) * t_size + np.abs(n) * (np.abs(w) * t_size * np.abs(n)).mean(-1, keepdims=True))
    return dx, (t * n).sum((0, 1)), size, (t_size * np.abs(n)).sum((0, 1))


def gradient_bar(dx, size, dtype):
    """Two factors r (2^-20 each), the mean (as many roundings as the sum of squares), the rotation 2^-21 and a few half steps: below 2^-18 of
    the terms' sizes; then one rounding."""
    return size * 2.0 ** -18 + np.abs(dx) * HALF_STEP[dtype] + (2.0 ** -25 if dtype == "f16" else 1e-37)


def weight_bar(size):
    """Terms: 2^-18 of their sizes as above.  A lane adds at most 64 rows' terms in these tests, a wavefront and a workgroup 8 such sums: 72
    half steps of what is summed, below 2^-17; 64 bits from there on."""
    return size * (2.0 ** -18 + 2.0 ** -17) + 1e-37


# ---- trees ------------------------------------------------------------------------------------------
def paths(parent):
    """For every token its ancestors among the new ones, itself first."""
    out = []
    for t, p in enumerate(parent):
        out.append([t] + (out[p] if 0 <= p < t else []))
    return out


def shows(spec, p, q):
    """Whether the mask shows a token at position p one at q <= p."""
    if p < 0 or p >= spec.L or q < 0:
        return False
    ng = spec.n_global if spec.kind == KIND_GLOBAL_LOCAL else 0
    return p - q <= spec.window or q < ng or p < ng


def tree(parent, ptr, length, spec, words):
    """(depth, seen) of the rows of sequences, as Python lists; seen: sets of indices."""
    depth, seen = [None] * len(parent), [None] * len(parent)
    for s in range(len(length)):
        a, b = int(ptr[s]), int(ptr[s + 1])
        base = int(length[s]) - (b - a)
        up = paths([int(x) for x in parent[a:min(b, a + 32 * words)]])
        for t in range(b - a):
            if t >= 32 * words:
                depth[a + t], seen[a + t] = -1, set()
                continue
            d = len(up[t]) - 1
            depth[a + t] = d
            seen[a + t] = {j for j in up[t] if shows(spec, base + d, base + len(up[j]) - 1)}
    return depth, seen


def unpack(bits):
    """int32 [T, words] -> a list of sets."""
    return [{32 * w + b for w, x in enumerate(row) for b in range(32) if int(x) >> b & 1} for row in bits]


def attend(Q, cache_k, cache_v, page_table, ptr, length, depth, seen, spec, scale, dtype, once=False):
    """(O, lse, bar of O, bar of lse), float64; rows of no sequence are NaN.  The bars are those of attention over a paged cache."""
    Hq, T, d = Q.shape
    n_pages, Hkv, page, _ = cache_k.shape
    O, lse = np.full((Hq, T, d), np.nan), np.full((Hq, T), np.nan)
    O_bar, lse_bar = np.zeros((Hq, T, d)), np.zeros((Hq, T))
    for s in range(len(length)):
        n = int(ptr[s + 1] - ptr[s])
        base = int(length[s]) - n
        for t in range(n):
            row = int(ptr[s]) + t
            O[:, row], lse[:, row] = 0.0, -np.inf
            p = base + depth[row]
            if depth[row] < 0 or p < 0 or p >= spec.L:
                continue
            j = [q for q in range(max(base, 0)) if q < spec.L and shows(spec, p, q)]
            j = np.array(j + [base + q for q in sorted(seen[row]) if q < n and base + q >= 0], dtype=np.int64)
            at, r = places(page_table, s, j, page, n_pages)
            at, r = at[at >= 0], r[at >= 0]
            if len(at) == 0:
                continue
            for g in range(Hkv):
                k, v = cache_k[at, g, r].astype(np.float64), cache_v[at, g, r].astype(np.float64)
                heads = slice(g * (Hq // Hkv), (g + 1) * (Hq // Hkv))
                q = Q[heads, row].astype(np.float64)
                z = scale * (q @ k.T)
                top = z.max(1, keepdims=True)
                e = np.exp(z - top)
                l = e.sum(1, keepdims=True)
                O[heads, row], lse[heads, row] = e @ v / l, (top + np.log(l))[:, 0]
                # scores: d products in 32 bits, scale, log2 e and the exponential a few half steps; probabilities as two numbers of the
                # storage type or rounded once; sums over n keys sqrt(n) half steps and to spare
                off = (d * 2.0 ** -24 * abs(scale) * (np.abs(q) @ np.abs(k).T)).max(1, keepdims=True) \
                    + 2.0 ** -22 * (1 + np.abs(z).max(1, keepdims=True))
                parts = {"f32": 0.0, "f16": 2.0 ** -21, "bf16": 2.0 ** -15}[dtype] if not once else HALF_STEP[dtype]
                share = e @ np.abs(v) / l
                O_bar[heads, row] = share * (2 * off + parts + (4 + np.sqrt(len(at))) * 2.0 ** -23) + np.abs(O[heads, row]) * HALF_STEP[dtype]
                if dtype == "f16":
                    O_bar[heads, row] += 2.0 ** -24 * np.abs(v).sum(0) / l + 2.0 ** -25
                lse_bar[heads, row] = (2 * off[:, 0]) + 2.0 ** -22 * (1 + np.abs(lse[heads, row]))
    return O, lse, O_bar, lse_bar


# ---- accepted tokens --------------------------------------------------------------------------------
def keep(cache, page_table, ptr, length, path, count):
    """cache [..., n_pages, Hkv, page, d] after the moves, all from what it held before."""
    out = cache.copy()
    n_pages, page = cache.shape[-4], cache.shape[-2]
    for s in range(len(length)):
        n = int(ptr[s + 1] - ptr[s])
        base = int(length[s]) - n
        for k in range(min(int(count[s]), path.shape[1])):
            p = int(path[s, k])
            if not k <= p < n or base + k < 0:
                continue
            (a, b), (r, q) = places(page_table, s, np.array([base + p, base + k]), page, n_pages)
            if a >= 0 and b >= 0:
                out[..., b, :, q, :] = cache[..., a, :, r, :]
    return out
