"""Plain 64-bit definitions of the serving operators (NumPy, host) and the error bars that follow from how the kernels
round.  Nothing here is shared with the library."""
import numpy as np

from sga_inputs import KIND_GLOBAL_LOCAL

HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def rotate(x, positions, freqs, layout="half", magnitude=1.0, inverse=False):
    """x float64 [H, T, d] -> (rotated, |a| + |b| of every channel's pair).  Angles in extended precision where the
    machine has it (a product of 2^31 and a frequency keeps 2^-33)."""
    c = 2 * len(freqs)
    one, two = (slice(0, c // 2), slice(c // 2, c)) if layout == "half" else (slice(0, c, 2), slice(1, c, 2))
    angle = np.asarray(positions, dtype=np.longdouble)[:, None] * np.asarray(freqs, dtype=np.longdouble)
    cos, sin = np.cos(angle).astype(np.float64), np.sin(angle).astype(np.float64)
    if inverse:
        sin = -sin
    y, size = x.copy(), np.abs(x)
    a, b = x[..., one], x[..., two]
    y[..., one], y[..., two] = magnitude * (a * cos - b * sin), magnitude * (a * sin + b * cos)
    size[..., one] = size[..., two] = abs(magnitude) * (np.abs(a) + np.abs(b))
    return y, size


def rotate_bar(y, size, dtype):
    """Sine and cosine: the reduced angle rounded to 32 bits (at most 2^-25 off), polynomials (2e-9), their evaluation and
    the product with the magnitude (a few half steps of 2^-24): below 2^-21 of the pair's size with the two products and
    their sum; then one rounding to the storage type (its smallest steps: 2^-25 for fp16)."""
    return size * 2.0 ** -21 + np.abs(y) * HALF_STEP[dtype] + (2.0 ** -25 if dtype == "f16" else 1e-37)


def neighbours(spec, i, length, causal):
    """Tokens that position i sees."""
    if i < 0 or i >= spec.L:
        return np.zeros(0, dtype=np.int64)
    j = np.arange(min(length, spec.L))
    see = np.abs(i - j) <= spec.window
    if spec.kind == KIND_GLOBAL_LOCAL:
        see |= (j < spec.n_global) | (i < spec.n_global)
    if causal:
        see &= j <= i
    return j[see]


def places(page_table, s, tokens, page_size, n_pages):
    """(page, row) of tokens of sequence s, page -1 where there is none."""
    column = tokens // page_size
    page = np.where(column < page_table.shape[1], page_table[s, np.minimum(column, page_table.shape[1] - 1)], -1)
    return np.where((page >= 0) & (page < n_pages), page, -1), tokens % page_size


def append(K, V, cache_k, cache_v, page_table, seq_ptr, seq_len, freqs, layout, magnitude, Q=None):
    """New contents of the caches and rotated queries (float64), with the bars' sizes of the keys and queries; what is not
    written keeps what it held.  Q_out of rows of no sequence is NaN."""
    ck, cv = cache_k.copy(), cache_v.copy()
    size = np.zeros_like(ck)
    page = cache_k.shape[2]
    q = np.full_like(Q, np.nan) if Q is not None else None
    q_size = np.zeros_like(Q) if Q is not None else None
    for s in range(len(seq_len)):
        rows = np.arange(seq_ptr[s], seq_ptr[s + 1])
        at = seq_len[s] - len(rows) + np.arange(len(rows))
        fine = (at >= 0) & (at < page_table.shape[1] * page)
        rows, at = rows[fine], at[fine]
        if len(rows) == 0:
            continue
        k, k_size = rotate(K[:, rows], at, freqs, layout, magnitude) if freqs is not None else (K[:, rows], 0 * K[:, rows])
        p, r = places(page_table, s, at, page, cache_k.shape[0])
        for n in range(len(rows)):
            if p[n] >= 0:
                ck[p[n], :, r[n]], cv[p[n], :, r[n]] = k[:, n], V[:, rows[n]]
                size[p[n], :, r[n]] = k_size[:, n]
        if Q is not None:
            q[:, rows], q_size[:, rows] = rotate(Q[:, rows], at, freqs, layout, magnitude)
    return ck, cv, size, q, q_size


def attend(Q, cache_k, cache_v, page_table, seq_ptr, seq_len, spec, scale, causal, dtype, once=False):
    """(O, lse, bar of O, bar of lse), float64; rows of no sequence are NaN.  once: probabilities are rounded to the
    storage type once, as the kernel of long chunks does."""
    Hq, T, d = Q.shape
    n_pages, Hkv, page, _ = cache_k.shape
    O, lse = np.full((Hq, T, d), np.nan), np.full((Hq, T), np.nan)
    O_bar, lse_bar = np.zeros((Hq, T, d)), np.zeros((Hq, T))
    for s in range(len(seq_len)):
        n = seq_ptr[s + 1] - seq_ptr[s]
        for t in range(n):
            row, i = seq_ptr[s] + t, seq_len[s] - n + t
            j = neighbours(spec, i, seq_len[s], causal)
            p, r = places(page_table, s, j, page, n_pages)
            p, r = p[p >= 0], r[p >= 0]
            O[:, row], lse[:, row] = 0.0, -np.inf
            if len(p) == 0:
                continue
            for g in range(Hkv):
                k, v = cache_k[p, g, r].astype(np.float64), cache_v[p, g, r].astype(np.float64)
                heads = slice(g * (Hq // Hkv), (g + 1) * (Hq // Hkv))
                q = Q[heads, row].astype(np.float64)
                z = scale * (q @ k.T)
                top = z.max(1, keepdims=True)
                e = np.exp(z - top)
                l = e.sum(1, keepdims=True)
                O[heads, row], lse[heads, row] = e @ v / l, (top + np.log(l))[:, 0]
                # A score is a sum of d products in 32 bits: d * 2^-24 of their sizes; scale, log2 e and the exponential add a
                # few half steps of the score's size and of 1.
                off = (d * 2.0 ** -24 * abs(scale) * (np.abs(q) @ np.abs(k).T)).max(1, keepdims=True) \
                    + 2.0 ** -22 * (1 + np.abs(z).max(1, keepdims=True))
                # probabilities enter the products as two numbers of the storage type: what is left is a half step of a half
                # step (fp16: or half its smallest step, 2^-25); sums over n keys in 32 bits: sqrt(n) half steps and to spare
                parts = {"f32": 0.0, "f16": 2.0 ** -21, "bf16": 2.0 ** -15}[dtype] if not once else HALF_STEP[dtype]
                share = e @ np.abs(v) / l
                O_bar[heads, row] = share * (2 * off + parts + (4 + np.sqrt(len(p))) * 2.0 ** -23) \
                    + np.abs(O[heads, row]) * HALF_STEP[dtype]
                if dtype == "f16":
                    O_bar[heads, row] += 2.0 ** -24 * np.abs(v).sum(0) / l + 2.0 ** -25
                lse_bar[heads, row] = (2 * off[:, 0]) + 2.0 ** -22 * (1 + np.abs(lse[heads, row]))
    return O, lse, O_bar, lse_bar
