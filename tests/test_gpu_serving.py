"""Rotary positions, appending to a paged cache and attention over it, against their definitions in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2502_01659_amd as sga
import serving_oracle as S
from sga_inputs import MaskSpec, KIND_GLOBAL_LOCAL, KIND_SLIDING

pytestmark = pytest.mark.gpu
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def host(t):
    return t.double().cpu().numpy()


def tokens(H, T, d, dtype, seed, layout="token"):
    """[H, T, d]: a view of [T, H, d] ("token"), of [T, H + 3, d + 16] ("slice"), or contiguous ("head")."""
    g = torch.Generator().manual_seed(seed)
    if layout == "head":
        x = torch.randn(H, T, d, generator=g)
        return x.to(DTYPE[dtype]).cuda()
    extra = (3, 16) if layout == "slice" else (0, 0)
    x = torch.randn(T, H + extra[0], d + extra[1], generator=g).to(DTYPE[dtype]).cuda()
    return x[:, :H, :d].transpose(0, 1)


def within(got, want, bar):
    got = host(got) if isinstance(got, torch.Tensor) else got
    assert np.array_equal(np.isfinite(got), np.isfinite(want))
    fine = np.isfinite(want)
    over = np.abs(got[fine] - want[fine]) - bar[fine]
    assert over.size == 0 or over.max() <= 0, (float(over.max()), float((np.abs(got[fine] - want[fine]) / (bar[fine] + 1e-300)).max()))
    return True


# ---- rotary ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("H,T,d,channels,memory", [
    (1, 1, 64, 64, "head"), (32, 1, 128, 128, "token"), (3, 65, 128, 64, "token"), (8, 257, 64, 32, "head"),
    (5, 33, 256, 256, "slice"), (2, 9, 32, 16, "token"), (4, 31, 80, 20, "token"), (3, 17, 7, 6, "head"),
    (1, 3000, 64, 64, "token"), (7, 13, 96, 2, "slice"), (2, 5, 1024, 1024, "head"),
])
def test_rotary(dtype, layout, H, T, d, channels, memory):
    freqs, _ = sga.rotary_frequencies(channels)
    rot = sga.Rotary(freqs, layout=layout, magnitude=1.25)
    x = tokens(H, T, d, dtype, T + d, memory)
    for inverse, positions, first in ((False, None, 0), (True, None, 131071), (False, torch.arange(T).cuda() * 7 - 3, 0)):
        print("rotary", dtype, layout, H, T, d, channels, memory, inverse, flush=True)
        at = positions.cpu().numpy() if positions is not None else first + np.arange(T)
        want, size = S.rotate(host(x), at, freqs.cpu().numpy(), layout, 1.25, inverse)
        bar = S.rotate_bar(want, size, dtype)
        bar[..., channels:] = 0                                # passed on as they are
        got = sga.rotary(x, rot, positions=positions, first=first, inverse=inverse)
        assert got.shape == x.shape and within(got, want, bar)
        same = x.clone() if memory != "slice" else tokens(H, T, d, dtype, T + d, memory)
        assert sga.rotary(same, rot, positions=positions, first=first, inverse=inverse, out=same) is same
        assert torch.equal(same, got)


def test_rotary_far_positions():
    """The angles keep their 2^-25 at 160 million tokens and at 2^50."""
    freqs, _ = sga.rotary_frequencies(64)
    x = tokens(2, 4096, 64, "f32", 5)
    for first in (160_000_000 - 4096, (1 << 31) - 5000, -(1 << 33), (1 << 50) + 12345):
        # the definition's product in exact integers: a frequency is m / 2^e, an angle modulo 2 pi needs pi to 160 bits
        two_pi = 2 * 314159265358979323846264338327950288419716939937510582097494459230781640628620899 * 10 ** 10
        angle = np.zeros((4096, 32))
        for k, f in enumerate(freqs.cpu().tolist()):
            num, den = f.as_integer_ratio()
            unit = 10 ** 90
            for t in range(0, 4096, 64):
                turns = (num * (first + t) * unit // den) % two_pi
                angle[t, k] = float(turns) / float(unit)
        rows = np.arange(0, 4096, 64)
        a, b = host(x)[:, rows, :32], host(x)[:, rows, 32:]
        cos, sin = np.cos(angle[rows]), np.sin(angle[rows])
        want = np.concatenate((a * cos - b * sin, a * sin + b * cos), -1)
        size = np.concatenate((np.abs(a) + np.abs(b),) * 2, -1)
        got = sga.rotary(x, sga.Rotary(freqs), first=first)
        assert within(host(got)[:, rows], want, S.rotate_bar(want, size, "f32"))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_gradient(layout):
    """The inverse of G is the gradient of <G, rotary(X)>: against differences in 64 bits and against the product."""
    freqs, magnitude = sga.rotary_frequencies(32, scaling="parts", factor=8.0, original_length=4096)
    rot = sga.Rotary(freqs, layout=layout, magnitude=magnitude)
    x, g = tokens(3, 70, 64, "f32", 1), tokens(3, 70, 64, "f32", 2)
    dx = host(sga.rotary(g, rot, first=900, inverse=True))
    f = lambda z: (S.rotate(z, 900 + np.arange(70), freqs.cpu().numpy(), layout, magnitude)[0] * host(g)).sum()
    X = host(x)
    for h, t, c in ((0, 0, 0), (1, 33, 17), (2, 69, 31), (0, 5, 40), (2, 1, 63)):
        up, down = X.copy(), X.copy()
        up[h, t, c] += 1e-3
        down[h, t, c] -= 1e-3
        # linear in x: the difference quotient is exact but for 64-bit rounding of the sum
        assert abs((f(up) - f(down)) / 2e-3 - dx[h, t, c]) <= 1e-6 * (1 + abs(dx[h, t, c]))
    y = host(sga.rotary(x, rot, first=900))
    # <G, Y> = <dX, X>: both sides are sums of 13,440 products, each off by less than 2^-20 of its pair's sizes
    assert abs((host(g) * y).sum() - (dx * X).sum()) <= 2.0 ** -20 * np.abs(X).sum() * 4


def test_rotary_without_rows_and_capture():
    freqs, _ = sga.rotary_frequencies(64)
    rot = sga.Rotary(freqs)
    assert sga.rotary(torch.empty(4, 0, 64, device="cuda"), rot).shape == (4, 0, 64)
    x, out = tokens(8, 300, 64, "f16", 3), torch.empty(8, 300, 64, dtype=torch.float16, device="cuda")
    at = torch.arange(300).cuda()
    sga.rotary(x, rot, positions=at, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sga.rotary(x, rot, positions=at, out=out)
    for step in range(3):
        at += 1000
        x.mul_(0.5)
        graph.replay()
        assert torch.equal(out, sga.rotary(x, rot, positions=at))


# ---- append ---------------------------------------------------------------------------------------
def batch_of(new, length, page, spare=2, padding=0, seed=0, columns=None, missing=()):
    """Random page tables for sequences of these lengths; `missing`: (sequence, column, entry) put in afterwards."""
    rng = np.random.default_rng(seed)
    columns = columns or max(1, max([-(-n // page) for n in length], default=1))
    need = [-(-n // page) for n in length]
    n_pages = max(1, sum(need) + spare)
    order = rng.permutation(n_pages)
    table = np.full((len(new), columns), -1, dtype=np.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n], at = order[at:at + n], at + n
    for s, c, entry in missing:
        table[s, c] = entry
    ptr = np.concatenate(([0], np.cumsum(new))).astype(np.int64)
    T = int(ptr[-1]) + padding
    dev = [torch.from_numpy(x).cuda() for x in (table, ptr, np.array(length, dtype=np.int32))]
    return sga.PagedBatch(*dev, T, page, n_pages), table, ptr, np.array(length), n_pages, T


def caches(n_pages, Hkv, page, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(n_pages, Hkv, page, d, generator=g).to(DTYPE[dtype]).cuda() for _ in range(2)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("new,length,page,Hq,Hkv,d,channels,layout,padding", [
    ([1], [1], 16, 4, 1, 64, 64, "half", 0),
    ([1] * 70, list(range(1, 71)), 16, 8, 8, 128, 128, "half", 3),
    ([5, 0, 130, 1], [5, 9, 300, 64], 24, 6, 2, 128, 64, "interleaved", 7),
    ([33, 2], [33, 1000], 1, 3, 3, 64, 64, "half", 0),
    ([40, 41], [100, 41], 7, 2, 1, 80, 20, "half", 1),
    ([300], [700], 256, 16, 4, 256, 256, "interleaved", 0),
    ([64, 1, 1, 17], [64, 65, 2000, 33], 64, 4, 4, 32, 32, "half", 0),
])
def test_append(dtype, new, length, page, Hq, Hkv, d, channels, layout, padding):
    print("append", dtype, new[:4], page, d, flush=True)
    batch, table, ptr, lens, n_pages, T = batch_of(new, length, page, padding=padding, seed=len(new))
    ck, cv = caches(n_pages, Hkv, page, d, dtype, 9)
    K, V, Q = tokens(Hkv, T, d, dtype, 1), tokens(Hkv, T, d, dtype, 2, "slice"), tokens(Hq, T, d, dtype, 3)
    freqs, magnitude = sga.rotary_frequencies(channels, scaling="linear", factor=2.0)
    want = S.append(host(K), host(V), host(ck), host(cv), table, ptr, lens, freqs.cpu().numpy(), layout, magnitude, host(Q))
    out = torch.full((Hq, T, d), 7.0, dtype=DTYPE[dtype], device="cuda")
    sga.cache_append(K, V, ck, cv, batch, rotary=sga.Rotary(freqs, layout, magnitude), Q=Q, Q_out=out)
    bar = S.rotate_bar(want[0], want[2], dtype)
    bar[want[2] == 0] = 0                                     # not written, or not turned
    assert within(ck, want[0], bar)
    assert np.array_equal(host(cv), want[1])
    q = host(out)
    real = np.isfinite(want[3])
    assert (q[~real] == 7.0).all()                           # padding rows are left as they were
    assert within(q[real], want[3][real], S.rotate_bar(want[3], want[4], dtype)[real])
    # without rotation, the values as they are
    ck2, cv2 = caches(n_pages, Hkv, page, d, dtype, 9)
    plain = S.append(host(K), host(V), host(ck2), host(cv2), table, ptr, lens, None, "half", 1.0)
    sga.cache_append(K, V, ck2, cv2, batch)
    assert np.array_equal(host(ck2), plain[0]) and np.array_equal(host(cv2), plain[1])
    # queries in place
    mine = Q.clone()
    assert sga.cache_append(K, V, ck2, cv2, batch, rotary=sga.Rotary(freqs, layout, magnitude), Q=mine, Q_out=mine) is mine
    assert torch.equal(mine[:, :int(ptr[-1])], out[:, :int(ptr[-1])])


def test_append_passes_over_missing_pages():
    """No page, a page that does not exist, positions before the first token and behind the table's last column."""
    batch, table, ptr, lens, n_pages, T = batch_of([40, 30, 50], [40, 64, 60], 16, columns=4,
                                                   missing=[(0, 1, -1), (1, 3, 10 ** 6), (2, 3, -7)])
    batch.seq_len[1] = 20                                     # its first ten tokens lie before position 0
    batch.seq_len[2] = 70                                     # its last six behind column 3
    lens[1], lens[2] = 20, 70
    ck, cv = caches(n_pages, 2, 16, 64, "f32", 4)
    K, V, Q = (tokens(2, T, 64, "f32", s) for s in (1, 2, 3))
    freqs, _ = sga.rotary_frequencies(64)
    want = S.append(host(K), host(V), host(ck), host(cv), table, ptr, lens, freqs.cpu().numpy(), "half", 1.0, host(Q))
    sga.cache_append(K, V, ck, cv, batch, rotary=sga.Rotary(freqs))
    bar = S.rotate_bar(want[0], want[2], "f32")
    bar[want[2] == 0] = 0
    assert within(ck, want[0], bar) and np.array_equal(host(cv), want[1])


# ---- attention ------------------------------------------------------------------------------------
def long_chunks(dtype, T, n_seqs, group, d, page):
    """16-bit calls whose sequences bring more than 32 rows on average take tiles of 128 rows, where a row of keys has 128 to
    512 bytes; there a probability is rounded once.  (In full precision neither kernel rounds it.)"""
    return dtype != "f32" and d >= 64 and T * group > 32 * n_seqs


def check_attention(dtype, new, length, page, Hq, Hkv, d, spec, causal=True, padding=0, memory="token", missing=(), scale=None,
                    workspace=True, rotten=True, seed=0, change=None, columns=None):
    print("attend", dtype, new[:6], length[:6], page, Hq, Hkv, d, spec, causal, flush=True)
    batch, table, ptr, lens, n_pages, T = batch_of(new, length, page, padding=padding, seed=seed, missing=missing, columns=columns)
    ck, cv = caches(n_pages, Hkv, page, d, dtype, seed + 1)
    if rotten:                                               # memory that no token was written to may hold anything
        used = torch.zeros(n_pages, page, dtype=torch.bool)
        for s, n in enumerate(length):
            p, r = S.places(table, s, np.arange(min(n, table.shape[1] * page)), page, n_pages)
            used[p[p >= 0], r[p >= 0]] = True
        used = used.cuda()[:, None, :, None]
        ck, cv = torch.where(used, ck, float("nan")), torch.where(used, cv, float("inf"))
    if change:
        change(ck, cv, table)
    Q = tokens(Hq, T, d, dtype, seed + 3, memory)
    scale = 1 / math.sqrt(d) if scale is None else scale
    long = long_chunks(dtype, T, len(new), Hq // Hkv, d, page)
    want, want_lse, bar, lse_bar = S.attend(host(Q), host(ck), host(cv), table, ptr, lens, spec, scale, causal, dtype, long)
    O = torch.full((Hq, T, d), 7.0, dtype=DTYPE[dtype], device="cuda")
    lse = torch.full((Hq, T), 7.0, device="cuda")
    ws = sga.alloc_paged_workspace(batch, spec, Hq, Hkv, d, dtype) if workspace else None
    assert sga.sga_profile_enable(1) == 0
    sga.attention_paged(Q, ck, cv, batch, spec, scale, causal=causal, O=O, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    kernel = sga.sga_profile_last_kernel()
    sga.sga_profile_enable(0)
    assert dtype == "f32" or kernel == ("paged_chunk_kernel" if long else "paged_kernel")
    end = int(ptr[-1])
    assert (host(O)[:, end:] == 7.0).all() and (host(lse)[:, end:] == 7.0).all()
    assert within(host(O)[:, :end], want[:, :end], bar[:, :end])
    assert within(host(lse)[:, :end], want_lse[:, :end], lse_bar[:, :end])
    return O, lse


def full(L):
    return MaskSpec(KIND_SLIDING, L, window=L)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("page", [16, 24, 1])
def test_attention_types(dtype, d, page):
    check_attention(dtype, [1, 3, 20], [77, 40, 20], page, 4, 2, d, full(96), padding=2)
    check_attention(dtype, [1, 9], [130, 50], page, 3, 1, d, MaskSpec(KIND_GLOBAL_LOCAL, 144, window=17, n_global=5))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (5, 5), (6, 2), (7, 1), (16, 2), (40, 2), (64, 1)])
def test_attention_shared_heads(dtype, Hq, Hkv):
    check_attention(dtype, [1, 1, 6], [1, 33, 100], 16, Hq, Hkv, 64, full(112))


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("spec", [
    full(160), MaskSpec(KIND_SLIDING, 160, window=0), MaskSpec(KIND_SLIDING, 160, window=1), MaskSpec(KIND_SLIDING, 160, window=31),
    MaskSpec(KIND_SLIDING, 160, window=70), MaskSpec(KIND_GLOBAL_LOCAL, 160, window=3, n_global=1),
    MaskSpec(KIND_GLOBAL_LOCAL, 160, window=20, n_global=40), MaskSpec(KIND_GLOBAL_LOCAL, 160, window=0, n_global=0),
    MaskSpec(KIND_GLOBAL_LOCAL, 160, window=5, n_global=160), MaskSpec(KIND_SLIDING, 100, window=40),
])
def test_attention_masks(dtype, causal, spec):
    # whole prompts, pieces in the middle, single tokens; sequences that pass the mask's length
    check_attention(dtype, [150, 37, 1, 0, 64], [150, 90, 144, 12, 64], 16, 4, 2, 64, spec, causal=causal)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_attention_split_sequences(dtype):
    """Few long sequences: pieces of the keys on workgroups of their own, joined afterwards."""
    for page in (16, 40):
        check_attention(dtype, [1, 2, 1], [5000, 1203, 1], page, 8, 2, 64, full(5008))
        check_attention(dtype, [1, 2, 1], [5000, 1203, 1], page, 8, 2, 64, full(5008), workspace=False)
        check_attention(dtype, [2, 1], [3000, 2999], page, 2, 1, 128, MaskSpec(KIND_GLOBAL_LOCAL, 3000, window=1500, n_global=70))


@pytest.mark.parametrize("memory", ["head", "token", "slice"])
def test_attention_strides(memory):
    check_attention("f16", [7, 1, 30], [40, 90, 30], 32, 6, 3, 64, full(96), memory=memory)


def test_attention_of_given_back_pages():
    """Pages behind a window are gone; a window that reaches into a missing page passes over it; a row may be left empty."""
    spec = MaskSpec(KIND_SLIDING, 400, window=50)
    gone = [(0, c, -1) for c in range(0, 21)]                # tokens 0 .. 335 of 400: all that the window leaves
    check_attention("f16", [1, 1], [400, 390], 16, 4, 4, 64, spec, missing=gone)
    check_attention("f32", [3, 1], [400, 390], 16, 4, 4, 64, spec, missing=gone + [(0, 22, -1), (1, 24, 10 ** 7)])
    check_attention("f32", [3, 1], [400, 390], 16, 4, 4, 64, spec, missing=[(0, c, -1) for c in range(25)])
    check_attention("bf16", [3, 1], [400, 390], 5, 4, 4, 64, spec, missing=[(1, c, -1) for c in range(70, 78)])


@pytest.mark.parametrize("page", [16, 24])
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_attention_of_infinities_that_are_not_seen(dtype, page):
    """Keys and values of a token hold infinities and NaN: rows that do not see it are as if it were not there."""
    def spoil(ck, cv, table):
        for token, k, v in ((20, float("nan"), 1.0), (41, 1.0, float("inf")), (60, 1.0, float("nan"))):
            ck[table[0, token // page], 0, token % page, 3] *= k
            cv[table[0, token // page], 0, token % page, 5] *= v

    for causal in (True, False):
        # 80 rows of a prompt whose windows of 4 hold one of the three tokens or none
        batch, table, ptr, lens, n_pages, T = batch_of([80], [80], page, seed=0)
        ck, cv = caches(n_pages, 2, page, 64, dtype, 1)
        clean = [ck.clone(), cv.clone()]
        spoil(ck, cv, table)
        spec = MaskSpec(KIND_SLIDING, 80, window=4)
        Q = tokens(2, T, 64, dtype, 3)
        got = host(sga.attention_paged(Q, ck, cv, batch, spec, 0.125, causal=causal))
        want, _, bar, _ = S.attend(host(Q), host(clean[0]), host(clean[1]), table, ptr, lens, spec, 0.125, causal, dtype,
                                   once=long_chunks(dtype, T, 1, 1, 64, page))
        i = np.arange(80)
        sees = lambda token: (np.abs(i - token) <= 4) & ((token <= i) | (not causal))
        assert np.isnan(got[0, sees(20)]).all()
        assert (~np.isfinite(got[0, sees(41), 5])).all() and (~np.isfinite(got[0, sees(60), 5])).all()
        for h in range(2):
            free = ~(sees(20) | sees(41) | sees(60)) if h == 0 else i >= 0
            assert within(got[h, free], want[h, free], bar[h, free])
        rest = [c for c in range(64) if c != 5]
        only_v = (sees(41) | sees(60)) & ~sees(20)
        assert within(got[0][only_v][:, rest], want[0][only_v][:, rest], bar[0][only_v][:, rest])


def test_attention_of_one_key_and_large_scores():
    O, lse = check_attention("bf16", [1, 1], [1, 1], 16, 4, 4, 128, full(16))
    check_attention("f32", [5], [64], 16, 2, 1, 64, full(64), scale=6.0)       # one key takes nearly all
    check_attention("f32", [5], [64], 16, 2, 1, 64, full(64), scale=-0.5)
    check_attention("f16", [5], [64], 16, 2, 1, 64, full(64), scale=0.0)


@pytest.mark.parametrize("dtype,d", [("f16", 64), ("f16", 128), ("f16", 256), ("bf16", 64), ("bf16", 128), ("bf16", 256),
                                     ("f32", 32), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("causal", [True, False])
def test_attention_long_chunks(dtype, d, causal):
    """Tiles of 128 rows: ragged ends, tiles of few rows, several pieces, global tokens before the window, missing pages."""
    check_attention(dtype, [129, 1, 300], [129, 40, 700], 16, 2, 2, d, full(704), causal=causal, padding=5)
    check_attention(dtype, [97], [600], 48, 3, 1, d, MaskSpec(KIND_SLIDING, 608, window=33), causal=causal, memory="slice")
    check_attention(dtype, [70, 0, 65], [3000, 7, 65], 16, 4, 1, d, MaskSpec(KIND_GLOBAL_LOCAL, 3008, window=1200, n_global=70),
                    causal=causal)
    check_attention(dtype, [130], [1000], 32, 2, 2, d, full(1000), causal=causal, missing=[(0, 3, -1), (0, 17, 10 ** 6), (0, 31, -9)])
    check_attention(dtype, [200], [150], 16, 2, 1, d, full(160), causal=causal)      # the first 50 lie before position 0
    check_attention(dtype, [100], [100], 16, 5, 5, d, MaskSpec(KIND_SLIDING, 80, window=0), causal=causal, workspace=False)


@pytest.mark.parametrize("d,dtype", [(64, "f16"), (128, "bf16"), (256, "f16"), (32, "f32"), (64, "f32"), (128, "f32")])
@pytest.mark.parametrize("page", [1, 5, 24, 100])
def test_attention_long_chunks_pages_of_any_size(d, dtype, page):
    check_attention(dtype, [129, 1, 300], [129, 40, 700], page, 2, 2, d, full(704), padding=5)
    check_attention(dtype, [60], [2500], page, 2, 1, d, full(2500), causal=False)          # more blocks than are asked for at once
    check_attention(dtype, [70, 0, 65], [3000, 7, 65], page, 4, 1, d, MaskSpec(KIND_GLOBAL_LOCAL, 3008, window=1200, n_global=70))
    last = (1000 - 1) // page
    check_attention(dtype, [130], [1000], page, 2, 2, d, full(1000), missing=[(0, 3, -1), (0, last // 2, 10 ** 6), (0, last, -9)])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_attention_long_chunks_of_uneven_scores(dtype):
    """Scores that grow along the keys raise the reference again and again; one key that takes all; a zero and a negative scale."""
    def grow(ck, cv, table):
        for t in range(400):
            ck[table[0, t // 16], :, t % 16] *= 0.02 * t
    for scale in (1.0, -1.0, 0.0, 0.01):
        check_attention(dtype, [140], [400], 16, 2, 1, 64, full(400), scale=scale, change=grow)
    check_attention(dtype, [200], [200], 16, 12, 12, 64, MaskSpec(KIND_SLIDING, 200, window=200))
    check_attention(dtype, [200], [200], 16, 4, 2, 64, MaskSpec(KIND_SLIDING, 200, window=200), causal=False)


def test_attention_far_pages():
    """A cache of more than 2^31 elements, the tokens in its last pages."""
    page, Hkv, d = 64, 8, 128
    n_pages = (1 << 31) // (page * Hkv * d) + 40
    ck, cv = (torch.empty(n_pages, Hkv, page, d, dtype=torch.float16, device="cuda") for _ in range(2))
    table = np.array([[n_pages - 1, 0, n_pages - 3]], dtype=np.int32)
    ptr, lens = np.array([0, 150]), np.array([150])
    batch = sga.PagedBatch(*(torch.from_numpy(x).cuda() for x in (table, ptr, lens.astype(np.int32))), 150, page, n_pages)
    K, V, Q = (tokens(h, 150, d, "f16", s) for h, s in ((8, 1), (8, 2), (16, 3)))
    sga.cache_append(K, V, ck, cv, batch)
    near = np.array([[0, 1, 2]], dtype=np.int32)
    small = [c[torch.from_numpy(table[0].astype(np.int64)).cuda()] for c in (ck, cv)]
    for t in range(150):
        assert torch.equal(small[0][t // page, :, t % page], K[:, t])
    spec = full(150)
    want, _, bar, _ = S.attend(host(Q), host(small[0]), host(small[1]), near, ptr, lens, spec, 0.1, True, "f16", True)
    assert within(sga.attention_paged(Q, ck, cv, batch, spec, 0.1), want, bar)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("seed", range(3))
def test_attention_of_many_sequences(dtype, seed):
    """More sequences than a wavefront looks at at a time, some without new tokens, tiles that are cut and tiles that are not."""
    rng = np.random.default_rng(seed)
    n = [150, 70, 200][seed]
    new = rng.integers(0, 3, n).tolist()
    length = [int(a + b) for a, b in zip(new, np.where(rng.random(n) < 0.03, 1500, rng.integers(0, 60, n)))]
    new[0] = new[-1] = 0
    check_attention(dtype, new, length, 16, 4, 2, 64, full(1600), seed=seed)
    check_attention(dtype, new, length, 7, 6, 2, 64, MaskSpec(KIND_GLOBAL_LOCAL, 1600, window=25, n_global=2), seed=seed, workspace=False)
    new = [x * 17 for x in new]
    length = [a + b for a, b in zip(new, length)]
    check_attention(dtype, new, length, 16, 4, 2, 64, full(1600), seed=seed, padding=3)


@pytest.mark.parametrize("seed", range(24))
def test_attention_drawn(seed):
    """Drawn sizes over the whole range of what a call may be."""
    rng = np.random.default_rng(1000 + seed)
    dtype, d = rng.choice(["f32", "f16", "bf16"]), int(rng.choice([32, 64, 128, 256]))
    Hkv, G, S = int(rng.integers(1, 4)), int(rng.choice([1, 1, 2, 3, 5, 8, 17])), int(rng.integers(1, 9))
    page = int(rng.choice([1, 3, 16, 17, 32, 48, 64, 200]))
    most = int(rng.choice([1, 4, 40, 150]))
    new = rng.integers(0, most + 1, S).tolist()
    length = [int(a + b) for a, b in zip(new, rng.integers(0, int(rng.choice([1, 50, 900])), S))]
    if rng.random() < 0.2:
        length[0] = max(0, new[0] - 3)                       # tokens before position 0
    L = max(1, max(length) - int(rng.choice([0, 0, 5])))
    w = int(rng.choice([0, 5, 40, 300, 10 ** 6]))
    spec = MaskSpec(KIND_SLIDING, L, window=w) if rng.random() < 0.5 else MaskSpec(KIND_GLOBAL_LOCAL, L, window=w, n_global=min(L, int(rng.choice([0, 1, 33, 70]))))
    missing = [(int(rng.integers(S)), int(rng.integers(max(1, -(-max(length) // page)))), int(rng.choice([-1, 1 << 30, -(1 << 31)])))
               for _ in range(int(rng.choice([0, 0, 3])))]
    check_attention(dtype, new, length, page, Hkv * G, Hkv, d, spec, causal=bool(rng.random() < 0.7), padding=int(rng.integers(3)),
                    memory=str(rng.choice(["head", "token", "slice"])), missing=missing, workspace=bool(rng.random() < 0.7),
                    seed=seed, scale=float(rng.choice([0.1, 1 / math.sqrt(d), -0.2])))


def test_attention_results_do_not_change():
    """The same call twice, and after another call has used the workspace, gives the same bits."""
    for new, length in (([1] * 5, [3000, 20, 700, 1, 1500]), ([100, 30, 1], [900, 500, 2000])):
        batch, table, ptr, lens, n_pages, T = batch_of(new, length, 16)
        ck, cv = caches(n_pages, 2, 16, 128, "bf16", 3)
        Q, spec = tokens(8, T, 128, "bf16", 4), full(3000)
        ws = sga.alloc_paged_workspace(batch, spec, 8, 2, 128, "bf16")
        a = sga.attention_paged(Q, ck, cv, batch, spec, 0.09, workspace=ws, want_lse=True)
        sga.attention_paged(Q * 2, ck, cv, batch, MaskSpec(KIND_SLIDING, 3000, window=100), 0.2, causal=False, workspace=ws)
        ws.fill_(255)
        b = sga.attention_paged(Q, ck, cv, batch, spec, 0.09, workspace=ws, want_lse=True)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_two_captured_graphs_share_a_workspace():
    batch, table, ptr, lens, n_pages, T = batch_of([1, 40, 1], [2500, 700, 64], 16)
    ck, cv = caches(n_pages, 2, 16, 64, "f16", 3)
    Q, spec = tokens(4, T, 64, "f16", 4), full(2500)
    ws = sga.alloc_paged_workspace(batch, spec, 4, 2, 64, "f16")
    want = [sga.attention_paged(Q * k, ck, cv, batch, spec, 0.125) for k in (1, 2)]
    X, out, graphs = [Q * 1, Q * 2], [torch.zeros_like(Q) for _ in range(2)], []
    torch.cuda.synchronize()
    for k in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            sga.attention_paged(X[k], ck, cv, batch, spec, 0.125, O=out[k], workspace=ws)
        graphs.append(g)
    eager = [sga.attention_paged(X[k], ck, cv, batch, spec, 0.125, workspace=ws) for k in range(2)]
    for _ in range(3):
        for k in (0, 1, 1, 0):
            out[k].zero_()
            graphs[k].replay()
            assert torch.equal(out[k], eager[k])
            # without a workspace no tile is cut: the same sums in another order
            assert ((out[k].float() - want[k].float()).abs() <= 2e-3 * (1 + want[k].float().abs())).all()
            sga.attention_paged(X[1 - k], ck, cv, batch, spec, 0.125, workspace=ws)


def test_refusals_of_device_tensors():
    batch, table, ptr, lens, n_pages, T = batch_of([2, 3], [20, 30], 16)
    ck, cv = caches(n_pages, 2, 16, 64, "f16", 3)
    Q, K = tokens(4, T, 64, "f16", 4), tokens(2, T, 64, "f16", 5)
    rot = sga.Rotary(sga.rotary_frequencies(64)[0])
    spec = full(32)
    for bad in (lambda: sga.attention_paged(Q[:, :4], ck, cv, batch, spec, 0.1), lambda: sga.attention_paged(Q.float(), ck, cv, batch, spec, 0.1),
                lambda: sga.attention_paged(Q, ck[:, :, :8], cv, batch, spec, 0.1), lambda: sga.attention_paged(Q, ck.transpose(1, 2), cv, batch, spec, 0.1),
                lambda: sga.attention_paged(Q, ck[:-1], cv[:-1], batch, spec, 0.1), lambda: sga.attention_paged(Q, ck, cv, batch, spec, 0.1, O=K),
                lambda: sga.attention_paged(Q, ck, cv, batch, spec, 0.1, lse=torch.empty(4, T, device="cuda", dtype=torch.float64)),
                lambda: sga.attention_paged(Q, ck, cv, batch, spec, 0.1, O=torch.empty(4, 1, 64, dtype=torch.float16, device="cuda").expand(4, T, 64)),
                lambda: sga.attention_paged(Q, ck, cv.float(), batch, spec, 0.1), lambda: sga.attention_paged(Q.cpu(), ck, cv, batch, spec, 0.1),
                lambda: sga.attention_paged(Q, ck, cv, batch, spec, 0.1, workspace=torch.empty(1000)),
                lambda: sga.cache_append(K[:1], K, ck, cv, batch), lambda: sga.cache_append(K, K, ck, cv, batch, Q=Q),
                lambda: sga.cache_append(K, K, ck, cv, batch, rotary=rot, Q_out=Q), lambda: sga.cache_append(K, Q, ck, cv, batch),
                lambda: sga.rotary(Q, rot, positions=torch.arange(T, device="cuda", dtype=torch.int32)),
                lambda: sga.rotary(Q, rot, positions=torch.arange(T + 1, device="cuda")), lambda: sga.rotary(Q, rot, out=Q[:, :-1]),
                lambda: sga.rotary(Q[..., ::2], rot), lambda: sga.Rotary(sga.rotary_frequencies(64)[0].float()),
                lambda: sga.Rotary(sga.rotary_frequencies(64)[0], layout="other")):
        with pytest.raises((ValueError, TypeError)):
            bad()
    with pytest.raises(sga.SgaError):                        # more channels than the head has
        sga.rotary(Q[..., :32], rot)
    with pytest.raises(sga.SgaError):                        # an address off 16 bytes
        sga.attention_paged(torch.empty(4 * T * 64 + 1, dtype=torch.float16, device="cuda")[1:].view(4, T, 64), ck, cv, batch, spec, 0.1)
    with pytest.raises(TypeError):
        sga.rotary(Q.double(), rot)
    with pytest.raises(sga.SgaError):                        # the other calls know nothing of bf16
        sga.attention_forward_implicit(*(torch.zeros(1, 8, 48, device="cuda"),) * 3, MaskSpec(KIND_SLIDING, 8, window=1), 0.1)


def test_attention_without_tokens():
    batch, *_ = batch_of([0, 0], [5, 9], 16)
    ck, cv = caches(batch.n_pages, 2, 16, 64, "f16", 1)
    Q = torch.empty(4, 0, 64, dtype=torch.float16, device="cuda")
    assert sga.attention_paged(Q, ck, cv, batch, full(16), 0.1).shape == (4, 0, 64)
    sga.cache_append(Q[:2], Q[:2], ck, cv, batch)


# ---- together --------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("d,G", [(64, 1), (128, 4)])
def test_generation_step_by_step_is_the_whole_sequence(dtype, d, G):
    """Prompts in pieces, then single tokens, through the cache; against the framework's call on the whole sequence,
    the mask as an explicit graph."""
    Hkv, page, w, g = 2, 16, 40, 3
    Hq, L = Hkv * G, [200, 131]
    spec = MaskSpec(KIND_GLOBAL_LOCAL, 208, window=w, n_global=g)
    freqs, magnitude = sga.rotary_frequencies(d, scaling="parts", factor=4.0, original_length=64)
    rot, scale = sga.Rotary(freqs, "half", magnitude), 1 / math.sqrt(d)
    Q, K, V = ([tokens(h, n, d, dtype, 10 * k + s) for s, n in enumerate(L)] for k, h in ((1, Hq), (2, Hkv), (3, Hkv)))
    batch0, table, *_ , n_pages, _ = batch_of([1, 1], L, page)
    ck, cv = caches(n_pages, Hkv, page, d, dtype, 1)
    done = [0, 0]
    O = [torch.empty_like(q) for q in Q]
    dev_table = batch0.page_table
    for take in [(64, 100), (1, 1), (70, 1), (33, 0), (0, 7)] + [(1, 1)] * 40:
        n = [min(t, L[s] - done[s]) for s, t in enumerate(take)]
        if sum(n) == 0:
            continue
        ptr = torch.tensor([0, n[0], n[0] + n[1]], device="cuda")
        lens = torch.tensor([done[0] + n[0], done[1] + n[1]], dtype=torch.int32, device="cuda")
        batch = sga.PagedBatch(dev_table, ptr, lens, sum(n), page, n_pages)
        q, k, v = (torch.cat([x[s][:, done[s]:done[s] + n[s]] for s in range(2)], 1) for x in (Q, K, V))
        q = sga.cache_append(k, v, ck, cv, batch, rotary=rot, Q=q)
        ws = sga.alloc_paged_workspace(batch, spec, Hq, Hkv, d, dtype)
        o = sga.attention_paged(q, ck, cv, batch, spec, scale, workspace=ws)
        for s in range(2):
            O[s][:, done[s]:done[s] + n[s]] = o[:, int(ptr[s]):int(ptr[s + 1])]
            done[s] += n[s]
    for s in range(2):
        n = done[s]
        i, j = np.arange(n)[:, None], np.arange(n)[None]
        see = (j <= i) & ((i - j <= w) | (j < g) | (i < g))
        row_ptr = torch.from_numpy(np.concatenate(([0], see.sum(1).cumsum())).astype(np.int64)).cuda()
        col = torch.from_numpy(np.nonzero(see)[1].astype(np.int32)).cuda()
        q = sga.rotary(Q[s][:, :n].contiguous(), rot)
        k = sga.rotary(K[s][:, :n].repeat_interleave(G, 0).contiguous(), rot)
        v = V[s][:, :n].repeat_interleave(G, 0).contiguous()
        whole = sga.attention_forward(q, k, v, row_ptr, col, scale)
        # two calls within the framework's bars of the same number: 1e-5 (fp32), 2e-3 (fp16), relative to 1 + |O|
        off = (whole.float() - O[s][:, :n].float()).abs() / (1 + whole.float().abs())
        assert off.max().item() <= 2 * {"f32": 1e-5, "f16": 2e-3}[dtype]


def test_captured_steps_follow_the_lengths():
    """Append and attention captured once, replayed while lengths and tokens change, against eager calls."""
    Hq, Hkv, d, page, L = 8, 2, 64, 16, 4000
    spec = MaskSpec(KIND_GLOBAL_LOCAL, L, window=1000, n_global=4)
    batch, table, *_, n_pages, T = batch_of([1, 1, 1], [L, L, L], page)
    batch.seq_len.copy_(torch.tensor([1, 700, 3000], dtype=torch.int32))
    ck, cv = caches(n_pages, Hkv, page, d, "f16", 2)
    freqs, _ = sga.rotary_frequencies(d)
    rot = sga.Rotary(freqs)
    ws = sga.alloc_paged_workspace(batch, spec, Hq, Hkv, d, "f16")
    K, V, Q = (tokens(h, T, d, "f16", s) for h, s in ((Hkv, 1), (Hkv, 2), (Hq, 3)))
    q, O = torch.empty_like(Q), torch.empty_like(Q)
    lse = torch.empty(Hq, T, device="cuda")

    def step(q, O, lse, ck, cv, ws):
        sga.cache_append(K, V, ck, cv, batch, rotary=rot, Q=Q, Q_out=q)
        sga.attention_paged(q, ck, cv, batch, spec, 0.125, O=O, lse=lse, workspace=ws)

    step(q, O, lse, ck, cv, ws)
    torch.cuda.synchronize()
    ck2, cv2 = ck.clone(), cv.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(q, O, lse, ck, cv, ws)
    side = torch.cuda.Stream()
    ws2 = torch.empty_like(ws)
    q2, O2, lse2 = torch.empty_like(q), torch.empty_like(O), torch.empty_like(lse)
    for k in range(5):
        batch.seq_len += 37
        K.add_(0.1)
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):                       # another stream, another workspace
            step(q2, O2, lse2, ck2, cv2, ws2)
        side.synchronize()
        assert torch.equal(O, O2) and torch.equal(lse, lse2) and torch.equal(q, q2)
    assert torch.isfinite(O).all()


@pytest.mark.parametrize("dtype,d,page,new", [("f16", 128, 16, [1, 3]), ("bf16", 64, 24, [90, 41]), ("f32", 64, 32, [100, 1]),
                                              ("f32", 32, 8, [2, 1]), ("f16", 256, 5, [70, 70])])
def test_caches_whose_pages_take_turns(dtype, d, page, new):
    """Keys and values page by page in one buffer, beside those of other layers: the same results as in two caches, and nothing
    written beside them."""
    Hq, Hkv, lens = 4, 2, [700, 300]
    spec = MaskSpec(KIND_GLOBAL_LOCAL, 768, window=200, n_global=5)
    batch, table, ptr, _, n_pages, T = batch_of(new, lens, page)
    ck, cv = caches(n_pages, Hkv, page, d, dtype, 1)
    whole = torch.full((n_pages, 6, Hkv, page, d), 7.0, dtype=DTYPE[dtype], device="cuda")
    pk, pv = whole[:, 2], whole[:, 3]
    pk.copy_(ck)
    pv.copy_(cv)
    rot = sga.Rotary(sga.rotary_frequencies(d)[0])
    Q, K, V = (tokens(h, T, d, dtype, s) for h, s in ((Hq, 1), (Hkv, 2), (Hkv, 3)))
    ws = sga.alloc_paged_workspace(batch, spec, Hq, Hkv, d, dtype)
    out = []
    for k, v in ((ck, cv), (pk, pv)):
        q = sga.cache_append(K, V, k, v, batch, rotary=rot, Q=Q)
        out.append((q, *sga.attention_paged(q, k, v, batch, spec, 0.1, workspace=ws, want_lse=True)))
    assert all(torch.equal(a, b) for a, b in zip(*out))
    assert torch.equal(pk, ck) and torch.equal(pv, cv)
    assert (whole[:, [0, 1, 4, 5]] == 7).all()


def test_two_streams_at_once():
    """Calls of two streams that overlap in time, each with a workspace of its own."""
    spec = MaskSpec(KIND_SLIDING, 4096, window=4096)
    work = []
    for s, new in enumerate(([1, 1, 1], [200, 3, 64])):
        batch, *_, n_pages, T = batch_of(new, [4000, 900, 2500], 16)
        ck, cv = caches(n_pages, 2, 16, 128, "bf16", s)
        work.append((tokens(8, T, 128, "bf16", s), ck, cv, batch, spec, 0.09))
    want = [sga.attention_paged(*w, workspace=sga.alloc_paged_workspace(w[3], spec, 8, 2, 128, "bf16")) for w in work]
    spaces = [sga.alloc_paged_workspace(w[3], spec, 8, 2, 128, "bf16") for w in work]
    outs = [[torch.zeros_like(w[0]) for _ in range(8)] for w in work]
    streams = [torch.cuda.Stream() for _ in work]
    torch.cuda.synchronize()
    for i in range(8):
        for w, space, out, stream in zip(work, spaces, outs, streams):
            with torch.cuda.stream(stream):
                sga.attention_paged(*w, O=out[i], workspace=space)
    torch.cuda.synchronize()
    assert all(torch.equal(o, x) for x, out in zip(want, outs) for o in out)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("new", [1, 20, 100])
@pytest.mark.parametrize("spoiled", [False, True])           # one value of a token is infinite: its channel is, the others are as they were
def test_attention_of_many_small_weights(dtype, new, spoiled):
    """Long contexts often give a few first tokens nearly all of the weight: here tokens 0, 32, 64 and 96, one for each wavefront's first
    block, whose values are 0, and 32,764 tokens `gap` below them, which alone decide O.  Their weights are far below the smallest
    number of fp16; together they are not.  Scores are 0 and gap exactly, so O = e^-gap sum(v) / (4 + 32,764 e^-gap)."""
    n, d, page = 32768, 64, 64
    long = kernel_of(dtype, new, 1, 1, d, full(n), False, n) == "paged_chunk_kernel"
    batch, table, ptr, lens, n_pages, T = batch_of([new], [n], page)
    ck, cv = (torch.zeros(n_pages, 1, page, d, dtype=DTYPE[dtype], device="cuda") for _ in range(2))
    values = torch.rand(n, d, generator=torch.Generator().manual_seed(1)).add_(0.5).to(DTYPE[dtype])
    values[[0, 32, 64, 96]] = 0
    if spoiled:
        values[1000, 5] = math.inf
    at = torch.from_numpy(table[0].astype(np.int64)).cuda()
    cv[at, 0] = values.view(-1, page, d).cuda()
    for t in (0, 32, 64, 96):
        ck[at[t // page], 0, t % page, 0] = 1
    Q = torch.zeros(1, T, d, dtype=DTYPE[dtype], device="cuda")
    Q[..., 0] = 1
    total = host(values).sum(0)
    for gap in (12.0, 14.5, 16.0, 16.75, 17.25, 17.5, 18.5, 20.0):
        for workspace in (None, sga.alloc_paged_workspace(batch, full(n), 1, 1, d, dtype)):
            print("small weights", dtype, new, spoiled, gap, flush=True)
            assert sga.sga_profile_enable(1) == 0
            O, lse = sga.attention_paged(Q, ck, cv, batch, full(n), gap, causal=False, workspace=workspace, want_lse=True)
            torch.cuda.synchronize()
            kernel = sga.sga_profile_last_kernel()
            sga.sga_profile_enable(0)
            assert kernel == ("paged_chunk_kernel" if long else "paged_kernel")
            sums = 4 + (n - 4) * math.exp(-gap)
            want = math.exp(-gap) * total / sums
            # The exponent is at most 29 and off by three half steps of it: 2^-17 of a weight.  Sums in 32 bits: an addition is off by
            # half a step of the sum, that of the four first tokens, and every lane makes at most n / 32 of them to l (2^-24 n / 32 in all),
            # n / 16 to O (of what O holds: sqrt(n) half steps and to spare).  Numerators enter the products
            # as two numbers of 16 bits or rounded once, fp16 ones that reach 2^10 at least with an absolute half step of 2^-25.
            parts = {"f32": 0.0, "f16": 2.0 ** -21, "bf16": 2.0 ** -15}[dtype] if not long else (0.0 if dtype == "f32" else S.HALF_STEP[dtype])
            relative = 2.0 ** -17 + parts + n / 32 * 2.0 ** -24 + (4 + math.sqrt(n)) * 2.0 ** -23
            bar = want * (relative + S.HALF_STEP[dtype]) + (2.0 ** -35 * total / sums + 2.0 ** -25 if dtype == "f16" else 0)
            assert within(O, np.broadcast_to(want, (1, T, d)), np.broadcast_to(bar, (1, T, d)))
            off = np.abs(host(lse) - (gap + math.log(sums))).max()
            assert off <= n / 32 * 2.0 ** -24 + 2.0 ** -22 * 32, (gap, off)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_up_to_the_last_position(layout):
    """|position| up to 2^52, and angles up to 2^62: the product's error is then hundreds of turns and is reduced too."""
    pi = 314159265358979323846264338327950288419716939937510582097494459230781640628620899      # 10^80 pi
    unit = 10 ** 80
    x = tokens(2, 64, 64, "f32", 5)
    near, _ = sga.rotary_frequencies(64)
    for freqs in (near, near * 1000.0, -near * 3.0):
        for first, step in (((1 << 50) + 12345, 977), ((1 << 51) - 64 * 977, 977), ((1 << 52) - 64 * 977, 977), (1 - (1 << 52), 12345)):
            at = [first + t * step for t in range(64)]
            assert max(map(abs, at)) < 1 << 52
            angle = np.zeros((64, 32))
            for k, f in enumerate(freqs.cpu().tolist()):
                num, den = f.as_integer_ratio()
                angle[:, k] = [float(num * p * unit // den % (2 * pi)) / float(unit) for p in at]
            a, b = (host(x)[..., :32], host(x)[..., 32:]) if layout == "half" else (host(x)[..., ::2], host(x)[..., 1::2])
            u, v = a * np.cos(angle) - b * np.sin(angle), a * np.sin(angle) + b * np.cos(angle)
            size = np.abs(a) + np.abs(b)
            if layout == "half":
                want, size = np.concatenate((u, v), -1), np.concatenate((size, size), -1)
            else:
                want, size = np.stack((u, v), -1).reshape(2, 64, 64), np.stack((size, size), -1).reshape(2, 64, 64)
            got = sga.rotary(x, sga.Rotary(freqs, layout=layout), positions=torch.tensor(at, device="cuda"))
            assert within(got, want, S.rotate_bar(want, size, "f32"))


def test_attention_of_sequences_that_go_back():
    """A seq_ptr that decreases brings more tiles than the call was planned for.  Rows may be wrong then, but no partial state is read from
    behind the workspace: that memory holds NaN here.  (Every sequence of tokens is the same one, so no row is NaN by itself.)"""
    T, d, page, length = 333 * 128, 64, 64, 4096
    g = torch.Generator(device="cuda").manual_seed(1)
    table = torch.arange(length // page, dtype=torch.int32, device="cuda").repeat(5, 1)
    ptr = torch.tensor([0, T, 0, T, 0, T], device="cuda")
    lens = torch.full((5,), length, dtype=torch.int32, device="cuda")
    batch = sga.PagedBatch(table, ptr, lens, T, page, length // page)
    ck, cv = (torch.randn(length // page, 1, page, d, generator=g, device="cuda", dtype=torch.float16) for _ in range(2))
    Q = torch.randn(1, T, d, generator=g, device="cuda", dtype=torch.float16)
    n = sga.paged_workspace_bytes(batch, full(length), 1, 1, d, torch.float16)
    assert n > 0
    # the tokens lie before position 0 but for the last 4,096: a cut tile of theirs is joined from its own records alone
    space = torch.full((n + (64 << 20),), 255, dtype=torch.uint8, device="cuda")
    O, lse = torch.zeros_like(Q), torch.zeros(1, T, device="cuda")
    sga.attention_paged(Q, ck, cv, batch, full(length), 0.125, O=O, lse=lse, workspace=space[:n])
    assert torch.isfinite(O).all() and not torch.isnan(lse).any()
    assert (space[n:] == 255).all()
    sga.cache_append(Q, Q, ck, cv, batch)
    assert torch.isfinite(ck).all() and torch.isfinite(cv).all()


def test_rotary_of_the_most_rows():
    """2^31 - 1 rows, the most that a call takes: the first, the last and some between them."""
    L = (1 << 31) - 1
    x = torch.zeros(1, L, 2, dtype=torch.float16, device="cuda")
    at = torch.tensor([0, 1, 4095, (1 << 22) + 3, (1 << 30) + 5, L - 4, L - 1], device="cuda")
    x[0, at] = torch.arange(1, 15, device="cuda").view(7, 2).half()
    rot = sga.Rotary(torch.full((1,), 0.37, dtype=torch.float64, device="cuda"))
    want, size = S.rotate(host(x[:, at]), at.cpu().numpy() - 7, np.array([0.37]))
    assert sga.rotary(x, rot, first=-7, out=x) is x
    assert within(x[:, at], want, S.rotate_bar(want, size, "f16"))
    assert int(torch.count_nonzero(x[0, :, 0])) <= 7


def test_append_of_the_most_sequences():
    """2^31 - 1 sequences, the most that a batch may have, all but three without new tokens; attention refuses as many."""
    S_, d, page = (1 << 31) - 1, 32, 16
    who = [5, (1 << 30) + 77, S_ - 1]
    table = torch.full((S_, 1), -1, dtype=torch.int32, device="cuda")
    ptr, lens = torch.zeros(S_ + 1, dtype=torch.int64, device="cuda"), torch.zeros(S_, dtype=torch.int32, device="cuda")
    for i, s in enumerate(who):
        table[s, 0] = 2 - i
        ptr[s + 1:] += 1
        lens[s] = 3 + i
    batch = sga.PagedBatch(table, ptr, lens, 3, page, 3)
    ck, cv = caches(3, 1, page, d, "f16", 1)
    before = [ck.clone(), cv.clone()]
    K, V = tokens(1, 3, d, "f16", 2), tokens(1, 3, d, "f16", 3)
    sga.cache_append(K, V, ck, cv, batch)
    for i in range(3):
        before[0][2 - i, :, 2 + i], before[1][2 - i, :, 2 + i] = K[:, i], V[:, i]
    assert torch.equal(ck, before[0]) and torch.equal(cv, before[1])
    with pytest.raises(sga.SgaError):
        sga.attention_paged(K, ck, cv, batch, full(16), 0.1)


# ---- which kernel takes a call, and calls of many sequences -----------------------------------------
def kernel_of(dtype, T, n_seqs, group, d, spec, causal, most):
    """Rows of keys of 128 to 512 bytes and more than 32 rows per sequence on average (full precision 96, 64 at d = 128, 32 up to d = 64 where a
    sequence has 256 tokens at most) take tiles of 128 rows, unless full precision at d = 64 meets a window of 256 keys or fewer."""
    row = d * (4 if dtype == "f32" else 2)
    narrow = dtype == "f32" and d == 64 and (1 if causal else 2) * spec.window <= 256
    rows = 32 if dtype != "f32" or (d <= 64 and min(spec.L, most) <= 256) else 64 if d > 64 else 96
    return "paged_chunk_kernel" if 128 <= row <= 512 and not narrow and T * group > rows * n_seqs else "paged_kernel"


def attend_on_device(Q, ck, cv, table, new, length, spec, scale, causal, dtype, once):
    """serving_oracle.attend for whole sequences at a time, in 64 bits on the device: (O, lse, bar of O, bar of lse) of the real rows."""
    page, Hkv, d = ck.shape[2], ck.shape[1], ck.shape[3]
    G, parts = Q.shape[0] // Hkv, {"f32": 0.0, "f16": 2.0 ** -21, "bf16": 2.0 ** -15}[dtype] if not once else S.HALF_STEP[dtype]
    out = [[], [], [], []]
    row = 0
    for s, (n, L) in enumerate(zip(new, length)):
        if n == 0:
            continue
        at = torch.arange(L, device="cuda")
        where = torch.from_numpy(table[s].astype(np.int64)).cuda()[at // page]
        k, v = (c[where, :, at % page].double().transpose(0, 1).unsqueeze(1) for c in (ck, cv))              # [Hkv, 1, L, d]
        q = Q[:, row:row + n].double().reshape(Hkv, G, n, d)
        i, j = torch.arange(L - n, L, device="cuda")[:, None], at[None]
        see = (i - j).abs() <= spec.window
        if spec.kind == KIND_GLOBAL_LOCAL:
            see |= (j < spec.n_global) | (i < spec.n_global)
        see &= (i < spec.L) & (j < spec.L)
        if causal:
            see &= j <= i
        z = scale * torch.matmul(q, k.transpose(-1, -2).contiguous())
        size = torch.matmul(q.abs(), k.abs().transpose(-1, -2).contiguous()).masked_fill_(~see, 0.0).amax(-1)
        off = d * 2.0 ** -24 * abs(scale) * size + 2.0 ** -22 * (1 + z.abs().masked_fill_(~see, 0.0).amax(-1))
        z.masked_fill_(~see, -math.inf)
        lse = torch.logsumexp(z, -1)
        w = (z - torch.where(lse.isinf(), 0.0, lse).unsqueeze(-1)).exp()
        O, share = torch.matmul(w, v), torch.matmul(w, v.abs())
        bar = share * (2 * off + parts + (4 + math.sqrt(L)) * 2.0 ** -23).unsqueeze(-1) + O.abs() * S.HALF_STEP[dtype]
        if dtype == "f16":
            bar += 2.0 ** -35 * v.abs().sum(-2, keepdim=True) + 2.0 ** -25        # (the largest numerator of a row is 2^10 or more)
        for x, y in zip(out, (O, lse, bar, 2 * off + 2.0 ** -22 * (1 + lse.abs()))):
            x.append(y.reshape(Hkv * G, n, *y.shape[3:]))
        row += n
    return [host(torch.cat(x, 1)) for x in out]


def check_on_device(dtype, new, length, page, Hq, Hkv, d, spec, causal=True, workspace=True, seed=0):
    print("attend", dtype, len(new), sum(new), max(length), page, Hq, Hkv, d, spec, causal, flush=True)
    batch, table, ptr, lens, n_pages, T = batch_of(new, length, page, seed=seed, padding=1)
    ck, cv = caches(n_pages, Hkv, page, d, dtype, seed + 1)
    Q, scale = tokens(Hq, T, d, dtype, seed + 3), 1 / math.sqrt(d)
    want = kernel_of(dtype, T, len(new), Hq // Hkv, d, spec, causal, table.shape[1] * page)
    ws = sga.alloc_paged_workspace(batch, spec, Hq, Hkv, d, dtype) if workspace else None
    O, lse = torch.full((Hq, T, d), 7.0, dtype=DTYPE[dtype], device="cuda"), torch.full((Hq, T), 7.0, device="cuda")
    assert sga.sga_profile_enable(1) == 0
    sga.attention_paged(Q, ck, cv, batch, spec, scale, causal=causal, O=O, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    kernel = sga.sga_profile_last_kernel()
    sga.sga_profile_enable(0)
    assert kernel == want
    o, l, bar, l_bar = attend_on_device(Q, ck, cv, table, new, length, spec, scale, causal, dtype, want == "paged_chunk_kernel" and dtype != "f32")
    assert within(O[:, :T - 1], o, bar) and within(lse[:, :T - 1], l, l_bar)
    assert (O[:, T - 1:] == 7).all() and (lse[:, T - 1:] == 7).all()
    return kernel


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,window,new,kernel", [
    (32, 1 << 20, 96, "paged_kernel"), (32, 1 << 20, 97, "paged_chunk_kernel"), (64, 1 << 20, 96, "paged_kernel"),
    (64, 1 << 20, 97, "paged_chunk_kernel"), (128, 1 << 20, 64, "paged_kernel"), (128, 1 << 20, 65, "paged_chunk_kernel"),
    (128, 100, 200, "paged_chunk_kernel"), (256, 1 << 20, 200, "paged_kernel"), (64, 257, 200, "paged_chunk_kernel"),
    (64, 128, 200, "paged_kernel"), (32, 20, 200, "paged_chunk_kernel"),
])
def test_attention_kernels_of_full_precision(d, window, new, kernel, causal):
    for page in (16, 24):
        spec = MaskSpec(KIND_SLIDING, 1300, window=window)
        # (padding counts: the one row of it is left out of the sequences' tokens)
        assert check_on_device("f32", [2 * new - 1 - new // 2, new // 2], [1300, 900], page, 2, 2, d, spec, causal) == kernel
    for length, short in ((256, "paged_chunk_kernel"), (257, "paged_kernel")):
        if d <= 64 and new <= 97:
            assert check_on_device("f32", [40, 50], [length, 60], 1, 2, 2, d, full(1300), causal) == short


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_attention_of_single_tokens_beside_prompts(dtype):
    """What a server sends at once: many single tokens and a prompt.  The kernel goes by the average."""
    rng = np.random.default_rng(1)
    behind = [int(x) for x in rng.integers(1, 900, 300)]
    for n, prompt, kernel in ((300, 4096, "paged_kernel"), (30, 4096, "paged_chunk_kernel")):
        new, length = [1] * n, behind[:n]
        new.insert(n // 3, prompt)
        length.insert(n // 3, prompt + 500)
        for spec in (full(5000), MaskSpec(KIND_GLOBAL_LOCAL, 5000, window=600, n_global=20)):
            assert check_on_device(dtype, new, length, 16, 2, 2, 64, spec) == kernel
    assert check_on_device(dtype, new, length, 24, 8, 2, 128, full(5000), workspace=False) == "paged_chunk_kernel"


@pytest.mark.parametrize("dtype,d", [("f16", 64), ("bf16", 128), ("f32", 64)])
def test_attention_of_thousands_of_sequences(dtype, d):
    rng = np.random.default_rng(2)
    length = [int(x) for x in rng.integers(1, 60, 3000)]
    length[17], length[2999] = 4000, 3000
    for n in (700, 3000):
        check_on_device(dtype, [1] * n, length[-n:], 16, 2, 1, d, full(4000))
    new = [int(x) for x in rng.integers(0, 90 if dtype != "f32" else 250, 150)]           # long chunks of more sequences than a wavefront looks at at a time, in pieces
    length = [a + int(b) for a, b in zip(new, rng.integers(0, 3000, 150))]
    assert check_on_device(dtype, new, length, 16, 1, 1, d, full(4000)) == "paged_chunk_kernel"
    assert check_on_device(dtype, new, length, 5, 1, 1, d, MaskSpec(KIND_GLOBAL_LOCAL, 4000, window=1500, n_global=9), causal=False) \
        == "paged_chunk_kernel"


@pytest.mark.parametrize("page", [64, 24])
@pytest.mark.parametrize("new", [1, 9, 150])
def test_attention_far_pages_of_every_kernel(new, page):
    """Offsets of more than 2^31 elements: single tokens, drafts and long chunks, pages of whole 16-key tiles and others."""
    Hkv, d, length = 8, 128, 150
    n_pages, columns = (1 << 31) // (page * Hkv * d) + 40, -(-length // page)
    ck, cv = (torch.empty(n_pages, Hkv, page, d, dtype=torch.float16, device="cuda") for _ in range(2))
    table = np.array([[n_pages - 1 - 2 * c if c % 2 == 0 else c for c in range(columns)]], dtype=np.int32)
    assert int(table[0, 0]) * page * Hkv * d > 1 << 31
    K, V, Q = (tokens(h, length, d, "f16", s) for h, s in ((Hkv, 1), (Hkv, 2), (16, 3)))
    dev = [torch.from_numpy(x).cuda() for x in (table, np.array([0, length]), np.array([length], dtype=np.int32))]
    sga.cache_append(K, V, ck, cv, sga.PagedBatch(*dev, length, page, n_pages))
    for t in range(length):
        assert torch.equal(ck[int(table[0, t // page]), :, t % page], K[:, t]) and torch.equal(cv[int(table[0, t // page]), :, t % page], V[:, t])
    dev[1] = torch.tensor([0, new], device="cuda")
    batch = sga.PagedBatch(*dev, new, page, n_pages)
    at = torch.from_numpy(table[0].astype(np.int64)).cuda()
    small = [c[at] for c in (ck, cv)]
    spec = MaskSpec(KIND_GLOBAL_LOCAL, length, window=100, n_global=3)
    want, lse, bar, lse_bar = S.attend(host(Q[:, :new]), host(small[0]), host(small[1]), np.arange(columns)[None], np.array([0, new]),
                                       np.array([length]), spec, 0.1, True, "f16", new * 2 > 32)
    got = sga.attention_paged(Q[:, :new], ck, cv, batch, spec, 0.1, want_lse=True)
    assert within(got[0], want, bar) and within(got[1], lse, lse_bar)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("new", [1, 20, 100])
def test_attention_of_huge_scores(dtype, new):
    """Scores so large that a step of theirs is more than what numerators are raised by: the tokens that share the largest one have the
    mean of their values as O, the others nothing."""
    n, d, page = 300, 64, 16
    batch, table, ptr, lens, n_pages, T = batch_of([new], [n], page)
    ck, cv = caches(n_pages, 1, page, d, dtype, 3)
    ck.zero_()
    at = torch.from_numpy(table[0].astype(np.int64)).cuda()
    seen = np.arange(n) % 3 == 1
    for t in np.nonzero(seen)[0]:
        ck[at[t // page], 0, t % page, 0] = 1
    v = host(cv[at, 0].reshape(-1, d)[:n])[seen]
    Q = torch.zeros(1, T, d, dtype=DTYPE[dtype], device="cuda")
    Q[..., 0] = 1
    long = kernel_of(dtype, T, 1, 1, d, full(n), False, n_pages * page) == "paged_chunk_kernel"
    parts = {"f32": 0.0, "f16": 2.0 ** -21, "bf16": 2.0 ** -15}[dtype] if not long else (0.0 if dtype == "f32" else S.HALF_STEP[dtype])
    for scale in [2.0 ** k * m for k in (10, 20, 22, 23, 24, 25, 26, 27, 28, 29, 30, 40) for m in (1.0, 1.4)]:
        print("huge scores", dtype, new, scale, flush=True)
        O, lse = sga.attention_paged(Q, ck, cv, batch, full(n), scale, causal=False, want_lse=True)
        bar = np.abs(v.mean(0)) * S.HALF_STEP[dtype] + np.abs(v).mean(0) * (parts + 16 * 2.0 ** -23) + 2.0 ** -25
        assert within(O, np.broadcast_to(v.mean(0), (1, T, d)), np.broadcast_to(bar, (1, T, d)))
        assert within(lse, np.full((1, T), scale + math.log(seen.sum())), np.full((1, T), 2.0 ** -21 * scale))
