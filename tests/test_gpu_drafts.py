"""Generation with drafted tokens against definitions in 64 bits: the next step's pages, norms of queries and keys with the rotation and their
gradient, trees of drafts, attention over them, accepted tokens moved into place, and a run of them together."""
import math

import numpy as np
import pytest
import torch

import drafts_oracle as D
import paper_2502_01659_amd as sga
import serving_oracle as S
from sga_inputs import MaskSpec, KIND_GLOBAL_LOCAL, KIND_SLIDING
from test_gpu_serving import DTYPE, batch_of, caches, full, host, long_chunks, tokens, within

pytestmark = pytest.mark.gpu


# ---- pages ------------------------------------------------------------------------------------------
def pages_case(rng, n_seqs, columns, page, kept, fill):
    """Sequences of random lengths with their pages, some columns without one, a ring that begins anywhere."""
    length = rng.integers(0, columns * page + 1, n_seqs)
    n_pages = max(1, int(sum(-(-length // page)) * fill) + 5)
    order = list(rng.permutation(n_pages))
    table = np.full((n_seqs, columns), -1, dtype=np.int32)
    rows = np.zeros(n_seqs, dtype=np.int64)
    for s in range(n_seqs):
        while -(-length[s] // page) > len(order):
            length[s] //= 2
        for c in range(-(-length[s] // page)):
            table[s, c] = order.pop() if rng.random() < 0.95 else (-1 if rng.random() < 0.7 else n_pages + 3)
        if kept:
            rows[s] = rng.integers(0, min(length[s], 9) + 1)
    ring = np.full(n_pages, -1, dtype=np.int32)
    first = int(rng.integers(0, n_pages))
    for i, p in enumerate(order):
        ring[(first + i) % n_pages] = p
    return table, np.concatenate(([0], rows.cumsum())), length.astype(np.int32), ring, np.array([first, len(order)]), n_pages


def run_pages(table, ptr, length, ring, state, ask, kept, T, page, n_pages, spec, in_place, maps=True):
    dev = lambda x, t: torch.from_numpy(np.ascontiguousarray(x)).to(t).cuda()
    batch = sga.PagedBatch(dev(table, torch.int32), dev(ptr, torch.int64), dev(length, torch.int32), T, page, n_pages)
    pool = sga.PagePool(dev(ring, torch.int32), dev(state, torch.int64))
    out, to, to_pool = None, batch, pool
    if not in_place:
        to = sga.PagedBatch(torch.full_like(batch.page_table, 77), torch.full_like(batch.seq_ptr, 77), torch.full_like(batch.seq_len, 77), T, page, n_pages)
        to_pool = sga.PagePool(pool.pages, torch.full_like(pool.state, 77))
        out = (to, to_pool)
    positions, slots = (torch.full((T,), -7, dtype=torch.int64, device="cuda") if maps else None for _ in range(2))
    got = sga.pages_advance(batch, pool, dev(ask, torch.int32), kept=dev(kept, torch.int32) if kept is not None else None, spec=spec,
                            positions=positions, slots=slots, out=out)
    assert got is to
    if not in_place:
        assert np.array_equal(batch.page_table.cpu().numpy(), table) and np.array_equal(batch.seq_len.cpu().numpy(), length)
        assert pool.state.tolist() == list(state)
    return to, to_pool, positions, slots


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n_seqs,columns,page,kept,spec,most", [
    (1, 1, 1, False, None, 3), (1, 700, 16, True, None, 2000), (7, 20, 16, True, MaskSpec(KIND_SLIDING, 64, window=40), 30),
    (64, 130, 16, True, MaskSpec(KIND_GLOBAL_LOCAL, 4000, window=300, n_global=33), 200), (300, 9, 5, False, None, 12),
    (1500, 64, 3, True, MaskSpec(KIND_SLIDING, 64, window=0), 5), (5000, 3, 8, True, None, 4), (3, 5000, 1, False, MaskSpec(KIND_SLIDING, 9, window=99), 900),
    (260, 100, 7, True, MaskSpec(KIND_GLOBAL_LOCAL, 9, window=7, n_global=9), 60), (65536, 2, 16, True, None, 9),
])
def test_pages(n_seqs, columns, page, kept, spec, most, in_place):
    rng = np.random.default_rng(n_seqs + columns)
    for fill, room in ((1.6, 1.2), (1.05, 0.6), (2.5, 0.0)):
        print("pages", n_seqs, columns, page, kept, spec, most, in_place, fill, flush=True)
        table, ptr, length, ring, state, n_pages = pages_case(rng, n_seqs, columns, page, kept, fill)
        ask = rng.integers(0, most + 1, n_seqs)
        ask[rng.random(n_seqs) < 0.1] = -1
        ask[rng.random(n_seqs) < 0.03] = columns * page + 1                   # more than a row of the table holds
        stay = rng.integers(-1, 11, n_seqs) if kept else None                 # (beyond 0 .. rows too)
        T = int(room * np.maximum(ask[ask <= columns * page], 0).sum())
        want = D.advance(table, ptr, length, ring, state, ask, stay, T, page, n_pages, spec)
        to, pool, positions, slots = run_pages(table, ptr, length, ring, state, ask, stay, T, page, n_pages, spec, in_place)
        assert np.array_equal(to.page_table.cpu().numpy(), want[0])
        assert np.array_equal(to.seq_ptr.cpu().numpy(), want[1]) and np.array_equal(to.seq_len.cpu().numpy(), want[2])
        assert np.array_equal(pool.pages.cpu().numpy(), want[3]) and pool.state.tolist() == want[4].tolist()
        end = int(want[1][-1])
        assert positions[:end].tolist() == want[5][:end] and slots[:end].tolist() == want[6][:end]
        assert (positions[end:] == -7).all() and (slots[end:] == -7).all()    # rows of no sequence are left as they were


def test_pages_of_nothing_and_of_bad_records():
    """No sequence; states out of range; a page that stands in two tables does not fill the ring beyond its size."""
    to, pool, *_ = run_pages(np.zeros((0, 4), dtype=np.int32), np.array([5]), np.zeros(0, dtype=np.int32), np.arange(6, dtype=np.int32), np.array([-1, 99]),
                             np.zeros(0), None, 3, 16, 6, None, False)
    assert to.seq_ptr.tolist() == [0] and pool.state.tolist() == [5, 6]
    for state in ([-3, 4], [17, 99], [5, -2]):
        table = np.array([[0, 1, -1], [1, 2, 3]], dtype=np.int32)
        args = (table, np.array([0, 0, 0]), np.array([30, 40], dtype=np.int32), np.arange(8, dtype=np.int32), np.array(state), np.array([-1, -1]), None, 4, 16, 8, None)
        want = D.advance(*args)
        to, pool, *_ = run_pages(*args, True, maps=False)
        assert np.array_equal(pool.pages.cpu().numpy(), want[3]) and pool.state.tolist() == want[4].tolist()


@pytest.mark.parametrize("asks,granted", [
    ([2 * 10 ** 9, 2 * 10 ** 9], 1), ([1 << 30, (1 << 30) - 1], 2), ([1 << 30, 1 << 30, 1], 1), ([1 << 30] * 4 + [5, 1 << 30], 1),
    ([(1 << 31) - 65536, 65535, 1], 2), ([7] + [2 * 10 ** 9] * 299, 2), ([1 << 30] * 130 + [1], 1),
])
def test_pages_of_requests_beyond_every_number(asks, granted):
    """As many rows as a batch may have, 2^31 - 1, and requests whose sum passes that, 2^32 and 2^33: those that fit are granted, the one that fills
    the rows to the last among them, and none behind the first that does not."""
    print("pages beyond", len(asks), asks[:4], flush=True)
    page, T = 65536, (1 << 31) - 1
    needs = [-(-a // page) for a in asks]
    columns, n_pages = min(max(needs), 32767), max(sum(needs), 5)
    table = torch.full((len(asks), columns), -1, dtype=torch.int32, device="cuda")
    batch = sga.PagedBatch(table, torch.zeros(len(asks) + 1, dtype=torch.int64, device="cuda"), torch.zeros(len(asks), dtype=torch.int32, device="cuda"),
                           T, page, n_pages)
    pool = sga.PagePool.full(n_pages)
    sga.pages_advance(batch, pool, torch.tensor(asks, dtype=torch.int32, device="cuda"))
    rows = [a if i < granted else 0 for i, a in enumerate(asks)]
    assert batch.seq_len.tolist() == rows and batch.seq_ptr.tolist() == [0] + np.cumsum(rows).tolist()
    taken = 0
    for i, n in enumerate(needs):
        n = n if i < granted else 0
        assert table[i, :n].tolist() == list(range(taken, taken + n)) and (table[i, n:] == -1).all()
        taken += n
    assert pool.state.tolist() == [taken % n_pages, n_pages - taken]


def test_pages_over_many_steps_captured():
    """A captured call, in place: pages are neither lost nor given twice, and every replay is the oracle's step."""
    rng = np.random.default_rng(5)
    S_, C, page, n_pages, T = 40, 30, 4, 500, 300
    spec = MaskSpec(KIND_GLOBAL_LOCAL, 1 << 20, window=30, n_global=5)
    batch = sga.PagedBatch(torch.full((S_, C), -1, dtype=torch.int32, device="cuda"), torch.zeros(S_ + 1, dtype=torch.int64, device="cuda"),
                           torch.zeros(S_, dtype=torch.int32, device="cuda"), T, page, n_pages)
    pool = sga.PagePool.full(n_pages)
    ask, kept = (torch.zeros(S_, dtype=torch.int32, device="cuda") for _ in range(2))
    positions, slots = (torch.zeros(T, dtype=torch.int64, device="cuda") for _ in range(2))
    ws = sga.alloc_pages_workspace(batch)
    call = lambda: sga.pages_advance(batch, pool, ask, kept=kept, spec=spec, positions=positions, slots=slots, workspace=ws)
    call()                                                    # (asks for nothing)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for step in range(60):
        before = [x.cpu().numpy().copy() for x in (batch.page_table, batch.seq_ptr, batch.seq_len, pool.pages, pool.state)]
        a = rng.integers(0, 13, S_)
        a[rng.random(S_) < 0.05] = -1
        k = rng.integers(0, 14, S_)
        ask.copy_(torch.from_numpy(a))
        kept.copy_(torch.from_numpy(k))
        graph.replay()
        torch.cuda.synchronize()
        want = D.advance(*before, a, k, T, page, n_pages, spec)
        got = [x.cpu().numpy() for x in (batch.page_table, batch.seq_ptr, batch.seq_len, pool.pages, pool.state)]
        assert all(np.array_equal(x, y) for x, y in zip(got, want)), step
        first, count = got[4]
        everywhere = np.concatenate((got[0][got[0] >= 0], got[3][(first + np.arange(count)) % n_pages]))
        assert np.array_equal(np.sort(everywhere), np.arange(n_pages))


# ---- norms ------------------------------------------------------------------------------------------
def weights_of(kind, d, dtype, offset, seed):
    if kind == "none":
        return None
    w = 1 - offset + 0.3 * torch.randn(d, generator=torch.Generator().manual_seed(seed))
    return w.to(DTYPE[dtype] if kind == "same" else DTYPE[kind]).cuda()


SHAPES = [
    # Hq, Hkv, T, d, channels, memory
    (1, 1, 1, 64, 64, "head"), (32, 8, 1, 128, 128, "token"), (4, 2, 65, 128, 64, "token"), (8, 1, 257, 64, 32, "head"), (5, 5, 33, 256, 256, "slice"),
    (2, 1, 9, 32, 16, "token"), (4, 3, 31, 80, 20, "token"), (4, 3, 31, 80, 80, "token"), (3, 2, 17, 7, 6, "head"), (2, 2, 700, 64, 64, "token"),
    (7, 1, 13, 96, 32, "slice"), (2, 1, 5, 1024, 1024, "head"), (1, 2, 6, 512, 64, "token"), (3, 1, 4, 2, 2, "head"), (2, 1, 3, 8, 4, "head"),
]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("Hq,Hkv,T,d,channels,memory", SHAPES)
def test_norm_rotary(dtype, layout, Hq, Hkv, T, d, channels, memory):
    freqs, _ = sga.rotary_frequencies(channels)
    rot, f = sga.Rotary(freqs, layout=layout, magnitude=1.25), freqs.cpu().numpy()
    Q, K = tokens(Hq, T, d, dtype, T + d, memory), tokens(Hkv, T, d, dtype, T + d + 1, memory)
    K[:, T // 2] *= 100
    for kind, offset, epsilon, positions, first in (("same", 0.0, 1e-6, None, 131071), ("f32", 1.0, 0.5, torch.arange(T).cuda() * 7 - 3, 0),
                                                    ("none", 3.0, 1e-5, None, -2)):
        print("norm", dtype, layout, Hq, Hkv, T, d, channels, memory, kind, flush=True)
        wq, wk = weights_of(kind, d, dtype, offset, 1), weights_of("bf16" if kind == "f32" else kind, d, dtype, offset, 2)
        at = positions.cpu().numpy() if positions is not None else first + np.arange(T)
        norms = sga.Norm(wq, epsilon, offset), sga.Norm(wk, epsilon, offset)
        out = sga.norm_rotary(Q, K, rotary=rot, q_norm=norms[0], k_norm=norms[1], positions=positions, first=first)
        for x, w, got in ((Q, wq, out[0]), (K, wk, out[1])):
            y, size = D.norm_rotate(host(x), at, f, layout, 1.25, host(w) if w is not None else None, epsilon, offset)
            assert within(got, y, D.norm_bar(y, size, dtype))
        # alone, in place, and one of the two only
        mine = Q.clone() if memory != "slice" else tokens(Hq, T, d, dtype, T + d, memory)
        assert sga.norm_rotary(mine, rotary=rot, q_norm=norms[0], positions=positions, first=first, Q_out=mine) is mine
        assert torch.equal(mine, out[0])
        half = sga.norm_rotary(Q, K, rotary=rot, k_norm=norms[1], positions=positions, first=first)
        assert torch.equal(half[1], out[1])
        y, size = S.rotate(host(Q), at, f, layout, 1.25)
        assert within(half[0], y, D.norm_bar(y, size, dtype))
        # no rotation
        y, size = D.norm_rotate(host(Q), at, None, layout, 1.0, host(wq) if wq is not None else None, epsilon, offset)
        assert within(sga.norm_rotary(Q, q_norm=norms[0]), y, D.norm_bar(y, size, dtype))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d", [64, 6])
def test_norm_rotary_of_the_farthest_positions(d, layout):
    """Positions are any 64-bit numbers, the lowest among them: in rows in lanes and one pair a lane, forward and back."""
    print("farthest", d, layout, flush=True)
    f = 1e-9 * 0.7 ** np.arange(d // 2)                       # (angles below 10^10: extended precision holds them to 2^-30)
    rot, n = sga.Rotary(torch.from_numpy(f).cuda(), layout=layout), sga.Norm()
    at = np.array([-2 ** 63, 5, -2 ** 63 + 1, 2 ** 63 - 1, -2 ** 63])
    Q, G = tokens(3, 5, d, "f32", 1), tokens(3, 5, d, "f32", 2)
    where = torch.from_numpy(at).cuda()
    y, size = D.norm_rotate(host(Q), at, f, layout, 1.0, None, 1e-6, 0.0)
    got = sga.norm_rotary(Q, rotary=rot, q_norm=n, positions=where)
    assert within(got, y, D.norm_bar(y, size, "f32"))
    dx, _ = sga.norm_rotary_backward(Q, G, rotary=rot, q_norm=n, positions=where)
    want, _, size, _ = D.norm_gradient(host(Q), host(G), at, f, layout, 1.0, None, 1e-6, 0.0)
    assert within(dx, want, D.gradient_bar(want, size, "f32"))
    first = sga.norm_rotary(Q[:, :1].contiguous(), rotary=rot, q_norm=n, first=-2 ** 63)
    assert torch.equal(first, got[:, :1])


@pytest.mark.parametrize("dtype,d,channels", [("bf16", 128, 64), ("f32", 10, 4)])
def test_norms_of_packed_and_of_broadcast_rows(dtype, d, channels):
    """Queries and keys that are slices of one projection, in place, values beside them untouched; one row that stands for all heads, and one for all
    tokens, forward and back."""
    rot, n = sga.Rotary(sga.rotary_frequencies(channels)[0]), sga.Norm(weights_of("f32", d, dtype, 0.0, 1))
    packed = tokens(1, 50, 8 * d, dtype, 1, "head").view(50, 8, d)
    Q, K, before = packed[:, :4].transpose(0, 1), packed[:, 4:6].transpose(0, 1), packed.clone()
    want = sga.norm_rotary(Q.clone(), K.clone(), rotary=rot, q_norm=n, k_norm=n, first=3)
    got = sga.norm_rotary(Q, K, rotary=rot, q_norm=n, k_norm=n, first=3, Q_out=Q, K_out=K)
    assert got[0] is Q and torch.equal(Q, want[0]) and torch.equal(K, want[1]) and torch.equal(packed[:, 6:], before[:, 6:])
    grads = tokens(1, 50, 8 * d, dtype, 2, "head").view(50, 8, d)
    G, GK, before = grads[:, :4].transpose(0, 1), grads[:, 4:6].transpose(0, 1), grads.clone()
    a = sga.norm_rotary_backward(Q, G.clone(), K, GK.clone(), rotary=rot, q_norm=n, k_norm=n, first=3)
    b = sga.norm_rotary_backward(Q, G, K, GK, rotary=rot, q_norm=n, k_norm=n, first=3, dQ=G, dK=GK)
    assert all(torch.equal(x, y) for x, y in zip(a, b)) and torch.equal(grads[:, 6:], before[:, 6:])
    for one in (tokens(1, 50, d, dtype, 3).expand(4, 50, d), tokens(4, 1, d, dtype, 3).expand(4, 50, d)):
        whole, g = one.contiguous(), tokens(4, 50, d, dtype, 4)
        assert torch.equal(sga.norm_rotary(one, rotary=rot, q_norm=n), sga.norm_rotary(whole, rotary=rot, q_norm=n))
        for x, y in ((one, g), (whole, one)):                 # (a gradient may be broadcast too)
            a, b = (sga.norm_rotary_backward(*z, rotary=rot, q_norm=n) for z in ((x, y), (x.contiguous(), y.contiguous())))
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("d,channels", [(128, 128), (7, 6)])
def test_norms_of_rows_with_infinities(d, channels):
    """A row that holds an infinity or a NaN says nothing about the others, in rows in lanes and one pair a lane."""
    rot, n = sga.Rotary(sga.rotary_frequencies(channels)[0]), sga.Norm(weights_of("f32", d, "f32", 0.0, 1))
    Q, G = tokens(3, 20, d, "f32", 1), tokens(3, 20, d, "f32", 2)
    y, dx = sga.norm_rotary(Q, rotary=rot, q_norm=n), sga.norm_rotary_backward(Q, G, rotary=rot, q_norm=n)[0]
    Q[1, 4, 2], Q[0, 19, 0], Q[2, 0, d - 1] = float("inf"), float("nan"), -float("inf")
    good = torch.ones(3, 20, dtype=torch.bool, device="cuda")
    good[1, 4] = good[0, 19] = good[2, 0] = False
    y2, dx2 = sga.norm_rotary(Q, rotary=rot, q_norm=n), sga.norm_rotary_backward(Q, G, rotary=rot, q_norm=n)[0]
    assert torch.equal(y[good], y2[good]) and torch.equal(dx[good], dx2[good])
    assert y2[~good].isnan().any(-1).all() and dx2[~good].isnan().any(-1).all()


def test_norm_of_rows_of_zeros_and_of_no_rows():
    x = torch.zeros(2, 3, 64, device="cuda")
    x[1, 1] = 1e-30
    got = sga.norm_rotary(x, q_norm=sga.Norm(epsilon=1e-12))
    y, size = D.norm_rotate(host(x), None, None, None, 1.0, None, 1e-12, 0.0)
    assert within(got, y, D.norm_bar(y, size, "f32"))
    e = torch.empty(4, 0, 64, dtype=torch.float16, device="cuda")
    w = torch.ones(64, device="cuda")
    assert sga.norm_rotary(e, q_norm=sga.Norm(w)).shape == (4, 0, 64)
    dx, dw = sga.norm_rotary_backward(e, e, q_norm=sga.Norm(w))
    assert dx.shape == (4, 0, 64) and (dw == 0).all()         # of no rows: nothing, not what memory held


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("Hq,Hkv,T,d,channels,memory", SHAPES)
def test_norm_gradient(dtype, layout, Hq, Hkv, T, d, channels, memory):
    freqs, _ = sga.rotary_frequencies(channels)
    rot, f = sga.Rotary(freqs, layout=layout, magnitude=0.8), freqs.cpu().numpy()
    Q, K, G, GK = (tokens(H, T, d, dtype, T + d + i, m) for i, (H, m) in enumerate(((Hq, memory), (Hkv, memory), (Hq, "token"), (Hkv, "head"))))
    for kind, offset, epsilon, r in (("same", 0.0, 1e-6, rot), ("f32", 1.0, 0.5, rot), ("none", 0.0, 1e-5, rot), ("f32", 0.0, 1e-6, None)):
        print("gradient", dtype, layout, Hq, Hkv, T, d, channels, memory, kind, r is None, flush=True)
        wq, wk = weights_of(kind, d, dtype, offset, 1), weights_of("f16" if kind == "f32" else kind, d, dtype, offset, 2)
        at = 900 + np.arange(T)
        qn, kn = sga.Norm(wq, epsilon, offset), sga.Norm(wk, epsilon, offset)
        dQ, dwq, dK, dwk = sga.norm_rotary_backward(Q, G, K, GK, rotary=r, q_norm=qn, k_norm=kn, first=900)
        for x, g, w, dx, dw in ((Q, G, wq, dQ, dwq), (K, GK, wk, dK, dwk)):
            want, want_w, size, w_size = D.norm_gradient(host(x), host(g), at, f if r is not None else None, layout, 0.8, host(w) if w is not None else None,
                                                         epsilon, offset)
            assert within(dx, want, D.gradient_bar(want, size, dtype))
            if w is None:
                assert dw is None
            else:
                assert dw.dtype == torch.float32 and within(dw, want_w, D.weight_bar(w_size))
        # the same bits again, alone, and in the place of the results' gradient
        mine = G.clone()
        again = sga.norm_rotary_backward(Q, mine, rotary=r, q_norm=qn, first=900, dQ=mine)
        assert again[0] is mine and torch.equal(mine, dQ)
    # without a norm the gradient is the rotation back
    got = sga.norm_rotary_backward(Q, G, K, GK, rotary=rot, k_norm=sga.Norm(wk, 1e-6, 0.0), first=900)
    want, _, size, _ = D.norm_gradient(host(Q), host(G), at, f, layout, 0.8, None, 1e-6, 0.0, normed=False)
    assert got[1] is None and within(got[0], want, D.gradient_bar(want, size, dtype))


# Calls whose workgroups and wavefronts take many tokens, one behind the other, with a remainder.  A lane adds at most 36 rows' terms of a weight's gradient in
# these (rows of one pair a lane: up to 16 tokens' heads over four wavefronts, up to four times; rows in lanes: up to eight tokens, four rounds of heads
# each), a wavefront and a workgroup up to 20 of its lanes' and wavefronts' sums in six steps: below the 72 half steps of weight_bar.
@pytest.mark.parametrize("dtype,Hq,Hkv,T,d,channels,memory,layout", [
    # one pair a lane: wide rows, of whose turns a workgroup holds fewer, odd sizes, several rounds
    ("f32", 2, 1, 4097, 1024, 1024, "token", "half"), ("bf16", 4, 1, 4100, 1000, 1000, "head", "interleaved"), ("f16", 3, 2, 4099, 7, 6, "token", "half"),
    ("f32", 3, 2, 40003, 7, 6, "head", "interleaved"), ("bf16", 3, 2, 4099, 80, 20, "token", "interleaved"), ("f16", 16, 1, 4101, 80, 20, "slice", "half"),
    # rows in lanes: one token and several a wavefront
    ("f16", 16, 2, 4099, 80, 80, "token", "half"), ("bf16", 8, 2, 16411, 64, 64, "token", "half"), ("f16", 32, 8, 9001, 128, 128, "token", "interleaved"),
    ("f32", 5, 5, 20011, 64, 32, "head", "half"),
])
def test_norms_of_many_tokens(dtype, Hq, Hkv, T, d, channels, memory, layout):
    print("many tokens", dtype, Hq, Hkv, T, d, channels, memory, layout, flush=True)
    freqs, _ = sga.rotary_frequencies(channels)
    rot, f = sga.Rotary(freqs, layout=layout, magnitude=0.9), freqs.cpu().numpy()
    Q, K, G, GK = (tokens(H, T, d, dtype, T + i, m) for i, (H, m) in enumerate(((Hq, memory), (Hkv, memory), (Hq, "token"), (Hkv, "head"))))
    wq, wk = weights_of("same", d, dtype, 0.0, 1), weights_of("f32", d, dtype, 1.0, 2)
    qn, kn = sga.Norm(wq), sga.Norm(wk, 0.25, 1.0)
    at = np.random.default_rng(d).integers(0, 1 << 20, T)
    where = torch.from_numpy(at).cuda()
    out = sga.norm_rotary(Q, K, rotary=rot, q_norm=qn, k_norm=kn, positions=where)
    grads = sga.norm_rotary_backward(Q, G, K, GK, rotary=rot, q_norm=qn, k_norm=kn, positions=where)
    for x, g, w, (epsilon, offset), y, dx, dw in ((Q, G, wq, (1e-6, 0.0), out[0], *grads[:2]), (K, GK, wk, (0.25, 1.0), out[1], *grads[2:])):
        want, size = D.norm_rotate(host(x), at, f, layout, 0.9, host(w), epsilon, offset)
        assert within(y, want, D.norm_bar(want, size, dtype))
        want, want_w, size, w_size = D.norm_gradient(host(x), host(g), at, f, layout, 0.9, host(w), epsilon, offset)
        assert within(dx, want, D.gradient_bar(want, size, dtype)) and within(dw, want_w, D.weight_bar(w_size))


def test_norms_of_far_rows():
    """Offsets of more than 2^32 elements, forward and back, in place."""
    L, d = (1 << 27) + 5, 32
    x = torch.zeros(1, L, d, dtype=torch.float16, device="cuda")
    g = torch.zeros_like(x)
    at = torch.tensor([0, 1, (1 << 26) + 3, (1 << 27) - 1, L - 1], device="cuda")
    x[0, at], g[0, at] = (torch.randn(5, d, generator=torch.Generator().manual_seed(s)).half().cuda() for s in (1, 2))
    w = weights_of("f32", d, "f16", 0.0, 3)
    freqs, _ = sga.rotary_frequencies(d)
    rot, n, f = sga.Rotary(freqs), sga.Norm(w), freqs.cpu().numpy()
    few_x, few_g, where = host(x[:, at]), host(g[:, at]), at.cpu().numpy() + 7
    dx, dw = sga.norm_rotary_backward(x, g, rotary=rot, q_norm=n, first=7, dQ=g)
    want, want_w, size, w_size = D.norm_gradient(few_x, few_g, where, f, "half", 1.0, host(w), 1e-6, 0.0)
    assert dx is g and within(g[:, at], want, D.gradient_bar(want, size, "f16")) and within(dw, want_w, D.weight_bar(w_size))
    assert int(torch.count_nonzero(g[0, :, 0])) <= 5
    assert sga.norm_rotary(x, rotary=rot, q_norm=n, first=7, Q_out=x) is x
    y, size = D.norm_rotate(few_x, where, f, "half", 1.0, host(w), 1e-6, 0.0)
    assert within(x[:, at], y, D.norm_bar(y, size, "f16")) and int(torch.count_nonzero(x[0, :, 0])) <= 5


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_norm_gradient_against_differences(layout):
    freqs, m = sga.rotary_frequencies(32, scaling="parts", factor=8.0, original_length=4096)
    rot, f = sga.Rotary(freqs, layout, m), freqs.cpu().numpy()
    Q, G = tokens(3, 40, 64, "f32", 1), tokens(3, 40, 64, "f32", 2)
    w = weights_of("f32", 64, "f32", 0.0, 3)
    dQ, dw = sga.norm_rotary_backward(Q, G, rotary=rot, q_norm=sga.Norm(w, 1e-3), first=50)
    at = 50 + np.arange(40)
    want, want_w, size, w_size = D.norm_gradient(host(Q), host(G), at, f, layout, m, host(w), 1e-3, 0.0)
    assert within(dQ, want, D.gradient_bar(want, size, "f32")) and within(dw, want_w, D.weight_bar(w_size))
    loss = lambda x, v: (D.norm_rotate(x, at, f, layout, m, v, 1e-3, 0.0)[0] * host(G)).sum()
    x, v = host(Q), host(w)
    # central differences of step h in 64 bits: third derivatives here are below 100, so they are off by 100 h^2 / 6, and by rounding / h
    h = 1e-4
    for i in ((0, 0, 0), (1, 33, 17), (2, 39, 31), (0, 5, 40), (2, 1, 63)):
        up, down = x.copy(), x.copy()
        up[i] += h
        down[i] -= h
        assert abs((loss(up, v) - loss(down, v)) / (2 * h) - want[i]) <= 1e-6 * (1 + abs(want[i]))
    for c in (0, 17, 40, 63):
        up, down = v.copy(), v.copy()
        up[c] += h
        down[c] -= h
        assert abs((loss(x, up) - loss(x, down)) / (2 * h) - want_w[c]) <= 1e-6 * (1 + abs(want_w[c]))


def test_norms_captured_and_on_two_streams():
    rot = sga.Rotary(sga.rotary_frequencies(128)[0])
    Q, K, G, GK = (tokens(H, 300, 128, "bf16", i) for i, H in enumerate((8, 2, 8, 2)))
    w = weights_of("f32", 128, "bf16", 0.0, 1)
    n = sga.Norm(w)
    at = torch.arange(300).cuda()
    out = [torch.empty_like(x) for x in (Q, K, G, GK)]
    dw = [torch.empty(128, device="cuda") for _ in range(2)]
    spaces = [sga.alloc_norm_workspace(300, 8, 2, 128) for _ in range(2)]

    def step(out, dw, space):
        sga.norm_rotary(Q, K, rotary=rot, q_norm=n, k_norm=n, positions=at, Q_out=out[0], K_out=out[1])
        sga.norm_rotary_backward(Q, G, K, GK, rotary=rot, q_norm=n, k_norm=n, positions=at, dQ=out[2], dK=out[3], dq_weight=dw[0], dk_weight=dw[1],
                                 workspace=space)
    step(out, dw, spaces[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, dw, spaces[0])
    side = torch.cuda.Stream()
    other, other_w = [torch.empty_like(x) for x in out], [torch.empty_like(x) for x in dw]
    for k in range(4):
        at += 1000
        w.mul_(0.9)
        Q.mul_(1.1)
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):                         # at the same time, another workspace
            step(other, other_w, spaces[1])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out + dw, other + other_w))


# ---- into the cache -----------------------------------------------------------------------------------
def tree_of(parent, batch, spec=None, words=None, most=None):
    p = torch.from_numpy(np.asarray(parent, dtype=np.int32)).cuda()
    made = None
    if words:
        made = sga.DraftTree(torch.full((len(parent),), -9, dtype=torch.int32, device="cuda"),
                             torch.full((len(parent), words), -9, dtype=torch.int32, device="cuda"))
    return sga.build_draft_tree(p, batch, spec or full(1 << 20), tree=made, **({"most": most} if most else {}))


def random_parents(new, padding, chain, seed):
    rng = np.random.default_rng(seed)
    out = []
    for n in new:
        out += [t - 1 if rng.random() < chain else int(rng.integers(-1, max(t, 1))) if t else -1 for t in range(n)]
    return np.array(out + [5] * padding, dtype=np.int32)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("new,length,page,Hq,Hkv,d,channels,layout,padding", [
    ([1], [1], 16, 4, 1, 64, 64, "half", 0), ([16] * 5, [200, 16, 33, 48, 4000], 16, 8, 2, 128, 128, "half", 3),
    ([5, 0, 70, 1], [5, 9, 300, 64], 24, 6, 2, 128, 64, "interleaved", 7), ([33, 2], [33, 1000], 1, 3, 3, 64, 64, "half", 0),
    ([40, 41], [100, 41], 7, 2, 1, 80, 20, "half", 1), ([20], [700], 256, 16, 4, 256, 256, "interleaved", 0),
])
def test_append_of_normed_drafts(dtype, new, length, page, Hq, Hkv, d, channels, layout, padding):
    print("append normed", dtype, new, page, d, flush=True)
    batch, table, ptr, lens, n_pages, T = batch_of(new, length, page, padding=padding, seed=len(new))
    ck, cv = caches(n_pages, Hkv, page, d, dtype, 9)
    K, V, Q = tokens(Hkv, T, d, dtype, 1), tokens(Hkv, T, d, dtype, 2, "slice"), tokens(Hq, T, d, dtype, 3)
    freqs, _ = sga.rotary_frequencies(channels)
    f, rot = freqs.cpu().numpy(), sga.Rotary(freqs, layout, 1.25)
    wq, wk = weights_of("same", d, dtype, 0.0, 1), weights_of("f32", d, dtype, 1.0, 2)
    qn, kn = sga.Norm(wq), sga.Norm(wk, 0.25, 1.0)
    parent = random_parents(new, padding, 0.3, 4)
    tree = tree_of(parent, batch, most=max(new))
    depth, _ = D.tree(parent, ptr, lens, full(1 << 20), 16)
    row = np.arange(T)
    seq = np.searchsorted(ptr[1:], row, side="right")
    real = seq < len(new)
    base = np.where(real, (lens - np.diff(ptr))[np.minimum(seq, len(new) - 1)], 0)
    at = base + np.array([x or 0 for x in depth])
    k, k_size = D.norm_rotate(host(K), at, f, layout, 1.25, host(wk), 0.25, 1.0)
    q, q_size = D.norm_rotate(host(Q), at, f, layout, 1.25, host(wq), 1e-6, 0.0)
    want_k, want_v, bar = host(ck), host(cv), np.zeros(ck.shape)
    for r in np.nonzero(real)[0]:
        slot = base[r] + r - ptr[seq[r]]
        p, i = table[seq[r], slot // page], slot % page
        want_k[p, :, i], want_v[p, :, i] = k[:, r], host(V[:, r])
        bar[p, :, i] = D.norm_bar(k[:, r], k_size[:, r], dtype)
    out = torch.full((Hq, T, d), 7.0, dtype=DTYPE[dtype], device="cuda")
    before = ck.clone(), cv.clone()
    assert sga.cache_append(K, V, ck, cv, batch, rotary=rot, Q=Q, Q_out=out, q_norm=qn, k_norm=kn, tree=tree) is out
    assert within(ck, want_k, bar) and np.array_equal(host(cv), want_v)
    assert (host(out)[:, ~real] == 7).all() and within(host(out)[:, real], q[:, real], D.norm_bar(q, q_size, dtype)[:, real])
    # the tree alone is a rotation by its positions; a chain's tree is the plain call
    ck2, cv2 = before[0].clone(), before[1].clone()
    sga.cache_append(K, V, ck2, cv2, batch, rotary=rot, tree=tree)
    y, size = S.rotate(host(K), at, f, layout, 1.25)
    for r in np.nonzero(real)[0]:
        slot = base[r] + r - ptr[seq[r]]
        p, i = table[seq[r], slot // page], slot % page
        want_k[p, :, i], bar[p, :, i] = y[:, r], S.rotate_bar(y[:, r], size[:, r], dtype)
    assert within(ck2, want_k, bar) and torch.equal(cv2, cv)
    chain = tree_of(random_parents(new, padding, 1.1, 0), batch, most=max(new))
    ck3, cv3, q3 = before[0].clone(), before[1].clone(), torch.full_like(out, 7.0)
    sga.cache_append(K, V, ck3, cv3, batch, rotary=rot, Q=Q, Q_out=q3, tree=chain)
    ck4, cv4, q4 = before[0].clone(), before[1].clone(), torch.full_like(out, 7.0)
    sga.cache_append(K, V, ck4, cv4, batch, rotary=rot, Q=Q, Q_out=q4)
    # (two kernels, each within the rotation's bar of the same number, which is at most that of a pair whose size is sqrt(2) |pair|)
    def near(a, b):
        a, b = host(a), host(b)
        pair = np.zeros_like(a)
        one, two = (slice(0, channels // 2), slice(channels // 2, channels)) if layout == "half" else (slice(0, channels, 2), slice(1, channels, 2))
        pair[..., one] = pair[..., two] = np.sqrt(2) * 1.01 * np.hypot(b[..., one], b[..., two])
        return (np.abs(a - b) <= 2 * S.rotate_bar(1.01 * np.abs(b) + 1e-30, pair, dtype)).all()
    assert near(ck3, ck4) and torch.equal(cv3, cv4) and near(q3, q4)
    # norms without rotation
    sga.cache_append(K, V, ck4, cv4, batch, Q=Q, Q_out=q4, q_norm=qn, k_norm=kn)
    y, size = D.norm_rotate(host(Q), None, None, None, 1.0, host(wq), 1e-6, 0.0)
    assert within(host(q4)[:, real], y[:, real], D.norm_bar(y, size, dtype)[:, real])


@pytest.mark.parametrize("dtype,new,length,page,Hq,Hkv,d,channels,tree", [
    # prompts: more tokens than the chip's wavefronts take at once, one and four of them a wavefront
    ("f16", [20000, 1, 0, 3011, 9990], [20000, 700, 5, 4000, 30000], 16, 8, 4, 128, 128, False),
    ("bf16", [20000, 1, 0, 3011, 19990], [20017, 1, 9, 3011, 20000], 24, 4, 1, 64, 64, False),
    # one pair a lane, four tokens a workgroup
    ("f16", [40] * 100 + [107], [90] * 50 + [40] * 50 + [107], 16, 3, 2, 80, 20, True), ("f32", [4096, 3], [5000, 3], 7, 3, 1, 7, 6, False),
    # ... and more of them than a grid's
    ("f16", [(1 << 22) + 9, 2], [(1 << 22) + 9, 4], 64, 1, 1, 3, 2, False),
])
def test_append_of_many_normed_tokens(dtype, new, length, page, Hq, Hkv, d, channels, tree):
    print("append many", dtype, new[:5], page, d, tree, flush=True)
    batch, table, ptr, lens, n_pages, T = batch_of(new, length, page, padding=5)
    ck, cv = caches(n_pages, Hkv, page, d, dtype, 9)
    K, V, Q = tokens(Hkv, T, d, dtype, 1), tokens(Hkv, T, d, dtype, 2), tokens(Hq, T, d, dtype, 3)
    freqs, _ = sga.rotary_frequencies(channels)
    f, rot = freqs.cpu().numpy(), sga.Rotary(freqs)
    wq, wk = weights_of("same", d, dtype, 0.0, 1), weights_of("f32", d, dtype, 1.0, 2)
    end = int(ptr[-1])
    seq = np.repeat(np.arange(len(new)), new)
    slot = (lens - np.diff(ptr))[seq] + np.arange(end) - ptr[seq]
    at, made = slot, None
    if tree:
        parent = random_parents(new, 5, 0.3, 4)
        made = tree_of(parent, batch, most=max(new))
        depth, _ = D.tree(parent, ptr, lens, full(1 << 20), 16)
        at = (lens - np.diff(ptr))[seq] + np.array(depth[:end])
    k, k_size = D.norm_rotate(host(K[:, :end]), at, f, "half", 1.0, host(wk), 0.25, 1.0)
    q, q_size = D.norm_rotate(host(Q[:, :end]), at, f, "half", 1.0, host(wq), 1e-6, 0.0)
    want_k, want_v, bar = host(ck), host(cv), np.zeros(ck.shape)
    p, i = table[seq, slot // page], slot % page
    want_k[p, :, i], want_v[p, :, i] = k.transpose(1, 0, 2), host(V[:, :end]).transpose(1, 0, 2)
    bar[p, :, i] = D.norm_bar(k, k_size, dtype).transpose(1, 0, 2)
    out = torch.full((Hq, T, d), 7.0, dtype=DTYPE[dtype], device="cuda")
    sga.cache_append(K, V, ck, cv, batch, rotary=rot, Q=Q, Q_out=out, q_norm=sga.Norm(wq), k_norm=sga.Norm(wk, 0.25, 1.0), tree=made)
    assert within(ck, want_k, bar) and np.array_equal(host(cv), want_v)
    assert (out[:, end:] == 7).all() and within(out[:, :end], q, D.norm_bar(q, q_size, dtype))


def test_append_leaves_out_what_the_tree_does_not_have():
    """Rows of depth -1, missing pages, places before 0 and behind the table."""
    batch, table, ptr, lens, n_pages, T = batch_of([40, 30, 50], [40, 64, 60], 16, columns=4, missing=[(0, 1, -1), (1, 3, 10 ** 6), (2, 3, -7)])
    batch.seq_len[1], batch.seq_len[2] = 20, 70
    tree = tree_of(random_parents([40, 30, 50], 0, 0.4, 1), batch, words=1)
    assert (tree.depth.cpu().numpy() == -1).sum() == 8 + 18                   # one word: 32 tokens a sequence
    ck, cv = caches(n_pages, 2, 16, 64, "f32", 4)
    k0, v0 = ck.clone(), cv.clone()
    K, V, Q = (tokens(2, T, 64, "f32", s) for s in (1, 2, 3))
    out = torch.full_like(Q, 7.0)
    sga.cache_append(K, V, ck, cv, batch, Q=Q, Q_out=out, q_norm=sga.Norm(), tree=tree)
    base = [0, -10, 20]
    for s, (n, b) in enumerate(zip([40, 30, 50], base)):
        for t in range(n):
            r, slot = int(ptr[s]) + t, b + t
            there = t < 32 and 0 <= slot < 64 and 0 <= table[s, slot // 16] < n_pages
            if there:
                k0[table[s, slot // 16], :, slot % 16], v0[table[s, slot // 16], :, slot % 16] = K[:, r], V[:, r]
            assert (out[:, r] == 7).all() == (t >= 32)
    assert torch.equal(ck, k0) and torch.equal(cv, v0)


# ---- trees --------------------------------------------------------------------------------------------
@pytest.mark.parametrize("words", [1, 2, 3, 7, 16])
@pytest.mark.parametrize("spec", [full(1 << 20), MaskSpec(KIND_SLIDING, 5000, window=0), MaskSpec(KIND_SLIDING, 60, window=3),
                                  MaskSpec(KIND_GLOBAL_LOCAL, 70, window=2, n_global=20), MaskSpec(KIND_GLOBAL_LOCAL, 5000, window=40, n_global=61)])
def test_tree(words, spec):
    most = 32 * words
    new = [1, most, 0, most - 1, 7, most + 3, 33, 2 * most, 16, 64, 65]
    length = [1, most + 10, 3, 4000, 50, most + 3, 20, 2 * most + 1, 66, 64, 80]                # (the 33 tokens: of a sequence of 20)
    for chain in (0.0, 0.5, 0.97, 1.1):
        print("tree", words, spec, chain, flush=True)
        batch, _, ptr, lens, _, T = batch_of(new, length, 16, padding=5)
        parent = random_parents(new, 5, chain, words)
        parent[int(ptr[1]) + 3] = 99                          # no earlier token: the last of the context
        parent[int(ptr[4]) + 2], parent[int(ptr[4]) + 5] = 2, -50
        tree = tree_of(parent, batch, spec, words)
        depth, seen = D.tree(parent, ptr, lens, spec, words)
        end = int(ptr[-1])
        assert tree.depth.tolist()[:end] == depth[:end] and D.unpack(tree.seen.cpu().numpy()[:end]) == seen[:end]
        assert (tree.depth[end:] == -9).all() and (tree.seen[end:] == -9).all()


def test_tree_captured_of_many_sequences():
    rng = np.random.default_rng(1)
    new = [int(x) for x in rng.integers(0, 20, 3000)]
    batch, _, ptr, lens, _, T = batch_of(new, [n + int(x) for n, x in zip(new, rng.integers(0, 50, 3000))], 16)
    spec = MaskSpec(KIND_SLIDING, 60, window=5)
    parent = torch.from_numpy(random_parents(new, 0, 0.5, 0)).cuda()
    for most in (20, 70):
        tree = sga.build_draft_tree(parent, batch, spec, most=most)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            sga.build_draft_tree(parent, batch, spec, tree=tree)
        for k in range(3):
            parent.copy_(torch.from_numpy(random_parents(new, 0, 0.2 * k, k)))
            tree.seen.fill_(3)
            graph.replay()
            depth, seen = D.tree(parent.cpu().numpy(), ptr, lens, spec, tree.seen.shape[1])
            assert tree.depth.tolist() == depth and D.unpack(tree.seen.cpu().numpy()) == seen


@pytest.mark.parametrize("n_seqs,words", [(70000, 3), (270000, 1)])
def test_trees_of_more_sequences_than_a_grid(n_seqs, words):
    print("trees", n_seqs, words, flush=True)
    rng = np.random.default_rng(words)
    new = rng.integers(0, 3, n_seqs)
    new[[0, 65535, 65536, n_seqs - 1]] = 3
    lens = new + rng.integers(0, 9, n_seqs)
    batch, _, ptr, lens, _, T = batch_of(new.tolist(), lens.tolist(), 16)
    parent = random_parents(new.tolist(), 0, 0.5, 1)
    spec = MaskSpec(KIND_GLOBAL_LOCAL, 1000, window=1, n_global=4)
    tree = tree_of(parent, batch, spec, words)
    depth, seen = D.tree(parent, ptr, lens, spec, words)
    assert tree.depth.tolist() == depth and D.unpack(tree.seen.cpu().numpy()) == seen


# ---- attention ------------------------------------------------------------------------------------------
def check_tree_attention(dtype, new, length, page, Hq, Hkv, d, spec, padding=0, memory="token", missing=(), scale=None, workspace=True, chain=0.3,
                         seed=0, words=None, columns=None, change=None):
    print("attend tree", dtype, new[:6], length[:6], page, Hq, Hkv, d, spec, words, flush=True)
    batch, table, ptr, lens, n_pages, T = batch_of(new, length, page, padding=padding, seed=seed, missing=missing, columns=columns)
    ck, cv = caches(n_pages, Hkv, page, d, dtype, seed + 1)
    used = torch.zeros(n_pages, page, dtype=torch.bool)      # memory that no token was written to may hold anything
    for s, n in enumerate(length):
        p, r = S.places(table, s, np.arange(min(n, table.shape[1] * page)), page, n_pages)
        used[p[p >= 0], r[p >= 0]] = True
    used = used.cuda()[:, None, :, None]
    ck, cv = torch.where(used, ck, float("nan")), torch.where(used, cv, float("inf"))
    parent = random_parents(new, padding, chain, seed)
    tree = tree_of(parent, batch, spec, words or max(1, -(-max(new) // 32)))
    if change:
        change(tree, ptr)
    depth = tree.depth.cpu().numpy()
    seen = D.unpack(tree.seen.cpu().numpy())
    if change is None:
        assert (depth[:ptr[-1]].tolist(), seen[:ptr[-1]]) == tuple(x[:ptr[-1]] for x in D.tree(parent, ptr, lens, spec, tree.seen.shape[1]))
    Q = tokens(Hq, T, d, dtype, seed + 3, memory)
    scale = 1 / math.sqrt(d) if scale is None else scale
    long = long_chunks(dtype, T, len(new), Hq // Hkv, d, page)
    want, want_lse, bar, lse_bar = D.attend(host(Q), host(ck), host(cv), table, ptr, lens, depth, seen, spec, scale, dtype, long)
    O = torch.full((Hq, T, d), 7.0, dtype=DTYPE[dtype], device="cuda")
    lse = torch.full((Hq, T), 7.0, device="cuda")
    ws = sga.alloc_paged_workspace(batch, spec, Hq, Hkv, d, dtype, tree=tree) if workspace else None
    assert sga.sga_profile_enable(1) == 0
    sga.attention_paged(Q, ck, cv, batch, spec, scale, O=O, lse=lse, workspace=ws, tree=tree)
    torch.cuda.synchronize()
    kernel = sga.sga_profile_last_kernel()
    sga.sga_profile_enable(0)
    assert dtype == "f32" or kernel == ("paged_chunk_kernel" if long else "paged_kernel")
    end = int(ptr[-1])
    assert (host(O)[:, end:] == 7).all() and (host(lse)[:, end:] == 7).all()
    assert within(host(O)[:, :end], want[:, :end], bar[:, :end]) and within(host(lse)[:, :end], want_lse[:, :end], lse_bar[:, :end])
    return kernel


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("page", [16, 24, 1])
def test_tree_attention_types(dtype, d, page):
    check_tree_attention(dtype, [1, 3, 20], [77, 40, 20], page, 4, 2, d, full(96), padding=2)
    check_tree_attention(dtype, [40, 9], [130, 50], page, 3, 1, d, MaskSpec(KIND_GLOBAL_LOCAL, 144, window=17, n_global=5))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (5, 5), (6, 2), (7, 1), (16, 2), (40, 2), (64, 1)])
def test_tree_attention_shared_heads(dtype, Hq, Hkv):
    check_tree_attention(dtype, [1, 13, 6], [1, 33, 100], 16, Hq, Hkv, 64, full(112))


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("chain", [0.0, 0.5, 1.1])
@pytest.mark.parametrize("spec", [
    full(160), MaskSpec(KIND_SLIDING, 160, window=0), MaskSpec(KIND_SLIDING, 160, window=1), MaskSpec(KIND_SLIDING, 160, window=31),
    MaskSpec(KIND_SLIDING, 160, window=70), MaskSpec(KIND_GLOBAL_LOCAL, 160, window=3, n_global=1), MaskSpec(KIND_GLOBAL_LOCAL, 160, window=20, n_global=40),
    MaskSpec(KIND_GLOBAL_LOCAL, 160, window=0, n_global=0), MaskSpec(KIND_GLOBAL_LOCAL, 160, window=5, n_global=160), MaskSpec(KIND_SLIDING, 60, window=40),
])
def test_tree_attention_masks(dtype, spec, chain):
    # trees alone, behind short and long contexts; sequences that pass the mask's length, in places only and in positions too
    for new, length in (([64, 37, 1, 0, 90], [64, 90, 144, 12, 150]), ([5, 7, 3], [64, 30, 60])):
        check_tree_attention(dtype, new, length, 16, 4, 2, 64, spec, chain=chain)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_tree_attention_split_sequences(dtype):
    """Few long contexts: pieces of the keys on workgroups of their own, joined afterwards."""
    for page in (16, 40):
        for new in ([4, 2, 7], [60, 41, 7], [200, 150, 130]):
            check_tree_attention(dtype, new, [3000, 1203, 200], page, 4, 2, 64, full(5008))
        check_tree_attention(dtype, [4, 2, 7], [3000, 1203, 200], page, 4, 2, 64, full(5008), workspace=False)
        check_tree_attention(dtype, [9, 30], [3000, 2999], page, 2, 1, 128, MaskSpec(KIND_GLOBAL_LOCAL, 3000, window=1500, n_global=70))


@pytest.mark.parametrize("memory", ["head", "token", "slice"])
def test_tree_attention_strides(memory):
    check_tree_attention("f16", [7, 1, 30], [40, 90, 30], 32, 6, 3, 64, full(96), memory=memory)


@pytest.mark.parametrize("scale", [-0.3, 0.0, 2.5])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_tree_attention_scales(dtype, scale):
    check_tree_attention(dtype, [7, 1, 12], [40, 90, 30], 16, 4, 2, 64, MaskSpec(KIND_GLOBAL_LOCAL, 96, window=20, n_global=3), scale=scale)
    check_tree_attention(dtype, [60, 80], [140, 90], 16, 4, 2, 64, MaskSpec(KIND_GLOBAL_LOCAL, 160, window=40, n_global=3), scale=scale)


def test_tree_attention_of_missing_pages_and_short_tables():
    spec = MaskSpec(KIND_SLIDING, 400, window=50)
    gone = [(0, c, -1) for c in range(0, 21)]
    check_tree_attention("f16", [5, 9], [400, 390], 16, 4, 4, 64, spec, missing=gone)
    check_tree_attention("f32", [33, 3], [400, 390], 16, 4, 4, 64, spec, missing=gone + [(0, 22, -1), (1, 24, 10 ** 7)])
    check_tree_attention("f16", [33, 3], [400, 390], 16, 4, 4, 64, spec, missing=gone + [(0, 22, -1), (1, 24, 10 ** 7)])
    check_tree_attention("f32", [3, 1], [400, 390], 16, 4, 4, 64, spec, missing=[(0, c, -1) for c in range(25)])       # rows that see nothing
    check_tree_attention("bf16", [40, 10], [400, 390], 5, 4, 4, 64, spec, missing=[(1, c, -1) for c in range(70, 78)])


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("new", [[9, 30, 2], [90, 64, 70]])
def test_tree_attention_of_any_bits(dtype, new):
    """What a program writes by itself: any bits, beyond the sequence's tokens too, any depths, rows that are none of the tree."""
    def scramble(tree, ptr):
        rng = np.random.default_rng(7)
        tree.seen.copy_(torch.from_numpy(rng.integers(-2 ** 31, 2 ** 31, tree.seen.shape).astype(np.int32)))
        d = rng.integers(0, 50, tree.depth.shape[0])
        d[::5] = -1 - d[::5]
        tree.depth.copy_(torch.from_numpy(d))
        tree.seen[1::7] = 0                                   # rows that see no new token
    for spec in (full(400), MaskSpec(KIND_GLOBAL_LOCAL, 150, window=60, n_global=9)):
        for extra in (0, 1, 60):
            check_tree_attention(dtype, new, [n + extra for n in new], 16, 4, 2, 64, spec, change=scramble, words=-(-max(new) // 32))
        check_tree_attention(dtype, new, [n + 5 for n in new], 24, 4, 2, 64, spec, change=scramble, words=1)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("page", [16, 24])
@pytest.mark.parametrize("n", [7, 100])
def test_tree_attention_of_infinities_that_are_not_seen(dtype, page, n):
    """A drafted token's key and value hold infinities and NaN: rows of other branches, and other heads, are as if it were not there."""
    batch, table, ptr, lens, n_pages, T = batch_of([n], [n + 70], page)
    ck, cv = caches(n_pages, 2, page, 64, dtype, 1)
    parent = np.array([-1] + [(t - 1) // 2 for t in range(1, n)])
    spec = full(400)
    tree = tree_of(parent, batch, spec, most=n)
    depth, seen = D.tree(parent, ptr, lens, spec, tree.seen.shape[1])
    Q = tokens(2, T, 64, dtype, 3)
    want, _, bar, _ = D.attend(host(Q), host(ck), host(cv), table, ptr, lens, depth, seen, spec, 0.125, dtype, long_chunks(dtype, T, 1, 1, 64, page))
    bad = 2
    at = 70 + bad
    ck[table[0, at // page], 0, at % page, 3] = float("nan")
    cv[table[0, at // page], 0, at % page, 5] = float("inf")
    got = host(sga.attention_paged(Q, ck, cv, batch, spec, 0.125, tree=tree))
    sees = np.array([bad in x for x in seen])
    assert sees.any() and not sees.all() and np.isnan(got[0, sees]).all()
    assert within(got[0, ~sees], want[0, ~sees], bar[0, ~sees]) and within(got[1], want[1], bar[1])


@pytest.mark.parametrize("dtype,d,new", [("f32", 64, 9), ("f16", 128, 9), ("bf16", 128, 90), ("f32", 128, 90)])
def test_a_chain_is_the_causal_call(dtype, d, new):
    """Drafts that follow each other are what attention over the cache has always computed: within the bars of both."""
    spec = MaskSpec(KIND_GLOBAL_LOCAL, 2000, window=300, n_global=7)
    batch, table, ptr, lens, n_pages, T = batch_of([new, 3], [1500, 700], 16)
    ck, cv = caches(n_pages, 2, 16, d, dtype, 1)
    Q = tokens(8, T, d, dtype, 2)
    tree = tree_of(random_parents([new, 3], 0, 1.1, 0), batch, spec, most=new)
    ws = sga.alloc_paged_workspace(batch, spec, 8, 2, d, dtype, tree=tree)
    a, la = sga.attention_paged(Q, ck, cv, batch, spec, 0.1, tree=tree, workspace=ws, want_lse=True)
    b, lb = sga.attention_paged(Q, ck, cv, batch, spec, 0.1, want_lse=True)
    _, _, bar, lse_bar = S.attend(host(Q), host(ck), host(cv), table, ptr, lens, spec, 0.1, True, dtype, long_chunks(dtype, T, 2, 4, d, 16))
    assert (np.abs(host(a) - host(b)) <= 2 * bar).all() and (np.abs(host(la) - host(lb)) <= 2 * lse_bar).all()


def tree_on_device(Q, ck, cv, table, ptr, new, length, has, depth, spec, scale, dtype, once):
    """drafts_oracle.attend, a sequence at a time in 64 bits on the device: (O, lse, bar of O, bar of lse).  has: [T][most] bits as booleans."""
    page, Hkv, d = ck.shape[2], ck.shape[1], ck.shape[3]
    G, parts = Q.shape[0] // Hkv, {"f32": 0.0, "f16": 2.0 ** -21, "bf16": 2.0 ** -15}[dtype] if not once else S.HALF_STEP[dtype]
    out = [[], [], [], []]
    for s, (n, L) in enumerate(zip(new, length)):
        base, rows = L - n, slice(int(ptr[s]), int(ptr[s]) + n)
        low = max(0, base - spec.window) if base >= spec.n_global else 0
        at = torch.cat((torch.arange(min(spec.n_global, low)), torch.arange(low, L))).cuda()
        where = torch.from_numpy(table[s].astype(np.int64)).cuda()[at // page]
        k, v = (c[where, :, at % page].double().transpose(0, 1).unsqueeze(1) for c in (ck, cv))              # [Hkv, 1, keys, d]
        q = Q[:, rows].double().reshape(Hkv, G, n, d)
        p = base + depth[rows].long()[:, None]
        see = ((p - at <= spec.window) | (at < spec.n_global) | (p < spec.n_global)) & (at < base)
        see[:, at >= base] = has[rows, :n]
        z = scale * torch.matmul(q, k.transpose(-1, -2).contiguous())
        size = torch.matmul(q.abs(), k.abs().transpose(-1, -2).contiguous()).masked_fill_(~see, 0.0).amax(-1)
        off = d * 2.0 ** -24 * abs(scale) * size + 2.0 ** -22 * (1 + z.abs().masked_fill_(~see, 0.0).amax(-1))
        z.masked_fill_(~see, -math.inf)
        lse = torch.logsumexp(z, -1)
        w = (z - lse.unsqueeze(-1)).exp()
        O, share = torch.matmul(w, v), torch.matmul(w, v.abs())
        bar = share * (2 * off + parts + (4 + math.sqrt(L)) * 2.0 ** -23).unsqueeze(-1) + O.abs() * S.HALF_STEP[dtype]
        if dtype == "f16":
            bar += 2.0 ** -35 * v.abs().sum(-2, keepdim=True) + 2.0 ** -25
        for x, y in zip(out, (O, lse, bar, 2 * off + 2.0 ** -22 * (1 + lse.abs()))):
            x.append(y.reshape(Hkv * G, n, *y.shape[3:]))
    return [host(torch.cat(x, 1)) for x in out]


@pytest.mark.parametrize("dtype,Hq,Hkv,d,page,n_seqs,new,alike", [
    ("f16", 16, 4, 128, 16, 130, 13, True), ("bf16", 16, 8, 64, 24, 100, 20, True), ("f16", 16, 8, 128, 16, 70, 30, False),
    ("bf16", 8, 1, 256, 16, 270, 9, True), ("f32", 4, 2, 128, 32, 140, 40, True), ("f16", 5, 5, 128, 16, 110, 40, True),
    ("f16", 16, 4, 128, 16, 65, 70, True), ("f16", 8, 8, 64, 1, 96, 33, True), ("bf16", 2, 2, 128, 16, 256, 40, True),
])
def test_tree_attention_of_many_tiles(dtype, Hq, Hkv, d, page, n_seqs, new, alike):
    """Tiles that are more than the places on the chip: alike, whole rounds of them uncut and the rest in pieces; all in one round; of all lengths."""
    rng = np.random.default_rng(n_seqs)
    n = [max(1, new - int(x)) for x in rng.integers(0, 3, n_seqs)]
    length = [a + int(b) for a, b in zip(n, rng.integers(1500, 2000, n_seqs) if alike else rng.integers(1, 2000, n_seqs))]
    spec = MaskSpec(KIND_GLOBAL_LOCAL, 2100, window=1000, n_global=7) if alike else MaskSpec(KIND_GLOBAL_LOCAL, 2100, window=2100, n_global=0)
    batch, table, ptr, lens, n_pages, T = batch_of(n, length, page, padding=2)
    ck, cv = caches(n_pages, Hkv, page, d, dtype, 1)
    Q = tokens(Hq, T, d, dtype, 2)
    parent = random_parents(n, 2, 0.4, 3)
    tree = tree_of(parent, batch, spec, most=max(n))
    _, seen = D.tree(parent, ptr, lens, spec, tree.seen.shape[1])
    has = torch.zeros(T, 32 * tree.seen.shape[1], dtype=torch.bool)
    for row, x in enumerate(seen[:int(ptr[-1])]):
        has[row, list(x)] = True
    once = long_chunks(dtype, T, n_seqs, Hq // Hkv, d, page)
    want = tree_on_device(Q, ck, cv, table, ptr, n, length, has.cuda(), tree.depth, spec, 0.1, dtype, once)
    end = int(ptr[-1])
    for ws in (sga.alloc_paged_workspace(batch, spec, Hq, Hkv, d, dtype, tree=tree), None):
        print("many tiles", dtype, Hq, Hkv, d, page, n_seqs, new, alike, ws is None, flush=True)
        got = sga.attention_paged(Q, ck, cv, batch, spec, 0.1, workspace=ws, want_lse=True, tree=tree)
        assert within(got[0][:, :end], want[0], want[2]) and within(got[1][:, :end], want[1], want[3])


def test_tree_attention_far_pages():
    """Offsets of more than 2^31 elements, in both kernels, and in the moves."""
    Hkv, d, page, length = 8, 128, 64, 150
    n_pages, columns = (1 << 31) // (page * Hkv * d) + 40, 3
    ck, cv = (torch.empty(n_pages, Hkv, page, d, dtype=torch.float16, device="cuda") for _ in range(2))
    table = np.array([[n_pages - 1, 5, n_pages - 9]], dtype=np.int32)
    at = torch.from_numpy(table[0].astype(np.int64)).cuda()
    for c, seed in ((ck, 1), (cv, 2)):
        c[at] = torch.randn(3, Hkv, page, d, generator=torch.Generator().manual_seed(seed)).half().cuda()
    small = [host(c[at]) for c in (ck, cv)]
    for new in (9, 60):
        dev = [torch.from_numpy(x).cuda() for x in (table, np.array([0, new]), np.array([length], dtype=np.int32))]
        batch = sga.PagedBatch(*dev, new, page, n_pages)
        parent = random_parents([new], 0, 0.3, 1)
        tree = tree_of(parent, batch, full(200), most=new)
        Q = tokens(16, new, d, "f16", 3)
        depth, seen = D.tree(parent, [0, new], [length], full(200), tree.seen.shape[1])
        want, lse, bar, lse_bar = D.attend(host(Q), *small, np.arange(3)[None], np.array([0, new]), [length], depth, seen, full(200), 0.1, "f16", new * 2 > 32)
        got = sga.attention_paged(Q, ck, cv, batch, full(200), 0.1, want_lse=True, tree=tree)
        assert within(got[0], want, bar) and within(got[1], lse, lse_bar)
    K, V, w = tokens(Hkv, new, d, "f16", 4), tokens(Hkv, new, d, "f16", 5), weights_of("same", d, "f16", 0.0, 6)
    sga.cache_append(K, V, ck, cv, batch, k_norm=sga.Norm(w), tree=tree)
    k, size = D.norm_rotate(host(K), None, None, None, 1.0, host(w), 1e-6, 0.0)
    for t in range(new):
        c, r = divmod(length - new + t, page)
        assert within(ck[int(table[0, c]), :, r], k[:, t], D.norm_bar(k[:, t], size[:, t], "f16")) and torch.equal(cv[int(table[0, c]), :, r], V[:, t])
    small = [host(c[at]) for c in (ck, cv)]
    path = torch.tensor([[3, 9, 40, 59]], dtype=torch.int32, device="cuda")
    sga.cache_keep(ck, cv, batch, path, torch.tensor([4], dtype=torch.int32, device="cuda"))
    for c, x in ((ck, small[0]), (cv, small[1])):
        assert np.array_equal(host(c[at]), D.keep(x, np.arange(3)[None], [0, 60], [length], path.cpu().numpy(), [4]))


# ---- accepted tokens -------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("layers,Hkv,d,page", [(0, 2, 64, 16), (1, 8, 128, 16), (3, 1, 7, 5), (2, 3, 80, 1), (5, 2, 256, 64), (2, 1, 1024, 3)])
def test_keep(dtype, layers, Hkv, d, page):
    new, length = [16, 1, 0, 90, 5, 200, 30], [40, 1, 9, 90, 64, 300, 20]     # (the last: more new tokens than the sequence has)
    batch, table, ptr, lens, n_pages, T = batch_of(new, length, page, padding=3, missing=[(4, 0, -1)] if page > 16 else [(5, -(-250 // page), -1), (5, 9, 10 ** 6)])
    g = torch.Generator().manual_seed(d)
    shape = (n_pages, Hkv, page, d) if layers == 0 else (layers, n_pages, Hkv, page, d)
    ck, cv = (torch.randn(shape, generator=g).to(DTYPE[dtype]).cuda() for _ in range(2))
    rng = np.random.default_rng(d)
    path = np.full((len(new), 100), 10 ** 6, dtype=np.int32)
    count = np.array([5, 1, 3, 90, -2, 100, 9], dtype=np.int32)
    for s, (n, c) in enumerate(zip(new, count)):
        if n > 0 and c > 0:
            chosen = np.sort(rng.permutation(n)[:min(c, n)])
            path[s, :len(chosen)] = chosen
    path[0, :5] = [2, 2, 7, 3, 99]                            # an index twice, falling ones, none of the tokens: what is not below k moves
    count[5] = 10 ** 6                                        # no more than the columns
    want = [D.keep(host(c), table, ptr, lens, path, count) for c in (ck, cv)]
    sga.cache_keep(ck, cv, batch, torch.from_numpy(path).cuda(), torch.from_numpy(count).cuda())
    assert np.array_equal(host(ck), want[0]) and np.array_equal(host(cv), want[1])


def test_keep_of_more_sequences_than_a_grid():
    S_, page = 40000, 4
    rng = np.random.default_rng(1)
    new = rng.integers(0, 4, S_)
    lens = -(-rng.integers(0, 5, S_) // page) * page + new   # (no two sequences have new tokens in one page, and each begins one)
    batch, table, ptr, lens, n_pages, T = batch_of(new.tolist(), lens.tolist(), page)
    ck, cv = caches(n_pages, 1, page, 8, "f16", 1)
    path = np.sort(rng.integers(0, 4, (S_, 3)), 1).astype(np.int32)
    count = rng.integers(0, 4, S_).astype(np.int32)
    want = [D.keep(host(c), table, ptr, lens, path, count) for c in (ck, cv)]
    sga.cache_keep(ck, cv, batch, torch.from_numpy(path).cuda(), torch.from_numpy(count).cuda())
    assert np.array_equal(host(ck), want[0]) and np.array_equal(host(cv), want[1])


def test_keep_of_layers_that_take_turns():
    """Layers, keys and values page by page in one buffer, and nothing written beside them."""
    batch, table, ptr, lens, n_pages, T = batch_of([9, 20], [30, 44], 8)
    whole = torch.randn(n_pages, 5, 2, 2, 8, 64, device="cuda")              # [pages][layers][keys, values][heads][tokens][channels]
    before = whole.clone()
    ck, cv = whole[:, 1:4, 0].transpose(0, 1), whole[:, 1:4, 1].transpose(0, 1)
    path = torch.tensor([[1, 4, 8], [0, 5, 19]], dtype=torch.int32, device="cuda")
    count = torch.tensor([3, 3], dtype=torch.int32, device="cuda")
    want = [D.keep(host(c), table, ptr, lens, path.cpu().numpy(), [3, 3]) for c in (ck, cv)]
    sga.cache_keep(ck, cv, batch, path, count)
    assert np.array_equal(host(ck), want[0]) and np.array_equal(host(cv), want[1])
    assert torch.equal(whole[:, [0, 4]], before[:, [0, 4]])
    with pytest.raises(ValueError):
        sga.cache_keep(torch.empty(1, device="cuda").expand(2, n_pages, 2, 8, 64), torch.empty(1, device="cuda").expand(2, n_pages, 2, 8, 64), batch, path, count)


def test_steps_on_two_streams_at_once():
    """Pages, trees, attention over them and moves of two batches on two streams that overlap in time, each with workspaces of its own."""
    work = []
    for s, (n, d) in enumerate((([5, 16, 3], 128), ([60, 33, 90], 64))):
        batch, table, ptr, lens, n_pages, T = batch_of(n, [4000, 900, 2500], 16, spare=40)
        spec = MaskSpec(KIND_GLOBAL_LOCAL, 4096, window=1500, n_global=3)
        ck, cv = caches(n_pages, 2, 16, d, "bf16", s)
        used = set(table[table >= 0].tolist())
        free = torch.tensor([p for p in range(n_pages) if p not in used] + [-1] * len(used), dtype=torch.int32, device="cuda")
        state = torch.tensor([0, n_pages - len(used)], device="cuda")
        parent = torch.from_numpy(random_parents(n, 0, 0.4, s)).cuda()
        ask = torch.tensor([3, 7, 1], dtype=torch.int32, device="cuda")
        path = torch.tensor([[1, 2], [0, 9], [2, 2]], dtype=torch.int32, device="cuda")
        count = torch.tensor([2, 2, 1], dtype=torch.int32, device="cuda")
        work.append((batch, spec, ck, cv, free, state, parent, ask, path, count, tokens(8, T, d, "bf16", s + 5), max(n)))

    def run(w, spaces=None):
        batch, spec, ck, cv, free, state, parent, ask, path, count, Q, most = w
        ck, cv, ring = ck.clone(), cv.clone(), free.clone()
        after = sga.PagedBatch(torch.empty_like(batch.page_table), torch.empty_like(batch.seq_ptr), torch.empty_like(batch.seq_len), batch.n_tokens, 16, batch.n_pages)
        pool = sga.PagePool(ring, torch.empty_like(state))
        tree = sga.build_draft_tree(parent, batch, spec, most=most)
        ws = sga.alloc_paged_workspace(batch, spec, 8, 2, Q.shape[2], "bf16", tree=tree)
        O, lse = sga.attention_paged(Q, ck, cv, batch, spec, 0.09, workspace=ws, tree=tree, want_lse=True)
        sga.cache_keep(ck, cv, batch, path, count)
        sga.pages_advance(batch, sga.PagePool(ring, state), ask, kept=count, spec=spec, out=(after, pool))
        return [tree.depth, tree.seen, O, lse, ck, cv, ring, pool.state, after.page_table, after.seq_ptr, after.seq_len]
    want = [run(w) for w in work]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in work], [[], []]
    for _ in range(6):
        for i, w in enumerate(work):
            with torch.cuda.stream(streams[i]):
                got[i].append(run(w))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for x, many in zip(want, got) for y in many for a, b in zip(x, y))


# ---- refusals of tensors -----------------------------------------------------------------------------------
def test_refusals():
    batch, *_, n_pages, T = batch_of([3, 2], [20, 9], 16)
    ck, cv = caches(n_pages, 2, 16, 64, "f16", 1)
    Q, K = tokens(4, T, 64, "f16", 1), tokens(2, T, 64, "f16", 2)
    rot, n, ints = sga.Rotary(sga.rotary_frequencies(64)[0]), sga.Norm(torch.ones(64, device="cuda")), lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    wrong = sga.Norm(torch.ones(32, device="cuda"))
    tree = sga.build_draft_tree(ints(T), batch, full(32))
    other = sga.DraftTree(ints(T + 1), ints(T + 1, 1))
    pool, small = sga.PagePool.full(n_pages), sga.PagePool.full(n_pages + 1)
    out = sga.PagedBatch(batch.page_table.clone(), batch.seq_ptr.clone(), batch.seq_len.clone(), T + 1, 16, n_pages)
    path, count = ints(2, 3), ints(2)
    for bad in (lambda: sga.norm_rotary(Q), lambda: sga.norm_rotary(Q, q_norm=wrong), lambda: sga.norm_rotary(Q, K[:, :-1], rotary=rot),
                lambda: sga.norm_rotary(Q, K.float(), rotary=rot), lambda: sga.norm_rotary(Q, rotary=rot, k_norm=n), lambda: sga.norm_rotary(Q, rotary=rot, Q_out=K),
                lambda: sga.norm_rotary(Q, rotary=rot, K_out=K), lambda: sga.norm_rotary(Q.cpu(), q_norm=n), lambda: sga.norm_rotary(Q[..., ::2], q_norm=sga.Norm()),
                lambda: sga.norm_rotary(Q, rotary=rot, positions=ints(T)), lambda: sga.norm_rotary_backward(Q, K, q_norm=n),
                lambda: sga.norm_rotary_backward(Q, Q, K, q_norm=n), lambda: sga.norm_rotary_backward(Q, Q, dK=K, q_norm=n),
                lambda: sga.norm_rotary_backward(Q, Q, rotary=rot, dq_weight=torch.empty(64, device="cuda")),
                lambda: sga.norm_rotary_backward(Q, Q, q_norm=n, dq_weight=torch.empty(64, device="cuda").half()),
                lambda: sga.norm_rotary_backward(Q, Q, q_norm=n, workspace=torch.empty(100)),
                lambda: sga.norm_rotary_backward(Q, Q, q_norm=n, dQ=torch.empty(4, 1, 64, dtype=torch.float16, device="cuda").expand(4, T, 64)),
                lambda: sga.cache_append(K, K, ck, cv, batch, q_norm=n), lambda: sga.cache_append(K, K, ck, cv, batch, k_norm=wrong),
                lambda: sga.cache_append(K, K, ck, cv, batch, tree=other), lambda: sga.cache_append(K, K, ck, cv, batch, Q=Q, k_norm=n),
                lambda: sga.attention_paged(Q, ck, cv, batch, full(32), 0.1, tree=other), lambda: sga.attention_paged(Q, ck, cv, batch, full(32), 0.1, tree=tree, causal=False),
                lambda: sga.alloc_paged_workspace(batch, full(32), 4, 2, 64, "f16", tree=other), lambda: sga.build_draft_tree(ints(T + 1), batch, full(32)),
                lambda: sga.build_draft_tree(ints(T).long(), batch, full(32)), lambda: sga.build_draft_tree(ints(T), batch, full(32), most=513),
                lambda: sga.build_draft_tree(ints(T), batch, full(32), tree=other), lambda: sga.pages_advance(batch, small, ints(2)),
                lambda: sga.pages_advance(batch, pool, ints(3)), lambda: sga.pages_advance(batch, pool, ints(2), kept=ints(3)),
                lambda: sga.pages_advance(batch, pool, ints(2), slots=ints(T)), lambda: sga.pages_advance(batch, pool, ints(2), out=(out, pool)),
                lambda: sga.pages_advance(batch, pool, ints(2), out=(batch, sga.PagePool.full(n_pages))), lambda: sga.cache_keep(ck, cv, batch, path.long(), count),
                lambda: sga.cache_keep(ck, cv[:-1], batch, path, count), lambda: sga.cache_keep(ck, cv, batch, ints(3, 3), count),
                lambda: sga.cache_keep(ck, cv, batch, path, ints(3)), lambda: sga.cache_keep(ck[None], cv, batch, path, count),
                lambda: sga.cache_keep(ck.cpu(), cv, batch, path, count)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(sga.SgaError):                        # a workspace that is too small
        sga.norm_rotary_backward(Q, Q, q_norm=n, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(sga.SgaError):
        sga.pages_advance(batch, pool, ints(2), workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))


# ---- together ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,d,captured", [("f32", 64, False), ("f16", 128, True), ("bf16", 64, True)])
def test_generation_with_drafts_is_the_whole_sequence(dtype, d, captured):
    """Steps of drafts, part of which stay, through pages that come and go, two layers, captured or not; then every token that stayed, against the
    definitions on the whole sequence: its key in the cache, and its output among what was there."""
    rng = np.random.default_rng(3)
    S_, Hkv, G, page, layers, n_pages, T = 3, 2, 2, 8, 2, 90, 60
    Hq, C = Hkv * G, 40
    spec = MaskSpec(KIND_GLOBAL_LOCAL, 1 << 20, window=50, n_global=5)
    freqs, _ = sga.rotary_frequencies(d)
    f, rot, scale = freqs.cpu().numpy(), sga.Rotary(freqs), 1 / math.sqrt(d)
    wq, wk = weights_of("same", d, dtype, 0.0, 1), weights_of("same", d, dtype, 0.0, 2)
    qn, kn = sga.Norm(wq), sga.Norm(wk)
    batch = sga.PagedBatch(torch.full((S_, C), -1, dtype=torch.int32, device="cuda"), torch.zeros(S_ + 1, dtype=torch.int64, device="cuda"),
                           torch.zeros(S_, dtype=torch.int32, device="cuda"), T, page, n_pages)
    pool = sga.PagePool.full(n_pages)
    ask, kept = (torch.zeros(S_, dtype=torch.int32, device="cuda") for _ in range(2))
    parent = torch.zeros(T, dtype=torch.int32, device="cuda")
    path, count = torch.zeros(S_, 20, dtype=torch.int32, device="cuda"), torch.zeros(S_, dtype=torch.int32, device="cuda")
    tree = sga.DraftTree(torch.zeros(T, dtype=torch.int32, device="cuda"), torch.zeros(T, 1, dtype=torch.int32, device="cuda"))
    ck, cv = (torch.full((layers, n_pages, Hkv, page, d), float("nan"), dtype=DTYPE[dtype], device="cuda") for _ in range(2))
    x = [[torch.zeros(T, H, d, dtype=DTYPE[dtype], device="cuda").transpose(0, 1) for H in (Hq, Hkv, Hkv)] for _ in range(layers)]
    q, O = ([torch.zeros_like(y[0]) for y in x] for _ in range(2))
    space, pages_space = sga.alloc_paged_workspace(batch, spec, Hq, Hkv, d, dtype, tree=tree), sga.alloc_pages_workspace(batch)

    def begin():
        sga.pages_advance(batch, pool, ask, kept=kept, spec=spec, workspace=pages_space)
        sga.build_draft_tree(parent, batch, spec, tree=tree)
        for l in range(layers):
            sga.cache_append(x[l][1], x[l][2], ck[l], cv[l], batch, rotary=rot, Q=x[l][0], Q_out=q[l], q_norm=qn, k_norm=kn, tree=tree)
            sga.attention_paged(q[l], ck[l], cv[l], batch, spec, scale, O=O[l], workspace=space, tree=tree)

    end = lambda: sga.cache_keep(ck, cv, batch, path, count)
    run_begin, run_end = begin, end
    if captured:
        begin()
        end()
        torch.cuda.synchronize()
        graphs = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        for graph, call in zip(graphs, (begin, end)):
            with torch.cuda.graph(graph):
                call()
        run_begin, run_end = (g.replay for g in graphs)
    done = [[[] for _ in range(S_)] for _ in range(layers)]       # the tokens that stayed: q, k, v as they came, and O
    for step in range(30):
        n = [int(rng.integers(1, 21)) for _ in range(S_)]
        if step == 17:
            n[1] = -1                                             # one sequence ends; its place is another's from the next step on
        kept.copy_(count)
        ask.copy_(torch.tensor(n))
        rows = [max(k, 0) for k in n]
        ptr = np.concatenate(([0], np.cumsum(rows)))
        p = random_parents(rows, T - ptr[-1], 0.5, step)
        parent.copy_(torch.from_numpy(p))
        for l in range(layers):
            for i, y in enumerate(x[l]):
                y.copy_(tokens(y.shape[0], T, d, dtype, 100 * step + 10 * l + i))
        run_begin()
        torch.cuda.synchronize()
        assert batch.seq_ptr.tolist() == ptr.tolist()
        path_, count_ = np.zeros((S_, 20), dtype=np.int32), np.zeros(S_, dtype=np.int32)
        for s in range(S_):
            if n[s] < 0:
                for l in range(layers):
                    done[l][s] = []
                continue
            assert int(batch.seq_len[s]) == len(done[0][s]) + n[s]
            leaf = int(rng.integers(0, n[s]))
            way = D.paths(p[ptr[s]:ptr[s + 1]].tolist())[leaf][::-1]
            path_[s, :len(way)], count_[s] = way, len(way)
            for l in range(layers):
                for t in way:
                    done[l][s].append([host(y[:, ptr[s] + t]) for y in x[l]] + [host(O[l][:, ptr[s] + t])])
        path.copy_(torch.from_numpy(path_))
        count.copy_(torch.from_numpy(count_))
        run_end()
    torch.cuda.synchronize()
    table = batch.page_table.cpu().numpy()
    once = long_chunks(dtype, T, S_, G, d, page)
    for l in range(layers):
        for s in range(S_):
            L = len(done[l][s])
            assert L > 15
            Q, K, V, out = (np.stack([z[i] for z in done[l][s]], 1) for i in range(4))
            k64, k_size = D.norm_rotate(K, np.arange(L), f, "half", 1.0, host(wk), 1e-6, 0.0)
            q64, q_size = D.norm_rotate(Q, np.arange(L), f, "half", 1.0, host(wq), 1e-6, 0.0)
            at = np.arange(L)
            pg, r = S.places(table, s, at, page, n_pages)
            there = pg >= 0
            assert there[max(0, L - 51):].all() and there[:5].all() and (L < 90 or not there.all())
            got_k, got_v = host(ck[l])[pg[there], :, r[there]].swapaxes(0, 1), host(cv[l])[pg[there], :, r[there]].swapaxes(0, 1)
            assert within(got_k, k64[:, there], D.norm_bar(k64, k_size, dtype)[:, there]) and np.array_equal(got_v, V[:, there])
            # the outputs: keys and queries are off by their bars, scores by what that makes of them; the weights' sum of changes is at
            # most 2 max |change of a score| of the mean of |V|
            kb, qb = D.norm_bar(k64, k_size, dtype), D.norm_bar(q64, q_size, dtype)
            one = lambda c: c.reshape(1, *c.shape).astype(np.float64)
            want, _, bar, _ = S.attend(q64, one(k64), one(V), np.zeros((1, 1), dtype=int), np.array([0, L]), np.array([L]), spec, scale, True, dtype, once)
            for h in range(Hq):
                g = h // G
                off = scale * (np.abs(q64[h]) @ kb[g].T + qb[h] @ np.abs(k64[g]).T + qb[h] @ kb[g].T).max(1)
                share = np.abs(V[g]).max(0)
                assert (np.abs(out[h] - want[h]) <= bar[h] + 2 * off[:, None] * share).all()
