"""Refusals of the calls for generation with drafted tokens (CPU only: nothing here launches a kernel)."""
import ctypes

import numpy as np
import pytest
import torch

import drafts_oracle as D
import paper_2502_01659_amd as sga
from paper_2502_01659_amd import binding as B
from sga_inputs import MaskSpec, KIND_BIGBIRD, KIND_DILATED, KIND_GLOBAL_LOCAL, KIND_SLIDING
from test_serving_args import OK, OnDevice, batch, desc, rows

SPEC = MaskSpec(KIND_SLIDING, 64, window=8)


def norm(**k):
    f = dict(struct_bytes=ctypes.sizeof(B._NormDesc), weight_dtype=1, weight=OK, epsilon=1e-6, offset=0.0)
    f.update(k)
    return B._NormDesc(*f.values())


def pool(**k):
    f = dict(struct_bytes=ctypes.sizeof(B._PagePool), reserved=0, pages=OK, state=OK)
    f.update(k)
    return B._PagePool(*f.values())


def tree(**k):
    f = dict(struct_bytes=ctypes.sizeof(B._DraftTree), words=2, depth=OK, seen=OK)
    f.update(k)
    return B._DraftTree(*f.values())


BAD_NORMS = (dict(struct_bytes=8), dict(weight_dtype=3), dict(weight_dtype=-1), dict(epsilon=0.0), dict(epsilon=-1.0), dict(epsilon=float("nan")),
             dict(epsilon=float("inf")), dict(weight=OK + 1))
BAD_TREES = (dict(struct_bytes=8), dict(words=0), dict(words=17), dict(depth=None), dict(seen=None), dict(depth=OK + 2), dict(seen=OK + 2))


def test_pages_argument_errors():
    need = sga.sga_pages_workspace_bytes(batch())
    assert need[0] == 0 and need[1] > 0

    def call(b=batch(), n=batch(), p=pool(), state=OK, ask=OK, kept=None, spec=SPEC, positions=None, slots=None, ws=OK, size=1 << 20):
        return sga.sga_pages_advance(b, n, p, state, ask, kept, spec, positions, slots, ws, size, None)
    for bad in (dict(b=None), dict(n=None), dict(p=None), dict(state=None), dict(ask=None), dict(state=OK + 4), dict(ask=OK + 2), dict(kept=OK + 2),
                dict(positions=OK + 4), dict(slots=OK + 4), dict(ws=OK + 16), dict(ws=None), dict(spec=MaskSpec(KIND_SLIDING, 0, window=1)),
                dict(p=pool(struct_bytes=0)), dict(p=pool(reserved=1)), dict(p=pool(pages=None)), dict(p=pool(state=None)),
                dict(p=pool(pages=OK + 2)), dict(p=pool(state=OK + 4))):
        assert call(**bad) == -1, bad
    for field, value in (("n_seqs", 3), ("n_tokens", 9), ("n_pages", 11), ("page_size", 8), ("pages_per_seq", 5), ("struct_bytes", 0),
                         ("page_table", None), ("seq_ptr", None), ("seq_len", OK + 2)):
        assert call(n=batch(**{field: value})) == -1, field
    for field, value in (("n_seqs", 65537), ("n_seqs", -1), ("page_size", 0), ("n_pages", 0), ("seq_ptr", None), ("page_table", None)):
        assert call(b=batch(**{field: value}), n=batch(**{field: value})) == -1, field
    assert call(b=batch(n_tokens=0, page_table=None), n=batch(n_tokens=0)) == -1            # sequences are read also where no row has room
    assert call(spec=MaskSpec(KIND_DILATED, 64, window=2, stride=2)) == -2 and call(spec=MaskSpec(KIND_BIGBIRD, 64, block=4)) == -2
    assert call(size=need[1] - 1) == -3 and call(ws=None, size=0) == -3
    assert sga.sga_pages_workspace_bytes(batch(n_seqs=65537))[0] == -1 and sga.sga_pages_workspace_bytes(None)[0] == -1
    assert sga.sga_pages_workspace_bytes(batch(n_seqs=65536, pages_per_seq=4096))[1] < 1 << 23


def test_norm_argument_errors():
    def call(Q=rows(), Q_out=rows(0x8000), qn=norm(), Hq=2, K=None, K_out=None, kn=None, Hkv=0, positions=None, L=4, d=64, r=desc(), dtype=1):
        return sga.sga_norm_rotary(Q, Q_out, qn, Hq, K, K_out, kn, Hkv, positions, 0, L, d, r, dtype, None)
    two = dict(K=rows(0x10000), K_out=rows(0x20000), Hkv=1)
    assert call(L=0) == 0 and call(L=0, Q=rows(None), Q_out=rows(None), r=None) == 0 and call(L=0, **two) == 0
    for bad in (dict(Q=None), dict(Q_out=None), dict(Q=rows(None)), dict(L=-1), dict(L=1 << 31), dict(Hq=0), dict(Hq=65536), dict(d=1), dict(d=1025),
                dict(d=62), dict(dtype=3), dict(qn=None, r=None), dict(K=rows()), dict(K_out=rows()), dict(kn=norm()), dict(positions=OK + 4),
                dict(Q=rows(OK + 1)), dict(Q_out=rows(OK, head=128)), dict(two, Hkv=0), dict(two, K_out=rows(0x8000)), dict(two, K=rows(None)),
                dict(two, K_out=rows(0x10000, row=256)), dict(r=desc(channels=63)), dict(r=desc(struct_bytes=1))):
        assert call(**bad) == -1, bad
    for bad in BAD_NORMS:
        assert call(qn=norm(**bad)) == -1 and call(kn=norm(**bad), **two) == -1, bad


def test_norm_gradient_argument_errors():
    def call(Q=rows(), g=rows(0x8000), dQ=rows(0x10000), qn=norm(), dw=None, Hq=2, K=None, gk=None, dK=None, kn=None, dwk=None, Hkv=0,
             positions=None, L=4, d=64, r=desc(), dtype=1, ws=None, size=0):
        return sga.sga_norm_rotary_backward(Q, g, dQ, qn, dw, Hq, K, gk, dK, kn, dwk, Hkv, positions, 0, L, d, r, dtype, ws, size, None)
    two = dict(K=rows(0x20000), gk=rows(0x30000), dK=rows(0x40000), Hkv=1, kn=norm())
    assert call(L=0) == 0 and call(L=0, **two) == 0
    for bad in (dict(Q=None), dict(g=None), dict(dQ=None), dict(Q=rows(None)), dict(L=-1), dict(L=1 << 31), dict(Hq=0), dict(d=1), dict(d=1025),
                dict(dtype=-1), dict(qn=None, r=None), dict(K=rows()), dict(dK=rows()), dict(gk=rows()), dict(kn=norm()), dict(dwk=OK),
                dict(qn=None, dw=OK), dict(qn=norm(weight=None), dw=OK), dict(dw=OK + 2), dict(dQ=rows(OK, head=128)), dict(dQ=rows(0x8000, row=64)),
                dict(two, K=None), dict(two, dK=rows(0x10000)), dict(two, Hkv=0), dict(two, dw=OK, dwk=OK, ws=OK, size=1 << 20),
                dict(ws=None, size=8), dict(ws=OK + 8, size=1 << 20), dict(positions=OK + 4), dict(g=rows(OK + 1))):
        assert call(**bad) == -1, bad
    for bad in BAD_NORMS:
        assert call(qn=norm(**bad)) == -1
    need = sga.sga_norm_workspace_bytes(4, 2, 0, 64)
    assert need[0] == 0 and need[1] >= 64 * 4
    assert call(dw=OK) == -3 and call(dw=OK, ws=OK, size=need[1] - 1) == -3
    for bad in ((-1, 2, 0, 64), (4, 0, 0, 64), (4, 2, -1, 64), (4, 2, 1, 1), (4, 2, 1, 1025), (1 << 31, 2, 1, 64)):
        assert sga.sga_norm_workspace_bytes(*bad)[0] == -1
    assert sga.sga_norm_workspace_bytes((1 << 31) - 1, 32, 8, 128)[1] < 1 << 21                # a few sums, however many rows


def test_outs_that_are_the_other_input():
    """What one tensor's rows are written to must not be what the other's are read from: rows run in any order."""
    a, b, c, d = (rows(x) for x in (0x10000, 0x20000, 0x30000, 0x40000))

    def forward(Q=a, Q_out=b, K=c, K_out=d):
        return sga.sga_norm_rotary(Q, Q_out, norm(), 2, K, K_out, norm(), 2, None, 0, 4, 64, desc(), 1, None)
    for bad in (dict(Q_out=c), dict(K_out=a), dict(Q_out=c, K_out=a), dict(K=a, Q_out=a), dict(K=a, K_out=a), dict(K=a, Q_out=a, K_out=a)):
        assert forward(**bad) == -1, bad
    e, f = rows(0x50000), rows(0x60000)

    def back(Q=a, g=b, dQ=c, K=d, gk=e, dK=f, qn=norm(), kn=norm()):
        return sga.sga_norm_rotary_backward(Q, g, dQ, qn, None, 2, K, gk, dK, kn, None, 2, None, 0, 4, 64, desc(), 1, None, 0, None)
    for bad in (dict(dQ=d), dict(dQ=e), dict(dK=a), dict(dK=b), dict(gk=b, dQ=b), dict(gk=b, dK=b), dict(K=a, dQ=a), dict(dQ=e, kn=None), dict(dK=b, qn=None)):
        assert back(**bad) == -1, bad

    def append(K=a, V=b, Q=c, Q_out=d):
        return sga.sga_cache_append_normed(K, V, OK, 0x4000, batch(), 2, 64, desc(), norm(), Q, Q_out, 4, norm(), None, 1, None)
    for bad in (dict(Q_out=a), dict(Q_out=b), dict(Q=a, Q_out=a)):
        assert append(**bad) == -1, bad


def test_tree_argument_errors():
    def call(parent=OK, b=batch(), spec=SPEC, t=tree()):
        return sga.sga_draft_tree_build(parent, b, spec, t, None)
    assert call(b=batch(n_tokens=0)) == 0 and call(b=batch(n_seqs=0)) == 0
    for bad in (dict(parent=None), dict(parent=OK + 2), dict(b=None), dict(t=None), dict(b=batch(struct_bytes=0)), dict(b=batch(seq_ptr=None)),
                dict(spec=MaskSpec(KIND_SLIDING, 64, window=-1))):
        assert call(**bad) == -1, bad
    for bad in BAD_TREES:
        assert call(t=tree(**bad)) == -1, bad
    assert call(spec=MaskSpec(KIND_BIGBIRD, 64, block=4)) == -2


def test_append_normed_argument_errors():
    def call(K=rows(), V=rows(), ck=OK, cv=0x4000, b=batch(), Hkv=2, d=64, r=desc(), kn=norm(), Q=None, Q_out=None, Hq=0, qn=None, t=None, dtype=1):
        return sga.sga_cache_append_normed(K, V, ck, cv, b, Hkv, d, r, kn, Q, Q_out, Hq, qn, t, dtype, None)
    assert call(b=batch(n_tokens=0)) == 0 and call(b=batch(n_seqs=0), t=tree()) == 0
    q = dict(Q=rows(), Q_out=rows(), Hq=4)
    for bad in (dict(K=None), dict(V=rows(None)), dict(ck=None), dict(cv=OK), dict(cv=OK + 1), dict(b=None), dict(Hkv=0), dict(d=1), dict(dtype=5),
                dict(Q=rows()), dict(Q_out=rows()), dict(qn=norm()), dict(q, r=None), dict(q, Hq=0), dict(q, Q_out=rows(head=32)),
                dict(r=desc(channels=128))):
        assert call(**bad) == -1, bad
    for bad in BAD_NORMS:
        assert call(kn=norm(**bad)) == -1 and call(qn=norm(**bad), **q) == -1
    for bad in BAD_TREES:
        assert call(t=tree(**bad)) == -1


def test_attention_tree_argument_errors():
    spec = MaskSpec(KIND_SLIDING, 64, window=64)

    def call(Q=rows(), ck=OK, cv=OK, b=batch(), t=tree(), mask=spec, O=rows(0x8000), Hq=4, Hkv=2, d=64, dtype=1, lse=None, ws=None, n=0):
        return sga.sga_attention_tree(Q, ck, cv, b, t, mask, O, Hq, Hkv, d, 0.1, dtype, lse, ws, n, None)
    assert call(b=batch(n_tokens=0)) == 0 and call(b=batch(n_seqs=0)) == 0
    for bad in (dict(Q=None), dict(O=None), dict(t=None), dict(ck=None), dict(cv=OK + 8), dict(Hq=3), dict(dtype=4), dict(O=rows(OK)), dict(lse=OK + 2),
                dict(ws=OK + 16, n=100), dict(mask=MaskSpec(KIND_SLIDING, 0, window=2))):
        assert call(**bad) == -1, bad
    for bad in BAD_TREES:
        assert call(t=tree(**bad)) == -1
    assert call(d=48) == -2 and call(mask=MaskSpec(KIND_BIGBIRD, 64, block=4)) == -2
    assert call(b=batch(n_tokens=(1 << 31) - 1), Hq=64, Hkv=1) == -4
    size = lambda t: sga.sga_tree_workspace_bytes(batch(n_seqs=1, n_tokens=4, pages_per_seq=4096), MaskSpec(KIND_SLIDING, 65536, window=65536), t, 4, 2, 64, 1)
    assert size(tree())[0] == 0 and size(tree())[1] > 0
    assert size(None)[0] == -1 and size(tree(words=0))[0] == -1


def test_keep_argument_errors():
    def call(ck=OK, cv=0x4000, b=batch(), Hkv=2, d=64, layers=1, apart=0, path=OK, columns=4, count=OK, dtype=1):
        return sga.sga_cache_keep(ck, cv, b, Hkv, d, layers, apart, path, columns, count, dtype, None)
    assert call(b=batch(n_tokens=0)) == 0 and call(b=batch(n_seqs=0)) == 0 and call(columns=0) == 0
    for bad in (dict(ck=None), dict(cv=None), dict(cv=OK), dict(ck=OK + 1), dict(b=None), dict(Hkv=0), dict(d=1), dict(d=2000), dict(layers=0),
                dict(layers=2, apart=2 * 16 * 64 - 1), dict(path=None), dict(count=None), dict(path=OK + 2), dict(count=OK + 2), dict(columns=-1),
                dict(dtype=3), dict(b=batch(page_stride=100))):
        assert call(**bad) == -1, bad
    assert call(layers=1 << 23, apart=1 << 20) == -4


def on_device(*shape, dtype=torch.int32):
    return OnDevice(torch.zeros(*shape, dtype=dtype))


def test_tensor_level_refusals_without_a_gpu():
    host = torch.zeros(4, dtype=torch.int32)
    for make in (lambda: sga.PagePool(host, torch.zeros(2, dtype=torch.int64)), lambda: sga.PagePool(on_device(4), on_device(2)),
                 lambda: sga.PagePool(on_device(4), on_device(3, dtype=torch.int64)), lambda: sga.Norm(torch.ones(4)),
                 lambda: sga.Norm(on_device(4, dtype=torch.float32), epsilon=0.0), lambda: sga.Norm(epsilon=float("inf")),
                 lambda: sga.Norm(on_device(2, 4, dtype=torch.float32)), lambda: sga.DraftTree(host, torch.zeros(4, 1, dtype=torch.int32)),
                 lambda: sga.DraftTree(on_device(4), on_device(4, 17)), lambda: sga.DraftTree(on_device(4), on_device(5, 1)),
                 lambda: sga.DraftTree(on_device(4, dtype=torch.int64), on_device(4, 1))):
        with pytest.raises(ValueError):
            make()
    with pytest.raises(TypeError):
        sga.Norm(on_device(4, dtype=torch.float64))
    for made in (sga.PagePool(on_device(4), on_device(2, dtype=torch.int64)), sga.Norm(on_device(4, dtype=torch.float16), offset=1.0),
                 sga.DraftTree(on_device(4), on_device(4, 2))):
        for name in list(made.__dict__):
            with pytest.raises(AttributeError):
                setattr(made, name, 7)


def test_the_oracle_of_pages():
    """By hand: pages of 4, a window of 4, one sequence of each kind."""
    table = np.array([[5, 6, 7, -1], [1, -1, -1, -1], [2, 3, -1, -1], [-1, -1, -1, -1]])
    ptr, length = np.array([0, 2, 3, 9, 9]), np.array([12, 4, 7, 0])
    ring, state = np.array([0, 0, 0, 0, 8, 9, 4, 0, 0, 0]), np.array([4, 3])
    # 0: keeps 1 of 2 rows (11 tokens), one more: nothing behind 11 - 4 = 7 but page 5.  1: all of its row, 5 more: two pages.  2: ends.
    # 3: 5 tokens are two pages, four needed up to it of three free.
    got = D.advance(table, ptr, length, ring, state, np.array([1, 5, -1, 5]), np.array([1, 1, 0, 0]), 20, 4, 10, MaskSpec(KIND_SLIDING, 99, window=4))
    assert got[0].tolist() == [[-1, 6, 7, -1], [1, 8, 9, -1], [-1] * 4, [-1] * 4]
    assert got[1].tolist() == [0, 1, 6, 6, 6] and got[2].tolist() == [12, 9, 0, 0]
    assert got[3].tolist() == [0, 0, 0, 0, 8, 9, 4, 5, 2, 3]
    assert got[4].tolist() == [6, 4]
    assert got[5][:7] == [11, 4, 5, 6, 7, 8, None] and got[6][:7] == [31, 32, 33, 34, 35, 36, None]


def test_the_oracle_of_trees():
    up = D.paths([-1, 0, 0, 2, -1, 9, 3])
    assert up == [[0], [1, 0], [2, 0], [3, 2, 0], [4], [5], [6, 3, 2, 0]]
    spec = MaskSpec(KIND_GLOBAL_LOCAL, 100, window=1, n_global=11)
    depth, seen = D.tree(np.array([-1, 0, 0, 2, -1, 9, 3]), [0, 7], [17], spec, 1)
    assert depth == [0, 1, 1, 2, 0, 0, 3] and seen[6] == {6, 3, 0} and seen[3] == {3, 2, 0}      # token 0 is at position 10: global
