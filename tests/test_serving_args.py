"""Refusals of the serving calls and the frequencies' formulas (CPU only: nothing here launches a kernel)."""
import ctypes
import math

import pytest
import torch

import paper_2502_01659_amd as sga
from paper_2502_01659_amd import binding as B
from sga_inputs import MaskSpec, KIND_BIGBIRD, KIND_DILATED, KIND_GLOBAL_LOCAL, KIND_NONLOCAL, KIND_SLIDING

OK = 0x1000        # any non-null aligned address: validation fails before it is used


def rows(data=OK, head=64, row=128):
    return B._Rows(data, head, row)


def desc(**k):
    f = dict(struct_bytes=ctypes.sizeof(B._RotaryDesc), layout=0, channels=64, magnitude=1.0, frequencies=OK)
    f.update(k)
    return B._RotaryDesc(*f.values())


def batch(**k):
    f = dict(struct_bytes=ctypes.sizeof(B._PagedBatch), n_seqs=2, n_tokens=8, n_pages=10, page_stride=2 * 16 * 64, page_size=16,
             pages_per_seq=4, page_table=OK, seq_ptr=OK, seq_len=OK)
    f.update(k)
    return B._PagedBatch(*f.values())


def test_rotary_argument_errors():
    def call(X=rows(), Y=rows(0x8000), positions=None, L=4, H=2, d=64, r=desc(), dtype=1):
        return sga.sga_rotary(X, Y, positions, 0, L, H, d, r, 0, dtype, None)
    assert call(L=0) == 0                                     # no row: nothing to do, no GPU needed
    assert call(X=rows(None), Y=rows(None), L=0) == 0
    assert call(X=None) == -1 and call(Y=None) == -1 and call(X=rows(None)) == -1 and call(Y=rows(None)) == -1
    assert call(L=-1) == -1 and call(L=1 << 31) == -1 and call(H=0) == -1 and call(H=65536) == -1
    assert call(d=1) == -1 and call(d=1025) == -1 and call(d=62) == -1       # channels beyond the head
    assert call(dtype=3) == -1 and call(dtype=-1) == -1
    assert call(r=None) == -1
    for bad in (dict(struct_bytes=8), dict(layout=2), dict(channels=0), dict(channels=63), dict(channels=66), dict(frequencies=None),
                dict(frequencies=OK + 4)):
        assert call(r=desc(**bad)) == -1
    assert call(X=rows(OK + 1)) == -1 and call(X=rows(OK + 2), dtype=0) == -1 and call(positions=OK + 4) == -1
    assert call(Y=rows(OK, head=128)) == -1                   # in place with other strides


def test_append_argument_errors():
    def call(K=rows(), V=rows(), ck=OK, cv=0x4000, b=batch(), Hkv=2, d=64, r=desc(), Q=None, Q_out=None, Hq=0, dtype=1):
        return sga.sga_cache_append(K, V, ck, cv, b, Hkv, d, r, Q, Q_out, Hq, dtype, None)
    assert call(b=batch(n_tokens=0)) == 0 and call(b=batch(n_seqs=0)) == 0
    assert call(b=batch(n_tokens=0, page_table=None, seq_ptr=None, seq_len=None), K=rows(None), V=rows(None)) == 0
    assert call(K=None) == -1 and call(V=rows(None)) == -1 and call(ck=None) == -1 and call(cv=OK + 1) == -1
    assert call(cv=OK) == -1                                  # keys and values in one place
    assert call(b=None) == -1 and call(Hkv=0) == -1 and call(d=1) == -1 and call(dtype=5) == -1
    for bad in (dict(struct_bytes=0), dict(n_seqs=-1), dict(n_tokens=-1), dict(n_tokens=1 << 31), dict(n_pages=0),
                dict(n_pages=1 << 31), dict(page_size=0), dict(page_size=65537), dict(pages_per_seq=0),
                dict(page_size=65536, pages_per_seq=1 << 15, page_stride=1 << 40), dict(page_stride=2 * 16 * 64 - 1),
                dict(page_table=None), dict(seq_ptr=None), dict(seq_len=None), dict(seq_ptr=OK + 4), dict(page_table=OK + 2)):
        assert call(b=batch(**bad)) == -1, bad
    assert call(Q=rows()) == -1 and call(Q_out=rows()) == -1                  # one without the other
    assert call(Q=rows(), Q_out=rows(), Hq=0) == -1
    assert call(Q=rows(), Q_out=rows(), Hq=4, r=None) == -1                   # nothing would turn them
    assert call(Q=rows(), Q_out=rows(head=32), Hq=4) == -1
    assert call(r=desc(channels=128)) == -1


def test_attention_argument_errors():
    spec = MaskSpec(KIND_SLIDING, 64, window=64)

    def call(Q=rows(), ck=OK, cv=OK, b=batch(), mask=spec, O=rows(0x8000), Hq=4, Hkv=2, d=64, dtype=1, lse=None, ws=None, n=0):
        return sga.sga_attention_paged(Q, ck, cv, b, mask, 1, O, Hq, Hkv, d, 0.1, dtype, lse, ws, n, None)
    assert call(b=batch(n_tokens=0)) == 0 and call(b=batch(n_seqs=0)) == 0
    assert call(Q=None) == -1 and call(O=None) == -1 and call(Q=rows(None)) == -1 and call(O=rows(OK)) == -1
    assert call(ck=None) == -1 and call(cv=OK + 8) == -1 and call(Q=rows(OK + 8)) == -1 and call(O=rows(0x8000, row=129)) == -1
    assert call(Q=rows(head=4)) == -1                                         # 8 bytes
    assert call(Hq=3) == -1 and call(Hq=0) == -1 and call(Hkv=0) == -1 and call(Hq=65536, Hkv=1) == -1
    assert call(d=48) == -2 and call(d=512) == -2 and call(dtype=4) == -1
    assert call(mask=MaskSpec(KIND_DILATED, 64, window=2, stride=2)) == -2
    assert call(mask=MaskSpec(KIND_NONLOCAL, 64, window=2, n_global=1)) == -2
    assert call(mask=MaskSpec(KIND_BIGBIRD, 64, block=4)) == -2
    assert call(mask=MaskSpec(KIND_SLIDING, 0, window=2)) == -1 and call(mask=MaskSpec(KIND_SLIDING, 64, window=-1)) == -1
    assert call(mask=MaskSpec(KIND_GLOBAL_LOCAL, 64, window=2, n_global=-1)) == -1
    assert call(b=batch(page_stride=2 * 16 * 64 + 4)) == -1                   # pages off 16 bytes
    assert call(ws=OK + 16, n=100) == -1 and call(ws=None, n=100) == -1 and call(lse=OK + 2) == -1
    assert call(b=batch(n_tokens=(1 << 31) - 1), Hq=64, Hkv=1) == -4


def test_workspace_rule():
    def size(S, T, L, window, Hq=32, Hkv=8, d=128, columns=None):
        b = batch(n_seqs=S, n_tokens=T, pages_per_seq=columns or -(-L // 16), page_stride=Hkv * 16 * d)
        st, n = sga.sga_paged_workspace_bytes(b, MaskSpec(KIND_SLIDING, L, window=window), Hq, Hkv, d, 2)
        assert st == 0
        return n
    assert size(1, 1, 65536, 65536) > 0                       # one long sequence is split
    assert size(1, 1, 65536, 65536) < 1 << 25
    assert size(64, 64, 65536, 65536) == size(4096, 4096, 1 << 20, 1 << 20) < 1 << 24      # two tiles for each share
    assert size(4, 32768, 65536, 65536) == 0                  # tiles of 128 rows enough for the chip
    assert 0 < size(4, 1024, 65536, 65536) < 1 << 29
    assert size(1, 1, 256, 256, Hq=1, Hkv=1) == 0             # a short one is one share
    assert size(1, 1, 65536, 100, Hq=1, Hkv=1) == 0           # a narrow window too
    assert size(1, 1, 1 << 20, 1 << 20, Hq=1, Hkv=1, columns=4) == 0          # the page table holds 64 tokens
    assert sga.sga_paged_workspace_bytes(batch(n_tokens=0), MaskSpec(KIND_SLIDING, 64), 4, 2, 64, 1) == (0, 0)
    assert sga.sga_paged_workspace_bytes(batch(n_tokens=0), MaskSpec(KIND_SLIDING, 0), 4, 2, 64, 1)[0] == -1


def test_tensor_level_refusals_without_a_gpu():
    x = torch.zeros(2, 3, 64)
    with pytest.raises(ValueError):
        sga.Rotary(torch.ones(32, dtype=torch.float64))       # host memory
    with pytest.raises(ValueError):
        sga.PagedBatch(torch.zeros(1, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int64),
                       torch.zeros(1, dtype=torch.int32), 1, 16, 4)
    with pytest.raises(ValueError):
        sga.PagedBatch(torch.zeros(1, 4, dtype=torch.int64), torch.zeros(2, dtype=torch.int64),
                       torch.zeros(1, dtype=torch.int32), 1, 16, 4)
    with pytest.raises(ValueError):
        sga.rotary(x, None)
    with pytest.raises(TypeError):
        B._serving_code(torch.float64)
    with pytest.raises(ValueError):
        B._strides(x[:, :, ::2], "X")
    for bad in (torch.zeros(1, 3, 64).expand(2, 3, 64), torch.zeros(2, 1, 64).expand(2, 3, 64),
                torch.as_strided(torch.zeros(1000), (2, 3, 64), (64, 100, 1)), torch.as_strided(torch.zeros(1000), (2, 3, 64), (32, 200, 1))):
        B._strides(bad, "X")                                  # may be read
        with pytest.raises(ValueError):
            B._strides(bad, "out", written=True)
    for good in (x, x.transpose(0, 1), torch.zeros(3, 7, 80)[:, :2, :64].transpose(0, 1), torch.zeros(1, 1, 64)):
        B._strides(good, "out", written=True)


def test_rotary_frequencies():
    f, m = sga.rotary_frequencies(8, base=100.0, device="cpu")
    assert f.dtype == torch.float64 and m == 1.0
    assert torch.allclose(f, torch.tensor([100.0 ** (-2 * i / 8) for i in range(4)], dtype=torch.float64), rtol=1e-15)
    g, m = sga.rotary_frequencies(8, base=100.0, scaling="linear", factor=4.0, device="cpu")
    assert torch.allclose(g, f / 4, rtol=1e-15) and m == 1.0
    g, m = sga.rotary_frequencies(8, base=100.0, scaling="base", factor=4.0, device="cpu")
    assert g[0] == f[0] and abs(g[3] / f[3] - 0.25) < 1e-14 and m == 1.0
    g, m = sga.rotary_frequencies(128, scaling="parts", factor=8.0, original_length=8192, device="cpu")
    f, _ = sga.rotary_frequencies(128, device="cpu")
    turns = 8192 * f / (2 * math.pi)
    assert torch.equal(g[turns >= 32], f[turns >= 32]) and torch.allclose(g[turns <= 1], f[turns <= 1] / 8, rtol=1e-15)
    middle = (turns > 1) & (turns < 32)
    assert ((g < f) & (g > f / 8))[middle].all() and middle.any()
    assert abs(m - (1 + 0.1 * math.log(8.0))) < 1e-15
    for bad in (dict(channels=3), dict(channels=0), dict(channels=8, scaling="other"), dict(channels=8, factor=0.5),
                dict(channels=8, base=-1.0), dict(channels=2, scaling="base"), dict(channels=8, scaling="parts", factor=2.0),
                dict(channels=8, scaling="parts", original_length=100, slow_turns=4.0, fast_turns=2.0)):
        with pytest.raises(ValueError):
            sga.rotary_frequencies(device="cpu", **bad)


def test_calls_too_large_for_one_grid():
    spec = MaskSpec(KIND_SLIDING, 1 << 20, window=1024)
    def size(n, Hq, Hkv, d, dtype=1, n_seqs=2):
        return sga.sga_paged_workspace_bytes(batch(n_tokens=n, n_seqs=n_seqs, page_stride=Hkv * 16 * d), spec, Hq, Hkv, d, dtype)[0]
    assert size(1 << 25, 64, 64, 128) == -4                   # 2^24 tiles of 128 rows over all heads
    assert size((1 << 25) - (1 << 14), 64, 64, 128) == 0
    assert size((1 << 31) - 1, 8, 1, 32) == -4 and size((1 << 31) - 1, 1, 1, 64) == -4


class OnDevice:
    """A host tensor that says it lies on device 0: enough to make the records that calls hand to the library."""
    is_cuda, device = True, torch.device("cuda", 0)

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return 0

    def __iadd__(self, x):
        self.t += x
        return self


def test_a_batch_and_a_rotation_keep_what_they_were_made_of():
    """The records for the library hold addresses and sizes: nothing that they were made of can be replaced behind them."""
    table, ptr, length = (OnDevice(torch.zeros(n, dtype=t)) for n, t in (((2, 4), torch.int32), (3, torch.int64), (2, torch.int32)))
    b = sga.PagedBatch(table, ptr, length, 8, 16, 10)
    record = b._struct(2048)
    for name, other in (("page_table", OnDevice(torch.zeros(2, 9, dtype=torch.int32))), ("seq_ptr", OnDevice(torch.zeros(3, dtype=torch.int64))),
                        ("seq_len", OnDevice(length.t + 1)), ("n_tokens", 7), ("page_size", 32), ("n_pages", 11), ("device", None),
                        ("device_index", 1)):
        held = getattr(b, name)
        with pytest.raises(AttributeError, match=name):
            setattr(b, name, other)
        with pytest.raises(AttributeError, match=name):
            delattr(b, name)
        assert getattr(b, name) is held
    b.seq_len += 1                                            # written into: the same array
    assert b.seq_len is length and length.t.tolist() == [1, 1]
    for stride in (2048, 4096):
        r = b._struct(stride)
        assert (r.page_table, r.seq_ptr, r.seq_len) == (table.data_ptr(), ptr.data_ptr(), length.data_ptr())
        assert (r.n_tokens, r.n_pages, r.page_size, r.pages_per_seq, r.n_seqs, r.page_stride) == (8, 10, 16, 4, 2, stride)
    assert b._struct(2048) is record

    f = OnDevice(torch.ones(32, dtype=torch.float64))
    rot = sga.Rotary(f, magnitude=0.5)
    for name, other in (("frequencies", OnDevice(torch.ones(16, dtype=torch.float64))), ("channels", 32), ("_desc", None), ("device_index", 1)):
        with pytest.raises(AttributeError, match=name):
            setattr(rot, name, other)
        with pytest.raises(AttributeError, match=name):
            delattr(rot, name)
    assert (rot._desc.frequencies, rot._desc.channels, rot.channels) == (f.data_ptr(), 64, 64)


def test_workspace_of_long_chunks_that_are_not_cut():
    """A tile of 128 rows is cut into pieces of at least 1,024 keys and their cost: up to 1,279 keys there is nothing to join."""
    def size(keys, dtype, window=None):
        b = batch(n_seqs=2, n_tokens=400, pages_per_seq=-(-keys // 16), page_stride=8 * 16 * 128)
        st, n = sga.sga_paged_workspace_bytes(b, MaskSpec(KIND_SLIDING, keys, window=keys if window is None else window), 8, 8, 128, dtype)
        assert st == 0
        return n
    assert size(1279, 2) == 0 and size(1280, 2) > 0 and size(1279, 1) == 0
    assert size(65536, 2, window=500) == 0 and size(65536, 2, window=1200) > 0
    assert size(512, 0) == 0 and size(513, 0) > 0             # full precision: pieces of 256, from 513 keys on
