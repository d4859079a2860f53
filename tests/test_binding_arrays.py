"""What the binding hands to the library for arrays of the batch that are no plain rows of memory: the calls run on CPU tensors against a
library that keeps their parameter blocks and enqueues nothing."""
import ctypes
import os
import types

import pytest
import torch

from paper_2605_15508_amd import binding, build


class Device(torch.Tensor):
    """A CPU tensor that the binding takes for one on the GPU."""
    is_cuda = property(lambda self: True)


def dev(t):
    return t.as_subclass(Device)


@pytest.fixture(scope="module")
def library():
    if not os.path.exists(binding.library_path()):
        build.build(force=True)
    return binding.load_library()


@pytest.fixture
def blocks(monkeypatch):
    """The parameter blocks of the calls made, in order."""
    seen = []

    def call(ref, *_):
        seen.append(ref._obj)
        return 0

    names = [n for n in binding.EXPORTS if n.startswith("sts_")]
    lib = types.SimpleNamespace(**{n: (lambda *_: 256) if n.endswith("_bytes") else call for n in names})
    monkeypatch.setattr(binding, "load_library", lambda: lib)
    monkeypatch.setattr(binding, "_current", lambda device: None)
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    monkeypatch.setattr(binding, "_workspace", lambda tag, nbytes, device: torch.empty(max(nbytes, 256), dtype=torch.uint8))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    return seen


def arrays(B, Hq=4, Hkv=2, N=40, d=64, Tq=3):
    q = dev(torch.zeros(B, Tq, Hq, d, dtype=torch.bfloat16))
    k, v = (dev(torch.zeros(B, Hkv, N, d, dtype=torch.bfloat16)) for _ in range(2))
    codes, scales = (dev(torch.zeros(B, Hkv, N, 2, n, dtype=torch.uint8)) for n in (d // 2, d // 32))
    return q, k, v, codes, scales


def with_lists(B, **kw):
    """The calls that take lists."""
    q, k, v, codes, scales = arrays(B)
    return [lambda **more: binding.sts_sparse_attn(q, k, v, scale=0.1, want_lse=False, **kw, **more), lambda **more: binding.sts_packed_attn(q, codes, scales, 0.1, want_lse=False, **kw, **more)]


def last_read(t, stride_b, B):
    """The bytes behind a tensor's address up to the end of batch element B - 1's rows, as the library reads them, and what the tensor has."""
    row = t.shape[1:].numel()
    return t.element_size() * ((B - 1) * stride_b + row), t.untyped_storage().nbytes() - t.storage_offset() * t.element_size()


@pytest.mark.parametrize("B", [1, 2, 5])
def test_lists_and_counts_are_read_where_they_are(blocks, B):
    wide, counts = dev(torch.zeros(B, 12, 7, dtype=torch.int32)), dev(torch.zeros(B, 12, dtype=torch.int32))
    for idx, cnt in ((wide[:, :4].contiguous(), counts[:, :4].contiguous()), (wide[:, 4:8], counts[:, 8:])):
        for call in with_lists(B, indices=idx, counts=cnt):
            for prepare in (False, True):
                before = len(blocks)
                r = call(prepare=prepare)
                if prepare:
                    r()
                assert len(blocks) == before + 1
                p = blocks[-1]
                assert (p.indices, p.counts, p.kmax) == (idx.data_ptr(), cnt.data_ptr(), 7)
                for t, stride, plain in ((idx, p.idx_stride_b, 4 * 7), (cnt, p.cnt_stride_b, 4)):
                    assert B == 1 or (stride or plain) == t.stride(0)              # (0: "not given")
                    end, there = last_read(t, stride or plain, B)
                    assert end <= there


@pytest.mark.parametrize("B", [2, 5])
@pytest.mark.parametrize("prepare", [False, True])
def test_one_list_for_the_whole_batch_is_refused(blocks, B, prepare):
    """A batch stride of 0 means "not given" to the library, which would read behind the tensor's end."""
    idx, cnt = (dev(torch.zeros(1, 4, *n, dtype=torch.int32)) for n in ((7,), ()))
    shared_idx, shared_cnt = idx.expand(B, -1, -1), cnt.expand(B, -1)
    for kw in (dict(indices=shared_idx), dict(indices=shared_idx.contiguous(), counts=shared_cnt), dict(indices=shared_idx, counts=shared_cnt.contiguous())):
        for call in with_lists(B, **kw):
            with pytest.raises(AssertionError, match="contiguous"):
                call(prepare=prepare)
    assert not blocks
    for call in with_lists(B, indices=shared_idx.contiguous(), counts=shared_cnt.contiguous()):
        call()
    for call in with_lists(1, indices=shared_idx[:1], counts=shared_cnt[:1]):          # one batch element has no batch stride
        call()
    for call in with_lists(B, indices=dev(torch.zeros(1, 4, 0, dtype=torch.int32)).expand(B, -1, -1)):          # lists without entries are not read
        call()
    assert len(blocks) == 6


@pytest.mark.parametrize("B", [1, 2, 5])
def test_lengths_with_gaps_are_refused(blocks, B):
    """The library reads B neighbouring words."""
    q, k, v, codes, scales = arrays(B)
    scores = dev(torch.zeros(B, 4, 3, 40))
    pages, table = (dev(torch.zeros(5 * B, 2, 8, 64, dtype=torch.bfloat16)) for _ in range(2)), dev(torch.zeros(B, 5, dtype=torch.int32))
    kp, vp = pages
    calls = [lambda n, **kw: binding.sts_select(scores, [0, 1, 2, 3], 5, seq_lens=n, **kw),
             lambda n, **kw: binding.sts_dense_attn(q, k, v, 0.1, seq_lens=n, want_lse=False, **kw),
             lambda n, **kw: binding.sts_dense_attn(q, kp, vp, 0.1, seq_lens=n, want_lse=False, page_size=8, block_table=table, N=40, **kw),
             lambda n, **kw: binding.sts_packed_attn(q, codes, scales, 0.1, seq_lens=n, want_lse=False, **kw),
             lambda n, **kw: binding.sts_window_attn(q, k, v, 0.1, 9, seq_lens=n, want_lse=False, **kw)]
    plain = dev(torch.zeros(B, dtype=torch.int32))
    for call in calls:
        for kw in ({}, {"prepare": True}):
            r = call(plain, **kw)
            if kw:
                r()
            assert blocks.pop().seq_lens == plain.data_ptr() and not blocks
            for n in (dev(torch.zeros(1, dtype=torch.int32)).expand(B), dev(torch.zeros(2 * B, dtype=torch.int32))[::2]):
                if B == 1:           # one length has no gaps
                    call(n, **kw)
                    continue
                with pytest.raises(AssertionError):
                    call(n, **kw)
            blocks.clear()


@pytest.mark.parametrize("prepare", [False, True])
def test_lists_of_an_empty_batch_and_lists_without_entries(library, blocks, prepare):
    """A tensor without elements has no address; the call is one with lists all the same."""
    lists = dev(torch.zeros(0, 4, 7, dtype=torch.int32)), dev(torch.zeros(0, 4, dtype=torch.int32))
    calls = [*with_lists(0, indices=lists[0]), *with_lists(0, indices=lists[0], counts=lists[1], head_map=[0, 0, 1, 1])]
    for B in (0, 2):
        calls += with_lists(B, indices=dev(torch.zeros(B, 4, 0, dtype=torch.int32)), head_map=[0, 0, 1, 1])
    for call in calls:
        r = call(prepare=prepare)
        if prepare:
            r()
        p = blocks.pop()
        assert not blocks and (p.indices or isinstance(p, binding.AttnParams))           # sts_sparse_attn is one by its name
        if p.B == 0:           # and what the library makes of it: nothing to do
            f = library.sts_sparse_attn if isinstance(p, binding.AttnParams) else library.sts_packed_attn
            assert f(ctypes.byref(p), None) == 0


@pytest.mark.parametrize("big", [2 ** 31, 2 ** 32, 2 ** 32 + 16, 10 ** 12, 2 ** 64])
def test_numbers_beyond_32_bits_do_not_wrap(library, blocks, big):
    """A window or sinks beyond any cache mean all of it; negative ones, and page sizes, are refused as smaller ones are."""
    q, k, v, codes, scales = arrays(2)
    rows = dev(torch.zeros(2, 3, 2, 64, dtype=torch.bfloat16))
    binding.sts_window_attn(q, k, v, 0.1, big, sinks=big, want_lse=False)
    assert (blocks[-1].window, blocks[-1].sinks) == (2 ** 31 - 1, 2 ** 31 - 1)
    binding.sts_window_attn(q, k, v, 0.1, -big, sinks=-big, want_lse=False)
    assert blocks[-1].window < 0 and blocks[-1].sinks < 0
    calls = [(lambda: binding.sts_window_attn(q, k, v, 0.1, 9, page_size=big, want_lse=False), library.sts_window_attn),
             (lambda: binding.sts_packed_attn(q, codes, scales, 0.1, page_size=big, want_lse=False), library.sts_packed_attn),
             (lambda: binding.sts_packed_store(rows, rows, codes, scales, page_size=big), library.sts_packed_store),
             (lambda: binding.sts_packed_load(codes, scales, 3, page_size=big, out=(rows, rows)), library.sts_packed_load)]
    for call, f in calls:
        call()
        p = blocks.pop()
        assert (p.cache if hasattr(p, "cache") else p).page_size == 2 ** 31 - 1
        assert f(ctypes.byref(p), None) == -2          # not supported: found before anything is enqueued


def test_scratch_that_is_not_on_the_device_is_refused(blocks):
    q, k, v, codes, scales = arrays(2)
    elsewhere = torch.empty(1 << 20, dtype=torch.uint8, device="meta")
    gaps = torch.empty(1 << 20, dtype=torch.uint8)[::2]
    for ws in (elsewhere, gaps):
        for prepare in (False, True):
            with pytest.raises(AssertionError):
                binding.sts_window_attn(q, k, v, 0.1, 9, want_lse=False, workspace=ws, prepare=prepare)
            with pytest.raises(AssertionError):
                binding.sts_packed_attn(q, codes, scales, 0.1, want_lse=False, workspace=ws, prepare=prepare)
    assert not blocks
