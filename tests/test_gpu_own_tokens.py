"""Own tokens of a block (k_new, v_new) whose numbers are none, over every kind of cache and however many workgroups share it."""
import math

import pytest
import torch

import paper_2605_15508_amd as sts
from cache_util import packed_cache

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def calls(B, Tq, Hq, Hkv, N, d, g, lens):
    """The attention calls that take own tokens, over caches of their own with `lens` cached tokens: {name: f(q, kn, vn) -> out, lse on the CPU}."""
    k, v = (torch.randn(B, Hkv, N, d, generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    codes, scales = (t.to(DEV) for t in packed_cache(B, Hkv, N, d, g)[:2])
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    lists = dict(indices=torch.arange(N, dtype=torch.int32, device=DEV).expand(B, Hq, N).contiguous(), counts=n[:, None].expand(B, Hq).contiguous())
    forms = {"sparse": lambda q, **kw: sts.sts_sparse_attn(q, k, v, scale=0.1, **lists, **kw), "dense": lambda q, **kw: sts.sts_dense_attn(q, k, v, 0.1, seq_lens=n, **kw),
             "packed": lambda q, **kw: sts.sts_packed_attn(q, codes, scales, 0.1, seq_lens=n, **kw),
             "packed lists": lambda q, **kw: sts.sts_packed_attn(q, codes, scales, 0.1, **lists, **kw),
             "window": lambda q, **kw: sts.sts_window_attn(q, k, v, 0.1, 10 ** 6, seq_lens=n, **kw)}

    def run(f):
        return lambda q, kn, vn: [t.cpu() for t in f(q.to(DEV), k_new=kn.to(DEV), v_new=vn.to(DEV), out_dtype=torch.float32)[:2]]
    return {name: run(f) for name, f in forms.items()}


@pytest.mark.parametrize("N", [40, 520, 600, 3000, 20000])
@pytest.mark.parametrize("Tq,bad", [(1, [0]), (3, [0]), (3, [2]), (4, [1, 2])])
@pytest.mark.parametrize("d", [64, 128])
def test_own_keys_that_are_no_numbers(d, Tq, bad, N):
    """Rows that see one are NaN, whatever else they see, nothing included; the others are as without."""
    B, Hq, Hkv = 3, 4, 2
    g = torch.Generator().manual_seed(N + Tq)
    q, kn, vn = (torch.randn(B, Tq, h, d, generator=g).to(torch.bfloat16) for h in (Hq, Hkv, Hkv))
    odd = kn.clone()
    odd[:, bad, 1, 5] = math.nan
    first = min(bad)
    for name, call in calls(B, Tq, Hq, Hkv, N, d, g, [0, 1, N]).items():
        want, got = call(q, kn, vn), call(q, odd, vn)
        assert torch.isfinite(want[0]).all(), name
        assert torch.isnan(got[0][:, first:, 2:]).all(), name
        assert not torch.isfinite(got[1][:, 2:, first:]).any(), name
        assert torch.equal(got[0][:, :, :2], want[0][:, :, :2]) and torch.equal(got[1][:, :2], want[1][:, :2]), name
        assert torch.equal(got[0][:, :first], want[0][:, :first]) and torch.equal(got[1][..., :first], want[1][..., :first]), name


@pytest.mark.parametrize("Tq,N", [(1, 40), (1, 3000), (4, 500), (4, 20000), (40, 300), (40, 2000)])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_are_no_numbers_have_no_logarithm(d, Tq, N):
    """A cached key that is NaN: the rows that see it are NaN, and their lse is -inf, from one workgroup or several."""
    Hq, Hkv = 4, 2
    g = torch.Generator().manual_seed(N + Tq)
    q = torch.randn(1, Tq, Hq, d, generator=g).to(torch.bfloat16).to(DEV)
    k, v = (torch.randn(1, Hkv, N, d, generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    codes, scales = (t.to(DEV) for t in packed_cache(1, Hkv, N, d, g)[:2])
    bad = N - 2
    k[:, 1, bad, 0] = math.nan
    scales[:, 1, bad, 0, 0] = 255
    idx = torch.arange(N, dtype=torch.int32, device=DEV).expand(1, Hq, N).contiguous()
    p = torch.arange(N - Tq, N)
    calls = {"window": (sts.sts_window_attn(q, k, v, 0.1, N), p >= bad), "short window": (sts.sts_window_attn(q, k, v, 0.1, 17), p >= bad)}
    if Tq <= 16:
        every = torch.ones(Tq, dtype=torch.bool)
        calls.update({"packed": (sts.sts_packed_attn(q, codes, scales, 0.1), every), "lists": (sts.sts_packed_attn(q, codes, scales, 0.1, indices=idx), every),
                      "sparse": (sts.sts_sparse_attn(q, k, v, idx, 0.1), every), "dense": (sts.sts_dense_attn(q, k, v, 0.1)[:2], every)})
    for name, ((o, l), hit) in calls.items():
        o, l = o.cpu(), l.cpu()
        assert torch.isnan(o[:, hit, 2:]).all() and torch.isneginf(l[:, 2:, hit]).all(), name
        assert torch.isfinite(o[:, :, :2]).all() and torch.isfinite(l[:, :2]).all(), name
        assert torch.isfinite(o[:, ~hit]).all() and torch.isfinite(l[..., ~hit]).all(), name
