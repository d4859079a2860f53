"""sts_linear_attn where it can go wrong at the ends of what it takes: pools named by several tensors, values, scales and states far from 1, against
the recurrence in 64 bits within bounds derived from the roundings (layers_util.linear)."""
import math

import pytest
import torch

import paper_2605_15508_amd as sts
from layers_util import check_linear, linear, starts_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def data(n, Hq, Hkv, d, seed, size=1.0):
    g = torch.Generator().manual_seed(seed)
    q, k, v = (torch.randn(n, h, d, generator=g) for h in (Hq, Hkv, Hkv))
    return q.to(torch.bfloat16), k.to(torch.bfloat16), (v * size).to(torch.bfloat16), torch.rand(n, Hkv, generator=g)


@pytest.mark.parametrize("n", [5, 70])
def test_in_place_through_two_slices_of_a_pool(n):
    """A layer's states out of a wider pool, sliced anew for each argument: the sequences' own slots are written, and no others."""
    B, Hkv, d = 2, 2, 64
    q, k, v, r = data(B * n, 4, Hkv, d, 1)
    decay = -0.1 * r
    wide = torch.randn(3, 6, 2 * Hkv, d, d, generator=torch.Generator().manual_seed(2)).to(DEV)
    before = wide.clone()
    slots = torch.tensor([4, 1], dtype=torch.int32, device=DEV)
    out, _ = sts.sts_linear_attn(q.to(DEV), k.to(DEV), v.to(DEV), decay.to(DEV), 0.1, starts=starts_of([n, n]).to(DEV), max_len=n, state=wide[1, :, Hkv:], slots=slots,
                                 state_out=wide[1, :, Hkv:], out_dtype=torch.float32)
    for b, s in enumerate((4, 1)):
        at = slice(b * n, b * n + n)
        ref, all_s, e, e_s = linear(q[at], k[at], v[at], decay[at], 0.1, before[1, s, Hkv:].cpu(), n > 16)
        check_linear(out[at], ref, e, f"sequence {b}")
        check_linear(wide[1, s, Hkv:], all_s[-1], e_s[-1], f"state {b}")
        wide[1, s, Hkv:] = before[1, s, Hkv:]
    assert torch.equal(wide, before)


def spread(r, bits):
    """Decays that make up 2^-bits a chunk of 32 rows, by a tenth more or less for each row."""
    return -bits * math.log(2) / 32 * (0.9 + 0.2 * r)


@pytest.mark.parametrize("Hq", [2, 4])          # one head to a workgroup, or two
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bits", [5, 20, 29, 31, 40, 50, 59, 65])
@pytest.mark.parametrize("size", [1.0, 1e-20])
def test_small_values_and_strong_decays(size, bits, d, Hq):
    """Seven chunks, so that the factor that the state is held by takes many values. Nothing is added to the bound: sums on the way are at most 2^46
    smaller than the results, 2^-112 for these values, where fp32's numbers of less than 2^-126 still have steps of 2^-149."""
    n, Hkv = 224, 2
    q, k, v, r = data(n, Hq, Hkv, d, 3, size)
    decay = spread(r, bits)
    first = torch.randn(1, Hkv, d, d, generator=torch.Generator().manual_seed(4)) * size
    out, S = sts.sts_linear_attn(q.to(DEV), k.to(DEV), v.to(DEV), decay.to(DEV), 0.1, starts=starts_of([n]).to(DEV), max_len=n, state=first.to(DEV),
                                 state_out=torch.empty(1, Hkv, d, d, device=DEV), out_dtype=torch.float32)
    ref, all_s, e, e_s = linear(q, k, v, decay, 0.1, first[0], True)
    check_linear(out, ref, e, f"{size} {bits}")
    check_linear(S[0], all_s[-1], e_s[-1], f"{size} {bits} state")


@pytest.mark.parametrize("Hq", [2, 4])          # one head to a workgroup, or two
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bits", [0, 5, 29, 50])
@pytest.mark.parametrize("scale,size", [(1e14, 1.0), (1e25, 1.0), (1e30, 1.0), (-1e38, 1e-20), (1e-30, 1e20)])
def test_scales_of_all_sizes(scale, size, bits, d, Hq):
    """A factor of the results is multiplied with the scale: the product must not leave fp32's range where results do not."""
    n, Hkv = 100, 2
    q, k, v, r = data(n, Hq, Hkv, d, 5, size)
    decay = spread(r, bits)
    out, _ = sts.sts_linear_attn(q.to(DEV), k.to(DEV), v.to(DEV), decay.to(DEV), scale, starts=starts_of([n]).to(DEV), max_len=n, out_dtype=torch.float32)
    ref, _, e, _ = linear(q, k, v, decay, scale, torch.zeros(Hkv, d, d), True)
    assert ref.abs().max() < 1e38 * 3
    check_linear(out, ref, e, f"{scale}")
    blocks = [t[:9].view(1, 9, *t.shape[1:]).to(DEV) for t in (q, k, v, decay)]
    out, _ = sts.sts_linear_attn(*blocks, scale, out_dtype=torch.float32)
    ref, _, e, _ = linear(q[:9], k[:9], v[:9], decay[:9], scale, torch.zeros(Hkv, d, d), False)
    check_linear(out[0], ref, e, f"{scale} row by row")


@pytest.mark.parametrize("Hq", [2, 4])          # one head to a workgroup, or two
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,at", [(9, 4), (100, 0), (100, 40), (1000, 700)])
def test_minus_infinity_forgets_states_of_any_size(n, at, d, Hq):
    """From row `at` on results and state are those of a sequence that begins there."""
    Hkv = 2
    q, k, v, r = data(n, Hq, Hkv, d, 6, 1e-10)
    decay = -0.05 * r
    decay[at] = -math.inf
    first = torch.full((1, Hkv, d, d), 3e38)
    out, S = sts.sts_linear_attn(q.to(DEV), k.to(DEV), v.to(DEV), decay.to(DEV), 0.1, starts=starts_of([n]).to(DEV), max_len=n, state=first.to(DEV),
                                 state_out=torch.empty(1, Hkv, d, d, device=DEV), out_dtype=torch.float32)
    ref, all_s, e, e_s = linear(q[at:], k[at:], v[at:], decay[at:], 0.1, torch.zeros(Hkv, d, d), n > 16)
    check_linear(out[at:], ref, e)
    check_linear(S[0], all_s[-1], e_s[-1], "state")
