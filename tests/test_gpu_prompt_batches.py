"""sts_prompt_attn over more sequences than one load looks through (64), of several blocks each: another order of the blocks, found in another way."""
import pytest
import torch

import paper_2605_15508_amd as sts
from layers_util import check_prompts, prompts, starts_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def batch(B, most, Hq, Hkv, d, seed):
    g = torch.Generator().manual_seed(seed)
    lens = torch.randint(0, most, (B,), generator=g).tolist()
    lens[0], lens[B // 2], lens[B - 1] = most, 0, most - 1
    return lens, starts_of(lens), [torch.randn(sum(lens), h, d, generator=g).to(torch.bfloat16) for h in (Hq, Hkv, Hkv)]


@pytest.mark.parametrize("d,Hq,Hkv", [(128, 8, 2), (64, 4, 4), (64, 16, 1), (128, 3, 1)])
@pytest.mark.parametrize("B", [64, 65, 130])
def test_many_prompts_of_several_blocks(B, d, Hq, Hkv):
    lens, starts, (q, k, v) = batch(B, 420, Hq, Hkv, d, B + Hq)
    out, lse = sts.sts_prompt_attn(q.to(DEV), k.to(DEV), v.to(DEV), starts.to(DEV), 0.1, out_dtype=torch.float32)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    for b in (0, 1, B // 3, 63, B - 2, B - 1):
        a, e = int(starts[b]), int(starts[b + 1])
        if e > a:
            check_prompts((out[a:e], lse[:, a:e]), prompts(q[a:e], k[a:e], v[a:e], starts_of([e - a]), 0.1), what=f"{b}")


@pytest.mark.parametrize("d", [64, 128])
def test_a_sequence_is_the_same_in_any_batch(d):
    """A block of a sequence that lies elsewhere in the batch, or in another one, comes to the same numbers: every sequence by itself, and among all."""
    lens, starts, (q, k, v) = batch(90, 300, 8, 2, d, 7)
    q, k, v = (t.to(DEV) for t in (q, k, v))
    out, lse = sts.sts_prompt_attn(q, k, v, starts.to(DEV), 0.1)
    for b in range(90):
        a, e = int(starts[b]), int(starts[b + 1])
        if e > a:
            one = sts.sts_prompt_attn(q[a:e], k[a:e], v[a:e], starts_of([e - a]).to(DEV), 0.1)
            assert torch.equal(one[0], out[a:e]) and torch.equal(one[1], lse[:, a:e]), b
