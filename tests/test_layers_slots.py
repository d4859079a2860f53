"""Which slots sts_linear_attn writes where the caller names none: on the CPU, by the parameter block of a prepared call that nothing launches."""
import pytest
import torch

import paper_2605_15508_amd as sts
from paper_2605_15508_amd import binding

B, n, Hkv, d = 3, 4, 2, 64


@pytest.fixture
def params(monkeypatch):
    """The parameter block of the call, made from CPU tensors."""
    monkeypatch.setattr(binding, "_current", lambda dev: None)
    k = torch.zeros(B, n, Hkv, d, dtype=torch.bfloat16)
    return lambda **kw: sts.sts_linear_attn(None, k, k, torch.zeros(Hkv), prepare=True, **kw)._p


def pools():
    wide = torch.zeros(4, 8, 3 * Hkv, d, d)           # [layers, slots, heads of three parts, d, d]
    return wide, torch.tensor([6, 1, 3], dtype=torch.int32)


@pytest.mark.parametrize("slice_of", [lambda w: w[2, :, :Hkv], lambda w: w[1, :, Hkv:2 * Hkv], lambda w: w[3, :, 2 * Hkv:], lambda w: w[0, 7:, :Hkv], lambda w: w[0, :, :Hkv].view(8, Hkv, d, d)])
def test_two_slices_of_one_pool_are_one_pool(params, slice_of):
    """Indexing makes a new tensor object every time."""
    wide, slots = pools()
    p = params(state=slice_of(wide), slots=slots, state_out=slice_of(wide))
    assert p.state == p.state_out and p.slots == slots.data_ptr() == p.slots_out
    one = slice_of(wide)
    p = params(state=one, slots=slots, state_out=one)
    assert p.slots == slots.data_ptr() == p.slots_out
    if one.shape[0] >= B:
        p = params(state=slice_of(wide), state_out=slice_of(wide))
        assert p.slots is None and p.slots_out is None


def test_slots_that_are_named_stay(params):
    wide, slots = pools()
    to = torch.tensor([0, 2, 4], dtype=torch.int32)
    for state_out in (wide[0, :, :Hkv], wide[0, 1:, :Hkv], wide[1, :, :Hkv]):
        assert params(state=wide[0, :, :Hkv], slots=slots, state_out=state_out, slots_out=to).slots_out == to.data_ptr()
    assert params(state_out=wide[0, :, :Hkv], slots_out=to).slots_out == to.data_ptr()


def test_pools_that_share_nothing_go_by_the_sequences(params):
    wide, slots = pools()
    one = wide[0, :, :Hkv]
    for state_out in (wide[1, :, :Hkv], wide[0, :, Hkv:2 * Hkv], wide[0, :, 2 * Hkv:], torch.zeros(B, Hkv, d, d)):
        p = params(state=one, slots=slots, state_out=state_out)
        assert p.slots_out is None and p.slots == slots.data_ptr()
        p = params(state=state_out, slots=slots, state_out=one)
        assert p.slots_out is None
    assert params(state=None, state_out=one).slots_out is None and params(state=one, slots=slots).slots_out is None
    # without lists sequence b reads slot b and writes slot b: what lies behind the sequences' slots is touched by none
    assert params(state=wide[0, :4, :Hkv], state_out=wide[0, :3, :Hkv]).slots_out is None
    assert params(state=wide[0, :4, :Hkv], state_out=wide[0, 3:, :Hkv]).slots_out is None


@pytest.mark.parametrize("state,state_out", [(lambda w: w[0, :, :Hkv], lambda w: w[0, 1:, :Hkv]), (lambda w: w[0, 1:, :Hkv], lambda w: w[0, :, :Hkv]), (lambda w: w[0, :, :Hkv], lambda w: w[0, :5, :Hkv]),
                                             (lambda w: w[0, :, :Hkv], lambda w: w[0, :, 1:1 + Hkv]), (lambda w: w[0, :, :Hkv], lambda w: w[0, ::2, :Hkv]), (lambda w: w[0, ::2, :Hkv], lambda w: w[0, :, :Hkv])])
def test_pools_that_overlap_otherwise_need_their_slots_named(params, state, state_out):
    """Where each sequence's state goes to would depend on which one of two is read first."""
    wide, slots = pools()
    with pytest.raises(AssertionError, match="slots_out"):
        params(state=state(wide), slots=slots, state_out=state_out(wide))
    to = torch.tensor([0, 1, 2], dtype=torch.int32)
    assert params(state=state(wide), slots=slots, state_out=state_out(wide), slots_out=to).slots_out == to.data_ptr()


def test_places_that_another_sequence_reads_are_refused_without_lists_too(params):
    wide, _ = pools()
    for to in (1, 2):
        with pytest.raises(AssertionError, match="slots_out"):
            params(state=wide[0, :5, :Hkv], state_out=wide[0, to:, :Hkv])


def test_no_sequences_and_empty_pools(params):
    wide, _ = pools()
    with pytest.raises((AssertionError, sts.StsError)):
        params(state=wide[0, :, :Hkv], slots=torch.zeros(1, dtype=torch.int32), state_out=wide[0, :, :Hkv])
    p = params(state=wide[0, :0, :Hkv], slots=torch.zeros(B, dtype=torch.int32), state_out=wide[0, :, :Hkv])
    assert p.slots_out is None and p.num_slots == 0
