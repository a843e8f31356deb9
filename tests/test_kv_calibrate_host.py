"""The calibration's batches over the instances that its limits allow.  No GPU."""

import pytest

from paper_2607_18253_amd import calibrate as K


@pytest.mark.parametrize("limits", [
    dict(token_budget=512, max_seqs=1024, chunk_cap=128), dict(token_budget=64, max_seqs=64, chunk_cap=512),
    dict(token_budget=1, max_seqs=8), dict(token_budget=300, max_seqs=1, chunk_cap=1), dict(chunk_cap=0),
    dict(max_ctx=2, kv_blocks=1), dict(max_ctx=9, kv_blocks=9, block_size=1), dict(kv_blocks=512, max_ctx=8192),
    dict(kv_blocks=1)])
def test_batches_of_any_instance(limits):
    inst = K.Instance(**limits)
    some = K.batches(inst, 45, seed=4)
    assert len(some) == 45
    for b in some:
        assert b.q_len.sum() <= inst.token_budget and 1 <= len(b.q_len) <= inst.max_seqs
        assert (b.q_len >= 1).all() and (b.q_len[:b.n_dec] == 1).all()
        assert not inst.chunk_cap or (b.q_len <= inst.chunk_cap).all()
        assert (b.ctx_len >= b.q_len).all() and (b.ctx_len <= inst.max_ctx).all()
        assert (-(-b.ctx_len // inst.block_size)).sum() <= inst.kv_blocks


@pytest.mark.parametrize("limits", [
    dict(token_budget=0), dict(max_seqs=0), dict(chunk_cap=-1), dict(max_ctx=1), dict(kv_blocks=0), dict(kv_blocks=15, block_size=1)])
def test_instances_that_cannot_run(limits):
    with pytest.raises(ValueError):
        K.Instance(**limits)
