"""The example's loss is a mean over the targets that there are: a target that is no token of the
vocabulary counts as none, as a negative one does, and is reported."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_targets_outside_the_vocabulary(sn):
    from paper_2506_01260_gb300 import lm_step
    results = []
    for bad in (-1, 300, 2 ** 31 - 1):
        m = lm_step.TwoStage(vocab=300, d=128, d_ff=192, k=12, seed=3)
        ids, target = lm_step.chain(500, m.vocab, seed=1)
        target[::3] = bad
        loss = m.backward(ids, target)
        if bad < 0:
            sn.sn_check_errors(m.basis)
        else:
            with pytest.raises(sn.SNError) as e:
                sn.sn_check_errors(m.basis)
            assert e.value.status == sn.SN_ERR_BAD_ID
        results.append([loss, *(g.clone() for g in m.grads.values())])
    for other in results[1:]:
        for a, b in zip(results[0], other):
            assert torch.equal(a, b)
