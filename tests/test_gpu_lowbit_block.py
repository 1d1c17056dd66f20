"""The operators together: a residual block trained in low precision."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("state_bits", [8, 32])
def test_a_block_learns_a_teacher(state_bits):
    """From another initialisation the loss has to fall to less than half of its start in 60 updates, and every update is reproducible."""
    import torch
    from paper_2003_10579_amd import lowbit_block
    assert torch.cuda.is_available(), "this test needs the GPU"
    block, losses = lowbit_block.train(60, rows=1000, width=200, hidden=330, state_bits=state_bits, report=None)
    assert np.all(np.isfinite(losses)) and losses[-1] < 0.5 * losses[0]
    again, losses2 = lowbit_block.train(60, rows=1000, width=200, hidden=330, state_bits=state_bits, report=None)
    assert losses == losses2 and torch.equal(block.w1, again.w1) and torch.equal(block.optimizer.m.view(torch.uint8), again.optimizer.m.view(torch.uint8))
    # a single row gives what it gives among others
    x, r = (torch.randn(70, 200, device="cuda").to(torch.bfloat16) for _ in range(2))
    block.quantize_weights()
    whole = block.answer(x, r)
    one = block.answer(x[3:4], r[3:4])
    assert torch.allclose(one.float(), whole[3:4].float(), rtol=2.0 ** -6, atol=2.0 ** -6 * float(whole.float().abs().max()))
