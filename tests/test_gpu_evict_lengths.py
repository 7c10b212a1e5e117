"""A decode iteration's weights where ctx_lens holds what no block table can describe: the same whichever launch adds them."""
import numpy as np
import pytest
import torch

import evict_common as ec
import gpu_common as gc
from test_gpu_evict import dev, handle, workspace

pytestmark = pytest.mark.gpu
DEV = gc.DEV


# by the launch itself (little to add) and by one behind it
@pytest.mark.parametrize("most", [160, 2112])
@pytest.mark.parametrize("fp8", [0, 1])
def test_length_beyond_the_block_table(most, fp8):
    """Longer than max_ctx_len, so no weight is added; the others' are."""
    c = ec.Cache([most, 30], 2, 64, 190, bool(fp8), room=[0, most - 30], extra_blocks=0)
    assert c.blocks * ec.PAGE == most
    h = handle(c, 8)
    bf = lambda n: torch.randn(2, n, 64, device=DEV).to(torch.bfloat16)
    w, out = dev(c.weights.clone()), torch.zeros(2, 8, 64, dtype=torch.bfloat16, device=DEV)
    work = workspace(h.tetri_decode_attn_weights_workspace(2, most))
    ctx = dev(np.array([most + 5, 30], dtype=np.int32))
    h.tetri_decode_attn_weights(bf(8), bf(2), bf(2), dev(c.pool), w, dev(c.bt), ctx, 2, most, 0.1, 0, fp8, ec.K_SCALE, ec.V_SCALE, work,
                                work.numel(), out)
    w, touched = w.cpu(), torch.zeros(c.weights.shape, dtype=torch.bool)
    p, s = c.slots(1, 30)
    touched[p, :, s] = True
    assert torch.equal(w.view(torch.int32)[~touched], c.weights.view(torch.int32)[~touched])
    assert (w[p, :, s] > c.weights[p, :, s]).all()
    h.close()


@pytest.mark.parametrize("most", [160, 2112])
@pytest.mark.parametrize("fp8", [0, 1])
@pytest.mark.parametrize("append", [0, 1])
def test_length_below_zero(most, append, fp8):
    """As length 0, as the attention and the cache take it: the new token has all the weight and the first slot."""
    c = ec.Cache([0, 30], 2, 64, 191, bool(fp8), room=most - 40, extra_blocks=0)
    h = handle(c, 8)
    g = 4
    bf = lambda n: torch.randn(2, n, 64, device=DEV).to(torch.bfloat16)
    w, out = dev(c.weights.clone()), torch.zeros(2, 8, 64, dtype=torch.bfloat16, device=DEV)
    longest = c.blocks * ec.PAGE - 1
    work = workspace(h.tetri_decode_attn_weights_workspace(2, longest))
    ctx = dev(np.array([-3, 30], dtype=np.int32))
    h.tetri_decode_attn_weights(bf(8), bf(2), bf(2), dev(c.pool), w, dev(c.bt), ctx, 2, longest, 0.1, append, fp8, ec.K_SCALE, ec.V_SCALE, work,
                                work.numel(), out)
    w, touched = w.cpu(), torch.zeros(c.weights.shape, dtype=torch.bool)
    p, s = c.slots(1, 30 + append)
    touched[p, :, s] = True
    if append:
        first = w[c.bt[0, 0], :, 0]
        # (g weights of exactly 1 but for the roundings of a score, its logarithm and the exponential: 2^-19)
        assert ((first - g).abs() <= g * 2.0 ** -19).all()
        touched[c.bt[0, 0], :, 0] = True
    assert torch.equal(w.view(torch.int32)[~touched], c.weights.view(torch.int32)[~touched])
    h.close()
