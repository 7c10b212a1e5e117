"""A decode iteration's weight of a token is summed over the query heads before it is added to what the token has."""
import pytest
import torch

import evict_common as ec
import gpu_common as gc
from test_gpu_evict import dev, handle, workspace

pytestmark = pytest.mark.gpu
DEV = gc.DEV


# cached tokens, and weights of which a query head's share, 1 / (L + 1) each, is a quarter of the last bit, all four's one
@pytest.mark.parametrize("L,held", [(511, 65536.0), (4095, 8192.0)], ids=["one-launch", "two"])
@pytest.mark.parametrize("fp8", [0, 1])
def test_small_weights_are_not_lost(L, held, fp8):
    hq, hkv, d, g = 8, 2, 64, 4
    c = ec.Cache([L], hkv, d, 210, bool(fp8))
    h = handle(c, hq)
    c.weights.fill_(held)
    w, q, kv = dev(c.weights), torch.zeros((1, hq, d), dtype=torch.bfloat16, device=DEV), torch.zeros((1, hkv, d), dtype=torch.bfloat16, device=DEV)
    out, work = torch.zeros_like(q), workspace(h.tetri_decode_attn_weights_workspace(1, L))
    h.tetri_decode_attn_weights(q, kv, kv, dev(c.pool), w, dev(c.bt), dev(c.ctx), 1, L, 0.1, 0, fp8, ec.K_SCALE, ec.V_SCALE, work, work.numel(), out)
    p, s = c.slots(0, L)
    got = w.cpu().double()[p, :, s] - held
    h.close()
    # (one addition: half of the last bit, held * 2^-24, and the exponentials' 2^-19 of a share)
    share = g / (L + 1.0)
    assert ((got - share).abs() <= held * 2.0 ** -24 + share * 2.0 ** -19).all(), (got.min(), got.max(), share)
