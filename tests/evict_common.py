"""Inputs of the eviction tests: requests of given lengths at random places of a pool whose other slots hold garbage."""
import numpy as np
import torch

PAGE = 16
K_SCALE, V_SCALE = 0.0137, 0.0171
NAN_CODE = 0x7F


class Cache:
    """A pool (16-bit values or codes), weights and block tables of requests with `lens` cached tokens and room for `room` more."""

    def __init__(self, lens, hkv, d, seed, fp8=False, room=1, extra_blocks=2, std=1.0):
        rng = np.random.default_rng(seed)
        gen = torch.Generator().manual_seed(seed)
        self.lens, self.hkv, self.d, self.fp8 = [int(n) for n in lens], hkv, d, fp8
        room = [room] * len(lens) if np.isscalar(room) else list(room)
        need = [-(-(n + m) // PAGE) for n, m in zip(self.lens, room)]
        self.pages = sum(need) + 3
        self.blocks = max(1, max(need)) + extra_blocks
        perm = rng.permutation(self.pages).astype(np.int32)
        self.bt = np.full((len(lens), self.blocks), 0x7FFFFFF0, dtype=np.int32)      # (entries that no token needs are no pages)
        at = 0
        for b, n in enumerate(need):
            self.bt[b, :n] = perm[at:at + n]
            at += n
        shape = (self.pages, 2, hkv, PAGE, d)
        values = torch.randn(shape, generator=gen) * std
        if fp8:
            scale = torch.tensor([K_SCALE, V_SCALE]).view(1, 2, 1, 1, 1)
            self.pool = (values / scale).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        else:
            self.pool = values.to(torch.bfloat16)
        self.weights = torch.rand((self.pages, hkv, PAGE), generator=gen) * 0.1
        # slots without a token: NaN
        used = torch.zeros((self.pages, PAGE), dtype=torch.bool)
        for b, n in enumerate(self.lens):
            j = np.arange(n)
            used[self.bt[b, j // PAGE], j % PAGE] = True
        spare = ~used
        self.pool.permute(0, 3, 1, 2, 4)[spare] = NAN_CODE if fp8 else float("nan")
        self.weights.permute(0, 2, 1)[spare] = float("nan")

    @property
    def ctx(self):
        return np.array(self.lens, dtype=np.int32)

    def float_pool(self):
        """The pool as float64 numpy values; garbage as 0."""
        if self.fp8:
            scale = torch.tensor([np.float32(K_SCALE), np.float32(V_SCALE)], dtype=torch.float64).view(1, 2, 1, 1, 1)
            x = self.pool.view(torch.float8_e4m3fn).double() * scale
        else:
            x = self.pool.double()
        return torch.nan_to_num(x, nan=0.0).numpy()

    def slots(self, b, count):
        """Pages and places of the first `count` slots of request b."""
        j = np.arange(count)
        return self.bt[b, j // PAGE], j % PAGE


def weight_bound(added, before, amplitude, d):
    """How far a weight may be off: the sum of what was added, each term with a relative error, and the last additions.

    A score is a sum of d products, exact ones, in fp32: off by at most d steps of 2^-24 of sum |q_i k_i| |scale| =: amplitude, whose
    largest value counts; it is multiplied by scale * log2(e) (rounded) and lse, made of such scores, is subtracted: three more
    roundings of numbers below amplitude * log2(e) + 20 each.  An exponential, a logarithm, and the sums over keys and rows (of terms that
    are all positive) stay below 2^-19 relative.  A term below 2^-126 may count as nothing: 2^-112 for all of a slot's.
    """
    rel = 2 * (d + 4) * 2.0 ** -24 * amplitude + 4 * 2.0 ** -24 * (amplitude * 1.45 + 20) + 2.0 ** -19
    return added * rel + (np.abs(before) + added) * 2.0 ** -23 + 2.0 ** -112


def amplitude(q, keys, scale):
    """Largest sum |q_i k_i| |scale| over rows of q [n,D] and keys [m,D]."""
    return float((np.abs(q) @ np.abs(keys).T).max() * abs(scale)) if len(q) and len(keys) else 0.0
