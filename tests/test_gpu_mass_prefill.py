"""The weights that a prefill by weight fills its cache with, on bf16 storage, to the precision of fp32 normalisers."""
import numpy as np
import pytest
import torch

from paper_2510_20787_amd import binding as B
from tests.test_gpu_mass_long import normalisers_and_weights

pytestmark = pytest.mark.gpu


def weights_of_a_prefill(Hq, Hkv, D, lens, last, q, k, v, sigma):
    """Device weights and those of 64-bit normalisers."""
    T = sum(lens)
    cfg = B.make_cfg(Hq, Hkv, D, 64, 100, 2, 0.0, sigma, "bf16")
    cu = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    mass = torch.zeros((Hkv, T), device="cuda")
    B.ltea_prefill_mass(cfg, q, k, v, cu, max(lens), B.alloc_cache(cfg, len(lens)), last=last, mass=mass)
    want, lo = torch.zeros((Hkv, T), dtype=torch.float64, device="cuda"), 0
    for n in lens:
        if n:
            want[:, lo:lo + n] = normalisers_and_weights(q[lo:lo + n], k[lo:lo + n], n, last, sigma)[1]
        lo += n
    return mass.double(), want


# A weight: 2^-17 of a term and half a rounding of 2^-24 for each term of its sum (some thousand: 2^-14 at most), as where normalisers are
# given.  The normaliser: the same 2^-18 of a probability, sums of 32 and of at most 63 blocks (47 roundings of 2^-24 on average), and its
# logarithm's roundings, 2^-22 of the 16 that it is at most.  2^-13 together.
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 64), (3, 3, 64), (4, 1, 128), (2, 2, 128)])
@pytest.mark.parametrize("lens,last", [((1, 33, 0, 300), 0), ((2000, 77), 0), ((2000, 500), 100), ((40, 64), 1)], ids=str)
def test_weights_of_a_prefill(Hq, Hkv, D, lens, last):
    g = torch.Generator(device="cuda").manual_seed(91)
    q, k, v = [torch.randn((sum(lens), h, D), generator=g, device="cuda").to(torch.bfloat16) for h in (Hq, Hkv, Hkv)]
    got, want = weights_of_a_prefill(Hq, Hkv, D, lens, last, q, k, v, D ** -0.5)
    err = (got - want).abs()
    assert bool((err <= 2.0 ** -13 * want + 1e-30).all()), float((err / want.clamp(min=1e-30)).max())


@pytest.mark.parametrize("Hq,Hkv,D", [(4, 1, 64), (2, 2, 128)])
def test_scores_that_grow_late(Hq, Hkv, D):
    """Scores that leave the range of a row's first reference value: the attention runs its tiles again."""
    g = torch.Generator(device="cuda").manual_seed(92)
    n = 700
    q, k, v = [torch.randn((n, h, D), generator=g, device="cuda") for h in (Hq, Hkv, Hkv)]
    k[400:] += 60.0 / D * torch.sign(q[:, :1].mean(0, keepdim=True))          # towards a direction that every query shares
    q += 3.0 * torch.sign(q[:, :1].mean(0, keepdim=True))
    q, k, v = (x.to(torch.bfloat16) for x in (q, k, v))
    got, want = weights_of_a_prefill(Hq, Hkv, D, (n,), 0, q, k, v, 1.0)
    top = float((q.double()[:, 0] @ k.double()[:, 0].T).max())
    assert top > 100                                                         # 144 powers of two above the first keys
    # as above, with exponents and normalisers of up to 2^9 in powers of two: 2^-15 each of their rounding
    err = (got - want).abs()
    assert bool((err <= (2.0 ** -13 + 4 * 2.0 ** -15) * want + 1e-30).all()), float((err / want.clamp(min=1e-30)).max())
