"""Weights of prompts whose keys are not all numbers: what a token received is the sum over the queries that see it and count, no other."""
import numpy as np
import pytest
import torch

from oracle import kept_oracle as ko
from paper_2510_20787_amd import binding as B
from tests.kept_util import f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("last", [0, 45])
@pytest.mark.parametrize("window", [2000, 77])
@pytest.mark.parametrize("lens", [(37, 90), (1111, 1, 300)], ids=str)
@pytest.mark.parametrize("dtype,Hq,Hkv,D", [("bf16", 4, 2, 64), ("bf16", 3, 1, 128), ("f32", 2, 1, 64), ("f32", 1, 1, 128)])
def test_keys_that_are_not_numbers(dtype, Hq, Hkv, D, lens, window, last):
    """Rows of NaN and of either infinity among the keys, queries without a normaliser, ends that fill no tile, several parts."""
    rng = np.random.default_rng(51)
    T, td, sigma = sum(lens), B.torch_dtype(dtype), 0.2
    q, k = [torch.from_numpy(rng.standard_normal((T, h, D))).to(dtype=td, device="cuda") for h in (Hq, Hkv)]
    q[..., 0] = q[..., 0].abs() + 0.25                       # a key of -inf there scores -inf against every query, one of inf inf
    cu = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    lse, lo = np.zeros((Hq, T), np.float32), 0
    for n in lens:                                           # (of the keys before they are spoiled: any finite number will do)
        lse[:, lo:lo + n] = ko.causal_lse(f64(q[lo:lo + n]), f64(k[lo:lo + n]), window, sigma)
        lo += n
    spoiled = {}
    for i, value in enumerate((np.nan, np.inf, -np.inf)):
        for j in rng.choice(T, 6, replace=False).tolist() + [int(cu[1]) - 1 - i, T - 1 - i]:
            spoiled[j] = value
    spoiled[5], spoiled[int(cu[1]) + 0] = np.nan, np.nan
    for j, value in spoiled.items():
        k[j, :, 0] = value
    lse[0, rng.choice(T, T // 6, replace=False)] = np.nan    # queries that count nothing, some heads all of them behind one key
    lse[:, 5:int(cu[1])] = np.where(rng.random((Hq, int(cu[1]) - 5)) < 0.5, np.inf, lse[:, 5:int(cu[1])])
    lse[:, int(cu[-2]):] = np.nan                            # nobody of the last sequence
    want, lo = np.zeros((Hkv, T)), 0
    for n in lens:
        with np.errstate(invalid="ignore"):
            want[:, lo:lo + n] = ko.attention_mass(f64(q[lo:lo + n]), f64(k[lo:lo + n]), lse[:, lo:lo + n].astype(np.float64), window, last, sigma)
        lo += n
    assert np.isnan(want).any() and np.isinf(want).any() or last > 0
    cfg = B.make_cfg(Hq, Hkv, D, window, 0, 0, 0.0, sigma, dtype)
    got = f64(B.ltea_attention_mass(cfg, q, k, cu, max(lens), torch.from_numpy(lse).cuda(), last=last))
    assert np.array_equal(np.isnan(got), np.isnan(want)), np.argwhere(np.isnan(got) != np.isnan(want))[:5]
    assert np.array_equal(np.isinf(got), np.isinf(want))
    fine = np.isfinite(want)
    # scores of a few units, sums of at most 1111 terms: 2^-17 of a term, and 2^-24 for each of half the terms on average: 2^-15
    assert (np.abs(got[fine] - want[fine]) <= 2.0 ** -15 * want[fine] + 1e-30).all()
    assert not got[:, int(cu[-2]):].any()
