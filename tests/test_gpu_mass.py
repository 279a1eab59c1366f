"""Attention weight that a prompt's tokens have received, and the prefill of a cache that keeps by it, against 64 bits."""
import numpy as np
import pytest
import torch

from oracle import kept_oracle as ko
from oracle import ltea_oracle as orc
from paper_2510_20787_amd import binding as B
from tests.kept_util import f64

pytestmark = pytest.mark.gpu


def prompt(lens, Hq, Hkv, D, dtype, seed, views=False):
    td = B.torch_dtype(dtype)
    rng = np.random.default_rng(seed)
    T = sum(lens)
    put = lambda x: torch.from_numpy(x).to(dtype=td, device="cuda")
    if views:        # q, k, v as slices of one projection's output, heads apart by more than a row
        x = put(rng.standard_normal((T, Hq + 2 * Hkv, D + 16)))
        q, k, v = x[:, :Hq, :D], x[:, Hq:Hq + Hkv, :D], x[:, Hq + Hkv:, :D]
    else:
        q, k, v = (put(rng.standard_normal((T, h, D))) for h in (Hq, Hkv, Hkv))
    cu = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    return q, k, v, cu


def reference(q, k, lens, window, last, sigma, lse=None):
    mass, all_lse, lo = [], [], 0
    for n in lens:
        x, y = f64(q[lo:lo + n]), f64(k[lo:lo + n])
        z = ko.causal_lse(x, y, window, sigma) if lse is None else lse[:, lo:lo + n]
        z = z.astype(np.float32).astype(np.float64)          # what the device is given
        all_lse.append(z)
        mass.append(ko.attention_mass(x, y, z, window, last, sigma))
        lo += n
    return np.concatenate(mass, 1), np.concatenate(all_lse, 1)


# The exponent is a fused multiply-add on numbers of some tens: its rounding, that of lse * log2(e) and the score's sum of at most 128
# terms leave 2^-17 of relative error in a term at most, a chain of sums of n terms n/2 roundings of 2^-24 on average and never more
# than n: 2^-15 together for the lengths here.
def check_mass(got, ref):
    err = np.abs(f64(got) - ref)
    assert (err <= 2.0 ** -15 * ref + 1e-30).all(), float((err / np.maximum(ref, 1e-30)).max())


@pytest.mark.parametrize("Hq,Hkv,D,dtype", [(2, 2, 64, "f32"), (4, 2, 128, "f32"), (2, 2, 64, "bf16"), (8, 2, 64, "bf16"),
                                            (3, 1, 128, "bf16"), (12, 3, 128, "bf16")])
@pytest.mark.parametrize("lens", [(1,), (31, 0, 64, 65), (300,), (257, 1, 511)], ids=str)
@pytest.mark.parametrize("window,last", [(0, 0), (40, 0), (1, 0), (0, 1), (0, 70), (100, 33)])
def test_mass(Hq, Hkv, D, dtype, lens, window, last):
    q, k, _, cu = prompt(lens, Hq, Hkv, D, dtype, 3, views=window == 40)
    w = window or max(lens)
    ref, lse = reference(q, k, lens, w, last, D ** -0.5)
    cfg = B.make_cfg(Hq, Hkv, D, w, 0, 0, 0.0, 0.0, dtype)
    got = B.ltea_attention_mass(cfg, q, k, cu, max(lens), torch.from_numpy(lse).float().cuda(), last=last)
    check_mass(got, ref)


@pytest.mark.parametrize("dtype,Hq,Hkv,D,lens,window", [("bf16", 4, 1, 64, (3000,), 3000), ("bf16", 1, 1, 128, (2500, 700), 1100),
                                                        ("f32", 2, 1, 64, (1500,), 1500)])
def test_long_prompts_in_parts(dtype, Hq, Hkv, D, lens, window):
    """Several parts of the queries per key, ends inside a tile; a scale of the caller's; same bits whatever the workspace held."""
    q, k, _, cu = prompt(lens, Hq, Hkv, D, dtype, 4)
    ref, lse = reference(q, k, lens, window, 0, 0.2)
    cfg = B.make_cfg(Hq, Hkv, D, window, 0, 0, 0.0, 0.2, dtype)
    lse = torch.from_numpy(lse).float().cuda()
    got = []
    for fill in (0, 255):
        ws = torch.full((B.ltea_mass_workspace_bytes(cfg, len(lens), sum(lens), max(lens)),), fill, dtype=torch.uint8, device="cuda")
        got.append(B.ltea_attention_mass(cfg, q, k, cu, max(lens), lse, workspace=ws))
    check_mass(got[0], ref)
    assert torch.equal(*got)


def test_queries_that_count_nothing():
    """A query whose lse is not finite counts nothing, whatever its row holds; the rest is as without it."""
    lens = (90, 40)
    q, k, _, cu = prompt(lens, 4, 2, 64, "bf16", 5)
    ref, lse = reference(q, k, lens, 90, 0, 0.125)
    dead = [(0, 3), (2, 89), (1, 100), (3, 129)]
    for value, row in ((np.nan, float("nan")), (np.inf, float("inf")), (-np.inf, 1.0)):
        z = lse.copy()
        x = q.clone()
        for hq, i in dead:
            z[hq, i] = value
            x[i, hq] = row
        good = q.clone()
        want, _ = reference(good, k, lens, 90, 0, 0.125, lse=z)
        cfg = B.make_cfg(4, 2, 64, 90, 0, 0, 0.0, 0.125, "bf16")
        check_mass(B.ltea_attention_mass(cfg, x, k, cu, 90, torch.from_numpy(z).float().cuda()), want)


@pytest.mark.parametrize("dtype,Hq,Hkv,D,lens,window,budget,last", [("f32", 2, 2, 64, (50, 7, 1), 12, 9, 0),
                                                                    ("bf16", 8, 2, 64, (300, 40, 0, 33), 64, 50, 0),
                                                                    ("bf16", 4, 4, 128, (200, 90), 16, 32, 20)])
def test_prefill_by_mass(dtype, Hq, Hkv, D, lens, window, budget, last):
    """Full causal attention of the prompt, its weights, and the cache that retention by them fills."""
    q, k, v, cu = prompt(lens, Hq, Hkv, D, dtype, 6, views=True)
    sigma, T, G = D ** -0.5, sum(lens), Hq // Hkv
    cfg = B.make_cfg(Hq, Hkv, D, window, budget, 3, 0.0, 0.0, dtype)
    cache = B.alloc_cache(cfg, len(lens))
    mass = torch.empty((Hkv, T), dtype=torch.float32, device="cuda")
    out = B.ltea_prefill_mass(cfg, q, k, v, cu, max(lens), cache, last=last, mass=mass)
    again = B.ltea_prefill_mass(cfg, q, k, v, cu, max(lens), B.alloc_cache(cfg, len(lens)), last=last)
    assert torch.equal(out, again)
    lo = 0
    for s, n in enumerate(lens):
        x, y, z = (f64(a[lo:lo + n]) for a in (q, k, v))
        lse = ko.causal_lse(x, y, max(n, 1), sigma) if n else np.zeros((Hq, 0))
        ref = ko.attention_mass(x, y, lse, max(n, 1), last, sigma)
        # 2^-13 for the weights themselves.  bf16: the attention sums the probabilities as it multiplies them, rounded to bf16, each off
        # by at most 2^-8 of itself; so is their sum, the normaliser e^lse, by which every weight of the query is divided.
        err = np.abs(f64(mass[:, lo:lo + n]) - ref)
        assert (err <= (2.0 ** -13 + (2.0 ** -8 if dtype == "bf16" else 0)) * ref + 1e-30).all()
        ago = np.arange(n)[:, None] - np.arange(n)[None]
        for hq in range(Hq):
            p = ko.softmax_rows(np.where(ago >= 0, sigma * (x[:, hq] @ y[:, hq // G].T), -np.inf)) if n else np.zeros((0, 0))
            want = p @ z[:, hq // G]
            tol = (2.0 ** -6 if dtype == "bf16" else 1e-5) * (np.abs(z).max() if n else 1)
            assert (np.abs(f64(out[lo:lo + n, hq]) - want) <= tol).all()
        for h in range(Hkv):
            keys = f64(mass[h, lo:lo + n])
            keep = orc.retain(keys, n, window, budget, 3, 0.0)
            cnt = int(cache.ret_count[s, h])
            assert np.array_equal(f64(cache.ret_pos[s, h, :cnt]), keep)
            assert np.array_equal(f64(cache.k_ret[s, h, :cnt]), y[keep.astype(int), h])
            for p in range(max(0, n - window), n):
                assert float(cache.win_score[s, h, p % window]) == keys[p]
                assert np.array_equal(f64(cache.v_win[s, h, p % window]), z[p, h])
        assert int(cache.n_seen[s]) == n and int(cache.n_scored[s]) == n
        lo += n
