"""Weights of long prompts, in more parts than one launch takes, against 64 bits on the device."""
import numpy as np
import pytest
import torch

from paper_2510_20787_amd import binding as B

pytestmark = pytest.mark.gpu


def normalisers_and_weights(q, k, window, last, sigma):
    """Of one sequence, in blocks of queries: lse [Hq, n] fp32, mass [Hkv, n] fp64 by that lse."""
    n, Hq, D = q.shape
    Hkv, first = k.shape[1], max(0, n - last) if last > 0 else 0
    lse = torch.zeros((Hq, n), dtype=torch.float32, device=q.device)
    mass = torch.zeros((Hkv, n), dtype=torch.float64, device=q.device)
    j = torch.arange(n, device=q.device)
    for hq in range(Hq):
        kt = k[:, hq // (Hq // Hkv)].double().T.contiguous()
        for i0 in range(0, n, 2048):
            i1 = min(n, i0 + 2048)
            j0 = max(0, i0 - window + 1)
            s = sigma * (q[i0:i1, hq].double() @ kt[:, j0:i1])
            ago = j[i0:i1, None] - j[None, j0:i1]
            s.masked_fill_((ago < 0) | (ago >= window), -torch.inf)
            lse[hq, i0:i1] = torch.logsumexp(s, 1).float()
            s.sub_(lse[hq, i0:i1, None].double()).exp_()
            mass[hq // (Hq // Hkv), j0:i1] += s[max(0, first - i0):].sum(0)
    return lse, mass


CASES = [  # dtype, Hq, Hkv, D, lengths, window (0: all), last
    ("bf16", 2, 1, 64, (40000,), 0, 0),               # 20 parts of 2048 queries: two pairs of launches
    ("bf16", 1, 1, 128, (34000, 300, 1, 5000), 0, 33500),
    ("bf16", 2, 2, 64, (40000,), 36000, 0),           # parts counted from the first that reaches a key, two pairs of launches
    ("bf16", 4, 1, 64, (36000, 0, 4100), 3000, 0),    # and one
    ("bf16", 2, 1, 128, (9000, 20000), 130, 7001),
    ("f32", 1, 1, 64, (34000,), 0, 0),
    ("f32", 1, 1, 128, (5000, 30000), 257, 0),
    ("bf16", 3, 1, 64, (3000,), 100, 0),
    ("bf16", 2, 1, 64, (5000,), 64, 1000),            # most keys out of the windows of all that count
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_long_prompts(case):
    dtype, Hq, Hkv, D, lens, window, last = case
    rng = torch.Generator(device="cuda").manual_seed(61)
    T, sigma, w = sum(lens), 0.1, window or max(lens)
    q, k = [torch.randn((T, h, D), generator=rng, device="cuda").to(B.torch_dtype(dtype)) for h in (Hq, Hkv)]
    cu = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    lse, want = torch.zeros((Hq, T), device="cuda"), torch.zeros((Hkv, T), dtype=torch.float64, device="cuda")
    lo = 0
    for n in lens:
        if n:
            lse[:, lo:lo + n], want[:, lo:lo + n] = normalisers_and_weights(q[lo:lo + n], k[lo:lo + n], w, last, sigma)
        lo += n
    cfg = B.make_cfg(Hq, Hkv, D, w, 0, 0, 0.0, sigma, dtype)
    got = []
    for fill in (0, 255):
        ws = torch.full((B.ltea_mass_workspace_bytes(cfg, len(lens), T, max(lens)),), fill, dtype=torch.uint8, device="cuda")
        got.append(B.ltea_attention_mass(cfg, q, k, cu, max(lens), lse, last=last, workspace=ws,
                                         mass=torch.full((Hkv, T), float("nan"), device="cuda")))
    assert torch.equal(*got)
    # lse of some ten: 2^-17 of a term as for short prompts; chains of 2048 sums of like terms, then of the parts: half of 2048 + 20
    # roundings of 2^-24 at most on average, 2^-14
    err = (got[0].double() - want).abs()
    assert bool((err <= (2.0 ** -17 + 2.0 ** -14) * want + 1e-30).all()), float((err / want.clamp(min=1e-30)).max())
