"""Every form of the step over kept entries against the oracle: heads on four waves and on eight, in shares, up to eight query heads and
more, both storage types; and the weights of many short prompts."""
import numpy as np
import pytest
import torch

from oracle import kept_oracle as ko
from paper_2510_20787_amd import binding as B
from tests.kept_util import f64, make_state, run_and_check

pytestmark = pytest.mark.gpu

# sequences, KV heads, window, budget, heads checked: every n-th
HEADS = {"four waves": (150, 2, 45, 70, 29), "few on four waves": (20, 2, 70, 100, 7), "eight waves": (70, 2, 70, 100, 23),
         "shares": (2, 2, 100, 2300, 1)}


@pytest.mark.parametrize("packed", [False, True], ids=["rows", "packed"])
@pytest.mark.parametrize("G", [1, 4, 9, 16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form", HEADS)
def test_forms_of_the_step(form, D, G, packed):
    nb, Hkv, window, budget, every = HEADS[form]
    cfg = B.make_cfg(G * Hkv, Hkv, D, window, budget, 2, 1e-3, 0.07, "bf16")
    seen = [window + budget + 11 + i for i in range(nb)]
    cache = make_state(cfg, seen, [budget if i % 3 else budget - 5 for i in range(nb)], 31)
    pk = B.ltea_kept_pack(cfg, cache) if packed else None
    for step in range(2):
        run_and_check(cfg, cache, pk, True, 500 + step, "bf16", heads=every)
    if packed:
        cache.n_scored += window
        run_and_check(cfg, cache, pk, False, 510, "bf16", heads=every)


@pytest.mark.parametrize("packed", [False, True], ids=["rows", "packed"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("nb,Hkv,window,budget,every", [(140, 2, 9, 40, 31), (60, 2, 9, 40, 17), (1, 2, 33, 2500, 1)])
def test_forms_of_the_step_in_fp32(nb, Hkv, window, budget, every, D, packed):
    cfg = B.make_cfg(3 * Hkv, Hkv, D, window, budget, 0, 0.0, 0.0, "f32")
    cache = make_state(cfg, [window + budget + i for i in range(nb)], [budget] * nb, 32)
    pk = B.ltea_kept_pack(cfg, cache) if packed else None
    for step in range(2):
        run_and_check(cfg, cache, pk, True, 520 + step, "f32", heads=every)


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_given_keys_without_a_budget(dtype, D):
    """Nothing is ever kept, and there are no packed rows to point at."""
    cfg = B.make_cfg(4, 2, D, 33, 0, 2, 0.0, 0.0, dtype)
    cache = make_state(cfg, [0, 7, 33, 200], [0, 0, 0, 0], 34)
    cache.n_scored += 33
    packed = B.alloc_packed(cfg, 4)
    assert packed.numel() == 0
    for step in range(3):
        run_and_check(cfg, cache, packed, False, 530 + step, dtype)
    assert B.ltea_kept_pack(cfg, cache).numel() == 0


def test_weights_of_many_short_prompts():
    """More sequences than a wave looks up at once, most of a few tokens, some of none."""
    rng = np.random.default_rng(33)
    lens = rng.integers(0, 6, 200)
    lens[[50, 130]] = 140, 33
    T, sigma = int(lens.sum()), 0.2
    q, k = [torch.from_numpy(rng.standard_normal((T, h, 64))).to(dtype=torch.bfloat16, device="cuda") for h in (4, 2)]
    cu = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)])).to(dtype=torch.int32, device="cuda")
    want, lse, lo = np.zeros((2, T)), np.zeros((4, T)), 0
    for n in lens:
        x, y = f64(q[lo:lo + n]), f64(k[lo:lo + n])
        if n:
            lse[:, lo:lo + n] = ko.causal_lse(x, y, 150, sigma).astype(np.float32)
            want[:, lo:lo + n] = ko.attention_mass(x, y, lse[:, lo:lo + n], 150, 3, sigma)
        lo += n
    cfg = B.make_cfg(4, 2, 64, 150, 0, 0, 0.0, sigma, "bf16")
    got = f64(B.ltea_attention_mass(cfg, q, k, cu, 140, torch.from_numpy(lse).float().cuda(), last=3))
    # as for longer prompts: 2^-15 of a weight
    assert (np.abs(got - want) <= 2.0 ** -15 * want + 1e-30).all()


def test_prompts_of_no_tokens_start_a_cache():
    cfg = B.make_cfg(4, 2, 64, 16, 20, 1, 0.0, 0.0, "bf16")
    cache = make_state(cfg, [50, 60], [20, 20], 35)
    q, k = [torch.empty((0, h, 64), dtype=torch.bfloat16, device="cuda") for h in (4, 2)]
    cu = torch.zeros(3, dtype=torch.int32, device="cuda")
    out = B.ltea_prefill_mass(cfg, q, k, k, cu, 0, cache)
    assert out.shape == (0, 4, 64) and not cache.n_seen.any() and not cache.n_scored.any() and not cache.ret_count.any()
    assert B.ltea_attention_mass(cfg, q, k, cu, 0, torch.empty((4, 0), device="cuda")).shape == (2, 0)
    for step in range(2):
        run_and_check(cfg, cache, None, True, 540 + step, "bf16")


@pytest.mark.parametrize("Hq,Hkv,D,dtype", [(5, 1, 64, "bf16"), (17, 1, 128, "bf16"), (60, 4, 64, "bf16"), (7, 1, 64, "f32")])
@pytest.mark.parametrize("n,last", [(1, 0), (70, 0), (300, 0), (900, 100)])
def test_weights_of_groups_in_parts(Hq, Hkv, D, dtype, n, last):
    """Short prompts: the heads of a group in parts that need not be equal."""
    rng = np.random.default_rng(36)
    q, k = [torch.from_numpy(rng.standard_normal((n, h, D))).to(dtype=B.torch_dtype(dtype), device="cuda") for h in (Hq, Hkv)]
    x, y = f64(q), f64(k)
    lse = ko.causal_lse(x, y, n, D ** -0.5).astype(np.float32)
    want = ko.attention_mass(x, y, lse.astype(np.float64), n, last, D ** -0.5)
    cfg = B.make_cfg(Hq, Hkv, D, n, 0, 0, 0.0, 0.0, dtype)
    cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    got = f64(B.ltea_attention_mass(cfg, q, k, cu, n, torch.from_numpy(lse).cuda(), last=last))
    assert (np.abs(got - want) <= 2.0 ** -15 * want + 1e-30).all()           # as above
