"""Infinite values and rows that go in the steps over kept entries, with bounds that stay finite whatever the rows hold."""
import numpy as np
import pytest
import torch

from oracle import kept_oracle as ko
from paper_2510_20787_amd import binding as B
from tests.kept_util import clone, f64, kept_values, make_state, step_inputs

pytestmark = pytest.mark.gpu

INF = float("inf")


def one_step(cfg, cache, packed, by_mass, seed, heads, added_infinity=None):
    """A step on the device and, for every n-th (sequence, head), the oracle's output, the value rows that it attends and its new state."""
    nb, G = cache.n_seen.numel(), cfg.Hq // cfg.Hkv
    before, packed_before = clone(cache), None if packed is None else packed.clone()
    q, k, v = step_inputs(cfg, nb, seed)
    if added_infinity is not None:
        v[:, :, added_infinity] = INF
    if by_mass:
        out = B.ltea_decode_step_mass(cfg, q, k, v, cache, packed=packed)
    else:
        out = B.ltea_decode_step_packed(cfg, q, k, v, cache, packed)
    torch.cuda.synchronize()
    sigma = cfg.softmax_scale if cfg.softmax_scale > 0 else cfg.D ** -0.5
    for b, h in [(i // cfg.Hkv, i % cfg.Hkv) for i in range(0, nb * cfg.Hkv, heads)]:
        t, n = int(before.n_seen[b]), int(before.ret_count[b, h])
        kr, vr = (f64(before.k_ret[b, h, :n]), f64(before.v_ret[b, h, :n])) if packed is None else kept_values(cfg, packed_before, b, h, n)
        with np.errstate(invalid="ignore"):
            ref, st = ko.kept_step(f64(q[b, h * G:(h + 1) * G]), f64(k[b, h]), f64(v[b, h]), f64(before.k_win[b, h]),
                                   f64(before.v_win[b, h]), f64(before.win_score[b, h]), kr, vr, f64(before.ret_score[b, h, :n]),
                                   f64(before.ret_pos[b, h, :n]), t, cfg.window, cfg.budget, cfg.sink, cfg.tau_logit, sigma, by_mass,
                                   packed is not None)
        rows = [st["v_win"][:min(t + 1, cfg.window)], vr[[i for i in range(n) if i != st["dst"]]]]
        if st["dst"] is not None:          # the leaving token as it is kept
            e = f64(before.v_win[b, h, t % cfg.window])
            rows.append((ko.as_kept(e) if packed is not None else e)[None])
        yield b, h, f64(out[b, h * G:(h + 1) * G]), ref, np.concatenate(rows), st


def check(got, ref, rows, where):
    """Infinities and what is not a number as in the reference.  The rest: half a step of bf16, and for probabilities held in 16 bits and
    more 2^-15 of the largest finite value that is attended (scores of a few units: 2^-18 of a probability, its two terms 2^-17 of it)."""
    largest = np.abs(rows[np.isfinite(rows)]).max()
    assert np.isfinite(largest)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), where
    assert np.array_equal(got[np.isinf(ref)], ref[np.isinf(ref)]), where
    fine = np.isfinite(ref)
    err = np.abs(got[fine] - ref[fine])
    assert (err <= 2.0 ** -8 * np.abs(ref[fine]) + 2.0 ** -15 * largest).all(), (where, float(err.max()))


# sequences, KV heads, window, budget, heads checked: every n-th
FORMS = {"four waves": (150, 2, 45, 70, 29), "few on four waves": (20, 2, 70, 100, 7), "eight waves": (70, 2, 70, 100, 23),
         "shares": (2, 2, 100, 2300, 1)}


@pytest.mark.parametrize("packed", [False, True], ids=["rows", "packed"])
@pytest.mark.parametrize("G", [1, 4, 5, 6, 8, 9, 17])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form", FORMS)
def test_infinite_values(form, D, G, packed):
    """A visible infinite value makes its column infinite (NaN where two of them cancel) and leaves the other columns alone."""
    nb, Hkv, window, budget, every = FORMS[form]
    cfg = B.make_cfg(G * Hkv, Hkv, D, window, budget, 2, 1e-3, 0.07, "bf16")
    cache = make_state(cfg, [window + budget + 11 + i for i in range(nb)], [budget] * nb, 41)
    rng = np.random.default_rng(42)
    segments = [cache.v_win] if packed else [cache.v_win, cache.v_ret]         # (a packed group with an infinity is NaN)
    for c in range(0, 40, 2):
        x = segments[c // 2 % len(segments)]
        x[:, :, rng.integers(x.shape[2]), c] = INF if c % 4 else -INF
    cache.v_win[:, :, 3, 50], cache.v_win[:, :, 30, 50] = INF, -INF
    cache.v_win[:, :, 17, 51] = float("nan")
    cache.v_win[:, :, 5, 52] = INF
    pk = B.ltea_kept_pack(cfg, cache) if packed else None
    seen = 0
    for by_mass in (True, False) if packed else (True,):
        cache.n_scored.copy_(cache.n_seen)
        for b, h, got, ref, rows, _ in one_step(cfg, cache, pk, by_mass, 43, every, added_infinity=45):
            check(got, ref, rows, (b, h))
            seen += int(np.isinf(ref).any()) + int(np.isfinite(ref).any())
    assert seen > 0


@pytest.mark.parametrize("packed", [False, True], ids=["rows", "packed"])
@pytest.mark.parametrize("G", [2, 7])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_that_go_hold_anything(D, G, packed):
    """The output next to a row that is dropped, and to one that is displaced, is finite and right to the same bound."""
    cfg = B.make_cfg(2 * G, 2, D, 40, 50, 0, 0.0, 0.0, "bf16")
    cache = make_state(cfg, [200, 200, 200], [50, 50, 50], 17)
    slot = 200 % 40
    cache.win_score[0, :, slot] = 0.0                                  # dropped by the threshold
    cache.k_win[0, :, slot], cache.v_win[0, :, slot] = INF, float("nan")
    cache.win_score[1, :, slot] = 5.0                                  # displaces the lowest
    cache.ret_score[1, :, 9] = 1e-6
    cache.k_ret[1, :, 9], cache.v_ret[1, :, 9] = float("nan"), INF
    cache.win_score[2, :, slot] = 5.0
    cache.ret_score[2, :, 33] = 1e-6
    cache.k_ret[2, :, 33], cache.v_ret[2, :, 33] = -INF, -INF
    pk = B.ltea_kept_pack(cfg, cache) if packed else None
    for b, h, got, ref, rows, st in one_step(cfg, cache, pk, True, 600, 1):
        assert st["dst"] == (None, 9, 33)[b] and np.isfinite(rows).all() and np.isfinite(ref).all()
        check(got, ref, rows, (b, h))


@pytest.mark.parametrize("segment", ["ring", "kept"])
@pytest.mark.parametrize("G", [1, 4, 5, 6, 8, 16, 17])
@pytest.mark.parametrize("D", [64, 128])
def test_probabilities_keep_32_bits(D, G, segment):
    """Three rows whose values cancel: two correct, to 8 bits each, what the first leaves, so that the output is below 2^-14 of the terms and
    its own rounding below 2^-22 of them.  What shows is the probabilities' precision.

    A score is the product of two bf16 values, exact.  Its exponent is a product with a rounded scale minus a rounded reference, of size
    up to 3: three roundings of 3 * 2^-24, 2^-21.3 of a probability by ln 2, and the exponential's and the sum's own, 2^-22 together.
    Bar 2^-20 of the terms; probabilities cut to 16 bits are off by up to 2^-17 of theirs."""
    rng = np.random.default_rng(8 * D + G)
    bf = lambda x: torch.as_tensor(np.asarray(x), dtype=torch.float64).to(torch.bfloat16).double().numpy()
    cfg = B.make_cfg(G, 1, D, 40, 40, 0, 0.0, 0.25, "bf16")
    kept = segment == "kept"
    cache = make_state(cfg, [43 if kept else 3], [3 if kept else 0], 44)
    # the query looks at channel 0: scores of a quarter of the product; the incoming token far below
    heads = bf(rng.uniform(1.0, 1.5, G))
    q, k = np.zeros((1, G, D)), np.zeros((1, 1, D))
    q[0, :, 0], k[0, 0, 0] = heads, -400.0
    keys = bf(rng.uniform(-4.0, 0.0, 3))
    x = 0.25 * heads[:, None] * keys[None]
    p = np.exp(x)                                                             # [G, 3]
    v = np.zeros((3, D))
    v[0] = bf(rng.standard_normal(D))
    for i in (1, 2):                                                          # channel d cancels for query head d % G
        for d in range(D):
            v[i, d] = bf(-(p[d % G, :i] @ v[:i, d]) / p[d % G, i])
    put = lambda a, dt=torch.bfloat16: torch.from_numpy(np.ascontiguousarray(a)).to(dtype=dt, device="cuda")
    if kept:                                                                  # a ring of rows that count nothing beside them
        cache.k_win[...] = 0.0
        cache.k_win[..., 0] = -400.0
        cache.v_win[...] = 0.0
    to_k, to_v = (cache.k_ret, cache.v_ret) if kept else (cache.k_win, cache.v_win)
    to_k[0, 0, :3] = 0.0
    to_k[0, 0, :3, 0], to_v[0, 0, :3] = put(keys), put(v)
    cache.win_score[...] = 0.0                                                # (what leaves is dropped)
    got = f64(B.ltea_decode_step_mass(cfg, put(q), put(k), put(np.zeros((1, 1, D))), cache))[0]
    total = p.sum(1, keepdims=True)
    ref, terms = (p @ v) / total, (p @ np.abs(v)) / total
    own = np.arange(D) % G == np.arange(G)[:, None]
    assert (np.abs(ref[own]) <= 2.0 ** -14 * terms[own]).all()
    err = np.abs(got - ref)
    assert (err <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -20 * terms)[own].all(), float((err / terms)[own].max() * 2 ** 20)


def check_added(got, before, after, where):
    """Keys against what they were and what 64 bits add: half a step of fp32 of the sum and 2^-15 of the weight that is added, whatever the
    key.  (A weight: 2^-18 of each of its probabilities, as in check(), their sum's and their normaliser's roundings; the numbers of some
    ten below 2^-126 that a probability in fp32 cannot be count as nothing.)"""
    fine = np.isfinite(after)
    assert np.array_equal(np.isinf(got), np.isinf(after)), where
    added = after[fine] - before[fine]
    err = np.abs(got[fine] - after[fine])
    assert (err <= 2.0 ** -24 * after[fine] + 2.0 ** -15 * added + 2.0 ** -120).all(), (where, float((err / after[fine]).max()))
    return float(np.median(added))


@pytest.mark.parametrize("packed", [False, True], ids=["rows", "packed"])
@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("small_keys", [False, True], ids=["keys", "small keys"])
@pytest.mark.parametrize("nb,G,window,budget,every", [(2, 2, 60, 5000, 1), (1, 8, 300, 3000, 1), (150, 4, 45, 70, 41), (60, 9, 70, 100, 17)])
def test_added_weights(nb, G, window, budget, every, small_keys, dtype, D, packed):
    """What a step adds to the keys of ring and kept entries, also where it is a small part of them."""
    cfg = B.make_cfg(2 * G, 2, D, window, budget, 1, 0.0, 0.0, dtype)
    cache = make_state(cfg, [window + budget + 5 + i for i in range(nb)], [budget] * nb, 45)
    if small_keys:
        cache.win_score.mul_(2.0 ** -20), cache.ret_score.mul_(2.0 ** -20)
    pk = B.ltea_kept_pack(cfg, cache) if packed else None
    before = clone(cache)
    medians = []
    for b, h, _, _, _, st in one_step(cfg, cache, pk, True, 46, every):
        slot, win, ret = int(before.n_seen[b]) % window, f64(before.win_score[b, h]), f64(before.ret_score[b, h])
        if st["dst"] is not None:
            ret[st["dst"]] = win[slot]
        win[slot] = 0.0
        medians += [check_added(f64(cache.win_score[b, h]), win, st["win_key"], (b, h)),
                    check_added(f64(cache.ret_score[b, h]), ret, st["ret_key"], (b, h))]
    assert 0 < min(medians) and max(medians) < 0.2
