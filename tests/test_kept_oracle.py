"""What pins the fp64 statement of eviction by accumulated weight and of rows in 4 bits (CPU): independent definitions, closed forms,
differences, and planted mistakes that the pins must notice."""
import numpy as np
import pytest

from oracle import kept_oracle as ko


def rows(rng, *shape):
    return rng.standard_normal(shape)


def mass_by_differences(q, k, window, last, sigma, eps=1e-5):
    """The weight of a token is the derivative of the counting queries' log normalisers with respect to a bias on its scores."""
    n, Hq, _ = q.shape
    Hkv = k.shape[1]
    out = np.zeros((Hkv, n))
    ago = np.arange(n)[:, None] - np.arange(n)[None, :]
    seen = (ago >= 0) & (ago < window)
    first = n - last if last > 0 else 0
    for h in range(Hkv):
        for j in range(n):
            for sign in (1, -1):
                bias = np.zeros(n)
                bias[j] = sign * eps
                for g in range(Hq // Hkv):
                    s = np.where(seen, sigma * (q[:, h * (Hq // Hkv) + g] @ k[:, h].T) + bias, -np.inf)
                    lse = np.logaddexp.reduce(s, axis=1)
                    out[h, j] += sign * lse[max(first, 0):].sum() / (2 * eps)
    return out


@pytest.mark.parametrize("window,last", [(40, 0), (5, 0), (40, 7), (6, 50), (1, 1)])
def test_weights_are_derivatives_of_the_normalisers(window, last):
    rng = np.random.default_rng(1)
    q, k = rows(rng, 23, 4, 8), rows(rng, 23, 2, 8)
    lse = ko.causal_lse(q, k, window, 0.3)
    got = ko.attention_mass(q, k, lse, window, last, 0.3)
    # central differences of lse: third derivative at most 1, eps^2 / 6 each, and 2^-50 / eps of rounding per term
    assert np.abs(got - mass_by_differences(q, k, window, last, 0.3)).max() < 23 * 2 * 1e-9
    n_counting = min(last, 23) if last > 0 else 23
    assert abs(got.sum() - 4 * n_counting) < 1e-9                   # every query spends weight one per head
    wrong = ko.attention_mass(q, k, lse, window + 1, last, 0.3)
    assert window >= 23 or np.abs(wrong - got).max() > 1e-3         # a window off by one is noticed


def test_queries_without_a_normaliser_count_nothing():
    rng = np.random.default_rng(2)
    q, k = rows(rng, 9, 1, 8), rows(rng, 9, 1, 8)
    lse = ko.causal_lse(q, k, 9, 1.0)
    whole = ko.attention_mass(q, k, lse, 9, 0, 1.0)
    for bad in (np.nan, np.inf, -np.inf):
        x = lse.copy()
        x[0, 4] = bad
        less = ko.attention_mass(q, k, x, 9, 0, 1.0)
        assert abs(whole.sum() - less.sum() - 1.0) < 1e-12 and np.isfinite(less).all()


def test_four_bit_values():
    eight = np.concatenate([ko.VALUES, -ko.VALUES, np.zeros(16)])
    for E in (-100, -2, 0, 3, 124):
        codes, byte = ko.encode(eight * 2.0 ** E)
        assert np.array_equal(ko.decode(codes, byte), eight * 2.0 ** E)       # exact values stay
        # the largest is 6 = 1.5 * 2^2: E = 2 - 2
        assert byte[0] == E + 127
    rng = np.random.default_rng(3)
    x = rows(rng, 50, 128) * 2.0 ** rng.integers(-60, 60, (50, 1))
    codes, byte = ko.encode(x)
    back = ko.decode(codes, byte)
    again = ko.encode(back)
    assert np.array_equal(again[0] & 7, codes & 7) and np.array_equal(ko.decode(*again), back)
    # of all multiples the nearest, unless the quotient is past 6
    grid = np.concatenate([-ko.VALUES, ko.VALUES])
    scale = np.repeat(2.0 ** (byte.astype(float) - 127), 32, axis=1)
    best = np.abs(x[..., None] / scale[..., None] - grid).min(axis=-1)
    assert np.allclose(np.abs(x - back) / scale, best, rtol=0, atol=1e-12)
    top = np.abs(x.reshape(50, 4, 32)).max(-1) / 2.0 ** (byte.astype(float) - 127)
    assert (top > 3.5).all() and (top <= 7.0).all()                             # m in (1.75, 2) * 2 or [1, 1.75] * 4
    assert np.array_equal(ko.decode(*ko.encode(2 * x)), 2 * back)


def test_halfway_goes_to_the_even_code_and_ends():
    x = np.zeros(32)
    x[:9] = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.0]
    x[9] = 6.5
    codes, byte = ko.encode(x)
    assert byte[0] == 127 and codes[:10].tolist() == [6, 0, 2, 2, 4, 4, 6, 6, 14, 7]
    for bad in (np.nan, np.inf):
        y = x.copy()
        y[20] = bad
        codes, byte = ko.encode(y)
        assert byte[0] == 255 and (codes == 7).all() and np.isnan(ko.decode(codes, byte)).all()
    codes, byte = ko.encode(np.full(32, -2.0 ** -121))
    assert byte[0] == 127 and (codes == 8).all() and not ko.decode(codes, byte).any()


@pytest.mark.parametrize("D", [64, 128])
def test_places_of_a_block_cover_it_once(D):
    code = sorted(p for r in range(32) for d in range(0, D, 2) for p in ko.code_places(r, d, D))
    exps = sorted(p for r in range(32) for g in range(D // 32) for p in ko.exponent_places(r, g, D))
    assert code == list(range(32 * D)) and exps == list(range(32 * D, 34 * D))


def run_steps(n, window, budget, sink, tau, by_mass, given=None, packed=False, seed=4, G=2, D=32):
    """n steps from an empty cache; returns every step's output, the final state and the inputs."""
    rng = np.random.default_rng(seed)
    q, k, v = rows(rng, n, G, D), rows(rng, n, D), rows(rng, n, D)
    kw, vw, key = np.zeros((window, D)), np.zeros((window, D)), np.zeros(window)
    kr, vr, rk, rp = np.zeros((0, D)), np.zeros((0, D)), np.zeros(0), np.zeros(0, int)
    outs = []
    for t in range(n):
        if given is not None and t >= window:
            key[t % window] = given[t - window]
        out, s = ko.kept_step(q[t], k[t], v[t], kw, vw, key, kr, vr, rk, rp, t, window, budget, sink, tau, D ** -0.5, by_mass, packed)
        dst = s["dst"]
        if dst is not None:
            e = t - window
            row = [ko.as_kept(x[e]) if packed else x[e] for x in (k, v)]
            if dst == len(kr):
                kr, vr = np.vstack([kr, row[0]]), np.vstack([vr, row[1]])
            else:
                kr[dst], vr[dst] = row
        kw, vw, key, rk, rp = s["k_win"], s["v_win"], s["win_key"], s["ret_key"], s["ret_pos"]
        outs.append(out)
    return np.array(outs), dict(key=key, ret_key=rk, ret_pos=rp), (q, k, v)


@pytest.mark.parametrize("n,window,budget,sink", [(30, 5, 4, 0), (40, 7, 6, 2), (12, 20, 4, 1), (25, 1, 1, 0), (20, 6, 0, 2)])
def test_steps_by_weight_against_the_whole_history(n, window, budget, sink):
    """Sets of positions and sums of probabilities, kept without rings or slots."""
    outs, state, (q, k, v) = run_steps(n, window, budget, sink, 0.0, True)
    got = {}                                      # position -> weight received while it was visible
    kept = {}                                     # position -> its key
    for t in range(n):
        e = t - window
        if e >= 0 and budget > 0:
            key = np.inf if e < sink else np.float32(got[e])
            if len(kept) < budget:
                kept[e] = key
            else:
                low = min(kept, key=lambda p: (np.float32(kept[p]), -p))
                if key > np.float32(kept[low]):
                    del kept[low]
                    kept[e] = key
        seen = [j for j in range(max(0, t - window + 1), t + 1)] + sorted(kept)
        s = (q[t] @ k[seen].T) * k.shape[1] ** -0.5
        p = np.exp(s - s.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        assert np.allclose(outs[t], p @ v[seen], atol=1e-12)
        got[t] = 0.0
        for j, w in zip(seen, p.sum(0)):
            if j in kept and j <= t - window:
                kept[j] = kept[j] + w
            else:
                got[j] += w
    assert sorted(state["ret_pos"].tolist()) == sorted(kept)
    order = np.argsort(state["ret_pos"])
    assert np.allclose(np.sort(state["ret_key"][order]), np.sort([kept[p] for p in sorted(kept)]), rtol=1e-6)
    for j in range(max(0, n - window), n):
        assert abs(state["key"][j % window] - got[j]) < 1e-9


def test_steps_by_given_keys_keep_the_largest():
    """The streaming rule keeps what one selection over all tokens that have left would keep."""
    rng = np.random.default_rng(5)
    n, window, budget, sink, tau = 60, 8, 10, 2, 0.1
    z = rng.standard_normal(n).astype(np.float32)
    _, state, _ = run_steps(n, window, budget, sink, tau, False, given=z)
    out = np.arange(n - window)
    cand = [j for j in out if j < sink or z[j] > np.float32(tau)]
    best = sorted(cand, key=lambda j: (-(np.inf if j < sink else z[j]), j))[:budget]
    assert sorted(state["ret_pos"].tolist()) == sorted(best)


def test_packed_rows_are_attended_as_they_are_kept():
    a, sa, (q, k, v) = run_steps(30, 5, 40, 0, 0.0, True, packed=True)
    seen = np.concatenate([ko.as_kept(k[:25]), k[25:]]), np.concatenate([ko.as_kept(v[:25]), v[25:]])
    p = ko.softmax_rows(q[29] @ seen[0].T * 32 ** -0.5)
    assert np.allclose(a[29], p @ seen[1], atol=1e-12)
    b, _, _ = run_steps(30, 5, 40, 0, 0.0, True, packed=False)
    assert np.allclose(a[:5], b[:5]) and np.abs(a[29] - b[29]).max() > 1e-4
