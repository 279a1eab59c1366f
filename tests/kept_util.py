"""Inputs and state of the steps over kept entries, read back from the device and compared with the oracle head by head."""
import numpy as np
import torch

from oracle import kept_oracle as ko
from paper_2510_20787_amd import binding as B

FIELDS = ("k_win", "v_win", "win_score", "k_ret", "v_ret", "ret_score", "ret_pos", "ret_count", "n_seen", "n_scored")


def clone(cache):
    return B.wrap_cache(*[getattr(cache, f).clone() for f in FIELDS])


def f64(x):
    return x.detach().double().cpu().numpy()


def make_state(cfg, seen, counts, seed, device="cuda"):
    """A cache of len(seen) sequences: seen tokens consumed, counts[b] (or [b][h]) entries kept.  What is not there holds NaN."""
    td = torch.float32 if cfg.dtype == B.LTEA_F32 else torch.bfloat16
    rng = np.random.default_rng(seed)
    nb, H, w, b, D = len(seen), cfg.Hkv, cfg.window, cfg.budget, cfg.D
    arr = dict(k_win=rng.standard_normal((nb, H, w, D)), v_win=rng.standard_normal((nb, H, w, D)),
               k_ret=rng.standard_normal((nb, H, max(b, 1), D)), v_ret=rng.standard_normal((nb, H, max(b, 1), D)))
    win = np.exp(rng.uniform(-6, 1, (nb, H, w)))
    ret = np.exp(rng.uniform(-6, 1, (nb, H, max(b, 1))))
    pos = np.full((nb, H, max(b, 1)), -7)
    cnt = np.broadcast_to(np.asarray(counts).reshape(nb, -1), (nb, H)).copy()
    for s in range(nb):
        for h in range(H):
            n = int(cnt[s, h])
            out = max(0, seen[s] - w)
            assert n <= min(b, out)
            pos[s, h, :n] = np.sort(rng.choice(out, n, replace=False))
            rng.shuffle(pos[s, h, :n])
            ret[s, h, :n][pos[s, h, :n] < cfg.sink] = np.inf
            for name in ("k_ret", "v_ret"):
                arr[name][s, h, n:] = np.nan
            ret[s, h, n:] = np.nan
            for name in ("k_win", "v_win"):
                arr[name][s, h, seen[s]:] = np.nan
            win[s, h, seen[s]:] = np.nan
    put = lambda x, dt: torch.from_numpy(np.ascontiguousarray(x)).to(dtype=dt, device=device)
    return B.wrap_cache(put(arr["k_win"], td), put(arr["v_win"], td), put(win, torch.float32), put(arr["k_ret"], td),
                        put(arr["v_ret"], td), put(ret, torch.float32), put(pos, torch.int32), put(cnt, torch.int32),
                        put(np.array(seen), torch.int32), put(np.array(seen), torch.int32))


def step_inputs(cfg, n_seqs, seed, device="cuda"):
    td = torch.float32 if cfg.dtype == B.LTEA_F32 else torch.bfloat16
    rng = np.random.default_rng(seed)
    return [torch.from_numpy(rng.standard_normal((n_seqs, h, cfg.D))).to(dtype=td, device=device) for h in (cfg.Hq, cfg.Hkv, cfg.Hkv)]


def kept_values(cfg, packed, b, h, count):
    """The values that a head's packed rows stand for."""
    blocks = packed[b, h].cpu().numpy()
    parts = [ko.read_block(blocks[i], cfg.D) for i in range((count + 31) // 32)]
    if not parts:
        return np.zeros((0, cfg.D)), np.zeros((0, cfg.D))
    kc, vc, ke, ve = (np.concatenate(x)[:count] for x in zip(*parts))
    return ko.decode(kc, ke), ko.decode(vc, ve)


# How far a result may be from 64 bits.  Scores: products of bf16 are exact, sums of at most 128 fp32 terms of size |q||k|/D each and
# the exponent's rounding leave 2^-18 of relative error in a probability at most (exponents of a few units); the bf16 value and the
# bf16 remainder of a probability hold 2^-17 of it.  Together under 2^-15 of the largest value, and the output's own rounding, half a step.
def check_out(got, ref, vmax, dtype):
    half_step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    err = np.abs(got - ref)
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    ok = err <= half_step * np.abs(ref) + 2.0 ** -15 * vmax
    assert ok[~np.isnan(ref)].all(), float(np.nanmax(err))


# A key: fp32 rounding of the sum, and 2^-15 of the weight that was added.
def check_key(got, ref, what):
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(np.isinf(got), np.isinf(ref)), what
    plain = np.isfinite(ref)
    err = np.abs(got[plain] - ref[plain])
    assert (err <= 2.0 ** -15 * np.minimum(np.abs(ref[plain]), 16) + 2.0 ** -30).all(), (what, float(err.max()))


def run_and_check(cfg, cache, packed, by_mass, seed, dtype, workspace=None, heads=None):
    """One step on the device, every (sequence, KV head) against the oracle started from the device's own state."""
    nb = cache.n_seen.numel()
    before, packed_before = clone(cache), None if packed is None else packed.clone()
    q, k, v = step_inputs(cfg, nb, seed)
    if by_mass:
        out = B.ltea_decode_step_mass(cfg, q, k, v, cache, packed=packed, workspace=workspace)
    else:
        out = B.ltea_decode_step_packed(cfg, q, k, v, cache, packed, workspace=workspace)
    torch.cuda.synchronize()
    G = cfg.Hq // cfg.Hkv
    sigma = cfg.softmax_scale if cfg.softmax_scale > 0 else cfg.D ** -0.5
    pairs = [(b, h) for b in range(nb) for h in range(cfg.Hkv)]
    for b, h in pairs if heads is None else [p for i, p in enumerate(pairs) if i % heads == 0]:
        t, n = int(before.n_seen[b]), int(before.ret_count[b, h])
        if packed is None:
            kr, vr = f64(before.k_ret[b, h, :n]), f64(before.v_ret[b, h, :n])
        else:
            kr, vr = kept_values(cfg, packed_before, b, h, n)
        ref, st = ko.kept_step(f64(q[b, h * G:(h + 1) * G]), f64(k[b, h]), f64(v[b, h]), f64(before.k_win[b, h]), f64(before.v_win[b, h]),
                               f64(before.win_score[b, h]), kr, vr, f64(before.ret_score[b, h, :n]), f64(before.ret_pos[b, h, :n]), t,
                               cfg.window, cfg.budget, cfg.sink, cfg.tau_logit, sigma, by_mass, packed is not None)
        where = f"sequence {b} head {h} t {t} count {n} dst {st['dst']}"
        live = min(t + 1, cfg.window)
        vmax = max(float(np.nanmax(np.abs(st["v_win"][:live]))), float(np.nanmax(np.abs(vr))) if n else 0.0, 6.0)
        check_out(f64(out[b, h * G:(h + 1) * G]), ref, vmax, dtype)
        assert np.array_equal(f64(cache.k_win[b, h]), st["k_win"], equal_nan=True), where
        assert np.array_equal(f64(cache.v_win[b, h]), st["v_win"], equal_nan=True), where
        if by_mass:
            check_key(f64(cache.win_score[b, h, :live]), st["win_key"][:live], where)
            assert np.array_equal(f64(cache.win_score[b, h, live:]), f64(before.win_score[b, h, live:]), equal_nan=True), where
        else:
            assert np.array_equal(f64(cache.win_score[b, h]), f64(before.win_score[b, h]), equal_nan=True), where
        m = len(st["ret_pos"])
        assert int(cache.ret_count[b, h]) == m, where
        assert np.array_equal(f64(cache.ret_pos[b, h, :m]), st["ret_pos"]), where
        check_key(f64(cache.ret_score[b, h, :m]), st["ret_key"], where)
        # slots that nothing was written to are as they were, the others hold the leaving token's row
        for i in range(max(cfg.budget, 0)):
            if i == st["dst"]:
                ek, ev = f64(before.k_win[b, h, t % cfg.window]), f64(before.v_win[b, h, t % cfg.window])
                if packed is None:
                    assert np.array_equal(f64(cache.k_ret[b, h, i]), ek, equal_nan=True) and np.array_equal(f64(cache.v_ret[b, h, i]), ev, equal_nan=True), where
                else:
                    kc, vc, ke, ve = (x[i % 32] for x in ko.read_block(packed[b, h, i // 32].cpu().numpy(), cfg.D))
                    for got, want in ((kc, ke), ko.encode(ek)), ((vc, ve), ko.encode(ev)):
                        assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1]), where
        if st["dst"] is None:
            same = packed is None or torch.equal(packed[b, h], packed_before[b, h])
            assert same, where
            if packed is None and cfg.budget:
                assert np.array_equal(f64(cache.k_ret[b, h]), f64(before.k_ret[b, h]), equal_nan=True), where
        elif packed is None:
            rest = [i for i in range(cfg.budget) if i != st["dst"]]
            assert np.array_equal(f64(cache.v_ret[b, h, rest]), f64(before.v_ret[b, h, rest]), equal_nan=True), where
        else:
            rest = [i for i in range(packed.shape[2]) if i != st["dst"] // 32]
            assert torch.equal(packed[b, h, rest], packed_before[b, h, rest]), where
    assert torch.equal(cache.n_seen, before.n_seen + 1)
    assert torch.equal(cache.n_scored, cache.n_seen if by_mass else before.n_scored)
    return out
