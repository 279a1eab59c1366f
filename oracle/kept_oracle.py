"""Plain fp64 statement of the cache that evicts by accumulated attention weight and of kept rows in 4 bits (NumPy, tests only).

An entry's key is the attention weight it has received, summed over the query heads of its KV head; the rules of eviction are
those of `ltea_oracle` with the key in the logit's place."""
from __future__ import annotations

import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def softmax_rows(s):
    m = s.max(axis=-1, keepdims=True, initial=-np.inf)
    p = np.exp(s - m)
    return p / p.sum(axis=-1, keepdims=True)


def attention_mass(q, k, lse, window, last, sigma):
    """q [n, Hq, D], k [n, Hkv, D], lse [Hq, n] of one sequence -> [Hkv, n]."""
    n, Hq, _ = q.shape
    Hkv = k.shape[1]
    ago = np.arange(n)[:, None] - np.arange(n)[None, :]
    counts = (ago >= 0) & (ago < window)
    if last > 0:
        counts &= (np.arange(n) >= n - last)[:, None]
    mass = np.zeros((Hkv, n))
    for hq in range(Hq):
        h = hq // (Hq // Hkv)
        good = np.isfinite(lse[hq])
        with np.errstate(over="ignore", invalid="ignore"):
            p = np.exp(sigma * (q[:, hq] @ k[:, h].T) - lse[hq][:, None])
        mass[h] += np.where(counts & good[:, None], p, 0.0).sum(axis=0)
    return mass


def causal_lse(q, k, window, sigma):
    """Log normalisers [Hq, n] of the queries of one sequence over the keys in their window."""
    n, Hq, _ = q.shape
    G = Hq // k.shape[1]
    ago = np.arange(n)[:, None] - np.arange(n)[None, :]
    out = np.zeros((Hq, n))
    for hq in range(Hq):
        s = np.where((ago >= 0) & (ago < window), sigma * (q[:, hq] @ k[:, hq // G].T), -np.inf)
        m = s.max(axis=1, initial=-np.inf)
        out[hq] = m + np.log(np.exp(s - m[:, None]).sum(axis=1))
    return out


# ---- 4-bit rows ------------------------------------------------------------------------------------------------------------
def encode(x):
    """x [..., D] -> codes [..., D] (0..15) and exponent bytes [..., D / 32]."""
    x = np.asarray(x, np.float64)
    g = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    codes = np.zeros(g.shape, np.uint8)
    byte = np.zeros(g.shape[:-1], np.uint8)
    for at in np.ndindex(*byte.shape):
        v = g[at]
        top = np.abs(v).max()
        sign = np.signbit(v).astype(np.uint8) << 3
        if not np.isfinite(v).all():
            codes[at], byte[at] = 7, 255
        elif top < 2.0 ** -120:
            codes[at], byte[at] = sign, 127
        else:
            m, e = np.frexp(top)                         # m in [0.5, 1)
            E = int(e) - 1 - 2 if 2 * m <= 1.75 or e == 128 else int(e) - 1 - 1
            a = np.minimum(np.abs(v) / 2.0 ** E, 6.0)
            far = np.abs(a[:, None] - VALUES)
            near = far.min(axis=1, keepdims=True)
            tied = far == near                           # at a halfway point both neighbours: the even code
            codes[at] = [min(np.flatnonzero(t), key=lambda c: c % 2) for t in tied] | sign
            byte[at] = E + 127
    return codes.reshape(x.shape), byte


def decode(codes, byte):
    mag = VALUES[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    g = mag.reshape(*mag.shape[:-1], mag.shape[-1] // 32, 32)
    scale = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))
    return (g * scale[..., None]).reshape(mag.shape)


def as_kept(x):
    return decode(*encode(x))


def code_places(r, d, D):
    """Byte offsets in its block of 32 slots of the codes of channel d of slot r: (K, V)."""
    a, j, b = r // 8, r // 4 % 2, r % 4
    if D == 128:
        k = (((j * 4 + d // 32) * 4 + a) * 4 + b) * 16 + d % 32 // 2
        v = (((j * 4 + a) * 16 + d // 8) * 4 + b) * 4 + d % 8 // 2
    else:
        k = (((d // 16 * 4 + a) * 4 + b) * 2 + j) * 8 + d % 16 // 2
        v = (((a * 16 + d // 4) * 2 + j) * 4 + b) * 2 + d % 4 // 2
    return k, 16 * D + v


def exponent_places(r, g, D):
    a, j, b = r // 8, r // 4 % 2, r % 4
    n = D // 32
    return 32 * D + ((a * 4 + b) * n + g) * 2 + j, 33 * D + ((a * n + g) * 2 + j) * 4 + b


def read_block(block, D):
    """One block's bytes [34 D] -> K codes, V codes [32, D], K, V exponent bytes [32, D / 32]."""
    kc, vc = np.zeros((32, D), np.uint8), np.zeros((32, D), np.uint8)
    ke, ve = np.zeros((32, D // 32), np.uint8), np.zeros((32, D // 32), np.uint8)
    for r in range(32):
        for d in range(D):
            k, v = code_places(r, d, D)
            kc[r, d], vc[r, d] = block[k] >> 4 * (d & 1) & 15, block[v] >> 4 * (d & 1) & 15
        for g in range(D // 32):
            k, v = exponent_places(r, g, D)
            ke[r, g], ve[r, g] = block[k], block[v]
    return kc, vc, ke, ve


# ---- one step of one (sequence, KV head) -------------------------------------------------------------------------------------
def kept_step(q, k_new, v_new, k_win, v_win, win_key, k_ret, v_ret, ret_key, ret_pos, t, window, budget, sink, tau, sigma,
              by_mass, packed):
    """q [G, D]; k_win, v_win [window, D], win_key [window]; k_ret, v_ret [count, D] (the values kept rows stand for), ret_key,
    ret_pos [count].  Keys are fp32.  Returns out [G, D] and the new state as a dict with `dst` (the compact slot that
    received the leaving token, or None)."""
    k_win, v_win, win_key = k_win.copy(), v_win.copy(), win_key.astype(np.float64)
    keys, pos = [np.float32(x) for x in ret_key], [int(p) for p in ret_pos]
    kr, vr = list(k_ret), list(v_ret)
    slot, e = t % window, t - window
    dst = None
    if e >= 0 and budget > 0 and (e < sink or np.float32(win_key[slot]) > np.float32(tau)):
        key = np.float32(np.inf) if e < sink else np.float32(win_key[slot])
        if len(keys) < budget:
            dst = len(keys)
            keys.append(None), pos.append(None), kr.append(None), vr.append(None)
        else:
            worst = min(range(budget), key=lambda i: (keys[i], -pos[i]))
            if key > keys[worst]:
                dst = worst
        if dst is not None:
            keys[dst], pos[dst] = key, e
            kr[dst], vr[dst] = (as_kept(k_win[slot]), as_kept(v_win[slot])) if packed else (k_win[slot].copy(), v_win[slot].copy())
    k_win[slot], v_win[slot] = k_new, v_new
    live = min(t + 1, window)
    K = np.concatenate([k_win[:live], np.array(kr).reshape(len(kr), -1)]) if kr else k_win[:live]
    V = np.concatenate([v_win[:live], np.array(vr).reshape(len(vr), -1)]) if vr else v_win[:live]
    p = softmax_rows(sigma * (q @ K.T))
    out = p @ V
    ret = np.array([float(x) for x in keys])
    if by_mass:
        w = np.where(np.isnan(p), 0.0, p).sum(axis=0)
        win_key[slot] = 0.0
        win_key[:live] += w[:live]
        ret = ret + w[live:]
    return out, dict(k_win=k_win, v_win=v_win, win_key=win_key, ret_key=ret, ret_pos=np.array(pos, np.int64), dst=dst)
