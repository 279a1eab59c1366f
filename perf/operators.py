"""Operators of a cache that evicts by accumulated attention weight and may hold its kept rows in 4 bits: the calls whose
speed matters to a user, their inputs, their unavoidable work, and their plain forms.

  weights   the attention weight that every token of a prompt has received (`ltea_attention_mass`)
  step      one decode step that evicts by accumulated weight, rows in the storage type (`ltea_decode_step_mass`)
  packed    one decode step over kept rows held in 4 bits, evicting by accumulated weight (`ltea_decode_step_mass`) or by given
            keys (`ltea_decode_step_packed`)
  pack      kept rows into 4 bits and back (`ltea_kept_pack`, `ltea_kept_unpack`)

Head shapes are those of `workloads.py`; windows, budgets and lengths run from one short prompt or one sequence to its largest
configuration, and for 4-bit rows to the budgets that they make room for.
"""
import math
import random

import torch

own = False

F32 = dict(dtype="f32", Hq=2, Hkv=2, D=64)
EVEN64 = dict(dtype="bf16", Hq=16, Hkv=16, D=64)
PAPER = dict(dtype="bf16", Hq=32, Hkv=8, D=64)
WIDE = dict(dtype="bf16", Hq=16, Hkv=16, D=128)
GROUPED = dict(dtype="bf16", Hq=32, Hkv=8, D=128)
LONG = dict(dtype="bf16", Hq=32, Hkv=32, D=128)


def listed():
    return [
        # the smallest call: one short fp32 prompt, as in a numerics check of a model
        dict(name="weights_f32_300", op="weights", B=1, n=300, ragged=0, window=0, last=0, fused=False, **F32),
        # an ordinary batch of prompts on the paper's grouped heads, every query counted
        dict(name="weights_paper_4x4096", op="weights", B=4, n=4096, ragged=0, window=0, last=0, fused=False, **PAPER),
        # prompts of a busy server packed without padding (q, k views of one projection's output), the last 256 queries of each counted
        dict(name="weights_ragged_12x6000", op="weights", B=12, n=6000, ragged=5, window=0, last=256, fused=True, **WIDE),
        # one whole document, every query counted
        dict(name="weights_long_32768", op="weights", B=1, n=32768, ragged=0, window=0, last=0, fused=False, **LONG),
        # interactive decode: one sequence
        dict(name="step_one", op="step", B=1, window=768, budget=512, sink=4, fill=1.0, **PAPER),
        # batched decode, 800 MB of cache read per step
        dict(name="step_wide_64", op="step", B=64, window=1024, budget=512, sink=0, fill=1.0, **WIDE),
        # interactive decode with a long kept set in 4 bits
        dict(name="packed_one_16384", op="packed", keys="mass", B=1, window=768, budget=16384, sink=4, fill=1.0, **PAPER),
        # batched decode, one query head per KV head, caches of different age
        dict(name="packed_16x4000", op="packed", keys="mass", B=16, window=1024, budget=4000, sink=0, fill=0.6, **WIDE),
        # a few sequences that evict by their learned scores, an odd budget
        dict(name="packed_scored_4x2001", op="packed", keys="given", B=4, window=768, budget=2001, sink=4, fill=1.0, **PAPER),
        # a busy server's batch by learned scores, 350 MB of cache read per step
        dict(name="packed_scored_32x8192", op="packed", keys="given", B=32, window=512, budget=8192, sink=4, fill=1.0, **GROUPED),
        # the kept rows of four prompts after their prefill
        dict(name="pack_4x500", op="pack", B=4, window=64, budget=500, sink=0, fill=0.7, **PAPER),
        # long kept sets: packed after a prefill, unpacked before the next chunk
        dict(name="pack_16x8192", op="pack", B=16, window=64, budget=8192, sink=0, fill=1.0, **GROUPED),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        op = rng.choice(["weights"] * 3 + ["step"] * 3 + ["packed"] * 4 + ["pack"])
        case = dict(op=op, **rng.choice([F32, EVEN64, PAPER, PAPER, WIDE, GROUPED, LONG]))
        f32 = case["dtype"] == "f32"
        if op == "weights":
            total = _log_int(rng, 64, 2048 if f32 else 49152)
            case["B"] = min(_log_int(rng, 1, 16), total // 32)
            case["n"] = min(total // case["B"], 24000)
            case["ragged"] = rng.randint(1, 1 << 20) if case["B"] > 1 and rng.random() < 0.6 else 0
            case["window"] = rng.choice([0, 0, rng.randint(1, case["n"])])
            case["last"] = rng.choice([0, 0, _log_int(rng, 1, 1024)])
            case["fused"] = rng.random() < 0.5
        else:
            case["B"] = _log_int(rng, 1, 4 if f32 else 64)
            case["window"] = _log_int(rng, 16, 2048)
            case["budget"] = _log_int(rng, 16, 2048 if op == "step" or f32 else 32768)
            case["sink"] = rng.choice([0, 1, 4])
            case["fill"] = rng.choice([1.0, 1.0, 0.5, 0.1])
            if op == "packed":
                case["keys"] = rng.choice(["mass", "given"])
        w = work(case)
        if w["flops"] <= 4.3e12 and 0 < w["bytes"] <= 8e8:
            return case


# ---- sizes -----------------------------------------------------------------------------------------------------------------
def _lengths(case):
    """Tokens per sequence of a packed batch."""
    if not case["ragged"]:
        return [case["n"]] * case["B"]
    r = random.Random(case["ragged"])
    return [r.randint(max(1, case["n"] // 16), case["n"]) for _ in range(case["B"])]


def _ages(case):
    """Tokens consumed and entries kept per sequence: at fill 1 all caches are full, below it their ages differ and the youngest
    are still filling their window."""
    w, b = case["window"], case["budget"]
    if case["fill"] >= 1.0:
        return [w + 3 * b + 37 * i for i in range(case["B"])], [b] * case["B"]
    r = random.Random(case["B"] * 1000003 + w * 1009 + b)
    seen = [r.randint(0, int((w + b) * 2 * case["fill"]) + 1) for _ in range(case["B"])]
    return seen, [min(b, max(0, n - w) * 2 // 3) for n in seen]


def _esz(case):
    return 4 if case["dtype"] == "f32" else 2


def _visible(n, window, last):
    """(query, key) pairs of one sequence: query i sees min(i + 1, window) keys, queries from n - last on."""
    w = min(window, n) if window > 0 else n
    upto = lambda m: m * (m + 1) // 2 if m <= w else w * (w + 1) // 2 + (m - w) * w     # of the first m queries
    return upto(n) - upto(max(0, n - last) if last > 0 else 0)


def work(case):
    D, Hq, Hkv, e = case["D"], case["Hq"], case["Hkv"], _esz(case)
    if case["op"] == "weights":
        ns = _lengths(case)
        counted = sum(min(n, case["last"]) if case["last"] > 0 else n for n in ns)
        reach = lambda n: min(n, case["last"] + case["window"] - 1) if case["last"] > 0 and case["window"] > 0 else n
        bytes_ = Hq * counted * (D * e + 4) + Hkv * sum(reach(n) for n in ns) * D * e + Hkv * sum(ns) * 4
        return dict(bytes=float(bytes_), flops=2.0 * D * Hq * sum(_visible(n, case["window"], case["last"]) for n in ns))
    seen, kept = _ages(case)
    row, packed_row = 2 * D * e, 2 * (D // 2 + D // 32)
    if case["op"] == "pack":         # one way and back
        return dict(bytes=float(Hkv * sum(kept) * 2 * (row + packed_row)), flops=float(Hkv * sum(kept) * 4 * D))
    ring = sum(min(n + 1, case["window"]) for n in seen)
    keys = 8 if case["op"] == "step" or case["keys"] == "mass" else 4      # read, and written back where weights are added
    per_kept = (packed_row if case["op"] == "packed" else row) + keys
    bytes_ = Hkv * (ring * (row + keys - 4) + sum(kept) * per_kept) + case["B"] * (2 * Hq * D * e + 2 * Hkv * 2 * D * e)
    return dict(bytes=float(bytes_), flops=4.0 * D * Hq * (ring + sum(kept)))


# ---- inputs ----------------------------------------------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _storage(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def prepare(case, seed):
    g = _gen(seed)
    return _prepare_weights(case, g) if case["op"] == "weights" else _prepare_cache(case, g)


def _prepare_weights(case, g):
    """Queries that look for something: every key carries a share of a direction common to its head, some tokens more of it."""
    dt, D, Hq, Hkv = _storage(case), case["D"], case["Hq"], case["Hkv"]
    ns = _lengths(case)
    T = sum(ns)
    cu = torch.tensor([0] + ns, device="cuda").cumsum(0).to(torch.int32)
    if case["fused"]:
        both = _normal(g, (T, Hq + 2 * Hkv, D), dt)
        q, k = both[:, :Hq], both[:, Hq:Hq + Hkv]
    else:
        q, k = _normal(g, (T, Hq, D), dt), _normal(g, (T, Hkv, D), dt)
    common = _normal(g, (1, Hkv, D), torch.float32)
    pull = torch.rand((T, Hkv, 1), generator=g, device="cuda").pow(4)
    k.copy_((k.float() + pull * common).to(dt))
    q.copy_((q.float() + 0.5 * common.repeat_interleave(Hq // Hkv, 1)).to(dt))
    window = case["window"] if case["window"] > 0 else max(ns)
    lse = torch.empty((Hq, T), dtype=torch.float32, device="cuda")
    lo = 0
    for n in ns:
        _per_query_block(q[lo:lo + n], k[lo:lo + n], window, 0, torch.float32,
                         lambda s, i0, j0, lo=lo: lse[:, lo + i0:lo + i0 + s.shape[2]].copy_(torch.logsumexp(s, 3).reshape(Hq, -1)))
        lo += n
    return dict(case=case, q=q, k=k, cu=cu, ns=ns, window=window, last=case["last"], lse=lse,
                mass=torch.empty((Hkv, T), dtype=torch.float32, device="cuda"))


def _prepare_cache(case, g):
    dt, D, Hq, Hkv, B, w, b = _storage(case), case["D"], case["Hq"], case["Hkv"], case["B"], case["window"], case["budget"]
    seen, kept = _ages(case)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    n_seen, count = i32(seen), i32(kept)
    s = dict(case=case, n_seen=n_seen, n_scored=n_seen.clone(), ret_count=count[:, None].repeat(1, Hkv).contiguous())
    kinds = ("k_ret", "v_ret") if case["op"] == "pack" else ("k_win", "v_win", "k_ret", "v_ret")
    for name in kinds:
        # channels of unequal size, as keys have them
        width = 0.3 + 1.4 * torch.rand((1, Hkv, 1, D), generator=g, device="cuda")
        s[name] = _normal(g, (B, Hkv, w if name.endswith("win") else b, D), torch.float32).mul_(width).to(dt)
    weight = lambda n: torch.rand((B, Hkv, n), generator=g, device="cuda").mul(7.0).sub(6.0).exp()
    s["win_score"], s["ret_score"] = weight(w), weight(b)
    if case["op"] == "packed" and case["keys"] == "given":
        s["win_score"], s["ret_score"] = s["win_score"].log(), s["ret_score"].add(0.01)
    # kept positions: distinct, below what is still in the window, the sinks among them
    span = (n_seen[:, None] - w).clamp(min=0).double() / count[:, None].clamp(min=1).double()
    pos = (torch.arange(b, device="cuda")[None] * span).floor().to(torch.int32)
    s["ret_pos"] = pos[:, None].repeat(1, Hkv, 1).contiguous()
    s["ret_score"] = torch.where(s["ret_pos"] < case["sink"], torch.full_like(s["ret_score"], math.inf), s["ret_score"])
    if case["op"] in ("packed", "pack"):
        s["packed"] = _encode_all(s["k_ret"], s["v_ret"])
    if case["op"] == "packed":
        del s["k_ret"], s["v_ret"]
    if case["op"] == "pack":
        s["k_out"], s["v_out"] = torch.zeros_like(s["k_ret"]), torch.zeros_like(s["v_ret"])
        return s
    s["q"], s["k"], s["v"] = (_normal(g, (B, h, D), dt) for h in (Hq, Hkv, Hkv))
    s["out"] = torch.empty((B, Hq, D), dtype=dt, device="cuda")
    s["until_scored"] = w        # steps until the ring's tokens need new scores
    return s


# ---- 4-bit rows ------------------------------------------------------------------------------------------------------------
# A value is +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} times a power of two that 32 channels of a row share; the layout is the header's.
_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _power(e):
    """2^e for whole e from -126 to 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _encode(x):
    """x [..., D] -> codes [..., D] (0..15), exponent bytes [..., D / 32]."""
    g = x.float().unflatten(-1, (-1, 32))
    top = g.abs().amax(-1)
    bad, tiny = ~torch.isfinite(top), top < 2.0 ** -120
    m, k = torch.frexp(torch.where(bad | tiny, torch.ones_like(top), top))       # top = m * 2^k, m in [0.5, 1)
    e = torch.where((m <= 0.875) | (k == 128), k - 3, k - 2)
    e = torch.where(bad | tiny, torch.zeros_like(e), e)
    a = g.abs() * _power(-e[..., None])
    code = sum(((a >= c) if even else (a > c)).to(torch.uint8)
               for c, even in ((0.25, 0), (0.75, 1), (1.25, 0), (1.75, 1), (2.5, 0), (3.5, 1), (5.0, 0)))
    code = torch.where(tiny[..., None], torch.zeros_like(code), code) | (torch.signbit(g).to(torch.uint8) << 3)
    code = torch.where(bad[..., None], torch.full_like(code, 7), code)
    byte = torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)
    return code.flatten(-2), byte


def _decode(code, byte):
    mag = torch.tensor(_VALUES, device=code.device)[(code & 7).long()]
    x = torch.where(code >= 8, -mag, mag).unflatten(-1, (-1, 32))
    x = x * _power(byte.to(torch.int32).clamp(max=254)[..., None] - 127)
    return torch.where((byte == 255)[..., None], torch.full_like(x, math.nan), x).flatten(-2)


# Blocks of 32 rows: K codes (16 D bytes), V codes (16 D), K exponents (D), V exponents (D).  Row r = 8 a + 4 j + b.
def _into_blocks(kc, vc, ke, ve):
    """kc, vc [..., 32, D] codes, ke, ve [..., 32, D / 32] bytes -> [..., 34 D] bytes."""
    D = kc.shape[-1]
    two = lambda c: c[..., 0::2] | (c[..., 1::2] << 4)                   # the even channel in the low half
    rows = lambda x: x.unflatten(-2, (4, 2, 4))                          # [..., a, j, b, bytes]
    k, v = rows(two(kc)), rows(two(vc))
    if D == 128:
        k = k.unflatten(-1, (4, 16)).movedim((-4, -2), (-5, -4))         # j, quarter, a, b, 16 bytes
        v = v.unflatten(-1, (16, 4)).movedim((-4, -2), (-5, -3))         # j, a, piece, b, 4 bytes
    else:
        k = k.unflatten(-1, (4, 8)).movedim((-2, -4), (-5, -2))          # quarter, a, b, j, 8 bytes
        v = v.unflatten(-1, (16, 2)).movedim(-2, -4)                     # a, piece, j, b, 2 bytes
    ke = rows(ke).movedim(-3, -1)                                        # a, b, group, j
    ve = rows(ve).movedim(-1, -3)                                        # a, group, j, b
    return torch.cat([k.flatten(-5), v.flatten(-5), ke.flatten(-4), ve.flatten(-4)], -1)


def _out_of_blocks(blocks):
    D = blocks.shape[-1] // 34
    k, v, ke, ve = blocks.split([16 * D, 16 * D, D, D], -1)
    if D == 128:
        k = k.unflatten(-1, (2, 4, 4, 4, 16)).movedim((-5, -4), (-4, -2))
        v = v.unflatten(-1, (2, 4, 16, 4, 4)).movedim((-5, -3), (-4, -2))
    else:
        k = k.unflatten(-1, (4, 4, 4, 2, 8)).movedim((-5, -2), (-2, -4))
        v = v.unflatten(-1, (4, 16, 2, 4, 2)).movedim(-4, -2)
    ke = ke.unflatten(-1, (4, 4, D // 32, 2)).movedim(-1, -3)
    ve = ve.unflatten(-1, (4, D // 32, 2, 4)).movedim(-3, -1)
    flat = lambda x: x.flatten(-2) if x.dim() > blocks.dim() + 3 else x
    row = lambda x: flat(x).flatten(-4, -2)
    apart = lambda c: torch.stack([c & 15, c >> 4], -1).flatten(-2)
    return apart(row(k)), apart(row(v)), row(ke), row(ve)


def _encode_all(k, v):
    """k, v [B, Hkv, budget, D] -> [B, Hkv, blocks, 34 D] bytes; rows that fill the last block up are zeros."""
    pad = -k.shape[2] % 32
    parts = []
    for x in (k, v):
        code, byte = _encode(x)
        grow = lambda y: torch.nn.functional.pad(y, (0, 0, 0, pad)).unflatten(2, (-1, 32))
        parts.append((grow(code), grow(byte)))
    return _into_blocks(parts[0][0], parts[1][0], parts[0][1], parts[1][1]).contiguous()


def _decode_all(packed, budget):
    kc, vc, ke, ve = (x.flatten(2, 3)[:, :, :budget] for x in _out_of_blocks(packed))
    return _decode(kc, ke), _decode(vc, ve)


# ---- one pass --------------------------------------------------------------------------------------------------------------
def run(state):
    op = state["case"]["op"]
    if op == "weights":
        return _weights_own(state) if own else _weights_plain(state)
    if op == "pack":
        return _pack_own(state) if own else _pack_plain(state)
    return _step_own(state) if own else _step_plain(state)


def _step_outputs(s):
    # packed rows come back as their bytes: encoding a row is exact, so equal values are equal bytes, and decoding all of them in
    # every step would be another operator's time
    rows = dict(packed=s["packed"]) if "packed" in s else dict(k_ret=s["k_ret"], v_ret=s["v_ret"])
    return dict(out=s["out"], k_win=s["k_win"], v_win=s["v_win"], win_score=s["win_score"], ret_score=s["ret_score"],
                ret_pos=s["ret_pos"], ret_count=s["ret_count"], n_seen=s["n_seen"], **rows)


def _score_again(s):
    """By given keys: the scores of what entered the ring count as known again, once a window."""
    if s["case"].get("keys") == "given":
        s["until_scored"] -= 1
        if s["until_scored"] == 0:
            s["until_scored"] = s["case"]["window"]
            s["n_scored"].copy_(s["n_seen"])


# plain forms: elementary tensor operations in 32 bits
def _per_query_block(q, k, window, first, dtype, use):
    """Calls use(scores [Hkv, G, rows, keys], first row, first key) for blocks of queries from `first` on; what a query does not
    see is -inf."""
    n, Hq, D = q.shape
    Hkv = k.shape[1]
    G = Hq // Hkv
    rows = max(64, (1 << 28) // (Hq * max(n, 1)))
    kt = k.permute(1, 2, 0).to(dtype).contiguous()
    for i0 in range(first, n, rows):
        i1 = min(n, i0 + rows)
        j0 = max(0, i0 - window + 1)
        x = q[i0:i1].unflatten(1, (Hkv, G)).permute(1, 2, 0, 3).to(dtype).reshape(Hkv, G * (i1 - i0), D)
        s = (x @ kt[:, :, j0:i1].contiguous()).mul_(D ** -0.5).unflatten(1, (G, i1 - i0))
        i = torch.arange(i0, i1, device=q.device)[:, None]
        j = torch.arange(j0, i1, device=q.device)[None]
        use(s.masked_fill_((j > i) | (j <= i - window), -math.inf), i0, j0)


def _weights_plain(s):
    mass = torch.zeros(s["mass"].shape, dtype=torch.float64, device="cuda")
    lo = 0
    for n in s["ns"]:
        lse = s["lse"][:, lo:lo + n].unflatten(0, (mass.shape[0], -1))

        def add(scores, i0, j0, lo=lo, lse=lse):
            p = scores.sub_(lse[:, :, i0:i0 + scores.shape[2], None]).exp_()
            mass[:, lo + j0:lo + j0 + scores.shape[3]] += p.sum((1, 2))
        _per_query_block(s["q"][lo:lo + n], s["k"][lo:lo + n], s["window"], max(0, n - s["last"]) if s["last"] > 0 else 0,
                         torch.float32, add)
        lo += n
    s["mass"].copy_(mass)
    return s["mass"]


def _pack_plain(s):
    live = (torch.arange(s["case"]["budget"], device="cuda") < s["ret_count"][..., None])[..., None]
    s["packed"].copy_(_encode_all(torch.where(live, s["k_ret"], 0), torch.where(live, s["v_ret"], 0)))
    k, v = _decode_all(s["packed"], s["case"]["budget"])
    s["k_out"].copy_(torch.where(live, k, s["k_out"]))
    s["v_out"].copy_(torch.where(live, v, s["v_out"]))
    return s["k_out"], s["v_out"]


def _step_plain(s):
    case = s["case"]
    B, Hkv, D, w, b = case["B"], case["Hkv"], case["D"], case["window"], case["budget"]
    mass = case["op"] == "step" or case["keys"] == "mass"
    at = torch.arange(B, device="cuda")[:, None], torch.arange(Hkv, device="cuda")[None]
    t = s["n_seen"].long()[:, None]
    slot, leaving = (t % w).expand(B, Hkv), t - w
    late = (leaving >= 0) & (s["n_scored"].long()[:, None] <= leaving) & (not mass)
    # where the leaving token goes: behind the kept ones, in the place of the lowest key (the latest of equal ones), or nowhere
    e_score = s["win_score"][(*at, slot)]
    sink = leaving < case["sink"]
    e_key = torch.where(sink, torch.full_like(e_score, math.inf), e_score)
    count = s["ret_count"].long()
    live = torch.arange(b, device="cuda") < count[..., None]
    keys = torch.where(live, s["ret_score"], torch.full_like(s["ret_score"], math.inf))
    low = keys.amin(-1)
    victim = torch.where(live & (keys == low[..., None]), s["ret_pos"], -1).argmax(-1)
    room = count < b
    moves = (leaving >= 0) & (sink | (e_score > 0.0)) & (room | (e_key > low))
    dst = torch.where(room, count, victim)
    put = lambda x, new: x.__setitem__((*at, dst), torch.where(moves if new.dim() == 2 else moves[..., None], new, x[(*at, dst)]))
    e_rows = s["k_win"][(*at, slot)].clone(), s["v_win"][(*at, slot)].clone()
    put(s["ret_score"], e_key)
    put(s["ret_pos"], leaving.to(torch.int32).expand(B, Hkv))
    if "packed" in s:
        (kc, ke), (vc, ve) = _encode(e_rows[0]), _encode(e_rows[1])
        block = s["packed"][(*at, dst // 32)]
        old = _out_of_blocks(block)
        here = ((torch.arange(32, device="cuda") == (dst % 32)[..., None]) & moves[..., None])[..., None]
        s["packed"][(*at, dst // 32)] = _into_blocks(*(torch.where(here, n[:, :, None], o) for o, n in zip(old, (kc, vc, ke, ve))))
        k_ret, v_ret = _decode_all(s["packed"], b)
    else:
        put(s["k_ret"], e_rows[0])
        put(s["v_ret"], e_rows[1])
        k_ret, v_ret = s["k_ret"].float(), s["v_ret"].float()
    s["ret_count"] += (moves & room).to(torch.int32)
    s["k_win"][(*at, slot)], s["v_win"][(*at, slot)] = s["k"], s["v"]
    s["n_seen"] += 1
    # the query over what is there now
    seen = torch.cat([(torch.arange(w, device="cuda")[None, None] < (t + 1)[..., None]).expand(B, Hkv, w),
                      torch.arange(b, device="cuda") < s["ret_count"][..., None]], -1)[:, :, None]
    keys_all = torch.cat([s["k_win"].float(), k_ret], 2).transpose(2, 3).contiguous()
    scores = (s["q"].float().unflatten(1, (Hkv, -1)) @ keys_all).mul_(D ** -0.5).masked_fill_(~seen, -math.inf)
    p = (scores - scores.amax(-1, keepdim=True)).exp()
    p = p / p.sum(-1, keepdim=True)
    values = torch.cat([s["v_win"].float(), v_ret], 2).masked_fill_(~seen.transpose(2, 3), 0.0)
    out = (p @ values).flatten(1, 2)
    s["out"].copy_(torch.where(late[..., None], torch.full_like(out, math.nan), out))
    if mass:
        got = p.sum(2)
        s["win_score"][(*at, slot)] = 0.0
        s["win_score"] += got[..., :w]
        s["ret_score"] += got[..., w:]
    else:
        _score_again(s)
    return _step_outputs(s)


# the framework's calls
def _binding():
    from paper_2510_20787_amd import binding
    return binding


def _handle(s):
    """What a program makes once and keeps: the config struct, the cache struct, a workspace."""
    if "handle" not in s:
        B, c = _binding(), s["case"]
        weights = c["op"] == "weights"
        cfg = B.make_cfg(c["Hq"], c["Hkv"], c["D"], s["window"] if weights else c["window"], 0 if weights else c["budget"],
                         0 if weights else c["sink"], 0.0, 0.0, c["dtype"])
        if weights:
            nbytes = B.ltea_mass_workspace_bytes(cfg, len(s["ns"]), s["q"].shape[0], max(s["ns"]))
            s["handle"] = dict(cfg=cfg, workspace=torch.empty(max(nbytes, 16), dtype=torch.uint8, device="cuda"))
        else:
            empty = torch.empty(0, dtype=_storage(c), device="cuda")
            cache = B.wrap_cache(s.get("k_win", empty), s.get("v_win", empty), s["win_score"], s.get("k_ret", empty),
                                 s.get("v_ret", empty), s["ret_score"], s["ret_pos"], s["ret_count"], s["n_seen"], s["n_scored"])
            s["handle"] = dict(cfg=cfg, cache=cache)
            if c["op"] == "pack":
                s["handle"]["back"] = B.wrap_cache(empty, empty, s["win_score"], s["k_out"], s["v_out"], s["ret_score"],
                                                   s["ret_pos"], s["ret_count"], s["n_seen"], s["n_scored"])
            else:
                nbytes = B.ltea_decode_kept_workspace_bytes(cfg, c["B"])
                s["handle"]["workspace"] = torch.empty(max(nbytes, 16), dtype=torch.uint8, device="cuda")
    return s["handle"]


def _weights_own(s):
    h = _handle(s)
    return _binding().ltea_attention_mass(h["cfg"], s["q"], s["k"], s["cu"], max(s["ns"]), s["lse"], last=s["last"], mass=s["mass"],
                                          workspace=h["workspace"])


def _pack_own(s):
    h, B = _handle(s), _binding()
    B.ltea_kept_pack(h["cfg"], h["cache"], packed=s["packed"])
    B.ltea_kept_unpack(h["cfg"], s["packed"], h["back"])
    return s["k_out"], s["v_out"]


def _step_own(s):
    h, B, c = _handle(s), _binding(), s["case"]
    if c["op"] == "step" or c["keys"] == "mass":
        B.ltea_decode_step_mass(h["cfg"], s["q"], s["k"], s["v"], h["cache"], packed=s.get("packed"), out=s["out"],
                                workspace=h["workspace"])
    else:
        B.ltea_decode_step_packed(h["cfg"], s["q"], s["k"], s["v"], h["cache"], s["packed"], out=s["out"],
                                  workspace=h["workspace"])
        _score_again(s)
    return _step_outputs(s)


# ---- from the definitions, in 64 bits ----------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"weights": _exact_weights, "pack": _exact_pack}.get(case["op"], _exact_step)(s)


def _exact_weights(s):
    c = s["case"]
    G = c["Hq"] // c["Hkv"]
    mass = torch.zeros(s["mass"].shape, dtype=torch.float64, device="cuda")
    lo = 0
    for n in s["ns"]:
        first = max(0, n - s["last"]) if s["last"] > 0 else 0
        for hq in range(c["Hq"]):
            k = s["k"][lo:lo + n, hq // G].double()
            for i0 in range(first, n, 4096):
                i = torch.arange(i0, min(n, i0 + 4096), device="cuda")
                z = s["q"][lo + i, hq].double() @ k.T / math.sqrt(c["D"]) - s["lse"][hq, lo + i].double()[:, None]
                ago = i[:, None] - torch.arange(n, device="cuda")[None]
                mass[hq // G, lo:lo + n] += torch.where((ago >= 0) & (ago < s["window"]), z.exp(), 0.0).sum(0)
        lo += n
    return mass


def _nearest(x):
    """Each group of 32 of x [..., D] at the nearest of its 15 values, in 64 bits, by the definition."""
    g = x.double().unflatten(-1, (-1, 32))
    top = g.abs().amax(-1, keepdim=True)
    k = torch.floor(torch.log2(top.clamp(min=2.0 ** -140)))
    k = k + (torch.exp2(k + 1) <= top).double() - (torch.exp2(k) > top).double()
    unit = torch.exp2(torch.where((top <= 1.75 * torch.exp2(k)) | (k == 127), k - 2, k - 1))
    grid = torch.tensor(_VALUES, dtype=torch.float64, device=x.device)
    far = (g.abs() / unit)[..., None] - grid
    even_first = far.abs() + torch.tensor([0, 1, 0, 1, 0, 1, 0, 1], dtype=torch.float64, device=x.device) * 1e-9
    return (torch.sign(g) * grid[even_first.argmin(-1)] * unit * (top >= 2.0 ** -120)).flatten(-2)


def _exact_pack(s):
    c = s["case"]
    if c["B"] * c["Hkv"] * c["budget"] * c["D"] > 1 << 28:
        return None
    out = []
    for x in (s["k_ret"], s["v_ret"]):
        y = torch.zeros(x.shape, dtype=torch.float64, device="cuda")
        for b in range(c["B"]):
            n = int(s["ret_count"][b, 0])
            for h in range(c["Hkv"]):
                y[b, h, :n] = _nearest(x[b, h, :n]) if n else 0.0
        out.append(y)
    return tuple(out)


def _exact_step(s):
    c = s["case"]
    w, G, D, tau = c["window"], c["Hq"] // c["Hkv"], c["D"], 0.0
    mass = c["op"] == "step" or c["keys"] == "mass"
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    win, ret = s["win_score"].double(), s["ret_score"].double()
    seen, counts = s["n_seen"].tolist(), s["ret_count"].tolist()
    for b in range(c["B"]):
        t = seen[b]
        slot, e = t % w, t - w
        for h in range(c["Hkv"]):
            n, dst = counts[b][h], -1
            if e >= 0:
                z = float(s["win_score"][b, h, slot])
                key = math.inf if e < c["sink"] else z
                if e < c["sink"] or z > tau:
                    if n < c["budget"]:
                        dst = n
                        n += 1
                    else:
                        low = s["ret_score"][b, h].min()
                        if key > float(low):
                            same = s["ret_score"][b, h] == low
                            dst = int(torch.where(same, s["ret_pos"][b, h], -1).argmax())
                    if dst >= 0:
                        ret[b, h, dst] = key
            m = min(t + 1, w)
            kw, vw = s["k_win"][b, h].double(), s["v_win"][b, h].double()
            ek, ev = kw[slot].clone(), vw[slot].clone()
            kw[slot], vw[slot] = s["k"][b, h].double(), s["v"][b, h].double()
            if "packed" in s:
                kr, vr = (x[0, 0].double() for x in _decode_all(s["packed"][b:b + 1, h:h + 1], c["budget"]))
                ek, ev = _nearest(ek[None])[0], _nearest(ev[None])[0]
            else:
                kr, vr = s["k_ret"][b, h].double(), s["v_ret"][b, h].double()
            if dst >= 0:
                kr[dst], vr[dst] = ek, ev
            K, V = torch.cat([kw[:m], kr[:n]]), torch.cat([vw[:m], vr[:n]])
            z = s["q"][b, h * G:(h + 1) * G].double() @ K.T / math.sqrt(D)
            p = torch.softmax(z, 1)
            out[b, h * G:(h + 1) * G] = p @ V
            if mass:
                win[b, h, slot] = 0.0
                win[b, h, :m] += p[:, :m].sum(0)
                ret[b, h, :n] += p[:, m:].sum(0)
    none = dict.fromkeys(("k_win", "v_win", "ret_pos", "ret_count", "n_seen", *(("packed",) if "packed" in s else ("k_ret", "v_ret"))))
    return dict(out=out, win_score=win if mass else None, ret_score=ret if mass else None, **none)
