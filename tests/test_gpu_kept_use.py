"""The calls of eviction by accumulated weight and of kept rows in 4 bits as a program makes them: one after another on one cache, recorded
in graphs, on another stream, at the ends of their ranges."""
import numpy as np
import pytest
import torch

from paper_2510_20787_amd import binding as B
from tests.gpu_util import DeviceWorkload
from tests.kept_util import FIELDS, clone, make_state, run_and_check, step_inputs
from tests.test_gpu_parity import make

pytestmark = pytest.mark.gpu


def prompt(cfg, lens, seed):
    td = torch.float32 if cfg.dtype == B.LTEA_F32 else torch.bfloat16
    rng = np.random.default_rng(seed)
    T = sum(lens)
    q, k, v = [torch.from_numpy(rng.standard_normal((T, h, cfg.D))).to(dtype=td, device="cuda") for h in (cfg.Hq, cfg.Hkv, cfg.Hkv)]
    return q, k, v, torch.from_numpy(np.concatenate([[0], np.cumsum(lens)])).to(dtype=torch.int32, device="cuda")


def valid(cache, f):
    """What of a member the contract defines: no slot past what is there."""
    x = getattr(cache, f)
    if f.startswith(("k_ret", "v_ret", "ret_score", "ret_pos")):
        return x[torch.arange(x.shape[2], device="cuda")[None, None] < cache.ret_count[:, :, None]]
    if f in ("k_win", "v_win", "win_score"):
        live = torch.arange(x.shape[2], device="cuda")[None] < cache.n_seen[:, None]
        return x[live[:, None].expand(x.shape[:3])]
    return x


def same(a, b, fields=FIELDS):
    return all(torch.equal(valid(a, f), valid(b, f)) for f in fields)


@pytest.mark.parametrize("dtype,Hq,Hkv,D", [("bf16", 8, 2, 64), ("bf16", 4, 4, 128), ("f32", 2, 2, 64)])
def test_prompt_steps_pack_steps_unpack_steps(dtype, Hq, Hkv, D):
    """A prompt by accumulated weight, steps on stored rows, the rows packed, steps on packed rows, unpacked, steps again."""
    cfg = B.make_cfg(Hq, Hkv, D, 24, 40, 2, 0.0, 0.0, dtype)
    lens = [150, 3, 24, 66]
    q, k, v, cu = prompt(cfg, lens, 1)
    cache = B.alloc_cache(cfg, len(lens))
    B.ltea_prefill_mass(cfg, q, k, v, cu, max(lens), cache)
    assert cache.n_seen.tolist() == lens and cache.n_scored.tolist() == lens
    assert cache.ret_count.max() <= 40 and int(cache.ret_count[0, 0]) == 40 and int(cache.ret_count[1, 0]) == 0
    for step in range(4):
        run_and_check(cfg, cache, None, True, 10 + step, dtype)
    packed = B.ltea_kept_pack(cfg, cache)
    for step in range(4):
        run_and_check(cfg, cache, packed, True, 20 + step, dtype)
    B.ltea_kept_unpack(cfg, packed, cache)
    assert torch.equal(B.ltea_kept_pack(cfg, cache), packed)
    for step in range(3):
        run_and_check(cfg, cache, None, True, 30 + step, dtype)


def test_scored_prompt_packed_steps_and_rescoring():
    """A prompt scored by the network, its kept rows packed, steps over them with the ring scored again in time; the eviction is that of the
    steps over stored rows, which have the same scores."""
    d = DeviceWorkload(make("bf16_d64"))
    cache = d.new_cache()
    B.ltea_prefill(d.cfg, d.cnn, d.q, d.k, d.v, d.cu, d.max_seqlen, cache)
    twin = clone(cache)
    packed = B.ltea_kept_pack(d.cfg, cache)
    cache.k_ret.fill_(float("nan")), cache.v_ret.fill_(float("nan"))           # not read any more
    period, n = B.ltea_lazy_period(d.cfg, d.cnn), cache.n_seen.numel()
    assert period >= 1
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for step in range(min(2 * period, 10)):
        if step % period == 0:
            B.ltea_rescore(d.cfg, d.cnn, cache), B.ltea_rescore(d.cfg, d.cnn, twin)
        q, k, v = step_inputs(d.cfg, n, 50 + step)
        out = B.ltea_decode_step_packed(d.cfg, q, k, v, cache, packed, status=status)
        B.ltea_decode_step_lazy(d.cfg, q, k, v, twin)
        assert bool(torch.isfinite(out).all())
        assert same(cache, twin, ("k_win", "v_win", "ret_score", "ret_pos", "ret_count", "n_seen", "n_scored")), step
    assert int(status) == 0
    again = torch.zeros_like(packed)                                            # the packed rows are the twin's, in 4 bits
    B.ltea_kept_pack(d.cfg, twin, again)
    assert torch.equal(again, packed)


SHAPES = [dict(B=2, Hq=8, Hkv=2, D=64, window=40, budget=30), dict(B=1, Hq=4, Hkv=1, D=128, window=100, budget=3000),
          dict(B=20, Hq=16, Hkv=16, D=128, window=33, budget=31)]


@pytest.mark.parametrize("use_packed", [False, True], ids=["rows", "packed"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_steps_replayed_from_a_graph(shape, use_packed):
    """Recorded steps give the bits of the same steps taken one by one, replay after replay, also where two graphs share a workspace."""
    nb = shape["B"]
    cfg = B.make_cfg(shape["Hq"], shape["Hkv"], shape["D"], shape["window"], shape["budget"], 1, 0.0, 0.0, "bf16")
    cache = make_state(cfg, [cfg.window + cfg.budget + 5 * i for i in range(nb)], [cfg.budget - (i == 0) for i in range(nb)], 5)
    for f in FIELDS:                                           # (nothing that is not a number, so that states compare by value)
        x = getattr(cache, f)
        if x.is_floating_point():
            x.nan_to_num_(nan=0.0, posinf=float("inf"))
    twin = clone(cache)
    packed = B.ltea_kept_pack(cfg, cache) if use_packed else None
    packed_twin = None if packed is None else packed.clone()
    ws = torch.full((max(B.ltea_decode_kept_workspace_bytes(cfg, nb), 16),), 0xFF, dtype=torch.uint8, device="cuda")
    steps = 2
    data = [step_inputs(cfg, nb, 70 + i) for i in range(steps)]
    outs = [torch.zeros(nb, cfg.Hq, cfg.D, dtype=torch.bfloat16, device="cuda") for _ in range(steps)]
    # warm up on copies: what is recorded does not run
    B.ltea_decode_step_mass(cfg, *data[0], clone(cache), packed=None if packed is None else packed.clone(), workspace=ws)
    graphs = []
    for i in range(steps):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.ltea_decode_step_mass(cfg, *data[i], cache, packed=packed, out=outs[i], workspace=ws)
        graphs.append(g)
    for replay in range(4):
        for i, (q, k, v) in enumerate(step_inputs(cfg, nb, 80 + 10 * replay + j) for j in range(steps)):
            for dst, src in zip(data[i], (q, k, v)):
                dst.copy_(src)
            graphs[i].replay()
            want = B.ltea_decode_step_mass(cfg, q, k, v, twin, packed=packed_twin)
            torch.cuda.synchronize()
            assert torch.equal(outs[i], want), (replay, i)
        assert same(cache, twin, FIELDS if packed is None else [f for f in FIELDS if f not in ("k_ret", "v_ret")]), replay
        assert packed is None or torch.equal(packed, packed_twin), replay


def test_prompt_and_conversions_replayed_from_a_graph():
    cfg = B.make_cfg(8, 2, 64, 32, 50, 1, 0.0, 0.0, "bf16")
    lens = [400, 33, 2100]
    q, k, v, cu = prompt(cfg, lens, 6)
    cache, twin = B.alloc_cache(cfg, 3), B.alloc_cache(cfg, 3)
    packed = B.alloc_packed(cfg, 3)
    ws = torch.full((B.ltea_prefill_mass_workspace_bytes(cfg, 3, sum(lens), max(lens)),), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(q)
    B.ltea_prefill_mass(cfg, q, k, v, cu, max(lens), twin, last=100, workspace=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.ltea_prefill_mass(cfg, q, k, v, cu, max(lens), cache, last=100, out=out, workspace=ws)
        B.ltea_kept_pack(cfg, cache, packed)
        B.ltea_kept_unpack(cfg, packed, cache)
    for replay in range(3):
        for x, y in zip((q, k, v), prompt(cfg, lens, 7 + replay)):
            x.copy_(y)
        g.replay()
        want = B.ltea_prefill_mass(cfg, q, k, v, cu, max(lens), twin, last=100)
        B.ltea_kept_unpack(cfg, B.ltea_kept_pack(cfg, twin), twin)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and same(cache, twin), replay


def test_another_stream():
    """Work goes to the caller's stream, in order with what is there."""
    cfg = B.make_cfg(8, 2, 64, 40, 60, 0, 0.0, 0.0, "bf16")
    first = make_state(cfg, [200, 150], [60, 60], 9)
    twin, side = clone(first), torch.cuda.Stream()
    q, k, v = step_inputs(cfg, 2, 90)
    want = B.ltea_decode_step_mass(cfg, q, k, v, twin)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        big = torch.randn(4096, 4096, device="cuda")
        for _ in range(4):
            big = big @ big * 1e-3
        late_q = q * 1                                        # (there only when the products are done)
        out = B.ltea_decode_step_mass(cfg, late_q, k, v, first)
    side.synchronize()
    assert torch.equal(out, want) and same(first, twin)


def test_tokens_behind_the_last_sequence_keep_their_weight():
    cfg = B.make_cfg(2, 1, 64, 5000, 0, dtype="bf16")
    q, k, v, cu = prompt(cfg, [3000, 60], 11)
    rng = np.random.default_rng(12)
    lse = torch.from_numpy(rng.uniform(8, 9, (2, 3060)).astype(np.float32)).cuda()
    mass = torch.full((1, 3060), 7.0, device="cuda")
    B.ltea_attention_mass(cfg, q, k, cu[:2].contiguous(), 3060, lse, mass=mass)
    full = B.ltea_attention_mass(cfg, q, k, cu, 3060, lse)
    assert torch.equal(mass[:, :3000], full[:, :3000]) and bool((mass[:, 3000:] == 7.0).all())


EDGES = [  # sequences, Hq, Hkv, D, window, budget, counts, heads checked: every n-th
    (1, 128, 1, 64, 40, 64, 64, 1),              # the largest group
    (1, 128, 1, 128, 700, 2000, 2000, 1),        # and cut into shares
    (2, 16, 1, 128, 100, 150, 149, 1),           # scores that just stay in LDS: 16 heads x (128 + 160) x 4 bytes + 33 KB of outputs
    (2, 16, 1, 128, 100, 190, 190, 1),           # and just not: 32 slots more
    (3, 9, 1, 64, 50, 90, 90, 1),                # more heads than a pass takes
    (1, 256, 256, 64, 20, 33, 33, 40),           # more KV heads than a counter holds
    (300, 1, 1, 64, 33, 64, 64, 37),             # more heads than CUs
    (1, 2, 1, 64, 1, 1, 1, 1),                   # one slot of each
    (1, 4, 2, 128, 2, 70000, 69999, 1),          # a budget past 16 bits
]


@pytest.mark.parametrize("packed", [False, True], ids=["rows", "packed"])
@pytest.mark.parametrize("case", EDGES, ids=lambda c: "-".join(map(str, c)))
def test_ends_of_the_ranges(case, packed):
    nb, Hq, Hkv, D, window, budget, count, every = case
    cfg = B.make_cfg(Hq, Hkv, D, window, budget, 0, 0.0, 0.0, "bf16")
    cache = make_state(cfg, [window + budget + 3 + i for i in range(nb)], [count] * nb, 20)
    pk = B.ltea_kept_pack(cfg, cache) if packed else None
    for step in range(2 if budget < 10000 else 1):
        run_and_check(cfg, cache, pk, True, 100 + step, "bf16", heads=every)


def test_wrong_tensors_are_refused():
    cfg = B.make_cfg(4, 2, 64, 16, 8, 0, 0.0, 0.0, "bf16")
    cache = make_state(cfg, [40, 41], [8, 8], 21)
    before = clone(cache)
    q, k, v = step_inputs(cfg, 2, 110)
    packed = B.ltea_kept_pack(cfg, cache)
    small = B.wrap_cache(*[getattr(cache, f)[:1].contiguous() if f == "ret_pos" else getattr(cache, f) for f in FIELDS])
    wide = B.wrap_cache(*[getattr(cache, f).double() if f == "win_score" else getattr(cache, f) for f in FIELDS])
    bad = [lambda: B.ltea_decode_step_mass(cfg, q.float(), k, v, cache), lambda: B.ltea_decode_step_mass(cfg, q, k[:1], v, cache),
           lambda: B.ltea_decode_step_mass(cfg, q.transpose(0, 1), k, v, cache), lambda: B.ltea_decode_step_mass(cfg, q, k, v, small),
           lambda: B.ltea_decode_step_mass(cfg, q, k, v, wide), lambda: B.ltea_decode_step_mass(cfg, q, k, v, cache, out=q.float()),
           lambda: B.ltea_decode_step_mass(cfg, q, k, v, cache, packed=packed[:1]),
           lambda: B.ltea_decode_step_mass(cfg, q, k, v, cache, workspace=torch.empty(1 << 20, device="cuda")),
           lambda: B.ltea_decode_step_packed(cfg, q, k, v, cache, packed, status=torch.zeros(1, device="cuda")),
           lambda: B.ltea_decode_step_packed(cfg, q, k, v, cache, packed.cpu()), lambda: B.ltea_decode_step_packed(cfg, q, k, v, cache, None),
           lambda: B.ltea_kept_unpack(cfg, packed[:1], cache), lambda: B.ltea_kept_pack(cfg, cache, packed.int())]
    for i, call in enumerate(bad):
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(B.LteaError):
        B.ltea_decode_step_mass(cfg, q, k, v, cache, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    for f in FIELDS:
        assert torch.equal(torch.nan_to_num(getattr(cache, f).float()), torch.nan_to_num(getattr(before, f).float())), f
