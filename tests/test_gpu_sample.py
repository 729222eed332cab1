"""jk_sample against the plain 64-bit rule: the token and the kept set exactly, the filtered logits to one rounding."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as pg
from paper_2502_06282_b200 import binding as jk
from paper_2502_06282_b200 import synth
from tests.jk_testutil import Guard, dev, host

pytestmark = pytest.mark.gpu


def make_ctx(vocab):
    return jk.Context(hidden=8, n_experts=1, top_k=1, inter=8, vocab=vocab, n_q_heads=1, n_kv_heads=1, head_dim=64,
                      max_batch=1, max_tree=1, max_depth=1, max_frontier=1, k_per_expert=1, dtype="f32")


def run(ctx, z, dtype, T=None, k=None, p=None, m=None, u=None, filtered=True, stride=None, offset=0):
    """Device call and plain rule, compared.  z [R, V] float64 holding values of the type."""
    R, V = z.shape
    g = Guard()
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    room = g.alloc((offset + R * (stride or V),), td)
    rows = room[offset:].view(R, stride or V)
    rows[:, :V] = dev(z.astype(np.float32)).to(td)
    tok = g.alloc((R,), torch.int32) if u is not None else None
    out = g.alloc((R, V), torch.float32) if filtered else None
    f = lambda x, t=np.float32: None if x is None else dev(np.broadcast_to(np.asarray(x, t), (R,)).copy())
    ctx.sample(rows[:, :V], f(T), f(k, np.int32), f(p), f(m), f(u), tok, out)
    torch.cuda.synchronize()
    g.check()
    at = lambda x, r, d, t=np.float32: d if x is None else (np.broadcast_to(np.asarray(x, t), (R,))[r].item())
    for r in range(R):
        want, kept = pg.sample_row(z[r], at(T, r, 1.0), at(k, r, 0, np.int32), at(p, r, 1.0), at(m, r, 0.0), at(u, r, 0.0))
        if tok is not None:
            assert int(tok[r]) == want, r
        if out is not None:
            got = host(out[r]).astype(np.float64)
            assert np.array_equal(got > -np.inf, kept), (r, int((got > -np.inf).sum()), int(kept.sum()))
            t = at(T, r, 1.0)
            big = float(np.finfo(np.float32).max)
            exact = np.clip(np.nan_to_num(z[r][kept], nan=0.0, posinf=big, neginf=-big) / t, -big, big) if t > 0 else np.zeros(kept.sum())
            # one division: half a step, 2^-24 (subnormal results: half of 2^-149)
            assert np.all(np.abs(got[kept] - exact) <= 2.0 ** -24 * np.abs(exact) + 2.0 ** -149), r
    return tok, out


def rows_of(rng, R, V, dtype, spread=3.0):
    z = rng.standard_normal((R, V)) * spread
    if V > 20:
        z[np.arange(R)[:, None], rng.integers(0, V, (R, 8))] += 3 * spread
    return synth.store_round(z, dtype).astype(np.float64)


FILTERS = [dict(), dict(k=1), dict(k=50), dict(p=0.9), dict(m=0.05), dict(k=40, p=0.8), dict(k=1000, p=0.95, m=0.01),
           dict(p=0.999999), dict(p=0.0), dict(m=1.0), dict(k=10 ** 9, p=0.5), dict(p=1.5, m=-1.0, k=-3)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 31, 1000, 4097, 32000, 128256])
def test_filters(V, dtype):
    rng = np.random.default_rng(V)
    ctx = make_ctx(V)
    for i, f in enumerate(FILTERS):
        R = 3 if V > 5000 else 7
        z = rows_of(rng, R, V, dtype, spread=(0.3, 2.0, 6.0)[i % 3])
        run(ctx, z, dtype, T=rng.uniform(0.3, 1.5, R), u=rng.random(R), **f)
    assert ctx.read_status() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_rows_with_their_own_parameters(dtype):
    rng = np.random.default_rng(3)
    R, V = 300, 3001
    ctx = make_ctx(V)
    run(ctx, rows_of(rng, R, V, dtype), dtype, T=rng.uniform(0.0, 2.0, R) * (rng.random(R) > 0.1),
        k=rng.integers(-1, 60, R), p=rng.uniform(0.1, 1.1, R), m=rng.uniform(-0.1, 0.2, R), u=rng.random(R))


@pytest.mark.parametrize("R", [60, 130, 250])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_one_two_and_four_blocks(R, dtype):
    """Enough rows that a row gets fewer blocks than the machine could give it."""
    rng = np.random.default_rng(R)
    V = 8300
    ctx = make_ctx(V)
    z = rows_of(rng, R, V, dtype)
    z[::5] = np.round(z[::5])                           # ties
    run(ctx, z, dtype, T=rng.uniform(0.4, 1.5, R), k=rng.integers(-1, 900, R), p=rng.uniform(0.3, 1.1, R),
        m=rng.uniform(-0.1, 0.05, R), u=rng.random(R))
    run(ctx, z, dtype, T=rng.uniform(0.4, 1.5, R), p=rng.uniform(0.6, 1.0, R), u=rng.random(R))


@pytest.mark.parametrize("V", [257, 32000])
def test_equal_logits(V):
    """Ties go to the lower index, whatever the filter cuts through them."""
    rng = np.random.default_rng(5)
    ctx = make_ctx(V)
    flat = np.zeros((6, V))
    # (a row of V equal tokens: top_p cuts where i < top_p V, away from whole numbers)
    run(ctx, flat, "f32", k=[0, 1, 7, 100, V - 1, V], p=[0.5003, 1.0, 0.4, 0.333, 1.0, 0.9001], u=rng.random(6))
    steps = rng.integers(0, 4, (6, V)).astype(np.float64)
    run(ctx, steps, "bf16", T=0.7, k=[0, 5, 60, V // 2, V - 2, 3], p=[0.31, 0.9, 0.77, 0.613, 0.2, 1.0], u=rng.random(6))
    run(ctx, -steps, "f32", m=[0.1, 0.2, 0.4, 0.9, 1.0, 0.0], u=rng.random(6))


@pytest.mark.parametrize("V", [6001, 40000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_crowded_values(V, dtype):
    """Rows whose values crowd where a threshold is looked for: a narrow band, next to zero, far below the weights that
    count, all negative, a scale of logits that one temperature leaves flat and another one sharp."""
    rng = np.random.default_rng(V)
    ctx = make_ctx(V)
    n = rng.standard_normal((10, V))
    z = np.empty((10, V))
    z[0] = 5.0 + 1e-4 * n[0]
    z[1] = 1e-6 * n[1]
    z[2] = -3.0 - 1e-5 * np.abs(n[2])
    z[3] = np.where(n[3] > -1.0, -1e4 - 1e3 * np.abs(n[3]), 2.0 * n[3])
    z[4] = 1e4 * n[4]
    z[5] = np.where(n[5] > 0, np.finfo(np.float32).min, n[5])
    z[6] = -50.0 * np.abs(n[6])
    z[7] = 1e-38 * n[7]
    z[8] = 1e30 * n[8]
    z[9] = np.round(n[9] * 8) / 8
    z = synth.store_round(z, dtype).astype(np.float64)
    f32 = np.float32
    for T in (1.0, 100.0, np.array([1e-4, 1e-6, 1e-5, 1e3, 1e4, 0.3, 50.0, 1e-38, 1e30, 0.2])):
        for f in (dict(p=0.5003), dict(k=300), dict(k=V // 2, p=0.731), dict(k=V - 3, p=0.99, m=0.2), dict(k=40, p=0.6)):
            run(ctx, z, dtype, T=T, u=rng.random(10).astype(f32), **f)


def test_infinities_nan_and_empty_rows():
    V = 1003
    rng = np.random.default_rng(7)
    ctx = make_ctx(V)
    z = rows_of(rng, 9, V, "f32")
    z[0] = -np.inf
    z[1] = np.nan
    z[2, :] = -np.inf
    z[2, 77] = -5.0
    z[3, ::2] = -np.inf
    z[4, ::3] = np.nan
    z[5, [3, 900]] = np.inf
    z[6] = np.finfo(np.float32).min
    z[7, 5] = np.finfo(np.float32).max
    z[8, 10:] = -np.inf
    for f in (dict(), dict(k=20), dict(p=0.7), dict(m=0.1), dict(k=5, p=0.9, m=0.3)):
        for u in (0.0, 0.6, np.float32(1.0) - np.float32(2.0) ** -24):
            run(ctx, z, "f32", u=u, **f)
    run(ctx, z, "f32", T=[0.0, -1.0, np.nan, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0], u=0.3)


def test_min_p_whose_bound_is_zero():
    """z_max + T ln(min_p) is 0 to the last bit, and the difference to z_max the same for hundreds of millions of floats around
    zero: finding the threshold must not go through them one by one.  (Tokens keep 1e-9 away from the border, where the
    logarithm's last bit decides nothing.)"""
    V = 1001
    rng = np.random.default_rng(19)
    ctx = make_ctx(V)
    T = np.array([0x3E8E9C82, 0x3F0E9C82, 0x3F0E9C82], np.uint32).view(np.float32)
    top = np.array([0x3F242FF9, 0x3FA42FF9, 0x3FA42FF9], np.uint32).view(np.float32)
    m = np.float32(0.1)
    assert all(float(z) + float(t) * np.log(float(m)) == 0.0 for z, t in zip(top, T))
    z = -np.abs(rng.standard_normal((3, V))) - 1e-3
    z[:, 5:400] = np.abs(rng.standard_normal((3, 395))) * 0.1 + 1e-3
    z[:, 600:604] = [1e-9, -1e-9, 1e-5, -1e-5]
    z[np.arange(3), [77, 0, V - 1]] = top
    z = synth.store_round(np.minimum(z, top[:, None]), "f32").astype(np.float64)
    for f in (dict(m=m), dict(m=m, p=0.9), dict(m=m, k=500)):
        run(ctx, z, "f32", T=T, u=rng.random(3), **f)
    assert ctx.read_status() == 0


def test_strides_alignment_and_missing_arguments():
    rng = np.random.default_rng(9)
    V = 1000
    ctx = make_ctx(V)
    for dtype in ("f32", "bf16"):
        z = rows_of(rng, 4, V, dtype)
        for stride, offset in ((V, 0), (V + 8, 0), (V + 3, 1), (V + 1, 3)):
            run(ctx, z, dtype, k=30, p=0.9, u=rng.random(4), stride=stride, offset=offset)
        run(ctx, z, dtype, k=30, p=0.9, u=None)
        run(ctx, z, dtype, p=0.9, u=rng.random(4), filtered=False)
        run(ctx, z, dtype, u=rng.random(4), filtered=False)


def test_replayed_from_a_graph_and_on_another_stream():
    """A captured call reads its inputs anew; a call on a side stream gives the same bits."""
    rng = np.random.default_rng(15)
    V, R = 32000, 5
    ctx = make_ctx(V)
    z, u = rows_of(rng, R, V, "f32"), rng.random(R).astype(np.float32)
    kw = dict(k=200, p=0.93, m=0.001)
    tok, out = run(ctx, z, "f32", T=0.9, u=u, **kw)
    f = lambda x, t: dev(np.full(R, x, t))
    zd, ud, par = dev(z.astype(np.float32)), dev(u), (f(0.9, np.float32), f(200, np.int32), f(0.93, np.float32), f(0.001, np.float32))
    tok2, out2 = torch.zeros_like(tok), torch.zeros_like(out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ctx.sample(zd, *par, ud, tok2, out2)
    side.synchronize()
    assert torch.equal(tok, tok2) and torch.equal(out, out2)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ctx.sample(zd, *par, ud, tok2, out2)
    for seed in (16, 17):
        z = rows_of(np.random.default_rng(seed), R, V, "f32")
        zd.copy_(dev(z.astype(np.float32)))
        g.replay()
        torch.cuda.synchronize()
        for r in range(R):
            want, kept = pg.sample_row(z[r], np.float32(0.9).item(), 200, np.float32(0.93).item(), np.float32(0.001).item(), u[r].item())
            assert int(tok2[r]) == want and np.array_equal(host(out2[r]) > -np.inf, kept)
    assert ctx.read_status() == 0


def test_the_draw_follows_the_distribution():
    """Over a grid of u the share of each token is its probability: exact up to the grid's step."""
    V, n = 50, 4000
    rng = np.random.default_rng(11)
    ctx = make_ctx(V)
    z = rows_of(rng, 1, V, "f32", 1.5)
    u = (np.arange(n) + 0.5) / n
    tok, _ = run(ctx, np.repeat(z, n, 0), "f32", T=0.8, u=u, filtered=False)
    p = np.exp((z[0] - z[0].max()) / np.float32(0.8))
    p /= p.sum()
    share = np.bincount(host(tok), minlength=V) / n
    assert np.all(np.abs(share - p) <= 1.0 / n + 1e-6)


def test_filtered_rows_feed_the_acceptance_walk():
    """Sampling acceptance on filtered target rows: only kept tokens are ever drawn or accepted, and without
    filters the walk's outcome is the one it has on the rows themselves."""
    rng = np.random.default_rng(13)
    w = synth.scaled(synth.WORKLOADS["tiny"], batch=1)
    ctx = jk.Context.for_workload(w)
    M, V, S, K = w.tree_size, w.vocab, w.n_slots, w.top_k
    parent = synth.random_tree(M, w.depth, 4)[None]
    depth = np.zeros((1, M), np.int32)
    for i in range(1, M):
        depth[0, i] = depth[0, parent[0, i]] + 1
    tok = rng.integers(0, V, (1, M)).astype(np.int32)
    logits = (rng.standard_normal((1, M, V)) * 2).astype(np.float32)
    for i in range(1, M):
        logits[0, parent[0, i], tok[0, i]] += 8.0
    draft = rng.standard_normal((1, S, K, V)).astype(np.float32)
    qslot = np.where(np.arange(M) < S, np.arange(M), -1).astype(np.int32)[None]
    tree = {"tok": dev(tok), "parent": dev(parent), "depth": dev(depth),
            "branch": torch.zeros(1, M, dtype=torch.int32, device="cuda"), "qslot": dev(qslot)}

    def accept(rows, T, ua, ub):
        kv_len = torch.tensor([64], dtype=torch.int32, device="cuda")
        n_acc, bonus = (torch.empty(1, dtype=torch.int32, device="cuda") for _ in "ab")
        idx, at = (torch.empty(1, w.depth, dtype=torch.int32, device="cuda") for _ in "ab")
        ctx.accept_and_compact(1, M, 1, T, rows, tree, dev(draft), S, dev(ua), dev(ub), 0, None, None, 0, 0, 200, kv_len,
                               n_acc, idx, at, bonus)
        return int(n_acc[0]), host(idx)[0].tolist(), int(bonus[0])

    filtered = torch.empty(M, V, device="cuda")
    for trial in range(12):
        ua, ub = rng.random((1, M)).astype(np.float32), rng.random((1, w.depth + 1)).astype(np.float32)
        ctx.sample(dev(logits[0]), dev(np.full(M, 0.8, np.float32)), out_logits=filtered)
        # (the draft's rows are divided by T inside the walk: hand it T = 1 on both sides)
        a = accept(filtered.view(1, M, V), 1.0, ua, ub)
        b = accept(dev((logits / np.float32(0.8)).astype(np.float32)), 1.0, ua, ub)
        assert a == b
        ctx.sample(dev(logits[0]), dev(np.full(M, 0.8, np.float32)), top_k=dev(np.full(M, 3, np.int32)), out_logits=filtered)
        n, idx, bonus = accept(filtered.view(1, M, V), 1.0, ua, ub)
        kept = host(filtered) > -np.inf
        path = [0] + idx[:n]
        for a_, b_ in zip(path, path[1:]):
            assert kept[a_, tok[0, b_]]
        assert kept[path[-1], bonus]
    assert ctx.read_status() == 0
