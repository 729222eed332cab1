"""Paged 8-bit KV cache on the device against the plain 64-bit model: bookkeeping, codes, scales and open rows bit
for bit, attention within a bound that is derived below."""
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as pg
from paper_2502_06282_b200 import binding as jk
from paper_2502_06282_b200 import synth
from tests.jk_testutil import Guard, dev, host

pytestmark = pytest.mark.gpu


def make_ctx(Hq, Hkv, d, B, M, dtype, depth=6, vocab=64):
    return jk.Context(hidden=64, n_experts=2, top_k=1, inter=64, vocab=vocab, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d,
                      max_batch=B, max_tree=M, max_depth=depth, max_frontier=1, k_per_expert=2, dtype=dtype)


class Pair:
    """A device cache and its model, side by side; every device array sits between canaries."""

    def __init__(self, ctx, L, n_pages, ps, max_seqs, max_pages):
        self.ctx, c = ctx, ctx.cfg
        self.ref = pg.Cache(L, n_pages, ps, max_seqs, max_pages, c.n_kv_heads, c.head_dim)
        plain = jk.PagedCache(ctx, n_layers=L, n_pages=n_pages, page_size=ps, max_seqs=max_seqs, max_pages=max_pages)
        self.guard = Guard()
        t = {n: self.guard.like(getattr(plain, n)) for n in jk.PagedCache._NAMES}
        for x in "kv":                                  # codes of NaN: a page nobody filled shows
            t[x + "_pages"].fill_(0x7F)
            t[x + "_scale"].fill_(1.0)
            t[x + "_open"].fill_(0.0)
        self.ref.pages[:] = 0x7F
        self.ref.scale[:] = 1.0
        self.dev = jk.PagedCache.from_tensors(ctx, t)
        ctx.paged_init(self.dev)
        self.dtype = ctx.dtype

    def draw(self, rng, shape, spread=1.0):
        x = synth.store_round(rng.standard_normal(shape) * spread, self.dtype)
        return x, dev(x, self.dtype)

    def same(self):
        """Everything the model says is on the device."""
        torch.cuda.synchronize()
        self.guard.check()
        r, d = self.ref, self.dev
        assert host(d.kv_len).tolist() == r.kv_len
        assert host(d.page_table).tolist() == r.table
        assert host(d.refcount).tolist() == r.refcount
        n = int(d.n_free[0])
        assert host(d.free_list)[:n].tolist() == r.free
        live = [e for e in range(r.n_pages) if r.refcount[e]]
        for i, x in enumerate("kv"):
            assert np.array_equal(host(getattr(d, x + "_pages"))[:, live], r.pages[i][:, live]), x
            assert np.array_equal(host(getattr(d, x + "_scale"))[:, live], r.scale[i][:, live]), x
            opened = host(getattr(d, x + "_open"))
            for b, length in enumerate(r.kv_len):
                for c in range(length // r.ps * r.ps, length):
                    at = c % (2 * r.ps)
                    assert np.array_equal(opened[:, b, :, at], r.open[i][:, b, :, at]), (x, b, c)


def ptrs(t):
    return torch.tensor([layer.data_ptr() for layer in t], dtype=torch.int64, device="cuda")


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def do_import(p, rng, seqs, lens, rows, layers=None, spread=1.0, src=None):
    r = p.ref
    n_l = layers or r.L
    shape = (n_l, len(lens), r.Hkv, rows, r.d)
    (k, kd), (v, vd) = src or (p.draw(rng, shape, spread), p.draw(rng, shape, spread))
    first = r.L - n_l
    p.ctx.paged_import(p.dev, len(lens), i32(lens), first, n_l, ptrs(kd), ptrs(vd), kd.stride(1), kd.stride(2), rows,
                       None if seqs is None else i32(seqs))
    return lambda: r.import_(list(range(len(lens))) if seqs is None else seqs, lens, first, k, v), (kd, vd)


def do_commit(p, rng, B, M, n_acc, idx, rows=None):
    r = p.ref
    shape = (r.L, B, r.Hkv, rows or M, r.d)
    (k, kd), (v, vd) = p.draw(rng, shape), p.draw(rng, shape)
    full = np.full((B, p.ctx.cfg.max_depth), -1, np.int32)
    for b in range(B):
        full[b, :len(idx[b])] = idx[b]
    acc = i32(n_acc)
    p.dev.kv_len[:B] += torch.where(acc >= 0, 1 + acc, acc * 0)
    r.kv_len[:B] = [n + (1 + a if a >= 0 else 0) for n, a in zip(r.kv_len, n_acc)]
    args = (p.dev, B, M, ptrs(kd), ptrs(vd), kd.stride(1), kd.stride(2), acc, dev(full))
    p.ctx.paged_commit(*args)
    return lambda: r.commit(k, v, n_acc, idx, M), args, (kd, vd)


SHAPES = [("bf16", 16, 128, 2), ("bf16", 64, 128, 3), ("bf16", 128, 128, 1), ("bf16", 32, 64, 2), ("f32", 16, 64, 1),
          ("f32", 128, 128, 2)]


@pytest.mark.parametrize("dtype,ps,d,Hkv", SHAPES)
def test_import_takes_prompts_of_any_length(dtype, ps, d, Hkv):
    rng = np.random.default_rng(ps + d)
    ctx = make_ctx(Hkv, Hkv, d, 2, 4, dtype)
    lens = [0, 1, ps - 1, ps, 5 * ps + 3]
    p = Pair(ctx, 2, 9, ps, 7, 6)
    src = []
    for _ in range(2):                                  # blocks of very different sizes, one all zero
        x, _ = p.draw(rng, (2, 5, Hkv, 5 * ps + 3, d))
        x *= np.exp2(rng.integers(-20, 20, size=(2, 5, Hkv, 1, 1))).astype(np.float32)
        x[:, 4, :, :ps] = 0.0
        x = synth.store_round(x, dtype)
        src.append((x, dev(x, dtype)))
    model, _ = do_import(p, rng, [6, 0, 3, 1, 4], lens, 5 * ps + 3, src=src)
    model()
    p.same()
    assert ctx.read_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_import_of_infinities_nan_and_tiny_values(dtype):
    """The scale follows the finite values; infinities become the largest code, NaN stays NaN."""
    rng = np.random.default_rng(6)
    ps, d = 32, 64
    ctx = make_ctx(2, 2, d, 1, 4, dtype)
    p = Pair(ctx, 1, 8, ps, 1, 7)
    big = float(np.finfo(np.float32).max) if dtype == "f32" else float(torch.finfo(torch.bfloat16).max)
    src = []
    for which in "kv":
        x, _ = p.draw(rng, (1, 1, 2, 6 * ps, d))
        x[0, 0, :, 3] = np.inf
        x[0, 0, :, ps + 1, ::3] = -np.inf
        x[0, 0, :, ps + 2, 5] = np.nan
        x[0, 0, :, 2 * ps:3 * ps] = np.nan             # nothing finite in the block
        x[0, 0, :, 3 * ps:4 * ps] *= np.float32(2.0 ** -40)
        x[0, 0, :, 4 * ps, 0] = big
        x[0, 0, :, 5 * ps:] = -0.0
        x = synth.store_round(x, dtype)
        src.append((x, dev(x, dtype)))
    model, _ = do_import(p, rng, None, [6 * ps], 6 * ps, src=src)
    model()
    torch.cuda.synchronize()
    p.guard.check()
    for i, name in enumerate("kv"):
        got, want = host(getattr(p.dev, name + "_pages"))[:, :6], p.ref.pages[i][:, :6]
        nan = (want & 0x7F) == 0x7F
        assert np.array_equal((got & 0x7F) == 0x7F, nan) and np.array_equal(got[~nan], want[~nan])
        assert np.array_equal(host(getattr(p.dev, name + "_scale"))[:, :6], p.ref.scale[i][:, :6])
    assert ctx.read_status() == 0


def test_import_layer_by_layer_and_again():
    rng = np.random.default_rng(5)
    ctx = make_ctx(2, 2, 64, 2, 4, "bf16")
    p = Pair(ctx, 3, 8, 16, 2, 4)
    src = p.draw(rng, (3, 2, 2, 50, 64)), p.draw(rng, (3, 2, 2, 50, 64))
    model, _ = do_import(p, rng, None, [50, 20], 50, layers=1, src=[(x[2:], xd[2:]) for x, xd in src])
    model()
    p.same()                                            # (last layer first; the others' codes are not set yet)
    model, _ = do_import(p, rng, None, [50, 20], 50, src=src)
    model()
    p.same()
    assert ctx.read_status() == 0


@pytest.mark.parametrize("dtype,ps,d,Hkv", SHAPES)
def test_commit_completes_pages(dtype, ps, d, Hkv):
    rng = np.random.default_rng(7 * ps + d)
    B, M = 5, 9
    ctx = make_ctx(Hkv, Hkv, d, B, M, dtype, depth=8)
    p = Pair(ctx, 2, 12 + 2 * B, ps, B + 1, 5)
    # a fresh sequence, one short of a page, at a page's border, past it, one that is skipped
    model, _ = do_import(p, rng, None, [0, ps - 1, ps, 2 * ps - 4, 7], 2 * ps)
    model()
    for n_acc, idx in (([0, 0, 3, 8, -1], [[], [], [2, 3, 8], [1, 2, 3, 4, 5, 6, 7, 8], []]),
                       ([4, 1, 0, 2, 0], [[1, 3, 5, 7], [8], [], [4, 6], []])):
        model, args, _keep = do_commit(p, rng, B, M, n_acc, idx, rows=M + 2)
        model()
        p.same()
        ctx.paged_commit(*args)                         # repeating it changes nothing
        p.same()
    assert ctx.read_status() == 0


def test_commit_can_complete_two_pages():
    rng = np.random.default_rng(9)
    ctx = make_ctx(1, 1, 64, 1, 32, "bf16", depth=16)
    p = Pair(ctx, 1, 6, 16, 1, 5)
    model, _keep1 = do_import(p, rng, None, [15], 15)
    model()
    model, _, _keep = do_commit(p, rng, 1, 32, [16], [list(range(3, 19))])
    model()
    p.same()
    assert p.ref.kv_len == [32] and ctx.read_status() == 0


def snapshot(p):
    return {n: getattr(p.dev, n).clone() for n in jk.PagedCache._NAMES}


def refuses(p, call, code):
    """The call sets `code` and changes nothing."""
    before = snapshot(p)
    call()
    assert p.ctx.read_status() == jk.ERR[code]
    for n, t in before.items():
        assert torch.equal(t.view(torch.uint8) if t.is_floating_point() else t,
                           getattr(p.dev, n).view(torch.uint8) if t.is_floating_point() else getattr(p.dev, n)), n
    p.guard.check()


def test_requests_that_cannot_be_met_change_nothing():
    rng = np.random.default_rng(11)
    ctx = make_ctx(1, 1, 64, 3, 4, "bf16", depth=4)
    p = Pair(ctx, 1, 5, 16, 4, 3)
    model, _keep = do_import(p, rng, [0, 1], [40, 17], 48)
    model()
    p.same()                                            # pages 0 1 | 2; free 4 3
    for seqs, lens, code in (([2, 2], [16, 16], "BOUNDS"), ([4], [1], "BOUNDS"), ([-1], [1], "BOUNDS"),
                             ([2], [49], "BOUNDS"), ([2], [-1], "BOUNDS"), ([0], [17], "BOUNDS"),
                             ([2], [48], "CAPACITY"), ([2, 3], [32, 16], "CAPACITY")):
        refuses(p, lambda: do_import(p, rng, seqs, lens, 48), code)
    big = [do_import(p, rng, [2], [32], 32, src=[p.draw(rng, (1, 1, 1, 32, 64)) for _ in "kv"])]
    big[0][0]()
    p.same()                                            # the pool is used up
    kt = torch.zeros(1, 3, 1, 4, 64, dtype=torch.bfloat16, device="cuda")

    def commit(n_acc, idx, B=3):
        full = np.full((B, 4), -1, np.int32)
        for b in range(B):
            full[b, :len(idx[b])] = idx[b]
        ctx.paged_commit(p.dev, B, 4, ptrs(kt), ptrs(kt), kt.stride(1), kt.stride(2), i32(n_acc), dev(full))

    p.dev.kv_len[:3] = i32([40 + 1, 17 + 1, 32 + 1])
    refuses(p, lambda: commit([0, 5, 0], [[], [], []]), "BOUNDS")           # n_acc > max_depth
    refuses(p, lambda: commit([0, 1, 0], [[], [4], []]), "BOUNDS")          # a node past the tree
    refuses(p, lambda: commit([0, 1, 0], [[], [-1], []]), "BOUNDS")
    p.dev.kv_len[1] = 1
    refuses(p, lambda: commit([0, 1, 0], [[], [1], []]), "BOUNDS")          # more accepted than there is
    p.dev.kv_len[:3] = i32([49, 18, 33])
    refuses(p, lambda: commit([0, 0, 0], [[], [], []]), "BOUNDS")           # past max_pages
    p.dev.kv_len[:3] = i32([48, 18, 33])
    refuses(p, lambda: commit([0, 0, 0], [[], [], []]), "CAPACITY")         # page 2 of row 0: none is free
    p.dev.kv_len[:3] = i32([40, 17, 32])
    p.same()
    for src, dst in (([0, 0], [3, 3]), ([0], [0]), ([3], [0]), ([0, 3], [3, 1]), ([0], [4]), ([-1], [3]), ([0], [1])):
        refuses(p, lambda: ctx.paged_fork(p.dev, i32(src), i32(dst)), "BOUNDS")
    for seqs in ([0, 0], [4], [-1]):
        refuses(p, lambda: ctx.paged_free(p.dev, i32(seqs)), "BOUNDS")
    # shared pages cannot be filled again
    ctx.paged_fork(p.dev, i32([0]), i32([3]))
    p.ref.fork([0], [3])
    p.same()
    refuses(p, lambda: do_import(p, rng, [0], [40], 48), "BOUNDS")
    # damaged bookkeeping: a page id outside the pool, a free list that names one, a count too low
    p.dev.page_table[1, 0] = 5
    refuses(p, lambda: ctx.paged_free(p.dev, i32([1])), "BOUNDS")
    refuses(p, lambda: do_import(p, rng, [1], [17], 48), "BOUNDS")
    p.dev.page_table[1, 0] = 0
    p.dev.refcount[0] = 2
    refuses(p, lambda: ctx.paged_free(p.dev, i32([0, 1, 3])), "BOUNDS")
    p.dev.page_table[1, 0] = 2
    p.same()
    ctx.paged_free(p.dev, i32([1]))
    p.ref.release([1])
    p.dev.free_list[0] = 5
    refuses(p, lambda: do_import(p, rng, [1], [16], 48), "BOUNDS")


@pytest.mark.parametrize("length", [-2 ** 31, -2 ** 31 + 1, -1, 0, 1, 2 ** 31 - 1])
def test_commit_refuses_lengths_that_cannot_be(length):
    rng = np.random.default_rng(12)
    ctx = make_ctx(1, 1, 64, 1, 4, "bf16", depth=4)
    p = Pair(ctx, 1, 4, 16, 1, 3)
    model, _keep = do_import(p, rng, None, [20], 20)
    model()
    kt = torch.zeros(1, 1, 1, 4, 64, dtype=torch.bfloat16, device="cuda")
    p.dev.kv_len.fill_(length)
    refuses(p, lambda: ctx.paged_commit(p.dev, 1, 4, ptrs(kt), ptrs(kt), kt.stride(1), kt.stride(2), i32([1]), i32([[1, 0, 0, 0]])),
            "BOUNDS")


@pytest.mark.parametrize("dtype,ps,d,Hkv", [("bf16", 16, 128, 2), ("f32", 32, 64, 1), ("bf16", 128, 64, 3)])
def test_fork_free_compact(dtype, ps, d, Hkv):
    rng = np.random.default_rng(13 + ps)
    ctx = make_ctx(Hkv, Hkv, d, 4, 6, dtype)
    p = Pair(ctx, 2, 30, ps, 9, 5)
    model, _keep = do_import(p, rng, [0, 1, 2, 3], [3 * ps + 5, 0, ps - 1, 4 * ps], 4 * ps)
    model()
    for src, dst in (([0, 0, 3], [8, 4, 6]), ([2, 4], [5, 7])):
        ctx.paged_fork(p.dev, i32(src), i32(dst))
        p.ref.fork(src, dst)
        p.same()
    model, _, _keep2 = do_commit(p, rng, 4, 6, [2, 0, 1, 5], [[1, 2], [], [3], [1, 2, 3, 4, 5]])
    model()
    p.same()                                            # forks keep what they had
    n_moved = torch.zeros(1, dtype=torch.int32, device="cuda")
    for gone in ([4], [0, 1, 5], [8, 6]):
        ctx.paged_free(p.dev, i32(gone))
        p.ref.release(gone)
        p.same()
        ctx.paged_compact(p.dev, n_moved)
        assert int(n_moved[0]) == p.ref.compact()
        p.same()
    ctx.paged_free(p.dev, i32(list(range(9))))
    p.ref.release(list(range(9)))
    ctx.paged_compact(p.dev)
    p.ref.compact()
    p.same()
    assert len(p.ref.free) == 30 and ctx.read_status() == 0


def test_compact_over_many_pages():
    """A pool of more pages than one round of the plan's block, holes everywhere."""
    rng = np.random.default_rng(17)
    ctx = make_ctx(1, 1, 64, 1, 1, "bf16")
    n_pages, seqs = 2600, 64
    p = Pair(ctx, 1, n_pages, 16, seqs, 40)
    perm = rng.permutation(n_pages)
    at = 0
    for b in range(seqs):
        n = int(rng.integers(0, 40))
        p.ref.table[b][:n] = perm[at:at + n].tolist()
        for e in perm[at:at + n]:
            p.ref.refcount[e] = 1
        p.ref.kv_len[b] = n * 16
        at += n
    p.ref.free = perm[at:].tolist()
    p.dev.page_table.copy_(i32(p.ref.table))
    p.dev.refcount.copy_(i32(p.ref.refcount))
    p.dev.kv_len.copy_(i32(p.ref.kv_len))
    p.dev.free_list[:len(p.ref.free)] = i32(p.ref.free)
    p.dev.n_free.fill_(len(p.ref.free))
    for x, kv in (("k", 0), ("v", 1)):
        p.ref.pages[kv] = rng.integers(0, 126, size=p.ref.pages[kv].shape)
        p.ref.scale[kv] = 2.0 ** rng.integers(-5, 5, size=p.ref.scale[kv].shape)
        getattr(p.dev, x + "_pages").copy_(dev(p.ref.pages[kv]))
        getattr(p.dev, x + "_scale").copy_(dev(p.ref.scale[kv].astype(np.float32)))
    p.same()
    gone = rng.permutation(seqs)[:23].tolist()
    ctx.paged_free(p.dev, i32(gone))
    p.ref.release(gone)
    p.same()
    n_moved = torch.zeros(1, dtype=torch.int32, device="cuda")
    ctx.paged_compact(p.dev, n_moved)
    assert int(n_moved[0]) == p.ref.compact() > 100
    p.same()


def test_free_and_compact_in_a_large_pool():
    """Pages far apart in a pool of many rounds of the plans' block; most rounds hold nothing."""
    rng = np.random.default_rng(18)
    ctx = make_ctx(1, 1, 64, 1, 1, "bf16")
    n_pages, seqs = 40000, 6
    p = Pair(ctx, 1, n_pages, 16, seqs, 30)
    perm = rng.permutation(n_pages)
    used = np.concatenate([perm[:100], np.arange(20), [n_pages - 1, 8191, 8192, 16384]])
    used = rng.permutation(np.unique(used))
    p.ref.refcount = [0] * n_pages
    for b in range(seqs):
        for t, e in enumerate(used[b * 20:(b + 1) * 20].tolist()):
            p.ref.table[b][t] = e
            p.ref.refcount[e] = 1
        p.ref.kv_len[b] = 16 * len(used[b * 20:(b + 1) * 20])
    p.ref.free = [e for e in perm.tolist() if not p.ref.refcount[e]]
    p.dev.page_table.copy_(i32(p.ref.table))
    p.dev.refcount.copy_(i32(p.ref.refcount))
    p.dev.kv_len.copy_(i32(p.ref.kv_len))
    p.dev.free_list[:len(p.ref.free)] = i32(p.ref.free)
    p.dev.n_free.fill_(len(p.ref.free))
    for x, kv in (("k", 0), ("v", 1)):
        p.ref.pages[kv] = rng.integers(0, 126, size=p.ref.pages[kv].shape)
        getattr(p.dev, x + "_pages").copy_(dev(p.ref.pages[kv]))
    for gone in ([1, 4], [0]):
        ctx.paged_free(p.dev, i32(gone))
        p.ref.release(gone)
        p.same()
        n_moved = torch.zeros(1, dtype=torch.int32, device="cuda")
        ctx.paged_compact(p.dev, n_moved)
        assert int(n_moved[0]) == p.ref.compact() > 0
        p.same()
    assert ctx.read_status() == 0


def test_copy_between_pools_and_inside_one():
    rng = np.random.default_rng(19)
    ctx = make_ctx(3, 3, 64, 2, 1, "bf16")
    a, b = Pair(ctx, 2, 9, 32, 2, 4), Pair(ctx, 2, 6, 32, 1, 4)
    model, _keep = do_import(a, rng, None, [128, 100], 128)
    model()
    ctx.paged_copy(a.dev, b.dev, i32([2, 6, 0]), i32([5, 0, 1]))
    torch.cuda.synchronize()
    for n in ("k_pages", "v_pages", "k_scale", "v_scale"):
        assert torch.equal(getattr(a.dev, n)[:, [2, 6, 0]], getattr(b.dev, n)[:, [5, 0, 1]])
    ctx.paged_copy(a.dev, a.dev, i32([1, 1]), i32([7, 8]))
    torch.cuda.synchronize()
    assert torch.equal(a.dev.k_pages[:, 7], a.dev.k_pages[:, 1]) and torch.equal(a.dev.v_scale[:, 8], a.dev.v_scale[:, 1])
    a.guard.check()
    b.guard.check()
    for src, dst in (([0, 1], [3, 3]), ([9], [0]), ([0], [6]), ([-1], [0]), ([0], [-1])):
        refuses(b, lambda: ctx.paged_copy(a.dev, b.dev, i32(src), i32(dst)), "BOUNDS")
    refuses(a, lambda: ctx.paged_copy(a.dev, a.dev, i32([0, 7]), i32([7, 8])), "BOUNDS")


# ------------------------------------------------------------------------------------------
# attention
# ------------------------------------------------------------------------------------------
def bound(out, size, dtype):
    """How far an element may be off.  bf16: the result is rounded once (2^-8 of it) and every softmax weight once:
    to bf16 over open and tree rows (2^-8 of sum p|v|), to fp16 over pages (2^-11); 2^-10 of that sum covers the rest:
    weights below 2^-31 of their row's reference that become 0 (2^-14 for 2^17 keys), fp32 products over 128
    elements (logits off by under 128 2^-24 sum|q k| scale = 2^-14 for these inputs) and the exponential (2^-22).
    f32, and one query row per kv head in bf16 (which rounds its result alone): the products' 2^-14 and as much for sums
    and the fast exponential."""
    if dtype == "bf16":
        return 2.0 ** -8 * np.abs(out) + (2.0 ** -8 + 2.0 ** -10) * size + 1e-30
    return 2.0 ** -13 * size + 1e-30


CASES = [
    # dtype, ps, d, Hq, Hkv, M, lens
    ("bf16", 16, 128, 2, 2, 1, [0, 1, 15, 16, 17, 333]),
    ("bf16", 64, 128, 8, 2, 1, [640, 127, 129]),
    ("bf16", 128, 128, 2, 2, 60, [127, 128, 1030]),
    ("bf16", 32, 128, 8, 1, 60, [95, 0, 700]),
    ("bf16", 64, 128, 16, 2, 128, [200, 63]),
    ("bf16", 64, 128, 3, 3, 17, [65, 66]),
    ("bf16", 16, 64, 4, 2, 33, [31, 250, 0]),
    ("bf16", 128, 64, 2, 1, 64, [257, 128]),
    ("bf16", 32, 64, 8, 1, 16, [40, 100]),
    ("f32", 16, 64, 4, 2, 16, [333, 7]),
    ("f32", 64, 128, 2, 1, 5, [130, 64, 0]),
]


def attention_case(dtype, ps, d, Hq, Hkv, M, lens, seed, layer=1, spread=1.0):
    rng = np.random.default_rng(seed)
    B = len(lens)
    ctx = make_ctx(Hq, Hkv, d, B, M, dtype)
    p = Pair(ctx, 2, sum(n // ps for n in lens) + 2, ps, B + 1, max(lens) // ps + 2)
    rows = max(max(lens), 1)
    shape = (2, B, Hkv, rows, d)
    src = []
    for which in "kv":                                   # pages whose sizes differ by up to 2^6
        x, _ = p.draw(rng, shape)
        x *= np.exp2(rng.integers(-3, 4, size=(2, B, Hkv, (rows + ps - 1) // ps))).repeat(ps, 3)[:, :, :, :rows, None]
        x = synth.store_round((x * (0.25 if which == "k" else 1.0)).astype(np.float32), dtype)
        src.append((x, dev(x, dtype)))
    model, keep = do_import(p, rng, None, lens, rows, src=src)
    model()
    torch.cuda.synchronize()
    q, qd = p.draw(rng, (B, M, Hq, d), spread)
    kt, ktd = p.draw(rng, (B, Hkv, M + 1, d))
    vt, vtd = p.draw(rng, (B, Hkv, M + 1, d))
    parent = np.stack([synth.random_tree(M, 6, seed + b) for b in range(B)])
    return ctx, p, q, qd, kt, ktd, vt, vtd, parent, layer


def check_attention(ctx, p, q, qd, kt, ktd, vt, vtd, parent, layer, scale=None):
    B, M, Hq, d = q.shape
    scale = scale or 1.0 / math.sqrt(d)
    g = Guard()
    out = g.alloc(q.shape, ctx.tdtype)
    ktd[:, :, M:] = float("nan")                        # rows behind the tree are nobody's
    vtd[:, :, M:] = float("nan")
    ctx.tree_verify_attn_paged(p.dev, layer, B, M, qd, ktd, vtd, dev(parent), scale, out)
    torch.cuda.synchronize()
    g.check()
    p.guard.check()
    assert ctx.read_status() == 0
    want, size = pg.tree_attention(p.ref, layer, q, kt[:, :, :M], vt[:, :, :M], parent, scale)
    off = np.abs(host(out) - want)
    assert np.all(off <= bound(want, size, p.dtype)), float((off / bound(want, size, p.dtype)).max())
    return out


@pytest.mark.parametrize("path", ["tensor", "cuda_core"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention(case, path):
    if path == "tensor" and CASES[case][0] == "f32":
        pytest.skip("one path in fp32")
    parts = attention_case(*CASES[case], seed=100 + case)
    parts[0].set_tensor_path(path == "tensor")
    # what lies in the open rows behind the live ones must not matter
    p = parts[1]
    for x in "kv":
        o = getattr(p.dev, x + "_open")
        for b, n in enumerate(p.ref.kv_len):
            dead = [r for r in range(2 * p.ref.ps) if r not in {c % (2 * p.ref.ps) for c in range(n // p.ref.ps * p.ref.ps, n)}]
            o[:, b, :, dead] = float("nan")
    a = check_attention(*parts)
    b = check_attention(*parts)
    assert torch.equal(a, b)                            # the same bits again


MORE = [
    # one query row per kv head: one to eight blocks of a cluster, runs that end inside a warp's step
    ("bf16", 16, 64, 3, 3, 1, [2049, 0, 127, 1024]),
    ("bf16", 64, 128, 1, 1, 1, [9000]),
    ("bf16", 128, 128, 40, 40, 1, [129] * 9),
    ("f32", 32, 64, 2, 2, 1, [4100, 3]),
    # few rows in fp32, and the first count that is not few
    ("f32", 32, 128, 4, 4, 4, [1500, 31]),
    ("f32", 16, 64, 8, 2, 4, [700, 3, 0]),
    ("f32", 64, 128, 1, 1, 17, [300]),
    # many units, so that partials are merged several rows per warp, in blocks of 16, 32 and 64 rows
    ("bf16", 16, 128, 16, 16, 9, [40, 7, 64, 0, 33] * 4),
    ("bf16", 16, 128, 16, 16, 20, [100, 16, 0, 47, 200, 31, 5, 64, 80, 1]),
    ("bf16", 32, 128, 10, 5, 60, [300, 17, 0, 129, 500, 64, 33, 200]),
    ("bf16", 32, 64, 10, 5, 60, [300, 17, 0, 129, 500, 64, 33, 200]),
    # a single unit over every CTA
    ("bf16", 64, 128, 1, 1, 5, [20000]),
]


@pytest.mark.parametrize("case", range(len(MORE)))
def test_attention_of_few_rows_and_of_many_units(case):
    parts = attention_case(*MORE[case], seed=200 + case)
    a = check_attention(*parts)
    b = check_attention(*parts)
    assert torch.equal(a, b)


def test_attention_with_a_sink_token_keeps_the_tail():
    """One key takes most of the weight, thousands share the rest: the small weights must not be lost."""
    rng = np.random.default_rng(23)
    d, n, M = 128, 4096, 4
    ctx = make_ctx(1, 1, d, 1, M, "bf16")
    p = Pair(ctx, 1, 70, 64, 1, 64)
    k = rng.standard_normal((1, 1, 1, n, d)) * 0.05
    q = np.ones((1, M, 1, d))
    k[0, 0, 0, 5] = 12.0 / (d * d ** -0.5)              # logit 12 against about 0: e^-12 = 2^-17.3 per other key
    v = rng.standard_normal((1, 1, 1, n, d)) * 0.1 + 1.0
    v[0, 0, 0, 5] = -1.0
    k, v = synth.store_round(k.astype(np.float32), "bf16"), synth.store_round(v.astype(np.float32), "bf16")
    model, _keep = do_import(p, rng, None, [n], n, src=[(k, dev(k, "bf16")), (v, dev(v, "bf16"))])
    model()
    kt, ktd = p.draw(rng, (1, 1, M + 1, d), 0.05)
    vt, vtd = p.draw(rng, (1, 1, M + 1, d), 0.1)
    q = q.astype(np.float32)
    check_attention(ctx, p, q, dev(q, "bf16"), kt, ktd, vt, vtd, np.array([[-1, 0, 1, 1]]), 0)


@pytest.mark.parametrize("spread", [1e-3, 30.0])
def test_attention_with_small_and_large_queries(spread):
    parts = attention_case("bf16", 64, 128, 4, 2, 20, [300, 70], seed=31, spread=spread)
    scale = 1.0 / math.sqrt(128) / max(1.0, spread)
    check_attention(*parts, scale=scale)


@pytest.mark.parametrize("d,Hq,M", [(128, 8, 6), (64, 4, 20), (128, 2, 3), (64, 1, 9)])
def test_attention_of_rows_of_very_different_size(d, Hq, M):
    """Rows 2^14 times as large as others of their block must not cost these their bits.  A query value may be off by 2^-13 of
    its row's largest, sums of products by 2^-16 of the products' sizes (256 additions in fp32): logits by Delta, weights and
    the result by exp(2 Delta) - 1 of sum p|v|."""
    ctx, p, q, qd, kt, ktd, vt, vtd, parent, layer = attention_case("bf16", 32, d, Hq, 1, M, [200, 70], seed=33)
    size_of = np.where(np.arange(Hq * M).reshape(M, Hq) % 3 == 0, 1.0, 2.0 ** -14)
    size_of[-1] = [0.0] + [2.0 ** -6] * (Hq - 1)        # a row of zeros, and rows between
    q = (q * size_of[None, :, :, None]).astype(np.float32)
    scale = 2.0 ** 12 / math.sqrt(d)
    out = torch.empty_like(qd)
    ctx.tree_verify_attn_paged(p.dev, layer, 2, M, dev(q, "bf16"), ktd, vtd, dev(parent), scale, out)
    want, size = pg.tree_attention(p.ref, layer, q, kt[:, :, :M], vt[:, :, :M], parent, scale)
    assert ctx.read_status() == 0
    for b in range(2):
        k = np.abs(p.ref.columns(0, layer, b, 0, kt[b, 0, :M]))
        aq = np.abs(q[b].astype(np.float64))
        delta = scale * (2.0 ** -13 * aq.max(-1) * k.sum(1).max() + 2.0 ** -16 * (aq @ k.T).max(-1))
        assert delta[size_of == 2.0 ** -14].max() < 2.0 ** -7
        off = np.abs(host(out)[b] - want[b])
        assert np.all(off <= bound(want[b], size[b], "bf16") + np.expm1(np.minimum(2 * delta, 50.0))[..., None] * size[b])


@pytest.mark.parametrize("path", ["tensor", "cuda_core"])
def test_attention_of_an_infinite_query_is_nan(path):
    """An infinite query value makes every logit of its row infinite or NaN, and the softmax NaN: not a number that was
    made finite on the way to 8 bits.  The other rows stay what they are."""
    ctx, p, q, qd, kt, ktd, vt, vtd, parent, layer = attention_case("bf16", 32, 128, 4, 1, 6, [200, 70], seed=34)
    ctx.set_tensor_path(path == "tensor")
    q[0, 2, 1, 7], q[1, 0, 3, 100] = np.inf, -np.inf
    kt[..., 7] = -1.0                                    # (the open and tree keys' logits -inf, the pages' of either sign)
    ktd[..., 7] = -1.0
    p.ref.open[0, ..., 7] = -1.0
    p.dev.k_open[..., 7] = -1.0
    out = torch.empty_like(qd)
    ctx.tree_verify_attn_paged(p.dev, layer, 2, 6, dev(q, "bf16"), ktd, vtd, dev(parent), 0.1, out)
    with np.errstate(invalid="ignore"):
        want, size = pg.tree_attention(p.ref, layer, q, kt[:, :, :6], vt[:, :, :6], parent, 0.1)
    got, nan = host(out), np.isnan(want)
    assert nan[0, 2, 1].all() and nan[1, 0, 3].all() and nan.sum() == 2 * 128
    assert np.array_equal(np.isnan(got), nan)
    assert np.all(np.abs(got - want)[~nan] <= bound(want, size, "bf16")[~nan])


@pytest.mark.parametrize("dtype,path,M", [("bf16", "tensor", 5), ("bf16", "tensor", 60), ("bf16", "tensor", 1),
                                          ("bf16", "cuda_core", 5), ("f32", "cuda_core", 1)])
@pytest.mark.parametrize("at", [0, 9984, 19840])
def test_attention_over_a_run_of_keys_that_are_nan(dtype, path, M, at):
    """A run of NaN keys that one block of threads has to itself is not lost when the blocks' parts are put together."""
    rng = np.random.default_rng(M)
    n, d = 20000, 128
    ctx = make_ctx(1, 1, d, 1, M, dtype)
    ctx.set_tensor_path(path == "tensor")
    p = Pair(ctx, 1, 157, 128, 1, 157)
    (k, kd), src_v = p.draw(rng, (1, 1, 1, n, d), 0.25), p.draw(rng, (1, 1, 1, n, d))
    kd[:, :, :, at:at + 128] = float("nan")
    _, _keep = do_import(p, rng, None, [n], n, src=[(k, kd), src_v])
    q, qd = p.draw(rng, (1, M, 1, d))
    (kt, ktd), (vt, vtd) = p.draw(rng, (1, 1, M, d)), p.draw(rng, (1, 1, M, d))
    out = torch.empty_like(qd)
    ctx.tree_verify_attn_paged(p.dev, 0, 1, M, qd, ktd, vtd, dev(synth.random_tree(M, 6, 1)[None]), 0.1, out)
    assert ctx.read_status() == 0 and bool(out.isnan().all())


def test_attention_refuses_what_is_out_of_range():
    parts = attention_case("bf16", 16, 128, 2, 2, 8, [40, 20], seed=41)
    ctx, p, q, qd, kt, ktd, vt, vtd, parent, layer = parts
    out = torch.empty_like(qd)

    def status():
        ctx.tree_verify_attn_paged(p.dev, layer, 2, 8, qd, ktd, vtd, dev(parent), 0.1, out)
        return ctx.read_status()

    assert status() == 0
    p.dev.page_table[0, 1] = p.ref.n_pages
    assert status() == jk.ERR["BOUNDS"]
    p.dev.page_table[0, 1] = -1
    assert status() == jk.ERR["BOUNDS"]
    p.dev.page_table[0, 1] = p.ref.table[0][1]
    for n in (-1, p.ref.max_pages * 16 + 1):
        p.dev.kv_len[1] = n
        assert status() == jk.ERR["BOUNDS"]
    p.dev.kv_len[1] = 20
    check_attention(*parts)


def test_attention_replayed_from_a_graph_and_on_another_stream():
    parts = attention_case("bf16", 32, 128, 4, 2, 12, [100, 33], seed=43)
    ctx, p, q, qd, kt, ktd, vt, vtd, parent, layer = parts
    want = check_attention(*parts)
    par = dev(parent)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.zeros_like(qd)
    with torch.cuda.stream(side):
        ctx.tree_verify_attn_paged(p.dev, layer, 2, 12, qd, ktd, vtd, par, 1.0 / math.sqrt(128), out)
    side.synchronize()
    assert torch.equal(out, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ctx.tree_verify_attn_paged(p.dev, layer, 2, 12, qd, ktd, vtd, par, 1.0 / math.sqrt(128), out)
    for length in (33, 20):                             # the graph reads the lengths anew
        p.dev.kv_len[1] = length
        p.ref.kv_len[1] = length
        p.ref.open[:, :, 1, :, :] = 0.0
        opened = torch.zeros_like(p.dev.k_open[:, 1])
        p.dev.k_open[:, 1] = opened
        p.dev.v_open[:, 1] = opened
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        want, size = pg.tree_attention(p.ref, layer, q, kt[:, :, :12], vt[:, :, :12], parent, 1.0 / math.sqrt(128))
        assert np.all(np.abs(host(out) - want) <= bound(want, size, "bf16"))


@pytest.mark.parametrize("M", [1, 20])
def test_two_contexts_read_one_cache_at_once(M):
    """Attention calls of different contexts may overlap on one cache: each has its own workspace."""
    parts = attention_case("bf16", 32, 128, 4, 4, M, [900, 333, 64], seed=51)
    ctx, p, q, qd, kt, ktd, vt, vtd, parent, layer = parts
    want = check_attention(*parts)
    other = make_ctx(4, 4, 128, 3, M, "bf16")
    seen = jk.PagedCache.from_tensors(other, {n: getattr(p.dev, n) for n in jk.PagedCache._NAMES})
    par, outs = dev(parent), [torch.zeros_like(qd) for _ in range(12)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for i, out in enumerate(outs):
        c, cache = (ctx, p.dev) if i % 2 else (other, seen)
        with torch.cuda.stream(streams[i % 2]):
            c.tree_verify_attn_paged(cache, layer, 3, M, qd, ktd, vtd, par, 1.0 / math.sqrt(128), out)
    torch.cuda.synchronize()
    assert all(torch.equal(out, want) for out in outs)
    assert ctx.read_status() == 0 and other.read_status() == 0


def test_verify_qkv_tree_is_verify_qkv_at_other_rows():
    for dtype in ("f32", "bf16"):
        w = synth.scaled(synth.WORKLOADS["tiny" if dtype == "f32" else "tiny_bf16"], batch=2)
        ctx = jk.Context.for_workload(w)
        B, M, T = 2, w.tree_size, ctx.tdtype
        g = torch.Generator(device="cuda").manual_seed(3)
        r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(T)
        wq = r((w.n_q_heads + 2 * w.n_kv_heads) * w.head_dim, w.hidden) * 0.02
        x, q = r(B, M, w.hidden), r(B, M, w.n_q_heads, w.head_dim)
        depth = torch.randint(0, 5, (B, M), generator=g, device="cuda").int()
        kv_len = i32([100, 3])
        kc, vc = (torch.zeros(B, w.n_kv_heads, 160, w.head_dim, dtype=T, device="cuda") for _ in "kv")
        ctx.verify_qkv(wq, B, M, x, depth, q, kc, vc, kv_len, 1e4)
        q2 = torch.zeros_like(q)
        kt, vt = (torch.zeros(B, w.n_kv_heads, M + 3, w.head_dim, dtype=T, device="cuda") for _ in "kv")
        ctx.verify_qkv_tree(wq, B, M, x, depth, q2, kt, vt, kv_len, 1e4)
        torch.cuda.synchronize()
        assert torch.equal(q, q2) and ctx.read_status() == 0
        for b, n in enumerate((100, 3)):
            assert torch.equal(kt[b, :, :M], kc[b, :, n:n + M]) and torch.equal(vt[b, :, :M], vc[b, :, n:n + M])
        assert not kt[:, :, M:].any() and not vt[:, :, M:].any()


# dtype, path, tree rows: one row per kv head, one row block of four and two of them, tensor blocks of 16 and 64 rows
FEW = [("bf16", "tensor", 1), ("f32", "cuda_core", 1), ("f32", "cuda_core", 3), ("bf16", "cuda_core", 5), ("bf16", "tensor", 5),
       ("bf16", "tensor", 40)]


def check_without_page_0(ps, d, dtype, path, M, owner):
    """Sequences that do not hold page 0, next to whatever lies there, at lengths that end inside a warp's step and a tile."""
    rng = np.random.default_rng(ps + d + M)
    lens = [ps, 3 * ps + 5, 0, 5 * ps, 9 * ps + 1]
    B, rows, Hkv = len(lens), 9 * ps + 1, 2
    ctx = make_ctx(Hkv, Hkv, d, B, M, dtype)
    ctx.set_tensor_path(path == "tensor")
    p = Pair(ctx, 2, sum(n // ps for n in lens) + 2, ps, B + 1, 11)
    seqs = list(range(B))
    if owner == "another sequence":                     # the row behind the call's takes page 0
        seqs, lens = [B] + seqs, [ps] + lens
    else:
        p.ref.free = [0] + list(range(p.ref.n_pages - 1, 0, -1))
        p.dev.free_list.copy_(i32(p.ref.free))
        for x in "kv":
            getattr(p.dev, x + "_scale").fill_(float("nan"))
    src = []
    for _ in "kv":
        x, _keep = p.draw(rng, (2, len(lens), Hkv, rows, d))
        if owner == "another sequence":
            x[:, 0, :, ::3] = np.nan
        src.append((x, dev(x, dtype)))
    model, _keep = do_import(p, rng, seqs, lens, rows, src=src)
    model()
    assert all(0 not in p.ref.table[b] for b in range(B))
    q, qd = p.draw(rng, (B, M, Hkv, d))
    (kt, ktd), (vt, vtd) = p.draw(rng, (B, Hkv, M + 1, d)), p.draw(rng, (B, Hkv, M + 1, d))
    parent = np.stack([synth.random_tree(M, 6, b) for b in range(B)])
    check_attention(ctx, p, q, qd, kt, ktd, vt, vtd, parent, 1)


@pytest.mark.parametrize("dtype,path,M", FEW)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("ps", [16, 32, 64, 128])
def test_attention_next_to_a_sequence_with_nan(ps, d, dtype, path, M):
    check_without_page_0(ps, d, dtype, path, M, "another sequence")


@pytest.mark.parametrize("dtype,path,M", FEW)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("ps", [16, 32, 64, 128])
def test_attention_next_to_a_page_nobody_filled(ps, d, dtype, path, M):
    """Codes and scales of NaN in the pages that no sequence holds."""
    check_without_page_0(ps, d, dtype, path, M, "nobody")


# ------------------------------------------------------------------------------------------
# the calls together, as a server uses them
# ------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_steps_of_a_server(dtype):
    rng = np.random.default_rng(51)
    B, M, L, ps, Hq, Hkv, d, V = 3, 12, 2, 16, 4, 2, 64, 64
    ctx = make_ctx(Hq, Hkv, d, B, M, dtype, vocab=V)
    p = Pair(ctx, L, 24, ps, 6, 8)
    model, _keep = do_import(p, rng, None, [37, 16, 0], 48)
    model()
    p.same()
    scale = d ** -0.5
    tok = np.tile(np.arange(M, dtype=np.int32), (B, 1))
    for step in range(4):
        parent = np.stack([synth.random_tree(M, 6, 60 + 10 * step + b) for b in range(B)])
        depth = np.zeros((B, M), np.int32)
        for b in range(B):
            for i in range(1, M):
                depth[b, i] = depth[b, parent[b, i]] + 1
        (k, kd), (v, vd) = p.draw(rng, (L, B, Hkv, M, d)), p.draw(rng, (L, B, Hkv, M, d))
        q, qd = p.draw(rng, (B, M, Hq, d))
        for layer in range(L):
            out = torch.empty_like(qd)
            ctx.tree_verify_attn_paged(p.dev, layer, B, M, qd, kd[layer], vd[layer], dev(parent), scale, out)
            want, size = pg.tree_attention(p.ref, layer, q, k[layer], v[layer], parent, scale)
            assert np.all(np.abs(host(out) - want) <= bound(want, size, dtype))
        # greedy acceptance along planted paths; the walk counts them into kv_len
        logits = rng.standard_normal((B, M, V)).astype(np.float32)
        for b in range(B):
            for i in range(1, M):
                if rng.random() < 0.6:
                    logits[b, parent[b, i], tok[b, i]] = 9.0 + rng.random()
        n_acc, acc_idx = torch.empty(B, dtype=torch.int32, device="cuda"), torch.empty(B, 6, dtype=torch.int32, device="cuda")
        acc_tok, bonus = torch.empty_like(acc_idx), torch.empty_like(n_acc)
        zero = torch.zeros(B, M, dtype=torch.int32, device="cuda")
        tree = {"tok": dev(tok), "parent": dev(parent), "depth": dev(depth), "branch": zero, "qslot": zero}
        before = list(p.ref.kv_len)
        ctx.accept_and_compact(B, M, 0, 1.0, dev(logits), tree, None, 0, None, None, 0, None, None, 0, 0,
                               p.ref.max_pages * ps, p.dev.kv_len, n_acc, acc_idx, acc_tok, bonus)
        ctx.paged_commit(p.dev, B, M, ptrs(kd), ptrs(vd), kd.stride(1), kd.stride(2), n_acc, acc_idx)
        na, idx = host(n_acc).tolist(), host(acc_idx).tolist()
        p.ref.kv_len[:B] = [n + 1 + a for n, a in zip(before, na)]
        p.ref.commit(k, v, na, idx, M)
        p.same()
    # two continuations of sequence 0, the others end, the pool is packed; attention reads the same numbers
    q, qd = p.draw(rng, (B, 1, Hq, d))
    (k, kd), (v, vd) = p.draw(rng, (B, Hkv, 1, d)), p.draw(rng, (B, Hkv, 1, d))
    root = torch.full((B, 1), -1, dtype=torch.int32, device="cuda")
    first, second = torch.empty_like(qd), torch.empty_like(qd)
    ctx.tree_verify_attn_paged(p.dev, 1, B, 1, qd, kd, vd, root, scale, first)
    ctx.paged_fork(p.dev, i32([0, 0]), i32([3, 5]))
    ctx.paged_free(p.dev, i32([1, 2]))
    ctx.paged_fork(p.dev, i32([3, 5]), i32([1, 2]))
    ctx.paged_free(p.dev, i32([3, 5, 0]))
    ctx.paged_compact(p.dev)
    p.ref.fork([0, 0], [3, 5])
    p.ref.release([1, 2])
    p.ref.fork([3, 5], [1, 2])
    p.ref.release([3, 5, 0])
    p.ref.compact()
    p.same()
    qd[1], kd[1], vd[1] = qd[0].clone(), kd[0].clone(), vd[0].clone()
    ctx.tree_verify_attn_paged(p.dev, 1, 2, 1, qd, kd, vd, root, scale, second)
    torch.cuda.synchronize()
    assert torch.equal(first[0], second[1]) or np.all(
        np.abs(host(first[0]) - host(second[1])) <= 2 * bound(host(first[0]), np.abs(host(first[0])) + 1.0, dtype))
    assert ctx.read_status() == 0


@pytest.mark.parametrize("dtype,path,M", FEW)
def test_attention_after_the_pool_was_packed(dtype, path, M):
    """Rows that came from forks, over pages that were shared, freed and moved, against the model within the bound."""
    rng = np.random.default_rng(61 + M)
    ps, d, Hq, Hkv, B = 16, 64, 4, 2, 3
    ctx = make_ctx(Hq, Hkv, d, B, M, dtype)
    ctx.set_tensor_path(path == "tensor")
    p = Pair(ctx, 2, 40, ps, 7, 9)
    model, _keep = do_import(p, rng, [0, 3, 1, 5, 2], [40, 133, 16, 90, 7], 133)
    model()
    for op, a, b in (("free", [0, 1], None), ("fork", [3, 5], [0, 1]), ("free", [3, 2], None), ("fork", [0, 5], [2, 6]), ("free", [5], None)):
        if op == "free":
            ctx.paged_free(p.dev, i32(a))
            p.ref.release(a)
        else:
            ctx.paged_fork(p.dev, i32(a), i32(b))
            p.ref.fork(a, b)
    moved = torch.zeros(1, dtype=torch.int32, device="cuda")
    ctx.paged_compact(p.dev, moved)
    assert int(moved[0]) == p.ref.compact() > 0
    p.same()
    assert p.ref.kv_len[:B] == [133, 90, 133] and p.ref.table[0][:8] == p.ref.table[2][:8]
    q, qd = p.draw(rng, (B, M, Hq, d))
    (kt, ktd), (vt, vtd) = p.draw(rng, (B, Hkv, M + 1, d)), p.draw(rng, (B, Hkv, M + 1, d))
    parent = np.stack([synth.random_tree(M, 6, b) for b in range(B)])
    check_attention(ctx, p, q, qd, kt, ktd, vt, vtd, parent, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_steps_replayed_from_a_graph(dtype):
    """Acceptance, commit and the next attention captured once; every replay works on the tree and the lengths it finds."""
    rng = np.random.default_rng(71)
    B, M, L, ps, Hq, Hkv, d, V = 2, 9, 2, 16, 4, 2, 64, 64
    ctx = make_ctx(Hq, Hkv, d, B, M, dtype, vocab=V)
    p = Pair(ctx, L, 24, ps, 3, 8)
    model, _keep = do_import(p, rng, None, [30, 15], 48)
    model()
    z32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    n_acc, acc_idx, acc_tok, bonus = z32(B), z32(B, 6), z32(B, 6), z32(B)
    parent, depth = z32(B, M), z32(B, M)
    tree = {"tok": dev(np.tile(np.arange(M, dtype=np.int32), (B, 1))), "parent": parent, "depth": depth, "branch": z32(B, M),
            "qslot": z32(B, M)}
    logits = torch.zeros(B, M, V, device="cuda")
    kd, vd = (torch.zeros(L, B, Hkv, M, d, dtype=ctx.tdtype, device="cuda") for _ in "kv")
    qd, out = (torch.zeros(B, M, Hq, d, dtype=ctx.tdtype, device="cuda") for _ in "ab")
    kp, vp = ptrs(kd), ptrs(vd)

    def step():
        ctx.accept_and_compact(B, M, 0, 1.0, logits, tree, None, 0, None, None, 0, None, None, 0, 0, p.ref.max_pages * ps,
                               p.dev.kv_len, n_acc, acc_idx, acc_tok, bonus)
        ctx.paged_commit(p.dev, B, M, kp, vp, kd.stride(1), kd.stride(2), n_acc, acc_idx)
        ctx.tree_verify_attn_paged(p.dev, 1, B, M, qd, kd[1], vd[1], parent, d ** -0.5, out)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(5):
        par = np.stack([synth.random_tree(M, 6, 80 + 10 * turn + b) for b in range(B)])
        dep, lg = np.zeros((B, M), np.int32), rng.standard_normal((B, M, V)).astype(np.float32)
        for b in range(B):
            for i in range(1, M):
                dep[b, i] = dep[b, par[b, i]] + 1
                if rng.random() < 0.6:
                    lg[b, par[b, i], i] = 9.0 + rng.random()
        (k, kx), (v, vx), (q, qx) = p.draw(rng, kd.shape), p.draw(rng, vd.shape), p.draw(rng, qd.shape)
        for t, x in ((parent, dev(par)), (depth, dev(dep)), (logits, dev(lg)), (kd, kx), (vd, vx), (qd, qx)):
            t.copy_(x)
        before = list(p.ref.kv_len)
        if turn < 4:
            graph.replay()
        else:
            step()                                       # and a call outside the graph goes on from there
        torch.cuda.synchronize()
        na, idx = host(n_acc).tolist(), host(acc_idx).tolist()
        p.ref.kv_len[:B] = [n + 1 + a for n, a in zip(before, na)]
        p.ref.commit(k, v, na, idx, M)
        p.same()
        want, size = pg.tree_attention(p.ref, 1, q, k[1], v[1], par, d ** -0.5)
        assert np.all(np.abs(host(out) - want) <= bound(want, size, dtype))
    assert ctx.read_status() == 0


@pytest.mark.parametrize("dtype,path,M", FEW)
def test_pages_past_32_bits_of_offset(dtype, path, M):
    """Pools of more than 4 GB, the pages in use at their end: the same bits as from a small pool."""
    rng = np.random.default_rng(81)
    ps, d, Hkv, L = 128, 128, 8, 2
    ctx = make_ctx(Hkv, Hkv, d, 2, M, dtype)
    ctx.set_tensor_path(path == "tensor")
    small = jk.PagedCache(ctx, n_layers=L, n_pages=8, page_size=ps, max_seqs=2, max_pages=5)
    large = jk.PagedCache(ctx, n_layers=L, n_pages=17000, page_size=ps, max_seqs=2, max_pages=5)
    assert large.k_pages.numel() > 2 ** 32
    large.free_list.copy_(torch.arange(17000, dtype=torch.int32, device="cuda"))      # 16999 first
    lens, rows = i32([3 * ps + 17, 2 * ps + 127]), 4 * ps
    T = ctx.tdtype
    r = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda().to(T)
    k, v, q = r(L, 2, Hkv, rows, d), r(L, 2, Hkv, rows, d), r(2, M, Hkv, d)
    kt, vt = r(L, 2, Hkv, M, d), r(L, 2, Hkv, M, d)
    parent = dev(np.stack([synth.random_tree(M, 6, b) for b in range(2)]))
    n_acc, idx = i32([0, 0]), torch.full((2, 6), -1, dtype=torch.int32, device="cuda")

    def attn(cache):
        out = torch.empty_like(q)
        ctx.tree_verify_attn_paged(cache, L - 1, 2, M, q, kt[-1], vt[-1], parent, d ** -0.5, out)
        return out

    first = []
    for cache in (small, large):
        ctx.paged_import(cache, 2, lens, 0, L, ptrs(k), ptrs(v), k.stride(1), k.stride(2), rows)
        first.append(attn(cache))
        cache.kv_len += 1                                # the root joins; sequence 1 completes a page
        ctx.paged_commit(cache, 2, M, ptrs(kt), ptrs(vt), kt.stride(1), kt.stride(2), n_acc, idx)
    assert torch.equal(*first) and not first[0].isnan().any()
    want = attn(small)
    assert host(large.page_table)[1].tolist() == [16996, 16995, 16994, -1, -1]
    assert torch.equal(attn(large), want)
    ctx.paged_copy(large, small, i32([16994, 16999]), i32([6, 7]))
    for n in ("k_pages", "v_pages", "k_scale", "v_scale"):
        assert torch.equal(getattr(small, n)[:, 6], getattr(large, n)[:, 16994])
        assert torch.equal(getattr(small, n)[:, 7], getattr(large, n)[:, 16999])
    ctx.paged_compact(large)
    assert sorted(host(large.page_table)[:, :3].ravel().tolist()) == list(range(6))
    assert torch.equal(attn(large), want) and ctx.read_status() == 0
