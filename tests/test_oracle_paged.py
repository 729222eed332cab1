"""Pins of the plain model of the paged 8-bit cache and of filtered sampling, and the refusals of the C entry
points that need no GPU."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as pg
from paper_2502_06282_b200 import binding as jk


def test_e4m3_table_is_torchs():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(pg.E4M3, want, equal_nan=True)


def test_e4m3_rounding_is_to_nearest_even():
    x = np.concatenate([np.linspace(-448, 448, 20001), np.geomspace(2.0 ** -12, 448, 4001),
                        (pg.E4M3[:126] + pg.E4M3[1:127]) / 2])                       # the ties
    want = torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    got = pg.e4m3_encode(x.astype(np.float32).astype(np.float64))
    assert np.array_equal(got, want)
    assert pg.e4m3_encode(np.array([1e9, -1e9, np.inf, np.nan])).tolist() == [0x7E, 0xFE, 0x7E, 0x7F]


@pytest.mark.parametrize("amax", [448.0, 448.0000305, 1.75, 1.7500001, 3.0, 2.0 ** -24, 1e-12, 0.0, 3e38])
def test_block_scale_is_the_smallest_power_of_two(amax):
    s = pg.block_scale(np.array([amax, -amax / 3]))
    assert math.frexp(s)[0] == 0.5 and s >= 2.0 ** -32
    assert amax <= 448 * s and (s == 2.0 ** -32 or amax > 448 * s / 2)


def test_attention_without_pages_is_tree_attention():
    from oracle import jakiro_oracle as orc
    rng = np.random.default_rng(0)
    c = pg.Cache(1, 2, 16, 1, 2, 2, 8)
    n, M = 11, 5
    src = rng.standard_normal((2, 1, 1, 2, n, 8))
    c.import_([0], [n], 0, src[0], src[1])
    q, kt, vt = rng.standard_normal((1, M, 4, 8)), rng.standard_normal((1, 2, M, 8)), rng.standard_normal((1, 2, M, 8))
    parent = np.array([[-1, 0, 0, 1, 2]])
    got, _ = pg.tree_attention(c, 0, q, kt, vt, parent, 0.3)
    want = orc.tree_verify_attn(q, np.concatenate([src[0][0], kt], 2), np.concatenate([src[1][0], vt], 2),
                                np.array([n]), parent, 0.3)
    assert np.allclose(got, want, rtol=1e-12, atol=1e-12)


def test_commit_and_import_agree():
    """Tokens that arrive one by one end up as the same pages as a whole prompt."""
    rng = np.random.default_rng(1)
    L, Hkv, d, ps, n = 2, 1, 4, 16, 53
    src = rng.standard_normal((2, L, 1, Hkv, n, d))
    a, b = (pg.Cache(L, 8, ps, 1, 4, Hkv, d) for _ in range(2))
    a.import_([0], [n], 0, src[0], src[1])
    for c in range(n):
        b.kv_len[0] = c + 1
        b.commit(src[0][:, :, :, c:c + 1], src[1][:, :, :, c:c + 1], [0], [[]], 1)
    assert a.table == b.table and a.free == b.free
    assert np.array_equal(a.pages, b.pages) and np.array_equal(a.scale, b.scale)
    r = slice(n // ps % 2 * ps, n // ps % 2 * ps + n % ps)
    assert np.array_equal(a.open[..., r, :], b.open[..., r, :])


def test_fork_free_compact_bookkeeping():
    rng = np.random.default_rng(2)
    c = pg.Cache(1, 12, 16, 5, 4, 1, 2)
    src = rng.standard_normal((2, 1, 3, 1, 60, 2))
    c.import_([0, 1, 2], [60, 33, 17], 0, src[0], src[1])
    c.fork([0, 0], [3, 4])
    assert [c.refcount[e] for e in c.table[0][:3]] == [3, 3, 3]
    before = c.columns(0, 0, 3, 0, [])
    c.release([0, 1])
    assert c.free[-2:] == [3, 4] and c.refcount[c.table[3][0]] == 2
    assert c.compact() == 1 and sorted(set(sum((r[:3] for r in c.table), []))) == [-1, 0, 1, 2, 3]
    assert np.array_equal(before, c.columns(0, 0, 3, 0, []))
    with pytest.raises(pg.Refused):
        c.fork([3], [4])


def test_sampling_rule_by_hand():
    z = np.log([0.4, 0.1, 0.1, 0.25, 0.15])
    tok, kept = pg.sample_row(z, top_k=3)
    assert kept.tolist() == [True, False, False, True, True] and tok == 0
    assert pg.sample_row(z, top_k=4)[1].tolist() == [True, True, False, True, True]      # tie: lower index
    assert pg.sample_row(z, top_p=0.6)[1].tolist() == [True, False, False, True, False]
    assert pg.sample_row(z, top_p=0.0)[1].tolist() == [True, False, False, False, False]
    assert pg.sample_row(z, min_p=0.3)[1].tolist() == [True, False, False, True, True]
    # cumulative sums in index order over the kept: 0.4, 0.65, 0.8 of 0.8
    assert [pg.sample_row(z, top_k=3, u=u)[0] for u in (0.0, 0.49, 0.51, 0.8, 0.82, 0.999)] == [0, 0, 3, 3, 4, 4]
    assert pg.sample_row(z, temperature=0.0, u=0.9)[0] == 0
    assert pg.sample_row([-np.inf, np.nan])[0] == -1
    assert pg.sample_row([np.nan, 1.0, np.inf, np.inf], u=0.7)[0] == 3


# ------------------------------------------------------------------------------------------
# refusals that come back before anything is launched
# ------------------------------------------------------------------------------------------
ALIGNED = 1 << 20


def _context(dtype="bf16", **kw):
    cfg = dict(hidden=64, n_experts=2, top_k=1, inter=64, vocab=64, n_q_heads=4, n_kv_heads=2, head_dim=64,
               max_batch=2, max_tree=8, max_depth=4, max_frontier=2, k_per_expert=2, dtype=dtype, allocate=False)
    ctx = jk.Context(**{**cfg, **kw})
    # a workspace nobody touches: the call itself may fail where there is no device, the pointer is kept
    jk.lib().jk_set_workspace(ctx._h, None, ALIGNED, ctx.workspace_bytes)
    return ctx


def _cache(**kw):
    f = dict(n_layers=2, n_pages=8, page_size=16, max_seqs=4, max_pages=4)
    p = {n: ALIGNED for n, _ in jk.JkPaged._fields_[5:]}
    return jk.JkPaged(**{**f, **p, **kw})


no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="a made-up workspace is only given without a device")


@no_gpu
@pytest.mark.parametrize("change,code", [
    (dict(page_size=48), "SHAPE"), (dict(page_size=0), "SHAPE"), (dict(n_pages=0), "SHAPE"),
    (dict(n_pages=(1 << 24) + 1), "SHAPE"), (dict(max_seqs=1025), "SHAPE"), (dict(max_pages=0), "SHAPE"),
    (dict(max_pages=1 << 30), "SHAPE"), (dict(n_layers=0), "SHAPE"), (dict(k_pages=None), "NULL"),
    (dict(scratch=None), "NULL"), (dict(v_open=ALIGNED + 8), "ALIGN"), (dict(k_scale=ALIGNED + 4), "ALIGN"),
    (dict(kv_len=ALIGNED + 2), "ALIGN")])
def test_descriptor_refusals(change, code):
    ctx, c = _context(), _cache(**change)
    L, want = jk.lib(), jk.ERR[code]
    r = C.byref(c)
    assert L.jk_paged_init(ctx._h, None, r) == want
    assert L.jk_paged_import(ctx._h, None, r, 1, None, ALIGNED, 0, 1, ALIGNED, ALIGNED, 2048, 1024, 16) == want
    assert L.jk_tree_verify_attn_paged(ctx._h, None, r, 0, 1, 1, ALIGNED, ALIGNED, ALIGNED, 128, 64, ALIGNED, 1.0,
                                     ALIGNED) == want
    assert L.jk_paged_commit(ctx._h, None, r, 1, 1, ALIGNED, ALIGNED, 128, 64, ALIGNED, ALIGNED) == want
    assert L.jk_paged_fork(ctx._h, None, r, 1, ALIGNED, ALIGNED) == want
    assert L.jk_paged_free(ctx._h, None, r, 1, ALIGNED) == want
    assert L.jk_paged_compact(ctx._h, None, r, None) == want
    assert L.jk_paged_copy(ctx._h, None, C.byref(_cache()), r, 1, ALIGNED, ALIGNED) == want


@no_gpu
def test_argument_refusals():
    ctx, c = _context(), _cache()
    L, E, A, r = jk.lib(), jk.ERR, ALIGNED, C.byref(c)
    attn = lambda layer=0, B=1, M=1, q=A, kt=A, sb=128, sh=64, par=A, scale=1.0, out=A: \
        L.jk_tree_verify_attn_paged(ctx._h, None, r, layer, B, M, q, kt, A, sb, sh, par, scale, out)
    assert attn(layer=2) == E["SHAPE"] and attn(layer=-1) == E["SHAPE"]
    assert attn(B=0) == E["SHAPE"] and attn(M=0) == E["SHAPE"] and attn(scale=0.0) == E["SHAPE"]
    assert attn(scale=math.nan) == E["SHAPE"]
    assert attn(B=3) == E["CAPACITY"] and attn(M=9, sh=1024) == E["CAPACITY"]
    assert attn(M=4) == E["SHAPE"]                               # a head's tree rows would overlap the next head's
    assert attn(q=None) == E["NULL"] and attn(par=None) == E["NULL"]
    assert attn(q=A + 8) == E["ALIGN"] and attn(out=A + 2) == E["ALIGN"] and attn(sh=68) == E["ALIGN"]
    imp = lambda B=1, n=A, l0=0, nl=2, k=A, sb=2048, sh=1024, rows=16: \
        L.jk_paged_import(ctx._h, None, r, B, None, n, l0, nl, k, A, sb, sh, rows)
    assert imp(B=5) == E["CAPACITY"] and imp(B=0) == E["SHAPE"] and imp(l0=1) == E["SHAPE"]
    assert imp(l0=-1) == E["SHAPE"] and imp(nl=0) == E["SHAPE"] and imp(n=None) == E["NULL"]
    assert imp(rows=17) == E["SHAPE"] and imp(sb=2044) == E["ALIGN"] and imp(sb=-8) == E["SHAPE"]
    com = lambda B=1, M=1, sh=64, n=A: L.jk_paged_commit(ctx._h, None, r, B, M, A, A, 128, sh, n, A)
    assert com(B=3) == E["CAPACITY"] and com(M=9, sh=640) == E["CAPACITY"] and com(M=2) == E["SHAPE"]
    assert com(n=None) == E["NULL"]
    assert L.jk_paged_fork(ctx._h, None, r, 5, A, A) == E["CAPACITY"]
    assert L.jk_paged_fork(ctx._h, None, r, 0, A, A) == E["SHAPE"]
    assert L.jk_paged_free(ctx._h, None, r, 5, A) == E["CAPACITY"]
    assert L.jk_paged_compact(ctx._h, None, r, A + 1) == E["ALIGN"]
    copy = lambda d, n=1: L.jk_paged_copy(ctx._h, None, r, C.byref(d), n, A, A)
    assert copy(_cache(page_size=32)) == E["SHAPE"] and copy(_cache(n_layers=1)) == E["SHAPE"]
    assert copy(_cache(), n=9) == E["CAPACITY"] and copy(_cache(n_pages=4)) == E["SHAPE"]     # the same arrays
    assert copy(_cache(v_pages=A + 4096)) == E["SHAPE"]
    assert L.jk_paged_init(None, None, r) == E["NULL"] and L.jk_paged_init(ctx._h, None, None) == E["NULL"]
    bare = jk.Context(hidden=64, n_experts=2, top_k=1, inter=64, vocab=64, n_q_heads=4, n_kv_heads=2, head_dim=64,
                      max_batch=2, max_tree=8, max_depth=4, max_frontier=2, k_per_expert=2, dtype="bf16",
                      allocate=False)
    assert L.jk_paged_init(bare._h, None, r) == E["WORKSPACE"]
    assert [L.jk_paged_scratch_ints(n) for n in (0, -1, (1 << 24) + 1, 1)] == [0, 0, 0, 67]


@no_gpu
def test_copy_refuses_pools_that_overlap_in_part():
    ctx = _context()                                    # 2 heads of 64: a block of codes is 1024 bytes, a pool 2 x 8 x 2 of them
    L, E, MB = jk.lib(), jk.ERR, 1 << 20
    at = dict(k_pages=1 * MB, v_pages=2 * MB, k_scale=3 * MB, v_scale=4 * MB)
    other = dict(k_pages=5 * MB, v_pages=6 * MB, k_scale=7 * MB, v_scale=8 * MB)
    copy = lambda **kw: L.jk_paged_copy(ctx._h, None, C.byref(_cache(**at)), C.byref(_cache(**{**other, **kw})), 1, ALIGNED, ALIGNED)
    codes, scales = 2 * 8 * 2 * 1024, 2 * 8 * 2 * 4
    for name in ("k_pages", "v_pages"):
        for a in (MB, 2 * MB):
            assert copy(**{name: a + codes - 16}) == E["SHAPE"] and copy(**{name: a - codes + 16}) == E["SHAPE"]
            assert copy(**{name: a + codes}) == E["CUDA"] and copy(**{name: a - codes}) == E["CUDA"]      # (no device here)
    for name in ("k_scale", "v_scale"):
        for a in (3 * MB, 4 * MB):
            assert copy(**{name: a}) == E["SHAPE"] and copy(**{name: a + scales - 16}) == E["SHAPE"]
            assert copy(**{name: a + scales}) == E["CUDA"]
    one = lambda **kw: L.jk_paged_copy(ctx._h, None, C.byref(_cache(**at)), C.byref(_cache(**{**at, **kw})), 1, ALIGNED, ALIGNED)
    assert one(k_scale=9 * MB) == E["SHAPE"] and one(v_scale=9 * MB) == E["SHAPE"] and one() == E["CUDA"]


@no_gpu
def test_sample_refusals():
    ctx = _context()
    L, E, A = jk.lib(), jk.ERR, ALIGNED
    s = lambda rows=1, z=A, dt=0, stride=64, T=None, u=A, tok=A, out=None: \
        L.jk_sample(ctx._h, None, rows, z, dt, stride, T, None, None, None, u, tok, out)
    assert s(rows=0) == E["SHAPE"] and s(stride=63) == E["SHAPE"] and s(dt=2) == E["DTYPE"]
    assert s(z=None) == E["NULL"] and s(u=None) == E["NULL"] and s(tok=None) == E["NULL"]
    assert s(z=A + 2) == E["ALIGN"] and s(T=A + 1) == E["ALIGN"] and s(tok=A + 2) == E["ALIGN"]


@no_gpu
def test_sample_refuses_filtered_rows_over_its_input():
    ctx = _context()
    L, E, A = jk.lib(), jk.ERR, ALIGNED
    s = lambda out, rows=3, dt=0, stride=80: L.jk_sample(ctx._h, None, rows, A, dt, stride, None, None, None, None, None, None, out)
    V = ctx.cfg.vocab
    end = (2 * 80 + V) * 4                              # of the logits, from their start
    for at in (0, 4, -4, end - 4, 4 - 3 * V * 4):
        assert s(A + at) == E["SHAPE"]
    assert s(A + (2 * 80 + V) * 2 - 4, dt=1) == E["SHAPE"]


# ------------------------------------------------------------------------------------------
# what the binding refuses before the library is called (a stand-in records the calls; nothing runs)
# ------------------------------------------------------------------------------------------
class _Recorder:
    def __init__(self):
        self.calls, self.real = [], jk.lib()

    def __getattr__(self, name):
        if name in ("jk_destroy", "jk_paged_scratch_ints"):
            return getattr(self.real, name)

        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


@pytest.fixture
def recorded(monkeypatch):
    ctx = jk.Context(hidden=64, n_experts=2, top_k=1, inter=64, vocab=64, n_q_heads=4, n_kv_heads=2, head_dim=64,
                     max_batch=2, max_tree=8, max_depth=4, max_frontier=2, k_per_expert=2, dtype="bf16", allocate=False)
    rec = _Recorder()
    monkeypatch.setattr(jk, "lib", lambda: rec)
    monkeypatch.setattr(jk, "_stream", lambda: 0)
    return ctx, rec


def _tensors(Hkv=2, d=64, T=torch.bfloat16):
    L, n, ps, seqs, cols = 2, 8, 16, 4, 4
    i32 = dict(dtype=torch.int32)
    page = lambda: torch.zeros(L, n, Hkv, ps, d, dtype=torch.uint8)
    opened = lambda: torch.zeros(L, seqs, Hkv, 2 * ps, d, dtype=T)
    return dict(k_pages=page(), v_pages=page(), k_scale=torch.zeros(L, n, Hkv), v_scale=torch.zeros(L, n, Hkv),
                k_open=opened(), v_open=opened(), kv_len=torch.zeros(seqs, **i32),
                page_table=torch.zeros(seqs, cols, **i32), refcount=torch.zeros(n, **i32),
                free_list=torch.zeros(n, **i32), n_free=torch.zeros(1, **i32))


def test_binding_refuses_tree_arrays_that_do_not_go_together(recorded):
    ctx, rec = recorded
    cache = jk.PagedCache.from_tensors(ctx, _tensors())
    B, M, T = 2, 3, torch.bfloat16
    z = lambda *s, t=T: torch.zeros(*s, dtype=t)
    good = dict(q=z(B, M, 4, 64), k=z(B, 2, 5, 64), v=z(B, 2, 5, 64), parent=z(B, M, t=torch.int32), out=z(B, M, 4, 64))
    wide = z(B, 2, 5, 128)
    bad = [dict(v=z(B, 2, 6, 64)), dict(v=z(B, 2, 6, 64)[:, :, :5]), dict(v=z(B, 5, 2, 64).transpose(1, 2)),
           dict(k=wide[..., :64], v=wide[..., :64]), dict(k=wide[..., ::2], v=wide[..., ::2]),
           dict(k=z(B, 2, 5, 64, t=torch.float32)), dict(v=z(B, 2, 5, 64, t=torch.float16)),
           dict(k=z(B, 2, 2, 64), v=z(B, 2, 2, 64)), dict(k=z(1, 2, 5, 64), v=z(1, 2, 5, 64)),
           dict(k=z(B, 3, 5, 64), v=z(B, 3, 5, 64)), dict(parent=z(B, M, t=torch.float32)), dict(parent=z(B, 2, t=torch.int32)),
           dict(parent=z(M, B, t=torch.int32).t()), dict(q=z(B, M, 4, 64, t=torch.float32)), dict(q=z(B, M, 3, 64)),
           dict(q=z(B, 4, M, 64).transpose(1, 2)), dict(out=z(B, M, 4, 64, t=torch.float32)),
           dict(out=z(B, M, 8, 64)[:, :, ::2])]

    def attn(change={}):
        a = {**good, **change}
        ctx.tree_verify_attn_paged(cache, 0, B, M, a["q"], a["k"], a["v"], a["parent"], 0.1, a["out"])

    for change in bad:
        with pytest.raises(ValueError):
            attn(change)
    wq, x, depth = z(8 * 64, 64), z(B, M, 64), z(B, M, t=torch.int32)
    n = z(B, t=torch.int32)
    ok = dict(w=wq, x=x, depth=depth, q=good["q"], k=good["k"], v=good["v"], n=n)

    def qkv(change={}):
        a = {**ok, **change}
        ctx.verify_qkv_tree(a["w"], B, M, a["x"], a["depth"], a["q"], a["k"], a["v"], a["n"], 1e4)

    for change in [b for b in bad if b.keys() <= {"k", "v"}] + [
            dict(depth=depth.long()), dict(x=x.float()), dict(x=z(B, M, 32)), dict(n=n.long()), dict(n=n[:1]), dict(w=wq[:7 * 64])]:
        with pytest.raises(ValueError):
            qkv(change)
    assert not rec.calls
    attn()
    qkv()
    wide_parent = z(B, M, t=torch.int64)
    attn(dict(parent=wide_parent))                      # converted, not read as 32-bit words
    assert rec.calls.pop()[1][11] != wide_parent.data_ptr()
    # the stride of a dimension of one does not count
    single = torch.zeros(B, 2, 64, dtype=T)
    both = dict(k=z(B, 2, 5, 64)[:, :, :1], v=torch.as_strided(z(B * 2 * 5 * 64), (B, 2, 1, 64), (640, 320, 7, 1)))
    q, root, out = z(B, 1, 4, 64), z(B, 1, t=torch.int32), z(B, 1, 4, 64)
    ctx.tree_verify_attn_paged(cache, 0, B, 1, q, both["k"], both["v"], root, 0.1, out)
    ctx.tree_verify_attn_paged(cache, 0, B, 1, q, single[:, :, None], single[:, :, None], root, 0.1, out)
    assert [n for n, _ in rec.calls] == ["jk_tree_verify_attn_paged", "jk_verify_qkv_tree"] + 2 * ["jk_tree_verify_attn_paged"]
    assert rec.calls[0][1][9:11] == (640, 320) and rec.calls[3][1][9:11] == (128, 64)


def test_binding_refuses_lists_of_another_type_or_length(recorded):
    ctx, rec = recorded
    cache = jk.PagedCache.from_tensors(ctx, _tensors())
    i = lambda *s, t=torch.int32: torch.zeros(*s, dtype=t)
    p = i(2, t=torch.int64)
    bad = [lambda: ctx.paged_import(cache, 2, i(2, t=torch.int64), 0, 2, p, p, 2048, 1024, 16),
           lambda: ctx.paged_import(cache, 2, i(1), 0, 2, p, p, 2048, 1024, 16),
           lambda: ctx.paged_import(cache, 2, i(2), 0, 2, p, p, 2048, 1024, 16, seqs=i(1)),
           lambda: ctx.paged_import(cache, 2, i(2), 0, 2, p, p, 2048, 1024, 16, seqs=i(2, t=torch.int64)),
           lambda: ctx.paged_import(cache, 2, i(2), 0, 2, p[:1], p, 2048, 1024, 16),
           lambda: ctx.paged_import(cache, 2, i(2), 0, 2, p, p.float(), 2048, 1024, 16),
           lambda: ctx.paged_commit(cache, 2, 1, p, p, 128, 64, i(1), i(2, 4)),
           lambda: ctx.paged_commit(cache, 2, 1, p, p, 128, 64, i(2), i(2, 3)),
           lambda: ctx.paged_commit(cache, 2, 1, p, p, 128, 64, i(2), i(4, 2).t()),
           lambda: ctx.paged_commit(cache, 2, 1, p[:1], p, 128, 64, i(2), i(2, 4)),
           lambda: ctx.paged_fork(cache, i(2, t=torch.int64), i(2)), lambda: ctx.paged_fork(cache, i(4)[::2], i(2)),
           lambda: ctx.paged_free(cache, i(2, t=torch.int64)), lambda: ctx.paged_free(cache, i(4)[::2]),
           lambda: ctx.paged_compact(cache, i(1, t=torch.int64)),
           lambda: ctx.paged_copy(cache, cache, i(1), i(1, t=torch.int64))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    z, f = torch.zeros(3, 64), torch.zeros(3)
    good = dict(temperature=f, top_k=i(3), top_p=f, min_p=f, u=f, out_tok=i(3), out_logits=torch.zeros(3, 64))
    for change in [{n: good[n].double()} for n in good] + [{n: good[n][:2]} for n in good] + [
            dict(top_k=f), dict(u=torch.zeros(6)[::2]), dict(out_tok=i(3, t=torch.int64)),
            dict(out_logits=torch.zeros(3, 128)[:, :64]), dict(out_logits=torch.zeros(64, 3).t())]:
        with pytest.raises(ValueError):
            ctx.sample(z, **{**good, **change})
    assert not rec.calls
    ctx.sample(z, **good)
    ctx.sample(z, u=f, out_tok=i(3))
    assert len(rec.calls) == 2


def test_binding_refuses_rows_laid_out_for_another_size(recorded):
    """Larger tensors, dense, whose rows lie further apart than the library reads them."""
    ctx, rec = recorded
    cache = jk.PagedCache.from_tensors(ctx, _tensors())
    B, M, T = 2, 3, torch.bfloat16
    z = lambda *s, t=T: torch.zeros(*s, dtype=t)
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)
    k, p = z(B, 2, 5, 64), torch.zeros(2, dtype=torch.int64)
    attn = lambda q=z(B, M, 4, 64), par=i(B, M), out=z(B, M, 4, 64), B=B: \
        ctx.tree_verify_attn_paged(cache, 0, B, M, q, k, k.clone(), par, 0.1, out)
    qkv = lambda x=z(B, M, 64), depth=i(B, M), q=z(B, M, 4, 64), B=B: \
        ctx.verify_qkv_tree(z(8 * 64, 64), B, M, x, depth, q, k, k.clone(), i(B), 1e4)
    f = torch.zeros(3)
    for call in (lambda: attn(q=z(B, 5, 4, 64)), lambda: attn(par=i(B, 5)), lambda: attn(out=z(B, 5, 4, 64)),
                 lambda: attn(par=torch.zeros(B, 5, dtype=torch.int64)), lambda: qkv(x=z(B, 5, 64)), lambda: qkv(depth=i(B, 5)),
                 lambda: qkv(q=z(B, 5, 4, 64)), lambda: ctx.paged_commit(cache, B, M, p, p, 640, 320, i(B), i(B, 6)),
                 lambda: ctx.sample(torch.zeros(3, 64), u=f, out_tok=i(3), out_logits=torch.zeros(3, 80))):
        with pytest.raises(ValueError):
            call()
    assert not rec.calls
    attn()
    attn(q=z(B * 5 * 4 * 64), par=i(B * 5))              # flat
    attn(q=z(1, 5, 4, 64), par=i(1, 5), out=z(1, 5, 4, 64), B=1)      # one sequence has one row
    qkv()
    ctx.paged_commit(cache, B, M, p, p, 640, 320, i(B), i(B, 4))
    assert len(rec.calls) == 5


def test_binding_refuses_a_cache_of_another_context(recorded):
    ctx, rec = recorded
    other = jk.Context.__new__(jk.Context)
    other.cfg, other.tdtype, other._h = jk.JkConfig(n_kv_heads=1, head_dim=64), torch.bfloat16, None
    other.kv_kind = (1, 64, torch.bfloat16)
    cache = jk.PagedCache.from_tensors(other, _tensors(Hkv=1))
    i = torch.zeros(1, dtype=torch.int32)
    q, k = torch.zeros(1, 1, 4, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 1, 64, dtype=torch.bfloat16)
    mine = jk.PagedCache.from_tensors(ctx, _tensors())
    for call in (lambda: ctx.paged_init(cache), lambda: ctx.paged_free(cache, i), lambda: ctx.paged_fork(cache, i, i),
                 lambda: ctx.paged_compact(cache), lambda: ctx.paged_copy(mine, cache, i, i),
                 lambda: ctx.tree_verify_attn_paged(cache, 0, 1, 1, q, k, k, i, 0.1, q.clone())):
        with pytest.raises(ValueError):
            call()
    assert not rec.calls
