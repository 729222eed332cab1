"""What the calls of a target layer refuse, before anything is launched (host only: no call here reaches a device)."""
import ctypes as C
import random
import sys

import pytest
import torch

from paper_2502_06282_b200 import binding as jk

E = jk.ERR
X, W, OUT, SCALE, RES, BIAS = 1 << 32, 2 << 32, 3 << 32, 4 << 32, 5 << 32, 6 << 32


@pytest.fixture(scope="module")
def lib():
    from paper_2502_06282_b200 import build
    build.build()
    return jk.lib()


def make_ctx(dtype="bf16", d=64):
    return jk.Context(hidden=8, n_experts=1, top_k=1, inter=8, vocab=8, n_q_heads=4, n_kv_heads=2, head_dim=d, max_batch=1,
                      max_tree=1, max_depth=1, max_frontier=1, k_per_expert=1, dtype=dtype, allocate=False)


@pytest.mark.parametrize("rows,n,want", [(1, 32, 512), (128, 128, 512), (129, 128, 1024), (1, 160, 1024), (0, 32, 0),
                                         (1, 0, 0), (1, 33, 0), (1 << 24, 32, (1 << 17) * 512), ((1 << 24) + 1, 32, 0),
                                         (1, (1 << 20) + 32, 0), (-5, 32, 0)])
def test_scale_bytes(lib, rows, n, want):
    assert lib.jk_row_scale_bytes(rows, n) == want


NORM = dict(rows=4, n=64, x=X, delta=None, weight=W, out_sum=None, out=OUT, mx8=None, scale=None)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("change,code", [
    (dict(x=None), "NULL"), (dict(out=None), "NULL"), (dict(mx8=SCALE), "NULL"), (dict(scale=SCALE), "NULL"),
    (dict(rows=0), "SHAPE"), (dict(rows=-1), "SHAPE"), (dict(n=0), "SHAPE"), (dict(n=12), "SHAPE"),
    (dict(n=32776), "SHAPE"), (dict(n=40, mx8=SCALE, scale=RES), "SHAPE"),
    (dict(x=X + 8), "ALIGN"), (dict(weight=W + 2), "ALIGN"), (dict(out=OUT + 8), "ALIGN"),
    (dict(out=X + 16), "SHAPE"), (dict(out=W), "SHAPE"), (dict(out_sum=OUT), "SHAPE"),
    (dict(delta=RES, out=RES + 32), "SHAPE"), (dict(mx8=X, scale=SCALE), "SHAPE"), (dict(mx8=SCALE, scale=SCALE), "SHAPE")])
def test_norm_refuses(lib, dtype, change, code):
    a, ctx = {**NORM, **change}, make_ctx(dtype)
    rc = lib.jk_add_norm(ctx._h, None, a["rows"], a["n"], a["x"], a["delta"], a["weight"], a["out_sum"], a["out"],
                         a["mx8"], a["scale"])
    assert rc == E[code]


@pytest.mark.parametrize("rows,n,x,stride,out,scale,code", [
    (1, 32, None, 0, OUT, SCALE, "NULL"), (1, 32, X, 0, None, SCALE, "NULL"), (1, 32, X, 0, OUT, None, "NULL"),
    (0, 32, X, 0, OUT, SCALE, "SHAPE"), (1, 40, X, 0, OUT, SCALE, "SHAPE"), (2, 64, X, 32, OUT, SCALE, "SHAPE"),
    (2, 64, X, 65, OUT, SCALE, "ALIGN"), (2, 64, X + 2, 0, OUT, SCALE, "ALIGN"), (2, 64, X, 0, X + 64, SCALE, "SHAPE"),
    (2, 64, X, 0, OUT, OUT + 16, "SHAPE")])
def test_quantize_refuses(lib, rows, n, x, stride, out, scale, code):
    ctx = make_ctx()
    assert lib.jk_quantize_rows(ctx._h, None, rows, n, x, stride, out, scale) == E[code]


OP = dict(n_out=64, n_in=64, operands=0, act=0, w=W, w_scale=None, bias=None, w_up=None, w_up_scale=None, bias_up=None)
CALL = dict(rows=4, x=X, x_scale=None, x_stride=0, residual=None, r_stride=0, out=OUT, out_type=0, out_scale=None, o_stride=0)
MX = dict(operands=2, w_scale=SCALE, x_scale=SCALE + (1 << 20))


@pytest.mark.parametrize("change,code", [
    (dict(w=None), "NULL"), (dict(x=None), "NULL"), (dict(out=None), "NULL"), (dict(operands=1), "DTYPE"),
    (dict(operands=7), "DTYPE"), (dict(out_type=3), "DTYPE"), (dict(out_type=2), "NULL"), ({**MX, "x_scale": None}, "NULL"),
    ({**MX, "w_scale": None}, "NULL"), ({**MX, "w_up": RES}, "NULL"), (dict(act=3), "SHAPE"), (dict(act=-1), "SHAPE"),
    (dict(bias_up=BIAS), "SHAPE"), (dict(rows=0), "SHAPE"), (dict(rows=(1 << 20) + 1), "SHAPE"), (dict(n_out=0), "SHAPE"),
    (dict(n_in=0), "SHAPE"), (dict(n_in=20), "SHAPE"), (dict(n_in=(1 << 17) + 8), "SHAPE"), ({**MX, "n_in": 72}, "SHAPE"),
    (dict(n_out=(1 << 20) + 1), "SHAPE"), (dict(n_out=40, out_type=2, out_scale=SCALE), "SHAPE"), (dict(x_stride=32), "SHAPE"),
    (dict(x_stride=-64), "SHAPE"), (dict(residual=RES, r_stride=63), "SHAPE"), (dict(o_stride=63), "SHAPE"),
    ({**MX, "x_stride": 128}, "SHAPE"), (dict(out_type=2, out_scale=SCALE, o_stride=96), "SHAPE"), (dict(x_stride=68), "ALIGN"),
    (dict(x=X + 8), "ALIGN"), (dict(w=W + 4), "ALIGN"), (dict(bias=BIAS + 2), "ALIGN"), (dict(out=OUT + 2), "ALIGN"),
    (dict(out=X), "SHAPE"), (dict(out=W + 128), "SHAPE"), (dict(residual=OUT + 128), "SHAPE"),
    (dict(residual=OUT, r_stride=128), "SHAPE"), (dict(residual=OUT, out_type=1), "SHAPE"), (dict(bias=OUT + 16), "SHAPE"),
    (dict(out_type=2, out_scale=OUT + 16), "SHAPE"), (dict(out_type=2, out_scale=X), "SHAPE"),
    ({**MX, "out": SCALE}, "SHAPE"), ({}, "WORKSPACE"), (dict(residual=OUT), "WORKSPACE"), (MX, "WORKSPACE")])
def test_linear_refuses(lib, change, code):
    a, ctx = {**OP, **CALL, **change}, make_ctx()
    op = jk.JkLinearOp(*[a[k] for k in OP])
    rc = lib.jk_linear(ctx._h, None, C.byref(op), a["rows"], a["x"], a["x_scale"], a["x_stride"], a["residual"],
                       a["r_stride"], a["out"], a["out_type"], a["out_scale"], a["o_stride"])
    assert rc == E[code]


@pytest.mark.parametrize("off,code", [(128, "WORKSPACE"), (112, "SHAPE"), (384, "WORKSPACE"), (400, "SHAPE"), (-128, "WORKSPACE"),
                                      (-112, "SHAPE"), (-384, "WORKSPACE"), (-400, "SHAPE"), (512 + 128, "WORKSPACE"),
                                      (512, "SHAPE"), (3 * 512 + 112, "SHAPE"), (3 * 512 + 128, "WORKSPACE"), (4 * 512, "WORKSPACE")])
@pytest.mark.parametrize("beside", ["x", "residual"])
def test_linear_columns_of_one_buffer(lib, beside, off, code):
    """Rows of 128 bytes, 512 apart: out may lie between the rows of x or of the residual, and may not reach into one."""
    op, ctx = jk.JkLinearOp(*OP.values()), make_ctx()
    x, res = (X, RES) if beside == "x" else (RES, X)
    assert lib.jk_linear(ctx._h, None, C.byref(op), 4, x, None, 256, res, 256, X + off, 0, None, 256) == E[code]


def test_linear_refuses_null_context_and_projection(lib):
    op, ctx = jk.JkLinearOp(*OP.values()), make_ctx()
    tail = (4, X, None, 0, None, 0, OUT, 0, None, 0)
    assert lib.jk_linear(None, None, C.byref(op), *tail) == E["NULL"]
    assert lib.jk_linear(ctx._h, None, None, *tail) == E["NULL"]


Q, K, V, POS = 7 << 32, 8 << 32, 9 << 32, 10 << 32
ROPE = dict(batch=2, n=3, qkv=X, stride=0, pos=POS, sections=(32,), theta=1e4, q=Q, k=K, v=V, sb=2 * 640, sh=640, rows=10,
            first=None)


@pytest.mark.parametrize("change,code", [
    (dict(qkv=None), "NULL"), (dict(pos=None), "NULL"), (dict(sections=None), "NULL"), (dict(q=None), "NULL"),
    (dict(k=None), "NULL"), (dict(v=None), "NULL"), (dict(batch=0), "SHAPE"), (dict(batch=65536), "SHAPE"), (dict(n=0), "SHAPE"),
    (dict(n=11), "SHAPE"), (dict(sections=()), "SHAPE"), (dict(sections=(8, 8, 8, 4, 4)), "SHAPE"), (dict(sections=(31,)), "SHAPE"),
    (dict(sections=(40, -8)), "SHAPE"), (dict(sections=(16, 8)), "SHAPE"), (dict(theta=0.0), "SHAPE"),
    (dict(theta=float("nan")), "SHAPE"), (dict(theta=float("inf")), "SHAPE"), (dict(stride=504), "SHAPE"),
    (dict(stride=516), "ALIGN"), (dict(sh=632), "SHAPE"), (dict(sb=640), "SHAPE"), (dict(sb=-1280), "SHAPE"),
    (dict(sb=1284), "ALIGN"), (dict(q=Q + 8), "ALIGN"), (dict(pos=POS + 2), "ALIGN"), (dict(first=POS + 1), "ALIGN"),
    (dict(q=X + 512), "SHAPE"), (dict(k=X), "SHAPE"), (dict(v=K), "SHAPE"), (dict(q=K + 512), "SHAPE"), ({}, "WORKSPACE"),
    (dict(sb=640, sh=1280), "WORKSPACE")])
def test_rope_refuses(lib, change, code):
    a, ctx = {**ROPE, **change}, make_ctx()
    s = a["sections"]
    rc = lib.jk_rope_qkv(ctx._h, None, a["batch"], a["n"], a["qkv"], a["stride"], a["pos"], 1 if s is None else len(s),
                         None if s is None else (C.c_int32 * max(1, len(s)))(*s), a["theta"], a["q"], a["k"], a["v"], a["sb"],
                         a["sh"], a["rows"], a["first"])
    assert rc == E[code]


def test_binding_refuses_other_arrays(lib):
    """The binding's own checks, on host tensors (which it refuses as well)."""
    ctx = make_ctx()
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="multiple of 32"):
        jk.Mx8(torch.zeros(2, 40, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8))
    with pytest.raises(ValueError, match="512 contiguous bytes"):
        jk.Mx8(torch.zeros(2, 64, dtype=torch.uint8), torch.zeros(8, dtype=torch.uint8))
    with pytest.raises(ValueError, match="contiguous 8-bit"):
        jk.Mx8(torch.zeros(2, 64), torch.zeros(512, dtype=torch.uint8))
    for bad in (torch.zeros(4, 64), bf(4, 128)[:, :64], bf(4, 64)):
        with pytest.raises(ValueError):
            jk.Linear(ctx, bad)
    with pytest.raises(ValueError, match="act"):
        jk.Linear(ctx, bf(4, 64), act="tanh")
    with pytest.raises(ValueError, match="bias_up"):
        jk.Linear(ctx, bf(4, 64), bias_up=bf(4))
    for x, kw in ((bf(4, 64), {}), (torch.zeros(4, 64), {}), (bf(64), {}), (bf(4, 128)[:, ::2], {})):
        with pytest.raises(ValueError):
            ctx.add_norm(x, out=x, **kw)
    with pytest.raises(ValueError):
        ctx.rope_qkv(1, 2, bf(1, 2, 512), torch.zeros(1, 2, 2, dtype=torch.int32), (32,), 1e4, bf(1, 2, 4, 64), bf(1, 2, 2, 64),
                     bf(1, 2, 2, 64))
    with pytest.raises(ValueError):
        ctx.rope_qkv(1, 2, bf(1, 3, 512), torch.zeros(1, 2, dtype=torch.int32), (32,), 1e4, bf(1, 2, 4, 64), bf(1, 2, 2, 64),
                     bf(1, 2, 2, 64))


def test_binding_refuses_expanded_rows(lib):
    """Rows that are one row in memory: the library would take the distance of 0 for dense rows and reach past that row.
    (On host tensors, whose strides are looked at before their device.)"""
    ctx = make_ctx()
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    x, w, out = bf(4, 64), bf(96, 64), bf(4, 96)
    op = jk.Linear.__new__(jk.Linear)
    op.kind, op.struct = ctx.tdtype, jk.JkLinearOp(96, 64, 0, 0, w.data_ptr())
    op.address = C.addressof(op.struct)
    near = bf(1000).as_strided((4, 64), (32, 1))          # rows that share elements without being one
    for bad in (bf(1, 64).expand(4, 64), bf(64).expand(4, 64), near):
        with pytest.raises(ValueError, match="rows overlap"):
            ctx.linear(op, bad, out)
    for a in ((x, bf(1, 96).expand(4, 96)), (x, torch.zeros(96).expand(4, 96))):
        with pytest.raises(ValueError, match="device"):   # (x comes first, and is on the host)
            ctx.linear(op, *a)
    Hq, Hkv, D, B, M = 4, 2, 64, 2, 3
    W = (Hq + 2 * Hkv) * D
    rest = dict(pos=torch.zeros(B, M, dtype=torch.int32), sections=(D // 2,), rope_theta=1e4, q_out=bf(B, M, Hq, D),
                k_out=bf(B, Hkv, 8, D), v_out=bf(B, Hkv, 8, D))
    for qkv in (bf(W).expand(B * M, W), bf(W).expand(B, M, W), bf(B * M * W).as_strided((B, M, W), (M * 8, 8, 1))):
        with pytest.raises(ValueError, match="rows overlap"):
            ctx.rope_qkv(B, M, qkv, **rest)
    with pytest.raises(ValueError, match="evenly"):
        ctx.rope_qkv(B, M, bf(1, M, W).expand(B, M, W), **rest)
    with pytest.raises(ValueError, match="device"):
        ctx.rope_qkv(B, M, bf(B, M, W), **rest)


@pytest.mark.parametrize("axes,shapes,bad", [
    (1, ((2, 3, 1), (2, 3), (6, 1), (6,), (3, 3), (5, 3, 1)), ((2, 4, 1), (2, 4), (7,), (7, 1), (3, 2), (2, 1, 3), (1, 6), (8,), (2, 2), (2, 3, 2))),
    (2, ((2, 3, 2), (6, 2), (3, 3, 2)), ((2, 4, 2), (7, 2), (2, 6), (2, 3), (12,), (14,), (2, 3, 3), (2, 2, 3), (3, 2, 2), (1, 2, 3, 2)))])
def test_binding_takes_positions_of_the_call_s_shape(lib, axes, shapes, bad):
    """Positions of more tokens than the call's are refused: read on as if dense, only the first sequence's would be right.
    Those of more sequences are read as they lie.
    (Tensors on the host: those of a right shape are refused for their device.)"""
    ctx = make_ctx()
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    B, M, sections = 2, 3, (32,) if axes == 1 else (8, 24)
    for group, match in ((shapes, "device"), (bad, "pos: expected a tensor")):
        for s in group:
            with pytest.raises(ValueError, match=match):
                ctx.rope_qkv(B, M, bf(B, M, 8 * 64), torch.zeros(s, dtype=torch.int32), sections, 1e4, bf(B, M, 4, 64),
                             bf(B, 2, 8, 64), bf(B, 2, 8, 64))


def rope_code(lib, ctx, a):
    s = a["sections"]
    return lib.jk_rope_qkv(ctx._h, None, a["batch"], a["n"], a["qkv"], a["stride"], a["pos"], len(s), (C.c_int32 * len(s))(*s),
                           a["theta"], a["q"], a["k"], a["v"], a["sb"], a["sh"], a["rows"], a["first"])


@pytest.mark.parametrize("change,code", [
    (dict(v=K + 16), "SHAPE"), (dict(v=K + 128), "SHAPE"), (dict(v=K - 128), "SHAPE"), (dict(v=K + 1280), "SHAPE"),
    (dict(v=K + 5120 - 16), "SHAPE"), (dict(v=K + 5120), "WORKSPACE"), (dict(v=K - 5120), "WORKSPACE"),
    # heads of K and V in turn: [batch, Hkv, 2, rows, d], [batch, 2, Hkv, rows, d], [2, Hkv, batch, rows, d]
    (dict(sh=1280, sb=2560, v=K + 1280), "WORKSPACE"), (dict(sh=1280, sb=2560, v=K + 1280 - 16), "SHAPE"),
    (dict(sh=1280, sb=2560, v=K + 1280 + 16), "SHAPE"), (dict(sh=640, sb=2560, v=K + 2560), "WORKSPACE"),
    (dict(sh=640, sb=2560, v=K + 1280), "SHAPE"), (dict(sb=640, sh=1280, v=K + 5120), "WORKSPACE"), (dict(sb=640, sh=1280, v=K + 2560), "SHAPE"),
    # rows of one buffer: the first ten are K's, the next V's
    (dict(sh=1280, sb=2560, v=K + 10 * 128), "WORKSPACE"), (dict(sh=1280, sb=2560, v=K + 9 * 128), "SHAPE"),
    (dict(batch=1, sb=0, v=K + 640), "SHAPE"), (dict(batch=1, sb=0, v=K + 2560), "WORKSPACE")])
def test_rope_refuses_k_and_v_that_meet(lib, change, code):
    assert rope_code(lib, make_ctx(), {**ROPE, **change}) == E[code]


def test_rope_k_and_v_against_every_pair_of_pieces(lib):
    """Random layouts of 2 heads and up to 5 sequences, with both nestings: what is refused is what shares a byte."""
    rng, ctx, seen = random.Random(5), make_ctx(), set()
    for _ in range(4000):
        B, rows, es, d, Hkv = rng.randint(1, 5), rng.randint(3, 6), 2, 64, 2
        part, gap = rows * d, lambda: 8 * rng.choice([0, 0, 1, rows * d // 8, rng.randint(0, 200)])
        if rng.random() < 0.5:
            sh = part + gap()
            sb = sh + part + gap()
        else:
            sb = part + gap()
            sh = (B - 1) * sb + part + gap()
        off = 16 * rng.choice([rng.randint(-60, 60), rng.randint(-800, 800), rng.choice([-1, 1]) * sb * es // 16, sh * es // 16,
                               part * es // 16 + rng.randint(-2, 2)])
        at = [(b * sb + h * sh) * es for b in range(B) for h in range(Hkv)]
        meet = any(abs(off + v - k) < part * es for v in at for k in at)
        code = rope_code(lib, ctx, {**ROPE, "batch": B, "rows": rows, "sb": sb, "sh": sh, "v": K + off})
        assert code == E["SHAPE" if meet else "WORKSPACE"], (B, rows, sb, sh, off)
        seen.add((meet, sb > sh))
    assert len(seen) == 4


@pytest.mark.parametrize("change,code", [(dict(sh=64), "WORKSPACE"), (dict(sh=0), "WORKSPACE"), (dict(sh=-4, sb=640), "WORKSPACE"),
                                         (dict(sh=64, sb=632), "SHAPE"), (dict(batch=1, sb=-1, sh=3), "WORKSPACE"), (dict(sh=64, v=K + 128), "SHAPE")])
def test_rope_takes_any_stride_of_a_dimension_of_one(lib, change, code):
    ctx = jk.Context(hidden=8, n_experts=1, top_k=1, inter=8, vocab=8, n_q_heads=4, n_kv_heads=1, head_dim=64, max_batch=1,
                     max_tree=1, max_depth=1, max_frontier=1, k_per_expert=1, dtype="bf16", allocate=False)
    assert rope_code(lib, ctx, {**ROPE, **change}) == E[code]


def test_library_loads_without_the_extension(lib, monkeypatch, tmp_path):
    """Only the target layer's four calls need it: without it, or with one that does not load, the rest is there and they
    say what is missing."""
    monkeypatch.setattr(jk, "_lib", None)
    monkeypatch.setattr(jk, "_calls", None)
    monkeypatch.setattr(jk, "CALLS_PATH", str(tmp_path / "none.so"))
    assert jk.lib().jk_row_scale_bytes(1, 32) == 512
    ctx, x = make_ctx(), torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(RuntimeError, match="none.so is missing"):
        ctx.add_norm(x, out=x)
    monkeypatch.undo()
    with pytest.raises(ValueError):                        # (the extension is there again, and refuses host tensors)
        ctx.add_norm(x, out=x)


def test_extension_that_does_not_load_is_named(lib, monkeypatch):
    import paper_2502_06282_b200 as package
    monkeypatch.setattr(jk, "_calls", None)
    monkeypatch.delattr(package, "_calls", raising=False)
    monkeypatch.setitem(sys.modules, "paper_2502_06282_b200._calls", None)
    with pytest.raises(RuntimeError, match="_calls.so does not load"):
        make_ctx().quantize_mx8(None, None)


def test_extension_is_built_again_for_another_torch(lib, monkeypatch):
    from paper_2502_06282_b200 import build
    assert not build.needs_build()
    monkeypatch.setattr(build, "_built_for", lambda: "another\n")
    assert build.needs_build() and build.calls_need_build() and not build.library_needs_build()
