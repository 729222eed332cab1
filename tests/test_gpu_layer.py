"""A target layer's steps around its attention against their 64-bit definitions: norm with the residual's addition and
8-bit rows, matrix products with their epilogue, rotary positions; and the whole layer.

Tolerances count roundings.  A value stored in a type is off by at most half a step (f32 2^-24, bf16 2^-8, e4m3
2^-4 relative, 2^-10 scales at the bottom of its grid).  A sum of K products in f32 is off by at most K steps of 2^-23
of the sum of their magnitudes (every addition may round, and a tensor core may cut instead of rounding)."""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as lo
from paper_2502_06282_b200 import binding as jk
from paper_2502_06282_b200 import synth
from tests.jk_testutil import Guard, dev, host

pytestmark = pytest.mark.gpu

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
TD = {"f32": torch.float32, "bf16": torch.bfloat16}


def make_ctx(dtype, Hq=1, Hkv=1, d=64, hidden=8, eps=1e-5, **kw):
    kw = {**dict(max_batch=1, max_tree=1), **kw}
    return jk.Context(hidden=hidden, n_experts=1, top_k=1, inter=8, vocab=8, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d,
                      max_depth=1, max_frontier=1, k_per_expert=1, dtype=dtype, rms_eps=eps, **kw)


def store(a, dtype):
    return synth.store_round(np.asarray(a, dtype=np.float32), dtype).astype(np.float64)


def to_dev(a, dtype):
    return dev(np.asarray(a, dtype=np.float32)).to(TD[dtype])


def mx8_guard(g, R, n):
    n_b = jk.lib().jk_row_scale_bytes(R, n)
    return jk.Mx8(g.alloc((R, n), torch.uint8), g.alloc((n_b,), torch.uint8))


def mx8_of(codes, e):
    """An array of the library's layout from the model's codes and exponents; bytes of no row or block are 0xFF."""
    R, n = codes.shape
    c = dev(codes.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8)
    s = np.full(jk.lib().jk_row_scale_bytes(R, n), 255, dtype=np.uint8)
    s[lo.tile_index(R, n).reshape(-1)] = (e + 127).reshape(-1).astype(np.uint8)
    return jk.Mx8(c.contiguous(), dev(s))


def read_mx8(m):
    """(codes' values, exponents) of a device array; the bytes that belong to no row or block are untouched."""
    R, n = m.shape
    codes = m.codes.view(torch.float8_e4m3fn).float().cpu().numpy().astype(np.float64)
    raw = m.scales.cpu().numpy()
    at = lo.tile_index(R, n)
    rest = np.ones(raw.size, bool)
    rest[at.reshape(-1)] = False
    assert np.all(raw[rest] == Guard.POISON), "a scale byte that belongs to no block was written"
    return codes, raw[at].astype(np.int64) - 127


def check_mx8(m, y, err):
    """y the exact rows, err what the f32 values may be off by: the scale is that of a value within err, the codes are
    off by half a step of the grid."""
    codes, e = read_mx8(m)
    fine = np.isfinite(y)
    mag = np.where(fine, np.abs(y), 0.0)
    low = lo.scale_exponents(np.maximum(mag - np.where(fine, err, 0), 0.0))
    high = lo.scale_exponents(mag + np.where(fine, err, 0))
    assert np.all((e >= low) & (e <= high))
    got, s = lo.dequantize(codes, e), np.repeat(np.exp2(e.astype(np.float64)), 32, axis=1)
    assert np.array_equal(np.isnan(got), np.isnan(y))
    inf = np.isinf(y)
    assert np.all(codes[inf] == np.sign(y[inf]) * 448.0)
    off = np.abs(got - np.where(fine, y, 0.0))
    assert np.all(off[fine] <= (2.0 ** -4 * (np.abs(y) + err) + 2.0 ** -10 * s + err)[fine])


def check_t(t, y, err, dtype):
    got = host(t).astype(np.float64)
    fine = np.isfinite(y)
    assert np.array_equal(np.isnan(got), np.isnan(y)) and np.array_equal(got[np.isinf(y)], y[np.isinf(y)])
    bound = HALF[dtype] * (np.abs(np.where(fine, y, 0.0)) + err) + err + 2.0 ** -133
    off = np.abs(got - y)
    assert np.all(off[fine] <= bound[fine]), float(np.max((off / bound)[fine]))


# ------------------------------------------------------------------------------------------ norm
def run_norm(dtype, R, n, add=True, weight=True, outs=("sum", "out", "mx8"), eps=1e-5, x=None, seed=0):
    rng = np.random.default_rng(seed + R * 7 + n)
    ctx, g = make_ctx(dtype, eps=eps), Guard()
    x = store(rng.standard_normal((R, n)) * np.exp(rng.standard_normal((R, 1))) if x is None else x, dtype)
    delta = store(rng.standard_normal((R, n)), dtype) if add else None
    w = store(1 + 0.2 * rng.standard_normal(n), dtype) if weight else None
    o_sum = g.alloc((R, n), TD[dtype]) if "sum" in outs else None
    o = g.alloc((R, n), TD[dtype]) if "out" in outs else None
    m = mx8_guard(g, R, n) if "mx8" in outs else None
    ctx.add_norm(to_dev(x, dtype), None if w is None else to_dev(w, dtype), None if delta is None else to_dev(delta, dtype),
                 o_sum, o, m)
    g.check()
    with np.errstate(invalid="ignore", over="ignore"):
        s, y = lo.add_norm(x, delta, w, float(np.float32(eps)))
    # s: one rounding.  The sum of squares: 8 + 4 + 5 + 5 + 2 steps in a row and a half step for each s, halved by the
    # root; root, quotient and two products four half steps
    rel = (24 + 2 + 4) * 2.0 ** -24
    err = np.where(np.isfinite(y), np.abs(y) * rel, 0.0)
    if delta is not None:
        err = err + np.where(np.isfinite(s), np.abs(s), 0) * 2.0 ** -24 * np.where(np.isfinite(y / s), np.abs(y / s), 0)
    if o_sum is not None:
        check_t(o_sum, s, np.where(np.isfinite(s), np.abs(s) * 2.0 ** -24, 0), dtype)
    if o is not None:
        check_t(o, y, err, dtype)
    if m is not None:
        check_mx8(m, y, err)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,n", [(1, 32), (3, 96), (129, 512), (2, 4096), (5, 5120), (300, 8192), (2, 16416), (3, 32768)])
def test_norm(R, n, dtype):
    run_norm(dtype, R, n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [8, 24, 1000, 4104])
def test_norm_widths_without_blocks(n, dtype):
    run_norm(dtype, 5, n, outs=("sum", "out"))


@pytest.mark.parametrize("add,weight,outs", [(False, True, ("out",)), (False, False, ("mx8",)), (True, False, ("sum",)),
                                             (True, True, ("sum", "mx8")), (False, True, ("sum", "out"))])
def test_norm_forms(add, weight, outs):
    run_norm("bf16", 7, 256, add, weight, outs, eps=0.5)


def test_norm_of_zeros_infinities_and_nan():
    x = np.random.default_rng(1).standard_normal((6, 128))
    x[0] = 0.0
    x[1, 5] = np.nan
    x[2, 7] = np.inf
    x[3] *= 1e-30
    x[4, :64] = 0.0
    run_norm("bf16", 6, 128, add=False, x=x)


def test_norm_in_place():
    rng = np.random.default_rng(4)
    ctx = make_ctx("bf16")
    x, d, w = (to_dev(rng.standard_normal(s), "bf16") for s in ((33, 512), (33, 512), (512,)))
    s, o = torch.empty_like(x), torch.empty_like(x)
    ctx.add_norm(x, w, d, s, o)
    x2, d2 = x.clone(), d.clone()
    ctx.add_norm(x2, w, d2, x2, d2)
    assert torch.equal(x2, s) and torch.equal(d2, o)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,n,wide", [(1, 32, 0), (130, 160, 8), (257, 1376, 0), (3, 28672, 64)])
def test_quantize(R, n, wide, dtype):
    """Exact: a scale is a power of two, a value is rounded once."""
    rng = np.random.default_rng(n)
    x = rng.standard_normal((R, n)) * np.exp2(rng.integers(-60, 40, (R, n // 32)).repeat(32, 1).astype(np.float64))
    x[0, :32] = 0.0
    x[-1, 3], x[-1, 4], x[-1, 5] = np.inf, -np.inf, np.nan
    x[0, -32:] = 448.0 * 2.0 ** rng.integers(-3, 3)      # on the border of a scale
    x = store(x, dtype)
    room = torch.full((R, n + wide), float("nan"), dtype=TD[dtype], device="cuda")
    room[:, :n] = to_dev(x, dtype)
    g, ctx = Guard(), make_ctx(dtype)
    m = mx8_guard(g, R, n)
    ctx.quantize_mx8(room[:, :n], m)
    g.check()
    codes, e = read_mx8(m)
    want, we = lo.quantize(x)
    assert np.array_equal(e, we)
    assert np.array_equal(codes, want, equal_nan=True)


# ------------------------------------------------------------------------------------------ product
def operands(rng, R, N, K, kind, dtype):
    """x, w as f64 values and as device arrays."""
    x = rng.standard_normal((R, K)) * np.exp(0.5 * rng.standard_normal((1, K)))
    w = 0.1 * rng.standard_normal((N, K))
    if kind == "mx8":
        (xc, xe), (wc, we) = lo.quantize(x), lo.quantize(w)
        return lo.dequantize(xc, xe), lo.dequantize(wc, we), mx8_of(xc, xe), mx8_of(wc, we)
    x, w = store(x, dtype), store(w, dtype)
    return x, w, to_dev(x, dtype), to_dev(w, dtype)


def run_linear(R, N, K, kind="T", dtype="bf16", gated=False, act="none", bias=False, residual=False, out="T", wide=0,
               in_place=False, seed=0, tensor=True):
    rng = np.random.default_rng(seed + R + 3 * N + 5 * K)
    ctx, g = make_ctx(dtype), Guard()
    ctx.set_tensor_path(tensor)
    x, w, xd, wd = operands(rng, R, N, K, kind, dtype)
    wu = bu = wud = None
    if gated:
        _, wu, _, wud = operands(rng, 1, N, K, kind, dtype)
    b = store(rng.standard_normal(N), dtype) if bias else None
    bu = store(rng.standard_normal(N), dtype) if bias and gated else None
    res = store(3 * rng.standard_normal((R, N)), dtype) if residual else None
    if wide and kind == "T":
        room = torch.full((R, K + wide), float("nan"), dtype=TD[dtype], device="cuda")
        room[:, :K] = xd
        xd = room[:, :K]
    dv = lambda a: None if a is None else to_dev(a, dtype)
    op = jk.Linear(ctx, wd, bias=dv(b), act=act, w_up=wud, bias_up=dv(bu))
    rd = dv(res)
    if out == "mx8":
        od = mx8_guard(g, R, N)
    else:
        room = g.alloc((R, N + wide), torch.float32 if out == "f32" else TD[dtype])
        od = room[:, :N]
        if in_place:
            od.copy_(rd)
            rd = od
    ctx.linear(op, xd, od, residual=rd)
    g.check()
    assert ctx.read_status() == 0
    if wide and out != "mx8":
        assert bool((room[:, N:].contiguous().view(torch.uint8) == Guard.POISON).all()), "wrote between the rows"
    y = lo.linear(x, w, b, act, wu, bu, res)
    ax = np.abs(x)
    ez = (K + 4) * 2.0 ** -23 * (ax @ np.abs(w).T + (0 if b is None else np.abs(b)))
    z = lo.linear(x, w, b)
    a = lo.act(z, act)
    # SiLU and GELU have slopes below 1.13.  What the functions themselves are off by, relative: a few units of f32 and the
    # rounding of an exponent of up to 2^5, 2^-18; GELU in outputs of 16 or 8 bits another 7.6e-6 (the fit): 2^-16
    own = 2.0 ** -16 if act == "gelu" and out != "f32" and dtype != "f32" else 2.0 ** -18
    e = 1.13 * ez + (own * (np.abs(a) + 2.0 ** -20) if act != "none" else 0.0)
    if gated:
        u = lo.linear(x, wu, bu)
        eu = (K + 4) * 2.0 ** -23 * (ax @ np.abs(wu).T + (0 if bu is None else np.abs(bu)))
        e = e * np.abs(u) + np.abs(a) * eu + e * eu + 2.0 ** -23 * np.abs(a * u)
    e = e + 2.0 ** -23 * (np.abs(y) + (0 if res is None else np.abs(res)))
    if out == "mx8":
        check_mx8(od, y, e)
    else:
        check_t(od, y, e, "f32" if out == "f32" else dtype)
    return od


ROWS = [1, 2, 15, 16, 17, 60, 127, 128, 129, 240, 256, 257, 480, 513]


@pytest.mark.parametrize("kind", ["T", "mx8"])
@pytest.mark.parametrize("R", ROWS)
def test_linear_rows(R, kind):
    run_linear(R, 160, 416, kind, residual=True)


@pytest.mark.parametrize("kind", ["T", "mx8"])
@pytest.mark.parametrize("R", [1, 17, 60, 129, 257, 513])
def test_gated_rows(R, kind):
    run_linear(R, 160, 416, kind, gated=True, act="silu", out="mx8")


@pytest.mark.parametrize("kind", ["T", "mx8"])
@pytest.mark.parametrize("N", [1, 7, 32, 127, 128, 129, 255, 1000, 2053])
def test_linear_outputs(N, kind):
    run_linear(60, N, 256, kind, bias=True, residual=True, act="gelu")
    run_linear(3, N, 256, kind, gated=True, bias=True, act="silu")


@pytest.mark.parametrize("kind,K", [("T", 8), ("T", 24), ("T", 72), ("T", 1376), ("T", 5000), ("T", 14336),
                                    ("mx8", 32), ("mx8", 96), ("mx8", 160), ("mx8", 1376), ("mx8", 14336)])
def test_linear_inner(kind, K):
    run_linear(33, 200, K, kind, residual=True)
    run_linear(5, 96, K, kind, gated=True, act="silu", out="mx8")


@pytest.mark.parametrize("kind", ["T", "mx8"])
@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("out", ["T", "f32", "mx8"])
def test_linear_epilogues(kind, act, gated, out):
    run_linear(70, 288, 192, kind, gated=gated, act=act, bias=True, residual=True, out=out)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("kind", ["T", "mx8"])
def test_linear_many_tiles(kind, gated):
    """More tiles than SMs, and tiles whose sum is split."""
    run_linear(300, 5000 if not gated else 4992, 640, kind, gated=gated, act="silu", out="mx8" if gated else "T")
    run_linear(31, 4096, 2048, kind, gated=gated, bias=True, residual=True)


@pytest.mark.parametrize("R,N", [(1, 97), (60, 130), (300, 97)])
def test_linear_strides(R, N):
    run_linear(R, N, 136, wide=24, residual=True)
    run_linear(R, N, 136, wide=8, residual=True, in_place=True)
    run_linear(R, N, 136, wide=8, residual=True, out="f32")


@pytest.mark.parametrize("out,N", [("T", 288), ("T", 290), ("T", 292), ("f32", 288), ("f32", 290), ("mx8", 288)])
def test_linear_many_rows_beside_aligned_rows(out, N):
    """Residuals and outputs of many rows whose rows begin at multiples of 16 bytes, or not, or one of the two."""
    rng = np.random.default_rng(11)
    R, K = 300, 200
    ctx = make_ctx("bf16")
    x, w, xd, wd = operands(rng, R, N, K, "T", "bf16")
    op = jk.Linear(ctx, wd, act="silu")
    res = store(rng.standard_normal((R, N)), "bf16")
    y = lo.linear(x, w, None, "silu", residual=res)
    e = 1.13 * (K + 4) * 2.0 ** -23 * (np.abs(x) @ np.abs(w).T) + 2.0 ** -18 * np.abs(y - res) + 2.0 ** -23 * (np.abs(y) + np.abs(res))
    for wide_r in (0, 8, 6, 3):
        room = torch.zeros(R, N + wide_r, dtype=torch.bfloat16, device="cuda")
        room[:, :N] = to_dev(res, "bf16")
        for wide_o in (0, 8, 6, 4, 5) if out != "mx8" else (0,):
            g = Guard()
            if out == "mx8":
                od = mx8_guard(g, R, N)
            else:
                od = g.alloc((R, N + wide_o), torch.float32 if out == "f32" else torch.bfloat16)[:, :N]
            ctx.linear(op, xd, od, residual=room[:, :N])
            g.check()
            if out == "mx8":
                check_mx8(od, y, e)
            else:
                check_t(od, y, e, "f32" if out == "f32" else "bf16")
                beside = g.regions[0][0][Guard.PAD:Guard.PAD + g.regions[0][1]].view(od.dtype).view(R, N + wide_o)[:, N:]
                assert bool((beside.contiguous().view(torch.uint8) == Guard.POISON).all()), "wrote between the rows"
    assert ctx.read_status() == 0


@pytest.mark.parametrize("gated,act,out", [(False, "none", "T"), (True, "silu", "T"), (False, "gelu", "mx8"),
                                           (True, "none", "mx8")])
@pytest.mark.parametrize("R,N,K", [(1, 32, 8), (16, 1376, 512), (17, 160, 2048), (33, 96, 1000), (130, 64, 40), (300, 640, 200),
                                   (500, 5024, 72)])
def test_linear_f32(R, N, K, gated, act, out):
    run_linear(R, N, K, dtype="f32", gated=gated, act=act, bias=True, residual=True, out=out, wide=4 if R < 20 else 0)


@pytest.mark.parametrize("dtype,tensor", [("f32", True), ("bf16", False)])
@pytest.mark.parametrize("kind", ["T", "mx8"])
def test_linear_cuda_cores(kind, dtype, tensor):
    run_linear(37, 160, 352, kind, dtype=dtype, gated=True, act="silu", out="T", bias=True, tensor=tensor)
    run_linear(37, 160, 352, kind, dtype=dtype, out="mx8", residual=True, tensor=tensor)


# blocks of 128 rows; of 64, alone and shared by 2, 4 and 8; warps of one and two outputs
@pytest.mark.parametrize("R,N,K,gated", [(1024, 1300, 256, False), (640, 640, 192, True), (1200, 2000, 520, True), (256, 4096, 1024, False),
                                         (100, 4101, 1032, False), (64, 512, 2048, True), (1, 2373, 136, False), (16, 4097, 264, False),
                                         (9, 1190, 1000, False), (5, 4099, 72, True)])
def test_linear_f32_deals(R, N, K, gated):
    """Against torch's product in 64 bits; sums of 32 products, then of those sums, within the bound of K + 4 roundings."""
    g = torch.Generator(device="cuda").manual_seed(R + N)
    ctx = make_ctx("f32")
    x, w, u, res = (torch.randn(s, generator=g, device="cuda") for s in ((R, K), (N, K), (N, K), (R, N)))
    op = jk.Linear(ctx, w, w_up=u if gated else None)
    outs = [torch.full((R, N), float("nan"), device="cuda") for _ in range(2)]
    for o in outs:
        ctx.linear(op, x, o, residual=res)
    assert ctx.read_status() == 0 and torch.equal(*outs)
    z = x.double() @ w.double().T
    e = (K + 4) * 2.0 ** -24 * (x.abs().double() @ w.abs().double().T)
    if gated:
        zu = x.double() @ u.double().T
        eu = (K + 4) * 2.0 ** -24 * (x.abs().double() @ u.abs().double().T)
        z, e = z * zu, e * zu.abs() + z.abs() * eu + e * eu + 2.0 ** -24 * (z * zu).abs()
    y = z + res.double()
    assert bool(((outs[0].double() - y).abs() <= e + 2.0 ** -23 * (y.abs() + e)).all())


def torch_mx8(x):
    """x [rows, n] f32 on the device -> (Mx8, the values it stands for), the exponent by frexp."""
    R, n = x.shape
    b = x.view(R, n // 32, 32)
    m, e = torch.frexp(b.abs().amax(2))
    e = torch.where(m > 0.875, e - 8, e - 9).clamp(min=-32)
    codes = (b * torch.exp2(-e.float())[..., None]).view(R, n).to(torch.float8_e4m3fn)
    full = torch.full((-(-R // 128) * 128, -(-n // 128) * 4), 255, dtype=torch.uint8, device="cuda")
    full[:R, :n // 32] = (e + 127).to(torch.uint8)
    tiles = full.view(-1, 4, 32, full.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).reshape(-1).contiguous()
    return jk.Mx8(codes.view(torch.uint8), tiles), (codes.double().view(R, n // 32, 32) * torch.exp2(e.double())[..., None]).view(R, n)


# Shapes that take each way a call can go: clusters of 8, 4 and 2 CTAs; even shares whose tiles span CTAs (with partials that
# come in several rounds); more tiles than SMs; many rows with whole tiles, with tiles cut among 2, 3 and 4 pairs, alone and before
# whole turns; widths that end inside a tile
@pytest.mark.parametrize("kind", ["T", "mx8"])
@pytest.mark.parametrize("R,N,K,gated", [
    (60, 640, 4096, False), (60, 4096, 4096, False), (17, 5120, 4096, False), (128, 1376, 4096, True), (60, 2048, 4096, True),
    (128, 11008, 8192, False), (250, 9000, 4096, False), (128, 11008, 2048, True), (1, 32000, 1024, False), (5, 20001, 512, True),
    (300, 2048, 8192, False), (300, 1300, 4096, True), (2047, 5120, 1024, False), (1500, 2500, 4096, True), (700, 5119, 2048, False),
    (257, 9000, 8192, False), (4099, 384, 256, True), (320, 4096, 1024, False), (500, 1000, 4096, False), (700, 640, 2048, False),
    (1500, 300, 1024, False), (300, 640, 1024, True), (513, 200, 4096, True), (260, 1376, 8192, False), (385, 128, 96, False),
    (1100, 2000, 8192, False), (256, 5120, 13824, False), (1100, 1200, 8192, True), (480, 4864, 4096, True)])
def test_linear_every_deal(R, N, K, gated, kind):
    """Against torch's product in 64 bits, twice for the same bits."""
    g = torch.Generator(device="cuda").manual_seed(R + N + K)
    ctx = make_ctx("bf16")
    make = lambda r, s: torch.randn(r, K, generator=g, device="cuda") * s
    pack = torch_mx8 if kind == "mx8" else (lambda x: (x.bfloat16(), x.bfloat16().double()))
    (xd, x), (wd, w) = pack(make(R, 1.0)), pack(make(N, 0.05))
    (ud, u) = pack(make(N, 0.05)) if gated else (None, None)
    res = torch.randn(R, N, generator=g, device="cuda").bfloat16()
    op = jk.Linear(ctx, wd, act="silu" if gated else "none", w_up=ud)
    outs = [torch.full((R, N), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for o in outs:
        ctx.linear(op, xd, o, residual=res)
    assert ctx.read_status() == 0
    assert torch.equal(*outs)
    z = x @ w.T
    ez = (K + 4) * 2.0 ** -23 * (x.abs() @ w.abs().T)
    if gated:
        a, zu = z * torch.sigmoid(z), x @ u.T
        eu = (K + 4) * 2.0 ** -23 * (x.abs() @ u.abs().T)
        y, e = a * zu, (1.13 * ez + 2.0 ** -18 * (a.abs() + 2.0 ** -20)) * zu.abs() + a.abs() * eu + 1.13 * ez * eu
    else:
        y, e = z, ez
    y = y + res.double()
    e = e + 2.0 ** -23 * (y.abs() + res.double().abs())
    off = (outs[0].double() - y).abs()
    assert bool((off <= HALF["bf16"] * (y.abs() + e) + e).all())


# Many rows: fewer tiles than pairs of SMs (1500 and 1100 rows), and more
@pytest.mark.parametrize("kind", ["T", "mx8"])
@pytest.mark.parametrize("R,N", [(1500, 2496), (2100, 4992)])
def test_linear_many_rows(R, N, kind):
    run_linear(R, N + 2, 96, kind, bias=True, residual=True, act="gelu", wide=8)
    run_linear(R, N, 96, kind, residual=True, wide=8, in_place=True)
    run_linear(R, N, 96, kind, residual=True, bias=True, out="f32", wide=8)
    run_linear(R, N, 96, kind, residual=True, bias=True, act="gelu", out="mx8")


@pytest.mark.parametrize("kind", ["T", "mx8"])
@pytest.mark.parametrize("R,N", [(1100, 1216), (1500, 2496)])
def test_gated_many_rows(R, N, kind):
    run_linear(R, N + 1, 96, kind, gated=True, bias=True, residual=True, act="silu", wide=8)
    run_linear(R, N, 96, kind, gated=True, bias=True, residual=True, act="silu", in_place=True)
    run_linear(R, N, 96, kind, gated=True, bias=True, act="gelu", out="f32")
    run_linear(R, N, 96, kind, gated=True, residual=True, act="silu", out="mx8")


@pytest.mark.parametrize("kind", ["T", "mx8"])
@pytest.mark.parametrize("R,N,K,gated", [(1100, 2016, 8192, False), (1100, 1216, 8192, True), (2047, 5120, 5120, False),
                                         (1100, 11008, 4096, True), (250, 4096, 4096, False), (120, 2048, 4096, True), (60, 512, 4096, False),
                                         (100, 11008, 4096, False)])
def test_linear_outputs_agree(R, N, K, gated, kind):
    """Tiles cut among CTAs: outputs in T and in 8 bits are those in f32, rounded; in place too."""
    g = torch.Generator(device="cuda").manual_seed(R + N + K)
    ctx = make_ctx("bf16")
    make = lambda r, s: torch.randn(r, K, generator=g, device="cuda") * s
    pack = torch_mx8 if kind == "mx8" else (lambda x: (x.bfloat16(), x.bfloat16().double()))
    (xd, x), (wd, w) = pack(make(R, 1.0)), pack(make(N, 0.05))
    (ud, u) = pack(make(N, 0.05)) if gated else (None, None)
    res, bias = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((R, N), (N,)))
    op = jk.Linear(ctx, wd, bias=bias, act="silu" if gated else "none", w_up=ud)
    y = torch.full((R, N), float("nan"), device="cuda")
    ctx.linear(op, xd, y, residual=res)
    z = x @ w.T + bias.double()
    ez = (K + 4) * 2.0 ** -23 * (x.abs() @ w.abs().T + bias.double().abs())
    if gated:
        a, zu = z * torch.sigmoid(z), x @ u.T
        eu = (K + 4) * 2.0 ** -23 * (x.abs() @ u.abs().T)
        z, ez = a * zu, (1.13 * ez + 2.0 ** -18 * (a.abs() + 2.0 ** -20)) * zu.abs() + a.abs() * eu + 1.13 * ez * eu + 2.0 ** -23 * (a * zu).abs()
    z = z + res.double()
    assert bool(((y.double() - z).abs() <= ez + 2.0 ** -23 * (z.abs() + res.double().abs())).all())
    t, place = torch.zeros(R, N, dtype=torch.bfloat16, device="cuda"), res.clone()
    ctx.linear(op, xd, t, residual=res)
    ctx.linear(op, xd, place, residual=place)
    assert torch.equal(t, y.bfloat16()) and torch.equal(place, t)
    m, (want, value) = jk.Mx8.empty(R, N), torch_mx8(y)
    ctx.linear(op, xd, m, residual=res)
    assert torch.equal(m.codes, want.codes)
    full = m.scales.view(-(-R // 128), -(-N // 128), 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-(-R // 128) * 128, -1)[:R, :N // 32]
    assert torch.equal(full.double(), torch.log2(value.abs().view(R, N // 32, 32).amax(2) / m.codes.view(torch.float8_e4m3fn).double().abs().view(
        R, N // 32, 32).amax(2)) + 127)
    assert ctx.read_status() == 0


def test_linear_two_contexts_at_once():
    """Two contexts on two streams, each with calls that hand sums over between CTAs, against the same calls alone."""
    rng = np.random.default_rng(12)
    shapes = [(60, 11008, 2048, "T"), (60, 1000, 4096, "mx8"), (300, 2048, 4096, "T"), (128, 9000, 4096, "mx8")]
    runs = []
    for c in range(2):
        ctx = make_ctx("bf16")
        for R, N, K, kind in shapes:
            g = torch.Generator(device="cuda").manual_seed(N + c)
            pack = torch_mx8 if kind == "mx8" else (lambda x: (x.bfloat16(), None))
            xd, wd = (pack(torch.randn(r, K, generator=g, device="cuda"))[0] for r in (R, N))
            op, out = jk.Linear(ctx, wd), torch.zeros(R, N, dtype=torch.bfloat16, device="cuda")
            ctx.linear(op, xd, out)
            torch.cuda.synchronize()
            runs.append((c, ctx, op, xd, out, out.clone()))
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for c, ctx, op, xd, out, _ in runs:
            with torch.cuda.stream(streams[c]):
                ctx.linear(op, xd, out)
    torch.cuda.synchronize()
    for c, ctx, op, xd, out, want in runs:
        assert torch.equal(out, want) and ctx.read_status() == 0


def test_rows_far_apart():
    """Offsets past 32 bits: rows 2^31 elements apart in x, residual and out; more than 2^32 elements in a norm."""
    R, N, K, far = 2, 136, 64, 1 << 31
    g = torch.Generator(device="cuda").manual_seed(3)
    ctx = make_ctx("bf16")
    x, w, res = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((R, K), (N, K), (R, N)))
    op, want = jk.Linear(ctx, w), torch.empty(R, N, dtype=torch.bfloat16, device="cuda")
    ctx.linear(op, x, want, residual=res)
    room = torch.empty(far + 4096, dtype=torch.bfloat16, device="cuda")
    at = lambda first, n: room[first:].as_strided((R, n), (far, 1), first)
    at(0, K).copy_(x)
    at(1024, N).copy_(res)
    ctx.linear(op, at(0, K), at(2048, N), residual=at(1024, N))
    assert torch.equal(at(2048, N), want)
    m, far_m = jk.Mx8.empty(R, K), jk.Mx8.empty(R, K)
    ctx.quantize_mx8(x, m)
    ctx.quantize_mx8(at(0, K), far_m)
    assert torch.equal(m.codes, far_m.codes)
    del room
    rows, n = (1 << 17) + 3, 32768
    big = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
    big[:2].normal_(generator=g)
    big[2:-2].zero_()
    big[-2:].normal_(generator=g)
    few = torch.cat([big[:2], big[-2:]])
    out, out8 = torch.empty_like(few), jk.Mx8.empty(4, n)
    ctx.add_norm(few, out=out, out_mx8=out8)
    codes = jk.Mx8.empty(rows, n)
    ctx.add_norm(big, out=big, out_mx8=codes)
    assert torch.equal(big[-2:], out[2:]) and torch.equal(big[:2], out[:2]) and not bool(big[rows // 2].any())
    assert torch.equal(codes.codes[-2:], out8.codes[2:])
    assert ctx.read_status() == 0


@pytest.mark.parametrize("kind", ["T", "mx8"])
def test_linear_nan_and_infinities_stay_in_their_row(kind):
    """A row of x with a NaN, and one with the type's largest value, reach no other row; padding reaches none."""
    rng = np.random.default_rng(5)
    R, N, K = 40, 96, 160
    x, w, _, wd = operands(rng, R, N, K, kind, "bf16")
    ctx = make_ctx("bf16")
    out = torch.empty(R, N, dtype=torch.bfloat16, device="cuda")

    def product(a):
        xd = mx8_of(*lo.quantize(a)) if kind == "mx8" else to_dev(a, "bf16")
        ctx.linear(jk.Linear(ctx, wd), xd, out)
        return host(out)

    want = product(x)
    y = x.copy()
    y[7, 3] = np.nan
    y[20, :] = 448.0 * 2.0 ** 100
    got = product(y)
    rest = [r for r in range(R) if r not in (7, 20)]
    assert np.array_equal(got[rest], want[rest])
    assert np.all(np.isnan(got[7]))


def test_linear_same_bits_every_time_replayed_and_on_another_stream():
    rng = np.random.default_rng(6)
    R, N, K = 60, 1000, 2048
    ctx = make_ctx("bf16")
    for kind in ("T", "mx8"):
        x, w, xd, wd = operands(rng, R, N, K, kind, "bf16")
        op = jk.Linear(ctx, wd)
        outs = [torch.empty(R, N, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
        ctx.linear(op, xd, outs[0])
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            ctx.linear(op, xd, outs[1])
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for _ in range(3):
                ctx.linear(op, xd, outs[2])
        for _ in range(4):
            outs[2].zero_()
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    assert ctx.read_status() == 0


def test_linear_chain_without_waiting():
    """Calls in a row on one stream, each reading what the one before wrote, against the same calls one by one."""
    rng = np.random.default_rng(7)
    R, H, I = 48, 256, 704
    ctx = make_ctx("bf16")
    up = jk.Linear(ctx, operands(rng, 1, I, H, "mx8", "bf16")[3], act="silu", w_up=operands(rng, 1, I, H, "mx8", "bf16")[3])
    down = jk.Linear(ctx, operands(rng, 1, H, I, "mx8", "bf16")[3])
    x0 = to_dev(rng.standard_normal((R, H)), "bf16")
    res = []
    for wait in (False, True):
        x, xn, h = x0.clone(), jk.Mx8.empty(R, H), jk.Mx8.empty(R, I)
        torch.cuda.synchronize()
        for _ in range(12):
            for call in (lambda: ctx.add_norm(x, out_mx8=xn), lambda: ctx.linear(up, xn, h),
                         lambda: ctx.linear(down, h, x, residual=x)):
                call()
                if wait:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        res.append(x)
    assert torch.equal(*res)


# ------------------------------------------------------------------------------------------ rotary positions
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,d", [(1, 1, 64), (8, 2, 128), (5, 5, 64), (40, 40, 128)])
@pytest.mark.parametrize("B,M,sections", [(1, 1, None), (3, 7, (0.25, 0.75)), (2, 61, (0.25, 0.375, 0.375)),
                                          (2, 5, (0.0, 0.5, 0.25, 0.25))])
def test_rope(B, M, sections, Hq, Hkv, d, dtype):
    rng = np.random.default_rng(B * 100 + M + Hq)
    half = d // 2
    sec = (half,) if sections is None else tuple(int(s * half) for s in sections)
    A, theta, wide = len(sec), (10000.0, 500000.0)[M % 2], 16 * (M % 3)
    ctx, g = make_ctx(dtype, Hq, Hkv, d), Guard()
    W = (Hq + 2 * Hkv) * d
    x = store(rng.standard_normal((B, M, W)), dtype)
    pos = rng.integers(0, 1 << 20, (B, M, A)).astype(np.int32)
    room = torch.full((B, M, W + wide), float("nan"), dtype=TD[dtype], device="cuda")
    room[..., :W] = to_dev(x, dtype)
    rows, first = M + 5, (np.arange(B) * 2 % 6).astype(np.int32)
    q = g.alloc((B, M, Hq, d), TD[dtype])
    k, v = (g.alloc((B, Hkv, rows, d), TD[dtype]) for _ in range(2))
    ctx.rope_qkv(B, M, room[..., :W], dev(pos if A > 1 else pos[..., 0]), sec, theta, q, k, v, first_row=dev(first))
    g.check()
    assert ctx.read_status() == 0
    wq, wk, wv = lo.rope(x, pos, sec, float(np.float32(theta)), Hq, Hkv, d)
    # angle: 64 bits (2^20 2^-53 at most), reduced to 32 (2^-24 of pi); sine and cosine 2 units; two products and a sum
    mag = np.abs(x).max()
    err = 2 * mag * (np.pi * 2.0 ** -24 + 2.0 ** -22 + 2.0 ** -23)
    check_t(q, wq, np.full(wq.shape, err), dtype)
    for b in range(B):
        r0 = int(first[b])
        check_t(k[b, :, r0:r0 + M], wk[b], np.full(wk[b].shape, err), dtype)
        assert np.array_equal(host(v[b, :, r0:r0 + M]), wv[b].astype(np.float32))
        for t in (k, v):
            other = torch.cat([t[b, :, :r0], t[b, :, r0 + M:]], 1).contiguous().view(torch.uint8)
            assert bool((other == Guard.POISON).all()), "rows beside the tokens' were written"


def test_rope_refuses_rows_and_positions_on_the_device():
    ctx = make_ctx("bf16", 2, 2, 64)
    qkv = torch.randn(2, 3, 6 * 64, device="cuda").bfloat16()
    pos = torch.ones(2, 3, dtype=torch.int32, device="cuda")
    for first, bad_pos, lost in (([0, 2], None, 1), ([-1, 0], None, 0), ([0, 0], (1, 2), None)):
        q = torch.full((2, 3, 2, 64), 7.0, device="cuda", dtype=torch.bfloat16)
        k, v = (torch.full((2, 2, 4, 64), 7.0, device="cuda", dtype=torch.bfloat16) for _ in range(2))
        p = pos.clone()
        if bad_pos:
            p[bad_pos] = -1
        ctx.rope_qkv(2, 3, qkv, p, (32,), 10000.0, q, k, v, first_row=torch.tensor(first, dtype=torch.int32, device="cuda"))
        assert ctx.read_status() == jk.ERR["BOUNDS"]
        if lost is not None:
            assert bool((k[lost] == 7).all()) and bool((v[lost] == 7).all())
            assert not bool((k[1 - lost] == 7).all())
        else:
            assert bool((k[1, :, 2] == 7).all()) and bool((v[1, :, 2] == 7).all()) and bool((q[1, 2] == 7).all())
            assert not bool((k[1, :, 1] == 7).any())
    ctx.rope_qkv(2, 3, qkv, pos, (32,), 10000.0, q, k, v)
    assert ctx.read_status() == 0


def test_rope_agrees_with_verify_qkv():
    """Projection by jk_linear and placing by jk_rope_qkv give what jk_verify_qkv gives, but for the projection's own
    rounding (qkv passes through T once: half a step of each of the two elements of a pair, and half a step at the end)."""
    rng = np.random.default_rng(9)
    B, M, Hq, Hkv, d, H = 2, 9, 4, 2, 64, 128
    ctx = make_ctx("bf16", Hq, Hkv, d, hidden=H, max_batch=B, max_tree=M)
    w = to_dev(0.1 * rng.standard_normal(((Hq + 2 * Hkv) * d, H)), "bf16")
    x = to_dev(rng.standard_normal((B, M, H)), "bf16")
    depth = dev(rng.integers(0, 5, (B, M)).astype(np.int32))
    kv_len = dev(np.array([3, 11], dtype=np.int32))
    new = lambda: [torch.zeros(s, device="cuda", dtype=torch.bfloat16) for s in ((B, M, Hq, d), (B, Hkv, 24, d), (B, Hkv, 24, d))]
    a, b = new(), new()
    ctx.verify_qkv(w, B, M, x, depth, *a, kv_len, 10000.0)
    qkv = torch.empty(B * M, w.shape[0], device="cuda", dtype=torch.bfloat16)
    ctx.linear(jk.Linear(ctx, w), x.view(B * M, H), qkv)
    ctx.rope_qkv(B, M, qkv, kv_len[:, None] + depth, (32,), 10000.0, *b, first_row=kv_len)
    assert ctx.read_status() == 0
    top = float(qkv.float().abs().max())
    for s, t in zip(a, b):
        assert float((s.float() - t.float()).abs().max()) <= 4 * 2.0 ** -8 * top


# ------------------------------------------------------------------------------------------ the whole layer
def exact_layer(x, p, parent, depth, kv_len, kc, vc, scale, Hq, Hkv, d, mx8, eps):
    """The layer in 64 bits; with mx8 its rows are quantised where the library's are."""
    q8 = (lambda a: lo.dequantize(*lo.quantize(a))) if mx8 else (lambda a: a)
    B, M = depth.shape
    _, xn = lo.add_norm(x, None, p["norm1"], eps)
    qkv = lo.linear(q8(xn), p["qkv"])
    q, k, v = lo.rope(qkv.reshape(B, M, -1), (kv_len[:, None] + depth)[..., None], (d // 2,), 10000.0, Hq, Hkv, d)
    att = np.empty((B, M, Hq, d))
    for b in range(B):
        n = int(kv_len[b])
        vis = np.zeros((M, n + M), bool)
        vis[:, :n] = True
        for i in range(M):
            j = i
            while j >= 0:
                vis[i, n + j] = True
                j = int(parent[b, j])
        for h in range(Hq):
            g = h // (Hq // Hkv)
            K = np.concatenate([kc[b, g, :n], k[b, g]])
            V = np.concatenate([vc[b, g, :n], v[b, g]])
            s = np.where(vis, q[b, :, h] @ K.T * scale, -np.inf)
            s = np.exp(s - s.max(1, keepdims=True))
            att[b, :, h] = (s / s.sum(1, keepdims=True)) @ V
    x = lo.linear(q8(att.reshape(B * M, -1)), p["o"], residual=x)
    _, xn = lo.add_norm(x, None, p["norm2"], eps)
    h = lo.linear(q8(xn), p["gate"], None, "silu", p["up"])
    return lo.linear(q8(h), p["down"], residual=x)


@pytest.mark.parametrize("mx8", [False, True])
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("dtype,B,M", [("bf16", 2, 13), ("bf16", 1, 1), ("bf16", 4, 60), ("f32", 2, 7)])
def test_target_layer(dtype, B, M, paged, mx8):
    """The calls as a pass makes them, twice in a row (two layers), eager and replayed from a graph."""
    rng = np.random.default_rng(B * M + mx8)
    H, I, Hq, Hkv, d, P = 256, 704, 4, 2, 64, 70
    ctx = make_ctx(dtype, Hq, Hkv, d, hidden=H, max_batch=B, max_tree=M)
    p = {"norm1": 1 + 0.1 * rng.standard_normal(H), "norm2": 1 + 0.1 * rng.standard_normal(H)}
    for n, s in (("qkv", ((Hq + 2 * Hkv) * d, H)), ("o", (H, Hq * d)), ("gate", (I, H)), ("up", (I, H)), ("down", (H, I))):
        p[n] = rng.standard_normal(s) / np.sqrt(s[1])
        p[n] = lo.dequantize(*lo.quantize(p[n])) if mx8 else store(p[n], dtype)
    p["norm1"], p["norm2"] = store(p["norm1"], dtype), store(p["norm2"], dtype)
    dv = (lambda a: mx8_of(*lo.quantize(a))) if mx8 else (lambda a: to_dev(a, dtype))
    layer = jk.TargetLayer(to_dev(p["norm1"], dtype), jk.Linear(ctx, dv(p["qkv"])), jk.Linear(ctx, dv(p["o"])),
                           to_dev(p["norm2"], dtype), jk.Linear(ctx, dv(p["gate"]), act="silu", w_up=dv(p["up"])),
                           jk.Linear(ctx, dv(p["down"])))
    bufs = jk.LayerBuffers(ctx, layer, B, M)
    x0 = store(rng.standard_normal((B * M, H)), dtype)
    kv_len = np.array([P - 3 * b for b in range(B)], dtype=np.int32)
    parent = np.array([[-1] + [int(rng.integers(0, i)) for i in range(1, M)] for _ in range(B)], dtype=np.int32)
    depth = np.zeros((B, M), dtype=np.int32)
    for i in range(1, M):
        depth[:, i] = depth[np.arange(B), parent[:, i]] + 1
    kc, vc = (store(rng.standard_normal((B, Hkv, P + M, d)), dtype) for _ in range(2))
    want = x0
    if paged:
        cache = jk.PagedCache(ctx, n_layers=1, n_pages=B * 6, page_size=16, max_seqs=B, max_pages=8)
        kd, vd = to_dev(kc, dtype), to_dev(vc, dtype)
        ptr = lambda t: torch.tensor([t.data_ptr()], dtype=torch.int64, device="cuda")
        ctx.paged_import(cache, B, dev(kv_len), 0, 1, ptr(kd), ptr(vd), kd.stride(0), kd.stride(1), P + M)
        ps, lens = 16, kv_len // 16 * 16
        for t in (kc, vc):                      # what the pages hold: one scale per page and head
            for b in range(B):
                for h in range(Hkv):
                    for a in range(0, int(lens[b]), ps):
                        blk = t[b, h, a:a + ps]
                        e = lo.scale_exponents(blk.reshape(1, -1)).max()
                        t[b, h, a:a + ps] = lo.e4m3(blk / 2.0 ** e) * 2.0 ** e
        lengths = cache.kv_len
        k, v = (torch.zeros(B, Hkv, M, d, dtype=TD[dtype], device="cuda") for _ in range(2))
    else:
        cache, lengths = None, dev(kv_len)
        k, v = to_dev(kc, dtype), to_dev(vc, dtype)
    for _ in range(2):
        want = exact_layer(want, p, parent, depth, kv_len, kc, vc, 0.125, Hq, Hkv, d, mx8, 1e-5)
    x = to_dev(x0, dtype)
    pd, dd = dev(parent), dev(depth)

    def run_pass():
        for _ in range(2):
            jk.run_target_layer(ctx, layer, bufs, B, M, x, pd, dd, 10000.0, 0.125, lengths, k, v, cache)

    run_pass()
    torch.cuda.synchronize()
    assert ctx.read_status() == 0
    got = host(x).astype(np.float64)
    # roundings to bf16 have an rms of 2^-8 / sqrt(3); about nine of them lie one behind the other in a layer, each of
    # at most the size of the stream: 2 * 9 * 0.00226 = 0.041 if all added up.  8-bit rows: a value that is off by
    # 2^-8 takes the next code in one of 2^-5 / 2^-8 = 8 cases, 2^-4 off: an rms of 0.022 at four places of each layer
    tol = {"f32": 1e-4, "bf16": 0.041}[dtype] + (2 * 4 * 0.022 if mx8 else 0.0)
    assert np.linalg.norm(got - want) <= tol * np.linalg.norm(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run_pass()
    for _ in range(2):
        x.copy_(to_dev(x0, dtype))
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(host(x).astype(np.float64), got)
    assert ctx.read_status() == 0


def test_binding_refuses_arrays_on_the_device():
    """Types, shapes and strides that the calls would read or write wrongly."""
    T, d = dict(dtype=torch.bfloat16, device="cuda"), dict(device="cuda")
    ctx = make_ctx("bf16", Hq=4, Hkv=2)
    x, w = torch.zeros(4, 64, **T), torch.zeros(96, 64, **T)
    m, op = jk.Mx8.empty(4, 64), jk.Linear(ctx, w)
    out = torch.zeros(4, 96, **T)

    def bad(call, *a, **kw):
        with pytest.raises(ValueError):
            call(*a, **kw)

    for kw in (dict(weight=torch.zeros(32, **T)), dict(weight=torch.zeros(1, 64, **T)), dict(delta=torch.zeros(4, 64, **d)),
               dict(delta=torch.zeros(4, 32, **T)), dict(out_sum=torch.zeros(2, 64, **T)), dict(out=torch.zeros(4, 128, **T)[:, ::2]),
               dict(out=torch.zeros(4, 128, **T)[:, :64]), dict(out=torch.zeros(4, 64, dtype=torch.bfloat16)), dict(out=[0]),
               dict(out_mx8=jk.Mx8.empty(4, 32)), dict(out_mx8=m.codes)):
        bad(ctx.add_norm, x, **{"out": torch.zeros_like(x), **kw})
    bad(ctx.add_norm, torch.zeros(4, 128, **T)[:, :64], out=x)
    bad(ctx.quantize_mx8, x.float(), m)
    bad(ctx.quantize_mx8, x[:2], m)
    bad(ctx.quantize_mx8, torch.zeros(64, 4, **T).T, m)
    bad(ctx.quantize_mx8, x, x)
    for a in ((x[:, :32], out), (x.float(), out), (m, out), (torch.zeros(64, 4, **T).T, out), (x, out[:2]), (x, out[:, :64]),
              (x, out.half()), (x, jk.Mx8.empty(4, 64)), (x, out, out[:2]), (x, out, out.float()), (x, torch.zeros(96, 4, **T).T),
              (x.cpu(), out), (None, out), (x, None), (x[0], out)):
        bad(ctx.linear, op, *a)
    bad(ctx.linear, jk.Linear(ctx, jk.Mx8.empty(96, 64)), x, out)
    bad(make_ctx("f32").linear, op, x, out)
    Hq, Hkv, D, B, M = ctx.cfg.n_q_heads, ctx.cfg.n_kv_heads, ctx.cfg.head_dim, 2, 3
    W = (Hq + 2 * Hkv) * D
    good = dict(batch=B, n_tokens=M, qkv=torch.zeros(B, M, W, **T), pos=torch.zeros(B, M, 1, dtype=torch.int32, **d), sections=(D // 2,),
                rope_theta=1e4, q_out=torch.zeros(B, M, Hq, D, **T), k_out=torch.zeros(B, Hkv, 8, D, **T),
                v_out=torch.zeros(B, Hkv, 8, D, **T), first_row=torch.zeros(B, dtype=torch.int32, **d))
    ctx.rope_qkv(**good)
    for kw in (dict(qkv=torch.zeros(B, M, W, **d)), dict(qkv=torch.zeros(B, M, W + D, **T)), dict(qkv=torch.zeros(B, M + 1, W, **T)),
               dict(qkv=torch.zeros(M, B, W, **T).transpose(0, 1)), dict(qkv=torch.zeros(B, 2 * M, W, **T)[:, :M]),
               dict(qkv=torch.zeros(M, B, 2 * W, **T)[:, :, :W]), dict(pos=torch.zeros(B, M, 2, dtype=torch.int32, **d)),
               dict(pos=torch.zeros(B, M, **d)), dict(pos=torch.zeros(B, 1, dtype=torch.int32, **d)), dict(sections=(1,) * 17),
               dict(q_out=torch.zeros(B, M, Hq, 2 * D, **T)[..., :D]), dict(q_out=torch.zeros(B, M, Hq, D, **d)),
               dict(k_out=torch.zeros(B, Hkv, 2, D, **T), v_out=torch.zeros(B, Hkv, 2, D, **T)), dict(k_out=torch.zeros(B, Hkv, 9, D, **T)),
               dict(k_out=torch.zeros(B, 8, Hkv, D, **T).transpose(1, 2)), dict(v_out=torch.zeros(B, Hkv, 8, D, **d)),
               dict(k_out=torch.zeros(1, Hkv, 8, D, **T), v_out=torch.zeros(1, Hkv, 8, D, **T)),
               dict(first_row=torch.zeros(B, dtype=torch.int64, **d)), dict(first_row=torch.zeros(1, dtype=torch.int32, **d)),
               dict(first_row=torch.zeros(B, dtype=torch.int32)), dict(batch=-1), dict(qkv=None)):
        bad(ctx.rope_qkv, **{**good, **kw})
    torch.cuda.synchronize()
    assert ctx.read_status() == 0


@pytest.mark.parametrize("R,N,K", [(60, 4096, 4096), (60, 11008, 2048), (700, 5120, 2048)])
def test_first_call_of_a_context_is_captured(R, N, K):
    """Nothing that a context finds out on its first call disturbs a capture; two graphs of it, replayed in turn."""
    g = torch.Generator(device="cuda").manual_seed(R)
    x, w = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((R, K), (N, K)))
    ctx = make_ctx("bf16")
    outs = [torch.zeros(R, N, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph, out in zip(graphs, outs):
        with torch.cuda.graph(graph):
            ctx.linear(jk.Linear(ctx, w), x, out)
    for _ in range(3):
        for graph, out in zip(graphs, outs):
            out.zero_()
            graph.replay()
    other = make_ctx("bf16")
    other.linear(jk.Linear(other, w), x, outs[2])
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[2])
    assert ctx.read_status() == 0


def test_binding_refuses_expanded_rows_on_the_device():
    """Arrays whose rows are one row in memory, as every operand; a single expanded row is an ordinary one."""
    T = dict(dtype=torch.bfloat16, device="cuda")
    ctx = make_ctx("bf16", Hq=4, Hkv=2)
    x, w, out, m = torch.randn(4, 64, **T), torch.randn(96, 64, **T), torch.zeros(4, 96, **T), jk.Mx8.empty(4, 64)
    op, one = jk.Linear(ctx, w), torch.randn(96, **T)
    for a in ((x[:1].expand(4, 64), out), (x[0].expand(4, 64), out), (x, one.expand(4, 96)), (x, one.float().expand(4, 96)),
              (x, out, one.expand(4, 96))):
        with pytest.raises(ValueError, match="rows overlap"):
            ctx.linear(op, *a)
    with pytest.raises(ValueError, match="rows overlap"):
        ctx.quantize_mx8(x[0].expand(4, 64), m)
    Hq, Hkv, D, B, M = 4, 2, 64, 2, 3
    W = (Hq + 2 * Hkv) * D
    new = lambda: [torch.zeros(s, **T) for s in ((B, M, Hq, D), (B, Hkv, 8, D), (B, Hkv, 8, D))]
    pos = torch.zeros(B, M, dtype=torch.int32, device="cuda")
    for qkv in (one.repeat(6)[:W].expand(B * M, W), one.repeat(6)[:W].expand(B, M, W)):
        with pytest.raises(ValueError, match="rows overlap"):
            ctx.rope_qkv(B, M, qkv, pos, (D // 2,), 1e4, *new())
    got = torch.zeros(1, 96, **T)
    ctx.linear(op, x[0].expand(1, 64), got, residual=one.expand(1, 96))
    ctx.linear(op, x, out, residual=one.repeat(4, 1))
    assert torch.equal(got[0], out[0]) and ctx.read_status() == 0


# More tiles than pairs of SMs, the last of the weights ending after 1 or 3 blocks of 32 outputs; few steps along k, so
# that a tile's stores follow the last one's closely
@pytest.mark.parametrize("kind", ["T", "mx8"])
@pytest.mark.parametrize("out", ["T", "mx8"])
@pytest.mark.parametrize("N,K,gated", [(1376, 128, False), (1312, 128, False), (1376, 512, False), (1184, 128, True), (1184, 384, True)])
def test_linear_many_rows_that_end_inside_a_tile(N, K, gated, out, kind):
    """No residual; outputs in T and in 8 bits are those in f32, rounded, over and over."""
    R = 4096
    g = torch.Generator(device="cuda").manual_seed(N + K)
    ctx = make_ctx("bf16")
    make = lambda r, s: torch.randn(r, K, generator=g, device="cuda") * s
    pack = torch_mx8 if kind == "mx8" else (lambda x: (x.bfloat16(), x.bfloat16().double()))
    (xd, x), (wd, w) = pack(make(R, 1.0)), pack(make(N, 0.05))
    (ud, u) = pack(make(N, 0.05)) if gated else (None, None)
    op = jk.Linear(ctx, wd, w_up=ud)
    y = torch.full((R, N), float("nan"), device="cuda")
    ctx.linear(op, xd, y)
    z, e = x @ w.T, (K + 4) * 2.0 ** -23 * (x.abs() @ w.abs().T)
    if gated:
        zu, eu = x @ u.T, (K + 4) * 2.0 ** -23 * (x.abs() @ u.abs().T)
        z, e = z * zu, e * zu.abs() + z.abs() * eu + e * eu + 2.0 ** -23 * (z * zu).abs()
    assert bool(((y.double() - z).abs() <= e + 2.0 ** -23 * z.abs()).all())
    want = torch_mx8(y)[0].codes if out == "mx8" else y.bfloat16()
    for _ in range(20):
        o = jk.Mx8.empty(R, N) if out == "mx8" else torch.zeros(R, N, dtype=torch.bfloat16, device="cuda")
        ctx.linear(op, xd, o)
        assert torch.equal(o.codes if out == "mx8" else o, want)
    assert ctx.read_status() == 0


@pytest.mark.parametrize("R,N,K,gated", [(64, 500, 2048, False), (64, 500, 2048, True), (33, 90, 1024, True), (50, 161, 4096, False),
                                         (20, 77, 2048, False), (30, 19, 1032, True)])
def test_linear_f32_shared_tiles_with_lanes_past_the_outputs(R, N, K, gated):
    """Against torch's product in 64 bits; sums of 32 products, then of those sums, within the bound of K + 4 roundings."""
    g = torch.Generator(device="cuda").manual_seed(R + N)
    ctx = make_ctx("f32")
    x, w, u = (torch.randn(s, generator=g, device="cuda") for s in ((R, K), (N, K), (N, K)))
    op, guard = jk.Linear(ctx, w, w_up=u if gated else None), Guard()
    outs = [guard.alloc((R, N), torch.float32) for _ in range(3)]
    for o in outs:
        ctx.linear(op, x, o)
    guard.check()
    assert ctx.read_status() == 0 and torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    z = x.double() @ w.double().T
    e = (K + 4) * 2.0 ** -24 * (x.abs().double() @ w.abs().double().T)
    if gated:
        zu = x.double() @ u.double().T
        eu = (K + 4) * 2.0 ** -24 * (x.abs().double() @ u.abs().double().T)
        z, e = z * zu, e * zu.abs() + z.abs() * eu + e * eu + 2.0 ** -24 * (z * zu).abs()
    assert bool(((outs[0].double() - z).abs() <= e + 2.0 ** -23 * (z.abs() + e)).all())


@pytest.mark.parametrize("sections", [(32,), (8, 24)])
def test_rope_positions_of_each_shape(sections):
    """Positions with and without the tokens in one line agree; those of a larger tree's buffer are refused whole and taken
    sliced."""
    B, M, Hq, Hkv, D, A = 2, 3, 4, 2, 64, len(sections)
    T = dict(dtype=torch.bfloat16, device="cuda")
    ctx = make_ctx("bf16", Hq, Hkv, D)
    qkv, large = torch.randn(B, M, (Hq + 2 * Hkv) * D, **T), torch.randint(0, 4096, (B, M + 2, A), dtype=torch.int32, device="cuda")
    new = lambda: [torch.zeros(s, **T) for s in ((B, M, Hq, D), (B, Hkv, 8, D), (B, Hkv, 8, D))]
    pos = large[:, :M].contiguous()
    shapes, outs = [pos, pos.view(B * M, A)] + ([pos.view(B, M), pos.view(-1)] if A == 1 else []), []
    for p in shapes:
        outs.append(new())
        ctx.rope_qkv(B, M, qkv, p, sections, 1e4, *outs[-1])
    for o in outs[1:]:
        assert all(torch.equal(s, t) for s, t in zip(outs[0], o))
    for p in [large, large.view(-1, A), large[:, :M]] + ([large.view(B, M + 2)] if A == 1 else []):
        with pytest.raises(ValueError, match="pos"):
            ctx.rope_qkv(B, M, qkv, p, sections, 1e4, *new())
    assert ctx.read_status() == 0


def test_rope_k_and_v_in_one_buffer():
    """K and V as halves of one buffer, by sequence, by head and by rows; where they would share a row the call is refused."""
    B, M, Hq, Hkv, D, rows = 3, 5, 4, 2, 64, 8
    T = dict(dtype=torch.bfloat16, device="cuda")
    ctx = make_ctx("bf16", Hq, Hkv, D)
    qkv, q = torch.randn(B, M, (Hq + 2 * Hkv) * D, **T), torch.zeros(B, M, Hq, D, **T)
    pos, first = torch.randint(0, 99, (B, M), dtype=torch.int32, device="cuda"), torch.tensor([0, 3, 1], dtype=torch.int32, device="cuda")
    k, v = (torch.zeros(B, Hkv, rows, D, **T) for _ in range(2))
    ctx.rope_qkv(B, M, qkv, pos, (D // 2,), 1e4, q, k, v, first_row=first)
    a, b, c = torch.zeros(B, 2, Hkv, rows, D, **T), torch.zeros(B, Hkv, 2, rows, D, **T), torch.zeros(B, Hkv, 2 * rows, D, **T)
    for k2, v2 in ((a[:, 0], a[:, 1]), (b[:, :, 0], b[:, :, 1]), (c[:, :, :rows], c[:, :, rows:])):
        ctx.rope_qkv(B, M, qkv, pos, (D // 2,), 1e4, q, k2, v2, first_row=first)
        assert torch.equal(k, k2) and torch.equal(v, v2)
    for k2, v2 in ((c[:, :, :rows], c[:, :, 1:rows + 1]), (c[:, :, rows - 1:-1], c[:, :, :rows]), (c, c)):
        with pytest.raises(RuntimeError, match="jk_rope_qkv"):
            ctx.rope_qkv(B, M, qkv, pos, (D // 2,), 1e4, q, k2, v2, first_row=first)
    assert ctx.read_status() == 0


def test_rope_one_head_of_k_and_v_of_any_stride():
    """One KV head, its rows [batch, rows, 1, d] seen as [batch, 1, rows, d]: the stride of the dimension of one is d."""
    B, M, Hq, D, rows = 2, 5, 4, 64, 8
    T = dict(dtype=torch.bfloat16, device="cuda")
    ctx = make_ctx("bf16", Hq, 1, D)
    qkv, q = torch.randn(B, M, (Hq + 2) * D, **T), torch.zeros(B, M, Hq, D, **T)
    pos = torch.randint(0, 99, (B, M), dtype=torch.int32, device="cuda")
    a, b = ([torch.zeros(s, **T) for _ in range(2)] for s in ((B, 1, rows, D), (B, rows, 1, D)))
    ctx.rope_qkv(B, M, qkv, pos, (D // 2,), 1e4, q, *a)
    ctx.rope_qkv(B, M, qkv, pos, (D // 2,), 1e4, q, *(t.as_strided((B, 1, rows, D), (rows * D, D, D, 1)) for t in b))
    for s, t in zip(a, b):
        assert torch.equal(s[:, 0], t[:, :, 0]) and bool(s[:, :, :M].any())
    assert ctx.read_status() == 0
