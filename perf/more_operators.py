"""The steps of a target layer around its attention, as cases that can be timed and compared: RMS norm with the
residual's addition (16-bit or 8-bit output), matrix products with bias, activation, gate and residual in their
epilogue (16-bit, 32-bit or 8-bit operands), and rotary positions with one or several axes that place K and V.

`own` chooses between the plain forms (elementary torch operations in 32 or 64 bits) and the calls a user makes of
this package.  Shapes are those of the package's workloads (LLaMA-2 7B / 13B / 70B and LLaMA-3 8B layers, trees of 60
nodes, the small test workload) and a range around them.

8-bit rows ("mx8"): e4m3 codes [rows, n] and one power-of-two scale for each 32 elements of a row, stored as the
exponent plus 127 in tiles of 128 rows x 4 blocks: row r, block k lies at byte
(r // 128 * ceil(n / 128) + k // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + k % 4.
"""
import math

import torch

own = False

DEV = "cuda"
E4M3 = torch.float8_e4m3fn
E8M0 = torch.float8_e8m0fnu
EPS = 1e-5


# --------------------------------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------------------------------
def _norm(name, R, n, dtype="bf16", add=True, norm=True, out="T"):
    c = dict(kind="norm", R=R, n=n, dtype=dtype, add=add, norm=norm, out=out)
    return {"name": name, **c} if name else c


def _linear(name, R, N, K, weights="T", dtype="bf16", gated=False, act="none", bias=False, residual=False, out="T",
            wide=0):
    c = dict(kind="linear", R=R, N=N, K=K, weights=weights, dtype=dtype, gated=gated, act=act, bias=bias,
             residual=residual, out=out, wide=wide)
    return {"name": name, **c} if name else c


def _rope(name, B, M, Hq, Hkv, d, axes, cache, dtype="bf16", far=4096):
    c = dict(kind="rope", B=B, M=M, Hq=Hq, Hkv=Hkv, d=d, axes=axes, cache=cache, dtype=dtype, far=far)
    return {"name": name, **c} if name else c


def listed():
    return [
        # before the attention when one token is decoded at the 7B width (latency)
        _norm("norm_token_7b", 1, 4096),
        # four trees of 60 nodes at the 8B width, for 8-bit projections
        _norm("norm_tree_8b_mx8", 240, 4096, out="both"),
        # a long prompt at the 70B width: bound by memory
        _norm("norm_prompt_70b_mx8", 8191, 8192, out="mx8"),
        # output projection of a verified tree, added to the residual stream
        _linear("o_tree_7b", 60, 4096, 4096, residual=True),
        # first half of the 7B FFN for a verified tree
        _linear("gated_tree_7b", 60, 11008, 4096, gated=True, act="silu"),
        # first half of the 8B FFN for a single token, all in 8 bits
        _linear("gated_token_8b_mx8", 1, 14336, 4096, weights="mx8", gated=True, act="silu", out="mx8"),
        # second half of the 13B FFN for eight trees, 8-bit operands
        _linear("down_tree_13b_b8_mx8", 480, 5120, 13824, weights="mx8", residual=True),
        # a projection with bias and GELU over a prompt of odd length, 13B width
        _linear("prompt_13b_gelu", 2047, 5120, 5120, act="gelu", bias=True),
        # first half of the 8B FFN over a long prompt, 8 bits: bound by the tensor cores
        _linear("gated_prompt_8b_mx8", 4099, 14336, 4096, weights="mx8", gated=True, act="silu", out="mx8"),
        # the single-precision test workload's FFN
        _linear("gated_f32", 16, 1376, 512, dtype="f32", gated=True, act="silu"),
        # rotary positions of four trees' nodes, K and V into the tree arrays (latency)
        _rope("rope_tree_8b", 4, 60, 32, 8, 128, 1, False),
        # a prompt with images: three axes, K and V into the cache
        _rope("rope_prompt_axes_7b", 2, 2047, 32, 32, 128, 3, True, far=100000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


WIDTHS = (512, 1376, 4096, 5120, 8192, 11008, 13824, 14336)


def draw(rng):
    c = _draw(rng)
    while work(c)["bytes"] > 470_000_000:              # no more than the largest listed case
        size = "N" if c["kind"] == "linear" else "M" if c["kind"] == "rope" else "R"
        c[size] //= 2
        if c.get("out") == "mx8" and size == "N":
            c[size] = max(1, c[size] // 32) * 32
    return c


def _draw(rng):
    kind = rng.choice(["norm", "linear", "linear", "linear", "rope"])
    if kind == "norm":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        n = rng.choice([rng.choice(WIDTHS), 32 * rng.randint(1, 600)])
        out = rng.choice(["T", "mx8", "both"])
        if out == "T":
            n = n + 8 * rng.randint(0, 3)
        norm = out != "mx8" or rng.random() < 0.6
        return _norm(None, max(1, min(_log(rng, 1, 16384), 30_000_000 // n)), n, dtype, norm and rng.random() < 0.7, norm,
                     out)
    if kind == "rope":
        Hkv = rng.choice([1, 2, 8, 8, 32, 40])
        Hq = Hkv * (rng.choice([1, 2, 4, 8]) if Hkv <= 8 else 1)
        B, M = _log(rng, 1, 16), _log(rng, 1, 4096)
        while B * M * (Hq + 2 * Hkv) > 1_000_000:
            B, M = max(1, B // 2), max(1, M * 3 // 4)
        return _rope(None, B, M, Hq, Hkv, rng.choice([128, 128, 64]), rng.choice([1, 2, 3]), rng.random() < 0.5,
                     rng.choice(["bf16", "bf16", "f32"]), _log(rng, 16, 1_000_000))
    weights = rng.choice(["T", "T", "mx8", "mx8"])
    dtype = "bf16" if weights == "mx8" else rng.choice(["bf16", "bf16", "bf16", "f32"])
    unit = 32 if weights == "mx8" else 8
    K = rng.choice([rng.choice(WIDTHS), unit * rng.randint(1, 14336 // unit)])
    gated = rng.random() < 0.4
    out = rng.choice(["T", "T", "mx8"]) if dtype == "bf16" else "T"
    N = rng.choice([rng.choice(WIDTHS), 32 * rng.randint(1, 448) if out == "mx8" else rng.randint(1, 14336)])
    R = rng.choice([_log(rng, 1, 4096), rng.randint(1, 64), 60])
    most = 2e11 if dtype == "f32" else 9e11            # operations of a case, at most the largest listed one's
    while 2.0 * R * N * K * (1 + gated) > most:
        R = max(1, R * 3 // 4)
    return _linear(None, R, N, K, weights, dtype, gated, rng.choice(["none", "silu", "gelu"]), rng.random() < 0.3,
                   out == "T" and rng.random() < 0.5, out, rng.choice([0, 0, 8, 64]) if weights == "T" else 0)


# --------------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------------
def _tdtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _exponent(amax):
    """The exponent of the smallest power of two s >= 2^-32 with amax <= 448 s, exactly (frexp)."""
    m, e = torch.frexp(amax)                           # amax = m 2^e, m in [1/2, 1); 448 = 7/8 2^9
    e = torch.where(m > 0.875, e - 8, e - 9)
    return torch.where(amax > 0, e, torch.full_like(e, -32)).clamp(min=-32)


def _quantise(y):
    """y [rows, n] f32 -> (e4m3 codes, exponents [rows, n / 32])."""
    b = y.unflatten(1, (-1, 32))
    e = _exponent(b.abs().amax(2))
    s = torch.exp2(-e.float())                         # exact: powers of two in the normal range
    return (b * s[..., None]).clamp(-448.0, 448.0).flatten(1).to(E4M3), e


def _scale_bytes(R, n):
    return -(-R // 128) * -(-n // 128) * 512


def _tile(e, n):
    """Exponents [rows, n / 32] in the order of the scale tiles; places that belong to no row or block are 0."""
    R, k = e.shape
    rt, kt = -(-R // 128), -(-n // 128)
    full = torch.zeros(rt * 128, kt * 4, dtype=torch.uint8, device=e.device)
    full[:R, :k] = (e + 127).to(torch.uint8)
    return full.view(rt, 4, 32, kt, 4).permute(0, 3, 2, 1, 4).reshape(-1)


def _untile(scales, R, n):
    """The scales as 32-bit numbers [rows, n / 32]."""
    rt, kt = -(-R // 128), -(-n // 128)
    full = scales.view(rt, kt, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(rt * 128, kt * 4)[:R, :n // 32]
    return torch.exp2(full.float() - 127.0)


def _values(codes, scales):
    """8-bit rows as the 32-bit values they stand for (a code times a power of two: exact)."""
    R, n = codes.shape
    return (codes.view(E4M3).float().unflatten(1, (-1, 32)) * _untile(scales, R, n)[..., None]).flatten(1)


def _hidden(R, n, g):
    """Hidden states as a layer sees them: channels of different size (a few large ones), rows too."""
    gain = torch.exp(0.5 * torch.randn(n, generator=g, device=DEV))
    gain[torch.randint(0, n, (max(1, n // 512),), generator=g, device=DEV)] *= 12.0
    x = torch.randn(R, n, generator=g, device=DEV)
    return x.mul_(gain).mul_(torch.exp(0.2 * torch.randn(R, 1, generator=g, device=DEV)))


def _weights(N, K, g):
    return torch.randn(N, K, generator=g, device=DEV).mul_(0.02)


def _mx8(x):
    codes, e = _quantise(x.float())
    return codes.view(torch.uint8), _tile(e, x.shape[1])


def _empty_mx8(R, n):
    return (torch.zeros(R, n, dtype=torch.uint8, device=DEV),
            torch.zeros(_scale_bytes(R, n), dtype=torch.uint8, device=DEV))


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed) * 7919 + 23)
    s = {"case": dict(case)}
    T = _tdtype(case["dtype"])
    kind = case["kind"]
    if kind == "norm":
        R, n = case["R"], case["n"]
        s["x"] = _hidden(R, n, g).to(T)
        s["delta"] = _hidden(R, n, g).mul_(0.3).to(T) if case["add"] else None
        s["w"] = (1.0 + 0.1 * torch.randn(n, generator=g, device=DEV)).to(T)
        s["sum"] = torch.empty_like(s["x"]) if case["add"] else None
        s["out"] = torch.empty_like(s["x"]) if case["out"] != "mx8" else None
        s["codes"], s["scales"] = _empty_mx8(R, n) if case["out"] != "T" else (None, None)
        if own:
            s["ctx"] = _context(case["dtype"])
            s["mx8"] = _handle(s["codes"], s["scales"])
    elif kind == "linear":
        R, N, K = case["R"], case["N"], case["K"]
        x = _hidden(R, K, g)
        ws = [_weights(N, K, g) for _ in range(1 + case["gated"])]
        if case["weights"] == "mx8":
            s["x"], s["w"] = _mx8(x), [_mx8(w) for w in ws]
        else:
            # rows of a wider array, as the columns of a fused projection's output are
            s["x"] = torch.zeros(R, K + case["wide"], dtype=T, device=DEV)[:, :K]
            s["x"].copy_(x)
            s["w"] = [w.to(T) for w in ws]
        del x, ws
        s["bias"] = [0.5 * torch.randn(N, generator=g, device=DEV) for _ in s["w"]] if case["bias"] else None
        if case["bias"]:
            s["bias"] = [b.to(T) for b in s["bias"]]
        s["residual"] = _hidden(R, N, g).to(T) if case["residual"] else None
        if case["out"] == "mx8":
            s["codes"], s["scales"] = _empty_mx8(R, N)
        else:
            s["out"] = torch.empty(R, N, dtype=T, device=DEV)
        if own:
            s["ctx"] = _context(case["dtype"])
            s["op"] = _op(s)
            s["xh"] = _handle(*s["x"]) if case["weights"] == "mx8" else s["x"]
            s["outh"] = _handle(s["codes"], s["scales"]) if case["out"] == "mx8" else s["out"]
    else:
        B, M, Hq, Hkv, d, A = (case[k] for k in ("B", "M", "Hq", "Hkv", "d", "axes"))
        s["qkv"] = torch.randn(B, M, (Hq + 2 * Hkv) * d, generator=g, device=DEV).to(T)
        first = torch.randint(0, 9, (B,), generator=g, device=DEV, dtype=torch.int32)
        # nodes of a tree share positions; images are grids at one time; text runs on
        s["pos"] = torch.randint(0, case["far"], (B, 1, A), generator=g, device=DEV, dtype=torch.int32) + torch.randint(
            0, min(M, case["far"]) + 1, (B, M, A), generator=g, device=DEV, dtype=torch.int32)
        rows = M + 8 if case["cache"] else M
        s["first"] = first if case["cache"] else None
        s["q"] = torch.empty(B, M, Hq, d, dtype=T, device=DEV)
        s["k"] = torch.zeros(B, Hkv, rows, d, dtype=T, device=DEV)
        s["v"] = torch.zeros(B, Hkv, rows, d, dtype=T, device=DEV)
        half = d // 2
        s["sections"] = {1: (half,), 2: (half // 4, half - half // 4),
                         3: (half // 4, half * 3 // 8, half * 3 // 8)}[A]
        if own:
            s["ctx"] = _context(case["dtype"], Hq, Hkv, d)
    return s


def _context(dtype, Hq=1, Hkv=1, d=64):
    from paper_2502_06282_b200 import binding
    return binding.Context(hidden=8, n_experts=1, top_k=1, inter=8, vocab=8, n_q_heads=Hq, n_kv_heads=Hkv,
                           head_dim=d, max_batch=1, max_tree=1, max_depth=1, max_frontier=1, k_per_expert=1,
                           dtype=dtype, rms_eps=EPS)


def _handle(codes, scales):
    from paper_2502_06282_b200 import binding
    return None if codes is None else binding.Mx8(codes, scales)


def _op(s):
    from paper_2502_06282_b200 import binding
    w = [_handle(*x) for x in s["w"]] if s["case"]["weights"] == "mx8" else s["w"]
    b = s["bias"] or [None, None]
    return binding.Linear(s["ctx"], w[0], bias=b[0], act=s["case"]["act"],
                          **(dict(w_up=w[1], bias_up=b[1]) if s["case"]["gated"] else {}))


# --------------------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------------------
def run(s):
    return {"norm": _run_norm, "linear": _run_linear, "rope": _run_rope}[s["case"]["kind"]](s)


def _codes(s):
    """8-bit outputs as the 8-bit numbers they are."""
    return {"codes": s["codes"].view(E4M3), "scales": s["scales"].view(E8M0)}


def _store_mx8(s, y):
    codes, e = _quantise(y)
    s["codes"].copy_(codes.view(torch.uint8))
    s["scales"].copy_(_tile(e, y.shape[1]))


def _run_norm(s):
    case = s["case"]
    if own and case["norm"]:
        s["ctx"].add_norm(s["x"], s["w"], delta=s["delta"], out_sum=s["sum"], out=s["out"], out_mx8=s["mx8"])
    elif own:
        s["ctx"].quantize_mx8(s["x"], s["mx8"])
    else:
        y = s["x"].float()
        if case["add"]:
            y = y + s["delta"].float()
            s["sum"].copy_(y)
        if case["norm"]:
            y = y * torch.rsqrt((y * y).mean(1, keepdim=True) + EPS) * s["w"].float()
        if case["out"] != "mx8":
            s["out"].copy_(y)
        if case["out"] != "T":
            _store_mx8(s, y)
    return {**({"sum": s["sum"]} if case["add"] else {}), **({"out": s["out"]} if case["out"] != "mx8" else {}),
            **(_codes(s) if case["out"] != "T" else {})}


def _act(z, act):
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def _run_linear(s):
    case = s["case"]
    if own:
        s["ctx"].linear(s["op"], s["xh"], s["outh"], residual=s["residual"])
    else:
        mx8 = case["weights"] == "mx8"
        x = _values(*s["x"]) if mx8 else s["x"].float()
        z = []
        for i, w in enumerate(s["w"]):
            y = x @ (_values(*w) if mx8 else w.float()).T
            z.append(y + s["bias"][i].float() if case["bias"] else y)
        y = _act(z[0], case["act"])
        if case["gated"]:
            y = y * z[1]
        if case["residual"]:
            y = y + s["residual"].float()
        if case["out"] == "mx8":
            _store_mx8(s, y)
        else:
            s["out"].copy_(y)
    return _codes(s) if case["out"] == "mx8" else s["out"]


def _axis_of(sections):
    return [a for a, n in enumerate(sections) for _ in range(n)]


def _run_rope(s):
    case = s["case"]
    B, M, Hq, Hkv, d = (case[k] for k in ("B", "M", "Hq", "Hkv", "d"))
    if own:
        s["ctx"].rope_qkv(B, M, s["qkv"], s["pos"], s["sections"], 10000.0, s["q"], s["k"], s["v"], first_row=s["first"])
    else:
        half = d // 2
        freq = torch.exp(torch.arange(half, device=DEV, dtype=torch.float64) * (-2.0 * math.log(10000.0) / d))
        angle = s["pos"].double()[..., _axis_of(s["sections"])] * freq                   # [B, M, d / 2]
        cos, sin = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]
        heads = s["qkv"].unflatten(2, (Hq + 2 * Hkv, d)).float()
        a, b = heads[:, :, :Hq + Hkv, :half], heads[:, :, :Hq + Hkv, half:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], 3)
        s["q"].copy_(turned[:, :, :Hq])
        at = torch.arange(M, device=DEV)[None].expand(B, M)
        if s["first"] is not None:
            at = at + s["first"][:, None]
        at = at[:, None, :, None].expand(B, Hkv, M, d)
        s["k"].scatter_(2, at, turned[:, :, Hq:].transpose(1, 2).to(s["k"].dtype))
        s["v"].scatter_(2, at, heads[:, :, Hq + Hkv:].transpose(1, 2).to(s["v"].dtype))
    return {"q": s["q"], "k": s["k"], "v": s["v"]}


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "norm":
        R, n = case["R"], case["n"]
        per = e * (1 + 2 * case["add"] + (case["out"] != "mx8")) + (1 + 1 / 32) * (case["out"] != "T")
        return {"bytes": R * n * per + n * e * case["norm"], "flops": 4.0 * R * n}
    if case["kind"] == "rope":
        heads = case["Hq"] + 2 * case["Hkv"]
        rows = case["B"] * case["M"]
        return {"bytes": 2.0 * rows * heads * case["d"] * e + 4 * rows * case["axes"],
                "flops": 3.0 * rows * (case["Hq"] + case["Hkv"]) * case["d"]}
    R, N, K = case["R"], case["N"], case["K"]
    g = 1 + case["gated"]
    unit = 33 / 32 if case["weights"] == "mx8" else e
    out = N * R * (33 / 32 if case["out"] == "mx8" else e)
    return {"bytes": (R * K + g * N * K) * unit + out + case["residual"] * R * N * e + case["bias"] * g * N * e,
            "flops": 2.0 * R * N * K * g}


# --------------------------------------------------------------------------------------------------
# definitions in 64 bits
# --------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "linear": _exact_linear, "rope": _exact_rope}[case["kind"]](s)


def _exact_mx8(y):
    """The elements in units of their block's scale, before they are rounded to 4 significant bits.  The scale itself
    has no such value: where a block's largest element lies next to the border, 32 bits may go either way."""
    b = y.unflatten(1, (-1, 32))
    e = torch.ceil(torch.log2(b.abs().amax(2) / 448.0)).clamp(min=-32.0)
    return {"codes": (b / torch.exp2(e)[..., None]).flatten(1), "scales": None}


def _exact_values(codes, scales):
    """Code bits and scale bytes to 64-bit values: sign, 4 exponent bits (bias 7), 3 bits of fraction."""
    R, n = codes.shape
    c = codes.to(torch.int64)
    sign, ex, frac = 1.0 - 2.0 * (c >> 7).double(), (c >> 3) & 15, (c & 7).double()
    v = torch.where(ex > 0, (1.0 + frac / 8.0) * torch.exp2(ex.double() - 7.0), frac * 2.0 ** -9) * sign
    r = torch.arange(R, device=DEV)[:, None]
    k = torch.arange(n // 32, device=DEV)[None]
    at = (r // 128 * -(-n // 128) + k // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + k % 4
    e = scales.to(torch.int64)[at].double() - 127.0
    return v * torch.exp2(e).repeat_interleave(32, 1)


def _exact_norm(s):
    case = s["case"]
    y = s["x"].double()
    out = {}
    if case["add"]:
        y = y + s["delta"].double()
        out["sum"] = y
    if case["norm"]:
        y = s["w"].double() * y / torch.sqrt(y.square().sum(1, keepdim=True) / case["n"] + EPS)
    if case["out"] != "mx8":
        out["out"] = y
    return {**out, **(_exact_mx8(y) if case["out"] != "T" else {})}


def _exact_linear(s):
    case = s["case"]
    x = _exact_values(*s["x"]) if case["weights"] == "mx8" else s["x"].double()
    zs = []
    for i, w in enumerate(s["w"]):
        w = _exact_values(*w) if case["weights"] == "mx8" else w.double()
        z = torch.einsum("rk,nk->rn", x, w)
        zs.append(z if s["bias"] is None else z + s["bias"][i].double())
    z = zs[0]
    y = z * torch.sigmoid(z) if case["act"] == "silu" else z
    if case["act"] == "gelu":
        y = z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
    if case["gated"]:
        y = y * zs[1]
    if s["residual"] is not None:
        y = y + s["residual"].double()
    return _exact_mx8(y) if case["out"] == "mx8" else y


def _exact_rope(s):
    case = s["case"]
    B, M, Hq, Hkv, d = (case[k] for k in ("B", "M", "Hq", "Hkv", "d"))
    half = d // 2
    axis = torch.tensor(_axis_of(s["sections"]), device=DEV)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV).expand(B, M, half),
                       s["pos"].double().index_select(2, axis) / 10000.0 ** (torch.arange(half, device=DEV).double() * 2 / d))
    rows = s["qkv"].double().view(B, M, Hq + 2 * Hkv, d)
    z = torch.complex(rows[:, :, :Hq + Hkv, :half].contiguous(), rows[:, :, :Hq + Hkv, half:].contiguous())
    z = z * turn[:, :, None]
    z = torch.cat([z.real, z.imag], 3)
    k, v = s["k"].double(), s["v"].double()
    for b in range(B):
        r0 = 0 if s["first"] is None else int(s["first"][b])
        k[b, :, r0:r0 + M] = z[b, :, Hq:].transpose(0, 1)
        v[b, :, r0:r0 + M] = rows[b, :, Hq + Hkv:].transpose(0, 1)
    return {"q": z[:, :, :Hq], "k": k, "v": v}
