"""The serving operators around the draft-and-verify step, as cases that can be timed and compared: tree
attention over a paged 8-bit KV cache, the calls that fill, extend, fork, free and compact such a cache, and
sampling with temperature, top-k, top-p and min-p.

`own` chooses between the plain forms (elementary torch operations in 32 or 64 bits) and the calls a user makes
of this package.  Shapes are those of the package's workloads (LLaMA-2 7B / 13B / 70B and LLaMA-3 8B heads, trees
of 60 nodes, 32 layers) and a range around them.
"""
import math

import torch

own = False

DEV = "cuda"
E4M3 = torch.float8_e4m3fn
MAX_DEPTH = 6                              # draft depth of the workloads: at most 6 accepted nodes


# --------------------------------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------------------------------
def _attn(name, B, Hq, Hkv, d, P, M, ps, dtype="bf16", ragged=False):
    c = dict(kind="attn", B=B, Hq=Hq, Hkv=Hkv, d=d, P=P, M=M, ps=ps, dtype=dtype, ragged=ragged)
    return {"name": name, **c} if name else c


def _commit(name, B, Hkv, d, P, M, ps, L, dtype="bf16"):
    c = dict(kind="commit", B=B, Hkv=Hkv, d=d, P=P, M=M, ps=ps, L=L, dtype=dtype)
    return {"name": name, **c} if name else c


def _import(name, B, Hkv, d, P, ps, L, dtype="bf16", ragged=False):
    c = dict(kind="import", B=B, Hkv=Hkv, d=d, P=P, ps=ps, L=L, dtype=dtype, ragged=ragged)
    return {"name": name, **c} if name else c


def _fork(name, n_src, n_fork, Hkv, d, P, ps, L):
    c = dict(kind="fork", n_src=n_src, n_fork=n_fork, Hkv=Hkv, d=d, P=P, ps=ps, L=L)
    return {"name": name, **c} if name else c


def _compact(name, n_seq, n_gone, Hkv, d, P, ps, L):
    c = dict(kind="compact", n_seq=n_seq, n_gone=n_gone, Hkv=Hkv, d=d, P=P, ps=ps, L=L)
    return {"name": name, **c} if name else c


def _copy(name, n_copy, Hkv, d, ps, L):
    c = dict(kind="copy", n_copy=n_copy, Hkv=Hkv, d=d, ps=ps, L=L)
    return {"name": name, **c} if name else c


def _sample(name, R, V, dtype, top_k, top_p, min_p, filtered, spread):
    c = dict(kind="sample", R=R, V=V, dtype=dtype, top_k=top_k, top_p=top_p, min_p=min_p, filtered=filtered,
             spread=spread)
    return {"name": name, **c} if name else c


def listed():
    return [
        # plain decoding of one sequence: a single token, one layer of the 7B heads (latency)
        _attn("attn_token_7b", 1, 32, 32, 128, 1024, 1, 64),
        # the verification call of the default workload: 60 tree nodes over a prefix of 1024
        _attn("attn_tree_7b", 1, 32, 32, 128, 1024, 60, 128),
        # grouped heads (8B), four sequences of uneven odd lengths, small pages
        _attn("attn_tree_8b_ragged", 4, 32, 8, 128, 4099, 60, 32, ragged=True),
        # a full server batch at a long prefix: bound by reading the cache
        _attn("attn_tree_13b_b8", 8, 40, 40, 128, 8192, 60, 64),
        # decoding a batch of long sequences with the 70B heads, eight query heads per kv head
        _attn("attn_token_70b_long", 32, 64, 8, 128, 16384, 1, 64, ragged=True),
        # the single-precision context with the small head size (the test workload's shape)
        _attn("attn_f32", 2, 8, 8, 64, 333, 16, 16, dtype="f32", ragged=True),
        # after a step: the accepted path of eight sequences joins the caches of all 32 layers
        _commit("commit_step", 8, 8, 128, 4096, 60, 64, 32),
        # after a prompt's pass: 32 layers of a 16-bit cache become pages
        _import("import_prompt", 1, 32, 128, 2047, 64, 32),
        # parallel sampling: sequences are forked, then the forks end
        _fork("fork_free", 4, 28, 8, 128, 2048 + 37, 64, 32),
        # finished sequences leave and the pool is packed (the pages that move are copied in all layers)
        _compact("free_compact", 24, 11, 8, 128, 2048 + 21, 64, 32),
        # one token for one sequence with the usual filters
        _sample("sample_token", 1, 32000, "f32", 50, 0.9, 0.0, False, 4.0),
        # the target rows of four trees, filtered for the acceptance walk, large vocabulary
        _sample("sample_tree_rows", 240, 128256, "bf16", 0, 0.95, 0.02, True, 3.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    c = _draw(rng)
    while work(c)["bytes"] > 1_600_000_000:            # no more than the largest listed case
        c["L" if c.get("L", 1) > 1 else "n_copy" if "n_copy" in c else "P"] //= 2
    return c


def _draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "commit", "import", "fork", "compact", "copy", "sample", "sample"])
    ps = rng.choice([16, 32, 64, 128])
    d = rng.choice([128, 128, 128, 64])
    if kind == "attn":
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        Hkv = rng.choice([1, 2, 4, 8, 8, 32, 40])
        G = rng.choice([1, 2, 4, 8]) if Hkv <= 8 else 1
        M = rng.choice([1, 1, rng.randint(2, 128), 60, 16])
        B = _log(rng, 1, 32)
        P = _log(rng, 1, 32768)
        cap = 5_000_000 if dtype == "f32" else 60_000_000     # (row, key, head) products a case may cost
        while B * P * Hkv * G * M > cap * 2 or B * P * Hkv > 4_000_000:
            B, P = max(1, B // 2), max(1, (P * 3) // 4)
        return _attn(None, B, Hkv * G, Hkv, d, P, M, ps, dtype, rng.random() < 0.5)
    if kind == "commit":
        return _commit(None, _log(rng, 1, 32), rng.choice([2, 8, 32]), d, _log(rng, 1, 4096),
                       rng.choice([1, 16, 60, rng.randint(2, 128)]), ps, rng.choice([1, 4, 16]),
                       rng.choice(["bf16", "bf16", "f32"]))
    if kind == "import":
        return _import(None, rng.randint(1, 4), rng.choice([2, 8]), d, _log(rng, 1, 8192), ps, rng.choice([1, 8, 32]),
                       rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.5)
    if kind == "fork":
        return _fork(None, rng.randint(1, 8), _log(rng, 1, 64), rng.choice([2, 8]), d, _log(rng, 1, 4096), ps,
                     rng.choice([1, 8, 32]))
    if kind == "compact":
        n = rng.randint(3, 32)
        return _compact(None, n, rng.randint(1, n), rng.choice([2, 8]), d, _log(rng, 200, 2048), ps,
                        rng.choice([1, 8, 24]))
    if kind == "copy":
        return _copy(None, _log(rng, 1, 512), rng.choice([2, 8]), d, ps, rng.choice([1, 8, 32]))
    V = rng.choice([32000, 128256, _log(rng, 17, 200000)])
    return _sample(None, max(1, min(_log(rng, 1, 480), 30_000_000 // V)), V, rng.choice(["f32", "bf16"]),
                   rng.choice([0, 0, 1, 40, 1000]), rng.choice([1.0, 0.9, 0.95, 0.5]), rng.choice([0.0, 0.0, 0.05]),
                   rng.random() < 0.5, rng.choice([0.5, 2.0, 4.0]))


# --------------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------------
def _tdtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _pow2_scale(amax):
    """The smallest power of two s >= 2^-32 with amax <= 448 s, exactly (frexp)."""
    m, e = torch.frexp(amax / 448.0)                   # amax / 448 = m 2^e, m in [1/2, 1)
    e = torch.where(m > 0.5, e, e - 1)
    e = torch.where(torch.ldexp(torch.full_like(amax, 448.0), e) < amax, e + 1, e)   # the division rounded
    e = torch.where(torch.ldexp(torch.full_like(amax, 448.0), e - 1) >= amax, e - 1, e)
    e = torch.where(amax > 0, e, torch.full_like(e, -32)).clamp(min=-32)
    return torch.ldexp(torch.ones_like(amax), e)


def _quantise(x):
    """x [..., ps, d] -> (e4m3 codes, scale [...]): one power-of-two scale per block."""
    x = x.float()
    s = _pow2_scale(x.abs().amax(dim=(-2, -1)))
    return (x / s[..., None, None]).clamp(-448.0, 448.0).to(E4M3), s


def _new_cache(L, n_pages, ps, max_seqs, max_pages, Hkv, d, dtype):
    i32 = dict(dtype=torch.int32, device=DEV)
    c = {"k_pages": torch.zeros(L, n_pages, Hkv, ps, d, dtype=torch.uint8, device=DEV),
         "v_pages": torch.zeros(L, n_pages, Hkv, ps, d, dtype=torch.uint8, device=DEV),
         "k_scale": torch.ones(L, n_pages, Hkv, device=DEV), "v_scale": torch.ones(L, n_pages, Hkv, device=DEV),
         "k_open": torch.zeros(L, max_seqs, Hkv, 2 * ps, d, dtype=_tdtype(dtype), device=DEV),
         "v_open": torch.zeros(L, max_seqs, Hkv, 2 * ps, d, dtype=_tdtype(dtype), device=DEV)}
    # the bookkeeping in one array, the parts of it under their names
    book = torch.zeros(max_seqs + max_seqs * max_pages + 2 * n_pages + 1, **i32)
    c["book"] = book
    c["kv_len"] = book[:max_seqs]
    at = max_seqs
    c["page_table"] = book[at:at + max_seqs * max_pages].view(max_seqs, max_pages)
    at += max_seqs * max_pages
    c["refcount"] = book[at:at + n_pages]
    c["free_list"] = book[at + n_pages:at + 2 * n_pages]
    c["n_free"] = book[at + 2 * n_pages:]
    c["page_table"].fill_(-1)
    c["free_list"].copy_(torch.arange(n_pages - 1, -1, -1, **i32))
    c["n_free"].fill_(n_pages)
    return c


def _fill_pages(c, g, like):
    """Codes and scales of plausible keys and values: normal rows, each block with a size of its own."""
    for name in ("k", "v"):
        pages, scale = c[name + "_pages"], c[name + "_scale"]
        for layer in range(pages.shape[0]):
            if layer and like != "all":                # one layer's values serve every layer, rolled by a page
                pages[layer].copy_(pages[layer - 1].roll(1, 0))
                scale[layer].copy_(scale[layer - 1].roll(1, 0))
                continue
            step = max(1, (1 << 26) // pages[0, 0].numel())
            for p0 in range(0, pages.shape[1], step):
                x = torch.randn(pages[layer, p0:p0 + step].shape, generator=g, device=DEV)
                size = torch.exp(0.5 * torch.randn(x.shape[:2], generator=g, device=DEV))
                q, s = _quantise((x * size[..., None, None]).bfloat16())
                pages[layer, p0:p0 + step] = q.view(torch.uint8)
                scale[layer, p0:p0 + step] = s
        c[name + "_open"].copy_(_randn_like(c[name + "_open"], g))


def _randn_like(t, g):
    out = torch.empty_like(t)
    flat, n = out.view(-1), 1 << 27
    for a in range(0, flat.numel(), n):
        flat[a:a + n] = torch.randn(flat[a:a + n].shape, generator=g, device=DEV)
    return out


def _give_pages(c, lens, g):
    """Rows of the table for sequences of these lengths, from shuffled pages; the rest is free."""
    ps, n_pages = c["k_pages"].shape[3], c["k_pages"].shape[1]
    perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    at = 0
    for b, n in enumerate(lens):
        c["page_table"][b, :n // ps] = perm[at:at + n // ps]
        at += n // ps
    c["refcount"][perm[:at].long()] = 1
    c["free_list"][:n_pages - at] = perm[at:]
    c["free_list"][n_pages - at:] = -1
    c["n_free"].fill_(n_pages - at)
    c["kv_len"][:len(lens)] = torch.tensor(lens, dtype=torch.int32, device=DEV)


def _spread(n):
    """n fractions in [0, 1), the same for every seed (the sizes of a case's arrays follow from it alone)."""
    return [(0.37 + 0.6180339887 * b) % 1.0 for b in range(n)]


def _lengths(B, P, ragged):
    if not ragged:
        return [P] * B
    return [P if b == 0 else int(P * (0.3 + 0.7 * x)) for b, x in enumerate(_spread(B))]


def _trees(B, M, g):
    """Random trees: parent[i] < i, bushier near the root; -1 for the root."""
    u = torch.rand(B, M, generator=g, device=DEV)
    i = torch.arange(M, device=DEV)
    par = (u * u * i).floor().to(torch.int32)
    par[:, 0] = -1
    return torch.minimum(par, (i - 1).to(torch.int32))


def _paths(B, M, g):
    """Accepted paths: n_acc node numbers, ascending, among the M - 1 nodes below the root."""
    n = (torch.rand(B, generator=g, device=DEV) * (min(MAX_DEPTH, M - 1) + 1)).floor().to(torch.int32)
    idx = torch.full((B, MAX_DEPTH), -1, dtype=torch.int32, device=DEV)
    if M > 1:
        k = min(MAX_DEPTH, M - 1)
        pick = torch.rand(B, M - 1, generator=g, device=DEV).argsort(1)[:, :k] + 1
        # the n_acc first picks, in ascending order
        live = torch.arange(k, device=DEV)[None] < n[:, None]
        pick = torch.where(live, pick, torch.full_like(pick, 1 << 20)).sort(1).values
        idx[:, :k] = torch.where(live, pick, torch.full_like(pick, -1)).to(torch.int32)
    return n, idx


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed) * 7919 + 11)
    s = {"case": dict(case)}
    kind = case["kind"]
    if kind == "sample":
        R, V = case["R"], case["V"]
        # a language model's rows: a wide normal body and a handful of likely tokens
        z = case["spread"] * torch.randn(R, V, generator=g, device=DEV)
        hot = torch.randint(0, V, (R, 12), generator=g, device=DEV)
        z.scatter_(1, hot, 3.0 * case["spread"] + 3.0 * torch.rand(R, 12, generator=g, device=DEV))
        s["logits"] = z.to(_tdtype(case["dtype"]))
        s["temperature"] = 0.6 + 0.8 * torch.rand(R, generator=g, device=DEV)
        s["top_k"] = torch.full((R,), case["top_k"], dtype=torch.int32, device=DEV)
        s["top_p"] = torch.full((R,), case["top_p"], device=DEV)
        s["min_p"] = torch.full((R,), case["min_p"], device=DEV)
        s["u"] = torch.rand(R, generator=g, device=DEV)
        s["tok"] = torch.empty(R, dtype=torch.int32, device=DEV)
        s["out"] = torch.empty(R, V, device=DEV) if case["filtered"] else None
        if own:
            s["ctx"] = _context(1, 1, 64, 1, 1, "f32", V)
        return s
    d, ps, Hkv, L = case["d"], case["ps"], case["Hkv"], case.get("L", 1)
    dtype = case.get("dtype", "bf16")
    T = _tdtype(dtype)
    if kind == "attn":
        B, M, Hq = case["B"], case["M"], case["Hq"]
        lens = _lengths(B, case["P"], case["ragged"])
        c = _new_cache(1, max(1, sum(n // ps for n in lens) + 3), ps, B, max(1, case["P"] // ps + 1), Hkv, d, dtype)
        _fill_pages(c, g, "all")
        _give_pages(c, lens, g)
        s["q"] = torch.randn(B, M, Hq, d, generator=g, device=DEV).to(T)
        s["k_tree"] = torch.randn(B, Hkv, M, d, generator=g, device=DEV).to(T)
        s["v_tree"] = torch.randn(B, Hkv, M, d, generator=g, device=DEV).to(T)
        s["parent"] = _trees(B, M, g)
        s["out"] = torch.empty_like(s["q"])
        if own:
            s["ctx"] = _context(Hq, Hkv, d, B, M, dtype)
    elif kind == "commit":
        B, M = case["B"], case["M"]
        n_acc, acc_idx = _paths(B, M, g)
        lens = [max(0, case["P"] - int(x * (ps + 8))) for x in _spread(B)]
        c = _new_cache(L, sum(n // ps for n in lens) + 2 * B + 3, ps, B, case["P"] // ps + 3, Hkv, d, dtype)
        _fill_pages(c, g, "one")
        _give_pages(c, lens, g)
        c["kv_len"].add_(1 + n_acc)                    # the acceptance walk has counted the path already
        s["k_tree"] = [_randn_like(torch.empty(B, Hkv, M, d, dtype=T, device=DEV), g) for _ in range(L)]
        s["v_tree"] = [_randn_like(torch.empty(B, Hkv, M, d, dtype=T, device=DEV), g) for _ in range(L)]
        s["n_acc"], s["acc_idx"] = n_acc, acc_idx
        s["k_ptrs"], s["v_ptrs"] = _ptrs(s["k_tree"]), _ptrs(s["v_tree"])
        if own:
            s["ctx"] = _context(Hkv, Hkv, d, B, M, dtype)
    elif kind == "import":
        B, P = case["B"], case["P"]
        lens = _lengths(B, P, case["ragged"])
        c = _new_cache(L, sum(n // ps for n in lens) + 5, ps, B, P // ps + 1, Hkv, d, dtype)
        s["k_src"] = [_randn_like(torch.empty(B, Hkv, P, d, dtype=T, device=DEV), g) for _ in range(L)]
        s["v_src"] = [_randn_like(torch.empty(B, Hkv, P, d, dtype=T, device=DEV), g) for _ in range(L)]
        s["n_tokens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
        s["k_ptrs"], s["v_ptrs"] = _ptrs(s["k_src"]), _ptrs(s["v_src"])
        if own:
            s["ctx"] = _context(Hkv, Hkv, d, B, 1, dtype)
    elif kind == "fork":
        n_src, n_fork, P = case["n_src"], case["n_fork"], case["P"]
        lens = [max(1, P - 5 * b) for b in range(n_src)]
        c = _new_cache(L, sum(n // ps for n in lens) + 3, ps, n_src + n_fork, P // ps + 1, Hkv, d, dtype)
        _fill_pages(c, g, "one")
        _give_pages(c, lens, g)
        s["src"] = torch.randint(0, n_src, (n_fork,), generator=g, device=DEV).to(torch.int32)
        s["dst"] = (n_src + torch.randperm(n_fork, generator=g, device=DEV)).to(torch.int32)
        s["gone"] = s["dst"].flip(0).contiguous()
        if own:
            s["ctx"] = _context(Hkv, Hkv, d, 1, 1, dtype)
    elif kind == "compact":
        n_seq, P = case["n_seq"], case["P"]
        lens = [max(1, int(P * (0.5 + 0.5 * x))) for x in _spread(n_seq)]
        c = _new_cache(L, sum(n // ps for n in lens) + 7, ps, n_seq, P // ps + 1, Hkv, d, dtype)
        _fill_pages(c, g, "one")
        _give_pages(c, lens, g)
        s["gone"] = torch.randperm(n_seq, generator=g, device=DEV)[:case["n_gone"]].to(torch.int32)
        s["book"] = c["book"].clone()                  # the bookkeeping as it was, for every further pass
        s["n_moved"] = torch.zeros(1, dtype=torch.int32, device=DEV)
        if own:
            s["ctx"] = _context(Hkv, Hkv, d, 1, 1, dtype)
    else:                                              # copy: pages to another pool (swapped out, or moved)
        n = case["n_copy"]
        c = _new_cache(L, n + 9, ps, 1, 1, Hkv, d, dtype)
        _fill_pages(c, g, "one")
        s["to"] = _new_cache(L, n + 2, ps, 1, 1, Hkv, d, dtype)
        s["src"] = torch.randperm(n + 9, generator=g, device=DEV)[:n].to(torch.int32)
        s["dst"] = torch.randperm(n + 2, generator=g, device=DEV)[:n].to(torch.int32)
        if own:
            s["ctx"] = _context(Hkv, Hkv, d, 1, 1, dtype)
            s["to_handle"] = _handle(s["ctx"], s["to"])
    s["cache"] = c
    if own:
        s["handle"] = _handle(s["ctx"], c)
    return s


def _ptrs(ts):
    return torch.tensor([t.data_ptr() for t in ts], dtype=torch.int64, device=DEV)


def _context(Hq, Hkv, d, B, M, dtype, vocab=8):
    from paper_2502_06282_b200 import binding
    return binding.Context(hidden=8, n_experts=1, top_k=1, inter=8, vocab=vocab, n_q_heads=Hq, n_kv_heads=Hkv,
                           head_dim=d, max_batch=B, max_tree=M, max_depth=MAX_DEPTH, max_frontier=1,
                           k_per_expert=1, dtype=dtype)


def _handle(ctx, c):
    from paper_2502_06282_b200 import binding
    names = ("k_pages", "v_pages", "k_scale", "v_scale", "k_open", "v_open", "kv_len", "page_table", "refcount",
             "free_list", "n_free")
    return binding.PagedCache.from_tensors(ctx, {n: c[n] for n in names})


# --------------------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------------------
def run(s):
    return {"attn": _run_attn, "commit": _run_commit, "import": _run_import, "fork": _run_fork,
            "compact": _run_compact, "copy": _run_copy, "sample": _run_sample}[s["case"]["kind"]](s)


def _cache_values(c):
    """The updated cache: codes as the 8-bit floats they are, scales, open rows, bookkeeping."""
    return {"k_pages": c["k_pages"].view(E4M3), "v_pages": c["v_pages"].view(E4M3), "k_scale": c["k_scale"],
            "v_scale": c["v_scale"], "k_open": c["k_open"], "v_open": c["v_open"], "kv_len": c["kv_len"],
            "page_table": c["page_table"], "refcount": c["refcount"], "n_free": c["n_free"]}


def _ancestors(parent):
    """[B, M, M] truth values: column j is row i itself or one of its ancestors."""
    B, M = parent.shape
    up = torch.zeros(B, M, M + 1, device=parent.device, dtype=torch.float64)
    up.scatter_(2, torch.where(parent < 0, torch.full_like(parent, M), parent).long()[..., None], 1.0)
    up = up[..., :M]
    # (1 + N)^127 of the parent step N is positive exactly where a path of at most 127 steps leads
    step = torch.eye(M, device=parent.device, dtype=torch.float64) + up
    return torch.linalg.matrix_power(step, 127) > 0


def _run_attn(s):
    case, c = s["case"], s["cache"]
    B, M, Hq, Hkv, d, ps = (case[k] for k in ("B", "M", "Hq", "Hkv", "d", "ps"))
    scale = 1.0 / math.sqrt(d)
    if own:
        s["ctx"].tree_verify_attn_paged(s["handle"], 0, B, M, s["q"], s["k_tree"], s["v_tree"], s["parent"], scale,
                                      s["out"])
        return s["out"]
    G = Hq // Hkv
    n = c["kv_len"][:B]
    nf = n // ps * ps
    T = c["page_table"].shape[1]
    ids = c["page_table"][:B].clamp(min=0).long()
    inside = torch.arange(T * ps, device=DEV)[None] < nf[:, None]            # [B, T ps]
    keys, values = (_rows(c[x + "_pages"][0], c[x + "_scale"][0], ids) for x in "kv")
    at = torch.arange(ps, device=DEV)
    opened = (nf[:, None] + at) % (2 * ps)                                    # rows of the open page
    o_in = at[None] < (n - nf)[:, None]
    pick = opened[:, None, :, None].expand(B, Hkv, ps, d)
    keys = torch.cat([keys, c["k_open"][0, :B].gather(2, pick).float(), s["k_tree"].float()], 2)
    values = torch.cat([values, c["v_open"][0, :B].gather(2, pick).float(), s["v_tree"].float()], 2)
    seen = torch.cat([inside, o_in], 1)[:, None].expand(B, M, T * ps + ps)
    seen = torch.cat([seen, _ancestors(s["parent"])], 2)                      # [B, M, columns]
    values = torch.where(seen.any(1)[:, None, :, None], values, torch.zeros((), device=DEV))
    q = s["q"].float().view(B, M, Hkv, G, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * M, d)
    z = (q @ keys.transpose(2, 3)) * scale
    z = z.view(B, Hkv, G, M, -1).masked_fill(~seen[:, None, None], -math.inf)
    p = torch.exp(z - z.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    o = p.reshape(B, Hkv, G * M, -1) @ values
    return o.view(B, Hkv, G, M, d).permute(0, 3, 1, 2, 4).reshape(B, M, Hq, d).to(s["q"].dtype)


def _rows(pages, scale, ids):
    """The rows of the pages `ids` [B, T] as numbers: [B, Hkv, T ps, d] in 32 bits."""
    B, T = ids.shape
    Hkv, ps, d = pages.shape[1:]
    x = pages[ids].view(E4M3).float() * scale[ids][..., None, None]
    return x.permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * ps, d)


def _take_pages(c, need):
    """Page numbers for the places `need` [n, 2] (row, column) of the table that have none: from the end of the
    free list on, in the order of the places."""
    have = c["page_table"][need[:, 0], need[:, 1]]
    new = have < 0
    order = torch.cumsum(new.int(), 0) - 1
    ids = torch.where(new, c["free_list"][(c["n_free"].long() - 1 - order).clamp(min=0)], have)
    c["page_table"][need[:, 0], need[:, 1]] = ids
    c["refcount"][ids.long()] = 1
    c["n_free"].sub_(new.sum().to(torch.int32))
    return ids.long()


def _run_commit(s):
    case, c = s["case"], s["cache"]
    B, M, ps, L = case["B"], case["M"], case["ps"], case["L"]
    if own:
        s["ctx"].paged_commit(s["handle"], B, M, s["k_ptrs"], s["v_ptrs"], s["k_tree"][0].stride(0),
                            s["k_tree"][0].stride(1), s["n_acc"], s["acc_idx"])
        return _cache_values(c)
    n = c["kv_len"][:B]
    old = n - 1 - s["n_acc"]
    rows = torch.cat([torch.zeros(B, 1, dtype=torch.int32, device=DEV), s["acc_idx"]], 1)     # root, then the path
    b, j = torch.nonzero(torch.arange(MAX_DEPTH + 1, device=DEV)[None] <= s["n_acc"][:, None], as_tuple=True)
    node, place = rows[b, j].long(), ((old[b] + j) % (2 * ps)).long()
    need = torch.nonzero((torch.arange(c["page_table"].shape[1], device=DEV)[None] >= (old // ps)[:, None]) &
                         (torch.arange(c["page_table"].shape[1], device=DEV)[None] < (n // ps)[:, None]))
    ids = _take_pages(c, need)
    half = (need[:, 1] % 2)[:, None] * ps + torch.arange(ps, device=DEV)
    for x in "kv":
        tree = torch.stack(s[x + "_tree"])
        c[x + "_open"][:, b, :, place] = tree[:, b, :, node]
        block = c[x + "_open"][:, need[:, 0][:, None], :, half]               # [pages, ps, L, Hkv, d]
        q, scale = _quantise(block.permute(2, 0, 3, 1, 4))
        c[x + "_pages"][:, ids] = q.view(torch.uint8)
        c[x + "_scale"][:, ids] = scale
    return _cache_values(c)


def _run_import(s):
    case, c = s["case"], s["cache"]
    B, P, ps, L = case["B"], case["P"], case["ps"], case["L"]
    if own:
        src = s["k_src"][0]
        s["ctx"].paged_import(s["handle"], B, s["n_tokens"], 0, L, s["k_ptrs"], s["v_ptrs"], src.stride(0),
                            src.stride(1), P)
        return _cache_values(c)
    n = s["n_tokens"]
    need = torch.nonzero(torch.arange(c["page_table"].shape[1], device=DEV)[None] < (n // ps)[:, None])
    ids = _take_pages(c, need)
    rest = torch.arange(ps, device=DEV)[None] < (n % ps)[:, None]
    b, j = torch.nonzero(rest, as_tuple=True)
    pos = (n // ps * ps)[b] + j
    full = need[:, 1][:, None] * ps + torch.arange(ps, device=DEV)
    for x in "kv":
        src = torch.stack(s[x + "_src"])
        c[x + "_open"][:, b, :, pos % (2 * ps)] = src[:, b, :, pos]
        q, scale = _quantise(src[:, need[:, 0][:, None], :, full].permute(2, 0, 3, 1, 4))
        c[x + "_pages"][:, ids] = q.view(torch.uint8)
        c[x + "_scale"][:, ids] = scale
    c["kv_len"][:B] = n
    return _cache_values(c)


def _free(c, gone):
    gone = gone.long()
    ids = c["page_table"][gone]
    ids = ids[ids >= 0].long()
    before = c["refcount"].clone()
    c["refcount"].index_add_(0, ids, torch.full_like(ids, -1).to(torch.int32))
    empty = torch.nonzero((before > 0) & (c["refcount"] == 0))[:, 0].to(torch.int32)
    c["free_list"][c["n_free"].long() + torch.arange(empty.numel(), device=DEV)] = empty
    c["n_free"].add_(empty.numel())
    c["page_table"][gone] = -1
    c["kv_len"][gone] = 0


def _run_fork(s):
    case, c = s["case"], s["cache"]
    ps = case["ps"]
    if own:
        s["ctx"].paged_fork(s["handle"], s["src"], s["dst"])
        forked = c["page_table"].clone(), c["kv_len"].clone()
        s["ctx"].paged_free(s["handle"], s["gone"])
    else:
        src, dst = s["src"].long(), s["dst"].long()
        c["page_table"][dst] = c["page_table"][src]
        c["kv_len"][dst] = c["kv_len"][src]
        ids = c["page_table"][dst]
        ids = ids[ids >= 0].long()
        c["refcount"].index_add_(0, ids, torch.ones_like(ids).to(torch.int32))
        n = c["kv_len"][src]
        i, j = torch.nonzero(torch.arange(ps, device=DEV)[None] < (n % ps)[:, None], as_tuple=True)
        row = (n // ps * ps)[i] % (2 * ps) + j
        for x in "kv":
            c[x + "_open"][:, dst[i], :, row] = c[x + "_open"][:, src[i], :, row]
        forked = c["page_table"].clone(), c["kv_len"].clone()
        _free(c, s["gone"])
    return {"forked": forked, "cache": _cache_values(c)}


def _run_compact(s):
    case, c = s["case"], s["cache"]
    c["book"].copy_(s["book"])
    if own:
        s["ctx"].paged_free(s["handle"], s["gone"])
        s["ctx"].paged_compact(s["handle"], s["n_moved"])
        return {"n_moved": s["n_moved"], "cache": _cache_values(c), "free_list": _live(c)}
    _free(c, s["gone"])
    n_pages = c["refcount"].numel()
    ids = torch.arange(n_pages, device=DEV)
    live = c["refcount"] > 0
    n_live = live.sum()
    src = torch.nonzero(live & (ids >= n_live))[:, 0]
    dst = torch.nonzero(~live & (ids < n_live))[:, 0]
    to = ids.clone()
    to[src] = dst
    for x in ("k_pages", "v_pages", "k_scale", "v_scale"):
        c[x][:, dst] = c[x][:, src]
    c["refcount"][dst] = c["refcount"][src]
    c["refcount"][src] = 0
    t = c["page_table"]
    t.copy_(torch.where(t >= 0, to[t.clamp(min=0).long()].to(torch.int32), t))
    c["free_list"].copy_(torch.where(ids < n_pages - n_live, n_pages - 1 - ids, -1))
    c["n_free"].copy_(n_pages - n_live)
    s["n_moved"].fill_(src.numel())
    return {"n_moved": s["n_moved"], "cache": _cache_values(c), "free_list": _live(c)}


def _live(c):
    """The entries of the free list that count."""
    at = torch.arange(c["free_list"].numel(), device=DEV)
    return torch.where(at < c["n_free"], c["free_list"], -1)


def _run_copy(s):
    c, to = s["cache"], s["to"]
    if own:
        s["ctx"].paged_copy(s["handle"], s["to_handle"], s["src"], s["dst"])
    else:
        src, dst = s["src"].long(), s["dst"].long()
        for x in ("k_pages", "v_pages", "k_scale", "v_scale"):
            to[x][:, dst] = c[x][:, src]
    return {x: to[x].view(E4M3) if "pages" in x else to[x] for x in ("k_pages", "v_pages", "k_scale", "v_scale")}


def _run_sample(s):
    if own:
        s["ctx"].sample(s["logits"], s["temperature"], s["top_k"], s["top_p"], s["min_p"], s["u"], s["tok"], s["out"])
        return {"token": s["tok"], "filtered": s["out"]}
    R, V = s["logits"].shape
    T = s["temperature"].double()[:, None]
    z, order = s["logits"].float().sort(dim=1, descending=True, stable=True)      # ties: the lower index first
    x = (z.double() - z[:, :1].double()) / T
    w = torch.exp(x)
    k = torch.where(s["top_k"] > 0, s["top_k"], torch.full_like(s["top_k"], V)).clamp(max=V)[:, None]
    rank = torch.arange(V, device=DEV)[None]
    w = torch.where(rank < k, w, torch.zeros_like(w))
    before = torch.cumsum(w, 1) - w
    top_p = s["top_p"].double()[:, None]
    keep = (rank < k) & ((before < top_p * w.sum(1, keepdim=True)) | (top_p >= 1))
    keep &= (z.double() - z[:, :1].double() >= T * torch.log(s["min_p"].double())[:, None]) | (rank == 0)
    keep |= rank == 0
    kept = torch.zeros(R, V, dtype=torch.bool, device=DEV).scatter_(1, order, keep)
    w = torch.zeros(R, V, dtype=torch.float64, device=DEV).scatter_(1, order, w * keep)
    cdf = torch.cumsum(w, 1)
    hit = (cdf > s["u"].double()[:, None] * cdf[:, -1:]) & kept
    tok = hit.int().argmax(1).to(torch.int32)
    out = None
    if s["out"] is not None:
        out = torch.where(kept, s["logits"].float() / s["temperature"][:, None], -math.inf)
    return {"token": tok, "filtered": out}


# --------------------------------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------------------------------
def work(case):
    kind, d = case["kind"], case.get("d", 0)
    w = 4 if case.get("dtype") == "f32" else 2
    if kind == "sample":
        R, V = case["R"], case["V"]
        return {"bytes": R * V * (w + (4 if case["filtered"] else 0)) + 24 * R, "flops": 12 * R * V}
    ps, Hkv, L = case["ps"], case["Hkv"], case.get("L", 1)
    page = 2 * Hkv * (ps * d + 4)                                             # K and V of a page with scales
    if kind == "attn":
        B, M, Hq = case["B"], case["M"], case["Hq"]
        lens = _lengths(B, case["P"], case["ragged"])
        pages, rest = sum(n // ps for n in lens), sum(n % ps for n in lens)
        return {"bytes": pages * (page + 4) + (rest + B * M) * 2 * Hkv * d * w + 2 * B * M * Hq * d * w,
                "flops": 4 * M * Hq * d * sum(n + M for n in lens)}
    if kind == "commit":
        B = case["B"]
        rows = 1 + min(MAX_DEPTH, case["M"] - 1) / 2
        full = rows / ps                                                      # pages completed per sequence
        return {"bytes": int(L * B * (rows * 4 * Hkv * d * w + full * (page + 2 * Hkv * (ps - rows) * d * w))),
                "flops": int(L * B * full * 4 * Hkv * ps * d)}
    if kind == "import":
        lens = _lengths(case["B"], case["P"], case["ragged"])
        n, pages = sum(lens), sum(x // ps for x in lens)
        return {"bytes": int(L * (n * 2 * Hkv * d * w + pages * page + (n - pages * ps) * 2 * Hkv * d * w)),
                "flops": int(L * n * 4 * Hkv * d)}
    if kind == "fork":
        n, P = case["n_fork"], case["P"]
        return {"bytes": int(n * (L * (P % ps) * 4 * Hkv * d * 2 + (P // ps) * 16)), "flops": int(n * (P // ps))}
    if kind == "compact":
        n, gone, P = case["n_seq"], case["n_gone"], case["P"]
        total = n * 0.75 * P / ps
        live = total * (1 - gone / n)
        moved = live * (gone / n)                                             # live pages above the cut
        return {"bytes": int(2 * L * moved * page + 24 * total), "flops": int(total)}
    return {"bytes": int(2 * L * case["n_copy"] * page), "flops": 0}


# --------------------------------------------------------------------------------------------------
# the definitions in 64 bits, one sequence or row at a time
# --------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "attn":
        return _exact_attn(s)
    if kind == "sample":
        return _exact_sample(s)
    if kind == "commit":
        return _exact_commit(s)
    if kind == "import":
        return _exact_import(s)
    return None                                        # bookkeeping and copies: every output is exact already


def _exact_attn(s):
    case, c = s["case"], s["cache"]
    M, Hq, Hkv, d, ps = (case[k] for k in ("M", "Hq", "Hkv", "d", "ps"))
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    parents = s["parent"].tolist()
    lens = c["kv_len"].tolist()
    for b in range(case["B"]):
        n, nf = lens[b], lens[b] // ps
        mask = torch.zeros(M, n + M, dtype=torch.bool, device=DEV)
        mask[:, :n] = True
        rows = []
        for i, p in enumerate(parents[b]):
            rows.append((rows[p] if p >= 0 else []) + [i])
        at = torch.tensor([(i, n + j) for i, r in enumerate(rows) for j in r], device=DEV)
        mask[at[:, 0], at[:, 1]] = True
        ids = c["page_table"][b, :nf].long()
        r0 = (nf % 2) * ps
        for h in range(Hkv):
            kv = []
            for x in "kv":
                paged = c[x + "_pages"][0, ids, h].view(E4M3).double() * c[x + "_scale"][0, ids, h].double()[:, None, None]
                kv.append(torch.cat([paged.reshape(nf * ps, d), c[x + "_open"][0, b, h, r0:r0 + n - nf * ps].double(),
                                     s[x + "_tree"][b, h].double()]))
            for g in range(Hq // Hkv):
                q = s["q"][b, :, h * (Hq // Hkv) + g].double()
                z = (q @ kv[0].T / math.sqrt(d)).masked_fill(~mask, -math.inf)
                out[b, :, h * (Hq // Hkv) + g] = torch.softmax(z, 1) @ kv[1]
    return out


def _exact_blocks(x):
    """[..., ps, d] -> the codes' values in 64 bits and the scale: code grid of 4 significant bits, steps of
    2^-9 at the bottom."""
    x = x.double()
    amax = x.abs().amax((-2, -1))
    e = torch.ceil(torch.log2(amax / 448.0)).clamp(min=-32)
    e = torch.where(amax > 0, e, torch.full_like(e, -32))
    scale = torch.exp2(e)
    y = x / scale[..., None, None]
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step, scale


def _exact_cache(s, x, values, at, scales):
    c = s["cache"]
    v = c[x + "_pages"].view(E4M3).to(torch.float32)
    sc = c[x + "_scale"].double()
    if len(at):
        v[:, at] = values.float()                      # 4 significant bits: exact in 32
        sc[:, at] = scales
    return v.double() if v.numel() < (1 << 28) else None, sc


def _exact_commit(s):
    case, c = s["case"], s["cache"]
    B, ps, L = case["B"], case["ps"], case["L"]
    if L * c["k_pages"].shape[1] * case["Hkv"] * ps * case["d"] > 1 << 31:
        return None
    lens, acc, path = c["kv_len"].tolist(), s["n_acc"].tolist(), s["acc_idx"].tolist()
    out = {}
    for x in "kv":
        opened = c[x + "_open"].double()
        tree = s[x + "_tree"]
        for b in range(B):
            for j in range(1 + acc[b]):
                node = 0 if j == 0 else path[b][j - 1]
                pos = lens[b] - 1 - acc[b] + j
                opened[:, b, :, pos % (2 * ps)] = torch.stack([t[b, :, node].double() for t in tree])
        at, blocks, taken = [], [], int(c["n_free"][0])
        for b in range(B):
            for t in range((lens[b] - 1 - acc[b]) // ps, lens[b] // ps):
                taken -= 1
                at.append(int(c["free_list"][taken]))
                blocks.append(opened[:, b, :, (t % 2) * ps:(t % 2) * ps + ps])
        v, sc = _exact_blocks(torch.stack(blocks, 1)) if at else (None, None)
        out[x + "_pages"], out[x + "_scale"] = _exact_cache(s, x, v, at, sc)
        out[x + "_open"] = opened
    return {**{k: out[k] for k in out}, "kv_len": None, "page_table": None, "refcount": None, "n_free": None}


def _exact_import(s):
    case, c = s["case"], s["cache"]
    ps, L = case["ps"], case["L"]
    if L * c["k_pages"].shape[1] * case["Hkv"] * ps * case["d"] > 1 << 31:
        return None
    lens = s["n_tokens"].tolist()
    out = {}
    for x in "kv":
        opened = c[x + "_open"].double()
        at, taken = [], int(c["n_free"][0])
        for b in range(case["B"]):
            n = lens[b]
            for t in range(n // ps):
                taken -= 1
                at.append(int(c["free_list"][taken]))
            for pos in range(n // ps * ps, n):
                opened[:, b, :, pos % (2 * ps)] = torch.stack([t[b, :, pos].double() for t in s[x + "_src"]])
        values, scales = [], []
        for layer in range(L):
            rows = torch.cat([s[x + "_src"][layer][b, :, :lens[b] // ps * ps].unflatten(1, (-1, ps)).transpose(0, 1)
                              for b in range(case["B"]) if lens[b] >= ps] or [torch.zeros(0)])
            if at:
                v, sc = _exact_blocks(rows)
                values.append(v.float())
                scales.append(sc)
        out[x + "_pages"], out[x + "_scale"] = _exact_cache(s, x, torch.stack(values) if at else None, at,
                                                            torch.stack(scales) if at else None)
        out[x + "_open"] = opened
    return {**out, "kv_len": None, "page_table": None, "refcount": None, "n_free": None}


def _exact_sample(s):
    R, V = s["logits"].shape
    toks, rows = [], []
    for r in range(R):
        z = s["logits"][r].double()
        T = s["temperature"][r].double()
        x = (z - z.max()) / T
        by = torch.sort(-x, stable=True).indices
        k = int(s["top_k"][r]) if int(s["top_k"][r]) > 0 else V
        first = by[:k]
        p = torch.softmax(x[first], 0)
        top_p = float(s["top_p"][r])
        n = len(first)
        if top_p < 1:
            n = min(n, int((torch.cumsum(p, 0) - p < top_p).sum()))
        min_p = float(s["min_p"][r])
        if min_p > 0:
            n = min(n, int((x[first] >= math.log(min_p)).sum()))
        first = first[:max(1, n)].sort().values
        cdf = torch.cumsum(torch.softmax(x[first], 0), 0)
        at = int((cdf <= s["u"][r].double() * cdf[-1]).sum())
        toks.append(int(first[min(at, len(first) - 1)]))
        if s["out"] is not None:
            row = torch.full((V,), -math.inf, dtype=torch.float64, device=DEV)
            row[first] = z[first] / T
            rows.append(row)
    return {"token": torch.tensor(toks, dtype=torch.int32, device=DEV), "filtered": torch.stack(rows) if rows else None}
