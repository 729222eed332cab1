"""ctypes binding of libjakiro.so: same entry points as include/jakiro.h.

Argument marshalling only.  Every arithmetic step runs in the CUDA kernels of
the library; torch is used for device memory and for the current stream.  If
the shared library has not been built the import of the library raises; there
is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, List, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libjakiro.so")

JK_F32, JK_BF16 = 0, 1
JK_OK = 0
ERR = {"NULL": -1, "SHAPE": -2, "ALIGN": -3, "DTYPE": -4, "CAPACITY": -5, "WORKSPACE": -6,
       "CUDA": -7, "TIMEOUT": -8, "BOUNDS": -9}

EXPORTS = ["jk_create", "jk_destroy", "jk_workspace_bytes", "jk_set_workspace", "jk_strerror",
           "jk_last_cuda_error", "jk_read_status", "jk_set_tensor_path", "jk_draft_expand",
           "jk_tree_finalize", "jk_tree_verify_attn", "jk_accept_and_compact",
           "jk_profile_enable", "jk_profile_collect", "jk_profile_stage_count",
           "jk_profile_stage_name", "jk_tree_verify_attn_static", "jk_tensor_path_active",
           "jk_set_attn_kernel", "jk_profile_read", "jk_draft_pre",
           "jk_verify_qkv", "jk_gather_accepted", "jk_paged_scratch_ints", "jk_paged_init",
           "jk_paged_import", "jk_tree_verify_attn_paged", "jk_verify_qkv_tree", "jk_paged_commit",
           "jk_paged_fork", "jk_paged_free", "jk_paged_compact", "jk_paged_copy", "jk_sample"]


class JkConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "hidden", "n_experts", "top_k", "inter", "vocab", "n_q_heads", "n_kv_heads", "head_dim",
        "max_batch", "max_tree", "max_depth", "max_frontier", "k_per_expert", "dtype")] + [
        ("rms_eps", C.c_float), ("use_pre_norm", C.c_int32), ("branch_residual", C.c_int32),
        ("head_mode", C.c_int32), ("contrast_alpha", C.c_float), ("contrast_beta", C.c_float)]


class JkDraftWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("router", "w_gate", "w_up", "w_down", "lm_head",
                                          "norm_weight")]


class JkPool(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("tok", "score", "parent", "qslot", "branch")] + [
        ("stride_b", C.c_int64)]


class JkPreWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("emb", "w_fc", "b_fc", "w_qkv", "w_o")]


class JkPreState(C.Structure):
    _fields_ = [("q", C.c_void_p), ("slot_parent", C.c_void_p), ("slot_depth", C.c_void_p),
                ("stride_b", C.c_int64)]


class JkPaged(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "n_pages", "page_size", "max_seqs",
                                         "max_pages")] + [
        (n, C.c_void_p) for n in ("k_pages", "v_pages", "k_scale", "v_scale", "k_open", "v_open",
                                  "kv_len", "page_table", "refcount", "free_list", "n_free",
                                  "scratch")]


_lib = None


def lib() -> C.CDLL:
    """The loaded shared library.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2502_06282_b200.build` "
                "(needs nvcc); there is no fallback implementation")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float
        L.jk_create.argtypes = [C.POINTER(vp), C.POINTER(JkConfig)]
        L.jk_destroy.argtypes = [vp]
        L.jk_workspace_bytes.argtypes = [vp]
        L.jk_workspace_bytes.restype = C.c_size_t
        L.jk_set_workspace.argtypes = [vp, vp, vp, C.c_size_t]
        L.jk_strerror.argtypes = [C.c_int]
        L.jk_strerror.restype = C.c_char_p
        L.jk_last_cuda_error.argtypes = [vp]
        L.jk_last_cuda_error.restype = C.c_char_p
        L.jk_read_status.argtypes = [vp, vp, C.POINTER(i32)]
        L.jk_set_tensor_path.argtypes = [vp, i32]
        L.jk_tensor_path_active.argtypes = [vp]
        L.jk_set_attn_kernel.argtypes = [vp, i32]
        L.jk_draft_expand.argtypes = [vp, vp, C.POINTER(JkDraftWeights), i32, i32, i32, vp, vp,
                                      vp, i32, i32, vp, vp, vp, C.POINTER(JkPool), vp, vp, vp,
                                      i64, vp, vp, vp, vp]
        L.jk_tree_finalize.argtypes = [vp, vp, i32, C.POINTER(JkPool), i32, vp, i32, vp, vp, vp,
                                       vp, vp, vp, vp]
        L.jk_tree_verify_attn.argtypes = [vp, vp, i32, i32, vp, vp, vp, i64, i64, i32, vp, vp,
                                          f32, vp]
        L.jk_tree_verify_attn_static.argtypes = L.jk_tree_verify_attn.argtypes + [vp]
        L.jk_accept_and_compact.argtypes = [vp, vp, i32, i32, i32, f32, vp, i32, vp, vp, vp, vp,
                                            vp, vp, i32, vp, vp, i32, vp, vp, i64, i64, i32, vp,
                                            vp, vp, vp, vp]
        L.jk_draft_pre.argtypes = [vp, vp, C.POINTER(JkPreWeights), C.POINTER(JkPreState), i32, i32,
                                   i32, vp, C.POINTER(JkPool), i32, i32, i32, vp, vp, vp, vp, i64,
                                   i64, i32, vp, f32, f32, vp]
        L.jk_verify_qkv.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, vp, vp, i64, i64, i32, vp, f32]
        L.jk_gather_accepted.argtypes = [vp, vp, i32, i32, vp, vp, vp, i32, vp]
        kv = C.POINTER(JkPaged)
        L.jk_paged_scratch_ints.argtypes = [i32]
        L.jk_paged_init.argtypes = [vp, vp, kv]
        L.jk_paged_import.argtypes = [vp, vp, kv, i32, vp, vp, i32, i32, vp, vp, i64, i64, i32]
        L.jk_tree_verify_attn_paged.argtypes = [vp, vp, kv, i32, i32, i32, vp, vp, vp, i64, i64, vp,
                                              f32, vp]
        L.jk_verify_qkv_tree.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, vp, vp, i64, i64, vp, f32]
        L.jk_paged_commit.argtypes = [vp, vp, kv, i32, i32, vp, vp, i64, i64, vp, vp]
        L.jk_paged_fork.argtypes = [vp, vp, kv, i32, vp, vp]
        L.jk_paged_free.argtypes = [vp, vp, kv, i32, vp]
        L.jk_paged_compact.argtypes = [vp, vp, kv, vp]
        L.jk_paged_copy.argtypes = [vp, vp, kv, kv, i32, vp, vp]
        L.jk_sample.argtypes = [vp, vp, i32, vp, i32, i64, vp, vp, vp, vp, vp, vp, vp]
        L.jk_profile_enable.argtypes = [vp, i32]
        L.jk_profile_collect.argtypes = [vp, vp, C.POINTER(f32), C.POINTER(i32)]
        L.jk_profile_read.argtypes = [vp, vp, C.POINTER(f32), C.POINTER(i32)]
        L.jk_profile_stage_count.argtypes = []
        L.jk_profile_stage_name.argtypes = [i32]
        L.jk_profile_stage_name.restype = C.c_char_p
        for name in EXPORTS:
            if name not in ("jk_workspace_bytes", "jk_strerror", "jk_last_cuda_error",
                            "jk_profile_stage_name", "jk_paged_scratch_ints"):
                getattr(L, name).restype = C.c_int
        L.jk_paged_scratch_ints.restype = i64
        _lib = L
    return _lib


class JakiroError(RuntimeError):
    def __init__(self, code: int, where: str, detail: str = ""):
        self.code = code
        msg = lib().jk_strerror(code).decode()
        super().__init__(f"{where}: {msg} ({code}) {detail}".strip())


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream() -> int:
    # (the handle alone: torch.cuda.current_stream() makes a Stream object, 3 us against 0.3)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _array(t: Optional[torch.Tensor], dtype: torch.dtype, n: int, name: str) -> Optional[int]:
    """The pointer of an array the library reads as n elements of one type in a row (None: not given)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() < n or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor of at least {n} elements")
    return t.data_ptr()


def _second_dim(n: int, **tensors):
    """Tensors of several rows of n: more dimensions than one, and a second one that is not n, would be read with a
    wrong distance between rows.  (A flat tensor is taken as it is.)"""
    for name, t in tensors.items():
        if t is not None and t.dim() > 1 and t.shape[1] != n:
            raise ValueError(f"{name}: the second dimension is {t.shape[1]}, not {n}")


def torch_dtype(dtype: str) -> torch.dtype:
    return torch.bfloat16 if dtype == "bf16" else torch.float32


class Context:
    """Owns a jk_ctx and its device workspace (a torch allocation)."""

    def __init__(self, *, hidden, n_experts, top_k, inter, vocab, n_q_heads, n_kv_heads,
                 head_dim, max_batch, max_tree, max_depth, max_frontier, k_per_expert, dtype,
                 rms_eps=1e-5, use_pre_norm=True, branch_residual=True, head_mode=0,
                 contrast_alpha=0.0, contrast_beta=1.0, device="cuda", allocate=True):
        self.cfg = JkConfig(hidden, n_experts, top_k, inter, vocab, n_q_heads, n_kv_heads,
                            head_dim, max_batch, max_tree, max_depth, max_frontier,
                            k_per_expert, JK_BF16 if dtype == "bf16" else JK_F32, rms_eps,
                            int(use_pre_norm), int(branch_residual), int(head_mode),
                            float(contrast_alpha), float(contrast_beta))
        self.dtype = dtype
        self.tdtype = torch_dtype(dtype)
        self.kv_kind = (n_kv_heads, head_dim, self.tdtype)     # what a paged cache has to hold
        self.q_row_bytes = n_q_heads * head_dim * self.tdtype.itemsize
        self._h = C.c_void_p()
        rc = lib().jk_create(C.byref(self._h), C.byref(self.cfg))
        if rc != JK_OK:
            self._h = C.c_void_p()
            raise JakiroError(rc, "jk_create")
        self.workspace = None
        self.device = device
        if allocate:
            n = lib().jk_workspace_bytes(self._h)
            self.workspace = torch.empty(n + 256, dtype=torch.uint8, device=device)
            base = (self.workspace.data_ptr() + 255) // 256 * 256
            self._check(lib().jk_set_workspace(self._h, _stream(), base, n), "jk_set_workspace")

    def set_workspace(self, buf: torch.Tensor, offset: int = 0):
        """jk_set_workspace on a caller-made uint8 device buffer: the workspace starts at the
        first 256-byte boundary at or after buf[offset]; the buffer must stay alive."""
        n = lib().jk_workspace_bytes(self._h)
        base = (buf.data_ptr() + offset + 255) // 256 * 256
        if base + n > buf.data_ptr() + buf.numel():
            raise ValueError("buffer too small for the workspace")
        self.workspace = buf
        self._check(lib().jk_set_workspace(self._h, _stream(), base, n), "jk_set_workspace")
        return base - buf.data_ptr()

    @classmethod
    def for_workload(cls, w, frontier_sizes=None, **kw) -> "Context":
        fs = w.frontier_sizes if frontier_sizes is None else frontier_sizes
        kw.setdefault("head_mode", getattr(w, "head_mode", 0))
        return cls(hidden=w.hidden, n_experts=w.n_experts, top_k=w.top_k, inter=w.inter,
                   vocab=w.vocab, n_q_heads=w.n_q_heads, n_kv_heads=w.n_kv_heads,
                   head_dim=w.head_dim, max_batch=w.batch, max_tree=w.tree_size,
                   max_depth=w.depth, max_frontier=max(fs),
                   k_per_expert=w.k_per_expert, dtype=w.dtype, **kw)

    def _check(self, rc: int, where: str):
        if rc != JK_OK:
            detail = lib().jk_last_cuda_error(self._h).decode() if rc == ERR["CUDA"] else ""
            raise JakiroError(rc, where, detail)

    @property
    def workspace_bytes(self) -> int:
        return lib().jk_workspace_bytes(self._h)

    def close(self):
        if self._h:
            lib().jk_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_attn_kernel(self, mode: int):
        self._check(lib().jk_set_attn_kernel(self._h, int(mode)), "jk_set_attn_kernel")

    def set_tensor_path(self, enable: bool):
        self._check(lib().jk_set_tensor_path(self._h, int(enable)), "jk_set_tensor_path")

    @property
    def tensor_path_active(self) -> bool:
        return bool(lib().jk_tensor_path_active(self._h))

    def read_status(self) -> int:
        out = C.c_int32(0)
        self._check(lib().jk_read_status(self._h, _stream(), C.byref(out)), "jk_read_status")
        return out.value

    def profile_enable(self, max_launches: int):
        self._check(lib().jk_profile_enable(self._h, max_launches), "jk_profile_enable")

    def profile_collect(self, keep: bool = False) -> Dict[str, tuple]:
        """{stage name: (total ms, launches)} since the last collect; synchronises.  keep=True
        leaves the recorded event pairs in place (jk_profile_read), for graph replays."""
        n = lib().jk_profile_stage_count()
        ms = (C.c_float * n)()
        cnt = (C.c_int32 * n)()
        fn = lib().jk_profile_read if keep else lib().jk_profile_collect
        self._check(fn(self._h, _stream(), ms, cnt), "jk_profile_collect")
        return {lib().jk_profile_stage_name(i).decode(): (float(ms[i]), int(cnt[i]))
                for i in range(n) if cnt[i]}

    # ------------------------------------------------------------------ calls
    @staticmethod
    def weights_struct(w: Dict[str, torch.Tensor]) -> JkDraftWeights:
        return JkDraftWeights(_ptr(w["router"]), _ptr(w["w_gate"]), _ptr(w["w_up"]),
                              _ptr(w["w_down"]), _ptr(w["lm_head"]), _ptr(w.get("norm_weight")))

    @staticmethod
    def pool_struct(pool: Dict[str, torch.Tensor]) -> JkPool:
        return JkPool(_ptr(pool["tok"]), _ptr(pool["score"]), _ptr(pool["parent"]),
                      _ptr(pool["qslot"]), _ptr(pool["branch"]), pool["tok"].stride(0))

    def draft_expand(self, weights, batch, n_frontier, width, u, parent_score, parent_gidx,
                     gidx_base, slot_base, out_probs, out_expert, out_gate, pool, out_lse,
                     out_feat, out_logits, next_frontier, next_parent_score, next_parent_gidx,
                     static_select=None):
        ws = weights if isinstance(weights, JkDraftWeights) else self.weights_struct(weights)
        ps = pool if isinstance(pool, JkPool) else self.pool_struct(pool)
        rc = lib().jk_draft_expand(
            self._h, _stream(), C.byref(ws), batch, n_frontier, width, _ptr(u),
            _ptr(parent_score), _ptr(parent_gidx), gidx_base, slot_base, _ptr(out_probs),
            _ptr(out_expert), _ptr(out_gate), C.byref(ps), _ptr(out_lse), _ptr(out_feat),
            _ptr(out_logits), 0 if out_logits is None else out_logits.stride(0),
            _ptr(next_frontier), _ptr(next_parent_score),
            _ptr(next_parent_gidx), _ptr(static_select))
        self._check(rc, "jk_draft_expand")

    @staticmethod
    def pre_weights_struct(w: Dict[str, torch.Tensor]) -> JkPreWeights:
        return JkPreWeights(_ptr(w["emb"]), _ptr(w["w_fc"]), _ptr(w.get("b_fc")), _ptr(w["w_qkv"]),
                            _ptr(w["w_o"]))

    def draft_pre(self, pre_weights, state: JkPreState, batch, n_frontier, slot_base, node_gidx,
                  pool, prev_gidx_base, prev_slot_base, prev_frontier, prev_feat, root_tok, k_cache,
                  v_cache, kv_len, rope_theta, scale, out_u, cache_rows=None):
        ws = pre_weights if isinstance(pre_weights, JkPreWeights) else self.pre_weights_struct(pre_weights)
        ps = pool if isinstance(pool, JkPool) else self.pool_struct(pool)
        rows = k_cache.shape[2] if cache_rows is None else cache_rows
        rc = lib().jk_draft_pre(self._h, _stream(), C.byref(ws), C.byref(state), batch, n_frontier,
                                slot_base, _ptr(node_gidx), C.byref(ps), prev_gidx_base,
                                prev_slot_base, prev_frontier, _ptr(prev_feat), _ptr(root_tok),
                                _ptr(k_cache), _ptr(v_cache), k_cache.stride(0), k_cache.stride(1),
                                rows, _ptr(kv_len), float(rope_theta), float(scale), _ptr(out_u))
        self._check(rc, "jk_draft_pre")

    def verify_qkv(self, w_qkv, batch, tree_size, x, depth, q_out, k_cache, v_cache, kv_len,
                   rope_theta, cache_rows=None):
        rows = k_cache.shape[2] if cache_rows is None else cache_rows
        rc = lib().jk_verify_qkv(self._h, _stream(), _ptr(w_qkv), batch, tree_size, _ptr(x),
                                 _ptr(depth), _ptr(q_out), _ptr(k_cache), _ptr(v_cache),
                                 k_cache.stride(0), k_cache.stride(1), rows, _ptr(kv_len),
                                 float(rope_theta))
        self._check(rc, "jk_verify_qkv")

    def gather_accepted(self, batch, tree_size, hidden, n_acc, acc_idx, rows_out, out):
        rc = lib().jk_gather_accepted(self._h, _stream(), batch, tree_size, _ptr(hidden),
                                      _ptr(n_acc), _ptr(acc_idx), rows_out, _ptr(out))
        self._check(rc, "jk_gather_accepted")

    def _tree_arrays(self, k_tree, v_tree, batch, tree_size):
        """Strides of the tree tokens' K and V, T [>= batch, Hkv, >= tree_size, d]: one pair for both."""
        Hkv, d, T = self.kv_kind
        s, shape = k_tree.stride(), k_tree.shape
        if k_tree.dtype is T and v_tree.dtype is T and v_tree.shape == shape and len(shape) == 4:
            b, h, m, x = shape
            if b >= batch and h == Hkv and m >= tree_size and x == d:
                if v_tree.stride() == s and s[2] == d and s[3] == 1:
                    return s
                # (the stride of a dimension of one does not count)
                if s[3] == 1 and (s[2] == d or m == 1) and all(
                        p == r or n == 1 for p, r, n in zip(s, v_tree.stride(), shape)):
                    return s
                raise ValueError("k_tree and v_tree must have the same strides and dense rows")
        raise ValueError(f"k_tree, v_tree: expected {T} tensors of one shape, [batch, {Hkv}, tree rows, {d}]")

    def verify_qkv_tree(self, w_qkv, batch, tree_size, x, depth, q_out, k_tree, v_tree, kv_len,
                        rope_theta):
        """jk_verify_qkv_tree: as verify_qkv, K and V of node i at row i of k_tree / v_tree."""
        s = self._tree_arrays(k_tree, v_tree, batch, tree_size)
        if batch > 1:
            _second_dim(tree_size, x=x, depth=depth, q_out=q_out)
        n, c, T = batch * tree_size, self.cfg, self.tdtype
        rc = lib().jk_verify_qkv_tree(
            self._h, _stream(),
            _array(w_qkv, T, (c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim * c.hidden, "w_qkv"), batch, tree_size,
            _array(x, T, n * c.hidden, "x"), _array(depth, torch.int32, n, "depth"),
            _array(q_out, T, n * c.n_q_heads * c.head_dim, "q_out"), k_tree.data_ptr(), v_tree.data_ptr(), s[0], s[1],
            _array(kv_len, torch.int32, batch, "kv_len"), float(rope_theta))
        self._check(rc, "jk_verify_qkv_tree")

    def tree_verify_attn_paged(self, cache: "PagedCache", layer, batch, tree_size, q, k_tree, v_tree,
                             parent, scale, out):
        """q, out [batch, tree_size, Hq, d]; k_tree, v_tree [batch, Hkv, tree rows, d] with the same strides and dense
        rows; parent i32 [batch, tree_size] (i64 is converted)."""
        s = self._tree_arrays(k_tree, v_tree, batch, tree_size)
        if batch > 1:
            _second_dim(tree_size, q=q, parent=parent, out=out)
        T, n = self.tdtype, batch * tree_size
        if parent.dtype is not torch.int32 or parent.nbytes < 4 * n or not parent.is_contiguous():
            if parent.dtype is not torch.int64:
                raise ValueError("parent: expected a contiguous int32 tensor [batch, tree_size]")
            parent = parent.int()
            _array(parent, torch.int32, n, "parent")
        n *= self.q_row_bytes
        if (q.dtype is not T or out.dtype is not T or q.nbytes < n or out.nbytes < n or not q.is_contiguous()
                or not out.is_contiguous()):
            raise ValueError(f"q, out: expected contiguous {T} tensors [batch, tree_size, {self.cfg.n_q_heads}, {self.cfg.head_dim}]")
        rc = lib().jk_tree_verify_attn_paged(
            self._h, _stream(), cache.of(self), layer, batch, tree_size, q.data_ptr(), k_tree.data_ptr(),
            v_tree.data_ptr(), s[0], s[1], parent.data_ptr(), scale, out.data_ptr())
        if rc:
            self._check(rc, "jk_tree_verify_attn_paged")

    def paged_init(self, cache: "PagedCache"):
        self._check(lib().jk_paged_init(self._h, _stream(), cache.of(self)), "jk_paged_init")

    def paged_import(self, cache: "PagedCache", batch, n_tokens, first_layer, n_layers, k_ptrs, v_ptrs,
                   stride_b, stride_h, src_rows, seqs=None):
        """k_ptrs, v_ptrs: int64 device tensors of n_layers pointers to T [batch, Hkv, src_rows, d]."""
        rc = lib().jk_paged_import(self._h, _stream(), cache.of(self), batch,
                                 _array(seqs, torch.int32, batch, "seqs"),
                                 _array(n_tokens, torch.int32, batch, "n_tokens"), first_layer, n_layers,
                                 _array(k_ptrs, torch.int64, n_layers, "k_ptrs"),
                                 _array(v_ptrs, torch.int64, n_layers, "v_ptrs"), stride_b, stride_h, src_rows)
        self._check(rc, "jk_paged_import")

    def paged_commit(self, cache: "PagedCache", batch, tree_size, k_ptrs, v_ptrs, stride_b, stride_h,
                   n_acc, acc_idx):
        """k_ptrs, v_ptrs: int64 device tensors of n_layers pointers to the layers' tree arrays; n_acc i32 [batch],
        acc_idx i32 [batch, max_depth]."""
        if batch > 1:
            _second_dim(self.cfg.max_depth, acc_idx=acc_idx)
        rc = lib().jk_paged_commit(self._h, _stream(), cache.of(self), batch, tree_size,
                                 _array(k_ptrs, torch.int64, cache.n_layers, "k_ptrs"),
                                 _array(v_ptrs, torch.int64, cache.n_layers, "v_ptrs"), stride_b, stride_h,
                                 _array(n_acc, torch.int32, batch, "n_acc"),
                                 _array(acc_idx, torch.int32, batch * self.cfg.max_depth, "acc_idx"))
        self._check(rc, "jk_paged_commit")

    def paged_fork(self, cache: "PagedCache", src, dst):
        if src.numel() != dst.numel():
            raise ValueError("src and dst name different numbers of sequences")
        n = src.numel()
        rc = lib().jk_paged_fork(self._h, _stream(), cache.of(self), n, _array(src, torch.int32, n, "src"),
                               _array(dst, torch.int32, n, "dst"))
        self._check(rc, "jk_paged_fork")

    def paged_free(self, cache: "PagedCache", seqs):
        n = seqs.numel()
        rc = lib().jk_paged_free(self._h, _stream(), cache.of(self), n, _array(seqs, torch.int32, n, "seqs"))
        self._check(rc, "jk_paged_free")

    def paged_compact(self, cache: "PagedCache", n_moved=None):
        self._check(lib().jk_paged_compact(self._h, _stream(), cache.of(self),
                                         _array(n_moved, torch.int32, 1, "n_moved")), "jk_paged_compact")

    def paged_copy(self, src: "PagedCache", dst: "PagedCache", src_ids, dst_ids):
        if src_ids.numel() != dst_ids.numel():
            raise ValueError("src_ids and dst_ids name different numbers of pages")
        n = src_ids.numel()
        rc = lib().jk_paged_copy(self._h, _stream(), src.of(self), dst.of(self), n,
                                     _array(src_ids, torch.int32, n, "src_ids"),
                                     _array(dst_ids, torch.int32, n, "dst_ids"))
        self._check(rc, "jk_paged_copy")

    def sample(self, logits, temperature=None, top_k=None, top_p=None, min_p=None, u=None,
               out_tok=None, out_logits=None):
        """jk_sample on logits [rows, V] (f32 or bf16; rows may be strided).  The per-row arrays (f32 [rows], top_k
        i32) and the outputs (i32 [rows], f32 [rows, V]) are contiguous device tensors or None."""
        if logits.dim() != 2 or logits.shape[1] != self.cfg.vocab or (
                logits.shape[1] > 1 and logits.stride(1) != 1):
            raise ValueError("logits must be [rows, vocab] with contiguous rows")
        dt = {torch.bfloat16: JK_BF16, torch.float32: JK_F32}.get(logits.dtype, -1)
        stride = logits.stride(0) if logits.shape[0] > 1 else logits.shape[1]
        R, f32, i32 = logits.shape[0], torch.float32, torch.int32
        if R > 1:
            _second_dim(self.cfg.vocab, out_logits=out_logits)
        rc = lib().jk_sample(self._h, _stream(), R, logits.data_ptr(), dt, stride,
                             _array(temperature, f32, R, "temperature"), _array(top_k, i32, R, "top_k"),
                             _array(top_p, f32, R, "top_p"), _array(min_p, f32, R, "min_p"), _array(u, f32, R, "u"),
                             _array(out_tok, i32, R, "out_tok"),
                             _array(out_logits, f32, R * self.cfg.vocab, "out_logits"))
        self._check(rc, "jk_sample")

    def tree_finalize(self, batch, pool, pool_n, root_tok, tree_size, tok, parent, depth, branch,
                      qslot, anc, static_keep=None):
        ps = pool if isinstance(pool, JkPool) else self.pool_struct(pool)
        rc = lib().jk_tree_finalize(self._h, _stream(), batch, C.byref(ps), pool_n,
                                    _ptr(root_tok), tree_size, _ptr(tok), _ptr(parent),
                                    _ptr(depth), _ptr(branch), _ptr(qslot), _ptr(anc),
                                    _ptr(static_keep))
        self._check(rc, "jk_tree_finalize")

    def tree_verify_attn(self, batch, tree_size, q, k_cache, v_cache, kv_len, parent, scale, out,
                         cache_rows=None):
        rows = k_cache.shape[2] if cache_rows is None else cache_rows
        rc = lib().jk_tree_verify_attn(self._h, _stream(), batch, tree_size, _ptr(q),
                                       _ptr(k_cache), _ptr(v_cache), k_cache.stride(0),
                                       k_cache.stride(1), rows, _ptr(kv_len), _ptr(parent),
                                       float(scale), _ptr(out))
        self._check(rc, "jk_tree_verify_attn")

    def tree_verify_attn_static(self, batch, tree_size, q, k_cache, v_cache, kv_len, parent,
                                scale, out, status, cache_rows=None):
        """jk_tree_verify_attn_static: the same attention without any workspace, for callers
        that cannot allocate device memory; scratch is the library's built-in 8 MiB array.
        `status` is a caller-owned int32 device word (cleared by the caller) that receives
        JK_ERR_BOUNDS when a cache is too short."""
        rows = k_cache.shape[2] if cache_rows is None else cache_rows
        rc = lib().jk_tree_verify_attn_static(self._h, _stream(), batch, tree_size, _ptr(q),
                                              _ptr(k_cache), _ptr(v_cache), k_cache.stride(0),
                                              k_cache.stride(1), rows, _ptr(kv_len),
                                              _ptr(parent), float(scale), _ptr(out),
                                              _ptr(status))
        if rc != JK_OK:
            detail = lib().jk_last_cuda_error(self._h).decode()
            raise JakiroError(rc, "jk_tree_verify_attn_static", detail)

    def accept_and_compact(self, batch, tree_size, mode, temperature, target_logits, tree,
                           draft_logits, n_slots, u_accept, u_bonus, n_layers, k_ptrs, v_ptrs,
                           cache_stride_b, cache_stride_h, cache_rows, kv_len, n_acc, acc_idx,
                           acc_tok, bonus_tok):
        tl_dtype = JK_BF16 if target_logits.dtype == torch.bfloat16 else JK_F32
        rc = lib().jk_accept_and_compact(
            self._h, _stream(), batch, tree_size, mode, float(temperature), _ptr(target_logits),
            tl_dtype, _ptr(tree["tok"]), _ptr(tree["parent"]), _ptr(tree["depth"]),
            _ptr(tree["branch"]), _ptr(tree["qslot"]), _ptr(draft_logits), n_slots,
            _ptr(u_accept), _ptr(u_bonus), n_layers, _ptr(k_ptrs), _ptr(v_ptrs), cache_stride_b,
            cache_stride_h, cache_rows, _ptr(kv_len), _ptr(n_acc), _ptr(acc_idx), _ptr(acc_tok),
            _ptr(bonus_tok))
        self._check(rc, "jk_accept_and_compact")


class PagedCache:
    """A paged 8-bit KV cache (jk_paged): the device tensors, as attributes, and the descriptor that
    the calls take.  `PagedCache(ctx, ...)` allocates an empty one; `from_tensors` wraps tensors the
    caller already has."""

    _NAMES = ("k_pages", "v_pages", "k_scale", "v_scale", "k_open", "v_open", "kv_len",
              "page_table", "refcount", "free_list", "n_free")

    def __init__(self, ctx: Context, *, n_layers, n_pages, page_size, max_seqs, max_pages,
                 device="cuda"):
        Hkv, d = ctx.cfg.n_kv_heads, ctx.cfg.head_dim
        u8 = dict(dtype=torch.uint8, device=device)
        f32 = dict(dtype=torch.float32, device=device)
        i32 = dict(dtype=torch.int32, device=device)
        T = dict(dtype=ctx.tdtype, device=device)
        blocks = (n_layers, n_pages, Hkv)
        opened = (n_layers, max_seqs, Hkv, 2 * page_size, d)
        self._wrap(ctx, {
            "k_pages": torch.empty(*blocks, page_size, d, **u8),
            "v_pages": torch.empty(*blocks, page_size, d, **u8),
            "k_scale": torch.empty(*blocks, **f32), "v_scale": torch.empty(*blocks, **f32),
            "k_open": torch.empty(*opened, **T), "v_open": torch.empty(*opened, **T),
            "kv_len": torch.empty(max_seqs, **i32),
            "page_table": torch.empty(max_seqs, max_pages, **i32),
            "refcount": torch.empty(n_pages, **i32), "free_list": torch.empty(n_pages, **i32),
            "n_free": torch.empty(1, **i32)})
        ctx.paged_init(self)

    @classmethod
    def from_tensors(cls, ctx: Context, tensors: Dict[str, torch.Tensor]) -> "PagedCache":
        """The tensors of a cache under the names of jk_paged (without scratch), already filled."""
        self = cls.__new__(cls)
        self._wrap(ctx, tensors)
        return self

    def _wrap(self, ctx, t):
        L, n_pages, Hkv, ps, d = t["k_pages"].shape
        max_seqs, max_pages = t["page_table"].shape
        want = {"k_pages": ((L, n_pages, Hkv, ps, d), None), "v_pages": ((L, n_pages, Hkv, ps, d), None),
                "k_scale": ((L, n_pages, Hkv), torch.float32), "v_scale": ((L, n_pages, Hkv), torch.float32),
                "k_open": ((L, max_seqs, Hkv, 2 * ps, d), ctx.tdtype),
                "v_open": ((L, max_seqs, Hkv, 2 * ps, d), ctx.tdtype),
                "kv_len": ((max_seqs,), torch.int32), "page_table": ((max_seqs, max_pages), torch.int32),
                "refcount": ((n_pages,), torch.int32), "free_list": ((n_pages,), torch.int32),
                "n_free": ((1,), torch.int32)}
        if (Hkv, d) != (ctx.cfg.n_kv_heads, ctx.cfg.head_dim):
            raise ValueError("the pages' kv heads or head size are not the context's")
        for n in self._NAMES:
            shape, dtype = want[n]
            ok = t[n].element_size() == 1 if dtype is None else t[n].dtype == dtype
            if not ok or tuple(t[n].shape) != shape or not t[n].is_contiguous():
                raise ValueError(f"{n}: expected a contiguous {shape} tensor of its type")
            if t[n].device != t["k_pages"].device:
                raise ValueError(f"{n} is on another device than k_pages")
            setattr(self, n, t[n])
        self.page_size, self.n_pages, self.n_layers = ps, n_pages, L
        self.max_seqs, self.max_pages = max_seqs, max_pages
        ints = lib().jk_paged_scratch_ints(n_pages)
        self.scratch = torch.empty(max(1, ints), dtype=torch.int32, device=t["k_pages"].device)
        self.struct = JkPaged(L, n_pages, ps, max_seqs, max_pages,
                            *[t[n].data_ptr() for n in self._NAMES], self.scratch.data_ptr())
        self.ref = C.byref(self.struct)
        self.kind = ctx.kv_kind

    def of(self, ctx):
        """The descriptor, for a context of the same kv heads, head size and type."""
        if self.kind is not ctx.kv_kind and self.kind != ctx.kv_kind:
            raise ValueError("the cache was made for other kv heads, another head size or type")
        return self.ref


class StepBuffers:
    """Device buffers of one draft-and-verify step for a workload, allocated once."""

    def __init__(self, ctx: Context, w, keep_logits: bool = True, device="cuda",
                 frontier_sizes=None):
        """frontier_sizes: the expanded nodes per draft pass when they do not follow from the
        workload's width (a predefined tree shape); default w.frontier_sizes."""
        B, K, ke, V, H = w.batch, w.top_k, w.k_per_expert, w.vocab, w.hidden
        fs = list(w.frontier_sizes if frontier_sizes is None else frontier_sizes)
        self.frontier_sizes = fs
        self.pool_n = sum(f * K * ke for f in fs)
        self.n_slots = sum(fs)
        i32 = dict(dtype=torch.int32, device=device)
        f32 = dict(dtype=torch.float32, device=device)
        self.w = w
        self.pool = {"tok": torch.empty(B, self.pool_n, **i32),
                     "score": torch.empty(B, self.pool_n, **f32),
                     "parent": torch.empty(B, self.pool_n, **i32),
                     "qslot": torch.empty(B, self.pool_n, **i32),
                     "branch": torch.empty(B, self.pool_n, **i32)}
        self.pool_struct = ctx.pool_struct(self.pool)
        self.probs = [torch.empty(B, F, w.n_experts, **f32) for F in fs]
        self.expert = [torch.empty(B, F, K, **i32) for F in fs]
        self.gate = [torch.empty(B, F, K, **f32) for F in fs]
        # log-sum-exp of every stored logits row: [B, S, K], laid out like the logits (a call
        # writes rows slot_base.. of every sequence); dense per-pass arrays when no logits are kept
        self.lse_all = torch.empty(B, self.n_slots, K, **f32) if keep_logits else None
        self.lse = self.lse_views() if keep_logits else [torch.empty(B, F, K, **f32) for F in fs]
        self.feat = [torch.empty(B, F, H, dtype=ctx.tdtype, device=device) for F in fs]
        self.logits = torch.empty(B, self.n_slots, K, V, **f32) if keep_logits else None
        nxt = fs[1:] + [1]                      # nodes chosen by pass l = nodes expanded by pass l+1
        self.frontier = [torch.empty(B, n, **i32) for n in nxt]
        self.parent_score = [torch.zeros(B, 1, **f32)] + [torch.empty(B, n, **f32) for n in nxt]
        self.parent_gidx = [torch.full((B, 1), -1, **i32)] + [torch.empty(B, n, **i32) for n in nxt]
        M = w.tree_size
        self.tree = {k: torch.empty(B, M, **i32) for k in ("tok", "parent", "depth", "branch",
                                                           "qslot")}
        self.anc = torch.empty(B, M, 2, dtype=torch.int64, device=device)
        self.n_acc = torch.empty(B, **i32)
        self.acc_idx = torch.empty(B, w.depth, **i32)
        self.acc_tok = torch.empty(B, w.depth, **i32)
        self.bonus = torch.empty(B, **i32)


def _lse_views(self):
    out, s0 = [], 0
    for F in self.frontier_sizes:
        out.append(self.lse_all[:, s0:s0 + F])
        s0 += F
    return out


StepBuffers.lse_views = _lse_views


def run_draft(ctx: Context, bufs: StepBuffers, weights, u_layers: Sequence[torch.Tensor],
              root_tok: torch.Tensor, finalize: bool = True, static_plan=None):
    """One jk_draft_expand call per draft pass, then jk_tree_finalize.  The expanded nodes'
    logits are kept in bufs.logits at slot order when that buffer exists.  static_plan (from
    static_tree.plan_from_paths, with device arrays): the predefined tree shape that replaces the
    score-driven choice of frontier and final tree."""
    w = bufs.w
    fs = bufs.frontier_sizes
    B, K, ke = w.batch, w.top_k, w.k_per_expert
    gidx_base = 0
    slot_base = 0
    for l, F in enumerate(fs):
        last = l == len(fs) - 1
        out_logits = None
        if bufs.logits is not None:      # rows slot_base..slot_base+F-1 of every sequence
            out_logits = bufs.logits[:, slot_base:slot_base + F]
        width = 0 if last else fs[l + 1]
        ctx.draft_expand(weights, B, F, width, u_layers[l],
                         bufs.parent_score[l], bufs.parent_gidx[l], gidx_base, slot_base,
                         bufs.probs[l], bufs.expert[l], bufs.gate[l], bufs.pool_struct,
                         bufs.lse[l], bufs.feat[l], out_logits,
                         None if last else bufs.frontier[l],
                         None if last else bufs.parent_score[l + 1],
                         None if last else bufs.parent_gidx[l + 1],
                         None if (last or static_plan is None) else static_plan["select"][l])
        gidx_base += F * K * ke
        slot_base += F
    if finalize:
        ctx.tree_finalize(B, bufs.pool_struct, bufs.pool_n, root_tok, w.tree_size,
                          bufs.tree["tok"], bufs.tree["parent"], bufs.tree["depth"],
                          bufs.tree["branch"], bufs.tree["qslot"], bufs.anc,
                          None if static_plan is None else static_plan["keep"])


class PreBuffers:
    """Device state of the draft layer's pre-MoE block for one step: the rotated queries and the
    partial tree (parent slot, depth) of every expanded node, and the hidden states u per pass."""

    def __init__(self, ctx: Context, bufs: StepBuffers, device="cuda"):
        w = bufs.w
        S = bufs.n_slots
        self.q = torch.empty(w.batch, S, w.n_q_heads, w.head_dim, dtype=ctx.tdtype, device=device)
        self.slot_parent = torch.empty(w.batch, S, dtype=torch.int32, device=device)
        self.slot_depth = torch.empty(w.batch, S, dtype=torch.int32, device=device)
        self.state = JkPreState(_ptr(self.q), _ptr(self.slot_parent), _ptr(self.slot_depth), S)
        self.u = [torch.empty(w.batch, F, w.hidden, dtype=ctx.tdtype, device=device)
                  for F in bufs.frontier_sizes]


def run_draft_chained(ctx: Context, bufs: StepBuffers, pre: PreBuffers, weights, pre_weights,
                      root_tok: torch.Tensor, root_feat: torch.Tensor, k_cache, v_cache, kv_len,
                      rope_theta: float, scale: float, finalize: bool = True):
    """The whole draft of one step with nothing synthetic in between: per pass jk_draft_pre turns
    the frontier's tokens and their parents' features into u (Eq. 1), jk_draft_expand grows the
    tree from u (Eq. 2-5) and hands back the features the next pass starts from."""
    w = bufs.w
    fs = bufs.frontier_sizes
    B, K, ke = w.batch, w.top_k, w.k_per_expert
    gidx_base = slot_base = 0
    prev = (0, 0, 1)                       # gidx_base, slot_base, F of the previous pass
    for l, F in enumerate(fs):
        last = l == len(fs) - 1
        ctx.draft_pre(pre_weights, pre.state, B, F, slot_base,
                      None if l == 0 else bufs.parent_gidx[l], bufs.pool_struct, prev[0], prev[1],
                      prev[2], root_feat if l == 0 else bufs.feat[l - 1], root_tok, k_cache,
                      v_cache, kv_len, rope_theta, scale, pre.u[l])
        out_logits = None if bufs.logits is None else bufs.logits[:, slot_base:slot_base + F]
        ctx.draft_expand(weights, B, F, 0 if last else fs[l + 1], pre.u[l], bufs.parent_score[l],
                         bufs.parent_gidx[l], gidx_base, slot_base, bufs.probs[l], bufs.expert[l],
                         bufs.gate[l], bufs.pool_struct, bufs.lse[l], bufs.feat[l], out_logits,
                         None if last else bufs.frontier[l],
                         None if last else bufs.parent_score[l + 1],
                         None if last else bufs.parent_gidx[l + 1])
        prev = (gidx_base, slot_base, F)
        gidx_base += F * K * ke
        slot_base += F
    if finalize:
        ctx.tree_finalize(B, bufs.pool_struct, bufs.pool_n, root_tok, w.tree_size,
                          bufs.tree["tok"], bufs.tree["parent"], bufs.tree["depth"],
                          bufs.tree["branch"], bufs.tree["qslot"], bufs.anc)
