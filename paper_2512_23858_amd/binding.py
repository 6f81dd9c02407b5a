"""Python binding of include/ygg.h: argument marshalling only.

Every function takes torch tensors that already live on the GPU, checks dtypes/contiguity,
passes raw device pointers and the current HIP stream to the C ABI, and raises on a non-zero
status.  The launching calls are marshalled by a small native module (csrc/python_calls.cpp), the
queries through ctypes.  There is no CPU or PyTorch fallback: if libygg.so is missing, loading fails.
"""
from __future__ import annotations

import ctypes
import importlib
import math
import os
from dataclasses import dataclass

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
OP_ATTENTION, OP_EXPAND, OP_ACCEPT, OP_ATTACH, OP_ATTENTION_BLOCK8, OP_CONSTRAIN = 0, 1, 2, 3, 4, 5
F32, BF16, FP8_E4M3, FP8_BLOCK = 0, 1, 2, 3
KV_BLOCK = 64      # tokens to a block of the 8-bit block cache


class _CShape(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("depth", ctypes.c_int32), ("width", ctypes.c_int32),
        ("n_nodes", ctypes.c_int32), ("vocab", ctypes.c_int32), ("kv_dtype", ctypes.c_int32),
        ("softmax_scale", ctypes.c_float), ("kv_capacity", ctypes.c_int64), ("max_seq_len", ctypes.c_int32),
    ]


@dataclass
class Shape:
    """Mirror of ygg_shape (see include/ygg.h for the meaning of every field)."""
    batch: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    depth: int
    width: int
    n_nodes: int
    vocab: int
    kv_dtype: int
    softmax_scale: float
    kv_capacity: int
    max_seq_len: int

    def c(self) -> _CShape:
        return _CShape(self.batch, self.n_q_heads, self.n_kv_heads, self.head_dim, self.depth, self.width,
                       self.n_nodes, self.vocab, self.kv_dtype, self.softmax_scale, self.kv_capacity,
                       self.max_seq_len)


@dataclass
class BlockCache:
    """The tensors of an 8-bit block cache (ygg_block8_cache in include/ygg.h), of one layer or with a leading layer dimension:
    codes [B,Hkv,nblk,64*Dh] uint8, scales [B,Hkv,nblk] fp32, tails [B,128,Hkv,Dh] bf16."""
    k_codes: torch.Tensor
    v_codes: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor
    k_tail: torch.Tensor
    v_tail: torch.Tensor

    def tensors(self):
        return self.k_codes, self.v_codes, self.k_scale, self.v_scale, self.k_tail, self.v_tail

    def layer(self, i: int) -> "BlockCache":
        """Views of one layer."""
        return BlockCache(*(t[i] for t in self.tensors()))


_lib = None


def lib_path() -> str:
    return os.path.join(_PKG, "libygg.so")


def load_library() -> ctypes.CDLL:
    """Loads libygg.so (built by paper_2512_23858_amd/build.py).  Raises if it is not there."""
    global _lib
    if _lib is None:
        path = lib_path()
        if not os.path.exists(path):
            raise RuntimeError(f"{path} not found: build it with `python -m paper_2512_23858_amd.build` "
                               "(there is no fallback path)")
        lib = ctypes.CDLL(path)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        shp = ctypes.POINTER(_CShape)
        lib.ygg_workspace_bytes.restype = sz
        lib.ygg_workspace_bytes.argtypes = [shp, i32, i32]
        lib.ygg_status_string.restype = ctypes.c_char_p
        lib.ygg_status_string.argtypes = [i32]
        lib.ygg_tree_attention.restype = i32
        lib.ygg_tree_attention.argtypes = [shp] + [vp] * 9 + [vp, sz, vp]
        lib.ygg_tree_attention_fp8kv.restype = i32
        lib.ygg_tree_attention_fp8kv.argtypes = [shp] + [vp] * 11 + [vp, sz, vp]
        lib.ygg_equal_growth_expand.restype = i32
        lib.ygg_equal_growth_expand.argtypes = [shp, i32] + [vp] * 4 + [vp, sz, vp]
        lib.ygg_equal_growth_expand_static.restype = i32
        lib.ygg_equal_growth_expand_static.argtypes = [shp, i32] + [vp] * 4 + [vp]
        lib.ygg_attach_pool_bytes.restype = sz
        lib.ygg_attach_pool_bytes.argtypes = [shp]
        lib.ygg_equal_growth_attach.restype = i32
        lib.ygg_equal_growth_attach.argtypes = [shp, i32] + [vp] * 4 + [vp, sz, vp, sz, vp]
        lib.ygg_prune_for_verification.restype = i32
        lib.ygg_prune_for_verification.argtypes = [shp, i32] + [vp] * 4 + [ctypes.c_float] + [vp] * 5 + [vp]
        lib.ygg_debug_validate.restype = i32
        lib.ygg_debug_validate.argtypes = [shp] + [vp] * 4 + [i32, vp, vp]
        lib.ygg_accept_and_compact.restype = i32
        lib.ygg_accept_and_compact.argtypes = [shp, i32] + [vp] * 12 + [vp, sz, vp]
        for name, args in (("ygg_tree_attention_block8", [shp] + [vp] * 8 + [vp, sz, vp]),
                           ("ygg_block8_append", [shp, i32, vp, vp, i32, vp, i32, vp, vp, vp, vp]),
                           ("ygg_tree_rotary", [shp, vp, ctypes.c_int64, vp, ctypes.c_int64] + [vp] * 3 + [i32, i32, ctypes.c_float] + [vp] * 4),
                           ("ygg_count_tokens", [shp, vp, i32, vp, i32, i32, vp, i32, vp, vp]),
                           ("ygg_constrain_logits", [shp, vp, i32, ctypes.c_int64] + [vp] * 5 + [vp, sz, vp])):
            getattr(lib, name).restype, getattr(lib, name).argtypes = i32, args
        lib.ygg_init.restype = i32
        lib.ygg_init.argtypes = []
        lib.ygg_debug_set_attention_plan.restype = i32
        lib.ygg_debug_set_attention_plan.argtypes = [i32, i32, i32, i32]
        lib.ygg_debug_attention_plan.restype = i32
        lib.ygg_debug_attention_plan.argtypes = [shp, ctypes.POINTER(i32)]
        lib.ygg_debug_attention_launch.restype = i32
        lib.ygg_debug_attention_launch.argtypes = [shp, ctypes.POINTER(i32)]
        lib.ygg_debug_block8_plan.restype = i32
        lib.ygg_debug_block8_plan.argtypes = [shp, ctypes.POINTER(i32)]
        lib.ygg_debug_tree_attention_main.restype = i32
        lib.ygg_debug_tree_attention_main.argtypes = [shp] + [vp] * 9 + [vp, sz, vp]
        _lib = lib
    return _lib


_native = None


def _calls():
    """The native marshalling module (linked against libygg.so, so that library is looked for first)."""
    global _native
    if _native is None:
        load_library()
        _native = importlib.import_module(__package__ + "._calls")
    return _native


def status_string(code: int) -> str:
    return load_library().ygg_status_string(code).decode()


def workspace_bytes(shape: Shape, op: int, n_layers: int = 0) -> int:
    cs = shape.c()
    return int(load_library().ygg_workspace_bytes(ctypes.byref(cs), op, n_layers))


def new_workspace(shape: Shape, op: int, n_layers: int = 0, device="cuda:0"):
    """Allocates a workspace for (shape, op) through torch (contents undefined, as the library expects)."""
    n = workspace_bytes(shape, op, n_layers)
    if n == 0:
        raise ValueError("invalid shape for a workspace")
    return torch.empty(n, dtype=torch.uint8, device=device)


def new_block_cache(shape: Shape, n_layers: int = 1, device="cuda:0") -> BlockCache:
    """Allocates an empty 8-bit block cache of n_layers layers through torch (zeros)."""
    if workspace_bytes(shape, OP_ATTENTION_BLOCK8) == 0:
        raise ValueError("invalid shape for a block cache")
    B, Hkv, Dh, nblk = shape.batch, shape.n_kv_heads, shape.head_dim, -(-shape.kv_capacity // KV_BLOCK)
    codes, scales, tails = (n_layers, B, Hkv, nblk, KV_BLOCK * Dh), (n_layers, B, Hkv, nblk), (n_layers, B, 2 * KV_BLOCK, Hkv, Dh)
    return BlockCache(*(torch.zeros(codes, dtype=torch.uint8, device=device) for _ in range(2)),
                      *(torch.ones(scales, dtype=torch.float32, device=device) for _ in range(2)),
                      *(torch.zeros(tails, dtype=torch.bfloat16, device=device) for _ in range(2)))


def rotary_frequencies(rotary_dim: int, base: float = 10000.0, factor: float = 1.0, original_len: int = 0,
                       low_turns: float = 1.0, high_turns: float = 4.0) -> torch.Tensor:
    """Frequency table [rotary_dim/2] of tree_rotary on the host, fp64: base^(-2j/rotary_dim) radians per position.
    factor > 1 stretches positions for long contexts: all frequencies alike where original_len is 0; else those that make at most
    low_turns turns over original_len positions in full, those that make high_turns or more not at all, with a ramp between."""
    if rotary_dim < 2 or rotary_dim % 2 or not base > 0 or not factor > 0 or original_len < 0 or not high_turns > low_turns:
        raise ValueError("rotary_dim must be even, base and factor positive, original_len not negative, high_turns above low_turns")
    f = float(base) ** (-torch.arange(rotary_dim // 2, dtype=torch.float64) * 2 / rotary_dim)
    keep = torch.zeros_like(f)
    if original_len:
        keep = ((original_len * f / (2 * math.pi) - low_turns) / (high_turns - low_turns)).clamp(0, 1)
    return f * keep + f / factor * (1 - keep)


def _dev(t, dtype=None, name="tensor"):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    return ctypes.c_void_p(t.data_ptr())


def _check(rc: int, what: str):
    if rc != 0:
        raise RuntimeError(f"{what} failed: {status_string(rc)} (status {rc})")


def _kv_torch_dtype(shape: Shape):
    """Element type of the K/V tensors (8-bit codes travel as uint8)."""
    return {F32: torch.float32, BF16: torch.bfloat16, FP8_E4M3: torch.uint8, FP8_BLOCK: torch.bfloat16}[shape.kv_dtype]


def _explain(shape: Shape, *checks, sizes=(), cache=()):
    """The native module refused an argument: run the same checks here, which raise what the caller should see.
    checks: (tensor or None, wanted dtype or None, name); sizes: as for _explain_sizes; cache: arguments of _explain_cache."""
    shape.c()
    for t, dtype, name in checks:
        _dev(t, dtype, name)
    _explain_sizes(*sizes)
    if cache:
        _explain_cache(shape, *cache)
    raise TypeError("an argument is neither a tensor nor None, or a number is out of range")


def tree_attention(shape: Shape, q, k_cache, v_cache, seq_lens, k_tree, v_tree, parent_idx, out, lse=None,
                   workspace=None, main_kernel_only=False):
    """ygg_tree_attention: writes `out` (and `lse` if given) on the current stream.
    main_kernel_only: the measurement hook ygg_debug_tree_attention_main (no merge of the key splits)."""
    rc = (_native or _calls()).tree_attention(shape, q, k_cache, v_cache, seq_lens, k_tree, v_tree, parent_idx, out, lse,
                                              workspace, True if main_kernel_only else False)
    if rc:
        if rc < 0:
            dt, i32 = _kv_torch_dtype(shape), torch.int32
            _explain(shape, (q, dt, "q"), (k_cache, dt, "k_cache"), (v_cache, dt, "v_cache"), (seq_lens, i32, "seq_lens"),
                     (k_tree, dt, "k_tree"), (v_tree, dt, "v_tree"), (parent_idx, i32, "parent_idx"), (out, dt, "out"),
                     (lse, torch.float32, "lse"), (workspace, None, "workspace"))
        _check(rc, "ygg_tree_attention")
    return out


def tree_attention_fp8kv(shape: Shape, q, k_cache, v_cache, seq_lens, k_tree, v_tree, k_scale, v_scale, parent_idx,
                         out, lse=None, workspace=None):
    """ygg_tree_attention_fp8kv: K/V as uint8 E4M3 codes with per-kv-head fp32 scales, Q and out bf16."""
    rc = (_native or _calls()).tree_attention_fp8kv(shape, q, k_cache, v_cache, seq_lens, k_tree, v_tree, k_scale, v_scale,
                                                    parent_idx, out, lse, workspace)
    if rc:
        if rc < 0:
            u8, bf, f32, i32 = torch.uint8, torch.bfloat16, torch.float32, torch.int32
            _explain(shape, (q, bf, "q"), (k_cache, u8, "k_cache"), (v_cache, u8, "v_cache"), (seq_lens, i32, "seq_lens"),
                     (k_tree, u8, "k_tree"), (v_tree, u8, "v_tree"), (k_scale, f32, "k_scale"), (v_scale, f32, "v_scale"),
                     (parent_idx, i32, "parent_idx"), (out, bf, "out"), (lse, f32, "lse"), (workspace, None, "workspace"))
        _check(rc, "ygg_tree_attention_fp8kv")
    return out


def _explain_growth(shape, draft_logits, parent_idx, token_ids, cum_logprob, *scratch):
    _explain(shape, (draft_logits, torch.float32, "draft_logits"), (parent_idx, torch.int32, "parent_idx"),
             (token_ids, torch.int32, "token_ids"), (cum_logprob, torch.float32, "cum_logprob"),
             *((t, None, "workspace") for t in scratch))


def equal_growth_expand(shape: Shape, d: int, draft_logits, parent_idx, token_ids, cum_logprob, workspace=None):
    """ygg_equal_growth_expand: fills the depth-d slots of parent_idx/token_ids/cum_logprob."""
    rc = (_native or _calls()).equal_growth_expand(shape, d, draft_logits, parent_idx, token_ids, cum_logprob, workspace)
    if rc:
        if rc < 0:
            _explain_growth(shape, draft_logits, parent_idx, token_ids, cum_logprob, workspace)
        _check(rc, "ygg_equal_growth_expand")


def equal_growth_expand_static(shape: Shape, d: int, draft_logits, parent_idx, token_ids, cum_logprob):
    """ygg_equal_growth_expand_static: the same draft step on the library's built-in scratch (no workspace)."""
    rc = (_native or _calls()).equal_growth_expand_static(shape, d, draft_logits, parent_idx, token_ids, cum_logprob)
    if rc:
        if rc < 0:
            _explain_growth(shape, draft_logits, parent_idx, token_ids, cum_logprob)
        _check(rc, "ygg_equal_growth_expand_static")


def attach_pool_bytes(shape: Shape) -> int:
    cs = shape.c()
    return int(load_library().ygg_attach_pool_bytes(ctypes.byref(cs)))


def equal_growth_attach(shape: Shape, t: int, draft_logits, parent_idx, token_ids, cum_logprob, pool, workspace=None):
    """ygg_equal_growth_attach: draft step t with free attachment; fills nodes 1+(t-1)W .. tW and updates `pool`."""
    rc = (_native or _calls()).equal_growth_attach(shape, t, draft_logits, parent_idx, token_ids, cum_logprob, pool, workspace)
    if rc:
        if rc < 0:
            _explain_growth(shape, draft_logits, parent_idx, token_ids, cum_logprob, workspace, pool)
        _check(rc, "ygg_equal_growth_attach")


def prune_for_verification(shape: Shape, w_verify: int, parent_idx, token_ids, cum_logprob, kept_nodes, new_parent,
                           new_token, expected_len=None, best_width=None, t_verifier=None, t_draft: float = 0.0):
    """ygg_prune_for_verification: keeps the w_verify most valuable nodes as a renumbered tree."""
    rc = (_native or _calls()).prune_for_verification(shape, w_verify, parent_idx, token_ids, cum_logprob, kept_nodes,
                                                      new_parent, new_token, expected_len, best_width, t_verifier, t_draft)
    if rc:
        if rc < 0:
            f32, i32 = torch.float32, torch.int32
            _explain(shape, (parent_idx, i32, "parent_idx"), (token_ids, i32, "token_ids"), (cum_logprob, f32, "cum_logprob"),
                     (t_verifier, f32, "t_verifier"), (kept_nodes, i32, "kept_nodes"), (new_parent, i32, "new_parent"),
                     (new_token, i32, "new_token"), (expected_len, f32, "expected_len"), (best_width, i32, "best_width"))
        _check(rc, "ygg_prune_for_verification")


def debug_validate(shape: Shape, flags, parent_idx=None, seq_lens=None, token_ids=None, logits=None):
    """ygg_debug_validate: per-sequence violation bit masks into `flags` ([B] int32 on the GPU)."""
    cs = shape.c()
    rows = 0 if logits is None else int(logits.shape[1])
    rc = load_library().ygg_debug_validate(
        ctypes.byref(cs), _dev(parent_idx, torch.int32, "parent_idx"), _dev(seq_lens, torch.int32, "seq_lens"),
        _dev(token_ids, torch.int32, "token_ids"), _dev(logits, torch.float32, "logits"), rows,
        _dev(flags, torch.int32, "flags"), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    _check(rc, "ygg_debug_validate")


def accept_and_compact(shape: Shape, n_layers: int, parent_idx, token_ids, k_tree, v_tree, k_cache, v_cache,
                       seq_lens, accept_len, accept_path, bonus_token, target_logits=None, target_tokens=None,
                       workspace=None):
    """ygg_accept_and_compact: updates the caches and seq_lens in place, fills the three outputs."""
    rc = (_native or _calls()).accept_and_compact(shape, n_layers, parent_idx, token_ids, k_tree, v_tree, k_cache, v_cache,
                                                  seq_lens, accept_len, accept_path, bonus_token, target_logits, target_tokens,
                                                  workspace)
    if rc:
        if rc < 0:
            dt, i32 = _kv_torch_dtype(shape), torch.int32
            _explain(shape, (target_logits, torch.float32, "target_logits"), (target_tokens, i32, "target_tokens"),
                     (parent_idx, i32, "parent_idx"), (token_ids, i32, "token_ids"), (k_tree, dt, "k_tree"),
                     (v_tree, dt, "v_tree"), (k_cache, dt, "k_cache"), (v_cache, dt, "v_cache"), (seq_lens, i32, "seq_lens"),
                     (accept_len, i32, "accept_len"), (accept_path, i32, "accept_path"), (bonus_token, i32, "bonus_token"),
                     (workspace, None, "workspace"))
        _check(rc, "ygg_accept_and_compact")


def _explain_rows(shape, rows, *checks, sizes=()):
    """_explain for calls with tensors whose rows may be strided: rows = (tensor, wanted dtype or None, name)."""
    for t, dtype, name in rows:
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError(f"{name} must be a GPU tensor")
        if dtype is not None and t.dtype != dtype:
            raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
        if t.dim() < 3:
            raise ValueError(f"{name} must have batch and token dimensions and dense ones behind them")
    for t, dtype, name in checks:
        _dev(t, dtype, name)
    for t, _, name in rows:
        if t is not None and not t.is_contiguous():
            raise ValueError(f"{name}: rows must be dense and lie evenly over batch and tokens")
    _explain(shape, sizes=sizes)


def _explain_sizes(*sizes):
    """sizes: (tensor or None, what the shape asks for, name): a pair, sequences and elements of each (more sequences may follow, and a
    single one may be longer); three numbers, the exact shape of strided rows; a list, all dimensions, the first as a minimum."""
    for t, n, name in sizes:
        if t is None:
            continue
        if isinstance(n, list):
            if t.dim() != len(n) or t.shape[0] < n[0] or list(t.shape[1:]) != n[1:]:
                raise ValueError(f"{name}: dimensions {n} are wanted, got {list(t.shape)}")
        elif len(n) == 3:
            if tuple(t.shape[:2]) != n[:2] or t.numel() != n[0] * n[1] * n[2]:
                raise ValueError(f"{name}: {n[0]} x {n[1]} rows of {n[2]} elements are wanted, got {tuple(t.shape)}")
        else:
            seqs, per = n
            if t.numel() != seqs * per and not (seqs == 1 and t.numel() >= per) and not (
                    t.dim() > 0 and t.shape[0] > seqs and t.numel() == t.shape[0] * per):
                raise ValueError(f"{name}: {seqs} x {per} elements are wanted, got {tuple(t.shape)}")


def _explain_cache(shape: Shape, cache: BlockCache, layers: int, alone: bool):
    """Sizes of a cache's tensors: of `layers` layers (alone: and no more), of the shape's batch and capacity."""
    B, Hkv, Dh, nblk = shape.batch, shape.n_kv_heads, shape.head_dim, -(-shape.kv_capacity // KV_BLOCK)
    forms = ((B, Hkv, nblk, KV_BLOCK * Dh), (B, Hkv, nblk), (B, 2 * KV_BLOCK, Hkv, Dh))
    for i, (t, _, name) in enumerate(_cache_checks(cache)):
        form = forms[i // 2]
        per = math.prod(form[1:])
        if t is None or t.numel() == layers * B * per:
            continue
        L, seqs = (t.shape[0], t.shape[1]) if t.dim() == len(form) + 1 else (1, t.shape[0]) if t.dim() == len(form) else (0, 0)
        if t.numel() != L * seqs * per or (L != 1 if alone else L < layers) or (seqs < B if L == 1 else seqs != B):
            raise ValueError(f"{name}: {layers} layer{'s' * (layers > 1)} of {list(form)} wanted, got {list(t.shape)}")


def _cache_checks(cache: BlockCache):
    want = (torch.uint8, torch.uint8, torch.float32, torch.float32, torch.bfloat16, torch.bfloat16)
    return list(zip(cache.tensors(), want, ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail")))


def tree_attention_block8(shape: Shape, q, cache: BlockCache, seq_lens, k_tree, v_tree, parent_idx, out, lse=None, workspace=None):
    """ygg_tree_attention_block8: tree attention of one layer over an 8-bit block cache (shape.kv_dtype FP8_BLOCK)."""
    rc = (_native or _calls()).tree_attention_block8(shape, q, cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale, cache.k_tail,
                                                     cache.v_tail, seq_lens, k_tree, v_tree, parent_idx, out, lse, workspace)
    if rc:
        if rc < 0:
            bf, i32 = torch.bfloat16, torch.int32
            B, N, q_row, kv_row = shape.batch, shape.n_nodes, shape.n_q_heads * shape.head_dim, shape.n_kv_heads * shape.head_dim
            _explain(shape, (q, bf, "q"), *_cache_checks(cache), (seq_lens, i32, "seq_lens"), (k_tree, bf, "k_tree"),
                     (v_tree, bf, "v_tree"), (parent_idx, i32, "parent_idx"), (out, bf, "out"), (lse, torch.float32, "lse"),
                     (workspace, None, "workspace"),
                     sizes=[(q, (B, N * q_row), "q"), (seq_lens, (B, 1), "seq_lens"), (k_tree, (B, N * kv_row), "k_tree"),
                            (v_tree, (B, N * kv_row), "v_tree"), (parent_idx, (B, N), "parent_idx"), (out, (B, N * q_row), "out"),
                            (lse, (B, N * shape.n_q_heads), "lse")],
                     cache=(cache, 1, True))
        _check(rc, "ygg_tree_attention_block8")
    return out


def block8_append(shape: Shape, n_layers: int, k_new, v_new, cache: BlockCache, seq_lens, n_new, rows=None):
    """ygg_block8_append: tokens seq_lens - n_new .. seq_lens - 1 of every layer, from rows of k_new and v_new
    [n_layers,B,n_rows,Hkv,Dh]; rows [B,max_new] picks them (an accept_path), else they are the first n_new.
    include/ygg.h (ygg_block8_cache) says to which lengths a sequence can be taken back."""
    rc = (_native or _calls()).block8_append(shape, n_layers, k_new, v_new, rows, n_new, seq_lens, cache.k_codes, cache.v_codes,
                                             cache.k_scale, cache.v_scale, cache.k_tail, cache.v_tail)
    if rc:
        if rc < 0:
            bf, i32 = torch.bfloat16, torch.int32
            form = [n_layers, shape.batch, k_new.shape[2] if k_new is not None and k_new.dim() > 2 else 0, shape.n_kv_heads, shape.head_dim]
            _explain(shape, (k_new, bf, "k_new"), (v_new, bf, "v_new"), (rows, i32, "rows"), (n_new, i32, "n_new"),
                     (seq_lens, i32, "seq_lens"), *_cache_checks(cache),
                     sizes=[(k_new, form, "k_new"), (v_new, form, "v_new"), (n_new, (shape.batch, 1), "n_new"), (seq_lens, (shape.batch, 1), "seq_lens"),
                            (rows, (shape.batch, 0 if rows is None else rows.shape[-1]), "rows")],
                     cache=(cache, n_layers, False))
        _check(rc, "ygg_block8_append")


def tree_rotary(shape: Shape, q, k, q_out, k_out, frequencies, seq_lens=None, parent_idx=None, positions=None, interleaved: bool = False,
                scale: float = 1.0):
    """ygg_tree_rotary: rotates 2 * len(frequencies) dimensions of every head of q [B,N,Hq,Dh] and k [B,N,Hkv,Dh] (either may be None
    with its output; tokens may be strided) at seq_lens + depth, or at positions [B,N].  frequencies: fp64 on the GPU."""
    rc = (_native or _calls()).tree_rotary(shape, q, k, q_out, k_out, frequencies, seq_lens, parent_idx, positions,
                                           True if interleaved else False, scale)
    if rc:
        if rc < 0:
            dt, i32 = torch.float32 if shape.kv_dtype == F32 else torch.bfloat16, torch.int32
            B, N = shape.batch, shape.n_nodes
            _explain_rows(shape, ((q, dt, "q"), (k, dt, "k")), (q_out, dt, "q_out"), (k_out, dt, "k_out"),
                          (frequencies, torch.float64, "frequencies"), (seq_lens, i32, "seq_lens"), (parent_idx, i32, "parent_idx"),
                          (positions, i32, "positions"),
                          sizes=[(q, (B, N, shape.n_q_heads * shape.head_dim), "q"), (k, (B, N, shape.n_kv_heads * shape.head_dim), "k"),
                                 (q_out, (B, N * shape.n_q_heads * shape.head_dim), "q_out"),
                                 (k_out, (B, N * shape.n_kv_heads * shape.head_dim), "k_out"), (positions, (B, N), "positions"),
                                 (seq_lens if positions is None else None, (B, 1), "seq_lens"),
                                 (parent_idx if positions is None else None, (B, N), "parent_idx")])
        _check(rc, "ygg_tree_rotary")


def count_tokens(shape: Shape, tokens, n_new, counts, rows=None, first: int = 0, prompt: bool = False):
    """ygg_count_tokens: adds n_new[b] tokens of tokens [B,T] (from `first` on, or those that rows [B,max_new] names) to counts [B,V]."""
    rc = (_native or _calls()).count_tokens(shape, tokens, n_new, counts, rows, first, True if prompt else False)
    if rc:
        if rc < 0:
            i32 = torch.int32
            _explain(shape, (tokens, i32, "tokens"), (n_new, i32, "n_new"), (counts, i32, "counts"), (rows, i32, "rows"),
                     sizes=[(tokens, (shape.batch, 0 if tokens is None else tokens.shape[-1]), "tokens"), (n_new, (shape.batch, 1), "n_new"),
                            (counts, (shape.batch, shape.vocab), "counts"), (rows, (shape.batch, 0 if rows is None else rows.shape[-1]), "rows")])
        _check(rc, "ygg_count_tokens")


def constrain_logits(shape: Shape, logits, parent_idx, token_ids, out=None, best=None, counts=None, repetition=None, presence=None,
                     frequency=None, bias=None, masks=None, mask_index=None, workspace=None):
    """ygg_constrain_logits: penalties, bias ([V] or [B,V]) and masks ([M, ceil(V/32)] int32 bit words) on logits [B,N,V] (fp32 or
    bf16, rows may be strided) into `out` (fp32) and / or the first maximum of each row into `best`."""
    rc = (_native or _calls()).constrain_logits(shape, logits, parent_idx, token_ids, out, best, counts, repetition, presence, frequency,
                                                bias, masks, mask_index, workspace)
    if rc:
        if rc < 0:
            f32, i32 = torch.float32, torch.int32
            B, N, V = shape.batch, shape.n_nodes, shape.vocab
            if logits is not None and logits.dtype not in (f32, torch.bfloat16):
                raise TypeError(f"logits: expected {f32} or {torch.bfloat16}, got {logits.dtype}")
            _explain_rows(shape, ((logits, None, "logits"),), (parent_idx, i32, "parent_idx"), (token_ids, i32, "token_ids"),
                          (out, f32, "out"), (best, i32, "best"), (counts, i32, "counts"), (repetition, f32, "repetition"),
                          (presence, f32, "presence"), (frequency, f32, "frequency"), (bias, f32, "bias"), (masks, i32, "masks"),
                          (mask_index, i32, "mask_index"), (workspace, None, "workspace"),
                          sizes=[(logits, (B, N, V), "logits"), (parent_idx, (B, N), "parent_idx"), (token_ids, (B, N), "token_ids"),
                                 (out, (B, N * V), "out"), (best, (B, N), "best"), (counts, (B, V), "counts"), (repetition, (B, 1), "repetition"),
                                 (presence, (B, 1), "presence"), (frequency, (B, 1), "frequency"),
                                 (bias, (1 if bias is not None and bias.dim() == 1 else B, V), "bias"),
                                 (masks, (0 if masks is None else masks.shape[0], -(-V // 32)), "masks"), (mask_index, (B, N), "mask_index")])
        _check(rc, "ygg_constrain_logits")


def attention_plan(shape: Shape) -> dict:
    """ygg_debug_attention_plan: the launch plan of tree_attention for this shape (host only)."""
    cs = shape.c()
    out = (ctypes.c_int32 * 5)()
    _check(load_library().ygg_debug_attention_plan(ctypes.byref(cs), out), "ygg_debug_attention_plan")
    return dict(matrix_cores=bool(out[0]), waves=out[1], key_shares=out[2], row_tiles=out[3], key_splits=out[4])


def attention_launch(shape: Shape) -> dict:
    """ygg_debug_attention_launch: more of the launch plan of tree_attention for this shape (host only)."""
    cs = shape.c()
    out = (ctypes.c_int32 * 3)()
    _check(load_library().ygg_debug_attention_launch(ctypes.byref(cs), out), "ygg_debug_attention_launch")
    return dict(opposite_phases=bool(out[0]), tree_cost=out[1], lds_bytes=out[2])


def block8_plan(shape: Shape) -> dict:
    """ygg_debug_block8_plan: the launch plan of tree_attention_block8 for this shape (host only)."""
    cs = shape.c()
    out = (ctypes.c_int32 * 7)()
    _check(load_library().ygg_debug_block8_plan(ctypes.byref(cs), out), "ygg_debug_block8_plan")
    return dict(row_blocks=out[0], row_tiles=out[1], rem_blocks=out[2], runs=out[3], rem_runs=out[4], wide=bool(out[5]), merge_lanes=out[6])


def init():
    """ygg_init: prepares the current device up front (otherwise done by the first launching call)."""
    _check(load_library().ygg_init(), "ygg_init")


def set_attention_plan(waves: int = 0, rblocks: int = 0, nsplit: int = 0, kshares: int = 0):
    """ygg_debug_set_attention_plan: tuning override of the attention launch plan (all zero: none)."""
    _check(load_library().ygg_debug_set_attention_plan(waves, rblocks, nsplit, kshares), "ygg_debug_set_attention_plan")
