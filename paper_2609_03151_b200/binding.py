"""ctypes binding of libbasp.so: same names as include/basp.h, argument marshalling only.

Importing this module loads the CUDA library and fails loudly if it has not been built
(``python -m paper_2609_03151_b200.build``).  There is no CPU fallback of any call.
"""
from __future__ import annotations

import ctypes
import os
import struct
from ctypes import POINTER, Structure, byref, c_char_p, c_float, c_int, c_longlong, c_size_t, c_void_p

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libbasp.so")
if not os.path.exists(_LIB_PATH):
    raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2609_03151_b200.build` "
                      "(there is no fallback path)")
lib = ctypes.CDLL(_LIB_PATH)
try:
    from ._marshal import addresses as _fast_addresses  # built beside the library, from csrc/marshal.cpp
except ImportError as e:
    raise ImportError(f"the binding's _marshal.so does not load ({e}): build it with `python -m paper_2609_03151_b200.build`") from e

BASP_OK = 0
BASP_ERR_INVALID, BASP_ERR_UNSUPPORTED, BASP_ERR_NULL, BASP_ERR_ALIGN = -1, -2, -3, -4
BASP_ERR_ALIAS, BASP_ERR_CUDA, BASP_ERR_TIMEOUT, BASP_ERR_WORKSPACE = -5, -6, -7, -8
BASP_MAX_RANKS = 32

EXPORTS = [
    "basp_plan_create", "basp_plan_destroy", "basp_plan_get_info", "basp_plan_get_rank",
    "basp_plan_group_ranks", "basp_reshard_s2h", "basp_reshard_h2s", "basp_reshard_qkv_s2h",
    "basp_attn_fwd", "basp_layer_fwd", "basp_workspace_bytes", "basp_layer_fwd_fused",
    "basp_layer_fwd_host", "basp_host_arena_bytes", "basp_layer_fwd_static",
    "basp_layer_workspace_shards", "basp_attn_bwd", "basp_attn_bwd_workspace_bytes", "basp_reshard_grads_h2s",
    "basp_layer_bwd", "basp_layer_bwd_workspace_bytes", "basp_get_status", "basp_clear_status",
    "basp_strerror", "basp_last_cuda_error", "basp_launch_count", "basp_selftest_wait_timeout", "basp_qkv_proj", "basp_out_proj",
    "basp_reshard_qkv_s2h_ranks", "basp_reshard_h2s_ranks", "basp_attn_fwd_ranks", "basp_layer_fwd_fused_ranks",
    "basp_qkv_proj_rope", "basp_layer_bwd_seq", "basp_layer_bwd_seq_workspace_bytes", "basp_plan_create_parts", "basp_attn_bwd_deterministic",
    "basp_qk_norm_rope", "basp_qk_norm_rope_bwd", "basp_qk_norm_rope_bwd_workspace_bytes",
    "basp_ckpt_bytes", "basp_ckpt_pack", "basp_ckpt_reshard_s2h", "basp_layer_bwd_ckpt",
    "basp_lm_loss_fwd", "basp_lm_loss_fwd_workspace_bytes", "basp_lm_loss_grad", "basp_lm_loss_grad_workspace_bytes",
    "basp_mask_bytes", "basp_mask_ranges", "basp_mask_packed", "basp_attn_masked_fwd", "basp_attn_masked_bwd",
    "basp_attn_masked_bwd_workspace_bytes", "basp_layer_masked_fwd", "basp_layer_masked_bwd", "basp_layer_masked_bwd_workspace_bytes", "basp_rope_make", "basp_rope",
    "basp_block_norm", "basp_block_norm_bwd", "basp_block_norm_bwd_workspace_bytes",
]


class basp_config(Structure):
    _fields_ = [(n, c_int) for n in ("n_ranks", "micro_batch", "num_groups", "seq_len", "n_q_heads",
                                     "n_kv_heads", "head_dim", "dtype", "causal")]


class basp_plan_info(Structure):
    _fields_ = [(n, c_int) for n in ("group_size", "num_groups", "seqs_per_group", "tokens_per_rank",
                                     "tokens_last_rank", "q_heads_per_rank", "kv_heads_per_rank")] + \
               [(n, c_size_t) for n in ("q_shard_elems", "kv_shard_elems", "lse_shard_elems")]


class basp_rank_info(Structure):
    _fields_ = [(n, c_int) for n in ("group", "local_rank", "seq_begin", "seq_end", "token_begin", "token_end",
                                     "q_head_begin", "q_head_end", "kv_head_begin", "kv_head_end")]


_PP = POINTER(c_void_p)
lib.basp_plan_create.argtypes = [POINTER(basp_config), POINTER(c_void_p)]
lib.basp_plan_destroy.argtypes = [c_void_p]
lib.basp_plan_get_info.argtypes = [c_void_p, POINTER(basp_plan_info)]
lib.basp_plan_get_rank.argtypes = [c_void_p, c_int, POINTER(basp_rank_info)]
lib.basp_plan_group_ranks.argtypes = [c_void_p, c_int, POINTER(c_int)]
lib.basp_reshard_s2h.argtypes = [c_void_p, c_int, _PP, _PP, c_void_p]
lib.basp_reshard_h2s.argtypes = [c_void_p, c_int, _PP, _PP, c_void_p]
lib.basp_reshard_qkv_s2h.argtypes = [c_void_p] + [_PP] * 6 + [c_void_p]
lib.basp_attn_fwd.argtypes = [c_void_p] + [_PP] * 5 + [c_float, c_void_p]
lib.basp_layer_fwd.argtypes = [c_void_p] + [_PP] * 5 + [c_void_p, c_size_t, c_float, c_void_p]
lib.basp_layer_fwd_fused.argtypes = [c_void_p] + [_PP] * 5 + [c_float, c_void_p]
lib.basp_reshard_qkv_s2h_ranks.argtypes = [c_void_p] + [_PP] * 6 + [c_int, c_int, c_void_p]
lib.basp_reshard_h2s_ranks.argtypes = [c_void_p, c_int, _PP, _PP, c_int, c_int, c_void_p]
lib.basp_attn_fwd_ranks.argtypes = [c_void_p] + [_PP] * 5 + [c_float, c_int, c_int, c_void_p]
lib.basp_layer_fwd_fused_ranks.argtypes = [c_void_p] + [_PP] * 5 + [c_float, c_int, c_int, c_void_p]
lib.basp_layer_fwd_static.argtypes = [c_void_p] + [_PP] * 5 + [c_float, c_void_p]
lib.basp_layer_fwd_host.argtypes = [c_void_p] + [_PP] * 4 + [c_void_p, c_size_t, c_float, c_void_p]
lib.basp_layer_workspace_shards.argtypes = [c_void_p, c_void_p] + [_PP] * 4
lib.basp_attn_bwd.argtypes = [c_void_p] + [_PP] * 9 + [c_void_p, c_size_t, c_float, c_void_p]
lib.basp_attn_bwd_deterministic.argtypes = lib.basp_attn_bwd.argtypes
lib.basp_reshard_grads_h2s.argtypes = [c_void_p] + [_PP] * 6 + [c_void_p]
lib.basp_layer_bwd.argtypes = [c_void_p] + [_PP] * 9 + [c_void_p, c_size_t, c_float, c_void_p]
lib.basp_layer_bwd_seq.argtypes = [c_void_p] + [_PP] * 9 + [c_void_p, c_size_t, c_float, c_void_p]
for _n in ("basp_attn_bwd_workspace_bytes", "basp_layer_bwd_workspace_bytes", "basp_layer_bwd_seq_workspace_bytes"):
    getattr(lib, _n).argtypes = [c_void_p]
    getattr(lib, _n).restype = c_size_t
lib.basp_workspace_bytes.argtypes = [c_void_p]
lib.basp_workspace_bytes.restype = c_size_t
lib.basp_host_arena_bytes.argtypes = [c_void_p]
lib.basp_host_arena_bytes.restype = c_size_t
lib.basp_get_status.argtypes = [c_void_p, POINTER(c_int)]
lib.basp_clear_status.argtypes = [c_void_p]
lib.basp_selftest_wait_timeout.argtypes = [ctypes.c_uint, c_void_p]
lib.basp_qkv_proj.argtypes = [c_void_p, c_int, _PP, c_void_p, _PP, _PP, _PP, c_void_p]
lib.basp_out_proj.argtypes = [c_void_p, c_int, _PP, c_void_p, _PP, c_void_p]
lib.basp_qkv_proj_rope.argtypes = [c_void_p, c_int, _PP, c_void_p, c_void_p, c_void_p, _PP, _PP, _PP, c_void_p]
# the calls below take their tables as addresses (see _Marshal)
lib.basp_qk_norm_rope.argtypes = [c_void_p] * 7 + [c_float] + [c_void_p] * 3
lib.basp_qk_norm_rope_bwd.argtypes = [c_void_p] * 7 + [c_float] + [c_void_p] * 7 + [c_size_t, c_void_p]
lib.basp_ckpt_pack.argtypes = [c_void_p] * 7
lib.basp_ckpt_reshard_s2h.argtypes = [c_void_p] * 7
lib.basp_layer_bwd_ckpt.argtypes = [c_void_p] * 8 + [c_size_t, c_float, c_void_p]
lib.basp_lm_loss_fwd.argtypes = [c_void_p, c_int, c_int] + [c_void_p] * 6 + [c_size_t, c_void_p]
lib.basp_lm_loss_grad.argtypes = [c_void_p, c_int, c_int] + [c_void_p] * 8 + [c_int, c_void_p, c_size_t, c_void_p]
for _n, _a in (("basp_qk_norm_rope_bwd_workspace_bytes", []), ("basp_ckpt_bytes", [c_int]),
               ("basp_lm_loss_fwd_workspace_bytes", [c_int]), ("basp_lm_loss_grad_workspace_bytes", [c_int] * 3)):
    getattr(lib, _n).argtypes = [c_void_p] + _a
    getattr(lib, _n).restype = c_size_t


class _Score(Structure):
    _fields_ = [("softcap", c_float), ("slopes", c_void_p), ("mask", c_void_p), ("mask_bytes", c_size_t)]


class basp_rope_config(Structure):
    _fields_ = [(n, c_int) for n in ("rotary_dim", "interleaved", "scaling")] + \
               [(n, ctypes.c_double) for n in ("base", "stretch", "original_len", "slow", "fast", "factor")]


class basp_rope_turns(Structure):
    _fields_ = [("rotary_dim", c_int), ("interleaved", c_int), ("factor", c_float), ("turns", ctypes.c_ulonglong * 64)]


lib.basp_mask_ranges.argtypes = [c_void_p] * 4 + [c_size_t, c_void_p]
lib.basp_mask_packed.argtypes = [c_void_p] * 3 + [c_int, c_void_p, c_size_t, c_void_p]
lib.basp_attn_masked_fwd.argtypes = [c_void_p, c_void_p] + [c_void_p] * 5 + [c_float, c_void_p]
lib.basp_attn_masked_bwd.argtypes = [c_void_p, c_void_p] + [c_void_p] * 10 + [c_size_t, c_float, c_void_p]
lib.basp_layer_masked_fwd.argtypes = [c_void_p, c_void_p] + [c_void_p] * 6 + [c_size_t, c_float, c_void_p]
lib.basp_layer_masked_bwd.argtypes = [c_void_p, c_void_p] + [c_void_p] * 10 + [c_size_t, c_float, c_void_p]
lib.basp_rope_make.argtypes = [POINTER(basp_rope_config), POINTER(basp_rope_turns)]
lib.basp_rope.argtypes = [c_void_p, POINTER(basp_rope_turns)] + [c_void_p] * 3 + [c_int] + [c_void_p] * 3
lib.basp_block_norm.argtypes = [c_void_p, c_int] + [c_void_p] * 5 + [c_float, c_float] + [c_void_p] * 3
lib.basp_block_norm_bwd.argtypes = [c_void_p, c_int] + [c_void_p] * 5 + [c_float, c_float] + [c_void_p] * 8 + [c_size_t, c_void_p]
for _n, _a in (("basp_mask_bytes", []), ("basp_attn_masked_bwd_workspace_bytes", []), ("basp_layer_masked_bwd_workspace_bytes", []),
               ("basp_block_norm_bwd_workspace_bytes", [c_int])):
    getattr(lib, _n).argtypes = [c_void_p] + _a
    getattr(lib, _n).restype = c_size_t
lib.basp_strerror.argtypes = [c_int]
lib.basp_strerror.restype = c_char_p
lib.basp_last_cuda_error.restype = c_char_p
lib.basp_launch_count.restype = c_longlong


class BaspError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = lib.basp_strerror(code).decode()
        cuda = lib.basp_last_cuda_error().decode() if code == BASP_ERR_CUDA else ""
        super().__init__(f"{where}: {msg} ({code}) {cuda}".strip())


def _check(code: int, where: str):
    if code != BASP_OK:
        raise BaspError(code, where)


def _ptrs(tensors, n: int):
    """Host array of n raw addresses from a list of tensors, raw integer addresses (peer memory mapped into this
    process) or None entries (-> NULL)."""
    if tensors is None:
        return None
    if len(tensors) != n:
        raise ValueError(f"expected {n} shards, got {len(tensors)}")
    return (c_void_p * n)(*[None if t is None else (t.data_ptr() if hasattr(t, "data_ptr") else int(t))
                            for t in tensors])


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


class Plan:
    """Owner of a basp_plan*; the N, K, ... attributes are what basp_plan_get_info reports."""

    def __init__(self, handle: int, cfg: basp_config):
        self.handle = c_void_p(handle)
        self.cfg = cfg
        info = basp_plan_info()
        _check(lib.basp_plan_get_info(self.handle, byref(info)), "basp_plan_get_info")
        self.info = info
        self.N = cfg.n_ranks
        self.K, self.G, self.Bl, self.T = info.group_size, info.num_groups, info.seqs_per_group, info.tokens_per_rank
        self.S, self.Hq, self.Hkv, self.D = cfg.seq_len, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim
        self.Hq_l, self.Hkv_l = info.q_heads_per_rank, info.kv_heads_per_rank
        self.T_last = info.tokens_last_rank
        self.sizes = {}        # elements of the ranks' shards, by elements per token

    def rank_tokens(self, r: int) -> int:
        """Tokens per sequence in rank r's sequence-sharded shards (the last rank of a group is short when the group
        size does not divide the sequence length)."""
        return self.T_last if r % self.K == self.K - 1 else self.T

    def __del__(self, _destroy=lib.basp_plan_destroy):
        h, self.handle = getattr(self, "handle", None), None
        if h:
            _destroy(h)


def basp_plan_create(n_ranks, micro_batch, seq_len, n_q_heads, n_kv_heads, head_dim, num_groups=0,
                     causal=True, dtype=0) -> Plan:
    cfg = basp_config(n_ranks, micro_batch, num_groups, seq_len, n_q_heads, n_kv_heads, head_dim, dtype, int(causal))
    out = c_void_p()
    _check(lib.basp_plan_create(byref(cfg), byref(out)), "basp_plan_create")
    return Plan(out.value, cfg)


class basp_plan_part(Structure):
    _fields_ = [("plan", c_void_p)] + [(n, c_int) for n in ("rank_begin", "n_ranks", "seq_begin", "n_seqs", "group_size")]


lib.basp_plan_create_parts.argtypes = [POINTER(basp_config), POINTER(basp_plan_part), POINTER(c_int)]


class PlanPart:
    """One uniform part of an unequal group formation: `plan` serves global ranks [rank_begin, rank_begin + n_ranks)
    and sequences [seq_begin, seq_begin + n_seqs); `shards(x)` cuts a per-rank list down to the part's ranks."""

    def __init__(self, plan: Plan, rank_begin: int, n_ranks: int, seq_begin: int, n_seqs: int, group_size: int):
        self.plan, self.rank_begin, self.n_ranks = plan, rank_begin, n_ranks
        self.seq_begin, self.n_seqs, self.group_size = seq_begin, n_seqs, group_size

    def shards(self, per_rank):
        return list(per_rank[self.rank_begin:self.rank_begin + self.n_ranks])


def basp_plan_create_parts(n_ranks, micro_batch, seq_len, n_q_heads, n_kv_heads, head_dim, causal=True, dtype=0):
    """Group formation for any micro_batch <= n_ranks (groups of ceil and floor(N/B) ranks): a list of one or two
    PlanPart.  Every call of the library is then made per part with part.plan and part.shards(...)."""
    cfg = basp_config(n_ranks, micro_batch, 0, seq_len, n_q_heads, n_kv_heads, head_dim, dtype, int(causal))
    arr = (basp_plan_part * 2)()
    n = c_int(0)
    _check(lib.basp_plan_create_parts(byref(cfg), arr, byref(n)), "basp_plan_create_parts")
    out = []
    for i in range(n.value):
        c = basp_config(arr[i].n_ranks, arr[i].n_seqs, 0, seq_len, n_q_heads, n_kv_heads, head_dim, dtype, int(causal))
        out.append(PlanPart(Plan(arr[i].plan, c), arr[i].rank_begin, arr[i].n_ranks, arr[i].seq_begin, arr[i].n_seqs,
                            arr[i].group_size))
    return out


def basp_plan_get_rank(plan: Plan, rank: int) -> dict:
    ri = basp_rank_info()
    _check(lib.basp_plan_get_rank(plan.handle, rank, byref(ri)), "basp_plan_get_rank")
    return {n: getattr(ri, n) for n, _ in basp_rank_info._fields_}


def basp_plan_group_ranks(plan: Plan, group: int) -> list[int]:
    out = (c_int * plan.K)()
    _check(lib.basp_plan_group_ranks(plan.handle, group, out), "basp_plan_group_ranks")
    return list(out)


def basp_reshard_s2h(plan, n_heads, seq_shards, head_shards, stream=None):
    _check(lib.basp_reshard_s2h(plan.handle, n_heads, _ptrs(seq_shards, plan.N), _ptrs(head_shards, plan.N),
                                _stream(stream)), "basp_reshard_s2h")


def basp_reshard_h2s(plan, n_heads, head_shards, seq_shards, stream=None):
    _check(lib.basp_reshard_h2s(plan.handle, n_heads, _ptrs(head_shards, plan.N), _ptrs(seq_shards, plan.N),
                                _stream(stream)), "basp_reshard_h2s")


def basp_reshard_qkv_s2h(plan, q_seq, k_seq, v_seq, q_head, k_head, v_head, stream=None):
    n = plan.N
    _check(lib.basp_reshard_qkv_s2h(plan.handle, _ptrs(q_seq, n), _ptrs(k_seq, n), _ptrs(v_seq, n),
                                    _ptrs(q_head, n), _ptrs(k_head, n), _ptrs(v_head, n), _stream(stream)),
           "basp_reshard_qkv_s2h")


def basp_attn_fwd(plan, q_head, k_head, v_head, o_head, lse_shards=None, softmax_scale=0.0, stream=None):
    n = plan.N
    _check(lib.basp_attn_fwd(plan.handle, _ptrs(q_head, n), _ptrs(k_head, n), _ptrs(v_head, n), _ptrs(o_head, n),
                             _ptrs(lse_shards, n), softmax_scale, _stream(stream)), "basp_attn_fwd")


def basp_workspace_bytes(plan) -> int:
    return int(lib.basp_workspace_bytes(plan.handle))


def basp_host_arena_bytes(plan) -> int:
    return int(lib.basp_host_arena_bytes(plan.handle))


def basp_layer_fwd(plan, q_seq, k_seq, v_seq, o_seq, workspace, lse_shards=None, softmax_scale=0.0, stream=None):
    n = plan.N
    _check(lib.basp_layer_fwd(plan.handle, _ptrs(q_seq, n), _ptrs(k_seq, n), _ptrs(v_seq, n), _ptrs(o_seq, n),
                              _ptrs(lse_shards, n), c_void_p(workspace.data_ptr()),
                              workspace.numel() * workspace.element_size(), softmax_scale, _stream(stream)),
           "basp_layer_fwd")


def basp_layer_fwd_fused(plan, q_seq, k_seq, v_seq, o_seq, lse_shards=None, softmax_scale=0.0, stream=None):
    n = plan.N
    _check(lib.basp_layer_fwd_fused(plan.handle, _ptrs(q_seq, n), _ptrs(k_seq, n), _ptrs(v_seq, n),
                                    _ptrs(o_seq, n), _ptrs(lse_shards, n), softmax_scale, _stream(stream)),
           "basp_layer_fwd_fused")


# ---- one physical GPU's share (ranks [rank_begin, rank_begin + rank_count)); shard lists may hold tensors, raw
# addresses of peer memory, or None for shards the call does not touch
def basp_reshard_qkv_s2h_ranks(plan, q_seq, k_seq, v_seq, q_head, k_head, v_head, rank_begin, rank_count, stream=None):
    n = plan.N
    _check(lib.basp_reshard_qkv_s2h_ranks(plan.handle, _ptrs(q_seq, n), _ptrs(k_seq, n), _ptrs(v_seq, n),
                                          _ptrs(q_head, n), _ptrs(k_head, n), _ptrs(v_head, n), rank_begin,
                                          rank_count, _stream(stream)), "basp_reshard_qkv_s2h_ranks")


def basp_reshard_h2s_ranks(plan, n_heads, head_shards, seq_shards, rank_begin, rank_count, stream=None):
    n = plan.N
    _check(lib.basp_reshard_h2s_ranks(plan.handle, n_heads, _ptrs(head_shards, n), _ptrs(seq_shards, n), rank_begin,
                                      rank_count, _stream(stream)), "basp_reshard_h2s_ranks")


def basp_attn_fwd_ranks(plan, q_head, k_head, v_head, o_head, rank_begin, rank_count, lse_shards=None,
                        softmax_scale=0.0, stream=None):
    n = plan.N
    _check(lib.basp_attn_fwd_ranks(plan.handle, _ptrs(q_head, n), _ptrs(k_head, n), _ptrs(v_head, n),
                                   _ptrs(o_head, n), _ptrs(lse_shards, n), softmax_scale, rank_begin, rank_count,
                                   _stream(stream)), "basp_attn_fwd_ranks")


def basp_layer_fwd_fused_ranks(plan, q_seq, k_seq, v_seq, o_seq, rank_begin, rank_count, lse_shards=None,
                               softmax_scale=0.0, stream=None):
    n = plan.N
    _check(lib.basp_layer_fwd_fused_ranks(plan.handle, _ptrs(q_seq, n), _ptrs(k_seq, n), _ptrs(v_seq, n),
                                          _ptrs(o_seq, n), _ptrs(lse_shards, n), softmax_scale, rank_begin,
                                          rank_count, _stream(stream)), "basp_layer_fwd_fused_ranks")


BASP_STATIC_SCRATCH_BYTES = 16 << 20


def basp_layer_fwd_static(plan, q_seq, k_seq, v_seq, o_seq, lse_shards=None, softmax_scale=0.0, stream=None):
    """The three-launch layer for callers that can neither allocate device memory nor pass a
    workspace: scratch is a fixed 16 MiB array inside the library (plans that need more are refused).
    Calls on one device share that array, so do not let two of them overlap on the GPU."""
    n = plan.N
    _check(lib.basp_layer_fwd_static(plan.handle, _ptrs(q_seq, n), _ptrs(k_seq, n), _ptrs(v_seq, n),
                                     _ptrs(o_seq, n), _ptrs(lse_shards, n), softmax_scale, _stream(stream)),
           "basp_layer_fwd_static")


def basp_layer_fwd_host(plan, q_seq_host, k_seq_host, v_seq_host, o_seq_host, device_arena, softmax_scale=0.0,
                        stream=None):
    n = plan.N
    _check(lib.basp_layer_fwd_host(plan.handle, _ptrs(q_seq_host, n), _ptrs(k_seq_host, n), _ptrs(v_seq_host, n),
                                   _ptrs(o_seq_host, n), c_void_p(device_arena.data_ptr()),
                                   device_arena.numel() * device_arena.element_size(), softmax_scale,
                                   _stream(stream)), "basp_layer_fwd_host")


def basp_layer_workspace_shards(plan, workspace):
    """Addresses (ints) of the head-sharded Q, K, V, O that basp_layer_fwd left in `workspace`:
    four lists of n_ranks device addresses."""
    n = plan.N
    arrs = [(c_void_p * n)() for _ in range(4)]
    _check(lib.basp_layer_workspace_shards(plan.handle, c_void_p(workspace.data_ptr()), *arrs),
           "basp_layer_workspace_shards")
    return [[int(a[i]) for i in range(n)] for a in arrs]


class _Addr:
    """A raw device address standing in for a tensor in the marshalling helpers."""

    def __init__(self, addr):
        self.addr = addr

    def data_ptr(self):
        return self.addr


def as_shards(addresses):
    return [_Addr(a) for a in addresses]


def basp_attn_bwd_workspace_bytes(plan) -> int:
    return int(lib.basp_attn_bwd_workspace_bytes(plan.handle))


def basp_layer_bwd_workspace_bytes(plan) -> int:
    return int(lib.basp_layer_bwd_workspace_bytes(plan.handle))


def basp_attn_bwd(plan, q_head, k_head, v_head, o_head, do_head, lse_shards, dq_head, dk_head, dv_head, workspace,
                  softmax_scale=0.0, stream=None, deterministic=False):
    n = plan.N
    fn = lib.basp_attn_bwd_deterministic if deterministic else lib.basp_attn_bwd
    _check(fn(plan.handle, *[_ptrs(t, n) for t in (q_head, k_head, v_head, o_head, do_head, lse_shards,
                                                                  dq_head, dk_head, dv_head)],
                             c_void_p(workspace.data_ptr()), workspace.numel() * workspace.element_size(),
                             softmax_scale, _stream(stream)), "basp_attn_bwd")


def basp_reshard_grads_h2s(plan, dq_head, dk_head, dv_head, dq_seq, dk_seq, dv_seq, stream=None):
    n = plan.N
    _check(lib.basp_reshard_grads_h2s(plan.handle, *[_ptrs(t, n) for t in (dq_head, dk_head, dv_head, dq_seq, dk_seq,
                                                                           dv_seq)], _stream(stream)),
           "basp_reshard_grads_h2s")


def basp_layer_bwd_seq_workspace_bytes(plan) -> int:
    return int(lib.basp_layer_bwd_seq_workspace_bytes(plan.handle))


def basp_layer_bwd_seq(plan, q_seq, k_seq, v_seq, o_seq, lse_shards, do_seq, dq_seq, dk_seq, dv_seq, workspace,
                       softmax_scale=0.0, stream=None):
    n = plan.N
    _check(lib.basp_layer_bwd_seq(plan.handle, *[_ptrs(t, n) for t in (q_seq, k_seq, v_seq, o_seq, lse_shards, do_seq,
                                                                       dq_seq, dk_seq, dv_seq)],
                                  c_void_p(workspace.data_ptr()), workspace.numel() * workspace.element_size(),
                                  softmax_scale, _stream(stream)), "basp_layer_bwd_seq")


def basp_layer_bwd(plan, q_head, k_head, v_head, o_head, lse_shards, do_seq, dq_seq, dk_seq, dv_seq, workspace,
                   softmax_scale=0.0, stream=None):
    n = plan.N
    _check(lib.basp_layer_bwd(plan.handle, *[_ptrs(t, n) for t in (q_head, k_head, v_head, o_head, lse_shards, do_seq,
                                                                   dq_seq, dk_seq, dv_seq)],
                              c_void_p(workspace.data_ptr()), workspace.numel() * workspace.element_size(),
                              softmax_scale, _stream(stream)), "basp_layer_bwd")


def basp_get_status(stream=None, raise_on_timeout=True):
    out = (c_int * 4)()
    rc = lib.basp_get_status(_stream(stream), out)
    if rc == BASP_ERR_TIMEOUT and not raise_on_timeout:
        return list(out)
    _check(rc, f"basp_get_status {list(out)}")
    return list(out)


def basp_clear_status(stream=None):
    _check(lib.basp_clear_status(_stream(stream)), "basp_clear_status")


def basp_qkv_proj(plan, hidden, x_seq, w_qkv, q_seq, k_seq, v_seq, stream=None):
    n = plan.N
    _check(lib.basp_qkv_proj(plan.handle, int(hidden), _ptrs(x_seq, n), c_void_p(w_qkv.data_ptr()), _ptrs(q_seq, n),
                             _ptrs(k_seq, n), _ptrs(v_seq, n), _stream(stream)), "basp_qkv_proj")


def basp_qkv_proj_rope(plan, hidden, x_seq, w_qkv, rope_cos, rope_sin, q_seq, k_seq, v_seq, stream=None):
    n = plan.N
    _check(lib.basp_qkv_proj_rope(plan.handle, int(hidden), _ptrs(x_seq, n), c_void_p(w_qkv.data_ptr()),
                                  c_void_p(rope_cos.data_ptr()), c_void_p(rope_sin.data_ptr()), _ptrs(q_seq, n),
                                  _ptrs(k_seq, n), _ptrs(v_seq, n), _stream(stream)), "basp_qkv_proj_rope")


def basp_out_proj(plan, hidden, o_seq, w_o, y_seq, stream=None):
    n = plan.N
    _check(lib.basp_out_proj(plan.handle, int(hidden), _ptrs(o_seq, n), c_void_p(w_o.data_ptr()), _ptrs(y_seq, n),
                             _stream(stream)), "basp_out_proj")


_BF16, _F32, _I64, _U8, _I32 = torch.bfloat16, torch.float32, torch.int64, torch.uint8, torch.int32


class _Marshal:
    """Pointer tables and checks of one call.  The library sees addresses only, so tensors that it would misread are refused
    here: wrong type or size, gaps between the elements, not in the current device's memory.  Raw addresses and objects with a
    data_ptr (as_shards) pass as they are."""

    __slots__ = ("device", "kept")

    def __init__(self):
        self.device = torch.cuda.current_device() if torch.cuda.is_initialized() else -2
        self.kept = None

    def _address(self, t, dtype, numel, what):
        if isinstance(t, torch.Tensor):
            if t.dtype != dtype or t.numel() != numel or not t.is_contiguous():
                raise ValueError(f"{what}: expected {numel} contiguous elements of {dtype}, got {tuple(t.shape)} of {t.dtype}"
                                 + ("" if t.is_contiguous() else ", not contiguous"))
            if not t.is_cuda:
                raise ValueError(f"{what} is on {t.device}: the library works on device memory")
            if t.get_device() != self.device:
                raise ValueError(f"{what} is on {t.device}, the current device is cuda:{self.device}")
            return t.data_ptr()
        return None if t is None else t.data_ptr() if hasattr(t, "data_ptr") else int(t)

    def addresses(self, *named):
        """One address for each (name, dtype, shards, sizes): of the table of a list's addresses (sizes: a tuple), of one tensor
        (sizes: its elements), None for None."""
        right = _fast_addresses(self.device, named)
        if right is not None:
            self.kept, out = right
            return out
        self.kept, out = [], []
        for what, dtype, shards, sizes in named:
            if shards is None:
                out.append(None)
            elif isinstance(sizes, int):
                out.append(self._address(shards, dtype, sizes, what))
            else:
                if len(shards) != len(sizes):
                    raise ValueError(f"expected {len(sizes)} shards, got {len(shards)}: {what}")
                table = (c_void_p * len(sizes))(*[self._address(t, dtype, n, f"{what}[{i}]")
                                                  for i, (t, n) in enumerate(zip(shards, sizes))])
                self.kept.append(table)
                out.append(ctypes.addressof(table))
        return out

    def space(self, workspace):
        """Address and size of a workspace tensor."""
        if workspace is None:
            return None, 0
        if workspace.get_device() != self.device or not workspace.is_contiguous():
            raise ValueError(f"workspace: expected contiguous memory of the current device, got a tensor on {workspace.device}")
        return workspace.data_ptr(), workspace.numel() * workspace.element_size()

    def stream(self, stream):
        if stream is None:
            return torch._C._cuda_getCurrentRawStream(self.device if self.device >= 0 else torch.cuda.current_device())
        return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _per_rank(plan, per_token):
    """Elements of every rank's sequence shard with `per_token` elements per token."""
    sizes = plan.sizes.get(per_token)
    if sizes is None:
        sizes = plan.sizes[per_token] = tuple(plan.Bl * plan.rank_tokens(r) * per_token for r in range(plan.N))
    return sizes


def _qk(plan):
    return _per_rank(plan, plan.Hq * plan.D), _per_rank(plan, plan.Hkv * plan.D)


def basp_qk_norm_rope(plan, q_seq, k_seq, w_q, w_k, rope_cos, rope_sin, q_out, k_out, eps=1e-6, stream=None):
    """Head norms of Q and K with the rotary embedding: z = x w / sqrt(mean(x^2) + eps), then the rotation of
    basp_qkv_proj_rope (same feature-major tables).  q_out[r] may be q_seq[r], k_out[r] may be k_seq[r]."""
    m, D, table = _Marshal(), plan.D, plan.D // 2 * plan.S
    q, k = _qk(plan)
    x, xk, wq, wk, cos, sin, y, yk = m.addresses(
        ("q_seq", _BF16, q_seq, q), ("k_seq", _BF16, k_seq, k), ("w_q", _BF16, w_q, D), ("w_k", _BF16, w_k, D),
        ("rope_cos", _F32, rope_cos, table), ("rope_sin", _F32, rope_sin, table), ("q_out", _BF16, q_out, q),
        ("k_out", _BF16, k_out, k))
    _check(lib.basp_qk_norm_rope(plan.handle, x, xk, wq, wk, cos, sin, eps, y, yk, m.stream(stream)), "basp_qk_norm_rope")


def basp_qk_norm_rope_bwd_workspace_bytes(plan) -> int:
    return int(lib.basp_qk_norm_rope_bwd_workspace_bytes(plan.handle))


def basp_qk_norm_rope_bwd(plan, q_seq, k_seq, w_q, w_k, rope_cos, rope_sin, dq_out, dk_out, dq_seq, dk_seq, dw_q, dw_k,
                          workspace, eps=1e-6, stream=None):
    """Gradients of basp_qk_norm_rope: dq_seq, dk_seq (bf16; may be dq_out, dk_out themselves) and dw_q, dw_k (fp32 [D])."""
    m, D, table = _Marshal(), plan.D, plan.D // 2 * plan.S
    q, k = _qk(plan)
    x, xk, wq, wk, cos, sin, dy, dyk, dx, dxk, gq, gk = m.addresses(
        ("q_seq", _BF16, q_seq, q), ("k_seq", _BF16, k_seq, k), ("w_q", _BF16, w_q, D), ("w_k", _BF16, w_k, D),
        ("rope_cos", _F32, rope_cos, table), ("rope_sin", _F32, rope_sin, table), ("dq_out", _BF16, dq_out, q),
        ("dk_out", _BF16, dk_out, k), ("dq_seq", _BF16, dq_seq, q), ("dk_seq", _BF16, dk_seq, k), ("dw_q", _F32, dw_q, D),
        ("dw_k", _F32, dw_k, D))
    _check(lib.basp_qk_norm_rope_bwd(plan.handle, x, xk, wq, wk, cos, sin, eps, dy, dyk, dx, dxk, gq, gk, *m.space(workspace),
                                     m.stream(stream)), "basp_qk_norm_rope_bwd")


def basp_ckpt_bytes(plan, rank) -> int:
    """Bytes of rank's 8-bit checkpoint of Q, K, V and O."""
    return int(lib.basp_ckpt_bytes(plan.handle, int(rank)))


def _ckpt_sizes(plan):
    sizes = plan.sizes.get("ckpt")
    if sizes is None:
        sizes = plan.sizes["ckpt"] = tuple(basp_ckpt_bytes(plan, r) for r in range(plan.N))
    return sizes


def basp_ckpt_pack(plan, q_seq, k_seq, v_seq, o_seq, ckpt, stream=None):
    """Q, K, V and O to 8 bits with one scale per head vector; ckpt[r]: uint8 tensor of basp_ckpt_bytes(plan, r)."""
    m = _Marshal()
    q, k = _qk(plan)
    a = m.addresses(("q_seq", _BF16, q_seq, q), ("k_seq", _BF16, k_seq, k), ("v_seq", _BF16, v_seq, k), ("o_seq", _BF16, o_seq, q),
                    ("ckpt", _U8, ckpt, _ckpt_sizes(plan)))
    _check(lib.basp_ckpt_pack(plan.handle, *a, m.stream(stream)), "basp_ckpt_pack")


def basp_ckpt_reshard_s2h(plan, ckpt, q_head, k_head, v_head, o_head, stream=None):
    """Checkpoints to head-sharded bf16 Q, K, V and O: the reading back and the all-to-all in one launch."""
    m, vec = _Marshal(), plan.Bl * plan.S * plan.D
    q, k = (vec * plan.Hq_l,) * plan.N, (vec * plan.Hkv_l,) * plan.N
    a = m.addresses(("ckpt", _U8, ckpt, _ckpt_sizes(plan)), ("q_head", _BF16, q_head, q), ("k_head", _BF16, k_head, k),
                    ("v_head", _BF16, v_head, k), ("o_head", _BF16, o_head, q))
    _check(lib.basp_ckpt_reshard_s2h(plan.handle, *a, m.stream(stream)), "basp_ckpt_reshard_s2h")


def basp_layer_bwd_ckpt(plan, ckpt, lse_shards, do_seq, dq_seq, dk_seq, dv_seq, workspace, softmax_scale=0.0, stream=None):
    """basp_layer_bwd_seq from the 8-bit checkpoints (workspace: basp_layer_bwd_seq_workspace_bytes)."""
    m = _Marshal()
    q, k = _qk(plan)
    a = m.addresses(("ckpt", _U8, ckpt, _ckpt_sizes(plan)),
                    ("lse_shards", _F32, lse_shards, (plan.Bl * plan.Hq_l * plan.S,) * plan.N), ("do_seq", _BF16, do_seq, q),
                    ("dq_seq", _BF16, dq_seq, q), ("dk_seq", _BF16, dk_seq, k), ("dv_seq", _BF16, dv_seq, k))
    _check(lib.basp_layer_bwd_ckpt(plan.handle, *a, *m.space(workspace), softmax_scale, m.stream(stream)), "basp_layer_bwd_ckpt")


def basp_lm_loss_fwd_workspace_bytes(plan, vocab) -> int:
    return int(lib.basp_lm_loss_fwd_workspace_bytes(plan.handle, int(vocab)))


def basp_lm_loss_grad_workspace_bytes(plan, hidden, vocab, piece_rows=0) -> int:
    return int(lib.basp_lm_loss_grad_workspace_bytes(plan.handle, int(hidden), int(vocab), int(piece_rows)))


def basp_lm_loss_fwd(plan, hidden, vocab, x_seq, w, labels, loss_seq, lse_seq, workspace, stream=None):
    """Per-token cross entropy of softmax(x W^T) against `labels` (int64; outside [0, vocab): no loss) and the log-sum-exp
    (lse_seq may be None), fp32."""
    m, n, hidden, vocab = _Marshal(), _per_rank(plan, 1), int(hidden), int(vocab)
    a = m.addresses(("x_seq", _BF16, x_seq, _per_rank(plan, hidden)), ("w", _BF16, w, vocab * hidden), ("labels", _I64, labels, n),
                    ("loss_seq", _F32, loss_seq, n), ("lse_seq", _F32, lse_seq, n))
    _check(lib.basp_lm_loss_fwd(plan.handle, hidden, vocab, *a, *m.space(workspace), m.stream(stream)),
           "basp_lm_loss_fwd")


def basp_lm_loss_grad(plan, hidden, vocab, x_seq, w, labels, token_weights, loss_seq, lse_seq, dx_seq, dw, workspace,
                      piece_rows=0, stream=None):
    """basp_lm_loss_fwd together with the gradients of sum(token_weights * loss): dx_seq and dw, bf16 (token_weights: fp32
    shards, or None for 1 each; dx_seq or dw None: not wanted)."""
    m, n, hidden, vocab = _Marshal(), _per_rank(plan, 1), int(hidden), int(vocab)
    wide = _per_rank(plan, hidden)
    a = m.addresses(("x_seq", _BF16, x_seq, wide), ("w", _BF16, w, vocab * hidden), ("labels", _I64, labels, n),
                    ("token_weights", _F32, token_weights, n), ("loss_seq", _F32, loss_seq, n), ("lse_seq", _F32, lse_seq, n),
                    ("dx_seq", _BF16, dx_seq, wide), ("dw", _BF16, dw, vocab * hidden))
    _check(lib.basp_lm_loss_grad(plan.handle, hidden, vocab, *a, int(piece_rows), *m.space(workspace), m.stream(stream)),
           "basp_lm_loss_grad")


def basp_mask_bytes(plan) -> int:
    return int(lib.basp_mask_bytes(plan.handle))


def _tokens(plan):
    """Tokens of the whole micro-batch, [B, S]."""
    return plan.cfg.micro_batch * plan.S


def _refilled(mask):
    """Tells torch that a mask object was written: a backward pass that has it saved is then refused, instead of taking another mask."""
    if not mask.is_inference():
        torch.autograd.graph.increment_version(mask)


def basp_mask_ranges(plan, key_begin, key_end, mask, stream=None):
    """The mask object of key ranges: query i of sequence b sees the keys [key_begin[b, i], key_end[b, i]) (int32 [B, S]);
    mask: uint8 tensor of basp_mask_bytes(plan)."""
    m, n = _Marshal(), _tokens(plan)
    a = m.addresses(("key_begin", _I32, key_begin, n), ("key_end", _I32, key_end, n))
    _check(lib.basp_mask_ranges(plan.handle, *a, *m.space(mask), m.stream(stream)), "basp_mask_ranges")
    _refilled(mask)


def basp_mask_packed(plan, positions, mask, prefix=None, window=0, stream=None):
    """The mask object of causal attention inside packed documents: positions in the own document (int32 [B, S], negative: padding),
    prefix: how many of the document's first tokens all of it sees (int32 [B, S] or None), window: keys back, itself included
    (0: all)."""
    m, n = _Marshal(), _tokens(plan)
    a = m.addresses(("positions", _I32, positions, n), ("prefix", _I32, prefix, n))
    _check(lib.basp_mask_packed(plan.handle, *a, int(window), *m.space(mask), m.stream(stream)), "basp_mask_packed")
    _refilled(mask)


_pack_score = struct.Struct("f4xPPN").pack          # the fields of _Score


class basp_score:
    """What a score goes through and which keys are seen: softcap c (0: none), slopes of the bias by distance (fp32 [Hq] or None),
    mask (a mask object, or None for the plan's own mask).  Holds its tensors."""

    def __init__(self, softcap=0.0, slopes=None, mask=None):
        self.softcap, self.slopes, self.mask = float(softcap), slopes, mask

    def pack(self, m, slopes):
        """The library's structure, `slopes`: the address."""
        mask, size = m.space(self.mask)
        return _pack_score(self.softcap, slopes or 0, mask or 0, size)


def _head_sizes(plan):
    sizes = plan.sizes.get("head")
    if sizes is None:
        vec, n = plan.Bl * plan.S, plan.N
        sizes = plan.sizes["head"] = ((vec * plan.Hq_l * plan.D,) * n, (vec * plan.Hkv_l * plan.D,) * n, (vec * plan.Hq_l,) * n)
    return sizes


def basp_attn_masked_fwd(plan, score, q_head, k_head, v_head, o_head, lse_shards=None, softmax_scale=0.0, stream=None):
    """basp_attn_fwd with capped, biased and masked scores (a basp_score); a query that sees no key has O = 0, LSE = -inf."""
    m, (q, k, rows) = _Marshal(), _head_sizes(plan)
    sl, *a = m.addresses(("slopes", _F32, score.slopes, plan.Hq), ("q_head", _BF16, q_head, q), ("k_head", _BF16, k_head, k),
                        ("v_head", _BF16, v_head, k), ("o_head", _BF16, o_head, q), ("lse_shards", _F32, lse_shards, rows))
    _check(lib.basp_attn_masked_fwd(plan.handle, score.pack(m, sl), *a, softmax_scale, m.stream(stream)), "basp_attn_masked_fwd")


def basp_attn_masked_bwd_workspace_bytes(plan) -> int:
    return int(lib.basp_attn_masked_bwd_workspace_bytes(plan.handle))


def basp_attn_masked_bwd(plan, score, q_head, k_head, v_head, o_head, do_head, lse_shards, dq_head, dk_head, dv_head, workspace,
                         softmax_scale=0.0, stream=None):
    """Gradients of basp_attn_masked_fwd from its O and LSE."""
    m, (q, k, rows) = _Marshal(), _head_sizes(plan)
    sl, *a = m.addresses(("slopes", _F32, score.slopes, plan.Hq), ("q_head", _BF16, q_head, q), ("k_head", _BF16, k_head, k), ("v_head", _BF16, v_head, k),
                    ("o_head", _BF16, o_head, q), ("do_head", _BF16, do_head, q), ("lse_shards", _F32, lse_shards, rows),
                    ("dq_head", _BF16, dq_head, q), ("dk_head", _BF16, dk_head, k), ("dv_head", _BF16, dv_head, k))
    _check(lib.basp_attn_masked_bwd(plan.handle, score.pack(m, sl), *a, *m.space(workspace), softmax_scale, m.stream(stream)), "basp_attn_masked_bwd")


def basp_layer_masked_fwd(plan, score, q_seq, k_seq, v_seq, o_seq, workspace, lse_shards=None, softmax_scale=0.0, stream=None):
    """basp_layer_fwd with such scores (same workspace)."""
    m, (q, k) = _Marshal(), _qk(plan)
    sl, *a = m.addresses(("slopes", _F32, score.slopes, plan.Hq), ("q_seq", _BF16, q_seq, q), ("k_seq", _BF16, k_seq, k), ("v_seq", _BF16, v_seq, k), ("o_seq", _BF16, o_seq, q),
                    ("lse_shards", _F32, lse_shards, _head_sizes(plan)[2]))
    _check(lib.basp_layer_masked_fwd(plan.handle, score.pack(m, sl), *a, *m.space(workspace), softmax_scale, m.stream(stream)), "basp_layer_masked_fwd")


def basp_layer_masked_bwd_workspace_bytes(plan) -> int:
    return int(lib.basp_layer_masked_bwd_workspace_bytes(plan.handle))


def basp_layer_masked_bwd(plan, score, q_head, k_head, v_head, o_head, lse_shards, do_seq, dq_seq, dk_seq, dv_seq, workspace,
                          softmax_scale=0.0, stream=None):
    """basp_layer_bwd with such scores (workspace: basp_layer_masked_bwd_workspace_bytes); q_head .. o_head as basp_layer_workspace_shards reports them."""
    m, (q, k) = _Marshal(), _qk(plan)
    qh, kh, rows = _head_sizes(plan)
    sl, *a = m.addresses(("slopes", _F32, score.slopes, plan.Hq), ("q_head", _BF16, q_head, qh), ("k_head", _BF16, k_head, kh), ("v_head", _BF16, v_head, kh),
                    ("o_head", _BF16, o_head, qh), ("lse_shards", _F32, lse_shards, rows), ("do_seq", _BF16, do_seq, q),
                    ("dq_seq", _BF16, dq_seq, q), ("dk_seq", _BF16, dk_seq, k), ("dv_seq", _BF16, dv_seq, k))
    _check(lib.basp_layer_masked_bwd(plan.handle, score.pack(m, sl), *a, *m.space(workspace), softmax_scale, m.stream(stream)), "basp_layer_masked_bwd")


_ROPE_SCALINGS = {"none": 0, "linear": 1, "yarn": 2, "wavelength": 3}


def basp_rope_make(rotary_dim, theta=10000.0, interleaved=False, scaling="none", factor=1.0, original_len=0.0, slow=0.0, fast=0.0,
                   attention_factor=0.0) -> basp_rope_turns:
    """The frequencies of a rotation, made once for a model.  scaling: "none", "linear", "yarn" (BASP_ROPE_BY_PARTS) or "wavelength",
    by `factor`; original_len: the length trained on; slow, fast: the borders in turns (0: the form's own); attention_factor: on the
    rotated features (0: the form's own)."""
    if scaling not in _ROPE_SCALINGS:
        raise ValueError(f"scaling: expected one of {sorted(_ROPE_SCALINGS)}, got {scaling!r}")
    cfg = basp_rope_config(int(rotary_dim), int(bool(interleaved)), _ROPE_SCALINGS[scaling], float(theta), float(factor),
                           float(original_len), float(slow), float(fast), float(attention_factor))
    out = basp_rope_turns()
    _check(lib.basp_rope_make(byref(cfg), byref(out)), "basp_rope_make")
    return out


def basp_rope(plan, rope, q_seq, k_seq, q_out, k_out, positions=None, inverse=False, stream=None):
    """Q and K rotated by their tokens' positions (int32 [B, S], None: the place in the sequence); inverse: the gradient of that.
    q_out[r] may be q_seq[r], k_out[r] may be k_seq[r]."""
    m, (q, k) = _Marshal(), _qk(plan)
    x, xk, pos, y, yk = m.addresses(("q_seq", _BF16, q_seq, q), ("k_seq", _BF16, k_seq, k), ("positions", _I32, positions, _tokens(plan)),
                                    ("q_out", _BF16, q_out, q), ("k_out", _BF16, k_out, k))
    _check(lib.basp_rope(plan.handle, byref(rope), x, xk, pos, int(bool(inverse)), y, yk, m.stream(stream)), "basp_rope")


def basp_block_norm(plan, hidden, x_seq, y_seq, h_seq, n_seq, w_post=None, gate=None, w_pre=None, res_scale=1.0, eps=1e-6, stream=None):
    """h = x + res_scale gate norm(y; w_post), n = norm(h; w_pre) on the ranks' rows of `hidden` features; w_post, gate (bf16 [hidden])
    None: not there; w_pre and n_seq None: no norm before the next block; y_seq and h_seq None: n of x alone."""
    m, hidden = _Marshal(), int(hidden)
    wide = _per_rank(plan, hidden)
    x, y, wp, g, wn, h, n = m.addresses(("x_seq", _BF16, x_seq, wide), ("y_seq", _BF16, y_seq, wide), ("w_post", _BF16, w_post, hidden),
                                        ("gate", _BF16, gate, hidden), ("w_pre", _BF16, w_pre, hidden), ("h_seq", _BF16, h_seq, wide),
                                        ("n_seq", _BF16, n_seq, wide))
    _check(lib.basp_block_norm(plan.handle, hidden, x, y, wp, g, wn, float(res_scale), float(eps), h, n, m.stream(stream)), "basp_block_norm")


def basp_block_norm_bwd_workspace_bytes(plan, hidden) -> int:
    return int(lib.basp_block_norm_bwd_workspace_bytes(plan.handle, int(hidden)))


def basp_block_norm_bwd(plan, hidden, h_seq, y_seq, dh_out, dn, dx_seq, dy_seq, dw_post, dgate, dw_pre, workspace, w_post=None,
                        gate=None, w_pre=None, res_scale=1.0, eps=1e-6, stream=None):
    """Gradients of basp_block_norm: dx_seq, dy_seq (bf16) and dw_post, dgate, dw_pre (fp32 [hidden]) from h, y and the gradients that
    reach h elsewhere (dh_out, None: none) and n (dn)."""
    m, hidden = _Marshal(), int(hidden)
    wide = _per_rank(plan, hidden)
    h, y, wp, g, wn, dh, d, dx, dy, gp, gg, gn = m.addresses(
        ("h_seq", _BF16, h_seq, wide), ("y_seq", _BF16, y_seq, wide), ("w_post", _BF16, w_post, hidden), ("gate", _BF16, gate, hidden),
        ("w_pre", _BF16, w_pre, hidden), ("dh_out", _BF16, dh_out, wide), ("dn", _BF16, dn, wide), ("dx_seq", _BF16, dx_seq, wide),
        ("dy_seq", _BF16, dy_seq, wide), ("dw_post", _F32, dw_post, hidden), ("dgate", _F32, dgate, hidden), ("dw_pre", _F32, dw_pre, hidden))
    _check(lib.basp_block_norm_bwd(plan.handle, hidden, h, y, wp, g, wn, float(res_scale), float(eps), dh, d, dx, dy, gp, gg, gn,
                                   *m.space(workspace), m.stream(stream)), "basp_block_norm_bwd")


def basp_selftest_wait_timeout(limit_us: int, stream=None):
    _check(lib.basp_selftest_wait_timeout(int(limit_us), _stream(stream)), "basp_selftest_wait_timeout")


def basp_launch_count() -> int:
    return int(lib.basp_launch_count())
