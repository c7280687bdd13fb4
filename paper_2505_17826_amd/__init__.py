"""MI355X (gfx950) core of a GRPO/PPO reinforcement fine-tuning trainer step.

A thin ctypes binding of ``librft.so``; every function keeps the name of the
C entry point it marshals (``include/rft.h``).  torch supplies device memory
and the current HIP stream; every step of the computation runs in the
library's HIP kernels.  There is no CPU fallback: if the library is missing
or no GPU is present the calls raise.
"""
from __future__ import annotations

import ctypes
import functools
import inspect
import math
import os
import struct
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librft.so")

RFT_OK, RFT_E_NULL, RFT_E_SHAPE, RFT_E_DTYPE, RFT_E_PARAM, RFT_E_WORKSPACE, \
    RFT_E_UNSUPPORTED, RFT_E_HIP = range(8)
RFT_F32, RFT_BF16 = 0, 1
RFT_AGG_SEQ_MEAN_TOKEN_MEAN, RFT_AGG_TOKEN_MEAN = 0, 1
RFT_ADV_GRPO, RFT_ADV_MEAN_CENTER, RFT_ADV_LEAVE_ONE_OUT = 0, 1, 2
RFT_BALANCE_BATCH, RFT_BALANCE_ROLLOUT = 0, 1
RFT_PRODUCTS_BY_TYPE, RFT_PRODUCTS_ONE, RFT_PRODUCTS_THREE = 0, 1, 3
(RFT_OP_TOKEN_LOGPROBS, RFT_OP_TOKEN_LOGPROBS_FROM_LOGITS, RFT_OP_PPO_FWD, RFT_OP_PPO_BWD,
 RFT_OP_PPO_BWD_LOGITS, RFT_OP_PPO_FUSED_LOGITS, RFT_OP_PPO_STEP, RFT_OP_SFT_FWD,
 RFT_OP_DPO_FWD) = range(9)

_p = ctypes.c_void_p
_i64 = ctypes.c_int64


class rft_tokens(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int64), ("n_seq", ctypes.c_int64), ("seq_start", _p),
                ("mask", _p), ("token_ids", _p), ("is_expert", _p)]


class rft_ppo_params(ctypes.Structure):
    _fields_ = [("eps_low", ctypes.c_float), ("eps_high", ctypes.c_float),
                ("kl_coef", ctypes.c_float), ("agg", ctypes.c_int32),
                ("denom_override", ctypes.c_double), ("mix_mu", ctypes.c_float),
                ("entropy_coef", ctypes.c_float)]


class rft_ppo_stats(ctypes.Structure):
    _fields_ = [("loss", ctypes.c_double), ("pg_loss", ctypes.c_double),
                ("kl_loss", ctypes.c_double), ("kl_mean", ctypes.c_double),
                ("entropy_mean", ctypes.c_double), ("ratio_mean", ctypes.c_double),
                ("clipfrac", ctypes.c_double), ("n_valid", ctypes.c_int64),
                ("n_seq_valid", ctypes.c_int64), ("n_clipped", ctypes.c_int64),
                ("n_bad_ids", ctypes.c_int64), ("sft_loss", ctypes.c_double),
                ("n_expert", ctypes.c_int64), ("entropy_loss", ctypes.c_double)]


class rft_dpo_stats(ctypes.Structure):
    _fields_ = [("loss", ctypes.c_double), ("chosen_reward", ctypes.c_double),
                ("rejected_reward", ctypes.c_double), ("reward_acc", ctypes.c_double),
                ("margin_mean", ctypes.c_double), ("n_pairs", ctypes.c_int64),
                ("n_valid", ctypes.c_int64), ("n_bad_ids", ctypes.c_int64)]


class rft_router_params(ctypes.Structure):
    _fields_ = [("n_experts", ctypes.c_int32), ("top_k", ctypes.c_int32),
                ("norm_topk", ctypes.c_int32), ("scope", ctypes.c_int32),
                ("balance_coef", ctypes.c_float), ("z_coef", ctypes.c_float)]


class rft_router_stats(ctypes.Structure):
    _fields_ = [("loss", ctypes.c_float), ("balance_loss", ctypes.c_float),
                ("z_loss", ctypes.c_float), ("max_count", ctypes.c_int32),
                ("n_valid", ctypes.c_int32), ("n_groups", ctypes.c_int32)]


class rft_param(ctypes.Structure):
    _fields_ = [("weight", _p), ("grad", _p), ("m", _p), ("v", _p), ("master", _p), ("n", _i64)]


class rft_clip(ctypes.Structure):
    _fields_ = [("norm", ctypes.c_float), ("scale", ctypes.c_float), ("finite", ctypes.c_int32)]


class rft_adamw_params(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("weight_decay", ctypes.c_double), ("step", _i64)]


class rft_matrices(ctypes.Structure):
    _fields_ = [("batch", _i64), ("rows", _i64), ("cols", _i64), ("row_stride", _i64),
                ("batch_stride", _i64)]


class rft_muon_params(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("momentum", ctypes.c_double),
                ("weight_decay", ctypes.c_double), ("scale", ctypes.c_double),
                ("a", ctypes.c_double), ("b", ctypes.c_double), ("c", ctypes.c_double),
                ("eps", ctypes.c_double), ("steps", ctypes.c_int32), ("nesterov", ctypes.c_int32),
                ("products", ctypes.c_int32)]


STATS_BYTES = ctypes.sizeof(rft_ppo_stats)
DPO_STATS_BYTES = ctypes.sizeof(rft_dpo_stats)

_SIGS = {
    "rft_abi_version": (ctypes.c_int, []),
    "rft_status_str": (ctypes.c_char_p, [ctypes.c_int]),
    "rft_last_error": (ctypes.c_char_p, []),
    "rft_workspace_bytes": (ctypes.c_size_t, [ctypes.c_int, ctypes.POINTER(rft_tokens), _i64, _i64,
                                              ctypes.c_int]),
    "rft_workspace_min_bytes": (ctypes.c_size_t, [ctypes.c_int, ctypes.POINTER(rft_tokens), _i64,
                                                  _i64, ctypes.c_int]),
    "rft_noalloc_scratch_bytes": (ctypes.c_size_t, []),
    "rft_ppo_clip_fused_logits_noalloc": (ctypes.c_int, [ctypes.POINTER(rft_tokens), _p, _i64, _p,
                                                         _p, _p, ctypes.POINTER(rft_ppo_params),
                                                         _p, _p, _p, _p, _p, _p, _p]),
    "rft_workspace_bytes_rows": (ctypes.c_size_t, [ctypes.c_int, ctypes.POINTER(rft_tokens), _i64,
                                                   _i64, ctypes.c_int, _i64]),
    "rft_chunk_rows": (_i64, [ctypes.c_int, ctypes.POINTER(rft_tokens), _i64, _i64, ctypes.c_int,
                              ctypes.c_size_t]),
    "rft_group_advantages": (ctypes.c_int, [_p, _i64, ctypes.c_int32, ctypes.c_float, ctypes.c_int32,
                                            _p, _p]),
    "rft_group_advantages_ids_workspace_bytes": (ctypes.c_size_t, [_i64, _i64]),
    "rft_group_advantages_ids": (ctypes.c_int, [_p, _p, _i64, _i64, ctypes.c_int32, ctypes.c_float,
                                                ctypes.c_int32, _p, _p, ctypes.c_size_t, _p]),
    "rft_token_logprobs": (ctypes.c_int, [ctypes.POINTER(rft_tokens), _p, _p, ctypes.c_int, _i64,
                                          _i64, _p, _p, _p, _p, ctypes.c_size_t, _p]),
    "rft_token_logprobs_from_logits": (ctypes.c_int, [ctypes.POINTER(rft_tokens), _p, _i64, _p,
                                                      _p, _p, _p, _p, ctypes.c_size_t, _p]),
    "rft_ppo_clip_loss_fwd": (ctypes.c_int, [ctypes.POINTER(rft_tokens), _i64, _p, _p, _p, _p, _p,
                                             ctypes.POINTER(rft_ppo_params), _p, _p, _p, _p,
                                             ctypes.c_size_t, _p]),
    "rft_ppo_clip_loss_bwd": (ctypes.c_int, [ctypes.POINTER(rft_tokens), _p, _p, ctypes.c_int, _i64,
                                             _i64, _p, _p, _p, _p, _p, _p, ctypes.c_int32, _p,
                                             ctypes.c_size_t, _p]),
    "rft_ppo_clip_loss_bwd_logits": (ctypes.c_int, [ctypes.POINTER(rft_tokens), _p, _i64, _p, _p,
                                                    _p, _p, _p, _p, ctypes.c_size_t, _p]),
    "rft_ppo_clip_fused_logits": (ctypes.c_int, [ctypes.POINTER(rft_tokens), _p, _i64, _p, _p, _p,
                                                 ctypes.POINTER(rft_ppo_params), _p, _p, _p, _p,
                                                 _p, _p, _p, ctypes.c_size_t, _p]),
    "rft_ppo_clip_step": (ctypes.c_int, [ctypes.POINTER(rft_tokens), _p, _p, ctypes.c_int, _i64,
                                         _i64, _p, _p, _p, ctypes.POINTER(rft_ppo_params), _p, _p,
                                         _p, _p, _p, _p, ctypes.c_int32, _p, _p, ctypes.c_size_t,
                                         _p]),
    "rft_sft_loss_fwd": (ctypes.c_int, [ctypes.POINTER(rft_tokens), _i64, _p, ctypes.c_int32,
                                        ctypes.c_double, _p, _p, _p, ctypes.c_size_t, _p]),
    "rft_dpo_loss_fwd": (ctypes.c_int, [ctypes.POINTER(rft_tokens), _i64, _p, _p, ctypes.c_float,
                                        ctypes.c_float, _p, _p, _p, _p, ctypes.c_size_t, _p]),
    "rft_router_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(rft_tokens),
                                                     ctypes.POINTER(rft_router_params)]),
    "rft_router_fwd": (ctypes.c_int, [ctypes.POINTER(rft_tokens), _p, ctypes.c_int, _i64,
                                      ctypes.POINTER(rft_router_params), _p, _p, _p, _p, _p, _p,
                                      _p, ctypes.c_size_t, _p]),
    "rft_router_bwd": (ctypes.c_int, [ctypes.POINTER(rft_tokens), _p, ctypes.c_int, _i64,
                                      ctypes.POINTER(rft_router_params), _p, _p, _p, _p, _p, _p,
                                      _i64, _p]),
    "rft_grad_norm_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(rft_param), _i64]),
    "rft_grad_norm": (ctypes.c_int, [ctypes.POINTER(rft_param), _i64, ctypes.c_int, ctypes.c_float,
                                     _p, _p, ctypes.c_size_t, _p]),
    "rft_adamw_step": (ctypes.c_int, [ctypes.POINTER(rft_param), _i64, ctypes.c_int, ctypes.c_int,
                                      ctypes.POINTER(rft_adamw_params), _p, _p]),
    "rft_orthogonalize_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(rft_matrices),
                                                            ctypes.POINTER(rft_muon_params),
                                                            ctypes.c_int]),
    "rft_orthogonalize": (ctypes.c_int, [ctypes.POINTER(rft_matrices), _p, ctypes.c_int,
                                         ctypes.POINTER(rft_muon_params), _p, ctypes.c_int, _p,
                                         ctypes.c_size_t, _p]),
    "rft_muon_step": (ctypes.c_int, [ctypes.POINTER(rft_matrices), _p, ctypes.c_int, _p, _p,
                                     ctypes.c_int, _p, ctypes.POINTER(rft_muon_params), _p, _p,
                                     ctypes.c_size_t, _p]),
}

_LIB = None


def lib() -> ctypes.CDLL:
    """Load librft.so (built in-tree by ``build_lib``); raise if it is missing."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run python -m paper_2505_17826_amd.build_lib")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _LIB = L
    return _LIB


class RftError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"{msg} (status {status})")
        self.status = status


def _check(st):
    if st != RFT_OK:
        L = lib()
        raise RftError(st, L.rft_last_error().decode())


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _need_gpu(*ts):
    for t in ts:
        if t is not None and t.device.type != "cuda":
            raise RuntimeError("librft works on device tensors only (no CPU fallback)")


def _dtype_code(t):
    if t.dtype == torch.bfloat16:
        return RFT_BF16
    if t.dtype == torch.float32:
        return RFT_F32
    raise TypeError(f"unsupported dtype {t.dtype}")


@dataclass
class Tokens:
    """Token layout of one batch: rollout row offsets, action mask, sampled ids
    (not needed by the router), and optionally per-rollout expert flags (MIX)."""
    seq_start: torch.Tensor   # int32 [n_seq + 1]
    mask: torch.Tensor        # uint8 [T]
    token_ids: torch.Tensor = None  # int32 [T]
    is_expert: torch.Tensor = None  # uint8 [n_seq] or None

    @property
    def T(self):
        return int(self.mask.numel())

    @property
    def n_seq(self):
        return int(self.seq_start.numel()) - 1

    def c(self) -> rft_tokens:
        for t, dt in ((self.seq_start, torch.int32), (self.mask, torch.uint8),
                      (self.token_ids, torch.int32)):
            if t is None and t is self.token_ids:
                continue
            if t.dtype != dt or not t.is_contiguous():
                raise TypeError("tokens: seq_start int32, mask uint8, token_ids int32, contiguous")
        ex = None
        if self.is_expert is not None:
            if (self.is_expert.dtype != torch.uint8 or not self.is_expert.is_contiguous()
                    or self.is_expert.numel() != self.n_seq):
                raise TypeError("tokens: is_expert must be contiguous uint8 [n_seq]")
            ex = self.is_expert.data_ptr()
        ids = None if self.token_ids is None else self.token_ids.data_ptr()
        return rft_tokens(self.T, self.n_seq, self.seq_start.data_ptr(), self.mask.data_ptr(),
                          ids, ex)


def ppo_params(eps_low=0.2, eps_high=0.2, kl_coef=0.0, agg=RFT_AGG_SEQ_MEAN_TOKEN_MEAN,
               denom_override=0.0, mix_mu=0.0, entropy_coef=0.0) -> rft_ppo_params:
    return rft_ppo_params(eps_low, eps_high, kl_coef, agg, denom_override, mix_mu, entropy_coef)


def stats_to_dict(buf: torch.Tensor, kind=None) -> dict:
    """Decode an rft_ppo_stats (or, with kind=rft_dpo_stats, an rft_dpo_stats)
    device buffer (synchronises on the copy)."""
    kind = rft_ppo_stats if kind is None else kind
    raw = bytes(buf.detach().cpu().numpy().tobytes())
    s = kind.from_buffer_copy(raw[:ctypes.sizeof(kind)])
    return {k: getattr(s, k) for k, _ in kind._fields_}


def workspace_bytes(op, tokens: Tokens, d=0, V=1, dtype=RFT_F32, minimum=False) -> int:
    L = lib()
    tk = tokens.c()
    f = L.rft_workspace_min_bytes if minimum else L.rft_workspace_bytes
    return int(f(op, ctypes.byref(tk), d, V, dtype))


def workspace_bytes_rows(op, tokens: Tokens, d, V, dtype, rows) -> int:
    """Workspace with which RFT_OP_PPO_BWD / RFT_OP_PPO_STEP runs row chunks of `rows` rows."""
    tk = tokens.c()
    return int(lib().rft_workspace_bytes_rows(op, ctypes.byref(tk), d, V, dtype, rows))


def chunk_rows(op, tokens: Tokens, d, V, dtype, ws_bytes) -> int:
    tk = tokens.c()
    return int(lib().rft_chunk_rows(op, ctypes.byref(tk), d, V, dtype, ws_bytes))


def _workspace(nbytes, device, ws=None):
    if nbytes == 0:
        return None, 0
    if ws is not None:
        return ws, ws.numel() * ws.element_size()
    return torch.empty(nbytes, dtype=torch.uint8, device=device), nbytes


def _used_on(stream, *ts):
    """Tells the allocator that arrays are used on a stream other than the one that they were
    allocated on (they may be freed before its work is done)."""
    for t in ts:
        if t is not None and t.numel():
            t.record_stream(stream)


def _arrays(x):
    """The tensors of an entry point's result."""
    if isinstance(x, torch.Tensor):
        return [x]
    if isinstance(x, tuple):
        return [t for y in x for t in _arrays(y)]
    return [] if x is None else [t for y in vars(x).values() for t in _arrays(y)]


def _allocates(f):
    """An entry point that makes its workspace, or results that are not given.  With stream=
    its body runs with that stream current, so that these are that stream's memory: a block
    of the caller's current stream may have been freed by it with work still pending there,
    and a fill there would not be ordered with the call.  The results then belong to the
    caller, whose stream reads them: the allocator is told so."""
    at = list(inspect.signature(f).parameters).index("stream")

    @functools.wraps(f)
    def call(*args, **kw):
        stream = args[at] if len(args) > at else kw.get("stream")
        if stream is None:
            return f(*args, **kw)
        for t in (*args, *kw.values()):
            if isinstance(t, torch.Tensor) and t.device != stream.device:
                raise RuntimeError(f"an array is on {t.device}, stream is of {stream.device}")
        callers = torch.cuda.current_stream(stream.device)
        with torch.cuda.stream(stream):
            out = f(*args, **kw)
        if callers != stream:
            _used_on(callers, *_arrays(out))
        return out

    return call


# ------------------------------------------------------------ entry points --
@_allocates
def rft_group_advantages(rewards, group_size, eps=1e-6, out=None, stream=None, unbiased=True):
    _need_gpu(rewards)
    out = torch.empty_like(rewards) if out is None else out
    n_groups = rewards.numel() // group_size if group_size > 0 else 0
    _check(lib().rft_group_advantages(_ptr(rewards), n_groups, group_size, eps,
                                      1 if unbiased else 0, _ptr(out), _stream(stream)))
    return out


@_allocates
def rft_group_advantages_ids(rewards, group_id, n_groups, mode=RFT_ADV_GRPO, eps=1e-6, out=None,
                             stream=None, unbiased=True, ws=None):
    _need_gpu(rewards, group_id)
    out = torch.empty_like(rewards) if out is None else out
    need = int(lib().rft_group_advantages_ids_workspace_bytes(rewards.numel(), n_groups))
    ws, nb = _workspace(need, rewards.device, ws)
    _check(lib().rft_group_advantages_ids(_ptr(rewards), _ptr(group_id), rewards.numel(), n_groups,
                                          mode, eps, 1 if unbiased else 0, _ptr(out), _ptr(ws), nb,
                                          _stream(stream)))
    return out


@_allocates
def rft_token_logprobs(tokens: Tokens, hidden, weight, logp=None, entropy=None, lse=None, ws=None,
                       stream=None, want_entropy=True):
    _need_gpu(hidden, weight)
    T, dev = tokens.T, hidden.device
    d, V = hidden.shape[1], weight.shape[0]
    dt = _dtype_code(hidden)
    logp = torch.empty(T, dtype=torch.float32, device=dev) if logp is None else logp
    lse = torch.empty(T, dtype=torch.float32, device=dev) if lse is None else lse
    if entropy is None and want_entropy:
        entropy = torch.empty(T, dtype=torch.float32, device=dev)
    need = workspace_bytes(RFT_OP_TOKEN_LOGPROBS, tokens, d, V, dt)
    ws, nb = _workspace(need, dev, ws)
    tk = tokens.c()
    _check(lib().rft_token_logprobs(ctypes.byref(tk), _ptr(hidden), _ptr(weight), dt, d, V,
                                    _ptr(logp), _ptr(entropy), _ptr(lse), _ptr(ws), nb,
                                    _stream(stream)))
    return logp, entropy, lse


@_allocates
def rft_token_logprobs_from_logits(tokens: Tokens, logits, logp=None, entropy=None, lse=None,
                                   gathered=None, want_gathered=False, stream=None):
    _need_gpu(logits)
    T, dev, V = tokens.T, logits.device, logits.shape[1]
    logp = torch.empty(T, dtype=torch.float32, device=dev) if logp is None else logp
    lse = torch.empty(T, dtype=torch.float32, device=dev) if lse is None else lse
    entropy = torch.empty(T, dtype=torch.float32, device=dev) if entropy is None else entropy
    if gathered is None and want_gathered:
        gathered = torch.empty(T, dtype=torch.float32, device=dev)
    tk = tokens.c()
    _check(lib().rft_token_logprobs_from_logits(ctypes.byref(tk), _ptr(logits), V, _ptr(logp),
                                                _ptr(entropy), _ptr(lse), _ptr(gathered), None, 0,
                                                _stream(stream)))
    return logp, entropy, lse, gathered


@_allocates
def rft_ppo_clip_loss_fwd(tokens: Tokens, V, logp, old_logp, ref_logp, adv, params, entropy=None,
                          grad_logp=None, stats=None, ws=None, stream=None, grad_entropy=None):
    """Returns (grad_logp, stats); grad_entropy, when given, receives e_t."""
    _need_gpu(logp, old_logp, adv)
    dev = logp.device
    grad_logp = torch.empty_like(logp) if grad_logp is None else grad_logp
    stats = torch.zeros(STATS_BYTES, dtype=torch.uint8, device=dev) if stats is None else stats
    need = workspace_bytes(RFT_OP_PPO_FWD, tokens, 0, V)
    ws, nb = _workspace(need, dev, ws)
    tk = tokens.c()
    _check(lib().rft_ppo_clip_loss_fwd(ctypes.byref(tk), V, _ptr(logp), _ptr(old_logp),
                                       _ptr(ref_logp), _ptr(adv), _ptr(entropy),
                                       ctypes.byref(params), _ptr(grad_logp), _ptr(grad_entropy),
                                       _ptr(stats), _ptr(ws), nb, _stream(stream)))
    return grad_logp, stats


@_allocates
def rft_ppo_clip_loss_bwd(tokens: Tokens, hidden, weight, lse, grad_logp, d_hidden=None,
                          d_weight=None, accumulate_dw=False, ws=None, stream=None,
                          grad_entropy=None, entropy=None):
    _need_gpu(hidden, weight, lse, grad_logp)
    dev = hidden.device
    T, d, V = tokens.T, hidden.shape[1], weight.shape[0]
    dt = _dtype_code(hidden)
    d_hidden = torch.empty((T, d), dtype=torch.float32, device=dev) if d_hidden is None else d_hidden
    d_weight = torch.empty((V, d), dtype=torch.float32, device=dev) if d_weight is None else d_weight
    need = workspace_bytes(RFT_OP_PPO_BWD, tokens, d, V, dt)
    ws, nb = _workspace(need, dev, ws)
    tk = tokens.c()
    _check(lib().rft_ppo_clip_loss_bwd(ctypes.byref(tk), _ptr(hidden), _ptr(weight), dt, d, V,
                                       _ptr(lse), _ptr(grad_logp), _ptr(grad_entropy),
                                       _ptr(entropy), _ptr(d_hidden), _ptr(d_weight),
                                       1 if accumulate_dw else 0, _ptr(ws), nb, _stream(stream)))
    return d_hidden, d_weight


@_allocates
def rft_ppo_clip_loss_bwd_logits(tokens: Tokens, logits, lse, grad_logp, d_logits=None,
                                 stream=None, grad_entropy=None, entropy=None):
    _need_gpu(logits, lse, grad_logp)
    d_logits = torch.empty_like(logits) if d_logits is None else d_logits
    tk = tokens.c()
    _check(lib().rft_ppo_clip_loss_bwd_logits(ctypes.byref(tk), _ptr(logits), logits.shape[1],
                                              _ptr(lse), _ptr(grad_logp), _ptr(grad_entropy),
                                              _ptr(entropy), _ptr(d_logits), None, 0,
                                              _stream(stream)))
    return d_logits


@_allocates
def rft_ppo_clip_fused_logits(tokens: Tokens, logits, old_logp, ref_logp, adv, params, logp=None,
                              entropy=None, lse=None, grad_logp=None, d_logits=None, stats=None,
                              ws=None, stream=None):
    _need_gpu(logits, old_logp, adv)
    T, dev, V = tokens.T, logits.device, logits.shape[1]
    logp = torch.empty(T, dtype=torch.float32, device=dev) if logp is None else logp
    d_logits = torch.empty_like(logits) if d_logits is None else d_logits
    stats = torch.zeros(STATS_BYTES, dtype=torch.uint8, device=dev) if stats is None else stats
    need = workspace_bytes(RFT_OP_PPO_FUSED_LOGITS, tokens, 0, V)
    ws, nb = _workspace(need, dev, ws)
    tk = tokens.c()
    _check(lib().rft_ppo_clip_fused_logits(ctypes.byref(tk), _ptr(logits), V, _ptr(old_logp),
                                           _ptr(ref_logp), _ptr(adv), ctypes.byref(params),
                                           _ptr(logp), _ptr(entropy), _ptr(lse), _ptr(grad_logp),
                                           _ptr(d_logits), _ptr(stats), _ptr(ws), nb,
                                           _stream(stream)))
    return logp, d_logits, stats


def rft_ppo_clip_fused_logits_noalloc(tokens: Tokens, logits, old_logp, ref_logp, adv, params,
                                      logp, d_logits, stats, entropy=None, lse=None,
                                      grad_logp=None, stream=None):
    """rft_ppo_clip_fused_logits without a workspace: the library's own scratch
    array is used and nothing is allocated, so every output must be given."""
    _need_gpu(logits, old_logp, adv, logp, d_logits, stats)
    tk = tokens.c()
    _check(lib().rft_ppo_clip_fused_logits_noalloc(
        ctypes.byref(tk), _ptr(logits), logits.shape[1], _ptr(old_logp), _ptr(ref_logp),
        _ptr(adv), ctypes.byref(params), _ptr(logp), _ptr(entropy), _ptr(lse), _ptr(grad_logp),
        _ptr(d_logits), _ptr(stats), _stream(stream)))
    return logp, d_logits, stats


@_allocates
def rft_ppo_clip_step(tokens: Tokens, hidden, weight, old_logp, ref_logp, adv, params,
                      logp=None, entropy=None, lse=None, grad_logp=None, d_hidden=None,
                      d_weight=None, accumulate_dw=False, stats=None, ws=None, stream=None):
    """Returns (logp, entropy, lse, grad_logp, d_hidden, d_weight, stats)."""
    _need_gpu(hidden, weight, old_logp, adv)
    dev = hidden.device
    T, d, V = tokens.T, hidden.shape[1], weight.shape[0]
    dt = _dtype_code(hidden)
    f32 = dict(dtype=torch.float32, device=dev)
    logp = torch.empty(T, **f32) if logp is None else logp
    entropy = torch.empty(T, **f32) if entropy is None else entropy
    lse = torch.empty(T, **f32) if lse is None else lse
    grad_logp = torch.empty(T, **f32) if grad_logp is None else grad_logp
    d_hidden = torch.empty((T, d), **f32) if d_hidden is None else d_hidden
    d_weight = torch.empty((V, d), **f32) if d_weight is None else d_weight
    stats = torch.zeros(STATS_BYTES, dtype=torch.uint8, device=dev) if stats is None else stats
    need = workspace_bytes(RFT_OP_PPO_STEP, tokens, d, V, dt)
    ws, nb = _workspace(need, dev, ws)
    tk = tokens.c()
    _check(lib().rft_ppo_clip_step(ctypes.byref(tk), _ptr(hidden), _ptr(weight), dt, d, V,
                                   _ptr(old_logp), _ptr(ref_logp), _ptr(adv), ctypes.byref(params),
                                   _ptr(logp), _ptr(entropy), _ptr(lse), _ptr(grad_logp),
                                   _ptr(d_hidden), _ptr(d_weight), 1 if accumulate_dw else 0,
                                   _ptr(stats), _ptr(ws), nb, _stream(stream)))
    return logp, entropy, lse, grad_logp, d_hidden, d_weight, stats


@_allocates
def rft_sft_loss_fwd(tokens: Tokens, V, logp, agg=RFT_AGG_TOKEN_MEAN, denom_override=0.0,
                     grad_logp=None, stats=None, ws=None, stream=None):
    """Returns (grad_logp, stats)."""
    _need_gpu(logp)
    dev = logp.device
    grad_logp = torch.empty_like(logp) if grad_logp is None else grad_logp
    stats = torch.zeros(STATS_BYTES, dtype=torch.uint8, device=dev) if stats is None else stats
    ws, nb = _workspace(workspace_bytes(RFT_OP_SFT_FWD, tokens, 0, V), dev, ws)
    tk = tokens.c()
    _check(lib().rft_sft_loss_fwd(ctypes.byref(tk), V, _ptr(logp), agg, denom_override,
                                  _ptr(grad_logp), _ptr(stats), _ptr(ws), nb, _stream(stream)))
    return grad_logp, stats


@_allocates
def rft_dpo_loss_fwd(tokens: Tokens, V, logp, ref_logp, beta=0.1, label_smoothing=0.0,
                     grad_logp=None, seq_logp=None, want_seq_logp=True, stats=None, ws=None,
                     stream=None):
    """Returns (grad_logp, seq_logp, stats); decode stats with
    stats_to_dict(stats, rft_dpo_stats)."""
    _need_gpu(logp, ref_logp)
    dev = logp.device
    grad_logp = torch.empty_like(logp) if grad_logp is None else grad_logp
    if seq_logp is None and want_seq_logp:
        seq_logp = torch.empty(tokens.n_seq, dtype=torch.float32, device=dev)
    stats = torch.zeros(DPO_STATS_BYTES, dtype=torch.uint8, device=dev) if stats is None else stats
    ws, nb = _workspace(workspace_bytes(RFT_OP_DPO_FWD, tokens, 0, V), dev, ws)
    tk = tokens.c()
    _check(lib().rft_dpo_loss_fwd(ctypes.byref(tk), V, _ptr(logp), _ptr(ref_logp), beta,
                                  label_smoothing, _ptr(grad_logp), _ptr(seq_logp), _ptr(stats),
                                  _ptr(ws), nb, _stream(stream)))
    return grad_logp, seq_logp, stats


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _call(fn, device, stream, *args):
    """Runs an entry point with `device` current, on `stream` or the device's current stream;
    the calls of a decode step take about as long on the host as on the GPU, so the device is
    set only where it is another one."""
    i = device.index
    if stream is None:
        s = _raw_stream(i)
    else:
        if stream.device != device:
            raise RuntimeError(f"stream is of {stream.device}, the call works on {device}")
        s = stream.cuda_stream
    if torch.cuda.current_device() == i:
        st = fn(*args, s)
    else:
        with torch.cuda.device(i):
            st = fn(*args, s)
    if st != RFT_OK:
        _check(st)


def _at(t):
    return None if t is None else t.data_ptr()


def _want(dev, t, dtype, shape, name):
    """A given array of a call: the dtype and shape that the entry point assumes, contiguous."""
    if t is None:
        raise TypeError(f"{name} is missing")
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous():
        raise TypeError(f"{name}: contiguous {dtype} {tuple(shape)} expected, "
                        f"got {t.dtype} {tuple(t.shape)}")
    if t.device != dev:
        raise RuntimeError(f"{name} is on {t.device}, the call works on {dev}")


def _same_device(dev, *named):
    for name, t in named:
        if t is not None and t.device != dev:
            raise RuntimeError(f"{name} is on {t.device}, the call works on {dev}")


# ------------------------------------------------------------------ router --
def router_params(n_experts, top_k, norm_topk=True, scope=RFT_BALANCE_BATCH, balance_coef=0.0,
                  z_coef=0.0) -> rft_router_params:
    return rft_router_params(n_experts, top_k, 1 if norm_topk else 0, scope, balance_coef, z_coef)


@dataclass
class RouterOut:
    """Outputs of rft_router_fwd; lse, counts, dprob and stats are None without the loss."""
    expert_ids: torch.Tensor      # int32 [T, k]
    gates: torch.Tensor           # f32 [T, k]
    lse: torch.Tensor = None      # f32 [T]
    counts: torch.Tensor = None   # int32 [G, E]
    dprob: torch.Tensor = None    # f32 [G, E]
    stats: torch.Tensor = None    # rft_router_stats (held as f32 [6]), see stats_to_dict

    @property
    def losses(self):
        """[loss, balance_loss, z_loss] as a view of the statistics (device, f32)."""
        return self.stats[:3]


_ROUTER_STATS_WORDS = ctypes.sizeof(rft_router_stats) // 4


def _router_rows(T, x, E, name):
    shape, stride = x.shape, x.stride()
    if len(shape) != 2 or shape[0] != T or shape[1] != E or (T and E > 1 and stride[1] != 1):
        raise TypeError(f"{name}: [{T}, {E}] with unit column stride expected, got "
                        f"{tuple(shape)} strides {stride}")
    # the stride of a single row may be anything
    return stride[0] if T > 1 else E


@_allocates
def rft_router_fwd(tokens: Tokens, logits, params, want_loss=True, out=None, ws=None, stream=None):
    """Returns a RouterOut; `out` (one of an earlier call with the same sizes) is written anew."""
    tk = tokens.c()
    dev, T, k, E = logits.device, tk.T, params.top_k, params.n_experts
    _need_gpu(logits)
    if not tokens.mask.device == dev == tokens.seq_start.device:
        _same_device(dev, ("mask", tokens.mask), ("seq_start", tokens.seq_start))
    if ws is not None:
        _same_device(dev, ("ws", ws))
    dt, ld = _dtype_code(logits), _router_rows(T, logits, E, "logits")
    G = tk.n_seq if params.scope == RFT_BALANCE_ROLLOUT else 1
    i32, f32 = torch.int32, torch.float32
    if out is None:
        new = torch.empty
        out = RouterOut(new((T, k), dtype=i32, device=dev), new((T, k), dtype=f32, device=dev))
        if want_loss:
            out.lse = new(T, dtype=f32, device=dev)
            out.counts = new((G, E), dtype=i32, device=dev)
            out.dprob = new((G, E), dtype=f32, device=dev)
            out.stats = new(_ROUTER_STATS_WORDS, dtype=f32, device=dev)
    else:
        _want(dev, out.expert_ids, i32, (T, k), "expert_ids")
        _want(dev, out.gates, f32, (T, k), "gates")
        if want_loss:
            _want(dev, out.lse, f32, (T,), "lse")
            _want(dev, out.counts, i32, (G, E), "counts")
            _want(dev, out.dprob, f32, (G, E), "dprob")
            _want(dev, out.stats, f32, (_ROUTER_STATS_WORDS,), "stats")
    L, rt, rp = lib(), ctypes.byref(tk), ctypes.byref(params)
    if not want_loss:
        _call(L.rft_router_fwd, dev, stream, rt, _at(logits), dt, ld, rp, _at(out.expert_ids),
              _at(out.gates), None, None, None, None, None, 0)
        if stream is not None:
            _used_on(stream, out.expert_ids, out.gates)
        return out
    ws, nb = _workspace(int(L.rft_router_workspace_bytes(rt, rp)), dev, ws)
    _call(L.rft_router_fwd, dev, stream, rt, _at(logits), dt, ld, rp, _at(out.expert_ids),
          _at(out.gates), _at(out.lse), _at(out.counts), _at(out.dprob), _at(out.stats), _at(ws), nb)
    if stream is not None:
        _used_on(stream, out.expert_ids, out.gates, out.lse, out.counts, out.dprob, out.stats, ws)
    return out


@_allocates
def rft_router_bwd(tokens: Tokens, logits, params, fwd: RouterOut, d_gates=None, d_logits=None,
                   stream=None):
    """Returns d_logits; `fwd` is what rft_router_fwd returned for the same inputs."""
    tk = tokens.c()
    dev, T, k, E = logits.device, tk.T, params.top_k, params.n_experts
    _need_gpu(logits)
    if not tokens.mask.device == dev == tokens.seq_start.device:
        _same_device(dev, ("mask", tokens.mask), ("seq_start", tokens.seq_start))
    dt, ld = _dtype_code(logits), _router_rows(T, logits, E, "logits")
    f32 = torch.float32
    if d_gates is not None:
        _want(dev, d_gates, f32, (T, k), "d_gates")
    if fwd.stats is None:
        raise TypeError("rft_router_bwd needs a forward with want_loss=True")
    _want(dev, fwd.expert_ids, torch.int32, (T, k), "expert_ids")
    _want(dev, fwd.lse, f32, (T,), "lse")
    _want(dev, fwd.dprob, f32, (tk.n_seq if params.scope == RFT_BALANCE_ROLLOUT else 1, E), "dprob")
    _want(dev, fwd.stats, f32, (_ROUTER_STATS_WORDS,), "stats")
    if d_logits is None:
        d_logits, ldd = torch.empty((T, E), dtype=logits.dtype, device=dev), E
    else:
        if d_logits.dtype != logits.dtype:
            raise TypeError("d_logits has the dtype of logits")
        ldd = _router_rows(T, d_logits, E, "d_logits")
        _same_device(dev, ("d_logits", d_logits))
    _call(lib().rft_router_bwd, dev, stream, ctypes.byref(tk), _at(logits), dt, ld,
          ctypes.byref(params), _at(fwd.expert_ids), _at(fwd.lse), _at(d_gates), _at(fwd.dprob),
          _at(fwd.stats), _at(d_logits), ldd)
    if stream is not None:
        _used_on(stream, d_logits)
    return d_logits


# ----------------------------------------------------------------- updates --
_data_ptr = torch.Tensor.data_ptr
_PARAM = struct.Struct("5Qq")  # an rft_param
_STATE_DTYPES = (torch.float32,) * 3  # of m, v and master


class Params:
    """Tensors of an update as (weight, grad, m, v[, master]) tuples, all contiguous and of one
    size each; a training program makes it once and keeps it.  For rft_grad_norm alone weight,
    m and v may be None.  A call uses the tensors where they lie when it is made (their storage
    may have been replaced); where the gradient given was the weight's .grad, it takes the .grad
    of that moment, which a backward pass may have made anew, and raises if there is none.
    Other gradients are the tensors given: a program that makes them anew makes Params anew."""

    def __init__(self, tensors):
        self.tensors = [tuple(t) + (None,) * (5 - len(t)) for t in tensors]
        self.device = None
        self.weight_dtype = self.grad_dtype = None
        self.c = (rft_param * max(1, len(self.tensors)))()
        self._follows = []  # tensors whose gradient is the weight's .grad
        for i, ts in enumerate(self.tensors):
            w, g = ts[:2]
            if self.device is None:
                _need_gpu(g)
                self.device, self.grad_dtype = g.device, g.dtype
                self._index = g.get_device()
            if w is not None:
                if self.weight_dtype is None:
                    self.weight_dtype = w.dtype
                if w.requires_grad and w.is_leaf and w.grad is g:
                    self._follows.append(i)
        self._bind()

    def _bind(self):
        held, ptrs = [], []
        kinds = (self.weight_dtype, self.grad_dtype, *_STATE_DTYPES)
        for i, ts in enumerate(self.tensors):
            n, at = ts[1].numel(), []
            for t, dt in zip(ts, kinds):
                if t is None:
                    at.append(0)
                elif (t.dtype is dt and t.numel() == n and t.get_device() == self._index
                      and t.is_contiguous()):
                    p = t.data_ptr()
                    at.append(p)
                    held.append(t)
                    ptrs.append(p)
                else:
                    raise TypeError(f"tensor {i}: contiguous {dt} of {n} elements on "
                                    f"{self.device} expected, got {t.dtype} {tuple(t.shape)} "
                                    f"on {t.device}")
            _PARAM.pack_into(self.c, i * _PARAM.size, *at, n)
        self._held, self._ptrs = held, ptrs

    def now(self):
        """The C list of the tensors as they are now."""
        moved = False
        for i in self._follows:
            w, g, *rest = self.tensors[i]
            if w.grad is not g:
                if w.grad is None:
                    raise RuntimeError(f"tensor {i}: the weight has no gradient")
                self.tensors[i] = (w, w.grad, *rest)
                moved = True
        if moved or list(map(_data_ptr, self._held)) != self._ptrs:
            self._bind()
        return self.c

    def __len__(self):
        return len(self.tensors)


class Clip:
    """Gradient norm and clip factor on the device (rft_clip, held as f32 [3])."""

    def __init__(self, device):
        self.buf = torch.empty(ctypes.sizeof(rft_clip) // 4, dtype=torch.float32, device=device)

    @property
    def norm(self):
        return self.buf[0]

    @property
    def scale(self):
        return self.buf[1]

    @property
    def finite(self):
        return self.buf.view(torch.int32)[2]


def _code(dtype):
    if dtype == torch.bfloat16:
        return RFT_BF16
    if dtype == torch.float32 or dtype is None:
        return RFT_F32
    raise TypeError(f"unsupported dtype {dtype}")


def _clip_at(dev, clip):
    if clip is None:
        return None
    if clip.buf.device != dev:
        raise RuntimeError(f"clip is on {clip.buf.device}, the call works on {dev}")
    return clip.buf.data_ptr()


@_allocates
def rft_grad_norm(params: Params, max_norm=0.0, clip=None, ws=None, stream=None) -> Clip:
    """Global gradient norm; the returned Clip feeds rft_adamw_step and rft_muon_step."""
    dev = params.device or torch.device("cuda", torch.cuda.current_device())
    clip = Clip(dev) if clip is None else clip
    if ws is not None:
        _same_device(dev, ("ws", ws))
    L, n, tensors = lib(), len(params), params.now()
    ws, nb = _workspace(int(L.rft_grad_norm_workspace_bytes(tensors, n)), dev, ws)
    _call(L.rft_grad_norm, dev, stream, tensors, n, _code(params.grad_dtype), max_norm,
          _clip_at(dev, clip), _at(ws), nb)
    if stream is not None:
        _used_on(stream, clip.buf, ws)
    return clip


def adamw_params(lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01,
                 step=1) -> rft_adamw_params:
    return rft_adamw_params(lr, beta1, beta2, eps, weight_decay, step)


def rft_adamw_step(params: Params, hyper, clip=None, stream=None):
    """One AdamW step in place over every tensor of `params`."""
    dev = params.device or torch.device("cuda", torch.cuda.current_device())
    _call(lib().rft_adamw_step, dev, stream, params.now(), len(params), _code(params.weight_dtype),
          _code(params.grad_dtype), ctypes.byref(hyper), _clip_at(dev, clip))


def muon_params(lr=0.02, momentum=0.95, nesterov=True, weight_decay=0.0, scale=1.0, steps=5,
                coefs=(3.4445, -4.7750, 2.0315), eps=1e-7,
                products=RFT_PRODUCTS_BY_TYPE) -> rft_muon_params:
    return rft_muon_params(lr, momentum, weight_decay, scale, *coefs, eps, steps,
                           1 if nesterov else 0, products)


def _matrices(first, *others):
    """The layout [rows, cols] or [batch, rows, cols] that every array of a call shares."""
    name, t = first
    if t.dim() not in (2, 3) or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise TypeError(f"{name}: [rows, cols] or [batch, rows, cols] with unit column stride")
    b = t.shape[0] if t.dim() == 3 else 1
    r, c = t.shape[-2:]
    # the strides that move: of several rows, and of several matrices
    key = lambda x: ((x.stride(-2) if r > 1 else c),  # noqa: E731
                     (x.stride(0) if x.dim() == 3 and b > 1 else 0))
    for n, x in others:
        if x is None:
            continue
        if x.shape != t.shape or (c > 1 and x.stride(-1) != 1) or key(x) != key(t):
            raise TypeError(f"{n}: the shape and strides of {name} expected")
        if x.device != t.device:
            raise RuntimeError(f"{n} is on {x.device}, {name} on {t.device}")
    return rft_matrices(b, r, c, *key(t))


@_allocates
def rft_orthogonalize(g, params, out=None, out_dtype=None, ws=None, stream=None):
    """Orthogonalises [rows, cols] or each of [batch, rows, cols]; out has g's strides."""
    _need_gpu(g, out)
    if out is None:
        out = torch.empty_strided(g.shape, g.stride(), dtype=out_dtype or g.dtype, device=g.device)
    elif out_dtype is not None and out.dtype != out_dtype:
        raise TypeError("out has another dtype than out_dtype")
    mats = _matrices(("g", g), ("out", out))
    _same_device(g.device, ("ws", ws))
    dt, odt = _dtype_code(g), _dtype_code(out)
    L, rm, rp = lib(), ctypes.byref(mats), ctypes.byref(params)
    ws, nb = _workspace(int(L.rft_orthogonalize_workspace_bytes(rm, rp, odt)), g.device, ws)
    _call(L.rft_orthogonalize, g.device, stream, rm, _at(g), dt, rp, _at(out), odt, _at(ws), nb)
    if stream is not None:
        _used_on(stream, out, ws)
    return out


@_allocates
def rft_muon_step(weight, grad, momentum, params, master=None, clip=None, ws=None, stream=None):
    """One orthogonalised momentum step in place; every array has the weight's strides."""
    _need_gpu(weight, grad, momentum, master)
    mats = _matrices(("weight", weight), ("grad", grad), ("momentum", momentum), ("master", master))
    for name, t in (("momentum", momentum), ("master", master)):
        if t is not None and t.dtype != torch.float32:
            raise TypeError(f"{name} is float32")
    dev = weight.device
    _same_device(dev, ("ws", ws))
    wdt, gdt = _dtype_code(weight), _dtype_code(grad)
    L, rm, rp = lib(), ctypes.byref(mats), ctypes.byref(params)
    need = int(L.rft_orthogonalize_workspace_bytes(rm, rp, RFT_F32 if master is not None else wdt))
    ws, nb = _workspace(need, dev, ws)
    _call(L.rft_muon_step, dev, stream, rm, _at(grad), gdt, _at(momentum), _at(weight), wdt,
          _at(master), rp, _clip_at(dev, clip), _at(ws), nb)
    if stream is not None:
        _used_on(stream, ws)


def loaded_library_path() -> str:
    return LIB_PATH if _LIB is not None else ""
