"""ctypes binding of libbanditspec.so: the same entry points as include/banditspec.h.

Argument marshalling only: tensors are passed as raw device pointers, every step of the
round runs in the library's CUDA kernels on torch's current stream.  PyTorch is used for
device memory and streams.  Importing this module loads the CUDA library and raises if it is
missing -- there is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbanditspec.so")
if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python __graft_entry__.py` "
                      "(the CUDA library is required; there is no fallback path)")
_lib = C.CDLL(LIB_PATH)

BS_OK = 0
BS_ERR_INVALID_ARG, BS_ERR_CUDA, BS_ERR_UNSUPPORTED, BS_ERR_WORKSPACE, BS_ERR_TIMEOUT, BS_ERR_DEVICE_DATA = 1, 2, 3, 4, 5, 6
BS_F32, BS_BF16 = 0, 1
BS_UCB, BS_EXP3, BS_UCB_REWARD = 0, 1, 2
BS_DEV_BAD_GAMMA, BS_DEV_BAD_TOKEN, BS_DEV_NONFINITE, BS_DEV_RESIDUAL_FALLBACK, BS_DEV_DRAFT_MISSING = 1, 2, 4, 8, 16
BS_DEV_BAD_TREE = 32
BS_DEV_BAD_LENGTH, BS_DEV_NO_BLOCKS, BS_DEV_NO_ROOM, BS_DEV_BAD_BLOCK, BS_DEV_TIMEOUT = 64, 128, 256, 512, 1024
BS_DEV_BAD_MASK = 2048
BS_ROTARY_PLAIN, BS_ROTARY_LINEAR, BS_ROTARY_BANDS, BS_ROTARY_YARN = 0, 1, 2, 3
BS_MAX_GAMMA, BS_MAX_ARMS, BS_MAX_BATCH, BS_MAX_SEQ_BLOCKS = 31, 32, 4096, 1 << 18

_vp, _i, _f, _d, _sz, _ll = C.c_void_p, C.c_int, C.c_float, C.c_double, C.c_size_t, C.c_longlong

# name -> (restype, argtypes); must list every symbol the header declares
SIGNATURES = {
    "bs_status_string": (C.c_char_p, [_i]),
    "bs_last_cuda_error": (C.c_char_p, []),
    "bs_workspace_bytes": (_sz, [_i, _i, _i]),
    "bs_workspace_init": (_i, [_vp, _sz, _vp]),
    "bs_get_device_status": (_i, [_vp, _sz, _i, _i, _i, _vp, _vp]),
    "bs_softmax_verify": (_i, [_vp, _vp, _i, _vp, _vp, _vp, _f, _i, _i, _i, _vp, _vp, _vp, _vp, _sz, _vp]),
    "bs_residual_sample": (_i, [_vp, _vp, _i, _vp, _vp, _vp, _vp, _f, _i, _i, _i, _vp, _vp, _vp, _sz, _vp]),
    "bs_softmax_verify_noalloc": (_i, [_vp, _vp, _i, _vp, _vp, _vp, _f, _i, _i, _i, _vp, _vp, _vp, _vp]),
    "bs_verify_walk": (_i, [_vp, _vp, _i, _vp, _vp, _vp, _vp, _f, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "bs_verify_walk_drafted": (_i, [_vp, _vp, _i, _vp, _vp, _vp, _vp, _f, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp, _sz,
                                    _vp]),
    "bs_draft_sample": (_i, [_vp, _i, _i, _vp, _vp, _f, _i, _i, _i, _vp, _vp, _sz, _vp]),
    "bs_softmax_verify_drafted": (_i, [_vp, _vp, _i, _vp, _vp, _vp, _f, _i, _i, _i, _vp, _vp, _vp, _vp, _sz, _vp]),
    "bs_tree_verify_greedy": (_i, [_vp, _i, _vp, _vp, _vp, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "bs_tree_expand_shapes": (_i, [_vp, _vp, _vp, _i, _i, _i, _vp, _vp, _vp]),
    "bs_lmhead_workspace_bytes": (_sz, [_i, _i, _i]),
    "bs_lmhead_verify": (_i, [_vp, _vp, _i, _vp, _vp, _i, _vp, _vp, _vp, _f, _i, _i, _i, _vp, _vp, _vp, _vp, _vp,
                              _vp, _sz, _vp]),
    "bs_cache_plan": (_i, [_vp, _vp, _vp, _i, _vp, _i, _i, _vp, _i, _vp, _vp, _i, _vp, _vp, _vp, _vp, _vp, _i, _vp, _vp]),
    "bs_cache_plan_next": (_i, [_vp, _vp, _vp, _vp, _vp, _i, _vp, _i, _i, _vp, _i, _vp, _vp, _i, _vp, _vp, _vp, _vp, _vp, _i, _vp, _vp]),
    "bs_cache_append": (_i, [_vp, _vp, _i, _ll, _ll, _ll, _ll, _vp, _i, _i, _i, _vp, _vp, _vp, _vp, _i, _i, _vp]),
    "bs_cache_workspace_bytes": (_sz, [_i, _i, _i]),
    "bs_cache_get_device_status": (_i, [_vp, _sz, _vp]),
    "bs_cache_attention": (_i, [_vp, _ll, _ll, _vp, _vp, _vp, _i, _vp, _i, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i,
                                _i, _f, _vp, _ll, _ll, _vp, _vp, _sz, _vp]),
    "bs_cache_keep_path": (_i, [_vp, _vp, _vp, _i, _i, _vp, _i, _i, _i, _vp, _vp, _vp, _vp, _i, _i, _vp, _vp]),
    "bs_rotary_frequencies": (_i, [_i, _i, _d, _d, _d, _d, _d, _vp, _vp]),
    "bs_rotary": (_i, [_vp, _ll, _ll, _vp, _ll, _ll, _i, _vp, _vp, _f, _i, _i, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp, _ll, _ll, _vp, _ll,
                       _ll, _vp]),
    "bs_prompt_attention": (_i, [_vp, _ll, _ll, _vp, _ll, _ll, _vp, _ll, _ll, _vp, _i, _i, _i, _i, _i, _f, _vp, _ll, _ll, _vp, _vp]),
    "bs_prompt_get_device_status": (_i, [_vp]),
    "bs_history_update": (_i, [_vp, _i, _i, _vp, _vp, _vp, _i, _vp, _vp, _i, _vp, _vp]),
    "bs_logits_adjust": (_i, [_vp, _vp, _i, _vp, _i, _i, _i, _vp, _vp, _i, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i, _vp, _i, _vp, _i, _i, _i,
                              _vp, _vp]),
    "bs_bandit_state_bytes": (_sz, [_i, _i, _i]),
    "bs_bandit_init": (_i, [_vp, _sz, _i, _i, _i, _vp, _d, _vp]),
    "bs_bandit_select": (_i, [_vp, _sz, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp]),
    "bs_bandit_update": (_i, [_vp, _sz, _i, _i, _i, _vp, _vp, _vp, _vp]),
    "bs_bandit_read": (_i, [_vp, _sz, _i, _i, _i, _vp, _vp, _vp, _vp, _vp]),
    "bs_bandit_step": (_i, [_vp, _sz, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "bs_bandit_init_reward": (_i, [_vp, _sz, _i, _i, _vp, _d, _d, _vp]),
    "bs_bandit_update_reward": (_i, [_vp, _sz, _i, _i, _vp, _vp, _vp, _vp]),
    "bs_throughput_reward": (_i, [_vp, _vp, _i, _d, _i, _vp, _vp]),
}
for _name, (_res, _args) in SIGNATURES.items():
    _fn = getattr(_lib, _name)
    _fn.restype, _fn.argtypes = _res, _args


class BanditSpecError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        detail = f" [{_lib.bs_last_cuda_error().decode()}]" if code == BS_ERR_CUDA else ""
        super().__init__(f"{where}: {_lib.bs_status_string(code).decode()} (bs_status {code}){detail}")


def _check(code: int, where: str) -> None:
    if code != BS_OK:
        raise BanditSpecError(code, where)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    assert t.is_contiguous(), "tensors must be contiguous"
    return t.data_ptr()


def _stream(stream=None) -> int:
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return BS_F32
    if t.dtype == torch.bfloat16:
        return BS_BF16
    raise TypeError(f"logits must be float32 or bfloat16, got {t.dtype}")


# ---- workspace ---------------------------------------------------------------------

def bs_workspace_bytes(B: int, Gmax: int, V: int) -> int:
    return int(_lib.bs_workspace_bytes(B, Gmax, V))


def bs_workspace_init(workspace: torch.Tensor, stream=None) -> None:
    _check(_lib.bs_workspace_init(_ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           "bs_workspace_init")


def new_workspace(B: int, Gmax: int, V: int, device="cuda") -> torch.Tensor:
    """Allocate (through torch) and clear a workspace for the given limits."""
    n = bs_workspace_bytes(B, Gmax, V)
    if n == 0:
        raise BanditSpecError(BS_ERR_UNSUPPORTED, "bs_workspace_bytes")
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    bs_workspace_init(ws)
    return ws


def bs_get_device_status(workspace: torch.Tensor, B: int, Gmax: int, V: int, stream=None) -> np.ndarray:
    """Per-sequence status bits of the last verify/residual pair (synchronises)."""
    host = np.zeros(B, dtype=np.int32)
    code = _lib.bs_get_device_status(_ptr(workspace), workspace.numel(), B, Gmax, V,
                                     host.ctypes.data_as(_vp), _stream(stream))
    if code not in (BS_OK, BS_ERR_DEVICE_DATA):
        raise BanditSpecError(code, "bs_get_device_status")
    return host


# ---- verification ---------------------------------------------------------------------

def bs_softmax_verify(target_logits, draft_logits, draft_tokens, gamma, u_accept, temperature: float,
                      accept_len, p_tok, q_tok, workspace, stream=None) -> None:
    B, G1, V = target_logits.shape
    _check(_lib.bs_softmax_verify(_ptr(target_logits), _ptr(draft_logits), _dtype_code(target_logits),
                                  _ptr(draft_tokens), _ptr(gamma), _ptr(u_accept), float(temperature),
                                  B, G1 - 1, V, _ptr(accept_len), _ptr(p_tok), _ptr(q_tok),
                                  _ptr(workspace), workspace.numel(), _stream(stream)), "bs_softmax_verify")


def bs_residual_sample(target_logits, draft_logits, draft_tokens, gamma, accept_len, u_resample,
                       temperature: float, out_tokens, out_len, workspace, stream=None) -> None:
    B, G1, V = target_logits.shape
    _check(_lib.bs_residual_sample(_ptr(target_logits), _ptr(draft_logits), _dtype_code(target_logits),
                                   _ptr(draft_tokens), _ptr(gamma), _ptr(accept_len), _ptr(u_resample),
                                   float(temperature), B, G1 - 1, V, _ptr(out_tokens), _ptr(out_len),
                                   _ptr(workspace), workspace.numel(), _stream(stream)), "bs_residual_sample")


BS_NOALLOC_SCRATCH_BYTES = 2 << 20


def bs_softmax_verify_noalloc(target_logits, draft_logits, draft_tokens, gamma, u_accept, temperature: float,
                              accept_len, p_tok, q_tok, stream=None) -> None:
    """bs_softmax_verify on the scratch array built into the library: for callers that cannot
    allocate device memory (fixed memory pools, buffer-only plugins, no-cudaMalloc paths).
    Sizes whose workspace exceeds BS_NOALLOC_SCRATCH_BYTES raise BS_ERR_WORKSPACE; calls that
    overlap on one GPU race on the shared array."""
    B, G1, V = target_logits.shape
    _check(_lib.bs_softmax_verify_noalloc(_ptr(target_logits), _ptr(draft_logits), _dtype_code(target_logits),
                                          _ptr(draft_tokens), _ptr(gamma), _ptr(u_accept), float(temperature),
                                          B, G1 - 1, V, _ptr(accept_len), _ptr(p_tok), _ptr(q_tok),
                                          _stream(stream)), "bs_softmax_verify_noalloc")


@dataclass
class RoundOutput:
    accept_len: torch.Tensor   # [B] int32, tau
    p_tok: torch.Tensor        # [B, Gmax] fp32
    q_tok: torch.Tensor        # [B, Gmax] fp32
    out_tokens: torch.Tensor   # [B, Gmax+1] int32
    out_len: torch.Tensor      # [B] int32, y = tau + 1
    workspace: torch.Tensor


def verify_round(target_logits, draft_logits, draft_tokens, gamma, u_accept, u_resample,
                 temperature: float, workspace: Optional[torch.Tensor] = None) -> RoundOutput:
    """Allocates the outputs and calls bs_softmax_verify then bs_residual_sample."""
    B, G1, V = target_logits.shape
    G = G1 - 1
    dev = target_logits.device
    if workspace is None:
        workspace = new_workspace(B, G, V, dev)
    accept_len = torch.empty(B, dtype=torch.int32, device=dev)
    p_tok = torch.empty(B, G, dtype=torch.float32, device=dev)
    q_tok = torch.empty(B, G, dtype=torch.float32, device=dev)
    out_tokens = torch.empty(B, G + 1, dtype=torch.int32, device=dev)
    out_len = torch.empty(B, dtype=torch.int32, device=dev)
    bs_softmax_verify(target_logits, draft_logits, draft_tokens, gamma, u_accept, temperature,
                      accept_len, p_tok, q_tok, workspace)
    bs_residual_sample(target_logits, draft_logits, draft_tokens, gamma, accept_len, u_resample,
                       temperature, out_tokens, out_len, workspace)
    return RoundOutput(accept_len, p_tok, q_tok, out_tokens, out_len, workspace)


def bs_verify_walk(target_logits, draft_logits, draft_tokens, gamma, u_accept, u_resample, temperature: float,
                   accept_len, p_tok, q_tok, out_tokens, out_len, workspace, stream=None) -> None:
    """Verification with early exit and resampling in one launch."""
    B, G1, V = target_logits.shape
    _check(_lib.bs_verify_walk(_ptr(target_logits), _ptr(draft_logits), _dtype_code(target_logits),
                               _ptr(draft_tokens), _ptr(gamma), _ptr(u_accept), _ptr(u_resample), float(temperature),
                               B, G1 - 1, V, _ptr(accept_len), _ptr(p_tok), _ptr(q_tok), _ptr(out_tokens),
                               _ptr(out_len), _ptr(workspace), workspace.numel(), _stream(stream)), "bs_verify_walk")


def bs_verify_walk_drafted(target_logits, draft_logits, draft_tokens, gamma, u_accept, u_resample, temperature: float,
                           accept_len, p_tok, q_tok, out_tokens, out_len, workspace, stream=None) -> None:
    """bs_verify_walk on the statistics bs_draft_sample left in the workspace: target rows only."""
    B, G1, V = target_logits.shape
    _check(_lib.bs_verify_walk_drafted(_ptr(target_logits), _ptr(draft_logits), _dtype_code(target_logits),
                                       _ptr(draft_tokens), _ptr(gamma), _ptr(u_accept), _ptr(u_resample),
                                       float(temperature), B, G1 - 1, V, _ptr(accept_len), _ptr(p_tok), _ptr(q_tok),
                                       _ptr(out_tokens), _ptr(out_len), _ptr(workspace), workspace.numel(),
                                       _stream(stream)), "bs_verify_walk_drafted")


def verify_round_walk(target_logits, draft_logits, draft_tokens, gamma, u_accept, u_resample,
                      temperature: float, workspace: Optional[torch.Tensor] = None) -> RoundOutput:
    """Allocates the outputs and calls bs_verify_walk."""
    B, G1, V = target_logits.shape
    G = G1 - 1
    dev = target_logits.device
    if workspace is None:
        workspace = new_workspace(B, G, V, dev)
    accept_len = torch.full((B,), -9, dtype=torch.int32, device=dev)
    p_tok = torch.full((B, G), -1.0, dtype=torch.float32, device=dev)
    q_tok = torch.full((B, G), -1.0, dtype=torch.float32, device=dev)
    out_tokens = torch.full((B, G + 1), -9, dtype=torch.int32, device=dev)
    out_len = torch.full((B,), -9, dtype=torch.int32, device=dev)
    bs_verify_walk(target_logits, draft_logits, draft_tokens, gamma, u_accept, u_resample, temperature,
                   accept_len, p_tok, q_tok, out_tokens, out_len, workspace)
    return RoundOutput(accept_len, p_tok, q_tok, out_tokens, out_len, workspace)


# ---- drafting on the device ------------------------------------------------------------

def bs_draft_sample(draft_logits, position: int, gamma, u_draft, temperature: float, draft_tokens, workspace,
                    stream=None) -> None:
    """Drafted token of `position` for every sequence with position < gamma_b, into draft_tokens[b, position]."""
    B, G, V = draft_logits.shape
    assert draft_tokens.shape == (B, G) and draft_tokens.dtype == torch.int32
    _check(_lib.bs_draft_sample(_ptr(draft_logits), _dtype_code(draft_logits), int(position), _ptr(gamma),
                                _ptr(u_draft), float(temperature), B, G, V, _ptr(draft_tokens),
                                _ptr(workspace), workspace.numel(), _stream(stream)), "bs_draft_sample")


def bs_softmax_verify_drafted(target_logits, draft_logits, draft_tokens, gamma, u_accept, temperature: float,
                              accept_len, p_tok, q_tok, workspace, stream=None) -> None:
    B, G1, V = target_logits.shape
    _check(_lib.bs_softmax_verify_drafted(_ptr(target_logits), _ptr(draft_logits), _dtype_code(target_logits),
                                          _ptr(draft_tokens), _ptr(gamma), _ptr(u_accept), float(temperature),
                                          B, G1 - 1, V, _ptr(accept_len), _ptr(p_tok), _ptr(q_tok),
                                          _ptr(workspace), workspace.numel(), _stream(stream)),
           "bs_softmax_verify_drafted")


# ---- greedy verification of a tree of drafts ---------------------------------------------------

def bs_tree_verify_greedy(target_logits, node_parent, node_tokens, n_nodes, accept_len, out_nodes, out_tokens,
                          out_len, workspace, stream=None) -> None:
    """target_logits [B, Nmax+1, V]: row n = the target's logits after the path to node n (row 0: the prompt)."""
    B, N1, V = target_logits.shape
    _check(_lib.bs_tree_verify_greedy(_ptr(target_logits), _dtype_code(target_logits), _ptr(node_parent),
                                      _ptr(node_tokens), _ptr(n_nodes), B, N1 - 1, V, _ptr(accept_len),
                                      _ptr(out_nodes), _ptr(out_tokens), _ptr(out_len), _ptr(workspace),
                                      workspace.numel(), _stream(stream)), "bs_tree_verify_greedy")


def bs_tree_expand_shapes(shape_parent, shape_nodes, arm, node_parent, n_nodes, stream=None) -> None:
    K, Nmax = shape_parent.shape
    B = arm.shape[0]
    _check(_lib.bs_tree_expand_shapes(_ptr(shape_parent), _ptr(shape_nodes), _ptr(arm), K, B, Nmax,
                                      _ptr(node_parent), _ptr(n_nodes), _stream(stream)), "bs_tree_expand_shapes")


# ---- fused LM head ----------------------------------------------------------------------

def bs_lmhead_workspace_bytes(B: int, Gmax: int, V: int) -> int:
    return int(_lib.bs_lmhead_workspace_bytes(B, Gmax, V))


def new_lmhead_workspace(B: int, Gmax: int, V: int, device="cuda") -> torch.Tensor:
    n = bs_lmhead_workspace_bytes(B, Gmax, V)
    if n == 0:
        raise BanditSpecError(BS_ERR_UNSUPPORTED, "bs_lmhead_workspace_bytes")
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    bs_workspace_init(ws)
    return ws


def bs_lmhead_verify(H_t, W_t, H_d, W_d, draft_tokens, gamma, u_accept, temperature: float, B: int, Gmax: int,
                     logits_t_out, logits_d_out, accept_len, p_tok, q_tok, workspace, stream=None) -> None:
    """H_t [B*(Gmax+1), d_t], W_t [d_t, V], H_d [B*Gmax, d_d], W_d [d_d, V] bf16; logits out fp32."""
    d_t, V = W_t.shape
    assert H_t.shape == (B * (Gmax + 1), d_t) and H_t.dtype == torch.bfloat16 and W_t.dtype == torch.bfloat16
    d_d = 0
    if W_d is not None:
        d_d = W_d.shape[0]
        assert W_d.shape[1] == V and H_d.shape == (B * Gmax, d_d)
        assert H_d.dtype == torch.bfloat16 and W_d.dtype == torch.bfloat16
    assert logits_t_out.dtype == torch.float32 and logits_t_out.numel() == B * (Gmax + 1) * V
    _check(_lib.bs_lmhead_verify(_ptr(H_t), _ptr(W_t), d_t, _ptr(H_d), _ptr(W_d), d_d, _ptr(draft_tokens),
                                 _ptr(gamma), _ptr(u_accept), float(temperature), B, Gmax, V,
                                 _ptr(logits_t_out), _ptr(logits_d_out), _ptr(accept_len), _ptr(p_tok), _ptr(q_tok),
                                 _ptr(workspace), workspace.numel(), _stream(stream)), "bs_lmhead_verify")


# ---- the key / value cache of a round ----------------------------------------------------------

# These calls are made once or more per layer: their checks are kept to a few attribute look-ups each.

# The current stream's handle without building a Stream object, and the current GPU without torch's check that CUDA is up (tensors
# are there already); where torch lacks these names (a build without CUDA), the long way.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_gpu = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_CODES, _f32, _bf16, _int32 = (torch.float8_e4m3fn, torch.uint8), torch.float32, torch.bfloat16, torch.int32
_ELSEWHERE = "every tensor of a call has to be on the same GPU"


def _i32(t, n: int, index: Optional[int] = None) -> Optional[int]:
    """Pointer of a contiguous int32 tensor of n elements, on GPU `index` if that is given (None stays NULL)."""
    if t is None:
        return None
    assert t.dtype is _int32 and t.numel() == n and t.is_contiguous(), f"contiguous int32 of {n} elements expected, got {t.dtype} {tuple(t.shape)}"
    assert index is None or t.get_device() == index, _ELSEWHERE
    return t.data_ptr()


def _gpu(t) -> int:
    """Index of the tensor's GPU.  All others of the call have to be there, too: a pointer into other memory would fault."""
    index = t.get_device()
    assert index >= 0, "the tensors have to be on a GPU"
    return index


def _call(fn, where: str, index: int, stream, *args) -> None:
    """fn(*args, stream) with GPU `index` current, on `stream` or that GPU's current stream."""
    if index == _current_gpu():
        code = fn(*args, _raw_stream(index) if stream is None else stream.cuda_stream)
    else:
        with torch.cuda.device(index):
            code = fn(*args, _raw_stream(index) if stream is None else stream.cuda_stream)
    if code != BS_OK:
        raise BanditSpecError(code, where)


def _cache_args(k_cache, k_scale, v_cache, v_scale):
    """The caches' GPU and shape: index, n_blocks, Hkv, block_tokens, d."""
    assert k_cache.dtype in _CODES and v_cache.dtype in _CODES, f"codes must be float8_e4m3fn, or uint8 that holds them, got {k_cache.dtype}, {v_cache.dtype}"
    shape = k_cache.shape
    n, H, bt, d = shape
    blocks = (n, H)
    assert v_cache.shape == shape and k_scale.shape == blocks and v_scale.shape == blocks
    assert k_scale.dtype is _f32 and v_scale.dtype is _f32
    assert k_cache.is_contiguous() and v_cache.is_contiguous() and k_scale.is_contiguous() and v_scale.is_contiguous()
    index = _gpu(k_cache)
    assert k_scale.get_device() == v_cache.get_device() == v_scale.get_device() == index, _ELSEWHERE
    return index, n, H, bt, d


def new_cache(n_blocks: int, Hkv: int, block_tokens: int, d: int, device="cuda"):
    """(codes, scales) of keys or values: float8_e4m3fn [n_blocks, Hkv, block_tokens, d], float32 [n_blocks, Hkv]."""
    return (torch.zeros(n_blocks, Hkv, block_tokens, d, dtype=torch.float8_e4m3fn, device=device),
            torch.ones(n_blocks, Hkv, dtype=torch.float32, device=device))


def bs_cache_plan(seq_len, kept, n_new, extra: int, active, block_tokens: int, block_table, n_held, free_blocks, n_free,
                  kv_len, cu_new, slot_map, positions, status, stream=None, last_cu=None,
                  n_shared=None) -> None:
    """Block tables, slots and positions of a round's new tokens; seq_len, block_table, n_held, free_blocks and n_free
    are updated in place.  last_cu: cu_new of the plan whose tokens `kept` counts (may be cu_new), so that a sequence it
    refused keeps none.  n_shared: leading blocks of each sequence that it shares with others and that are never returned."""
    B, W = block_table.shape
    n_blocks, T = free_blocks.numel(), slot_map.numel()
    index = _gpu(seq_len)
    if active is not None:
        assert active.dtype is torch.uint8 and active.numel() == B and active.is_contiguous()
        assert active.get_device() == index, _ELSEWHERE
    fn, more = _lib.bs_cache_plan, ()
    if last_cu is not None or n_shared is not None:
        fn, more = _lib.bs_cache_plan_next, (_i32(last_cu, B + 1, index), _i32(n_shared, B, index))
    _call(fn, "bs_cache_plan", index, stream, _i32(seq_len, B, index), _i32(kept, B, index), *more, _i32(n_new, B, index), extra,
          None if active is None else active.data_ptr(), B, block_tokens, _i32(block_table, B * W, index), W, _i32(n_held, B, index),
          _i32(free_blocks, n_blocks, index), n_blocks, _i32(n_free, 1, index), _i32(kv_len, B, index), _i32(cu_new, B + 1, index), _i32(slot_map, T, index),
          _i32(positions, T, index), T, _i32(status, B, index))


def bs_cache_append(k, v, slot_map, k_cache, k_scale, v_cache, v_scale, stream=None) -> None:
    """k, v [T, Hkv, d] (bf16 or fp32, last dimension contiguous) into their slots."""
    index, n_blocks, Hkv, bt, d = _cache_args(k_cache, k_scale, v_cache, v_scale)
    T = slot_map.numel()
    assert k.get_device() == v.get_device() == index, _ELSEWHERE
    assert k.shape == v.shape == (T, Hkv, d) and k.dtype is v.dtype
    kt, kh, k1 = k.stride()
    vt, vh, v1 = v.stride()
    assert k1 == 1 and v1 == 1, "the last dimension must be contiguous"
    _call(_lib.bs_cache_append, "bs_cache_append", index, stream, k.data_ptr(), v.data_ptr(), _dtype_code(k), kt, kh, vt, vh,
          _i32(slot_map, T, index), T, Hkv, d, k_cache.data_ptr(), k_scale.data_ptr(), v_cache.data_ptr(), v_scale.data_ptr(), n_blocks, bt)


def new_cache_workspace(Hq: int, Hkv: int, d: int, device="cuda") -> torch.Tensor:
    """Scratch of bs_cache_attention, cleared."""
    with torch.cuda.device(device):
        n = int(_lib.bs_cache_workspace_bytes(Hq, Hkv, d))
        if n == 0:
            raise BanditSpecError(BS_ERR_UNSUPPORTED, "bs_cache_workspace_bytes")
        ws = torch.empty(n, dtype=torch.uint8, device=device)
        bs_workspace_init(ws)
    return ws


def bs_cache_get_device_status(workspace, stream=None) -> None:
    """Raises BanditSpecError (BS_ERR_TIMEOUT) if a bounded wait gave up in an attention on this workspace since it was cleared
    (synchronises)."""
    _call(_lib.bs_cache_get_device_status, "bs_cache_get_device_status", _gpu(workspace), stream,
          workspace.data_ptr(), workspace.numel())


def bs_cache_attention(q, cu_new, kv_len, block_table, node_parent, k_cache, k_scale, v_cache, v_scale, max_new: int,
                       softmax_scale: float, out, status, workspace, stream=None) -> None:
    """q, out [T, Hq, d] bf16 (last dimension contiguous): attention of the new tokens over the cache.  node_parent
    None: chains; [B, Nmax] int32: trees of drafts."""
    index, n_blocks, Hkv, bt, d = _cache_args(k_cache, k_scale, v_cache, v_scale)
    B, W = block_table.shape
    T, Hq, dq = q.shape
    assert q.get_device() == out.get_device() == workspace.get_device() == index, _ELSEWHERE
    assert q.dtype is _bf16 and out.dtype is _bf16 and dq == d and out.shape == q.shape
    qt, qh, q1 = q.stride()
    ot, oh, o1 = out.stride()
    assert q1 == 1 and o1 == 1, "the last dimension must be contiguous"
    Nmax = 0 if node_parent is None else node_parent.shape[1]
    parent = _i32(node_parent, B * Nmax, index)
    if node_parent is not None and Nmax == 0:             # trees of a root alone: nothing to read, but NULL would mean chains
        parent = kv_len.data_ptr()
    _call(_lib.bs_cache_attention, "bs_cache_attention", index, stream, q.data_ptr(), qt, qh, _i32(cu_new, B + 1, index),
          _i32(kv_len, B, index), _i32(block_table, B * W, index), W, parent, Nmax, k_cache.data_ptr(), k_scale.data_ptr(),
          v_cache.data_ptr(), v_scale.data_ptr(), n_blocks, bt, B, T, Hq, Hkv, d, max_new, softmax_scale, out.data_ptr(), ot, oh,
          _i32(status, B, index), workspace.data_ptr(), workspace.numel())


def bs_cache_keep_path(out_nodes, accept_len, seq_len, block_table, k_cache, k_scale, v_cache, v_scale, status,
                       stream=None) -> None:
    """The accepted path of bs_tree_verify_greedy to the front of its tree."""
    index, n_blocks, Hkv, bt, d = _cache_args(k_cache, k_scale, v_cache, v_scale)
    B, W = block_table.shape
    Nmax = out_nodes.shape[1]
    _call(_lib.bs_cache_keep_path, "bs_cache_keep_path", index, stream, _i32(out_nodes, B * Nmax, index), _i32(accept_len, B, index),
          _i32(seq_len, B, index), B, Nmax, _i32(block_table, B * W, index), W, Hkv, d, k_cache.data_ptr(), k_scale.data_ptr(), v_cache.data_ptr(),
          v_scale.data_ptr(), n_blocks, bt, _i32(status, B, index))


def _of(t, dtype, n: int, index: int) -> Optional[int]:
    """Pointer of a contiguous tensor of n elements of that type on GPU `index` (None stays NULL)."""
    if t is None:
        return None
    assert t.dtype is dtype and t.numel() == n and t.is_contiguous(), f"contiguous {dtype} of {n} elements expected, got {t.dtype} {tuple(t.shape)}"
    assert t.get_device() == index, _ELSEWHERE
    return t.data_ptr()


# ---- rotary positions --------------------------------------------------------------------------

@dataclass
class RotaryTable:
    """Frequencies of bs_rotary on one GPU."""
    freq: torch.Tensor         # [rot / 2] int64: turns a position x 2^64
    amplitude: float
    rot: int                   # rotated elements of a head


_SCALINGS = {"none": BS_ROTARY_PLAIN, "linear": BS_ROTARY_LINEAR, "bands": BS_ROTARY_BANDS, "yarn": BS_ROTARY_YARN}


def new_rotary_table(rot: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, low: float = 1.0,
                     high: float = 32.0, original: float = 8192.0, device="cuda") -> RotaryTable:
    """Frequencies base^(-2 i / rot), scaled: "none", "linear", "bands" or "yarn" (bs_rotary_frequencies)."""
    freq, amplitude = np.zeros(max(int(rot), 0) // 2 + 1, dtype=np.uint64), C.c_float(0.0)
    _check(_lib.bs_rotary_frequencies(_SCALINGS[scaling], rot, base, factor, low, high, original, freq.ctypes.data_as(_vp),
                                      C.byref(amplitude)), "bs_rotary_frequencies")
    return RotaryTable(torch.from_numpy(freq[: rot // 2].view(np.int64)).to(device), amplitude.value, rot)


def _heads(x, index: int):
    """Pointer, strides and heads of [T, H, d] on GPU `index`, last dimension contiguous; an absent one has no heads."""
    if x is None:
        return 0, 0, 0, 0
    assert x.get_device() == index, _ELSEWHERE
    t, h, one = x.stride()
    assert one == 1 or x.shape[2] == 1, "the last dimension must be contiguous"
    return x.data_ptr(), t, h, x.shape[1]


def bs_rotary(q, k, positions, table: RotaryTable, interleaved: bool, q_out, k_out, cu_new=None, node_parent=None, stream=None) -> None:
    """q, q_out [T, Hq, d] and k, k_out [T, Hkv, d] (bf16 or fp32; either pair may be None; q_out may be q) rotated to `positions`
    [T] int32.  node_parent [B, Nmax] with cu_new [B + 1]: trees of drafts, a node stands its depth behind its root."""
    some = q if q is not None else k
    T, _, d = some.shape
    index, dtype, freq = _gpu(some), some.dtype, table.freq
    assert (q is None) == (q_out is None) and (k is None) == (k_out is None)
    assert q is None or (q.shape[0] == T and q.shape[2] == d and q_out.shape == q.shape and q.dtype is dtype and q_out.dtype is dtype)
    assert k is None or (k.shape[0] == T and k.shape[2] == d and k_out.shape == k.shape and k.dtype is dtype and k_out.dtype is dtype)
    table_at = _of(freq, torch.int64, table.rot // 2, index)
    B, Nmax = (0, 0) if node_parent is None else node_parent.shape
    parent = _i32(node_parent, B * Nmax, index)
    if node_parent is not None:
        assert cu_new is not None, "trees need cu_new"
        if Nmax == 0:                                        # an empty tensor has no address, and NULL would mean chains
            parent = positions.data_ptr()
    qp, qt, qh, Hq = _heads(q, index)
    kp, kt, kh, Hkv = _heads(k, index)
    qop, qot, qoh, _ = _heads(q_out, index)
    kop, kot, koh, _ = _heads(k_out, index)
    _call(_lib.bs_rotary, "bs_rotary", index, stream, qp, qt, qh, kp, kt, kh, _dtype_code(some), _i32(positions, T, index), table_at,
          table.amplitude, table.rot, 1 if interleaved else 0, None if node_parent is None else _i32(cu_new, B + 1, index), parent, B, Nmax,
          T, Hq, Hkv, d, qop, qot, qoh, kop, kot, koh)


# ---- attention of whole prompts ------------------------------------------------------------------

def bs_prompt_attention(q, k, v, cu_seqlens, softmax_scale: float, out, status=None, stream=None) -> None:
    """q, out [T, Hq, d], k, v [T, Hkv, d] bf16 (last dimension contiguous): causal attention within the sequences of cu_seqlens [B + 1]."""
    T, Hq, d = q.shape
    index, B = _gpu(q), cu_seqlens.numel() - 1
    assert q.dtype is _bf16 and k.dtype is _bf16 and v.dtype is _bf16 and out.dtype is _bf16
    assert out.shape == q.shape and k.shape == v.shape and k.shape[0] == T and k.shape[2] == d
    qp, qt, qh, _ = _heads(q, index)
    kp, kt, kh, Hkv = _heads(k, index)
    vp, vt, vh, _ = _heads(v, index)
    op, ot, oh, _ = _heads(out, index)
    _call(_lib.bs_prompt_attention, "bs_prompt_attention", index, stream, qp, qt, qh, kp, kt, kh, vp, vt, vh, _i32(cu_seqlens, B + 1, index),
          B, T, Hq, Hkv, d, softmax_scale, op, ot, oh, _i32(status, B, index))


def bs_prompt_get_device_status(device="cuda", stream=None) -> None:
    """Raises BanditSpecError (BS_ERR_TIMEOUT) if a bounded wait gave up in a bs_prompt_attention on that GPU since the last such answer
    (synchronises the stream)."""
    device = torch.device(device)
    index = torch.cuda.current_device() if device.index is None else device.index
    _call(_lib.bs_prompt_get_device_status, "bs_prompt_get_device_status", index, stream)


# ---- logits before the verification ------------------------------------------------------------

def new_history(B: int, V: int, device="cuda") -> torch.Tensor:
    """Token histories without an entry: int16 [B, V]."""
    return torch.zeros(B, V, dtype=torch.int16, device=device)


def bs_history_update(history, fresh=None, cu_prompt=None, prompt_tokens=None, out_tokens=None, out_len=None, status=None,
                      stream=None) -> None:
    """Enters prompt_tokens (packed by cu_prompt) and the first out_len[b] of out_tokens [B, W] in history [B, V] int16; histories
    with fresh[b] begin anew."""
    B, V = history.shape
    index = _gpu(history)
    assert (out_tokens is None) == (out_len is None) and (cu_prompt is None) == (prompt_tokens is None)
    Tp = 0 if prompt_tokens is None else prompt_tokens.numel()
    W = 0 if out_tokens is None else out_tokens.shape[1]
    _call(_lib.bs_history_update, "bs_history_update", index, stream, _of(history, torch.int16, B * V, index), B, V,
          _of(fresh, torch.uint8, B, index), _i32(cu_prompt, B + 1, index), _i32(prompt_tokens, Tp, index), Tp,
          _i32(out_tokens, B * W, index), _i32(out_len, B, index), W, _i32(status, B, index))


def bs_logits_adjust(logits, out, gamma, extra: int, rows=None, draft_tokens=None, node_parent=None, history=None, repetition=None,
                     presence=None, frequency=None, bias_begin=None, bias_tokens=None, bias_values=None, masks=None, mask_row=None,
                     status=None, stream=None) -> None:
    """Penalties, biases and grammar masks on rows (begin, end) of logits [B, R, V] below gamma_b + extra; out may be logits."""
    B, R, V = logits.shape
    index = _gpu(logits)
    begin, end = (0, R) if rows is None else rows
    N = 0 if draft_tokens is None else draft_tokens.shape[1]
    n_bias = 0 if bias_tokens is None else bias_tokens.numel()
    assert (bias_begin is None) == (bias_tokens is None) == (bias_values is None)
    assert (masks is None) == (mask_row is None)
    n_masks = 0 if masks is None else masks.shape[0]
    tokens, parent = _i32(draft_tokens, B * N, index), _i32(node_parent, B * N, index)
    if draft_tokens is not None and N == 0:                  # an empty tensor has no address; nothing of it is read
        tokens, parent = logits.data_ptr(), None
    _call(_lib.bs_logits_adjust, "bs_logits_adjust", index, stream, _of(logits, logits.dtype, B * R * V, index),
          _of(out, logits.dtype, B * R * V, index), _dtype_code(logits), _i32(gamma, B, index), extra, begin, end, tokens, parent, N,
          _of(history, torch.int16, B * V, index), _of(repetition, _f32, B, index), _of(presence, _f32, B, index),
          _of(frequency, _f32, B, index), _i32(bias_begin, B + 1, index), _i32(bias_tokens, n_bias, index),
          _of(bias_values, _f32, n_bias, index), n_bias, _i32(masks, n_masks * ((V + 31) // 32), index), n_masks,
          _i32(mask_row, B * R, index), B, R, V, _i32(status, B, index))


# ---- bandits ---------------------------------------------------------------------------

def bs_bandit_state_bytes(alg: int, B: int, K: int) -> int:
    return int(_lib.bs_bandit_state_bytes(alg, B, K))


def bs_bandit_init(state: torch.Tensor, alg: int, B: int, K: int, arm_gamma: Sequence[int],
                   delta: float = 0.5, stream=None) -> None:
    ag = np.ascontiguousarray(arm_gamma, dtype=np.int32)
    assert ag.shape == (K,)
    _check(_lib.bs_bandit_init(_ptr(state), state.numel(), alg, B, K, ag.ctypes.data_as(_vp),
                               float(delta), _stream(stream)), "bs_bandit_init")


def bs_bandit_select(state, alg: int, B: int, K: int, u_arm, active, arm, gamma, index_out=None,
                     stream=None) -> None:
    _check(_lib.bs_bandit_select(_ptr(state), state.numel(), alg, B, K, _ptr(u_arm), _ptr(active),
                                 _ptr(arm), _ptr(gamma), _ptr(index_out), _stream(stream)), "bs_bandit_select")


def bs_bandit_update(state, alg: int, B: int, K: int, arm, reward_y, active=None, stream=None) -> None:
    _check(_lib.bs_bandit_update(_ptr(state), state.numel(), alg, B, K, _ptr(arm), _ptr(reward_y),
                                 _ptr(active), _stream(stream)), "bs_bandit_update")


def bs_bandit_step(state, alg: int, B: int, K: int, reward, u_arm_next, active, arm, gamma, index_out=None,
                   stream=None) -> None:
    """Update with this round's reward (int32 accepted lengths, or fp64 rewards for BS_UCB_REWARD) and
    select the next round's arms, in one launch; `arm` is read and overwritten."""
    ry, rr = (None, reward) if alg == BS_UCB_REWARD else (reward, None)
    assert (rr.dtype == torch.float64) if rr is not None else (ry.dtype == torch.int32)
    _check(_lib.bs_bandit_step(_ptr(state), state.numel(), alg, B, K, _ptr(ry), _ptr(rr), _ptr(u_arm_next),
                               _ptr(active), _ptr(arm), _ptr(gamma), _ptr(index_out), _stream(stream)),
           "bs_bandit_step")


def bs_bandit_read(state, alg: int, B: int, K: int, stream=None) -> dict:
    """Sufficient statistics as host arrays: UCBSpec {n, sumY, t}; EXP3Spec {S, n, t}; real-reward
    UCBSpec {S (the reward sums), n, t}."""
    t = np.zeros(B, dtype=np.int64)
    if alg == BS_UCB:
        n = np.zeros((B, K), dtype=np.int64)
        sy = np.zeros((B, K), dtype=np.int64)
        _check(_lib.bs_bandit_read(_ptr(state), state.numel(), alg, B, K, n.ctypes.data_as(_vp),
                                   sy.ctypes.data_as(_vp), None, t.ctypes.data_as(_vp), _stream(stream)),
               "bs_bandit_read")
        return {"n": n, "sumY": sy, "t": t}
    S = np.zeros((B, K), dtype=np.float64)
    n = np.zeros((B, K), dtype=np.int64)
    _check(_lib.bs_bandit_read(_ptr(state), state.numel(), alg, B, K, n.ctypes.data_as(_vp), None,
                               S.ctypes.data_as(_vp), t.ctypes.data_as(_vp), _stream(stream)), "bs_bandit_read")
    return {"S": S, "n": n, "t": t}


def bs_bandit_init_reward(state: torch.Tensor, B: int, K: int, arm_gamma: Sequence[int], delta: float,
                          reward_width: float, stream=None) -> None:
    ag = np.ascontiguousarray(np.asarray(arm_gamma, dtype=np.int32))
    assert ag.shape == (K,)
    _check(_lib.bs_bandit_init_reward(_ptr(state), state.numel(), B, K, ag.ctypes.data_as(_vp), float(delta),
                                      float(reward_width), _stream(stream)), "bs_bandit_init_reward")


def bs_bandit_update_reward(state, B: int, K: int, arm, reward, active=None, stream=None) -> None:
    assert reward.dtype == torch.float64
    _check(_lib.bs_bandit_update_reward(_ptr(state), state.numel(), B, K, _ptr(arm), _ptr(reward), _ptr(active),
                                        _stream(stream)), "bs_bandit_update_reward")


def bs_throughput_reward(out_len, active, B: int, seconds: float, whole_batch: bool, reward, stream=None) -> None:
    assert out_len.dtype == torch.int32 and reward.dtype == torch.float64
    _check(_lib.bs_throughput_reward(_ptr(out_len), _ptr(active), B, float(seconds), int(bool(whole_batch)),
                                     _ptr(reward), _stream(stream)), "bs_throughput_reward")


def new_bandit(alg: int, B: int, arm_gamma: Sequence[int], delta: float = 0.5, device="cuda",
               reward_width: Optional[float] = None) -> torch.Tensor:
    K = len(arm_gamma)
    n = bs_bandit_state_bytes(alg, B, K)
    if n == 0:
        raise BanditSpecError(BS_ERR_UNSUPPORTED, "bs_bandit_state_bytes")
    state = torch.empty(n, dtype=torch.uint8, device=device)
    if alg == BS_UCB_REWARD:
        bs_bandit_init_reward(state, B, K, arm_gamma, delta, reward_width)
    else:
        bs_bandit_init(state, alg, B, K, arm_gamma, delta)
    return state
