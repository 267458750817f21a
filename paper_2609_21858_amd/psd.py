"""Thin ctypes binding of libpsd (the C ABI in include/psd.h).

Argument marshalling only: every step of the sampler runs in the HIP kernels of
libpsd.  PyTorch provides device memory and the current stream.  If the built
library is missing, importing this module raises -- there is no fallback.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "lib", "libpsd.so")

PSD_OK, PSD_E_ARG, PSD_E_UNSUPPORTED, PSD_E_HIP, PSD_E_WORKSPACE = 0, -1, -2, -3, -4
PSD_F32, PSD_BF16 = 0, 1
PSD_MODE_HET, PSD_MODE_MPFR = 0, 1
PSD_CLOCKS_TREE, PSD_CLOCKS_FLAT = 0, 1
ERR_SPIN, ERR_CAND = 1, 2


class PsdError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"psd status {status}: {msg}")
        self.status = status


class Params(ctypes.Structure):
    _fields_ = [
        ("key", ctypes.c_uint64),
        ("vocab", ctypes.c_int32),
        ("num_drafts", ctypes.c_int32),
        ("ctx_window", ctypes.c_int32),
        ("temp_target", ctypes.c_float),
        ("temp_draft", ctypes.c_float),
        ("dtype", ctypes.c_int32),
        ("mode", ctypes.c_int32),
        ("clocks", ctypes.c_int32),
        ("top_k", ctypes.c_int32),
        ("top_p", ctypes.c_float),
    ]


class Block(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32),
        ("gamma", ctypes.c_int32),
        ("prefix_tokens", ctypes.c_void_p),
        ("start_pos", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p),
        ("workspace_bytes", ctypes.c_size_t),
        ("status", ctypes.c_void_p),
    ]


class Cache(ctypes.Structure):
    """psd_cache: keys and values in pages (make_cache)."""
    _fields_ = [
        ("k", ctypes.c_void_p),
        ("v", ctypes.c_void_p),
        ("dtype", ctypes.c_int32),
        ("heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("page_tokens", ctypes.c_int32),
        ("pages", ctypes.c_int32),
        ("layers", ctypes.c_int32),
        ("stride_layer", ctypes.c_int64),
        ("stride_page", ctypes.c_int64),
        ("stride_token", ctypes.c_int64),
        ("stride_head", ctypes.c_int64),
    ]


class Seqs(ctypes.Structure):
    """psd_seqs: the sequences of one call (make_seqs)."""
    _fields_ = [
        ("batch", ctypes.c_int32),
        ("rows", ctypes.c_int32),
        ("max_new", ctypes.c_int32),
        ("max_kv", ctypes.c_int32),
        ("table_width", ctypes.c_int32),
        ("table_stride", ctypes.c_int64),
        ("new_start", ctypes.c_void_p),
        ("kv_len", ctypes.c_void_p),
        ("table", ctypes.c_void_p),
    ]


class Rows(ctypes.Structure):
    """psd_rows: packed rows of heads."""
    _fields_ = [("data", ctypes.c_void_p), ("stride_row", ctypes.c_int64), ("stride_head", ctypes.c_int64)]


class Rotation(ctypes.Structure):
    """psd_rotation: norms and position rotation of psd_kv_append."""
    _fields_ = [
        ("rotary", ctypes.c_int32),
        ("interleaved", ctypes.c_int32),
        ("positions_max", ctypes.c_int32),
        ("cos", ctypes.c_void_p),
        ("sin", ctypes.c_void_p),
        ("positions", ctypes.c_void_p),
        ("q_norm", ctypes.c_void_p),
        ("k_norm", ctypes.c_void_p),
        ("eps", ctypes.c_float),
    ]


class ToyLM(ctypes.Structure):
    """psd_toy_lm: the synthetic position-indexed model of psd_toy_logits / psd_generate."""
    _fields_ = [
        ("seed", ctypes.c_uint64),
        ("draft_seed", ctypes.c_uint64),
        ("sigma", ctypes.c_float),
        ("alpha", ctypes.c_float),
        ("tau", ctypes.c_float * 2),
        ("tau_split", ctypes.c_int32),
    ]


def make_toy_lm(seed: int, draft_seed: int, sigma: float, alpha: float, tau=(1.0, 1.0), tau_split: int = 0) -> ToyLM:
    lm = ToyLM(seed & 0xFFFFFFFFFFFFFFFF, draft_seed & 0xFFFFFFFFFFFFFFFF, sigma, alpha)
    lm.tau[0], lm.tau[1] = float(tau[0]), float(tau[1])
    lm.tau_split = int(tau_split)
    return lm


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built: run __graft_entry__.build() (hipcc, gfx950)")
    lib = ctypes.CDLL(LIB_PATH)
    P = ctypes.POINTER(Params)
    Bp = ctypes.POINTER(Block)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    sigs = {
        "psd_abi_version": ([], i32),
        "psd_last_error": ([], ctypes.c_char_p),
        "psd_workspace_bytes": ([P, i32, i32], sz),
        "psd_workspace_clear": ([vp, sz, vp], i32),
        "psd_workspace_errors": ([vp, vp, ctypes.POINTER(ctypes.c_uint32)], i32),
        "psd_draft": ([P, Bp, i32, i32, vp, vp, vp, vp], i32),
        "psd_verify": ([P, Bp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp], i32),
        "psd_verify_static": ([P, Bp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp], i32),
        "psd_detect": ([P, i32, i32, vp, vp, vp, vp, vp, vp], i32),
        "psd_detect_pvalue": ([i32, vp, vp, vp, vp, vp], i32),
        "psd_philox": ([i32, vp, vp, vp, vp], i32),
        "psd_context_keys": ([P, i32, vp, vp, vp, vp], i32),
        "psd_clock_values": ([P, i32, vp, vp, vp, vp, vp], i32),
        "psd_set_spin_limit": ([ctypes.c_uint32], None),
        "psd_detect_scores": ([P, vp, i32, i32, i32, vp, vp, vp, vp, vp], i32),
        "psd_detect_scores_pvalue": ([vp, i32, vp, vp, vp, vp], i32),
        "psd_detection_rate": ([i32, vp, i32, ctypes.c_double, vp, vp], i32),
        "psd_advance": ([P, i32, i32, ctypes.c_int64, vp, vp, vp, ctypes.c_int64, vp, vp, vp, vp, vp], i32),
        "psd_toy_logits": ([P, ctypes.POINTER(ToyLM), i32, i32, vp, vp, vp, vp], i32),
        "psd_generate_workspace_bytes": ([P, i32, i32], sz),
        "psd_generate": ([P, ctypes.POINTER(ToyLM), i32, i32, i32, vp, ctypes.c_int64, vp, sz, i32, i32,
                          ctypes.POINTER(i32), ctypes.POINTER(ctypes.c_uint32), vp], i32),
        # structs by address: a Cache, Seqs, Rows or Rotation (or None for a NULL pointer) goes in by byref()
        "psd_kv_append": ([vp, vp, vp, vp, vp, vp, vp, i32, vp], i32),
        "psd_attention": ([vp, vp, vp, i32, ctypes.c_float, i32, vp, i32, vp, vp, vp, sz, vp], i32),
        "psd_attention_workspace_bytes": ([vp, vp, i32], sz),
        "psd_kv_keep": ([vp, vp, vp, ctypes.c_int64, i32, vp, vp, vp], i32),
        "psd_verify_given": ([P, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp], i32),
        "psd_verify_given_workspace_bytes": ([P, i32, i32], sz),
    }
    for name, (args, res) in sigs.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = res
    return lib


_lib = _load()
EXPORTS = ("psd_abi_version", "psd_last_error", "psd_workspace_bytes", "psd_workspace_clear",
           "psd_workspace_errors", "psd_draft", "psd_verify", "psd_verify_static", "psd_detect", "psd_detect_pvalue", "psd_philox",
           "psd_context_keys", "psd_clock_values", "psd_set_spin_limit", "psd_detect_scores",
           "psd_detect_scores_pvalue", "psd_detection_rate", "psd_advance", "psd_toy_logits",
           "psd_generate_workspace_bytes", "psd_generate", "psd_kv_append", "psd_attention",
           "psd_attention_workspace_bytes", "psd_kv_keep", "psd_verify_given", "psd_verify_given_workspace_bytes")


def lib():
    return _lib


def _check(status: int):
    if status != PSD_OK:
        raise PsdError(status, (_lib.psd_last_error() or b"").decode())


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    if stream is None:
        # the current stream's handle without a Stream object around it (0.1 us instead of 2.8)
        return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))
    return ctypes.c_void_p(stream.cuda_stream)


def make_params(key: int, vocab: int, num_drafts: int, ctx_window: int, temp_target: float = 1.0,
                temp_draft: float = 1.0, dtype=torch.bfloat16, mode: int = PSD_MODE_HET,
                clocks: int = PSD_CLOCKS_TREE, top_k: int = 0, top_p: float = 1.0) -> Params:
    dt = dtype if isinstance(dtype, int) else (PSD_BF16 if dtype == torch.bfloat16 else PSD_F32)
    return Params(key & 0xFFFFFFFFFFFFFFFF, vocab, num_drafts, ctx_window, temp_target, temp_draft, dt, mode,
                  clocks, top_k, top_p)


def workspace_bytes(params: Params, batch: int, gamma: int) -> int:
    return int(_lib.psd_workspace_bytes(ctypes.byref(params), batch, gamma))


def new_workspace(params: Params, batch: int, gamma: int, device="cuda") -> torch.Tensor:
    """Zero-filled device workspace (torch allocation, 256-byte aligned)."""
    n = workspace_bytes(params, batch, gamma)
    if n == 0:
        raise PsdError(PSD_E_ARG, "invalid parameters for workspace sizing")
    return torch.zeros(n, dtype=torch.uint8, device=device)


def workspace_clear(ws: torch.Tensor, stream=None):
    _check(_lib.psd_workspace_clear(_ptr(ws), ws.numel(), _stream(stream)))


def workspace_errors(ws: torch.Tensor, stream=None) -> int:
    out = ctypes.c_uint32(0)
    _check(_lib.psd_workspace_errors(_ptr(ws), _stream(stream), ctypes.byref(out)))
    return int(out.value)


def _block(batch, gamma, prefix, start_pos, ws, status=None):
    return Block(batch, gamma, prefix.data_ptr() if prefix is not None and prefix.numel() else None,
                 start_pos.data_ptr(), ws.data_ptr(), ws.numel(), None if status is None else status.data_ptr())


def set_spin_limit(polls: int = 0):
    """Test hook: polls of a bounded wait before it gives up (0 = default)."""
    _lib.psd_set_spin_limit(polls)


def draft(params: Params, ws, prefix_tokens, start_pos, gamma: int, s_begin: int, draft_logits, draft_tokens,
          draft_lse=None, stream=None, status=None):
    """psd_draft: draft depths [s_begin, s_begin + draft_logits.shape[2]).  status: optional
    int32 [1] device tensor receiving the call's error bits."""
    B = int(start_pos.shape[0])
    blk = _block(B, gamma, prefix_tokens, start_pos, ws, status)
    _check(_lib.psd_draft(ctypes.byref(params), ctypes.byref(blk), s_begin, int(draft_logits.shape[2]),
                          _ptr(draft_logits), _ptr(draft_tokens), _ptr(draft_lse), _stream(stream)))


def verify(params: Params, ws, prefix_tokens, start_pos, target_logits, draft_logits=None, draft_tokens=None,
           target_rows: int = 1, want_lse: bool = False, want_targets: bool = False, out=None, stream=None,
           status=None):
    """psd_verify; allocates the outputs it is not given.  Returns a dict of tensors.  status:
    optional int32 [1] device tensor receiving the call's error bits."""
    B = int(start_pos.shape[0])
    K = params.num_drafts
    gamma = int(target_logits.shape[-2]) - 1
    dev = target_logits.device
    o = {} if out is None else dict(out)
    if draft_tokens is None:
        draft_tokens = torch.empty((B, K, gamma), dtype=torch.int32, device=dev)
    o["draft_tokens"] = draft_tokens
    o.setdefault("out_tokens", torch.empty((B, gamma + 1), dtype=torch.int32, device=dev))
    o.setdefault("out_len", torch.empty((B,), dtype=torch.int32, device=dev))
    tshape = (B, gamma + 1) if target_rows == 1 else (B, K, gamma + 1)
    if want_lse:
        o.setdefault("target_lse", torch.empty(tshape, dtype=torch.float32, device=dev))
        if draft_logits is not None:
            o.setdefault("draft_lse", torch.empty((B, K, gamma), dtype=torch.float32, device=dev))
    if want_targets:
        o.setdefault("target_tokens", torch.empty(tshape, dtype=torch.int32, device=dev))
    blk = _block(B, gamma, prefix_tokens, start_pos, ws, status)
    _check(_lib.psd_verify(ctypes.byref(params), ctypes.byref(blk), target_rows, _ptr(target_logits),
                           _ptr(draft_logits), _ptr(draft_tokens), _ptr(o["out_tokens"]), _ptr(o["out_len"]),
                           _ptr(o.get("target_lse")), _ptr(o.get("draft_lse")), _ptr(o.get("target_tokens")),
                           _stream(stream)))
    return o


def verify_static(params: Params, prefix_tokens, start_pos, target_logits, draft_logits=None, draft_tokens=None,
                  target_rows: int = 1, out=None, status=None, stream=None):
    """psd_verify_static (the library's fixed scratch, no workspace).  Outputs come
    from `out` (a dict of tensors: draft_tokens, out_tokens, out_len and optionally
    target_lse, draft_lse, target_tokens) or are allocated here by torch when missing."""
    B = int(start_pos.shape[0])
    K = params.num_drafts
    gamma = int(target_logits.shape[-2]) - 1
    dev = target_logits.device
    o = {} if out is None else dict(out)
    if draft_tokens is None:
        draft_tokens = o.get("draft_tokens")
    if draft_tokens is None:
        draft_tokens = torch.empty((B, K, gamma), dtype=torch.int32, device=dev)
    o["draft_tokens"] = draft_tokens
    o.setdefault("out_tokens", torch.empty((B, gamma + 1), dtype=torch.int32, device=dev))
    o.setdefault("out_len", torch.empty((B,), dtype=torch.int32, device=dev))
    blk = Block(B, gamma, prefix_tokens.data_ptr() if prefix_tokens is not None and prefix_tokens.numel() else None,
                start_pos.data_ptr(), None, 0, None if status is None else status.data_ptr())
    _check(_lib.psd_verify_static(ctypes.byref(params), ctypes.byref(blk), target_rows, _ptr(target_logits),
                                  _ptr(draft_logits), _ptr(draft_tokens), _ptr(o["out_tokens"]), _ptr(o["out_len"]),
                                  _ptr(o.get("target_lse")), _ptr(o.get("draft_lse")), _ptr(o.get("target_tokens")),
                                  _stream(stream)))
    return o


def detect(params: Params, tokens, n0, per_token: bool = False, stream=None):
    """psd_detect -> (score f64 [n_seq], count i32 [n_seq], per-token f32 or None)."""
    n_seq, seq_len = int(tokens.shape[0]), int(tokens.shape[1])
    dev = tokens.device
    score = torch.empty((n_seq,), dtype=torch.float64, device=dev)
    count = torch.empty((n_seq,), dtype=torch.int32, device=dev)
    per = torch.empty((n_seq, seq_len), dtype=torch.float32, device=dev) if per_token else None
    _check(_lib.psd_detect(ctypes.byref(params), n_seq, seq_len, _ptr(tokens), _ptr(n0), _ptr(score), _ptr(count),
                           _ptr(per), _stream(stream)))
    return score, count, per


class ScoreParams(ctypes.Structure):
    _fields_ = [("li_delta", ctypes.c_double), ("pl_eps", ctypes.c_double)]


def detect_scores(params: Params, tokens, n0, li_delta: float, pl_eps: float, seq_len: int = None, stream=None):
    """psd_detect_scores -> (scores f64 [n_seq][4] = S_A, S_U, S_Li, S_PL; count i32 [n_seq]).
    seq_len < tokens.shape[1] scores that prefix of every row."""
    n_seq, stride = int(tokens.shape[0]), int(tokens.shape[1])
    seq_len = stride if seq_len is None else int(seq_len)
    sp = ScoreParams(li_delta, pl_eps)
    scores = torch.empty((n_seq, 4), dtype=torch.float64, device=tokens.device)
    count = torch.empty((n_seq,), dtype=torch.int32, device=tokens.device)
    _check(_lib.psd_detect_scores(ctypes.byref(params), ctypes.byref(sp), n_seq, seq_len, stride, _ptr(tokens),
                                  _ptr(n0), _ptr(scores), _ptr(count), _stream(stream)))
    return scores, count


def detect_scores_pvalue(scores, count, li_delta: float, pl_eps: float, stream=None):
    """psd_detect_scores_pvalue -> ln p f64 [n_seq][4] (A exact; U, Li, PL Chernoff bounds)."""
    n = int(scores.shape[0])
    sp = ScoreParams(li_delta, pl_eps)
    out = torch.empty((n, 4), dtype=torch.float64, device=scores.device)
    _check(_lib.psd_detect_scores_pvalue(ctypes.byref(sp), n, _ptr(scores), _ptr(count), _ptr(out),
                                         _stream(stream)))
    return out


def detection_rate(log_p, alpha: float, stream=None):
    """psd_detection_rate over a column of log p-values ([n] or [n][c] with one column
    selected by the caller's view) -> int32 [1] count with ln p <= ln alpha."""
    n = int(log_p.shape[0])
    stride = int(log_p.stride(0))
    out = torch.empty((1,), dtype=torch.int32, device=log_p.device)
    _check(_lib.psd_detection_rate(n, _ptr(log_p), stride, alpha, _ptr(out), _stream(stream)))
    return out


def detect_pvalue(score, count, stream=None):
    """psd_detect_pvalue -> (ln p_A f64 [n_seq], ANLPPT_A f64 [n_seq]) of S_A ~ Gamma(M, 1) under the null."""
    n = int(score.shape[0])
    log_p = torch.empty((n,), dtype=torch.float64, device=score.device)
    anl = torch.empty((n,), dtype=torch.float64, device=score.device)
    _check(_lib.psd_detect_pvalue(n, _ptr(score), _ptr(count), _ptr(log_p), _ptr(anl), _stream(stream)))
    return log_p, anl


def philox(ctr, key, stream=None):
    n = int(ctr.shape[0])
    out = torch.empty((n, 4), dtype=torch.int32, device=ctr.device)
    _check(_lib.psd_philox(n, _ptr(ctr), _ptr(key), _ptr(out), _stream(stream)))
    return out


def context_keys(params: Params, t, windows, stream=None):
    n = int(t.shape[0])
    out = torch.empty((n, 2), dtype=torch.int32, device=t.device)
    _check(_lib.psd_context_keys(ctypes.byref(params), n, _ptr(t), _ptr(windows) if windows is not None and
                                 windows.numel() else None, _ptr(out), _stream(stream)))
    return out


def clock_values(params: Params, kappa, slot, token, stream=None):
    n = int(slot.shape[0])
    out = torch.empty((n,), dtype=torch.float64, device=slot.device)
    _check(_lib.psd_clock_values(ctypes.byref(params), n, _ptr(kappa), _ptr(slot), _ptr(token), _ptr(out),
                                 _stream(stream)))
    return out


# ---------------------------------------------------------------- multi-block generation

def advance(params: Params, gamma: int, max_len: int, text, length, prefix, start_pos, n_active, out_tokens=None,
            out_len=None, stream=None):
    """psd_advance: commit one block (out_len None: set up the first block from the prompts)."""
    B = int(text.shape[0])
    _check(_lib.psd_advance(ctypes.byref(params), B, gamma, int(max_len), _ptr(out_tokens), _ptr(out_len),
                            _ptr(text), int(text.stride(0)), _ptr(length),
                            _ptr(prefix) if prefix is not None and prefix.numel() else None, _ptr(start_pos),
                            _ptr(n_active), _stream(stream)))


def toy_logits(params: Params, lm: ToyLM, gamma: int, start_pos, drafts: bool = True, stream=None):
    """psd_toy_logits -> (target rows [B][gamma+1][V], draft rows [B][K][gamma][V] or None)."""
    B, V, K = int(start_pos.shape[0]), params.vocab, params.num_drafts
    dt = torch.bfloat16 if params.dtype == PSD_BF16 else torch.float32
    tl = torch.empty((B, gamma + 1, V), dtype=dt, device=start_pos.device)
    dl = torch.empty((B, K, gamma, V), dtype=dt, device=start_pos.device) if drafts else None
    _check(_lib.psd_toy_logits(ctypes.byref(params), ctypes.byref(lm), B, gamma, _ptr(start_pos), _ptr(tl), _ptr(dl),
                               _stream(stream)))
    return tl, dl


def generate_workspace_bytes(params: Params, batch: int, gamma: int) -> int:
    return int(_lib.psd_generate_workspace_bytes(ctypes.byref(params), batch, gamma))


def generate(params: Params, lm: ToyLM, prompts, n_pos: int, gamma: int, check_every: int = 16,
             use_graph: bool = False, ws=None, stream=None):
    """psd_generate: n_pos tokens after each prompt (int32 [B][m], m = ctx_window) on the device.
    Returns (text int32 [B][m + n_pos], blocks, error bits)."""
    B, m = int(prompts.shape[0]), params.ctx_window
    assert prompts.shape[1] == m
    text = torch.full((B, m + n_pos), -1, dtype=torch.int32, device=prompts.device)
    text[:, :m] = prompts
    if ws is None:
        n = generate_workspace_bytes(params, B, gamma)
        if n == 0:
            raise PsdError(PSD_E_ARG, "invalid parameters for generation")
        ws = torch.empty(n, dtype=torch.uint8, device=prompts.device)
    blocks = ctypes.c_int32(0)
    bits = ctypes.c_uint32(0)
    _check(_lib.psd_generate(ctypes.byref(params), ctypes.byref(lm), B, gamma, n_pos, _ptr(text), int(text.stride(0)),
                             _ptr(ws), ws.numel(), check_every, 1 if use_graph else 0, ctypes.byref(blocks),
                             ctypes.byref(bits), _stream(stream)))
    return text, int(blocks.value), int(bits.value)



# ---------------------------------------------------------------- the target's pass over a block's new tokens

# A refusal builds its message only when it refuses: a call's checks cost about a microsecond.

def _refuse(msg: str):
    raise PsdError(PSD_E_ARG, msg)


_DTYPES = {torch.bfloat16: PSD_BF16, torch.float32: PSD_F32}


def _dtype(t) -> int:
    d = _DTYPES.get(t.dtype)
    if d is None:
        _refuse(f"dtype {t.dtype} is neither bfloat16 nor float32")
    return d


def _ints(t, what: str, dim: int, rows: int = 0):
    if t.dtype != torch.int32 or t.dim() != dim or (t.shape[-1] > 1 and t.stride(-1) != 1) or t.shape[0] < rows:
        _refuse(f"{what}: int32 with {dim} dimensions, at least {rows} long, the last dimension contiguous")


def _row_stride(t, what: str) -> int:
    """Elements from one row of a matrix of indices to the next; rows that overlap (an expanded tensor's lie on one
    another) have no stride that the calls could take."""
    rows, width = t.shape
    if rows == 1:
        return width
    if t.stride(0) < width:
        _refuse(f"{what}: rows overlap (stride {t.stride(0)}, width {width}); .contiguous() gives each its own")
    return t.stride(0)


def make_cache(k, v) -> Cache:
    """Pools [pages][page tokens][heads][head dim] (or [layers][pages]...) of any strides with a contiguous
    last dimension; keeps both tensors alive."""
    if k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype:
        _refuse("k and v pools differ in layout")
    if k.dim() not in (4, 5) or k.stride(-1) != 1:
        _refuse("pools are [layers][pages][page tokens][heads][head dim]")
    pages, page, heads, dim = k.shape[-4:]
    st = k.stride()
    c = Cache(k.data_ptr(), v.data_ptr(), _dtype(k), heads, dim, page, pages, k.shape[0] if k.dim() == 5 else 1,
              st[0] if k.dim() == 5 else 0, st[-4], st[-3], st[-2])
    c.tensors = (k, v)
    return c


def make_seqs(new_start, kv_len, table, rows: int, max_new: int, max_kv: int) -> Seqs:
    """Sequences of one call: new_start int32 [B+1], kv_len int32 [B], table int32 [B][width]; rows, max_new and
    max_kv bound the lengths, which may change on the device.  Keeps the tensors alive."""
    _ints(new_start, "new_start", 1)
    _ints(kv_len, "kv_len", 1)
    _ints(table, "table", 2)
    B = int(kv_len.shape[0])
    if new_start.shape[0] != B + 1 or table.shape[0] != B:
        _refuse("new_start [B+1], kv_len [B] and table [B][width] disagree")
    s = Seqs(B, int(rows), int(max_new), int(max_kv), table.shape[1], _row_stride(table, "table"),
             new_start.data_ptr(), kv_len.data_ptr(), table.data_ptr())
    s.tensors = (new_start, kv_len, table)
    return s


def _rows(t, what: str, cache: Cache, rows: int, heads: int) -> Rows:
    shape, stride = t.shape, t.stride()
    if (len(shape) != 3 or shape[0] < rows or shape[1] != heads or shape[2] != cache.head_dim or stride[2] != 1
            or _DTYPES.get(t.dtype) != cache.dtype):
        _refuse(f"{what}: [{rows}][{heads}][{cache.head_dim}] in the cache's dtype with a contiguous last dimension")
    return Rows(t.data_ptr(), stride[0], stride[1])


def _ref(s):
    return None if s is None else ctypes.byref(s)


def kv_append(cache: Cache, seqs: Seqs, k, v, q=None, q_out=None, cos=None, sin=None, interleaved: bool = False,
              positions=None, q_norm=None, k_norm=None, eps: float = 1e-6, stream=None):
    """psd_kv_append: keys (normed with k_norm, turned by cos and sin float32 [positions][R/2]) and values into the
    cache; returns the queries, treated the same way, in q_out (allocated when missing), or None without q."""
    rows, heads = seqs.rows, cache.heads
    rk, rv = _rows(k, "k", cache, rows, heads), _rows(v, "v", cache, rows, heads)
    rq = ro = None
    H = 0
    if q is not None:
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        H = q.shape[1]
        rq, ro = _rows(q, "q", cache, rows, H), _rows(q_out, "q_out", cache, rows, H)
    R = P = 0
    if cos is not None:
        if (sin is None or cos.shape != sin.shape or cos.dim() != 2 or cos.dtype != torch.float32
                or sin.dtype != torch.float32 or not cos.is_contiguous() or not sin.is_contiguous()):
            _refuse("cos and sin: contiguous float32 [positions][R/2]")
        P, R = cos.shape
        R *= 2
    if positions is not None:
        _ints(positions, "positions", 1, rows)
    for w in (q_norm, k_norm):
        if w is not None and (w.shape != (cache.head_dim,) or not w.is_contiguous() or _dtype(w) != cache.dtype):
            _refuse("q_norm and k_norm: [head dim] in the cache's dtype")
    rot = Rotation(R, 1 if interleaved else 0, P, _ptr(cos), _ptr(sin), _ptr(positions), _ptr(q_norm), _ptr(k_norm), eps)
    _check(_lib.psd_kv_append(ctypes.byref(cache), ctypes.byref(seqs), ctypes.byref(rot), ctypes.byref(rk),
                              ctypes.byref(rv), _ref(rq), _ref(ro), H, _stream(stream)))
    return q_out


def attention_workspace_bytes(cache: Cache, seqs: Seqs, q_heads: int) -> int:
    n = int(_lib.psd_attention_workspace_bytes(ctypes.byref(cache), ctypes.byref(seqs), q_heads))
    if n == ctypes.c_size_t(-1).value:
        raise PsdError(PSD_E_ARG, (_lib.psd_last_error() or b"").decode())
    return n


def new_attention_workspace(cache: Cache, seqs: Seqs, q_heads: int, device="cuda") -> torch.Tensor:
    """Zero-filled device workspace of psd_attention for these bounds (may be empty)."""
    return torch.zeros(attention_workspace_bytes(cache, seqs, q_heads), dtype=torch.uint8, device=device)


def attention(cache: Cache, seqs: Seqs, q, ws, scale: float = None, window: int = 0, mask=None, out=None,
              want_lse: bool = False, lse=None, stream=None):
    """psd_attention of q [rows][H][head dim] over the cache -> {"out", and "lse" float32 [rows][H] with
    want_lse}.  mask: int32 [rows][words], bit j % 32 of word j / 32 for new token j (draft paths).  scale
    defaults to 1 / sqrt(head dim)."""
    H, rows = q.shape[1], seqs.rows
    rq = _rows(q, "q", cache, rows, H)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    ro = _rows(out, "out", cache, rows, H)
    o = {"out": out}
    if want_lse:
        if lse is None:
            lse = torch.empty((q.shape[0], H), dtype=torch.float32, device=q.device)
        elif lse.dtype != torch.float32 or not lse.is_contiguous() or lse.shape[0] < rows or lse.shape[1:] != (H,):
            _refuse("lse: contiguous float32 [rows][H]")
        o["lse"] = lse
    words = 0
    if mask is not None:
        _ints(mask, "mask", 2, rows)
        if not mask.is_contiguous():
            _refuse("mask: contiguous int32 [rows][words]")
        words = mask.shape[1]
    if scale is None:
        scale = cache.head_dim ** -0.5
    _check(_lib.psd_attention(ctypes.byref(cache), ctypes.byref(seqs), ctypes.byref(rq), H, scale, window, _ptr(mask), words,
                              ctypes.byref(ro), _ptr(o.get("lse")), _ptr(ws), 0 if ws is None else ws.numel(),
                              _stream(stream)))
    return o


def kv_keep(cache: Cache, seqs: Seqs, keep, n_keep, kv_out=None, stream=None):
    """psd_kv_keep: new tokens keep[b][i] (int32 [B][width], strictly ascending), i < n_keep[b] (int32 [B]), move to the
    first new positions in every layer of the cache; returns the sequences' new lengths (int32 [B])."""
    B = seqs.batch
    _ints(keep, "keep", 2)
    _ints(n_keep, "n_keep", 1)
    if keep.shape[0] != B or n_keep.shape[0] != B:
        _refuse("keep [B][width], n_keep [B]")
    if kv_out is None:
        kv_out = torch.empty((B,), dtype=torch.int32, device=keep.device)
    else:
        _ints(kv_out, "kv_out", 1, B)
    _check(_lib.psd_kv_keep(ctypes.byref(cache), ctypes.byref(seqs), _ptr(keep), _row_stride(keep, "keep"), keep.shape[1],
                            _ptr(n_keep), _ptr(kv_out), _stream(stream)))
    return kv_out


# ---------------------------------------------------------------- verification from given random numbers

def verify_given_workspace_bytes(params: Params, batch: int, gamma: int) -> int:
    return int(_lib.psd_verify_given_workspace_bytes(ctypes.byref(params), batch, gamma))


def new_verify_given_workspace(params: Params, batch: int, gamma: int, device="cuda") -> torch.Tensor:
    """Device workspace of psd_verify_given (uninitialised)."""
    n = verify_given_workspace_bytes(params, batch, gamma)
    if n == 0:
        raise PsdError(PSD_E_ARG, (_lib.psd_last_error() or b"").decode())
    return torch.empty(n, dtype=torch.uint8, device=device)


def verify_given(params: Params, ws, target_logits, draft_logits, draft_tokens, u, e, n_drafts=None,
                 want_lse: bool = False, out=None, stream=None):
    """psd_verify_given: target rows [B][gamma+1][V], draft rows [B][gamma][V], drafts int32 [B][gamma], u float32
    [B][gamma], e float32 [B][V] -> {"out_tokens" int32 [B][gamma+1], "out_len" int32 [B], and with want_lse
    "target_lse", "draft_lse"}."""
    B, gamma = int(draft_tokens.shape[0]), int(draft_tokens.shape[1])
    V, dev = params.vocab, draft_tokens.device
    if (target_logits.shape != (B, gamma + 1, V) or draft_logits.shape != (B, gamma, V)
            or _dtype(target_logits) != params.dtype or _dtype(draft_logits) != params.dtype
            or not target_logits.is_contiguous() or not draft_logits.is_contiguous()):
        _refuse(f"target_logits ({B}, {gamma + 1}, {V}) and draft_logits ({B}, {gamma}, {V}): contiguous, in params' dtype")
    if draft_tokens.dtype != torch.int32 or not draft_tokens.is_contiguous():
        _refuse("draft_tokens: contiguous int32 [B][gamma]")
    if (u.shape != (B, gamma) or e.shape != (B, V) or u.dtype != torch.float32 or e.dtype != torch.float32
            or not u.is_contiguous() or not e.is_contiguous()):
        _refuse(f"u ({B}, {gamma}) and e ({B}, {V}): contiguous float32")
    if n_drafts is not None:
        _ints(n_drafts, "n_drafts", 1)
        if n_drafts.shape[0] != B:
            _refuse("n_drafts: int32 [B]")
    o = {} if out is None else dict(out)
    for name, shape, dt in (("out_tokens", (B, gamma + 1), torch.int32), ("out_len", (B,), torch.int32),
                            ("target_lse", (B, gamma + 1), torch.float32), ("draft_lse", (B, gamma), torch.float32)):
        if name not in o:
            if dt is torch.int32 or want_lse:
                o[name] = torch.empty(shape, dtype=dt, device=dev)
        elif o[name].shape != shape or o[name].dtype != dt or not o[name].is_contiguous():
            _refuse(f"{name}: contiguous {dt} {shape}")
    _check(_lib.psd_verify_given(ctypes.byref(params), B, gamma, _ptr(target_logits), _ptr(draft_logits), _ptr(draft_tokens),
                                 _ptr(n_drafts), _ptr(u), _ptr(e), _ptr(o["out_tokens"]), _ptr(o["out_len"]),
                                 _ptr(o.get("target_lse")), _ptr(o.get("draft_lse")), _ptr(ws), ws.numel(),
                                 _stream(stream)))
    return o
