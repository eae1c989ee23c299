"""Python binding of liblopa, the MI355X (gfx950) LoPA branch-verification step.

Argument marshalling only: every step of the method runs in the HIP kernels
behind the C ABI declared in include/lopa.h. PyTorch supplies device memory and
the stream. The functions keep the C names:

    lopa_build_branches            Eq. 1 + top-k lookahead branches (Alg. 1 steps 1-2)
    lopa_verify_forward            one batched forward of all branches (Alg. 1 step 3)
    lopa_branch_confidence_select  Eq. 2 scores, argmax, next state (Sec. 3.2 logit reuse)
    lopa_commit_kv                 winner K/V -> static cache (Sec. 3.4)

and, for callers that keep the K / V of many sequences in pages of their own:

    lopa_paged_append              head norms + rotation of new rows, K / V to their pages
    lopa_paged_attention           a ragged batch's rows over their pages
    lopa_token_logprobs            log probability, entropy and top tokens of rows of logits

Importing this module loads liblopa.so built in-tree by build.py (or
__graft_entry__.build()); there is no fallback: a missing library raises.
"""
from __future__ import annotations

import ctypes as C

import torch

from ._abi import (EXPORTS, LIB_PATH, LOPA_BF16, LOPA_ECAPACITY, LOPA_EHIP, LOPA_EINVAL,  # noqa: F401
                   LOPA_ENOMEM, LOPA_ESHAPE, LOPA_F16, LOPA_F32, LOPA_OK, MAX_BLOCK, MAX_ROWS, MAX_TOP,
                   METRIC_LOWEST_SEGMENT, METRIC_MEAN, METRIC_WINDOW_MIN, PRECISIONS, PROF_KINDS,
                   WINDOW_MAX_BLOCKS, LopaError, lib, lopa_layer_weights, lopa_model_cfg,
                   lopa_paged_batch, lopa_pages, lopa_weight_ptrs, lopa_window)


def _check(status: int):
    if status != LOPA_OK:
        raise LopaError(status, lib.lopa_last_error().decode())


def _ptr(t, dtype=None, name="tensor"):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name}: must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    return C.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


# ------------------------------------------------------------------ handles
class Model:
    """Repacked model weights on the device (lopa_model)."""

    def __init__(self, cfg: dict, weights: dict, stream=None, precision: str = "bf16"):
        """precision: "bf16", or "fp8_mlp" (gate / up / down in W8A8 E4M3 with
        per-channel weight and per-row activation scales)."""
        if precision not in PRECISIONS:
            raise ValueError(f"precision {precision!r} not in {sorted(PRECISIONS)}")
        c = lopa_model_cfg(cfg["layers"], cfg["hidden"], cfg["heads"], cfg["kv_heads"],
                           cfg["head_dim"], cfg["ffn"], cfg["vocab"], cfg["mask_id"],
                           cfg["rms_eps"], cfg["rope_theta"], 1 if cfg["qkv_bias"] else 0)
        bf = torch.bfloat16
        n = cfg["layers"]
        arr = (lopa_layer_weights * n)()
        for i, lw in enumerate(weights["layers"]):
            f = {}
            for key in ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down", "ln1", "ln2"):
                f[key] = _ptr(lw[key], bf, key)
            for key in ("bq", "bk", "bv"):
                f[key] = _ptr(lw[key], bf, key) if cfg["qkv_bias"] else None
            arr[i] = lopa_layer_weights(**f)
        w = lopa_weight_ptrs(_ptr(weights["embed"], bf, "embed"), arr,
                             _ptr(weights["final_norm"], bf, "final_norm"),
                             _ptr(weights["lm_head"], bf, "lm_head"))
        h = C.c_void_p()
        _check(lib.lopa_model_create_ex(C.byref(c), C.byref(w), PRECISIONS[precision],
                                        _stream(stream), C.byref(h)))
        self.handle, self.cfg, self.precision = h, dict(cfg), precision

    def close(self):
        if getattr(self, "handle", None) and lib is not None:
            lib.lopa_model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        self.close()


class KV:
    """Static KV cache + per-branch staging + verify workspace (lopa_kv)."""

    def __init__(self, model: Model, max_len: int, max_branches: int, max_block: int):
        h = C.c_void_p()
        _check(lib.lopa_kv_create(model.handle, max_len, max_branches, max_block, C.byref(h)))
        self.handle, self.model = h, model
        self.max_len, self.max_branches, self.max_block = max_len, max_branches, max_block
        self.block_causal = 0

    def read(self, layer: int, start: int, length: int, stream=None):
        c = self.model.cfg
        shp = (c["kv_heads"], length, c["head_dim"])
        k = torch.empty(shp, dtype=torch.bfloat16, device="cuda")
        v = torch.empty_like(k)
        _check(lib.lopa_kv_read(self.handle, layer, start, length, _ptr(k), _ptr(v), _stream(stream)))
        return k, v

    def write(self, layer: int, start: int, k: torch.Tensor, v: torch.Tensor, stream=None):
        _check(lib.lopa_kv_write(self.handle, layer, start, k.shape[1], _ptr(k, torch.bfloat16),
                                 _ptr(v, torch.bfloat16), _stream(stream)))

    def read_staging(self, branch: int, layer: int, L: int, stream=None):
        c = self.model.cfg
        k = torch.empty((c["kv_heads"], L, c["head_dim"]), dtype=torch.bfloat16, device="cuda")
        v = torch.empty_like(k)
        _check(lib.lopa_kv_read_staging(self.handle, branch, layer, _ptr(k), _ptr(v), _stream(stream)))
        return k, v

    def set_block_causal(self, sub_block: int):
        """0: full attention inside the block; c > 0 (multiple of 16): rows of
        sub-block b see the prefix and sub-blocks 0..b of their branch."""
        _check(lib.lopa_kv_set_block_causal(self.handle, sub_block))
        self.block_causal = sub_block

    def profile(self, kinds=()):
        """Time launches of the given kinds (names from PROF_KINDS) with HIP events."""
        mask = 0
        for kd in kinds:
            mask |= 1 << PROF_KINDS.index(kd)
        _check(lib.lopa_kv_profile(self.handle, mask))

    def profile_read(self) -> dict:
        """{kind: (total_ms, launches)} since the last read."""
        n = len(PROF_KINDS)
        ms = (C.c_double * n)()
        cnt = (C.c_int64 * n)()
        _check(lib.lopa_kv_profile_read(self.handle, ms, cnt))
        return {PROF_KINDS[i]: (ms[i], cnt[i]) for i in range(n)}

    def close(self):
        if getattr(self, "handle", None) and lib is not None:
            lib.lopa_kv_destroy(self.handle)
            self.handle = None

    def __del__(self):
        self.close()


# ------------------------------------------------------------- entry points
I32, F32, U8 = torch.int32, torch.float32, torch.uint8


def lopa_build_branches(tokens, conf, pred, L, mask_id, tau, k, branch_tokens, fill_pos, valid,
                        n_valid, stream=None):
    _check(lib.lopa_build_branches(_ptr(tokens, I32, "tokens"), _ptr(conf, F32, "conf"),
                                   _ptr(pred, I32, "pred"), L, mask_id, float(tau), k,
                                   _ptr(branch_tokens, I32, "branch_tokens"),
                                   _ptr(fill_pos, I32, "fill_pos"), _ptr(valid, U8, "valid"),
                                   _ptr(n_valid, I32, "n_valid"), _stream(stream)))


def lopa_build_branches_window(tokens, conf, pred, L, n_eligible, mask_id, tau, k, branch_tokens,
                               fill_pos, valid, n_valid, stream=None):
    _check(lib.lopa_build_branches_window(_ptr(tokens, I32, "tokens"), _ptr(conf, F32, "conf"),
                                          _ptr(pred, I32, "pred"), L, n_eligible, mask_id,
                                          float(tau), k, _ptr(branch_tokens, I32, "branch_tokens"),
                                          _ptr(fill_pos, I32, "fill_pos"), _ptr(valid, U8, "valid"),
                                          _ptr(n_valid, I32, "n_valid"), _stream(stream)))


def lopa_verify_forward(model: Model, kv: KV, prefix_len, branch_tokens, n_branches, L, conf, pred,
                        stream=None):
    _check(lib.lopa_verify_forward(model.handle, kv.handle, prefix_len,
                                   _ptr(branch_tokens, I32, "branch_tokens"), n_branches, L,
                                   _ptr(conf, F32, "conf"), _ptr(pred, I32, "pred"),
                                   _stream(stream)))


def lopa_prefill(model: Model, kv: KV, prefix_len, tokens, block, stream=None):
    _check(lib.lopa_prefill(model.handle, kv.handle, prefix_len, _ptr(tokens, I32, "tokens"),
                            tokens.numel(), block, _stream(stream)))


def lopa_verify_forward_noalloc(model: Model, kv: KV, prefix_len, branch_tokens, n_branches, L,
                                conf, pred, stream=None):
    _check(lib.lopa_verify_forward_noalloc(model.handle, kv.handle, prefix_len,
                                           _ptr(branch_tokens, I32, "branch_tokens"), n_branches,
                                           L, _ptr(conf, F32, "conf"), _ptr(pred, I32, "pred"),
                                           _stream(stream)))


def lopa_branch_confidence_select(branch_tokens, conf, pred, valid, n_branches, L, mask_id, scores,
                                  winner, next_tokens, next_conf, next_pred, next_unfilled,
                                  stream=None):
    _check(lib.lopa_branch_confidence_select(
        _ptr(branch_tokens, I32, "branch_tokens"), _ptr(conf, F32, "conf"), _ptr(pred, I32, "pred"),
        _ptr(valid, U8, "valid"), n_branches, L, mask_id, _ptr(scores, F32, "scores"),
        _ptr(winner, I32, "winner"), _ptr(next_tokens, I32, "next_tokens"),
        _ptr(next_conf, F32, "next_conf"), _ptr(next_pred, I32, "next_pred"),
        _ptr(next_unfilled, I32, "next_unfilled"), _stream(stream)))


def lopa_branch_confidence_select_metric(branch_tokens, conf, pred, valid, n_branches, L, mask_id,
                                         metric, window, eta, scores, winner, next_tokens,
                                         next_conf, next_pred, next_unfilled, stream=None):
    _check(lib.lopa_branch_confidence_select_metric(
        _ptr(branch_tokens, I32, "branch_tokens"), _ptr(conf, F32, "conf"), _ptr(pred, I32, "pred"),
        _ptr(valid, U8, "valid"), n_branches, L, mask_id, metric, window, eta,
        _ptr(scores, F32, "scores"), _ptr(winner, I32, "winner"),
        _ptr(next_tokens, I32, "next_tokens"), _ptr(next_conf, F32, "next_conf"),
        _ptr(next_pred, I32, "next_pred"), _ptr(next_unfilled, I32, "next_unfilled"),
        _stream(stream)))


def lopa_debug_hidden(model: Model, kv: KV, prefix_len, branch_tokens, n_branches, L, n_layers,
                      x_out, stream=None):
    _check(lib.lopa_debug_hidden(model.handle, kv.handle, prefix_len,
                                 _ptr(branch_tokens, I32, "branch_tokens"), n_branches, L, n_layers,
                                 _ptr(x_out, F32, "x_out"), _stream(stream)))


def lopa_commit_kv(kv: KV, winner, prefix_len, L, append_offset, stream=None):
    _check(lib.lopa_commit_kv(kv.handle, _ptr(winner, I32, "winner"), prefix_len, L,
                              _ptr(append_offset, I32, "append_offset"), _stream(stream)))


def lopa_commit_kv_rows(kv: KV, winner, prefix_len, L, n_rows, append_offset, stream=None):
    _check(lib.lopa_commit_kv_rows(kv.handle, _ptr(winner, I32, "winner"), prefix_len, L, n_rows,
                                   _ptr(append_offset, I32, "append_offset"), _stream(stream)))


# ---------------------------------------------------- multi-block window
WINDOW_WORDS = C.sizeof(lopa_window) // 4  # int32 words of the device window state


def window_state(device="cuda") -> torch.Tensor:
    """Device memory for one lopa_window (int32 words)."""
    return torch.zeros(WINDOW_WORDS, dtype=torch.int32, device=device)


def window_read(win: torch.Tensor) -> lopa_window:
    """The window state copied to the host (a synchronising read)."""
    host = win.cpu().numpy()
    return lopa_window.from_buffer_copy(host.tobytes())


def lopa_window_init(win, tokens, conf, pred, L, w_max, n_blocks, prefix_len, mask_id, tau_add,
                     tau_act, stream=None):
    _check(lib.lopa_window_init(_ptr(win, I32, "win"), _ptr(tokens, I32, "tokens"),
                                _ptr(conf, F32, "conf"), _ptr(pred, I32, "pred"), L, w_max,
                                n_blocks, prefix_len, mask_id, float(tau_add), float(tau_act),
                                _stream(stream)))


def lopa_window_update(win, tokens, conf, pred, out_tokens, stream=None):
    _check(lib.lopa_window_update(_ptr(win, I32, "win"), _ptr(tokens, I32, "tokens"),
                                  _ptr(conf, F32, "conf"), _ptr(pred, I32, "pred"),
                                  _ptr(out_tokens, I32, "out_tokens"), _stream(stream)))


def lopa_window_commit(kv: KV, winner, win, stream=None):
    _check(lib.lopa_window_commit(kv.handle, _ptr(winner, I32, "winner"), _ptr(win, I32, "win"),
                                  _stream(stream)))


# ------------------------------------------------------ serving: paged cache
_DTYPES = {torch.bfloat16: LOPA_BF16, torch.float16: LOPA_F16, torch.float32: LOPA_F32}


def _on(t, name):
    """The device (its index) of a call: that of its first tensor."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch tensor")
    if not t.is_cuda:
        raise ValueError(f"{name}: must be a device tensor")
    return t.get_device()


def _arg(t, dtype, dev, name, shape=None):
    """Address of a contiguous tensor on dev, None for None."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch tensor")
    if t.get_device() != dev:
        raise ValueError(f"{name}: must be a device tensor on cuda:{dev}")
    if dtype is not None and t.dtype is not dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name}: expected shape {shape}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    return t.data_ptr()


def _rows_arg(t, dtype, dev, name, shape):
    """Address and row stride of a [rows][heads][head_dim] tensor with contiguous heads."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch tensor")
    if t.get_device() != dev:
        raise ValueError(f"{name}: must be a device tensor on cuda:{dev}")
    if t.dtype is not dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name}: expected shape {shape}, got {tuple(t.shape)}")
    n, h, d = shape
    ld, sh, sd = t.stride()
    if n and (sd != 1 or (h > 1 and sh != d)):
        raise ValueError(f"{name}: the heads of a row must be contiguous")
    return t.data_ptr(), ld if n > 1 else h * d


def _call(f, dev, stream, *args):
    """f(*args, stream) on the device that holds the arrays, on its current stream or the given one."""
    if stream is None:
        st = torch._C._cuda_getCurrentRawStream(dev)  # current_stream(dev).cuda_stream without its object
    else:
        if hasattr(stream, "device") and stream.device.index != dev:
            raise ValueError(f"stream of {stream.device}, the tensors on cuda:{dev}")
        st = _stream(stream)
    if torch.cuda.current_device() == dev:
        status = f(*args, st)
    else:
        with torch.cuda.device(dev):
            status = f(*args, st)
    if status:
        _check(status)


def _paged(k_pages, v_pages, table, q_start, kv_len, rows, dev):
    dtype = k_pages.dtype
    if dtype is not torch.bfloat16 and dtype is not torch.float16:
        raise TypeError(f"k_pages: expected bfloat16 or float16, got {dtype}")
    if k_pages.dim() != 4:
        raise ValueError("k_pages: expected [pages][kv_heads][page_size][head_dim]")
    n, hkv, ps, d = k_pages.shape
    n_seq, ld = table.shape if table.dim() == 2 else (-1, 0)
    pages = lopa_pages(_arg(k_pages, dtype, dev, "k_pages"),
                       _arg(v_pages, dtype, dev, "v_pages", k_pages.shape), n, hkv, ps, d, _DTYPES[dtype])
    batch = lopa_paged_batch(_arg(table, I32, dev, "table", (n_seq, ld)),
                             _arg(q_start, I32, dev, "q_start", (n_seq + 1,)),
                             _arg(kv_len, I32, dev, "kv_len", (n_seq,)), n_seq, ld, rows)
    return pages, batch


def lopa_paged_append(k_pages, v_pages, table, q_start, kv_len, q, k, v, q_norm, k_norm, eps,
                      rope_theta, q_out, stream=None):
    """q [rows][heads][d], k and v [rows][kv_heads][d] (row strides are free, so views of a
    packed projection output do); q_norm / k_norm [d] or None; q_out like q."""
    dev = _on(k_pages, "k_pages")
    rows, heads, d = q.shape
    pages, batch = _paged(k_pages, v_pages, table, q_start, kv_len, rows, dev)
    t, hkv = k_pages.dtype, pages.kv_heads
    if d != pages.head_dim:
        raise ValueError(f"q: head_dim {d}, the pages' {pages.head_dim}")
    qp, ldq = _rows_arg(q, t, dev, "q", (rows, heads, d))
    kp, ldk = _rows_arg(k, t, dev, "k", (rows, hkv, d))
    vp, ldv = _rows_arg(v, t, dev, "v", (rows, hkv, d))
    op, ldo = _rows_arg(q_out, t, dev, "q_out", (rows, heads, d))
    _call(lib.lopa_paged_append, dev, stream, C.byref(pages), C.byref(batch), heads, qp, ldq, kp, ldk, vp,
          ldv, _arg(q_norm, t, dev, "q_norm", (d,)), _arg(k_norm, t, dev, "k_norm", (d,)), eps, rope_theta,
          op, ldo)


def lopa_paged_attention_workspace(heads, kv_heads, head_dim, n_seq, rows, max_rows, max_len) -> int:
    """Bytes of workspace that lopa_paged_attention needs for these sizes."""
    n = lib.lopa_paged_attention_workspace(heads, kv_heads, head_dim, n_seq, rows, max_rows, max_len)
    if n < 0:
        _check(n)
    return n


def lopa_paged_attention(q, k_pages, v_pages, table, q_start, kv_len, max_rows, max_len, block, scale,
                         softcap, out, lse=None, workspace=None, stream=None):
    """q and out [rows][heads][d] (free row strides); block 0 full, 1 causal, c block-causal;
    lse [rows][heads] fp32 or None; workspace: a contiguous tensor of the bytes that
    lopa_paged_attention_workspace gives, or None."""
    dev = _on(k_pages, "k_pages")
    rows, heads, d = q.shape
    pages, batch = _paged(k_pages, v_pages, table, q_start, kv_len, rows, dev)
    if d != pages.head_dim:
        raise ValueError(f"q: head_dim {d}, the pages' {pages.head_dim}")
    t = k_pages.dtype
    qp, ldq = _rows_arg(q, t, dev, "q", (rows, heads, d))
    op, ldo = _rows_arg(out, t, dev, "out", (rows, heads, d))
    _call(lib.lopa_paged_attention, dev, stream, C.byref(pages), C.byref(batch), heads, max_rows, max_len,
          qp, ldq, block, scale, softcap, op, ldo, _arg(lse, F32, dev, "lse", (rows, heads)),
          _arg(workspace, None, dev, "workspace"), workspace.nbytes if workspace is not None else 0)


def lopa_token_logprobs_workspace(rows, vocab, n_top) -> int:
    """Bytes of workspace that lopa_token_logprobs needs for these sizes."""
    n = lib.lopa_token_logprobs_workspace(rows, vocab, n_top)
    if n < 0:
        _check(n)
    return n


def lopa_token_logprobs(logits, tokens, exclude, logprob=None, entropy=None, top_ids=None,
                        top_logprobs=None, workspace=None, stream=None):
    """logits [rows][vocab] of bfloat16, float16 or float32 (free row stride); tokens [rows] with
    logprob [rows]; entropy [rows]; top_ids and top_logprobs [rows][n]; each output may be None.
    exclude: a token outside the support, or -1."""
    if getattr(top_ids, "shape", None) != getattr(top_logprobs, "shape", None):
        raise ValueError("top_ids and top_logprobs go together, of one shape: both or neither")
    dev = _on(logits, "logits")
    dtype = _DTYPES.get(logits.dtype)
    if dtype is None or logits.dim() != 2:
        raise TypeError("logits: expected [rows][vocab] of bfloat16, float16 or float32")
    rows, vocab = logits.shape
    ld, unit = logits.stride()
    if rows and vocab > 1 and unit != 1:
        raise ValueError("logits: a row must be contiguous")
    n = top_ids.shape[-1] if top_ids is not None else 0
    if n == 0:
        top_ids = top_logprobs = None
    _call(lib.lopa_token_logprobs, dev, stream, logits.data_ptr(), dtype, ld if rows > 1 else vocab, rows,
          vocab, exclude, _arg(tokens, I32, dev, "tokens", (rows,)), n,
          _arg(logprob, F32, dev, "logprob", (rows,)), _arg(entropy, F32, dev, "entropy", (rows,)),
          _arg(top_ids, I32, dev, "top_ids", (rows, n)), _arg(top_logprobs, F32, dev, "top_logprobs", (rows, n)),
          _arg(workspace, None, dev, "workspace"), workspace.nbytes if workspace is not None else 0)


from .decoder import Decoder, WindowDecoder  # noqa: E402,F401
