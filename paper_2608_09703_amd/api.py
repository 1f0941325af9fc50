"""PyTorch front end of the fused multi-sub-model LM head + CE + KL.

``distill(h_list, W_list, labels, ...)`` returns the per-sub-model
cross-entropies ``ce[M]``, the distillation values ``kl[M]`` (KL from the
teacher's softmax at temperature tau) and the mean teacher entropy, with
autograd support: the backward pass feeds the upstream gradients of ``ce``
and ``kl`` to the library as the coefficients of the objective, so any
objective linear in them (eq. (3) of the paper with its sum over
sub-models, or per-sub-model weights) differentiates correctly with no host
synchronisation.

``forward`` / ``backward`` are the same two library calls without autograd,
on caller-visible buffers (used by the tests and the benchmark).
"""

from __future__ import annotations

import contextlib
import ctypes
import functools
from typing import List, Optional, Sequence

import torch
from torch.autograd import forward_ad

from . import binding as B

# Descriptors are built once per set of values (bounded) and only ever read: a
# decoding loop makes the same few calls over and over, and filling the ctypes
# fields costs about as much as the launch.
_make_junction = functools.lru_cache(maxsize=256)(B.make_junction)
_make_sampling = functools.lru_cache(maxsize=256)(B.make_sampling)
_make_layer_norm = functools.lru_cache(maxsize=256)(B.make_layer_norm)
_layer_norm_workspace = functools.lru_cache(maxsize=256)(
    lambda *key: B.layer_norm_workspace(_make_layer_norm(*key)))


def _sampling(V, temperature, top_p, greedy) -> B.Sampling:
    # by value (a tensor hashes by identity), through the fields' own conversion:
    # what a descriptor refuses (a text, say) is refused
    return _make_sampling(V, ctypes.c_float(temperature).value, ctypes.c_float(top_p).value, bool(greedy))


def _dtype_code(dt: torch.dtype) -> int:
    if dt == torch.bfloat16:
        return B.MLS_BF16
    if dt == torch.float32:
        return B.MLS_F32
    raise TypeError(f"unsupported dtype {dt}; use bfloat16 or float32")


def make_problem(h: Sequence[torch.Tensor], W: Sequence[torch.Tensor], labels: torch.Tensor, *,
                 alpha: float = 0.0, tau: float = 1.0, teacher: int = -1,
                 ignore_index: int = -100, flags: int = 0, vocab_chunk: int = 0,
                 grad_h_dtype: torch.dtype = torch.float32) -> B.Problem:
    M = len(h)
    if M < 1 or len(W) != M:
        raise ValueError("need one head per sub-model")
    dev = h[0].device
    if dev.type != "cuda":
        raise RuntimeError("the fused loss runs on the GPU only; got tensors on " + str(dev))
    dt = h[0].dtype
    T = h[0].shape[0]
    V = W[0].shape[0]
    for i in range(M):
        for x in (h[i], W[i]):
            if x.device != dev or x.dtype != dt or x.dim() != 2 or not x.is_contiguous():
                raise ValueError("h_i / W_i must be contiguous 2-D tensors of one dtype on one device")
        if h[i].shape[0] != T or W[i].shape[0] != V or h[i].shape[1] != W[i].shape[1]:
            raise ValueError(f"shape mismatch in sub-model {i}")
    if labels.device != dev or labels.dtype != torch.int64 or labels.shape != (T,) \
            or not labels.is_contiguous():
        raise ValueError("labels must be a contiguous int64 [T] tensor on the same device")
    return B.make_problem(M, T, V, [x.shape[1] for x in h], [x.data_ptr() for x in h],
                          [x.data_ptr() for x in W], labels.data_ptr(), dtype=_dtype_code(dt),
                          teacher=teacher, ignore_index=ignore_index, alpha=alpha, tau=tau,
                          flags=flags, vocab_chunk=vocab_chunk,
                          grad_h_dtype=_dtype_code(grad_h_dtype))


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # not a public name


def _stream(dev) -> int:
    """Handle of the device's current stream (of a tensor's device without building a Stream object)."""
    if _raw_stream is not None and isinstance(dev, torch.device) and dev.index is not None:
        return _raw_stream(dev.index)
    return torch.cuda.current_stream(dev).cuda_stream


_HERE = contextlib.nullcontext()


def _on(dev: torch.device):
    """The device the tensors live on as the current one, for the launches inside."""
    return _HERE if dev.index == torch.cuda.current_device() else torch.cuda.device(dev)


def _primal(name: str, *xs: Optional[torch.Tensor]):
    """Refuses tensors that carry a tangent: addresses do not, so that the result would be
    without one, which later operations take for a derivative of zero."""
    # (outside of dual levels no tensor does: a tenth of the three questions' 1 us, which
    # the smallest calls would show; a torch without this number is asked them always)
    if getattr(forward_ad, "_current_level", 0) < 0:
        return
    for x in xs:
        if x is not None and forward_ad.unpack_dual(x).tangent is not None:
            raise NotImplementedError(f"{name}: forward-mode derivatives are not available")


def _once(name: str, g: Optional[torch.Tensor]):
    """Backward passes run with gradients enabled only where their own are asked for."""
    if torch.is_grad_enabled():
        raise RuntimeError(f"{name}: gradients of gradients are not available")
    _primal(name, g)


# Backward passes below run on the engine's thread, where every step costs about twice
# what it does on the caller's. The engine has made the forward's device and stream the
# current ones; what the forward has checked is not checked again, and the library is
# called without a wrapper in between.


class Buffers:
    """Caller-owned device buffers of one problem shape (workspace + statistics)."""

    def __init__(self, p: B.Problem, device):
        self.ws_bytes, self.stats_bytes = B.query_sizes(p)
        self.workspace = torch.empty(max(self.ws_bytes, 256), dtype=torch.uint8, device=device)
        self.stats = torch.empty(self.stats_bytes, dtype=torch.uint8, device=device)
        M = p.M
        self.ce = torch.empty(M, dtype=torch.float32, device=device)
        self.kl = torch.empty(M, dtype=torch.float32, device=device)
        self.entropy = torch.empty(1, dtype=torch.float32, device=device)

    def stats_view(self, M: int, T: int):
        """(lse1, lset, ce_row, kl_row, h_row) views into the statistics buffer."""
        f = self.stats[: (4 * M * T + T) * 4].view(torch.float32)
        return (f[: M * T].view(M, T), f[M * T: 2 * M * T].view(M, T),
                f[2 * M * T: 3 * M * T].view(M, T), f[3 * M * T: 4 * M * T].view(M, T),
                f[4 * M * T:])


def forward(p: B.Problem, buf: Buffers, device) -> None:
    B.distill_fwd(p, buf.stats.data_ptr(), buf.ce.data_ptr(), buf.kl.data_ptr(),
                  buf.entropy.data_ptr(), buf.workspace.data_ptr(), buf.workspace.numel(),
                  _stream(device))


def backward(p: B.Problem, buf: Buffers, device, g_ce: Optional[torch.Tensor],
             g_kl: Optional[torch.Tensor], grad_h: Sequence[Optional[torch.Tensor]],
             grad_W: Sequence[Optional[torch.Tensor]]) -> None:
    gh_dt = torch.bfloat16 if p.grad_h_dtype == B.MLS_BF16 else torch.float32
    for g in grad_h:
        if g is not None and (g.dtype != gh_dt or not g.is_contiguous()):
            raise ValueError(f"grad_h tensors are contiguous {gh_dt} tensors")
    gW_dt = torch.bfloat16 if p.flags & B.MLS_GRAD_W_BF16 else torch.float32
    for g in grad_W:
        if g is not None and (g.dtype != gW_dt or not g.is_contiguous()):
            raise ValueError(f"grad_W tensors are contiguous {gW_dt} tensors")
    gc = g_ce.data_ptr() if g_ce is not None else None
    gk = g_kl.data_ptr() if g_kl is not None else None
    B.distill_bwd(p, buf.stats.data_ptr(), gc, gk,
                  [g.data_ptr() if g is not None else None for g in grad_h],
                  [g.data_ptr() if g is not None else None for g in grad_W],
                  buf.workspace.data_ptr(), buf.workspace.numel(), _stream(device))


class _Distill(torch.autograd.Function):
    @staticmethod
    def forward(ctx, labels, opts, *hw):
        M = len(hw) // 2
        h, W = list(hw[:M]), list(hw[M:])
        # bf16 hidden states and heads get bf16 gradients straight from the library
        p = make_problem(h, W, labels, grad_h_dtype=h[0].dtype,
                         flags=B.MLS_GRAD_W_BF16 if h[0].dtype == torch.bfloat16 else 0, **opts)
        dev = h[0].device
        buf = Buffers(p, dev)
        forward(p, buf, dev)
        # the losses are the function's outputs; the context keeps the rest
        ce, kl, entropy = buf.ce, buf.kl, buf.entropy
        buf.ce = buf.kl = buf.entropy = None
        ctx.p = p
        ctx.buf = buf
        ctx.M = M
        ctx.save_for_backward(labels, *hw)
        ctx.mark_non_differentiable(entropy)
        return ce, kl, entropy

    @staticmethod
    def backward(ctx, g_ce, g_kl, g_ent):
        # saved-tensor hooks (offloading to the host, say) hand back other tensors
        # than forward() saw, which may be gone: the addresses are taken anew
        labels, *hw = (x.contiguous() for x in ctx.saved_tensors)
        M = ctx.M
        dev = hw[0].device
        p = B.Problem.from_buffer_copy(ctx.p)
        p.labels = labels.data_ptr()
        for i in range(M):
            p.h[i] = hw[i].data_ptr()
            p.W[i] = hw[M + i].data_ptr()
        if g_ce is None:
            g_ce = torch.zeros(M, dtype=torch.float32, device=dev)
        if g_kl is None:
            g_kl = torch.zeros(M, dtype=torch.float32, device=dev)
        g_ce = g_ce.to(torch.float32).contiguous()
        g_kl = g_kl.to(torch.float32).contiguous()
        need = ctx.needs_input_grad[2:]
        gh: List[Optional[torch.Tensor]] = []
        gW: List[Optional[torch.Tensor]] = []
        for i in range(M):  # of the inputs' dtype, as forward() set the problem up
            gh.append(torch.empty_like(hw[i]) if need[i] else None)
            gW.append(torch.empty_like(hw[M + i]) if need[M + i] else None)
        backward(p, ctx.buf, dev, g_ce, g_kl, gh, gW)
        return (None, None, *gh, *gW)


def distill(h_list: Sequence[torch.Tensor], W_list: Sequence[torch.Tensor], labels: torch.Tensor,
            *, tau: float = 1.0, teacher: int = -1, ignore_index: int = -100,
            vocab_chunk: int = 0):
    """Per-sub-model ``(ce[M], kl[M], entropy[1])`` with autograd through the HIP kernels."""
    opts = dict(tau=tau, teacher=teacher, ignore_index=ignore_index, vocab_chunk=vocab_chunk)
    return _Distill.apply(labels, opts, *h_list, *W_list)


def run_diagnostics(p: B.Problem, buf: Buffers, device, kl_pair: torch.Tensor, agree: torch.Tensor,
                    argmax: Optional[torch.Tensor]) -> None:
    """Pairwise diagnostics into caller tensors (one pass; ``buf.workspace`` is used)."""
    B.diagnostics(p, kl_pair.data_ptr(), agree.data_ptr(),
                  argmax.data_ptr() if argmax is not None else None, buf.workspace.data_ptr(),
                  buf.workspace.numel(), _stream(device))


@torch.no_grad()
def diagnostics(h_list: Sequence[torch.Tensor], W_list: Sequence[torch.Tensor],
                labels: torch.Tensor, *, ignore_index: int = -100, want_argmax: bool = False):
    """Cross-model ``(kl[M, M], agree[M, M], argmax[M, T] or None)`` of the sub-model heads.

    ``kl[i, j]`` is the mean over valid tokens of KL(p_i || p_j) at temperature 1 and
    ``agree[i, j]`` the fraction of valid tokens whose top-1 predictions coincide.
    One self-normalising pass over the logits of all sub-models.
    """
    p = make_problem(h_list, W_list, labels, ignore_index=ignore_index)
    dev = h_list[0].device
    buf = Buffers(p, dev)
    M, T = len(h_list), h_list[0].shape[0]
    kl = torch.empty(M, M, dtype=torch.float32, device=dev)
    agree = torch.empty(M, M, dtype=torch.float32, device=dev)
    am = torch.empty(M, T, dtype=torch.int32, device=dev) if want_argmax else None
    run_diagnostics(p, buf, dev, kl, agree, am)
    return kl, agree, am


_JUNCTION_LAYOUTS = {"prev_first": B.MLS_JUNCTION_PREV_FIRST, "fresh_first": B.MLS_JUNCTION_FRESH_FIRST}


def _junction_desc(o, e, grad_dtype, layout, flags=0):
    if not o.is_cuda or e.device != o.device:
        raise RuntimeError("the junction runs on the GPU only")
    if o.dim() != 2 or e.dim() != 2 or o.size(0) != e.size(0) or o.dtype != e.dtype:
        raise ValueError("o [T, d_prev] and e [T, d_fresh] must share T and dtype")
    if not (o.is_contiguous() and e.is_contiguous()):
        raise ValueError("o and e must be contiguous")
    return _make_junction(o.size(0), o.size(1), e.size(1), _dtype_code(o.dtype),
                          _dtype_code(grad_dtype), _JUNCTION_LAYOUTS[layout], flags)


def junction_forward(o: torch.Tensor, e: torch.Tensor, *, layout: str = "prev_first",
                     out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Eq. (1): ``x = [o * ||e|| / ||o|| | e]`` per token (no autograd)."""
    j = _junction_desc(o, e, o.dtype, layout)
    x = out if out is not None else o.new_empty((j.T, j.d_prev + j.d_fresh))
    B.junction_fwd(j, o.data_ptr(), e.data_ptr(), x.data_ptr(), _stream(o.device))
    return x


def junction_backward(o: torch.Tensor, e: torch.Tensor, g_x: torch.Tensor, *,
                      layout: str = "prev_first", g_o: Optional[torch.Tensor] = None,
                      g_e: Optional[torch.Tensor] = None, accumulate: bool = False):
    """``(g_o, g_e)`` of the junction for the upstream gradient ``g_x`` (dtype of ``g_x``)."""
    if not g_x.is_contiguous() or g_x.shape != (o.shape[0], o.shape[1] + e.shape[1]):
        raise ValueError("g_x must be a contiguous [T, d_prev + d_fresh] tensor")
    j = _junction_desc(o, e, g_x.dtype, layout, B.MLS_JUNCTION_ACCUMULATE if accumulate else 0)
    if g_o is None:
        g_o = g_x.new_empty(o.shape, device=o.device)
    if g_e is None:
        g_e = g_x.new_empty(e.shape, device=o.device)
    for g in (g_o, g_e):
        if g.dtype != g_x.dtype or not g.is_contiguous():
            raise ValueError("g_o / g_e must be contiguous and of g_x's dtype")
    B.junction_bwd(j, o.data_ptr(), e.data_ptr(), g_x.data_ptr(), g_o.data_ptr(), g_e.data_ptr(),
                   _stream(o.device))
    return g_o, g_e


class _Junction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, o, e, layout):
        ctx.save_for_backward(o, e)
        ctx.layout = layout
        return junction_forward(o, e, layout=layout)

    @staticmethod
    def backward(ctx, g_x):
        o, e = ctx.saved_tensors
        g_o, g_e = junction_backward(o, e, g_x.contiguous(), layout=ctx.layout)
        return g_o.to(o.dtype), g_e.to(e.dtype), None


def junction(o: torch.Tensor, e: torch.Tensor, *, layout: str = "prev_first") -> torch.Tensor:
    """Inter-model junction of eq. (1) with autograd through the HIP kernels."""
    return _Junction.apply(o, e, layout)


# ---------------------------------------------------------------------------
# post-training: the norm in front of a head, token log-probabilities, the policy
# loss on them and the clipping of the gradients
# ---------------------------------------------------------------------------

def _norm_rows(x: torch.Tensor):
    """``x [..., d]`` as rows: (2-D view, elements between rows)."""
    if x.dim() < 1 or x.numel() == 0 or (x.size(-1) > 1 and x.stride(-1) != 1):
        raise ValueError("x must be a non-empty [..., d] tensor with neighbouring elements in a row")
    rows = x
    if x.dim() != 2:
        try:
            rows = x.view(-1, x.size(-1))
        except RuntimeError as e:
            raise ValueError("the rows of x must lie at one distance from each other") from e
    ld = rows.stride(0) if rows.size(0) > 1 else rows.size(1)
    if ld < rows.size(1):
        raise ValueError("the rows of x must not overlap (an expanded x: call .contiguous())")
    return rows, ld


def _norm_desc(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor], eps: float):
    if not x.is_cuda or weight.device != x.device or (bias is not None and bias.device != x.device):
        raise RuntimeError("layer_norm runs on the GPU only, on tensors of one device")
    rows, ld = _norm_rows(x)
    d = rows.size(1)
    for p in (weight, bias):
        if p is not None and (p.shape != (d,) or not p.is_contiguous() or p.dtype != weight.dtype):
            raise ValueError("weight and bias must be contiguous [d] tensors of one dtype")
    return rows, (rows.size(0), d, ld, _dtype_code(x.dtype), _dtype_code(weight.dtype),
                  ctypes.c_float(eps).value)


def layer_norm_forward(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, *,
                       eps: float = 1e-5, want_stats: bool = False):
    """``y`` of :func:`layer_norm` (no autograd), and with ``want_stats`` the float32
    ``[2, rows]`` means and inverse deviations that :func:`layer_norm_backward` reads."""
    rows, key = _norm_desc(x, weight, bias, eps)
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    stats = torch.empty(2, key[0], dtype=torch.float32, device=x.device) if want_stats else None
    with _on(x.device):
        B.layer_norm_fwd(_make_layer_norm(*key), rows.data_ptr(), weight.data_ptr(),
                         bias.data_ptr() if bias is not None else None, y.data_ptr(),
                         stats.data_ptr() if want_stats else None, _stream(x.device))
    return (y, stats) if want_stats else y


def layer_norm_backward(x: torch.Tensor, weight: torch.Tensor, stats: torch.Tensor, g_y: torch.Tensor, *,
                        eps: float = 1e-5, want_x: bool = True, want_weight: bool = True,
                        want_bias: bool = False):
    """``(g_x, g_weight, g_bias)`` for the gradient ``g_y`` of ``y`` (None where not wanted)."""
    rows, key = _norm_desc(x, weight, None, eps)
    if g_y.shape != x.shape or g_y.dtype != x.dtype or g_y.device != x.device or not g_y.is_contiguous():
        raise ValueError("g_y must be a contiguous tensor of x's shape, dtype and device")
    if stats.shape != (2, key[0]) or stats.dtype != torch.float32 or stats.device != x.device \
            or not stats.is_contiguous():
        raise ValueError("stats must be the forward's [2, rows] float32 tensor")
    n = _make_layer_norm(*key)
    g_x = torch.empty(x.shape, dtype=x.dtype, device=x.device) if want_x else None
    g_w = torch.empty_like(weight) if want_weight else None
    g_b = torch.empty_like(weight) if want_bias else None
    ws_bytes = _layer_norm_workspace(*key) if want_weight or want_bias else 0
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device=x.device) if ws_bytes else None
    ptr = (lambda t: t.data_ptr() if t is not None else None)
    with _on(x.device):
        B.layer_norm_bwd(n, rows.data_ptr(), weight.data_ptr(), stats.data_ptr(), g_y.data_ptr(), ptr(g_x),
                         ptr(g_w), ptr(g_b), ptr(ws), ws_bytes, _stream(x.device))
    return g_x, g_w, g_b


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        rows, key = _norm_desc(x, weight, bias, eps)
        dev = x.device
        y = torch.empty(x.shape, dtype=x.dtype, device=dev)
        stats = torch.empty(2, key[0], dtype=torch.float32, device=dev)
        n = _make_layer_norm(*key)
        with _on(dev):
            B.layer_norm_fwd(n, rows.data_ptr(), weight.data_ptr(), bias.data_ptr() if bias is not None else None,
                             y.data_ptr(), stats.data_ptr(), _stream(dev))
        ctx.save_for_backward(x, weight, stats)
        ctx.n, ctx.ws_bytes = n, _layer_norm_workspace(*key)
        return y

    @staticmethod
    def backward(ctx, g_y):
        _once("layer_norm", g_y)
        x, weight, stats = ctx.saved_tensors
        if not g_y.is_contiguous():
            g_y = g_y.contiguous()
        dev, n = g_y.device, ctx.n
        # (behind saved-tensor hooks the layout of x may be another)
        if x.dim() != 2 or x.stride() != (n.ld_x, 1):
            x, ld = _norm_rows(x)
            if ld != n.ld_x:
                n = B.make_layer_norm(n.T, n.d, ld, n.act_dtype, n.param_dtype, n.eps)
        need_x, need_w, need_b, _ = ctx.needs_input_grad
        g_x = torch.empty_like(g_y) if need_x else None
        g_w = torch.empty_like(weight) if need_w else None
        g_b = torch.empty_like(weight) if need_b else None
        ws = torch.empty(ctx.ws_bytes, dtype=torch.uint8, device=dev) if need_w or need_b else None
        st = B.lib().mls_layer_norm_bwd(
            n, x.data_ptr(), weight.data_ptr(), stats.data_ptr(), g_y.data_ptr(),
            g_x.data_ptr() if need_x else None, g_w.data_ptr() if need_w else None,
            g_b.data_ptr() if need_b else None, ws.data_ptr() if ws is not None else None, ctx.ws_bytes, _stream(dev))
        if st:
            B.check(st, "mls_layer_norm_bwd")
        return g_x, g_w, g_b, None


def layer_norm(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, *,
               eps: float = 1e-5) -> torch.Tensor:
    """Layer norm over the last dimension of ``x [..., d]`` with autograd through the HIP kernels.

    ``x`` is bf16 or float32; its rows may be columns of a wider tensor (a nested
    sub-model's channels). ``weight`` and ``bias [d]`` are bf16 or float32, whatever
    ``x`` is; their gradients are summed in float32 and rounded once.
    """
    _primal("layer_norm", x, weight, bias)
    if torch.is_grad_enabled() and (x.requires_grad or weight.requires_grad or
                                    (bias is not None and bias.requires_grad)):
        return _LayerNorm.apply(x, weight, bias, eps)
    return layer_norm_forward(x, weight, bias, eps=eps)


# Logits that token_logp keeps for its backward by itself: at most this many bytes
# (of 288 GB); beyond, the backward computes them again. T = 4,096, d = 4,352,
# V = 49,152: 0.4 GiB, and both passes take 3,580 us in place of 4,595.
KEEP_LOGITS_BYTES = 2 << 30


def _token_logp_forward(h, W, tokens, opts, keep_logits):
    dev = h.device
    p = make_problem([h], [W], tokens, grad_h_dtype=h.dtype,
                     flags=B.MLS_GRAD_W_BF16 if h.dtype == torch.bfloat16 else 0, **opts)
    ws_bytes, bwd_bytes, kept_bytes = B.token_logp_workspace(p)
    if keep_logits is None:
        keep_logits = kept_bytes <= KEEP_LOGITS_BYTES
    kept = torch.empty(kept_bytes, dtype=torch.uint8, device=dev) if keep_logits and kept_bytes else None
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
    stats = torch.empty(B.query_sizes(p)[1], dtype=torch.uint8, device=dev)
    logp = torch.empty(p.T, dtype=torch.float32, device=dev)
    entropy = torch.empty(p.T, dtype=torch.float32, device=dev)
    with _on(dev):
        B.token_logp_fwd(p, stats.data_ptr(), logp.data_ptr(), entropy.data_ptr(),
                         kept.data_ptr() if kept is not None else None, ws.data_ptr(), ws_bytes, _stream(dev))
    return logp, entropy, p, stats, kept, bwd_bytes


class _TokenLogp(torch.autograd.Function):
    @staticmethod
    def forward(ctx, tokens, opts, keep_logits, h, W):
        logp, entropy, ctx.p, ctx.stats, kept, ctx.ws_bytes = _token_logp_forward(h, W, tokens, opts, keep_logits)
        ctx.save_for_backward(tokens, h, W, kept)  # (freed by the backward)
        ctx.mark_non_differentiable(entropy)
        ctx.set_materialize_grads(False)  # no zeros for the entropy
        return logp, entropy

    @staticmethod
    def backward(ctx, g_logp, g_entropy):
        _once("token_logp", g_logp)
        if g_logp is None:
            return None, None, None, None, None
        # the saved tensors' addresses are taken anew, as in the loss's backward
        tokens, h, W, kept = ctx.saved_tensors
        if not (tokens.is_contiguous() and h.is_contiguous() and W.is_contiguous()):
            tokens, h, W = tokens.contiguous(), h.contiguous(), W.contiguous()
        g_logp = g_logp.contiguous()
        p = ctx.p
        if (p.labels, p.h[0], p.W[0]) != (tokens.data_ptr(), h.data_ptr(), W.data_ptr()):
            p = B.Problem.from_buffer_copy(p)
            p.labels, p.h[0], p.W[0] = tokens.data_ptr(), h.data_ptr(), W.data_ptr()
        _, _, _, need_h, need_W = ctx.needs_input_grad
        gh = torch.empty_like(h) if need_h else None
        gW = torch.empty_like(W) if need_W else None
        ws = torch.empty(ctx.ws_bytes, dtype=torch.uint8, device=h.device)
        st = B.lib().mls_token_logp_bwd(p, ctx.stats.data_ptr(), kept.data_ptr() if kept is not None else None,
                                        g_logp.data_ptr(), gh.data_ptr() if need_h else None,
                                        gW.data_ptr() if need_W else None, ws.data_ptr(), ctx.ws_bytes,
                                        _stream(h.device))
        if st:
            B.check(st, "mls_token_logp_bwd")
        return None, None, None, gh, gW


def token_logp(h: torch.Tensor, W: torch.Tensor, tokens: torch.Tensor, *, temperature: float = 1.0,
               ignore_index: int = -100, vocab_chunk: int = 0, keep_logits: Optional[bool] = None):
    """``(logp [T], entropy [T])`` (float32) of ``tokens [T]`` under the head ``W [V, d]`` on ``h [T, d]``.

    ``logp[t] = log softmax(W h[t] / temperature)[tokens[t]]``, with autograd through
    the HIP kernels for any gradient per token; ``entropy`` (of the same softmax) is
    for monitoring and not differentiated. Both are 0 where the token is
    ``ignore_index``. Ignored tokens cost no product, and what their rows of ``h`` hold
    does not matter.

    bf16 gradients are sums of bf16 products: each softmax entry over 1 - p (the token's
    own one is exact), for ``W`` each entry of ``h`` times its token's factor, and the
    results are rounded to bf16 once (the whole of it is 0.0022 of a gradient's norm in
    large batches, of which the results' own rounding is 0.0017). float32 has none of these.

    ``keep_logits``: whether the backward finds the logits kept (16 bits each, which is up
    to 2^-12 of a softmax entry; ``2 T V`` bytes until it is done; bf16 inputs only) or
    computes them again; by itself, kept up to ``KEEP_LOGITS_BYTES``. It forms the logit gradients a chunk of the vocabulary at a
    time (``vocab_chunk`` columns, or as many as fit 256 MiB).
    """
    opts = dict(tau=temperature, ignore_index=ignore_index, vocab_chunk=vocab_chunk)
    _primal("token_logp", h, W)
    if torch.is_grad_enabled() and (h.requires_grad or W.requires_grad):
        return _TokenLogp.apply(tokens, opts, keep_logits, h, W)
    return _token_logp_forward(h, W, tokens, opts, False)[:2]


_POLICY_REDUCTIONS = {"token": 0, "sequence": B.MLS_POLICY_MEAN_OF_SEQUENCES}


def _policy_forward(logp, args, want_grad):
    old, adv, ref, mask, cu, desc = args
    dev = logp.device
    loss, kl, clipped = (torch.empty((), dtype=torch.float32, device=dev) for _ in range(3))
    grad = torch.empty(desc.N + 1, dtype=torch.float32, device=dev) if want_grad else None
    ws_bytes = B.policy_loss_workspace(desc)
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
    with _on(dev):
        B.policy_loss_fwd(desc, logp.data_ptr(), old.data_ptr(), adv.data_ptr(),
                          ref.data_ptr() if ref is not None else None,
                          mask.data_ptr() if mask is not None else None,
                          cu.data_ptr() if cu is not None else None, loss.data_ptr(), kl.data_ptr(),
                          clipped.data_ptr(), grad.data_ptr() if want_grad else None, ws.data_ptr(), ws_bytes,
                          _stream(dev))
    return loss, kl, clipped, grad


class _PolicyLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logp, args):
        loss, kl, clipped, grad = _policy_forward(logp, args, True)
        ctx.save_for_backward(grad)
        ctx.shape = logp.shape
        ctx.mark_non_differentiable(kl, clipped)
        ctx.set_materialize_grads(False)  # no zeros for the other two
        return loss, kl, clipped

    @staticmethod
    def backward(ctx, g_loss, g_kl, g_clipped):
        _once("policy_loss", g_loss)
        if g_loss is None:
            return None, None
        grad, = ctx.saved_tensors
        dev = grad.device
        g_logp = torch.empty(ctx.shape, dtype=torch.float32, device=dev)
        st = B.lib().mls_policy_loss_bwd(grad.numel() - 1, grad.data_ptr(), g_loss.data_ptr(), g_logp.data_ptr(),
                                         _stream(dev))
        if st:
            B.check(st, "mls_policy_loss_bwd")
        return g_logp, None


def policy_loss(logp: torch.Tensor, old_logp: torch.Tensor, advantages: torch.Tensor, *,
                ref_logp: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
                cu_seqlens: Optional[torch.Tensor] = None, per_sequence: bool = False, clip_low: float = 0.2,
                clip_high: float = 0.2, kl_coef: float = 0.0, reduction: str = "token"):
    """``(loss, kl, clipped)``: the clipped policy loss on token log-probabilities.

    Per token with advantage ``A`` and ``r = exp(logp - old_logp)`` the loss is
    ``-min(r A, clip(r, 1 - clip_low, 1 + clip_high) A) + kl_coef k`` with
    ``k = exp(ref_logp - logp) - (ref_logp - logp) - 1``. ``reduction="token"`` takes
    the mean over the tokens that count, ``"sequence"`` the mean over the sequences of
    their tokens' means. ``kl`` is the same mean of ``k`` (0 without ``ref_logp``) and
    ``clipped`` the share of clipped tokens. Only ``logp`` is differentiated, and only
    in ``loss``.

    ``logp``, ``old_logp``, ``ref_logp`` (float32) and ``mask`` (bool: the tokens that
    count) are of one shape, ``[N]`` packed or ``[B, L]`` padded. Packed sequences are
    ``cu_seqlens`` (int32 ``[S + 1]``, ascending; tokens outside of them do not count);
    the rows of ``[B, L]`` are sequences by themselves. ``advantages`` is per token, or
    with ``per_sequence`` one per sequence ``[S]``.
    """
    if not logp.is_cuda:
        raise RuntimeError("policy_loss runs on the GPU only; got tensors on " + str(logp.device))
    if reduction not in _POLICY_REDUCTIONS:
        raise ValueError(f"reduction must be one of {sorted(_POLICY_REDUCTIONS)}, got {reduction!r}")
    dev, shape, N = logp.device, logp.shape, logp.numel()
    for name, x in (("logp", logp), ("old_logp", old_logp), ("ref_logp", ref_logp)):
        if x is not None and (x.dtype != torch.float32 or x.shape != shape or x.device != dev or
                              not x.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous float32 tensor of logp's shape and device")
    if mask is not None and (mask.dtype != torch.bool or mask.shape != logp.shape or mask.device != dev or
                             not mask.is_contiguous()):
        raise ValueError("mask must be a contiguous bool tensor of logp's shape and device")
    flags = _POLICY_REDUCTIONS[reduction] | (B.MLS_POLICY_ADV_PER_SEQUENCE if per_sequence else 0)
    if cu_seqlens is not None:
        if logp.dim() != 1:
            raise ValueError("cu_seqlens goes with packed [N] tokens")
        if cu_seqlens.dtype != torch.int32 or cu_seqlens.dim() != 1 or cu_seqlens.numel() < 2 or \
                cu_seqlens.device != dev or not cu_seqlens.is_contiguous():
            raise ValueError("cu_seqlens must be a contiguous int32 [S + 1] tensor on logp's device")
    elif flags:
        if logp.dim() != 2 or N == 0:
            raise ValueError("sequences are cu_seqlens or the rows of a [B, L] logp")
        cu_seqlens = torch.arange(0, N + 1, logp.size(1), dtype=torch.int32, device=dev)
    S = cu_seqlens.numel() - 1 if cu_seqlens is not None else 0
    if advantages.dtype != torch.float32 or advantages.device != dev or not advantages.is_contiguous() or \
            advantages.shape != ((S,) if per_sequence else logp.shape):
        raise ValueError("advantages must be a contiguous float32 tensor of " +
                         ("[S]" if per_sequence else "logp's shape"))
    desc = B.make_policy(N, S, clip_low, clip_high, kl_coef, flags)
    args = (old_logp, advantages, ref_logp, mask, cu_seqlens, desc)
    _primal("policy_loss", logp)
    if torch.is_grad_enabled() and logp.requires_grad:
        return _PolicyLoss.apply(logp, args)
    return _policy_forward(logp, args, False)[:3]


_GRAD_CODES = {torch.bfloat16: B.MLS_BF16, torch.float32: B.MLS_F32}


def _clip(grads, max_norm: float, out) -> torch.Tensor:
    # (one pass over the list for each property: hundreds of tensors, whose properties
    # cost more than the launches when asked for one by one)
    T = torch.Tensor
    entries = list(grads)
    grads = [g for g in entries if g is not None]
    if out is not None:
        out = list(out)
        if len(out) != len(entries):
            raise ValueError("out must hold one entry for each entry of grads")
        if len(grads) != len(entries):
            out = [o for g, o in zip(entries, out) if g is not None]
    if not grads:
        raise ValueError("no gradients given: the norm would be on no device")
    dev = grads[0].device
    if dev.type != "cuda":
        raise RuntimeError("gradient norms run on the GPU only; got tensors on " + str(dev))
    on = {grads[0].get_device()}
    if {*map(T.get_device, grads)} != on or not all(map(T.is_contiguous, grads)):
        raise ValueError("gradients must be contiguous tensors on one device")
    dtypes = [g.dtype for g in grads]
    codes = [*map(_GRAD_CODES.get, dtypes)]
    if None in codes:
        raise TypeError(f"unsupported dtype {dtypes[codes.index(None)]}; use bfloat16 or float32")
    sizes, data = [*map(T.numel, grads)], [*map(T.data_ptr, grads)]
    to = data
    if out is not None:
        if type(None) in map(type, out) or [*map(T.numel, out)] != sizes or [o.dtype for o in out] != dtypes or \
                {*map(T.get_device, out)} != on or not all(map(T.is_contiguous, out)):
            raise ValueError("out must hold for each gradient one contiguous tensor of its size, dtype and device")
        to = [*map(T.data_ptr, out)]
    tensors = B.make_grad_tensors(data, to, sizes, codes)
    norm = torch.empty((), dtype=torch.float32, device=dev)
    ws_bytes = B.clip_grad_norm_workspace(len(data), tensors)
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
    with _on(dev):
        B.clip_grad_norm(len(data), tensors, max_norm, norm.data_ptr(), ws.data_ptr(), ws_bytes, _stream(dev))
    if max_norm:  # written through addresses: graphs that saved these tensors are told
        torch.autograd.graph.increment_version(grads if out is None else out)
    return norm


@torch.no_grad()
def grad_norm(grads: Sequence[Optional[torch.Tensor]]) -> torch.Tensor:
    """The global L2 norm (float32, on the device, not differentiated) of a list of bf16 or
    float32 gradients; entries that are None are left out."""
    return _clip(grads, 0.0, None)


@torch.no_grad()
def clip_grad_norm(grads: Sequence[Optional[torch.Tensor]], max_norm: float, *,
                   out: Optional[Sequence[Optional[torch.Tensor]]] = None) -> torch.Tensor:
    """Scales gradients by ``min(1, max_norm / norm)`` and returns their global L2 norm before.

    The norm is a float32 scalar on the device: nothing waits for it. The gradients
    (bf16 and float32 mixed) are scaled in place, or into the tensors ``out`` of the
    same sizes and dtypes. Entries that are None are left out, and with them their
    entries of ``out``; one gradient there has to be. A norm that is NaN or infinite
    scales nothing.
    """
    if not max_norm > 0:
        raise ValueError(f"max_norm must be > 0, got {max_norm}")
    return _clip(grads, max_norm, out)


def head_logits(o: torch.Tensor, W: torch.Tensor, out: Optional[torch.Tensor] = None):
    """``logits [T, V] = o W^T`` in fp32 through the HIP head kernel (decode regime)."""
    if not o.is_cuda or W.device != o.device or o.dtype != W.dtype:
        raise RuntimeError("o and W must be GPU tensors of one dtype")
    if not (o.is_contiguous() and W.is_contiguous()) or o.shape[1] != W.shape[1]:
        raise ValueError("o [T, d] and W [V, d] must be contiguous with a shared d")
    T, V = o.shape[0], W.shape[0]
    out = out if out is not None else torch.empty(T, V, dtype=torch.float32, device=o.device)
    B.head_logits(T, V, o.shape[1], _dtype_code(o.dtype), o.data_ptr(), W.data_ptr(),
                  out.data_ptr(), _stream(o.device))
    return out


def sample(logits: torch.Tensor, u: Optional[torch.Tensor], *, temperature: float = 1.0,
           top_p: float = 1.0, greedy: bool = False,
           params: Optional[torch.Tensor] = None) -> torch.Tensor:
    """int32 tokens, one per row of ``logits [rows, V]`` (fp32), with uniforms ``u [rows]``.

    ``params``: optional uint8 tensor of ``rows * ROW_PARAMS_BYTES`` bytes that
    receives the rows' distribution records (for ``spec_verify(draft_params=)``).
    """
    if logits.dtype != torch.float32 or not logits.is_contiguous() or logits.dim() != 2:
        raise ValueError("logits must be a contiguous float32 [rows, V] tensor")
    rows, V = logits.shape
    if u is not None and (u.dtype != torch.float32 or u.shape != (rows,) or not u.is_contiguous()):
        raise ValueError("u must be a contiguous float32 [rows] tensor")
    if params is not None and (params.dtype != torch.uint8 or not params.is_contiguous() or
                               params.numel() < rows * B.ROW_PARAMS_BYTES):
        raise ValueError("params must be a contiguous uint8 tensor of rows * ROW_PARAMS_BYTES")
    tok = torch.empty(rows, dtype=torch.int32, device=logits.device)
    B.sample(_sampling(V, temperature, top_p, greedy), rows, logits.data_ptr(),
             u.data_ptr() if u is not None else None, tok.data_ptr(), _stream(logits.device),
             params.data_ptr() if params is not None else None)
    return tok


def spec_verify(draft_logits: Optional[torch.Tensor], target_logits: torch.Tensor,
                draft_tokens: Optional[torch.Tensor], u_accept: Optional[torch.Tensor],
                u_sample: Optional[torch.Tensor], *, temperature: float = 1.0, top_p: float = 1.0,
                greedy: bool = False, draft_params: Optional[torch.Tensor] = None):
    """``(n_accepted [B], next_token [B])`` (int32) of speculative verification.

    Draft-side arrays in drafting order: ``draft_logits [gamma, B, V]`` (fp32),
    ``draft_tokens [gamma, B]`` (int32), ``u_accept [gamma, B]``; verifier side
    ``target_logits [B, gamma + 1, V]`` (fp32) and ``u_sample [B]``.
    ``draft_params``: optional uint8 records ``[gamma, B]`` from ``sample(params=)``
    on the draft rows with the same settings (then not recomputed).
    """
    Bt, G1, V = target_logits.shape
    G = G1 - 1
    dev = target_logits.device
    for x in (draft_logits, target_logits, u_accept, u_sample):
        if x is not None and (x.dtype != torch.float32 or not x.is_contiguous()):
            raise ValueError("logits and uniforms must be contiguous float32")
    if draft_tokens is not None and (draft_tokens.dtype != torch.int32 or
                                     not draft_tokens.is_contiguous()):
        raise ValueError("draft_tokens must be contiguous int32")
    if G > 0 and (draft_logits is None or draft_logits.shape != (G, Bt, V) or
                  draft_tokens is None or draft_tokens.shape != (G, Bt)):
        raise ValueError("draft_logits [gamma, B, V] and draft_tokens [gamma, B] are required")
    if G > 0 and not greedy and (u_accept is None or u_accept.shape != (G, Bt)):
        raise ValueError("u_accept [gamma, B] is required")
    n_acc = torch.empty(Bt, dtype=torch.int32, device=dev)
    nxt = torch.empty(Bt, dtype=torch.int32, device=dev)
    ws_bytes = 0 if greedy else B.spec_verify_workspace(Bt, G)
    ws = torch.empty(max(ws_bytes, 256), dtype=torch.uint8, device=dev) if not greedy else None
    ptr = (lambda x: x.data_ptr() if x is not None else None)
    if draft_params is not None and (draft_params.dtype != torch.uint8 or
                                     not draft_params.is_contiguous() or
                                     draft_params.numel() < G * Bt * B.ROW_PARAMS_BYTES):
        raise ValueError("draft_params must be contiguous uint8 of gamma * B records")
    B.spec_verify(_sampling(V, temperature, top_p, greedy), Bt, G, ptr(draft_logits),
                  target_logits.data_ptr(), ptr(draft_tokens), ptr(u_accept), ptr(u_sample),
                  n_acc.data_ptr(), nxt.data_ptr(), ptr(ws), ws_bytes, _stream(dev),
                  draft_params=ptr(draft_params))
    return n_acc, nxt


# ---------------------------------------------------------------------------
# decoding with a tree of drafted tokens: cache entries, attention, verification, and
# the head in 8-bit integers
# ---------------------------------------------------------------------------

def _no_grad(name: str, *xs: Optional[torch.Tensor]):
    """Refuses tensors that a gradient is wanted for: the result would be without one."""
    if torch.is_grad_enabled():
        for x in xs:
            if x is not None and x.requires_grad:
                raise RuntimeError(f"{name}: gradients are not available; call it under torch.no_grad()")
    _primal(name, *xs)


def _written(*xs: torch.Tensor):
    """Tells autograd of tensors that were written through their addresses."""
    xs = [x for x in xs if not x.is_inference()]
    if xs:
        torch.autograd.graph.increment_version(xs)


# What a call checks and works out from the tensors' types, shapes and strides alone is
# kept per set of these (bounded, as the descriptors above): 8 of a call's 18 us.

def _meta(x: Optional[torch.Tensor]):
    return None if x is None else (x.dtype, x.get_device(), x.shape, x.stride())


def _kv_cache(name: str, k_pages, v_pages, page_table, lengths, all_layers: bool = False) -> B.KVCache:
    """The descriptor without addresses; the tensors as their :func:`_meta`."""
    dtype, dev, shape, stride = k_pages
    if dev < 0:
        raise RuntimeError(f"{name} runs on the GPU only")
    dims = len(shape)
    if v_pages != k_pages or not (dims == 4 or (all_layers and dims == 5)):
        raise ValueError(f"{name}: k_pages and v_pages are [pages, kv_heads, page_size, head_dim] tensors" +
                         (", or such of several layers," if all_layers else "") + " of one layout, dtype and device")
    if dims == 4:
        layers, ld_layer = 1, 0
    else:
        layers, ld_layer, shape, stride = shape[0], stride[0], shape[1:], stride[1:]
    if stride[3] != 1 and shape[3] > 1:
        raise ValueError(f"{name}: the elements of an entry must be neighbours")
    t_dtype, t_dev, t_shape, t_stride = page_table
    if t_dtype != torch.int32 or len(t_shape) != 2 or t_dev != dev or (t_shape[1] > 1 and t_stride[1] != 1):
        raise ValueError(f"{name}: page_table must be an int32 [B, pages of a sequence] tensor on the pages' device")
    Bt, width = t_shape
    _ints(name, "lengths", lengths, (Bt,), dev)
    far = [s if n > 1 else 0 for n, s in zip((layers,) + tuple(shape), (ld_layer,) + tuple(stride))]
    return B.KVCache(_dtype_code(dtype), shape[2], shape[1], shape[3], layers, shape[0], Bt, width, *far[:4],
                     t_stride[0] if Bt > 1 else width)


def _step_rows(name: str, x, what: str, c: B.KVCache, like, heads: Optional[int] = None):
    """Checks ``x [B, n, heads, head_dim]`` and returns its strides."""
    dtype, dev, shape, stride = x
    if dev != like[1] or dtype != like[0] or len(shape) != 4 or shape[0] != c.batch or shape[3] != c.head_dim or \
            shape[1] == 0 or (heads is not None and shape[2] != heads) or (stride[3] != 1 and shape[3] > 1):
        raise ValueError(f"{name}: {what} must be a [B, n, heads, head_dim] tensor of the pages' dtype and device")
    return tuple(stride[i] if shape[i] > 1 else 0 for i in range(3))


def _ints(name: str, what: str, x, shape, dev):
    if x is not None and (x[0] != torch.int32 or x[2] != shape or x[1] != dev or not _packed(x[2], x[3])):
        raise ValueError(f"{name}: {what} must be a contiguous int32 {list(shape)} tensor on the same device")


def _packed(shape, stride) -> bool:
    want = 1
    for n, s in zip(reversed(shape), reversed(stride)):
        if n != 1 and s != want:
            return False
        want *= n
    return True


def _with_addresses(c: B.KVCache, k_pages, v_pages, page_table, lengths) -> B.KVCache:
    c = B.KVCache.from_buffer_copy(c)
    c.k, c.v, c.page_table, c.lengths = k_pages.data_ptr(), v_pages.data_ptr(), page_table.data_ptr(), lengths.data_ptr()
    return c


@functools.lru_cache(maxsize=256)
def _write_plan(k, v, k_pages, v_pages, page_table, lengths, counts):
    c = _kv_cache("cache_write", k_pages, v_pages, page_table, lengths)
    ld = _step_rows("cache_write", k, "k", c, k_pages, c.kv_heads)
    if v[2] != k[2]:
        raise ValueError("cache_write: k and v must be of one shape")
    same = _step_rows("cache_write", v, "v", c, k_pages, c.kv_heads) == ld
    _ints("cache_write", "counts", counts, (c.batch,), k[1])
    return c, k[2][1], ld, same


@functools.lru_cache(maxsize=256)
def _compact_plan(k_pages, v_pages, page_table, lengths, path, n_accepted):
    c = _kv_cache("cache_compact", k_pages, v_pages, page_table, lengths, all_layers=True)
    if len(path[2]) != 2:
        raise ValueError("cache_compact: path must be an int32 [B, n] tensor")
    _ints("cache_compact", "path", path, (c.batch, path[2][1]), k_pages[1])
    _ints("cache_compact", "n_accepted", n_accepted, (c.batch,), k_pages[1])
    return c, path[2][1]


@functools.lru_cache(maxsize=256)
def _attention_plan(q, k_pages, v_pages, page_table, lengths, parents):
    c = _kv_cache("tree_attention", k_pages, v_pages, page_table, lengths)
    ld = _step_rows("tree_attention", q, "q", c, k_pages)
    n, heads = q[2][1], q[2][2]
    _ints("tree_attention", "parents", parents, (c.batch, n), q[1])
    c.k = c.v = c.page_table = c.lengths = 16  # (no address is looked at for the size)
    return c, n, heads, ld, c.head_dim ** -0.5, B.tree_attention_workspace(c, n, heads)


@functools.lru_cache(maxsize=256)
def _verify_plan(target, tokens, parents, u_accept, u_sample, draft, draft_params, temperature, top_p, greedy):
    _, dev, shape, _ = target
    if dev < 0:
        raise RuntimeError("tree_verify runs on the GPU only")
    if len(shape) != 3:
        raise ValueError("tree_verify: target_logits must be a [B, n, V] tensor")
    Bt, n, V = shape
    for what, x, want in (("target_logits", target, (Bt, n, V)), ("draft_logits", draft, (Bt, n, V)),
                          ("u_accept", u_accept, (Bt, n)), ("u_sample", u_sample, (Bt,))):
        if x is not None and (x[0] != torch.float32 or x[2] != want or x[1] != dev or not _packed(x[2], x[3])):
            raise ValueError(f"tree_verify: {what} must be a contiguous float32 {list(want)} tensor on one device")
    if tokens is None:
        raise ValueError("tree_verify: tokens are required")
    _ints("tree_verify", "tokens", tokens, (Bt, n), dev)
    _ints("tree_verify", "parents", parents, (Bt, n), dev)
    if draft_params is not None:
        count = 1
        for k in draft_params[2]:
            count *= k
        if draft_params[0] != torch.uint8 or draft_params[1] != dev or not _packed(draft_params[2], draft_params[3]) or \
                count < Bt * n * B.ROW_PARAMS_BYTES:
            raise ValueError("tree_verify: draft_params must be contiguous uint8 of B * n records")
    s = B.make_sampling(V, temperature, top_p, greedy)
    return Bt, n, s, B.tree_verify_workspace(s, Bt, n)


@functools.lru_cache(maxsize=256)
def _quant_plan(x):
    dtype, dev, shape, stride = x
    if dev < 0:
        raise RuntimeError("quantize_rows runs on the GPU only")
    if len(shape) != 2 or 0 in shape or (shape[1] > 1 and stride[1] != 1):
        raise ValueError("quantize_rows: x must be a non-empty [T, d] tensor with neighbouring elements in a row")
    T, d = shape
    ld = stride[0] if T > 1 else d
    if ld < d:
        raise ValueError("quantize_rows: the rows of x must not overlap (an expanded x: call .contiguous())")
    return T, d, ld, _dtype_code(dtype)


@functools.lru_cache(maxsize=256)
def _int8_plan(o, W, W_scale, out):
    if o[1] < 0 or W[1] != o[1] or W_scale[1] != o[1]:
        raise RuntimeError("head_logits_int8 runs on the GPU only, on tensors of one device")
    if W[0] != torch.int8 or W_scale[0] != torch.float32:
        raise TypeError("head_logits_int8: W must be int8 and W_scale float32")
    if len(o[2]) != 2 or len(W[2]) != 2 or o[2][1] != W[2][1] or W_scale[2] != (W[2][0],) or \
            not all(_packed(x[2], x[3]) for x in (o, W, W_scale)):
        raise ValueError("o [T, d], W [V, d] and W_scale [V] must be contiguous with a shared d")
    (T, d), V = o[2], W[2][0]
    if out is not None and (out[0] != torch.float32 or out[2] != (T, V) or out[1] != o[1] or
                            not _packed(out[2], out[3])):
        raise ValueError("out must be a contiguous float32 [T, V] tensor")
    return T, d, V, _dtype_code(o[0]), B.head_logits_int8_workspace(T, d)


def cache_write(k: torch.Tensor, v: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor,
                page_table: torch.Tensor, lengths: torch.Tensor, *, counts: Optional[torch.Tensor] = None) -> None:
    """Writes new entries ``k``, ``v [B, n, kv_heads, head_dim]`` behind the ``lengths [B]`` that each sequence has.

    ``k_pages`` and ``v_pages`` are ``[pages, kv_heads, page_size, head_dim]`` (bf16 or float32, any strides of whole
    16 bytes), ``page_table`` (int32 ``[B, pages of a sequence]``; columns of a wider table will do) names the pages
    of each sequence: entry ``t`` is row ``t % page_size`` of page ``page_table[b, t // page_size]``. ``counts``
    (int32 ``[B]``): how many of the ``n`` a sequence has (a padded batch of prompts or trees). A sequence of length
    below 0 takes no part, and pages outside the pool are not written. ``lengths`` stay as they are.
    """
    _no_grad("cache_write", k, v, k_pages, v_pages)
    c, n, ld, same = _write_plan(_meta(k), _meta(v), _meta(k_pages), _meta(v_pages), _meta(page_table),
                                 _meta(lengths), _meta(counts))
    if not same:  # one set of strides for both
        return cache_write(k.contiguous(), v.contiguous(), k_pages, v_pages, page_table, lengths, counts=counts)
    c = _with_addresses(c, k_pages, v_pages, page_table, lengths)
    dev = k.device
    with _on(dev):
        B.cache_write(c, n, k.data_ptr(), v.data_ptr(), ld, counts.data_ptr() if counts is not None else None,
                      _stream(dev))
    _written(k_pages, v_pages)


def cache_compact(k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor,
                  path: torch.Tensor, n_accepted: torch.Tensor) -> torch.Tensor:
    """Moves the entries of an accepted path together and returns the sequences' new lengths (int32 ``[B]``).

    ``path [B, n]`` and ``n_accepted [B]`` are those of :func:`tree_verify` for a tree whose entries
    :func:`cache_write` put behind ``lengths``: entry ``lengths + j`` takes what entry ``lengths + path[:, j]`` held,
    for ``j`` up to ``n_accepted``. The pages may be those of all layers, ``[layers, pages, kv_heads, page_size,
    head_dim]``, for one call. Where ``lengths`` or ``n_accepted`` is below 0, nothing moves.
    """
    _no_grad("cache_compact", k_pages, v_pages)
    c, n = _compact_plan(_meta(k_pages), _meta(v_pages), _meta(page_table), _meta(lengths), _meta(path),
                         _meta(n_accepted))
    c = _with_addresses(c, k_pages, v_pages, page_table, lengths)
    dev = k_pages.device
    new = torch.empty(c.batch, dtype=torch.int32, device=dev)
    with _on(dev):
        B.cache_compact(c, n, path.data_ptr(), n_accepted.data_ptr(), new.data_ptr(), _stream(dev))
    _written(k_pages, v_pages)
    return new


def tree_attention(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor,
                   lengths: torch.Tensor, parents: Optional[torch.Tensor] = None, *,
                   scale: Optional[float] = None) -> torch.Tensor:
    """Attention from the nodes of each sequence's tree of drafted tokens, ``q [B, n, heads, head_dim]``.

    Pages, ``page_table`` and ``lengths`` as in :func:`cache_write`, which has put the ``n`` nodes' entries behind the
    ``lengths`` of the context. Node ``i`` attends to the whole context, to its ancestors and to itself. ``parents``
    (int32 ``[B, n]``): -1 for a node behind the context, else an earlier node; any other number marks a node that
    the tree does not have (nor any below it), whose rows are zeros. Without ``parents`` the nodes are a chain, and
    ``n = 1`` is a decoding step without a draft. Up to 64 nodes; ``heads`` is a multiple of the pages' ``kv_heads``
    (consecutive heads share one); ``head_dim`` 32, 64, 96, 128, 192 or 256; ``scale`` is ``head_dim ** -0.5`` by
    itself. bf16 or float32, sums in float32; the weights of bf16 values are rounded to bf16. What a node does not
    attend to does not change a bit of its result, whatever it holds. The entries are taken in parts as the table's
    width has it, so pass the columns that are in use.
    """
    _no_grad("tree_attention", q, k_pages, v_pages)
    c, n, heads, ld, default, ws_bytes = _attention_plan(_meta(q), _meta(k_pages), _meta(v_pages),
                                                         _meta(page_table), _meta(lengths), _meta(parents))
    c = _with_addresses(c, k_pages, v_pages, page_table, lengths)
    dev = q.device
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device=dev) if ws_bytes else None
    out = torch.empty(q.shape, dtype=q.dtype, device=dev)
    with _on(dev):
        B.tree_attention(c, n, heads, q.data_ptr(), ld, parents.data_ptr() if parents is not None else None,
                         default if scale is None else scale, out.data_ptr(),
                         ws.data_ptr() if ws is not None else None, ws_bytes, _stream(dev))
    return out


def tree_verify(target_logits: torch.Tensor, tokens: torch.Tensor, parents: Optional[torch.Tensor],
                u_accept: Optional[torch.Tensor], u_sample: Optional[torch.Tensor], *,
                draft_logits: Optional[torch.Tensor] = None, draft_params: Optional[torch.Tensor] = None,
                temperature: float = 1.0, top_p: float = 1.0, greedy: bool = False):
    """``(n_accepted [B], path [B, n], next_token [B])`` (int32): speculative verification of drafted trees.

    Node 0 of each tree is the last decided token. ``target_logits [B, n, V]`` (fp32) are the verifier's at every
    node, ``tokens [B, n]`` (int32) the drafted ones and ``parents [B, n]`` (int32) the tree: an earlier node, or any
    other number for a node that is not there; None is a chain. ``draft_logits [B, n, V]``: the draft's at every
    node, from which its children were drawn, each by itself (rows of nodes without children are not used); without
    them the children are taken as proposals without probabilities, such as the draft's most likely tokens. Children
    are tried in node order with ``u_accept [B, n]``; where none is taken the next token is drawn with ``u_sample
    [B]`` from what is left of the verifier's distribution, which the tokens follow in either case.
    ``path`` holds the taken nodes from node 0 on, then -1 (:func:`cache_compact` takes it). ``draft_params``: optional
    uint8 records ``[B, n]`` from ``sample(params=)`` on the draft's rows with the same settings.
    """
    _no_grad("tree_verify", target_logits, draft_logits)
    Bt, n, s, ws_bytes = _verify_plan(_meta(target_logits), _meta(tokens), _meta(parents), _meta(u_accept),
                                      _meta(u_sample), _meta(draft_logits), _meta(draft_params),
                                      ctypes.c_float(temperature).value, ctypes.c_float(top_p).value, bool(greedy))
    dev = target_logits.device
    ptr = (lambda x: x.data_ptr() if x is not None else None)
    out = torch.empty(Bt * (n + 2), dtype=torch.int32, device=dev)
    n_acc, path, nxt = out[:Bt], out[Bt:Bt * (n + 1)].view(Bt, n), out[Bt * (n + 1):]
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device=dev) if ws_bytes else None
    to = out.data_ptr()
    with _on(dev):
        B.tree_verify(s, Bt, n, target_logits.data_ptr(), ptr(draft_logits), tokens.data_ptr(), ptr(parents),
                      ptr(u_accept), ptr(u_sample), to, to + 4 * Bt, to + 4 * Bt * (n + 1), ptr(ws), ws_bytes,
                      _stream(dev), draft_params=ptr(draft_params))
    return n_acc, path, nxt


def quantize_rows(x: torch.Tensor):
    """``(q int8 [T, d], scale float32 [T])`` of the rows of ``x [T, d]`` (bf16 or float32; rows may lie apart).

    ``scale = max |x| / 127`` of a row (float32) and ``q`` the integers next to ``x / scale``: the form in which
    :func:`head_logits_int8` takes a head's weights.
    """
    _no_grad("quantize_rows", x)
    T, d, ld, code = _quant_plan(_meta(x))
    dev = x.device
    q = torch.empty(T, d, dtype=torch.int8, device=dev)
    scale = torch.empty(T, dtype=torch.float32, device=dev)
    with _on(dev):
        B.quantize_rows(T, d, ld, code, x.data_ptr(), q.data_ptr(), scale.data_ptr(), _stream(dev))
    return q, scale


def head_logits_int8(o: torch.Tensor, W: torch.Tensor, W_scale: torch.Tensor, out: Optional[torch.Tensor] = None):
    """:func:`head_logits` with the head's weights as 8-bit integers, ``W int8 [V, d]`` and ``W_scale [V]`` of
    :func:`quantize_rows`: half the bytes of bf16. The rows of ``o [T, d]`` (bf16 or float32) are made 8-bit integers
    in the same way, and the products are summed exactly. ``d`` is a multiple of 16.
    """
    _no_grad("head_logits_int8", o, W_scale, out)
    T, d, V, code, ws_bytes = _int8_plan(_meta(o), _meta(W), _meta(W_scale), _meta(out))
    dev = o.device
    given = out is not None
    if not given:
        out = torch.empty(T, V, dtype=torch.float32, device=dev)
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
    with _on(dev):
        B.head_logits_int8(T, V, d, code, o.data_ptr(), W.data_ptr(), W_scale.data_ptr(), out.data_ptr(),
                           ws.data_ptr(), ws_bytes, _stream(dev))
    if given:
        _written(out)
    return out


def coefficients(M: int, *, alpha: float, tau: float = 1.0, teacher: int = -1,
                 mode: str = "paper", weights: Optional[Sequence[float]] = None):
    """``(g_ce, g_kl)`` lists of eq. (3) (``mode="paper"``) or the additive form."""
    m = B.MLS_MODE_PAPER if mode == "paper" else B.MLS_MODE_ADDITIVE
    return B.coeffs(M, teacher, alpha, tau, m, weights)
