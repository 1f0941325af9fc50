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


def coefficients(M: int, *, alpha: float, tau: float = 1.0, teacher: int = -1,
                 mode: str = "paper", weights: Optional[Sequence[float]] = None):
    """``(g_ce, g_kl)`` lists of eq. (3) (``mode="paper"``) or the additive form."""
    m = B.MLS_MODE_PAPER if mode == "paper" else B.MLS_MODE_ADDITIVE
    return B.coeffs(M, teacher, alpha, tau, m, weights)
