"""The post-training entry points write nothing outside of their workspaces and outputs.

Every buffer lies between two guard areas of a fixed pattern in one allocation, and is
exactly as large as the queries and the documentation say; the pattern has to be there
afterwards. (Writes inside the allocation: nothing here can fault.)
"""

import pytest
import torch

from paper_2608_09703_amd import api as D
from paper_2608_09703_amd import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
GUARD = 4 << 20


class _Guarded:
    def __init__(self):
        self.all = []

    def __call__(self, nbytes, name):
        raw = torch.full((GUARD + (nbytes + 255) // 256 * 256 + GUARD,), 0xA5, dtype=torch.uint8, device=DEV)
        self.all.append((name, raw, GUARD, GUARD + nbytes))
        return raw[GUARD:GUARD + nbytes]

    def check(self, what):
        torch.cuda.synchronize()
        for name, raw, a, b in self.all:
            assert bool((raw[:a] == 0xA5).all()) and bool((raw[b:] == 0xA5).all()), f"{what}: {name}"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d,V", [(1, 64, 300), (129, 64, 257), (129, 2048, 300), (300, 2048, 1000),
                                   (641, 2080, 777), (300, 200, 515), (260, 96, 5000)])
@pytest.mark.parametrize("chunk", [0, 256])
def test_token_logp(T, d, V, chunk, dtype):
    h = torch.randn(T, d, device=DEV).to(dtype)
    W = (torch.randn(V, d, device=DEV) * 0.05).to(dtype)
    tokens = torch.randint(0, V, (T,), device=DEV)
    tokens[1::4] = -100
    g = _Guarded()
    es = h.element_size()
    for flags, keep in ((0, False), (0, True), (B.MLS_ACCUMULATE_GRAD_H, False)):
        p = D.make_problem([h], [W], tokens, grad_h_dtype=dtype, vocab_chunk=chunk,
                           flags=flags | (B.MLS_GRAD_W_BF16 if es == 2 else 0))
        fwd, bwd, kb = B.token_logp_workspace(p)
        kept = g(kb, "kept").data_ptr() if keep and kb else None
        stats, logp, ent = g(B.query_sizes(p)[1], "stats"), g(4 * T, "logp"), g(4 * T, "entropy")
        gh, gW = g(T * d * es, "grad_h"), g(V * d * es, "grad_W")
        gl = torch.randn(T, device=DEV)
        s = D._stream(h.device)
        w1, w2 = g(fwd, "forward workspace"), g(bwd, "backward workspace")
        B.token_logp_fwd(p, stats.data_ptr(), logp.data_ptr(), ent.data_ptr(), kept, w1.data_ptr(), fwd, s)
        B.token_logp_bwd(p, stats.data_ptr(), kept, gl.data_ptr(), gh.data_ptr(), gW.data_ptr(), w2.data_ptr(), bwd, s)
        g.check(f"T={T} d={d} V={V} chunk={chunk}")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d", [(1, 1), (3, 7), (5, 513), (700, 1001), (2050, 64), (40, 4352), (3, 16384)])
def test_layer_norm(T, d, dtype):
    g = _Guarded()
    es = torch.empty((), dtype=dtype).element_size()
    x, w = torch.randn(T, d, device=DEV).to(dtype), torch.randn(d, device=DEV)
    gy = torch.randn(T, d, device=DEV).to(dtype)
    n = D._make_layer_norm(T, d, d, D._dtype_code(dtype), B.MLS_F32, 1e-5)
    y, st, gx = g(T * d * es, "y"), g(8 * T, "stats"), g(T * d * es, "g_x")
    gw, gb, nb = g(4 * d, "g_weight"), g(4 * d, "g_bias"), B.layer_norm_workspace(n)
    ws, s = g(nb, "workspace"), D._stream(x.device)
    B.layer_norm_fwd(n, x.data_ptr(), w.data_ptr(), w.data_ptr(), y.data_ptr(), st.data_ptr(), s)
    B.layer_norm_bwd(n, x.data_ptr(), w.data_ptr(), st.data_ptr(), gy.data_ptr(), gx.data_ptr(), gw.data_ptr(),
                     gb.data_ptr(), ws.data_ptr(), nb, s)
    g.check(f"T={T} d={d}")


@pytest.mark.parametrize("lens", [[1], [3, 0, 5], [1000, 24], [1, 4096], [2000] * 5])
def test_policy_loss(lens):
    g = _Guarded()
    S, N = len(lens), sum(lens)
    cu = torch.tensor([0] + lens, dtype=torch.int32, device=DEV).cumsum(0).int()
    x = torch.randn(N, device=DEV)
    mask = torch.rand(N, device=DEV) < 0.5
    p = B.make_policy(N, S, 0.2, 0.2, 0.1, B.MLS_POLICY_MEAN_OF_SEQUENCES)
    nb = B.policy_loss_workspace(p)
    out = [g(4, k) for k in ("loss", "kl", "clipped")]
    grad, ws, gl, s = g(4 * (N + 1), "grad"), g(nb, "workspace"), g(4 * N, "g_logp"), D._stream(x.device)
    one = torch.ones((), device=DEV)
    B.policy_loss_fwd(p, x.data_ptr(), x.data_ptr(), x.data_ptr(), x.data_ptr(), mask.data_ptr(), cu.data_ptr(),
                      *[o.data_ptr() for o in out], grad.data_ptr(), ws.data_ptr(), nb, s)
    B.policy_loss_bwd(N, grad.data_ptr(), one.data_ptr(), gl.data_ptr(), s)
    g.check(f"{lens}")


@pytest.mark.parametrize("sizes", [[1], [16384, 16385, 7], [5] * 300, [100001, 3, 0, 40000]])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_clip_grad_norm(sizes, dtype):
    g = _Guarded()
    es = torch.empty((), dtype=dtype).element_size()
    grads = [torch.randn(n, device=DEV).to(dtype) for n in sizes]
    out = [g(max(n, 1) * es, f"out {i}") for i, n in enumerate(sizes[:40])]
    to = [o.data_ptr() for o in out] + [x.data_ptr() for x in grads[40:]]
    t = B.make_grad_tensors([x.data_ptr() for x in grads], to, sizes, [D._dtype_code(dtype)] * len(sizes))
    nb = B.clip_grad_norm_workspace(len(sizes), t)
    ws, norm = g(nb, "workspace"), g(4, "norm")
    B.clip_grad_norm(len(sizes), t, 0.1, norm.data_ptr(), ws.data_ptr(), nb, D._stream(grads[0].device))
    g.check(f"{len(sizes)} tensors")
