"""A decoder layer on the library's operators: its gradients against autograd in 64 bits, and its blocks through the optimizer's path."""
import pytest
import torch

import paper_2605_16184_amd as ast
from paper_2605_16184_amd.layer import DecoderLayer, gradient_blocks
from paper_2605_16184_amd import workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _reference(layer, r, cu, dout, step):
    """Output and gradients of the layer in 64 bits; the masks come from the library's dropout, which has tests of its own."""
    p, rows, d = layer.dropout, layer.rows, layer.d

    def mask(offset):
        if not p:
            return torch.ones(rows, d, dtype=torch.float64, device=DEV)
        one = torch.ones(rows, d, device=DEV)
        ast.dropout(one, one, p, seed=layer.seed, offset=offset)
        return one.double()

    w = {k: getattr(layer, k).double().requires_grad_() for k in ("qkv", "o", "gate_up", "down", "norm1", "norm2")}
    x = r.double().requires_grad_()
    norm = lambda t, g: t * torch.rsqrt(t.square().mean(1, keepdim=True) + layer.eps) * g
    qkv = (norm(x, w["norm1"]) @ w["qkv"].T).view(rows, -1, layer.dim)
    group = layer.heads // layer.kv_heads
    parts = []
    for j in range(layer.heads):
        kv = layer.heads + j // group
        q, k, v = qkv[:, j], qkv[:, kv], qkv[:, kv + layer.kv_heads]
        out = torch.zeros(rows, layer.dim, dtype=torch.float64, device=DEV)
        for s, e in zip(cu[:-1], cu[1:]):
            z = q[s:e] @ k[s:e].T * layer.dim ** -0.5
            z = z.masked_fill(torch.ones(e - s, e - s, device=DEV).triu(1).bool(), float("-inf"))
            out = torch.cat([out[:s], torch.softmax(z, 1) @ v[s:e], out[e:]])
        parts.append(out)
    H = x + (torch.cat(parts, 1) @ w["o"].T) * mask(2 * step)
    gu = norm(H, w["norm2"]) @ w["gate_up"].T
    f = (torch.nn.functional.silu(gu[:, :layer.ffn]) * gu[:, layer.ffn:]) @ w["down"].T
    y = H + f * mask(2 * step + 1)
    y.backward(dout.double())
    kv, d_ = layer.kv_heads * layer.dim, layer.d
    g = {"q": w["qkv"].grad[:d_], "k": w["qkv"].grad[d_:d_ + kv], "v": w["qkv"].grad[d_ + kv:], "o": w["o"].grad, "gate": w["gate_up"].grad[:layer.ffn],
         "up": w["gate_up"].grad[layer.ffn:], "down": w["down"].grad, "norm1": w["norm1"].grad, "norm2": w["norm2"].grad}
    return y.detach(), x.grad, g


# A result passes through about a dozen roundings of relative size u (the operands of every product, the stored activations), each at
# most once amplified by sums that cancel: 16 u in the norm
@pytest.mark.parametrize("dtype,tol", [(torch.float32, 1e-4), (torch.bfloat16, 16 * 2.0 ** -8)])
@pytest.mark.parametrize("dropout", [0.0, 0.25])
def test_layer_gradients_against_autograd(dtype, tol, dropout):
    rows, lens = 200, [70, 1, 100, 20]
    layer = DecoderLayer(rows, d=96, heads=6, kv_heads=2, ffn=200, dtype=dtype, dropout=dropout, seed=7)
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    g = torch.Generator(device=DEV).manual_seed(3)
    r, dout = torch.randn(rows, 96, generator=g, device=DEV), torch.randn(rows, 96, generator=g, device=DEV)
    y = layer.forward(r, torch.tensor(cu, dtype=torch.int32, device=DEV), step=5)
    dr, grads = layer.backward(dout)
    y64, dr64, g64 = _reference(layer, r, cu, dout, 5)
    rel = lambda a, b: float(torch.linalg.norm(a.double() - b) / torch.linalg.norm(b))
    assert rel(y, y64) <= tol and rel(dr, dr64) <= tol
    for k in g64:
        assert rel(grads[k], g64[k]) <= tol, k


def test_layer_with_other_sequences_at_every_step():
    # few sequences take a larger workspace of the attention's backward pass than many
    rows = 1024
    layer = DecoderLayer(rows, d=64, heads=8, kv_heads=1, ffn=96, seed=2)
    g = torch.Generator(device=DEV).manual_seed(4)
    for n in (512, 1, 64):
        cu = torch.arange(0, rows + 1, rows // n, dtype=torch.int32, device=DEV)
        r, dout = torch.randn(rows, 64, generator=g, device=DEV), torch.randn(rows, 64, generator=g, device=DEV)
        fresh = DecoderLayer(rows, d=64, heads=8, kv_heads=1, ffn=96, seed=2)
        assert torch.equal(layer.forward(r, cu), fresh.forward(r, cu))
        (dr, grads), (want, wants) = layer.backward(dout), fresh.backward(dout)
        assert torch.equal(dr, want) and all(torch.equal(grads[k], wants[k]) for k in grads)


def test_layer_gradients_through_statistics_roots_and_update():
    rows = 384
    layer = DecoderLayer(rows, d=256, heads=4, kv_heads=2, ffn=320, dropout=0.125)
    g = torch.Generator(device=DEV).manual_seed(1)
    cu = torch.tensor([0, 130, 384], dtype=torch.int32, device=DEV)
    mats = [(n, layer.d if n in "qo" else layer.kv_heads * layer.dim if n in "kv" else layer.d if n == "down" else layer.ffn,
             layer.ffn if n == "down" else layer.d) for n in DecoderLayer.MATRICES]
    shapes = W.block_shapes(mats, 200)
    Ls, Rs = [torch.eye(m, device=DEV) * 1e-8 for m, _ in shapes], [torch.eye(n, device=DEV) * 1e-8 for _, n in shapes]
    for step in range(3):
        r, dout = torch.randn(rows, 256, generator=g, device=DEV), torch.randn(rows, 256, generator=g, device=DEV) * 1e-2
        layer.forward(r, cu, step=step)
        _, grads = layer.backward(dout)
        Gs = gradient_blocks(grads, 200)
        assert [tuple(G.shape) for G in Gs] == shapes
        ast.stats_update(list(zip(Gs, Ls, Rs)), 0.95)
    XLs, XRs = [torch.empty_like(L) for L in Ls], [torch.empty_like(R) for R in Rs]
    info = torch.full((2 * len(shapes),), -1, dtype=torch.int32, device=DEV)
    ast.inverse_root(list(zip(Ls, XLs)) + list(zip(Rs, XRs)), 1e-5, info=info)
    Ps = [torch.empty(s, device=DEV) for s in shapes]
    ast.precondition(list(zip(XLs, Gs, XRs, Ps)))
    assert int(info.abs().sum()) == 0
    for G, L, R, P in zip(Gs, Ls, Rs, Ps):
        assert bool(torch.isfinite(P).all())
        # the update is the gradient under the statistics' inverse roots, in 64 bits
        want = G.double()
        for A, left in ((L, True), (R, False)):
            lam, V = torch.linalg.eigh(A.double())
            X = (V * (lam + 1e-5 * lam[-1]).clamp_min(1e-30).pow(-0.25)) @ V.T.contiguous()
            want = X @ want if left else want @ X
        assert float(torch.linalg.norm(P.double() - want) / torch.linalg.norm(want)) <= 2e-2
