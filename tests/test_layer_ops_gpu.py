"""Norm, dropout and attention against plain implementations in 64 bits, at the sizes and layouts where they can go wrong.

Tolerances are bounds from the roundings made: U[t] = eps / 2 of an output's or operand's type, relative to the value; sums in fp32
(F = 2^-24 an addition) relative to the sum of the terms' magnitudes."""
import math

import numpy as np
import pytest
import torch

import paper_2605_16184_amd as ast

pytestmark = pytest.mark.gpu
DEV = "cuda"
F = 2.0 ** -24
TINY = 2.0 ** -126
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float8_e4m3fn: 2.0 ** -4}
f32, bf16, e4m3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn


def _randn(*shape, dtype=f32, seed=0, std=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed * 7919 + 11)
    return (std * torch.randn(*shape, generator=g, device=DEV)).to(dtype)


def _inside(got, ref, tol, what):
    err = (got.double() - ref).abs()
    assert torch.isfinite(got.double()).all(), what
    worst = (err / tol.clamp_min(1e-300)).max() if err.numel() else 0.0
    assert bool((err <= tol).all()), f"{what}: {float(worst):.3g} of the tolerance"


# ---- dropout --------------------------------------------------------------------------------------
def _philox(seed, offset, rows, cols):
    """The 16-bit numbers of every element, by the definition, in Python's own integers on the host."""
    out = np.empty((rows, (cols + 7) // 8 * 8), dtype=np.int64)
    mask = 0xFFFFFFFF
    for r in range(rows):
        for c in range(out.shape[1] // 8):
            x = [c, r, offset & mask, offset >> 32]
            k = [seed & mask, seed >> 32]
            for _ in range(10):
                p, q = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57
                x = [(q >> 32) ^ x[1] ^ k[0], q & mask, (p >> 32) ^ x[3] ^ k[1], p & mask]
                k = [(k[0] + 0x9E3779B9) & mask, (k[1] + 0xBB67AE85) & mask]
            out[r, 8 * c:8 * c + 8] = [(x[e // 2] >> (16 * (e % 2))) & 0xFFFF for e in range(8)]
    return torch.from_numpy(out[:, :cols]).to(DEV)


def test_generator_gives_the_published_vector():
    # key and counter of all ones: the first known answer of the method's publication with ten rounds that is not all zeros
    n = (1 << 64) - 1
    c = 0xFFFFFFFF
    x, k = [c, c, c, c], [c, c]
    for _ in range(10):
        p, q = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57
        x = [(q >> 32) ^ x[1] ^ k[0], q & c, (p >> 32) ^ x[3] ^ k[1], p & c]
        k = [(k[0] + 0x9E3779B9) & c, (k[1] + 0xBB67AE85) & c]
    assert x == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    # and the kernel at the largest seed and offset
    X = torch.ones(3, 17, device=DEV)
    Y = torch.empty_like(X)
    ast.dropout(X, Y, 0.5, seed=n, offset=n)
    assert torch.equal(Y != 0, _philox(n, n, 3, 17) >= 32768)


@pytest.mark.parametrize("dtype", [f32, bf16])
@pytest.mark.parametrize("rows,cols,ld,p", [(1, 1, 1, 0.5), (3, 7, 9, 0.25), (5, 8, 8, 0.1), (17, 333, 340, 0.9), (2, 1000, 1001, 2.0 ** -16),
                                            (300, 9, 9, 65535 / 65536)])
def test_dropout_is_the_definition(rows, cols, ld, p, dtype):
    X = _randn(rows, ld, dtype=dtype, seed=rows)[:, :cols]
    full = torch.full((rows, ld + 3), -7.0, dtype=dtype, device=DEV)
    Y = full[:, 2:2 + cols] if cols + 2 <= ld + 3 else full[:, :cols]
    seed, offset = 0x123456789ABCDEF0 + rows, (5 << 32) + cols
    ast.dropout(X, Y, p, seed=seed, offset=offset)
    t = round(p * 65536)
    keep = _philox(seed, offset, rows, cols) >= t
    scale = torch.tensor(65536.0 / (65536 - t), dtype=torch.float64).float().item()
    assert torch.equal(Y, torch.where(keep, X.float() * scale, 0.0).to(dtype))
    Y.fill_(-7.0)
    assert bool((full == -7.0).all())                      # nothing beside the view was written


def test_dropout_in_place_infinities_state_and_gradient():
    X = _randn(64, 1030, seed=3)
    X[5, 7] = math.inf
    X[6, 8] = math.nan
    Y, Z = torch.empty_like(X), X.clone()
    state = torch.tensor([77, 5], dtype=torch.int64, device=DEV)
    ast.dropout(X, Y, 0.3, seed=77, offset=5)
    ast.dropout(Z, Z, 0.3, rng=state)
    assert torch.equal(torch.nan_to_num(Y, 123.0), torch.nan_to_num(Z, 123.0))
    keep = Y != 0
    assert bool((Y[~keep] == 0).all()) and abs(keep.float().mean().item() - 0.7) < 5 * math.sqrt(0.21 / X.numel())
    G = torch.empty_like(X)
    ast.dropout(torch.ones_like(X), G, 0.3, seed=77, offset=5)
    assert torch.equal(G != 0, _philox(77, 5, 64, 1030) >= round(0.3 * 65536))
    W = torch.empty_like(X)
    ast.dropout(X, W, 0.0, seed=1)
    assert torch.equal(torch.nan_to_num(W, 123.0), torch.nan_to_num(X, 123.0))
    ast.dropout(X, W, 0.3, seed=77, offset=6)
    assert not torch.equal(W != 0, keep)


# ---- norm -----------------------------------------------------------------------------------------
def _factor(seed, offset, rows, cols, p):
    t = round(p * 65536)
    if t == 0:
        return torch.ones(rows, cols, dtype=torch.float64, device=DEV)
    ones, out = torch.ones(rows, cols, device=DEV), torch.empty(rows, cols, device=DEV)
    ast.dropout(ones, out, p, seed=seed, offset=offset)     # its mask is held against the definition above
    return (out != 0).double() * 65536.0 / (65536 - t)


# roundings on the way to y, relative to (|x| / (1 - p) + |R|) r |w|: x / (1 - p), the sum and y's two products 1 each; the mean of squares:
# at most 32 terms in a thread, 6 + 16 joins, each twice for the square: half of that in its root, and 3 for root, quotient and mean
NORM_ROUNDINGS = 4 + 28 + 3


def _norm_ref(X, R, W, factor, eps):
    h = X.double() * factor + (R.double() if R is not None else 0.0)
    r = 1.0 / torch.sqrt(h.square().mean(1, keepdim=True) + eps)
    w = W.double() if W is not None else torch.ones(X.shape[1], dtype=torch.float64, device=DEV)
    size = X.double().abs() * factor + (R.double().abs() if R is not None else 0.0)
    return h, h * r * w, size, size * r * w.abs()


WIDTHS = [1, 7, 8, 64, 127, 128, 129, 511, 512, 513, 777, 1024, 1025, 2047, 2048, 2049, 4097, 5632, 8193, 16384]


@pytest.mark.parametrize("cols", WIDTHS)
@pytest.mark.parametrize("xt,ht,yt,wt", [(bf16, bf16, bf16, bf16), (bf16, f32, bf16, f32), (f32, f32, f32, f32), (f32, bf16, f32, bf16)])
def test_norm_against_64_bits(cols, xt, ht, yt, wt):
    rows, pad = 9, 3
    X, R = _randn(rows, cols + pad, dtype=xt, seed=cols)[:, pad:], _randn(rows, cols + 1, dtype=ht, seed=cols + 1, std=2.0)[:, :cols]
    W = _randn(cols, dtype=wt, seed=cols + 2)
    H = torch.full((rows, cols + 5), 3.0, dtype=ht, device=DEV)
    Y = torch.full((rows, cols + 1), 3.0, dtype=yt, device=DEV)
    for p in (0.0, 0.25):
        ast.rms_norm(X, Y[:, 1:], W=W, R=R, H=H[:, :cols], eps=1e-5, p=p, seed=9, offset=2)
        h, y, hs, ys = _norm_ref(X, R, W, _factor(9, 2, rows, cols, p), 1e-5)
        _inside(H[:, :cols], h, U[ht] * 1.01 * h.abs() + 2 * F * hs, "H")
        _inside(Y[:, 1:], y, U[yt] * 1.01 * y.abs() + NORM_ROUNDINGS * F * ys, "Y")
        assert bool((H[:, cols:] == 3.0).all()) and bool((Y[:, 0] == 3.0).all())


@pytest.mark.parametrize("cols", [1, 100, 128, 136, 777, 2048, 2500, 8192, 16000])
@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("xt", [bf16, f32])
def test_norm_with_8_bit_output(cols, group, xt):
    rows = 5
    X, R, W = _randn(rows, cols, dtype=xt, seed=1), _randn(rows, cols, dtype=xt, seed=2), _randn(cols, seed=3)
    X[2], R[2] = 0, 0                                       # a row of zeros
    X[3] *= 1e-20
    R[3] = 0
    groups = -(-cols // 128) if group else 1
    Y = torch.zeros(rows, cols + 1, dtype=torch.uint8, device=DEV).view(e4m3)[:, :cols]
    S = torch.empty(rows, groups, device=DEV)
    ast.rms_norm(X, Y, W=W, R=R, scale=S, group=group, eps=1e-30)
    h, y, _, ys = _norm_ref(X, R, W, 1.0, 1e-30)
    z = torch.zeros(rows, groups * (group or cols), dtype=torch.float64, device=DEV)
    z[:, :cols] = y
    top = z.view(rows, groups, -1).abs().amax(2)
    tops = torch.zeros_like(z)
    tops[:, :cols] = ys
    near = (NORM_ROUNDINGS + 2) * F
    _inside(S, top.clamp_min(2.0 ** -100) / 448, near * tops.view(rows, groups, -1).amax(2) / 448 + 1e-40, "scale")
    spread = S.double().repeat_interleave(group or cols, 1)[:, :cols]
    # half a step: 2^-4 of the value, 2^-10 below the smallest normal number
    _inside(Y.float() * 1.0, y / spread, (U[e4m3] * 1.001 * y.abs() + 2 * near * ys) / spread + 2.0 ** -10, "Y")
    assert float(Y.float().abs().max()) <= 448.0
    assert bool((Y[2].float() == 0).all())


def test_norm_options_and_aliases():
    rows, cols = 33, 640
    X, R, W = _randn(rows, cols, seed=1), _randn(rows, cols, seed=2), _randn(cols, seed=3)
    H, Y = torch.empty_like(X), torch.empty_like(X)
    ast.rms_norm(X, Y, W=W, R=R, H=H, p=0.5, seed=3)
    for alias in ("R", "X", "Y", "RY"):
        x, r = X.clone(), R.clone()
        h = r if "R" in alias else x if alias == "X" else torch.empty_like(X)
        y = x if "Y" in alias else torch.empty_like(X)
        ast.rms_norm(x, y, W=W, R=r, H=h, p=0.5, rng=torch.tensor([3, 0], device=DEV))
        assert torch.equal(h, H) and torch.equal(y, Y), alias
    ast.rms_norm(X, Y)                                      # no weight, no residual, no sum
    _, y, _, ys = _norm_ref(X, None, None, 1.0, 1e-6)
    _inside(Y, y, F * y.abs() + NORM_ROUNDINGS * F * ys, "Y")
    ast.rms_norm(X, Y, H=H)
    assert torch.equal(H, X)


def test_norm_keeps_what_is_no_number_in_its_row():
    X = _randn(6, 300, dtype=bf16, seed=1)
    X[1, 3], X[4, 299] = math.nan, math.inf
    Y, S = torch.empty(6, 300, device=DEV).to(e4m3), torch.empty(6, 3, device=DEV)
    Z = torch.empty(6, 300, device=DEV)
    ast.rms_norm(X, Z)
    ast.rms_norm(X, Y, scale=S, group=128)
    good = [0, 2, 3, 5]
    for r in (1, 4):
        assert not bool(torch.isfinite(Z[r]).all()) and not bool(torch.isfinite(Y[r].float() * 1.0).all())
    assert bool(torch.isfinite(Z[good]).all()) and bool(torch.isfinite(Y[good].float()).all()) and bool(torch.isfinite(S[good]).all())


def _norm_grad_ref(H, dY, W, dH, eps):
    h, dy = H.double(), dY.double()
    w = W.double() if W is not None else torch.ones(H.shape[1], dtype=torch.float64, device=DEV)
    r = 1.0 / torch.sqrt(h.square().mean(1, keepdim=True) + eps)
    n = dy * w
    base = dH.double() if dH is not None else torch.zeros_like(h)
    dr = base + r * (n - h * r * r * (n * h).mean(1, keepdim=True))
    size = base.abs() + r * (n.abs() + h.abs() * r * r * (n * h).abs().mean(1, keepdim=True))
    return dr, size, (dy * h * r).sum(0), (dy * h * r).abs().sum(0)


@pytest.mark.parametrize("cols", WIDTHS)
@pytest.mark.parametrize("rows", [1, 13, 5000])
@pytest.mark.parametrize("xt,ht,yt,wt", [(bf16, bf16, bf16, bf16), (bf16, f32, bf16, f32), (f32, f32, f32, f32), (f32, bf16, f32, bf16)])
def test_norm_backward_against_64_bits(rows, cols, xt, ht, yt, wt):
    if rows * cols > 1 << 24:
        rows = (1 << 24) // cols
    H, dY, dH = _randn(rows, cols, dtype=ht, seed=1), _randn(rows, cols + 1, dtype=yt, seed=2)[:, 1:], _randn(rows, cols, dtype=ht, seed=3)
    W = _randn(cols, dtype=wt, seed=4)
    dX, dR = torch.full((rows, cols + 3), 5.0, dtype=xt, device=DEV), torch.empty(rows, cols, dtype=ht, device=DEV)
    dW = torch.empty(cols, dtype=wt, device=DEV)
    ast.rms_norm_backward(H, dY, W=W, dH=dH, dX=dX[:, :cols], dR=dR, dW=dW, eps=1e-5, p=0.25, seed=4, offset=8)
    dr, size, dw, dws = _norm_grad_ref(H, dY, W, dH, 1e-5)
    k = 3 * NORM_ROUNDINGS                                  # two means and three uses of r
    _inside(dR, dr, U[ht] * 1.01 * dr.abs() + k * F * size, "dR")
    f = _factor(4, 8, rows, cols, 0.25)
    _inside(dX[:, :cols], dr * f, U[xt] * 1.01 * (dr * f).abs() + (k + 1) * F * size * f, "dX")
    assert bool((dX[:, cols:] == 5.0).all())
    # a term has NORM_ROUNDINGS roundings; a column is added up over the rows of a workgroup, its wavefronts, the workgroups
    adds = rows // 1024 + 2 + 4 + 32 + 32
    _inside(dW, dw, U[wt] * 1.01 * dw.abs() + (NORM_ROUNDINGS + adds) * F * dws, "dW")


def test_norm_backward_parts_aliases_and_differences():
    rows, cols = 37, 520
    H, dY, dH, W = (_randn(*s, seed=i) for i, s in enumerate([(rows, cols), (rows, cols), (rows, cols), (cols,)]))
    dX, dR, dW = torch.empty_like(H), torch.empty_like(H), torch.empty_like(W)
    ast.rms_norm_backward(H, dY, W=W, dH=dH, dX=dX, dR=dR, dW=dW, p=0.25, seed=1)
    one = torch.empty_like(H)
    ast.rms_norm_backward(H, dY, W=W, dH=dH, dR=one)
    assert torch.equal(one, dR)
    ast.rms_norm_backward(H, dY, W=W, dH=dH, dX=one, p=0.25, seed=1)
    assert torch.equal(one, dX)
    w2 = torch.empty_like(W)
    ast.rms_norm_backward(H, dY, W=W, dW=w2)
    assert torch.equal(w2, dW)
    a, b = dH.clone(), dY.clone()
    ast.rms_norm_backward(H, b, W=W, dH=a, dX=b, dR=a, dW=w2, p=0.25, seed=1)
    assert torch.equal(a, dR) and torch.equal(b, dX) and torch.equal(w2, dW)
    ast.rms_norm_backward(H, dY, dR=one)                    # no weight, no gradient by the residual path
    dr, size, _, _ = _norm_grad_ref(H, dY, None, None, 1e-6)
    _inside(one, dr, F * dr.abs() + 3 * NORM_ROUNDINGS * F * size, "dR")
    # against differences of the forward pass in 64 bits along a random direction: error of order t^2 times the third derivative
    ast.rms_norm_backward(H, dY, W=W, dR=one)
    D, t = _randn(rows, cols, seed=9).double(), 1e-4

    def value(h):
        return (dY.double() * h * W.double() / torch.sqrt(h.square().mean(1, keepdim=True) + 1e-6)).sum()

    num = (value(H.double() + t * D) - value(H.double() - t * D)) / (2 * t)
    mag = float((one.double().abs() * D.abs()).sum())
    assert abs(float(num) - float((one.double() * D).sum())) <= mag * (3 * NORM_ROUNDINGS * F + 10 * t * t)


# ---- attention -------------------------------------------------------------------------------------
def _attention_ref(Q, K, V, cu, scale, dO=None):
    """O, lse and the gradients in 64 bits, and bounds on what the kernels' roundings change of them."""
    total, heads, dim = Q.shape
    group, dt = heads // K.shape[1], Q.dtype
    up = U[bf16] if dt == bf16 else 0.0                     # P and dS as operands of the second product
    names = ["O", "dQ", "dK", "dV"]
    shapes = [Q.shape, Q.shape, K.shape, K.shape]
    ref = {k: torch.zeros(s, dtype=torch.float64, device=DEV) for k, s in zip(names, shapes)}
    tol = {k: torch.zeros(s, dtype=torch.float64, device=DEV) for k, s in zip(names, shapes)}
    ref["lse"], tol["lse"] = torch.zeros(heads, total, dtype=torch.float64, device=DEV), torch.zeros(heads, total, dtype=torch.float64, device=DEV)
    mm = lambda a, b: torch.mm(a.contiguous(), b.contiguous())
    largest = 0.0
    by_d = {"O": 0.0, "dQ": 0.0, "dK": 0.0, "dV": 0.0}      # squares of what the rounding of the stored O can change by way of D
    for s, e in zip(cu[:-1], cu[1:]):
        n = e - s
        for j in range(heads if n else 0):
            q, k, v = Q[s:e, j].double(), K[s:e, j // group].double(), V[s:e, j // group].double()
            seen = torch.ones(n, n, device=DEV).tril().bool()
            z = torch.where(seen, scale * mm(q, k.T), -math.inf)
            lse = torch.logsumexp(z, 1)
            largest = max(largest, float(torch.where(seen, z.abs(), 0.0).max()))
            p = torch.exp(z - lse[:, None])
            # the exponent: a sum of dim products, the scale, a difference; exp2 and the sum of n terms
            top = torch.where(seen, scale * mm(q.abs(), k.abs().T), 0.0).amax(1, keepdim=True)
            ez = top * (dim + 4) * F + 4 * F * (1 + lse.abs()[:, None])
            ep = 2 * ez + (n + 8) * F
            ref["O"][s:e, j] = mm(p, v)
            tol["O"][s:e, j] = U[dt] * 1.01 * mm(p, v).abs() + (ep + up * 1.01 + (n + 2) * F) * mm(p, v.abs())
            ref["lse"][j, s:e] = lse
            tol["lse"][j, s:e] = (ez + (n + 8) * F).squeeze(1) + 2 * F * lse.abs()
            if dO is None:
                continue
            g = dO[s:e, j].double()
            dp = mm(g, v.T)
            o = mm(p, v)
            ds = p * (dp - (g * o).sum(1, keepdim=True))
            size = mm(g.abs(), v.abs().T) + (g.abs() * mm(p, v.abs())).sum(1, keepdim=True)
            # D is made from O as stored; what P is off by
            eo = (tol["O"][s:e, j] * g.abs()).sum(1, keepdim=True)
            # below 2^-126, fp32's smallest normal number, P and every product count as zero: 2^-126 (|dP| + |D|) of a dS, 2^-126 a term
            es = (up * 1.01 + 2 * ep) * ds.abs() + p * (eo + (dim + 3) * F * size) + TINY * size
            kt, jk = (n + 2) * F, j // group
            tol["dQ"][s:e, j] += n * TINY
            tol["dK"][s:e, jk] += n * TINY
            tol["dV"][s:e, jk] += n * TINY + TINY * g.abs().sum(0)
            by_d["dQ"] += float((scale * mm(p * eo, k.abs())).square().sum())
            by_d["dK"] += float((scale * mm((p * eo).T, q.abs())).square().sum()) * group
            ref["dQ"][s:e, j] = scale * mm(ds, k)
            tol["dQ"][s:e, j] += U[dt] * 1.01 * ref["dQ"][s:e, j].abs() + scale * (mm(es, k.abs()) + kt * mm(ds.abs(), k.abs()))
            ref["dK"][s:e, jk] += scale * mm(ds.T, q)
            tol["dK"][s:e, jk] += scale * (mm(es.T, q.abs()) + (group + 1) * kt * mm(ds.abs().T, q.abs()))
            ref["dV"][s:e, jk] += mm(p.T, g)
            tol["dV"][s:e, jk] += mm(((up * 1.01 + 2 * ep + (group + 1) * kt) * p).T, g.abs())
    for k in ("dK", "dV"):
        tol[k] += U[dt] * 1.01 * ref[k].abs()
    ref["by_d"], ref["z"] = by_d, largest
    return ref, tol


def _attention_check(lens, heads, kv_heads, dim, dtype, lead=0, tail=0, layout="packed", scale=None, seed=0):
    total = lead + sum(lens) + tail
    if layout == "packed":                                  # one projection's output
        qkv = _randn(total, heads + 2 * kv_heads, dim, dtype=dtype, seed=seed)
        Q, K, V = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
    elif layout == "heads":                                 # head-major
        Q, K, V = (_randn(h, total, dim, dtype=dtype, seed=seed + i).transpose(0, 1) for i, h in enumerate((heads, kv_heads, kv_heads)))
    else:                                                   # rows at odd places
        Q, K, V = (_randn(total, h, dim + 3, dtype=dtype, seed=seed + i)[:, :, 1:dim + 1] for i, h in enumerate((heads, kv_heads, kv_heads)))
    like = (lambda t: torch.full_like(t.transpose(0, 1).contiguous(), 9.0).transpose(0, 1)) if layout == "heads" else \
        (lambda t: torch.full((t.shape[0], t.shape[1], dim + (3 if layout == "odd" else 0)), 9.0, dtype=dtype, device=DEV)[:, :, :dim])
    O, dQ, dK, dV = like(Q), like(Q), like(K), like(V)
    dO = _randn(total, heads, dim, dtype=dtype, seed=seed + 5)
    cu = [lead]
    for n in lens:
        cu.append(cu[-1] + n)
    dcu = torch.tensor(cu, dtype=torch.int32, device=DEV)
    if lead:                                                # rows of no sequence are not read
        for t in (Q, K, V, dO):
            t[:lead] = math.nan
    if tail:
        for t in (Q, K, V, dO):
            t[cu[-1]:] = math.nan
    lse = torch.full((heads, total), 9.0, device=DEV)
    sc = dim ** -0.5 if scale is None else scale
    ast.attention(Q, K, V, O, lse=lse, cu=dcu, scale=scale)
    ast.attention_backward(Q, K, V, O, lse, dO, dQ, dK, dV, cu=dcu, scale=scale)
    ref, tol = _attention_ref(Q, K, V, cu, sc, dO)
    s, e = cu[0], cu[-1]
    for name, t in (("O", O), ("dQ", dQ), ("dK", dK), ("dV", dV)):
        _inside(t[s:e], ref[name][s:e], tol[name][s:e], name)
        assert bool((t[:s] == 9.0).all()) and bool((t[e:] == 9.0).all()), name
        # all over a bf16 result: independent roundings of P or dS and of the result, each within its half step, and the rounding of
        # O, which dP - D does not scale down where one key has nearly all of a row (dP and D are then nearly equal)
        norm = torch.linalg.norm(ref[name][s:e]).clamp_min(1e-30)
        whole = float(torch.linalg.norm(t[s:e].double() - ref[name][s:e]) / norm)
        if max(lens) > 1:
            by_d = math.sqrt(ref["by_d"][name]) / float(norm)
            # P is as far off as its exponent z, relative to 1: the sum of dim products of rounding F each, sqrt(dim) F |z| in the mean
            by_z = math.sqrt(dim) * F * ref["z"]
            assert whole <= (math.sqrt(2 * U[bf16] ** 2 + by_d ** 2 + by_z ** 2) if dtype == bf16 else 1e-5 + by_d + by_z), (name, whole)
    _inside(lse[:, s:e], ref["lse"][:, s:e], tol["lse"][:, s:e], "lse")
    assert bool((lse[:, :s] == 9.0).all()) and bool((lse[:, e:] == 9.0).all())
    return Q, K, V, O, lse, dO, dQ, dK, dV, dcu


@pytest.mark.parametrize("dtype", [bf16, f32])
@pytest.mark.parametrize("lens", [[1], [2], [31], [32], [33], [63, 64, 65], [127], [128], [129], [0, 1, 0, 255, 256, 257, 0], [500, 3]])
@pytest.mark.parametrize("dim", [64, 128])
def test_attention_at_the_edges_of_its_tiles(lens, dim, dtype):
    _attention_check(lens, 4, 2, dim, dtype, lead=3, tail=5)


@pytest.mark.parametrize("dtype", [bf16, f32])
@pytest.mark.parametrize("dim", [1, 3, 8, 20, 32, 40, 63, 65, 80, 96, 127])
def test_attention_of_other_widths(dim, dtype):
    _attention_check([70, 9, 140], 2, 1, dim, dtype, tail=2)


@pytest.mark.parametrize("dtype", [bf16, f32])
@pytest.mark.parametrize("layout", ["packed", "heads", "odd"])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 3), (6, 2), (8, 1)])
def test_attention_of_heads_and_layouts(heads, kv_heads, layout, dtype):
    _attention_check([150, 41], heads, kv_heads, 64, dtype, tail=1, layout=layout)


@pytest.mark.parametrize("lens", [[5] * 64, [1] * 65 + [300], [0] * 100 + [200, 17] + [0] * 30, [129, 1] * 100])
def test_attention_of_many_sequences(lens):
    _attention_check(lens, 2, 1, 64, bf16, tail=7)


@pytest.mark.parametrize("dtype", [bf16, f32])
@pytest.mark.parametrize("heads,kv_heads", [(64, 16), (48, 48), (96, 2)])
@pytest.mark.parametrize("lens,dim,layout", [
    ([129, 257, 31, 300, 64], 64, "packed"), ([129, 257, 0, 300, 64, 1], 64, "odd"), ([400, 127, 128], 128, "packed"),
    ([385, 2, 250], 128, "odd"), ([300, 300], 96, "heads"), ([97, 480], 80, "packed"), ([280, 150, 33], 33, "packed")])
def test_attention_of_many_heads(lens, dim, layout, heads, kv_heads, dtype):
    # enough tiles of 128 rows for all of the chip; heads that share keys dealt to several workgroups
    _attention_check(lens, heads, kv_heads, dim, dtype, lead=2, tail=4, layout=layout)


@pytest.mark.parametrize("scale", [2.0 ** -100, 1e-12, 1e-3, 1.0, 4.0, 64.0])
@pytest.mark.parametrize("dtype", [bf16, f32])
def test_attention_with_flat_and_sharp_scores(scale, dtype):
    # at 4 a row is one key almost everywhere and scores grow by hundreds from tile to tile
    _attention_check([260], 2, 2, 64, dtype, scale=scale)


@pytest.mark.parametrize("dtype", [bf16, f32])
def test_attention_longer(dtype):
    _attention_check([1300, 700], 4, 2, 64, dtype)
    _attention_check([1100], 2, 1, 128, dtype)


def test_attention_without_offsets_and_with_broadcast_keys():
    Q, dO = _randn(200, 4, 64, dtype=bf16, seed=1), _randn(200, 4, 64, dtype=bf16, seed=2)
    K = _randn(1, 1, 64, dtype=bf16, seed=3).expand(200, 2, 64)          # strides of zero: read only
    V = _randn(200, 1, 64, dtype=bf16, seed=4).expand(200, 2, 64)
    O, dQ, lse = torch.empty_like(Q), torch.empty_like(Q), torch.empty(4, 200, device=DEV)
    dK, dV = torch.empty(200, 2, 64, dtype=bf16, device=DEV), torch.empty(200, 2, 64, dtype=bf16, device=DEV)
    ast.attention(Q, K, V, O)
    first = O.clone()
    ast.attention(Q, K, V, O, lse=lse)
    assert torch.equal(first, O)
    ast.attention_backward(Q, K, V, O, lse, dO, dQ, dK, dV)
    ref, tol = _attention_ref(Q, K, V, [0, 200], 64 ** -0.5, dO)
    for name, t in (("O", O), ("dQ", dQ), ("dK", dK), ("dV", dV)):
        _inside(t, ref[name], tol[name], name)
    with pytest.raises(ast.AsteriaError):
        ast.attention(Q, K, V, torch.empty(1, 4, 64, dtype=bf16, device=DEV).expand(200, 4, 64))


@pytest.mark.parametrize("dtype", [bf16, f32])
def test_attention_keeps_sequences_apart(dtype):
    Q, K, V = (_randn(300, 2, 64, dtype=dtype, seed=i) for i in range(3))
    cu = torch.tensor([0, 100, 220, 300], dtype=torch.int32, device=DEV)
    O, dO = torch.empty_like(Q), _randn(300, 2, 64, dtype=dtype, seed=4)
    lse = torch.empty(2, 300, device=DEV)
    dQ, dK, dV = (torch.empty_like(Q) for _ in range(3))

    def run():
        ast.attention(Q, K, V, O, lse=lse, cu=cu)
        ast.attention_backward(Q, K, V, O, lse, dO, dQ, dK, dV, cu=cu)
        return [t.clone() for t in (O, dQ, dK, dV)]

    clean = run()
    Q[150], K[160], V[170], dO[180] = math.nan, math.inf, -math.inf, math.nan
    for a, b in zip(clean, run()):
        assert torch.equal(a[:100], b[:100]) and torch.equal(a[220:], b[220:])
        assert not bool(torch.isfinite(b[100:220]).all())


def test_attention_scores_of_the_lowest_values():
    # the first keys give scores of minus infinity: they count for nothing
    Q, K, V = (_randn(96, 1, 64, seed=i).abs() for i in range(3))
    K[:40] = -3e38
    Q[:40] = 0.0
    Q[40:] += 1.0
    O, lse = torch.empty_like(Q), torch.empty(1, 96, device=DEV)
    ast.attention(Q, K, V, O, lse=lse, scale=1.0)
    ref, _ = _attention_ref(Q[40:], K[40:], V[40:], [0, 56], 1.0)
    assert bool(torch.isfinite(O).all())
    assert float(torch.linalg.norm(O[40:].double() - ref["O"]) / torch.linalg.norm(ref["O"])) <= 1e-5
    # those rows that see nothing else have equal scores
    mean = V[:40, 0].double().cumsum(0) / torch.arange(1, 41, device=DEV)[:, None]
    assert float(torch.linalg.norm(O[:40, 0].double() - mean) / torch.linalg.norm(mean)) <= 1e-5


@pytest.mark.parametrize("dtype", [bf16, f32])
@pytest.mark.parametrize("heads", [1, 192])
def test_attention_scores_that_rise_and_fall(heads, dtype):
    # no score to go by for several tiles, then scores of -500, then steps up by hundreds and down again, at places within tiles
    n = 700
    Q, K, V = torch.zeros(n, heads, 64, device=DEV), torch.zeros(n, 1, 64, device=DEV), _randn(n, 1, 64, seed=3)
    Q[:, :, 0] = 1.0
    K[:, 0, 0] = -3e38
    K[:, 0, 1] = -3e38
    Q[:, :, 1] = 1.0                                        # the sum of both passes the range: minus infinity
    K[210:, 0, 1] = 0.0
    K[210:, 0, 0] = -500.0
    K[333:, 0, 0] = -100.0
    K[350:, 0, 0] = -480.0
    K[420:, 0, 0] = 300.0
    K[421:, 0, 0] = 304.0
    K[640:, 0, 0] = 295.0
    Q, K, V = Q.to(dtype), K.to(dtype), V.to(dtype)
    O, lse = torch.empty_like(Q), torch.empty(heads, n, device=DEV)
    ast.attention(Q, K, V, O, lse=lse, scale=1.0)
    z = K[210:, 0, 0].double().expand(n - 210, n - 210)
    z = torch.where(torch.ones(n - 210, n - 210, device=DEV).tril().bool(), z, -math.inf)
    ref = torch.softmax(z, 1) @ V[210:, 0].double()
    tol = (U[dtype] * 1.01 + (U[bf16] * 1.01 if dtype == bf16 else 0.0) + 2 * 504 * 4 * F + 1000 * F) * (torch.softmax(z, 1) @ V[210:, 0].double().abs())
    for j in (0, heads - 1):
        _inside(O[210:, j], ref, tol, "O")
        _inside(lse[j, 210:], torch.logsumexp(z, 1), torch.full((n - 210,), 504 * 8 * F, dtype=torch.float64, device=DEV), "lse")


@pytest.mark.parametrize("dtype", [bf16, f32])
@pytest.mark.parametrize("heads", [1, 192])
@pytest.mark.parametrize("step", [4.0, 15.0, 20.0, 45.0, -20.0])
@pytest.mark.parametrize("dim", [64, 33, 120])
def test_attention_scores_in_steps(dim, step, heads, dtype):
    # every 90 keys the scores are a step higher: sums grow by 2^6, 2^21, 2^29, 2^65 at a time
    n = 500
    Q, K, V = torch.zeros(n, heads, dim, device=DEV), torch.zeros(n, 1, dim, device=DEV), _randn(n, 1, dim, seed=3)
    Q[:, :, 0] = 1.0
    K[:, 0, 0] = step * (torch.arange(n, device=DEV) // 90)
    Q, K, V = Q.to(dtype), K.to(dtype), V.to(dtype)
    O, lse = torch.empty_like(Q), torch.empty(heads, n, device=DEV)
    ast.attention(Q, K, V, O, lse=lse, scale=1.0)
    top = abs(step) * 5 + 10
    z = torch.where(torch.ones(n, n, device=DEV).tril().bool(), K[:, 0, 0].double().expand(n, n), -math.inf)
    P = torch.softmax(z, 1)
    # roundings of the result, of P, of the exponents and of the sums
    tol = (U[dtype] * 1.01 + (U[bf16] * 1.01 if dtype == bf16 else 0.0) + 2 * top * 4 * F + 1000 * F) * (P @ V[:, 0].double().abs())
    for j in (0, heads - 1):
        _inside(O[:, j], P @ V[:, 0].double(), tol, "O")
        _inside(lse[j], torch.logsumexp(z, 1), torch.full((n,), top * 8 * F, dtype=torch.float64, device=DEV), "lse")


@pytest.mark.parametrize("dim", [64, 50, 128])
@pytest.mark.parametrize("n,heads", [(3, 1), (20, 1), (20, 400), (64, 1), (64, 400), (300, 1), (300, 200)])
def test_attention_gradients_without_the_rounding_of_o(n, heads, dim):
    # values around 64, where O is stored in steps of 1/2: D from it would be off by a tenth of dP - D.  The gradient of K is free of
    # that at every length, that of Q where a row's keys lie in one tile
    Q, K, dO = _randn(n, heads, dim, dtype=bf16, seed=1), _randn(n, 1, dim, dtype=bf16, seed=2), _randn(n, heads, dim, dtype=bf16, seed=4)
    V = (64 + _randn(n, 1, dim, seed=3)).to(bf16)
    O, lse, dQ, dK, dV = torch.empty_like(Q), torch.empty(heads, n, device=DEV), torch.empty_like(Q), torch.empty_like(K), torch.empty_like(V)
    ast.attention(Q, K, V, O, lse=lse)
    ast.attention_backward(Q, K, V, O, lse, dO, dQ, dK, dV)
    some = sorted({0, heads - 1})
    q, k, v, g, scale = Q.double(), K[:, 0].double().contiguous(), V[:, 0].double().contiguous(), dO.double(), dim ** -0.5
    wantK = torch.zeros_like(k)
    # independent roundings of dS and of the result, each within half a step; sums of dim products of size 64, in fp32, against differences of size 1
    bound = math.sqrt(2) * U[bf16] + 64 * dim * F
    for j in range(heads):
        qj, gj = q[:, j].contiguous(), g[:, j].contiguous()
        z = torch.where(torch.ones(n, n, device=DEV).tril().bool(), scale * torch.mm(qj, k.T.contiguous()), -math.inf)
        P = torch.softmax(z, 1)
        dP = torch.mm(gj, v.T.contiguous())
        dS = P * (dP - (P * dP).sum(1, keepdim=True))
        wantK += scale * torch.mm(dS.T.contiguous(), qj)
        if n <= 64 and j in some:
            want = scale * torch.mm(dS, k)
            assert float(torch.linalg.norm(dQ[:, j].double() - want) / torch.linalg.norm(want)) <= bound
    assert float(torch.linalg.norm(dK[:, 0].double() - wantK) / torch.linalg.norm(wantK)) <= bound


def test_attention_gradient_against_differences():
    # of the forward pass in 64 bits, along one random direction of all three inputs
    Q, K, V, dO = (_randn(130, h, 40, seed=i) for i, h in enumerate((4, 2, 2, 4)))
    O, lse = torch.empty_like(Q), torch.empty(4, 130, device=DEV)
    dQ, dK, dV = torch.empty_like(Q), torch.empty_like(K), torch.empty_like(V)
    ast.attention(Q, K, V, O, lse=lse)
    ast.attention_backward(Q, K, V, O, lse, dO, dQ, dK, dV)
    A, B, C = (_randn(130, h, 40, seed=10 + i).double() for i, h in enumerate((4, 2, 2)))
    t = 1e-4

    def value(s):
        return (_attention_ref(Q.double() + s * A, K.double() + s * B, V.double() + s * C, [0, 130], 40 ** -0.5)[0]["O"] * dO.double()).sum()

    U[torch.float64] = 0.0
    num = float((value(t) - value(-t)) / (2 * t))
    parts = [(dQ, A), (dK, B), (dV, C)]
    got = sum(float((d.double() * x).sum()) for d, x in parts)
    mag = sum(float((d.double().abs() * x.abs()).sum()) for d, x in parts)
    assert abs(num - got) <= mag * (1e-5 + 100 * t * t)


def test_same_bits_every_run_and_in_every_batch():
    Q, K, V, O, lse, dO, dQ, dK, dV, cu = _attention_check([300, 40, 200], 8, 2, 64, bf16)
    again = [torch.empty_like(t) for t in (O, lse, dQ, dK, dV)]
    ast.attention(Q, K, V, again[0], lse=again[1], cu=cu)
    ast.attention_backward(Q, K, V, again[0], again[1], dO, *again[2:], cu=cu)
    for a, b in zip((O, lse, dQ, dK, dV), again):
        assert torch.equal(a, b)
    # the middle sequence alone
    s = slice(300, 340)
    one = [torch.empty_like(t[s].contiguous()) for t in (O, dQ, dK, dV)]
    l1 = torch.empty(8, 40, device=DEV)
    ast.attention(Q[s], K[s], V[s], one[0], lse=l1)
    ast.attention_backward(Q[s], K[s], V[s], one[0], l1, dO[s], *one[1:])
    for a, b in zip((O[s], dQ[s], dK[s], dV[s]), one):
        assert torch.equal(a, b)


def test_captured_graph_follows_new_inputs_offsets_and_random_numbers():
    rows, d = 260, 128
    X, R = _randn(rows, d, dtype=bf16, seed=1), _randn(rows, d, dtype=bf16, seed=2)
    H, Y = torch.empty_like(X), torch.empty_like(X)
    W = _randn(d, dtype=bf16, seed=3)
    state = torch.tensor([1, 1], dtype=torch.int64, device=DEV)
    cu = torch.tensor([0, 100, 260, 260], dtype=torch.int32, device=DEV)
    O, lse = torch.zeros(rows, 2, 64, dtype=bf16, device=DEV), torch.zeros(2, rows, device=DEV)
    dQ, dK, dV = torch.zeros_like(O), torch.zeros(rows, 1, 64, dtype=bf16, device=DEV), torch.zeros(rows, 1, 64, dtype=bf16, device=DEV)
    dX, dR, dW, Z = torch.zeros_like(X), torch.zeros_like(X), torch.zeros_like(W), torch.zeros_like(X)
    outs = (H, Y, O, lse, dQ, dK, dV, dX, dR, dW, Z)
    wn = torch.empty(max(1, ast.rms_norm_backward_workspace_bytes(H, Y, W, None, dX, dR, dW)), dtype=torch.uint8, device=DEV)
    kv = Y.view(rows, 2, 64)[:, :1]
    wa = torch.empty(ast.attention_backward_workspace_bytes(O, kv, kv, O), dtype=torch.uint8, device=DEV)

    def run():
        ast.rms_norm(X, Y, W=W, R=R, H=H, p=0.2, rng=state)
        q, k = Y.view(rows, 2, 64), Y.view(rows, 2, 64)[:, :1]
        ast.attention(q, k, k, O, lse=lse, cu=cu)
        ast.attention_backward(q, k, k, O, lse, O, dQ, dK, dV, cu=cu, ws=wa)
        ast.rms_norm_backward(H, dQ.view(rows, d), W=W, dX=dX, dR=dR, dW=dW, p=0.2, rng=state, ws=wn)
        ast.dropout(dX, Z, 0.4, rng=state)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(4):
        X.copy_(_randn(rows, d, dtype=bf16, seed=20 + i))
        state.copy_(torch.tensor([i, 7 * i]))
        cu.copy_(torch.tensor([0, 50 + i, 120, 250 - i], dtype=torch.int32))
        for t in outs:
            t.zero_()
        run()
        want = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, outs):
            assert torch.equal(a, b)


def test_on_a_stream_of_the_caller():
    side = torch.cuda.Stream()
    X = _randn(2000, 2048, seed=1)
    Y, Z, H = torch.empty_like(X), torch.empty_like(X), torch.empty_like(X)
    dW = torch.empty(2048, device=DEV)
    ast.rms_norm(X, Y, H=H)
    ast.rms_norm_backward(H, Y, dX=Z, dW=dW)
    want = [t.clone() for t in (Y, Z, dW)]
    for t in (Y, Z, dW):
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    ast.rms_norm(X, Y, H=H, stream=side)
    ast.rms_norm_backward(H, Y, dX=Z, dW=dW, stream=side)   # its workspace is allocated on that stream
    junk = [torch.full((1 << 20,), 7.0, device=DEV) for _ in range(8)]
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(want, (Y, Z, dW)):
        assert torch.equal(a, b)
    del junk


def test_two_graphs_on_one_workspace_and_calls_side_by_side():
    # two captured backward passes that share a workspace, replayed in turn, and the same calls on two streams with workspaces of their own
    sets = []
    for i, (heads, kv) in enumerate(((64, 16), (32, 4))):
        Q, K, V, dO = (_randn(700, h, 64, dtype=bf16, seed=10 * i + j) for j, h in enumerate((heads, kv, kv, heads)))
        O, lse = torch.empty_like(Q), torch.empty(heads, 700, device=DEV)
        sets.append((Q, K, V, O, lse, dO, torch.empty_like(Q), torch.empty_like(K), torch.empty_like(V)))
        ast.attention(Q, K, V, O, lse=lse)
    ws = torch.empty(max(ast.attention_backward_workspace_bytes(*s[:5]) for s in sets), dtype=torch.uint8, device=DEV)
    want, graphs = [], []
    for s in sets:
        ast.attention_backward(*s)
        want.append([t.clone() for t in s[6:]])
    torch.cuda.synchronize()
    for s in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ast.attention_backward(*s, ws=ws)
        graphs.append(g)
    for turn in range(3):
        for s in sets:
            for t in s[6:]:
                t.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for s, w in zip(sets, want):
            for a, b in zip(s[6:], w):
                assert torch.equal(a, b)
    streams = [torch.cuda.Stream() for _ in sets]
    for s in sets:
        for t in s[6:]:
            t.zero_()
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    for turn in range(3):
        for s, st in zip(sets, streams):
            ast.attention_backward(*s, stream=st)
    torch.cuda.synchronize()
    for s, w in zip(sets, want):
        for a, b in zip(s[6:], w):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [bf16, f32])
def test_attention_offsets_outside_the_rows_are_brought_inside(dtype):
    Q, K, V = (_randn(200, 2, 64, dtype=dtype, seed=i) for i in range(3))
    O, P = torch.full_like(Q, 9.0), torch.full_like(Q, 9.0)
    ast.attention(Q, K, V, O, cu=torch.tensor([-50, 90, 90, 1 << 30], dtype=torch.int32, device=DEV))
    ast.attention(Q, K, V, P, cu=torch.tensor([0, 90, 90, 200], dtype=torch.int32, device=DEV))
    assert torch.equal(O, P)


def test_attention_rows_far_into_a_large_array():
    # element offsets beyond 2^32: rows 3 apart by strides of a wide buffer, read through registers (the direct loads take 31 bits)
    ld = 1 << 25
    buf = torch.zeros(200 * ld, dtype=bf16, device=DEV)
    view = lambda at, h: torch.as_strided(buf, (200, h, 64), (ld, 64, 1), at)
    Q, K, V = view(0, 2), view(4096, 2), view(8192, 2)
    for i, t in enumerate((Q, K, V)):
        t.copy_(_randn(200, 2, 64, dtype=bf16, seed=i))
    dO = _randn(200, 2, 64, dtype=bf16, seed=5)
    got, want = [], []
    for q, k, v, like, out in ((Q, K, V, lambda at: view(at, 2), got), (Q.contiguous(), K.contiguous(), V.contiguous(), lambda at: torch.empty_like(dO), want)):
        O, lse = like(12288), torch.empty(2, 200, device=DEV)
        dQ, dK, dV = like(16384), like(20480), like(24576)
        ast.attention(q, k, v, O, lse=lse)
        ast.attention_backward(q, k, v, O, lse, dO, dQ, dK, dV)
        out += [O, lse, dQ, dK, dV]
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_norm_and_dropout_rows_far_into_a_large_array():
    ld = (1 << 30) + 8
    buf = torch.zeros(4 * ld + 4096, device=DEV)
    X = torch.as_strided(buf, (5, 600), (ld, 1), 0)
    Y = torch.as_strided(buf, (5, 600), (ld, 1), 1024)
    x = _randn(5, 600, seed=1)
    X.copy_(x)
    y = torch.empty_like(x)
    ast.rms_norm(X, Y, p=0.5, seed=2)
    ast.rms_norm(x, y, p=0.5, seed=2)
    assert torch.equal(Y, y)
    ast.dropout(X, Y, 0.5, seed=2)
    ast.dropout(x, y, 0.5, seed=2)
    assert torch.equal(Y, y)
