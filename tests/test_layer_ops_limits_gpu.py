"""Norm and attention where their definitions are easily missed: values far from zero mean, sequences of one row, elements that a mask
hides, values next to a border of their type.  References in 64 bits; U[t] = eps / 2 of a type, F = 2^-24 a rounding of an fp32 sum."""
import math

import pytest
import torch

import paper_2605_16184_amd as ast

pytestmark = pytest.mark.gpu
DEV = "cuda"
F = 2.0 ** -24
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
f32, bf16 = torch.float32, torch.bfloat16


def _randn(*shape, dtype=f32, seed=0, mean=0.0):
    g = torch.Generator(device=DEV).manual_seed(seed * 104729 + 29)
    return (mean + torch.randn(*shape, generator=g, device=DEV)).to(dtype)


def _offsets(lens, lead=0):
    cu = [lead]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu, torch.tensor(cu, dtype=torch.int32, device=DEV)


def _train(Q, K, V, dO, cu=None, scale=None):
    O, lse = torch.full_like(Q, 9.0), torch.full((Q.shape[1], Q.shape[0]), 9.0, device=DEV)
    dQ, dK, dV = torch.full_like(Q, 9.0), torch.full_like(K, 9.0), torch.full_like(V, 9.0)
    ast.attention(Q, K, V, O, lse=lse, cu=cu, scale=scale)
    ast.attention_backward(Q, K, V, O, lse, dO, dQ, dK, dV, cu=cu, scale=scale)
    return O, lse, dQ, dK, dV


# ---- sequences of one row ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [bf16, f32])
@pytest.mark.parametrize("heads,kv_heads,dim", [(1, 1, 64), (32, 4, 80), (6, 2, 33)])
@pytest.mark.parametrize("lens", [[1], [0, 1, 0, 1, 1], [1] * 600])
def test_sequences_of_one_row_have_no_gradient_through_the_softmax(lens, heads, kv_heads, dim, dtype):
    cu, dcu = _offsets(lens)
    total = cu[-1]
    Q, dO = _randn(total, heads, dim, dtype=dtype, seed=1), _randn(total, heads, dim, dtype=dtype, seed=4)
    K, V = _randn(total, kv_heads, dim, dtype=dtype, seed=2, mean=3.0), _randn(total, kv_heads, dim, dtype=dtype, seed=3, mean=3.0)
    O, lse, dQ, dK, dV = _train(Q, K, V, dO, dcu)
    group = heads // kv_heads
    k, v = K.double().repeat_interleave(group, 1), V.double().repeat_interleave(group, 1)
    assert not bool(dQ.any()) and not bool(dK.any())
    # P = 1: forward by a quotient of two equal numbers (six products of fp32 terms, two roundings each, the reciprocal and its product),
    # backward by an exponent of z - lse: z twice, a sum of dim products, and its factor.  In bf16 an operand P near 1 is 1
    z = dim ** -0.5 * (Q.double().abs() * k.abs()).sum(2)
    ez = ((dim + 4) * z + 4 * (1 + z) + 8) * F
    if dtype == bf16:
        assert torch.equal(O.double(), v) and float(ez.max()) < 2.0 ** -9
        ez = 0 * ez
    assert bool(((O.double() - v).abs() <= 14 * F * 1.01 * v.abs()).all())
    sums = lambda t: t.view(total, kv_heads, group, dim).sum(2)
    want, size, off = sums(dO.double()), sums(dO.double().abs()), sums(2 * ez[:, :, None] * dO.double().abs())
    assert bool(((dV.double() - want).abs() <= U[dtype] * 1.01 * want.abs() + (2 * 6 * group + 1) * F * size + off).all())


# ---- values far from zero mean ----------------------------------------------------------------------
def _gradients(Q, K, V, dO, cu, scale, heads):
    """dQ of some heads and dK, dV in 64 bits, and what independent roundings, each of at most half a step, change of dQ and dK in the
    norm: dS before its sum is taken out (off by P times the rounding of O), P beside it, the results, and fp32 sums of dim products."""
    group, dim = Q.shape[1] // K.shape[1], Q.shape[2]
    ref = {"dQ": {}, "dK": torch.zeros(K.shape, dtype=torch.float64, device=DEV), "dV": torch.zeros(V.shape, dtype=torch.float64, device=DEV)}
    off = {"dQ": {}, "dK": torch.zeros(K.shape, dtype=torch.float64, device=DEV)}         # squares
    mm = lambda a, b: torch.mm(a.contiguous(), b.contiguous())
    u = U[bf16] if Q.dtype == bf16 else 0.0
    for j in range(Q.shape[1]):
        jk = j // group
        if j in heads:
            ref["dQ"][j] = torch.zeros(Q.shape[0], dim, dtype=torch.float64, device=DEV)
            off["dQ"][j] = torch.zeros(Q.shape[0], dim, dtype=torch.float64, device=DEV)
        for s, e in zip(cu[:-1], cu[1:]):
            n = e - s
            if n == 0:
                continue
            q, k, v, g = Q[s:e, j].double(), K[s:e, jk].double(), V[s:e, jk].double(), dO[s:e, j].double()
            seen = torch.ones(n, n, device=DEV).tril().bool()
            z = torch.where(seen, scale * mm(q, k.T), -math.inf)
            P = torch.softmax(z, 1)
            dP = mm(g, v.T)
            dS = P * (dP - (P * dP).sum(1, keepdim=True))
            by_o = (g.abs() * mm(P, v).abs() * U[Q.dtype]).sum(1, keepdim=True)            # of D, by O as stored
            # P by its exponent and dP, D: sums of dim products, sqrt(dim) F of their size in the mean
            ez = torch.where(seen, scale * mm(q.abs(), k.abs().T), 0.0).amax(1, keepdim=True) * math.sqrt(dim) * F + 4 * F
            ed = math.sqrt(dim) * F * (mm(g.abs(), v.abs().T) + (g.abs() * mm(P, v.abs())).sum(1, keepdim=True))
            each = (u * (dS.abs() + 2 * P * by_o)).square() + (2 * ez * dS.abs() + 2 * P * ed).square()
            ref["dK"][s:e, jk] += scale * mm(dS.T, q)
            ref["dV"][s:e, jk] += mm(P.T, g)
            off["dK"][s:e, jk] += scale ** 2 * mm(each.T, q.square())
            if j in heads:
                ref["dQ"][j][s:e] = scale * mm(dS, k)
                off["dQ"][j][s:e] = scale ** 2 * mm(each, k.square()) + (U[Q.dtype] * ref["dQ"][j][s:e]).square()
    off["dK"] += (U[Q.dtype] * ref["dK"]).square()
    return ref, off


@pytest.mark.parametrize("dtype", [bf16, f32])
@pytest.mark.parametrize("lens,heads,kv_heads", [([300], 200, 2), ([129, 0, 700, 65, 1], 2, 1), ([129, 0, 700, 65, 1], 96, 4), ([1500], 40, 8)])
@pytest.mark.parametrize("dim", [64, 50, 96, 128])
@pytest.mark.parametrize("mean_v,mean_k", [(1.0, 0.0), (64.0, 0.0), (1.0, 4.0)])
def test_gradients_do_not_carry_the_rounding_of_o(mean_v, mean_k, dim, lens, heads, kv_heads, dtype):
    cu, dcu = _offsets(lens)
    total = cu[-1]
    Q, dO = _randn(total, heads, dim, dtype=dtype, seed=1), _randn(total, heads, dim, dtype=dtype, seed=4)
    K, V = _randn(total, kv_heads, dim, dtype=dtype, seed=2, mean=mean_k), _randn(total, kv_heads, dim, dtype=dtype, seed=3, mean=mean_v)
    _, _, dQ, dK, dV = _train(Q, K, V, dO, dcu)
    some = sorted({0, heads // 2, heads - 1})
    ref, off = _gradients(Q, K, V, dO, cu, dim ** -0.5, some)
    for j in some:
        for s, e in zip(cu[:-1], cu[1:]):                    # the first tile's rows and the later ones apart
            for a, b in ((s, min(e, s + 64)), (s + 64, e)):
                if b > a + 1:
                    err = float(torch.linalg.norm(dQ[a:b, j].double() - ref["dQ"][j][a:b]))
                    assert err <= math.sqrt(float(off["dQ"][j][a:b].sum())), (j, a, b, err / float(torch.linalg.norm(ref["dQ"][j][a:b])))
    assert float(torch.linalg.norm(dK.double() - ref["dK"])) <= math.sqrt(float(off["dK"].sum()))
    assert float(torch.linalg.norm(dV.double() - ref["dV"]) / torch.linalg.norm(ref["dV"])) <= (math.sqrt(2) * U[bf16] if dtype == bf16 else 1e-5)


# ---- elements that the mask hides ----------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [bf16, f32])
@pytest.mark.parametrize("dim", [64, 40, 80, 128, 127])
@pytest.mark.parametrize("heads", [2, 200])                 # four wavefronts (two) for the same rows; one wavefront for every 32 rows
@pytest.mark.parametrize("at", [31, 32, 63, 127, 191, 300])
def test_what_the_mask_hides_reaches_no_row_32_or_more_before_it(at, heads, dim, dtype):
    n = 340
    cu, dcu = _offsets([n, 3], lead=5)
    s, e, r = cu[0], cu[1], cu[0] + at
    block = s + at // 32 * 32                               # rows before it see nothing of row r's block of 32
    Q, dO = _randn(cu[-1], heads, dim, dtype=dtype, seed=1), _randn(cu[-1], heads, dim, dtype=dtype, seed=4)
    K, V = _randn(cu[-1], 1, dim, dtype=dtype, seed=2), _randn(cu[-1], 1, dim, dtype=dtype, seed=3)
    O, lse, dQ, dK, dV = _train(Q, K, V, dO, dcu)
    # of an exponent and of a sum of n: twice the dim products of a score, the sum's additions, the logarithm
    z = dim ** -0.5 * float(torch.linalg.norm(Q.double(), dim=2).max() * torch.linalg.norm(K.double(), dim=2).max())
    ez = ((2 * dim + 4) * z + n + 8 + 2 * float(lse[:, s:e].abs().max())) * F
    largest = float(V.abs().max())
    for bad in (math.inf, -math.inf, math.nan):
        for t in (K, V):
            keep = t[r].clone()
            t[r, 0, dim // 2] = bad
            o, l, dq = torch.empty_like(O), torch.empty_like(lse), torch.empty_like(dQ)
            ast.attention(Q, K, V, o, lse=l, cu=dcu)
            ast.attention_backward(Q, K, V, O, lse, dO, dq, torch.empty_like(dK), torch.empty_like(dV), cu=dcu)
            t[r] = keep
            assert torch.equal(dq[s:block], dQ[s:block])
            # 128 rows share a workgroup, which in bf16 counts its exponents from other maxima where a sum is no number: roundings only
            tile = block if dtype == f32 else s + at // 128 * 128
            assert torch.equal(o[s:tile], O[s:tile]) and torch.equal(l[:, s:tile], lse[:, s:tile])
            off = (o[tile:block].double() - O[tile:block].double()).abs()
            assert bool((off <= 2 * (2.02 * U[bf16] + 2 * ez) * largest).all())
            assert bool(((l[:, tile:r] - lse[:, tile:r]).abs() <= 2 * ez).all())
            if t is V or math.isnan(bad):                   # a score of minus infinity only takes the key away
                assert not bool(torch.isfinite(o[r]).all())
            assert torch.equal(o[e:cu[-1]], O[e:cu[-1]]) and torch.equal(dq[e:cu[-1]], dQ[e:cu[-1]])
        for t in (Q, dO):
            keep = t[r].clone()
            t[r, 0, dim // 2] = bad
            dq, dk, dv = torch.empty_like(dQ), torch.empty_like(dK), torch.empty_like(dV)
            ast.attention_backward(Q, K, V, O, lse, dO, dq, dk, dv, cu=dcu)
            t[r] = keep
            assert torch.equal(dq[s:r], dQ[s:r]) and torch.equal(dq[r + 1:cu[-1]], dQ[r + 1:cu[-1]])
            for a, b in ((dk, dK), (dv, dV)):
                assert torch.equal(a[block + 32:cu[-1]], b[block + 32:cu[-1]])


# ---- 8-bit output ------------------------------------------------------------------------------------
@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("rows,cols,dtype", [(4096, 2048, bf16), (3000, 777, f32), (5000, 100, bf16), (300, 5632, f32)])
def test_norm_rounds_quotients_to_8_bits(rows, cols, group, dtype):
    # Y is the nearest 8-bit value, ties to even, of the fp32 quotient of y (a call with fp32 output gives it) and the scale
    e4m3 = torch.float8_e4m3fn
    X, R, W = _randn(rows, cols, dtype=dtype, seed=1), _randn(rows, cols, dtype=dtype, seed=2), _randn(cols, seed=3)
    y, Y = torch.empty(rows, cols, device=DEV), torch.empty(rows, cols, dtype=torch.uint8, device=DEV).view(e4m3)
    S = torch.empty(rows, -(-cols // 128) if group else 1, device=DEV)
    W[cols // 2:] *= 1e-32                                  # groups next to the smallest scale
    X[5], R[5] = X[5] * 2.0 ** -90, 0                       # and a row, with 1 / sqrt(eps) = 1000
    ast.rms_norm(X, y, W=W, R=R)
    ast.rms_norm(X, Y, W=W, R=R, scale=S, group=group)
    spread = S.repeat_interleave(group or cols, 1)[:, :cols]
    # on the host: the quotient of two fp32 numbers in 64 bits rounds to the same 24 bits, and those to 8 bits by comparison with the
    # neighbours' middle
    q = (y.cpu().double() / spread.cpu().double()).float().double()
    step = torch.exp2(torch.floor(torch.log2(q.abs().clamp_min(2.0 ** -6))) - 3)
    want = torch.clamp(torch.round(q / step) * step, -448.0, 448.0)
    assert bool((Y.cpu().float().double() == want).all())
    assert int((S <= 2.0 ** -80).sum()) >= 1


# ---- fp32's lowest and largest numbers ------------------------------------------------------------------
@pytest.mark.parametrize("heads", [2, 200])
@pytest.mark.parametrize("dim", [64, 50, 128])
@pytest.mark.parametrize("lowest", [torch.finfo(f32).min, -3.397e38, -3.39e38])
def test_attention_in_fp32_with_numbers_that_round_to_no_bf16(lowest, dim, heads):
    # keys that are so far down that they count for nothing: results are those of the rows without them
    n, hidden = 300, [1, 40, 70, 128, 200]
    Q, K, V, dO = (_randn(n, h, dim, seed=i) for i, h in enumerate((heads, 1, 1, heads)))
    Q[:, :, 0] = 1.0
    K[hidden] = 0.0
    K[hidden, 0, 0] = lowest
    keep = [i for i in range(n) if i not in hidden]
    O, lse, dQ, dK, dV = _train(Q, K, V, dO, scale=1.0)
    q, k, v, z0 = Q.double(), K[keep].double(), V[keep].double(), torch.ones(len(keep), len(keep), device=DEV).tril().bool()
    for j in (0, heads - 1):
        z = torch.where(z0, torch.mm(q[keep, j].contiguous(), k[:, 0].T.contiguous()), -math.inf)
        P = torch.softmax(z, 1)
        ref = torch.mm(P, v[:, 0].contiguous())
        # exponents twice, dim products each, and sums of n
        e = float(torch.where(z0, torch.mm(q[keep, j].abs().contiguous(), k[:, 0].abs().T.contiguous()), 0.0).max()) * (dim + 4) * F
        tol = (2 * (e + 4 * F) + (2 * n + 10) * F) * torch.mm(P, v[:, 0].abs()) + F * ref.abs()
        assert bool(((O[keep, j].double() - ref).abs() <= tol).all())
        want = torch.logsumexp(z, 1)
        assert bool(((lse[j, keep].double() - want).abs() <= e + (n + 8) * F + 2 * F * want.abs()).all())
    # the largest and lowest value of one key comes out as it is, in sequences of one row
    cu = torch.arange(n + 1, dtype=torch.int32, device=DEV)
    big = V.clone()
    big[:, 0, 0], big[:, 0, 1] = torch.finfo(f32).max, lowest
    ast.attention(torch.zeros_like(Q), K, big, O, cu=cu)
    assert torch.equal(O, big.expand(n, heads, dim))
    # finite gradients, none to keys that count for nothing
    assert all(bool(torch.isfinite(t).all()) for t in (dQ, dK, dV)) and not bool(dK[hidden].any()) and not bool(dV[hidden].any())


@pytest.mark.parametrize("exponent", [-100, -115, -126, -133])
@pytest.mark.parametrize("dtype", [bf16, f32])
def test_attention_with_the_smallest_numbers(exponent, dtype):
    # sequences of one row give V back: fp32 as three bf16 terms, of which the last ends at bf16's smallest step, 2^-133
    n = 64
    V = ((1 + torch.rand(n, 2, 64, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)) * 2.0 ** exponent).to(dtype)
    Z, O = torch.zeros_like(V), torch.empty_like(V)
    ast.attention(Z, Z, V, O, cu=torch.arange(n + 1, dtype=torch.int32, device=DEV))
    assert float((O.double() - V.double()).abs().max()) <= (0.0 if dtype == bf16 else 2.0 ** -134)


@pytest.mark.parametrize("group", [0, 128])
def test_norm_in_8_bits_keeps_the_sign_of_zero(group):
    X, W = _randn(40, 300, seed=1), _randn(300, seed=2)
    X[:, ::3] = 0.0
    X[:, 1::7] = 0.0                                        # times weights of both signs
    y, Y = torch.empty_like(X), torch.empty(40, 300, dtype=torch.uint8, device=DEV)
    S = torch.empty(40, 3 if group else 1, device=DEV)
    ast.rms_norm(X, y, W=W)
    ast.rms_norm(X, Y.view(torch.float8_e4m3fn), W=W, scale=S, group=group)
    assert torch.equal(Y >= 128, torch.signbit(y)) and bool((torch.signbit(y) & (y == 0)).any())


def test_norm_of_rows_that_hold_no_number_or_pass_the_range():
    X = _randn(8, 300, seed=1)
    clean, S0 = torch.empty(8, 300, device=DEV).to(torch.float8_e4m3fn), torch.empty(8, 3, device=DEV)
    ast.rms_norm(X, clean, scale=S0, group=128)
    X[1, 5], X[3, 299], X[5] = math.nan, -math.inf, 1e20
    Y, S, Z = torch.empty_like(clean), torch.empty_like(S0), torch.empty(8, 300, device=DEV)
    ast.rms_norm(X, Y, scale=S, group=128)
    ast.rms_norm(X, Z)
    same = [0, 2, 4, 6, 7]
    assert torch.equal(Y[same].view(torch.uint8), clean[same].view(torch.uint8)) and torch.equal(S[same], S0[same])
    for r in (1, 3):
        assert not bool(torch.isfinite(Y[r].float()).all()) and not bool(torch.isfinite(Z[r]).all())
    assert not bool(Y[5].float().any()) and not bool(Z[5].any())
