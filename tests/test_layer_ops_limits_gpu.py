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

