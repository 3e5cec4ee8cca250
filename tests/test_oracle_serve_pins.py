"""Pins for the oracle's norm and 8-bit experts: closed forms, torch autograd, central differences, and what 8 bits may
cost.  No GPU is used."""
import numpy as np
import pytest
import torch

import oracle

EPS = 1e-6


def _case(T=5, d=24, seed=0):
    g = np.random.default_rng(seed)
    return g.standard_normal((T, d)), 1.0 + 0.2 * g.standard_normal(d), g.standard_normal((T, d)), g.standard_normal((T, d))


def test_norm_closed_forms():
    h, gain, _, _ = _case()
    y, r = oracle.add_rmsnorm(h, np.ones(24), 0.0)
    np.testing.assert_allclose((y * y).mean(axis=1), 1.0, rtol=1e-14)            # unit mean square
    np.testing.assert_allclose(oracle.add_rmsnorm(-3.0 * h, gain, 0.0)[0], -oracle.add_rmsnorm(h, gain, 0.0)[0], rtol=1e-13)
    assert np.all(oracle.add_rmsnorm(np.zeros((2, 7)), np.ones(7), EPS)[0] == 0)
    np.testing.assert_allclose(oracle.add_rmsnorm(np.full((1, 5), 2.0), np.ones(5), 0.0)[1], 0.5, rtol=1e-15)


def test_norm_backward_is_the_formulas_gradient():
    h, gain, dy, dh = _case(seed=1)
    th, tg = (torch.tensor(a, dtype=torch.float64, requires_grad=True) for a in (h, gain))
    y = th / torch.sqrt((th * th).mean(1, keepdim=True) + EPS) * tg
    ((y * torch.tensor(dy)).sum() + (th * torch.tensor(dh)).sum()).backward()
    dx, dgain = oracle.add_rmsnorm_bwd(dy, dh, h, gain, EPS)
    np.testing.assert_allclose(dx, th.grad.numpy(), rtol=1e-12, atol=1e-13)
    np.testing.assert_allclose(dgain, tg.grad.numpy(), rtol=1e-12, atol=1e-13)


def test_norm_backward_against_differences():
    h, gain, dy, _ = _case(T=2, d=7, seed=2)
    dx, dgain = oracle.add_rmsnorm_bwd(dy, None, h, gain, EPS)
    step = 1e-6

    def loss(a, b):
        return (oracle.add_rmsnorm(a, b, EPS)[0] * dy).sum()

    for i in np.ndindex(h.shape):
        e = np.zeros_like(h)
        e[i] = step
        assert abs((loss(h + e, gain) - loss(h - e, gain)) / (2 * step) - dx[i]) < 1e-8
    for i in range(7):
        e = np.zeros(7)
        e[i] = step
        assert abs((loss(h, gain + e) - loss(h, gain - e)) / (2 * step) - dgain[i]) < 1e-8
    assert abs((oracle.add_rmsnorm_bwd(dy, None, h, gain, 0.0)[0] * h).sum()) < 1e-12   # scale invariance: dx is orthogonal to h


def test_quantised_rows():
    v = np.random.default_rng(3).standard_normal((6, 50))
    q, s = oracle.quantize_rows(v)
    assert np.abs(q).max(axis=1).tolist() == [127] * 6 and np.abs(q * s[:, None] - v).max() <= 0.5 * s.max()
    assert oracle.quantize_rows(np.array([[0.5, 1.5, 2.5, 127.0]]))[0].tolist() == [[0, 2, 2, 127]]      # ties to even
    assert oracle.quantize_rows(np.zeros((1, 3)))[1][0] == 0.0
    # a row's scale does not change its integers; float32 steps give the same ones away from a tie
    assert np.array_equal(oracle.quantize_rows(v * 4.0)[0], q)
    qf, m = oracle.quantize_rows_f32(v)
    away = np.abs(np.abs(v / s[:, None] % 1.0) - 0.5) > 1e-4
    assert np.array_equal(qf[away], q[away]) and np.array_equal(m, np.abs(v.astype(np.float32)).max(axis=1))


@pytest.mark.parametrize("rows", [[3, 0, 1, 6], [0, 0, 0, 1]])
def test_experts_on_exact_integers_are_the_float_experts(rows):
    """The result follows expert_ffn_fwd on the values that integers and scales stand for, up to what quantising the
    activation costs: half a step of each row, through the down projection."""
    g = np.random.default_rng(5)
    E, d, f, B = 4, 12, 9, sum(rows)
    off = np.concatenate([[0], np.cumsum(rows)])
    xq, w = g.integers(-127, 128, (B, d)), [g.integers(-127, 128, s) for s in ((E, f, d), (E, f, d), (E, d, f))]
    xs, ws = g.uniform(0.01, 0.02, B), [g.uniform(0.001, 0.002, s) for s in ((E, f), (E, f), (E, d))]
    Y, A, AQ, AS = oracle.expert_ffn_q8(xq, xs, np.arange(B), off, w[0], ws[0], w[1], ws[1], w[2], ws[2])
    values = [(a * s[:, :, None]).transpose(0, 2, 1) for a, s in zip(w, ws)]
    ref_Y, G, U = oracle.expert_ffn_fwd(xq * xs[:, None], off, *values)
    ref_A = oracle.silu(G) * U
    np.testing.assert_allclose(A, ref_A, rtol=1e-12, atol=1e-14)
    e_of = np.repeat(np.arange(E), rows)
    reach = 0.5 * AS[:, None] * np.abs(values[2][e_of]).sum(axis=1)
    assert np.all(np.abs(Y - ref_Y) <= reach * (1 + 1e-9))
