"""Pins for the oracle's layer normalisation, 8-bit checkpoints and products by groups of rows, CPU only: torch's autograd in
float64, finite differences, the formats' own invariants."""
import numpy as np
import pytest
import torch

import oracle


def test_layer_norm_matches_autograd_and_differences():
    rng = np.random.default_rng(1)
    x, gy = rng.standard_normal((40, 9)) * 3.0 + 5.0, rng.standard_normal((40, 9))
    gamma, beta = rng.standard_normal(9), rng.standard_normal(9)
    xt, gt, bt = (torch.tensor(v, requires_grad=True) for v in (x, gamma, beta))
    yt = torch.nn.functional.layer_norm(xt, (9,), gt, bt, eps=1e-5)
    (yt * torch.tensor(gy)).sum().backward()
    y, mean, rstd, xhat = oracle.ln_forward(x, 1e-5, gamma, beta)
    gx, dgamma, dbeta = oracle.ln_backward(xhat, rstd, gy, gamma)
    for got, want in ((y, yt.detach()), (gx, xt.grad), (dgamma, gt.grad), (dbeta, bt.grad)):
        assert np.allclose(got, want.numpy(), rtol=1e-10, atol=1e-12)
    # a central difference of step t is off by t^2 times the third derivative and 1e-16 / t of cancellation
    i, c, t = 7, 3, 1e-5
    up, down = x.copy(), x.copy()
    up[i, c] += t
    down[i, c] -= t
    slope = ((oracle.ln_forward(up, 1e-5, gamma, beta)[0] - oracle.ln_forward(down, 1e-5, gamma, beta)[0]) * gy).sum() / (2 * t)
    assert abs(slope - gx[i, c]) < 1e-6


def test_layer_norm_of_a_constant_row_is_beta():
    y, mean, rstd, xhat = oracle.ln_forward(np.full((2, 5), 3.0), 1e-5, np.full(5, 2.0), np.arange(5.0))
    assert np.array_equal(y, np.tile(np.arange(5.0), (2, 1))) and np.array_equal(xhat, np.zeros((2, 5)))


@pytest.mark.parametrize("c", [1, 31, 32, 33, 100])
def test_checkpoint_comes_back_within_a_step_and_repacks_to_itself(c):
    rng = np.random.default_rng(c)
    x = (rng.standard_normal((50, c)) * np.exp(rng.standard_normal((50, 1)) * 20)).astype(np.float32)
    codes, scales = oracle.ckpt8_pack(x)
    v = oracle.ckpt8_unpack(codes, scales)
    step = np.repeat(np.ldexp(1.0, scales.astype(int) - 127), 32, axis=1)[:, :c]
    top = np.stack([np.abs(x[:, 32 * b:32 * b + 32]).max(axis=1) for b in range(scales.shape[1])], axis=1)
    assert (np.ldexp(1.0, scales.astype(int) - 127) <= top.astype(np.float64) / 64).all()
    assert (np.abs(v - x) <= step).all()
    assert (np.abs(v - x)[np.abs(codes) < 127] <= step[np.abs(codes) < 127] / 2).all()
    again = oracle.ckpt8_pack(v)   # the largest value may have moved to a power of two above, never by more
    assert (np.abs(oracle.ckpt8_unpack(*again) - v) <= step).all()


def test_checkpoint_of_special_values():
    big, tiny = np.finfo(np.float32).max, np.float32(1e-45)
    x = np.zeros((6, 40), np.float32)
    x[1, 0], x[2, 33], x[3, 5], x[4, 0], x[5, 0] = np.inf, np.nan, -big, tiny, -0.0
    codes, scales = oracle.ckpt8_pack(x)
    assert scales[0].tolist() == [0, 0] and scales[1].tolist() == [255, 0] and scales[2].tolist() == [0, 255]
    assert scales[3, 0] == 127 - 6 + 127 and codes[3, 5] == -127 and scales[4, 0] == 1 and codes[4, 0] == 0 and scales[5, 0] == 0
    v = oracle.ckpt8_unpack(codes, scales)
    assert np.isnan(v[1, :32]).all() and (v[1, 32:] == 0).all() and np.isnan(v[2, 32:]).all() and np.isfinite(v[3]).all()


def test_grouped_product_matches_autograd():
    rng = np.random.default_rng(2)
    h, w, dz = rng.standard_normal((30, 4)), rng.standard_normal((5, 4, 3)), rng.standard_normal((30, 3))
    offsets = np.array([2, 2, 10, 11, 11, 27])
    ht, wt = torch.tensor(h, requires_grad=True), torch.tensor(w, requires_grad=True)
    zt = torch.cat([torch.zeros(2, 3, dtype=torch.float64)] + [ht[a:b] @ wt[g] for g, (a, b) in enumerate(zip(offsets, offsets[1:]))] +
                   [torch.zeros(3, 3, dtype=torch.float64)])
    (zt * torch.tensor(dz)).sum().backward()
    dh, dw = oracle.grouped_linear_bwd(h, w, offsets, dz)
    assert np.allclose(oracle.grouped_linear(h, w, offsets), zt.detach().numpy(), rtol=1e-12, atol=1e-14)
    assert np.allclose(dh, ht.grad.numpy(), rtol=1e-12, atol=1e-14) and np.allclose(dw, wt.grad.numpy(), rtol=1e-12, atol=1e-14)


def test_offsets_that_descend_or_leave_the_array():
    assert oracle.group_rows([-3, 5, 2, 99], 10) == [(0, 5), (5, 5), (5, 10)]
