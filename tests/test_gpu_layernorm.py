"""GPU parity of the layer normalisation, forward and backward, from the rows and from their 8-bit checkpoint, with the float64
oracle: every width class of the kernels, offsets that cancel, special values, in place, under capture, on another stream.

Tolerances.  u = 2^-24 is half a unit of a float32.  A sum of C terms that passes k additions one after the other is off by at
most k u times the sum of the magnitudes, and k is what a lane adds up itself plus the steps that join the lanes: at most
`links(C)`.  A bf16 result is rounded once more: half a step, 2^-8 of the value."""
import numpy as np
import pytest
import torch

import oracle

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24
WIDTHS = [1, 3, 4, 5, 8, 16, 20, 31, 32, 33, 47, 64, 72, 96, 100, 128, 200, 256, 264, 512, 520, 1000, 1024, 1025, 2048, 2056, 5000]


def links(c):
    return (c + 3) // 4 + 16 if c <= 128 else max(64, c // 32 * 2) + 16


def within(got, want, tol, what):
    err = np.abs(np.asarray(got, np.float64) - want)
    both_nan = np.isnan(got) & np.isnan(want)
    bad = ~((err <= tol) | both_nan)
    assert not bad.any(), (what, int(bad.sum()), float(np.nanmax(err / np.broadcast_to(tol, err.shape))))


def half(dt, v):
    return 2.0 ** -8 * np.abs(v) + 2.0 ** -134 if dt == "bf16" else 0.0


def np64(t):
    return t.detach().double().cpu().numpy()


def problem(n, c, dt, offset, seed, affine=True):
    gen = torch.Generator().manual_seed(seed)
    x = ((torch.randn(n, c, generator=gen) * torch.exp(torch.randn(n, 1, generator=gen)) + offset)).to(DT[dt])
    gy = torch.randn(n, c, generator=gen).to(DT[dt])
    gamma = torch.randn(c, generator=gen) if affine else None
    beta = torch.randn(c, generator=gen) if affine else None
    return [t.cuda() if t is not None else None for t in (x, gy, gamma, beta)]


def forward_bounds(x, gamma, beta, eps):
    """(y, mean, rstd, xhat) of the oracle and their bounds: an error dm of the mean moves xhat by dm rstd; the deviations'
    rounding and the sum of their squares move rstd by (links + 4) u of itself, and the mean's error by (dm rstd)^2 / 2 more."""
    y, mean, rstd, xhat = oracle.ln_forward(x, eps, gamma, beta)
    k = links(x.shape[1])
    dm = (k + 2) * U * np.abs(x).mean(axis=1)
    # x - mean is rounded to float32 once: u of its size
    slack = dm + U * (np.abs(x).max(axis=1) + np.abs(mean))
    rel = (k + 6) * U + (slack * rstd) ** 2
    dx = slack[:, None] * rstd[:, None] + (rel[:, None] + 3 * U) * np.abs(xhat)
    ga = 1.0 if gamma is None else np.abs(gamma)
    be = 0.0 if beta is None else np.abs(beta)
    return (y, mean, rstd, xhat), (dx * ga + 2 * U * (np.abs(xhat) * ga + be), dm + U * np.abs(mean), rel * rstd + 2 * U * rstd, dx)


@pytest.mark.parametrize("c", WIDTHS)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,offset", [(1, 0.0), (77, 3.0), (1500, 100.0)])
def test_forward(n, c, dt, offset):
    from paper_2111_06483_b200 import api
    x, _, gamma, beta = problem(n, c, dt, offset, 7 * n + c, affine=n != 1)
    y, (mean, rstd) = api.ln_forward(x, 1e-5, gamma, beta)
    assert y.dtype == x.dtype and mean.shape == (n,) and rstd.shape == (n,)
    want, tol = forward_bounds(np64(x), None if gamma is None else np64(gamma), None if beta is None else np64(beta), 1e-5)
    within(np64(mean), want[1], tol[1], "mean")
    within(np64(rstd), want[2], tol[2], "rstd")
    within(np64(y), want[0], tol[0] + half(dt, np.abs(want[0]) + tol[0]), "y")


@pytest.mark.parametrize("c", WIDTHS)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,offset", [(1, 0.0), (77, 3.0), (1500, 1.0)])
def test_forward_with_the_checkpoint_of_its_rows(n, c, dt, offset):
    """y and rstd bit for bit those of the plain call.  A code is xhat / step rounded, so within half a step and xhat's own error;
    a block's step is that of the largest xhat, which may lie on either side of a power of two: within its error, too."""
    from paper_2111_06483_b200 import api
    x, _, gamma, beta = problem(n, c, dt, offset, 7 * n + c, affine=n != 1)
    y, (mean, rstd) = api.ln_forward(x, 1e-5, gamma, beta)
    y8, (ck, rstd8) = api.ln_forward(x, 1e-5, gamma, beta, checkpoint=True)
    assert torch.equal(y8, y) and torch.equal(rstd8, rstd)
    want, tol = forward_bounds(np64(x), None, None, 1e-5)
    got = oracle.ckpt8_unpack(ck.codes.cpu().numpy(), ck.scales.cpu().numpy())
    step = np.repeat(np.where(ck.scales.cpu().numpy() == 0, 0.0, np.ldexp(1.0, ck.scales.cpu().numpy().astype(int) - 127)), 32, axis=1)[:, :c]
    cut = np.where(np.abs(ck.codes.cpu().numpy()) == 127, 0.5, 0.0)   # 127.5 to 128 is held as 127
    within(got, want[3], (0.5 + cut) * step + tol[3], "xhat")
    top = np.stack([np.abs(want[3][:, b * 32:b * 32 + 32]).max(axis=1) for b in range(ck.scales.shape[1])], axis=1)
    near = np.stack([tol[3][:, b * 32:b * 32 + 32].max(axis=1) for b in range(ck.scales.shape[1])], axis=1)
    unit = np.where(ck.scales.cpu().numpy() == 0, 0.0, np.ldexp(64.0, ck.scales.cpu().numpy().astype(int) - 127))
    assert (unit <= top + near).all() and (2 * unit >= top - near).all()


def backward_bounds(xhat, dxhat, rstd, gy, gamma, rows_in_a_row):
    gx, dgamma, dbeta = oracle.ln_backward(xhat, rstd, gy, gamma)
    k = links(xhat.shape[1])
    g = np.abs(gy if gamma is None else gy * gamma)
    ax = np.abs(xhat)
    d_level = (k + 3) * U * g.mean(axis=1, keepdims=True)
    d_along = (k + 4) * U * (g * ax).mean(axis=1, keepdims=True) + (g * dxhat).mean(axis=1, keepdims=True)
    along = (g * ax).mean(axis=1, keepdims=True)
    inner = g + g.mean(axis=1, keepdims=True) + ax * along
    t_gx = rstd[:, None] * (d_level + ax * d_along + dxhat * along + 4 * U * inner)
    t_dg = (rows_in_a_row + 2) * U * (np.abs(gy) * ax).sum(axis=0) + (np.abs(gy) * dxhat).sum(axis=0)
    t_db = (rows_in_a_row + 2) * U * np.abs(gy).sum(axis=0)
    return (gx, dgamma, dbeta), (t_gx, t_dg, t_db)


def chain(n):
    """Rows that one float32 sum passes at most: a lane group's own, and the 8 to 64 groups that a block joins."""
    return n // 8 + 80


@pytest.mark.parametrize("c", WIDTHS)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,offset", [(1, 0.0), (77, 3.0), (1500, 1.0)])
def test_backward(n, c, dt, offset):
    from paper_2111_06483_b200 import api
    x, gy, gamma, beta = problem(n, c, dt, offset, 7 * n + c, affine=n != 1)
    _, (mean, rstd) = api.ln_forward(x, 1e-5, gamma, beta)
    gx, dgamma, dbeta = api.ln_backward(x, gy, (mean, rstd), gamma)
    assert gx.dtype == x.dtype and dgamma.shape == (c,) and dbeta.shape == (c,)
    # from the mean and rstd that the call is given: x - mean and the product with rstd round xhat twice
    m, r = np64(mean), np64(rstd)
    xhat = (np64(x) - m[:, None]) * r[:, None]
    want, tol = backward_bounds(xhat, 3 * U * np.abs(xhat), r, np64(gy), None if gamma is None else np64(gamma), chain(n))
    within(np64(gx), want[0], tol[0] + half(dt, np.abs(want[0]) + tol[0]), "gx")
    within(np64(dgamma), want[1], tol[1], "dgamma")
    within(np64(dbeta), want[2], tol[2], "dbeta")


@pytest.mark.parametrize("c", WIDTHS)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 77, 1500])
def test_backward_from_the_checkpoint(n, c, dt):
    from paper_2111_06483_b200 import api
    x, gy, gamma, beta = problem(n, c, dt, 1.0, 7 * n + c, affine=n != 1)
    _, (ck, rstd) = api.ln_forward(x, 1e-5, gamma, beta, checkpoint=True)
    gx, dgamma, dbeta = api.ln_backward(None, gy, (ck, rstd), gamma)
    xhat = oracle.ckpt8_unpack(ck.codes.cpu().numpy(), ck.scales.cpu().numpy())   # exact
    want, tol = backward_bounds(xhat, 0.0 * xhat, np64(rstd), np64(gy), None if gamma is None else np64(gamma), chain(n))
    within(np64(gx), want[0], tol[0] + half(dt, np.abs(want[0]) + tol[0]), "gx")
    within(np64(dgamma), want[1], tol[1], "dgamma")
    within(np64(dbeta), want[2], tol[2], "dbeta")


@pytest.mark.parametrize("c,dt", [(64, "f32"), (256, "bf16"), (47, "f32"), (100, "bf16")])
def test_many_rows(c, dt):
    """More rows than the grid has groups: each takes several, asked for together, and a remainder."""
    from paper_2111_06483_b200 import api
    n = 150_003
    x, gy, gamma, beta = problem(n, c, dt, 2.0, c)
    y, (mean, rstd) = api.ln_forward(x, 1e-5, gamma, beta)
    want, tol = forward_bounds(np64(x), np64(gamma), np64(beta), 1e-5)
    within(np64(y), want[0], tol[0] + half(dt, np.abs(want[0]) + tol[0]), "y")
    _, (ck, rstd8) = api.ln_forward(x, 1e-5, gamma, beta, checkpoint=True)
    for first, xhat, dx in ((mean, (np64(x) - np64(mean)[:, None]) * np64(rstd)[:, None], 3 * U),
                            (ck, oracle.ckpt8_unpack(ck.codes.cpu().numpy(), ck.scales.cpu().numpy()), 0.0)):
        gx, dgamma, dbeta = api.ln_backward(x, gy, (first, rstd), gamma)
        want, tol = backward_bounds(xhat, dx * np.abs(xhat), np64(rstd), np64(gy), np64(gamma), 400)   # 150,003 rows over 1,184 blocks of 8 groups at least, and their joining
        within(np64(gx), want[0], tol[0] + half(dt, np.abs(want[0]) + tol[0]), "gx")
        within(np64(dgamma), want[1], tol[1], "dgamma")
        within(np64(dbeta), want[2], tol[2], "dbeta")


@pytest.mark.parametrize("c", [127, 129, 166, 249, 250, 253, 254, 333, 505, 506, 761, 762, 1017, 1018, 1021, 1022, 1023])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 9, 4003])
def test_rows_that_are_no_whole_vectors(n, c, dt):
    """Rows that start anywhere within a vector, to one column more or less than a kernel's lanes cover, all four passes."""
    test_forward(n, c, dt, 1.0)
    test_forward_with_the_checkpoint_of_its_rows(n, c, dt, 1.0)
    test_backward(n, c, dt, 1.0)
    test_backward_from_the_checkpoint(n, c, dt)


@pytest.mark.parametrize("c", [772, 1020, 1027, 1028, 1032, 1536, 2044, 2047, 2049, 2052, 4096, 4100, 8188, 8192, 8196])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 78, 1501])
def test_rows_that_a_block_shares(n, c, dt):
    """Rows of more columns than a warp holds, to the most that a block does and one vector more, all four passes."""
    test_forward(n, c, dt, 1.0)
    test_forward_with_the_checkpoint_of_its_rows(n, c, dt, 1.0)
    test_backward(n, c, dt, 1.0)
    test_backward_from_the_checkpoint(n, c, dt)


@pytest.mark.parametrize("c", [388, 392, 508, 512, 516, 520, 764, 768, 776, 1016, 1024, 1280, 1532, 1536, 1540, 1544, 2040])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 2, 3, 79, 1502])
def test_rows_that_several_warps_share(n, c, dt):
    """Rows of more than a warp's columns, several to a block, whose last ones have no row."""
    test_forward(n, c, dt, 1.0)
    test_forward_with_the_checkpoint_of_its_rows(n, c, dt, 1.0)
    test_backward(n, c, dt, 1.0)
    test_backward_from_the_checkpoint(n, c, dt)


@pytest.mark.parametrize("c", [1021, 2000, 2047, 4100, 8192])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_wide_rows_in_place(c, dt):
    """The result over x or over gy, as for other rows; without weight gradients the same gx."""
    from paper_2111_06483_b200 import api, binding as B
    test_in_place(c, dt)
    x, gy, gamma, beta = problem(700, c, dt, 1.0, c)
    _, saved = api.ln_forward(x, 1e-5, gamma, beta)
    gx, _, _ = api.ln_backward(x, gy, saved, gamma)
    alone = torch.empty_like(gx)
    B.sar_ln_bwd(x, *saved, gamma, gy, alone, None, None, None)
    assert torch.equal(alone, gx)


@pytest.mark.parametrize("c", [5, 47, 127, 333, 1021])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_what_lies_before_and_behind_stays(c, dt):
    """y, gx, codes and scales are written to the last value and not a byte further, and infinities behind x and gy reach nothing."""
    from paper_2111_06483_b200 import api, binding as B
    n = 37
    x, gy, gamma, beta = problem(n, c, dt, 1.0, c)
    want_y, (ck, rstd) = api.ln_forward(x, 1e-5, gamma, beta, checkpoint=True)
    want_gx, dgamma, dbeta = api.ln_backward(None, gy, (ck, rstd), gamma)

    def room(like, fill):
        t = torch.full((like.numel() + 32,), fill, dtype=like.dtype, device="cuda")
        t[16:-16] = like.reshape(-1)
        return t, t[16:-16].view(like.shape)

    (_, xs), (_, gs) = room(x, float("inf")), room(gy, float("nan"))
    (ry, y), (rc, codes), (rs, scales) = room(torch.zeros_like(x), 3.0), room(torch.zeros_like(ck.codes), 99), room(torch.zeros_like(ck.scales), 77)
    B.sar_ln_fwd_ckpt8(xs, gamma, beta, 1e-5, y, rstd, codes, scales)
    assert torch.equal(y, want_y) and torch.equal(codes, ck.codes) and torch.equal(scales, ck.scales)
    (rg, gx), ws = room(torch.zeros_like(x), 3.0), torch.empty(B.sar_ln_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    dg, db = torch.empty_like(dgamma), torch.empty_like(dbeta)
    B.sar_ln_bwd_ckpt8(codes, scales, rstd, gamma, gs, gx, dg, db, ws)
    assert torch.equal(gx, want_gx) and torch.equal(dg, dgamma) and torch.equal(db, dbeta)
    for r, v in ((ry, 3), (rg, 3), (rc, 99), (rs, 77)):
        assert (r[:16] == v).all() and (r[-16:] == v).all()


def test_gradient_against_differences():
    """The loss sum(y * gy) in float64 on the oracle's forward pass, moved along random directions: what the backward pass says
    of its slope.  A central difference of step 1e-4 on values of order 1 is off by 1e-8 and the float32 gradient by 1e-5."""
    from paper_2111_06483_b200 import api
    x, gy, gamma, beta = problem(40, 24, "f32", 0.5, 11)
    _, saved = api.ln_forward(x, 1e-5, gamma, beta)
    grads = [np64(t) for t in api.ln_backward(x, gy, saved, gamma)]
    rng = np.random.default_rng(0)
    at = [np64(t) for t in (x, gamma, beta)]
    for _ in range(4):
        move = [rng.standard_normal(a.shape) for a in at]
        loss = [(oracle.ln_forward(at[0] + s * move[0], 1e-5, at[1] + s * move[1], at[2] + s * move[2])[0] * np64(gy)).sum() for s in (1e-4, -1e-4)]
        slope = (loss[0] - loss[1]) / 2e-4
        size = sum(np.abs(g * m).sum() for g, m in zip(grads, move))
        assert abs(slope - sum((g * m).sum() for g, m in zip(grads, move))) < 1e-5 * size


@pytest.mark.parametrize("c", [64, 47, 1500])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_in_place(c, dt):
    from paper_2111_06483_b200 import api, binding as B
    x, gy, gamma, beta = problem(513, c, dt, 1.0, c)
    y, (mean, rstd) = api.ln_forward(x, 1e-5, gamma, beta)
    gx, dgamma, dbeta = api.ln_backward(x, gy, (mean, rstd), gamma)
    over = x.clone()
    B.sar_ln_fwd(over, gamma, beta, 1e-5, over, None, None)   # mean and rstd not asked for
    assert torch.equal(over, y)
    ws = torch.empty(B.sar_ln_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    dg, db = torch.empty_like(dgamma), torch.empty_like(dbeta)
    for over in (x.clone(), gy.clone()):
        xin, gin = (over, gy) if torch.equal(over, x) else (x, over)
        B.sar_ln_bwd(xin, mean, rstd, gamma, gin, over, dg, db, ws)
        assert torch.equal(over, gx) and torch.equal(dg, dgamma) and torch.equal(db, dbeta)
    _, (ck, rstd8) = api.ln_forward(x, 1e-5, gamma, beta, checkpoint=True)
    want = api.ln_backward(None, gy, (ck, rstd8), gamma)
    over = gy.clone()
    B.sar_ln_bwd_ckpt8(ck.codes, ck.scales, rstd8, gamma, over, over, dg, None, ws)   # one of the two sums
    assert torch.equal(over, want[0]) and torch.equal(dg, want[1])
    over = gy.clone()
    B.sar_ln_bwd(x, mean, rstd, gamma, over, over, None, None, None)   # no sums, no scratch
    assert torch.equal(over, gx)


@pytest.mark.parametrize("c", [64, 47, 1500])
def test_rows_with_infinities_and_nan_spoil_no_other_row(c):
    from paper_2111_06483_b200 import api
    x, gy, gamma, beta = problem(100, c, "f32", 0.0, c)
    clean = x.clone()
    x[13, 3], x[40, 0], x[77, c - 1] = float("nan"), float("inf"), float("-inf")
    good = torch.ones(100, dtype=torch.bool, device="cuda")
    good[[13, 40, 77]] = False
    y, (mean, rstd) = api.ln_forward(x, 1e-5, gamma, beta)
    y0, (mean0, rstd0) = api.ln_forward(clean, 1e-5, gamma, beta)
    assert torch.equal(y[good], y0[good]) and y[~good].isnan().all() and torch.equal(mean[good], mean0[good])
    y8, (ck, _) = api.ln_forward(x, 1e-5, gamma, beta, checkpoint=True)
    _, (ck0, _) = api.ln_forward(clean, 1e-5, gamma, beta, checkpoint=True)
    assert torch.equal(ck.codes[good], ck0.codes[good]) and torch.equal(ck.scales[good], ck0.scales[good])
    assert (ck.scales[~good] == 255).all() and not ck.codes[~good].any()
    gx = api.ln_backward(None, gy, (ck, rstd0), gamma)[0]
    gx0 = api.ln_backward(None, gy, (ck0, rstd0), gamma)[0]
    assert torch.equal(gx[good], gx0[good]) and gx[~good].isnan().all()


@pytest.mark.parametrize("c", [64, 300, 1000])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_addresses_that_are_not_aligned(c, dt):
    from paper_2111_06483_b200 import api, binding as B
    n = 65
    x, gy, gamma, beta = problem(n, c, dt, 1.0, 3)
    want, tol = forward_bounds(np64(x), np64(gamma), np64(beta), 1e-5)
    room = torch.full((n * c + 2,), 9.0, dtype=DT[dt], device="cuda")
    off = room[1:-1].view(n, c)
    mean, rstd = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    B.sar_ln_fwd(x, gamma, beta, 1e-5, off, mean, rstd)
    within(np64(off), want[0], tol[0] + half(dt, np.abs(want[0]) + tol[0]), "y")
    codes = torch.zeros(n * c + 1, dtype=torch.int8, device="cuda")[1:].view(n, c)
    scales = torch.empty(n, (c + 31) // 32, dtype=torch.uint8, device="cuda")
    B.sar_ln_fwd_ckpt8(x, gamma, beta, 1e-5, off, rstd, codes, scales)
    B.sar_ln_bwd_ckpt8(codes, scales, rstd, gamma, gy, off, None, None, None)
    gx = oracle.ln_backward(oracle.ckpt8_unpack(codes.cpu().numpy(), scales.cpu().numpy()), np64(rstd), np64(gy), np64(gamma))[0]
    within(np64(off), gx, (links(c) + 48) * U * (np.abs(gx) + np64(rstd)[:, None] * 30) + half(dt, gx), "gx")   # |xhat| and |gy gamma| below 5 or so each
    assert room[0] == 9 and room[-1] == 9


def test_more_than_2_31_values():
    from paper_2111_06483_b200 import api
    n, c = 8_600_000, 256
    x = torch.zeros(n, c, dtype=torch.bfloat16, device="cuda")
    gy = torch.zeros_like(x)
    small_x, small_g, gamma, beta = problem(129, c, "bf16", 1.0, 5)
    x[-129:], gy[-129:] = small_x, small_g
    y, (ck, rstd) = api.ln_forward(x, 1e-5, gamma, beta, checkpoint=True)
    y0, (ck0, rstd0) = api.ln_forward(small_x, 1e-5, gamma, beta, checkpoint=True)
    assert torch.equal(y[-129:], y0) and torch.equal(ck.codes[-129:], ck0.codes) and torch.equal(ck.scales[-129:], ck0.scales)
    del y
    gx, dgamma, dbeta = api.ln_backward(None, gy, (ck, rstd), gamma)
    gx0, dg0, db0 = api.ln_backward(None, small_g, (ck0, rstd0), gamma)
    assert torch.equal(gx[-129:], gx0) and not gx[:-129].any()
    size = np64(small_g.float().abs()).sum(axis=0)
    within(np64(dbeta), np64(db0), 200 * U * size, "dbeta")
    within(np64(dgamma), np64(dg0), 200 * U * 16 * size, "dgamma")   # |xhat| <= sqrt(256)


def test_no_rows():
    from paper_2111_06483_b200 import api
    x = torch.empty(0, 48, device="cuda")
    y, saved = api.ln_forward(x)
    gx, dgamma, dbeta = api.ln_backward(x, x, saved)
    assert y.shape == (0, 48) and gx.shape == (0, 48) and dgamma.shape == (48,) and not dgamma.any() and not dbeta.any()
    _, saved = api.ln_forward(x, checkpoint=True)
    assert not api.ln_backward(None, x, saved)[1].any()


@pytest.mark.parametrize("c", [64, 47, 1500])
def test_the_same_bits_every_time_captured_and_on_another_stream(c):
    from paper_2111_06483_b200 import api
    x, gy, gamma, beta = problem(5000, c, "bf16", 1.0, c)

    def step():
        y, (ck, rstd) = api.ln_forward(x, 1e-5, gamma, beta, checkpoint=True)
        _, (mean, r) = api.ln_forward(x, 1e-5, gamma, beta)
        return (y, ck.codes, *api.ln_backward(None, gy, (ck, rstd), gamma), *api.ln_backward(x, gy, (mean, r), gamma))

    want = [t.clone() for t in step()]
    assert all(torch.equal(a, b) for a, b in zip(step(), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    x2 = problem(5000, c, "bf16", 2.0, c + 1)[0]
    keep = x.clone()
    x.copy_(x2)
    graph.replay()
    assert not torch.equal(held[0], want[0])
    x.copy_(keep)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_refusals():
    from paper_2111_06483_b200 import api
    x, gy, gamma, beta = problem(20, 64, "bf16", 0.0, 1)
    y, saved = api.ln_forward(x, 1e-5, gamma, beta)
    y, saved8 = api.ln_forward(x, 1e-5, gamma, beta, checkpoint=True)
    ck, rstd = saved8
    for call in (lambda: api.ln_forward(x, 1e-5, gamma[:-1], beta), lambda: api.ln_forward(x, 1e-5, gamma.bfloat16(), beta),
                 lambda: api.ln_forward(x, 1e-5, gamma, beta.cpu()), lambda: api.ln_forward(x.t(), 1e-5),
                 lambda: api.ln_backward(x, gy[:-1], saved, gamma), lambda: api.ln_backward(x, gy.float(), saved, gamma),
                 lambda: api.ln_backward(x, gy, (saved[0][:-1], saved[1]), gamma), lambda: api.ln_backward(None, gy[:, :32].contiguous(), saved8, gamma),
                 lambda: api.ln_backward(None, gy, (api.Checkpoint8(ck.codes, ck.scales[:-1]), rstd), gamma),
                 lambda: api.ln_backward(None, gy, (ck, rstd[:-1]), gamma)):
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(TypeError):   # the rows are needed where saved holds no checkpoint
        api.ln_backward(None, gy, saved, gamma)
    with pytest.raises(ValueError):
        api.ln_forward(x.view(20, 2, 32))
    from paper_2111_06483_b200 import binding as B
    with pytest.raises(B.SarError) as e:
        api.ln_forward(x, -1.0)
    assert e.value.code == -1
