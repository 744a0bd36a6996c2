"""Calls of the layer normalisation, the 8-bit checkpoints and the products by group at the edges of what they take."""
import numpy as np
import pytest
import torch

import oracle

pytestmark = pytest.mark.gpu


def test_codes_and_scales_of_different_shapes_are_refused():
    """A checkpoint that was cut along one of its arrays: every row behind the first would be decoded with another row's scales."""
    from paper_2111_06483_b200 import api, binding as B
    n, C = 10, 64
    x = torch.randn(n, C, device="cuda").bfloat16()
    c, rstd = api.ckpt8_pack(x), torch.ones(n, device="cuda")
    o = torch.tensor([0, n], device="cuda")
    codes, narrow = c.codes[:, :32].contiguous(), x[:, :32].contiguous()
    ws, dw = torch.empty(1 << 20, dtype=torch.uint8, device="cuda"), torch.empty(1, 32, C, device="cuda")
    for scales in (c.scales, c.scales.view(-1), c.scales[:, :1].repeat(2, 1), c.scales[:, :1].contiguous().view(1, -1)):
        cut = api.Checkpoint8(codes, scales)
        for call in (lambda: api.ckpt8_unpack(cut), lambda: api.ln_backward(None, narrow, (cut, rstd)), lambda: api.typed_linear_backward_weight(cut, o, x),
                     lambda: B.sar_ckpt8_unpack(codes, scales, narrow), lambda: B.sar_ln_bwd_ckpt8(codes, scales, rstd, None, narrow, narrow, None, None, None),
                     lambda: B.sar_linear_grouped_bwd_weight_ckpt8(codes, scales, None, None, x, o, dw, ws)):
            with pytest.raises(AssertionError):
                call()
    api.ckpt8_unpack(api.Checkpoint8(codes, c.scales[:, :1].contiguous()))


def test_a_layer_refuses_a_checkpoint_of_another_width():
    from paper_2111_06483_b200 import api
    n, d = 60, 64
    gen = torch.Generator().manual_seed(3)
    g = api.Graph.from_coo(n, *(torch.randint(0, n, (400,), generator=gen, dtype=torch.int32).cuda() for _ in range(2)))
    h, W = torch.randn(n, d, generator=gen).bfloat16().cuda(), torch.randn(d, d, generator=gen).bfloat16().cuda()
    _, (c, inv) = api.sage_layer_forward(g, h, W, W, checkpoint=True)
    for bad in (api.Checkpoint8(c.codes, torch.cat([c.scales, c.scales], 1)), api.Checkpoint8(torch.cat([c.codes, c.codes], 1), c.scales),
                api.Checkpoint8(c.codes.view(n * 2, d // 2), c.scales.view(n * 2, -1))):
        with pytest.raises(AssertionError):
            api.sage_layer_backward(g, h, W, W, (bad, inv), h)


def test_sizes_beyond_32_bits_are_refused():
    """2^32 + 64 columns are not 64.  Arrays without rows hold no memory, whatever their width."""
    from paper_2111_06483_b200 import api, binding as B
    C = 2 ** 32 + 64
    def none(*shape, dtype=torch.bfloat16):
        return torch.empty(0, *shape, dtype=dtype, device="cuda")
    x, few, o = none(C), none(64), torch.zeros(2, dtype=torch.int64, device="cuda")
    row = none(dtype=torch.float32)
    c = api.Checkpoint8(none(C, dtype=torch.int8), none(C // 32, dtype=torch.uint8))
    W = torch.empty(1, C, 0, dtype=torch.bfloat16, device="cuda")
    for call in (lambda: api.ln_forward(x), lambda: api.ln_forward(x, checkpoint=True), lambda: api.ln_backward(x, x, (row, row)), lambda: api.ln_backward(None, x, (c, row)),
                 lambda: api.ckpt8_pack(x), lambda: api.ckpt8_unpack(c), lambda: api.typed_linear_forward(x, W, o), lambda: api.typed_linear_forward(none(0), W.view(1, 0, C), o),
                 lambda: api.typed_linear_backward_weight(x, o, few), lambda: api.typed_linear_backward_weight(few, o, x), lambda: api.typed_linear_backward_weight(c, o, few)):
        with pytest.raises(B.SarError) as e:
            call()
        assert e.value.code == -2


def test_scratch_of_more_rows_serves_fewer():
    from paper_2111_06483_b200 import binding as B
    d = 256
    gen = torch.Generator().manual_seed(4)
    h, dz = (torch.randn(4737, d, generator=gen).bfloat16().cuda() for _ in range(2))
    ws = torch.empty(B.sar_linear_grouped_workspace_bytes(4737, 1, d, d), dtype=torch.uint8, device="cuda")
    for n in (4737, 4736, 64, 1):
        dw = torch.empty(1, d, d, device="cuda")
        B.sar_linear_grouped_bwd_weight(h[:n], dz[:n], None, dw, ws)
        want = h[:n].double().t() @ dz[:n].double()
        size = h[:n].double().abs().t() @ dz[:n].double().abs()
        assert ((dw[0].double() - want).abs() <= (34 * 2.0 ** -22 + 160 * 2.0 ** -24) * size + 1e-30).all()   # the bound of the products' own tests


@pytest.mark.parametrize("c", [3, 4, 12, 47, 64, 72, 100, 127, 191, 256, 333, 500, 764, 1000, 1021, 1500, 2048, 3001, 8192, 9001])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("level,steps", [(1000.0, 0), (12345.678, 0), (-10000.0 - 1 / 3, 0), (1000.0, 1), (-7777.7, 3)])
def test_rows_of_little_spread_about_a_high_level(c, dt, level, steps):
    """Constant rows, and rows within a few units in the last place of a level: xhat and 1 / sigma from the mean itself, not from one
    that was rounded.  u = 2^-24, w a unit in the last place of the level.
    The mean first taken is off by e <= (k + 2) u |level| with k additions one after the other (k as in the normalisation's tests), and so
    are the deviations from it, exactly (Sterbenz).  They are small multiples of w in float32, and their sums exact.  What is left: the
    rounding of e, of the deviation times 1 / sigma and of 1 / sigma itself, whose variance is a difference of at most v + 2 e^2 to
    (k + 6) u of that.  The stored mean is rounded once more.  bf16: the row's sum is exact (whole multiples of 2^-7 of the level, less
    than 2^24 of them) and so is what the quotient is off, so the deviations are taken from the mean rounded to float32 after one more
    addition: 2 u |mean|, nothing in a constant row, whose mean is a float32.  That adds its square to the variance.  bf16 results:
    half a step."""
    from paper_2111_06483_b200 import api
    U, n, eps = 2.0 ** -24, 9, 1e-5
    gen = torch.Generator().manual_seed(c)
    x = torch.full((n, c), level, dtype=torch.float32).to(dt)
    w = torch.tensor(torch.finfo(dt).eps * 2.0 ** np.floor(np.log2(abs(level))))
    x = (x.double() + torch.randint(-steps, steps + 1, (n, c), generator=gen) * w.double()).to(dt)
    X = x.double().numpy()
    _, mean, rstd, xhat = oracle.ln_forward(X, eps)
    x = x.cuda()
    y, (got_mean, got_rstd) = api.ln_forward(x, eps)
    k = (c + 3) // 4 + 16 if c <= 128 else max(64, c // 32 * 2) + 16
    e = np.abs(X).max() * (k + 2) * U if dt == torch.float32 else np.abs(X).max() * 2 * U   # bf16: the sum is exact
    var = 1.0 / rstd ** 2 - eps
    rel = (k + 6) * U * (var + 2 * e * e) / (var + eps)
    rel = rel / 2 + rel * rel + 3 * U
    if dt == torch.bfloat16 and steps:
        rel = rel + (2 * U * np.abs(mean) * rstd) ** 2
    tol = 4 * U * (np.abs(xhat) + 2 * e * rstd[:, None]) + np.abs(xhat) * rel[:, None]
    if dt == torch.bfloat16 and steps:
        tol = tol + 2 * U * np.abs(mean)[:, None] * rstd[:, None]
    half = 0.0 if dt == torch.float32 else 2.0 ** -8 * (np.abs(xhat) + tol)
    assert (np.abs(got_mean.double().cpu().numpy() - mean) <= 2 * U * np.abs(mean) + 4 * U * e).all()
    assert (np.abs(got_rstd.double().cpu().numpy() - rstd) <= (rel + 2 * U) * rstd).all()
    assert (np.abs(y.double().cpu().numpy() - xhat) <= tol + half).all()
    y8, (ck, rstd8) = api.ln_forward(x, eps, checkpoint=True)
    assert torch.equal(y8, y) and torch.equal(rstd8, got_rstd)
    if steps == 0:
        v = api.ckpt8_unpack(ck, torch.float32).double().cpu().numpy()
        assert (np.abs(v) <= 2 * tol).all()   # of blocks whose largest value is within tol of zero


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("c", [1, 47, 64, 333, 1024, 1027, 2048, 4095, 8192, 8193])
@pytest.mark.parametrize("n", [1, 3, 65, 9473])
def test_the_scratch_for_these_rows_is_enough(n, c, dt):
    """The backward passes write no byte behind it, and give what they give with more."""
    from paper_2111_06483_b200 import api, binding as B
    gen = torch.Generator().manual_seed(n + c)
    x, gy = (torch.randn(n, c, generator=gen).to(dt).cuda() for _ in range(2))
    gamma = torch.randn(c, generator=gen).cuda()
    _, (mean, rstd) = api.ln_forward(x)
    _, (ck, _) = api.ln_forward(x, checkpoint=True)
    size, most = B.sar_ln_workspace_bytes_rows(n, c), B.sar_ln_workspace_bytes(c)
    assert size <= most
    for backward in (lambda gx, dg, db, ws: B.sar_ln_bwd(x, mean, rstd, gamma, gy, gx, dg, db, ws),
                     lambda gx, dg, db, ws: B.sar_ln_bwd_ckpt8(ck.codes, ck.scales, rstd, gamma, gy, gx, dg, db, ws)):
        got = []
        for room in (size, most):
            buffer = torch.full((room + 4096,), 0xAB, dtype=torch.uint8, device="cuda")
            out = [torch.empty_like(x), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")]
            backward(*out, buffer[:room])
            assert (buffer[room:] == 0xAB).all()
            got.append(out)
        assert all(torch.equal(a, b) for a, b in zip(*got))


def test_a_backward_pass_over_few_wide_rows_takes_little_memory():
    from paper_2111_06483_b200 import api
    x = torch.randn(2, 1 << 20, device="cuda")
    _, saved = api.ln_forward(x)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    api.ln_backward(x, x, saved)
    assert torch.cuda.max_memory_allocated() - before < 64 << 20   # gx, dgamma, dbeta and one record: 24 MB


@pytest.mark.parametrize("d_in,d_out", [(136, 8), (136, 72), (264, 40), (456, 104), (1032, 24), (200, 120), (256, 72), (200, 48)])
@pytest.mark.parametrize("sizes", [[50_000], [20_001, 0, 1, 39_000, 65], [2500] * 24])
def test_weight_gradients_of_many_rows_taken_turned_or_not(sizes, d_in, d_out):
    """Widths whose transposed gradient takes fewer tiles, on either side of the rule, with rows of no group around them that hold NaN.
    The bound is that of the products by group: 34 additions by truncation, 2^-22, and the joined runs and chunks, 2^-24 each."""
    from paper_2111_06483_b200 import api
    gen = torch.Generator(device="cuda").manual_seed(d_in + len(sizes))
    n, before = sum(sizes) + 40, 7
    h, dz = (torch.randn(n, d, generator=gen, device="cuda").bfloat16() for d in (d_in, d_out))
    edges = (before + np.cumsum([0] + sizes)).tolist()
    for t in (h, dz):
        t[:before], t[edges[-1]:] = float("nan"), float("inf")
    dw = api.typed_linear_backward_weight(h, torch.tensor(edges, device="cuda"), dz)
    for g, (a, b) in enumerate(zip(edges, edges[1:])):
        x, y = h[a:b].double(), dz[a:b].double()
        size = x.abs().t() @ y.abs()
        assert ((dw[g].double() - x.t() @ y).abs() <= (34 * 2.0 ** -22 + (n // 512 + 160) * 2.0 ** -24) * size).all()


@pytest.mark.parametrize("c", [1, 24, 47, 64, 100, 333, 1024, 1027, 2048, 5000, 8200])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offsets", [[30, 30, 200, 333], [0, 400], [390, 400, 400], [400, 400], [50, 20, 90, 60], [-5, 2 ** 40]])
def test_the_normalisation_s_gradients_over_the_rows_of_some_group(c, dt, offsets):
    """Rows of no group hold NaN and infinities in every array: all results are those of a call where these rows are zeros, bit for bit."""
    from paper_2111_06483_b200 import api
    n = 400
    gen = torch.Generator().manual_seed(c)
    x, gy = (torch.randn(n, c, generator=gen).to(dt).cuda() for _ in range(2))
    gamma = torch.randn(c, generator=gen).cuda()
    _, (mean, rstd) = api.ln_forward(x)
    _, (ck, _) = api.ln_forward(x, checkpoint=True)
    o = torch.tensor(offsets, device="cuda")
    rows = oracle.group_rows(offsets, n)
    out = torch.ones(n, dtype=torch.bool, device="cuda")
    out[rows[0][0]:rows[-1][1]] = False

    def filled(t, value):
        return torch.where(out.view(-1, *[1] * (t.dim() - 1)), torch.full_like(t, value), t)
    nan, inf = float("nan"), float("inf")
    clean = [filled(t, 0) for t in (x, gy, mean, rstd, ck.codes, ck.scales)]
    dirty = [filled(t, v) for t, v in ((x, nan), (gy, inf), (mean, inf), (rstd, nan), (ck.codes, 99), (ck.scales, 255))]
    for checkpoint in (False, True):
        def gradients(arrays, *more):
            x, gy, mean, rstd, codes, scales = arrays
            return api.ln_backward(x, gy, (api.Checkpoint8(codes, scales) if checkpoint else mean, rstd), gamma, *more)
        want, got = gradients(clean), gradients(dirty, o)
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and not got[0][out].any()


@pytest.mark.parametrize("checkpoint", [False, True])
def test_what_rows_of_no_type_hold_reaches_nothing_in_a_typed_layer(checkpoint):
    """A padded batch: NaN and infinities behind the last node and before the first, in x and in the upstream gradient."""
    from paper_2111_06483_b200 import api
    n, d_in, d_out = 300, 96, 72
    gen = torch.Generator().manual_seed(5)
    x, gz = (torch.randn(n, d, generator=gen).bfloat16().cuda() for d in (d_in, d_out))
    W = (torch.randn(2, d_in, d_out, generator=gen) / d_in ** 0.5).bfloat16().cuda()
    gamma, beta = torch.rand(d_in, generator=gen).cuda() + 0.5, torch.randn(d_in, generator=gen).cuda()
    o = torch.tensor([20, 100, 250], device="cuda")

    def step():
        z, saved = api.typed_layer_forward(x, W, o, gamma, beta, checkpoint=checkpoint)
        return (z, *api.typed_layer_backward(W, o, saved, gz, gamma, beta))
    want = step()
    x[:20], x[250:], gz[:20], gz[250:] = float("nan"), float("inf"), float("inf"), float("nan")
    got = step()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert not got[0][:20].any() and not got[1][250:].any() and not any(t.isnan().any() for t in got)


def test_rows_whose_squares_leave_float32():
    """As documented: 1 / sigma is zero and y is beta, from the mean or from the checkpoint alike; other rows are not touched."""
    from paper_2111_06483_b200 import api
    for c in (64, 333, 9000):
        x = torch.randn(5, c, device="cuda")
        clean, _ = api.ln_forward(x)
        x[2] *= 1e20
        beta = torch.randn(c, device="cuda")
        y, (mean, rstd) = api.ln_forward(x, beta=beta)
        assert torch.equal(y[2], beta) and rstd[2] == 0 and mean[2].isfinite()
        assert torch.equal(api.ln_forward(x)[0][[0, 1, 3, 4]], clean[[0, 1, 3, 4]])
        y8, (ck, rstd8) = api.ln_forward(x, beta=beta, checkpoint=True)
        assert torch.equal(y8, y) and not ck.scales[2].any() and not ck.codes[2].any()
