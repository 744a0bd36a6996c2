"""GPU parity of the products by groups of rows (a projection per node type) and of their gradients, from bf16 rows and from 8-bit
checkpoints, with the float64 oracle.

Tolerances.  A product of two bf16 is exact in float32.  The tensor cores add 16 of them to a float32 sum and cut off what does
not fit: each addition takes at most 2 units, 2^-22, of what has been added up, so K products are off by (K / 16 + 2) 2^-22 of the
sum of their magnitudes.  A weight gradient's sum runs over 512 rows at most (34 additions); the runs and chunks are joined by
at most `joins` additions that round by 2^-24.  A bf16 result is rounded once more, by 2^-8 of the value."""
import numpy as np
import pytest
import torch

import oracle

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
NAN = float("nan")


def np64(t):
    return t.detach().double().cpu().numpy()


def within(got, want, tol, what):
    err = np.abs(got - want)
    bad = ~(err <= tol)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3].tolist(), float(np.nanmax(err / tol)))


def problem(sizes, d_in, d_out, before=0, behind=0, seed=0):
    """(h, W, dz, offsets) with groups of these sizes; the rows of no group hold NaN and infinities."""
    gen = torch.Generator().manual_seed(seed + 31 * d_in + d_out + sum(sizes))
    n = before + sum(sizes) + behind
    h, dz = torch.randn(n, d_in, generator=gen), torch.randn(n, d_out, generator=gen)
    W = torch.randn(len(sizes), d_in, d_out, generator=gen)
    offsets = torch.tensor([before] + (before + np.cumsum(sizes)).tolist())
    for t in (h, dz):
        t[:before], t[n - behind:] = NAN, float("inf")
    return [t.bfloat16().cuda() for t in (h, W, dz)] + [offsets.cuda()]


def rows_bound(a, b_abs, want, offsets):
    k = a.shape[1]
    size = oracle.grouped_linear(np.abs(a), b_abs, offsets)
    tol = (k / 16 + 2) * 2.0 ** -22 * size
    return tol + 2.0 ** -8 * (np.abs(want) + tol)


def weight_bound(h, dz, W, offsets, joins):
    return (34 * 2.0 ** -22 + joins * U) * oracle.grouped_linear_bwd(np.abs(h), np.abs(W), offsets, np.abs(dz))[1]


def joins(n):
    return n // 512 + 160


def clean(x):
    return np.where(np.isfinite(x), x, 0.0)


def run_all(h, W, dz, offsets):
    from paper_2111_06483_b200 import binding as B
    n, d_in = h.shape
    G, _, d_out = W.shape
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    z = torch.full((n, d_out), 7.0, dtype=torch.bfloat16, device="cuda")
    dh = torch.full((n, d_in), 7.0, dtype=torch.bfloat16, device="cuda")
    dw = torch.full((G, d_in, d_out), NAN, device="cuda")
    ws = torch.full((B.sar_linear_grouped_workspace_bytes(n, G, d_in, d_out),), 255, dtype=torch.uint8, device="cuda")   # NaN
    B.sar_linear_grouped(h, W, offsets, z, 0, flag)
    B.sar_linear_grouped_bwd_input(dz, W, offsets, dh, 0, flag)
    B.sar_linear_grouped_bwd_weight(h, dz, offsets, dw, ws, flag)
    assert flag.item() == 0
    return z, dh, dw


def check_all(h, W, dz, offsets):
    z, dh, dw = run_all(h, W, dz, offsets)
    H, w, Z, o = clean(np64(h)), np64(W), clean(np64(dz)), offsets.cpu().numpy()
    want_z = oracle.grouped_linear(H, w, o, rest=7.0)
    want_dh, want_dw = oracle.grouped_linear_bwd(H, w, o, Z, rest=7.0)
    within(np64(z), want_z, rows_bound(H, np.abs(w), want_z, o), "z")
    within(np64(dh), want_dh, rows_bound(Z, np.abs(w.transpose(0, 2, 1)), want_dh, o), "dh")
    within(np64(dw), want_dw, weight_bound(H, Z, w, o, joins(h.shape[0])) + 1e-30, "dw")
    rest = np.ones(h.shape[0], bool)
    for a, b in oracle.group_rows(o, h.shape[0]):
        rest[a:b] = False
    assert (np64(z)[rest] == 7).all() and (np64(dh)[rest] == 7).all()   # left as they were


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300, 513])
def test_one_group_of_few_rows(n):
    check_all(*problem([n], 64, 64))


@pytest.mark.parametrize("d_in,d_out", [(8, 8), (16, 136), (64, 64), (72, 40), (128, 256), (136, 72), (256, 256), (264, 264), (320, 392), (512, 520), (520, 512), (1032, 48), (40, 1032)])
def test_widths(d_in, d_out):
    check_all(*problem([200, 0, 1, 333], d_in, d_out))


@pytest.mark.parametrize("d_in,d_out", [(136, 8), (264, 40), (456, 72), (520, 200), (1032, 120)])
@pytest.mark.parametrize("sizes", [[5], [200, 0, 1, 333], [7, 900, 0, 65] * 16])
def test_weight_gradients_taken_turned(sizes, d_in, d_out):
    """Widths whose transposed gradient takes fewer tiles, with few outputs and with many, rows of no group around them."""
    check_all(*problem(sizes, d_in, d_out, 3, 70))


@pytest.mark.parametrize("sizes", [[0], [0, 0, 5], [128, 128], [127, 1, 129], [1] * 40, [3, 700, 0, 0, 65, 2000], [31, 33, 0] * 11])
@pytest.mark.parametrize("before,behind", [(0, 0), (5, 0), (0, 9), (130, 200)])
def test_groups_and_rows_of_no_group(sizes, before, behind):
    """Tiles end inside groups, groups inside tiles; the rows of no group hold NaN and infinities and reach nothing."""
    if before + sum(sizes) + behind == 0:
        return
    check_all(*problem(sizes, 72, 80, before, behind))


@pytest.mark.parametrize("sizes", [[40_000, 3, 0, 25_001, 7_777], [100] * 500, [0] * 1000 + [5000] + [1] * 23])
@pytest.mark.parametrize("d_in,d_out", [(64, 128), (136, 264)])
def test_more_tiles_than_blocks(sizes, d_in, d_out):
    check_all(*problem(sizes, d_in, d_out, 3, 4))


def test_neighbours_hold_nan():
    """A tile takes in the next group's rows, a contraction's last step as well, and the weights lie one after the other: NaN and
    infinities in another group stay there."""
    h, W, dz, o = problem([70, 50, 90], 72, 40)
    clean_z, clean_dh, clean_dw = run_all(h, W, dz, o)
    h[70:120], dz[70:120], W[1] = NAN, float("inf"), NAN
    z, dh, dw = run_all(h, W, dz, o)
    for a, b in ((z, clean_z), (dh, clean_dh)):
        assert torch.equal(a[:70], b[:70]) and torch.equal(a[120:], b[120:]) and a[70:120].isnan().all()
    assert torch.equal(dw[0], clean_dw[0]) and torch.equal(dw[2], clean_dw[2]) and dw[1].isnan().all()


def test_offsets_that_descend_or_leave_the_array():
    """Read as the header says; every access stays in bounds."""
    h, W, dz, _ = problem([300], 64, 64)
    W = W.repeat(5, 1, 1).contiguous() * torch.arange(1, 6, device="cuda").view(5, 1, 1).bfloat16()
    check_all(h, W, dz, torch.tensor([-7, 100, 40, 2 ** 40, 5, -2 ** 60], device="cuda"))


def test_weight_sums_do_not_drift():
    """65,536 rows of one group with means apart from zero, which one float32 sum on the tensor cores would leave 1e-4 off: 512
    rows by truncation are 32 steps of at most 2^-23 of a sum that grows evenly, half of that on average: 32 / 2 / 2 2^-23 = 1e-6, and the
    sums that round add a tenth.  Within 2e-6 of the 64-bit value."""
    from paper_2111_06483_b200 import api
    gen = torch.Generator(device="cuda").manual_seed(0)
    h, dz = ((torch.randn(65536, 256, generator=gen, device="cuda") + 1).bfloat16() for _ in range(2))
    dw = api.typed_linear_backward_weight(h, torch.tensor([0, 65536], device="cuda"), dz)
    want = h.double().t() @ dz.double()
    assert ((dw[0].double() - want).norm() / want.norm()).item() < 2e-6


@pytest.mark.parametrize("d_in,d_out,types", [(256, 256, 8), (136, 72, 64), (64, 128, 200), (264, 40, 5)])
def test_long_chunks_with_many_ragged_ends(d_in, d_out, types):
    """Hundreds of steps a block, several segments with ragged ends in each: what a role takes for the stage that it waits for must be
    that stage's latest round.  The bound is the one above, of the whole result."""
    from paper_2111_06483_b200 import api
    n = 1_000_000
    gen = torch.Generator(device="cuda").manual_seed(d_in)
    h, dz = (torch.randn(n, d, generator=gen, device="cuda").bfloat16() for d in (d_in, d_out))
    cut = torch.randint(0, n, (types - 1,), generator=gen, device="cuda").sort().values
    o = torch.cat([cut.new_zeros(1), cut, cut.new_full((1,), n)])
    host = o.tolist()
    want = torch.stack([h[a:b].double().t() @ dz[a:b].double() for a, b in zip(host, host[1:])])
    for _ in range(3):
        dw = api.typed_linear_backward_weight(h, o, dz)
        assert ((dw.double() - want).norm() / want.norm()).item() < 2e-6
    p = api.ckpt8_pack(h)
    v = api.ckpt8_unpack(p, torch.float32).double()
    want = torch.stack([(v[a:b] + 0.5).t() @ dz[a:b].double() for a, b in zip(host, host[1:])])
    half = torch.full((d_in,), 0.5, device="cuda")
    for _ in range(3):
        dw = api.typed_linear_backward_weight(p, o, dz, beta=half)
        assert ((dw.double() - want).norm() / want.norm()).item() < 2e-6


def checkpoint_of(h):
    codes, scales = oracle.ckpt8_pack(np64(h.float()))
    return torch.tensor(codes).cuda(), torch.tensor(scales).cuda()


@pytest.mark.parametrize("sizes,d_in,d_out", [([1], 64, 64), ([17], 8, 8), ([200, 0, 1, 333], 136, 72), ([128, 600], 256, 256), ([70, 2000], 264, 264),
                                              ([31, 33, 0] * 11, 72, 520), ([40_000, 3, 25_001], 64, 128), ([5000], 520, 40)])
@pytest.mark.parametrize("affine", ["none", "gamma", "beta", "both"])
def test_weights_from_a_checkpoint(sizes, d_in, d_out, affine):
    from paper_2111_06483_b200 import binding as B
    h, W, dz, o = problem(sizes, d_in, d_out, 3, 70)
    h[0], h[-1] = 0.0, 1.0
    codes, scales = checkpoint_of(torch.nan_to_num(h.float(), posinf=1.0))
    gen = torch.Generator().manual_seed(1)
    gamma = torch.randn(d_in, generator=gen).cuda() if affine in ("gamma", "both") else None
    beta = torch.randn(d_in, generator=gen).cuda() if affine in ("beta", "both") else None
    n, G = h.shape[0], len(sizes)
    dw = torch.full((G, d_in, d_out), NAN, device="cuda")
    ws = torch.full((B.sar_linear_grouped_workspace_bytes(n, G, d_in, d_out),), 255, dtype=torch.uint8, device="cuda")
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.sar_linear_grouped_bwd_weight_ckpt8(codes, scales, gamma, beta, dz, o, dw, ws, flag)
    assert flag.item() == 0
    v, Z, off = oracle.ckpt8_unpack(codes.cpu().numpy(), scales.cpu().numpy()), clean(np64(dz)), o.cpu().numpy()
    ga = np.ones(d_in) if gamma is None else np64(gamma)
    be = np.zeros(d_in) if beta is None else np64(beta)
    want = oracle.grouped_linear_bwd(v * ga + be, np64(W), off, Z)[1]
    # the product times gamma, and beta times the column sums of dz, each in float32
    tol = weight_bound(v * ga, Z, np64(W), off, joins(n) + 4)
    tol += (32 + joins(n) + 4) * U * oracle.grouped_linear_bwd(np.broadcast_to(np.abs(be), v.shape), np64(W), off, np.abs(Z))[1]
    within(np64(dw), want, tol + 1e-30, "dw")


def test_a_checkpoint_block_of_nan_reaches_its_columns_alone():
    from paper_2111_06483_b200 import api
    h, W, dz, o = problem([100, 60], 96, 64)
    codes, scales = checkpoint_of(h)
    clean_dw = api.typed_linear_backward_weight(api.Checkpoint8(codes, scales), o, dz)
    scales[130, 1] = 255
    dw = api.typed_linear_backward_weight(api.Checkpoint8(codes, scales), o, dz)
    assert torch.equal(dw[0], clean_dw[0]) and dw[1, 32:64].isnan().all()
    assert torch.equal(dw[1, :32], clean_dw[1, :32]) and torch.equal(dw[1, 64:], clean_dw[1, 64:])


def test_one_group_without_offsets():
    from paper_2111_06483_b200 import binding as B
    h, W, dz, o = problem([777], 64, 72)
    z, dh, dw = run_all(h, W, dz, o)
    z2, dh2, dw2 = run_all(h, W, dz, None)
    assert torch.equal(z, z2) and torch.equal(dh, dh2) and torch.equal(dw, dw2)


def test_api_writes_zeros_or_leaves_rows_of_no_type():
    from paper_2111_06483_b200 import api
    h, W, dz, o = problem([100, 200], 64, 72, 40, 50)
    z, dh = api.typed_linear_forward(h, W, o), api.typed_linear_backward_input(dz, W, o)
    for out in (z, dh):
        assert not out[:40].any() and not out[-50:].any() and out[40:-50].any()
    given = torch.full((390, 72), 5.0, dtype=torch.bfloat16, device="cuda")
    again = api.typed_linear_forward(h, W, o, out=given)
    assert (given[:40] == 5).all() and (given[-50:] == 5).all() and torch.equal(given[40:-50], z[40:-50]) and again.data_ptr() == given.data_ptr()


def test_captured_and_replayed_with_other_offsets_and_values():
    from paper_2111_06483_b200 import api
    h, W, dz, o = problem([100, 0, 300], 64, 72)
    codes, scales = checkpoint_of(h)

    def step():
        return (api.typed_linear_forward(h, W, o), *api.typed_linear_backward(h, W, o, dz),
                api.typed_linear_backward_weight(api.Checkpoint8(codes, scales), o, dz, beta=torch.ones(64, device="cuda")))

    first = step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(held, first))
    o.copy_(torch.tensor([7, 7, 250, 399]))
    h2, _, dz2, _ = problem([100, 0, 300], 64, 72, seed=9)
    h.copy_(h2)
    dz.copy_(dz2)
    graph.replay()
    got = [t.clone() for t in held]
    assert all(torch.equal(a, b) for a, b in zip(got, step())) and not torch.equal(got[0], first[0])


def test_two_streams_at_once():
    from paper_2111_06483_b200 import api
    work = [problem([5000, 3, 9000], 128, 128, seed=s) for s in (1, 2)]
    want = [(api.typed_linear_forward(h, W, o), *api.typed_linear_backward(h, W, o, dz)) for h, W, dz, o in work]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in work], [None, None]
    for _ in range(3):
        for i, (h, W, dz, o) in enumerate(work):
            with torch.cuda.stream(streams[i]):
                got[i] = (api.typed_linear_forward(h, W, o), *api.typed_linear_backward(h, W, o, dz))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_more_than_2_31_values():
    from paper_2111_06483_b200 import api
    n, d = 8_600_000, 256
    h, W, dz, _ = problem([700], d, d)
    big_h, big_z = torch.zeros(n, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, d, dtype=torch.bfloat16, device="cuda")
    big_h[-700:], big_z[-700:] = h, dz
    W = torch.cat([W * 2, W])
    o = torch.tensor([0, n - 700, n], device="cuda")
    small = torch.tensor([0, 0, 700], device="cuda")
    z = api.typed_linear_forward(big_h, W, o)
    assert torch.equal(z[-700:], api.typed_linear_forward(h, W, small)[-700:]) and not z[:-700].any()
    del z
    dh = api.typed_linear_backward_input(big_z, W, o)
    assert torch.equal(dh[-700:], api.typed_linear_backward_input(dz, W, small)) and not dh[:-700].any()
    del dh
    dw = api.typed_linear_backward_weight(big_h, o, big_z)
    want = oracle.grouped_linear_bwd(np64(h), np64(W), [0, 0, 700], np64(dz))[1]
    within(np64(dw), want, weight_bound(np64(h), np64(dz), np64(W), [0, 0, 700], 4) + 1e-30, "dw")
    codes, scales = torch.zeros(n, d, dtype=torch.int8, device="cuda"), torch.zeros(n, d // 32, dtype=torch.uint8, device="cuda")
    codes[-700:], scales[-700:] = checkpoint_of(h)
    dw = api.typed_linear_backward_weight(api.Checkpoint8(codes, scales), o, big_z)
    v = oracle.ckpt8_unpack(codes[-700:].cpu().numpy(), scales[-700:].cpu().numpy())
    want = oracle.grouped_linear_bwd(v, np64(W), [0, 0, 700], np64(dz))[1]
    within(np64(dw), want, weight_bound(v, np64(dz), np64(W), [0, 0, 700], 4) + 1e-30, "dw from the checkpoint")


def test_no_rows():
    from paper_2111_06483_b200 import api
    W, o = torch.ones(2, 16, 24, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    h, gz = torch.empty(0, 16, dtype=torch.bfloat16, device="cuda"), torch.empty(0, 24, dtype=torch.bfloat16, device="cuda")
    assert api.typed_linear_forward(h, W, o).shape == (0, 24)
    dh, dW = api.typed_linear_backward(h, W, o, gz)
    assert dh.shape == (0, 16) and dW.shape == (2, 16, 24) and not dW.any()
    c = api.Checkpoint8(torch.empty(0, 16, dtype=torch.int8, device="cuda"), torch.empty(0, 1, dtype=torch.uint8, device="cuda"))
    assert not api.typed_linear_backward_weight(c, o, gz).any()


def test_refusals():
    from paper_2111_06483_b200 import api, binding as B
    h, W, dz, o = problem([30, 10], 64, 72)
    api.typed_linear_backward(h, W, o, dz)
    c = api.Checkpoint8(*checkpoint_of(h))
    for call in (lambda: api.typed_linear_forward(h, W[:, :56].contiguous(), o), lambda: api.typed_linear_forward(h, W, o[:-1]),
                 lambda: api.typed_linear_forward(h, W, o.int()), lambda: api.typed_linear_forward(h, W, o.cpu()), lambda: api.typed_linear_forward(h, W.float(), o),
                 lambda: api.typed_linear_forward(h, W[0], o), lambda: api.typed_linear_forward(h, W, o, out=h), lambda: api.typed_linear_forward(h[:, ::2], W, o),
                 lambda: api.typed_linear_backward_input(h, W, o), lambda: api.typed_linear_backward_weight(h, o, dz[:-1]),
                 lambda: api.typed_linear_backward_weight(h, o, dz.float()), lambda: api.typed_linear_backward_weight(h, o[:1], dz),
                 lambda: api.typed_linear_backward_weight(c, o, dz[:-1]), lambda: api.typed_linear_backward_weight(c, o, dz, gamma=torch.ones(63, device="cuda")),
                 lambda: api.typed_linear_backward_weight(api.Checkpoint8(c.codes, c.scales[1:]), o, dz)):
        with pytest.raises(AssertionError):
            call()
    square = problem([40], 64, 64)
    with pytest.raises(AssertionError):   # over the rows that it reads
        api.typed_linear_forward(square[0], square[1], square[3], out=square[0])
    for bad in (h.float(), ):
        with pytest.raises(B.SarError) as e:
            api.typed_linear_forward(bad, W.float(), o)
        assert e.value.code == -2
    with pytest.raises(B.SarError) as e:
        api.typed_linear_forward(h[:, :60].contiguous(), W[:, :60].contiguous(), o)
    assert e.value.code == -2


# ---- together ------------------------------------------------------------------------------------------------------------

def layer_loss_gradients(x, W, offsets, gamma, beta, gz):
    """The gradients of sum(z * gz), z = LN(x) W[type], by autograd in float64."""
    xt, Wt, gt, bt = (t.double().cpu().requires_grad_(True) for t in (x, W, gamma, beta))
    y = torch.nn.functional.layer_norm(xt, (x.shape[1],), gt, bt, 1e-5)
    z = torch.cat([y[a:b] @ Wt[g] for g, (a, b) in enumerate(oracle.group_rows(offsets.cpu().numpy(), x.shape[0]))])
    (z * gz.double().cpu()).sum().backward()
    return z.detach(), xt.grad, Wt.grad, gt.grad, bt.grad


@pytest.mark.parametrize("checkpoint", [False, True])
def test_a_typed_layer_forward_and_backward(checkpoint):
    """The normalised projection as a training step runs it, against autograd in float64.  Kept rows: bf16 roundings of y and gy, 2^-8
    each on random signs.  Checkpoint: xhat within half a 64th of its block's largest, at most 2^-6 of it, about 2% of a value's size
    in a block of 32 normal values, which the sums over rows average out."""
    from paper_2111_06483_b200 import api
    gen = torch.Generator().manual_seed(5)
    n, d_in, d_out = 3000, 96, 72
    x, gz = (torch.randn(n, d, generator=gen).bfloat16().cuda() for d in (d_in, d_out))
    W = (torch.randn(3, d_in, d_out, generator=gen) / d_in ** 0.5).bfloat16().cuda()
    gamma, beta = torch.rand(d_in, generator=gen).cuda() + 0.5, torch.randn(d_in, generator=gen).cuda()
    o = torch.tensor([0, 1000, 1000, n]).cuda()
    z, saved = api.typed_layer_forward(x, W, o, gamma, beta, checkpoint=checkpoint)
    gx, dW, dgamma, dbeta = api.typed_layer_backward(W, o, saved, gz, gamma, beta)
    want = layer_loss_gradients(x, W, o, gamma, beta, gz)
    for got, ref, tol in zip((z, gx, dW, dgamma, dbeta), want, (0.01,) + ((0.03,) * 4 if checkpoint else (0.01,) * 4)):
        assert ((got.double().cpu() - ref).norm() / ref.norm()).item() < tol
    if checkpoint:
        ck, rstd = saved
        assert ck.nbytes == n * (d_in + 3) and rstd.numel() == n
        # a longer chain of the same calls gives the same bits
        z2, saved2 = api.typed_layer_forward(x, W, o, gamma, beta)
        assert torch.equal(z, z2) and all(torch.equal(a, b) for a, b in zip(api.typed_layer_backward(W, o, saved2, gz, gamma, beta), (gx, dW, dgamma, dbeta)))


@pytest.mark.parametrize("k", [1, 3])
def test_a_sage_layer_that_keeps_its_aggregate_in_8_bits(k):
    """Everything but dW is the plain layer's bit for bit; dW is h^T dz of the values that the checkpoint of the aggregate stands for."""
    from paper_2111_06483_b200 import api
    gen = torch.Generator().manual_seed(3)
    n, d_in, d_out = 500, 64, 72
    src, dst = (torch.randint(0, n, (4000,), generator=gen, dtype=torch.int32).cuda() for _ in range(2))
    g = api.Graph.from_coo(n, src, dst, k=k, build_parts=k > 1)
    h, gpre = (torch.randn(n, d, generator=gen).bfloat16().cuda() for d in (d_in, d_out))
    W, W_res = (torch.randn(d_in, d_out, generator=gen).bfloat16().cuda() for _ in range(2))
    pre, saved = api.sage_layer_forward(g, h, W, W_res)
    pre8, saved8 = api.sage_layer_forward(g, h, W, W_res, checkpoint=True)
    assert torch.equal(pre, pre8) and isinstance(saved8[0], api.Checkpoint8) and saved8[0].nbytes == n * (d_in + 2)
    dh, dW, dW_res = api.sage_layer_backward(g, h, W, W_res, saved, gpre)
    dh8, dW8, dW_res8 = api.sage_layer_backward(g, h, W, W_res, saved8, gpre)
    assert torch.equal(dh, dh8) and torch.equal(dW_res, dW_res8)
    codes, scales = oracle.ckpt8_pack(np64(saved[0]))
    assert np.array_equal(saved8[0].codes.cpu().numpy(), codes) and np.array_equal(saved8[0].scales.cpu().numpy(), scales)
    v, Z = oracle.ckpt8_unpack(codes, scales), np64(gpre)
    within(np64(dW8), v.T @ Z, (34 * 2.0 ** -22 + joins(n) * U) * (np.abs(v).T @ np.abs(Z)), "dW")
    with pytest.raises(AssertionError):
        api.sage_layer_backward(g, h, W, W_res, (api.Checkpoint8(saved8[0].codes[1:], saved8[0].scales), saved8[1]), gpre)
