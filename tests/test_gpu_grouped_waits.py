"""Waits inside the products by group that run out: with a limit of 0 a wait gives up that is not over at the first look, which the
first copy of every block never is.  A block that gives up leaves nothing in flight, and the device goes on."""
import pytest
import torch

pytestmark = pytest.mark.gpu
SHAPES = [([5], 64, 64), ([200, 0, 1, 333], 72, 40), ([700, 900], 256, 256), ([3000, 1, 40_000], 264, 264), ([500, 70], 520, 392)]


def problem(sizes, d_in, d_out):
    gen = torch.Generator().manual_seed(d_in + sum(sizes))
    n = sum(sizes)
    h, dz, W = torch.randn(n, d_in, generator=gen), torch.randn(n, d_out, generator=gen), torch.randn(len(sizes), d_in, d_out, generator=gen)
    offsets = torch.tensor([0, *sizes]).cumsum(0)
    return [t.bfloat16().cuda() for t in (h, W, dz)] + [offsets.cuda()]


def calls(sizes, d_in, d_out):
    """The four calls on prepared arrays: (call(flag), result) each."""
    from paper_2111_06483_b200 import api, binding as B
    h, W, dz, o = problem(sizes, d_in, d_out)
    n, G = h.shape[0], len(sizes)
    c = api.ckpt8_pack(h)
    half = torch.full((d_in,), 0.5, device="cuda")
    z, dh = torch.empty_like(dz), torch.empty_like(h)
    dw, dw8 = (torch.empty(G, d_in, d_out, device="cuda") for _ in range(2))
    ws = torch.empty(B.sar_linear_grouped_workspace_bytes(n, G, d_in, d_out), dtype=torch.uint8, device="cuda")
    return [(lambda f: B.sar_linear_grouped(h, W, o, z, 0, f), z), (lambda f: B.sar_linear_grouped_bwd_input(dz, W, o, dh, 0, f), dh),
            (lambda f: B.sar_linear_grouped_bwd_weight(h, dz, o, dw, ws, f), dw),
            (lambda f: B.sar_linear_grouped_bwd_weight_ckpt8(c.codes, c.scales, half, half, dz, o, dw8, ws, f), dw8)]


@pytest.fixture
def no_patience():
    """Inside the returned call a launch has no time to wait."""
    from paper_2111_06483_b200 import binding as B

    def run(call, *args):
        B.sar_set_wait_limit(0)
        try:
            call(*args)
        finally:
            assert B.sar_set_wait_limit(-1) == 0
        torch.cuda.synchronize()
    return run


@pytest.mark.parametrize("sizes,d_in,d_out", SHAPES)
def test_a_wait_that_runs_out_is_told_and_the_device_goes_on(sizes, d_in, d_out, no_patience):
    for call, out in calls(sizes, d_in, d_out):
        flag = torch.zeros(1, dtype=torch.int32, device="cuda")
        call(flag)
        want = out.clone()
        assert flag.item() == 0
        for _ in range(3):
            flag.zero_()
            no_patience(call, flag)
            assert flag.item() == 1
        flag.zero_()
        out.fill_(float("nan"))
        call(flag)
        assert flag.item() == 0 and torch.equal(out, want)


@pytest.mark.parametrize("sizes,d_in,d_out", SHAPES)
def test_results_of_a_launch_that_gave_up_are_nan(sizes, d_in, d_out, no_patience):
    """Whatever the arrays and the scratch held before: each value is NaN, or right where its block did not have to wait."""
    for call, out in calls(sizes, d_in, d_out):
        flag = torch.zeros(1, dtype=torch.int32, device="cuda")
        call(flag)
        want = out.clone()
        assert not want.isnan().any()
        out.fill_(7.0)
        no_patience(call, flag)
        assert flag.item() == 1 and out.isnan().any() and (out.isnan() | (out == want)).all()


def test_the_next_call_of_the_api_reports_it(no_patience):
    from paper_2111_06483_b200 import api, binding as B
    n, d = 500, 64
    h, W, dz, o = problem([200, 300], d, d)
    c, square = api.ckpt8_pack(h), W[0].contiguous()
    gen = torch.Generator().manual_seed(3)
    g = api.Graph.from_coo(n, *(torch.randint(0, n, (4000,), generator=gen, dtype=torch.int32).cuda() for _ in range(2)))
    _, saved = api.sage_layer_forward(g, h, square, square, checkpoint=True)
    for call in (lambda: api.typed_linear_forward(h, W, o), lambda: api.typed_linear_backward_input(dz, W, o), lambda: api.typed_linear_backward_weight(h, o, dz),
                 lambda: api.typed_linear_backward_weight(c, o, dz), lambda: api.sage_layer_backward(g, h, square, square, saved, dz)[1]):
        want, got = call(), []
        no_patience(lambda: got.append(call()))
        assert got[0].isnan().any()
        with pytest.raises(B.SarError) as e:
            call()
        assert e.value.code == B.SAR_ERR_WAIT
        assert torch.equal(call(), want)   # reported once


def test_a_replayed_graph_reports_it_to_the_next_call(no_patience):
    from paper_2111_06483_b200 import api, binding as B
    h, W, dz, o = problem([200, 300], 64, 64)
    want = api.typed_linear_forward(h, W, o)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        no_wait_z = []
        B.sar_set_wait_limit(0)
        no_wait_z.append(api.typed_linear_forward(h, W, o))
        B.sar_set_wait_limit(-1)
    graph.replay()
    torch.cuda.synchronize()
    assert no_wait_z[0].isnan().any()
    with pytest.raises(B.SarError):
        api.typed_linear_forward(h, W, o)
    assert torch.equal(api.typed_linear_forward(h, W, o), want)


def test_the_first_call_of_a_process_may_be_captured():
    """The word that tells of waits is set up by the first call, whose host memory a capture must not refuse."""
    import subprocess
    import sys
    code = """
import torch
from paper_2111_06483_b200 import api
h = torch.randn(300, 64, device="cuda").bfloat16()
W = torch.randn(2, 64, 72, device="cuda").bfloat16()
o = torch.tensor([0, 100, 300], device="cuda")
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    z = api.typed_linear_forward(h, W, o)
graph.replay()
torch.cuda.synchronize()
assert torch.equal(z, api.typed_linear_forward(h, W, o)) and z.any()
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
