"""GPU parity of the 8-bit checkpoints with the float64 oracle: codes, scales and the values they stand for, bit for bit, at every
width class of the kernels, with special values, strided addresses, large arrays and under capture."""
import numpy as np
import pytest
import torch

import oracle

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def rows(n, c, dt, seed):
    """Rows of very different sizes, zeros, whole zero blocks, infinities, NaN, the type's extremes and subnormals."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, c)) * np.exp(rng.standard_normal((n, 1)) * 10)
    x[rng.random((n, c)) < 0.05] = 0.0
    x = torch.tensor(x, dtype=torch.float32)
    special = [float("inf"), float("-inf"), float("nan"), 3.38e38, -3.38e38, 1e-45, 1e-39, 0.0]
    for i in range(0, n, 7):
        x[i, rng.integers(c)] = special[i // 7 % len(special)]
    for i in range(3, n, 11):
        x[i, :32] = 0.0
    for i in range(5, n, 13):   # everything on a border between two codes: ties
        x[i] = (torch.arange(c) % 127 + 0.5) * 2.0 ** (i % 40 - 20)
    return x.to(DT[dt])


def same(a, b):
    return np.array_equal(a, b, equal_nan=True)


def check(x, codes, scales):
    from paper_2111_06483_b200 import api
    want_codes, want_scales = oracle.ckpt8_pack(x.float().cpu().numpy())
    assert np.array_equal(scales.cpu().numpy(), want_scales)
    assert np.array_equal(codes.cpu().numpy(), want_codes)
    want = oracle.ckpt8_unpack(want_codes, want_scales)
    for dt in (torch.float32, torch.bfloat16):   # exact in both
        got = api.ckpt8_unpack(api.Checkpoint8(codes, scales), dt)
        assert got.dtype == dt and same(got.double().cpu().numpy(), want)


@pytest.mark.parametrize("c", [1, 4, 8, 12, 31, 32, 33, 47, 64, 100, 256, 1000, 4104])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 203])
def test_pack_and_unpack(n, c, dt):
    from paper_2111_06483_b200 import api
    x = rows(n, c, dt, 1000 * n + c).cuda()
    p = api.ckpt8_pack(x)
    assert p.nbytes == n * c + n * ((c + 31) // 32)
    check(x, p.codes, p.scales)


@pytest.mark.parametrize("c", [2, 3, 5, 7, 9, 15, 17, 23, 36, 50, 57, 63, 95, 121, 122, 127, 166, 249, 250, 333, 505, 506, 761, 1017, 1018, 1021, 1022, 1023, 1025, 1030, 1036, 1100])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 2, 9, 5001])
def test_rows_that_are_no_whole_vectors(n, c, dt):
    """Every place within a vector that a row can start at, the last vectors of the array, and one column more or less than a kernel's
    lanes cover; many rows a lane group.  The bytes behind the codes and the values stay as they were."""
    from paper_2111_06483_b200 import binding as B
    x = rows(min(n, 203), c, dt, 1000 * n + c).repeat(-(-n // 203), 1)[:n].contiguous().cuda()
    codes = torch.full((n * c + 16,), 99, dtype=torch.int8, device="cuda")
    scales = torch.full((n * ((c + 31) // 32) + 16,), 77, dtype=torch.uint8, device="cuda")
    own, s = codes[:n * c].view(n, c), scales[:-16].view(n, -1)
    B.sar_ckpt8_pack(x, own, s)
    assert (codes[n * c:] == 99).all() and (scales[-16:] == 77).all()
    want_codes, want_scales = oracle.ckpt8_pack(x.float().cpu().numpy())
    assert np.array_equal(s.cpu().numpy(), want_scales) and np.array_equal(own.cpu().numpy(), want_codes)
    back = torch.full((n * c + 16,), 7.0, dtype=DT[dt], device="cuda")
    B.sar_ckpt8_unpack(own, s, back[:n * c].view(n, c))
    assert (back[n * c:] == 7).all() and same(back[:n * c].view(n, c).double().cpu().numpy(), oracle.ckpt8_unpack(want_codes, want_scales))


@pytest.mark.parametrize("c", [1027, 1028, 1500, 2044, 2047, 2049, 2052, 4100, 8188, 8196])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 2, 1203])
def test_rows_that_a_block_shares(n, c, dt):
    test_pack_and_unpack(n, c, dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("skip_x,skip_codes", [(1, 0), (0, 1), (4, 4), (2, 0)])
def test_addresses_that_are_not_aligned(dt, skip_x, skip_codes):
    from paper_2111_06483_b200 import binding as B
    n, c = 37, 64
    x = rows(n, c, dt, 5)
    room = torch.zeros(n * c + 8, dtype=DT[dt], device="cuda")
    xs = room[skip_x:skip_x + n * c].view(n, c)
    xs.copy_(x)
    codes = torch.full((n * c + 8,), 99, dtype=torch.int8, device="cuda")
    scales = torch.zeros(n, 2, dtype=torch.uint8, device="cuda")
    own = codes[skip_codes:skip_codes + n * c].view(n, c)
    B.sar_ckpt8_pack(xs, own, scales)
    check(x, own, scales)
    assert (codes[:skip_codes] == 99).all() and (codes[skip_codes + n * c:] == 99).all()
    back = torch.full((n * c + 8,), 7.0, dtype=DT[dt], device="cuda")
    B.sar_ckpt8_unpack(own, scales, back[skip_x:skip_x + n * c].view(n, c))
    assert same(back[skip_x:skip_x + n * c].view(n, c).double().cpu().numpy(), oracle.ckpt8_unpack(own.cpu().numpy(), scales.cpu().numpy()))
    assert (back[:skip_x] == 7).all() and (back[skip_x + n * c:] == 7).all()


def test_whatever_the_codes_the_bytes_0_and_255_stand_for_zeros_and_nan():
    from paper_2111_06483_b200 import api
    codes = torch.arange(-127, 128, dtype=torch.int8, device="cuda")[:128].repeat(3, 1).contiguous()
    scales = torch.tensor([[0, 255, 127, 1]] * 3, dtype=torch.uint8, device="cuda")
    v = api.ckpt8_unpack(api.Checkpoint8(codes, scales), torch.float32)
    assert same(v.double().cpu().numpy(), oracle.ckpt8_unpack(codes.cpu().numpy(), scales.cpu().numpy()))
    assert (v[:, :32] == 0).all() and v[:, 32:64].isnan().all()


def test_no_rows():
    from paper_2111_06483_b200 import api
    p = api.ckpt8_pack(torch.empty(0, 40, device="cuda"))
    assert p.codes.shape == (0, 40) and p.scales.shape == (0, 2) and api.ckpt8_unpack(p).shape == (0, 40)


@pytest.mark.parametrize("c", [256, 100])
def test_more_than_2_31_values(c):
    """Offsets beyond 32 bits: the last rows of an array of 2.2 thousand million values."""
    from paper_2111_06483_b200 import api
    n = 2_200_000_000 // c
    x = torch.zeros(n, c, dtype=torch.bfloat16, device="cuda")
    x[-301:] = rows(301, c, "bf16", 3).cuda()
    x[:7] = rows(7, c, "bf16", 4).cuda()
    p = api.ckpt8_pack(x)
    for part in (slice(0, 7), slice(n - 301, n)):
        codes, scales = oracle.ckpt8_pack(x[part].float().cpu().numpy())
        assert np.array_equal(p.codes[part].cpu().numpy(), codes) and np.array_equal(p.scales[part].cpu().numpy(), scales)
    back = api.ckpt8_unpack(p)
    want = oracle.ckpt8_unpack(p.codes[-301:].cpu().numpy(), p.scales[-301:].cpu().numpy())
    assert same(back[-301:].double().cpu().numpy(), want) and not back[7:-301].any()


def test_captured_and_replayed_on_other_values():
    from paper_2111_06483_b200 import api
    x = rows(64, 96, "bf16", 1).cuda()
    api.ckpt8_unpack(api.ckpt8_pack(x))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p = api.ckpt8_pack(x)
        v = api.ckpt8_unpack(p)
    other = rows(64, 96, "bf16", 2).cuda()
    x.copy_(other)
    graph.replay()
    check(other, p.codes, p.scales)
    assert same(v.double().cpu().numpy(), oracle.ckpt8_unpack(p.codes.cpu().numpy(), p.scales.cpu().numpy()))


def test_refusals():
    from paper_2111_06483_b200 import api, binding as B
    x = torch.zeros(8, 64, device="cuda")
    p = api.ckpt8_pack(x)
    for bad in (x.half(), x.double(), x.long()):
        with pytest.raises(TypeError):
            api.ckpt8_pack(bad)
    for bad in (x.t(), x[:, ::2]):
        with pytest.raises(AssertionError):
            api.ckpt8_pack(bad)
    with pytest.raises(ValueError):
        api.ckpt8_pack(x.view(-1))
    for codes, scales in ((p.codes.int(), p.scales), (p.codes, p.scales.int()), (p.codes, p.scales[:-1]), (p.codes, p.scales.cpu())):
        with pytest.raises(AssertionError):
            api.ckpt8_unpack(api.Checkpoint8(codes, scales))
    with pytest.raises(AssertionError):
        B.sar_ckpt8_pack(x, p.codes[:-1], p.scales)
