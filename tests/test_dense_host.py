"""Host-side rules of the layer normalisation, the 8-bit checkpoints and the products by group that need no device."""
import pytest

from paper_2111_06483_b200 import binding as B, build


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


def test_the_wait_limit_is_told_back_and_a_negative_one_brings_the_default_back():
    assert B.sar_set_wait_limit(7) == 4_000_000_000
    assert B.sar_set_wait_limit(0) == 7
    assert B.sar_set_wait_limit(-1) == 0
    assert B.sar_set_wait_limit(-5) == 4_000_000_000


def test_a_wait_that_ran_out_has_a_status_of_its_own():
    assert B.lib().sar_status_string(B.SAR_ERR_WAIT).startswith(b"a wait inside a kernel ran out")


@pytest.mark.parametrize("groups,d_in,d_out", [(1, 256, 256), (8, 64, 64), (64, 136, 72), (3, 200, 120), (2, 520, 392), (1024, 8, 8)])
def test_scratch_for_many_rows_suffices_for_fewer(groups, d_in, d_out):
    """The rows are cut into chunks of whole steps, so one row more can mean half as many chunks (256 x 256: 74 of 64 rows for 4,736
    rows, 38 of 128 for 4,737)."""
    rows = [1, 63, 64, 65, *range(100, 20_000, 61), 4736, 4737, 9472, 9473, 10 ** 6, 10 ** 6 + 1, 2 * 10 ** 9]
    size = [B.sar_linear_grouped_workspace_bytes(n, groups, d_in, d_out) for n in sorted(rows)]
    assert size == sorted(size)


def test_scratch_of_the_normalisation_follows_the_records():
    record = 2 * 4
    for C in (1, 47, 64, 1000, 8192, 8193, 1 << 20):
        size = [B.sar_ln_workspace_bytes_rows(n, C) for n in (0, 1, 2, 3, 64, 65, 300, 5000, 10 ** 6, 2 ** 40)]
        assert size == sorted(size) and size[-1] <= B.sar_ln_workspace_bytes(C)
        assert size[1] >= record * C
    assert B.sar_ln_workspace_bytes_rows(300, 1000) < 160 * record * 1000
    assert B.sar_ln_workspace_bytes_rows(300, 1 << 20) < 6 * record * (1 << 20)
    assert B.sar_ln_workspace_bytes(1 << 20) < 150 * record * (1 << 20)
    for n, C in ((-1, 64), (5, 0), (5, (1 << 20) + 1)):
        assert B.sar_ln_workspace_bytes_rows(n, C) == 0
    assert B.sar_ln_workspace_bytes((1 << 20) + 1) == 0   # which the calls refuse


def test_refusals_of_the_normalisation_s_gradients_by_group():
    from ctypes import c_int32, c_int64, c_size_t, c_void_p
    lib, P, odd, null, lots = B.lib(), c_void_p(1 << 20), c_void_p((1 << 20) + 4), c_void_p(0), c_size_t(1 << 40)
    rows = (c_int64(10), c_int32(3), c_int32(64), 0, P, P, P, P, P, P, P, P, P, P, lots, null)      # n, groups, C, t, offsets, x, mean, rstd, gamma, gy, gx, ...
    packed = (c_int64(10), c_int32(3), c_int32(64), 0, P, P, P, P, P, P, P, P, P, P, lots, null)    # ... offsets, codes, scales, rstd, gamma, gy, gx, ...
    for fn, good in ((lib.sar_ln_bwd_grouped, rows), (lib.sar_ln_bwd_ckpt8_grouped, packed)):
        for status, at, value in ((-1, 0, c_int64(-1)), (-1, 1, c_int32(0)), (-2, 1, c_int32(1025)), (-1, 2, c_int32(0)), (-1, 3, 7), (-1, 4, null), (-3, 4, odd),
                                  (-1, 5, null), (-1, 6, null), (-1, 7, null), (-1, 9, null), (-1, 10, null), (-4, 13, null), (-4, 14, c_size_t(64))):
            args = list(good)
            args[at] = value
            assert fn(*args) == status, (fn.__name__, at)
