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
