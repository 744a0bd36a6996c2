"""Refusals of the layer normalisation, the 8-bit checkpoints and the products by groups of rows.  The library checks its
arguments on the host before anything is launched, so these run without a device: the addresses are never followed."""
import ctypes
from ctypes import c_float, c_int32, c_int64, c_size_t, c_uint32, c_void_p

import pytest
import torch

F32, BF16 = 0, 1
INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE = -1, -2, -3, -4
P = c_void_p(1 << 20)          # aligned to everything
ODD = c_void_p((1 << 20) + 1)
HALF = c_void_p((1 << 20) + 8)
NULL = c_void_p(0)
LOTS = c_size_t(1 << 40)


@pytest.fixture(scope="module")
def lib():
    from paper_2111_06483_b200 import binding, build
    build.build()
    return binding.lib()


def refused(fn, good, *cases):
    """fn(*good) with the arguments of each case replaced ({position: value}) returns the case's status."""
    for status, change in cases:
        args = list(good)
        for at, value in change.items():
            args[at] = value
        assert fn(*args) == status, (fn.__name__, change)


def test_checkpoint(lib):
    n, C = c_int64(10), c_int32(64)
    pack = (n, C, F32, P, P, P, NULL)        # x, codes, scales
    unpack = (n, C, F32, P, P, P, NULL)      # codes, scales, x
    common = [(INVALID, {0: c_int64(-1)}), (INVALID, {1: c_int32(0)}), (INVALID, {2: 7}), (UNSUPPORTED, {1: c_int32((1 << 20) + 1)}),
              (INVALID, {3: NULL}), (INVALID, {4: NULL}), (INVALID, {5: NULL})]
    refused(lib.sar_ckpt8_pack, pack, *common, (ALIGNMENT, {3: ODD}))
    refused(lib.sar_ckpt8_unpack, unpack, *common, (ALIGNMENT, {5: ODD}))
    assert lib.sar_ckpt8_pack(c_int64(0), C, BF16, NULL, NULL, NULL, NULL) == 0
    assert lib.sar_ckpt8_unpack(c_int64(0), C, BF16, NULL, NULL, NULL, NULL) == 0


def test_layer_norm(lib):
    n, C = c_int64(10), c_int32(64)
    eps = c_float(1e-5)
    fwd = (n, C, F32, P, P, P, eps, P, P, P, NULL)                  # x, gamma, beta, eps, y, mean, rstd
    refused(lib.sar_ln_fwd, fwd, (INVALID, {0: c_int64(-1)}), (INVALID, {1: c_int32(0)}), (INVALID, {2: 5}), (INVALID, {3: NULL}),
            (INVALID, {7: NULL}), (INVALID, {6: c_float(-1.0)}), (INVALID, {6: c_float(float("nan"))}), (UNSUPPORTED, {1: c_int32((1 << 20) + 1)}),
            (ALIGNMENT, {3: ODD}), (ALIGNMENT, {7: ODD}), (ALIGNMENT, {4: ODD}), (ALIGNMENT, {8: ODD}), (ALIGNMENT, {9: ODD}))
    packed = (n, C, BF16, P, P, P, eps, P, P, P, P, NULL)           # ..., y, rstd, codes, scales
    refused(lib.sar_ln_fwd_ckpt8, packed, (INVALID, {8: NULL}), (INVALID, {9: NULL}), (INVALID, {10: NULL}), (ALIGNMENT, {8: ODD}))
    bwd = (n, C, F32, P, P, P, P, P, P, P, P, P, LOTS, NULL)        # x, mean, rstd, gamma, gy, gx, dgamma, dbeta, ws
    refused(lib.sar_ln_bwd, bwd, (INVALID, {3: NULL}), (INVALID, {4: NULL}), (INVALID, {5: NULL}), (INVALID, {7: NULL}), (INVALID, {8: NULL}),
            (WORKSPACE, {11: NULL}), (WORKSPACE, {11: ODD}), (WORKSPACE, {12: c_size_t(64)}), (WORKSPACE, {12: c_size_t(64), 9: NULL}),
            (ALIGNMENT, {7: ODD}), (ALIGNMENT, {9: ODD}), (UNSUPPORTED, {1: c_int32((1 << 20) + 1)}))
    bwd8 = (n, C, BF16, P, P, P, P, P, P, P, P, P, LOTS, NULL)      # codes, scales, rstd, gamma, gy, gx, dgamma, dbeta, ws
    refused(lib.sar_ln_bwd_ckpt8, bwd8, (INVALID, {3: NULL}), (INVALID, {4: NULL}), (INVALID, {5: NULL}), (INVALID, {7: NULL}),
            (WORKSPACE, {11: NULL}), (ALIGNMENT, {8: ODD}))
    for C in (1, 64, 5000):
        assert lib.sar_ln_workspace_bytes(c_int32(C)) >= 2 * C * 4
    assert lib.sar_ln_workspace_bytes(c_int32(0)) == 0


def test_grouped_products(lib):
    n, G, di, do = c_int64(100), c_int32(3), c_int32(64), c_int32(32)
    rows = (n, G, di, do, BF16, P, P, P, P, c_uint32(0), NULL, NULL)   # offsets, h, w, z, flags, flag
    bad_sizes = [(INVALID, {0: c_int64(-1)}), (INVALID, {1: c_int32(0)}), (INVALID, {2: c_int32(0)}), (INVALID, {3: c_int32(-8)}), (UNSUPPORTED, {4: F32}),
                 (INVALID, {4: 9}), (UNSUPPORTED, {1: c_int32(1025)}), (UNSUPPORTED, {2: c_int32(60)}), (UNSUPPORTED, {3: c_int32(4)}),
                 (UNSUPPORTED, {0: c_int64(2 ** 31)}), (UNSUPPORTED, {0: c_int64(2 ** 31 - 100)}), (UNSUPPORTED, {2: c_int32((1 << 20) + 8)})]
    for fn in (lib.sar_linear_grouped, lib.sar_linear_grouped_bwd_input):
        refused(fn, rows, *bad_sizes, (INVALID, {5: NULL}), (INVALID, {6: NULL}), (INVALID, {7: NULL}), (INVALID, {8: NULL}), (INVALID, {9: c_uint32(2)}),
                (ALIGNMENT, {5: c_void_p((1 << 20) + 4)}), (ALIGNMENT, {6: HALF}), (ALIGNMENT, {7: HALF}), (ALIGNMENT, {8: HALF}))
        assert fn(c_int64(0), G, di, do, BF16, P, NULL, NULL, NULL, c_uint32(0), NULL, NULL) == 0
        assert fn(c_int64(0), G, di, do, F32, P, NULL, NULL, NULL, c_uint32(0), NULL, NULL) == UNSUPPORTED
    weight = (n, G, di, do, BF16, P, P, P, P, NULL, P, LOTS, NULL)     # offsets, h, dz, dw, flag, ws
    refused(lib.sar_linear_grouped_bwd_weight, weight, *bad_sizes, (INVALID, {5: NULL}), (INVALID, {6: NULL}), (INVALID, {7: NULL}), (INVALID, {8: NULL}),
            (ALIGNMENT, {7: HALF}), (WORKSPACE, {10: NULL}), (WORKSPACE, {10: HALF}), (WORKSPACE, {11: c_size_t(1000)}))
    packed = (n, G, di, do, BF16, P, P, P, P, P, P, P, NULL, P, LOTS, NULL)   # offsets, codes, scales, gamma, beta, dz, dw, flag, ws
    refused(lib.sar_linear_grouped_bwd_weight_ckpt8, packed, *bad_sizes, (INVALID, {6: NULL}), (INVALID, {7: NULL}), (INVALID, {10: NULL}), (INVALID, {11: NULL}),
            (ALIGNMENT, {6: c_void_p((1 << 20) + 4)}), (ALIGNMENT, {8: ODD}), (WORKSPACE, {13: NULL}), (WORKSPACE, {14: c_size_t(1000)}))
    # one record per chunk and group at least, whatever the sizes
    for n, G, di, do in ((1, 1, 8, 8), (100, 3, 64, 32), (10 ** 6, 1024, 256, 256), (2 * 10 ** 9, 7, 512, 1032)):
        assert lib.sar_linear_grouped_workspace_bytes(c_int64(n), c_int32(G), c_int32(di), c_int32(do)) >= (G + 1) * di * do * 4
    assert lib.sar_linear_grouped_workspace_bytes(c_int64(0), c_int32(1), c_int32(8), c_int32(8)) == 0


def test_results_over_operands_are_refused(lib):
    """z over any part of the rows (n d 2 bytes) or of the weights, from either side."""
    n, G, di, do, z = 100, 3, 64, 32, 1 << 24
    for fn, rows, result in ((lib.sar_linear_grouped, n * di * 2, n * do * 2), (lib.sar_linear_grouped_bwd_input, n * do * 2, n * di * 2)):
        for at, size, far in ((6, rows, 7), (7, G * di * do * 2, 6)):
            for start in (z, z + result - 16, z - size + 16):
                args = [c_int64(n), c_int32(G), c_int32(di), c_int32(do), BF16, P, P, P, c_void_p(z), c_uint32(0), NULL, NULL]
                args[at], args[far] = c_void_p(start), c_void_p(1 << 30)
                assert fn(*args) == INVALID


def test_tensors_that_are_not_on_a_device_are_refused():
    from paper_2111_06483_b200 import api
    x, o = torch.zeros(4, 32, dtype=torch.bfloat16), torch.tensor([0, 4])
    c = api.Checkpoint8(torch.zeros(4, 32, dtype=torch.int8), torch.zeros(4, 1, dtype=torch.uint8))
    for call in (lambda: api.ln_forward(x), lambda: api.ckpt8_pack(x), lambda: api.ckpt8_unpack(c), lambda: api.typed_linear_forward(x, x.view(1, 4, 32), o),
                 lambda: api.ln_backward(None, x, (c, torch.zeros(4))), lambda: api.typed_linear_backward_weight(c, o, x)):
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(AssertionError):   # gamma without a checkpoint
        api.typed_linear_backward_weight(x, o, x, gamma=torch.zeros(32))
    with pytest.raises(TypeError):
        api.ckpt8_unpack(c, torch.float16)
    assert c.nbytes == 4 * 32 + 4 and tuple(c.shape) == (4, 32)
