"""The 4-bit operators at the ends of what their arguments may be: factors, rows and scores far from what models hold."""
import numpy as np
import pytest
import torch

import fp4_reference as F
from paper_2607_14107_b200 import binding as Bd
from test_gpu_fp4 import check_rows, f32

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def quantised(x, fmt, t):
    codes = torch.full((x.shape[0], x.shape[1] // 2), 0x55, dtype=torch.uint8, device="cuda")
    scales = torch.full((x.shape[0], x.shape[1] // F.group(fmt)), 0x55, dtype=torch.uint8, device="cuda")
    deq = torch.full_like(x, 3.0)
    Bd.polestar_k_fp4_quantize(x, codes, scales, fmt, tensor_scale=torch.tensor([t], device="cuda"), deq=deq)
    return codes, scales, deq


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", [F.NV, F.MX])
@pytest.mark.parametrize("t,size", [(1e-30, 3e9), (1e-25, 1e15), (2e-13, 1.2e30), (1.3e-30, 1.2e30)])
def test_scale_of_a_quotient_beyond_fp32(t, size, fmt, dtype):
    # maximum and divisor are ordinary numbers, their quotient is not one of fp32: the scale saturates
    x = (torch.rand((8, 64), generator=torch.Generator().manual_seed(1)) * 0.9 + 0.1) * size          # (positive: the codes' signs are the next test's)
    x = x.to(DT[dtype]).cuda()
    codes, scales, deq = quantised(x, fmt, t)
    check_rows(x, codes.cpu().numpy(), scales.cpu().numpy(), deq, fmt, t, Bd.SCALES_ROWS)
    assert (scales.cpu() == (0x7E if fmt == F.NV else 0xFE)).all()


def far_rows(rows, d, dtype, seed):
    """Ordinary rows with entries of either sign up to the type's largest, in every place of a group."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, d), generator=g)
    top = torch.finfo(DT[dtype]).max
    big = torch.tensor([-top, top, -3.3e37, 3.3e37, -1.3e36, 1e30, -1e20, -1e10])
    for r in range(rows):
        x[r, torch.randperm(d, generator=g)[:1 + d // 40]] = big[r % 8] * (1.0 if r % 3 else 0.75)
    return x.to(DT[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", [F.NV, F.MX])
@pytest.mark.parametrize("t", [1e-3, 2.5e-4, 0.00021, 1e-12, 2.0 ** -126, 0.7, 1e6])
def test_codes_of_quotients_beyond_fp32(t, fmt, dtype):
    # |x| / (s t) of a saturated group overflows: the code is 6 with the sign of x
    x = far_rows(64, 160, dtype, 2).cuda()
    codes, scales, deq = quantised(x, fmt, t)
    check_rows(x, codes.cpu().numpy(), scales.cpu().numpy(), deq, fmt, t, Bd.SCALES_ROWS)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t", [1e-3, 0.00021, 1e-12])
def test_appended_rows_beyond_fp32(t, dtype):
    b, R, nkv, dh = 2, 24, 2, 64
    k, v = (far_rows(b * R, nkv * dh, dtype, s).view(b, R, nkv * dh).cuda() for s in (3, 4))
    kc, vc = (torch.zeros((b, R, nkv, dh // 2), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros((b, R, nkv, dh // 16), dtype=torch.uint8, device="cuda") for _ in range(2))
    ts = torch.tensor([t], device="cuda")
    Bd.polestar_k_kv4_append(k, v, None, None, kc, ks, vc, vs, ts, ts)
    for x, c, s in ((k, kc, ks), (v, vc, vs)):
        want_c, want_s, _ = F.quantize(f32(x).reshape(b, R, nkv, dh), F.NV, t)
        assert np.array_equal(c.cpu().numpy(), F.pack(want_c)) and np.array_equal(s.cpu().numpy(), want_s)
