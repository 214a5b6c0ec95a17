"""The 4-bit operators at the ends of what their arguments may be: factors, rows and scores far from what models hold."""
import pytest
import torch

import fp4_reference as F
from paper_2607_14107_b200 import binding as Bd
from test_gpu_fp4 import check_rows

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
