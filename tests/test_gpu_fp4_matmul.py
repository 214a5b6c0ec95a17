"""Products of microscaled 4-bit matrices against float64 products of the values that their codes stand for."""
import numpy as np
import pytest
import torch

import fp4_reference as F
from paper_2607_14107_b200 import binding as Bd

pytestmark = pytest.mark.gpu


def matrix(rows, K, fmt, seed, spread=0.5):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, K), generator=g) * torch.exp(spread * torch.randn(K, generator=g))
    x[rows // 2] = 0.0
    c, b, _ = F.quantize(x.numpy(), fmt, 0.01)
    return torch.from_numpy(F.pack(c)).cuda(), torch.from_numpy(F.tile_scales(b)).cuda(), torch.from_numpy(F.values(c, b, fmt))


def check(M, N, K, fmt, out_dtype, ta=0.01, tb=0.37, ld=None, seed=0):
    ac, asc, av = matrix(M, K, fmt, 2 * seed + 1)
    bc, bsc, bv = matrix(N, K, fmt, 2 * seed + 2)
    ld = ld or N
    buf = torch.full((M, ld), 123.0, dtype=out_dtype, device="cuda")
    t = lambda x: None if x is None else torch.tensor([x], device="cuda")  # noqa: E731
    Bd.polestar_k_fp4_matmul(ac, asc, bc, bsc, buf[:, :N], fmt, t(ta), t(tb))
    want = (av @ bv.T) * float(np.float32(1 if ta is None else ta)) * float(np.float32(1 if tb is None else tb))
    size = (av.abs() @ bv.abs().T) * (1 if ta is None else ta) * (1 if tb is None else tb)
    got = buf[:, :N].double().cpu()
    # products are exact; every partial sum (K / 64 instructions, at most 8 parts) loses at most 2^-22 of the sum of magnitudes in the tensor
    # core's accumulator (truncation), the factor and the product with it 2^-24 each; then the output's rounding
    tol = size * (2.0 ** -22 * (K / 64 + 8) + 2.0 ** -22) + want.abs() * torch.finfo(out_dtype).eps / 2
    bad = (got - want).abs() > tol + 1e-30
    assert not bad.any(), ((got - want).abs() / (tol + 1e-30)).max().item()
    assert (buf[:, N:] == 123.0).all()
    return buf


@pytest.mark.parametrize("fmt", [F.NV, F.MX])
@pytest.mark.parametrize("M,N,K", [
    (1, 1, 64), (1, 128, 256), (3, 200, 320), (32, 256, 512), (17, 1000, 1024), (33, 130, 192), (64, 384, 2048), (40, 4096, 4096),
    (65, 129, 448), (128, 256, 256), (100, 700, 1728), (129, 300, 640), (300, 520, 960),
])
def test_products(M, N, K, fmt):
    check(M, N, K, fmt, torch.float32)


@pytest.mark.parametrize("fmt", [F.NV, F.MX])
@pytest.mark.parametrize("M,N,K,dtype", [
    (256, 256, 256, torch.float32), (257, 255, 64, torch.float32), (1000, 1100, 2048, torch.bfloat16), (513, 20000, 448, torch.bfloat16),
    (2100, 2500, 704, torch.float32), (997, 4099, 1600, torch.float32), (130, 30000, 1152, torch.bfloat16),
])
def test_products_of_many_rows(M, N, K, dtype, fmt):
    # several tiles per CTA pair, ragged last tiles, K that ends inside a ring slot
    check(M, N, K, fmt, dtype, seed=7)


@pytest.mark.parametrize("kernel", [1, 2])
@pytest.mark.parametrize("M,N,K,dtype", [
    (1, 1, 64, torch.float32), (7, 130, 448, torch.bfloat16), (128, 300, 2304, torch.float32),          # one row tile; K split in two, four, eight
    (64, 128, 4096, torch.float32), (20, 900, 8192, torch.bfloat16), (130, 400, 4160, torch.float32), (300, 520, 960, torch.bfloat16),
    (257, 1255, 1088, torch.float32), (100, 20100, 320, torch.bfloat16), (513, 9000, 448, torch.float32), (1000, 1100, 2048, torch.bfloat16),
])
def test_both_kernels(monkeypatch, kernel, M, N, K, dtype):
    monkeypatch.setenv("POLESTAR_FP4_KERNEL", str(kernel))
    Bd.polestar_reload_env()
    check(M, N, K, F.NV, dtype, ld=N + 3, seed=11)
    check(M, N, K, F.MX, dtype, seed=12)


@pytest.mark.parametrize("fmt", [F.NV, F.MX])
@pytest.mark.parametrize("M,N,K,pad", [(5, 131, 128, 3), (70, 515, 1088, 1), (260, 250, 512, 6)])
def test_products_in_bf16_with_strided_rows(M, N, K, pad, fmt):
    check(M, N, K, fmt, torch.bfloat16, ld=N + pad, seed=3)
    check(M, N, K, fmt, torch.float32, ta=None, tb=None, ld=N + pad, seed=4)


@pytest.mark.parametrize("fmt", [F.NV, F.MX])
def test_codes_and_scales_meet(fmt):
    # one non-zero group per row, every group a scale and a code of its own: a product is right only if bytes, nibbles and scale ids are
    K, G = 512, F.group(fmt)
    rows = 420
    c = np.zeros((rows, K), np.uint8)
    b = np.full((rows, K // G), 0 if fmt == F.NV else 1, np.uint8)
    for r in range(rows):
        for g in range(K // G):
            if (r + g) % 3 == 0:
                c[r, g * G + (r * 7 + g) % G] = 1 + (r + 5 * g) % 15
                b[r, g] = (40 + (3 * r + 11 * g) % 40) if fmt == F.NV else 118 + (3 * r + 5 * g) % 18
    v = torch.from_numpy(F.values(c, b, fmt))
    codes, scales = torch.from_numpy(F.pack(c)).cuda(), torch.from_numpy(F.tile_scales(b)).cuda()
    one_c = np.tile(np.array([2], np.uint8), (K, K)) * np.eye(K, dtype=np.uint8)        # code 2 is 1.0: the identity
    one_b = np.full((K, K // G), 56 if fmt == F.NV else 127, np.uint8)                   # scale 1.0
    eye_c, eye_s = torch.from_numpy(F.pack(one_c)).cuda(), torch.from_numpy(F.tile_scales(one_b)).cuda()
    for M in (rows, 31, 64, 160):
        out = torch.zeros((M, K), device="cuda")
        a_scales = torch.from_numpy(F.tile_scales(b[:M])).cuda()
        Bd.polestar_k_fp4_matmul(codes[:M].contiguous(), a_scales, eye_c, eye_s, out, fmt)
        assert torch.equal(out.cpu().double(), v[:M])
    out = torch.zeros((K, rows), device="cuda")
    Bd.polestar_k_fp4_matmul(eye_c, eye_s, codes, scales, out, fmt)
    assert torch.equal(out.cpu().double(), v.T)


def test_quantised_rows_into_a_product():
    # activations quantised on the device, NaN in one row: that row alone is NaN
    M, N, K = 37, 260, 512
    x = torch.randn((M, K), generator=torch.Generator().manual_seed(1)).bfloat16()
    x[5, 77] = float("nan")
    x[6, 3] = float("-inf")
    xc = torch.empty((M, K // 2), dtype=torch.uint8, device="cuda")
    xs = torch.empty(Bd.polestar_k_fp4_scale_bytes(M, K, F.NV, Bd.SCALES_TILED), dtype=torch.uint8, device="cuda")
    t = torch.tensor([0.02], device="cuda")
    Bd.polestar_k_fp4_quantize(x.cuda(), xc, xs, F.NV, Bd.SCALES_TILED, tensor_scale=t)
    wc, ws, wv = matrix(N, K, F.NV, 9)
    out = torch.zeros((M, N), device="cuda")
    Bd.polestar_k_fp4_matmul(xc, xs, wc, ws, out, F.NV, t)
    c, b, v = F.quantize(x.float().numpy(), F.NV, 0.02)
    want = torch.from_numpy(v) @ wv.T
    rows = [r for r in range(M) if r not in (5, 6)]
    got = out.double().cpu()
    assert torch.isnan(got[[5, 6]]).all()
    size = torch.from_numpy(np.abs(v)) @ wv.abs().T
    assert ((got - want).abs()[rows] <= size[rows] * 2.0 ** -22 * (K / 64 + 9)).all()


def test_nothing_to_compute():
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda")  # noqa: E731
    Bd.polestar_k_fp4_matmul(u8(0, 32), u8(0), u8(5, 32), u8(512), torch.empty((0, 5), device="cuda"), F.NV)
    Bd.polestar_k_fp4_matmul(u8(5, 32), u8(512), u8(0, 32), u8(0), torch.empty((5, 0), device="cuda"), F.NV)
    torch.cuda.synchronize()
