"""Rows in microscaled 4-bit floating point and rows of a 4-bit K/V cache, byte for byte against their definition."""
import numpy as np
import pytest
import torch

import fp4_reference as F
from paper_2607_14107_b200 import binding as Bd

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def rows_of(shape, seed, dtype, special=False):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * torch.exp(0.7 * torch.randn(shape[-1], generator=g))
    x[..., 3::7] = torch.round(x[..., 3::7] * 4) / 4              # values next to and on the middles between codes
    if special:
        r = x.reshape(-1, 32)
        r[0] = 0.0
        r[1 % len(r), 5] = float("nan")
        r[2 % len(r), 31] = float("inf")
        r[3 % len(r), :16] = -float("inf")
        r[4 % len(r)] = 1e-42                                        # subnormal: the scale is zero (nv) or the smallest (mx)
        r[5 % len(r)] *= 1e37                                        # the scale saturates
        r[6 % len(r)] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] * 2 + [-0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, -6.0] * 2)
        r[7 % len(r)] = -0.0
        r[8 % len(r)] *= 1e-37
        r[9 % len(r)] = 2.0 ** -7                                    # between zero and the smallest scale
    return x.to(dtype)


def f32(t):
    return t.detach().float().cpu().numpy()


def check_rows(x, codes, scales, deq, fmt, t, layout):
    c, b, v = F.quantize(f32(x), fmt, t)
    assert np.array_equal(codes, F.pack(c))
    assert np.array_equal(scales.reshape(-1), (F.tile_scales(b) if layout == Bd.SCALES_TILED else b).reshape(-1))
    if deq is not None:
        # (value times factor in fp32, then the row's type: each rounds once, float64 products of the formats' values are exact)
        with np.errstate(over="ignore"):
            grid_s = F.values(c, b, fmt).astype(np.float32)
            want = torch.from_numpy((grid_s * np.float32(t)).astype(np.float32)).to(deq.dtype)
        assert torch.equal(torch.nan_to_num(deq.cpu().float(), nan=12345.0), torch.nan_to_num(want.float(), nan=12345.0))


@pytest.mark.parametrize("fmt", [F.NV, F.MX])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d,t,layout", [
    (1, 32, None, 0), (1, 32, 0.0123, 1), (3, 64, None, 1), (130, 96, 0.37, 0), (130, 96, 0.37, 1), (33, 4096, 0.0123, 1),
    (257, 160, None, 1), (128, 128, 1.0, 1), (127, 18944, 2.5e-4, 0), (9000, 1024, 0.5, 1), (2500, 4096, None, 0),
])
def test_quantize_rows(dtype, fmt, rows, d, t, layout):
    x = rows_of((rows, d), rows + d, DT[dtype], special=True).cuda()
    codes = torch.full((rows, d // 2), 0xAA, dtype=torch.uint8, device="cuda")
    scales = torch.full((Bd.polestar_k_fp4_scale_bytes(rows, d, fmt, layout),), 0xAA, dtype=torch.uint8, device="cuda")
    deq = torch.full_like(x, 77.0)
    ts = None if t is None else torch.tensor([t], device="cuda")
    Bd.polestar_k_fp4_quantize(x, codes, scales, fmt, layout, tensor_scale=ts, deq=deq)
    check_rows(x, codes.cpu().numpy(), scales.cpu().numpy(), deq, fmt, 1.0 if t is None else t, layout)
    # without the stored values, and from rows that lie in a wider matrix
    wide = torch.full((rows, d + 64), float("nan"), dtype=x.dtype, device="cuda")
    wide[:, 32:32 + d] = x
    c2, s2 = torch.full_like(codes, 0x55), torch.full_like(scales, 0x55)
    Bd.polestar_k_fp4_quantize(wide[:, 32:32 + d], c2, s2, fmt, layout, tensor_scale=ts)
    assert torch.equal(codes, c2) and torch.equal(scales, s2)


@pytest.mark.parametrize("t", [1e-30, 2.0 ** -130, 1e30, 3.0])
@pytest.mark.parametrize("fmt", [F.NV, F.MX])
def test_quantize_far_factors(fmt, t):
    # units beyond the range of the reciprocal's correction step divide
    x = (torch.randn((64, 256), generator=torch.Generator().manual_seed(3)) * (t if t > 1e-35 else 1e-36)).cuda()
    codes = torch.empty((64, 128), dtype=torch.uint8, device="cuda")
    scales = torch.empty((64, 256 // F.group(fmt)), dtype=torch.uint8, device="cuda")
    Bd.polestar_k_fp4_quantize(x, codes, scales, fmt, tensor_scale=torch.tensor([t], device="cuda"))
    check_rows(x, codes.cpu().numpy(), scales.cpu().numpy(), None, fmt, t, Bd.SCALES_ROWS)


def test_quantize_quotients_next_to_the_middles():
    # every unit of a sweep against numerators within three ulps of (middle x unit): the decision is the IEEE quotient's
    g = torch.Generator().manual_seed(5)
    t = 0.7310585
    rows = []
    for i in range(512):
        amax = np.float32(torch.rand((), generator=g).item() * 10 + 0.01)
        s = F.E4M3[F.e4m3_byte(np.array([amax / np.float32(np.float32(t) * np.float32(6))], np.float32))[0]]
        u = np.float32(np.float32(s) * np.float32(t))
        row = [amax]
        for mid in (0.25, 0.75, 1.25, 1.75, 2.5):
            x = np.float32(np.float32(mid) * u)
            row += [np.nextafter(x, np.float32(0)), x, np.nextafter(x, np.float32(100))]
        rows.append([v if abs(v) <= amax else np.float32(0) for v in row] * 2)
    x = torch.tensor(np.array(rows, np.float32)).cuda()
    codes = torch.empty((512, 16), dtype=torch.uint8, device="cuda")
    scales = torch.empty((512, 2), dtype=torch.uint8, device="cuda")
    Bd.polestar_k_fp4_quantize(x, codes, scales, F.NV, tensor_scale=torch.tensor([t], device="cuda"))
    check_rows(x, codes.cpu().numpy(), scales.cpu().numpy(), None, F.NV, t, Bd.SCALES_ROWS)


def test_empty_inputs_touch_nothing():
    e = torch.empty((0, 64), device="cuda")
    u8 = lambda *s: torch.empty(s, dtype=torch.uint8, device="cuda")  # noqa: E731
    Bd.polestar_k_fp4_quantize(e, u8(0, 32), u8(0), F.NV)
    Bd.polestar_k_kv4_append(torch.empty((2, 0, 128), device="cuda"), torch.empty((2, 0, 128), device="cuda"), None, None,
                             u8(2, 5, 2, 32), u8(2, 5, 2, 4), u8(2, 5, 2, 32), u8(2, 5, 2, 4))
    torch.cuda.synchronize()


def cache(b, cap, nkv, dh, fill):
    mk = lambda w: torch.full((b, cap, nkv, w), fill, dtype=torch.uint8, device="cuda")  # noqa: E731
    return mk(dh // 2), mk(dh // 16), mk(dh // 2), mk(dh // 16)


@pytest.mark.parametrize("dtype,b,R,cap,nkv,dh,tk,tv", [
    ("bf16", 1, 1, 1, 1, 64, None, None),
    ("bf16", 3, 37, 200, 4, 128, 0.0173, 0.0031),
    ("f32", 3, 29, 1021, 4, 64, 0.02, None),
    ("f32", 2, 70, 70, 1, 128, None, 0.01),
    ("bf16", 2, 300, 512, 32, 128, 0.02, 0.02),
    ("bf16", 5, 777, 800, 1, 64, 0.02, 0.02),
])
def test_append(dtype, b, R, cap, nkv, dh, tk, tv):
    k, v = (rows_of((b, R, nkv * dh), s, DT[dtype], special=s == 1).cuda() for s in (1, 2))
    rng = np.random.default_rng(R)
    idx = np.full((b, R), -7, np.int32)
    counts = np.zeros(b, np.int32)
    for s in range(b):
        counts[s] = (R, 0, max(1, R - 3))[s % 3]
        idx[s] = rng.integers(-2, cap + 2, R) if s == 2 else np.sort(rng.permutation(cap)[:R]) if cap >= R else rng.integers(0, cap, R)
        if s == 2 and R > 4:
            idx[s, [0, R // 2, R - 4]] = idx[s, 1]                     # the same position several times, also far apart
    kc, ks, vc, vs = cache(b, cap, nkv, dh, 0xCC)
    kd, vd = torch.full_like(k, 5.0), torch.full_like(v, 5.0)
    t = lambda x: None if x is None else torch.tensor([x], device="cuda")  # noqa: E731
    Bd.polestar_k_kv4_append(k, v, torch.from_numpy(idx).cuda(), torch.from_numpy(counts).cuda(), kc, ks, vc, vs, t(tk), t(tv), kd, vd)
    for x, c, sc, d, tt in ((k, kc, ks, kd, tk), (v, vc, vs, vd, tv)):
        want_c, want_s = np.full(tuple(c.shape), 0xCC, np.uint8), np.full(tuple(sc.shape), 0xCC, np.uint8)
        codes, bytes_, val = F.quantize(f32(x).reshape(b, R, nkv, dh), F.NV, 1.0 if tt is None else tt)
        for s in range(b):
            for i in range(counts[s]):                                 # in order: the last row listed stays
                if 0 <= idx[s, i] < cap:
                    want_c[s, idx[s, i]], want_s[s, idx[s, i]] = F.pack(codes[s, i]), bytes_[s, i]
            live = torch.from_numpy((F.values(codes[s], bytes_[s], F.NV).astype(np.float32) * np.float32(1.0 if tt is None else tt))).to(d.dtype)
            n = counts[s]
            assert torch.equal(torch.nan_to_num(d[s, :n].cpu().float(), nan=-3.0), torch.nan_to_num(live.reshape(R, -1)[:n].float(), nan=-3.0))
            assert (d[s, n:] == 5.0).all()
        assert np.array_equal(c.cpu().numpy(), want_c) and np.array_equal(sc.cpu().numpy(), want_s)


def test_append_defaults_and_negative_counts():
    b, R, cap, nkv, dh = 2, 11, 20, 2, 64
    k, v = rows_of((b, R, nkv * dh), 8, torch.bfloat16).cuda(), rows_of((b, R, nkv * dh), 9, torch.bfloat16).cuda()
    kc, ks, vc, vs = cache(b, cap, nkv, dh, 0)
    Bd.polestar_k_kv4_append(k, v, None, None, kc, ks, vc, vs)          # row i at position i
    c, s, _ = F.quantize(f32(v).reshape(b, R, nkv, dh), F.NV)
    assert np.array_equal(vc[:, :R].cpu().numpy(), F.pack(c)) and np.array_equal(vs[:, :R].cpu().numpy(), s) and not vc[:, R:].any()
    before = kc.clone()
    Bd.polestar_k_kv4_append(v, k, None, torch.tensor([-5, 0], dtype=torch.int32, device="cuda"), kc, ks, vc, vs)
    assert torch.equal(before, kc)
    Bd.polestar_k_kv4_append(v, k, None, torch.tensor([99, 1], dtype=torch.int32, device="cuda"), kc, ks, vc, vs)   # clamped to R
    c, s, _ = F.quantize(f32(v).reshape(b, R, nkv, dh), F.NV)
    assert np.array_equal(kc[0, :R].cpu().numpy(), F.pack(c[0])) and torch.equal(kc[1, 1:], before[1, 1:])
