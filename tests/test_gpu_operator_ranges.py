"""The 4-bit operators at the ends of what their arguments may be: factors, rows and scores far from what models hold."""
import math

import numpy as np
import pytest
import torch

import fp4_reference as F
from paper_2607_14107_b200 import binding as Bd
from test_gpu_fp4 import check_rows, f32
from test_gpu_kv4 import reference, run

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


def cache_of(k, v, tk, tv):
    """Rows [b, cap, n_kv, dh] -> a 4-bit cache and the values that it stands for."""
    got = []
    for x, t in ((k, tk), (v, tv)):
        c, s, _ = F.quantize(x.numpy(), F.NV, t)
        got.append((torch.from_numpy(F.pack(c)).cuda(), torch.from_numpy(s).cuda(), torch.from_numpy(F.values(c, s, F.NV, t))))
    return got


def force(monkeypatch, kernel):
    monkeypatch.setenv("POLESTAR_KV4_KERNEL", str(kernel))
    Bd.polestar_reload_env()


@pytest.mark.parametrize("kernel,dtype,dh", [(1, "bf16", 128), (2, "bf16", 128), (0, "f32", 128), (0, "bf16", 64)])
@pytest.mark.parametrize("tk", [1.0, 4e-7, 1e-7, 2.0 ** -126])
@pytest.mark.parametrize("R,cap,lens", [(5, 300, [300, 129, 128]), (300, 257, [257, 1, 100]), (3, 4200, [4199, 4096, 130])])
def test_zero_rows_are_the_mean_of_the_values(monkeypatch, kernel, dtype, dh, tk, R, cap, lens):
    # a row of zeros (padding) weighs every key alike, whatever the keys' factor and wherever the length ends in a tile
    force(monkeypatch, kernel)
    b, nh, nkv, tv = 3, 4, 2, 0.005
    g = torch.Generator().manual_seed(5)
    k, v = torch.randn((b, cap, nkv, dh), generator=g) * tk * 50, torch.randn((b, cap, nkv, dh), generator=g)
    (kc, ks, k64), (vc, vs, v64) = cache_of(k, v, tk, tv)
    q = torch.randn((b, R, nh, dh), generator=g)
    q[:, ::2] = 0.0
    if tk < 1:
        q[:, 1] = 1e-38                                            # its scores are as good as 0
    out, lse = run(q.flatten(2).to(DT[dtype]).cuda(), kc, ks, vc, vs, tk, tv, lens)
    want, want_lse, size = reference(q.to(DT[dtype]).double(), k64, v64, lens, nh)
    got, got_lse = out.double().cpu().view_as(want), lse.double().cpu()
    rows = torch.zeros(R, dtype=torch.bool)
    rows[::2] = True
    if tk < 1:
        rows[1] = True
    # probabilities are 2^7 or, at factors of 2^-126, off by less than 2^-100: exact in fp16.  Sums of up to `cap` values of 128 |v| add 2^-23 (truncated)
    # per addition of 16 keys; then the factor, the quotient and the output's rounding
    tol = size * 2.0 ** -23 * (cap / 16 + 16) + want.abs() * (2.0 ** -22 + torch.finfo(DT[dtype]).eps / 2)
    assert ((got - want).abs() <= tol)[:, rows].all(), ((got - want).abs() / tol)[:, rows].max().item()
    assert ((got_lse - want_lse).abs() <= 2.0 ** -22 * want_lse.abs() + 2.0 ** -20)[:, rows].all()
    assert torch.isfinite(got).all() and torch.isfinite(got_lse).all()


@pytest.mark.parametrize("kernel", [1, 2])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("fmt", [F.NV, F.MX])
@pytest.mark.parametrize("M,N,K", [(5, 131, 64), (70, 256, 2048), (300, 520, 192)])
@pytest.mark.parametrize("ta,tb,shrink", [(1e-22, 3e-22, 1.0), (1e-30, 1e-14, 1.0), (1e25, 1e14, 1e-4), (2.0 ** 100, 2.0 ** 30, 1e-4), (2.0 ** -126, 2.0 ** -100, 1.0),
                                          (2.0 ** 127, 2.0 ** 126, 1e-4), (3e-20, 1e-19, 1.0), (0.013, 3e5, 1.0)])
def test_far_factors_of_a_product(monkeypatch, kernel, M, N, K, fmt, dtype, ta, tb, shrink):
    # the two factors' product may lie outside fp32 although the result does not, and a row of zeros stays one
    monkeypatch.setenv("POLESTAR_FP4_KERNEL", str(kernel))
    Bd.polestar_reload_env()
    g = torch.Generator().manual_seed(M)
    x = torch.randn((M, K), generator=g) * shrink
    x[M // 2] = 0.0
    c, s, _ = F.quantize(x.numpy(), fmt, 0.01)
    av = torch.from_numpy(F.values(c, s, fmt))
    y = torch.randn((N, K), generator=g) * shrink
    bc, bs, _ = F.quantize(y.numpy(), fmt, 0.01)
    bv = torch.from_numpy(F.values(bc, bs, fmt))
    ta, tb = (torch.tensor([t], dtype=torch.float32, device="cuda") for t in (ta, tb))
    out = torch.full((M, N), 5.0, dtype=dtype, device="cuda")
    Bd.polestar_k_fp4_matmul(torch.from_numpy(F.pack(c)).cuda(), torch.from_numpy(F.tile_scales(s)).cuda(), torch.from_numpy(F.pack(bc)).cuda(),
                             torch.from_numpy(F.tile_scales(bs)).cuda(), out, fmt, ta, tb)
    factor = ta.double().cpu().item() * tb.double().cpu().item()
    want, size = av @ bv.T * factor, av.abs() @ bv.abs().T * factor
    got = out.double().cpu()
    # as in the tests of the product: 2^-22 of the magnitudes per instruction and part, 2^-24 for each factor and the product with it, the output's rounding; results
    # below the normal range are rounded to its step
    tol = size * (2.0 ** -22 * (K / 64 + 8) + 2.0 ** -22) + want.abs() * torch.finfo(dtype).eps / 2 + 2.0 ** -126 * torch.finfo(dtype).eps
    top = torch.finfo(dtype).max
    fits = want.abs() + tol < top
    assert fits.any() or factor > 1e60
    assert ((got - want).abs() <= tol)[fits].all(), ((got - want).abs() / tol)[fits].max().item()
    over = want.abs() - tol > 1.01 * top
    assert (torch.isinf(got) & (torch.sign(got) == torch.sign(want)))[over].all()
    assert not torch.isnan(got).any() and (got[M // 2] == 0).all()


@pytest.mark.parametrize("kernel,dtype,dh", [(1, "bf16", 128), (2, "bf16", 128), (0, "f32", 128), (0, "bf16", 64)])
@pytest.mark.parametrize("cap,lens", [(1, [1, 0]), (200, [200, 130]), (5000, [5000, 64])])
def test_scores_beyond_fp32(monkeypatch, kernel, dtype, dh, cap, lens):
    # -inf weighs nothing beside other scores; rows whose scores are all -inf have no softmax: NaN, and not the zero row of a sequence without keys
    force(monkeypatch, kernel)
    b, R, nh, tk, tv = 2, 4, 2, 1e7, 0.01
    g = torch.Generator().manual_seed(6)
    k, v = torch.rand((b, cap, 1, dh), generator=g) * 1e10 + 1e9, torch.randn((b, cap, 1, dh), generator=g)
    k[:, 1::2] = 0.0                                                # every second key scores 0
    (kc, ks, k64), (vc, vs, v64) = cache_of(k, v, tk, tv)
    q = torch.full((b, R, nh, dh), -1e30)
    q[:, 1] = 1e-12
    q = q.to(DT[dtype])
    out, lse = run(q.flatten(2).cuda(), kc, ks, vc, vs, tk, tv, lens)
    want, want_lse, size = reference(q.double(), k64, v64, lens, nh)
    got, got_lse = out.double().cpu().view_as(want), lse.double().cpu()
    for i, n in enumerate(lens):
        for r in (0, 2, 3):
            if n == 0:
                assert not got[i, r].any() and (got_lse[i, r] == -math.inf).all()
            elif n == 1:
                assert torch.isnan(got[i, r]).all() and torch.isnan(got_lse[i, r]).all()
            else:
                tol = size * (2.0 ** -23 * (cap / 16 + 16)) + want.abs() * (2.0 ** -22 + torch.finfo(DT[dtype]).eps / 2)
                assert ((got - want).abs() <= tol)[i, r].all()
                assert ((got_lse - want_lse).abs() <= 1e-5)[i, r].all()
    # all keys: every one of them far below
    k[:, 1::2] = k[:, :1]
    (kc, ks, k64), _ = cache_of(k, v, tk, tv)
    out, lse = run(q.flatten(2).cuda(), kc, ks, vc, vs, tk, tv, lens)
    got, got_lse = out.cpu().view_as(want), lse.cpu()
    for i, n in enumerate(lens):
        for r in (0, 2, 3):
            assert torch.isnan(got[i, r]).all() and torch.isnan(got_lse[i, r]).all() if n else not got[i, r].any() and (got_lse[i, r] == -math.inf).all()
        assert torch.isfinite(got[i, 1]).all()


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("R,cap", [(1, 3000), (20, 700)])
def test_fp32_rows_of_wide_range(dh, R, cap):
    # one large entry that meets keys of zero: the scores are those of the small entries, which have to keep their places
    g = torch.Generator().manual_seed(9)
    k, v = torch.randn((1, cap, 1, dh), generator=g) * 3e5, torch.randn((1, cap, 1, dh), generator=g)
    k[..., :16] = 0.0
    (kc, ks, k64), (vc, vs, v64) = cache_of(k, v, 200.0, 0.005)
    q = torch.randn((1, R, 2, dh), generator=g) * 1e-6
    q[..., 3] = 1.5
    out, lse = run(q.flatten(2).cuda(), kc, ks, vc, vs, 200.0, 0.005, None)
    want, want_lse, size = reference(q.double(), k64, v64, [cap], 2)
    # q is held to 2^-22 of an entry, or 2^-37 of twice the row's largest; then sums of dh terms in fp32, one rounding each for unit and score
    qk = torch.stack([q[0, :, h].double().abs() @ k64[0, :, 0].abs().T for h in range(2)], 1).amax(-1)[None] / math.sqrt(dh)
    s_err = qk * 2.0 ** -21 + 3.0 * 2.0 ** -37 * k64[0, :, 0].abs().sum(-1).max() / math.sqrt(dh)
    rel = 2 * s_err + 2.0 ** -20 + 2.0 ** -24 * (cap / 8 + 64)
    got = out.double().cpu().view_as(want)
    tol = (rel + 2.0 ** -22)[..., None] * size + want.abs() * 2.0 ** -24
    assert ((got - want).abs() <= tol).all(), ((got - want).abs() / tol).max().item()
    assert ((lse.double().cpu() - want_lse).abs() <= rel + 2.0 ** -22 * want_lse.abs()).all()


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("R", [1, 12])
def test_fp32_probabilities_far_below_the_largest(R, dh):
    # a few keys take nearly all the weight and have the value 0 in half of the channels: what the others add there is the output
    cap = 20000
    g = torch.Generator().manual_seed(10)
    k, v = torch.zeros((1, cap, 1, dh)), torch.rand((1, cap, 1, dh), generator=g) + 0.5
    k[0, :, 0, 17] = torch.randint(0, 2, (cap,), generator=g).float()          # scores 0 or about 0.1 ...
    j = torch.arange(cap)
    top = (j % 16 == 3) & (j // 16 % 8 < 4)
    k[0, top, 0, 0] = 6.0                                                      # ... and about 23: the others' probabilities are near 2^-33 of the largest
    v[0, top, 0, dh // 2:] = 0.0
    (kc, ks, k64), (vc, vs, v64) = cache_of(k, v, 0.01, 0.01)
    q = torch.zeros((1, R, 2, dh))
    q[..., 0] = math.log(2) * 34 * math.sqrt(dh) / 6.0
    q[..., 17] = 0.1 * math.sqrt(dh)
    out, _ = run(q.flatten(2).cuda(), kc, ks, vc, vs, 0.01, 0.01, None)
    want, lse, size = reference(q.double(), k64, v64, [cap], 2)
    most = torch.exp(torch.stack([(q[0, :, h].double() @ k64[0, :, 0].T).amax(-1) for h in range(2)], -1)[None] / math.sqrt(dh) - lse)
    # a probability is held to 2^-22 of itself, or to half of fp16's last step lifted by 2^7 and 2^12: 2^-25 2^-19 of the row's largest; scores of up to 24 are off by
    # 2^-21 of that at worst, sums as in the other tests
    rel = 2 * 24.0 * 2.0 ** -21 + 2.0 ** -20 + 2.0 ** -24 * (cap / 8 + 64) + 2.0 ** -22
    tol = rel * size + (2.0 ** -44 * most)[..., None] * v64[0].abs().sum(0).sum(0) + want.abs() * 2.0 ** -24
    got = out.double().cpu().view_as(want)
    assert ((got - want).abs() <= tol).all(), ((got - want).abs() / tol).max().item()


@pytest.mark.parametrize("mask_id", [2 ** 32 + 3, 3 - 2 ** 32, 2 ** 31, 100, -1])
def test_mask_token_out_of_range_leaves_nothing_out(mask_id):
    x = torch.randn((2, 100), generator=torch.Generator().manual_seed(1))
    x[:, 3] = 9.0
    ids, tops = torch.empty((2, 1), dtype=torch.int32, device="cuda"), torch.empty((2, 1), device="cuda")
    Bd.polestar_k_token_logprobs(x.cuda(), None, mask_id, None, None, ids, tops)
    assert (ids == 3).all()


@pytest.mark.parametrize("kernel", [1, 2])
@pytest.mark.parametrize("b,R,cap,nh,nkv,lens", [
    (1, 300, 2, 2, 1, None), (2, 65, 3, 4, 2, [3, 2]), (1, 200, 7, 1, 1, None), (2, 40, 130, 2, 2, [130, 129]), (3, 16, 700, 4, 1, [700, 257, 5]), (1, 600, 40, 1, 1, None),
])
def test_bf16_rows_hold_probabilities_to_11_bits(monkeypatch, kernel, b, R, cap, nh, nkv, lens):
    # few keys whose values nearly cancel show a probability's rounding, which the outputs' own hides elsewhere
    force(monkeypatch, kernel)
    g = torch.Generator().manual_seed(21)
    k, v = torch.randn((b, cap, nkv, 128), generator=g), torch.randn((b, cap, nkv, 128), generator=g)
    (kc, ks, k64), (vc, vs, v64) = cache_of(k, v, 0.02, 0.005)
    q = (torch.randn((b, R, nh, 128), generator=g) * 0.5).bfloat16()
    out, _ = run(q.flatten(2).cuda(), kc, ks, vc, vs, 0.02, 0.005, lens)
    n = lens or [cap] * b
    want, _, size = reference(q.double(), k64, v64, n, nh)
    # scores as in the other tests: 2^-21 sum |q k| / sqrt(dh) at worst; a probability is off by twice that, by 2^-20 of the exponential and by fp16's half step
    # 2^-11; sums of `cap` terms in instructions of 16 add 2^-23 (truncated) each; then the output's rounding
    s_err = torch.zeros((b, R, nh), dtype=torch.float64)
    for i in range(b):
        for h in range(nh):
            s_err[i, :, h] = (q[i, :, h].double().abs() @ k64[i, :n[i], h // (nh // nkv)].abs().T).amax(-1) / math.sqrt(128) * 2.0 ** -21
    rel = 2 * s_err + 2.0 ** -20 + 2.0 ** -11 + 2.0 ** -23 * (cap / 16 + 8)
    tol = rel[..., None] * size + want.abs() * 2.0 ** -8
    got = out.double().cpu().view_as(want)
    assert ((got - want).abs() <= tol).all(), ((got - want).abs() / tol).max().item()


@pytest.mark.parametrize("dh", [64, 128])
def test_fp32_rows_over_many_keys_keep_their_last_places(dh):
    # values of one sign and probabilities spread over 20000 keys that no CTAs share out: every warp adds 312 times to its sums, a third of them each.  Rounded to nearest,
    # the additions' errors (2^-24 of the running sum at most, 2^-25.8 on average in square) have no direction: 3 2^-24 sqrt(312 / 3) 2^-1.8 = 9 2^-24 would be
    # three of their standard deviations for one output, and their mean square over all outputs is near 3 2^-24.  Probabilities add 2^-22 (their two terms; the
    # exponential's 2^-22 weighs on sums and values alike), scores 2^-22 here.  Together below 2e-6; sums truncated at every step lose 7e-6 of
    # themselves (312 additions, each a half of the running sum's last place on average).
    cap, R, nh = 20000, 260, 28
    g = torch.Generator().manual_seed(22)
    k, v = torch.randn((1, cap, 4, dh), generator=g), torch.rand((1, cap, 4, dh), generator=g) + 0.5
    (kc, ks, k64), (vc, vs, v64) = cache_of(k, v, 0.02, 0.005)
    q = torch.randn((1, R, nh, dh), generator=g) * 0.05
    out, lse = run(q.flatten(2).cuda(), kc, ks, vc, vs, 0.02, 0.005, None)
    rows = torch.tensor([0, 7, 16, 100, 259])
    want, want_lse, _ = reference(q[:, rows].double(), k64, v64, [cap], nh)
    got = out.double().cpu().view(1, R, nh, dh)[:, rows]
    assert ((got - want).norm() / want.norm()).item() <= 2e-6
    assert (lse.double().cpu()[:, rows] - want_lse).abs().max().item() <= 2e-6 * 10.0


@pytest.mark.parametrize("kernel,dtype,dh", [(1, "bf16", 128), (2, "bf16", 128), (0, "f32", 128), (0, "bf16", 64)])
def test_a_score_above_fp32_makes_its_row_nan(monkeypatch, kernel, dtype, dh):
    force(monkeypatch, kernel)
    cap, R, tk = 300, 3, 1e7
    k, v = torch.zeros((1, cap, 1, dh)), torch.ones((1, cap, 1, dh))
    k[0, 200] = 1e10
    (kc, ks, _), (vc, vs, _) = cache_of(k, v, tk, 0.01)
    q = torch.full((1, R, dh), 1e-12)
    q[0, 1] = 1e30
    out, lse = run(q.to(DT[dtype]).cuda(), kc, ks, vc, vs, tk, 0.01, [cap])
    assert torch.isnan(out[0, 1]).all() and torch.isnan(lse[0, 1]).all()
    assert torch.isfinite(out[0, ::2]).all() and torch.isfinite(lse[0, ::2]).all()
