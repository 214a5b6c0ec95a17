"""Attention over a K/V cache held in 4 bits against float64 attention over the values that the cache stands for."""
import math

import numpy as np
import pytest
import torch

import fp4_reference as F
from paper_2607_14107_b200 import binding as Bd

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def make_cache(b, cap, nkv, dh, seed, tk, tv, peaked=0.0):
    """Codes of random rows; a few keys far larger than the rest (peaked), so that the running maximum moves late."""
    g = torch.Generator().manual_seed(seed)
    out = []
    for i, t in enumerate((tk, tv)):
        x = torch.randn((b, cap, nkv, dh), generator=g) * torch.exp(0.5 * torch.randn(dh, generator=g))
        if i == 0 and peaked:
            x[:, ::37] *= peaked
        c, s, _ = F.quantize(x.numpy(), F.NV, 1.0 if t is None else t)
        out.append((torch.from_numpy(F.pack(c)).cuda(), torch.from_numpy(s).cuda(), torch.from_numpy(F.values(c, s, F.NV, 1.0 if t is None else t))))
    return out


def reference(q, k, v, lens, nh):
    """float64: q [b, R, nh, dh], k / v [b, cap, nkv, dh] -> out, lse, and sum p |v| (what the rounding of p can move)."""
    b, R, _, dh = q.shape
    nkv = k.shape[2]
    out, size = torch.zeros((b, R, nh, dh), dtype=torch.float64), torch.zeros((b, R, nh, dh), dtype=torch.float64)
    lse = torch.full((b, R, nh), -math.inf, dtype=torch.float64)
    for i in range(b):
        n = int(lens[i])
        if n == 0:
            continue
        for h in range(nh):
            g = h // (nh // nkv)
            s = q[i, :, h] @ k[i, :n, g].T / math.sqrt(dh)
            p = torch.softmax(s, -1)
            lse[i, :, h] = torch.logsumexp(s, -1)
            out[i, :, h], size[i, :, h] = p @ v[i, :n, g], p @ v[i, :n, g].abs()
    return out, lse, size


def run(q, kc, ks, vc, vs, tk, tv, lens, with_lse=True, fill=7.0):
    b, R, w = q.shape
    dh = 2 * kc.shape[3]
    nh = w // dh
    out = torch.full_like(q, fill)
    lse = torch.full((b, R, nh), fill, device="cuda") if with_lse else None
    scratch = torch.full((Bd.polestar_k_kv4_scratch_bytes(b, R, kc.shape[1], nh, kc.shape[2], dh),), 0xFF, dtype=torch.uint8, device="cuda")
    t = lambda x: None if x is None else torch.tensor([x], device="cuda")  # noqa: E731
    Bd.polestar_k_kv4_attention(q, kc, ks, vc, vs, t(tk), t(tv), None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda"), out, lse, scratch)
    return out, lse


def check(dtype, b, R, cap, nh, nkv, dh, lens, tk=0.02, tv=0.005, q_size=0.5, peaked=0.0, seed=0):
    (kc, ks, k), (vc, vs, v) = make_cache(b, cap, nkv, dh, seed, tk, tv, peaked)
    g = torch.Generator().manual_seed(seed + 50)
    q = (q_size * torch.randn((b, R, nh * dh), generator=g) * torch.exp(torch.randn(dh, generator=g) * 0.3).repeat(nh)).to(DT[dtype])
    out, lse = run(q.cuda(), kc, ks, vc, vs, tk, tv, lens)
    n = [cap] * b if lens is None else [min(max(x, 0), cap) for x in lens]
    q64 = q.double().view(b, R, nh, dh)
    want, want_lse, size = reference(q64, k, v, n, nh)
    # Scores: products are exact up to q's terms (16 bits: bf16 is exact in them, fp32 2^-22), sums of at most dh terms in fp32, one rounding each
    # for unit and score: |ds| <= 2^-21 sum |q k| / sqrt(dh) at worst.  A probability is off by that, by its rounding (bf16 forms: 2^-9 where
    # tensor memory holds it as bf16, fp16 2^-11; fp32: 2^-22) and the exponential's 2^-21; sums of up to `cap` terms of like sign add 2^-24
    # per addition in each of several chains: 2^-24 * (cap / 8 + 64) covers them.
    # Probabilities below fp16's range.  They are held as p 2^7 relative to a maximum that lags by no more than it lifts, and fp16's steps are never
    # finer than 2^-24: each p is off by up to 2^-25 2^-7 = 2^-32 of the row's largest, whatever its own size.  That moves an output by up to
    # 2^-32 sum_j |v_j| (a row whose one likely key has the value 0 in a channel shows it: there sum p |v| is of the order of 2^-30), and the
    # sum of probabilities, taken from the unrounded ones, not at all.
    s_err = torch.zeros_like(want_lse)
    for i in range(b):
        if n[i]:
            for h in range(nh):
                s_err[i, :, h] = (q64[i, :, h].abs() @ k[i, :n[i], h // (nh // nkv)].abs().T).amax(-1) / math.sqrt(dh) * 2.0 ** -21
    p_round = 2.0 ** -9 if dtype == "bf16" else 2.0 ** -22
    rel = 2 * s_err + 2.0 ** -20 + 2.0 ** -24 * (cap / 8 + 64)
    lost = torch.stack([v[i, :n[i]].abs().sum(0).repeat_interleave(nh // nkv, 0) for i in range(b)])[:, None] * 2.0 ** -32
    tol = (rel + p_round)[..., None] * size + lost + want.abs() * torch.finfo(DT[dtype]).eps / 2 + 1e-12
    got = out.double().cpu().view(b, R, nh, dh)
    assert ((got - want).abs() <= tol).all(), ((got - want).abs() / tol).max().item()
    got_lse = lse.double().cpu()
    assert torch.equal(torch.isinf(got_lse), torch.isinf(want_lse))
    fin = torch.isfinite(want_lse)
    lse_tol = rel + 2.0 ** -22 * want_lse.abs()
    assert ((got_lse - want_lse).abs()[fin] <= lse_tol[fin]).all(), (got_lse - want_lse).abs()[fin].max().item()
    return out, lse, (kc, ks, vc, vs), q


SHAPES = [
    # b, R, cap, nh, nkv, dh, lens
    (1, 1, 1, 1, 1, 64, None), (1, 1, 1, 2, 1, 128, [1]), (2, 1, 5, 4, 2, 128, [5, 3]),
    (1, 16, 16, 2, 2, 64, None), (1, 17, 33, 3, 3, 128, None), (3, 29, 1021, 4, 4, 64, [1021, 0, 517]),
    (2, 32, 512, 4, 4, 128, [512, 511]), (2, 5, 2100, 14, 2, 128, [2100, 1]), (4, 1, 8192, 28, 4, 128, [8192, 4097, 4096, 33]),
    (1, 130, 300, 7, 1, 128, None), (1, 1, 65536, 2, 1, 64, [65535]), (2, 70, 777, 8, 8, 64, [-4, 9999]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("b,R,cap,nh,nkv,dh,lens", SHAPES)
def test_attention(dtype, b, R, cap, nh, nkv, dh, lens):
    check(dtype, b, R, cap, nh, nkv, dh, lens)


@pytest.mark.parametrize("kernel", [1, 2])
@pytest.mark.parametrize("b,R,cap,nh,nkv,lens", [
    (1, 1, 1, 1, 1, None), (2, 1, 700, 2, 1, [700, 130]), (3, 29, 1021, 4, 4, [1021, 0, 517]),       # one row tile: the streams split the keys
    (2, 128, 129, 2, 2, [129, 128]), (1, 129, 127, 1, 1, None),                                        # a full row tile, a second one of a single row
    (2, 70, 600, 7, 1, [600, 257]), (1, 520, 384, 1, 1, None), (2, 260, 1300, 2, 2, [1300, 3]),        # odd and even numbers of row tiles
    (1, 3, 9000, 7, 1, [8999]), (2, 40, 5000, 4, 1, [5000, 700]),                                      # keys split over CTAs, some without any
])
def test_both_kernels(monkeypatch, kernel, b, R, cap, nh, nkv, lens):
    monkeypatch.setenv("POLESTAR_KV4_KERNEL", str(kernel))
    Bd.polestar_reload_env()
    check("bf16", b, R, cap, nh, nkv, 128, lens, seed=kernel)
    check("bf16", b, R, cap, nh, nkv, 128, lens, q_size=6.0, peaked=5.0, seed=kernel + 10)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_size,peaked", [(8.0, 6.0), (1e-4, 0.0), (3e4, 0.0), (1e-30, 0.0)])
def test_attention_peaked_and_flat_rows(dtype, q_size, peaked):
    check(dtype, 2, 19, 900, 4, 2, 128, [900, 641], q_size=q_size, peaked=peaked, tk=None if q_size < 1 else 1e-3 if q_size > 100 else 0.02, tv=None, seed=4)


@pytest.mark.parametrize("dtype,R", [("bf16", 1), ("f32", 1), ("bf16", 40), ("bf16", 300)])
def test_what_lies_behind_a_sequence_is_not_seen(dtype, R):
    # codes and scales behind the lengths are NaN scales; nothing of them shows, and the same rows come out whatever lies there
    b, cap, nh, nkv, dh = 3, 700, 4, 2, 128
    lens = [700, 129, 0]
    out, lse, (kc, ks, vc, vs), q = check(dtype, b, R, cap, nh, nkv, dh, lens, seed=2)
    for i, n in enumerate(lens):
        for t in (ks, vs):
            t[i, n:] = 0x7F
        for t in (kc, vc):
            t[i, n:] = 0xFF
    again, lse2 = run(q.cuda(), kc, ks, vc, vs, 0.02, 0.005, lens)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    assert not out[2].any() and torch.isinf(lse[2]).all()
    # a NaN scale in front of the length is seen: keys poison the head's rows, values one group of channels
    vs[0, 5, 1, 2] = 0x7F
    bad, _ = run(q.cuda(), kc, ks, vc, vs, 0.02, 0.005, lens)
    bad = bad.view(b, R, nh, dh)
    assert torch.isnan(bad[0, :, 2:, 32:48]).all() and not torch.isnan(bad[0, :, :2]).any() and not torch.isnan(bad[0, :, 2:, :32]).any()
    ks[0, 600, 0, 7] = 0x7F
    bad, l3 = run(q.cuda(), kc, ks, vc, vs, 0.02, 0.005, lens)
    assert torch.isnan(bad.view(b, R, nh, dh)[0, :, :2]).all() and torch.isnan(l3[0, :, :2]).all() and not torch.isnan(bad[1]).any()


def test_nan_rows_stay_their_own():
    b, R, cap, nh, nkv, dh = 1, 37, 300, 4, 2, 128
    (kc, ks, k), (vc, vs, v) = make_cache(b, cap, nkv, dh, 3, 0.02, 0.005)
    q = torch.randn((b, R, nh * dh), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    clean, _ = run(q, kc, ks, vc, vs, 0.02, 0.005, None)
    q[0, 7, 3] = float("nan")
    q[0, 20, dh + 5] = float("inf")
    out, lse = run(q, kc, ks, vc, vs, 0.02, 0.005, None)
    o = out.view(R, nh, dh)
    assert torch.isnan(o[7, 0]).all() and torch.isnan(lse[0, 7, 0])
    keep = torch.ones((R, nh), dtype=torch.bool)
    keep[7, 0] = keep[20, 1] = False
    assert torch.equal(o[keep], clean.view(R, nh, dh)[keep])


@pytest.mark.parametrize("kernel,dtype", [(1, "bf16"), (2, "bf16"), (0, "f32")])
@pytest.mark.parametrize("cap", [1, 77, 3000])
def test_infinite_q_is_nan_whatever_its_scores_sign(monkeypatch, kernel, dtype, cap):
    # every score is -inf: softmax over them is NaN, and not the zero row of a sequence without keys
    monkeypatch.setenv("POLESTAR_KV4_KERNEL", str(kernel))
    Bd.polestar_reload_env()
    R, dh, t = 3, 128, torch.tensor([0.02], device="cuda")
    k = torch.ones((2, cap, dh), dtype=DT[dtype], device="cuda")
    c = [torch.empty((2, cap, 1, n), dtype=torch.uint8, device="cuda") for n in (dh // 2, dh // 16, dh // 2, dh // 16)]
    Bd.polestar_k_kv4_append(k, k, None, None, *c, t, t)
    q = torch.ones((2, R, dh), dtype=DT[dtype], device="cuda")
    q[:, 1, 5] = -math.inf
    out, lse = run(q, *c, 0.02, 0.02, [cap, 0])
    assert torch.isnan(out[0, 1]).all() and torch.isnan(lse[0, 1]).all()
    assert not out[1].any() and torch.isinf(lse[1]).all()                  # (no keys: zeros)
    assert torch.isfinite(out[0, ::2]).all() and torch.isfinite(lse[0, ::2]).all()


@pytest.mark.parametrize("kernel,dtype", [(1, "bf16"), (2, "bf16"), (0, "f32")])
def test_more_sequences_than_are_cut_to_measure(monkeypatch, kernel, dtype):
    monkeypatch.setenv("POLESTAR_KV4_KERNEL", str(kernel))
    Bd.polestar_reload_env()
    check(dtype, 40, 1, 2200, 4, 2, 128, [2200, 0, 1, 64, 65] + [(97 * i) % 2201 for i in range(35)], seed=8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_without_lse_and_without_lengths(dtype):
    out, lse, c, q = check(dtype, 2, 9, 400, 4, 4, 64, None)
    again, none = run(q.cuda(), *c, 0.02, 0.005, None, with_lse=False)
    assert none is None and torch.equal(out, again)


def test_append_then_attend_joins_with_plain_attention():
    """A denoising step: rows go into the cache, query rows attend over it, and lse joins the result with attention over other keys."""
    b, R, cap, nh, nkv, dh = 2, 32, 512, 8, 2, 128
    g = torch.Generator().manual_seed(0)
    (kc, ks, k), (vc, vs, v) = make_cache(b, cap, nkv, dh, 6, 0.02, 0.005)
    new_k, new_v = (torch.randn((b, R, nkv * dh), generator=g).bfloat16() for _ in range(2))
    q = torch.randn((b, R, nh * dh), generator=g).bfloat16()
    idx = torch.stack([torch.randperm(cap, generator=g)[:R].sort()[0] for _ in range(b)]).int()
    tk, tv = torch.tensor([0.02], device="cuda"), torch.tensor([0.005], device="cuda")
    kd, vd = torch.zeros_like(new_k).cuda(), torch.zeros_like(new_v).cuda()
    Bd.polestar_k_kv4_append(new_k.cuda(), new_v.cuda(), idx.cuda(), None, kc, ks, vc, vs, tk, tv, kd, vd)
    lens = [512, 400]
    out, lse = run(q.cuda(), kc, ks, vc, vs, 0.02, 0.005, lens)
    for x, name, t in ((k, new_k, 0.02), (v, new_v, 0.005)):
        c, s, val = F.quantize(name.float().numpy().reshape(b, R, nkv, dh), F.NV, t)
        for i in range(b):
            x[i, idx[i].long()] = torch.from_numpy(val[i])
    q64 = q.double().view(b, R, nh, dh)
    want, want_lse, size = reference(q64, k, v, lens, nh)
    assert ((out.double().cpu().view_as(want) - want).abs() <= size * 2.0 ** -8 + want.abs() * 2.0 ** -8).all()
    # the same keys in two calls, joined by their log-sum-exps
    halves = [run(q.cuda(), *(t[:, lo:hi].contiguous() for t in (kc, ks, vc, vs)), 0.02, 0.005, [min(max(n - lo, 0), hi - lo) for n in lens])
              for lo, hi in ((0, 200), (200, 512))]
    w = torch.softmax(torch.stack([h[1] for h in halves]).double(), 0)
    joined = sum(wi[..., None] * h[0].double().view(b, R, nh, dh) for wi, h in zip(w, halves)).cpu()
    assert ((joined - want).abs() <= size * 2.0 ** -7 + want.abs() * 2.0 ** -8).all()


def test_results_do_not_depend_on_the_run():
    b, R, cap, nh, nkv, dh = 2, 3, 5000, 8, 2, 128
    (kc, ks, _), (vc, vs, _) = make_cache(b, cap, nkv, dh, 8, 0.02, 0.005)
    q = torch.randn((b, R, nh * dh), generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    first = run(q, kc, ks, vc, vs, 0.02, 0.005, [5000, 1700])
    for _ in range(3):
        again = run(q, kc, ks, vc, vs, 0.02, 0.005, [5000, 1700], fill=0.0)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
