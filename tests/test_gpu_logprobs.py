"""Token log-probabilities, entropy and alternatives against float64."""
import numpy as np
import pytest
import torch

from paper_2607_14107_b200 import binding as Bd

pytestmark = pytest.mark.gpu


def reference(x, target, mask_id, k):
    """x float64 [rows][V] -> logprob, entropy, ids, tops as the header defines them."""
    rows, V = x.shape
    lp, h = np.zeros(rows), np.zeros(rows)
    ids, tops = np.full((rows, k), -1, np.int64), np.full((rows, k), -np.inf)
    for r in range(rows):
        ok = not np.isnan(x[r]).any() and x[r].max() < np.inf and x[r].max() > -np.inf
        order = [v for v in np.argsort(-x[r], kind="stable") if v != mask_id and not np.isnan(x[r, v])][:k]
        ids[r, :len(order)] = order
        if ok:
            z = x[r] - x[r].max()
            e = np.exp(z)
            ls = np.log(e.sum())
            h[r] = ls - (e * np.where(e > 0, z, 0)).sum() / e.sum()
            tops[r, :len(order)] = z[order] - ls
            lp[r] = z[target[r]] - ls if 0 <= target[r] < V else (0.0 if target[r] < 0 else np.nan)
        else:
            h[r] = np.nan
            tops[r, :len(order)] = np.nan
            lp[r] = 0.0 if target[r] < 0 else np.nan
    return lp, h, ids, tops


def run(x, target, mask_id, k, ld=None, off=0):
    rows, V = x.shape
    ld = ld or V
    buf = torch.full((off + rows * ld,), 1e30, dtype=x.dtype, device="cuda")      # what lies between the rows would be seen
    m = buf[off:].view(rows, ld)[:, :V]
    m.copy_(x)
    lp, h = torch.full((rows,), -1.0, device="cuda"), torch.full((rows,), -1.0, device="cuda")
    ids = torch.full((rows, k), -9, dtype=torch.int32, device="cuda")
    tops = torch.full((rows, k), -9.0, device="cuda")
    Bd.polestar_k_token_logprobs(m, torch.from_numpy(target).int().cuda(), mask_id, lp, h, ids, tops)
    return [t.cpu().numpy().astype(np.float64) for t in (lp, h, ids, tops)]


def check(x, target, mask_id, k, **kw):
    got = run(x, target, mask_id, k, **kw)
    want = reference(x.cpu().double().numpy(), target, mask_id, k)
    # fp32: a term's error is 2^-22 of ex2 and 2^-24 per unit of its exponent (32 covers what carries weight); a thread adds up to V / 128 terms
    # in two chains, all errors in one direction at worst
    V = x.shape[1]
    eps = 2.0 ** -24 * (4 + 32 + V / 256 + 24)
    with np.errstate(invalid="ignore"):
        span = np.nan_to_num(np.abs(np.where(np.isfinite(want[0]), want[0], 0)))
    assert np.array_equal(np.isnan(got[0]), np.isnan(want[0])) and np.array_equal(np.isnan(got[1]), np.isnan(want[1]))
    inf = np.isinf(want[0])
    assert np.array_equal(got[0][inf], want[0][inf])
    fin = np.isfinite(want[0])
    assert (np.abs(got[0] - want[0])[fin] <= (eps + 2.0 ** -23 * span)[fin]).all(), np.abs(got[0] - want[0])[fin].max()
    fin = np.isfinite(want[1])
    # entropy: the same errors weighted with |z| <= H + 1 on average, twice (sum and weighted sum)
    assert (np.abs(got[1] - want[1])[fin] <= (2 * eps * (2 + want[1]))[fin]).all(), np.abs(got[1] - want[1])[fin].max()
    assert np.array_equal(got[2], want[2])
    a, b = got[3], want[3]
    assert np.array_equal(np.isnan(a), np.isnan(b)) and np.array_equal(a[np.isinf(b)], b[np.isinf(b)])
    fin = np.isfinite(b)
    assert (np.abs(a - b)[fin] <= (eps + 2.0 ** -23 * np.abs(b))[fin]).all()


def logits(rows, V, seed, dtype, sigma=3.0):
    g = torch.Generator().manual_seed(seed)
    return (sigma * torch.randn((rows, V), generator=g)).to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,V,k", [(1, 1, 1), (2, 2, 3), (3, 5, 32), (7, 31, 8), (5, 1000, 0), (4, 4097, 20), (3, 50257, 32), (2, 126464, 8),
                                      (32, 126464, 1), (300, 2003, 5), (600, 640, 32), (40, 20001, 7)])
def test_logprobs(dtype, rows, V, k):
    x = logits(rows, V, V + rows, dtype)
    target = np.random.default_rng(V).integers(0, V, rows)
    target[0] = -1
    if rows > 2:
        target[1], target[2] = V, V - 1
    check(x, target, V // 2, k)


@pytest.mark.parametrize("dtype,off,pad", [(torch.float32, 1, 3), (torch.float32, 3, 0), (torch.bfloat16, 1, 5), (torch.bfloat16, 7, 1), (torch.bfloat16, 0, 8)])
def test_rows_at_any_address(dtype, off, pad):
    x = logits(9, 5003, 4, dtype)
    check(x, np.arange(9), 17, 6, ld=5003 + pad, off=off)
    check(logits(5, 3, 4, dtype), np.arange(5) % 3, 1, 2, ld=3 + pad, off=off)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [640, 40000])
def test_equal_logits(dtype, V):
    # whole rows of one value, of few values, ascending and descending rows: the lowest indices among equals, however many reach the bound
    x = torch.zeros((8, V))
    x[1] = (torch.arange(V) % 3).float()
    x[2] = torch.arange(V).float() / 64
    x[3] = -torch.arange(V).float() / 64
    x[4, V // 2:] = 1.0
    x[5, :V // 3] = float("-inf")
    x[6, :] = float("-inf"); x[6, 5] = 2.0; x[6, V - 1] = 2.0
    x[7] = (torch.arange(V) // (V // 4)).float()
    check(x.to(dtype), np.array([0, 1, V - 1, 0, 0, V - 1, 5, 3]), 1, 32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_without_a_distribution(dtype):
    x = logits(7, 3001, 2, dtype)
    x[0] = float("-inf")
    x[1, 77] = float("nan")
    x[2, 2999] = float("inf")
    x[3, ::2] = float("-inf")
    x[4] = float("nan")
    x[5] = torch.finfo(dtype).min
    x[6, 1:] = float("-inf")                      # one token alone: log-probability 0, entropy 0
    target = np.array([4, 5, 6, 7, -1, 8, 0])
    got = run(x, target, -1, 4)
    want = reference(x.double().numpy(), target, -1, 4)
    for g, w in zip((got[0], got[1], got[3]), (want[0], want[1], want[3])):
        rows = [0, 1, 2, 3, 5, 6] if g is not got[3] else [0, 1, 3, 5, 6]
        assert np.array_equal(np.isnan(g[rows]), np.isnan(w[rows]))
    assert np.array_equal(got[2][[0, 1, 3, 5, 6]], want[2][[0, 1, 3, 5, 6]])
    assert (got[2][4] == -1).all() and got[0][6] == 0.0 and got[1][6] == 0.0
    assert np.isnan(got[0][[0, 1, 2]]).all() and np.isnan(got[1][[0, 1, 2, 4]]).all()


def test_nearly_certain_rows_keep_their_small_values():
    # one token 20 above 50 others: logprob -50 e^-20, entropy 50 e^-20 (20 + 1): relative to the maximum, not to the logits' size
    x = torch.full((2, 51), 1000.0)
    x[:, 7] = 1020.0
    x[1, 7] = 1008.0
    got = run(x, np.array([7, 7]), -1, 1)
    want = reference(x.double().numpy(), np.array([7, 7]), -1, 1)
    assert np.abs(got[0] - want[0]).max() <= 2.0 ** -22 and np.abs(got[1] - want[1]).max() <= 2.0 ** -20 and (got[1] >= 0).all()


def test_optional_outputs_and_determinism():
    x = logits(33, 30011, 12, torch.bfloat16).cuda()
    t = torch.arange(33, dtype=torch.int32, device="cuda")
    outs = []
    for _ in range(2):
        lp, h = torch.empty(33, device="cuda"), torch.empty(33, device="cuda")
        ids, tops = torch.empty((33, 16), dtype=torch.int32, device="cuda"), torch.empty((33, 16), device="cuda")
        Bd.polestar_k_token_logprobs(x, t, 5, lp, h, ids, tops)
        outs.append([lp, h, ids, tops])
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    only_h = torch.empty(33, device="cuda")
    Bd.polestar_k_token_logprobs(x, None, None, None, only_h)
    assert torch.equal(only_h, outs[0][1])
