"""The 4-bit and log-probability entry points as programs use them: composed into a step, captured, on other streams, far into large buffers."""
import math

import numpy as np
import pytest
import torch

import fp4_reference as F
from paper_2607_14107_b200 import binding as Bd

pytestmark = pytest.mark.gpu


def u8(*shape):
    return torch.zeros(shape, dtype=torch.uint8, device="cuda")


class Layer:
    """Buffers of one attention layer in 4 bits and the calls of a denoising step over it."""

    def __init__(self, rows=24, cap=300, nh=4, nkv=2, dh=128, vocab=1000, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.g, self.rows, self.cap, self.nh, self.nkv, self.dh, self.vocab = g, rows, cap, nh, nkv, dh, vocab
        d = nh * dh
        self.w = {}
        for name, n, k in (("qkv", (nh + 2 * nkv) * dh, d), ("o", d, d), ("lm", vocab, d)):
            c, b, v = F.quantize((0.05 * torch.randn((n, k), generator=g)).numpy(), F.NV, 0.001)
            self.w[name] = (torch.from_numpy(F.pack(c)).cuda(), torch.from_numpy(F.tile_scales(b)).cuda(), torch.from_numpy(v))
        self.x = torch.randn((rows, d), generator=g).bfloat16().cuda()
        self.xc, self.xs = u8(rows, d // 2), u8(Bd.polestar_k_fp4_scale_bytes(rows, d, F.NV, Bd.SCALES_TILED))
        self.kc, self.ks, self.vc, self.vs = u8(1, cap, nkv, dh // 2), u8(1, cap, nkv, dh // 16), u8(1, cap, nkv, dh // 2), u8(1, cap, nkv, dh // 16)
        new = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.qkv, self.q, self.k, self.v = new(rows, (nh + 2 * nkv) * dh), new(1, rows, d), new(1, rows, nkv * dh), new(1, rows, nkv * dh)
        self.attn, self.o = new(1, rows, d), new(rows, d)
        self.logits = torch.zeros((rows, vocab), device="cuda")
        self.idx = torch.sort(torch.randperm(cap, generator=g)[:rows])[0].int().view(1, rows).cuda()
        self.lens = torch.tensor([cap], dtype=torch.int32, device="cuda")
        self.scratch = u8(Bd.polestar_k_kv4_scratch_bytes(1, rows, cap, nh, nkv, dh))
        self.t = {n: torch.tensor([t], device="cuda") for n, t in (("x", 0.01), ("w", 0.001), ("k", 0.01), ("v", 0.01))}
        self.target = torch.zeros(rows, dtype=torch.int32, device="cuda")
        self.lp, self.h = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
        self.ids, self.tops = torch.zeros((rows, 4), dtype=torch.int32, device="cuda"), torch.zeros((rows, 4), device="cuda")

    def project(self, x, name, out):
        Bd.polestar_k_fp4_quantize(x, self.xc, self.xs, F.NV, Bd.SCALES_TILED, tensor_scale=self.t["x"])
        Bd.polestar_k_fp4_matmul(self.xc, self.xs, *self.w[name][:2], out, F.NV, self.t["x"], self.t["w"])

    def step(self):
        nq, nk = self.nh * self.dh, self.nkv * self.dh
        self.project(self.x, "qkv", self.qkv)
        self.q[0].copy_(self.qkv[:, :nq]); self.k[0].copy_(self.qkv[:, nq:nq + nk]); self.v[0].copy_(self.qkv[:, nq + nk:])
        Bd.polestar_k_kv4_append(self.k, self.v, self.idx, None, self.kc, self.ks, self.vc, self.vs, self.t["k"], self.t["v"])
        Bd.polestar_k_kv4_attention(self.q, self.kc, self.ks, self.vc, self.vs, self.t["k"], self.t["v"], self.lens, self.attn, None, self.scratch)
        self.project(self.attn[0], "o", self.o)
        self.project(self.o, "lm", self.logits)
        Bd.polestar_k_token_logprobs(self.logits, self.target, 7, self.lp, self.h, self.ids, self.tops)

    def outputs(self):
        return [t.clone() for t in (self.qkv, self.kc, self.ks, self.vc, self.vs, self.attn, self.o, self.logits, self.lp, self.h, self.ids, self.tops)]


def test_a_step_from_end_to_end():
    """Every stage against float64 from the stage before as the library left it."""
    s = Layer()
    s.step()
    val = lambda x, t: torch.from_numpy(F.quantize(x.float().cpu().numpy(), F.NV, t)[2])  # noqa: E731
    for x, name, out in ((s.x, "qkv", s.qkv), (s.attn[0], "o", s.o), (s.o, "lm", s.logits)):
        a = val(x, 0.01)
        want = a @ s.w[name][2].T
        size = a.abs() @ s.w[name][2].abs().T
        assert ((out.double().cpu() - want).abs() <= size * 2.0 ** -18 + want.abs() * torch.finfo(out.dtype).eps / 2 + 1e-9).all(), name
    for rows, c, sc in ((s.k, s.kc, s.ks), (s.v, s.vc, s.vs)):
        code, byte, _ = F.quantize(rows[0].float().cpu().numpy().reshape(s.rows, s.nkv, s.dh), F.NV, 0.01)
        at = s.idx[0].cpu().long()
        assert np.array_equal(c[0].cpu().numpy()[at], F.pack(code)) and np.array_equal(sc[0].cpu().numpy()[at], byte)
    k, v = (torch.from_numpy(F.values(F.unpack(c[0].cpu().numpy()), sc[0].cpu().numpy(), F.NV, 0.01)) for c, sc in ((s.kc, s.ks), (s.vc, s.vs)))
    q = s.q[0].double().cpu().view(s.rows, s.nh, s.dh)
    for h in range(s.nh):
        p = torch.softmax(q[:, h] @ k[:, h // 2].T / math.sqrt(s.dh), -1)
        got = s.attn[0].double().cpu().view(s.rows, s.nh, s.dh)[:, h]
        assert ((got - p @ v[:, h // 2]).abs() <= (p @ v[:, h // 2].abs()) * 2.0 ** -8 + got.abs() * 2.0 ** -8 + 1e-9).all()
    lp = torch.log_softmax(s.logits.double(), -1)
    assert (s.lp.double() - lp[:, 0]).abs().max() < 1e-5
    lp[:, 7] = -math.inf
    assert torch.equal(s.ids.long().sort(-1)[0], lp.topk(4, -1).indices.sort(-1)[0])


def test_a_captured_step_replays_on_new_inputs():
    s, ref = Layer(seed=1), Layer(seed=1)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        s.step()
        with torch.cuda.graph(graph, stream=stream):
            s.step()
    torch.cuda.synchronize()
    for seed in (5, 6):
        x = torch.randn(s.x.shape, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()
        idx = torch.sort(torch.randperm(s.cap, generator=torch.Generator().manual_seed(seed))[:s.rows])[0].int().view(1, -1).cuda()
        for l in (s, ref):
            l.x.copy_(x); l.idx.copy_(idx); l.lens.fill_(100 * (seed - 4))
            for t in (l.kc, l.ks, l.vc, l.vs):
                t.zero_()
        graph.replay()
        ref.step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(s.outputs(), ref.outputs()))


def test_steps_on_two_streams_at_once():
    layers = [Layer(seed=2), Layer(seed=3, rows=70, cap=2000)]
    for l in layers:
        l.step()
    torch.cuda.synchronize()
    want = [l.outputs() for l in layers]
    streams = [torch.cuda.Stream() for _ in layers]
    for _ in range(5):
        for l in layers:
            for t in (l.attn, l.logits, l.kc, l.vc):
                t.zero_()
        torch.cuda.synchronize()
        for l, st in zip(layers, streams):
            with torch.cuda.stream(st):
                l.step()
        torch.cuda.synchronize()
        for l, w in zip(layers, want):
            assert all(torch.equal(a, b) for a, b in zip(l.outputs(), w))


# ------------------------------------------------------------------ offsets beyond 32 bits
def test_quantised_rows_beyond_four_gigabytes():
    rows, d = 70000, 32768                      # 2.3e9 elements
    x = torch.zeros((rows, d), dtype=torch.bfloat16, device="cuda")
    some = torch.randn((3, d), generator=torch.Generator().manual_seed(0)).bfloat16()
    at = [0, 65537, rows - 1]
    x[at] = some.cuda()
    codes, scales = torch.full((rows, d // 2), 0xEE, dtype=torch.uint8, device="cuda"), torch.full((rows, d // 16), 0xEE, dtype=torch.uint8, device="cuda")
    Bd.polestar_k_fp4_quantize(x, codes, scales, F.NV)
    c, b, _ = F.quantize(some.float().numpy(), F.NV)
    assert np.array_equal(codes[at].cpu().numpy(), F.pack(c)) and np.array_equal(scales[at].cpu().numpy(), b)
    assert not codes[at[0] + 1:at[1]].any() and not scales[at[1] + 1:at[2]].any()


def test_products_beyond_four_gigabytes():
    M, N, K = 66000, 33000, 64                  # 2.2e9 outputs
    g = torch.Generator().manual_seed(1)
    ac, ab, av = F.quantize(torch.randn((300, K), generator=g).numpy(), F.NV)
    bc, bb, bv = F.quantize(torch.randn((N, K), generator=g).numpy(), F.NV)
    at = np.arange(M) % 300
    out = torch.zeros((M, N), dtype=torch.bfloat16, device="cuda")
    Bd.polestar_k_fp4_matmul(torch.from_numpy(F.pack(ac)[at]).cuda(), torch.from_numpy(F.tile_scales(ab[at])).cuda(), torch.from_numpy(F.pack(bc)).cuda(),
                             torch.from_numpy(F.tile_scales(bb)).cuda(), out, F.NV)
    rows = [0, 32767, 65535, 65536, M - 1]
    want = torch.from_numpy(av[at[rows]]) @ torch.from_numpy(bv).T
    size = torch.from_numpy(np.abs(av[at[rows]])) @ torch.from_numpy(np.abs(bv)).T
    assert ((out[rows].double().cpu() - want).abs() <= size * 2.0 ** -18 + want.abs() * 2.0 ** -8).all()


@pytest.mark.parametrize("R", [1, 80])
def test_cache_beyond_four_gigabytes(R):
    # more sequences than are cut to measure, the last one far behind 2^32 bytes of codes
    b, cap, nkv, dh = 34, 65536, 32, 128
    kc, ks, vc, vs = u8(b, cap, nkv, dh // 2), u8(b, cap, nkv, dh // 16), u8(b, cap, nkv, dh // 2), u8(b, cap, nkv, dh // 16)
    g = torch.Generator().manual_seed(2)
    n = 200
    k, v = (torch.randn((b, n, nkv * dh), generator=g).bfloat16() for _ in range(2))
    idx = torch.arange(cap - n, cap, dtype=torch.int32).repeat(b, 1)
    idx[0] = torch.arange(n, dtype=torch.int32)
    lens = torch.full((b,), 0, dtype=torch.int32)
    lens[0], lens[-1] = n, cap
    Bd.polestar_k_kv4_append(k.cuda(), v.cuda(), idx.cuda(), None, kc, ks, vc, vs)
    q = torch.randn((b, R, nkv * dh), generator=g).bfloat16()
    out = torch.full_like(q, 3.0, device="cuda")
    lse = torch.zeros((b, R, nkv), device="cuda")
    scratch = u8(Bd.polestar_k_kv4_scratch_bytes(b, R, cap, nkv, nkv, dh))
    Bd.polestar_k_kv4_attention(q.cuda(), kc, ks, vc, vs, None, None, lens.cuda(), out, lse, scratch)
    assert not out[1:-1].any() and torch.isinf(lse[1:-1]).all()
    for i, zeros in ((0, 0), (b - 1, cap - n)):                         # rows of zeros score 0 and are worth 0
        kv = [torch.from_numpy(F.quantize(x[i].float().numpy().reshape(n, nkv, dh), F.NV)[2]) for x in (k, v)]
        for h in (0, 17, 31):
            s = q[i, :, h * dh:(h + 1) * dh].double() @ kv[0][:, h].T / math.sqrt(dh)
            total = s.exp().sum(-1) + zeros
            want, size = (s.exp() @ kv[1][:, h]) / total[:, None], (s.exp() @ kv[1][:, h].abs()) / total[:, None]
            got = out[i, :, h * dh:(h + 1) * dh].double().cpu()
            assert ((got - want).abs() <= size * 2.0 ** -8 + want.abs() * 2.0 ** -8 + 1e-9).all()
            assert ((lse[i, :, h].double().cpu() - total.log()).abs() <= 1e-4).all()


def test_logits_rows_beyond_four_gigabytes():
    rows, V, ld = 3, 5000, 1 << 31
    buf = torch.zeros((rows - 1) * ld + V, dtype=torch.bfloat16, device="cuda")
    m = buf.as_strided((rows, V), (ld, 1))
    x = torch.randn((rows, V), generator=torch.Generator().manual_seed(3)).bfloat16()
    m.copy_(x)
    lp, h = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    ids, tops = torch.zeros((rows, 3), dtype=torch.int32, device="cuda"), torch.zeros((rows, 3), device="cuda")
    Bd.polestar_k_token_logprobs(m, torch.arange(rows, dtype=torch.int32, device="cuda"), None, lp, h, ids, tops)
    want = torch.log_softmax(x.double(), -1)
    assert (lp.double().cpu() - want[range(rows), range(rows)]).abs().max() < 1e-5
    assert torch.equal(tops.double().cpu().argsort(-1, descending=True), torch.arange(3).repeat(rows, 1))
    assert (tops.double().cpu() - want.topk(3, -1).values).abs().max() < 1e-5
