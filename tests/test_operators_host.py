"""The 4-bit and log-probability entry points refuse what they cannot take before they touch the device (no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2607_14107_b200 import binding as Bd
from paper_2607_14107_b200 import build as build_mod


@pytest.fixture(scope="module")
def lib():
    build_mod.build()
    return Bd.load()


OK = 0x7000001000          # an aligned address that nothing reads


def p(off=0):
    return C.c_void_p(OK + off)


def test_scale_bytes(lib):
    f = lib.polestar_k_fp4_scale_bytes
    assert f(5, 64, Bd.FP4_NV, Bd.SCALES_ROWS) == 5 * 4 and f(5, 64, Bd.FP4_MX, Bd.SCALES_ROWS) == 5 * 2
    assert f(1, 64, Bd.FP4_NV, Bd.SCALES_TILED) == 512 and f(129, 96, Bd.FP4_NV, Bd.SCALES_TILED) == 2 * 2 * 512
    assert f(128, 128, Bd.FP4_MX, Bd.SCALES_TILED) == 512 and f(128, 160, Bd.FP4_MX, Bd.SCALES_TILED) == 1024
    assert f(0, 64, Bd.FP4_NV, Bd.SCALES_ROWS) == 0
    for bad in ((-1, 64, 0, 0), (4, 48, 0, 0), (4, 0, 0, 0), (4, 64, 2, 0), (4, 64, 0, 2), (1 << 31, 64, 0, 0)):
        assert f(*bad) == 0
    assert f((1 << 31) - 1, 1 << 20, Bd.FP4_NV, Bd.SCALES_ROWS) == ((1 << 31) - 1) << 16


def quantize(lib, x=p(), ld=64, rows=2, d=64, dtype=1, fmt=0, layout=0, t=None, codes=p(), scales=p(), deq=None):
    return lib.polestar_k_fp4_quantize(x, ld, rows, d, dtype, fmt, layout, t, codes, scales, deq, None)


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(d=0), dict(d=48, ld=48), dict(d=-32), dict(ld=32), dict(ld=68), dict(dtype=2), dict(fmt=2), dict(fmt=-1), dict(layout=2),
    dict(x=None), dict(codes=None), dict(scales=None), dict(x=p(8)), dict(codes=p(2)), dict(deq=p(4)), dict(t=p(2)), dict(layout=1, scales=p(2)),
    dict(dtype=0, ld=66),
])
def test_quantize_refuses(lib, bad):
    assert quantize(lib, **bad) == Bd.E_INVAL
    assert quantize(lib, rows=0, x=None, codes=None, scales=None) == Bd.OK


def matmul(lib, ac=p(), asc=p(), bc=p(), bs=p(), ta=None, tb=None, out=p(), ld=8, M=4, N=8, K=64, fmt=0, dtype=1):
    return lib.polestar_k_fp4_matmul(ac, asc, bc, bs, ta, tb, out, ld, M, N, K, fmt, dtype, None)


@pytest.mark.parametrize("bad", [
    dict(M=-1), dict(N=-1), dict(K=0), dict(K=32), dict(K=96), dict(ld=7), dict(fmt=2), dict(dtype=2), dict(ac=None), dict(asc=None), dict(bc=None),
    dict(bs=None), dict(out=None), dict(ac=p(8)), dict(asc=p(4)), dict(bc=p(8)), dict(bs=p(8)), dict(out=p(1)), dict(dtype=0, out=p(2)), dict(ta=p(1)), dict(tb=p(2)),
])
def test_matmul_refuses(lib, bad):
    assert matmul(lib, **bad) == Bd.E_INVAL
    assert matmul(lib, M=0, ac=None, out=None) == Bd.OK and matmul(lib, N=0, ld=0, bc=None) == Bd.OK


def append(lib, k=p(), v=p(), idx=None, cnt=None, batch=1, R=2, cap=8, n_kv=2, dh=128, dtype=1, tk=None, tv=None, c=(p(),) * 4, kd=None, vd=None):
    return lib.polestar_k_kv4_append(k, v, idx, cnt, batch, R, cap, n_kv, dh, dtype, tk, tv, *c, kd, vd, None)


@pytest.mark.parametrize("bad", [
    dict(batch=-1), dict(batch=65536), dict(R=-1), dict(R=65537), dict(cap=0), dict(cap=65537), dict(n_kv=0), dict(n_kv=1025), dict(dh=96), dict(dh=256),
    dict(dtype=2), dict(k=None), dict(v=None), dict(c=(None, p(), p(), p())), dict(c=(p(), p(), p(), None)), dict(k=p(8)), dict(kd=p(2)), dict(idx=p(2)),
    dict(c=(p(2), p(), p(), p())), dict(tk=p(2)), dict(cnt=p(1)),
])
def test_append_refuses(lib, bad):
    assert append(lib, **bad) == Bd.E_INVAL
    assert append(lib, R=0, k=None, v=None) == Bd.OK and append(lib, batch=0, k=None, v=None) == Bd.OK


def attention(lib, q=p(), c=(p(),) * 4, tk=None, tv=None, lens=None, out=p(), lse=None, batch=1, R=2, cap=8, nh=4, n_kv=2, dh=128, dtype=1, scratch=p(), size=1 << 40):
    return lib.polestar_k_kv4_attention(q, *c, tk, tv, lens, out, lse, batch, R, cap, nh, n_kv, dh, dtype, scratch, size, None)


@pytest.mark.parametrize("bad", [
    dict(batch=-1), dict(R=-1), dict(R=65537), dict(cap=0), dict(cap=65537), dict(nh=3), dict(nh=0), dict(n_kv=0), dict(nh=2048, n_kv=2), dict(dh=32), dict(dtype=2),
    dict(q=None), dict(out=None), dict(scratch=None), dict(c=(p(), None, p(), p())), dict(q=p(8)), dict(out=p(4)), dict(c=(p(), p(8), p(), p())), dict(scratch=p(8)),
    dict(lens=p(2)), dict(lse=p(2)), dict(tv=p(1)),
])
def test_attention_refuses(lib, bad):
    assert attention(lib, **bad) == Bd.E_INVAL
    assert attention(lib, R=0, q=None, out=None, scratch=None) == Bd.OK


def test_attention_scratch(lib):
    f = lib.polestar_k_kv4_scratch_bytes
    assert f(1, 1, 8, 4, 3, 128) == 0 and f(1, 1, 8, 4, 2, 96) == 0 and f(1, -1, 8, 4, 2, 128) == 0
    for shape in ((1, 1, 65536, 28, 4, 128), (8, 1, 32768, 28, 4, 128), (1, 2048, 2048, 32, 32, 128), (64, 65536, 65536, 1024, 1024, 128), (0, 0, 1, 1, 1, 64)):
        n = f(*shape)
        assert n >= 256
        b, R, cap, nh, n_kv, dh = shape
        if b and R:
            assert attention(lib, batch=b, R=R, cap=cap, nh=nh, n_kv=n_kv, dh=dh, size=n - 1) == Bd.E_NOSPACE
    assert f(1, 1, 65536, 28, 4, 128) < 8 << 20


def logprobs(lib, x=p(), ld=100, rows=2, V=100, dtype=0, target=p(), mask=-1, k=0, lp=p(), h=None, ids=None, tops=None):
    return lib.polestar_k_token_logprobs(x, ld, rows, V, dtype, target, mask, k, lp, h, ids, tops, None)


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(V=0), dict(ld=99), dict(dtype=2), dict(k=-1), dict(k=33, ids=p(), tops=p()), dict(x=None), dict(target=None), dict(k=1), dict(k=1, ids=p()),
    dict(x=p(2)), dict(dtype=1, x=p(1)), dict(lp=p(2)), dict(h=p(1)), dict(target=p(2)), dict(k=1, ids=p(2), tops=p()),
])
def test_logprobs_refuses(lib, bad):
    assert logprobs(lib, **bad) == Bd.E_INVAL
    assert logprobs(lib, rows=0, x=None, target=None, lp=None) == Bd.OK


def test_binding_refuses_what_the_library_cannot_see():
    # tensors on another device, of another type or shape, or with holes: the library gets addresses only
    x = torch.zeros((2, 64))
    for call in (lambda: Bd.polestar_k_fp4_quantize(x, x, x, Bd.FP4_NV),
                 lambda: Bd.polestar_k_fp4_matmul(x.byte(), x.byte(), x.byte(), x.byte(), x, Bd.FP4_NV),
                 lambda: Bd.polestar_k_token_logprobs(x, None, 0, None, None),
                 lambda: Bd.polestar_k_kv4_append(x, x, None, None, *(torch.zeros((1, 4, 2, 64), dtype=torch.uint8),) * 4),
                 lambda: Bd.polestar_k_kv4_attention(x, *(torch.zeros((1, 4, 2, 64), dtype=torch.uint8),) * 4, None, None, None, x, None, x)):
        with pytest.raises(Bd.PolestarError) as e:
            call()
        assert e.value.code == Bd.E_INVAL


def test_binding_refuses_sizes_beyond_32_bits():
    # ctypes cuts integers to 32 bits without a word: 2^32 + 64 channels would become 64
    Bd._sizes(rows=0, d=2 ** 31 - 1)
    for n in (2 ** 31, 2 ** 32, 2 ** 32 + 64):
        with pytest.raises(Bd.PolestarError) as e:
            Bd._sizes(rows=1, d=n)
        assert e.value.code == Bd.E_INVAL
        with pytest.raises(Bd.PolestarError):
            Bd.polestar_k_fp4_scale_bytes(1, n, Bd.FP4_NV, Bd.SCALES_ROWS)


@pytest.mark.parametrize("sizes", [dict(M=2 ** 31 - 1), dict(M=2 ** 31 - 255), dict(N=2 ** 31 - 1, ld=2 ** 31), dict(K=2 ** 31 - 64)])
def test_matmul_refuses_sizes_that_do_not_round_up_in_32_bits(lib, sizes):
    # tiles are counted in 32 bits: the last size with a whole tile behind it is 2^31 - 256
    assert matmul(lib, **sizes) == Bd.E_INVAL
