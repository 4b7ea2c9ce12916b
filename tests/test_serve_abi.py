"""The serving operators' C ABI on the CPU: what it refuses before anything is enqueued, and workspace sizes (no kernel is
launched by these tests)."""
import ctypes
import os

import pytest

from paper_2505_14022_amd import msda

INVALID, UNSUPPORTED, OK = msda.MSDA_ERROR_INVALID_VALUE, msda.MSDA_ERROR_NOT_SUPPORTED, msda.MSDA_SUCCESS
FAILED = msda.MSDA_ERROR_LAUNCH_FAILED  # every check passed: there is no GPU


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(msda.LIB_PATH):
        pytest.skip("libmsda.so not built")
    return msda.lib()


@pytest.fixture
def no_gpu():
    """Fabricated device addresses are only passed where no GPU is visible."""
    import torch

    if torch.cuda.device_count() > 0:
        pytest.skip("fabricated device addresses are only passed where no GPU is visible")


# ---------------------------------------------------------------- norm and rows in 8 bits


def rms(L, entry="msda_rmsnorm_forward", rows=4, C=8, eps=1e-6, dtype=0, x=0x1000, out=0x2000, scale=0x3000, weight=None,
        residual=None, sum=None):
    return getattr(L, entry)(x, residual, weight, out, *((sum, scale) if entry.endswith("forward") else (scale, sum)), rows, C,
                             eps, dtype, None)


@pytest.mark.parametrize("entry", ["msda_rmsnorm_forward", "msda_rmsnorm_quantize"])
@pytest.mark.parametrize("kw,status,needle", [
    (dict(rows=-1), INVALID, "rows"), (dict(C=0), INVALID, "C=0"), (dict(dtype=3), INVALID, "dtype"),
    (dict(dtype=-1), INVALID, "dtype"), (dict(eps=-1e-6), INVALID, "eps"), (dict(eps=float("nan")), INVALID, "eps"),
    (dict(eps=float("inf")), INVALID, "eps"), (dict(C=16385), UNSUPPORTED, "16384"),
    (dict(rows=1 << 58), UNSUPPORTED, "too large"), (dict(x=None), INVALID, "non-null"), (dict(out=None), INVALID, "non-null"),
    (dict(x=0x1002), INVALID, "misaligned"), (dict(weight=0x1002), INVALID, "misaligned"),
    (dict(scale=0x3001), INVALID, "misaligned"), (dict(dtype=1, residual=0x1001), INVALID, "misaligned"),
    (dict(sum=0x1002), INVALID, "misaligned"),
])
def test_rmsnorm_refuses(L, no_gpu, entry, kw, status, needle):
    assert rms(L, entry, **kw) == status and needle in msda.last_error()


def test_quantize_refuses(L, no_gpu):
    def call(x=0x1000, codes=0x2001, scale=0x3000, rows=3, C=5, dtype=2):
        return L.msda_quantize_rows(x, codes, scale, rows, C, dtype, None)

    assert rms(L, "msda_rmsnorm_quantize", scale=None) == INVALID and "non-null" in msda.last_error()
    for kw in (dict(x=None), dict(codes=None), dict(scale=None), dict(x=0x1001), dict(scale=0x3002), dict(rows=-1), dict(C=0),
               dict(dtype=5)):
        assert call(**kw) == INVALID, kw
    assert call(C=1 << 20) == UNSUPPORTED
    assert call(rows=0, x=None, codes=None, scale=None) == OK
    assert call() == FAILED


def test_rmsnorm_backward_refuses(L, no_gpu):
    def call(rows=4, C=8, dtype=0, x=0x1000, rstd=0x3000, gx=0x4000, gw=0x5000, ws=0x10000, nbytes=1 << 20, gs=None):
        return L.msda_rmsnorm_backward(x, None, None, 0x2000, gs, rstd, gx, gw, ws, nbytes, rows, C, dtype, None)

    for kw, needle in ((dict(x=None), "non-null"), (dict(rstd=None), "non-null"), (dict(gx=None), "non-null"),
                       (dict(gw=0x5002), "misaligned"), (dict(gx=0x4001), "misaligned"), (dict(gs=0x4002), "misaligned"),
                       (dict(ws=None, nbytes=0), "workspace"), (dict(nbytes=31), "workspace"), (dict(ws=0x10008), "aligned"),
                       (dict(rows=-2), "rows"), (dict(dtype=9), "dtype")):
        assert call(**kw) == INVALID and needle in msda.last_error(), kw
    assert call(rows=0, gw=None, x=None, rstd=None, gx=None, ws=None, nbytes=0) == OK


@pytest.mark.parametrize("rows,C,dtype", [(1, 1, 0), (300, 256, 1), (39894, 1024, 2), (2, 16384, 0)])
def test_rmsnorm_workspace_size(L, rows, C, dtype):
    # a sum of C columns for each of at most 1024 workgroups
    n = msda.rmsnorm_workspace_size(rows, C, dtype)
    assert n % (4 * C) == 0 and 4 * C <= n <= 1024 * 4 * C
    assert msda.rmsnorm_workspace_size(0, C, dtype) == 0
    with pytest.raises(msda.MsdaError):
        msda.rmsnorm_workspace_size(rows, 0, dtype)


# ---------------------------------------------------------------- products


def product(L, T=4, K=64, O=32, dtype=0, a=0x1000, b=0x2000, a_scale=0x3000, b_scale=0x4000, bias=None, out=0x5000):
    return L.msda_quantized_matmul(a, b, a_scale, b_scale, bias, out, T, K, O, dtype, None)


@pytest.mark.parametrize("kw,status,needle", [
    (dict(T=-1), INVALID, "T="), (dict(O=-1), INVALID, "O="), (dict(K=0), INVALID, "K="), (dict(dtype=3), INVALID, "dtype"),
    (dict(K=131072), UNSUPPORTED, "131071"), (dict(T=(1 << 31) - 1000), UNSUPPORTED, "2^31"), (dict(O=1 << 33), UNSUPPORTED, "2^31"),
    (dict(a=None), INVALID, "non-null"), (dict(b=None), INVALID, "non-null"), (dict(a_scale=None), INVALID, "non-null"),
    (dict(b_scale=None), INVALID, "non-null"), (dict(out=None), INVALID, "non-null"), (dict(a_scale=0x3001), INVALID, "misaligned"),
    (dict(bias=0x3002), INVALID, "misaligned"), (dict(out=0x5002), INVALID, "misaligned"), (dict(out=0x5001, dtype=1), INVALID, "misaligned"),
    (dict(T=1 << 30, O=1 << 30), UNSUPPORTED, "launch"), (dict(T=1 << 30, O=1 << 30, K=7), UNSUPPORTED, "launch"),
    (dict(T=64, O=(1 << 31) - 2048, K=7), UNSUPPORTED, "launch"),
])
def test_product_refuses(L, no_gpu, kw, status, needle):
    assert product(L, **kw) == status and needle in msda.last_error()


def test_product_takes_any_codes(L, no_gpu):
    for kw in (dict(), dict(a=0x1001, K=7), dict(O=1), dict(T=1), dict(T=1 << 20, O=1 << 12), dict(K=131071), dict(out=0x5002, dtype=2)):
        assert product(L, **kw) == FAILED, kw
    assert product(L, T=0, a=None, b=None, a_scale=None, b_scale=None, out=None) == OK
    assert product(L, O=0, a=None, b=None, a_scale=None, b_scale=None, out=None) == OK


# ---------------------------------------------------------------- paged cache


def cache(**kw):
    d = dict(N=3, pages=20, page_size=16, Mkv=2, D=32, width=5, table_stride=5, k=0x1000, v=0x2000, k_scale=0x3000, v_scale=0x4000,
             table=0x5000, length=0x6000, start=0x7000)
    d.update(kw)
    return msda.CacheDescription(*d.values())


def append(L, c, k=0x10000, ks=(64, 32), v=0x20000, vs=(64, 32), pos=0x30000, freqs=0x40000, T=9, A=1, R=16, dtype=2):
    two = ctypes.c_int64 * 2
    return L.msda_cache_append(ctypes.byref(c) if c else None, k, two(*ks) if ks else None, v, two(*vs) if vs else None, pos, freqs, T,
                               A, R, 0, dtype, None)


def attention(L, c, q=0x10000, qs=(128, 32), out=0x20000, lse=0x30000, T=9, M=4, scale=0.1, softcap=0.0, dtype=2, ws=0x100000,
              nbytes=1 << 40):
    return L.msda_cache_attention(ctypes.byref(c) if c else None, q, (ctypes.c_int64 * 2)(*qs) if qs else None, out, lse, T, M, scale,
                                  softcap, 1, dtype, ws, nbytes, None)


def size(L, c, T=9, M=4, dtype=2):
    n = ctypes.c_size_t(77)
    return L.msda_cache_attention_workspace_size(ctypes.byref(c), T, M, dtype, ctypes.byref(n)), n.value


@pytest.mark.parametrize("kw,status,needle", [
    (dict(N=-1), INVALID, "N="), (dict(pages=-1), INVALID, "pages="), (dict(width=-1), INVALID, "width="), (dict(Mkv=0), INVALID, "Mkv="),
    (dict(D=0), INVALID, "D="), (dict(page_size=8), UNSUPPORTED, "page_size=8"), (dict(page_size=48), UNSUPPORTED, "page_size=48"),
    (dict(page_size=512), UNSUPPORTED, "page_size=512"), (dict(D=40), UNSUPPORTED, "multiple of 16"), (dict(D=144), UNSUPPORTED, "128"),
    (dict(Mkv=65537), UNSUPPORTED, "65536"), (dict(N=1 << 24), UNSUPPORTED, "2^24"), (dict(pages=1 << 31), UNSUPPORTED, "pages="),
    (dict(width=1 << 27), UNSUPPORTED, "width="), (dict(table_stride=4), INVALID, "table_stride"), (dict(start=None), INVALID, "T=9"),
    (dict(k=None), INVALID, "non-null"), (dict(v_scale=None), INVALID, "non-null"), (dict(table=None), INVALID, "non-null"),
    (dict(length=None), INVALID, "non-null"), (dict(k=0x1008), INVALID, "16 bytes"), (dict(v=0x2001), INVALID, "16 bytes"),
    (dict(k_scale=0x3002), INVALID, "misaligned"), (dict(table=0x5001), INVALID, "misaligned"), (dict(start=0x7002), INVALID, "misaligned"),
])
def test_cache_refuses(L, no_gpu, kw, status, needle):
    c = cache(**kw)
    M = 4 if c.Mkv == 2 else max(c.Mkv, 1)
    assert append(L, c, R=min(16, max(c.D // 2, 0))) == status and needle in msda.last_error()
    assert attention(L, c, M=M) == status and needle in msda.last_error()


@pytest.mark.parametrize("kw,status,needle", [
    (dict(T=-1), INVALID, "T="), (dict(dtype=3), INVALID, "dtype"), (dict(A=0), INVALID, "A=0"), (dict(A=5), INVALID, "A=5"),
    (dict(A=2, pos=None), INVALID, "pos"), (dict(R=-1), INVALID, "R=-1"), (dict(R=17), INVALID, "R=17"), (dict(k=None), INVALID, "non-null"),
    (dict(v=None), INVALID, "non-null"), (dict(freqs=None), INVALID, "non-null"), (dict(ks=None), INVALID, "stride"),
    (dict(vs=None), INVALID, "stride"), (dict(ks=(-64, 32)), INVALID, "stride"), (dict(vs=(64, -32)), INVALID, "stride"),
    (dict(k=0x10001), INVALID, "misaligned"), (dict(v=0x20001), INVALID, "misaligned"), (dict(pos=0x30002), INVALID, "misaligned"),
    (dict(T=(1 << 31) - 1000), UNSUPPORTED, "2^31"),
])
def test_append_refuses(L, no_gpu, kw, status, needle):
    assert append(L, cache(), **kw) == status and needle in msda.last_error()


def test_append_takes_what_it_documents(L, no_gpu):
    assert append(L, None) == INVALID
    assert append(L, cache(), T=0, k=None, v=None, pos=None, freqs=None) == OK
    assert append(L, cache(N=0, table_stride=0, k=None, v=None), T=4) == OK
    assert append(L, cache(pages=0, k=None, v=None, k_scale=None, v_scale=None)) == OK  # no page exists: nothing is stored
    for kw in (dict(), dict(pos=None), dict(R=0, freqs=None, pos=None), dict(ks=(0, 0)), dict(k=0x10002), dict(dtype=0, A=4)):
        assert append(L, cache(), **kw) == FAILED, kw
    assert append(L, cache(start=None), T=3) == FAILED
    assert append(L, cache(N=1 << 23, Mkv=2048), R=0) == UNSUPPORTED and "launch" in msda.last_error()


@pytest.mark.parametrize("kw,status,needle", [
    (dict(T=-1), INVALID, "T="), (dict(dtype=3), INVALID, "dtype"), (dict(M=0), INVALID, "M=0"), (dict(M=3), INVALID, "M=3"),
    (dict(M=65538), UNSUPPORTED, "65536"), (dict(scale=0.0), INVALID, "scale"), (dict(scale=-1.0), INVALID, "scale"),
    (dict(scale=float("nan")), INVALID, "scale"), (dict(scale=2e38), INVALID, "scale"), (dict(softcap=-1.0), INVALID, "softcap"),
    (dict(softcap=float("inf")), INVALID, "softcap"), (dict(softcap=1e-38), INVALID, "softcap"), (dict(qs=None), INVALID, "stride"),
    (dict(qs=(-1, 32)), INVALID, "stride"), (dict(q=None), INVALID, "non-null"), (dict(out=None), INVALID, "non-null"),
    (dict(q=0x10001), INVALID, "misaligned"), (dict(out=0x20008), INVALID, "16 bytes"), (dict(lse=0x30002), INVALID, "misaligned"),
    (dict(T=1 << 28), UNSUPPORTED, "launch"),
])
def test_cache_attention_refuses(L, no_gpu, kw, status, needle):
    assert attention(L, cache(), **kw) == status and needle in msda.last_error()
    if set(kw) <= {"T", "M", "dtype"}:
        assert size(L, cache(), **kw) == (status, 0)


def test_cache_attention_workspace(L, no_gpu):
    long = cache(width=1000, table_stride=1000)
    st, need = size(L, long)
    assert st == OK and need > 0
    for kw in (dict(ws=None), dict(nbytes=need - 1), dict(ws=0x100008)):
        assert attention(L, long, **kw) == INVALID and "workspace" in msda.last_error()
    assert attention(L, long, nbytes=need) == FAILED
    assert size(L, cache()) == (OK, 0) and attention(L, cache(), ws=None, nbytes=0, lse=None) == FAILED
    assert attention(L, None) == INVALID and L.msda_cache_attention_workspace_size(None, 1, 1, 0, None) == INVALID
    assert attention(L, cache(), T=0, q=None, out=None) == OK and size(L, cache(), T=0) == (OK, 0)
    # the partial results of splits stay within half a GB, or there are none
    for T in (1, 300, 70000, 1 << 20):
        for N in (1, 64, 5000):
            for width in (1, 100, 8000, 100000):
                st, need = size(L, cache(N=N, width=width, table_stride=width, Mkv=8, D=128), T=T, M=64)
                assert st == OK and need <= 1 << 29


def test_python_checks_its_tensors(L):
    import torch

    x = torch.zeros(4, 32)
    codes = torch.zeros(4, 32, dtype=torch.int8)
    with pytest.raises(ValueError, match="device tensors"):
        msda.rmsnorm_forward(x)
    with pytest.raises(ValueError, match="dtype"):
        msda.rmsnorm_quantize(x.double())
    with pytest.raises(ValueError, match="device tensors"):
        msda.quantize_rows(x)
    with pytest.raises(ValueError, match="must be torch.int8"):
        msda.quantized_matmul(x, codes, x[:, 0], x[:, 0])
    with pytest.raises(ValueError, match="b must be"):
        msda.quantized_matmul(codes, codes[0], x[:, 0], x[:, 0])
    pool = torch.zeros(5, 1, 16, 32, dtype=torch.int8)
    scale, table, n = torch.zeros(5, 1), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    k = x.view(4, 1, 32)
    with pytest.raises(ValueError, match="device tensors"):
        msda.cache_append(k, k, pool, pool, scale, scale, table, n)
    with pytest.raises(ValueError, match="pos needs freqs"):
        msda.cache_append(k, k, pool, pool, scale, scale, table, n, pos=x)
    with pytest.raises(ValueError, match="k must be"):
        msda.cache_append(x, x, pool, pool, scale, scale, table, n)
    with pytest.raises(ValueError, match="k_cache must be"):
        msda.cache_attention(k, pool[0], pool[0], scale, scale, table, n)
    with pytest.raises(ValueError, match="q must be"):
        msda.cache_attention(x, pool, pool, scale, scale, table, n)
