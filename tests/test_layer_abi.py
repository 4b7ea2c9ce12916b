"""The layer operators' C ABI on the CPU: what it refuses before anything is enqueued, and workspace sizes (no kernel
is launched by these tests)."""
import ctypes
import os

import pytest

from paper_2505_14022_amd import msda

INVALID, UNSUPPORTED, OK = msda.MSDA_ERROR_INVALID_VALUE, msda.MSDA_ERROR_NOT_SUPPORTED, msda.MSDA_SUCCESS


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


def ln_forward(L, rows=4, C=8, eps=1e-5, dtype=0, x=0x1000, out=0x2000, weight=None, residual=None, mean=None):
    return L.msda_layernorm_forward(x, residual, weight, None, out, None, mean, None, rows, C, eps, dtype, None)


@pytest.mark.parametrize("kw,status,needle", [
    (dict(rows=-1), INVALID, "rows"), (dict(C=0), INVALID, "C=0"), (dict(dtype=3), INVALID, "dtype"),
    (dict(dtype=-1), INVALID, "dtype"), (dict(eps=-1e-6), INVALID, "eps"), (dict(eps=float("nan")), INVALID, "eps"),
    (dict(eps=float("inf")), INVALID, "eps"), (dict(C=16385), UNSUPPORTED, "16384"),
    (dict(rows=1 << 58), UNSUPPORTED, "too large"), (dict(x=None), INVALID, "non-null"), (dict(out=None), INVALID, "non-null"),
    (dict(x=0x1002), INVALID, "misaligned"), (dict(weight=0x1002), INVALID, "misaligned"),
    (dict(mean=0x1001), INVALID, "misaligned"), (dict(dtype=1, residual=0x1001), INVALID, "misaligned"),
])
def test_layernorm_forward_refuses(L, no_gpu, kw, status, needle):
    assert ln_forward(L, **kw) == status and needle in msda.last_error()


def test_layernorm_empty_is_a_no_op(L):
    assert ln_forward(L, rows=0, x=None, out=None) == OK


def ln_backward(L, rows=4, C=8, dtype=0, x=0x1000, mean=0x3000, gx=0x4000, gw=0x5000, gb=None, ws=0x10000, nbytes=1 << 20):
    return L.msda_layernorm_backward(x, None, None, 0x2000, None, mean, 0x3800, gx, gw, gb, ws, nbytes, rows, C, dtype, None)


@pytest.mark.parametrize("kw,needle", [
    (dict(x=None), "non-null"), (dict(mean=None), "non-null"), (dict(gx=None), "non-null"), (dict(gw=0x5002), "misaligned"),
    (dict(gx=0x4001), "misaligned"), (dict(ws=None, nbytes=0), "workspace"), (dict(nbytes=63), "workspace"),
    (dict(ws=0x10008), "aligned"), (dict(gw=None, gb=0x5000, nbytes=0), "workspace"), (dict(rows=-2), "rows"),
])
def test_layernorm_backward_refuses(L, no_gpu, kw, needle):
    assert ln_backward(L, **kw) == INVALID and needle in msda.last_error()


@pytest.mark.parametrize("rows,C,dtype", [(1, 1, 0), (300, 256, 1), (87296, 1024, 1), (39894, 256, 2), (2, 16384, 0)])
def test_layernorm_workspace_size(L, rows, C, dtype):
    # two sums of C columns for each of at most 1024 workgroups
    n = msda.layernorm_workspace_size(rows, C, dtype)
    assert n % (8 * C) == 0 and 8 * C <= n <= 1024 * 8 * C
    assert msda.layernorm_workspace_size(0, C, dtype) == 0
    with pytest.raises(msda.MsdaError):
        msda.layernorm_workspace_size(rows, 0, dtype)


def rotary(L, N=2, T=3, M=4, D=16, A=2, R=8, items=2, dtype=0, x=0x1000, out=0x9000, xs=None, os_=None, pos=0x2000,
           freqs=0x3000, entry="msda_rotary_forward"):
    arr = ctypes.c_int64 * 3
    return getattr(L, entry)(x, arr(*xs) if xs else None, pos, freqs, out, arr(*os_) if os_ else None, N, T, M, D, A, R,
                             items, 0, dtype, None)


@pytest.mark.parametrize("entry", ["msda_rotary_forward", "msda_rotary_backward"])
@pytest.mark.parametrize("kw,status,needle", [
    (dict(N=-1), INVALID, "N="), (dict(T=-1), INVALID, "T="), (dict(M=0), INVALID, "M="), (dict(D=0), INVALID, "D="),
    (dict(A=0), INVALID, "A=0"), (dict(A=5), INVALID, "A=5"), (dict(R=9), INVALID, "R=9"), (dict(R=-1), INVALID, "R="),
    (dict(items=3), INVALID, "pos_items"), (dict(dtype=7), INVALID, "dtype"), (dict(D=1025, R=4), UNSUPPORTED, "1024"),
    (dict(M=4097), UNSUPPORTED, "65536"), (dict(x=None), INVALID, "non-null"), (dict(pos=None), INVALID, "non-null"),
    (dict(x=0x1002), INVALID, "misaligned"), (dict(os_=(192, 0, 16)), INVALID, "stride of 0"),
    (dict(N=1 << 32, items=1), UNSUPPORTED, "2^31"),
])
def test_rotary_refuses(L, no_gpu, entry, kw, status, needle):
    assert rotary(L, entry=entry, **kw) == status and needle in msda.last_error()


def test_rotary_empty_is_a_no_op(L):
    assert rotary(L, T=0, x=None, out=None, pos=None, freqs=None) == OK
    assert rotary(L, N=0, items=0, x=None, out=None, pos=None, freqs=None) == OK


def description(**kw):
    d = dict(N=2, Lq=70, Lk=90, M=4, Mkv=2, D=32, dtype=2, causal=0, unaligned=0, scale=0.1, softcap=0.0)
    tables = {k: kw.pop(k, None) for k in ("slopes", "q_pos", "k_pos", "q_doc", "k_doc", "prefix")}
    d.update(kw)
    arr = ctypes.c_int64 * 3
    return msda.AttentionDescription(*(d[k] for k in ("N", "Lq", "Lk", "M", "Mkv", "D", "dtype", "causal", "unaligned", "scale", "softcap")),
                                     arr(d["Lq"] * d["M"] * d["D"], d["M"] * d["D"], d["D"]),
                                     *(arr(d["Lk"] * d["Mkv"] * d["D"], d["Mkv"] * d["D"], d["D"]) for _ in range(2)),
                                     *tables.values())


def forward(L, a, q=0x1000, k=0x2000, v=0x3000, out=0x4000, lse=0x5000, ws=0x10000, nbytes=1 << 30):
    return L.msda_attention_forward(ctypes.byref(a), q, k, v, out, lse, ws, nbytes, None)


def backward(L, a, lse=0x5000, go=0x6000, gq=0x7000, gk=0x8000, gv=0x9000, ws=0x10000, nbytes=1 << 30):
    return L.msda_attention_backward(ctypes.byref(a), 0x1000, 0x2000, 0x3000, 0x4000, lse, go, gq, gk, gv, ws, nbytes, None)


@pytest.mark.parametrize("kw,status,needle", [
    (dict(N=-1), INVALID, "N="), (dict(Lq=-1), INVALID, "Lq="), (dict(Lk=-3), INVALID, "Lk="), (dict(M=0), INVALID, "M="),
    (dict(Mkv=0), INVALID, "Mkv="), (dict(M=5), INVALID, "multiple"), (dict(D=0), INVALID, "D="), (dict(D=129), UNSUPPORTED, "128"),
    (dict(dtype=3), INVALID, "dtype"), (dict(scale=0.0), INVALID, "scale"), (dict(scale=-1.0), INVALID, "scale"),
    (dict(scale=float("nan")), INVALID, "scale"), (dict(scale=float("inf")), INVALID, "scale"),
    (dict(softcap=-1.0), INVALID, "softcap"), (dict(softcap=float("nan")), INVALID, "softcap"),
    (dict(causal=1, Lq=91), INVALID, "causal"), (dict(q_doc=0x100), INVALID, "q_doc"), (dict(k_doc=0x100), INVALID, "q_doc"),
    (dict(slopes=0x100), INVALID, "slopes"), (dict(slopes=0x100, q_pos=0x100, k_pos=0x104), INVALID, "misaligned"),
    (dict(prefix=0x102), INVALID, "misaligned"), (dict(Lk=1 << 31), UNSUPPORTED, "2^31"),
    (dict(Lq=1 << 30), UNSUPPORTED, "2^31"), (dict(N=1 << 30, M=1 << 10, Mkv=1 << 10), UNSUPPORTED, "launch"),
    (dict(N=1 << 20, Lk=1 << 20), UNSUPPORTED, "launch"), (dict(M=32770), UNSUPPORTED, "32768"),
])
def test_attention_refuses(L, no_gpu, kw, status, needle):
    a = description(**kw)
    size = ctypes.c_size_t(0)
    assert L.msda_attention_workspace_size(ctypes.byref(a), 0, ctypes.byref(size)) == status and needle in msda.last_error()
    assert forward(L, a) == status and needle in msda.last_error()
    assert backward(L, a) == status and needle in msda.last_error()


def test_attention_refuses_bad_pointers_and_workspaces(L, no_gpu):
    a = description(q_doc=0x100, k_doc=0x200)
    need = []
    for b in (0, 1):
        size = ctypes.c_size_t(0)
        assert L.msda_attention_workspace_size(ctypes.byref(a), b, ctypes.byref(size)) == OK
        need.append(size.value)
    assert 0 < need[0] < need[1]
    for kw in (dict(q=None), dict(k=None), dict(out=None), dict(q=0x1008), dict(v=0x3002), dict(out=0x4008), dict(lse=0x5002),
               dict(ws=None, nbytes=0), dict(nbytes=need[0] - 1), dict(ws=0x10008)):
        assert forward(L, a, **kw) == INVALID, kw
    loose = description(unaligned=1)  # may start anywhere but off its elements
    assert forward(L, loose, q=0x1001) == INVALID and "misaligned" in msda.last_error()
    assert forward(L, loose, q=0x1002, nbytes=0) == INVALID and "workspace" in msda.last_error()
    for kw in (dict(lse=None), dict(go=None), dict(gq=None), dict(gk=None), dict(gv=None), dict(go=0x6008), dict(gv=0x9002),
               dict(ws=None, nbytes=0), dict(nbytes=need[1] - 1)):
        assert backward(L, a, **kw) == INVALID, kw
    assert L.msda_attention_forward(None, None, None, None, None, None, None, 0, None) == INVALID
    assert L.msda_attention_workspace_size(ctypes.byref(a), 0, None) == INVALID


@pytest.mark.parametrize("which", ["q_stride", "k_stride", "v_stride"])
def test_attention_refuses_negative_strides(L, no_gpu, which):
    for i in range(3):
        a = description()
        getattr(a, which)[i] = -8
        assert forward(L, a) == INVALID and "strides" in msda.last_error()
        assert backward(L, a) == INVALID and "strides" in msda.last_error()


@pytest.mark.parametrize("which,rows", [("q_stride", 70 * 4), ("k_stride", 90 * 2), ("v_stride", 90 * 2)])
def test_attention_copies_rows_that_lie_far_apart(L, which, rows):
    """The kernels' offsets within a tile of 128 tokens have 31 bits: tokens of 2^24 bytes are copied to rows of 64."""
    def need(stride, backward):
        a = description()
        if stride:
            getattr(a, which)[1] = stride
            getattr(a, which)[0] = stride * 90
        size = ctypes.c_size_t(0)
        assert L.msda_attention_workspace_size(ctypes.byref(a), backward, ctypes.byref(size)) == OK
        return size.value

    for b in (0, 1):
        assert need(1 << 22, b) == need(0, b)
        for stride in (1 << 23, 3 << 22, 1 << 24, 1 << 33):
            assert need(stride, b) >= need(0, b) + 2 * rows * 64


def test_attention_empty_is_a_no_op(L):
    for kw in (dict(N=0), dict(Lq=0)):
        assert forward(L, description(**kw), None, None, None, None, None, None, 0) == OK
    assert backward(L, description(Lq=0, Lk=0), None, None, None, None, None, None, 0) == OK


def test_python_checks_its_tensors(L):
    import torch

    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="device tensors"):
        msda.layernorm_forward(x)
    with pytest.raises(ValueError, match="dtype"):
        msda.layernorm_forward(x.double())
    with pytest.raises(ValueError, match="freqs"):
        msda.rotary_forward(x, x, x)
    q = torch.zeros(1, 2, 4, 8)
    with pytest.raises(ValueError, match="device tensors"):
        msda.attention_forward(q, q, q)
    with pytest.raises(ValueError, match="k must be|q must be"):
        msda.attention_forward(q, x, x)


def attention_size(L, grads, **kw):
    size = ctypes.c_size_t(0)
    return L.msda_attention_workspace_size(ctypes.byref(description(**kw)), grads, ctypes.byref(size))


@pytest.mark.parametrize("most,grads,kw", [
    # a workgroup of 256 a head in the backward, of 64 in the forward of few rows
    (2 ** 21 - 1, 1, dict(M=8, Mkv=8, Lq=1, Lk=1)), (2 ** 23 - 1, 0, dict(M=8, Mkv=8, Lq=1, Lk=1)),
    # tables of documents, a wave for each tile and block of a batch item: 2 in the forward, 4 with the backward's
    (2 ** 25 - 2, 0, dict(M=1, Mkv=1, Lq=1, Lk=1, q_doc=0x100, k_doc=0x200)),
    # copies of 16 bytes, of 2^22 an item here
    (2 ** 10 - 1, 0, dict(M=32, Mkv=4, Lq=2 ** 15, Lk=100, unaligned=1)),
])
def test_attention_refuses_grids_that_the_runtime_does_not_take(L, no_gpu, most, grads, kw):
    call = backward if grads else forward
    assert attention_size(L, grads, N=most, **kw) == OK
    for n in (most + 1, most + 9, 2 * most):
        assert attention_size(L, grads, N=n, **kw) == UNSUPPORTED and "launch" in msda.last_error()
        # with all pointers and a workspace said to be large enough: refused before anything is enqueued
        assert call(L, description(N=n, **kw), nbytes=1 << 60) == UNSUPPORTED and "launch" in msda.last_error()


@pytest.mark.parametrize("entry", ["msda_rotary_forward", "msda_rotary_backward"])
@pytest.mark.parametrize("kw", [dict(M=8, D=1024, R=0, dtype=1), dict(M=8, D=1024, R=64, dtype=0, x=0x1004),
                                dict(M=513, D=1, R=0, dtype=2)])
def test_rotary_refuses_grids_that_the_runtime_does_not_take(L, no_gpu, entry, kw):
    assert rotary(L, entry=entry, N=1, T=2 ** 24, A=1, items=1, **kw) == UNSUPPORTED and "launch" in msda.last_error()
    assert rotary(L, entry=entry, N=1, T=2 ** 24 - 1, A=1, items=1, **kw) == msda.MSDA_ERROR_LAUNCH_FAILED  # there is no GPU


@pytest.mark.parametrize("kw,needle", [
    (dict(scale=3e38), "scale"), (dict(softcap=3e38), "softcap"), (dict(scale=1.0, softcap=1e-39), "softcap"),
    (dict(scale=100.0, softcap=4e-37), "softcap"), (dict(scale=1e-3, softcap=1e-45), "softcap"),
])
def test_attention_refuses_factors_that_overflow(L, no_gpu, kw, needle):
    # zero scores times such a factor would be NaN
    assert attention_size(L, 0, **kw) == INVALID and needle in msda.last_error()
    assert forward(L, description(**kw)) == INVALID and needle in msda.last_error()
    assert backward(L, description(**kw)) == INVALID and needle in msda.last_error()


@pytest.mark.parametrize("kw", [dict(scale=1e38), dict(softcap=1e38), dict(scale=1e-3, softcap=1e-38), dict(scale=1e-45)])
def test_attention_takes_factors_up_to_there(L, no_gpu, kw):
    assert attention_size(L, 1, **kw) == OK
