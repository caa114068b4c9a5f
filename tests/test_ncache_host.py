"""The 4-bit cache without a GPU: its oracle against independent definitions, argument checks of the C entry points
(every refusal comes before any HIP call) and of the binding."""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import ncache as on
from paper_2609_36835_amd import arckv as A


# ------------------------------------------------------------------------------------------------ the oracle's pins
def test_rounding_goes_to_the_nearest_code():
    """Every border between two codes, the values next to it and random values, against a search for the nearest."""
    m = np.array(on.MAGNITUDES)
    mid = (m[1:] + m[:-1]) / 2
    g = np.random.default_rng(0)
    y = np.concatenate([m, mid, np.nextafter(mid, 0), np.nextafter(mid, 9), g.uniform(0, 6, 3000), [6.5, 7.0, 8.0, 100.0]])
    for x, got in zip(y, on.n_round(y)):
        d = np.abs(m - x)
        best = np.flatnonzero(d == d.min())
        want = best[0] if len(best) == 1 else best[best % 2 == 0][0]
        assert got == m[want], x
    assert np.array_equal(on.n_round(-y), -on.n_round(y))
    assert np.signbit(on.n_round(np.array([-0.1, -0.0]))).all()


def test_scale_is_the_smallest_power_of_two():
    for a in (6.0, np.nextafter(6.0, 9), 3.0, 1e-3, 1e30, 1.0, 0.9):
        s = on.n_scale(float(a))
        assert math.frexp(s)[0] == 0.5 and a <= 6 * s and a > 3 * s
    assert on.n_scale(0.0) == on.n_scale(1e-38) == 2.0 ** -100
    assert on.n_scale(3.4e38) == 2.0 ** 125
    assert math.isnan(on.n_scale(math.inf)) and math.isnan(on.n_scale(math.nan))


def test_stored_values_are_within_half_a_step_and_stay():
    g = np.random.default_rng(1)
    x = g.standard_normal((100, 128)) * np.exp(g.uniform(-3, 3, (1, 128)))
    codes, scales = on.n_rows(x)
    v = on.n_values(codes, scales)
    s = np.repeat(scales, 32, axis=1)
    assert (np.abs(v - x) <= np.maximum(np.abs(x), s) / 4).all()
    again = on.n_rows(v)
    assert np.array_equal(on.n_values(*again), v)
    assert np.array_equal(on.n_unpack(*on.n_bytes(codes, scales)), v)


def test_bytes_of_a_row():
    x = np.zeros((1, 128))
    x[0, :8] = [0.5, -0.5, 1, 6, -6, 3, 0, -0.0]
    x[0, 96] = math.inf
    b, s = on.n_bytes(*on.n_rows(x))
    assert b[0, :4].tolist() == [0x91, 0x72, 0x5f, 0x80] and (b[0, 4:] == 0).all()
    assert s[0].tolist() == [127, 27, 27, 255]
    assert np.isnan(on.n_unpack(b, s)[0, 96:]).all()


# ------------------------------------------------------------------------------------------------ refusals, C ABI
FAKE, ODD, WS = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1002), ctypes.c_void_p(0x10000)
needs_no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="invented pointers: only where no GPU is visible")


def cache(P=2, rows=100, d=128, K=FAKE, V=FAKE, Ks=FAKE, Vs=FAKE):
    return ctypes.byref(A.NCacheStruct(P, rows, d, K, V, Ks, Vs))


BAD_CACHES = [(dict(P=0), A.ERR_INVALID_ARG), (dict(rows=0), A.ERR_INVALID_ARG), (dict(d=64), A.ERR_UNSUPPORTED),
              (dict(rows=(1 << 26) + 1), A.ERR_UNSUPPORTED), (dict(P=(1 << 20) + 1), A.ERR_UNSUPPORTED),
              (dict(K=None), A.ERR_INVALID_ARG), (dict(V=None), A.ERR_INVALID_ARG), (dict(Ks=None), A.ERR_INVALID_ARG),
              (dict(Vs=None), A.ERR_INVALID_ARG), (dict(K=ODD), A.ERR_INVALID_ARG), (dict(Vs=ODD), A.ERR_INVALID_ARG),
              (dict(V=ctypes.c_void_p(0x1008)), A.ERR_INVALID_ARG), (dict(rows=-2 ** 31), A.ERR_INVALID_ARG)]


@needs_no_gpu
def test_write_refuses():
    f = A.lib().arckv_ncache_write
    for kw, want in BAD_CACHES:
        assert f(cache(**kw), 1, A.BF16, FAKE, FAKE, None, None, None) == want, kw
    assert f(None, 1, A.BF16, FAKE, FAKE, None, None, None) == A.ERR_INVALID_ARG
    for n, dtype, K, V, start, want in [
            (0, A.BF16, FAKE, FAKE, None, A.ERR_INVALID_ARG), (101, A.BF16, FAKE, FAKE, None, A.ERR_INVALID_ARG),
            (1, 2, FAKE, FAKE, None, A.ERR_UNSUPPORTED), (1, A.F32, None, FAKE, None, A.ERR_INVALID_ARG),
            (1, A.F32, FAKE, ODD, None, A.ERR_INVALID_ARG), (1, A.F32, FAKE, FAKE, ODD, A.ERR_INVALID_ARG),
            (2 ** 31 - 1, A.F32, FAKE, FAKE, None, A.ERR_INVALID_ARG)]:
        assert f(cache(), n, dtype, K, V, start, None, None) == want, (n, dtype)


@needs_no_gpu
def test_read_refuses():
    f = A.lib().arckv_ncache_read
    for kw, want in BAD_CACHES:
        assert f(cache(**kw), 0, 1, A.BF16, None, FAKE, FAKE, None) == want, kw
    for first, n, dtype, K, want in [
            (-1, 1, A.BF16, FAKE, A.ERR_INVALID_ARG), (0, 0, A.BF16, FAKE, A.ERR_INVALID_ARG),
            (1, 100, A.BF16, FAKE, A.ERR_INVALID_ARG), (2 ** 31 - 1, 1, A.BF16, FAKE, A.ERR_INVALID_ARG),
            (0, 1, 7, FAKE, A.ERR_UNSUPPORTED), (0, 1, A.F32, None, A.ERR_INVALID_ARG), (0, 1, A.F32, ODD, A.ERR_INVALID_ARG)]:
        assert f(cache(), first, n, dtype, None, K, FAKE, None) == want, (first, n, dtype)


@needs_no_gpu
def test_attend_refuses():
    f = A.lib().arckv_attend_ncache
    call = lambda c=None, G=4, F=0, scale=0.0, Q=FAKE, beta=None, length=None, Kf=None, Vf=None, lf=None, out=FAKE, ws=WS, \
        nbytes=1 << 40: f(c or cache(), G, F, scale, Q, beta, length, Kf, Vf, lf, out, ws, nbytes, None)
    for kw, want in BAD_CACHES:
        assert call(cache(**kw)) == want, kw
    for kw, want in [
            (dict(G=0), A.ERR_INVALID_ARG), (dict(G=17), A.ERR_UNSUPPORTED), (dict(F=-1), A.ERR_INVALID_ARG),
            (dict(F=(1 << 26) + 1, Kf=FAKE, Vf=FAKE), A.ERR_UNSUPPORTED), (dict(F=3), A.ERR_INVALID_ARG),
            (dict(F=3, Kf=FAKE), A.ERR_INVALID_ARG), (dict(F=3, Kf=FAKE, Vf=ODD), A.ERR_INVALID_ARG),
            (dict(Q=None), A.ERR_INVALID_ARG), (dict(Q=ODD), A.ERR_INVALID_ARG), (dict(out=None), A.ERR_INVALID_ARG),
            (dict(out=ODD), A.ERR_INVALID_ARG), (dict(scale=math.nan), A.ERR_INVALID_ARG),
            (dict(scale=math.inf), A.ERR_INVALID_ARG), (dict(beta=ODD), A.ERR_INVALID_ARG),
            (dict(length=ODD), A.ERR_INVALID_ARG), (dict(lf=ODD), A.ERR_INVALID_ARG)]:
        assert call(**kw) == want, kw
    big = cache(rows=100000)
    need = A.attend_ncache_workspace_size(2, 100000, 4)
    if need:
        assert call(big, nbytes=need - 1) == call(big, ws=None) == call(big, ws=ctypes.c_void_p(0x10010)) == A.ERR_WORKSPACE


def test_workspace_size():
    for args, want in [((0, 1, 1, 0), A.ERR_INVALID_ARG), ((1, 0, 1, 0), A.ERR_INVALID_ARG), ((1, 1, 0, 0), A.ERR_INVALID_ARG),
                       ((1, 1, 1, -1), A.ERR_INVALID_ARG), ((1, 1, 17, 0), A.ERR_UNSUPPORTED),
                       (((1 << 20) + 1, 1, 1, 0), A.ERR_UNSUPPORTED), ((1, (1 << 26) + 1, 1, 0), A.ERR_UNSUPPORTED)]:
        with pytest.raises(A.ArckvError) as e:
            A.attend_ncache_workspace_size(*args)
        assert e.value.status == want, args
    with pytest.raises(ValueError):
        A.attend_ncache_workspace_size(1 << 32, 1, 1)
    sizes = (1, 2, 63, 64, 65, 768, 769, 4096, 1 << 20, 1 << 26)
    most = max(A.attend_ncache_workspace_size(P, rows, 16, F) for P in sizes if P <= 1 << 20 for rows in sizes for F in sizes)
    assert most <= 128 << 20, most


# ------------------------------------------------------------------------------------------------ refusals, binding
@needs_no_gpu
def test_binding_refuses_host_tensors(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    c = A.ncache(2, 10, device="cpu")
    x = torch.zeros(2, 1, 128, dtype=torch.bfloat16)
    for f in (lambda: A.ncache_write(c, x, x), lambda: A.ncache_read(c), lambda: A.attend_ncache(x, c)):
        with pytest.raises(ValueError, match="GPU"):
            f()


def test_the_cache_has_the_documented_arrays():
    c = A.ncache(3, 70, device="cpu")
    assert [tuple(t.shape) for t in c] == [(3, 70, 64), (3, 70, 64), (3, 70, 4), (3, 70, 4)]
    assert all(t.dtype == torch.uint8 for t in c)


@needs_no_gpu
def test_host_code_under_sanitizers():
    """Refusals, workspace sizes and frequencies under AddressSanitizer and UndefinedBehaviorSanitizer (no GPU)."""
    from paper_2609_36835_amd import build as B
    from tests.test_host_sanitizers import HOST_SAN, OUT, PKG, ROOT, _kernel_objects
    objs = _kernel_objects()
    if not objs:
        pytest.skip("kernel objects not built (run paper_2609_36835_amd.build first)")
    os.makedirs(OUT, exist_ok=True)
    hipcc, inc = B._hipcc(), ["-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc")]
    host_o, drv_o, exe = (os.path.join(OUT, n) for n in ("arckv_host_nc.o", "ncache_checks.o", "ncache_checks"))
    for cmd in ([hipcc, "-std=c++17", "-fPIC", *HOST_SAN, *inc, "-c", os.path.join(PKG, "csrc", "arckv_host.cpp"), "-o", host_o],
                [hipcc, "-std=c++17", *HOST_SAN, *inc, "-c", os.path.join(ROOT, "tests", "sanitize", "ncache_checks.cpp"),
                 "-o", drv_o],
                [hipcc, f"--offload-arch={B.ARCH}", *HOST_SAN, drv_o, host_o, *objs, "-o", exe]):
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, (" ".join(cmd), r.stderr[-4000:])
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1", HIP_VISIBLE_DEVICES="")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0 and "ok: 0 failures" in r.stdout, (r.stdout[-4000:], r.stderr[-4000:])


def test_chunks_by_the_kernel_that_runs():
    """A pair that eight waves take whole in less time than several chunks of four waves is one chunk, which needs no workspace;
    long pairs that leave CUs without work, or many, are cut."""
    from paper_2609_36835_amd import arckv
    size = arckv.attend_ncache_workspace_size
    for P, R in ((256, 9000), (224, 46849), (200, 6621), (200, 20254), (192, 4353), (160, 2500), (256, 4000), (64, 1500), (8, 819)):
        assert size(P, R, 4) == size(P, R, 16) == 0, (P, R)
    for P, R in ((1, 131072), (8, 131072), (8, 4000), (64, 2500), (96, 10069), (128, 10069), (160, 46849), (192, 20254), (256, 20254)):
        assert size(P, R, 4) > 0, (P, R)
