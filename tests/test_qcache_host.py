"""The 8-bit cache without a GPU: its oracle against independent definitions, argument checks of the C entry points
(every refusal comes before any HIP call) and of the binding."""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import qcache as oq
from paper_2609_36835_amd import arckv as A


# ------------------------------------------------------------------------------------------------ the oracle's pins
def test_e4m3_rounding_is_the_types():
    """Every border between two codes, the values next to it and random values, against torch's conversion."""
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    mid = (codes[1:] + codes[:-1]) / 2
    g = np.random.default_rng(0)
    y = np.concatenate([codes, mid, np.nextafter(mid, 0), np.nextafter(mid, 1e9), g.uniform(0, 448, 5000),
                        np.exp(g.uniform(-12, 6, 5000))]).astype(np.float32).astype(np.float64)
    y = np.concatenate([y, -y])
    want = torch.from_numpy(y).float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oq.q_round(y, "e4m3"), want)


def test_int8_rounding_ties_to_even():
    y = np.array([0.5, 1.5, 2.5, -0.5, -1.5, 126.5, 0.49999, 63.5])
    assert oq.q_round(y, "int8").tolist() == [0, 2, 2, 0, -2, 126, 0, 64]


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_scale_is_the_smallest_power_of_two(fmt):
    M = oq.LARGEST[fmt]
    for a in (M, np.nextafter(M, 1e9), M / 2, M * 3, 1e-3, 1e30, 1.0, 0.9):
        s = oq.q_scale(float(a), fmt)
        assert math.frexp(s)[0] == 0.5 and a <= M * s and a > M * s / 2
    assert oq.q_scale(0.0, fmt) == oq.q_scale(1e-38, fmt) == 2.0 ** -100
    assert math.isnan(oq.q_scale(math.inf, fmt)) and math.isnan(oq.q_scale(math.nan, fmt))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_stored_values_are_within_half_a_step_and_stay(fmt):
    g = np.random.default_rng(1)
    x = g.standard_normal((200, 16)) * np.exp(g.uniform(-3, 3, (1, 16)))
    codes, scales = np.zeros((200, 16)), np.full(4, 2.0 ** -100)
    oq.q_write(codes, scales, x, 0, fmt)
    v = oq.q_values(codes, scales)
    s = np.repeat(scales, 64)[:200, None]
    half = s / 2 if fmt == "int8" else np.maximum(np.abs(x) * 2.0 ** -4, s * 2.0 ** -10)
    assert (np.abs(v - x) <= half).all()
    c2, s2 = np.zeros((200, 16)), np.full(4, 2.0 ** -100)
    oq.q_write(c2, s2, v, 0, fmt)
    assert np.array_equal(oq.q_values(c2, s2), v)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_block_scores_bound_every_logit(fmt):
    g = np.random.default_rng(2)
    x, Q = g.standard_normal((150, 128)), g.standard_normal((3, 128))
    beta = g.uniform(-3, 3, 150)
    codes, scales, bounds = np.zeros((150, 128)), np.zeros(3), np.zeros((3, 2, 128))
    oq.q_write(codes, scales, x, 0, fmt, bounds)
    K = oq.q_values(codes, scales)
    sc = oq.q_block_scores(Q, bounds, scales, 150, 0.1, beta)
    for b in range(3):
        rows = slice(64 * b, min(64 * b + 64, 150))
        assert (0.1 * Q @ K[rows].T + beta[rows]).max() <= sc[b] + 1e-12
    assert oq.q_block_scores(Q, bounds, scales, 64, 0.1)[1:].tolist() == [-math.inf, -math.inf]


def test_attend_matches_a_plain_softmax_and_drops_masked_rows():
    g = np.random.default_rng(3)
    Q, K, V = g.standard_normal((2, 8)), g.standard_normal((5, 8)), g.standard_normal((5, 8))
    beta = np.array([0.0, -math.inf, 1.0, -math.inf, -2.0])
    V[1] = math.nan
    w = np.exp(Q @ K.T + beta)[:, [0, 2, 4]]
    want = (w / w.sum(1, keepdims=True)) @ V[[0, 2, 4]]
    assert np.allclose(oq.q_attend(Q, K, V, beta, None, None, 1.0)[0], want, rtol=1e-12)
    assert (oq.q_attend(Q, K, V, np.full(5, -math.inf), None, None, 1.0)[0] == 0).all()


# ------------------------------------------------------------------------------------------------ refusals, C ABI
FAKE, ODD, WS = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1002), ctypes.c_void_p(0x10000)
needs_no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="invented pointers: only where no GPU is visible")


def cache(P=2, rows=100, d=128, fmt=A.E4M3, K=FAKE, V=FAKE, Ks=FAKE, Vs=FAKE, bounds=FAKE):
    return ctypes.byref(A.QCacheStruct(P, rows, d, fmt, K, V, Ks, Vs, bounds))


BAD_CACHES = [(dict(P=0), A.ERR_INVALID_ARG), (dict(rows=0), A.ERR_INVALID_ARG), (dict(d=64), A.ERR_UNSUPPORTED),
              (dict(fmt=2), A.ERR_UNSUPPORTED), (dict(rows=(1 << 26) + 1), A.ERR_UNSUPPORTED),
              (dict(P=(1 << 20) + 1), A.ERR_UNSUPPORTED), (dict(Ks=None), A.ERR_INVALID_ARG),
              (dict(bounds=ODD), A.ERR_INVALID_ARG), (dict(K=ODD), A.ERR_INVALID_ARG)]


@needs_no_gpu
def test_write_refuses():
    f = A.lib().arckv_qcache_write
    for kw, want in BAD_CACHES + [(dict(V=None), A.ERR_INVALID_ARG), (dict(Vs=None), A.ERR_INVALID_ARG)]:
        assert f(cache(**kw), 1, A.BF16, FAKE, FAKE, None, None, None) == want, kw
    assert f(None, 1, A.BF16, FAKE, FAKE, None, None, None) == A.ERR_INVALID_ARG
    for n, dtype, K, V, start, want in [
            (0, A.BF16, FAKE, FAKE, None, A.ERR_INVALID_ARG), (101, A.BF16, FAKE, FAKE, None, A.ERR_INVALID_ARG),
            (1, 2, FAKE, FAKE, None, A.ERR_UNSUPPORTED), (1, A.F32, None, FAKE, None, A.ERR_INVALID_ARG),
            (1, A.F32, FAKE, ODD, None, A.ERR_INVALID_ARG), (1, A.F32, FAKE, FAKE, ODD, A.ERR_INVALID_ARG)]:
        assert f(cache(), n, dtype, K, V, start, None, None) == want, (n, dtype)


@needs_no_gpu
def test_read_refuses():
    f = A.lib().arckv_qcache_read
    for kw, want in BAD_CACHES:
        assert f(cache(**kw), 0, 1, A.BF16, None, FAKE, FAKE, None) == want, kw
    for first, n, dtype, K, want in [
            (-1, 1, A.BF16, FAKE, A.ERR_INVALID_ARG), (0, 0, A.BF16, FAKE, A.ERR_INVALID_ARG),
            (1, 100, A.BF16, FAKE, A.ERR_INVALID_ARG), (2 ** 31 - 1, 1, A.BF16, FAKE, A.ERR_INVALID_ARG),
            (0, 1, 5, FAKE, A.ERR_UNSUPPORTED), (0, 1, A.F32, ODD, A.ERR_INVALID_ARG)]:
        assert f(cache(), first, n, dtype, None, K, FAKE, None) == want, (first, n)


@needs_no_gpu
def test_select_blocks_refuses():
    f = A.lib().arckv_select_blocks
    for kw, want in BAD_CACHES + [(dict(bounds=None), A.ERR_INVALID_ARG)]:
        assert f(cache(**kw), 4, 0.0, FAKE, None, None, 1, FAKE, FAKE, None) == want, kw
    for G, scale, Q, k, scores, want in [
            (0, 0.0, FAKE, 1, FAKE, A.ERR_INVALID_ARG), (17, 0.0, FAKE, 1, FAKE, A.ERR_UNSUPPORTED),
            (4, math.nan, FAKE, 1, FAKE, A.ERR_INVALID_ARG), (4, 0.0, None, 1, FAKE, A.ERR_INVALID_ARG),
            (4, 0.0, ODD, 1, FAKE, A.ERR_INVALID_ARG), (4, 0.0, FAKE, 0, FAKE, A.ERR_INVALID_ARG),
            (4, 0.0, FAKE, 3, FAKE, A.ERR_INVALID_ARG), (4, 0.0, FAKE, 1, None, A.ERR_INVALID_ARG)]:
        assert f(cache(), G, scale, Q, None, None, k, scores, FAKE, None) == want, (G, k)


@needs_no_gpu
def test_attend_qcache_refuses():
    f, big = A.lib().arckv_attend_qcache, 1 << 30

    def call(c=None, G=4, nsel=0, F=0, scale=0.0, Q=FAKE, beta=None, blocks=None, K_f=None, out=FAKE, ws=WS, n=big):
        return f(c or cache(), G, nsel, F, scale, Q, beta, None, blocks, K_f, K_f, None, out, ws, n, None)
    for kw, want in BAD_CACHES:
        assert call(cache(**kw)) == want, kw
    for kw, want in [(dict(G=0), A.ERR_INVALID_ARG), (dict(G=17), A.ERR_UNSUPPORTED), (dict(F=-1), A.ERR_INVALID_ARG),
                     (dict(nsel=-1), A.ERR_INVALID_ARG), (dict(nsel=2), A.ERR_INVALID_ARG),
                     (dict(blocks=FAKE), A.ERR_INVALID_ARG), (dict(F=2), A.ERR_INVALID_ARG),
                     (dict(F=2, K_f=ODD), A.ERR_INVALID_ARG), (dict(scale=math.inf), A.ERR_INVALID_ARG),
                     (dict(Q=ODD), A.ERR_INVALID_ARG), (dict(out=None), A.ERR_INVALID_ARG),
                     (dict(beta=ODD), A.ERR_INVALID_ARG), (dict(c=cache(rows=2000), ws=None), A.ERR_WORKSPACE),
                     (dict(c=cache(rows=2000), ws=ODD), A.ERR_WORKSPACE),
                     (dict(c=cache(rows=100000), n=1000), A.ERR_WORKSPACE)]:
        assert call(**kw) == want, kw


def test_attend_qcache_workspace_size():
    size = A.attend_qcache_workspace_size
    assert size(512, 16384, 4) > size(8, 16384, 4, nsel=64) > 0
    assert size(1, 64, 4) == 0                                         # one workgroup's work
    assert size(1 << 20, 1 << 26, 16) == 0 < size(100, 1 << 26, 16) < 1 << 26   # however large the cache
    for args, want in [((0, 1, 1), A.ERR_INVALID_ARG), ((1, 0, 1), A.ERR_INVALID_ARG), ((1, 1, 0), A.ERR_INVALID_ARG),
                       ((1, 1, 17), A.ERR_UNSUPPORTED), ((1, 1, 1, -1), A.ERR_INVALID_ARG),
                       ((1, 1, 1, 0, -1), A.ERR_INVALID_ARG), ((1, 1, 1, (1 << 20) + 1), A.ERR_UNSUPPORTED)]:
        with pytest.raises(A.ArckvError) as e:
            size(*args)
        assert e.value.status == want, args


# ------------------------------------------------------------------------------------------------ refusals, binding
def test_binding_checks_shapes_types_and_devices():
    x = torch.zeros(2, 3, 128)
    assert A._qptr(None, (1,), torch.float32, 0, "x") is None
    with pytest.raises(TypeError):
        A._qptr(x, x.shape, torch.bfloat16, 0, "x")
    with pytest.raises(ValueError, match="shape"):
        A._qptr(x, (2, 3, 64), torch.float32, 0, "x")
    with pytest.raises(ValueError, match="current GPU"):
        A._qptr(x, x.shape, torch.float32, 0, "x")                     # a CPU tensor
    with pytest.raises(ValueError, match="contiguous"):
        A._qptr(x[:, :, ::2], (2, 3, 64), torch.float32, -1, "x")
    for dtype in (torch.uint8, torch.float8_e5m2, torch.bfloat16):
        with pytest.raises(TypeError):
            A.qcache(1, 64, dtype, device="cpu")
    c = A.qcache(3, 130, torch.int8, device="cpu")
    assert [tuple(t.shape) for t in c] == [(3, 130, 128), (3, 130, 128), (3, 3), (3, 3), (3, 3, 2, 128)]
    assert A.qcache(1, 1, device="cpu", bounds=False).K_bounds is None


def test_host_code_under_sanitizers():
    """The entry points' argument checks and workspace arithmetic with AddressSanitizer and UndefinedBehaviorSanitizer on
    the host code alone (built as tests/test_host_sanitizers.py builds the rest)."""
    from paper_2609_36835_amd import build as B
    from tests.test_host_sanitizers import HOST_SAN, OUT, PKG, ROOT, _kernel_objects
    objs = _kernel_objects()
    if not objs:
        pytest.skip("kernel objects not built (run paper_2609_36835_amd.build first)")
    os.makedirs(OUT, exist_ok=True)
    hipcc, inc = B._hipcc(), ["-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc")]
    host_o, drv_o, exe = (os.path.join(OUT, n) for n in ("arckv_host_q.o", "qcache_checks.o", "qcache_checks"))
    for cmd in ([hipcc, "-std=c++17", "-fPIC", *HOST_SAN, *inc, "-c", os.path.join(PKG, "csrc", "arckv_host.cpp"), "-o", host_o],
                [hipcc, "-std=c++17", *HOST_SAN, *inc, "-c", os.path.join(ROOT, "tests", "sanitize", "qcache_checks.cpp"),
                 "-o", drv_o],
                [hipcc, f"--offload-arch={B.ARCH}", *HOST_SAN, drv_o, host_o, *objs, "-o", exe]):
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, (" ".join(cmd), r.stderr[-4000:])
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1", HIP_VISIBLE_DEVICES="")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0 and "ok: 0 failures" in r.stdout, (r.stdout[-4000:], r.stderr[-4000:])


@pytest.mark.parametrize("R", [130, 20000])
def test_exact_sums_show_any_row(R):
    """The inputs of the GPU test of attention's sums: a row left out, doubled or taken for its neighbour in the oracle
    moves a result by more than that test allows, wherever the row lies."""
    from tests.test_gpu_qcache_sums import exact_sums
    g = np.random.default_rng(R)
    K, V = (torch.from_numpy(g.integers(0, 2, (1, R, 128)).astype(np.float32)) for _ in range(2))
    Q = torch.zeros(1, 2, 128)
    Q[0, 1, 17] = 4096.0
    ones = torch.ones(1, R)
    want = exact_sums(Q, -K, V, ones, None, None, None, None)
    for row in [0, 1, 63, 64, 65, R // 2, R - 3, R - 2]:
        for change in ("left out", "twice", "its neighbour's value", "its neighbour's key"):
            w, k, v = ones.clone(), -K.clone(), V.clone()
            if change == "left out":
                w[0, row] = 0
            elif change == "twice":
                w[0, row] = 2
            elif change == "its neighbour's value":
                v[0, row] = V[0, row + 1]
            else:
                k[0, row] = -K[0, row + 1]
            got = exact_sums(Q, k, v, w, None, None, None, None)
            seen = bool(((got - want).abs() > 2.0 ** -22 * want).any())
            assert seen or (change == "its neighbour's key" and K[0, row, 17] == K[0, row + 1, 17]), (row, change)


def step_by_step(fmt, growth):
    """64 rows, each `growth` times the one before, written one at a time: rows, stored values, and for each row the
    largest scale since it was written."""
    g = np.random.default_rng(4)
    x = g.standard_normal((64, 16)) * np.exp(math.log(growth) * np.arange(64))[:, None]
    codes, scales, largest = np.zeros((64, 16)), np.full(1, 2.0 ** -100), np.zeros((64, 1))
    for i in range(64):
        oq.q_write(codes, scales, x[i:i + 1], i, fmt)
        largest[:i + 1] = np.maximum(largest[:i + 1], scales[0])
    return x, oq.q_values(codes, scales), largest


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("growth", [1.0, 1.02, 1.1, 1.4])
def test_rows_kept_in_a_growing_block_stay_within_a_step(fmt, growth):
    """Each doubling of the scale can add half a step of the new one: s / 2 + s / 4 + ... < s in all.  In e4m3 only values
    below 2^-6 scale are rounded again, in steps of 2^-9 scale."""
    x, v, s = step_by_step(fmt, growth)
    err = np.abs(v - x)
    if fmt == "int8":
        assert (err < s).all()
    else:
        large = np.abs(x) >= 2.0 ** -6 * s
        assert (err[large] <= 2.0 ** -4 * np.abs(x[large])).all() and (err < 2.0 ** -9 * s)[~large].all()


@pytest.mark.parametrize("fmt,growth", [("int8", 1.02), ("e4m3", 1.1)])
def test_rows_kept_in_a_growing_block_pass_half_a_step(fmt, growth):
    x, v, s = step_by_step(fmt, growth)
    half = s / 2 if fmt == "int8" else np.maximum(np.abs(x) * 2.0 ** -4, s * 2.0 ** -10)
    assert (np.abs(v - x) > half).any()


def test_binding_refuses_what_32_bits_do_not_hold():
    """A C argument of 32 bits takes a larger number modulo 2^32: row 2^32 would be row 0."""
    c = A.qcache(2, 100, device="cpu")
    Q = torch.zeros(2, 4, 128, dtype=torch.bfloat16)
    for big in (1 << 31, 1 << 32, (1 << 32) + 1, -(1 << 31) - 1):
        with pytest.raises(ValueError, match="first"):
            A.qcache_read(c, big, 4)
        with pytest.raises(ValueError, match="n:"):
            A.qcache_read(c, 0, big)
        with pytest.raises(ValueError, match="k:"):
            A.select_blocks(Q, c, big)
        for i in range(5):
            args = [2, 100, 4, 0, 0]
            args[i] = big
            with pytest.raises(ValueError, match="32 bits"):
                A.attend_qcache_workspace_size(*args)


@needs_no_gpu
def test_no_workspace_under_sanitizers():
    """A call that needs no workspace forms no address from the null pointer in its place."""
    from paper_2609_36835_amd import build as B
    from tests.test_host_sanitizers import HOST_SAN, OUT, PKG, ROOT, _kernel_objects
    objs = _kernel_objects()
    if not objs:
        pytest.skip("kernel objects not built (run paper_2609_36835_amd.build first)")
    os.makedirs(OUT, exist_ok=True)
    hipcc, inc = B._hipcc(), ["-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc")]
    host_o, drv_o, exe = (os.path.join(OUT, n) for n in ("arckv_host_n.o", "qcache_no_workspace.o", "qcache_no_workspace"))
    for cmd in ([hipcc, "-std=c++17", "-fPIC", *HOST_SAN, *inc, "-c", os.path.join(PKG, "csrc", "arckv_host.cpp"), "-o", host_o],
                [hipcc, "-std=c++17", *HOST_SAN, *inc, "-c",
                 os.path.join(ROOT, "tests", "sanitize", "qcache_no_workspace.cpp"), "-o", drv_o],
                [hipcc, f"--offload-arch={B.ARCH}", *HOST_SAN, drv_o, host_o, *objs, "-o", exe]):
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, (" ".join(cmd), r.stderr[-4000:])
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0 and "ok: size 0, 0 bytes" in r.stdout, (r.stdout[-4000:], r.stderr[-4000:])
