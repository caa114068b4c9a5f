"""Rotary positions without a GPU: frequencies against their formulas, and argument checks of the C entry points and of
the binding (every refusal comes before any HIP call)."""
import ctypes
import math

import numpy as np
import pytest
import torch

import synth
from oracle import rotary as orot
from paper_2609_36835_amd import arckv as A

FAKE, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008)
needs_no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="invented pointers: only where no GPU is visible")


# ------------------------------------------------------------------------------------------------ frequencies
@pytest.mark.parametrize("d_rot", [2, 4, 34, 64, 126, 128])
@pytest.mark.parametrize("mode", A.STRETCHES)
def test_frequencies(d_rot, mode):
    """Each is formed by a handful of float64 operations (pow within an ulp or two): 2^-48 relative."""
    if mode == "base" and d_rot == 2:
        return
    for base, stretch, length, few, many in [(10000.0, 4.0, 4096.0, 1.0, 32.0), (500000.0, 8.0, 8192.0, 1.0, 4.0),
                                             (10000.0, 1.0, 100.0, 0.5, 1e6), (1.5, 3.0, 50.0, 2.0, 2.5)]:
        got = A.rotary_frequencies(d_rot, base, mode, stretch, length, few, many, device="cpu")
        want = orot.frequencies(d_rot, base, mode, stretch, length, few, many)
        assert got.dtype == torch.float64 and got.shape == (d_rot // 2,)
        np.testing.assert_allclose(got.numpy(), want, rtol=2.0 ** -48)


def test_turns_are_the_bands_of_the_synthetic_inputs():
    """synth's scaled frequencies (8 times 8192 positions, between one turn and four) are the turns' ramp, and its way of
    turning is that of halves."""
    got = A.rotary_frequencies(128, synth.ROPE_THETA, "turns", 8.0, 8192.0, 1.0, 4.0, device="cpu").numpy()
    np.testing.assert_allclose(got, synth.llama3_inv_freq(), rtol=2.0 ** -46)
    x = np.random.default_rng(0).standard_normal((9, 128))
    at = np.array([0, 1, 5, 100, 1000, 8191, 30000, 65535, 131071])
    np.testing.assert_allclose(orot.rotary(x[:, None], at, got)[:, 0], synth.apply_rope(x, at), atol=1e-6)


def test_ramps_end_where_they_should():
    f = A.rotary_frequencies(128, 10000.0, device="cpu")
    for mode in ("turns", "index"):
        g = A.rotary_frequencies(128, 10000.0, mode, 16.0, 4096.0, 1.0, 32.0, device="cpu")
        assert torch.equal(g[:8], f[:8]) and torch.allclose(g[-8:], f[-8:] / 16, rtol=1e-15)
        assert (g[1:] <= g[:-1]).all()


def test_frequencies_refuse():
    for args, want in [
            ((0, 1e4, "none"), A.ERR_INVALID_ARG), ((3, 1e4, "none"), A.ERR_INVALID_ARG), ((130, 1e4, "none"), A.ERR_INVALID_ARG),
            ((64, 1.0, "none"), A.ERR_INVALID_ARG), ((64, math.inf, "none"), A.ERR_INVALID_ARG),
            ((64, math.nan, "none"), A.ERR_INVALID_ARG), ((64, 1e4, "linear", 0.5), A.ERR_INVALID_ARG),
            ((64, 1e4, "linear", math.inf), A.ERR_INVALID_ARG), ((2, 1e4, "base", 2.0), A.ERR_INVALID_ARG),
            ((4, 1e300, "base", 1e10), A.ERR_INVALID_ARG), ((64, 1e4, "turns", 2.0, 0.0), A.ERR_INVALID_ARG),
            ((64, 1e4, "turns", 2.0, math.nan), A.ERR_INVALID_ARG), ((64, 1e4, "index", 2.0, 10.0, 0.0, 1.0), A.ERR_INVALID_ARG),
            ((64, 1e4, "index", 2.0, 10.0, 2.0, 2.0), A.ERR_INVALID_ARG)]:
        with pytest.raises(A.ArckvError) as e:
            A.rotary_frequencies(*args, device="cpu")
        assert e.value.status == want, args
    with pytest.raises(ValueError):
        A.rotary_frequencies(64, mode="other", device="cpu")
    f = A.lib().arckv_rotary_frequencies
    assert f(64, 1e4, 0, 1.0, 0.0, 0.0, 0.0, None) == A.ERR_INVALID_ARG
    buf = (ctypes.c_double * 64)()
    assert f(64, 1e4, 5, 1.0, 0.0, 0.0, 0.0, buf) == f(64, 1e4, -1, 1.0, 0.0, 0.0, 0.0, buf) == A.ERR_UNSUPPORTED


# ------------------------------------------------------------------------------------------------ refusals
def params(N=5, d=128, d_rot=128, layout=0, dtype=A.BF16, transpose=0, factor=1.0):
    return ctypes.byref(A.RotaryParams(N, d, d_rot, layout, dtype, transpose, factor))


def rows(heads=3, x=FAKE, xt=384, xh=128, y=ctypes.c_void_p(0x9000), yt=384, yh=128):
    return ctypes.byref(A.RotaryRows(heads, x, xt, xh, y, yt, yh))


@needs_no_gpu
def test_rotary_refuses():
    f = A.lib().arckv_rotary
    for kw, want in [
            (dict(N=0), A.ERR_INVALID_ARG), (dict(N=-1), A.ERR_INVALID_ARG), (dict(N=(1 << 26) + 1), A.ERR_UNSUPPORTED),
            (dict(d=64), A.ERR_UNSUPPORTED), (dict(d_rot=0), A.ERR_INVALID_ARG), (dict(d_rot=3), A.ERR_INVALID_ARG),
            (dict(d_rot=130), A.ERR_INVALID_ARG), (dict(layout=2), A.ERR_UNSUPPORTED), (dict(layout=-1), A.ERR_UNSUPPORTED),
            (dict(dtype=2), A.ERR_UNSUPPORTED), (dict(transpose=2), A.ERR_INVALID_ARG),
            (dict(factor=math.nan), A.ERR_INVALID_ARG), (dict(factor=math.inf), A.ERR_INVALID_ARG)]:
        assert f(params(**kw), None, FAKE, rows(), None, None) == want, kw
    assert f(None, None, FAKE, rows(), None, None) == A.ERR_INVALID_ARG
    assert f(params(), None, FAKE, None, rows(), None) == A.ERR_INVALID_ARG
    assert f(params(), None, None, rows(), None, None) == A.ERR_INVALID_ARG
    assert f(params(), ctypes.c_void_p(0x1002), FAKE, rows(), None, None) == A.ERR_INVALID_ARG
    assert f(params(), None, ctypes.c_void_p(0x1004), rows(), None, None) == A.ERR_INVALID_ARG
    bad = [(dict(heads=0), A.ERR_INVALID_ARG), (dict(heads=(1 << 20) + 1, yh=128, yt=1 << 28), A.ERR_UNSUPPORTED),
           (dict(x=None), A.ERR_INVALID_ARG), (dict(y=None), A.ERR_INVALID_ARG), (dict(x=ODD), A.ERR_INVALID_ARG),
           (dict(y=ODD), A.ERR_INVALID_ARG), (dict(xt=-128), A.ERR_INVALID_ARG), (dict(xt=4), A.ERR_INVALID_ARG),
           (dict(yh=132), A.ERR_INVALID_ARG), (dict(xh=(1 << 34) + 8), A.ERR_UNSUPPORTED),
           (dict(yh=0), A.ERR_INVALID_ARG), (dict(yt=0), A.ERR_INVALID_ARG), (dict(yt=120), A.ERR_INVALID_ARG),
           (dict(yt=256), A.ERR_INVALID_ARG),                    # the next token begins inside this one's heads
           (dict(yt=128, yh=632), A.ERR_INVALID_ARG),            # the next head inside this one's tokens
           (dict(x=FAKE, y=FAKE, xt=384, yt=768), A.ERR_INVALID_ARG)]
    for kw, want in bad:
        assert f(params(), None, FAKE, rows(**kw), None, None) == want, kw
        assert f(params(), None, FAKE, rows(), rows(**kw), None) == want, kw
    many = dict(heads=1 << 10, xt=1 << 18, yt=1 << 18)
    assert f(params(N=(1 << 20) + 1), None, FAKE, rows(**many), None, None) == A.ERR_UNSUPPORTED
    assert f(params(N=1 << 20), None, FAKE, rows(**many), rows(), None) == A.ERR_UNSUPPORTED


@needs_no_gpu
def test_binding_refuses(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    x, freq = torch.zeros(3, 2, 128), torch.zeros(64, dtype=torch.float64)
    with pytest.raises(ValueError, match="GPU"):
        A.rotary(x, freq)
    with pytest.raises(TypeError):
        A.rotary(x.half(), freq)
    with pytest.raises(TypeError, match="output"):
        A.rotary(x, freq, out=x.bfloat16())
    with pytest.raises(ValueError, match="shape"):
        A.rotary(x[:, :, :64], freq)
    with pytest.raises(ValueError, match="shape"):
        A.rotary(x, freq, out=x[:2])
    with pytest.raises(ValueError):
        A.rotary(x[:, 0], freq)
