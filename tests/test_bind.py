"""The binding's native short way: it leaves everything that is not as documented to the long way, whose errors say what is
wrong, and where it takes a call it does what the long way does."""
import concurrent.futures
import ctypes
import math
import os

import pytest
import torch

from paper_2609_36835_amd import arckv as A
from paper_2609_36835_amd import build as B

NAMES = ("ncache_write", "ncache_read", "attend_ncache", "rotary")


class LongWay:
    """Stands in for the native module and takes nothing."""

    def __getattr__(self, name):
        return lambda *a: None


class Counted:
    def __init__(self, m):
        self.m, self.taken, self.left = m, 0, 0

    def __getattr__(self, name):
        def call(*a):
            r = getattr(self.m, name)(*a)
            self.taken, self.left = self.taken + (r is not None), self.left + (r is None)
            return r
        return call


def test_host_tensors_and_other_objects_are_left_to_the_long_way():
    m = A._bind()
    c = A.ncache(2, 10, device="cpu")
    x, i = torch.zeros(2, 3, 128, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    f = torch.zeros(64, dtype=torch.float64)
    assert m.ncache_write(0, c, x, x, i, i) is None
    assert m.ncache_read(0, c, 0, 3, False, i) is None
    assert m.attend_ncache(0, x, c, None, i, None, None, None, None, None, None) is None
    assert m.rotary(0, x, f, None, None, False, False, 1.0, x, None) is None
    for junk in (None, 1, "x", (), (1, 2, 3, 4), [], object(), 1.5):
        assert m.ncache_write(0, junk, junk, junk, junk, junk) is None
        assert m.ncache_read(0, junk, junk, junk, junk, junk) is None
        assert m.attend_ncache(0, *[junk] * 10) is None
        assert m.rotary(0, *[junk] * 9) is None
    for name in NAMES:
        assert getattr(m, name)() is None and getattr(m, name)(0) is None


def both_ways(monkeypatch, call):
    """The call's results by the short way, which has to take it, and by the long one."""
    short = Counted(A._bind())
    monkeypatch.setattr(A, "_BIND", short)
    a = call()
    assert (short.taken, short.left) == (1, 0)
    monkeypatch.setattr(A, "_BIND", LongWay())
    b = call()
    monkeypatch.undo()
    return a, b


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_both_ways_write_and_read_the_same(monkeypatch, dtype):
    K, V = torch.randn(3, 20, 128, device="cuda").to(dtype), torch.randn(3, 20, 128, device="cuda").to(dtype)
    start, count = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([0, 5, 90], [20, 3, 20]))
    for args in ((), (start,), (None, count), (start, count)):
        caches = []

        def call():
            c = A.ncache(3, 100)
            for t in c:
                t.zero_()
            A.ncache_write(c, K, V, *args)
            caches.append(c)
        both_ways(monkeypatch, call)
        assert all(torch.equal(a, b) for a, b in zip(*caches))
    for args in ((), (7,), (90, 10), (0, 100, dtype), (3, None, dtype, count)):
        (k, v), (k2, v2) = both_ways(monkeypatch, lambda: A.ncache_read(caches[0], *args))
        assert k.dtype == k2.dtype and k.is_contiguous() and v.is_contiguous() and torch.equal(k, k2) and torch.equal(v, v2)
        assert k.untyped_storage().data_ptr() != caches[0].K.data_ptr()


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [100, 20000])
def test_both_ways_attend_the_same(monkeypatch, rows):
    P, G, F = 3, 4, 9
    c = A.ncache(P, rows)
    K = torch.randn(P, rows, 128, device="cuda")
    A.ncache_write(c, K, K)
    Q, Kf = torch.randn(P, G, 128, device="cuda").bfloat16(), torch.randn(P, F, 128, device="cuda").bfloat16()
    beta, n = torch.randn(P, rows, device="cuda"), torch.tensor([1, 50, rows], dtype=torch.int32, device="cuda")
    nf = torch.tensor([0, 9, 4], dtype=torch.int32, device="cuda")
    out = torch.empty(P, G, 128, device="cuda")
    ws = torch.empty(max(256, A.attend_ncache_workspace_size(P, rows, G, F)), dtype=torch.uint8, device="cuda")
    for kw in (dict(), dict(beta=beta), dict(length=n, K_f=Kf, V_f=Kf, length_f=nf), dict(scale=0.25), dict(out=out), dict(ws=ws),
               dict(beta=beta, length=n, K_f=Kf, V_f=Kf, length_f=nf, scale=0.1, out=out, ws=ws)):
        def call():
            r = A.attend_ncache(Q, c, **kw)
            assert (r is out) == ("out" in kw)
            return r.clone()
        a, b = both_ways(monkeypatch, call)
        assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_both_ways_turn_the_same(monkeypatch, dtype):
    qkv = torch.randn(11, 7, 128, device="cuda").to(dtype)
    pos = torch.arange(11, dtype=torch.int32, device="cuda") * 1000
    for d_rot in (128, 34):
        freq = A.rotary_frequencies(d_rot)
        ko = torch.empty(2, 11, 128, dtype=dtype, device="cuda").transpose(0, 1)
        for kw in (dict(), dict(positions=pos), dict(other=qkv[:, 4:6]), dict(positions=pos, other=qkv[:, 4:6], out_other=ko, factor=1.5),
                   dict(interleaved=True, transpose=True)):
            a, b = both_ways(monkeypatch, lambda: A.rotary(qkv[:, :4], freq, **kw))
            for x, y in zip(a, b) if isinstance(a, tuple) else ((a, b),):
                assert torch.equal(x, y)
        a, b = both_ways(monkeypatch, lambda: A.rotary(qkv[:1, :1], freq, pos[:1]))
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_what_the_short_way_leaves_works_or_says_why():
    c = A.ncache(2, 50)
    x = torch.randn(2, 3, 128, device="cuda").bfloat16()
    for t in c:
        t.zero_()
    A.ncache_write(list(c), x, x)                                  # a list of the arrays
    k, _ = A.ncache_read(list(c), 0, 3)
    assert torch.equal(k, A.ncache_read(c, 0, 3)[0])
    assert torch.equal(A.attend_ncache(x, c, scale=1), A.attend_ncache(x, c, scale=1.0))   # a whole number
    f = A.rotary_frequencies(64)
    assert torch.equal(A.rotary(x, f, factor=2), A.rotary(x, f, factor=2.0))
    with pytest.raises(A.ArckvError):
        A.ncache_write(c, *[torch.zeros(2, 51, 128, device="cuda")] * 2)
    with pytest.raises(A.ArckvError):
        A.ncache_read(c, 50, 1)
    with pytest.raises(A.ArckvError):
        A.attend_ncache(x, c, scale=math.nan)
    with pytest.raises(A.ArckvError):
        A.attend_ncache(torch.zeros(2, 17, 128, dtype=torch.bfloat16, device="cuda"), c)
    with pytest.raises(A.ArckvError):
        A.rotary(x, f, factor=math.inf)
    with pytest.raises(TypeError):
        A.rotary(x, f, torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        A.rotary(x.transpose(1, 2).contiguous().transpose(1, 2), f)


def test_an_output_without_its_rows_is_refused():
    """rotary's out_other is where `other` goes: without rows to turn nothing would be written there."""
    x, f = torch.zeros(2, 3, 128), torch.zeros(64, dtype=torch.float64)
    with pytest.raises(ValueError, match="out_other"):
        A.rotary(x, f, out_other=torch.empty(2, 1, 128))


def test_the_library_is_built_without_a_host_compiler(monkeypatch, tmp_path, capfd):
    """hipcc alone makes the library; a native part that an earlier build left does not stay beside it."""
    stale = tmp_path / "_arckv_bind.so"
    stale.write_bytes(b"stale")
    monkeypatch.setenv("CXX", str(tmp_path / "no-compiler"))
    monkeypatch.setattr(B, "BIND", str(stale))
    monkeypatch.setattr(B, "LIB", str(tmp_path / "libarckv.so"))
    monkeypatch.setattr(B, "BUILD_DIR", str(tmp_path / "objects"))
    monkeypatch.setattr(B, "sources", lambda: [os.path.join(B.CSRC, "util.hip")])
    assert B.build() == B.LIB and os.path.exists(B.LIB)
    assert not stale.exists()
    assert "no-compiler" in capfd.readouterr().err


def unfit(monkeypatch, tmp_path, why):
    monkeypatch.setattr(A, "_BIND", None)
    if why == "another torch's":
        monkeypatch.setattr(torch, "__version__", "0.1")
        return
    path = tmp_path / "_arckv_bind.so"
    if why == "no library":
        path.write_bytes(b"not one")
    monkeypatch.setattr(A, "BIND_PATH", str(path))


@pytest.mark.parametrize("why", ["missing", "no library", "another torch's"])
def test_without_a_native_part_that_fits_all_calls_go_the_long_way(monkeypatch, tmp_path, why):
    unfit(monkeypatch, tmp_path, why)
    with pytest.warns(RuntimeWarning, match="_arckv_bind.so"):
        m = A._bind()
    assert m is A._bind()
    for name in NAMES:
        assert getattr(m, name)(0, 1, 2) is None
    monkeypatch.undo()
    assert A._bind() is not m


@pytest.mark.gpu
@pytest.mark.parametrize("why", ["missing", "no library", "another torch's"])
def test_calls_work_without_a_native_part(monkeypatch, tmp_path, why):
    x, f = torch.randn(3, 20, 128, device="cuda").bfloat16(), A.rotary_frequencies(64)
    pos = torch.arange(3, dtype=torch.int32, device="cuda")

    def calls():
        c = A.ncache(3, 30)
        for t in c:
            t.zero_()
        y = A.rotary(x, f, pos)
        A.ncache_write(c, y, x)
        return (y, *c, *A.ncache_read(c, 2, 9), A.attend_ncache(x[:, :4].contiguous(), c))
    want = calls()
    unfit(monkeypatch, tmp_path, why)
    with pytest.warns(RuntimeWarning):
        got = calls()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.gpu
def test_the_library_is_called_without_the_interpreters_lock():
    """A launch may wait, for room in a queue say; other Python threads go on meanwhile.  In place of each entry point stands
    Python's own question whether this thread holds the lock: 0, which is also the entry points' OK, where it does not."""
    m, L = A._bind(), A.lib()
    at = lambda *f: tuple(ctypes.cast(x, ctypes.c_void_p).value for x in f)
    held = ctypes.pythonapi.PyGILState_Check
    c, dev = A.ncache(2, 50), torch.cuda.current_device()
    x, f = torch.zeros(2, 3, 128, dtype=torch.bfloat16, device="cuda"), A.rotary_frequencies(64)
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    m.init(at(*[held] * 5), torch._C._cuda_getCurrentRawStream)
    try:
        taken = [m.ncache_write(dev, c, x, x, None, None), m.ncache_read(dev, c, 0, 3, False, None),
                 m.attend_ncache(dev, x, c, None, None, None, None, None, None, None, ws),
                 m.rotary(dev, x, f, None, None, False, False, 1.0, torch.empty_like(x), None)]
    finally:
        m.init(at(L.arckv_ncache_write, L.arckv_ncache_read, L.arckv_attend_ncache_workspace_size, L.arckv_attend_ncache,
                  L.arckv_rotary), torch._C._cuda_getCurrentRawStream)
    assert all(t is not None for t in taken)


@pytest.mark.gpu
def test_calls_from_two_threads_at_once():
    """Each thread's calls, on a stream of its own, give what they give alone."""
    x = [torch.randn(6, 200, 128, device="cuda").bfloat16() for _ in range(2)]
    f = A.rotary_frequencies(64)

    def calls(i):
        out = []
        with torch.cuda.stream(streams[i]):
            for _ in range(50):
                c = A.ncache(6, 200)
                y = A.rotary(x[i], f)
                A.ncache_write(c, y, x[i])
                out = [y, *A.ncache_read(c), A.attend_ncache(x[i][:, :4].contiguous(), c)]
        streams[i].synchronize()
        return out
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    want = [calls(0), calls(1)]
    with concurrent.futures.ThreadPoolExecutor(2) as ex:
        got = list(ex.map(calls, (0, 1)))
    for a, b in zip(want, got):
        assert all(torch.equal(s, t) for s, t in zip(a, b))
