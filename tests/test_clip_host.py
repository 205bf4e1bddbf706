"""Host side of the norm, clipping and update entry points, without a GPU:
tensor tables, workspace sizes and every refusal of the C ABI (all of them
come before anything is enqueued); and the host code under sanitizers."""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2108_02416_amd import aspis

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = "/opt/rocm"
SIZE = {0: 4, 1: 2, 2: 2}


def _table(numels, dtypes, base=1 << 40):
    """The table of tensors laid one after another from an invented address."""
    L = aspis.lib()
    n = len(numels)
    numel = np.array(numels, dtype=np.int64)
    dtype = np.array(dtypes, dtype=np.int32)
    ptr, at = np.zeros(n, dtype=np.uint64), base
    for i in range(n):
        at += -at % SIZE[dtypes[i]]
        ptr[i] = at
        at += numels[i] * SIZE[dtypes[i]]
    entries = L.aspis_tensor_entries(numel.ctypes.data, n)
    out = np.zeros((entries, 2), dtype=np.uint64)
    st = L.aspis_tensor_table(ptr.ctypes.data, numel.ctypes.data, dtype.ctypes.data, n,
                              out.ctypes.data, entries)
    assert st == aspis.OK
    chunks = [aspis.Chunk.from_buffer_copy(out[i].tobytes()) for i in range(entries)]
    return ptr, chunks, L.aspis_tensor_chunks(numel.ctypes.data, n)


@pytest.mark.parametrize("numels,dtypes", [
    ([7840, 10], [0, 0]), ([], []), ([0], [1]), ([0, 5, 0, 0, 3, 0], [0, 1, 2, 0, 2, 1]),
    ([1, 4096, 4097, 8192, 100_000], [2, 0, 1, 0, 2])])
def test_a_table_covers_every_element_once(numels, dtypes):
    ptr, entries, n_chunks = _table(numels, dtypes)
    chunks, tensors = entries[:n_chunks], entries[n_chunks:]
    assert len(tensors) == len(numels)
    k = filled = 0
    for i, (n, t) in enumerate(zip(numels, dtypes)):
        assert (tensors[i].addr, tensors[i].info) == (k, filled)
        at = 0
        for _ in range(tensors[i].n):
            c = chunks[k]
            assert c.addr == int(ptr[i]) + at * SIZE[t] and 0 < c.n <= 4096
            assert c.info == filled * 4 + t
            at += c.n
            k += 1
        assert at == n
        filled += n > 0
    assert k == n_chunks


def test_table_refusals():
    L = aspis.lib()
    one = np.array([5], dtype=np.int64)
    kind = np.array([0], dtype=np.int32)
    out = np.zeros((2, 2), dtype=np.uint64)

    def table(ptr=4096, numel=one, dtype=kind, count=1, buf=out, cap=2):
        p = np.array([ptr], dtype=np.uint64)
        return L.aspis_tensor_table(p.ctypes.data, numel.ctypes.data, dtype.ctypes.data, count,
                                    buf.ctypes.data if buf is not None else None, cap)

    assert table() == aspis.OK
    assert table(ptr=0) == aspis.ERR_INVALID_ARG
    assert table(ptr=4098) == aspis.ERR_INVALID_ARG            # misaligned float32
    assert table(ptr=4098, dtype=np.array([1], dtype=np.int32)) == aspis.OK
    assert table(dtype=np.array([3], dtype=np.int32)) == aspis.ERR_INVALID_ARG
    assert table(numel=np.array([-1], dtype=np.int64)) == aspis.ERR_INVALID_ARG
    assert table(numel=np.array([1 << 39], dtype=np.int64)) == aspis.ERR_OVERFLOW
    assert table(numel=np.array([1 << 62], dtype=np.int64)) == aspis.ERR_OVERFLOW
    assert table(count=-1) == aspis.ERR_INVALID_ARG
    assert table(buf=None) == aspis.ERR_INVALID_ARG
    out[:] = 7
    assert table(cap=1) == aspis.ERR_BUFFER_SMALL
    assert (out == 7).all()
    assert table(ptr=0, numel=np.array([0], dtype=np.int64)) == aspis.OK
    assert L.aspis_tensor_chunks(None, 1) == -1 and L.aspis_tensor_entries(None, 0) == 0
    assert L.aspis_norm_workspace(-1) == 0 and L.aspis_norm_workspace(0) > 0


P = 1 << 20   # an address that nothing reads: every call below is refused


def _list_calls():
    L = aspis.lib()
    sgd = lambda **k: aspis.SgdOptions(**{"lr": 0.1, "momentum": 0.9, "max_norm": 1.0, **k})
    adam = lambda **k: aspis.AdamwOptions(**{"lr": 0.1, "beta_one": 0.9, "beta_two": 0.99,
                                             "eps": 1e-8, "max_norm": 1.0, "step": 1, **k})
    ws = 1 << 20
    bad, small = aspis.ERR_INVALID_ARG, aspis.ERR_BUFFER_SMALL
    norm = lambda t=P, n=3, k=1, s=P, o=P, w=P, b=ws: L.aspis_grad_norm(t, n, k, s, o, None, w, b, None)
    clip = lambda t=P, out=None, n=3, m=1.0, s=P, o=P, f=0, w=P, b=ws: \
        L.aspis_clip_grads(t, out, n, m, s, o, f, w, b, None)
    up = lambda p=P, g=P, m=P, c=None, n=3, o=None, s=P, r=P, w=P, b=ws, **k: L.aspis_clipped_sgd(
        p, g, m, c, n, ctypes.byref(sgd(**k) if o is None else o), s, r, w, b, None)
    ad = lambda p=P, g=P, m=P, v=P, c=None, n=3, s=P, r=P, w=P, b=ws, **k: L.aspis_clipped_adamw(
        p, g, m, v, c, n, ctypes.byref(adam(**k)), s, r, w, b, None)
    nan, inf = math.nan, math.inf
    yield from [(bad, norm, {"t": None}), (bad, norm, {"n": -1}), (bad, norm, {"n": 1 << 40}),
                (bad, norm, {"s": None}), (bad, norm, {"o": None}), (bad, norm, {"t": P + 8}),
                (bad, norm, {"w": P + 8}), (bad, norm, {"k": -1}), (small, norm, {"w": None}),
                (small, norm, {"b": 16})]
    yield from [(bad, clip, {"t": None}), (bad, clip, {"m": -1.0}), (bad, clip, {"m": nan}),
                (bad, clip, {"out": P + 4}), (bad, clip, {"f": 2}), (small, clip, {"b": 0})]
    yield from [(bad, up, {"p": None}), (bad, up, {"g": None}), (bad, up, {"m": None}),
                (bad, up, {"p": P + 8}), (bad, up, {"m": P + 8}), (bad, up, {"c": P + 8}),
                (bad, up, {"lr": nan}), (bad, up, {"lr": inf}), (bad, up, {"momentum": 1.0}),
                (bad, up, {"momentum": -0.1}), (bad, up, {"weight_decay": -1.0}),
                (bad, up, {"max_norm": nan}), (bad, up, {"flags": 4}), (small, up, {"b": 8})]
    yield from [(bad, ad, {"v": None}), (bad, ad, {"m": None}), (bad, ad, {"step": 0}),
                (bad, ad, {"beta_one": 1.0}), (bad, ad, {"beta_two": nan}), (bad, ad, {"eps": -1.0}),
                (bad, ad, {"weight_decay": inf}), (bad, ad, {"c": P + 8}), (bad, ad, {"flags": 8})]
    rows = lambda x=P, r=4, d=8, ld=8, t=0, n=P, w=P, b=ws: L.aspis_row_norms(x, r, d, ld, t, n, w, b, None)
    crows = lambda x=P, r=4, d=8, ld=8, t=0, m=1.0, o=1 << 30, ldo=8, n=P, f=0, w=P, b=ws: \
        L.aspis_clip_rows(x, r, d, ld, t, m, o, ldo, n, f, w, b, None)
    yield from [(bad, rows, {"x": None}), (bad, rows, {"x": P + 2}), (bad, rows, {"ld": 7}),
                (bad, rows, {"r": -1}), (bad, rows, {"d": -1}), (bad, rows, {"t": 3}),
                (bad, rows, {"n": None}), (small, rows, {"d": 1 << 20, "ld": 1 << 20, "b": 8}),
                (aspis.ERR_OVERFLOW, rows, {"r": 1 << 40, "ld": 1 << 40}),
                (aspis.ERR_OVERFLOW, rows, {"d": 1 << 35, "ld": 1 << 35})]
    yield from [(bad, crows, {"m": -1.0}), (bad, crows, {"m": nan}), (bad, crows, {"o": None}),
                (bad, crows, {"o": (1 << 30) + 1}), (bad, crows, {"ldo": 7}), (bad, crows, {"f": 1}),
                (bad, crows, {"o": P + 4}), (bad, crows, {"o": P + 32}),      # overlaps
                (bad, crows, {"o": P, "ldo": 9}), (bad, crows, {"o": P - 64})]


def test_every_refusal():
    for status, call, args in _list_calls():
        assert call(**args) == status, (args, aspis.lib().aspis_last_error())
        assert aspis.lib().aspis_last_error()


def test_workspaces_grow_with_the_work():
    L = aspis.lib()
    assert L.aspis_norm_workspace(1 << 20) > L.aspis_norm_workspace(1) > 0
    assert L.aspis_row_workspace(1000, 30_000, 0) == 0        # in registers
    assert L.aspis_row_workspace(1000, 40_000, 0) > 0
    assert L.aspis_row_workspace(1000, 60_000, 1) == 0
    assert L.aspis_row_workspace(0, 1 << 30, 0) == 0
    for bad in ((-1, 5, 0), (5, -1, 0), (5, 5, 7), (1 << 40, 1 << 40, 0), (1, 1 << 35, 0)):
        assert L.aspis_row_workspace(*bad) == 2 ** 64 - 1, bad


def test_missing_library_raises(monkeypatch, tmp_path):
    monkeypatch.setattr(aspis, "LIB_PATH", str(tmp_path / "libaspis.so"))
    monkeypatch.setattr(aspis, "_lib", None)
    import torch
    with pytest.raises(ImportError, match="libaspis.so is missing"):
        aspis.TensorList([], device=torch.device("cuda", 0))


def test_the_state_of_a_list_of_tensors():
    import torch
    a, b = torch.zeros(12, dtype=torch.bfloat16), torch.zeros(5)
    now = aspis._tensor_state([a, b])
    assert now == aspis._tensor_state([a, b])
    assert aspis._tensor_state([]) == b""
    for other in ([b, a], [a], [a.view(torch.float16), b], [a[:11], b], [a[1:], b], [a, b.clone()]):
        assert aspis._tensor_state(other) != now
    # the same elements in another shape, but not in another order
    assert aspis._tensor_state([a.reshape(3, 4), b]) == now
    turned = aspis._tensor_state([a.reshape(3, 4).t(), b])
    assert turned != now and turned != aspis._tensor_state([a.reshape(2, 6).t(), b])
    for wrong in ((a, b), [a, 1], None):
        with pytest.raises(TypeError):
            aspis._tensor_state(wrong)


def test_lists_that_share_memory():
    import itertools
    import random
    native = aspis._tensors()

    def pack(spans):
        spans = sorted(spans)
        return np.array([*(x for s in spans for x in s), max((b for _, b in spans), default=0)],
                        dtype=np.uint64).tobytes()
    rng = random.Random(5)
    seen = set()
    for _ in range(3000):
        room = rng.choice([20, 60, 400])
        lists = []
        for _ in range(rng.randint(1, 4)):
            starts = [rng.randrange(room) for _ in range(rng.randint(0, 4))]
            lists.append([(a, a + rng.randint(1, 9)) for a in starts])
        want = all(x[1] <= y[0] or y[1] <= x[0] for p, q in itertools.combinations(lists, 2)
                   for x in p for y in q)
        assert native.apart(*map(pack, lists)) == want, lists
        seen.add(want)
    assert seen == {True, False}
    assert native.apart()
    for wrong in ((b"",), (b"0" * 16,), ([1],), (pack([]),) * 9):
        with pytest.raises(TypeError):
            native.apart(*wrong)


def test_the_native_checks_take_gpu_tensors_only():
    """None sends the binding to the Python checks, which say what is wrong."""
    import torch
    t = torch.zeros(6)
    native = aspis._tensors()
    assert native.buffer(t, torch.float32, 6, 0) is None
    assert native.buffer(None, torch.float32, 6, 0) is None
    assert native.rows(t) is None and native.rows([t]) is None
    for wrong in ((t,), (t, 0, 6, 0), (t, torch.float32, "6", 0), (t, torch.float32, 1 << 70, 0)):
        with pytest.raises((TypeError, OverflowError)):
            native.buffer(*wrong)
    with pytest.raises(aspis.AspisError, match="norms"):
        aspis._buffer("norms", t, torch.float32, 6, torch.device("cuda", 0))


def test_missing_module_raises(monkeypatch):
    import sys
    import torch
    monkeypatch.setattr(aspis, "_native", None)
    import paper_2108_02416_amd
    monkeypatch.delattr(paper_2108_02416_amd, "_tensors", raising=False)
    monkeypatch.setitem(sys.modules, "paper_2108_02416_amd._tensors", None)
    with pytest.raises(ImportError, match="_tensors.so is missing"):
        aspis.TensorList([], device=torch.device("cuda", 0))


@pytest.mark.skipif(shutil.which("g++") is None
                    or not os.path.exists(os.path.join(ROCM, "lib", "libamdhip64.so")),
                    reason="needs g++ and the ROCm host runtime library")
def test_host_code_under_sanitizers(tmp_path):
    src = os.path.join(ROOT, "tests", "host_sanitize")
    csrc = os.path.join(ROOT, "paper_2108_02416_amd", "csrc")
    exe = tmp_path / "clip_sanitize"
    subprocess.run(["g++", "-std=c++17", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=undefined", "-fno-omit-frame-pointer", "-g", "-O1",
                    "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"),
                    os.path.join(src, "clip_driver.cpp"), os.path.join(src, "device_stubs.cpp"),
                    os.path.join(csrc, "aspis_clip.cpp"), os.path.join(csrc, "aspis_host.cpp"),
                    "-L", os.path.join(ROCM, "lib"), f"-Wl,-rpath,{ROCM}/lib", "-lamdhip64",
                    "-lpthread", "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300,
                         env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0"))
    assert out.returncode == 0, out.stdout + out.stderr
    assert out.stdout.strip().endswith("ok")
    assert "runtime error" not in out.stderr and "AddressSanitizer" not in out.stderr, out.stderr


def _host_list(monkeypatch, tensors):
    """A TensorList of host tensors: its reading without a GPU."""
    import torch
    monkeypatch.setattr(aspis, "_raw_stream", lambda device: 0)
    handle = aspis.TensorList.__new__(aspis.TensorList)
    handle.tensors, handle.device = list(tensors), torch.device("cpu")
    handle._read()
    return handle


def _follows(handle):
    """The table names the tensors as they are now."""
    entries = handle._table.numpy().view(np.uint64)
    assert handle.table() == handle._table.data_ptr()
    sizes = [t.numel() for t in handle.tensors]
    assert handle.numels == sizes and handle.n_chunks == sum(-(-n // 4096) for n in sizes)
    starts = [int(entries[int(e[0]), 0]) for e in entries[handle.n_chunks:]]
    assert starts == [t.data_ptr() for t in handle.tensors]


def test_a_list_that_could_not_be_read_is_read_again(monkeypatch):
    """Tensors that turn unusable are refused at every call until they are
    usable again: never answered with the table of what they were."""
    import torch
    good = torch.zeros(600)
    for wrong in (torch.zeros(600, dtype=torch.float64),           # type
                  torch.zeros(1200)[::2],                          # gaps
                  torch.zeros(1).expand(600),                      # overlaps
                  torch.zeros(600, device="meta")):                # another device
        t = torch.zeros(600)
        t.data = good
        handle = _host_list(monkeypatch, [t, torch.zeros(5)])
        _follows(handle)
        if wrong.device.type == "meta":
            handle.tensors[0] = wrong
        else:
            t.data = wrong
        for _ in range(3):
            with pytest.raises((aspis.AspisError, RuntimeError)):
                handle.table()
        if wrong.device.type == "meta":
            handle.tensors[0] = t
        t.data = torch.zeros(200_000)
        handle.table()
        _follows(handle)


def test_a_table_that_could_not_be_uploaded_is_uploaded_again(monkeypatch):
    import torch
    t = torch.zeros(10)
    handle = _host_list(monkeypatch, [t])
    address = handle.table()
    t.data = torch.zeros(200_000)

    def full(array):
        raise torch.OutOfMemoryError("no memory for the table")
    with monkeypatch.context() as m:
        m.setattr(torch, "from_numpy", full)
        for _ in range(2):
            with pytest.raises(torch.OutOfMemoryError):
                handle.table()
            assert handle.n_chunks == 1 and handle._address == address
    handle.table()
    _follows(handle)


def test_buffers_hold_the_sum_a_call_went_by(monkeypatch):
    """A given sum of squares is what the call's buffers hold afterwards, new
    ones and kept ones, and the given tensor stays the caller's."""
    import types
    import torch
    monkeypatch.setattr(aspis, "_buffer", lambda name, t, dtype, n, device: t.data_ptr())
    grads = types.SimpleNamespace(device=torch.device("cpu"), ws_bytes=64)
    kept = aspis.NormBuffers.empty("cpu")
    kept.sumsq.fill_(7.0)
    for given in (torch.tensor([25.0], dtype=torch.float64), torch.tensor(36.0, dtype=torch.float64)):
        for bufs in (None, kept):
            got, _, total, _, _, _, flags = aspis._scratch(grads, bufs, None, given)
            assert bufs is None or got is bufs
            assert flags == aspis.CLIP_HAVE_SUMSQ and total == got.sumsq.data_ptr()
            assert got.sumsq.tolist() == [float(given)] and got.sumsq.data_ptr() != given.data_ptr()
    _, _, total, _, _, _, _ = aspis._scratch(grads, kept, None, kept.sumsq)
    assert total == kept.sumsq.data_ptr() and kept.sumsq.tolist() == [36.0]


def test_lists_match_tensor_by_tensor(monkeypatch):
    """A contiguous tensor may have any shape, whatever its neighbours are;
    one that is not has to have the gradient's shape and strides."""
    import torch
    make = lambda *ts: _host_list(monkeypatch, ts)
    turned = lambda: torch.zeros(3, 5).t()
    grads = make(turned(), torch.zeros(12))
    aspis._check_match("params", make(turned(), torch.zeros(3, 4)), grads)
    aspis._check_match("params", make(torch.zeros(15), torch.zeros(3, 4)),
                       make(torch.zeros(5, 3), torch.zeros(12)))
    for wrong in (make(torch.zeros(5, 3), torch.zeros(12)), make(torch.zeros(15), torch.zeros(12)),
                  make(turned(), torch.zeros(4, 3).t()), make(torch.zeros(5, 3).t(), torch.zeros(12))):
        for a, b in ((wrong, grads), (grads, wrong)):
            with pytest.raises(aspis.AspisError, match="not contiguous"):
                aspis._check_match("params", a, b)


def test_lists_see_negated_views(monkeypatch):
    """The imaginary part of a conjugate shares memory that holds its
    opposite."""
    import torch
    x = torch.complex(torch.tensor([3.0]), torch.tensor([4.0]))
    turned = x.conj().imag
    assert turned.is_neg() and turned.data_ptr() == x.imag.data_ptr()
    assert aspis._tensor_state([turned]) != aspis._tensor_state([x.imag])
    with pytest.raises(aspis.AspisError, match="negated"):
        _host_list(monkeypatch, [turned])
    _follows(_host_list(monkeypatch, [turned.resolve_neg()]))
