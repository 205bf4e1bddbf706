"""Host side of the token operators, without a GPU: every refusal of the C
ABI comes before anything is enqueued; workspaces; the plain forms the GPU
tests compare with; and the host code under sanitizers."""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2108_02416_amd import aspis

from _tokens import Policy, embed_sums, kept, philox, policy_inputs, softmax_loss

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = "/opt/rocm"
# addresses that nothing reads: every call below is refused
P, Q, W = 1 << 40, 1 << 41, 1 << 42
BAD, SMALL, OVER = aspis.ERR_INVALID_ARG, aspis.ERR_BUFFER_SMALL, aspis.ERR_OVERFLOW
WS = 1 << 24


def _embed(table=P, vocab=9, d=6, ld=6, kind=0, tokens=P, n=4, index=1, scale=1.0, out=Q, ldo=6,
           to=0):
    return aspis.lib().aspis_embed(table, vocab, d, ld, kind, tokens, n, index, scale, out, ldo, to,
                                   None)


def _embed_grad(grad=P, n=4, d=6, ld=6, kind=0, tokens=P, index=1, scale=1.0, out=Q, vocab=9,
                ldo=6, to=0, flags=0, ws=W, size=WS):
    return aspis.lib().aspis_embed_grad(grad, n, d, ld, kind, tokens, index, scale, out, vocab, ldo,
                                        to, flags, ws, size, None)


def _dropout(x=P, rows=4, d=6, ld=6, kind=0, p=0.1, seed=1, at=None, offset=0, res=None, ldr=6,
             out=Q, ldo=6):
    return aspis.lib().aspis_dropout(x, rows, d, ld, kind, p, seed, at, offset, res, ldr, out, ldo,
                                     None)


def _logps(z=P, rows=4, vocab=6, ld=6, kind=0, tokens=P, index=1, temperature=1.0, logps=Q, ws=W,
           size=WS):
    return aspis.lib().aspis_token_logps(z, rows, vocab, ld, kind, tokens, index, temperature, logps,
                                         ws, size, None)


def _policy(z=P, rows=4, vocab=6, ld=6, kind=0, tokens=P, index=1, old=P, adv=P, weight=P, ref=P,
            sums=P + 4096, logps=P + 8192, grad=Q, ldg=6, ws=W, size=WS, low=0.2, high=0.2, kl=0.0,
            temperature=1.0, scale=1.0):
    opt = aspis.PolicyOptions(low, high, kl, temperature, scale)
    return aspis.lib().aspis_policy_loss(z, rows, vocab, ld, kind, tokens, index, old, adv, weight,
                                         ref, ctypes.byref(opt), sums, logps, grad, ldg, ws, size,
                                         None)


NAN, INF = math.nan, math.inf


@pytest.mark.parametrize("status,call,args", [
    *[(BAD, _embed, a) for a in (
        {"table": None}, {"table": P + 2}, {"tokens": None}, {"tokens": P + 4}, {"out": None},
        {"out": Q + 1}, {"vocab": -1}, {"d": -1}, {"n": -1}, {"ld": 5}, {"ldo": 5}, {"kind": 3},
        {"to": -1}, {"index": 2}, {"scale": NAN}, {"scale": INF}, {"scale": 1e39},
        {"out": P + 24}, {"out": P, "ldo": 12})],
    *[(OVER, _embed, a) for a in ({"vocab": 1 << 31}, {"ld": 1 << 60}, {"n": 1 << 59, "ldo": 99})],
    *[(BAD, _embed_grad, a) for a in (
        {"grad": None}, {"grad": P + 2}, {"tokens": None}, {"tokens": P + 2, "index": 0},
        {"out": None}, {"out": Q + 2}, {"vocab": -1}, {"d": -1}, {"n": -1}, {"ld": 5}, {"ldo": 5},
        {"kind": 3}, {"to": 5}, {"index": -1}, {"scale": NAN}, {"flags": 2}, {"ws": W + 8, "n": 2000},
        {"out": P + 48})],
    *[(SMALL, _embed_grad, a) for a in ({"ws": None}, {"size": 100}, {"n": 1 << 20, "size": 1 << 20})],
    *[(OVER, _embed_grad, a) for a in ({"vocab": 1 << 31}, {"n": (1 << 30) + 1},
                                       {"d": 1 << 58, "ld": 1 << 58, "ldo": 1 << 58, "vocab": 1})],
    *[(BAD, _dropout, a) for a in (
        {"x": None}, {"x": P + 1}, {"out": None}, {"rows": -1}, {"d": -2}, {"ld": 5}, {"ldo": 5},
        {"kind": 9}, {"p": -0.1}, {"p": 1.1}, {"p": NAN}, {"at": P + 4}, {"res": P + 1, "ldr": 6},
        {"res": P, "ldr": 4}, {"out": P + 4}, {"out": P, "ldo": 7}, {"res": Q + 4})],
    *[(OVER, _dropout, a) for a in ({"ld": 1 << 59}, {"rows": 1 << 58})],
    *[(BAD, _logps, a) for a in (
        {"z": None}, {"z": P + 1}, {"rows": -1}, {"vocab": -1}, {"ld": 5}, {"kind": 4},
        {"tokens": None}, {"tokens": P + 4}, {"index": 7}, {"temperature": 0.0},
        {"temperature": -1.0}, {"temperature": NAN}, {"temperature": INF}, {"temperature": 1e-31},
        {"logps": None}, {"logps": Q + 2}, {"ws": W + 4})],
    *[(SMALL, _logps, a) for a in ({"ws": None}, {"size": 0})],
    *[(OVER, _logps, a) for a in ({"vocab": (1 << 24) + 1, "ld": 1 << 25},
                                  {"rows": (1 << 30) + 1})],
    *[(BAD, _policy, a) for a in (
        {"z": None}, {"old": None}, {"old": P + 2}, {"adv": None}, {"weight": None},
        {"weight": P + 1}, {"ref": P + 3}, {"ref": None, "kl": 0.1}, {"sums": None},
        {"logps": None}, {"grad": Q + 2}, {"ldg": 5}, {"grad": P + 4}, {"grad": P, "ldg": 8},
        {"low": -0.1}, {"low": 1.1}, {"low": NAN}, {"high": -1.0}, {"high": INF}, {"high": NAN},
        {"kl": -1.0}, {"kl": NAN}, {"kl": 1e39}, {"temperature": 0.0}, {"scale": INF},
        {"scale": NAN}, {"scale": 1e30, "temperature": 1e-20}, {"ws": W + 2}, {"logps": P},
        {"logps": P + 12}, {"logps": P - 12}, {"sums": P + 8}, {"sums": P - 8})],
    *[(SMALL, _policy, a) for a in ({"ws": None}, {"size": 10})],
])
def test_refusals(status, call, args):
    assert call(**args) == status, args
    assert aspis.lib().aspis_last_error()


# what is written shares no memory with anything else
@pytest.mark.parametrize("call,args", [
    *[(_embed, a) for a in ({"tokens": Q}, {"tokens": Q + 88}, {"tokens": Q - 24},
                            {"out": P + 24, "tokens": Q}, {"table": Q + 20, "ld": 6})],
    *[(_embed_grad, a) for a in ({"tokens": Q}, {"ws": P}, {"ws": Q}, {"ws": Q + 208},
                                 {"tokens": W}, {"tokens": W + 16})],
    *[(_dropout, a) for a in ({"at": Q}, {"at": Q + 88}, {"out": P + 24, "ldo": 7},
                              {"x": P, "ld": 12, "out": P + 20, "ldo": 12},
                              {"x": P, "ld": 12, "out": P + 28, "ldo": 12},
                              {"x": P, "ld": 12, "out": P + 24, "ldo": 13})],
    *[(_logps, a) for a in ({"logps": P}, {"logps": P + 92}, {"tokens": Q, "index": 0},
                            {"tokens": W}, {"ws": P}, {"ws": Q}, {"rows": 1, "vocab": 1, "logps": P})],
    *[(_policy, a) for a in (
        {"tokens": Q}, {"tokens": P + 8192}, {"tokens": P + 4096}, {"sums": P + 8196},
        {"sums": Q}, {"logps": Q + 92}, {"logps": P + 92}, {"ws": P}, {"ws": Q},
        {"ws": P + 4096}, {"old": W}, {"ref": W + 16}, {"adv": Q},
        {"weight": Q + 4}, {"ref": Q}, {"ldg": 12, "ld": 12, "grad": P + 20})],
])
def test_outputs_over_inputs(call, args):
    assert call(**args) == BAD, args
    assert b"overlap" in aspis.lib().aspis_last_error()


def test_null_options():
    assert aspis.lib().aspis_policy_loss(P, 1, 1, 1, 0, P, 1, P, P, P, P, None, P, P, None, 0, P, WS,
                                         None) == BAD


def test_workspaces():
    L, none = aspis.lib(), 2 ** 64 - 1
    assert L.aspis_embed_workspace(1 << 16, 1024) > L.aspis_embed_workspace(1 << 12, 64) > 0
    # two arrays of pairs and at most a quarter of the gradient's elements
    assert L.aspis_embed_workspace(1 << 20, 2048) < 16 * (1 << 20) + (1 << 20) * 2048
    for bad in ((-1, 4), (4, -1), ((1 << 30) + 1, 1), (1 << 30, 1 << 40)):
        assert L.aspis_embed_workspace(*bad) == none, bad
    assert L.aspis_policy_workspace(0, 1000, 1) % 16 == 0
    assert L.aspis_policy_workspace(4096, 32_003, 1) > L.aspis_policy_workspace(4, 32_003, 1) > 0
    for bad in ((-1, 4, 0), (4, -1, 0), (4, (1 << 24) + 1, 0), (4, 4, 3), (1 << 60, 1 << 20, 0)):
        assert L.aspis_policy_workspace(*bad) == none, bad


def test_the_generator_gives_the_published_number():
    """A known answer that comes with the generator's paper."""
    assert philox(0, np.zeros(1, np.uint64))[0].tolist() == [
        0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]


def test_positions_continue_across_blocks_and_wrap():
    whole = kept(100, 0.3, 7, 5)
    for at in (1, 3, 8, 64):
        assert (kept(100 - at, 0.3, 7, 5 + at) == whole[at:]).all()
    wrapped = kept(40, 0.3, 7, 2 ** 64 - 11)
    assert (wrapped[11:] == kept(29, 0.3, 7, 0)).all()


def test_the_plain_policy_gradient_is_the_slope_of_its_loss():
    z, t, old, adv, w, ref = policy_inputs(5, 7, seed=1, masked=0.0)
    z = z.double().numpy()
    args = (t, old.astype(float), adv.astype(float), w.astype(float), ref.astype(float), (0.2, 0.2),
            0.3, 0.9)
    plain = Policy(z, t, old, adv, w, ref, (0.2, 0.2), 0.3, 0.9)
    assert abs(plain.sums[0] - softmax_loss(z, *args)) < 1e-12
    h = 1e-6
    for i in range(5):
        for v in range(7):
            up, down = z.copy(), z.copy()
            up[i, v] += h
            down[i, v] -= h
            slope = (softmax_loss(up, *args) - softmax_loss(down, *args)) / (2 * h)
            assert abs(slope - plain.grad[i, v]) < 1e-8


def test_the_plain_sums_by_token():
    g = np.arange(12.0).reshape(6, 2)
    sums, sizes, count = embed_sums(g, [2, -1, 0, 2, 3, 7], 3)
    assert sums.tolist() == [[4, 5], [0, 0], [6, 8]] and count.tolist() == [1, 0, 2]
    assert (sizes == np.abs(sums)).all()


@pytest.mark.skipif(shutil.which("g++") is None
                    or not os.path.exists(os.path.join(ROCM, "lib", "libamdhip64.so")),
                    reason="needs g++ and the ROCm host runtime library")
def test_host_code_under_sanitizers(tmp_path):
    src = os.path.join(ROOT, "tests", "host_sanitize")
    csrc = os.path.join(ROOT, "paper_2108_02416_amd", "csrc")
    exe = tmp_path / "tokens_sanitize"
    subprocess.run(["g++", "-std=c++17", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=undefined", "-fno-omit-frame-pointer", "-g", "-O1",
                    "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"),
                    os.path.join(src, "tokens_driver.cpp"), os.path.join(src, "device_stubs.cpp"),
                    os.path.join(csrc, "aspis_tokens.cpp"), os.path.join(csrc, "aspis_host.cpp"),
                    "-L", os.path.join(ROCM, "lib"), f"-Wl,-rpath,{ROCM}/lib", "-lamdhip64",
                    "-lpthread", "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300,
                         env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0"))
    assert out.returncode == 0, out.stdout + out.stderr
    assert out.stdout.strip().endswith("ok")
    assert "runtime error" not in out.stderr and "AddressSanitizer" not in out.stderr, out.stderr
