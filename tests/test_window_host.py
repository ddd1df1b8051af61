"""The host layer of the masked attention and of the 4-bit conversions on the CPU: refusals through the binding, and the whole
layer under AddressSanitizer and UndefinedBehaviorSanitizer (tests/host/window_driver.cpp), whose stand-ins for the launchers
check what every launch would index."""

import os
import subprocess

import pytest

import paper_2603_00907_amd as kvs
from test_abi_host import FakeBuf, status_of

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HOST = os.path.join(ROOT, "tests", "host")
CSRC = os.path.join(ROOT, "paper_2603_00907_amd", "csrc")


def test_window_host_layer_under_sanitizers(tmp_path):
    hipcc = "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not installed")
    exe = str(tmp_path / "window_driver")
    cmd = [hipcc, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-x", "hip",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xarch_host", "-fno-omit-frame-pointer",
           "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, os.path.join(CSRC, "kvs_window_api.hip"),
           os.path.join(HOST, "window_driver.cpp"), "-fsanitize=address", "-fsanitize=undefined", "-fno-gpu-sanitize",
           "-o", exe]
    build = subprocess.run(cmd, capture_output=True, text=True)
    assert build.returncode == 0, build.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert run.returncode == 0, (run.stdout[-3000:], run.stderr[-3000:])
    assert "all checks passed" in run.stdout
    assert "runtime error" not in run.stderr and "AddressSanitizer" not in run.stderr


def problem(**kw):
    base = dict(lens=[1024, 500], budgets=[1024, 500], group=2, window=4, head_dim=64, dtype="f32", n_sink=3, causal=True)
    return kvs.Problem(**{**base, **kw})


@pytest.mark.parametrize("kw,span,want", [
    (dict(), 0, kvs.KVS_OK),
    (dict(lens=[0, 3]), 0, kvs.KVS_OK),
    (dict(in_rows=[0, 1000]), 5, kvs.KVS_OK),                # units may share rows
    (dict(), -1, kvs.KVS_ERR_INVALID_ARG),
    (dict(head_dim=32), 0, kvs.KVS_ERR_INVALID_ARG),
    (dict(group=1 << 12, window=(1 << 10) + 1), 0, kvs.KVS_ERR_INVALID_ARG),
    (dict(n_sink=-1), 0, kvs.KVS_ERR_INVALID_ARG),
    (dict(lens=[-1, 3]), 0, kvs.KVS_ERR_INVALID_ARG),
    (dict(lens=[(1 << 22) + 1, 3]), 0, kvs.KVS_ERR_INVALID_ARG),
    (dict(scale=float("inf")), 0, kvs.KVS_ERR_INVALID_ARG),
    (dict(dtype=2), 0, kvs.KVS_ERR_DTYPE),
])
def test_window_problem_validation(kw, span, want):
    assert status_of(kvs.kvs_window_attention_workspace_size, problem(**kw), span=span) == want


def test_window_buffers_are_checked_on_the_host():
    p = problem()
    buf = lambda i, n=1 << 24: FakeBuf((i + 1) << 30, n)  # noqa: E731
    call = lambda fn, *a, **k: status_of(fn, p, *a, **k)  # noqa: E731
    need = kvs.kvs_window_attention_workspace_size(p)
    win = lambda **o: call(kvs.kvs_window_attention, o.get("Q", buf(0)), o.get("K", buf(1)), buf(2), o.get("counts"),  # noqa: E731
                           o.get("out", buf(3)), o.get("ws", buf(4)), ws_bytes=o.get("ws_bytes"))
    assert win(Q=None) == kvs.KVS_ERR_INVALID_ARG
    assert win(K=FakeBuf(buf(1).addr + 8, 16)) == kvs.KVS_ERR_INVALID_ARG
    assert win(out=buf(1)) == kvs.KVS_ERR_ALIAS
    assert win(counts=buf(3)) == kvs.KVS_ERR_ALIAS
    if need:
        assert win(ws=None) == kvs.KVS_ERR_WORKSPACE
        assert win(ws_bytes=need - 1) == kvs.KVS_ERR_WORKSPACE
    packed = lambda **o: call(kvs.kvs_window_attention_packed, buf(0), buf(1), o.get("ks", buf(5)), buf(2), buf(6), None,  # noqa: E731
                              o.get("out", buf(3)), buf(4))
    assert packed(ks=None) == kvs.KVS_ERR_INVALID_ARG
    assert packed(out=buf(6)) == kvs.KVS_ERR_ALIAS
    assert call(kvs.kvs_pack, buf(0), buf(1), buf(2), buf(3), buf(4), buf(4)) == kvs.KVS_ERR_ALIAS
    assert call(kvs.kvs_pack, buf(0), buf(1), buf(2), buf(3), None, buf(5)) == kvs.KVS_ERR_INVALID_ARG
    assert call(kvs.kvs_unpack, buf(2), buf(3), buf(4), buf(5), buf(0), buf(0)) == kvs.KVS_ERR_ALIAS
    shared = problem(out_rows=[0, 1000])
    assert status_of(kvs.kvs_pack, shared, buf(0), buf(1), buf(2), buf(3), buf(4), buf(5)) == kvs.KVS_ERR_INVALID_ARG
