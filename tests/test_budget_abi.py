"""Refusals of the operators of a budget before anything is launched, their workspace
sizes, and their host layer under sanitizers (no GPU)."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

from paper_2606_29207_amd import kf

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000      # non-null, 256-byte aligned stand-in; never dereferenced here
HUGE = 1 << 40


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(kf._LIB_PATH):
        from paper_2606_29207_amd import build
        build.build()
    return kf.load()


def _shape(**kw):
    a = dict(num_seqs=2, num_q_heads=8, num_kv_heads=2, kv_dtype=kf.KV_BF16, num_pages=10,
             num_page_ids=8, scale=0.1)
    a.update(kw)
    return kf.make_shape(**a)


def _window(lib, shape=None, **kw):
    a = dict(q=FAKE, num_rows=5, q_stride=1024, begin=FAKE, first=FAKE, sinks=4, window=9,
             k_pool=FAKE, v_pool=FAKE, ks=None, vs=None, routes=FAKE, num_routes=3, max_pages=4,
             page_ids=FAKE, csr=FAKE, out=FAKE, lse=FAKE, ws=FAKE, ws_bytes=HUGE, err=FAKE)
    a.update(kw)
    return lib.kf_window_attn(
        ctypes.byref(shape or _shape()), a["q"], a["num_rows"], a["q_stride"], a["begin"], a["first"],
        a["sinks"], a["window"], a["k_pool"], a["v_pool"], a["ks"], a["vs"], a["routes"],
        a["num_routes"], a["max_pages"], a["page_ids"], a["csr"], a["out"], a["lse"], a["ws"],
        a["ws_bytes"], a["err"], None)


def _weights(lib, shape=None, **kw):
    a = dict(q=FAKE, num_rows=5, q_stride=1024, lse=FAKE, begin=FAKE, first=FAKE, k_pool=FAKE,
             ks=None, routes=FAKE, num_routes=3, max_pages=4, page_ids=FAKE, decay=1.0,
             weights=FAKE, ws=FAKE, ws_bytes=HUGE, err=FAKE)
    a.update(kw)
    return lib.kf_attn_weights(
        ctypes.byref(shape or _shape()), a["q"], a["num_rows"], a["q_stride"], a["lse"], a["begin"],
        a["first"], a["k_pool"], a["ks"], a["routes"], a["num_routes"], a["max_pages"],
        a["page_ids"], a["decay"], a["weights"], a["ws"], a["ws_bytes"], a["err"], None)


def _evict(lib, shape=None, **kw):
    a = dict(k_pool=FAKE, v_pool=FAKE, ks=None, vs=None, weights=FAKE, routes=FAKE, num_routes=3,
             max_pages=4, page_ids=FAKE, csr=FAKE, into=FAKE, keep=FAKE, max_keep=20, first=1,
             last=2, ws=FAKE, ws_bytes=HUGE, err=FAKE)
    a.update(kw)
    return lib.kf_kv_evict(
        ctypes.byref(shape or _shape()), a["k_pool"], a["v_pool"], a["ks"], a["vs"], a["weights"],
        a["routes"], a["num_routes"], a["max_pages"], a["page_ids"], a["csr"], a["into"], a["keep"],
        a["max_keep"], a["first"], a["last"], a["ws"], a["ws_bytes"], a["err"], None)


FP8 = dict(kv_dtype=kf.KV_FP8_E4M3)


@pytest.mark.parametrize("shape_kw,kw,status", [
    ({}, dict(sinks=-1), -1), ({}, dict(window=-1), -1), ({}, dict(first=None), -1),
    ({}, dict(first=FAKE + 2), -1), ({}, dict(q=None), -1), ({}, dict(q=FAKE + 8), -1),
    ({}, dict(begin=None), -1), ({}, dict(csr=FAKE + 1), -1), ({}, dict(out=FAKE + 8), -1),
    ({}, dict(lse=None), -1), ({}, dict(err=None), -1), ({}, dict(num_rows=-1), -1),
    ({}, dict(q_stride=1016), -1), ({}, dict(ws=None), -3), ({}, dict(ws=FAKE + 128), -3),
    ({}, dict(ws_bytes=256), -3), (FP8, {}, -1), (dict(kv_dtype=7), {}, -2),
    (dict(num_q_heads=34), {}, -2), (dict(scale=float("nan")), {}, -1)])
def test_window_host_checks(lib, shape_kw, kw, status):
    assert _window(lib, _shape(**shape_kw), **kw) == status


@pytest.mark.parametrize("shape_kw,kw,status", [
    ({}, dict(q=None), -1), ({}, dict(q=FAKE + 8), -1), ({}, dict(lse=None), -1),
    ({}, dict(lse=FAKE + 2), -1), ({}, dict(begin=None), -1), ({}, dict(first=None), -1),
    ({}, dict(first=FAKE + 1), -1), ({}, dict(k_pool=None), -1), ({}, dict(k_pool=FAKE + 8), -1),
    ({}, dict(routes=None), -1), ({}, dict(page_ids=None), -1), ({}, dict(weights=None), -1),
    ({}, dict(weights=FAKE + 2), -1), ({}, dict(err=None), -1), ({}, dict(decay=float("nan")), -1),
    ({}, dict(decay=float("inf")), -1), ({}, dict(num_rows=-1), -1), ({}, dict(num_routes=-1), -1),
    ({}, dict(max_pages=-1), -1), ({}, dict(q_stride=1016), -1), ({}, dict(q_stride=1028), -1),
    (FP8, {}, -1), (FP8, dict(ks=FAKE + 2), -1), (dict(kv_dtype=7), {}, -2),
    (dict(num_q_heads=34), {}, -2), (dict(num_q_heads=7), {}, -1),
    ({}, dict(num_routes=70000), -2), ({}, dict(num_rows=1 << 27), -2),
    ({}, dict(num_rows=2000, max_pages=128, ws=None), -3),
    ({}, dict(num_rows=2000, max_pages=128, ws=FAKE + 8), -3),
    ({}, dict(num_rows=2000, max_pages=128, ws_bytes=1000), -3)])
def test_weights_host_checks(lib, shape_kw, kw, status):
    assert _weights(lib, _shape(**shape_kw), **kw) == status


@pytest.mark.parametrize("shape_kw,kw,status", [
    ({}, dict(k_pool=None), -1), ({}, dict(v_pool=FAKE + 8), -1), ({}, dict(weights=None), -1),
    ({}, dict(weights=FAKE + 2), -1), ({}, dict(routes=None), -1), ({}, dict(page_ids=None), -1),
    ({}, dict(csr=None), -1), ({}, dict(into=None), -1), ({}, dict(into=FAKE + 2), -1),
    ({}, dict(keep=None), -1), ({}, dict(keep=FAKE + 1), -1), ({}, dict(err=None), -1),
    ({}, dict(max_keep=-1), -1), ({}, dict(first=-1), -1), ({}, dict(last=-1), -1),
    ({}, dict(num_routes=-1), -1), ({}, dict(max_pages=-1), -1), ({}, dict(ws=None), -3),
    ({}, dict(ws=FAKE + 8), -3), ({}, dict(ws_bytes=64), -3), (FP8, {}, -1), (FP8, dict(ks=FAKE), -1),
    (FP8, dict(ks=FAKE, vs=FAKE + 2), -1), (dict(kv_dtype=7), {}, -2),
    (dict(num_seqs=70000), {}, -2), (dict(num_pages=1 << 27), {}, -2),
    (dict(num_seqs=60000), dict(max_keep=1 << 20), -2)])
def test_evict_host_checks(lib, shape_kw, kw, status):
    assert _evict(lib, _shape(**shape_kw), **kw) == status


def test_nothing_to_do_is_a_no_op(lib):
    assert _window(lib, num_rows=0, q=None, out=None, ws=None, first=None) == 0
    assert _weights(lib, num_rows=0, q=None, lse=None, ws=None) == 0
    assert _weights(lib, num_routes=0, routes=None, weights=None) == 0
    assert _weights(lib, _shape(num_seqs=0), begin=None, first=None) == 0
    assert _evict(lib, _shape(num_seqs=0), into=None, keep=None, ws=None) == 0
    assert _evict(lib, num_routes=0, routes=None, ws=None) == 0


def test_workspace_sizes(lib):
    s = _shape()
    assert kf.attn_weights_workspace_bytes(s, 2, 3, 4) == 256
    assert 256 < kf.attn_weights_workspace_bytes(s, 2000, 3, 128) <= 4 << 20
    assert kf.attn_weights_workspace_bytes(s, -1, 3, 4) == 0
    assert kf.attn_weights_workspace_bytes(s, 2, 70000, 4) == 0
    assert kf.attn_weights_workspace_bytes(_shape(kv_dtype=7), 2, 3, 4) == 0
    n = kf.kv_evict_workspace_bytes(s, 100)
    assert 2 * 2 * 100 * 4 <= n <= 2 * 2 * 100 * 4 + 1024
    assert kf.kv_evict_workspace_bytes(s, -1) == 0
    assert kf.kv_evict_workspace_bytes(_shape(num_seqs=70000), 1) == 0


def test_binding_refuses_host_tensors_and_odd_sizes():
    s = _shape()
    i = torch.zeros(8, dtype=torch.int32)
    bf = torch.zeros((2, 8, 128), dtype=torch.bfloat16)
    pool = torch.zeros((10, 2, 16, 128), dtype=torch.bfloat16)
    with pytest.raises(kf.KFError):
        kf.bind_window_attn(s, bf, i, 1, 2, pool, pool, i, 4, i, i, i, bf, bf, i, i)
    with pytest.raises(kf.KFError):
        kf.bind_attn_weights(s, bf, bf.float(), i, pool, i, 4, i, i, 1.0, pool.float(), i)
    with pytest.raises(kf.KFError):
        kf.bind_kv_evict(s, pool, pool, pool.float(), i, 4, i, i, i, i, 20, 1, 2, i)


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_host_layer_under_asan_and_ubsan(tmp_path):
    """kf_budget_api.cpp built with g++ under both sanitizers against a host-only HIP test
    double, its launchers replaced by checking ones (tests/c/budget_stress.cpp)."""
    san = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer"]
    src = os.path.join(ROOT, "paper_2606_29207_amd", "csrc")
    inc = ["-I", os.path.join(ROOT, "tests", "c", "hipstub"), "-I", os.path.join(ROOT, "include"),
           "-I", src]
    exe = tmp_path / "budget_stress"
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-Wall", *san, *inc, os.path.join(src, "kf_api.cpp"),
           os.path.join(src, "kf_budget_api.cpp"),
           os.path.join(ROOT, "tests", "c", "budget_stress.cpp"), "-o", str(exe), "-lm"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, " ".join(cmd) + "\n" + res.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0",
               UBSAN_OPTIONS="print_stacktrace=1")
    env.pop("LD_PRELOAD", None)
    run = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300, env=env)
    assert run.returncode == 0 and "budget_stress ok" in run.stdout, run.stdout + run.stderr[-4000:]
