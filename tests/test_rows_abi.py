"""Refusals of the row operators before anything is launched, their workspace
sizes, and the host layer under sanitizers (no GPU)."""
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
    head_dim, page = kw.pop("head_dim", 128), kw.pop("page_size", 16)
    a.update(kw)
    s = kf.make_shape(**a)
    s.head_dim, s.page_size = head_dim, page
    return s


ROW_ARGS = dict(q=FAKE, num_rows=5, q_stride=1024, seq_row_begin=FAKE, k_pool=FAKE, v_pool=FAKE,
                k_scale=None, v_scale=None, routes=FAKE, num_routes=3, max_pages=4, page_ids=FAKE,
                seq_route_begin=FAKE, out=FAKE, lse=FAKE, workspace=FAKE, ws_bytes=HUGE, err=FAKE)


def _prompt(lib, shape=None, first_pos=FAKE, **kw):
    a = dict(ROW_ARGS, **kw)
    return lib.kf_prompt_attn(
        ctypes.byref(shape or _shape()), a["q"], a["num_rows"], a["q_stride"], a["seq_row_begin"],
        first_pos, a["k_pool"], a["v_pool"], a["k_scale"], a["v_scale"], a["routes"],
        a["num_routes"], a["max_pages"], a["page_ids"], a["seq_route_begin"], a["out"], a["lse"],
        a["workspace"], a["ws_bytes"], a["err"], None)


def _tree(lib, shape=None, k_draft=FAKE, v_draft=FAKE, kv_stride=256, tree_mask=FAKE, **kw):
    a = dict(ROW_ARGS, **kw)
    return lib.kf_tree_attn(
        ctypes.byref(shape or _shape()), a["q"], a["num_rows"], a["q_stride"], k_draft, v_draft,
        kv_stride, tree_mask, a["seq_row_begin"], a["k_pool"], a["v_pool"], a["k_scale"],
        a["v_scale"], a["routes"], a["num_routes"], a["max_pages"], a["page_ids"],
        a["seq_route_begin"], a["out"], a["lse"], a["workspace"], a["ws_bytes"], a["err"], None)


def _append(lib, shape=None, **kw):
    a = dict(k_pool=FAKE, v_pool=FAKE, k_scale=None, v_scale=None, k_rows=FAKE, v_rows=FAKE,
             num_rows=40, row_stride=256, row_list=None, num_entries=40, begin=FAKE, routes=FAKE,
             num_routes=3, page_ids=FAKE, workspace=FAKE, ws_bytes=48, err=FAKE)
    a.update(kw)
    return lib.kf_kv_append_rows(
        ctypes.byref(shape or _shape()), a["k_pool"], a["v_pool"], a["k_scale"], a["v_scale"],
        a["k_rows"], a["v_rows"], a["num_rows"], a["row_stride"], a["row_list"], a["num_entries"],
        a["begin"], a["routes"], a["num_routes"], a["page_ids"], a["workspace"], a["ws_bytes"],
        a["err"], None)


SHARED = [
    (dict(), dict(q=None), -1), (dict(), dict(q=FAKE + 8), -1), (dict(), dict(k_pool=None), -1),
    (dict(), dict(v_pool=FAKE + 4), -1), (dict(), dict(routes=None), -1),
    (dict(), dict(routes=FAKE + 2), -1), (dict(), dict(page_ids=None), -1),
    (dict(), dict(seq_row_begin=None), -1), (dict(), dict(seq_route_begin=None), -1),
    (dict(), dict(seq_row_begin=FAKE + 1), -1), (dict(), dict(out=None), -1),
    (dict(), dict(out=FAKE + 8), -1), (dict(), dict(lse=None), -1), (dict(), dict(lse=FAKE + 2), -1),
    (dict(), dict(err=None), -1), (dict(), dict(num_rows=-1), -1), (dict(), dict(num_routes=-1), -1),
    (dict(), dict(max_pages=-1), -1), (dict(), dict(q_stride=1016), -1),
    (dict(), dict(q_stride=1028), -1), (dict(), dict(q_stride=-1024), -1),
    (dict(), dict(workspace=None), -3), (dict(), dict(workspace=FAKE + 128), -3),
    (dict(), dict(ws_bytes=256), -3),
    (dict(kv_dtype=kf.KV_FP8_E4M3), dict(), -1),
    (dict(kv_dtype=kf.KV_FP8_E4M3), dict(k_scale=FAKE), -1),
    (dict(kv_dtype=kf.KV_FP8_E4M3), dict(k_scale=FAKE, v_scale=FAKE + 2), -1),
    (dict(kv_dtype=7), dict(), -2), (dict(head_dim=64), dict(), -2), (dict(page_size=32), dict(), -2),
    (dict(num_q_heads=7), dict(), -1), (dict(num_q_heads=34), dict(), -2),
    (dict(scale=float("nan")), dict(), -1), (dict(scale=float("inf")), dict(), -1),
    (dict(num_seqs=-1), dict(), -1),
    (dict(), dict(num_rows=2 ** 31 - 1), -2),
    (dict(num_q_heads=70000, num_kv_heads=70000), dict(q_stride=128 * 70000), -2),
]


@pytest.mark.parametrize("shape_kw,call_kw,status", SHARED)
def test_attention_host_checks(lib, shape_kw, call_kw, status):
    assert _prompt(lib, _shape(**shape_kw), **call_kw) == status
    assert _tree(lib, _shape(**shape_kw), kv_stride=128 * 70000, **call_kw) == status


def test_checks_of_one_operator_alone(lib):
    assert _prompt(lib, first_pos=None) == -1
    assert _prompt(lib, first_pos=FAKE + 2) == -1
    for kw in (dict(k_draft=None), dict(v_draft=None), dict(k_draft=FAKE + 8), dict(v_draft=FAKE + 2),
               dict(tree_mask=None), dict(tree_mask=FAKE + 4), dict(kv_stride=248),
               dict(kv_stride=260), dict(kv_stride=-256)):
        assert _tree(lib, **kw) == -1, kw


def test_no_rows_are_a_no_op(lib):
    assert _prompt(lib, num_rows=0, q=None, out=None, workspace=None, first_pos=None) == 0
    assert _tree(lib, num_rows=0, k_draft=None, tree_mask=None, workspace=None) == 0
    assert _append(lib, num_entries=0, k_rows=None, workspace=None) == 0
    assert _append(lib, num_routes=0, num_entries=0, routes=None) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(k_pool=None), -1), (dict(v_pool=FAKE + 8), -1), (dict(k_rows=None), -1),
    (dict(k_rows=FAKE + 8), -1), (dict(v_rows=FAKE + 4), -1), (dict(begin=None), -1),
    (dict(begin=FAKE + 2), -1), (dict(routes=None), -1), (dict(page_ids=None), -1),
    (dict(err=None), -1), (dict(row_list=FAKE + 1), -1), (dict(num_rows=-1), -1),
    (dict(num_entries=-1), -1), (dict(num_routes=-1), -1), (dict(num_entries=41), -1),
    (dict(row_stride=248), -1), (dict(row_stride=260), -1), (dict(workspace=None), -3),
    (dict(workspace=FAKE + 8), -3), (dict(ws_bytes=47), -3),
    (dict(num_rows=2 ** 31 - 1, num_entries=2 ** 31 - 1, num_routes=65535, ws_bytes=HUGE), -2),
    (dict(num_routes=65536, ws_bytes=HUGE), -2),
])
def test_append_rows_host_checks(lib, kw, status):
    assert _append(lib, **kw) == status


def test_append_rows_fp8_needs_scales(lib):
    s = _shape(kv_dtype=kf.KV_FP8_E4M3)
    assert _append(lib, s) == -1 and _append(lib, s, k_scale=FAKE) == -1
    assert _append(lib, s, k_scale=FAKE + 2, v_scale=FAKE) == -1


def test_workspace_sizes(lib):
    def size(rows, **kw):
        return kf.rows_attn_workspace_bytes(_shape(**kw), rows)

    assert size(2 ** 28) == 0 and size(2 ** 28, num_q_heads=2) > 0  # threads of a grid: 32 bits
    assert size(-1) == 0 and size(5, head_dim=64) == 0 and size(2 ** 31 - 1) == 0
    assert size(5, num_q_heads=70000, num_kv_heads=70000) == 0
    assert 0 < size(0) <= size(1) <= size(100) <= size(100000)
    # tables, pages and lengths do not matter
    assert size(100, num_page_ids=8) == size(100, num_page_ids=1 << 20) == size(100, num_pages=1 << 20)
    # records of at most eight (row tile, KV head) parts per compute unit
    assert size(1 << 20) < 400e6
    assert lib.kf_kv_append_rows_workspace_bytes(-1) == 0
    assert lib.kf_kv_append_rows_workspace_bytes(0) == 16
    assert lib.kf_kv_append_rows_workspace_bytes(100) == 1600


def test_binding_refuses_host_tensors():
    s = _shape()
    z = torch.zeros
    with pytest.raises(kf.KFError, match="device tensor"):
        kf.bind_prompt_attn(s, z((5, 8, 128), dtype=torch.bfloat16), z(2, dtype=torch.int32), None,
                            None, None, 4, None, None, None, None, None, None, None)
    with pytest.raises(kf.KFError, match="device tensor"):
        kf.bind_tree_attn(s, z((5, 8, 128), dtype=torch.bfloat16), z((5, 2, 128), dtype=torch.bfloat16),
                          None, None, None, None, None, 4, None, None, None, None, None, None, None)
    with pytest.raises(kf.KFError, match="device tensor"):
        kf.bind_kv_append_rows(s, z(1), z(1), z(1), z(1), z((1, 6)), z(1), z(1), z(1))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_host_layer_under_asan_and_ubsan(tmp_path):
    """kf_rows_api.cpp (with the planner of kf_api.cpp) built with g++ under both
    sanitizers against the host-only HIP test double, its launchers replaced by
    checkers (tests/c/rows_stress.cpp)."""
    inc = ["-I", os.path.join(ROOT, "tests", "c", "hipstub"), "-I", os.path.join(ROOT, "include"),
           "-I", os.path.join(ROOT, "paper_2606_29207_amd", "csrc")]
    exe = tmp_path / "rows_stress"
    csrc = os.path.join(ROOT, "paper_2606_29207_amd", "csrc")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-Wall", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", *inc,
           os.path.join(csrc, "kf_api.cpp"), os.path.join(csrc, "kf_rows_api.cpp"),
           os.path.join(ROOT, "tests", "c", "rows_stress.cpp"), "-o", str(exe), "-lm"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, " ".join(cmd) + "\n" + res.stderr
    env = dict(os.environ)
    env.pop("LD_PRELOAD", None)
    run = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300, env=env)
    assert run.returncode == 0 and "rows_stress ok" in run.stdout, run.stdout + run.stderr[-4000:]
