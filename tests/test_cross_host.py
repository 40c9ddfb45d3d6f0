"""Plans of cross attention: host checks, no device."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_1511_06416_amd as same

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("code,args", [
    (same.SAME_EINVAL, dict(heads_q=3, heads_kv=2)),
    (same.SAME_EINVAL, dict(heads_q=0)),
    (same.SAME_EINVAL, dict(head_dim=0)),
    (same.SAME_EINVAL, dict(head_dim=12)),
    (same.SAME_EINVAL, dict(head_dim=136)),
    (same.SAME_EINVAL, dict(dtype=torch.float32)),
    (same.SAME_EINVAL, dict(dtype=torch.int8)),
    (same.SAME_EINVAL, dict(q_ptr=[1, 3])),
    (same.SAME_EINVAL, dict(q_ptr=[0, 3, 2], k_ptr=[0, 1, 1])),
    (same.SAME_EINVAL, dict(q_ptr=[0, 3, 4])),
    (same.SAME_ESIZE, dict(k_ptr=[0, 1 << 30])),
    (same.SAME_ESIZE, dict(q_ptr=[0, 1 << 28])),
    (same.SAME_ESIZE, dict(heads_q=1 << 17)),
])
def test_refused_plans(code, args):
    ok = dict(q_ptr=[0, 3], k_ptr=[0, 5], heads_q=4, heads_kv=1, head_dim=64, dtype=torch.bfloat16)
    with pytest.raises(same.SameError) as e:
        same.same_cross_create(**dict(ok, **args))
    assert e.value.code == code and str(e.value)


def test_workspace():
    """The gradient keeps delta, except of small segments; parts are needed
    where few rows meet many keys."""
    p = same.same_cross_create([0, 3], [0, 5], 4, 1, 64, torch.bfloat16)
    assert p.workspace_bytes() == p.workspace_bytes(True) == 0
    p = same.same_cross_create([0, 3], [0, 50], 4, 1, 64, torch.bfloat16)
    assert p.workspace_bytes() == 0 and p.workspace_bytes(True) >= 3 * 4 * 4
    p = same.same_cross_create([0, 1], [0, 100_000], 4, 1, 64, torch.bfloat16)
    assert p.workspace_bytes() > 0
    p = same.same_cross_create([0, 100_000], [0, 3], 4, 1, 64, torch.bfloat16)
    assert p.workspace_bytes(True) > 100_000 * 4 * 4


def test_empty_plans():
    for q_ptr, k_ptr in (([0], [0]), ([0, 0], [0, 0]), ([0, 0, 0], [0, 4, 4])):
        p = same.same_cross_create(q_ptr, k_ptr, 1, 1, 8, torch.float16)
        assert p.workspace_bytes() == 0
        same.same_cross_destroy(p)
        same.same_cross_destroy(p)


def test_pointers_are_copied():
    q_ptr = np.array([0, 5], dtype=np.int64)
    p = same.same_cross_create(q_ptr, [0, 7], 1, 1, 8, torch.float16)
    q_ptr[1] = 1 << 40
    assert p.n_q == 5 and p.workspace_bytes(True) < 1 << 20


def test_spilled_kernels_are_found():
    from paper_1511_06416_amd.build import spilled

    remarks = "\n".join("a.hip:1:1: remark: %s [-Rpass-analysis=kernel-resource-usage]" % line for line in [
        "Function Name: one", "    VGPRs: 256", "    SGPRs Spill: 6", "    VGPRs Spill: 0",
        "Function Name: two", "    VGPRs: 256", "    SGPRs Spill: 0", "    VGPRs Spill: 12"])
    assert spilled(remarks) == ["two"]
    assert spilled("") == []


@pytest.mark.parametrize("scale", [0.0, -1.0, 1e-46, 1e-39, 2.5e38, 3e38, 1e39, float("inf"), float("nan")])
@pytest.mark.parametrize("q_ptr", [[0], [0, 0]])
def test_refused_scales(scale, q_ptr):
    """Scales that are no positive normal number in 32 bits, before and after
    log2(e): a plan without tokens would otherwise have nothing to do."""
    p = same.same_cross_create(q_ptr, q_ptr, 1, 1, 8, torch.float16)
    lib = same.load_library()
    none = (None, 0, 0)
    args = (*none, *none, *none, None, scale, 0.0, 0, 0)
    assert lib.same_cross_attention(p.handle, *args, None, None, None, None) == same.SAME_EINVAL
    assert lib.same_cross_attention_backward(p.handle, *args, None, None, *none, None, None, None, None,
                                             None) == same.SAME_EINVAL
    args = (*none, *none, *none, None, 1.2e-38, 0.0, 0, 0)
    assert lib.same_cross_attention(p.handle, *args, None, None, None, None) == same.SAME_OK


@pytest.mark.parametrize("n_segs,code", [(-1, "SAME_EINVAL"), (1 << 31, "SAME_ESIZE"), (1 << 60, "SAME_ESIZE"),
                                         (1 << 61, "SAME_ESIZE"), ((1 << 63) - 1, "SAME_ESIZE")])
def test_refused_numbers_of_segments(n_segs, code):
    """Refused before the pointers are read or anything is sized by them; in a
    process of its own, which an exception through the C entry would end."""
    run = """
import ctypes, numpy as np, paper_1511_06416_amd as same
a, h = np.zeros(4, np.int64), ctypes.c_void_p()
rc = same.load_library().same_cross_create(%d, a.ctypes.data, a.ctypes.data, 1, 1, 8, same.SAME_F16, ctypes.byref(h))
assert rc == same.%s and not h.value, rc
""" % (n_segs, code)
    done = subprocess.run([sys.executable, "-c", run], cwd=ROOT, capture_output=True, text=True)
    assert done.returncode == 0, (done.returncode, done.stderr)


def test_workspaces_are_whole():
    """An expanded workspace has the numbers of bytes, not the memory."""
    p = same.same_cross_create([0, 1], [0, 100_000], 4, 1, 64, torch.bfloat16)
    q, k = torch.zeros(1, 4, 64, dtype=torch.bfloat16), torch.zeros(100_000, 1, 64, dtype=torch.bfloat16)
    need = p.workspace_bytes(True)
    for ws in (torch.zeros(1, dtype=torch.uint8).expand(need), torch.zeros(2 * need, dtype=torch.uint8)[::2]):
        with pytest.raises(same.SameError, match="contiguous"):
            same.same_cross_attention(p, q, k, k, q, None, ws)
        with pytest.raises(same.SameError, match="contiguous"):
            same.same_cross_attention_backward(p, q, k, k, q, None, q, q, k, k, ws)


def test_every_kernel_source_is_checked():
    from paper_1511_06416_amd import build

    sources = sorted(f for f in os.listdir(build.CSRC) if f.endswith(".hip"))
    assert sources == sorted(f for f in build.SOURCES if f.endswith(".hip")) and "kernels.hip" in sources
    for src in sources:
        flags = build.command(src, "x.o")
        assert "-fno-slp-vectorize" in flags and "-Rpass-analysis=kernel-resource-usage" in flags, src
    one = "a.hip:1:1: remark: Function Name: one [-R]\na.hip:1:1: remark:     VGPRs Spill: %d [-R]\n"
    build.check_remarks("a.hip", one % 0)
    for text in (one % 1, "", "a.hip:1:1: remark:     VGPRs Spill: 0 [-R]\n"):
        with pytest.raises(RuntimeError, match="a.hip"):
            build.check_remarks("a.hip", text)
