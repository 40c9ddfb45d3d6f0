"""Refusals of a training step's operators at the C entries: found before
anything is enqueued, so no device is needed."""
import ctypes as C
import re
import subprocess

import numpy as np
import pytest
import torch

import paper_1511_06416_amd as same
from paper_1511_06416_amd import build

A = 1 << 20   # an address that is never read
OK = same.SAME_OK


@pytest.fixture(scope="module")
def lib():
    return same.load_library()


NORM = dict(dtype=same.SAME_BF16, head_dim=64, q=A, q_row=128, q_head=64, q_tokens=0, heads_q=2, q_weight=None,
            q_positions=None, k=A, k_row=64, k_head=64, k_tokens=0, heads_kv=1, k_weight=None, k_positions=None, eps=1e-6,
            rot_dim=0, angles=None)


def norm_rc(lib, backward=False, **kw):
    a = dict(NORM, **kw)
    a["angles"] = None if a["angles"] is None else a["angles"].ctypes.data
    if backward:
        return lib.same_qk_norm_backward(*a.values(), A << 8, 128, 64, A << 9, 64, 64, A << 10, A << 11, None, None, None, None)
    return lib.same_qk_norm(*a.values(), A << 8, A << 9, None)


@pytest.mark.parametrize("code,kw", [
    (same.SAME_EINVAL, dict(dtype=3)),
    (same.SAME_EINVAL, dict(head_dim=0)), (same.SAME_EINVAL, dict(head_dim=136)), (same.SAME_EINVAL, dict(head_dim=12)),
    (same.SAME_EINVAL, dict(eps=0.0)), (same.SAME_EINVAL, dict(eps=1e-46)), (same.SAME_EINVAL, dict(eps=float("inf"))),
    (same.SAME_EINVAL, dict(rot_dim=-2)), (same.SAME_EINVAL, dict(rot_dim=7)), (same.SAME_EINVAL, dict(rot_dim=66)),
    (same.SAME_EINVAL, dict(rot_dim=8)),
    (same.SAME_EINVAL, dict(rot_dim=2, angles=np.array([np.inf]))),
    (same.SAME_EINVAL, dict(rot_dim=2, angles=np.array([-1.1e12]))),
    (same.SAME_EINVAL, dict(rot_dim=2, angles=np.array([1.0]), q_tokens=1)),
    (same.SAME_EINVAL, dict(q_tokens=-1)), (same.SAME_EINVAL, dict(heads_kv=0)), (same.SAME_ESIZE, dict(heads_q=65537)),
    (same.SAME_ESIZE, dict(q_tokens=1 << 40)), (same.SAME_ESIZE, dict(q_tokens=1 << 39, q_row=1 << 40)),
    (same.SAME_EINVAL, dict(q=None, q_tokens=1)), (same.SAME_EALIGN, dict(q=A + 2, q_tokens=1)),
    (same.SAME_EALIGN, dict(k_row=60, k_tokens=2)), (same.SAME_EINVAL, dict(q_head=-8, q_tokens=1)),
    (same.SAME_EALIGN, dict(q_weight=A + 1)),
])
def test_norm_refusals(lib, code, kw):
    assert norm_rc(lib, **kw) == code and same.same_last_error()
    assert norm_rc(lib, True, **kw) == code


def test_norm_overlaps(lib):
    n = dict(q_tokens=4, k_tokens=4)
    assert norm_rc(lib, q=A << 8, q_row=136, **n) == same.SAME_EINVAL     # out over strided q
    assert norm_rc(lib, k=A << 8, **n) == same.SAME_EINVAL                # q_out over k
    assert norm_rc(lib, q_weight=A << 8, **n) == same.SAME_EINVAL
    assert norm_rc(lib, True, q=A << 10, **n) == same.SAME_EINVAL         # dq over q
    assert norm_rc(lib) == OK and norm_rc(lib, True) == OK                # no tokens


def probs_rc(lib, **kw):
    a = dict(dict(dtype=same.SAME_F32, logits=A, row_stride=10, rows=4, cols=10, counts=None, targets=A << 3,
                  log_probs=A << 4, sums=None, entropy=None, n_top=0, top_ids=None, top_log_probs=None, workspace=None), **kw)
    return lib.same_log_probs(*a.values(), None)


@pytest.mark.parametrize("code,kw", [
    (same.SAME_EINVAL, dict(dtype=7)), (same.SAME_EINVAL, dict(rows=-1)), (same.SAME_EINVAL, dict(cols=-1)),
    (same.SAME_ESIZE, dict(cols=(1 << 21) + 1)), (same.SAME_ESIZE, dict(rows=1 << 40)),
    (same.SAME_ESIZE, dict(rows=1 << 30, row_stride=1 << 40)),
    (same.SAME_EINVAL, dict(logits=None)), (same.SAME_EALIGN, dict(logits=A + 1)), (same.SAME_EINVAL, dict(row_stride=-1)),
    (same.SAME_EINVAL, dict(n_top=65)), (same.SAME_EINVAL, dict(n_top=-1)), (same.SAME_EINVAL, dict(n_top=1)),
    (same.SAME_EINVAL, dict(targets=None)), (same.SAME_EALIGN, dict(sums=A + 4)),
    (same.SAME_EINVAL, dict(log_probs=A)), (same.SAME_EINVAL, dict(entropy=A << 4)),
    (same.SAME_EINVAL, dict(cols=1 << 20, row_stride=1 << 20, rows=1, targets=A << 12, log_probs=A << 13)),
    (same.SAME_EALIGN, dict(cols=1 << 20, row_stride=1 << 20, rows=1, targets=A << 12, log_probs=A << 13,
                            workspace=(A << 10) + 128)),
])
def test_log_probs_refusals(lib, code, kw):
    assert probs_rc(lib, **kw) == code and same.same_last_error()


@pytest.mark.parametrize("code,kw", [
    (same.SAME_EINVAL, dict(sums=None)), (same.SAME_EINVAL, dict(targets=None)), (same.SAME_EINVAL, dict(dentropy=A << 7)),
    (same.SAME_EINVAL, dict(dlogits=A + 40)), (same.SAME_EINVAL, dict(dlogits_row=9)), (same.SAME_EINVAL, dict(dlogits=None)),
    (same.SAME_EINVAL, dict(dlogits=A, row_stride=12)), (same.SAME_EINVAL, dict(dlogits=A << 4)),
    (same.SAME_EALIGN, dict(dlog_probs=(A << 5) + 2)), (same.SAME_ESIZE, dict(cols=1 << 22)),
])
def test_log_probs_gradient_refusals(lib, code, kw):
    a = dict(dict(dtype=same.SAME_F32, logits=A, row_stride=10, rows=4, cols=10, counts=None, targets=A << 3, sums=A << 4,
                  entropy=None, dlog_probs=A << 5, dentropy=None, dlogits=A << 6, dlogits_row=10), **kw)
    assert lib.same_log_probs_backward(*a.values(), None) == code and same.same_last_error()


def test_nothing_to_do(lib):
    assert probs_rc(lib, rows=0) == OK
    a = (same.SAME_F16, None, 0, 0, 5, None, None, None, None, None, None, None, 5, None)
    assert lib.same_log_probs_backward(*a) == OK


def ortho_rc(lib, **kw):
    coefs = np.ascontiguousarray(kw.pop("coefs", same.NEWTON_SCHULZ), dtype=np.float64)
    a = dict(dict(dtype=same.SAME_F32, g=A, g_mat=21000, g_row=150, n_mats=2, rows=140, cols=150, coefs=coefs.ctypes.data,
                  steps=len(coefs), eps=1e-7, scale=1.0, out=A << 1, out_mat=21000, out_row=150, workspace=A << 2), **kw)
    return lib.same_orthogonalise(*a.values(), None)


@pytest.mark.parametrize("code,kw", [
    (same.SAME_EINVAL, dict(dtype=-1)), (same.SAME_EINVAL, dict(rows=-1)), (same.SAME_EINVAL, dict(n_mats=-1)),
    (same.SAME_ESIZE, dict(rows=1 << 16, cols=1 << 16)), (same.SAME_ESIZE, dict(rows=1, cols=1 << 25)),
    (same.SAME_ESIZE, dict(n_mats=1 << 40)), (same.SAME_EINVAL, dict(coefs=[(30.0, 0.0, 0.0)])),
    (same.SAME_EINVAL, dict(coefs=[(1.0, 0.0, 20.0)])), (same.SAME_EINVAL, dict(coefs=[(np.nan, 0.0, 0.0)])),
    (same.SAME_EINVAL, dict(coefs=[(0.0, 0.0, 0.0), (0.5, 1e39, 0.0)])), (same.SAME_ESIZE, dict(out_row=1 << 62)),
    (same.SAME_EINVAL, dict(coefs=[(3.0, 0.0, 0.0)] * 3)), (same.SAME_EINVAL, dict(steps=0)), (same.SAME_EINVAL, dict(steps=33)),
    (same.SAME_EINVAL, dict(eps=0.0)), (same.SAME_EINVAL, dict(eps=np.inf)), (same.SAME_EINVAL, dict(scale=1e39)),
    (same.SAME_EINVAL, dict(g=None)), (same.SAME_EINVAL, dict(out=None)), (same.SAME_EALIGN, dict(g=A + 2)),
    (same.SAME_EINVAL, dict(g_row=-1)), (same.SAME_EINVAL, dict(out_row=149)), (same.SAME_EINVAL, dict(out_mat=20999)),
    (same.SAME_ESIZE, dict(g_mat=1 << 61)), (same.SAME_EINVAL, dict(workspace=None)), (same.SAME_EALIGN, dict(workspace=A + 64)),
    (same.SAME_EINVAL, dict(out=A + 4)), (same.SAME_EINVAL, dict(workspace=A)), (same.SAME_EINVAL, dict(out=A << 2)),
    (same.SAME_EINVAL, dict(out=A, workspace=A)),
])
def test_orthogonalise_refusals(lib, code, kw):
    assert ortho_rc(lib, **kw) == code and same.same_last_error()


def test_orthogonalise_nothing_to_do(lib):
    for kw in (dict(n_mats=0), dict(rows=0), dict(cols=0)):
        assert ortho_rc(lib, **kw) == OK


def test_workspace_sizes():
    assert same.same_log_probs_workspace_size(1000, 64, 20) == 0
    assert same.same_log_probs_workspace_size(3, 1 << 21, 20) >= 3 * 64 * (12 + 20 * 8)
    assert same.same_qk_norm_workspace_size(64, 0, 1, 0, 1) == 0
    assert 4 * 64 <= same.same_qk_norm_workspace_size(64, 1 << 30, 8, 1, 1) <= 1 << 21
    assert same.same_orthogonalise_workspace_size(0, 5, 5, torch.float32) == 0
    # many matrices share their planes; those that a block holds need none
    few, many = (same.same_orthogonalise_workspace_size(n, 200, 300, torch.float32) for n in (1 << 14, 1 << 20))
    assert 0 < few == many
    for rows, cols in ((32, 1023), (256, 64), (96, 256), (128, 128)):
        assert same.same_orthogonalise_workspace_size(1 << 20, rows, cols, torch.float32) == 0
    for call, args in ((same.same_log_probs_workspace_size, (-1, 5, 0)), (same.same_log_probs_workspace_size, (1, 5, 65)),
                       (same.same_qk_norm_workspace_size, (12, 1, 1, 1, 1)),
                       (same.same_orthogonalise_workspace_size, (1, -1, 1, torch.float32))):
        with pytest.raises(same.SameError):
            call(*args)


def test_host_tensors_are_refused():
    x = torch.zeros(4, 2, 8, dtype=torch.float16)
    with pytest.raises(same.SameError, match="device"):
        same.same_qk_norm(x, x, x, x)
    with pytest.raises(same.SameError, match="device"):
        same.same_log_probs(x[0], None, None, None)
    with pytest.raises(same.SameError, match="device"):
        same.same_orthogonalise(x, x, None)


def test_shares_of_heads(tmp_path):
    """Every head of a token is in one share, and none is empty: a wave reads its share's first head."""
    source, lib = tmp_path / "shares.cpp", tmp_path / "shares.so"
    source.write_text('''#include "norm_shares.hpp"
extern "C" int wrong(int heads, int split) {
    const same::NormShares s = same::norm_shares(heads, split);
    return s.cut < 1 || s.cut > split || (s.cut - 1) * s.part >= heads || s.cut * s.part < heads;
}
''')
    subprocess.check_call(["g++", "-std=c++17", "-shared", "-fPIC", "-I", build.CSRC, "-o", str(lib), str(source)])
    wrong = C.CDLL(str(lib)).wrong
    for heads in list(range(1, 140)) + [4096, 65535, 65536]:
        for split in list(range(1, 140)) + [4096]:
            assert not wrong(heads, split), (heads, split)


def closest_read(listing):
    """The fewest wait states from a 64-bit matrix product to an instruction that reads its result
    as no sum, over every path of a listing's kernels."""
    def registers(operand):
        m = re.match(r"-?\|?([av])\[(\d+):(\d+)\]|-?\|?([av])(\d+)\b", operand)
        if not m:
            return set()
        if m[1]:
            return {(m[1], i) for i in range(int(m[2]), int(m[3]) + 1)}
        return {(m[4], int(m[5]))}

    least, products = 99, 0
    for body in re.findall(r"^_ZN\S*kernel\S*:.*?\n(.*?)s_endpgm", listing, re.M | re.S):
        lines = [line.split(";")[0].split() for line in body.split("\n")]
        lines = [[x.strip(",") for x in line] for line in lines if line and not (line[0].startswith(".") and ":" not in line[0])]
        labels = {line[0][:-1]: i for i, line in enumerate(lines) if line[0].endswith(":")}
        for start, line in enumerate(lines):
            if not line[0].startswith("v_mfma_f64"):
                continue
            products += 1
            result, paths, seen = registers(line[1]), [(start + 1, 0)], {}
            while paths:
                at, states = paths.pop()
                while at < len(lines) and states < least and seen.get(at, 99) > states:
                    seen[at] = states
                    op, *args = lines[at]
                    at += 1
                    if op.endswith(":"):
                        continue
                    if op.startswith("v_mfma"):
                        if any(registers(a) & result for a in args[1:3]):
                            least = states
                        if registers(args[0]) & result:
                            break   # its own sum goes on: that product is looked at by itself
                        states += 16 if "f64" in op else 4
                        continue
                    reads = args[1:] if op.startswith("v_") else args if op.startswith(("ds_write", "global_store", "buffer_store")) else []
                    if any(registers(a) & result for a in reads):
                        least = states
                    if op == "s_branch":
                        at, states = labels[args[0]], states + 1
                        continue
                    if op.startswith("s_cbranch"):
                        paths.append((labels[args[0]], states + 1))
                    states += int(args[0]) + 1 if op == "s_nop" else 1
    return least, products


def test_results_of_64_bit_products_are_waited_for(tmp_path):
    """A compiler has read such a result behind a branch too few wait states after its product, and
    a step of a small update was lost without an error: it takes 18 of them to be there."""
    listing = tmp_path / "small.s"
    command = build.command("ortho_small.hip", str(listing))
    at = command.index("-c")
    subprocess.check_call(command[:at] + ["--cuda-device-only", "-S"] + command[at + 1:], stderr=subprocess.DEVNULL)
    least, products = closest_read(listing.read_text())
    assert products >= 34 and least >= 18, (products, least)   # of 34 kernels, each with one at least


def test_reads_behind_branches_are_found():
    kernel = "_ZN4same6kernelE:\n v_mfma_f64_16x16x4_f64 v[0:7], v[8:9], v[10:11], 0\n %s\n s_endpgm\n"
    assert closest_read(kernel % "s_nop 15\n s_nop 1\n v_add_f64 v[8:9], v[2:3], v[2:3]")[0] == 18
    assert closest_read(kernel % "s_cbranch_scc1 .LBB0_2\n s_nop 15\n s_nop 3\n.LBB0_2:\n s_nop 4\n ds_write_b64 v20, v[6:7]")[0] == 6
    assert closest_read(kernel % "v_mfma_f64_16x16x4_f64 v[0:7], v[12:13], v[14:15], v[0:7]\n s_nop 6\n v_mov_b32 v9, v0")[0] == 7
