"""Launch geometry of uniprefill_attention, taken from the host side of the library built with a plain C++ compiler."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

import paper_2605_06221_amd as up
from attention_form_cases import FORMS, TYPES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HOST_BUILD = os.path.join(ROOT, "tests", "host_build")
CSRC = os.path.join(ROOT, "paper_2605_06221_amd", "csrc")


@pytest.fixture(scope="module")
def host_lib(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    lib = str(tmp_path_factory.mktemp("host") / "libuniprefill_host.so")
    cmd = [gxx, "-std=c++17", "-O1", "-fPIC", "-shared", "-x", "c++", "-I", HOST_BUILD, "-I", CSRC,
           os.path.join(HOST_BUILD, "attn_form.cpp"), os.path.join(HOST_BUILD, "launch_stubs.cpp"), "-o", lib]
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert res.returncode == 0, res.stdout
    return ctypes.CDLL(lib)


def form(lib, lengths, earlier, hq, hkv, D, f32):
    """(rows of a work-group, whether the keys are cut)"""
    cu = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    ck = np.concatenate([[0], np.cumsum(np.add(lengths, earlier))]).astype(np.int32)
    p = up.make_params(num_seqs=len(lengths), total_tokens=int(cu[-1]), block_size=64, num_q_heads=hq, num_kv_heads=hkv, head_dim=D,
                       qk_dtype=up.UP_F32 if f32 else up.UP_BF16)
    out = (ctypes.c_int32 * 2)()
    assert lib.attn_form(ctypes.byref(p), ctypes.c_void_p(cu.ctypes.data), ctypes.c_void_p(ck.ctypes.data), out) == 0
    return out[0], out[1] > 0


@pytest.mark.parametrize("lengths,earlier,hq,hkv,cut", FORMS)
@pytest.mark.parametrize("D,f32", TYPES)
def test_batches_of_the_gpu_tests_reach_their_form(host_lib, lengths, earlier, hq, hkv, cut, D, f32):
    assert form(host_lib, lengths, earlier, hq, hkv, D, f32) == (256, cut)


@pytest.mark.parametrize("lengths,earlier,hq,hkv,want", [
    ([2048], [0], 32, 8, (128, False)), ([2048], [6000], 32, 8, (256, False)), ([32768], [0], 32, 8, (256, False)),
    ([1], [20000], 8, 1, (128, True)), ([4096, 1], [0, 131072], 32, 8, (256, True)), ([1] * 131072, [0] * 131072, 64, 64, (128, False)),
])
def test_forms_of_ordinary_batches(host_lib, lengths, earlier, hq, hkv, want):
    """Prompts, a chunk after cached tokens, decode rows alone and beside a chunk, more sequences than work-groups of 512 threads."""
    assert form(host_lib, lengths, earlier, hq, hkv, 128, False) == want
