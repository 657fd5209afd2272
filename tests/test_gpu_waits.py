"""The bounded waits of tree attention's warps: how long one lasts on a barrier that nothing completes."""
import ctypes
import os
import subprocess

import pytest
import torch

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))
LIMIT = 1_000_000_000          # ns of a wait on which nothing comes; what 128 polls and a block's start take comes on top


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("probe") / "wait_probe.so")
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-DGVA_WITH_MMA", "-shared", "-Xcompiler", "-fPIC",
                    "-I", os.path.join(HERE, "..", "paper_2609_13285_b200", "csrc"), os.path.join(HERE, "wait_probe.cu"), "-o", lib], check=True)
    f = ctypes.CDLL(lib).wait_probe
    f.argtypes = [ctypes.c_int, ctypes.c_int] + [ctypes.c_void_p] * 3

    def run(mode, flag):
        result, elapsed = torch.full((32,), 7, dtype=torch.int32, device="cuda"), torch.zeros(32, dtype=torch.int64, device="cuda")
        assert f(mode, flag, result.data_ptr(), elapsed.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        return set(result.tolist()), min(elapsed.tolist()), max(elapsed.tolist())
    return run


def test_a_complete_phase_is_seen_at_once(probe):
    for flag in (0, 1):
        said, _, most = probe(0, flag)
        assert said == {1} and most < LIMIT // 100


@pytest.mark.parametrize("mode", [1, 2, 3])
def test_a_wait_on_nothing_ends_after_its_time(probe, mode):
    said, least, most = probe(mode, 0)
    assert said == {0} and LIMIT <= least and most < 3 * LIMIT


@pytest.mark.parametrize("mode", [1, 2])
def test_a_wait_ends_early_where_another_warp_has_given_up(probe, mode):
    said, _, most = probe(mode, 1)
    assert said == {0} and most < LIMIT
