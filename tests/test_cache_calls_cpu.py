"""The order of what bdkv_attention queues in the library's own workspace, without a GPU (tests/cache_calls.cu)."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_33887_gb300", "csrc")
REPLACED = ["cudaGetDevice", "cudaSetDevice", "cudaGetLastError", "cudaDeviceGetAttribute", "cudaStreamIsCapturing",
            "cudaEventCreateWithFlags", "cudaEventDestroy", "cudaEventRecord", "cudaStreamWaitEvent", "cudaMalloc",
            "cudaFree"]


def _nvcc():
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    return None


@pytest.fixture(scope="module")
def queued(tmp_path_factory):
    nvcc = _nvcc()
    if nvcc is None:
        pytest.skip("no CUDA toolkit")
    exe = str(tmp_path_factory.mktemp("calls") / "cache_calls")
    cmd = [nvcc, "-gencode", "arch=compute_103a,code=sm_103a", "-std=c++17", "-O1", "--expt-relaxed-constexpr",
           "-I" + CSRC, "-I" + os.path.join(CSRC, "cache"), "-I" + os.path.join(ROOT, "include")]
    cmd += [f for name in REPLACED for f in ("-Xlinker", "--wrap=" + name)]
    r = subprocess.run(cmd + [os.path.join(ROOT, "tests", "cache_calls.cu"), "-o", exe, "-ldl"], capture_output=True,
                       text=True)
    assert r.returncode == 0, r.stderr

    def run(*calls):
        out = subprocess.run([exe] + ["%d:%d" % c for c in calls], capture_output=True, text=True, check=True).stdout
        return [line.split() for line in out.strip().split("\n")]

    return run


def test_every_call_waits_for_the_one_before(queued):
    """Also on the same handle: a stream that was destroyed may give its handle to the next one while its work still
    runs, and the handle of the per-thread default stream (2) is another stream in every thread."""
    calls = [(2, 4000), (2, 4000), (64, 4000), (64, 4000), (0, 4000), (2, 4000)]
    for i, (line, (st, _)) in enumerate(zip(queued(*calls), calls)):
        first = ["malloc"] if i == 0 else ["wait(%d)" % st]
        assert line == ["0"] + first + ["parts(%d)" % st, "join(%d)" % st, "record(%d)" % st], i


def test_a_larger_workspace_takes_the_place_of_one_that_no_call_uses(queued):
    """cudaFree returns once the device has finished what was queued: no wait is needed behind it."""
    lines = queued((1024, 4000), (1024, 60000), (1088, 4000))
    assert [line[1:-3] for line in lines] == [["malloc"], ["free", "malloc"], ["wait(1088)"]]
    assert all(line[0] == "0" for line in lines)


def test_a_call_in_one_part_leaves_the_workspace_alone(queued):
    assert queued((1024, 100), (1024, 4000), (1088, 100))[::2] == [["0", "parts(1024)"], ["0", "parts(1088)"]]
