"""The status word of the single operations (nnc_op_status)."""
import os
import subprocess
import sys
import textwrap

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def planting_lib(tmp_path_factory):
    """The library with one function more: it stores a code the way a tensor-core kernel does whose wait ran out."""
    from paper_2512_21571_b200 import build
    build.build()
    work = tmp_path_factory.mktemp("status")
    api = os.path.join(build.CSRC, "nnc_api.cu")
    (work / "plant.cu").write_text('#include "%s"\n' % api + textwrap.dedent("""
        static __global__ void plant_kernel(int *status, int code) { atomicExch(status, code); }
        extern "C" int plant(int code, void *stream) {
            LaunchCtx lc;
            if (op_ctx(lc, stream)) return NNC_ERR_CUDA;
            plant_kernel<<<1, 1, 0, lc.stream>>>(lc.status, code);
            return cudaGetLastError() == cudaSuccess ? NNC_OK : NNC_ERR_CUDA;
        }
    """))
    lib = str(work / "libplant.so")
    objects = [s[:-3] + ".o" for s in build.sources() if s != api]
    r = subprocess.run(["nvcc", *build.NVCC_FLAGS, "-I", build.CSRC, "-shared", "-cudart", "static", "-o", lib, str(work / "plant.cu"), *objects],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return lib


def test_the_planting_library_builds(planting_lib):
    assert os.path.getsize(planting_lib)


_CHILD = """
import ctypes as C, sys, torch
sys.path.insert(0, %r)
from paper_2512_21571_b200 import binding as nnc
nnc.lib.plant.argtypes = [C.c_int, C.c_void_p]
cache = nnc.PagedKV.empty(1, 16, 1, 64, torch.bfloat16, 1, 1)      # a table of -1: no page
pos = torch.zeros(1, dtype=torch.int32, device="cuda")
stream = torch.cuda.current_stream().cuda_stream
assert nnc.op_status() == 0
nnc.op_kv_read_paged(cache, pos)
assert nnc.lib.plant(5, stream) == 0
assert nnc.op_status() == 0x105 and nnc.op_status() == 0           # the code leaves the address's bit
assert nnc.lib.plant(7, stream) == 0
nnc.op_attn_decode_paged(torch.zeros(1, 1, 64, dtype=torch.bfloat16, device="cuda"), cache, pos + 1)
assert nnc.op_status() == 0x107 and nnc.op_status() == 0
assert nnc.lib.plant(9, stream) == 0
assert nnc.op_status() == 9
nnc.op_kv_read_paged(cache, pos)
assert nnc.op_status() == 0x100 and nnc.op_status() == 0
print("done")
""" % ROOT


@pytest.mark.gpu
def test_codes_and_the_bit_of_bad_addresses_leave_one_another(planting_lib):
    r = subprocess.run([sys.executable, "-c", _CHILD], capture_output=True, text=True, timeout=300, env={**os.environ, "NNC_LIBRARY": planting_lib})
    assert r.returncode == 0 and "done" in r.stdout, r.stdout + r.stderr


@pytest.mark.gpu
def test_the_status_waits_for_every_stream():
    """Streams that do not synchronise with the default one included."""
    import torch
    from paper_2512_21571_b200 import binding as nnc
    cache = nnc.PagedKV.empty(1, 16, 1, 64, torch.bfloat16, 1, 1)
    pos = torch.zeros(1, dtype=torch.int32, device="cuda")
    nnc.op_kv_read_paged(cache, pos)
    assert nnc.op_status() == 0x100
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)      # some 50 ms
            nnc.op_kv_read_paged(cache, pos)
        assert nnc.op_status() == 0x100
    assert nnc.op_status() == 0
