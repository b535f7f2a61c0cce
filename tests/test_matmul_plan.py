"""Which launch mixaq_fp8_matmul asks for (csrc/fp8_gemm.cu over a stand-in for the CUDA runtime).  The parts that a product's k-blocks are
added in decide its last bits, and they are promised to depend on the arguments alone: not on how many SMs a device has, or how many
clusters fit onto its chip."""
import ctypes as C
import os
import random
import subprocess

import pytest

from paper_2507_19131_b200 import build as mq_build

HERE = os.path.dirname(os.path.abspath(__file__))
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")


class Device(C.Structure):
    _fields_ = [("sms", C.c_int), ("clusters", C.c_int * 4)]


class Launch(C.Structure):
    _fields_ = [("kernel", C.c_char * 128), ("grid", C.c_int), ("cluster", C.c_int), ("threads", C.c_int)]


# SMs; clusters of 1, 2, 4, 8 CTAs at once.  The first two are B200s, whose chips differ in the SMs of a GPC; the others parts of one.
DEVICES = [(148, 148, 74, 36, 17), (148, 148, 74, 33, 15), (132, 132, 66, 28, 12), (16, 16, 8, 4, 1)]


@pytest.fixture(scope="module")
def L(tmp_path_factory):
    if not os.path.exists(NVCC):
        pytest.skip("no nvcc")
    out = str(tmp_path_factory.mktemp("plan") / "libplan.so")
    flags = [f for f in mq_build.NVCC_FLAGS if f not in ("-O3", "-lineinfo")]
    subprocess.check_call([NVCC] + flags + ["-cudart", "none", "-Xlinker", "-Bsymbolic", "-o", out, os.path.join(mq_build.CSRC, "fp8_gemm.cu"),
                                            os.path.join(HERE, "host_path", "ask_matmul.cu"), os.path.join(HERE, "host_path", "fake_device.cpp")])
    lib = C.CDLL(out)
    lib.ask_matmul.argtypes = [C.c_long, C.c_long, C.c_long, C.c_int, C.c_long]
    devices = (Device * 8).in_dll(lib, "fake_devices")
    for i, d in enumerate(DEVICES):
        devices[i] = Device(d[0], (C.c_int * 4)(*d[1:]))
    return lib


def ask(L, device, m, n, k, w_rows, offset=0):
    C.c_int.in_dll(L, "fake_device").value = device
    before = C.c_long.in_dll(L, "launches").value
    assert L.ask_matmul(m, n, k, w_rows, offset) == 1 and C.c_long.in_dll(L, "launches").value == before + 1
    p = Launch.in_dll(L, "last_launch")
    return p.kernel, p.cluster, p.grid


SHAPES = [(1, 1, 1), (49, 288, 96), (1, 4096, 4096), (37, 2000, 4090), (2048, 4096, 16384), (8192, 8192, 8192), (1536, 384, 66800), (300, 1000, 1000),
          (256, 4096, 4096), (512, 2048, 2048), (1000, 64, 10000), (5000, 4300, 700), (129, 1030, 8192), (4096, 256, 512)]


@pytest.mark.parametrize("w_rows", [1, 128])
def test_the_parts_of_a_product_do_not_depend_on_the_device(L, w_rows):
    rng = random.Random(5)
    drawn = [tuple(int(2 ** rng.uniform(0, 14)) for _ in range(3)) for _ in range(400)]
    for shape in SHAPES + drawn:
        asked = [ask(L, d, *shape, w_rows, offset) for d in range(len(DEVICES)) for offset in (0, 4096)]
        assert len({(kernel, cluster) for kernel, cluster, _ in asked}) == 1, (shape, asked)


@pytest.mark.parametrize("w_rows", [1, 128])
def test_launches_fit_the_device(L, w_rows):
    """Grids are whole clusters; tiles that are walked over get no more CTAs or pairs than run at once."""
    kinds = set()
    for shape in SHAPES:
        for d, device in enumerate(DEVICES):
            kernel, cluster, grid = ask(L, d, *shape, w_rows)
            assert grid % cluster == 0 and cluster in (1, 2, 4, 8)
            pair = b"ILi256E" in kernel
            assert (cluster == 2) if pair else True
            if pair or cluster == 1:
                assert grid // cluster <= device[2 if pair else 1]
            kinds.add((kernel, cluster))
    assert len(kinds) >= 6                                  # every width, with and without parts
