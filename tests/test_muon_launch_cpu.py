"""The orthogonaliser's C entries on a stand-in for the CUDA runtime (fake_cudart.cpp): what a call
leaves behind when a query or a launch fails, and which device it works on.  No GPU: kernels are
recorded, not run."""
import ctypes
import os
import shutil
import subprocess

import pytest

import paper_1806_08054_b200 as ecq

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_1806_08054_b200", "csrc")
ECQ_ERR_CUDA = 2
P = 1 << 20       # a non-null, aligned stand-in for the address of a vector; no kernel runs on it
NVCC = os.environ.get("NVCC") or shutil.which("nvcc")


@pytest.fixture(scope="module")
def built(tmp_path_factory):
    if not NVCC:
        pytest.skip("no nvcc")
    so = str(tmp_path_factory.mktemp("fake") / "libmuon_fake.so")
    # the kernels are not run: no machine code for them
    subprocess.check_call([NVCC, "-gencode", "arch=compute_100a,code=compute_100a", "-std=c++17", "-O1", "-shared",
                           "-Xcompiler", "-fPIC", "-cudart", "none", "-Xlinker", "-Bsymbolic", "--threads", "0", "-o", so,
                           os.path.join(HERE, "fake_cudart.cpp"),
                           os.path.join(HERE, "fake_kernels.cu"), os.path.join(CSRC, "ecq_muon.cu")])
    return so


@pytest.fixture
def lib(built, tmp_path):
    """A copy of its own for each test: nothing of another's is known to it."""
    L = ctypes.CDLL(shutil.copy(built, str(tmp_path)))
    vp, u32, u64, f32, i32 = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_float, ctypes.c_int
    L.ecq_muon_create.argtypes = [ctypes.POINTER(vp), u32, vp, vp, vp, vp, vp, u32, vp, i32]
    L.ecq_muon_destroy.argtypes = [vp]
    L.ecq_muon_workspace_bytes.argtypes, L.ecq_muon_workspace_bytes.restype = [vp], u64
    L.ecq_muon_set_tiles.argtypes = [vp, i32]
    L.ecq_muon_bind.argtypes = [vp, vp, u64, vp]
    L.ecq_muon_orthogonalize.argtypes = [vp, vp, i32, vp, i32, vp]
    L.ecq_muon_step.argtypes = [vp, vp, vp, f32, i32, f32, f32, vp, vp, i32, vp]
    L.ecq_muon_status.argtypes = [vp, vp]
    L.fake_fail.argtypes = [ctypes.c_char_p, i32]
    L.fake_events.restype = ctypes.c_char_p
    L.fake_device.restype = i32
    L.cudaSetDevice.argtypes = [i32]
    return L


class Plan:
    def __init__(self, L, rows, cols, count=1, precision=0, bind=True):
        self.L = L
        self.h = ctypes.c_void_p()
        size = rows * cols
        assert L.ecq_muon_create(ctypes.byref(self.h), count, (ctypes.c_uint64 * count)(*[i * size for i in range(count)]),
                                 (ctypes.c_uint32 * count)(*[rows] * count), (ctypes.c_uint32 * count)(*[cols] * count),
                                 None, None, 5, None, precision) == ecq.ECQ_OK
        if bind:
            assert self.bind() == ecq.ECQ_OK
        L.fake_events()

    def bind(self):
        return self.L.ecq_muon_bind(self.h, P, self.L.ecq_muon_workspace_bytes(self.h), None)

    def step(self):
        return self.L.ecq_muon_step(self.h, P, 2 * P, 0.9, 1, 0.1, 0.0, 3 * P, None, 0, None)

    def events(self):
        return self.L.fake_events().decode().split()

    def close(self):
        self.L.fake_fail(b"", -1)
        self.L.ecq_muon_destroy(self.h)


SMALL, LARGE = (96, 160, 1), (1024, 1024, 8)      # one launch in front of the products, and two


@pytest.mark.parametrize("size,ahead", [(SMALL, 1), (LARGE, 2)])
def test_a_call_that_succeeds(lib, size, ahead):
    p = Plan(lib, *size)
    for _ in range(2):
        assert p.step() == ecq.ECQ_OK
        assert p.events() == ["prepare"] * ahead + ["iterate"]
    p.close()


@pytest.mark.parametrize("call,size", [("attribute", (128, 128, 1)), ("attribute", (1024, 4096, 1)), ("occupancy", (1024, 2048, 8)),
                                       ("occupancy", (2497, 85, 1))])
def test_a_query_that_fails_launches_nothing_and_is_asked_again(lib, call, size):
    p = Plan(lib, *size)
    lib.fake_fail(call.encode(), 0)
    assert p.step() == ECQ_ERR_CUDA and p.events() == []
    assert p.step() == ecq.ECQ_OK and p.events()[-1] == "iterate"
    p.close()


@pytest.mark.parametrize("size,call,skip", [(SMALL, "iterate", 0), (LARGE, "iterate", 0), (LARGE, "prepare", 1), (SMALL, "prepare", 0)])
def test_a_launch_that_fails_leaves_no_counts_to_the_next_call(lib, size, call, skip):
    """The counts of the launches that did happen would send the next call's beyond their lists."""
    p = Plan(lib, *size)
    assert p.step() == ecq.ECQ_OK
    p.events()
    lib.fake_fail(call.encode(), skip)
    assert p.step() == ECQ_ERR_CUDA
    assert "iterate" not in p.events()
    assert p.step() == ecq.ECQ_OK
    after = p.events()
    assert "stale" not in after and after[0] == "memset" and after[-1] == "iterate"
    assert p.step() == ecq.ECQ_OK
    assert p.events()[0] == "prepare"                       # and only once
    p.close()


def test_a_reset_that_fails_is_tried_again(lib):
    p = Plan(lib, *SMALL)
    lib.fake_fail(b"iterate", 0)
    assert p.step() == ECQ_ERR_CUDA
    p.events()
    lib.fake_fail(b"memset", 0)
    assert p.step() == ECQ_ERR_CUDA and p.events() == []
    assert p.step() == ecq.ECQ_OK and p.events()[:2] == ["memset", "prepare"]
    p.close()


def test_a_plan_stays_on_its_device(lib):
    """Binding and tile choices leave the caller's device as it is; with another one than the plan's
    current, calls are refused."""
    lib.cudaSetDevice(3)
    p = Plan(lib, *SMALL, bind=False)
    lib.cudaSetDevice(1)
    assert p.bind() == ecq.ECQ_OK and lib.fake_device() == 1
    assert lib.ecq_muon_set_tiles(p.h, ecq.ECQ_MUON_TILES_128X128) == ecq.ECQ_OK and lib.fake_device() == 1
    assert p.step() == ecq.ECQ_ERR_ARG
    assert lib.ecq_muon_orthogonalize(p.h, P, 0, 2 * P, 0, None) == ecq.ECQ_ERR_ARG
    assert lib.ecq_muon_status(p.h, None) == ecq.ECQ_ERR_ARG
    assert p.events() == []
    lib.cudaSetDevice(3)
    assert p.step() == ecq.ECQ_OK and lib.ecq_muon_status(p.h, None) == ecq.ECQ_OK
    p.close()
