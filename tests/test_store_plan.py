"""How the K/V store's host side cuts a call, with the CUDA runtime and the launchers replaced by stand-ins: the machine here
has two devices of 148 and 40 multiprocessors.  Needs no GPU."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2306_14048_b200", "csrc")
HERE = 0x10000  # an aligned address nobody reads

FAKE = r"""
struct CUstream_st; struct CUtensorMap_st; struct h2o_store_config_t;
static int current = 0;
extern "C" {
int cudaGetDevice(int* d) { *d = current; return 0; }
int cudaSetDevice(int d) { current = d; return 0; }
int cudaGetDeviceCount(int* n) { *n = 2; return 0; }
int cudaGetLastError() { return 0; }
int cudaDeviceGetAttribute(int* v, int attr, int dev) { *v = attr == 16 ? (dev ? 40 : 148) : 10; return 0; }
void** __cudaRegisterFatBinary(void*) { return 0; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
}
namespace h2o {
struct AttendView;
typedef CUstream_st* S;
bool make_store_map(CUtensorMap_st*, h2o_store_config_t const&, void const*, int) { return true; }
int launch_attend_tc(AttendView const&, int, int, int, void const*, void const*, S) { return 0; }
int launch_attend_fma(AttendView const&, int, int, int, S) { return 0; }
int launch_attend_mma(AttendView const&, int, bool, int const*, int, void const*, void const*, S) { return 0; }
int launch_store_read(h2o_store_config_t const&, void*, void*, int, long, long, long const*, long, S) { return 0; }
int launch_store_write(h2o_store_config_t const&, void const*, void const*, int, long, long, long const*, long, S) { return 0; }
int launch_attend_join(AttendView const&, int, S) { return 0; }
int attend_tc_box_rows(int, int, int) { return 80; }
int attend_fma_row_tile(long rows) { return rows <= 4 ? 4 : 64; }
int attend_mma_row_tile(long rows) { return rows <= 8 ? 8 : rows <= 16 ? 16 : 32; }
int attend_mma_blocks_per_sm(int, int) { return 2; }
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    import __graft_entry__

    __graft_entry__.build()
    from paper_2306_14048_b200 import binding as b

    at = tmp_path_factory.mktemp("plan")
    (at / "fake.cpp").write_text(FAKE)
    nvcc = os.environ.get("NVCC", "nvcc")
    for cmd in ([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"),
                 "-I", CSRC, "-c", os.path.join(CSRC, "store_api.cu"), "-o", str(at / "api.o")],
                ["g++", "-shared", "-fPIC", "-Wl,-Bsymbolic", "-o", str(at / "plan.so"), str(at / "fake.cpp"), str(at / "api.o")]):
        res = subprocess.run(cmd, capture_output=True, text=True)
        assert res.returncode == 0, res.stderr
    so = ctypes.CDLL(str(at / "plan.so"))
    for name in ("h2o_store_create", "h2o_store_destroy", "h2o_cross_scratch_bytes", "h2o_cross_attend", "h2o_prefix_scratch_bytes", "h2o_prefix_attend"):
        getattr(so, name).argtypes, getattr(so, name).restype = getattr(b.lib, name).argtypes, getattr(b.lib, name).restype
    so.binding = b
    return so


def _store(lib, device):
    b = lib.binding
    h = ctypes.c_void_p()
    cfg = b.h2o_store_config_t(n_heads=4, head_dim=128, format=b.H2O_BF16, device=device, rows=200000, k=HERE, v=HERE)
    assert lib.h2o_store_create(ctypes.byref(h), ctypes.byref(cfg)) == 0
    return h


@pytest.mark.parametrize("tokens", [1, 200])
@pytest.mark.parametrize("keys", [100, 3000, 100000])
def test_a_call_is_cut_for_the_stores_device(lib, tokens, keys):
    """Whichever device is current: a thread that asks for the scratch may have another one than the thread that calls."""
    b = lib.binding
    q = b.h2o_queries_t(q=HERE, out=2 * HERE, cu_q=HERE, q_rows=tokens, dtype=b.H2O_BF16, query_group=1, batch=1, max_q=tokens)
    r = b.h2o_ranges_t(HERE, HERE, keys)
    need = {}
    for device in (0, 1):
        h = _store(lib, device)
        for current in (0, 1):
            lib.cudaSetDevice(current)
            need[device, current] = (lib.h2o_cross_scratch_bytes(h, ctypes.byref(q), ctypes.byref(r)),
                                     lib.h2o_prefix_scratch_bytes(h, ctypes.byref(q), ctypes.byref(r), 1, None, 1, ctypes.byref(r)))
            for got, rc in ((need[device, current][0], lib.h2o_cross_attend(h, ctypes.byref(q), ctypes.byref(r), HERE, need[device, 0][0], None)),
                            (need[device, current][1], lib.h2o_prefix_attend(h, ctypes.byref(q), ctypes.byref(r), 1, None, 1, ctypes.byref(r), HERE,
                                                                             need[device, 0][1], None))):
                assert rc == 0
        lib.h2o_store_destroy(h)
        assert need[device, 0] == need[device, 1]
    if keys == 100000:
        assert need[0, 0][0] > need[1, 0][0] > 0  # more blocks, more pieces
