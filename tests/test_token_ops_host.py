"""Host side of the token-model calls on a stand-in for the CUDA runtime: shapes of their launches, the order of their
copies, and what they do when the host has no memory.  The stand-in is preloaded into a child process, where it
answers as a B200 would, keeps a record and runs no kernel."""
import os
import subprocess
import sys
import textwrap

import pytest

from paper_1805_10387_b200 import build

RUNTIME = r"""
#include <cuda_runtime.h>
#include <new>
#include <cstdio>
#include <cstdlib>
#include <cstring>
static bool no_memory = false;
static char record[1 << 16];
static unsigned long long at_symbol[8];
static void note(const char* what) { strncat(record, what, sizeof(record) - strlen(record) - 1); }
static cudaError_t launch(dim3 g, dim3 b, size_t smem) {
  char line[128];
  snprintf(line, sizeof line, "launch %u %u %u x %u %zu\n", g.x, g.y, g.z, b.x, smem);
  note(line);
  const bool fits = g.x && g.x <= 2147483647u && g.y && g.y <= 65535 && g.z && g.z <= 65535 && b.x && b.x * b.y * b.z <= 1024;
  return fits && smem <= (227 << 10) ? cudaSuccess : cudaErrorInvalidConfiguration;
}
void* operator new(size_t n) {
  void* p = no_memory ? nullptr : malloc(n ? n : 1);
  if (!p) throw std::bad_alloc();
  return p;
}
void* operator new(size_t n, const std::nothrow_t&) noexcept { return no_memory ? nullptr : malloc(n ? n : 1); }
extern "C" {
void fake_no_memory(int on) { no_memory = on; }
const char* fake_record() { return record; }
void fake_clear() { record[0] = 0; }
cudaError_t cudaGetDevice(int* d) { *d = 0; return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int* v, cudaDeviceAttr a, int) {
  *v = a == cudaDevAttrComputeCapabilityMajor ? 10 : a == cudaDevAttrMultiProcessorCount ? 148 : 0;
  return cudaSuccess;
}
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { note("attribute\n"); return cudaSuccess; }
cudaError_t cudaOccupancyMaxActiveClusters(int* n, const void*, const cudaLaunchConfig_t*) { *n = 16; return cudaSuccess; }
cudaError_t cudaOccupancyMaxActiveBlocksPerMultiprocessor(int* n, const void*, int, size_t) { *n = 2; return cudaSuccess; }
cudaError_t cudaOccupancyMaxActiveBlocksPerMultiprocessorWithFlags(int* n, const void*, int, size_t, unsigned) { *n = 2; return cudaSuccess; }
cudaError_t cudaGetSymbolAddress(void** p, const void*) { *p = at_symbol; return cudaSuccess; }
cudaError_t cudaMalloc(void** p, size_t n) { *p = aligned_alloc(256, (n + 255) / 256 * 256); return cudaSuccess; }
cudaError_t cudaFree(void* p) { free(p); return cudaSuccess; }
cudaError_t cudaMemcpy(void* d, const void* s, size_t n, cudaMemcpyKind) { note("copy\n"); memcpy(d, s, n); return cudaSuccess; }
cudaError_t cudaStreamSynchronize(cudaStream_t) { note("wait\n"); return cudaSuccess; }
cudaError_t cudaDeviceSynchronize() { note("wait\n"); return cudaSuccess; }
cudaError_t cudaLaunchKernel(const void*, dim3 g, dim3 b, void**, size_t smem, cudaStream_t) { return launch(g, b, smem); }
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void*, void**) {
  return launch(c->gridDim, c->blockDim, c->dynamicSmemBytes);
}
}
"""

# The child has the binding's declarations, without torch, and P: an address that no call reads.
CHILD = """
import ctypes as C, sys, types
class Any(types.ModuleType):
    def __getattr__(self, name):
        if name.startswith("__"):
            raise AttributeError(name)
        return Any(name)
sys.modules["torch"] = Any("torch")
sys.path.insert(0, {root!r})
from paper_1805_10387_b200 import mp
fake = C.CDLL({fake!r})
fake.fake_record.restype = C.c_char_p
L = mp.lib()
buf = (C.c_uint8 * 65536)()
P = (C.addressof(buf) + 255) // 256 * 256
def record():
    text = fake.fake_record().decode().split("\\n")[:-1]
    fake.fake_clear()
    return text
def embed_bwd(n, V, D, ld):
    return L.mp_embedding_bwd(P, 8, P, ld, P, ld, n, V, D, -1, 1.0, None, P, 1 << 60, None)
def norm_fwd(M, D, x_bytes=2):
    return L.mp_block_norm_fwd(0, 1e-6, 1.0, P, x_bytes, D, P, D, P, None, 0, P, D, P, P, D, P, M, D, None)
def norm_bwd(M, D, x_bytes=2):
    return L.mp_block_norm_bwd(0, 1.0, P, D, None, 0, P, x_bytes, D, P, D, P, None, 0, P, P, P + 32768, D, P + 4096, D, P, None, 0, P,
                               M, D, None, P, 1 << 40, None)
def loss(N, V):
    cfg = mp.PolicyConfig(0.2, 0.2, 0.0, 1.0)
    ld = -(-V // 8) * 8
    return L.mp_policy_loss(P, ld, P, 8, P, None, P, P, N, V, C.byref(cfg), P, ld, P, P, P, None, None)
def plan(count, bits=32):
    arr = (C.c_void_p * 1)(P)
    out = C.c_void_p()
    s = arr if bits == 8 else None
    return L.mp_adamw_plan_create(1, arr, arr, arr, arr, arr, (C.c_int64 * 1)(count), None, bits, s, s, C.byref(out)), out
def update(p):
    opt = mp.AdamWConfig(1e-3, 0.9, 0.99, 1e-8, 0.0)
    return L.mp_adamw_update(p, P, C.byref(opt), 1, None)
"""


@pytest.fixture(scope="module")
def child(tmp_path_factory):
    build.build()
    at = tmp_path_factory.mktemp("runtime")
    src, fake = at / "fake.cpp", str(at / "libfake.so")
    src.write_text(RUNTIME)
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", "-I/usr/local/cuda/include", str(src), "-o", fake], check=True)
    head = CHILD.format(root=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), fake=fake)

    def run(body):
        env = dict(os.environ, LD_PRELOAD=fake)
        r = subprocess.run([sys.executable, "-c", head + textwrap.dedent(body)], env=env, capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, (r.returncode, r.stdout[-2000:], r.stderr[-2000:])
    return run


def test_the_embedding_gradient_of_very_wide_rows_fits_the_grid(child):
    """Widths up to the documented 2^31 - 9: no dimension of a launch passes what a grid may have."""
    child("""
    for D in (1024, 1 << 24, (1 << 24) + 8, 1 << 27, (1 << 27) + 4096, (1 << 31) - 16):
        for n in (1, 300, 5000, 70000):
            assert embed_bwd(n, 3, D, D) == 0, (D, n, L.mp_last_error())
            lines = record()
            assert sum(l.startswith("launch") for l in lines) in (2, 3), lines
    """)


def test_no_exception_leaves_a_call_on_a_host_without_memory(child):
    """A first call of every kind while the host can allocate nothing: it returns (an error or not), it does not end the process."""
    child("""
    p32, p8 = plan(1000)[1], plan(1000, 8)[1]
    fake.fake_no_memory(1)
    results = [embed_bwd(100, 50, 64, 64), embed_bwd(20000, 50, 64, 64), update(p32), update(p8)]
    results += [norm_fwd(4, D, xb) for D in (64, 512, 1024, 2048, 4096, 8192, 16384) for xb in (2, 4)]
    results += [norm_bwd(4, D, xb) for D in (64, 512, 1024, 2048, 4096, 8192, 16384) for xb in (2, 4)]
    results += [loss(4, V) for V in (29, 600, 20000, 50000, 131072)]
    rc, _ = plan(1000)
    fake.fake_no_memory(0)
    assert results == [0] * len(results), results
    assert rc == mp.MP_ERR_NOMEM
    """)


def test_attributes_and_occupancies_are_asked_once(child):
    child("""
    def asked(call):
        assert call() == 0
        return record().count("attribute")
    for call in (lambda: embed_bwd(100, 50, 64, 64), lambda: norm_fwd(4, 512), lambda: norm_bwd(4, 512), lambda: norm_bwd(4, 16384),
                 lambda: loss(4, 600), lambda: loss(4, 131072)):
        assert asked(call) > 0 and asked(call) == 0
    assert asked(lambda: norm_fwd(4, 1024)) > 0           # another kernel
    assert asked(lambda: norm_fwd(4, 512, 4)) > 0
    """)


def test_a_plan_waits_for_its_table(child):
    """A copy from pageable memory returns when the bytes are staged; a stream that does not wait for the default
    one may read the table at once, so the plan's call waits for the copy itself."""
    child("""
    for bits in (32, 8):
        assert plan(1000, bits)[0] == 0
        assert record() == ["copy", "wait"]
    """)


def test_a_gradient_in_the_place_of_the_norms_input_needs_its_pitch(child):
    """With another pitch a row's gradient would lie over rows that other threads have yet to read."""
    child("""
    def call(dx, ld, M=40, D=64, x_bytes=2):
        return L.mp_block_norm_bwd(0, 1.0, P, 64, None, 0, P + 8192, x_bytes, 64, None, 0, None, None, 0, P, P, dx, ld, None, 0, None,
                                   None, 0, P, M, D, None, P, 1 << 40, None)
    for xb in (2, 4):
        assert call(P + 8192, 64, x_bytes=xb) == 0 and call(P + 16384, 72, x_bytes=xb) == 0
        assert call(P + 8192, 72, x_bytes=xb) == mp.MP_ERR_INVALID_ARG
        assert b"place" in L.mp_last_error()
    """)


def test_the_bounds_of_the_embedding_gradient_are_the_documented_ones(child):
    child("""
    def call(n, V):
        rc = L.mp_embedding_bwd(P, 8, P, 8, P, 8, n, V, 8, -1, 1.0, None, P, 16, None)
        return rc, L.mp_last_error().decode()
    last = 2 ** 31 - 130
    assert call(last, 5)[0] == mp.MP_ERR_NOMEM and mp.mp_embedding_bwd_workspace_bytes(last, 5, 8) > 16 * last
    rc, text = call(last + 1, 5)
    assert rc == mp.MP_ERR_TOO_LARGE and "n must be below 2^31 - 129" in text, text
    assert mp.mp_embedding_bwd_workspace_bytes(last + 1, 5, 8) == 0
    last = 2 ** 31 - 2
    assert call(5, last)[0] == mp.MP_ERR_NOMEM
    rc, text = call(5, last + 1)
    assert rc == mp.MP_ERR_TOO_LARGE and "V below 2^31 - 1" in text, text
    header = " ".join(open({root!r} + "/include/mp.h").read().replace(" * ", " ").split())
    assert "n below 2^31 - 129, V below 2^31 - 1" in header
    """.replace("{root!r}", repr(os.path.dirname(os.path.dirname(os.path.abspath(__file__))))))


def test_the_stream_is_found_without_the_private_functions_of_torch(monkeypatch):
    import importlib.util
    import types
    import torch
    for gone in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
        with monkeypatch.context() as m:
            m.delattr(torch._C, gone, raising=False)
            m.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=1234))
            spec = importlib.util.find_spec("paper_1805_10387_b200.mp")
            fresh = importlib.util.module_from_spec(spec)          # a second copy: the first one keeps its functions
            spec.loader.exec_module(fresh)
            assert fresh._stream() == 1234, gone
