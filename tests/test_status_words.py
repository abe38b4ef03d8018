"""A status that has been read is cleared: when the call returns, not at some later time.

The entries are linked to a stand-in for the CUDA runtime (no device is needed): work on a stream is queued, and done
when the stream is waited for, the latest that the runtime allows.  Another stream may use the handle as soon as the
call has returned, and what its kernels latch then must not be cleared by work that is still queued."""

import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2608_02703_gb300 import archead
from paper_2608_02703_gb300.build import BUILD, CSRC, INCLUDE, build

RUNTIME = r"""
#include <string.h>
#include <functional>
#include <map>
#include <vector>
#include "int8.h"
#include "internal.h"
#include "loss.h"

static std::map<cudaStream_t, std::vector<std::function<void()>>> queued;
static void finish(cudaStream_t s) {
  for (auto &work : queued[s]) work();
  queued[s].clear();
}

extern "C" {
void **__cudaRegisterFatBinary(void *) { static void *none; return &none; }
void __cudaRegisterFatBinaryEnd(void **) {}
void __cudaUnregisterFatBinary(void **) {}
cudaError_t cudaSetDevice(int) { return cudaSuccess; }
cudaError_t cudaStreamSynchronize(cudaStream_t s) { finish(s); return cudaSuccess; }
cudaError_t cudaMemsetAsync(void *p, int v, size_t n, cudaStream_t s) {
  queued[s].push_back([=] { memset(p, v, n); });
  return cudaSuccess;
}
cudaError_t cudaMemcpyAsync(void *to, const void *from, size_t n, cudaMemcpyKind, cudaStream_t s) {
  queued[s].push_back([=] { memcpy(to, from, n); });
  return cudaSuccess;
}
cudaError_t cudaMemset(void *p, int v, size_t n) { return cudaMemsetAsync(p, v, n, nullptr); }
cudaError_t cudaMemcpy(void *to, const void *from, size_t n, cudaMemcpyKind) {
  finish(nullptr);
  memcpy(to, from, n);
  return cudaSuccess;
}
}

// What a kernel does that latches a bit, queued on a stream.
extern "C" void latch(int *word, int bit, cudaStream_t s) { queued[s].push_back([=] { *word |= bit; }); }
extern "C" void *loss_handle(int *word) { auto *h = new archead_loss(); h->err = word; return h; }
extern "C" void *int8_handle(int *word) { auto *h = new archead_int8_weight(); h->err = word; return h; }
extern "C" void *pack_handle(int *word) { auto *h = new archead_pack(); h->err = word; return h; }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    build()
    where = tmp_path_factory.mktemp("status")
    source, out = where / "runtime.cc", where / "libstatus.so"
    source.write_text(RUNTIME)
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include")
    objects = [os.path.join(BUILD, f"{name}.o") for name in ("api", "int8_api", "loss_api")]
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", f"-I{INCLUDE}", f"-I{CSRC}", f"-I{cuda}", str(source), *objects,
                    "-Wl,-Bsymbolic", "-Wl,-z,lazy", "-o", str(out)], check=True)
    return ctypes.CDLL(str(out), mode=os.RTLD_LAZY)


@pytest.mark.parametrize("kind,entry", [("loss", "archead_loss_sync_status"), ("int8", "archead_int8_sync_status"),
                                        ("pack", "archead_sync_status")])
def test_a_status_is_cleared_when_it_has_been_read(lib, kind, entry):
    word = ctypes.c_int(0)
    make, sync = getattr(lib, kind + "_handle"), getattr(lib, entry)
    make.restype = ctypes.c_void_p
    handle, one, two = ctypes.c_void_p(make(ctypes.byref(word))), ctypes.c_void_p(8), ctypes.c_void_p(16)
    timeout = 1  # the error word's bit of a wait that gave up
    assert sync(handle, one) == archead.OK and word.value == 0
    lib.latch(ctypes.byref(word), timeout, one)
    assert sync(handle, one) == archead.ERR_DEVICE_TIMEOUT
    assert word.value == 0
    # The next call's kernels, on another stream: what they latch is there when that stream is waited for.
    lib.latch(ctypes.byref(word), timeout, two)
    lib.cudaStreamSynchronize(two)
    assert sync(handle, one) == archead.ERR_DEVICE_TIMEOUT  # (whatever was left queued on `one` ran before)
    assert word.value == 0
