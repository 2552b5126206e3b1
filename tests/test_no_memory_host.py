"""No C++ exception leaves a C entry: error texts that the host has no memory for."""

import os
import shutil
import subprocess

import pytest

from paper_2306_08881_amd import _lib as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <new>
#include "acp.h"

static bool none = false;  // no more memory from operator new, which the library shares
void* operator new(std::size_t n) {
  void* p = none ? nullptr : std::malloc(n);
  if (!p) throw std::bad_alloc();
  return p;
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }

int main() {
  const int32_t ndims[] = {2};
  const int64_t dims[] = {64, 64};
  int64_t k = 0;
  const float* f = nullptr;
  acp_adamw* opt = nullptr;
  acp_ctx* ctx = nullptr;
  acp_adamw_grad grad = {};
  acp_adamw_hyper hyper = {};
  if (acp_adamw_init(&opt, 1, ndims, dims, 32, nullptr, 0) != ACP_OK) return 2;
  if (acp_init(&ctx, 1, ndims, dims, 4, 0, 1 << 20, 1, ACP_FLAG_REUSE | ACP_FLAG_EF) != ACP_OK) return 2;
  none = true;
  bool ok = true;
  acp_adamw* another = nullptr;
  ok = ok && acp_adamw_init(&another, 1, ndims, dims, 32, nullptr, 0) == ACP_E_STATE && !another;
  ok = ok && acp_adamw_state_bytes(opt, nullptr) == ACP_E_INVALID;
  ok = ok && acp_adamw_tensor_info(opt, 1, &k, nullptr, nullptr, nullptr, nullptr) == ACP_E_INVALID;
  ok = ok && acp_adamw_grads_bytes(opt, &grad, &k) != ACP_OK;
  ok = ok && acp_adamw_bind(opt, reinterpret_cast<void*>(257), 1, nullptr, nullptr, nullptr) != ACP_OK;
  ok = ok && acp_adamw_set_grads(opt, 4, &grad, nullptr, 0, nullptr) != ACP_OK;
  ok = ok && acp_adamw_norm(opt, 4, 1.f, 1.f, nullptr, nullptr) != ACP_OK;
  ok = ok && acp_adamw_step(opt, 4, 1, &hyper, nullptr, nullptr) != ACP_OK;
  ok = ok && acp_advance_all(ctx, 1, nullptr, nullptr) == ACP_E_INVALID;
  ok = ok && acp_advance(ctx, 1, 0, nullptr, nullptr) == ACP_E_STATE;
  ok = ok && acp_factor_address(ctx, 0, 0, 0, &f) == ACP_E_STATE;
  none = false;
  acp_adamw_destroy(opt);
  acp_destroy(ctx);
  std::puts(ok ? "ok" : "wrong status");
  return ok ? 0 : 1;
}
"""


def test_refusals_without_memory(tmp_path):
    if not shutil.which("g++"):
        pytest.skip("no host compiler")
    L.load()  # built
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(PROGRAM)
    lib = os.path.dirname(os.path.abspath(L.__file__))
    subprocess.run(["g++", "-std=c++17", f"-I{ROOT}/include", str(src), "-o", str(exe), f"-L{lib}", "-l:libacp.so",
                    f"-Wl,-rpath,{lib}", "-Wl,--allow-shlib-undefined"], check=True)
    env = dict(os.environ, LD_LIBRARY_PATH="/opt/rocm/lib:" + os.environ.get("LD_LIBRARY_PATH", ""))
    p = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120, env=env)
    assert p.returncode == 0 and p.stdout.strip() == "ok", (p.returncode, p.stdout, p.stderr)
