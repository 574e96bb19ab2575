"""Host side of the attention calls without a device, on a context made by hand: the error of kernels that could not be set up comes
back from the calls (nothing may reach a launch: the error recorded is the one given, not that of a missing device), and the bounds of
the sizes are those that the header states."""
import os
import subprocess

from paper_2603_02883_b200 import fb4

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

HEAD = r"""
#include <stdio.h>
#include <string.h>
#include "fb4_internal.h"

alignas(256) static unsigned char room[1 << 16];

int main() {
  static fb4_ctx ctx;
  fb4_default_config(&ctx.cfg);
  ctx.fast_ok = 1;
  ctx.sm_count = 148;
  fb4_cache cache;
  memset(&cache, 0, sizeof cache);
  cache.k_codes = cache.v_codes = room;
  cache.k_meta = cache.v_meta = reinterpret_cast<uint16_t*>(room);
  cache.n_pages = 1;
  cache.page_tokens = 16;
  cache.n_heads = 1;
  cache.head_dim = 64;
  const int32_t* lens = reinterpret_cast<const int32_t*>(room);
"""

SET_UP = r"""
  const int64_t* slot = reinterpret_cast<const int64_t*>(room);
  ctx.append_error = cudaErrorInvalidValue;
  int rc = fb4_cache_append(&ctx, &cache, slot, room, 64, room, 64, 1, 0, 0.0f, 0, 0, 0, 0, 0, 0, 0, 0);
  if (rc != FB4_ERR_CUDA || fb4_last_cuda_error() != (int)cudaErrorInvalidValue) return 1;
  ctx.attend_error = cudaErrorInvalidConfiguration;
  for (int many = 0; many < 2; ++many) {
    rc = fb4_cache_attention(&ctx, room, 64, 1, 100, &cache, lens, 1, lens, lens, 1, many ? 100 : 1, 16, 0.1f, 1, 0, room, 64, 1, 0, 0, 0, 0);
    if (rc != FB4_ERR_CUDA || fb4_last_cuda_error() != (int)cudaErrorInvalidConfiguration) return 2;
  }
  if (ctx.launches != 0) return 3;
  // arguments are checked first
  if (fb4_cache_attention(&ctx, room, 64, 1, 100, &cache, lens, 1, lens, 0, 1, 1, 16, 0.1f, 1, 0, room, 64, 1, 0, 0, 0, 0) != FB4_ERR_INVALID_ARG) return 4;
  puts("ok");
  return 0;
}
"""


BOUNDS = r"""
  auto size = [&](int q_heads, int n_seqs, int max_q, int max_kv, int window) {
    return fb4_cache_attention_workspace(&ctx, q_heads, 1, 64, n_seqs, max_q, max_kv, window);
  };
  if (size(1, 1, 1 << 30, 16, 0) < 0 || size(1, 1, (1 << 30) + 1, 16, 0) != -1) return 1;
  if (size(1024, 1, 1 << 20, 16, 0) < 0 || size(1024, 1, (1 << 20) + 1, 16, 0) != -1) return 2;
  if (size(1, 1, 1, 1 << 30, 0) < 0 || size(1, 1, 1, (1 << 30) + 1, 0) != -1) return 3;
  if (size(1, 0x7fffffff, 1, 16, 0) < 0 || size(1, 1 << 30, 2, 16, 0) != -1 || size(2, 1 << 30, 1, 16, 0) != -1) return 4;
  if (size(1, 1, 1, 16, 0x7fffffff) < 0 || size(1, 1, 1, 16, -1) != -1) return 5;
  const int too_many[][2] = {{(1 << 30) + 1, 16}, {1, (1 << 30) + 1}};
  for (const auto& b : too_many)
    if (fb4_cache_attention(&ctx, room, 64, 1, 100, &cache, lens, 1, lens, lens, 1, b[0], b[1], 0.1f, 1, 0, room, 64, 1, 0, 0, 0, 0) != FB4_ERR_SHAPE) return 6;
  if (ctx.launches != 0) return 7;
  puts("ok");
  return 0;
}
"""


def run(tmp_path, body):
    fb4.lib()
    libdir = os.path.dirname(fb4.library_path())
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    src, exe = tmp_path / "host.cpp", tmp_path / "host"
    src.write_text(HEAD + body)
    subprocess.check_call(["g++", "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2603_02883_b200", "csrc"),
                           "-I", os.path.join(cuda, "include"), str(src), "-o", str(exe), "-L", libdir, "-lfb4", f"-Wl,-rpath,{libdir}"])
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout == "ok\n", r


def test_kernels_that_could_not_be_set_up_are_an_error(tmp_path):
    run(tmp_path, SET_UP)


def test_bounds_of_the_sizes(tmp_path):
    run(tmp_path, BOUNDS)


def test_the_header_states_every_bound():
    text = open(os.path.join(ROOT, "include", "fb4.h")).read()
    assert "max_kv <= 2^30" in text and "max_q * q_heads <= 2^30" in text and "n_seqs * max_q * q_heads < 2^31" in text
