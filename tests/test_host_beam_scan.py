"""The scan of a beam selection without a GPU, built for the host as in test_host_beam_join: what it leaves is what that file makes, and of a row that is finished nothing is
looked at (its logits are pages that nobody may read)."""
import os
import struct
import subprocess

import numpy as np
import pytest
import torch

from paper_2407_20272_amd import build
from test_host_beam_join import RUNTIME, gen, join_source, scanned

PROGRAM = r"""
#include <sys/mman.h>
#include <ucontext.h>
#include <vector>
#include "join_source.h"

namespace emu {
struct Lane { ucontext_t c; dim3 id; bool at_barrier, over; };
static Lane lanes[1024];
static ucontext_t here;
static unsigned long long slots[16][2][64];
static unsigned turn[1024];
static int cur;
dim3* tid;
int outside;
static ee::BeamArgs args;
static void (*kernel)(ee::BeamArgs);
static void leave() { swapcontext(&lanes[cur].c, &here); }
int lane() { return cur & 63; }
unsigned long long exchange(unsigned long long v, int l) {
  const int t = cur, wave = t >> 6, set = turn[t]++ & 1;
  slots[wave][set][t & 63] = v;
  leave();
  return slots[wave][set][l];
}
unsigned long long ballot(bool x) {
  const int t = cur, wave = t >> 6, set = turn[t]++ & 1;
  slots[wave][set][t & 63] = x;
  leave();
  unsigned long long bits = 0;
  for (int l = 0; l < 64; ++l) bits |= slots[wave][set][l] << l;
  return bits;
}
void meet() { lanes[cur].at_barrier = true; leave(); }
static void body() { kernel(args); lanes[cur].over = true; leave(); }
static void workgroup(int threads) {
  static std::vector<char> stacks(1024 * 65536);
  for (int t = 0; t < threads; ++t) {
    lanes[t] = Lane{};
    lanes[t].id = {(unsigned)t, 0, 0};
    turn[t] = 0;
    getcontext(&lanes[t].c);
    lanes[t].c.uc_stack.ss_sp = &stacks[(size_t)t * 65536];
    lanes[t].c.uc_stack.ss_size = 65536;
    lanes[t].c.uc_link = nullptr;
    makecontext(&lanes[t].c, body, 0);
  }
  for (;;) {
    bool any = false;
    for (int w = 0; w < threads / 64; ++w)
      for (bool again = true; again;) {
        again = false;
        for (int l = 0; l < 64; ++l) {
          cur = w * 64 + l;
          if (lanes[cur].at_barrier || lanes[cur].over) continue;
          tid = &lanes[cur].id;
          swapcontext(&here, &lanes[cur].c);
          again = true;
        }
      }
    for (int t = 0; t < threads; ++t)
      if (!lanes[t].over) lanes[t].at_barrier = false, any = true;
    if (!any) return;
  }
}
}

int main(int argc, char** argv) {                                // file, bf16, threads, each, beams, vocab, n_out, chunks, bytes in front of a row
  const int bf16 = atoi(argv[2]), threads = atoi(argv[3]), each = atoi(argv[4]), beams = atoi(argv[5]), vocab = atoi(argv[6]), n = atoi(argv[7]), chunks = atoi(argv[8]);
  const int off = atoi(argv[9]), size = bf16 ? 2 : 4;
  FILE* f = fopen(argv[1], "rb");
  std::vector<int32_t> finished(beams);
  if (fread(finished.data(), 4, beams, f) != (size_t)beams) exit(2);
  const size_t stride = ((size_t)vocab * size + off + 4095) / 4096 * 4096;
  char* z = (char*)mmap(0, stride * beams, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0);
  for (int b = 0; b < beams; ++b) {
    if (fread(z + b * stride + off, size, vocab, f) != (size_t)vocab) exit(2);
    if (finished[b]) mprotect(z + b * stride, stride, PROT_NONE);
  }
  std::vector<double2> stats((size_t)beams * chunks, double2{-7, -7});
  std::vector<uint64_t> found((size_t)n * beams * chunks, 7);
  ee::BeamArgs a{};
  a.logits = z + off, a.stride = stride / size, a.groups = 1, a.beams = beams, a.vocab = vocab, a.n_out = n, a.chunks = chunks, a.threads = threads, a.each = each;
  a.finished = finished.data(), a.stats = stats.data(), a.found = found.data();
  emu::args = a;
  emu::kernel = threads == 1024 ? bf16 ? ee::beam_scan_kernel<ee::bf16_t, 1024, 16> : ee::beam_scan_kernel<float, 1024, 16>
                : each == 32    ? bf16 ? ee::beam_scan_kernel<ee::bf16_t, 256, 32> : ee::beam_scan_kernel<float, 256, 32>
                                : bf16 ? ee::beam_scan_kernel<ee::bf16_t, 256, 16> : ee::beam_scan_kernel<float, 256, 16>;
  for (unsigned row = 0; row < (unsigned)beams; ++row)
    for (unsigned c = 0; c < (unsigned)chunks; ++c) blockIdx = {c, row, 0}, emu::workgroup(threads);
  fwrite(stats.data(), sizeof(double2), stats.size(), stdout);
  fwrite(found.data(), 8, found.size(), stdout);
  fflush(stdout);
  _Exit(emu::outside ? 3 : 0);
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("host_beam_scan")
    (d / "hip").mkdir()
    (d / "hip" / "hip_runtime.h").write_text(RUNTIME)
    (d / "join_source.h").write_text(join_source())
    (d / "program.cpp").write_text(PROGRAM)
    clang = os.path.join(os.path.dirname(os.path.realpath(build._hipcc())), "..", "llvm", "bin", "clang++")
    subprocess.run([clang if os.path.exists(clang) else "/opt/rocm/llvm/bin/clang++", "-x", "c++", "-std=c++17", "-O1", "-Wno-everything", "-I" + str(d),
                    "-I" + os.path.join(build.ROOT, "include"), "-I" + build.CSRC, str(d / "program.cpp"), "-o", str(d / "program")],
                   check=True, capture_output=True, text=True)
    return str(d / "program")


@pytest.mark.parametrize("threads,each,n", [(256, 16, 4), (256, 32, 20), (1024, 16, 128)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab,off", [(2048, 0), (20000, 0), (9001, 0), (20000, 4)])
def test_a_finished_row_is_not_looked_at(program, tmp_path, threads, each, n, dtype, vocab, off):
    beams, bf16 = 3, dtype is torch.bfloat16
    logits = (torch.randn((beams, vocab), generator=gen(vocab)) * 3).to(dtype)
    finished = np.array([0, 1, 0], dtype=np.int32)
    raw = (logits.view(torch.int16) if bf16 else logits).numpy()
    with open(tmp_path / "in", "wb") as f:
        f.write(finished.tobytes() + raw.tobytes())
    chunks, stats, found = scanned(logits.float(), n, threads * each)
    out = subprocess.run([program, str(tmp_path / "in"), *map(str, (int(bf16), threads, each, beams, vocab, n, chunks, off))], capture_output=True, timeout=300)
    assert out.returncode == 0, (out.returncode, out.stderr)      # (-11: a page of the finished row)
    got = np.frombuffer(out.stdout[:stats.nbytes], dtype=np.float64).reshape(stats.shape)
    # a thread adds `each` exponentials (off by 2^-22 of themselves) in float: 2^-22 + each 2^-24 of the sum
    assert (got[[0, 2], :, 0] == stats[[0, 2], :, 0]).all() and (abs(got[[0, 2], :, 1] / stats[[0, 2], :, 1] - 1) <= 2.0 ** -22 + each * 2.0 ** -23).all()
    got = np.frombuffer(out.stdout[stats.nbytes:], dtype=np.uint64).reshape(n, beams, chunks)
    there = found.reshape(n, beams, chunks) if len(found) == n else np.concatenate([found, np.zeros((n - len(found), beams, chunks), np.uint64)])
    there = np.where(there >> np.uint64(32), there, 0)
    assert (got[:, [0, 2]] == there[:, [0, 2]]).all()
