"""How dllm_adapters finds a tile's rows among 32 neighbours (up to 64 rows), by the kernels' own tile_of, run on the CPU:
64 threads in the place of a wave's lanes, the wave's instructions as functions in which they meet (CPU only)."""
import os
import subprocess

import pytest

from paper_2608_22646_amd import build

PROGRAM = r"""
#include <pthread.h>
#include <cstdio>
#include <thread>
#include <vector>
#include <hip/hip_runtime.h>
#undef __device__
#define __device__ __attribute__((host)) __attribute__((device))
#define __builtin_amdgcn_readlane host_readlane
#define __builtin_amdgcn_readfirstlane host_readfirstlane
static pthread_barrier_t meet;
static int lanes[64];
static unsigned long long votes;
// every lane's value is there between the two meetings
static int host_readlane(int x, int lane);
static int host_readfirstlane(int x);
struct Here { unsigned x; };
static thread_local Here here;
#define threadIdx here
__attribute__((host)) unsigned long long __ballot(int);
__attribute__((host)) void __syncthreads();
__attribute__((host)) int __popcll(unsigned long long x) { return __builtin_popcountll(x); }
__attribute__((host)) int __ffsll(unsigned long long x) { return __builtin_ffsll((long long)x); }
#include "%s"
static int host_readlane(int x, int lane) {
  lanes[here.x] = x;
  pthread_barrier_wait(&meet);
  const int r = lanes[lane];
  pthread_barrier_wait(&meet);
  return r;
}
static int host_readfirstlane(int x) { return host_readlane(x, 0); }
unsigned long long __ballot(int p) {
  lanes[here.x] = p != 0;
  pthread_barrier_wait(&meet);
  unsigned long long r = 0;
  for (int i = 0; i < 64; ++i) r |= (unsigned long long)lanes[i] << i;
  pthread_barrier_wait(&meet);
  return r;
}
void __syncthreads() { pthread_barrier_wait(&meet); }
namespace dllm { int device_cu_count() { return 256; } }
using namespace dllm;

int main() {
  constexpr int N = 4, NONE = 0x5eed;
  pthread_barrier_init(&meet, nullptr, 64);
  for (int rows : {1, 31, 32, 33, 40, 50, 63, 64})
    for (int kind = 0; kind < 4; ++kind) {
      std::vector<int> which(rows);
      for (int m = 0; m < rows; ++m) which[m] = kind == 0 ? 2 : kind == 1 ? m * 3 %% (N + 2) - 1 : kind == 2 ? -1 : m * N / rows;
      AdaptersArgs a{};
      a.rows = rows;
      a.adapters = N;
      a.rank = 8;
      a.slices = 1;
      a.d_in = a.d_out = a.slice_end[0] = 64;
      a.which = which.data();
      const AdaptersPlan p = plan_of(a);
      if (p.sorted) printf("sorted at %%d rows\n", rows);
      std::vector<int> had(rows, 0);
      for (int i = 0; i < p.tiles; ++i) {
        int place[128];  // int rows[TM], and what lies behind it
        for (int& x : place) x = NONE;
        struct Found { int adapter, count; } t[64];
        std::vector<std::thread> wave;
        for (unsigned l = 0; l < 64; ++l)
          wave.emplace_back([&, l] {
            here.x = l;
            const auto r = tile_of(a, p, i, place);
            t[l] = Found{r.adapter, r.count};
          });
        for (auto& w : wave) w.join();
        for (int l = 1; l < 64; ++l)
          if (t[l].adapter != t[0].adapter || t[l].count != t[0].count) printf("rows %%d kind %%d tile %%d: lanes disagree\n", rows, kind, i);
        for (int k = TM; k < 128; ++k)
          if (place[k] != NONE) printf("rows %%d kind %%d tile %%d: store to rows[%%d]\n", rows, kind, i, k);
        if (t[0].count < 0 || t[0].count > TM) printf("rows %%d kind %%d tile %%d: %%d rows\n", rows, kind, i, t[0].count);
        for (int k = 0; k < t[0].count && k < TM; ++k) {
          const int m = place[k], w = m >= 0 && m < rows ? (which[m] >= 0 && which[m] < N ? which[m] : -1) : -2;
          if (w == -2 || w != t[0].adapter) printf("rows %%d kind %%d tile %%d: row %%d\n", rows, kind, i, m);
          if (w != -2) ++had[m];
        }
      }
      for (int m = 0; m < rows; ++m)
        if (had[m] != 1) printf("rows %%d kind %%d: row %%d in %%d tiles\n", rows, kind, m, had[m]);
      printf("looked at %%d rows kind %%d\n", rows, kind);
    }
}
"""


@pytest.fixture(scope="module")
def output(tmp_path_factory):
    d = tmp_path_factory.mktemp("tiles")
    src, exe = d / "tiles.hip", d / "tiles"
    src.write_text(PROGRAM % os.path.join(build.CSRC, "k_adapters.hip"))
    # host code only: the kernels are not compiled, so their code object is missing at link time
    subprocess.run([build.hipcc(), "--cuda-host-only", f"--offload-arch={build.ARCH}", "-O1", "-std=c++17", "-w", "-pthread",
                    "-x", "hip", str(src), "-o", str(exe), "-Wl,--unresolved-symbols=ignore-all"], check=True, timeout=300)
    env = dict(os.environ, HIP_VISIBLE_DEVICES="", ROCR_VISIBLE_DEVICES="")  # no GPU is shown to it
    return subprocess.run([str(exe)], capture_output=True, text=True, check=True, timeout=120, env=env).stdout.split("\n")


def test_rows_among_neighbours(output):
    """Every row in one tile of its adapter, and no store behind a tile's 32 places."""
    assert len([l for l in output if l.startswith("looked")]) == 8 * 4
    wrong = [l for l in output if l and not l.startswith("looked")]
    assert not wrong, f"{len(wrong)}: {wrong[:5]}"
