// Host program: what the recurrence's loads read of rows that end early.  Every
// element lies on a page of its own, and the pages behind a row's length cannot
// be read: a load that touches one ends the program.
#include <hip/hip_runtime.h>
#include <sys/mman.h>

#include <cstdio>
#include <cstring>

#undef __device__
#define __device__ __attribute__((device)) __attribute__((host))
#define __builtin_amdgcn_sched_barrier(x)
#include "gated_scan.h"

using namespace st::ops;

constexpr int kPage = 4096, kSteps = 70, kN = 16;

// Pages whose first `live` may be read, filled with `byte`.
char* pages(int live, int byte) {
  char* p = (char*)mmap(nullptr, kSteps * kPage, PROT_READ | PROT_WRITE,
                        MAP_PRIVATE | MAP_ANONYMOUS, -1, 0);
  memset(p, byte, kSteps * kPage);
  mprotect(p + live * kPage, (kSteps - live) * kPage, PROT_NONE);
  return p;
}

int main() {
  const int b = 5;
  static int lengths[kPage];
  for (int len : {0, 1, 15, 16, 17, 40, 69, 70}) {
    char* x = pages(len, 1);
    char* reset = pages(len, 1);
    for (int reverse = 0; reverse < 2; ++reverse) {
      ScanArgs a{};
      lengths[b] = len;
      a.q = SeqAxes{kSteps, kPage, 1, reverse, lengths, (uint8_t*)reset};
      const SeqTensor v{x, kPage / 4, 1};
      const Row r = row_of(a.q, b);
      for (int s0 = 0; s0 < kSteps; s0 += kN) {
        printf("len %d, reverse %d, step %d\n", len, reverse, s0);
        fflush(stdout);
        Pack<float, 1> out[kN];
        load_steps<kN, false>(v, a, r, b, 0, s0, false, out);
        const bool whole = s0 + kN <= len;
        if (whole) load_steps<kN, false>(v, a, r, b, 0, s0, true, out);
        const unsigned cuts = cuts_of<kN, false>(a, r, b, s0);
        for (int k = 0; k < kN; ++k) {
          const bool live = s0 + k < len;
          if ((cuts >> k & 1) != live) return 2;
          float one;
          memset(&one, 1, 4);
          if (live && out[k].e[0] != one) return 3;
        }
      }
    }
  }
  puts("ok");
}
