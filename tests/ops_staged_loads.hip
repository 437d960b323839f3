// The register-staged loads of the matrix product's operands (gemm.h), run on the CPU: every operand lies against a page that
// cannot be read, once with its end and once with its beginning, and what the loads leave of each tile is the operand's
// elements, with zeros past its end along k.  Prints the first case that reads outside or leaves something else.
#include <signal.h>
#include <stdio.h>
#include <string.h>
#include <sys/mman.h>
#include <unistd.h>

#include "../paper_2510_21048_amd/csrc/ops/gemm.h"

using namespace xops;

static char now[256];
static void outside(int) {
  static const char what[] = "a load outside of the operand: ";
  (void)!write(1, what, sizeof(what) - 1);
  (void)!write(1, now, strlen(now));
  _exit(1);
}

constexpr size_t kPage = 4096, kRoom = 512 * kPage;  // between two pages that cannot be read
static char* room;

static bool same(f16 got, f16 want) { return memcmp(&got, &want, 2) == 0; }

// rows x k elements, ks of k summed over; the rows lie ld apart where KC, the k do else
template <int R, bool KC>
static void operand(int64_t rows, int64_t k, int64_t ks, int64_t ld, bool at_end) {
  constexpr int THREADS = 256;
  typedef Tile<f16, R, KC> Ti;
  const int64_t high = KC ? rows : k, wide = KC ? k : rows, bytes = ((high - 1) * ld + wide) * 2;
  f16* p = reinterpret_cast<f16*>(at_end ? room + kRoom - bytes : room);
  const auto value = [&](int64_t r, int64_t c) { return f16(float((r * 37 + c * 11) % 2039 + 1)); };
  for (int64_t h = 0; h < high; ++h)
    for (int64_t w = 0; w < wide; ++w) p[h * ld + w] = KC ? value(h, w) : value(w, h);
  static char lds[Ti::kBytes];
  for (int64_t r0 = 0; r0 < rows; r0 += R)
    for (int t = 0; t < (ks + kBK - 1) / kBK + 3; ++t) {
      snprintf(now, sizeof(now), "R=%d KC=%d rows=%ld k=%ld ks=%ld ld=%ld r0=%ld tile=%d at_end=%d\n", R, int(KC), long(rows), long(k), long(ks),
               long(ld), long(r0), t, int(at_end));
      for (int tid = 0; tid < THREADS; ++tid) {
        Staged<f16, Ti, R, KC, THREADS> s;
        s.init(tid, ld, r0, rows, int(ks));
        s.load(tid, p, ld, r0, rows, t, int(ks));
        s.store(tid, lds);
      }
      for (int i = 0; i < Ti::kChunks; ++i) {
        int row, c;
        Ti::at(i, row, c);
        for (int j = 0; j < 8; ++j) {
          const int64_t r = r0 + row + (KC ? 0 : j), kk = int64_t(t) * kBK + c + (KC ? j : 0);
          f16 got;
          memcpy(&got, lds + i * 16 + j * 2, 2);
          if (r < rows && !same(got, kk < ks ? value(r, kk) : f16(0.0f))) {
            printf("another element at row %ld, k %ld: %s", long(r), long(kk), now);
            exit(1);
          }
        }
      }
    }
}

template <int R, bool KC>
static long all() {
  long cases = 0;
  const int64_t ks[] = {1, 7, 8, 63, 64, 65, 128, 130};
  for (int64_t rows = 1; rows < 2 * R + 10; ++rows)
    for (int64_t k : ks)
      for (int64_t end : {k, int64_t(64)})  // the end of a split, or of k
        for (int pad : {0, 3})
          for (int at_end : {0, 1}) {
            if (end > k) continue;
            operand<R, KC>(rows, k, end, (KC ? k : rows) + pad, at_end);
            ++cases;
          }
  return cases;
}

int main() {
  char* all_room = static_cast<char*>(mmap(nullptr, kRoom + 2 * kPage, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0));
  if (all_room == MAP_FAILED) return 2;
  mprotect(all_room, kPage, PROT_NONE);
  mprotect(all_room + kPage + kRoom, kPage, PROT_NONE);
  room = all_room + kPage;
  signal(SIGSEGV, outside);
  signal(SIGBUS, outside);
  const long cases = all<64, false>() + all<64, true>() + all<128, false>() + all<128, true>();
  printf("%ld operands ok\n", cases);
  return 0;
}
