// Test driver: how many tables the checked mode of the append calls allocates.  Built and run by
// tests/test_append_checks.py.  The last new token goes where the first one does, so that the calls
// are refused after they have looked at every token and before anything is launched.
#include <cstdio>
#include <cstdlib>
#include <new>
#include <vector>

#include "kvt.h"

static long g_large = 0;   // allocations of more than a kilobyte (a set's nodes are smaller)

void* operator new(std::size_t n) {
  if (n > 1024) ++g_large;
  if (void* p = std::malloc(n)) return p;
  throw std::bad_alloc();
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }

int main(int argc, char** argv) {
  const int32_t tokens = argc > 1 ? std::atoi(argv[1]) : 0, pages = (tokens + 15) / 16;
  std::vector<int32_t> table(2 * (size_t)pages);
  for (int32_t i = 0; i < pages; ++i) table[i] = table[pages + i] = i;
  const int32_t prefix[2] = {0, 0}, suffix[2] = {tokens, 1};
  const kvt_pool pool = {(void*)0x10000000, (void*)0x20000000000, pages, 1, 64, KVT_DTYPE_BF16};
  const kvt_seqs seqs = {2, prefix, suffix, (const int32_t*)0x30000000000, table.data(), pages};
  void *k = (void*)0x40000000000, *v = (void*)0x50000000000;

  g_large = 0;
  const kvt_status plain = kvt_append_kv(&pool, &seqs, k, v, nullptr);
  const long of_plain = g_large;

  std::vector<float> freq(8, 0.5f);
  const kvt_rotary rotary = {freq.data(), nullptr, nullptr, 1, 16, 1, 0};
  const kvt_rows k_rows = {k, 64}, v_rows = {v, 64};
  g_large = 0;
  const kvt_status turned = kvt_append_kv_rotary(&pool, &seqs, &rotary, &k_rows, &v_rows, nullptr, 0, nullptr, nullptr);
  std::printf("%d %ld %d %ld\n", (int)plain, of_plain, (int)turned, g_large);
  return 0;
}
