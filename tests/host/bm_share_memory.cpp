// Block manager under failing allocations: a fork, a copy, an eviction in shared
// blocks, a compaction and the groups whose k-th allocation fails, for every k
// they make, give kCapacity and leave the free blocks, the tables and the live
// entries as they were; the same call then succeeds.
// Prints "ok" and exits 0, or names the first failure.
#include <cstdio>
#include <cstdlib>
#include <functional>
#include <new>
#include <vector>

#include "kvs_cache.h"

static long g_left = -1;   // allocations until one fails; -1: none fails

void* operator new(std::size_t n) {
  if (g_left >= 0 && g_left-- == 0) throw std::bad_alloc();
  if (void* p = std::malloc(n ? n : 1)) return p;
  throw std::bad_alloc();
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }

int main() {
  constexpr int NB = 900, BS = 4, N = 1100, S = 4;
  std::vector<int32_t> pos(N), slots(N), from(N), to(N), odd, group(S), blocks(S);
  for (int i = 0; i < N; ++i) pos[i] = 200 + i;
  for (int i = 0; i < N; i += 2) odd.push_back(200 + i);
  int n = 0;
  using Call = std::function<int(kvs::BlockManager&, std::string*)>;
  const std::vector<std::pair<const char*, Call>> calls = {
      {"fork", [&](kvs::BlockManager& bm, std::string* e) { return bm.fork(0, 3, e); }},
      {"copy", [&](kvs::BlockManager& bm, std::string* e) { return bm.copy(0, 3, from.data(), to.data(), &n, e); }},
      {"evict",
       [&](kvs::BlockManager& bm, std::string* e) {
         return bm.evict_shared(1, odd.data(), 300, slots.data(), from.data(), to.data(), &n, e);
       }},
      {"compact", [&](kvs::BlockManager& bm, std::string* e) { return bm.compact(2, from.data(), to.data(), &n, e); }},
      {"groups", [&](kvs::BlockManager& bm, std::string* e) { return bm.groups(group.data(), blocks.data(), &n, e); }},
  };
  for (const auto& [name, call] : calls) {
    long failures = 0;
    for (long k = 0;; ++k) {
      kvs::BlockManager bm(NB, BS, S, NB);
      std::string err;
      err.reserve(256);
      if (bm.append(0, pos.data(), N, slots.data(), &err) || bm.fork(0, 1, &err) ||
          bm.append(2, pos.data(), N, slots.data(), &err) || bm.evict(2, odd.data(), (int)odd.size(), slots.data(), &err))
        return 1;
      std::vector<int32_t> table(S * NB), before(S * NB), nblk(S), nbefore(S);
      bm.tables(before.data(), nbefore.data());
      const int free_before = bm.free_blocks();
      int live[S], code = -1;
      for (int s = 0; s < S; ++s) live[s] = bm.live(s);
      g_left = k;
      try {
        code = call(bm, &err);
      } catch (const std::bad_alloc&) {
        g_left = -1;
        std::printf("%s, allocation %ld: the exception leaves the call\n", name, k);
        return 1;
      }
      const bool failed = g_left < 0;   // the k-th allocation took place
      g_left = -1;
      if (failed && code == kvs::BlockManager::kOk) continue;   // one that the call can do without (a sort's buffer)
      if (failed) {
        ++failures;
        bm.tables(table.data(), nblk.data());
        bool same = table == before && nblk == nbefore && bm.free_blocks() == free_before;
        for (int s = 0; s < S; ++s) same = same && bm.live(s) == live[s];
        if (code != kvs::BlockManager::kCapacity || !same) {
          std::printf("%s, allocation %ld: code %d, %d free blocks (%d before)\n", name, k, code, bm.free_blocks(), free_before);
          return 1;
        }
        code = call(bm, &err);
      }
      if (code != kvs::BlockManager::kOk) {
        std::printf("%s, allocation %ld: the call after it gives %d\n", name, k, code);
        return 1;
      }
      int all = 0;
      for (int s = 0; s < S; ++s)
        if (bm.release(s, slots.data(), &all, &err)) return 1;
      if (bm.free_blocks() != NB) {
        std::printf("%s, allocation %ld: %d free blocks at the end\n", name, k, bm.free_blocks());
        return 1;
      }
      if (!failed) break;
    }
    std::printf("%s: %ld failed allocations\n", name, failures);
    if (failures < 2) return 1;
  }
  std::printf("ok\n");
  return 0;
}
