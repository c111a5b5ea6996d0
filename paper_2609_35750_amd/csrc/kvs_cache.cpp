// Host-side bookkeeping of the streamed paged KV cache (the inference side of
// KV-streams, Section 2 "KV-streams" and Section 4 "Inference engine
// implementation"): cache blocks of block_size slots, a free list, and per
// sequence the list of its blocks in allocation order.  Tokens are appended
// at the tail of a sequence's last block; evicted entries are dropped for
// good (their slots are never refilled) and a block returns to the free list
// once none of its entries is live.  The device side (slot contents and the
// live marks read by the decode kernel) is updated by the caller with the
// slot lists these calls return.
//
// Sequences may share blocks (fork).  A slot has one position and one live mark
// on the device, so all that hold a block see the same entries of it: nothing is
// appended to a shared block, and a sequence that evicts some of its entries gets
// a block of its own for the others (evict).
#include "kvs_cache.h"

#include <algorithm>
#include <climits>
#include <cstdio>
#include <new>

namespace kvs {

SlotMap::Page* SlotMap::page(int idx) {
  if (idx == last_idx_) return last_;
  const auto it = pages_.find(idx);
  if (it == pages_.end()) return nullptr;
  last_idx_ = idx;
  return last_ = it->second.get();
}

int* SlotMap::make(int pos) {
  const int idx = pos >> kBits;
  Page* p = page(idx);
  if (!p) {
    auto fresh = std::make_unique<Page>();
    for (int& s : fresh->slot) s = kNone;
    p = fresh.get();
    pages_.emplace(idx, std::move(fresh));
    last_idx_ = idx;
    last_ = p;
  }
  return &p->slot[pos & kMask];
}

void SlotMap::count(int pos, int d) {
  const int idx = pos >> kBits;
  Page* p = page(idx);
  if (!p) return;
  p->live += d;
  live_ += d;
  if (p->live == 0) {
    pages_.erase(idx);
    last_idx_ = -1;
    last_ = nullptr;
  }
}

void SlotMap::copy_to(SlotMap* to) const {
  for (const auto& kv : pages_) to->pages_.emplace(kv.first, std::make_unique<Page>(*kv.second));
  to->live_ = live_;
}

void SlotMap::clear() {
  pages_.clear();
  last_idx_ = -1;
  last_ = nullptr;
  live_ = 0;
}

BlockManager::BlockManager(int num_blocks, int block_size, int num_seqs, int max_blocks)
    : nb_(num_blocks), bs_(block_size), ns_(num_seqs), mb_(max_blocks),
      blocks_(num_seqs), tail_fill_(num_seqs, block_size), live_(num_blocks, 0),
      refs_(num_blocks, 0), slot_of_(num_seqs) {
  free_.reserve(num_blocks);
  for (int b = num_blocks - 1; b >= 0; --b) free_.push_back(b);   // block 0 is handed out first
}

static int fail_msg(std::string* err, int code, const char* msg, long long a = 0) {
  if (err) {
    char buf[256];
    snprintf(buf, sizeof(buf), msg, a);
    *err = buf;
  }
  return code;
}

int BlockManager::append(int seq, const int32_t* pos, int n, int32_t* slots, std::string* err) {
  if (seq < 0 || seq >= ns_) return fail_msg(err, kBadArg, "sequence index %lld out of range", seq);
  auto& map = slot_of_[seq];
  // Reserve every position first (a marker no slot has), counted as live so that its page stays, and room for the
  // new blocks; a failure, of an allocation too, takes the markers back.
  constexpr int kReserved = -2;
  int done = 0, code = kOk;
  for (; done < n; ++done) {
    const int p = pos[done];
    if (p < 0) {
      code = fail_msg(err, kBadArg, "negative trace position %lld", p);
      break;
    }
    int* s = nullptr;
    try {
      s = map.make(p);
    } catch (const std::bad_alloc&) {
      code = fail_msg(err, kCapacity, "out of host memory at trace position %lld", p);
      break;
    }
    if (*s != SlotMap::kNone) {
      code = fail_msg(err, kBadState, "trace position %lld is already in the cache", p);
      break;
    }
    *s = kReserved;
    map.count(p, 1);
  }
  // blocks this append needs, checked before anything else changes
  const int room = bs_ - tail_fill_[seq];
  const long long need = n > room ? (n - room + bs_ - 1) / bs_ : 0;
  if (code == kOk && need > (long long)free_.size())
    code = fail_msg(err, kCapacity, "out of cache blocks (%lld more needed)", need);
  if (code == kOk && (long long)blocks_[seq].size() + need > mb_)
    code = fail_msg(err, kCapacity, "sequence would hold more than max_blocks (%lld) blocks", mb_);
  if (code == kOk) try {
      blocks_[seq].reserve(blocks_[seq].size() + need);
    } catch (const std::bad_alloc&) {
      code = fail_msg(err, kCapacity, "out of host memory for %lld blocks", need);
    }
  if (code != kOk) {
    for (int i = 0; i < done; ++i) {
      *map.find(pos[i]) = SlotMap::kNone;
      map.count(pos[i], -1);
    }
    return code;
  }
  for (int i = 0; i < n; ++i) {
    if (tail_fill_[seq] == bs_) {
      blocks_[seq].push_back(free_.back());
      free_.pop_back();
      tail_fill_[seq] = 0;
    }
    const int blk = blocks_[seq].back();
    refs_[blk] = 1;
    const int slot = blk * bs_ + tail_fill_[seq]++;
    ++live_[blk];
    *map.find(pos[i]) = slot;
    slots[i] = slot;
  }
  return kOk;
}

// at: where the caller's last block stood in the list, and where this one does; an eviction of consecutive positions
// touches consecutive blocks, so the search for each ends where the last one did, or one behind it.
std::vector<int>::iterator BlockManager::find_block(int seq, int blk, size_t* at) {
  auto& bl = blocks_[seq];
  const size_t i = *at;
  const auto it = i < bl.size() && bl[i] == blk           ? bl.begin() + i
                  : i + 1 < bl.size() && bl[i + 1] == blk ? bl.begin() + i + 1
                                                          : std::find(bl.begin(), bl.end(), blk);
  *at = it - bl.begin();
  return it;
}

// The block leaves the sequence's table, and if no other one holds it returns to the free list.
void BlockManager::drop_block(int seq, int blk, size_t* at) {
  auto& bl = blocks_[seq];
  const bool tail = !bl.empty() && bl.back() == blk;
  bl.erase(find_block(seq, blk, at));
  if (--refs_[blk] == 0) free_.push_back(blk);
  else --extra_;
  if (tail) tail_fill_[seq] = bs_;   // the next append opens a new block
}

int BlockManager::evict_shared(int seq, const int32_t* pos, int n, int32_t* slots, int32_t* from, int32_t* to,
                               int* n_copies, std::string* err) {
  if (seq < 0 || seq >= ns_) return fail_msg(err, kBadArg, "sequence index %lld out of range", seq);
  auto& map = slot_of_[seq];
  // Mark every entry as taken first (the sign bit of its slot; no slot gives kNone), so that a repeated position
  // shows; a failure takes the marks back.
  constexpr int kTaken = INT_MIN;
  auto untake = [&](int k) {
    while (--k >= 0) *map.find(pos[k]) ^= kTaken;
  };
  for (int i = 0; i < n; ++i) {
    int* s = pos[i] < 0 ? nullptr : map.find(pos[i]);
    if (!s || *s < 0) {
      const int code = s && *s != SlotMap::kNone
                           ? fail_msg(err, kBadState, "trace position %lld evicted twice", pos[i])
                           : fail_msg(err, kBadState, "trace position %lld is not in the cache", pos[i]);
      untake(i);
      return code;
    }
    *s ^= kTaken;
  }
  if (n_copies) *n_copies = 0;
  // Entries taken of each shared block; those that keep some are replaced, in the order they are met.
  struct Replaced {
    int blk, fresh, used;
  };
  std::vector<Replaced> replaced;
  std::unordered_map<int, int> taken, which;   // by block: entries taken; its place in `replaced`
  try {
    int last = -1, *count = nullptr;
    for (int i = 0; i < n && extra_ > 0; ++i) {
      const int blk = (*map.find(pos[i]) ^ kTaken) / bs_;
      if (refs_[blk] < 2) continue;
      if (blk != last) count = &taken[last = blk];
      ++*count;
    }
    for (int i = 0; i < n && !taken.empty(); ++i) {
      const int blk = (*map.find(pos[i]) ^ kTaken) / bs_;
      if (refs_[blk] < 2 || taken[blk] == live_[blk]) continue;
      if (!from) {
        untake(n);
        return fail_msg(err, kBadState, "trace position %lld is in a block that stays shared: its other entries need a copy",
                        pos[i]);
      }
      if (which.emplace(blk, (int)replaced.size()).second) replaced.push_back({blk, -1, 0});
    }
  } catch (const std::bad_alloc&) {
    untake(n);
    return fail_msg(err, kCapacity, "out of host memory for %lld positions", n);
  }
  if (replaced.size() > free_.size()) {
    untake(n);
    return fail_msg(err, kCapacity, "out of cache blocks (%lld more needed)", (long long)replaced.size());
  }
  if (!replaced.empty()) {   // what stays of them, by position: the copies, and the map's new slots
    std::vector<std::pair<int, int>> stay;
    try {
      map.each([&](int p, int slot) {
        if (slot >= 0 && refs_[slot / bs_] > 1 && which.count(slot / bs_)) stay.emplace_back(p, slot);
      });
    } catch (const std::bad_alloc&) {
      untake(n);
      return fail_msg(err, kCapacity, "out of host memory for %lld positions", n);
    }
    std::sort(stay.begin(), stay.end());
    size_t at = 0;
    for (Replaced& r : replaced) {
      r.fresh = free_.back();
      free_.pop_back();
      refs_[r.fresh] = 1;
      live_[r.fresh] = live_[r.blk] - taken.find(r.blk)->second;
      *find_block(seq, r.blk, &at) = r.fresh;
      --refs_[r.blk];
      --extra_;
    }
    int k = 0;
    for (const auto& e : stay) {
      Replaced& r = replaced[which.find(e.second / bs_)->second];
      from[k] = e.second;
      *map.find(e.first) = to[k++] = r.fresh * bs_ + r.used++;
    }
    *n_copies = k;
    for (const Replaced& r : replaced)   // a last block has room for appends behind what it holds
      if (blocks_[seq].back() == r.fresh) tail_fill_[seq] = r.used;
  }
  size_t at = 0;
  const bool shared = !taken.empty();
  for (int i = 0; i < n; ++i) {
    const int p = pos[i];
    int* s = map.find(p);
    const int slot = *s ^ kTaken;
    *s = SlotMap::kNone;
    map.count(p, -1);
    const int blk = slot / bs_;
    if (shared) {   // the others keep it
      const auto t = taken.find(blk);
      if (t != taken.end()) {
        slots[i] = -1;
        if (--t->second == 0 && !which.count(blk)) drop_block(seq, blk, &at);
        continue;
      }
    }
    slots[i] = slot;
    if (--live_[blk] == 0) drop_block(seq, blk, &at);
  }
  return kOk;
}

int BlockManager::release(int seq, int32_t* slots, int* n_slots, std::string* err) {
  if (seq < 0 || seq >= ns_) return fail_msg(err, kBadArg, "sequence index %lld out of range", seq);
  int k = 0;
  slot_of_[seq].each([&](int, int slot) {
    if (refs_[slot / bs_] == 1) slots[k++] = slot;
  });
  std::sort(slots, slots + k);
  *n_slots = k;
  slot_of_[seq].clear();
  for (int blk : blocks_[seq]) {
    if (--refs_[blk] > 0) {
      --extra_;
      continue;
    }
    live_[blk] = 0;
    free_.push_back(blk);
  }
  blocks_[seq].clear();
  tail_fill_[seq] = bs_;
  return kOk;
}

int BlockManager::check_pair(int src, int dst, std::string* err) const {
  for (int s : {src, dst})
    if (s < 0 || s >= ns_) return fail_msg(err, kBadArg, "sequence index %lld out of range", s);
  if (src == dst) return fail_msg(err, kBadArg, "source and destination are both sequence %lld", src);
  if (!blocks_[dst].empty()) return fail_msg(err, kBadState, "sequence %lld is not empty", dst);
  return kOk;
}

int BlockManager::fork(int src, int dst, std::string* err) {
  if (const int code = check_pair(src, dst, err)) return code;
  try {
    SlotMap map;
    slot_of_[src].copy_to(&map);
    blocks_[dst] = blocks_[src];
    slot_of_[dst].swap(map);
  } catch (const std::bad_alloc&) {
    return fail_msg(err, kCapacity, "out of host memory for %lld entries", slot_of_[src].live());
  }
  for (int blk : blocks_[src]) ++refs_[blk];
  extra_ += (long long)blocks_[src].size();
  tail_fill_[src] = tail_fill_[dst] = bs_;
  return kOk;
}

int BlockManager::copy(int src, int dst, int32_t* from, int32_t* to, int* n, std::string* err) {
  *n = 0;
  if (const int code = check_pair(src, dst, err)) return code;
  const int live = slot_of_[src].live();
  const long long need = ((long long)live + bs_ - 1) / bs_;
  if (need > (long long)free_.size())
    return fail_msg(err, kCapacity, "out of cache blocks (%lld needed)", need);
  if (need > mb_) return fail_msg(err, kCapacity, "sequence would hold more than max_blocks (%lld) blocks", mb_);
  std::vector<std::pair<int, int>> entries;
  SlotMap map;
  try {
    entries.reserve(live);
    slot_of_[src].each([&](int p, int slot) { entries.emplace_back(p, slot); });
    slot_of_[src].copy_to(&map);
    blocks_[dst].reserve(need);
  } catch (const std::bad_alloc&) {
    return fail_msg(err, kCapacity, "out of host memory for %lld entries", live);
  }
  std::sort(entries.begin(), entries.end());
  for (int i = 0; i < live; ++i) {
    if (i % bs_ == 0) {
      blocks_[dst].push_back(free_.back());
      free_.pop_back();
      refs_[blocks_[dst].back()] = 1;
    }
    const int blk = blocks_[dst].back();
    ++live_[blk];
    from[i] = entries[i].second;
    *map.find(entries[i].first) = to[i] = blk * bs_ + i % bs_;
  }
  slot_of_[dst].swap(map);
  tail_fill_[dst] = live % bs_ ? live % bs_ : bs_;
  *n = live;
  return kOk;
}

int BlockManager::compact(int seq, int32_t* from, int32_t* to, int* n, std::string* err) {
  *n = 0;
  if (seq < 0 || seq >= ns_) return fail_msg(err, kBadArg, "sequence index %lld out of range", seq);
  auto& bl = blocks_[seq];
  // Blocks that take part, by their place in the table: the fullest stay, as many as hold all their entries.
  const size_t end = bl.size() - (!bl.empty() && tail_fill_[seq] < bs_ ? 1 : 0);
  std::vector<int> mine, state;   // state, by place: kOut, kStays, kLeaves
  enum { kOut, kStays, kLeaves };
  struct Row {
    int place, row, pos;
  };
  std::vector<Row> leaving;
  std::vector<uint64_t> held;     // by place: rows with an entry
  std::unordered_map<int, int> place_of;
  try {
    state.assign(bl.size(), kOut);
    held.assign(bl.size(), 0);
    long long live = 0;
    for (size_t i = 0; i < end; ++i)
      if (refs_[bl[i]] == 1) {
        mine.push_back((int)i);
        live += live_[bl[i]];
      }
    const size_t keep = (size_t)((live + bs_ - 1) / bs_);
    if (keep >= mine.size()) return kOk;
    std::stable_sort(mine.begin(), mine.end(), [&](int a, int b) { return live_[bl[a]] > live_[bl[b]]; });
    for (size_t i = 0; i < mine.size(); ++i) {
      state[mine[i]] = i < keep ? kStays : kLeaves;
      place_of.emplace(bl[mine[i]], mine[i]);
    }
    slot_of_[seq].each([&](int p, int slot) {
      const auto it = place_of.find(slot / bs_);
      if (it == place_of.end()) return;
      if (state[it->second] == kLeaves) leaving.push_back({it->second, slot % bs_, p});
      else held[it->second] |= 1ull << (slot % bs_);
    });
  } catch (const std::bad_alloc&) {
    return fail_msg(err, kCapacity, "out of host memory for %lld entries", slot_of_[seq].live());
  }
  std::sort(leaving.begin(), leaving.end(), [](const Row& a, const Row& b) {
    return a.place != b.place ? a.place < b.place : a.row < b.row;
  });
  size_t place = 0;
  int row = 0, k = 0;
  for (const Row& e : leaving) {
    while (state[place] != kStays || row >= bs_ || ((held[place] >> row) & 1ull)) {
      if (state[place] == kStays && row < bs_) ++row;
      else ++place, row = 0;
    }
    from[k] = bl[e.place] * bs_ + e.row;
    to[k] = bl[place] * bs_ + row++;
    ++live_[bl[place]];
    *slot_of_[seq].find(e.pos) = to[k++];
  }
  *n = k;
  size_t out = 0;
  for (size_t i = 0; i < bl.size(); ++i) {
    if (state[i] == kLeaves) {
      live_[bl[i]] = refs_[bl[i]] = 0;
      free_.push_back(bl[i]);
    } else {
      bl[out++] = bl[i];
    }
  }
  bl.resize(out);   // a last block with room for appends takes no part, so there is still room, or still none
  return kOk;
}

// Sequences in the order of their tables' leading shared blocks; a run of them whose tables begin with the same l
// blocks saves (length - 1) l block reads as one group.  The runs nest (those with a larger l inside), so from the inside
// out each one is worth the larger of its own saving and the sum of what is inside it, and from the outside in the
// first run that is worth its own becomes a group.
int BlockManager::groups(int32_t* seq_group, int32_t* group_blocks, int* n, std::string* err) const {
  *n = 0;
  for (int s = 0; s < ns_; ++s) seq_group[s] = -1;
  if (extra_ == 0) return kOk;
  struct Run {
    long long own, inner;   // block reads saved by the run as a group; by the runs inside it
    int first, last, blocks;
  };
  try {
    std::vector<int> order, lead(ns_, 0);   // leading shared blocks
    for (int s = 0; s < ns_; ++s) {
      const auto& bl = blocks_[s];
      int k = 0;
      while (k < (int)bl.size() && refs_[bl[k]] > 1) ++k;
      lead[s] = k;
      if (k) order.push_back(s);
    }
    std::stable_sort(order.begin(), order.end(), [&](int a, int b) {
      return std::lexicographical_compare(blocks_[a].begin(), blocks_[a].begin() + lead[a], blocks_[b].begin(),
                                          blocks_[b].begin() + lead[b]);
    });
    const int m = (int)order.size();
    auto alike = [&](int i) {   // blocks that sequences i - 1 and i of the order begin with
      if (i >= m) return -1;
      const int a = order[i - 1], b = order[i];
      const int most = std::min(lead[a], lead[b]);
      return (int)(std::mismatch(blocks_[a].begin(), blocks_[a].begin() + most, blocks_[b].begin()).first -
                   blocks_[a].begin());
    };
    std::vector<Run> runs{{0, 0, 0, m - 1, 0}};
    std::vector<int> open{0};
    for (int i = 1; i <= m; ++i) {
      const int l = alike(i);
      int first = i - 1, inside = -1;
      while (!open.empty() && runs[open.back()].blocks > l) {
        const int r = open.back();
        open.pop_back();
        runs[r].last = i - 1;
        runs[r].own = (long long)(runs[r].last - runs[r].first) * runs[r].blocks;
        first = runs[r].first;
        inside = r;
        if (!open.empty() && runs[open.back()].blocks >= l) {
          runs[open.back()].inner += std::max(runs[r].own, runs[r].inner);
          inside = -1;
        }
      }
      if (l > 0 && (open.empty() || runs[open.back()].blocks < l)) {
        const long long inner = inside < 0 ? 0 : std::max(runs[inside].own, runs[inside].inner);
        open.push_back((int)runs.size());
        runs.push_back({0, inner, first, i - 1, l});
      }
    }
    // A run was made before or behind the ones inside it; take the larger runs first.
    std::vector<int> by_size;
    for (int r = 1; r < (int)runs.size(); ++r) by_size.push_back(r);
    std::stable_sort(by_size.begin(), by_size.end(), [&](int a, int b) {
      return runs[a].last - runs[a].first != runs[b].last - runs[b].first
                 ? runs[a].last - runs[a].first > runs[b].last - runs[b].first
                 : runs[a].blocks < runs[b].blocks;
    });
    for (int r : by_size) {
      const Run& x = runs[r];
      if (x.own <= 0 || x.own < x.inner || seq_group[order[x.first]] >= 0) continue;
      for (int i = x.first; i <= x.last; ++i) seq_group[order[i]] = *n;
      group_blocks[(*n)++] = x.blocks;
    }
  } catch (const std::bad_alloc&) {
    *n = 0;
    return fail_msg(err, kCapacity, "out of host memory for %lld sequences", ns_);
  }
  return kOk;
}

int BlockManager::shared(int seq) const {
  if (seq < 0 || seq >= ns_) return -1;
  int k = 0;
  if (extra_ > 0)   // a cache that has not forked asks this at every eviction
    for (int blk : blocks_[seq]) k += refs_[blk] > 1;
  return k;
}

void BlockManager::tables(int32_t* block_table, int32_t* seq_blocks) const {
  for (int s = 0; s < ns_; ++s) {
    const auto& bl = blocks_[s];
    seq_blocks[s] = (int32_t)bl.size();
    for (int i = 0; i < mb_; ++i) block_table[(size_t)s * mb_ + i] = i < (int)bl.size() ? bl[i] : 0;
  }
}

int BlockManager::live(int seq) const {
  return (seq >= 0 && seq < ns_) ? slot_of_[seq].live() : -1;
}

}  // namespace kvs
