// The launches of calls on packed prompts and of slot copies, looked at on the CPU: the library's host code (address and undefined-behaviour sanitizers
// on, no device code) over a stand-in for the HIP runtime that launches nothing and hands every launch's arguments to a check.  The items of a call have to
// cover every row over every key that it sees, once; what they point at has to lie inside its list; the copies of a call, done one
// after the other, have to leave what they leave when done at once.  Built and run by tests/test_packed_lists.py.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <new>
#include <random>
#include <set>
#include <string>
#include <vector>

#include "launch_lists.hpp"

// ------------------------------------------------------------------------------------------------ the stand-in
namespace {
std::map<const void *, std::string> &kernels() {   // host stub -> name (filled while objects of other files are built)
  static auto *names = new std::map<const void *, std::string>;
  return *names;
}
struct Call {
  dim3 grid, block;
  size_t lds;
  hipStream_t stream;
} pushed;
char scratch_of_the_device[64];

using namespace pc::packed;
struct Packed {
  bool merge, in_args;
  dim3 grid;
  Args a;
  std::vector<int32_t> words;
};
std::vector<Packed> packed;
size_t list_words;   // of the list copied last
struct Fork { dim3 grid; pc::fork::Moves moves; int blocks; bool eight; };
std::vector<Fork> forks;

long allocations_left = -1;   // -1: as many as are asked for
int bad;
int seen_merges, seen_long, seen_short, seen_kind[2], seen_rings, seen_store[2], seen_uneven;   // that the calls reach all of this
void expect(bool ok, const char *what) {
  if (!ok) {
    if (++bad < 20) std::printf("FAILED: %s\n", what);
  }
}
}  // namespace

extern "C" {
void **__hipRegisterFatBinary(const void *) { static void *handle; return &handle; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *stub, char *, const char *name, unsigned, void *, void *, void *, void *, int *) { kernels()[stub] = name; }
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream) { pushed = {grid, block, lds, stream}; return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *stream) {
  *grid = pushed.grid, *block = pushed.block, *lds = pushed.lds, *stream = pushed.stream;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void *stub, dim3 grid, dim3, void **args, size_t, hipStream_t) {
  const std::string &name = kernels()[stub];
  const long left = allocations_left;   // (the records' own do not count)
  allocations_left = -1;
  if (name.find("packed_attention") != std::string::npos || name.find("packed_merge") != std::string::npos) {
    Packed p;
    p.merge = name.find("packed_merge") != std::string::npos;
    p.in_args = name.find("words") != std::string::npos;
    p.grid = grid;
    if (p.in_args) {
      const auto *aw = (const ArgsAndWords *)args[0];
      p.a = aw->a;
      p.words.assign(aw->words, aw->words + kArgWords);
    } else {
      p.a = *(const Args *)args[0];
      p.words.assign(p.a.words, p.a.words + list_words);
    }
    packed.push_back(p);
  }
  if (name.find("kv_fork_kernel") != std::string::npos)
    forks.push_back({grid, *(const pc::fork::Moves *)args[0], *(int *)args[1], name.find("Li1EEE") != std::string::npos});
  allocations_left = left;
  return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
const char *hipGetErrorString(hipError_t) { return "none"; }
hipError_t hipFuncSetAttribute(const void *, hipFuncAttribute, int) { return hipSuccess; }
hipError_t hipGetDevice(int *d) { *d = 0; return hipSuccess; }
hipError_t hipGetDevicePropertiesR0600(hipDeviceProp_tR0600 *p, int) { p->multiProcessorCount = 256; return hipSuccess; }
hipError_t hipGetSymbolAddress(void **p, const void *) { *p = scratch_of_the_device; return hipSuccess; }
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipEventCreate(hipEvent_t *e) { *e = nullptr; return hipSuccess; }
hipError_t hipEventCreateWithFlags(hipEvent_t *e, unsigned) { *e = nullptr; return hipSuccess; }
hipError_t hipEventDestroy(hipEvent_t) { return hipSuccess; }
hipError_t hipEventElapsedTime(float *ms, hipEvent_t, hipEvent_t) { *ms = 0.f; return hipSuccess; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipSuccess; }
hipError_t hipEventSynchronize(hipEvent_t) { return hipSuccess; }
hipError_t hipHostMalloc(void **p, size_t n, unsigned) { *p = std::malloc(n); return hipSuccess; }
hipError_t hipHostFree(void *p) { std::free(p); return hipSuccess; }
hipError_t hipMemcpy(void *to, const void *from, size_t n, hipMemcpyKind) { memcpy(to, from, n); return hipSuccess; }
hipError_t hipMemcpyAsync(void *to, const void *from, size_t n, hipMemcpyKind, hipStream_t) { memcpy(to, from, n); list_words = n / 4; return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *s) { *s = hipStreamCaptureStatusNone; return hipSuccess; }
}

// ------------------------------------------------------------------------------------------------ host memory that runs out
void *operator new(size_t n) {
  if (allocations_left == 0) throw std::bad_alloc();
  if (allocations_left > 0) --allocations_left;
  void *p = std::malloc(n ? n : 1);
  if (!p) throw std::bad_alloc();
  return p;
}
void *operator new(size_t n, const std::nothrow_t &) noexcept { return std::malloc(n ? n : 1); }
void operator delete(void *p) noexcept { std::free(p); }
void operator delete(void *p, size_t) noexcept { std::free(p); }

// ------------------------------------------------------------------------------------------------ the calls
namespace {
void *aligned(size_t bytes) {
  void *p = std::aligned_alloc(256, (bytes + 255) / 256 * 256);
  if (!p) std::abort();
  return p;
}
struct Context {
  percache_config c;
  percache_ctx *ctx = nullptr;
  void *arena;
  Context(int Hq, int Hkv, int D, int n_slots, int n8, int capacity, int n_layers = 1) : c{n_layers, 128, Hq, Hkv, D, n_slots, capacity, 4096, 10000.0f, 0, 0, 0, n8} {
    const size_t bytes = percache_arena_bytes(&c);
    arena = aligned(bytes);
    if (bytes == 0 || percache_create(&c, arena, bytes, &ctx) != PC_OK) std::abort();
  }
  ~Context() {
    percache_destroy(ctx);
    std::free(arena);
  }
  void put(int layer, int slot, int tokens) {
    if (percache_kv_put(ctx, layer, slot, arena, arena, tokens, nullptr) != PC_OK) std::abort();
  }
};

void packed_call(Context &x, std::mt19937 &rng, const std::vector<int> &T, int max_chunks, int n_splits, int gap) {
  const char *what = "packed";
  const percache_config &c = x.c;
  const int B = (int)T.size(), G = c.n_q_heads / c.n_kv_heads;
  std::vector<int32_t> start(B + 1, gap), ids((size_t)B * max_chunks, 0), used((size_t)B * max_chunks, 0), n_chunks(B, 0);
  for (int b = 0; b < B; ++b) {
    start[b + 1] = start[b] + T[b];
    n_chunks[b] = max_chunks ? (int)(rng() % (max_chunks + 1)) : 0;
    int sum = 0;
    for (int j = 0; j < n_chunks[b]; ++j) {
      const int slot = (int)(rng() % c.n_slots), have = percache_kv_len(x.ctx, 0, slot);
      ids[(size_t)b * max_chunks + j] = slot;
      int u = rng() % 4 == 0 ? 0 : 1 + (int)(rng() % have);
      if (sum + u + 1 > c.max_pos) u = 0;
      used[(size_t)b * max_chunks + j] = u;
      sum += u;
    }
  }
  const int N = start[B] + gap;
  const size_t bytes = percache_packed_workspace_bytes(x.ctx, B, N, max_chunks);
  void *ws = aligned(bytes);
  n_splits = std::min(n_splits, percache_packed_max_splits(x.ctx, B, N));
  packed.clear();
  const pc_status st = percache_attention_packed(x.ctx, 0, x.arena, x.arena, x.arena, N, start.data(), B, ids.data(), used.data(), n_chunks.data(), max_chunks, n_splits, x.arena,
                                                 nullptr, ws, bytes, nullptr);
  expect(st == PC_OK, "packed: call");
  if (start[B] == start[0]) {
    expect(packed.empty(), "packed: nothing to launch");
    std::free(ws);
    return;
  }
  expect(!packed.empty() && !packed[0].merge && packed.size() <= 2, "packed: launches");
  const Packed &p = packed[0];
  const Args &a = p.a;
  ++(p.in_args ? seen_short : seen_long);
  const int n_items = a.merges_at / kItemWords, n_words = (int)p.words.size();
  expect(a.merges_at % kItemWords == 0 && (int)p.grid.x == n_items * c.n_kv_heads, "packed: one workgroup an item and kv head");
  expect(a.ents_at % 2 == 0 && a.ents_at >= a.merges_at && a.ents_at + 2 * a.n_ents <= n_words, "packed: entries inside the list");
  if (!p.in_args) expect((size_t)n_words * 4 <= (size_t)((char *)a.part_o - (char *)a.words), "packed: the list in front of the partial rows");
  expect((char *)(a.part_ml + 2 * a.part_rows * c.n_kv_heads) <= (char *)ws + (bytes + 255) / 256 * 256, "packed: partial rows inside the workspace");
  // expected tiles of every request, entry by entry
  std::vector<std::vector<std::pair<int, int>>> want(B);   // (slot, used)
  std::vector<int> cached(B, 0);
  for (int b = 0; b < B; ++b)
    if (T[b])
      for (int j = 0; j < n_chunks[b]; ++j) {
        const int u = used[(size_t)b * max_chunks + j];
        if (u) {
          want[b].push_back({ids[(size_t)b * max_chunks + j], u});
          cached[b] += (u + 63) / 64;
        }
      }
  std::map<int, int> seq_at;   // first row -> request with rows
  for (int b = 0; b < B; ++b)
    if (T[b]) seq_at[start[b]] = b;
  struct Part { int begin, end, part, rows; };
  std::vector<std::map<int, std::vector<Part>>> blocks(B);   // of a request: first stacked row -> partitions
  std::vector<std::map<int, int>> heights(B);
  for (int i = 0; i < n_items; ++i) {
    Item it;
    memcpy(&it, p.words.data() + (size_t)i * kItemWords, sizeof it);
    const auto at = seq_at.find(it.row0);
    if (at == seq_at.end()) {
      expect(false, "packed: an item of no request");
      continue;
    }
    ++seen_kind[it.kind()];
    const int b = at->second, r = it.i0 * G + it.rem0;
    expect(it.T == T[b] && it.rem0 < G && it.rows() >= 1 && it.rows() <= (it.kind() == kWide ? kWideRows : kNarrowRows) && r + it.rows() <= G * T[b], "packed: rows of an item");
    expect(it.n_cached >= 0 && it.f0 >= 0 && it.f1 >= it.f0 && it.n_cached + it.f1 - it.f0 >= 1 && it.f1 <= (T[b] + 63) / 64, "packed: tiles of an item");
    int begin = cached[b] + it.f0;
    if (it.n_cached) {
      int before = 0, e = -1;
      for (int k = 0; k < (int)want[b].size() && e < 0; ++k) {   // which of the request's entries it starts in: by its place among all entries
        int first = 0;
        for (int s = 0; s < b; ++s) first += (int)want[s].size();
        if (it.ent == first + k) e = k;
        else before += (want[b][k].second + 63) / 64;
      }
      expect(e >= 0 && it.ent < a.n_ents, "packed: entry of an item");
      if (e >= 0) {
        begin = before + it.tile0;
        expect(it.slot0 == want[b][e].first && it.used0 == want[b][e].second && it.tile0 >= 0 && it.tile0 * 64 < it.used0, "packed: first entry");
        int tiles = -it.tile0, k = e;
        while (tiles < it.n_cached && k < (int)want[b].size()) {
          expect(p.words[a.ents_at + 2 * (it.ent + k - e)] == want[b][k].first && p.words[a.ents_at + 2 * (it.ent + k - e) + 1] == want[b][k].second, "packed: entries");
          tiles += (want[b][k++].second + 63) / 64;
        }
        expect(tiles >= it.n_cached, "packed: cached tiles of an item");
      }
      expect(it.f1 == it.f0 || (it.f0 == 0 && begin + it.n_cached == cached[b]), "packed: fresh tiles behind all cached ones");
    }
    blocks[b][r].push_back({begin, begin + it.n_cached + it.f1 - it.f0, it.part, it.rows()});
    heights[b][r] = it.rows();
  }
  std::vector<std::pair<int, int>> rows_used;   // partial rows
  std::map<int, Merge> merges;
  int n_merges = 0;
  if (packed.size() == 2) {
    n_merges = (int)packed[1].grid.x;
    seen_merges += n_merges;
    for (int i = 0; i < n_merges; ++i) {
      Merge m;
      memcpy(&m, p.words.data() + a.merges_at + (size_t)i * kMergeWords, sizeof m);
      merges[m.part] = m;
      expect(m.rows <= (int)packed[1].grid.y * 256 / (c.head_dim / 8) && packed[1].grid.z == (unsigned)c.n_kv_heads, "packed: rows of the merge");
    }
    expect(a.merges_at + n_merges * kMergeWords <= a.ents_at, "packed: merges in front of the entries");
  }
  int merged = 0;
  for (int b = 0; b < B; ++b) {
    int r = 0;
    for (auto &kv : blocks[b]) {
      expect(kv.first == r, "packed: every row in one block");
      const int rows = heights[b][kv.first], tiles = cached[b] + ((kv.first + rows - 1) / G) / 64 + 1;
      auto &parts = kv.second;
      std::sort(parts.begin(), parts.end(), [](const Part &x, const Part &y) { return x.begin < y.begin; });
      int t = 0, shortest = tiles, longest = 0;
      for (const Part &q : parts) {
        shortest = std::min(shortest, q.end - q.begin);
        longest = std::max(longest, q.end - q.begin);
        expect(q.begin == t && q.rows == rows, "packed: every key in one partition");
        t = q.end;
        expect((parts.size() == 1) == (q.part < 0), "packed: partial results");
        if (q.part >= 0) rows_used.push_back({q.part, q.part + rows});
      }
      expect(t == tiles, "packed: all keys");
      seen_uneven += longest > shortest + 1;
      if (parts.size() > 1) {
        ++merged;
        const auto m = merges.find(parts[0].part);
        expect(m != merges.end() && m->second.n == (int)parts.size() && m->second.rows == rows && m->second.row0 == start[b] && m->second.i0 * G + m->second.rem0 == kv.first,
               "packed: a merge for every cut block");
        for (size_t j = 0; j < parts.size(); ++j) expect(parts[j].part == parts[0].part + (int)j * rows, "packed: a merge finds its partitions");
        if (n_splits > 0) expect((int)parts.size() <= n_splits, "packed: partitions asked for");
      }
      r += rows;
    }
    expect(r == G * T[b], "packed: all rows");
  }
  expect(merged == n_merges, what);
  std::sort(rows_used.begin(), rows_used.end());
  for (size_t i = 0; i < rows_used.size(); ++i) expect(rows_used[i].second <= (i + 1 < rows_used.size() ? rows_used[i + 1].first : (int)a.part_rows), "packed: partial rows apart");
  std::free(ws);
}

void packed_calls() {
  std::mt19937 rng(1);
  const int heads[][3] = {{16, 8, 128}, {14, 2, 64}, {3, 3, 128}, {71, 1, 64}, {32, 8, 128}, {24, 8, 128}, {8, 1, 64}};
  for (const auto &h : heads) {
    if ((h[0] + 2 * h[1]) * h[2] % 128) continue;
    Context x(h[0], h[1], h[2], 24, 9, 192);
    for (int s = 0; s < 24; ++s) x.put(0, s, 1 + (int)(rng() % 192));
    for (int round = 0; round < 120; ++round) {
      const int B = 1 + (int)(rng() % (round % 10 == 0 ? 300 : 12)), most = round % 7 == 0 ? 3000 : round % 3 == 0 ? 300 : 20;
      std::vector<int> T(B);
      for (int &t : T) t = rng() % 5 == 0 ? 0 : rng() % 3 == 0 ? 1 : (int)(rng() % (B > 20 ? 40 : most));
      const int chunks = round % 4 == 0 ? 0 : (int)(rng() % (round % 11 == 0 ? 90 : 14)), splits = round % 2 ? 0 : (int)(rng() % 65);
      packed_call(x, rng, T, chunks, splits, round % 5 == 0 ? (int)(rng() % 40) : 0);
    }
    packed_call(x, rng, {0, 0, 0}, 3, 0, 7);
    packed_call(x, rng, {1}, 0, 0, 0);
    packed_call(x, rng, {9000, 1, 4500}, 2, 0, 0);
  }
}

// The moves of a call, list by list, over slots that hold their own number and length.
void fork_call(Context &x, const std::vector<int32_t> &src, const std::vector<int32_t> &dst, const std::vector<int32_t> &cut) {
  const int S = x.c.n_slots, n16 = S - x.c.n_slots_8bit;
  std::vector<std::vector<int>> was(S), now;   // tokens
  for (int s = 0; s < S; ++s) was[s].assign(std::max(0, percache_kv_len(x.ctx, 0, s)), s);
  std::vector<std::vector<int>> want = was;
  for (size_t i = 0; i < src.size(); ++i) {
    want[dst[i]] = was[src[i]];
    if (!cut.empty()) want[dst[i]].resize(cut[i]);
  }
  forks.clear();
  expect(percache_kv_fork(x.ctx, 0, 1, src.data(), dst.data(), cut.empty() ? nullptr : cut.data(), (int32_t)src.size(), nullptr) == PC_OK, "fork: call");
  now = was;
  for (auto &s : now) s.resize(x.c.slot_capacity, -1);
  for (const Fork &f : forks) {
    const int off = f.eight ? n16 : 0, count = f.eight ? S - n16 : n16, lists = (int)f.grid.x / f.blocks / x.c.n_kv_heads;
    expect(lists >= 1 && f.moves.start[lists] <= pc::fork::kMoves, "fork: moves of a launch");
    ++seen_store[f.eight];
    std::map<int, int> owner;   // slot -> list that touches it (others run beside it)
    for (int l = 0; l < lists; ++l) {
      std::vector<int> held;
      for (int m = f.moves.start[l]; m < f.moves.start[l + 1]; ++m) {
        const pc::fork::Move &v = f.moves.m[m];
        expect(v.src >= -1 && v.src < count && v.dst >= -1 && v.dst < count && v.len >= 1 && v.len <= f.blocks * 64 && v.len <= x.c.slot_capacity, "fork: a move");
        for (int s : {v.src, v.dst})
          if (s >= 0) {
            if (owner.count(s)) expect(owner[s] == l, "fork: lists that run beside each other");
            owner[s] = l;
          }
        seen_rings += v.dst < 0;
        if (v.dst < 0) held.assign(now[off + v.src].begin(), now[off + v.src].begin() + v.len);
        else {
          const std::vector<int> &from = v.src < 0 ? held : now[off + v.src];
          expect((int)from.size() >= v.len, "fork: tokens that were held");
          std::vector<int> copy(from.begin(), from.begin() + std::min<size_t>(v.len, from.size()));
          std::copy(copy.begin(), copy.end(), now[off + v.dst].begin());
        }
      }
    }
  }
  for (int s = 0; s < S; ++s) {
    expect(percache_kv_len(x.ctx, 0, s) == (int)want[s].size(), "fork: lengths");
    now[s].resize(want[s].size());
    expect(now[s] == want[s], "fork: what a slot holds");
  }
}

void fork_calls() {
  std::mt19937 rng(2);
  for (int round = 0; round < 400; ++round) {
    const int S = 2 + (int)(rng() % (round % 20 == 0 ? 1500 : 40)), n8 = (int)(rng() % (S + 1));
    Context x(2, 1, 64, S, n8, 128);
    std::vector<int> full[2];
    for (int s = 0; s < S; ++s)
      if (rng() % 6) {
        x.put(0, s, 1 + (int)(rng() % 128));
        full[s >= S - n8].push_back(s);
      }
    std::vector<int32_t> src, dst, cut;
    for (int f = 0; f < 2; ++f) {
      if (full[f].empty()) continue;
      std::vector<int> to;
      for (int s = f ? S - n8 : 0; s < (f ? S : S - n8); ++s) to.push_back(s);
      std::shuffle(to.begin(), to.end(), rng);
      to.resize(1 + rng() % to.size());
      std::vector<int> from = full[f];
      if (round % 3 == 0) {   // one ring of all of them, or a permutation
        to = full[f];
        if (round % 2) std::shuffle(from.begin(), from.end(), rng);
        else std::rotate(from.begin(), from.begin() + 1, from.end());
      }
      for (size_t i = 0; i < to.size(); ++i) {
        src.push_back(round % 3 == 0 ? from[i] : from[rng() % from.size()]);
        dst.push_back(to[i]);
      }
    }
    if (round % 2)
      for (int s : src) cut.push_back(1 + (int)(rng() % percache_kv_len(x.ctx, 0, s)));
    fork_call(x, src, dst, cut);
  }
}

// Calls that find no host memory say so and have done nothing; calls that a grid does not hold are refused.
void refusals() {
  Context x(4, 2, 64, 12, 6, 128);
  for (int s = 0; s < 12; ++s) x.put(0, s, 100);
  const std::vector<int32_t> src = {0, 1, 2, 2, 6, 7}, dst = {1, 2, 0, 5, 7, 6}, cut = {10, 20, 30, 40, 50, 60};
  const std::vector<int32_t> start = {0, 400, 401, 900}, ids(60, 3), used(60, 64), n_chunks(3, 20);
  const size_t bytes = percache_packed_workspace_bytes(x.ctx, 3, 900, 20);
  void *ws = aligned(bytes);
  for (int call = 0; call < 2; ++call)
    for (long k = 0;; ++k) {
      packed.clear();
      forks.clear();
      packed.reserve(4);
      forks.reserve(4);
      allocations_left = k;
      const pc_status st = call ? percache_kv_fork(x.ctx, 0, 1, src.data(), dst.data(), cut.data(), 6, nullptr)
                                : percache_attention_packed(x.ctx, 0, x.arena, x.arena, x.arena, 900, start.data(), 3, ids.data(), used.data(), n_chunks.data(), 20, 0, x.arena,
                                                            nullptr, ws, bytes, nullptr);
      const bool ran_out = allocations_left == 0;
      allocations_left = -1;
      if (st == PC_OK) break;
      expect(ran_out && st == PC_ENOMEM && packed.empty() && forks.empty() && k < 10000, "refusals: no host memory");
      for (int s = 0; s < 12; ++s) expect(percache_kv_len(x.ctx, 0, s) == 100, "refusals: lengths stay");
    }
  expect(percache_kv_len(x.ctx, 0, 5) == 40 && percache_kv_len(x.ctx, 0, 0) == 30 && percache_kv_len(x.ctx, 0, 6) == 60, "refusals: the call that had enough");
  std::free(ws);
  // (the workspaces are not looked at by a call that is refused)
  const int many = 1 << 23;
  std::vector<int32_t> one_each(many / 2 + 1), none(many / 2, 0);
  for (int i = 0; i <= many / 2; ++i) one_each[i] = i;
  packed.clear();
  expect(percache_attention_packed(x.ctx, 0, x.arena, x.arena, x.arena, many / 2, one_each.data(), many / 2, none.data(), none.data(), none.data(), 0, 0, x.arena, nullptr, x.arena,
                                   percache_packed_workspace_bytes(x.ctx, many / 2, many / 2, 0), nullptr) == PC_ESHAPE && packed.empty(), "refusals: workgroups");
  int32_t *const ints = (int32_t *)x.arena;
  float *const floats = (float *)x.arena;
  expect(percache_beam_select(x.ctx, x.arena, 1, 8, floats, many, 1, 8, 1, ints, ints, floats, x.arena, (size_t)1 << 40, nullptr) == PC_ESHAPE, "refusals: rows of logits");
  expect(percache_qkv_norm_rope(x.ctx, x.arena, 512, INT32_MAX, ints, 1, nullptr, nullptr, nullptr, nullptr, 0.f, x.arena, x.arena, x.arena, nullptr) == PC_ESHAPE, "refusals: rows of a projection");
}

// A block's rows are told apart by the upper half of a product in place of a division by the heads a kv head.
void rows_of_heads() {
  for (uint64_t G = 1; G <= 32767; ++G) {
    const uint64_t per = (uint32_t)((0xffffffffull + G) / G);
    bool ok = true;
    for (uint64_t at : {(uint64_t)1, G - 1, G, 2 * G - 1, 2 * G, (uint64_t)255, (uint64_t)256, G + 254})
      for (uint64_t x : {at - 1, at, at + 1})
        if (x < G + 256) ok &= (G == 1 ? x : x * per >> 32) == x / G;
    expect(ok, "rows: heads of a block");
  }
}

// workspaces of the selection: never smaller than what its launches write
void selection_sizes() {
  Context x(2, 1, 64, 1, 0, 64);
  for (int batch : {1, 3, 64, 500})
    for (int beams : {1, 4, 32, 64})
      for (int best : {1, 8, 32, 64})
        for (int vocab : {1, 999, 32000, 151936}) {
          const size_t n = percache_beam_select_workspace_bytes(x.ctx, batch, beams, vocab, best);
          expect((n == 0) == (beams * best > 2048) && (n == 0 || n >= (size_t)batch * beams * best * 8), "selection: workspace");
        }
  expect(percache_beam_select_workspace_bytes(x.ctx, 1, 65, 10, 1) == 0 && percache_beam_select_workspace_bytes(nullptr, 1, 1, 1, 1) == 0, "selection: refused");
}
}  // namespace

int main() {
  packed_calls();
  fork_calls();
  refusals();
  rows_of_heads();
  selection_sizes();
  expect(seen_merges && seen_long && seen_short && seen_kind[0] && seen_kind[1] && seen_rings && seen_store[0] && seen_store[1] && seen_uneven, "calls of every kind");
  std::printf(bad ? "packed driver: %d FAILED checks\n" : "packed driver: ok\n", bad);
  return bad ? 1 : 0;
}
