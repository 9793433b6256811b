// The launches of calls on drafted tokens, looked at on the CPU: the library's host code (address and undefined-behaviour sanitizers on, no device
// code) over a stand-in for the HIP runtime that launches nothing and hands every launch's arguments to a check.  What a kernel would read from
// a list that travels as a launch argument has to lie inside it.  Built and run by tests/test_launch_lists.py.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <string>
#include <vector>

#include "percache_internal.hpp"

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

struct PathLaunch {   // kv_path_kernel
  pc::ListWords lists;
  int record, queries, blocks, T;
  const void *k;
};
std::vector<PathLaunch> paths;
int other_launches;

int bad;
void expect(bool ok, const char *what) {
  if (!ok) {
    ++bad;
    std::printf("FAILED: %s\n", what);
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
  if (kernels()[stub].find("kv_path_kernel") == std::string::npos) {
    ++other_launches;
    return hipSuccess;
  }
  // (stores, bf16 slots, k, v, weights, capacity, T, lists, record)
  PathLaunch p;
  p.k = *(const void **)args[3];
  p.T = *(int *)args[7];
  p.lists = *(const pc::ListWords *)args[8];
  p.record = *(int *)args[9];
  p.queries = (int)grid.z;
  p.blocks = (int)grid.x;
  paths.push_back(p);
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
hipError_t hipMemcpyAsync(void *to, const void *from, size_t n, hipMemcpyKind, hipStream_t) { memcpy(to, from, n); return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *s) { *s = hipStreamCaptureStatusNone; return hipSuccess; }
}

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
  Context(int n_slots, int capacity) : c{1, 64, 2, 1, 64, n_slots, capacity, 16384, 10000.0f, 0, 0, 0, 0} {
    const size_t bytes = percache_arena_bytes(&c);
    arena = aligned(bytes);
    if (bytes == 0 || percache_create(&c, arena, bytes, &ctx) != PC_OK) std::abort();
  }
  ~Context() {
    percache_destroy(ctx);
    std::free(arena);
  }
  void put(int slot, int tokens) {
    if (percache_kv_put(ctx, 0, slot, arena, arena, tokens, nullptr) != PC_OK) std::abort();
  }
};

// what kv_path_kernel reads of its lists: a record's four words (slot, token, nodes, query), then as many nodes as the third says
constexpr int kHeader = 4;
void check_records(const char *what) {
  for (const PathLaunch &p : paths) {
    expect(p.record >= kHeader && (long)p.record * p.queries <= pc::kListWords, what);
    for (int z = 0; z < p.queries && (z + 1) * p.record <= pc::kListWords; ++z) {
      const int32_t *rec = p.lists.v + z * p.record;
      expect(rec[0] >= 0 && rec[2] >= 0 && kHeader + rec[2] <= p.record, what);
      expect((rec[1] + rec[2] + 63) / 64 - rec[1] / 64 <= p.blocks, what);
      for (int j = 0; j < rec[2] && kHeader + j < p.record; ++j) expect(rec[kHeader + j] >= 0 && rec[kHeader + j] < p.T, what);
    }
  }
}

pc_status append(Context &x, int T, const std::vector<std::vector<int32_t>> &nodes, const std::vector<int32_t> &slots, const int32_t *start = nullptr) {
  size_t most = 1;
  for (const auto &p : nodes) most = p.size() > most ? p.size() : most;
  std::vector<int32_t> path(nodes.size() * most, 0), n_path;
  for (size_t b = 0; b < nodes.size(); ++b) {
    std::copy(nodes[b].begin(), nodes[b].end(), path.begin() + b * most);
    n_path.push_back((int32_t)nodes[b].size());
  }
  paths.clear();
  return percache_kv_append_path(x.ctx, 0, x.arena, x.arena, (int32_t)nodes.size(), T, path.data(), n_path.data(), (int32_t)most, slots.data(), start, nullptr, nullptr, nullptr);
}

// a query without a slot whose path is longer than that of any query that has one
void skipped_queries() {
  const char *what = "a skipped query's record";
  {
    Context x(2, 64);
    expect(append(x, 2000, {{5}, std::vector<int32_t>(2000, 7)}, {0, -1}) == PC_OK, "call");
    expect(paths.size() == 1 && percache_kv_len(x.ctx, 0, 0) == 1, "one launch, one token");
    check_records(what);
  }
  {   // as the last record of a full list
    Context x(207, 64);
    std::vector<std::vector<int32_t>> nodes(207, std::vector<int32_t>(1, 3));
    std::vector<int32_t> slots(207);
    for (int b = 0; b < 207; ++b) slots[b] = b;
    nodes.push_back(std::vector<int32_t>(200, 9));
    slots.push_back(-5);
    expect(append(x, 256, nodes, slots) == PC_OK, "call");
    check_records(what);
  }
  {   // nobody has a slot
    Context x(1, 64);
    expect(append(x, 900, {std::vector<int32_t>(900, 1), {}}, {-1, -1}) == PC_OK && paths.empty(), "nothing to launch");
  }
}

// paths that a launch's list does not hold go in pieces that end with a block of their slot
void long_paths() {
  const char *what = "a long path's pieces";
  for (int have : {0, 1, 37, 63, 64, 700})
    for (int n : {827, 828, 829, 830, 892, 1656, 3000}) {
      Context x(3, 4096);
      if (have) x.put(0, have);
      x.put(2, 9);
      std::vector<std::vector<int32_t>> nodes(4);
      for (int j = 0; j < n; ++j) nodes[0].push_back((j * 7 + 3) % 5000);
      nodes[1] = {1, 2, 3};
      nodes[2].assign(4000, 8);
      nodes[3] = {4999};
      expect(append(x, 5000, nodes, {0, 1, -1, 2}) == PC_OK, "call");
      expect(percache_kv_len(x.ctx, 0, 0) == have + n && percache_kv_len(x.ctx, 0, 1) == 3 && percache_kv_len(x.ctx, 0, 2) == 10, "lengths");
      check_records(what);
      int at[3] = {have, 0, 9};
      for (const PathLaunch &p : paths)
        for (int z = 0; z < p.queries; ++z) {
          const int32_t *rec = p.lists.v + z * p.record;
          const int b = rec[3], slot = rec[0], base = slot == 0 ? have : slot == 1 ? 0 : 9;
          expect(slot == (b == 3 ? 2 : b) && rec[1] == at[slot], what);
          for (int j = 0; j < rec[2]; ++j) expect(rec[kHeader + j] == nodes[b][rec[1] - base + j], what);
          at[slot] += rec[2];
          expect(at[slot] == base + (int)nodes[b].size() || at[slot] % 64 == 0, what);
        }
      expect(at[0] == have + n && at[1] == 3 && at[2] == 10, what);
    }
}

// weights for slots none of whose rows counts (the query with a long path has no chunks): their number of row blocks is no limit for anybody
void weights_without_counting_rows() {
  Context x(1, 64);
  x.put(0, 60);
  const int T = 200;
  std::vector<int32_t> ids = {0, 0}, used = {60, 0}, n_chunks = {1, 0}, path(2 * T), n_path = {0, T};
  for (int j = 0; j < T; ++j) path[j] = path[T + j] = j;
  const size_t bytes = percache_draft_workspace_bytes(x.ctx, 2, T, 1);
  void *ws = aligned(bytes);
  std::vector<float> w(64);
  const int before = other_launches;
  expect(percache_attention_weights(x.ctx, 0, x.arena, nullptr, w.data(), 2, T, ids.data(), used.data(), n_chunks.data(), 1, nullptr, path.data(), n_path.data(), T,
                                    nullptr, w.data(), nullptr, ws, bytes, nullptr) == PC_OK, "weights");
  expect(other_launches > before, "weights: launches");
  std::free(ws);
}
}  // namespace

int main() {
  skipped_queries();
  long_paths();
  weights_without_counting_rows();
  std::printf(bad ? "launch driver: %d FAILED checks\n" : "launch driver: ok\n", bad);
  return bad ? 1 : 0;
}
