// What calls of given shapes plan: the stand-in runtime of packed_driver.cpp, the calls from standard input, one a line:
//   Hq Hkv D n_slots n_slots_8bit capacity  tokens of every slot  n_splits n_requests chunks  rows of every request  slots, used lengths of its chunks
// and for each call a line "call STATUS ITEMS MERGES LISTS_IN_ARGUMENTS" and its items, a line each:
//   rows kind cached_tiles fresh_tiles partial entries bf16 8-bit    (partial: 1 for one of several partitions; bf16, 8-bit: whether it walks such chunks)
// "rotations": Hq Hkv D rows, answered by the workgroups of the launch.
// Built and run by tests/test_packed_shapes.py.
#define main main_of_packed_driver
#include "packed_driver.cpp"
#undef main

#include <iostream>

namespace {
// Rows of a projection: as many as a launch of fewer than 2^32 threads holds, and one more.
void rows_of_a_launch() {
  struct Heads { int q, kv, D, threads; };   // threads a row, two heads a group of D / 16 lanes
  for (const Heads &h : {Heads{3, 3, 128, 40}, Heads{4, 2, 128, 32}, Heads{14, 2, 64, 36}, Heads{4, 2, 64, 16}}) {
    Context x(h.q, h.kv, h.D, 1, 0, 64);
    const long most = (((1L << 24) - 1) * 256) / h.threads;   // (2^24 workgroups of 256 are 2^32 threads)
    auto rows = [&](long n) {
      return percache_qkv_norm_rope(x.ctx, x.arena, (h.q + 2 * h.kv) * h.D, (int32_t)n, (int32_t *)x.arena, 1, nullptr, nullptr, nullptr, nullptr, 0.f, x.arena, x.arena, x.arena, nullptr);
    };
    expect(rows(std::min<long>(most, INT32_MAX)) == PC_OK, "rows: what a launch holds");
    if (most < INT32_MAX) expect(rows(most + 1) == PC_ESHAPE && rows(std::min<long>(2 * most, INT32_MAX)) == PC_ESHAPE, "rows: more than a launch holds");
  }
}

// Workspaces: what is enough for a call is enough for every smaller one, and partial rows are kept for no more blocks than are ever cut.
void packed_sizes() {
  for (const auto &h : {std::array<int, 3>{32, 8, 128}, {2, 1, 128}, {14, 2, 64}, {16, 16, 64}}) {
    Context x(h[0], h[1], h[2], 1, 0, 64);
    const int G = h[0] / h[1];
    size_t before = 0;
    long rows_before = 0;
    for (long n = 1; n < 9000000; n += 1 + n / 3) {
      const size_t bytes = percache_packed_workspace_bytes(x.ctx, 3, (int32_t)n, 2);
      expect(bytes >= before, "sizes: smaller calls");
      if (rows_before * G / 256 > 8L * 256 / h[1])   // (8 blocks a CU and more: every further row only lengthens the lists)
        expect(bytes - before <= (size_t)((n - rows_before) * G / kNarrowRows + 1) * (kItemWords + kMergeWords) * 4 + 3 * 256, "sizes: rows that are never cut");
      before = bytes;
      rows_before = n;
    }
  }
}

void one_call(int Hq, int Hkv, int D, int n_slots, int n8, int C) {
  auto read = [](int n) {
    std::vector<int32_t> v(n);
    for (int32_t &x : v) std::cin >> x;
    return v;
  };
  Context x(Hq, Hkv, D, n_slots, n8, C);
  const std::vector<int32_t> tokens = read(n_slots);
  for (int s = 0; s < n_slots; ++s)
    if (tokens[s]) x.put(0, s, tokens[s]);
  const std::vector<int32_t> head = read(3), T = read(head[1]);
  const int n_splits = head[0], B = head[1], chunks = head[2];
  std::vector<int32_t> start(B + 1, 0), n_chunks(B, chunks), ids, used;
  for (int b = 0; b < B; ++b) {
    start[b + 1] = start[b] + T[b];
    for (int j = 0; j < chunks; ++j) {
      const auto e = read(2);
      ids.push_back(e[0]);
      used.push_back(e[1]);
    }
  }
  const size_t bytes = percache_packed_workspace_bytes(x.ctx, B, start[B], chunks);
  void *ws = aligned(bytes);
  packed.clear();
  const pc_status st = percache_attention_packed(x.ctx, 0, x.arena, x.arena, x.arena, start[B], start.data(), B, ids.data(), used.data(), n_chunks.data(), chunks,
                                                 std::min(n_splits, percache_packed_max_splits(x.ctx, B, start[B])), x.arena, nullptr, ws, bytes, nullptr);
  const int n_items = packed.empty() ? 0 : packed[0].a.merges_at / kItemWords;
  std::printf("call %d %d %d %d\n", (int)st, n_items, packed.size() == 2 ? (int)packed[1].grid.x : 0, packed.empty() || packed[0].in_args);
  for (int i = 0; i < n_items; ++i) {
    const Packed &p = packed[0];
    Item it;
    memcpy(&it, p.words.data() + (size_t)i * kItemWords, sizeof it);
    int entries = 0, formats[2] = {0, 0};
    for (int tiles = -it.tile0; it.n_cached && tiles < it.n_cached; ++entries) {
      const int32_t *e = p.words.data() + p.a.ents_at + 2 * (it.ent + entries);
      formats[e[0] >= n_slots - n8] = 1;
      tiles += (e[1] + 63) / 64;
    }
    std::printf("%d %d %d %d %d %d %d %d\n", it.rows(), it.kind(), it.n_cached, it.f1 - it.f0, it.part >= 0, entries, formats[0], formats[1]);
  }
  std::free(ws);
}
}  // namespace

int main(int argc, char **argv) {
  const std::string what = argc > 1 ? argv[1] : "";
  if (what == "rows") rows_of_a_launch();
  if (what == "sizes") packed_sizes();
  int Hq, Hkv, D, n_slots, n8, C, rows;
  while (what == "rotations" && std::cin >> Hq >> Hkv >> D >> rows) {
    Context x(Hq, Hkv, D, 1, 0, 64);
    expect(percache_qkv_norm_rope(x.ctx, x.arena, (Hq + 2 * Hkv) * D, rows, (int32_t *)x.arena, 1, nullptr, nullptr, nullptr, nullptr, 0.f, x.arena, x.arena, x.arena, nullptr) == PC_OK,
           "rotations: call");
    std::printf("workgroups %u\n", pushed.grid.x);
  }
  while (what == "calls" && std::cin >> Hq >> Hkv >> D >> n_slots >> n8 >> C) one_call(Hq, Hkv, D, n_slots, n8, C);
  std::printf(bad ? "shapes driver: %d FAILED checks\n" : "shapes driver: ok\n", bad);
  return bad ? 1 : 0;
}
