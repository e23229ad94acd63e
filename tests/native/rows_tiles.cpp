// The tiles of the attention of chunks, worked out on the CPU: a wave is 64 lanes that run in turn and meet at each exchange.  Tables of offsets,
// sorted and not; what a tile names has to lie in the call's rows, and over sorted offsets every column has to be in one tile.
// Prints the first thing that is wrong and returns 1.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>
#include <ucontext.h>

#define __device__
#define __forceinline__ inline
using std::max;
using std::min;

namespace wave {
constexpr int LANES = 64;
struct { int x; } at;
ucontext_t main_ctx, lane_ctx[LANES];
char stacks[LANES][32768];
int64_t slot[2][LANES];                          // what the lanes brought to this exchange, and to the one before
int exchanges[LANES];
bool done[LANES];
void (*body)();

// brings v, waits for the other lanes, and gives what all of them brought
const int64_t* meet(int64_t v) {
  const int l = at.x, which = exchanges[l]++ & 1;
  slot[which][l] = v;
  swapcontext(&lane_ctx[l], &main_ctx);
  return slot[which];
}
void lane_main() {
  body();
  done[at.x] = true;
}
bool run(void (*f)()) {
  body = f;
  for (int l = 0; l < LANES; ++l) {
    exchanges[l] = 0;
    done[l] = false;
    getcontext(&lane_ctx[l]);
    lane_ctx[l].uc_stack = {stacks[l], 0, sizeof stacks[l]};
    lane_ctx[l].uc_link = &main_ctx;
    makecontext(&lane_ctx[l], lane_main, 0);
  }
  for (;;) {
    int ended = 0;
    for (int l = 0; l < LANES; ++l) {
      at.x = l;
      swapcontext(&main_ctx, &lane_ctx[l]);
      ended += done[l];
    }
    if (ended == LANES) return true;
    if (ended) return false;                     // some lanes wait for others that have left
  }
}
}  // namespace wave

#define threadIdx wave::at
inline uint64_t __ballot(bool v) {
  const int64_t* s = wave::meet(v);
  uint64_t b = 0;
  for (int l = 0; l < 64; ++l) b |= (uint64_t)(s[l] != 0) << l;
  return b;
}
inline int __popcll(uint64_t v) { return __builtin_popcountll(v); }
inline int __shfl_down(int v, int by, int) { const int l = wave::at.x; const int64_t* s = wave::meet(v); return (int)s[l + by < 64 ? l + by : l]; }
inline int __shfl_up(int v, int by, int) { const int l = wave::at.x; const int64_t* s = wave::meet(v); return (int)s[l >= by ? l - by : l]; }
inline int read_lane(int v, int from) { return (int)wave::meet(v)[from]; }
#define __builtin_amdgcn_readlane read_lane
#define __builtin_amdgcn_readfirstlane(v) read_lane(v, 0)

#include "../../paper_2604_13519_amd/csrc/ts_rows_tiles.h"

static ts_kv_attend_rows_args args;
static int G, T, seq_tiles, got_seq[64], got_m0[64], got_cols[64];
static RowSeq got_rows[64];

template <int TM, int UNIT>
static void one_tile() {
  const int l = wave::at.x;
  int m0 = 0, cols = 0;
  RowSeq rs{};
  const int seq = tile_of<TM, UNIT>(args, G, seq_tiles, T, m0, cols, rs);
  got_seq[l] = seq; got_m0[l] = m0; got_cols[l] = cols; got_rows[l] = rs;
}

static bool fail(const char* what, const std::vector<int32_t>& off, int tm, int n) {
  printf("%s: %d rows, %d heads a KV head, %d columns a tile, tile %d: sequence %d, first column %d of %d; offsets", what, n, G, tm, T, got_seq[0], got_m0[0], got_cols[0]);
  for (size_t i = 0; i < off.size() && i < 70; ++i) printf(" %d", off[i]);
  printf("\n");
  return false;
}

// all tiles of a call
static bool check(const std::vector<int32_t>& off, const std::vector<int32_t>& len, int n_rows, bool sorted, int which) {
  static const int TM[4] = {16, 32, 128, 256};
  static void (*const body[4])() = {one_tile<16, 16>, one_tile<32, 16>, one_tile<128, 32>, one_tile<256, 32>};
  const int n = (int)len.size(), tm = TM[which];
  args = {};
  args.row_offsets = off.data(); args.lengths = len.data();
  args.n_seqs = n; args.n_rows = n_rows; args.max_len = 4096; args.table_width = 256;
  seq_tiles = (G + tm - 1) / tm;
  const int slots = (int)((int64_t)n_rows * G / tm + n);
  std::vector<std::vector<char>> hit(sorted ? n : 0);        // columns that had a tile
  for (int s = 0; s < (int)hit.size(); ++s) hit[s].assign((size_t)(off[s + 1] - off[s]) * G, 0);
  for (T = 0; T < slots; ++T) {
    if (!wave::run(body[which])) return fail("lanes go different ways", off, tm, n_rows);
    const int seq = got_seq[0], m0 = got_m0[0], cols = got_cols[0];
    for (int l = 1; l < 64; ++l)
      if (got_seq[l] != seq || (seq >= 0 && (got_m0[l] != m0 || got_cols[l] != cols))) return fail("lanes differ", off, tm, n_rows);
    if (seq < 0) continue;
    const RowSeq& r = got_rows[0];
    if (seq >= n || m0 < 0 || cols < 1 || cols > tm) return fail("no tile", off, tm, n_rows);
    const int64_t first = (int64_t)r.first + m0 / G, last = (int64_t)r.first + (m0 + cols - 1) / G;
    if (r.first < 0 || r.end > n_rows || first < r.first || last >= r.end) return fail("rows that are not the sequence's", off, tm, n_rows);
    if (sorted)
      for (int m = m0; m < m0 + cols; ++m)
        if (hit[seq][m]++) return fail("a column twice", off, tm, n_rows);
  }
  for (auto& h : hit)
    for (char c : h)
      if (!c) return fail("a column in no tile", off, tm, n_rows);
  return true;
}

int main(int argc, char** argv) {
  const bool sorted = argc > 1 && argv[1][0] == 's';
  std::mt19937 rng(5);
  auto below = [&](int n) { return (int)(rng() % (unsigned)n); };
  if (!sorted) {                                 // sequences whose places lie behind the tile that is asked for; an empty one
    std::vector<int32_t> off(65, 0), len(64, 7);
    off[0] = 500; off[1] = 2000;
    G = 4;
    if (!check(off, len, 2000, false, 2)) return 1;
    off.assign(65, 5);
    off[0] = off[1] = off[2] = 2000;
    if (!check(off, len, 2000, false, 2)) return 1;
  }
  for (int round = 0; round < (sorted ? 160 : 200); ++round) {
    static const int around[] = {63, 64, 65};
    const int n = round % 4 == 0 ? around[round / 4 % 3] : round % 4 == 1 ? 1 + below(62) : 64 + below(140);
    const int n_rows = 1 + below(round % 3 == 0 ? 40 : 600);
    std::vector<int32_t> off(n + 1), len(n);
    for (auto& l : len) l = below(300);
    for (auto& o : off) o = below(n_rows + 1);
    if (sorted) {
      if (round % 5 == 0)                        // few that are not empty
        for (auto& o : off) o = below(4) ? (below(2) ? 0 : n_rows) : o;
      std::sort(off.begin(), off.end());
    } else {
      static const int odd[] = {-1, -5, INT32_MIN, INT32_MAX, 1 << 30, 0};
      for (auto& o : off)
        if (below(20) == 0) o = below(6) == 5 ? n_rows : odd[below(6)];
      for (auto& l : len)
        if (below(20) == 0) l = odd[below(6)];
      if (round % 3 == 1) std::sort(off.begin(), off.end(), [](int a, int b) { return a > b; });
    }
    static const int groups[] = {1, 2, 3, 4, 5, 7, 8, 16, 17};
    G = groups[below(9)];
    if (!check(off, len, n_rows, sorted, below(4))) return 1;
  }
  printf("ok\n");
  return 0;
}
