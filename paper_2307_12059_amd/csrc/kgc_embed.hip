// Host side of the operators on embedding tables (see include/kgc.h): argument checks and launches.  They take no scratch of
// the handle and do not wait for the device, so that they can be captured into graphs and enqueued on any stream.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "kgc_embed.h"
#include "kgc_handle.h"

using namespace kgc;

namespace {

constexpr int kLimitD = 960;
constexpr int64_t kLimitRows = 2147483647ll - 64;
constexpr int kLookupItems = 1024;               // vectors of a lookup's tile: four a thread
constexpr int64_t kScores4Queries = 1048560;     // a grid holds 65,535 sets of 16 queries
constexpr int64_t kScores4Lds = 80 * 1024;       // most staged queries of a workgroup, where it need not hold more
constexpr int64_t kAdjustRowsFirst = 262144;     // a MiB of biases
constexpr int64_t kMaxLds = 160 * 1024, kComputeUnits = 256;
// Up to this many ids a tile of the sort holds 1,024 of them, up to a quarter of it 512, beyond 4,096.  10,000 ids in 400,000 rows: 42 us in
// tiles of 512, 47 of 1,024; a million in a million rows: 181 us in tiles of 4,096, 209 of 1,024
constexpr int64_t kSortSmall = 262144;
// Fewer ids take shorter digits, whose tables cost a workgroup less, more of them longer ones and fewer passes: 32,768 ids in a million rows
// of 64: 67 us with 9 bits, 73 with 11; 400,000: 156, 128; 400,000 in 1,345 rows: 68, 58
constexpr int64_t kSortShort = 131072;
constexpr int kSortShortBits = 9;
constexpr int64_t kGradTeams = 4096;             // teams that k_grad_sum cuts the sorted ids for, as far as its chunks of 8 to 256 allow
// Few ids, sums that are not added to dW: a workgroup for each of up to this many rows looks for its ids; beyond, one for each id looks for
// the others of its row, after dW was cleared.  500 ids: 4,000 rows 7.1 us a workgroup a row, 9.2 us a workgroup an id; 8,000 rows 10.0, 9.1.
// (A row with many of the ids is one workgroup's work all the same: 8,192 ids for 4 rows of 512 take 93 us, 8,193 on the way of more ids 22; for 18
// rows of 100 10.5 and 10.5, for 200 rows 7 and 14; 3,500 ids of one row among 15,000 rows of 512 142 us, 3,501 22.)
constexpr int64_t kFewByRow = 4096;
constexpr int64_t kGradFewById = 3500;

// the checks that every operator begins with
int begin(kgc_handle* hd, int32_t d, HandleView* v) {
  if (!hd) return KGC_E_INVALID;
  *v = handle_view(hd);
  const int max_d = v->max_d > 0 ? std::min(v->max_d, kLimitD) : kLimitD;
  if (d < 1 || d > max_d) return handle_fail(hd, KGC_E_INVALID, "d must be in [1, max_d]");
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev != v->device)
    return handle_fail(hd, KGC_E_INVALID, "the handle's device is not the current device");
  handle_clear(hd);
  return KGC_OK;
}

int finish(kgc_handle* hd) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? KGC_OK : handle_fail(hd, KGC_E_HIP, "kernel launch", e);
}

bool is_type(int32_t t) { return t == KGC_F32 || t == KGC_BF16; }
int64_t size_of(int32_t t) { return t == KGC_BF16 ? 2 : 4; }
bool aligned(const void* p, int64_t a) { return ((uintptr_t)p % (uintptr_t)a) == 0; }
// bytes from the first to the last element of `rows` rows of `cols` elements
uint64_t span(int64_t rows, int64_t ld, int64_t cols, int64_t size) {
  return rows > 0 ? (uint64_t)((rows - 1) * ld + cols) * (uint64_t)size : 0;
}
bool overlap(const void* p, uint64_t pb, const void* q, uint64_t qb) {
  const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
  return pb && qb && a < b + qb && b < a + pb;
}
// a row stride that no offset computed with it can overflow: 2^31 rows of 2^31 elements stay below 2^62.  Outputs need at least
// the length of a row, inputs may repeat one (0)
bool is_stride(int64_t ld, int64_t least) { return ld >= least && ld <= kLimitRows; }

// workgroups for `items` work items of which each takes `per`: kernels that are given fewer than they need walk in strides
unsigned groups_for(int64_t items, int64_t per, int64_t most = 1 << 20) {
  return (unsigned)std::max<int64_t>(1, std::min(most, (items + per - 1) / per));
}

template <typename TI, typename TO, int V>
void launch_lookup(hipStream_t st, LookupArgs a) {
  a.vpr = (a.d + V - 1) / V;
  a.rows = std::max(1, std::min(kLookupRows, kLookupItems / a.vpr));
  a.magic = ((1u << 20) + a.vpr - 1) / a.vpr;
  const unsigned grid = groups_for(a.n, a.rows);
  if (a.B) k_lookup<TI, TO, true, V><<<grid, 256, 0, st>>>(a);
  else k_lookup<TI, TO, false, V><<<grid, 256, 0, st>>>(a);
}

template <typename TI, typename TO>
void launch_lookup_any(hipStream_t st, const LookupArgs& a) {
  constexpr int V = 16 / (int)sizeof(TI);
  if (a.d >= V) launch_lookup<TI, TO, V>(st, a);
  else launch_lookup<TI, TO, 1>(st, a);
}

// rows x cols elements of the type `kind`, a row ld elements from the next
void launch_zero(hipStream_t st, void* p, int32_t kind, int64_t rows, int64_t cols, int64_t ld) {
  const ZeroArgs z{p, ld == cols ? 1 : rows, ld == cols ? rows * cols : cols, ld, 0};
  const unsigned grid = groups_for(z.rows * ((z.cols + 3) / 4), 256, 16384);
  if (kind == KGC_BF16) k_zero_rows<uint16_t><<<grid, 256, 0, st>>>(z);
  else k_zero_rows<float><<<grid, 256, 0, st>>>(z);
}

// ---- gradient of a lookup: the plan of a call, the same for the size of its workspace and for its launches ----
struct GradPlan {
  bool few, table, scanned;
  int passes, bits, tile, tiles, chunk, dp, rows;
  size_t once;                                     // LDS bytes of k_sort_once; 0: the radix sort
  int64_t chunks, per_team;
  int blocks;
  size_t lds;
  uint64_t o_pair[2], o_hist, o_total, o_head, o_tail, o_ids, bytes;
};

// lanes that take a row of d columns, four each (several times beyond 256)
int lanes_for(int d) { return d <= 64 ? 16 : d <= 128 ? 32 : 64; }

GradPlan plan_grad(int64_t n, int64_t N, int d) {
  GradPlan p{};
  // A workgroup per id or row that goes through all ids, or the sort.  Measured, us, us with the sort: 3,000 ids in 15,000 rows: 12.9, 15.2 (4,000
  // ids: 17.3, 15.6); with 1,345 rows a workgroup a row: 4,000 ids: 6.8, 14.5; 8,000: 8.8, 14.7
  p.few = n <= kGradFewById || (n <= kGradFew && N <= n / 4);
  if (p.few) return p;
  p.dp = (d + 3) / 4 * 4;
  auto carve = [&](uint64_t bytes) {
    const uint64_t at = p.bytes;
    p.bytes += (bytes + 255) / 256 * 256;
    return at;
  };
  const int T = lanes_for(d), teams = 256 / T;
  p.lds = (size_t)(N < 65536 ? N + 1 : 65536) * (teams * p.dp + 1) * 4;
  p.table = d >= 4 && d <= 256 && p.lds <= (size_t)(T <= 32 ? kTableLdsOne : kTableLds);
  if (p.table) {
    p.blocks = (int)std::min<int64_t>(p.lds > kTableLds ? 256 : 512, (n + 16 * teams - 1) / (16 * teams));
    p.per_team = (n + (int64_t)p.blocks * teams - 1) / ((int64_t)p.blocks * teams);
    p.o_head = carve((uint64_t)p.blocks * N * p.dp * 4);
    p.o_total = carve((uint64_t)p.blocks * N * 4);
    return p;
  }
  int bits = 0;
  while (bits < 32 && (N >> bits) != 0) ++bits;                 // ids 0 .. N - 1, and N for those that name no row
  const int most = n <= kSortShort ? kSortShortBits : kSortBits;
  p.passes = std::max(1, (bits + most - 1) / most);
  p.bits = std::max(1, (bits + p.passes - 1) / p.passes);
  p.tile = n <= kSortSmall / 4 ? 512 : n <= kSortSmall ? 1024 : 4096;
  p.tiles = (int)((n + p.tile - 1) / p.tile);
  p.scanned = ((int64_t)p.tiles << p.bits) > (n <= kSortSmall ? kSortSums : kSortSums / 4);
  p.rows = (int)std::min<int64_t>(kOnceRows + 1, (N + kOnceGroups - 1) / kOnceGroups);
  if (n <= (p.passes == 1 ? kOnceIds / 3 : kOnceIds) && p.rows <= kOnceRows) {
    p.once = (size_t)4 * kOnceWaves * p.rows + (size_t)2 * kOnceWaves * once_share(n);
    if (p.once > 156 * 1024) p.once = 0;
  }
  p.chunk = 8;
  while (p.chunk < kGradChunk && n / p.chunk > kGradTeams) p.chunk *= 2;
  p.chunks = (n + p.chunk - 1) / p.chunk;
  for (int k = 0; k < (p.once ? 1 : std::min(p.passes, 2)); ++k) p.o_pair[k] = carve((uint64_t)n * 8);
  if (p.once) {
    p.o_ids = carve((uint64_t)n * 4);
  } else {
    p.o_hist = carve(((uint64_t)p.tiles << p.bits) * 4);
    p.o_total = carve(4ull << p.bits);
  }
  p.o_head = carve((uint64_t)p.chunks * p.dp * 4);
  p.o_tail = carve((uint64_t)p.chunks * p.dp * 4);
  return p;
}

template <typename TG, typename TW, int T, bool NARROW>
void launch_grad_few(hipStream_t st, const GradArgs& a, bool by_row) {
  if (by_row) k_grad_few<TG, TW, true, T, NARROW><<<(unsigned)a.N, 256, 0, st>>>(a);
  else k_grad_few<TG, TW, false, T, NARROW><<<(unsigned)a.n, 256, 0, st>>>(a);
}

// The sorted pairs of a call.  What of dW has to be cleared is shared out among the launches, half as much to a counting one as to a
// scattering one.
template <typename TW, int K>
const uint2* launch_sort(hipStream_t st, const GradArgs& a, const GradPlan& p, char* work, ZeroArgs z) {
  SortArgs s{};
  s.ids = a.ids; s.sid = a.sid; s.N = (uint32_t)a.N; s.n = a.n; s.tiles = p.tiles; s.bits = p.bits; s.scanned = p.scanned;
  s.hist = (uint32_t*)(work + p.o_hist);
  s.total = (uint32_t*)(work + p.o_total);
  const int64_t vectors = z.rows * ((z.cols + 3) / 4), third = (vectors + 3 * p.passes - 1) / (3 * p.passes);
  auto extra = [&](int64_t share) {                             // workgroups that clear: up to four a compute unit
    s.zero = z;
    s.zero.per_launch = share;
    return (unsigned)(p.tiles + (share > 0 ? groups_for(share, 1024, 1024) : 0));
  };
  const size_t lds = (size_t)6 * 4 << p.bits;
  for (int k = 0; k < p.passes; ++k) {
    s.shift = k * p.bits;
    s.in = (const uint2*)(work + p.o_pair[(k + 1) & 1]);
    s.out = (uint2*)(work + p.o_pair[k & 1]);
    const unsigned count = extra(third);
    if (k == 0) k_sort_count<TW, true, K><<<count, 256, 0, st>>>(s);
    else k_sort_count<TW, false, K><<<count, 256, 0, st>>>(s);
    s.zero_first += third;
    if (p.scanned) k_sort_scan<<<((1 << p.bits) + 63) / 64, 1024, 0, st>>>(s.hist, s.total, p.tiles, 1 << p.bits);
    const unsigned scatter = extra(2 * third);
    if (k == 0) k_sort_scatter<TW, true, K><<<scatter, 256, lds, st>>>(s);
    else k_sort_scatter<TW, false, K><<<scatter, 256, lds, st>>>(s);
    s.zero_first += 2 * third;
  }
  return s.out;
}

template <typename TW>
const uint2* launch_once(hipStream_t st, const GradArgs& a, const GradPlan& p, char* work, const ZeroArgs& z) {
  SortArgs s{};
  s.ids = a.ids; s.sid = a.sid; s.N = (uint32_t)a.N; s.n = a.n; s.tiles = kOnceGroups; s.rows = p.rows;
  if (a.sid > kOnceStride) {
    int32_t* ids = (int32_t*)(work + p.o_ids);
    k_ids<<<(unsigned)((a.n + 255) / 256), 256, 0, st>>>(a.ids, a.sid, (int)a.n, ids);
    s.ids = ids; s.sid = 1;
  }
  while ((1 << s.bits) < p.rows) ++s.bits;
  s.out = (uint2*)(work + p.o_pair[0]);
  s.zero = z;
  s.zero.per_launch = z.rows * ((z.cols + 3) / 4);
  const unsigned grid = kOnceGroups + (z.rows ? groups_for(s.zero.per_launch, 4096, 256) : 0);
  if (p.once > 64 * 1024) (void)hipFuncSetAttribute((const void*)k_sort_once<TW>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)p.once);
  k_sort_once<TW><<<grid, kOnceWaves * 64, p.once, st>>>(s);
  return s.out;
}

template <typename TG, int T>
void launch_table(hipStream_t st, const TableArgs& t, size_t lds) {
  if (lds > 64 * 1024) (void)hipFuncSetAttribute((const void*)k_grad_table<TG, T>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  k_grad_table<TG, T><<<t.blocks, 256, lds, st>>>(t);
}

template <typename TG, typename TW>
void launch_grad(hipStream_t st, GradArgs a, const GradPlan& p, char* work) {
  const bool by_row = p.few && a.n > 0 && (a.N < a.n || (!a.accumulate && a.N <= kFewByRow));
  ZeroArgs z{};
  if (!a.accumulate) {
    const bool whole = a.ldw == a.d;
    z.p = a.dW;
    z.rows = whole ? 1 : a.N;
    z.cols = whole ? a.N * a.d : a.d;
    z.ld = a.ldw;
  }
  const int T = lanes_for(a.d);
  if (p.few) {
    if (!a.accumulate && !by_row) launch_zero(st, a.dW, sizeof(TW) == 2 ? KGC_BF16 : KGC_F32, a.N, a.d, a.ldw);
    if (a.n == 0) return;
    if (a.d < 4) launch_grad_few<TG, TW, 16, true>(st, a, by_row);
    else if (T == 16) launch_grad_few<TG, TW, 16, false>(st, a, by_row);
    else if (T == 32) launch_grad_few<TG, TW, 32, false>(st, a, by_row);
    else launch_grad_few<TG, TW, 64, false>(st, a, by_row);
    return;
  }
  if (p.table) {
    TableArgs t{};
    t.G = a.G; t.ids = a.ids; t.dW = a.dW; t.n = a.n; t.ldg = a.ldg; t.sid = a.sid; t.ldw = a.ldw; t.per_team = p.per_team;
    t.d = a.d; t.dp = p.dp; t.N = (int)a.N; t.blocks = p.blocks; t.accumulate = a.accumulate; t.scale = a.scale;
    t.parts = (float*)(work + p.o_head); t.named = (uint32_t*)(work + p.o_total);
    const dim3 joins((unsigned)a.N, (unsigned)((a.d + 63) / 64), 1);
    if (T == 16) launch_table<TG, 16>(st, t, p.lds);
    else if (T == 32) launch_table<TG, 32>(st, t, p.lds);
    else launch_table<TG, 64>(st, t, p.lds);
    k_grad_table_join<TW><<<joins, 256, 0, st>>>(t);
    return;
  }
  a.pair = p.once           ? launch_once<TW>(st, a, p, work, z)
           : p.tile == 512  ? launch_sort<TW, 2>(st, a, p, work, z)
           : p.tile == 1024 ? launch_sort<TW, 4>(st, a, p, work, z)
                            : launch_sort<TW, 16>(st, a, p, work, z);
  a.head = (float*)(work + p.o_head); a.tail = (float*)(work + p.o_tail);
  a.chunks = p.chunks; a.chunk = p.chunk; a.dp = p.dp;
  const unsigned grid = (unsigned)((p.chunks * T + 255) / 256);
  const int per_wave = (int)std::min<int64_t>(64, (p.chunks + 16383) / 16384);
  const unsigned joins = (unsigned)((p.chunks + 16 * per_wave - 1) / (16 * per_wave));
  const size_t lds = (size_t)16 * p.dp * 4;
  if (a.d < 4) k_grad_sum<TG, TW, 16, 1, true><<<grid, 256, 0, st>>>(a);
  else if (a.d <= 64) k_grad_sum<TG, TW, 16, 1, false><<<grid, 256, 0, st>>>(a);
  else if (a.d <= 128) k_grad_sum<TG, TW, 32, 1, false><<<grid, 256, 0, st>>>(a);
  else if (a.d <= 256) k_grad_sum<TG, TW, 64, 1, false><<<grid, 256, 0, st>>>(a);
  else if (a.d <= 512) k_grad_sum<TG, TW, 64, 2, false><<<grid, 256, 0, st>>>(a);
  else k_grad_sum<TG, TW, 64, 4, false><<<grid, 256, 0, st>>>(a);
  if (T == 16) k_grad_join<TW, 16><<<joins, 1024, lds, st>>>(a, per_wave);
  else if (T == 32) k_grad_join<TW, 32><<<joins, 1024, lds, st>>>(a, per_wave);
  else k_grad_join<TW, 64><<<joins, 1024, lds, st>>>(a, per_wave);
}

// ---- scores against a 4-bit table ----
template <typename TX, typename TO, int CT>
void launch_scores4(hipStream_t st, const Scores4Args& a) {
  const int64_t blocks = (a.N + kTable4Rows - 1) / kTable4Rows;
  const size_t lds = (size_t)a.groups * CT * (sizeof(TX) == 4 ? 3 : 1) * 1024;
  // As many workgroups as run at once (two on a compute unit, as their registers allow, where the LDS does), each wave as many blocks
  // of rows as the others: a second round of workgroups would stage the queries again while most of the chip waits.  Workgroups go to
  // the eight XCDs in turn, so with a multiple of eight in a row those that read the same rows for other queries share an L2: 128
  // queries, 100,000 rows, d = 200: 27.2 us, without 28.0; 256 queries: 46.6, 48.4.
  const int64_t sets = (a.n + 16 * CT - 1) / (16 * CT), per_cu = std::max<int64_t>(1, std::min<int64_t>(2, kMaxLds / lds));
  const int64_t at_once = std::max<int64_t>(1, kComputeUnits * per_cu / sets);
  const int64_t per_wave = (blocks + at_once * kScores4Waves - 1) / (at_once * kScores4Waves);
  const int64_t groups = (blocks + per_wave * kScores4Waves - 1) / (per_wave * kScores4Waves);
  const dim3 grid((unsigned)(sets > 1 ? (groups + 7) / 8 * 8 : groups), (unsigned)sets, 1);
  // (more LDS than a launch gets unasked; where this fails, the launch does and reports it)
  if (lds > 64 * 1024)
    (void)hipFuncSetAttribute((const void*)k_scores4<TX, TO, CT>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  k_scores4<TX, TO, CT><<<grid, kScores4Waves * 64, lds, st>>>(a);
}

template <typename TX, typename TO>
void launch_scores4_any(hipStream_t st, const Scores4Args& a) {
  const int64_t tile = (int64_t)a.groups * (sizeof(TX) == 4 ? 3 : 1) * 1024;      // LDS bytes of 16 queries
  if (a.n > 16 && 2 * tile <= kScores4Lds) launch_scores4<TX, TO, 2>(st, a);
  else launch_scores4<TX, TO, 1>(st, a);
}

template <typename T>
void launch_adjust(hipStream_t st, AdjustArgs a, bool in_place) {
  const bool dense = !in_place || a.bias || a.allowed;
  if (!dense && !a.seen) {
    const int64_t per_row = a.n_known / a.n;
    const unsigned parts = (unsigned)std::max<int64_t>(1, std::min<int64_t>(64, per_row / 1024));
    k_adjust_known<T><<<dim3(parts, (unsigned)std::min<int64_t>(a.n, 65535), 1), 256, 0, st>>>(a);
    return;
  }
  // Biases that the L2s do not keep are read once for all rows, chunk by chunk (32 rows of a million, bfloat16: 24 us, 36 row by row);
  // otherwise a row is read from end to end (float32 without biases: 39 us, 42 chunk by chunk)
  a.rows_first = a.bias && a.N >= kAdjustRowsFirst;
  const int64_t chunks = (a.N + kAdjustChunk - 1) / kAdjustChunk;
  const unsigned grid = groups_for(a.n * chunks, 1, 1 << 22);
  if (dense) a.seen ? k_adjust<T, true, true><<<grid, 256, 0, st>>>(a) : k_adjust<T, true, false><<<grid, 256, 0, st>>>(a);
  else k_adjust<T, false, true><<<grid, 256, 0, st>>>(a);
}

}  // namespace

extern "C" {

int kgc_lookup(kgc_handle* hd, const void* A, int64_t Na, int64_t lda, const int32_t* ia, int64_t sia, float sa, const void* B,
               int64_t Nb, int64_t ldb, const int32_t* ib, int64_t sib, float sb, int64_t n, int32_t d, void* out, int64_t ldo,
               int32_t out_dtype) {
  HandleView v;
  const int rc = begin(hd, d, &v);
  if (rc != KGC_OK) return rc;
  const bool two = B || ib;
  if (!is_type(out_dtype)) return handle_fail(hd, KGC_E_INVALID, "out_dtype must be KGC_F32 or KGC_BF16");
  if (n < 0 || n > kLimitRows || Na < 0 || Na > kLimitRows || (two && (Nb < 0 || Nb > kLimitRows)))
    return handle_fail(hd, KGC_E_INVALID, "n, Na or Nb out of range");
  if (!is_stride(ldo, d)) return handle_fail(hd, KGC_E_INVALID, "ldo must be at least d");
  if (!is_stride(lda, 0) || !is_stride(sia, 0) || (two && (!is_stride(ldb, 0) || !is_stride(sib, 0))))
    return handle_fail(hd, KGC_E_INVALID, "strides must not be negative");
  if (n == 0) return KGC_OK;
  if ((Na > 0 && !A) || !ia || !out || (two && ((Nb > 0 && !B) || !ib)))
    return handle_fail(hd, KGC_E_INVALID, "NULL where data is required");
  const int64_t si = size_of(v.dtype), so = size_of(out_dtype);
  if (!aligned(A, si) || !aligned(out, so) || !aligned(ia, 4) || (two && (!aligned(B, si) || !aligned(ib, 4))))
    return handle_fail(hd, KGC_E_INVALID, "misaligned pointer");
  const uint64_t ob = span(n, ldo, d, so);
  if (overlap(out, ob, A, span(Na, lda, d, si)) || overlap(out, ob, ia, span(n, sia, 1, 4)) ||
      (two && (overlap(out, ob, B, span(Nb, ldb, d, si)) || overlap(out, ob, ib, span(n, sib, 1, 4)))))
    return handle_fail(hd, KGC_E_INVALID, "out overlaps an input");
  LookupArgs a{};
  a.A = A; a.ia = ia; a.na = Na; a.lda = lda; a.sia = sia; a.sa = sa;
  a.out = out; a.n = n; a.ldo = ldo; a.d = d;
  // an empty table has no row to read in the place of a missing one: its part is left out
  if (two && Nb > 0) {
    if (Na > 0) { a.B = B; a.ib = ib; a.nb = Nb; a.ldb = ldb; a.sib = sib; a.sb = sb; }
    else { a.A = B; a.ia = ib; a.na = Nb; a.lda = ldb; a.sia = sib; a.sa = sb; }
  }
  const bool bi = v.dtype == KGC_BF16, bo = out_dtype == KGC_BF16;
  if (a.na == 0) launch_zero(v.stream, out, out_dtype, n, d, ldo);
  else if (bi) bo ? launch_lookup_any<uint16_t, uint16_t>(v.stream, a) : launch_lookup_any<uint16_t, float>(v.stream, a);
  else bo ? launch_lookup_any<float, uint16_t>(v.stream, a) : launch_lookup_any<float, float>(v.stream, a);
  return finish(hd);
}

uint64_t kgc_lookup_grad_bytes(int64_t n, int64_t N, int32_t d) {
  if (n < 0 || n > kLimitRows || N < 0 || N > kLimitRows || d < 1 || d > kLimitD) return 0;
  return plan_grad(n, N, d).bytes;
}

int kgc_lookup_grad(kgc_handle* hd, const void* G, int32_t g_dtype, int64_t ldg, const int32_t* ids, int64_t sid, int64_t n, int32_t d,
                    float scale, int32_t accumulate, void* dW, int32_t dw_dtype, int64_t N, int64_t ldw, void* work,
                    uint64_t work_bytes) {
  HandleView v;
  const int rc = begin(hd, d, &v);
  if (rc != KGC_OK) return rc;
  if (!is_type(g_dtype) || !is_type(dw_dtype)) return handle_fail(hd, KGC_E_INVALID, "g_dtype and dw_dtype must be KGC_F32 or KGC_BF16");
  if (accumulate != 0 && accumulate != 1) return handle_fail(hd, KGC_E_INVALID, "accumulate must be 0 or 1");
  if (n < 0 || n > kLimitRows || N < 0 || N > kLimitRows) return handle_fail(hd, KGC_E_INVALID, "n or N out of range");
  if (!is_stride(ldw, d)) return handle_fail(hd, KGC_E_INVALID, "ldw must be at least d");
  if (!is_stride(ldg, 0) || !is_stride(sid, 0)) return handle_fail(hd, KGC_E_INVALID, "strides must not be negative");
  if (N == 0 || (n == 0 && accumulate)) return KGC_OK;
  if (!dW || (n > 0 && (!G || !ids))) return handle_fail(hd, KGC_E_INVALID, "NULL where data is required");
  const int64_t sg = size_of(g_dtype), sw = size_of(dw_dtype);
  if (!aligned(dW, sw) || (n > 0 && (!aligned(G, sg) || !aligned(ids, 4)))) return handle_fail(hd, KGC_E_INVALID, "misaligned pointer");
  const GradPlan p = plan_grad(n, N, d);
  if (p.bytes && (!work || work_bytes < p.bytes || !aligned(work, 16)))
    return handle_fail(hd, KGC_E_INVALID, "work must be 16-byte aligned and hold kgc_lookup_grad_bytes(n, N, d) bytes");
  const uint64_t wb = span(N, ldw, d, sw), gb = span(n, ldg, d, sg), ib = span(n, sid, 1, 4);
  if (overlap(dW, wb, G, gb) || overlap(dW, wb, ids, ib) || overlap(work, p.bytes, G, gb) || overlap(work, p.bytes, ids, ib) ||
      overlap(work, p.bytes, dW, wb))
    return handle_fail(hd, KGC_E_INVALID, "dW and work must not overlap another argument");
  GradArgs a{};
  a.G = G; a.ids = ids; a.dW = dW; a.n = n; a.ldg = ldg; a.sid = sid; a.N = N; a.ldw = ldw; a.d = d;
  a.accumulate = accumulate; a.scale = scale;
  const bool bg = g_dtype == KGC_BF16, bw = dw_dtype == KGC_BF16;
  if (bg) bw ? launch_grad<uint16_t, uint16_t>(v.stream, a, p, (char*)work) : launch_grad<uint16_t, float>(v.stream, a, p, (char*)work);
  else bw ? launch_grad<float, uint16_t>(v.stream, a, p, (char*)work) : launch_grad<float, float>(v.stream, a, p, (char*)work);
  return finish(hd);
}

uint64_t kgc_table4_bytes(int64_t N, int32_t d) {
  if (N < 0 || N > kLimitRows || d < 1 || d > kLimitD) return 0;
  return (uint64_t)((N + kTable4Rows - 1) / kTable4Rows) * (uint64_t)((d + kTable4Group - 1) / kTable4Group) * kTable4Bytes;
}

int kgc_pack4(kgc_handle* hd, const void* W, int64_t N, int64_t ldw, int32_t d, void* table, uint64_t table_bytes, float* sq) {
  HandleView v;
  const int rc = begin(hd, d, &v);
  if (rc != KGC_OK) return rc;
  if (N < 0 || N > kLimitRows) return handle_fail(hd, KGC_E_INVALID, "N out of range");
  if (!is_stride(ldw, 0)) return handle_fail(hd, KGC_E_INVALID, "strides must not be negative");
  if (N == 0) return KGC_OK;
  if (!W || !table) return handle_fail(hd, KGC_E_INVALID, "NULL where data is required");
  const int64_t sw = size_of(v.dtype);
  const uint64_t need = kgc_table4_bytes(N, d), wb = span(N, ldw, d, sw), qb = sq ? (uint64_t)N * 4 : 0;
  if (!aligned(W, sw) || !aligned(sq, 4)) return handle_fail(hd, KGC_E_INVALID, "misaligned pointer");
  if (table_bytes < need || !aligned(table, 16))
    return handle_fail(hd, KGC_E_INVALID, "table must be 16-byte aligned and hold kgc_table4_bytes(N, d) bytes");
  if (overlap(table, need, W, wb) || overlap(sq, qb, W, wb) || overlap(sq, qb, table, need))
    return handle_fail(hd, KGC_E_INVALID, "table and sq must not overlap another argument");
  Pack4Args a{};
  a.W = W; a.N = N; a.ldw = ldw; a.d = d; a.groups = (d + kTable4Group - 1) / kTable4Group;
  a.table = (char*)table; a.sq = sq;
  const unsigned grid = (unsigned)((N + 255) / 256);            // (below 2^24)
  if (v.dtype == KGC_BF16) k_pack4<uint16_t><<<grid, 256, 0, v.stream>>>(a);
  else k_pack4<float><<<grid, 256, 0, v.stream>>>(a);
  return finish(hd);
}

int kgc_scores4(kgc_handle* hd, const void* table, int64_t N, int32_t d, const void* x, int32_t x_dtype, int64_t ldx, int64_t n,
                float alpha, const float* c, float beta, void* y, int32_t y_dtype, int64_t ldy) {
  HandleView v;
  const int rc = begin(hd, d, &v);
  if (rc != KGC_OK) return rc;
  if (!is_type(x_dtype) || !is_type(y_dtype)) return handle_fail(hd, KGC_E_INVALID, "x_dtype and y_dtype must be KGC_F32 or KGC_BF16");
  if (N < 0 || N > kLimitRows) return handle_fail(hd, KGC_E_INVALID, "N out of range");
  if (n < 0 || n > kScores4Queries) return handle_fail(hd, KGC_E_INVALID, "n must be in [0, 1048560]");
  if (!is_stride(ldx, 0)) return handle_fail(hd, KGC_E_INVALID, "strides must not be negative");
  if (!is_stride(ldy, N)) return handle_fail(hd, KGC_E_INVALID, "ldy must be at least N");
  if (N == 0 || n == 0) return KGC_OK;
  if (!table || !x || !y) return handle_fail(hd, KGC_E_INVALID, "NULL where data is required");
  const int64_t sx = size_of(x_dtype), sy = size_of(y_dtype);
  if (!aligned(table, 16) || !aligned(x, sx) || !aligned(y, sy) || !aligned(c, 4)) return handle_fail(hd, KGC_E_INVALID, "misaligned pointer");
  const uint64_t yb = span(n, ldy, N, sy);
  if (overlap(y, yb, table, kgc_table4_bytes(N, d)) || overlap(y, yb, x, span(n, ldx, d, sx)) || overlap(y, yb, c, c ? (uint64_t)N * 4 : 0))
    return handle_fail(hd, KGC_E_INVALID, "y overlaps an input");
  Scores4Args a{};
  a.table = (const char*)table; a.N = N; a.d = d; a.groups = (d + kTable4Group - 1) / kTable4Group;
  a.x = x; a.ldx = ldx; a.n = n; a.alpha = alpha; a.c = c; a.beta = beta; a.y = y; a.ldy = ldy;
  const bool bx = x_dtype == KGC_BF16, by = y_dtype == KGC_BF16;
  if (bx) by ? launch_scores4_any<uint16_t, uint16_t>(v.stream, a) : launch_scores4_any<uint16_t, float>(v.stream, a);
  else by ? launch_scores4_any<float, uint16_t>(v.stream, a) : launch_scores4_any<float, float>(v.stream, a);
  return finish(hd);
}

int kgc_adjust(kgc_handle* hd, const kgc_adjustment* j) {
  if (!hd) return KGC_E_INVALID;
  if (!j) return handle_fail(hd, KGC_E_INVALID, "the adjustment is NULL");
  HandleView v;
  const int rc = begin(hd, 1, &v);
  if (rc != KGC_OK) return rc;
  if (!is_type(j->dtype)) return handle_fail(hd, KGC_E_INVALID, "dtype must be KGC_F32 or KGC_BF16");
  if (j->reserved != 0) return handle_fail(hd, KGC_E_INVALID, "reserved must be zero");
  if (j->n < 0 || j->n > kLimitRows || j->N < 0 || j->N > kLimitRows) return handle_fail(hd, KGC_E_INVALID, "n or N out of range");
  const int64_t n = j->n, N = j->N, words = (N + 31) / 32, sz = size_of(j->dtype);
  if (!is_stride(j->ld_scores, 0) || (j->allowed && !is_stride(j->ld_allowed, 0)))
    return handle_fail(hd, KGC_E_INVALID, "strides must not be negative");
  if (!is_stride(j->ld_out, N)) return handle_fail(hd, KGC_E_INVALID, "ld_out must be at least N");
  if (j->allowed && (j->masks < 1 || j->masks > kLimitRows)) return handle_fail(hd, KGC_E_INVALID, "masks out of range");
  if (j->allowed && !j->mask_row && j->masks != 1 && j->masks != n)
    return handle_fail(hd, KGC_E_INVALID, "without mask_row there is one mask, or one for each row");
  if (j->mask_row && !j->allowed) return handle_fail(hd, KGC_E_INVALID, "mask_row without allowed");
  const bool known = j->known_offsets != nullptr, seen = j->seen_offsets != nullptr;
  if (j->known_count < 0 || j->seen_count < 0 || (!known && (j->known_ids || j->known_count)) || (!seen && (j->seen_ids || j->seen_count)) ||
      (j->known_count > 0 && !j->known_ids) || (j->seen_count > 0 && !j->seen_ids))
    return handle_fail(hd, KGC_E_INVALID, "a list is offsets, ids and the number of ids");
  if (!std::isfinite(j->repeat) || !(j->repeat > 0.f) || !std::isfinite(j->presence) || !std::isfinite(j->frequency))
    return handle_fail(hd, KGC_E_INVALID, "repeat must be positive, presence and frequency finite");
  if (n == 0 || N == 0) return KGC_OK;
  if (!j->scores || !j->out) return handle_fail(hd, KGC_E_INVALID, "NULL where data is required");
  if (!aligned(j->scores, sz) || !aligned(j->out, sz) || !aligned(j->bias, 4) || !aligned(j->allowed, 4) || !aligned(j->mask_row, 4) ||
      !aligned(j->known_offsets, 8) || !aligned(j->known_ids, 4) || !aligned(j->seen_offsets, 8) || !aligned(j->seen_ids, 4))
    return handle_fail(hd, KGC_E_INVALID, "misaligned pointer");
  const bool in_place = j->scores == j->out;
  if (in_place && j->ld_scores != j->ld_out) return handle_fail(hd, KGC_E_INVALID, "in place, ld_scores and ld_out must be equal");
  const uint64_t ob = span(n, j->ld_out, N, sz);
  if ((!in_place && overlap(j->out, ob, j->scores, span(n, j->ld_scores, N, sz))) || overlap(j->out, ob, j->bias, j->bias ? (uint64_t)N * 4 : 0) ||
      overlap(j->out, ob, j->allowed, j->allowed ? span(j->masks, j->ld_allowed, words, 4) : 0) ||
      overlap(j->out, ob, j->mask_row, j->mask_row ? (uint64_t)n * 4 : 0) ||
      overlap(j->out, ob, j->known_offsets, known ? (uint64_t)(n + 1) * 8 : 0) || overlap(j->out, ob, j->known_ids, (uint64_t)j->known_count * 4) ||
      overlap(j->out, ob, j->seen_offsets, seen ? (uint64_t)(n + 1) * 8 : 0) || overlap(j->out, ob, j->seen_ids, (uint64_t)j->seen_count * 4))
    return handle_fail(hd, KGC_E_INVALID, "out overlaps an input");
  AdjustArgs a{};
  a.in = j->scores; a.out = j->out; a.n = n; a.N = N; a.ldi = j->ld_scores; a.ldo = j->ld_out;
  a.bias = j->bias; a.allowed = j->allowed; a.masks = j->masks; a.ldm = j->ld_allowed; a.mask_row = j->mask_row;
  if (j->known_count > 0) { a.known_off = j->known_offsets; a.known = j->known_ids; a.n_known = j->known_count; }
  if (j->seen_count > 0) { a.seen_off = j->seen_offsets; a.seen = j->seen_ids; a.n_seen = j->seen_count; }
  a.repeat = j->repeat; a.presence = j->presence; a.frequency = j->frequency;
  if (in_place && !a.bias && !a.allowed && !a.known && !a.seen) return KGC_OK;
  if (j->dtype == KGC_BF16) launch_adjust<uint16_t>(v.stream, a, in_place);
  else launch_adjust<float>(v.stream, a, in_place);
  return finish(hd);
}

}  // extern "C"
