// Kernels of the operators on embedding tables (gfx950, wave64).
#pragma once
#include <hip/hip_runtime.h>

#include "kgc_device.h"

namespace kgc {

// Vectors of a row.  Rows start wherever the caller's stride puts them, so the types ask for the alignment of an element
// only; global loads and stores of 8 and 16 bytes need no more on this chip.
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));

// to bfloat16: nearest, ties to even, a NaN of any payload stays a NaN
__device__ __forceinline__ uint16_t to_bf16(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// four elements from p on, `left` of them there (the others are 0)
template <typename T>
__device__ __forceinline__ f32x4_t ld4(const T* p, int left) {
  f32x4_t v = {0.f, 0.f, 0.f, 0.f};
  if (left >= 4) {
    if constexpr (sizeof(T) == 4) {
      const u32x4_any w = *(const u32x4_any*)p;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
    } else {
      const u32x2_any w = *(const u32x2_any*)p;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < left) {
        if constexpr (sizeof(T) == 4) v[i] = p[i];
        else v[i] = bf16_to_f32(p[i]);
      }
  }
  return v;
}

// A float32 result in the storage type: the one rounding of an output (nearest, ties to even).  STREAM: stored past the caches, for
// what is written once beside tables and gradients that are read again.
template <typename T, bool STREAM = false>
__device__ __forceinline__ void st4(T* p, f32x4_t v, int left) {
  if (left >= 4) {
    if constexpr (sizeof(T) == 4) {
      u32x4_any w;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(v[i]);
      if constexpr (STREAM) __builtin_nontemporal_store(w, (u32x4_any*)p);
      else *(u32x4_any*)p = w;
    } else {
      const u32x2_any w = __builtin_bit_cast(u32x2_any, __builtin_convertvector(v, bf16x4_t));
      if constexpr (STREAM) __builtin_nontemporal_store(w, (u32x2_any*)p);
      else *(u32x2_any*)p = w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < left) {
        if constexpr (sizeof(T) == 4) p[i] = v[i];
        else p[i] = to_bf16(v[i]);
      }
  }
}

// V elements as they lie in memory, and as float32.  Loads are asked for without a branch and widened where they are used: a branch or a
// conversion between two loads has the second wait for the first.
template <typename T, int V>
struct Raw {
  static constexpr int kWords = V * (int)sizeof(T) / 4;
  uint32_t w[kWords ? kWords : 1];
};
template <typename T, int V>
__device__ __forceinline__ Raw<T, V> ld_raw(const T* p) {
  Raw<T, V> r;
  if constexpr (V * sizeof(T) >= 16) {
#pragma unroll
    for (int k = 0; k < Raw<T, V>::kWords / 4; ++k) {
      const u32x4_any v = ((const u32x4_any*)p)[k];
#pragma unroll
      for (int i = 0; i < 4; ++i) r.w[4 * k + i] = v[i];
    }
  } else if constexpr (V * sizeof(T) == 8) {
    const u32x2_any v = *(const u32x2_any*)p;
    r.w[0] = v[0];
    r.w[1] = v[1];
  } else {
    static_assert(V == 1, "");
    if constexpr (sizeof(T) == 4) r.w[0] = __float_as_uint(*p);
    else r.w[0] = *p;
  }
  return r;
}
template <typename T, int V>
__device__ __forceinline__ float raw_elem(const Raw<T, V>& r, int i) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(r.w[i]);
  else return __uint_as_float(i & 1 ? r.w[i / 2] & 0xFFFF0000u : r.w[i / 2] << 16);
}
template <typename T, int V, bool STREAM>
__device__ __forceinline__ void st_vec(T* p, const float (&v)[V]) {
  if constexpr (V == 1) {
    if constexpr (sizeof(T) == 4) *p = v[0];
    else *p = to_bf16(v[0]);
  } else if constexpr (V == 8 && sizeof(T) == 2) {
    typedef __bf16 bf16x8_v __attribute__((ext_vector_type(8)));
    typedef float f32x8_v __attribute__((ext_vector_type(8)));
    const u32x4_any w = __builtin_bit_cast(u32x4_any, __builtin_convertvector(f32x8_v{v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]}, bf16x8_v));
    if constexpr (STREAM) __builtin_nontemporal_store(w, (u32x4_any*)p);
    else *(u32x4_any*)p = w;
  } else {
#pragma unroll
    for (int k = 0; k < V / 4; ++k) st4<T, STREAM>(p + 4 * k, f32x4_t{v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]}, 4);
  }
}

// ---- lookup: out[i] = sa A[ia[i]] + sb B[ib[i]] ----
struct LookupArgs {
  const void* A; const int32_t* ia; int64_t na, lda, sia; float sa;
  const void* B; const int32_t* ib; int64_t nb, ldb, sib; float sb;
  void* out; int64_t n, ldo;
  int d, vpr, rows;            // rows: output rows of a workgroup's tile; vpr: vectors of a row
  uint32_t magic;              // ceil(2^20 / vpr): item / vpr for the fewer than 4,096 items of a tile
};
constexpr int kLookupRows = 256;      // most rows of a tile

// A workgroup takes a tile of whole rows: their ids to the LDS, then a thread four vectors of V elements (16 bytes; single elements
// where a row is shorter) at a time.  A row's last vector ends with the row and overlaps the one before, which writes the same
// values.  Bound by bytes: a million rows of 128 in bfloat16 from two tables (Zipf's law, 321 MB with every table row once) take 78 to 83
// us, 4 TB/s; with every lane reading its own id and checking its own row's end 174, stored through the caches 98.
template <typename TI, typename TO, bool TWO, int V>
__global__ __launch_bounds__(256) void k_lookup(const LookupArgs a) {
  __shared__ int32_t id[2][kLookupRows];
  for (int64_t row0 = (int64_t)blockIdx.x * a.rows; row0 < a.n; row0 += (int64_t)gridDim.x * a.rows) {
    const int rows = (int)min((int64_t)a.rows, a.n - row0), items = rows * a.vpr;
    if ((int)threadIdx.x < rows) {
      id[0][threadIdx.x] = a.ia[(row0 + threadIdx.x) * a.sia];
      if (TWO) id[1][threadIdx.x] = a.ib[(row0 + threadIdx.x) * a.sib];
    }
    __syncthreads();
    for (int base = threadIdx.x; base < items; base += 1024) {
      int row[4], col[4];
      bool in_a[4], in_b[4];
      Raw<TI, V> x[4], y[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int it = min(base + 256 * u, items - 1);          // (the last vector once more)
        row[u] = (int)(((uint32_t)it * a.magic) >> 20);
        col[u] = min((it - row[u] * a.vpr) * V, a.d - V);
        const int32_t i = id[0][row[u]];
        in_a[u] = i >= 0 && i < a.na;
        x[u] = ld_raw<TI, V>((const TI*)a.A + (in_a[u] ? (int64_t)i * a.lda : 0) + col[u]);
        if (TWO) {
          const int32_t j = id[1][row[u]];
          in_b[u] = j >= 0 && j < a.nb;
          y[u] = ld_raw<TI, V>((const TI*)a.B + (in_b[u] ? (int64_t)j * a.ldb : 0) + col[u]);
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        float v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          v[i] = in_a[u] ? a.sa * raw_elem(x[u], i) : 0.f;
          if (TWO) v[i] += in_b[u] ? a.sb * raw_elem(y[u], i) : 0.f;
        }
        st_vec<TO, V, true>((TO*)a.out + (row0 + row[u]) * a.ldo + col[u], v);
      }
    }
    __syncthreads();
  }
}

// ---- gradient of a lookup: dW[v] (+)= scale * sum over i with ids[i] == v of G[i] ----
//
// The sums are taken in an order that depends on the ids and on n, N and d alone, not on strides, types or what they are added to, so that two
// calls give the same bits.  Few ids: a workgroup looks its id up in all of them (k_grad_few).  More: the ids are grouped with their positions in order (k_sort_once, or a stable radix sort, least significant digit first),
// the sorted list is cut into chunks that a team of lanes each sums row by row (k_grad_sum), and sums that reach over chunk borders are
// joined from the chunks' parts (k_grad_join): a row that occurs once and one that occurs a million times cost the same per
// occurrence.
struct GradArgs {
  const void* G; const int32_t* ids; void* dW;
  int64_t n, ldg, sid, N, ldw;
  int d, dp, accumulate; float scale;
  const uint2* pair;                               // sorted: id (N: names no row) and where it stood
  float* head; float* tail;                        // chunks x dp: the sum a chunk begins with, ends with, if it is a part
  int64_t chunks; int chunk;
};

// A lane's four columns from col on, asked for without a branch: where fewer than four are left, the last four of the row instead
// (rows of fewer: those that are there, repeated).
template <typename TG, bool NARROW>
__device__ __forceinline__ Raw<TG, 4> grad_load(const GradArgs& a, int64_t row, int col) {
  const TG* p = (const TG*)a.G + row * a.ldg;
  if constexpr (!NARROW) return ld_raw<TG, 4>(p + min(col, a.d - 4));
  Raw<TG, 4> r;
  if constexpr (sizeof(TG) == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) r.w[i] = __float_as_uint(p[min(i, a.d - 1)]);
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) r.w[i] = (uint32_t)p[min(2 * i, a.d - 1)] | ((uint32_t)p[min(2 * i + 1, a.d - 1)] << 16);
  }
  return r;
}
template <typename TG>
__device__ __forceinline__ f32x4_t widen(const Raw<TG, 4>& r) {
  return f32x4_t{raw_elem(r, 0), raw_elem(r, 1), raw_elem(r, 2), raw_elem(r, 3)};
}

// the sum of columns that grad_load asked for, to a row of dW; no ids: the row is 0 whatever the scale
template <typename TW>
__device__ __forceinline__ void grad_store(const GradArgs& a, int64_t row, int col, f32x4_t sum, bool named = true) {
  TW* p = (TW*)a.dW + row * a.ldw;
  const int left = a.d - col;
  f32x4_t v = sum * (named ? a.scale : 0.f);
  if (left >= 4) {
    if (a.accumulate) v = v + ld4((const TW*)p + col, 4);
    st4<TW, true>(p + col, v, 4);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = a.d >= 4 ? a.d - 4 + i : i;
      if (c >= col && c < a.d) {
        float x = v[i];
        if constexpr (sizeof(TW) == 4) p[c] = a.accumulate ? p[c] + x : x;
        else p[c] = to_bf16(a.accumulate ? bf16_to_f32(p[c]) + x : x);
      }
    }
  }
}

// rows of zeros: the vectors first, first + step, ... below last of rows x cols elements
struct ZeroArgs {
  void* p; int64_t rows, cols, ld, per_launch;     // per_launch: vectors that one of the sort's launches clears
};
template <typename T>
__device__ __forceinline__ void zero_rows(const ZeroArgs& z, int64_t first, int64_t step, int64_t last) {
  const int64_t vpr = (z.cols + 3) / 4;
  last = min(last, z.rows * vpr);
  for (int64_t it = first; it < last; it += step) {
    const int64_t r = z.rows == 1 ? 0 : it / vpr, c = (it - r * vpr) * 4, left = z.cols - c;
    st4<T, true>((T*)z.p + r * z.ld + c, f32x4_t{0.f, 0.f, 0.f, 0.f}, (int)(left < 4 ? left : 4));
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_zero_rows(const ZeroArgs z) {
  zero_rows<T>(z, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256, z.rows * ((z.cols + 3) / 4));
}

constexpr int kGradFew = 8192;                      // most ids that k_grad_few can list

// One workgroup per id (BY_ROW: per row of dW, which then needs no clearing); that of an id that stands further up has nothing to do,
// nor has that of a row that none names when the sums are added to it.
// Each wave lists the places of its share of the ids that match and sums their rows, T lanes a row.  Bound by latency: 128 ids in 2,000
// rows of 32: 4.2 us, 1,000 in 1,345 rows of 100: 4.4, 8,000: 10.7.
template <typename TG, typename TW, bool BY_ROW, int T, bool NARROW>
__global__ __launch_bounds__(256) void k_grad_few(const GradArgs a) {
  __shared__ uint16_t place[4][kGradFew / 4];
  __shared__ __align__(16) float red[4][T * 4];
  __shared__ int named[4];
  const int n = (int)a.n, lane = lane_id(), wave = threadIdx.x >> 6;
  const int target = blockIdx.x;
  const int32_t id = BY_ROW ? target : a.ids[target * a.sid];
  if (!BY_ROW && (id < 0 || id >= a.N)) return;
  int found = 0;
  bool earlier = false;
  for (int j0 = wave * 64; j0 < n; j0 += 1024) {
    int32_t x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int j = j0 + 256 * u + lane;
      x[u] = j < n ? a.ids[j * a.sid] : -1;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int j = j0 + 256 * u + lane;
      const bool is = j < n && x[u] == id;
      const unsigned long long m = __ballot(is);
      if (is) {
        place[wave][found + __popcll(m & ((1ull << lane) - 1))] = (uint16_t)j;
        earlier = earlier || (!BY_ROW && j < target);
      }
      found += __popcll(m);
    }
  }
  bool any = true;
  if (BY_ROW && !a.accumulate) {                    // (0.4 us less than __syncthreads_or)
    if (lane == 0) named[wave] = found;
    __syncthreads();
    any = (named[0] | named[1] | named[2] | named[3]) != 0;
  } else if (BY_ROW ? !__syncthreads_or(found) : __syncthreads_or(earlier)) {
    return;
  }
  const int team = lane / T, sub = lane % T;
  constexpr int kTeams = 64 / T;
  for (int col0 = 0; col0 < a.d; col0 += T * 4) {
    const int col = col0 + sub * 4;
    f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
    for (int k = team; k < found; k += 8 * kTeams) {
      Raw<TG, 4> x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = grad_load<TG, NARROW>(a, place[wave][min(k + u * kTeams, found - 1)], col);
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (k + u * kTeams < found) sum = sum + widen(x[u]);
    }
#pragma unroll
    for (int o = T; o < 64; o <<= 1)
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] += __shfl_xor(sum[i], o);
    if (lane < T) *(f32x4_t*)&red[wave][sub * 4] = sum;
    __syncthreads();
    if (threadIdx.x < T && col < a.d) {
#pragma unroll
      for (int w = 1; w < 4; ++w) sum = sum + *(const f32x4_t*)&red[w][sub * 4];
      grad_store<TW>(a, id, col, sum, any);
    }
    __syncthreads();
  }
}

// ---- the sort ----
//
// A pass counts the digits of every tile, then scatters.  Its launches hold more workgroups than there are tiles where dW has to be
// cleared: the sort waits for memory most of the time and leaves the bandwidth to them (14,000 ids in 640,000 rows of 64: 57 us for both,
// 68 with all of the clearing in the first launch).  Bound by latency, 4 us a count and 7 a scatter, up to 100,000 ids; a million in three
// columns (12 MB to read twice) take 92 us without clearing.
constexpr int kSortBits = 11;                       // most bits of a digit
// Up to this many counts (a quarter of it in tiles of 4,096 ids) every scattering workgroup adds them up itself, beyond them k_sort_scan does:
// 100,000 ids in 15,000 rows 35 us, 39 with k_sort_scan; 400,000 ids 83, 70
constexpr int kSortSums = 16384;

struct SortArgs {
  const int32_t* ids; int64_t sid; uint32_t N;      // first pass: the caller's ids
  const uint2* in; uint2* out;                      // later passes; pairs of id and position
  uint32_t* hist; uint32_t* total;                  // hist[tile][digit] (with k_sort_scan: of the tiles before), total[digit]
  int64_t n; int tiles, shift, bits, scanned, rows;
  ZeroArgs zero; int64_t zero_first;                // vectors of dW from zero_first on are cleared beside this launch
};

__device__ __forceinline__ uint32_t sort_key(const SortArgs& a, int64_t i, bool first) {
  if (!first) return a.in[i].x;
  const uint32_t id = (uint32_t)a.ids[i * a.sid];
  return id < a.N ? id : a.N;                       // (negative ids are large as unsigned numbers)
}

template <typename TW>
__device__ __forceinline__ void sort_zero(const SortArgs& a) {
  const int64_t b = (int64_t)blockIdx.x - a.tiles, groups = (int64_t)gridDim.x - a.tiles;
  zero_rows<TW>(a.zero, a.zero_first + b * blockDim.x + threadIdx.x, groups * blockDim.x, a.zero_first + a.zero.per_launch);
}

// K: ids per thread; a tile holds 256 K
template <typename TW, bool FIRST, int K>
__global__ __launch_bounds__(256) void k_sort_count(const SortArgs a) {
  __shared__ uint32_t c[1 << kSortBits];
  if ((int)blockIdx.x >= a.tiles) return sort_zero<TW>(a);
  const int bins = 1 << a.bits;
  for (int b = threadIdx.x; b < bins; b += 256) c[b] = 0;
  const int64_t base = (int64_t)blockIdx.x * (256 * K);
  uint32_t key[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int64_t i = base + k * 256 + threadIdx.x;
    key[k] = i < a.n ? sort_key(a, i, FIRST) : 0u;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k)
    if (base + k * 256 + threadIdx.x < a.n) atomicAdd(&c[(key[k] >> a.shift) & (bins - 1)], 1u);
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += 256) a.hist[(int64_t)blockIdx.x * bins + b] = c[b];
}

// Many counts: sixteen threads a digit turn its tiles' counts into the counts before them.
__global__ __launch_bounds__(1024) void k_sort_scan(uint32_t* hist, uint32_t* total, int tiles, int bins) {
  __shared__ uint32_t part[16][64];
  const int lane = lane_id(), g = threadIdx.x >> 6, b = blockIdx.x * 64 + lane;
  const int per = (tiles + 15) / 16, t0 = g * per, t1 = min(t0 + per, tiles);
  uint32_t sum = 0;
  if (b < bins) {
#pragma unroll 8
    for (int t = t0; t < t1; ++t) sum += hist[(int64_t)t * bins + b];
  }
  part[g][lane] = sum;
  __syncthreads();
  uint32_t run = 0, all = 0;
  for (int k = 0; k < 16; ++k) {
    if (k < g) run += part[k][lane];
    all += part[k][lane];
  }
  if (b >= bins) return;
#pragma unroll 8
  for (int t = t0; t < t1; ++t) {
    const uint32_t x = hist[(int64_t)t * bins + b];
    hist[(int64_t)t * bins + b] = run;
    run += x;
  }
  if (g == 0) total[b] = all;
}

// the lanes whose digit is this lane's, of those that have one
__device__ __forceinline__ unsigned long long same_digit(uint32_t digit, int bits, bool in) {
  unsigned long long same = __ballot(in);
  for (int b = 0; b < bits; ++b) {
    const unsigned long long one = __ballot((digit >> b) & 1u);
    same &= (digit >> b) & 1u ? one : ~one;
  }
  return same;
}

// A wave takes its share of the tile in rounds of 64 ids; in a round the lanes of one digit find one another by ballots over its bits, so
// ranks within the wave follow the order of the ids.
template <typename TW, bool FIRST, int K>
__global__ __launch_bounds__(256) void k_sort_scatter(const SortArgs a) {
  constexpr int kThreads = 256, W = 4;
  extern __shared__ __align__(16) uint32_t lds[];   // c[W][bins], all[bins], first[bins]
  __shared__ uint32_t wsum[W];
  if ((int)blockIdx.x >= a.tiles) return sort_zero<TW>(a);
  const int bins = 1 << a.bits, wave = threadIdx.x >> 6, lane = lane_id();
  uint32_t *c = lds, *all = lds + W * bins, *first = all + bins;
  const int64_t tile = (int64_t)blockIdx.x * (kThreads * K), base = tile + wave * (64 * K);
  uint32_t key[K], pos[K], rank[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int64_t i = base + k * 64 + lane;
    key[k] = pos[k] = 0;
    if (i < a.n) {
      if (FIRST) {
        key[k] = sort_key(a, i, true);
        pos[k] = (uint32_t)i;
      } else {
        const uint2 p = a.in[i];
        key[k] = p.x;
        pos[k] = p.y;
      }
    }
  }
  for (int b = threadIdx.x; b < (W + 2) * bins; b += kThreads) lds[b] = 0;
  __syncthreads();
  // ids of every digit in all tiles and in the tiles before this one
  if (a.scanned) {
    for (int b = threadIdx.x; b < bins; b += kThreads) {
      first[b] = a.hist[(int64_t)blockIdx.x * bins + b];
      all[b] = a.total[b];
    }
  } else {
    const int sets = bins < kThreads ? kThreads / bins : 1;      // threads that share a digit, each every sets-th tile
    for (int b = threadIdx.x % bins; b < bins; b += kThreads) {
      uint32_t sum = 0, before = 0;
#pragma unroll 8
      for (int t = threadIdx.x / bins % sets; t < a.tiles; t += sets) {
        const uint32_t x = a.hist[(int64_t)t * bins + b];
        sum += x;
        if (t < (int)blockIdx.x) before += x;
      }
      if (sum) atomicAdd(&all[b], sum);
      if (before) atomicAdd(&first[b], before);
    }
  }
  const unsigned long long below = (1ull << lane) - 1;
  uint32_t* mine_c = c + wave * bins;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const bool in = base + k * 64 + lane < a.n;
    const uint32_t dg = (key[k] >> a.shift) & (bins - 1);
    const unsigned long long same = same_digit(dg, a.bits, in);
    uint32_t before = 0;
    if (in) {
      before = __hip_atomic_load(mine_c + dg, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      rank[k] = before + __popcll(same & below);
    }
    __builtin_amdgcn_wave_barrier();                // every lane has read the count before the first of a digit moves it on
    if (in && (same & below) == 0)
      __hip_atomic_store(mine_c + dg, before + (uint32_t)__popcll(same), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  // where the digits of this tile go: all ids of smaller digits, those of this digit in earlier tiles, and in earlier waves
  const int per = (bins + kThreads - 1) / kThreads; // digits of a thread, neighbours
  uint32_t mine = 0;
  for (int k = 0; k < per; ++k)
    if ((int)threadIdx.x * per + k < bins) mine += all[threadIdx.x * per + k];
  uint32_t sum = mine;
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t up = __shfl_up(sum, o);
    if (lane >= o) sum += up;
  }
  if (lane == 63) wsum[wave] = sum;
  __syncthreads();
  uint32_t run = sum - mine;
  for (int w = 0; w < wave; ++w) run += wsum[w];
  for (int k = 0; k < per; ++k) {
    const int b = threadIdx.x * per + k;
    if (b < bins) {
      uint32_t at = run + first[b];
      for (int w = 0; w < W; ++w) {
        const uint32_t x = c[w * bins + b];
        c[w * bins + b] = at;
        at += x;
      }
      run += all[b];
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k)
    if (base + k * 64 + lane < a.n) a.out[mine_c[(key[k] >> a.shift) & (bins - 1)] + rank[k]] = make_uint2(key[k], pos[k]);
}

// Not too many ids and rows: one launch in place of all passes.  The sums need the ids of a row side by side and in order, not the rows in
// order; so workgroup g takes the rows v with v % 256 == g, goes through all ids for theirs, which it lists and counts, and for the number of
// those of the workgroups before it, where its pairs begin.  (Rows side by side would leave the frequent ones to one workgroup where they have the
// smallest numbers.)  A call, us, us with the radix sort: 10,000 ids in 40,000 rows of 64: 16, 28; 32,768 in 15,000 of 100: 19, 27; of those, by
// Zipf's law: 24, 30; one id for all 32,768: 48, 44.  Bound by the trips to memory, then by the vector instructions for every id in every workgroup,
// which is why it ends at 49,152 ids (in 15,000 rows: 23, 31; by Zipf's law 28, 34; one id for all 52, 43) and, where the radix sort takes one pass
// (N < 512), at 16,384; and where the LDS ends: at 49,152 ids with 245,760 rows, at 47,104 with 262,144.
constexpr int kOnceAsk = 8;                        // ids of a lane asked for at a time (16: 1 us more for 5,000 ids)
constexpr int kOnceGroups = 256, kOnceRows = 1024, kOnceWaves = 16;
constexpr int kOnceStride = 4;                      // every workgroup reads what lies between the ids too: those further apart are copied first
constexpr int kOnceIds = 49152;                     // (places are kept in 16 bits)
__host__ __device__ inline int once_share(int64_t n) { return (int)((n + kOnceWaves * 64 - 1) / (kOnceWaves * 64)) * 64; }    // ids of a wave

// Ids further apart than kOnceStride, side by side.  The radix sort would put the rows in another order, and chunks would cut their sums in other
// places: the stride would show in the bits.  A call at a stride of 8, us, us with the radix sort: 5,000 ids in 100,000 rows of 64: 17.8, 28.8; 32,768 in
// 15,000 of 100: 21, 27; one id for all of them: 49, 43.
__global__ __launch_bounds__(256) void k_ids(const int32_t* ids, int64_t sid, int n, int32_t* out) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) out[i] = ids[i * sid];
}

// (registers for two workgroups a compute unit, so that clearing ones run beside these: 5,000 ids in 100,000 rows 22 -> 19 us)
template <typename TW>
__global__ __launch_bounds__(kOnceWaves * 64) __attribute__((amdgpu_waves_per_eu(8))) void k_sort_once(const SortArgs a) {
  extern __shared__ __align__(16) uint32_t lds[];   // c[waves][rows], then the places of every wave's ids
  __shared__ uint32_t wsum[kOnceWaves], wbelow[kOnceWaves], wnamed[kOnceWaves];
  if ((int)blockIdx.x >= kOnceGroups) return sort_zero<TW>(a);
  const int rows = a.rows, wave = threadIdx.x >> 6, lane = lane_id(), n = (int)a.n, share = once_share(n);
  const uint32_t group = blockIdx.x, sid = (uint32_t)a.sid;       // (at most kOnceStride: an id's offset has 32 bits)
  uint32_t* c = lds + wave * rows;
  uint16_t* place = (uint16_t*)(lds + kOnceWaves * rows) + wave * share;
  for (int b = threadIdx.x; b < kOnceWaves * rows; b += kOnceWaves * 64) lds[b] = 0;
  __syncthreads();
  const unsigned long long under = (1ull << lane) - 1;
  const int begin = __builtin_amdgcn_readfirstlane(wave) * share, end = min(begin + share, n);
  int found = 0, before = 0, named = 0;             // the wave's ids of this group, of earlier ones, of all
  // (masks of the lanes are counted beside the vector instructions, which bound this loop)
  auto look = [&](uint32_t key, int j, unsigned long long in) {
    const unsigned long long row = __ballot(key < a.N) & in, mine = row & __ballot(key % kOnceGroups == group);
    named += __popcll(row);
    before += __popcll(row & __ballot(key % kOnceGroups < group));
    if (!mine) return;
    if ((mine >> lane) & 1) place[found + __popcll(mine & under)] = (uint16_t)j;
    found += __popcll(mine);
  };
  int j0 = begin;
  for (; j0 + 64 * kOnceAsk <= end; j0 += 64 * kOnceAsk) {
    uint32_t key[kOnceAsk];
    const int32_t* p = a.ids + (uint32_t)j0 * sid;
#pragma unroll
    for (int u = 0; u < kOnceAsk; ++u) key[u] = (uint32_t)p[u * 64 * sid + lane * sid];
#pragma unroll
    for (int u = 0; u < kOnceAsk; ++u) look(key[u], j0 + u * 64 + lane, ~0ull);
  }
  if (j0 < end) {
    uint32_t key[kOnceAsk];
#pragma unroll
    for (int u = 0; u < kOnceAsk; ++u) key[u] = (uint32_t)a.ids[(uint32_t)min(j0 + u * 64 + lane, n - 1) * sid];
#pragma unroll
    for (int u = 0; u < kOnceAsk; ++u) look(key[u], j0 + u * 64 + lane, __ballot(j0 + u * 64 + lane < end));
  }
  if (lane == 0) wbelow[wave] = before, wnamed[wave] = named;
  // how many of them a row has.  A frequent row's are counted together: atomics on one address take their turns
  uint32_t pos[4], key[4];
  auto load = [&](int j0) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      pos[u] = place[min(j0 + u * 64 + lane, found - 1)];
      key[u] = (uint32_t)a.ids[pos[u] * sid];
    }
  };
  for (int j0 = 0; j0 < found; j0 += 64 * 4) {
    load(j0);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (j0 + u * 64 >= found) break;
      const bool in = j0 + u * 64 + lane < found;
      const uint32_t row = key[u] / kOnceGroups, one = __builtin_amdgcn_readfirstlane(row);
      const unsigned long long same = __ballot(in && row == one);
      if (lane == 0) atomicAdd(&c[one], (uint32_t)__popcll(same));
      if (in && row != one) atomicAdd(&c[row], 1u);
    }
  }
  __syncthreads();
  // where the rows of this workgroup go, a thread a row
  const int b = threadIdx.x;
  uint32_t mine = 0;
  if (b < rows)
    for (int w = 0; w < kOnceWaves; ++w) mine += lds[w * rows + b];
  uint32_t sum = mine;
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t up = __shfl_up(sum, o);
    if (lane >= o) sum += up;
  }
  if (lane == 63) wsum[wave] = sum;
  __syncthreads();
  uint32_t at = sum - mine, all = 0;
  for (int w = 0; w < kOnceWaves; ++w) {
    at += wbelow[w] + (w < wave ? wsum[w] : 0u);
    all += wnamed[w];
  }
  if (b < rows)
    for (int w = 0; w < kOnceWaves; ++w) {
      const uint32_t x = lds[w * rows + b];
      lds[w * rows + b] = at;
      at += x;
    }
  __syncthreads();
  for (int j0 = 0; j0 < found; j0 += 64 * 4) {
    if (found > 64 * 4) load(j0);                   // (fewer are there still)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (j0 + u * 64 >= found) break;
      const bool in = j0 + u * 64 + lane < found;
      const uint32_t row = key[u] / kOnceGroups;
      const uint32_t one = __builtin_amdgcn_readfirstlane(row);
      unsigned long long same = __ballot(in && row == one);
      if (same != __ballot(in)) same = same_digit(row, a.bits, in);
      const uint32_t first = __hip_atomic_load(c + row, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      if (in) a.out[first + __popcll(same & under)] = make_uint2(key[u], pos[u]);
      __builtin_amdgcn_wave_barrier();              // every lane has read the count before the first of a row moves it on
      if (in && (same & under) == 0)
        __hip_atomic_store(c + row, first + (uint32_t)__popcll(same), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      __builtin_amdgcn_wave_barrier();
    }
  }
  // ids that name no row come last
  for (int64_t i = (int64_t)all + blockIdx.x * (kOnceWaves * 64) + threadIdx.x; i < n; i += kOnceGroups * kOnceWaves * 64)
    a.out[i] = make_uint2(a.N, 0u);
}

// ---- the sums ----
// T lanes per chunk, M vectors of four columns per lane.  The chunk's pairs go to the LDS; rows of G are asked for U at a time, one step
// ahead of their sums, into two sets of registers in turn.  The sum moves on to the next row of dW where the id changes.  Bound by bytes:
// 250,000 rows of 100 in float32 for 18 rows: 22 us, 4.6 TB/s; a million of 128 in bfloat16 for 220,000 (Zipf's law, 370 MB): 90 us, 4.1 TB/s,
// 125 stored through the caches.
constexpr int kGradChunk = 256;                     // most ids of a chunk
template <typename TG, typename TW, int T, int M, bool NARROW>
__global__ __launch_bounds__(256) void k_grad_sum(const GradArgs a) {
  constexpr int U = M == 1 ? 8 : 8 / M;
  __shared__ uint2 pairs[256 / T][kGradChunk];
  const int team = threadIdx.x / T, lane = threadIdx.x % T;
  const int64_t ch = (int64_t)blockIdx.x * (256 / T) + team, b = ch * a.chunk;
  const int len = (int)max((int64_t)0, min((int64_t)a.chunk, a.n - b));
  uint32_t prior = ~0u, follow = ~0u;
  if (len > 0) {
    if (b > 0) prior = a.pair[b - 1].x;
    if (b + len < a.n) follow = a.pair[b + len].x;
  }
  for (int j = lane; j < len; j += T) pairs[team][j] = a.pair[b + j];
  __syncthreads();
  if (len == 0) return;
  const uint2* p = pairs[team];
  auto rows = [&](Raw<TG, 4> (&x)[U][M], int i) {                // (past the end the last row again)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = p[min(i + u, len - 1)].y;
#pragma unroll
      for (int m = 0; m < M; ++m) x[u][m] = grad_load<TG, NARROW>(a, at, (m * T + lane) * 4);
    }
  };
  uint32_t cur = p[0].x;
  bool part = prior == cur;                                      // the current sum began in an earlier chunk
  const bool goes_on = follow == p[len - 1].x;
  f32x4_t acc[M];
#pragma unroll
  for (int m = 0; m < M; ++m) acc[m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  auto emit = [&](float* parts) {
    if (cur >= (uint32_t)a.N) return;
#pragma unroll
    for (int m = 0; m < M; ++m) {
      const int col = (m * T + lane) * 4;
      if (col < a.d) {
        if (parts) *(f32x4_t*)(parts + ch * a.dp + col) = acc[m];
        else grad_store<TW>(a, cur, col, acc[m]);
      }
    }
  };
  auto add = [&](const Raw<TG, 4> (&x)[U][M], int i) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool in = i + u < len;
      const uint32_t id = p[min(i + u, len - 1)].x;
      if (id != cur) {
        emit(part ? a.head : nullptr);
        part = false;
        cur = id;
#pragma unroll
        for (int m = 0; m < M; ++m) acc[m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      }
#pragma unroll
      for (int m = 0; m < M; ++m)
        if (in) acc[m] = acc[m] + widen(x[u][m]);
    }
  };
  Raw<TG, 4> x0[U][M], x1[U][M];
  rows(x0, 0);
  for (int i = 0; i < len; i += 2 * U) {
    rows(x1, i + U);
    add(x0, i);
    rows(x0, i + 2 * U);
    add(x1, i + U);
  }
  emit(part ? a.head : (goes_on ? a.tail : nullptr));
}

constexpr int kJoinLong = 64;                        // parts from which on a sum is the whole workgroup's

// How many parts the sum of `id` that begins in chunk c has: its own and one in each following chunk that begins with the id.  The
// wave looks at the next 64 chunks; if they all do, it closes in from the widest steps on.
__device__ __forceinline__ int64_t grad_parts(const GradArgs& a, int64_t c, uint32_t id) {
  const int lane = lane_id();
  int64_t parts = 1;
  for (int64_t step = 1;;) {
    const int64_t q = c + parts + (lane + 1) * step - 1;
    const unsigned long long on = __ballot(q < a.chunks && a.pair[q * a.chunk].x == id);
    const int run = on == ~0ull ? 64 : __builtin_ctzll(~on);
    parts += run * step;
    if (run == 64) step *= 64;
    else if (step == 1) return parts;
    else step /= 64;
  }
}

// Sums that begin in a chunk and reach past it: the chunk's last part, then the first parts of the chunks it reaches into, each of
// the teams of a wave taking every (number of teams)-th part.  A wave takes `per_wave` chunks; long sums are left to the whole
// workgroup.  Bound by latency: 3 to 8 us.
template <typename TW, int T>
__global__ __launch_bounds__(1024) void k_grad_join(const GradArgs a, int per_wave) {
  extern __shared__ __align__(16) float red[];       // 16 x dp
  __shared__ int64_t long_chunk[32];                 // (long sums begin more than kJoinLong chunks apart, in 1,024 chunks at most)
  __shared__ int64_t long_parts[32];
  __shared__ int n_long;
  const int lane = lane_id(), wave = threadIdx.x >> 6;
  if (threadIdx.x == 0) n_long = 0;
  __syncthreads();
  const int64_t c0 = ((int64_t)blockIdx.x * 16 + wave) * per_wave;
  bool begins = false;
  if (lane < per_wave && c0 + lane < a.chunks) {
    const int64_t b = (c0 + lane) * a.chunk, e = b + a.chunk;
    if (e < a.n) {
      const uint32_t last = a.pair[e - 1].x, next = a.pair[e].x, prior = b > 0 ? a.pair[b - 1].x : ~0u;
      begins = last < (uint32_t)a.N && next == last && prior != last;
    }
  }
  // parts first, first + step, ... of the sum that begins in chunk c, columns from col on
  auto gather = [&](int64_t c, int64_t parts, int64_t first, int64_t step, int col) {
    f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
    for (int64_t j = first; j < parts; j += 4 * step) {
      f32x4_t x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int64_t q = j + u * step;
        x[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if (q < parts && col < a.d) x[u] = *(const f32x4_t*)((q ? a.head : a.tail) + (c + q) * a.dp + col);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) sum = sum + x[u];
    }
#pragma unroll
    for (int o = T; o < 64; o <<= 1)
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] += __shfl_xor(sum[i], o);
    return sum;
  };
  for (unsigned long long m = __ballot(begins); m; m &= m - 1) {
    const int64_t c = c0 + __builtin_ctzll(m);
    const uint32_t id = a.pair[c * a.chunk + a.chunk - 1].x;
    const int64_t parts = grad_parts(a, c, id);
    if (parts > kJoinLong) {
      if (lane == 0) {
        const int l = atomicAdd(&n_long, 1);
        long_chunk[l] = c;
        long_parts[l] = parts;
      }
      continue;
    }
    for (int col = (lane % T) * 4; col - (lane % T) * 4 < a.d; col += T * 4) {
      const f32x4_t sum = gather(c, parts, lane / T, 64 / T, col);
      if (lane < T && col < a.d) grad_store<TW>(a, id, col, sum);
    }
  }
  __syncthreads();
  const int longs = n_long;
  for (int l = 0; l < longs; ++l) {
    const int64_t c = long_chunk[l], parts = long_parts[l];
    const uint32_t id = a.pair[c * a.chunk + a.chunk - 1].x;
    for (int col = (lane % T) * 4; col - (lane % T) * 4 < a.d; col += T * 4) {
      const f32x4_t sum = gather(c, parts, wave * (64 / T) + lane / T, 16 * (64 / T), col);
      if (lane < T && col < a.d) *(f32x4_t*)(red + wave * a.dp + col) = sum;
    }
    __syncthreads();
    for (int col = threadIdx.x * 4; col < a.d; col += 4096) {
      f32x4_t sum = *(const f32x4_t*)(red + col);
      for (int w = 1; w < 16; ++w) sum = sum + *(const f32x4_t*)(red + w * a.dp + col);
      grad_store<TW>(a, id, col, sum);
    }
    __syncthreads();
  }
}

// ---- small tables ----
//
// A table of few and short rows (the relations' side of a graph with two dozen of them): no sort.  Every team of lanes keeps the whole
// table's sums in the LDS and adds its stretch of G to them in order, the workgroup adds up its teams' tables, and k_grad_table_join
// the workgroups'.  Bound by the bytes of G: 250,000 rows of 100 in float32 for 18 rows take 22 + 7 us, a call 29 (42 with the sort), for 44
// rows 30 (41); a million in bfloat16 for 18 rows 54 (80); 20,000 for 18 rows 12 (19).
struct TableArgs {
  const void* G; const int32_t* ids; void* dW;
  int64_t n, ldg, sid, ldw, per_team;
  int d, dp, N, blocks, accumulate; float scale;
  float* parts; uint32_t* named;                   // blocks x N x dp; blocks x N: ids of the row
};
// Two workgroups a compute unit; rows of at most 128 columns, with eight teams or more in a workgroup, may take one a compute unit (with four
// teams, 44 rows of 200 in bfloat16, a million ids: 144 us, 119 with the sort).
constexpr int kTableLds = 80 * 1024, kTableLdsOne = 156 * 1024;

template <typename TG, int T>
__global__ __launch_bounds__(256) void k_grad_table(const TableArgs a) {
  constexpr int kTeams = 256 / T, U = 8;
  extern __shared__ __align__(16) float acc[];     // [kTeams][N + 1][dp] (the last row: of ids that name none), then [N + 1] counts
  const int team = threadIdx.x / T, lane = threadIdx.x % T, col = min(lane * 4, a.dp - 4), words = kTeams * (a.N + 1) * a.dp;
  uint32_t* count = (uint32_t*)(acc + words);
  for (int k = threadIdx.x; k < words + a.N + 1; k += 256) acc[k] = 0.f;
  __syncthreads();
  const int64_t b = ((int64_t)blockIdx.x * kTeams + team) * a.per_team, e = min(b + a.per_team, a.n);
  float* mine = acc + team * (a.N + 1) * a.dp + col;
  auto ask = [&](Raw<TG, 4> (&x)[U], int32_t (&id)[U], int64_t i) {          // (past the end the last row again)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = min(i + u, a.n - 1);
      x[u] = ld_raw<TG, 4>((const TG*)a.G + at * a.ldg + min(lane * 4, a.d - 4));
      id[u] = a.ids[at * a.sid];
    }
  };
  auto add = [&](const Raw<TG, 4> (&x)[U], const int32_t (&id)[U], int64_t i) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int row = i + u < e && (uint32_t)id[u] < (uint32_t)a.N ? id[u] : a.N;
      if (lane * 4 < a.d) {
        f32x4_t* p = (f32x4_t*)(mine + row * a.dp);
        *p = *p + widen(x[u]);
      }
      if (lane == 0) atomicAdd(&count[row], 1u);
    }
  };
  Raw<TG, 4> x0[U], x1[U];
  int32_t id0[U], id1[U];
  if (b < e) {
    ask(x0, id0, b);
    for (int64_t i = b; i < e; i += 2 * U) {
      ask(x1, id1, i + U);
      add(x0, id0, i);
      ask(x0, id0, i + 2 * U);
      add(x1, id1, i + U);
    }
  }
  __syncthreads();
  float* parts = a.parts + (int64_t)blockIdx.x * a.N * a.dp;
  for (int k = threadIdx.x * 4; k < a.N * a.dp; k += 1024) {
    f32x4_t sum = *(const f32x4_t*)(acc + k);
#pragma unroll
    for (int t = 1; t < kTeams; ++t) sum = sum + *(const f32x4_t*)(acc + t * (a.N + 1) * a.dp + k);
    *(f32x4_t*)(parts + k) = sum;
  }
  for (int k = threadIdx.x; k < a.N; k += 256) a.named[(int64_t)blockIdx.x * a.N + k] = count[k];
}

// One workgroup per row and 64 columns: 16 threads side by side, 16 of them one above the other for every 16th part.
template <typename TW>
__global__ __launch_bounds__(256) void k_grad_table_join(const TableArgs a) {
  __shared__ __align__(16) float red[16][64];
  const int row = blockIdx.x, col = blockIdx.y * 64 + (threadIdx.x % 16) * 4, seg = threadIdx.x / 16;
  f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
  uint32_t named = 0;
  for (int k = seg; k < a.blocks; k += 8 * 16) {
    f32x4_t x[8];
    uint32_t c[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int q = min(k + 16 * u, a.blocks - 1);
      x[u] = *(const f32x4_t*)(a.parts + ((int64_t)q * a.N + row) * a.dp + min(col, a.dp - 4));
      c[u] = a.named[(int64_t)q * a.N + row];
    }
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (k + 16 * u < a.blocks) {
        sum = sum + x[u];
        named |= c[u];
      }
  }
  *(f32x4_t*)&red[seg][(threadIdx.x % 16) * 4] = sum;
  const bool any = __syncthreads_or((int)(named != 0));
  if (!any && a.accumulate) return;
  if (seg == 0 && col < a.d) {
#pragma unroll
    for (int k = 1; k < 16; ++k) sum = sum + *(const f32x4_t*)&red[k][threadIdx.x * 4];
    GradArgs g{};
    g.dW = a.dW; g.ldw = a.ldw; g.d = a.d; g.accumulate = a.accumulate; g.scale = a.scale;
    grad_store<TW>(g, row, col, sum, any);
  }
}

// ---- tables in 4 bits ----
//
// A value is an e2m1 code (a sign and a magnitude of 0, 0.5, 1, 1.5, 2, 3, 4, 6) times the bfloat16 scale of its 32 dimensions.  The
// code is the type that this chip widens to bfloat16 by itself, two values an instruction, exactly; so products go through the
// bf16 matrix pipes and the scale multiplies the float32 sum of a group.
//
// Layout: 64 rows x 32 dimensions are one block of 1,152 bytes, blocks of a row range one after the other.  First 64 x 16 bytes of
// codes: lane l of a wave finds in dword t of its 16 bytes the eight dimensions 8 (l / 16) ... of row 16 t + l % 16, which is the
// operand of the 16 x 16 x 32 matrix instruction; then 64 scales in the order of its results (lane's rows 16 t + 4 (l / 16) + i).
constexpr int kTable4Rows = 64, kTable4Group = 32;
constexpr int64_t kTable4Bytes = 1024 + 128;

struct Pack4Args {
  const void* W; int64_t N, ldw; int d, groups;
  char* table; float* sq;
};

// A wave packs 64 rows, a block of 32 dimensions at a time: lane l the dimensions 8 (l / 16) ... of the four rows 16 t + l % 16, whose four
// lanes share the largest magnitude.  Products of a scale (8 significant bits) with the middles between levels (3) and with the
// levels (2) are exact in float32, so the code is that of the nearest level, the even code of two as near; sq is the sum of exact
// squares in double, rounded once.  A million rows of 128 in bfloat16 (332 MB): 120 to 131 us (float32, 588 MB: 135); a thread a row took 393.  Smaller tables
// are bound by latency: a wave's groups follow one another, each after its loads, and N / 256 workgroups are few (15,000 rows of 100: 19 us, either type;
// 100,000 of 200: 42).
template <typename T>
__global__ __launch_bounds__(256) void k_pack4(const Pack4Args a) {
  const int lane = lane_id(), q = lane / 16, m = lane % 16;
  const int64_t rb = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (rb * kTable4Rows >= a.N) return;
  const bool whole = (rb + 1) * kTable4Rows <= a.N;
  double sq[4] = {0.0, 0.0, 0.0, 0.0};
  for (int g = 0; g < a.groups; ++g) {
    char* block = a.table + (rb * a.groups + g) * kTable4Bytes;
    const int col = g * kTable4Group + q * 8;
    Raw<T, 8> r[4];
    if (whole && (g + 1) * kTable4Group <= a.d) {
#pragma unroll
      for (int t = 0; t < 4; ++t) r[t] = ld_raw<T, 8>((const T*)a.W + (rb * kTable4Rows + t * 16 + m) * a.ldw + col);
    } else {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int64_t row = rb * kTable4Rows + t * 16 + m;
        r[t] = Raw<T, 8>{};
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (row < a.N && col + i < a.d) {
            if constexpr (sizeof(T) == 4) r[t].w[i] = __float_as_uint(((const float*)a.W)[row * a.ldw + col + i]);
            else r[t].w[i / 2] |= (uint32_t)((const uint16_t*)a.W)[row * a.ldw + col + i] << (16 * (i & 1));
          }
      }
    }
    u32x4_t codes;
    uint16_t scale = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      uint32_t most = 0;                                       // (magnitudes in the order of their bits: infinities and NaN on top)
#pragma unroll
      for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(raw_elem(r[t], i)) & 0x7FFFFFFFu);
      most = max(most, (uint32_t)__shfl_xor((int)most, 16));
      most = max(most, (uint32_t)__shfl_xor((int)most, 32));
      const bool finite = most < 0x7F800000u;
      const uint16_t sb = finite ? to_bf16(__uint_as_float(most) / 6.0f) : (uint16_t)0x7FC0u;      // (a group with no number stands for none)
      const float s = bf16_to_f32(sb);
      uint32_t word = 0;
      if (s > 0.f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x = raw_elem(r[t], i), y = fabsf(x);
          uint32_t code = (uint32_t)(y > 0.25f * s) + (uint32_t)(y >= 0.75f * s) + (uint32_t)(y > 1.25f * s) + (uint32_t)(y >= 1.75f * s) +
                          (uint32_t)(y > 2.5f * s) + (uint32_t)(y >= 3.5f * s) + (uint32_t)(y > 5.0f * s);
          const float level = code < 4 ? 0.5f * (float)code : code < 6 ? (float)(code - 2) : 2.0f * (float)(code - 4);
          sq[t] += (double)(level * s) * (double)(level * s);
          if (code && x < 0.f) code |= 8u;
          word |= code << (4 * i);
        }
      }
      if (!finite) sq[t] = __builtin_nan("");
      codes[t] = word;
      if (q == t) scale = sb;
    }
    *(u32x4_t*)(block + lane * 16) = codes;
    *(uint16_t*)(block + 1024 + ((m / 4) * 16 + q * 4 + m % 4) * 2) = scale;
  }
  if (a.sq) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      sq[t] += __shfl_xor(sq[t], 16);
      sq[t] += __shfl_xor(sq[t], 32);
      const int64_t row = rb * kTable4Rows + t * 16 + m;
      if (q == t && row < a.N) a.sq[row] = (float)sq[t];
    }
  }
}

// eight 4-bit values as bfloat16
__device__ __forceinline__ bf16x8_t widen4(uint32_t code) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, 1.0f, 1);
  const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, 1.0f, 3);
  return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

struct Scores4Args {
  const char* table; int64_t N; int d, groups;
  const void* x; int64_t ldx, n;
  float alpha, beta; const float* c;
  void* y; int64_t ldy;
};

constexpr int kScores4Waves = 8;

// Eight float32 as three sets of eight bfloat16 whose sums they are (24 significant bits in pieces of 8, cut off and not rounded, so that
// none of them overflows); infinities and NaN stand in the first.
__device__ __forceinline__ void split3(const float (&x)[8], u32x4_t (&p)[3]) {
  uint32_t u[8], most = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    u[i] = __float_as_uint(x[i]);
    most = max(most, u[i] & 0x7FFFFFFFu);
  }
  float r[8], l[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    r[i] = x[i] - __uint_as_float(u[i] & 0xFFFF0000u);
    l[i] = r[i] - __uint_as_float(__float_as_uint(r[i]) & 0xFFFF0000u);
  }
  if (most >= 0x7F800000u) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if ((u[i] & 0x7FFFFFFFu) >= 0x7F800000u) {
        r[i] = l[i] = 0.f;
        if (u[i] & 0x007FFFFFu) u[i] = 0x7FC00000u;
      }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {                               // (the upper halves of two words side by side)
    p[0][i] = __builtin_amdgcn_perm(u[2 * i + 1], u[2 * i], 0x07060302u);
    p[1][i] = __builtin_amdgcn_perm(__float_as_uint(r[2 * i + 1]), __float_as_uint(r[2 * i]), 0x07060302u);
    p[2][i] = __builtin_amdgcn_perm(__float_as_uint(l[2 * i + 1]), __float_as_uint(l[2 * i]), 0x07060302u);
  }
}

// y[q][row] = alpha x_q . t^_row + beta c[row].  A workgroup keeps 16 CT queries in the LDS as matrix operands (float32 ones as three
// bfloat16 pieces: three matrix instructions instead of one); a wave takes 64 rows of the table at a time, group by group.  Few queries
// are bound by the table's bytes (4 queries, a million rows of 128, 92 MB: 18 to 21 us, 4.4 to 5.1 TB/s).  128 queries, 100,000 rows of 200: 25 to 28 us
// in float32, 21 to 23 in bfloat16; by the counters the vector instructions that widen and scale take 8 us of that, the matrix ones 7 (bfloat16: 2),
// the results' bytes 9.  They do not overlap well: a wave waits for memory a third of its time, and as long for its turn to issue.
template <typename TX, typename TO, int CT>
__global__ __launch_bounds__(kScores4Waves * 64) void k_scores4(const Scores4Args a) {
  constexpr int NS = sizeof(TX) == 4 ? 3 : 1;
  extern __shared__ __align__(16) u32x4_t xs[];               // [group][CT][NS][64]
  const int64_t q0 = (int64_t)blockIdx.y * 16 * CT;
  const int lane = lane_id();
  const int64_t blocks = (a.N + kTable4Rows - 1) / kTable4Rows, stride = (int64_t)gridDim.x * kScores4Waves;
  if ((int64_t)blockIdx.x * kScores4Waves >= blocks) return;
  // (the wave's number as a scalar: so are the addresses that come from it)
  int64_t rb = (int64_t)blockIdx.x * kScores4Waves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // Blocks of the table one after the other, the next one asked for before the last is multiplied, into two sets of registers in turn.
  struct Block { u32x4_t code, scale[2]; };
  Block w0, w1;
  int64_t ahead_rb = rb;                                      // the block asked for last
  int ahead_g = 0;
  auto load = [&](Block& w) {
    const char* p = a.table + (ahead_rb * a.groups + ahead_g) * kTable4Bytes;
    w.code = *(const u32x4_t*)(p + lane * 16);
    w.scale[0] = *(const u32x4_t*)(p + 1024 + (lane / 16) * 32);
    w.scale[1] = *(const u32x4_t*)(p + 1024 + (lane / 16) * 32 + 16);
  };
  auto next = [&] {                                           // (the last one again at the end)
    if (ahead_g + 1 < a.groups) ++ahead_g;
    else if (ahead_rb + stride < blocks) ahead_g = 0, ahead_rb += stride;
  };
  if (rb < blocks) {                                          // (under the staging of the queries)
    load(w0);
    next();
    load(w1);
    next();
  }
  // the queries as matrix operands: eight dimensions of one query an item; two items' loads in flight.  Past the last query it stands
  // there again, and so do its results: stores under a condition would have each block wait for those of the one before
  const int items = a.groups * CT * 64;
  for (int it0 = threadIdx.x; it0 < items; it0 += 2 * kScores4Waves * 64) {
    Raw<TX, 4> r[2][2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int it = min(it0 + u * kScores4Waves * 64, items - 1);
      const int64_t q = min(q0 + (it >> 6) % CT * 16 + (it & 15), a.n - 1);
      const int k = (it >> 6) / CT * kTable4Group + (it & 63) / 16 * 8;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (a.d >= 4) r[u][h] = ld_raw<TX, 4>((const TX*)a.x + q * a.ldx + min(k + 4 * h, a.d - 4));
        else r[u][h] = Raw<TX, 4>{};
      }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int it = it0 + u * kScores4Waves * 64;
      if (it >= items) continue;
      const int64_t q = min(q0 + (it >> 6) % CT * 16 + (it & 15), a.n - 1);
      const int k = (it >> 6) / CT * kTable4Group + (it & 63) / 16 * 8;
      float x[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f32x4_t v = widen(r[u][h]);
        const int left = a.d - k - 4 * h;
        if (left < 4) v = left > 0 ? ld4((const TX*)a.x + q * a.ldx + k + 4 * h, left) : f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[4 * h + i] = v[i];
      }
      u32x4_t p[3];
      split3(x, p);                                           // (a bfloat16 is its first piece)
#pragma unroll
      for (int s = 0; s < NS; ++s) xs[((it >> 6) * NS + s) * 64 + (it & 63)] = p[s];
    }
  }
  __syncthreads();
  if (rb >= blocks) return;
  f32x4_t sum[4][CT];
  int g = 0;
  auto clear = [&] {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) sum[t][ct] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  };
  auto multiply = [&](const Block& w) {
    bf16x8_t x[CT][NS];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int s = 0; s < NS; ++s) x[ct][s] = __builtin_bit_cast(bf16x8_t, xs[((g * CT + ct) * NS + s) * 64 + lane]);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const bf16x8_t v = widen4(w.code[t]);
      f32x4_t scale;
      scale[0] = __uint_as_float(w.scale[t / 2][2 * (t % 2)] << 16);
      scale[1] = __uint_as_float(w.scale[t / 2][2 * (t % 2)] & 0xFFFF0000u);
      scale[2] = __uint_as_float(w.scale[t / 2][2 * (t % 2) + 1] << 16);
      scale[3] = __uint_as_float(w.scale[t / 2][2 * (t % 2) + 1] & 0xFFFF0000u);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = NS - 1; s >= 0; --s) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, x[ct][s], acc, 0, 0, 0);
        sum[t][ct] = sum[t][ct] + scale * acc;
      }
    }
  };
  auto store = [&] {
    // a whole block of rows without the checks of the last one, so that the loads of c do not wait for one another
    if ((rb + 1) * kTable4Rows <= a.N) {
      Raw<float, 4> c[4];
      if (a.c) {
#pragma unroll
        for (int t = 0; t < 4; ++t) c[t] = ld_raw<float, 4>(a.c + rb * kTable4Rows + t * 16 + (lane / 16) * 4);
      }
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          const int64_t q = min(q0 + ct * 16 + lane % 16, a.n - 1);
          f32x4_t v = sum[t][ct] * a.alpha;
          if (a.c) v = v + widen(c[t]) * a.beta;
          st4((TO*)a.y + q * a.ldy + rb * kTable4Rows + t * 16 + (lane / 16) * 4, v, 4);
        }
      return;
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int64_t row = rb * kTable4Rows + t * 16 + (lane / 16) * 4;
      if (row >= a.N) continue;
      const int left = (int)min(a.N - row, (int64_t)4);
      f32x4_t c = {0.f, 0.f, 0.f, 0.f};
      if (a.c) c = ld4(a.c + row, left) * a.beta;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        const int64_t q = q0 + ct * 16 + lane % 16;
        if (q < a.n) st4((TO*)a.y + q * a.ldy + row, sum[t][ct] * a.alpha + c, left);
      }
    }
  };
  clear();
  auto step = [&](const Block& w) {                           // true: that was the last
    multiply(w);
    if (++g < a.groups) return false;
    store();
    clear();
    g = 0;
    rb += stride;
    return rb >= blocks;
  };
  for (;;) {                                                  // (the barriers keep the loads ahead of the next products)
    if (step(w0)) return;
    load(w0);
    next();
    __builtin_amdgcn_sched_barrier(0);
    if (step(w1)) return;
    load(w1);
    next();
    __builtin_amdgcn_sched_barrier(0);
  }
}

// ---- adjusted scores ----
struct AdjustArgs {
  const void* in; void* out; int64_t n, N, ldi, ldo;
  const float* bias;
  const uint32_t* allowed; int64_t masks, ldm; const int32_t* mask_row;
  const int64_t* known_off; const int32_t* known; int64_t n_known;
  const int64_t* seen_off; const int32_t* seen; int64_t n_seen;
  float repeat, presence, frequency;
  int rows_first;              // the same chunk of all rows, then the next one
};

constexpr int kAdjustChunk = 4096;

// ids first .. last of row b's list, whatever the offsets hold: never past the list
__device__ __forceinline__ void list_range(const int64_t* off, int64_t count, int64_t b, int64_t* first, int64_t* last) {
  *first = min(max(off[b], (int64_t)0), count);
  *last = min(max(off[b + 1], *first), count);
}

// A workgroup takes 4,096 scores of one row: it looks through the row's lists for the entities of this chunk (a bit for the known
// ones, a count for the seen ones, both in the LDS), then passes once over the scores.  Integer atomics only: the order does not
// matter.  DENSE: every score is written; otherwise (in place, lists only) those of named entities and their neighbours in a vector,
// chunk by chunk all the same (60 ids a row: 512 rows of 40,000: 11.5 us, 600 of a million: 164).
// Bound by bytes and by the trips to the lists: 256 x 100,000 in bfloat16 with everything 27 us (106 MB, 3.9 TB/s), without lists 18, a
// plain copy 15.
template <typename T, bool DENSE, bool SEEN>
__global__ __launch_bounds__(256) void k_adjust(const AdjustArgs a) {
  __shared__ uint32_t gone[kAdjustChunk / 32];
  __shared__ __align__(16) uint32_t times[SEEN ? kAdjustChunk : 4];
  const int64_t chunks = (a.N + kAdjustChunk - 1) / kAdjustChunk;
  for (int64_t job = blockIdx.x; job < a.n * chunks; job += gridDim.x) {
    const int64_t b = a.rows_first ? job % a.n : job / chunks, n0 = (a.rows_first ? job / a.n : job - b * chunks) * kAdjustChunk;
    const int size = (int)min(a.N - n0, (int64_t)kAdjustChunk);
    const uint32_t* mask = nullptr;
    if (DENSE && a.allowed) {
      const int64_t m = a.mask_row ? (int64_t)a.mask_row[b] : (a.masks == 1 ? 0 : b);
      if (m >= 0 && m < a.masks) mask = a.allowed + m * a.ldm + n0 / 32;
    }
    const T* in = (const T*)a.in + b * a.ldi + n0;
    T* out = (T*)a.out + b * a.ldo + n0;
    // a whole chunk's scores are asked for before the lists are looked through, 16 bytes a vector
    constexpr int V = 16 / (int)sizeof(T), U = kAdjustChunk / (256 * V);
    const int k0 = threadIdx.x * V;
    const bool whole = DENSE && size == kAdjustChunk;
    Raw<T, V> x[U];
    if (whole) {
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = ld_raw<T, V>(in + k0 + 256 * V * u);
    }
    if (threadIdx.x < kAdjustChunk / 32) gone[threadIdx.x] = 0;
    if (SEEN)
      for (int k = threadIdx.x * 4; k < kAdjustChunk; k += 1024) *(u32x4_t*)(times + k) = u32x4_t{0, 0, 0, 0};
    __syncthreads();
    // the row's entities of this chunk; four of a thread's ids under way at a time
    auto look = [&](const int64_t* off, const int32_t* ids, int64_t count, auto&& found) {
      int64_t first, last;
      list_range(off, count, b, &first, &last);
      for (int64_t i = first + threadIdx.x; i < last; i += 1024) {
        int32_t id[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) id[u] = ids[min(i + 256 * u, last - 1)];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int64_t k = (int64_t)id[u] - n0;
          if (i + 256 * u < last && k >= 0 && k < size) found((int)k);
        }
      }
    };
    if (a.known) look(a.known_off, a.known, a.n_known, [&](int k) { atomicOr(&gone[k >> 5], 1u << (k & 31)); });
    if (SEEN) look(a.seen_off, a.seen, a.n_seen, [&](int k) { atomicAdd(&times[k], 1u); });
    __syncthreads();
    auto change = [&](int k, uint32_t allowed, f32x4_t x, f32x4_t bias) {
      uint32_t off = (gone[k >> 5] >> (k & 31)) & 15u;
      if (DENSE) off |= ~(allowed >> (k & 31)) & 15u;
      if (DENSE && a.bias) x = x + bias;
      u32x4_t c = {0, 0, 0, 0};
      if (SEEN) c = *(const u32x4_t*)(times + k);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (SEEN && c[i]) x[i] = (x[i] > 0.f ? x[i] / a.repeat : x[i] * a.repeat) - (a.presence + a.frequency * (float)c[i]);
        if ((off >> i) & 1u) x[i] = -__builtin_inff();
      }
      return x;
    };
    if (whole) {
      Raw<float, V> bias[U];
      uint32_t allowed[U];
      if (a.bias) {
#pragma unroll
        for (int u = 0; u < U; ++u) bias[u] = ld_raw<float, V>(a.bias + n0 + k0 + 256 * V * u);
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u) bias[u] = Raw<float, V>{};
      }
#pragma unroll
      for (int u = 0; u < U; ++u) allowed[u] = mask ? mask[(k0 + 256 * V * u) >> 5] : ~0u;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float y[V];
#pragma unroll
        for (int h = 0; h < V / 4; ++h) {
          const f32x4_t xs = {raw_elem(x[u], 4 * h), raw_elem(x[u], 4 * h + 1), raw_elem(x[u], 4 * h + 2), raw_elem(x[u], 4 * h + 3)};
          const f32x4_t bs = {raw_elem(bias[u], 4 * h), raw_elem(bias[u], 4 * h + 1), raw_elem(bias[u], 4 * h + 2), raw_elem(bias[u], 4 * h + 3)};
          const f32x4_t r = change(k0 + 256 * V * u + 4 * h, allowed[u], xs, bs);
#pragma unroll
          for (int i = 0; i < 4; ++i) y[4 * h + i] = r[i];
        }
        st_vec<T, V, false>(out + k0 + 256 * V * u, y);
      }
    } else {
      for (int k = threadIdx.x * 4; k < size; k += 1024) {
        if (!DENSE) {
          uint32_t touched = (gone[k >> 5] >> (k & 31)) & 15u;
          if (SEEN)
#pragma unroll
            for (int i = 0; i < 4; ++i) touched |= times[k + i];
          if (!touched) continue;
        }
        const f32x4_t bias = DENSE && a.bias ? ld4(a.bias + n0 + k, size - k) : f32x4_t{0.f, 0.f, 0.f, 0.f};
        st4(out + k, change(k, mask ? mask[k >> 5] : ~0u, ld4(in + k, size - k), bias), size - k);
      }
    }
    __syncthreads();
  }
}

// in place and nothing but known entities: they leave one by one
template <typename T>
__global__ __launch_bounds__(256) void k_adjust_known(const AdjustArgs a) {
  for (int64_t b = blockIdx.y; b < a.n; b += gridDim.y) {
    int64_t first, last;
    list_range(a.known_off, a.n_known, b, &first, &last);
    for (int64_t i = first + (int64_t)blockIdx.x * 256 + threadIdx.x; i < last; i += (int64_t)gridDim.x * 256) {
      const int32_t k = a.known[i];
      if (k >= 0 && k < a.N) {
        if constexpr (sizeof(T) == 4) ((float*)a.out)[b * a.ldo + k] = -__builtin_inff();
        else ((uint16_t*)a.out)[b * a.ldo + k] = 0xFF80u;
      }
    }
  }
}

}  // namespace kgc
