// dfssm_adapters.hip -- low-rank adapters of many requests beside a shared
// projection, gfx950:  out[m] = y[m] + s[m] * (beta_a * (B_a (A_a q_m))) with
// a = ids[m], int8 or packed int4 factors.
//
// The integers are exact (acc_a int32, acc_b int64), and each of the four
// fp32 operations after them is rounded once, so results do not depend on
// which rows share a call.
//
// Rows are taken in windows of 64.  The rows of a window that name one adapter
// make sets of up to 16, the columns of an MFMA, whatever order they come in: a
// wave holds the window's ids in its lanes and finds a set with two ballots, so
// nothing has to be sorted.  Two launches: acc_a per row and rank, left in the
// workspace as four signed base-256 digits, and the product with B with the
// fp32 operations and y in its epilogue; or, for few rows, one that takes acc_a
// itself.  y is read once, a factor once for each set of a window that names its
// adapter (A once more per column block in that one launch), which is little beside
// y where prompts make runs.  So bytes bound it from a few hundred rows on: 7001 rows x 10576 columns at rank 16, 619 MB, adapter_down
// 10.5 and adapter_up 126 us (4.7 TB/s of y and out, a large copy's rate); below
// that the launches and the round trips to memory do.
#include <algorithm>
#include <type_traits>

#include "dfssm_adapters.hpp"
#include "dfssm_linear.hpp"

namespace {

using dfssm_lin::mfma;
using dfssm_lin::v4i;
using dfssm_lin::zero4;

constexpr int kWindow = 64;     // rows
constexpr int kSet = 16;        // rows of a set
constexpr int kWaves = 4;       // of adapter_up
constexpr int kThreads = 64 * kWaves;
constexpr int kDownWaves = 8;   // of adapter_down, which split K
constexpr int kCols = 64;       // output columns of a wave of adapter_up
typedef float f4 __attribute__((ext_vector_type(4)));

struct Args {
  const int8_t* q;     // [M][K]
  const float* s;      // [M]
  int64_t M;
  int K, N, r, rp;     // rp: r rounded up to 16
  const int32_t* ids;  // [M]
  int64_t n;           // adapters
  const int8_t* A;     // [n][r][K], or K / 2 bytes a row
  const int8_t* B;     // [n][N][r], or r / 2 bytes a row
  const float* beta;   // [n][N]
  const float* y;
  float* out;          // [M][N]
  int8_t* limbs;       // [M][4][rp] digits of acc_a, zeros from r on
  int blocks;          // column blocks of adapter_up, rank tiles of adapter_down
  int parts;           // workgroups that share a window's sets
};

// The window's adapter of lane's row: -1 for none, -2 past the last row.
__device__ __forceinline__ int window_id(const Args& a, int64_t row) {
  if (row >= a.M) return -2;
  const int32_t id = a.ids[row];
  return id >= 0 && id < a.n ? id : -1;
}

// The rows of a window that name the adapter of row z, from row z on, up to 16.
struct Set {
  int id;        // adapter, -1: rows without one
  int count;
  int at;        // lane c < count: row of the window of column c
  __device__ __forceinline__ int row(int c) const { return __builtin_amdgcn_ds_bpermute(c * 4, at); }
};

__device__ __forceinline__ Set set_of(int id, int z, int lane) {
  Set s;
  s.id = __builtin_amdgcn_readlane(id, z);
  const uint64_t same = __ballot(id == s.id) >> z << z;
  const int rank = __popcll(same & ((1ull << lane) - 1));
  const bool mine = id == s.id && lane >= z && rank < kSet;
  s.count = __popcll(__ballot(mine));
  // the set's rows push their lane to the lane of their rank, the others to one
  // that no column reads; columns without a row repeat row z
  s.at = __builtin_amdgcn_ds_permute((mine ? rank : 63) * 4, lane);
  if (lane >= s.count) s.at = z;
  return s;
}

// First rows of the window's sets (every 16th row of an adapter's), as a mask.
__device__ __forceinline__ uint64_t set_starts(int id, int lane) {
  uint64_t rest = __ballot(id >= -1);
  bool start = false;
  while (rest) {
    const int a = __builtin_amdgcn_readlane(id, __ffsll((unsigned long long)rest) - 1);
    const uint64_t same = __ballot(id == a);
    if (id == a) start = __popcll(same & ((1ull << lane) - 1)) % kSet == 0;
    rest &= ~same;
  }
  return __ballot(start);
}

// The sets of a window that are part `part` of `parts`, as their first rows: with a
// part for every row, the set that starts with row `part`, if one does; else every
// parts-th set.
__device__ __forceinline__ uint64_t my_sets(const Args& a, int id, int lane, int part) {
  if (a.parts >= std::min<int64_t>(a.M, kWindow)) {
    const int own = __builtin_amdgcn_readlane(id, part);
    const uint64_t same = __ballot(id == own);
    return own >= -1 && __popcll(same & ((1ull << part) - 1)) % kSet == 0 ? 1ull << part : 0ull;
  }
  uint64_t all = set_starts(id, lane), mine = 0;
  for (int k = 0; all; ++k, all &= all - 1)
    if (k % a.parts == part) mine |= all & -all;     // parts: a power of two
  return mine;
}

// How the rows of B can be read: ranks in whole pieces of 16, in whole 4-byte words,
// or any number.
enum Ranks { kPieces, kWords, kAny };

// Values start .. start + 15 of a factor row of len values, zero from len on.
template <bool L4, int RANKS>
__device__ __forceinline__ v4i load_ranks(const int8_t* row, int start, int len) {
  if (start >= len) return zero4();
  if constexpr (RANKS == kPieces) {
    const uint4 u = dfssm_lin::load_row16<L4>(row, start);
    return v4i{(int)u.x, (int)u.y, (int)u.z, (int)u.w};
  } else if constexpr (RANKS == kAny) {
    return dfssm_lin::load16_row_guarded<L4>(row, start, len, false);
  } else if constexpr (L4) {
    const uint32_t* p = reinterpret_cast<const uint32_t*>(row + start / 2);
    const uint4 u = dfssm_lin::expand_i4(make_uint2(p[0], start + 8 < len ? p[1] : 0u));
    return v4i{(int)u.x, (int)u.y, (int)u.z, (int)u.w};
  } else {
    const int* p = reinterpret_cast<const int*>(row + start);
    v4i o = zero4();
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (start + 4 * e < len) o[e] = p[e];
    return o;
  }
}

// acc_a of a set's rows and 16 ranks, K split over the waves.
template <bool L4>
__global__ __launch_bounds__(64 * kDownWaves) void adapter_down(Args a) {
  __shared__ v4i part_s[kDownWaves][64];
  const int tile = blockIdx.x % a.blocks;
  const int64_t row0 = (int64_t)(blockIdx.x / a.blocks) * kWindow;
  const int lane = threadIdx.x & 63, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int id = window_id(a, row0 + lane);
  const int rank = 16 * tile + (lane & 15);
  const int64_t stride = L4 ? a.K / 2 : a.K;
  for (uint64_t sets = my_sets(a, id, lane, blockIdx.y); sets; sets &= sets - 1) {
    const Set s = set_of(id, __ffsll((unsigned long long)sets) - 1, lane);
    if (s.id < 0) continue;
    const int64_t m = row0 + s.row(lane & 15);
    const int8_t* Ar = a.A + ((int64_t)s.id * a.r + std::min(rank, a.r - 1)) * stride;
    const int8_t* qr = a.q + m * a.K;
    v4i acc = zero4();
    constexpr int U = 8;
    for (int k0 = 64 * wave; k0 < a.K; k0 += 64 * kDownWaves * U) {
      v4i av[U], qv[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int k = k0 + 64 * kDownWaves * u + 16 * g;
        av[u] = qv[u] = zero4();
        if (k < a.K) {
          const uint4 w = dfssm_lin::load_row16<L4>(Ar, k);
          av[u] = v4i{(int)w.x, (int)w.y, (int)w.z, (int)w.w};
          qv[u] = dfssm_lin::load16(qr + k);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) acc = mfma(av[u], qv[u], acc);
    }
    part_s[wave][lane] = acc;
    __syncthreads();
    if (wave == 0 && (lane & 15) < s.count) {
#pragma unroll
      for (int w = 1; w < kDownWaves; ++w) acc += part_s[w][lane];
      // lane: column (row of the set) lane % 16, ranks 16 tile + 4 g ..
      uint32_t word[4] = {0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (16 * tile + 4 * g + e >= a.r) continue;
        int8_t d[4];
        dfssm_dev::split_limbs(acc[e], d);
#pragma unroll
        for (int t = 0; t < 4; ++t) word[t] |= (uint32_t)(uint8_t)d[t] << (8 * e);
      }
      int8_t* o = a.limbs + m * 4 * a.rp + 16 * tile + 4 * g;
#pragma unroll
      for (int t = 0; t < 4; ++t) *reinterpret_cast<uint32_t*>(o + t * a.rp) = word[t];
    }
    __syncthreads();
  }
}

// Columns n .. n + 3 of a row of N, the last ones again past its end (VEC: N is a
// multiple of 4, and n at most N - 4).
template <bool VEC>
__device__ __forceinline__ f4 load4(const float* row, int n, int N) {
  if (VEC) return *reinterpret_cast<const f4*>(row + n);
  f4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = row[std::min(n + e, N - 1)];
  return v;
}
template <bool VEC>
__device__ __forceinline__ void store4(float* row, int n, int N, f4 v) {
  if (VEC) {
    *reinterpret_cast<f4*>(row + n) = v;
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (n + e < N) row[n + e] = v[e];
}

// y + s (beta acc_b), acc_b from row r of its four digits' products
__device__ __forceinline__ float add_adapter(float y, float s, float beta, const v4i (&acc)[4], int r) {
  const int32_t lo = acc[1][r] * 256 + acc[0][r], hi = acc[3][r] * 256 + acc[2][r];
  const float fb = (float)__builtin_fma((double)hi, 65536.0, (double)lo);   // exact, then rounded once
  const float t = beta * fb;
  const float u = s * t;
  return y + u;
}

// A set's rows by 64 columns a wave: MFMA column l % 16 of tile t is output column
// 4 (l % 16) + t, so that a lane ends with four neighbouring columns of four rows
// and 16 lanes with 256 bytes of one.
template <bool L4, int RANKS, bool VEC, bool ONE>
__global__ __launch_bounds__(kThreads) void adapter_up(Args a) {
  const int64_t row0 = (int64_t)(blockIdx.x / a.blocks) * kWindow;
  const int lane = threadIdx.x & 63, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int n0 = ((int)(blockIdx.x % a.blocks) * kWaves + wave) * kCols;
  if (n0 >= a.N) return;
  const int id = window_id(a, row0 + lane);
  const bool in_place = a.out == a.y;
  const int64_t stride = L4 ? a.r / 2 : a.r;
  const int n = n0 + 4 * (lane & 15), nl = VEC ? std::min(n, a.N - 4) : n;   // nl: for loads
  for (uint64_t sets = my_sets(a, id, lane, blockIdx.y); sets; sets &= sets - 1) {
    const Set s = set_of(id, __ffsll((unsigned long long)sets) - 1, lane);
    if (s.id < 0 && in_place) continue;
    int64_t m[4];
    f4 yv[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      m[r] = row0 + s.row(4 * g + r);
      yv[r] = load4<VEC>(a.y + m[r] * a.N, nl, a.N);
    }
    if (s.id >= 0) {
      const f4 bv = load4<VEC>(a.beta + (int64_t)s.id * a.N, nl, a.N);
      float sc[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) sc[r] = a.s[m[r]];
      const int8_t* lim = a.limbs + (row0 + s.row(lane & 15)) * 4 * a.rp;
      auto digits = [&](int j, v4i (&lm)[4]) {
#pragma unroll
        for (int d = 0; d < 4; ++d) lm[d] = j < a.rp ? dfssm_lin::load16(lim + d * a.rp + j) : zero4();
      };
      auto ranks = [&](int t, int j) {
        return load_ranks<L4, RANKS>(a.B + ((int64_t)s.id * a.N + std::min(n + t, a.N - 1)) * stride, j, a.r);
      };
      auto finish = [&](int t, const v4i (&acc)[4]) {
#pragma unroll
        for (int r = 0; r < 4; ++r) yv[r][t] = add_adapter(yv[r][t], sc[r], bv[t], acc, r);
      };
      if constexpr (ONE) {   // one step of ranks: a column tile at a time keeps few sums
        v4i lm[4], b[4];
        digits(16 * g, lm);
#pragma unroll
        for (int t = 0; t < 4; ++t) b[t] = ranks(t, 16 * g);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          v4i acc[4];
#pragma unroll
          for (int d = 0; d < 4; ++d) acc[d] = mfma(lm[d], b[t], zero4());
          finish(t, acc);
          __builtin_amdgcn_sched_barrier(0);
        }
      } else {
        v4i acc[4][4];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int d = 0; d < 4; ++d) acc[t][d] = zero4();
        for (int j0 = 0; j0 < a.rp; j0 += 64) {
          v4i lm[4];
          digits(j0 + 16 * g, lm);
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const v4i b = ranks(t, j0 + 16 * g);
#pragma unroll
            for (int d = 0; d < 4; ++d) acc[t][d] = mfma(lm[d], b, acc[t][d]);
          }
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) finish(t, acc[t]);
      }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (4 * g + r < s.count && n < a.N) store4<VEC>(a.out + m[r] * a.N, n, a.N, yv[r]);
  }
}

// Few rows in one launch: every workgroup takes acc_a of its set by itself, K
// split over the waves and summed through LDS, and then its columns as adapter_up
// does.  Up to rank 64, whose digits are one step of the product.
template <bool L4, int RANKS, bool VEC>
__global__ __launch_bounds__(kThreads) void adapter_few(Args a) {
  __shared__ v4i part_s[kWaves][4][64];
  const int64_t row0 = (int64_t)(blockIdx.x / a.blocks) * kWindow;
  const int lane = threadIdx.x & 63, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int n0 = ((int)(blockIdx.x % a.blocks) * kWaves + wave) * kCols;
  const int id = window_id(a, row0 + lane);
  const bool in_place = a.out == a.y;
  const int64_t strideA = L4 ? a.K / 2 : a.K, strideB = L4 ? a.r / 2 : a.r;
  const int n = n0 + 4 * (lane & 15), nl = VEC ? std::min(n, a.N - 4) : n;
  const int tiles = a.rp / 16;
  for (uint64_t sets = my_sets(a, id, lane, blockIdx.y); sets; sets &= sets - 1) {
    const Set s = set_of(id, __ffsll((unsigned long long)sets) - 1, lane);
    if (s.id < 0 && in_place) continue;
    int64_t m[4];
    f4 yv[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      m[r] = row0 + s.row(4 * g + r);
      yv[r] = load4<VEC>(a.y + m[r] * a.N, nl, a.N);
    }
    if (s.id >= 0) {
      const int8_t* qr = a.q + (row0 + s.row(lane & 15)) * a.K;
      const f4 bv = load4<VEC>(a.beta + (int64_t)s.id * a.N, nl, a.N);
      v4i b[4];
#pragma unroll
      for (int t = 0; t < 4; ++t)
        b[t] = load_ranks<L4, RANKS>(a.B + ((int64_t)s.id * a.N + std::min(n + t, a.N - 1)) * strideB, 16 * g, a.r);
      float sc[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) sc[r] = a.s[m[r]];
      v4i sum[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) sum[t] = zero4();
      constexpr int U = 4;
      for (int k0 = 64 * wave; k0 < a.K; k0 += 64 * kWaves * U) {
        v4i qv[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int k = k0 + 64 * kWaves * u + 16 * g;
          qv[u] = k < a.K ? dfssm_lin::load16(qr + k) : zero4();
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          if (t >= tiles) continue;
          const int8_t* Ar = a.A + ((int64_t)s.id * a.r + std::min(16 * t + (lane & 15), a.r - 1)) * strideA;
          v4i av[U];
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int k = k0 + 64 * kWaves * u + 16 * g;
            av[u] = zero4();
            if (k < a.K) {
              const uint4 w = dfssm_lin::load_row16<L4>(Ar, k);
              av[u] = v4i{(int)w.x, (int)w.y, (int)w.z, (int)w.w};
            }
          }
#pragma unroll
          for (int u = 0; u < U; ++u) sum[t] = mfma(av[u], qv[u], sum[t]);
        }
      }
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (t < tiles) part_s[wave][t][lane] = sum[t];
      __syncthreads();
      // lane: row lane % 16 of the set, ranks 16 g ..; tiles past the last meet
      // zeros of B
      uint32_t word[16];
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const int at = 16 * h + (lane & 15), tile = std::min(g, tiles - 1);
        v4i v = part_s[0][tile][at];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) v += part_s[w][tile][at];
#pragma unroll
        for (int e = 0; e < 4; ++e) word[4 * h + e] = dfssm_lin::pack_limbs(v[e]);
      }
      v4i lm[4];
      dfssm_lin::limb_operands(word, lm);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        v4i acc[4];
#pragma unroll
        for (int d = 0; d < 4; ++d) acc[d] = mfma(lm[d], b[t], zero4());
#pragma unroll
        for (int r = 0; r < 4; ++r) yv[r][t] = add_adapter(yv[r][t], sc[r], bv[t], acc, r);
      }
      __syncthreads();   // the next set's sums
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (4 * g + r < s.count && n < a.N) store4<VEC>(a.out + m[r] * a.N, n, a.N, yv[r]);
  }
}

// Workgroups that share a window's sets: one per row while they stay below
// `most`, else a power of two from 4 (the sets of a window that is one run) on.  A
// workgroup without a set costs its start and a look at the ids: 7001 rows in
// runs, adapter_down with 64 parts 20 us, with 8 (most = 1024) 10 us; adapter_up,
// whose workgroups are half the size and hold a fifth of the work, takes 8192.
int window_parts(int64_t M, int64_t blocks, int64_t most) {
  const int64_t groups = dfssm::ceil_div(M, kWindow) * blocks;
  int p = 4;
  while (p < kWindow && groups * p * 2 <= most) p *= 2;
  return (int)std::min<int64_t>(M, p);
}

// Whether adapter_few is the faster one.  Every workgroup of it reads its set's A
// again, which beats a second launch while there is one tile of ranks or K is
// short, and while its workgroups (one per row and column block, those of rows that
// start no set included) are at home on the card at once.  us of a call in a graph,
// two launches / adapter_few, 16 adapters:
//  - int8 rank 16, 768 x 3352: 1 row 6.0 / 4.3, 64 rows (896 workgroups) 7.2 / 5.8,
//    128 rows 7.8 / 8.9; 2048 x 8512: 1 row 6.7 / 5.2, 16 rows (544) 7.5 / 7.3, 32
//    rows (1088) 8.6 / 10.9; 4096 x 2048: 64 rows (512) 8.9 / 7.5, 128 rows (1024)
//    9.4 / 10.3
//  - int8 rank 64, 768 x 3352: 1 row 6.3 / 5.6; 2048 x 8512: 1 row 7.1 / 8.3
//  - int4 rank 16, 768 x 3352: 1 row 7.0 / 5.2; rank 64: 6.8 / 7.0
// and with ids in any order, up to 64 rows of 900 workgroups or fewer:
//  - int8 rank 32, K 256 .. 2304: 6.0 .. 6.9 / 4.3 .. 6.7 at 1 row, 7.9 / 7.4 at 64 rows of
//    2304 x 1152; K 4096: 8.0 / 8.6.  Rank 48, K 256 .. 1024: 5.9 .. 6.4 / 4.5 .. 5.5 at 1
//    row; K 1536: 6.4 .. 7.4 / 6.4 .. 6.9; K 2048 and 2304: 6.9 / 7.2 .. 7.9.  Rank 64, K 1024:
//    6.6 / 6.2 at 1 row, 7.5 / 8.9 at 16 of 4384 columns; K 1536: 6.7 / 7.3
//  - int4 rank 32, K 256 .. 1024: 6.4 .. 6.9 / 5.0 .. 6.1 at 1 row; K 1536: 7.0 / 7.1.  Rank 48,
//    K 512: 6.7 / 5.9; K 768: 6.9 / 6.4; K 1024: 6.9 / 6.9.  Rank 64, K 256: 6.6 / 5.6; K 512:
//    6.8 / 6.3; K 768: 6.9 / 7.0
//  - wrong by most near the limit of workgroups, where it depends on the ids: rank 16,
//    4096 x 2048, 64 rows of one adapter 10.0 / 11.9, of 16 in runs 9.3 / 10.4, in any order
//    9.0 / 9.7, in turn 8.4 / 7.2; 2048 x 8512, 16 rows of one adapter 7.7 / 6.1, in any order
//    7.4 / 7.1, each its own 7.8 / 10.3, rank 32 7.7 / 9.1
template <bool L4>
bool few_is_best(const Args& a) {
  const int64_t tiles = a.rp / 16;
  return a.rp <= 64 && (tiles - 1) * a.K <= (L4 ? 1024 : 2304) && a.blocks * a.M <= 900;
}

template <bool L4>
hipError_t launch(Args a, hipStream_t st) {
  const int64_t windows = dfssm::ceil_div(a.M, kWindow);
  a.blocks = (int)dfssm::ceil_div(a.N, kCols * kWaves);
  if (a.n > 0 && few_is_best<L4>(a)) {
    a.parts = window_parts(a.M, a.blocks, 8192);
    const dim3 grid((unsigned)(windows * a.blocks), (unsigned)a.parts), block(kThreads);
    const bool vec = a.N % 4 == 0;
    if (a.r % 16 == 0 && vec) adapter_few<L4, kPieces, true><<<grid, block, 0, st>>>(a);
    else if (a.r % (L4 ? 8 : 4) == 0 && vec) adapter_few<L4, kWords, true><<<grid, block, 0, st>>>(a);
    else adapter_few<L4, kAny, false><<<grid, block, 0, st>>>(a);
    return hipGetLastError();
  }
  if (a.n > 0) {
    a.blocks = (int)dfssm::ceil_div(a.r, 16);
    a.parts = window_parts(a.M, a.blocks, 1024);
    adapter_down<L4><<<dim3((unsigned)(windows * a.blocks), (unsigned)a.parts), dim3(64 * kDownWaves), 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  a.blocks = (int)dfssm::ceil_div(a.N, kCols * kWaves);
  a.parts = window_parts(a.M, a.blocks, 8192);
  const dim3 grid((unsigned)(windows * a.blocks), (unsigned)a.parts), block(kThreads);
  const bool vec = a.N % 4 == 0, one = a.rp <= 64;
  auto up = [&](auto ranks, auto v, auto o) {
    adapter_up<L4, decltype(ranks)::value, decltype(v)::value, decltype(o)::value><<<grid, block, 0, st>>>(a);
  };
  auto pick = [&](auto ranks) {
    if (vec && one) up(ranks, std::true_type{}, std::true_type{});
    else if (vec) up(ranks, std::true_type{}, std::false_type{});
    else if (one) up(ranks, std::false_type{}, std::true_type{});
    else up(ranks, std::false_type{}, std::false_type{});
  };
  if (a.r % 16 == 0)
    pick(std::integral_constant<int, kPieces>{});
  else if (a.r % (L4 ? 8 : 4) == 0)
    pick(std::integral_constant<int, kWords>{});
  else
    up(std::integral_constant<int, kAny>{}, std::false_type{}, std::false_type{});
  return hipGetLastError();
}

}  // namespace

namespace dfssm {

size_t lora_adapters_workspace_bytes(int64_t M, int64_t r) { return (size_t)round_up(M * 4 * round_up(r, 16), 256); }

hipError_t launch_lora_adapters(const int8_t* q, const float* s, int64_t M, int64_t K, int64_t N, int64_t r,
                                const int32_t* ids, int64_t n_adapters, const void* A, const void* B, bool l4,
                                const float* beta, const float* y, float* out, void* ws, hipStream_t st) {
  if (M == 0 || N == 0) return hipSuccess;
  Args a{q, s, M, (int)K, (int)N, (int)r, (int)round_up(r, 16), ids, r > 0 ? n_adapters : 0,
         static_cast<const int8_t*>(A), static_cast<const int8_t*>(B), beta, y, out, static_cast<int8_t*>(ws), 0, 0};
  return l4 ? launch<true>(a, st) : launch<false>(a, st);
}

}  // namespace dfssm
