// dfssm_prompt.hip -- the short causal convolution and the selective scan of
// Mamba-2 over packed prompts of different lengths, gfx950.
//
// The recurrence h_t = exp(a_t) h_{t-1} + (dt_t x_t) B_t^T, y_t = h_t C_t + D x_t
// (a_t = dt_t A) is taken 64 tokens at a time.  With c_i = a_1 + .. + a_i inside a
// chunk that starts from h,
//   y_i = exp(c_i) C_i h + sum_{j <= i} M_ij x_j,
//   M_ij = exp(c_i - c_j) (C_i . B_j) dt_j + D [i = j]
//   h' = exp(c_64) h + sum_j (exp(c_64 - c_j) dt_j x_j) B_j^T
// which is three matrix products a chunk and head, on the matrix cores.  They
// are fp32 products in fp16 halves: v = 2^-e (hi + lo), hi = fp16(2^e v), lo =
// fp16(2^e v - hi), both rounded to nearest, e such that the largest of a tile's
// (or column's) values lies in [2^14, 2^15).  hi + lo holds 23 bits of a value
// down to 2^-17 of the largest, 2^-39 of the largest below that, and a product
// takes hi hi + hi lo + lo hi (the fourth is below 2^-23 of it): three MFMAs of 16
// clocks for what the fp32 MFMA takes sixteen of 32.
//
// Launches, with their times for one prompt of 2048 tokens at d_inner 4096 and of
// 7001 at d_inner 5120 (N = 128):
//   prompt_chunks  11, 16 us   cuts the sequences into chunks and segments (the
//                  tables of the next launches), and prepares what all heads of a
//                  chunk share: B and C after convolution and silu as MFMA operands,
//                  C B^T, and per head dt, its decays and their sums
//   prompt_ends    18, 52 us   only for sequences of more than one segment: each
//                  segment's final state from a zero state
//   prompt_starts  12, 12 us   then turns those into the state before each segment
//   prompt_scan    32, 109 us  walks each segment chunk by chunk with the state in
//                  registers
// A sequence of many chunks is split into segments where its heads alone would
// leave most of the card idle.  73 and 186 to 196 us in all; one copy of what must be read
// and written would take 15 and 64 us.  What bounds them is the instructions of
// prompt_scan and prompt_ends, not memory (1.0 and 1.6 TB/s): of the 1460 vector
// instructions of a chunk of prompt_scan beside its 228 MFMAs a third turn fp32
// values into halves and a fifth convolve; of the 840 of prompt_ends beside 96 a
// third convolve and a ninth make halves.  In 60 % of prompt_scan's clocks one is
// issued; in the rest both waves of a SIMD wait for results, LDS or memory.
#include <algorithm>
#include <atomic>

#include "dfssm_linear.hpp"
#include "dfssm_mamba.hpp"

namespace {

constexpr int kHeadDim = 64;
constexpr int kChunk = 64;         // tokens
constexpr int kHeads = 2;          // of a scan workgroup, two waves of 32 channels each
constexpr int kWaves = 2 * kHeads;
constexpr int kThreads = 64 * kWaves;
constexpr int kChunkThreads = 512;
constexpr float kLog2e = 1.44269504088896341f;

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));

struct Header {
  int n_segs, n_splits;
  int pad[2];
};

struct Seg {
  int64_t row0;    // first row of the sequence
  int len;         // tokens of the sequence
  int chunk0;      // first chunk of the segment
  int k, count;    // segment of the sequence, and how many it has
  int k0, k1;      // its chunks of the sequence, up to k1
  int slot;        // of the pool, or -1: nothing is read or kept
  int fresh;       // starts from zeros
  int pos;         // position of the first token, & 3
  int entry;       // place of the segment among those of split sequences
};

// Per chunk and head, 2 KB.  The exponents c_i - c_j (in units of log2) are sums of
// non-positive numbers only, never differences, so that a weak decay behind a
// strong one keeps its digits: inside a group of eight tokens the sum of the
// tokens' own a (kA), across groups p_i + (groups between) + q_j.
enum Tok {
  kP = 0,              // [64] sum of a over the token's group, up to and with it
  kQ = kChunk,         // [64] over its group behind it
  kA = 2 * kChunk,     // [64] a
  kDt = 3 * kChunk,    // [64] dt
  kW = 4 * kChunk,     // [64] exp(c_64 - c_j) dt_j
  kE = 5 * kChunk,     // [64] exp(c_i)
  kBd = 6 * kChunk,    // [8][8] sum over the groups between groups [i] and [j]
  kAll = 7 * kChunk,   // sum of a
  kDtMax,              // largest dt
  kEb, kEc,            // of all heads: exponents of B's and C's operands (as integers)
  kGMax,               // and the largest |C_i . B_j|, j <= i
  kTokFloats = 8 * kChunk
};

// Operand pieces of 1 KB: lane l's 16 bytes at 16 l.
template <int N>
struct Lay {
  static constexpr int NT = N / 16, KS = N / 32;
  static constexpr int c_units = 4 * KS * 2;      // [row tile][k step][hi, lo]
  static constexpr int g_units = 6 * 2;           // [tile][4 + 4 tokens]
  static constexpr int b_units = NT * 2 * 2;      // [state tile][token half][hi, lo]
  // a chunk's: C, C B^T, then B
  static constexpr int head_units = c_units + g_units, units = head_units + b_units;
  static constexpr int b_global = head_units * 1024;
  // LDS of prompt_scan: C, C B^T, the heads' tokens and B; 80 KB, two workgroups a CU
  static constexpr int tok_off = head_units * 1024;
  static constexpr int b_off = tok_off + kHeads * kTokFloats * 4;
  // and M of the heads, over C where it has the room
  static constexpr int m_units = 6 * 2;           // [tile][hi, lo]
  static constexpr int m_off = c_units >= kHeads * m_units ? 0 : b_off + b_units * 1024;
  static constexpr int scan_lds = b_off + b_units * 1024 + (m_off ? kHeads * m_units * 1024 : 0);
  // LDS of prompt_ends: two buffers of B and half of the tokens' values
  static constexpr int e_buf = (b_units + kHeads) * 1024;
  // LDS of prompt_chunks: B and C [64][2 N + 4] (then C B^T [64][68]), and 32 words
  static constexpr int chunk_lds = (kChunk * (2 * N + 4) + 32) * 4;
};

struct Args {
  const float* zx;
  int64_t ld;
  int T;
  const int32_t* cu;
  int S;
  const int32_t* slots;
  const int32_t* positions;
  int64_t n_slots;
  int d_inner, H;
  float* ring;
  const float* conv_w;
  const float* conv_b;
  const float* dt_bias;
  const float* A_log;
  const float* D;
  float* state;
  float* y;
  int chunks, segments;   // of a sequence of all rows
  int groups;      // of kHeads heads
  // workspace
  Header* head;
  Seg* segs;
  int* splits;     // first segment of each split sequence
  char* ops;       // [chunk][units] operands of all heads: C, G, B
  float* tok;      // [chunk][H][kTokFloats]
  float* halo;     // [entry][3][d_inner] inputs before a split sequence (at its first entry)
  float* ends;     // [entry][H][2][N / 16][2][64][4] states of split sequences
  float* decay;    // [entry][H] sum of a log2(e) over a segment
};

// ---------------------------------------------------------------- places
struct Place {
  int seq;          // -1: the chunk index is past the last
  int row0, len;    // of the sequence
  int k, nch;       // chunk of the sequence, and how many it has
  int seg, entry;   // of the sequence's first segment
  int split;        // split sequences before it
  int slot, pos;    // of the sequence, as given
  int n_segs, n_splits;   // of the call, when `total` was asked for
};

// Inclusive scans over the 64 lanes, on the vector ALU: shifts inside the rows
// of 16, then the last lane of a row (of two rows) to the rows behind it.
template <int CTRL, int ROWS>
__device__ __forceinline__ int from_lane(int none, int v) {
  return __builtin_amdgcn_update_dpp(none, v, CTRL, ROWS, 0xF, false);
}
__device__ __forceinline__ int scan_max(int v) {   // not negative
  v = max(v, from_lane<0x111, 0xF>(0, v));   // row_shr:1, 2, 4, 8
  v = max(v, from_lane<0x112, 0xF>(0, v));
  v = max(v, from_lane<0x114, 0xF>(0, v));
  v = max(v, from_lane<0x118, 0xF>(0, v));
  v = max(v, from_lane<0x142, 0xA>(0, v));   // row_bcast:15, 31
  return max(v, from_lane<0x143, 0xC>(0, v));
}
__device__ __forceinline__ int scan_sum(int v) {
  v += from_lane<0x111, 0xF>(0, v);
  v += from_lane<0x112, 0xF>(0, v);
  v += from_lane<0x114, 0xF>(0, v);
  v += from_lane<0x118, 0xF>(0, v);
  v += from_lane<0x142, 0xA>(0, v);
  return v + from_lane<0x143, 0xC>(0, v);
}
__device__ __forceinline__ int lane_of(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }

__device__ __forceinline__ int clip(int v, int T) { return min(max(v, 0), T); }

// Segments of a sequence of nch chunks: none is longer than those of all rows.
__device__ __forceinline__ int segments_of(const Args& a, int nch) {
  return (nch * a.segments + a.chunks - 1) / a.chunks;
}

// First chunk of segment k of `count`: those that are one chunk longer come first, so that
// two of them seldom share a CU (the second workgroup of a CU comes half a card later):
// 109 us of prompt_scan at 7001 tokens of d_inner 5120, in 12 segments, for 117 with them
// spread evenly.
__device__ __forceinline__ int segment_start(int k, int nch, int count) {
  return k * (nch / count) + min(k, nch % count);
}

// Where chunk c lies.  Offsets below 0, above T or below an earlier one are
// raised or cut to the nearest that is not.  Every wave scans the offsets
// itself, 64 sequences at a time.
__device__ Place find_chunk(const Args& a, int c, bool total) {
  const int lane = threadIdx.x & 63;
  Place p{-1, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
  int chunks = 0, segs = 0, entries = 0, splits = 0;
  int top = clip(a.cu[0], a.T);
  for (int i0 = 0; i0 < a.S; i0 += 64) {
    const int i = i0 + lane, at = min(i, a.S - 1);
    const int offset = a.cu[at + 1];
    const int slot = a.slots ? a.slots[at] : at, pos = a.positions ? a.positions[at] : 0;
    const int e = scan_max(max(i < a.S ? clip(offset, a.T) : 0, top));
    const int up = __builtin_amdgcn_ds_bpermute((lane - 1) * 4, e);
    const int b = lane ? up : top;
    const int len = e - b;
    const int nch = (len + kChunk - 1) / kChunk;
    const int nsg = segments_of(a, nch);
    const int nen = nsg > 1 ? nsg : 0, nsp = nsg > 1 ? 1 : 0;
    const int ci = scan_sum(nch), si = scan_sum(nsg), ei = scan_sum(nen), pi = scan_sum(nsp);
    const int c0 = chunks + ci - nch;
    const uint64_t hit = __ballot(c >= c0 && c < c0 + nch);
    if (hit) {
      const int l = __ffsll((unsigned long long)hit) - 1;
      p.seq = i0 + l;
      p.row0 = lane_of(b, l);
      p.len = lane_of(len, l);
      p.nch = lane_of(nch, l);
      p.k = c - lane_of(c0, l);
      p.seg = segs + lane_of(si - nsg, l);
      p.entry = entries + lane_of(ei - nen, l);
      p.split = splits + lane_of(pi - nsp, l);
      p.slot = lane_of(slot, l);
      p.pos = lane_of(pos, l);
      if (!total) return p;
    }
    chunks += lane_of(ci, 63);
    segs += lane_of(si, 63);
    entries += lane_of(ei, 63);
    splits += lane_of(pi, 63);
    top = lane_of(e, 63);
  }
  p.n_segs = segs;
  p.n_splits = splits;
  return p;
}

// Slot that a sequence keeps its state in, or -1: outside the pool, or named
// by an earlier sequence with tokens.
__device__ int kept_slot(const Args& a, int seq, int slot) {
  if (slot < 0 || slot >= a.n_slots) return -1;
  if (!a.slots) return slot;
  const int lane = threadIdx.x & 63;
  bool hit = false;
  int top = clip(a.cu[0], a.T);
  for (int j0 = 0; j0 < seq; j0 += 64) {
    const int j = j0 + lane;
    const int e = scan_max(max(j < seq ? clip(a.cu[j + 1], a.T) : 0, top));
    const int up = __builtin_amdgcn_ds_bpermute((lane - 1) * 4, e);
    hit |= j < seq && e > (lane ? up : top) && a.slots[j] == slot;
    top = lane_of(e, 63);
  }
  return __ballot(hit) ? -1 : slot;
}

// ---------------------------------------------------------------- arithmetic
// Keeps the phases of a chunk apart: the compiler would start the loads and
// conversions of later ones early, and run out of registers.
#define PHASE() __builtin_amdgcn_sched_barrier(0)

// A value that the compiler takes for new: what depends on it is computed where
// it is used, not once before the loop and kept in registers.
__device__ __forceinline__ int anew(int lane_value) {
  asm volatile("" : "+v"(lane_value));
  return lane_value;
}
__device__ __forceinline__ uint32_t anew_uniform(uint32_t value) {
  asm volatile("" : "+s"(value));
  return value;
}

__device__ __forceinline__ f4 mfma(h8 a, h8 b, f4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// v_exp_f32 and v_rcp_f32 are within an ulp; below v = -88 exp is inf and the
// result -0, where v / (1 + exp(-v)) is below 1e-36
__device__ __forceinline__ float silu(float v) {
  const float e = __builtin_amdgcn_exp2f(-kLog2e * v);
  return v * __builtin_amdgcn_rcpf(1.0f + e);
}
__device__ __forceinline__ float softplus(float v) { return v > 20.0f ? v : log1pf(expf(v)); }

// Exponent that scales values of magnitude up to m into fp16's range, [2^14,
// 2^15) for the largest; at most 60, so that two of them still have a factor that
// takes them back.  (Values that are all below 2^-46 keep an error of 2^-85.)
__device__ __forceinline__ int scale_exp(float m) {
  const int e = (__float_as_int(m) >> 23) & 255;
  return 141 - max(e, 81);
}
__device__ __forceinline__ float pow2(int e) { return __int_as_float((127 + e) << 23); }
// 2^-e for the sum of two of them: from 2^-120 up, and infinity from 2^128 on, where
// the product of the largest values is past fp32 by 2^28: no finite value is wrong for
// want of a second factor, which every sum would have to be multiplied with.
__device__ __forceinline__ float unscale(int e) { return pow2(min(-e, 128)); }

// Two products, a packed conversion, two v_fma_mix_f32 (what is left of a value, exact
// since the scale is a power of two) and a packed conversion for two values: 23 clocks
// with two waves a SIMD.  v_fma_mixlo / mixhi_f16, one instruction a half, take 8.8
// clocks each.
__device__ __forceinline__ void split8(const float (&v)[8], float scale, h8& hi, h8& lo) {
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const h2 p = __builtin_convertvector((f2{v[e] * scale, v[e + 1] * scale}), h2);
    const float l0 = __builtin_fmaf(v[e], scale, -(float)p[0]), l1 = __builtin_fmaf(v[e + 1], scale, -(float)p[1]);
    const h2 q = __builtin_convertvector((f2{l0, l1}), h2);
    hi[e] = p[0], hi[e + 1] = p[1];
    lo[e] = q[0], lo[e + 1] = q[1];
  }
}

// The same for values that are in range as they are; one: 1, unknown to the
// compiler, which would convert back and subtract otherwise.
__device__ __forceinline__ void split8(const float (&v)[8], h8& hi, h8& lo, float one) {
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const h2 p = __builtin_convertvector((f2{v[e], v[e + 1]}), h2);
    const float l0 = __builtin_fmaf(v[e], one, -(float)p[0]), l1 = __builtin_fmaf(v[e + 1], one, -(float)p[1]);
    const h2 q = __builtin_convertvector((f2{l0, l1}), h2);
    hi[e] = p[0], hi[e + 1] = p[1];
    lo[e] = q[0], lo[e + 1] = q[1];
  }
}

// maximum over the lanes l, l ^ 16, l ^ 32, l ^ 48 (not negative: ordered as bits)
__device__ __forceinline__ float max_groups(float f) {
  unsigned v = (unsigned)__float_as_int(f);
  auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(p[0], p[1]);
  p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return __int_as_float((int)max(p[0], p[1]));
}

// ---------------------------------------------------------------- chunks
// Chunk, shared part: the convolution and silu of B and C, their operands and C B^T.
template <int N>
__device__ void chunk_operands(const Args& a, int c, const Place& p, int slot, bool fresh, int pos, int n,
                               char* lds) {
  using L = Lay<N>;
  constexpr int CH = 2 * N, ROW = CH + 4;      // + 4: rows of a read in different banks
  constexpr int PARTS = kChunkThreads / CH, TP = kChunk / PARTS;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  float* xs = reinterpret_cast<float*>(lds);   // [64][ROW]: B, then C
  float* gs = xs;                              // [64][68] C B^T, once nobody reads xs
  float* red = xs + kChunk * ROW;              // [8][2], [8]
  {
    const int ch = tid % CH, t0 = (tid / CH) * TP;
    const int cc = a.d_inner + ch, conv_dim = a.d_inner + CH;
    const float* u = a.zx + ((int64_t)p.row0 + p.k * kChunk) * a.ld + a.d_inner + cc;
    const float4 w = *reinterpret_cast<const float4*>(a.conv_w + 4 * (int64_t)cc);
    const float b = a.conv_b[cc];
    float v[TP + 3];
#pragma unroll
    for (int e = 0; e < TP + 3; ++e) {
      const int t = t0 + e - 3;
      v[e] = 0.f;
      if (t >= 0 || p.k > 0)
        v[e] = u[(int64_t)min(t, n - 1) * a.ld];
      else if (!fresh)
        v[e] = a.ring[((int64_t)slot * 4 + ((pos + t) & 3)) * conv_dim + cc];
    }
    float m = 0.f;
#pragma unroll
    for (int e = 0; e < TP; ++e) {
      const float s = silu(fmaf(w.w, v[e + 3], fmaf(w.z, v[e + 2], fmaf(w.y, v[e + 1], fmaf(w.x, v[e], b)))));
      xs[(t0 + e) * ROW + ch] = s;
      m = fmaxf(m, fabsf(s));
    }
    // a wave holds channels of one of the two
    m = __int_as_float((int)dfssm_px::wave_max_bits_u((uint32_t)__float_as_int(m)));
    if (lane == 0) {
      red[2 * wave] = ch < N ? m : 0.f;
      red[2 * wave + 1] = ch < N ? 0.f : m;
    }
  }
  __syncthreads();
  float mb = 0.f, mc = 0.f;
#pragma unroll
  for (int i = 0; i < kChunkThreads / 64; ++i) {
    mb = fmaxf(mb, red[2 * i]);
    mc = fmaxf(mc, red[2 * i + 1]);
  }
  const int eb = scale_exp(mb), ec = scale_exp(mc);
  const float sb = pow2(eb), sc = pow2(ec);
  char* ops = a.ops + (int64_t)c * L::units * 1024;

  // C: rows i = 16 rt + l % 16, k slot 8 g + e is state column 32 ks + 4 g + e (+ 12 from e = 4 on), the
  // order in which an MFMA result holds the state
  auto gather = [&](int i, int col, float (&v)[8]) {
    const float* s = xs + i * ROW + col;
    const float4 lo4 = *reinterpret_cast<const float4*>(s), hi4 = *reinterpret_cast<const float4*>(s + 16);
    v[0] = lo4.x, v[1] = lo4.y, v[2] = lo4.z, v[3] = lo4.w, v[4] = hi4.x, v[5] = hi4.y, v[6] = hi4.z, v[7] = hi4.w;
  };
  for (int i = wave; i < 4 * L::KS; i += kChunkThreads / 64) {
    const int rt = i / L::KS, ks = i % L::KS;
    float v[8];
    gather(16 * rt + lane % 16, N + 32 * ks + 4 * (lane / 16), v);
    h8 hi, lo;
    split8(v, sc, hi, lo);
    h8* o = reinterpret_cast<h8*>(ops + (i * 2) * 1024) + lane;
    o[0] = hi;
    o[64] = lo;
  }
  // B transposed: rows n = 16 nt + l % 16, k slot 8 g + e is token 32 s + 8 g + e
  for (int i = wave; i < L::NT * 2; i += kChunkThreads / 64) {
    const int nt = i / 2, s = i % 2;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = xs[(32 * s + 8 * (lane / 16) + e) * ROW + 16 * nt + lane % 16];
    h8 hi, lo;
    split8(v, sb, hi, lo);
    h8* o = reinterpret_cast<h8*>(ops + L::b_global + i * 2048) + lane;
    o[0] = hi;
    o[64] = lo;
  }
  // C B^T, the tiles on and below the diagonal: at most two a wave
  float gm = 0.f;
  f4 g[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int i = wave + u * (kChunkThreads / 64);
    if (i >= 10) break;
    const int rt = i < 1 ? 0 : i < 3 ? 1 : i < 6 ? 2 : 3, jt = i - rt * (rt + 1) / 2;
    g[u] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < L::KS; ++ks) {
      float vc[8], vb[8];
      gather(16 * rt + lane % 16, N + 32 * ks + 4 * (lane / 16), vc);
      gather(16 * jt + lane % 16, 32 * ks + 4 * (lane / 16), vb);
      h8 ch, cl, bh, bl;
      split8(vc, sc, ch, cl);
      split8(vb, sb, bh, bl);
      g[u] = mfma(ch, bh, g[u]);
      g[u] = mfma(ch, bl, g[u]);
      g[u] = mfma(cl, bh, g[u]);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      g[u][r] *= unscale(eb + ec);
      gm = fmaxf(gm, fabsf(g[u][r]));
    }
  }
  gm = __int_as_float((int)dfssm_px::wave_max_bits_u((uint32_t)__float_as_int(gm)));
  if (lane == 0) red[16 + wave] = gm;
  __syncthreads();
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int i = wave + u * (kChunkThreads / 64);
    if (i >= 10) break;
    const int rt = i < 1 ? 0 : i < 3 ? 1 : i < 6 ? 2 : 3, jt = i - rt * (rt + 1) / 2;
#pragma unroll
    for (int r = 0; r < 4; ++r) gs[(16 * rt + 4 * (lane / 16) + r) * 68 + 16 * jt + lane % 16] = g[u][r];
  }
  for (int i = 0; i < kChunkThreads / 64; ++i) gm = fmaxf(gm, red[16 + i]);
  for (int h = tid; h < a.H; h += kChunkThreads) {
    float* o = a.tok + ((int64_t)c * a.H + h) * kTokFloats;
    o[kEb] = __int_as_float(eb);
    o[kEc] = __int_as_float(ec);
    o[kGMax] = gm;
  }
  __syncthreads();
  // C B^T as an operand: rows i, k slot 8 g + e is token 32 s + 8 g + e; zeros above
  // the diagonal
  for (int i = wave; i < 6; i += kChunkThreads / 64) {
    const int rt = i < 2 ? i : i < 4 ? 2 : 3, s = i < 2 ? 0 : i & 1;
    const int row = 16 * rt + lane % 16, j = 32 * s + 8 * (lane / 16);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = j + e <= row ? gs[row * 68 + j + e] : 0.f;
    float4* o = reinterpret_cast<float4*>(ops + (L::c_units + 2 * i) * 1024) + lane;
    o[0] = make_float4(v[0], v[1], v[2], v[3]);
    o[64] = make_float4(v[4], v[5], v[6], v[7]);
  }
}

// Chunk, kDecayHeads heads: dt, the sums of its decays and what the scan takes of
// them; a wave holds the 64 tokens of a head.
constexpr int kDecayHeads = 32;
template <int N>
__device__ void chunk_decays(const Args& a, int c, const Place& p, int n, int h0, char* lds) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  float* raw = reinterpret_cast<float*>(lds);  // [64 tokens][kDecayHeads + 1]
  const float* z = a.zx + ((int64_t)p.row0 + p.k * kChunk) * a.ld + 2 * a.d_inner + 2 * N + h0;
  const int nh = min(kDecayHeads, a.H - h0);
  for (int i = tid; i < kChunk * kDecayHeads; i += kChunkThreads) {
    const int t = i / kDecayHeads, h = i % kDecayHeads;
    if (t < n && h < nh) raw[t * (kDecayHeads + 1) + h] = z[t * a.ld + h];
  }
  // A log2(e) of all of them, a lane each
  const double Ahead = -1.4426950408889634 * exp((double)a.A_log[h0 + min(lane, nh - 1)]);
  const float bhead = a.dt_bias[h0 + min(lane, nh - 1)];
  __syncthreads();
  for (int h = wave; h < nh; h += kChunkThreads / 64) {
    const double A = __hiloint2double(lane_of(__double2hiint(Ahead), h), lane_of(__double2loint(Ahead), h));
    const float bias = __int_as_float(lane_of(__float_as_int(bhead), h));
    float dt = 0.f, own = 0.f;
    if (lane < n) {
      dt = softplus(raw[lane * (kDecayHeads + 1) + h] + bias);
      // one rounding: an error of A would be the same in every token of the sum
      own = (float)((double)dt * A);
    }
    float up = own, down = own;
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) {
      const float u = __shfl_up(up, d, 8), v = __shfl_down(down, d, 8);
      if ((lane & 7) >= d) up += u;
      if ((lane & 7) + d < 8) down += v;
    }
    down = __shfl_down(down, 1, 8);
    if ((lane & 7) == 7) down = 0.f;
    const int g = lane >> 3;
    float before = 0.f, behind = 0.f, between = 0.f, all = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float s = __int_as_float(lane_of(__float_as_int(up), 8 * k + 7));
      all += s;
      before += k < g ? s : 0.f;
      behind += k > g ? s : 0.f;
      between += k < g && k > (lane & 7) ? s : 0.f;
    }
    const float m = __int_as_float((int)dfssm_px::wave_max_bits_u((uint32_t)__float_as_int(dt)));
    float* o = a.tok + ((int64_t)c * a.H + h0 + h) * kTokFloats;
    o[kP + lane] = up;
    o[kQ + lane] = down;
    o[kA + lane] = own;
    o[kDt + lane] = dt;
    o[kW + lane] = dt * __builtin_amdgcn_exp2f(down + behind);
    o[kE + lane] = __builtin_amdgcn_exp2f(before + up);
    o[kBd + lane] = between;
    if (lane == 0) o[kAll] = all, o[kDtMax] = m;
  }
}

// Workgroups of a chunk: the shared part, then kDecayHeads heads each.  The shared parts
// come first, since they take longest, and with 32 heads a workgroup instead of 16
// most calls have no second round: at 7001 tokens of d_inner 5120 20.6 us with 16 and
// the parts in the order of the chunks, 15.5 us so.  11 us at 2048 tokens of d_inner
// 4096, which is how long one shared part takes: its loads, then convolution, operands
// and C B^T one after another through LDS.
template <int N>
__global__ __launch_bounds__(kChunkThreads) void prompt_chunks(Args a) {
  extern __shared__ char lds[];
  const int parts = 1 + (a.H + kDecayHeads - 1) / kDecayHeads;
  const int all = gridDim.x / parts, c = blockIdx.x % all, part = blockIdx.x / all, tid = threadIdx.x;
  const Place p = find_chunk(a, c, blockIdx.x == 0);
  if (blockIdx.x == 0 && tid == 0) a.head->n_segs = p.n_segs, a.head->n_splits = p.n_splits;
  if (p.seq < 0) return;
  const int n = min(kChunk, p.len - p.k * kChunk);
  const int count = segments_of(a, p.nch);
  const bool copies = part > 0 && p.k == 0 && count > 1;      // the inputs before a split sequence
  const int at = p.k / (p.nch / count + 1), first =           // the chunk's segment
      at < p.nch % count ? at : (p.k - p.nch % count) / (p.nch / count);
  const bool starts = part == 1 && segment_start(first, p.nch, count) == p.k;
  // the slot, where the ring is read or the segment written
  int slot = -1;
  const int pos = p.pos & 3;
  if (starts || copies || (part == 0 && p.k == 0 && p.pos > 0)) slot = kept_slot(a, p.seq, p.slot);
  const bool fresh = slot < 0 || p.pos <= 0;
  if (part == 0) {
    chunk_operands<N>(a, c, p, slot, fresh, pos, n, lds);
    return;
  }
  if (starts && tid == 0) {
    const int end = segment_start(first + 1, p.nch, count);
    a.segs[p.seg + first] = Seg{p.row0, p.len, c, first, count, p.k, end, slot, fresh ? 1 : 0, pos, p.entry + first};
    if (first == 0 && count > 1) a.splits[p.split] = p.seg;
  }
  const int h0 = (part - 1) * kDecayHeads;
  if (copies && !fresh) {
    // of the channels of these heads; all loads before the stores, which might alias them
    constexpr int kChannels = kDecayHeads * kHeadDim, kEach = kChannels / kChunkThreads;
    float v[3][kEach];
#pragma unroll
    for (int e = 0; e < 3; ++e)
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        v[e][i] = a.ring[((int64_t)slot * 4 + ((pos + 1 + e) & 3)) * (a.d_inner + 2 * N) +
                         min(h0 * kHeadDim + i * kChunkThreads + tid, a.d_inner - 1)];
#pragma unroll
    for (int e = 0; e < 3; ++e)
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int ch = h0 * kHeadDim + i * kChunkThreads + tid;
        if (ch < a.d_inner) a.halo[((int64_t)p.entry * 3 + e) * a.d_inner + ch] = v[e][i];
      }
  }
  chunk_decays<N>(a, c, p, n, h0, lds);
}

// ---------------------------------------------------------------- scan
// A workgroup has two heads of a segment and four waves, two of 32 channels a head.
// It takes 80 KB of LDS and at most 256 registers a lane, so that two are on a CU: a
// second wave on a SIMD is what hides waits here, and one head a workgroup would
// bring B and C into LDS twice as often.  Its inputs x are convolved in the lanes
// that hold them as MFMA operands, in prompt_ends and again in prompt_scan: kept in
// memory in between they cost 286 MB at 7001 tokens of d_inner 5120, and 15 us more
// than computing them again.
//
// Lane l of a wave: channels 2 (l % 16) and + 1 of the wave's 32 (operand
// columns of its two tiles), tokens 32 s + 8 (l / 16) + e (operand rows).
struct Wave {
  int id, h;                // uniform: the wave and its head
  bool on;                  // false: a wave past the last head, which repeats it and stores nothing
  int lane, g;
  int ch;                   // first channel of the lane in its head
  __device__ __forceinline__ void renew() {
    lane = anew(lane);
    g = lane >> 4;
    ch = 32 * (id & 1) + 2 * (lane & 15);
  }
};

__device__ __forceinline__ Wave wave_of(const Args& a, int group) {
  Wave v;
  v.id = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  v.lane = threadIdx.x & 63;
  v.h = kHeads * group + (v.id >> 1);
  v.on = v.h < a.H;
  v.h = min(v.h, a.H - 1);
  v.renew();
  return v;
}

// One of the wave, in scalar registers.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ Seg uniform(const Seg& s) {
  const uint32_t lo = (uint32_t)uniform((int)s.row0), hi = (uint32_t)uniform((int)(s.row0 >> 32));
  return Seg{(int64_t)((uint64_t)hi << 32 | lo), uniform(s.len), uniform(s.chunk0), uniform(s.k), uniform(s.count),
             uniform(s.k0), uniform(s.k1), uniform(s.slot), uniform(s.fresh), uniform(s.pos), uniform(s.entry)};
}

struct Pair {
  float a, b;
};
__device__ __forceinline__ Pair load_pair(const float* p) {  // 4-byte aligned
  Pair v;
  __builtin_memcpy(&v, p, 8);
  return v;
}

// The convolution of the lane's two channels.
struct Taps {
  float4 w0, w1;
  Pair b;
};
__device__ __forceinline__ Taps taps_of(const Args& a, const Wave& v) {
  const int c = v.h * kHeadDim + v.ch;
  return Taps{*reinterpret_cast<const float4*>(a.conv_w + 4 * (int64_t)c),
              *reinterpret_cast<const float4*>(a.conv_w + 4 * (int64_t)c + 4), load_pair(a.conv_b + c)};
}

// Buffer over memory of `bytes` from a uniform address.
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef __amdgpu_buffer_rsrc_t Rows;
__device__ __forceinline__ Rows rows_of(const float* p, uint32_t bytes) {
  const uint64_t at = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32));
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>((uint64_t)hi << 32 | lo), 0,
                                           __builtin_amdgcn_readfirstlane((int)bytes), 0x00027000);
}

// The lane's inputs of chunk k: raw[s][e] is token 32 s + 8 g + e - 3.  Past the
// sequence there are zeros (its dt is 0, so nothing comes of them); the three inputs
// before the sequence come from the ring or its copy, or are zeros.  Offsets from the
// chunk's row - 3 stay below 2^32: ld <= 2^22.
struct XRows {
  Rows rows;
  uint32_t step, first;
};
__device__ __forceinline__ XRows x_rows(const Args& a, const Wave& v, const Seg& sg, int k) {
  const uint32_t step = anew_uniform((uint32_t)a.ld * 4u);
  return XRows{rows_of(a.zx + (sg.row0 + (int64_t)k * kChunk - 3) * a.ld + a.d_inner + v.h * kHeadDim,
                       (uint32_t)(min(kChunk, sg.len - k * kChunk) + 3) * step),
               step, 8u * (uint32_t)v.g * step + 4u * (uint32_t)v.ch};
}
constexpr int kXLoads = 22;
__device__ __forceinline__ void load_x(const XRows& x, int i, uint32_t least, Pair (&raw)[2][11]) {
  const int s = i / 11, e = i % 11;
  uint32_t off = x.first + (uint32_t)(32 * s + e) * x.step;
  if (s == 0 && e < 3) off = max(off, least);
  const u2 p = __builtin_amdgcn_raw_buffer_load_b64(x.rows, (int)off, 0, 0);
  raw[s][e] = Pair{__int_as_float((int)p[0]), __int_as_float((int)p[1])};
}
// All of the first chunk of a segment, which may be the sequence's.
template <int N>
__device__ __forceinline__ void load_first_x(const Args& a, const Wave& v, const Seg& sg, int k, Pair (&raw)[2][11]) {
  const XRows x = x_rows(a, v, sg, k);
  const uint32_t least = k == 0 ? 3u * x.step + 4u * (uint32_t)v.ch : 0u;
#pragma unroll
  for (int i = 0; i < kXLoads; ++i) load_x(x, i, least, raw);
  if (k == 0) {
    const int conv_dim = a.d_inner + 2 * N;
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (v.g == 0) {
        raw[0][e] = Pair{0.f, 0.f};
        if (!sg.fresh) {
          const float* from = sg.count > 1 ? a.halo + ((int64_t)sg.entry * 3 + e) * a.d_inner
                                           : a.ring + ((int64_t)sg.slot * 4 + ((sg.pos + 1 + e) & 3)) * conv_dim;
          raw[0][e] = load_pair(from + v.h * kHeadDim + v.ch);
        }
      }
  }
}

// Without new values in its place the old ones would hold their registers to the
// loop's end.
__device__ __forceinline__ void forget(Pair (&raw)[2][11]) {
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int e = 0; e < 11; ++e) raw[s][e] = Pair{0.f, 0.f};
}

// x[tile][s][e] after the convolution and silu
__device__ __forceinline__ void convolve(const Taps& w, const Pair (&raw)[2][11], float (&x)[2][2][8]) {
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const Pair *r = raw[s] + e;
      x[0][s][e] = silu(fmaf(w.w0.w, r[3].a, fmaf(w.w0.z, r[2].a, fmaf(w.w0.y, r[1].a, fmaf(w.w0.x, r[0].a, w.b.a)))));
      x[1][s][e] = silu(fmaf(w.w1.w, r[3].b, fmaf(w.w1.z, r[2].b, fmaf(w.w1.y, r[1].b, fmaf(w.w1.x, r[0].b, w.b.b)))));
      if (e % 4 == 3) PHASE();
    }
}

__device__ __forceinline__ float max16(const float (&x)[2][8]) {
  float m = 0.f;
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(x[s][e]));
  return m;
}

// operands (hi, lo) of x and the exponent of the lane's column
__device__ __forceinline__ int operands(const float (&x)[2][8], h8 (&hi)[2], h8 (&lo)[2]) {
  const int e = scale_exp(max_groups(max16(x)));
  const float sc = pow2(e);
  split8(x[0], sc, hi[0], lo[0]);
  split8(x[1], sc, hi[1], lo[1]);
  return e;
}

__device__ __forceinline__ void read8(const float* p, float (&v)[8]) {
  const float4 lo = *reinterpret_cast<const float4*>(p), hi = *reinterpret_cast<const float4*>(p + 4);
  v[0] = lo.x, v[1] = lo.y, v[2] = lo.z, v[3] = lo.w, v[4] = hi.x, v[5] = hi.y, v[6] = hi.z, v[7] = hi.w;
}

// A column's inputs times w, as they enter the state at the chunk's end.
__device__ __forceinline__ void weigh(const float* w, int g, float (&x)[2][8]) {
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    float t[8];
    read8(w + 32 * s + 8 * g, t);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[s][e] *= t[e];
  }
}

// state = decay * state + B^T xw; state[nt][tile] is column 2 (l % 16) + tile, rows 16 nt + 4 g ..
// The operands of a tile are read while the products of the one before run, and its
// sums are added while those of the one behind do: the waves of a workgroup come
// here together and would wait for LDS and the matrix cores in turn.
// between(i), i < 6 NT: what else the wave has to ask for, behind every second product.
template <int NT, class Between>
__device__ __forceinline__ void update(const h8* B, int lane, float decay, int eb, const h8 (&hi)[2][2],
                                       const h8 (&lo)[2][2], const int (&ex)[2], f4 (&state)[NT][2],
                                       const Between& between) {
  h8 b[4];                     // [s][hi, lo]
  f4 last[2];
  const float f[2] = {unscale(eb + ex[0]), unscale(eb + ex[1])};
  // a product and a v_fmac, at twice the rate of ldexp and v_fma
  auto finish = [&](int nt, int t) {
#pragma unroll
    for (int r = 0; r < 4; ++r) state[nt][t][r] = fmaf(last[t][r], f[t], state[nt][t][r] * decay);
  };
#pragma unroll
  for (int i = 0; i < 4; ++i) b[i] = B[i * 64 + lane];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    h8 next[4];
    if (nt + 1 < NT) {
#pragma unroll
      for (int i = 0; i < 4; ++i) next[i] = B[((nt + 1) * 4 + i) * 64 + lane];
    }
    PHASE();
    f4 acc[2] = {f4{0.f, 0.f, 0.f, 0.f}, f4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int p = 0; p < 6; ++p) {
      const int s = p / 3;
#pragma unroll
      for (int t = 0; t < 2; ++t)
        acc[t] = mfma(b[2 * s + (p % 3 == 1)], p % 3 == 2 ? lo[t][s] : hi[t][s], acc[t]);
      between(6 * nt + p);
      if (nt > 0 && (p == 2 || p == 3)) finish(nt - 1, p - 2);
      PHASE();
    }
    last[0] = acc[0];
    last[1] = acc[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = next[i];
  }
  finish(NT - 1, 0);
  finish(NT - 1, 1);
}

// Copies `units` KB from src to LDS at dst, the workgroup's waves in turn.
__device__ __forceinline__ void fetch_piece(const Wave& v, const char* src, uint32_t dst, int i) {
  dfssm_lin::dma16((uint32_t)(v.lane * 16 + i * kWaves * 1024), src + v.id * 1024,
                   dst + (uint32_t)(i * kWaves + v.id) * 1024u);
}
template <int UNITS>
__device__ __forceinline__ void fetch(const Wave& v, const char* src, uint32_t dst) {
  static_assert(UNITS % kWaves == 0, "every wave copies as many");
#pragma unroll
  for (int i = 0; i < UNITS / kWaves; ++i) fetch_piece(v, src, dst, i);
}
// The values of the workgroup's heads: all of them, or the half from kW on.
__device__ __forceinline__ void fetch_tok(const Args& a, const Wave& v, int c, int group, uint32_t dst) {
  const int h = min(kHeads * group + (v.id >> 1), a.H - 1);
  dfssm_lin::dma16((uint32_t)v.lane * 16u, a.tok + ((int64_t)c * a.H + h) * kTokFloats + (v.id & 1) * 256,
                   dst + (uint32_t)v.id * 1024u);
}
__device__ __forceinline__ void fetch_tok_half(const Args& a, const Wave& v, int c, int group, uint32_t dst) {
  if (v.id & 1) return;
  const int h = min(kHeads * group + (v.id >> 1), a.H - 1);
  dfssm_lin::dma16((uint32_t)v.lane * 16u, a.tok + ((int64_t)c * a.H + h) * kTokFloats + kW,
                   dst + (uint32_t)(v.id >> 1) * 1024u);
}
// Two workgroups share a CU, and the older one's waves go first wherever both could:
// it would finish with the other half done, which then runs alone, at two thirds of
// the rate of the two.  So the fewer chunks a workgroup has left, the lower its priority
// (at 7001 tokens of d_inner 5120 223 us in all for 235).
__device__ __forceinline__ void yield(int chunks_left) {
  if (chunks_left > 5)
    __builtin_amdgcn_s_setprio(3);
  else if (chunks_left > 2)
    __builtin_amdgcn_s_setprio(2);
  else if (chunks_left > 1)
    __builtin_amdgcn_s_setprio(1);
  else
    __builtin_amdgcn_s_setprio(0);
}
constexpr int kYStores = 16;
// All of the wave's loads but the last n have arrived, and its LDS reads are done;
// then the others', too.
template <int n>
__device__ __forceinline__ void arrive() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(n) : "memory");
}

// The same for what the waves have read from and written to LDS.
__device__ __forceinline__ void arrive_lds() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// the wave's part of entry e of the split sequences' states
template <int N>
__device__ __forceinline__ f4* entry_of(const Args& a, int e, const Wave& v) {
  return reinterpret_cast<f4*>(a.ends) + (((int64_t)e * a.H + v.h) * 2 + (v.id & 1)) * (N / 16) * 2 * 64 + v.lane;
}
// the lane's float4 of state tile (nt, t) in a slot
template <int N>
__device__ __forceinline__ f4* slot_of(const Args& a, int slot, const Wave& v, int nt, int t) {
  return reinterpret_cast<f4*>(a.state + (((int64_t)slot * a.H + v.h) * kHeadDim + v.ch + t) * N + 16 * nt + 4 * v.g);
}

// Final states of the segments of split sequences but the last, from zeros; the
// first one also copies the slot's state before the last one overwrites it.
// 52 us at 7001 tokens of d_inner 5120: the inputs are 143 MB, 31 us at the rate of a
// copy, and the instructions of a chunk about 5000 clocks a wave, 35 us with two waves
// a SIMD.
template <int N>
__global__ __launch_bounds__(kThreads, 2) void prompt_ends(Args a) {
  using L = Lay<N>;
  extern __shared__ char lds[];
  const int group = blockIdx.x % a.groups, si = blockIdx.x / a.groups;
  const Seg sg = uniform(a.segs[si]);        // with the count, not after it
  if (si >= a.head->n_segs || sg.k == sg.count - 1) return;
  Wave v = wave_of(a, group);
  const uint32_t base = dfssm_px::lds_addr(lds);
  auto get = [&](int c, int i) {
    const uint32_t to = base + (uint32_t)(i & 1) * L::e_buf;
    fetch<L::b_units>(v, a.ops + (int64_t)c * L::units * 1024 + L::b_global, to);
    fetch_tok_half(a, v, c, group, to + L::b_units * 1024);
  };
  if (v.on && sg.k == 0) {
#pragma unroll
    for (int nt = 0; nt < L::NT; ++nt)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        entry_of<N>(a, sg.entry, v)[(nt * 2 + t) * 64] =
            sg.fresh ? f4{0.f, 0.f, 0.f, 0.f} : *slot_of<N>(a, sg.slot, v, nt, t);
  }
  f4 state[L::NT][2];
#pragma unroll
  for (int nt = 0; nt < L::NT; ++nt) state[nt][0] = state[nt][1] = f4{0.f, 0.f, 0.f, 0.f};
  float sum = 0.f;
  Pair raw[2][11];
  const int k0 = sg.k0, chunks = sg.k1 - k0;
  get(sg.chunk0, 0);
  const Taps taps = taps_of(a, v);
  load_first_x<N>(a, v, sg, k0, raw);
  for (int i = 0; i < chunks; ++i) {
    const int c = sg.chunk0 + i;
    const bool more = i + 1 < chunks;
    yield(chunks - i);
    v.renew();
    float x[2][2][8];
    convolve(taps, raw, x);
    PHASE();
    // B of this chunk, asked for a chunk ago
    arrive<0>();
    // what the next one needs goes between the products and conversions: the four waves
    // come here together, and would stand behind each other's loads
    const XRows rows = x_rows(a, v, sg, min(k0 + i + 1, (sg.len - 1) / kChunk));
    const char* buf = lds + (i & 1) * L::e_buf;
    const float* tok = reinterpret_cast<const float*>(buf + L::b_units * 1024) + (v.id >> 1) * 256;
    h8 hi[2][2], lo[2][2];
    int ex[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if (more) {
#pragma unroll
        for (int e = 0; e < kXLoads / 2; ++e) load_x(rows, 2 * e + t, 0u, raw);
      }
      weigh(tok, v.g, x[t]);
      ex[t] = operands(x[t], hi[t], lo[t]);
      PHASE();
    }
    if (!more) forget(raw);
    const float all = tok[kAll - kW];
    const int eb = uniform(__float_as_int(tok[kEb - kW]));
    sum += all;
    constexpr int kPieces = L::b_units / kWaves;
    const uint32_t to = base + (uint32_t)(~i & 1) * L::e_buf;
    const char* next = a.ops + (int64_t)(c + 1) * L::units * 1024 + L::b_global;
    update<L::NT>(reinterpret_cast<const h8*>(buf), v.lane, __builtin_amdgcn_exp2f(all), eb, hi, lo, ex,
                  state, [&](int at) {
                    if (at < kPieces && more) fetch_piece(v, next, to, at);
                    if (at == kPieces && more) fetch_tok_half(a, v, c + 1, group, to + L::b_units * 1024);
                  });
  }
  if (!v.on) return;
  v.renew();
#pragma unroll
  for (int nt = 0; nt < L::NT; ++nt)
#pragma unroll
    for (int t = 0; t < 2; ++t) entry_of<N>(a, sg.entry + 1, v)[(nt * 2 + t) * 64] = state[nt][t];
  if (v.lane == 0 && !(v.id & 1)) a.decay[(int64_t)sg.entry * a.H + v.h] = sum;
}

// States before the segments of split sequences, in the place of the final states
// that the segments reach from zeros: start 0 is the sequence's, start k + 1 is
// exp(segment k's sum) start k + end k.  A thread walks four elements, and loads all of
// its segments' before the first sum.  12 us for 16 segments of d_inner 4096: 65 MB, 5.5
// TB/s.
constexpr int kMaxSegs = 16;
__global__ __launch_bounds__(256) void prompt_starts(Args a, int elements, int shift) {
  const int i = blockIdx.x * 256 + threadIdx.x;      // f4 of a state; 2^shift of them a head
  if (i >= elements) return;
  const int splits = a.head->n_splits;
  for (int q = blockIdx.y; q < splits; q += gridDim.y) {
    const Seg sg = a.segs[a.splits[q]];
    f4* e = reinterpret_cast<f4*>(a.ends) + (int64_t)sg.entry * elements + i;
    const float* d = a.decay + (int64_t)sg.entry * a.H + (i >> shift);
    f4 v[kMaxSegs];
    float s[kMaxSegs];
#pragma unroll
    for (int k = 0; k < kMaxSegs; ++k) {
      const int at = min(k, sg.count - 1);      // past the last: not used
      v[k] = e[(int64_t)at * elements];
      s[k] = d[(int64_t)min(k, sg.count - 2) * a.H];
    }
#pragma unroll
    for (int k = 1; k < kMaxSegs; ++k) {
      const float f = __builtin_amdgcn_exp2f(s[k - 1]);
#pragma unroll
      for (int r = 0; r < 4; ++r) v[k][r] = fmaf(v[k - 1][r], f, v[k][r]);
      if (k < sg.count) e[(int64_t)k * elements] = v[k];
    }
  }
}

// A chunk: exp(c_i) C h and M while its inputs are on their way, then their convolution
// and M x, and with B, which took the place of the last chunk's, the state's update, while
// the next chunk's C, C B^T, tokens and inputs are asked for and the outputs stored.
// 107 to 112 us at 7001 tokens of d_inner 5120.  A chunk is 3650 clocks of MFMA and 5300 of
// other vector instructions for a wave, and the two waves of a SIMD hide little of the
// one behind the other's: 75 us or more.  Preparing the operands of C h between its products
// instead of before them changed nothing; x taken back from its halves for the update
// instead of kept, and convolved before M, took 122 us where this took 115.
template <int N>
__global__ __launch_bounds__(kThreads, 2) void prompt_scan(Args a) {
  using L = Lay<N>;
  extern __shared__ char lds[];
  const int group = blockIdx.x % a.groups, si = blockIdx.x / a.groups;
  const Seg sg = uniform(a.segs[si]);        // with the count, not after it
  if (si >= a.head->n_segs) return;
  Wave v = wave_of(a, group);
  const uint32_t base = dfssm_px::lds_addr(lds);
  const h8* Bs = reinterpret_cast<const h8*>(lds + L::b_off);
  const int k0 = sg.k0, k1 = sg.k1;
  const float Dh = a.D[v.h];

  auto get_c = [&](int c) {
    fetch<L::head_units>(v, a.ops + (int64_t)c * L::units * 1024, base);
    fetch_tok(a, v, c, group, base + L::tok_off);
  };
  Pair raw[2][11];             // the next chunk's inputs
  // the state before the segment
  f4 state[L::NT][2];
  if (sg.count > 1) {
#pragma unroll
    for (int nt = 0; nt < L::NT; ++nt)
#pragma unroll
      for (int t = 0; t < 2; ++t) state[nt][t] = entry_of<N>(a, sg.entry, v)[(nt * 2 + t) * 64];
  } else {
#pragma unroll
    for (int nt = 0; nt < L::NT; ++nt)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        state[nt][t] = !sg.fresh ? *slot_of<N>(a, sg.slot, v, nt, t) : f4{0.f, 0.f, 0.f, 0.f};
  }
  get_c(sg.chunk0);
  load_first_x<N>(a, v, sg, k0, raw);
  v.renew();
  // arrived here, so that no chunk waits for it behind its own loads
#pragma unroll
  for (int nt = 0; nt < L::NT; ++nt)
#pragma unroll
    for (int t = 0; t < 2; ++t) asm volatile("" : "+v"(state[nt][t]));

  f4 yv[4][2];
  // C, C B^T and the tokens have arrived
  dfssm_lin::wait_vm<kXLoads>();
  // Outputs of chunk k go to a buffer that ends behind the last row, and what lies past
  // it is dropped: branches would leave open how many stores there are to wait for.
  const uint32_t ystep = (uint32_t)a.d_inner * 4u;
  auto y_rows = [&](int k) {
    return rows_of(a.y + (sg.row0 + (int64_t)k * kChunk) * a.d_inner + v.h * kHeadDim,
                   v.on ? (uint32_t)min(kChunk, sg.len - k * kChunk) * ystep : 0u);
  };
  auto store = [&](const Rows& rows, uint32_t first, uint32_t step, int i) {
    const int rt = i / 4, r = i % 4;
    __builtin_amdgcn_raw_buffer_store_b64(
        u2{(uint32_t)__float_as_int(yv[rt][0][r]), (uint32_t)__float_as_int(yv[rt][1][r])}, rows,
        (int)(first + (uint32_t)(16 * rt + r) * step), 0, 0);
  };
  h8 xh[2][2], xl[2][2];
  int ex[2], k = k0;
  int eb;
  float decay;
  for (;;) {
    const int c = sg.chunk0 + k - k0;
    yield(k1 - k);
    v.renew();
    const int i16 = v.lane & 15;
    const h8* Cs = reinterpret_cast<const h8*>(lds);
    const float* Gs = reinterpret_cast<const float*>(lds + L::c_units * 1024);
    const float* tok = reinterpret_cast<const float*>(lds + L::tok_off) + (v.id >> 1) * kTokFloats;
    float x[2][2][8];
    // C, C B^T and the tokens of this chunk, asked for before its x and the last one's
    // outputs; nobody reads the last one's B any more
    arrive<kXLoads + kYStores>();
    PHASE();
    const Taps taps = taps_of(a, v);      // kept over the chunk they would take ten registers
    PHASE();
    decay = __builtin_amdgcn_exp2f(tok[kAll]);             // exp(c_64)
    eb = uniform(__float_as_int(tok[kEb]));
    const int ec = uniform(__float_as_int(tok[kEc]));
    {
      // exp(c_i) C_i h, two row tiles and a k step at a time; operands read one ahead
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) yv[rt][0] = yv[rt][1] = f4{0.f, 0.f, 0.f, 0.f};
      if (!(k == 0 && sg.fresh)) {
        int eh[2];
        h8 hh[2], hl[2], cf[4];          // cf: [row tile][hi, lo]
        auto read_c = [&](int step, h8 (&f)[4]) {
          const int ks = step >> 1, r0 = 2 * (step & 1);
#pragma unroll
          for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int p = 0; p < 2; ++p) f[2 * r + p] = Cs[(((r0 + r) * L::KS + ks) * 2 + p) * 64 + v.lane];
        };
        auto split_state = [&](int ks, h8 (&hi)[2], h8 (&lo)[2]) {
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const f4 p = state[2 * ks][t], q = state[2 * ks + 1][t];
            const float s[8] = {p[0], p[1], p[2], p[3], q[0], q[1], q[2], q[3]};
            split8(s, pow2(eh[t]), hi[t], lo[t]);
          }
        };
        read_c(0, cf);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          float m = 0.f;
#pragma unroll
          for (int nt = 0; nt < L::NT; ++nt)
#pragma unroll
            for (int r = 0; r < 4; ++r) m = fmaxf(m, fabsf(state[nt][t][r]));
          eh[t] = scale_exp(max_groups(m));
        }
#pragma unroll
        for (int step = 0; step < 2 * L::KS; ++step) {
          const int r0 = 2 * (step & 1);
          h8 nf[4];
          if (step + 1 < 2 * L::KS) read_c(step + 1, nf);
          PHASE();
          if (!(step & 1)) split_state(step >> 1, hh, hl);
#pragma unroll
          for (int r = 0; r < 2; ++r) {
#pragma unroll
            for (int t = 0; t < 2; ++t) yv[r0 + r][t] = mfma(cf[2 * r], hh[t], yv[r0 + r][t]);
          }
#pragma unroll
          for (int r = 0; r < 2; ++r) {
#pragma unroll
            for (int t = 0; t < 2; ++t) yv[r0 + r][t] = mfma(cf[2 * r + 1], hh[t], yv[r0 + r][t]);
          }
#pragma unroll
          for (int r = 0; r < 2; ++r) {
#pragma unroll
            for (int t = 0; t < 2; ++t) yv[r0 + r][t] = mfma(cf[2 * r], hl[t], yv[r0 + r][t]);
          }
          PHASE();
#pragma unroll
          for (int i = 0; i < 4; ++i) cf[i] = nf[i];
        }
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) {
          const float4 E = *reinterpret_cast<const float4*>(tok + kE + 16 * rt + 4 * v.g);
          const float Er[4] = {E.x, E.y, E.z, E.w};
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const float f = unscale(ec + eh[t]);
#pragma unroll
            for (int r = 0; r < 4; ++r) yv[rt][t][r] = (yv[rt][t][r] * f) * Er[r];
          }
        }
        PHASE();
      }
      // + M x.  M is the head's: each of its two waves prepares half of the tiles (rows
      // 16 rt .., tokens 32 s ..): those on the diagonal of 32 rows, and one below
      if (L::m_off == 0) arrive_lds();      // C is read
      // the diagonal adds D to its own C_i . B_i dt_i: the bound is that of the sum
      const int em = scale_exp(tok[kGMax] * tok[kDtMax] + fabsf(Dh));
      const float sm = pow2(em);
      h8* Ms = reinterpret_cast<h8*>(lds + L::m_off + (v.id >> 1) * L::m_units * 1024) + v.lane;
      {
        const float one = __int_as_float((int)anew_uniform(0x3f800000u));
        const int half = v.id & 1;
        struct Tile {
          float4 lo, hi;       // C B^T
          float p, bd;         // sums over the row's group up to the row, and between the groups
        };
        auto read_tile = [&](int rt, int s, Tile& f) {
          const int tile = rt < 2 ? rt : 2 * rt - 2 + s, row = 16 * rt + i16;
          f.lo = *reinterpret_cast<const float4*>(Gs + (2 * tile) * 256 + 4 * v.lane);
          f.hi = *reinterpret_cast<const float4*>(Gs + (2 * tile + 1) * 256 + 4 * v.lane);
          f.p = tok[kP + row];
          f.bd = tok[kBd + 8 * (row >> 3) + 4 * s + v.g];
        };
        Tile cur;
        read_tile(2 * half, half, cur);
        float qj[8], dj[8], aj[8];
        read8(tok + kQ + 32 * half + 8 * v.g, qj);
        read8(tok + kDt + 32 * half + 8 * v.g, dj);
        read8(tok + kA + 32 * half + 8 * v.g, aj);
#pragma unroll
        for (int i = 0; i < 3; ++i) {
          const int rt = i < 2 ? 2 * half + i : 2 + half, s = i < 2 ? half : 0;
          const int tile = rt < 2 ? rt : 2 * rt - 2 + s;
          Tile next;
          float nq[8], nd[8];
          if (i == 0) read_tile(2 * half + 1, half, next);
          if (i == 1) {
            read_tile(2 + half, 0, next);
            read8(tok + kQ + 8 * v.g, nq);
            read8(tok + kDt + 8 * v.g, nd);
          }
          PHASE();
          const float top = cur.p + cur.bd;
          const float gb[8] = {cur.lo.x, cur.lo.y, cur.lo.z, cur.lo.w, cur.hi.x, cur.hi.y, cur.hi.z, cur.hi.w};
          float d[8], m[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) d[e] = qj[e] + top;
          float here = 0.f;           // D on the diagonal
          if (i < 2) {
            // the row's own group: the tokens behind j up to the row
            const bool own = 2 * i + (i16 >> 3) == v.g;
            float sum = 0.f;
#pragma unroll
            for (int e = 7; e >= 0; --e) {
              d[e] = own ? sum : d[e];
              sum = e <= (i16 & 7) ? sum + aj[e] : 0.f;
            }
            here = own ? Dh * sm : 0.f;
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            // C B^T is 0 above the diagonal, where the exponent means nothing (it is never above 0)
            m[e] = gb[e] * (__builtin_amdgcn_exp2f(d[e]) * (dj[e] * sm));
            if (i < 2) m[e] += e == (i16 & 7) ? here : 0.f;
          }
          h8 mh, ml;
          split8(m, mh, ml, one);
          Ms[(2 * tile) * 64] = mh;
          Ms[(2 * tile + 1) * 64] = ml;
          PHASE();
          cur = next;
          if (i == 1) {
#pragma unroll
            for (int e = 0; e < 8; ++e) qj[e] = nq[e], dj[e] = nd[e];
          }
        }
      }
      convolve(taps, raw, x);
#pragma unroll
      for (int t = 0; t < 2; ++t) ex[t] = operands(x[t], xh[t], xl[t]);
      PHASE();
      fetch<L::b_units>(v, a.ops + (int64_t)c * L::units * 1024 + L::b_global, base + L::b_off);
      const float mf[2] = {unscale(em + ex[0]), unscale(em + ex[1])};
      arrive_lds();
      h8 mc[2];
      f4 macc[2];
      auto read_m = [&](int i, h8 (&f)[2]) {
        f[0] = Ms[(2 * i) * 64];
        f[1] = Ms[(2 * i + 1) * 64];
      };
      read_m(0, mc);
#pragma unroll
      for (int i = 0; i < 6; ++i) {
        const int rt = i < 2 ? i : i / 2 + 1, s = i < 2 ? 0 : i & 1;
        h8 next[2];
        if (i < 5) read_m(i + 1, next);
        PHASE();
        if (s == 0) macc[0] = macc[1] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < 2; ++t) macc[t] = mfma(mc[0], xh[t][s], macc[t]);
#pragma unroll
        for (int t = 0; t < 2; ++t) macc[t] = mfma(mc[1], xh[t][s], macc[t]);
#pragma unroll
        for (int t = 0; t < 2; ++t) macc[t] = mfma(mc[0], xl[t][s], macc[t]);
        if (s == rt >> 1) {
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) yv[rt][t][r] = fmaf(macc[t][r], mf[t], yv[rt][t][r]);
        }
        PHASE();
        mc[0] = next[0], mc[1] = next[1];
      }
    }
    // the inputs as they enter the state at the chunk's end
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      weigh(tok + kW, v.g, x[t]);
      ex[t] = operands(x[t], xh[t], xl[t]);
      PHASE();
    }
    // B of this chunk; nobody reads its C, C B^T and tokens any more
    arrive<0>();
    if (k + 1 == k1) break;
    // What there is to store and to ask for goes between the products: the four waves
    // come here together, and would stand behind each other's loads.
    constexpr int kPieces = L::head_units / kWaves, kOps = kPieces + 1 + kYStores + kXLoads;
    const uint32_t step = anew_uniform(ystep), first = 4u * (uint32_t)v.g * step + 4u * (uint32_t)v.ch;
    const Rows out = y_rows(k);
    const XRows in = x_rows(a, v, sg, k + 1);
    const char* next = a.ops + (int64_t)(c + 1) * L::units * 1024;
    update<L::NT>(Bs, v.lane, decay, eb, xh, xl, ex, state, [&](int at) {
#pragma unroll
      for (int i = 0; i < kOps; ++i)
        if (i * 6 * L::NT / kOps == at) {
          if (i < kPieces)
            fetch_piece(v, next, base, i);
          else if (i == kPieces)
            fetch_tok(a, v, c + 1, group, base + L::tok_off);
          else if (i < kPieces + 1 + 2 * kYStores) {
            if ((i - kPieces) % 2)
              store(out, first, step, (i - kPieces - 1) / 2);
            else
              load_x(in, (i - kPieces - 2) / 2, 0u, raw);
          } else
            load_x(in, i - kPieces - 1 - kYStores, 0u, raw);
        }
    });
    ++k;
  }
  {
    const uint32_t step = anew_uniform(ystep), first = 4u * (uint32_t)v.g * step + 4u * (uint32_t)v.ch;
    const Rows out = y_rows(k);
    update<L::NT>(Bs, v.lane, decay, eb, xh, xl, ex, state, [&](int at) {
#pragma unroll
      for (int i = 0; i < kYStores; ++i)
        if (i * 6 * L::NT / kYStores == at) store(out, first, step, i);
    });
  }
  if (sg.k != sg.count - 1 || sg.slot < 0) return;
  v.renew();
  // the state and the ring as sg.len single steps would leave them: the newest
  // inputs, at most four, and zeros before the first of a new sequence
  if (v.on) {
#pragma unroll
    for (int nt = 0; nt < L::NT; ++nt)
#pragma unroll
      for (int t = 0; t < 2; ++t) *slot_of<N>(a, sg.slot, v, nt, t) = state[nt][t];
  }
  const int conv_dim = a.d_inner + 2 * N;
  auto keep = [&](int ch) {
    float x[4];                 // loaded before the stores, which might alias them
#pragma unroll
    for (int i = 1; i <= 4; ++i) x[i - 1] = a.zx[(sg.row0 + sg.len - min(i, sg.len)) * a.ld + a.d_inner + ch];
#pragma unroll
    for (int i = 1; i <= 4; ++i)
      if (i <= sg.len || sg.fresh)
        a.ring[((int64_t)sg.slot * 4 + ((sg.pos + sg.len - i) & 3)) * conv_dim + ch] = i <= sg.len ? x[i - 1] : 0.f;
  };
  if (v.on && v.lane < 32) keep(v.h * kHeadDim + 32 * (v.id & 1) + v.lane);
  if (group == 0)
    for (int i = 64 * v.id + v.lane; i < 2 * N; i += kThreads) keep(a.d_inner + i);
}

// ---------------------------------------------------------------- host
struct Sizes {
  int64_t full, segments;      // chunks and segments of a sequence of all rows
  int64_t chunks, segs, splits, entries;
  int64_t table;               // room for segs that does not fall as T grows
};

// Segments of a sequence of all rows: such that they and the pairs of heads come to
// at most two workgroups a CU (at 7001 tokens of d_inner 5120 192 us, with one a CU 228),
// with two chunks or more each (at 2048 tokens of d_inner 4096 73 us, with three or
// more 85, with four or more 76), 16 at most.  Below six chunks prompt_ends and
// prompt_starts cost more than they save: at 320 tokens 44 us whole and 50 split, at
// 384 tokens 50 and 47.
// The others are upper limits over every way to cut T rows into S sequences.  With f
// chunks and g segments for all rows, f >= 2 g, a sequence of n chunks has ceil(n g / f)
// segments, and s sequences have at most f + s - 1 chunks, so at most
//   (sum of n g + s (f - 1)) / f <= g + s + ((s - 1) g - s) / f
// segments; the last term is below (s - 1) / 2, so that is at most g + s - 1 + s / 2.
// Split ones have more than f / g chunks each, so that there are no more than
// f / floor(f / g) <= (3 g - 1) / 2 of them.  None of the limits that the workspace
// follows falls as T or S grows, so that one made for the largest call serves every
// smaller one.
Sizes sizes(int64_t T, int64_t S, int64_t H) {
  Sizes z;
  const int64_t seqs = std::min(S, T);
  z.full = dfssm::ceil_div(T, kChunk);
  const int64_t fit = std::max<int64_t>(1, 512 / dfssm::ceil_div(H, kHeads));
  z.segments = z.full < 6 ? 1 : std::min({(int64_t)kMaxSegs, fit, z.full / 2});
  z.chunks = T / kChunk + seqs;
  if (z.segments == 1) {
    z.segs = z.table = seqs;
    z.splits = z.entries = 0;
    return z;
  }
  z.segs = z.chunks * z.segments / z.full + seqs;
  z.table = z.segments + seqs + seqs / 2;      // segs is one below it at most
  z.splits = std::min(seqs, (3 * z.segments - 1) / 2);
  z.entries = z.segments + z.splits - 1 + z.splits / 2;
  return z;
}

struct Carve {
  size_t head, segs, splits, ops, tok, halo, ends, decay, bytes;
};

Carve carve(int64_t T, int64_t S, int64_t d_inner, int64_t N) {
  size_t off = 0;
  auto take = [&](int64_t n) {
    const size_t o = off;
    off += ((size_t)n + 255) & ~(size_t)255;
    return o;
  };
  const int64_t H = d_inner / kHeadDim;
  const Sizes z = sizes(T, S, H);
  Carve c;
  c.head = take(sizeof(Header));
  c.segs = take((int64_t)sizeof(Seg) * z.table);
  c.splits = take(4 * z.splits);
  c.ops = take(z.chunks * (N == 128 ? Lay<128>::units : Lay<64>::units) * 1024);
  c.tok = take(z.chunks * H * kTokFloats * 4);
  c.halo = take(z.entries * 3 * d_inner * 4);
  c.ends = take(z.entries * d_inner * N * 4);
  c.decay = take(z.entries * H * 4);
  c.bytes = off;
  return c;
}

template <int N>
hipError_t launch(const Args& a, const Sizes& z, hipStream_t st) {
  using L = Lay<N>;
  constexpr int chunk_lds = L::chunk_lds, ends_lds = 2 * L::e_buf;
  // above 64 KB a kernel has to be told that it may, once a device
  static std::atomic<uint64_t> told{0};
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  if (e != hipSuccess) return e;
  const uint64_t bit = device < 64 ? (uint64_t)1 << device : 0;
  if (!(told.load(std::memory_order_relaxed) & bit)) {
    auto tell = [&](const void* kernel, int bytes) {
      if (e == hipSuccess) e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    };
    tell(reinterpret_cast<const void*>(prompt_chunks<N>), chunk_lds);
    tell(reinterpret_cast<const void*>(prompt_ends<N>), ends_lds);
    tell(reinterpret_cast<const void*>(prompt_scan<N>), L::scan_lds);
    if (e != hipSuccess) return e;
    told.fetch_or(bit, std::memory_order_relaxed);
  }
  const dim3 parts((unsigned)(z.chunks * (1 + dfssm::ceil_div(a.H, kDecayHeads))));
  prompt_chunks<N><<<parts, dim3(kChunkThreads), chunk_lds, st>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)(z.segs * a.groups));
  if (z.segments > 1) {
    prompt_ends<N><<<grid, dim3(kThreads), ends_lds, st>>>(a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int elements = a.d_inner * N / 4;
    const dim3 starts((unsigned)dfssm::ceil_div(elements, 256), (unsigned)std::min<int64_t>(z.splits, 2));
    prompt_starts<<<starts, dim3(256), 0, st>>>(a, elements, N == 128 ? 11 : 10);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  prompt_scan<N><<<grid, dim3(kThreads), L::scan_lds, st>>>(a);
  return hipGetLastError();
}

}  // namespace

namespace dfssm {

size_t ssm_prompt_workspace_bytes(int64_t T, int64_t S, int64_t d_inner, int64_t d_state) {
  return T > 0 && S > 0 ? carve(T, S, d_inner, d_state).bytes : 0;
}

hipError_t launch_ssm_prompt(const float* zx, int64_t ld, int64_t T, const int32_t* cu, int64_t S, int64_t d_inner,
                             int64_t d_state, const int32_t* slots, const int32_t* positions, int64_t n_slots,
                             float* ring, const float* conv_w, const float* conv_b, const float* dt_bias,
                             const float* A_log, const float* D, float* state, float* y, void* ws, hipStream_t st) {
  if (T == 0 || S == 0) return hipSuccess;
  const int64_t H = d_inner / kHeadDim;
  const Carve c = carve(T, S, d_inner, d_state);
  const Sizes z = sizes(T, S, H);
  char* b = static_cast<char*>(ws);
  auto f = [&](size_t o) { return reinterpret_cast<float*>(b + o); };
  Args a{zx, ld, (int)T, cu, (int)S, slots, positions, n_slots, (int)d_inner, (int)H, ring, conv_w, conv_b, dt_bias,
         A_log, D, state, y, (int)z.full, (int)z.segments, (int)ceil_div(H, kHeads),
         reinterpret_cast<Header*>(b + c.head), reinterpret_cast<Seg*>(b + c.segs),
         reinterpret_cast<int*>(b + c.splits), b + c.ops, f(c.tok),
         f(c.halo), f(c.ends), f(c.decay)};
  return d_state == 128 ? launch<128>(a, z, st) : launch<64>(a, z, st);
}

}  // namespace dfssm
