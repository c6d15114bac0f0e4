// 4-bit expert weights with group scales: quantisation, the values they stand for, the packed order, and the expert network computed
// from them (occult_expert_ffn_w4) with the arguments and results of occult_expert_ffn.
//
//   w = scale * (code - zero), code 0..15, one scale (bf16) and zero point (8 unless given) per `group` weights along K
//
// The products are bound by streaming the active experts' codes (half a byte per weight, against two in bf16), with the vector
// instructions that turn codes into matrix operands next: v_mfma_f32_16x16x32_bf16 wants 8 bf16 per lane.  Two codes at a time are
// put, by a shift and one and-or, into the mantissas of bf16 numbers in [16, 32): the operand is 16 + code exactly, 7
// instructions per 8 weights.  What is too much, (16 + zero) * sum x, is itself a matrix product with a constant operand, whose result
// is where the accumulation of a group starts; a group's f32 sum is then scaled once, in f32, by the scale of the lane's own weight
// row (weights are the column operand: an accumulator's lane has one weight row).  No weight is rounded on the way.
// f32 layers: x is split into three bf16 parts whose sum it is exactly, and each goes through the matrix instruction.
#include "common.h"
#include "gemm.h"
#include "stream_gemm.h"

#include <type_traits>

namespace occult {

namespace w4 {

constexpr int kBlockK = 128;         // K elements of a code block: one 16-byte load per lane
constexpr int kUnit = 16;            // weight rows of a code block
constexpr int kBlockBytes = kUnit * kBlockK / 2;

// Packed order of one weight matrix (or gate/up pair: NW = 2): codes [unit][K block][matrix of the pair] of 1 KiB, where 16 bytes
// of lane l are its row l % 16 and, dword by dword, K elements j * 32 + (l / 16) * 8 .. + 8; scales likewise
// [unit][K block][matrix][16 rows][128 / group], as bf16, or with zero points as (bf16 scale << 16 | bf16 of -(16 + zero)).
struct Layout {
  int units, kblocks, per_block;     // per_block: scales of a row in a K block
  long long code_bytes, scale_bytes; // of one matrix (pair)
};
static Layout layout(int N, int K, int NW, int group, bool zeros) {
  Layout L;
  L.units = (N + kUnit - 1) / kUnit;
  L.kblocks = (K + kBlockK - 1) / kBlockK;
  L.per_block = kBlockK / group;
  const long long blocks = (long long)L.units * L.kblocks * NW;
  L.code_bytes = blocks * kBlockBytes;
  L.scale_bytes = blocks * kUnit * L.per_block * (zeros ? 4 : 2);
  return L;
}
struct Packed {
  Layout gu, down;
  long long gu_codes, gu_scales, down_codes, down_scales, total;   // byte offsets of the four regions
};
static Packed packed_layout(const occult_cfg_t& c, int group, bool zeros) {
  Packed p;
  const long long n = c.E + c.S;
  auto up = [](long long v) { return (v + 255) & ~255ll; };
  p.gu = layout(c.f, c.d, 2, group, zeros);
  p.down = layout(c.d, c.f, 1, group, zeros);
  p.gu_codes = 0;
  p.gu_scales = up(n * p.gu.code_bytes);
  p.down_codes = p.gu_scales + up(n * p.gu.scale_bytes);
  p.down_scales = p.down_codes + up(n * p.down.code_bytes);
  p.total = p.down_scales + up(n * p.down.scale_bytes);
  return p;
}

// ---- one problem of the products ------------------------------------------------------------------------------------------
struct Args {
  GemmArgs g;                        // A, lda, a_rows, C, ldc, columns of C, groups and their rows, N, K, kseg
  const char *codes, *scales;
  long long code_stride, scale_stride;   // bytes between weight matrices (pairs)
  int kblocks;                       // K blocks of one weight matrix
  int mats;                          // weight matrices that K walks (the shared experts' down projection: S)
};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// `sixteen`: 0x41804180, two bf16 16, in a vector register that the compiler does not know the value of: it then makes one and-or of the
// two operations, which takes one constant from a scalar register and none from the instruction
__device__ __forceinline__ unsigned two_sixteens() {
  unsigned v = 0x41804180u;
  asm volatile("" : "+v"(v));
  return v;
}
__device__ __forceinline__ bf16x8 operand_of(unsigned v, unsigned sixteen) {
  constexpr unsigned kMask = 0x00780078u;
  const u32x4 r = {(v & kMask) | sixteen, (v >> 4 & kMask) | sixteen, (v >> 8 & kMask) | sixteen,
                   (__builtin_amdgcn_alignbit(v, v, 12) & kMask) | sixteen};
  return __builtin_bit_cast(bf16x8, r);
}
// the inverse: 8 codes of consecutive K elements -> the dword that operand_of reads
__device__ __forceinline__ unsigned dword_of(const int (&code)[8]) {
  unsigned v = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) v |= (unsigned)code[2 * i] << (4 * i) | (unsigned)code[2 * i + 1] << (16 + 4 * i);
  return v << 3 | v >> 29;
}
__device__ __forceinline__ bf16x8 splat_bf16(unsigned bits) {
  const unsigned two = bits << 16 | (bits & 0xFFFFu);
  const u32x4 r = {two, two, two, two};
  return __builtin_bit_cast(bf16x8, r);
}

// code - zero itself as an operand, for f32 layers: three times the instructions, and no sum of 16 * x to be taken off again (an f32
// result would show the last bits that cancelling it costs)
__device__ __forceinline__ bf16x8 exact_operand_of(unsigned v, unsigned sixteen, float minus_zero) {
  const u32x4 biased = __builtin_bit_cast(u32x4, operand_of(v, sixteen));
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    r[i] = __float_as_uint(bf16_lo(biased[i]) + minus_zero) >> 16 | (__float_as_uint(bf16_hi(biased[i]) + minus_zero) & 0xFFFF0000u);
  return __builtin_bit_cast(bf16x8, r);
}

// A lane's codes and scales of a K block of one weight matrix, as loaded (nothing is computed from them before they are used, or the
// computation would wait for the load): G scales, in pairs of bf16, or with zero points in words of scale and -(16 + zero).
template <int G, bool ZERO>
struct Block {
  static constexpr int kScaleBytes = G * (ZERO ? 4 : 2), kWords = ZERO ? G : (G + 1) / 2;
  u32x4 q;
  unsigned s[kWords];
  __device__ __forceinline__ void load(const char* codes, const char* scales, unsigned lane16, unsigned scale_off) {
    q = *reinterpret_cast<const u32x4*>(codes + (size_t)lane16);
    const char* sp = scales + (size_t)scale_off;
    if constexpr (kScaleBytes == 2) s[0] = *reinterpret_cast<const uint16_t*>(sp);
    else {
      typedef unsigned Words __attribute__((ext_vector_type(kWords)));
      const Words w = *reinterpret_cast<const Words*>(sp);
#pragma unroll
      for (int i = 0; i < kWords; ++i) s[i] = w[i];
    }
  }
  __device__ __forceinline__ float scale(int g) const {
    if constexpr (ZERO) return __uint_as_float(s[g] & 0xFFFF0000u);
    else return __uint_as_float(g & 1 ? s[g / 2] & 0xFFFF0000u : s[g / 2] << 16);
  }
  __device__ __forceinline__ float minus_zero(int g) const { return ZERO ? __uint_as_float(s[ZERO ? g : 0] << 16) : -24.0f; }
};

// 8 elements of x along K as matrix operands: one, or three whose sum they are (truncations: the rest is exact every time)
template <bool F32>
struct XFrag;
template <>
struct XFrag<false> {
  static constexpr int kParts = 1;
  u32x4 raw;
  __device__ void load(const char* row, int k, int K) {
    raw = u32x4{0, 0, 0, 0};
    if (k < K) raw = *reinterpret_cast<const u32x4*>(row + (size_t)k * 2);
  }
  __device__ void parts(bf16x8 (&p)[1]) const { p[0] = __builtin_bit_cast(bf16x8, raw); }
};
template <>
struct XFrag<true> {
  static constexpr int kParts = 3;
  f32x4 raw[2];
  __device__ void load(const char* row, int k, int K) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      raw[h] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      if (k + 4 * h < K) raw[h] = *reinterpret_cast<const f32x4*>(row + (size_t)(k + 4 * h) * 4);
    }
  }
  __device__ void parts(bf16x8 (&p)[3]) const {
    u32x4 out[3];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a = raw[i / 2][i % 2 * 2], b = raw[i / 2][i % 2 * 2 + 1];
#pragma unroll
      for (int n = 0; n < 3; ++n) {
        const unsigned ua = __float_as_uint(a) & 0xFFFF0000u, ub = __float_as_uint(b) & 0xFFFF0000u;
        out[n][i] = ua >> 16 | ub;
        a -= __uint_as_float(ua);
        b -= __uint_as_float(ub);
      }
    }
#pragma unroll
    for (int n = 0; n < 3; ++n) p[n] = __builtin_bit_cast(bf16x8, out[n]);
  }
};

// Sum over this and the lower lanes: shifts inside rows of 16 lanes, then a row's last lane to the next row, then lane 31 to the upper half
__device__ __forceinline__ int wave_prefix_sum(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);   // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // row_bcast:15, rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // row_bcast:31, rows 2 and 3
  return v;
}

// Row tile and column block of a workgroup.  Workgroups [0, b_blocks) work on the second problem (the shared experts, whose down
// projection has the longest K: they start first), the rest on the first.  The row tiles that read the same weights get ids 8
// apart: they run on the same XCD, at about the same time, and all but the first find the codes in its L2 (500 tokens, 6 of 64 experts:
// with the tiles spread over the XCDs the codes came 2.4 times from memory).  A pair (group, column block) belongs to XCD
// (group * n_cb + block) % 8, so that column blocks that are no multiple of 8 leave no XCD with more of them.
// b_rows, b_units: rows and units of a workgroup of the second problem.
// group = -1: nothing to do.  Called by the whole workgroup, whose first wave does the work.
struct Place {
  TileInfo ti;
  int cb, matrix;                    // column block; weight matrix
};
template <int BM>
__device__ __forceinline__ Place find_place(const Args& first, const Args& second, int b_blocks, int units_per_block, int b_rows,
                                            int b_units, Place* s_place) {
  if (threadIdx.x < 64) {
    const int bid = (int)blockIdx.x, lane = threadIdx.x;
    const GemmArgs& g = (bid < b_blocks ? second : first).g;
    const int per_block = bid < b_blocks ? b_units : units_per_block;
    const int n_cb = ((g.N + kUnit - 1) / kUnit + per_block - 1) / per_block;
    Place p;
    p.ti.group = -1;
    p.ti.m0 = p.ti.rows = p.ti.row_base = p.cb = p.matrix = 0;
    if (bid < b_blocks) {
      const int tiles = (g.M + b_rows - 1) / b_rows;
      const int unit = bid / (8 * tiles) * 8 + (bid & 7);
      if (unit < g.ngroups * n_cb) {
        p.ti.group = unit / n_cb;
        p.ti.m0 = (bid >> 3) % tiles * b_rows;
        p.ti.rows = g.M;
        p.cb = unit % n_cb;
        p.matrix = g.w_base + p.ti.group;
      }
      if (lane == 0) *s_place = p;
    } else {
      const int xcd = (bid - b_blocks) & 7, at = (bid - b_blocks) >> 3;
      if (lane == 0) *s_place = p;
      int before = 0;   // workgroups of this XCD before the groups at hand
      for (int c0 = 0; c0 < g.ngroups; c0 += 64) {
        const int group = c0 + lane;
        const int lo = group < g.ngroups ? g.grp_offset[group] : 0, hi = group < g.ngroups ? g.grp_offset[group + 1] : 0;
        const int matrix = group < g.ngroups ? g.grp_widx[group] : 0;   // beside the offsets: the codes' addresses wait for it
        const int tiles = (hi - lo + BM - 1) / BM;
        const int cb0 = (xcd - group * n_cb) & 7;   // this group's first column block on this XCD
        const int mine = cb0 < n_cb ? (n_cb - cb0 + 7) / 8 : 0;
        const int incl = wave_prefix_sum(tiles * mine);
        const int excl = before + incl - tiles * mine;
        if (at >= excl && at < excl + tiles * mine) {   // at most one lane over all chunks
          p.ti.group = group;
          p.ti.m0 = (at - excl) % tiles * BM;
          p.ti.rows = hi - lo;
          p.ti.row_base = lo;
          p.cb = cb0 + (at - excl) / tiles * 8;
          p.matrix = matrix;
          *s_place = p;
        }
        before += __builtin_amdgcn_readlane(incl, 63);
        if (before > at) break;   // uniform
      }
    }
  }
  __syncthreads();
  Place p = *s_place;
  p.ti.group = __builtin_amdgcn_readfirstlane(p.ti.group);
  p.ti.m0 = __builtin_amdgcn_readfirstlane(p.ti.m0);
  p.ti.rows = __builtin_amdgcn_readfirstlane(p.ti.rows);
  p.ti.row_base = __builtin_amdgcn_readfirstlane(p.ti.row_base);
  p.cb = __builtin_amdgcn_readfirstlane(p.cb);
  p.matrix = __builtin_amdgcn_readfirstlane(p.matrix);
  return p;
}

// The waves of a workgroup take equal parts of K of NB units of 16 output columns (NW matrices each: gate and up, or down) for up
// to 16 rows of one group, and add their sums through LDS in the order of K.  For few rows, where the length of a wave's stream is
// what counts; every wave has kRing - 1 K blocks in flight (gate/up, whose waves have four: one in flight, in fewer registers,
// 10.6 us, three 12.7; 2 tokens, 64 experts and 2 shared).
template <int NB, int NW, int G, bool ZERO, bool F32, int kRing, int WAVES>
__device__ __forceinline__ void split_product(const Args& a, const TileInfo& ti, long long matrix, int unit0, float (*s_red)[NB * NW * 4][64]) {
  constexpr int kSteps = kBlockK / 32, kGroupSteps = kSteps / G;
  constexpr int P = XFrag<F32>::kParts;
  typedef Block<G, ZERO> B;
  const int units = (a.g.N + kUnit - 1) / kUnit;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, c = lane >> 4;
  // this wave's K blocks, counted through the matrices that K walks
  const int blocks = a.kblocks * a.mats;
  const int kb_begin = blocks * wave / WAVES, kb_end = blocks * (wave + 1) / WAVES;

  const char* xrow;
  {
    int lr = ti.m0 + r;
    if (lr >= ti.rows) lr = ti.rows - 1;   // rows past the group's end repeat its last one; dropped at the end
    const long long logical = ti.row_base + lr;
    const long long src = a.g.a_rows ? a.g.a_rows[logical] : logical;
    xrow = static_cast<const char*>(a.g.A) + src * a.g.lda * (F32 ? 4 : 2);
  }
  const unsigned lane16 = lane * 16, scale_off = r * B::kScaleBytes;
  struct Stage {
    B w[NB][NW];
    XFrag<F32> x[kSteps];
  };
  auto load = [&](Stage& st, int kb) {
    const int mat = a.mats == 1 ? 0 : kb / a.kblocks, kin = kb - mat * a.kblocks;   // uniform
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int unit = min(unit0 + nb, units - 1);   // past the last unit: read it again, dropped at the end
      const long long block = ((long long)unit * a.kblocks + kin) * NW;
#pragma unroll
      for (int m = 0; m < NW; ++m)
        st.w[nb][m].load(a.codes + (matrix + mat) * a.code_stride + (block + m) * kBlockBytes,
                         a.scales + (matrix + mat) * a.scale_stride + (block + m) * (kUnit * B::kScaleBytes), lane16, scale_off);
    }
#pragma unroll
    for (int j = 0; j < kSteps; ++j)
      st.x[j].load(xrow + (size_t)mat * a.g.kseg * (F32 ? 4 : 2), kin * kBlockK + j * 32 + c * 8, a.g.kseg);
  };

  f32x4 acc[NB][NW];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int m = 0; m < NW; ++m) acc[nb][m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  const bf16x8 minus24 = splat_bf16(0xC1C0u), ones = splat_bf16(0x3F80u);   // -(16 + 8); 1
  const unsigned sixteen = two_sixteens();
  auto multiply = [&](const Stage& st) {
    bf16x8 xp[kSteps][P];
#pragma unroll
    for (int j = 0; j < kSteps; ++j) st.x[j].parts(xp[j]);
#pragma unroll
    for (int gi = 0; gi < G; ++gi) {
      f32x4 start = {0.0f, 0.0f, 0.0f, 0.0f};   // -24 * sum x, or with zero points sum x
      if constexpr (!F32) {
#pragma unroll
        for (int j = gi * kGroupSteps; j < (gi + 1) * kGroupSteps; ++j)
          start = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xp[j][0], ZERO ? ones : minus24, start, 0, 0, 0);
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int m = 0; m < NW; ++m) {
          const B& w = st.w[nb][m];
          f32x4 part = start;
          if constexpr (ZERO && !F32) {
#pragma unroll
            for (int e = 0; e < 4; ++e) part[e] *= w.minus_zero(gi);
          }
#pragma unroll
          for (int j = gi * kGroupSteps; j < (gi + 1) * kGroupSteps; ++j) {
            const bf16x8 v = F32 ? exact_operand_of(w.q[j], sixteen, w.minus_zero(gi)) : operand_of(w.q[j], sixteen);
#pragma unroll
            for (int n = 0; n < P; ++n) part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xp[j][n], v, part, 0, 0, 0);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[nb][m][e] = fmaf(w.scale(gi), part[e], acc[nb][m][e]);
        }
    }
  };

  Stage ring[kRing];
#pragma unroll
  for (int i = 0; i < kRing - 1; ++i)
    if (kb_begin + i < kb_end) load(ring[i], kb_begin + i);
  for (int kb = kb_begin; kb < kb_end;) {   // wave-uniform
#pragma unroll
    for (int i = 0; i < kRing; ++i) {
      if (kb + kRing - 1 < kb_end) load(ring[(i + kRing - 1) % kRing], kb + kRing - 1);
      multiply(ring[i]);
      if (++kb == kb_end) break;
    }
  }

  // the waves' sums, added in the order of K; wave e < 4 finishes element e of every accumulator
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int m = 0; m < NW; ++m)
#pragma unroll
      for (int e = 0; e < 4; ++e) s_red[wave][(nb * NW + m) * 4 + e][lane] = acc[nb][m][e];
  __syncthreads();
  if (wave >= 4) return;
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    float v[NW];
#pragma unroll
    for (int m = 0; m < NW; ++m) {
      const int at = (nb * NW + m) * 4 + wave;
      v[m] = s_red[0][at][lane];
#pragma unroll
      for (int k = 1; k < WAVES; ++k) v[m] += s_red[k][at][lane];
    }
    const int token = ti.m0 + c * 4 + wave, col = (unit0 + nb) * kUnit + r;
    if (token < ti.rows && col < a.g.N) {
      const float y = NW == 2 ? v[0] / (1.0f + expf(-v[0])) * v[NW - 1] : v[0];
      const size_t at = (size_t)(ti.row_base + token) * a.g.ldc + group_col0(a.g, ti.group) + col;
      if constexpr (F32) static_cast<float*>(a.g.C)[at] = y;
      else static_cast<__bf16*>(a.g.C)[at] = (__bf16)y;   // rounded to nearest: the layer's type between the two products
    }
  }
}

template <int NB, int NW, int G, bool ZERO, bool F32, int kRing, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void w4_gemm(const Args first, const Args second, const int b_blocks) {
  __shared__ Place s_place;
  __shared__ float s_red[WAVES][NB * NW * 4][64];
  const Place place = find_place<16>(first, second, b_blocks, NB, 16, NB, &s_place);
  if (place.ti.group < 0) return;
  split_product<NB, NW, G, ZERO, F32, kRing, WAVES>((int)blockIdx.x < b_blocks ? second : first, place.ti, place.matrix, place.cb * NB, s_red);
}

// The same product for more rows: the four waves of a workgroup take NB units each over the whole K, and share x: a K block of it
// is brought to LDS once per workgroup, in whole cache lines, while the block before it is multiplied.  (With K split over the waves, each
// would read its own quarter of x, row by row: from 8 rows per expert on more bytes than its codes, and 16 cache lines per load.)
constexpr int kPitch = kBlockK * 2 + 16;   // bytes between rows in LDS: 16 rows' 16-byte pieces fall on different banks

// MB: blocks of 16 rows that are multiplied (of the MT that a row tile may have)
template <int MB, int NB, int NW, int G, bool ZERO, int kRing>
__device__ __forceinline__ void tile_product(const Args& a, const TileInfo& ti, long long matrix, int unit0, char* s_x) {
  constexpr int kSteps = kBlockK / 32, kGroupSteps = kSteps / G;
  typedef Block<G, ZERO> B;
  constexpr int kBuffer = 16 * MB * kPitch;
  const int lane = threadIdx.x & 63;
  const int r = lane & 15, c = lane >> 4;
  const int units = (a.g.N + kUnit - 1) / kUnit;

  // staging: thread owns 16-byte piece `piece` of rows tid / 16 + 16 * i
  const int piece = threadIdx.x & 15, row_in = threadIdx.x >> 4;
  int src[MB];
#pragma unroll
  for (int i = 0; i < MB; ++i)   // rows past the group's end repeat its last one; dropped at the end
    src[i] = ti.row_base + min(ti.m0 + row_in + 16 * i, ti.rows - 1);
  if (a.g.a_rows) {
#pragma unroll
    for (int i = 0; i < MB; ++i) src[i] = a.g.a_rows[src[i]];
  }
  const char* xrow[MB];
  auto set_rows = [&]() {   // when the first codes have been asked for
#pragma unroll
    for (int i = 0; i < MB; ++i) xrow[i] = static_cast<const char*>(a.g.A) + (long long)src[i] * a.g.lda * 2 + piece * 16;
  };
  const int blocks = a.kblocks * a.mats;

  struct Stage {
    B w[NB][NW];
    u32x4 x[MB];
  };
  // codes and scales: scalar bases that walk the K blocks (and the matrices), and one 32-bit offset per lane
  const char* code_at[NB];
  const char* scale_at[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const long long block = (long long)min(unit0 + nb, units - 1) * a.kblocks * NW;   // past the last unit: read it again, dropped
    code_at[nb] = a.codes + matrix * a.code_stride + block * kBlockBytes;
    scale_at[nb] = a.scales + matrix * a.scale_stride + block * (kUnit * B::kScaleBytes);
  }
  const unsigned lane16 = lane * 16, scale_off = r * B::kScaleBytes;
  int code_kin = 0;
  // the K block that `code_at` stands at, one weight matrix of it; and on to the next K block
  auto load_code = [&](B& w, int nb, int m) {
    w.load(code_at[nb] + m * kBlockBytes, scale_at[nb] + m * (kUnit * B::kScaleBytes), lane16, scale_off);
  };
  auto advance_codes = [&]() {
    const bool wraps = NW == 1 && ++code_kin == a.kblocks;   // on to the next matrix (gate and up have one)
    if (wraps) code_kin = 0;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      code_at[nb] += NW * kBlockBytes;
      scale_at[nb] += NW * kUnit * B::kScaleBytes;
      if (wraps) {
        code_at[nb] += a.code_stride - (long long)a.kblocks * NW * kBlockBytes;
        scale_at[nb] += a.scale_stride - (long long)a.kblocks * NW * kUnit * B::kScaleBytes;
      }
      // held in scalar registers: the compiler would carry base plus lane offset along per lane, a 64-bit addition for every load
      asm volatile("" : "+s"(code_at[nb]), "+s"(scale_at[nb]));
    }
  };
  auto load_codes = [&](B (&w)[NB][NW]) {   // the next K block's
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int m = 0; m < NW; ++m) load_code(w[nb][m], nb, m);
    advance_codes();
  };
  int x_kin = 0;
  auto load_x = [&](u32x4 (&x)[MB]) {   // the next K block's
    const bool in = x_kin * kBlockK + piece * 8 < a.g.kseg;
    const bool wraps = ++x_kin == a.kblocks && NW == 1;
    const int step = wraps ? (a.g.kseg - (a.kblocks - 1) * kBlockK) * 2 : kBlockK * 2;
    if (wraps) x_kin = 0;
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      x[i] = u32x4{0, 0, 0, 0};
      if (in) x[i] = *reinterpret_cast<const u32x4*>(xrow[i]);
      xrow[i] += step;
    }
  };
  auto store_x = [&](const u32x4 (&x)[MB], int buf) {
#pragma unroll
    for (int i = 0; i < MB; ++i) *reinterpret_cast<u32x4*>(s_x + buf * kBuffer + (row_in + 16 * i) * kPitch + piece * 16) = x[i];
  };

  f32x4 acc[NB][NW][MB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int m = 0; m < NW; ++m)
#pragma unroll
      for (int tb = 0; tb < MB; ++tb) acc[nb][m][tb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  const bf16x8 minus24 = splat_bf16(0xC1C0u), ones = splat_bf16(0x3F80u);   // -(16 + 8); 1
  const unsigned sixteen = two_sixteens();
  // refill: each matrix's registers are loaded again, with the next K block, as soon as its last group has been multiplied
  auto multiply = [&](B (&w_all)[NB][NW], int buf, auto refill) {
#pragma unroll
    for (int gi = 0; gi < G; ++gi) {
      bf16x8 xp[kGroupSteps][MB];
      f32x4 start[MB];   // -24 * sum x, or with zero points sum x
#pragma unroll
      for (int tb = 0; tb < MB; ++tb) {
        start[tb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < kGroupSteps; ++j) {
          xp[j][tb] = *reinterpret_cast<const bf16x8*>(s_x + buf * kBuffer + (tb * 16 + r) * kPitch + (gi * kGroupSteps + j) * 64 + c * 16);
          start[tb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xp[j][tb], ZERO ? ones : minus24, start[tb], 0, 0, 0);
        }
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int m = 0; m < NW; ++m) {
          B& w = w_all[nb][m];
          const float scale = w.scale(gi);
          f32x4 part[MB];
#pragma unroll
          for (int tb = 0; tb < MB; ++tb) {
            part[tb] = start[tb];
            if constexpr (ZERO) {
#pragma unroll
              for (int e = 0; e < 4; ++e) part[tb][e] *= w.minus_zero(gi);
            }
          }
#pragma unroll
          for (int j = 0; j < kGroupSteps; ++j) {
            const bf16x8 v = operand_of(w.q[gi * kGroupSteps + j], sixteen);
#pragma unroll
            for (int tb = 0; tb < MB; ++tb) part[tb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xp[j][tb], v, part[tb], 0, 0, 0);
          }
#pragma unroll
          for (int tb = 0; tb < MB; ++tb)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[nb][m][tb][e] = fmaf(scale, part[tb][e], acc[nb][m][tb][e]);
          if constexpr (decltype(refill)::value) {
            if (gi == G - 1) load_code(w, nb, m);
          }
        }
      if constexpr (G > 1) __builtin_amdgcn_sched_barrier(0);   // or the next groups' x would be read early, and registers spilled
    }
  };

  // x one K block ahead in LDS; one barrier per K block: whoever passes it has read the buffer that is written next
  if constexpr (kRing == 1) {   // codes one K block ahead in the registers of the block before
    B w[NB][NW];
    u32x4 x[MB];
    load_codes(w);   // before x, whose addresses wait for the row indices
    set_rows();
    load_x(x);
    store_x(x, 0);
    __syncthreads();
    for (int kb = 0; kb + 1 < blocks; ++kb) {   // uniform over the workgroup
      load_x(x);
      multiply(w, kb & 1, std::true_type{});
      advance_codes();
      store_x(x, 1 - (kb & 1));
      __syncthreads();
    }
    multiply(w, (blocks - 1) & 1, std::false_type{});
  } else {                      // codes and x kRing - 1 K blocks ahead in registers
    Stage ring[kRing];
#pragma unroll
    for (int i = 0; i < kRing - 1; ++i)
      if (i < blocks) load_codes(ring[i].w);
    set_rows();
#pragma unroll
    for (int i = 0; i < kRing - 1; ++i)
      if (i < blocks) load_x(ring[i].x);
    store_x(ring[0].x, 0);
    __syncthreads();
    for (int kb = 0; kb < blocks;) {   // uniform over the workgroup
#pragma unroll
      for (int i = 0; i < kRing; ++i) {
        Stage& next = ring[(i + kRing - 1) % kRing];
        if (kb + kRing - 1 < blocks) {
          load_x(next.x);
          load_codes(next.w);
        }
        multiply(ring[i].w, i & 1, std::false_type{});
        if (++kb == blocks) break;
        store_x(ring[(i + 1) % kRing].x, 1 - (i & 1));
        __syncthreads();
      }
    }
  }

#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int col = (unit0 + nb) * kUnit + r;
    if (col >= a.g.N) continue;
    __bf16* out = static_cast<__bf16*>(a.g.C) + (size_t)ti.row_base * a.g.ldc + group_col0(a.g, ti.group) + col;
#pragma unroll
    for (int tb = 0; tb < MB; ++tb)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int token = ti.m0 + tb * 16 + c * 4 + e;
        const float g = acc[nb][0][tb][e];
        if (token < ti.rows) out[(size_t)token * a.g.ldc] = (__bf16)(NW == 2 ? g / (1.0f + expf(-g)) * acc[nb][NW - 1][tb][e] : g);
      }
  }
}

// SPLIT: the second problem's workgroups take 16 rows of SPLIT units with K split over the waves, as in w4_gemm (0: they are like the
// first's).  The shared experts' down projection walks the matrices of all of them: with 4 of them and the whole K to a wave,
// 44 K blocks one after the other, which takes longer than the routed experts' whole product up to 64 tokens.
template <int MT, int NB, int NW, int G, bool ZERO, int kRing, int SPLIT>
__global__ __launch_bounds__(256, kRing == 1 ? 2 : 4) void w4_tile_gemm(const Args first, const Args second, const int b_blocks) {
  constexpr int BM = 16 * MT;
  static_assert(MT <= 2, "one or two blocks of rows");
  static_assert(kRing == 1 || kRing % 2 == 0, "the LDS buffers alternate");
  __shared__ Place s_place;
  constexpr int kLds = 2 * BM * kPitch > SPLIT * NW * 4096 ? 2 * BM * kPitch : SPLIT * NW * 4096;
  __shared__ __attribute__((aligned(16))) char s_x[kLds];
  const Place place = find_place<BM>(first, second, b_blocks, 4 * NB, SPLIT ? 16 : BM, SPLIT ? SPLIT : 4 * NB, &s_place);
  const TileInfo& ti = place.ti;
  if (ti.group < 0) return;
  const bool is_second = (int)blockIdx.x < b_blocks;   // uniform
  if constexpr (SPLIT) {
    if (is_second) {
      static_assert(sizeof(float[4][SPLIT * NW * 4][64]) <= sizeof(s_x), "the sums fit where x would be");
      split_product<SPLIT, NW, G, ZERO, false, 3, 4>(second, ti, place.matrix, place.cb * SPLIT,
                                                  reinterpret_cast<float (*)[SPLIT * NW * 4][64]>(s_x));
      return;
    }
  }
  const Args& a = is_second ? second : first;
  const int unit0 = (place.cb * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * NB;
  const int left = ti.rows - ti.m0;   // a tile's empty blocks of 16 rows are not multiplied
  if (MT == 1 || left <= 16) tile_product<1, NB, NW, G, ZERO, kRing>(a, ti, place.matrix, unit0, s_x);
  else tile_product<MT, NB, NW, G, ZERO, kRing>(a, ti, place.matrix, unit0, s_x);
}

// ---- quantisation, values, packing ----------------------------------------------------------------------------------------
// double -> bf16, to nearest even, in one rounding
__device__ __forceinline__ uint16_t bf16_of(double v) {
  float f = (float)v;
  // the float on the far side of a bf16 tie would round twice: step back towards v, whose own rounding the low bits then show
  if (((__float_as_uint(f) & 0xFFFFu) == 0x8000u) && (double)f != v) {
    const bool up = fabs((double)f) < fabs(v);
    return (uint16_t)((__float_as_uint(f) >> 16) + (up ? 1 : 0));
  }
  const unsigned u = __float_as_uint(f);
  return (uint16_t)((u + 0x7FFFu + (u >> 16 & 1)) >> 16);
}
__device__ __forceinline__ float bf16_value(uint16_t b) { return __uint_as_float((unsigned)b << 16); }

// group / 8 neighbouring lanes per group, 8 weights each.  Codes by division in double: the quotient of two floats is never so close to a
// rounding border that double would put it on the other side.  (One thread per group of 128 read a line for every two bytes: 1.1 GB
// of weights 20.7 ms, so 0.7.)
template <bool BF16>
__global__ __launch_bounds__(256) void quantize_kernel(const void* w, long long rows, int K, int group, uint8_t* codes, uint16_t* scales,
                                                       uint8_t* zeros) {
  const int groups = (K + group - 1) / group, lanes = group / 8;
  const long long n = rows * groups * lanes;   // a multiple of `lanes`, like the stride: a group's lanes stay together
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
    const long long at = i / lanes, row = at / groups;
    const int k0 = (int)(at - row * groups) * group + (int)(i % lanes) * 8;
    const size_t base = (size_t)row * K + k0;
    float v[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {   // K is a multiple of 4
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * h + e] = 0.0f;
      if (k0 + 4 * h < K) {
        if constexpr (BF16) {
          const uint2 u = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(w) + base + 4 * h);
          v[4 * h] = bf16_lo(u.x); v[4 * h + 1] = bf16_hi(u.x);
          v[4 * h + 2] = bf16_lo(u.y); v[4 * h + 3] = bf16_hi(u.y);
        } else {
          const f32x4 u = *reinterpret_cast<const f32x4*>(static_cast<const float*>(w) + base + 4 * h);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[4 * h + e] = u[e];
        }
      }
    }
    float lo = 0.0f, hi = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      lo = fminf(lo, v[e]);
      hi = fmaxf(hi, v[e]);
    }
    for (int o = 1; o < lanes; o <<= 1) {
      lo = fminf(lo, __shfl_xor(lo, o, 64));
      hi = fmaxf(hi, __shfl_xor(hi, o, 64));
    }
    const uint16_t sb = bf16_of(zeros ? ((double)hi - (double)lo) / 15.0 : (double)fmaxf(hi, -lo) / 7.0);
    const double s = (double)bf16_value(sb);
    const int z = zeros && s > 0.0 ? (int)fmin(fmax(rint(-(double)lo / s), 0.0), 15.0) : 8;
    if (i % lanes == 0) {
      scales[at] = sb;
      if (zeros) zeros[at] = (uint8_t)z;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (k0 + 4 * h < K) {
        unsigned q = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const double t = s > 0.0 ? rint((double)v[4 * h + e] / s) + z : (double)z;
          q |= (unsigned)fmin(fmax(t, 0.0), 15.0) << (4 * e);
        }
        reinterpret_cast<uint16_t*>(codes)[(base + 4 * h) / 4] = (uint16_t)q;
      }
  }
}

// 4 weights per thread (K is a multiple of 4, and of the group only where a row ends with one)
template <bool BF16>
__global__ __launch_bounds__(256) void dequantize_kernel(const uint8_t* codes, const uint16_t* scales, const uint8_t* zeros,
                                                         long long rows, int K, int group, void* w) {
  const int groups = (K + group - 1) / group, quads = K / 4;
  const long long n = rows * quads;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
    const long long row = i / quads;
    const int k = (int)(i - row * quads) * 4;
    const long long g = row * groups + k / group;
    const float s = bf16_value(scales[g]);
    const float z = zeros ? (float)(zeros[g] & 15) : 8.0f;
    const unsigned q = reinterpret_cast<const uint16_t*>(codes)[((size_t)row * K + k) / 4];
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = s * ((float)(q >> (4 * e) & 15) - z);
    if constexpr (BF16) reinterpret_cast<uint2*>(w)[i] = uint2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    else reinterpret_cast<float4*>(w)[i] = float4{v[0], v[1], v[2], v[3]};
  }
}

// one thread per dword of a code block, all matrices of one kind; matrix m of a pair goes between the other's blocks
__global__ __launch_bounds__(256) void pack_codes_kernel(const uint8_t* codes, long long mats, int N, int K, int units, int kblocks, int NW,
                                                         int m, unsigned* out) {
  const long long per_mat = (long long)units * kblocks * 256, n = mats * per_mat;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
    const long long mat = i / per_mat, rest = i - mat * per_mat, block = rest / 256;
    const int in = (int)(rest & 255), lane = in >> 2, j = in & 3;
    const int row = (int)(block / kblocks) * kUnit + (lane & 15);
    const int k = (int)(block % kblocks) * kBlockK + j * 32 + (lane >> 4) * 8;
    int q[8];
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      unsigned byte = 0x88;   // past the matrix: the value is never used, or multiplied by zeros
      if (row < N && k + e < K) byte = codes[(((size_t)mat * N + row) * K + k + e) / 2];
      q[e] = byte & 15;
      q[e + 1] = byte >> 4;
    }
    out[(mat * units * kblocks * NW + block * NW + m) * 256 + in] = dword_of(q);
  }
}
__global__ __launch_bounds__(256) void pack_scales_kernel(const uint16_t* scales, const uint8_t* zeros, long long mats, int N, int K,
                                                          int group, int units, int kblocks, int NW, int m, void* out) {
  const int G = kBlockK / group, groups = (K + group - 1) / group, per_block = kUnit * G;
  const long long per_mat = (long long)units * kblocks * per_block, n = mats * per_mat;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
    const long long mat = i / per_mat, rest = i - mat * per_mat, block = rest / per_block;
    const int in = (int)(rest % per_block);
    const int row = (int)(block / kblocks) * kUnit + in / G, g = (int)(block % kblocks) * G + in % G;
    unsigned s = 0, z = 8;
    if (row < N && g < groups) {
      const size_t at = ((size_t)mat * N + row) * groups + g;
      s = scales[at];
      if (zeros) z = zeros[at] & 15;
    }
    const size_t at = (size_t)(mat * units * kblocks * NW + block * NW + m) * per_block + in;
    if (zeros) static_cast<unsigned*>(out)[at] = s << 16 | (__float_as_uint(-(16.0f + (float)z)) >> 16);
    else static_cast<uint16_t*>(out)[at] = (uint16_t)s;
  }
}

static int check_group(int group) {
  OCC_REQUIRE(group == 32 || group == 64 || group == 128, OCCULT_EINVAL, "group=%d must be 32, 64 or 128", group);
  return OCCULT_OK;
}
static int check_rows(const occult_cfg_t& c) {
  const int es = elem_size(c);
  OCC_REQUIRE(((size_t)c.d * es) % 16 == 0 && ((size_t)c.f * es) % 16 == 0, OCCULT_EALIGN,
              "rows of d=%d or f=%d elements are not multiples of 16 bytes", c.d, c.f);
  return OCCULT_OK;
}
static int check_codes(const occult_cfg_t& c, const occult_w4_weights_t* q) {
  int rc = check_rows(c);
  if (rc) return rc;
  OCC_REQUIRE(q, OCCULT_ENULLPTR, "codes are NULL");
  rc = check_group(q->group);
  if (rc) return rc;
  for (int i = 0; i < 3; ++i) {
    OCC_REQUIRE(q->codes[i] && q->scales[i], OCCULT_ENULLPTR, "codes[%d] or scales[%d] is NULL", i, i);
    OCC_REQUIRE((q->zeros[i] != nullptr) == (q->zeros[0] != nullptr), OCCULT_ENULLPTR,
                "zero points of some matrices and not of others");
    OCC_REQUIRE(aligned16(q->codes[i]) && ((uintptr_t)q->scales[i] & 1) == 0, OCCULT_EALIGN, "codes[%d] or scales[%d] is not aligned",
                i, i);
  }
  return OCCULT_OK;
}
static int grid_for(long long threads) {
  const long long blocks = (threads + 255) / 256;
  return (int)(blocks < 16384 ? blocks : 16384);
}

// TILE: w4_tile_gemm, whose workgroups have 4 * NB units (of the second problem SPLIT, if not 0); else w4_gemm with NB.
// MIN_GROUP: the finest groups that the caller's rule sends here.
template <bool TILE, int MT, int NB, int NW, bool F32, int RING, int SPLIT = 0, int WAVES = 4, int MIN_GROUP = 32>
static int launch_typed(const Args& a, const Args* b, int group, bool zeros, int total_rows, hipStream_t s) {
  constexpr int BM = 16 * MT, UNITS = TILE ? 4 * NB : NB, B_ROWS = SPLIT ? 16 : BM, B_UNITS = SPLIT ? SPLIT : UNITS;
  const int n_cb = ((a.g.N + kUnit - 1) / kUnit + UNITS - 1) / UNITS;
  // row tiles of the grouped rows: at most one partly filled one per group, and none without a row
  long long m_tiles = ((long long)total_rows + (long long)a.g.ngroups * (BM - 1)) / BM;
  if (m_tiles > total_rows) m_tiles = total_rows;
  const long long a_blocks = m_tiles * ((n_cb + 7) / 8) * 8;   // an XCD has at most ceil(n_cb / 8) column blocks of a group
  const int b_cb = ((a.g.N + kUnit - 1) / kUnit + B_UNITS - 1) / B_UNITS;
  const long long b_blocks = b ? (b->g.ngroups * (long long)b_cb + 7) / 8 * 8 * ((b->g.M + B_ROWS - 1) / B_ROWS) : 0;
  const long long grid = a_blocks + b_blocks;
  OCC_REQUIRE(grid < (1ll << 24), OCCULT_ESHAPE, "%lld workgroups are too many for one launch", grid);
  const Args& second = b ? *b : a;
#define OCC_W4_CASE(G_, Z_)                                                                                                \
  if (group == kBlockK / G_ && zeros == Z_) {                                                                              \
    if constexpr (TILE) w4_tile_gemm<MT, NB, NW, G_, Z_, RING, SPLIT><<<(int)grid, 256, 0, s>>>(a, second, (int)b_blocks); \
    else w4_gemm<NB, NW, G_, Z_, F32, RING, WAVES><<<(int)grid, 64 * WAVES, 0, s>>>(a, second, (int)b_blocks);             \
    OCC_LAUNCH_CHECK(TILE ? "w4_tile_gemm" : "w4_gemm");                                                                   \
    return OCCULT_OK;                                                                                                      \
  }
  OCC_W4_CASE(1, false)
  OCC_W4_CASE(2, false)
  OCC_W4_CASE(1, true)
  OCC_W4_CASE(2, true)
  if constexpr (MIN_GROUP == 32) {
    OCC_W4_CASE(4, false)
    OCC_W4_CASE(4, true)
  }
#undef OCC_W4_CASE
  OCC_FAIL(OCCULT_EINVAL, "group=%d", group);
}

// a: the routed experts' grouped rows; b: the shared experts', or NULL.  Times below: gate/up or down product of the layers with 60 (4 per
// token, 4 shared) and 64 experts (8 per token), K = 2048 and 1408 or 1024.
template <int NW>
static int launch(const occult_cfg_t& c, const Args& a, const Args* b, int group, bool zeros, hipStream_t s) {
  const int rows = c.T * c.k;
  if (c.dtype == OCCULT_F32) return launch_typed<false, 1, 2, NW, true, 2>(a, b, group, zeros, rows, s);
  // K split over the waves while whole-K workgroups would not fill the chip two or three times: gate/up, 1 token 8.9 against
  // 13.0 us (60 experts), 2 tokens 10.9 against 15.8 (64, none shared), 3 tokens 15.5 against 18.9 (64, 6 per token, 2 shared: 440
  // workgroups); equal from 6 tokens on (60: 616).  Down: 2 tokens 10.0 against 15.0 (64, 2 shared: 416), 3 tokens 11.0 against 17.2 (608).
  const long long tiles = min_i(rows, rows / 16 + c.E) + (b ? (long long)b->g.ngroups * ((c.T + 15) / 16) : 0);
  // Eight waves for the down product, which may have a long sum over shared experts beside short ones (1 token, 4 shared 8.8 against 10.6 us
  // with four, 2 tokens 9.4 against 10.9; none shared 5.9 against 6.0); four for gate/up (2 tokens 10.5 against 11.1).
  if (tiles * ((a.g.N + 4 * kUnit - 1) / (4 * kUnit)) <= 640)
    return launch_typed<false, 1, NW == 2 ? 1 : 2, NW, false, 2, 0, NW == 2 ? 4 : 8>(a, b, group, zeros, rows, s);
  const long long per_expert = rows / c.E;
  if constexpr (NW == 1) {
    // A long sum over the shared experts' matrices beside short routed ones (K blocks: 44 of 4 shared experts, 22 of 2): 4 tokens split 12.2
    // against 24.3 us, 17 tokens 20.8 against 33.1, 64 tokens 27.7 against 38.4 (29.1 with codes three blocks ahead), 128 tokens 38.9
    // against 40.7 (36.2 with codes three blocks ahead).  With 2 shared, 4 tokens 11.1 against 13.7, 17 tokens 22.8 against 22.7.
    // Nothing between 22 and 44 K blocks, or below 22, was measured: the borders at 20 and 32 stand for those two.
    const int chain = b ? b->mats * b->kblocks : 0;
    if ((chain >= 20 && chain >= c.T) || (chain >= 32 && c.T <= 64)) return launch_typed<true, 1, 1, 1, false, 1, 2>(a, b, group, zeros, rows, s);
    if (chain >= 32 && per_expert < 12) return launch_typed<true, 1, 1, 1, false, 4>(a, b, group, zeros, rows, s);
  }
  // Tiles of 32 rows decode an expert's codes half as often as tiles of 16, and with two units per wave x is read half as often; both take
  // registers, and so waves that hide latency.  Gate/up, us, 16 rows | 32 rows | 32 rows and two units: 4 rows per expert 38.4 | 41.5 |
  // 39.2; 8 rows 47.6 | 45.7 | 52.6; 16 rows 65.7 | 59.8 | 56.7; 23 rows 65.0 | 59.7 | 57.7; 46 rows 108 | 92 | 83; with groups
  // of 32, whose four scalings per block take registers, 23 rows 72.3 | 67.0 | 71.0, 46 rows 137 | 119 | 125.  Down product: 12 rows
  // 34.1 | 32.3 | 32.5; 16 rows 41.5 | 42.6 | 50.6; 23 rows 43.8 | 41.4 | 37.9; 46 rows 72 | 64 | 52.
  if (per_expert >= (NW == 2 ? 16 : 20) && (NW == 1 || group != 32))
    return launch_typed<true, 2, 2, NW, false, 1, 0, 4, NW == 2 ? 64 : 32>(a, b, group, zeros, rows, s);
  if (per_expert >= 8) return launch_typed<true, 2, 1, NW, false, 1>(a, b, group, zeros, rows, s);
  return launch_typed<true, 1, 1, NW, false, 1>(a, b, group, zeros, rows, s);
}

}  // namespace w4

}  // namespace occult

using namespace occult;
using namespace occult::w4;

extern "C" int occult_quantize_weights(const occult_cfg_t* cfg, const occult_weights_t* weights, const occult_w4_weights_t* out,
                                       occult_stream_t stream) {
  int rc = check_cfg(cfg);
  if (rc) return rc;
  const occult_cfg_t& c = *cfg;
  rc = check_codes(c, out);
  if (rc) return rc;
  OCC_REQUIRE(weights && weights->w_gate && weights->w_up && weights->w_down, OCCULT_ENULLPTR, "weights or one of its tensors is NULL");
  const void* w[3] = {weights->w_gate, weights->w_up, weights->w_down};
  for (int i = 0; i < 3; ++i) OCC_REQUIRE(aligned16(w[i]), OCCULT_EALIGN, "a weight tensor is not 16-byte aligned");
  hipStream_t s = static_cast<hipStream_t>(stream);
  for (int i = 0; i < 3; ++i) {
    const int N = i < 2 ? c.f : c.d, K = i < 2 ? c.d : c.f;
    const long long rows = (long long)(c.E + c.S) * N;
    const int grid = grid_for(rows * ((K + out->group - 1) / out->group) * (out->group / 8));
    if (c.dtype == OCCULT_BF16)
      quantize_kernel<true><<<grid, 256, 0, s>>>(w[i], rows, K, out->group, out->codes[i], out->scales[i], out->zeros[i]);
    else
      quantize_kernel<false><<<grid, 256, 0, s>>>(w[i], rows, K, out->group, out->codes[i], out->scales[i], out->zeros[i]);
    OCC_LAUNCH_CHECK("quantize_kernel");
  }
  return OCCULT_OK;
}

extern "C" int occult_dequantize_weights(const occult_cfg_t* cfg, const occult_w4_weights_t* q, void* w_gate, void* w_up, void* w_down,
                                         occult_stream_t stream) {
  int rc = check_cfg(cfg);
  if (rc) return rc;
  const occult_cfg_t& c = *cfg;
  rc = check_codes(c, q);
  if (rc) return rc;
  OCC_REQUIRE(w_gate && w_up && w_down, OCCULT_ENULLPTR, "w_gate, w_up or w_down is NULL");
  OCC_REQUIRE(aligned16(w_gate) && aligned16(w_up) && aligned16(w_down), OCCULT_EALIGN, "a weight tensor is not 16-byte aligned");
  void* w[3] = {w_gate, w_up, w_down};
  hipStream_t s = static_cast<hipStream_t>(stream);
  for (int i = 0; i < 3; ++i) {
    const int N = i < 2 ? c.f : c.d, K = i < 2 ? c.d : c.f;
    const long long rows = (long long)(c.E + c.S) * N;
    const int grid = grid_for(rows * (K / 4));
    if (c.dtype == OCCULT_BF16)
      dequantize_kernel<true><<<grid, 256, 0, s>>>(q->codes[i], q->scales[i], q->zeros[i], rows, K, q->group, w[i]);
    else
      dequantize_kernel<false><<<grid, 256, 0, s>>>(q->codes[i], q->scales[i], q->zeros[i], rows, K, q->group, w[i]);
    OCC_LAUNCH_CHECK("dequantize_kernel");
  }
  return OCCULT_OK;
}

extern "C" int occult_pack_w4_bytes(const occult_cfg_t* cfg, int group, int zeros, size_t* bytes) {
  int rc = check_cfg(cfg);
  if (rc == OCCULT_OK) rc = check_rows(*cfg);
  if (rc == OCCULT_OK) rc = check_group(group);
  if (rc) return rc;
  OCC_REQUIRE(zeros == 0 || zeros == 1, OCCULT_EINVAL, "zeros=%d must be 0 or 1", zeros);
  OCC_REQUIRE(bytes, OCCULT_ENULLPTR, "output pointer is NULL");
  *bytes = (size_t)packed_layout(*cfg, group, zeros != 0).total;
  return OCCULT_OK;
}

extern "C" int occult_pack_w4(const occult_cfg_t* cfg, const occult_w4_weights_t* q, void* packed, size_t packed_size,
                              occult_stream_t stream) {
  int rc = check_cfg(cfg);
  if (rc) return rc;
  const occult_cfg_t& c = *cfg;
  rc = check_codes(c, q);
  if (rc) return rc;
  const bool zeros = q->zeros[0] != nullptr;
  const Packed p = packed_layout(c, q->group, zeros);
  OCC_REQUIRE(packed, OCCULT_ENULLPTR, "packed is NULL");
  OCC_REQUIRE(aligned16(packed), OCCULT_EALIGN, "packed is not 16-byte aligned");
  OCC_REQUIRE(packed_size >= (size_t)p.total, OCCULT_EWORKSPACE, "packed buffer of %zu bytes < required %lld", packed_size, p.total);
  char* out = static_cast<char*>(packed);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const long long mats = c.E + c.S;
  for (int i = 0; i < 3; ++i) {
    const int N = i < 2 ? c.f : c.d, K = i < 2 ? c.d : c.f, NW = i < 2 ? 2 : 1, m = i == 1;
    const Layout& L = i < 2 ? p.gu : p.down;
    const long long blocks = mats * L.units * L.kblocks;
    pack_codes_kernel<<<grid_for(blocks * 256), 256, 0, s>>>(q->codes[i], mats, N, K, L.units, L.kblocks, NW, m,
                                                              reinterpret_cast<unsigned*>(out + (i < 2 ? p.gu_codes : p.down_codes)));
    OCC_LAUNCH_CHECK("pack_codes_kernel");
    pack_scales_kernel<<<grid_for(blocks * kUnit * L.per_block), 256, 0, s>>>(q->scales[i], q->zeros[i], mats, N, K, q->group, L.units,
                                                                               L.kblocks, NW, m,
                                                                               out + (i < 2 ? p.gu_scales : p.down_scales));
    OCC_LAUNCH_CHECK("pack_scales_kernel");
  }
  return OCCULT_OK;
}

extern "C" int occult_expert_ffn_w4(const occult_cfg_t* cfg, const occult_plan_t* plan, const void* sfd_x, const void* x,
                                    const void* packed, size_t packed_size, int group, int zeros, void* epd_h, void* epd_y,
                                    void* h_shared, void* y_shared, occult_stream_t stream) {
  size_t need = 0;
  int rc = occult_pack_w4_bytes(cfg, group, zeros, &need);
  if (rc) return rc;
  const occult_cfg_t& c = *cfg;
  OCC_REQUIRE(plan && plan->exp_offset && plan->pos_expert && plan->epd_sfd_row, OCCULT_ENULLPTR, "plan or one of its tables is NULL");
  OCC_REQUIRE(packed, OCCULT_ENULLPTR, "packed is NULL");
  OCC_REQUIRE(packed_size >= need, OCCULT_EWORKSPACE, "packed buffer of %zu bytes < required %zu", packed_size, need);
  OCC_REQUIRE(aligned16(packed) && aligned16(sfd_x) && aligned16(x) && aligned16(epd_h) && aligned16(epd_y) && aligned16(h_shared) &&
                  aligned16(y_shared),
              OCCULT_EALIGN, "a buffer is not 16-byte aligned");
  if (c.T == 0) return OCCULT_OK;
  OCC_REQUIRE(sfd_x && epd_h && epd_y, OCCULT_ENULLPTR, "sfd_x, epd_h or epd_y is NULL");
  if (c.S > 0) OCC_REQUIRE(x && h_shared && y_shared, OCCULT_ENULLPTR, "x, h_shared or y_shared is NULL with S=%d", c.S);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const Packed p = packed_layout(c, group, zeros != 0);
  const char* base = static_cast<const char*>(packed);
  if (c.ffn_phase != 2) {   // h = silu(x W_gate^T) * (x W_up^T)
    Args a{};
    a.codes = base + p.gu_codes; a.scales = base + p.gu_scales;
    a.code_stride = p.gu.code_bytes; a.scale_stride = p.gu.scale_bytes;
    a.kblocks = p.gu.kblocks; a.mats = 1;
    a.g.lda = a.g.K = a.g.kseg = c.d;
    a.g.N = c.f;
    Args b = a;
    a.g.A = sfd_x; a.g.a_rows = plan->epd_sfd_row; a.g.C = epd_h; a.g.ldc = c.f;
    a.g.grp_offset = plan->exp_offset; a.g.grp_widx = plan->pos_expert; a.g.ngroups = c.E;
    b.g.A = x; b.g.C = h_shared; b.g.ldc = c.S * c.f; b.g.c_group_cols = c.f;
    b.g.w_base = c.E; b.g.ngroups = c.S; b.g.M = c.T;
    rc = launch<2>(c, a, c.S > 0 ? &b : nullptr, group, zeros != 0, s);
    if (rc) return rc;
  }
  if (c.ffn_phase != 1) {   // y = h W_down^T; the shared experts as one product whose K walks their down matrices
    Args a{};
    a.codes = base + p.down_codes; a.scales = base + p.down_scales;
    a.code_stride = p.down.code_bytes; a.scale_stride = p.down.scale_bytes;
    a.kblocks = p.down.kblocks; a.mats = 1;
    a.g.kseg = c.f;
    a.g.N = a.g.ldc = c.d;
    Args b = a;
    a.g.A = epd_h; a.g.lda = a.g.K = c.f; a.g.C = epd_y;
    a.g.grp_offset = plan->exp_offset; a.g.grp_widx = plan->pos_expert; a.g.ngroups = c.E;
    b.g.A = h_shared; b.g.lda = b.g.K = c.S * c.f; b.g.C = y_shared; b.mats = c.S;
    b.g.w_base = c.E; b.g.ngroups = 1; b.g.M = c.T;
    rc = launch<1>(c, a, c.S > 0 ? &b : nullptr, group, zeros != 0, s);
  }
  return rc;
}

extern "C" int occult_forward_w4(const occult_cfg_t* cfg, const occult_plan_t* plan, const float* logits, const void* x,
                                 const void* packed, size_t packed_size, int group, int zeros,
                                 const occult_forward_buffers_t* buffers, occult_stream_t stream) {
  int rc = check_cfg(cfg);
  if (rc) return rc;
  OCC_REQUIRE(buffers, OCCULT_ENULLPTR, "buffers is NULL");
  const occult_forward_buffers_t& b = *buffers;
  rc = occult_route(cfg, logits, b.ids, b.w, stream);
  if (rc == OCCULT_OK)
    rc = plan_and_dispatch(cfg, b.ids, b.w, plan, b.plan_ws, b.plan_ws_bytes, x, b.sfd_x, static_cast<hipStream_t>(stream));
  if (rc == OCCULT_OK)
    rc = occult_expert_ffn_w4(cfg, plan, b.sfd_x, x, packed, packed_size, group, zeros, b.epd_h, b.epd_y, b.h_shared, b.y_shared, stream);
  return rc ? rc : occult_combine(cfg, plan, b.epd_y, b.sfd_y, b.y_shared, b.y, stream);
}
