// 4-bit expert weights with group scales: quantisation, the values they stand for, the packed order, and the expert network computed
// from them (occult_expert_ffn_w4) with the arguments and results of occult_expert_ffn.
//
//   w = scale * (code - zero), code 0..15, one scale (bf16) and zero point (8 unless given) per `group` weights along K
//
// The products are bound by streaming the active experts' codes (half a byte per weight, against two in bf16), with the vector
// instructions that turn codes into matrix operands next: v_mfma_f32_16x16x32_bf16 wants 8 bf16 per lane.  Two codes at a time are
// put, by a rotation and one and-or, into the mantissas of bf16 numbers in [16, 32): the operand is 16 + code exactly, 7
// instructions per 8 weights.  What is too much, (16 + zero) * sum x, is itself a matrix product with a constant operand, whose result
// is where the accumulation of a group starts; a group's f32 sum is then scaled once, in f32, by the scale of the lane's own weight
// row (weights are the column operand: an accumulator's lane has one weight row).  No weight is rounded on the way.
// f32 layers: x is split into three bf16 parts whose sum it is exactly, and each goes through the matrix instruction.
#include "common.h"
#include "gemm.h"
#include "stream_gemm.h"

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

__device__ __forceinline__ bf16x8 operand_of(unsigned v) {
  constexpr unsigned kMask = 0x00780078u, kSixteen = 0x41804180u;
  const u32x4 r = {(v & kMask) | kSixteen, (__builtin_amdgcn_alignbit(v, v, 4) & kMask) | kSixteen,
                   (__builtin_amdgcn_alignbit(v, v, 8) & kMask) | kSixteen, (__builtin_amdgcn_alignbit(v, v, 12) & kMask) | kSixteen};
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

// The four waves of a workgroup take the quarters of K of NB units of 16 output columns (NW matrices each: gate and up, or down) for up
// to 16 * MT rows of one group, and add their sums through LDS in the order of K.  G: scales per row and K block; ZERO: with zero points.
template <int MT, int NB, int NW, int G, bool ZERO, bool F32>
__global__ __launch_bounds__(256) void w4_gemm(const Args first, const Args second, const int a_blocks) {
  constexpr int BM = 16 * MT;
  constexpr int kSteps = kBlockK / 32, kGroupSteps = kSteps / G;
  constexpr int P = XFrag<F32>::kParts;
  constexpr int kScaleBytes = (ZERO ? 4 : 2);
  __shared__ TileInfo s_info;
  int bid = (int)blockIdx.x;
  const bool is_second = bid >= a_blocks;   // uniform
  const Args& a = is_second ? second : first;
  const int units = (a.g.N + kUnit - 1) / kUnit, n_cb = (units + NB - 1) / NB;
  int mt, cb;
  if (!is_second) {
    mt = bid / n_cb;
    cb = bid % n_cb;
  } else {   // the row tiles that read the same weights 8 ids apart: on the same XCD, whose L2 then has them
    const int b = bid - a_blocks;
    const int tiles = (a.g.M + BM - 1) / BM;
    const int unit = b / (8 * tiles) * 8 + (b & 7), m = (b >> 3) % tiles;
    if (unit >= a.g.ngroups * n_cb) return;
    mt = unit / n_cb * tiles + m;
    cb = unit % n_cb;
  }
  TileInfo ti = find_tile<BM>(a.g, mt, &s_info);
  if (ti.group < 0) return;
  ti.group = __builtin_amdgcn_readfirstlane(ti.group);
  ti.m0 = __builtin_amdgcn_readfirstlane(ti.m0);
  ti.rows = __builtin_amdgcn_readfirstlane(ti.rows);
  ti.row_base = __builtin_amdgcn_readfirstlane(ti.row_base);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, c = lane >> 4;
  const int unit0 = cb * NB;
  const long long matrix = __builtin_amdgcn_readfirstlane(a.g.grp_widx ? a.g.grp_widx[ti.group] : a.g.w_base + ti.group);
  const int nblk = min(MT, (ti.rows - ti.m0 + 15) / 16);   // token blocks with any valid row

  const char* xrow[MT];
#pragma unroll
  for (int tb = 0; tb < MT; ++tb) {
    int lr = ti.m0 + tb * 16 + r;
    if (lr >= ti.rows) lr = ti.rows - 1;   // rows past the group's end repeat its last one; dropped at the end
    const long long logical = ti.row_base + lr;
    const long long src = a.g.a_rows ? a.g.a_rows[logical] : logical;
    xrow[tb] = static_cast<const char*>(a.g.A) + src * a.g.lda * (F32 ? 4 : 2);
  }

  struct Stage {
    u32x4 q[NB][NW];
    unsigned s[NB][NW][G];   // bf16 scale in the high half; with zero points the bf16 of -(16 + zero) in the low one
    XFrag<F32> x[MT][kSteps];
  };
  // one K block: kb counts through the matrices that K walks
  auto load = [&](Stage& st, int kb) {
    const int mat = kb / a.kblocks, kin = kb - mat * a.kblocks;
    const long long w = matrix + mat;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int unit = min(unit0 + nb, units - 1);   // past the last unit: read it again, dropped at the end
      const long long block = ((long long)unit * a.kblocks + kin) * NW;
#pragma unroll
      for (int m = 0; m < NW; ++m) {
        st.q[nb][m] = *reinterpret_cast<const u32x4*>(a.codes + w * a.code_stride + (block + m) * kBlockBytes + lane * 16);
        const char* sp = a.scales + w * a.scale_stride + ((block + m) * kUnit + r) * (G * kScaleBytes);
#pragma unroll
        for (int i = 0; i < G; ++i) {
          if constexpr (ZERO) st.s[nb][m][i] = reinterpret_cast<const unsigned*>(sp)[i];
          else st.s[nb][m][i] = (unsigned)reinterpret_cast<const uint16_t*>(sp)[i] << 16;
        }
      }
    }
#pragma unroll
    for (int tb = 0; tb < MT; ++tb)
      if (tb < nblk) {
#pragma unroll
        for (int j = 0; j < kSteps; ++j)
          st.x[tb][j].load(xrow[tb] + (size_t)mat * a.g.kseg * (F32 ? 4 : 2), kin * kBlockK + j * 32 + c * 8, a.g.kseg);
      }
  };

  f32x4 acc[NB][NW][MT];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int m = 0; m < NW; ++m)
#pragma unroll
      for (int tb = 0; tb < MT; ++tb) acc[nb][m][tb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  const bf16x8 minus24 = splat_bf16(0xC1C0u);   // -(16 + 8)
  auto multiply = [&](const Stage& st) {
#pragma unroll
    for (int tb = 0; tb < MT; ++tb)
      if (tb < nblk) {
        bf16x8 xp[kSteps][P];
#pragma unroll
        for (int j = 0; j < kSteps; ++j) st.x[tb][j].parts(xp[j]);
#pragma unroll
        for (int gi = 0; gi < G; ++gi) {
          f32x4 start = {0.0f, 0.0f, 0.0f, 0.0f};
          if constexpr (!ZERO) {
#pragma unroll
            for (int j = gi * kGroupSteps; j < (gi + 1) * kGroupSteps; ++j)
#pragma unroll
              for (int n = 0; n < P; ++n) start = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xp[j][n], minus24, start, 0, 0, 0);
          }
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int m = 0; m < NW; ++m) {
              f32x4 part = start;
              if constexpr (ZERO) {
                const bf16x8 minus = splat_bf16(st.s[nb][m][gi]);
#pragma unroll
                for (int j = gi * kGroupSteps; j < (gi + 1) * kGroupSteps; ++j)
#pragma unroll
                  for (int n = 0; n < P; ++n) part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xp[j][n], minus, part, 0, 0, 0);
              }
#pragma unroll
              for (int j = gi * kGroupSteps; j < (gi + 1) * kGroupSteps; ++j) {
                const bf16x8 w = operand_of(st.q[nb][m][j]);
#pragma unroll
                for (int n = 0; n < P; ++n) part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xp[j][n], w, part, 0, 0, 0);
              }
              const float scale = __uint_as_float(st.s[nb][m][gi] & 0xFFFF0000u);
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[nb][m][tb][e] = fmaf(scale, part[e], acc[nb][m][tb][e]);
            }
        }
      }
  };

  const int blocks = a.kblocks * a.mats;
  const int kb_begin = blocks * wave / 4, kb_end = blocks * (wave + 1) / 4;
  if (kb_begin < kb_end) {   // wave-uniform
    Stage s0, s1;
    load(s0, kb_begin);
    for (int kb = kb_begin; kb < kb_end; kb += 2) {
      const bool more1 = kb + 1 < kb_end, more2 = kb + 2 < kb_end;   // past the end the last block is fetched again and not used
      load(s1, more1 ? kb + 1 : kb);
      multiply(s0);
      load(s0, more2 ? kb + 2 : more1 ? kb + 1 : kb);
      if (more1) multiply(s1);
    }
  }

  // the four waves' sums, added in the order of K; wave e finishes element e of every accumulator
  __shared__ float s_red[4][NB * NW * MT * 4][64];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int m = 0; m < NW; ++m)
#pragma unroll
      for (int tb = 0; tb < MT; ++tb)
#pragma unroll
        for (int e = 0; e < 4; ++e) s_red[wave][((nb * NW + m) * MT + tb) * 4 + e][lane] = acc[nb][m][tb][e];
  __syncthreads();
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int tb = 0; tb < MT; ++tb) {
      float v[NW];
#pragma unroll
      for (int m = 0; m < NW; ++m) {
        const int at = ((nb * NW + m) * MT + tb) * 4 + wave;
        v[m] = ((s_red[0][at][lane] + s_red[1][at][lane]) + s_red[2][at][lane]) + s_red[3][at][lane];
      }
      const int token = ti.m0 + tb * 16 + c * 4 + wave, col = (unit0 + nb) * kUnit + r;
      if (token < ti.rows && col < a.g.N) {
        const float y = NW == 2 ? v[0] / (1.0f + expf(-v[0])) * v[NW - 1] : v[0];
        const size_t at = (size_t)(ti.row_base + token) * a.g.ldc + group_col0(a.g, ti.group) + col;
        if constexpr (F32) static_cast<float*>(a.g.C)[at] = y;
        else static_cast<__bf16*>(a.g.C)[at] = (__bf16)y;   // rounded to nearest: the layer's type between the two products
      }
    }
}

// ---- quantisation, values, packing ----------------------------------------------------------------------------------------
template <bool BF16>
__device__ __forceinline__ float load_weight(const void* p, size_t i) {
  if constexpr (BF16) return __uint_as_float((unsigned)static_cast<const uint16_t*>(p)[i] << 16);
  else return static_cast<const float*>(p)[i];
}
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

// One thread per group.  Codes by division in double: the quotient of two floats is never so close to a rounding border that double
// would put it on the other side.
template <bool BF16>
__global__ __launch_bounds__(256) void quantize_kernel(const void* w, long long rows, int K, int group, uint8_t* codes, uint16_t* scales,
                                                       uint8_t* zeros) {
  const int groups = (K + group - 1) / group;
  const long long n = rows * groups;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
    const long long row = i / groups;
    const int k0 = (int)(i - row * groups) * group, k1 = min(K, k0 + group);
    const size_t base = (size_t)row * K;
    float lo = 0.0f, hi = 0.0f;
    for (int k = k0; k < k1; ++k) {
      const float v = load_weight<BF16>(w, base + k);
      lo = fminf(lo, v);
      hi = fmaxf(hi, v);
    }
    const double span = zeros ? ((double)hi - (double)lo) / 15.0 : (double)fmaxf(hi, -lo) / 7.0;
    const uint16_t sb = bf16_of(span);
    const double s = (double)bf16_value(sb);
    int z = 8;
    if (zeros) {
      z = s > 0.0 ? (int)fmin(fmax(rint(-(double)lo / s), 0.0), 15.0) : 8;
      zeros[i] = (uint8_t)z;
    }
    scales[i] = sb;
    for (int k = k0; k < k1; k += 2) {
      int q[2];
      for (int e = 0; e < 2; ++e) {
        const double t = s > 0.0 ? rint((double)load_weight<BF16>(w, base + k + e) / s) + z : (double)z;
        q[e] = (int)fmin(fmax(t, 0.0), 15.0);
      }
      codes[(base + k) / 2] = (uint8_t)(q[0] | q[1] << 4);
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
    const float z = zeros ? (float)zeros[g] : 8.0f;
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

template <int MT, int NB, int NW, bool F32>
static int launch_typed(const Args& a, const Args* b, int group, bool zeros, int total_rows, hipStream_t s) {
  constexpr int BM = 16 * MT;
  const int n_cb = ((a.g.N + kUnit - 1) / kUnit + NB - 1) / NB;
  // row tiles of the grouped rows: at most one partly filled one per group, and none without a row
  long long m_tiles = ((long long)total_rows + (long long)a.g.ngroups * (BM - 1)) / BM;
  if (m_tiles > total_rows) m_tiles = total_rows;
  const long long a_blocks = m_tiles * n_cb;
  long long grid = a_blocks;
  if (b) grid += (b->g.ngroups * (long long)n_cb + 7) / 8 * 8 * ((b->g.M + BM - 1) / BM);
  if (grid == 0) return OCCULT_OK;
  OCC_REQUIRE(grid < (1ll << 24), OCCULT_ESHAPE, "%lld workgroups are too many for one launch", grid);
  const Args& second = b ? *b : a;
#define OCC_W4_CASE(G_, Z_)                                                                                                \
  if (group == kBlockK / G_ && zeros == Z_) {                                                                              \
    w4_gemm<MT, NB, NW, G_, Z_, F32><<<(int)grid, 256, 0, s>>>(a, second, (int)a_blocks);                                  \
    OCC_LAUNCH_CHECK("w4_gemm");                                                                                           \
    return OCCULT_OK;                                                                                                      \
  }
  OCC_W4_CASE(1, false)
  OCC_W4_CASE(2, false)
  OCC_W4_CASE(4, false)
  OCC_W4_CASE(1, true)
  OCC_W4_CASE(2, true)
  OCC_W4_CASE(4, true)
#undef OCC_W4_CASE
  OCC_FAIL(OCCULT_EINVAL, "group=%d", group);
}

// a: the routed experts' grouped rows; b: the shared experts', or NULL
template <int NW>
static int launch(const occult_cfg_t& c, const Args& a, const Args* b, int group, bool zeros, hipStream_t s) {
  const int rows = c.T * c.k;
  if (c.dtype == OCCULT_F32) return launch_typed<1, 2, NW, true>(a, b, group, zeros, rows, s);
  if (rows <= 8ll * c.E) return launch_typed<1, 2, NW, false>(a, b, group, zeros, rows, s);
  return launch_typed<2, 2, NW, false>(a, b, group, zeros, rows, s);
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
    const int grid = grid_for(rows * ((K + out->group - 1) / out->group));
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
