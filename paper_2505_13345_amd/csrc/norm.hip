// occult_block_norm and its backward pass: the norms around a block, fused with its gate, its residual scale and the residual sum.
//
//   forward   out = x_scale * x + y_scale * gate * N_post(y);   h = N_pre(out)
//   backward  D = dout + N_pre'(dh);   dx = x_scale * D;   dz = y_scale * gate * D;   dy = N_post'(dz);   dgate = y_scale * z * D
//   (without y, the pre norm alone: h = N_pre(x), dx = D)
//   with N(v) = vh * w + b, vh = (v - mu) * r, r = 1 / sqrt(mean((v - mu)^2) + eps), mu = 0 (RMS) or mean(v) (LAYER), and
//   N'(g) = r * (q - vh * mean(q * vh) - [LAYER] mean(q)), q = g * w.
//
// Bound by HBM: a handful of operations per element.  Every row is read once and written once: the lanes that share a row keep it in
// registers from the first sum to the last store, so the row statistics cost no second read, and the backward pass
// recomputes them from the rows that it reads anyway instead of reading kept ones.  A row of up to 64 vectors of 16 bytes
// belongs to the smallest power of two of lanes that holds it (a wave then works on several rows).  Longer rows, forward: two vectors
// per lane, on one wave and beyond that on 2, 4, 8 or 16, which exchange their sums through LDS; backward, where the column sums
// take registers: one vector per lane on 2, 3, 4, 5 or 8 waves, then two and four vectors on eight.  All sums are f32; which
// lanes add what depends on the row length alone, so a token's results do not depend on the batch around it.
#include "common.h"

#include <math.h>

#include <type_traits>

namespace occult {

namespace norm {

constexpr int kMaxRowBytes = 32768;
constexpr int kColSums = 5;          // post weight, post bias, pre weight, pre bias, channel gate
constexpr int kBackwardBlocks = 256; // workgroups of the backward pass that keep column sums, at most

struct Args {
  const void *x, *y, *gate, *post_w, *post_b, *pre_w, *pre_b;
  void *out, *h;
  int T, row_vecs, lanes;            // lanes: lanes of a row where a wave holds several rows
  int post, pre, gate_kind;
  float x_scale, y_scale, post_eps, pre_eps, offset, inv_d;
};

struct BackwardArgs {
  const void *y, *out, *dout, *dh, *gate, *post_w, *post_b, *pre_w;
  void *dx, *dy, *dgate;             // dgate: per token (f32) or per element (rows); a channel gate's goes through ws
  float* ws;                         // [workgroup][column sum][d]
  int T, row_vecs, lanes;
  int post, pre, gate_kind, sums;    // sums: bit i = column sum i is wanted
  float x_scale, y_scale, post_eps, pre_eps, offset, inv_d;
};

// Waves of a workgroup, a multiple of those of a row: at least 4 in the forward pass, about 8 in the backward pass, whose workgroups each
// leave a set of column sums.
constexpr int block_waves(int W, bool backward) {
  return backward ? (W == 3 ? 9 : W == 5 ? 10 : 8) : W <= 4 ? 4 : W;
}

// Which lanes hold which rows.  V vectors per lane, W waves per row.
template <int V, int W, bool BACKWARD>
struct Place {
  static constexpr int kWaves = block_waves(W, BACKWARD);
  int row, lane, stride;             // row inside the workgroup, lane inside the row, lanes of the row
  __device__ Place(int lanes) {
    const int wave = threadIdx.x >> 6, l = threadIdx.x & 63;
    if constexpr (W == 1) {
      row = wave * (64 / lanes) + l / lanes;
      lane = l & (lanes - 1);
      stride = lanes;
    } else {
      row = wave / W;
      lane = (wave % W) * 64 + l;
      stride = 64 * W;
    }
  }
  __device__ static int rows_per_block(int lanes) { return W == 1 ? kWaves * (64 / lanes) : kWaves / W; }
};

// Sum over aligned groups of `lanes` lanes (a power of two), in each of them.  Inside 16 lanes by DPP operands (neighbours, pairs, then
// mirrored halves and rows, whose partners hold the sum of the other half), beyond them from a row's lane; a lane exchange
// through LDS takes longer than all four additions.
__device__ __forceinline__ float group_sum(float v, int lanes) {
  auto add = [&](auto ctrl) {
    const int o = __builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, true);
    v += __int_as_float(o);
  };
  if (lanes >= 2) add(std::integral_constant<int, 0xB1>{});    // quad_perm [1,0,3,2]
  if (lanes >= 4) add(std::integral_constant<int, 0x4E>{});    // quad_perm [2,3,0,1]
  if (lanes >= 8) add(std::integral_constant<int, 0x141>{});   // row_half_mirror
  if (lanes >= 16) add(std::integral_constant<int, 0x140>{});  // row_mirror
  if (lanes == 32) v += __shfl_xor(v, 16, 64);
  if (lanes == 64) {
    const auto row = [&](int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l)); };
    v = (row(0) + row(16)) + (row(32) + row(48));
  }
  return v;
}

// The sums of N values over the lanes of a row, in every lane.  `slot`: alternates between two LDS areas, so that one barrier per
// exchange is enough.
template <int W, int WAVES, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], int lanes, int& slot) {
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = group_sum(v[n], W > 1 ? 64 : lanes);
  if constexpr (W > 1) {
    __shared__ float s_sum[2][N][WAVES];
    const int wave = threadIdx.x >> 6, first = wave / W * W;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int n = 0; n < N; ++n) s_sum[slot][n][wave] = v[n];
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float s = s_sum[slot][n][first];
#pragma unroll
      for (int w = 1; w < W; ++w) s += s_sum[slot][n][first + w];
      v[n] = s;
    }
    slot ^= 1;
  }
}

// A lane's vectors of a row as loaded; vectors past the row's end are zero.
template <bool BF16, int V>
struct RowRegs {
  using R = Row<BF16>;
  typename R::Raw raw[V];
  __device__ void load(const void* base, size_t t, int row_vecs, int lane, int stride, bool valid) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = lane + i * stride;
      raw[i] = typename R::Raw{};
      if (valid && c < row_vecs) raw[i] = R::load_raw(base, t, row_vecs, c);
    }
  }
  // one value per channel, read by every workgroup: kept in the caches
  __device__ void load_channels(const void* base, int row_vecs, int lane, int stride) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = lane + i * stride;
      raw[i] = typename R::Raw{};
      if (base && c < row_vecs) raw[i] = static_cast<const typename R::Raw*>(base)[c];
    }
  }
  // Makes the compiler take the values for new ones: what is kept across rows stays as loaded, in half the registers of its floats.
  __device__ void keep_raw() {
#pragma unroll
    for (int i = 0; i < V; ++i) asm volatile("" : "+v"(raw[i]));
  }
  __device__ void unpack(int i, float* v) const { R::unpack(raw[i], v); }
};

template <bool BF16>
__device__ __forceinline__ float load_scalar(const void* base, size_t t) {
  if constexpr (BF16) return __uint_as_float((unsigned)static_cast<const uint16_t*>(base)[t] << 16);
  else return static_cast<const float*>(base)[t];
}

// factor of a norm's weight: 1 where there is none
template <int NE>
__device__ __forceinline__ void weight_of(bool has, float offset, float* w) {
#pragma unroll
  for (int e = 0; e < NE; ++e) w[e] = has ? w[e] + offset : 1.0f;
}

template <bool BF16, int V, int W>
__global__ __launch_bounds__(64 * block_waves(W, false)) void block_norm_kernel(const Args a) {
  using R = Row<BF16>;
  constexpr int NE = R::kElems;
  typedef Place<V, W, false> P;
  const P p(a.lanes);
  const int rows = P::rows_per_block(a.lanes);
  int slot = 0;

  RowRegs<BF16, V> post_w, post_b, pre_w, pre_b, cgate;
  post_w.load_channels(a.post_w, a.row_vecs, p.lane, p.stride);
  post_b.load_channels(a.post_b, a.row_vecs, p.lane, p.stride);
  pre_w.load_channels(a.pre_w, a.row_vecs, p.lane, p.stride);
  pre_b.load_channels(a.pre_b, a.row_vecs, p.lane, p.stride);
  cgate.load_channels(a.gate_kind == OCCULT_GATE_CHANNEL ? a.gate : nullptr, a.row_vecs, p.lane, p.stride);

  // one pass = one row per group of lanes; uniform over the workgroup, which meets in row_sums
  for (long long t0 = (long long)blockIdx.x * rows; t0 < a.T; t0 += (long long)gridDim.x * rows) {
    const bool valid = t0 + p.row < a.T;
    const size_t t = valid ? t0 + p.row : 0;
    post_w.keep_raw();
    post_b.keep_raw();
    pre_w.keep_raw();
    pre_b.keep_raw();
    cgate.keep_raw();
    RowRegs<BF16, V> xr, yr;
    xr.load(a.x, t, a.row_vecs, p.lane, p.stride, valid);
    float s[V][NE];   // the residual stream
#pragma unroll
    for (int i = 0; i < V; ++i) xr.unpack(i, s[i]);
    if (a.y) {
      yr.load(a.y, t, a.row_vecs, p.lane, p.stride, valid);
      RowRegs<BF16, V> gr;
      if (a.gate_kind == OCCULT_GATE_ELEMENT) gr.load(a.gate, t, a.row_vecs, p.lane, p.stride, valid);
      float token_gate = 1.0f;
      if (a.gate_kind == OCCULT_GATE_TOKEN) token_gate = load_scalar<BF16>(a.gate, t);
      float z[V][NE];
#pragma unroll
      for (int i = 0; i < V; ++i) yr.unpack(i, z[i]);
      if (a.post) {
        float mu = 0.0f;
        if (a.post == OCCULT_NORM_LAYER) {
          float sum[1] = {0.0f};
#pragma unroll
          for (int i = 0; i < V; ++i)
#pragma unroll
            for (int e = 0; e < NE; ++e) sum[0] += z[i][e];
          row_sums<W, P::kWaves>(sum, a.lanes, slot);
          mu = sum[0] * a.inv_d;
        }
        float sq[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const bool in = p.lane + i * p.stride < a.row_vecs;
#pragma unroll
          for (int e = 0; e < NE; ++e) {
            z[i][e] = in ? z[i][e] - mu : 0.0f;
            sq[0] = fmaf(z[i][e], z[i][e], sq[0]);
          }
        }
        row_sums<W, P::kWaves>(sq, a.lanes, slot);
        const float r = 1.0f / sqrtf(fmaf(sq[0], a.inv_d, a.post_eps));
#pragma unroll
        for (int i = 0; i < V; ++i) {
          float w[NE], b[NE];
          post_w.unpack(i, w);
          post_b.unpack(i, b);
          weight_of<NE>(a.post_w != nullptr, a.offset, w);
#pragma unroll
          for (int e = 0; e < NE; ++e) z[i][e] = fmaf(z[i][e] * r, w[e], b[e]);
        }
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int c = p.lane + i * p.stride;
        float g[NE];
        if (a.gate_kind == OCCULT_GATE_CHANNEL) cgate.unpack(i, g);
        else if (a.gate_kind == OCCULT_GATE_ELEMENT) gr.unpack(i, g);
        else
#pragma unroll
          for (int e = 0; e < NE; ++e) g[e] = token_gate;
#pragma unroll
        for (int e = 0; e < NE; ++e) s[i][e] = fmaf(a.y_scale * g[e], z[i][e], a.x_scale * s[i][e]);
        // rounds s to what is stored: the next norm is taken of the values that the backward pass, and the next block, will read
        if (valid && c < a.row_vecs) R::store_round(a.out, t, a.row_vecs, c, s[i]);
      }
    }
    if (a.pre) {
      float mu = 0.0f;
      if (a.pre == OCCULT_NORM_LAYER) {
        float sum[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const bool in = p.lane + i * p.stride < a.row_vecs;
#pragma unroll
          for (int e = 0; e < NE; ++e) sum[0] += in ? s[i][e] : 0.0f;
        }
        row_sums<W, P::kWaves>(sum, a.lanes, slot);
        mu = sum[0] * a.inv_d;
      }
      float sq[1] = {0.0f};
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const bool in = p.lane + i * p.stride < a.row_vecs;
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          s[i][e] = in ? s[i][e] - mu : 0.0f;
          sq[0] = fmaf(s[i][e], s[i][e], sq[0]);
        }
      }
      row_sums<W, P::kWaves>(sq, a.lanes, slot);
      const float r = 1.0f / sqrtf(fmaf(sq[0], a.inv_d, a.pre_eps));
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int c = p.lane + i * p.stride;
        float w[NE], b[NE];
        pre_w.unpack(i, w);
        pre_b.unpack(i, b);
        weight_of<NE>(a.pre_w != nullptr, a.offset, w);
#pragma unroll
        for (int e = 0; e < NE; ++e) s[i][e] = fmaf(s[i][e] * r, w[e], b[e]);
        if (valid && c < a.row_vecs) R::store_round(a.h, t, a.row_vecs, c, s[i]);
      }
    }
  }
}

// Gradients of what is summed over tokens (weights, biases, a channel gate): every lane adds its columns' contributions over the rows of
// its workgroup in registers, the workgroup's row groups are added through LDS in their order, and the workgroups' sums go to ws, where
// column_sums_kernel adds them in order: no atomics, the same bits every time.
template <bool BF16, int V, int W, bool LAYER>
__global__ __launch_bounds__(64 * block_waves(W, true)) void block_norm_backward_kernel(const BackwardArgs a) {
  using R = Row<BF16>;
  constexpr int NE = R::kElems;
  // without a mean-subtracting norm or a bias there are three column sums: weights and gate
  constexpr int NS = LAYER ? kColSums : 3;
  constexpr int kPostW = 0, kPreW = 1, kGate = 2, kPostB = LAYER ? 3 : 0, kPreB = LAYER ? 4 : 0;
  typedef Place<V, W, true> P;
  const P p(a.lanes);
  const int rows = P::rows_per_block(a.lanes);
  int slot = 0;

  // With four vectors per lane, or two of bf16 and five column sums, the parameters are read again for every row (from L2) and no row is
  // requested ahead: kept in registers both would spill (2195 rows of 7640 f32: 298 us, so 76; 2048 of 5000 bf16 69.6, so 61.8).
  constexpr bool kTight = V == 4 || (V == 2 && LAYER && BF16);
  RowRegs<BF16, V> post_w, post_b, pre_w, cgate;
  const void* const gate_channels = a.gate_kind == OCCULT_GATE_CHANNEL ? a.gate : nullptr;
  if constexpr (!kTight) {
    post_w.load_channels(a.post_w, a.row_vecs, p.lane, p.stride);
    post_b.load_channels(a.post_b, a.row_vecs, p.lane, p.stride);
    pre_w.load_channels(a.pre_w, a.row_vecs, p.lane, p.stride);
    cgate.load_channels(gate_channels, a.row_vecs, p.lane, p.stride);
  }
  // (loads and their unpacked values stay inside a phase of a row)
  auto phase = [&]() {
    if constexpr (kTight) asm volatile("" ::: "memory");
  };
  auto channels = [&](const RowRegs<BF16, V>& kept, const void* base, int i, float* v) {
    if constexpr (kTight) {
      const int c = p.lane + i * p.stride;
      typename R::Raw raw{};
      if (base && c < a.row_vecs) raw = static_cast<const typename R::Raw*>(base)[c];
      R::unpack(raw, v);
    } else {
      kept.unpack(i, v);
    }
  };
  const bool need_y = a.dy && (a.post || a.gate_kind);

  float col[NS][V][NE];
#pragma unroll
  for (int n = 0; n < NS; ++n)
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int e = 0; e < NE; ++e) col[n][i][e] = 0.0f;

  struct Rows {
    RowRegs<BF16, V> y, out, dout, dh, gate;
    float token_gate;
  };
  auto load = [&](Rows& r, long long t0) {
    const bool valid = t0 + p.row < a.T;
    const size_t t = valid ? t0 + p.row : 0;
    r.dout.load(a.dout, t, a.row_vecs, p.lane, p.stride, valid && a.dout);
    r.out.load(a.out, t, a.row_vecs, p.lane, p.stride, valid && a.pre);
    r.dh.load(a.dh, t, a.row_vecs, p.lane, p.stride, valid && a.pre);
    r.y.load(a.y, t, a.row_vecs, p.lane, p.stride, valid && need_y);
    r.gate.load(a.gate, t, a.row_vecs, p.lane, p.stride, valid && a.gate_kind == OCCULT_GATE_ELEMENT);
    r.token_gate = 1.0f;   // also where there is no token: 0 * another one's infinity would go into the column sums
    if (a.gate_kind == OCCULT_GATE_TOKEN && valid) r.token_gate = load_scalar<BF16>(a.gate, t);
  };
  const long long step = (long long)gridDim.x * rows;
  Rows next;
  if constexpr (!kTight) load(next, (long long)blockIdx.x * rows);
  for (long long t0 = (long long)blockIdx.x * rows; t0 < a.T; t0 += step) {
    const bool valid = t0 + p.row < a.T;
    const size_t t = valid ? t0 + p.row : 0;
    if constexpr (kTight) {
      load(next, t0);
    } else {
      post_w.keep_raw();
      post_b.keep_raw();
      pre_w.keep_raw();
      cgate.keep_raw();
    }
    const Rows cur = next;
    // requested before this pass's sums, whose exchanges would otherwise leave memory idle
    if (!kTight && t0 + step < a.T) load(next, t0 + step);
    const RowRegs<BF16, V>&yr = cur.y, &outr = cur.out, &doutr = cur.dout, &dhr = cur.dh, &gr = cur.gate;
    const float token_gate = cur.token_gate;

    float D[V][NE], o[V][NE], y[V][NE];   // gradient of the stream, the stream and y (less their means)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      doutr.unpack(i, D[i]);
      outr.unpack(i, o[i]);
      yr.unpack(i, y[i]);
    }
    if constexpr (LAYER) {
      float mean[2] = {0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          mean[0] += o[i][e];
          mean[1] += y[i][e];
        }
      row_sums<W, P::kWaves>(mean, a.lanes, slot);
      const float mo = a.pre == OCCULT_NORM_LAYER ? mean[0] * a.inv_d : 0.0f;
      const float my = a.post == OCCULT_NORM_LAYER ? mean[1] * a.inv_d : 0.0f;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const bool in = p.lane + i * p.stride < a.row_vecs;
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          o[i][e] = in ? o[i][e] - mo : 0.0f;
          y[i][e] = in ? y[i][e] - my : 0.0f;
        }
      }
    }
    // squares of both rows, and the two sums of the pre norm's gradient, in one exchange
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float w[NE], g[NE];
      channels(pre_w, a.pre_w, i, w);
      dhr.unpack(i, g);
      weight_of<NE>(a.pre_w != nullptr, a.offset, w);
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        s[0] = fmaf(o[i][e], o[i][e], s[0]);
        s[1] = fmaf(y[i][e], y[i][e], s[1]);
        s[2] = fmaf(g[e] * w[e], o[i][e], s[2]);
        if (LAYER) s[3] = fmaf(g[e], w[e], s[3]);
      }
    }
    row_sums<W, P::kWaves>(s, a.lanes, slot);
    phase();
    if (a.pre) {
      const float r = 1.0f / sqrtf(fmaf(s[0], a.inv_d, a.pre_eps));
      const float m2 = s[2] * r * a.inv_d, m1 = LAYER && a.pre == OCCULT_NORM_LAYER ? s[3] * a.inv_d : 0.0f;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float w[NE], g[NE];
        channels(pre_w, a.pre_w, i, w);
        dhr.unpack(i, g);
        weight_of<NE>(a.pre_w != nullptr, a.offset, w);
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          const float hat = o[i][e] * r;
          D[i][e] = fmaf(r, fmaf(-hat, m2, fmaf(g[e], w[e], -m1)), D[i][e]);
          col[kPreW][i][e] = fmaf(g[e], hat, col[kPreW][i][e]);
          if constexpr (LAYER) col[kPreB][i][e] += g[e];
        }
      }
    }
    phase();
    if (a.dx) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int c = p.lane + i * p.stride;
        float v[NE];
#pragma unroll
        for (int e = 0; e < NE; ++e) v[e] = a.x_scale * D[i][e];
        if (valid && c < a.row_vecs) R::store_round(a.dx, t, a.row_vecs, c, v);
      }
    }
    if (!a.dy) continue;   // uniform over the grid
    phase();
    const float r = a.post ? 1.0f / sqrtf(fmaf(s[1], a.inv_d, a.post_eps)) : 1.0f;
    // D becomes q = dz * w, the gradient of the normalised row; sums of the post norm's gradient and of a token's gate
    float u[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = p.lane + i * p.stride;
      const bool in = c < a.row_vecs;
      float w[NE], b[NE], g[NE], dg[NE];
      channels(post_w, a.post_w, i, w);
      channels(post_b, a.post_b, i, b);
      weight_of<NE>(a.post_w != nullptr, a.offset, w);
      if (a.gate_kind == OCCULT_GATE_CHANNEL) channels(cgate, gate_channels, i, g);
      else if (a.gate_kind == OCCULT_GATE_ELEMENT) gr.unpack(i, g);
      else
#pragma unroll
        for (int e = 0; e < NE; ++e) g[e] = token_gate;
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        const float hat = y[i][e] * r, sD = in ? a.y_scale * D[i][e] : 0.0f;
        dg[e] = fmaf(hat, w[e], b[e]) * sD;
        const float dz = g[e] * sD;
        col[kPostW][i][e] = fmaf(dz, hat, col[kPostW][i][e]);
        if constexpr (LAYER) col[kPostB][i][e] += dz;
        D[i][e] = dz * w[e];
        u[0] = fmaf(D[i][e], hat, u[0]);
        u[1] += D[i][e];
        u[2] += dg[e];
        col[kGate][i][e] += dg[e];
      }
      if (a.gate_kind == OCCULT_GATE_ELEMENT && a.dgate && valid && in) R::store_round(a.dgate, t, a.row_vecs, c, dg);
    }
    if (a.post || a.gate_kind == OCCULT_GATE_TOKEN) row_sums<W, P::kWaves>(u, a.lanes, slot);
    if (a.gate_kind == OCCULT_GATE_TOKEN && a.dgate && valid && p.lane == 0) static_cast<float*>(a.dgate)[t] = u[2];
    phase();
    const float m2 = u[0] * a.inv_d, m1 = LAYER && a.post == OCCULT_NORM_LAYER ? u[1] * a.inv_d : 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = p.lane + i * p.stride;
      float v[NE];
#pragma unroll
      for (int e = 0; e < NE; ++e)   // without a post norm no value of y is in it: 0 * y is not 0 for an infinity or NaN
        v[e] = a.post ? r * (D[i][e] - m1 - y[i][e] * r * m2) : D[i][e];
      if (valid && c < a.row_vecs) R::store_round(a.dy, t, a.row_vecs, c, v);
    }
  }

  if (!a.sums) return;
  // A wave's row groups are added across its lanes, then the workgroup's waves (W == 1) or rows through LDS in their order.
  constexpr int kGroups = W == 1 ? P::kWaves : P::kWaves / W;
  const int wave = threadIdx.x >> 6, group = W == 1 ? wave : p.row;
  const bool leads = W > 1 || (int)(threadIdx.x & 63) < a.lanes;   // one of its wave's row groups
  __shared__ float s_col[kGroups > 1 ? P::kWaves * 64 * V * NE : 1];
  const int d = a.row_vecs * NE;
  float* ws = a.ws + (size_t)blockIdx.x * __popc(a.sums) * d;
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    // bits of `sums`: post weight, post bias, pre weight, pre bias, channel gate
    constexpr int kBit[kColSums] = {0, 2, 4, 1, 3};
    if (!(a.sums >> kBit[n] & 1)) continue;   // uniform
    if constexpr (W == 1) {
      for (int o = a.lanes; o < 64; o <<= 1)
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
          for (int e = 0; e < NE; ++e) col[n][i][e] += __shfl_xor(col[n][i][e], o, 64);
    }
    if constexpr (kGroups > 1) {
      __syncthreads();
      if (group > 0 && leads) {
        float* mine = s_col + (group * p.stride + p.lane) * V * NE;
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
          for (int e = 0; e < NE; ++e) mine[i * NE + e] = col[n][i][e];
      }
      __syncthreads();
    }
    if (group == 0 && leads) {
      float* dst = ws + (size_t)__popc(a.sums & ((1 << kBit[n]) - 1)) * d;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int c = p.lane + i * p.stride;
#pragma unroll
        for (int g = 1; g < kGroups; ++g)
#pragma unroll
          for (int e = 0; e < NE; ++e) col[n][i][e] += s_col[(g * p.stride + p.lane) * V * NE + i * NE + e];
        if (c < a.row_vecs)
#pragma unroll
          for (int e = 0; e < NE; ++e) dst[c * NE + e] = col[n][i][e];
      }
    }
  }
}

struct ColumnArgs {
  const float* ws;
  float* dst[kColSums];
  int blocks, nsums, d, accumulate;
};

// 64 columns per workgroup, 16 slices of the workgroups' sums, added in order
__global__ __launch_bounds__(1024) void column_sums_kernel(const ColumnArgs a) {
  __shared__ float s_part[16][64];
  const int lane = threadIdx.x & 63, slice = threadIdx.x >> 6;
  const long long n = (long long)a.nsums * a.d, col = (long long)blockIdx.x * 64 + lane;
  const int lo = (int)((long long)a.blocks * slice / 16), hi = (int)((long long)a.blocks * (slice + 1) / 16);
  float sum = 0.0f;
  if (col < n) {
#pragma unroll 8
    for (int b = lo; b < hi; ++b) sum += a.ws[(size_t)b * n + col];
  }
  s_part[slice][lane] = sum;
  __syncthreads();
  if (slice == 0 && col < n) {
#pragma unroll
    for (int i = 1; i < 16; ++i) sum += s_part[i][lane];
    const int which = (int)(col / a.d), c = (int)(col % a.d);
    float* dst = a.dst[0];
#pragma unroll
    for (int i = 1; i < kColSums; ++i)
      if (which == i) dst = a.dst[i];
    dst[c] = a.accumulate ? dst[c] + sum : sum;
  }
}

// Vectors per lane, waves per row and lanes per row of a row length: V and W of the kernels above.  Forward: two vectors per lane before a
// second wave (16384 rows of 2048 bf16: 47 us, with one 51, with four 51; one row 3.3, 2.8, 4.6).  Backward: one vector per lane up to eight
// waves (the column sums take registers: 1000 rows of 2048 12.8 us, with two 15.8; 16384 rows the same 76, with
// means and biases 92 against 126), then two and four (sixteen waves of two leave 128 registers: 2195 rows of 7640 f32 134 us, eight
// of four 75; 2048 rows of 16384 bf16 299 and 208, both of which spill, as do means and biases there: 320).
struct Shape {
  int V, W, lanes;
};
static Shape shape_of(int row_vecs, bool backward) {
  Shape s{1, 1, 64};
  if (row_vecs <= 64) {
    while (s.lanes > 1 && s.lanes / 2 >= row_vecs) s.lanes /= 2;
    return s;
  }
  s.V = !backward ? 2 : row_vecs <= 512 ? 1 : row_vecs <= 1024 ? 2 : 4;
  while (64 * s.V * s.W < row_vecs) s.W *= 2;   // rows up to kMaxRowBytes: 16 waves of 2, 8 of 4
  // Powers of two alone leave up to half of a row's lanes idle: backward 16384 rows of 1032 bf16 92 us, on three waves 81; 12000 of 2056
  // 104, on five 72; six gain nothing (3000: 107 and 109), and forward three lose (60000 rows of 2056 241 us, 303).
  if (backward && s.V == 1 && s.W == 4 && row_vecs <= 192) s.W = 3;
  if (backward && s.V == 1 && s.W == 8 && row_vecs <= 320) s.W = 5;
  return s;
}
static int rows_per_block(const Shape& s, bool backward) {
  const int waves = block_waves(s.W, backward);
  return s.W == 1 ? waves * (64 / s.lanes) : waves / s.W;
}

static int backward_blocks(const occult_cfg_t& c) {
  const int rows = rows_per_block(shape_of(c.d * elem_size(c) / 16, true), true);
  const long long need = ((long long)c.T + rows - 1) / rows;
  return need < kBackwardBlocks ? (int)need : kBackwardBlocks;
}

static int check(const occult_cfg_t* cfg, const occult_block_norm_t* n) {
  int rc = check_cfg(cfg);
  if (rc) return rc;
  OCC_REQUIRE(n, OCCULT_ENULLPTR, "norm description is NULL");
  const occult_cfg_t& c = *cfg;
  const size_t row = (size_t)c.d * elem_size(c);
  OCC_REQUIRE(row % 16 == 0, OCCULT_EALIGN, "rows of d=%d elements are not multiples of 16 bytes", c.d);
  OCC_REQUIRE(row <= (size_t)kMaxRowBytes, OCCULT_ESHAPE, "rows of %zu bytes are longer than %d", row, kMaxRowBytes);
  OCC_REQUIRE(n->post_kind >= OCCULT_NORM_NONE && n->post_kind <= OCCULT_NORM_LAYER && n->pre_kind >= OCCULT_NORM_NONE &&
                  n->pre_kind <= OCCULT_NORM_LAYER,
              OCCULT_EINVAL, "unknown norm (post %d, pre %d)", n->post_kind, n->pre_kind);
  OCC_REQUIRE(n->gate_kind >= OCCULT_GATE_NONE && n->gate_kind <= OCCULT_GATE_ELEMENT, OCCULT_EINVAL, "unknown gate %d",
              n->gate_kind);
  OCC_REQUIRE(isfinite(n->x_scale) && isfinite(n->y_scale) && isfinite(n->weight_offset), OCCULT_EINVAL,
              "x_scale, y_scale or weight_offset is not finite");
  if (n->post_kind)
    OCC_REQUIRE(isfinite(n->post_eps) && n->post_eps > 0.0f, OCCULT_EINVAL, "post_eps=%g must be positive", (double)n->post_eps);
  else
    OCC_REQUIRE(!n->post_weight && !n->post_bias, OCCULT_EINVAL, "post_weight or post_bias without a post norm");
  if (n->pre_kind)
    OCC_REQUIRE(isfinite(n->pre_eps) && n->pre_eps > 0.0f, OCCULT_EINVAL, "pre_eps=%g must be positive", (double)n->pre_eps);
  else
    OCC_REQUIRE(!n->pre_weight && !n->pre_bias, OCCULT_EINVAL, "pre_weight or pre_bias without a pre norm");
  OCC_REQUIRE((n->gate != nullptr) == (n->gate_kind != OCCULT_GATE_NONE) || c.T == 0, OCCULT_ENULLPTR,
              "gate and gate_kind=%d do not belong together", n->gate_kind);
  OCC_REQUIRE(aligned16(n->post_weight) && aligned16(n->post_bias) && aligned16(n->pre_weight) && aligned16(n->pre_bias) &&
                  (n->gate_kind == OCCULT_GATE_TOKEN ? (uintptr_t)n->gate % elem_size(c) == 0 : aligned16(n->gate)),
              OCCULT_EALIGN, "a parameter is not 16-byte aligned");
  return OCCULT_OK;
}

// column sums of a description, as bits: post weight, post bias, pre weight, pre bias, channel gate
static int wanted_sums(const occult_block_norm_t& n) {
  return (n.post_weight ? 1 : 0) | (n.post_bias ? 2 : 0) | (n.pre_weight ? 4 : 0) | (n.pre_bias ? 8 : 0) |
         (n.gate_kind == OCCULT_GATE_CHANNEL ? 16 : 0);
}

static int popcount(int v) { return __builtin_popcount((unsigned)v); }

template <bool BF16>
static int launch_forward(const Args& a, const Shape& s, hipStream_t stream) {
  const int rows = rows_per_block(s, false);
  const long long need = ((long long)a.T + rows - 1) / rows;
  const int grid = need < 4096 ? (int)need : 4096;
#define OCC_NORM_CASE(V_, W_)                                                                             \
  if (s.V == V_ && s.W == W_) {                                                                           \
    block_norm_kernel<BF16, V_, W_><<<grid, 64 * block_waves(W_, false), 0, stream>>>(a);                 \
    OCC_LAUNCH_CHECK("block_norm_kernel");                                                                \
    return OCCULT_OK;                                                                                     \
  }
  OCC_NORM_CASE(1, 1)
  OCC_NORM_CASE(2, 1)
  OCC_NORM_CASE(2, 2)
  OCC_NORM_CASE(2, 4)
  OCC_NORM_CASE(2, 8)
  OCC_NORM_CASE(2, 16)
#undef OCC_NORM_CASE
  OCC_FAIL(OCCULT_ESHAPE, "no kernel for rows of %d vectors", a.row_vecs);
}

template <bool BF16, bool LAYER>
static int launch_backward(const BackwardArgs& a, const Shape& s, int grid, hipStream_t stream) {
#define OCC_NORM_CASE(V_, W_)                                                                             \
  if (s.V == V_ && s.W == W_) {                                                                           \
    block_norm_backward_kernel<BF16, V_, W_, LAYER><<<grid, 64 * block_waves(W_, true), 0, stream>>>(a);  \
    OCC_LAUNCH_CHECK("block_norm_backward_kernel");                                                       \
    return OCCULT_OK;                                                                                     \
  }
  OCC_NORM_CASE(1, 1)
  OCC_NORM_CASE(1, 2)
  OCC_NORM_CASE(1, 3)
  OCC_NORM_CASE(1, 4)
  OCC_NORM_CASE(1, 5)
  OCC_NORM_CASE(1, 8)
  OCC_NORM_CASE(2, 8)
  OCC_NORM_CASE(4, 8)
#undef OCC_NORM_CASE
  OCC_FAIL(OCCULT_ESHAPE, "no kernel for rows of %d vectors", a.row_vecs);
}

}  // namespace norm

}  // namespace occult

using namespace occult;
using namespace occult::norm;

extern "C" int occult_block_norm(const occult_cfg_t* cfg, const occult_block_norm_t* n, const void* x, const void* y, void* out,
                                 void* h, occult_stream_t stream) {
  int rc = check(cfg, n);
  if (rc) return rc;
  const occult_cfg_t& c = *cfg;
  if (y == nullptr && c.T > 0)
    OCC_REQUIRE(n->post_kind == OCCULT_NORM_NONE && n->gate_kind == OCCULT_GATE_NONE && n->pre_kind != OCCULT_NORM_NONE,
                OCCULT_EINVAL, "without y there is nothing but a pre norm to do");
  if (c.T == 0) return OCCULT_OK;
  OCC_REQUIRE(x, OCCULT_ENULLPTR, "x is NULL");
  OCC_REQUIRE(!y || out, OCCULT_ENULLPTR, "out is NULL");
  OCC_REQUIRE(!n->pre_kind || h, OCCULT_ENULLPTR, "h is NULL with a pre norm");
  OCC_REQUIRE(aligned16(x) && aligned16(y) && aligned16(out) && aligned16(h), OCCULT_EALIGN, "a buffer is not 16-byte aligned");
  OCC_REQUIRE(!n->pre_kind || !y || h != out, OCCULT_EINVAL, "out and h are the same buffer");
  Args a{};
  a.x = x; a.y = y; a.gate = n->gate; a.out = out; a.h = h;
  a.post_w = n->post_weight; a.post_b = n->post_bias; a.pre_w = n->pre_weight; a.pre_b = n->pre_bias;
  a.T = c.T; a.row_vecs = c.d * elem_size(c) / 16;
  a.post = n->post_kind; a.pre = n->pre_kind; a.gate_kind = n->gate_kind;
  a.x_scale = n->x_scale; a.y_scale = n->y_scale; a.post_eps = n->post_eps; a.pre_eps = n->pre_eps;
  a.offset = n->weight_offset; a.inv_d = 1.0f / (float)c.d;
  const Shape s = shape_of(a.row_vecs, false);
  a.lanes = s.lanes;
  hipStream_t st = static_cast<hipStream_t>(stream);
  return c.dtype == OCCULT_BF16 ? launch_forward<true>(a, s, st) : launch_forward<false>(a, s, st);
}

extern "C" int occult_block_norm_backward_ws_bytes(const occult_cfg_t* cfg, const occult_block_norm_t* n, size_t* ws_bytes) {
  int rc = check(cfg, n);
  if (rc) return rc;
  OCC_REQUIRE(ws_bytes, OCCULT_ENULLPTR, "output pointer is NULL");
  *ws_bytes = (size_t)backward_blocks(*cfg) * popcount(wanted_sums(*n)) * (size_t)cfg->d * 4;
  return OCCULT_OK;
}

extern "C" int occult_block_norm_backward(const occult_cfg_t* cfg, const occult_block_norm_t* n, const void* y, const void* out,
                                          const void* dout, const void* dh, void* dx, void* dy,
                                          const occult_block_norm_grads_t* grads, int accumulate, void* ws, size_t ws_bytes,
                                          occult_stream_t stream) {
  int rc = check(cfg, n);
  if (rc) return rc;
  const occult_cfg_t& c = *cfg;
  OCC_REQUIRE(accumulate == 0 || accumulate == 1, OCCULT_EINVAL, "accumulate=%d must be 0 or 1", accumulate);
  OCC_REQUIRE(grads, OCCULT_ENULLPTR, "grads is NULL");
  const occult_block_norm_grads_t& g = *grads;
  OCC_REQUIRE((!g.post_weight || n->post_weight) && (!g.post_bias || n->post_bias) && (!g.pre_weight || n->pre_weight) &&
                  (!g.pre_bias || n->pre_bias) && (!g.gate || n->gate_kind),
              OCCULT_EINVAL, "a gradient is asked for of a parameter that is not there");
  OCC_REQUIRE(dy || c.T == 0 || (!g.post_weight && !g.post_bias && !g.gate), OCCULT_ENULLPTR,
              "gradients of the post norm or the gate without dy");
  OCC_REQUIRE(aligned16(y) && aligned16(out) && aligned16(dout) && aligned16(dh) && aligned16(dx) && aligned16(dy) && aligned16(ws) &&
                  aligned16(g.gate) && aligned16(g.post_weight) && aligned16(g.post_bias) && aligned16(g.pre_weight) &&
                  aligned16(g.pre_bias),
              OCCULT_EALIGN, "a buffer is not 16-byte aligned");
  float* const all[kColSums] = {g.post_weight, g.post_bias, g.pre_weight, g.pre_bias,
                                n->gate_kind == OCCULT_GATE_CHANNEL ? static_cast<float*>(g.gate) : nullptr};
  int sums = 0;
  for (int i = 0; i < kColSums; ++i) sums |= all[i] ? 1 << i : 0;
  const int blocks = backward_blocks(c);
  if (c.T > 0) {
    OCC_REQUIRE(!n->pre_kind || (out && dh), OCCULT_ENULLPTR, "out or dh is NULL with a pre norm");
    OCC_REQUIRE(n->pre_kind || dout, OCCULT_ENULLPTR, "dout is NULL without a pre norm");
    OCC_REQUIRE(dx || dy, OCCULT_ENULLPTR, "dx and dy are NULL");
    OCC_REQUIRE(!dy || y || (!n->post_kind && !n->gate_kind), OCCULT_ENULLPTR, "y is NULL with a post norm or a gate");
    OCC_REQUIRE(dx != dy, OCCULT_EINVAL, "dx and dy are the same buffer");
    if (sums)
      OCC_REQUIRE(ws && ws_bytes >= (size_t)blocks * popcount(sums) * (size_t)c.d * 4, OCCULT_EWORKSPACE,
                  "workspace of %zu bytes < required %zu", ws ? ws_bytes : (size_t)0, (size_t)blocks * popcount(sums) * (size_t)c.d * 4);
  }
  BackwardArgs a{};
  a.y = y; a.out = out; a.dout = dout; a.dh = dh; a.gate = n->gate; a.dx = dx; a.dy = dy; a.dgate = g.gate;
  a.post_w = n->post_weight; a.post_b = n->post_bias; a.pre_w = n->pre_weight;
  a.ws = static_cast<float*>(ws);
  a.T = c.T; a.row_vecs = c.d * elem_size(c) / 16;
  a.post = n->post_kind; a.pre = n->pre_kind; a.gate_kind = n->gate_kind; a.sums = sums;
  // the pre norm alone: h = N_pre(x) has no x_scale in it (without a pre norm there is no such call, and a y was there)
  const bool alone = !y && !dy && n->pre_kind && n->post_kind == OCCULT_NORM_NONE && n->gate_kind == OCCULT_GATE_NONE;
  a.x_scale = alone ? 1.0f : n->x_scale; a.y_scale = n->y_scale; a.post_eps = n->post_eps; a.pre_eps = n->pre_eps;
  a.offset = n->weight_offset; a.inv_d = 1.0f / (float)c.d;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (c.T > 0) {
    const Shape s = shape_of(a.row_vecs, true);
    a.lanes = s.lanes;
    const bool layer = n->post_kind == OCCULT_NORM_LAYER || n->pre_kind == OCCULT_NORM_LAYER || (sums & 10);
    if (c.dtype == OCCULT_BF16)
      rc = layer ? launch_backward<true, true>(a, s, blocks, st) : launch_backward<true, false>(a, s, blocks, st);
    else
      rc = layer ? launch_backward<false, true>(a, s, blocks, st) : launch_backward<false, false>(a, s, blocks, st);
    if (rc) return rc;
  }
  if (sums && (c.T > 0 || !accumulate)) {
    ColumnArgs ca{};
    ca.ws = a.ws;
    ca.blocks = c.T > 0 ? blocks : 0;
    ca.d = c.d;
    ca.accumulate = accumulate;
    for (int i = 0; i < kColSums; ++i)
      if (all[i]) ca.dst[ca.nsums++] = all[i];
    const long long cols = (long long)ca.nsums * c.d;
    column_sums_kernel<<<(int)((cols + 63) / 64), 1024, 0, st>>>(ca);
    OCC_LAUNCH_CHECK("column_sums_kernel");
  }
  return OCCULT_OK;
}
