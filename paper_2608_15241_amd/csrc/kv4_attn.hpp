// Attention of up to 16 query rows of one KV head over blocks of the 4-bit pool, in one
// wave and its registers: what decode attention and prefill attention of few rows share.
//
// Blocks are taken in pairs: S^T[16 keys x 16 rows] = K Q^T of each on
// v_mfma_f32_16x16x32_bf16, then O^T += V^T P^T over their 32 keys. A score tile's
// layout (lane: 4 keys of one row) is that of the value product's B operand, and the
// pool's codes lie as the A operands do, so nothing crosses lanes but a row's maximum
// when it rises and its sums at the end. Scores, maximum, sums and output are float32; the
// weights are rounded to bf16 for the value product (2^-8 of each at most), which the
// matrix instruction needs. They are summed unrounded, for the log-sum-exp and the join
// with other parts, and as rounded, which the output is divided by: an output is then an
// average of values by weights that add up to one, and what one key dominates, or values
// that agree, keep every bit. (The rest of each weight as a second product would take
// decode 1 to 5% longer at D = 128, up to 10% at D = 64, and 128-row prefill 25%.)
#pragma once

#include <type_traits>

#include "kv4.hpp"

namespace localk {
namespace {

constexpr float kLazy4 = 8.f;        // log2 of the largest weight before the maximum rises
constexpr float kNegBig4 = -1.0e30f;  // the running maximum before any key

// One pair of blocks in registers, as loaded.
template <int D>
struct Regs4 {
  uint32_t k[2][D / 32];  // this lane's codes of K and V
  uint32_t v[2][D / 32];
  uint32_t ks[2], vs[2];  // the scale of its K dims; the scales of its 4 tokens of V
};

template <int D>
__device__ __forceinline__ void load_codes(__amdgpu_buffer_rsrc_t r, uint32_t off,
                                           uint32_t (&c)[D / 32]) {
  if constexpr (D == 128) {
    const u32x4 v = buf_load16_stream(r, off);
    c[0] = v.x, c[1] = v.y, c[2] = v.z, c[3] = v.w;
  } else {
    const u32x2 v = buf_load8_stream(r, off);
    c[0] = v.x, c[1] = v.y;
  }
}

// Block e of a pair: tile p * Hkv + g of the pool (nothing is read, and zeros come, where
// there is no block). The codes are read once; the scales share their lines.
template <int D>
__device__ __forceinline__ void load_block4(Regs4<D>& R, int e, const uint8_t* kv4, int64_t tile,
                                            bool live) {
  using L4 = Kv4<D>;
  const int lane = threadIdx.x % kWave, col = lane % 16, kgrp = lane / 16;
  const __amdgpu_buffer_rsrc_t r = make_rsrc(kv4 + tile * L4::kTile, live ? L4::kTile : 0u);
  load_codes<D>(r, lane * L4::kLane, R.k[e]);
  load_codes<D>(r, L4::kV + lane * L4::kLane, R.v[e]);
  R.ks[e] = __builtin_amdgcn_raw_buffer_load_b8(r, L4::k_scale(L4::k_group(kgrp), col), 0, 0);
  R.vs[e] =
      __builtin_amdgcn_raw_buffer_load_b32(r, L4::v_scale(L4::v_group(col), 4 * kgrp), 0, 0);
}

// c plus both bf16 values of a dword.
__device__ __forceinline__ float add_pair(uint32_t w, float c) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w),
                                         __builtin_bit_cast(bf16x2, 0x3f803f80u), c, false);
}

// What turns a sum of values by rounded weights (of sum w) into one that is divided by the
// sum l of the unrounded ones. No weight (or none above the smallest floats): 1.
__device__ __forceinline__ float rounded_fit(float l, float w) { return w == 0.f ? 1.f : l / w; }

template <int D>
struct Attn4 {
  static constexpr int KC = D / 32, VT = D / 16;
  bf16x8 qv[KC];  // row lane % 16, the dims of the lane's codes of K
  f32x4 acc[VT];  // tile t, element i: dim (4 (lane / 16) + i) * VT + t of row lane % 16
  float m_run, rise;   // running maximum (log2); raw score that raises it
  float l_run, w_run;  // sums of the weights, and of the weights as rounded

  __device__ __forceinline__ void init(float inv_scale) {
#pragma unroll
    for (int t = 0; t < VT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    m_run = kNegBig4;
    l_run = w_run = 0.f;
    rise = (kNegBig4 + kLazy4) * inv_scale;
  }

  __device__ __forceinline__ void load_q(const uint16_t* row, bool in, uint32_t q_xor,
                                         uint32_t q_and) {
    const int kgrp = threadIdx.x % kWave / 16;
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      u32x4 v = {0u, 0u, 0u, 0u};
      if (in) v = ld_global<u32x4>(row + (D / 4) * kgrp + 8 * c);
      qv[c] = as_bf16x8((v ^ q_xor) & q_and);
    }
  }

  // Raw scores of block e: keys 4 (lane / 16) .. of row lane % 16.
  __device__ __forceinline__ f32x4 scores(const Regs4<D>& R, int e) const {
    const float ks = scale4(R.ks[e]);
    f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      const uint32_t w = R.k[e][c];
      const u32x4 kf = {unpack4<0>(w, ks), unpack4<1>(w, ks), unpack4<2>(w, ks),
                        unpack4<3>(w, ks)};
      sc = mfma16x16x32(as_bf16x8(kf), qv[c], sc);
    }
    return sc;
  }

  // Scores (-inf: not seen) -> weights as the value product's operand; ps: this lane's
  // sums of the two blocks' weights. The running maximum rises only when a weight would
  // pass 2^kLazy4: below, float32 holds the weights as well as below 1, and nothing has to
  // cross lanes or be rescaled. scale: > 0, log2 units, inv_scale its reciprocal.
  __device__ __forceinline__ void weigh(const f32x4 (&sc)[2], float scale, float inv_scale,
                                        float (&ps)[2], u32x4& pf) {
    const float mx = max3f(max3f(sc[0][0], sc[0][1], sc[0][2]),
                           max3f(sc[0][3], sc[1][0], sc[1][1]),
                           __builtin_elementwise_maximum(sc[1][2], sc[1][3]));
    if (__ballot(mx > rise)) {
      const float m_new = fmaxf(m_run, max_xor32(max_xor16(mx)) * scale);
      const float alpha = fast_exp2(m_run - m_new);
      l_run *= alpha;
      w_run *= alpha;
      m_run = m_new;
      rise = (m_new + kLazy4) * inv_scale;
#pragma unroll
      for (int t = 0; t < VT; ++t) acc[t] *= alpha;
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float p[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) p[k] = fast_exp2(fmaf(sc[e][k], scale, -m_run));
      ps[e] = (p[0] + p[1]) + (p[2] + p[3]);
      pf[2 * e] = pack_bf16x2(p[0], p[1]);
      pf[2 * e + 1] = pack_bf16x2(p[2], p[3]);
    }
    l_run += ps[0] + ps[1];
#pragma unroll
    for (int k = 0; k < 4; ++k) w_run = add_pair(pf[k], w_run);
  }

  // Tiles 2 I and 2 I + 1 of the value product: byte I of a token's codes.
  template <int I>
  __device__ __forceinline__ void pair_tiles(const Regs4<D>& R, const float (&vs)[2][4],
                                             u32x4 pf) {
    u32x4 lo, hi;
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t x0 = unpack4<I>(v_token<D>(R.v[e], 2 * k), vs[e][2 * k]);
        const uint32_t x1 = unpack4<I>(v_token<D>(R.v[e], 2 * k + 1), vs[e][2 * k + 1]);
        lo[2 * e + k] = __builtin_amdgcn_perm(x1, x0, 0x05040100u);
        hi[2 * e + k] = __builtin_amdgcn_perm(x1, x0, 0x07060302u);
      }
    acc[2 * I] = mfma16x16x32(as_bf16x8(lo), as_bf16x8(pf), acc[2 * I]);
    acc[2 * I + 1] = mfma16x16x32(as_bf16x8(hi), as_bf16x8(pf), acc[2 * I + 1]);
  }

  __device__ __forceinline__ void values(const Regs4<D>& R, u32x4 pf) {
    float vs[2][4];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      vs[e][0] = scale4_of<0>(R.vs[e]);
      vs[e][1] = scale4_of<1>(R.vs[e]);
      vs[e][2] = scale4_of<2>(R.vs[e]);
      vs[e][3] = scale4_of<3>(R.vs[e]);
    }
    pair_tiles<0>(R, vs, pf);
    pair_tiles<1>(R, vs, pf);
    if constexpr (D == 128) {
      pair_tiles<2>(R, vs, pf);
      pair_tiles<3>(R, vs, pf);
    }
  }

  // put(row, d, the row's unnormalised output at dims d .. d + 3, its maximum, its sum) for
  // every row below `rows` and d, of W waves' results joined through mg (W > 1:
  // join4_bytes of LDS). Sums the rows over the lanes first.
  template <int W, typename Put>
  __device__ __forceinline__ void finish(int rows, float* mg, Put put) {
    const int lane = threadIdx.x % kWave, col = lane % 16, kgrp = lane / 16;
    l_run = sum_kgroups(l_run);
    const float fit = rounded_fit(l_run, sum_kgroups(w_run));
#pragma unroll
    for (int t = 0; t < VT; ++t) acc[t] *= fit;
    auto lane_dims = [&](int i, int t4) {  // tiles 4 t4 .. + 3 of element i
      return f32x4{acc[4 * t4][i], acc[4 * t4 + 1][i], acc[4 * t4 + 2][i], acc[4 * t4 + 3][i]};
    };
    if constexpr (W > 1) {
      constexpr int kRow = D + 4;
      float* mg_ml = mg + W * rows * kRow;
      if (col < rows) {
        const int row = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) * rows + col;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int t4 = 0; t4 < VT / 4; ++t4)
            *reinterpret_cast<f32x4*>(mg + row * kRow + (4 * kgrp + i) * VT + 4 * t4) =
                lane_dims(i, t4);
        if (kgrp == 0) {
          mg_ml[2 * row] = m_run;
          mg_ml[2 * row + 1] = l_run;
        }
      }
      __syncthreads();
      for (int e = threadIdx.x; e < rows * (D / 4); e += kWave * W) {
        const int row = e / (D / 4), d = 4 * (e % (D / 4));
        float M = kNegBig4;
#pragma unroll
        for (int w = 0; w < W; ++w) M = fmaxf(M, mg_ml[2 * (w * rows + row)]);
        float den = 0.f;
        f32x4 num = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < W; ++w) {  // a wave without a block: weight x 0
          const int at = w * rows + row;
          const float f = fast_exp2(mg_ml[2 * at] - M);
          den += mg_ml[2 * at + 1] * f;
          num += *reinterpret_cast<const f32x4*>(mg + at * kRow + d) * f;
        }
        put(row, d, num, M, den);
      }
    } else if (col < rows) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int t4 = 0; t4 < VT / 4; ++t4)
          put(col, (4 * kgrp + i) * VT + 4 * t4, lane_dims(i, t4), m_run, l_run);
    }
  }
};

// LDS of W waves' results of `rows` rows: a padded row of output, its maximum and sum.
template <int D>
constexpr int join4_bytes(int W, int rows) {
  return W > 1 ? W * rows * (D + 4 + 2) * static_cast<int>(sizeof(float)) : 0;
}

}  // namespace
}  // namespace localk
