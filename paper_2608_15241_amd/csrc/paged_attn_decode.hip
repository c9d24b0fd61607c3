// local_paged_attn_decode: one new token per request attends over its paged
// KV cache; blocks whose adapter-version tag differs from the request's
// version are excluded (§5.1 validity key; §1 challenge (2)).
//
// Design (HBM-bound: every valid KV byte is read once, stale blocks are never
// read):
//  * Split-KV. A workgroup owns a partition of 16 to 64 logical blocks of one
//    request and one KV head; it is one wave, or two or four where there are
//    few partitions (its valid blocks are dealt to the waves, whose results
//    meet in LDS). Partitions are counted from the end of the context. Up to
//    512 requests the dispatch slots take every full partition first, request
//    by request, then the requests' partial ones (their oldest blocks), longest
//    first, which shortens the tail when context lengths vary; with more
//    requests the partition index is the slowest grid dimension and the partial
//    ones come last in the order of the requests. A wave reads the partition's
//    table entries and tags first, keeps the non-stale blocks and walks them in
//    order through a ring of DEPTH register sets, so that DEPTH-1 blocks'
//    K/V loads are in flight while one block is computed. Block loads are
//    buffer loads issued unconditionally (a block past the end gets a
//    zero-size descriptor: zeros, no traffic) and the new token is merged in
//    with selects, so the loop has no data-dependent branch and each block
//    waits only for its own loads.
//  * Matrix cores, transposed. Per block, S^T[16 keys x 16 cols] =
//    K[16 x D] * Q^T[D x 16] on v_mfma_f32_16x16x32_bf16, where the columns
//    are the Hq/Hkv query heads that share KV head g (zero-padded to 16).
//    The K layout [D/8][16][8] makes each lane's 16-byte A-operand slice
//    contiguous and each MFMA's 64 loads one contiguous kilobyte. The score
//    tile's accumulator layout (lane: 4 keys of one column) is exactly the
//    B-operand layout of the next product O^T[D x 16] += V^T[D x 16] P^T on
//    v_mfma_f32_16x16x16_bf16, whose A operand comes straight from the V
//    layout [D][16] (each lane: 4 keys of one dim, 8 bytes).
//  * Online softmax in the log2 domain per column. A request that fits one
//    partition is finished in place; otherwise each partition leaves its
//    (max, sum, unnormalised O) and a second kernel merges them.
//  * The new token's K/V are written at position L-1 by the wave that owns
//    that block, which also substitutes them for the cache slot it reads, so
//    no other workgroup and no second launch is involved.
#include <mutex>

#include "paged_attn_decode.hpp"

namespace localk {
namespace {

// The 4 V values a lane holds for one block (slots slot0..slot0+3), with
// slots past s_live set to 0 (their cache contents are undefined and must not
// reach the product) and slot s_new replaced by vnew. For a block that is
// neither the last nor the appended one, s_live = 15 and s_new = -1 leave it
// unchanged; everything is a select.
__device__ __forceinline__ u32x2 fix_v(u32x2 v, int slot0, int s_live, int s_new,
                                       uint32_t vnew) {
  uint32_t h[4] = {v.x & 0xffffu, v.x >> 16, v.y & 0xffffu, v.y >> 16};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int slot = slot0 + e;
    h[e] = slot > s_live ? 0u : (slot == s_new ? vnew : h[e]);
  }
  u32x2 r;
  r.x = h[0] | (h[1] << 16);
  r.y = h[2] | (h[3] << 16);
  return r;
}

#ifndef LOCAL_DECODE_APPEND_NT
#define LOCAL_DECODE_APPEND_NT 1  // non-temporal stores: measured 9 us faster on the 7B batch
#endif
// Store of a piece of the appended token.
template <typename T>
__device__ __forceinline__ void st_append(uint16_t* p, T v) {
#if LOCAL_DECODE_APPEND_NT
  __builtin_nontemporal_store(v, reinterpret_cast<T*>(p));
#else
  *reinterpret_cast<T*>(p) = v;
#endif
}

// K/V registers of one block.
template <int D>
struct BlockRegs {
  u32x4 k[D / 32];
  u32x2 v[D / 16];
};

// WEIGHTED: each block's share of the softmax is recorded (DecodeArgs::blk_lse).
template <int D, int DEPTH, bool RANKED, int W, bool WEIGHTED>
__global__ __launch_bounds__(kWave* W) void decode_attn_kernel(DecodeArgs a, int B) {
  constexpr int KC = D / 32;  // 32-dim chunks of the QK product
  constexpr int VT = D / 16;  // 16-dim tiles of the PV product

  const int lane = threadIdx.x % kWave;
  const int wave = W == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int col = lane % 16, kgrp = lane / 16;
  // Partition p covers blocks [nb - P(p+1), nb - Pp) of b (P = a.pb): the full ones
  // counted from the end of the context, then at most one partial one at the
  // start. An empty context runs partition 0 with no block (zero output,
  // lse = -inf). The grid is 1D, KV heads fastest, sized for n_parts + 1
  // partitions of every request; the slots map to units longest first (full
  // partitions, then the partial ones by decreasing length), so the last
  // waves to start are the shortest and the idle slots come last. Batches
  // wider than the ranking takes dispatch each partition row in request
  // order instead, the partial partitions last.
  const int g = blockIdx.x % a.Hkv;
  const int slot = blockIdx.x / a.Hkv;
  int b, part;
  if (RANKED) {
    b = decode_unit(a, B, slot, &part);
    if (b < 0) return;
  } else {
    b = slot % B;
    part = slot / B;
  }
  const int L = a.ctx_lens[b];
  const int nb = owned_blocks(L, a.max_blocks);
  const int n_full = full_parts(nb, a.pb), rem = nb - n_full * a.pb;
  if (!RANKED) {
    if (part < a.n_parts) {
      if (part >= n_full && !(nb == 0 && part == 0)) return;
    } else {
      if (rem == 0) return;
      part = n_full;
    }
  }
  const int j_end_part = nb - part * a.pb;
  const int j0 = max(0, j_end_part - a.pb);
  const int n_parts_b = max(1, n_full + (rem > 0 ? 1 : 0));
  const int rv = a.req_version[b];
  const int32_t* table = a.block_table + static_cast<int64_t>(b) * a.max_blocks;
  const int G = a.group;

  // This partition's blocks: table entries and tags, keep the non-stale ones.
  const int jend = j_end_part;
  int my_phys = 0;
  bool ok = false;
  if (lane < a.pb && j0 + lane < jend) {
    my_phys = table[j0 + lane];
    ok = my_phys >= 0 && my_phys < a.num_blocks && a.block_version[my_phys] == rv;
    if (!ok) my_phys = 0;  // an id outside the pool is never dereferenced
  }
  // The valid blocks are dealt to the waves in turn: the i-th to wave i % W.
  const uint64_t part_valid = __ballot(ok);
  uint64_t valid_mask = part_valid;
  if (W > 1)
    valid_mask = __ballot(ok && __popcll(part_valid & ((1ull << lane) - 1ull)) % W == wave);
  if (a.vc_mask && g == 0 && wave == 0) {  // the version check of this partition's blocks
    const bool owned = lane < a.pb && j0 + lane < jend;
    const uint64_t stale = __ballot(owned && !ok);
    int live = ok ? min(kBlockSize, L - kBlockSize * (j0 + lane)) : 0;
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) live += __shfl_xor(live, off);
    if (lane == 0) {
      const int64_t slot = static_cast<int64_t>(b) * a.n_parts + part;
      a.vc_mask[slot] = stale;
      a.vc_valid[slot] = live;
    }
  }
  if constexpr (WEIGHTED) {  // stale blocks of this partition have no weight
    if (wave == 0 && lane < a.pb && j0 + lane < jend && !ok) {
      float* bl = blk_lse_at(a, b, g, j0 + lane);
      for (int h = 0; h < G; ++h) bl[h] = -INFINITY;
    }
  }

  // Query heads of this KV head, as the B operand (column = head).
  bf16x8 qv[KC];
  {
    const int h = g * G + col;
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      u32x4 v = {0u, 0u, 0u, 0u};
      if (col < G)
        v = ld_global<u32x4>(a.q + (static_cast<int64_t>(b) * a.Hq + h) * D + 32 * c +
                             8 * kgrp);
      qv[c] = as_bf16x8(v);
    }
  }

  // The new token (position L-1), if its block is in this partition: its K/V
  // rows are substituted for the slot while the block is read, and written to
  // the pool after the last block (an id outside the pool is not written).
  const int j_new = (L - 1) / kBlockSize, s_last = (L - 1) % kBlockSize;
  const bool has_new = a.k_new != nullptr;
  const int64_t kvrow = (static_cast<int64_t>(b) * a.Hkv + g) * D;
  bool append = has_new && j_new >= j0 && j_new < jend;
  if (W > 1 && append)  // by the wave that reads the block (a stale one: wave 0)
    append = (part_valid >> (j_new - j0) & 1ull) ? (valid_mask >> (j_new - j0) & 1ull) != 0ull
                                                 : wave == 0;
  const int p_new = append ? table[j_new] : -1;

  f32x4 acc[VT];
#pragma unroll
  for (int t = 0; t < VT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = kNegBig, l_run = 0.f;

  // the new token's K/V fragments, for the lanes that hold its slot
  u32x4 kn[KC];
  uint32_t vn[VT];
#pragma unroll
  for (int c = 0; c < KC; ++c) kn[c] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
  for (int t = 0; t < VT; ++t) vn[t] = 0u;
  if (append) {
#pragma unroll
    for (int c = 0; c < KC; ++c) kn[c] = ld_global<u32x4>(a.k_new + kvrow + 32 * c + 8 * kgrp);
#pragma unroll
    for (int t = 0; t < VT; ++t) vn[t] = a.v_new[kvrow + 16 * t + col];
  }

  // next valid block (partition-relative index), -1 when none is left
  auto next_block = [&]() -> int {
    if (!valid_mask) return -1;
    const int i = __builtin_ctzll(valid_mask);
    valid_mask &= valid_mask - 1;
    return i;
  };
  constexpr uint32_t kTileBytes = kBlockSize * D * 2;
  auto load_block = [&](BlockRegs<D>& R, int i) {
    const bool live = i >= 0;
    // the block id is the same in every lane: keep it (and the descriptors)
    // in scalar registers
    const int p = live ? __builtin_amdgcn_readlane(my_phys, i) : 0;
    const int64_t tile = (static_cast<int64_t>(p) * a.Hkv + g) * (kBlockSize * D);
    const __amdgpu_buffer_rsrc_t rk = make_rsrc(a.k_cache + tile, live ? kTileBytes : 0u);
    const __amdgpu_buffer_rsrc_t rv2 = make_rsrc(a.v_cache + tile, live ? kTileBytes : 0u);
#pragma unroll
    for (int c = 0; c < KC; ++c) R.k[c] = buf_load16_stream(rk, (c * 512 + lane * 8) * 2);
#pragma unroll
    for (int t = 0; t < VT; ++t)
      R.v[t] = buf_load8_stream(rv2, ((16 * t + col) * kBlockSize + 4 * kgrp) * 2);
  };
  auto compute_block = [&](BlockRegs<D>& R, int i) {
    const int j = j0 + i;
    const bool last = j == j_new;
    const int s_live = last ? s_last : kBlockSize - 1;
    const int s_new = (last && has_new) ? s_last : -1;
#pragma unroll
    for (int c = 0; c < KC; ++c) R.k[c] = col == s_new ? kn[c] : R.k[c];
#pragma unroll
    for (int t = 0; t < VT; ++t) R.v[t] = fix_v(R.v[t], 4 * kgrp, s_live, s_new, vn[t]);
    f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < KC; ++c) sc = mfma16x16x32(as_bf16x8(R.k[c]), qv[c], sc);
    float s[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      s[e] = j * kBlockSize + 4 * kgrp + e < L ? sc[e] * a.scale_log2 : -INFINITY;
    float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
    mx = max_xor32(max_xor16(mx));
    const float m_new = fmaxf(m_run, mx);
    const float alpha = fast_exp2(m_run - m_new);
    bf16x4 pb;
    float psum = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float p = fast_exp2(s[e] - m_new);
      psum += p;
      pb[e] = static_cast<__bf16>(p);
    }
    l_run = l_run * alpha + psum;
    m_run = m_new;
    if constexpr (WEIGHTED) {  // (log2 of 0 is -inf)
      const float sum = sum_kgroups(psum);
      if (kgrp == 0 && col < G) blk_lse_at(a, b, g, j)[col] = m_new + __log2f(sum);
    }
#pragma unroll
    for (int t = 0; t < VT; ++t) {
      acc[t] *= alpha;
      acc[t] = mfma16x16x16(as_bf16x4(R.v[t]), pb, acc[t]);
    }
  };

  // ring of DEPTH register sets: DEPTH-1 blocks load while one computes
  BlockRegs<D> R[DEPTH];
  int idx[DEPTH];
#pragma unroll
  for (int d = 0; d < DEPTH - 1; ++d) {
    idx[d] = next_block();
    load_block(R[d], idx[d]);
  }

  bool done = false;
  while (!done) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      const int fill = (d + DEPTH - 1) % DEPTH;
      idx[fill] = next_block();
      load_block(R[fill], idx[fill]);
      if (idx[d] < 0) {
        done = true;
        break;
      }
      compute_block(R[d], idx[d]);
    }
  }

  // ---- append: the new token's K/V rows from the registers that hold them
  // (K: k-group c8 = 4c + kgrp of the row in the 4 lanes of column 0; V: dim
  // 16t + col in the lanes of k-group 0), after every read of the block.
  // Written here rather than before the loop, a store ahead of the block
  // loads would hold them back (measured: 5 us per launch on the 7B batch).
  if (append && p_new >= 0 && p_new < a.num_blocks) {
    const int64_t tile = (static_cast<int64_t>(p_new) * a.Hkv + g) * (kBlockSize * D);
    if (col == 0) {
#pragma unroll
      for (int c = 0; c < KC; ++c)
        st_append<u32x4>(a.k_cache + tile + (4 * c + kgrp) * (kBlockSize * 8) + s_last * 8,
                         kn[c]);
    }
    if (kgrp == 0) {
#pragma unroll
      for (int t = 0; t < VT; ++t)
        st_append<uint16_t>(a.v_cache + tile + (16 * t + col) * kBlockSize + s_last,
                            static_cast<uint16_t>(vn[t]));
    }
  }

  // ---- finish: the column's sum over the 4 lane groups, then write
  l_run += __shfl_xor(l_run, 16);
  l_run += __shfl_xor(l_run, 32);
  if constexpr (W > 1) {
    // the waves' results meet in LDS; each thread then finishes 4 dims of a head
    extern __shared__ __attribute__((aligned(16))) float mg[];
    constexpr int kRow = D + 4;
    float* mg_ml = mg + W * G * kRow;
    if (col < G) {
      const int row = wave * G + col;
#pragma unroll
      for (int t = 0; t < VT; ++t)
        *reinterpret_cast<f32x4*>(mg + row * kRow + 16 * t + 4 * kgrp) = acc[t];
      if (kgrp == 0) {
        mg_ml[2 * row] = m_run;
        mg_ml[2 * row + 1] = l_run;
      }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < G * (D / 4); e += kWave * W) {
      const int hc = e / (D / 4), d = 4 * (e % (D / 4));
      float M = kNegBig;
#pragma unroll
      for (int w = 0; w < W; ++w) M = fmaxf(M, mg_ml[2 * (w * G + hc)]);
      float den = 0.f;
      f32x4 num = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < W; ++w) {  // a wave without a block: weight x 0
        const int row = w * G + hc;
        const float f = fast_exp2(mg_ml[2 * row] - M);
        den += mg_ml[2 * row + 1] * f;
        num += *reinterpret_cast<const f32x4*>(mg + row * kRow + d) * f;
      }
      const int64_t bh = static_cast<int64_t>(b) * a.Hq + g * G + hc;
      if (n_parts_b == 1) {
        num *= den > 0.f ? 1.f / den : 0.f;
        *reinterpret_cast<u32x2*>(a.out + bh * D + d) =
            u32x2{pack_bf16x2(num[0], num[1]), pack_bf16x2(num[2], num[3])};
        if (d == 0 && a.lse) a.lse[bh] = den > 0.f ? (M + __log2f(den)) * kLn2 : -INFINITY;
        if (WEIGHTED && d == 0) {
          a.part_ml[bh * a.n_parts * 2] = M;
          a.part_ml[bh * a.n_parts * 2 + 1] = den;
        }
      } else {
        const int64_t pi = bh * a.n_parts + part;
        *reinterpret_cast<f32x4*>(a.part_o + pi * D + d) = num;
        if (d == 0) {
          a.part_ml[pi * 2] = M;
          a.part_ml[pi * 2 + 1] = den;
        }
      }
    }
  } else if (col < G) {
    const int h = g * G + col;
    const int64_t bh = static_cast<int64_t>(b) * a.Hq + h;
    if (n_parts_b == 1) {
      const float inv = l_run > 0.f ? 1.f / l_run : 0.f;
#pragma unroll
      for (int t = 0; t < VT; ++t)
        *reinterpret_cast<u32x2*>(a.out + bh * D + 16 * t + 4 * kgrp) =
            u32x2{pack_bf16x2(acc[t][0] * inv, acc[t][1] * inv),
                  pack_bf16x2(acc[t][2] * inv, acc[t][3] * inv)};
      if (kgrp == 0 && a.lse)
        a.lse[bh] = l_run > 0.f ? (m_run + __log2f(l_run)) * kLn2 : -INFINITY;
      if (WEIGHTED && kgrp == 0) {
        a.part_ml[bh * a.n_parts * 2] = m_run;
        a.part_ml[bh * a.n_parts * 2 + 1] = l_run;
      }
    } else {
      const int64_t pi = bh * a.n_parts + part;
#pragma unroll
      for (int t = 0; t < VT; ++t)
        *reinterpret_cast<f32x4*>(a.part_o + pi * D + 16 * t + 4 * kgrp) = acc[t];
      if (kgrp == 0) {
        a.part_ml[pi * 2] = m_run;
        a.part_ml[pi * 2 + 1] = l_run;
      }
    }
  }
}

// Blocks in flight per wave: 4 with one query head per KV head, 3 with
// grouped heads (measured: 4 is 1.7% faster on the MHA decode step and 1.2%
// slower on the GQA one, whose waves do four heads' softmax per block).
#ifndef LOCAL_DECODE_DEPTH_MHA
#define LOCAL_DECODE_DEPTH_MHA 4
#endif
#ifndef LOCAL_DECODE_DEPTH
#define LOCAL_DECODE_DEPTH 3
#endif

template <int D, int DEPTH, bool RANKED, bool WEIGHTED>
void launch_attn(const DecodeArgs& a, int B, unsigned grid, int W, hipStream_t s) {
  const int lds = merge_lds_bytes<D>(W, a.group);
  if (W == 4)
    decode_attn_kernel<D, DEPTH, RANKED, 4, WEIGHTED><<<grid, 4 * kWave, lds, s>>>(a, B);
  else if (W == 2)
    decode_attn_kernel<D, DEPTH, RANKED, 2, WEIGHTED><<<grid, 2 * kWave, lds, s>>>(a, B);
  else
    decode_attn_kernel<D, DEPTH, RANKED, 1, WEIGHTED><<<grid, kWave, 0, s>>>(a, B);
}

template <int D, int DEPTH>
void launch_ranked(const DecodeArgs& a, int B, unsigned grid, int W, hipStream_t s) {
  if (B <= kRankChunks * kWave) {
    if (a.w_out)
      launch_attn<D, DEPTH, true, true>(a, B, grid, W, s);
    else
      launch_attn<D, DEPTH, true, false>(a, B, grid, W, s);
  } else {
    if (a.w_out)
      launch_attn<D, DEPTH, false, true>(a, B, grid, W, s);
    else
      launch_attn<D, DEPTH, false, false>(a, B, grid, W, s);
  }
}

// Waves that share a partition. What a wave does before its first block (three
// dependent loads) and its in-flight blocks bound a partition, so few units
// want more waves each, and many units want one (three waves of one unit hold
// the registers of three units). Units are counted from the table's width, since
// the host knows no lengths: half of them or less run. Measured in us with 1 / 2 / 4
// waves: one query head per KV head: 96 units 30 / 19 / 15; 512 31 / 22 / 27; 1536 to
// 3072 44 / 50 / 61, 79 / 82 / 99, 85 / 91 / 116, and with contexts of 10 blocks in
// tables of 64 19 / 22 / 28; 8192 199 / 202 / 238. Grouped heads: 248 units 31 / 21 /
// 17; 384 20 / 18 / 17; 768 33 / 28 / 26; 1024 33 / 34 / 33; 1280 37 / 42 / 40; 1536 to
// 2560 46 / 46 / 47, 54 / 51 / 53, 63 / 58 / 60, 76 / 72 / 75 (contexts that fill a
// third of the table 32 / 28, 34 / 36, 40 / 42, 52 / 50; with 64-block partitions 148 /
// 152 / 142); 3072 to 4096 84 / 87 / 86, 95 / 97 / 99, 117 / 111 / 112; 16384 719 / 715 /
// 725. So one wave from 768 units on, two for grouped heads from 1536 to 2560.
int waves_of(const DecodeArgs& a, int B) {
  const int64_t units = static_cast<int64_t>(a.Hkv) * B * a.n_parts;
  const bool mha = a.group == 1;
  if (units < (mha ? 257 : kFewUnits)) return 4;
  if (units < kFewUnits) return 2;
  const bool pair = !mha && units >= 1536 && units <= 2560;
  return pair && a.max_blocks >= 64 && a.pb < 64 ? 2 : 1;
}

template <int D>
local_status_t launch_decode(const DecodeArgs& a, int B, hipStream_t s) {
  const int64_t wgs = std::max(static_cast<int64_t>(a.Hkv) * B * (a.n_parts + 1),
                               a.w_out ? merge_grid<D>(a, B) : 0);
  if (wgs >= (1LL << 31))
    return local_fail(LOCAL_ERR_UNSUPPORTED, "paged_attn_decode: grid of %lld workgroups",
                      (long long)wgs);
  const unsigned grid = static_cast<unsigned>(a.Hkv) * B * (a.n_parts + 1);
  const int W = waves_of(a, B);
  if (a.group == 1)
    launch_ranked<D, LOCAL_DECODE_DEPTH_MHA>(a, B, grid, W, s);
  else
    launch_ranked<D, LOCAL_DECODE_DEPTH>(a, B, grid, W, s);
  if (a.w_out)
    decode_merge_kernel<D, false, true>
        <<<static_cast<unsigned>(merge_grid<D>(a, B)), D, a.Hq * sizeof(float), s>>>(a, B);
  else if (a.n_parts > 1 || a.vc_mask)
    decode_merge_kernel<D, false, false><<<B * a.Hq, D, 0, s>>>(a, B);
  return local_check_launch("paged_attn_decode");
}

}  // namespace
}  // namespace localk

using namespace localk;

// Host-side validation shared by the entry points: fills *a (without the
// partials' pointers) and *part, the split-KV partials of the call.
static local_status_t decode_setup(const uint16_t* q, int32_t B, int32_t Hq, int32_t Hkv,
                                   int32_t D, const uint16_t* k_new, const uint16_t* v_new,
                                   uint16_t* k_cache, uint16_t* v_cache, int64_t num_blocks,
                                   int32_t block_size, const int32_t* block_table,
                                   int32_t max_blocks, const int32_t* ctx_lens,
                                   const int32_t* block_version, const int32_t* req_version,
                                   float sm_scale, uint16_t* out, float* lse, const char* who,
                                   DecodeArgs* a, DecodeParts* part) {
  if (B < 0 || Hq <= 0 || Hkv <= 0 || max_blocks < 1 || num_blocks < 1 || Hq % Hkv != 0)
    return local_fail(LOCAL_ERR_SHAPE, "%s: B=%d Hq=%d Hkv=%d max_blocks=%d num_blocks=%lld",
                      who, B, Hq, Hkv, max_blocks, (long long)num_blocks);
  if (block_size != kBlockSize || (D != 64 && D != 128) || Hq / Hkv > 16)
    return local_fail(LOCAL_ERR_UNSUPPORTED,
                      "%s: block_size=%d D=%d group=%d (need 16, 64|128, <=16)", who,
                      block_size, D, Hq / Hkv);
  if ((k_new == nullptr) != (v_new == nullptr))
    return local_fail(LOCAL_ERR_NULL, "%s: k_new and v_new must both be set", who);
  a->q = q;
  a->k_new = k_new;
  a->v_new = v_new;
  a->k_cache = k_cache;
  a->v_cache = v_cache;
  a->block_table = block_table;
  a->ctx_lens = ctx_lens;
  a->block_version = block_version;
  a->req_version = req_version;
  a->out = out;
  a->lse = lse;
  a->part_o = nullptr;
  a->part_ml = nullptr;
  a->vc_mask = nullptr;
  a->vc_valid = nullptr;
  a->vc_pairs = nullptr;
  a->vc_cap = 0;
  a->vc_n_stale = nullptr;
  a->vc_valid_tokens = nullptr;
  a->blk_lse = nullptr;
  a->w_in = nullptr;
  a->w_out = nullptr;
  a->w_decay = 1.f;
  a->kv4 = nullptr;
  a->q_xor = 0u;
  a->q_and = ~0u;
  a->Hq = Hq;
  a->Hkv = Hkv;
  a->group = Hq / Hkv;
  a->num_blocks = num_blocks;
  a->max_blocks = max_blocks;
  a->scale_log2 = sm_scale * kLog2e;
  *part = decode_parts(*a, B, D, true);
  return LOCAL_OK;
}

static local_status_t decode_pointers_ok(const DecodeArgs& a, const char* who) {
  if (!a.q || !a.k_cache || !a.v_cache || !a.block_table || !a.ctx_lens ||
      !a.block_version || !a.req_version || !a.out)
    return local_fail(LOCAL_ERR_NULL, "%s: NULL pointer argument", who);
  return LOCAL_OK;
}

static local_status_t decode_launch(DecodeArgs& a, int B, int D, void* partials,
                                    size_t part_elems, void* stream) {
  a.part_o = static_cast<float*>(partials);
  a.part_ml = a.part_o + part_elems * D;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return D == 64 ? launch_decode<64>(a, B, s) : launch_decode<128>(a, B, s);
}

extern "C" local_status_t local_paged_attn_decode(
    const uint16_t* q, int32_t B, int32_t Hq, int32_t Hkv, int32_t D,
    const uint16_t* k_new, const uint16_t* v_new, uint16_t* k_cache, uint16_t* v_cache,
    int64_t num_blocks, int32_t block_size, const int32_t* block_table,
    int32_t max_blocks, const int32_t* ctx_lens, const int32_t* block_version,
    const int32_t* req_version, float sm_scale, uint16_t* out, float* lse, void* ws,
    size_t* ws_bytes, void* stream) {
  const char* who = "paged_attn_decode";
  if (!ws_bytes) return local_fail(LOCAL_ERR_WORKSPACE, "%s: ws_bytes is NULL", who);
  DecodeArgs a;
  DecodeParts part;
  local_status_t st = decode_setup(q, B, Hq, Hkv, D, k_new, v_new, k_cache, v_cache,
                                   num_blocks, block_size, block_table, max_blocks, ctx_lens,
                                   block_version, req_version, sm_scale, out, lse, who, &a,
                                   &part);
  if (st != LOCAL_OK) return st;
  if (!ws) {
    *ws_bytes = part.bytes;
    return LOCAL_OK;
  }
  if (*ws_bytes < part.bytes) part = decode_parts(a, B, D, false);
  if (*ws_bytes < part.bytes)
    return local_fail(LOCAL_ERR_WORKSPACE, "%s: workspace %zu < %zu", who, *ws_bytes, part.bytes);
  if (B == 0) return LOCAL_OK;
  if ((st = decode_pointers_ok(a, who)) != LOCAL_OK) return st;
  return decode_launch(a, B, D, ws, part.elems, stream);
}

// The partition length and waves that a call's size selects, as blocks + 256 x
// waves (for the tests, which name the form that they mean; not in local.h).
extern "C" int32_t localk_decode_form(int32_t B, int32_t Hq, int32_t Hkv, int32_t max_blocks) {
  DecodeArgs a{};
  a.Hkv = Hkv;
  a.group = Hq / Hkv;
  a.max_blocks = max_blocks;
  decode_parts(a, B, 128, true);
  return a.pb + 256 * waves_of(a, B);
}

// ---------------------------------------------------------------- checked
namespace {
__global__ void decode_vc_empty_kernel(int32_t* n_stale) { *n_stale = 0; }
}  // namespace

extern "C" local_status_t local_paged_attn_decode_checked(
    const uint16_t* q, int32_t B, int32_t Hq, int32_t Hkv, int32_t D,
    const uint16_t* k_new, const uint16_t* v_new, uint16_t* k_cache, uint16_t* v_cache,
    int64_t num_blocks, int32_t block_size, const int32_t* block_table,
    int32_t max_blocks, const int32_t* ctx_lens, const int32_t* block_version,
    const int32_t* req_version, float sm_scale, uint16_t* out, float* lse,
    int32_t* stale_pairs, int64_t cap, int32_t* n_stale, int32_t* valid_tokens, void* ws,
    size_t* ws_bytes, void* stream) {
  const char* who = "paged_attn_decode_checked";
  if (!ws_bytes) return local_fail(LOCAL_ERR_WORKSPACE, "%s: ws_bytes is NULL", who);
  DecodeArgs a;
  DecodeParts part;
  local_status_t st = decode_setup(q, B, Hq, Hkv, D, k_new, v_new, k_cache, v_cache,
                                   num_blocks, block_size, block_table, max_blocks, ctx_lens,
                                   block_version, req_version, sm_scale, out, lse, who, &a,
                                   &part);
  if (st != LOCAL_OK) return st;
  if (cap < 0) return local_fail(LOCAL_ERR_SHAPE, "%s: cap=%lld", who, (long long)cap);
  if (a.n_parts > D)
    return local_fail(LOCAL_ERR_UNSUPPORTED, "%s: max_blocks=%d over %d blocks", who,
                      max_blocks, D * a.pb);
  auto total = [](const DecodeParts& p) {
    return align256(p.bytes) + align256(p.units * sizeof(uint64_t)) +
           align256(p.units * sizeof(int32_t));
  };
  if (!ws) {
    *ws_bytes = total(part);
    return LOCAL_OK;
  }
  if (*ws_bytes < total(part)) part = decode_parts(a, B, D, false);
  if (*ws_bytes < total(part))
    return local_fail(LOCAL_ERR_WORKSPACE, "%s: workspace %zu < %zu", who, *ws_bytes, total(part));
  if (!n_stale || (B > 0 && !valid_tokens) || (cap > 0 && !stale_pairs))
    return local_fail(LOCAL_ERR_NULL, "%s: NULL version-check output", who);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (B == 0) {
    decode_vc_empty_kernel<<<1, 1, 0, s>>>(n_stale);
    return local_check_launch(who);
  }
  if ((st = decode_pointers_ok(a, who)) != LOCAL_OK) return st;
  char* base = static_cast<char*>(ws);
  a.vc_mask = reinterpret_cast<uint64_t*>(base + align256(part.bytes));
  a.vc_valid = reinterpret_cast<int32_t*>(base + align256(part.bytes) +
                                          align256(part.units * sizeof(uint64_t)));
  a.vc_pairs = stale_pairs;
  a.vc_cap = cap;
  a.vc_n_stale = n_stale;
  a.vc_valid_tokens = valid_tokens;
  return decode_launch(a, B, D, ws, part.elems, stream);
}

// ---------------------------------------------------------------- no-alloc
// Scratch of local_paged_attn_decode_noalloc: the split-KV partials of up to
// 131072 (request, query head, partition) triples at D = 128, held
// by the library in device memory (one copy per GPU, for the life of the
// process). In host code `scratch` names a host-side stand-in, not the device
// copy: its device address is taken once per device with
// hipGetSymbolAddress and only that address is ever passed to a kernel.
constexpr size_t kNoAllocBytes = LOCAL_DECODE_NOALLOC_SCRATCH_BYTES;
static_assert(kNoAllocBytes == 131072 * (128 + 2) * sizeof(float), "partials at D = 128");
__device__ __align__(256) float scratch[kNoAllocBytes / sizeof(float)];

namespace {
constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void* g_scratch_ptr[kMaxDevices] = {};

// The device address of `scratch` on the current device (taken on its first
// use there, with that device current). NULL with *st set on failure.
void* scratch_of_current_device(local_status_t* st) {
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess || dev < 0 || dev >= kMaxDevices) {
    *st = local_fail(LOCAL_ERR_HIP, "paged_attn_decode_noalloc: hipGetDevice: %s (device %d)",
                     hipGetErrorString(e), dev);
    return nullptr;
  }
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  if (!g_scratch_ptr[dev]) {
    void* p = nullptr;
    e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
    if (e != hipSuccess || !p) {
      *st = local_fail(LOCAL_ERR_HIP, "paged_attn_decode_noalloc: hipGetSymbolAddress: %s",
                       hipGetErrorString(e));
      return nullptr;
    }
    g_scratch_ptr[dev] = p;
  }
  return g_scratch_ptr[dev];
}
}  // namespace

extern "C" local_status_t local_paged_attn_decode_noalloc(
    const uint16_t* q, int32_t B, int32_t Hq, int32_t Hkv, int32_t D,
    const uint16_t* k_new, const uint16_t* v_new, uint16_t* k_cache, uint16_t* v_cache,
    int64_t num_blocks, int32_t block_size, const int32_t* block_table,
    int32_t max_blocks, const int32_t* ctx_lens, const int32_t* block_version,
    const int32_t* req_version, float sm_scale, uint16_t* out, float* lse, void* stream) {
  const char* who = "paged_attn_decode_noalloc";
  DecodeArgs a;
  DecodeParts part;
  local_status_t st = decode_setup(q, B, Hq, Hkv, D, k_new, v_new, k_cache, v_cache,
                                   num_blocks, block_size, block_table, max_blocks, ctx_lens,
                                   block_version, req_version, sm_scale, out, lse, who, &a,
                                   &part);
  if (st != LOCAL_OK) return st;
  if (part.bytes > kNoAllocBytes)
    return local_fail(LOCAL_ERR_UNSUPPORTED,
                      "%s: B*Hq*ceil(max_blocks/%d)*(D+2)*4 = %zu bytes of partials exceed the "
                      "library's fixed scratch of %zu bytes (use local_paged_attn_decode with a "
                      "workspace)", who, a.pb, part.bytes, kNoAllocBytes);
  if (B == 0) return LOCAL_OK;
  if ((st = decode_pointers_ok(a, who)) != LOCAL_OK) return st;
  void* partials = scratch_of_current_device(&st);
  if (!partials) return st;
  return decode_launch(a, B, D, partials, part.elems, stream);
}

// ---------------------------------------------------------------- weighted
// Decode attention with the weight of each block. The attention launch records
// each (block, query head)'s log-sum-exp as it passes (B * max_blocks * Hq floats:
// 4 bytes where the block's K and V of one KV head take 64 D), and the merge
// launch, which knows every head's sum, turns them into weights: no launch and no
// pass over K of its own.
extern "C" local_status_t local_paged_attn_decode_weighted(
    const uint16_t* q, int32_t B, int32_t Hq, int32_t Hkv, int32_t D,
    const uint16_t* k_new, const uint16_t* v_new, uint16_t* k_cache, uint16_t* v_cache,
    int64_t num_blocks, int32_t block_size, const int32_t* block_table,
    int32_t max_blocks, const int32_t* ctx_lens, const int32_t* block_version,
    const int32_t* req_version, float sm_scale, uint16_t* out, float* lse,
    const float* weight_in, float weight_decay, float* weight_out, void* ws,
    size_t* ws_bytes, void* stream) {
  const char* who = "paged_attn_decode_weighted";
  if (!ws_bytes) return local_fail(LOCAL_ERR_WORKSPACE, "%s: ws_bytes is NULL", who);
  DecodeArgs a;
  DecodeParts part;
  local_status_t st = decode_setup(q, B, Hq, Hkv, D, k_new, v_new, k_cache, v_cache,
                                   num_blocks, block_size, block_table, max_blocks, ctx_lens,
                                   block_version, req_version, sm_scale, out, lse, who, &a,
                                   &part);
  if (st != LOCAL_OK) return st;
  if ((st = decode_weights_ok(Hq, weight_decay, who)) != LOCAL_OK) return st;
  const size_t need = align256(part.bytes) + block_lse_bytes(B, Hq, max_blocks);
  if (!ws) {
    *ws_bytes = need;
    return LOCAL_OK;
  }
  if (*ws_bytes < need)
    return local_fail(LOCAL_ERR_WORKSPACE, "%s: workspace %zu < %zu", who, *ws_bytes, need);
  if (B == 0) return LOCAL_OK;
  if ((st = decode_pointers_ok(a, who)) != LOCAL_OK) return st;
  if (!weight_out) return local_fail(LOCAL_ERR_NULL, "%s: weight_out is NULL", who);
  if ((st = decode_weights_apart(weight_in, weight_out, B, max_blocks, who)) != LOCAL_OK)
    return st;
  a.blk_lse = reinterpret_cast<float*>(static_cast<char*>(ws) + align256(part.bytes));
  a.w_in = weight_in;
  a.w_out = weight_out;
  a.w_decay = weight_decay;
  return decode_launch(a, B, D, ws, part.elems, stream);
}
