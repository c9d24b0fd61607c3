// local_paged_attn_decode_kv4: decode attention over the 4-bit pool, with the new
// token's append and, when asked for, the weight of each block.
//
// Mathematics: s = sm_scale q K^, w = softmax(s), out = w V^ over the valid keys, K^
// and V^ the values that the pool's codes stand for (the new token's too). Those are
// bf16 values exactly, so the products and sums are those of bf16 decode attention.
//
// Bound by HBM: a block and KV head is one tile of 17 D bytes, read once, against
// 64 D in bf16. What the smaller tile changes against the bf16 kernel:
//  * Unpacking must not cost more than the loads: 2176 bytes hold 4096 values, so at
//    6 TB/s the chip has some 3 vector instructions a value. The codes lie in operand
//    order (kv4.hpp), a conversion makes two scaled values, and V needs one lane-local
//    permute per two values to pair neighbouring tokens: 1.3 instructions a value and
//    lane group, of which the scales are 0.2.
//  * Blocks are taken in pairs (kv4_attn.hpp).
//  * Partitions, dispatch order, waves per partition and merge: as for bf16.
// 128 contexts of 1024 to 16384 tokens, 8 KV heads of 128, weights of the blocks too:
// 218 us, 5.0 TB/s (the loads alone take 95% of it).
#include "kv4_attn.hpp"
#include "paged_attn_decode.hpp"

namespace localk {
namespace {

// The new token as a lane holds it: its K dims (D/4, one scale) where the lane's
// column is the token's slot, its V dims (D/16) where its k-group holds the slot.
template <int D>
struct NewToken {
  uint32_t k[D / 32], v, ks, vs;
};

template <int D>
__device__ __forceinline__ void quantise_new(const uint16_t* k_new, const uint16_t* v_new,
                                             int col, int kgrp, NewToken<D>& n) {
  u32x4 kv[D / 32], vv = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int c = 0; c < D / 32; ++c) kv[c] = ld_global<u32x4>(k_new + (D / 4) * kgrp + 8 * c);
  if constexpr (D == 128) {
    vv = ld_global<u32x4>(v_new + 8 * col);
  } else {
    const u32x2 w = ld_global<u32x2>(v_new + 4 * col);
    vv = u32x4{w.x, w.y, 0u, 0u};
  }
  n.ks = round_k<D>(kv, n.k);
  n.vs = round_v<D>(vv, n.v);
}

// __launch_bounds__: three waves a SIMD (registers permitting, and they do: two ran the
// 128 contexts of 1K to 16K tokens 3% slower).
template <int D, int DEPTH, bool RANKED, int W, bool WEIGHTED>
__global__ __launch_bounds__(kWave* W, 3) void decode_kv4_kernel(DecodeArgs a, int B) {
  using L4 = Kv4<D>;
  constexpr int KC = D / 32;

  const int lane = threadIdx.x % kWave;
  const int wave = W == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int col = lane % 16, kgrp = lane / 16;
  // Ranked units and their order: as decode_attn_kernel, partitions counted from the end.
  // Otherwise partition p is blocks [pb p, pb (p + 1)), so that the table's entries are
  // on their way before the length is known.
  const int g = blockIdx.x % a.Hkv;
  const int slot = blockIdx.x / a.Hkv;
  int b, part, L, nb, n_full, j0, jend;
  int my_phys = -1;
  const int32_t* table = a.block_table;
  if constexpr (RANKED) {
    b = decode_unit(a, B, slot, &part);
    if (b < 0) return;
    L = a.ctx_lens[b];
    nb = owned_blocks(L, a.max_blocks);
    n_full = full_parts(nb, a.pb);
    jend = nb - part * a.pb;
    j0 = max(0, jend - a.pb);
    table += static_cast<int64_t>(b) * a.max_blocks;
    if (lane < a.pb && j0 + lane < jend) my_phys = table[j0 + lane];
  } else {
    b = slot % B;
    part = slot / B;
    L = a.ctx_lens[b];
    j0 = part * a.pb;
    table += static_cast<int64_t>(b) * a.max_blocks;
    if (lane < a.pb && j0 + lane < a.max_blocks) my_phys = table[j0 + lane];
    nb = owned_blocks(L, a.max_blocks);
    if (j0 >= max(nb, 1)) return;
    n_full = full_parts(nb, a.pb);
    jend = min(nb, j0 + a.pb);
  }
  const int n_parts_b = max(1, n_full + (nb > n_full * a.pb ? 1 : 0));
  const int rv = a.req_version[b];
  const int G = a.group;

  const bool owned = lane < a.pb && j0 + lane < jend;
  bool ok = false;
  if (owned) ok = my_phys >= 0 && my_phys < a.num_blocks && a.block_version[my_phys] == rv;
  if (!ok) my_phys = 0;  // an id outside the pool is never dereferenced
  const uint64_t part_valid = __ballot(ok);
  uint64_t valid_mask = part_valid;
  if (W > 1)
    valid_mask = __ballot(ok && __popcll(part_valid & ((1ull << lane) - 1ull)) % W == wave);
  if constexpr (WEIGHTED) {  // stale blocks of this partition have no weight
    if (wave == 0 && owned && !ok) {
      float* none = blk_lse_at(a, b, g, j0 + lane);
      for (int h = 0; h < G; ++h) none[h] = -INFINITY;
    }
  }

  // Rows: the query heads of this KV head.
  const int64_t bh0 = static_cast<int64_t>(b) * a.Hq + g * G;
  Attn4<D> at;
  at.load_q(a.q + (bh0 + col) * D, col < G, a.q_xor, a.q_and);
  const float inv_scale = 1.f / a.scale_log2;
  at.init(inv_scale);

  // The new token (position L-1), if its block is in this partition: substituted while
  // the block is read, written after the last block.
  const int j_new = (L - 1) / kBlockSize, s_last = (L - 1) % kBlockSize;
  const bool has_new = a.k_new != nullptr;
  bool append = has_new && j_new >= j0 && j_new < jend;
  if (W > 1 && append)  // by the wave that reads the block (a stale one: wave 0)
    append = (part_valid >> (j_new - j0) & 1ull) ? (valid_mask >> (j_new - j0) & 1ull) != 0ull
                                                 : wave == 0;
  const int p_new = append ? table[j_new] : -1;
  NewToken<D> fresh{};
  if (append) {
    const int64_t row = (static_cast<int64_t>(b) * a.Hkv + g) * D;
    quantise_new<D>(a.k_new + row, a.v_new + row, col, kgrp, fresh);
  }

  // (WEIGHTED) where this lane records block j0's weight
  float* bl = blk_lse_at(a, b, g, j0) + col;

  auto next_block = [&]() -> int {
    if (!valid_mask) return -1;
    const int i = __builtin_ctzll(valid_mask);
    valid_mask &= valid_mask - 1;
    return i;
  };
  auto load_block = [&](Regs4<D>& R, int e, int i) {
    const int p = i >= 0 ? __builtin_amdgcn_readlane(my_phys, i) : 0;
    load_block4<D>(R, e, a.kv4, static_cast<int64_t>(p) * a.Hkv + g, i >= 0);
  };
  // The block that holds the last position: the new token's codes for its slot; slots
  // past it as zeros (their contents are undefined and must not reach the product).
  auto fix_last = [&](Regs4<D>& R, int e) {
    if (has_new && col == s_last) {
#pragma unroll
      for (int c = 0; c < KC; ++c) R.k[e][c] = fresh.k[c];
      R.ks[e] = fresh.ks;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int s = 4 * kgrp + i;
      const bool dead = s > s_last, put = has_new && s == s_last;
      const uint32_t byte = 0xffu << (8 * i);
      R.vs[e] = dead ? R.vs[e] & ~byte : put ? (R.vs[e] & ~byte) | fresh.vs << (8 * i) : R.vs[e];
      if constexpr (D == 128) {
        R.v[e][i] = dead ? 0u : put ? fresh.v : R.v[e][i];
      } else {
        const int sh = 16 * (i % 2);
        const uint32_t rest = R.v[e][i / 2] & ~(0xffffu << sh);
        R.v[e][i / 2] = dead ? rest : put ? rest | (fresh.v & 0xffffu) << sh : R.v[e][i / 2];
      }
    }
  };
  auto compute = [&](Regs4<D>& R, int i0, int i1) {
    f32x4 sc[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int i = e ? i1 : i0;
      const bool tail = i < 0 || j0 + i == j_new;
      if (tail && i >= 0) fix_last(R, e);
      sc[e] = at.scores(R, e);
      if (tail) {  // no block, or one with slots past the context's end
        const int live = i < 0 ? 0 : L - (j0 + i) * kBlockSize;
#pragma unroll
        for (int k = 0; k < 4; ++k) sc[e][k] = 4 * kgrp + k < live ? sc[e][k] : -INFINITY;
      }
    }
    float ps[2];
    u32x4 pf;
    at.weigh(sc, a.scale_log2, inv_scale, ps, pf);
    if constexpr (WEIGHTED) {
      // k-group 0 ends up with the first block's sum, k-group 1 with the second's
      const int i = kgrp == 0 ? i0 : i1;
      const float sum = sum_kgroups2(ps[0], ps[1]);
      if (kgrp < 2 && col < G && i >= 0) bl[i * G] = at.m_run + __log2f(sum);
    }
    at.values(R, pf);
  };

  // ring of DEPTH pairs: DEPTH-1 pairs load while one computes
  Regs4<D> R[DEPTH];
  int i0[DEPTH], i1[DEPTH];
  auto fill = [&](int d) {
    i0[d] = next_block();
    i1[d] = next_block();
    load_block(R[d], 0, i0[d]);
    load_block(R[d], 1, i1[d]);
  };
#pragma unroll
  for (int d = 0; d < DEPTH - 1; ++d) fill(d);
  bool done = false;
  while (!done) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      fill((d + DEPTH - 1) % DEPTH);
      if (i0[d] < 0) {
        done = true;
        break;
      }
      compute(R[d], i0[d], i1[d]);
    }
  }

  // ---- append, after every read of the block
  if (append && p_new >= 0 && p_new < a.num_blocks) {
    uint8_t* tile = a.kv4 + (static_cast<int64_t>(p_new) * a.Hkv + g) * L4::kTile;
    if (col == 0) {  // K: the slot's codes of each k-group
      uint32_t* to = reinterpret_cast<uint32_t*>(tile + (kgrp * kBlockSize + s_last) * L4::kLane);
#pragma unroll
      for (int c = 0; c < KC; ++c) to[c] = fresh.k[c];
      if (D == 128 || kgrp % 2 == 0)
        tile[L4::k_scale(L4::k_group(kgrp), s_last)] = static_cast<uint8_t>(fresh.ks);
    }
    if (kgrp == 1) {  // V: the slot's codes of each column's dims
      uint8_t* to = tile + L4::kV + ((s_last / 4 * 16 + col) * 4 + s_last % 4) * L4::kTokenV;
      if constexpr (D == 128)
        *reinterpret_cast<uint32_t*>(to) = fresh.v;
      else
        *reinterpret_cast<uint16_t*>(to) = static_cast<uint16_t>(fresh.v);
      if (col % (16 / L4::kGroups) == 0)
        tile[L4::v_scale(L4::v_group(col), s_last)] = static_cast<uint8_t>(fresh.vs);
    }
  }

  extern __shared__ __attribute__((aligned(16))) float mg[];
  at.template finish<W>(G, mg, [&](int hc, int d, f32x4 num, float M, float den) {
    const int64_t bh = bh0 + hc;
    if (n_parts_b == 1) {
      num *= den == 0.f ? 0.f : 1.f / den;
      *reinterpret_cast<u32x2*>(a.out + bh * D + d) =
          u32x2{pack_bf16x2(num[0], num[1]), pack_bf16x2(num[2], num[3])};
      if (d == 0 && a.lse) a.lse[bh] = den == 0.f ? -INFINITY : (M + __log2f(den)) * kLn2;
    } else {
      *reinterpret_cast<f32x4*>(a.part_o + (bh * a.n_parts + part) * D + d) = num;
    }
    if (d == 0 && (WEIGHTED || n_parts_b > 1)) {
      const int64_t to = (bh * a.n_parts + part) * 2;
      a.part_ml[to] = M;
      a.part_ml[to + 1] = den;
    }
  });
}

constexpr int kKv4Depth = 2;  // pairs of blocks in registers

template <int D, bool RANKED, bool WEIGHTED>
void launch_kv4(const DecodeArgs& a, int B, unsigned grid, int W, hipStream_t s) {
  const int lds = join4_bytes<D>(W, a.group);
  if (W == 4)
    decode_kv4_kernel<D, kKv4Depth, RANKED, 4, WEIGHTED><<<grid, 4 * kWave, lds, s>>>(a, B);
  else if (W == 2)
    decode_kv4_kernel<D, kKv4Depth, RANKED, 2, WEIGHTED><<<grid, 2 * kWave, lds, s>>>(a, B);
  else
    decode_kv4_kernel<D, kKv4Depth, RANKED, 1, WEIGHTED><<<grid, kWave, 0, s>>>(a, B);
}

// Waves that share a partition, by units as for bf16, but later: a block takes a quarter
// of the time, so what a wave does before its first block weighs more. Measured in us
// with 1 / 2 / 4 waves, 8 KV heads of 4 query heads: 1024 units 27 / 21 / 19 (16 requests
// of up to 4000 tokens), 1200 28 / 22.5 / 21.6, 2112 34 / 31 / 33, 4224 37.8 / 36.7 / 38.6;
// one query head per KV head: 1024 20 / 15.8 / 15.2, 8192 61 / 64 / 71. Requests of one
// partition fill it in part only: 1024 units 16.4 / 15.2 / 18.8.
int kv4_waves(const DecodeArgs& a, int B) {
  const int64_t units = static_cast<int64_t>(a.Hkv) * B * a.n_parts;
  if (units < (a.n_parts > 1 ? 1536 : 512)) return 4;
  return units < (a.n_parts > 1 ? 5120 : 2048) ? 2 : 1;
}

// Whether units are dispatched longest first. Units that are about all resident at once
// need no order, and finding it takes a call of 4 requests 1 us of 6.7; 128 short requests,
// 4096 waves, 15.4 us with and 14.1 without, 16 of up to 4000 tokens, 4352 waves, 18.0 with
// and 18.7 without.
bool kv4_ranked(const DecodeArgs& a, int B) {
  const int64_t wgs = static_cast<int64_t>(a.Hkv) * B * (a.n_parts + 1);
  return B <= kRankChunks * kWave && wgs * kv4_waves(a, B) > 4096;
}

template <int D>
local_status_t launch_decode_kv4(const DecodeArgs& a, int B, hipStream_t s) {
  const int64_t wgs = static_cast<int64_t>(a.Hkv) * B * (a.n_parts + 1);
  const int64_t merge = merge_grid<D>(a, B);
  if (std::max(wgs, merge) >= (1LL << 31))
    return local_fail(LOCAL_ERR_UNSUPPORTED, "paged_attn_decode_kv4: grid of %lld workgroups",
                      (long long)std::max(wgs, merge));
  const int W = kv4_waves(a, B);
  const bool ranked = kv4_ranked(a, B);
  const unsigned grid =
      static_cast<unsigned>(a.Hkv) * B * static_cast<unsigned>(a.n_parts + (ranked ? 1 : 0));
  if (ranked)
    a.w_out ? launch_kv4<D, true, true>(a, B, grid, W, s)
            : launch_kv4<D, true, false>(a, B, grid, W, s);
  else
    a.w_out ? launch_kv4<D, false, true>(a, B, grid, W, s)
            : launch_kv4<D, false, false>(a, B, grid, W, s);
  if (a.w_out)
    decode_merge_kernel<D, true, true>
        <<<static_cast<unsigned>(merge), D, a.Hq * sizeof(float), s>>>(a, B);
  else if (a.n_parts > 1)
    decode_merge_kernel<D, true, false><<<static_cast<unsigned>(merge), D, 0, s>>>(a, B);
  return local_check_launch("paged_attn_decode_kv4");
}

}  // namespace
}  // namespace localk

using namespace localk;

extern "C" local_status_t local_paged_attn_decode_kv4(
    const uint16_t* q, int32_t B, int32_t Hq, int32_t Hkv, int32_t D,
    const uint16_t* k_new, const uint16_t* v_new, uint8_t* kv4, int64_t num_blocks,
    int32_t block_size, const int32_t* block_table, int32_t max_blocks,
    const int32_t* ctx_lens, const int32_t* block_version, const int32_t* req_version,
    float sm_scale, uint16_t* out, float* lse, const float* weight_in, float weight_decay,
    float* weight_out, void* ws, size_t* ws_bytes, void* stream) {
  const char* who = "paged_attn_decode_kv4";
  if (!ws_bytes) return local_fail(LOCAL_ERR_WORKSPACE, "%s: ws_bytes is NULL", who);
  if (B < 0 || Hq <= 0 || Hkv <= 0 || max_blocks < 1 || num_blocks < 1 || Hq % Hkv != 0)
    return local_fail(LOCAL_ERR_SHAPE, "%s: B=%d Hq=%d Hkv=%d max_blocks=%d num_blocks=%lld",
                      who, B, Hq, Hkv, max_blocks, (long long)num_blocks);
  if (block_size != kBlockSize || (D != 64 && D != 128) || Hq / Hkv > 16)
    return local_fail(LOCAL_ERR_UNSUPPORTED,
                      "%s: block_size=%d D=%d group=%d (need 16, 64|128, <=16)", who,
                      block_size, D, Hq / Hkv);
  if ((k_new == nullptr) != (v_new == nullptr))
    return local_fail(LOCAL_ERR_NULL, "%s: k_new and v_new must both be set", who);
  if (weight_in && !weight_out)
    return local_fail(LOCAL_ERR_NULL, "%s: weight_in without weight_out", who);
  local_status_t st = weight_out ? decode_weights_ok(Hq, weight_decay, who) : LOCAL_OK;
  if (st != LOCAL_OK) return st;
  DecodeArgs a{};
  a.q = q;
  a.k_new = k_new;
  a.v_new = v_new;
  a.kv4 = kv4;
  a.block_table = block_table;
  a.ctx_lens = ctx_lens;
  a.block_version = block_version;
  a.req_version = req_version;
  a.out = out;
  a.lse = lse;
  a.num_blocks = num_blocks;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.group = Hq / Hkv;
  a.max_blocks = max_blocks;
  const Scale4 scale = scale_of(sm_scale);
  a.scale_log2 = scale.log2;
  a.q_xor = scale.q_xor;
  a.q_and = scale.q_and;
  const DecodeParts part = decode_parts(a, B, D, true);
  // (the same with and without weights, so that one query serves both)
  const size_t need = align256(part.bytes) + block_lse_bytes(B, Hq, max_blocks);
  if (!ws) {
    *ws_bytes = need;
    return LOCAL_OK;
  }
  if (*ws_bytes < need)
    return local_fail(LOCAL_ERR_WORKSPACE, "%s: workspace %zu < %zu", who, *ws_bytes, need);
  if (B == 0) return LOCAL_OK;
  if (!q || !kv4 || !block_table || !ctx_lens || !block_version || !req_version || !out)
    return local_fail(LOCAL_ERR_NULL, "%s: NULL pointer argument", who);
  if (!aligned16(q) || !aligned16(kv4) || !aligned16(out) || !aligned16(k_new) ||
      !aligned16(v_new) || !aligned16(ws))
    return local_fail(LOCAL_ERR_UNSUPPORTED, "%s: q, k_new, v_new, kv4, out and ws must start "
                      "on 16 bytes", who);
  if ((st = decode_weights_apart(weight_in, weight_out, B, max_blocks, who)) != LOCAL_OK)
    return st;
  a.part_o = static_cast<float*>(ws);
  a.part_ml = a.part_o + part.elems * D;
  a.blk_lse = reinterpret_cast<float*>(static_cast<char*>(ws) + align256(part.bytes));
  a.w_in = weight_in;
  a.w_out = weight_out;
  a.w_decay = weight_decay;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return D == 64 ? launch_decode_kv4<64>(a, B, s) : launch_decode_kv4<128>(a, B, s);
}

// The partition length, the waves and the dispatch order that a call's size selects, as
// blocks + 256 x waves + 4096 if longest first (for the tests, which name the form that they
// mean; not in local.h).
extern "C" int32_t localk_decode_kv4_form(int32_t B, int32_t Hq, int32_t Hkv,
                                          int32_t max_blocks) {
  DecodeArgs a{};
  a.Hkv = Hkv;
  a.group = Hq / Hkv;
  a.max_blocks = max_blocks;
  decode_parts(a, B, 128, true);
  return a.pb + 256 * kv4_waves(a, B) + (kv4_ranked(a, B) ? 4096 : 0);
}
