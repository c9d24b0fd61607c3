// Pieces shared by the decode attention kernels of the bf16 and the 4-bit pool:
// partitions of the contexts, the dispatch order of their units and the merge of
// the partitions' results.
#pragma once

#include <algorithm>

#include "common.hpp"

namespace localk {
namespace {

// Blocks per partition, by the width of the block table: 32 up to 256 blocks,
// 48 up to 512, 64 beyond (at most 64: one bit per lane in the stale masks).
// Measured: the 32-layer decode with contexts up to 16K tokens (1024-block
// tables) is 3.2% faster a step with 64 than with 32, the GQA decode with
// 512-block tables 2% faster with 48, and the MHA decode with 256-block tables
// fastest with 32 (fewer, longer partitions: less merge traffic and fewer
// waves; shorter ones: more parallelism per request).
//
// A call with fewer than kFewUnits (KV head, request, partition) units leaves
// compute units idle or unevenly loaded, and halves the partitions until it
// has that many, down to 16 blocks and up to kMaxFine partitions a request
// (whose merge is a serial pass). Measured, 8 KV heads of 4 query heads:
// 5 requests of up to 15K tokens 55 us with 64 blocks and 36 with 32 (600 and
// 1200 units); 8 of up to 4000 tokens 31 us with 32 and 21 with 16; one of
// 16000 tokens (4 waves each) 22 us with 64, 17 with 32, 20 with 16 (62
// partitions).
constexpr int kFewUnits = 768;
constexpr int kMaxFine = 32;

int parts_of_table(int max_blocks, int pb) { return (max_blocks + pb - 1) / pb; }

int longest_part_blocks(int max_blocks) {
  return max_blocks <= 256 ? 32 : max_blocks <= 512 ? 48 : 64;
}

int part_blocks(int max_blocks, int64_t heads) {  // heads: B * Hkv
  int pb = longest_part_blocks(max_blocks);
  while (pb > 16 && heads * parts_of_table(max_blocks, pb) < kFewUnits) {
    const int half = pb == 64 ? 32 : 16;
    if (parts_of_table(max_blocks, half) > kMaxFine) break;
    pb = half;
  }
  return pb;
}

// Units that the partials are sized for at least, so that a call with fewer
// requests never asks for a larger workspace than one with more: halving (or a
// step from 48 to 16) starts below kFewUnits, so no fine call has more.
constexpr int64_t kFineUnits = 3 * kFewUnits;
constexpr float kNegBig = -1.0e30f;

struct DecodeArgs {
  const uint16_t* q;
  const uint16_t* k_new;
  const uint16_t* v_new;
  uint16_t* k_cache;
  uint16_t* v_cache;
  const int32_t* block_table;
  const int32_t* ctx_lens;
  const int32_t* block_version;
  const int32_t* req_version;
  uint16_t* out;
  float* lse;
  float* part_o;   // [B][Hq][n_parts][D]
  float* part_ml;  // [B][Hq][n_parts][2]  (max in log2 units, sum)
  // The version check of the same call (null when not asked for): per
  // (request, partition), the stale blocks as a bit mask (bit i = block
  // j0 + i) and the live tokens of the valid ones, written by KV head 0's
  // waves; the merge launch turns them into the canonical outputs.
  uint64_t* vc_mask;    // [B][n_parts]
  int32_t* vc_valid;    // [B][n_parts]
  int32_t* vc_pairs;    // [cap][2] (b, j), or null when cap == 0
  int64_t vc_cap;
  int32_t* vc_n_stale;  // one int32
  int32_t* vc_valid_tokens;  // [B]
  int64_t num_blocks;
  int Hq, Hkv, group, max_blocks, n_parts;
  int pb;            // blocks per partition (part_blocks of max_blocks)
  float scale_log2;  // sm_scale * log2(e)
  // Attention weight by block (null w_out when not asked for). blk_lse: per
  // (request, block, query head) the log2 of the sum of exp2(scores) over the
  // block's keys, -inf for a stale block; the merge launch turns it into weights
  // once it knows each head's sum over all blocks.
  float* blk_lse;  // [B][Hkv][max_blocks][group]
  const float* w_in;
  float* w_out;    // [B][max_blocks]
  float w_decay;
  uint8_t* kv4;    // the 4-bit pool, instead of k_cache and v_cache
  uint32_t q_xor, q_and;  // (4-bit pool) the sign of sm_scale on q's bits, or none of it
};

constexpr size_t align256(size_t v) { return (v + 255) & ~static_cast<size_t>(255); }

// Logical blocks request b owns: ceil(L/16), at most the table's width.
__device__ __forceinline__ int owned_blocks(int L, int max_blocks) {
  return L <= 0 ? 0 : min((L - 1) / kBlockSize + 1, max_blocks);  // (L may be INT_MAX)
}

// Set bits of m below this lane.
__device__ __forceinline__ int bits_below(uint64_t m) {
  return __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(m >> 32),
                                   __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(m), 0u));
}

// Full partitions of nb blocks (part_blocks is 16, 32, 48 or 64).
__device__ __forceinline__ int full_parts(int nb, int pb) {
  const unsigned u = static_cast<unsigned>(nb);
  return static_cast<int>(pb == 48 ? u / 48u : u >> (pb == 16 ? 4 : pb == 32 ? 5 : 6));
}

// Requests a wavefront ranks at once: 64 per register, up to this many
// registers (larger batches use the grid order below without ranking).
constexpr int kRankChunks = 8;

// The unit of work of dispatch slot k, longest first: every full partition,
// request by request (they are equally long), then each request's partial
// partition, longest first (ties: smaller b); an empty context is a partial
// partition of no block. Returns the request (-1 past the last unit) and, in
// *part, its partition index (a partial one is numbered n_full, as in the
// merge). Every lane returns the same.
//
// Every wave of every slot runs this before it knows what to load, so its
// instructions count (with 128 requests and 1000 units, 30 us of issue slots over
// the chip when the partial partitions were searched length by length and
// the k-th set bit by clearing k of them): the full partitions are found by
// prefix sums over the bits of n_full, the partial ones by a radix selection
// over the 6 bits of their length, all with ballots.
__device__ int decode_unit(const DecodeArgs& a, int B, int k, int* part) {
  const int lane = threadIdx.x % kWave;
  const int nc = (B + kWave - 1) / kWave;
  int nf[kRankChunks], rem[kRankChunks], pre[kRankChunks];
  uint64_t cand[kRankChunks];  // requests with a partial partition
#pragma unroll
  for (int c = 0; c < kRankChunks; ++c) {
    if (c >= nc) break;
    const int b = c * kWave + lane;
    rem[c] = b < B ? a.ctx_lens[b] : -1;
  }
  int n_partial = 0;
#pragma unroll
  for (int c = 0; c < kRankChunks; ++c) {
    if (c >= nc) break;
    const bool in = c * kWave + lane < B;
    const int nb = in ? owned_blocks(rem[c], a.max_blocks) : 0;
    nf[c] = full_parts(nb, a.pb);
    rem[c] = nb - nf[c] * a.pb;
    cand[c] = __ballot(in && (nb == 0 || rem[c] > 0));
    n_partial += __popcll(cand[c]);
  }
  // exclusive prefix sums of n_full over the requests, bit by bit
  int full = 0;
#pragma unroll
  for (int c = 0; c < kRankChunks; ++c) {
    if (c >= nc) break;
    pre[c] = full;
    for (int bit = 0; (1 << bit) <= a.n_parts; ++bit) {
      const uint64_t m = __ballot((nf[c] >> bit) & 1);
      pre[c] += bits_below(m) << bit;
      full += __popcll(m) << bit;
    }
  }
  if (k >= full + n_partial) return -1;
  if (k < full) {
#pragma unroll
    for (int c = 0; c < kRankChunks; ++c) {
      if (c >= nc) break;
      const uint64_t m = __ballot(k >= pre[c] && k < pre[c] + nf[c]);
      if (m) {
        const int l = __builtin_ctzll(m);
        *part = k - __builtin_amdgcn_readlane(pre[c], l);
        return c * kWave + l;
      }
    }
  }
  k -= full;
  for (int bit = 5; bit >= 0; --bit) {  // (a partial partition has at most 63 blocks)
    int longer = 0;
#pragma unroll
    for (int c = 0; c < kRankChunks; ++c) {
      if (c >= nc) break;
      longer += __popcll(cand[c] & __ballot((rem[c] >> bit) & 1));
    }
    const bool take = k < longer;
    if (!take) k -= longer;
#pragma unroll
    for (int c = 0; c < kRankChunks; ++c) {
      if (c >= nc) break;
      const uint64_t m = __ballot((rem[c] >> bit) & 1);
      cand[c] &= take ? m : ~m;
    }
  }
#pragma unroll
  for (int c = 0; c < kRankChunks; ++c) {
    if (c >= nc) break;
    const int n = __popcll(cand[c]);
    if (k < n) {
      const bool mine = (cand[c] >> lane & 1ull) && bits_below(cand[c]) == k;
      const int l = __builtin_ctzll(__ballot(mine));
      *part = __builtin_amdgcn_readlane(nf[c], l);
      return c * kWave + l;
    }
    k -= n;
  }
  return -1;
}

// Bytes of LDS a workgroup of W > 1 waves merges its waves' results in: per
// (wave, column) an unnormalised O row (padded by 16 bytes, so that the columns
// a wave writes together fall in distinct banks), its maximum and its sum.
template <int D>
constexpr int merge_lds_bytes(int W, int group) {
  return W * group * (D + 4 + 2) * static_cast<int>(sizeof(float));
}

// Merge the partitions of every (request, head) that has more than one.
// The version check from the partitions' stale masks (one workgroup per
// request, D threads): the request's offset in the canonical list is the
// number of stale blocks of the requests before it; its own stale blocks
// follow in ascending j (partitions in descending index). Deterministic, no
// atomics.
__device__ void decode_version_check(const DecodeArgs& a, int b, int B, int* sh) {
  const int tid = threadIdx.x, nt = blockDim.x;
  auto parts_of = [&](int bb) {
    const int nbb = owned_blocks(a.ctx_lens[bb], a.max_blocks);
    return max(1, full_parts(nbb + a.pb - 1, a.pb));
  };
  int before = 0;
  for (int e = tid; e < b * a.n_parts; e += nt) {
    const int bb = e / a.n_parts, pp = e % a.n_parts;
    if (pp < parts_of(bb)) before += __popcll(a.vc_mask[e]);
  }
  const int np = parts_of(b);
  // this request's partitions in ascending j: t-th is partition np - 1 - t
  int cnt = 0, valid = 0;
  uint64_t mask = 0ull;
  if (tid < np) {
    const int64_t slot = static_cast<int64_t>(b) * a.n_parts + (np - 1 - tid);
    mask = a.vc_mask[slot];
    cnt = __popcll(mask);
    valid = a.vc_valid[slot];
  }
  // block-wide sums of `before` and `valid`, exclusive prefix of `cnt` over t
  sh[tid] = cnt;
  __syncthreads();
  int pre = 0;
  for (int t = 0; t < tid && t < np; ++t) pre += sh[t];
  __syncthreads();
  sh[tid] = before;
  __syncthreads();
  for (int w = nt / 2; w > 0; w >>= 1) {
    if (tid < w) sh[tid] += sh[tid + w];
    __syncthreads();
  }
  const int offset = sh[0];
  __syncthreads();
  sh[tid] = valid;
  __syncthreads();
  for (int w = nt / 2; w > 0; w >>= 1) {
    if (tid < w) sh[tid] += sh[tid + w];
    __syncthreads();
  }
  if (tid == 0) a.vc_valid_tokens[b] = sh[0];
  if (tid < np) {  // (np <= n_parts <= nt: the host checks)
    const int nbb = owned_blocks(a.ctx_lens[b], a.max_blocks);
    const int p = np - 1 - tid;
    const int j0 = max(0, nbb - a.pb * (p + 1));
    int64_t pos = static_cast<int64_t>(offset) + pre;
    for (uint64_t m = mask; m; m &= m - 1ull, ++pos) {
      if (pos < a.vc_cap) {
        a.vc_pairs[2 * pos] = b;
        a.vc_pairs[2 * pos + 1] = j0 + __ffsll(static_cast<long long>(m)) - 1;
      }
    }
    if (b == B - 1 && tid == np - 1) *a.vc_n_stale = offset + pre + cnt;
  }
}

// Where block j of request b, KV head g, records its heads' weights.
__device__ __forceinline__ float* blk_lse_at(const DecodeArgs& a, int b, int g, int j) {
  return a.blk_lse + ((static_cast<int64_t>(b) * a.Hkv + g) * a.max_blocks + j) * a.group;
}

// Attention weight of D blocks of one request: w_out = decay * w_in + the sum over
// the query heads of exp2(blk_lse - lse), with each head's lse over all blocks
// taken from the partitions' sums again (a few KB from L2) rather than from the
// workgroups that merge them, which run in the same launch. Blocks past the
// context's end get 0. One thread adds a block's heads in order: no atomics.
template <int D>
__device__ void decode_block_weights(const DecodeArgs& a, int unit, float* lse2) {
  const int chunks = (a.max_blocks + D - 1) / D;
  const int b = unit / chunks, j = unit % chunks * D + static_cast<int>(threadIdx.x);
  const int nb = owned_blocks(a.ctx_lens[b], a.max_blocks);
  const int np = max(1, full_parts(nb + a.pb - 1, a.pb));
  // The block's own values first: they need no sum, and their loads run beside those of
  // the partitions' sums.
  constexpr int kAhead = 8;  // groups of 4 heads read ahead
  const int64_t at = static_cast<int64_t>(b) * a.max_blocks + j;
  const bool mine = j < nb, fours = a.group % 4 == 0;
  auto values = [&](int q) {  // heads 4 q ..
    const int per = a.group / 4;
    return *reinterpret_cast<const f32x4*>(blk_lse_at(a, b, q / per, j) + q % per * 4);
  };
  f32x4 ahead[kAhead];
  if (mine && fours) {
#pragma unroll
    for (int q = 0; q < kAhead; ++q)
      if (4 * q < a.Hq) ahead[q] = values(q);
  }
  const float old = mine && a.w_in ? a.w_in[at] : 0.f;
  if (unit % chunks * D < nb) {
    constexpr int kPer = 4, kBatch = 4;  // lanes that share a head's partitions
    const int p0 = threadIdx.x % kPer;
    for (int h0 = 0; h0 < a.Hq; h0 += D / kPer) {
      const int h = min(h0 + static_cast<int>(threadIdx.x) / kPer, a.Hq - 1);
      const float2* ml = reinterpret_cast<const float2*>(
          a.part_ml + (static_cast<int64_t>(b) * a.Hq + h) * a.n_parts * 2);
      float M = kNegBig, den = 0.f;
      for (int p = p0; p < np; p += kPer * kBatch) {
        float2 v[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
          v[i] = p + kPer * i < np ? ml[p + kPer * i] : float2{kNegBig, 0.f};
        float top = M;
#pragma unroll
        for (int i = 0; i < kBatch; ++i) top = fmaxf(top, v[i].x);
        den *= fast_exp2(M - top);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) den += v[i].y * fast_exp2(v[i].x - top);
        M = top;
      }
      float top = fmaxf(M, __shfl_xor(M, 1));
      top = fmaxf(top, __shfl_xor(top, 2));
      den *= fast_exp2(M - top);
      den += __shfl_xor(den, 1);
      den += __shfl_xor(den, 2);
      // (no valid key: every blk_lse is -inf)
      if (p0 == 0) lse2[h] = den == 0.f ? 0.f : top + __log2f(den);
    }
  }
  __syncthreads();
  if (j >= a.max_blocks) return;
  float w = 0.f;
  if (mine) {
    if (fours) {
      for (int q0 = 0; 4 * q0 < a.Hq; q0 += kAhead) {
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
          if (4 * (q0 + q) >= a.Hq) break;
          const f32x4 v = q0 == 0 ? ahead[q] : values(q0 + q);
#pragma unroll
          for (int i = 0; i < 4; ++i) w += fast_exp2(v[i] - lse2[4 * (q0 + q) + i]);
        }
      }
    } else {
      for (int h = 0; h < a.Hq; ++h)
        w += fast_exp2(blk_lse_at(a, b, h / a.group, j)[h % a.group] - lse2[h]);
    }
    if (a.w_in) w = fmaf(a.w_decay, old, w);
  }
  a.w_out[at] = w;
}

// Workgroups of the merge launch: one for each (request, query head), then with
// weights one for each D blocks of a request's table row.
template <int D>
int64_t merge_grid(const DecodeArgs& a, int B) {
  const int64_t chunks = a.w_out ? (a.max_blocks + D - 1) / D : 0;
  return static_cast<int64_t>(B) * (a.Hq + chunks);
}

// NANS: a NaN among the sums reaches the outputs (the 4-bit pool stores them on
// purpose). WEIGHTED: the launch has the workgroups of the block weights (and Hq
// floats of LDS).
template <int D, bool NANS, bool WEIGHTED>
__global__ __launch_bounds__(D) void decode_merge_kernel(DecodeArgs a, int B) {
  if constexpr (WEIGHTED) {
    extern __shared__ float merge_lse2[];
    if (blockIdx.x >= static_cast<unsigned>(B * a.Hq)) {
      decode_block_weights<D>(a, blockIdx.x - B * a.Hq, merge_lse2);
      return;
    }
  }
  const int bh = blockIdx.x;
  const int b = bh / a.Hq;
  const int d = threadIdx.x;
  if (a.vc_mask && bh % a.Hq == 0) {
    __shared__ int sh[D];
    decode_version_check(a, b, B, sh);
  }
  const int L = a.ctx_lens[b];
  const int nb = owned_blocks(L, a.max_blocks);
  const int np = max(1, full_parts(nb + a.pb - 1, a.pb));
  if (np == 1) return;  // written by the main kernel
  // one pass over the partitions, 8 at a time (16 of the 4-bit pool's, whose calls are
  // shorter) with all their loads in flight; the running sums are rescaled when a batch
  // raises the maximum
  constexpr int kMergeBatch = NANS ? 16 : 8;
  const float* ml = a.part_ml + static_cast<int64_t>(bh) * a.n_parts * 2;
  const float* po = a.part_o + static_cast<int64_t>(bh) * a.n_parts * D;
  float M = kNegBig, den = 0.f, num = 0.f;
  for (int p0 = 0; p0 < np; p0 += kMergeBatch) {
    float2 mlv[kMergeBatch];
    float ov[kMergeBatch];
#pragma unroll
    for (int q = 0; q < kMergeBatch; ++q) {
      const bool in = p0 + q < np;
      mlv[q] = in ? *reinterpret_cast<const float2*>(ml + 2 * (p0 + q)) : float2{kNegBig, 0.f};
      ov[q] = in ? po[static_cast<int64_t>(p0 + q) * D + d] : 0.f;
    }
    float Mb = M;
#pragma unroll
    for (int q = 0; q < kMergeBatch; ++q) Mb = fmaxf(Mb, mlv[q].x);
    const float c = fast_exp2(M - Mb);
    den *= c;
    num *= c;
#pragma unroll
    for (int q = 0; q < kMergeBatch; ++q) {
      const float f = fast_exp2(mlv[q].x - Mb);
      den += mlv[q].y * f;
      num += ov[q] * f;
    }
    M = Mb;
  }
  const bool some = NANS ? den != 0.f : den > 0.f;
  a.out[static_cast<int64_t>(bh) * D + d] = f32_to_bf16(some ? num / den : 0.f);
  if (d == 0 && a.lse) a.lse[bh] = some ? (M + __log2f(den)) * kLn2 : -INFINITY;
}

// Host checks and workspace of the block weights.
inline local_status_t decode_weights_ok(int Hq, float decay, const char* who) {
  if (!(decay >= 0.f && decay <= 1.f))
    return local_fail(LOCAL_ERR_UNSUPPORTED, "%s: weight_decay=%g (need 0 <= decay <= 1)", who,
                      static_cast<double>(decay));
  if (Hq > 8192)  // (one float of LDS each in the merge launch)
    return local_fail(LOCAL_ERR_UNSUPPORTED, "%s: Hq=%d (need <= 8192)", who, Hq);
  return LOCAL_OK;
}

// weight_out is weight_in itself (a thread reads and writes the same element) or apart.
inline local_status_t decode_weights_apart(const float* in, const float* out, int B,
                                           int max_blocks, const char* who) {
  const size_t bytes = static_cast<size_t>(B) * max_blocks * sizeof(float);
  if (in && in != out && overlap(in, bytes, out, bytes))
    return local_fail(LOCAL_ERR_SHAPE, "%s: weight_out overlaps weight_in in part", who);
  return LOCAL_OK;
}

inline size_t block_lse_bytes(int B, int Hq, int max_blocks) {
  return align256(static_cast<size_t>(B > 0 ? B : 1) * Hq * max_blocks * sizeof(float));
}

// Split-KV partials of a call: the partition length (a->pb, a->n_parts) and what
// the partials take.
struct DecodeParts {
  size_t elems, bytes;  // (request, query head, partition) triples; their bytes
  size_t units;         // (request, partition) pairs of the version masks
};

// fine: the partitions that the call's size asks for, with room for any call of
// fewer requests; else the longest ones of its table and exactly their partials,
// for a workspace that has no room for more.
inline DecodeParts decode_parts(DecodeArgs& a, int B, int D, bool fine) {
  a.pb = fine ? part_blocks(a.max_blocks, static_cast<int64_t>(B) * a.Hkv)
              : longest_part_blocks(a.max_blocks);
  a.n_parts = parts_of_table(a.max_blocks, a.pb);
  DecodeParts p;
  p.units = static_cast<size_t>(B > 0 ? B : 1) * a.n_parts;
  p.elems = p.units * a.Hq;
  if (fine) {
    p.units = std::max(p.units, static_cast<size_t>(kFineUnits));
    p.elems = std::max(p.elems, static_cast<size_t>(kFineUnits) * a.group);
  }
  p.bytes = p.elems * (D + 2) * sizeof(float);
  return p;
}

}  // namespace
}  // namespace localk
