// local_paged_attn_prefill_kv4: a chunk of new tokens per request is put into the
// 4-bit pool, then attends causally over cached prefix plus chunk.
//
// Mathematics: as prefill attention over the bf16 pool, with K^ and V^ the values that
// the codes stand for (the chunk's own tokens too); those are exact in bf16.
//
// Bound by the matrix cores and the softmax's vector instructions; the pool's 4-bit
// tiles make the memory side four times lighter than bf16, at the price of unpacking.
//  * Append: a wave per (block of a request's chunk, KV head) rounds up to 16 tokens and
//    writes them as the whole tile that they mostly are. One more workgroup of that
//    launch plans the attention: it knows every tile's keys, splits the long ones into
//    key ranges where a call has too few tiles to fill the chip, and orders the units
//    longest first.
//  * A workgroup takes 128 rows of one request and one KV head, a row being a (token,
//    query head of the group): every query head of the group shares what is unpacked.
//    8 waves: two halves of 4 waves of 32 rows, which take the steps of 64 keys in
//    turn and join their results in LDS at the end. (4 waves with every step ran the
//    same work, but a unit then takes twice as long, and the longest sets the end.)
//  * Each wave of a half unpacks one of a step's four blocks into LDS, in the order of
//    the matrix operands (lane l's 16 bytes at 16 l), so that operand reads are
//    contiguous kilobytes. Two buffers a half: the codes of the step after next load
//    into registers while the next is unpacked and this one computed; one barrier.
//  * S^T = K Q^T, O^T += V^T P^T on v_mfma_f32_16x16x32_bf16, as in decode, and as
//    there the running maximum rises only when a weight would pass 2^8.
//  * An infinity or a NaN in V (scale byte 255) must reach the rows that see its token
//    and no other, which 0 * NaN in a product would not do: its values enter the
//    product as zeros, and a mask of such tokens then puts NaN into those rows.
#include <algorithm>
#include <climits>

#include "kv4.hpp"

namespace localk {
namespace {

constexpr int kP4Waves = 4;                            // of a half
constexpr int kP4Halves = 2;
constexpr int kP4Threads = kP4Halves * kP4Waves * kWave;
constexpr int kP4RowTiles = 2;                         // 16-row tiles of a wave
constexpr int kP4Rows = kP4Waves * 16 * kP4RowTiles;   // rows of a workgroup
constexpr int kP4Step = 4;                             // blocks a step
constexpr int kP4Window = kP4Threads;                  // table entries listed at a time
constexpr int kP4MinRange = 8;                         // blocks a key range has at least
constexpr int kP4MaxRanges = 16;
constexpr int kP4Units = 256;                          // a workgroup for every compute unit
constexpr int kApThreads = 256;                        // of the append launch
constexpr int kApWaves = kApThreads / kWave;
constexpr float kP4NegBig = -1.0e30f;
constexpr float kP4Lazy = 8.f;  // log2 of the largest weight before the maximum rises

struct Prefill4Args {
  const uint16_t* q;
  const int32_t* q_indptr;
  const uint16_t* k_new;
  const uint16_t* v_new;
  uint8_t* kv4;
  const int32_t* block_table;
  const int32_t* ctx_lens;
  const int32_t* block_version;
  const int32_t* req_version;
  uint16_t* out;
  float* lse;
  // workspace
  int* counts;     // units of the plan, tiles
  int4* plan;      // units, longest first: request, tile, range, ranges of the tile
  int4* tiles;     // request, tile, blocks that its last row sees, ranges
  float* part_o;   // [T][Hq][ranges][D]
  float* part_ml;  // [T][Hq][ranges][2]
  int64_t T, num_blocks;
  int B, Hq, Hkv, group, max_blocks;
  int ranges;      // the most a tile may be split into
  int max_tiles;   // tiles that the plan has room for
  float scale_log2;
  uint32_t q_xor, q_and;
};

__device__ __forceinline__ bool rows_ok4(int r0, int r1, int64_t T) {
  return r0 >= 0 && r1 >= r0 && r1 <= T;
}

// What a workgroup has to know of its tile of 128 rows.
struct Tile4 {
  int b, r0, row0, rows;   // request, its first token, first row of the tile, its rows
  int prefix;              // cached tokens before the chunk
  int blocks;              // blocks that the tile's last row sees
};

__device__ __forceinline__ Tile4 tile_of(const Prefill4Args& a, int b, int tile) {
  Tile4 t;
  t.b = b;
  t.r0 = a.q_indptr[b];
  const int n = a.q_indptr[b + 1] - t.r0, L = a.ctx_lens[b];
  t.row0 = tile * kP4Rows;
  t.rows = min(kP4Rows, n * a.group - t.row0);
  t.prefix = L - n;
  const int last = t.prefix + (t.row0 + t.rows - 1) / a.group;  // its position
  t.blocks = last < 0 ? 0 : min(last / kBlockSize + 1, a.max_blocks);
  return t;
}

// Inclusive prefix sum over the append launch's workgroup.
__device__ __forceinline__ int scan_ap(int v, int* wave_sums) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const int up = __shfl_up(v, off);
    if (lane >= off) v += up;
  }
  __syncthreads();  // (the sums of the call before have been read)
  if (lane == kWave - 1) wave_sums[wave] = v;
  __syncthreads();
  for (int w = 0; w < wave; ++w) v += wave_sums[w];
  return v;
}

// ---------------------------------------------------------------- plan
// One workgroup. Units are ordered by a counting sort of their lengths in 256 steps
// (the order among equals does not matter to any result).
__device__ void plan_kv4(const Prefill4Args& a) {
  __shared__ int first[kApThreads + 1], wave_sums[kApWaves], hist[256], longest;
  __shared__ unsigned long long work;
  const int tid = threadIdx.x;
  int n_tiles = 0;
  if (tid == 0) work = 0ull, longest = 1;
  for (int b0 = 0; b0 < a.B; b0 += kApThreads) {
    int n = 0;
    if (b0 + tid < a.B) {
      const int r0 = a.q_indptr[b0 + tid], r1 = a.q_indptr[b0 + tid + 1];
      if (rows_ok4(r0, r1, a.T)) n = ((r1 - r0) * a.group + kP4Rows - 1) / kP4Rows;
    }
    const int incl = scan_ap(n, wave_sums);
    first[tid + 1] = incl;
    if (tid == 0) first[0] = 0;
    __syncthreads();
    const int all = first[kApThreads];
    // (a plan is sized for row ranges that do not overlap)
    for (int t = tid; t < all && n_tiles + t < a.max_tiles; t += kApThreads) {
      int lo = 0, hi = kApThreads;
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (first[mid] <= t)
          lo = mid;
        else
          hi = mid;
      }
      const int tile = t - first[lo], blocks = tile_of(a, b0 + lo, tile).blocks;
      a.tiles[n_tiles + t] = int4{b0 + lo, tile, blocks, 1};
      atomicAdd(&work, static_cast<unsigned long long>(blocks));
      atomicMax(&longest, blocks);
    }
    n_tiles = min(n_tiles + all, a.max_tiles);
    __syncthreads();
  }
  // No unit longer than a compute unit's share of the work.
  hist[tid] = 0;
  __syncthreads();
  const int64_t share = (static_cast<int64_t>(work) * a.Hkv + kP4Units - 1) / kP4Units;
  auto ranges_of = [&](int blocks) {
    const int64_t want = (blocks + share - 1) / max(share, static_cast<int64_t>(1));
    const int most = min(a.ranges, blocks / kP4MinRange);
    return static_cast<int>(max(static_cast<int64_t>(1), min(want, static_cast<int64_t>(most))));
  };
  auto bucket = [&](int blocks, int n) {
    return 255 - static_cast<int>(static_cast<int64_t>(blocks) * 255 /
                                  (static_cast<int64_t>(longest) * n));
  };
  // (tile t of a.tiles is read by the thread that wrote it or after a barrier)
  for (int t = tid; t < n_tiles; t += kApThreads) {
    const int blocks = a.tiles[t].z, n = ranges_of(blocks);
    atomicAdd(&hist[bucket(blocks, n)], n);
  }
  __syncthreads();
  const int mine = hist[tid], incl = scan_ap(mine, wave_sums);
  if (tid == kApThreads - 1) {
    a.counts[0] = incl;
    a.counts[1] = n_tiles;
  }
  hist[tid] = incl - mine;
  __syncthreads();
  for (int t = tid; t < n_tiles; t += kApThreads) {
    const int4 e = a.tiles[t];
    const int n = ranges_of(e.z);
    a.tiles[t].w = n;
    const int at = atomicAdd(&hist[bucket(e.z, n)], n);
    for (int r = 0; r < n; ++r) a.plan[at + r] = int4{e.x, e.y, r, n};
  }
}

// ---------------------------------------------------------------- append
// The k-th block of new tokens: requests in order. Every lane returns the same; false
// past the last.
__device__ bool find_new_block(const Prefill4Args& a, int64_t k, int* b, int* j) {
  const int lane = threadIdx.x % kWave;
  for (int b0 = 0; b0 < a.B; b0 += kWave) {
    int n = 0, j0 = 0;
    if (b0 + lane < a.B) {
      const int r0 = a.q_indptr[b0 + lane], r1 = a.q_indptr[b0 + lane + 1];
      const int L = a.ctx_lens[b0 + lane];
      if (rows_ok4(r0, r1, a.T) && r1 > r0 && L > 0) {
        j0 = max(L - (r1 - r0), 0) / kBlockSize;
        n = min((L - 1) / kBlockSize + 1, a.max_blocks) - j0;
        n = max(n, 0);
      }
    }
    int incl = n;
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
      const int up = __shfl_up(incl, off);
      if (lane >= off) incl += up;
    }
    const uint64_t past = __ballot(incl > k);
    if (past) {
      const int l = __builtin_ctzll(past);
      *b = b0 + l;
      *j = __shfl(j0, l) + static_cast<int>(k) - (__shfl(incl, l) - __shfl(n, l));
      return true;
    }
    k -= __shfl(incl, kWave - 1);
  }
  return false;
}

template <int D>
__global__ __launch_bounds__(kApThreads) void append_kv4_kernel(Prefill4Args a) {
  using L4 = Kv4<D>;
  constexpr int VT = D / 16;
  if (blockIdx.x == 0) {
    plan_kv4(a);
    return;
  }
  const int64_t unit =
      (static_cast<int64_t>(blockIdx.x) - 1) * kApWaves + threadIdx.x / kWave;
  const int lane = threadIdx.x % kWave, col = lane % 16, kgrp = lane / 16;
  const int g = static_cast<int>(unit % a.Hkv);
  int b, j;
  if (!find_new_block(a, unit / a.Hkv, &b, &j)) return;
  const int p = a.block_table[static_cast<int64_t>(b) * a.max_blocks + j];
  if (p < 0 || p >= a.num_blocks) return;
  const int r0 = a.q_indptr[b], n = a.q_indptr[b + 1] - r0;
  const int first = a.ctx_lens[b] - n;  // position of the chunk's first token
  // Slot s of the block is token row s + off of the chunk where that is one of its n.
  const int off = j * kBlockSize - first;
  auto fresh = [&](int slot) { return slot + off >= 0 && slot + off < n; };
  auto row = [&](int slot) {
    return (static_cast<int64_t>(r0 + slot + off) * a.Hkv + g) * D;
  };
  uint8_t* o = a.kv4 + (static_cast<int64_t>(p) * a.Hkv + g) * L4::kTile;
  // K: slot col, dims (D/4) kgrp ..; V: slots 4 kgrp .., dims VT col ..
  u32x4 kv[D / 32];
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    kv[c] = u32x4{0u, 0u, 0u, 0u};
    if (fresh(col)) kv[c] = ld_global<u32x4>(a.k_new + row(col) + (D / 4) * kgrp + 8 * c);
  }
  u32x4 vv[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    vv[e] = u32x4{0u, 0u, 0u, 0u};
    if (fresh(4 * kgrp + e)) {
      const uint16_t* from = a.v_new + row(4 * kgrp + e) + VT * col;
      if constexpr (D == 128) {
        vv[e] = ld_global<u32x4>(from);
      } else {
        const u32x2 w = ld_global<u32x2>(from);
        vv[e] = u32x4{w.x, w.y, 0u, 0u};
      }
    }
  }
  uint32_t code[D / 32], vcode[4], vs[4];
  const uint32_t ks = round_k<D>(kv, code);
#pragma unroll
  for (int e = 0; e < 4; ++e) vs[e] = round_v<D>(vv[e], vcode[e]);
  if (fresh(col)) {
    uint32_t* to = reinterpret_cast<uint32_t*>(o + lane * L4::kLane);
#pragma unroll
    for (int c = 0; c < D / 32; ++c) to[c] = code[c];
    if (D == 128 || kgrp % 2 == 0)
      o[L4::k_scale(L4::k_group(kgrp), col)] = static_cast<uint8_t>(ks);
  }
  uint8_t* vo = o + L4::kV + lane * L4::kLane;
  const bool head = col % (16 / L4::kGroups) == 0;
  if (fresh(4 * kgrp) && fresh(4 * kgrp + 3)) {  // the lane's four slots at once
    if constexpr (D == 128)
      *reinterpret_cast<u32x4*>(vo) = u32x4{vcode[0], vcode[1], vcode[2], vcode[3]};
    else
      *reinterpret_cast<u32x2*>(vo) = u32x2{(vcode[0] & 0xffffu) | vcode[1] << 16,
                                            (vcode[2] & 0xffffu) | vcode[3] << 16};
    if (head)
      *reinterpret_cast<uint32_t*>(o + L4::v_scale(L4::v_group(col), 4 * kgrp)) =
          vs[0] | vs[1] << 8 | vs[2] << 16 | vs[3] << 24;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (!fresh(4 * kgrp + e)) continue;
      if constexpr (D == 128)
        reinterpret_cast<uint32_t*>(vo)[e] = vcode[e];
      else
        reinterpret_cast<uint16_t*>(vo)[e] = static_cast<uint16_t>(vcode[e]);
      if (head)
        o[L4::v_scale(L4::v_group(col), 4 * kgrp + e)] = static_cast<uint8_t>(vs[e]);
    }
  }
}

__global__ __launch_bounds__(kApThreads) void plan_kv4_kernel(Prefill4Args a) { plan_kv4(a); }

// ---------------------------------------------------------------- attention
template <int D>
struct Codes4 {  // the block that a wave unpacks, as loaded
  uint32_t k[D / 32], v[D / 32];
  uint32_t ks, vs;
};

template <int D>
__device__ __forceinline__ void load_cached(__amdgpu_buffer_rsrc_t r, uint32_t off,
                                            uint32_t (&c)[D / 32]) {
  if constexpr (D == 128) {
    const u32x4 v = buf_load16(r, off);
    c[0] = v.x, c[1] = v.y, c[2] = v.z, c[3] = v.w;
  } else {
    const u32x2 v = buf_load8(r, off);
    c[0] = v.x, c[1] = v.y;
  }
}

template <int D>
struct Stage4 {  // one step's operands in LDS
  u32x4 k[kP4Step][D / 32][kWave];
  u32x2 v[kP4Step / 2][D / 16][kWave][2];  // by (pair, tile, lane): of either block
  uint32_t nan[kP4Step][4];  // by (block, group): tokens whose V is not finite
};

template <int D>
__global__ __launch_bounds__(kP4Threads, 2) void prefill_kv4_kernel(Prefill4Args a) {
  using L4 = Kv4<D>;
  constexpr int KC = D / 32, VT = D / 16, RT = kP4RowTiles;
  __shared__ Stage4<D> stage[kP4Halves][2];
  __shared__ __attribute__((aligned(16))) int list_id[kP4Window + 2 * kP4Step],
      list_j[kP4Window + 2 * kP4Step];
  __shared__ int wave_n[kP4Halves * kP4Waves];
  static_assert(sizeof(stage) >= kP4Rows * (D + 4 + 2) * sizeof(float), "joins in the stages");

  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave_all = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int wave = wave_all % kP4Waves, half = wave_all / kP4Waves;
  const int col = lane % 16, kgrp = lane / 16;
  const int g = blockIdx.x % a.Hkv;
  const int slot = blockIdx.x / a.Hkv;
  if (slot >= a.counts[0]) return;
  const int4 unit = a.plan[slot];
  const int b = unit.x, range = unit.z, n_ranges = unit.w;
  const Tile4 tl = tile_of(a, b, unit.y);
  const int lo = static_cast<int>(static_cast<int64_t>(tl.blocks) * range / n_ranges);
  const int hi = static_cast<int>(static_cast<int64_t>(tl.blocks) * (range + 1) / n_ranges);
  const int L = a.ctx_lens[b], rv = a.req_version[b];
  const int32_t* table = a.block_table + static_cast<int64_t>(b) * a.max_blocks;

  // This wave's rows: column col of row tile r is row 32 wave + 16 r + col of the tile.
  int pos[RT];        // its position, -1 for none
  int64_t qrow[RT];   // token * Hq + head
  bf16x8 qv[RT][KC];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int row = 16 * RT * wave + 16 * r + col;
    const bool in = row < tl.rows;
    const int at = tl.row0 + (in ? row : 0);
    const int i = at / a.group;
    pos[r] = in ? tl.prefix + i : -1;
    qrow[r] = static_cast<int64_t>(tl.r0 + i) * a.Hq + g * a.group + at % a.group;
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      u32x4 v = {0u, 0u, 0u, 0u};
      if (in) v = ld_global<u32x4>(a.q + qrow[r] * D + (D / 4) * kgrp + 8 * c);
      qv[r][c] = as_bf16x8((v ^ a.q_xor) & a.q_and);
    }
  }
  // Positions of the wave's first and last row: bounds of what it may see.
  const int wrow = tl.row0 + 16 * RT * wave;
  const bool wave_in = 16 * RT * wave < tl.rows, wave_full = 16 * RT * (wave + 1) <= tl.rows;
  const int first_pos = tl.prefix + wrow / a.group;
  const int last_pos =
      wave_in ? tl.prefix + (min(wrow + 16 * RT, tl.row0 + tl.rows) - 1) / a.group : -1;

  f32x4 acc[RT][VT];
  float m_run[RT], l_run[RT], rise[RT];
  const float inv_scale = 1.f / a.scale_log2;
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    m_run[r] = kP4NegBig;
    l_run[r] = 0.f;
    rise[r] = (kP4NegBig + kP4Lazy) * inv_scale;
#pragma unroll
    for (int t = 0; t < VT; ++t) acc[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // This wave unpacks block `wave` of its half's steps.
  auto load = [&](Codes4<D>& c, int s) {
    const int id = __builtin_amdgcn_readfirstlane(list_id[kP4Step * s + wave]);
    const int64_t tile = (static_cast<int64_t>(max(id, 0)) * a.Hkv + g) * L4::kTile;
    const __amdgpu_buffer_rsrc_t r = make_rsrc(a.kv4 + tile, id >= 0 ? L4::kTile : 0u);
    load_cached<D>(r, lane * L4::kLane, c.k);
    load_cached<D>(r, L4::kV + lane * L4::kLane, c.v);
    c.ks = __builtin_amdgcn_raw_buffer_load_b8(r, L4::k_scale(L4::k_group(kgrp), col), 0, 0);
    c.vs = __builtin_amdgcn_raw_buffer_load_b32(r, L4::v_scale(L4::v_group(col), 4 * kgrp), 0, 0);
  };
  auto unpack = [&](Codes4<D>& c, Stage4<D>& st, int s) {
    const float ks = scale4(c.ks);
#pragma unroll
    for (int i = 0; i < KC; ++i)
      st.k[wave][i][lane] = u32x4{unpack4<0>(c.k[i], ks), unpack4<1>(c.k[i], ks),
                                  unpack4<2>(c.k[i], ks), unpack4<3>(c.k[i], ks)};
    // V: slots past the context's end, and tokens that are not finite, as zeros
    const int j = __builtin_amdgcn_readfirstlane(list_j[kP4Step * s + wave]);
    const bool last = L - j * kBlockSize < kBlockSize;
    // (a byte of 255 is a zero byte of the complement)
    const bool bad = ((~c.vs - 0x01010101u) & c.vs & 0x80808080u) != 0u;
    uint32_t odd = 0u;
    if (last || __ballot(bad)) {
      const int live = L - j * kBlockSize - 4 * kgrp;  // (no block: far below 0)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t byte = 0xffu << (8 * i);
        const bool dead = i >= live, is = (c.vs & byte) == byte;
        if (is && !dead) odd |= 1u << i;
        if (is || dead) {
          c.vs &= ~byte;
          if constexpr (D == 128)
            c.v[i] = 0u;
          else
            c.v[i / 2] &= ~(0xffffu << (16 * (i % 2)));
        }
      }
    }
    u32x2 x[VT];
    unpack_v<D>(c.v, c.vs, x);
#pragma unroll
    for (int t = 0; t < VT; ++t) st.v[wave / 2][t][lane][wave % 2] = x[t];
    uint32_t mine = 0u;  // the block's tokens, for group `lane`
    if (__ballot(odd != 0u)) {
      const int at = lane % L4::kGroups * (16 / L4::kGroups);  // a column of the group
      for (int kg = 0; kg < 4; ++kg) mine |= __shfl(odd, kg * 16 + at) << (4 * kg);
    }
    if (lane < L4::kGroups) st.nan[wave][lane] = mine;
  };
  auto compute = [&](const Stage4<D>& st, int s) {
    int j[kP4Step];
#pragma unroll
    for (int e = 0; e < kP4Step; ++e)
      j[e] = __builtin_amdgcn_readfirstlane(list_j[kP4Step * s + e]);
    if (j[0] * kBlockSize > last_pos) return;  // (ascending: no key of the step is seen)
    f32x4 sc[RT][kP4Step];
#pragma unroll
    for (int e = 0; e < kP4Step; ++e) {
#pragma unroll
      for (int r = 0; r < RT; ++r) sc[r][e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        const bf16x8 kf = as_bf16x8(st.k[e][c][lane]);
#pragma unroll
        for (int r = 0; r < RT; ++r) sc[r][e] = mfma16x16x32(kf, qv[r][c], sc[r][e]);
      }
    }
    // Keys past a row's position (those of no block lie past every position).
    if (!wave_full || j[kP4Step - 1] * kBlockSize + kBlockSize - 1 > first_pos) {
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int e = 0; e < kP4Step; ++e) {
          const int seen = pos[r] - j[e] * kBlockSize - 4 * kgrp;
#pragma unroll
          for (int k = 0; k < 4; ++k) sc[r][e][k] = k <= seen ? sc[r][e][k] : -INFINITY;
        }
    }
    u32x4 pf[RT][kP4Step / 2];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      float mx = max3f(sc[r][0][0], sc[r][0][1], sc[r][0][2]);
      mx = max3f(mx, sc[r][0][3], sc[r][1][0]);
      mx = max3f(mx, sc[r][1][1], sc[r][1][2]);
      mx = max3f(mx, sc[r][1][3], sc[r][2][0]);
      mx = max3f(mx, sc[r][2][1], sc[r][2][2]);
      mx = max3f(mx, sc[r][2][3], sc[r][3][0]);
      mx = max3f(mx, sc[r][3][1], sc[r][3][2]);
      mx = max2f(mx, sc[r][3][3]);
      if (__ballot(mx > rise[r])) {
        const float m_new = fmaxf(m_run[r], max_xor32(max_xor16(mx)) * a.scale_log2);
        const float alpha = fast_exp2(m_run[r] - m_new);
        l_run[r] *= alpha;
        m_run[r] = m_new;
        rise[r] = (m_new + kP4Lazy) * inv_scale;
#pragma unroll
        for (int t = 0; t < VT; ++t) acc[r][t] *= alpha;
      }
      float sum[kP4Step];
#pragma unroll
      for (int e = 0; e < kP4Step; ++e) {
        float p[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          p[k] = fast_exp2(fmaf(sc[r][e][k], a.scale_log2, -m_run[r]));
        sum[e] = (p[0] + p[1]) + (p[2] + p[3]);
        pf[r][e / 2][2 * (e % 2)] = pack_bf16x2(p[0], p[1]);
        pf[r][e / 2][2 * (e % 2) + 1] = pack_bf16x2(p[2], p[3]);
      }
      l_run[r] += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    }
#pragma unroll
    for (int pr = 0; pr < kP4Step / 2; ++pr)
#pragma unroll
      for (int t = 0; t < VT; ++t) {
        const bf16x8 vf =
            as_bf16x8(*reinterpret_cast<const u32x4*>(&st.v[pr][t][lane][0]));
#pragma unroll
        for (int r = 0; r < RT; ++r)
          acc[r][t] = mfma16x16x32(vf, as_bf16x8(pf[r][pr]), acc[r][t]);
      }
    // Tokens whose V is not finite, in the rows that see them (a lane's dims all lie
    // in one group).
    uint32_t bad[kP4Step], any = 0u;
#pragma unroll
    for (int e = 0; e < kP4Step; ++e) any |= bad[e] = st.nan[e][L4::k_group(kgrp)];
    if (__ballot(any != 0u)) {
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        bool hit = false;
#pragma unroll
        for (int e = 0; e < kP4Step; ++e) {
          const int n = min(max(pos[r] - j[e] * kBlockSize + 1, 0), kBlockSize);
          hit |= (bad[e] & ((1u << n) - 1u)) != 0u;
        }
        if (hit) {
          const float nan = __builtin_nanf("");
#pragma unroll
          for (int t = 0; t < VT; ++t) acc[r][t] = f32x4{nan, nan, nan, nan};
        }
      }
    }
  };

  for (int w0 = lo; w0 < hi; w0 += kP4Window) {
    // the window's valid blocks, in ascending order
    const int j = w0 + tid;
    int id = -1;
    if (j < hi) {
      const int p = table[j];
      if (p >= 0 && p < a.num_blocks && a.block_version[p] == rv) id = p;
    }
    const uint64_t m = __ballot(id >= 0);
    if (lane == 0) wave_n[wave_all] = __popcll(m);
    __syncthreads();
    int before = 0, n = 0;
#pragma unroll
    for (int w = 0; w < kP4Halves * kP4Waves; ++w) {
      before += w < wave_all ? wave_n[w] : 0;
      n += wave_n[w];
    }
    if (id >= 0) {
      const int at = before + __popcll(m & ((1ull << lane) - 1ull));
      list_id[at] = id;
      list_j[at] = j;
    }
    if (tid < 2 * kP4Step) {  // the rest of the halves' last steps: no block
      list_id[n + tid] = -1;
      list_j[n + tid] = (INT_MAX - kBlockSize) / kBlockSize;
    }
    __syncthreads();
    // step 2 i + half is this half's i-th
    const int steps = (n + kP4Halves * kP4Step - 1) / (kP4Halves * kP4Step);
    if (steps > 0) {
      Codes4<D> c;
      load(c, half);
      unpack(c, stage[half][0], half);
      if (steps > 1) load(c, kP4Halves + half);
      __syncthreads();
      for (int i = 0; i < steps; ++i) {
        if (i + 1 < steps) {
          unpack(c, stage[half][(i + 1) % 2], kP4Halves * (i + 1) + half);
          if (i + 2 < steps) load(c, kP4Halves * (i + 2) + half);
        }
        compute(stage[half][i % 2], kP4Halves * i + half);
        __syncthreads();
      }
    }
    __syncthreads();  // (the list is written again)
  }

  // ---- finish: the rows' sums over the k-groups, the halves joined through LDS (the
  // second writes, the first adds), then the outputs. A lane's dims are 4 * VT
  // neighbours: (4 kgrp + i) * VT + t.
  constexpr int kRow = D + 4;
  float* join = reinterpret_cast<float*>(&stage[0][0]);
  float* join_ml = join + kP4Rows * kRow;
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    l_run[r] += __shfl_xor(l_run[r], 16);
    l_run[r] += __shfl_xor(l_run[r], 32);
  }
  if (half == 1) {
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int row = 16 * RT * wave + 16 * r + col;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int t = 0; t < VT; t += 4)
          *reinterpret_cast<f32x4*>(join + row * kRow + (4 * kgrp + i) * VT + t) =
              f32x4{acc[r][t][i], acc[r][t + 1][i], acc[r][t + 2][i], acc[r][t + 3][i]};
      if (kgrp == 0) {
        join_ml[2 * row] = m_run[r];
        join_ml[2 * row + 1] = l_run[r];
      }
    }
  }
  __syncthreads();
  if (half == 1) return;
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int row = 16 * RT * wave + 16 * r + col;
    if (row >= tl.rows) continue;
    const float m1 = join_ml[2 * row], l1 = join_ml[2 * row + 1];
    const float M = fmaxf(m_run[r], m1);
    const float f0 = fast_exp2(m_run[r] - M), f1 = fast_exp2(m1 - M);
    const float l = l_run[r] * f0 + l1 * f1;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int64_t at = qrow[r] * a.ranges + range;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < VT; t += 4) {
        const int d = (4 * kgrp + i) * VT + t;
        const f32x4 o1 = *reinterpret_cast<const f32x4*>(join + row * kRow + d);
        f32x4 o = {acc[r][t][i], acc[r][t + 1][i], acc[r][t + 2][i], acc[r][t + 3][i]};
        o = o * f0 + o1 * f1;
        if (n_ranges == 1) {
          o *= inv;
          *reinterpret_cast<u32x2*>(a.out + qrow[r] * D + d) =
              u32x2{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
        } else {
          *reinterpret_cast<f32x4*>(a.part_o + at * D + d) = o;
        }
      }
    if (kgrp == 0) {
      if (n_ranges > 1) {
        a.part_ml[2 * at] = M;
        a.part_ml[2 * at + 1] = l;
      } else if (a.lse) {
        a.lse[qrow[r]] = l == 0.f ? -INFINITY : (M + __log2f(l)) * kLn2;
      }
    }
  }
}

// Joins the key ranges of the tiles that have more than one: a workgroup a quarter of a
// tile and KV head, a thread 4 dims of a row.
constexpr int kMgRows = kP4Rows / 4;

template <int D>
__global__ __launch_bounds__(kApThreads) void merge_kv4_kernel(Prefill4Args a) {
  const int g = blockIdx.x % a.Hkv;
  const int rest = blockIdx.x / a.Hkv;
  if (rest / 4 >= a.counts[1]) return;
  const int4 e = a.tiles[rest / 4];
  const int n = e.w;
  if (n == 1) return;
  const Tile4 tl = tile_of(a, e.x, e.y);
  for (int x = threadIdx.x; x < kMgRows * (D / 4); x += kApThreads) {
    const int row = rest % 4 * kMgRows + x / (D / 4), d = 4 * (x % (D / 4));
    if (row >= tl.rows) break;
    const int at = tl.row0 + row;
    const int64_t q =
        static_cast<int64_t>(tl.r0 + at / a.group) * a.Hq + g * a.group + at % a.group;
    const float2* ml = reinterpret_cast<const float2*>(a.part_ml + q * a.ranges * 2);
    const float* po = a.part_o + q * a.ranges * D + d;
    float M = kP4NegBig, den = 0.f;
    f32x4 num = {0.f, 0.f, 0.f, 0.f};
    for (int r = 0; r < n; ++r) M = fmaxf(M, ml[r].x);
    for (int r = 0; r < n; ++r) {
      const float f = fast_exp2(ml[r].x - M);
      den += ml[r].y * f;
      num += *reinterpret_cast<const f32x4*>(po + static_cast<int64_t>(r) * D) * f;
    }
    num *= den == 0.f ? 0.f : 1.f / den;
    *reinterpret_cast<u32x2*>(a.out + q * D + d) =
        u32x2{pack_bf16x2(num[0], num[1]), pack_bf16x2(num[2], num[3])};
    if (d == 0 && a.lse) a.lse[q] = den == 0.f ? -INFINITY : (M + __log2f(den)) * kLn2;
  }
}

template <int D>
local_status_t launch_prefill_kv4(const Prefill4Args& a, hipStream_t s) {
  const char* who = "paged_attn_prefill_kv4";
  const int64_t grid = static_cast<int64_t>(a.max_tiles) * a.ranges * a.Hkv;
  // blocks that hold a chunk's tokens: at most one more than the chunk fills, each side
  const int64_t blocks = a.T / kBlockSize + 2 * static_cast<int64_t>(a.B);
  const int64_t append = 1 + (blocks * a.Hkv + kApWaves - 1) / kApWaves;
  const int64_t merge = a.ranges > 1 ? static_cast<int64_t>(a.max_tiles) * 4 * a.Hkv : 0;
  if (grid >= (1LL << 31) || append >= (1LL << 31) || merge >= (1LL << 31))
    return local_fail(LOCAL_ERR_UNSUPPORTED, "%s: grids of %lld, %lld and %lld workgroups", who,
                      (long long)grid, (long long)append, (long long)merge);
  if (a.k_new)
    append_kv4_kernel<D><<<static_cast<unsigned>(append), kApThreads, 0, s>>>(a);
  else
    plan_kv4_kernel<<<1, kApThreads, 0, s>>>(a);
  prefill_kv4_kernel<D><<<static_cast<unsigned>(grid), kP4Threads, 0, s>>>(a);
  if (merge) merge_kv4_kernel<D><<<static_cast<unsigned>(merge), kApThreads, 0, s>>>(a);
  return local_check_launch(who);
}

// Key ranges that a tile of a call may be split into: as many as give every compute unit
// a workgroup where there are few tiles, counted from the sizes that the host knows.
int ranges_of_call(int64_t tiles, int Hkv, int max_blocks) {
  const int64_t want = (2 * kP4Units + tiles * Hkv - 1) / (tiles * Hkv);
  const int64_t most = std::max(1, max_blocks / kP4MinRange);
  return static_cast<int>(std::min<int64_t>({want, most, kP4MaxRanges}));
}

}  // namespace
}  // namespace localk

using namespace localk;

extern "C" local_status_t local_paged_attn_prefill_kv4(
    const uint16_t* q, const int32_t* q_indptr, int32_t B, int64_t T, int32_t Hq, int32_t Hkv,
    int32_t D, const uint16_t* k_new, const uint16_t* v_new, uint8_t* kv4, int64_t num_blocks,
    int32_t block_size, const int32_t* block_table, int32_t max_blocks,
    const int32_t* ctx_lens, const int32_t* block_version, const int32_t* req_version,
    float sm_scale, uint16_t* out, float* lse, void* ws, size_t* ws_bytes, void* stream) {
  const char* who = "paged_attn_prefill_kv4";
  if (!ws_bytes) return local_fail(LOCAL_ERR_WORKSPACE, "%s: ws_bytes is NULL", who);
  if (B < 0 || T < 0 || Hq <= 0 || Hkv <= 0 || max_blocks < 1 || num_blocks < 1 || Hq % Hkv != 0)
    return local_fail(LOCAL_ERR_SHAPE,
                      "%s: B=%d T=%lld Hq=%d Hkv=%d max_blocks=%d num_blocks=%lld", who, B,
                      (long long)T, Hq, Hkv, max_blocks, (long long)num_blocks);
  if (block_size != kBlockSize || (D != 64 && D != 128) || Hq / Hkv > 16)
    return local_fail(LOCAL_ERR_UNSUPPORTED,
                      "%s: block_size=%d D=%d group=%d (need 16, 64|128, <=16)", who,
                      block_size, D, Hq / Hkv);
  if (T * (Hq / Hkv) >= (1LL << 30))  // (rows of a request are counted in 32 bits)
    return local_fail(LOCAL_ERR_UNSUPPORTED, "%s: T=%lld", who, (long long)T);
  if ((k_new == nullptr) != (v_new == nullptr))
    return local_fail(LOCAL_ERR_NULL, "%s: k_new and v_new must both be set", who);
  Prefill4Args a{};
  // (B tiles more than the rows fill: each request's last one)
  const int64_t tiles = T * (Hq / Hkv) / kP4Rows + B;
  if (tiles * kP4MaxRanges >= (1LL << 31))
    return local_fail(LOCAL_ERR_UNSUPPORTED, "%s: T=%lld B=%d", who, (long long)T, B);
  a.max_tiles = static_cast<int>(tiles);
  a.ranges = B > 0 && T > 0 ? ranges_of_call(tiles, Hkv, max_blocks) : 1;
  const size_t rows = static_cast<size_t>(T) * Hq * (a.ranges > 1 ? a.ranges : 0);
  const size_t plan_at = 256, tiles_at = plan_at + sizeof(int4) * tiles * a.ranges;
  const size_t part_at = round256(tiles_at + sizeof(int4) * tiles);
  const size_t need = part_at + rows * (D + 2) * sizeof(float);
  if (!ws) {
    *ws_bytes = need;
    return LOCAL_OK;
  }
  if (*ws_bytes < need)
    return local_fail(LOCAL_ERR_WORKSPACE, "%s: workspace %zu < %zu", who, *ws_bytes, need);
  if (B == 0 || T == 0) return LOCAL_OK;
  if (!q || !q_indptr || !kv4 || !block_table || !ctx_lens || !block_version || !req_version ||
      !out)
    return local_fail(LOCAL_ERR_NULL, "%s: NULL pointer argument", who);
  if (!aligned16(q) || !aligned16(kv4) || !aligned16(out) || !aligned16(k_new) ||
      !aligned16(v_new) || !aligned16(ws))
    return local_fail(LOCAL_ERR_UNSUPPORTED, "%s: q, k_new, v_new, kv4, out and ws must start "
                      "on 16 bytes", who);
  a.q = q;
  a.q_indptr = q_indptr;
  a.k_new = k_new;
  a.v_new = v_new;
  a.kv4 = kv4;
  a.block_table = block_table;
  a.ctx_lens = ctx_lens;
  a.block_version = block_version;
  a.req_version = req_version;
  a.out = out;
  a.lse = lse;
  char* base = static_cast<char*>(ws);
  a.counts = reinterpret_cast<int*>(base);
  a.plan = reinterpret_cast<int4*>(base + plan_at);
  a.tiles = reinterpret_cast<int4*>(base + tiles_at);
  a.part_o = reinterpret_cast<float*>(base + part_at);
  a.part_ml = a.part_o + rows * D;
  a.T = T;
  a.num_blocks = num_blocks;
  a.B = B;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.group = Hq / Hkv;
  a.max_blocks = max_blocks;
  const Scale4 scale = scale_of(sm_scale);
  a.scale_log2 = scale.log2;
  a.q_xor = scale.q_xor;
  a.q_and = scale.q_and;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return D == 64 ? launch_prefill_kv4<64>(a, s) : launch_prefill_kv4<128>(a, s);
}
