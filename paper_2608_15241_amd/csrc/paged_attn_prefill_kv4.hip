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
//    there the running maximum rises only when a weight would pass 2^8, and the weights
//    are rounded to bf16 for the product and summed both ways. 4 x 512 tokens on 0 to
//    2048, 32 heads of 128: 78 us, the steps at about 850 TFLOP/s.
//  * An infinity or a NaN in V (scale byte 255) must reach the rows that see its token
//    and no other, which 0 * NaN in a product would not do: its values enter the
//    product as zeros, and a mask of such tokens then puts NaN into those rows.
#include <algorithm>
#include <climits>

#include "kv4_attn.hpp"
#include "paged_attn_decode.hpp"

namespace localk {
namespace {

constexpr int kP4Waves = 4;                            // of a half
constexpr int kP4Halves = 2;
constexpr int kP4Threads = kP4Halves * kP4Waves * kWave;
constexpr int kP4RowTiles = 2;                         // 16-row tiles of a wave
constexpr int kP4Rows = kP4Waves * 16 * kP4RowTiles;   // rows of a workgroup
constexpr int kP4Step = 4;                             // blocks a step
constexpr int kP4Window = kP4Threads;                  // table entries listed at a time
constexpr int kP4MinRange = 16;                        // blocks a key range has at least
constexpr int kP4MaxRanges = 16;
constexpr int kP4Units = 256;                          // a workgroup for every compute unit
constexpr int kApThreads = 256;                        // of the append launch
constexpr int kApWaves = kApThreads / kWave;

// Blocks of a key range below which tiles (times KV heads) of this number are not cut
// further. A range's partial result, 128 rows in float32, is written and read again, which
// takes as long as some 24 blocks' products; with more tiles fewer compute units are idle
// without it. Against ranges of 8 blocks or a compute unit's share, whichever is longer,
// calls took 0.58 to 1.12 of the time, 0.92 to 0.93 on average over two sets of 40 (202
// tiles of 1 to 31 blocks 39 -> 24 us); one bound for all, 24 or 48, 0.94.
__host__ __device__ inline int least_range(int64_t units) {
  return static_cast<int>(units < 4 * kP4MinRange ? kP4MinRange : units < 256 ? units / 4 : 64);
}

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
  int4* plan;      // units (Unit4), longest first, then ones of no request
  int4* tiles;     // first token, first row, rows, ranges; then ones of no rows
  float* part_o;   // [T][Hq][ranges][D]
  float* part_ml;  // [T][Hq][ranges][2]
  int64_t T, num_blocks;
  int B, Hq, Hkv, group, max_blocks;
  int ranges;      // the most a tile may be split into
  int max_tiles;   // tiles that the plan has room for (of few rows: that there may be)
  int pb;          // few rows: blocks of a partition (few_part), else 0
  float scale_log2;
  uint32_t q_xor, q_and;
};

__device__ __forceinline__ bool rows_ok4(int r0, int r1, int64_t T) {
  return r0 >= 0 && r1 >= r0 && r1 <= T;
}

// A unit of work: a tile of 128 rows of a request, or a range of its keys.
struct Unit4 {
  int b, range, n_ranges, r0;     // request (-1: none), range of so many, first token
  int row0, rows, prefix, lo;     // first row and rows, cached tokens, blocks [lo, hi)
  int hi, L, rv, none;            // context length and version of the request
};
constexpr int kUnitInt4s = sizeof(Unit4) / sizeof(int4);

// Blocks that the tile at row0 of a chunk of n tokens sees with its last row.
__device__ __forceinline__ int blocks_of(const Prefill4Args& a, int n, int L, int row0) {
  const int rows = min(kP4Rows, n * a.group - row0);
  const int last = L - n + (row0 + rows - 1) / a.group;  // its position
  return last < 0 ? 0 : min(last / kBlockSize + 1, a.max_blocks);
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
constexpr int kPlanCache = 1024;  // tiles whose entries stay in LDS
constexpr int kPlanChoices = 3;

__device__ void plan_kv4(const Prefill4Args& a) {
  __shared__ int4 cache[kPlanCache];
  __shared__ int4 req[kApThreads];  // first token, tokens, context length, version
  __shared__ int first[kApThreads + 1], wave_sums[kApWaves], hist[256], longest;
  __shared__ int n_units[kPlanChoices];
  __shared__ unsigned long long work;
  const int tid = threadIdx.x;
  int n_tiles = 0;
  if (tid == 0) work = 0ull, longest = 1;
  hist[tid] = 0;
  if (tid < kPlanChoices) n_units[tid] = 0;
  for (int b0 = 0; b0 < a.B; b0 += kApThreads) {
    int n = 0;
    if (b0 + tid < a.B) {
      const int r0 = a.q_indptr[b0 + tid], r1 = a.q_indptr[b0 + tid + 1];
      req[tid] = int4{r0, r1 - r0, a.ctx_lens[b0 + tid], a.req_version[b0 + tid]};
      if (rows_ok4(r0, r1, a.T)) n = ((r1 - r0) * a.group + kP4Rows - 1) / kP4Rows;
    }
    const int incl = scan_ap(n, wave_sums);
    first[tid + 1] = incl;
    if (tid == 0) first[0] = 0;
    __syncthreads();
    const int all = first[kApThreads];
    // (a plan is sized for row ranges that do not overlap)
    for (int t = tid; t < all && n_tiles + t < a.max_tiles; t += kApThreads) {
      int lo = 0, hi = min(a.B - b0, kApThreads);
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (first[mid] <= t)
          lo = mid;
        else
          hi = mid;
      }
      const int b = b0 + lo, row0 = (t - first[lo]) * kP4Rows, at = n_tiles + t;
      const int blocks = blocks_of(a, req[lo].y, req[lo].z, row0);
      const int4 e = {b, row0, blocks, 0};
      if (at < kPlanCache)
        cache[at] = e;
      else
        a.tiles[at] = e;
      atomicAdd(&work, static_cast<unsigned long long>(blocks));
      atomicMax(&longest, blocks);
    }
    n_tiles = min(n_tiles + all, a.max_tiles);
    __syncthreads();
  }
  // No unit longer than a compute unit's share of the work (and least_range), or an eighth
  // or a quarter more where that leaves no compute unit a second one (units of one length, 270 of them
  // by the share alone, took two rounds: 52 us instead of 43).
  const float share = fmaxf(static_cast<float>(work) * a.Hkv / kP4Units,
                            least_range(static_cast<int64_t>(n_tiles) * a.Hkv));
  auto ranges_of = [&](int blocks, float inv_len) {
    const int want = static_cast<int>(static_cast<float>(blocks) * inv_len + 0.999f);
    return max(1, min(want, min(a.ranges, blocks / kP4MinRange)));
  };
  auto bucket = [&](int blocks, int n) {
    const float part = static_cast<float>(blocks) / (static_cast<float>(longest) * n);
    return 255 - min(255, static_cast<int>(part * 255.f));
  };
  auto entry = [&](int t) { return t < kPlanCache ? cache[t] : a.tiles[t]; };
  float inv_len = 1.f / share;
  if (a.ranges > 1) {
    constexpr float kLonger[kPlanChoices] = {1.f, 1.125f, 1.25f};
    int n[kPlanChoices] = {0, 0, 0};
    for (int t = tid; t < n_tiles; t += kApThreads) {
      const int blocks = entry(t).z;
#pragma unroll
      for (int c = 0; c < kPlanChoices; ++c) n[c] += ranges_of(blocks, inv_len / kLonger[c]);
    }
#pragma unroll
    for (int c = 0; c < kPlanChoices; ++c) {
#pragma unroll
      for (int off = kWave / 2; off > 0; off >>= 1) n[c] += __shfl_xor(n[c], off);
      if (tid % kWave == 0) atomicAdd(&n_units[c], n[c]);
    }
    __syncthreads();
#pragma unroll
    for (int c = kPlanChoices - 1; c >= 0; --c)
      if (static_cast<int64_t>(n_units[c]) * a.Hkv <= kP4Units)
        inv_len = 1.f / (share * kLonger[c]);
  }
  for (int t = tid; t < n_tiles; t += kApThreads) {
    const int blocks = entry(t).z, n = ranges_of(blocks, inv_len);
    atomicAdd(&hist[bucket(blocks, n)], n);
  }
  __syncthreads();
  const int mine = hist[tid], incl = scan_ap(mine, wave_sums);
  const int before = incl - mine;
  __syncthreads();
  hist[tid] = before;
  if (tid == kApThreads - 1) first[0] = incl;
  __syncthreads();
  const int units = first[0];
  for (int t = tid; t < a.max_tiles; t += kApThreads) {
    if (t >= n_tiles) {
      a.tiles[t] = int4{0, 0, 0, 1};
      continue;
    }
    const int4 e = entry(t);
    const int b = e.x, row0 = e.y, blocks = e.z, n = ranges_of(blocks, inv_len);
    int4 q;
    if (a.B <= kApThreads) {
      q = req[b];
    } else {  // (only the last requests are still in LDS)
      const int r0 = a.q_indptr[b];
      q = int4{r0, a.q_indptr[b + 1] - r0, a.ctx_lens[b], a.req_version[b]};
    }
    const int r0 = q.x, tokens = q.y, L = q.z, rv = q.w;
    const int rows = min(kP4Rows, tokens * a.group - row0);
    a.tiles[t] = int4{r0, row0, rows, n};
    const int at = atomicAdd(&hist[bucket(blocks, n)], n);
    for (int r = 0; r < n; ++r) {
      int4* u = a.plan + static_cast<int64_t>(at + r) * kUnitInt4s;
      u[0] = int4{b, r, n, r0};
      u[1] = int4{row0, rows, L - tokens,
                  static_cast<int>(static_cast<int64_t>(blocks) * r / n)};
      u[2] = int4{static_cast<int>(static_cast<int64_t>(blocks) * (r + 1) / n), L, rv, 0};
    }
  }
  for (int u = units + tid; u < a.max_tiles * a.ranges; u += kApThreads)
    a.plan[static_cast<int64_t>(u) * kUnitInt4s] = int4{-1, 0, 0, 0};
}

// ---------------------------------------------------------------- append
// The k-th block of new tokens: requests in order. Every lane returns the same; false
// past the last.
struct NewBlock {
  int b, j;       // request, block of its table
  int r0, n, L;   // the request's first token row and tokens, its context length
};

__device__ bool find_new_block(const Prefill4Args& a, int64_t k, NewBlock* f) {
  const int lane = threadIdx.x % kWave;
  for (int b0 = 0; b0 < a.B; b0 += kWave) {
    int n = 0, j0 = 0, r0 = 0, r1 = 0, L = 0;
    if (b0 + lane < a.B) {
      r0 = a.q_indptr[b0 + lane], r1 = a.q_indptr[b0 + lane + 1];
      L = a.ctx_lens[b0 + lane];
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
      f->b = b0 + l;
      f->r0 = __builtin_amdgcn_readlane(r0, l);
      f->n = __builtin_amdgcn_readlane(r1, l) - f->r0;
      f->L = __builtin_amdgcn_readlane(L, l);
      f->j = __builtin_amdgcn_readlane(j0, l) + static_cast<int>(k) -
             __builtin_amdgcn_readlane(incl - n, l);
      return true;
    }
    k -= __builtin_amdgcn_readlane(incl, kWave - 1);
  }
  return false;
}

template <int D>
__global__ __launch_bounds__(kApThreads) void append_kv4_kernel(Prefill4Args a) {
  using L4 = Kv4<D>;
  constexpr int VT = D / 16;
  if (a.plan && blockIdx.x == 0) {
    plan_kv4(a);
    return;
  }
  const int64_t unit = (static_cast<int64_t>(blockIdx.x) - (a.plan ? 1 : 0)) * kApWaves +
                       threadIdx.x / kWave;
  const int lane = threadIdx.x % kWave, col = lane % 16, kgrp = lane / 16;
  const int g = static_cast<int>(unit % a.Hkv);
  NewBlock f;
  if (!find_new_block(a, unit / a.Hkv, &f)) return;
  const int p = a.block_table[static_cast<int64_t>(f.b) * a.max_blocks + f.j];
  const int r0 = f.r0, n = f.n, j = f.j;
  const int first = f.L - n;  // position of the chunk's first token
  // Slot s of the block is token row s + off of the chunk where that is one of its n.
  const int off = j * kBlockSize - first;
  auto fresh = [&](int slot) { return slot + off >= 0 && slot + off < n; };
  auto row = [&](int slot) {
    return (static_cast<int64_t>(r0 + slot + off) * a.Hkv + g) * D;
  };
  // A lane takes the same dims of K and V, VT col .., of slots 4 kgrp .. (whole rows are
  // read side by side; K by the lane that holds its codes in attention read 64 places).
  auto read = [&](const uint16_t* x, int e) {
    u32x4 v = {0u, 0u, 0u, 0u};
    if (fresh(4 * kgrp + e)) {
      const uint16_t* from = x + row(4 * kgrp + e) + VT * col;
      if constexpr (D == 128) {
        v = ld_global<u32x4>(from);
      } else {
        const u32x2 w = ld_global<u32x2>(from);
        v = u32x4{w.x, w.y, 0u, 0u};
      }
    }
    return v;
  };
  u32x4 kv[4], vv[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) kv[e] = read(a.k_new, e), vv[e] = read(a.v_new, e);
  if (p < 0 || p >= a.num_blocks) return;  // (read while the id was on its way)
  uint8_t* o = a.kv4 + (static_cast<int64_t>(p) * a.Hkv + g) * L4::kTile;
  uint32_t kcode[4], ks[4], vcode[4], vs[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    ks[e] = round_v<D>(kv[e], kcode[e]);
    vs[e] = round_v<D>(vv[e], vcode[e]);
  }
  const int d = VT * col, group = L4::v_group(col);
  const bool head = col % (16 / L4::kGroups) == 0;  // of the group's lanes
  uint8_t* vo = o + L4::kV + lane * L4::kLane;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int s = 4 * kgrp + e;
    if (!fresh(s)) continue;
    uint8_t* ko = o + (d / (D / 4) * kBlockSize + s) * L4::kLane + d % (D / 4) / 2;
    if constexpr (D == 128)
      *reinterpret_cast<uint32_t*>(ko) = kcode[e];
    else
      *reinterpret_cast<uint16_t*>(ko) = static_cast<uint16_t>(kcode[e]);
  }
  if (fresh(4 * kgrp) && fresh(4 * kgrp + 3)) {  // the lane's four slots at once
    if constexpr (D == 128)
      *reinterpret_cast<u32x4*>(vo) = u32x4{vcode[0], vcode[1], vcode[2], vcode[3]};
    else
      *reinterpret_cast<u32x2*>(vo) = u32x2{(vcode[0] & 0xffffu) | vcode[1] << 16,
                                            (vcode[2] & 0xffffu) | vcode[3] << 16};
    if (head) {
      *reinterpret_cast<uint32_t*>(o + L4::k_scale(group, 4 * kgrp)) =
          ks[0] | ks[1] << 8 | ks[2] << 16 | ks[3] << 24;
      *reinterpret_cast<uint32_t*>(o + L4::v_scale(group, 4 * kgrp)) =
          vs[0] | vs[1] << 8 | vs[2] << 16 | vs[3] << 24;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (!fresh(4 * kgrp + e)) continue;
      if constexpr (D == 128)
        reinterpret_cast<uint32_t*>(vo)[e] = vcode[e];
      else
        reinterpret_cast<uint16_t*>(vo)[e] = static_cast<uint16_t>(vcode[e]);
      if (head) {
        o[L4::k_scale(group, 4 * kgrp + e)] = static_cast<uint8_t>(ks[e]);
        o[L4::v_scale(group, 4 * kgrp + e)] = static_cast<uint8_t>(vs[e]);
      }
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
  static_assert(sizeof(stage) >= kP4Rows * (D + 4 + 2) * sizeof(float), "joined in the stages");

  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave_all = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int wave = wave_all % kP4Waves, half = wave_all / kP4Waves;
  const int col = lane % 16, kgrp = lane / 16;
  // Unit p * gridDim + i of pass p, by falling length, every other pass the other way
  // round (in steps of 8 workgroups, the XCDs: a KV head's units stay on one).
  const uint32_t units = static_cast<uint32_t>(a.max_tiles) * a.ranges * a.Hkv;
  auto unit_of = [&](uint32_t pass) {  // (below 2^31 + 256: the host checks)
    const uint32_t i = blockIdx.x, n = gridDim.x;
    const uint32_t turned = n % 8 == 0 ? (n / 8 - 1 - i / 8) * 8 + i % 8 : n - 1 - i;
    return pass * n + (pass % 2 ? turned : i);
  };
  auto read_unit = [&](uint32_t u) {
    Unit4 e;
    e.b = -1;
    if (u < units) {
      // (read-only here and the same for the workgroup: scalar loads)
      typedef const __attribute__((address_space(4))) u32x4* ScalarPtr;
      const int64_t at = u / static_cast<uint32_t>(a.Hkv);
      const ScalarPtr from = (ScalarPtr)(a.plan + at * kUnitInt4s);
      u32x4 w[kUnitInt4s];
#pragma unroll
      for (int i = 0; i < kUnitInt4s; ++i) w[i] = from[i];
      __builtin_memcpy(&e, w, sizeof e);
    }
    return e;
  };
  // A table entry where it names a block of the pool, else -1; then with its tag.
  auto read_id = [&](const Unit4& e, int j) {
    const int p = j < e.hi ? a.block_table[static_cast<int64_t>(e.b) * a.max_blocks + j] : -1;
    return p >= 0 && p < a.num_blocks ? p : -1;
  };
  auto read_tag = [&](int p) { return p >= 0 ? a.block_version[p] : 0; };

  uint32_t pass = 0;
  Unit4 e = read_unit(unit_of(0));
  if (e.b < 0) return;
  int g = static_cast<int>(unit_of(0) % static_cast<uint32_t>(a.Hkv));
  int id = read_id(e, e.lo + tid);
  if (read_tag(id) != e.rv) id = -1;

  // This wave's rows: column col of row tile r is row 32 wave + 16 r + col of the tile.
  auto row_of = [&](const Unit4& u, int head, int r, int* position) {
    const int row = 16 * RT * wave + 16 * r + col;
    const bool in = row < u.rows;
    const int at = u.row0 + (in ? row : 0);
    const int i = at / a.group;
    *position = in ? u.prefix + i : -1;
    return static_cast<int64_t>(u.r0 + i) * a.Hq + head * a.group + at % a.group;
  };
  int pos[RT];  // a row's position, -1 for none
  bf16x8 qv[RT][KC];
  auto read_q = [&](const Unit4& u, int head) {
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int64_t row = row_of(u, head, r, &pos[r]);
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        u32x4 v = {0u, 0u, 0u, 0u};
        if (16 * RT * wave + 16 * r + col < u.rows)
          v = ld_global<u32x4>(a.q + row * D + (D / 4) * kgrp + 8 * c);
        qv[r][c] = as_bf16x8((v ^ a.q_xor) & a.q_and);
      }
    }
  };
  read_q(e, g);

  f32x4 acc[RT][VT];
  float m_run[RT], rise[RT], l_run[RT], w_run[RT];  // as in Attn4
  const float inv_scale = 1.f / a.scale_log2;
  // Positions of the wave's first and last row: bounds of what it may see.
  bool wave_full = false;
  int first_pos = 0, last_pos = -1;

  // Lane i holds what the half's i-th step of a window takes: its blocks' logical
  // indices and the id of the one that this wave unpacks.
  static_assert(kP4Window == kWave * kP4Halves * kP4Step, "a lane a step");
  int my_id = -1;
  int4 my_j4 = {0, 0, 0, 0};
  auto j_of = [&](int s, int e) {
    return __builtin_amdgcn_readlane(e == 0 ? my_j4.x : e == 1 ? my_j4.y : e == 2 ? my_j4.z
                                                                                : my_j4.w, s);
  };
  // This wave unpacks block `wave` of its half's steps.
  auto load = [&](Codes4<D>& c, int s) {
    const int p = __builtin_amdgcn_readlane(my_id, s);
    const int64_t tile = (static_cast<int64_t>(max(p, 0)) * a.Hkv + g) * L4::kTile;
    const __amdgpu_buffer_rsrc_t r = make_rsrc(a.kv4 + tile, p >= 0 ? L4::kTile : 0u);
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
    const int j = j_of(s, wave);
    const bool last = e.L - j * kBlockSize < kBlockSize;
    // (a byte of 255 is a zero byte of the complement)
    const bool bad = ((~c.vs - 0x01010101u) & c.vs & 0x80808080u) != 0u;
    uint32_t odd = 0u;
    if (last || __ballot(bad)) {
      const int live = e.L - j * kBlockSize - 4 * kgrp;  // (no block: far below 0)
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
    for (int e = 0; e < kP4Step; ++e) j[e] = j_of(s, e);
    if (j[0] * kBlockSize > last_pos) return;  // (ascending: no key of the step is seen)
    // Operands are read a block of K (half a pair of V) ahead of their products; left to
    // itself the compiler reads two at a time and waits for each.
    f32x4 sc[RT][kP4Step];
    u32x4 kf[2][KC];
#pragma unroll
    for (int c = 0; c < KC; ++c) kf[0][c] = st.k[0][c][lane];
#pragma unroll
    for (int e = 0; e < kP4Step; ++e) {
      if (e + 1 < kP4Step) {
#pragma unroll
        for (int c = 0; c < KC; ++c) kf[(e + 1) % 2][c] = st.k[e + 1][c][lane];
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int r = 0; r < RT; ++r) sc[r][e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < KC; ++c)
#pragma unroll
        for (int r = 0; r < RT; ++r)
          sc[r][e] = mfma16x16x32(as_bf16x8(kf[e % 2][c]), qv[r][c], sc[r][e]);
      __builtin_amdgcn_sched_barrier(0);
    }
    constexpr int VG = VT / 2, kGroups = kP4Step / 2 * 2;  // groups of V tiles
    u32x4 vf[2][VG];
    auto read_v = [&](int q) {
#pragma unroll
      for (int t = 0; t < VG; ++t)
        vf[q % 2][t] = *reinterpret_cast<const u32x4*>(&st.v[q / 2][q % 2 * VG + t][lane][0]);
    };
    read_v(0);
    // Keys past a row's position (those of no block lie past every position).
    if (!wave_full || j[kP4Step - 1] * kBlockSize + kBlockSize - 1 > first_pos) {
      asm volatile("");  // (a branch: as selects it costs every step 64 instructions)
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
      mx = __builtin_elementwise_maximum(mx, sc[r][3][3]);
      if (__ballot(mx > rise[r])) {
        const float m_new = fmaxf(m_run[r], max_xor32(max_xor16(mx)) * a.scale_log2);
        const float alpha = fast_exp2(m_run[r] - m_new);
        l_run[r] *= alpha;
        w_run[r] *= alpha;
        m_run[r] = m_new;
        rise[r] = (m_new + kLazy4) * inv_scale;
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
#pragma unroll
      for (int e = 0; e < kP4Step / 2; ++e)
#pragma unroll
        for (int k = 0; k < 4; ++k) w_run[r] = add_pair(pf[r][e][k], w_run[r]);
    }
#pragma unroll
    for (int q = 0; q < kGroups; ++q) {
      if (q + 1 < kGroups) read_v(q + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < VG; ++t)
#pragma unroll
        for (int r = 0; r < RT; ++r)
          acc[r][q % 2 * VG + t] = mfma16x16x32(as_bf16x8(vf[q % 2][t]), as_bf16x8(pf[r][q / 2]),
                                                acc[r][q % 2 * VG + t]);
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

  // A window's valid blocks in ascending order: counted, then (behind a barrier) listed.
  auto count_ids = [&](int p) {
    const uint64_t m = __ballot(p >= 0);
    if (lane == 0) wave_n[wave_all] = __popcll(m);
  };
  auto list_ids = [&](int p, int j) {
    const uint64_t m = __ballot(p >= 0);
    int before = 0, n = 0;
#pragma unroll
    for (int w = 0; w < kP4Halves * kP4Waves; ++w) {
      before += w < wave_all ? wave_n[w] : 0;
      n += wave_n[w];
    }
    if (p >= 0) {
      const int at = before + __popcll(m & ((1ull << lane) - 1ull));
      list_id[at] = p;
      list_j[at] = j;
    }
    if (tid < 2 * kP4Step) {  // the rest of the halves' last steps: no block
      list_id[n + tid] = -1;
      list_j[n + tid] = (INT_MAX - kBlockSize) / kBlockSize;
    }
    return n;
  };

  // The halves' results are joined through LDS: half h finishes row tile h of each wave
  // pair, the other half hands its part over. A lane's dims are 4 * VT neighbours:
  // (4 kgrp + i) * VT + t.
  static_assert(RT == kP4Halves, "a row tile a half");
  constexpr int kRow = D + 4;
  float* join = reinterpret_cast<float*>(&stage[0][0]);
  float* join_ml = join + kP4Rows * kRow;
  auto hand_over = [&](const f32x4(&x)[VT], float m, float l, int r) {
    const int row = 16 * RT * wave + 16 * r + col;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < VT; t += 4)
        *reinterpret_cast<f32x4*>(join + row * kRow + (4 * kgrp + i) * VT + t) =
            f32x4{x[t][i], x[t + 1][i], x[t + 2][i], x[t + 3][i]};
    if (kgrp == 0) {
      join_ml[2 * row] = m;
      join_ml[2 * row + 1] = l;
    }
  };
  auto finish = [&](const Unit4& u, int head, const f32x4(&x)[VT], float m, float l0, int r) {
    const int row0 = 16 * RT * wave + 16 * r;  // of this wave's 16 rows
    if (row0 >= u.rows) return;
    int position;
    const int64_t to = row_of(u, head, r, &position);
    float* mine = join + (row0 + col) * kRow;
    const float m1 = join_ml[2 * (row0 + col)], l1 = join_ml[2 * (row0 + col) + 1];
    const float M = fmaxf(m, m1);
    const float f0 = fast_exp2(m - M), f1 = fast_exp2(m1 - M);
    const float l = l0 * f0 + l1 * f1;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    f32x4 o[4][VT / 4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < VT / 4; ++t) {
        const f32x4 o1 = *reinterpret_cast<const f32x4*>(mine + (4 * kgrp + i) * VT + 4 * t);
        o[i][t] = f32x4{x[4 * t][i], x[4 * t + 1][i], x[4 * t + 2][i], x[4 * t + 3][i]} * f0 +
                  o1 * f1;
      }
    // The wave's rows go back into their places in LDS and out in whole rows: stored from
    // here, 8 bytes a lane and row, they took 12 us of the 4 x 512 tokens' 81.
    asm volatile("" ::: "memory");  // (each row's old contents are read by now)
    const bool whole = u.n_ranges == 1;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < VT / 4; ++t) {
        const int d = (4 * kgrp + i) * VT + 4 * t;
        if (whole) {
          const f32x4 v = o[i][t] * inv;
          *reinterpret_cast<u32x2*>(reinterpret_cast<uint16_t*>(mine) + d) =
              u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
        } else {
          *reinterpret_cast<f32x4*>(mine + d) = o[i][t];
        }
      }
    asm volatile("" ::: "memory");
    const int per_row = whole ? D / 8 : D / 4;  // lanes of 16 bytes
    for (int k = 0; k < per_row / 4; ++k) {
      const int row = k * (kWave / per_row) + lane / per_row, piece = lane % per_row;
      const u32x4 v = *reinterpret_cast<const u32x4*>(
          reinterpret_cast<const char*>(join + (row0 + row) * kRow) + 16 * piece);
      const int64_t q = static_cast<int64_t>(__shfl(static_cast<long long>(to), row));
      if (row0 + row < u.rows) {
        if (whole)
          *reinterpret_cast<u32x4*>(a.out + q * D + 8 * piece) = v;
        else
          *reinterpret_cast<u32x4*>(a.part_o + (q * a.ranges + u.range) * D + 4 * piece) = v;
      }
    }
    if (kgrp == 0 && row0 + col < u.rows) {
      if (!whole) {
        const int64_t at = to * a.ranges + u.range;
        a.part_ml[2 * at] = M;
        a.part_ml[2 * at + 1] = l;
      } else if (a.lse) {
        a.lse[to] = l == 0.f ? -INFINITY : (M + __log2f(l)) * kLn2;
      }
    }
  };

  // Units one after the other. What the next one starts from (its entry, its first
  // window's ids and tags, q) is read while this one runs (1% of the 4 x 512 tokens: a
  // second unit's chain of dependent loads otherwise shows between two units only).
  count_ids(id);
  __syncthreads();
  int n = list_ids(id, e.lo + tid);
  for (;;) {
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      m_run[r] = kNegBig4;
      l_run[r] = w_run[r] = 0.f;
      rise[r] = (kNegBig4 + kLazy4) * inv_scale;
#pragma unroll
      for (int t = 0; t < VT; ++t) acc[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int wrow = 16 * RT * wave;
    wave_full = wrow + 16 * RT <= e.rows;
    first_pos = e.prefix + (e.row0 + wrow) / a.group;
    last_pos =
        wrow < e.rows ? e.prefix + (e.row0 + min(wrow + 16 * RT, e.rows) - 1) / a.group : -1;
    __syncthreads();

    Unit4 next;
    int next_id = -1, next_tag = 0;
    for (int w0 = e.lo;;) {
      // step 2 i + half is this half's i-th
      const int steps = (n + kP4Halves * kP4Step - 1) / (kP4Halves * kP4Step);
      const int mine = kP4Step * (kP4Halves * lane + half);  // (lanes past `steps`: unused)
      my_id = list_id[mine + wave];
      my_j4 = *reinterpret_cast<const int4*>(&list_j[mine]);
      Codes4<D> c;
      if (steps > 0) load(c, 0);
      const bool start = w0 == e.lo;
      if (start) {
        next = read_unit(unit_of(pass + 1));
        if (next.b >= 0) next_id = read_id(next, next.lo + tid);
      }
      if (steps > 0) unpack(c, stage[half][0], 0);
      if (start && next.b >= 0) next_tag = read_tag(next_id);
      if (steps > 1) load(c, 1);
      __syncthreads();
      for (int i = 0; i < steps; ++i) {
        if (i + 1 < steps) {
          unpack(c, stage[half][(i + 1) % 2], i + 1);
          if (i + 2 < steps) load(c, i + 2);
        }
        compute(stage[half][i % 2], i);
        __syncthreads();
      }
      w0 += kP4Window;
      if (w0 >= e.hi) break;
      int p = read_id(e, w0 + tid);
      if (read_tag(p) != e.rv) p = -1;
      count_ids(p);
      __syncthreads();
      n = list_ids(p, w0 + tid);
      __syncthreads();
    }

    const int next_g = static_cast<int>(unit_of(pass + 1) % static_cast<uint32_t>(a.Hkv));
    if (next.b >= 0) {
      read_q(next, next_g);
      id = next_tag == next.rv ? next_id : -1;
      count_ids(id);
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      l_run[r] += __shfl_xor(l_run[r], 16);
      l_run[r] += __shfl_xor(l_run[r], 32);
      const float fit = rounded_fit(l_run[r], sum_kgroups(w_run[r]));
#pragma unroll
      for (int t = 0; t < VT; ++t) acc[r][t] *= fit;
    }
    if (half == 0)
      hand_over(acc[1], m_run[1], l_run[1], 1);
    else
      hand_over(acc[0], m_run[0], l_run[0], 0);
    __syncthreads();
    if (half == 0)
      finish(e, g, acc[0], m_run[0], l_run[0], 0);
    else
      finish(e, g, acc[1], m_run[1], l_run[1], 1);
    if (next.b < 0) return;
    n = list_ids(id, next.lo + tid);
    e = next;
    g = next_g;
    ++pass;
  }
}

__device__ __forceinline__ void write_row(const Prefill4Args& a, int64_t q, int d, int D,
                                          f32x4 num, float M, float den) {
  num *= den == 0.f ? 0.f : 1.f / den;
  *reinterpret_cast<u32x2*>(a.out + q * D + d) =
      u32x2{pack_bf16x2(num[0], num[1]), pack_bf16x2(num[2], num[3])};
  if (d == 0 && a.lse) a.lse[q] = den == 0.f ? -INFINITY : (M + __log2f(den)) * kLn2;
}

// Joins the n parts (key ranges) of dims d .. d + 3 of row q (token * Hq + query head).
template <int D, int kBatch>
__device__ __forceinline__ void merge_row(const Prefill4Args& a, int64_t q, int d, int n) {
  const float2* ml = reinterpret_cast<const float2*>(a.part_ml + q * a.ranges * 2);
  const float* po = a.part_o + q * a.ranges * D + d;
  // every part's loads in flight at once, kBatch at a time (up to 8 it stops at the last;
  // 16 as branches would take 110 registers)
  float M = kNegBig4, den = 0.f;
  f32x4 num = {0.f, 0.f, 0.f, 0.f};
  for (int p = 0; p < n; p += kBatch) {
    float2 m[kBatch];
    f32x4 o[kBatch];
#pragma unroll
    for (int r = 0; r < kBatch; ++r) {
      const int at_r = min(p + r, n - 1);
      m[r] = ml[at_r];
      o[r] = *reinterpret_cast<const f32x4*>(po + static_cast<int64_t>(at_r) * D);
    }
    float top = M;
#pragma unroll
    for (int r = 0; r < kBatch; ++r) top = fmaxf(top, m[r].x);
    const float f = fast_exp2(M - top);
    den *= f;
    num *= f;
#pragma unroll
    for (int r = 0; r < kBatch; ++r) {
      if (kBatch <= 8 && p + r >= n) break;
      const float w = kBatch <= 8 || p + r < n ? fast_exp2(m[r].x - top) : 0.f;
      den += m[r].y * w;
      num += o[r] * w;
    }
    M = top;
  }
  write_row(a, q, d, D, num, M, den);
}

// Joins the key ranges of the tiles that have more than one: a thread takes 4 dims of a
// row, a workgroup the rows that its threads make.
template <int D>
constexpr int merge_rows() { return kApThreads / (D / 4); }

template <int D>
__global__ __launch_bounds__(kApThreads) void merge_kv4_kernel(Prefill4Args a) {
  const int g = blockIdx.x % a.Hkv;
  const int rest = blockIdx.x / a.Hkv;
  constexpr int kParts = kP4Rows / merge_rows<D>();
  const int4 e = a.tiles[rest / kParts];
  const int r0 = e.x, row0 = e.y, rows = e.z, n = e.w;
  const int row = rest % kParts * merge_rows<D>() + threadIdx.x / (D / 4);
  const int d = 4 * (threadIdx.x % (D / 4));
  if (n == 1 || row >= rows) return;
  const int at = row0 + row;
  const int64_t q = static_cast<int64_t>(r0 + at / a.group) * a.Hq + g * a.group + at % a.group;
  merge_row<D, 8>(a, q, d, n);
}

// ---------------------------------------------------------------- few rows
// Requests that bring few rows each (a token or a few behind a long context) leave most
// of a 128-row tile empty, and their time is that of reading the cache: as in decode, one
// wave (or two or four, whose results meet in LDS) takes 16 rows of a request and KV head
// over a partition of the blocks, in its registers (kv4_attn.hpp). A request with
// more rows takes several such units, which read the same blocks.
constexpr int kFewRows = 16;

// The slot-th tile of kFewRows rows: requests in order. Every lane returns the same;
// false past the last.
struct FewTile {
  int b, r0, L;
  int row0, rows;  // of the request's (token, query head of the group) rows
  int prefix;      // cached tokens before the chunk
  int first;       // position of the first row
  int blocks;      // blocks that the last row sees
};

__device__ bool find_few(const Prefill4Args& a, int slot, FewTile* t) {
  const int lane = threadIdx.x % kWave;
  for (int b0 = 0; b0 < a.B; b0 += kWave) {
    int n = 0, r0 = 0, rows = 0, L = 0;
    if (b0 + lane < a.B) {
      r0 = a.q_indptr[b0 + lane];
      const int r1 = a.q_indptr[b0 + lane + 1];
      L = a.ctx_lens[b0 + lane];
      if (rows_ok4(r0, r1, a.T)) rows = (r1 - r0) * a.group;
      n = (rows + kFewRows - 1) / kFewRows;
    }
    int incl = n;
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
      const int up = __shfl_up(incl, off);
      if (lane >= off) incl += up;
    }
    const uint64_t past = __ballot(incl > slot);
    if (past) {
      const int l = __builtin_ctzll(past);
      rows = __builtin_amdgcn_readlane(rows, l);
      t->b = b0 + l;
      t->r0 = __builtin_amdgcn_readlane(r0, l);
      t->L = __builtin_amdgcn_readlane(L, l);
      t->row0 = (slot - __builtin_amdgcn_readlane(incl - n, l)) * kFewRows;
      t->rows = min(kFewRows, rows - t->row0);
      t->prefix = t->L - rows / a.group;
      t->first = t->prefix + t->row0 / a.group;
      const int last = t->prefix + (t->row0 + t->rows - 1) / a.group;
      t->blocks = last < 0 ? 0 : min(last / kBlockSize + 1, a.max_blocks);
      return true;
    }
    slot -= __builtin_amdgcn_readlane(incl, kWave - 1);
  }
  return false;
}

// Blocks of a partition of a tile that sees so many: as in decode where the call's ranges
// hold them, else as many times 64 as they need (the host bounds the ranges by what the
// table's width would leave of partial results; most contexts are shorter than that).
__device__ __forceinline__ int few_part(const Prefill4Args& a, int blocks) {
  if (blocks <= a.ranges * a.pb) return a.pb;
  return (blocks + kWave * a.ranges - 1) / (kWave * a.ranges) * kWave;
}

// Row r of a tile: token * Hq + query head.
__device__ __forceinline__ int64_t few_row(const Prefill4Args& a, const FewTile& t, int g, int r) {
  const int at = t.row0 + r;
  return static_cast<int64_t>(t.r0 + at / a.group) * a.Hq + g * a.group + at % a.group;
}

template <int D, int W>
__global__ __launch_bounds__(kWave* W, 3) void few_kv4_kernel(Prefill4Args a) {
  using L4 = Kv4<D>;
  constexpr int DEPTH = 2;  // pairs of blocks in registers
  const int lane = threadIdx.x % kWave, col = lane % 16, kgrp = lane / 16;
  const int wave = W == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int g = blockIdx.x % a.Hkv;
  const int rest = blockIdx.x / a.Hkv;
  const int part = rest % a.ranges;
  FewTile t;
  if (!find_few(a, rest / a.ranges, &t)) return;
  const int pb = few_part(a, t.blocks);
  const int n_parts = max(1, (t.blocks + pb - 1) / pb);
  if (part >= n_parts) return;
  // Partitions count from the end, as in decode.
  const int jend = t.blocks - part * pb, j0 = max(0, jend - pb);
  const int32_t* table = a.block_table + static_cast<int64_t>(t.b) * a.max_blocks;
  const int rv = a.req_version[t.b];
  // A group of 64 blocks from jg on, a lane each: this wave's share of the valid ones.
  int jg = j0, my_phys = 0;
  uint64_t valid = 0ull;
  auto take = [&](int id) {
    const bool ok =
        jg + lane < jend && id >= 0 && id < a.num_blocks && a.block_version[id] == rv;
    my_phys = ok ? id : 0;  // an id outside the pool is never dereferenced
    const uint64_t all = __ballot(ok);
    valid = all;
    if (W > 1) valid = __ballot(ok && __popcll(all & ((1ull << lane) - 1ull)) % W == wave);
  };
  auto read_id = [&](int j) { return j + lane < jend ? table[j + lane] : -1; };
  take(read_id(jg));

  Attn4<D> at;
  const bool in = col < t.rows;
  at.load_q(a.q + (in ? few_row(a, t, g, col) : 0) * D, in, a.q_xor, a.q_and);
  const float inv_scale = 1.f / a.scale_log2;
  at.init(inv_scale);
  const int pos = in ? t.prefix + (t.row0 + col) / a.group : INT_MAX - kBlockSize;

  auto next_block = [&]() -> int {
    if (!valid) return -1;
    const int i = __builtin_ctzll(valid);
    valid &= valid - 1;
    return i;
  };
  // V of a block at the end of what is seen: slots past the context's end, and tokens that
  // are not finite, as zeros; returns the latter for the group of this lane's output dims.
  auto settle = [&](Regs4<D>& R, int e, int j) {
    uint32_t odd = 0u, bad = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t byte = 0xffu << (8 * i);
      const bool dead = j * kBlockSize + 4 * kgrp + i >= t.L, is = (R.vs[e] & byte) == byte;
      if (is && !dead) odd |= 1u << i;
      if (is || dead) {
        R.vs[e] &= ~byte;
        if constexpr (D == 128)
          R.v[e][i] = 0u;
        else
          R.v[e][i / 2] &= ~(0xffffu << (16 * (i % 2)));
      }
    }
    if (__ballot(odd != 0u)) {
      const int from = L4::k_group(kgrp) * (16 / L4::kGroups);  // a column of the group
      for (int kg = 0; kg < 4; ++kg) bad |= __shfl(odd, kg * 16 + from) << (4 * kg);
    }
    return bad;
  };
  auto compute = [&](Regs4<D>& R, int i0, int i1) {
    f32x4 sc[2];
    bool hit = false;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int i = e ? i1 : i0, j = jg + i;
      // a block that some row sees in part, or none
      const bool tail = i < 0 || j * kBlockSize + kBlockSize - 1 > t.first;
      const int seen = i < 0 ? 0 : min(max(pos - j * kBlockSize + 1, 0), kBlockSize);
      if (tail && i >= 0) hit |= (settle(R, e, j) & ((1u << seen) - 1u)) != 0u;
      sc[e] = at.scores(R, e);
      if (tail) {
#pragma unroll
        for (int k = 0; k < 4; ++k) sc[e][k] = 4 * kgrp + k < seen ? sc[e][k] : -INFINITY;
      }
    }
    float ps[2];
    u32x4 pf;
    at.weigh(sc, a.scale_log2, inv_scale, ps, pf);
    at.values(R, pf);
    if (hit) {
      const float nan = __builtin_nanf("");
#pragma unroll
      for (int k = 0; k < D / 16; ++k) at.acc[k] = f32x4{nan, nan, nan, nan};
    }
  };

  Regs4<D> R[DEPTH];
  int i0[DEPTH], i1[DEPTH];
  auto fill = [&](int d) {
    i0[d] = next_block();
    i1[d] = next_block();
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int i = e ? i1[d] : i0[d];
      const int p = i >= 0 ? __builtin_amdgcn_readlane(my_phys, i) : 0;
      load_block4<D>(R[d], e, a.kv4, static_cast<int64_t>(p) * a.Hkv + g, i >= 0);
    }
  };
  for (;;) {
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
    jg += kWave;
    if (jg >= jend) break;
    take(read_id(jg));
  }

  extern __shared__ __attribute__((aligned(16))) float mg[];
  at.template finish<W>(t.rows, mg, [&](int r, int d, f32x4 num, float M, float den) {
    const int64_t q = few_row(a, t, g, r);
    if (n_parts == 1) {
      write_row(a, q, d, D, num, M, den);
    } else {
      const int64_t to = q * a.ranges + part;
      *reinterpret_cast<f32x4*>(a.part_o + to * D + d) = num;
      if (d == 0) {
        a.part_ml[2 * to] = M;
        a.part_ml[2 * to + 1] = den;
      }
    }
  });
}

template <int D>
__global__ __launch_bounds__(kFewRows* D / 4) void few_merge_kernel(Prefill4Args a) {
  FewTile t;
  if (!find_few(a, blockIdx.x / a.Hkv, &t)) return;
  const int pb = few_part(a, t.blocks), n = (t.blocks + pb - 1) / pb;
  if (n <= 1) return;
  const int row = threadIdx.x / (D / 4);
  if (row >= t.rows) return;
  const int64_t q = few_row(a, t, blockIdx.x % a.Hkv, row);
  // (8 and 16 at a time: one request of 8 tokens behind 4000 18.8 and 16.1 us, 5 requests
  // of 56 to 242 tokens, of 2 or 3 partitions, 28.5 and 30.5)
  const int d = 4 * (threadIdx.x % (D / 4));
  if (n <= 8)
    merge_row<D, 8>(a, q, d, n);
  else
    merge_row<D, 16>(a, q, d, n);
}

template <int D>
void launch_few(const Prefill4Args& a, unsigned grid, int W, hipStream_t s) {
  const int lds = join4_bytes<D>(W, kFewRows);
  if (W == 4)
    few_kv4_kernel<D, 4><<<grid, 4 * kWave, lds, s>>>(a);
  else if (W == 2)
    few_kv4_kernel<D, 2><<<grid, 2 * kWave, lds, s>>>(a);
  else
    few_kv4_kernel<D, 1><<<grid, kWave, 0, s>>>(a);
}

template <int D>
local_status_t launch_prefill_kv4(const Prefill4Args& a, hipStream_t s) {
  const char* who = "paged_attn_prefill_kv4";
  const int64_t units = static_cast<int64_t>(a.max_tiles) * a.ranges * a.Hkv;
  // blocks that hold a chunk's tokens: at most one more than the chunk fills, each side
  const int64_t blocks = a.T / kBlockSize + 2 * static_cast<int64_t>(a.B);
  const int64_t append = 1 + (blocks * a.Hkv + kApWaves - 1) / kApWaves;
  const int64_t per_tile = a.pb ? 1 : kP4Rows / merge_rows<D>();
  const int64_t merge = a.ranges > 1 ? a.max_tiles * per_tile * a.Hkv : 0;
  if (units >= (1LL << 31) || append >= (1LL << 31) || merge >= (1LL << 31))
    return local_fail(LOCAL_ERR_UNSUPPORTED, "%s: %lld units, grids of %lld and %lld workgroups",
                      who, (long long)units, (long long)append, (long long)merge);
  if (a.k_new)
    append_kv4_kernel<D><<<static_cast<unsigned>(append), kApThreads, 0, s>>>(a);
  else if (a.plan)
    plan_kv4_kernel<<<1, kApThreads, 0, s>>>(a);
  if (a.pb) {
    launch_few<D>(a, static_cast<unsigned>(units), units < 1536 ? 4 : units < 5120 ? 2 : 1, s);
    if (merge)
      few_merge_kernel<D><<<static_cast<unsigned>(merge), kFewRows * D / 4, 0, s>>>(a);
  } else {
    const int64_t grid = std::min<int64_t>(units, kP4Units);
    prefill_kv4_kernel<D><<<static_cast<unsigned>(grid), kP4Threads, 0, s>>>(a);
    if (merge) merge_kv4_kernel<D><<<static_cast<unsigned>(merge), kApThreads, 0, s>>>(a);
  }
  return local_check_launch(who);
}

// Calls of at most this many rows a request, on average, go by 16 rows. Measured in us by
// 16 rows / by 128, 8 KV heads of 4 query heads, 8 requests behind 500 to 8000 tokens: 16
// rows 28 / 42, 32 rows 37 / 41, 64 rows 49 / 42; 32 KV heads, 4 requests behind 100 to
// 2000: 16 rows 21 / 31, 32 rows 26 / 31, 64 rows 33 / 32.
//
// So do calls of more rows whose 16-row tiles, times KV heads, times entries of a request's
// table (a bound on the blocks that they unpack) are at most kFewWork: the plan and the
// 128-row workgroups' start and joins outlast their steps there. Over 140 calls of 1 to 8
// requests with 1 to 700 new tokens, 16 rows take 0.60 to 1.03 of the time of 128 up to
// 32768 (one of 115 longer, 1.15), 0.72 to 1.66 beyond.
constexpr int kFewMeanRows = 32;
constexpr int64_t kFewWork = 32768;

bool few_rows(int64_t all_rows, int B, int Hkv, int max_blocks) {
  return all_rows <= static_cast<int64_t>(B) * kFewMeanRows ||
         all_rows / kFewRows + B <= kFewWork / max_blocks / Hkv;
}

// Partitions that a tile of such a call may be split into: those of the whole table while
// they leave at most kFewPartials partial results, 136 MB at D = 128 (128 requests of 32
// tokens with 32 heads and a 1024-block table would ask for 1.1 GB); fewer beyond. Calls
// whose contexts are as long as their table take 0.98 to 1.00 of the time with the bound;
// where the table is wider, workgroups without a partition go too: 64 requests of 8 tokens
// behind up to 8000, 32/8 heads, 8192-block table, 156 us instead of 191, 100 single tokens
// behind up to 4000 104 instead of 134. (Partitions made longer by the table's width
// instead took those 314 and 183.)
constexpr int64_t kFewPartials = 1 << 18;

int few_ranges(int parts, int64_t rows) {  // rows: T * Hq
  return static_cast<int>(
      std::min<int64_t>(parts, std::max<int64_t>(1, kFewPartials / std::max<int64_t>(1, rows))));
}

// Key ranges that a tile of a call may be split into: as many as give every compute unit
// a workgroup where there are few tiles, counted from the sizes that the host knows.
int ranges_of_call(int64_t tiles, int Hkv, int max_blocks) {
  if (tiles == 0) return 1;
  const int64_t want = (2 * kP4Units + tiles * Hkv - 1) / (tiles * Hkv);
  const int least = least_range(tiles * Hkv);
  const int64_t most = std::max(1, (max_blocks + least / 2) / least);
  return static_cast<int>(std::min<int64_t>({want, most, kP4MaxRanges}));
}

// Tiles of a call; sets a's partitions (few rows) or else pb = 0, and its ranges.
int64_t tiles_of_call(Prefill4Args& a, int64_t all_rows, int B, int Hkv, int max_blocks) {
  const bool few = few_rows(all_rows, B, Hkv, max_blocks);
  // (B tiles more than the rows fill: each request's last one)
  const int64_t tiles = all_rows / (few ? kFewRows : kP4Rows) + B;
  a.pb = few ? part_blocks(max_blocks, tiles * Hkv) : 0;
  a.ranges = few ? few_ranges(parts_of_table(max_blocks, a.pb), all_rows * Hkv)
                 : ranges_of_call(tiles, Hkv, max_blocks);
  return tiles;
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
  const int64_t tiles = tiles_of_call(a, T * (Hq / Hkv), B, Hkv, max_blocks);
  if (tiles * kP4MaxRanges >= (1LL << 31))
    return local_fail(LOCAL_ERR_UNSUPPORTED, "%s: T=%lld B=%d", who, (long long)T, B);
  a.max_tiles = static_cast<int>(tiles);
  const bool few = a.pb != 0;
  const size_t rows = static_cast<size_t>(T) * Hq * (a.ranges > 1 ? a.ranges : 0);
  const size_t tiles_at = few ? 0 : sizeof(Unit4) * tiles * a.ranges;
  const size_t part_at = few ? 0 : align256(tiles_at + sizeof(int4) * tiles);
  // (never 0: a caller's allocation of nothing may be NULL, which asks for the size)
  const size_t need = std::max<size_t>(part_at + rows * (D + 2) * sizeof(float), 256);
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
  a.plan = few ? nullptr : reinterpret_cast<int4*>(base);
  a.tiles = few ? nullptr : reinterpret_cast<int4*>(base + tiles_at);
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

// What a call's size selects: the most key ranges of a tile, with 16 rows at a time plus 1000
// times the blocks of a partition, with 128 rows negative (for the tests, which name the form
// that they mean; not in local.h).
extern "C" int32_t localk_prefill_kv4_form(int64_t T, int32_t B, int32_t Hq, int32_t Hkv,
                                           int32_t max_blocks) {
  Prefill4Args a{};
  tiles_of_call(a, T * (Hq / Hkv), B, Hkv, max_blocks);
  return a.pb ? a.ranges + 1000 * a.pb : -a.ranges;
}
