// local_paged_attn_prefill_kv4: a chunk of new tokens per request is put into the
// 4-bit pool, then attends causally over cached prefix plus chunk.
//
// Mathematics: as prefill attention over the bf16 pool, with K^ and V^ the values that
// the codes stand for (the chunk's own tokens too); those are exact in bf16.
//
// Bound by the matrix cores and the softmax's vector instructions; the pool's 4-bit
// tiles make the memory side four times lighter than bf16, at the price of unpacking.
//  * A workgroup takes 128 rows of one request and one KV head, a row being a (token,
//    query head of the group): every query head of the group shares what is unpacked.
//    4 waves of 32 rows.
//  * 64 keys a step: each wave unpacks a quarter of the step's K and V into LDS, in
//    the order of the matrix operands (lane l's 16 bytes at 16 l), so that every LDS
//    access is a contiguous kilobyte a wave. Two buffers: the codes of step s + 2 load
//    into registers while step s + 1 is unpacked and step s is computed; one barrier a
//    step.
//  * S^T = K Q^T, O^T += V^T P^T on v_mfma_f32_16x16x32_bf16, as in decode.
//  * Calls with few tiles split each tile's keys into ranges, joined by a merge launch.
//  * An infinity or a NaN in V (scale byte 255) must reach the rows that see its token
//    and no other, which 0 * NaN in a product would not do: its values enter the
//    product as zeros, and a mask of such tokens then puts NaN into those rows.
#include <algorithm>
#include <climits>

#include "kv4.hpp"

namespace localk {
namespace {

constexpr int kP4Waves = 4;
constexpr int kP4Threads = kP4Waves * kWave;
constexpr int kP4RowTiles = 2;                         // 16-row tiles of a wave
constexpr int kP4Rows = kP4Waves * 16 * kP4RowTiles;   // rows of a workgroup
constexpr int kP4Step = 4;                             // blocks a step
constexpr int kP4Window = kP4Threads;                  // table entries listed at a time
constexpr int kP4MinRange = 8;                         // blocks a key range has at least
constexpr int kP4MaxRanges = 16;
constexpr int kP4WantUnits = 512;                      // two workgroups a compute unit
constexpr float kP4NegBig = -1.0e30f;

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
  float* part_o;   // [T][Hq][ranges][D]
  float* part_ml;  // [T][Hq][ranges][2]
  int64_t T, num_blocks;
  int B, Hq, Hkv, group, max_blocks, ranges;
  float scale_log2;
};

__device__ __forceinline__ bool rows_ok4(int r0, int r1, int64_t T) {
  return r0 >= 0 && r1 >= r0 && r1 <= T;
}

// The request whose rows hold row t (the last one with q_indptr[b] <= t), or -1.
__device__ __forceinline__ int request_of(const Prefill4Args& a, int64_t t) {
  int lo = 0, hi = a.B;  // q_indptr[lo] <= t < q_indptr[hi] where the rows are in order
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a.q_indptr[mid] <= t)
      lo = mid;
    else
      hi = mid;
  }
  const int r0 = a.q_indptr[lo], r1 = a.q_indptr[lo + 1];
  return rows_ok4(r0, r1, a.T) && r0 <= t && t < r1 ? lo : -1;
}

// ---------------------------------------------------------------- append
// D/8 lanes a (token, KV head): each rounds 8 dims of K and 8 of V.
template <int D>
__global__ __launch_bounds__(kP4Threads) void append_kv4_kernel(Prefill4Args a) {
  using L4 = Kv4<D>;
  constexpr int kLanes = D / 8;
  const int64_t unit =
      (static_cast<int64_t>(blockIdx.x) * kP4Threads + threadIdx.x) / kLanes;
  const int i = threadIdx.x % kLanes;
  const int64_t t = unit / a.Hkv;
  const int g = static_cast<int>(unit % a.Hkv);
  const bool in = t < a.T;  // (no early exit: the lanes of a group exchange maxima)
  u32x4 kv = {0u, 0u, 0u, 0u}, vv = {0u, 0u, 0u, 0u};
  int p = -1, slot = 0;
  if (in) {
    const int b = request_of(a, t);
    if (b >= 0) {
      const int r0 = a.q_indptr[b], n = a.q_indptr[b + 1] - r0;
      const int pos = a.ctx_lens[b] - n + static_cast<int>(t - r0);
      if (pos >= 0 && pos / kBlockSize < a.max_blocks) {
        p = a.block_table[static_cast<int64_t>(b) * a.max_blocks + pos / kBlockSize];
        if (p >= a.num_blocks) p = -1;
        slot = pos % kBlockSize;
      }
    }
    if (p >= 0) {
      kv = ld_global<u32x4>(a.k_new + (t * a.Hkv + g) * D + 8 * i);
      vv = ld_global<u32x4>(a.v_new + (t * a.Hkv + g) * D + 8 * i);
    }
  }
  float x[8], y[8], mk = 0.f, mv = 0.f;
  split8(kv, x);
  split8(vv, y);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    mk = amax_bits(mk, x[e]);
    mv = amax_bits(mv, y[e]);
  }
  mk = amax_xor(amax_xor(mk, 1), 2);
  mv = amax_xor(amax_xor(mv, 1), 2);
  if (p < 0) return;
  const uint32_t ks = scale_byte(mk), vs = scale_byte(mv);
  uint8_t* tile = a.kv4 + (static_cast<int64_t>(p) * a.Hkv + g) * L4::kTile;
  // K: dims 8 i .. of the slot lie in k-group 8 i / (D/4)
  constexpr int kDims = D / 4;
  *reinterpret_cast<uint32_t*>(tile + (8 * i / kDims * kBlockSize + slot) * L4::kLane +
                               8 * i % kDims / 2) = pack4x8(x, ks);
  // V: in columns 8 i / (D/16) ..
  uint8_t* vo = tile + L4::kV;
  const uint32_t w = pack4x8(y, vs);
  if constexpr (D == 128) {
    *reinterpret_cast<uint32_t*>(vo + ((slot / 4 * 16 + i) * 4 + slot % 4) * 4) = w;
  } else {
    uint8_t* to = vo + ((slot / 4 * 16 + 2 * i) * 4 + slot % 4) * 2;
    *reinterpret_cast<uint16_t*>(to) = static_cast<uint16_t>(w);
    *reinterpret_cast<uint16_t*>(to + 8) = static_cast<uint16_t>(w >> 16);
  }
  if (i % 4 == 0) {
    tile[L4::k_scale(i / 4, slot)] = static_cast<uint8_t>(ks);
    tile[L4::v_scale(i / 4, slot)] = static_cast<uint8_t>(vs);
  }
}

// ---------------------------------------------------------------- units
// What a workgroup (or a merged row) has to know of its tile of 128 rows.
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

// Key ranges of a tile.
__device__ __forceinline__ int ranges_of(const Prefill4Args& a, int blocks) {
  return min(a.ranges, max(1, (blocks + kP4MinRange - 1) / kP4MinRange));
}

// The slot-th tile: requests in order, a request's tiles from its last. Every lane
// returns the same; false past the last.
__device__ bool find_tile(const Prefill4Args& a, int slot, int* b, int* tile) {
  const int lane = threadIdx.x % kWave;
  for (int b0 = 0; b0 < a.B; b0 += kWave) {
    int n = 0;
    if (b0 + lane < a.B) {
      const int r0 = a.q_indptr[b0 + lane], r1 = a.q_indptr[b0 + lane + 1];
      if (rows_ok4(r0, r1, a.T)) n = ((r1 - r0) * a.group + kP4Rows - 1) / kP4Rows;
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
      *b = b0 + l;
      *tile = __shfl(incl, l) - 1 - slot;
      return true;
    }
    slot -= __shfl(incl, kWave - 1);
  }
  return false;
}

// ---------------------------------------------------------------- attention
template <int D>
struct Codes4 {  // a wave's share of a step, as loaded
  uint32_t k[D / 32], v[2][D / 32];
  uint32_t ks, vs[2];
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
  u32x4 v[kP4Step / 2][D / 16][kWave];
  uint32_t nan[kP4Step / 2][4];  // by (pair, group): tokens whose V is not finite
};

template <int D>
__global__ __launch_bounds__(kP4Threads, 2) void prefill_kv4_kernel(Prefill4Args a) {
  using L4 = Kv4<D>;
  constexpr int KC = D / 32, VT = D / 16, RT = kP4RowTiles;
  __shared__ Stage4<D> stage[2];
  __shared__ int list_id[kP4Window + kP4Step], list_j[kP4Window + kP4Step];
  __shared__ int wave_n[kP4Waves];

  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int col = lane % 16, kgrp = lane / 16;
  const int g = blockIdx.x % a.Hkv;
  const int rest = blockIdx.x / a.Hkv;
  const int range = rest % a.ranges;
  int b, tile_i;
  if (!find_tile(a, rest / a.ranges, &b, &tile_i)) return;
  const Tile4 tl = tile_of(a, b, tile_i);
  const int n_ranges = ranges_of(a, tl.blocks);
  if (range >= n_ranges) return;
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
      qv[r][c] = as_bf16x8(v);
    }
  }
  // Positions of the wave's first and last row: bounds of what it may see.
  const int wrow = tl.row0 + 16 * RT * wave;
  const bool wave_in = 16 * RT * wave < tl.rows;
  const int first_pos = tl.prefix + wrow / a.group;
  const int last_pos =
      wave_in ? tl.prefix + (min(wrow + 16 * RT, tl.row0 + tl.rows) - 1) / a.group : -1;

  f32x4 acc[RT][VT];
  float m_run[RT], l_run[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    m_run[r] = kP4NegBig;
    l_run[r] = 0.f;
#pragma unroll
    for (int t = 0; t < VT; ++t) acc[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // Which quarter of a step this wave unpacks: K of block `wave`; V of the pair wave/2,
  // the half of its tiles that byte pair wave % 2 of a token's codes holds.
  const int pair = wave / 2, half = wave % 2;
  auto rsrc_of = [&](int at) {
    const int id = __builtin_amdgcn_readfirstlane(list_id[at]);
    const int64_t tile = (static_cast<int64_t>(max(id, 0)) * a.Hkv + g) * L4::kTile;
    return make_rsrc(a.kv4 + tile, id >= 0 ? L4::kTile : 0u);
  };
  auto load = [&](Codes4<D>& c, int s) {
    const __amdgpu_buffer_rsrc_t rk = rsrc_of(kP4Step * s + wave);
    load_cached<D>(rk, lane * L4::kLane, c.k);
    c.ks = __builtin_amdgcn_raw_buffer_load_b8(rk, L4::k_scale(L4::k_group(kgrp), col), 0, 0);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const __amdgpu_buffer_rsrc_t rv2 = rsrc_of(kP4Step * s + 2 * pair + e);
      load_cached<D>(rv2, L4::kV + lane * L4::kLane, c.v[e]);
      c.vs[e] = __builtin_amdgcn_raw_buffer_load_b32(
          rv2, L4::v_scale(L4::v_group(col), 4 * kgrp), 0, 0);
    }
  };
  auto unpack = [&](Codes4<D>& c, Stage4<D>& st, int s) {
    const float ks = scale4(c.ks);
#pragma unroll
    for (int i = 0; i < KC; ++i)
      st.k[wave][i][lane] = u32x4{unpack4<0>(c.k[i], ks), unpack4<1>(c.k[i], ks),
                                  unpack4<2>(c.k[i], ks), unpack4<3>(c.k[i], ks)};
    // V: slots past the context's end and tokens that are not finite as zeros
    uint32_t odd = 0u;  // bit 4 e + i: token 4 kgrp + i of block e
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int j = list_j[kP4Step * s + 2 * pair + e];
      const int live = L - j * kBlockSize - 4 * kgrp;  // (absent: far below 0)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t byte = 0xffu << (8 * i);
        const bool dead = i >= live, bad = (c.vs[e] & byte) == byte;
        if (bad && !dead) odd |= 1u << (4 * e + i);
        if (bad || dead) {
          c.vs[e] &= ~byte;
          if constexpr (D == 128)
            c.v[e][i] = 0u;
          else
            c.v[e][i / 2] &= ~(0xffffu << (16 * (i % 2)));
        }
      }
    }
    u32x2 va[VT], vb[VT];
    unpack_v<D>(c.v[0], c.vs[0], va);
    unpack_v<D>(c.v[1], c.vs[1], vb);
#pragma unroll
    for (int t = 0; t < VT; ++t)
      if (t / (VT / 2) == half)
        st.v[pair][t][lane] = u32x4{va[t].x, va[t].y, vb[t].x, vb[t].y};
    if (half == 0) {
      uint32_t mine = 0u;  // bit 16 e + token, for group `lane`
      if (__ballot(odd != 0u)) {
        const int at = lane % L4::kGroups * (16 / L4::kGroups);  // a column of the group
        for (int kg = 0; kg < 4; ++kg) {
          const uint32_t o = __shfl(odd, kg * 16 + at);
          mine |= (o & 15u) << (4 * kg) | (o >> 4) << (16 + 4 * kg);
        }
      }
      if (lane < L4::kGroups) st.nan[pair][lane] = mine;
    }
  };
  auto compute = [&](const Stage4<D>& st, int s) {
    int j[kP4Step], top = 0;
#pragma unroll
    for (int e = 0; e < kP4Step; ++e) {
      j[e] = __builtin_amdgcn_readfirstlane(list_j[kP4Step * s + e]);
      top = max(top, j[e]);
    }
    if (j[0] * kBlockSize > last_pos) return;  // (ascending: no key of the step is seen)
    const bool mask = top * static_cast<int64_t>(kBlockSize) + kBlockSize - 1 > first_pos ||
                      16 * RT * (wave + 1) > tl.rows;
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
    u32x4 pf[RT][kP4Step / 2];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      float mx = -INFINITY;
#pragma unroll
      for (int e = 0; e < kP4Step; ++e)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          float v = sc[r][e][k] * a.scale_log2;
          if (mask) {
            // keys of block j[e] that the row sees: those up to its position
            const int64_t key = static_cast<int64_t>(j[e]) * kBlockSize + 4 * kgrp + k;
            v = key <= pos[r] ? v : -INFINITY;
          }
          sc[r][e][k] = v;
          mx = fmaxf(mx, v);
        }
      mx = max_xor32(max_xor16(mx));
      const float m_new = fmaxf(m_run[r], mx);
      const float alpha = fast_exp2(m_run[r] - m_new);
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < kP4Step; ++e) {
        float p[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          p[k] = fast_exp2(sc[r][e][k] - m_new);
          sum += p[k];
        }
        pf[r][e / 2][2 * (e % 2)] = pack_bf16x2(p[0], p[1]);
        pf[r][e / 2][2 * (e % 2) + 1] = pack_bf16x2(p[2], p[3]);
      }
      l_run[r] = l_run[r] * alpha + sum;
      m_run[r] = m_new;
#pragma unroll
      for (int t = 0; t < VT; ++t) acc[r][t] *= alpha;
    }
#pragma unroll
    for (int pr = 0; pr < kP4Step / 2; ++pr)
#pragma unroll
      for (int t = 0; t < VT; ++t) {
        const bf16x8 vf = as_bf16x8(st.v[pr][t][lane]);
#pragma unroll
        for (int r = 0; r < RT; ++r)
          acc[r][t] = mfma16x16x32(vf, as_bf16x8(pf[r][pr]), acc[r][t]);
      }
    // Tokens whose V is not finite, in the rows that see them (a lane's dims all lie
    // in group kgrp * kGroups / 4).
#pragma unroll
    for (int pr = 0; pr < kP4Step / 2; ++pr) {
      const uint32_t bad = st.nan[pr][L4::k_group(kgrp)];
      if (!__ballot(bad != 0u)) continue;
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        uint32_t see = 0u;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int64_t n = pos[r] - static_cast<int64_t>(j[2 * pr + e]) * kBlockSize + 1;
          const int w = n < 0 ? 0 : n > kBlockSize ? kBlockSize : static_cast<int>(n);
          see |= ((1u << w) - 1u) << (16 * e);
        }
        if (see & bad) {
#pragma unroll
          for (int t = 0; t < VT; ++t)
            acc[r][t] = f32x4{__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""),
                              __builtin_nanf("")};
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
    if (lane == 0) wave_n[wave] = __popcll(m);
    __syncthreads();
    int before = 0, n = 0;
#pragma unroll
    for (int w = 0; w < kP4Waves; ++w) {
      before += w < wave ? wave_n[w] : 0;
      n += wave_n[w];
    }
    if (id >= 0) {
      const int at = before + __popcll(m & ((1ull << lane) - 1ull));
      list_id[at] = id;
      list_j[at] = j;
    }
    if (tid < kP4Step) {  // the rest of the last step: no block
      list_id[n + tid] = -1;
      list_j[n + tid] = INT_MAX / kBlockSize;
    }
    __syncthreads();
    const int steps = (n + kP4Step - 1) / kP4Step;
    if (steps > 0) {
      Codes4<D> c;
      load(c, 0);
      unpack(c, stage[0], 0);
      if (steps > 1) load(c, 1);
      __syncthreads();
      for (int s = 0; s < steps; ++s) {
        if (s + 1 < steps) {
          unpack(c, stage[(s + 1) % 2], s + 1);
          if (s + 2 < steps) load(c, s + 2);
        }
        compute(stage[s % 2], s);
        __syncthreads();
      }
    }
    __syncthreads();  // (the list is written again)
  }

  // ---- finish
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    float l = l_run[r];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    const int row = 16 * RT * wave + 16 * r + col;
    if (row >= tl.rows) continue;
    if (n_ranges == 1) {
      const float inv = l == 0.f ? 0.f : 1.f / l;
      uint16_t* o = a.out + qrow[r] * D;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int t = 0; t < VT; t += 4)
          *reinterpret_cast<u32x2*>(o + (4 * kgrp + i) * VT + t) =
              u32x2{pack_bf16x2(acc[r][t][i] * inv, acc[r][t + 1][i] * inv),
                    pack_bf16x2(acc[r][t + 2][i] * inv, acc[r][t + 3][i] * inv)};
      if (kgrp == 0 && a.lse)
        a.lse[qrow[r]] = l == 0.f ? -INFINITY : (m_run[r] + __log2f(l)) * kLn2;
    } else {
      const int64_t at = qrow[r] * a.ranges + range;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int t = 0; t < VT; t += 4)
          *reinterpret_cast<f32x4*>(a.part_o + at * D + (4 * kgrp + i) * VT + t) =
              f32x4{acc[r][t][i], acc[r][t + 1][i], acc[r][t + 2][i], acc[r][t + 3][i]};
      if (kgrp == 0) {
        a.part_ml[2 * at] = m_run[r];
        a.part_ml[2 * at + 1] = l;
      }
    }
  }
}

// Joins the key ranges of each (token, query head) that has more than one.
template <int D>
__global__ __launch_bounds__(D) void merge_kv4_kernel(Prefill4Args a) {
  const int64_t row = blockIdx.x;
  const int64_t t = row / a.Hq;
  const int d = threadIdx.x;
  const int b = request_of(a, t);
  if (b < 0) return;
  const int in_group = static_cast<int>(t - a.q_indptr[b]) * a.group +
                       static_cast<int>(row % a.Hq) % a.group;
  const int n = ranges_of(a, tile_of(a, b, in_group / kP4Rows).blocks);
  if (n == 1) return;
  const float* ml = a.part_ml + row * a.ranges * 2;
  const float* po = a.part_o + row * a.ranges * D;
  float M = kP4NegBig, den = 0.f, num = 0.f;
  for (int r = 0; r < n; ++r) M = fmaxf(M, ml[2 * r]);
  for (int r = 0; r < n; ++r) {
    const float f = fast_exp2(ml[2 * r] - M);
    den += ml[2 * r + 1] * f;
    num += po[static_cast<int64_t>(r) * D + d] * f;
  }
  a.out[row * D + d] = f32_to_bf16(den == 0.f ? 0.f : num / den);
  if (d == 0 && a.lse) a.lse[row] = den == 0.f ? -INFINITY : (M + __log2f(den)) * kLn2;
}

template <int D>
local_status_t launch_prefill_kv4(const Prefill4Args& a, hipStream_t s) {
  const char* who = "paged_attn_prefill_kv4";
  const int64_t tiles = a.T * a.group / kP4Rows + a.B;
  const int64_t grid = tiles * a.ranges * a.Hkv;
  const int64_t append = (a.T * a.Hkv * (D / 8) + kP4Threads - 1) / kP4Threads;
  const int64_t merge = a.ranges > 1 ? a.T * a.Hq : 0;
  if (grid >= (1LL << 31) || append >= (1LL << 31) || merge >= (1LL << 31))
    return local_fail(LOCAL_ERR_UNSUPPORTED, "%s: grids of %lld, %lld and %lld workgroups", who,
                      (long long)grid, (long long)append, (long long)merge);
  if (a.k_new) append_kv4_kernel<D><<<static_cast<unsigned>(append), kP4Threads, 0, s>>>(a);
  prefill_kv4_kernel<D><<<static_cast<unsigned>(grid), kP4Threads, 0, s>>>(a);
  if (merge) merge_kv4_kernel<D><<<static_cast<unsigned>(merge), D, 0, s>>>(a);
  return local_check_launch(who);
}

// Key ranges of a call: as many as give every compute unit two workgroups, counted
// from the sizes that the host knows.
int ranges_of_call(int64_t T, int B, int group, int Hkv, int max_blocks) {
  const int64_t units = (T * group / kP4Rows + B) * Hkv;
  const int64_t want = (kP4WantUnits + units - 1) / units;
  const int64_t most = (max_blocks + kP4MinRange - 1) / kP4MinRange;
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
  a.ranges = B > 0 && T > 0 ? ranges_of_call(T, B, Hq / Hkv, Hkv, max_blocks) : 1;
  const size_t rows = static_cast<size_t>(T) * Hq * (a.ranges > 1 ? a.ranges : 0);
  const size_t need = rows * (D + 2) * sizeof(float);
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
  a.part_o = static_cast<float*>(ws);
  a.part_ml = a.part_o + rows * D;
  a.T = T;
  a.num_blocks = num_blocks;
  a.B = B;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.group = Hq / Hkv;
  a.max_blocks = max_blocks;
  a.scale_log2 = sm_scale * kLog2e;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return D == 64 ? launch_prefill_kv4<64>(a, s) : launch_prefill_kv4<128>(a, s);
}
