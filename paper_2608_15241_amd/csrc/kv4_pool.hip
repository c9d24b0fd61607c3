// local_kv4_pool_import / local_kv4_pool_export: blocks of the bf16 pool to the 4-bit
// pool and back, all or those of a list (block ids, slots and tags unchanged).
//
// Bound by HBM: a (block, KV head) is 64 D bytes in bf16 and 17 D in 4 bits; there is
// half a conversion a value beside them and the maxima of the groups. One wave takes
// one (block, KV head) and its lanes hold what they hold in attention (kv4.hpp): of K
// the 16-byte pieces of one token, of V 4 tokens of D/16 dims, 8 bytes a dim. On
// the way out V goes through LDS, so that memory sees whole kilobytes: 32768 blocks of 8
// heads (D = 128) go in in 452 us and out in 469 (6.0 and 5.8 TB/s), out without it in 531.
#include "kv4.hpp"

namespace localk {
namespace {

constexpr int kPoolWaves = 4;

struct PoolArgs {
  uint16_t* k;
  uint16_t* v;
  uint8_t* kv4;
  const int32_t* ids;  // n block ids, or null: block i for i < n
  int64_t n, num_blocks;
  int Hkv;
};

// The tile (block * Hkv + head) of a wave, -1 for none (past the end, or an id outside
// the pool).
__device__ __forceinline__ int64_t pool_tile(const PoolArgs& a) {
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * kPoolWaves + threadIdx.x / kWave;
  const int64_t i = unit / a.Hkv;
  if (i >= a.n) return -1;
  const int64_t p = a.ids ? a.ids[i] : i;
  return p >= 0 && p < a.num_blocks ? p * a.Hkv + unit % a.Hkv : -1;
}

// A lane's codes of K or V: 16 or 8 bytes, aligned as the pool is.
template <int D>
__device__ __forceinline__ void get_codes(const uint8_t* p, uint32_t (&c)[D / 32]) {
  if constexpr (D == 128) {
    const u32x4 v = ld_global<u32x4>(p);
    c[0] = v.x, c[1] = v.y, c[2] = v.z, c[3] = v.w;
  } else {
    const u32x2 v = ld_global<u32x2>(p);
    c[0] = v.x, c[1] = v.y;
  }
}

template <int D>
__device__ __forceinline__ void put_codes(uint8_t* p, const uint32_t (&c)[D / 32]) {
  if constexpr (D == 128)
    *reinterpret_cast<u32x4*>(p) = u32x4{c[0], c[1], c[2], c[3]};
  else
    *reinterpret_cast<u32x2*>(p) = u32x2{c[0], c[1]};
}

// A wave's tile of V in LDS: D rows of 32 bytes (16 tokens), 16 bytes of padding behind
// the rows of one column of lanes, which spreads the lanes' rows over the banks.
template <int D>
struct VTile {
  static constexpr int kRows = D / 16;  // rows of a lane
  static constexpr int kBytes = 16 * (32 * kRows + 16);
  static __device__ __forceinline__ int at(int d, int byte) {
    return d * 32 + byte + d / kRows * 16;
  }
};

template <int D>
__global__ __launch_bounds__(kPoolWaves* kWave) void kv4_import_kernel(PoolArgs a) {
  using L4 = Kv4<D>;
  constexpr int VT = D / 16;
  const int64_t tile = pool_tile(a);
  if (tile < 0) return;
  const int lane = threadIdx.x % kWave, col = lane % 16, kgrp = lane / 16;
  const uint16_t* k = a.k + tile * (kBlockSize * D);
  const uint16_t* v = a.v + tile * (kBlockSize * D);
  uint8_t* o = a.kv4 + tile * L4::kTile;
  // K: token col, dims (D/4) kgrp ..
  u32x4 kv[D / 32];
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
    kv[c] = ld_stream<u32x4>(k + ((D / 32 * kgrp + c) * kBlockSize + col) * 8);
  // V: dims VT col .., tokens 4 kgrp .. (8 bytes of a row a lane; through LDS, as export
  // stores them, 477 us instead of 451)
  u32x2 vv[VT];
#pragma unroll
  for (int t = 0; t < VT; ++t)
    vv[t] = ld_global<u32x2>(v + (VT * col + t) * kBlockSize + 4 * kgrp);

  uint32_t kc[D / 32];
  const uint32_t ks = round_k<D>(kv, kc);
  put_codes<D>(o + lane * L4::kLane, kc);
  if (D == 128 || kgrp % 2 == 0)
    o[L4::k_scale(L4::k_group(kgrp), col)] = static_cast<uint8_t>(ks);

  uint32_t vs = 0u, code[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {  // token e of the lane's four: its dims as pairs
    u32x4 y = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < VT / 2; ++i) {
      const uint32_t w0 = e < 2 ? vv[2 * i].x : vv[2 * i].y;
      const uint32_t w1 = e < 2 ? vv[2 * i + 1].x : vv[2 * i + 1].y;
      y[i] = __builtin_amdgcn_perm(w1, w0, e % 2 ? 0x07060302u : 0x05040100u);
    }
    vs |= round_v<D>(y, code[e]) << (8 * e);
  }
  uint32_t vc[D / 32];
  if constexpr (D == 128) {
#pragma unroll
    for (int e = 0; e < 4; ++e) vc[e] = code[e];
  } else {
    vc[0] = (code[0] & 0xffffu) | code[1] << 16;
    vc[1] = (code[2] & 0xffffu) | code[3] << 16;
  }
  put_codes<D>(o + L4::kV + lane * L4::kLane, vc);
  if (col % (16 / L4::kGroups) == 0)
    *reinterpret_cast<uint32_t*>(o + L4::v_scale(L4::v_group(col), 4 * kgrp)) = vs;
}

template <int D>
__global__ __launch_bounds__(kPoolWaves* kWave) void kv4_export_kernel(PoolArgs a) {
  using L4 = Kv4<D>;
  constexpr int VT = D / 16;
  const int64_t tile = pool_tile(a);
  if (tile < 0) return;
  const int lane = threadIdx.x % kWave, col = lane % 16, kgrp = lane / 16;
  uint16_t* k = a.k + tile * (kBlockSize * D);
  uint16_t* v = a.v + tile * (kBlockSize * D);
  const uint8_t* o = a.kv4 + tile * L4::kTile;
  uint32_t kc[D / 32], vc[D / 32];
  get_codes<D>(o + lane * L4::kLane, kc);
  get_codes<D>(o + L4::kV + lane * L4::kLane, vc);
  const float ks = scale4(o[L4::k_scale(L4::k_group(kgrp), col)]);
  const uint32_t vs = ld_global<uint32_t>(o + L4::v_scale(L4::v_group(col), 4 * kgrp));
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
    *reinterpret_cast<u32x4*>(k + ((D / 32 * kgrp + c) * kBlockSize + col) * 8) =
        u32x4{unpack4<0>(kc[c], ks), unpack4<1>(kc[c], ks), unpack4<2>(kc[c], ks),
              unpack4<3>(kc[c], ks)};
  u32x2 x[VT];
  unpack_v<D>(vc, vs, x);
  __shared__ __attribute__((aligned(16))) char lds[kPoolWaves][VTile<D>::kBytes];
  char* mine = lds[threadIdx.x / kWave];
#pragma unroll
  for (int t = 0; t < VT; ++t)
    *reinterpret_cast<u32x2*>(mine + VTile<D>::at(VT * col + t, 8 * kgrp)) = x[t];
  asm volatile("" ::: "memory");  // (the wave's own rows: its accesses stay in order)
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    const int piece = c * kWave + lane;
    const u32x4 row =
        *reinterpret_cast<const u32x4*>(mine + VTile<D>::at(piece / 2, piece % 2 * 16));
    __builtin_nontemporal_store(row, reinterpret_cast<u32x4*>(v + piece * 8));
  }
}

local_status_t pool4_convert(bool import, PoolArgs a, int D, int block_size, void* stream) {
  const char* who = import ? "kv4_pool_import" : "kv4_pool_export";
  if (a.num_blocks < 0 || a.n < -1 || a.Hkv < 1)
    return local_fail(LOCAL_ERR_SHAPE, "%s: num_blocks=%lld n_ids=%lld Hkv=%d", who,
                      (long long)a.num_blocks, (long long)a.n, a.Hkv);
  if (block_size != kBlockSize || (D != 64 && D != 128))
    return local_fail(LOCAL_ERR_UNSUPPORTED, "%s: block_size=%d D=%d (need 16, 64|128)", who,
                      block_size, D);
  if (a.n < 0) {
    a.ids = nullptr;
    a.n = a.num_blocks;
  } else if (a.n > 0 && !a.ids) {
    return local_fail(LOCAL_ERR_NULL, "%s: block_ids is NULL for %lld ids", who, (long long)a.n);
  }
  if (a.n == 0 || a.num_blocks == 0) return LOCAL_OK;
  if (!a.k || !a.v || !a.kv4)
    return local_fail(LOCAL_ERR_NULL, "%s: NULL pointer argument", who);
  if (!aligned16(a.k) || !aligned16(a.v) || !aligned16(a.kv4))
    return local_fail(LOCAL_ERR_UNSUPPORTED, "%s: the pools must start on 16 bytes", who);
  // (in 64 bits: num_blocks < 2^31 blocks of ids, at most 2^31 - 1 heads)
  if (a.num_blocks >= (1LL << 31) || a.n > (1LL << 40) / a.Hkv)
    return local_fail(LOCAL_ERR_UNSUPPORTED, "%s: num_blocks=%lld n_ids=%lld Hkv=%d", who,
                      (long long)a.num_blocks, (long long)a.n, a.Hkv);
  const size_t tiles = static_cast<size_t>(a.num_blocks) * a.Hkv;
  const size_t wide = tiles * kBlockSize * D * sizeof(uint16_t), narrow = tiles * 17 * D;
  if (overlap(a.k, wide, a.v, wide) || overlap(a.k, wide, a.kv4, narrow) ||
      overlap(a.v, wide, a.kv4, narrow))
    return local_fail(LOCAL_ERR_SHAPE, "%s: the pools overlap", who);
  const int64_t grid = (a.n * a.Hkv + kPoolWaves - 1) / kPoolWaves;
  if (grid >= (1LL << 31))
    return local_fail(LOCAL_ERR_UNSUPPORTED, "%s: grid of %lld workgroups", who, (long long)grid);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const unsigned wgs = static_cast<unsigned>(grid);
  constexpr int threads = kPoolWaves * kWave;
  if (import)
    D == 64 ? kv4_import_kernel<64><<<wgs, threads, 0, s>>>(a)
            : kv4_import_kernel<128><<<wgs, threads, 0, s>>>(a);
  else
    D == 64 ? kv4_export_kernel<64><<<wgs, threads, 0, s>>>(a)
            : kv4_export_kernel<128><<<wgs, threads, 0, s>>>(a);
  return local_check_launch(who);
}

}  // namespace
}  // namespace localk

using namespace localk;

extern "C" local_status_t local_kv4_pool_import(const uint16_t* k_cache, const uint16_t* v_cache,
                                                int64_t num_blocks, int32_t Hkv, int32_t D,
                                                int32_t block_size, const int32_t* block_ids,
                                                int64_t n_ids, uint8_t* kv4, void* stream) {
  const PoolArgs a = {const_cast<uint16_t*>(k_cache), const_cast<uint16_t*>(v_cache), kv4,
                      block_ids, n_ids, num_blocks, Hkv};
  return pool4_convert(true, a, D, block_size, stream);
}

extern "C" local_status_t local_kv4_pool_export(const uint8_t* kv4, int64_t num_blocks,
                                                int32_t Hkv, int32_t D, int32_t block_size,
                                                const int32_t* block_ids, int64_t n_ids,
                                                uint16_t* k_cache, uint16_t* v_cache,
                                                void* stream) {
  const PoolArgs a = {k_cache, v_cache, const_cast<uint8_t*>(kv4), block_ids, n_ids,
                      num_blocks, Hkv};
  return pool4_convert(false, a, D, block_size, stream);
}
