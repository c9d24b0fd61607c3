// local_kv_evict: a request's blocks down to a budget, the ones that attention used
// least first (by accumulated weight), with the block table, the weights and the
// lengths closed up behind them.
//
// Bound by latency: a request is a row of a few hundred to a few thousand ids and
// weights. One workgroup takes one request: it reads the row and its blocks' tags once
// (the first block of each thread stays in registers, the keys in LDS), finds the weight
// of the last block that stays by radix selection (up to four histograms of 8 bits,
// integer counts, so the order of the atomics does not matter; it ends as soon as a
// digit's keys all stay), and closes the row up by prefix sums in ascending order, which
// reads every chunk before it writes at or below it and so works in place. Rows wider
// than 256 blocks get 1024 threads: 128 rows of up to 1024 blocks take 7.5 us replayed
// from a graph, 10.0 with 256 threads.
#include "common.hpp"

namespace localk {
namespace {

constexpr int kEvKeys = 8192;  // keys held in LDS; those of longer rows are formed again

struct EvictArgs {
  const int32_t* table;
  const int32_t* ctx_lens;
  const float* weight;
  const int32_t* keep;
  const int32_t* block_version;
  const int32_t* req_version;
  int32_t* table_out;
  int32_t* ctx_out;
  float* weight_out;
  int32_t* evicted;
  int32_t* n_evicted;
  int64_t num_blocks;
  int max_blocks, sink, recent;
};

// Exclusive prefix sum of a flag over the workgroup, and the total.
template <int THREADS>
__device__ __forceinline__ int flag_prefix(bool f, int* wave_sums, int* total) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const uint64_t m = __ballot(f);
  __syncthreads();  // (the sums of the call before have been read)
  if (lane == 0) wave_sums[wave] = __popcll(m);
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < THREADS / kWave; ++w) {
    before += w < wave ? wave_sums[w] : 0;
    all += wave_sums[w];
  }
  *total = all;
  return before + __popcll(m & ((1ull << lane) - 1ull));
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void kv_evict_kernel(EvictArgs a) {
  __shared__ uint32_t keys[kEvKeys];
  __shared__ int hist[256];
  __shared__ int wave_sums[THREADS / kWave];
  __shared__ int found[3];
  const int b = blockIdx.x, tid = threadIdx.x;
  const int64_t row = static_cast<int64_t>(b) * a.max_blocks;
  const int id0 = tid < a.max_blocks ? a.table[row + tid] : 0;  // this thread's first block
  const float w0 = tid < a.max_blocks ? a.weight[row + tid] : 0.f;
  const int L = a.ctx_lens[b];
  const int nb = L <= 0 ? 0 : min((L - 1) / kBlockSize + 1, a.max_blocks);
  const int rv = a.req_version[b];
  // Protected: the first `sink` and the last `recent` blocks.
  const int sink = min(a.sink, nb), late = max(sink, nb - a.recent);
  const int n_prot = sink + (nb - late);
  const int n_keep = min(nb, max(a.keep[b], n_prot));
  int need = n_keep - n_prot;  // blocks of [sink, late) that stay

  // Order of the blocks: by weight (what is not positive, NaN too, as 0), stale ones
  // below all.
  auto key = [&](int p, float w) -> uint32_t {
    if (p < 0 || p >= a.num_blocks || a.block_version[p] != rv) return 0u;
    return w > 0.f ? __float_as_uint(w) + 1u : 1u;
  };
  auto make_key = [&](int j) {
    return j == tid ? key(id0, w0) : key(a.table[row + j], a.weight[row + j]);
  };
  auto key_of = [&](int j) { return j < kEvKeys ? keys[j] : make_key(j); };

  // The need-th largest key (`least`) and how many of that key stay, lowest j first.
  const bool select = need > 0 && need < late - sink;
  uint32_t least = need > 0 ? 0u : 0xffffffffu;
  int of_least = need > 0 ? nb : 0;
  if (select) {
    for (int j = sink + tid; j < late; j += THREADS) {
      const uint32_t k = make_key(j);
      if (j < kEvKeys) keys[j] = k;
    }
    __syncthreads();
    least = 0u;
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      const uint32_t mask = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
      for (int j = sink + tid; j < late; j += THREADS) {
        const uint32_t k = key_of(j);
        if ((k & mask) == least) atomicAdd(&hist[k >> shift & 255u], 1);
      }
      __syncthreads();
      if (tid < kWave) {  // counts of the digits above: 4 digits a lane, from the top
        int c[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          c[i] = hist[255 - (4 * tid + i)];
          sum += c[i];
        }
        int incl = sum;
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
          const int up = __shfl_up(incl, off);
          if (tid >= off) incl += up;
        }
        int above = incl - sum;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (above < need && need <= above + c[i]) {
            found[0] = 255 - (4 * tid + i);
            found[1] = above;
            found[2] = c[i];
          }
          above += c[i];
        }
      }
      __syncthreads();
      least |= static_cast<uint32_t>(found[0]) << shift;
      need -= found[1];
      if (need == found[2]) {  // every key of this digit stays: those from `least` on
        need = nb;
        break;
      }
    }
    of_least = need;
  }

  // Close the row up, a block a thread at a time.
  int kept_at = 0, gone_at = 0, same_at = 0;
  for (int j0 = 0; j0 < nb; j0 += THREADS) {
    const int j = j0 + tid;
    const bool in = j < nb, held = in && (j < sink || j >= late);
    const uint32_t k = in && !held && select ? key_of(j) : 0u;
    const int id = j == tid ? id0 : in ? a.table[row + j] : 0;
    const float w = j == tid ? w0 : in ? a.weight[row + j] : 0.f;
    const bool same = in && !held && k == least;
    int n_same = 0, n_kept = 0;
    const int rank = same_at + flag_prefix<THREADS>(same, wave_sums, &n_same);
    const bool keep = held || (in && !held && (k > least || (same && rank < of_least)));
    const int at = kept_at + flag_prefix<THREADS>(keep, wave_sums, &n_kept);
    if (keep) {
      a.table_out[row + at] = id;
      a.weight_out[row + at] = w;
    } else if (in) {
      a.evicted[row + gone_at + (j - j0) - (at - kept_at)] = id;
    }
    same_at += n_same;
    kept_at += n_kept;
    gone_at += min(THREADS, nb - j0) - n_kept;
  }
  __syncthreads();
  for (int j = tid; j < a.max_blocks; j += THREADS) {
    if (j >= kept_at) {
      a.table_out[row + j] = -1;
      a.weight_out[row + j] = 0.f;
    }
    if (j >= gone_at) a.evicted[row + j] = -1;
  }
  if (tid == 0) {
    // (a length past the table's end, which owns no more blocks, counts as its end)
    const int64_t end = static_cast<int64_t>(kBlockSize) * a.max_blocks;
    a.ctx_out[b] = gone_at == 0 ? L
                                : static_cast<int>(min(static_cast<int64_t>(L), end) -
                                                   kBlockSize * gone_at);
    a.n_evicted[b] = gone_at;
  }
}

}  // namespace
}  // namespace localk

using namespace localk;

extern "C" local_status_t local_kv_evict(const int32_t* block_table, int32_t B,
                                         int32_t max_blocks, const int32_t* ctx_lens,
                                         int32_t block_size, const float* block_weight,
                                         const int32_t* keep_blocks, int32_t sink_blocks,
                                         int32_t recent_blocks, const int32_t* block_version,
                                         int64_t num_blocks, const int32_t* req_version,
                                         int32_t* table_out, int32_t* ctx_out,
                                         float* weight_out, int32_t* evicted,
                                         int32_t* n_evicted, void* stream) {
  const char* who = "kv_evict";
  if (B < 0 || max_blocks < 1 || num_blocks < 1 || sink_blocks < 0 || recent_blocks < 1)
    return local_fail(LOCAL_ERR_SHAPE,
                      "%s: B=%d max_blocks=%d num_blocks=%lld sink_blocks=%d recent_blocks=%d "
                      "(the last block is always kept: recent_blocks >= 1)", who, B, max_blocks,
                      (long long)num_blocks, sink_blocks, recent_blocks);
  if (block_size != kBlockSize)
    return local_fail(LOCAL_ERR_UNSUPPORTED, "%s: block_size=%d (need 16)", who, block_size);
  if (B == 0) return LOCAL_OK;
  if (!block_table || !ctx_lens || !block_weight || !keep_blocks || !block_version ||
      !req_version || !table_out || !ctx_out || !weight_out || !evicted || !n_evicted)
    return local_fail(LOCAL_ERR_NULL, "%s: NULL pointer argument", who);
  // The first three outputs may be the inputs that they follow; a workgroup of one row
  // would read what another has written anywhere else.
  struct Array {
    const void* p;
    size_t bytes;
  };
  const size_t rows = static_cast<size_t>(B) * max_blocks * sizeof(int32_t);
  const size_t each = static_cast<size_t>(B) * sizeof(int32_t);
  const size_t tags = static_cast<size_t>(num_blocks) * sizeof(int32_t);
  const Array in[] = {{block_table, rows}, {ctx_lens, each}, {block_weight, rows},
                      {keep_blocks, each}, {req_version, each}, {block_version, tags}};
  const Array o[] = {{table_out, rows}, {ctx_out, each}, {weight_out, rows},
                     {evicted, rows}, {n_evicted, each}};
  for (int i = 0; i < 5; ++i) {
    bool bad = false;
    for (int k = 0; k < 6; ++k)
      bad |= !(i < 3 && k == i && o[i].p == in[k].p) &&
             overlap(o[i].p, o[i].bytes, in[k].p, in[k].bytes);
    for (int k = 0; k < i; ++k) bad |= overlap(o[i].p, o[i].bytes, o[k].p, o[k].bytes);
    if (bad)
      return local_fail(LOCAL_ERR_SHAPE, "%s: an output overlaps another array (only table_out, "
                        "ctx_out and weight_out may be their inputs)", who);
  }
  const EvictArgs a = {block_table, ctx_lens,   block_weight, keep_blocks, block_version,
                       req_version, table_out,  ctx_out,      weight_out,  evicted,
                       n_evicted,   num_blocks, max_blocks,   sink_blocks, recent_blocks};
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (max_blocks > 256)
    kv_evict_kernel<1024><<<B, 1024, 0, s>>>(a);
  else
    kv_evict_kernel<256><<<B, 256, 0, s>>>(a);
  return local_check_launch(who);
}
