// Eviction from the persistent KV cache by accumulated attention weight.
//
// Of the n tokens that sequence b holds, keep = min(n, room of the destination, max(budget_b, number
// of protected ones)) stay: the protected first, then by weight, ties to the lowest slot. Kept slots
// in front of `keep` stay where they are, and the i-th kept slot behind it moves to the i-th hole in
// front of it, so in place only as many rows move as there are holes (sources lie behind `keep`,
// destinations in front of it: no row is read after it was written). The order of the slots means
// nothing to attention, which goes by their positions.
//
// Two launches. The first, a workgroup per sequence, finds the weight of the last slot that stays by a
// radix selection over order-preserving 32-bit keys (three digits of 11, 11 and 10 bits, counted in
// LDS), then ranks holes and movers by prefix sums, and does the bookkeeping arrays. The second
// copies the K and V rows.
#include "cp_common.h"

namespace cp {
namespace {

struct EvictParams {
  // source
  const uint4* k;
  const uint4* v;
  int32_t* kv_pos;
  float* weight;
  const int32_t* cu;
  int32_t* used;
  // destination (the same in place)
  uint4* k_to;
  uint4* v_to;
  int32_t* pos_to;
  float* weight_to;
  const int32_t* cu_to;
  int32_t* used_to;
  const int32_t* budget;
  const int32_t* protect_from;   // or NULL
  int64_t slots, slots_to;
  int32_t batch, sinks, chunks;
  bool in_place;
  // workspace: what is copied where, [slots] at the sequence's first slot; and how many
  int32_t* from;    // destination slot -> source slot, both within the sequence (in place: of move t)
  int32_t* to;      // in place: destination slot of move t
  int32_t* count;   // [batch]
};

__device__ __forceinline__ int64_t clamp64(int64_t x, int64_t lo, int64_t hi) {
  return x < lo ? lo : x > hi ? hi : x;
}
struct Range {
  int64_t first, room;
};
__device__ __forceinline__ Range range_of(const int32_t* cu, int b, int64_t slots) {
  Range r;
  r.first = clamp64(cu[b], 0, slots);
  r.room = clamp64(cu[b + 1], r.first, slots) - r.first;
  return r;
}

constexpr int SEL_THREADS = 1024, SEL_WAVES = SEL_THREADS / 64;
constexpr int BINS = 2048;

// Order-preserving key of a weight; protected slots are above all, NaN below all.
__device__ __forceinline__ uint32_t key_of(float w, bool safe) {
  if (safe) return 0xffffffffu;
  if (w != w) return 0;
  const uint32_t x = __builtin_bit_cast(uint32_t, w + 0.f);   // (-0 counts as 0)
  return (x & 0x80000000u) ? ~x : x | 0x80000000u;
}

// Prefix sum over the workgroup of x (exclusive), and the total.
__device__ __forceinline__ int block_scan(int x, int* wave_sums, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int end = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(end, o, 64);
    if (lane >= o) end += y;
  }
  __syncthreads();
  if (lane == 63) wave_sums[wave] = end;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < SEL_WAVES; ++w) {
    const int y = wave_sums[w];
    if (w < wave) before += y;
    all += y;
  }
  *total = all;
  return before + end - x;
}

__global__ __launch_bounds__(SEL_THREADS) void evict_select_kernel(const EvictParams p) {
  __shared__ int hist[BINS];
  __shared__ int wave_sums[SEL_WAVES];
  __shared__ int found_bin, found_above;
  const int b = blockIdx.x, tid = threadIdx.x;
  const Range src = range_of(p.cu, b, p.slots), dst = range_of(p.cu_to, b, p.slots_to);
  const int n = (int)clamp64(p.used[b], 0, src.room);
  const int32_t from_pos = p.protect_from != nullptr ? p.protect_from[b] : CP_POS_PAD_KV;
  const int32_t* const pos = p.kv_pos + src.first;
  const float* const weight = p.weight + src.first;
  auto key = [&](int i) -> uint32_t {
    const int32_t at = pos[i];
    // (a padded token can be seen by no query: nothing protects it)
    return key_of(weight[i], at != CP_POS_PAD_KV && (at < p.sinks || at >= from_pos));
  };
  int protected_n = 0;
  for (int i = tid; i < n; i += SEL_THREADS) protected_n += key(i) == 0xffffffffu;
  int all;
  block_scan(protected_n, wave_sums, &all);
  int64_t want = p.budget[b];
  if (want < all) want = all;
  const int keep = (int)clamp64(want, 0, n < dst.room ? n : dst.room);

  // the key of the last slot that stays, and how many slots with that key do
  uint32_t bar = 0;
  int ties = 0;
  if (keep > 0 && keep < n) {
    uint32_t prefix = 0, prefix_mask = 0;
    int left = keep;
    for (int d = 0; d < 3; ++d) {
      const int shift = d == 0 ? 21 : d == 1 ? 10 : 0;
      const uint32_t digit = d == 2 ? 1023u : 2047u;
      __syncthreads();
      for (int i = tid; i < BINS; i += SEL_THREADS) hist[i] = 0;
      __syncthreads();
      for (int i = tid; i < n; i += SEL_THREADS) {
        const uint32_t x = key(i);
        if ((x & prefix_mask) == prefix) atomicAdd(&hist[(x >> shift) & digit], 1);
      }
      __syncthreads();
      // bins from the top: thread t has bins BINS-1-2t and BINS-2-2t
      const int hi = BINS - 1 - 2 * tid;
      const int c1 = hist[hi], c0 = hist[hi - 1];
      const int above = block_scan(c0 + c1, wave_sums, &all);
      if (above < left && left <= above + c1) {
        found_bin = hi;
        found_above = above;
      } else if (above + c1 < left && left <= above + c1 + c0) {
        found_bin = hi - 1;
        found_above = above + c1;
      }
      __syncthreads();
      prefix |= (uint32_t)found_bin << shift;
      prefix_mask |= digit << shift;
      left -= found_above;
    }
    bar = prefix;
    ties = left;
  }

  // ranks of the holes in front of `keep` and of the movers behind it
  int32_t* const from = p.from + src.first;
  int32_t* const to = p.to + src.first;
  int tie_base = 0, hole_base = 0, mover_base = 0;
  for (int i0 = 0; i0 < n; i0 += SEL_THREADS) {
    const int i = i0 + tid;
    bool stays = false, tie = false;
    if (i < n) {
      if (keep == n) stays = true;
      else if (keep > 0) {
        const uint32_t x = key(i);
        stays = x > bar;
        tie = x == bar;
      }
    }
    const int rank = block_scan(tie ? 1 : 0, wave_sums, &all);
    if (tie && tie_base + rank < ties) stays = true;
    tie_base += all;
    const bool hole = i < keep && !stays, mover = i >= keep && i < n && stays;
    // (holes lie in front of movers: one scan serves both)
    const int r = block_scan((hole ? 1 : 0) | (mover ? 1 << 16 : 0), wave_sums, &all);
    if (hole) to[hole_base + (r & 0xffff)] = i;
    if (mover) from[mover_base + (r >> 16)] = i;
    hole_base += all & 0xffff;
    mover_base += all >> 16;
  }
  __threadfence_block();
  __syncthreads();
  const int moves = hole_base;
  if (p.in_place) {
    for (int t = tid; t < moves; t += SEL_THREADS) {
      const int d = to[t], s = from[t];
      p.kv_pos[src.first + d] = pos[s];
      p.weight[src.first + d] = weight[s];
    }
    __syncthreads();
    for (int i = keep + tid; i < n; i += SEL_THREADS) {
      p.kv_pos[src.first + i] = CP_POS_PAD_KV;
      p.weight[src.first + i] = 0.f;
    }
  } else {
    for (int i = tid; i < keep; i += SEL_THREADS) {
      p.pos_to[dst.first + i] = pos[i];
      p.weight_to[dst.first + i] = weight[i];
    }
    for (int64_t i = keep + tid; i < dst.room; i += SEL_THREADS) {
      p.pos_to[dst.first + i] = CP_POS_PAD_KV;
      p.weight_to[dst.first + i] = 0.f;
    }
    __syncthreads();
    for (int t = tid; t < moves; t += SEL_THREADS) {
      const int d = to[t], s = from[t];
      p.pos_to[dst.first + d] = pos[s];
      p.weight_to[dst.first + d] = weight[s];
    }
  }
  if (tid == 0) {
    p.used_to[b] = keep;
    p.count[2 * b] = keep;
    p.count[2 * b + 1] = moves;
  }
}

// Rows of K and V: in place the moves, otherwise first what stays in its slot and then the moves.
__global__ __launch_bounds__(256) void evict_move_kernel(const EvictParams p) {
  const int b = blockIdx.y;
  const Range src = range_of(p.cu, b, p.slots), dst = range_of(p.cu_to, b, p.slots_to);
  const int keep = p.count[2 * b], moves = p.count[2 * b + 1];
  const int32_t* const from = p.from + src.first;
  const int32_t* const to = p.to + src.first;
  const int64_t stride = (int64_t)gridDim.x * 256;
  const int64_t first = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (p.in_place) {
    for (int64_t e = first; e < (int64_t)moves * p.chunks; e += stride) {
      const int64_t t = e / p.chunks, c = e - t * p.chunks;
      const int64_t s = (src.first + from[t]) * p.chunks + c, d = (dst.first + to[t]) * p.chunks + c;
      p.k_to[d] = p.k[s];
      p.v_to[d] = p.v[s];
    }
    return;
  }
  for (int64_t e = first; e < (int64_t)keep * p.chunks; e += stride) {
    const int64_t i = e / p.chunks, c = e - i * p.chunks;
    // is slot i a hole? `to` is ascending
    int lo = 0, hi = moves;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (to[mid] < i) lo = mid + 1;
      else hi = mid;
    }
    const int64_t s0 = lo < moves && to[lo] == i ? from[lo] : i;
    const int64_t s = (src.first + s0) * p.chunks + c, d = (dst.first + i) * p.chunks + c;
    p.k_to[d] = p.k[s];
    p.v_to[d] = p.v[s];
  }
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
inline size_t round256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

size_t evict_workspace_bytes(const cp_shape& s) {
  return 2 * round256((size_t)s.total_kv * 4) + round256((size_t)s.batch * 8);
}

}  // namespace cp

extern "C" int cp_kv_evict(const cp_shape* shape, void* k_cache, void* v_cache, int32_t* kv_pos_cache,
                           float* weight, const int32_t* cu_seqlens_kv, int32_t* seq_used,
                           const int32_t* budget, const int32_t* protect_from, int32_t sinks,
                           void* k_to, void* v_to, int32_t* kv_pos_to, float* weight_to,
                           const int32_t* cu_seqlens_to, int32_t* seq_used_to, int64_t slots_to,
                           void* workspace, size_t workspace_bytes, void* stream) {
  using namespace cp;
  const int rc = check_cache_shape(shape);
  if (rc != CP_OK) return rc;
  const cp_shape& s = *shape;
  if (sinks < 0) return CP_ERR_SHAPE;
  if (cu_seqlens_kv == nullptr || seq_used == nullptr || budget == nullptr) return CP_ERR_NULL;
  const bool in_place = k_to == nullptr;
  if (in_place) {
    if (v_to != nullptr || kv_pos_to != nullptr || weight_to != nullptr || cu_seqlens_to != nullptr ||
        seq_used_to != nullptr)
      return CP_ERR_NULL;   // all of the destination or nothing
    k_to = k_cache; v_to = v_cache; kv_pos_to = kv_pos_cache; weight_to = weight;
    cu_seqlens_to = cu_seqlens_kv; seq_used_to = seq_used; slots_to = s.total_kv;
  } else {
    if (v_to == nullptr || kv_pos_to == nullptr || weight_to == nullptr || cu_seqlens_to == nullptr ||
        seq_used_to == nullptr)
      return CP_ERR_NULL;
    if (slots_to < 0 || slots_to > INT32_MAX) return CP_ERR_SHAPE;
    if (k_to == k_cache || v_to == v_cache || kv_pos_to == kv_pos_cache || weight_to == weight ||
        seq_used_to == seq_used)
      return CP_ERR_SHAPE;  // another cache, or in place
  }
  if (s.total_kv > 0 &&
      (k_cache == nullptr || v_cache == nullptr || kv_pos_cache == nullptr || weight == nullptr))
    return CP_ERR_NULL;
  if (!aligned16(k_cache) || !aligned16(v_cache) || !aligned16(k_to) || !aligned16(v_to))
    return CP_ERR_ALIGN;
  if (s.batch > 65535) return CP_ERR_SHAPE;   // the grid's second dimension
  if (workspace == nullptr || ((uintptr_t)workspace & 255u) != 0 ||
      workspace_bytes < evict_workspace_bytes(s))
    return CP_ERR_WORKSPACE;
  EvictParams p = {};
  p.k = (const uint4*)k_cache; p.v = (const uint4*)v_cache; p.kv_pos = kv_pos_cache; p.weight = weight;
  p.cu = cu_seqlens_kv; p.used = seq_used;
  p.k_to = (uint4*)k_to; p.v_to = (uint4*)v_to; p.pos_to = kv_pos_to; p.weight_to = weight_to;
  p.cu_to = cu_seqlens_to; p.used_to = seq_used_to;
  p.budget = budget; p.protect_from = protect_from;
  p.slots = s.total_kv; p.slots_to = slots_to;
  p.batch = s.batch; p.sinks = sinks;
  p.chunks = (int32_t)((int64_t)s.n_kv_heads * s.head_dim * (s.dtype == CP_BF16 ? 2 : 4) / 16);
  p.in_place = in_place;
  char* const ws = (char*)workspace;
  p.from = (int32_t*)ws;
  p.to = (int32_t*)(ws + round256((size_t)s.total_kv * 4));
  p.count = (int32_t*)(ws + 2 * round256((size_t)s.total_kv * 4));
  hipStream_t st = (hipStream_t)stream;
  hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)s.batch), dim3(SEL_THREADS), 0, st, p);
  if (check_launch() != CP_OK) return CP_ERR_LAUNCH;
  // enough workgroups for every CU, no more than there are chunks
  const int64_t rows = in_place ? s.total_kv : slots_to < s.total_kv ? slots_to : s.total_kv;
  int64_t parts = (2048 + s.batch - 1) / s.batch;
  const int64_t most = (rows * p.chunks / s.batch + 255) / 256;
  if (parts > most) parts = most;
  if (parts < 1) parts = 1;
  hipLaunchKernelGGL(evict_move_kernel, dim3((unsigned)parts, (unsigned)s.batch), dim3(256), 0, st, p);
  return check_launch();
}
