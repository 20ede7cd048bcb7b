// Accumulated attention weight of the cached keys: for every slot j of a sequence's cache
//   w_j <- decay * w_j + sum over the sequence's queries i that see j and all heads h of
//          exp(scale q_ih . k_j - LSE_ih),
// with the LSE of the finished attention (over all ranks' keys, after the merge), so that the terms
// are the softmax probabilities themselves. K is read, V is not.
//
// S = Q K^T on 32x32 MFMAs with the rows (query, head of the KV head's group) on the M side and the
// keys on the N side: a key's terms of 32 rows then lie in the registers of one lane pair, and
// summing over rows costs one addition a score. A wavefront keeps 64 keys in registers and walks the
// row blocks. Sums are fp32 in a fixed order (no atomics): a workgroup owns 256 keys of a KV head and
// a range of the row blocks; with several ranges or KV heads the parts go to the workspace and a
// second launch adds them up in order.
#include <math.h>

#include "cp_common.h"

namespace cp {
namespace {

constexpr int NW = 4;                  // wavefronts of a workgroup
constexpr int KEYS = 32;               // keys of a fragment
constexpr int KB = 2;                  // fragments of a wavefront
constexpr int WG_KEYS = NW * KB * KEYS;
constexpr int ROWS = 32;               // rows of a row block

struct WeightParams {
  const void* q;
  const int32_t* q_pos;
  const int32_t* cu_q;
  const void* k;
  const int32_t* kv_pos;
  const int32_t* cu_kv;
  const int32_t* used;   // or NULL
  const float* lse;
  float* weight;
  float* part;           // [n_ranges * n_kv_heads][total_kv], or NULL: one part, straight to weight
  int64_t total_q, total_kv;
  int32_t batch, n_q_heads, n_kv_heads, group, n_ranges;
  float scale_log2, decay;
};

__device__ __forceinline__ int64_t clamp64(int64_t x, int64_t lo, int64_t hi) {
  return x < lo ? lo : x > hi ? hi : x;
}
struct Seq {
  int64_t q0, k0;
  int32_t n, used;
};
// (boundaries that contradict each other or the totals are cut to what is there)
__device__ __forceinline__ Seq seq_of(const WeightParams& p, int b) {
  Seq s;
  s.q0 = clamp64(p.cu_q[b], 0, p.total_q);
  s.n = (int32_t)(clamp64(p.cu_q[b + 1], s.q0, p.total_q) - s.q0);
  s.k0 = clamp64(p.cu_kv[b], 0, p.total_kv);
  const int64_t room = clamp64(p.cu_kv[b + 1], s.k0, p.total_kv) - s.k0;
  s.used = (int32_t)(p.used != nullptr ? clamp64(p.used[b], 0, room) : room);
  return s;
}

// The sequence that block x of the line of all sequences' key blocks belongs to, and its first block.
__device__ __forceinline__ int find_block(const WeightParams& p, int x, int* begin) {
  const int lane = threadIdx.x & 63;
  int base = 0;
  for (int b0 = 0; b0 < p.batch; b0 += 64) {
    int c = 0;
    if (b0 + lane < p.batch) c = (seq_of(p, b0 + lane).used + WG_KEYS - 1) / WG_KEYS;
    int end = c;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(end, o, 64);
      if (lane >= o) end += y;
    }
    const uint64_t behind = __builtin_amdgcn_ballot_w64(base + end > x);
    if (behind != 0) {
      const int l = __builtin_ctzll(behind);
      *begin = base + __shfl(end - c, l, 64);
      return b0 + l;
    }
    base += __shfl(end, 63, 64);
  }
  return -1;
}

__device__ __forceinline__ floatx16_t product(const uint4& a, const uint4& b, floatx16_t c, bf16_t) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a),
                                                 __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
__device__ __forceinline__ floatx16_t product(const uint4& a, const uint4& b, floatx16_t c, float) {
  const floatx4_t x = __builtin_bit_cast(floatx4_t, a), y = __builtin_bit_cast(floatx4_t, b);
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], y[i], c, 0, 0, 0);
  return c;
}

template <typename TI, int D>
__global__ __launch_bounds__(NW * 64) void kv_weight_kernel(const WeightParams p) {
  constexpr int NKS = D * (int)sizeof(TI) / 32;   // pairs of 16-byte chunks of a row
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rl = lane & 31, hf = lane >> 5;
  __shared__ __align__(16) float lse_of[NW][ROWS];
  __shared__ __align__(16) int32_t pos_of[NW][ROWS];
  int begin = 0;
  const int b = find_block(p, blockIdx.x, &begin);
  if (b < 0) return;
  const Seq sq = seq_of(p, b);
  const int range = blockIdx.y % p.n_ranges, kvh = blockIdx.y / p.n_ranges;
  const int key0 = ((int)blockIdx.x - begin) * WG_KEYS + wave * KB * KEYS;
  if (key0 >= sq.used) return;   // (no barrier below)
  const int64_t tok_q = (int64_t)p.n_q_heads * D, tok_kv = (int64_t)p.n_kv_heads * D;

  // lane (rl, hf): 16-byte chunk 2 ks + hf of key rl of the fragment
  uint4 kf[KB][NKS];
  int32_t kp[KB];
  int32_t k_max = INT32_MIN, k_min = INT32_MAX;
#pragma unroll
  for (int f = 0; f < KB; ++f) {
    const int64_t key = sq.k0 + min(key0 + f * KEYS + rl, sq.used - 1);
    const uint4* src = (const uint4*)((const TI*)p.k + key * tok_kv + kvh * D) + hf;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) kf[f][ks] = src[2 * ks];
    kp[f] = p.kv_pos[key];
    k_max = max(k_max, kp[f]);
    k_min = min(k_min, kp[f]);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    k_max = max(k_max, __shfl_xor(k_max, o, 64));
    k_min = min(k_min, __shfl_xor(k_min, o, 64));
  }

  float sum[KB];
#pragma unroll
  for (int f = 0; f < KB; ++f) sum[f] = 0.f;
  const int64_t n_rows = (int64_t)sq.n * p.group;
  const int64_t blocks = (n_rows + ROWS - 1) / ROWS;
  const int64_t r0 = blocks * range / p.n_ranges, r1 = blocks * (range + 1) / p.n_ranges;
  for (int64_t rb = r0; rb < r1; ++rb) {
    const int64_t row = rb * ROWS + rl;
    const bool ok = row < n_rows;
    const int64_t nd = ok ? row / p.group : 0;
    const int head = kvh * p.group + (ok ? (int)(row - nd * p.group) : 0);
    const int64_t tok = sq.q0 + nd;
    const int32_t qp = ok ? p.q_pos[tok] : INT32_MIN;
    const uint64_t some = __builtin_amdgcn_ballot_w64(ok && qp >= k_min);
    if (some == 0) continue;   // none of the rows sees any of the keys
    const bool masked = __builtin_amdgcn_ballot_w64(ok && qp < k_max) != 0;
    uint4 qf[NKS];
    const uint4* src = (const uint4*)((const TI*)p.q + tok * tok_q + head * D) + hf;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {
      qf[ks] = make_uint4(0, 0, 0, 0);
      if (ok) qf[ks] = src[2 * ks];
    }
    // a row that sees no key anywhere (LSE = -inf), and one behind the last, weighs nothing
    float l2 = ok ? p.lse[tok * p.n_q_heads + head] * kLog2e : INFINITY;
    if (l2 == -INFINITY) l2 = INFINITY;
    __builtin_amdgcn_wave_barrier();
    if (hf == 0) {
      lse_of[wave][rl] = l2;
      pos_of[wave][rl] = qp;
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    // score i of lane (rl, hf): key rl, row (i / 4) * 8 + hf * 4 + i % 4
    floatx4_t lr[4];
#pragma unroll
    for (int a = 0; a < 4; ++a) lr[a] = *(const floatx4_t*)&lse_of[wave][a * 8 + hf * 4];
#pragma unroll
    for (int f = 0; f < KB; ++f) {
      floatx16_t s;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) s = product(qf[ks], kf[f][ks], s, TI());
      float t = 0.f;
      if (masked) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float e = __builtin_amdgcn_exp2f(fmaf(s[i], p.scale_log2, -lr[i >> 2][i & 3]));
          t += pos_of[wave][(i >> 2) * 8 + hf * 4 + (i & 3)] >= kp[f] ? e : 0.f;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          t += __builtin_amdgcn_exp2f(fmaf(s[i], p.scale_log2, -lr[i >> 2][i & 3]));
      }
      sum[f] += t;
    }
    __builtin_amdgcn_wave_barrier();
  }
#pragma unroll
  for (int f = 0; f < KB; ++f) {
    const float t = sum[f] + __shfl_xor(sum[f], 32, 64);
    const int key = key0 + f * KEYS + rl;
    if (hf == 0 && key < sq.used) {
      const int64_t at = sq.k0 + key;
      if (p.part != nullptr)
        p.part[(int64_t)blockIdx.y * p.total_kv + at] = t;
      else
        p.weight[at] = p.decay != 0.f ? fmaf(p.weight[at], p.decay, t) : t;
    }
  }
}

// weight <- decay * weight + the parts, in their order.
__global__ __launch_bounds__(256) void kv_weight_sum_kernel(const WeightParams p) {
  int begin = 0;
  const int b = find_block(p, blockIdx.x, &begin);
  if (b < 0) return;
  const Seq sq = seq_of(p, b);
  const int key = ((int)blockIdx.x - begin) * WG_KEYS + threadIdx.x;
  if (key >= sq.used) return;
  const int64_t at = sq.k0 + key;
  const int n = p.n_ranges * p.n_kv_heads;
  float t = 0.f;
  for (int i = 0; i < n; ++i) t += p.part[(int64_t)i * p.total_kv + at];
  p.weight[at] = p.decay != 0.f ? fmaf(p.weight[at], p.decay, t) : t;
}
static_assert(WG_KEYS == 256, "a thread of the second launch per key");

struct WeightPlan {
  int64_t blocks;   // key blocks there can be
  int n_ranges;
  size_t bytes;
};
WeightPlan weight_plan(const cp_shape& s) {
  WeightPlan pl = {};
  pl.blocks = s.total_kv / WG_KEYS + s.batch;
  // Row blocks of a sequence, on average; ranges of them until there are four workgroups per CU
  const int64_t rows = (s.total_q * (s.n_q_heads / s.n_kv_heads) + s.batch - 1) / s.batch;
  int64_t n = 1;
  while (n < 32 && pl.blocks * s.n_kv_heads * n < 1024 && rows > n * 4 * ROWS) n *= 2;
  pl.n_ranges = (int)n;
  const int64_t parts = n * s.n_kv_heads;
  pl.bytes = parts > 1 ? (size_t)parts * s.total_kv * 4 : 0;
  return pl;
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

}  // namespace

size_t weight_workspace_bytes(const cp_shape& s) {
  return weight_plan(s).bytes;
}

}  // namespace cp

extern "C" int cp_kv_attn_weight(const cp_shape* shape, const void* q, const int32_t* q_pos,
                                 const int32_t* cu_seqlens_q, const float* lse, const void* k_cache,
                                 const int32_t* kv_pos_cache, const int32_t* cu_seqlens_kv,
                                 const int32_t* seq_used, float decay, float* weight, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  using namespace cp;
  const int rc = check_shape(shape);
  if (rc != CP_OK) return rc;
  const cp_shape& s = *shape;
  if (!(decay >= 0.f) || isinf(decay)) return CP_ERR_SHAPE;
  if (cu_seqlens_q == nullptr || cu_seqlens_kv == nullptr) return CP_ERR_NULL;
  if (s.total_q > 0 && (q == nullptr || q_pos == nullptr || lse == nullptr)) return CP_ERR_NULL;
  if (s.total_kv > 0 && (k_cache == nullptr || kv_pos_cache == nullptr || weight == nullptr))
    return CP_ERR_NULL;
  if (!aligned16(q) || !aligned16(k_cache)) return CP_ERR_ALIGN;
  if (s.total_kv == 0) return CP_OK;
  if (s.total_kv > INT32_MAX - WG_KEYS) return CP_ERR_SHAPE;
  const WeightPlan pl = weight_plan(s);
  if (pl.bytes > 0 && (workspace == nullptr || ((uintptr_t)workspace & 255u) != 0 ||
                       workspace_bytes < pl.bytes))
    return CP_ERR_WORKSPACE;
  const int64_t parts = (int64_t)pl.n_ranges * s.n_kv_heads;
  if (parts > 65535) return CP_ERR_SHAPE;   // the grid's second dimension
  WeightParams p = {};
  p.q = q; p.q_pos = q_pos; p.cu_q = cu_seqlens_q;
  p.k = k_cache; p.kv_pos = kv_pos_cache; p.cu_kv = cu_seqlens_kv; p.used = seq_used;
  p.lse = lse; p.weight = weight;
  p.part = pl.bytes > 0 ? (float*)workspace : nullptr;
  p.total_q = s.total_q; p.total_kv = s.total_kv; p.batch = s.batch;
  p.n_q_heads = s.n_q_heads; p.n_kv_heads = s.n_kv_heads; p.group = s.n_q_heads / s.n_kv_heads;
  p.n_ranges = pl.n_ranges;
  p.scale_log2 = (s.softmax_scale > 0.f ? s.softmax_scale : 1.0f / sqrtf((float)s.head_dim)) * kLog2e;
  p.decay = decay;
  hipStream_t st = (hipStream_t)stream;
  const dim3 grid((unsigned)pl.blocks, (unsigned)parts);
#define CP_WEIGHT(TI, D) hipLaunchKernelGGL((kv_weight_kernel<TI, D>), grid, dim3(NW * 64), 0, st, p)
  if (s.dtype == CP_FP32) {
    if (s.head_dim == 64) CP_WEIGHT(float, 64);
    else CP_WEIGHT(float, 128);
  } else {
    if (s.head_dim == 64) CP_WEIGHT(bf16_t, 64);
    else CP_WEIGHT(bf16_t, 128);
  }
#undef CP_WEIGHT
  if (check_launch() != CP_OK) return CP_ERR_LAUNCH;
  if (p.part == nullptr) return CP_OK;
  hipLaunchKernelGGL(kv_weight_sum_kernel, dim3((unsigned)pl.blocks), dim3(256), 0, st, p);
  return check_launch();
}
