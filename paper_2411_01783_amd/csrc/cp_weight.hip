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
constexpr int TILE = 64;               // rows of a tile

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
  int32_t wg_keys;       // keys of a workgroup
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
    if (b0 + lane < p.batch) c = (seq_of(p, b0 + lane).used + p.wg_keys - 1) / p.wg_keys;
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

// Row r of a (sequence, KV head): node r / group, head r % group of the group; kept per lane and moved
// on by a constant number of rows.
struct RowAt {
  int32_t node, head;
  __device__ __forceinline__ void set(int64_t r, int group) {
    node = (int32_t)(r / group);
    head = (int32_t)(r - (int64_t)node * group);
  }
  __device__ __forceinline__ void advance(int by_node, int by_head, int group) {
    node += by_node;
    head += by_head;
    if (head >= group) {
      head -= group;
      ++node;
    }
  }
};

// KB: fragments of 32 keys that a wavefront holds. A tile of 64 rows travels through registers into
// one of two LDS buffers while the tile before it is used (16-byte chunk c of row r lies at
// c ^ (r % chunks): 16 lanes that read the same chunk of neighbouring rows touch all banks).
template <typename TI, int D, int KB>
__global__ __launch_bounds__(NW * 64, KB == 1 && sizeof(TI) == 2 ? 4 : 2) void kv_weight_kernel(const WeightParams p) {
  constexpr int ROW = D * (int)sizeof(TI), CH = ROW / 16, NKS = CH / 2;
  constexpr int ST = TILE * CH / (NW * 64);        // chunks of a tile that a lane brings
  constexpr int RPI = NW * 64 / CH;                // rows that the workgroup brings at a time
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rl = lane & 31, hf = lane >> 5;
  __shared__ __align__(16) char tile[2][TILE * ROW];
  __shared__ __align__(16) float lse_of[2][NW][TILE];
  __shared__ __align__(16) int32_t pos_of[2][NW][TILE];
  __shared__ int32_t wg_k_min[NW], wg_first[NW], wg_last[NW];
  int begin = 0;
  const int b = find_block(p, blockIdx.x, &begin);
  if (b < 0) return;
  const Seq sq = seq_of(p, b);
  const int range = blockIdx.y % p.n_ranges, kvh = blockIdx.y / p.n_ranges;
  const int key0 = ((int)blockIdx.x - begin) * p.wg_keys + wave * KB * KEYS;
  const int64_t tok_q = (int64_t)p.n_q_heads * D, tok_kv = (int64_t)p.n_kv_heads * D;

  // lane (rl, hf): 16-byte chunk 2 ks + hf of key rl of the fragment (keys behind the last repeat it)
  uint4 kf[KB][NKS];
  int32_t kp[KB];
  int32_t k_max = INT32_MIN, k_min = INT32_MAX;
#pragma unroll
  for (int f = 0; f < KB; ++f) {
    const int64_t key = sq.k0 + min(key0 + f * KEYS + rl, sq.used - 1);
    kp[f] = p.kv_pos[key];
    const uint4* src = (const uint4*)((const TI*)p.k + key * tok_kv + kvh * D) + hf;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) kf[f][ks] = src[2 * ks];
  }
#pragma unroll
  for (int f = 0; f < KB; ++f) {
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
  const int64_t tiles = (n_rows + TILE - 1) / TILE;
  int64_t t0 = tiles * range / p.n_ranges, t1 = tiles * (range + 1) / p.n_ranges;
  if (t1 - t0 > 2) {
    // the tiles between the first and the last row that sees any key of the workgroup
    if (lane == 0) wg_k_min[wave] = k_min;
    __syncthreads();
    int32_t lo = wg_k_min[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) lo = min(lo, wg_k_min[w]);
    const int n0 = (int)(t0 * TILE / p.group), n1 = (int)min<int64_t>(sq.n, (t1 * TILE - 1) / p.group + 1);
    int first = INT32_MAX, last = -1;
    for (int i = n0 + tid; i < n1; i += NW * 64)
      if (p.q_pos[sq.q0 + i] >= lo) {
        first = min(first, i);
        last = i;
      }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      first = min(first, __shfl_xor(first, o, 64));
      last = max(last, __shfl_xor(last, o, 64));
    }
    if (lane == 0) {
      wg_first[wave] = first;
      wg_last[wave] = last;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      first = min(first, wg_first[w]);
      last = max(last, wg_last[w]);
    }
    if (last < 0) {
      t1 = t0;
    } else {
      t0 = max(t0, (int64_t)first * p.group / TILE);
      t1 = min(t1, ((int64_t)(last + 1) * p.group - 1) / TILE + 1);
    }
  }

  // ---- a tile on its way: ST chunks of Q a lane, and of every row its LSE and position ----
  RowAt at[ST], mine;
#pragma unroll
  for (int i = 0; i < ST; ++i) at[i].set(t0 * TILE + i * RPI + tid / CH, p.group);
  mine.set(t0 * TILE + lane, p.group);
  const int by_node = TILE / p.group, by_head = TILE % p.group;
  uint4 st[ST];
  float st_lse;
  int32_t st_pos;
  auto fetch = [&]() {
#pragma unroll
    for (int i = 0; i < ST; ++i) {
      st[i] = make_uint4(0, 0, 0, 0);
      if (at[i].node < sq.n)
        st[i] = ((const uint4*)((const TI*)p.q + (sq.q0 + at[i].node) * tok_q +
                                (kvh * p.group + at[i].head) * D))[tid % CH];
      at[i].advance(by_node, by_head, p.group);
    }
    st_lse = INFINITY;
    st_pos = INT32_MIN;
    if (mine.node < sq.n) {
      st_lse = p.lse[(sq.q0 + mine.node) * p.n_q_heads + kvh * p.group + mine.head];
      st_pos = p.q_pos[sq.q0 + mine.node];
    }
    mine.advance(by_node, by_head, p.group);
  };
  // a row that sees no key anywhere (LSE = -inf), and one behind the last, weighs nothing
  auto put = [&](int to) {
#pragma unroll
    for (int i = 0; i < ST; ++i) {
      const int r = i * RPI + tid / CH;
      *(uint4*)(tile[to] + r * ROW + (((tid % CH) ^ (r & (CH - 1))) << 4)) = st[i];
    }
    lse_of[to][wave][lane] = st_lse == -INFINITY ? INFINITY : st_lse * kLog2e;
    pos_of[to][wave][lane] = st_pos;
  };

  if (t0 < t1) {
    fetch();
    put((int)(t0 & 1));
  }
  for (int64_t t = t0; t < t1; ++t) {
    const int cur = (int)(t & 1);
    // which of the tile's row blocks see any of the wavefront's keys, and which not all
    const bool real = st_pos != INT32_MIN;
    const uint64_t some = __builtin_amdgcn_ballot_w64(real && st_pos >= k_min);
    const uint64_t hide = __builtin_amdgcn_ballot_w64(real && st_pos < k_max);
    __syncthreads();
    if (t + 1 < t1) fetch();
#pragma unroll
    for (int rb = 0; rb < TILE / 32; ++rb) {
      if ((uint32_t)(some >> (32 * rb)) == 0) continue;
      const bool masked = (uint32_t)(hide >> (32 * rb)) != 0;
      floatx16_t s[KB];
#pragma unroll
      for (int f = 0; f < KB; ++f)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[f][i] = 0.f;
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) {
        const int r = rb * 32 + rl;
        const uint4 qf = *(const uint4*)(tile[cur] + r * ROW + (((2 * ks + hf) ^ (r & (CH - 1))) << 4));
#pragma unroll
        for (int f = 0; f < KB; ++f) s[f] = product(qf, kf[f][ks], s[f], TI());
      }
      // score i of lane (rl, hf): key rl, row (i / 4) * 8 + hf * 4 + i % 4
      floatx4_t lr[4];
#pragma unroll
      for (int a = 0; a < 4; ++a)
        lr[a] = *(const floatx4_t*)&lse_of[cur][wave][rb * 32 + a * 8 + hf * 4];
#pragma unroll
      for (int f = 0; f < KB; ++f) {
        float e[16];
#pragma unroll
        for (int i = 0; i < 16; ++i)
          e[i] = __builtin_amdgcn_exp2f(fmaf(s[f][i], p.scale_log2, -lr[i >> 2][i & 3]));
        if (masked) {
#pragma unroll
          for (int a = 0; a < 4; ++a) {
            const int4 q = *(const int4*)&pos_of[cur][wave][rb * 32 + a * 8 + hf * 4];
            e[4 * a] = q.x >= kp[f] ? e[4 * a] : 0.f;
            e[4 * a + 1] = q.y >= kp[f] ? e[4 * a + 1] : 0.f;
            e[4 * a + 2] = q.z >= kp[f] ? e[4 * a + 2] : 0.f;
            e[4 * a + 3] = q.w >= kp[f] ? e[4 * a + 3] : 0.f;
          }
        }
        float x = (e[0] + e[1]) + (e[2] + e[3]);
#pragma unroll
        for (int a = 1; a < 4; ++a)
          x += (e[4 * a] + e[4 * a + 1]) + (e[4 * a + 2] + e[4 * a + 3]);
        sum[f] += x;
      }
    }
    if (t + 1 < t1) put(cur ^ 1);
  }
#pragma unroll
  for (int f = 0; f < KB; ++f) {
    const float x = sum[f] + __shfl_xor(sum[f], 32, 64);
    const int key = key0 + f * KEYS + rl;
    if (hf == 0 && key < sq.used) {
      const int64_t to = sq.k0 + key;
      if (p.part != nullptr)
        p.part[(int64_t)blockIdx.y * p.total_kv + to] = x;
      else
        p.weight[to] = p.decay != 0.f ? fmaf(p.weight[to], p.decay, x) : x;
    }
  }
}

// weight <- decay * weight + the parts, in their order.
__global__ __launch_bounds__(256) void kv_weight_sum_kernel(const WeightParams p) {
  int begin = 0;
  const int b = find_block(p, blockIdx.x, &begin);
  if (b < 0) return;
  const Seq sq = seq_of(p, b);
  const int key = ((int)blockIdx.x - begin) * p.wg_keys + threadIdx.x;
  if ((int)threadIdx.x >= p.wg_keys || key >= sq.used) return;
  const int64_t at = sq.k0 + key;
  const int n = p.n_ranges * p.n_kv_heads;
  float t = 0.f;
  for (int i = 0; i < n; ++i) t += p.part[(int64_t)i * p.total_kv + at];
  p.weight[at] = p.decay != 0.f ? fmaf(p.weight[at], p.decay, t) : t;
}

struct WeightPlan {
  int kb;           // fragments of a wavefront
  int64_t blocks;   // key blocks there can be
  int n_ranges;
  size_t bytes;
};
WeightPlan weight_plan(const cp_shape& s) {
  WeightPlan pl = {};
  const int64_t rows = (s.total_q * (s.n_q_heads / s.n_kv_heads) + s.batch - 1) / s.batch;
  const int64_t tiles = (rows + TILE - 1) / TILE;   // of a sequence, on average
  pl.kb = tiles <= 1 || s.dtype == CP_FP32 ? 1 : 2;
  const int wg_keys = NW * pl.kb * KEYS;
  pl.blocks = s.total_kv / wg_keys + s.batch;
  // ranges of the rows until there are eight workgroups per CU, of four tiles at least
  int64_t n = 1;
  while (n < 64 && pl.blocks * s.n_kv_heads * n < 2048 && tiles >= n * 2 * 4) n *= 2;
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
  if (s.total_kv > INT32_MAX - 256) return CP_ERR_SHAPE;   // key indices in 31 bits
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
  p.wg_keys = NW * pl.kb * KEYS;
  p.scale_log2 = (s.softmax_scale > 0.f ? s.softmax_scale : 1.0f / sqrtf((float)s.head_dim)) * kLog2e;
  p.decay = decay;
  hipStream_t st = (hipStream_t)stream;
  const dim3 grid((unsigned)pl.blocks, (unsigned)parts);
#define CP_WEIGHT(TI, D, KB) \
  hipLaunchKernelGGL((kv_weight_kernel<TI, D, KB>), grid, dim3(NW * 64), 0, st, p)
  if (s.dtype == CP_FP32) {
    if (s.head_dim == 64) CP_WEIGHT(float, 64, 1);
    else CP_WEIGHT(float, 128, 1);
  } else if (s.head_dim == 64) {
    if (pl.kb == 1) CP_WEIGHT(bf16_t, 64, 1);
    else CP_WEIGHT(bf16_t, 64, 2);
  } else {
    if (pl.kb == 1) CP_WEIGHT(bf16_t, 128, 1);
    else CP_WEIGHT(bf16_t, 128, 2);
  }
#undef CP_WEIGHT
  if (check_launch() != CP_OK) return CP_ERR_LAUNCH;
  if (p.part == nullptr) return CP_OK;
  hipLaunchKernelGGL(kv_weight_sum_kernel, dim3((unsigned)pl.blocks), dim3(256), 0, st, p);
  return check_launch();
}
