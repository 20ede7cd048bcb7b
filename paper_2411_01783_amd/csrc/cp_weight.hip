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

#include "cp_scan.h"

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

struct Seq {
  int32_t q0, n, k0, used;   // first query, queries, first slot, tokens in the cache
  __device__ __forceinline__ Seq of_lane(int l) const {
    Seq r;
    r.q0 = __builtin_amdgcn_readlane(q0, l);
    r.n = __builtin_amdgcn_readlane(n, l);
    r.k0 = __builtin_amdgcn_readlane(k0, l);
    r.used = __builtin_amdgcn_readlane(used, l);
    return r;
  }
};
// (boundaries that contradict each other or the totals are cut to what is there)
__device__ __forceinline__ Seq seq_of(const WeightParams& p, int b) {
  const int32_t a0 = p.cu_q[b], a1 = p.cu_q[b + 1], c0 = p.cu_kv[b], c1 = p.cu_kv[b + 1];
  const int32_t u = p.used != nullptr ? p.used[b] : INT32_MAX;
  Seq s;
  s.q0 = (int32_t)clamp64(a0, 0, p.total_q);
  s.n = (int32_t)clamp64(a1, s.q0, p.total_q) - s.q0;
  s.k0 = (int32_t)clamp64(c0, 0, p.total_kv);
  s.used = (int32_t)clamp64(u, 0, clamp64(c1, s.k0, p.total_kv) - s.k0);
  return s;
}
// The sequence that block x of all sequences' key blocks belongs to, and its first block.
__device__ __forceinline__ int find_block(const WeightParams& p, int x, int* begin, Seq* sq) {
  return find_sequence_of_block(
      p.batch, x, begin, sq, [&](int b) { return seq_of(p, b); },
      [&](const Seq& s) { return (s.used + p.wg_keys - 1) / p.wg_keys; });
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
  __device__ __forceinline__ void set(uint32_t r, uint32_t group) {
    node = (int32_t)(r / group);
    head = (int32_t)(r - (uint32_t)node * group);
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

// A wavefront holds KB fragments of 32 keys: two of bf16 (one would halve the use of a row tile; us, one and two: 16
// heads on one over 32 sequences of 2048 to 8192 keys, a query each 14.1 and 12.2, 16 queries each 28.3 and 24.5;
// 32 heads on 8 over 8 sequences 63 and 28; 8192 queries over their own prompt 237 and 198; 16 queries over 8
// times 4096 keys 11.4 and 13.2), one of fp32, of which two have no registers. FLAT: one KV head, whose rows lie one behind the
// other in Q. A tile of 64 rows travels through registers into one of two LDS buffers while the
// tile before it is used (16-byte chunk c of row r lies at c ^ (r % chunks): 16 lanes that read the same
// chunk of neighbouring rows touch all banks).
// A score costs a wavefront 24 clocks of vector issue (fma, exp at a quarter of the rate, add) and 16 of the
// matrix pipe, so the products of a row and key block are issued between the exponentials of the one before it. That
// does not make them run at once: over a prompt of 8192 queries vector instructions are issued for 55 % of the busy
// cycles and the matrix pipe works for 34 %, nearly all of it together, so that neither of them alone binds.
template <typename TI>
constexpr int frags() { return sizeof(TI) == 2 ? 2 : 1; }
template <typename TI, int D, bool FLAT>
__global__ __launch_bounds__(NW * 64, 2) void kv_weight_kernel(const WeightParams p) {
  constexpr int KB = frags<TI>();
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
  Seq sq;
  if (find_block(p, blockIdx.x, &begin, &sq) < 0) return;
  const int range = blockIdx.y % p.n_ranges, kvh = blockIdx.y / p.n_ranges;
  const int key0 = ((int)blockIdx.x - begin) * p.wg_keys + wave * KB * KEYS;
  const int64_t tok_q = (int64_t)p.n_q_heads * D, tok_kv = (int64_t)p.n_kv_heads * D;

  // lane (rl, hf): 16-byte chunk 2 ks + hf of key rl of the fragment (keys behind the last repeat it)
  uint4 kf[KB][NKS];
  int32_t kp[KB];
#pragma unroll
  for (int f = 0; f < KB; ++f) {
    const int64_t key = (int64_t)sq.k0 + min(key0 + f * KEYS + rl, sq.used - 1);
    kp[f] = max(p.kv_pos[key], INT32_MIN + 1);   // (INT32_MIN is the position of rows that are none)
    const uint4* src = (const uint4*)((const TI*)p.k + key * tok_kv + kvh * D) + hf;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) kf[f][ks] = src[2 * ks];
  }
  const int n_rows = sq.n * p.group;
  const int tiles = (n_rows + TILE - 1) / TILE;
  int t0 = (int)((int64_t)tiles * range / p.n_ranges), t1 = (int)((int64_t)tiles * (range + 1) / p.n_ranges);

  // ---- a tile on its way: ST chunks of Q a lane, and of every row its LSE and position ----
  const TI* const q0 = (const TI*)p.q + sq.q0 * tok_q;
  const float* const lse0 = p.lse + (int64_t)sq.q0 * p.n_q_heads;
  const int32_t* const pos0 = p.q_pos + sq.q0;
  RowAt at[FLAT ? 1 : ST], mine;
  const int by_node = TILE / p.group, by_head = TILE % p.group;
  auto start = [&](int t) {
    mine.set(t * TILE + lane, p.group);
    if (!FLAT)
#pragma unroll
      for (int i = 0; i < ST; ++i) at[FLAT ? 0 : i].set(t * TILE + i * RPI + tid / CH, p.group);
  };
  uint4 st[ST];
  float st_lse;
  int32_t st_pos;
  auto fetch = [&](int t) {
#pragma unroll
    for (int i = 0; i < ST; ++i) {
      st[i] = make_uint4(0, 0, 0, 0);
      if (FLAT) {
        const int r = t * TILE + i * RPI + tid / CH;
        if (r < n_rows) st[i] = ((const uint4*)(q0 + (int64_t)r * D))[tid % CH];
      } else {
        RowAt& a = at[FLAT ? 0 : i];
        if (a.node < sq.n)
          st[i] = ((const uint4*)(q0 + a.node * tok_q + (kvh * p.group + a.head) * D))[tid % CH];
        a.advance(by_node, by_head, p.group);
      }
    }
    st_lse = INFINITY;
    st_pos = INT32_MIN;
    if (mine.node < sq.n) {
      st_lse = FLAT ? lse0[t * TILE + lane] : lse0[(int64_t)mine.node * p.n_q_heads + kvh * p.group + mine.head];
      st_pos = pos0[mine.node];
    }
    mine.advance(by_node, by_head, p.group);
  };
  // a row that sees no key anywhere (LSE = -inf), and one behind the last, is none: it weighs nothing
  auto put = [&](int to) {
    if (st_lse == -INFINITY) {
      st_lse = INFINITY;
      st_pos = INT32_MIN;
    }
#pragma unroll
    for (int i = 0; i < ST; ++i) {
      const int r = i * RPI + tid / CH;
      *(uint4*)(tile[to] + r * ROW + (((tid % CH) ^ (r & (CH - 1))) << 4)) = st[i];
    }
    lse_of[to][wave][lane] = st_lse * kLog2e;
    pos_of[to][wave][lane] = st_pos;
  };

  const bool look = t1 - t0 > 2;
  if (!look && t0 < t1) {   // (requested with the keys)
    start(t0);
    fetch(t0);
  }
  float old[KB];
#pragma unroll
  for (int f = 0; f < KB; ++f) {
    old[f] = 0.f;
    if (p.part == nullptr && p.decay != 0.f && key0 + f * KEYS + rl < sq.used)
      old[f] = p.weight[(int64_t)sq.k0 + key0 + f * KEYS + rl];
  }
  int32_t k_max = INT32_MIN, k_min = INT32_MAX;
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
  if (look) {
    // the tiles between the first and the last row that sees any key of the workgroup
    if (lane == 0) wg_k_min[wave] = k_min;
    __syncthreads();
    int32_t lo = wg_k_min[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) lo = min(lo, wg_k_min[w]);
    const int n0 = t0 * TILE / p.group, n1 = min(sq.n, (t1 * TILE - 1) / p.group + 1);
    int first = INT32_MAX, last = -1;
    for (int i = n0 + tid; i < n1; i += NW * 64)
      if (pos0[i] >= lo) {
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
    first = __builtin_amdgcn_readfirstlane(first);
    last = __builtin_amdgcn_readfirstlane(last);
    if (last < 0) {
      t1 = t0;
    } else {
      t0 = max(t0, first * p.group / TILE);
      t1 = min(t1, ((last + 1) * p.group - 1) / TILE + 1);
    }
    if (t0 < t1) {
      start(t0);
      fetch(t0);
    }
  }
  if (t0 < t1) put(t0 & 1);

  float sum[KB];
#pragma unroll
  for (int f = 0; f < KB; ++f) sum[f] = 0.f;
  for (int t = t0; t < t1; ++t) {
    const int cur = t & 1;
    // which of the tile's rows see any of the wavefront's keys, and which not all
    const bool real = st_pos != INT32_MIN;
    const uint64_t none = __builtin_amdgcn_ballot_w64(!real);
    const uint64_t some = __builtin_amdgcn_ballot_w64(real && st_pos >= k_min);
    const uint64_t hide = __builtin_amdgcn_ballot_w64(real && st_pos < k_max);
    __syncthreads();
    if (t + 1 < t1) fetch(t + 1);
    // score i of lane (rl, hf) in a row and key block: key rl, row (i / 4) * 8 + hf * 4 + i % 4
    auto q_chunk = [&](int rb, int ks) -> uint4 {
      const int r = rb * 32 + rl;
      return *(const uint4*)(tile[cur] + r * ROW + (((2 * ks + hf) ^ (r & (CH - 1))) << 4));
    };
    auto lse_rows = [&](int rb, floatx4_t (&lr)[4]) {
#pragma unroll
      for (int a = 0; a < 4; ++a)
        lr[a] = *(const floatx4_t*)&lse_of[cur][wave][rb * 32 + a * 8 + hf * 4];
    };
    auto term = [&](const floatx16_t& s, const floatx4_t (&lr)[4], int i) {
      return __builtin_amdgcn_exp2f(fmaf(s[i], p.scale_log2, -lr[i >> 2][i & 3]));
    };
    bool masked = some != 0;
    if (KB > 1 && some != 0 && hide == 0) {
      float before[KB];
#pragma unroll
      for (int f = 0; f < KB; ++f) before[f] = sum[f];
      constexpr int RB = TILE / 32, NB = RB * KB, PER = 16 / NKS > 0 ? 16 / NKS : 1;
      floatx16_t s[2];
      floatx4_t lr[RB][4];
      uint4 qf[NKS];
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) qf[ks] = q_chunk(0, ks);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) lse_rows(rb, lr[rb]);
#pragma unroll
      for (int j = 0; j <= NB; ++j) {   // products of block j, exponentials of block j - 1
        float x[2] = {0.f, 0.f};
        if (j < NB)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[j & 1][i] = 0.f;
        // a step behind a product: arguments of PER scores, exponentials of the PER before them, the
        // sum of those before (neither waits for the instruction in front of it)
        float e[16];
#pragma unroll
        for (int ks = 0; ks < NKS + 2; ++ks) {
          if (j < NB && ks < NKS) {
            s[j & 1] = product(qf[ks], kf[j % KB][ks], s[j & 1], TI());
            if (j % KB == KB - 1 && j / KB + 1 < RB) qf[ks] = q_chunk(j / KB + 1, ks);
          }
          if (j > 0) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
              const int a = ks * PER + i, b = a - PER, c = b - PER;
              if (c >= 0 && c < 16) x[c & 1] += e[c];
              if (b >= 0 && b < 16) e[b] = __builtin_amdgcn_exp2f(e[b]);
              if (a < 16) e[a] = fmaf(s[(j - 1) & 1][a], p.scale_log2, -lr[(j - 1) / KB][a >> 2][a & 3]);
            }
          }
          if (j < NB) __builtin_amdgcn_sched_barrier(0);
        }
        if (j > 0) sum[(j - 1) % KB] += x[0] + x[1];
      }
      // A row that is none adds exp(-inf) = 0, or a NaN where its product with a key that is not finite is one: then
      // the tile is done with its mask.
      masked = false;
      if (none != 0) {
        bool nan = false;
#pragma unroll
        for (int f = 0; f < KB; ++f) nan |= sum[f] != sum[f];
        masked = __builtin_amdgcn_ballot_w64(nan) != 0;
        if (masked)
#pragma unroll
          for (int f = 0; f < KB; ++f) sum[f] = before[f];
      }
    }
    if (__builtin_expect(masked, KB == 1)) {
#pragma unroll
      for (int rb = 0; rb < TILE / 32; ++rb) {
        floatx4_t lr[4];
        lse_rows(rb, lr);
        floatx16_t s[KB];
#pragma unroll
        for (int f = 0; f < KB; ++f)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[f][i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) {
          const uint4 qf = q_chunk(rb, ks);
#pragma unroll
          for (int f = 0; f < KB; ++f) s[f] = product(qf, kf[f][ks], s[f], TI());
        }
#pragma unroll
        for (int f = 0; f < KB; ++f) {
          float x[2] = {0.f, 0.f};
#pragma unroll
          for (int a = 0; a < 4; ++a) {
            const int4 q = *(const int4*)&pos_of[cur][wave][rb * 32 + a * 8 + hf * 4];
            const int32_t qp[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float e = term(s[f], lr, 4 * a + i);
              x[i & 1] += qp[i] >= kp[f] ? e : 0.f;
            }
          }
          sum[f] += x[0] + x[1];
        }
      }
    }
    if (t + 1 < t1) put(cur ^ 1);
  }
#pragma unroll
  for (int f = 0; f < KB; ++f) {
    const float x = sum[f] + __shfl_xor(sum[f], 32, 64);
    const int key = key0 + f * KEYS + rl;
    if (hf == 0 && key < sq.used) {
      const int64_t to = (int64_t)sq.k0 + key;
      if (p.part != nullptr)
        p.part[(int64_t)blockIdx.y * p.total_kv + to] = x;
      else
        p.weight[to] = p.decay != 0.f ? fmaf(old[f], p.decay, x) : x;
    }
  }
}

// weight <- decay * weight + the parts: four threads a key, each every fourth part in order, then theirs
// in order.
constexpr int SUM_KEYS = 64;
__global__ __launch_bounds__(256) void kv_weight_sum_kernel(const WeightParams p) {
  __shared__ float sums[4][SUM_KEYS];
  int begin = 0;
  Seq sq;
  const int per = p.wg_keys / SUM_KEYS;
  const int x = (int)wide_block();
  if (find_block(p, x / per, &begin, &sq) < 0) return;
  const int lane = threadIdx.x & 63, quarter = threadIdx.x >> 6;
  const int key = (x / per - begin) * p.wg_keys + x % per * SUM_KEYS + lane;
  const int64_t at = (int64_t)sq.k0 + min(key, sq.used - 1);
  const int n = p.n_ranges * p.n_kv_heads;
  const float old = quarter == 0 && p.decay != 0.f ? p.weight[at] : 0.f;
  float t = 0.f;
  constexpr int U = 8;   // parts in flight
  for (int i = quarter; i < n; i += 4 * U) {
    float x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = i + 4 * u < n ? p.part[(int64_t)(i + 4 * u) * p.total_kv + at] : 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) t += x[u];
  }
  sums[quarter][lane] = t;
  __syncthreads();
  if (quarter == 0 && key < sq.used) {
    t = ((sums[0][lane] + sums[1][lane]) + sums[2][lane]) + sums[3][lane];
    p.weight[at] = p.decay != 0.f ? fmaf(old, p.decay, t) : t;
  }
}

constexpr int64_t kMaxParts = 65535;   // the grid's second dimension
struct WeightPlan {
  int wg_keys;      // keys of a block
  int64_t blocks;   // there can be
  int n_ranges;
  size_t bytes;
};
// (what a workgroup's start costs, in tiles. us for 1, 3 and 5: 16 queries over 32 sequences 31.1, 24.4, 24.4; 64 over 2
// of 8192 keys 14.3, 14.1, 18.3; 512 over 4 of 4096 55.2, 50.3, 50.3)
constexpr double kStartTiles = 3;
// (and the launch that adds the parts up: 16 queries over 8 times 4096 keys in one range 11.0 us, in two 13.1, 32 over 3 times
// 5000 to 20000 16.8 and 18.4)
constexpr double kSumTiles = 3;
WeightPlan weight_plan(const cp_shape& s) {
  WeightPlan pl = {};
  const int64_t rows = (s.total_q * (s.n_q_heads / s.n_kv_heads) + s.batch - 1) / s.batch;
  const int64_t tiles = (rows + TILE - 1) / TILE;   // of a sequence, on average
  pl.wg_keys = NW * KEYS * (s.dtype == CP_FP32 ? frags<float>() : frags<bf16_t>());
  pl.blocks = s.total_kv / pl.wg_keys + s.batch;
  // Ranges of the rows: as many as make the least of (rounds of workgroups, two a CU, and one for the
  // tail) times (tiles of one, and what it costs to begin). Which of them see nothing is not known here.
  int64_t n = 1;
  double least = 1e30;
  for (int64_t i = 1; i <= 128 && i <= tiles && i * s.n_kv_heads <= kMaxParts; ++i) {
    const double cost = ((double)(pl.blocks * s.n_kv_heads * i) / 512 + 1) *
                        (kStartTiles + (double)((tiles + i - 1) / i)) +
                        (i * s.n_kv_heads > 1 ? kSumTiles : 0);
    if (cost < least) {
      least = cost;
      n = i;
    }
  }
  pl.n_ranges = (int)n;
  const int64_t parts = n * s.n_kv_heads;
  pl.bytes = parts > 1 ? (size_t)parts * s.total_kv * 4 : 0;
  return pl;
}

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
  if (s.batch > kMaxWalkedBatch) return CP_ERR_SHAPE;
  if (s.total_kv == 0) return CP_OK;
  // key indices, rows and a token's channels in 31 bits
  if (s.total_kv > INT32_MAX - 256 || s.total_q * s.n_q_heads > INT32_MAX - TILE ||
      (int64_t)s.n_q_heads * s.head_dim > INT32_MAX)
    return CP_ERR_SHAPE;
  const WeightPlan pl = weight_plan(s);
  if (pl.bytes > 0 && (workspace == nullptr || ((uintptr_t)workspace & 255u) != 0 ||
                       workspace_bytes < pl.bytes))
    return CP_ERR_WORKSPACE;
  const int64_t parts = (int64_t)pl.n_ranges * s.n_kv_heads;
  if (parts > kMaxParts) return CP_ERR_SHAPE;
  WeightParams p = {};
  p.q = q; p.q_pos = q_pos; p.cu_q = cu_seqlens_q;
  p.k = k_cache; p.kv_pos = kv_pos_cache; p.cu_kv = cu_seqlens_kv; p.used = seq_used;
  p.lse = lse; p.weight = weight;
  p.part = pl.bytes > 0 ? (float*)workspace : nullptr;
  p.total_q = s.total_q; p.total_kv = s.total_kv; p.batch = s.batch;
  p.n_q_heads = s.n_q_heads; p.n_kv_heads = s.n_kv_heads; p.group = s.n_q_heads / s.n_kv_heads;
  p.n_ranges = pl.n_ranges;
  p.wg_keys = pl.wg_keys;
  p.scale_log2 = (s.softmax_scale > 0.f ? s.softmax_scale : 1.0f / sqrtf((float)s.head_dim)) * kLog2e;
  p.decay = decay;
  hipStream_t st = (hipStream_t)stream;
  const dim3 grid((unsigned)pl.blocks, (unsigned)parts);
#define CP_WEIGHT(TI, D)                                                                            \
  if (s.n_kv_heads == 1)                                                                            \
    hipLaunchKernelGGL((kv_weight_kernel<TI, D, true>), grid, dim3(NW * 64), 0, st, p);              \
  else                                                                                              \
    hipLaunchKernelGGL((kv_weight_kernel<TI, D, false>), grid, dim3(NW * 64), 0, st, p)
  if (s.dtype == CP_FP32) {
    if (s.head_dim == 64) { CP_WEIGHT(float, 64); }
    else { CP_WEIGHT(float, 128); }
  } else {
    if (s.head_dim == 64) { CP_WEIGHT(bf16_t, 64); }
    else { CP_WEIGHT(bf16_t, 128); }
  }
#undef CP_WEIGHT
  if (check_launch() != CP_OK) return CP_ERR_LAUNCH;
  if (p.part == nullptr) return CP_OK;
  hipLaunchKernelGGL(kv_weight_sum_kernel, wide_grid(pl.blocks * (p.wg_keys / SUM_KEYS)), dim3(256), 0, st, p);
  return check_launch();
}
