// Attention of trees of drafted tokens over the persistent KV cache (speculative decoding on a
// rank's share of it), and the commit of the accepted paths.
//
// Sequence b has n_b drafted nodes. Node i sees cache slot j < used_b iff kv_pos[j] <= q_pos[i],
// and node t of its own tree iff bit t of its mask is set. With s_j = scale q.k_j over what it sees,
//   O = sum_j e^(s_j - m) v_j / sum_j e^(s_j - m),   LSE = m + log sum_j e^(s_j - m),
// in one pass over the keys with a running maximum m and sum (online softmax).
//
// The n_b nodes times the `group` query heads of a KV head are the rows of one product against that
// head's keys; rows are cut into row blocks and keys into sub-tiles of 32, first the cached ones,
// then the tree's own. S^T = K Q^T and O^T += V^T P^T run on 32x32 MFMAs with the keys (channels) on
// the M side and the rows on the N side, which keeps a row's statistics in one lane pair and
// feeds P to the second product from the registers the first one left it in.
//
// All (KV head, sequence, row block) spans, cut into tiles, form one line that is dealt out to the
// workgroups in equal shares, whatever the sequences' lengths; a span that falls into several
// shares leaves fp32 parts that a second launch joins (the merge of Appendix B, Equation 4).
#include <math.h>

#include "cp_scan.h"

namespace cp {
namespace {

#define CP_LDS_AS __attribute__((address_space(3)))
#define CP_GLB_AS __attribute__((address_space(1)))

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef short shortx4_t __attribute__((ext_vector_type(4)));

constexpr int SUB = 32;   // keys of a sub-tile

// ---------------------------------------------------------------------------
// The line of tiles
// ---------------------------------------------------------------------------
struct TreeParams {
  const void* q;
  const int32_t* q_pos;
  const int32_t* cu_q;
  const void* k_new;       // NULL: the tree's own keys are another rank's
  const void* v_new;
  const uint64_t* mask;    // [total_q][words]
  const void* k;
  const void* v;
  const int32_t* kv_pos;
  const int32_t* cu_kv;
  const int32_t* used;     // or NULL: all slots of a sequence's range
  void* out;
  float* lse;
  float* part_o;           // [2 * n_wg][row block][D], not normalised
  float* part_ml;          // [2 * n_wg][row block][2]: running maximum (log2 domain), sum
  int64_t total_q, total_kv;
  int32_t batch, words, n_q_heads, n_kv_heads, group;
  int32_t n_wg, log2_wg;   // workgroups among which the line is dealt out, a power of two
  int32_t min_share;
  float scale_log2;
};

// What a sequence holds. Boundaries that contradict each other or the totals (they are read on the
// device, where nothing can be refused) are cut to what is there.
struct TreeSeq {
  int32_t q0, n, k0, used;   // first node, nodes, first cache slot, tokens in the cache
  int32_t spans, tiles;      // row blocks of a KV head, tiles of each
  __device__ __forceinline__ TreeSeq of_lane(int l) const {
    TreeSeq r;
    r.q0 = __builtin_amdgcn_readlane(q0, l);
    r.n = __builtin_amdgcn_readlane(n, l);
    r.k0 = __builtin_amdgcn_readlane(k0, l);
    r.used = __builtin_amdgcn_readlane(used, l);
    r.spans = __builtin_amdgcn_readlane(spans, l);
    r.tiles = __builtin_amdgcn_readlane(tiles, l);
    return r;
  }
  __device__ __forceinline__ int cached_subs() const { return (used + SUB - 1) / SUB; }
};

__device__ __forceinline__ int64_t wave_scan64(int64_t x) {   // of numbers from 0 to 2^48
  const int lo = wave_scan((int)(x & 0xffffff)), hi = wave_scan((int)(x >> 24));
  return ((int64_t)hi << 24) + lo;
}
__device__ __forceinline__ int64_t readlane64(int64_t x, int l) {
  return ((int64_t)__builtin_amdgcn_readlane((int)(x >> 32), l) << 32) |
         (uint32_t)__builtin_amdgcn_readlane((int)x, l);
}
__device__ __forceinline__ uint32_t div64(uint64_t a, uint32_t b) {   // quotient in 32 bits
  return (a >> 32) == 0 ? (uint32_t)a / b : (uint32_t)(a / b);
}

// The line of all tiles: KV heads, in each the sequences, in each the row blocks (RM rows), in each the
// tiles (SPT sub-tiles). Up to 64 sequences are described by one round trip, a lane each; of more, the
// lanes hold 64 at a time.
template <int RM, int SPT>
struct TreeLine {
  const TreeParams& p;
  TreeSeq mine;
  int64_t end;        // tiles of the sequences up to the lane's, of those held
  int held;           // first of the sequences held
  int64_t head_tiles, share;

  __device__ __forceinline__ void hold(int b0) {
    held = b0;
    const int b = min(b0 + (int)(threadIdx.x & 63), p.batch - 1);
    const int32_t a0 = p.cu_q[b], a1 = p.cu_q[b + 1], c0 = p.cu_kv[b], c1 = p.cu_kv[b + 1];
    const int32_t u = p.used != nullptr ? p.used[b] : INT32_MAX;
    mine.q0 = (int32_t)clamp64(a0, 0, p.total_q);
    mine.n = (int32_t)clamp64(a1, mine.q0, p.total_q) - mine.q0;
    mine.k0 = (int32_t)clamp64(c0, 0, p.total_kv);
    mine.used = (int32_t)clamp64(u, 0, clamp64(c1, mine.k0, p.total_kv) - mine.k0);
    mine.spans = (mine.n * p.group + RM - 1) / RM;   // (rows of a KV head in 31 bits: the host checks)
    const int subs = mine.cached_subs() + (p.k_new != nullptr ? (mine.n + SUB - 1) / SUB : 0);
    mine.tiles = subs > 0 ? (subs + SPT - 1) / SPT : 1;   // (nothing to see: one tile, empty)
    end = wave_scan64(b0 + (int)(threadIdx.x & 63) < p.batch ? (int64_t)mine.spans * mine.tiles : 0);
  }
  __device__ __forceinline__ explicit TreeLine(const TreeParams& params) : p(params) {
    head_tiles = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 64) {
      hold(b0);
      head_tiles += readlane64(end, 63);
    }
    const int64_t all = head_tiles * p.n_kv_heads;
    share = (all + p.n_wg - 1) >> p.log2_wg;
    if (share < p.min_share) share = p.min_share;
  }
  // The sequence of tile u of a KV head (-1: behind the last), and the tile where it begins.
  __device__ __forceinline__ int find(int64_t u, int64_t* begin, TreeSeq* sq) {
    int64_t base = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 64) {
      if (b0 != held) hold(b0);
      const uint64_t behind = __builtin_amdgcn_ballot_w64(base + end > u);
      if (behind != 0) {
        const int l = __builtin_ctzll(behind);
        *sq = mine.of_lane(l);
        *begin = base + readlane64(end, l) - (int64_t)sq->spans * sq->tiles;
        return b0 + l;
      }
      base += readlane64(end, 63);
    }
    return -1;
  }
  // The sequence that node t belongs to (-1: behind the last tree), and the tiles before it.
  __device__ __forceinline__ int find_node(int t, int64_t* begin, TreeSeq* sq) {
    int64_t base = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 64) {
      if (b0 != held) hold(b0);
      const bool in = b0 + (int)(threadIdx.x & 63) < p.batch;
      const uint64_t hit = __builtin_amdgcn_ballot_w64(in && t >= mine.q0 && t < mine.q0 + mine.n);
      if (hit != 0) {
        const int l = __builtin_ctzll(hit);
        *sq = mine.of_lane(l);
        *begin = base + readlane64(end, l) - (int64_t)sq->spans * sq->tiles;
        return b0 + l;
      }
      base += readlane64(end, 63);
    }
    return -1;
  }
};

// A workgroup's share of a span: tiles [t0, t1) of row block `span` of KV head kvh of a sequence.
struct TreePiece {
  TreeSeq sq;
  int kvh, span, t0, t1;
  int n_cached, n_subs;
  bool whole;        // the span is all in this piece: its result goes to the output
  int slot;          // otherwise: where the part goes
};
template <int RM, int SPT>
__device__ __forceinline__ bool tree_piece(TreeLine<RM, SPT>& line, int64_t u, int64_t u_end, TreePiece* x) {
  int64_t v = u, begin;
  x->kvh = 0;
  while (v >= line.head_tiles) {
    v -= line.head_tiles;
    ++x->kvh;
  }
  if (line.find(v, &begin, &x->sq) < 0) return false;
  const int64_t in = v - begin;
  x->span = (int)div64((uint64_t)in, (uint32_t)x->sq.tiles);
  x->t0 = (int)(in - (int64_t)x->span * x->sq.tiles);
  x->t1 = (int)min<int64_t>(x->sq.tiles, x->t0 + (u_end - u));
  x->n_cached = x->sq.cached_subs();
  x->n_subs = x->n_cached + (line.p.k_new != nullptr ? (x->sq.n + SUB - 1) / SUB : 0);
  x->whole = x->t0 == 0 && x->t1 == x->sq.tiles;
  // a share has at most one part that ends a span and one that begins one
  x->slot = 2 * (int)blockIdx.x + (x->t0 == 0 ? 1 : 0);
  return true;
}

// ---------------------------------------------------------------------------
// The kernel
// ---------------------------------------------------------------------------
__device__ __forceinline__ floatx16_t mfma32(bf16x8_t a, bf16x8_t b, floatx16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ floatx16_t mfma32(float a, float b, floatx16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ void to_lds16(const void* src, char* dst_wave_uniform) {
  __builtin_amdgcn_global_load_lds((const CP_GLB_AS void*)src, (CP_LDS_AS void*)dst_wave_uniform,
                                   16, 0, 0);
}
__device__ __forceinline__ float xor32(float x) { return __shfl_xor(x, 32, 64); }

// A sub-tile in LDS: 32 K rows, 32 V rows (16-byte chunks of a row permuted, see below), positions.
template <typename TI, int D>
struct SubTile {
  static constexpr int ROW = D * (int)sizeof(TI);
  static constexpr int CH = ROW / 16;              // 16-byte chunks of a row
  static constexpr int V_OFF = SUB * ROW;
  static constexpr int POS_OFF = 2 * SUB * ROW;
  static constexpr int BYTES = POS_OFF + 256;
  // Chunk c of K row r lies at c ^ k_perm(r): lanes that read the same chunk of neighbouring rows
  // touch different banks. V of bf16: a transposed read takes 32 bytes of four neighbouring rows;
  // chunk c lies at c ^ v_perm(r), which puts the 32-byte pieces of the four rows, and of the two
  // 16-lane groups that read neighbouring channels, into different banks. (V of fp32 is read along
  // its rows.)
  __device__ static constexpr int k_perm(int r) { return r & (CH - 1); }
  __device__ static constexpr int v_perm(int r) {
    if (sizeof(TI) == 4) return 0;
    return D == 128 ? (((r & 1) * 2) ^ (((r >> 1) & 1) * 5)) << 1 : (r & 3) << 1;
  }
};

template <typename TO>
__device__ __forceinline__ void store4(TO* dst, floatx4_t x);
template <>
__device__ __forceinline__ void store4<float>(float* dst, floatx4_t x) {
  *(floatx4_t*)dst = x;
}
template <>
__device__ __forceinline__ void store4<bf16_t>(bf16_t* dst, floatx4_t x) {
  bf16x4_t y;
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = static_cast<bf16_t>(x[i]);
  *(bf16x4_t*)dst = y;
}

// bf16 pairs: 1.0 where the element is not finite and not of sign `minus` (a NaN counts for both),
// else 0; and the pair with what is not finite replaced by zero.
__device__ __forceinline__ uint32_t not_finite(uint32_t x, bool minus) {
  uint32_t r = 0;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t e = (x >> (16 * h)) & 0xffffu;
    const bool nan = (e & 0x7fffu) > 0x7f80u;
    if (nan || e == (minus ? 0xff80u : 0x7f80u)) r |= 0x3f80u << (16 * h);
  }
  return r;
}
__device__ __forceinline__ uint32_t only_finite(uint32_t x) {
  if ((x & 0x7f80u) == 0x7f80u) x &= 0xffff0000u;
  if ((x & 0x7f800000u) == 0x7f800000u) x &= 0xffffu;
  return x;
}
__device__ __forceinline__ uint32_t any_not_finite(uint32_t x) {   // 1 or 0, without a branch
  return (uint32_t)((x & 0x7f80u) == 0x7f80u) | (uint32_t)((x & 0x7f800000u) == 0x7f800000u);
}

// KS: the wavefronts of a workgroup hold the same 32 C rows and take turns at the sub-tiles (few
// rows: the keys are what there is to share out). Otherwise every wavefront holds 32 C rows of its
// own and all read every sub-tile of a tile.
template <bool KS, int C, int NW>
struct Form {
  static constexpr int RW = 32 * C;                    // rows of a wavefront
  static constexpr int RM = KS ? RW : RW * NW;         // rows of a row block
  static constexpr int SPT = KS ? NW : 2;              // sub-tiles of a tile
};
template <typename TI, int D, bool KS, int C, int NW>
constexpr int tree_smem() {
  using F = Form<KS, C, NW>;
  const int tiles = F::SPT * SubTile<TI, D>::BYTES;
  const int join = KS ? NW * (F::RW * (D + 4) + 2 * F::RW) * 4 : 0;
  return tiles > join ? tiles : join;
}

// TI: K, V and Q. TO: O. P goes into the second product as TERMS bf16 terms (bf16 inputs): one
// where O is rounded to bf16 itself, three (24 bits) where it stays fp32.
template <typename TI, int D, bool KS, int C, int NW, int TERMS, typename TO>
__global__ __launch_bounds__(NW * 64) void tree_attn_kernel(const TreeParams p) {
  using F = Form<KS, C, NW>;
  using T = SubTile<TI, D>;
  constexpr bool F32 = sizeof(TI) == 4;
  constexpr int NKS = T::ROW / 32, NCB = D / 32;
  extern __shared__ __align__(16) char smem[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rl = lane & 31, hf = lane >> 5;   // row (N side) or key / channel (M side), half
  TreeLine<F::RM, F::SPT> line(p);
  int64_t u = blockIdx.x * line.share;
  const int64_t u_end = min(line.head_tiles * p.n_kv_heads, u + line.share);
  const int64_t tok_q = (int64_t)p.n_q_heads * D, tok_kv = (int64_t)p.n_kv_heads * D;

  while (u < u_end) {
    TreePiece pc;
    if (!tree_piece(line, u, u_end, &pc)) break;
    const TreeSeq& sq = pc.sq;
    const int kvh = pc.kvh, t0 = pc.t0, t1 = pc.t1, n_cached = pc.n_cached, n_subs = pc.n_subs;
    const int n_rows = sq.n * p.group;

    // ---- the wavefront's rows ----
    int row[C];            // within (sequence, KV head)
    int node[C];           // of all nodes; -1: a row behind the last one
    int32_t qp[C];
    uint4 qf[C][NKS];      // lane (rl, hf): 16-byte chunk 2 ks + hf of row rl
    int32_t q_min = INT32_MAX, q_max = INT32_MIN;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      row[c] = pc.span * F::RM + (KS ? 0 : wave * F::RW) + c * 32 + rl;
      const bool ok = row[c] < n_rows;
      const int nd = ok ? (uint32_t)row[c] / (uint32_t)p.group : 0;
      node[c] = ok ? sq.q0 + nd : -1;
      const int head = kvh * p.group + (ok ? row[c] - nd * p.group : 0);
      const uint4* src = (const uint4*)((const TI*)p.q + (ok ? node[c] : 0) * tok_q + head * D) + hf;
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) {
        qf[c][ks] = make_uint4(0, 0, 0, 0);
        if (ok) qf[c][ks] = src[2 * ks];
      }
      qp[c] = ok ? p.q_pos[node[c]] : INT32_MIN;
      if (ok) {
        q_min = min(q_min, qp[c]);
        q_max = max(q_max, qp[c]);
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      q_min = min(q_min, __shfl_xor(q_min, o, 64));
      q_max = max(q_max, __shfl_xor(q_max, o, 64));
    }

    float m_run[C], l_run[C];
    floatx16_t o_acc[C][NCB];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      m_run[c] = -INFINITY;
      l_run[c] = 0.f;
#pragma unroll
      for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
        for (int i = 0; i < 16; ++i) o_acc[c][cb][i] = 0.f;
    }

    // Requests for sub-tile `st` into LDS at `dst`: rows behind its last one repeat that one (and are
    // masked by their index). `w` of `nw` wavefronts share the requests out.
    auto request = [&](int st, char* dst, int w, int nw) {
      const bool own = st >= n_cached;
      const int first = (own ? st - n_cached : st) * SUB;
      const int last = min(SUB, (own ? sq.n : sq.used) - first) - 1;
      const int64_t base = (int64_t)(own ? sq.q0 : sq.k0) + first;
      const TI* kt = (const TI*)(own ? p.k_new : p.k) + base * tok_kv + kvh * D;
      const TI* vt = (const TI*)(own ? p.v_new : p.v) + base * tok_kv + kvh * D;
      constexpr int RPI = 64 / T::CH;          // rows of a request
      for (int i = w; i < SUB / RPI; i += nw) {
        const int r = i * RPI + lane / T::CH, slot = lane % T::CH;
        const int64_t off = (int64_t)min(r, last) * tok_kv;
        to_lds16((const uint4*)(kt + off) + (slot ^ T::k_perm(r)), dst + i * 1024);
        to_lds16((const uint4*)(vt + off) + (slot ^ T::v_perm(r)), dst + T::V_OFF + i * 1024);
      }
      if (!own && w == 0)
        __builtin_amdgcn_global_load_lds((const CP_GLB_AS void*)(p.kv_pos + base + min(rl, last)),
                                         (CP_LDS_AS void*)(dst + T::POS_OFF), 4, 0, 0);
    };

    // S, P and O of one sub-tile that lies in LDS at `buf`.
    auto compute = [&](int st, const char* buf) {
      const bool own = st >= n_cached;
      const int first = (own ? st - n_cached : st) * SUB;
      const int cnt = min(SUB, (own ? sq.n : sq.used) - first);
      bool masked = own || cnt < SUB;
      if (!own) {
        const int32_t kp = *(const int32_t*)(buf + T::POS_OFF + rl * 4);
        if (__builtin_amdgcn_ballot_w64(kp <= q_max) == 0) return;   // none of the rows sees any
        masked = masked || __builtin_amdgcn_ballot_w64(kp > q_min) != 0;
      }
      floatx16_t s[C];
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[c][i] = 0.f;
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) {
        const uint4 a = *(const uint4*)(buf + rl * T::ROW + (((2 * ks + hf) ^ T::k_perm(rl)) << 4));
#pragma unroll
        for (int c = 0; c < C; ++c) {
          if constexpr (F32) {
            const floatx4_t af = __builtin_bit_cast(floatx4_t, a);
            const floatx4_t qv = __builtin_bit_cast(floatx4_t, qf[c][ks]);
#pragma unroll
            for (int x = 0; x < 4; ++x) s[c] = mfma32(af[x], qv[x], s[c]);
          } else {
            s[c] = mfma32(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, qf[c][ks]),
                          s[c]);
          }
        }
      }
      // score i of lane (rl, hf): key (i / 4) * 8 + hf * 4 + i % 4
      bool odd_v = false;   // V holds what is not finite, which rows that do not see it must not meet
      if (masked) {
        const uint32_t there = cnt == SUB ? ~0u : (1u << cnt) - 1;
        int32_t kp[16];
        if (!own) {
#pragma unroll
          for (int a = 0; a < 4; ++a) {
            const int4 x = *(const int4*)(buf + T::POS_OFF + (a * 8 + hf * 4) * 4);
            kp[4 * a] = x.x; kp[4 * a + 1] = x.y; kp[4 * a + 2] = x.z; kp[4 * a + 3] = x.w;
          }
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
          uint32_t see = there;
          if (own) {
            const int word = (st - n_cached) >> 1;
            see = 0;
            if (node[c] >= 0 && word < p.words)
              see = (uint32_t)(p.mask[(int64_t)node[c] * p.words + word] >> (((st - n_cached) & 1) * 32)) & there;
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const bool vis = ((see >> ((i >> 2) * 8 + hf * 4 + (i & 3))) & 1) != 0 &&
                             (own || kp[i] <= qp[c]);
            s[c][i] = vis ? s[c][i] : -INFINITY;
          }
        }
#pragma unroll
        for (int i = 0; i < SUB * T::ROW / 1024; ++i) {
          const uint4 x = *(const uint4*)(buf + T::V_OFF + i * 1024 + lane * 16);
          if constexpr (F32)
            odd_v |= (x.x & 0x7f800000u) == 0x7f800000u || (x.y & 0x7f800000u) == 0x7f800000u ||
                     (x.z & 0x7f800000u) == 0x7f800000u || (x.w & 0x7f800000u) == 0x7f800000u;
          else
            odd_v |= (any_not_finite(x.x) | any_not_finite(x.y) | any_not_finite(x.z) |
                      any_not_finite(x.w)) != 0;
        }
        odd_v = __builtin_amdgcn_ballot_w64(odd_v) != 0;
      }
      u32x4_t pb[C][TERMS][2];   // P^T of keys 0..15 and 16..31, per term
      float pf[C][F32 ? 16 : 1];
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float mx = s[c][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[c][i]);
        mx = fmaxf(mx, xor32(mx));
        const float m_new = fmaxf(m_run[c], mx * p.scale_log2);
        const float m_use = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m_run[c] - m_use);
        m_run[c] = m_new;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float e = __builtin_amdgcn_exp2f(fmaf(s[c][i], p.scale_log2, -m_use));
          sum += e;
          if constexpr (F32) {
            pf[c][i] = e;
          } else {
#pragma unroll
            for (int t = 0; t < TERMS; ++t) {
              const bf16_t x = static_cast<bf16_t>(e);
              const uint32_t bits = __builtin_bit_cast(uint16_t, x);
              if ((i & 1) == 0) pb[c][t][i >> 3][(i & 7) >> 1] = bits;
              else pb[c][t][i >> 3][(i & 7) >> 1] |= bits << 16;
              e -= static_cast<float>(x);
            }
          }
        }
        l_run[c] = fmaf(l_run[c], alpha, sum);
        if (__builtin_amdgcn_ballot_w64(alpha != 1.f) != 0) {
#pragma unroll
          for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
            for (int i = 0; i < 16; ++i) o_acc[c][cb][i] *= alpha;
        }
      }
      if constexpr (F32) {
        // O^T += V^T P^T, a key pair a step: k slot hf of step i is the key of score i
#pragma unroll
        for (int cb = 0; cb < NCB; ++cb) {
          floatx16_t plus[C], minus[C];   // how many visible infinities of either sign (a NaN: both)
#pragma unroll
          for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) plus[c][i] = minus[c][i] = 0.f;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int r = (i >> 2) * 8 + hf * 4 + (i & 3);
            float v = *(const float*)(buf + T::V_OFF + r * T::ROW + (cb * 32 + rl) * 4);
            if (odd_v) {
              const bool fin = fabsf(v) < INFINITY;
              const float up = fin || v == -INFINITY ? 0.f : 1.f, dn = fin || v == INFINITY ? 0.f : 1.f;
#pragma unroll
              for (int c = 0; c < C; ++c) {
                const float seen = pf[c][i] != 0.f ? 1.f : 0.f;
                plus[c] = mfma32(up, seen, plus[c]);
                minus[c] = mfma32(dn, seen, minus[c]);
              }
              v = fin ? v : 0.f;
            }
#pragma unroll
            for (int c = 0; c < C; ++c) o_acc[c][cb] = mfma32(v, pf[c][i], o_acc[c][cb]);
          }
          if (odd_v) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
              for (int i = 0; i < 16; ++i)
                o_acc[c][cb][i] += (plus[c][i] > 0.f ? INFINITY : 0.f) + (minus[c][i] > 0.f ? -INFINITY : 0.f);
          }
        }
      } else {
        // O^T += V^T P^T: k slot j of half hf in step kb is key kb*16 + (j/4)*8 + hf*4 + j%4
        const int vj = (lane & 15) >> 2, vq = lane & 3, vg = (lane >> 4) & 1;
#pragma unroll
        for (int cb = 0; cb < NCB; ++cb) {
          u32x4_t v[2];
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const int r = kb * 16 + x * 8 + hf * 4 + vj;
              const int chunk = cb * 4 + vg * 2 + (vq >> 1);
              const char* at = buf + T::V_OFF + r * T::ROW + ((chunk ^ T::v_perm(r)) << 4) + (vq & 1) * 8;
              const u32x2_t z = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                                (CP_LDS_AS shortx4_t*)at));
              v[kb][2 * x] = z[0];
              v[kb][2 * x + 1] = z[1];
            }
          if (__builtin_expect(odd_v, 0)) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
              floatx16_t sign[2];   // how many visible infinities of either sign (a NaN: both)
#pragma unroll
              for (int m = 0; m < 2; ++m) {
#pragma unroll
                for (int i = 0; i < 16; ++i) sign[m][i] = 0.f;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                  u32x4_t a, seen;
#pragma unroll
                  for (int x = 0; x < 4; ++x) {
                    a[x] = not_finite(v[kb][x], m == 1);
                    seen[x] = ((pb[c][0][kb][x] & 0xffffu) != 0 ? 0x3f80u : 0) |
                              ((pb[c][0][kb][x] >> 16) != 0 ? 0x3f800000u : 0);
                  }
                  sign[m] = mfma32(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, seen),
                                   sign[m]);
                }
              }
#pragma unroll
              for (int i = 0; i < 16; ++i)
                o_acc[c][cb][i] += (sign[0][i] > 0.f ? INFINITY : 0.f) + (sign[1][i] > 0.f ? -INFINITY : 0.f);
            }
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
              for (int x = 0; x < 4; ++x) v[kb][x] = only_finite(v[kb][x]);
          }
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
              for (int t = 0; t < TERMS; ++t)
                o_acc[c][cb] = mfma32(__builtin_bit_cast(bf16x8_t, v[kb]),
                                      __builtin_bit_cast(bf16x8_t, pb[c][t][kb]), o_acc[c][cb]);
        }
      }
    };

    for (int t = t0; t < t1; ++t) {
      __syncthreads();   // the tile before has been read
      if (KS) {
        const int st = t * F::SPT + wave;
        if (st < n_subs) request(st, smem + wave * T::BYTES, 0, 1);
      } else {
        for (int x = 0; x < F::SPT; ++x)
          if (t * F::SPT + x < n_subs) request(t * F::SPT + x, smem + x * T::BYTES, wave, NW);
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      if (KS) {
        const int st = t * F::SPT + wave;
        if (st < n_subs) compute(st, smem + wave * T::BYTES);
      } else {
        for (int x = 0; x < F::SPT; ++x)
          if (t * F::SPT + x < n_subs) compute(t * F::SPT + x, smem + x * T::BYTES);
      }
    }
#pragma unroll
    for (int c = 0; c < C; ++c) l_run[c] += xor32(l_run[c]);

    // ---- the span's result, or this share's part of it ----
    auto write = [&](int r, int in_block, float m, float l, int ch, floatx4_t o4) {
      if (r >= n_rows) return;
      if (pc.whole) {
        const int nd = (uint32_t)r / (uint32_t)p.group;
        const int64_t at = (int64_t)(sq.q0 + nd) * p.n_q_heads + kvh * p.group + (r - nd * p.group);
        const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;   // (a NaN stays one)
        store4<TO>((TO*)p.out + at * D + ch, o4 * inv);
        if (ch == 0) p.lse[at] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
      } else {
        const int64_t at = (int64_t)pc.slot * F::RM + in_block;
        *(floatx4_t*)(p.part_o + at * D + ch) = o4;
        if (ch == 0) {
          p.part_ml[at * 2] = m;
          p.part_ml[at * 2 + 1] = l;
        }
      }
    };
    if constexpr (KS) {
      // the wavefronts' disjoint subsets of the keys are joined in LDS
      constexpr int OS = D + 4;                      // floats of a row
      constexpr int WS = F::RW * OS + 2 * F::RW;     // of a wavefront
      float* const cb0 = (float*)smem;
      __syncthreads();
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float* const mine = cb0 + wave * WS + (c * 32 + rl) * OS;
#pragma unroll
        for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
          for (int a = 0; a < 4; ++a)
            *(floatx4_t*)(mine + cb * 32 + a * 8 + hf * 4) =
                floatx4_t{o_acc[c][cb][4 * a], o_acc[c][cb][4 * a + 1], o_acc[c][cb][4 * a + 2],
                          o_acc[c][cb][4 * a + 3]};
        if (hf == 0) {
          cb0[wave * WS + F::RW * OS + c * 32 + rl] = m_run[c];
          cb0[wave * WS + F::RW * OS + F::RW + c * 32 + rl] = l_run[c];
        }
      }
      __syncthreads();
      for (int e = tid; e < F::RW * (D / 4); e += NW * 64) {
        const int r = e / (D / 4), ch = (e % (D / 4)) * 4;
        float m = -INFINITY, l = 0.f;
        floatx4_t o4 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) m = fmaxf(m, cb0[w * WS + F::RW * OS + r]);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          const float lw = cb0[w * WS + F::RW * OS + F::RW + r];
          const float f = m == -INFINITY ? lw   // (0, or a NaN)
                                         : __builtin_amdgcn_exp2f(cb0[w * WS + F::RW * OS + r] - m);
          const floatx4_t x = *(const floatx4_t*)(cb0 + w * WS + r * OS + ch);
          l = fmaf(lw, f, l);
          o4 += x * f;
        }
        write(pc.span * F::RM + r, r, m, l, ch, o4);
      }
      __syncthreads();
    } else {
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
          for (int a = 0; a < 4; ++a)
            write(row[c], wave * F::RW + c * 32 + rl, m_run[c], l_run[c], cb * 32 + a * 8 + hf * 4,
                  floatx4_t{o_acc[c][cb][4 * a], o_acc[c][cb][4 * a + 1], o_acc[c][cb][4 * a + 2],
                            o_acc[c][cb][4 * a + 3]});
    }
    u += t1 - t0;
  }
}

// ---------------------------------------------------------------------------
// Many rows (bf16): eight wavefronts with 32 rows each, a tile of 64 keys for all of them.
//
// Bound by the matrix pipe and, about as much, by the LDS reads that feed it (a fragment serves 32 rows).
// A step works on three sub-tiles: the products S^T of the next one and O^T of the one before are issued
// between the softmax arithmetic of the current one, which needs neither. The reference that the
// exponentials are taken against is raised only when a score exceeds it by 2^8 (O and the sum are
// rescaled then): they cancel in O / l, and what is rounded has the same relative error at any scale.
// A tile travels through registers into one of three LDS buffers: one holds the values of the
// sub-tile before, one the current tile, and one is being filled; one barrier a tile.
// ---------------------------------------------------------------------------
constexpr int MANY_WAVES = 8;
constexpr int MANY_ROWS = 32 * MANY_WAVES;
constexpr float kSlack = 8.f;

template <int J>
struct IntC {
  static constexpr int value = J;
};
// max over the two halves of a wavefront that share a row (inline assembly: through the builtin the
// compiler takes the two results of a swap of equal operands for equal; the s_nop covers the wait states
// that a lane swap needs after a vector write of its operands)
__device__ __forceinline__ float halves_max(float x) {
  float a = x, b = x;
  asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(b));
  return fmaxf(a, b);
}
// Keeps the computation of x where it is in the instruction stream.
__device__ __forceinline__ void pin(float& x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ void pin(u32x4_t& x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ void pin(floatx16_t& x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  bf16x2_t t;
  t[0] = static_cast<bf16_t>(a);
  t[1] = static_cast<bf16_t>(b);
  return __builtin_bit_cast(uint32_t, t);
}

template <int D>
struct ManyTile {
  using T = SubTile<bf16_t, D>;
  static constexpr int KEYS = 2 * SUB;
  static constexpr int V_OFF = KEYS * T::ROW;
  static constexpr int POS_OFF = 2 * KEYS * T::ROW;
  static constexpr int BYTES = POS_OFF + KEYS * 4;
  static constexpr int ZERO_OFF = 3 * BYTES;           // a sub-tile's worth of V, zeros
  static constexpr int SMEM = ZERO_OFF + SUB * T::ROW;
};

template <int D, int TERMS, typename TO>
__global__ __launch_bounds__(MANY_WAVES * 64) void tree_many_kernel(const TreeParams p) {
  using M = ManyTile<D>;
  using T = SubTile<bf16_t, D>;
  constexpr int NKS = D / 16, NCB = D / 32, NVF = 2 * NCB;
  constexpr int THREADS = MANY_WAVES * 64, RPI = THREADS / T::CH, CPT = M::KEYS / RPI;
  static_assert(NKS == NVF, "a V^T fragment takes the registers of a K fragment");
  extern __shared__ __align__(16) char smem[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rl = lane & 31, hf = lane >> 5;
  for (int i = tid * 16; i < SUB * T::ROW; i += THREADS * 16)
    *(uint4*)(smem + M::ZERO_OFF + i) = make_uint4(0, 0, 0, 0);
  int64_t u = 0, u_end = 1;
  const int64_t tok_q = (int64_t)p.n_q_heads * D, tok_kv = (int64_t)p.n_kv_heads * D;
  // LDS offsets of this lane inside a sub-tile: K fragment chunk 2 ks + hf of row rl; V^T fragments
  // (cb, kb): channels of block cb, keys kb*16 + x*8 + hf*4 + 0..3 (v_perm of a row depends on vj alone).
  // Chunks are permuted by exclusive-or, and so are the offsets of the others (ks * 32, cb * 64).
  const int koff = rl * T::ROW + ((hf ^ T::k_perm(rl)) << 4);
  const int vj = (lane & 15) >> 2, vq = lane & 3, vg = (lane >> 4) & 1;
  const int voff = (hf * 4 + vj) * T::ROW + (((vg * 2 + (vq >> 1)) ^ T::v_perm(vj)) << 4) + (vq & 1) * 8;
  static_assert(M::BYTES % 256 == 0 && M::V_OFF % 256 == 0 && SUB * T::ROW % 256 == 0, "as the permutation asks");

  for (bool first = true; first || u < u_end; first = false) {
    TreePiece pc;
    {
      // (described anew for every piece: the lanes' sequences would take registers all along)
      TreeLine<MANY_ROWS, 2> line(p);
      if (first) {
        u = blockIdx.x * line.share;
        u_end = min(line.head_tiles * p.n_kv_heads, u + line.share);
        if (u >= u_end) return;
      }
      if (!tree_piece(line, u, u_end, &pc)) return;
    }
    const TreeSeq& sq = pc.sq;
    const int kvh = pc.kvh, n_cached = pc.n_cached, n_subs = pc.n_subs;
    const int n_rows = sq.n * p.group;
    const int row = pc.span * MANY_ROWS + wave * 32 + rl;
    const bool ok = row < n_rows;
    const int nd = ok ? (uint32_t)row / (uint32_t)p.group : 0;
    const int node = sq.q0 + nd;
    const int head = kvh * p.group + (ok ? row - nd * p.group : 0);

    // ---- a tile on its way: K and V rows by 16-byte chunks, positions of the cached ones ----
    const bf16_t* const kc = (const bf16_t*)p.k + sq.k0 * tok_kv + kvh * D;
    const bf16_t* const vc = (const bf16_t*)p.v + sq.k0 * tok_kv + kvh * D;
    const bf16_t* const kt = (const bf16_t*)p.k_new + sq.q0 * tok_kv + kvh * D;
    const bf16_t* const vt = (const bf16_t*)p.v_new + sq.q0 * tok_kv + kvh * D;
    const bool has_tree = p.k_new != nullptr;
    static_assert(CPT <= 2, "chunks of a lane");
    uint4 st_k0, st_k1, st_v0, st_v1;   // (scalars: an array of these ends up in memory)
    int32_t st_pos = 0;
    auto fetch_row = [&](int idx, uint4& k, uint4& v) __attribute__((always_inline)) {
      // (keys behind the last of either kind repeat it, and are masked by their index; a choice between
      // values, since one between the variables would put them into memory)
      const bool own = has_tree && idx >= n_cached * SUB;
      const int key = own ? min(idx - n_cached * SUB, sq.n - 1) : min(idx, sq.used - 1);
      const int64_t off = key * tok_kv;
      const bf16_t* const kr = own ? kt + off : kc + off;
      const bf16_t* const vr = own ? vt + off : vc + off;
      k = ((const uint4*)kr)[tid % T::CH];
      v = ((const uint4*)vr)[tid % T::CH];
    };
    auto fetch = [&](int t) __attribute__((always_inline)) {
      fetch_row(t * M::KEYS + tid / T::CH, st_k0, st_v0);
      if constexpr (CPT > 1) fetch_row(t * M::KEYS + RPI + tid / T::CH, st_k1, st_v1);
      if (tid < M::KEYS) {
        const int idx = t * M::KEYS + tid;
        st_pos = idx < sq.used ? p.kv_pos[sq.k0 + idx] : CP_POS_PAD_KV;
      }
    };
    auto put_row = [&](char* buf, int r, const uint4& k, const uint4& v) __attribute__((always_inline)) {
      const int c = tid % T::CH;
      *(uint4*)(buf + r * T::ROW + ((c ^ T::k_perm(r & 31)) << 4)) = k;
      *(uint4*)(buf + M::V_OFF + r * T::ROW + ((c ^ T::v_perm(r & 31)) << 4)) = v;
    };
    auto put = [&](char* buf) __attribute__((always_inline)) {
      put_row(buf, tid / T::CH, st_k0, st_v0);
      if constexpr (CPT > 1) put_row(buf, RPI + tid / T::CH, st_k1, st_v1);
      if (tid < M::KEYS) *(int32_t*)(buf + M::POS_OFF + tid * 4) = st_pos;
    };
    if (n_subs > 0) fetch(pc.t0);

    uint4 qf[NKS];
    const uint4* const q_src = (const uint4*)((const bf16_t*)p.q + node * tok_q + head * D) + hf;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {
      qf[ks] = make_uint4(0, 0, 0, 0);
      if (ok) qf[ks] = q_src[2 * ks];
    }
    const int32_t qp = ok ? p.q_pos[node] : INT32_MIN;
    int32_t q_min = ok ? qp : INT32_MAX;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) q_min = min(q_min, __shfl_xor(q_min, o, 64));

    float ref = -INFINITY, l_run = 0.f;
    floatx16_t o_acc[NCB], s[2];
    u32x4_t pb[2][TERMS][2];               // P of the current sub-tile and the one before, in bf16 pairs per
                                           // term (keys 0..15, 16..31)
#pragma unroll
    for (int k = 0; k < TERMS; ++k) pb[1][k][0] = pb[1][k][1] = u32x4_t{0, 0, 0, 0};
    bool pending = false;                  // O^T of the sub-tile before has not been added yet
#pragma unroll
    for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
      for (int i = 0; i < 16; ++i) o_acc[cb][i] = 0.f;

    // (LDS addresses as numbers: `sub` is one of the wavefront's, uniform)
    auto lds = [](const char* sub) { return (uint32_t)(size_t)(CP_LDS_AS const char*)sub; };
    auto k_frag = [&](const char* sub, int ks) __attribute__((always_inline)) {
      return __builtin_bit_cast(uint4, *(CP_LDS_AS const u32x4_t*)(size_t)((lds(sub) + koff) ^ (ks * 32)));
    };
    auto v_frag = [&](const char* sub, int f) __attribute__((always_inline)) -> uint4 {   // f = cb * 2 + kb
      u32x4_t v;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const u32x2_t z = __builtin_bit_cast(
            u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((CP_LDS_AS shortx4_t*)(size_t)(
                         (((lds(sub) + M::V_OFF + voff) ^ ((f >> 1) * 64)) + ((f & 1) * 16 + x * 8) * T::ROW))));
        v[2 * x] = z[0];
        v[2 * x + 1] = z[1];
      }
      return __builtin_bit_cast(uint4, v);
    };
    // O^T of a sub-tile with nothing in between. ODD: V holds what is not finite, which reaches the rows
    // that see it, and no other.
    auto value_product = [&](auto parc, auto oddc, const char* sub) __attribute__((always_inline)) {
      constexpr int par = decltype(parc)::value;
      constexpr bool odd_v = decltype(oddc)::value != 0;
#pragma unroll
      for (int cb = 0; cb < NCB; ++cb) {
        u32x4_t v[2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) v[kb] = __builtin_bit_cast(u32x4_t, v_frag(sub, cb * 2 + kb));
        if constexpr (odd_v) {
          const u32x4_t t[2] = {pb[par][0][0], pb[par][0][1]};
#pragma unroll
            for (int m = 0; m < 2; ++m) {
              floatx16_t sign;   // how many visible infinities of this sign (a NaN counts for both)
#pragma unroll
              for (int i = 0; i < 16; ++i) sign[i] = 0.f;
#pragma unroll
              for (int kb = 0; kb < 2; ++kb) {
                u32x4_t a, seen;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                  a[x] = not_finite(v[kb][x], m == 1);
                  seen[x] = ((t[kb][x] & 0xffffu) != 0 ? 0x3f80u : 0) | ((t[kb][x] >> 16) != 0 ? 0x3f800000u : 0);
                }
                sign = mfma32(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, seen), sign);
              }
#pragma unroll
              for (int i = 0; i < 16; ++i) o_acc[cb][i] += sign[i] > 0.f ? (m == 0 ? INFINITY : -INFINITY) : 0.f;
            }
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
              for (int x = 0; x < 4; ++x) v[kb][x] = only_finite(v[kb][x]);
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int k = 0; k < TERMS; ++k)
            o_acc[cb] = mfma32(__builtin_bit_cast(bf16x8_t, v[kb]), __builtin_bit_cast(bf16x8_t, pb[par][k][kb]),
                               o_acc[cb]);
      }
    };

    // One step: softmax of sub-tile st (scores s[PAR], positions at `pos`, values at v_here), products S^T
    // of the next one (K rows at k_next) and O^T of the one before (V rows at v_prev). Returns whether
    // the sub-tile's V holds what is not finite and is hidden from a row.
    auto step = [&](auto parc, int st, const int32_t* pos, const char* v_here, const char* k_next,
                    const char* v_prev) __attribute__((always_inline)) -> bool {
      constexpr int PAR = decltype(parc)::value;
      // K fragments 0 .. NKS-1 of the next sub-tile, then V^T fragments of the one before: AHEAD of them
      // are on their way
      constexpr int FRAGS = NKS + NVF, AHEAD = 4;
      uint4 fr[AHEAD];
      auto request = [&](int g) __attribute__((always_inline)) {
        if (g < NKS) fr[g % AHEAD] = k_frag(k_next, g);
        else if (g < FRAGS) fr[g % AHEAD] = v_frag(v_prev, (g - NKS) % NCB * 2 + (g - NKS) / NCB);
      };
#pragma unroll
      for (int g = 0; g < AHEAD; ++g) request(g);
      const bool own = st >= n_cached;
      const int cnt = own ? sq.n - (st - n_cached) * SUB : sq.used - st * SUB;   // keys, if not SUB
      bool masked = own || cnt < SUB;
      if (!masked) masked = __builtin_amdgcn_ballot_w64(pos[rl] > q_min) != 0;
      uint32_t odd_here = 0;
      if (masked) {
        const uint32_t there = st >= n_subs ? 0 : cnt >= SUB ? ~0u : (1u << cnt) - 1;
        uint32_t see = there;
        if (own) {
          const int word = (st - n_cached) >> 1;
          see = 0;
          if (ok && word < p.words && there != 0)
            see = (uint32_t)(p.mask[(int64_t)node * p.words + word] >> (((st - n_cached) & 1) * 32)) & there;
        }
        see >>= hf * 4;   // (bit a * 8 + i: score 4 a + i)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const int4 x = *(const int4*)(pos + a * 8 + hf * 4);
          const int32_t kp[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int vis = (int)((see & (1u << (a * 8 + i))) != 0) & ((int)own | (int)(kp[i] <= qp));
            s[PAR][4 * a + i] = vis != 0 ? s[PAR][4 * a + i] : -INFINITY;
          }
        }
#pragma unroll
        for (int i = 0; i < SUB * T::ROW / 1024; ++i) {
          const uint4 x = *(const uint4*)(v_here + M::V_OFF + i * 1024 + lane * 16);
          odd_here |= any_not_finite(x.x) | any_not_finite(x.y) | any_not_finite(x.z) | any_not_finite(x.w);
        }
        odd_here = __builtin_amdgcn_ballot_w64(odd_here != 0) != 0;
      }
      float mx = fmaxf(fmaxf(s[PAR][0], s[PAR][1]), s[PAR][2]);
#pragma unroll
      for (int i = 3; i < 15; i += 2) mx = fmaxf(fmaxf(mx, s[PAR][i]), s[PAR][i + 1]);
      mx = halves_max(fmaxf(mx, s[PAR][15])) * p.scale_log2;
      const bool raise = mx > ref + kSlack;
      const bool any_raise = __builtin_amdgcn_ballot_w64(raise) != 0;
      float alpha = 1.f;
      if (any_raise) {
        if (raise) {
          alpha = __builtin_amdgcn_exp2f(ref - mx);
          ref = mx;
        }
        l_run *= alpha;
      }
      const float use = ref == -INFINITY ? 0.f : ref;

      // Softmax arithmetic in units, two MFMA slots or so apart: argument of score w, exponential of the
      // one before, sum and rounding of the one before that.
      constexpr int UNITS = 18, SLOTS = NKS + NVF * TERMS;
      float e[16], sum[2] = {0.f, 0.f};
      auto unit = [&](int w) __attribute__((always_inline)) {
        if (w >= 2) {
          const int i = w - 2;
          sum[i & 1] += e[i];
          if ((i & 1) == 1)
#pragma unroll
            for (int k = 0; k < TERMS; ++k) {
              const uint32_t x = pack_bf16(e[i - 1], e[i]);
              pb[PAR][k][i >> 3][(i & 7) >> 1] = x;
              if (k + 1 < TERMS) {   // what the term leaves over (exact)
                e[i - 1] -= __builtin_bit_cast(float, x << 16);
                e[i] -= __builtin_bit_cast(float, x & 0xffff0000u);
              }
            }
        }
        if (w >= 1 && w < 17) e[w - 1] = __builtin_amdgcn_exp2f(e[w - 1]);
        if (w < 16) e[w] = fmaf(s[PAR][w], p.scale_log2, -use);
      };
      auto units = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
        for (int w = slot * UNITS / SLOTS; w < (slot + 1) * UNITS / SLOTS; ++w) unit(w);
        __builtin_amdgcn_sched_barrier(0);
      };
#pragma unroll
      for (int i = 0; i < 16; ++i) s[PAR ^ 1][i] = 0.f;
#pragma unroll
      for (int g = 0; g < FRAGS; ++g) {
        const bf16x8_t a = __builtin_bit_cast(bf16x8_t, fr[g % AHEAD]);
        if (g < NKS) {
          s[PAR ^ 1] = mfma32(a, __builtin_bit_cast(bf16x8_t, qf[g < NKS ? g : 0]), s[PAR ^ 1]);
          request(g + AHEAD);
          units(g);
        } else {
          // (neighbouring fragments belong to different blocks of O)
          const int f = g - NKS, cb = f % NCB, kb = f / NCB;
#pragma unroll
          for (int k = 0; k < TERMS; ++k) {
            o_acc[cb] = mfma32(a, __builtin_bit_cast(bf16x8_t, pb[PAR ^ 1][k][kb]), o_acc[cb]);
            if (k == TERMS - 1) request(g + AHEAD);
            units(NKS + f * TERMS + k);
          }
        }
      }
      l_run += sum[0] + sum[1];
      // (all of this belongs in front of the branch below: the optimiser would sink it behind it)
      pin(s[PAR ^ 1]);
      pin(l_run);
#pragma unroll
      for (int k = 0; k < TERMS; ++k)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) pin(pb[PAR][k][kb]);
#pragma unroll
      for (int cb = 0; cb < NCB; ++cb) pin(o_acc[cb]);
      if (any_raise) {
#pragma unroll
        for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
          for (int i = 0; i < 16; ++i) o_acc[cb][i] *= alpha;
      }
      return odd_here != 0;
    };
    auto run_step = [&](auto parc, int st, const int32_t* pos, const char* v_here, const char* k_next,
                        const char* v_prev) __attribute__((always_inline)) {
      // (no product is pending: P times zeros)
      const bool odd = step(parc, st, pos, v_here, k_next, pending ? v_prev : smem + M::ZERO_OFF - M::V_OFF);
      if (__builtin_expect(odd, 0)) value_product(parc, IntC<1>{}, v_here);
      pending = !odd;
    };

    if (n_subs > 0) {
      constexpr int HALF = SUB * T::ROW;   // bytes from a tile's first sub-tile to its second
      char *prev = smem, *cur = smem + M::BYTES, *next = smem + 2 * M::BYTES;
      lds_barrier();   // the piece before has been read
      put(cur);
      if (pc.t0 + 1 < pc.t1) fetch(pc.t0 + 1);
      lds_barrier();
#pragma unroll
      for (int i = 0; i < 16; ++i) s[0][i] = 0.f;
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks)
        s[0] = mfma32(__builtin_bit_cast(bf16x8_t, k_frag(cur, ks)), __builtin_bit_cast(bf16x8_t, qf[ks]), s[0]);
      for (int t = pc.t0; t < pc.t1; ++t) {
        const int32_t* const pos = (const int32_t*)(cur + M::POS_OFF);
        run_step(IntC<0>{}, 2 * t, pos, cur, cur + HALF, prev + HALF);
        if (t + 1 < pc.t1) {
          put(next);
          if (t + 2 < pc.t1) fetch(t + 2);
        }
        lds_barrier();
        // (a second sub-tile that is not there holds copies of the last key, none of which counts)
        run_step(IntC<1>{}, 2 * t + 1, pos + SUB, cur + HALF, next, cur);
        char* const x = prev;
        prev = cur;
        cur = next;
        next = x;
      }
      if (pending) value_product(IntC<1>{}, IntC<0>{}, prev + HALF);
    }
    l_run += xor32(l_run);

    // ---- the span's result, or this share's part of it ----
    if (ok) {
      float inv = 1.f;
      TO* out = nullptr;
      float* part = nullptr;
      if (pc.whole) {
        const int64_t at = (int64_t)node * p.n_q_heads + head;
        inv = l_run > 0.f ? 1.f / l_run : l_run == 0.f ? 0.f : l_run;   // (a NaN stays one)
        out = (TO*)p.out + at * D;
        if (hf == 0) p.lse[at] = l_run == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(l_run)) * kLn2;
      } else {
        const int64_t at = (int64_t)pc.slot * MANY_ROWS + wave * 32 + rl;
        part = p.part_o + at * D;
        if (hf == 0) {
          p.part_ml[at * 2] = ref;
          p.part_ml[at * 2 + 1] = l_run;
        }
      }
#pragma unroll
      for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const floatx4_t x = {o_acc[cb][4 * a], o_acc[cb][4 * a + 1], o_acc[cb][4 * a + 2], o_acc[cb][4 * a + 3]};
          const int ch = cb * 32 + a * 8 + hf * 4;
          if (pc.whole) store4<TO>(out + ch, x * inv);
          else *(floatx4_t*)(part + ch) = x;
        }
    }
    u += pc.t1 - pc.t0;
  }
}

// Joins the parts of the spans that fell into several shares, a wavefront per row: lane l knows the
// maximum and sum of part l, and the rows of eight parts are in flight at a time.
template <int D, int RM, int SPT, typename TO>
__global__ __launch_bounds__(256) void tree_join_kernel(const TreeParams p) {
  constexpr int V = D / 64, U = 8;
  typedef float vec_t __attribute__((ext_vector_type(V)));
  const int lane = threadIdx.x & 63;
  const int64_t idx = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (idx >= p.total_q * p.n_q_heads) return;
  const int node = (uint32_t)idx / (uint32_t)p.n_q_heads;
  const int head = (int)idx - node * p.n_q_heads, kvh = (uint32_t)head / (uint32_t)p.group;
  TreeLine<RM, SPT> line(p);
  TreeSeq sq;
  int64_t before;
  if (line.find_node(node, &before, &sq) < 0) return;   // behind the last tree
  const int row = (node - sq.q0) * p.group + (head - kvh * p.group);
  const int span = row / RM;
  const int64_t a = kvh * line.head_tiles + before + (int64_t)span * sq.tiles;
  const int w0 = (int)div64((uint64_t)a, (uint32_t)line.share);
  const int n = (int)div64((uint64_t)(a + sq.tiles - 1), (uint32_t)line.share) - w0 + 1;
  if (n == 1) return;
  // (the first part begins the span)
  auto at = [&](int k) { return (int64_t)(2 * (w0 + k) + (k == 0 ? 1 : 0)) * RM + (row - span * RM); };
  float m = -INFINITY, l = 0.f;
  vec_t o = {};
  for (int k0 = 0; k0 < n; k0 += 64) {
    const int cnt = min(64, n - k0);
    float mw = -INFINITY, lw = 0.f;
    if (lane < cnt) {
      const float2 x = *(const float2*)(p.part_ml + at(k0 + lane) * 2);
      mw = x.x;
      lw = x.y;
    }
    vec_t x[U];
    auto rows = [&](int k) {
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = *(const vec_t*)(p.part_o + at(k0 + min(k + u, cnt - 1)) * D + lane * V);
    };
    rows(0);
    float top = mw;
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor(top, s, 64));
    const float mn = fmaxf(m, top);
    const float old = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
    // (a part that saw nothing has weight 0; one that saw a NaN alone has no maximum and that sum)
    const float f = lw == 0.f ? 0.f : mw == -INFINITY ? lw : __builtin_amdgcn_exp2f(mw - mn);
    float sum = lw * f;
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) sum += __shfl_xor(sum, s, 64);
    l = fmaf(l, old, sum);
    m = mn;
    o *= old;
    for (int k = 0; k < cnt; k += U) {
      if (k > 0) rows(k);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float fu = k + u < cnt ? __builtin_bit_cast(float, __builtin_amdgcn_readlane(
                                           __builtin_bit_cast(int, f), k + u)) : 0.f;
        if (k + u < cnt) o += x[u] * fu;
      }
    }
  }
  const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
  o *= inv;
#pragma unroll
  for (int i = 0; i < V; ++i) ((TO*)p.out)[idx * D + lane * V + i] = from_float<TO>(o[i]);
  if (lane == 0) p.lse[idx] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// ---------------------------------------------------------------------------
// Commit of the accepted paths: a workgroup per sequence lists the nodes that the accepted node's
// mask names and copies their rows behind what the cache holds. Pure data movement of a few rows,
// bound by its chain of latencies {accepted, used} -> mask -> rows.
// ---------------------------------------------------------------------------
struct AcceptParams {
  const uint4* k_new;
  const uint4* v_new;
  const int32_t* pos_new;
  const int32_t* cu_new;
  const uint64_t* mask;
  const int32_t* accepted;
  uint4* k;
  uint4* v;
  int32_t* kv_pos;
  const int32_t* cu_kv;
  int32_t* used;
  int32_t* dropped;
  int64_t total_new, slots;
  int32_t words, chunks;   // 16-byte chunks of a row
};
constexpr int ACCEPT_THREADS = 256;

__global__ __launch_bounds__(ACCEPT_THREADS) void tree_accept_kernel(const AcceptParams p) {
  __shared__ int16_t path[CP_TREE_MAX_WORDS * 64];
  __shared__ int count;
  const int b = blockIdx.x, tid = threadIdx.x;
  const int64_t q0 = clamp64(p.cu_new[b], 0, p.total_new);
  const int64_t n = clamp64(p.cu_new[b + 1], q0, p.total_new) - q0;
  const int64_t k0 = clamp64(p.cu_kv[b], 0, p.slots);
  const int64_t room = clamp64(p.cu_kv[b + 1], k0, p.slots) - k0;
  const int64_t used = clamp64(p.used[b], 0, room);
  const int acc = p.accepted[b];
  if (acc < 0 || acc >= n) return;   // uniform
  if (tid < 64) {   // a word a lane
    uint64_t m = tid < p.words ? p.mask[(q0 + acc) * p.words + tid] : 0;
    const int64_t left = n - tid * 64;
    if (left < 64) m &= left > 0 ? (1ull << left) - 1 : 0;
    const int c = __builtin_popcountll(m);
    int end = c;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(end, o, 64);
      if (tid >= o) end += y;
    }
    int at = end - c;
    for (; m != 0; m &= m - 1) path[at++] = (int16_t)(tid * 64 + __builtin_ctzll(m));
    if (tid == 63) count = end;
  }
  __syncthreads();
  const int taken = (int)min<int64_t>(count, room - used);
  for (int e = tid; e < taken * p.chunks; e += ACCEPT_THREADS) {
    const int i = e / p.chunks, c = e - i * p.chunks;
    const int64_t src = (q0 + path[i]) * p.chunks + c, dst = (k0 + used + i) * p.chunks + c;
    p.k[dst] = p.k_new[src];
    p.v[dst] = p.v_new[src];
  }
  for (int i = tid; i < taken; i += ACCEPT_THREADS) p.kv_pos[k0 + used + i] = p.pos_new[q0 + path[i]];
  if (tid == 0) {   // (every thread has read used[b] before the barrier above)
    if (taken > 0) p.used[b] = (int32_t)(used + taken);
    if (p.dropped != nullptr && count > taken) atomicAdd(p.dropped, count - taken);
  }
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
inline size_t round256(size_t x) { return (x + 255) & ~(size_t)255; }

enum TreeForm { kFew32, kFew64, kMany };
struct TreePlan {
  TreeForm form;
  int rm, spt, n_wg, log2_wg, min_share;
  size_t o_bytes, ml_bytes;
};
TreePlan tree_plan(const cp_shape& s) {
  TreePlan pl = {};
  const int64_t group = s.n_q_heads / s.n_kv_heads;
  const int64_t rows = s.total_q * group / s.batch;   // of a sequence, on average
  pl.form = s.dtype == CP_FP32 || rows <= 32 ? kFew32 : rows <= 128 ? kFew64 : kMany;
  pl.rm = pl.form == kFew32 ? 32 : pl.form == kFew64 ? 64 : MANY_ROWS;
  pl.spt = pl.form == kMany ? 2 : 4;
  pl.min_share = 1;
  // no more workgroups than there can be tiles
  const int64_t spans = s.total_q * group / pl.rm + s.batch;
  const int64_t tiles = (s.total_kv + s.total_q) / (SUB * pl.spt) + 2 * (int64_t)s.batch;
  const int64_t most = pl.form == kMany ? 256 : 512;
  const int64_t any = spans > most || tiles > most ? most : spans * tiles * s.n_kv_heads;
  while ((1 << pl.log2_wg) < any && (1 << pl.log2_wg) < most) ++pl.log2_wg;
  pl.n_wg = 1 << pl.log2_wg;
  pl.o_bytes = round256((size_t)2 * pl.n_wg * pl.rm * s.head_dim * 4);
  pl.ml_bytes = round256((size_t)2 * pl.n_wg * pl.rm * 2 * 4);
  return pl;
}

template <typename TI, int D, bool KS, int C, int NW, int TERMS, typename TO>
int launch_form(const TreeParams& p, hipStream_t st) {
  using F = Form<KS, C, NW>;
  constexpr int smem = tree_smem<TI, D, KS, C, NW>();
  static_assert(smem <= 160 * 1024, "LDS of a CU");
  auto kernel = tree_attn_kernel<TI, D, KS, C, NW, TERMS, TO>;
  if (hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, smem) !=
      hipSuccess)
    return CP_ERR_LAUNCH;
  hipLaunchKernelGGL(kernel, dim3(p.n_wg), dim3(NW * 64), smem, st, p);
  if (check_launch() != CP_OK) return CP_ERR_LAUNCH;
  const int64_t rows = p.total_q * p.n_q_heads;
  hipLaunchKernelGGL((tree_join_kernel<D, F::RM, F::SPT, TO>), dim3((unsigned)((rows + 3) / 4)),
                     dim3(256), 0, st, p);
  return check_launch();
}

template <int D, int TERMS, typename TO>
int launch_many(const TreeParams& p, hipStream_t st) {
  static_assert(ManyTile<D>::SMEM <= 160 * 1024, "LDS of a CU");
  auto kernel = tree_many_kernel<D, TERMS, TO>;
  if (hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize,
                          ManyTile<D>::SMEM) != hipSuccess)
    return CP_ERR_LAUNCH;
  hipLaunchKernelGGL(kernel, dim3(p.n_wg), dim3(MANY_WAVES * 64), ManyTile<D>::SMEM, st, p);
  if (check_launch() != CP_OK) return CP_ERR_LAUNCH;
  const int64_t rows = p.total_q * p.n_q_heads;
  hipLaunchKernelGGL((tree_join_kernel<D, MANY_ROWS, 2, TO>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, st,
                     p);
  return check_launch();
}

template <int D, int TERMS, typename TO>
int launch_bf16(const TreeParams& p, TreeForm form, hipStream_t st) {
  switch (form) {
    case kFew32: return launch_form<bf16_t, D, true, 1, 4, TERMS, TO>(p, st);
    case kFew64: return launch_form<bf16_t, D, true, 2, 4, TERMS, TO>(p, st);
    default: return launch_many<D, TERMS, TO>(p, st);
  }
}

}  // namespace

size_t tree_workspace_bytes(const cp_shape& s) {
  if (s.total_q == 0) return 0;
  const TreePlan pl = tree_plan(s);
  return pl.o_bytes + pl.ml_bytes;
}

}  // namespace cp

extern "C" {

int cp_tree_mask(int32_t batch, const int32_t* cu_seqlens, const int32_t* parents, int32_t mask_words,
                 uint64_t* mask_out) {
  if (cu_seqlens == nullptr) return CP_ERR_NULL;
  if (batch < 1 || mask_words < 1 || mask_words > CP_TREE_MAX_WORDS || cu_seqlens[0] != 0)
    return CP_ERR_SHAPE;
  for (int b = 0; b < batch; ++b) {
    const int64_t n = (int64_t)cu_seqlens[b + 1] - cu_seqlens[b];
    if (n < 0 || n > 64 * (int64_t)mask_words) return CP_ERR_SHAPE;
  }
  if (cu_seqlens[batch] > 0 && (parents == nullptr || mask_out == nullptr)) return CP_ERR_NULL;
  for (int b = 0; b < batch; ++b)
    for (int32_t i = 0; i < cu_seqlens[b + 1] - cu_seqlens[b]; ++i) {
      const int32_t parent = parents[cu_seqlens[b] + i];
      if (parent < -1 || parent >= i) return CP_ERR_SHAPE;
    }
  for (int b = 0; b < batch; ++b) {
    uint64_t* const tree = mask_out + (int64_t)cu_seqlens[b] * mask_words;
    for (int32_t i = 0; i < cu_seqlens[b + 1] - cu_seqlens[b]; ++i) {
      const int32_t parent = parents[cu_seqlens[b] + i];
      uint64_t* const m = tree + (int64_t)i * mask_words;
      for (int w = 0; w < mask_words; ++w)
        m[w] = parent < 0 ? 0 : tree[(int64_t)parent * mask_words + w];
      m[i / 64] |= 1ull << (i % 64);
    }
  }
  return CP_OK;
}

int cp_tree_attn(const cp_shape* shape, const void* q, const int32_t* q_pos,
                 const int32_t* cu_seqlens_q, const void* k_new, const void* v_new,
                 const uint64_t* tree_mask, int32_t mask_words, const void* k_cache,
                 const void* v_cache, const int32_t* kv_pos_cache, const int32_t* cu_seqlens_kv,
                 const int32_t* seq_used, void* out, float* lse, int32_t out_dtype, void* workspace,
                 size_t workspace_bytes, void* stream) {
  using namespace cp;
  const int rc = check_shape(shape);
  if (rc != CP_OK) return rc;
  const cp_shape& s = *shape;
  if (out_dtype != CP_BF16 && out_dtype != CP_FP32) return CP_ERR_UNSUPPORTED;
  if ((k_new == nullptr) != (v_new == nullptr)) return CP_ERR_NULL;
  if (k_new != nullptr && (mask_words < 1 || mask_words > CP_TREE_MAX_WORDS)) return CP_ERR_SHAPE;
  if (cu_seqlens_q == nullptr || cu_seqlens_kv == nullptr) return CP_ERR_NULL;
  if (s.total_q > 0 && (q == nullptr || q_pos == nullptr || out == nullptr || lse == nullptr))
    return CP_ERR_NULL;
  if (s.total_q > 0 && k_new != nullptr && tree_mask == nullptr) return CP_ERR_NULL;
  if (s.total_q > 0 && s.total_kv > 0 &&
      (k_cache == nullptr || v_cache == nullptr || kv_pos_cache == nullptr))
    return CP_ERR_NULL;
  if (!aligned16(q) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(k_cache) ||
      !aligned16(v_cache) || !aligned16(out))
    return CP_ERR_ALIGN;
  if (s.total_q == 0) return CP_OK;
  // rows of the merge's grid, nodes and tokens of a sequence with their sub-tiles are kept in 31 bits
  if (s.total_q * s.n_q_heads > INT32_MAX - 1024 || s.total_kv > INT32_MAX - 1024 || s.batch > (1 << 24))
    return CP_ERR_SHAPE;
  const TreePlan pl = tree_plan(s);
  if (workspace == nullptr || ((uintptr_t)workspace & 255u) != 0 ||
      workspace_bytes < pl.o_bytes + pl.ml_bytes)
    return CP_ERR_WORKSPACE;
  TreeParams p = {};
  p.q = q; p.q_pos = q_pos; p.cu_q = cu_seqlens_q;
  p.k_new = k_new; p.v_new = v_new; p.mask = tree_mask; p.words = mask_words;
  p.k = k_cache; p.v = v_cache; p.kv_pos = kv_pos_cache; p.cu_kv = cu_seqlens_kv; p.used = seq_used;
  p.out = out; p.lse = lse;
  p.part_o = (float*)workspace;
  p.part_ml = (float*)((char*)workspace + pl.o_bytes);
  p.total_q = s.total_q; p.total_kv = s.total_kv; p.batch = s.batch;
  p.n_q_heads = s.n_q_heads; p.n_kv_heads = s.n_kv_heads; p.group = s.n_q_heads / s.n_kv_heads;
  p.n_wg = pl.n_wg; p.log2_wg = pl.log2_wg; p.min_share = pl.min_share;
  p.scale_log2 = (s.softmax_scale > 0.f ? s.softmax_scale : 1.0f / sqrtf((float)s.head_dim)) * kLog2e;
  hipStream_t st = (hipStream_t)stream;
  const bool f32_out = out_dtype == CP_FP32;
  if (s.dtype == CP_FP32) {
    if (s.head_dim == 64)
      return f32_out ? launch_form<float, 64, true, 1, 4, 1, float>(p, st)
                     : launch_form<float, 64, true, 1, 4, 1, bf16_t>(p, st);
    return f32_out ? launch_form<float, 128, true, 1, 4, 1, float>(p, st)
                   : launch_form<float, 128, true, 1, 4, 1, bf16_t>(p, st);
  }
  if (s.head_dim == 64)
    return f32_out ? launch_bf16<64, 3, float>(p, pl.form, st) : launch_bf16<64, 1, bf16_t>(p, pl.form, st);
  return f32_out ? launch_bf16<128, 3, float>(p, pl.form, st) : launch_bf16<128, 1, bf16_t>(p, pl.form, st);
}

int cp_tree_accept(const cp_shape* shape, const void* k_new, const void* v_new,
                   const int32_t* pos_new, const int32_t* cu_seqlens_new, const uint64_t* tree_mask,
                   int32_t mask_words, const int32_t* accepted, void* k_cache, void* v_cache,
                   int32_t* kv_pos_cache, const int32_t* cu_seqlens_kv, int32_t* seq_used,
                   int32_t* dropped, void* stream) {
  using namespace cp;
  const int rc = check_cache_shape(shape);
  if (rc != CP_OK) return rc;
  const cp_shape& s = *shape;
  if (mask_words < 1 || mask_words > CP_TREE_MAX_WORDS) return CP_ERR_SHAPE;
  if (cu_seqlens_new == nullptr || cu_seqlens_kv == nullptr || seq_used == nullptr ||
      accepted == nullptr)
    return CP_ERR_NULL;
  if (s.total_q > 0 && (k_new == nullptr || v_new == nullptr || pos_new == nullptr ||
                        tree_mask == nullptr))
    return CP_ERR_NULL;
  if (s.total_q > 0 && s.total_kv > 0 &&
      (k_cache == nullptr || v_cache == nullptr || kv_pos_cache == nullptr))
    return CP_ERR_NULL;
  if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(k_cache) || !aligned16(v_cache))
    return CP_ERR_ALIGN;
  if (s.total_q == 0) return CP_OK;
  AcceptParams p;
  p.k_new = (const uint4*)k_new; p.v_new = (const uint4*)v_new;
  p.pos_new = pos_new; p.cu_new = cu_seqlens_new; p.mask = tree_mask; p.accepted = accepted;
  p.k = (uint4*)k_cache; p.v = (uint4*)v_cache; p.kv_pos = kv_pos_cache; p.cu_kv = cu_seqlens_kv;
  p.used = seq_used; p.dropped = dropped;
  p.total_new = s.total_q; p.slots = s.total_kv; p.words = mask_words;
  const int64_t chunks = (int64_t)s.n_kv_heads * s.head_dim * (s.dtype == CP_BF16 ? 2 : 4) / 16;
  // a path's chunks are counted in 31 bits
  if (chunks * CP_TREE_MAX_WORDS * 64 > INT32_MAX) return CP_ERR_SHAPE;
  p.chunks = (int32_t)chunks;
  hipLaunchKernelGGL(tree_accept_kernel, dim3((unsigned)s.batch), dim3(ACCEPT_THREADS), 0,
                     (hipStream_t)stream, p);
  return check_launch();
}

}  // extern "C"
