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
  float scale_log2;
};

// What a sequence holds. Boundaries that contradict each other or the totals (they are read on the
// device, where nothing can be refused) are cut to what is there.
struct TreeSeq {
  int32_t q0, n, k0, used;   // first node, nodes, first cache slot, tokens in the cache
  int32_t spans, tiles;      // row blocks of a KV head, tiles of each
  int32_t rm;                // rows of a row block: a multiple of 32, much the same for all of them
  int32_t parts;             // of each, where every workgroup takes one
  __device__ __forceinline__ TreeSeq of_lane(int l) const {
    TreeSeq r;
    r.q0 = __builtin_amdgcn_readlane(q0, l);
    r.n = __builtin_amdgcn_readlane(n, l);
    r.k0 = __builtin_amdgcn_readlane(k0, l);
    r.used = __builtin_amdgcn_readlane(used, l);
    r.spans = __builtin_amdgcn_readlane(spans, l);
    r.tiles = __builtin_amdgcn_readlane(tiles, l);
    r.rm = __builtin_amdgcn_readlane(rm, l);
    r.parts = __builtin_amdgcn_readlane(parts, l);
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
// It is cut into equal shares wherever they end, or, where there are few spans, so that no share
// has tiles of two: a span takes as many workgroups as it needs at `share` tiles each. A workgroup with a second
// piece (its Q, first tiles and result anew) is done as late as one with kPiece tiles more. us, anywhere and at spans'
// ends: 61 nodes of 16 heads over 131072 keys 98.9 and 88.7, 16 sequences of 2048 to 8192 keys 63.0 and 58.7, 64 of 500 to
// 4000 with 16 nodes 59.8 and 52.9, 8 of 900 to 6000 with head_dim 64 and 30 to 100 nodes 40.0 and 35.0 (with 64 nodes each
// 29.8 and 31.8), 32 of 1000 to 8000 with two nodes 28.2 and 25.3.
template <int RM, int SPT>
struct TreeLine {
  static constexpr int kPiece = SPT == 2 ? 8 : 4;
  const TreeParams& p;
  TreeSeq mine;
  int64_t end;        // units (tiles, or parts) of the sequences up to the lane's, of those held
  int held;           // first of the sequences held
  int64_t head_units; // of a KV head
  int64_t share;      // tiles
  bool single;        // a part each

  __device__ __forceinline__ void hold(int b0) {
    held = b0;
    const int b = min(b0 + (int)(threadIdx.x & 63), p.batch - 1);
    const int32_t a0 = p.cu_q[b], a1 = p.cu_q[b + 1], c0 = p.cu_kv[b], c1 = p.cu_kv[b + 1];
    const int32_t u = p.used != nullptr ? p.used[b] : INT32_MAX;
    mine.q0 = (int32_t)clamp64(a0, 0, p.total_q);
    mine.n = (int32_t)clamp64(a1, mine.q0, p.total_q) - mine.q0;
    mine.k0 = (int32_t)clamp64(c0, 0, p.total_kv);
    mine.used = (int32_t)clamp64(u, 0, clamp64(c1, mine.k0, p.total_kv) - mine.k0);
    const int rows = mine.n * p.group;               // (in 31 bits: the host checks)
    mine.spans = (rows + RM - 1) / RM;
    // (blocks of the same height: the longest share decides. us, full blocks and a rest against equal ones: 272 rows on
    // 8192 keys 26.0 and 24.2, on 8 times 4096 of 8 KV heads 100 and 84, 384 rows 105 and 98, 640 152 and 151)
    const uint32_t groups = (uint32_t)(rows + 31) / 32, spans = (uint32_t)max(mine.spans, 1);
    mine.rm = RM == 32 ? 32 : (int)((groups + spans - 1) / spans) * 32;
    if (b0 + (int)(threadIdx.x & 63) >= p.batch) mine.spans = 0;
    const int subs = mine.cached_subs() + (p.k_new != nullptr ? (mine.n + SUB - 1) / SUB : 0);
    mine.tiles = subs > 0 ? (subs + SPT - 1) / SPT : 1;   // (nothing to see: one tile, empty)
    mine.parts = 0;
    if (single) cut();
    else end = wave_scan64((int64_t)mine.spans * mine.tiles);
  }
  __device__ __forceinline__ void cut() {
    mine.parts = ((uint32_t)mine.tiles + (uint32_t)share - 1) / (uint32_t)share;
    end = wave_scan64((int64_t)mine.spans * mine.parts);
  }
  __device__ __forceinline__ explicit TreeLine(const TreeParams& params) : p(params) {
    single = false;
    head_units = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 64) {
      hold(b0);
      head_units += readlane64(end, 63);
    }
    const int64_t all = head_units * p.n_kv_heads;
    share = (all + p.n_wg - 1) >> p.log2_wg;
    if (share <= 1) return;   // (no share has two pieces)
    int64_t spans = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 64) {
      if (b0 != held) hold(b0);
      spans += readlane64(wave_scan64(mine.spans), 63);
    }
    spans *= p.n_kv_heads;
    if (2 * spans > p.n_wg) return;
    const int64_t one = div64((uint64_t)(all + p.n_wg - spans - 1), (uint32_t)(p.n_wg - spans));
    if (one > share + kPiece) return;
    single = true;            // (n_wg - spans + spans parts at most)
    share = one;
    head_units = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 64) {
      if (b0 != held) hold(b0);
      else cut();
      head_units += readlane64(end, 63);
    }
  }
  // The units of a workgroup.
  __device__ __forceinline__ void mine_to_do(int64_t* u, int64_t* u_end) const {
    const int64_t each = single ? 1 : share;
    *u = blockIdx.x * each;
    *u_end = min(head_units * p.n_kv_heads, *u + each);
  }
  __device__ __forceinline__ int64_t units(const TreeSeq& sq) const {
    return (int64_t)sq.spans * (single ? sq.parts : sq.tiles);
  }
  // The sequence of unit u of a KV head (-1: behind the last), and the unit where it begins.
  __device__ __forceinline__ int find(int64_t u, int64_t* begin, TreeSeq* sq) {
    int64_t base = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 64) {
      if (b0 != held) hold(b0);
      const uint64_t behind = __builtin_amdgcn_ballot_w64(base + end > u);
      if (behind != 0) {
        const int l = __builtin_ctzll(behind);
        *sq = mine.of_lane(l);
        *begin = base + readlane64(end, l) - units(*sq);
        return b0 + l;
      }
      base += readlane64(end, 63);
    }
    return -1;
  }
  // The sequence that node t belongs to (-1: behind the last tree), and the units before it.
  __device__ __forceinline__ int find_node(int t, int64_t* begin, TreeSeq* sq) {
    int64_t base = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 64) {
      if (b0 != held) hold(b0);
      const bool in = b0 + (int)(threadIdx.x & 63) < p.batch;
      const uint64_t hit = __builtin_amdgcn_ballot_w64(in && t >= mine.q0 && t < mine.q0 + mine.n);
      if (hit != 0) {
        const int l = __builtin_ctzll(hit);
        *sq = mine.of_lane(l);
        *begin = base + readlane64(end, l) - units(*sq);
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
  int units;
};
template <int RM, int SPT>
__device__ __forceinline__ bool tree_piece(TreeLine<RM, SPT>& line, int64_t u, int64_t u_end, TreePiece* x) {
  int64_t v = u, begin;
  x->kvh = 0;
  if (v >= line.head_units) {
    x->kvh = ((v | line.head_units) >> 32) == 0 ? (uint32_t)v / (uint32_t)line.head_units : (int)(v / line.head_units);
    v -= x->kvh * line.head_units;
  }
  if (line.find(v, &begin, &x->sq) < 0) return false;
  const int64_t in = v - begin;
  const int tiles = x->sq.tiles;
  if (line.single) {
    x->span = (int)div64((uint64_t)in, (uint32_t)x->sq.parts);
    const int part = (int)(in - (int64_t)x->span * x->sq.parts);
    const int each = ((uint32_t)tiles + (uint32_t)x->sq.parts - 1) / (uint32_t)x->sq.parts;
    x->t0 = part * each;   // (no part is empty: fewer tiles each make no fewer parts)
    x->t1 = min(tiles, x->t0 + each);
    x->slot = 2 * (int)blockIdx.x;
    x->units = 1;
  } else {
    x->span = (int)div64((uint64_t)in, (uint32_t)tiles);
    x->t0 = (int)(in - (int64_t)x->span * tiles);
    x->t1 = (int)min<int64_t>(tiles, x->t0 + (u_end - u));
    // a share has at most one part that ends a span and one that begins one
    x->slot = 2 * (int)blockIdx.x + (x->t0 == 0 ? 1 : 0);
    x->units = x->t1 - x->t0;
  }
  x->n_cached = x->sq.cached_subs();
  x->n_subs = x->n_cached + (line.p.k_new != nullptr ? (x->sq.n + SUB - 1) / SUB : 0);
  x->whole = x->t0 == 0 && x->t1 == tiles;
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

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  bf16x2_t t;
  t[0] = static_cast<bf16_t>(a);
  t[1] = static_cast<bf16_t>(b);
  return __builtin_bit_cast(uint32_t, t);
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
// bf16 pair: 1.0 where bit i (low half), bit i + 1 (high half) of `bits` is set.
__device__ __forceinline__ uint32_t ones_of(uint32_t bits, int i) {
  return ((bits >> i) & 1u ? 0x3f80u : 0) | ((bits >> (i + 1)) & 1u ? 0x3f800000u : 0);
}

// V that is not finite. A row that does not see it must not meet it (its weight is 0, and 0 times it is a NaN), and
// one that sees an infinity has it as its result, whatever the weight (which may have become 0, and whose second and third
// term may be negative: a NaN again). What the plain product leaves in such a row is the right infinity or a NaN, never
// a finite number or the wrong sign. So nothing looks for such values on the way; where a result holds a NaN, the piece is
// gone through a second time, with the values that are not finite set apart from the others in every sub-tile. (Where
// every piece needs that, 16 trees over 2048 to 8192 keys with an fp32 result take 360 us instead of 92, 8 over 900 to
// 6000 with head_dim 64 102 instead of 36; looking for such values in every masked sub-tile cost the others 1 to 7 us.)
// NaN if the blocks hold one (or maybe an infinity: then the second pass is in vain).
template <int N>
__device__ __forceinline__ float nan_of(const floatx16_t (&o)[N]) {
  float x = 0.f;
#pragma unroll
  for (int b = 0; b < N; ++b)
#pragma unroll
    for (int i = 0; i < 16; i += 2) x = fmaf(o[b][i], o[b][i + 1], x);
  return x;
}
// x * f of the second pass: an infinity that has been seen stays, however small the factor.
__device__ __forceinline__ float scaled(float x, float f) {
  return fabsf(x) == INFINITY ? x : x * f;
}
template <int J>
struct IntC {
  static constexpr int value = J;
};

// Few rows: the four wavefronts of a workgroup hold the same 32 rows and take turns at the sub-tiles (the keys
// are what there is to share out), each with a buffer of its own; a tile is a sub-tile for each of them.
constexpr int FEW_WAVES = 4, FEW_ROWS = 32;
template <typename TI, int D>
constexpr int few_smem() {
  const int tiles = FEW_WAVES * SubTile<TI, D>::BYTES;
  const int join = FEW_WAVES * FEW_ROWS * (D + 4 + 2) * 4;
  return tiles > join ? tiles : join;
}

// Bound by latencies: the chain {sequence boundaries} -> K, V, Q -> products -> join in LDS -> parts, and the
// second launch; 8 nodes of 16 heads over 430 keys take 8 us here and 4 in the join, 32 sequences of 4096 keys at
// 32 rows each 26.0 us (67 MB, 2.6 TB/s).
// TI: K, V and Q. TO: O. P goes into the second product as TERMS bf16 terms (bf16 inputs): one at head_dim 128
// where O is rounded to bf16 itself, three (24 bits) at head_dim 64, where cp_attn_partial keeps them too, and where O
// stays fp32.
template <typename TI, int D, int TERMS, typename TO>
__global__ __launch_bounds__(FEW_WAVES * 64, sizeof(TI) * D == 512 ? 1 : 2) void tree_few_kernel(const TreeParams p) {
  using T = SubTile<TI, D>;
  constexpr bool F32 = sizeof(TI) == 4;
  constexpr int NKS = T::ROW / 32, NCB = D / 32;
  extern __shared__ __align__(16) char smem[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rl = lane & 31, hf = lane >> 5;   // row (N side) or key / channel (M side), half
  TreeLine<FEW_ROWS, FEW_WAVES> line(p);
  int64_t u, u_end;
  line.mine_to_do(&u, &u_end);
  const int64_t tok_q = (int64_t)p.n_q_heads * D, tok_kv = (int64_t)p.n_kv_heads * D;

  while (u < u_end) {
    TreePiece pc;
    if (!tree_piece(line, u, u_end, &pc)) break;
    const TreeSeq& sq = pc.sq;
    const int kvh = pc.kvh, t0 = pc.t0, t1 = pc.t1, n_cached = pc.n_cached, n_subs = pc.n_subs;
    const int n_rows = sq.n * p.group;

    // Requests for sub-tile `st`: rows behind its last one repeat that one (and are masked by their index).
    char* const buf = smem + wave * T::BYTES;
    auto request = [&](int st) __attribute__((always_inline)) {
      const bool own = st >= n_cached;
      const int first = (own ? st - n_cached : st) * SUB;
      const int last = min(SUB, (own ? sq.n : sq.used) - first) - 1;
      const int64_t base = (int64_t)(own ? sq.q0 : sq.k0) + first;
      const TI *kt = (const TI*)p.k, *vt = (const TI*)p.v;
      if (own) {
        kt = (const TI*)p.k_new;
        vt = (const TI*)p.v_new;
      }
      kt += base * tok_kv + kvh * D;
      vt += base * tok_kv + kvh * D;
      constexpr int RPI = 64 / T::CH;          // rows of a request
#pragma unroll
      for (int i = 0; i < SUB / RPI; ++i) {
        const int r = i * RPI + lane / T::CH, slot = lane % T::CH;
        const int64_t off = min(r, last) * tok_kv;
        to_lds16((const uint4*)(kt + off) + (slot ^ T::k_perm(r)), buf + i * 1024);
        to_lds16((const uint4*)(vt + off) + (slot ^ T::v_perm(r)), buf + T::V_OFF + i * 1024);
      }
      if (!own)
        __builtin_amdgcn_global_load_lds((const CP_GLB_AS void*)(p.kv_pos + base + min(rl, last)),
                                         (CP_LDS_AS void*)(buf + T::POS_OFF), 4, 0, 0);
    };
    lds_barrier();   // what the piece before joined has been read
    if (t0 * FEW_WAVES + wave < n_subs) request(t0 * FEW_WAVES + wave);

    // ---- the wavefront's rows ----
    const int row = pc.span * FEW_ROWS + rl;   // within (sequence, KV head)
    const bool ok = row < n_rows;
    const int nd = ok ? (uint32_t)row / (uint32_t)p.group : 0;
    const int node = sq.q0 + nd;
    const int head = kvh * p.group + (ok ? row - nd * p.group : 0);
    const uint4* const q_src = (const uint4*)((const TI*)p.q + node * tok_q + head * D) + hf;
    uint4 qf[NKS];      // lane (rl, hf): 16-byte chunk 2 ks + hf of row rl
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {
      qf[ks] = make_uint4(0, 0, 0, 0);
      if (ok) qf[ks] = q_src[2 * ks];
    }
    const int32_t qp = ok ? p.q_pos[node] : INT32_MIN;
    int32_t q_min = ok ? qp : INT32_MAX, q_max = qp;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      q_min = min(q_min, __shfl_xor(q_min, o, 64));
      q_max = max(q_max, __shfl_xor(q_max, o, 64));
    }

    float m_run, l_run;
    floatx16_t o_acc[NCB];
    // f(i, whether the lane's row sees the key of score i) for sub-tile st of `cnt` keys; score i of lane
    // (rl, hf): key (i / 4) * 8 + hf * 4 + i % 4
    auto each_score = [&](int st, bool own, int cnt, auto f) __attribute__((always_inline)) {
      const uint32_t there = cnt == SUB ? ~0u : (1u << cnt) - 1;
      uint32_t see = there;
      if (own) {
        const int word = (st - n_cached) >> 1;
        see = 0;
        if (ok && word < p.words)
          see = (uint32_t)(p.mask[(int64_t)node * p.words + word] >> (((st - n_cached) & 1) * 32)) & there;
      }
      see >>= hf * 4;   // (bit a * 8 + i: score 4 a + i)
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const int4 x = *(const int4*)(buf + T::POS_OFF + (a * 8 + hf * 4) * 4);
        const int32_t kp[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
          f(4 * a + i, ((int)((see & (1u << (a * 8 + i))) != 0) & ((int)own | (int)(kp[i] <= qp))) != 0);
      }
    };
    // S, P and O of one sub-tile that lies in LDS at `buf`. AGAIN: of the second pass.
    auto compute = [&](auto againc, int st) __attribute__((always_inline)) {
      constexpr bool AGAIN = decltype(againc)::value != 0;
      const bool own = st >= n_cached;
      const int first = (own ? st - n_cached : st) * SUB;
      const int cnt = min(SUB, (own ? sq.n : sq.used) - first);
      bool masked = AGAIN || own || cnt < SUB;
      if (!own) {
        const int32_t kp = *(const int32_t*)(buf + T::POS_OFF + rl * 4);
        if (__builtin_amdgcn_ballot_w64(kp <= q_max) == 0) return;   // none of the rows sees any
        masked = masked || __builtin_amdgcn_ballot_w64(kp > q_min) != 0;
      }
      floatx16_t s;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) {
        const uint4 a = *(const uint4*)(buf + rl * T::ROW + (((2 * ks + hf) ^ T::k_perm(rl)) << 4));
        if constexpr (F32) {
          const floatx4_t af = __builtin_bit_cast(floatx4_t, a);
          const floatx4_t qv = __builtin_bit_cast(floatx4_t, qf[ks]);
#pragma unroll
          for (int x = 0; x < 4; ++x) s = mfma32(af[x], qv[x], s);
        } else {
          s = mfma32(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, qf[ks]), s);
        }
      }
      uint32_t seen_bits = 0;   // of the second pass: bit i, the row sees the key of score i
      if (masked)
        each_score(st, own, cnt, [&](int i, bool vis) {
          s[i] = vis ? s[i] : -INFINITY;
          if (AGAIN) seen_bits |= (uint32_t)vis << i;
        });
      u32x4_t pb[TERMS][2];   // P^T of keys 0..15 and 16..31, per term
      float e[16];
      float mx = s[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
      mx = fmaxf(mx, xor32(mx));
      const float m_new = fmaxf(m_run, mx * p.scale_log2);
      const float m_use = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_use);
      m_run = m_new;
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        e[i] = __builtin_amdgcn_exp2f(fmaf(s[i], p.scale_log2, -m_use));
        sum += e[i];
        if (!F32 && (i & 1) == 1)
#pragma unroll
          for (int t = 0; t < TERMS; ++t) {
            const uint32_t x = pack_bf16(e[i - 1], e[i]);
            pb[t][i >> 3][(i & 7) >> 1] = x;
            e[i - 1] -= __builtin_bit_cast(float, x << 16);   // what the term leaves over (exact)
            e[i] -= __builtin_bit_cast(float, x & 0xffff0000u);
          }
      }
      l_run = fmaf(l_run, alpha, sum);
      if (__builtin_amdgcn_ballot_w64(alpha != 1.f) != 0) {
#pragma unroll
        for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
          for (int i = 0; i < 16; ++i) o_acc[cb][i] = AGAIN ? scaled(o_acc[cb][i], alpha) : o_acc[cb][i] * alpha;
      }
      if constexpr (F32) {
        // O^T += V^T P^T, a key pair a step: k slot hf of step i is the key of score i
#pragma unroll
        for (int cb = 0; cb < NCB; ++cb) {
          floatx16_t plus, minus;   // how many visible infinities of either sign (a NaN: both)
#pragma unroll
          for (int i = 0; i < 16; ++i) plus[i] = minus[i] = 0.f;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int r = (i >> 2) * 8 + hf * 4 + (i & 3);
            float v = *(const float*)(buf + T::V_OFF + r * T::ROW + (cb * 32 + rl) * 4);
            if constexpr (AGAIN) {
              const bool fin = fabsf(v) < INFINITY;
              const float up = fin || v == -INFINITY ? 0.f : 1.f, dn = fin || v == INFINITY ? 0.f : 1.f;
              const float seen = (seen_bits >> i) & 1u ? 1.f : 0.f;
              plus = mfma32(up, seen, plus);
              minus = mfma32(dn, seen, minus);
              v = fin ? v : 0.f;
            }
            o_acc[cb] = mfma32(v, e[i], o_acc[cb]);
          }
          if constexpr (AGAIN) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
              o_acc[cb][i] += (plus[i] > 0.f ? INFINITY : 0.f) + (minus[i] > 0.f ? -INFINITY : 0.f);
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
          if constexpr (AGAIN) {
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
                  seen[x] = ones_of(seen_bits, kb * 8 + 2 * x);
                }
                sign[m] = mfma32(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, seen), sign[m]);
              }
            }
#pragma unroll
            for (int i = 0; i < 16; ++i)
              o_acc[cb][i] += (sign[0][i] > 0.f ? INFINITY : 0.f) + (sign[1][i] > 0.f ? -INFINITY : 0.f);
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
              for (int x = 0; x < 4; ++x) v[kb][x] = only_finite(v[kb][x]);
          }
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int t = 0; t < TERMS; ++t)
              o_acc[cb] = mfma32(__builtin_bit_cast(bf16x8_t, v[kb]), __builtin_bit_cast(bf16x8_t, pb[t][kb]),
                                 o_acc[cb]);
        }
      }
    };

    auto pass = [&](auto againc) __attribute__((always_inline)) {
      m_run = -INFINITY;
      l_run = 0.f;
#pragma unroll
      for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
        for (int i = 0; i < 16; ++i) o_acc[cb][i] = 0.f;
      for (int t = t0; t < t1; ++t) {   // (a wavefront waits for its own sub-tiles alone)
        const int st = t * FEW_WAVES + wave;
        if (st >= n_subs) break;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        compute(againc, st);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (t + 1 < t1 && st + FEW_WAVES < n_subs) request(st + FEW_WAVES);
      }
      l_run += xor32(l_run);
    };
    pass(IntC<0>{});
    const float x = nan_of<NCB>(o_acc);
    // (a row whose sum is a NaN is NaN in any case; without a sub-tile O is 0)
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(ok && l_run == l_run && x != x) != 0, 0)) {
      request(t0 * FEW_WAVES + wave);
      pass(IntC<1>{});
    }

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
        const int64_t at = (int64_t)pc.slot * FEW_ROWS + in_block;
        *(floatx4_t*)(p.part_o + at * D + ch) = o4;
        if (ch == 0) {
          p.part_ml[at * 2] = m;
          p.part_ml[at * 2 + 1] = l;
        }
      }
    };
    // the wavefronts' disjoint subsets of the keys are joined in LDS
    constexpr int OS = D + 4;                      // floats of a row
    constexpr int WS = FEW_ROWS * OS + 2 * FEW_ROWS;     // of a wavefront
    float* const cb0 = (float*)smem;
    lds_barrier();
    float* const mine = cb0 + wave * WS;
#pragma unroll
    for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
      for (int a = 0; a < 4; ++a)
        *(floatx4_t*)(mine + rl * OS + cb * 32 + a * 8 + hf * 4) =
            floatx4_t{o_acc[cb][4 * a], o_acc[cb][4 * a + 1], o_acc[cb][4 * a + 2], o_acc[cb][4 * a + 3]};
    if (hf == 0) {
      mine[FEW_ROWS * OS + rl] = m_run;
      mine[FEW_ROWS * OS + FEW_ROWS + rl] = l_run;
    }
    lds_barrier();
    constexpr int LPR = D / 4, RPI = FEW_WAVES * 64 / LPR;   // lanes of a row, rows at a time
#pragma unroll 4
    for (int i = 0; i < FEW_ROWS / RPI; ++i) {
      const int r = i * RPI + tid / LPR, ch = (tid % LPR) * 4;
      float m = -INFINITY, l = 0.f;
      floatx4_t o4 = {0.f, 0.f, 0.f, 0.f};
      float mw[FEW_WAVES], lw[FEW_WAVES], f[FEW_WAVES];
      floatx4_t x[FEW_WAVES];
#pragma unroll
      for (int w = 0; w < FEW_WAVES; ++w) {
        mw[w] = cb0[w * WS + FEW_ROWS * OS + r];
        lw[w] = cb0[w * WS + FEW_ROWS * OS + FEW_ROWS + r];
        x[w] = *(const floatx4_t*)(cb0 + w * WS + r * OS + ch);
        m = fmaxf(m, mw[w]);
      }
#pragma unroll
      for (int w = 0; w < FEW_WAVES; ++w) {
        f[w] = m == -INFINITY ? lw[w]   // (0, or a NaN)
                              : __builtin_amdgcn_exp2f(mw[w] - m);
        l = fmaf(lw[w], f[w], l);
        o4 += x[w] * f[w];
      }
      if (const float y = fmaf(o4[0], o4[1], o4[2] * o4[3]); __builtin_expect(y != y, 0))
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          o4[i] = 0.f;
#pragma unroll
          for (int w = 0; w < FEW_WAVES; ++w) o4[i] += scaled(x[w][i], f[w]);
        }
      write(pc.span * FEW_ROWS + r, r, m, l, ch, o4);
    }
    u += pc.units;
  }
}

// ---------------------------------------------------------------------------
// Many rows (bf16): eight wavefronts with 32 rows each, a tile of 64 keys for all of them.
//
// A step works on three sub-tiles: the products S^T of the next one and O^T of the one before are issued
// between the softmax arithmetic of the current one, which needs neither, and so is the maximum of the
// next one's scores. The reference that the exponentials are taken against is raised only when a
// score exceeds it by 8 in powers of two (O and the sum are rescaled then): it cancels in O / l, and what is
// rounded has the same relative error at any scale.
// A tile goes straight into one of four LDS buffers: the tile before (its values), the current one, the next
// and the one being filled; one barrier a tile. (When that was taken, against tiles through registers with fragments
// requested four products ahead where now eight fit: 97 and 104 us for 61 nodes of 16 heads over 131072 keys, 88 and 95
// for 16 sequences of 2048 to 8192 keys with three terms.)
// Measured: 61 nodes of 16 heads over 131072 keys of one, 83.5 us, 784 TFLOP/s, of which 69 us are the loop (the matrix
// pipe takes 2050 cycles of a tile's 3570), 12 the way to the first product and 4 the parts' way out. The matrix pipe is
// busy for 43 % of the kernel and vector instructions are issued for 47 %: the two wavefronts of a SIMD come out of
// a barrier together and mostly take turns at them, as do a wavefront's own (the prefill kernel's loop, whose LDS reads
// are ordered by hand with counted waits, has the matrix pipe at 58 %). Without its LDS reads the call takes 0.92 of the
// time, without the exponentials 0.98, without the loads 0.92; the wavefronts' priorities in turn change nothing.
// ---------------------------------------------------------------------------
constexpr int MANY_WAVES = 8;
constexpr int MANY_ROWS = 32 * MANY_WAVES;
constexpr float kSlack = 8.f;

// max over the two halves of a wavefront that share a row (inline assembly: through the builtin the
// compiler takes the two results of a swap of equal operands for equal; the s_nop covers the wait states
// that a lane swap needs after a vector write of its operands)
__device__ __forceinline__ float halves_max(float x) {
  float a = x, b = x;
  asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(b));
  return fmaxf(a, b);
}
// Requests from memory into LDS, 16 or 4 bytes a lane at `dst` (uniform) and on. In assembly: in front of
// every LDS read the compiler would wait for the requests that it knows of. landed_barrier() waits for them.
// (No vector register is written. m0 is the compiler's own: it holds nothing across statements, each use sets
// it. The s_nop 0 is the wait state between its write and its use. A base in scalar registers may have been written
// by the vector instruction in front of the statement, a v_readlane that brings a spilled one back: a memory instruction
// may read it 5 wait states later, which the compiler keeps for instructions of its own alone.)
__device__ __forceinline__ void dma16(const void* base, uint32_t lane_bytes, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %0, %1"
               :: "v"(lane_bytes), "s"(base), "s"(dst) : "memory");
}
__device__ __forceinline__ void dma16(const void* src, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
               :: "v"(src), "s"(dst) : "memory");
}
__device__ __forceinline__ void dma4(const void* src, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off"
               :: "v"(src), "s"(dst) : "memory");
}
// Every wavefront's requests have landed and its LDS reads have returned.
__device__ __forceinline__ void landed_barrier() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}
// Keeps the computation of x where it is in the instruction stream.
__device__ __forceinline__ void pin(float& x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ void pin(u32x4_t& x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ void pin(floatx16_t& x) { asm volatile("" : "+v"(x)); }

template <int D>
struct ManyTile {
  using T = SubTile<bf16_t, D>;
  static constexpr int KEYS = 2 * SUB;   // (one position a lane of a wavefront)
  static constexpr int V_OFF = KEYS * T::ROW;
  static constexpr int POS_OFF = 2 * KEYS * T::ROW;
  static constexpr int BYTES = POS_OFF + KEYS * 4;
  static constexpr int ZERO_OFF = 4 * BYTES;           // a sub-tile's worth of V, zeros
  static constexpr int AGAIN_OFF = ZERO_OFF + SUB * T::ROW;
  static constexpr int SMEM = AGAIN_OFF + 16;
};

template <int D, int TERMS, typename TO>
__global__ __launch_bounds__(MANY_WAVES * 64) void tree_many_kernel(const TreeParams p) {
  using M = ManyTile<D>;
  using T = SubTile<bf16_t, D>;
  constexpr int NKS = D / 16, NCB = D / 32, NVF = 2 * NCB;
  constexpr int THREADS = MANY_WAVES * 64;
  constexpr int RPT = THREADS / T::CH, REQ = M::KEYS / RPT;   // rows of a request of all wavefronts, requests
  static_assert(NKS == NVF, "a V^T fragment takes the registers of a K fragment");
  extern __shared__ __align__(16) char smem[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rl = lane & 31, hf = lane >> 5;
  for (int i = tid * 16; i < SUB * T::ROW; i += THREADS * 16)
    *(uint4*)(smem + M::ZERO_OFF + i) = make_uint4(0, 0, 0, 0);
  const int r0 = tid / T::CH, slot = tid % T::CH;   // of a request: row and 16-byte slot in LDS
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
        line.mine_to_do(&u, &u_end);
        if (u >= u_end) return;
      }
      if (!tree_piece(line, u, u_end, &pc)) return;
    }
    const TreeSeq& sq = pc.sq;
    const int kvh = pc.kvh, n_cached = pc.n_cached, n_subs = pc.n_subs;
    const int n_rows = sq.n * p.group;
    const int row = pc.span * sq.rm + wave * 32 + rl;
    const bool busy = wave * 32 < sq.rm && pc.span * sq.rm + wave * 32 < n_rows;
    const bool ok = busy && row < n_rows;
    const int nd = ok ? (uint32_t)row / (uint32_t)p.group : 0;
    const int node = sq.q0 + nd;
    const int head = kvh * p.group + (ok ? row - nd * p.group : 0);

    // ---- tiles on their way ----
    auto buf = [&](int t) { return smem + (t & 3) * M::BYTES; };
    const bf16_t* const kc = (const bf16_t*)p.k + sq.k0 * tok_kv + kvh * D;
    const bf16_t* const vc = (const bf16_t*)p.v + sq.k0 * tok_kv + kvh * D;
    // Requests of tile t into `buf`: the wavefront's K and V rows and, the first one, the positions. Keys
    // behind the last cached or tree's own one repeat it (and are masked by their index).
    const int k_l = (slot ^ T::k_perm(r0 & 31)) * 8, v_l = (slot ^ T::v_perm(r0 & 31)) * 8;
    // (32 bits hold a lane's offset inside a tile; of wider rows every address is computed)
    const bool narrow = tok_kv < (1 << 23);
    const uint32_t k_lane = ((uint32_t)r0 * (uint32_t)tok_kv + k_l) * 2;
    const uint32_t v_lane = ((uint32_t)r0 * (uint32_t)tok_kv + v_l) * 2;
    auto request_tile = [&](int t, const char* buf) __attribute__((always_inline)) {
      const uint32_t dst = (uint32_t)(size_t)(CP_LDS_AS const char*)buf;
      const uint32_t at = dst + wave * 1024;
      const int key0 = t * M::KEYS;
      if (narrow && key0 + M::KEYS <= sq.used) {   // cached keys alone
        const int64_t base = key0 * tok_kv;
#pragma unroll
        for (int i = 0; i < REQ; ++i) {
          dma16(kc + (base + i * RPT * tok_kv), k_lane, at + i * RPT * T::ROW);
          dma16(vc + (base + i * RPT * tok_kv), v_lane, at + i * RPT * T::ROW + M::V_OFF);
        }
      } else {
        const bf16_t* const kt = (const bf16_t*)p.k_new + sq.q0 * tok_kv + kvh * D;
        const bf16_t* const vt = (const bf16_t*)p.v_new + sq.q0 * tok_kv + kvh * D;
#pragma unroll
        for (int i = 0; i < REQ; ++i) {
          const int idx = key0 + i * RPT + r0;
          const bool own = p.k_new != nullptr && idx >= n_cached * SUB;
          const int key = own ? min(idx - n_cached * SUB, sq.n - 1) : min(idx, sq.used - 1);
          const int64_t off = key * tok_kv;
          // (a choice between values: one between the variables would put them into memory)
          dma16((own ? kt + off : kc + off) + k_l, at + i * RPT * T::ROW);
          dma16((own ? vt + off : vc + off) + v_l, at + i * RPT * T::ROW + M::V_OFF);
        }
      }
      if (wave == 0 && sq.used > 0)
        dma4(p.kv_pos + sq.k0 + min(key0 + lane, sq.used - 1), dst + M::POS_OFF);
    };
    int* const again = (int*)(smem + M::AGAIN_OFF);   // a wavefront wants the second pass
    if (n_subs > 0) {
      lds_barrier();   // the piece before has been read
      if (tid == 0) *again = 0;
      request_tile(pc.t0, buf(pc.t0));
      if (pc.t0 + 1 < pc.t1) request_tile(pc.t0 + 1, buf(pc.t0 + 1));
    }
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
    float top = -INFINITY;                 // the next sub-tile's largest score (log2 domain; if it needs no mask)
    bool masked = false;                   // the next sub-tile needs a mask
    floatx16_t o_acc[NCB], s[2];
    u32x4_t pb[2][TERMS][2];               // P of the current sub-tile and the one before, in bf16 pairs per
                                           // term (keys 0..15, 16..31)
#pragma unroll
    for (int k = 0; k < TERMS; ++k) pb[1][k][0] = pb[1][k][1] = u32x4_t{0, 0, 0, 0};
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
    // O^T of a sub-tile with nothing in between. AGAIN: of the second pass, what is not finite by the bits of the
    // scores whose keys the row sees.
    auto value_product = [&](auto parc, auto againc, const char* sub, uint32_t seen_bits) __attribute__((always_inline)) {
      constexpr int par = decltype(parc)::value;
#pragma unroll
      for (int cb = 0; cb < NCB; ++cb) {
        u32x4_t v[2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) v[kb] = __builtin_bit_cast(u32x4_t, v_frag(sub, cb * 2 + kb));
        if constexpr (decltype(againc)::value != 0) {
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
                  seen[x] = ones_of(seen_bits, kb * 8 + 2 * x);
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

    // K fragments 0 .. NKS-1 of the next sub-tile, then V^T fragments of the one before, then K fragments
    // of the sub-tile after the next: AHEAD of them are on their way
    constexpr int FRAGS = NKS + NVF, AHEAD = NKS;
    uint4 fr[AHEAD];

    // Sub-tile st has keys that some row does not see: the tree's own, keys behind the last, or a position
    // (this lane's `pos`, of key rl) behind a query's.
    auto needs_mask = [&](int st, int32_t pos) -> bool {   // (cached keys end before the tree's begin)
      return ((int)(__builtin_amdgcn_ballot_w64(pos > q_min) != 0) | (int)(st * SUB + SUB > sq.used)) != 0;
    };
    // Masks the scores s[PAR] of sub-tile st; bit i of the result: the row sees the key of score i.
    auto mask = [&](auto parc, int st, const int32_t* pos) __attribute__((always_inline)) -> uint32_t {
      constexpr int PAR = decltype(parc)::value;
      const bool own = st >= n_cached;
      const int cnt = own ? sq.n - (st - n_cached) * SUB : sq.used - st * SUB;   // keys, if not SUB
      const uint32_t there = st >= n_subs ? 0 : cnt >= SUB ? ~0u : (1u << cnt) - 1;
      uint32_t see = there;
      if (own) {
        const int word = (st - n_cached) >> 1;
        see = 0;
        if (ok && word < p.words && there != 0)
          see = (uint32_t)(p.mask[(int64_t)node * p.words + word] >> (((st - n_cached) & 1) * 32)) & there;
      }
      see >>= hf * 4;   // (bit a * 8 + i: score 4 a + i)
      uint32_t seen_bits = 0;
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const int4 x = *(const int4*)(pos + a * 8 + hf * 4);
        const int32_t kp[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int vis = (int)((see & (1u << (a * 8 + i))) != 0) & ((int)own | (int)(kp[i] <= qp));
          s[PAR][4 * a + i] = vis != 0 ? s[PAR][4 * a + i] : -INFINITY;
          seen_bits |= (uint32_t)vis << (4 * a + i);
        }
      }
      return seen_bits;
    };
    // largest score of the row in s[PAR], log2 domain
    auto row_max = [&](auto parc) __attribute__((always_inline)) {
      constexpr int PAR = decltype(parc)::value;
      float mx = fmaxf(fmaxf(s[PAR][0], s[PAR][1]), s[PAR][2]);
#pragma unroll
      for (int i = 3; i < 15; i += 2) mx = fmaxf(fmaxf(mx, s[PAR][i]), s[PAR][i + 1]);
      return halves_max(fmaxf(mx, s[PAR][15])) * p.scale_log2;
    };

    // One step: softmax of sub-tile st (scores s[PAR], its positions at `pos`), products S^T
    // of the next one (its K fragments on their way, the others at k_next) and O^T of the one before (V rows
    // at v_prev); the K fragments of the one after the next (k_after) are requested.
    auto step = [&](auto parc, int st, const int32_t* pos, const char* k_next,
                    const int32_t* pos_next, const char* k_after, const char* v_prev) __attribute__((always_inline)) {
      constexpr int PAR = decltype(parc)::value;
      auto request = [&](int g) __attribute__((always_inline)) {
        if (g < NKS) fr[g % AHEAD] = k_frag(k_next, g);
        else if (g < FRAGS) fr[g % AHEAD] = v_frag(v_prev, (g - NKS) % NCB * 2 + (g - NKS) / NCB);
        else fr[g % AHEAD] = k_frag(k_after, g - FRAGS);
      };
      if (__builtin_expect(masked, 0)) {
        mask(parc, st, pos);
        top = row_max(parc);
      }
      const bool raise = top > ref + kSlack;
      const bool any_raise = __builtin_amdgcn_ballot_w64(raise) != 0;
      float alpha = 1.f;
      if (__builtin_expect(any_raise, 0)) {
        if (raise) {
          alpha = __builtin_amdgcn_exp2f(ref - top);
          ref = top;
        }
        l_run *= alpha;
      }

      // Softmax arithmetic in units, two MFMA slots or so apart: argument of score w, exponential of the
      // one before, sum and rounding of the one before that.
      constexpr int UNITS = 18, SLOTS = NKS + NVF * TERMS, MAX_SLOTS = SLOTS - NKS - 2 >= 4 ? 4 : 2;
      const float use = ref == -INFINITY ? 0.f : ref;
      float e[16], sum[2] = {0.f, 0.f}, mx = -INFINITY;
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
      int32_t next_pos = 0;
      auto units = [&](int slot) __attribute__((always_inline)) {
        if (slot == 1) next_pos = pos_next[rl];
#pragma unroll
        for (int w = slot * UNITS / SLOTS; w < (slot + 1) * UNITS / SLOTS; ++w) unit(w);
        // the largest score of the next sub-tile, whose products are complete two slots after their last
        if (slot >= NKS + 2 && slot < NKS + 2 + MAX_SLOTS) {
          const int i0 = (slot - NKS - 2) * (16 / MAX_SLOTS);
#pragma unroll
          for (int i = i0; i < i0 + 16 / MAX_SLOTS; i += 2) mx = fmaxf(fmaxf(mx, s[PAR ^ 1][i]), s[PAR ^ 1][i + 1]);
        }
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
      // (all of this belongs in front of the branch below: the optimiser would sink it behind it)
      pin(s[PAR ^ 1]);
      l_run += sum[0] + sum[1];
      pin(l_run);
      top = halves_max(mx) * p.scale_log2;
#pragma unroll
      for (int k = 0; k < TERMS; ++k)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) pin(pb[PAR][k][kb]);
#pragma unroll
      for (int cb = 0; cb < NCB; ++cb) pin(o_acc[cb]);
      masked = needs_mask(st + 1, next_pos);
      if (__builtin_expect(any_raise, 0)) {
#pragma unroll
        for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
          for (int i = 0; i < 16; ++i) o_acc[cb][i] *= alpha;
      }
    };

    if (n_subs > 0) {
      constexpr int HALF = SUB * T::ROW;   // bytes from a tile's first sub-tile to its second
      auto pos_of = [](const char* b) { return (const int32_t*)(b + M::POS_OFF); };
      landed_barrier();
      if (pc.t0 + 2 < pc.t1) request_tile(pc.t0 + 2, buf(pc.t0 + 2));
      if (!busy) {
        // none of the block's rows: the wavefront brings its part of the tiles and leaves the units to the others (64 rows
        // of 32 sequences of 4096 keys 34.8 -> 29.4 us, 128 37.1 -> 31.5)
        for (int t = pc.t0; t < pc.t1; ++t) {
          landed_barrier();
          if (t + 3 < pc.t1) request_tile(t + 3, buf(t + 3));
        }
      } else {
        {
          const char* const b = buf(pc.t0);
#pragma unroll
          for (int i = 0; i < 16; ++i) s[0][i] = 0.f;
#pragma unroll
          for (int ks = 0; ks < NKS; ++ks)
            s[0] = mfma32(__builtin_bit_cast(bf16x8_t, k_frag(b, ks)), __builtin_bit_cast(bf16x8_t, qf[ks]), s[0]);
#pragma unroll
          for (int g = 0; g < AHEAD; ++g) fr[g] = k_frag(b + HALF, g);
          masked = needs_mask(2 * pc.t0, pos_of(b)[rl]);
          top = row_max(IntC<0>{});
        }
        const char* const zeros = smem + M::ZERO_OFF - M::V_OFF;   // (of the first step: P = 0 times zeros)
        for (int t = pc.t0; t < pc.t1; ++t) {
          const char* const b = buf(t);
          const char* const b_next = buf(t + 1);
          step(IntC<0>{}, 2 * t, pos_of(b), b + HALF, pos_of(b) + SUB, b_next,
               t > pc.t0 ? buf(t - 1) + HALF : zeros);
          // (the next tile but one has landed everywhere, and the values of the one before have been read)
          landed_barrier();
          if (t + 3 < pc.t1) request_tile(t + 3, buf(t + 3));
          // (a second sub-tile that is not there holds copies of the last key, none of which counts)
          step(IntC<1>{}, 2 * t + 1, pos_of(b) + SUB, b_next, pos_of(b_next), b_next + HALF, b);
        }
        value_product(IntC<1>{}, IntC<0>{}, buf(pc.t1 - 1) + HALF, 0);
      }
      l_run += xor32(l_run);
      // (a row whose sum is a NaN is NaN in any case)
      const float x = nan_of<NCB>(o_acc);
      if (__builtin_amdgcn_ballot_w64(ok && l_run == l_run && x != x) != 0 && lane == 0) *again = 1;
      lds_barrier();
      if (__builtin_expect(__builtin_amdgcn_readfirstlane(*again) != 0, 0)) {
        // The second pass, a tile after the other, by the arithmetic of the first.
        ref = -INFINITY;
        l_run = 0.f;
#pragma unroll
        for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
          for (int i = 0; i < 16; ++i) o_acc[cb][i] = 0.f;
        for (int st = 2 * pc.t0; st < min(2 * pc.t1, n_subs); ++st) {
          if ((st & 1) == 0) {
            lds_barrier();   // the tile before has been read
            request_tile(st >> 1, smem);
            landed_barrier();
          }
          if (!busy) continue;
          const char* const b = smem + (st & 1) * HALF;
#pragma unroll
          for (int i = 0; i < 16; ++i) s[0][i] = 0.f;
#pragma unroll
          for (int ks = 0; ks < NKS; ++ks)
            s[0] = mfma32(__builtin_bit_cast(bf16x8_t, k_frag(b, ks)), __builtin_bit_cast(bf16x8_t, qf[ks]), s[0]);
          const uint32_t seen_bits = mask(IntC<0>{}, st, pos_of(smem) + (st & 1) * SUB);
          top = row_max(IntC<0>{});
          float alpha = 1.f;
          if (top > ref + kSlack) {
            alpha = __builtin_amdgcn_exp2f(ref - top);
            ref = top;
          }
          l_run *= alpha;
#pragma unroll
          for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
            for (int i = 0; i < 16; ++i) o_acc[cb][i] = scaled(o_acc[cb][i], alpha);
          const float use = ref == -INFINITY ? 0.f : ref;
          float sum[2] = {0.f, 0.f};
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            float e0 = __builtin_amdgcn_exp2f(fmaf(s[0][i], p.scale_log2, -use));
            float e1 = __builtin_amdgcn_exp2f(fmaf(s[0][i + 1], p.scale_log2, -use));
            sum[0] += e0;
            sum[1] += e1;
#pragma unroll
            for (int k = 0; k < TERMS; ++k) {
              const uint32_t y = pack_bf16(e0, e1);
              pb[0][k][i >> 3][(i & 7) >> 1] = y;
              e0 -= __builtin_bit_cast(float, y << 16);
              e1 -= __builtin_bit_cast(float, y & 0xffff0000u);
            }
          }
          l_run += sum[0] + sum[1];
          value_product(IntC<0>{}, IntC<1>{}, b, seen_bits);
        }
        l_run += xor32(l_run);
      }
    }

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
    u += pc.units;
  }
}

// Joins the parts of the spans that fell into several shares, W wavefronts per row: lane l knows the
// maximum and sum of its wavefront's part l, and the rows of eight parts are in flight at a time. Bound by the
// parts' bytes where there are many rows (10 us for 33 MB); few rows (and so, many parts of each) take four
// wavefronts each: 9.1 us instead of 10.7 for 976 rows in 64 parts.
template <int D, int RM, int SPT, int W, typename TO>
__global__ __launch_bounds__(256) void tree_join_kernel(const TreeParams p) {
  constexpr int V = D / 64, U = 8, CHUNK = 64 / W;
  typedef float vec_t __attribute__((ext_vector_type(V)));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t idx = wide_block() * (4 / W) + wave / W;
  if (idx >= p.total_q * p.n_q_heads) return;
  const int node = (uint32_t)idx / (uint32_t)p.n_q_heads;
  const int head = (int)idx - node * p.n_q_heads, kvh = (uint32_t)head / (uint32_t)p.group;
  TreeLine<RM, SPT> line(p);
  TreeSeq sq;
  int64_t before;
  if (line.find_node(node, &before, &sq) < 0) return;   // behind the last tree
  const int row = (node - sq.q0) * p.group + (head - kvh * p.group);
  const int span = (uint32_t)row / (uint32_t)sq.rm;
  const int64_t a = kvh * line.head_units + before + (int64_t)span * (line.single ? sq.parts : sq.tiles);
  int w0 = (int)a, n = sq.parts;
  if (!line.single) {
    w0 = (int)div64((uint64_t)a, (uint32_t)line.share);
    n = (int)div64((uint64_t)(a + sq.tiles - 1), (uint32_t)line.share) - w0 + 1;
  }
  if (n == 1) return;
  // (in a line cut anywhere the first part begins the span)
  const int begins = line.single ? 0 : 1;
  auto at = [&](int k) __attribute__((always_inline)) {
    return (int64_t)(2 * (w0 + k) + (k == 0 ? begins : 0)) * RM + (row - span * sq.rm);
  };
  float m, l;
  vec_t o;
  auto pass = [&](auto againc) __attribute__((always_inline)) {
    auto by = [](vec_t v, float w) __attribute__((always_inline)) {
      if constexpr (decltype(againc)::value != 0) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = scaled(v[i], w);
        return v;
      } else {
        return v * w;
      }
    };
    m = -INFINITY;
    l = 0.f;
    o = vec_t{};
    for (int k0 = wave % W * CHUNK; k0 < n; k0 += 64) {
      const int cnt = min(CHUNK, n - k0);
      float mw = -INFINITY, lw = 0.f;
      if (lane < cnt) {
        const float2 x = *(const float2*)(p.part_ml + at(k0 + lane) * 2);
        mw = x.x;
        lw = x.y;
      }
      vec_t x[U];
      auto rows = [&](int k) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = *(const vec_t*)(p.part_o + at(k0 + min(k + u, cnt - 1)) * D + lane * V);
      };
      rows(0);
      float top = mw;
#pragma unroll
      for (int s = CHUNK / 2; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor(top, s, CHUNK));
      const float mn = fmaxf(m, __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, top))));
      const float old = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
      // (a part that saw nothing has weight 0; one that saw a NaN alone has no maximum and that sum)
      const float f = lw == 0.f ? 0.f : mw == -INFINITY ? lw : __builtin_amdgcn_exp2f(mw - mn);
      float sum = lw * f;
#pragma unroll
      for (int s = CHUNK / 2; s > 0; s >>= 1) sum += __shfl_xor(sum, s, CHUNK);
      l = fmaf(l, old, __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, sum))));
      m = mn;
      o = by(o, old);
      for (int k = 0; k < cnt; k += U) {
        if (k > 0) rows(k);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const float fu = k + u < cnt ? __builtin_bit_cast(float, __builtin_amdgcn_readlane(
                                             __builtin_bit_cast(int, f), k + u)) : 0.f;
          if (k + u < cnt) o += by(x[u], fu);
        }
      }
    }
  };
  pass(IntC<0>{});
  float y = o[0];
  if constexpr (V > 1) y *= o[1];
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(y != y && l == l) != 0, 0)) pass(IntC<1>{});
  if constexpr (W > 1) {   // (all of a workgroup's wavefronts have come this far: one row)
    __shared__ vec_t other[W][64];
    __shared__ float2 ml[W];
    other[wave][lane] = o;
    if (lane == 0) ml[wave] = make_float2(m, l);
    __syncthreads();
    if (wave > 0) return;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < W; ++w) top = fmaxf(top, ml[w].x);
    l = 0.f;
    o = vec_t{};
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = ml[w].y == 0.f ? 0.f : ml[w].x == -INFINITY ? ml[w].y : __builtin_amdgcn_exp2f(ml[w].x - top);
      l = fmaf(ml[w].y, f, l);
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] += scaled(other[w][lane][i], f);
    }
    m = top;
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

constexpr int64_t kFewBlocks = 1 << 26, kFewOneBlock = 1 << 27, kFewTiles = 768;
struct TreePlan {
  bool many;
  int rm, spt, n_wg, log2_wg;
  size_t o_bytes, ml_bytes;
};
TreePlan tree_plan(const cp_shape& s) {
  TreePlan pl = {};
  const int64_t group = s.n_q_heads / s.n_kv_heads;
  // 32-row blocks (of a sequence on average) times sub-tiles of all, weighed by head_dim: the form for many rows reads a
  // key once for 256 rows and has three times the matrix rate, the other starts and ends sooner, and one block of it
  // is all the work there is up to 32 rows. us (few rows, many; * the one that the rule takes, where it is the slower):
  // head_dim 128, 16 heads on one: 8 sequences of 4096 keys, 32 rows 17.5 and 18.4, 128 26.5 and 25.3, 256 36.5 and
  // 30.8; 1 of 8192 keys, 256 rows 18.2 and 27.7, 640 24.1 and 29.0*; 1 of 16384, 256 rows 23.5 and 30.7*, 640 28.9
  // and 30.9*; 32 sequences of 16 rows 24.4 and 25.4, of 64 36.2 and 29.8; 32 heads on 8, 8 sequences of 32 rows 42.0
  // and 49.1*, 32 of 32 125 and 118, of 64 175 and 122. Head_dim 64, 8 heads on two: 8 sequences of 128 rows 25.7 and
  // 26.8, of 256 36.1 and 32.7; 32 sequences of 32 rows 25.4 and 41.1, of 64 35.0 and 40.4*, of 128 56.8 and 44.9.
  // (total_kv are the slots that there are, used or not, and the rows of a sequence are the batch's average.)
  const int64_t blocks = (s.total_q * group / s.batch + 31) / 32;
  const int64_t subs = ((s.total_kv + s.total_q) / SUB + s.batch) * s.n_kv_heads;
  const int64_t limit = (blocks > 1 ? kFewBlocks : kFewOneBlock) / (s.head_dim * s.head_dim);
  pl.many = s.dtype == CP_BF16 && blocks > 0 && subs > limit / blocks;
  pl.rm = pl.many ? MANY_ROWS : FEW_ROWS;
  pl.spt = pl.many ? 2 : FEW_WAVES;
  // no more workgroups than there can be tiles
  const int64_t spans = s.total_q * group / pl.rm + s.batch;
  const int64_t tiles = (s.total_kv + s.total_q) / (SUB * pl.spt) + 2 * (int64_t)s.batch;
  // (two workgroups of the form for few rows share a CU, which pays from a few tiles each. us for 256 and 512: 1 sequence
  // of 8192 keys, 256 rows 18.2 and 20.2, 640 rows 24.2 and 23.7; 8 of 1024, 128 rows 17.7 and 18.9, 8 of 4096, 256
  // rows 39.2 and 36.5; 32 heads on 8, 2048 keys, 64 rows 17.5 and 18.0)
  const int64_t most = pl.many || blocks * subs / FEW_WAVES <= kFewTiles ? 256 : 512;
  const int64_t any = spans > most || tiles > most ? most : spans * tiles * s.n_kv_heads;
  while ((1 << pl.log2_wg) < any && (1 << pl.log2_wg) < most) ++pl.log2_wg;
  pl.n_wg = 1 << pl.log2_wg;
  pl.o_bytes = round256((size_t)2 * pl.n_wg * pl.rm * s.head_dim * 4);
  pl.ml_bytes = round256((size_t)2 * pl.n_wg * pl.rm * 2 * 4);
  return pl;
}

constexpr int64_t kJoinRows = 2048;   // (four wavefronts a row fill the card's 8192 places)
template <int D, int RM, int SPT, typename TO>
int launch_join(const TreeParams& p, hipStream_t st) {
  const int64_t rows = p.total_q * p.n_q_heads;
  if (rows <= kJoinRows)
    hipLaunchKernelGGL((tree_join_kernel<D, RM, SPT, 4, TO>), wide_grid(rows), dim3(256), 0, st, p);
  else
    hipLaunchKernelGGL((tree_join_kernel<D, RM, SPT, 1, TO>), wide_grid((rows + 3) / 4), dim3(256), 0, st, p);
  return check_launch();
}

template <typename TI, int D, int TERMS, typename TO>
int launch_few(const TreeParams& p, hipStream_t st) {
  constexpr int smem = few_smem<TI, D>();
  static_assert(smem <= 160 * 1024, "LDS of a CU");
  auto kernel = tree_few_kernel<TI, D, TERMS, TO>;
  if (hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, smem) !=
      hipSuccess)
    return CP_ERR_LAUNCH;
  hipLaunchKernelGGL(kernel, dim3(p.n_wg), dim3(FEW_WAVES * 64), smem, st, p);
  if (check_launch() != CP_OK) return CP_ERR_LAUNCH;
  return launch_join<D, FEW_ROWS, FEW_WAVES, TO>(p, st);
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
  return launch_join<D, MANY_ROWS, 2, TO>(p, st);
}

template <int D, int TERMS, typename TO>
int launch_bf16(const TreeParams& p, bool many, hipStream_t st) {
  return many ? launch_many<D, TERMS, TO>(p, st) : launch_few<bf16_t, D, TERMS, TO>(p, st);
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
  if (s.batch > kMaxWalkedBatch) return CP_ERR_SHAPE;
  if (s.total_q == 0) return CP_OK;
  // rows, a token's channels, and a sequence's tokens and nodes in one line are counted in 31 bits
  if (s.total_q * s.n_q_heads > INT32_MAX - 1024 || s.total_kv + s.total_q > INT32_MAX - 1024 ||
      (int64_t)s.n_q_heads * s.head_dim > INT32_MAX)
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
  p.n_wg = pl.n_wg; p.log2_wg = pl.log2_wg;
  p.scale_log2 = (s.softmax_scale > 0.f ? s.softmax_scale : 1.0f / sqrtf((float)s.head_dim)) * kLog2e;
  hipStream_t st = (hipStream_t)stream;
  const bool f32_out = out_dtype == CP_FP32;
  if (s.dtype == CP_FP32) {
    if (s.head_dim == 64)
      return f32_out ? launch_few<float, 64, 1, float>(p, st)
                     : launch_few<float, 64, 1, bf16_t>(p, st);
    return f32_out ? launch_few<float, 128, 1, float>(p, st)
                   : launch_few<float, 128, 1, bf16_t>(p, st);
  }
  if (s.head_dim == 64)
    return f32_out ? launch_bf16<64, 3, float>(p, pl.many, st) : launch_bf16<64, 3, bf16_t>(p, pl.many, st);
  return f32_out ? launch_bf16<128, 3, float>(p, pl.many, st) : launch_bf16<128, 1, bf16_t>(p, pl.many, st);
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
  // the grid's threads
  if (s.batch > INT32_MAX / ACCEPT_THREADS) return CP_ERR_SHAPE;
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
