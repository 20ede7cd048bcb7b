// Eviction from the persistent KV cache by accumulated attention weight.
//
// Of the n tokens that sequence b holds, keep = min(n, room of the destination, max(budget_b, number
// of protected ones)) stay: the protected first, then by weight, ties to the lowest slot. Kept slots
// in front of `keep` stay where they are, and the i-th kept slot behind it moves to the i-th hole in
// front of it, so in place only as many rows move as there are holes (sources lie behind `keep`,
// destinations in front of it: no row is read after it was written). The order of the slots means
// nothing to attention, which goes by their positions.
//
// The weight of the last slot that stays is found by a radix selection over order-preserving 32-bit
// keys (three digits of 11, 11 and 10 bits); then ties, holes and movers are ranked by prefix sums
// over 64-slot ballots. Sequences that one workgroup reads quickly are one launch, a workgroup
// each, with the keys in LDS; longer ones are cut into chunks and take a launch per digit. The last
// launch moves the rows and does the bookkeeping.
#include "cp_scan.h"

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
  // workspace, [slots] each, at the sequence's first slot
  int32_t* to;      // in place: destination slot of move t; else, per slot that is filled, its source
                    // slot, or -1 - t where move t fills it
  int32_t* from;    // source slot of move t
  int32_t* count;   // [batch][2]: slots that stay, moves
  // of sequences in chunks
  int32_t* hist;    // [batch][HIST]
  int32_t* chunk;   // [chunk][4]: slots above the bar, at it; the same in front of `keep`
};

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
// Slots of a chunk. More chunks are read in fewer rounds but add more counts up: us for 8192, 4096 and 2048, 4 sequences of
// 32768 slots 42, 34, 30, 16 of 65536 47, 39, 44, 64 of 32768 60, 64, 78.
constexpr int CHUNK = 4096;
constexpr int64_t kMaxSlots = INT32_MAX - 64 * CHUNK;   // slots, and the ends of steps over them, are counted in 31 bits
constexpr int HIST = 3 * BINS + 64;       // three digits' counts, and the number of protected slots

// Order-preserving key of a weight; protected slots are above all, NaN below all.
__device__ __forceinline__ uint32_t key_of(float w, bool safe) {
  if (safe) return 0xffffffffu;
  if (w != w) return 0;
  const uint32_t x = __builtin_bit_cast(uint32_t, w + 0.f);   // (-0 counts as 0)
  return (x & 0x80000000u) ? ~x : x | 0x80000000u;
}

// Prefix sum over the workgroup of x (exclusive), and the total.
__device__ __forceinline__ int block_scan(int x, int* wave_sums, int* total) {
  static_assert(SEL_WAVES == 16, "the wavefronts' sums are one row of lanes");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int end = wave_scan(x);
  __syncthreads();
  if (lane == 63) wave_sums[wave] = end;
  __syncthreads();
  const int sums = row_scan(wave_sums[lane & 15]);
  *total = __builtin_amdgcn_readlane(sums, 15);
  return (wave > 0 ? __builtin_amdgcn_readlane(sums, wave - 1) : 0) + end - x;
}

// What a sequence keeps, and its slots' keys.
struct EvictSeq {
  Range src, dst;
  int32_t n, from_pos, budget;
  __device__ __forceinline__ EvictSeq() {}
  __device__ __forceinline__ EvictSeq(const EvictParams& p, int b) {
    src = range_of(p.cu, b, p.slots);
    dst = range_of(p.cu_to, b, p.slots_to);
    n = (int)clamp64(p.used[b], 0, src.room);
    from_pos = p.protect_from != nullptr ? p.protect_from[b] : CP_POS_PAD_KV;
    budget = p.budget[b];
  }
  __device__ __forceinline__ EvictSeq of_lane(int l) const {
    // (slots are counted in 31 bits; in scalar registers from here on)
    EvictSeq r;
    r.src.first = __builtin_amdgcn_readlane((int)src.first, l);
    r.src.room = __builtin_amdgcn_readlane((int)src.room, l);
    r.dst.first = __builtin_amdgcn_readlane((int)dst.first, l);
    r.dst.room = __builtin_amdgcn_readlane((int)dst.room, l);
    r.n = __builtin_amdgcn_readlane(n, l);
    r.from_pos = __builtin_amdgcn_readlane(from_pos, l);
    r.budget = __builtin_amdgcn_readlane(budget, l);
    return r;
  }
  __device__ __forceinline__ uint32_t key(const EvictParams& p, int32_t at, float w) const {
    // (a padded token can be seen by no query: nothing protects it)
    return key_of(w, at != CP_POS_PAD_KV && (at < p.sinks || at >= from_pos));
  }
  __device__ __forceinline__ uint32_t key(const EvictParams& p, int i) const {
    return key(p, p.kv_pos[src.first + i], p.weight[src.first + i]);
  }
  __device__ __forceinline__ int keep(int protected_n) const {
    const int64_t want = budget < protected_n ? protected_n : budget;
    return (int)clamp64(want, 0, n < dst.room ? n : dst.room);
  }
};
// The keys of the K slots i, i + step, ... that lie in front of `end`, all requested at once.
template <int K>
__device__ __forceinline__ void load_keys(const EvictParams& p, const EvictSeq& sq, int i, int step, int end,
                                          uint32_t (&x)[K]) {
  int32_t at[K];
  float w[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int j = i + k * step;
    at[k] = CP_POS_PAD_KV;
    w[k] = 0.f;
    if (j < end) {
      at[k] = p.kv_pos[sq.src.first + j];
      w[k] = p.weight[sq.src.first + j];
    }
  }
#pragma unroll
  for (int k = 0; k < K; ++k) x[k] = sq.key(p, at[k], w[k]);
}

// The digit at which `left` slots, counted from the largest, are reached: c1 and c0 are the counts of
// this thread's bins BINS-1-2t and BINS-2-2t. What lies above it is taken off `left`. (Uniform; two words of
// LDS, free again after the next barrier.)
__device__ __forceinline__ int find_digit(int c1, int c0, int& left, int* wave_sums, int* found) {
  int all;
  const int above = block_scan(c0 + c1, wave_sums, &all);
  const int hi = BINS - 1 - 2 * (int)threadIdx.x;
  if (above < left && left <= above + c1) {
    found[0] = hi;
    found[1] = above;
  } else if (above + c1 < left && left <= above + c1 + c0) {
    found[0] = hi - 1;
    found[1] = above + c1;
  }
  __syncthreads();
  left -= __builtin_amdgcn_readfirstlane(found[1]);
  return __builtin_amdgcn_readfirstlane(found[0]);
}
__device__ constexpr int digit_shift(int d) { return d == 0 ? 21 : d == 1 ? 10 : 0; }
__device__ constexpr uint32_t digit_mask(int d) { return d == 2 ? 1023u : 2047u; }

// Of the slots of a sequence in front of some slot: ties with the bar, holes, movers.
struct Ranks {
  int ties, holes, movers;
};
// The lanes in front of `end` of 64 slots from g on.
__device__ __forceinline__ uint64_t lanes_before(int g, int end) {
  const int left = end - g;
  return left <= 0 ? 0 : left >= 64 ? ~0ull : (1ull << left) - 1;
}
__device__ __forceinline__ int rank_in(uint64_t mask) {   // set lanes in front of this one
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}
// The slots [g, g + 64) in front of `end`, this lane's of key x: moves are listed, and in place the
// bookkeeping of what goes is cleared. (Keys are read by the wavefront that lists them.) Which slots
// stay is a matter of lane masks, in scalar registers; lanes are asked only where there is a move.
__device__ __forceinline__ void list_moves(const EvictParams& p, const EvictSeq& sq, int g0, int end, uint32_t x,
                                           int keep, uint32_t bar, int ties, Ranks& r) {
  const int g = __builtin_amdgcn_readfirstlane(g0), i = g + (int)(threadIdx.x & 63);
  const uint64_t in = lanes_before(g, end), front = lanes_before(g, keep) & in;
  uint64_t stays = in;
  if (keep < sq.n) {
    const uint64_t up = __builtin_amdgcn_ballot_w64(x > bar) & in, at = __builtin_amdgcn_ballot_w64(x == bar) & in;
    const int left = ties - r.ties, tied = __builtin_popcountll(at);
    uint64_t kept = at;
    if (left <= 0) kept = 0;
    else if (left < tied) kept = __builtin_amdgcn_ballot_w64(rank_in(at) < left) & at;
    stays = keep > 0 ? up | kept : 0;
    r.ties += tied;
  }
  const uint64_t holes = front & ~stays, movers = stays & ~front, gone = in & ~front & ~stays;
  auto mine = [&](uint64_t m) { return ((m >> (threadIdx.x & 63)) & 1) != 0; };
  if (!p.in_place && front != 0) {
    if (mine(front)) p.to[sq.src.first + i] = mine(holes) ? -1 - (r.holes + rank_in(holes)) : i;
  } else if (holes != 0) {
    if (mine(holes)) p.to[sq.src.first + r.holes + rank_in(holes)] = i;
  }
  if (movers != 0 && mine(movers)) p.from[sq.src.first + r.movers + rank_in(movers)] = i;
  if (p.in_place && gone != 0 && mine(gone)) {
    p.kv_pos[sq.src.first + i] = CP_POS_PAD_KV;
    p.weight[sq.src.first + i] = 0.f;
  }
  r.holes += __builtin_popcountll(holes);
  r.movers += __builtin_popcountll(movers);
}

// Slots above the bar and at it among [g, g + 64) in front of `end`, all and those in front of `keep`.
__device__ __forceinline__ void count_slots(int g0, int end, uint32_t x, int keep, uint32_t bar, int (&c)[4]) {
  const int g = __builtin_amdgcn_readfirstlane(g0);
  const uint64_t in = lanes_before(g, end), front = lanes_before(g, keep);
  const uint64_t up = keep > 0 ? __builtin_amdgcn_ballot_w64(x > bar) & in : 0;
  const uint64_t at = __builtin_amdgcn_ballot_w64(x == bar) & in;
  c[0] += __builtin_popcountll(up);
  c[1] += __builtin_popcountll(at);
  c[2] += __builtin_popcountll(up & front);
  c[3] += __builtin_popcountll(at & front);
}

// Parts of a sequence, one a lane in their order, by their counts y: added to `r` what the parts before
// part `a` hold, and to `e` what those before part `z` do. The first part begins behind the r.ties
// (e.ties) ties that there are so far.
__device__ __forceinline__ void add_parts(bool in, int4 y, int first, int last, int keep, int ties, int a,
                                          Ranks& r, int z, Ranks& e) {
  const int tied = wave_scan(y.y);
  const int left = max(0, ties - (r.ties + tied - y.y));
  const int front = y.z + min(left, y.w);
  const int holes = wave_scan(in ? min(keep, last) - min(keep, first) - front : 0);
  const int movers = wave_scan(in ? y.x + min(left, y.y) - front : 0);
  auto add = [&](int k, Ranks& to) {   // k uniform
    if (k == 0) return;
    to.ties += __builtin_amdgcn_readlane(tied, k - 1);
    to.holes += __builtin_amdgcn_readlane(holes, k - 1);
    to.movers += __builtin_amdgcn_readlane(movers, k - 1);
  };
  const Ranks base = r;
  add(a, r);
  if (&e != &r) {
    e = base;
    add(z, e);
  }
}

// A workgroup per sequence. The keys of the first `cached` slots are kept in LDS.
__global__ __launch_bounds__(SEL_THREADS) void evict_select_kernel(const EvictParams p, int cached) {
  extern __shared__ __align__(16) uint32_t keys[];
  __shared__ int hist[BINS];
  __shared__ int wave_sums[SEL_WAVES];
  __shared__ int found[2];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const EvictSeq sq(p, b);
  for (int i = tid; i < BINS; i += SEL_THREADS) hist[i] = 0;
  __syncthreads();
  int protected_n = 0;
  constexpr int AT_ONCE = 8;   // keys of a lane in flight
  for (int i0 = tid; i0 < sq.n; i0 += AT_ONCE * SEL_THREADS) {
    uint32_t x[AT_ONCE];
    load_keys(p, sq, i0, SEL_THREADS, sq.n, x);
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      const int i = i0 + k * SEL_THREADS;
      if (i >= sq.n) break;
      if (i < cached) keys[i] = x[k];
      protected_n += x[k] == 0xffffffffu;
      atomicAdd(&hist[x[k] >> digit_shift(0)], 1);
    }
  }
  int all;
  block_scan(protected_n, wave_sums, &all);   // (and the counts are complete)
  const int keep = sq.keep(all);
  // f(i, key of slot i) for the slots i, i + step, ... in front of `end` (behind it with a key of 0, up
  // to AT_ONCE steps), the keys of AT_ONCE slots requested together
  auto each_key = [&](int i0, int step, int end, auto f) {
    for (int i = i0; __builtin_amdgcn_ballot_w64(i < end) != 0; i += AT_ONCE * step) {
      uint32_t x[AT_ONCE];
      if (sq.n <= cached) {
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) x[k] = keys[min(i + k * step, sq.n - 1)];
      } else {
        load_keys(p, sq, i, step, end, x);
      }
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) f(i + k * step, x[k]);
    }
  };

  // the key of the last slot that stays, and how many slots with that key do
  uint32_t bar = 0;
  int ties = keep;
  if (keep > 0 && keep < sq.n) {
#pragma unroll
    for (int d = 0; d < 3; ++d) {
      if (d > 0) {
        __syncthreads();
        for (int i = tid; i < BINS; i += SEL_THREADS) hist[i] = 0;
        __syncthreads();
        const int above = digit_shift(d - 1);
        each_key(tid, SEL_THREADS, sq.n, [&](int i, uint32_t x) {
          if (i < sq.n && ((x ^ bar) >> above) == 0)
            atomicAdd(&hist[(x >> digit_shift(d)) & digit_mask(d)], 1);
        });
        __syncthreads();
      }
      const int hi = BINS - 1 - 2 * tid;
      bar |= (uint32_t)find_digit(hist[hi], hist[hi - 1], ties, wave_sums, found) << digit_shift(d);
    }
  }
  if (keep < sq.n) {
    // a contiguous part per wavefront: first how many of its slots lie above and at the bar, ...
    const int part = ((sq.n + SEL_THREADS - 1) / SEL_THREADS) * 64;
    const int i0 = min(sq.n, wave * part), i1 = min(sq.n, i0 + part);
    int c[4] = {0, 0, 0, 0};
    each_key(i0 + lane, 64, i1, [&](int i, uint32_t x) { count_slots(i - lane, i1, x, keep, bar, c); });
    __shared__ __align__(16) int counts[SEL_WAVES][4];
    if (lane == 0)
#pragma unroll
      for (int k = 0; k < 4; ++k) counts[wave][k] = c[k];
    __syncthreads();
    // ... then their ranks
    Ranks r = {0, 0, 0}, end = {0, 0, 0};
    {
      // (unsigned: of the lanes that stand for no wavefront the product may wrap)
      const int w0 = (int)min((uint32_t)sq.n, (uint32_t)lane * part), w1 = min(sq.n, w0 + part);
      add_parts(lane < SEL_WAVES, lane < SEL_WAVES ? *(const int4*)counts[lane] : make_int4(0, 0, 0, 0), w0, w1,
                keep, ties, wave, r, SEL_WAVES, end);
    }
    each_key(i0 + lane, 64, i1, [&](int i, uint32_t x) {
      list_moves(p, sq, i - lane, i1, x, keep, bar, ties, r);
    });
    if (tid == 0) p.count[2 * b + 1] = end.holes;
  } else {
    if (!p.in_place)
      for (int i = tid; i < keep; i += SEL_THREADS) p.to[sq.src.first + i] = i;
    if (tid == 0) p.count[2 * b + 1] = 0;
  }
  if (tid == 0) p.count[2 * b] = keep;
}

// ---- sequences in chunks, a workgroup each ----

// The sequence that chunk x of all sequences belongs to, what it holds, and its first chunk.
__device__ __forceinline__ int find_chunk(const EvictParams& p, int x, int* begin, EvictSeq* sq) {
  return find_sequence_of_block(
      p.batch, x, begin, sq, [&](int b) { return EvictSeq(p, b); },
      [](const EvictSeq& s) { return (s.n + CHUNK - 1) / CHUNK; });
}

__global__ __launch_bounds__(256) void evict_clear_kernel(const EvictParams p) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < (int64_t)p.batch * HIST) p.hist[i] = 0;
  if (i < (int64_t)p.batch * 2) p.count[i] = 0;   // (a sequence that holds nothing has no chunk)
}

// The bar as far as the digits before STEP tell it, and the slots with those digits that stay. The
// counts are requested by the constructor.
template <int STEP>
struct Bar {
  int c1[STEP > 0 ? STEP : 1], c0[STEP > 0 ? STEP : 1], protected_n;
  uint32_t value = 0;
  int keep = 0, ties = 0;
  __device__ __forceinline__ Bar(const EvictParams& p, int b) {
    const int32_t* const h = p.hist + (int64_t)b * HIST;
    const int hi = BINS - 1 - 2 * (int)threadIdx.x;
#pragma unroll
    for (int d = 0; d < STEP; ++d) {
      c1[d] = h[d * BINS + hi];
      c0[d] = h[d * BINS + hi - 1];
    }
    protected_n = h[3 * BINS];
  }
  // (uniform)
  __device__ __forceinline__ void find(const EvictSeq& sq, int* wave_sums, int* found) {
    keep = ties = sq.keep(__builtin_amdgcn_readfirstlane(protected_n));
    if (keep == 0 || keep == sq.n) return;
#pragma unroll
    for (int d = 0; d < STEP; ++d)
      value |= (uint32_t)find_digit(c1[d], c0[d], ties, wave_sums, found) << digit_shift(d);
  }
};
constexpr int PART = CHUNK / SEL_WAVES, PER = PART / 64;   // slots of a chunk's wavefront, of a lane

// Counts of digit D among the slots that share the bar's digits before it.
template <int D>
__global__ __launch_bounds__(SEL_THREADS) void evict_digit_kernel(const EvictParams p) {
  __shared__ int hist[BINS];
  __shared__ int wave_sums[SEL_WAVES];
  __shared__ int found[2];
  int begin = 0;
  EvictSeq sq;
  const int b = find_chunk(p, blockIdx.x, &begin, &sq), tid = threadIdx.x;
  if (b < 0) return;
  const int i0 = ((int)blockIdx.x - begin) * CHUNK, i1 = min(sq.n, i0 + CHUNK);
  Bar<D> bar(p, b);
  uint32_t x[PER];
  load_keys(p, sq, i0 + tid, SEL_THREADS, i1, x);
  for (int i = tid; i < BINS; i += SEL_THREADS) hist[i] = 0;
  if (D > 0) {
    bar.find(sq, wave_sums, found);
    if (bar.keep == 0 || bar.keep == sq.n) return;
  }
  __syncthreads();
  int protected_n = 0;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    if (i0 + tid + k * SEL_THREADS >= i1) break;
    if (D == 0) protected_n += x[k] == 0xffffffffu;
    if (D == 0 || ((x[k] ^ bar.value) >> digit_shift(D > 0 ? D - 1 : 0)) == 0)
      atomicAdd(&hist[(x[k] >> digit_shift(D)) & digit_mask(D)], 1);
  }
  int all;
  block_scan(protected_n, wave_sums, &all);   // (and the counts are complete)
  int32_t* const h = p.hist + (int64_t)b * HIST;
  if (D == 0 && tid == 0 && all > 0) atomicAdd(&h[3 * BINS], all);
  for (int i = tid; i < BINS; i += SEL_THREADS)
    if (hist[i] != 0) atomicAdd(&h[D * BINS + i], hist[i]);
}

// LIST false: the counts of every chunk. True: the moves, given those.
template <bool LIST>
__global__ __launch_bounds__(SEL_THREADS) void evict_chunk_kernel(const EvictParams p) {
  __shared__ int wave_sums[SEL_WAVES];
  __shared__ int found[2];
  __shared__ __align__(16) int counts[SEL_WAVES][4];
  int begin = 0;
  EvictSeq sq;
  const int b = find_chunk(p, blockIdx.x, &begin, &sq), tid = threadIdx.x;
  if (b < 0) return;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i0 = ((int)blockIdx.x - begin) * CHUNK, i1 = min(sq.n, i0 + CHUNK);
  const int p0 = min(i1, i0 + wave * PART), p1 = min(i1, p0 + PART);
  Bar<3> bar(p, b);
  uint32_t x[PER];
  load_keys(p, sq, p0 + lane, 64, p1, x);
  int4 before = make_int4(0, 0, 0, 0);   // of the first 64 chunks before, a lane each
  if (LIST && begin + lane < (int)blockIdx.x) before = *(const int4*)(p.chunk + (int64_t)(begin + lane) * 4);
  bar.find(sq, wave_sums, found);
  const int keep = bar.keep, ties = bar.ties;
  int c[4] = {0, 0, 0, 0};
#pragma unroll
  for (int k = 0; k < PER; ++k)
    count_slots(p0 + k * 64, p1, x[k], keep, bar.value, c);
  if (lane == 0)
#pragma unroll
    for (int k = 0; k < 4; ++k) counts[wave][k] = c[k];
  __syncthreads();
  if (!LIST) {
    if (tid < 4) {
      int sum = 0;
#pragma unroll
      for (int w = 0; w < SEL_WAVES; ++w) sum += counts[w][tid];
      p.chunk[(int64_t)blockIdx.x * 4 + tid] = sum;
    }
    return;
  }
  Ranks r = {0, 0, 0}, end = {0, 0, 0};
  if (keep < sq.n) {
    const int mine = (int)blockIdx.x - begin;   // chunks before
    for (int k0 = 0; k0 < mine; k0 += 64) {
      const int k = k0 + lane;
      const bool in = k < mine;
      const int4 y = k0 == 0 ? before
                     : in ? *(const int4*)(p.chunk + (int64_t)(begin + k) * 4) : make_int4(0, 0, 0, 0);
      add_parts(in, y, k * CHUNK, (k + 1) * CHUNK, keep, ties, min(64, mine - k0), r, 0, r);
    }
    const int w0 = min(i1, i0 + lane * PART), w1 = min(i1, w0 + PART);
    add_parts(lane < SEL_WAVES, lane < SEL_WAVES ? *(const int4*)counts[lane] : make_int4(0, 0, 0, 0), w0, w1,
              keep, ties, wave, r, SEL_WAVES, end);
  }
  if (i1 == sq.n && tid == 0) {
    p.count[2 * b] = keep;
    p.count[2 * b + 1] = end.holes;
  }
  if (keep < sq.n || !p.in_place) {
#pragma unroll
    for (int k = 0; k < PER; ++k)
      list_moves(p, sq, p0 + k * 64, p1, x[k], keep, bar.value, ties, r);
  }
}

// (Where sequences' ranges overlap, against the layout, the lists of one may hold slots of another.)
__device__ __forceinline__ int within(int slot, const Range& r) {
  return (int)min((uint32_t)slot, (uint32_t)r.room - 1);   // (a range with rows has slots)
}

// Rows and bookkeeping: in place the moves, otherwise all slots that are filled, and those behind.
__global__ __launch_bounds__(256) void evict_move_kernel(const EvictParams p) {
  const int b = blockIdx.y;
  const Range from = range_of(p.cu, b, p.slots), to = range_of(p.cu_to, b, p.slots_to);
  const int keep = p.count[2 * b], moves = p.count[2 * b + 1];
  const int64_t s0 = from.first, d0 = to.first;
  const int stride = gridDim.x * 256, first = blockIdx.x * 256 + threadIdx.x;
  const int rows = p.in_place ? moves : keep;
  for (int64_t e = first; e < (int64_t)rows * p.chunks; e += stride) {
    const int i = (int)(e / p.chunks), c = (int)(e - (int64_t)i * p.chunks);
    int s, d;
    if (p.in_place) {
      s = p.from[s0 + i];
      d = p.to[s0 + i];
    } else {
      const int m = p.to[s0 + i];
      s = m >= 0 ? m : p.from[s0 + within(-1 - m, from)];
      d = i;
    }
    s = within(s, from);
    d = within(d, to);
    const int64_t src = (s0 + s) * p.chunks + c, dst = (d0 + d) * p.chunks + c;
    const uint4 k = p.k[src], v = p.v[src];
    p.k_to[dst] = k;
    p.v_to[dst] = v;
    if (c == 0) {
      p.pos_to[d0 + d] = p.kv_pos[s0 + s];
      p.weight_to[d0 + d] = p.weight[s0 + s];
      if (p.in_place) {   // (no other thread reads the slot's entries)
        p.kv_pos[s0 + s] = CP_POS_PAD_KV;
        p.weight[s0 + s] = 0.f;
      }
    }
  }
  if (!p.in_place)
    for (int64_t i = (int64_t)keep + first; i < to.room; i += stride) {
      p.pos_to[d0 + i] = CP_POS_PAD_KV;
      p.weight_to[d0 + i] = 0.f;
    }
  if (first == 0) p.used_to[b] = keep;
}

// Above this many slots a sequence, on average, they are cut into chunks. us (a workgroup each, chunks): 4 sequences
// of 8192 slots 19 and 34, of 16384 29 and 34, of 32768 48 and 34, of 131072 232 and 35; 64 of 16384 43 and 50,
// of 32768 63 and 64, of 65536 139 and 103.
constexpr int64_t kChunkedSlots = 24 * 1024;
constexpr int kCachedKeys = 32768;   // keys in LDS at most: 128 KB

struct EvictPlan {
  bool chunked;
  int64_t chunks;   // there can be
  size_t list, count, hist, chunk, bytes;
};
EvictPlan evict_plan(const cp_shape& s) {
  EvictPlan pl = {};
  pl.chunked = s.total_kv / s.batch > kChunkedSlots;
  pl.chunks = s.total_kv / CHUNK + s.batch;
  pl.list = round256((size_t)s.total_kv * 4);
  pl.count = round256((size_t)s.batch * 8);
  pl.hist = pl.chunked ? round256((size_t)s.batch * HIST * 4) : 0;
  pl.chunk = pl.chunked ? round256((size_t)pl.chunks * 16) : 0;
  pl.bytes = 2 * pl.list + pl.count + pl.hist + pl.chunk;
  return pl;
}

}  // namespace

size_t evict_workspace_bytes(const cp_shape& s) { return evict_plan(s).bytes; }

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
  if (sinks < 0 || s.total_kv > kMaxSlots) return CP_ERR_SHAPE;
  // 16-byte chunks of a row are counted in 31 bits
  if ((int64_t)s.n_kv_heads * s.head_dim > INT32_MAX / 4) return CP_ERR_SHAPE;
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
    if (slots_to < 0 || slots_to > kMaxSlots) return CP_ERR_SHAPE;
    if (k_to == k_cache || v_to == v_cache || kv_pos_to == kv_pos_cache || weight_to == weight ||
        seq_used_to == seq_used)
      return CP_ERR_SHAPE;  // another cache, or in place
  }
  if (s.total_kv > 0 &&
      (k_cache == nullptr || v_cache == nullptr || kv_pos_cache == nullptr || weight == nullptr))
    return CP_ERR_NULL;
  if (!aligned16(k_cache) || !aligned16(v_cache) || !aligned16(k_to) || !aligned16(v_to))
    return CP_ERR_ALIGN;
  static_assert(kMaxWalkedBatch <= 65535, "the grid's second dimension");
  if (s.batch > kMaxWalkedBatch) return CP_ERR_SHAPE;
  const EvictPlan pl = evict_plan(s);
  if (workspace == nullptr || ((uintptr_t)workspace & 255u) != 0 || workspace_bytes < pl.bytes)
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
  char* ws = (char*)workspace;
  auto take = [&ws](size_t bytes) {
    char* const at = ws;
    ws += bytes;
    return at;
  };
  p.to = (int32_t*)take(pl.list);
  p.from = (int32_t*)take(pl.list);
  p.count = (int32_t*)take(pl.count);
  p.hist = (int32_t*)take(pl.hist);
  p.chunk = (int32_t*)take(pl.chunk);
  hipStream_t st = (hipStream_t)stream;
  if (pl.chunked) {
    const dim3 grid((unsigned)pl.chunks), block(SEL_THREADS);
    hipLaunchKernelGGL(evict_clear_kernel, dim3((unsigned)(((int64_t)s.batch * HIST + 255) / 256)), dim3(256),
                       0, st, p);
    hipLaunchKernelGGL(evict_digit_kernel<0>, grid, block, 0, st, p);
    hipLaunchKernelGGL(evict_digit_kernel<1>, grid, block, 0, st, p);
    hipLaunchKernelGGL(evict_digit_kernel<2>, grid, block, 0, st, p);
    hipLaunchKernelGGL(evict_chunk_kernel<false>, grid, block, 0, st, p);
    hipLaunchKernelGGL(evict_chunk_kernel<true>, grid, block, 0, st, p);
  } else {
    // (a batch of more sequences than CUs: two workgroups share one)
    const int64_t most = s.batch > 256 ? kCachedKeys / 4 : kCachedKeys;
    const int cached = (int)(s.total_kv < most ? s.total_kv : most);
    if (hipFuncSetAttribute((const void*)evict_select_kernel, hipFuncAttributeMaxDynamicSharedMemorySize,
                            kCachedKeys * 4) != hipSuccess)
      return CP_ERR_LAUNCH;
    hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)s.batch), dim3(SEL_THREADS), cached * 4, st, p,
                       cached);
  }
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
