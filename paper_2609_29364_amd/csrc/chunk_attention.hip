// Attention of each request's new tokens (a prompt chunk, or one token) over
// its paged cache.
//
// Query row (token j, head h) of request r sits at position p = L_r - n_r + j
// and sees token t iff t < prefix_r, or first_j <= t <= p (first_j = 0 where no
// first keys are given), in a block whose id is valid:
//     x_t = f(scale <q, k_t>) - slope_h |p - t|,  f(x) = cap tanh(x / cap) or x
//     o   = sum_t e^(x_t - m) v_t / sum_t e^(x_t - m),  m = max_t x_t
// in one pass over the tokens with the running maximum and sum in fp32.
//
// The (query tokens x heads of a group) rows of one KV head are one product's
// columns: S^T = K Q^T and O^T = V^T P^T on 32x32x16 bf16 MFMAs.  A workgroup
// of four waves takes 128 rows, 32 a wave, whose Q operands stay in registers;
// stages of 64 tokens (four blocks) go to LDS by direct loads, double-buffered,
// and serve all four waves.  Two workgroups share a CU, so one's softmax runs
// under the other's MFMAs.  The cache's layout feeds the MFMAs as it is: a K
// operand is 16 bytes of one slot (8 dimensions), a V^T operand 16 bytes of one
// dimension (8 slots).  The K rows enter with bits 2 and 3 of their slot
// swapped, which makes the eight S^T values a lane holds of a block those of
// the 8 slots its V^T operand has: P^T goes from accumulator to operand
// (rounded to bf16, an error of at most 2^-8 of each weight) without leaving
// its lane.
//
// The softmax rescale is skipped while no row's maximum grows by more than 8 in log2
// (weights then stay below 2^8, far from any limit of fp32), a published refinement of the one-pass
// softmax.  Tokens hidden from a row get weight 0; as 0 times an infinity or NaN is NaN, a V operand
// of a stage with hidden tokens is looked through for them, and where one has any they are taken out
// of the product and added to the rows that see them.
//
// Items of at most 64 rows (single tokens, ends of chunks) are bound by memory: their
// waves stream K and V into registers, each its own tokens.  Larger ones are bound by the
// matrix cores and, about as much, the ALU that runs the softmax.  Measured (32/8 heads,
// head_dim 128): 8192 tokens after 24000 3240-3340 us, 1130-1163 TFLOP/s, the matrix cores busy
// 63 % of the cycles (the card's library product reaches 1120-1580 TFLOP/s by size); four prompts
// of 4096 tokens 530-546 us, 1007-1038 TFLOP/s; 256 single tokens at 1-4k 412-416 us, 6.5 TB/s; 128
// of them at 2-8k, capped, in a window of 1024 behind a prefix 97-99 us, 5.8 TB/s.  128 rows rather
// than 256: two workgroups of four waves on a CU rather than one of eight, which all wait at one
// barrier.
#include "chunk_plan.h"
#include "nsd_internal.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;

constexpr int kThreads = 64 * kWaves;
constexpr int kStageBlocks = kStage / NSD_BLOCK_SIZE;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kSlack = 8.f;                // log2 of the weights' bound
constexpr int kUnits = 32;                   // of an item's rows, at most, in the join
// CAP of the templates below: scores are not capped, capped at up to kUsual, or at more.
enum { kNoCap, kUsualCap, kLargeCap };
constexpr float kUsual = 256.f;

struct Params {
  const uint16_t* q;
  const uint16_t *k, *v;
  const int32_t* first;
  const float* slopes;
  uint16_t* out;
  // Split items: how many a KV head has, a record of each (splits | first place << 8, first
  // query token, first row, rows); and by place, one a part, the rows' (max, sum) and
  // normalised values.
  int32_t* split_items;
  int4* records;      // [split items][hkv]
  float2* part_ml;    // [places][hkv][kRows]
  float* part;        // [places][hkv][kRows][D]
  int64_t num_blocks;
  float scale, cap;   // scale log2 e > 0 (a negative scale's sign is in `negate`)
  uint32_t negate;    // 0x80008000: Q's signs are flipped
  int32_t width, bs, total_q, hq, hkv, group, max_len, tile, items, max_places, parted, units;
};

__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ inline uint32_t pack(float a, float b) {
  const bf16x2 v = __builtin_convertvector(f32x2{a, b}, bf16x2);
  return __builtin_bit_cast(uint32_t, v);
}

// x of the lane 32 away (a register swapped with a copy of itself holds both halves' values).
__device__ inline float other_half(float x) {
  uint32_t a = __float_as_uint(x), b = a;
  asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1\n\ts_nop 1" : "+v"(a), "+v"(b));
  return __uint_as_float((threadIdx.x & 32) ? a : b);
}

// The first item of request r: its rows' tiles are items first_item(r) .. first_item(r + 1) - 1,
// which are at least ceil(rows / tile) of them whatever the rows, so no prefix sum is needed.
__device__ inline int first_item(const Params& P, const int32_t* indptr, int r) {
  const int64_t a = min(max(indptr[r], 0), P.total_q);
  return (int)(a * P.group / P.tile) + r;
}

// The last request whose first item is at most `item`, by 64 lanes' probes a round.
__device__ inline int find_request(const Params& P, const int32_t* indptr, int item) {
  int lo = 0, n = P.bs;
  while (n > 1) {
    const int step = (n + 63) / 64, i = lo + (int)(threadIdx.x & 63) * step;
    const bool in = i < lo + n && (i == lo || first_item(P, indptr, i) <= item);
    const uint64_t m = __ballot(in);
    const int last = 63 - __builtin_clzll(m);
    n = min(step, n - last * step);
    lo += last * step;
  }
  return uniform(lo);
}

// Sums and maxima over the wave's lanes up to each.
template <class T, class Op>
__device__ inline T wave_scan(T x, T none, Op op) {
  auto step = [&](auto ctrl, auto rows) {
    const int y = __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none),
                                              __builtin_bit_cast(int, x), decltype(ctrl)::value,
                                              decltype(rows)::value, 0xf, false);
    x = op(x, __builtin_bit_cast(T, y));
  };
  using std::integral_constant;
  const integral_constant<int, 0xf> all{};
  step(integral_constant<int, 0x111>{}, all);   // from 1, 2, 4 and 8 lanes below in a row of 16
  step(integral_constant<int, 0x112>{}, all);
  step(integral_constant<int, 0x114>{}, all);
  step(integral_constant<int, 0x118>{}, all);
  step(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});   // the row below's last
  step(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});   // the lower half's last
  return x;
}
template <class T>
__device__ inline T last_lane(T x) {
  return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}
__device__ inline int sum_scan(int x) { return wave_scan(x, 0, [](int a, int b) { return a + b; }); }

// What a workgroup does for its KV head: split `split` of `splits` of a request's tile of rows;
// place: of its partial result; record: of its item.  r < 0: nothing.
struct Piece {
  int r, tile, split, splits, place, record;
  int a0, a1, length;   // the request's query rows; its length, at most max_len
};

// The idx-th piece of a batch of at most kPartedBatch requests, found by every wave from the
// batch's lengths (a lane has up to four requests), so that no launch and no list goes before.
//
// A tile's cost is the stages its request's tokens span (split_limit() and last_round() say
// which are split).  Long pieces go first, in five classes of length.  All waves compute the same
// from the same lengths.
//
// Offsets that fall (no valid batch's) count tokens twice, and the items may pass the host's
// bound: such a batch is not split, so that no part or record lacks its workgroup, and items past
// the grid are left out.
__device__ inline Piece find_piece(const Params& P, const int32_t* indptr, const int32_t* lens,
                                   const int32_t* prefixes, int idx) {
  const int lane = threadIdx.x & 63, per = (P.bs + 63) / 64;
  int tiles[kPerLane], stages[kPerLane], splits[kPerLane], base[kPerLane], nth[kPerLane];
  float cost = 0.f;
  int count = 0;
  bool falls = false;
  int a[kPerLane], b[kPerLane], L[kPerLane], prefix[kPerLane], first[kPerLane];
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) {   // (all the loads in flight)
    const int r = min(i * 64 + lane, P.bs - 1);
    a[i] = indptr[r];
    b[i] = indptr[r + 1];
    L[i] = lens[r];
    prefix[i] = prefixes ? prefixes[r] : 0;
  }
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) {
    a[i] = min(max(a[i], 0), P.total_q);
    b[i] = min(max(b[i], 0), P.total_q);
    falls |= b[i] < a[i];
    b[i] = max(b[i], a[i]);
    first[i] = P.first ? P.first[min(a[i], P.total_q - 1)] : 0;
  }
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) {
    const bool in = i * 64 + lane < P.bs;
    const int length = min(max(L[i], 0), P.max_len);
    const int from = min(max(first[i], 0), length);
    const int seen = min(max(prefix[i], 0), from);
    tiles[i] = in ? (int)(((int64_t)(b[i] - a[i]) * P.group + P.tile - 1) / P.tile) : 0;
    stages[i] = in ? max((length - from + seen + kStage - 1) / kStage, 1) : 0;
    splits[i] = 1;
    cost += (float)tiles[i] * stages[i];
    count += tiles[i];
  }
  const auto add = [](float x, float y) { return x + y; };
  const auto larger = [](float x, float y) { return fmaxf(x, y); };
  const float total = last_lane(wave_scan(cost, 0.f, add));
  const int items = last_lane(sum_scan(count));
  Tail tail{0, 1};
  if (P.max_places) {
    const bool rising = !__ballot(falls);
    const float limit = rising ? split_limit(items, total, P.hkv) : INFINITY;
    int places = 0, split_items = 0;
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
      if (i >= per) continue;
      splits[i] = parts_of(stages[i], limit);
      const int y = splits[i] > 1 ? tiles[i] : 0, x = y * splits[i];
      const int upto = sum_scan(x), nth_upto = sum_scan(y);
      base[i] = places + upto - x;
      nth[i] = split_items + nth_upto - y;
      places += last_lane(upto);
      split_items += last_lane(nth_upto);
    }
    if (places > P.max_places) {   // cannot be, by the bound the host took
#pragma unroll
      for (int i = 0; i < kPerLane; ++i) splits[i] = 1;
      split_items = 0;
    }
    if (rising && split_items == 0) {
      tail = last_round(items, P.hkv);
      split_items = tail.items;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) *P.split_items = split_items;
  }
  int mine = 0;
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) mine += tiles[i] * splits[i];
  const int whole = last_lane(sum_scan(mine)) - tail.items, pieces = whole + tail.items * tail.parts;
  if (idx >= pieces) return Piece{-1};
  const int part = idx < whole ? 0 : (idx - whole) % tail.parts;
  const int nth_tail = idx < whole ? -1 : (idx - whole) / tail.parts;
  if (nth_tail >= 0) idx = whole + nth_tail;
  float most = 0.f, each[kPerLane];
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) {
    each[i] = (float)stages[i] / splits[i];
    if (tiles[i]) most = fmaxf(most, each[i]);
  }
  // pieces that all run at once are one class
  most = pieces * P.hkv > kSlots ? last_lane(wave_scan(most, 0.f, larger)) : -1.f;
  const float bounds[6] = {INFINITY, 0.75f * most, 0.5f * most, 0.35f * most, 0.2f * most, -1.f};
  int before = 0;
#pragma unroll
  for (int k = 0; k < 5; ++k)
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
      if (i >= per) continue;
      const int x = each[i] <= bounds[k] && each[i] > bounds[k + 1] ? tiles[i] * splits[i] : 0;
      const int upto = before + sum_scan(x);
      const uint64_t m = __ballot(upto > idx);
      if (m) {
        const int l = __builtin_ctzll(m);
        auto at = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
        const int local = idx - at(upto - x), n = at(splits[i]), t = at(tiles[i]);
        Piece p;
        p.r = i * 64 + l;
        p.splits = n;
        p.split = local % n;
        p.tile = t - 1 - local / n;   // a request's last rows see the most tokens
        p.place = n > 1 ? at(base[i]) + p.tile * n + p.split : 0;
        p.record = n > 1 ? at(nth[i]) + p.tile : 0;
        if (nth_tail >= 0) {   // (no request is split besides)
          p.splits = tail.parts;
          p.split = part;
          p.place = nth_tail * tail.parts + part;
          p.record = nth_tail;
        }
        p.a0 = at(a[i]);
        p.a1 = at(b[i]);
        p.length = min(max(at(L[i]), 0), P.max_len);
        return p;
      }
      before = last_lane(upto);
    }
  return Piece{-1};
}

// 1 KiB from src + OFFSET to dst + OFFSET, 16 bytes a lane.
template <int OFFSET>
__device__ inline void load_lds(const uint16_t* src, void* dst) {
  __builtin_amdgcn_global_load_lds(
      (const __attribute__((address_space(1))) uint32_t*)(src + (threadIdx.x & 63) * 8),
      (__attribute__((address_space(3))) uint32_t*)dst, 16, OFFSET, 0);
}

template <int D>
struct Acc {
  f32x16 o[D / 32];   // O^T: row of the wave = lane % 32, dimension 32 t + 8 (i / 4) + 4 (lane / 32) + i % 4
  float m, l;         // running maximum (log2 domain) and this lane's sum
  bool odd;           // an infinity or NaN was left out of the product
};

// One row's mask: what its position, first key and prefix let it see.
struct Sight {
  int p, first, prefix;
  float slope;   // log2 domain
  int length;    // of the request

  // of the block at t0, the 8 tokens this lane's operands hold: a bit for each that it sees
  __device__ inline uint32_t sees(int t0) const {
    t0 += (threadIdx.x & 32) >> 2;
    return (below(p - t0 + 1) & ~below(first - t0)) | below(prefix - t0);
  }
  // the lowest n bits of 8
  static __device__ inline uint32_t below(int n) { return (1u << min(max(n, 0), 8)) - 1; }
};

// MFMA operands from a block's tiles.
template <int D>
struct Tile {
  static constexpr int kHalf = D * 16;   // elements of a block's K or V tile

  // This lane's K operand in its block's tile (the two halves of the lanes' 16s take a block
  // each): its slot with bits 2 and 3 swapped.
  static __device__ inline int key_offset() {
    const int lane = threadIdx.x & 63, r = lane & 15;
    return (lane >> 5) * 128 + ((r & 3) | (r & 4) << 1 | (r & 8) >> 1) * 8;
  }
  static __device__ inline int value_offset() {
    const int lane = threadIdx.x & 63;
    return (lane & 31) * 16 + (lane >> 5) * 8;
  }

  // S^T of 32 tokens x 32 rows.  k: two blocks' tiles [D/8][16][8].
  static __device__ inline f32x16 scores(const uint16_t* k, const bf16x8 (&q)[D / 16]) {
    const uint16_t* p = k + (threadIdx.x >> 4 & 1) * kHalf + key_offset();
    f32x16 s = {};
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk)
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8*)(p + kk * 256), q[kk], s, 0, 0, 0);
    return s;
  }

  // V^T operand of block b's dimensions 32 t ..: [D][16] as it is in the cache.
  static __device__ inline bf16x8 values(const uint16_t* v, int b, int t) {
    return *(const bf16x8*)(v + b * kHalf + t * 512 + value_offset());
  }
};

// bf16 pairs: the larger of two by 16-bit halves.
__device__ inline uint32_t max16(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a),
                                                                __builtin_bit_cast(u16x2, b)));
}
// Whether any of the bf16 values of an operand is an infinity or NaN: m collects their
// exponents.
__device__ inline uint32_t exponents(uint32_t m, bf16x8 v) {
  const u32x4 x = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int e = 0; e < 4; ++e) m = max16(m, x[e] & 0x7f807f80u);
  return m;
}
__device__ inline bool unusual(uint32_t m) { return (m & 0xffffu) == 0x7f80u || m >> 16 == 0x7f80u; }

// The operand's values at bits m (a bit each); the others 0.
__device__ inline bf16x8 keep(bf16x8 v, uint32_t m) {
  u32x4 x = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int e = 0; e < 4; ++e)
    x[e] &= (m >> (2 * e) & 1 ? 0xffffu : 0u) | (m >> (2 * e + 1) & 1 ? 0xffff0000u : 0u);
  return __builtin_bit_cast(bf16x8, x);
}

// A bit for each value of an operand that is +infinity (sign 0), -infinity (sign 1) or NaN.
__device__ inline uint32_t infinite(bf16x8 v, uint32_t sign) {
  const u32x4 x = __builtin_bit_cast(u32x4, v);
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t h = x[e / 2] >> (16 * (e % 2)) & 0xffffu;
    m |= (uint32_t)(((h & 0x7fffu) > 0x7f80u) | (h == (0x7f80u | sign << 15))) << e;
  }
  return m;
}

// bf16 1 at bits m, else 0.
__device__ inline bf16x8 ones(uint32_t m) {
  const u32x4 one = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
  return keep(__builtin_bit_cast(bf16x8, one), m);
}

// Scores of NSUB x 32 tokens from t0 on, capped and biased, to the log2 domain (c: scale log2 e).
//
// The cap as 1 - 2 / (1 + e^(2 x / cap)) takes two numbers of its own size from one another: off by
// 2^-22 of the cap or so whatever the score, which up to kUsual is 2^-14 of a weight, a 64th of
// its rounding to bf16.  kLargeCap, for caps beyond: the series of tanh where |x / cap| < 1/4 (its
// next term is 2^-26 of the score there), so that the error is about 5 2^-23 of the score itself.
// It costs prompts of packed documents 106 -> 141 us, single tokens 97 -> 98.
template <int CAP, bool BIAS, int NSUB>
__device__ inline void to_log2(f32x16 (&s)[NSUB], float c, float cap, const Sight& w, int t0,
                               int half) {
  const float y = CAP ? fminf(2.f * c / cap, 3e38f) : 0.f;
  const float top = fminf(cap * kLog2e, 3e38f), u1 = c / top;
  const float d0 = (float)(w.p - t0 - 8 * half);
#pragma unroll
  for (int u = 0; u < NSUB; ++u)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float x;
      if constexpr (CAP == kUsualCap) {
        // cap tanh(x / cap): 1 - 2 / (1 + e^(2 x / cap))
        const float e = __builtin_amdgcn_exp2f(s[u][i] * y);
        x = fmaf(-2.f * top, __builtin_amdgcn_rcpf(1.f + e), top);
      } else if constexpr (CAP == kLargeCap) {
        const float v = s[u][i] * u1, vv = v * v;
        const float e = __builtin_amdgcn_exp2f(s[u][i] * y);
        const float far = top * fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + e), 1.f);
        const float series =
            vv * fmaf(vv, fmaf(vv, fmaf(vv, 62.f / 2835, -17.f / 315), 2.f / 15), -1.f / 3);
        x = s[u][i] * c;
        x = fabsf(v) < 0.25f ? fmaf(x, series, x) : far;
      } else {
        x = s[u][i] * c;
      }
      if constexpr (BIAS) x = fmaf(-w.slope, fabsf(d0 - (float)(u * 32 + i / 8 * 16 + i % 8)), x);
      s[u][i] = x;
    }
}

// The running maximum takes `top` (of this lane's tokens) in, where some row's grew by more
// than kSlack: only then do the row's two lanes meet.
template <int D>
__device__ inline void grow(Acc<D>& a, float top) {
  if (!__ballot(top > a.m + kSlack)) return;
  top = fmaxf(top, other_half(top));
  const float m = fmaxf(a.m, top);
  const float f = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(a.m - m);
  a.m = m;
  a.l *= f;
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) a.o[t][i] *= f;
}

// Softmax and the second product of NSUB x 32 tokens from t0 on for a wave's rows: s their
// S^T, values(b, t) the V^T operand of block b's dimensions 32 t...  hidden: some row may not
// see some token.  valid: bit b set if block b may be read.
template <int D, int CAP, bool BIAS, int NSUB, class Values>
__device__ inline void weigh(Acc<D>& a, f32x16 (&s)[NSUB], const Values& values, const Params& P,
                             const Sight& w, int t0, uint32_t valid, bool hidden) {
  const int half = (threadIdx.x & 63) >> 5;
  const float c = P.scale;
  if constexpr (CAP || BIAS) to_log2<CAP, BIAS, NSUB>(s, c, P.cap, w, t0, half);
  constexpr bool kLog2 = CAP || BIAS;   // scores are in the log2 domain already
  if (hidden) {
#pragma unroll
    for (int b = 0; b < NSUB * 2; ++b) {
      const uint32_t seen = valid >> b & 1 ? w.sees(t0 + b * 16) : 0u;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int i = b % 2 * 8 + e;
        const uint32_t on = (uint32_t)((int32_t)(seen << (31 - e)) >> 31);
        s[b / 2][i] = __uint_as_float((__float_as_uint(s[b / 2][i]) & on) | (0xff800000u & ~on));
      }
    }
  }
  float top = s[0][0];
#pragma unroll
  for (int u = 0; u < NSUB; ++u)
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, s[u][i]);
  if constexpr (!kLog2) top *= c;
  grow(a, top);
  const float sub = a.m == -INFINITY ? 0.f : a.m;
  u32x4 p[NSUB * 2];
#pragma unroll
  for (int u = 0; u < NSUB; ++u)
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      float e[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        e[j] = __builtin_amdgcn_exp2f(kLog2 ? s[u][i + j] - sub : fmaf(s[u][i + j], c, -sub));
        a.l += e[j];
      }
      p[u * 2 + i / 8][i % 8 / 2] = pack(e[0], e[1]);
    }
#pragma unroll
  for (int b = 0; b < NSUB * 2; ++b) {
    bf16x8 vt[D / 32];
#pragma unroll
    for (int t = 0; t < D / 32; ++t) vt[t] = values(b, t);
    if (hidden) {
      // slots past the request's last token, and blocks that may not be read, hold anything
      const int left = w.length - (t0 + b * 16);
      if (!(valid >> b & 1) || left < 16) {
        const int mine = left - 8 * half;
        const uint32_t in = !(valid >> b & 1) || mine <= 0 ? 0u : mine < 8 ? (1u << mine) - 1 : 0xffu;
#pragma unroll
        for (int t = 0; t < D / 32; ++t) vt[t] = keep(vt[t], in);
      }
      uint32_t m = 0;
#pragma unroll
      for (int t = 0; t < D / 32; ++t) m = exponents(m, vt[t]);
      if (__ballot(unusual(m))) {
        a.odd = true;
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
          vt[t] = keep(vt[t], ~(infinite(vt[t], 0) | infinite(vt[t], 1)));
      }
    }
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
      a.o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vt[t], __builtin_bit_cast(bf16x8, p[b]),
                                                       a.o[t], 0, 0, 0);
  }
}

// Adds to the rows what weigh() left out: the infinities and NaN of the V operands (v: their
// place in this lane) of the block at t0 that each row sees.  Their numbers per row and
// dimension are products of flags.
template <int D>
__device__ inline void add_infinities(Acc<D>& a, const uint16_t* v, const Sight& w, int t0) {
  const int left = w.length - t0 - (threadIdx.x & 32) / 4;
  const uint32_t in = left <= 0 ? 0u : left < 8 ? (1u << left) - 1 : 0xffu;
  const bf16x8 see = ones(w.sees(t0) & in);
#pragma unroll
  for (int t = 0; t < D / 32; ++t) {
    const bf16x8 x = *(const bf16x8*)(v + t * 512);
#pragma unroll
    for (uint32_t sign = 0; sign < 2; ++sign) {
      f32x16 n = {};
      n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ones(infinite(x, sign) & in), see, n, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 16; ++i) a.o[t][i] += n[i] > 0.f ? (sign ? -INFINITY : INFINITY) : 0.f;
    }
  }
}

// weigh() from a stage's tiles in LDS.
template <int D, int CAP, bool BIAS, int NSUB>
__device__ inline void stage(Acc<D>& a, const uint16_t* k, const uint16_t* v,
                             const bf16x8 (&q)[D / 16], const Params& P, const Sight& w, int t0,
                             uint32_t valid, bool hidden) {
  using T = Tile<D>;
  f32x16 s[NSUB];
#pragma unroll
  for (int u = 0; u < NSUB; ++u) s[u] = T::scores(k + u * 2 * T::kHalf, q);
  weigh<D, CAP, BIAS, NSUB>(a, s, [&](int b, int t) { return T::values(v, b, t); }, P, w, t0,
                            valid, hidden);
}

// stage() of 64 tokens that every row sees: the hot one.  Left to itself the compiler has two
// LDS reads in flight and waits for them before every other MFMA, so the order is given:
// eight K operands ahead of the first MFMA, the first V operands under the last ones, the
// weights of a block under the MFMAs of the one before.
template <int D>
__device__ inline void open_stage(Acc<D>& a, const uint16_t* k, const uint16_t* v,
                                  const bf16x8 (&q)[D / 16], float c) {
  using T = Tile<D>;
  constexpr int KK = D / 16, VT = D / 32;
  const uint16_t* kp = k + (threadIdx.x >> 4 & 1) * T::kHalf + T::key_offset();
  bf16x8 kf[2][KK], vf[4][VT];
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) kf[u][kk] = *(const bf16x8*)(kp + u * 2 * T::kHalf + kk * 256);
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int t = 0; t < VT; ++t) vf[b][t] = T::values(v, b, t);
  f32x16 s[2] = {};
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
      s[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[u][kk], q[kk], s[u], 0, 0, 0);
  float top = s[0][0];
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, s[u][i]);
  __builtin_amdgcn_sched_group_barrier(0x100, KK, 0);
#pragma unroll
  for (int i = 0; i < KK; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  }
#pragma unroll
  for (int i = 0; i < KK; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x002, 1, 0);
  }
  // The waves of a SIMD drift out of step where the one that weighs goes first: 8192 tokens after
  // 24000 3364 -> 3283 us, a mixed step 162 -> 156 (2 ragged chunks 2830 -> 2886).
  __builtin_amdgcn_s_setprio(1);
  grow(a, top * c);
  const float sub = a.m == -INFINITY ? 0.f : a.m;
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    u32x4 p;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      float e[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float x = s[b / 2][b % 2 * 8 + i + j];
        e[j] = __builtin_amdgcn_exp2f(fmaf(x, c, -sub));
        a.l += e[j];
      }
      p[i / 2] = pack(e[0], e[1]);
    }
    if (b < 2) {
#pragma unroll
      for (int t = 0; t < VT; ++t) vf[b + 2][t] = T::values(v, b + 2, t);
    }
#pragma unroll
    for (int t = 0; t < VT; ++t)
      a.o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[b][t], __builtin_bit_cast(bf16x8, p),
                                                       a.o[t], 0, 0, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x002, 28, 1);
  __builtin_amdgcn_s_setprio(0);
#pragma unroll
  for (int b = 0; b < 3; ++b)
#pragma unroll
    for (int t = 0; t < VT; ++t) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
      if (b < 2) __builtin_amdgcn_sched_group_barrier(0x100, 1, 1);
      __builtin_amdgcn_sched_group_barrier(0x002, 28 / VT, 1);
    }
  __builtin_amdgcn_sched_group_barrier(0x008, VT, 1);
}

template <int D, int CAP, bool BIAS>
__global__ __launch_bounds__(kThreads, 2) void chunk_kernel(
    const Params P, const int32_t* __restrict__ tables, const int32_t* __restrict__ lens,
    const int32_t* __restrict__ indptr, const int32_t* __restrict__ prefixes) {
  constexpr int kTile = D * 16;                     // elements of a block's K or V tile
  constexpr int kPlane = kStageBlocks * kTile;      // of a stage's K or V
  __shared__ __attribute__((aligned(16))) uint16_t buf0[2 * kPlane], buf1[2 * kPlane];
  __shared__ float2 meet[kWaves][64];
  using T = Tile<D>;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  // heads fastest: with 8 KV heads the workgroups of a head share an XCD's L2
  const int x = blockIdx.x, g = x % P.hkv;
  Piece piece;
  if (P.parted) {
    piece = find_piece(P, indptr, lens, prefixes, x / P.hkv);
    if (piece.r < 0) return;
  } else {
    // the items as they come, the last first, none split
    const int item = P.items - 1 - x / P.hkv;
    const int r = find_request(P, indptr, item);
    piece = Piece{r, item - first_item(P, indptr, r), 0, 1, 0, 0};
    piece.a0 = min(max(indptr[r], 0), P.total_q);
    piece.a1 = min(max(indptr[r + 1], piece.a0), P.total_q);
    piece.length = min(max(lens[r], 0), P.max_len);
  }
  const int r = piece.r;
  const int a0 = piece.a0, n = piece.a1 - a0;
  const int64_t rows = (int64_t)n * P.group;
  const int64_t row0 = (int64_t)piece.tile * P.tile;
  if (row0 < 0 || row0 >= rows) return;
  const int L = min(piece.length, P.width < (1 << 26) ? P.width * 16 : 1 << 30);
  const int last = L - 1;
  const int prefix = prefixes ? min(max(prefixes[r], 0), L) : 0;

  // few rows: the waves share them (one or two groups of 32) and part the tokens
  const int count = (int)min(rows - row0, (int64_t)P.tile);
  const int rgroups = count <= kWaveRows ? 1 : count <= 2 * kWaveRows ? 2 : kWaves;
  const int rg = wave & (rgroups - 1), tgroups = kWaves / rgroups, tg = wave / rgroups;
  const bool idle = rg * kWaveRows >= count;   // a wave without rows

  // this lane's row
  const int64_t row = row0 + rg * kWaveRows + (lane & 31);
  const bool mine = row < row0 + count;
  const int j = mine ? (int)(row / P.group) : 0, h = mine ? (int)(row - (int64_t)j * P.group) : 0;
  Sight w;
  w.p = mine ? min(L - n + j, last) : -1;
  w.first = mine && P.first ? max(P.first[a0 + j], 0) : 0;
  w.prefix = mine ? prefix : 0;
  w.length = L;
  w.slope = BIAS && mine ? P.slopes[g * P.group + h] * kLog2e : 0.f;
  bf16x8 q[D / 16];
  {
    const uint16_t* src = P.q + ((int64_t)(a0 + j) * P.hq + g * P.group + h) * D + (lane >> 5) * 8;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      u32x4 t = {};
      if (mine) t = *(const u32x4*)(src + kk * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) t[e] ^= P.negate;
      q[kk] = __builtin_bit_cast(bf16x8, t);
    }
  }
  // the lowest and highest first key of the wave's rows and of the workgroup's (at most 128
  // query tokens), and the wave's first and last position
  int fmin = 0, fmax = 0, from = 0, high = 0;
  if (P.first) {
    const int j0 = (int)(row0 / P.group), j1 = (int)((row0 + count - 1) / P.group);
    const int f0 = P.first[a0 + min(j0 + lane, j1)], f1 = P.first[a0 + min(j0 + 64 + lane, j1)];
    const auto less = [](int x, int y) { return min(x, y); };
    const auto more = [](int x, int y) { return max(x, y); };
    fmin = last_lane(wave_scan(mine ? w.first : INT32_MAX, INT32_MAX, less));
    fmax = last_lane(wave_scan(mine ? w.first : INT32_MIN, INT32_MIN, more));
    from = max(last_lane(wave_scan(min(f0, f1), INT32_MAX, less)), 0);
    high = max(last_lane(wave_scan(max(f0, f1), INT32_MIN, more)), 0);
  }
  const int64_t wave_last = min(row0 + count, row0 + (rg + 1) * kWaveRows) - 1;
  const int pmin = min(L - n + (int)((row0 + rg * kWaveRows) / P.group), last);
  const int pmax = min(L - n + (int)(wave_last / P.group), last);
  const int low = min(L - n + (int)(row0 / P.group), last);   // the workgroup's first position
  const int to = min(L - n + (int)((row0 + count - 1) / P.group), last) + 1;   // past its last key
  // stages: those of the prefix, then from the first key's on
  const int n1 = (prefix + kStage - 1) / kStage;
  const int s2 = max(n1, from / kStage);
  const int n2 = to > 0 ? max((to + kStage - 1) / kStage - s2, 0) : 0;
  const int stages = n1 + n2;
  const int per = (stages + piece.splits - 1) / piece.splits;
  const int i0 = min(piece.split * per, stages), i1 = min(i0 + per, stages);

  Acc<D> a;
#pragma unroll
  for (int t = 0; t < D / 32; ++t) a.o[t] = f32x16{};
  a.m = -INFINITY;
  a.l = 0.f;
  a.odd = false;

  const int32_t* table = tables + (int64_t)r * P.width;
  const int blocks = (L + 15) / 16;
  auto start = [&](int i) { return (i < n1 ? i : i - n1 + s2) * kStage; };
  // The ids of 64 blocks (16 stages), a lane each, and of the 64 after them: a scalar load and
  // its wait per stage would cost every stage its latency.
  int chunk = -2, now = 0, ahead = 0;
  uint64_t good = 0;   // which of them may be read
  auto ids = [&](int c) { return table[min(c * 64 + lane, blocks - 1)]; };
  auto seek = [&](int t0) {   // ids for the stage at t0; which of its blocks may be read
    const int c = t0 >> 10;
    if (c != chunk) {
      now = c == chunk + 1 ? ahead : ids(c);
      ahead = ids(c + 1);
      good = __ballot((now >= 0) & (now < P.num_blocks) & (c * 64 + lane < blocks));
      chunk = c;
    }
    return (uint32_t)(good >> (t0 >> 4 & 63)) & ((1u << kStageBlocks) - 1);
  };
  // wave w loads block w of the stage sought; an unreadable one's place gets block 0
  auto load = [&](int t0, uint32_t valid, uint16_t* buf) {
    const int id = valid >> wave & 1 ? __builtin_amdgcn_readlane(now, (t0 >> 4 & 63) + wave) : 0;
    const int64_t at = ((int64_t)id * P.hkv + g) * kTile;
    uint16_t *kd = buf + wave * kTile, *vd = kd + kPlane;
    load_lds<0>(P.k + at, kd);
    load_lds<1024>(P.k + at, kd);
    if constexpr (D == 128) {
      load_lds<2048>(P.k + at, kd);
      load_lds<3072>(P.k + at, kd);
    }
    load_lds<0>(P.v + at, vd);
    load_lds<1024>(P.v + at, vd);
    if constexpr (D == 128) {
      load_lds<2048>(P.v + at, vd);
      load_lds<3072>(P.v + at, vd);
    }
  };
  auto arrived = [&] {
    __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0): this wave's part of the stage is in LDS
    __syncthreads();
  };
  // every row of the workgroup sees every token of such a stage
  auto open = [&](int i, uint32_t valid) {
    const int t0 = start(i);
    return (((t0 + kStage - 1 <= low) & (t0 >= high)) | (t0 + kStage <= prefix)) &
           (valid == (1u << kStageBlocks) - 1);
  };
  auto seen_by_all = [&](int i, const uint16_t* buf) {
    if constexpr (CAP || BIAS)
      stage<D, CAP, BIAS, 2>(a, buf, buf + kPlane, q, P, w, start(i), 0xf, false);
    else
      open_stage<D>(a, buf, buf + kPlane, q, P.scale);
  };
  auto seen_by_some = [&](int i, uint32_t valid, const uint16_t* buf) {
    const int t0 = start(i);
    if (idle) return;
    for (int u = 0; u < 2; ++u) {
      const int t = t0 + u * 32;
      const uint32_t ok = valid >> (2 * u) & 3;
      if (((t > pmax) | (t + 32 <= fmin)) & (t >= prefix)) continue;
      const bool all = ((t + 31 <= pmin) & (t >= fmax)) | (t + 32 <= prefix);
      stage<D, CAP, BIAS, 1>(a, buf + u * 2 * kTile, buf + kPlane + u * 2 * kTile, q, P, w, t, ok,
                             !(all & (ok == 3)));
    }
  };
  auto infinities = [&] {
    if (!a.odd) return;   // rare: the pieces once more
    for (int j = 2 * i0 + tg; j < 2 * i1; j += tgroups)
      for (int b = 0; b < 2; ++b) {
        const int t0 = start(j >> 1) + (j & 1) * 32 + b * 16;
        const int id = table[min(t0 / 16, blocks - 1)];
        if (t0 < L && id >= 0 && id < P.num_blocks)
          add_infinities<D>(a, P.v + ((int64_t)id * P.hkv + g) * kTile + T::value_offset(), w, t0);
      }
  };
  if (tgroups > 1) {
    // Few rows: bound by the bytes in flight.  Every wave streams its own 32-token pieces from
    // memory into registers, without a barrier: K of the next piece is requested once the
    // scores have consumed this one's, V once the second product has.
    const int j1 = 2 * i1;
    bf16x8 kr[D / 16], vr[2][D / 32];
    const int own = lane >> 4 & 1;   // this lane's block of the piece
    int id[2];
    uint32_t valid = 0;
    auto place = [&](int j) { return start(j >> 1) + (j & 1) * 32; };
    auto find = [&](int j) {
      valid = 0;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int blk = place(j) / 16 + b;
        id[b] = table[min(blk, blocks - 1)];
        const bool ok = (blk < blocks) & (id[b] >= 0) & (id[b] < P.num_blocks);
        valid |= ok ? 1u << b : 0u;
        id[b] = ok ? id[b] : 0;
      }
    };
    auto keys = [&] {
      const uint16_t* p = P.k + ((int64_t)(own ? id[1] : id[0]) * P.hkv + g) * kTile + T::key_offset();
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
        kr[kk] = __builtin_nontemporal_load((const bf16x8*)(p + kk * 256));
    };
    auto values = [&] {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const uint16_t* p = P.v + ((int64_t)id[b] * P.hkv + g) * kTile + T::value_offset();
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
          vr[b][t] = __builtin_nontemporal_load((const bf16x8*)(p + t * 512));
      }
    };
    int j = 2 * i0 + tg;
    if (j < j1) {
      find(j);
      keys();
      values();
    }
    while (j < j1) {
      const int t0 = place(j), next = j + tgroups;
      const uint32_t ok = valid;
      f32x16 s[1] = {};
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
        s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kr[kk], q[kk], s[0], 0, 0, 0);
      if (next < j1) {
        find(next);
        keys();
      }
      const bool all = ((t0 + 31 <= pmin) & (t0 >= fmax)) | (t0 + 32 <= prefix);
      weigh<D, CAP, BIAS, 1>(a, s, [&](int b, int t) { return vr[b][t]; }, P, w, t0, ok,
                             !(all & (ok == 3)));
      if (next < j1) values();
      j = next;
    }
    infinities();
    // the token groups' results meet in LDS
    a.l += other_half(a.l);
    auto region = [&](int v) { return (float*)((v & 2 ? buf1 : buf0) + (v & 1) * kPlane) + lane; };
    if (tg) {
      float* to = region(wave);
#pragma unroll
      for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) to[(t * 16 + i) * 64] = a.o[t][i];
      meet[wave][lane] = make_float2(a.m, a.l);
    }
    __syncthreads();
    if (tg) return;
    for (int o = 1; o < tgroups; ++o) {
      const float2 y = meet[o * rgroups + rg][lane];
      const float* from = region(o * rgroups + rg);
      const float m = fmaxf(a.m, y.x);
      const float f = a.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(a.m - m);
      const float e = y.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(y.x - m);
      a.m = m;
      a.l = a.l * f + y.y * e;
#pragma unroll
      for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) a.o[t][i] = a.o[t][i] * f + from[(t * 16 + i) * 64] * e;
    }
  } else {
    // Stages in pairs, a buffer each.  va, vb: which blocks of a pair's stages may be read.
    uint32_t va = 0, vb = 0;
    auto first = [&](int i) {   // stage i goes to buf0
      if (i >= i1) return;
      va = seek(start(i));
      load(start(i), va, buf0);
    };
    first(i0);
    for (int i = i0; i < i1; i += 2) {
      while (i + 1 < i1) {   // the hot loop
        vb = seek(start(i + 1));
        if (!(open(i, va) & open(i + 1, vb)) | idle) break;
        arrived();
        load(start(i + 1), vb, buf1);
        seen_by_all(i, buf0);
        arrived();
        first(i + 2);
        seen_by_all(i + 1, buf1);
        i += 2;
      }
      if (i >= i1) break;
      arrived();
      const uint32_t ok = va;
      if (i + 1 < i1) load(start(i + 1), vb, buf1);
      seen_by_some(i, ok, buf0);
      if (i + 1 >= i1) break;
      arrived();
      first(i + 2);
      seen_by_some(i + 1, vb, buf1);
    }
    infinities();
    a.l += other_half(a.l);
  }

  const int64_t place = (int64_t)piece.place * P.hkv + g;
  if (piece.splits > 1 && piece.split == 0 && tid == 0)
    P.records[(int64_t)piece.record * P.hkv + g] =
        make_int4(piece.splits | piece.place << 8, a0, (int)row0, count);
  if (!mine) return;
  const float l = a.l;
  const float f = l == 0.f ? 0.f : 1.f / l;   // no visible token: 0
  if (piece.splits == 1) {
    uint16_t* dst = P.out + ((int64_t)(a0 + j) * P.hq + g * P.group + h) * D + (lane >> 5) * 4;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        u32x2 y;
        y[0] = pack(a.o[t][4 * c] * f, a.o[t][4 * c + 1] * f);
        y[1] = pack(a.o[t][4 * c + 2] * f, a.o[t][4 * c + 3] * f);
        *(u32x2*)(dst + t * 32 + c * 8) = y;
      }
    return;
  }
  const int64_t at = place * kRows + rg * kWaveRows + (lane & 31);
  float* dst = P.part + at * D + (lane >> 5) * 4;
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      float4 y = {a.o[t][4 * c] * f, a.o[t][4 * c + 1] * f, a.o[t][4 * c + 2] * f, a.o[t][4 * c + 3] * f};
      *(float4*)(dst + t * 32 + c * 8) = y;
    }
  if (lane < 32) P.part_ml[at] = make_float2(a.m, l);
}

// The splits of an item's rows joined: D/4 threads take a row's columns, several such teams
// part many splits and meet in LDS.  A row of 64 splits, or many rows of 16, are loads after one
// another, so the rows of an item (and KV head) are up to 32 units of work: as many as there are
// workgroups for, of the items the host bounds (P.units) where they are few and mostly all
// split, of those the device counts where they are a last round's.
template <int D>
__global__ __launch_bounds__(kThreads) void join_kernel(const Params P) {
  constexpr int kTeam = D / 4, kTeams = kThreads / kTeam;
  __shared__ float4 sums[kTeams][kTeam];
  __shared__ float2 meet[kTeams];   // (max, sum)
  const int team = threadIdx.x / kTeam, c = threadIdx.x % kTeam;
  // records fastest: neighbouring workgroups, on different XCDs, have as many rows to join
  const int room = P.units ? (int)gridDim.x / P.units : 1;
  int4 rec = P.records[blockIdx.x % room];   // (not after the count: a latency less)
  const int records = *P.split_items * P.hkv, stride = P.units ? room : max(records, 1);
  const int each = P.units ? P.units : max(1, min(kUnits, (int)gridDim.x / stride));
  for (int unit = blockIdx.x; unit < stride * each; unit += gridDim.x) {
    const int nth = unit % stride, part = unit / stride;
    if (nth >= records) return;
    if (!P.units) rec = P.records[nth];
    const int splits = rec.x & 0xff, count = rec.w, g = nth % P.hkv;
    const int64_t place = (int64_t)(rec.x >> 8) * P.hkv + g;
    const int teams = splits > 16 ? 8 : splits > 8 ? 4 : splits > 4 ? 2 : 1, rows = kTeams / teams;
    const int first = team & (teams - 1);
    for (int row0 = part * rows; row0 < count; row0 += each * rows) {
      const int row = row0 + team / teams;
      const bool in = row < count;
      const int64_t at = place * kRows + row, step = (int64_t)P.hkv * kRows;
      float m = -INFINITY, sum = 0.f;
      float4 o = {0.f, 0.f, 0.f, 0.f};
      for (int s0 = first; in && s0 < splits; s0 += 4 * teams) {
        float2 x[4];
        float4 y[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {   // the four loads in flight; past the last split: nothing seen
          const int s = min(s0 + u * teams, splits - 1);
          x[u] = P.part_ml[at + s * step];
          y[u] = *(const float4*)(P.part + (at + s * step) * D + c * 4);
          if (s0 + u * teams >= splits || x[u].y == 0.f) x[u] = make_float2(-INFINITY, 0.f);
        }
        const float top = fmaxf(fmaxf(m, fmaxf(x[0].x, x[1].x)), fmaxf(x[2].x, x[3].x));
        const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
        m = top;
        sum *= keep;
        o.x *= keep, o.y *= keep, o.z *= keep, o.w *= keep;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          if (x[u].y == 0.f) continue;
          const float f = __builtin_amdgcn_exp2f(x[u].x - m) * x[u].y;
          sum += f;
          o.x += f * y[u].x, o.y += f * y[u].y, o.z += f * y[u].z, o.w += f * y[u].w;
        }
      }
      if (teams > 1) {
        __syncthreads();
        sums[team][c] = o;
        if (c == 0) meet[team] = make_float2(m, sum);
        __syncthreads();
        float top = m;
        for (int t = 1; t < teams; ++t) top = fmaxf(top, meet[team - first + t].x);
        const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
        sum *= keep;
        o.x *= keep, o.y *= keep, o.z *= keep, o.w *= keep;
        for (int t = 1; t < teams; ++t) {
          const float2 x = meet[team - first + t];
          if (x.y == 0.f) continue;   // (the sum of NaN scores is NaN, their maximum -infinity)
          const float f = __builtin_amdgcn_exp2f(x.x - top);
          const float4 y = sums[team - first + t][c];
          sum += f * x.y;
          o.x += f * y.x, o.y += f * y.y, o.z += f * y.z, o.w += f * y.w;
        }
      }
      if (in && first == 0) {
        const float f = sum == 0.f ? 0.f : 1.f / sum;
        const int r = rec.z + row, j = r / P.group, h = r - j * P.group;
        u32x2 y;
        y[0] = pack(o.x * f, o.y * f);
        y[1] = pack(o.z * f, o.w * f);
        *(u32x2*)(P.out + ((int64_t)(rec.y + j) * P.hq + g * P.group + h) * D + c * 4) = y;
      }
    }
  }
}

bool sizes_ok(int32_t bs, int32_t total_q, int32_t hq, int32_t hkv, int32_t d, int32_t max_q,
              int32_t max_len) {
  return bs >= 0 && bs <= kMaxBatch && total_q >= 0 && hkv >= 1 && hq >= hkv && hq % hkv == 0 &&
         (d == 64 || d == 128) && max_q >= 1 && max_len >= 1 &&
         (int64_t)total_q * hq <= INT32_MAX;
}

}  // namespace

extern "C" size_t nsd_chunk_attention_workspace_size(int32_t bs, int32_t total_q,
                                                     int32_t num_q_heads, int32_t num_kv_heads,
                                                     int32_t head_dim, int32_t max_q_per_seq,
                                                     int32_t max_seq_len) {
  if (!sizes_ok(bs, total_q, num_q_heads, num_kv_heads, head_dim, max_q_per_seq, max_seq_len))
    return 0;
  return workspace_bytes(plan(bs, total_q, num_q_heads, num_kv_heads, max_seq_len), num_kv_heads,
                         head_dim);
}

extern "C" size_t nsd_chunk_attention_workspace_bound(int32_t num_kv_heads, int32_t head_dim) {
  if (num_kv_heads < 1 || (head_dim != 64 && head_dim != 128)) return 0;
  return workspace_bound(num_kv_heads, head_dim);
}

extern "C" nsd_status nsd_chunk_attention(
    const void* q, const void* k_cache, const void* v_cache, int64_t num_blocks,
    const int32_t* block_table, int32_t max_blocks_per_seq, const int32_t* seq_lens,
    const int32_t* q_indptr, int32_t bs, int32_t total_q, int32_t num_q_heads,
    int32_t num_kv_heads, int32_t head_dim, int32_t block_size, int32_t max_q_per_seq,
    int32_t max_seq_len, float scale, float softcap, const float* slopes,
    const int32_t* first_keys, const int32_t* prefix_lens, void* out, void* workspace,
    size_t workspace_size, void* stream) {
  using namespace nsd;
  const char* fn = "chunk_attention";
  if (bs < 0 || bs > kMaxBatch)
    return fail(NSD_ERR_SHAPE, "%s: bs must be in [0, %d]", fn, kMaxBatch);
  if (block_size != NSD_BLOCK_SIZE)
    return fail(NSD_ERR_UNSUPPORTED, "%s: block_size must be 16 (got %d)", fn, block_size);
  if (head_dim != 64 && head_dim != 128)
    return fail(NSD_ERR_UNSUPPORTED, "%s: head_dim must be 64 or 128 (got %d)", fn, head_dim);
  if (num_kv_heads < 1 || num_q_heads < 1 || num_q_heads % num_kv_heads)
    return fail(NSD_ERR_SHAPE, "%s: num_q_heads (%d) must be a positive multiple of "
                "num_kv_heads (%d)", fn, num_q_heads, num_kv_heads);
  if (total_q < 0 || max_q_per_seq < 1 || max_seq_len < 1 || max_blocks_per_seq < 1 ||
      num_blocks < 0)
    return fail(NSD_ERR_SHAPE, "%s: total_q, max_q_per_seq, max_seq_len, max_blocks_per_seq or "
                "num_blocks out of range", fn);
  if ((int64_t)total_q * num_q_heads > INT32_MAX)
    return fail(NSD_ERR_UNSUPPORTED, "%s: more than 2^31-1 query rows", fn);
  if (num_blocks > INT32_MAX || num_blocks * num_kv_heads > INT32_MAX)
    return fail(NSD_ERR_UNSUPPORTED, "%s: more than 2^31-1 (block, KV head) tiles in a pool", fn);
  if (!std::isfinite(scale)) return fail(NSD_ERR_SHAPE, "%s: scale must be finite", fn);
  if (!(softcap >= 0.f) || std::isinf(softcap))
    return fail(NSD_ERR_SHAPE, "%s: softcap must be finite and not negative (0: none)", fn);
  if (bs == 0 || total_q == 0) return NSD_OK;
  if (!q || !block_table || !seq_lens || !q_indptr || !out || (num_blocks && (!k_cache || !v_cache)))
    return fail(NSD_ERR_NULL, "%s: NULL pointer argument", fn);
  if (((uintptr_t)q | (uintptr_t)k_cache | (uintptr_t)v_cache | (uintptr_t)out) % 16)
    return fail(NSD_ERR_SHAPE, "%s: q, out and the caches must be 16-byte aligned", fn);
  const Plan pl = plan(bs, total_q, num_q_heads, num_kv_heads, max_seq_len);
  const size_t need = workspace_bytes(pl, num_kv_heads, head_dim);
  if (need && (!workspace || workspace_size < need || (uintptr_t)workspace % 16))
    return fail(NSD_ERR_WORKSPACE, "%s: a 16-byte aligned workspace of %zu bytes needed, %zu given",
                fn, need, workspace ? workspace_size : (size_t)0);
  const int64_t groups = pieces(pl, num_kv_heads) * num_kv_heads;
  if (groups * kThreads > UINT32_MAX)   // a launch's threads
    return fail(NSD_ERR_UNSUPPORTED, "%s: too many workgroups", fn);
  Params P;
  P.q = (const uint16_t*)q;
  P.k = (const uint16_t*)k_cache;
  P.v = (const uint16_t*)v_cache;
  P.first = first_keys;
  P.slopes = slopes;
  P.out = (uint16_t*)out;
  const int64_t places = (int64_t)pl.places * num_kv_heads;
  const int64_t split_items = (int64_t)pl.split_items * num_kv_heads;
  P.split_items = (int32_t*)workspace;
  P.records = (int4*)((char*)workspace + 16);
  P.part_ml = (float2*)(P.records + split_items);
  P.part = (float*)(P.part_ml + places * kRows);
  P.max_places = pl.places;
  // The order matters where the items do not all run at once and differ: of few or short requests,
  // many rounds, or more requests than find_piece() holds, they start as they come.
  P.parted = pl.places || (max_seq_len > 12 * kStage && bs >= 16 && bs <= kPartedBatch && pl.items * num_kv_heads > kSlots &&
                           pl.items * num_kv_heads <= 8 * kSlots);
  P.num_blocks = num_blocks;
  // 0 becomes a factor too small to move a weight, as 0 times a hidden token's -infinity is NaN;
  // nor is it infinite, as that times a score of 0 is too
  P.scale = std::min(std::max(std::fabs(scale) * kLog2e, 1e-37f), 3e38f);
  P.cap = softcap;
  P.negate = std::signbit(scale) ? 0x80008000u : 0u;
  P.width = max_blocks_per_seq;
  P.bs = bs;
  P.total_q = total_q;
  P.hq = num_q_heads;
  P.hkv = num_kv_heads;
  P.group = num_q_heads / num_kv_heads;
  P.max_len = num_blocks ? max_seq_len : 0;   // without a pool nothing is visible
  P.tile = pl.tile;
  P.items = (int32_t)pl.items;
  clear_stale_error();
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((uint32_t)groups), dim3(kThreads), 0, (hipStream_t)stream, P,
                       block_table, seq_lens, q_indptr, prefix_lens);
  };
  const bool bias = slopes != nullptr;
  auto capped = [&](auto d, auto biased) {
    constexpr int D = decltype(d)::value;
    constexpr bool kBias = decltype(biased)::value;
    if (softcap == 0.f) go(chunk_kernel<D, kNoCap, kBias>);
    else if (softcap <= kUsual) go(chunk_kernel<D, kUsualCap, kBias>);
    else go(chunk_kernel<D, kLargeCap, kBias>);
  };
  auto dims = [&](auto d) { bias ? capped(d, std::true_type{}) : capped(d, std::false_type{}); };
  if (head_dim == 64) dims(std::integral_constant<int, 64>{});
  else dims(std::integral_constant<int, 128>{});
  if (const nsd_status st = check_launch(fn)) return st;
  if (pl.places) {
    // about four workgroups a CU
    P.units = pl.items * num_kv_heads > kSlots
                  ? 0 : (int)std::max<int64_t>(1, std::min<int64_t>(kUnits, 2 * kSlots / split_items));
    const dim3 grid((uint32_t)(P.units ? split_items * P.units
                                       : std::min<int64_t>(split_items * kUnits, 2 * kSlots)));
    if (head_dim == 64)
      hipLaunchKernelGGL(join_kernel<64>, grid, dim3(kThreads), 0, (hipStream_t)stream, P);
    else
      hipLaunchKernelGGL(join_kernel<128>, grid, dim3(kThreads), 0, (hipStream_t)stream, P);
    return check_launch(fn);
  }
  return NSD_OK;
}
