// Rotary positions for a step's query and key rows, and its K/V rows into
// their slots of the paged cache.
//
// Pair i of a head (dimensions i and i + R/2 of the R rotated ones, or 2i and
// 2i + 1) belongs to axis a(i) of the positions (time, height, width for
// images) and turns by angle = pos[a(i)][row] * inv_freq[i]:
//     (x, y) -> (x cos - y sin, x sin + y cos)
// in fp32, rounded once to bf16.  A position of 10^6 at frequency 1 has no
// fractional turn left in fp32 (its steps are 0.06 there), so the angle is
// formed and reduced to a turn in fp64, once per row and pair for all heads.
//
// The work is memory traffic: (2 Hq + 4 Hkv) D 2 bytes a row.  Workgroups are of three kinds, so
// that each waits for as few loads in a row as it can: query rows (angles, no slots), key rows
// (both) and value rows (slots, no angles).  One takes `rows` consecutive rows and some heads,
// which share the angles in LDS.
//
// The cache's K plane takes a row's 8 dimensions as 16 bytes with the slots adjacent, its V plane
// 2 bytes a row with the 16 slots of a dimension adjacent, so value rows that follow each other
// in one block (a run) are written together, a whole 32-byte V sector where the run fills its
// block.  A run is at most 16 rows; the workgroup whose rows hold its first row takes all of
// it.  Slots that a run does not fill are not touched (narrower stores), so rows may name slots
// in any order.
//
// Measured (head_dim 128): 15555 rows of 32/8 heads, three axes, 383 MB, 76-90 us, the rate of a
// copy; 1280 rows in windows of 5 15 us, 24.0 MB written where 15.7 are needed as most V sectors are
// written in part (a run as pairs, fours and eights of slots 14.8 us, slot by slot 17.7); 64 single
// rows of 16/8 heads 4.1 us (all kinds in one workgroup, one after the other, 9.9).
#include "nsd_internal.h"

#include <algorithm>

namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;

constexpr int kThreads = 256;
constexpr int kMaxAxes = 4;
constexpr int kRows = 16;              // rows of a workgroup, at most
constexpr int kSpan = kRows + 15;      // with the rest of a run begun in them

// The grid's part of one kind: `heads` heads a workgroup, `groups` such groups.
struct Kind {
  int32_t first, heads, groups;
};

struct RopeArgs {
  const uint16_t *q, *k, *v;
  uint16_t *q_out, *k_pool, *v_pool;
  const int32_t *pos, *slots;
  const float* freq;
  int64_t q_stride, k_stride, v_stride;   // elements between rows
  int64_t num_slots;
  int32_t cuts[kMaxAxes];                 // pairs below cuts[a] belong to axes up to a
  int32_t total, hq, hkv, rot, rows;      // rows of a workgroup: a power of two
  Kind query, key, value;
};

__device__ inline float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float hi_f(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// two fp32 to bf16 (nearest even), the first in the low half
__device__ inline uint32_t pack(float a, float b) {
  const bf16x2 v = __builtin_convertvector(f32x2{a, b}, bf16x2);
  return __builtin_bit_cast(uint32_t, v);
}

// The first row of a run: not the slot after its predecessor's within one block.
__device__ inline bool begins(const int32_t* slots, int64_t i) {
  if (i == 0) return true;
  const int32_t s = slots[i];
  return s < 0 || s % 16 == 0 || slots[i - 1] != s - 1;
}

// Two sets of 8 dimensions turned: half layout x = dims 8c.., y = dims R/2 + 8c..
__device__ inline void turn_half(u32x4& x, u32x4& y, const float2* cs) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 a = cs[2 * e], b = cs[2 * e + 1];
    const float x0 = lo_f(x[e]), x1 = hi_f(x[e]), y0 = lo_f(y[e]), y1 = hi_f(y[e]);
    x[e] = pack(x0 * a.x - y0 * a.y, x1 * b.x - y1 * b.y);
    y[e] = pack(x0 * a.y + y0 * a.x, x1 * b.y + y1 * b.x);
  }
}
// pairs of adjacent dimensions: x's pairs have angles cs[0..3], y's cs[4..7]
__device__ inline void turn_adjacent(u32x4& x, u32x4& y, const float2* cs) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 a = cs[e], b = cs[4 + e];
    const float x0 = lo_f(x[e]), x1 = hi_f(x[e]), y0 = lo_f(y[e]), y1 = hi_f(y[e]);
    x[e] = pack(x0 * a.x - x1 * a.y, x0 * a.y + x1 * a.x);
    y[e] = pack(y0 * b.x - y1 * b.y, y0 * b.y + y1 * b.x);
  }
}

// Unit c of a head: 16 dimensions at offsets *x and *y.  The first rot/16 units are turned,
// with the angles 8c.. of their row; the others pass.
template <bool ADJ>
__device__ inline bool unit(int c, int rot, int* x, int* y) {
  const bool turned = c < rot / 16;
  *x = !turned || ADJ ? 16 * c : 8 * c;
  *y = !turned || ADJ ? 16 * c + 8 : rot / 2 + 8 * c;
  return turned;
}

// (cos, sin) of rows base .. base + n - 1.
template <int D>
__device__ inline void angles(const RopeArgs& A, int64_t base, int n, float2 (*turns)[D / 2]) {
  const int pairs = A.rot / 2;
  for (int u = threadIdx.x; u < n * (D / 2); u += kThreads) {
    const int row = u / (D / 2), p = u % (D / 2);
    if (p >= pairs) continue;
    int axis = 0;
#pragma unroll
    for (int a = 0; a < kMaxAxes - 1; ++a) axis += p >= A.cuts[a];
    const double t = (double)A.pos[(int64_t)axis * A.total + base + row] * (double)A.freq[p] *
                     0.15915494309189533577;   // turns
    float s, c;
    sincospif((float)(2.0 * (t - rint(t))), &s, &c);
    turns[row][p] = make_float2(c, s);
  }
}

// 16 dimensions of a row: loaded, turned where they are, and their places in the head.
template <int D, bool ADJ>
struct Unit {
  u32x4 x, y;
  int xo, yo;
  bool turned;
  __device__ inline void load(const uint16_t* head, int c, int rot) {
    turned = unit<ADJ>(c, rot, &xo, &yo);
    x = *(const u32x4*)(head + xo);
    y = *(const u32x4*)(head + yo);
  }
  __device__ inline void turn(const float2* cs) {
    if (!turned) return;
    if (ADJ) turn_adjacent(x, y, cs);
    else turn_half(x, y, cs);
  }
};

template <int D, bool ADJ>
__device__ inline void query_rows(const RopeArgs& A, int64_t base, int g, float2 (*turns)[D / 2]) {
  constexpr int U = D / 16, kStep = kThreads / U;
  const int n = (int)min((int64_t)A.rows, A.total - base);
  const int h0 = g * A.query.heads, hn = min(A.query.heads, A.hq - h0);
  const int c = threadIdx.x % U, units = n * hn;
  // this thread's (row, head)s, kStep units apart; the first one's row is loaded under the angles
  int i = threadIdx.x / U, row = i / hn, h = i - row * hn;
  const int row_step = kStep / hn, h_step = kStep - row_step * hn;
  Unit<D, ADJ> x;
  auto load = [&] { x.load(A.q + (base + row) * A.q_stride + (h0 + h) * D, c, A.rot); };
  if (i < units) load();
  angles<D>(A, base, n, turns);
  __syncthreads();
  while (i < units) {
    x.turn(&turns[row][8 * c]);
    uint16_t* dst = A.q_out + ((base + row) * A.hq + h0 + h) * D;
    *(u32x4*)(dst + x.xo) = x.x;
    *(u32x4*)(dst + x.yo) = x.y;
    i += kStep;
    row += row_step;
    h += h_step;
    if (h >= hn) h -= hn, ++row;
    if (i < units) load();
  }
}

template <int D, bool ADJ>
__device__ inline void key_rows(const RopeArgs& A, int64_t base, int g, float2 (*turns)[D / 2]) {
  constexpr int U = D / 16;
  const int n = (int)min((int64_t)A.rows, A.total - base);
  const int g0 = g * A.key.heads, gn = min(A.key.heads, A.hkv - g0);
  // neighbouring lanes take neighbouring rows, whose slots are adjacent in the plane
  const int row = threadIdx.x & (A.rows - 1), step = kThreads / A.rows;
  int i = threadIdx.x / A.rows;
  const int units = row < n ? gn * U : 0;
  const int64_t s = row < n ? A.slots[base + row] : -1;
  Unit<D, ADJ> x;
  auto load = [&] {
    x.load(A.k + (base + row) * A.k_stride + (g0 + i / U) * D, i % U, A.rot);
  };
  if (i < units) load();
  angles<D>(A, base, n, turns);
  __syncthreads();
  const bool cached = s >= 0 && s < A.num_slots;
  while (i < units) {
    x.turn(&turns[row][8 * (i % U)]);
    if (cached) {
      uint16_t* dst = A.k_pool + (s / 16 * A.hkv + g0 + i / U) * (D * 16) + s % 16 * 8;
      *(u32x4*)(dst + x.xo * 16) = x.x;
      *(u32x4*)(dst + x.yo * 16) = x.y;
    }
    i += step;
    if (i < units) load();
  }
}

// Slots [s0, s1) of a dimension's 16 (w: all 16, in pairs), in the widest stores that hold no
// other slot: a store of 2 bytes costs as much as one of 16.
__device__ inline void put_run(uint16_t* dst, const u32x4 (&w)[2], int s0, int s1) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (s0 <= 8 * h && s1 >= 8 * h + 8) {
      *(u32x4*)(dst + 8 * h) = w[h];
      continue;
    }
#pragma unroll
    for (int f = 0; f < 2; ++f) {
      const int t = 8 * h + 4 * f;
      if (s0 <= t && s1 >= t + 4) {
        *(u32x2*)(dst + t) = u32x2{w[h][2 * f], w[h][2 * f + 1]};
        continue;
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int p = t + 2 * e;
        const uint32_t x = w[h][2 * f + e];
        if (s0 <= p && s1 >= p + 2) *(uint32_t*)(dst + p) = x;
        else if (s0 <= p && s1 == p + 1) dst[p] = (uint16_t)x;
        else if (s0 == p + 1 && s1 >= p + 2) dst[p + 1] = (uint16_t)(x >> 16);
      }
    }
  }
}

template <int D>
__device__ inline void value_rows(const RopeArgs& A, int64_t i0, int g) {
  __shared__ int32_t slot[kSpan], first[kSpan + 1];   // rows' slots; runs' first rows
  __shared__ int32_t span[2];                         // past the last row; runs
  const int tid = threadIdx.x;
  const int g0 = g * A.value.heads, gn = min(A.value.heads, A.hkv - g0);
  // rows from the first run begun at or after i0 to the first begun at or after i0 + rows
  if (tid < 64) {
    const int64_t i = i0 + tid;
    const bool b = tid < kSpan + 1 && (i >= A.total || begins(A.slots, i));
    const uint64_t m = __ballot(b);
    // a run is at most 16 rows, so both searches end within 16
    const int lo = __builtin_ctzll(m), hi = A.rows + __builtin_ctzll(m >> A.rows);
    const bool mine = b && tid >= lo && tid < hi && i < A.total;
    const uint64_t mm = __ballot(mine);
    if (mine) first[__popcll(mm & ((1ull << tid) - 1))] = tid;
    if (tid < kSpan) slot[tid] = i < A.total ? A.slots[i] : -1;
    if (tid == 0) {
      span[0] = min(hi, (int)min(A.total - i0, (int64_t)kSpan));
      span[1] = __popcll(mm);
    }
  }
  __syncthreads();
  const int runs = span[1];
  // two dimensions of a run
  for (int u = tid; u < runs * gn * (D / 2); u += kThreads) {
    const int c = u % (D / 2), v = u / (D / 2), run = v / gn, head = g0 + v - run * gn;
    const int a = first[run], b = run + 1 < runs ? first[run + 1] : span[0];
    const int64_t s = slot[a];
    if (s < 0 || s >= A.num_slots) continue;
    const int s0 = (int)(s % 16);
    const uint16_t* src = A.v + (i0 + a) * A.v_stride + head * D + 2 * c;
    uint16_t* dst = A.v_pool + ((s / 16 * A.hkv + head) * D + 2 * c) * 16;
    if (b - a == 1) {   // a single token
      const uint32_t x = *(const uint32_t*)src;
      dst[s0] = (uint16_t)x;
      dst[16 + s0] = (uint16_t)(x >> 16);
      continue;
    }
    uint32_t w[16];   // slots beside the run get some row of it: no load waits for a comparison
#pragma unroll
    for (int p = 0; p < 16; ++p)
      w[p] = *(const uint32_t*)(src + min(max(p - s0, 0), b - a - 1) * A.v_stride);
    // the two dimensions' slots, in pairs; [s0, s1) are the run's
    u32x4 even[2], odd[2];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      even[e / 4][e % 4] = (w[2 * e] & 0xffffu) | w[2 * e + 1] << 16;
      odd[e / 4][e % 4] = w[2 * e] >> 16 | (w[2 * e + 1] & 0xffff0000u);
    }
    const int s1 = s0 + b - a;
    put_run(dst, even, s0, s1);
    put_run(dst + 16, odd, s0, s1);
  }
}

template <int D, bool ADJ>
__global__ __launch_bounds__(kThreads) void rope_append_kernel(RopeArgs A) {
  __shared__ float2 turns[kRows][D / 2];
  const int b = blockIdx.x;
  auto place = [&](const Kind& k, int* g) {
    const int i = b - k.first;
    *g = i % k.groups;
    return (int64_t)(i / k.groups) * A.rows;
  };
  int g;
  if (b < A.key.first) {
    const int64_t base = place(A.query, &g);
    query_rows<D, ADJ>(A, base, g, turns);
  } else if (b < A.value.first) {
    const int64_t base = place(A.key, &g);
    key_rows<D, ADJ>(A, base, g, turns);
  } else {
    const int64_t base = place(A.value, &g);
    value_rows<D>(A, base, g);
  }
}

}  // namespace

extern "C" nsd_status nsd_rope_append(void* k_pool, void* v_pool, int64_t num_blocks,
                                      const void* q, int64_t q_stride, const void* k_new,
                                      int64_t k_stride, const void* v_new, int64_t v_stride,
                                      const int32_t* positions, const float* inv_freq,
                                      const int32_t* sections, int32_t n_axes, int32_t rot_dim,
                                      int32_t interleaved, const int32_t* slots, int32_t total_q,
                                      int32_t num_q_heads, int32_t num_kv_heads,
                                      int32_t block_size, int32_t head_dim, void* q_out,
                                      void* stream) {
  using namespace nsd;
  const char* fn = "rope_append";
  if (block_size != NSD_BLOCK_SIZE)
    return fail(NSD_ERR_UNSUPPORTED, "%s: block_size must be 16 (got %d)", fn, block_size);
  if (head_dim != 64 && head_dim != 128)
    return fail(NSD_ERR_UNSUPPORTED, "%s: head_dim must be 64 or 128 (got %d)", fn, head_dim);
  if (num_kv_heads < 1 || num_q_heads < 1 || num_q_heads % num_kv_heads || num_q_heads > 65535)
    return fail(NSD_ERR_SHAPE, "%s: num_q_heads (%d) must be a positive multiple of "
                "num_kv_heads (%d), at most 65535", fn, num_q_heads, num_kv_heads);
  if (total_q < 0 || num_blocks < 0) return fail(NSD_ERR_SHAPE, "%s: negative size", fn);
  if (num_blocks > (1 << 27) || num_blocks * num_kv_heads > 0x7fffffff)
    return fail(NSD_ERR_UNSUPPORTED, "%s: more than 2^27 blocks or 2^31-1 (block, KV head) "
                "tiles in a pool", fn);
  if (rot_dim < 0 || rot_dim > head_dim || rot_dim % 16)
    return fail(NSD_ERR_SHAPE, "%s: rot_dim must be a multiple of 16 in [0, head_dim] (got %d)",
                fn, rot_dim);
  if (n_axes < 1 || n_axes > kMaxAxes)
    return fail(NSD_ERR_SHAPE, "%s: n_axes must be in [1, %d]", fn, kMaxAxes);
  if (n_axes > 1 && !sections) return fail(NSD_ERR_NULL, "%s: sections is NULL", fn);
  RopeArgs A;
  int64_t upto = 0;
  for (int a = 0; a < kMaxAxes; ++a) {
    if (a < n_axes) {
      const int32_t n = n_axes > 1 || sections ? sections[a] : rot_dim / 2;
      if (n < 0) return fail(NSD_ERR_SHAPE, "%s: a negative section", fn);
      upto += n;
    }
    A.cuts[a] = a < n_axes - 1 ? (int32_t)(upto < head_dim ? upto : head_dim) : head_dim;
  }
  if (upto != rot_dim / 2)
    return fail(NSD_ERR_SHAPE, "%s: the sections must hold rot_dim / 2 = %d pairs (got %lld)", fn,
                rot_dim / 2, (long long)upto);
  if (total_q == 0) return NSD_OK;
  if (!q || !k_new || !v_new || !slots || !q_out || (rot_dim && (!positions || !inv_freq)) ||
      (num_blocks && (!k_pool || !v_pool)))
    return fail(NSD_ERR_NULL, "%s: NULL pointer argument", fn);
  const int64_t q_row = (int64_t)num_q_heads * head_dim, kv_row = (int64_t)num_kv_heads * head_dim;
  const int64_t most = (int64_t)1 << 40;
  if (q_stride < q_row || k_stride < kv_row || v_stride < kv_row || q_stride > most ||
      k_stride > most || v_stride > most)
    return fail(NSD_ERR_SHAPE, "%s: a row stride is shorter than its row", fn);
  if ((q_stride | k_stride | v_stride) % 8 ||
      ((uintptr_t)q | (uintptr_t)k_new | (uintptr_t)v_new | (uintptr_t)q_out |
       (uintptr_t)k_pool | (uintptr_t)v_pool) % 16)
    return fail(NSD_ERR_SHAPE, "%s: rows and planes must be 16-byte aligned", fn);
  if (q_out == q && q_stride != q_row)
    return fail(NSD_ERR_SHAPE, "%s: q is turned in place only where its rows are dense", fn);
  A.q = (const uint16_t*)q;
  A.k = (const uint16_t*)k_new;
  A.v = (const uint16_t*)v_new;
  A.q_out = (uint16_t*)q_out;
  A.k_pool = (uint16_t*)k_pool;
  A.v_pool = (uint16_t*)v_pool;
  A.pos = positions;
  A.slots = slots;
  A.freq = inv_freq;
  A.q_stride = q_stride;
  A.k_stride = k_stride;
  A.v_stride = v_stride;
  A.num_slots = num_blocks * NSD_BLOCK_SIZE;
  A.total = total_q;
  A.hq = num_q_heads;
  A.hkv = num_kv_heads;
  A.rot = rot_dim;
  // Few rows: few of them a workgroup, and a workgroup for each group of heads, until the device
  // has enough workgroups (four a CU).
  A.rows = total_q <= 256 ? 4 : kRows;
  const int64_t tiles = ((int64_t)total_q + A.rows - 1) / A.rows;
  int64_t blocks = 0;
  auto kind = [&](int32_t heads, int32_t most) {
    Kind k;
    k.first = (int32_t)blocks;
    k.heads = std::min(heads, most);
    while (k.heads > 1 && tiles * ((heads + k.heads - 1) / k.heads) < 1024) k.heads = (k.heads + 1) / 2;
    k.groups = (heads + k.heads - 1) / k.heads;
    blocks += tiles * k.groups;
    return k;
  };
  A.query = kind(num_q_heads, 32);
  A.key = kind(num_kv_heads, 32);
  A.value = kind(num_kv_heads, 32);
  if (blocks * kThreads > UINT32_MAX)   // a launch's threads
    return fail(NSD_ERR_UNSUPPORTED, "%s: too many workgroups", fn);
  const dim3 grid((uint32_t)blocks);
  clear_stale_error();
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, (hipStream_t)stream, A);
  };
  if (head_dim == 64) interleaved ? go(rope_append_kernel<64, true>) : go(rope_append_kernel<64, false>);
  else interleaved ? go(rope_append_kernel<128, true>) : go(rope_append_kernel<128, false>);
  return check_launch(fn);
}
