// Attention over the paged cache (bf16 or 4 bits) with a sliding window and
// first tokens that stay visible.
//
// out = sum_j 2^(c s_j - m) v_j / sum_j 2^(c s_j - m), s = q . k, c = scale *
// log2 e, in one pass over the keys: a running m, and sums rescaled when it
// moves.  The query heads of a key head are rows beside each other, so a key
// is read once for all of them: with few rows a call is bound by the cache's
// bytes (a row of 128 dims: 512 bytes a token and head in bf16, 136 in 4 bits),
// with many by the two products, 4 dh operations a row and key.  Two kernels
// for the two ends: few rows, keys straight to registers, all workgroups'
// shares of the keys alike; many rows, tiles of keys in LDS that 128 rows
// share.  Both keep the scores transposed (K Q^T), which leaves the weights
// where the second product takes its operand from: no weight goes through LDS.
// The weights are rounded to bf16 for that product, each by at most 2^-8 of it:
// outputs of the timed cases are off by 0.0023 of their size, where rounding them
// alone is 0.0017.  With what is left of each weight in a second product they are
// off by 0.0017, but prompts take 375 us for 300, chunks on 4-bit keys 778 for 575
// and 64 rows 159 for 133; single tokens 0 to 3% more, and are rounded alike so
// that a row is as exact as a token as it is in a chunk.
#include <algorithm>
#include <climits>
#include <cmath>
#include <type_traits>

#include "conv_common.hpp"
#include "kv_cache.hpp"

namespace dstack {

namespace {

typedef __attribute__((__vector_size__(2 * sizeof(int)))) int i32x2;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;

constexpr float LOG2E = 1.4426950408889634f;
// Sums are rescaled once a score passes their reference by 2^SLACK, not at
// every new maximum: weights stay below 2^SLACK, as exact relative to their
// sum as those below 1.
constexpr float SLACK = 8.f;
constexpr int COUNTERS = 4096;            // arrival counters at the workspace's start
constexpr int MERGE_ROWS = 2048;          // splits times rows that one merge holds

struct AttendArgs {
  const bf16* q;
  long q_stride;
  bf16* out;
  float* part;          // partial results: per unit [splits][rows][DH], then [splits][rows][2]
  unsigned* counters;
  int heads, group, max_q, window, sinks;
  FastDiv by_group;
  int splits, chunk;    // workgroups per unit, key tiles of one
  int part_rows;        // rows of a unit's partial result
  float scale;
};

// What the rows of one sequence see: keys below `end`, of them those below
// `sink_tiles` tiles and those from tile `first` on.
struct Range {
  int p0;               // position of the first row
  int end;              // one past the last key that any row sees
  int lo_first, lo_last;  // first key of the first and of the last row's window
  int sinks;
};

__device__ __forceinline__ int window_start(int p, int window) {
  return window ? (int)max(0L, (long)p - window + 1) : 0;
}

__device__ __forceinline__ Range key_range(const KVView& kv, int len, int n, int first_row, int rows, int window,
                                           int sinks) {
  Range r;
  r.p0 = len > 0 ? len - n + first_row : -1;
  const int p1 = len > 0 ? r.p0 + rows - 1 : -1;
  r.end = max(0, min(min(len, (int)((long)kv.max_pages << kv.shift)), p1 + 1));
  r.lo_first = window_start(r.p0, window);
  r.lo_last = window_start(p1, window);
  r.sinks = window ? sinks : 0;
  return r;
}

// Tiles of `size` keys that hold visible ones: [0, sink) and [first, last).
struct Tiles {
  int sink, first, count;
  __device__ __forceinline__ Tiles(const Range& r, int size) {
    const int last = (r.end + size - 1) / size;
    first = min(r.lo_first / size, last);
    sink = min((min(r.sinks, r.end) + size - 1) / size, first);
    count = sink + last - first;
  }
  __device__ __forceinline__ int operator[](int t) const { return t < sink ? t : first + t - sink; }
};

// maximum over the lanes that share lane % 32
__device__ __forceinline__ float half_max(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

// maximum over the lanes that share lane % 16
__device__ __forceinline__ float quad_max(float v) {
  v = half_max(v);
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

// sum over the lanes that share lane % 16
__device__ __forceinline__ float quad_sum(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// exp2(x - m) with m = -inf standing for "no key yet"
__device__ __forceinline__ float known(float m) { return m == -INFINITY ? 0.f : m; }

// whether a sum of products with zero is finite: NaN if any value of w is not
__device__ __forceinline__ float poison(unsigned w, float acc) {
  const bf16x2 z = {(bf16)0.f, (bf16)0.f};
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), z, acc, false);
}

template <int WORDS>
__device__ __forceinline__ bool not_finite(const unsigned (&val)[8][WORDS]) {
  float bad = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int w = 0; w < WORDS; ++w) bad = poison(val[j][w], bad);
  return bad != 0.f;
}

// Infinities and NaN among values: 0 * infinity is NaN in a row that does not
// see the key, in one whose weight of it is below what fp32 holds, and in sums
// rescaled past it.  They are taken out of the values and noted in LDS for the
// rows that see them, two bits a dim (+inf 1, -inf 2, NaN 3), to be added to the
// rows' sums at the end.  The few-row kernel looks for them on the way (bf16: one
// operation for two values, which costs nothing beside the reads; 4 bits: the
// scales alone, 2 to 3% where vector work bounds it); the tile kernel, whose
// values go through LDS, takes a unit again, looking, where a sum ended as NaN.
__device__ __forceinline__ unsigned odd_bits(unsigned x) {  // of a bf16 value
  const unsigned a = x & 0x7fffu;
  return a > 0x7f80u ? 3u : a < 0x7f80u ? 0u : x >> 15 ? 2u : 1u;
}
__device__ __forceinline__ unsigned without_odd(unsigned w) {  // of two values
  return ((w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu) | ((w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u);
}
template <int DH>
__device__ __forceinline__ float odd_of(const unsigned* notes, int row, int dim) {
  const unsigned b = notes[row * (DH / 16) + (dim >> 4)] >> (2 * (dim & 15)) & 3u;
  return b == 0u ? 0.f : b == 1u ? INFINITY : b == 2u ? -INFINITY : __uint_as_float(0x7fc00000u);
}
// Notes what is not finite of the two values w at dims dim, dim + 1 of a key for the rows that see it.
template <int DH, typename Sees>
__device__ __forceinline__ void note_odd(unsigned* notes, unsigned w, int dim, int rows, Sees sees) {
  const unsigned bits = odd_bits(w & 0xffffu) | odd_bits(w >> 16) << 2;
  if (bits)
#pragma unroll 1
    for (int r = 0; r < rows; ++r)
      if (sees(r)) atomicOr(notes + r * (DH / 16) + (dim >> 4), bits << (2 * (dim & 15)));
}

// Eight dims of a query row (not live: zeros).
__device__ __forceinline__ bf16x8 query(const bf16* p, bool aligned, bool live) {
  bf16x8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (bf16)0.f;
  if (live && aligned) v = *reinterpret_cast<const bf16x8*>(p);
  if (live && !aligned)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = p[e];
  return v;
}
__device__ __forceinline__ bf16x8 with_sign(bf16x8 v, float sign) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (bf16)((float)v[e] * sign);
  return v;
}

// a row's output from its sums (0: no visible key)
__device__ __forceinline__ f32x4 normed(f32x4 v, float sum) {
  return sum == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : v * (1.f / sum);
}

// The factor of a part whose maximum is m beside the whole's M: at least fp32's
// least value, so that a part's infinities stay what they are (0 * infinity is
// NaN).  It adds at most 2^-149 of the part's sums to the whole's.
__device__ __forceinline__ float part_factor(float m, float M) { return fmaxf(exp2_fast(m - known(M)), 0x1p-149f); }

__device__ __forceinline__ void store_out(bf16* p, f32x4 v, bool aligned) {
  const bf16x4 o = {(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
  if (aligned) {
    *reinterpret_cast<bf16x4*>(p) = o;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = o[e];
  }
}

// The last of a unit's workgroups to arrive joins their parts, in order.  Every
// thread's device-scope stores of this workgroup's part come before.
template <int DH, typename Dst>
__device__ __forceinline__ void join_parts(const AttendArgs& a, __amdgpu_buffer_rsrc_t pr, size_t unit, int parts,
                                           int rows, float* lds, int* arrived, Dst dst) {
  const unsigned ml_at = (unsigned)a.splits * a.part_rows * DH * 4;
  wait_vmcnt<0>();
  __syncthreads();
  if (threadIdx.x == 0)
    *arrived = (int)__hip_atomic_fetch_add(a.counters + unit, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (*arrived != parts - 1) return;
  if (threadIdx.x == 0) __hip_atomic_store(a.counters + unit, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  for (int x = threadIdx.x; x < parts * rows; x += 256) {  // at most MERGE_ROWS
    const int sp = x / rows, rr = x - sp * rows;
    const auto ml = __builtin_amdgcn_raw_buffer_load_b64(pr, (int)(ml_at + ((unsigned)sp * a.part_rows + rr) * 8), 0, CPOL_SC1);
    lds[x] = __builtin_bit_cast(float, (int)ml[0]);
    lds[MERGE_ROWS + x] = __builtin_bit_cast(float, (int)ml[1]);
  }
  __syncthreads();
  const bool o16 = ((uintptr_t)a.out & 15) == 0;
  for (int x = threadIdx.x; x < rows * (DH / 4); x += 256) {
    const int rr = x / (DH / 4), d = x % (DH / 4) * 4;
    float mm = -INFINITY;
    for (int sp = 0; sp < parts; ++sp) mm = fmaxf(mm, lds[sp * rows + rr]);
    float sum = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < parts; s0 += 8) {
      f32x4 v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k)
        v[k] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                             pr, (int)(((unsigned)min(s0 + k, parts - 1) * a.part_rows + rr) * (DH * 4) + d * 4), 0, CPOL_SC1));
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (s0 + k < parts) {
          const float f = part_factor(lds[(s0 + k) * rows + rr], mm);
          sum += lds[MERGE_ROWS + (s0 + k) * rows + rr] * f;
          o += v[k] * f;
        }
    }
    store_out(dst(rr) + d, normed(o, sum), o16);
  }
}

// ------------------------------------------------------------- few rows --

// The pages of a step's keys, in groups of 16, each of which lies in one page:
// looked up (look) a step before they are needed (use).  Pages that hold a
// whole step take one lookup and one address.
template <int SUBS>
struct Groups {
  static constexpr int N = 2 * SUBS;
  int raw[N], page[N], key0, have;  // have: bits of the groups whose page is there
  bool one;
  __device__ __forceinline__ void look(const KVView& kv, int seq, int key) {
    const kv_uniform_ints table = kv_uniform(kv.table + (long)seq * kv.max_pages);
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i == 0 || !one) raw[i] = table[min((key + 16 * i) >> kv.shift, kv.max_pages - 1)];
  }
  __device__ __forceinline__ void use(const KVView& kv, int key) {
    key0 = key;
    have = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (i && one) continue;
      const int p = __builtin_amdgcn_readfirstlane(raw[i]);
      const bool there = p >= 0 && p < kv.n_pages && (key + 16 * i) >> kv.shift < kv.max_pages;
      page[i] = there ? p : 0;
      have |= there ? (one ? (1 << N) - 1 : 1 << i) : 0;
    }
  }
  // f(i, where group i starts) in values of BYTES a token
  template <int BYTES, typename F>
  __device__ __forceinline__ void each(const KVView& kv, const char* base, int head, F f) const {
    const int slot = key0 & ((1 << kv.shift) - 1);
    if (one) {
      const char* p = base + kv_token(kv, page[0], head, slot) * BYTES;
#pragma unroll
      for (int i = 0; i < N; ++i) f(i, p + i * 16 * BYTES);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) f(i, base + kv_token(kv, page[i], head, (slot + 16 * i) & ((1 << kv.shift) - 1)) * BYTES);
    }
  }
  template <int DH, typename F>
  __device__ __forceinline__ void scales(const KVView& kv, const unsigned char* base, int head, F f) const {
    const int slot = key0 & ((1 << kv.shift) - 1);
    if (one) {
      const unsigned char* p = base + kv_scale(kv, page[0], head, slot, 0, DH / KV_BLOCK);
#pragma unroll
      for (int i = 0; i < N; ++i) f(i, p + i * 16);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) f(i, base + kv_scale(kv, page[i], head, (slot + 16 * i) & ((1 << kv.shift) - 1), 0, DH / KV_BLOCK));
    }
  }
};

// One step of a wave: SUBS * 32 keys in registers.  Lane (c = lane % 16, g =
// lane / 16).  Scores are S^T = K Q^T on 16x16 tiles (a lane: row c of 16, keys
// 4 g + r of each 16), which makes the weights the second operand of O^T = V^T
// P^T as they are: contraction slot (g, j) stands for key 4 g + j (j < 4) or 16
// + 4 g + j - 4 of 32.  V: a lane loads dims DH / 16 * c .. of those eight
// keys, whole rows by 16 lanes, and pairs of keys' values are put together
// dim by dim (frag): no LDS, no transposed copy.
template <int DH, int FORMAT, int SUBS>
struct Step;

// A lane's dims of its query row: eight for each product, product j those from
// 32 j + 8 g on (STRIDE 8, STEP 32) or from DH / 4 g + 8 j on (STRIDE DH / 4, STEP
// 8), as the keys' lanes have them.
template <int DH, int STRIDE, int STEP>
struct QueryRow {
  bf16x8 q[DH / 32];
  __device__ __forceinline__ void load(const bf16* p, bool aligned, bool live, int g) {
#pragma unroll
    for (int j = 0; j < DH / 32; ++j) q[j] = query(p + STRIDE * g + STEP * j, aligned, live);
  }
  __device__ __forceinline__ void convert(float sign) {
    if (sign == 1.f) return;
#pragma unroll
    for (int j = 0; j < DH / 32; ++j) q[j] = with_sign(q[j], sign);
  }
};

// bf16: K fragments straight from memory, a tile's 32 dims at a time.
template <int DH, int SUBS>
struct Step<DH, KV_BF16, SUBS> {
  static constexpr int WORDS = DH / 32;  // of a lane's dims of a value row
  typedef QueryRow<DH, 8, 32> Query;
  bf16x8 k[SUBS * 2][DH / 32];
  unsigned v[SUBS][8][WORDS];
  __device__ __forceinline__ void load_k(const Groups<SUBS>& gr, const KVView& kv, int head, int c, int g) {
    const unsigned at = c * (DH * 2) + g * 16;
    gr.template each<DH * 2>(kv, kv.k, head, [&](int i, const char* p) {
#pragma unroll
      for (int j = 0; j < DH / 32; ++j) k[i][j] = *reinterpret_cast<const bf16x8*>(p + (at + 64 * j));
    });
  }
  __device__ __forceinline__ void load_v(const Groups<SUBS>& gr, const KVView& kv, int head, int c, int g) {
    const unsigned at = g * (4 * DH * 2) + c * (DH / 8);
    gr.template each<DH * 2>(kv, kv.v, head, [&](int i, const char* p) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (DH == 128) {
          const u32x4 t = *reinterpret_cast<const u32x4*>(p + (at + j * DH * 2));
#pragma unroll
          for (int w = 0; w < WORDS; ++w) v[i >> 1][4 * (i & 1) + j][w] = t[w];
        } else {
          const u32x2 t = *reinterpret_cast<const u32x2*>(p + (at + j * DH * 2));
#pragma unroll
          for (int w = 0; w < WORDS; ++w) v[i >> 1][4 * (i & 1) + j][w] = t[w];
        }
      }
    });
  }
  __device__ __forceinline__ f32x4 scores(int i, const Query& q) const {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < DH / 32; ++j) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[i][j], q.q[j], s, 0, 0, 0);
    return s;
  }
  __device__ __forceinline__ void values(int b, unsigned (&out)[8][WORDS]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int w = 0; w < WORDS; ++w) out[j][w] = v[b][j][w];
  }
  // whether all values are known to be finite
  __device__ __forceinline__ bool finite() const { return false; }
};

// 4 bits: a lane loads dims DH / 4 g .. of key c, eight to a word, and turns each
// word to bf16 for its product.  (The scaled product takes 4-bit keys as they lie,
// but its other operand has 8 bits: a query row in two e4m3 parts under one scale
// is exact only for dims down to 2^-9 of its largest, and in three e5m2 parts down
// to 2^-23; the rest of a small dim is lost.  48 sequences of one row, 128 units
// of 32 rows and 64 of 35 take 103, 46 and 43.8 us with two parts, 117, 51 and 48.7
// with three and 100.5, 46.7 and 44.8 by conversion.)
template <int DH, int SUBS>
struct Step<DH, KV_FP4, SUBS> {
  static constexpr int WORDS = DH / 32;
  typedef QueryRow<DH, DH / 4, 8> Query;
  unsigned k[SUBS * 2][DH / 32];
  unsigned ks[SUBS * 2];
  unsigned v[SUBS][8];
  unsigned vs[SUBS][2];  // scales of four keys each
  __device__ __forceinline__ void load_k(const Groups<SUBS>& gr, const KVView& kv, int head, int c, int g) {
    const unsigned at = c * (DH / 2) + g * (DH / 8), sat = ((g * (DH / 4) / KV_BLOCK) << kv.shift) + c;
    gr.template each<DH / 2>(kv, kv.k, head, [&](int i, const char* p) {
      if constexpr (DH == 128) {
        const u32x4 t = *reinterpret_cast<const u32x4*>(p + at);
#pragma unroll
        for (int w = 0; w < 4; ++w) k[i][w] = t[w];
      } else {
        const u32x2 t = *reinterpret_cast<const u32x2*>(p + at);
        k[i][0] = t[0];
        k[i][1] = t[1];
      }
    });
    gr.template scales<DH>(kv, kv.ks, head, [&](int i, const unsigned char* p) { ks[i] = *(p + sat); });
  }
  __device__ __forceinline__ void load_v(const Groups<SUBS>& gr, const KVView& kv, int head, int c, int g) {
    const unsigned at = g * (2 * DH) + c * (DH / 32), sat = ((c * (DH / 16) / KV_BLOCK) << kv.shift) + 4 * g;
    gr.template each<DH / 2>(kv, kv.v, head, [&](int i, const char* p) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        v[i >> 1][4 * (i & 1) + j] = DH == 128 ? *reinterpret_cast<const unsigned*>(p + (at + j * (DH / 2)))
                                               : *reinterpret_cast<const unsigned short*>(p + (at + j * (DH / 2)));
    });
    gr.template scales<DH>(kv, kv.vs, head, [&](int i, const unsigned char* p) {
      vs[i >> 1][i & 1] = *reinterpret_cast<const unsigned*>(p + sat);
    });
  }
  __device__ __forceinline__ f32x4 scores(int i, const Query& q) const {
    const float scale = kv_scale_of(ks[i]);
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < DH / 32; ++j)
      s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kv_fp4_values(k[i][j], scale), q.q[j], s, 0, 0, 0);
    return s;
  }
  __device__ __forceinline__ void values(int b, unsigned (&out)[8][WORDS]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const unsigned w = vs[b][j >> 2];
      const float s = __uint_as_float((j & 3) == 3 ? w >> 1 : w << (23 - 8 * (j & 3)));  // its exponent is all that counts
      out[j][0] = kv_fp4_pair<0>(v[b][j], s);
      out[j][1] = kv_fp4_pair<1>(v[b][j], s);
      if constexpr (DH == 128) {
        out[j][2] = kv_fp4_pair<2>(v[b][j], s);
        out[j][3] = kv_fp4_pair<3>(v[b][j], s);
      }
    }
  }
  // by the scales: of less than 252, 2^125, no value is past bf16's range
  __device__ __forceinline__ bool finite() const {
    unsigned large = 0;  // the top bits of bytes of 252 and more
#pragma unroll
    for (int b = 0; b < SUBS; ++b)
#pragma unroll
      for (int h = 0; h < 2; ++h) large |= ((vs[b][h] & 0x7f7f7f7fu) + 0x04040404u) & vs[b][h];
    return !__any(large & 0x80808080u);
  }
};

// Row m of dim tile i stands for dim DH / 16 * m + i.
template <int WORDS>
__device__ __forceinline__ u32x4 frag(const unsigned (&val)[8][WORDS], int i) {
  u32x4 t;
#pragma unroll
  for (int w = 0; w < 4; ++w)
    t[w] = __builtin_amdgcn_perm(val[2 * w + 1][i >> 1], val[2 * w][i >> 1], i & 1 ? 0x07060302u : 0x05040100u);
  return t;
}

// Measured: 64 sequences of 6000 to 32000 keys, windows of 4096 (8 heads of 128,
// bf16) 192 us, 5.6 TB/s; 48 sequences of 1000 to 16000 4-bit keys 96 us, 4.6 TB/s;
// one of 131071 4-bit keys 36 us, 4.0 TB/s; one with 12 heads of 64 and a window of
// 128 keys 8 us (the launch, the lookups and one join).
//
// One unit = the rows of a sequence on one key head, FEW_ROWS at most.  The
// call's units, each so many key tiles long, lie one behind the other; the
// workgroups take equal stretches of the whole, so that long and short
// sequences load all CUs alike whatever their lengths.  A unit's rows are
// taken by groups of 16, each by its share of the workgroup's waves, which
// take the piece's tiles in turn, every wave with its own running maximum and
// sums; they are joined in LDS, and units that several workgroups hold a piece
// of in memory, by the last of them to arrive.  (Waves of 32 rows, which read a
// key half as often but whose sums leave no registers for loads ahead of the
// join: 32 units of 32 rows on up to 8000 bf16 keys 39.5 us for 33.5.)
// Tiles of a stretch at least: one a wave.  Of 2: 12 units of 132 keys 12.9 us for
// 10.6, 16 of 64 rows on 4-bit keys 40 for 36; of 32: 64 units of 35 rows on up to
// 7001 4-bit keys 67 us for 46.
constexpr int FEW_MIN_TILES = 8;
constexpr int FEW_ROWS = 64;

struct Unit {
  int seq, head, r0, toks, count;
  int sink, first;  // of its tiles (see Tiles)
  Range rg;
};

// A sequence's rows and keys as they are in memory.
struct Extent {
  int r0, n, len;
};

// A sequence's tiles of KEYS keys (0: it has no rows).
template <int KEYS>
__device__ __forceinline__ int few_tiles(const KVView& kv, const AttendArgs& a, const Extent& e, int* toks, Range* rg) {
  *toks = min(e.n, a.max_q);
  *rg = key_range(kv, e.len, e.n, 0, *toks, a.window, a.sinks);
  return e.r0 < 0 || *toks <= 0 || (long)e.r0 + *toks > kv.rows ? 0 : max(1, Tiles(*rg, KEYS).count);
}

__device__ __forceinline__ long uniform64(long v) {
  return (long)(((unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32) |
                (unsigned)__builtin_amdgcn_readfirstlane((int)v));
}

// n / d for 0 <= n < 2^52, d > 0
__device__ __forceinline__ long quotient(long n, long d) {
  long q = (long)((double)n / (double)d);
  if (q * d > n) --q;
  if ((q + 1) * d <= n) ++q;
  return uniform64(q);
}

// sum over the lanes up to this one
__device__ __forceinline__ unsigned sum_upto(unsigned v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // within rows of 16: from 1, 2, 4, 8 lanes below
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // last lanes of rows 0 and 2 to rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // lane 31 to rows 2 and 3
  return v;
}

template <int DH, int FORMAT, int SUBS, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void attend_few_kernel(KVView kv, AttendArgs a) {
  typedef Step<DH, FORMAT, SUBS> S;
  constexpr int KEYS = 32 * SUBS;
  constexpr int PITCH = DH + 4;
  constexpr int THREADS = 64 * WAVES;
  __shared__ __attribute__((aligned(16))) float lds[WAVES * 16 * PITCH];
  __shared__ float ms[WAVES][16], ls[WAVES][16];
  __shared__ unsigned notes[FEW_ROWS * (DH / 16)];
  __shared__ int arrived, noted;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
  const kv_uniform_ints starts = kv_uniform(kv.q_start), lens = kv_uniform(kv.kv_len);
  const bool pieces = a.part != nullptr;  // else whole units are dealt out
  const float sign = a.scale > 0.f ? 1.f : a.scale < 0.f ? -1.f : 0.f;
  const float cs = a.scale == 0.f ? 1.f : fabsf(a.scale) * LOG2E;
  const bool q16 = (((uintptr_t)a.q | (uintptr_t)(a.q_stride * 2)) & 15) == 0, o16 = ((uintptr_t)a.out & 15) == 0;

  // This workgroup's stretch [x, x_end) of the whole, and the sequence it
  // starts in, whose first unit's first tile is at `at`.  64 sequences at a
  // time, one a lane: first the sum of all, then the place of x in it.
  Unit un;
  un.seq = -1;
  auto weight = [&](int tiles) { return pieces ? tiles : min(tiles, 1); };
  auto take = [&](int seq, const Extent& e) {
    un.seq = seq;
    un.r0 = e.r0;
    un.count = few_tiles<KEYS>(kv, a, e, &un.toks, &un.rg);
    const Tiles tiles(un.rg, KEYS);
    un.sink = tiles.sink;
    un.first = tiles.first;
  };
  long x = 0, x_end = 0, at = 0, whole_tiles = 0, blocks = 0, each = 0;
  unsigned upto = 0, rest = 0;
  int some = 0, count = 0, chunk = 0, parts = 1, part = 0;
  auto border = [&](unsigned b) { return b * each + b * rest / (unsigned)blocks; };  // = whole_tiles * b / blocks
  Extent ext{0, 0, 0};
  if (kv.n_seq == 1) {
    take(0, Extent{starts[0], starts[1] - starts[0], lens[0]});
    whole_tiles = weight(un.count);
    some = un.count > 0;
  }
  for (int pass = kv.n_seq == 1; pass < 2; ++pass) {
    if (pass) {
      whole_tiles *= kv.kv_heads;
      const long busy = (long)some * kv.kv_heads;
      blocks = min((long)gridDim.x, pieces ? max((whole_tiles + FEW_MIN_TILES - 1) / FEW_MIN_TILES, busy) : busy);
      if (blocks == 0) return;
      each = quotient(whole_tiles, blocks);
      rest = (unsigned)(whole_tiles - each * blocks);
      const unsigned b = blockIdx.x;
      if (pieces && 2 * busy <= blocks && kv.n_seq <= 64) {
        // Few units: each is cut into equal parts of at most `chunk` tiles, one a workgroup, which then has one
        // piece and ends after it (128 units of 32 rows 49 us, by stretches 51; 64 units of one token 19, 25).
        for (int k = 0; k < 2; ++k) {
          chunk = (int)(k ? quotient(whole_tiles, blocks - busy) : each) + 1;
          if (k == 0 && rest == 0) --chunk;
          const int n = kv.n_seq == 1 ? un.count : lane < kv.n_seq ? count : 0;
          upto = (unsigned)(n + chunk - 1) / (unsigned)chunk;
          if (kv.n_seq > 1) upto = sum_upto(upto);
          x_end = (long)(unsigned)__builtin_amdgcn_readlane((int)upto, 63) * kv.kv_heads;
          if (x_end <= gridDim.x) break;
        }
        if (b >= x_end) return;
        x = b;
      } else {
        if (b >= blocks) return;
        x = border(b);
        x_end = border(b + 1);
      }
      if (kv.n_seq == 1) break;
    }
    long before = 0;
    for (int s0 = 0; s0 < kv.n_seq; s0 += 64) {
      if (pass == 0 || kv.n_seq > 64) {
        const int s = min(s0 + lane, kv.n_seq - 1), r1 = kv.q_start[s + 1];
        ext.r0 = kv.q_start[s];
        ext.n = r1 - ext.r0;
        ext.len = kv.kv_len[s];
        int toks;
        Range rg;
        count = few_tiles<KEYS>(kv, a, ext, &toks, &rg);
        upto = sum_upto(s0 + lane < kv.n_seq ? weight(count) : 0);
        some += pass ? 0 : __builtin_popcountll(__ballot(s0 + lane < kv.n_seq && count > 0));
      }
      const unsigned long long past = pass ? __ballot((before + upto) * kv.kv_heads > x) : 0;
      if (past) {
        const int k = __builtin_ctzll(past);
        at = (before + (k ? (unsigned)__builtin_amdgcn_readlane((int)upto, k - 1) : 0u)) * kv.kv_heads;
        take(s0 + k, Extent{__builtin_amdgcn_readlane(ext.r0, k), __builtin_amdgcn_readlane(ext.n, k),
                            __builtin_amdgcn_readlane(ext.len, k)});
        break;
      }
      before += (unsigned)__builtin_amdgcn_readlane((int)upto, 63);
    }
    if (pass == 0) whole_tiles = before;
  }
  if (un.seq < 0) return;  // (the lengths changed under the call)
  if (chunk) parts = (int)((unsigned)(un.count + chunk - 1) / (unsigned)chunk);
  const int step = chunk ? parts : weight(un.count);
  un.head = (int)((unsigned)(x - at) / (unsigned)step);
  at += (long)un.head * step;
  part = (int)(x - at);
  // A border within `near` tiles of a unit's end moves there: equal units that
  // miss the borders by a tile are not cut for it (64 equal windows on 512
  // workgroups: 200 -> 194 us).
  const int near = pieces && !chunk ? (int)min(each / 16, 4L) : 0;
  bool skip = false;  // the unit is left to the workgroup before
  if (near && part) {
    if (part <= near)
      part = 0;
    else if (un.count - part <= near)
      skip = true;
  }
  if (skip) at += un.count;

  int ta = 0, tb = 0;  // the piece of the unit: its tiles [ta, tb)
  S st;
  typename S::Query qf;
  int pos, low;  // of the lane's row
  // The waves of a unit: one, two or four groups of 16 rows, which take all of
  // the piece's tiles each; the `kw` waves of a group take them in turn.
  int kw, row_base, t_first;
  Groups<SUBS> gr;
  gr.one = (1 << kv.shift) >= KEYS;
  auto key_of = [&](int t) { return (t < un.sink ? t : un.first + t - un.sink) * KEYS; };
  // the first loads of a piece: its rows, and this wave's first tile
  auto begin = [&]() {
    const int rows = un.toks * a.group;
    const int group = rows <= 16 ? 0 : rows <= 32 ? wave / (WAVES / 2) : wave / (WAVES / 4);
    kw = rows <= 16 ? WAVES : rows <= 32 ? WAVES / 2 : WAVES / 4;
    row_base = 16 * group;
    t_first = row_base < rows ? ta + wave - group * kw : tb;
    if (t_first < tb) gr.look(kv, un.seq, key_of(t_first));
    const int r = row_base + c, tok = a.by_group.div(r), hd = r - tok * a.group;
    pos = un.rg.p0 + tok;
    low = window_start(pos, a.window);
    qf.load(a.q + (long)(un.r0 + tok) * a.q_stride + (long)(un.head * a.group + hd) * DH, q16, tok < un.toks, g);
    if (t_first < tb) {
      gr.use(kv, key_of(t_first));
      st.load_k(gr, kv, un.head, c, g);
      st.load_v(gr, kv, un.head, c, g);
      gr.look(kv, un.seq, key_of(min(t_first + kw, tb - 1)));
    }
    qf.convert(sign);
  };
  // A piece: its first loads are issued, then the sums of the one before are
  // joined while they fly, then its tiles are taken.
  f32x4 acc[DH / 16];
  float m, l;
  Unit done;
  int done_ta = 0, done_tb = 0, done_kw = 1, done_base = 0;
  long done_at = 0;
  bool first = true, more = true;
  const unsigned slot_bytes = (unsigned)a.part_rows * (DH + 2) * 4;
  const __amdgpu_buffer_rsrc_t room =
      __builtin_amdgcn_make_buffer_rsrc(pieces ? a.part : (float*)a.out, (short)0, pieces ? (int)(2 * gridDim.x * slot_bytes) : 0, 0x00020000);
  for (;;) {
    if (more) {
      const bool next = !first || skip;
      skip = false;
      if (next && ++un.head == kv.kv_heads) {
        un.head = 0;
        int s = un.seq;
        do {
          ++s;
          const int r0 = starts[s];
          take(s, Extent{r0, starts[s + 1] - r0, lens[s]});
        } while (un.count == 0 && s + 1 < kv.n_seq);
      }
      ta = next || !pieces ? 0 : chunk ? (int)((long)part * un.count / parts) : part;
      tb = un.count;
      if (chunk) {
        tb = (int)((long)(part + 1) * un.count / parts);
      } else if (pieces) {
        const long left = x_end - at;  // of the unit's tiles before the border
        if (left < un.count) {
          if (left <= near) more = false;
          if (un.count - left > near) tb = (int)left;
        }
      }
    }
    if (more) begin();
    if (!first) {
      const int rows = done.toks * a.group;
      const bool single = done_ta == 0 && done_tb == done.count;
      auto result = [&](int rr, int d) {
        const int tok = a.by_group.div(rr);
        return a.out + ((long)(done.r0 + tok) * a.heads + done.head * a.group + rr - tok * a.group) * DH + d;
      };
      // where workgroup b keeps its piece: the one it starts in (0) or the one it ends in (1)
      const unsigned mine = (2 * blockIdx.x + (done_ta == 0 ? 1 : 0)) * slot_bytes;
      const int ml_at = a.part_rows * DH * 4;
      const float sum_l = quad_sum(l);
      if (g == 0) {
        ms[wave][c] = m;
        ls[wave][c] = sum_l;
      }
      if (done_base + c < rows) {
        float* to = lds + (wave * 16 + c) * PITCH;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int i = 0; i < DH / 16; i += 4)
            *reinterpret_cast<f32x4*>(to + DH / 16 * (4 * g + r) + i) = f32x4{acc[i][r], acc[i + 1][r], acc[i + 2][r], acc[i + 3][r]};
      }
      __syncthreads();
      auto join = [&](auto waves) {
        constexpr int KW = decltype(waves)::value;
        for (int y = threadIdx.x; y < rows * (DH / 4); y += THREADS) {
          const int rr = y / (DH / 4), d = y % (DH / 4) * 4, s0 = rr / 16 * KW, row = rr % 16;
          float wm[KW], mm = -INFINITY, sum = 0.f;
#pragma unroll
          for (int w = 0; w < KW; ++w) {
            wm[w] = ms[s0 + w][row];
            mm = fmaxf(mm, wm[w]);
          }
          const float M = known(mm);
          f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int w = 0; w < KW; ++w) {
            const float f = exp2_fast(wm[w] - M);
            sum += ls[s0 + w][row] * f;
            o += *reinterpret_cast<const f32x4*>(lds + ((s0 + w) * 16 + row) * PITCH + d) * f;
          }
          if (noted) {
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += odd_of<DH>(notes, rr, d + e);
          }
          if (single) {
            store_out(result(rr, d), normed(o, sum), o16);
          } else {
            __builtin_amdgcn_raw_buffer_store_b128(o, room, (int)(mine + (rr * DH + d) * 4), 0, CPOL_SC1);
            if (d == 0) {
              const i32x2 ml = {(int)__float_as_uint(mm), (int)__float_as_uint(sum)};
              __builtin_amdgcn_raw_buffer_store_b64(ml, room, (int)(mine + ml_at + rr * 8), 0, CPOL_SC1);
            }
          }
        }
      };
      if (done_kw == WAVES)
        join(std::integral_constant<int, WAVES>());
      else if (done_kw == WAVES / 2)
        join(std::integral_constant<int, WAVES / 2>());
      else
        join(std::integral_constant<int, WAVES / 4>());
      __syncthreads();
      if (!single) {
        // the workgroups that hold a piece of this unit; the last of them to arrive joins the pieces, in order
        int b0 = blockIdx.x - part, b1 = b0 + parts - 1;
        if (!chunk) {
          const long end = done_at + done.count;
          b0 = (int)quotient((done_at + 1) * blocks - 1, whole_tiles);
          b1 = (int)quotient(end * blocks - 1, whole_tiles);
          if (border(b0 + 1) < end && border(b0 + 1) - done_at <= near) ++b0;
          if (border(b1) > done_at && border(b1) - done_at > near && end - border(b1) <= near) --b1;
        }
        const size_t unit = (size_t)done.seq * kv.kv_heads + done.head;
        wait_vmcnt<0>();
        __syncthreads();
        if (threadIdx.x == 0)
          arrived = (int)__hip_atomic_fetch_add(a.counters + unit, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (arrived == b1 - b0) {
          if (threadIdx.x == 0) __hip_atomic_store(a.counters + unit, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          // Four dims of a row a thread; where that leaves threads over, `groups` of them take every groups-th piece.
          const int shares = rows * (DH / 4), groups = max(1, min(THREADS / shares, 8));
          for (int y0 = 0; y0 < shares; y0 += THREADS) {
            const int group = groups == 1 ? 0 : threadIdx.x / shares, y = y0 + threadIdx.x - group * shares;
            const int rr = y / (DH / 4), d = y % (DH / 4) * 4;
            float pm = -INFINITY, pl = 0.f;
            f32x4 po = {0.f, 0.f, 0.f, 0.f};
            if (y < shares && group < groups)
              for (int b = b0 + group; b <= b1; b += 8 * groups) {  // eight pieces' loads in flight
                i32x2 ml[8];
                f32x4 v[8];
                float nm = pm;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                  const int bk = min(b + k * groups, b1);
                  const unsigned slot = (2 * bk + (bk == b0 ? 1 : 0)) * slot_bytes;
                  const auto t = __builtin_amdgcn_raw_buffer_load_b64(room, (int)(slot + ml_at + rr * 8), 0, CPOL_SC1);
                  ml[k] = i32x2{(int)t[0], (int)t[1]};
                  v[k] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(room, (int)(slot + (rr * DH + d) * 4), 0, CPOL_SC1));
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) nm = fmaxf(nm, __int_as_float(ml[k][0]));
                const float f = part_factor(pm, nm);
                pm = nm;
                pl *= f;
                po *= f;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                  if (b + k * groups > b1) continue;
                  const float h = part_factor(__int_as_float(ml[k][0]), nm);
                  pl += __int_as_float(ml[k][1]) * h;
                  po += v[k] * h;
                }
              }
            if (groups > 1) {
              if (group < groups) {
                float* to = lds + (group * shares + y) * 8;
                *reinterpret_cast<f32x4*>(to) = po;
                to[4] = pm;
                to[5] = pl;
              }
              __syncthreads();
              if (group == 0) {
                for (int k = 1; k < groups; ++k) {
                  const float* from = lds + (k * shares + y) * 8;
                  const float nm = fmaxf(pm, from[4]), f = part_factor(pm, nm), h = part_factor(from[4], nm);
                  pm = nm;
                  pl = pl * f + from[5] * h;
                  po = po * f + *reinterpret_cast<const f32x4*>(from) * h;
                }
              }
            }
            if (y < shares && group == 0) store_out(result(rr, d), normed(po, pl), o16);
          }
          __syncthreads();
        }
      }
    }
    if (!more) return;
    first = false;
    const Range rg = un.rg;
    const int rows = un.toks * a.group;
    if (threadIdx.x == 0) noted = 0;
    for (int y = threadIdx.x; y < rows * (DH / 16); y += THREADS) notes[y] = 0u;
    __syncthreads();
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int t = t_first; t < tb; t += kw) {
      const int key0 = key_of(t), have = gr.have;
      const bool whole = have == (1 << (SUBS * 2)) - 1 && key0 + KEYS - 1 <= rg.p0 && key0 + KEYS <= rg.end &&
                         (key0 >= rg.lo_last || key0 + KEYS <= rg.sinks);
      f32x4 s[SUBS * 2];
#pragma unroll
      for (int i = 0; i < SUBS * 2; ++i) s[i] = st.scores(i, qf);
      const bool more = t + kw < tb;
      if (more) {
        gr.use(kv, key_of(t + kw));
        st.load_k(gr, kv, un.head, c, g);
      }
      if (!whole) {
#pragma unroll
        for (int i = 0; i < SUBS * 2; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int j = key0 + 16 * i + 4 * g + r;
            const bool seen = (have >> i & 1) && j < rg.end && j <= pos && (j >= low || j < rg.sinks);
            s[i][r] = seen ? s[i][r] : -INFINITY;
          }
      }
      float mx = s[0][0];
#pragma unroll
      for (int i = 0; i < SUBS * 2; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[i][r]);
      mx = quad_max(mx) * cs;
      if (__any(mx > m + SLACK)) {
        const float nm = fmaxf(m, mx), f = exp2_fast(m - known(nm));
        m = nm;
        l *= f;
#pragma unroll
        for (int i = 0; i < DH / 16; ++i) acc[i] *= f;
      }
      const float ref = known(m);
      bf16x8 p[SUBS];
#pragma unroll
      for (int b = 0; b < SUBS; ++b) {
        float e[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          e[r] = exp2_fast(s[2 * b + (r >> 2)][r & 3] * cs - ref);
          l += e[r];
        }
        const u32x4 w = {pack_bf16x2(e[0], e[1]), pack_bf16x2(e[2], e[3]), pack_bf16x2(e[4], e[5]), pack_bf16x2(e[6], e[7])};
        p[b] = __builtin_bit_cast(bf16x8, w);
      }
      const bool plain = whole && st.finite();
#pragma unroll
      for (int b = 0; b < SUBS; ++b) {
        unsigned val[8][S::WORDS];
        st.values(b, val);
        if (!plain) {
          if (!whole) {
            // a value that no row sees counts nothing, whatever it is
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const int key = key0 + 32 * b + (j >> 2) * 16 + 4 * g + (j & 3);
              const bool seen = (have >> (2 * b + (j >> 2)) & 1) && key < rg.end && (key >= rg.lo_first || key < rg.sinks);
#pragma unroll
              for (int w = 0; w < S::WORDS; ++w) val[j][w] = seen ? val[j][w] : 0u;
            }
          }
          if (__any(not_finite(val))) {
            if (lane == 0) noted = 1;
            static_assert(64 * 8 * S::WORDS <= 16 * PITCH, "a wave's values fit where it leaves its sums");
            unsigned* mine = reinterpret_cast<unsigned*>(lds) + wave * (16 * PITCH) + lane * (8 * S::WORDS);
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
              for (int w = 0; w < S::WORDS; ++w) {
                mine[j * S::WORDS + w] = val[j][w];
                val[j][w] = without_odd(val[j][w]);
              }
#pragma unroll 1
            for (int y = 0; y < 8 * S::WORDS; ++y) {
              const int j = y / S::WORDS, key = key0 + 32 * b + (j >> 2) * 16 + 4 * g + (j & 3);
              note_odd<DH>(notes, mine[y], DH / 16 * c + 2 * (y % S::WORDS), rows, [&](int r) {
                const int pr = rg.p0 + a.by_group.div(r);
                return key <= pr && (key >= window_start(pr, a.window) || key < rg.sinks);
              });
            }
          }
        }
#pragma unroll
        for (int i = 0; i < DH / 16; ++i) {
          const bf16x8 f = __builtin_bit_cast(bf16x8, frag(val, i));
          acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, p[b], acc[i], 0, 0, 0);
        }
      }
      if (more) {
        st.load_v(gr, kv, un.head, c, g);
        gr.look(kv, un.seq, key_of(min(t + 2 * kw, tb - 1)));
      }
    }

    done = un;
    done_ta = ta;
    done_tb = tb;
    done_kw = kw;
    done_base = row_base;
    done_at = at;
    x = pieces ? at + tb : at + 1;
    at += weight(un.count);
    more = x < x_end && tb == un.count && !chunk;
  }
}

// ------------------------------------------------------------ many rows --

constexpr int TILE_ROWS = 128;  // (token, head of the group) rows of a workgroup, 32 a wave
constexpr int TILE_KEYS = 64;

// LDS place of 16-byte piece p of a key's row: pieces are exchanged so that the
// 32 rows (keys) or the 4 rows (values) that a read touches at once lie in
// different banks.
template <int DH>
__device__ __forceinline__ int k_piece(int key, int p) { return p ^ (DH == 128 ? key & 15 : (key >> 1) & 7); }
template <int DH>
__device__ __forceinline__ int v_piece(int key, int p) { return p ^ (DH == 128 ? 4 * (key & 3) : 4 * ((key >> 1) & 1)); }

// A tile of 64 keys, from the cache to LDS, 16 keys a wave (which lie in one
// page).  start() issues the loads, finish() ends with the wave's part in LDS.
// A page that is not there reads as zeros.  bf16: straight to LDS, 1 KB a load.
template <int DH, int FORMAT>
struct Loader;

template <int DH>
struct Loader<DH, KV_BF16> {
  static constexpr int LOADS = DH / 32;        // of 1 KB each, for 16 keys
  static constexpr int ROWS = 1024 / (DH * 2);  // keys of one load
  unsigned ko[LOADS], vo[LOADS];
  __device__ __forceinline__ Loader() {
    const int lane = threadIdx.x & 63, r = lane / (DH / 8), p = lane % (DH / 8);
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int key = j * ROWS + r;
      ko[j] = (unsigned)(key * DH * 2 + k_piece<DH>(key, p) * 16);
      vo[j] = (unsigned)(key * DH * 2 + v_piece<DH>(key, p) * 16);
    }
  }
  __device__ __forceinline__ void start(const KVView& kv, int page, int head, int slot, unsigned lds, int wave) {
    const long at = kv_token(kv, max(page, 0), head, slot) * (DH * 2);
    const unsigned bytes = page < 0 ? 0u : 16u * DH * 2;
    load_group<LOADS>(make_rsrc(kv.k + at, bytes), ko, lds + wave * 16 * DH * 2);
    load_group<LOADS>(make_rsrc(kv.v + at, bytes), vo, lds + (TILE_KEYS + wave * 16) * DH * 2);
  }
  __device__ __forceinline__ void finish(unsigned char*) { wait_vmcnt<0>(); }
};

// 4 bits: a quarter of a key and of a value a thread, to bf16 on the way.
template <int DH>
struct Loader<DH, KV_FP4> {
  static constexpr int WORDS = DH / 32;
  unsigned k[WORDS], v[WORDS];
  unsigned ks, vs;  // scale bytes
  bool there;
  __device__ __forceinline__ void start(const KVView& kv, int page, int head, int slot0, unsigned, int) {
    const int key = (threadIdx.x & 63) >> 2, b = threadIdx.x & 3;
    there = page >= 0;
    const char* pk = kv.k + kv_token(kv, max(page, 0), head, slot0) * (DH / 2);
    const char* pv = kv.v + kv_token(kv, max(page, 0), head, slot0) * (DH / 2);
    const long sc = kv_scale(kv, max(page, 0), head, slot0, 0, DH / KV_BLOCK);
    const unsigned at = key * (DH / 2) + b * (DH / 8), sat = ((DH == 128 ? b : b >> 1) << kv.shift) + key;
    if constexpr (DH == 128) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(pk + at), y = *reinterpret_cast<const u32x4*>(pv + at);
#pragma unroll
      for (int w = 0; w < WORDS; ++w) k[w] = x[w], v[w] = y[w];
    } else {
      const u32x2 x = *reinterpret_cast<const u32x2*>(pk + at), y = *reinterpret_cast<const u32x2*>(pv + at);
#pragma unroll
      for (int w = 0; w < WORDS; ++w) k[w] = x[w], v[w] = y[w];
    }
    ks = *(kv.ks + sc + sat);
    vs = *(kv.vs + sc + sat);
  }
  __device__ __forceinline__ void finish(unsigned char* lds) {
    const int key = threadIdx.x >> 2, b = threadIdx.x & 3;
    const float fk = kv_scale_of(ks), fv = kv_scale_of(vs);
    if (!there) {
#pragma unroll
      for (int w = 0; w < WORDS; ++w) k[w] = v[w] = 0u;  // (of a finite scale or not: not seen)
    }
    // Eight lanes (two keys) write at once: words are stored in an order that
    // differs between a key's halves, for values between the keys too, so that
    // the eight 16-byte pieces lie in different banks.
    const int ko = DH == 128 ? b & 2 : 0, vo = DH == 128 ? ko ^ (key & 1) : 0;
    turn(k, ko);
    turn(v, vo);
    unsigned char* at = lds + key * (DH * 2);
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
      *reinterpret_cast<bf16x8*>(at + k_piece<DH>(key, WORDS * b + (w ^ ko)) * 16) = kv_fp4_values(k[w], fk);
      *reinterpret_cast<bf16x8*>(at + TILE_KEYS * DH * 2 + v_piece<DH>(key, WORDS * b + (w ^ vo)) * 16) = kv_fp4_values(v[w], fv);
    }
  }
  // words w ^ by
  __device__ __forceinline__ static void turn(unsigned (&x)[WORDS], int by) {
    if constexpr (DH == 128) {
      const unsigned y[4] = {by & 1 ? x[1] : x[0], by & 1 ? x[0] : x[1], by & 1 ? x[3] : x[2], by & 1 ? x[2] : x[3]};
#pragma unroll
      for (int w = 0; w < 4; ++w) x[w] = by & 2 ? y[w ^ 2] : y[w];
    }
  }
};

// One unit = 128 rows of a sequence on one key head, 32 rows a wave; the four
// waves take the same 64 keys from LDS, the next 64 on their way meanwhile.
// Two workgroups a CU: one's products run while the other's weights (a maximum,
// exponentials and a sum) are computed.  For 128 dims a wave reads the tile's 32
// KB from LDS for 32 products of 32x32x16; 64 rows a wave would halve the reads,
// but their sums and scores spill, and two groups of waves half a tile apart
// took 355 us where this takes 308.  Bound by the vector work between the
// products.  Measured: one prompt of 8192 rows, windows of 2048, 32 heads of 128
// on 8: 284 us, 850 TFLOP/s of the pairs that are visible; 2 x 1024 rows on up to
// 16000 4-bit keys 546 us, 910 TFLOP/s.
template <int DH, int FORMAT>
__global__ __launch_bounds__(256, 2) void attend_tile_kernel(KVView kv, AttendArgs a) {
  constexpr int TILE_BYTES = TILE_KEYS * DH * 2;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * TILE_BYTES];  // K, V of two tiles
  __shared__ unsigned notes[TILE_ROWS * (DH / 16)];
  __shared__ int there[2][4];  // whether a tile's 16-key groups have a page
  __shared__ int arrived;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 31, h = lane >> 5;
  const int kvh = blockIdx.x % kv.kv_heads, tile = gridDim.x / kv.kv_heads - 1 - blockIdx.x / kv.kv_heads, split = blockIdx.y;

  // tiles of sequence s start at q_start[s] * group / TILE_ROWS + s: room for all of its rows before the next one's
  int seq = 0, left = kv.n_seq;
  auto base = [&](int s) { return (long)kv.q_start[s] * a.group / TILE_ROWS + s; };
  while (left > 1) {
    const int step = (left + 63) >> 6;
    const unsigned long long below = __ballot(lane * step < left && base(min(seq + lane * step, kv.n_seq - 1)) <= tile);
    const int k = below ? 63 - __builtin_clzll(below) : 0;
    seq += k * step;
    left = min(step, left - k * step);
  }
  seq = __builtin_amdgcn_readfirstlane(seq);
  const int r0 = kv.q_start[seq], n = kv.q_start[seq + 1] - r0, len = kv.kv_len[seq];
  const int toks = min(n, a.max_q);
  if (r0 < 0 || toks <= 0 || (long)r0 + toks > kv.rows) return;
  const long in_seq = tile - base(seq);
  const long total = (long)toks * a.group, row0 = in_seq * TILE_ROWS;
  if (in_seq < 0 || row0 >= total) return;
  const int rows = (int)min((long)TILE_ROWS, total - row0);
  const int tok0 = (int)(row0 / a.group), head0 = (int)(row0 - (long)tok0 * a.group);  // of the tile's first row
  auto token = [&](int r) { return a.by_group.div(head0 + r); };                           // after tok0
  const Range rg = key_range(kv, len, n, tok0, token(rows - 1) + 1, a.window, a.sinks);
  const Tiles tiles(rg, TILE_KEYS);
  const int parts = max(1, min(a.splits, (tiles.count + a.chunk - 1) / a.chunk));
  if (split >= parts) return;
  const int t0 = split * a.chunk, t_end = split == parts - 1 ? tiles.count : t0 + a.chunk;
  const float sign = a.scale > 0.f ? 1.f : a.scale < 0.f ? -1.f : 0.f;
  const float cs = a.scale == 0.f ? 1.f : fabsf(a.scale) * LOG2E;
  const bool q16 = (((uintptr_t)a.q | (uintptr_t)(a.q_stride * 2)) & 15) == 0, o16 = ((uintptr_t)a.out & 15) == 0;

  // the lane's row (past the end: the last one again), and those of the wave's first and last row
  const int row = min(wave * 32 + c, rows - 1);
  const int tok = token(row), first_tok = token(min(wave * 32, rows - 1)), last_tok = token(min(wave * 32 + 31, rows - 1));
  const int pos = rg.p0 + tok, low = window_start(pos, a.window);
  const int pos_first = rg.p0 + first_tok, pos_last = rg.p0 + last_tok;
  const int low_first = window_start(pos_first, a.window), low_last = window_start(pos_last, a.window);
  const long row_at = (long)(r0 + tok0 + tok), head = kvh * a.group + (head0 + row) - tok * a.group;
  bf16x8 qf[DH / 16];
#pragma unroll
  for (int j = 0; j < DH / 16; ++j) qf[j] = query(a.q + row_at * a.q_stride + head * DH + 16 * j + 8 * h, q16, true);
  if (sign != 1.f) {
#pragma unroll
    for (int j = 0; j < DH / 16; ++j) qf[j] = with_sign(qf[j], sign);
  }

  f32x16 acc[DH / 32];
  float m, l;
  bool careful = false;  // the second time: a sum was NaN
  for (int x = threadIdx.x; x < TILE_ROWS * (DH / 16); x += 256) notes[x] = 0u;

  Loader<DH, FORMAT> ld;
  const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_address(lds));
  // the page of this wave's 16 keys of a tile: looked up a tile before it is loaded
  const kv_uniform_ints table = kv_uniform(kv.table + (long)seq * kv.max_pages);
  int raw = 0;
  auto look = [&](int t) { raw = table[min((tiles[min(t, t_end - 1)] * TILE_KEYS + 16 * wave) >> kv.shift, kv.max_pages - 1)]; };
  auto load = [&](int t) {
    const int key = tiles[t] * TILE_KEYS + 16 * wave, p = __builtin_amdgcn_readfirstlane(raw);
    const int page = p >= 0 && p < kv.n_pages && key >> kv.shift < kv.max_pages ? p : -1;
    if (lane == 0) there[t & 1][wave] = page >= 0;
    ld.start(kv, page, kvh, key & ((1 << kv.shift) - 1), lds0 + ((t - t0) & 1 ? 2 * TILE_BYTES : 0), wave);
  };
  for (;;) {
#pragma unroll
    for (int i = 0; i < DH / 32; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][r] = 0.f;
    m = -INFINITY;
    l = 0.f;
    if (t0 < t_end) {
      look(t0);
      load(t0);
      look(t0 + 1);
    }
    for (int t = t0; t < t_end; ++t) {
      const int key0 = tiles[t] * TILE_KEYS;
      const unsigned buf = (t - t0) & 1 ? 2 * TILE_BYTES : 0;
      ld.finish(lds + buf);
      __syncthreads();  // the tile is in LDS; every wave is done with the one before, whose place the next one takes
      const int have = __builtin_amdgcn_readfirstlane(there[t & 1][0] | there[t & 1][1] << 1 | there[t & 1][2] << 2 | there[t & 1][3] << 3);
      if (t + 1 < t_end) {
        load(t + 1);
        look(t + 2);
      }
      unsigned char* K = lds + buf;
      unsigned char* V = K + TILE_BYTES;
      // values of 16 keys x: lanes of one half take keys 4 h + j and 8 + 4 h + j, dim 32 i + c
      auto value = [&](int i, int x) {
        u32x4 r;
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const int key = 16 * x + 8 * y + 4 * h + ((lane & 15) >> 2), piece = 4 * i + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
          const unsigned char* at = V + key * (DH * 2) + v_piece<DH>(key, piece) * 16 + (lane & 1) * 8;
          const auto w = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) s16x4*)(const __attribute__((address_space(3))) void*)at);
          const u32x2 d = __builtin_bit_cast(u32x2, w);
          r[2 * y] = d[0];
          r[2 * y + 1] = d[1];
        }
        return r;
      };
      if (careful || have != 15 || key0 + TILE_KEYS - 1 > rg.p0 || key0 + TILE_KEYS > rg.end ||
          (key0 < rg.lo_last && key0 + TILE_KEYS > rg.sinks)) {
        // Some rows do not see all of it: values that none sees become zero, whatever they are.
        constexpr int PER = DH / 4 / 8;  // 16-byte pieces of a thread: a quarter of a key
        const int key = threadIdx.x >> 2, j = key0 + key;
        const bool seen = (have >> (key >> 4) & 1) && j < rg.end && (j >= rg.lo_first || j < rg.sinks);
        u32x4* mine = reinterpret_cast<u32x4*>(V + key * (DH * 2)) + (threadIdx.x & 3) * PER;
        if (!seen) {
#pragma unroll
          for (int x = 0; x < PER; ++x) mine[x] = u32x4{0u, 0u, 0u, 0u};
        } else if (careful) {
#pragma unroll 1
          for (int x = 0; x < PER; ++x) {
            u32x4 w = mine[x];
            const int dim = 8 * v_piece<DH>(key, (threadIdx.x & 3) * PER + x);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              note_odd<DH>(notes, w[e], dim + 2 * e, rows, [&](int r) {
                const int pr = rg.p0 + token(r);
                return j <= pr && (j >= window_start(pr, a.window) || j < rg.sinks);
              });
              w[e] = without_odd(w[e]);
            }
            mine[x] = w;
          }
        }
        __syncthreads();
      }
      if (key0 <= pos_last && (key0 + TILE_KEYS > low_first || key0 < rg.sinks)) {
        f32x16 s[2];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[b][r] = 0.f;
#pragma unroll
        for (int j = 0; j < DH / 16; ++j)
#pragma unroll
          for (int b = 0; b < 2; ++b) {  // two sums in turn: neither waits for its last product
            const int key = 32 * b + c;
            const bf16x8 kf = *reinterpret_cast<const bf16x8*>(K + key * (DH * 2) + k_piece<DH>(key, 2 * j + h) * 16);
            s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[j], s[b], 0, 0, 0);
          }
        // eight reads ahead of the products (as the compiler orders them: 2-4% slower)
        __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
#pragma unroll
        for (int j = 0; j < DH / 8; ++j) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        const bool whole = have == 15 && key0 + TILE_KEYS - 1 <= pos_first && key0 + TILE_KEYS <= rg.end &&
                           (key0 >= low_last || key0 + TILE_KEYS <= rg.sinks);
        if (!whole) {
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int j = key0 + 32 * b + 8 * (r >> 2) + 4 * h + (r & 3);
              const bool seen = (have >> (2 * b + (r >> 3)) & 1) && j < rg.end && j <= pos && (j >= low || j < rg.sinks);
              s[b][r] = seen ? s[b][r] : -INFINITY;
            }
        }
        float mx = s[0][0];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[b][r]);
        mx = half_max(mx) * cs;
        if (__any(mx > m + SLACK)) {
          const float nm = fmaxf(m, mx), f = exp2_fast(m - known(nm));
          m = nm;
          l *= f;
#pragma unroll
          for (int i = 0; i < DH / 32; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][r] *= f;
        }
        const float ref = known(m);
        bf16x8 p[4];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            float e[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) {
              e[r] = exp2_fast(s[b][8 * x + r] * cs - ref);
              l += e[r];
            }
            const u32x4 w = {pack_bf16x2(e[0], e[1]), pack_bf16x2(e[2], e[3]), pack_bf16x2(e[4], e[5]), pack_bf16x2(e[6], e[7])};
            p[2 * b + x] = __builtin_bit_cast(bf16x8, w);
          }
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int i = 0; i < DH / 32; ++i)
            acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, value(i, x)), p[x], acc[i], 0, 0, 0);
      }
    }
    bool nan = false;
#pragma unroll
    for (int i = 0; i < DH / 32; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) nan |= acc[i][r] != acc[i][r];
    if (careful || !__syncthreads_or(nan)) break;
    careful = true;
  }

  if (careful) {
#pragma unroll
    for (int i = 0; i < DH / 32; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][r] += odd_of<DH>(notes, row, 32 * i + 8 * (r >> 2) + 4 * h + (r & 3));
  }
  l += __shfl_xor(l, 32, 64);
  const bool valid = wave * 32 + c < rows;
  if (parts == 1) {
    const float inv = 1.f / l;
    bf16* dst = a.out + (row_at * a.heads + head) * DH;
#pragma unroll
    for (int i = 0; i < DH / 32; ++i)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        // dims 16 x + 4 h .. and 16 x + 8 + 4 h ..: exchanged between the halves into eight in a row
        unsigned w[2][2];
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            w[y][e] = l == 0.f ? 0u : pack_bf16x2(acc[i][8 * x + 4 * y + 2 * e] * inv, acc[i][8 * x + 4 * y + 2 * e + 1] * inv);
        u32x4 o;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const auto z = __builtin_amdgcn_permlane32_swap(w[0][e], w[1][e], false, false);
          o[e] = z[0];
          o[2 + e] = z[1];
        }
        if (!valid) continue;
        bf16* to = dst + 32 * i + 16 * x + 8 * h;
        if (o16) {
          *reinterpret_cast<u32x4*>(to) = o;
        } else {
          const bf16x8 b = __builtin_bit_cast(bf16x8, o);
#pragma unroll
          for (int e = 0; e < 8; ++e) to[e] = b[e];
        }
      }
    return;
  }
  const size_t unit = (size_t)tile * kv.kv_heads + kvh;
  const size_t unit_floats = (size_t)a.splits * a.part_rows * (DH + 2);
  const __amdgpu_buffer_rsrc_t pr =
      __builtin_amdgcn_make_buffer_rsrc(a.part + unit * unit_floats, (short)0, (int)(unit_floats * 4), 0x00020000);
  if (valid) {
    const unsigned at = ((unsigned)split * a.part_rows + row) * (DH * 4) + 16 * h;
#pragma unroll
    for (int i = 0; i < DH / 32; ++i)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        __builtin_amdgcn_raw_buffer_store_b128(f32x4{acc[i][4 * x], acc[i][4 * x + 1], acc[i][4 * x + 2], acc[i][4 * x + 3]}, pr,
                                               (int)(at + (32 * i + 8 * x) * 4), 0, CPOL_SC1);
    if (h == 0) {
      const i32x2 ml = {__builtin_bit_cast(int, m), __builtin_bit_cast(int, l)};
      __builtin_amdgcn_raw_buffer_store_b64(ml, pr, (int)((unsigned)a.splits * a.part_rows * DH * 4 + ((unsigned)split * a.part_rows + row) * 8), 0, CPOL_SC1);
    }
  }
  join_parts<DH>(a, pr, unit, parts, rows, reinterpret_cast<float*>(lds), &arrived, [&](int rr) {
    const int k = token(rr);
    return a.out + ((long)(r0 + tok0 + k) * a.heads + kvh * a.group + head0 + rr - k * a.group) * DH;
  });
}

}  // namespace

// A call's launch.  few: workgroups that share all key tiles alike, or (no
// room for pieces) whole units; else tiles of 128 rows, their
// keys in `splits` parts of `chunk` tiles.  bytes: workspace used.
struct AttendPlan {
  bool few, pieces;
  int waves;
  long units;
  int blocks;
  int splits, chunk, part_rows;
  size_t bytes;
};

static AttendPlan attend_plan(int rows, int n_seq, int heads, int kv_heads, int dh, int format, int max_q, int max_kv, int window,
                              int sinks, int n_cu, size_t ws_bytes) {
  AttendPlan p{};
  const long group = heads / kv_heads, most = std::min(max_q, rows) * group;
  const size_t room = ws_bytes > COUNTERS * 4 ? ws_bytes - COUNTERS * 4 : 0;
  // Up to 32 rows a unit the few-row kernel: 128 units of 32 rows on up to 8000
  // 4-bit keys 48 us (by tiles 106), 32 units on bf16 keys 33 (41).  Up to 64
  // rows on 4-bit keys, which the tiles turn to bf16 for every wave alike: 48
  // rows 74 (127), 35 rows 46 (60); four groups of rows read bf16 keys four
  // times, 256 units of 64 rows 190 us (133).
  p.few = most <= (format == KV_FP4 ? FEW_ROWS : 32);
  if (p.few) {
    p.units = (long)n_seq * kv_heads;
    p.part_rows = (int)most;
    const size_t slots = 2 * (size_t)p.part_rows * (dh + 2) * 4;  // of a workgroup
    // Eight waves a workgroup join more of a unit in LDS and fewer pieces in
    // memory: 8 units of 131071 4-bit keys 34 us (four waves: 38), 64 units of 35
    // rows 46 (53).  Four leave less over between many units: 384 units 100 us
    // (eight: 113), 192 units 27 (32).
    p.waves = p.units <= n_cu / 4 ? 8 : 4;
    const long most_blocks = (long)n_cu * 8 / p.waves;  // two waves a SIMD
    const long whole = std::min(most_blocks, p.units), pieces = std::min<size_t>(room / slots, most_blocks);
    p.pieces = p.units <= COUNTERS && pieces >= whole && pieces > 0;
    p.blocks = (int)(p.pieces ? pieces : whole);
    p.splits = p.chunk = 1;
    p.bytes = p.pieces ? COUNTERS * 4 + slots * p.blocks : 0;
    return p;
  }
  p.units = ((long)rows * group / TILE_ROWS + n_seq) * kv_heads;
  p.part_rows = TILE_ROWS;
  // key tiles of the longest unit
  const long row_toks = std::min<long>(max_q, TILE_ROWS / group + 2);
  long tiles = ((long)max_kv + TILE_KEYS - 1) / TILE_KEYS;
  if (window)
    tiles = std::min(tiles, ((long)window + row_toks + TILE_KEYS - 2) / TILE_KEYS + 1 + ((long)sinks + TILE_KEYS - 1) / TILE_KEYS);
  tiles = std::max(tiles, 1L);
  long splits = 1;
  const size_t one = (size_t)p.units * p.part_rows * (dh + 2) * 4;
  if (p.units <= COUNTERS) {
    // Parts for one workgroup a CU where each keeps 8 tiles, for two where it
    // keeps 16: four chunks of 64 rows on 8192 4-bit keys 131 -> 94 us by the
    // second, 256 rows on 32768 keys 255 -> 187; but units of 19 tiles cut in
    // two 43 -> 53.
    splits = std::max(std::min(n_cu / p.units, tiles / 8), std::min(2 * n_cu / p.units, tiles / 16));
    splits = std::min(splits, (long)(MERGE_ROWS / p.part_rows));
    splits = std::max(1L, std::min(splits, (long)std::min<size_t>(room / one, MERGE_ROWS)));
  }
  p.chunk = (int)std::min<long>((tiles + splits - 1) / splits, INT_MAX);
  p.splits = (int)((tiles + p.chunk - 1) / p.chunk);
  p.bytes = p.splits > 1 ? COUNTERS * 4 + one * p.splits : 0;
  return p;
}

size_t attention_cache_workspace_bytes(int rows, int n_seq, int heads, int kv_heads, int dh, int max_q, int max_kv,
                                       int window, int sinks, int n_cu) {
  if (rows < 1 || n_seq < 1 || kv_heads < 1 || heads < 1 || heads % kv_heads || (dh != 64 && dh != 128) || max_q < 1 ||
      max_kv < 0 || window < 0 || sinks < 0)
    return 0;
  size_t most = 0;  // of both formats
  for (int f : {KV_BF16, KV_FP4})
    most = std::max(most, attend_plan(rows, n_seq, heads, kv_heads, dh, f, max_q, max_kv, window, sinks, n_cu, SIZE_MAX).bytes);
  return most;
}

template <int DH, int FORMAT, int WAVES>
static void attend_few_launch(const KVView& kv, const AttendArgs& a, const AttendPlan& p, hipStream_t st) {
  constexpr int SUBS = FORMAT == KV_FP4 || DH == 64 ? 2 : 1;
  launch(attend_few_kernel<DH, FORMAT, SUBS, WAVES>, dim3((unsigned)p.blocks), dim3(64 * WAVES), 0, st, kv, a);
}

template <int DH, int FORMAT>
static void attend_launch(const KVView& kv, const AttendArgs& a, const AttendPlan& p, hipStream_t st) {
  if (!p.few)
    launch(attend_tile_kernel<DH, FORMAT>, dim3((unsigned)p.units, (unsigned)p.splits), dim3(256), 0, st, kv, a);
  else if (p.waves == 4)
    attend_few_launch<DH, FORMAT, 4>(kv, a, p, st);
  else
    attend_few_launch<DH, FORMAT, 8>(kv, a, p, st);
}

dstack_status launch_attention_cache(const dstack_kv_cache* c, const dstack_kv_batch* b, const bf16* q,
                                     int64_t q_stride, int heads, int max_q, int max_kv, int window, int sinks,
                                     float scale, bf16* out, void* ws, size_t ws_bytes, int n_cu, hipStream_t st) {
  KVView kv;
  dstack_status s = kv_view(c, b, "attention_cache", &kv);
  if (s != DSTACK_OK) return s;
  DS_CHECK(q && out, DSTACK_E_INVALID, "attention_cache: null pointer");
  DS_CHECK(heads >= 1 && heads <= 65535 && heads % c->kv_heads == 0, DSTACK_E_INVALID,
           "attention_cache: heads must be a multiple of the cache's");
  DS_CHECK(q_stride >= (int64_t)heads * c->dh, DSTACK_E_INVALID, "attention_cache: rows shorter than their heads");
  DS_CHECK(max_q >= 1 && max_kv >= 0 && window >= 0 && sinks >= 0, DSTACK_E_INVALID,
           "attention_cache: max_q >= 1, max_kv, window and sinks >= 0");
  DS_CHECK(scale == 0.f || (std::fabs(scale) >= 0x1p-126f && std::fabs(scale) <= 0x1p126f), DSTACK_E_INVALID,
           "attention_cache: scale must be 0 or of magnitude 2^-126 to 2^126");
  DS_CHECK(((uintptr_t)q & 1) == 0 && ((uintptr_t)out & 1) == 0, DSTACK_E_INVALID,
           "attention_cache: misaligned pointer");
  DS_CHECK(((uintptr_t)ws & 255) == 0, DSTACK_E_INVALID, "attention_cache: workspace must be 256-byte aligned");
  const AttendPlan p = attend_plan(b->rows, b->n_seq, heads, c->kv_heads, c->dh, c->format, max_q, max_kv, window, sinks, n_cu,
                                   ws ? ws_bytes : 0);
  // a launch has fewer than 2^32 threads (few rows: at most two workgroups a CU)
  DS_CHECK(p.few || p.units < 1L << 24, DSTACK_E_UNSUPPORTED, "attention_cache: too many rows");
  char* base = static_cast<char*>(ws);
  const AttendArgs a{q, q_stride, out, p.bytes ? reinterpret_cast<float*>(base + COUNTERS * 4) : nullptr,
                     reinterpret_cast<unsigned*>(base), heads, heads / c->kv_heads, max_q, window, sinks,
                     FastDiv::make(heads / c->kv_heads), p.splits, p.chunk, p.part_rows, scale};
  if (c->dh == 64 && c->format == KV_BF16)
    attend_launch<64, KV_BF16>(kv, a, p, st);
  else if (c->dh == 64)
    attend_launch<64, KV_FP4>(kv, a, p, st);
  else if (c->format == KV_BF16)
    attend_launch<128, KV_BF16>(kv, a, p, st);
  else
    attend_launch<128, KV_FP4>(kv, a, p, st);
  DS_HIP(hipGetLastError());
  return DSTACK_OK;
}

}  // namespace dstack
