// The key/value cache of generating transformers: rows appended with their
// position rotation on the way, and read back.
//
// Append: y = x, its first `rot` dims turned by the position's angles: pairs
// (a, b) -> (a c - b s, a s + b c).  A product of a bf16 and an fp32 value is
// exact in fp64, so y is one rounding to 53 bits away from the formula, and is
// then rounded once to its place's type: through fp32 with the last bit made
// odd wherever that step was inexact, which leaves the final rounding what it
// would have been from 53 bits (Boldo & Melquiond, "When double rounding is
// odd", 2005).  The 4-bit block: amax = max |y| over 32 dims, scale 2^e with
// the least e for which amax <= 7 * 2^e: 7 is where rounding to 6 is off by
// half of the step below 6 and by half of what the next scale's step would be,
// so no value is off by more than 2^e (a scale of the power of two below
// amax / 4, the other common choice, is off by up to twice that at the top).
#include <algorithm>

#include "kv_cache.hpp"

namespace dstack {

namespace {

// fp32 with the last bit set where y is between two values of it
__device__ __forceinline__ float round_odd(double y) {
  const float f = (float)y;
  const double r = y - (double)f;
  unsigned b = __builtin_bit_cast(unsigned, f);
  if (fabs(r) > 0.0 && !(b & 1)) b += ((r > 0.0) == ((int)b >= 0)) ? 1u : (unsigned)-1;
  return __builtin_bit_cast(float, b);
}

// scale * y (scale 1/4 to 1) as round_odd gives it.  Where all are normal fp32
// numbers: the 23 leading bits of y's mantissa, the last one set where bits
// below them are, and the exponent moved; nine 32-bit operations a value in
// place of two conversions and a difference in 64 bits.
__device__ __forceinline__ void narrow(const double (&y)[8], float scale, float (&f)[8]) {
  constexpr unsigned LEAST = 0x38300000u, PAST = 0x47f00000u;  // high words of 2^-124 and 2^128
  unsigned far = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const unsigned long long b = __builtin_bit_cast(unsigned long long, y[e]);
    const unsigned hi = (unsigned)(b >> 32), lo = (unsigned)b;
    far = max(far, (hi & 0x7fffffffu) - LEAST);
    const unsigned m = __builtin_amdgcn_alignbit(hi, lo, 29) + 0x40000000u;  // exponent bias 1023 to 127
    const unsigned w = (m & 0x7fffffffu) | (hi & 0x80000000u) | min(lo << 3, 1u);
    f[e] = scale * __uint_as_float(w);
  }
  if (far >= PAST - LEAST) {  // a zero, a tiny or a huge value, an infinity or NaN among them
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = round_odd(scale * y[e]);
  }
}

// a c + b s in fp32, and whether its nearest bf16 value is that of the exact
// sum.  The sum r is off by half its last place and half that of the product p,
// together less than 1/2 + |p / r| of r's last places.  Its lower 16 bits are
// d such places from 2^15, where the rounding turns (at a power of two d / 2
// below it, where the places halve), so it is sure for (d - 1) / 2 > |p / r|;
// tiny, infinite and NaN sums are not.  Of 1024 values, as a wave has, one is
// unsure about one time in five.
__device__ __forceinline__ float turned_fast(float a, float c, float b, float s, bool& sure) {
  const float p = b * s, r = fmaf(a, c, p);
  const float far = (float)(int)((__float_as_uint(r) << 16) + 0x80000000u);  // 2^16 d
  sure &= fmaf(fmaf(fabsf(far), 0x1p-17f, -0.5f), fabsf(r), -fabsf(p)) > 0x1p-80f;
  return r;
}

struct AppendArgs {
  const bf16* qkv;
  long stride;
  const float* cs;
  bf16* q_out;
  int heads, table_len, rot, pairs;
};

// the eight values of dims d0 .. d0 + 7 of head row x at the position's angles
template <int DH>
__device__ __forceinline__ void rotated(const bf16* x, int d0, const float* cs, int rot, bool pairs, double (&y)[8]) {
  const int half = rot >> 1;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int d = d0 + e;
    double v = (double)(float)x[d];
    if (d < rot) {
      const bool low = pairs ? !(d & 1) : d < half;
      const int p = pairs ? d ^ 1 : (low ? d + half : d - half), i = pairs ? d >> 1 : (low ? d : d - half);
      const double c = cs[i], s = cs[half + i], w = (double)(float)x[p];
      v = low ? v * c - w * s : w * s + v * c;
    }
    y[e] = v;
  }
}

// The codes of eight values given as quarters f, of a block whose largest
// quarter is mx (infinite: the block is not finite), and the block's scale byte.
__device__ __forceinline__ unsigned fp4_words(const float (&f)[8], float mx, unsigned* byte) {
  const unsigned b = __builtin_bit_cast(unsigned, mx);
  // amax = 4 mx = 4 m 2^x, m in [1, 2): at most 7 * 2^e = 1.75 * 2^(e + 2) from e = x on, or x + 1 where m > 1.75
  const int ex = min(max((int)(b >> 23) - 127 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0), KV_MIN_EXP), 127);
  const bool bad = b >= 0x7f800000u;
  *byte = bad ? 255u : (unsigned)(ex + 127);
  // the quarters' scale; of the least one, which is no normal number, twice that and twice the values
  const float up = ex == KV_MIN_EXP ? 2.f : 1.f;
  const float s = __builtin_bit_cast(float, (unsigned)(max(bad ? 0 : ex, KV_MIN_EXP + 1) - 2 + 127) << 23);
  unsigned w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, up * f[0], up * f[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, up * f[2], up * f[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, up * f[4], up * f[5], s, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, up * f[6], up * f[7], s, 3);
  return bad ? 0u : w;
}

// Any rotation, strides and alignment: eight values a thread, element by
// element (16384 rows of 32 + 2 * 8 heads of 128 into 4 bits and back: 343 us
// with this one, 118 with the next).
template <int DH, int FORMAT>
__global__ __launch_bounds__(256) void kv_append_kernel(KVView kv, AppendArgs a) {
  const int row = blockIdx.x;
  const int seq = kv_find(kv.q_start, kv.n_seq, row);
  if (seq < 0) return;
  const int r0 = kv.q_start[seq], r1 = kv.q_start[seq + 1];
  const long pos = (long)kv.kv_len[seq] - ((long)r1 - r0) + (row - r0);
  if (pos < 0) return;
  const int page = kv_page(kv, seq, pos), slot = (int)(pos & ((1 << kv.shift) - 1));
  const int units = (a.heads + 2 * kv.kv_heads) * (DH / 8);
  const float* cs = a.cs + min(pos, (long)a.table_len - 1) * a.rot;
  // whole blocks of 32 dims stay together: units is a multiple of 4
  for (int u = threadIdx.x; u < units; u += 256) {
    const int head = u / (DH / 8), d0 = u % (DH / 8) * 8;
    const bool is_q = head < a.heads, is_k = !is_q && head < a.heads + kv.kv_heads;
    double y[8];
    rotated<DH>(a.qkv + (long)row * a.stride + head * DH, d0, cs, is_q || is_k ? a.rot : 0, a.pairs, y);
    if (is_q) {
      if (a.q_out)
        for (int e = 0; e < 8; ++e) a.q_out[((long)row * a.heads + head) * DH + d0 + e] = (bf16)round_odd(y[e]);
      continue;
    }
    const int h = head - a.heads - (is_k ? 0 : kv.kv_heads);
    char* dst = is_k ? kv.k : kv.v;
    if (FORMAT == KV_BF16) {
      if (page < 0) continue;
      bf16x8 o;
      for (int e = 0; e < 8; ++e) o[e] = (bf16)round_odd(y[e]);
      *reinterpret_cast<bf16x8*>(dst + (kv_token(kv, page, h, slot) * DH + d0) * 2) = o;
      continue;
    }
    // a quarter of y: a turned pair can pass fp32's largest value, and the largest scale's 7 * 2^127 is past it too
    float f[8], mx = 0.f;
    bool bad = false;
    for (int e = 0; e < 8; ++e) {
      f[e] = round_odd(0.25 * y[e]);
      bad |= !(fabs(y[e]) <= 1e300);
      mx = fmaxf(mx, fabsf(f[e]));
    }
    if (bad) mx = INFINITY;
    mx = fmaxf(mx, __shfl_xor(mx, 1, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 2, 64));
    if (page < 0) continue;
    unsigned byte;
    const unsigned w = fp4_words(f, mx, &byte);
    *reinterpret_cast<unsigned*>(dst + (kv_token(kv, page, h, slot) * DH + d0) / 2) = w;
    if ((u & 3) == 0)
      (is_k ? kv.ks : kv.vs)[kv_scale(kv, page, h, slot, d0 / KV_BLOCK, DH / KV_BLOCK)] =
          (unsigned char)byte;
  }
}

// The same, 16 values a thread in two 16-byte pieces: for halves the pair's
// dims d .. d + 7 and half + d .., else 16 dims in a row.  One workgroup a row;
// nothing a thread loads of its row waits for the row's sequence.  A block of
// 32 dims is four threads' pieces (halves) or two threads' (else).  Values that
// are rounded to bf16 are turned in fp32, and in fp64 where that is not sure.
// Registers for five waves a SIMD (six: 16384 rows alike, ragged prompts of 2199
// rows 12.9 -> 15.4 us; eight spill): the row's way through the lookups (its
// sequence, length, angles) is hidden only by other rows'.  Several rows a
// workgroup, the next one's loads ahead, took more registers than that gained
// (148 -> 165 us); all values in fp64 139 us where this takes 118 (append and
// read of 16384 rows of 32 + 2 * 8 heads of 128 into 4 bits).  Alone: those 95
// us, 3.7 TB/s; one row 3 us; 64 rows 5.2, of which 1.5 are the angles, whose load
// waits for the row's position (without rotation 3.7 us; into bf16 5.0 and 3.6).
template <int DH, int FORMAT>
__global__ __launch_bounds__(512, 5) void kv_append_vec_kernel(KVView kv, AppendArgs a) {
  const int row = blockIdx.x;
  const int units = (a.heads + 2 * kv.kv_heads) * (DH / 16), half = a.rot >> 1;
  // head, and first dims of the two pieces, of unit u
  auto dims = [&](int u, int& head, int& d0, int& d1, bool& turned, bool& split) {
    head = u / (DH / 16);
    const int piece = u % (DH / 16);
    turned = head < a.heads + kv.kv_heads && 16 * piece < a.rot;
    split = turned && !a.pairs;  // halves: units 0 .. half / 8 - 1 of a head are its turned dims
    d0 = split ? 8 * piece : 16 * piece;
    d1 = split ? half + d0 : d0 + 8;
  };
  int head, d0, d1;
  bool turned, split;
  bf16x8 in[2];
  auto load = [&]() {
    const bf16* x = a.qkv + (long)row * a.stride + (long)head * DH;
    in[0] = *reinterpret_cast<const bf16x8*>(x + d0);
    in[1] = *reinterpret_cast<const bf16x8*>(x + d1);
  };
  dims(min((int)threadIdx.x, units - 1), head, d0, d1, turned, split);
  load();
  const int seq = kv_find(kv.q_start, kv.n_seq, row);
  if (seq < 0) return;
  const int r0 = kv.q_start[seq], r1 = kv.q_start[seq + 1];
  const long pos = (long)kv.kv_len[seq] - ((long)r1 - r0) + (row - r0);
  if (pos < 0) return;
  const float* cs = a.cs + min(pos, (long)a.table_len - 1) * a.rot;
  const int page = kv_page(kv, seq, pos), slot = (int)(pos & ((1 << kv.shift) - 1));
  for (int u = threadIdx.x; u < units; u += blockDim.x) {
    if (u != (int)threadIdx.x) {
      dims(u, head, d0, d1, turned, split);
      load();
    }
    const bool is_q = head < a.heads, is_v = head >= a.heads + kv.kv_heads;
    if (is_q && !a.q_out) continue;
    const float scale = FORMAT == KV_FP4 && !is_q ? 0.25f : 1.f;  // of a 4-bit block: see above
    float f[2][8];
    if (turned) {
      // cosines and sines of the thread's pairs: (d0 + e, d1 + e) of halves, else neighbours
      float c[8], n[8];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (split || d0 + 8 * t < a.rot) {
          const float* at = cs + (split ? d0 : d0 >> 1) + 4 * t;
          const f32x4 cc = *reinterpret_cast<const f32x4*>(at), ss = *reinterpret_cast<const f32x4*>(at + half);
#pragma unroll
          for (int e = 0; e < 4; ++e) c[4 * t + e] = cc[e], n[4 * t + e] = ss[e];
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) c[4 * t + e] = 1.f, n[4 * t + e] = 0.f;
        }
      }
      // (pairs) values 2 e and 2 e + 1 of the thread's 16 are a pair; halves: e of each piece
      if (FORMAT == KV_BF16 || is_q) {
        bool sure = true;
        auto turn = [&](bf16 x, bf16 z, int e, float& lo, float& hi) {
          const float p = (float)x, q = (float)z;
          lo = turned_fast(p, c[e], -q, n[e], sure);
          hi = turned_fast(q, c[e], p, n[e], sure);
        };
        auto turn_exact = [&](bf16 x, bf16 z, int e, float& lo, float& hi) {
          const double p = (double)(float)x, q = (double)(float)z, cc = c[e], ss = n[e];
          lo = round_odd(p * cc - q * ss);
          hi = round_odd(p * ss + q * cc);
        };
        auto all = [&](auto f_pair) {
          if (split) {
#pragma unroll
            for (int e = 0; e < 8; ++e) f_pair(in[0][e], in[1][e], e, f[0][e], f[1][e]);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int t = e >> 2, d = 2 * (e & 3);
              f_pair(in[t][d], in[t][d + 1], e, f[t][d], f[t][d + 1]);
            }
          }
        };
        all(turn);
        if (!sure) {
          all(turn_exact);
          if (!split && d1 >= a.rot)  // not turned, whatever its neighbour is
#pragma unroll
            for (int e = 0; e < 8; ++e) f[1][e] = (float)in[1][e];
        }
      } else {
#pragma unroll
        for (int t = 0; t < 2; ++t) {  // four pairs at a time
          double y[8];
          float g[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p = (float)(split ? in[0][4 * t + e] : in[t][2 * e]), q = (float)(split ? in[1][4 * t + e] : in[t][2 * e + 1]);
            const double cc = c[4 * t + e], ss = n[4 * t + e], x = p, z = q;
            const bool turn = split || d0 + 8 * t < a.rot;
            y[2 * e] = turn ? x * cc - z * ss : x;
            y[2 * e + 1] = turn ? x * ss + z * cc : z;
          }
          narrow(y, scale, g);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (split) {
              f[0][4 * t + e] = g[2 * e];
              f[1][4 * t + e] = g[2 * e + 1];
            } else {
              f[t][2 * e] = g[2 * e];
              f[t][2 * e + 1] = g[2 * e + 1];
            }
          }
        }
      }
    } else {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 8; ++e) f[t][e] = scale * (float)in[t][e];
    }
    if (is_q || FORMAT == KV_BF16) {
      bf16x8 o[2];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 8; ++e) o[t][e] = (bf16)f[t][e];
      if (is_q) {
        bf16* dst = a.q_out + ((long)row * a.heads + head) * DH;
        *reinterpret_cast<bf16x8*>(dst + d0) = o[0];
        *reinterpret_cast<bf16x8*>(dst + d1) = o[1];
      } else if (page >= 0) {
        const int h = head - a.heads - (is_v ? kv.kv_heads : 0);
        bf16* dst = reinterpret_cast<bf16*>(is_v ? kv.v : kv.k) + kv_token(kv, page, h, slot) * DH;
        *reinterpret_cast<bf16x8*>(dst + d0) = o[0];
        *reinterpret_cast<bf16x8*>(dst + d1) = o[1];
      }
      continue;
    }
    float mx[2] = {0.f, 0.f};
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float odd = 0.f;  // NaN if a value is not finite
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        mx[t] = fmaxf(mx[t], fabsf(f[t][e]));
        odd = fmaf(f[t][e], 0.f, odd);
      }
      if (odd != 0.f) mx[t] = INFINITY;
    }
    if (!split) mx[0] = mx[1] = fmaxf(mx[0], mx[1]);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      mx[t] = fmaxf(mx[t], __shfl_xor(mx[t], 1, 64));
      const float o = __shfl_xor(mx[t], 2, 64);
      if (split) mx[t] = fmaxf(mx[t], o);
    }
    if (page < 0) continue;
    const int h = head - a.heads - (is_v ? kv.kv_heads : 0);
    char* dst = (is_v ? kv.v : kv.k) + kv_token(kv, page, h, slot) * (DH / 2);
    unsigned char* sc = is_v ? kv.vs : kv.ks;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      unsigned byte;
      const unsigned w = fp4_words(f[t], mx[t], &byte);
      const int d = t ? d1 : d0;
      *reinterpret_cast<unsigned*>(dst + d / 2) = w;
      if (d % KV_BLOCK == 0) sc[kv_scale(kv, page, h, slot, d / KV_BLOCK, DH / KV_BLOCK)] = (unsigned char)byte;
    }
  }
}

// Eight values a thread, one workgroup a row; bound by the bytes that it
// writes: 16384 rows of 2 * 8 heads of 128 from 4 bits 21 us, 4.0
// TB/s, from bf16 22.5 us, 6.0 TB/s.
template <int DH, int FORMAT>
__global__ __launch_bounds__(512) void kv_read_kernel(KVView kv, bf16* __restrict__ k_out, bf16* __restrict__ v_out,
                                                      bool vec) {
  const int row = blockIdx.x;
  const int seq = kv_find(kv.q_start, kv.n_seq, row);
  if (seq < 0) return;
  const int r0 = kv.q_start[seq], r1 = kv.q_start[seq + 1];
  const long pos = (long)kv.kv_len[seq] - ((long)r1 - r0) + (row - r0);
  const int page = kv_page(kv, seq, pos), slot = (int)(pos & ((1 << kv.shift) - 1));
  if (page < 0) return;
  const int units = 2 * kv.kv_heads * (DH / 8);
  for (int u = threadIdx.x; u < units; u += blockDim.x) {
    int h = u / (DH / 8);
    const int d0 = u % (DH / 8) * 8;
    const bool is_k = h < kv.kv_heads;
    h -= is_k ? 0 : kv.kv_heads;
    bf16* dst = (is_k ? k_out : v_out) + ((long)row * kv.kv_heads + h) * DH + d0;
    const char* src = is_k ? kv.k : kv.v;
    const long at = kv_token(kv, page, h, slot) * DH + d0;
    bf16x8 o;
    if (FORMAT == KV_BF16) {
      o = *reinterpret_cast<const bf16x8*>(src + at * 2);
    } else {
      const unsigned byte =
          (is_k ? kv.ks : kv.vs)[kv_scale(kv, page, h, slot, d0 / KV_BLOCK, DH / KV_BLOCK)];
      o = kv_fp4_values(*reinterpret_cast<const unsigned*>(src + at / 2), kv_scale_of(byte));
    }
    if (vec) {
      *reinterpret_cast<bf16x8*>(dst) = o;
    } else {
      for (int e = 0; e < 8; ++e) dst[e] = o[e];
    }
  }
}

// A launch has fewer than 2^32 threads.
bool fits(long blocks, unsigned threads) { return blocks * threads < 1L << 32; }

bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

}  // namespace

dstack_status kv_view(const dstack_kv_cache* c, const dstack_kv_batch* b, const char* who, KVView* out) {
  const std::string w(who);
  DS_CHECK(c && b, DSTACK_E_INVALID, w + ": null cache or batch");
  DS_CHECK(c->format == KV_BF16 || c->format == KV_FP4, DSTACK_E_UNSUPPORTED, w + ": format must be 0 (bf16) or 1 (fp4)");
  DS_CHECK(c->k && c->v && b->q_start && b->kv_len && b->page_table, DSTACK_E_INVALID, w + ": null pointer");
  DS_CHECK(c->format == KV_BF16 || (c->k_scale && c->v_scale), DSTACK_E_INVALID, w + ": an fp4 cache needs its scales");
  DS_CHECK(c->kv_heads >= 1 && c->n_pages >= 1 && c->page_size >= 1 && b->n_seq >= 1 && b->max_pages >= 1 &&
               b->rows >= 1,
           DSTACK_E_INVALID, w + ": bad shape");
  DS_CHECK(c->dh == 64 || c->dh == 128, DSTACK_E_UNSUPPORTED, w + ": head width 64 or 128");
  DS_CHECK(c->page_size >= 16 && c->page_size <= 1024 && (c->page_size & (c->page_size - 1)) == 0,
           DSTACK_E_UNSUPPORTED, w + ": a page holds 16, 32, ..., 1024 tokens");
  DS_CHECK(c->kv_heads <= 65535 && b->n_seq <= 65535, DSTACK_E_UNSUPPORTED, w + ": at most 65535 heads and sequences");
  DS_CHECK((int64_t)b->max_pages * c->page_size <= (1 << 30), DSTACK_E_UNSUPPORTED,
           w + ": a sequence's pages hold at most 2^30 tokens");
  DS_CHECK((__int128)c->n_pages * c->kv_heads * c->page_size <= UINT32_MAX, DSTACK_E_UNSUPPORTED,
           w + ": a cache holds fewer than 2^32 tokens of a head");
  DS_CHECK(aligned(c->k, 16) && aligned(c->v, 16) &&
               (c->format == KV_BF16 || (aligned(c->k_scale, 16) && aligned(c->v_scale, 16))),
           DSTACK_E_INVALID, w + ": the cache's tensors must be 16-byte aligned");
  DS_CHECK(aligned(b->q_start, 4) && aligned(b->kv_len, 4) && aligned(b->page_table, 4), DSTACK_E_INVALID,
           w + ": misaligned int32 pointer");
  out->k = static_cast<char*>(c->k);
  out->v = static_cast<char*>(c->v);
  out->ks = static_cast<unsigned char*>(c->k_scale);
  out->vs = static_cast<unsigned char*>(c->v_scale);
  out->q_start = b->q_start;
  out->kv_len = b->kv_len;
  out->table = b->page_table;
  out->n_pages = c->n_pages;
  out->kv_heads = c->kv_heads;
  out->shift = __builtin_ctz((unsigned)c->page_size);
  out->n_seq = b->n_seq;
  out->max_pages = b->max_pages;
  out->rows = b->rows;
  return DSTACK_OK;
}

dstack_status launch_kv_append(const dstack_kv_cache* c, const dstack_kv_batch* b, const bf16* qkv, int64_t stride,
                               int heads, const float* cs, int table_len, int rot, int pairs, bf16* q_out,
                               hipStream_t st) {
  KVView kv;
  dstack_status s = kv_view(c, b, "kv_append", &kv);
  if (s != DSTACK_OK) return s;
  DS_CHECK(qkv, DSTACK_E_INVALID, "kv_append: null pointer");
  DS_CHECK(heads >= 0 && heads <= 65535, DSTACK_E_INVALID, "kv_append: heads out of range");
  DS_CHECK(stride >= (int64_t)(heads + 2 * (int64_t)c->kv_heads) * c->dh, DSTACK_E_INVALID,
           "kv_append: rows shorter than their heads");
  DS_CHECK(cs ? rot >= 2 && rot % 2 == 0 && rot <= c->dh && table_len >= 1 : rot == 0, DSTACK_E_INVALID,
           "kv_append: an even rotation of at most the head's width with a table, none without");
  DS_CHECK(aligned(qkv, 2) && aligned(q_out, 2) && aligned(cs, 4), DSTACK_E_INVALID, "kv_append: misaligned pointer");
  const AppendArgs a{qkv, stride, cs, q_out, heads, table_len, rot, pairs};
  const bool vec = aligned(qkv, 16) && stride % 8 == 0 && aligned(q_out, 16) && aligned(cs, 16) &&
                   (pairs ? rot % 8 == 0 : rot % (c->format == KV_FP4 ? 64 : 16) == 0);
  const int units = (heads + 2 * c->kv_heads) * (c->dh / 16);
  const dim3 grid((unsigned)b->rows), block(vec ? (unsigned)std::min(512, (units + 63) / 64 * 64) : 256);
  DS_CHECK(fits(b->rows, block.x), DSTACK_E_UNSUPPORTED, "kv_append: too many rows");
  if (vec) {
    if (c->dh == 64 && c->format == KV_BF16)
      launch(kv_append_vec_kernel<64, KV_BF16>, grid, block, 0, st, kv, a);
    else if (c->dh == 64)
      launch(kv_append_vec_kernel<64, KV_FP4>, grid, block, 0, st, kv, a);
    else if (c->format == KV_BF16)
      launch(kv_append_vec_kernel<128, KV_BF16>, grid, block, 0, st, kv, a);
    else
      launch(kv_append_vec_kernel<128, KV_FP4>, grid, block, 0, st, kv, a);
  } else if (c->dh == 64 && c->format == KV_BF16) {
    launch(kv_append_kernel<64, KV_BF16>, grid, block, 0, st, kv, a);
  } else if (c->dh == 64) {
    launch(kv_append_kernel<64, KV_FP4>, grid, block, 0, st, kv, a);
  } else if (c->format == KV_BF16) {
    launch(kv_append_kernel<128, KV_BF16>, grid, block, 0, st, kv, a);
  } else {
    launch(kv_append_kernel<128, KV_FP4>, grid, block, 0, st, kv, a);
  }
  DS_HIP(hipGetLastError());
  return DSTACK_OK;
}

dstack_status launch_kv_read(const dstack_kv_cache* c, const dstack_kv_batch* b, bf16* k_out, bf16* v_out,
                             hipStream_t st) {
  KVView kv;
  dstack_status s = kv_view(c, b, "kv_read", &kv);
  if (s != DSTACK_OK) return s;
  DS_CHECK(k_out && v_out, DSTACK_E_INVALID, "kv_read: null pointer");
  DS_CHECK(aligned(k_out, 2) && aligned(v_out, 2), DSTACK_E_INVALID, "kv_read: misaligned pointer");
  const bool vec = aligned(k_out, 16) && aligned(v_out, 16);
  const dim3 grid((unsigned)b->rows), block((unsigned)std::min(512, (2 * c->kv_heads * (c->dh / 8) + 63) / 64 * 64));
  DS_CHECK(fits(b->rows, block.x), DSTACK_E_UNSUPPORTED, "kv_read: too many rows");
  if (c->dh == 64 && c->format == KV_BF16)
    launch(kv_read_kernel<64, KV_BF16>, grid, block, 0, st, kv, k_out, v_out, vec);
  else if (c->dh == 64)
    launch(kv_read_kernel<64, KV_FP4>, grid, block, 0, st, kv, k_out, v_out, vec);
  else if (c->format == KV_BF16)
    launch(kv_read_kernel<128, KV_BF16>, grid, block, 0, st, kv, k_out, v_out, vec);
  else
    launch(kv_read_kernel<128, KV_FP4>, grid, block, 0, st, kv, k_out, v_out, vec);
  DS_HIP(hipGetLastError());
  return DSTACK_OK;
}

}  // namespace dstack
