// oscar_q8_attn: attention from the new tokens over the paged 8-bit cache.
//
//   out[r] = sum_j exp(c <q_r, k_j> - m) v_j / sum_j exp(c <q_r, k_j> - m)     over positions j <= pos(r)
//
// in one pass over the cache, with a reference m that follows the largest logit.  A code is exact in bf16 and in
// fp16, so keys are multiplied as they are with queries as they are, and a block's scale (a power of two) goes
// onto its logits; value codes times their scale are exact in bf16.  Probabilities are rounded, to two bf16 limbs
// (2^-17), each a matrix product of its own: with one, 2^-9 a token would add to the output's own rounding.  With two, fp32 outputs over
// 1000 tokens are 6 .. 12 parts in 10^7 off, 3 .. 6 with probabilities of 24 bits; of 4096 rounded to bf16 0 .. 4 differ by it.
//
// A workgroup takes 16 or 32 rows (row = new token * g + query head of the group) of one kv head and a range of
// pages; of a page each of its four waves takes a step of 32 tokens.  S^T = K Q^T: a lane gets logits of tokens of
// one row, and these are, as they stand, its part of the operand of O^T = V^T P^T.  What is loaded lies one step
// ahead of its use, and logits are worked out a step ahead of their probabilities.  No barrier until the waves' sums
// are joined at the end.
//
// Up to 16 rows (a decoding step) take products of 16 x 16 x 32: the cache's bytes bound it (8 sequences of 32K: 82 us,
// 6.6 TB/s with the start, the end and the joining launch; a plain read of as many bytes takes 80).  More rows take products of
// 32 x 32 x 16 and are bound by issue: 172 vector instructions a step of 32 x 32 (64 conversions, 48 for limbs, 16
// exponentials) beside 24 products of 32 clocks, and the two hide little of each other: over pieces of up to 500 tokens the
// matrix cores are busy 37 % of the time and other vector instructions issued 43 % (8 sequences of 4100, 32 heads:
// 130 us, 565 TFLOP/s of the formula's products).  A product keeps vector instructions out for 8 clocks whatever
// its size (measured, of two waves side by side), which speaks for the larger one; two tiles of 16 x 16 x 32 took 1 .. 5 % more.
// Three waves a SIMD instead of two (queries in LDS) spill, four tiles of 16 rows leave one wave: 261 and 303 us where two
// took 232.  Scales through the lanes instead of scalar loads take 5 .. 25 % more.

#include <algorithm>

#include "oscar_q8.h"

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int O_PITCH = 132;       // of a row of sums in LDS: 16 rows' pieces on different banks
constexpr int V_PITCH = 264;       // bytes of a window row in LDS (a wave's 32 rows take the place of its 16 rows of sums)
static_assert(32 * V_PITCH <= 16 * O_PITCH * 4, "a wave's window rows fit its sums' place");
constexpr float NO_REF = -3e38f;   // reference of a row that has seen no token
// A reference moves when a logit passes it by this much (in powers of two): probabilities stay below 2^8, and a wave
// seldom has to multiply its sums.
constexpr float REF_SLACK = 8.0f;

struct AttnParams {
  Q8Cache c;
  Q8Rows r;
  const uint16_t* q;
  int64_t q_stride;
  void* out;
  float* ws;          // [sequence][new token][query head][split][130]: sums of values, sum and reference
  float scale_log2;   // of logits, in powers of two
  int hq, g, splits, row_blocks, out_f32;
};

__device__ __forceinline__ bf16x8 bf16_operand(u32x2 codes, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[0], scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[0], scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[1], scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[1], scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ f16x8 f16_operand(u32x2 codes) {
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes[0], 1.0f, false);
  const f16x2 b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes[0], 1.0f, true);
  const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes[1], 1.0f, false);
  const f16x2 d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes[1], 1.0f, true);
  return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Queries and keys are of the io type, everything else of the product is bf16.
template <bool F16> struct Io;
template <> struct Io<false> {
  using Op = bf16x8;
  static __device__ __forceinline__ Op keys(u32x2 codes) { return bf16_operand(codes, 1.0f); }
  static __device__ __forceinline__ f32x4 mul(Op a, Op b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ f32x16 mul32(Op a, Op b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Io<true> {
  using Op = f16x8;
  static __device__ __forceinline__ Op keys(u32x2 codes) { return f16_operand(codes); }
  static __device__ __forceinline__ f32x4 mul(Op a, Op b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ f32x16 mul32(Op a, Op b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

__device__ __forceinline__ f32x4 mul_bf16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ f32x16 mul32_bf16(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// An output as the io type holds it: values of an fp16 cache are up to 65536, which goes out as the largest fp16 number.
template <bool F16> __device__ __forceinline__ float io_number(float x) {
  return F16 ? __builtin_amdgcn_fmed3f(x, -65504.0f, 65504.0f) : x;
}
__device__ __forceinline__ uint32_t two_bf16(float a, float b) { return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b}); }

// ONCE: past the caches.
template <bool ONCE, typename T> __device__ __forceinline__ T fetch(const uint8_t* p) {
  return ONCE ? __builtin_nontemporal_load(reinterpret_cast<const T*>(p)) : *reinterpret_cast<const T*>(p);
}

// What a wave does with a step of 32 tokens, by the shape of its products.  LOGITS: of a lane; pairs of its
// probabilities make OPERANDS operands of the value products.  keys / values: raw pages' bytes as Q8_STEP_BYTES has
// them; window_keys: 16-bit keys at `row0`.
//
// 16 rows: lane 16 * q4 + n has row n and tokens 16 * (i / 4) + 4 * q4 + i % 4.
template <bool F16> struct Rows16 {
  using Op = typename Io<F16>::Op;
  using Acc = f32x4;
  using Logits = float[8];
  static constexpr int ROWS = 16, LOGITS = 8, KEYS = 4, TILES = 8, OPERANDS = 1;
  static __device__ __forceinline__ int row(int lane) { return lane & 15; }
  static __device__ __forceinline__ int token(int lane, int i) { return 16 * (i / 4) + 4 * (lane >> 4) + i % 4; }
  static __device__ __forceinline__ int channel(int lane, int tile, int i) { return 16 * tile + 4 * (lane >> 4) + i; }
  static __device__ __forceinline__ int query_channel(int lane, int kk) { return 64 * (kk / 2) + 16 * (lane >> 4) + 8 * (kk % 2); }
  static __device__ __forceinline__ float over_lanes(float x) {   // the largest of the lanes that share a row
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
  }
  static __device__ __forceinline__ float sum_lanes(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
  }
  static __device__ __forceinline__ void put(Logits& s, int tile, f32x4 x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) s[4 * tile + i] = x[i];
  }
  template <bool ONCE> static __device__ __forceinline__ void load_keys(const uint8_t* step, int lane, u32x4* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = fetch<ONCE, u32x4>(step + i * 1024 + lane * 16);
  }
  template <bool ONCE> static __device__ __forceinline__ void load_values(const uint8_t* step, int lane, u32x4* x) {
    load_keys<ONCE>(step, lane, x);
  }
  static __device__ __forceinline__ void keys(const u32x4* k, const Op* q, Logits& s) {
#pragma unroll
    for (int tile = 0; tile < 2; ++tile) {
      f32x4 x = {};
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        const u32x4 c = k[2 * tile + kk / 2];
        x = Io<F16>::mul(Io<F16>::keys(u32x2{c[2 * (kk % 2)], c[2 * (kk % 2) + 1]}), q[kk], x);
      }
      put(s, tile, x);
    }
  }
  static __device__ __forceinline__ void window_keys(const uint16_t* row0, int lane, const Op* q, Logits& s) {
#pragma unroll
    for (int tile = 0; tile < 2; ++tile) {
      const uint16_t* in = row0 + (16 * tile + (lane & 15)) * D;
      f32x4 x = {};
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
        x = Io<F16>::mul(__builtin_bit_cast(Op, *reinterpret_cast<const u32x4*>(in + query_channel(lane, kk))), q[kk], x);
      put(s, tile, x);
    }
  }
  static __device__ __forceinline__ bf16x8 operand(const uint32_t* pairs, int) {
    return __builtin_bit_cast(bf16x8, u32x4{pairs[0], pairs[1], pairs[2], pairs[3]});
  }
  static __device__ __forceinline__ void values(const u32x4* v, float scale, const bf16x8* hi, const bf16x8* lo, Acc* o) {
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const u32x4 x = v[c / 2];
      const bf16x8 val = bf16_operand(u32x2{x[2 * (c % 2)], x[2 * (c % 2) + 1]}, scale);
      o[c] = mul_bf16(val, lo[0], mul_bf16(val, hi[0], o[c]));
    }
  }
  static __device__ __forceinline__ Acc mul(bf16x8 a, bf16x8 b, Acc c) { return mul_bf16(a, b, c); }
  static __device__ __forceinline__ int value_channel(int lane, int tile) { return 16 * tile + (lane & 15); }
  static __device__ __forceinline__ int value_token(int lane, int, int i) { return token(lane, i); }
};

// 32 rows: lane 32 * g + n has row n and tokens 8 * (i / 4) + 4 * g + i % 4.  Lanes ask for the bytes of their own token (of
// their own channel, 8 at a time), in stretches of 256 bytes; as they lie, 24 exchanges between lanes a step take 5 % of the time.
template <bool F16> struct Rows32 {
  using Op = typename Io<F16>::Op;
  using Acc = f32x16;
  using Logits = f32x16;
  static constexpr int ROWS = 32, LOGITS = 16, KEYS = 8, TILES = 4, OPERANDS = 2;
  static __device__ __forceinline__ int row(int lane) { return lane & 31; }
  static __device__ __forceinline__ int token(int lane, int i) { return 8 * (i / 4) + 4 * (lane >> 5) + i % 4; }
  static __device__ __forceinline__ int channel(int lane, int tile, int i) { return 32 * tile + 8 * (i / 4) + 4 * (lane >> 5) + i % 4; }
  // product kk: half of the channels kk / 4, even or odd sixteens of it kk / 2 % 2, eight of those kk % 2
  static __device__ __forceinline__ int query_channel(int lane, int kk) {
    return 64 * (kk / 4) + 16 * (2 * (lane >> 5) + kk / 2 % 2) + 8 * (kk % 2);
  }
  static __device__ __forceinline__ float over_lanes(float x) { return fmaxf(x, __shfl_xor(x, 32)); }
  static __device__ __forceinline__ float sum_lanes(float x) { return x + __shfl_xor(x, 32); }
  template <bool ONCE> static __device__ __forceinline__ void load_keys(const uint8_t* step, int lane, u32x4* x) {
    const uint8_t* in = step + (lane >> 4 & 1) * 2048 + (lane >> 5) * 512 + (lane & 15) * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = fetch<ONCE, u32x4>(in + (i & 1) * 1024 + (i >> 1) * 256);   // half i % 2 of the channels
  }
  template <bool ONCE> static __device__ __forceinline__ void load_values(const uint8_t* step, int lane, u32x4* x) {
    const uint8_t* in = step + (lane >> 5) * 256 + (lane & 15) * 16 + (lane >> 4 & 1) * 8;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const u32x2 a = fetch<ONCE, u32x2>(in + c * 1024), b = fetch<ONCE, u32x2>(in + c * 1024 + 512);
      x[c] = u32x4{a[0], a[1], b[0], b[1]};
    }
  }
  static __device__ __forceinline__ void keys(const u32x4* k, const Op* q, Logits& s) {
    f32x16 x = {};
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        const u32x4 c = k[half + kk / 2 * 2];
        x = Io<F16>::mul32(Io<F16>::keys(u32x2{c[2 * (kk % 2)], c[2 * (kk % 2) + 1]}), q[4 * half + kk], x);
      }
    }
    s = x;
  }
  static __device__ __forceinline__ void window_keys(const uint16_t* row0, int lane, const Op* q, Logits& s) {
    const uint16_t* in = row0 + (lane & 31) * D;
    f32x16 x = {};
#pragma unroll
    for (int kk = 0; kk < 8; ++kk)
      x = Io<F16>::mul32(__builtin_bit_cast(Op, *reinterpret_cast<const u32x4*>(in + query_channel(lane, kk))), q[kk], x);
    s = x;
  }
  // product j of the values takes the tokens of quarters g (j = 0) and 2 + g (j = 1) of a page's step
  static __device__ __forceinline__ bf16x8 operand(const uint32_t* pairs, int j) {
    return __builtin_bit_cast(bf16x8, u32x4{pairs[2 * j], pairs[2 * j + 1], pairs[4 + 2 * j], pairs[5 + 2 * j]});
  }
  static __device__ __forceinline__ void values(const u32x4* v, float scale, const bf16x8* hi, const bf16x8* lo, Acc* o) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {   // (a sum's products lie four apart)
      bf16x8 val[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c] = mul32_bf16(val[c] = bf16_operand(u32x2{v[c][2 * j], v[c][2 * j + 1]}, scale), hi[j], o[c]);
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c] = mul32_bf16(val[c], lo[j], o[c]);
    }
  }
  static __device__ __forceinline__ Acc mul(bf16x8 a, bf16x8 b, Acc c) { return mul32_bf16(a, b, c); }
  static __device__ __forceinline__ int value_channel(int lane, int tile) { return 32 * tile + (lane & 31); }
  static __device__ __forceinline__ int value_token(int lane, int j, int i) { return token(lane, 4 * j + i + (i / 4) * 4); }
};

// A wave's rows: queries, sums of values (transposed), sum and reference.
template <class S> struct State {
  typename S::Op q[S::KEYS];
  typename S::Acc o[S::TILES];
  float sum, ref;        // sum: of the lane's own tokens
  int pos;               // the lane's row's position, -1: no row
  int min_pos, max_pos;  // of the rows there are
};

// Logits of tokens that a row does not see, of a step from t0 on: from `limit` on, or behind the row's own.
template <class S> __device__ __forceinline__ void hide(const State<S>& w, typename S::Logits& s, int t0, int lane, int limit) {
  const int last = min(w.pos, limit - 1) - t0;
#pragma unroll
  for (int i = 0; i < S::LOGITS; ++i) s[i] = S::token(lane, i) <= last ? s[i] : -INFINITY;
}
// The reference follows the step's largest logit, all sums with it.
template <class S> __device__ __forceinline__ void move_reference(State<S>& w, const typename S::Logits& s, float scale) {
  float top = s[0];
#pragma unroll
  for (int i = 1; i < S::LOGITS; ++i) top = fmaxf(top, s[i]);
  top *= scale;
  if (!__any(top > w.ref + REF_SLACK)) return;
  const float ref = fmaxf(w.ref, S::over_lanes(top));
  const float f = __builtin_amdgcn_exp2f(w.ref - ref);
  w.ref = ref;
  w.sum *= f;
#pragma unroll
  for (int c = 0; c < S::TILES; ++c) w.o[c] *= f;
}
// Probabilities, two limbs of the operands.  (The product is not rounded before the reference, which was taken from a
// rounded one, is subtracted: all powers of a row may be off by the same half step, which is less than 2^6 for logits below 2^30.)
template <class S> __device__ __forceinline__ void probabilities(State<S>& w, const typename S::Logits& s, float scale, bf16x8* hi, bf16x8* lo) {
  uint32_t h[S::LOGITS / 2], l[S::LOGITS / 2];
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < S::LOGITS / 2; ++i) {   // (two at a time: the conversion takes two)
    const float a = __builtin_amdgcn_exp2f(fmaf(s[2 * i], scale, -w.ref)), b = __builtin_amdgcn_exp2f(fmaf(s[2 * i + 1], scale, -w.ref));
    sum += a + b;
    h[i] = two_bf16(a, b);
    asm("" : "+v"(h[i]));   // (else what is taken from it is converted once more)
    l[i] = two_bf16(a - __uint_as_float(h[i] << 16), b - __uint_as_float(h[i] & 0xffff0000u));
  }
  w.sum += sum;
#pragma unroll
  for (int j = 0; j < S::OPERANDS; ++j) hi[j] = S::operand(h, j), lo[j] = S::operand(l, j);
}

__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Where the waves' sums meet, 16 rows at a time.
struct __align__(16) Joined {
  float o[4][16 * O_PITCH];
  float sum[4][32], ref[4][32];
};

// The rows from row0 on (of a sequence and kv head) over the pages of a split, by a workgroup.
// ONCE: no other workgroup reads these pages, and they are asked for past the caches (caches of 1 GB in all, one after the
// other: 1 x 1000 tokens 15.1 -> 12.9 us, 8 x 4000 21.1 -> 18.7, 8 x 32K 95 -> 82, with 32 rows 115 -> 102; the same cache
// again and again, 8 x 4000, 18.4 -> 19.0; pages that several blocks of rows read, 35 rows over 128K, 39 -> 44)
template <bool F16, class S, bool ONCE>
__device__ __forceinline__ void attend(const AttnParams& P, const Q8Seq& seq, int b, int h, int split, int row0, Joined& J) {
  using Op = typename S::Op;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rows = seq.n * P.g;
  State<S> w;
  w.min_pos = seq.old + row0 / P.g;
  w.max_pos = seq.old + (min(row0 + S::ROWS, rows) - 1) / P.g;
  {
    const int row = row0 + S::row(lane), t = row / P.g;
    const int64_t at = seq.row + t;
    const bool is = row < rows && at >= 0 && at < P.r.n_rows;
    w.pos = is ? seq.old + t : -1;
    const uint16_t* q = P.q + at * P.q_stride + (h * P.g + row % P.g) * D;
#pragma unroll
    for (int kk = 0; kk < S::KEYS; ++kk) {
      u32x4 x = {};
      if (is) x = *reinterpret_cast<const u32x4*>(q + S::query_channel(lane, kk));
      w.q[kk] = __builtin_bit_cast(Op, x);
    }
    w.sum = 0.0f;
    w.ref = NO_REF;
#pragma unroll
    for (int c = 0; c < S::TILES; ++c) w.o[c] = typename S::Acc{};
  }

  // pages of whole blocks, and the window behind them
  const int coded = seq.len / P.c.block * P.c.block;
  const int end = min(coded, w.max_pos + 1);                 // tokens of pages that some row sees
  const int pages = min(max(end + R - 1, 0) / R, P.c.max_pages);
  const int per = (pages + P.splits - 1) / P.splits;
  const int p0 = min(split * per, pages), p1 = min(p0 + per, pages);
  const int per_page = R / P.c.block;
  const int32_t* table = P.c.table + (int64_t)b * P.c.max_pages;

  u32x4 k[4] = {}, v[4] = {};
  float ks = 1.0f, vs = 1.0f;
  // (no less than the smallest number: hidden logits times 0 are none)
  const auto logit_scale = [&](float block) { return fmaxf(block * P.scale_log2, 0x1p-126f); };
  const auto page_of = [&](int p) -> int {
    if (p >= p1 || p * R + wave * Q8_STEP_TOKENS >= end) return -1;
    const int page = __builtin_amdgcn_readfirstlane(table[p]);
    return (uint32_t)page < (uint32_t)P.c.num_pages ? page : -1;
  };
  const auto load_keys = [&](int page, u32x4* x, float& scale) {
    if (page < 0) return;
    const int64_t at = (int64_t)page * P.c.heads + h;
    S::template load_keys<ONCE>(P.c.k_codes + at * Q8_PAGE_BYTES + wave * Q8_STEP_BYTES, lane, x);
    scale = P.c.k_scales[at * per_page + wave * Q8_STEP_TOKENS / P.c.block];
  };
  const auto load_values = [&](int page, u32x4* x, float& scale) {
    if (page < 0) return;
    const int64_t at = (int64_t)page * P.c.heads + h;
    S::template load_values<ONCE>(P.c.v_codes + at * Q8_PAGE_BYTES + wave * Q8_STEP_BYTES, lane, x);
    scale = P.c.v_scales[at * per_page + wave * Q8_STEP_TOKENS / P.c.block];
  };

  int page = page_of(p0), next = page_of(p0 + 1);
  if (p0 < p1) {
    load_keys(page, k, ks);
    load_values(page, v, vs);
  }

  // the window, its steps by the last split's waves, while the first pages are on their way
  if (split == P.splits - 1) {
    const int64_t win = ((int64_t)b * P.c.heads + h) * (2 * P.c.block * D);
    const int stop = min(seq.len, w.max_pos + 1);
    for (int t0 = coded + wave * Q8_STEP_TOKENS; t0 < stop; t0 += 4 * Q8_STEP_TOKENS) {
      const int slot = t0 % (2 * P.c.block);   // (a step does not wrap)
      // values go through LDS, because an operand wants 8 tokens of a channel in a lane; what no token owns becomes zero
      u32x4 rows_v[8];
      uint8_t* tile_v = reinterpret_cast<uint8_t*>(J.o[wave]);
      const int tr = lane >> 4, tc = lane & 15;
#pragma unroll
      for (int i = 0; i < 8; ++i) rows_v[i] = *reinterpret_cast<const u32x4*>(P.c.win_v + win + (slot + 4 * i + tr) * D + 8 * tc);
      typename S::Logits s;
      S::window_keys(P.c.win_k + win + slot * D, lane, w.q, s);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const u32x4 x = t0 + 4 * i + tr < stop ? rows_v[i] : u32x4{};
        u32x2* to = reinterpret_cast<u32x2*>(tile_v + (4 * i + tr) * V_PITCH + 16 * tc);
        to[0] = u32x2{x[0], x[1]};
        to[1] = u32x2{x[2], x[3]};
      }
      wave_fence();
      hide(w, s, t0, lane, stop);
      move_reference(w, s, P.scale_log2);
      bf16x8 hi[S::OPERANDS], lo[S::OPERANDS];
      probabilities(w, s, P.scale_log2, hi, lo);
#pragma unroll
      for (int c = 0; c < S::TILES; ++c)
#pragma unroll
        for (int j = 0; j < S::OPERANDS; ++j) {
          bf16x8 val, rest;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const uint16_t x = *reinterpret_cast<const uint16_t*>(tile_v + S::value_token(lane, j, i) * V_PITCH + 2 * S::value_channel(lane, c));
            if constexpr (F16) {   // 11 bits in two limbs, each by both of the probabilities'
              const float f = (float)__builtin_bit_cast(_Float16, x);
              val[i] = (__bf16)f;
              rest[i] = (__bf16)(f - (float)val[i]);
            } else {
              val[i] = __builtin_bit_cast(__bf16, x);
            }
          }
          w.o[c] = S::mul(val, lo[j], S::mul(val, hi[j], w.o[c]));
          if constexpr (F16) w.o[c] = S::mul(rest, lo[j], S::mul(rest, hi[j], w.o[c]));
        }
      wave_fence();
    }
  }

  typename S::Logits s = {};
  if (p0 < p1) S::keys(k, w.q, s);
  float scale = logit_scale(ks);
  load_keys(next, k, ks);
  for (int p = p0; p < p1; ++p) {
    const int after = page_of(p + 2);
    const int t0 = p * R + wave * Q8_STEP_TOKENS;
    if (page < 0 || t0 + Q8_STEP_TOKENS - 1 > w.min_pos) {
      hide(w, s, t0, lane, page < 0 ? 0 : end);
      if (page < 0)   // (what stands for a page's values must be numbers)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = u32x4{};
    }
    move_reference(w, s, scale);
    bf16x8 hi[S::OPERANDS], lo[S::OPERANDS];
    probabilities(w, s, scale, hi, lo);
    S::keys(k, w.q, s);
    scale = logit_scale(ks);
    S::values(v, vs, hi, lo, w.o);
    load_keys(after, k, ks);
    load_values(next, v, vs);
    page = next;
    next = after;
  }

  // the four waves' sums
  w.sum = S::sum_lanes(w.sum);
  if (lane < S::ROWS) J.sum[wave][lane] = w.sum, J.ref[wave][lane] = w.ref;
#pragma unroll
  for (int r = 0; r < S::ROWS; r += 16) {
    if (r > 0) __syncthreads();
    if (S::ROWS == 16 || (S::row(lane) & 16) == r) {
      constexpr int NUMBERS = sizeof(typename S::Acc) / 4;
#pragma unroll
      for (int c = 0; c < S::TILES; ++c)
#pragma unroll
        for (int i = 0; i < NUMBERS; i += 4)
          *reinterpret_cast<f32x4*>(&J.o[wave][(S::row(lane) & 15) * O_PITCH + S::channel(lane, c, i)]) =
              f32x4{w.o[c][i], w.o[c][i + 1], w.o[c][i + 2], w.o[c][i + 3]};
    }
    __syncthreads();
    const int j = tid >> 4, row = row0 + r + j, t = row / P.g;
    const int64_t at = seq.row + t;
    if (row < rows && at >= 0 && at < P.r.n_rows) {
      float ref = NO_REF, sum = 0.0f, x[8] = {};
#pragma unroll
      for (int i = 0; i < 4; ++i) ref = fmaxf(ref, J.ref[i][r + j]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float f = __builtin_amdgcn_exp2f(J.ref[i][r + j] - ref);
        sum += f * J.sum[i][r + j];
        const f32x4 *o = reinterpret_cast<const f32x4*>(&J.o[i][j * O_PITCH + (tid & 15) * 8]), first = o[0], last = o[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] += f * first[e], x[4 + e] += f * last[e];
      }
      const int head = h * P.g + row % P.g, c0 = (tid & 15) * 8;
      if (P.splits == 1) {
        const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= inv;
        const int64_t to = (at * P.hq + head) * D + c0;
        if (P.out_f32) {
          float* out = reinterpret_cast<float*>(P.out) + to;
          *reinterpret_cast<f32x4*>(out) = f32x4{x[0], x[1], x[2], x[3]};
          *reinterpret_cast<f32x4*>(out + 4) = f32x4{x[4], x[5], x[6], x[7]};
        } else {
          Op y;
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = io_number<F16>(x[e]);
          *reinterpret_cast<Op*>(reinterpret_cast<uint16_t*>(P.out) + to) = y;
        }
      } else {
        float* ws = P.ws + ((((int64_t)b * P.r.T + t) * P.hq + head) * P.splits + split) * 130;
#pragma unroll
        for (int e = 0; e < 8; e += 2) *reinterpret_cast<float2*>(ws + c0 + e) = make_float2(x[e], x[e + 1]);
        if (c0 == 0) *reinterpret_cast<float2*>(ws + 128) = make_float2(sum, ref);
      }
    }
  }
}

// F16: the io type; ROWS: of a workgroup; ONCE: one workgroup has all of a sequence's rows.
template <bool F16, int ROWS, bool ONCE> __global__ __launch_bounds__(256, 2) void oscar_q8_attn_kernel(AttnParams P) {
  __shared__ Joined J;
  // row blocks of one range of pages lie on one die of eight, next to each other; the ranges that are left over when every
  // die has as many share the dies (300 rows x 2 kv heads over 30000: on two dies 549 us, on all 150)
  uint32_t id = blockIdx.x;
  int rb = 0;
  if (!ONCE) {
    const uint32_t units = (uint32_t)P.c.batch * P.c.heads * P.splits, even = units / 8 * 8, blocks = P.row_blocks;
    if (id < even * blocks) {
      const uint32_t group = id / (8 * blocks), in = id % (8 * blocks);
      rb = in / 8;
      id = group * 8 + in % 8;
    } else {
      const uint32_t rest = (units - even) * blocks, in = id - even * blocks, at = in % 8 * ((rest + 7) / 8) + in / 8;
      if (at >= rest) return;
      rb = at % blocks;
      id = even + at / blocks;
    }
    rb = P.row_blocks - 1 - rb;   // (the last rows see the most)
  }
  const int split = id % P.splits;
  id /= P.splits;
  const int h = id % P.c.heads, b = id / P.c.heads;
  if (b >= P.c.batch) return;
  const Q8Seq seq = q8_seq(P.r, b);
  const int row0 = rb * ROWS, left = seq.n * P.g - row0;
  if (left <= 0) return;
  if (left <= 16)   // (all, or a sequence's last rows)
    attend<F16, Rows16<F16>, ONCE>(P, seq, b, h, split, row0, J);
  else if constexpr (ROWS == 32)
    attend<F16, Rows32<F16>, ONCE>(P, seq, b, h, split, row0, J);
}

// Joins the splits of a row and query head: a workgroup, each wave a quarter of the splits.
template <bool F16> __global__ __launch_bounds__(256) void oscar_q8_join_kernel(AttnParams P) {
  __shared__ float2 s_o[4][64];
  __shared__ float s_ref[4], s_sum[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t unit = blockIdx.x;   // [sequence][new token][head]
  const int head = unit % P.hq, t = unit / P.hq % P.r.T;
  const int64_t b = unit / P.hq / P.r.T;
  const Q8Seq s = q8_seq(P.r, b);
  const int64_t at = s.row + t;
  if (t >= s.n || at < 0 || at >= P.r.n_rows) return;
  const int per = (P.splits + 3) / 4, i0 = wave * per, i1 = min(i0 + per, P.splits);
  const float* ws = P.ws + unit * P.splits * 130;
  // statistics of up to 64 splits a round, then their sums
  float ref = NO_REF, sum = 0.0f, x = 0.0f, y = 0.0f;
  for (int c0 = i0; c0 < i1; c0 += 64) {
    const float2 st = c0 + lane < i1 ? *reinterpret_cast<const float2*>(ws + (c0 + lane) * 130 + 128) : make_float2(0.0f, NO_REF);
    float top = st.y;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    top = fmaxf(top, ref);
    const float back = __builtin_amdgcn_exp2f(ref - top), f = __builtin_amdgcn_exp2f(st.y - top);
    ref = top;
    float part = f * st.x;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) part += __shfl_xor(part, d);
    sum = sum * back + part;
    x *= back, y *= back;
    const int n = min(i1 - c0, 64);
    for (int j = 0; j < n; j += 16) {   // (16 loads on the way at a time; what is past the end weighs nothing)
      float2 o[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) o[i] = *reinterpret_cast<const float2*>(ws + (c0 + min(j + i, n - 1)) * 130 + 2 * lane);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float g = j + i < n ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), j + i)) : 0.0f;
        x += g * o[i].x;
        y += g * o[i].y;
      }
    }
  }
  s_o[wave][lane] = make_float2(x, y);
  if (lane == 0) s_ref[wave] = ref, s_sum[wave] = sum;
  __syncthreads();
  if (wave > 0) return;
  ref = fmaxf(fmaxf(s_ref[0], s_ref[1]), fmaxf(s_ref[2], s_ref[3]));
  sum = x = y = 0.0f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float f = __builtin_amdgcn_exp2f(s_ref[w] - ref);
    sum += f * s_sum[w];
    x += f * s_o[w][lane].x;
    y += f * s_o[w][lane].y;
  }
  const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
  x *= inv, y *= inv;
  const int64_t to = (at * P.hq + head) * D + 2 * lane;
  if (P.out_f32) {
    *reinterpret_cast<float2*>(reinterpret_cast<float*>(P.out) + to) = make_float2(x, y);
  } else if constexpr (F16) {
    *reinterpret_cast<f16x2*>(reinterpret_cast<uint16_t*>(P.out) + to) = f16x2{(_Float16)io_number<F16>(x), (_Float16)io_number<F16>(y)};
  } else {
    *reinterpret_cast<bf16x2*>(reinterpret_cast<uint16_t*>(P.out) + to) = bf16x2{(__bf16)x, (__bf16)y};
  }
}

// Rows of a workgroup.
int rows_of(int64_t rows) { return rows <= 16 ? 16 : 32; }

template <bool F16> void launch(const AttnParams& P, int block_rows, uint32_t grid, hipStream_t st) {
  if (block_rows == 16)
    hipLaunchKernelGGL((oscar_q8_attn_kernel<F16, 16, true>), dim3(grid), dim3(256), 0, st, P);
  else if (P.row_blocks == 1)
    hipLaunchKernelGGL((oscar_q8_attn_kernel<F16, 32, true>), dim3(grid), dim3(256), 0, st, P);
  else
    hipLaunchKernelGGL((oscar_q8_attn_kernel<F16, 32, false>), dim3(grid), dim3(256), 0, st, P);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool heads_fit(const oscar_q8_cache* c, int32_t hq) {
  return hq >= 1 && hq % c->n_kv_heads == 0 && hq / c->n_kv_heads <= OSCAR_Q8_MAX_GROUP;
}

}  // namespace

extern "C" int32_t oscar_q8_auto_splits(const oscar_q8_cache* cache, int32_t n_q_heads, int32_t T, int32_t max_seq_len) {
  if (oscar_check_q8_sizes(cache) != OSCAR_OK || !heads_fit(cache, n_q_heads) || T < 1 || max_seq_len < 1) return 1;
  const int64_t rows = (int64_t)T * (n_q_heads / cache->n_kv_heads);
  const int block = rows_of(rows);
  const int64_t units = (int64_t)cache->batch * cache->n_kv_heads * ((rows + block - 1) / block);
  const int64_t pages = ((int64_t)max_seq_len + OSCAR_R - 1) / OSCAR_R;
  const int64_t cus = oscar_compute_units();
  // The one that takes least.  16 rows read: a page of a split takes 0.75 us, and more workgroups than compute units do not
  // read faster (8 sequences of 32K, 4 / 8 splits 82 / 86 us).  32 rows compute: a page takes 1.05 us, of each of two
  // workgroups that share a unit 2 * 0.88.  The joining launch takes 5.5 us (3.5 of them on the GPU), a row's sums of a split
  // 0.5 ns.  One row over 1000, 8 / 1 splits: 10.1 / 10.9 us of graph, 12.4 / 10.9 of calls; 8 rows of 8 sequences over 1000,
  // 8 / 1 splits 20.4 / 14.4; 35 rows over 128K, 32 / 64 45.6 / 37.9; 700 of 2 sequences over 54539, 1 / 4 443 / 286.
  const double row_us = 0.0005 * (double)cache->batch * T * n_q_heads;
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>({block == 16 ? cus / units : 4 * cus / units, pages, 512}));
  int64_t best = 1;
  double least = 0.0;
  for (int64_t s = 1; s <= most; ++s) {
    const int64_t rounds = block == 16 ? 1 : (units * s + cus - 1) / cus, share = (pages + s - 1) / s;
    double us = (double)(rounds * share) * (block == 16 ? 0.75 : rounds == 1 ? 1.05 : rounds == 2 ? 0.88 : 0.9);
    if (s > 1) us = 1.07 * (us + 5.5 + row_us * (double)s);   // (one split unless several gain a little)
    if (s == 1 || us < least) best = s, least = us;
  }
  return (int32_t)best;
}

extern "C" size_t oscar_q8_workspace_bytes(const oscar_q8_cache* cache, int32_t n_q_heads, int32_t T, int32_t num_splits) {
  if (oscar_check_q8_sizes(cache) != OSCAR_OK || !heads_fit(cache, n_q_heads) || T < 1 || num_splits <= 1) return 0;
  return (size_t)cache->batch * T * n_q_heads * num_splits * 130 * sizeof(float);
}

extern "C" int oscar_q8_attn(const void* q, int64_t q_stride, int64_t n_rows, int32_t n_q_heads, int32_t T,
                             const int32_t* row_starts, const int32_t* new_lens, const int32_t* lens,
                             const oscar_q8_cache* cache, void* out, int32_t out_dtype, float softmax_scale,
                             int32_t max_seq_len_hint, int32_t num_splits, void* workspace, size_t workspace_bytes,
                             void* stream) {
  const int rc = oscar_check_q8_cache(cache);
  if (rc != OSCAR_OK) return rc;
  if (n_q_heads < 1 || n_q_heads % cache->n_kv_heads != 0) return OSCAR_ERR_INVALID_ARG;
  if (!heads_fit(cache, n_q_heads)) return OSCAR_ERR_UNSUPPORTED;
  if (out_dtype != OSCAR_F32 && out_dtype != cache->io_dtype) return OSCAR_ERR_INVALID_ARG;
  if (T < 0 || n_rows < 0 || max_seq_len_hint < 0 || num_splits < 0 || num_splits > 512) return OSCAR_ERR_INVALID_ARG;
  if (T == 0 || n_rows == 0) return OSCAR_OK;
  if (!q || !lens || !out || !aligned16(q) || !aligned16(out)) return OSCAR_ERR_INVALID_ARG;
  if (q_stride < (int64_t)n_q_heads * OSCAR_D || q_stride % 8 != 0) return OSCAR_ERR_INVALID_ARG;
  const int splits = num_splits ? num_splits : oscar_q8_auto_splits(cache, n_q_heads, T, max_seq_len_hint);
  const int g = n_q_heads / cache->n_kv_heads;
  const int64_t rows = (int64_t)T * g;
  if (rows > INT32_MAX / 2) return OSCAR_ERR_INVALID_ARG;
  const int block = rows_of(rows);
  const int64_t row_blocks = (rows + block - 1) / block, units = (int64_t)cache->batch * cache->n_kv_heads * splits;
  const int64_t grid = row_blocks == 1 ? units : (units * row_blocks + 7) / 8 * 8;
  const int64_t join = (int64_t)cache->batch * T * n_q_heads;
  // a grid's threads are counted in 32 bits
  if (row_blocks > INT32_MAX / 8 || grid * 256 > UINT32_MAX || (splits > 1 && join * 256 > UINT32_MAX)) return OSCAR_ERR_INVALID_ARG;
  if (splits > 1 && (!workspace || !aligned16(workspace) || workspace_bytes < oscar_q8_workspace_bytes(cache, n_q_heads, T, splits)))
    return OSCAR_ERR_WORKSPACE;
  AttnParams P = {};
  P.c = q8_device_view(cache);
  P.r = {row_starts, new_lens, lens, T, n_rows};
  P.q = reinterpret_cast<const uint16_t*>(q);
  P.q_stride = q_stride;
  P.out = out;
  P.ws = reinterpret_cast<float*>(workspace);
  P.scale_log2 = (softmax_scale > 0.0f ? softmax_scale : 0.08838834764831845f) * 1.4426950408889634f;
  P.hq = n_q_heads;
  P.g = g;
  P.splits = splits;
  P.row_blocks = (int)row_blocks;
  P.out_f32 = out_dtype == OSCAR_F32;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const bool f16 = cache->io_dtype == OSCAR_F16;
  f16 ? launch<true>(P, block, (uint32_t)grid, st) : launch<false>(P, block, (uint32_t)grid, st);
  if (splits > 1) {
    if (f16)
      hipLaunchKernelGGL((oscar_q8_join_kernel<true>), dim3((uint32_t)join), dim3(256), 0, st, P);
    else
      hipLaunchKernelGGL((oscar_q8_join_kernel<false>), dim3((uint32_t)join), dim3(256), 0, st, P);
  }
  if (hipGetLastError() != hipSuccess) return OSCAR_ERR_HIP;
  return OSCAR_OK;
}
