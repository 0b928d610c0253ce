// oscar_rope: rotary positions on queries and keys, with up to four position axes.
//
// Pair i of a vector (channels i and i + r/2, or 2i and 2i + 1) turns by the angle
//   a = position[axis(i)][token] * inv_freq[i],   y1 = x1 cos a - x2 sin a,   y2 = x2 cos a + x1 sin a.
// The angle is worked out in 64 bits and their rest: the product of a 32-bit position and a 24-bit frequency has up to
// 56 bits, 1 / 2 pi is held to 106, and of turns the fraction counts, to 2^-52 at any position (in 64 bits alone the
// largest ones were off by 3e-7).  Sine and cosine are 64-bit series about the nearest quarter turn, rounded once to
// 32 bits: the turn's own roundings are all there is.
//
// What bounds it: every channel is read and written once, a few operations each: memory.  The sines are the dear
// part, and all heads of a token share them: a workgroup takes one to four tokens, one thread works out the
// sine and cosine of one (token, pair), and LDS hands them to the threads that turn the heads' channels,
// 16 bytes of each half a thread.  32768 tokens of 28 + 4 heads in bf16, three axes: 98 us, 5.5 TB/s read + written
// (a copy reaches 5.0); 2999 of 32 + 8 in fp32, half of the channels in adjacent pairs: 19.9 us, 6.2 TB/s, part of
// it out of the caches; one token 2.8 us, a launch.
#include "oscar_common.h"

namespace {

constexpr int kMaxTokens = 4;   // tokens a workgroup takes

struct RopeParams {
  const void* in[2];     // queries, keys
  void* out[2];
  int64_t in_stride[2], out_stride[2];   // elements between tokens
  int heads[2];
  int64_t n_tokens;
  const int32_t* positions;   // [axes][n_tokens]
  const float* inv_freq;      // [half]
  uint64_t axis_lo, axis_hi;  // 2 bits a pair
  int half;                   // rotated pairs
  int tokens;                 // of a workgroup
  float sign;                 // -1: the turn taken back
};

enum { PAIRS_HALVES, PAIRS_ADJACENT, PAIRS_SCALAR };

// 16 bytes of elements as fp32 and back
template <typename T> struct Vec {
  static constexpr int N = 16 / sizeof(T);
  float x[N];
  __device__ __forceinline__ void load(const T* p) {
    const uint4 w = *reinterpret_cast<const uint4*>(p);
    const T* e = reinterpret_cast<const T*>(&w);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = to_f32<T>(e[i]);
  }
  __device__ __forceinline__ void store(T* p) const {
    uint4 w;
    T* e = reinterpret_cast<T*>(&w);
#pragma unroll
    for (int i = 0; i < N; ++i) e[i] = from_f32<T>(x[i]);
    *reinterpret_cast<uint4*>(p) = w;
  }
};

// (cos, sin) of 2 pi times position times frequency / 2 pi.
__device__ __forceinline__ float2 cos_sin(int32_t position, float inv_freq) {
#pragma clang fp contract(off)   // (products are rounded where their rests are taken)
  constexpr double kHi = 0.15915494309189535, kLo = -9.839338337591243e-18;   // 1 / 2 pi
  const double p = position, f = inv_freq;
  const double a = p * f, a_rest = fma(p, f, -a);   // exact together
  const double t = a * kHi, t_rest = fma(a, kHi, -t) + fma(a, kLo, a_rest * kHi);
  const double r = (t - rint(t)) + t_rest;          // turns, within half a turn
  const double quarter = rint(4.0 * r);
  const double y = fma(quarter, -0.25, r) * 6.283185307179586, z = y * y;   // |y| <= pi / 4
  // the series' next terms are 7e-12 and 5e-13 there
  double s = fma(z, fma(z, fma(z, fma(z, -1.0 / 39916800, 1.0 / 362880), -1.0 / 5040), 1.0 / 120), -1.0 / 6);
  double c = fma(z, fma(z, fma(z, fma(z, fma(z, 1.0 / 479001600, -1.0 / 3628800), 1.0 / 40320), -1.0 / 720), 1.0 / 24), -0.5);
  s = fma(y * z, s, y);
  c = fma(z, c, 1.0);
  const int q = (int)quarter & 3;
  const float cf = (float)(q & 1 ? s : c), sf = (float)(q & 1 ? c : s);
  return make_float2(q == 1 || q == 2 ? -cf : cf, q >= 2 ? -sf : sf);
}

__device__ __forceinline__ void turn(float& a, float& b, float2 cs) {
  const float y = a * cs.x - b * cs.y;
  b = b * cs.x + a * cs.y;
  a = y;
}

template <typename T, int PAIRS> __global__ __launch_bounds__(256) void oscar_rope_kernel(RopeParams P) {
  constexpr int N = Vec<T>::N;
  constexpr int ITEMS = PAIRS == PAIRS_SCALAR ? 64 : D / (2 * N);   // pieces of a head
  __shared__ __align__(16) float2 s_cs[kMaxTokens][64];
  const int tid = threadIdx.x;
  const int64_t t0 = (int64_t)blockIdx.x * P.tokens;
  const int nt = (int)min((int64_t)P.tokens, P.n_tokens - t0);
  {
    const int t = tid >> 6, i = tid & 63;
    if (t < nt && i < P.half) {
      const int axis = (int)((i < 32 ? P.axis_lo >> (2 * i) : P.axis_hi >> (2 * i - 64)) & 3);
      const float2 cs = cos_sin(P.positions[axis * P.n_tokens + t0 + t], P.inv_freq[i]);
      s_cs[t][i] = make_float2(cs.x, cs.y * P.sign);
    }
  }
  __syncthreads();
  const int heads = P.heads[0] + P.heads[1];
  const int j = tid % ITEMS;
  int t = 0, h = tid / ITEMS;
  for (;; h += 256 / ITEMS) {
    while (h >= heads) {
      h -= heads;
      ++t;
    }
    if (t >= nt) break;
    const bool key = h >= P.heads[0];
    const int hh = key ? h - P.heads[0] : h;
    const T* src = reinterpret_cast<const T*>(P.in[key]) + (t0 + t) * P.in_stride[key] + hh * D;
    T* dst = reinterpret_cast<T*>(P.out[key]) + (t0 + t) * P.out_stride[key] + hh * D;
    if (PAIRS == PAIRS_HALVES) {
      // vectors j and j + half / N turn together; those behind the rotated channels are copied
      const int per = P.half / N;
      const bool on = j < per;
      // (a copied pair: 2 per + (j - per), and D / (2 N) further)
      const int a = on ? j : per + j, b = on ? j + per : D / (2 * N) + j;
      Vec<T> x, y;
      x.load(src + a * N);
      y.load(src + b * N);
      if (on) {
#pragma unroll
        for (int e = 0; e < N; ++e) turn(x.x[e], y.x[e], s_cs[t][j * N + e]);
      }
      x.store(dst + a * N);
      y.store(dst + b * N);
    } else if (PAIRS == PAIRS_ADJACENT) {
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        Vec<T> x;
        const int at = j + v * ITEMS;   // (lanes side by side: a wave's access takes whole lines)
        x.load(src + at * N);
#pragma unroll
        for (int e = 0; e < N; e += 2) {
          const int i = (at * N + e) / 2;
          if (i < P.half) turn(x.x[e], x.x[e + 1], s_cs[t][i]);
        }
        x.store(dst + at * N);
      }
    } else {
      // halves that do not start on 16 bytes: one pair a thread, and one of the channels behind
      const int a = j < P.half ? j : P.half + j, b = j < P.half ? j + P.half : 64 + j;
      float x = to_f32<T>(src[a]), y = to_f32<T>(src[b]);
      if (j < P.half) turn(x, y, s_cs[t][j]);
      dst[a] = from_f32<T>(x);
      dst[b] = from_f32<T>(y);
    }
  }
}

template <typename T> void launch(const RopeParams& P, bool adjacent, dim3 grid, hipStream_t st) {
  if (adjacent)
    hipLaunchKernelGGL((oscar_rope_kernel<T, PAIRS_ADJACENT>), grid, dim3(256), 0, st, P);
  else if (P.half % Vec<T>::N == 0)
    hipLaunchKernelGGL((oscar_rope_kernel<T, PAIRS_HALVES>), grid, dim3(256), 0, st, P);
  else
    hipLaunchKernelGGL((oscar_rope_kernel<T, PAIRS_SCALAR>), grid, dim3(256), 0, st, P);
}

}  // namespace

extern "C" int oscar_rope(const void* q, const void* k, void* q_out, void* k_out, int64_t n_tokens,
                          int32_t n_q_heads, int32_t n_kv_heads, int64_t q_stride, int64_t k_stride,
                          int64_t q_out_stride, int64_t k_out_stride, const int32_t* positions,
                          const float* inv_freq, const uint8_t* pair_axis, int32_t n_axes, int32_t rotary_dim,
                          int32_t io_dtype, uint32_t flags, void* stream) {
  if (n_tokens < 0 || n_q_heads < 0 || n_kv_heads < 0 || n_axes < 1 || n_axes > 4 || rotary_dim < 2 ||
      rotary_dim > D || rotary_dim % 2 != 0)
    return OSCAR_ERR_INVALID_ARG;
  if (io_dtype != OSCAR_F32 && io_dtype != OSCAR_BF16 && io_dtype != OSCAR_F16) return OSCAR_ERR_INVALID_ARG;
  if (flags & ~(uint32_t)(OSCAR_ROPE_ADJACENT | OSCAR_ROPE_INVERSE)) return OSCAR_ERR_INVALID_ARG;
  RopeParams P = {};
  const int64_t vec = io_dtype == OSCAR_F32 ? 4 : 8;
  const void* in[2] = {q, k};
  void* out[2] = {q_out, k_out};
  const int heads[2] = {n_q_heads, n_kv_heads};
  const int64_t in_stride[2] = {q_stride, k_stride}, out_stride[2] = {q_out_stride, k_out_stride};
  for (int i = 0; i < 2; ++i) {
    if (heads[i] == 0 || n_tokens == 0) continue;   // (tensors of no tokens have no addresses)
    if (!in[i] || !out[i] || heads[i] > 65536) return OSCAR_ERR_INVALID_ARG;
    // 16-byte accesses; tokens do not overlap
    if (((reinterpret_cast<uintptr_t>(in[i]) | reinterpret_cast<uintptr_t>(out[i])) & 15) != 0 ||
        in_stride[i] % vec != 0 || out_stride[i] % vec != 0)
      return OSCAR_ERR_INVALID_ARG;
    if (n_tokens > 1 && (in_stride[i] < (int64_t)heads[i] * D || out_stride[i] < (int64_t)heads[i] * D))
      return OSCAR_ERR_INVALID_ARG;
    P.in[i] = in[i];
    P.out[i] = out[i];
    P.heads[i] = heads[i];
    P.in_stride[i] = in_stride[i];
    P.out_stride[i] = out_stride[i];
  }
  if (n_tokens > 0 && (!positions || !inv_freq)) return OSCAR_ERR_INVALID_ARG;
  P.half = rotary_dim / 2;
  if (pair_axis) {
    for (int i = 0; i < P.half; ++i) {
      if (pair_axis[i] >= n_axes) return OSCAR_ERR_INVALID_ARG;
      (i < 32 ? P.axis_lo : P.axis_hi) |= (uint64_t)pair_axis[i] << (2 * (i % 32));
    }
  } else if (n_axes != 1) {
    return OSCAR_ERR_INVALID_ARG;
  }
  if (n_tokens == 0 || n_q_heads + n_kv_heads == 0) return OSCAR_OK;
  P.n_tokens = n_tokens;
  P.positions = positions;
  P.inv_freq = inv_freq;
  P.sign = flags & OSCAR_ROPE_INVERSE ? -1.0f : 1.0f;
  // One token a workgroup, or up to four where there are many and one's pieces leave threads idle.  32768 tokens in
  // bf16: of 5 heads 33 us with one, 22 with four, of 18 68 and 58, of 32 103, 98 with two, 101 with four, of 40 117
  // and 123; in fp32, with twice the bytes a sine: of 5 heads 38 and 32, of 9 52 and 57.  1000 tokens of 18 heads in
  // bf16, which do not fill the chip twice over: 4.4 and 5.5.
  const bool adjacent = flags & OSCAR_ROPE_ADJACENT;
  const int64_t pieces = (n_q_heads + n_kv_heads) * (int64_t)(adjacent || P.half % vec == 0 ? D / 2 / vec : D / 2);
  const int64_t fit = (io_dtype == OSCAR_F32 ? 256 : 512) / pieces;
  P.tokens = n_tokens <= 8 * (int64_t)oscar_compute_units() || fit < 1 ? 1 : fit < kMaxTokens ? (int)fit : kMaxTokens;
  const int64_t blocks = (n_tokens + P.tokens - 1) / P.tokens;
  if (blocks >= 1 << 24) return OSCAR_ERR_INVALID_ARG;   // (fewer than 2^32 threads)
  const dim3 grid((unsigned)blocks);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (io_dtype == OSCAR_F32)
    launch<float>(P, adjacent, grid, st);
  else if (io_dtype == OSCAR_BF16)
    launch<__hip_bfloat16>(P, adjacent, grid, st);
  else
    launch<__half>(P, adjacent, grid, st);
  if (hipGetLastError() != hipSuccess) return OSCAR_ERR_HIP;
  return OSCAR_OK;
}
