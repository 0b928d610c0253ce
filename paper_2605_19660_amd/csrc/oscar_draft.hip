// oscar_draft_attn: attention of several new tokens of every sequence over its packed cache and, causally,
// over each other.
//
//   logit[t][h][i] = scale n_i sum_j Q_j (Delta_k c_k + b_k)_ij      cached token i, Q = H(q_th)/sqrt(128),
//                                                                    b = -Delta z (integer zero-points) or zero
//   logit[t][h][j] = scale <q_th, k_j>                               new token j <= t
//   out[t][h]      = softmax over both, times the values
//
// The T tokens' g query heads of a kv head are T g rows that read the same keys and values.  A wave holds
// 16 or 32 of them (16 a matrix tile) and takes whole pages of 128 tokens on its own, with its own running
// maximum and sum; four waves and the splits of the sequence are joined at the end.
//
//   S^T = K Q^T : v_mfma_f32_16x16x32_f16, rows = 16 tokens, columns = 16 query rows, over 128 channels
//   O^T = V^T P^T: rows = 16 channels, columns = query rows, over 128 tokens
// Row n of a token tile is token 4 (n % 4) + n / 4 of it, so that a lane's four results of tile T are its
// tokens 16 T + 4 r + lane / 16: exactly the tokens whose value codes the lane's chunk of the page holds for
// step r.  The probabilities are packed where they are and nothing is exchanged between lanes but the row
// maxima.
//
// Codes become fp16 operands with a mask (a code parked in the mantissa of a subnormal: c 2^(s - 24)); the
// steps go to the other operand, Q Delta_k once a group of tokens and P Delta_v once a group of channels, and
// 2^-s with them.  Q Delta and P Delta are rounded to fp16: half a step of 2^-11, a fourth of the output's
// own in bf16.  The zero terms (b) are products of their own on the matrix cores: for the keys they are
// what a tile's sums start from, for the values they and the row sums are rows of one extra tile.
// The probabilities are scaled by 2^15 (less where a value step of 2 or more would carry P Delta past the
// fp16 range): a token counts down to 2^-39 of the largest.  Sums, maxima and outputs are fp32.
#include "oscar_decode_common.h"

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kHalfMax = 65504.0f;
constexpr int kQShift = 2;           // the queries carry 2^2
constexpr int TAIL = 32;             // tokens of a 16-bit piece (window, new tokens)

struct DraftParams {
  const void *q, *k_new, *v_new;
  void* out;
  float* ws;
  const int32_t* new_lens;
  oscar_cache c;
  PageGeom g;
  int T, num_splits;
  float scale_log2;
};

template <int BITS> struct Codes {
  static constexpr int BPMIN = BITS == 2 ? 4 : 2, BPMAX = BITS == 2 ? 8 : 6;
  static constexpr int WORDS = BITS;   // dwords of a chunk
  // the operand of k-step kk from a chunk
  __device__ static __forceinline__ half8 operand(const uint32_t* w, int kk) {
    u32x4 r;
    if (BITS == 2) {
      const uint32_t x = w[kk / 2];
      if (kk % 2 == 0) {
        const uint32_t l = x << 4;
        r[0] = l & 0x00300030u, r[1] = l & 0x00C000C0u, r[2] = x & 0x00300030u, r[3] = x & 0x00C000C0u;
      } else {
        const uint32_t l = x >> 6;
        r[0] = x & 0x03000300u, r[1] = l & 0x00300030u, r[2] = l & 0x00C000C0u, r[3] = l & 0x03000300u;
      }
    } else {
      const uint32_t x = w[kk], l = x << 2, s = x >> 6;
      r[0] = l & 0x003C003Cu, r[1] = l & 0x03C003C0u, r[2] = s & 0x003C003Cu, r[3] = s & 0x03C003C0u;
    }
    return __builtin_bit_cast(half8, r);
  }
  // what an element's bit position is above the lowest
  __device__ static constexpr int above(int kk, int e) { return slot_bitpos(BITS, kk, e) - BPMIN; }
  // 2^(above - (BPMAX - BPMIN)), the other operand's counterweight for what is no code
  __device__ static __forceinline__ half8 counterweight(int kk) {
    half8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (_Float16)(1.0f / (float)(1 << (BPMAX - BPMIN - above(kk, e))));
    return r;
  }
};

// 8 numbers of a page's metadata, as fp16 (fp32 metadata: rounded, and kept inside the range)
template <bool M32> __device__ __forceinline__ half8 load_step(const uint8_t* base, int idx) {
  if (!M32) return *reinterpret_cast<const half8*>(base + (size_t)idx * 2);
  half8 r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = (_Float16)fminf(reinterpret_cast<const float*>(base)[idx + e], kHalfMax);
  return r;
}
// and the zero term b that belongs to steps `idx` and zeros `zidx`
template <bool M32> __device__ __forceinline__ half8 load_b(const uint8_t* base, int idx, int zidx, bool zp_min) {
  half8 r;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float s, z;
    if (M32) {
      s = reinterpret_cast<const float*>(base)[idx + e];
      z = reinterpret_cast<const float*>(base)[zidx + e];
    } else {
      s = (float)reinterpret_cast<const _Float16*>(base)[idx + e];
      z = (float)reinterpret_cast<const _Float16*>(base)[zidx + e];
    }
    r[e] = (_Float16)__builtin_amdgcn_fmed3f(zp_min ? z : -z * s, -kHalfMax, kHalfMax);
  }
  return r;
}

__device__ __forceinline__ float4v mfma(half8 a, half8 b, float4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ half2v pack2(float a, float b) {
  return __builtin_convertvector((float2v){a, b}, half2v);
}
__device__ __forceinline__ float max_of_row(float v) {   // over the four lanes that hold a query row
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}

// The running state of one tile of 16 query rows: lane's row = lane % 16.
struct RowTile {
  float4v o[8];   // channels 16 ct + 4 (lane / 16) + r, in units of the codes once pages have begun
  float4v x;      // of rows 4 (lane / 16) + r of the extra tile: zero terms of the value groups, then the row sum
  float m;        // running maximum, log2 units
};

template <int BITS, bool M32, int NR>
__global__ __launch_bounds__(256, 2) void oscar_draft_kernel(DraftParams P) {
  using C = Codes<BITS>;
  constexpr int ROWS = NR * 16;
  constexpr int OROW = D + 4;
  __shared__ __align__(16) float s_o[4][ROWS][OROW];
  __shared__ float s_m[4][ROWS], s_l[4][ROWS];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, q4 = lane >> 4;
  const int Hkv = P.c.cfg.n_kv_heads, Hq = P.c.cfg.n_q_heads, g = Hq / Hkv;
  const int split = blockIdx.x % P.num_splits, unit = blockIdx.x / P.num_splits;
  const int kvh = unit % Hkv, b = unit / Hkv;
  const int row0 = blockIdx.y * ROWS;

  const int n_new = P.new_lens ? min(max(P.new_lens[b], 0), P.T) : P.T;
  const int seq_len = max(P.c.seq_lens[b], 0);
  const int res = min(max(P.c.res_lens[b], 0), min(R, seq_len));
  const int pages = min((seq_len - res) / R, P.c.max_pages_per_seq);
  const int rows = min(max(n_new * g - row0, 0), ROWS);         // of this block that are there
  const bool zp_min = P.c.cfg.zp_mode == OSCAR_ZP_MIN;
  const bool bf16 = P.c.cfg.io_dtype == OSCAR_BF16;

  RowTile tile[NR];
#pragma unroll
  for (int i = 0; i < NR; ++i) {
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) tile[i].o[ct] = (float4v){0, 0, 0, 0};
    tile[i].x = (float4v){0, 0, 0, 0};
    tile[i].m = -INFINITY;
  }
  int eoff = 15;

  if (rows > 0) {
    // ---- queries: lane's row, channels 32 q4 .. + 31 ----
    half8 qh[NR][4];
    const uint16_t* q = reinterpret_cast<const uint16_t*>(P.q);
    int row_t[NR];
    const uint16_t* q_row[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int row = row0 + 16 * i + n;
      row_t[i] = row / g;
      const bool there = row < n_new * g;
      q_row[i] = q + (((size_t)b * P.T + (there ? row_t[i] : 0)) * Hq + (size_t)kvh * g + (there ? row % g : 0)) * D + 32 * q4;
      float x[32];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(q_row[i] + 8 * u);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint16_t v = (uint16_t)(w[e / 2] >> (16 * (e % 2)));
          const float f = bf16 ? __uint_as_float((uint32_t)v << 16) : __half2float(__ushort_as_half(v));
          x[8 * u + e] = there ? f : 0.0f;
        }
      }
      float mul = P.scale_log2 * (float)(1 << kQShift);
      if (P.c.cfg.rotation == OSCAR_ROTATION_ON) {
#pragma unroll
        for (int h = 1; h < 32; h <<= 1) {
#pragma unroll
          for (int u = 0; u < 32; ++u) {
            if ((u & h) == 0) {
              const float a = x[u], c = x[u | h];
              x[u] = a + c;
              x[u | h] = a - c;
            }
          }
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const float sg = (q4 >> s) & 1 ? -1.0f : 1.0f;
#pragma unroll
          for (int u = 0; u < 32; ++u) x[u] = fmaf(x[u], sg, __shfl_xor(x[u], 16 << s, 64));
        }
        mul *= 0.08838834764831845f;
      }
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          qh[i][kk][e] = (_Float16)(x[8 * kk + e] * mul);
    }

    // ---- 16-bit tokens: the window's pieces, then the new tokens', dealt to the waves of all splits ----
    const int waves = P.num_splits * 4, own = split * 4 + wave;
    const int n_win = (res + TAIL - 1) / TAIL;
    const int last_t = (row0 + rows - 1) / g;                            // last new token any row here sees
    const int n_tail = n_win + (min(n_new, last_t + 1) + TAIL - 1) / TAIL;
    for (int u = own; u < n_tail; u += waves) {
      const bool win = u < n_win;
      const int t0 = (win ? u : u - n_win) * TAIL, count = win ? res : n_new;
      const size_t head = (size_t)b * Hkv + kvh;
      const uint16_t *kb, *vb;
      size_t stride;
      if (win) {
        kb = reinterpret_cast<const uint16_t*>(P.c.res_k) + head * R * D;
        vb = reinterpret_cast<const uint16_t*>(P.c.res_v) + head * R * D;
        stride = D;
      } else {
        kb = reinterpret_cast<const uint16_t*>(P.k_new) + ((size_t)b * P.T * Hkv + kvh) * D;
        vb = reinterpret_cast<const uint16_t*>(P.v_new) + ((size_t)b * P.T * Hkv + kvh) * D;
        stride = (size_t)Hkv * D;
      }
      // logits: tile s holds tokens t0 + 16 s + .., row n of the tile = token n of it
      float4v S[NR][2];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int t = min(t0 + 16 * s + n, count - 1);
        u32x4 a[4];
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) a[kk] = *reinterpret_cast<const u32x4*>(kb + (size_t)t * stride + 32 * q4 + 8 * kk);
#pragma unroll
        for (int i = 0; i < NR; ++i) {
          float4v acc = {0, 0, 0, 0};
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            if (win) {
              acc = mfma(__builtin_bit_cast(half8, a[kk]), qh[i][kk], acc);
            } else {
              const u32x4 r = *reinterpret_cast<const u32x4*>(q_row[i] + 8 * kk);
              if (bf16)
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[kk]),
                                                              __builtin_bit_cast(bf16x8, r), acc, 0, 0, 0);
              else
                acc = mfma(__builtin_bit_cast(half8, a[kk]), __builtin_bit_cast(half8, r), acc);
            }
          }
          S[i][s] = acc;
        }
      }
      float f[2][4];
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int t = t0 + 16 * s + 4 * q4 + r;
          f[s][r] = win ? load_meta(P.c.res_norm, head * R + min(t, R - 1), M32 ? 4 : 2) * (1.0f / (1 << kQShift)) : P.scale_log2;
        }
      half8 pr[NR];
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        float mx = -INFINITY;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int t = t0 + 16 * s + 4 * q4 + r;
            const bool seen = t < count && (win || t <= row_t[i]);
            const float v = seen ? S[i][s][r] * f[s][r] : -INFINITY;
            S[i][s][r] = v;
            mx = fmaxf(mx, v);
          }
        const float m = fmaxf(tile[i].m, max_of_row(mx));
        const float M = m == -INFINITY ? 0.0f : m - eoff;
        const float alpha = tile[i].m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(tile[i].m - m);
        tile[i].m = m;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int r = 0; r < 4; ++r) pr[i][4 * s + r] = (_Float16)__builtin_amdgcn_exp2f(S[i][s][r] - M);
#pragma unroll
        for (int ct = 0; ct < 8; ++ct) tile[i].o[ct] *= alpha;
        tile[i].x *= alpha;
        half8 one;
#pragma unroll
        for (int e = 0; e < 8; ++e) one[e] = (_Float16)(n == 4 ? 1.0f / (1 << (C::BPMAX - C::BPMIN)) : 0.0f);
        tile[i].x = mfma(one, pr[i], tile[i].x);
      }
      // values: channel 16 ct + n of tokens t0 + 16 s + 4 q4 + r
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) {
        half8 a;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int t = t0 + 16 * s + 4 * q4 + r;
            const uint16_t v = vb[(size_t)min(t, count - 1) * stride + 16 * ct + n];
            const float x = bf16 ? __uint_as_float((uint32_t)v << 16) : __half2float(__ushort_as_half(v));
            a[4 * s + r] = (_Float16)(t < count ? __builtin_amdgcn_fmed3f(x, -kHalfMax, kHalfMax) : 0.0f);
          }
#pragma unroll
        for (int i = 0; i < NR; ++i) tile[i].o[ct] = mfma(a, pr[i], tile[i].o[ct]);
      }
    }

    // ---- pages ----
    // queries in the codes' order, with the counterweights of their bit positions
    half8 qc[NR][4];
#pragma unroll
    for (int i = 0; i < NR; ++i)
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int u = slot_index(BITS, kk, e);
          qc[i][kk][e] = qh[i][u / 8][u % 8] * (_Float16)(1.0f / (float)(1 << C::above(kk, e)));
        }
    constexpr float kCodeUnit = 1.0f / (float)(1 << (24 - C::BPMIN));     // of a code in the sums
#pragma unroll
    for (int i = 0; i < NR; ++i)
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) tile[i].o[ct] *= kCodeUnit;
    const int row_of_tile = 4 * (n % 4) + n / 4;                          // token of a tile that this lane's row is

    for (int u = own < n_tail ? own + (n_tail - own + waves - 1) / waves * waves : own; u - n_tail < pages; u += waves) {
      const int phys = P.c.block_table[(size_t)b * P.c.max_pages_per_seq + (u - n_tail)];
      if (phys < 0 || phys >= P.c.num_pages) continue;
      const size_t pg = (size_t)phys * Hkv + kvh;
      const uint8_t* kcodes = reinterpret_cast<const uint8_t*>(P.c.k_codes) + pg * P.g.k_codes_bytes;
      const uint8_t* kmeta = reinterpret_cast<const uint8_t*>(P.c.k_meta) + pg * P.g.k_meta_bytes;
      const uint8_t* knorm = reinterpret_cast<const uint8_t*>(P.c.k_norms) + pg * P.g.k_norms_bytes;
      const uint8_t* vcodes = reinterpret_cast<const uint8_t*>(P.c.v_codes) + pg * P.g.v_codes_bytes;
      const uint8_t* vmeta = reinterpret_cast<const uint8_t*>(P.c.v_meta) + pg * P.g.v_meta_bytes;
      uint32_t kc[4][2 * BITS], vc[4][2 * BITS];
#pragma unroll
      for (int w = 0; w < 4; ++w)
#pragma unroll
        for (int j = 0; j < BITS / 2; ++j) {
          *reinterpret_cast<u32x4*>(&kc[w][4 * j]) =
              *reinterpret_cast<const u32x4*>(kcodes + chunk_offset(BITS, 2 * w, row_of_tile, q4) + 16 * j);
          *reinterpret_cast<u32x4*>(&vc[w][4 * j]) =
              *reinterpret_cast<const u32x4*>(vcodes + chunk_offset(BITS, 2 * w, n, q4) + 16 * j);
        }

      // logits of 128 tokens
      float4v S[NR][8];
      half8 qd[NR][4];
      float4v start[NR];
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if (w * 32 % P.g.k_group == 0) {
          const int gk = w * 32 / P.g.k_group;
#pragma unroll
          for (int i = 0; i < NR; ++i) start[i] = (float4v){0, 0, 0, 0};
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            const int at = gk * D + 32 * q4 + 8 * kk;
            const half8 step = load_step<M32>(kmeta, at);
            const half8 zb = load_b<M32>(kmeta, at, P.g.ngk * D + at, zp_min) * C::counterweight(kk);
#pragma unroll
            for (int i = 0; i < NR; ++i) {
              qd[i][kk] = qc[i][kk] * step;
              start[i] = mfma(zb, qc[i][kk], start[i]);
            }
          }
#pragma unroll
          for (int i = 0; i < NR; ++i) start[i] *= 1.0f / (float)(1 << (24 - C::BPMAX));
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
          for (int i = 0; i < NR; ++i) S[i][2 * w + j] = start[i];
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            const half8 a = C::operand(kc[w] + j * BITS, kk);
#pragma unroll
            for (int i = 0; i < NR; ++i) S[i][2 * w + j] = mfma(a, qd[i][kk], S[i][2 * w + j]);
          }
        }
      }

      // the extra tile's rows: zero terms of the value groups (0 .. 3), row sum (4)
      half8 extra[4];
      uint32_t big = 0;   // largest value step (fp16 bits) of this lane's group
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        const int at = min(n, P.g.ngv - 1) * R + (4 * kk + q4) * 8;
        const half8 step = load_step<M32>(vmeta, at);
        const half8 zb = load_b<M32>(vmeta, at, P.g.ngv * R + at, zp_min);
        const half8 cw = C::counterweight(kk);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          extra[kk][e] = n == 4 ? cw[e] : zb[e] * cw[e];
          big = max(big, (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)step[e]));
        }
      }
      int page_off = 15;
      if (__any(big >= 0x4000u)) {
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) big = max(big, (uint32_t)__shfl_xor((int)big, s, 64));
        page_off = __builtin_amdgcn_readfirstlane(15 - max((int)(big >> 10) - 14, 0));
      }
      const int off = min(eoff, page_off);

      // probabilities
      float nrm[4][8];
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int t = 0; t < 8; ++t)
          nrm[r][t] = load_meta(knorm, (4 * r + q4) * 8 + t, M32 ? 4 : 2) * (float)(1 << (24 - C::BPMIN - kQShift));
      half8 pr[NR][4];
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        float mx = -INFINITY;
#pragma unroll
        for (int t = 0; t < 8; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            S[i][t][r] *= nrm[r][t];
            mx = fmaxf(mx, S[i][t][r]);
          }
        const float m = fmaxf(tile[i].m, max_of_row(mx));
        if (__any(m > tile[i].m) || off != eoff) {
          const float alpha = tile[i].m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(tile[i].m - m + (float)(off - eoff));
#pragma unroll
          for (int ct = 0; ct < 8; ++ct) tile[i].o[ct] *= alpha;
          tile[i].x *= alpha;
          tile[i].m = m;
        }
        const float M = m - (float)off;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int t = 0; t < 8; t += 2) {
            const float Mk = M + (float)C::above(r, t);
            const half2v p = pack2(__builtin_amdgcn_exp2f(S[i][t][r] - Mk), __builtin_amdgcn_exp2f(S[i][t + 1][r] - Mk));
            pr[i][r][t] = p[0];
            pr[i][r][t + 1] = p[1];
          }
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) tile[i].x = mfma(extra[kk], pr[i][kk], tile[i].x);
      }
      eoff = off;

      // values
      half8 pd[NR][4];
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if (w * 32 % P.g.v_group == 0) {
          const int gv = w * 32 / P.g.v_group;
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            const half8 step = load_step<M32>(vmeta, gv * R + (4 * kk + q4) * 8);
#pragma unroll
            for (int i = 0; i < NR; ++i) pd[i][kk] = pr[i][kk] * step;
          }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            const half8 a = C::operand(vc[w] + j * BITS, kk);
#pragma unroll
            for (int i = 0; i < NR; ++i) tile[i].o[2 * w + j] = mfma(a, pd[i][kk], tile[i].o[2 * w + j]);
          }
      }
    }
    // back to numbers: codes' unit, zero terms of each channel's value group
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      tile[i].x *= (float)(1 << (C::BPMAX - C::BPMIN));
      float zb[4];
#pragma unroll
      for (int gv = 0; gv < 4; ++gv) zb[gv] = __shfl(tile[i].x[gv], n, 64);
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) {
        const int gv = ct * 16 / P.g.v_group;
        const float z = gv == 0 ? zb[0] : gv == 1 ? zb[1] : gv == 2 ? zb[2] : zb[3];
        tile[i].o[ct] = tile[i].o[ct] * (float)(1 << (24 - C::BPMIN)) + z;
      }
    }
  }

  // ---- the four waves joined ----
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const float l = __shfl(tile[i].x[0], 16 + n, 64);
    if (q4 == 0) {
      s_m[wave][16 * i + n] = tile[i].m == -INFINITY ? -INFINITY : tile[i].m - (float)eoff;
      s_l[wave][16 * i + n] = l;
    }
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) *reinterpret_cast<float4v*>(&s_o[wave][16 * i + n][16 * ct + 4 * q4]) = tile[i].o[ct];
  }
  __syncthreads();
  const int c4 = (tid & 31) * 4;
  for (int row = tid >> 5; row < ROWS; row += 8) {
    if (row0 + row >= P.T * g) break;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) M = fmaxf(M, s_m[w][row]);
    float4v o = {0, 0, 0, 0};
    float l = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if (s_m[w][row] == -INFINITY) continue;
      const float f = __builtin_amdgcn_exp2f(s_m[w][row] - M);
      o += *reinterpret_cast<const float4v*>(&s_o[w][row][c4]) * f;
      l = fmaf(s_l[w][row], f, l);
    }
    const bool there = row < rows;
    const int t = (row0 + row) / g, h = kvh * g + (row0 + row) % g;
    const size_t out_row = ((size_t)b * P.T + t) * Hq + h;
    if (P.num_splits > 1) {
      float* rec = P.ws + (out_row * P.num_splits + split) * WS_STRIDE;
      *reinterpret_cast<float2v*>(rec + c4) = there ? (float2v){o[0], o[1]} : (float2v){0, 0};
      *reinterpret_cast<float2v*>(rec + c4 + 2) = there ? (float2v){o[2], o[3]} : (float2v){0, 0};
      if (c4 == 0) *reinterpret_cast<float2v*>(rec + D) = there ? (float2v){M, l} : (float2v){-INFINITY, 0};
    } else {
      const float inv = there && l > 0.0f ? 1.0f / l : 0.0f;
      uint16_t* dst = reinterpret_cast<uint16_t*>(P.out) + out_row * D + c4;
      uint16_t v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = there ? o[e] * inv : 0.0f;
        v[e] = bf16 ? __builtin_bit_cast(uint16_t, __float2bfloat16(x)) : __builtin_bit_cast(uint16_t, __float2half_rn(x));
      }
      *reinterpret_cast<uint2*>(dst) = make_uint2(v[0] | (uint32_t)v[1] << 16, v[2] | (uint32_t)v[3] << 16);
    }
  }
}

template <int BITS, bool M32> void launch(const DraftParams& P, int nr, dim3 grid, hipStream_t st) {
  if (nr == 1)
    hipLaunchKernelGGL((oscar_draft_kernel<BITS, M32, 1>), grid, dim3(256), 0, st, P);
  else
    hipLaunchKernelGGL((oscar_draft_kernel<BITS, M32, 2>), grid, dim3(256), 0, st, P);
}

// tiles of 16 query rows a wave holds
int row_tiles(const oscar_config& cfg, int T) { return (int64_t)T * (cfg.n_q_heads / cfg.n_kv_heads) <= 16 ? 1 : 2; }
int64_t row_blocks(const oscar_config& cfg, int T) {
  const int rows = 16 * row_tiles(cfg, T);
  return ((int64_t)T * (cfg.n_q_heads / cfg.n_kv_heads) + rows - 1) / rows;
}

int check_draft_config(const oscar_config* cfg) {
  const int rc = oscar_validate_config(cfg);
  if (rc != OSCAR_OK) return rc;
  return cfg->io_dtype == OSCAR_F32 ? OSCAR_ERR_UNSUPPORTED : OSCAR_OK;
}

}  // namespace

extern "C" int32_t oscar_draft_auto_splits(const oscar_config* cfg, int32_t batch, int32_t T, int32_t max_seq_len) {
  if (check_draft_config(cfg) != OSCAR_OK || batch <= 0 || T <= 0) return 1;
  const int64_t units = (int64_t)batch * cfg->n_kv_heads * row_blocks(*cfg, T);
  const int64_t pages = max_seq_len > 0 ? ((int64_t)max_seq_len + R - 1) / R : 1;
  int64_t splits = 2 * (int64_t)oscar_compute_units() / units;
  if (splits > (pages + 3) / 4) splits = (pages + 3) / 4;
  if (splits > 512) splits = 512;
  return splits < 1 ? 1 : (int32_t)splits;
}

extern "C" size_t oscar_draft_workspace_bytes(const oscar_config* cfg, int32_t batch, int32_t T, int32_t num_splits) {
  if (!cfg || batch <= 0 || T <= 0 || num_splits <= 1 || cfg->n_q_heads <= 0) return 0;
  return (size_t)batch * T * cfg->n_q_heads * num_splits * WS_STRIDE * sizeof(float);
}

extern "C" int oscar_draft_attn(const void* q, const void* k_new, const void* v_new, int32_t T,
                                const int32_t* new_lens, const oscar_cache* cache, void* out,
                                float softmax_scale, int32_t max_seq_len_hint, int32_t num_splits,
                                void* workspace, size_t workspace_bytes, void* stream) {
  int rc = oscar_check_cache(cache);
  if (rc != OSCAR_OK) return rc;
  const oscar_config& cfg = cache->cfg;
  rc = check_draft_config(&cfg);
  if (rc != OSCAR_OK) return rc;
  if (T < 0 || max_seq_len_hint < 0 || num_splits < 0 || num_splits > 512 || cache->num_pages <= 0)
    return OSCAR_ERR_INVALID_ARG;
  if (T == 0) return OSCAR_OK;
  if (!q || !k_new || !v_new || !out) return OSCAR_ERR_INVALID_ARG;
  if (((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(k_new) | reinterpret_cast<uintptr_t>(v_new) |
        reinterpret_cast<uintptr_t>(out)) & 15) != 0)
    return OSCAR_ERR_INVALID_ARG;
  if (num_splits == 0) num_splits = oscar_draft_auto_splits(&cfg, cache->batch, T, max_seq_len_hint);
  const int64_t blocks = row_blocks(cfg, T), units = (int64_t)cache->batch * cfg.n_kv_heads * num_splits;
  if (blocks > 65535 || units > 0x7fffffff || cache->batch > 65535 || (int64_t)T * cfg.n_q_heads > 0x7fffffff)
    return OSCAR_ERR_INVALID_ARG;
  const size_t need = oscar_draft_workspace_bytes(&cfg, cache->batch, T, num_splits);
  if (need > 0 && (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 7) != 0))
    return OSCAR_ERR_WORKSPACE;
  DraftParams P;
  P.q = q;
  P.k_new = k_new;
  P.v_new = v_new;
  P.out = out;
  P.ws = reinterpret_cast<float*>(workspace);
  P.new_lens = new_lens;
  P.c = *cache;
  P.g = make_geom(cfg.bits, cfg.k_group, cfg.v_group, cfg.meta_dtype);
  P.T = T;
  P.num_splits = num_splits;
  P.scale_log2 = (softmax_scale > 0.0f ? softmax_scale : 0.08838834764831845f) * 1.4426950408889634f;
  // row blocks of one page range are a multiple of the XCDs' number apart wherever the ranges are
  const dim3 grid((unsigned)units, (unsigned)blocks);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const int nr = row_tiles(cfg, T);
  const bool m32 = cfg.meta_dtype == OSCAR_F32;
  if (cfg.bits == 2) {
    if (m32) launch<2, true>(P, nr, grid, st); else launch<2, false>(P, nr, grid, st);
  } else {
    if (m32) launch<4, true>(P, nr, grid, st); else launch<4, false>(P, nr, grid, st);
  }
  if (num_splits > 1)
    oscar_launch_decode_reduce(P.ws, out, num_splits, cfg.io_dtype, T * cfg.n_q_heads, cache->batch, st);
  if (hipGetLastError() != hipSuccess) return OSCAR_ERR_HIP;
  return OSCAR_OK;
}
