// oscar_cache_read: keys and values of a range of tokens, out of the packed cache.
//
//   k_t = H(n_t K_u,t) / sqrt(128),  K_u,tj = Delta_gj (c_tj - z_gj)      (H is its own inverse)
//   v_tj = Delta_tg (c_tj - z_tg)
// and from the window K_u and V as they stand (float zero-points: Delta c + zero).
//
// What bounds it: 86 bytes a token and kv head are read (2-bit codes) and 512 written (16-bit), so it is a
// stream of writes, and the vector ALU is the next wall (400 operations a wave and tile of 16 tokens).  A workgroup
// takes the keys or the values of one page of one kv head: a wave 32 tokens' keys (two tiles, whose chunks a lane
// loads with one access, 1 KB a wave) or 32 channels' values.  A lane holds 32 channels of a token: five Hadamard
// stages are in its registers, two are exchanges inside a quad of lanes.  Either goes through LDS so that rows of
// 128 channels are written whole, and past the caches, where nothing reads them soon (145 us with ordinary stores).
// 4 x 32768 tokens of 8 kv heads, 2-bit to bf16: 124 us, 5.1 TB/s read + written (a copy reaches 5.0, a fill 6.9);
// 8 x 900 4-bit to fp32: 17 us, 4.0 TB/s; 1000 tokens: 5.9 us, the chain of lengths, table and page.
#include "oscar_decode_common.h"
#include "oscar_rowops.h"

namespace {

struct ReadParams {
  void *k, *v;
  const int32_t* starts;
  oscar_cache c;
  PageGeom g;
  int64_t T;
};

// The 32 codes of a lane's chunk as floats, in their natural order: spread over the bytes of a register, which
// convert without being cut out.
template <int BITS> __device__ __forceinline__ void unpack_chunk(const uint32_t* w, float (&x)[32]) {
  constexpr int PER = 8 / BITS;   // codes of a byte
#pragma unroll
  for (int i = 0; i < BITS; ++i)
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const uint32_t v = w[i] >> (k * BITS) & (BITS == 2 ? 0x03030303u : 0x0f0f0f0fu);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[(4 * i + j) * PER + k] = (float)(v >> (8 * j) & 0xffu);
    }
}

// A lane's 32 steps or zeros as they are stored, in operand order (8 kk + e); widened where they are used.
template <bool M32> struct Meta32 {
  uint4 q[M32 ? 8 : 4];
  // 8 of them every `stride` numbers from `idx` on
  __device__ __forceinline__ void load(const uint8_t* base, int idx, int stride) {
    constexpr int PER = M32 ? 2 : 1;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int i = 0; i < PER; ++i)
        q[kk * PER + i] = reinterpret_cast<const uint4*>(base + (size_t)(idx + kk * stride) * (M32 ? 4 : 2))[i];
  }
  // what is worked out of them is not carried beyond this point
  __device__ __forceinline__ void keep() {
#pragma unroll
    for (int i = 0; i < (M32 ? 8 : 4); ++i) asm volatile("" : "+v"(q[i].x), "+v"(q[i].y), "+v"(q[i].z), "+v"(q[i].w));
  }
  __device__ __forceinline__ float at(int i) const {
    if (M32) return __uint_as_float(reinterpret_cast<const uint32_t*>(q)[i]);
    return __half2float(__ushort_as_half((uint16_t)(reinterpret_cast<const uint32_t*>(q)[i / 2] >> (16 * (i % 2)))));
  }
};
// H over 128 channels, 32 consecutive ones in each lane of a quad (lane % 4 = which), times mul
__device__ __forceinline__ void rotate_quad(float (&x)[32], float mul) {
#pragma unroll
  for (int h = 1; h < 32; h <<= 1) {
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      if ((i & h) == 0) {
        const float a = x[i], b = x[i | h];
        x[i] = a + b;
        x[i | h] = a - b;
      }
    }
  }
  // Across the quad: own += partner * s with s = +1 in the lower lane and -1 in the upper one, which leaves the
  // upper lane b - a for a - b; the sign a lane has collected goes into the factor.  (A DPP operand must not be read
  // in the two issue slots after it was written: the block starts with that wait, and inside it every element is
  // rewritten eight instructions before it is read again.)
  const int q4 = threadIdx.x & 3;
  const float s0 = q4 & 1 ? -1.0f : 1.0f, s1 = q4 & 2 ? -1.0f : 1.0f;
#define OSCAR_QUAD_STAGE(S, CTRL)                                            \
  "v_fmac_f32_dpp %0, %0, " S " " CTRL " row_mask:0xf bank_mask:0xf\n\t"      \
  "v_fmac_f32_dpp %1, %1, " S " " CTRL " row_mask:0xf bank_mask:0xf\n\t"      \
  "v_fmac_f32_dpp %2, %2, " S " " CTRL " row_mask:0xf bank_mask:0xf\n\t"      \
  "v_fmac_f32_dpp %3, %3, " S " " CTRL " row_mask:0xf bank_mask:0xf\n\t"      \
  "v_fmac_f32_dpp %4, %4, " S " " CTRL " row_mask:0xf bank_mask:0xf\n\t"      \
  "v_fmac_f32_dpp %5, %5, " S " " CTRL " row_mask:0xf bank_mask:0xf\n\t"      \
  "v_fmac_f32_dpp %6, %6, " S " " CTRL " row_mask:0xf bank_mask:0xf\n\t"      \
  "v_fmac_f32_dpp %7, %7, " S " " CTRL " row_mask:0xf bank_mask:0xf\n\t"
#pragma unroll
  for (int i = 0; i < 32; i += 8)
    asm volatile("s_nop 1\n\t"
                 OSCAR_QUAD_STAGE("%8", "quad_perm:[1,0,3,2]")
                 OSCAR_QUAD_STAGE("%9", "quad_perm:[2,3,0,1]")
                 : "+v"(x[i]), "+v"(x[i + 1]), "+v"(x[i + 2]), "+v"(x[i + 3]), "+v"(x[i + 4]), "+v"(x[i + 5]),
                   "+v"(x[i + 6]), "+v"(x[i + 7])
                 : "v"(s0), "v"(s1));
#undef OSCAR_QUAD_STAGE
  mul *= s0 * s1;
#pragma unroll
  for (int i = 0; i < 32; ++i) x[i] *= mul;
}

// Two numbers to the output's type, in one conversion.
typedef float float2v __attribute__((ext_vector_type(2)));
template <typename OUT> struct Pair;
template <> struct Pair<float> {
  typedef float2v Type;
};
template <> struct Pair<__half> {
  typedef _Float16 Type __attribute__((ext_vector_type(2)));
};
template <> struct Pair<__hip_bfloat16> {
  typedef __bf16 Type __attribute__((ext_vector_type(2)));
};
template <typename OUT> __device__ __forceinline__ typename Pair<OUT>::Type pair(float a, float b) {
  return __builtin_convertvector((float2v){a, b}, typename Pair<OUT>::Type);
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void store_row(uint8_t* p, const uint4& v) {
  __builtin_nontemporal_store((u32x4){v.x, v.y, v.z, v.w}, reinterpret_cast<u32x4*>(p));
}

// 8 numbers of the window's type
__device__ __forceinline__ void load8_io(const void* base, int64_t at, int dt, float (&x)[8]) {
  if (dt == OSCAR_F32) {
    const float4* p = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(base) + at);
    const float4 a = p[0], b = p[1];
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  } else {
    const uint4 v = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(base) + at);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint16_t e = (uint16_t)(w[i / 2] >> (16 * (i % 2)));
      x[i] = dt == OSCAR_BF16 ? bf16_bits_to_f32(e) : __half2float(__ushort_as_half(e));
    }
  }
}

template <int BITS, typename OUT, bool M32, bool ZP_MIN>
__global__ __launch_bounds__(256, sizeof(OUT) == 2 && !M32 ? 4 : 2) void oscar_cache_read_kernel(ReadParams P) {
  typedef typename Pair<OUT>::Type Two;
  // a wave's 16 tokens of keys, or the workgroup's 128 tokens of values; padded so that rows written at once by
  // different lanes fall on other banks
  constexpr int KROW = D * sizeof(OUT) + 32, VROW = D * sizeof(OUT) + 32;
  __shared__ __align__(16) uint8_t s_rows[4][R / 4 * VROW];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  uint8_t* rows = s_rows[wave];
  const int h = blockIdx.y, b = blockIdx.z, Hkv = P.c.cfg.n_kv_heads;
  const bool values = P.k == nullptr || (P.v != nullptr && blockIdx.x % 2 == 1);
  const int block = P.k && P.v ? blockIdx.x / 2 : blockIdx.x;
  const int seq_len = max(P.c.seq_lens[b], 0);
  const int res = min(max(P.c.res_lens[b], 0), min(R, seq_len));
  const int pages = min((seq_len - res) / R, P.c.max_pages_per_seq);
  const int64_t start = P.starts ? P.starts[b] : 0;
  const int64_t t_begin = max(start, (int64_t)0), t_end = min(start + P.T, (int64_t)pages * R + res);
  const int64_t page = t_begin / R + block;
  const int64_t lo = max(t_begin, page * R), hi = min(t_end, (page + 1) * R);
  if (lo >= hi) return;
  const int t_lo = (int)(lo - page * R), t_hi = (int)(hi - page * R);   // of this page's tokens
  const bool window = page == pages;
  int64_t phys = 0;
  if (!window) {
    phys = P.c.block_table[(int64_t)b * P.c.max_pages_per_seq + page];
    if (phys < 0 || phys >= P.c.num_pages) return;
  }
  const int64_t unit = window ? (int64_t)b * Hkv + h : phys * Hkv + h;
  const int n = lane >> 2, q4 = lane & 3;
  // row `page * R + t` of the outputs
  const int64_t out_row = (((int64_t)b * P.T + page * R - start) * Hkv + h) * D;
  const int64_t row_bytes = (int64_t)Hkv * D * sizeof(OUT);

  if (!values) {
    uint8_t* out = reinterpret_cast<uint8_t*>(reinterpret_cast<OUT*>(P.k) + out_row);
    const bool rotated = P.c.cfg.rotation == OSCAR_ROTATION_ON;
    uint32_t w[2 * BITS];
    float norm[2];
    Meta32<M32> step, zero;   // (widened for each tile: as 64 floats they cost registers, and waves, 83 -> 162 us)
    if (!window) {
      const uint8_t* codes = reinterpret_cast<const uint8_t*>(P.c.k_codes) + unit * P.g.k_codes_bytes;
      const uint4* src = reinterpret_cast<const uint4*>(codes + chunk_offset(BITS, 2 * wave, n, q4));
#pragma unroll
      for (int i = 0; i < BITS / 2; ++i) *reinterpret_cast<uint4*>(w + 4 * i) = src[i];
      // the two tiles lie in one group of 32, 64 or 128 tokens
      const uint8_t* meta = reinterpret_cast<const uint8_t*>(P.c.k_meta) + unit * P.g.k_meta_bytes;
      const int group = wave * 32 / P.g.k_group;
      step.load(meta, group * D + 32 * q4, 8);
      zero.load(meta, (P.g.ngk + group) * D + 32 * q4, 8);
#pragma unroll
      for (int i = 0; i < 2; ++i)
        norm[i] = load_meta(reinterpret_cast<const uint8_t*>(P.c.k_norms) + unit * P.g.k_norms_bytes,
                            tok_meta_pos((2 * wave + i) * 16 + n), M32 ? 4 : 2);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int t0 = (2 * wave + i) * 16;
      if (t0 >= t_hi || t0 + 16 <= t_lo) continue;
      float x[32], nm;
      if (!window) {
        step.keep();
        zero.keep();
        unpack_chunk<BITS>(w + i * BITS, x);
#pragma unroll
        for (int u = 0; u < 32; ++u) {
          const float a = step.at(kmeta_pos_of_chan(BITS, u)), z = zero.at(kmeta_pos_of_chan(BITS, u));
          x[u] = ZP_MIN ? fmaf(x[u], a, z) : (x[u] - z) * a;
        }
        nm = norm[i];
      } else {
#pragma unroll
        for (int u = 0; u < 4; ++u)
          load8_io(P.c.res_k, (unit * R + t0 + n) * D + 32 * q4 + 8 * u, OSCAR_F16, reinterpret_cast<float(&)[8]>(x[8 * u]));
        nm = load_meta(P.c.res_norm, unit * R + t0 + n, M32 ? 4 : 2);
      }
      if (rotated) {
        rotate_quad(x, nm * 0.08838834764831845f);
      } else {
#pragma unroll
        for (int u = 0; u < 32; ++u) x[u] *= nm;
      }
      Two* row = reinterpret_cast<Two*>(rows + n * KROW + 32 * q4 * sizeof(OUT));
#pragma unroll
      for (int u = 0; u < 32; u += 2) row[u / 2] = pair<OUT>(x[u], x[u + 1]);
      wave_lds_fence();
      constexpr int LANES = D * sizeof(OUT) / 16;   // of a row
#pragma unroll
      for (int r = 0; r < 16; r += 64 / LANES) {
        const int t = t0 + r + lane / LANES, c = lane % LANES * 16;
        const uint4 v = *reinterpret_cast<const uint4*>(rows + (r + lane / LANES) * KROW + c);
        if (t >= t_lo && t < t_hi) store_row(out + t * row_bytes + c, v);
      }
      wave_lds_fence();
    }
    return;
  }

  uint8_t* out = reinterpret_cast<uint8_t*>(reinterpret_cast<OUT*>(P.v) + out_row);
  if (window) {
    // 8 channels of a token a thread
    for (int t = t_lo + tid / 16; t < t_hi; t += 16) {
      float x[8];
      load8_io(P.c.res_v, (unit * R + t) * D + 8 * (tid % 16), P.c.cfg.io_dtype, x);
      Two* row = reinterpret_cast<Two*>(out + t * row_bytes) + 4 * (tid % 16);
#pragma unroll
      for (int u = 0; u < 4; ++u) row[u] = pair<OUT>(x[2 * u], x[2 * u + 1]);
    }
    return;
  }
  const uint8_t* codes = reinterpret_cast<const uint8_t*>(P.c.v_codes) + unit * P.g.v_codes_bytes;
  const uint4* src = reinterpret_cast<const uint4*>(codes + chunk_offset(BITS, 2 * wave, n, q4));
  uint32_t w[2 * BITS];
#pragma unroll
  for (int i = 0; i < BITS / 2; ++i) *reinterpret_cast<uint4*>(w + 4 * i) = src[i];
  const uint8_t* meta = reinterpret_cast<const uint8_t*>(P.c.v_meta) + unit * P.g.v_meta_bytes;
  const int group = wave * 32 / P.g.v_group;
  Meta32<M32> step, zero;
  step.load(meta, group * R + q4 * 8, 32);
  zero.load(meta, (P.g.ngv + group) * R + q4 * 8, 32);
  // channels 32 w + n and 32 w + 16 + n of a token lie side by side in LDS: one write for both
  uint8_t* image = &s_rows[0][0];
  uint8_t* column = image + q4 * VROW + (16 * wave + n) * sizeof(Two);
  constexpr int PER = 8 / BITS;   // codes of a byte
#pragma unroll
  for (int i = 0; i < BITS; ++i)
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      constexpr uint32_t mask = BITS == 2 ? 0x03030303u : 0x0f0f0f0fu;
      const uint32_t v0 = w[i] >> (k * BITS) & mask, v1 = w[BITS + i] >> (k * BITS) & mask;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int m = kmeta_pos_of_chan(BITS, (4 * i + j) * PER + k);   // 8 kk + e: token 16 e + 4 kk + q4
        const float a = step.at(m), z = zero.at(m);
        const float c0 = (float)(v0 >> (8 * j) & 0xffu), c1 = (float)(v1 >> (8 * j) & 0xffu);
        *reinterpret_cast<Two*>(column + (16 * (m % 8) + 4 * (m / 8)) * VROW) =
            ZP_MIN ? pair<OUT>(fmaf(c0, a, z), fmaf(c1, a, z)) : pair<OUT>((c0 - z) * a, (c1 - z) * a);
      }
    }
  __syncthreads();
  // a lane's 16 bytes are N channels of one of the two: the same half of N pairs
  constexpr int N = 16 / sizeof(OUT), LANES = D / N;
  const int c = tid % LANES * N, second = c / 16 % 2;
#pragma unroll 4
  for (int t = t_lo + tid / LANES; t < t_hi; t += 256 / LANES) {
    const uint4* p = reinterpret_cast<const uint4*>(image + t * VROW + (c / 32 * 16 + c % 16) * sizeof(Two));
    const uint4 lo4 = p[0], hi4 = p[1];
    uint4 v;
    if (sizeof(OUT) == 2) {
      const uint32_t half = second ? 0x07060302u : 0x05040100u;
      v = make_uint4(__builtin_amdgcn_perm(lo4.y, lo4.x, half), __builtin_amdgcn_perm(lo4.w, lo4.z, half),
                     __builtin_amdgcn_perm(hi4.y, hi4.x, half), __builtin_amdgcn_perm(hi4.w, hi4.z, half));
    } else {
      v = second ? make_uint4(lo4.y, lo4.w, hi4.y, hi4.w) : make_uint4(lo4.x, lo4.z, hi4.x, hi4.z);
    }
    store_row(out + t * row_bytes + c * sizeof(OUT), v);
  }
}

template <int BITS, typename OUT, bool M32> void launch(const ReadParams& P, dim3 grid, hipStream_t st) {
  if (P.c.cfg.zp_mode == OSCAR_ZP_MIN)
    hipLaunchKernelGGL((oscar_cache_read_kernel<BITS, OUT, M32, true>), grid, dim3(256), 0, st, P);
  else
    hipLaunchKernelGGL((oscar_cache_read_kernel<BITS, OUT, M32, false>), grid, dim3(256), 0, st, P);
}
template <int BITS, typename OUT> void launch(const ReadParams& P, dim3 grid, hipStream_t st) {
  if (P.g.meta_bytes == 4)
    launch<BITS, OUT, true>(P, grid, st);
  else
    launch<BITS, OUT, false>(P, grid, st);
}
template <typename OUT> void launch(const ReadParams& P, dim3 grid, hipStream_t st) {
  if (P.g.bits == 2)
    launch<2, OUT>(P, grid, st);
  else
    launch<4, OUT>(P, grid, st);
}

}  // namespace

extern "C" int oscar_cache_read(const oscar_cache* cache, const int32_t* starts, int32_t T, void* k, void* v,
                                int32_t out_dtype, void* stream) {
  const int rc = oscar_check_cache(cache);
  if (rc != OSCAR_OK) return rc;
  if (T < 0 || cache->num_pages <= 0) return OSCAR_ERR_INVALID_ARG;
  if (out_dtype != OSCAR_F32 && out_dtype != OSCAR_BF16 && out_dtype != OSCAR_F16) return OSCAR_ERR_INVALID_ARG;
  if (((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15) != 0) return OSCAR_ERR_INVALID_ARG;
  if (cache->cfg.n_kv_heads > 65535 || cache->batch > 65535) return OSCAR_ERR_INVALID_ARG;
  if (T == 0) return OSCAR_OK;
  if (!k && !v) return OSCAR_ERR_INVALID_ARG;
  ReadParams P;
  P.k = k;
  P.v = v;
  P.starts = starts;
  P.c = *cache;
  P.g = make_geom(cache->cfg.bits, cache->cfg.k_group, cache->cfg.v_group, cache->cfg.meta_dtype);
  P.T = T;
  // pages that T tokens from anywhere can touch, and no more than a sequence has with its window
  int64_t blocks = starts ? ((int64_t)T - 1) / R + 2 : ((int64_t)T - 1) / R + 1;
  if (blocks > (int64_t)cache->max_pages_per_seq + 1) blocks = (int64_t)cache->max_pages_per_seq + 1;
  if (k && v) blocks *= 2;
  if (blocks >= 1 << 24) return OSCAR_ERR_INVALID_ARG;   // (fewer than 2^32 threads)
  const dim3 grid((unsigned)blocks, cache->cfg.n_kv_heads, cache->batch);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (out_dtype == OSCAR_F32)
    launch<float>(P, grid, st);
  else if (out_dtype == OSCAR_BF16)
    launch<__hip_bfloat16>(P, grid, st);
  else
    launch<__half>(P, grid, st);
  if (hipGetLastError() != hipSuccess) return OSCAR_ERR_HIP;
  return OSCAR_OK;
}
