// oscar_cache_read: keys and values of a range of tokens, out of the packed cache.
//
//   k_t = H(n_t K_u,t) / sqrt(128),  K_u,tj = Delta_gj (c_tj - z_gj)      (H is its own inverse)
//   v_tj = Delta_tg (c_tj - z_tg)
// and from the window K_u and V as they stand (float zero-points: Delta c + zero).
//
// What bounds it: 86 bytes a token and kv head are read (2-bit codes) and 512 written (16-bit), so it is a
// stream of writes.  A workgroup takes the keys or the values of one page of one kv head, and each of its waves a
// quarter without waiting for the others: 32 tokens' keys (two tiles, whose chunks a lane loads with one access,
// 1 KB a wave) or 32 channels' values.  A lane holds 32 channels of a token: five Hadamard stages are in its
// registers, two are exchanges inside a quad of lanes.  Either goes through LDS so that a wave writes rows of
// 256 (keys) or 64 bytes (values) whole.
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

// the 32 codes of a lane's chunk as floats, in their natural order
template <int BITS> __device__ __forceinline__ void unpack_chunk(const uint32_t* w, float (&x)[32]) {
#pragma unroll
  for (int u = 0; u < 32; ++u) x[u] = (float)((w[u * BITS / 32] >> (u * BITS % 32)) & ((1u << BITS) - 1u));
}

// 8 metadata numbers from 16-byte aligned storage
template <bool M32> __device__ __forceinline__ void load_meta8(const uint8_t* base, int idx, float (&x)[8]) {
  if (M32) {
    const float4* p = reinterpret_cast<const float4*>(base + (size_t)idx * 4);
    const float4 a = p[0], b = p[1];
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  } else {
    const uint4 w = *reinterpret_cast<const uint4*>(base + (size_t)idx * 2);
    const __half* h = reinterpret_cast<const __half*>(&w);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __half2float(h[i]);
  }
}

__device__ __forceinline__ float dequant(float c, float step, float zero, bool zp_min) {
  return zp_min ? fmaf(c, step, zero) : (c - zero) * step;
}

// Between a wave's writes to its own LDS and its reads of what other lanes wrote: LDS operations of one wave
// execute in order, the compiler must not move them.
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

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
  const int q4 = threadIdx.x & 3;
  const float s0 = q4 & 1 ? -1.0f : 1.0f, s1 = q4 & 2 ? -1.0f : 1.0f;
#pragma unroll
  for (int i = 0; i < 32; ++i) x[i] = fmaf(x[i], s0, partner<0>(x[i]));
#pragma unroll
  for (int i = 0; i < 32; ++i) x[i] = fmaf(x[i], s1, partner<1>(x[i])) * mul;
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

template <int BITS, typename OUT, bool M32>
__global__ __launch_bounds__(256) void oscar_cache_read_kernel(ReadParams P) {
  typedef typename Pair<OUT>::Type Two;
  // a wave's rows: 16 tokens' keys, or 128 tokens' values of 32 channels; padded so that rows written at once by
  // different lanes fall on other banks
  constexpr int KROW = D * sizeof(OUT) + 32, VROW = 32 * sizeof(OUT) + 16;
  constexpr int BYTES = 16 * KROW > R * VROW ? 16 * KROW : R * VROW;
  __shared__ __align__(16) uint8_t s_rows[4][BYTES];
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
  const bool zp_min = P.c.cfg.zp_mode == OSCAR_ZP_MIN;
  // row `page * R + t` of the outputs
  const int64_t out_row = (((int64_t)b * P.T + page * R - start) * Hkv + h) * D;
  const int64_t row_bytes = (int64_t)Hkv * D * sizeof(OUT);

  if (!values) {
    uint8_t* out = reinterpret_cast<uint8_t*>(reinterpret_cast<OUT*>(P.k) + out_row);
    const bool rotated = P.c.cfg.rotation == OSCAR_ROTATION_ON;
    uint32_t w[2 * BITS];
    float norm[2], step[32], zero[32];
    if (!window) {
      const uint8_t* codes = reinterpret_cast<const uint8_t*>(P.c.k_codes) + unit * P.g.k_codes_bytes;
      const uint4* src = reinterpret_cast<const uint4*>(codes + chunk_offset(BITS, 2 * wave, n, q4));
#pragma unroll
      for (int i = 0; i < BITS / 2; ++i) *reinterpret_cast<uint4*>(w + 4 * i) = src[i];
      // the two tiles lie in one group of 32, 64 or 128 tokens
      const uint8_t* meta = reinterpret_cast<const uint8_t*>(P.c.k_meta) + unit * P.g.k_meta_bytes;
      const int group = wave * 32 / P.g.k_group;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        float a[8], z[8];
        load_meta8<M32>(meta, group * D + 32 * q4 + 8 * kk, a);
        load_meta8<M32>(meta, (P.g.ngk + group) * D + 32 * q4 + 8 * kk, z);
#pragma unroll
        for (int e = 0; e < 8; ++e) step[slot_index(BITS, kk, e)] = a[e], zero[slot_index(BITS, kk, e)] = z[e];
      }
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
        unpack_chunk<BITS>(w + i * BITS, x);
#pragma unroll
        for (int u = 0; u < 32; ++u) x[u] = dequant(x[u], step[u], zero[u], zp_min);
        nm = norm[i];
      } else {
        const __half* src = reinterpret_cast<const __half*>(P.c.res_k) + (unit * R + t0 + n) * D + 32 * q4;
#pragma unroll
        for (int u = 0; u < 32; ++u) x[u] = __half2float(src[u]);
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
        if (t >= t_lo && t < t_hi) *reinterpret_cast<uint4*>(out + t * row_bytes + c) = v;
      }
      wave_lds_fence();
    }
    return;
  }

  uint8_t* out = reinterpret_cast<uint8_t*>(reinterpret_cast<OUT*>(P.v) + out_row) + 32 * wave * sizeof(OUT);
  if (window) {
    // 32 channels of a token a lane
    for (int t = t_lo + lane; t < t_hi; t += 64) {
      Two* row = reinterpret_cast<Two*>(out + t * row_bytes);
      const int64_t at = (unit * R + t) * D + 32 * wave;
#pragma unroll 4
      for (int u = 0; u < 32; u += 2)
        row[u / 2] = pair<OUT>(load_io(P.c.res_v, at + u, P.c.cfg.io_dtype), load_io(P.c.res_v, at + u + 1, P.c.cfg.io_dtype));
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
  float a[4][8], z[4][8];
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) {
    load_meta8<M32>(meta, group * R + (4 * kk + q4) * 8, a[kk]);
    load_meta8<M32>(meta, (P.g.ngv + group) * R + (4 * kk + q4) * 8, z[kk]);
  }
  float x[2][32];
  unpack_chunk<BITS>(w, x[0]);
  unpack_chunk<BITS>(w + BITS, x[1]);
#pragma unroll
  for (int kk = 0; kk < 4; ++kk)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // channels n and 16 + n of a token lie side by side in LDS: one write for both
      const int t = 16 * e + 4 * kk + q4, u = slot_index(BITS, kk, e);
      *reinterpret_cast<Two*>(rows + t * VROW + n * sizeof(Two)) =
          pair<OUT>(dequant(x[0][u], a[kk][e], z[kk][e], zp_min), dequant(x[1][u], a[kk][e], z[kk][e], zp_min));
    }
  wave_lds_fence();
  // a lane takes 16 bytes of channels n .. and the 16 bytes of channels 16 + n .. beside them
  constexpr int N = 16 / sizeof(OUT), LANES = 16 / N;
#pragma unroll 4
  for (int t = t_lo + lane / LANES; t < t_hi; t += 64 / LANES) {
    const int c = lane % LANES;
    const uint4* p = reinterpret_cast<const uint4*>(rows + t * VROW + c * 32);
    const uint4 lo4 = p[0], hi4 = p[1];
    uint4 first, second;
    if (sizeof(OUT) == 2) {
      first = make_uint4(__builtin_amdgcn_perm(lo4.y, lo4.x, 0x05040100u), __builtin_amdgcn_perm(lo4.w, lo4.z, 0x05040100u),
                         __builtin_amdgcn_perm(hi4.y, hi4.x, 0x05040100u), __builtin_amdgcn_perm(hi4.w, hi4.z, 0x05040100u));
      second = make_uint4(__builtin_amdgcn_perm(lo4.y, lo4.x, 0x07060302u), __builtin_amdgcn_perm(lo4.w, lo4.z, 0x07060302u),
                          __builtin_amdgcn_perm(hi4.y, hi4.x, 0x07060302u), __builtin_amdgcn_perm(hi4.w, hi4.z, 0x07060302u));
    } else {
      first = make_uint4(lo4.x, lo4.z, hi4.x, hi4.z);
      second = make_uint4(lo4.y, lo4.w, hi4.y, hi4.w);
    }
    *reinterpret_cast<uint4*>(out + t * row_bytes + c * 16) = first;
    *reinterpret_cast<uint4*>(out + t * row_bytes + 16 * sizeof(OUT) + c * 16) = second;
  }
}

template <int BITS, typename OUT> void launch(const ReadParams& P, dim3 grid, hipStream_t st) {
  if (P.g.meta_bytes == 4)
    hipLaunchKernelGGL((oscar_cache_read_kernel<BITS, OUT, true>), grid, dim3(256), 0, st, P);
  else
    hipLaunchKernelGGL((oscar_cache_read_kernel<BITS, OUT, false>), grid, dim3(256), 0, st, P);
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
  const dim3 grid((unsigned)(k && v ? 2 * blocks : blocks), cache->cfg.n_kv_heads, cache->batch);
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
