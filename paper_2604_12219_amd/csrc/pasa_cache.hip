// Writing rows of K and V into the 4-bit cache, and reading them back.
//
// A thread owns 8 channels (16 bytes of bf16, one code word) of one token and head, d/8 threads a token, so that a group of 32, 64 or
// 128 channels is 4, 8 or 16 neighbouring lanes and its extremes take two to four exchanges inside a row of 16 lanes.
// Both kernels are one pass over their data: 2 bytes a value on one side, 4 bits and the parameters on the other.
#include "pasa_cache.hpp"

namespace {

constexpr int kThreads = 256;
constexpr uint32_t kMostKey = 0x46800000u, kMostValue = 0x71800000u;  // 16384, 2^100

template <int CTRL>
PASA_DEVICE float dpp_f(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), CTRL, 0xf, 0xf, true));
}
template <int CTRL>
PASA_DEVICE uint32_t dpp_u(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xf, 0xf, true);
}
constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;  // lane ^ 1, lane ^ 2, 7 - lane of 8, 15 - lane of 16

PASA_DEVICE uint32_t bf16_round(float x) {  // to nearest, ties to even; x is finite
  const uint32_t u = __float_as_uint(x);
  return (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}

// The codes and the parameter word of 8 channels (four words of bf16 pairs) whose group is the G/8 lanes around this one.
//   s = bf16(binary32((max - min) / 15)), 0 below 2^-126;  code = nearest integer to (x - min) / s, ties to even
// with the real quotients: binary32 decides where its error cannot matter, the rest is done over in 64 bits.
// most: the largest bit pattern of |x| that can be held
template <int G>
PASA_DEVICE uint32_t quantise8(const uint4& raw, uint32_t& param, uint32_t most) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
  float x[8];
  uint32_t top = 0u;  // largest |x| as a bit pattern (infinities and NaN are larger than any number)
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = bf16_low(w[i]);
    x[2 * i + 1] = bf16_high(w[i]);
    top = max(top, max((w[i] << 16) & 0x7fff0000u, w[i] & 0x7fff0000u));
  }
  float lo = x[0], hi = x[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    lo = fminf(lo, x[i]);
    hi = fmaxf(hi, x[i]);
  }
  lo = fminf(lo, dpp_f<kSwap1>(lo)); hi = fmaxf(hi, dpp_f<kSwap1>(hi)); top = max(top, dpp_u<kSwap1>(top));
  lo = fminf(lo, dpp_f<kSwap2>(lo)); hi = fmaxf(hi, dpp_f<kSwap2>(hi)); top = max(top, dpp_u<kSwap2>(top));
  if constexpr (G >= 64) {
    lo = fminf(lo, dpp_f<kHalfMirror>(lo)); hi = fmaxf(hi, dpp_f<kHalfMirror>(hi)); top = max(top, dpp_u<kHalfMirror>(top));
  }
  if constexpr (G >= 128) {
    lo = fminf(lo, dpp_f<kMirror>(lo)); hi = fmaxf(hi, dpp_f<kMirror>(hi)); top = max(top, dpp_u<kMirror>(top));
  }
  if (top > most) {  // the whole group reads back as NaN
    param = 0x7fc07fc0u;
    return 0u;
  }
  // halves: the difference of the largest and the smallest bf16 exceeds binary32
  const float lo_half = 0.5f * lo;
  float t = fmaf(0.5f, hi, -lo_half) * (2.0f / 15.0f);
  const int from_middle = (int)(__float_as_uint(t) & 0xffffu) - 0x8000;
  if (from_middle >= -64 && from_middle <= 64) t = (float)(((double)hi - (double)lo) / 15.0);  // (t is within 4 units in the last place)
  uint32_t s_bits = bf16_round(t);
  if (s_bits < 0x0080u) s_bits = 0u;  // below 2^-126, the smallest normal number
  // the minimum is one of the group's own bf16 values; adding 0 makes -0 and +0 the same
  param = s_bits | (__float_as_uint(lo + 0.0f) & 0xffff0000u);
  if (s_bits == 0u) return 0u;
  const float s = __uint_as_float(s_bits << 16);
  const float inv2 = 2.0f * __builtin_amdgcn_rcpf(s);
  uint32_t word = 0u;
  float worst = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float y = fmaf(0.5f, x[i], -lo_half) * inv2;
    const float r = rintf(y);
    worst = fmaxf(worst, fabsf(y - r));
    word |= (uint32_t)fminf(r, 15.0f) << (4 * i);
  }
  if (worst > 0.49998f) {  // |y - exact| < 15.1 * 5 * 2^-24 < 1e-5: only such quotients can be rounded the wrong way
    word = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) word |= (uint32_t)fmin(rint(((double)x[i] - (double)lo) / (double)s), 15.0) << (4 * i);
  }
  return word;
}

// which token this thread works on, and where it lies in the pool (null: nowhere)
struct Place {
  uint8_t* run;
  uint32_t slot;
  int64_t row_off;
};
template <int D, int G>
PASA_DEVICE Place place(const CacheRowsParams& p) {
  constexpr int TPT = D / 8;  // threads of a token
  const int i = blockIdx.x * (kThreads / TPT) + (int)threadIdx.x / TPT, h = blockIdx.y, b = blockIdx.z;
  Place a{nullptr, 0u, 0};
  const CacheSequence s = cache_sequence(p.c, b, p.n);
  const int64_t pos = s.first + i;
  if (i >= s.rows || pos < 0 || pos >= ((int64_t)p.c.max_pages << p.c.log_page)) return a;
  const int page = p.c.pages[(int64_t)b * p.c.max_pages + (pos >> p.c.log_page)];
  if (page < 0 || page >= p.c.n_pages) return a;
  a.run = p.c.pool + ((int64_t)page * p.c.H_kv + h) * p.c.head_bytes;
  a.slot = (uint32_t)pos & ((1u << p.c.log_page) - 1u);
  a.row_off = b * p.stride_b + h * p.stride_h + i * p.stride_n;
  return a;
}

template <int D>
PASA_DEVICE uint32_t k_word(uint32_t chunk) { return (chunk & 3u) * (D / 32) + (chunk >> 2); }  // word of channels 8 chunk ..

template <int D, int G>
__global__ void __launch_bounds__(kThreads) cache_write_kernel(CacheRowsParams p) {
  typedef CacheLayout<D, G> L;
  const Place a = place<D, G>(p);
  if (!a.run) return;
  const uint32_t chunk = threadIdx.x % (D / 8), page = 1u << p.c.log_page;
  const uint4 kr = *reinterpret_cast<const uint4*>(p.k + a.row_off + 8 * chunk);
  const uint4 vr = *reinterpret_cast<const uint4*>(p.v + a.row_off + 8 * chunk);
  uint32_t kp, vp;
  const uint32_t kc = quantise8<G>(kr, kp, kMostKey), vc = quantise8<G>(vr, vp, kMostValue);
  *reinterpret_cast<uint32_t*>(a.run + L::k_codes(page) + a.slot * L::CODE + 4 * k_word<D>(chunk)) = kc;
  *reinterpret_cast<uint32_t*>(a.run + L::v_codes(page) + a.slot * L::CODE + 4 * chunk) = vc;
  if (chunk % (G / 8) == 0) {
    const uint32_t at = a.slot * L::PARAM + 4 * (chunk / (G / 8));
    *reinterpret_cast<uint32_t*>(a.run + L::k_params(page) + at) = kp;
    *reinterpret_cast<uint32_t*>(a.run + L::v_params(page) + at) = vp;
  }
}

PASA_DEVICE uint4 values8(uint32_t codes, uint32_t param) {
  const float s = bf16_low(param), m = bf16_high(param);
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {  // s c is exact (12 bits), so a value is rounded once to binary32 and once to bf16
    const float a = fmaf(s, (float)((codes >> (8 * i)) & 15u), m), b = fmaf(s, (float)((codes >> (8 * i + 4)) & 15u), m);
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 r = {(__bf16)a, (__bf16)b};
    w[i] = __builtin_bit_cast(uint32_t, r);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int D, int G>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(CacheRowsParams p) {
  typedef CacheLayout<D, G> L;
  const Place a = place<D, G>(p);
  if (!a.run) return;
  const uint32_t chunk = threadIdx.x % (D / 8), page = 1u << p.c.log_page;
  const uint32_t at = a.slot * L::PARAM + 4 * (chunk / (G / 8));
  const uint32_t kc = *reinterpret_cast<const uint32_t*>(a.run + L::k_codes(page) + a.slot * L::CODE + 4 * k_word<D>(chunk));
  const uint32_t vc = *reinterpret_cast<const uint32_t*>(a.run + L::v_codes(page) + a.slot * L::CODE + 4 * chunk);
  const uint32_t kp = *reinterpret_cast<const uint32_t*>(a.run + L::k_params(page) + at);
  const uint32_t vp = *reinterpret_cast<const uint32_t*>(a.run + L::v_params(page) + at);
  *reinterpret_cast<uint4*>(p.k + a.row_off + 8 * chunk) = values8(kc, kp);
  *reinterpret_cast<uint4*>(p.v + a.row_off + 8 * chunk) = values8(vc, vp);
}

template <int D, int G>
hipError_t launch_rows(const CacheRowsParams& p, bool write, hipStream_t stream) {
  constexpr int rows = kThreads / (D / 8);
  const dim3 grid((p.n + rows - 1) / rows, p.c.H_kv, p.c.B);
  if (write) cache_write_kernel<D, G><<<grid, kThreads, 0, stream>>>(p);
  else cache_read_kernel<D, G><<<grid, kThreads, 0, stream>>>(p);
  return hipGetLastError();
}

hipError_t launch_rows(const CacheRowsParams& p, bool write, hipStream_t stream) {
  if (p.c.d == 64) return p.c.group == 32 ? launch_rows<64, 32>(p, write, stream) : launch_rows<64, 64>(p, write, stream);
  return p.c.group == 32 ? launch_rows<128, 32>(p, write, stream)
       : p.c.group == 64 ? launch_rows<128, 64>(p, write, stream) : launch_rows<128, 128>(p, write, stream);
}

}  // namespace

hipError_t pasa_launch_cache_write(const CacheRowsParams& p, hipStream_t stream) { return launch_rows(p, true, stream); }
hipError_t pasa_launch_cache_read(const CacheRowsParams& p, hipStream_t stream) { return launch_rows(p, false, stream); }
