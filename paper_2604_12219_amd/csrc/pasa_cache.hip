// Writing rows of K and V into the 4-bit cache, and reading them back.
//
// A thread owns 8 channels (16 bytes of bf16, one code word) of one token and head, d/8 threads a token, so that a group of 32, 64 or
// 128 channels is 4, 8 or 16 neighbouring lanes and its extremes take two to four exchanges inside a row of 16 lanes.
// Both kernels are one pass over their data: 2 bytes a value on one side, 4 bits and the parameters on the other.  A wave's requests and stores are
// 1 KB of rows and 256 bytes of codes, each in whole lines (a page holds a token's codes together), and a thread has both tensors in flight.
//   Writing is bound by vector instructions beside the reads: 10,800 tokens of 40 heads, d = 128, groups of 64, 221 MB read and 62 MB written in 60 us, 4.7
//   TB/s.  Reading back is bound by the stores: 75,600 tokens of 40 heads, groups of 32, 484 MB read and 1548 MB written in 375 us, 5.4 TB/s (a large
//   copy reaches 4.8, a large fill 6.8).  One token of 8 sequences is latency, 3.3 and 2.6 us.
#include "pasa_cache.hpp"

namespace {

constexpr int kThreads = 256;
constexpr float kMostKey = 16384.f, kMostValue = 0x1p100f;

template <int CTRL>
PASA_DEVICE float dpp_f(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), CTRL, 0xf, 0xf, true));
}
constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;  // lane ^ 1, lane ^ 2, 7 - lane of 8, 15 - lane of 16

PASA_DEVICE uint32_t bf16_round(float x) {  // to nearest, ties to even; x is finite
  const uint32_t u = __float_as_uint(x);
  return (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}

PASA_DEVICE float min_nan(float a, float b) { return __builtin_elementwise_minimum(a, b); }  // NaN if either is
PASA_DEVICE float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// The codes and the parameter word of 8 channels (four words of bf16 pairs) whose group is the G/8 lanes around this one.
//   s = bf16(binary32((max - min) / 15)), 0 below 2^-126;  code = nearest integer to (x - min) / s, ties to even
// with the real quotients.  most: the largest magnitude that can be held.
// Vector instructions are what bounds writing (155 a wave and tensor), so the quotients are binary32, refined by one step: an exact tie, one value in
// 560 of normally distributed ones, then comes out exact and is rounded right.  What lies within 2e-6 of a tie and is not
// shown to be one (the remainder is zero and the difference was exact) is done over in 64 bits, which hardly ever happens; with every tie done over
// in 64 bits, 10,800 tokens of 40 heads took 97 us instead of 60.
template <int G>
PASA_DEVICE uint32_t quantise8(const uint4& raw, uint32_t& param, float most) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
  float x[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = bf16_low(w[i]);
    x[2 * i + 1] = bf16_high(w[i]);
  }
  float lo = x[0], hi = x[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    lo = min_nan(lo, x[i]);
    hi = max_nan(hi, x[i]);
  }
  lo = min_nan(lo, dpp_f<kSwap1>(lo)); hi = max_nan(hi, dpp_f<kSwap1>(hi));
  lo = min_nan(lo, dpp_f<kSwap2>(lo)); hi = max_nan(hi, dpp_f<kSwap2>(hi));
  if constexpr (G >= 64) { lo = min_nan(lo, dpp_f<kHalfMirror>(lo)); hi = max_nan(hi, dpp_f<kHalfMirror>(hi)); }
  if constexpr (G >= 128) { lo = min_nan(lo, dpp_f<kMirror>(lo)); hi = max_nan(hi, dpp_f<kMirror>(hi)); }
  if (!(hi <= most && lo >= -most)) {  // the whole group reads back as NaN
    param = 0x7fc07fc0u;
    return 0u;
  }
  float t = (hi - lo) * (1.0f / 15.0f);
  const int from_middle = (int)(__float_as_uint(t) & 0xffffu) - 0x8000;
  if (from_middle >= -64 && from_middle <= 64) t = (float)(((double)hi - (double)lo) / 15.0);  // (t is within 4 units in the last place)
  uint32_t s_bits = bf16_round(t);
  if (s_bits < 0x0080u) s_bits = 0u;  // below 2^-126, the smallest normal number
  // the minimum is one of the group's own bf16 values; adding 0 makes -0 and +0 the same
  param = s_bits | (__float_as_uint(lo + 0.0f) & 0xffff0000u);
  if (s_bits == 0u) return 0u;
  const float s = __uint_as_float(s_bits << 16), inv = __builtin_amdgcn_rcpf(s);
  float d[8], y[8], r[8], worst = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    d[i] = x[i] - lo;
    const float y0 = d[i] * inv;
    y[i] = fmaf(fmaf(-y0, s, d[i]), inv, y0);
    r[i] = rintf(y[i]);  // at most 15: (max - min) / s <= 15 (1 + 2^-8)
    worst = fmaxf(worst, fabsf(y[i] - r[i]));
  }
  if (worst > 0.499998f) {  // |y - exact| < 16 * 2^-24
    bool doubt = false;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      doubt |= fabsf(y[i] - r[i]) > 0.499998f && (fmaf(-y[i], s, d[i]) != 0.f || d[i] + lo != x[i]);
    if (doubt) {
#pragma unroll
      for (int i = 0; i < 8; ++i) r[i] = (float)rint(((double)x[i] - (double)lo) / (double)s);
    }
  }
  const float a = fmaf(fmaf(fmaf(r[3], 16.f, r[2]), 16.f, r[1]), 16.f, r[0]), b = fmaf(fmaf(fmaf(r[7], 16.f, r[6]), 16.f, r[5]), 16.f, r[4]);
  return (uint32_t)a | ((uint32_t)b << 16);
}

// the row this thread works on (i < 0: none), and where its token lies in the pool (null: nowhere)
struct Row {
  int i, b, h;
  int64_t pos;
};
template <int D>
PASA_DEVICE Row row_of(const CacheRowsParams& p) {
  constexpr int TPT = D / 8;  // threads of a token
  Row r;
  r.i = blockIdx.x * (kThreads / TPT) + (int)threadIdx.x / TPT;
  r.h = blockIdx.y;
  r.b = blockIdx.z;
  const CacheSequence s = cache_sequence(p.c, r.b, p.n);
  r.pos = s.first + r.i;
  if (r.i >= s.rows || r.pos < 0 || r.pos >= ((int64_t)p.c.max_pages << p.c.log_page)) r.i = -1;
  return r;
}
PASA_DEVICE int64_t row_offset(const CacheRowsParams& p, const Row& r) { return r.b * p.stride_b + r.h * p.stride_h + r.i * p.stride_n; }
PASA_DEVICE uint8_t* run_of(const CacheRowsParams& p, const Row& r) {
  const int page = p.c.pages[(int64_t)r.b * p.c.max_pages + (r.pos >> p.c.log_page)];
  return page < 0 || page >= p.c.n_pages ? nullptr : p.c.pool + ((int64_t)page * p.c.H_kv + r.h) * p.c.head_bytes;
}

template <int D>
PASA_DEVICE uint32_t k_word(uint32_t chunk) { return (chunk & 3u) * (D / 32) + (chunk >> 2); }  // word of channels 8 chunk ..

template <int D, int G>
__global__ void __launch_bounds__(kThreads) cache_write_kernel(CacheRowsParams p) {
  typedef CacheLayout<D, G> L;
  const Row row = row_of<D>(p);
  if (row.i < 0) return;
  const uint32_t chunk = threadIdx.x % (D / 8), page = 1u << p.c.log_page, slot = (uint32_t)row.pos & (page - 1u);
  const int64_t off = row_offset(p, row) + 8 * chunk;
  const uint4 kr = *reinterpret_cast<const uint4*>(p.k + off);
  const uint4 vr = *reinterpret_cast<const uint4*>(p.v + off);
  uint8_t* const run = run_of(p, row);  // (after the rows have been requested)
  uint32_t kp, vp;
  const uint32_t kc = quantise8<G>(kr, kp, kMostKey), vc = quantise8<G>(vr, vp, kMostValue);
  if (!run) return;
  *reinterpret_cast<uint32_t*>(run + L::k_codes(page) + slot * L::CODE + 4 * k_word<D>(chunk)) = kc;
  *reinterpret_cast<uint32_t*>(run + L::v_codes(page) + slot * L::CODE + 4 * chunk) = vc;
  if (chunk % (G / 8) == 0) {
    const uint32_t at = slot * L::PARAM + 4 * (chunk / (G / 8));
    *reinterpret_cast<uint32_t*>(run + L::k_params(page) + at) = kp;
    *reinterpret_cast<uint32_t*>(run + L::v_params(page) + at) = vp;
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
  const Row row = row_of<D>(p);
  if (row.i < 0) return;
  const uint8_t* const run = run_of(p, row);
  if (!run) return;
  const uint32_t chunk = threadIdx.x % (D / 8), page = 1u << p.c.log_page, slot = (uint32_t)row.pos & (page - 1u);
  const uint32_t at = slot * L::PARAM + 4 * (chunk / (G / 8));
  const uint32_t kc = *reinterpret_cast<const uint32_t*>(run + L::k_codes(page) + slot * L::CODE + 4 * k_word<D>(chunk));
  const uint32_t vc = *reinterpret_cast<const uint32_t*>(run + L::v_codes(page) + slot * L::CODE + 4 * chunk);
  const uint32_t kp = *reinterpret_cast<const uint32_t*>(run + L::k_params(page) + at);
  const uint32_t vp = *reinterpret_cast<const uint32_t*>(run + L::v_params(page) + at);
  const int64_t off = row_offset(p, row) + 8 * chunk;
  *reinterpret_cast<uint4*>(p.k + off) = values8(kc, kp);
  *reinterpret_cast<uint4*>(p.v + off) = values8(vc, vp);
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
