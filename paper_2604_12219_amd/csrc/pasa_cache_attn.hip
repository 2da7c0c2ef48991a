// Attention of new rows over the 4-bit cache.
//   o = sum_t w_t v_t / sum_t w_t,  w_t = exp(scale q . k_t),  over the cached tokens t that a row may see
// in one pass with a running maximum and sum per row.
#include "pasa_cache.hpp"

namespace {

constexpr float kLn2 = 0.6931471805599453f;

// One wave per row.  A lane holds one key of a tile of 64 for the logits and D/64 channels for the sums over the values.
template <int D, int G>
__global__ void __launch_bounds__(64) cache_attn_kernel(CacheAttnParams p) {
  typedef CacheLayout<D, G> L;
  const int lane = threadIdx.x, i = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const CacheSequence seq = cache_sequence(p.c, b, p.n);
  if (i >= seq.rows) return;
  const int hkv = h / (p.H / p.c.H_kv);
  const uint32_t page = 1u << p.c.log_page;
  int64_t limit = seq.length;
  if (p.causal && seq.first + i + 1 < limit) limit = seq.first + i + 1;
  __shared__ float q[D];
  __shared__ float w[64];
  const uint16_t* const qrow = p.q + b * p.stride_b + h * p.stride_h + i * p.stride_n;
  for (int ch = lane; ch < D; ch += 64) q[ch] = __uint_as_float((uint32_t)qrow[ch] << 16);
  __syncthreads();
  float m = -INFINITY, l = 0.f, o[D / 64] = {};
  const int32_t* const table = p.c.pages + (int64_t)b * p.c.max_pages;
  auto run_of = [&](int64_t pos) -> const uint8_t* {  // null: a page number that is not followed
    const int pg = table[pos >> p.c.log_page];
    return pg < 0 || pg >= p.c.n_pages ? nullptr : p.c.pool + ((int64_t)pg * p.c.H_kv + hkv) * p.c.head_bytes;
  };
  for (int64_t base = 0; base < limit; base += 64) {
    const int64_t pos = base + lane;
    const uint8_t* const run = pos < limit ? run_of(pos) : nullptr;
    float z = -INFINITY;
    if (run) {
      const uint32_t slot = (uint32_t)pos & (page - 1u);
      float dot = 0.f;
      for (int word = 0; word < D / 8; ++word) {
        const uint32_t c = *reinterpret_cast<const uint32_t*>(run + L::k_codes(page) + slot * L::CODE + 4 * word);
        const int ch = 32 * (word % (D / 32)) + 8 * (word / (D / 32));
        const uint32_t par = *reinterpret_cast<const uint32_t*>(run + L::k_params(page) + slot * L::PARAM + 4 * (ch / G));
        for (int e = 0; e < 8; ++e) dot = fmaf(q[ch + e], fmaf(bf16_low(par), (float)((c >> (4 * e)) & 15u), bf16_high(par)), dot);
      }
      z = dot * p.scale;
    }
    float top = z;
    for (int x = 32; x >= 1; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
    const float m_new = fmaxf(m, top), ref = m_new == -INFINITY ? 0.f : m_new;
    const float corr = exp2f(m - ref), weight = exp2f(z - ref);
    float sum = weight;
    for (int x = 32; x >= 1; x >>= 1) sum += __shfl_xor(sum, x);
    m = m_new;
    l = l * corr + sum;
    w[lane] = weight;
    __syncthreads();
    for (int t = 0; t < D / 64; ++t) o[t] *= corr;
    for (int key = 0; key < 64; ++key) {
      const int64_t at = base + key;
      const uint8_t* const vrun = at < limit ? run_of(at) : nullptr;
      if (!vrun) continue;
      const uint32_t slot = (uint32_t)at & (page - 1u);
      for (int t = 0; t < D / 64; ++t) {
        const int ch = 64 * t + lane;
        const uint32_t c = vrun[L::v_codes(page) + slot * L::CODE + ch / 2] >> (4 * (ch & 1));
        const uint32_t par = *reinterpret_cast<const uint32_t*>(vrun + L::v_params(page) + slot * L::PARAM + 4 * (ch / G));
        o[t] = fmaf(w[key], fmaf(bf16_low(par), (float)(c & 15u), bf16_high(par)), o[t]);
      }
    }
    __syncthreads();
  }
  // a row that sees nothing is zero, its normaliser empty
  uint16_t* const orow = p.o + b * p.stride_b + h * p.stride_h + i * p.stride_n;
  for (int t = 0; t < D / 64; ++t) {
    const __bf16 r = (__bf16)(l == 0.f ? 0.f : o[t] / l);
    orow[64 * t + lane] = __builtin_bit_cast(uint16_t, r);
  }
  if (p.lse && lane == 0) p.lse[((int64_t)b * p.H + h) * p.n + i] = l == 0.f ? -INFINITY : m * kLn2 + logf(l);
}

template <int D, int G>
hipError_t launch(const CacheAttnParams& p, hipStream_t stream) {
  cache_attn_kernel<D, G><<<dim3(p.n, p.H, p.c.B), 64, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t pasa_launch_cache_attn(const CacheAttnParams& p, hipStream_t stream) {
  if (p.c.d == 64) return p.c.group == 32 ? launch<64, 32>(p, stream) : launch<64, 64>(p, stream);
  return p.c.group == 32 ? launch<128, 32>(p, stream) : p.c.group == 64 ? launch<128, 64>(p, stream) : launch<128, 128>(p, stream);
}
