// The 4-bit key/value cache on the device: where a token's codes and parameters lie, and what they stand for.
//
// A pool is [n_pages][H_kv] runs of head_bytes bytes, one run per page and key/value head (the layout of pasa.h):
//   K codes [page][d/2] | V codes [page][d/2] | K parameters [page][d/group] | V parameters [page][d/group]
// A parameter is one 32-bit word: the scale s (bf16) in its low half, the minimum m (bf16) in its high half; a code c of
// its group stands for s c + m.  A code word holds 8 channels, channel i of the 8 in bits 4i .. 4i+3.  V word w holds the channels
// 8w .. 8w+7.  K word q * (d/32) + j holds the channels 32j + 8q .. + 7: the d/32 words of one q are one load, and each of
// them lies in another run of 32 channels, so that a matrix instruction over one word per lane stays inside a group.
#pragma once
#include "pasa_cache_kernels.hpp"
#include "pasa_device.hpp"

PASA_DEVICE float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
PASA_DEVICE float bf16_high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

constexpr float kLn2 = 0.6931471805599453f;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(4))) const int32_t const_i32;  // read by scalar loads

// N words at once
template <int N>
PASA_DEVICE void load_words(const uint8_t* base, uint32_t off, uint32_t (&w)[N]) {
  if constexpr (N == 4) {
    const uint4 v = *reinterpret_cast<const uint4*>(base + off);
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
  } else if constexpr (N == 2) {
    const uint2 v = *reinterpret_cast<const uint2*>(base + off);
    w[0] = v.x; w[1] = v.y;
  } else {
    static_assert(N == 1, "");
    w[0] = *reinterpret_cast<const uint32_t*>(base + off);
  }
}

// offsets inside a head's run of a page
template <int D, int G>
struct CacheLayout {
  static constexpr int NG = D / G;         // groups
  static constexpr int CODE = D / 2;       // bytes of a token's codes
  static constexpr int PARAM = 4 * NG;     // bytes of a token's parameters
  PASA_DEVICE static uint32_t k_codes(uint32_t) { return 0u; }
  PASA_DEVICE static uint32_t v_codes(uint32_t page) { return page * CODE; }
  PASA_DEVICE static uint32_t k_params(uint32_t page) { return page * (2 * CODE); }
  PASA_DEVICE static uint32_t v_params(uint32_t page) { return page * (2 * CODE + PARAM); }
};

// the sequence of one batch entry: its tokens, its new rows, and where row 0 of them lies
struct CacheSequence {
  int32_t length;   // cached tokens that the page table can hold
  int32_t rows;     // new rows
  int64_t first;    // position of row 0 (negative if more rows than tokens are declared)
};
PASA_DEVICE CacheSequence cache_sequence(const CacheParams& p, int b, int n) {
  CacheSequence s;
  const int32_t len = max(p.len[b], 0);
  s.rows = p.n_new ? min(max(p.n_new[b], 0), n) : n;
  s.first = (int64_t)len - s.rows;
  s.length = min(len, p.max_pages << p.log_page);
  return s;
}
// how many of the sequence's tokens row r of `share` rows a token sees
PASA_DEVICE int cache_limit(const CacheSequence& s, int causal, int share, int r) {
  if (!causal) return s.length;
  const int64_t own = s.first + r / share + 1;
  return own < 0 ? 0 : own < s.length ? (int)own : s.length;
}
