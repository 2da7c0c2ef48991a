// Attention of many new rows over the 4-bit cache: the matrix-core side of pasa_cache_attn.hip.
//
// Bound by the matrix cores, as attention over bf16 is: tiles of 64 tokens in LDS, and instruction streams over them (pasa_cache_pipes.hpp).
// What differs is how a tile gets there: a thread holds a few code words of one token, of K and of V, converts them and writes them
// to the other half of the ring while this tile is worked on.  The conversion is shared by all rows of a workgroup, hence eight waves
// and 256 rows: with four waves and 128 it costs twice as much a row.
// Measured (median of 23 passes in a row, this kernel alone): 3600 rows of 40 heads over 75,600 tokens, d = 128, groups of 32, 5.99 ms, 930 TFLOP/s; 4680 rows
// of 12 heads over 32,760, 1.03 ms.  Per wave and tile 34
// matrix and 252 vector instructions (150 in attention over bf16), the matrix cores busy 0.56 and the vector units 0.59 of the cycles at the 1.79 GHz that
// the power leaves (bf16: 0.70 at 1.6).  A conversion that costs nothing would take 10 % off, keys rounded to bf16 3 %.
//
//   V: bf16(s c + m).  An and-or (and one shift for half of a word) makes fp16 numbers 1024 + c or 64 + c of two codes, a mixed fma
//     s c + m of each (s (1024 + c) + (m - 1024 s): the rounding of that is 2^-13 of s), a conversion rounds two of them to bf16: 2.1 instructions a
//     value.  Values beyond +-2^100 do not exist in a cache (pasa_cache_write), so 1024 s is finite.
//   K: fp16 2^f s (c - 8): a shift and an and-or make 1 + c/16 of two codes, a packed fma 16 s (1 + c/16) - 24 s: 1.5 instructions a value.  What that
//     leaves out, sum_g (m_g + 8 s_g) sum_{i in g} q_i, is one more matrix instruction per 32 keys, with both factors as sums of two fp16 numbers
//     (22 bits).  With keys rounded to bf16 instead lse would be off by 1e-5.
//   Powers of two.  s has 8 bits and c - 8 at most 3 or is a power of two, so s (c - 8) is exact where fp16 has the exponents for it: s from 2^-17 to
//     2^11.  A cache holds scales down to 2^-126.  So the groups of a key/value head are shifted to the top of fp16's range, each by the power 2^f that
//     its largest operand over the sequence's tokens allows (cache_key_range_kernel; 2^13 to 2^14 then), and the queries by 2^-f; a row's queries
//     then by one more power that puts the largest of them between 2^7 and 2^8 (the sum of 128 is an fp16 number), which the row's logit scale takes
//     back.  So K is exact for scales down to 2^-30 of its group's largest operand and q down to 2^-24 of the row's largest; what is smaller is rounded to 2^-25, that is
//     2^-38 and 2^-32 of the largest.
#include "pasa_cache.hpp"
#include "pasa_cache_pipes.hpp"

namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// 8 values of a word of codes in bf16; b0 = m - 1024 s, b1 = m - 64 s
PASA_DEVICE uint4 values8(uint32_t x, float s, float b0, float b1) {
  float v[8];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const f16x2 a = __builtin_bit_cast(f16x2, ((x >> (8 * i)) & 0x000f000fu) | 0x64006400u);  // 1024 + c of channels 2 i and 2 i + 4
    const f16x2 b = __builtin_bit_cast(f16x2, ((x >> (8 * i)) & 0x00f000f0u) | 0x54005400u);  // 64 + c of channels 2 i + 1 and 2 i + 5
    v[2 * i] = fmaf((float)a[0], s, b0);
    v[2 * i + 4] = fmaf((float)a[1], s, b0);
    v[2 * i + 1] = fmaf((float)b[0], s, b1);
    v[2 * i + 5] = fmaf((float)b[1], s, b1);
  }
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bf16x2 p = {(__bf16)v[2 * i], (__bf16)v[2 * i + 1]};
    r[i] = __builtin_bit_cast(uint32_t, p);
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}

// 8 keys' values s (c - 8) of a word of codes in fp16, in the order 0 4 1 5 2 6 3 7; f = (16 s, -24 s)
PASA_DEVICE uint4 keys8(uint32_t x, uint32_t f) {
  const f16x2 a = __builtin_shufflevector(__builtin_bit_cast(f16x2, f), __builtin_bit_cast(f16x2, f), 0, 0);
  const f16x2 b = __builtin_shufflevector(__builtin_bit_cast(f16x2, f), __builtin_bit_cast(f16x2, f), 1, 1);
  const uint32_t h[4] = {((x << 6) & 0x03c003c0u) | 0x3c003c00u, ((x << 2) & 0x03c003c0u) | 0x3c003c00u, ((x >> 2) & 0x03c003c0u) | 0x3c003c00u,
                         ((x >> 6) & 0x03c003c0u) | 0x3c003c00u};
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(f16x2, h[i]), a, b));
  return make_uint4(r[0], r[1], r[2], r[3]);
}

PASA_DEVICE bool finite_param(uint32_t w) { return (w & 0x7f80u) != 0x7f80u && (w & 0x7f800000u) != 0x7f800000u; }

// What a thread converts of a group of 128 tokens: the quarter q of one token's K (its code words q * (d/32) ..) and a quarter of its V, with
// the parameters they need.  The 16 tokens of a wave lie in one page, so what depends on the page is scalar and the lane's offsets stay the same.
template <int D, int G>
struct Quarter {
  typedef CacheLayout<D, G> L;
  static constexpr int N = D / 32;  // code words of K, and of V
  // The lane's tokens among the wave's 16: 4 lanes a token.  16 neighbouring lanes write 16-byte chunks of 4 tokens at a time; K's (chunk 4 j + q of a row)
  // fall into different banks for 4 tokens in a row, V's (chunk (d/32) q + j) for 4 tokens that differ in the two bits which the LDS layout puts
  // into the low bits of a chunk's place (lds_chunk_off): a four-way conflict otherwise, 450 cycles a tile.
  static PASA_DEVICE int k_token(int lane) { return lane >> 2; }
  static PASA_DEVICE int v_token(int lane) {
    const int t = lane >> 2;
    return D == 128 ? ((t & 3) << 2) | (t >> 2) : (t & 1) | ((t & 2) << 1) | ((t & 4) >> 1) | (t & 8);
  }
  struct Offsets {
    uint32_t k_code, k_par, v_code, v_par;
    PASA_DEVICE void init(int lane) {
      const int q = lane & 3, kt = k_token(lane), vt = v_token(lane);
      k_code = kt * L::CODE + 4 * N * q;
      k_par = kt * L::PARAM;
      v_code = vt * L::CODE + 4 * N * q;
      v_par = vt * L::PARAM + 4 * (8 * N * q / G);
    }
  };
  uint32_t k_code[N], k_par[L::NG], v_code[N], v_par;
  // run, slot: page and slot of the wave's first token.  (The offsets are hidden from the compiler, or else it adds them to the page's address
  // as 64-bit numbers on the vector unit, instead of using the instruction's scalar base.)
  PASA_DEVICE void load_k(const uint8_t* run, uint32_t page, uint32_t slot, const Offsets& at) {
    uint32_t code = at.k_code, par = at.k_par;
    asm("" : "+v"(code), "+v"(par));
    load_words<N>(run + (L::k_codes(page) + slot * L::CODE), code, k_code);
    load_words<L::NG>(run + (L::k_params(page) + slot * L::PARAM), par, k_par);
  }
  PASA_DEVICE void load_v(const uint8_t* run, uint32_t page, uint32_t slot, const Offsets& at) {
    uint32_t code = at.v_code, par = at.v_par, w[1];
    asm("" : "+v"(code), "+v"(par));
    load_words<N>(run + (L::v_codes(page) + slot * L::CODE), code, v_code);
    load_words<1>(run + (L::v_params(page) + slot * L::PARAM), par, w);
    v_par = w[0];
  }
};
// 2^f of K's groups: 16 2^f and -24 2^f of each, 2^f of the lane's own quarter's
template <int NG>
struct KeyFactors {
  float f16[NG], f24[NG], own;
};
// the same, taken for conversion
template <int D, int G>
struct Taken {
  typedef CacheLayout<D, G> L;
  static constexpr int N = D / 32;
  uint32_t kc[N], kf[N], vc[N], v_par;  // kf: 2^f times 16 s and -24 s of a K word's group in fp16
  float vs, vm0, vm1;                   // s, m - 1024 s, m - 64 s of the V words' group
  uint2 bias;  // the token's offset operands of group q: (hi, hi, lo, 0) of 2^f (m + 8 s), to be multiplied with (hi, lo, hi, 0) of the group's sum of q
  PASA_DEVICE void take_k(const Quarter<D, G>& x, int q, const KeyFactors<D / G>& up) {
    uint32_t own = x.k_par[0];
#pragma unroll
    for (int g = 1; g < L::NG; ++g) own = q == g ? x.k_par[g] : own;
    const float mid = fmaf(8.f, bf16_low(own), bf16_high(own)) * up.own;
    const _Float16 hi = (_Float16)mid, lo = (_Float16)(mid - (float)hi);
    const f16x2 x0 = {hi, hi}, x1 = {lo, (_Float16)0.f};
    bias = make_uint2(__builtin_bit_cast(uint32_t, x0), __builtin_bit_cast(uint32_t, x1));
    if (q >= L::NG) bias = make_uint2(0u, 0u);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float s = bf16_low(x.k_par[j * 32 / G]);
      const f16x2 f = {(_Float16)(up.f16[j * 32 / G] * s), (_Float16)(up.f24[j * 32 / G] * s)};
      kf[j] = __builtin_bit_cast(uint32_t, f);
      kc[j] = x.k_code[j];
    }
  }
  PASA_DEVICE void factors(uint32_t par) {
    vs = bf16_low(par);
    vm0 = fmaf(-1024.f, vs, bf16_high(par));
    vm1 = fmaf(-64.f, vs, bf16_high(par));
  }
  PASA_DEVICE void take_v(const Quarter<D, G>& x) {
    v_par = x.v_par;
    factors(v_par);
#pragma unroll
    for (int j = 0; j < N; ++j) vc[j] = x.v_code[j];
  }
};

// The largest magnitude of an operand that K makes, max(8 |s|, |m + 8 s|), of every group of a head over the sequence's tokens, as its biased exponent (0:
// all are zero), byte g of a word for group g; parameters that are not finite do not count.  Workgroup (j, head, sequence) takes the j-th of key_parts
// runs of tokens.  Bound by a chain of loads (length, page, parameters): 12 heads of 32,760 tokens 5 us, 40 heads of 75,600, 48 MB of parameters, 11 us.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
PASA_DEVICE uint32_t max_u16x2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
constexpr int kRangeThreads = 256;
template <int D, int G>
__global__ void __launch_bounds__(kRangeThreads) cache_key_range_kernel(CacheAttnParams p) {
  typedef CacheLayout<D, G> L;
  constexpr int NG = D / G, U = 4, WAVES = kRangeThreads / 64;
  __shared__ uint32_t s_even[WAVES], s_odd[WAVES];
  const int j = blockIdx.x, hkv = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  const CacheSequence seq = cache_sequence(p.c, b, p.n);
  const int per = (seq.length + p.key_parts - 1) / p.key_parts, first = j * per, last = seq.rows > 0 ? min(first + per, seq.length) : 0;
  const uint32_t page = 1u << p.c.log_page;
  const int32_t* const table = p.c.pages + (int64_t)b * p.c.max_pages;
  float top[NG];
#pragma unroll
  for (int g = 0; g < NG; ++g) top[g] = 0.f;
  for (int at = first; at < last; at += U * kRangeThreads) {  // (the threads behind the last token look at that one again)
    int pos[U], pg[U];
    uint32_t w[U][NG];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      pos[u] = min(at + u * kRangeThreads + tid, last - 1);
      pg[u] = table[pos[u] >> p.c.log_page];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool ok = pg[u] >= 0 && pg[u] < p.c.n_pages;
      const uint8_t* const run = p.c.pool + ((int64_t)(ok ? pg[u] : 0) * p.c.H_kv + hkv) * p.c.head_bytes;
      load_words<NG>(run, L::k_params(page) + ((uint32_t)pos[u] & (page - 1u)) * L::PARAM, w[u]);
      if (!ok)
#pragma unroll
        for (int g = 0; g < NG; ++g) w[u][g] = 0u;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const float s = bf16_low(w[u][g]), m = bf16_high(w[u][g]), size = fmaxf(8.f * fabsf(s), fabsf(fmaf(8.f, s, m)));
        if (finite_param(w[u][g])) top[g] = fmaxf(top[g], size);
      }
  }
  uint32_t pair[2] = {0u, 0u};  // groups 0 and 2, 1 and 3
#pragma unroll
  for (int g = 0; g < NG; ++g) pair[g & 1] |= (top[g] == 0.f ? 0u : max(__float_as_uint(top[g]) >> 23, 1u)) << (8 * (g & 2));
  for (int d = 32; d >= 1; d >>= 1)
#pragma unroll
    for (int i = 0; i < 2; ++i) pair[i] = max_u16x2(pair[i], (uint32_t)__shfl_xor((int)pair[i], d));
  if ((tid & 63) == 0) { s_even[tid >> 6] = pair[0]; s_odd[tid >> 6] = pair[1]; }
  __syncthreads();
  if (tid != 0) return;
#pragma unroll
  for (int w = 1; w < WAVES; ++w) {
    pair[0] = max_u16x2(pair[0], s_even[w]);
    pair[1] = max_u16x2(pair[1], s_odd[w]);
  }
  p.key_range[((int64_t)b * p.c.H_kv + hkv) * p.key_parts + j] = pair[0] | (pair[1] << 8);
}

// ---- who does what ----
// An item is a (sequence, run of ROWS rows), numbered e = b * row_tiles + run, of one key/value head; its weight is the number of tiles that its rows
// see (at least one where there are rows: somebody has to write them).  All items of all heads in a row, head by head, are a line of
// tiles that the workgroups divide evenly, each a piece of `piece` of them: so an item can be shared by several workgroups, and the last ones have no
// less to do than the first, whatever the lengths are (they are known on the device only).  Against one workgroup an item: 40 heads of 15 items,
// 600 workgroups on 256 compute units, 14,400 rows and 75,600 tokens, 7640 -> 6300 us.
// A workgroup's piece holds at most two parts of items: one at its start (slot 2 w of the partial results) and one at its end (slot 2 w + 1).  The last
// workgroup's end is the end of an item: its second slot holds K's magnitudes (cache_attn_plan).
struct CacheItem {
  int b, row0, rows;  // rows: of the sequence, times the share of heads
  CacheSequence seq;
};
PASA_DEVICE CacheItem cache_item(const CacheAttnParams& p, int e) {
  CacheItem it;
  it.b = e / p.row_tiles;
  it.row0 = (e % p.row_tiles) * p.wg_rows;
  it.seq = cache_sequence(p.c, it.b, p.n);
  it.rows = p.share * it.seq.rows;
  return it;
}
PASA_DEVICE int row_limit(const CacheAttnParams& p, const CacheSequence& seq, int r) { return cache_limit(seq, p.causal, p.share, r); }
PASA_DEVICE int item_tiles(const CacheAttnParams& p, const CacheItem& it) { return (row_limit(p, it.seq, min(it.row0 + p.wg_rows, it.rows) - 1) + 63) >> 6; }
PASA_DEVICE int item_weight(const CacheAttnParams& p, int e) {
  const CacheItem it = cache_item(p, e);
  return it.row0 >= it.rows ? 0 : max(item_tiles(p, it), 1);
}
// the first item from e on that has rows (p.c.B * row_tiles if there is none); e is uniform, the lanes look at 64 sequences at once
PASA_DEVICE int next_item(const CacheAttnParams& p, int e, int lane) {
  const int end = p.c.B * p.row_tiles;
  if (e >= end) return end;
  const CacheItem it = cache_item(p, e);
  if (it.row0 < it.rows) return e;
  for (int b0 = it.b + 1; b0 < p.c.B; b0 += 64) {
    const uint64_t there = __builtin_amdgcn_ballot_w64(b0 + lane < p.c.B && cache_sequence(p.c, min(b0 + lane, p.c.B - 1), p.n).rows > 0);
    if (there != 0u) return (b0 + __builtin_ctzll(there)) * p.row_tiles;
  }
  return end;
}
PASA_DEVICE int64_t wave_inclusive_sum(int64_t x, int lane) {
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t y = __shfl_up((long long)x, d);
    if (lane >= d) x += y;
  }
  return x;
}

constexpr int kTileWaves = 8, kTileRows = 32 * kTileWaves;

template <int D, int G>
__global__ void __launch_bounds__(kTileWaves * 64, 2) cache_tile_kernel(CacheAttnParams p) {
  typedef CacheLayout<D, G> L;
  constexpr int WAVES = kTileWaves, ROWS = kTileRows, TILE = 64 * 2 * D, GROUP = 2 * TILE, BIAS = 64 * 32;
  // Two groups of two tiles (128 tokens) of K, two of V, the offset operands of K's tokens.  V group v holds the tiles 2 v and 2 v + 1, K group v the
  // tiles 2 v + 1 and 2 v + 2 (counted from the workgroup's first one): the logits are a tile ahead.  Group v lies in half v & 1.
  __shared__ __attribute__((aligned(1024))) char ring[4 * GROUP + 4 * BIAS];
  __shared__ bool bad[2][128];  // V tokens that not every row sees: has values that are not finite
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), ql = lane & 31, h = lane >> 5;

  // ---- this workgroup's piece ----
  __shared__ int64_t s_sum[WAVES], s_at[2];
  const int items = p.c.B * p.row_tiles;
  int64_t head_tiles = 0;  // of one key/value head
  for (int e = tid; e < items; e += WAVES * 64) head_tiles += item_weight(p, e);
  head_tiles = wave_inclusive_sum(head_tiles, lane);
  if (lane == 63) s_sum[wave] = head_tiles;
  __syncthreads();
  head_tiles = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) head_tiles += s_sum[w];
  const int64_t all_tiles = head_tiles * p.c.H_kv, piece = max((all_tiles + gridDim.x - 1) / gridDim.x, (int64_t)kCacheMinPiece);
  int64_t at = blockIdx.x * piece;
  const int64_t end = min(at + piece, all_tiles);
  if (tid == 0) p.merge[blockIdx.x].parts = 0;
  if (at >= end) return;
  int hkv = (int)(at / head_tiles), item = 0, off = 0;  // where the piece starts: tile `off` of the item
  {
    const int64_t want = at - hkv * head_tiles;
    int64_t before = 0;  // tiles of the items before e0
    for (int e0 = 0;; e0 += WAVES * 64) {
      const int e = e0 + tid, weight = e < items ? item_weight(p, e) : 0;
      const int64_t incl = wave_inclusive_sum(weight, lane);
      __syncthreads();  // s_sum has been read
      if (lane == 63) s_sum[wave] = incl;
      __syncthreads();
      int64_t first = before + incl - weight, all = before;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        if (w < wave) first += s_sum[w];
        all += s_sum[w];
      }
      if (want >= first && want < first + weight) { s_at[0] = e; s_at[1] = want - first; }
      if (want < all) break;
      before = all;
    }
    __syncthreads();
    item = __builtin_amdgcn_readfirstlane((int)s_at[0]);
    off = __builtin_amdgcn_readfirstlane((int)s_at[1]);
    hkv = __builtin_amdgcn_readfirstlane(hkv);
  }

  for (bool first_part = true; at < end; first_part = false) {
  const CacheItem it = cache_item(p, item);
  const int b = it.b, row0 = it.row0, rows = it.rows, share = p.share, last_row = min(row0 + ROWS, rows) - 1;
  const CacheSequence seq = it.seq;
  const int limit_all = __builtin_amdgcn_readfirstlane(row_limit(p, seq, row0)), limit_any = __builtin_amdgcn_readfirstlane(row_limit(p, seq, last_row));
  const int tiles = (limit_any + 63) >> 6, weight = max(tiles, 1);
  const int take_tiles = (int)min((int64_t)(weight - off), end - at);
  const int t_begin = __builtin_amdgcn_readfirstlane(min(off, tiles)), t_end = __builtin_amdgcn_readfirstlane(min(off + take_tiles, tiles));
  const bool whole_item = take_tiles == weight;
  const uint32_t page = 1u << p.c.log_page;
  const_i32* const table = (const_i32*)(p.c.pages + (int64_t)b * p.c.max_pages);

  // this wave's rows, a lane's row in either half-wave
  const int row = row0 + wave * 32 + ql;
  const int own = min(row, last_row), i_own = own / share, h_own = hkv * share + own % share;
  const int64_t row_off = b * p.stride_b + h_own * p.stride_h + i_own * p.stride_n;
  const int limit = row_limit(p, seq, own);
  const int limit_wave = __builtin_amdgcn_readfirstlane(row_limit(p, seq, min(row0 + wave * 32 + 31, last_row)));
  uint4 q_raw[D / 16];
#pragma unroll
  for (int s = 0; s < D / 16; ++s) q_raw[s] = *reinterpret_cast<const uint4*>(p.q + row_off + 16 * s + 8 * h);
  uint32_t range = lane < p.key_parts ? p.key_range[((int64_t)b * p.c.H_kv + hkv) * p.key_parts + lane] : 0u;

  f32x16 o[D / 32];
#pragma unroll
  for (int t = 0; t < D / 32; ++t) o[t] = f32x16{0};
  float m = -INFINITY, l = 0.f;

  const uint32_t ring_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)ring;
  // the lane's addresses of the operand fetches in the first K tile, its offset operands and the first V tile
  uint32_t ka[D / 16], va[2 * (D / 32)];
  const uint32_t ab = ring_base + (uint32_t)(4 * GROUP + h * (BIAS / 2) + ql * 16);
#pragma unroll
  for (int s = 0; s < D / 16; ++s) ka[s] = (ring_base + (uint32_t)lds_chunk_off<D>(ql, h)) ^ (uint32_t)(s << 5);
  {
    const int i = lane & 15, r = 4 * h + (i >> 2), c = 16 * ((lane >> 4) & 1) + 4 * (i & 3);
#pragma unroll
    for (int t = 0; t < D / 32; ++t) {
      va[2 * t] = (ring_base + (uint32_t)(2 * GROUP + lds_chunk_off<D>(r, c >> 3) + (c & 7) * 2)) ^ (uint32_t)(t << 6);
      va[2 * t + 1] = (ring_base + (uint32_t)(2 * GROUP + lds_chunk_off<D>(r + 8, c >> 3) + (c & 7) * 2)) ^ (uint32_t)(t << 6);
    }
  }

  // ---- how tiles get into LDS ----
  typedef Quarter<D, G> Raw;
  const int token0 = wave * 16, quarter = lane & 3, k_token = token0 + Raw::k_token(lane), v_token = token0 + Raw::v_token(lane);  // of a group
  Raw raw;
  typename Raw::Offsets raw_at;
  raw_at.init(lane);
  auto is_page = [&](int pg) -> bool { return pg >= 0 && pg < p.c.n_pages; };
  // Whether all pages of the workgroup's tokens are followed (or else every tile is masked: `followed` below looks each of them up)
  bool pages_good = true;
  {
    const int first = t_begin * 64 >> p.c.log_page, last = (min(64 * t_end, seq.length) - 1) >> p.c.log_page;
    for (int j = first + tid; j <= last; j += WAVES * 64) pages_good &= is_page(p.c.pages[(int64_t)b * p.c.max_pages + j]);
    pages_good = __syncthreads_and(pages_good);
  }
  auto followed = [&](int tile) -> uint32_t {  // bit t: the page of tokens 64 tile + 16 t .. is followed
    uint32_t bits = 0u;
#pragma unroll
    for (int t = 0; t < 4; ++t) bits |= (uint32_t)is_page(table[min(64 * tile + 16 * t, seq.length - 1) >> p.c.log_page]) << t;
    return bits;
  };
  const int t_whole = pages_good ? max(min(limit_all >> 6, t_end), t_begin) : t_begin;  // before it every row sees every token
  // The page of a wave's tokens is looked up a step (of two tiles) before their codes are requested, these a step before they are converted.
  // (Before the first and behind the last tile: some tokens of the sequence, converted and not used)
  const int64_t pool_page = (int64_t)p.c.H_kv * p.c.head_bytes;
  const uint8_t* const pool_head = p.c.pool + (int64_t)hkv * p.c.head_bytes;
  auto k_pos = [&](int v) -> int { return 64 * (t_begin + 2 * v + 1) + token0; };  // first of the wave's tokens of K group v
  auto v_pos = [&](int v) -> int { return 64 * (t_begin + 2 * v) + token0; };
  auto look_up = [&](int pos) -> int { return table[min(max(pos, 0), seq.length - 1) >> p.c.log_page]; };
  auto run_of = [&](int pg) -> const uint8_t* { return pool_head + (is_page(pg) ? pg : 0) * pool_page; };
  auto slot_of = [&](int pos) -> uint32_t { return (uint32_t)pos & (page - 1u); };
  int k_page, v_page;  // of the groups to be requested next
  Taken<D, G> cv;
  KeyFactors<D / G> up;
  auto request = [&](int v) {  // groups v, whose pages have been looked up
    raw.load_k(run_of(k_page), page, slot_of(k_pos(v)), raw_at);
    raw.load_v(run_of(v_page), page, slot_of(v_pos(v)), raw_at);
    k_page = look_up(k_pos(v + 1));
    v_page = look_up(v_pos(v + 1));
  };
  auto take = [&](int v) {  // the groups v, which have been requested; the ones after them are
    cv.take_k(raw, quarter, up);
    cv.take_v(raw);
    request(v + 1);
  };
  auto store_bias = [&](int v) {
    *reinterpret_cast<uint2*>(ring + 4 * GROUP + (2 * (v & 1) + (k_token >> 6)) * BIAS + (quarter >> 1) * (BIAS / 2) + (k_token & 63) * 16 + (quarter & 1) * 8) = cv.bias;
  };
  auto store_k = [&](int v) {
    store_bias(v);
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
      *reinterpret_cast<uint4*>(ring + (v & 1) * GROUP + lds_chunk_off<D>(k_token, 4 * j + quarter)) = keys8(cv.kc[j], cv.kf[j]);
  };
  // Weights of zero do not hide values that are not finite from the rows that do not see them: in a tile that is not whole such values
  // become zeros, and `bad` says so to the rows that do see the token (whose outputs are NaN then in all channels, not only in those of that group)
  auto store_v = [&](int v) {
    if (t_begin + 2 * v + 2 > t_whole) {
      const int pos = v_pos(v) + Raw::v_token(lane);
      const bool finite = finite_param(cv.v_par);
      const bool hide = pos >= 64 * t_whole && (!finite || pos >= limit_any || (!pages_good && !is_page(look_up(v_pos(v)))));
      const uint64_t not_finite = __builtin_amdgcn_ballot_w64(!finite) >> (lane & 60);
      if (quarter == 0) bad[v & 1][v_token] = (not_finite & 15u) != 0u;
      if (hide) cv.factors(0u);
    }
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
      *reinterpret_cast<uint4*>(ring + 2 * GROUP + (v & 1) * GROUP + lds_chunk_off<D>(v_token, D / 32 * quarter + j)) = values8(cv.vc[j], cv.vs, cv.vm0, cv.vm1);
  };
  auto meet = [&]() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

  // the addresses for tile x of the four in the ring
  struct At {
    uint32_t ka[D / 16], ab, va[2 * (D / 32)];
  };
  auto k_at = [&](At& at, int x) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) at.ka[s] = ka[s] + (uint32_t)(x * TILE);
    at.ab = ab + (uint32_t)(x * BIAS);
  };
  auto v_at = [&](At& at, int x) {
#pragma unroll
    for (int t = 0; t < 2 * (D / 32); ++t) at.va[t] = va[t] + (uint32_t)(x * TILE);
  };

  if (t_begin < t_end) {  // K group -1 is requested
    k_page = look_up(k_pos(-1));
    raw.load_k(run_of(k_page), page, slot_of(k_pos(-1)), raw_at);
    k_page = look_up(k_pos(0));
    v_page = look_up(v_pos(0));
  }

  // the powers of two of K's groups: the largest operand between 2^13 and 2^14, so that 24 s is an fp16 number (2^120 at most: 24 s 2^f in binary32)
  constexpr int NG = D / G;
  constexpr int kNoKeys = 1 << 12;  // of a group whose keys are zero: q does not matter and becomes zero
  int f[NG];
  {
    uint32_t even = range & 0x00ff00ffu, odd = (range >> 8) & 0x00ff00ffu;
    for (int d = 32; d >= 1; d >>= 1) {
      even = max_u16x2(even, (uint32_t)__shfl_xor((int)even, d));
      odd = max_u16x2(odd, (uint32_t)__shfl_xor((int)odd, d));
    }
    even = __builtin_amdgcn_readfirstlane(even);
    odd = __builtin_amdgcn_readfirstlane(odd);
    up.own = 0.f;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const int e = (int)(((g & 1 ? odd : even) >> (8 * (g & 2))) & 0xffu), own_f = min(140 - e, 120);
      f[g] = e == 0 ? kNoKeys : own_f;
      const uint32_t pow16 = (uint32_t)(own_f + 131) << 23;  // (put together from bits, so that they are scalars)
      up.f16[g] = __uint_as_float(pow16);
      up.f24[g] = __uint_as_float(pow16 | 0x80400000u);
      if (quarter == g) up.own = __uint_as_float((uint32_t)(own_f + 127) << 23);
    }
  }
  // 2^(7 - e - f) q in fp16, 2^e the power of two at the largest 2^-f |q| of the row, in the order of a word's codes; qb: the groups' sums of that
  f16x8 qf[D / 16], qb;
  float c_row;  // logit scale times log2(e) times 2^(e - 7)
  {
    int e = -kNoKeys;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      uint32_t top = 0u;
#pragma unroll
      for (int s = g * (G / 16); s < (g + 1) * (G / 16); ++s) {
        const uint32_t w[4] = {q_raw[s].x, q_raw[s].y, q_raw[s].z, q_raw[s].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) top = max(top, max((w[i] << 16) & 0x7fff0000u, w[i] & 0x7fff0000u));
      }
      const u32x2 both = __builtin_amdgcn_permlane32_swap(top, top, false, false);
      top = max(both[0], both[1]);
      if (top != 0u && f[g] != kNoKeys) e = max(e, (int)max(top >> 23, 1u) - 127 - f[g]);
    }
    if (e == -kNoKeys) e = 0;
    c_row = fmaxf(__builtin_ldexpf(p.scale, e - 7), 0x1p-126f);  // (never zero: -inf, the logit of a key that is not seen, has to stay that)
    float sum[D / G];
#pragma unroll
    for (int g = 0; g < D / G; ++g) sum[g] = 0.f;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      const uint32_t w[4] = {q_raw[s].x, q_raw[s].y, q_raw[s].z, q_raw[s].w};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = i & 1 ? bf16_high(w[i / 2]) : bf16_low(w[i / 2]);
        const _Float16 y = (_Float16)__builtin_ldexpf(x, 7 - e - f[s * 16 / G]);
        qf[s][i < 4 ? 2 * i : 2 * i - 7] = y;
        sum[s * 16 / G] += (float)y;
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {  // quarters 2 h and 2 h + 1
      float t = 0.f;
#pragma unroll
      for (int g = 0; g < D / G; ++g) {
        const float all = half_swap_sum(sum[g]);
        if (2 * h + i == g) t = all;
      }
      const _Float16 hi = (_Float16)t, lo = (_Float16)(t - (float)hi);
      qb[4 * i] = hi; qb[4 * i + 1] = lo; qb[4 * i + 2] = hi; qb[4 * i + 3] = (_Float16)0.f;
    }
  }

  // ---- a tile of which not every row sees every token; k, v: where its K and V are ----
  auto masked_tile = [&](int tile, int k, int v) {
    if (64 * tile >= limit_wave) return;  // none of the wave's rows sees any of it
    At at;
    k_at(at, k);
    v_at(at, v);
    f32x16 s0, s1;
    bf16x8 pf[4];
    cache_pipes::logits(at.ka, at.ab, qf, qb, s0, s1);
    const int rel = limit - 64 * tile - 4 * h;
    const uint32_t bits = followed(tile);
    int lim[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) lim[t] = (bits >> t) & 1u ? rel : -64;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int key = mfma_row(r, 0);
      if (key >= lim[r >> 3]) s0[r] = -INFINITY;
      if (key + 32 >= lim[2 + (r >> 3)]) s1[r] = -INFINITY;
    }
    float mx = fmaxf(s0[0], s1[0]);
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(fmaxf(mx, s0[r]), s1[r]);
    mx = half_swap_max(mx) * c_row;
    if (__builtin_amdgcn_ballot_w64(mx > m)) {
      const float m_new = mx > m ? mx + 8.f : m;  // (as in the pipelined steps)
      const float corr = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      l *= corr;
#pragma unroll
      for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] *= corr;
    }
    const float neg = m == -INFINITY ? 0.f : -m;  // nothing seen yet: every weight is exp2(-inf) = 0
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s0[r] = __builtin_amdgcn_exp2f(fmaf(s0[r], c_row, neg));
      s1[r] = __builtin_amdgcn_exp2f(fmaf(s1[r], c_row, neg));
      sum += s0[r] + s1[r];
    }
    l += sum;
#pragma unroll
    for (int i = 0; i < 8; ++i) {  // the weights to bf16, the type of the matrix operands
      pf[0][i] = (__bf16)s0[i];
      pf[1][i] = (__bf16)s0[8 + i];
      pf[2][i] = (__bf16)s1[i];
      pf[3][i] = (__bf16)s1[8 + i];
    }
    pipes::cols_x_p64(at.va[0], at.va[1], pf, o);
    uint64_t not_finite = __builtin_amdgcn_ballot_w64(bad[v >> 1][64 * (v & 1) + lane]);
    if (not_finite != 0u) {  // hardly ever
      float add = 0.f;
      for (; not_finite != 0u; not_finite &= not_finite - 1u) {
        const int key = __builtin_ctzll(not_finite);
        if (64 * tile + key < limit && ((bits >> (key >> 4)) & 1u)) add = NAN;
      }
#pragma unroll
      for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] += add;
    }
  };

  if (t_begin < t_end) {
    // K groups -1 (for the first tile) and 0, V group 0; groups 1 requested
    cv.take_k(raw, quarter, up);
    request(0);
    store_k(-1);
    take(0);
    store_k(0);
    store_v(0);
    meet();
    int tile = t_begin, v = 0;  // V group v and K groups v - 1 and v are in LDS, groups v + 1 requested
    if (tile < t_whole) {
      // a run of whole tiles in pipelined steps, each with P V of one tile and the logits of the next, two steps between meetings
      pipes::PipeState st;
      At at;
      k_at(at, 3);  // tile 0 is the second one of K group -1
      cache_pipes::pipe_start(at.ka, at.ab, qf, qb, m, l, c_row, st);
      meet();  // K group -1 may be overwritten
      const uint32_t kst = ring_base + (uint32_t)lds_chunk_off<D>(k_token, quarter), vst = ring_base + (uint32_t)(2 * GROUP + lds_chunk_off<D>(v_token, D / 32 * quarter));
#pragma unroll 1
      for (; tile + 3 < t_whole; tile += 2) {
        take(v + 1);
        store_bias(v + 1);
        // the conversion runs in the shadow of the matrix instructions
        cache_pipes::pipe_steps(v & 1, ka, ab, va, qf, qb, o, m, l, st, c_row, cv.kc, cv.kf, cv.vc, cv.vs, cv.vm0, cv.vm1, kst, vst);
        ++v;
        meet();
      }
      const bool three = tile + 2 < t_whole;  // whole tiles that are left (or one or two): the next V group holds one that is not whole, or is none
      if (three) {
        take(v + 1);
        store_k(v + 1);
        store_v(v + 1);
      }
#pragma unroll 1
      for (int x = 0; x < 2 && tile + 1 < t_whole; ++x, ++tile) {
        k_at(at, 2 * (v & 1) + x);
        v_at(at, 2 * (v & 1) + x);
        cache_pipes::pipe_step(at.ka, at.ab, at.va, qf, qb, o, m, l, st, c_row);
      }
      if (three) {
        ++v;
        meet();
      }
      v_at(at, 2 * (v & 1) + ((tile - t_begin) & 1));
      cache_pipes::pipe_end(at.va, o, m, l, st, c_row);
      ++tile;
      if (((tile - t_begin) & 1) == 0 && tile < t_end) {  // V group v is used up
        take(v + 1);
        meet();
        store_k(v + 1);
        store_v(v + 1);
        ++v;
        meet();
      }
    }
#pragma unroll 1
    while (tile < t_end) {
      // the two tiles of V group v: their K is the second one of K group v - 1 and the first one of K group v
      if (((tile - t_begin) & 1) == 0) {
        masked_tile(tile, 2 * ((v - 1) & 1) + 1, 2 * (v & 1));
        ++tile;
      }
      if (tile < t_end) {
        masked_tile(tile, 2 * (v & 1), 2 * (v & 1) + 1);
        ++tile;
      }
      if (tile < t_end) {
        take(v + 1);
        meet();
        store_k(v + 1);
        store_v(v + 1);
        ++v;
        meet();
      }
    }
  }
  meet();  // the next part's tiles may be written

  l = half_swap_sum(l);
  if (row <= last_row) {
    const int64_t line = ((int64_t)b * p.H + h_own) * p.n + i_own;
    if (whole_item) {  // a row that sees nothing is zero, its normaliser empty
      const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
      for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const bf16x2 x0 = {(__bf16)(o[t][4 * g] * inv), (__bf16)(o[t][4 * g + 1] * inv)};
          const bf16x2 x1 = {(__bf16)(o[t][4 * g + 2] * inv), (__bf16)(o[t][4 * g + 3] * inv)};
          *reinterpret_cast<uint2*>(p.o + row_off + 32 * t + 8 * g + 4 * h) = make_uint2(__builtin_bit_cast(uint32_t, x0), __builtin_bit_cast(uint32_t, x1));
        }
      if (p.lse && h == 0) p.lse[line] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
    } else {
      const int64_t part_row = (2 * blockIdx.x + (first_part ? 0 : 1)) * (int64_t)ROWS + (row - row0);
#pragma unroll
      for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<float4*>(p.part_o + part_row * D + 32 * t + 8 * g + 4 * h) = make_float4(o[t][4 * g], o[t][4 * g + 1], o[t][4 * g + 2], o[t][4 * g + 3]);
      if (h == 0) { p.part_ml[2 * part_row] = m; p.part_ml[2 * part_row + 1] = l; }
    }
  }
  if (tid == 0 && off != 0) {  // not the first part of a shared item: cache_merge_items puts it together
    const int64_t start = at - off;
    const int w0 = (int)(start / piece);
    p.merge[blockIdx.x] = {hkv, item, 2 * w0 + (start % piece != 0 ? 1 : 0), (int)((start + weight - 1) / piece) - w0 + 1};
  }
  at += take_tiles;
  off = 0;
  item = next_item(p, item + 1, lane);
  if (item == items) {
    ++hkv;
    item = next_item(p, 0, lane);
  }
  item = __builtin_amdgcn_readfirstlane(item);
  }
}

// Items that several workgroups share, from their parts (67 MB of them where all 256 workgroups have two of 256 rows of 128 channels: 22 us).  Its time is
// a chain of loads, so four rows go side by side: few parts by one wave, its lanes on 64/LANES parts at a time, workgroup (w, y) on rows 16 y .. of the
// item whose last part workgroup w of cache_tile_kernel had; many parts, of few rows if they are not that many, by the four waves of a workgroup, each
// a quarter, and by the workgroups (w, y) of all parts but the first.
template <int D>
__global__ void __launch_bounds__(256) cache_merge_items(CacheAttnParams p) {
  constexpr int LANES = D / 4, PP = 64 / LANES, R = 4, WAVES = 4;  // lanes of a part's row, parts at a time in a wave, rows
  __shared__ f32x4 s_o[WAVES - 1][R][LANES];
  __shared__ float s_sum[WAVES - 1][R];
  const CacheMerge mg = p.merge[blockIdx.x];
  if (mg.parts == 0) return;
  const CacheItem it = cache_item(p, mg.item);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int part = (int)blockIdx.x - mg.first_slot / 2, last = min((int)(gridDim.y * WAVES * R), it.rows - it.row0) - 1;
  const bool shared = mg.parts > 2 * PP && last < (mg.parts - 1) * (int)gridDim.y * R;  // by the waves, all rows at once
  if (!shared && part != mg.parts - 1) return;
  const int r0 = (shared ? (part - 1) * (int)gridDim.y + (int)blockIdx.y : (int)blockIdx.y * WAVES + wave) * R;
  if (r0 > last) return;
  const int share = p.share, sub = lane / LANES, ch = lane % LANES * 4;
  // part 0 in slot first_slot, the others at the starts of the workgroups after that; rows behind the last one are the last one again, not written
  auto place = [&](int j, int k) -> int64_t {
    return (j == 0 ? mg.first_slot : (int64_t)2 * (mg.first_slot / 2 + j)) * p.wg_rows + min(r0 + k, last);
  };
  float top[R], sum[R];
  f32x4 o[R];
#pragma unroll
  for (int k = 0; k < R; ++k) { top[k] = -INFINITY; sum[k] = 0.f; o[k] = f32x4{0.f, 0.f, 0.f, 0.f}; }
  for (int j = lane; j < mg.parts; j += 64)
#pragma unroll
    for (int k = 0; k < R; ++k) top[k] = fmaxf(top[k], p.part_ml[2 * place(j, k)]);
#pragma unroll
  for (int k = 0; k < R; ++k) {
    for (int d = 32; d >= 1; d >>= 1) top[k] = fmaxf(top[k], __shfl_xor(top[k], d));
    if (top[k] == -INFINITY) top[k] = 0.f;
  }
#pragma unroll 4
  for (int j = (shared ? wave * PP : 0) + sub; j < mg.parts; j += shared ? WAVES * PP : PP) {
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int64_t at = place(j, k);
      const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + 2 * at);
      const f32x4 x = *reinterpret_cast<const f32x4*>(p.part_o + at * D + ch);
      const float f = __builtin_amdgcn_exp2f(ml.x - top[k]);
      sum[k] = fmaf(f, ml.y, sum[k]);
#pragma unroll
      for (int i = 0; i < 4; ++i) o[k][i] = fmaf(f, x[i], o[k][i]);
    }
  }
#pragma unroll
  for (int k = 0; k < R; ++k) {
#pragma unroll
    for (int d = LANES; d < 64; d <<= 1) {
      sum[k] += __shfl_xor(sum[k], d);
#pragma unroll
      for (int i = 0; i < 4; ++i) o[k][i] += __shfl_xor(o[k][i], d);
    }
    if (shared && wave > 0 && sub == 0) {
      s_o[wave - 1][k][lane] = o[k];
      s_sum[wave - 1][k] = sum[k];
    }
  }
  if (shared) {
    __syncthreads();
    if (wave > 0) return;
  }
  if (sub != 0) return;
#pragma unroll
  for (int k = 0; k < R; ++k) {
    if (r0 + k > last) break;
    if (shared)
#pragma unroll
      for (int w = 0; w < WAVES - 1; ++w) {
        o[k] += s_o[w][k][lane];
        sum[k] += s_sum[w][k];
      }
    const int row = it.row0 + r0 + k, i = row / share, h = mg.hkv * share + row % share;
    const float inv = sum[k] == 0.f ? 0.f : 1.f / sum[k];
    const bf16x2 x0 = {(__bf16)(o[k][0] * inv), (__bf16)(o[k][1] * inv)}, x1 = {(__bf16)(o[k][2] * inv), (__bf16)(o[k][3] * inv)};
    *reinterpret_cast<uint2*>(p.o + it.b * p.stride_b + h * p.stride_h + i * p.stride_n + ch) =
        make_uint2(__builtin_bit_cast(uint32_t, x0), __builtin_bit_cast(uint32_t, x1));
    if (p.lse && ch == 0) p.lse[((int64_t)it.b * p.H + h) * p.n + i] = sum[k] == 0.f ? -INFINITY : (top[k] + __builtin_amdgcn_logf(sum[k])) * kLn2;
  }
}

template <int D, int G>
hipError_t launch(const CacheAttnParams& p, hipStream_t stream) {
  cache_key_range_kernel<D, G><<<dim3(p.key_parts, p.c.H_kv, p.c.B), kRangeThreads, 0, stream>>>(p);
  cache_tile_kernel<D, G><<<p.pieces, kTileWaves * 64, 0, stream>>>(p);
  cache_merge_items<D><<<dim3(p.pieces, p.wg_rows / 16), 256, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t pasa_launch_cache_tiles(const CacheAttnParams& p, hipStream_t stream) {
  if (p.c.d == 64) return p.c.group == 32 ? launch<64, 32>(p, stream) : launch<64, 64>(p, stream);
  return p.c.group == 32 ? launch<128, 32>(p, stream) : p.c.group == 64 ? launch<128, 64>(p, stream) : launch<128, 128>(p, stream);
}
