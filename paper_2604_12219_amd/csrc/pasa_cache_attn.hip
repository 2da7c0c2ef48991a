// Attention of new rows over the 4-bit cache.
//   o = sum_t w_t v_t / sum_t w_t,  w_t = exp(scale q . k_t),  over the cached tokens t that a row may see
// in one pass with a running maximum and sum per row.
//
// Rows.  The share = H / H_kv query heads of a key/value head see the same keys, so (row, head of the share) pairs are numbered
// through, r = row * share + head, and a workgroup takes a run of them.
//
// cache_rows_kernel: at most 16 such rows a workgroup, four waves that take tiles of 64 tokens in turn.
//   Bound by memory: d + 8 d/G bytes a token and head are read once, and everything else has to fit beside that.  A code
//   never becomes a number of its own: the bf16 with bits 0x4180 | c << 3 is 16 + c exactly, so one shift and one and-or per two codes
//   make matrix operands of whole words, and scales and minima are applied to the products in binary32:
//     S = sum_g s_g (sum_i q_i (16 + c_i) - 16 sum_i q_i) + m_g sum_i q_i           over the channels i of group g
//     O_i = sum_t (p_t s_t)(16 + c_ti) - 23.5 sum_t (p_t s_t) + sum_t p_t (m_t + 7.5 s_t)
//   (the first subtraction is the accumulator's start value; the second sum, of the rounded p_t s_t, is one more product with ones.  The
//   weights p_t s_t are rounded to bf16; splitting the value at the middle of its range, m + 7.5 s, keeps what that rounding
//   multiplies as small as a value is, |v - middle|, where splitting at m would let it multiply up to twice as much.)
//   Logits: A = Q (rows), B = K codes (columns: keys), 16 keys a matrix instruction, one instruction per 32 channels.  A lane so holds
//   one key, whose scales are one load, and needs a group's scale once for each of its rows.  The rows of a workgroup sit in slots
//   4 x + i of the 16 (x = lane / 16 of the result, i < NR), so a lane computes NR logits a key instead of four.
//   Values: A = weights, B = V codes (columns: channels).  The transposing 4-bit LDS read hands a lane 16 tokens of one channel.
//   A lane's weights of the tokens 16 t + (lane & 15), t = 0..3, are neighbours in the contraction, so they leave as one 8-byte LDS write.
//   Measured: one token of 75,600, 40 heads of 128 channels, 484 MB in 92 us, 5.3 TB/s; 32 sequences of 800 to 8000 tokens, 8 heads with 4 query heads each,
//   184 MB in 38 us, 4.8 TB/s.  With 16 rows vector instructions bound it, some 540 a wave and tile with one group a head and 900 with four: 64 heads of
//   4000 tokens, 33 rows each (three runs of 16), 47 us with the launch.
// Longer sequences are divided among workgroups, each leaving (m, l, o), and cache_merge_kernel puts these together.
#include "pasa_cache.hpp"

#include <type_traits>

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

PASA_DEVICE f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// a word of 8 codes as 16 + c in bf16, in the order 0 4 1 5 2 6 3 7.  The constants come in registers (CodeBits), where an and-or can have them.
struct CodeBits {
  uint32_t mask = 0x00780078u, sixteen = 0x41804180u;
  PASA_DEVICE CodeBits() { asm("" : "+s"(mask), "+v"(sixteen)); }
};
PASA_DEVICE bf16x8 codes_bf16(uint32_t x, const CodeBits& k) {
  const u32x4 w = {((x << 3) & k.mask) | k.sixteen, ((x >> 1) & k.mask) | k.sixteen, ((x >> 5) & k.mask) | k.sixteen, ((x >> 9) & k.mask) | k.sixteen};
  return __builtin_bit_cast(bf16x8, w);
}
// 8 bf16 in that order
PASA_DEVICE bf16x8 code_order(const uint4& w) {
  const u32x4 r = {(w.x & 0xffffu) | (w.z << 16), (w.x >> 16) | (w.z & 0xffff0000u), (w.y & 0xffffu) | (w.w << 16), (w.y >> 16) | (w.w & 0xffff0000u)};
  return __builtin_bit_cast(bf16x8, r);
}

// sum or maximum over the 16 lanes of a row, in every one of them
template <int N>
PASA_DEVICE float row_rotate(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), 0x120 + N, 0xf, 0xf, true));
}
PASA_DEVICE float row16_max(float x) {
  x = fmaxf(x, row_rotate<8>(x)); x = fmaxf(x, row_rotate<4>(x)); x = fmaxf(x, row_rotate<2>(x));
  return fmaxf(x, row_rotate<1>(x));
}
PASA_DEVICE float row16_sum(float x) {
  x += row_rotate<8>(x); x += row_rotate<4>(x); x += row_rotate<2>(x);
  return x + row_rotate<1>(x);
}

PASA_DEVICE void wave_fence() {  // LDS written by lanes of this wave is read by others of it
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// result of row r (of `rows` of sequence b, key/value head hkv), column ch: output or partial result
struct RowPlace {
  int64_t out, lse;
};
PASA_DEVICE RowPlace row_place(const CacheAttnParams& p, int b, int hkv, int share, int r) {
  const int i = r / share, h = hkv * share + r % share;
  return {b * p.stride_b + h * p.stride_h + i * p.stride_n, ((int64_t)b * p.H + h) * p.n + i};
}

constexpr int kWaves = 4;

template <int D, int G, int NR>
__global__ void __launch_bounds__(kWaves * 64, 2) cache_rows_kernel(CacheAttnParams p) {
  typedef CacheLayout<D, G> L;
  constexpr int NG = D / G, NW = D / 32, CT = D / 16;  // groups; words of codes a lane loads of 16 tokens; column tiles of 16 channels
  constexpr int ROWS = 4 * NR, WPG = G / 32;           // rows of the workgroup; code words of a group
  struct Work {
    uint8_t v[kWaves][64 * L::CODE];
    uint16_t w[kWaves][NG][ROWS][64];
  };
  struct Result {
    float o[kWaves][ROWS][D + 4];  // (4 more: the four rows that a wave writes at once fall into different banks)
    float m[kWaves][ROWS], l[kWaves][ROWS];
  };
  __shared__ __attribute__((aligned(16))) union { Work work; Result res; } sh;
  // With 8 or 16 rows every step fetches Q's operands and the sums below anew, which saves 32 registers: 60 spilled with 16 rows and groups of 32, eight
  // sequences of 8 heads, 4000 tokens, 33 rows each 85 us held, 51 fetched.  With 4 rows they stay (one token of 75,600, 40 heads: fetched 113 us, held 108).
  constexpr bool FETCH = NR > 1;
  __shared__ bf16x8 s_q[FETCH ? NW : 1][64];
  __shared__ f32x4 s_start[FETCH ? NG : 1][4];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, x = lane >> 4;
  const int split = blockIdx.x % p.splits, row0 = (int)(blockIdx.x / p.splits) * ROWS, hkv = blockIdx.y, b = blockIdx.z;
  const CacheSequence seq = cache_sequence(p.c, b, p.n);
  const int share = p.share, rows = share * seq.rows;
  if (row0 >= rows) return;
  const int last_row = min(row0 + ROWS, rows) - 1;
  auto limit_of = [&](int r) -> int { return cache_limit(seq, p.causal, share, r); };
  const int limit_all = limit_of(row0), limit_any = limit_of(last_row);
  const int tiles = (limit_any + 63) >> 6, per = (tiles + p.splits - 1) / p.splits;
  const int t_end = min(tiles, (split + 1) * per);
  const uint32_t page = 1u << p.c.log_page;
  const_i32* const table = (const_i32*)(p.c.pages + (int64_t)b * p.c.max_pages);

  // queries: slot col of the 16 holds row x' NR + i for col = 4 x' + i, i < NR
  bf16x8 qf[NW];
  {
    const int r = row0 + (col >> 2) * NR + (col & 3);
    const bool there = (col & 3) < NR && r <= last_row;
    const uint16_t* const qr = p.q + row_place(p, b, hkv, share, there ? r : row0).out + 8 * x;
#pragma unroll
    for (int j = 0; j < NW; ++j) {
      uint4 raw = {0u, 0u, 0u, 0u};
      if (there) raw = *reinterpret_cast<const uint4*>(qr + 32 * j);
      qf[j] = code_order(raw);
    }
  }
  const u32x4 ones_bits = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
  const bf16x8 ones = __builtin_bit_cast(bf16x8, ones_bits);
  f32x4 start[NG];  // -16 sum of a group's q
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = g * WPG; j < (g + 1) * WPG; ++j) sum = mfma16(qf[j], ones, sum);
    start[g] = sum * -16.f;
  }
  if constexpr (FETCH) {
    if (wave == 0) {
#pragma unroll
      for (int j = 0; j < NW; ++j) s_q[j][lane] = qf[j];
      if (col == 0)
#pragma unroll
        for (int g = 0; g < NG; ++g) s_start[g][x] = start[g];
    }
    __syncthreads();
  }
  int limit[NR];
#pragma unroll
  for (int i = 0; i < NR; ++i) limit[i] = limit_of(min(row0 + x * NR + i, last_row));

  float m[NR], l[NR], mid[NG][NR];  // running maximum (log2 units); this lane's shares of the sums of p and of p (m + 7.5 s)
  f32x4 o[CT], wsum[NG];            // sums of (p s)(16 + c) and of p s
#pragma unroll
  for (int i = 0; i < NR; ++i) { m[i] = -INFINITY; l[i] = 0.f; }
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    wsum[g] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NR; ++i) mid[g][i] = 0.f;
  }
#pragma unroll
  for (int c = 0; c < CT; ++c) o[c] = f32x4{0.f, 0.f, 0.f, 0.f};

  // a tile's tokens: 16 each in the page and slot that hold them (a page is a multiple of 16 tokens)
  uint32_t kc[4][NW], kp[4][NG], vc[4][NW], vp[4][NG];
  const uint8_t* run[4];
  uint32_t slot[4];
  int key0[4];  // position of the sub-tile's first token; beyond every limit if its page is not followed
  auto find = [&](int tile) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int pos = 64 * tile + 16 * t;
      const int pg = table[min(pos, seq.length - 1) >> p.c.log_page];  // (behind the last token: masked, but some page of the sequence)
      const bool ok = pg >= 0 && pg < p.c.n_pages;
      key0[t] = ok ? pos : 0x7fffff00;
      run[t] = p.c.pool + ((int64_t)(ok ? pg : 0) * p.c.H_kv + hkv) * p.c.head_bytes;
      slot[t] = (uint32_t)pos & (page - 1u);
    }
  };
  auto load_k = [&]() {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      load_words<NW>(run[t], L::k_codes(page) + slot[t] * L::CODE + (uint32_t)(col * L::CODE + x * (L::CODE / 4)), kc[t]);
      load_words<NG>(run[t], L::k_params(page) + slot[t] * L::PARAM + (uint32_t)(col * L::PARAM), kp[t]);
    }
  };
  auto load_v = [&]() {
#pragma unroll
    for (int t = 0; t < 4; ++t) load_words<NW>(run[t], L::v_codes(page) + slot[t] * L::CODE + (uint32_t)(lane * (L::CODE / 4)), vc[t]);
  };
  auto load_vp = [&]() {
#pragma unroll
    for (int t = 0; t < 4; ++t) load_words<NG>(run[t], L::v_params(page) + slot[t] * L::PARAM + (uint32_t)(col * L::PARAM), vp[t]);
  };

  uint8_t* const vl = sh.work.v[wave];
  // the transposing read: lane `col` of block x points at the token that stands in nibble `col` of every result
  const int nib = col & 7, ord = nib < 4 ? 2 * nib : 2 * nib - 7;  // nibble -> place in the contraction (0 4 1 5 2 6 3 7)
  const int v_token = 16 * (ord & 3) + 4 * x + 2 * (col >> 3) + (ord >> 2);
  const uint8_t* const v_read = vl + v_token * L::CODE;
  const int w_row = (col >> 2) * NR + min(col & 3, NR - 1);  // the row of slot col (or, unused slots, any)

  const CodeBits bits16;
  int tile = split * per + wave;
  if (tile < t_end) {
    find(tile);
    load_v();
    load_k();
    load_vp();
  }
  for (; tile < t_end; tile += kWaves) {
    wave_fence();
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      uint8_t* const at = vl + 16 * t * L::CODE + lane * (L::CODE / 4);
      if constexpr (NW == 4) *reinterpret_cast<uint4*>(at) = make_uint4(vc[t][0], vc[t][1], vc[t][2], vc[t][3]);
      else *reinterpret_cast<uint2*>(at) = make_uint2(vc[t][0], vc[t][1]);
    }
    int key[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) key[t] = key0[t] + col;
    const bool whole = max(max(key0[0], key0[1]), max(key0[2], key0[3])) + 16 <= limit_all;  // every row sees every token
    // Every operand of the next tile is requested where this tile's is used up, most of a step ahead.  (The last step requests
    // its own tile again: requests under a condition cost the compiler copies of all these registers.)
    find(tile + kWaves < t_end ? tile + kWaves : tile);
    load_v();
    float s[4][NR];
    if constexpr (FETCH) {
#pragma unroll
      for (int j = 0; j < NW; ++j) qf[j] = s_q[j][lane];
#pragma unroll
      for (int g = 0; g < NG; ++g) start[g] = s_start[g][x];
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        f32x4 acc = start[g];
#pragma unroll
        for (int j = g * WPG; j < (g + 1) * WPG; ++j) acc = mfma16(qf[j], codes_bf16(kc[t][j], bits16), acc);
        const float sc = bf16_low(kp[t][g]), mn = bf16_high(kp[t][g]) * -0.0625f;  // (times start: the minimum times the sum of q)
#pragma unroll
        for (int i = 0; i < NR; ++i) s[t][i] = fmaf(sc, acc[i], g == 0 ? mn * start[g][i] : fmaf(mn, start[g][i], s[t][i]));
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    load_k();
    __builtin_amdgcn_sched_barrier(0);
    if (!whole)
#pragma unroll
      for (int i = 0; i < NR; ++i)
#pragma unroll
        for (int t = 0; t < 4; ++t) s[t][i] = key[t] < limit[i] ? s[t][i] : -INFINITY;
    // The maximum follows the logits only when one is 64 times its weight's due ahead: o and l are as exact with weights up to 64 as with weights up to
    // 1, and the maximum over the lanes is rarely needed.
    float mx[NR];
    bool grows = false;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      mx[i] = fmaxf(fmaxf(s[0][i], s[1][i]), fmaxf(s[2][i], s[3][i]));
      grows |= fmaf(mx[i], p.scale, -m[i]) > 6.f;
    }
    if (__builtin_amdgcn_ballot_w64(grows)) {
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        mx[i] = row16_max(mx[i]) * p.scale;
        const float m_new = fmaxf(m[i], mx[i]);
        const float corr = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[i] - m_new);
        m[i] = m_new;
        l[i] *= corr;
#pragma unroll
        for (int g = 0; g < NG; ++g) { mid[g][i] *= corr; wsum[g][i] *= corr; }
#pragma unroll
        for (int c = 0; c < CT; ++c) o[c][i] *= corr;
      }
    }
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const float neg = m[i] == -INFINITY ? 0.f : -m[i];  // nothing seen yet: every weight is exp2(-inf) = 0
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        s[t][i] = __builtin_amdgcn_exp2f(fmaf(s[t][i], p.scale, neg));
        l[i] += s[t][i];
      }
    }
    auto weights = [&](auto masked) {
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        float sc[4], mm[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          sc[t] = bf16_low(vp[t][g]);
          mm[t] = fmaf(7.5f, sc[t], bf16_high(vp[t][g]));
        }
#pragma unroll
        for (int i = 0; i < NR; ++i) {
          bf16x8 w;  // (the upper half unused)
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            float ps = s[t][i] * sc[t], pm = s[t][i] * mm[t];
            if constexpr (decltype(masked)::value) {  // a token that is not seen may have any parameters, NaN among them
              ps = key[t] < limit[i] ? ps : 0.f;
              pm = key[t] < limit[i] ? pm : 0.f;
            }
            w[t] = (__bf16)ps;
            mid[g][i] += pm;
          }
          const u32x4 bits = __builtin_bit_cast(u32x4, w);
          *reinterpret_cast<uint2*>(&sh.work.w[wave][g][x * NR + i][4 * col]) = make_uint2(bits[0], bits[1]);
        }
      }
    };
    if (whole) weights(std::false_type{});
    else weights(std::true_type{});
    load_vp();
    __builtin_amdgcn_sched_barrier(0);
    wave_fence();
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const bf16x8 w0 = *reinterpret_cast<const bf16x8*>(&sh.work.w[wave][g][w_row][16 * x]);
      const bf16x8 w1 = *reinterpret_cast<const bf16x8*>(&sh.work.w[wave][g][w_row][16 * x + 8]);
      wsum[g] = mfma16(w0, ones, wsum[g]);
      wsum[g] = mfma16(w1, ones, wsum[g]);
#pragma unroll
      for (int c = g * (G / 16); c < (g + 1) * (G / 16); ++c) {
        const i32x2 v = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_i32x2*)(v_read + 8 * c));
        o[c] = mfma16(w0, codes_bf16((uint32_t)v[0], bits16), o[c]);
        o[c] = mfma16(w1, codes_bf16((uint32_t)v[1], bits16), o[c]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // the four waves' results are put together
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    l[i] = row16_sum(l[i]);
#pragma unroll
    for (int g = 0; g < NG; ++g) mid[g][i] = row16_sum(mid[g][i]) - 23.5f * wsum[g][i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const int r = x * NR + i;
#pragma unroll
    for (int c = 0; c < CT; ++c) sh.res.o[wave][r][16 * c + col] = o[c][i] + mid[c / (G / 16)][i];
    if (col == 0) { sh.res.m[wave][r] = m[i]; sh.res.l[wave][r] = l[i]; }
  }
  __syncthreads();
  constexpr int TPR = D / 4;  // threads of a row, four channels each
  for (int r = tid / TPR; r < ROWS; r += kWaves * 64 / TPR) {
    const int ch = tid % TPR * 4;
    if (row0 + r > last_row) break;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sh.res.m[w][r]);
    const float ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    f32x4 val = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(sh.res.m[w][r] - ref);
      const f32x4 part = *reinterpret_cast<const f32x4*>(&sh.res.o[w][r][ch]);
      sum = fmaf(f, sh.res.l[w][r], sum);
#pragma unroll
      for (int i = 0; i < 4; ++i) val[i] = fmaf(f, part[i], val[i]);
    }
    const RowPlace at = row_place(p, b, hkv, share, row0 + r);
    if (p.splits == 1) {  // a row that sees nothing is zero, its normaliser empty
      bf16x4 y;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = (__bf16)(sum == 0.f ? 0.f : val[i] / sum);
      *reinterpret_cast<bf16x4*>(p.o + at.out + ch) = y;
      if (p.lse && ch == 0) p.lse[at.lse] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
    } else {
      const int64_t part = at.lse * p.splits + split;
      *reinterpret_cast<f32x4*>(p.part_o + part * D + ch) = val;
      if (ch == 0) { p.part_ml[2 * part] = top; p.part_ml[2 * part + 1] = sum; }
    }
  }
}

// out and lse of a row from the results of its splits: a workgroup a row, each wave every fourth split.  A chain of loads of some 4 us, whatever the size.
template <int D>
__global__ void __launch_bounds__(256) cache_merge_kernel(CacheAttnParams p) {
  __shared__ float part[4][D];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const CacheSequence seq = cache_sequence(p.c, b, p.n);
  if (i >= seq.rows) return;
  const int64_t row = ((int64_t)b * p.H + h) * p.n + i, first = row * p.splits;
  float m = -INFINITY, l = 0.f;
  if (lane < p.splits) { m = p.part_ml[2 * (first + lane)]; l = p.part_ml[2 * (first + lane) + 1]; }
  float top = m;
  for (int d = 32; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float f = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.f : top));
  float sum = f * l;
  for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d);
  float o[D / 64] = {};
  const float* const src = p.part_o + first * D + lane;
#pragma unroll 8
  for (int s = wave; s < p.splits; s += 4) {
    const float fs = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(f), s));
#pragma unroll
    for (int t = 0; t < D / 64; ++t) o[t] = fmaf(fs, src[s * D + 64 * t], o[t]);
  }
#pragma unroll
  for (int t = 0; t < D / 64; ++t) part[wave][64 * t + lane] = o[t];
  __syncthreads();
  const int ch = threadIdx.x;
  if (ch < D) {
    const float val = (part[0][ch] + part[1][ch]) + (part[2][ch] + part[3][ch]);
    const __bf16 y = (__bf16)(sum == 0.f ? 0.f : val / sum);
    p.o[b * p.stride_b + h * p.stride_h + i * p.stride_n + ch] = __builtin_bit_cast(uint16_t, y);
  }
  if (p.lse && threadIdx.x == 0) p.lse[row] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <int D, int G>
hipError_t launch_rows(const CacheAttnParams& p, hipStream_t stream) {
  const int rows = p.share * p.n;
  const dim3 grid((rows + p.wg_rows - 1) / p.wg_rows * p.splits, p.c.H_kv, p.c.B);
  if (p.wg_rows == 4) cache_rows_kernel<D, G, 1><<<grid, kWaves * 64, 0, stream>>>(p);
  else if (p.wg_rows == 8) cache_rows_kernel<D, G, 2><<<grid, kWaves * 64, 0, stream>>>(p);
  else cache_rows_kernel<D, G, 4><<<grid, kWaves * 64, 0, stream>>>(p);
  return hipGetLastError();
}

hipError_t launch_rows(const CacheAttnParams& p, hipStream_t stream) {
  if (p.c.d == 64) return p.c.group == 32 ? launch_rows<64, 32>(p, stream) : launch_rows<64, 64>(p, stream);
  return p.c.group == 32 ? launch_rows<128, 32>(p, stream)
       : p.c.group == 64 ? launch_rows<128, 64>(p, stream) : launch_rows<128, 128>(p, stream);
}

}  // namespace

hipError_t pasa_launch_cache_attn(const CacheAttnParams& p, hipStream_t stream) {
  if (p.wg_rows == 256) return pasa_launch_cache_tiles(p, stream);
  const hipError_t rc = launch_rows(p, stream);
  if (rc != hipSuccess || p.splits == 1) return rc;
  const dim3 grid(p.n, p.H, p.c.B);
  if (p.c.d == 64) cache_merge_kernel<64><<<grid, 256, 0, stream>>>(p);
  else cache_merge_kernel<128><<<grid, 256, 0, stream>>>(p);
  return hipGetLastError();
}
