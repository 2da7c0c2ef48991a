// Host-side launch interface of the 4-bit key/value cache's kernels (format: pasa_cache.hpp).  As in pasa_kernels.hpp the launchers
// validate nothing, return hipGetLastError() after their last launch and never synchronise.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

struct CacheParams {
  uint8_t* pool;
  const int32_t* pages;  // [B][max_pages]: page of the pool that holds tokens i * page .. of a sequence; numbers outside [0, n_pages) are not followed
  const int32_t* len;    // [B]: tokens of a sequence, the new ones among them
  const int32_t* n_new;  // [B] or null: new rows of a sequence; row i is token len - n_new + i (null: n of them)
  int32_t B, H_kv, d, group, log_page, n_pages, max_pages;
  int64_t head_bytes;    // bytes of one head's run in a page
};

struct CacheRowsParams {  // write: K and V rows -> cache; read: cache -> rows
  CacheParams c;
  uint16_t* k;  // write: not written
  uint16_t* v;
  int64_t stride_b, stride_h, stride_n;
  int32_t n;
};
hipError_t pasa_launch_cache_write(const CacheRowsParams& p, hipStream_t stream);
hipError_t pasa_launch_cache_read(const CacheRowsParams& p, hipStream_t stream);

struct CacheAttnParams {
  CacheParams c;
  const uint16_t* q;
  uint16_t* o;
  float* lse;  // nullable
  int64_t stride_b, stride_h, stride_n;
  int32_t H, n, causal;
  float scale;  // of the logits, times log2(e)
  int32_t wg_rows;  // (row, head of a key/value head's share) pairs of a workgroup: 4, 8, 16 (pasa_cache_attn.hip), 128 or 256 (pasa_cache_tile.hip)
  int32_t splits;   // workgroups among which a sequence's tokens are divided, at most kCacheMaxSplits
  float* part_o;    // splits > 1: fp32 [B][H][n][splits][d], sums against the maximum of their split
  float* part_ml;   //             fp32 [B][H][n][splits][2], that maximum (log2 units) and the sum of the weights
};
constexpr int kCacheMaxSplits = 64;  // a wave of the merging kernel holds one per lane
hipError_t pasa_launch_cache_tiles(const CacheAttnParams& p, hipStream_t stream);  // the attention kernel alone
hipError_t pasa_launch_cache_attn(const CacheAttnParams& p, hipStream_t stream);
