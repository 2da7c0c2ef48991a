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

struct CacheMerge {  // an item that several workgroups of cache_tile_kernel share (pasa_cache_tile.hip)
  int32_t hkv, item, first_slot, parts;  // parts = 0: none
};
struct CacheAttnParams {
  CacheParams c;
  const uint16_t* q;
  uint16_t* o;
  float* lse;  // nullable
  int64_t stride_b, stride_h, stride_n;
  int32_t H, share, n, causal;  // share = H / H_kv
  float scale;  // of the logits, times log2(e)
  int32_t wg_rows;  // (row, head of a key/value head's share) pairs of a workgroup: 4, 8, 16 (pasa_cache_attn.hip) or 256 (pasa_cache_tile.hip)
  // 4, 8, 16: a sequence's tokens are divided among `splits` workgroups, at most kCacheMaxSplits, and with splits > 1
  int32_t splits;
  float* part_o;   // fp32 [B][H][n][splits][d]: sums against the maximum of their split
  float* part_ml;  // fp32 [B][H][n][splits][2]: that maximum (log2 units) and the sum of the weights
  // 256: all the work is divided among `pieces` workgroups; part_o, part_ml are [2 pieces][wg_rows][d], [..][2]
  int32_t pieces, row_tiles;  // row_tiles = runs of wg_rows rows that a sequence can have
  CacheMerge* merge;          // [pieces]
  uint32_t* key_range;        // [B][H_kv][key_parts]: largest magnitudes of K's groups (pasa_cache_tile.hip), each of a run of a sequence's tokens
  int32_t key_parts;          // at most kCacheMaxKeyParts
};
constexpr int kCacheMaxKeyParts = 64;  // a wave of cache_tile_kernel holds one per lane
constexpr int kCacheMinPiece = 2;  // tiles of a piece, at least
constexpr int kCacheMaxSplits = 64;  // a wave of the merging kernel holds one per lane
hipError_t pasa_launch_cache_tiles(const CacheAttnParams& p, hipStream_t stream);  // wg_rows 256
hipError_t pasa_launch_cache_attn(const CacheAttnParams& p, hipStream_t stream);
