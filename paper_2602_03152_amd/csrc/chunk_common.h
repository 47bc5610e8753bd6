// Shared by the kernels around chunks of new tokens (cache.hip, chunk.hip, chunk_wide.hip): the cache and the chunk as the kernels see
// them, and 8-bit values.
#pragma once

#include "attend_common.h"

namespace fasa {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// for lambdas over register arrays: one that is called twice and not inlined has them in memory
#define FASA_INLINE __attribute__((always_inline))

enum CacheFmt { kPlain = FASA_CACHE_PLAIN, kInt8 = FASA_CACHE_INT8, kE4m3 = FASA_CACHE_E4M3 };

// A cached row's storage: values of ET, or bytes.
template <typename ET, CacheFmt F> struct RowType { using type = uint8_t; };
template <typename ET> struct RowType<ET, kPlain> { using type = ET; };

struct CacheView {
  void *K, *V;
  float *ks, *vs;               // null: rows of dtype
  long long sb, sh, sn;         // elements between blocks (paged) or sequences, heads, tokens
  long long ssb, ssh;           // of the scales
  PageMap pm;
};
// Block (without paging: sequence) and token in it of token n of sequence b.  In two steps, where the table is read ahead: the entry as it is, and
// clamped into the pool.
__device__ __forceinline__ int cache_block(const PageMap& pm, int b, int n) {
  return pm.table ? pm.table[(size_t)b * pm.max_blocks + (n >> pm.shift)] : b;
}
__device__ __forceinline__ int cache_clamp(const PageMap& pm, int blk) { return pm.table ? min(max(blk, 0), pm.n_pool - 1) : blk; }
__device__ __forceinline__ int cache_offset(const PageMap& pm, int n) { return pm.table ? n & ((1 << pm.shift) - 1) : n; }
__device__ __forceinline__ void cache_place(const PageMap& pm, int b, int n, int& blk, int& off) {
  blk = cache_clamp(pm, cache_block(pm, b, n));
  off = cache_offset(pm, n);
}

struct ChunkView {
  const int32_t *n_new_seq, *n_ctx_seq, *row_start;
  int n_new, n_rows, n_ctx;
};
struct SeqChunk { int n_ctx, n_new, row; };      // a sequence's tokens, new tokens, first row
__device__ __forceinline__ SeqChunk seq_chunk(const ChunkView& c, int b) {
  SeqChunk s;
  s.n_ctx = c.n_ctx_seq ? min(max(c.n_ctx_seq[b], 0), c.n_ctx) : c.n_ctx;
  s.row = c.row_start ? min(max(c.row_start[b], 0), c.n_rows) : b * c.n_new;
  int n = min(c.n_new_seq ? c.n_new_seq[b] : c.n_new, min(c.n_new, s.n_ctx));
  if (c.row_start) n = min(n, c.n_rows - s.row);
  s.n_new = max(n, 0);
  return s;
}

// Work on a chunk goes by tiles of a sequence's items (rows, rows times heads).  Without row_start the rows of a sequence that
// has fewer than n_new are padding that the caller has room for: every sequence gets the same number of tiles, and those behind its end have
// nothing to do.  With row_start there may be many short sequences beside a long one, and batch * (tiles of the longest) of
// workgroups would find nothing to do; there are n_rows in all, so n_rows * per_row / TILE + batch tiles are enough, and a
// workgroup finds its own by counting them, 64 sequences at a time.  False: no tile left for it.
template <int TILE>
__device__ __forceinline__ bool find_chunk_tile(const ChunkView& c, int batch, int per_row, int tiles_each, unsigned id, int& b, int& tile) {
  if (c.row_start == nullptr) {
    b = (int)(id / (unsigned)tiles_each);
    tile = (int)(id - (unsigned)b * tiles_each);
    return b < batch;
  }
  uint32_t left = id;
  for (int b0 = 0; b0 < batch; b0 += kWave) {
    const int mine = b0 + lane_id();
    const uint32_t v = mine < batch ? (uint32_t)(((long long)seq_chunk(c, mine).n_new * per_row + TILE - 1) / TILE) : 0u;
    const uint32_t incl = wave_prefix_sum(v);
    const uint32_t total = (uint32_t)__builtin_amdgcn_readlane((int)incl, kWave - 1);
    if (left < total) {
      const int at = __builtin_ctzll(__ballot(incl > left));
      b = b0 + at;
      tile = (int)(left - (uint32_t)__builtin_amdgcn_readlane((int)(incl - v), at));
      return true;
    }
    left -= total;
  }
  return false;
}
// A workgroup's part of the work: tokens [split * share, ..) of a query tile of a sequence.  first: the place of the tile's split 0 among the partial results.
struct ChunkUnit {
  SeqChunk seq;
  int b, tile, split, splits, first;
  int share;                    // 0: the tile's tokens in equal parts
  int slot;                     // of the tile among a row's (sequence's and KV head's) that are split: below the workgroups of a KV head
};
// Unit y of the grid.  Uniform: the first `whole` tiles are a unit each, every other one is in `splits` parts.  By length (units != 0; up to 64 sequences): a batch of mixed lengths would wait for its longest
// sequence, so all parts are of about as many tokens, and a sequence has as many of them as it takes: the smallest share (a multiple of 64 tokens, of
// least_share or more) with which all the tiles' parts are no more than the units.  Every wave finds it by itself, a lane a sequence.
template <int TILE>
__device__ __forceinline__ bool find_chunk_unit(const ChunkView& c, int batch, int G, int tiles_each, int whole, int splits, int units, int least_share, unsigned y, ChunkUnit& u) {
  if (units == 0) {
    const bool one = y < (unsigned)whole;
    const unsigned part = one ? 0u : y - (unsigned)whole, id = one ? y : (unsigned)whole + part / (unsigned)splits;
    u.splits = one ? 1 : splits;
    u.split = one ? 0 : (int)(part % (unsigned)splits);
    u.first = (int)part - u.split;
    u.share = 0;
    u.slot = (int)(part / (unsigned)splits);
    if (!find_chunk_tile<TILE>(c, batch, G, tiles_each, id, u.b, u.tile)) return false;
    u.seq = seq_chunk(c, u.b);
    return u.tile < (int)(((long long)u.seq.n_new * G + TILE - 1) / TILE);
  }
  SeqChunk s = {0, 0, 0};
  if (lane_id() < batch) s = seq_chunk(c, lane_id());
  const int nt = (int)(((long long)s.n_new * G + TILE - 1) / TILE);
  const int s64 = nt ? (int)(((long long)s.n_ctx + 63) / 64) : 0;
  const auto parts = [&](int q) {                                      // of a tile, with a share of q times 64 tokens
    int n = (int)ceilf((float)s64 * __builtin_amdgcn_rcpf((float)q));
    if ((long long)n * q < s64) ++n;
    return n;
  };
  int hi = max((int)wave_max((float)s64) + 1, 1);                      // (holds all; + 1 for what the conversion may round off)
  int lo = min(max((int)(wave_sum((float)nt * (float)s64) / (float)units), least_share / 64), hi);
  for (int i = 0; i < 8 && lo < hi; ++i) {
    const int mid = (lo + hi) / 2;
    if (wave_sum((float)nt * (float)parts(mid)) <= (float)units) hi = mid;
    else lo = mid + 1;
  }
  const int n = parts(hi);
  const uint32_t v = (uint32_t)(nt * n), incl = wave_prefix_sum(v);
  const unsigned long long reached = __ballot(incl > y);
  // (more parts than units: only if the sequences' rows overlap, so that there are more new tokens than rows)
  if (reached == 0ull || __builtin_amdgcn_readlane((int)incl, kWave - 1) > units) return false;
  u.b = __builtin_ctzll(reached);
  const int local = (int)y - __builtin_amdgcn_readlane((int)(incl - v), u.b);
  u.splits = __builtin_amdgcn_readlane(n, u.b);
  u.tile = local / u.splits;
  u.split = local - u.tile * u.splits;
  u.first = (int)y - u.split;
  u.share = 64 * hi;
  u.slot = u.tile;
  u.seq = SeqChunk{__builtin_amdgcn_readlane(s.n_ctx, u.b), __builtin_amdgcn_readlane(s.n_new, u.b), __builtin_amdgcn_readlane(s.row, u.b)};
  return true;
}
// tiles that the grid needs (an upper bound)
inline long long chunk_tiles(bool by_row_start, int batch, int n_new, int n_rows, int per_row, int tile) {
  return by_row_start ? (long long)n_rows * per_row / tile + batch : (long long)batch * (((long long)n_new * per_row + tile - 1) / tile);
}

// ---- 8-bit values ---------------------------------------------------------------------------------
// Four bytes as two words of bf16 pairs.  Exact: an int8 has 8 significant bits, an e4m3 number 4.
template <CacheFmt F> __device__ __forceinline__ uint2 bytes_to_bf16(uint32_t w) {
  if constexpr (F == kE4m3) {
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true)));
  } else {
    const float f0 = (float)(int8_t)w, f1 = (float)(int8_t)(w >> 8), f2 = (float)(int8_t)(w >> 16), f3 = (float)((int32_t)w >> 24);
    return make_uint2(__builtin_amdgcn_perm(__float_as_uint(f1), __float_as_uint(f0), 0x07060302u),
                      __builtin_amdgcn_perm(__float_as_uint(f3), __float_as_uint(f2), 0x07060302u));
  }
}
template <CacheFmt F> __device__ __forceinline__ f32x4_t bytes_to_f32(uint32_t w) {
  if constexpr (F == kE4m3) {
    const uint2 p = bytes_to_bf16<F>(w);
    return f32x4_t{bf16_lo(p.x), bf16_hi(p.x), bf16_lo(p.y), bf16_hi(p.y)};
  } else {
    return f32x4_t{(float)(int8_t)w, (float)(int8_t)(w >> 8), (float)(int8_t)(w >> 16), (float)((int32_t)w >> 24)};
  }
}
// two float32 numbers as a word of bf16, to the nearest, ties to even
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const bf16x2_t r = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, r);
}

// ---- launchers (shapes are validated) ----------------------------------------------------------------
hipError_t launch_cache_write(const fasa_shape& s, const CacheView& cv, CacheFmt fmt, const ChunkView& ch, long long kv_stride, const void* k_new,
                              const void* v_new, hipStream_t st);
hipError_t launch_cache_read(const fasa_shape& s, const CacheView& cv, CacheFmt fmt, const int32_t* T, const int32_t* n_ctx_seq,
                             int n_begin, int n_end, void* K_out, void* V_out, hipStream_t st);

// The forms of chunk attention, and what each divides a call into: tiles of `rows` query rows (new token, head of the group) of a sequence and KV head, whose tokens go to
// parts of `least` or more, `splits` a tile at most, for rounds of `resident` workgroups, `resident_by_length` where parts go by the sequences' lengths.  No more than `parts`
// workgroups of a call have partial results.  What a workgroup's begin and end cost beside its tokens, and what a part costs to be joined, in tokens of a tile: begin, join.
struct ChunkForm {
  int rows, resident, resident_by_length, least, splits, parts, begin, join;
};
constexpr ChunkForm kTokenForm{16, kAssumedCUs, 2 * kAssumedCUs, 64, 256, 4 * kAssumedCUs, 800, 0};            // chunk.hip
constexpr ChunkForm kShortForm{128, 2 * kAssumedCUs, 2 * kAssumedCUs, 256, 64, 2 * kAssumedCUs, 500, 1};       // chunk_wide.hip
constexpr ChunkForm kDeepForm{256, kAssumedCUs, kAssumedCUs, 256, 64, 2 * kAssumedCUs, 320, 2};

struct ChunkPlan {
  ChunkForm form;
  bool apart;         // rows are looked up one by one
  bool by_length;     // parts by the sequences' lengths
  int tile_rows;      // query rows that a tile of this call has: form.rows, or all that there are
  int per_seq;        // query tiles of the longest sequence
  int whole;          // tiles before those that are split (0: by_length)
  int splits;         // parts of a tile behind, where it is not by_length
  int units;          // workgroups of a KV head, at most
  int parts;          // of them with partial results: all behind `whole`, where there are any
  size_t part_acc_bytes, part_ml_bytes;
};
// apart: chunk_wide.hip has to look rows up one by one - pages of fewer tokens than a wave's load has rows, or strides beyond what it multiplies in 32 bits
inline bool chunk_rows_apart(const CacheView& cv, CacheFmt fmt) {
  return (cv.pm.table != nullptr && ((1 << cv.pm.shift) < (fmt == kPlain ? 4 : 8) || cv.sb >= (1ll << 31))) || cv.sn >= (1ll << 27);
}
ChunkPlan plan_chunk(const fasa_shape& s, bool apart, const ChunkView& ch);
// rows of partial results that no call with this one's batch and heads and at most its new tokens, rows and context goes beyond
size_t most_chunk_parts(const fasa_shape& s, const ChunkView& ch);
constexpr size_t kChunkAccBytes = kHeadDim * 4, kChunkMlBytes = 8;                    // of a row of partial results
struct ChunkArgs {
  CacheView cv;
  ChunkView ch;
  CacheFmt fmt;
  const void* q;
  void* O;
  long long q_stride, o_stride;
  float *part_acc, *part_ml;
  uint32_t* tickets;            // [row][kChunkTickets], zero
};
constexpr int kChunkTickets = kHistBins;      // the words of a row's histogram, which are zero between calls
hipError_t launch_chunk(const fasa_shape& s, const ChunkPlan& p, const ChunkArgs& a, hipStream_t st);
hipError_t launch_chunk_wide(const fasa_shape& s, const ChunkPlan& p, const ChunkArgs& a, hipStream_t st);

}  // namespace fasa
