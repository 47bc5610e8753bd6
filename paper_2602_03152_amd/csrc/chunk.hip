// Attention of a few query rows of a KV head over its cache: single tokens, a few drafted ones, and float32 chunks of any length.
// Query rows (new token i, head g of the group) of a sequence and KV head go by tiles of 16, the columns of the matrix cores' 16-row
// tile engine (mfma_tile.h); a tile's tokens are shared out to `splits` workgroups of eight waves, a wave takes 16 at a time, and the
// last workgroup of a tile by ticket merges the partial results.  Bound by reading the rows, once per tile: 2 d bytes e a token.
#include "chunk_common.h"
#include "mfma_tile.h"

namespace fasa {

constexpr int kChunkThreads = 512, kChunkWaves = kChunkThreads / kWave;
constexpr int kChunkRows = 16;                           // query rows of a tile
constexpr int kChunkStep = 16 * kChunkWaves;             // tokens of a round of the waves

// One lane's share of 16 rows as stored; K: chunks hi, hi + 4, .. of 16 bytes of row lo, V: dims 8lo .. 8lo + 7 of rows 4hi .. 4hi + 3
template <typename ET, CacheFmt F> struct RawKV {
  uint4 k[2];
  uint2 v[4];
  __device__ __forceinline__ void load_k(const uint8_t* p) { k[0] = load_u128<>(p); k[1] = load_u128<>(p + 64); }
  __device__ __forceinline__ void load_v(int e, const uint8_t* p) { v[e] = *reinterpret_cast<const uint2*>(p); }
  __device__ __forceinline__ void k_to(TileKV<ET>& t) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t w[4] = {k[i].x, k[i].y, k[i].z, k[i].w};
      if constexpr (sizeof(ET) == 2) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint2 a = bytes_to_bf16<F>(w[2 * j]), b = bytes_to_bf16<F>(w[2 * j + 1]);
          t.kc[2 * i + j] = make_uint4(a.x, a.y, b.x, b.y);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) t.kc[4 * i + j] = bytes_to_f32<F>(w[j]);
      }
    }
  }
  __device__ __forceinline__ void v_to(TileKV<ET>& t) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(ET) == 2) {
        const uint2 a = bytes_to_bf16<F>(v[e].x), b = bytes_to_bf16<F>(v[e].y);
        t.vr[e] = make_uint4(a.x, a.y, b.x, b.y);
      } else {
        t.vr[e][0] = bytes_to_f32<F>(v[e].x);
        t.vr[e][1] = bytes_to_f32<F>(v[e].y);
      }
    }
  }
};
// head dim at which chunk i of a lane's K begins, of the chunks that TileKV<ET> holds
template <typename ET, CacheFmt F> __device__ __forceinline__ int chunk_dim(int i, int hi) {
  constexpr int C = kChunk<ET>;
  if constexpr (F == kPlain) return C * (hi + 4 * i);
  else return 16 * (hi + 4 * (i / (16 / C))) + C * (i % (16 / C));
}

// SMALL: pages of fewer than 16 tokens, whose rows are looked up one by one; else the 16 rows of a tile lie in one block.
template <typename ET, CacheFmt F, bool SMALL>
__global__ __launch_bounds__(kChunkThreads, 2) void chunk_kernel(const ET* __restrict__ q, const typename RowType<ET, F>::type* __restrict__ K,
                                                                 const typename RowType<ET, F>::type* __restrict__ V, ET* __restrict__ O,
                                                                 float* __restrict__ part_acc, float* __restrict__ part_ml,
                                                                 uint32_t* __restrict__ tickets, CacheView cv, ChunkView ch, int batch, int Hkv,
                                                                 int G, int tiles_each, int splits, int cap, long long q_stride,
                                                                 long long o_stride, float scale_log2e) {
  constexpr int D = kHeadDim;
  constexpr bool F32 = sizeof(ET) == 4;
  using RT = typename RowType<ET, F>::type;
  // waves' totals: [wave][cap][D], then m, l [wave][cap]; the merge: weights [split][cap], then the partitions' sums
  extern __shared__ __align__(16) float lds[];
  __shared__ __align__(16) float scs[kChunkWaves][16];
  __shared__ float red[kChunkRows];
  __shared__ uint32_t ticket;

  // workgroups: heads fastest (the blocks of a paged cache often hold all heads' rows side by side), then splits
  unsigned id = blockIdx.x;
  const int h = (int)(id % (unsigned)Hkv);
  id /= (unsigned)Hkv;
  const int split = (int)(id % (unsigned)splits);
  id /= (unsigned)splits;
  int b, qt;
  if (!find_chunk_tile<kChunkRows>(ch, batch, G, tiles_each, id, b, qt)) return;
  const SeqChunk sc = seq_chunk(ch, b);
  const int rows = min(cap, sc.n_new * G - qt * kChunkRows);        // of this tile
  if (rows <= 0) return;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int lo = lane & 15, hi = lane >> 4;
  const int pos0 = sc.n_ctx - sc.n_new;
  const auto token_of = [&](int r) FASA_INLINE { return (qt * kChunkRows + r) / G; };
  // tokens [0, seen) are seen by the last row of the tile
  const int seen = pos0 + token_of(rows - 1) + 1;
  const int share = ((seen + splits - 1) / splits + 15) & ~15;
  const int s0 = min(split * share, seen), s1 = min(seen, s0 + share);

  MfmaTile<kChunkRows, ET> tile;
  const int my = min(lo, rows - 1), my_tok = token_of(my);
  const int my_end = min(s1, pos0 + my_tok + 1);                     // of query row lo
  {
    const ET* p = q + (long long)(sc.row + my_tok) * q_stride + (long long)(h * G + (qt * kChunkRows + my) - my_tok * G) * D;
#pragma unroll
    for (int i = 0; i < (F32 ? 8 : 4); ++i)
      tile.qb[i] = __builtin_bit_cast(typename MfmaTile<kChunkRows, ET>::QT, *reinterpret_cast<const uint4*>(p + chunk_dim<ET, F>(i, hi)));
  }
  tile.reset();

  const RT* Kh = K + h * cv.sh + (F == kPlain ? kChunk<ET> : 16) * hi;
  const RT* Vh = V + h * cv.sh + 8 * lo;
  const float* ksh = F == kPlain ? nullptr : cv.ks + h * cv.ssh;
  const float* vsh = F == kPlain ? nullptr : cv.vs + h * cv.ssh;
  typename std::conditional<F == kPlain, TileKV<ET>, RawKV<ET, F>>::type raw;
  f32x4_t ks = {1.f, 1.f, 1.f, 1.f}, vs = ks;
  struct Place { long long k, v[4], vs[4]; } pl;       // rows and scales of the next tile
  // the tile's rows from token j0 on; tokens behind the split's last are the last again
  auto find_rows = [&](int j0) FASA_INLINE {
    if constexpr (SMALL) {
      int blk, off;
      cache_place(cv.pm, b, min(j0 + lo, s1 - 1), blk, off);
      pl.k = blk * cv.sb + off * cv.sn;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        cache_place(cv.pm, b, min(j0 + 4 * hi + e, s1 - 1), blk, off);
        pl.v[e] = blk * cv.sb + off * cv.sn;
        pl.vs[e] = blk * cv.ssb + off;
      }
    } else {
      int blk, off;
      cache_place(cv.pm, b, min(j0, (s1 - 1) & ~15), blk, off);      // (j0 is a multiple of 16, the same for the wave)
      const int last = s1 - 1 - min(j0, (s1 - 1) & ~15);
      const long long base = blk * cv.sb + off * cv.sn, sbase = blk * cv.ssb + off;
      pl.k = base + (long long)min(lo, last) * cv.sn;
#pragma unroll
      for (int e = 0; e < 4; ++e) pl.v[e] = base + (long long)min(4 * hi + e, last) * cv.sn;
      pl.vs[0] = sbase + min(4 * hi, last & ~3);                     // four at once: rows of scales are whole fours
    }
  };
  auto load_k = [&]() FASA_INLINE {
    raw.load_k(Kh + pl.k);
    if constexpr (F != kPlain) {
      if constexpr (SMALL) {
#pragma unroll
        for (int e = 0; e < 4; ++e) ks[e] = ksh[pl.vs[e]];
      } else {
        ks = *reinterpret_cast<const f32x4_t*>(ksh + pl.vs[0]);
      }
    }
  };
  auto load_v = [&]() FASA_INLINE {
#pragma unroll
    for (int e = 0; e < 4; ++e) raw.load_v(e, Vh + pl.v[e]);
    if constexpr (F != kPlain) {
      if constexpr (SMALL) {
#pragma unroll
        for (int e = 0; e < 4; ++e) vs[e] = vsh[pl.vs[e]];
      } else {
        vs = *reinterpret_cast<const f32x4_t*>(vsh + pl.vs[0]);
      }
    }
  };
  int j0 = s0 + 16 * wave;
  if (j0 < s1) {
    find_rows(j0);
    load_k();
    load_v();
    TileKV<ET> kv;
    for (; j0 < s1; j0 += kChunkStep) {
      float sv[4];
      f32x4_t k_by = ks, v_by = vs;
      if constexpr (F == kPlain) kv = raw; else { raw.k_to(kv); raw.v_to(kv); }
      find_rows(min(j0 + kChunkStep, s1 - 1) & ~15);                 // (behind the last tile: a tile that nobody takes)
      load_k();
      load_v();
      tile.logits(kv, scale_log2e, sv);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int n = j0 + 4 * hi + e;
        // rows behind the split's end were not loaded, and the scales read there may be anything
        if constexpr (F != kPlain) { sv[e] *= k_by[e]; v_by[e] = n < s1 ? v_by[e] : 0.f; }
        sv[e] = n < my_end ? sv[e] : -INFINITY;
      }
      if constexpr (F == kPlain) tile.accumulate_full(kv, sv, &scs[wave][0], lo, hi);
      else tile.accumulate_full(kv, sv, &scs[wave][0], lo, hi, [&](int e, float w) { return w * v_by[e]; });
    }
  }
  float* sm_m = lds + kChunkWaves * cap * D;
  float* sm_l = sm_m + kChunkWaves * cap;
  tile.finish(sm_m + wave * cap, sm_l + wave * cap, lds + wave * cap * D, lo, hi, rows);
  __syncthreads();

  // row r of the tile, to O
  auto store_row = [&](int r, int d4, float4 a) FASA_INLINE {
    const int tok = token_of(r);
    ET* o = O + (long long)(sc.row + tok) * o_stride + (long long)(h * G + (qt * kChunkRows + r) - tok * G) * D + 4 * d4;
    if constexpr (F32) *reinterpret_cast<float4*>(o) = a;
    else *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16(a.x, a.y), pack_bf16(a.z, a.w));
  };
  const size_t tile_id = (size_t)(b * Hkv + h) * tiles_each + qt;
  float* pa = part_acc + tile_id * splits * cap * D;
  float2* pm = reinterpret_cast<float2*>(part_ml) + tile_id * splits * cap;
  for (int x = t; x < rows * (D / 4); x += kChunkThreads) {
    const int r = x / (D / 4), d4 = x % (D / 4);
    float mn = kNegBig, l = 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kChunkWaves; ++w) mn = fmaxf(mn, sm_m[w * cap + r]);
#pragma unroll
    for (int w = 0; w < kChunkWaves; ++w) {
      const float by = exp2f(sm_m[w * cap + r] - mn);
      l = fmaf(sm_l[w * cap + r], by, l);
      const float4 o = *reinterpret_cast<const float4*>(lds + (size_t)(w * cap + r) * D + 4 * d4);
      a.x = fmaf(o.x, by, a.x); a.y = fmaf(o.y, by, a.y); a.z = fmaf(o.z, by, a.z); a.w = fmaf(o.w, by, a.w);
    }
    if (splits == 1) {
      store_row(r, d4, make_float4(a.x / l, a.y / l, a.z / l, a.w / l));
    } else {
      float2* to = reinterpret_cast<float2*>(pa + ((size_t)split * cap + r) * D + 4 * d4);
      st_agent(to, make_float2(a.x, a.y));
      st_agent(to + 1, make_float2(a.z, a.w));
      if (d4 == 0) st_agent(pm + split * cap + r, make_float2(mn, l));
    }
  }
  if (splits == 1) return;
  publish_barrier();
  uint32_t* tk = tickets + (size_t)(b * Hkv + h) * kChunkTickets + qt;
  if (t == 0) ticket = atomicAdd(tk, 1u);
  __syncthreads();
  if (ticket != (uint32_t)splits - 1u) return;
  if (t == 0) *tk = 0;                                                // clean for the next call

  // ---- the tile's last workgroup merges ----
  float* w = lds;                                                     // [row][split]
  for (int r = wave; r < rows; r += kChunkWaves) {
    float mx = kNegBig, sum = 0.f;
    for (int sp = lane; sp < splits; sp += kWave) mx = fmaxf(mx, ld_agent(pm + sp * cap + r).x);
    mx = wave_max(mx);
    for (int sp = lane; sp < splits; sp += kWave) {
      const float2 ml = ld_agent(pm + sp * cap + r);
      const float by = exp2f(ml.x - mx);
      w[r * splits + sp] = by;
      sum = fmaf(ml.y, by, sum);
    }
    sum = wave_sum(sum);
    if (lane == 0) red[r] = 1.0f / sum;
  }
  __syncthreads();
  const __amdgpu_buffer_rsrc_t rs = agent_buffer(pa);
  for (int x = t; x < rows * (D / 4); x += kChunkThreads) {
    const int r = x / (D / 4), d4 = x % (D / 4);
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int sp0 = 0; sp0 < splits; sp0 += 8) {
      uint4 o[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) o[u] = agent_load_u128(rs, (uint32_t)(((min(sp0 + u, splits - 1) * cap + r) * D + 4 * d4) * 4));
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float by = sp0 + u < splits ? w[r * splits + min(sp0 + u, splits - 1)] : 0.f;
        a.x = fmaf(__uint_as_float(o[u].x), by, a.x); a.y = fmaf(__uint_as_float(o[u].y), by, a.y);
        a.z = fmaf(__uint_as_float(o[u].z), by, a.z); a.w = fmaf(__uint_as_float(o[u].w), by, a.w);
      }
    }
    const float by = red[r];
    store_row(r, d4, make_float4(a.x * by, a.y * by, a.z * by, a.w * by));
  }
}

// Splits: as many as fill the compute units once, of 64 tokens or more, 256 at most (the merge's weights lie in LDS).
ChunkPlan plan_chunk(const fasa_shape& s, bool apart, int n_new, int n_rows, bool by_row_start) {
  ChunkPlan p{};
  const int G = s.n_q_heads / s.n_kv_heads;
  if (s.dtype == FASA_BF16 && (long long)n_new * G > kChunkRows) return plan_chunk_wide(s, apart, n_new, n_rows, by_row_start);
  p.tile_rows = n_new * (long long)G < kChunkRows ? n_new * G : kChunkRows;
  p.tiles = (int)chunk_tiles(by_row_start, s.batch, n_new, n_rows, G, kChunkRows);
  p.per_seq = (int)(((long long)n_new * G + kChunkRows - 1) / kChunkRows);
  const long long wgs = (long long)p.tiles * s.n_kv_heads;
  long long n = kAssumedCUs / wgs;
  const int most = (s.n_ctx + 63) / 64;
  if (n > most) n = most;
  if (n > 256) n = 256;
  if (p.per_seq > kChunkTickets) n = 1;
  p.splits = n < 1 ? 1 : (int)n;
  const size_t parts = p.splits == 1 ? 0 : (size_t)s.batch * s.n_kv_heads * p.per_seq * p.splits * p.tile_rows;
  p.part_acc_bytes = parts * kHeadDim * 4;
  p.part_ml_bytes = parts * 8;
  return p;
}

template <typename ET, CacheFmt F>
static hipError_t chunk_t(const fasa_shape& s, const ChunkPlan& p, const ChunkArgs& a, hipStream_t st) {
  using RT = typename RowType<ET, F>::type;
  const bool small = a.cv.pm.table != nullptr && a.cv.pm.shift < 4;
  const size_t totals = (size_t)kChunkWaves * p.tile_rows * (kHeadDim + 2) * 4, merge = (size_t)p.tile_rows * p.splits * 4;
  const auto kernel = small ? chunk_kernel<ET, F, true> : chunk_kernel<ET, F, false>;
  return launch_lds("fasa_chunk_attend", kernel, dim3((unsigned)((long long)p.tiles * s.n_kv_heads * p.splits)), dim3(kChunkThreads),
                    totals > merge ? totals : merge, st, (const ET*)a.q, (const RT*)a.cv.K, (const RT*)a.cv.V, (ET*)a.O, a.part_acc, a.part_ml,
                    a.tickets, a.cv, a.ch, s.batch, s.n_kv_heads, s.n_q_heads / s.n_kv_heads, p.per_seq, p.splits, p.tile_rows, a.q_stride,
                    a.o_stride, 1.4426950408889634f / sqrtf((float)s.head_dim));
}

hipError_t launch_chunk(const fasa_shape& s, const ChunkPlan& p, const ChunkArgs& a, hipStream_t st) {
  if (s.dtype == FASA_BF16)
    return a.fmt == kPlain ? chunk_t<uint16_t, kPlain>(s, p, a, st) : a.fmt == kInt8 ? chunk_t<uint16_t, kInt8>(s, p, a, st) : chunk_t<uint16_t, kE4m3>(s, p, a, st);
  return a.fmt == kPlain ? chunk_t<float, kPlain>(s, p, a, st) : a.fmt == kInt8 ? chunk_t<float, kInt8>(s, p, a, st) : chunk_t<float, kE4m3>(s, p, a, st);
}

}  // namespace fasa
