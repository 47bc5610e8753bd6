// Attention of a few query rows of a KV head over its cache: single tokens, a few drafted ones, and float32 chunks of any length.
// Query rows (new token i, head g of the group) of a sequence and KV head go by tiles of 16, the columns of the matrix cores' 16-row
// tile engine (mfma_tile.h); a tile's tokens are shared out to workgroups, a wave of which takes 16 at a time, and the
// last workgroup of a tile by ticket merges the partial results.  Bound by reading the rows, once per tile.
#include <algorithm>

#include "chunk_common.h"
#include "mfma_tile.h"

namespace fasa {

// Waves of a workgroup.  A wave has a tile of 16 tokens in flight: 8 KB of bf16 rows, 4 KB of 8-bit ones, of which a compute unit needs eight for what four of the former
// do.  us, four / eight waves: bf16, 8 rows of 8192: 12.0 / 13.0, of 32768: 29.9 / 31.8, 128 of 4864 - 16384: 134 / 138; e4m3, 8 of 131072: 69.8 / 52.4 (with two tiles in
// flight 58.0); float32, 37 new tokens over 4096: 18.2 / 15.9.
template <typename ET, CacheFmt F> constexpr int kChunkWaves = F == kPlain && sizeof(ET) == 2 ? 4 : 8;
constexpr int kChunkRows = kTokenForm.rows;
constexpr int kTicketWords = 8;                          // from a tile's ticket to the next: tickets of different rows, whose workgroups run on different XCDs, share no line
static_assert(kTokenForm.resident <= kTokenForm.resident_by_length && kTokenForm.resident_by_length * kTicketWords <= kChunkTickets, "a ticket for each tile that is split");

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
__global__ __launch_bounds__((64 * kChunkWaves<ET, F>), 2) void chunk_kernel(
    const ET* __restrict__ q, const typename RowType<ET, F>::type* __restrict__ K, const typename RowType<ET, F>::type* __restrict__ V, ET* __restrict__ O,
    float* __restrict__ part_acc, float2* __restrict__ part_ml, uint32_t* __restrict__ tickets, CacheView cv, ChunkView ch, int batch, int Hkv, int G,
    int tiles_each, int whole, int all_splits, int units, int all_parts, int cap, long long q_stride, long long o_stride, float scale_log2e) {
  constexpr int D = kHeadDim, NWV = kChunkWaves<ET, F>, NT = 64 * NWV, ROUND = 16 * NWV;     // tokens of a round of the waves
  constexpr bool F32 = sizeof(ET) == 4;
  using RT = typename RowType<ET, F>::type;
  // waves' totals: [wave][cap][D], then m, l [wave][cap]; the merge: weights [row][split]
  extern __shared__ __align__(16) float lds[];
  __shared__ __align__(16) float scs[NWV][16];
  __shared__ float red[kChunkRows];
  __shared__ uint32_t ticket;

  // workgroups: heads fastest (the blocks of a paged cache often hold all heads' rows side by side)
  const int h = (int)(blockIdx.x % (unsigned)Hkv);
  ChunkUnit u;
  if (!find_chunk_unit<kChunkRows>(ch, batch, G, tiles_each, whole, all_splits, units, kTokenForm.least, blockIdx.x / (unsigned)Hkv, u)) return;
  const int b = u.b, splits = u.splits, qrow = ((u.seq.n_new * G - 1) / kChunkRows - u.tile) * kChunkRows;     // the longest first
  const int rows = min(cap, u.seq.n_new * G - qrow);                 // of this tile
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int lo = lane & 15, hi = lane >> 4;
  const int pos0 = u.seq.n_ctx - u.seq.n_new;
  const auto token_of = [&](int r) FASA_INLINE { return (qrow + r) / G; };
  const int seen = pos0 + token_of(rows - 1) + 1;                    // by the last row of the tile
  const int share = u.share ? u.share : ((seen + splits - 1) / splits + 15) & ~15;
  const int s0 = (int)min((long long)u.split * share, (long long)seen), s1 = min(seen, s0 + share);

  MfmaTile<kChunkRows, ET> tile;
  const int my = min(lo, rows - 1), my_tok = token_of(my);
  const int my_end = min(s1, pos0 + my_tok + 1);                     // of query row lo
  {
    const ET* p = q + (long long)(u.seq.row + my_tok) * q_stride + (long long)(h * G + (qrow + my) - my_tok * G) * D;
#pragma unroll
    for (int i = 0; i < (F32 ? 8 : 4); ++i)
      tile.qb[i] = __builtin_bit_cast(typename MfmaTile<kChunkRows, ET>::QT, *reinterpret_cast<const uint4*>(p + chunk_dim<ET, F>(i, hi)));
  }
  tile.reset();

  const bool paged = cv.pm.table != nullptr;
  const long long seq = (paged ? 0 : b * cv.sb) + h * cv.sh, sseq = (paged ? 0 : b * cv.ssb) + h * cv.ssh;
  const RT* Kh = K + seq + (F == kPlain ? kChunk<ET> : 16) * hi;
  const RT* Vh = V + seq + 8 * lo;
  const float* ksh = F == kPlain ? nullptr : cv.ks + sseq;
  const float* vsh = F == kPlain ? nullptr : cv.vs + sseq;
  const long long sb = paged ? cv.sb : 0, ssb = paged ? cv.ssb : 0;
  const int32_t* const table = paged ? cv.pm.table + (size_t)b * cv.pm.max_blocks : reinterpret_cast<const int32_t*>(q);   // (an entry is read in any case)
  const int shift = paged ? cv.pm.shift : 31, in_block = paged ? (1 << cv.pm.shift) - 1 : 0x7fffffff, blk_max = paged ? cv.pm.n_pool - 1 : 0;
  const auto block_of = [&](int n) FASA_INLINE { return min(max(table[n >> shift], 0), blk_max); };
  typename std::conditional<F == kPlain, TileKV<ET>, RawKV<ET, F>>::type raw;
  f32x4_t ks = {1.f, 1.f, 1.f, 1.f}, vs = ks;
  struct Place { long long k, v[4], vs[4]; } pl;                     // rows and scales of the next tile
  // Lane l: the block of this wave's l-th tile from here on.  A lookup between a tile's loads and the next one's would wait for the former.
  int entries = 0;
  auto look_up = [&](int j0) FASA_INLINE {
    if constexpr (!SMALL) entries = block_of((int)min((long long)j0 + (long long)ROUND * lane, (long long)s1 - 1));
  };
  // rows from token j0 on, this wave's i-th tile since the lookup; tokens behind the split's last are the last again
  auto find_rows = [&](int j0, int i) FASA_INLINE {
    if constexpr (SMALL) {
      const int nk = min(j0 + lo, s1 - 1);
      pl.k = block_of(nk) * sb + (nk & in_block) * cv.sn;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int n = min(j0 + 4 * hi + e, s1 - 1), blk = block_of(n);
        pl.v[e] = blk * sb + (n & in_block) * cv.sn;
        pl.vs[e] = blk * ssb + (n & in_block);
      }
    } else {
      const int last = min(s1 - 1 - j0, 15), blk = __builtin_amdgcn_readlane(entries, i);     // (j0 is a multiple of 16)
      const long long base = blk * sb + (j0 & in_block) * cv.sn;
      pl.k = base + min(lo, last) * cv.sn;
#pragma unroll
      for (int e = 0; e < 4; ++e) pl.v[e] = base + min(4 * hi + e, last) * cv.sn;
      pl.vs[0] = blk * ssb + (j0 & in_block) + min(4 * hi, last & ~3);                        // four at once: rows of scales are whole fours
    }
  };
  auto scales = [&](const float* from) FASA_INLINE {
    f32x4_t x = {1.f, 1.f, 1.f, 1.f};
    if constexpr (F != kPlain) {
      if constexpr (SMALL) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = from[pl.vs[e]];
      } else {
        x = *reinterpret_cast<const f32x4_t*>(from + pl.vs[0]);
      }
    }
    return x;
  };
  auto load_k = [&]() FASA_INLINE { raw.load_k(Kh + pl.k); ks = scales(ksh); };
  auto load_v = [&]() FASA_INLINE {
#pragma unroll
    for (int e = 0; e < 4; ++e) raw.load_v(e, Vh + pl.v[e]);
    vs = scales(vsh);
  };
  int j0 = s0 + 16 * wave;
  if (j0 < s1) {
    look_up(j0);
    find_rows(j0, 0);
    load_k();
    load_v();
    for (int i = 1; j0 < s1; j0 += ROUND, ++i) {
      if ((i & 63) == 0) look_up(j0 + ROUND);
      const bool more = j0 + ROUND < s1;
      find_rows(more ? j0 + ROUND : j0, (more ? i : i - 1) & 63);     // (behind the last tile that tile again, for nobody)
      float sv[4];
      auto seen_only = [&]() FASA_INLINE {
#pragma unroll
        for (int e = 0; e < 4; ++e) sv[e] = j0 + 4 * hi + e < my_end ? sv[e] : -INFINITY;
      };
      if constexpr (F == kPlain) {
        // One set of registers: the next tile's K goes where this one's has been used, and runs under this tile's P . V, its V under the next logits.
        tile.logits(raw, scale_log2e, sv);
        __builtin_amdgcn_sched_barrier(0);
        load_k();
        __builtin_amdgcn_sched_barrier(0);
        seen_only();
        tile.accumulate_full(raw, sv, &scs[wave][0], lo, hi);
        __builtin_amdgcn_sched_barrier(0);
        load_v();
        __builtin_amdgcn_sched_barrier(0);
      } else {
        // Values go into registers of their own, and all of the next tile is asked for at once.
        TileKV<ET> kv;
        const f32x4_t k_by = ks;
        f32x4_t v_by;
        // (scales of tokens that the query does not see may be anything, a NaN too)
#pragma unroll
        for (int e = 0; e < 4; ++e) v_by[e] = j0 + 4 * hi + e < my_end ? vs[e] : 0.f;
        raw.k_to(kv);
        raw.v_to(kv);
        load_k();
        load_v();
        tile.logits(kv, scale_log2e, sv);
#pragma unroll
        for (int e = 0; e < 4; ++e) sv[e] *= k_by[e];
        seen_only();
        tile.accumulate_full(kv, sv, &scs[wave][0], lo, hi, [&](int e, float w) FASA_INLINE { return w * v_by[e]; });
      }
    }
  }
  float* sm_m = lds + NWV * cap * D;
  float* sm_l = sm_m + NWV * cap;
  tile.finish(sm_m + wave * cap, sm_l + wave * cap, lds + wave * cap * D, lo, hi, rows);
  __syncthreads();

  // row r of the tile, to O
  auto store_row = [&](int r, int d4, float4 a) FASA_INLINE {
    const int tok = token_of(r);
    ET* o = O + (long long)(u.seq.row + tok) * o_stride + (long long)(h * G + (qrow + r) - tok * G) * D + 4 * d4;
    if constexpr (F32) *reinterpret_cast<float4*>(o) = a;
    else *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16(a.x, a.y), pack_bf16(a.z, a.w));
  };
  // partial results: [head][unit][cap]
  const size_t part0 = ((size_t)h * all_parts + u.first) * cap;
  float* pa = part_acc + part0 * D;
  float2* pm = part_ml + part0;
  for (int x = t; x < rows * (D / 4); x += NT) {
    const int r = x / (D / 4), d4 = x % (D / 4);
    float mn = kNegBig, l = 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < NWV; ++w) mn = fmaxf(mn, sm_m[w * cap + r]);
#pragma unroll
    for (int w = 0; w < NWV; ++w) {
      const float by = exp2f(sm_m[w * cap + r] - mn);
      l = fmaf(sm_l[w * cap + r], by, l);
      const float4 o = *reinterpret_cast<const float4*>(lds + (size_t)(w * cap + r) * D + 4 * d4);
      a.x = fmaf(o.x, by, a.x); a.y = fmaf(o.y, by, a.y); a.z = fmaf(o.z, by, a.z); a.w = fmaf(o.w, by, a.w);
    }
    if (splits == 1) {
      store_row(r, d4, make_float4(a.x / l, a.y / l, a.z / l, a.w / l));
    } else {
      float2* to = reinterpret_cast<float2*>(pa + ((size_t)u.split * cap + r) * D + 4 * d4);
      st_agent(to, make_float2(a.x, a.y));
      st_agent(to + 1, make_float2(a.z, a.w));
      if (d4 == 0) st_agent(pm + (size_t)u.split * cap + r, make_float2(mn, l));
    }
  }
  if (splits == 1) return;
  publish_barrier();
  uint32_t* tk = tickets + (size_t)(b * Hkv + h) * kChunkTickets + kTicketWords * u.slot;
  if (t == 0) ticket = atomicAdd(tk, 1u);
  __syncthreads();
  if (ticket != (uint32_t)splits - 1u) return;
  if (t == 0) *tk = 0;                                                // clean for the next call

  // ---- the tile's last workgroup merges ----
  float* w = lds;                                                     // [row][split]
  for (int r = wave; r < rows; r += NWV) {
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
  for (int x = t; x < rows * (D / 4); x += NT) {
    const int r = x / (D / 4), d4 = x % (D / 4);
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int sp0 = 0; sp0 < splits; sp0 += 8) {
      uint4 o[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) o[k] = agent_load_u128(rs, (uint32_t)(((min(sp0 + k, splits - 1) * cap + r) * D + 4 * d4) * 4));
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float by = sp0 + k < splits ? w[r * splits + min(sp0 + k, splits - 1)] : 0.f;
        a.x = fmaf(__uint_as_float(o[k].x), by, a.x); a.y = fmaf(__uint_as_float(o[k].y), by, a.y);
        a.z = fmaf(__uint_as_float(o[k].z), by, a.z); a.w = fmaf(__uint_as_float(o[k].w), by, a.w);
      }
    }
    const float by = red[r];
    store_row(r, d4, make_float4(a.x * by, a.y * by, a.z * by, a.w * by));
  }
}
// Float32, and up to 16 query rows of a KV head: by 16-row tiles (20 rows, 32768 tokens: those 36.9 us, chunk_wide.hip 36.4; 8-bit 31.1 / 30.2).  Up to 128, or where rows
// have to be looked up one by one: the short form (32 heads over 8, 32768 tokens, 32 new ones: 50.4 us, the deep form 58.0; 33: 59.5 / 58.0, 64: 70 / 65).  That one also where
// tiles of 256 rows in the least parts would leave half of the compute units without work (us, short / deep: 512 tokens, 256 new ones 20.6 / 25.7; 2048, 128: 21.7 / 26.3;
// 4096, 64: 21.6 / 26.1; and with twice as many parts 2048, 256: 31.5 / 31.1, 8192, 64: 31.6 / 30.8), and for contexts of up to 1024 tokens, of which a workgroup has so few that its
// begin and end count, which two on a compute unit hide (prompts, 4 of 1024: 63 / 73, 8 of 512: 43 / 50, 4 of 2048: 195 / 189).
static ChunkForm chunk_form(const fasa_shape& s, bool apart, const ChunkView& ch) {
  const int G = s.n_q_heads / s.n_kv_heads;
  const long long m = (long long)ch.n_new * G;
  if (s.dtype == FASA_F32 || m <= kTokenForm.rows) return kTokenForm;
  if (m <= kShortForm.rows || apart || s.n_ctx <= 1024) return kShortForm;
  const long long tiles = chunk_tiles(ch.row_start != nullptr, s.batch, ch.n_new, ch.n_rows, G, kDeepForm.rows);
  return tiles * s.n_kv_heads * ((s.n_ctx + kDeepForm.least - 1) / kDeepForm.least) <= kDeepForm.resident / 2 ? kShortForm : kDeepForm;
}

ChunkPlan plan_chunk(const fasa_shape& s, bool apart, const ChunkView& ch) {
  const int G = s.n_q_heads / s.n_kv_heads;
  const long long m = (long long)ch.n_new * G;
  ChunkPlan p{};
  p.form = chunk_form(s, apart, ch);
  p.apart = apart;
  p.tile_rows = p.form.rows == kTokenForm.rows && m < p.form.rows ? (int)m : p.form.rows;
  p.per_seq = (int)((m + p.tile_rows - 1) / p.tile_rows);
  const long long tiles = chunk_tiles(ch.row_start != nullptr, s.batch, ch.n_new, ch.n_rows, G, p.tile_rows);
  const long long units = p.form.resident / s.n_kv_heads;
  // By length: parts of a sequence are whole, so its last is half a part too long on average, tiles / 2 of them in all; with twice the workgroups half of that, but then a
  // compute unit has two after each other, which costs about what 800 tokens take.  (us, once / twice, 8 KV heads, int8: 4 sequences of 670 - 1531 9.7 / 15.2, 8 of 2816 - 8192
  // 25.1 / 31.7, 16 of 2432 - 8192 49.0 / 50.7, 4 of 28672 - 65536 86.7 / 91.2, 16 of 4864 - 16384 88.6 / 84.6, bf16 138.6 / 139.1.)
  const bool once = tiles <= units && (long long)s.batch * s.n_ctx * tiles < 3200 * units * units;
  const long long units_by_length = once ? units : p.form.resident_by_length / s.n_kv_heads;
  p.by_length = (ch.n_ctx_seq || ch.n_new_seq) && s.batch > 1 && s.batch <= kWave && tiles <= units_by_length;
  const long long by_tokens = (s.n_ctx + p.form.least - 1) / p.form.least, most = std::min(by_tokens, (long long)p.form.splits);
  p.splits = 1;
  // Uniform: as many tiles whole as make full rounds, and the others in parts, so many that what they take in rounds of workgroups is the least.
  // us without / with: 32 heads over 8, 32768 tokens: 700 new ones (88 tiles for 256 workgroups) 499 / 445, 1100 (144) 953 / 702, 2200 (280) 1912 / 1200, 3000 (376) 1893 / 1578; over
  // 4096: 700 82.6 / 82.8, 1100 127 / 110, 2200 159 / 148.  A token each, int8 and bf16, 8 KV heads, of 12000: 20 sequences 137 / 108, 198 / 185, 12: 74.7 / 70.1, 114 / 114; of 4000: 20:
  // 49.8 / 44.1, 69 / 67, 36: 96 / 69, 152 / 110, 5: 14.3 / 14.4, 17.1 / 17.2.  72 x 8 drafted ones 279 / 230.  Float32, 150 new ones over 4096: 174 / 113.
  if (!p.by_length && units > 0) {
    const long long left = tiles % units, all = p.form.parts / s.n_kv_heads;
    p.whole = (int)(tiles - left);
    const long long seen = p.whole && s.batch == 1 ? s.n_ctx - ch.n_new + left * p.tile_rows / G : s.n_ctx;      // (of one sequence the shortest tiles are left)
    const auto cost = [&](long long n) { return (left * n + units - 1) / units * (seen / n + p.form.begin) + (n > 1 ? left * n * s.n_kv_heads * p.form.join + 40 : 0); };
    for (long long n = 2; n <= most && left * n <= all; ++n)
      if (cost(n) < cost(p.splits)) p.splits = (int)n;
  }
  if (p.splits == 1 && !p.by_length) p.whole = (int)tiles;
  p.units = (int)(p.by_length ? std::min(units_by_length, tiles * by_tokens) : p.whole + (tiles - p.whole) * p.splits);
  p.parts = p.by_length ? p.units : p.units - p.whole;
  const size_t parts = (size_t)p.parts * s.n_kv_heads * p.tile_rows;
  p.part_acc_bytes = parts * kChunkAccBytes;
  p.part_ml_bytes = parts * kChunkMlBytes;
  return p;
}

// A call's tiles have `query` rows together at most and one unfinished tile for each sequence; parts are at most `most` to a tile, and as many as workgroups are resident.
size_t most_chunk_parts(const fasa_shape& s, const ChunkView& ch) {
  const long long G = s.n_q_heads / s.n_kv_heads, query = (ch.row_start ? (long long)ch.n_rows : (long long)s.batch * ch.n_new) * G;
  size_t parts = 0;
  for (const ChunkForm& f : {kTokenForm, kShortForm, kDeepForm}) {
    if (f.rows != kTokenForm.rows && (s.dtype == FASA_F32 || ch.n_new * G <= kTokenForm.rows)) continue;
    const long long most = (s.n_ctx + f.least - 1) / f.least;
    const long long by_tokens = std::min(most, (long long)f.parts) * (query + (long long)s.batch * f.rows) * s.n_kv_heads;
    parts = std::max(parts, (size_t)std::min(by_tokens, (long long)f.parts * f.rows));
  }
  return parts;
}

template <typename ET, CacheFmt F>
static hipError_t chunk_t(const fasa_shape& s, const ChunkPlan& p, const ChunkArgs& a, hipStream_t st) {
  using RT = typename RowType<ET, F>::type;
  const bool small = a.cv.pm.table != nullptr && a.cv.pm.shift < 4;
  const int hkv = s.n_kv_heads, G = s.n_q_heads / hkv;
  const size_t totals = (size_t)kChunkWaves<ET, F> * p.tile_rows * (kHeadDim + 2) * 4, merge = (size_t)p.tile_rows * (p.by_length ? p.units : p.splits) * 4;
  const auto kernel = small ? chunk_kernel<ET, F, true> : chunk_kernel<ET, F, false>;
  return launch_lds("fasa_chunk_attend", kernel, dim3((unsigned)p.units * (unsigned)hkv), dim3(64 * kChunkWaves<ET, F>), totals > merge ? totals : merge, st,
                    (const ET*)a.q, (const RT*)a.cv.K, (const RT*)a.cv.V, (ET*)a.O, a.part_acc, (float2*)a.part_ml, a.tickets, a.cv, a.ch, s.batch, hkv, G,
                    p.per_seq, p.whole, p.splits, p.by_length ? p.units : 0, p.parts, p.tile_rows, a.q_stride, a.o_stride, 1.4426950408889634f / sqrtf((float)s.head_dim));
}

hipError_t launch_chunk(const fasa_shape& s, const ChunkPlan& p, const ChunkArgs& a, hipStream_t st) {
  if (s.dtype == FASA_BF16)
    return a.fmt == kPlain ? chunk_t<uint16_t, kPlain>(s, p, a, st) : a.fmt == kInt8 ? chunk_t<uint16_t, kInt8>(s, p, a, st) : chunk_t<uint16_t, kE4m3>(s, p, a, st);
  return a.fmt == kPlain ? chunk_t<float, kPlain>(s, p, a, st) : a.fmt == kInt8 ? chunk_t<float, kInt8>(s, p, a, st) : chunk_t<float, kE4m3>(s, p, a, st);
}

}  // namespace fasa
