// Attention of a chunk of bf16 query rows over a bf16 or 8-bit cache: many query rows of a KV head (new token, head of the group) against the same K and V,
// both products on the matrix cores, K and V tiles of 64 tokens shared by the workgroup through LDS.
//
//   S^T = K Q^T   (tokens x queries; 32 x 32 x 16 MFMAs, K from LDS, Q in registers): the result's column, a lane's own, is one query, its 16
//                 registers are tokens 8 (i / 4) + 4 (lane / 32) + i % 4.  Maximum, exponentials and sum of a query are the lane's own but for one exchange
//                 with the lane 32 on.
//   O^T += V^T P^T (dims x queries): what the lane has of P^T, as bf16, is the second operand as it stands: its k-slots 0-3, 4-7 are the tokens of registers
//                 8 s .. 8 s + 7 of k-step s.  V^T with tokens in that order comes out of LDS by transposing reads (ds_read_b64_tr_b16: 16 lanes get
//                 one column each of four rows).  A new maximum rescales a lane's own accumulators.
// LDS rows are 256 bytes of 16-byte chunks; chunk c of token t is stored at c ^ (t mod 16) (K) or c ^ 2 (t mod 8) (V), so that the lanes
// of a read fall on all banks.
#include "chunk_common.h"

namespace fasa {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

constexpr int kWideTok = 64;                              // tokens of a tile
constexpr int kTileBytes = kWideTok * kHeadDim * 2;       // of K or V in LDS

__device__ __forceinline__ int swz_k(int t) { return t & 15; }
__device__ __forceinline__ int swz_v(int t) { return 2 * (t & 7); }

// Four bf16 of one column of V for each of 16 lanes, out of four rows of LDS
__device__ __forceinline__ uint2 lds_read_tr(__attribute__((address_space(3))) const unsigned char* p) {
  const s16x4_t r = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)p);
  return __builtin_bit_cast(uint2, r);
}

template <CacheFmt F, int NW>
__global__ __launch_bounds__(64 * NW, 2) void chunk_wide_kernel(const uint16_t* __restrict__ q, const typename RowType<uint16_t, F>::type* __restrict__ K,
                                                                const typename RowType<uint16_t, F>::type* __restrict__ V, uint16_t* __restrict__ O,
                                                                float* __restrict__ part_acc, float2* __restrict__ part_ml, CacheView cv, ChunkView ch,
                                                                int batch, int Hkv, int G, int tiles_each, int splits, long long q_stride,
                                                                long long o_stride, float scale_log2e) {
  constexpr int D = kHeadDim, NT = 64 * NW, TR = 32 * NW;
  constexpr bool BYTES = F != kPlain;
  using RT = typename RowType<uint16_t, F>::type;
  constexpr int PER_ROW = BYTES ? 8 : 16;                 // 16-byte pieces of a stored row
  constexpr int NL = kWideTok * PER_ROW / NT;             // pieces of K, and of V, a thread
  extern __shared__ __align__(16) unsigned char smem[];   // [2][K tile, V tile], then scales [2][k 64, v 64]
  float* sm_scale = reinterpret_cast<float*>(smem + 4 * kTileBytes);

  unsigned id = blockIdx.x;
  const int h = (int)(id % (unsigned)Hkv);
  id /= (unsigned)Hkv;
  const int split = (int)(id % (unsigned)splits);
  id /= (unsigned)splits;
  int b, qt;
  if (!find_chunk_tile<TR>(ch, batch, G, tiles_each, id, b, qt)) return;
  const SeqChunk sc = seq_chunk(ch, b);
  const int m = sc.n_new * G, m_tiles = (m + TR - 1) / TR;
  if (qt >= m_tiles) return;
  qt = m_tiles - 1 - qt;                                   // the longest first
  const int rows = min(TR, m - qt * TR);
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int pos0 = sc.n_ctx - sc.n_new;
  const auto token_of = [&](int r) FASA_INLINE { return (qt * TR + r) / G; };
  const int seen = pos0 + token_of(rows - 1) + 1;          // tokens that the tile's last row sees
  const int share = ((seen + splits - 1) / splits + kWideTok - 1) / kWideTok * kWideTok;
  const int s0 = min(split * share, seen), s1 = min(seen, s0 + share);
  const int n_tiles = (s1 - s0 + kWideTok - 1) / kWideTok;

  // this lane's query
  const int my = min(32 * wave + col, rows - 1), my_tok = token_of(my);
  const int my_end = min(s1, pos0 + my_tok + 1);
  const int wave_all = min(s1, pos0 + token_of(min(32 * wave, rows - 1)) + 1);         // tokens that all of the wave's queries see
  const int wave_end = 32 * wave < rows ? min(s1, pos0 + token_of(min(32 * wave + 31, rows - 1)) + 1) : s0;
  bf16x8_t qb[8];
  {
    const uint16_t* p = q + (long long)(sc.row + my_tok) * q_stride + (long long)(h * G + (qt * TR + my) - my_tok * G) * D + 8 * half;
#pragma unroll
    for (int i = 0; i < 8; ++i) qb[i] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const uint4*>(p + 16 * i));
  }
  f32x16_t oc[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) oc[i] = f32x16_t{};
  float m_run = kNegBig, l_run = 0.f;

  // ---- loader: piece x of a tile is 16 bytes of row x / PER_ROW ----
  uint4 rk[NL], rv[NL];
  float rs = 0.f;                                          // threads 0-63: scale of K row t, 64-127: of V row t - 64
  const RT* Kh = K + h * cv.sh;
  const RT* Vh = V + h * cv.sh;
  // A tile's blocks are looked up a tile ahead of its loads: a lookup between loads would wait for all loads before it.
  int blk[NL], sblk = 0;
  auto look_up = [&](int j0) FASA_INLINE {
#pragma unroll
    for (int i = 0; i < NL; ++i) blk[i] = cache_block(cv.pm, b, min(j0 + (t + NT * i) / PER_ROW, s1 - 1));
    if constexpr (BYTES) sblk = cache_block(cv.pm, b, min(j0 + (t & 63), s1 - 1));
  };
  auto load_tile = [&](int j0) FASA_INLINE {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int x = t + NT * i;
      const long long at = cache_clamp(cv.pm, blk[i]) * cv.sb + cache_offset(cv.pm, min(j0 + x / PER_ROW, s1 - 1)) * cv.sn + (x % PER_ROW) * (16 / (int)sizeof(RT));
      rk[i] = *reinterpret_cast<const uint4*>(Kh + at);
      rv[i] = *reinterpret_cast<const uint4*>(Vh + at);
    }
    if constexpr (BYTES) {
      if (t < 2 * kWideTok) rs = (t < kWideTok ? cv.ks : cv.vs)[cache_clamp(cv.pm, sblk) * cv.ssb + h * cv.ssh + cache_offset(cv.pm, min(j0 + (t & 63), s1 - 1))];
    }
    look_up(j0 + kWideTok);
  };
  auto store_tile = [&](int buf) FASA_INLINE {
    unsigned char* k = smem + buf * 2 * kTileBytes;
    unsigned char* v = k + kTileBytes;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int x = t + NT * i, r = x / PER_ROW, c = x % PER_ROW;
      if constexpr (BYTES) {
        const uint32_t wk[4] = {rk[i].x, rk[i].y, rk[i].z, rk[i].w}, wv[4] = {rv[i].x, rv[i].y, rv[i].z, rv[i].w};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint2 ka = bytes_to_bf16<F>(wk[2 * j]), kb = bytes_to_bf16<F>(wk[2 * j + 1]);
          const uint2 va = bytes_to_bf16<F>(wv[2 * j]), vb = bytes_to_bf16<F>(wv[2 * j + 1]);
          *reinterpret_cast<uint4*>(k + r * 256 + (((2 * c + j) ^ swz_k(r)) << 4)) = make_uint4(ka.x, ka.y, kb.x, kb.y);
          *reinterpret_cast<uint4*>(v + r * 256 + (((2 * c + j) ^ swz_v(r)) << 4)) = make_uint4(va.x, va.y, vb.x, vb.y);
        }
      } else {
        *reinterpret_cast<uint4*>(k + r * 256 + ((c ^ swz_k(r)) << 4)) = rk[i];
        *reinterpret_cast<uint4*>(v + r * 256 + ((c ^ swz_v(r)) << 4)) = rv[i];
      }
    }
    if constexpr (BYTES) {
      if (t < 2 * kWideTok) sm_scale[buf * 2 * kWideTok + t] = t < kWideTok ? rs * scale_log2e : rs;
    }
  };

  if (n_tiles > 0) {
    look_up(s0);
    load_tile(s0);
    store_tile(0);
    if (n_tiles > 1) load_tile(s0 + kWideTok);
    __syncthreads();
  }
  for (int j = 0; j < n_tiles; ++j) {
    const int j0 = s0 + j * kWideTok, buf = j & 1;
    const unsigned char* kt = smem + buf * 2 * kTileBytes;
    const unsigned char* vt = kt + kTileBytes;
    const bool work = j0 < wave_end;
    f32x16_t sv[2];
    if (work) {
      sv[0] = f32x16_t{};
      sv[1] = f32x16_t{};
#pragma unroll
      for (int s = 0; s < 8; ++s)
#pragma unroll
        for (int nb = 0; nb < 2; ++nb) {
          const int r = 32 * nb + col;
          const uint4 a = *reinterpret_cast<const uint4*>(kt + r * 256 + (((2 * s + half) ^ swz_k(r)) << 4));
          sv[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), qb[s], sv[nb], 0, 0, 0);
        }
    }
    if (j + 1 < n_tiles) store_tile(buf ^ 1);
    if (j + 2 < n_tiles) load_tile(j0 + 2 * kWideTok);
    if (work) {
      float mul = scale_log2e;
      if constexpr (BYTES) {
        const float* ks = sm_scale + buf * 2 * kWideTok;
#pragma unroll
        for (int nb = 0; nb < 2; ++nb)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const float4 f = *reinterpret_cast<const float4*>(ks + 32 * nb + 8 * g + 4 * half);
            sv[nb][4 * g] *= f.x; sv[nb][4 * g + 1] *= f.y; sv[nb][4 * g + 2] *= f.z; sv[nb][4 * g + 3] *= f.w;
          }
        mul = 1.f;
      }
      if (j0 + kWideTok > wave_all) {
#pragma unroll
        for (int nb = 0; nb < 2; ++nb)
#pragma unroll
          for (int i = 0; i < 16; ++i) sv[nb][i] = j0 + 32 * nb + 8 * (i / 4) + 4 * half + i % 4 < my_end ? sv[nb][i] : -INFINITY;
      }
      float mx = sv[0][0];
#pragma unroll
      for (int nb = 0; nb < 2; ++nb)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sv[nb][i]);
      mx = xor32_max(mx) * mul;
      const float m_new = fmaxf(m_run, mx);
      if (__ballot(m_new != m_run) != 0ull) {
        const float by = __builtin_amdgcn_exp2f(m_run - m_new);
        m_run = m_new;
        l_run *= by;
#pragma unroll
        for (int d = 0; d < 4; ++d) oc[d] *= by;
      }
      uint32_t pw[2][8];
#pragma unroll
      for (int nb = 0; nb < 2; ++nb) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          sv[nb][i] = __builtin_amdgcn_exp2f(BYTES ? sv[nb][i] - m_new : __builtin_fmaf(sv[nb][i], mul, -m_new));
          l_run += sv[nb][i];
        }
        if constexpr (BYTES) {
          const float* vs = sm_scale + buf * 2 * kWideTok + kWideTok;
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const float4 f = *reinterpret_cast<const float4*>(vs + 32 * nb + 8 * g + 4 * half);
            sv[nb][4 * g] *= f.x; sv[nb][4 * g + 1] *= f.y; sv[nb][4 * g + 2] *= f.z; sv[nb][4 * g + 3] *= f.w;
          }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) pw[nb][i] = pack_bf16(sv[nb][2 * i], sv[nb][2 * i + 1]);
      }
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const bf16x8_t p = __builtin_bit_cast(bf16x8_t, make_uint4(pw[s / 2][4 * (s & 1)], pw[s / 2][4 * (s & 1) + 1], pw[s / 2][4 * (s & 1) + 2], pw[s / 2][4 * (s & 1) + 3]));
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          const int r = 16 * s + 4 * half + ((lane & 15) >> 2), c = 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
          const unsigned char* at = vt + ((c ^ swz_v(r)) << 4) + 8 * (lane & 1) + r * 256;
          const unsigned char* at8 = vt + ((c ^ swz_v(r + 8)) << 4) + 8 * (lane & 1) + (r + 8) * 256;
          const uint2 lo = lds_read_tr((__attribute__((address_space(3))) const unsigned char*)at), hi = lds_read_tr((__attribute__((address_space(3))) const unsigned char*)at8);
          oc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, make_uint4(lo.x, lo.y, hi.x, hi.y)), p, oc[d], 0, 0, 0);
        }
      }
    }
    __syncthreads();
  }
  l_run = xor32_sum(l_run);
  if (32 * wave + col >= rows) return;
  if (splits == 1) {
    const float by = 1.0f / l_run;
    uint16_t* o = O + (long long)(sc.row + my_tok) * o_stride + (long long)(h * G + (qt * TR + my) - my_tok * G) * D + 4 * half;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<uint2*>(o + 32 * d + 8 * g) = make_uint2(pack_bf16(oc[d][4 * g] * by, oc[d][4 * g + 1] * by), pack_bf16(oc[d][4 * g + 2] * by, oc[d][4 * g + 3] * by));
    return;
  }
  const size_t at = (((size_t)(b * Hkv + h) * tiles_each + qt) * splits + split) * TR + my;
  float* pa = part_acc + at * D + 4 * half;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<float4*>(pa + 32 * d + 8 * g) = make_float4(oc[d][4 * g], oc[d][4 * g + 1], oc[d][4 * g + 2], oc[d][4 * g + 3]);
  if (half == 0) part_ml[at] = make_float2(m_run, l_run);
}

// largest of a lane's sixteen logits
__device__ __forceinline__ float largest(const f32x16_t& v) {
  float m = __builtin_fmaxf(v[0], v[1]);
#pragma unroll
  for (int i = 2; i < 16; i += 2) m = __builtin_fmaxf(m, __builtin_fmaxf(v[i], v[i + 1]));
  return m;
}

// The same for long chunks, eight waves of 32 queries (256 rows a tile), two a SIMD.  In steps of 32 tokens: step u runs the logits of step u + 1 and the
// output of step u - 1 beside its own exponentials, in one block of straight code, so that the matrix cores have work while a wave is at its softmax.
constexpr int kDeepWaves = 8, kDeepRows = 32 * kDeepWaves;
constexpr int kDeepSlots = 3;                             // tiles of K, and of V, in LDS: K of tiles T, T + 1 and V of T - 1, T are read while K of T + 2 and V of T + 1 are written
template <CacheFmt F>
__global__ __launch_bounds__(64 * kDeepWaves, 2) void chunk_deep_kernel(const uint16_t* __restrict__ q, const typename RowType<uint16_t, F>::type* __restrict__ K,
                                                            const typename RowType<uint16_t, F>::type* __restrict__ V, uint16_t* __restrict__ O,
                                                            float* __restrict__ part_acc, float2* __restrict__ part_ml, CacheView cv, ChunkView ch,
                                                            int batch, int Hkv, int G, int tiles_each, int splits, long long q_stride,
                                                            long long o_stride, float scale_log2e) {
  constexpr int D = kHeadDim, NT = 64 * kDeepWaves, TR = kDeepRows;
  constexpr bool BYTES = F != kPlain;
  using RT = typename RowType<uint16_t, F>::type;
  constexpr int PER_ROW = BYTES ? 8 : 16;                 // 16-byte pieces of a stored row
  constexpr int NL = kWideTok * PER_ROW / NT;             // pieces of K, and of V, a thread
  constexpr int WROWS = 64 / PER_ROW;                     // rows of a wave's load
  extern __shared__ __align__(16) unsigned char smem[];   // [slot] K tiles, [slot] V tiles, then scales [slot][k 64], [slot][v 64]
  unsigned char* const smk = smem;
  unsigned char* const smv = smem + kDeepSlots * kTileBytes;
  float* const ssk = reinterpret_cast<float*>(smem + 2 * kDeepSlots * kTileBytes);
  float* const ssv = ssk + kDeepSlots * kWideTok;

  unsigned id = blockIdx.x;
  const int h = (int)(id % (unsigned)Hkv);
  id /= (unsigned)Hkv;
  const int split = (int)(id % (unsigned)splits);
  id /= (unsigned)splits;
  int b, qt;
  if (!find_chunk_tile<TR>(ch, batch, G, tiles_each, id, b, qt)) return;
  const SeqChunk sc = seq_chunk(ch, b);
  const int m = sc.n_new * G, m_tiles = (m + TR - 1) / TR;
  if (qt >= m_tiles) return;
  qt = m_tiles - 1 - qt;                                   // the longest first
  const int rows = min(TR, m - qt * TR);
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int pos0 = sc.n_ctx - sc.n_new;
  const auto token_of = [&](int r) FASA_INLINE { return (qt * TR + r) / G; };
  const int seen = pos0 + token_of(rows - 1) + 1;          // tokens that the tile's last row sees
  const int share = ((seen + splits - 1) / splits + kWideTok - 1) / kWideTok * kWideTok;
  const int s0 = min(split * share, seen), s1 = min(seen, s0 + share);
  const int n_tiles = (s1 - s0 + kWideTok - 1) / kWideTok;

  // this lane's query
  const int my = min(32 * wave + col, rows - 1), my_tok = token_of(my);
  const int my_end = min(s1, pos0 + my_tok + 1);
  const int wave_all = min(s1, pos0 + token_of(min(32 * wave, rows - 1)) + 1);         // tokens that all of the wave's queries see
  bf16x8_t qb[8];
  {
    const uint16_t* p = q + (long long)(sc.row + my_tok) * q_stride + (long long)(h * G + (qt * TR + my) - my_tok * G) * D + 8 * half;
#pragma unroll
    for (int i = 0; i < 8; ++i) qb[i] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const uint4*>(p + 16 * i));
  }
  f32x16_t oc[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) oc[i] = f32x16_t{};
  float m_run = kNegBig, l_run = 0.f;

  // ---- loader ----
  // A wave's load is WROWS rows, which lie in one block (pages of that many tokens or more): where they begin is the wave's, in scalar registers, and the same for
  // K and V; what is a lane's is its row and piece in there, clamped to the last row that there is.  Lane l looks up the block of a tile's token l.
  const bool paged = cv.pm.table != nullptr;
  const int32_t* const table = paged ? cv.pm.table + (size_t)b * cv.pm.max_blocks : reinterpret_cast<const int32_t*>(q);
  const int shift = paged ? cv.pm.shift : 31, in_block = paged ? (1 << cv.pm.shift) - 1 : 0x7fffffff;
  const int blk_max = paged ? cv.pm.n_pool - 1 : 0;
  const uint32_t blk_bytes = paged ? (uint32_t)(cv.sb * (int)sizeof(RT)) : 0, row_bytes = (uint32_t)(cv.sn * (int)sizeof(RT));
  const long long seq = (paged ? 0 : b * cv.sb) + h * cv.sh;
  const char* const Kh = reinterpret_cast<const char*>(K + seq);
  const char* const Vh = reinterpret_cast<const char*>(V + seq);
  const uint32_t my_row = (uint32_t)(lane / PER_ROW) * row_bytes, my_piece = (uint32_t)(lane % PER_ROW) * 16;
  typedef uint32_t u32xl __attribute__((ext_vector_type(4 * NL)));
  struct Rows { uint64_t at[NL]; uint32_t last[NL]; int blk; };     // of a tile: where this wave's loads begin, bytes to the last row of them; lane l: block of token l
  auto look_up = [&](int j0) FASA_INLINE { return table[min(j0 + lane, s1 - 1) >> shift]; };
  auto rows_of = [&](int j0, int blks) FASA_INLINE {
    Rows r;
    r.blk = min(max(blks, 0), blk_max);
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int g = min(j0 + WROWS * (wave + kDeepWaves * i), (s1 - 1) & ~(WROWS - 1));
      const uint32_t blk = (uint32_t)__builtin_amdgcn_readlane(r.blk, max(g - j0, 0));
      r.at[i] = (uint64_t)blk * blk_bytes + (uint64_t)(uint32_t)(g & in_block) * row_bytes;
      r.last[i] = (uint32_t)min(s1 - 1 - g, WROWS - 1) * row_bytes;
    }
    return r;
  };
  auto load_rows = [&](const char* H, const Rows& r) FASA_INLINE {
    u32xl v;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const uint4 x = *reinterpret_cast<const uint4*>(H + r.at[i] + (min(my_row, r.last[i]) + my_piece));
      v[4 * i] = x.x; v[4 * i + 1] = x.y; v[4 * i + 2] = x.z; v[4 * i + 3] = x.w;
    }
    return v;
  };
  const float* const ks_h = BYTES ? cv.ks + (paged ? 0 : b * cv.ssb) + h * cv.ssh : nullptr;
  const float* const vs_h = BYTES ? cv.vs + (paged ? 0 : b * cv.ssb) + h * cv.ssh : nullptr;
  auto load_scale = [&](const float* s, int j0, const Rows& r) FASA_INLINE {
    return s[r.blk * (paged ? cv.ssb : 0) + (min(j0 + lane, s1 - 1) & in_block)];
  };
  auto store_rows = [&](unsigned char* to, u32xl r, auto swz) FASA_INLINE {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int row = WROWS * (wave + kDeepWaves * i) + lane / PER_ROW, c = lane % PER_ROW;
      if constexpr (BYTES) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint2 lo = bytes_to_bf16<F>(r[4 * i + 2 * j]), hi = bytes_to_bf16<F>(r[4 * i + 2 * j + 1]);
          *reinterpret_cast<uint4*>(to + row * 256 + (((2 * c + j) ^ swz(row)) << 4)) = make_uint4(lo.x, lo.y, hi.x, hi.y);
        }
      } else {
        *reinterpret_cast<uint4*>(to + row * 256 + ((c ^ swz(row)) << 4)) = make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
      }
    }
  };

  // ---- products ----
  typedef __attribute__((address_space(3))) const unsigned char* lds_ptr;
  lds_ptr k_at[8], v_at[4];                                // places of this lane's operands in slot 0, of its first 32 (16) tokens
#pragma unroll
  for (int s = 0; s < 8; ++s) k_at[s] = (lds_ptr)smk + col * 256 + (((2 * s + half) ^ swz_k(col)) << 4);
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    const int r = 4 * half + ((lane & 15) >> 2), c = 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    v_at[d] = (lds_ptr)smv + r * 256 + ((c ^ swz_v(r)) << 4) + 8 * (lane & 1);
  }
  struct Weights { uint32_t w[8]; };
  // at: where the 32 tokens begin, in bytes from slot 0
  auto logits = [&](int at, f32x16_t& sv) FASA_INLINE {
#pragma unroll
    for (int s = 0; s < 8; ++s)
      sv = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, *(__attribute__((address_space(3))) const u32x4_t*)(k_at[s] + at)), qb[s], s == 0 ? f32x16_t{} : sv, 0, 0, 0);
  };
  auto output = [&](int at, const Weights& p) FASA_INLINE {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const lds_ptr from = v_at[d] + (at + s * 16 * 256);
        const uint2 lo = lds_read_tr(from), hi = lds_read_tr(from + 8 * 256);            // (rows r and r + 8 have the same swizzle)
        oc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, make_uint4(lo.x, lo.y, hi.x, hi.y)),
                                                        __builtin_bit_cast(bf16x8_t, make_uint4(p.w[4 * s], p.w[4 * s + 1], p.w[4 * s + 2], p.w[4 * s + 3])), oc[d], 0, 0, 0);
      }
  };
  auto by_scale = [&](f32x16_t& sv, const float* f) FASA_INLINE {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float4 x = *reinterpret_cast<const float4*>(f + 8 * g + 4 * half);
      sv[4 * g] *= x.x; sv[4 * g + 1] *= x.y; sv[4 * g + 2] *= x.z; sv[4 * g + 3] *= x.w;
    }
  };
  // Weights of logits sv (tokens n0 .. n0 + 31); by: the factor by which the running sums go down.
  auto softmax = [&](f32x16_t& sv, Weights& p, float& by, int n0, const float* ks, const float* vs) FASA_INLINE {
    if constexpr (BYTES) by_scale(sv, ks);
    if (n0 + 32 > wave_all) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sv[i] = n0 + 8 * (i / 4) + 4 * half + i % 4 < my_end ? sv[i] : kNegBig;
    }
    float mx = xor32_max(largest(sv));
    if constexpr (!BYTES) mx *= scale_log2e;
    const float m_new = fmaxf(m_run, mx);
    by = __builtin_amdgcn_exp2f(m_run - m_new);
    m_run = m_new;
#pragma unroll
    for (int i = 0; i < 16; ++i) sv[i] = __builtin_amdgcn_exp2f(BYTES ? sv[i] - m_new : __builtin_fmaf(sv[i], scale_log2e, -m_new));
    l_run *= by;
    if constexpr (BYTES) {
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 16; ++i) sum[i & 1] += sv[i];
      l_run += sum[0] + sum[1];
      by_scale(sv, vs);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) p.w[i] = pack_bf16(sv[2 * i], sv[2 * i + 1]);
    if constexpr (!BYTES) {                                // the sum of the weights as the product has them: two at a time
      const bf16x2_t ones = {(__bf16)1.0f, (__bf16)1.0f};
      float other = 0.f;
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        l_run = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, p.w[i]), ones, l_run, false);
        other = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, p.w[i + 1]), ones, other, false);
      }
      l_run += other;
    }
  };
  // step: logits of the next 32 tokens -> nxt, output of the ones before (pp), weights of these (cur -> pc)
  auto step = [&](f32x16_t& cur, f32x16_t& nxt, const Weights& pp, Weights& pc, int k_next, int v_last, int n0, const float* ks, const float* vs) FASA_INLINE {
    float by;
    logits(k_next, nxt);
    output(v_last, pp);
    softmax(cur, pc, by, n0, ks, vs);
    if (__ballot(by != 1.f) != 0ull) {
#pragma unroll
      for (int d = 0; d < 4; ++d) oc[d] *= by;
    }
  };

  if (n_tiles > 0) {
    f32x16_t sa, sb;
    Weights pa = {}, pb;
    const auto of_k = [](int r) { return swz_k(r); };
    const auto of_v = [](int r) { return swz_v(r); };
    float rsk = 0.f, rsv = 0.f;
    // K of tiles 0 and 1, V of tile 0; zeros for V of the tile before the first, which has no weights, but what 0 is multiplied by has to be a number
    Rows ra = rows_of(s0, look_up(s0)), rb = rows_of(s0 + kWideTok, look_up(s0 + kWideTok)), rc = rows_of(s0 + 2 * kWideTok, look_up(s0 + 2 * kWideTok));
    store_rows(smk, load_rows(Kh, ra), of_k);
    store_rows(smv, load_rows(Vh, ra), of_v);
    store_rows(smk + kTileBytes, load_rows(Kh, rb), of_k);
    if constexpr (BYTES) {
      ssk[lane] = load_scale(ks_h, s0, ra) * scale_log2e;                               // (all waves, the same)
      ssv[lane] = load_scale(vs_h, s0, ra);
      ssk[kWideTok + lane] = load_scale(ks_h, s0 + kWideTok, rb) * scale_log2e;
      rsk = load_scale(ks_h, s0 + 2 * kWideTok, rc);
    }
    for (int x = t; x < kTileBytes / 16; x += NT) reinterpret_cast<uint4*>(smv + (kDeepSlots - 1) * kTileBytes)[x] = make_uint4(0, 0, 0, 0);
    u32xl raw = load_rows(Kh, rc);
    int blks = look_up(s0 + 3 * kWideTok);
    __syncthreads();
    logits(0, sa);
    // Tile T, in slot c0 (c1, c2: slots of T + 1 and T + 2, the latter T - 1's too).  Before it: raw is K of tile T + 2, r1 and r2 are the rows of T + 1 and T + 2,
    // blks the blocks of T + 3, whose rows r0 becomes.
    auto tile = [&](int T, int c0, int c1, int c2, Rows& r0, const Rows& r1) FASA_INLINE {
      constexpr int B = kTileBytes;
      const int j0 = s0 + T * kWideTok;
      store_rows(smk + c2 * B, raw, of_k);
      raw = load_rows(Vh, r1);
      if constexpr (BYTES) {
        ssk[c2 * kWideTok + lane] = rsk * scale_log2e;
        rsv = load_scale(vs_h, j0 + kWideTok, r1);
      }
      step(sa, sb, pa, pb, c0 * B + 32 * 256, c2 * B + 32 * 256, j0, ssk + c0 * kWideTok, ssv + c0 * kWideTok);
      store_rows(smv + c1 * B, raw, of_v);
      r0 = rows_of(j0 + 3 * kWideTok, blks);
      raw = load_rows(Kh, r0);
      if constexpr (BYTES) {
        ssv[c1 * kWideTok + lane] = rsv;
        rsk = load_scale(ks_h, j0 + 3 * kWideTok, r0);
      }
      blks = look_up(j0 + 4 * kWideTok);
      step(sb, sa, pb, pa, c1 * B, c0 * B, j0 + 32, ssk + c0 * kWideTok + 32, ssv + c0 * kWideTok + 32);
      __syncthreads();
    };
    int c0 = 0, c1 = 1, c2 = 2;
    for (int T = 0; T < n_tiles; ++T) {
      tile(T, c0, c1, c2, ra, rb);
      const Rows r = ra; ra = rb; rb = rc; rc = r;
      const int c = c0; c0 = c1; c1 = c2; c2 = c;
    }
    output(c2 * kTileBytes + 32 * 256, pa);
  }
  l_run = xor32_sum(l_run);
  if (32 * wave + col >= rows) return;
  if (splits == 1) {
    const float by = 1.0f / l_run;
    uint16_t* o = O + (long long)(sc.row + my_tok) * o_stride + (long long)(h * G + (qt * TR + my) - my_tok * G) * D + 4 * half;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<uint2*>(o + 32 * d + 8 * g) = make_uint2(pack_bf16(oc[d][4 * g] * by, oc[d][4 * g + 1] * by), pack_bf16(oc[d][4 * g + 2] * by, oc[d][4 * g + 3] * by));
    return;
  }
  const size_t at = (((size_t)(b * Hkv + h) * tiles_each + qt) * splits + split) * TR + my;
  float* to = part_acc + at * D + 4 * half;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<float4*>(to + 32 * d + 8 * g) = make_float4(oc[d][4 * g], oc[d][4 * g + 1], oc[d][4 * g + 2], oc[d][4 * g + 3]);
  if (half == 0) part_ml[at] = make_float2(m_run, l_run);
}

// Joins the splits of a tile's rows: 32 lanes a row, four dims each.
template <int TR>
__global__ __launch_bounds__(256) void chunk_merge_kernel(const float* __restrict__ part_acc, const float2* __restrict__ part_ml, uint16_t* __restrict__ O,
                                                          ChunkView ch, int batch, int Hkv, int G, int tiles_each, int splits, long long o_stride) {
  const int h = blockIdx.y;
  unsigned id = blockIdx.x / (TR / 8);
  const int r = (int)(blockIdx.x % (TR / 8)) * 8 + (int)(threadIdx.x >> 5), c = threadIdx.x & 31;
  int b, qt;
  if (!find_chunk_tile<TR>(ch, batch, G, tiles_each, id, b, qt)) return;
  const SeqChunk sc = seq_chunk(ch, b);
  if (qt * (long long)TR + r >= (long long)sc.n_new * G) return;
  const size_t at = ((size_t)(b * Hkv + h) * tiles_each + qt) * splits * TR + r;
  float mx = kNegBig, l = 0.f;
  for (int s = 0; s < splits; ++s) mx = fmaxf(mx, part_ml[at + (size_t)s * TR].x);
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int s = 0; s < splits; ++s) {
    const float2 ml = part_ml[at + (size_t)s * TR];
    const float by = exp2f(ml.x - mx);
    const float4 x = *reinterpret_cast<const float4*>(part_acc + (at + (size_t)s * TR) * kHeadDim + 4 * c);
    l = fmaf(ml.y, by, l);
    a.x = fmaf(x.x, by, a.x); a.y = fmaf(x.y, by, a.y); a.z = fmaf(x.z, by, a.z); a.w = fmaf(x.w, by, a.w);
  }
  const int row = qt * TR + r, tok = row / G;
  const float by = 1.0f / l;
  *reinterpret_cast<uint2*>(O + (long long)(sc.row + tok) * o_stride + (long long)(h * G + row - tok * G) * kHeadDim + 4 * c) =
      make_uint2(pack_bf16(a.x * by, a.y * by), pack_bf16(a.z * by, a.w * by));
}

template <CacheFmt F, int NW>
static hipError_t wide_t(const fasa_shape& s, const ChunkPlan& p, const ChunkArgs& a, hipStream_t st) {
  using RT = typename RowType<uint16_t, F>::type;
  const int hkv = s.n_kv_heads, G = s.n_q_heads / hkv;
  hipError_t e = launch_lds("fasa_chunk_attend", chunk_wide_kernel<F, NW>, dim3((unsigned)((long long)p.tiles * hkv * p.splits)), dim3(64 * NW),
                            4 * kTileBytes + (F == kPlain ? 0 : 4 * kWideTok * 4), st, (const uint16_t*)a.q, (const RT*)a.cv.K, (const RT*)a.cv.V,
                            (uint16_t*)a.O, a.part_acc, (float2*)a.part_ml, a.cv, a.ch, s.batch, hkv, G, p.per_seq, p.splits, a.q_stride, a.o_stride,
                            1.4426950408889634f / sqrtf((float)s.head_dim));
  if (e != hipSuccess || p.splits == 1) return e;
  return launch("fasa_chunk_merge", chunk_merge_kernel<32 * NW>, dim3((unsigned)p.tiles * 4 * NW, hkv), dim3(256), st, (const float*)a.part_acc,
                (const float2*)a.part_ml, (uint16_t*)a.O, a.ch, s.batch, hkv, G, p.per_seq, p.splits, a.o_stride);
}

template <CacheFmt F> static hipError_t deep_t(const fasa_shape& s, const ChunkPlan& p, const ChunkArgs& a, hipStream_t st) {
  using RT = typename RowType<uint16_t, F>::type;
  const int hkv = s.n_kv_heads, G = s.n_q_heads / hkv;
  const hipError_t e = launch_lds("fasa_chunk_attend", chunk_deep_kernel<F>, dim3((unsigned)((long long)p.tiles * hkv * p.splits)), dim3(64 * kDeepWaves),
                                  2 * kDeepSlots * (kTileBytes + (F == kPlain ? 0 : kWideTok * 4)), st, (const uint16_t*)a.q, (const RT*)a.cv.K, (const RT*)a.cv.V,
                                  (uint16_t*)a.O, a.part_acc, (float2*)a.part_ml, a.cv, a.ch, s.batch, hkv, G, p.per_seq, p.splits, a.q_stride, a.o_stride,
                                  1.4426950408889634f / sqrtf((float)s.head_dim));
  if (e != hipSuccess || p.splits == 1) return e;
  return launch("fasa_chunk_merge", chunk_merge_kernel<kDeepRows>, dim3((unsigned)p.tiles * (kDeepRows / 8), hkv), dim3(256), st, (const float*)a.part_acc,
                (const float2*)a.part_ml, (uint16_t*)a.O, a.ch, s.batch, hkv, G, p.per_seq, p.splits, a.o_stride);
}

hipError_t launch_chunk_wide(const fasa_shape& s, const ChunkPlan& p, const ChunkArgs& a, hipStream_t st) {
  if (p.tile_rows == 128)
    return a.fmt == kPlain ? wide_t<kPlain, 4>(s, p, a, st) : a.fmt == kInt8 ? wide_t<kInt8, 4>(s, p, a, st) : wide_t<kE4m3, 4>(s, p, a, st);
  // pages of fewer tokens than a wave's load has rows, or rows far apart: tokens are looked up one by one
  const bool apart = (a.cv.pm.table != nullptr && (1 << a.cv.pm.shift) < (a.fmt == kPlain ? 4 : 8)) ||
                     a.cv.sn >= (1ll << 27) || a.cv.sb >= (1ll << 31);
  if (apart) return a.fmt == kPlain ? wide_t<kPlain, 8>(s, p, a, st) : a.fmt == kInt8 ? wide_t<kInt8, 8>(s, p, a, st) : wide_t<kE4m3, 8>(s, p, a, st);
  return a.fmt == kPlain ? deep_t<kPlain>(s, p, a, st) : a.fmt == kInt8 ? deep_t<kInt8>(s, p, a, st) : deep_t<kE4m3>(s, p, a, st);
}

}  // namespace fasa
