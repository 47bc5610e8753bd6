// Attention of a chunk of bf16 query rows over a bf16 or 8-bit cache: many query rows of a KV head (new token, head of the group) against the same K and V,
// both products on the matrix cores, tiles of 64 tokens of K and V shared by the workgroup through LDS, a wave for every 32 query rows.
//
//   S^T = K Q^T   (tokens x queries; 32 x 32 x 16 MFMAs, K from LDS, Q in registers): the result's column, a lane's own, is one query, its 16
//                 registers are tokens 8 (i / 4) + 4 (lane / 32) + i % 4.  Maximum, exponentials and sum of a query are the lane's own but for one exchange
//                 with the lane 32 on.
//   O^T += V^T P^T (dims x queries): what the lane has of P^T, as bf16, is the second operand as it stands: its k-slots 0-3, 4-7 are the tokens of registers
//                 8 s .. 8 s + 7 of k-step s.  V^T with tokens in that order comes out of LDS by transposing reads (ds_read_b64_tr_b16: 16 lanes get
//                 one column each of four rows).  A new maximum rescales a lane's own accumulators.
// LDS rows are 256 bytes of 16-byte chunks; chunk c of token t is stored at c ^ (t mod 16) (K) or c ^ 4 (t mod 4) ^ (t / 4 mod 2) (V), so that the lanes that
// are served at once fall on all banks: 16 lanes of a read of K, 32 of a transposing one (four rows, 64 bytes each).  8-bit rows become bf16 (exactly) on their way into
// LDS, once for all waves; their scales multiply logits and weights in float32.
#include "chunk_common.h"

namespace fasa {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) const unsigned char* lds_ptr;

constexpr int kWideTok = 64;                              // tokens of a tile
constexpr int kTileBytes = kWideTok * kHeadDim * 2;       // of K or V in LDS

__device__ __forceinline__ int swz_k(int t) { return t & 15; }
__device__ __forceinline__ int swz_v(int t) { return (4 * (t & 3)) ^ ((t >> 2) & 1); }

// Four bf16 of one column of V for each of 16 lanes, out of four rows of LDS
__device__ __forceinline__ uint2 lds_read_tr(lds_ptr p) {
  const s16x4_t r = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)p);
  return __builtin_bit_cast(uint2, r);
}

// What a workgroup works on: query rows [qt TR, qt TR + rows) of sequence b and KV head h, tokens [s0, s1).  part: where its partial result goes.
constexpr int kWideLeast = kShortForm.least;
static_assert(kShortForm.least == kDeepForm.least);
template <int TR> struct WideJob {
  int b, h, qt, splits, rows, row0, pos0, s0, s1, n_tiles;
  size_t part;
  __device__ __forceinline__ int token_of(int r, int G) const { return (qt * TR + r) / G; }      // new token of the tile's row r
  // False: nothing to do.  Workgroups: heads fastest (those of a sequence read the same blocks, and a head's lie on one XCD where there are eight).
  __device__ __forceinline__ bool find(const ChunkView& ch, int batch, int Hkv, int G, int tiles_each, int whole, int all_splits, int units, int all_parts) {
    h = (int)(blockIdx.x % (unsigned)Hkv);
    ChunkUnit u;
    if (!find_chunk_unit<TR>(ch, batch, G, tiles_each, whole, all_splits, units, kWideLeast, blockIdx.x / (unsigned)Hkv, u)) return false;
    b = u.b;
    splits = u.splits;
    const int m = u.seq.n_new * G;
    qt = (m + TR - 1) / TR - 1 - u.tile;                   // the longest first
    rows = min(TR, m - qt * TR);
    row0 = u.seq.row;
    pos0 = u.seq.n_ctx - u.seq.n_new;
    const int seen = pos0 + token_of(rows - 1, G) + 1;     // tokens that the tile's last row sees
    const int share = u.share ? u.share : ((seen + splits - 1) / splits + kWideTok - 1) / kWideTok * kWideTok;
    s0 = (int)min((long long)u.split * share, (long long)seen);
    s1 = min(seen, s0 + share);
    n_tiles = (s1 - s0 + kWideTok - 1) / kWideTok;
    part = (size_t)h * all_parts + u.first + u.split;
    return true;
  }
};

// Rows of the cache, 16 bytes a lane and load, into registers and on to LDS.
// A wave's load is WROWS rows, which lie in one block (pages of that many tokens or more): where they begin is the wave's, in scalar registers, and the same for K
// and V; what is a lane's is its row and piece in there, clamped to the last row that there is.  Lane l looks up the block of a tile's token l, a tile or more
// ahead of the rows: a lookup between two loads would wait for the first one's.  APART: smaller pages (or strides that 32 bits do not hold): every lane
// finds its own rows.
template <CacheFmt F, int NW, bool APART> struct WideLoader {
  static constexpr bool BYTES = F != kPlain;
  using RT = typename RowType<uint16_t, F>::type;
  static constexpr int PER_ROW = BYTES ? 8 : 16;           // 16-byte pieces of a stored row
  static constexpr int NL = kWideTok * PER_ROW / (64 * NW);     // pieces of K, and of V, a thread
  static constexpr int WROWS = 64 / PER_ROW;               // rows of a wave's load
  typedef uint32_t u32xl __attribute__((ext_vector_type(4 * NL)));
  struct Rows {                                            // of a tile: where this wave's loads begin (APART: this lane's), bytes from there to the last row
    uint64_t at[NL];
    uint32_t last[NL];
    int blk;                                               // lane l: block of token l
  };
  const int32_t* table;
  const char *Kh, *Vh;
  const float *ks, *vs;
  long long ssb, sb, sn;
  uint32_t blk_bytes, row_bytes, my_row, my_piece;
  int shift, in_block, blk_max, s1, wave, lane;

  __device__ __forceinline__ WideLoader(const CacheView& cv, const void* K, const void* V, const void* any, int b, int h, int s1_, int wave_, int lane_) {
    const bool paged = cv.pm.table != nullptr;
    table = paged ? cv.pm.table + (size_t)b * cv.pm.max_blocks : reinterpret_cast<const int32_t*>(any);     // (an entry is read in any case)
    shift = paged ? cv.pm.shift : 31;
    in_block = paged ? (1 << cv.pm.shift) - 1 : 0x7fffffff;
    blk_max = paged ? cv.pm.n_pool - 1 : 0;
    const long long seq = (paged ? 0 : b * cv.sb) + h * cv.sh;
    Kh = reinterpret_cast<const char*>((const RT*)K + seq);
    Vh = reinterpret_cast<const char*>((const RT*)V + seq);
    sb = paged ? cv.sb * (int)sizeof(RT) : 0;
    sn = cv.sn * (int)sizeof(RT);
    blk_bytes = (uint32_t)sb;
    row_bytes = (uint32_t)sn;
    if constexpr (BYTES) {
      ks = cv.ks + (paged ? 0 : b * cv.ssb) + h * cv.ssh;
      vs = cv.vs + (paged ? 0 : b * cv.ssb) + h * cv.ssh;
      ssb = paged ? cv.ssb : 0;
    }
    s1 = s1_;
    wave = wave_;
    lane = lane_;
    my_row = (uint32_t)(lane / PER_ROW) * row_bytes;
    my_piece = (uint32_t)(lane % PER_ROW) * 16;
  }
  // the table's entry for token j0 + lane (tokens behind the last one: the last one's)
  __device__ __forceinline__ int look_up(int j0) const { return table[min(j0 + lane, s1 - 1) >> shift]; }
  __device__ __forceinline__ Rows rows_of(int j0, int entry) const {
    Rows r;
    r.blk = min(max(entry, 0), blk_max);
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      if constexpr (APART) {
        const int n = min(j0 + WROWS * (wave + NW * i) + lane / PER_ROW, s1 - 1);
        const int blk = __shfl(r.blk, max(n - j0, 0));
        r.at[i] = (uint64_t)(blk * sb + (n & in_block) * sn);
        r.last[i] = 0;
      } else {
        const int g = min(j0 + WROWS * (wave + NW * i), (s1 - 1) & ~(WROWS - 1));
        const uint32_t blk = (uint32_t)__builtin_amdgcn_readlane(r.blk, max(g - j0, 0));
        r.at[i] = (uint64_t)blk * blk_bytes + (uint64_t)(uint32_t)(g & in_block) * row_bytes;
        r.last[i] = (uint32_t)min(s1 - 1 - g, WROWS - 1) * row_bytes;
      }
    }
    return r;
  }
  __device__ __forceinline__ u32xl load(const char* H, const Rows& r) const {
    u32xl v;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const uint4 x = *reinterpret_cast<const uint4*>(H + r.at[i] + ((APART ? 0 : min(my_row, r.last[i])) + my_piece));
      v[4 * i] = x.x; v[4 * i + 1] = x.y; v[4 * i + 2] = x.z; v[4 * i + 3] = x.w;
    }
    return v;
  }
  // of token j0 + lane
  __device__ __forceinline__ float load_scale(const float* s, int j0, const Rows& r) const { return s[r.blk * ssb + (min(j0 + lane, s1 - 1) & in_block)]; }
  template <class Swz> __device__ __forceinline__ void store(unsigned char* to, u32xl r, Swz swz) const {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int row = WROWS * (wave + NW * i) + lane / PER_ROW, c = lane % PER_ROW;
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
  }
  __device__ __forceinline__ void store_k(unsigned char* to, u32xl r) const { store(to, r, [](int t) { return swz_k(t); }); }
  __device__ __forceinline__ void store_v(unsigned char* to, u32xl r) const { store(to, r, [](int t) { return swz_v(t); }); }
};

// The 32 queries of a wave: products with tiles in LDS, softmax, result.
template <bool BYTES> struct WideQueries {
  struct Weights { uint32_t w[8]; };                       // of 32 tokens
  bf16x8_t qb[8];
  f32x16_t oc[4];
  float m_run, l_run;                                      // of this lane's query: what the weights are relative to (log2 domain), their sum over this lane's tokens
  uint32_t k_at[8], v_at[4];                               // places of this lane's operands in a tile, of its first 32 (16) tokens
  int my, my_end, all, half;                               // row in the tile, tokens that it sees, tokens that all rows of the wave see
  long long at;                                            // of the row, in elements of q

  template <int TR>
  __device__ __forceinline__ WideQueries(const WideJob<TR>& job, const uint16_t* q, long long q_stride, int G, int wave, int lane) {
    constexpr int D = kHeadDim;
    const int col = lane & 31;
    half = lane >> 5;
    my = min(32 * wave + col, job.rows - 1);
    const int tok = job.token_of(my, G);
    my_end = min(job.s1, job.pos0 + tok + 1);
    all = min(job.s1, job.pos0 + job.token_of(min(32 * wave, job.rows - 1), G) + 1);
    const uint16_t* p = q + (long long)(job.row0 + tok) * q_stride + (long long)(job.h * G + (job.qt * TR + my) - tok * G) * D + 8 * half;
#pragma unroll
    for (int i = 0; i < 8; ++i) qb[i] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const uint4*>(p + 16 * i));
#pragma unroll
    for (int i = 0; i < 4; ++i) oc[i] = f32x16_t{};
    m_run = kNegBig;
    l_run = 0.f;
#pragma unroll
    for (int s = 0; s < 8; ++s) k_at[s] = col * 256 + (((2 * s + half) ^ swz_k(col)) << 4);
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const int r = 4 * half + ((lane & 15) >> 2), c = 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
      v_at[d] = r * 256 + ((c ^ swz_v(r)) << 4) + 8 * (lane & 1);
    }
  }
  // logits of 32 tokens of K at kt
  __device__ __forceinline__ f32x16_t logits(lds_ptr kt) const {
    f32x16_t sv = {};
#pragma unroll
    for (int s = 0; s < 8; ++s)
      sv = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, *(__attribute__((address_space(3))) const u32x4_t*)(kt + k_at[s])), qb[s], sv, 0, 0, 0);
    return sv;
  }
  // the weighted 32 tokens of V at vt
  __device__ __forceinline__ void output(lds_ptr vt, const Weights& p) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const lds_ptr from = vt + v_at[d] + s * 16 * 256;
        const uint2 lo = lds_read_tr(from), hi = lds_read_tr(from + 8 * 256);            // (rows r and r + 8 have the same swizzle)
        oc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, make_uint4(lo.x, lo.y, hi.x, hi.y)),
                                                        __builtin_bit_cast(bf16x8_t, make_uint4(p.w[4 * s], p.w[4 * s + 1], p.w[4 * s + 2], p.w[4 * s + 3])), oc[d], 0, 0, 0);
      }
  }
  __device__ __forceinline__ void by_scale(f32x16_t& sv, const float* f) const {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float4 x = *reinterpret_cast<const float4*>(f + 8 * g + 4 * half);
      sv[4 * g] *= x.x; sv[4 * g + 1] *= x.y; sv[4 * g + 2] *= x.z; sv[4 * g + 3] *= x.w;
    }
  }
  // Weights of logits sv (tokens n0 .. n0 + 31; 8-bit: ks, vs their scales, ks with the softmax's).  What they are relative to follows the running maximum only
  // where that has grown by more than 2^8 (weights of up to 256 are as exact as those below 1): with 32 queries a wave, one of them has a new maximum in every
  // step of the first 32, and in 32 / u of the steps u behind, and 64 accumulators would be multiplied there.
  __device__ __forceinline__ void softmax(f32x16_t& sv, Weights& p, int n0, const float* ks, const float* vs, float scale_log2e) {
    if constexpr (BYTES) by_scale(sv, ks);
    if (n0 + 32 > all) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sv[i] = n0 + 8 * (i / 4) + 4 * half + i % 4 < my_end ? sv[i] : kNegBig;
    }
    float mx = __builtin_fmaxf(sv[0], sv[1]);
#pragma unroll
    for (int i = 2; i < 16; i += 2) mx = __builtin_fmaxf(mx, __builtin_fmaxf(sv[i], sv[i + 1]));
    mx = xor32_max(mx);
    if constexpr (!BYTES) mx *= scale_log2e;
    if (__ballot(mx > m_run + 8.f) != 0ull) {
      const float m_new = __builtin_fmaxf(m_run, mx), by = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= by;
#pragma unroll
      for (int d = 0; d < 4; ++d) oc[d] *= by;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) sv[i] = __builtin_amdgcn_exp2f(BYTES ? sv[i] - m_run : __builtin_fmaf(sv[i], scale_log2e, -m_run));
    if constexpr (BYTES) {
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 16; ++i) sum[i & 1] += sv[i];
      l_run += sum[0] + sum[1];
      by_scale(sv, vs);
      if (n0 + 32 > all) {                                 // (a scale may be a NaN)
#pragma unroll
        for (int i = 0; i < 16; ++i) sv[i] = n0 + 8 * (i / 4) + 4 * half + i % 4 < my_end ? sv[i] : 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) p.w[i] = pack_bf16(sv[2 * i], sv[2 * i + 1]);
    if constexpr (!BYTES) {                                // the sum of the weights as the product has them, two at a time
      const bf16x2_t ones = {(__bf16)1.0f, (__bf16)1.0f};
      float other = 0.f;
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        l_run = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, p.w[i]), ones, l_run, false);
        other = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, p.w[i + 1]), ones, other, false);
      }
      l_run += other;
    }
  }
  // To O, or where there are splits to their places.  row: of the tile, before it was clamped.
  template <int TR>
  __device__ __forceinline__ void finish(const WideJob<TR>& job, int row, uint16_t* O, long long o_stride, int G, float* part_acc, float2* part_ml) {
    constexpr int D = kHeadDim;
    const float l = xor32_sum(l_run);
    if (row >= job.rows) return;
    if (job.splits == 1) {
      const float by = 1.0f / l;
      const int tok = job.token_of(my, G);
      uint16_t* o = O + (long long)(job.row0 + tok) * o_stride + (long long)(job.h * G + (job.qt * TR + my) - tok * G) * D + 8 * half;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int g = 0; g < 4; g += 2) {                   // eight dims in a row to a lane: the lower half of the wave takes those of g, the upper of g + 1
          uint32_t w[4];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const auto x = __builtin_amdgcn_permlane32_swap(pack_bf16(oc[d][4 * g + 2 * i] * by, oc[d][4 * g + 2 * i + 1] * by),
                                                            pack_bf16(oc[d][4 * g + 4 + 2 * i] * by, oc[d][4 * g + 5 + 2 * i] * by), false, false);
            w[i] = x[0];
            w[2 + i] = x[1];
          }
          *reinterpret_cast<uint4*>(o + 32 * d + 8 * g) = make_uint4(w[0], w[1], w[2], w[3]);
        }
      return;
    }
    const size_t to = job.part * TR + my;
    float* pa = part_acc + to * D + 4 * half;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<float4*>(pa + 32 * d + 8 * g) = make_float4(oc[d][4 * g], oc[d][4 * g + 1], oc[d][4 * g + 2], oc[d][4 * g + 3]);
    if (half == 0) part_ml[to] = make_float2(m_run, l);
  }
};

// Few query rows, or few tokens: bound by reading the rows, which four waves share; two workgroups a compute unit have 64 KB of loads in flight.  (8 x 4 heads of 32905, 35 query
// rows each: 106 us, 5.1 TB/s.)
constexpr int kShortWaves = 4, kShortRows = kShortForm.rows;
static_assert(kShortRows == 32 * kShortWaves);
template <CacheFmt F, bool APART>
__global__ __launch_bounds__(64 * kShortWaves, 2) void chunk_short_kernel(const uint16_t* __restrict__ q, const void* __restrict__ K, const void* __restrict__ V,
                                                                         uint16_t* __restrict__ O, float* __restrict__ part_acc,
                                                                         float2* __restrict__ part_ml, CacheView cv, ChunkView ch, int batch, int Hkv,
                                                                         int G, int tiles_each, int whole, int splits, int units, int all_parts, long long q_stride, long long o_stride,
                                                                         float scale_log2e) {
  constexpr bool BYTES = F != kPlain;
  extern __shared__ __align__(16) unsigned char smem[];    // [2][K tile, V tile], then scales [2][k 64, v 64]
  float* const sm_scale = reinterpret_cast<float*>(smem + 4 * kTileBytes);
  WideJob<kShortRows> job;
  if (!job.find(ch, batch, Hkv, G, tiles_each, whole, splits, units, all_parts)) return;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  using Loader = WideLoader<F, kShortWaves, APART>;
  const Loader ld(cv, K, V, q, job.b, job.h, job.s1, wave, lane);
  WideQueries<BYTES> wq(job, q, q_stride, G, wave, lane);
  const bool mine = 32 * wave < job.rows;                  // waves without a row only load
  if (job.n_tiles > 0) {
    typename Loader::u32xl rk, rv;
    float sk = 0.f, sv = 0.f;
    int next = ld.look_up(job.s0);                         // of the tile to be loaded next
    auto load = [&](int j0) FASA_INLINE {
      const typename Loader::Rows r = ld.rows_of(j0, next);
      rk = ld.load(ld.Kh, r);
      rv = ld.load(ld.Vh, r);
      if constexpr (BYTES) {
        sk = ld.load_scale(ld.ks, j0, r);
        sv = ld.load_scale(ld.vs, j0, r);
      }
      next = ld.look_up(j0 + kWideTok);
    };
    auto store = [&](int buf) FASA_INLINE {
      ld.store_k(smem + buf * 2 * kTileBytes, rk);
      ld.store_v(smem + buf * 2 * kTileBytes + kTileBytes, rv);
      if constexpr (BYTES) {                               // (all waves, the same)
        sm_scale[buf * 2 * kWideTok + lane] = sk * scale_log2e;
        sm_scale[buf * 2 * kWideTok + kWideTok + lane] = sv;
      }
    };
    load(job.s0);
    store(0);
    load(job.s0 + kWideTok);
    __syncthreads();
    for (int T = 0; T < job.n_tiles; ++T) {
      const int j0 = job.s0 + T * kWideTok, buf = T & 1;
      store(buf ^ 1);                                      // tile T + 1; behind the last: the last row, for nobody
      load(j0 + 2 * kWideTok);
      if (mine) {
        const lds_ptr kt = (lds_ptr)smem + buf * 2 * kTileBytes;
        const float* ks = sm_scale + buf * 2 * kWideTok;
        f32x16_t s[2];
        typename WideQueries<BYTES>::Weights p;
        s[0] = wq.logits(kt);
        s[1] = wq.logits(kt + 32 * 256);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          wq.softmax(s[i], p, j0 + 32 * i, ks + 32 * i, ks + kWideTok + 32 * i, scale_log2e);
          wq.output(kt + kTileBytes + i * 32 * 256, p);
        }
      }
      __syncthreads();
    }
  }
  wq.finish(job, 32 * wave + (lane & 31), O, o_stride, G, part_acc, part_ml);
}

// Many: eight waves (256 rows a tile), two a SIMD.  In steps of 32 tokens: step u runs the logits of step u + 1 and the output of step u - 1 ahead of its own
// softmax, so that the matrix cores have sixteen products in a row to do that wait for nothing.  Bound by power: 2048 new tokens over 32768, 32 heads over 8, take 1080 us
// (0.99 PFLOP/s) at 1.9 GHz, and 860 at 2.4 on a cache of zeros; the products alone would take 52 % of the cycles.  (One wave of 64 queries a SIMD would read half as much
// from LDS, but a lone wave issues a vector instruction only every 6 - 10 cycles where two issue one every 3.  Exponentials between the products: 4 - 18 % slower.)
constexpr int kDeepWaves = 8, kDeepRows = kDeepForm.rows;
static_assert(kDeepRows == 32 * kDeepWaves);
constexpr int kDeepSlots = 3;                             // tiles of K, and of V, in LDS: K of tiles T, T + 1 and V of T - 1, T are read while K of T + 2 and V of T + 1 are written
template <CacheFmt F>
__global__ __launch_bounds__(64 * kDeepWaves, 2) void chunk_deep_kernel(const uint16_t* __restrict__ q, const void* __restrict__ K, const void* __restrict__ V,
                                                                       uint16_t* __restrict__ O, float* __restrict__ part_acc,
                                                                       float2* __restrict__ part_ml, CacheView cv, ChunkView ch, int batch, int Hkv,
                                                                       int G, int tiles_each, int whole, int splits, int units, int all_parts, long long q_stride, long long o_stride,
                                                                       float scale_log2e) {
  constexpr int NT = 64 * kDeepWaves, B = kTileBytes;
  constexpr bool BYTES = F != kPlain;
  extern __shared__ __align__(16) unsigned char smem[];   // [slot] K tiles, [slot] V tiles, then scales [slot][k 64], [slot][v 64]
  unsigned char* const smk = smem;
  unsigned char* const smv = smem + kDeepSlots * B;
  float* const ssk = reinterpret_cast<float*>(smem + 2 * kDeepSlots * B);
  float* const ssv = ssk + kDeepSlots * kWideTok;
  WideJob<kDeepRows> job;
  if (!job.find(ch, batch, Hkv, G, tiles_each, whole, splits, units, all_parts)) return;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  using Loader = WideLoader<F, kDeepWaves, false>;
  using Rows = typename Loader::Rows;
  const Loader ld(cv, K, V, q, job.b, job.h, job.s1, wave, lane);
  WideQueries<BYTES> wq(job, q, q_stride, G, wave, lane);
  using Weights = typename WideQueries<BYTES>::Weights;
  const int s0 = job.s0;
  // step: logits of the next 32 tokens -> nxt, output of the ones before (pp), weights of these (cur -> pc)
  auto step = [&](f32x16_t& cur, f32x16_t& nxt, const Weights& pp, Weights& pc, int k_next, int v_last, int n0, const float* ks, const float* vs) FASA_INLINE {
    nxt = wq.logits((lds_ptr)smk + k_next);
    wq.output((lds_ptr)smv + v_last, pp);
    wq.softmax(cur, pc, n0, ks, vs, scale_log2e);
  };
  if (job.n_tiles > 0) {
    f32x16_t sa, sb;
    Weights pa = {}, pb;
    float rsk = 0.f, rsv = 0.f;
    // K of tiles 0 and 1, V of tile 0; zeros for V of the tile before the first, which has no weights, but what 0 is multiplied by has to be a number
    const int e0 = ld.look_up(s0), e1 = ld.look_up(s0 + kWideTok), e2 = ld.look_up(s0 + 2 * kWideTok);
    Rows ra = ld.rows_of(s0, e0), rb = ld.rows_of(s0 + kWideTok, e1), rc = ld.rows_of(s0 + 2 * kWideTok, e2);
    const auto k0 = ld.load(ld.Kh, ra), v0 = ld.load(ld.Vh, ra), k1 = ld.load(ld.Kh, rb);
    auto raw = ld.load(ld.Kh, rc);
    int entry = ld.look_up(s0 + 3 * kWideTok);
    ld.store_k(smk, k0);
    ld.store_v(smv, v0);
    ld.store_k(smk + B, k1);
    if constexpr (BYTES) {
      ssk[lane] = ld.load_scale(ld.ks, s0, ra) * scale_log2e;                             // (all waves, the same)
      ssv[lane] = ld.load_scale(ld.vs, s0, ra);
      ssk[kWideTok + lane] = ld.load_scale(ld.ks, s0 + kWideTok, rb) * scale_log2e;
      rsk = ld.load_scale(ld.ks, s0 + 2 * kWideTok, rc);
    }
    for (int x = t; x < B / 16; x += NT) reinterpret_cast<uint4*>(smv + (kDeepSlots - 1) * B)[x] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    sa = wq.logits((lds_ptr)smk);
    // Tile T in slot c0; c1, c2: slots of T + 1 and T + 2, the latter T - 1's too.  Before it: raw is K of tile T + 2, rb and rc are the rows of T + 1 and T + 2,
    // entry of T + 3.  (Every wave runs all tiles, for the barriers.)
    int c0 = 0, c1 = 1, c2 = 2;
    for (int T = 0; T < job.n_tiles; ++T) {
      const int j0 = s0 + T * kWideTok;
      ld.store_k(smk + c2 * B, raw);
      raw = ld.load(ld.Vh, rb);
      if constexpr (BYTES) {
        ssk[c2 * kWideTok + lane] = rsk * scale_log2e;
        rsv = ld.load_scale(ld.vs, j0 + kWideTok, rb);
      }
      step(sa, sb, pa, pb, c0 * B + 32 * 256, c2 * B + 32 * 256, j0, ssk + c0 * kWideTok, ssv + c0 * kWideTok);
      ld.store_v(smv + c1 * B, raw);
      rb = rc;
      rc = ld.rows_of(j0 + 3 * kWideTok, entry);
      raw = ld.load(ld.Kh, rc);
      if constexpr (BYTES) {
        ssv[c1 * kWideTok + lane] = rsv;
        rsk = ld.load_scale(ld.ks, j0 + 3 * kWideTok, rc);
      }
      entry = ld.look_up(j0 + 4 * kWideTok);
      step(sb, sa, pb, pa, c1 * B, c0 * B, j0 + 32, ssk + c0 * kWideTok + 32, ssv + c0 * kWideTok + 32);
      __syncthreads();
      const int c = c0; c0 = c1; c1 = c2; c2 = c;
    }
    wq.output((lds_ptr)smv + c2 * B + 32 * 256, pa);
  }
  wq.finish(job, 32 * wave + (lane & 31), O, o_stride, G, part_acc, part_ml);
}

// Joins the parts of a tile's rows: as many workgroups for each part, which take as many rows as the others, 32 lanes a row, four dims each.
template <int TR> constexpr int kMergeWgs = TR / 64;
template <int TR>
__global__ __launch_bounds__(256) void chunk_merge_kernel(const float* __restrict__ part_acc, const float2* __restrict__ part_ml, uint16_t* __restrict__ O,
                                                          ChunkView ch, int batch, int Hkv, int G, int tiles_each, int whole, int all_splits, int units, int all_parts,
                                                          long long o_stride) {
  extern __shared__ float weights[];                                   // [8][parts]
  const int h = (int)(blockIdx.x % (unsigned)Hkv);
  ChunkUnit u;
  if (!find_chunk_unit<TR>(ch, batch, G, tiles_each, whole, all_splits, units, kWideLeast, (unsigned)whole + blockIdx.x / (unsigned)Hkv, u) || u.splits == 1) return;
  const int wgs = u.splits * kMergeWgs<TR>, wg = u.split * kMergeWgs<TR> + (int)blockIdx.y;
  const int n = u.splits, m = u.seq.n_new * G, qt = (m + TR - 1) / TR - 1 - u.tile, rows = min(TR, m - qt * TR);
  const int group = threadIdx.x >> 5, c = threadIdx.x & 31;
  const size_t part0 = ((size_t)h * all_parts + u.first) * TR;
  float* const w = weights + group * n;
  const int per = (rows + wgs - 1) / wgs, r1 = min(rows, (wg + 1) * per);
  for (int r = wg * per + group; r < r1; r += 8) {
    const float2* ml = part_ml + part0 + r;
    float mx = kNegBig, l = 0.f;
    for (int s = c; s < n; s += 32) mx = fmaxf(mx, ml[(size_t)s * TR].x);
    mx = xor16_max(row16_max(mx));                                     // (of 32 lanes)
    for (int s = c; s < n; s += 32) {
      const float2 x = ml[(size_t)s * TR];
      w[s] = exp2f(x.x - mx);
      l = fmaf(x.y, w[s], l);
    }
    l = xor16_sum(row16_sum(l));
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");             // (a wave's LDS operations complete in order)
    const float* pa = part_acc + (part0 + r) * kHeadDim + 4 * c;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = 0; s0 < n; s0 += 8) {
      float4 x[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = *reinterpret_cast<const float4*>(pa + (size_t)min(s0 + k, n - 1) * TR * kHeadDim);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float by = s0 + k < n ? w[min(s0 + k, n - 1)] : 0.f;
        a.x = fmaf(x[k].x, by, a.x); a.y = fmaf(x[k].y, by, a.y); a.z = fmaf(x[k].z, by, a.z); a.w = fmaf(x[k].w, by, a.w);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int row = qt * TR + r, tok = row / G;
    const float by = 1.0f / l;
    *reinterpret_cast<uint2*>(O + (long long)(u.seq.row + tok) * o_stride + (long long)(h * G + row - tok * G) * kHeadDim + 4 * c) =
        make_uint2(pack_bf16(a.x * by, a.y * by), pack_bf16(a.z * by, a.w * by));
  }
}

template <int TR, class Kernel>
static hipError_t wide_t(Kernel kernel, size_t lds, const fasa_shape& s, const ChunkPlan& p, const ChunkArgs& a, hipStream_t st) {
  const int hkv = s.n_kv_heads, G = s.n_q_heads / hkv, units = p.by_length ? p.units : 0;
  const hipError_t e = launch_lds("fasa_chunk_attend", kernel, dim3((unsigned)p.units * (unsigned)hkv), dim3(2 * TR), lds, st, (const uint16_t*)a.q,
                                  (const void*)a.cv.K, (const void*)a.cv.V, (uint16_t*)a.O, a.part_acc, (float2*)a.part_ml, a.cv, a.ch, s.batch, hkv, G,
                                  p.per_seq, p.whole, p.splits, units, p.parts, a.q_stride, a.o_stride, 1.4426950408889634f / sqrtf((float)s.head_dim));
  if (e != hipSuccess || p.parts == 0) return e;
  return launch_lds("fasa_chunk_merge", chunk_merge_kernel<TR>, dim3((unsigned)p.parts * (unsigned)hkv, kMergeWgs<TR>), dim3(256), (p.by_length ? p.units : p.splits) * 8 * sizeof(float),
                    st, (const float*)a.part_acc, (const float2*)a.part_ml, (uint16_t*)a.O, a.ch, s.batch, hkv, G, p.per_seq, p.whole, p.splits, units, p.parts, a.o_stride);
}
template <CacheFmt F> static hipError_t wide_f(const fasa_shape& s, const ChunkPlan& p, const ChunkArgs& a, hipStream_t st) {
  const size_t scales = F == kPlain ? 0 : kWideTok * 4;
  if (p.tile_rows == kDeepRows) return wide_t<kDeepRows>(chunk_deep_kernel<F>, 2 * kDeepSlots * (kTileBytes + scales), s, p, a, st);
  return wide_t<kShortRows>(p.apart ? chunk_short_kernel<F, true> : chunk_short_kernel<F, false>, 4 * (kTileBytes + scales), s, p, a, st);
}
hipError_t launch_chunk_wide(const fasa_shape& s, const ChunkPlan& p, const ChunkArgs& a, hipStream_t st) {
  return a.fmt == kPlain ? wide_f<kPlain>(s, p, a, st) : a.fmt == kInt8 ? wide_f<kInt8>(s, p, a, st) : wide_f<kE4m3>(s, p, a, st);
}

}  // namespace fasa
