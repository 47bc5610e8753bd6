// Rows of new tokens into the cache, in its format, and rows of the cache back in dtype.  Both move memory and little else:
// a row is 16 lanes' work, eight values (16 bytes of bf16) a lane, one row of K and one of V each.  (More rows a lane in flight, and fewer waves, are slower: 1 / 2 / 4 / 8
// rows, 32768 x 8 written as e4m3 46 / 48 / 54 / 62 us, read from int8 41 / 41 / 43.5 / 48.)
#include "chunk_common.h"

namespace fasa {

constexpr int kCacheTile = 16;                         // rows of K, and of V, of a workgroup of 256

// largest of the 16 lanes of a row
__device__ __forceinline__ uint32_t row16_max_u32(uint32_t x) {
  x = max(x, dpp_u32<0xB1, 0xF>(x));
  x = max(x, dpp_u32<0x4E, 0xF>(x));
  x = max(x, dpp_u32<0x141, 0xF>(x));
  return max(x, dpp_u32<0x140, 0xF>(x));
}

template <typename ET> struct Vals8 { uint4 w[sizeof(ET) / 2]; };      // eight values as they are stored
template <typename ET> __device__ __forceinline__ Vals8<ET> load_vals(const ET* p) {
  Vals8<ET> v;
#pragma unroll
  for (int i = 0; i < (int)sizeof(ET) / 2; ++i) v.w[i] = reinterpret_cast<const uint4*>(p)[i];
  return v;
}
template <typename ET> __device__ __forceinline__ void floats_of(const Vals8<ET>& v, float (&f)[8]) {
  if constexpr (sizeof(ET) == 2) {
    const uint32_t w[4] = {v.w[0].x, v.w[0].y, v.w[0].z, v.w[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = bf16_lo(w[i]); f[2 * i + 1] = bf16_hi(w[i]); }
  } else {
    const uint32_t w[8] = {v.w[0].x, v.w[0].y, v.w[0].z, v.w[0].w, v.w[1].x, v.w[1].y, v.w[1].z, v.w[1].w};
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[i]);
  }
}

// Four quotients' codes; the format's own rounding instruction (to the nearest, ties to even).
template <CacheFmt F> __device__ __forceinline__ uint32_t codes_of(const float* y) {
  if constexpr (F == kE4m3) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
  } else {
    const uint32_t a = (uint32_t)__float2int_rn(y[0]), b = (uint32_t)__float2int_rn(y[1]);
    const uint32_t c = (uint32_t)__float2int_rn(y[2]), d = (uint32_t)__float2int_rn(y[3]);
    const uint32_t ab = __builtin_amdgcn_perm(b, a, 0x0c0c0400u), cd = __builtin_amdgcn_perm(d, c, 0x0c0c0400u);
    return __builtin_amdgcn_perm(cd, ab, 0x05040100u);
  }
}

// A row's eight values of this lane -> codes, and the row's scale.  codes: the nearest to x / s, decided as if the quotient were exact.  A product with 1 / s is off
// by less than 2^-22 of itself, which matters only within that of a tie: where the codes of 2^-21 less and 2^-21 more differ (a lane in 10^3 for int8, in 10^4 for e4m3) the
// nearest is one of the two, and x is compared with the middle between them times s: the difference is rounded once and has its exact sign.  (Dividing every value
// takes ten instructions more each.)
template <typename ET, CacheFmt F> __device__ __forceinline__ uint2 quantise_row(const Vals8<ET>& v, float& scale) {
  constexpr float Q = F == kE4m3 ? 448.f : 127.f;
  float f[8];
  floats_of<ET>(v, f);
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(f[i]) & 0x7fffffffu);
  most = row16_max_u32(most);
  const bool finite = most < 0x7f800000u;
  float s = __uint_as_float(most) / Q;
  scale = finite ? s : __uint_as_float(0x7fc00000u);
  const bool some = finite && s > 0.f, tiny = s < 0x1p-60f;
  if (__ballot(some && tiny) != 0ull) {                    // (1 / s would be infinite, and differences below what float32 holds)
    const float up = tiny ? 0x1p80f : 1.f;
    s *= up;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] *= up;
  }
  const float inv = __builtin_amdgcn_rcpf(s);              // (within 2^-23)
  float lo[8], hi[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float y = f[i] * inv;
    lo[i] = y * (1.0f - 0x1p-21f);
    hi[i] = y * (1.0f + 0x1p-21f);
  }
  uint2 c = make_uint2(codes_of<F>(lo), codes_of<F>(lo + 4));
  const uint2 d = make_uint2(codes_of<F>(hi), codes_of<F>(hi + 4));
  const bool near = some && (c.x != d.x || c.y != d.y || tiny);
  if (__ballot(near) != 0ull) {
    if (near) {
      if (tiny) {                                          // (a scale of a few bits may leave quotients beyond Q)
#pragma unroll
        for (int i = 0; i < 8; ++i) { lo[i] = fminf(fmaxf(lo[i], -Q), Q); hi[i] = fminf(fmaxf(hi[i], -Q), Q); }
        c = make_uint2(codes_of<F>(lo), codes_of<F>(lo + 4));
      }
      const uint2 e = make_uint2(codes_of<F>(hi), codes_of<F>(hi + 4));
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x4_t vl = bytes_to_f32<F>(h ? c.y : c.x), vh = bytes_to_f32<F>(h ? e.y : e.x);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float mid = 0.5f * (vl[i] + vh[i]), over = fmaf(-mid, s, f[4 * h + i]);
          // (a tie: the middle itself, which goes to the even code)
          lo[4 * h + i] = over > 0.f ? fmaxf(vl[i], vh[i]) : over < 0.f ? fminf(vl[i], vh[i]) : mid;
        }
      }
      c = make_uint2(codes_of<F>(lo), codes_of<F>(lo + 4));
    }
  }
  return some ? c : make_uint2(0u, 0u);
}

// grid: tiles of 16 (token, head) items of a sequence, as they lie in k_new.  (16 tokens of a head, whose scales are then written 64 bytes at a time, are 1 us faster
// at 46, and 1 us slower for rows of dtype.)
template <typename ET, CacheFmt F>
__global__ __launch_bounds__(256) void cache_write_kernel(const ET* __restrict__ k_new, const ET* __restrict__ v_new, CacheView cv, ChunkView ch,
                                                          int batch, int Hkv, uint32_t m_hkv, int tiles_each, long long kv_stride) {
  using RT = typename RowType<ET, F>::type;
  int b, tile;
  if (!find_chunk_tile<kCacheTile>(ch, batch, Hkv, tiles_each, blockIdx.x, b, tile)) return;
  const SeqChunk sc = seq_chunk(ch, b);
  const int n_items = sc.n_new * Hkv;
  const int group = threadIdx.x >> 4, c = threadIdx.x & 15;
  if (tile * kCacheTile >= n_items) return;
  // (items behind the last are the last again: their lanes compute and do not store)
  const int item = min(tile * kCacheTile + group, n_items - 1);
  const int i = (int)fast_div((uint32_t)item, (uint32_t)Hkv, m_hkv), h = item - i * Hkv;
  const long long from = (long long)(sc.row + i) * kv_stride + h * kHeadDim + 8 * c;
  const Vals8<ET> k = load_vals<ET>(k_new + from), v = load_vals<ET>(v_new + from);
  int blk, off;
  cache_place(cv.pm, b, sc.n_ctx - sc.n_new + i, blk, off);
  const bool mine = tile * kCacheTile + group < n_items;
  const long long at = blk * cv.sb + h * cv.sh + off * cv.sn + 8 * c;
  if constexpr (F == kPlain) {
    if (mine) {
#pragma unroll
      for (int x = 0; x < (int)sizeof(ET) / 2; ++x) {
        reinterpret_cast<uint4*>((RT*)cv.K + at)[x] = k.w[x];
        reinterpret_cast<uint4*>((RT*)cv.V + at)[x] = v.w[x];
      }
    }
  } else {
    float ks, vs;
    const uint2 kc = quantise_row<ET, F>(k, ks), vc = quantise_row<ET, F>(v, vs);
    if (mine) {
      *reinterpret_cast<uint2*>((RT*)cv.K + at) = kc;
      *reinterpret_cast<uint2*>((RT*)cv.V + at) = vc;
      const long long sat = blk * cv.ssb + h * cv.ssh + off;
      if (c == 0) {
        cv.ks[sat] = ks;
        cv.vs[sat] = vs;
      }
    }
  }
}

// Eight values of this lane of a cached row, as they are stored, and on to dtype.
template <typename ET, CacheFmt F> struct Stored { uint2 w; };
template <typename ET> struct Stored<ET, kPlain> { Vals8<ET> w; };
template <typename ET, CacheFmt F> __device__ __forceinline__ Stored<ET, F> load_stored(const typename RowType<ET, F>::type* p) {
  if constexpr (F == kPlain) return {load_vals<ET>(p)};
  else return {*reinterpret_cast<const uint2*>(p)};
}
template <typename ET, CacheFmt F> __device__ __forceinline__ void store_vals(ET* dst, const Stored<ET, F>& x, float scale) {
  if constexpr (F == kPlain) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(ET) / 2; ++i) reinterpret_cast<uint4*>(dst)[i] = x.w.w[i];
  } else {
    const f32x4_t a = bytes_to_f32<F>(x.w.x) * scale, b = bytes_to_f32<F>(x.w.y) * scale;
    if constexpr (sizeof(ET) == 2) {
      *reinterpret_cast<uint4*>(dst) = make_uint4(pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3]), pack_bf16(b[0], b[1]), pack_bf16(b[2], b[3]));
    } else {
      reinterpret_cast<f32x4_t*>(dst)[0] = a;
      reinterpret_cast<f32x4_t*>(dst)[1] = b;
    }
  }
}

// grid (tiles of kCacheTile tokens or list entries, rows).  (Heads fastest: 42.0 / 40.8 us, 32768 x 8 int8; a selection 38.8 / 37.6.)
template <typename ET, CacheFmt F>
__global__ __launch_bounds__(256) void cache_read_kernel(ET* __restrict__ K_out, ET* __restrict__ V_out, CacheView cv, const int32_t* __restrict__ T,
                                                         int t_pitch, const int32_t* __restrict__ n_ctx_seq, int n_ctx, int Hkv,
                                                         uint32_t m_hkv, int n_begin, int n_end) {
  using RT = typename RowType<ET, F>::type;
  const int row = blockIdx.y;
  int b, h;
  head_of_row(row, Hkv, m_hkv, b, h);
  const int N = n_ctx_seq ? min(max(n_ctx_seq[b], 0), n_ctx) : n_ctx;
  const int end = min(n_end, T ? min(t_pitch, N) : N);
  const int c = threadIdx.x & 15, j = n_begin + (int)blockIdx.x * kCacheTile + (int)(threadIdx.x >> 4);
  if (j >= end) return;
  const int n = T ? min(max(T[(size_t)row * t_pitch + j], 0), N - 1) : j;
  int blk, off;
  cache_place(cv.pm, b, n, blk, off);
  const long long at = blk * cv.sb + h * cv.sh + off * cv.sn + 8 * c;
  const long long sat = F == kPlain ? 0 : blk * cv.ssb + h * cv.ssh + off;
  Stored<ET, F> k, v;
  float ks = 1.f, vs = 1.f;
  if (K_out) {
    k = load_stored<ET, F>((const RT*)cv.K + at);
    if constexpr (F != kPlain) ks = cv.ks[sat];
  }
  if (V_out) {
    v = load_stored<ET, F>((const RT*)cv.V + at);
    if constexpr (F != kPlain) vs = cv.vs[sat];
  }
  const long long to = ((long long)row * (n_end - n_begin) + (j - n_begin)) * kHeadDim + 8 * c;
  if (K_out) store_vals<ET, F>(K_out + to, k, ks);
  if (V_out) store_vals<ET, F>(V_out + to, v, vs);
}

template <typename ET, CacheFmt F>
static hipError_t write_t(const fasa_shape& s, const CacheView& cv, const ChunkView& ch, long long kv_stride, const void* k_new, const void* v_new,
                          hipStream_t st) {
  const int hkv = s.n_kv_heads;
  const long long each = ((long long)ch.n_new * hkv + kCacheTile - 1) / kCacheTile;
  const long long tiles = chunk_tiles(ch.row_start != nullptr, s.batch, ch.n_new, ch.n_rows, hkv, kCacheTile);
  return launch("fasa_cache_write", cache_write_kernel<ET, F>, dim3((unsigned)tiles), dim3(256), st, (const ET*)k_new, (const ET*)v_new, cv, ch, s.batch,
                hkv, div_magic(hkv, (long long)ch.n_new * hkv), (int)each, kv_stride);
}
template <typename ET, CacheFmt F>
static hipError_t read_t(const fasa_shape& s, const CacheView& cv, const int32_t* T, const int32_t* n_ctx_seq, int n_begin, int n_end, void* K_out,
                         void* V_out, hipStream_t st) {
  const int rows = s.batch * s.n_kv_heads, pitch = s.budget < s.n_ctx ? s.budget : s.n_ctx;
  return launch("fasa_cache_read", cache_read_kernel<ET, F>, dim3((n_end - n_begin + kCacheTile - 1) / kCacheTile, rows), dim3(256), st, (ET*)K_out, (ET*)V_out,
                cv, T, pitch, n_ctx_seq, s.n_ctx, s.n_kv_heads, div_magic(s.n_kv_heads, rows), n_begin, n_end);
}

#define FASA_BY_FORMAT(call, ...)                                                                                   \
  (s.dtype == FASA_BF16 ? (fmt == kPlain  ? call<uint16_t, kPlain>(__VA_ARGS__)                                     \
                           : fmt == kInt8 ? call<uint16_t, kInt8>(__VA_ARGS__) : call<uint16_t, kE4m3>(__VA_ARGS__)) \
                        : (fmt == kPlain  ? call<float, kPlain>(__VA_ARGS__)                                        \
                           : fmt == kInt8 ? call<float, kInt8>(__VA_ARGS__) : call<float, kE4m3>(__VA_ARGS__)))

hipError_t launch_cache_write(const fasa_shape& s, const CacheView& cv, CacheFmt fmt, const ChunkView& ch, long long kv_stride, const void* k_new,
                              const void* v_new, hipStream_t st) {
  return FASA_BY_FORMAT(write_t, s, cv, ch, kv_stride, k_new, v_new, st);
}
hipError_t launch_cache_read(const fasa_shape& s, const CacheView& cv, CacheFmt fmt, const int32_t* T, const int32_t* n_ctx_seq, int n_begin,
                             int n_end, void* K_out, void* V_out, hipStream_t st) {
  return FASA_BY_FORMAT(read_t, s, cv, T, n_ctx_seq, n_begin, n_end, K_out, V_out, st);
}

}  // namespace fasa
