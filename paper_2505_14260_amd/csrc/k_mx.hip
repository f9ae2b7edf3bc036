// Microscaled 4-bit operators: quantisation, the norms and activations that
// end in it, and the product of quantised matrices.
//
// A row is cut into blocks of 32 values that share a power of two,
//   s = 2^(floor(log2 max|x|) - 2), held as its exponent + 127 (0 .. 252),
// and x / s is rounded to E2M1 (0 .5 1 1.5 2 3 4 6 and their negatives), to the
// nearest, ties to the even code, saturating at 6: the OCP Microscaling Formats'
// MXFP4.  A block that holds a NaN or an infinity has the scale 255 and stands
// for NaN; a block of zeros has the scale code 0.
//
// Activations take two such terms, hi = MX(x) and lo = MX(x - hi) (x - hi is
// exact in float32): 8 bits and two scales stand for hi + lo.  On the matrix cores
// a product with an E4M3 operand keeps its sums to 3e-5 of the sum of |x w| (2e-4
// at worst) where 4-bit operands keep float32 (6e-8), two 4-bit products take the
// cycles of one with an 8-bit operand, and the rounding of two terms is half
// E4M3's (normal values: 1.5% against 2.9% of their norm; one term 11.5%).
//
// Layout: tiles of 16 rows x 128 columns of one term, 1 KB in the order in which the
// product's lanes read them: lane l's 16 bytes (row l % 16, block l / 16 of four, two
// values a byte, the lower nibble first) at 16 l.  A row of tiles lies in sequence,
// per 16 rows first that of term 0, then of term 1.  The scales of four neighbouring
// tiles (a group, 512 columns) take 256 bytes, lane l's four at 4 l, so that a dword
// of scales serves four tiles.  Columns past K are zero, scales too (255 in a row that
// the norm made all NaN); rows past the last are zero in weights and left as they were
// in activations, whose products are not stored.  Weights (one term) and activations
// differ in nothing else.
#include <hip/hip_fp16.h>

#include <type_traits>

#include "msd_internal.h"
#include "mx_plan.h"

namespace msd {

namespace {

constexpr int BLK = 32;     // values per scale
constexpr int KT = 128;     // columns of a tile
constexpr int GROUP = MX_GROUP;  // columns of a group of scales
constexpr int TILE_BYTES = 16 * KT / 2;

constexpr int GROUP_SCALES = 256;  // bytes of scales of 16 rows of a group

// Bytes from a row of tiles, and from its scales, to the next.
MSD_DEV size_t tiles_pitch(int nkt) { return (size_t)nkt * TILE_BYTES; }
MSD_DEV size_t scales_pitch(int groups) { return (size_t)groups * GROUP_SCALES; }

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// Sixteen bytes at the alignment of the elements: rows may begin anywhere, and the
// hardware takes such loads and stores whole.
template <int TYPE>
struct Unit;
template <>
struct Unit<MX_F32> {
  typedef uint32_t u32x4_a __attribute__((ext_vector_type(4), aligned(4)));
  typedef u32x4_a type;
};
template <>
struct Unit<MX_BF16> {
  typedef uint32_t u32x4_a __attribute__((ext_vector_type(4), aligned(2)));
  typedef u32x4_a type;
};
template <>
struct Unit<MX_F16> : Unit<MX_BF16> {};

template <int TYPE>
MSD_DEV float from16(uint16_t h) {
  return TYPE == MX_BF16 ? bf2f(h) : __half2float(__builtin_bit_cast(__half, h));
}

template <int TYPE>
MSD_DEV uint16_t to16(float v) {
  return TYPE == MX_BF16 ? f2bf(v) : __builtin_bit_cast(uint16_t, __float2half(v));
}

// Eight neighbouring values of a float matrix; those at and past n are zero.
template <int TYPE>
MSD_DEV void load8(const void* p, size_t at, int n, float* v) {
  typedef typename Unit<TYPE>::type U;
  if (n >= 8) {
    if constexpr (TYPE == MX_F32) {
      const U* q = reinterpret_cast<const U*>(static_cast<const float*>(p) + at);
      const U a = q[0], b = q[1];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = __uint_as_float(a[i]);
        v[4 + i] = __uint_as_float(b[i]);
      }
    } else {
      const U a = *reinterpret_cast<const U*>(static_cast<const uint16_t*>(p) + at);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = from16<TYPE>((uint16_t)(a[i / 2] >> (16 * (i & 1))));
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = 0.f;
    if (i >= n) continue;
    if constexpr (TYPE == MX_F32)
      v[i] = static_cast<const float*>(p)[at + i];
    else
      v[i] = from16<TYPE>(static_cast<const uint16_t*>(p)[at + i]);
  }
}

template <int TYPE>
MSD_DEV void store8(void* p, size_t at, int n, const float* v) {
  typedef typename Unit<TYPE>::type U;
  if (n >= 8) {
    if constexpr (TYPE == MX_F32) {
      U* q = reinterpret_cast<U*>(static_cast<float*>(p) + at);
      U a, b;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        a[i] = __float_as_uint(v[i]);
        b[i] = __float_as_uint(v[4 + i]);
      }
      q[0] = a;
      q[1] = b;
    } else {
      U w;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] = to16<TYPE>(v[2 * i]) | (uint32_t)to16<TYPE>(v[2 * i + 1]) << 16;
      *reinterpret_cast<U*>(static_cast<uint16_t*>(p) + at) = w;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (i >= n) continue;
    if constexpr (TYPE == MX_F32)
      static_cast<float*>(p)[at + i] = v[i];
    else
      static_cast<uint16_t*>(p)[at + i] = to16<TYPE>(v[i]);
  }
}

typedef float f32x2 __attribute__((ext_vector_type(2)));

// The eight values of a lane's codes under their block's scale (below 255).  The
// conversion instructions take a scale from the exponent bits alone (0: 2^-127).
MSD_DEV void values8(uint32_t codes, uint32_t sc, float* v) {
  const float s = __uint_as_float(sc << 23);
  const f32x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 0),
                      __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 1),
                      __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 2),
                      __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 3)};
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = p[i / 2][i & 1];
}

// One term of a block whose 32 values lie in four neighbouring lanes, eight
// each: the codes of this lane's (the return value) and the block's scale; v
// becomes what is left, exactly.
MSD_DEV uint32_t quantise8(float* v, uint32_t* scale) {
  uint32_t top = 0;  // as bits, so that a NaN is largest
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  // over four lanes, by moves within quads: lanes 1 0 3 2, then 2 3 0 1
  top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0xB1, 0xF, 0xF, true));
  top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x4E, 0xF, 0xF, true));
  const uint32_t e = top >> 23;
  if (e == 255u) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(0x7FC00000u);
    *scale = 255u;
    return 0u;
  }
  const uint32_t sc = e > 2u ? e - 2u : 0u;
  *scale = sc;
  // the conversions round to the nearest, ties to even, and saturate
  const float s = __uint_as_float(sc << 23);
  uint32_t codes = 0;
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[0], v[1], s, 0);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[2], v[3], s, 1);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[4], v[5], s, 2);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[6], v[7], s, 3);
  float q[8];
  values8(codes, sc, q);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] -= q[i];
  return codes;
}

// A quantised matrix of activations.
struct RowsOut {
  uint8_t* codes;
  uint8_t* scales;
  int nkt, groups;
};

// Byte offsets of the codes from column k0 on and of the scale of their block.
MSD_DEV size_t code_at(size_t row, int t, int k0, int terms, int nkt) {
  const int lane = ((k0 >> 5) & 3) * 16 + (int)(row & 15);
  return ((row >> 4) * terms + t) * tiles_pitch(nkt) + (k0 >> 7) * TILE_BYTES + lane * 16 +
         ((k0 & 31) >> 1);
}
MSD_DEV size_t scale_at(size_t row, int t, int k0, int terms, int groups) {
  const int lane = ((k0 >> 5) & 3) * 16 + (int)(row & 15);
  return ((row >> 4) * terms + t) * scales_pitch(groups) + (k0 >> 9) * GROUP_SCALES + lane * 4 +
         ((k0 >> 7) & 3);
}

// Quantises a wave's 512 columns of a row, this lane's eight from k0 on.
template <int TX>
MSD_DEV void put_rows(const RowsOut& o, size_t row, int k0, float* v) {
#pragma unroll
  for (int t = 0; t < TX; ++t) {
    uint32_t sc;
    const uint32_t c = quantise8(v, &sc);
    if (k0 < o.nkt * KT)
      *reinterpret_cast<uint32_t*>(o.codes + code_at(row, t, k0, TX, o.nkt)) = c;
    if (!(threadIdx.x & 3)) o.scales[scale_at(row, t, k0, TX, o.groups)] = (uint8_t)sc;
  }
}

// ------------------------------------------------------------ quantise ----
// A float matrix [rows][cols] whose rows lie ld values apart; or a bf16 weight
// in the packed order of k_gemm.hip, or split rows (MX_SPLIT: hi, then lo).
struct Source {
  const void* p;
  size_t ld;
  int cols;
  int nkt;  // 128-column blocks (packed)
};

template <int TYPE>
MSD_DEV void load_src(const Source& s, size_t row, int k0, float* v) {
  if constexpr (TYPE == MX_PACKED) {
    const size_t blk = (row >> 6) * s.nkt + (k0 >> 7);
    const size_t unit = (((row >> 4) & 3) * 4 + ((k0 >> 3) & 3)) * 64 + (row & 15) + 16 * ((k0 >> 5) & 3);
    load8<MX_BF16>(s.p, blk * 8192 + unit * 8, 8, v);
  } else if constexpr (TYPE == MX_SPLIT) {
    float lo[8];
    load8<MX_BF16>(s.p, row * s.ld + k0, s.cols - k0, v);
    load8<MX_BF16>(s.p, row * s.ld + s.cols + k0, s.cols - k0, lo);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += lo[i];
  } else {
    load8<TYPE>(s.p, row * s.ld + k0, s.cols - k0, v);
  }
}

// Activations: a workgroup takes 16 rows of 512 columns, a wave one of them, a lane
// eight columns; the rows' 16-byte pieces of a tile so meet in one L2.  (Four rows per
// wave, their loads together, are slower: 3,136 x 11,008 float32 52 us against 40.)
// Bound by memory once large, by the launch before: 10 x 4,096
// in 3 us; 3,136 x 11,008 float32 in 40, 175 MB with the codes at 4.4 TB/s of a copy's 4.8.
constexpr int ROW_THREADS = 16 * 64;
template <int TYPE, int TX>
__global__ __launch_bounds__(ROW_THREADS) void k_mx_rows(Source s, int rows, RowsOut o) {
  const size_t tile = blockIdx.x / o.groups;
  const size_t row = tile * 16 + (threadIdx.x >> 6);
  if (row >= (size_t)rows) return;
  const int k0 = (int)(blockIdx.x - tile * o.groups) * GROUP + (threadIdx.x & 63) * 8;
  float v[8];
  load_src<TYPE>(s, row, k0, v);
  put_rows<TX>(o, row, k0, v);
}

// Weights: a workgroup takes 16 rows of 512 columns, a lane eight columns of a row in
// each of the four tiles, so that it has its dword of scales.  Bound by memory: 4,096 x 8,192
// bf16, 85 MB, in 20 us (4.2 TB/s).
template <int TYPE>
__global__ __launch_bounds__(256) void k_mx_weight(Source s, int rows, int groups, int nkt,
                                                   uint8_t* codes, uint32_t* scales) {
  const size_t t = blockIdx.x / groups;
  const int g = (int)(blockIdx.x - t * groups);
  const int r = threadIdx.x >> 4, c = threadIdx.x & 15;
  const size_t row = t * 16 + r;
  uint32_t sc4 = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int kt = g * 4 + j;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
    if (row < (size_t)rows && kt < nkt) load_src<TYPE>(s, row, kt * KT + c * 8, v);
    uint32_t sc;
    const uint32_t q = quantise8(v, &sc);
    sc4 |= sc << (8 * j);
    if (kt < nkt)
      *reinterpret_cast<uint32_t*>(codes + t * tiles_pitch(nkt) + kt * TILE_BYTES +
                                   ((c >> 2) * 16 + r) * 16 + (c & 3) * 4) = q;
  }
  if (!(c & 3)) scales[t * (scales_pitch(groups) / 4) + g * 64 + (c >> 2) * 16 + r] = sc4;
}

// ---------------------------------------------------------- dequantise ----
// The same workgroups; a wave takes R of the rows.  Bound by memory: 4,096 x 8,192 of
// one term to bf16, 85 MB, in 17 us (5.1 TB/s).
template <int TYPE, int TX, int R>
__global__ __launch_bounds__(ROW_THREADS / R) void k_mx_values(RowsOut q, int rows, int cols,
                                                               void* out, size_t ld) {
  const size_t tile = blockIdx.x / q.groups;
  const size_t row = tile * 16 + (threadIdx.x >> 6) * R;
  const int k0 = (int)(blockIdx.x - tile * q.groups) * GROUP + (threadIdx.x & 63) * 8;
  if (k0 >= cols) return;
  uint32_t c[R][TX], sc[R][TX];
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int t = 0; t < TX; ++t) {
      if (row + i >= (size_t)rows) continue;
      c[i][t] = *reinterpret_cast<const uint32_t*>(q.codes + code_at(row + i, t, k0, TX, q.nkt));
      sc[i][t] = q.scales[scale_at(row + i, t, k0, TX, q.groups)];
    }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (row + i >= (size_t)rows) continue;
    float v[8], w[8];
    values8(c[i][0], sc[i][0], v);
    if constexpr (TX == 2) {
      values8(c[i][1], sc[i][1], w);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] += w[k];
    }
    if (sc[i][0] == 255u) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(0x7FC00000u);
    }
    store8<TYPE>(out, (row + i) * ld + k0, cols - k0, v);
  }
}

// ---------------------------------------------------------------- norm ----
// One workgroup per row, the row's sum in registers between its two uses.  The
// mean square and the scaling are in float64: 4-bit values change with the last
// bit of what is rounded to them, and the operator is bound by memory: 3,136 x 4,096
// float32, 168 MB with the codes, in 37 us (4.5 TB/s); 26 rows of 3,584 bf16 in 4.5, the launch.
// From so many rows on, the 16 rows of a tile run on one XCD (workgroup i runs on XCD
// i mod 8), so that their 16-byte pieces of its codes leave one L2 in whole lines.
constexpr int NORM_TILE_ROWS = 128;
template <int TYPE, int NT>
__global__ __launch_bounds__(NT) void k_mx_norm(const void* x, size_t ldx, const void* y, size_t ldy,
                                                void* xo, size_t ldo, const uint16_t* gain, int rows,
                                                int d, double eps, RowsOut o, const int* dst,
                                                float* feat) {
  __shared__ double sh[NT / 64];
  size_t row = blockIdx.x;
  if (rows >= NORM_TILE_ROWS) {
    const int i = blockIdx.x >> 3;
    row = (size_t)((i >> 4) * 8 + (blockIdx.x & 7)) * 16 + (i & 15);
    if (row >= (size_t)rows) return;
  }
  const int k0 = (int)threadIdx.x * 8, n = d - k0;
  float v[8], g[8];
  load8<TYPE>(x, row * ldx + k0, n, v);
  if (y) {
    float u[8];
    load8<TYPE>(y, row * ldy + k0, n, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += u[i];
  }
  if (xo) store8<TYPE>(xo, row * ldo + k0, n, v);
  if (!gain) {
    if (feat && dst[row] >= 0) store8<MX_F32>(feat, (size_t)dst[row] * d + k0, n, v);
    if (k0 / GROUP < o.groups) put_rows<2>(o, row, k0, v);
    return;
  }
  load8<MX_BF16>(gain, k0, n, g);
  double ss = 0.0;
#pragma unroll
  for (int i = 0; i < 8; ++i) ss = fma((double)v[i], (double)v[i], ss);
  for (int k = 32; k > 0; k >>= 1) ss += __shfl_xor(ss, k);
  if (!(threadIdx.x & 63)) sh[threadIdx.x >> 6] = ss;
  __syncthreads();
  ss = 0.0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) ss += sh[w];
  if (k0 / GROUP >= o.groups) return;  // a wave past the last group
  const double r = 1.0 / sqrt(ss / d + eps);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)((double)v[i] * r * (double)g[i]);
  put_rows<2>(o, row, k0, v);
}

// -------------------------------------------------------------- swiglu ----
// silu(g) u = g u r for g >= 0, g u t r below, with t = e^-|g| = f 2^n and r = 1 / (1 + t)
// (1 ulp).  f is the hardware's 2^x (1 ulp) of -|g| log2(e) - n, the product in two parts;
// past |g| = 1000 all of it is zero.  2^n takes its place last, so that neither t nor
// silu(g) has to be a normal float32 value for g u t r to be right: g f is exact for a
// denormal g (f = 1), and u r rounds a denormal u by 2^-150, which g <= 17 (r < 1) cannot
// make more than 2^-145 (the smallest 4-bit step is 2^-128).  HALVES: half of 2^n before
// the product with u r, which overflows without it where |u| is 2^119 and more; calls
// without come first, and again with it where the value is not finite (640 x 11,008
// float32: 13.2 us, 12.9 with expf and silu(g) rounded first, 13.7 with HALVES at once).
template <bool HALVES>
MSD_DEV float silu_times(float g, float u) {
  const float a = -__builtin_amdgcn_fmed3f(fabsf(g), 0.f, 1000.f);
  const float L = 0x1.715476p+0f, M = 0x1.4ae0cp-26f;  // log2(e) = L + M
  const float m = rintf(a * L);
  const float f = __builtin_amdgcn_exp2f(fmaf(a, M, fmaf(a, L, -m)));
  const int n = (int)m;
  const float r = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_ldexpf(f, n));
  const int e = g < 0.f ? n : 0, h = HALVES ? e >> 1 : 0;
  float w = g < 0.f ? g * f : g;
  if (HALVES) w = __builtin_amdgcn_ldexpf(w, h);
  return __builtin_amdgcn_ldexpf(w * (u * r), e - h);
}

// Activations' split (k_mx_rows).  Bound by memory, near its arithmetic's time: 640 x 11,008
// float32, 64 MB with the codes, in 13.2 us (4.9 TB/s); 10 rows 3.7 us.
template <int TYPE>
__global__ __launch_bounds__(ROW_THREADS) void k_mx_swiglu(const void* gate, const void* up,
                                                           size_t ldg, size_t ldu, int rows, int F,
                                                           RowsOut o) {
  const size_t tile = blockIdx.x / o.groups;
  const size_t row = tile * 16 + (threadIdx.x >> 6);
  if (row >= (size_t)rows) return;
  const int k0 = (int)(blockIdx.x - tile * o.groups) * GROUP + (threadIdx.x & 63) * 8;
  float g[8], u[8];
  load8<TYPE>(gate, row * ldg + k0, F - k0, g);
  load8<TYPE>(up, row * ldu + k0, F - k0, u);
  float v[8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = silu_times<false>(g[i], u[i]);
    top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  }
  if (__builtin_expect(__any(top >= 0x7F800000u), 0)) {  // out of the common path's way
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (!__builtin_isfinite(v[i])) v[i] = silu_times<true>(g[i], u[i]);
  }
  put_rows<2>(o, row, k0, v);
}

// ------------------------------------------------------------- product ----
struct ProductArgs {
  const uint8_t *xc, *xs;  // activations
  const uint8_t *wc, *ws;  // weight
  int M, N, nkt, groups;   // 128-column tiles and groups of four along K
  void* out;
  size_t ldo;
  bool vec;  // rows of out take stores of four values
};

// Four neighbouring columns of an output row.
template <int TYPE>
MSD_DEV void store4(const ProductArgs& a, int m, int n, const f32x4& v) {
  const size_t at = (size_t)m * a.ldo + n;
  if (a.vec && n + 4 <= a.N) {
    if constexpr (TYPE == MX_F32) {
      *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + at) = v;
    } else {
      const uint2 w = make_uint2(to16<TYPE>(v[0]) | (uint32_t)to16<TYPE>(v[1]) << 16,
                                 to16<TYPE>(v[2]) | (uint32_t)to16<TYPE>(v[3]) << 16);
      *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + at) = w;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (n + i >= a.N) break;
    if constexpr (TYPE == MX_F32)
      static_cast<float*>(a.out)[at + i] = v[i];
    else
      static_cast<uint16_t*>(a.out)[at + i] = to16<TYPE>(v[i]);
  }
}

// acc += a 16 x 128 tile of W (rows) times one of X (columns): lane l gets the
// products of X row l % 16 and W rows 4 (l / 16) .. + 3.  The scales are bytes
// `byte` (known when compiled) of ws and xs.
MSD_DEV f32x4 mfma_mx(i32x4 w, i32x4 x, f32x4 acc, int ws, int xs, int byte) {
  const i32x8 w8 = __builtin_shufflevector(w, w, 0, 1, 2, 3, -1, -1, -1, -1);
  const i32x8 x8 = __builtin_shufflevector(x, x, 0, 1, 2, 3, -1, -1, -1, -1);
#define MX_BYTE(B) __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w8, x8, acc, 4, 4, B, ws, B, xs)
  switch (byte) {
    case 0: return MX_BYTE(0);
    case 1: return MX_BYTE(1);
    case 2: return MX_BYTE(2);
    default: return MX_BYTE(3);
  }
#undef MX_BYTE
}

// Few rows or few columns: a workgroup takes 16 MT rows and 16 CT columns whole, its
// eight waves the groups of K in turn, straight from memory to registers, D - 1 tiles
// ahead, with no barrier on the way.  Their sums meet in LDS: of waves w and w + 4
// first, then of the four.  Eight waves share K so that few columns still fill the
// chip's memory queues, and each reads 1 KB of W in a row.  Up to 16 rows two workgroups
// share a CU (128 registers, so fewer tiles ahead; 10 x 152,064 x 3,584: 62 us with one).
// Bound by W's bytes: 10 rows by 152,064 x 3,584 (290 MB) in 50 us, 5.8 TB/s; by 4,096 x
// 4,096 (8.9 MB) in 4.4.  Over few columns and more rows by X, which every workgroup reads:
// 64 x 4,096 x 11,008 in 16.4 us, 190 MB of X for 24 MB of W.
template <int MT, int CT, int TX, int TYPE>
__global__ __launch_bounds__(64 * SPLIT_WAVES, MT == 1 ? 4 : 2) void k_mx_split(ProductArgs a, int n_ct) {
  constexpr int NW = SPLIT_WAVES, U = MT * CT;
  __shared__ f32x4 sh[NW / 2][U][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m0 = (int)(blockIdx.x / n_ct) * MT, n0 = (int)(blockIdx.x % n_ct) * CT;  // in tiles
  const int xlast = (a.M - 1) >> 4, wlast = (a.N - 1) >> 4, nkt = a.nkt, groups = a.groups;
  // tiles past the last repeat it; their sums are not stored
  const uint8_t *xc[MT][TX], *xs[MT][TX], *wc[CT], *ws[CT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int t = 0; t < TX; ++t) {
      const size_t u = (size_t)min(m0 + m, xlast) * TX + t;
      xc[m][t] = a.xc + u * tiles_pitch(nkt);
      xs[m][t] = a.xs + u * scales_pitch(groups);
    }
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const size_t u = min(n0 + c, wlast);
    wc[c] = a.wc + u * tiles_pitch(nkt);
    ws[c] = a.ws + u * scales_pitch(groups);
  }
  constexpr int D = MT * TX + CT <= 5 ? 4 : 2;  // tiles in registers
  i32x4 fx[D][MT][TX], fw[D][CT];
  int sx[MT][TX], sw[CT], sxn[MT][TX], swn[CT];
  // tile kt along K; those past the last repeat it, with scales of zero
  const auto load = [&](int i, int kt) {
    const unsigned at = (unsigned)min(kt, nkt - 1) * TILE_BYTES + lane * 16;
#pragma unroll
    for (int c = 0; c < CT; ++c)
      fw[i][c] = __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(wc[c] + at));
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int t = 0; t < TX; ++t) fx[i][m][t] = *reinterpret_cast<const i32x4*>(xc[m][t] + at);
  };
  const auto load_s = [&](int g) {
    const unsigned at = (unsigned)min(g, groups - 1) * GROUP_SCALES + lane * 4;
#pragma unroll
    for (int c = 0; c < CT; ++c) swn[c] = *reinterpret_cast<const int*>(ws[c] + at);
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int t = 0; t < TX; ++t) sxn[m][t] = *reinterpret_cast<const int*>(xs[m][t] + at);
  };
  f32x4 acc[MT][CT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int c = 0; c < CT; ++c) acc[m][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  // the four tiles of group g; `more`: the wave has another one
  const auto group = [&](int g, bool more) {
#pragma unroll
    for (int c = 0; c < CT; ++c) sw[c] = swn[c];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int t = 0; t < TX; ++t) sx[m][t] = sxn[m][t];
    if (more) load_s(g + NW);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      // the tile D - 1 further along the wave's
      if (j + D - 1 < 4) load((j + D - 1) % D, 4 * g + j + D - 1);
      else if (more) load((j + D - 1) % D, 4 * (g + NW) + j + D - 5);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int t = 0; t < TX; ++t)
#pragma unroll
          for (int c = 0; c < CT; ++c)
            acc[m][c] = mfma_mx(fw[j % D][c], fx[j % D][m][t], acc[m][c], sw[c], sx[m][t], j);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  if (wave < groups) {
    load_s(wave);
#pragma unroll
    for (int j = 0; j < D - 1; ++j) load(j, wave * 4 + j);
    int g = wave;
#pragma unroll 1
    for (; g + NW < groups; g += NW) group(g, true);
    group(g, false);
  }
  if (wave >= NW / 2) {
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int c = 0; c < CT; ++c) sh[wave - NW / 2][m * CT + c][lane] = acc[m][c];
  }
  __syncthreads();
  if (wave < NW / 2) {
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int c = 0; c < CT; ++c) sh[wave][m * CT + c][lane] += acc[m][c];
  }
  __syncthreads();
  for (int q = threadIdx.x; q < U * 64; q += 64 * NW) {
    const int u = q >> 6, l = q & 63;
    f32x4 v = sh[0][u][l];
#pragma unroll
    for (int w = 1; w < NW / 2; ++w) v += sh[w][u][l];
    const int row = (m0 + u / CT) * 16 + (l & 15), n = (n0 + u % CT) * 16 + (l >> 4) * 4;
    if (row < a.M && n < a.N) store4<TYPE>(a, row, n, v);
  }
}

// Column tiles that run side by side on an XCD, so that the row tiles' X is read once for
// all of them (640 x 22,016 x 4,096: 59 us with 8 or 16, 64 with 2, 66 with 1).
constexpr int COLUMN_GROUP = 8;
constexpr int RSRC_RAW = 0x00020000;       // raw buffer: 32-bit data format, stride 0
constexpr int PAST = (int)0x80000000u;     // a byte offset past every buffer
MSD_DEV constexpr int vmcnt_imm(int n) { return 0x0f70 | (n & 15) | ((n >> 4) << 14); }

// Many rows: a workgroup of RW x CW waves takes 16 WM RW rows and 16 WN CW columns, a
// wave 16 WM x 16 WN of them.  The tiles of X and W go to LDS by buffer loads with the
// lds bit, in NB buffers, NB - 1 steps (tiles along K) ahead.
// The buffers are arrays of their own and the loads into them buffer loads: the
// compiler then knows that reads of one need not wait for loads into another.  One
// barrier per step: before it every wave waits for its own loads into the next buffer;
// later loads stay in flight.  With four buffers a step's loads go between its matrix
// instructions (640 x 4,096 x 11,008: 41 us, 43 with all of them first); with two, first:
// the step's end waits for them (3,136 x 4,096 x 11,008: 83 us, 99 in between).
// Raw buffer loads check voffset against the record count less soffset, so soffset
// stays inside the buffer: row and column tiles past the last and tiles past K
// (voffset 2^31) read zeros.
// Bound by feeding the matrix units: 640 x 22,016 x 4,096, two terms, in 59 us, 3.9
// PFLOP/s of 4-bit products where the same instructions on registers alone reach about 7;
// its 430 workgroups fill 84% of the places, the units are busy 39% of the time, LDS has
// no bank conflicts.  W read from memory to registers instead of through LDS is slower
// (65), a third buffer and K split over two sets of waves are no faster.
template <int WM, int WN, int RW, int CW, int NB, int OCC, int TX, int TYPE>
__global__ __launch_bounds__(64 * RW * CW, OCC) void k_mx_tile(ProductArgs a, int n_mt, int n_nt,
                                                               int gc) {
  constexpr int NW = RW * CW, BM = 16 * WM * RW, BN = 16 * WN * CW;
  constexpr int UX = WM * RW * TX, UW = WN * CW;  // 1 KB pieces of X and of W per step
  constexpr int XLX = UX / NW, XL = XLX + UW / NW;  // of them per wave: of X, all
  static_assert(UX % NW == 0 && UW % NW == 0, "pieces divide over the waves");
  static_assert(NB == 2 || NB == 4, "buffers and bytes of scales repeat every four steps");
  constexpr bool PRE = NB == 4;  // a step's first fragments are read in the step before
  constexpr int P = (UX + UW) * 64;
  __shared__ i32x4 sh0[P];
  __shared__ i32x4 sh1[P];
  __shared__ i32x4 sh2[NB == 4 ? P : 1];
  __shared__ i32x4 sh3[NB == 4 ? P : 1];
  const auto buf = [&](int i) -> i32x4* {
    return i % NB == 0 ? sh0 : i % NB == 1 ? sh1 : i % NB == 2 ? sh2 : sh3;
  };
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int items = n_mt * n_nt, per = (items + 7) >> 3;
  const int t = ((int)blockIdx.x & 7) * per + ((int)blockIdx.x >> 3);
  if (((int)blockIdx.x >> 3) >= per || t >= items) return;
  // groups of gc column tiles, columns innermost
  const int cg = t / (n_mt * gc), tr = t - cg * n_mt * gc, wide = min(gc, n_nt - cg * gc);
  const int mt = tr / wide, nt = cg * gc + tr - mt * wide, m0 = mt * BM;
  const int rw = wave / CW, cw = wave % CW;
  const int nkt = a.nkt, xtile0 = m0 / 16, xtiles = min((a.M + 15) / 16 - xtile0, BM / 16);
  const int tiles = (a.N + 15) / 16, tile0 = nt * (BN / 16), ntile = min(tiles - tile0, BN / 16);
  const int tp = (int)tiles_pitch(nkt), sp = (int)scales_pitch(a.groups);
  const __amdgpu_buffer_rsrc_t rxc = __builtin_amdgcn_make_buffer_rsrc(
      (void*)(a.xc + (size_t)xtile0 * TX * tp), 0, xtiles * TX * tp, RSRC_RAW);
  const __amdgpu_buffer_rsrc_t rxs = __builtin_amdgcn_make_buffer_rsrc(
      (void*)(a.xs + (size_t)xtile0 * TX * sp), 0, xtiles * TX * sp, RSRC_RAW);
  const __amdgpu_buffer_rsrc_t rwc = __builtin_amdgcn_make_buffer_rsrc(
      (void*)(a.wc + (size_t)tile0 * tp), 0, ntile * tp, RSRC_RAW);
  const __amdgpu_buffer_rsrc_t rws = __builtin_amdgcn_make_buffer_rsrc(
      (void*)(a.ws + (size_t)tile0 * sp), 0, ntile * sp, RSRC_RAW);
  int wso[WN], xso[WM][TX];
#pragma unroll
  for (int j = 0; j < WN; ++j) wso[j] = (cw * WN + j) * sp + lane * 4;
#pragma unroll
  for (int m = 0; m < WM; ++m)
#pragma unroll
    for (int tt = 0; tt < TX; ++tt) xso[m][tt] = ((rw * WM + m) * TX + tt) * sp + lane * 4;
  // piece q of the wave (those of X, then those of W) of tile kt along K
  const auto load1 = [&](i32x4* b, int q, int kt) {
    const bool isx = q < XLX;
    const int u = isx ? wave * XLX + q : wave * (XL - XLX) + q - XLX;
    const int at = u * tp + lane * 16, vo = kt < nkt ? at : PAST;
    const int so = min(kt, nkt - 1) * TILE_BYTES;
    i32x4* const to = b + (isx ? u : UX + u) * 64;
    if (isx)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rxc, (__attribute__((address_space(3))) void*)to, 16, vo, so, 0, 0);
    else
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rwc, (__attribute__((address_space(3))) void*)to, 16, vo, so, 0, 0);
  };
  constexpr int U = WM * TX, PF = U < 4 ? U : 4;  // X fragments of a step; read PF ahead
  constexpr int S = WN + U;                       // loads of scales per group
  i32x4 fw[PRE ? 2 : 1][WN], fx[PF];
  int sw[WN], sx[WM][TX], swn[WN], sxn[WM][TX];
  f32x4 acc[WM][WN];
#pragma unroll
  for (int m = 0; m < WM; ++m)
#pragma unroll
    for (int j = 0; j < WN; ++j) acc[m][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  // the scales of group g
  const auto load_s = [&](int g) {
    const bool in = g < a.groups;
    const int at = min(g, a.groups - 1) * GROUP_SCALES;
#pragma unroll
    for (int j = 0; j < WN; ++j)
      swn[j] = __builtin_amdgcn_raw_buffer_load_b32(rws, in ? wso[j] : PAST, at, 0);
#pragma unroll
    for (int m = 0; m < WM; ++m)
#pragma unroll
      for (int tt = 0; tt < TX; ++tt)
        sxn[m][tt] = __builtin_amdgcn_raw_buffer_load_b32(rxs, in ? xso[m][tt] : PAST, at, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  load_s(0);
#pragma unroll
  for (int i = 0; i < NB - 1; ++i) {
#pragma unroll
    for (int q = 0; q < XL; ++q) load1(buf(i), q, i);
    __builtin_amdgcn_sched_barrier(0);
  }
  constexpr int AHEAD = PRE ? NB - 3 : NB - 2;  // steps whose loads may be in flight at a turn
  const auto turn = [&](bool scales) {
    if (AHEAD == 0) __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    else if (scales) __builtin_amdgcn_s_waitcnt(vmcnt_imm(AHEAD * XL + S));
    else __builtin_amdgcn_s_waitcnt(vmcnt_imm(AHEAD * XL));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  turn(false);
  const int xo = rw * U * 64 + lane, wo = (UX + cw * WN) * 64 + lane;
  const auto first = [&](const i32x4* b, int i) {
#pragma unroll
    for (int u = 0; u < PF; ++u) fx[u] = b[xo + u * 64];
#pragma unroll
    for (int j = 0; j < WN; ++j) fw[PRE ? i & 1 : 0][j] = b[wo + j * 64];
  };
  if (PRE) first(sh0, 0);
  // Step i of a group (known when compiled), tile kt along K.
  const auto step = [&](int i, int kt) {
    const i32x4 *const b = buf(i), *const bn = buf(i + 1);
    if (!PRE) {
#pragma unroll
      for (int q = 0; q < XL; ++q) load1(buf(i + NB - 1), q, kt + NB - 1);
      __builtin_amdgcn_sched_barrier(0);
      first(b, i);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int m = u / TX, tt = u % TX;
#pragma unroll
      for (int j = 0; j < WN; ++j)
        acc[m][j] = mfma_mx(fw[PRE ? i & 1 : 0][j], fx[u % PF], acc[m][j], sw[j], sx[m][tt], i);
      if (u + PF < U) fx[u % PF] = b[xo + (u + PF) * 64];
      else if (PRE) fx[u % PF] = bn[xo + (u + PF - U) * 64];
      if (PRE) {
#pragma unroll
        for (int j = u * WN / U; j < (u + 1) * WN / U; ++j) fw[(i + 1) & 1][j] = bn[wo + j * 64];
      }
      if (PRE) {
#pragma unroll
        for (int q = u * XL / U; q < (u + 1) * XL / U; ++q) load1(buf(i + NB - 1), q, kt + NB - 1);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    // the scales of the next group were loaded in a group's first step, before X and W
    turn(i == 0);
  };
#pragma unroll 1
  for (int g = 0; g < a.groups; ++g) {
#pragma unroll
    for (int j = 0; j < WN; ++j) sw[j] = swn[j];
#pragma unroll
    for (int m = 0; m < WM; ++m)
#pragma unroll
      for (int tt = 0; tt < TX; ++tt) sx[m][tt] = sxn[m][tt];
    load_s(g + 1);
    step(0, 4 * g);
    step(1, 4 * g + 1);
    step(2, 4 * g + 2);
    step(3, 4 * g + 3);
  }
#pragma unroll
  for (int m = 0; m < WM; ++m) {
    const int row = m0 + (rw * WM + m) * 16 + (lane & 15);
    if (row >= a.M) continue;
#pragma unroll
    for (int j = 0; j < WN; ++j) {
      const int n = (tile0 + cw * WN + j) * 16 + (lane >> 4) * 4;
      if (n < a.N) store4<TYPE>(a, row, n, acc[m][j]);
    }
  }
}

RowsOut rows_out(const MxMat& q) {
  return {static_cast<uint8_t*>(q.codes), static_cast<uint8_t*>(q.scales), mx_tiles(q.cols),
          mx_groups(q.cols)};
}

// Workgroups of 16 rows x 512 columns.
unsigned tile_blocks(const MxMat& q) {
  return (unsigned)((size_t)((q.rows + 15) / 16) * mx_groups(q.cols));
}

int type_size(int type) { return type == MX_F32 ? 4 : 2; }

}  // namespace

#define MX_TYPES(type, go)             \
  do {                                 \
    if (type == MX_F32) go(MX_F32);    \
    else if (type == MX_BF16) go(MX_BF16); \
    else go(MX_F16);                   \
  } while (0)

void launch_mx_quantise(const void* src, int type, size_t ld, const MxMat& q, hipStream_t st) {
  if (q.rows <= 0) return;
  const Source s{src, ld, q.cols, mx_tiles(q.cols)};
  if (q.weight) {
    const auto go = [&](auto k) {
      hipLaunchKernelGGL(k, dim3(tile_blocks(q)), dim3(256), 0, st, s, q.rows, mx_groups(q.cols),
                         mx_tiles(q.cols), static_cast<uint8_t*>(q.codes),
                         static_cast<uint32_t*>(q.scales));
    };
    if (type == MX_PACKED) go(k_mx_weight<MX_PACKED>);
    else if (type == MX_F32) go(k_mx_weight<MX_F32>);
    else if (type == MX_BF16) go(k_mx_weight<MX_BF16>);
    else go(k_mx_weight<MX_F16>);
    return;
  }
  const auto go = [&](auto k) {
    hipLaunchKernelGGL(k, dim3(tile_blocks(q)), dim3(ROW_THREADS), 0, st, s, q.rows, rows_out(q));
  };
#define GO(T)                                 \
  do {                                        \
    if (q.terms == 2) go(k_mx_rows<T, 2>);    \
    else go(k_mx_rows<T, 1>);                 \
  } while (0)
  if (type == MX_SPLIT) GO(MX_SPLIT);
  else MX_TYPES(type, GO);
#undef GO
}

void launch_mx_dequantise(const MxMat& q, void* dst, int type, size_t ld, hipStream_t st) {
  if (q.rows <= 0) return;
  const unsigned blocks = tile_blocks(q);
  const auto go = [&](auto k, int R) {
    hipLaunchKernelGGL(k, dim3(blocks), dim3(ROW_THREADS / R), 0, st, rows_out(q), q.rows, q.cols,
                       dst, ld);
  };
  // four rows per wave where one term leaves a wave little to load and there are many
  // (4,096 x 8,192: 17.5 us against 21.0; with fewer or two terms one row is faster)
#define GO(T)                                              \
  do {                                                     \
    if (q.terms == 2) go(k_mx_values<T, 2, 1>, 1);         \
    else if (blocks < 2048) go(k_mx_values<T, 1, 1>, 1);   \
    else go(k_mx_values<T, 1, 4>, 4);                      \
  } while (0)
  MX_TYPES(type, GO);
#undef GO
}

void launch_mx_norm(const void* x, size_t ldx, const void* y, size_t ldy, void* xo, size_t ldo,
                    int type, const uint16_t* gain, float eps, const MxMat& q, hipStream_t st,
                    const int* dst, float* feat) {
  if (q.rows <= 0) return;
  const int d = q.cols;
  const auto go = [&](auto k, int threads) {
    hipLaunchKernelGGL(k, dim3(q.rows < NORM_TILE_ROWS ? q.rows : (q.rows + 127) / 128 * 128),
                       dim3(threads), 0, st, x, ldx, y, ldy, xo, ldo, gain, q.rows, d, (double)eps,
                       rows_out(q), dst, feat);
  };
#define GO(T)                                          \
  do {                                                 \
    if (d <= 2048) go(k_mx_norm<T, 256>, 256);         \
    else if (d <= 4096) go(k_mx_norm<T, 512>, 512);    \
    else go(k_mx_norm<T, 1024>, 1024);                 \
  } while (0)
  MX_TYPES(type, GO);
#undef GO
}

void launch_mx_swiglu(const void* gate, size_t ldg, const void* up, size_t ldu, int type,
                      const MxMat& q, hipStream_t st) {
  if (q.rows <= 0) return;
#define GO(T)                                                                                    \
  hipLaunchKernelGGL(k_mx_swiglu<T>, dim3(tile_blocks(q)), dim3(ROW_THREADS), 0, st, gate, up, ldg, \
                     ldu, q.rows, q.cols, rows_out(q))
  MX_TYPES(type, GO);
#undef GO
}

namespace {

template <int TX, int TYPE>
void product(const ProductArgs& a, hipStream_t st) {
  const ProductPlan p = plan_product(a.M, a.N, a.groups, TX);
  const int n_mt = p.CT ? 0 : (a.M + p.BM - 1) / p.BM, n_nt = p.CT ? 0 : (a.N + p.BN - 1) / p.BN;
  const auto tile = [&](auto k, int threads) {
    hipLaunchKernelGGL(k, dim3(8 * ((n_mt * n_nt + 7) / 8)), dim3(threads), 0, st, a, n_mt, n_nt,
                       COLUMN_GROUP);
  };
  const auto split = [&](auto k) {
    const int n_ct = (a.N + 16 * p.CT - 1) / (16 * p.CT);
    hipLaunchKernelGGL(k, dim3((unsigned)n_ct * ((a.M + 16 * p.MT - 1) / (16 * p.MT))),
                       dim3(64 * SPLIT_WAVES), 0, st, a, n_ct);
  };
  if (p.BM == 64) tile(k_mx_tile<2, 4, 2, 2, 4, 2, TX, TYPE>, 256);
  else if (p.BM == 128) tile(k_mx_tile<4, 8, 2, 2, 2, 2, TX, TYPE>, 256);
  else if (p.BM == 256) tile(k_mx_tile<4, 8, 4, 2, 2, 2, TX, TYPE>, 512);
#define GO(M)                                             \
  else if (p.MT == M) {                                   \
    if (p.CT == 1) split(k_mx_split<M, 1, TX, TYPE>);     \
    else if (p.CT == 2) split(k_mx_split<M, 2, TX, TYPE>); \
    else split(k_mx_split<M, 4, TX, TYPE>);               \
  }
  GO(1) GO(2) GO(4)
#undef GO
}

}  // namespace

void launch_mx_product(const MxMat& x, const MxMat& w, void* out, int type, size_t ldo,
                       hipStream_t st) {
  if (x.rows <= 0 || w.rows <= 0) return;
  ProductArgs a{static_cast<const uint8_t*>(x.codes), static_cast<const uint8_t*>(x.scales),
                static_cast<const uint8_t*>(w.codes), static_cast<const uint8_t*>(w.scales),
                x.rows, w.rows, mx_tiles(w.cols), mx_groups(w.cols), out, ldo, false};
  const int sz = type_size(type);
  a.vec = !((uintptr_t)out & (4 * sz - 1)) && ldo % 4 == 0;
#define GO(T)                               \
  do {                                      \
    if (x.terms == 2) product<2, T>(a, st); \
    else product<1, T>(a, st);              \
  } while (0)
  MX_TYPES(type, GO);
#undef GO
}

}  // namespace msd
