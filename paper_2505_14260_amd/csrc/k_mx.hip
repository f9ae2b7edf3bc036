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
// Layouts, both in the order in which the product's lanes read a 16 x 128 tile
// (lane l: row l % 16, block l / 16 of four):
//  rows    row r: the codes of term 0, of term 1, K padded to 128 columns, two
//          values a byte, the lower nibble first; its scales, per term groups of
//          16 blocks (512 columns), block b of a group at byte 4 (b % 4) + b / 4;
//  weight  tiles (16 rows x 128 columns) of 1 KB, along a row of tiles first, lane
//          l's 16 bytes at 16 l; the scales of four neighbouring tiles in 256
//          bytes, lane l's four at 4 l.
// A lane's dword of scales so serves four tiles.  Padding is zero.
#include <hip/hip_fp16.h>

#include "msd_internal.h"

namespace msd {

namespace {

constexpr int BLK = 32;     // values per scale
constexpr int KT = 128;     // columns of a tile
constexpr int GROUP = 512;  // columns of a group of scales
constexpr int TILE_BYTES = 16 * KT / 2;

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// Eight neighbouring values of a float matrix; those at and past n are zero.
template <int TYPE>
MSD_DEV void load8(const void* p, size_t at, int n, bool vec, float* v) {
  if (vec && n >= 8) {
    if constexpr (TYPE == MX_F32) {
      const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
      const float4 a = q[0], b = q[1];
      v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
      v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
      const uint4 a = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + at);
      const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint16_t h = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
        v[i] = TYPE == MX_BF16 ? bf2f(h) : __half2float(__builtin_bit_cast(__half, h));
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = 0.f;
    if (i >= n) continue;
    if constexpr (TYPE == MX_F32) {
      v[i] = static_cast<const float*>(p)[at + i];
    } else {
      const uint16_t h = static_cast<const uint16_t*>(p)[at + i];
      v[i] = TYPE == MX_BF16 ? bf2f(h) : __half2float(__builtin_bit_cast(__half, h));
    }
  }
}

template <int TYPE>
MSD_DEV uint16_t to16(float v) {
  return TYPE == MX_BF16 ? f2bf(v) : __builtin_bit_cast(uint16_t, __float2half(v));
}

template <int TYPE>
MSD_DEV void store8(void* p, size_t at, int n, bool vec, const float* v) {
  if (vec && n >= 8) {
    if constexpr (TYPE == MX_F32) {
      float4* q = reinterpret_cast<float4*>(static_cast<float*>(p) + at);
      q[0] = make_float4(v[0], v[1], v[2], v[3]);
      q[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] = to16<TYPE>(v[2 * i]) | (uint32_t)to16<TYPE>(v[2 * i + 1]) << 16;
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + at) = make_uint4(w[0], w[1], w[2], w[3]);
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

// 2^(code - 127), code 0 .. 254
MSD_DEV float scale_value(uint32_t code) {
  return __uint_as_float(code ? code << 23 : 0x00400000u);
}

// One term of a block whose 32 values lie in four neighbouring lanes, eight
// each: the codes of this lane's (the return value) and the block's scale; v
// becomes what is left, exactly.
MSD_DEV uint32_t quantise8(float* v, uint32_t* scale) {
  uint32_t top = 0;  // as bits, so that a NaN is largest
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  top = max(top, (uint32_t)__shfl_xor((int)top, 1));
  top = max(top, (uint32_t)__shfl_xor((int)top, 2));
  const int e = (int)(top >> 23);
  const bool nan = e == 255;
  const uint32_t sc = nan ? 255u : (uint32_t)max(e - 2, 0);
  *scale = sc;
  const float inv = __uint_as_float((254u - (nan ? 127u : sc)) << 23), s = scale_value(nan ? 127u : sc);
  uint32_t codes = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = fabsf(v[i]) * inv;
    // the step is 1/2 below 2, 1 below 4, then 2
    const float step = a < 2.f ? 0.5f : a < 4.f ? 1.f : 2.f;
    const float per = a < 2.f ? 2.f : a < 4.f ? 1.f : 0.5f;
    const float q = fminf(__builtin_rintf(a * per) * step, 6.f);
    // the code of q: 2q up to 2, q + 2 up to 4, q / 2 + 4
    const uint32_t c = (uint32_t)(q < 2.f ? 2.f * q : q < 4.f ? q + 2.f : 0.5f * q + 4.f);
    codes |= (c | (__float_as_uint(v[i]) >> 31 << 3)) << (4 * i);
    v[i] = fmaf(-copysignf(q, v[i]), s, v[i]);
  }
  if (nan) {
    codes = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(0x7FC00000u);
  }
  return codes;
}

// Eight values from their codes and scale, added to v.
MSD_DEV void add_values8(uint32_t codes, uint32_t sc, float* v) {
  const float s = sc == 255u ? __uint_as_float(0x7FC00000u) : scale_value(sc);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t c = codes >> (4 * i) & 7u;
    const float q = c < 4u ? 0.5f * c : c < 6u ? c - 2.f : 2.f * c - 8.f;
    v[i] += (codes >> (4 * i) & 8u ? -q : q) * s;
  }
}

// Where a lane's eight columns from k0 of a row of the rows layout lie.
struct RowsOut {
  uint8_t* codes;
  uint8_t* scales;
  int term_codes, term_scales;  // bytes of a row per term
  int terms;
};

MSD_DEV int scale_at(int b) { return (b >> 4) * 16 + (b & 3) * 4 + ((b >> 2) & 3); }

MSD_DEV void put_rows(const RowsOut& o, size_t row, int k0, float* v) {
  for (int t = 0; t < o.terms; ++t) {
    uint32_t sc;
    const uint32_t c = quantise8(v, &sc);
    if (k0 / 2 < o.term_codes)
      *reinterpret_cast<uint32_t*>(o.codes + (row * o.terms + t) * o.term_codes + k0 / 2) = c;
    if (!(threadIdx.x & 3))
      o.scales[(row * o.terms + t) * o.term_scales + scale_at(k0 / BLK)] = (uint8_t)sc;
  }
}

// ------------------------------------------------------------ quantise ----
// A float matrix [rows][cols] whose rows lie ld values apart; or a bf16 weight
// in the packed order of k_gemm.hip, or split rows (MX_SPLIT: hi, then lo).
struct Source {
  const void* p;
  size_t ld;
  int cols;
  bool vec;
  int nkt;  // 128-column blocks (packed)
};

template <int TYPE>
MSD_DEV void load_src(const Source& s, size_t row, int k0, float* v) {
  if constexpr (TYPE == MX_PACKED) {
    const size_t blk = (row >> 6) * s.nkt + (k0 >> 7);
    const size_t unit = (((row >> 4) & 3) * 4 + ((k0 >> 3) & 3)) * 64 + (row & 15) + 16 * ((k0 >> 5) & 3);
    load8<MX_BF16>(s.p, blk * 8192 + unit * 8, 8, true, v);
  } else if constexpr (TYPE == MX_SPLIT) {
    float lo[8];
    load8<MX_BF16>(s.p, row * s.ld + k0, s.cols - k0, s.vec, v);
    load8<MX_BF16>(s.p, row * s.ld + s.cols + k0, s.cols - k0, s.vec, lo);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += lo[i];
  } else {
    load8<TYPE>(s.p, row * s.ld + k0, s.cols - k0, s.vec, v);
  }
}

// Rows layout: a wave takes 512 columns of a row, a lane eight.
template <int TYPE>
__global__ __launch_bounds__(256) void k_mx_rows(Source s, int rows, int groups, RowsOut o) {
  const size_t w = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const size_t row = w / groups;
  if (row >= (size_t)rows) return;
  const int k0 = (int)(w - row * groups) * GROUP + (threadIdx.x & 63) * 8;
  float v[8];
  load_src<TYPE>(s, row, k0, v);
  put_rows(o, row, k0, v);
}

// Weight layout: a workgroup takes 16 rows of 512 columns, a lane eight columns
// of a row in each of the four tiles, so that it has its dword of scales.
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
      *reinterpret_cast<uint32_t*>(codes + (t * nkt + kt) * TILE_BYTES + ((c >> 2) * 16 + r) * 16 +
                                   (c & 3) * 4) = q;
  }
  if (!(c & 3)) scales[(t * groups + g) * 64 + (c >> 2) * 16 + r] = sc4;
}

// ---------------------------------------------------------- dequantise ----
template <int TYPE, bool WEIGHT>
__global__ __launch_bounds__(256) void k_mx_values(const uint8_t* codes, const uint8_t* scales,
                                                   int terms, int rows, int cols, int units,
                                                   int nkt, int groups, void* out, size_t ld,
                                                   bool vec) {
  const size_t q = (size_t)blockIdx.x * 256 + threadIdx.x;
  const size_t row = q / units;
  if (row >= (size_t)rows) return;
  const int k0 = (int)(q - row * units) * 8;
  const int b = k0 / BLK;
  float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int t = 0; t < terms; ++t) {
    uint32_t c, sc;
    if constexpr (WEIGHT) {
      const size_t tile = row / 16;
      const int lane = (b & 3) * 16 + (int)(row & 15), kt = k0 / KT;
      c = *reinterpret_cast<const uint32_t*>(codes + (tile * nkt + kt) * TILE_BYTES + lane * 16 +
                                             (k0 & 31) / 2);
      sc = scales[(tile * groups + kt / 4) * 256 + lane * 4 + (kt & 3)];
    } else {
      c = *reinterpret_cast<const uint32_t*>(codes + (row * terms + t) * (size_t)(nkt * KT / 2) + k0 / 2);
      sc = scales[(row * terms + t) * (size_t)(groups * 16) + scale_at(b)];
    }
    add_values8(c, sc, v);
  }
  store8<TYPE>(out, row * ld + k0, cols - k0, vec, v);
}

// ---------------------------------------------------------------- norm ----
// One workgroup per row, the row's sum in registers between its two uses.  The
// mean square and the scaling are in float64: 4-bit values change with the last
// bit of what is rounded to them, and the operator is bound by memory.
constexpr int NORM_THREADS = 256;
template <int TYPE, int CH>
__global__ __launch_bounds__(NORM_THREADS) void k_mx_norm(const void* x, size_t ldx, const void* y,
                                                          size_t ldy, void* xo, size_t ldo,
                                                          const uint16_t* gain, int d, double eps,
                                                          bool vec, bool gvec, RowsOut o) {
  __shared__ double sh[NORM_THREADS / 64];
  const size_t row = blockIdx.x;
  float v[CH][8];
  double ss = 0.0;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int k0 = (c * NORM_THREADS + (int)threadIdx.x) * 8, n = d - k0;
    load8<TYPE>(x, row * ldx + k0, n, vec, v[c]);
    if (y) {
      float u[8];
      load8<TYPE>(y, row * ldy + k0, n, vec, u);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c][i] += u[i];
    }
    if (xo) store8<TYPE>(xo, row * ldo + k0, n, vec, v[c]);
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fma((double)v[c][i], (double)v[c][i], ss);
  }
  for (int k = 32; k > 0; k >>= 1) ss += __shfl_xor(ss, k);
  if (!(threadIdx.x & 63)) sh[threadIdx.x >> 6] = ss;
  __syncthreads();
  ss = 0.0;
#pragma unroll
  for (int w = 0; w < NORM_THREADS / 64; ++w) ss += sh[w];
  const double r = 1.0 / sqrt(ss / d + eps);
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int k0 = (c * NORM_THREADS + (int)threadIdx.x) * 8;
    if (k0 / 8 / 64 * 64 * 8 >= o.term_scales * BLK) continue;  // a wave past the last group
    float g[8];
    load8<MX_BF16>(gain, k0, d - k0, gvec, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[c][i] = (float)((double)v[c][i] * r * (double)g[i]);
    put_rows(o, row, k0, v[c]);
  }
}

// -------------------------------------------------------------- swiglu ----
template <int TYPE>
__global__ __launch_bounds__(256) void k_mx_swiglu(const void* gate, const void* up, size_t ldg,
                                                   size_t ldu, int rows, int F, int groups,
                                                   bool vec, RowsOut o) {
  const size_t w = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const size_t row = w / groups;
  if (row >= (size_t)rows) return;
  const int k0 = (int)(w - row * groups) * GROUP + (threadIdx.x & 63) * 8;
  float g[8], u[8];
  load8<TYPE>(gate, row * ldg + k0, F - k0, vec, g);
  load8<TYPE>(up, row * ldu + k0, F - k0, vec, u);
#pragma unroll
  for (int i = 0; i < 8; ++i) g[i] = g[i] / (1.f + expf(-g[i])) * u[i];
  put_rows(o, row, k0, g);
}

// ------------------------------------------------------------- product ----
struct ProductArgs {
  const uint8_t *xc, *xs;  // rows layout
  const uint8_t *wc, *ws;  // weight layout
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
// products of X row l % 16 and W rows 4 (l / 16) .. + 3.  The scales are the low
// bytes of ws and xs.
MSD_DEV f32x4 mfma_mx(i32x4 w, i32x4 x, f32x4 acc, int ws, int xs) {
  const i32x8 w8 = __builtin_shufflevector(w, w, 0, 1, 2, 3, -1, -1, -1, -1);
  const i32x8 x8 = __builtin_shufflevector(x, x, 0, 1, 2, 3, -1, -1, -1, -1);
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w8, x8, acc, 4, 4, 0, ws, 0, xs);
}

// Few rows: a workgroup takes 16 columns and 16 MT rows, its waves the groups of
// K in turn; their sums meet in LDS and are added in the order of the waves.
template <int MT, int TX, int NW, int TYPE>
__global__ __launch_bounds__(64 * NW) void k_mx_product(ProductArgs a) {
  __shared__ f32x4 sh[NW][MT][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned tiles = (a.N + 15) / 16;
  const int m0 = (int)(blockIdx.x / tiles) * 16 * MT;
  const size_t tile = blockIdx.x % tiles;
  const int term_c = a.nkt * (KT / 2), term_s = a.groups * 16;
  const uint8_t* wc = a.wc + tile * a.nkt * TILE_BYTES + lane * 16;
  const uint8_t* ws = a.ws + tile * a.groups * 256 + lane * 4;
  const uint8_t *xc[MT], *xs[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    // rows past the last repeat it; their sums are not stored
    const size_t row = min(m0 + m * 16 + (lane & 15), a.M - 1);
    xc[m] = a.xc + row * TX * term_c + (lane >> 4) * 16;
    xs[m] = a.xs + row * TX * term_s + (lane >> 4) * 4;
  }
  f32x4 acc[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) acc[m] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int g = wave; g < a.groups; g += NW) {
    const int sw = *reinterpret_cast<const int*>(ws + (size_t)g * 256);
    int sx[MT][TX];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int t = 0; t < TX; ++t)
        sx[m][t] = *reinterpret_cast<const int*>(xs[m] + t * term_s + g * 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int kt = g * 4 + j;
      if (kt >= a.nkt) break;
      const i32x4 w = *reinterpret_cast<const i32x4*>(wc + (size_t)kt * TILE_BYTES);
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int t = 0; t < TX; ++t) {
          const i32x4 x = *reinterpret_cast<const i32x4*>(xc[m] + t * term_c + kt * (KT / 2));
          acc[m] = mfma_mx(w, x, acc[m], sw >> (8 * j), sx[m][t] >> (8 * j));
        }
    }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m) sh[wave][m][lane] = acc[m];
  __syncthreads();
  for (int u = threadIdx.x; u < MT * 64; u += 64 * NW) {
    const int m = u >> 6, l = u & 63;
    f32x4 v = sh[0][m][l];
#pragma unroll
    for (int w = 1; w < NW; ++w) v += sh[w][m][l];
    const int row = m0 + m * 16 + (l & 15), n = (int)tile * 16 + (l >> 4) * 4;
    if (row < a.M && n < a.N) store4<TYPE>(a, row, n, v);
  }
}

RowsOut rows_out(const MxMat& q) {
  return {static_cast<uint8_t*>(q.codes), static_cast<uint8_t*>(q.scales), mx_tiles(q.cols) * KT / 2,
          mx_groups(q.cols) * 16, q.terms};
}

unsigned wave_blocks(int rows, int groups) {
  return (unsigned)(((size_t)rows * groups + 3) / 4);
}

// Whether rows of values of `size` bytes take 16-byte accesses.
bool rows_aligned(const void* p, size_t ld, int size) {
  return !((uintptr_t)p & 15) && !(ld * size & 15);
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
  const int groups = mx_groups(q.cols);
  Source s{src, ld, q.cols, false, mx_tiles(q.cols)};
  s.vec = rows_aligned(src, ld, type == MX_F32 ? 4 : 2);
  if (type == MX_SPLIT) s.vec = s.vec && q.cols % 8 == 0;
  if (q.weight) {
    const unsigned grid = (unsigned)((size_t)((q.rows + 15) / 16) * groups);
    const auto go = [&](auto k) {
      hipLaunchKernelGGL(k, dim3(grid), dim3(256), 0, st, s, q.rows, groups, mx_tiles(q.cols),
                         static_cast<uint8_t*>(q.codes), static_cast<uint32_t*>(q.scales));
    };
    if (type == MX_PACKED) go(k_mx_weight<MX_PACKED>);
    else if (type == MX_F32) go(k_mx_weight<MX_F32>);
    else if (type == MX_BF16) go(k_mx_weight<MX_BF16>);
    else go(k_mx_weight<MX_F16>);
  } else {
    const auto go = [&](auto k) {
      hipLaunchKernelGGL(k, dim3(wave_blocks(q.rows, groups)), dim3(256), 0, st, s, q.rows, groups,
                         rows_out(q));
    };
    if (type == MX_SPLIT) go(k_mx_rows<MX_SPLIT>);
    else if (type == MX_F32) go(k_mx_rows<MX_F32>);
    else if (type == MX_BF16) go(k_mx_rows<MX_BF16>);
    else go(k_mx_rows<MX_F16>);
  }
}

void launch_mx_dequantise(const MxMat& q, void* dst, int type, size_t ld, hipStream_t st) {
  if (q.rows <= 0) return;
  const int units = (q.cols + 7) / 8;
  const dim3 grid((unsigned)(((size_t)q.rows * units + 255) / 256));
  const bool vec = rows_aligned(dst, ld, type_size(type));
#define GO(T)                                                                                      \
  do {                                                                                             \
    if (q.weight)                                                                                  \
      hipLaunchKernelGGL((k_mx_values<T, true>), grid, dim3(256), 0, st, (const uint8_t*)q.codes,  \
                         (const uint8_t*)q.scales, 1, q.rows, q.cols, units, mx_tiles(q.cols),     \
                         mx_groups(q.cols), dst, ld, vec);                                         \
    else                                                                                           \
      hipLaunchKernelGGL((k_mx_values<T, false>), grid, dim3(256), 0, st, (const uint8_t*)q.codes, \
                         (const uint8_t*)q.scales, q.terms, q.rows, q.cols, units,                 \
                         mx_tiles(q.cols), mx_groups(q.cols), dst, ld, vec);                       \
  } while (0)
  MX_TYPES(type, GO);
#undef GO
}

void launch_mx_norm(const void* x, size_t ldx, const void* y, size_t ldy, void* xo, size_t ldo,
                    int type, const uint16_t* gain, float eps, const MxMat& q, hipStream_t st) {
  if (q.rows <= 0) return;
  const int sz = type_size(type), d = q.cols;
  const bool vec = rows_aligned(x, ldx, sz) && (!y || rows_aligned(y, ldy, sz)) &&
                   (!xo || rows_aligned(xo, ldo, sz));
  const bool gvec = !((uintptr_t)gain & 15);
  const RowsOut o = rows_out(q);
  const auto go = [&](auto k) {
    hipLaunchKernelGGL(k, dim3(q.rows), dim3(NORM_THREADS), 0, st, x, ldx, y, ldy, xo, ldo, gain, d,
                       (double)eps, vec, gvec, o);
  };
  const int per = NORM_THREADS * 8;
#define GO(T)                                \
  do {                                       \
    if (d <= per) go(k_mx_norm<T, 1>);       \
    else if (d <= 2 * per) go(k_mx_norm<T, 2>); \
    else go(k_mx_norm<T, 4>);                \
  } while (0)
  MX_TYPES(type, GO);
#undef GO
}

void launch_mx_swiglu(const void* gate, size_t ldg, const void* up, size_t ldu, int type,
                      const MxMat& q, hipStream_t st) {
  if (q.rows <= 0) return;
  const int groups = mx_groups(q.cols), sz = type_size(type);
  const bool vec = rows_aligned(gate, ldg, sz) && rows_aligned(up, ldu, sz);
#define GO(T)                                                                                    \
  hipLaunchKernelGGL((k_mx_swiglu<T>), dim3(wave_blocks(q.rows, groups)), dim3(256), 0, st, gate, \
                     up, ldg, ldu, q.rows, q.cols, groups, vec, rows_out(q))
  MX_TYPES(type, GO);
#undef GO
}

void launch_mx_product(const MxMat& x, const MxMat& w, void* out, int type, size_t ldo,
                       hipStream_t st) {
  if (x.rows <= 0 || w.rows <= 0) return;
  ProductArgs a{static_cast<const uint8_t*>(x.codes), static_cast<const uint8_t*>(x.scales),
                static_cast<const uint8_t*>(w.codes), static_cast<const uint8_t*>(w.scales),
                x.rows, w.rows, mx_tiles(w.cols), mx_groups(w.cols), out, ldo, false};
  const int sz = type_size(type);
  a.vec = !((uintptr_t)out & (4 * sz - 1)) && ldo % 4 == 0;
  const int MT = x.rows <= 16 ? 1 : 4;
  const dim3 grid((unsigned)((w.rows + 15) / 16) * ((x.rows + 16 * MT - 1) / (16 * MT)));
  constexpr int NW = 8;
  const auto go = [&](auto k) { hipLaunchKernelGGL(k, grid, dim3(64 * NW), 0, st, a); };
#define GO(T)                                              \
  do {                                                     \
    if (x.terms == 2) {                                    \
      if (MT == 1) go(k_mx_product<1, 2, NW, T>);          \
      else go(k_mx_product<4, 2, NW, T>);                  \
    } else {                                               \
      if (MT == 1) go(k_mx_product<1, 1, NW, T>);          \
      else go(k_mx_product<4, 1, NW, T>);                  \
    }                                                      \
  } while (0)
  MX_TYPES(type, GO);
#undef GO
}

}  // namespace msd
