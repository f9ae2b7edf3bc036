// Operators on rows of logits: the largest of a row, the choice of tokens under a
// temperature, top-k, top-p and min-p (drawn from, or written back as logits), and
// distillation from a teacher's top logits with its gradient.
//
// A row's tokens are ranked by value, then by id (lowest first); a NaN counts as -inf.
// Everything that is kept under top-k, top-p and min-p is a prefix of that order, so
// one threshold (a key, and how many of the tokens that share it) describes it.  Keys
// are the values' bits made to ascend with them.  The threshold is found digit by
// digit from histograms of counts (top-k) or of weights (top-p).
//
// Weights exp((x - max) / T) decide which token lies next to a border, so they are
// computed in 64 bits and held as whole numbers of 2^-45: at most 2^18 of them sum
// exactly, in any order.
#include <hip/hip_fp16.h>

#include "msd_internal.h"

namespace msd {

namespace {

constexpr int LB = 1024;  // threads of a row
constexpr int LW = LB / 64;
constexpr uint32_t KEY_NINF = 0x007FFFFFu;  // the key of -inf; no key is smaller

template <int TYPE>
MSD_DEV float value_at(const void* p, size_t i) {
  if constexpr (TYPE == MX_F32) return static_cast<const float*>(p)[i];
  const uint16_t h = static_cast<const uint16_t*>(p)[i];
  if constexpr (TYPE == MX_BF16) return bf2f(h);
  return __half2float(__builtin_bit_cast(__half, h));
}

template <int TYPE>
MSD_DEV void put_at(void* p, size_t i, float v) {
  if constexpr (TYPE == MX_F32)
    static_cast<float*>(p)[i] = v;
  else if constexpr (TYPE == MX_BF16)
    static_cast<uint16_t*>(p)[i] = f2bf(v);
  else
    static_cast<uint16_t*>(p)[i] = __builtin_bit_cast(uint16_t, __float2half(v));
}

template <int TYPE>
MSD_DEV const void* row_of(const void* p, size_t ld) {
  return static_cast<const char*>(p) + (size_t)blockIdx.x * ld * (TYPE == MX_F32 ? 4 : 2);
}

MSD_DEV uint32_t key_of(float x) {
  if (!(x > -INFINITY)) return KEY_NINF;
  const uint32_t u = __float_as_uint(x + 0.f);  // -0 ranks as 0
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
MSD_DEV float of_key(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}

struct Lds {
  uint64_t hist[2048];
  uint64_t part[LW];
  uint32_t key[LW];
  uint64_t found[2];
  int bin;
};

MSD_DEV uint64_t block_sum(uint64_t v, Lds& s) {
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor((unsigned long long)v, o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s.part[threadIdx.x >> 6] = v;
  __syncthreads();
  uint64_t t = 0;
  for (int i = 0; i < LW; ++i) t += s.part[i];
  return t;
}

MSD_DEV double block_sum(double v, Lds& s) {
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s.part[threadIdx.x >> 6] = __double_as_longlong(v);
  __syncthreads();
  double t = 0;
  for (int i = 0; i < LW; ++i) t += __longlong_as_double((long long)s.part[i]);
  return t;
}

// The sum over the threads before this one.
MSD_DEV uint64_t block_before(uint64_t v, Lds& s) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  uint64_t in = v;
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t y = __shfl_up((unsigned long long)in, o);
    if (lane >= o) in += y;
  }
  __syncthreads();
  if (lane == 63) s.part[w] = in;
  __syncthreads();
  uint64_t before = in - v;
  for (int i = 0; i < w; ++i) before += s.part[i];
  return before;
}

MSD_DEV uint32_t block_max(uint32_t v, Lds& s) {
  for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s.key[threadIdx.x >> 6] = v;
  __syncthreads();
  uint32_t t = 0;
  for (int i = 0; i < LW; ++i) t = max(t, s.key[i]);
  return t;
}

// Whole number of 2^-45 next to exp((x - m) / T), c = log2(e) / T.
constexpr double ONE = 0x1p45;
MSD_DEV uint64_t weight(float x, float m, double c) {
  if (!(x > -INFINITY)) return 0;
  if (x == m) return (uint64_t)ONE;
  return (uint64_t)rint(exp2(((double)x - (double)m) * c) * ONE);
}

// What is kept of a row: keys above `key`, and of those equal to it the ids up to
// `last`.
struct Kept {
  uint32_t key;
  int last;
};
MSD_DEV bool in(Kept k, uint32_t key, int id) {
  return key > k.key || (key == k.key && id <= k.last);
}

// The shortest prefix of the ranked row whose counts (c == 0) or weights sum to at
// least `want` (1 <= want <= their sum).
template <int TYPE>
MSD_DEV Kept shortest(const void* x, int V, float m, double c, uint64_t want, Lds& s) {
  uint32_t prefix = 0;  // the digits found so far
  int left = 32;        // bits below them
  uint64_t ties = 0, each = 1;
  while (left > 0) {
    const int bits = left > 11 ? 11 : left;
    const int low = left - bits;
    __syncthreads();
    for (int i = threadIdx.x; i < 2048; i += LB) s.hist[i] = 0;
    __syncthreads();
    for (int v = threadIdx.x; v < V; v += LB) {
      const float z = value_at<TYPE>(x, v);
      const uint32_t k = key_of(z);
      if (left < 32 && (k ^ prefix) >> left) continue;
      const uint64_t w = c == 0 ? 1 : weight(z, m, c);
      if (w) atomicAdd((unsigned long long*)&s.hist[(k >> low) & ((1u << bits) - 1)], w);
    }
    __syncthreads();
    // from the largest digit down, two digits a thread
    const int b1 = 2047 - 2 * threadIdx.x;
    const uint64_t h1 = s.hist[b1], h2 = s.hist[b1 - 1];
    const uint64_t before = block_before(h1 + h2, s);
    if (before < want && want <= before + h1 + h2) {
      const bool second = want > before + h1;
      s.bin = second ? b1 - 1 : b1;
      s.found[0] = second ? before + h1 : before;
      s.found[1] = second ? h2 : h1;
    }
    __syncthreads();
    prefix |= (uint32_t)s.bin << low;
    want -= s.found[0];
    ties = s.found[1];
    left = low;
  }
  if (c != 0) each = weight(of_key(prefix), m, c);
  const uint64_t n = (want + each - 1) / each;  // of the equal ones, at least 1
  if (n * each >= ties) return {prefix, V};
  // the n-th of them in the order of their ids
  uint64_t seen = 0;
  for (int v0 = 0; v0 < V; v0 += LB) {
    const int v = v0 + threadIdx.x;
    const uint64_t hit = v < V && key_of(value_at<TYPE>(x, v)) == prefix;
    const uint64_t before = seen + block_before(hit, s);
    if (hit && before + 1 == n) s.bin = v;
    seen += block_sum(hit, s);
    if (seen >= n) break;
  }
  __syncthreads();
  return {prefix, s.bin};
}

template <int TYPE>
MSD_DEV float row_max(const void* x, int V, Lds& s) {
  uint32_t k = KEY_NINF;
  for (int v = threadIdx.x; v < V; v += LB) k = max(k, key_of(value_at<TYPE>(x, v)));
  return of_key(block_max(k, s));
}

// The tokens that stay (m > -inf).
template <int TYPE>
MSD_DEV Kept choose(const void* x, int V, float m, const LogitsChoice& how, Lds& s) {
  Kept k{KEY_NINF + 1, V};
  if (how.top_k > 0 && how.top_k < V) {
    const Kept t = shortest<TYPE>(x, V, m, 0, how.top_k, s);
    if (t.key > KEY_NINF) k = t;
  }
  if (how.top_p < 1) {
    uint64_t sum = 0;
    for (int v = threadIdx.x; v < V; v += LB) {
      const float z = value_at<TYPE>(x, v);
      if (in(k, key_of(z), v)) sum += weight(z, m, how.c);
    }
    sum = block_sum(sum, s);
    const uint64_t want = (uint64_t)fmax(ceil((double)sum * how.top_p), 1.0);
    const Kept t = shortest<TYPE>(x, V, m, how.c, want < sum ? want : sum, s);
    if (t.key > k.key || (t.key == k.key && t.last < k.last)) k = t;
  }
  if (how.min_d > -INFINITY) {
    // x - m >= T log(min_p): the least such key
    uint32_t least = 0xFFFFFFFFu;
    for (int v = threadIdx.x; v < V; v += LB) {
      const float z = value_at<TYPE>(x, v);
      if (z == m || (double)z - (double)m >= how.min_d) least = min(least, key_of(z));
    }
    least = ~block_max(~least, s);
    if (least > k.key) k = {least, V};
  }
  return k;
}

template <int TYPE>
__global__ __launch_bounds__(LB) void k_filter(const void* logits, size_t ld, int V,
                                               LogitsChoice how, void* out, size_t ldo,
                                               int* kept) {
  __shared__ Lds s;
  const void* x = row_of<TYPE>(logits, ld);
  void* o = const_cast<void*>(row_of<TYPE>(out, ldo));
  const float m = row_max<TYPE>(x, V, s);
  const Kept k = m > -INFINITY ? choose<TYPE>(x, V, m, how, s) : Kept{0xFFFFFFFFu, -1};
  uint64_t n = 0;
  for (int v = threadIdx.x; v < V; v += LB) {
    const float z = value_at<TYPE>(x, v);
    const bool stays = in(k, key_of(z), v);
    put_at<TYPE>(o, v, stays ? z : -INFINITY);
    n += stays;
  }
  n = block_sum(n, s);
  if (kept && threadIdx.x == 0) kept[blockIdx.x] = (int)n;
}

template <int TYPE>
__global__ __launch_bounds__(LB) void k_sample(const void* logits, size_t ld, int V,
                                               LogitsChoice how, const float* uniforms, int* tokens,
                                               float* logprobs) {
  __shared__ Lds s;
  const void* x = row_of<TYPE>(logits, ld);
  const float m = row_max<TYPE>(x, V, s);
  if (!(m > -INFINITY)) {
    if (threadIdx.x == 0) {
      tokens[blockIdx.x] = -1;
      if (logprobs) logprobs[blockIdx.x] = -INFINITY;
    }
    return;
  }
  const Kept k = choose<TYPE>(x, V, m, how, s);
  // each thread sums a stretch of ids
  const int per = (V + LB - 1) / LB;
  const int v0 = min(V, (int)threadIdx.x * per), v1 = min(V, v0 + per);
  uint64_t part = 0;
  for (int v = v0; v < v1; ++v) {
    const float z = value_at<TYPE>(x, v);
    if (in(k, key_of(z), v)) part += weight(z, m, how.c);
  }
  const uint64_t before = block_before(part, s);
  const uint64_t total = block_sum(part, s);
  const float u = uniforms[blockIdx.x];
  // the first id whose running sum is above u times the total
  const uint64_t at = u >= 1.f ? total - 1 : u > 0.f ? (uint64_t)((double)u * (double)total) : 0;
  if (before <= at && at < before + part) {
    uint64_t run = before;
    for (int v = v0; v < v1; ++v) {
      const float z = value_at<TYPE>(x, v);
      if (!in(k, key_of(z), v)) continue;
      run += weight(z, m, how.c);
      if (run <= at) continue;
      tokens[blockIdx.x] = v;
      if (logprobs)
        logprobs[blockIdx.x] =
            (float)((z == m ? 0.0 : ((double)z - (double)m) * how.c * 0.69314718055994530942) -
                    log((double)total * (1 / ONE)));
      break;
    }
  }
}

template <int TYPE>
__global__ __launch_bounds__(LB) void k_top(const void* logits, size_t ld, int V, int n,
                                            float* values, int* ids, float* lse) {
  __shared__ Lds s;
  __shared__ uint64_t list[LOGITS_TOP_MAX];
  __shared__ int count;
  const void* x = row_of<TYPE>(logits, ld);
  if (threadIdx.x == 0) count = 0;
  const float m = row_max<TYPE>(x, V, s);
  const Kept k = shortest<TYPE>(x, V, m, 0, n, s);
  double sum = 0;
  for (int v = threadIdx.x; v < V; v += LB) {
    const float z = value_at<TYPE>(x, v);
    const uint32_t key = key_of(z);
    // a place among them: by the key, then by the lower id
    if (in(k, key, v)) list[atomicAdd(&count, 1)] = ((uint64_t)key << 32) | (uint32_t)~v;
    if (z == m)
      sum += 1;
    else if (z > -INFINITY)
      sum += exp((double)z - (double)m);
  }
  sum = block_sum(sum, s);
  if (threadIdx.x < n) {
    const uint64_t mine = list[threadIdx.x];
    int rank = 0;
    for (int i = 0; i < n; ++i) rank += list[i] > mine;
    const size_t o = (size_t)blockIdx.x * n + rank;
    values[o] = of_key((uint32_t)(mine >> 32));
    ids[o] = (int)~(uint32_t)mine;
  }
  if (lse && threadIdx.x == 0)
    lse[blockIdx.x] = fabsf(m) < INFINITY ? (float)((double)m + log(sum)) : m;
}

// A row's teacher entry of this thread (id < 0: none).
struct Entry {
  int id;
  double lq, q;
};

// q = softmax(t / T) over the row's entries; all zero where none has a value above
// -inf, NaN where one is NaN or +inf.
MSD_DEV Entry teacher_entry(const LogitsTeacher& t, int V, Lds& s) {
  Entry e{-1, 0, 0};
  float z = -INFINITY;
  if (threadIdx.x < (unsigned)t.k) {
    const size_t o = (size_t)blockIdx.x * t.k + threadIdx.x;
    e.id = t.ids[o];
    if (e.id < 0 || e.id >= V) e.id = -1;
    if (e.id >= 0) z = t.values[o];
  }
  const float top = of_key(block_max(key_of(z), s));
  const double d = ((double)z - (double)top) * t.inv_t;
  const double w = z == -INFINITY ? 0 : exp(d);
  const double sum = block_sum(w, s);
  if (w != 0) {
    e.lq = d - log(sum);
    e.q = w / sum;
  }
  return e;
}

template <int TYPE>
__global__ __launch_bounds__(LB) void k_distill(const void* logits, size_t ld, int V,
                                                LogitsTeacher t, float* loss, float* lse,
                                                const float* grad, void* dx, size_t ldd) {
  __shared__ Lds s;
  __shared__ int sid[LOGITS_TOP_MAX];
  __shared__ double sq[LOGITS_TOP_MAX];
  const void* x = row_of<TYPE>(logits, ld);
  const Entry e = teacher_entry(t, V, s);
  // the entry's logit, before a gradient in the logits' place is written
  const float zk = e.id >= 0 ? value_at<TYPE>(x, e.id) : 0.f;
  float m = -INFINITY;
  for (int v = threadIdx.x; v < V; v += LB) m = fmaxf(m, value_at<TYPE>(x, v));
  m = of_key(block_max(key_of(m), s));
  double sum = 0;
  for (int v = threadIdx.x; v < V; v += LB)
    sum += exp(((double)value_at<TYPE>(x, v) - (double)m) * t.inv_t);
  sum = block_sum(sum, s);
  const double dk = ((double)zk - (double)m) * t.inv_t;
  if (loss) {
    const double l = block_sum(e.q != 0 ? e.q * (e.lq - (dk - log(sum))) : 0, s);
    if (threadIdx.x == 0) loss[blockIdx.x] = (float)l;
  }
  if (lse && threadIdx.x == 0)
    lse[blockIdx.x] = (float)(m * t.inv_t + log(sum));
  if (!dx) return;
  void* o = const_cast<void*>(row_of<TYPE>(dx, ldd));
  const double mass = block_sum(e.q, s);  // 1 (or NaN); 0 without entries
  const double g = mass == 0 ? 0 : grad[blockIdx.x] * t.inv_t * mass;
  if (threadIdx.x < (unsigned)t.k) {
    sid[threadIdx.x] = e.id;
    sq[threadIdx.x] = e.q;
  }
  for (int v = threadIdx.x; v < V; v += LB) {
    const double p = exp(((double)value_at<TYPE>(x, v) - (double)m) * t.inv_t) / sum;
    put_at<TYPE>(o, v, mass == 0 ? 0.f : (float)(g * p));
  }
  __syncthreads();
  if (e.id < 0 || mass == 0) return;
  // the first entry of an id carries the others'
  double q = 0;
  for (int i = 0; i < t.k; ++i) {
    if (sid[i] != e.id) continue;
    if (i < (int)threadIdx.x) return;
    q += sq[i];
  }
  put_at<TYPE>(o, e.id, (float)(g * (exp(dk) / sum - q)));
}

}  // namespace

#define LOGITS_TYPES(type, K, ...)                                                       \
  do {                                                                                   \
    if (type == MX_F32)                                                                  \
      hipLaunchKernelGGL(K<MX_F32>, dim3(rows), dim3(LB), 0, st, __VA_ARGS__);           \
    else if (type == MX_BF16)                                                            \
      hipLaunchKernelGGL(K<MX_BF16>, dim3(rows), dim3(LB), 0, st, __VA_ARGS__);          \
    else                                                                                 \
      hipLaunchKernelGGL(K<MX_F16>, dim3(rows), dim3(LB), 0, st, __VA_ARGS__);           \
  } while (0)

void launch_logits_top(const void* x, int type, size_t ld, int rows, int cols, int k, float* values,
                       int* ids, float* lse, hipStream_t st) {
  if (rows <= 0) return;
  LOGITS_TYPES(type, k_top, x, ld, cols, k, values, ids, lse);
}

void launch_logits_sample(const void* x, int type, size_t ld, int rows, int cols,
                          const LogitsChoice& how, const float* uniforms, int* tokens,
                          float* logprobs, hipStream_t st) {
  if (rows <= 0) return;
  LOGITS_TYPES(type, k_sample, x, ld, cols, how, uniforms, tokens, logprobs);
}

void launch_logits_filter(const void* x, int type, size_t ld, int rows, int cols,
                          const LogitsChoice& how, void* out, size_t ldo, int* kept,
                          hipStream_t st) {
  if (rows <= 0) return;
  LOGITS_TYPES(type, k_filter, x, ld, cols, how, out, ldo, kept);
}

void launch_logits_distill(const void* x, int type, size_t ld, int rows, int cols,
                           const LogitsTeacher& t, float* loss, float* lse, const float* grad,
                           void* dx, size_t ldd, hipStream_t st) {
  if (rows <= 0) return;
  LOGITS_TYPES(type, k_distill, x, ld, cols, t, loss, lse, grad, dx, ldd);
}

}  // namespace msd
