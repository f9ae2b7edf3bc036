// Operators on rows of logits: the largest of a row, the choice of tokens under a
// temperature, top-k, top-p and min-p (drawn from, or written back as logits), and
// distillation from a teacher's top logits with its gradient.
//
// A row's tokens are ranked by value, then by id (lowest first); a NaN counts as -inf.
// Everything that is kept under top-k, top-p and min-p is a prefix of that order, so
// its last token describes it (Kept).
//
// Weights exp((x - max) / T) decide which token lies next to a border, so they are
// computed in 64 bits and held as whole numbers of 2^-45: 2^18 of them sum exactly, in
// any order, atomics included.
//
// One workgroup a row.
#include <hip/hip_fp16.h>

#include <type_traits>

#include "msd_internal.h"

namespace msd {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// sixteen bytes at the alignment of the elements: rows may begin anywhere
typedef u32x4 u32x4_4 __attribute__((aligned(4)));
typedef u32x4 u32x4_2 __attribute__((aligned(2)));

template <int TYPE>
struct Type {  // 16 bits
  static constexpr int E = 8, SIZE = 2;
  typedef u32x4_2 unit;
  static constexpr uint32_t NINF = TYPE == MX_BF16 ? 0xFF80FF80u : 0xFC00FC00u;  // -inf, twice
};
template <>
struct Type<MX_F32> {
  static constexpr int E = 4, SIZE = 4;
  typedef u32x4_4 unit;
  static constexpr uint32_t NINF = 0xFF800000u;
};

template <int TYPE>
MSD_DEV float from_bits(uint32_t h) {
  if constexpr (TYPE == MX_F32) return __uint_as_float(h);
  if constexpr (TYPE == MX_BF16) return __uint_as_float(h << 16);
  return __half2float(__builtin_bit_cast(__half, (uint16_t)h));
}
template <int TYPE>
MSD_DEV uint32_t to_bits(float v) {
  if constexpr (TYPE == MX_F32) return __float_as_uint(v);
  if constexpr (TYPE == MX_BF16) return f2bf(v);
  return __builtin_bit_cast(uint16_t, __float2half(v));
}
template <int TYPE>
MSD_DEV uint32_t bits_at(const char* p, int i) {
  if constexpr (TYPE == MX_F32) return reinterpret_cast<const uint32_t*>(p)[i];
  return reinterpret_cast<const uint16_t*>(p)[i];
}
template <int TYPE>
MSD_DEV void put_bits(char* p, int i, uint32_t h) {
  if constexpr (TYPE == MX_F32)
    reinterpret_cast<uint32_t*>(p)[i] = h;
  else
    reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)h;
}
// Element e of a unit, and its place.
template <int TYPE>
MSD_DEV uint32_t lift(const u32x4& u, int e) {
  if constexpr (TYPE == MX_F32) return u[e];
  return e & 1 ? u[e / 2] >> 16 : u[e / 2] & 0xFFFFu;
}
template <int TYPE>
MSD_DEV void lower(u32x4& u, int e, uint32_t h) {
  if constexpr (TYPE == MX_F32)
    u[e] = h;
  else
    u[e / 2] = e & 1 ? (u[e / 2] & 0xFFFFu) | h << 16 : (u[e / 2] & 0xFFFF0000u) | h;
}

// A row of V logits over LB threads, in tiles of a unit of 16 bytes each: unit j of a
// thread begins at element (j LB + thread) E; places past V hold -inf.
template <int TYPE, int LB_>
struct Row {
  static constexpr int T = TYPE, LB = LB_, E = Type<TYPE>::E, TILE = LB * E, W = LB / 64;
  typedef typename Type<TYPE>::unit unit;
  const char* p;
  int V;

  MSD_DEV Row(const void* base, size_t ld, int V_)
      : p(static_cast<const char*>(base) + (size_t)blockIdx.x * ld * Type<TYPE>::SIZE), V(V_) {}
  MSD_DEV int id(int j) const { return (j * LB + (int)threadIdx.x) * E; }
  MSD_DEV u32x4 load(int j) const {
    return *reinterpret_cast<const unit*>(p + (size_t)id(j) * Type<TYPE>::SIZE);
  }
  // Of the last tile, where V may end inside a unit.
  MSD_DEV u32x4 load_tail(int j) const {
    const int i = id(j);
    if (i + E <= V) return load(j);
    u32x4 u = Type<TYPE>::NINF;
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (i + e < V) lower<TYPE>(u, e, bits_at<TYPE>(p, i + e));
    return u;
  }
  // f(j, id, unit) for every tile in order, read from memory, AHEAD tiles at a time.
  template <int AHEAD, class F>
  MSD_DEV void each(F f) const {
    const int full = V / TILE, n = (V + TILE - 1) / TILE;
    for (int j = 0; j < n; j += AHEAD) {
      u32x4 t[AHEAD];
#pragma unroll
      for (int b = 0; b < AHEAD; ++b)
        if (j + b < full) t[b] = load(j + b);
      if (full < n && full < j + AHEAD) {
        const u32x4 last = load_tail(full);
#pragma unroll
        for (int b = 0; b < AHEAD; ++b)
          if (j + b == full) t[b] = last;
      }
#pragma unroll
      for (int b = 0; b < AHEAD; ++b)
        if (j + b < n) f(j + b, id(j + b), t[b]);
    }
  }
  MSD_DEV void store(char* o, int i, const u32x4& u) const {
    if (i + E <= V) {
      *reinterpret_cast<unit*>(o + (size_t)i * Type<TYPE>::SIZE) = u;
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (i + e < V) put_bits<TYPE>(o, i + e, lift<TYPE>(u, e));
    }
  }
};

// The same with up to U whole tiles and the last one in registers.
template <int TYPE, int LB, int U>
struct HeldRow : Row<TYPE, LB> {
  typedef Row<TYPE, LB> Base;
  u32x4 r[U], last;
  MSD_DEV HeldRow(const void* base, size_t ld, int V) : Base(base, ld, V) {
    const int full = V / Base::TILE;
#pragma unroll
    for (int j = 0; j < U; ++j) r[j] = j < full ? this->load(j) : u32x4(Type<TYPE>::NINF);
    last = Type<TYPE>::NINF;
    if (V % Base::TILE) last = this->load_tail(full);
  }
  template <int AHEAD, class F>
  MSD_DEV void each(F f) const {
    const int full = this->V / Base::TILE;
#pragma unroll
    for (int j = 0; j < U; ++j)
      if (j < full) f(j, this->id(j), r[j]);
    if (this->V % Base::TILE) f(full, this->id(full), last);
  }
};
template <int TYPE, int LB>
struct HeldRow<TYPE, LB, 0> : Row<TYPE, LB> {  // too long for that
  using Row<TYPE, LB>::Row;
};

// ----------------------------------------------------------- keys and weights ----

constexpr uint32_t KEY_NINF = 0x007FFFFFu;  // the key of -inf; no key is smaller
// Bits that ascend with the value.
MSD_DEV uint32_t key_of(float x) {
  if (!(x > -INFINITY)) return KEY_NINF;
  const uint32_t u = __float_as_uint(x + 0.f);  // -0 ranks as 0
  return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}
MSD_DEV float of_key(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}
// A token's place in the order: the larger, the earlier.
MSD_DEV uint64_t place_of(uint32_t key, int id) { return ((uint64_t)key << 32) | (uint32_t)~id; }

// exp((x - m) / T) as a whole number of 2^-45, to 2^-44 of itself before that rounding;
// c = log2(e) / T.  2^t = 2^k 2^r, r in [-1/2, 1/2], and 2^r = 1 + r q(r) with q the
// Chebyshev interpolation of (2^r - 1) / r of degree 8 (3.7e-14 off at most).
constexpr double ONE = 0x1p45;
struct Scale {
  double m, c;
  bool finite;  // an infinite maximum leaves itself alone
};
MSD_DEV uint64_t weight(float x, const Scale& s) {
  if (!s.finite) return x == (float)s.m ? (uint64_t)ONE : 0;
  const double t = fmax(((double)x - s.m) * s.c, -64.0);  // (a NaN too)
  const double k = t + 0x1.8p52;                          // rounded in its last bits
  const double r = t - (k - 0x1.8p52);
  double q = 0x1.b63880a30e9ffp-24;
  q = fma(q, r, 0x1.63d136366db24p-20);
  q = fma(q, r, 0x1.ffcb9515a8016p-17);
  q = fma(q, r, 0x1.4308ac85aa947p-13);
  q = fma(q, r, 0x1.5d87fe86fe88ep-10);
  q = fma(q, r, 0x1.3b2ab7181b755p-7);
  q = fma(q, r, 0x1.c6b08d7047e52p-5);
  q = fma(q, r, 0x1.ebfbdff823cedp-3);
  q = fma(q, r, 0x1.62e42fefa39efp-1);
  q = fma(q, r, 1.0);
  const double w = __builtin_amdgcn_ldexp(q, (int)__double2loint(k));
  // the last bit of a double in [128, 256) is 2^-45
  return (uint64_t)(__double_as_longlong(w + 128.0) - 0x4060000000000000ll);
}

// ------------------------------------------------------- waves and workgroups ----

// v of the lanes `ctrl` names, `none` where there is none (data-parallel primitives).
template <int CTRL, int ROWS>
MSD_DEV uint32_t dpp(uint32_t v, uint32_t none) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, CTRL, ROWS, 0xF, false);
}
template <int CTRL, int ROWS>
MSD_DEV uint64_t dpp(uint64_t v, uint64_t none) {
  return ((uint64_t)dpp<CTRL, ROWS>((uint32_t)(v >> 32), (uint32_t)(none >> 32)) << 32) |
         dpp<CTRL, ROWS>((uint32_t)v, (uint32_t)none);
}
template <int CTRL, int ROWS>
MSD_DEV double dpp(double v, double none) {
  return __longlong_as_double((long long)dpp<CTRL, ROWS>(
      (uint64_t)__double_as_longlong(v), (uint64_t)__double_as_longlong(none)));
}
// Inclusive over the lanes before; the last lane has the whole.
template <class V, class F>
MSD_DEV V wave_scan(V v, V none, F f) {
  v = f(v, dpp<0x111, 0xF>(v, none));  // from 1, 2, 4 and 8 lanes before, in rows of 16
  v = f(v, dpp<0x112, 0xF>(v, none));
  v = f(v, dpp<0x114, 0xF>(v, none));
  v = f(v, dpp<0x118, 0xF>(v, none));
  v = f(v, dpp<0x142, 0xA>(v, none));  // the last of a row to rows 1 and 3
  v = f(v, dpp<0x143, 0xC>(v, none));  // lane 31 to rows 2 and 3
  return v;
}
struct Sum {
  template <class V>
  MSD_DEV V operator()(V a, V b) const {
    return a + b;
  }
};
struct Max {
  MSD_DEV uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; }
};

constexpr int LISTED = 1024;  // tokens that are ranked among each other
constexpr int BINS = 2048;
constexpr int SLOTS = 4;
struct Lds {
  uint64_t hist[BINS];    // also the weights of a list, and sums of a row's stretches
  uint64_t list[LISTED];
  uint64_t sorted[LOGITS_TOP_MAX];
  int rank[LISTED];
  uint64_t part[SLOTS][16];
  uint64_t found[2];
  int bin, count;
};

// Reductions over the workgroup; each writes another slot, so that one barrier does.
template <int W>
struct Group {
  Lds& s;
  int turn = 0;
  MSD_DEV uint64_t* swap(uint64_t of_last_lane) {
    uint64_t* const p = s.part[turn];
    turn = (turn + 1) % SLOTS;
    if ((threadIdx.x & 63) == 63) p[threadIdx.x >> 6] = of_last_lane;
    lds_barrier();
    return p;
  }
  MSD_DEV uint32_t max(uint32_t v) {
    const uint64_t* p = swap(wave_scan(v, 0u, Max()));
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) t = Max()(t, (uint32_t)p[i]);
    return t;
  }
  MSD_DEV uint64_t sum(uint64_t v) {
    const uint64_t* p = swap(wave_scan(v, (uint64_t)0, Sum()));
    uint64_t t = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) t += p[i];
    return t;
  }
  MSD_DEV double sum(double v) {
    const uint64_t* p = swap((uint64_t)__double_as_longlong(wave_scan(v, 0.0, Sum())));
    double t = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) t += __longlong_as_double((long long)p[i]);
    return t;
  }
  // The sum over the threads before this one, and the whole.
  MSD_DEV uint64_t before(uint64_t v, uint64_t* all) {
    const uint64_t in = wave_scan(v, (uint64_t)0, Sum());
    const uint64_t* p = swap(in);
    uint64_t b = in - v, t = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      if (i == (int)(threadIdx.x >> 6)) b += t;
      t += p[i];
    }
    *all = t;
    return b;
  }
};

// The last token that is kept of a row.
struct Kept {
  uint32_t key;
  int id;
};
struct Keeps {  // the same as values
  float x;
  int id;
  MSD_DEV explicit Keeps(Kept k) : x(of_key(k.key)), id(k.id) {}
  MSD_DEV bool operator()(float v, int i) const { return v > x || (v == x && i <= id); }
};

// ------------------------------------------------------------------ thresholds ----

// The bin of s.hist in which the running sum reaches `want`, with the sum before it and
// its own in s.found.  Bins ascend from bin 0 on, or descend from the last.
template <int W, bool DOWN>
MSD_DEV void find_bin(uint64_t want, Group<W>& g) {
  Lds& s = g.s;
  constexpr int PER = BINS / (W * 64);
  uint64_t h[PER], sum = 0, all;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int b = threadIdx.x * PER + i;
    sum += h[i] = s.hist[DOWN ? BINS - 1 - b : b];
  }
  uint64_t run = g.before(sum, &all);
  if (run < want && want <= run + sum) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (run < want && want <= run + h[i]) {
        const int b = threadIdx.x * PER + i;
        s.bin = DOWN ? BINS - 1 - b : b;
        s.found[0] = run;
        s.found[1] = h[i];
      }
      run += h[i];
    }
  }
  lds_barrier();
}

template <int W>
MSD_DEV void clear_bins(Lds& s) {
  lds_barrier();
  for (int i = threadIdx.x; i < BINS; i += W * 64) s.hist[i] = 0;
  lds_barrier();
}

// The shortest prefix of the ranked row whose counts (null) or weights sum to at least
// `want` (1 <= want <= their sum), digit by digit of the keys: for any row.
template <class R>
MSD_DEV Kept shortest(const R& row, const Scale* sc, uint64_t want, Group<R::W>& g) {
  Lds& s = g.s;
  uint32_t prefix = 0;  // the digits found so far
  int left = 32;        // bits below them
  uint64_t ties = 0, each = 1;
  while (left > 0) {
    const int bits = left > 11 ? 11 : left;
    const int low = left - bits;
    clear_bins<R::W>(s);
    row.template each<4>([&](int, int i, const u32x4& u) {
#pragma unroll
      for (int e = 0; e < R::E; ++e) {
        const float x = from_bits<R::T>(lift<R::T>(u, e));
        const uint32_t k = key_of(x);
        if (i + e >= row.V || (left < 32 && (k ^ prefix) >> left)) continue;
        const uint64_t w = sc ? weight(x, *sc) : 1;
        if (w) atomicAdd((unsigned long long*)&s.hist[(k >> low) & ((1u << bits) - 1)], w);
      }
    });
    lds_barrier();
    find_bin<R::W, true>(want, g);
    prefix |= (uint32_t)s.bin << low;
    want -= s.found[0];
    ties = s.found[1];
    left = low;
  }
  if (sc) each = weight(of_key(prefix), *sc);
  const uint64_t n = (want + each - 1) / each;  // of the equal ones, at least 1
  if (n * each >= ties) return {prefix, row.V};
  // the n-th of them in the order of their ids
  uint64_t seen = 0;
  row.template each<4>([&](int, int i, const u32x4& u) {
    if (seen >= n) return;
    int hits = 0;
#pragma unroll
    for (int e = 0; e < R::E; ++e)
      hits += i + e < row.V && key_of(from_bits<R::T>(lift<R::T>(u, e))) == prefix;
    uint64_t all;
    uint64_t before = seen + g.before(hits, &all);
    seen += all;
    if (before >= n || before + hits < n) return;
#pragma unroll
    for (int e = 0; e < R::E; ++e)
      if (i + e < row.V && key_of(from_bits<R::T>(lift<R::T>(u, e))) == prefix && ++before == n)
        s.bin = i + e;
  });
  lds_barrier();
  return {prefix, s.bin};
}

// Tokens of the row that `takes` into s.list, in any order; their number, which may be
// more than fit.
template <class R, class F>
MSD_DEV int make_list(const R& row, Lds& s, F takes) {
  lds_barrier();
  if (threadIdx.x == 0) s.count = 0;
  lds_barrier();
  row.template each<4>([&](int, int i, const u32x4& u) {
#pragma unroll
    for (int e = 0; e < R::E; ++e) {
      const float x = from_bits<R::T>(lift<R::T>(u, e));
      if (!takes(x, i + e) || i + e >= row.V) continue;
      const int at = atomicAdd(&s.count, 1);
      if (at < LISTED) s.list[at] = place_of(key_of(x), i + e);
    }
  });
  lds_barrier();
  return s.count;
}

// The first n (at most LOGITS_TOP_MAX and V) tokens of the row in order, in s.sorted.
// A wave's r-th largest of its threads' largest, r = n / W rounded up, is reached by r
// tokens of that wave; the least of these over the waves, so by n tokens of the row,
// and by few more of most rows.  Those are ranked by counting.
template <class R>
MSD_DEV void first_tokens(const R& row, uint32_t mine, int n, Group<R::W>& g) {
  Lds& s = g.s;
  const int r = (n + R::W - 1) / R::W;
  uint32_t least = 0;  // its first 20 bits: at most the r-th largest
#pragma unroll
  for (int b = 31; b >= 12; --b) {
    const uint32_t up = least | 1u << b;
    if (__popcll(__ballot(mine >= up)) >= r) least = up;
  }
  const uint32_t floor_key = ~g.max(~least);
  const float at_least = of_key(floor_key);
  int C = floor_key > KEY_NINF ? make_list(row, s, [&](float x, int) { return x >= at_least; })
                               : make_list(row, s, [&](float, int) { return true; });
  if (C > LISTED) {  // very many equal ones, or the largest in few threads
    const Kept k = shortest(row, nullptr, n, g);
    C = make_list(row, s, [&](float x, int i) {
      const uint32_t key = key_of(x);
      return key > k.key || (key == k.key && i <= k.id);
    });
  }
  for (int i = threadIdx.x; i < C; i += R::LB) s.rank[i] = 0;
  lds_barrier();
  // the list in parts, so that every wave counts
  const int pad = (C + 63) & ~63;
  const int parts = pad < R::LB ? R::LB / pad : 1;
  const int per = (C + parts - 1) / parts;
  for (int i0 = threadIdx.x; i0 < pad * parts; i0 += R::LB) {
    const int q = i0 / pad, i = i0 - q * pad;
    if (i >= C) continue;
    const uint64_t me = s.list[i];
    int above = 0;
    const int end = min(C, (q + 1) * per);
    for (int k = q * per; k < end; ++k) above += s.list[k] > me;
    if (above) atomicAdd(&s.rank[i], above);
  }
  lds_barrier();
  for (int i = threadIdx.x; i < C; i += R::LB)
    if (s.rank[i] < n) s.sorted[s.rank[i]] = s.list[i];
  lds_barrier();
}

// Bins of a row's weights, 44 to a factor of two, that ascend as they fall: weights of
// the last are below 2^-46.
constexpr float BINS_PER_2 = 44.f;
MSD_DEV float bin_of(float x, float m, float c) {
  return x == m ? 0.f : fminf((m - x) * c, (float)BINS);
}

// The shortest prefix of the ranked row within `limit` whose weights sum to at least
// top_p of that of `limit`.
template <class R>
MSD_DEV Kept by_weight(const R& row, const Scale& sc, double top_p, Kept limit, Group<R::W>& g) {
  Lds& s = g.s;
  const float m = (float)sc.m;
  const float c = (float)(sc.c * (double)BINS_PER_2);
  const Keeps in(limit);
  clear_bins<R::W>(s);
  row.template each<4>([&](int, int i, const u32x4& u) {
#pragma unroll
    for (int e = 0; e < R::E; ++e) {
      const float x = from_bits<R::T>(lift<R::T>(u, e));
      const float b = bin_of(x, m, c);
      if (b < (float)BINS && in(x, i + e))
        atomicAdd((unsigned long long*)&s.hist[(int)b], weight(x, sc));
    }
  });
  lds_barrier();
  uint64_t sum = 0, all;
  for (int i = threadIdx.x; i < BINS; i += R::LB) sum += s.hist[i];
  all = g.sum(sum);
  uint64_t want = (uint64_t)ceil((double)all * top_p);
  want = want < 1 ? 1 : want > all ? all : want;
  const uint64_t whole = want;
  find_bin<R::W, false>(want, g);
  const float bin = (float)s.bin;
  want -= s.found[0];
  // the tokens of a bin are nearly alike, which tells their number
  const bool many =
      (double)s.found[1] > 0.9 * LISTED * ONE * (double)__builtin_amdgcn_exp2f(-bin / BINS_PER_2);
  float sub = -1.f;
  if (many) {  // bins of that bin
    clear_bins<R::W>(s);
    row.template each<4>([&](int, int i, const u32x4& u) {
#pragma unroll
      for (int e = 0; e < R::E; ++e) {
        const float x = from_bits<R::T>(lift<R::T>(u, e));
        const float b = bin_of(x, m, c);
        if (floorf(b) == bin && in(x, i + e))
          atomicAdd((unsigned long long*)&s.hist[(int)((b - bin) * BINS)], weight(x, sc));
      }
    });
    lds_barrier();
    find_bin<R::W, false>(want, g);
    sub = (float)s.bin;
    want -= s.found[0];
  }
  const int C = make_list(row, s, [&](float x, int i) {
    const float b = bin_of(x, m, c);
    return floorf(b) == bin && (sub < 0 || floorf((b - bin) * BINS) == sub) && in(x, i);
  });
  if (C > LISTED) return shortest(row, &sc, whole, g);
  for (int i = threadIdx.x; i < C; i += R::LB)
    s.hist[i] = weight(of_key((uint32_t)(s.list[i] >> 32)), sc);
  lds_barrier();
  for (int i = threadIdx.x; i < C; i += R::LB) {
    const uint64_t me = s.list[i];
    uint64_t before = 0;
    for (int k = 0; k < C; ++k) before += s.list[k] > me ? s.hist[k] : 0;
    if (before < want && want <= before + s.hist[i]) s.found[0] = me;
  }
  lds_barrier();
  return {(uint32_t)(s.found[0] >> 32), (int)~(uint32_t)s.found[0]};
}

// The first of the values that min_p keeps: x - m >= min_d.
MSD_DEV uint32_t min_key(float m, double min_d) {
  const double least = (double)m + min_d;
  const uint32_t k = key_of((float)least);
  return k + ((double)of_key(k) < least);  // the next one up
}

// A few tokens at most stay (0 < top_k <= LOGITS_TOP_MAX): their number, in order in
// s.sorted, with their weights in s.hist and *all their sum.
template <class R>
MSD_DEV int choose_few(const R& row, uint32_t mine, const Scale& sc, const LogitsChoice& how,
                       uint64_t* all, Group<R::W>& g) {
  Lds& s = g.s;
  const int n = min(how.top_k, row.V);
  first_tokens(row, mine, n, g);
  uint32_t key = 0;
  uint64_t w = 0;
  if ((int)threadIdx.x < n) {
    key = (uint32_t)(s.sorted[threadIdx.x] >> 32);
    w = weight(of_key(key), sc);
    s.hist[threadIdx.x] = w;
  }
  uint64_t sum;
  const uint64_t before = g.before(w, &sum);
  bool stays = key > KEY_NINF;
  if (how.top_p < 1) {
    const uint64_t want = (uint64_t)ceil((double)sum * how.top_p);
    stays = stays && (before < want || threadIdx.x == 0);
  }
  if (how.min_d > -INFINITY) stays = stays && key >= min_key((float)sc.m, how.min_d);
  const int left = (int)g.sum((uint64_t)stays);
  *all = g.sum(stays ? w : 0);
  return left;
}

// The last token that stays.
template <class R>
MSD_DEV Kept choose_many(const R& row, const Scale& sc, const LogitsChoice& how, Group<R::W>& g) {
  Kept k{KEY_NINF + 1, row.V};
  if (how.top_k > 0 && how.top_k < row.V) {
    const Kept t = shortest(row, nullptr, how.top_k, g);
    if (t.key > KEY_NINF) k = t;
  }
  if (how.top_p < 1) k = by_weight(row, sc, how.top_p, k, g);
  if (how.min_d > -INFINITY) {
    const uint32_t least = min_key((float)sc.m, how.min_d);
    if (least > k.key) k = {least, row.V};
  }
  return k;
}

// ------------------------------------------------------------------- operators ----

// The key of the thread's largest.
template <class R>
MSD_DEV uint32_t thread_max(const R& row) {
  float m = -INFINITY;
  row.template each<4>([&](int, int, const u32x4& u) {
#pragma unroll
    for (int e = 0; e < R::E; ++e) m = fmaxf(m, from_bits<R::T>(lift<R::T>(u, e)));
  });
  return key_of(m);
}

template <class R>
MSD_DEV Scale scale_of(float m, double c) {
  return {(double)m, c, m < INFINITY};
}

template <class R>
__global__ __launch_bounds__(R::LB) void k_filter(const void* logits, size_t ld, int V,
                                                  LogitsChoice how, void* out, size_t ldo,
                                                  int* kept) {
  __shared__ Lds s;
  Group<R::W> g{s};
  const R row(logits, ld, V);
  char* const o = static_cast<char*>(out) + (size_t)blockIdx.x * ldo * Type<R::T>::SIZE;
  const uint32_t mine = thread_max(row);
  const float m = of_key(g.max(mine));
  const Scale sc = scale_of<R>(m, how.c);
  Kept k{0xFF800000u, -1};  // nothing: +inf of no id
  if (m > -INFINITY) {
    if (how.top_k > 0 && how.top_k <= LOGITS_TOP_MAX) {
      uint64_t all;
      const uint64_t last = s.sorted[choose_few(row, mine, sc, how, &all, g) - 1];
      k = {(uint32_t)(last >> 32), (int)~(uint32_t)last};
    } else {
      k = choose_many(row, sc, how, g);
    }
  }
  const Keeps stays(k);
  uint32_t n = 0;
  row.template each<4>([&](int, int i, const u32x4& u) {
    u32x4 y = u;
#pragma unroll
    for (int e = 0; e < R::E; ++e) {
      const bool in = stays(from_bits<R::T>(lift<R::T>(u, e)), i + e);
      if (!in) lower<R::T>(y, e, Type<R::T>::NINF & (R::T == MX_F32 ? ~0u : 0xFFFFu));
      n += in;
    }
    row.store(o, i, y);
  });
  const uint64_t all = g.sum((uint64_t)n);
  if (kept && threadIdx.x == 0) kept[blockIdx.x] = (int)all;
}

// The place of u in a whole of `all`.
MSD_DEV uint64_t drawn(float u, uint64_t all) {
  return u >= 1.f ? all - 1 : u > 0.f ? (uint64_t)((double)u * (double)all) : 0;
}
MSD_DEV void put_token(int id, float x, uint64_t all, const Scale& sc, int* tokens,
                       float* logprobs) {
  tokens[blockIdx.x] = id;
  if (logprobs)
    logprobs[blockIdx.x] = (float)((x == (float)sc.m ? 0.0 : ((double)x - sc.m) * sc.c * M_LN2) -
                                   log((double)all * (1 / ONE)));
}

template <class R>
__global__ __launch_bounds__(R::LB) void k_sample(const void* logits, size_t ld, int V,
                                                  LogitsChoice how, const float* uniforms,
                                                  int* tokens, float* logprobs) {
  __shared__ Lds s;
  Group<R::W> g{s};
  const float u = uniforms[blockIdx.x];
  const R row(logits, ld, V);
  const uint32_t mine = thread_max(row);
  const float m = of_key(g.max(mine));
  const Scale sc = scale_of<R>(m, how.c);
  if (!(m > -INFINITY)) {
    if (threadIdx.x == 0) {
      tokens[blockIdx.x] = -1;
      if (logprobs) logprobs[blockIdx.x] = -INFINITY;
    }
    return;
  }
  uint64_t all;
  if (how.top_k > 0 && how.top_k <= LOGITS_TOP_MAX) {
    const int n = choose_few(row, mine, sc, how, &all, g);
    if ((int)threadIdx.x >= n) return;
    // the running sum in the order of the ids, of which ~ makes the lower the greater
    const uint32_t me = (uint32_t)s.sorted[threadIdx.x];
    uint64_t before = 0;
    for (int i = 0; i < n; ++i) before += (uint32_t)s.sorted[i] > me ? s.hist[i] : 0;
    const uint64_t at = drawn(u, all);
    if (before <= at && at < before + s.hist[threadIdx.x])
      put_token((int)~me, of_key((uint32_t)(s.sorted[threadIdx.x] >> 32)), all, sc, tokens, logprobs);
    return;
  }
  const Keeps stays(choose_many(row, sc, how, g));
  // sums of stretches of 64 units, one for each tile and wave, in the order of the ids
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  lds_barrier();
  row.template each<4>([&](int j, int i, const u32x4& un) {
    uint64_t sum = 0;
#pragma unroll
    for (int e = 0; e < R::E; ++e) {
      const float x = from_bits<R::T>(lift<R::T>(un, e));
      if (stays(x, i + e)) sum += weight(x, sc);
    }
    sum = wave_scan(sum, (uint64_t)0, Sum());
    if (lane == 63) s.hist[j * R::W + w] = sum;
  });
  lds_barrier();
  // the stretch that holds the place
  const int n = (V + R::TILE - 1) / R::TILE * R::W;
  const int per = (n + R::LB - 1) / R::LB;
  uint64_t sum = 0;
  for (int i = 0; i < per; ++i) {
    const int q = threadIdx.x * per + i;
    if (q < n) sum += s.hist[q];
  }
  uint64_t run = g.before(sum, &all);
  const uint64_t at = drawn(u, all);
  if (run <= at && at < run + sum) {
    int q = threadIdx.x * per;
    while (run + s.hist[q] <= at) run += s.hist[q++];
    s.bin = q;
    s.found[0] = run;
  }
  lds_barrier();
  if (s.bin % R::W != w) return;
  const int j = __builtin_amdgcn_readfirstlane(s.bin / R::W);
  const u32x4 un = row.load_tail(j);
  uint64_t ws[R::E];
  sum = 0;
#pragma unroll
  for (int e = 0; e < R::E; ++e) {
    const float x = from_bits<R::T>(lift<R::T>(un, e));
    ws[e] = stays(x, row.id(j) + e) ? weight(x, sc) : 0;
    sum += ws[e];
  }
  run = s.found[0] + wave_scan(sum, (uint64_t)0, Sum()) - sum;
#pragma unroll
  for (int e = 0; e < R::E; ++e) {
    if (run <= at && at < run + ws[e])
      put_token(row.id(j) + e, from_bits<R::T>(lift<R::T>(un, e)), all, sc, tokens, logprobs);
    run += ws[e];
  }
}

// The thread's sum of e^((x - m) / T), c = log2(e) / T, in 32 bits.
template <class R>
MSD_DEV float exp_sum(const R& row, float m, float c) {
  float sum = 0.f;
  row.template each<4>([&](int, int, const u32x4& u) {
#pragma unroll
    for (int e = 0; e < R::E; ++e)
      sum += __builtin_amdgcn_exp2f((from_bits<R::T>(lift<R::T>(u, e)) - m) * c);
  });
  return sum;
}

template <class R>
__global__ __launch_bounds__(R::LB) void k_top(const void* logits, size_t ld, int V, int n,
                                               float* values, int* ids, float* lse) {
  __shared__ Lds s;
  Group<R::W> g{s};
  const R row(logits, ld, V);
  const uint32_t mine = thread_max(row);
  const float m = of_key(g.max(mine));
  first_tokens(row, mine, n, g);
  if ((int)threadIdx.x < n) {
    const size_t o = (size_t)blockIdx.x * n + threadIdx.x;
    const uint64_t t = s.sorted[threadIdx.x];
    values[o] = of_key((uint32_t)(t >> 32));
    ids[o] = (int)~(uint32_t)t;
  }
  if (!lse) return;
  float l = m;
  if (fabsf(m) < INFINITY) {
    // (a NaN is no token)
    float sum = 0.f;
    row.template each<4>([&](int, int, const u32x4& u) {
#pragma unroll
      for (int e = 0; e < R::E; ++e)
        sum += __builtin_amdgcn_exp2f(
            fmaxf(from_bits<R::T>(lift<R::T>(u, e)) - m, -INFINITY) * (float)M_LOG2E);
    });
    l = (float)((double)m + log(g.sum((double)sum)));
  }
  if (threadIdx.x == 0) lse[blockIdx.x] = l;
}

// A row's teacher entry of this thread (id < 0: none).
struct Entry {
  int id;
  float value;
  double lq, q;
};

// q = softmax(t / T) over the row's entries; all zero where none has a value above
// -inf, NaN where one is NaN or +inf.
template <int W>
MSD_DEV void soften(Entry& e, double inv_t, Group<W>& g) {
  const float top = of_key(g.max(key_of(e.value)));
  const double d = ((double)e.value - (double)top) * inv_t;
  const double w = e.value == -INFINITY ? 0 : exp(d);
  const double sum = g.sum(w);
  e.lq = e.q = 0;
  if (w != 0) {
    e.lq = d - log(sum);
    e.q = w / sum;
  }
}

template <class R>
__global__ __launch_bounds__(R::LB) void k_distill(const void* logits, size_t ld, int V,
                                                   LogitsTeacher t, float* loss, float* lse,
                                                   const float* grad, void* dx, size_t ldd) {
  __shared__ Lds s;
  Group<R::W> g{s};
  Entry e{-1, -INFINITY, 0, 0};
  if ((int)threadIdx.x < t.k) {
    const size_t o = (size_t)blockIdx.x * t.k + threadIdx.x;
    e.id = t.ids[o];
    if (e.id < 0 || e.id >= V) e.id = -1;
    if (e.id >= 0) e.value = t.values[o];
    s.list[threadIdx.x] = (uint32_t)e.id;
  }
  const R row(logits, ld, V);
  const float zk = e.id >= 0 ? from_bits<R::T>(bits_at<R::T>(row.p, e.id)) : 0.f;
  soften(e, t.inv_t, g);
  const float c = (float)(t.inv_t * M_LOG2E);
  // a NaN is passed over here and found again by the sum
  const float m = of_key(g.max(thread_max(row)));
  const double sum = g.sum((double)exp_sum(row, m, c));
  const double dk = ((double)zk - (double)m) * t.inv_t;
  const double l = g.sum(e.q != 0 ? e.q * (e.lq - (dk - log(sum))) : 0.0);
  if (loss && threadIdx.x == 0) loss[blockIdx.x] = (float)l;
  if (lse && threadIdx.x == 0) lse[blockIdx.x] = (float)(m * t.inv_t + log(sum));
  if (!dx) return;
  // the entries' logits are read before a gradient in their place is written
  asm volatile("" ::"v"(zk));
  if ((int)threadIdx.x < t.k) s.hist[threadIdx.x] = (uint64_t)__double_as_longlong(e.q);
  const double mass = g.sum(e.q);  // 1 (or NaN); 0 without entries
  const double gr = mass == 0 ? 0 : grad[blockIdx.x] * t.inv_t * mass;
  char* const o = static_cast<char*>(dx) + (size_t)blockIdx.x * ldd * Type<R::T>::SIZE;
  if (mass == 0) {
    const u32x4 none = 0u;
    row.template each<4>([&](int, int i, const u32x4&) { row.store(o, i, none); });
    return;
  }
  const float f = (float)(gr / sum);
  row.template each<4>([&](int, int i, const u32x4& u) {
    u32x4 y;
#pragma unroll
    for (int e = 0; e < R::E; ++e)
      lower<R::T>(y, e,
                  to_bits<R::T>(f * __builtin_amdgcn_exp2f(
                                        (from_bits<R::T>(lift<R::T>(u, e)) - m) * c)));
    row.store(o, i, y);
  });
  __syncthreads();
  if (e.id < 0) return;
  // the first entry of an id carries the others'
  double q = 0;
  for (int i = 0; i < t.k; ++i) {
    if ((int)(uint32_t)s.list[i] != e.id) continue;
    if (i < (int)threadIdx.x) return;
    q += __longlong_as_double((long long)s.hist[i]);
  }
  put_bits<R::T>(o, e.id, to_bits<R::T>((float)(gr * (exp(dk) / sum - q))));
}

}  // namespace

namespace {

template <class F>
void by_type(int type, F f) {
  if (type == MX_F32)
    f(std::integral_constant<int, MX_F32>());
  else if (type == MX_BF16)
    f(std::integral_constant<int, MX_BF16>());
  else
    f(std::integral_constant<int, MX_F16>());
}

// Rows of up to this many bytes take a workgroup of 256 threads.
constexpr int SHORT_ROW = 256 * 8 * 16;

}  // namespace

void launch_logits_top(const void* x, int type, size_t ld, int rows, int cols, int k, float* values,
                       int* ids, float* lse, hipStream_t st) {
  if (rows <= 0) return;
  by_type(type, [&](auto t_) {
    constexpr int TYPE = decltype(t_)::value;
    if (cols * Type<TYPE>::SIZE <= SHORT_ROW)
      k_top<Row<TYPE, 256>><<<rows, 256, 0, st>>>(x, ld, cols, k, values, ids, lse);
    else
      k_top<Row<TYPE, 1024>><<<rows, 1024, 0, st>>>(x, ld, cols, k, values, ids, lse);
  });
}

void launch_logits_sample(const void* x, int type, size_t ld, int rows, int cols,
                          const LogitsChoice& how, const float* uniforms, int* tokens,
                          float* logprobs, hipStream_t st) {
  if (rows <= 0) return;
  by_type(type, [&](auto t_) {
    constexpr int TYPE = decltype(t_)::value;
    if (cols * Type<TYPE>::SIZE <= SHORT_ROW)
      k_sample<Row<TYPE, 256>><<<rows, 256, 0, st>>>(x, ld, cols, how, uniforms, tokens, logprobs);
    else
      k_sample<Row<TYPE, 1024>>
          <<<rows, 1024, 0, st>>>(x, ld, cols, how, uniforms, tokens, logprobs);
  });
}

void launch_logits_filter(const void* x, int type, size_t ld, int rows, int cols,
                          const LogitsChoice& how, void* out, size_t ldo, int* kept,
                          hipStream_t st) {
  if (rows <= 0) return;
  by_type(type, [&](auto t_) {
    constexpr int TYPE = decltype(t_)::value;
    if (cols * Type<TYPE>::SIZE <= SHORT_ROW)
      k_filter<Row<TYPE, 256>><<<rows, 256, 0, st>>>(x, ld, cols, how, out, ldo, kept);
    else
      k_filter<Row<TYPE, 1024>><<<rows, 1024, 0, st>>>(x, ld, cols, how, out, ldo, kept);
  });
}

void launch_logits_distill(const void* x, int type, size_t ld, int rows, int cols,
                           const LogitsTeacher& t, float* loss, float* lse, const float* grad,
                           void* dx, size_t ldd, hipStream_t st) {
  if (rows <= 0) return;
  by_type(type, [&](auto t_) {
    constexpr int TYPE = decltype(t_)::value;
    const int tiles = cols / (1024 * Type<TYPE>::E);  // whole ones
    if (cols * Type<TYPE>::SIZE <= SHORT_ROW)
      k_distill<HeldRow<TYPE, 256, 8>>
          <<<rows, 256, 0, st>>>(x, ld, cols, t, loss, lse, grad, dx, ldd);
    else if (tiles <= 8)
      k_distill<HeldRow<TYPE, 1024, 8>>
          <<<rows, 1024, 0, st>>>(x, ld, cols, t, loss, lse, grad, dx, ldd);
    else if (tiles <= 19)
      k_distill<HeldRow<TYPE, 1024, 19>>
          <<<rows, 1024, 0, st>>>(x, ld, cols, t, loss, lse, grad, dx, ldd);
    else
      k_distill<HeldRow<TYPE, 1024, 0>>
          <<<rows, 1024, 0, st>>>(x, ld, cols, t, loss, lse, grad, dx, ldd);
  });
}

}  // namespace msd
