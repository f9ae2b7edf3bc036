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
// any order, atomics included: no result depends on the order of the atomics.
//
// One workgroup a row; no memory but the operands and the workgroup's own LDS, so calls on
// several streams and captured graphs share nothing.  Offsets of a row are 64-bit, within a
// row 32-bit (at most 2^18 logits).
//
// Times here are of one MI355X, on which a copy of 82 MB reads and writes 7.0 TB/s, one of
// 2 GiB 5.0 TB/s, a long read alone 6.9 to 7.1, and the smallest launch takes 4.2 us in a row
// of launches.  They are means over launches in a row, over inputs in turn; "a -> b us" are
// those before and after a step, both of the time when it was taken.
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

// A unit of E values, rounded by the hardware's conversions.
template <int TYPE>
MSD_DEV u32x4 pack(const float (&v)[Type<TYPE>::E]) {
  u32x4 u;
  if constexpr (TYPE == MX_F32) {
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = __float_as_uint(v[e]);
  } else {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (TYPE == MX_BF16)
        u[e] = __builtin_bit_cast(uint32_t, b2{(__bf16)v[2 * e], (__bf16)v[2 * e + 1]});
      else
        u[e] = __builtin_bit_cast(uint32_t, h2{(_Float16)v[2 * e], (_Float16)v[2 * e + 1]});
    }
  }
  return u;
}

// A row of V logits over the W waves of LB threads, in units of 16 bytes a lane: 64 units,
// a stretch, for a wave at a time.  A wave's stretches lie W apart (tiles of the whole
// workgroup), or with RUNS one after the other, so that its sums are of neighbouring ids.
// Places past V hold -inf.
template <int TYPE, int LB_, bool RUNS = false>
struct Row {
  static constexpr int T = TYPE, LB = LB_, E = Type<TYPE>::E, TILE = LB * E, W = LB / 64;
  static constexpr int STRETCH = 64 * E;
  typedef typename Type<TYPE>::unit unit;
  const char* p;
  int V;
  int at, full, part;  // the thread's first id; the wave's whole stretches, and any after them

  MSD_DEV Row(const void* base, size_t ld, int V_)
      : p(static_cast<const char*>(base) + (size_t)blockIdx.x * ld * Type<TYPE>::SIZE), V(V_) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if constexpr (RUNS) {
      const int n = per_wave(), first = wave * n;
      full = min(max(V / STRETCH - first, 0), n);
      part = full < n && (first + full) * STRETCH < V;
      at = first * STRETCH + (threadIdx.x & 63) * E;
    } else {
      full = V / TILE;
      part = V % TILE != 0;
      at = threadIdx.x * E;
    }
  }
  // The other order of the same row.
  MSD_DEV explicit Row(const Row<TYPE, LB_, !RUNS>& o) : p(o.p), V(o.V) {
    static_assert(!RUNS, "in tiles");
    full = V / TILE;
    part = V % TILE != 0;
    at = threadIdx.x * E;
  }
  MSD_DEV int per_wave() const { return (V + TILE - 1) / TILE; }
  MSD_DEV int id(int j) const { return at + j * (RUNS ? STRETCH : TILE); }
  MSD_DEV u32x4 load(int j) const {
    return *reinterpret_cast<const unit*>(p + (size_t)id(j) * Type<TYPE>::SIZE);
  }
  // One that V may end in.
  MSD_DEV u32x4 load_tail(int j) const {
    const int i = id(j);
    if (i + E <= V) return load(j);
    u32x4 u = Type<TYPE>::NINF;
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (i + e < V) lower<TYPE>(u, e, bits_at<TYPE>(p, i + e));
    return u;
  }
  // f(j, id, unit) for every unit of the wave in order, read from memory, the next AHEAD
  // under way while f works on these.
  template <int AHEAD, class F>
  MSD_DEV void each(F f) const {
    u32x4 next[AHEAD], last = Type<TYPE>::NINF;
#pragma unroll
    for (int b = 0; b < AHEAD; ++b) next[b] = b < full ? load(b) : last;
    if (part) last = load_tail(full);
    for (int j = 0; j < full; j += AHEAD) {
      u32x4 t[AHEAD];
#pragma unroll
      for (int b = 0; b < AHEAD; ++b) {
        t[b] = next[b];
        if (j + AHEAD + b < full) next[b] = load(j + AHEAD + b);
      }
#pragma unroll
      for (int b = 0; b < AHEAD; ++b)
        if (j + b < full) f(j + b, id(j + b), t[b]);
    }
    if (part) f(full, id(full), last);
  }
  // Past the caches: a row's outputs are not read again by this call, and in the caches they
  // would push out rows that are (gradients of 639 x 32,000 f32 52 -> 44 us, of 1,151 x
  // 152,064 bf16 319 -> 288; filter of 488 x 152,064 f32 190 -> 178).
  MSD_DEV void store(char* o, int i, const u32x4& u) const {
    if (i + E <= V) {
      __builtin_nontemporal_store(u, reinterpret_cast<unit*>(o + (size_t)i * Type<TYPE>::SIZE));
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (i + e < V) put_bits<TYPE>(o, i + e, lift<TYPE>(u, e));
    }
  }
};

// The same with up to U whole tiles and the last one in registers: for a second pass that
// needs every logit again (the gradient), HBM is read once.
template <int TYPE, int LB, int U>
struct HeldRow : Row<TYPE, LB> {
  static constexpr int UNITS = U;
  mutable u32x4 r[U], last;
  MSD_DEV HeldRow(const void* base, size_t ld, int V) : Row<TYPE, LB>(base, ld, V) {
#pragma unroll
    for (int j = 0; j < U; ++j) r[j] = j < this->full ? this->load(j) : u32x4(Type<TYPE>::NINF);
    last = Type<TYPE>::NINF;
    if (this->part) last = this->load_tail(this->full);
  }
  template <int AHEAD, class F>
  MSD_DEV void each(F f) const {
#pragma unroll
    for (int j = 0; j < U; ++j) {
      // so that no pass keeps its converted values for the next one
      asm("" : "+v"(r[j]));
      if (j < this->full) f(j, this->id(j), r[j]);
    }
    asm("" : "+v"(last));
    if (this->part) f(this->full, this->id(this->full), last);
  }
};
template <int TYPE, int LB>
struct HeldRow<TYPE, LB, 0> : Row<TYPE, LB> {  // too long for that
  using Row<TYPE, LB>::Row;
};

// A row that is read once, of up to U whole tiles, AHEAD of them under way at a time, whose
// units' largest (of each PER of them) stay in registers: they tell which few units to read
// again.  A quarter of a held row's registers or less, so that long rows share a CU too (top
// 128 of 1,151 x 152,064 bf16 161 -> 114 us).
template <int TYPE, int LB, int U, int AHEAD, int PER = 1>
struct ToppedRow : Row<TYPE, LB> {
  using Row<TYPE, LB>::Row;
  static constexpr int UNITS = U, TOPS = U / PER;
  static_assert(U % PER == 0 && U <= 64, "a bit for each unit");
  float top[TOPS + 1];
  // m = f(unit) for every unit in order, m its largest.
  template <class F>
  MSD_DEV void read(F f) {
    u32x4 next[AHEAD], last = Type<TYPE>::NINF;
#pragma unroll
    for (int b = 0; b < AHEAD; ++b) next[b] = b < this->full ? this->load(b) : last;
    if (this->part) last = this->load_tail(this->full);
#pragma unroll
    for (int j = 0; j < U; ++j) {
      if (j % PER == 0) top[j / PER] = -INFINITY;
      if (j < this->full) {
        const u32x4 t = next[j % AHEAD];
        if (j + AHEAD < this->full) next[j % AHEAD] = this->load(j + AHEAD);
        top[j / PER] = fmaxf(top[j / PER], f(t));
      }
    }
    top[TOPS] = this->part ? f(last) : -INFINITY;
  }
  // The units that may reach x (others may be among them).
  MSD_DEV uint64_t reach(float x) const {
    uint64_t m = 0;
#pragma unroll
    for (int j = 0; j < TOPS; ++j)
      m |= (uint64_t)(top[j] >= x ? (1u << PER) - 1 : 0u) << (j * PER);
    if (this->full < 64) m &= (1ull << this->full) - 1;
    if (this->part && top[TOPS] >= x) m |= 1ull << this->full;
    return m;
  }
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
  float m;
  double c, m64;
  bool finite;  // an infinite maximum weighs 1 and leaves nothing to the others
  MSD_DEV Scale(float m_, double c_)
      : m(m_), c(c_), m64(m_ < INFINITY ? m_ : 0.0), finite(m_ < INFINITY) {}
  MSD_DEV float operator()(float x) const {  // what weighs
    return finite ? x : x == INFINITY ? 0.f : -INFINITY;
  }
};
// About 25 vector instructions, of 64 bits at the rate of 32-bit ones here (0.59 ns for a
// wave's on one CU); the library's exp takes more, and its last bits are not a contract.
// With 128 added, as a double: sums of n such bits are n times 128's more than the sum.
// d: x - m.
MSD_DEV uint64_t bits_at_distance(double d, const Scale& s) {
  const double t = fmax(d * s.c, -64.0);  // (a NaN too)
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
  return (uint64_t)__double_as_longlong(w + 128.0);
}
constexpr uint64_t BITS_128 = 0x4060000000000000ull;
MSD_DEV uint64_t bits_of(float x, const Scale& s) {
  return bits_at_distance((double)x - s.m64, s);
}
MSD_DEV uint64_t weight(float x, const Scale& s) { return bits_of(s(x), s) - BITS_128; }

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

constexpr int BINS = 2048;
constexpr int SLOTS = 4;
struct Lds {  // of every kernel
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

// A bound for a row's n first tokens without a search over the row: the key of its largest,
// and one that the r largest of the threads' largest reach in every wave: so W r tokens at
// least reach it, and few more of most rows.
struct Tops {
  uint32_t max, floor;
};
template <int W>
MSD_DEV Tops tops(uint32_t mine, int r, Group<W>& g) {
  uint32_t least = 0;  // the first 20 bits of the r-th largest: at most that
#pragma unroll
  for (int b = 31; b >= 12; --b) {
    const uint32_t up = least | 1u << b;
    if (__popcll(__ballot(mine >= up)) >= r) least = up;
  }
  const uint64_t* p = g.swap((uint64_t)wave_scan(mine, 0u, Max()) << 32 | least);
  Tops t{0, 0xFFFFFFFFu};
#pragma unroll
  for (int i = 0; i < W; ++i) {
    t.max = Max()(t.max, (uint32_t)(p[i] >> 32));
    t.floor = min(t.floor, (uint32_t)p[i]);
  }
  return t;
}

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

// The bin of hist in which the running sum reaches `want`, with the sum before it and its
// own in s.found; *all: the whole sum.  Bins ascend from bin 0 on, or descend from the last.
template <int W, bool DOWN>
MSD_DEV void find_bin(const uint64_t* hist, uint64_t want, uint64_t* all, Group<W>& g) {
  constexpr int PER = BINS / (W * 64);
  uint64_t h[PER], sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int b = threadIdx.x * PER + i;
    sum += h[i] = hist[DOWN ? BINS - 1 - b : b];
  }
  uint64_t run = g.before(sum, all);
  if (run < want && want <= run + sum) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (run < want && want <= run + h[i]) {
        const int b = threadIdx.x * PER + i;
        g.s.bin = DOWN ? BINS - 1 - b : b;
        g.s.found[0] = run;
        g.s.found[1] = h[i];
      }
      run += h[i];
    }
  }
  lds_barrier();
}

template <int W>
MSD_DEV void clear_bins(uint64_t* hist) {
  lds_barrier();
  for (int i = threadIdx.x; i < BINS; i += W * 64) hist[i] = 0;
  lds_barrier();
}

// The shortest prefix of the ranked row whose counts (null) or weights sum to at least
// `want` (1 <= want <= their sum), digit by digit of the keys: for any row, in up to
// four passes over it.
template <class R>
MSD_DEV Kept shortest(const R& row, const Scale* sc, uint64_t want, uint64_t* hist,
                      Group<R::W>& g) {
  Lds& s = g.s;
  uint32_t prefix = 0;  // the digits found so far
  int left = 32;        // bits below them
  uint64_t ties = 0, each = 1, all;
  while (left > 0) {
    const int bits = left > 11 ? 11 : left;
    const int low = left - bits;
    clear_bins<R::W>(hist);
    row.template each<2>([&](int, int i, const u32x4& u) {
#pragma unroll
      for (int e = 0; e < R::E; ++e) {
        const float x = from_bits<R::T>(lift<R::T>(u, e));
        const uint32_t k = key_of(x);
        if (i + e >= row.V || (left < 32 && (k ^ prefix) >> left)) continue;
        const uint64_t w = sc ? weight(x, *sc) : 1;
        if (w) atomicAdd((unsigned long long*)&hist[(k >> low) & ((1u << bits) - 1)], w);
      }
    });
    lds_barrier();
    find_bin<R::W, true>(hist, want, &all, g);
    prefix |= (uint32_t)s.bin << low;
    want -= s.found[0];
    ties = s.found[1];
    left = low;
  }
  if (sc) each = weight(of_key(prefix), *sc);
  const uint64_t n = (want + each - 1) / each;  // of the equal ones, at least 1
  if (n * each >= ties) return {prefix, row.V};
  // the n-th of them in the order of their ids, a tile at a time
  const Row<R::T, R::LB> tiles(row);
  const int end = (row.V + R::TILE - 1) / R::TILE;
  uint64_t seen = 0;
  for (int j = 0; j < end && seen < n; ++j) {
    const u32x4 u = tiles.load_tail(j);
    const int i = tiles.id(j);
    int hits = 0;
#pragma unroll
    for (int e = 0; e < R::E; ++e)
      hits += i + e < row.V && key_of(from_bits<R::T>(lift<R::T>(u, e))) == prefix;
    uint64_t before = seen + g.before(hits, &all);
    seen += all;
    if (before >= n || before + hits < n) continue;
#pragma unroll
    for (int e = 0; e < R::E; ++e)
      if (i + e < row.V && key_of(from_bits<R::T>(lift<R::T>(u, e))) == prefix && ++before == n)
        s.bin = i + e;
  }
  lds_barrier();
  return {prefix, s.bin};
}

// Places of the unit's tokens that `takes` at the end of a list of `room`; s.count counts
// those that found none too.
template <class R, class F>
MSD_DEV void append(const R& row, int i, const u32x4& u, uint64_t* list, int room, Lds& s, F takes) {
  int c = 0;
#pragma unroll
  for (int e = 0; e < R::E; ++e)
    c += i + e < row.V && takes(from_bits<R::T>(lift<R::T>(u, e)), i + e);
  if (!c) return;
  int at = atomicAdd(&s.count, c);
#pragma unroll
  for (int e = 0; e < R::E; ++e) {
    const float x = from_bits<R::T>(lift<R::T>(u, e));
    if (i + e >= row.V || !takes(x, i + e)) continue;
    if (at < room) list[at] = place_of(key_of(x), i + e);
    ++at;
  }
}
MSD_DEV void clear_count(Lds& s) {
  lds_barrier();
  if (threadIdx.x == 0) s.count = 0;
  lds_barrier();
}

// The first of the values that min_p keeps: x - m >= min_d.
MSD_DEV uint32_t min_key(float m, double min_d) {
  const double least = (double)m + min_d;
  const uint32_t k = key_of((float)least);
  return k + ((double)of_key(k) < least);  // the next one up
}

// A unit's largest.
template <class R>
MSD_DEV float unit_max(const u32x4& u) {
  float m = -INFINITY;
#pragma unroll
  for (int e = 0; e < R::E; ++e) m = fmaxf(m, from_bits<R::T>(lift<R::T>(u, e)));
  return m;
}

// The key of the thread's largest.
template <class R>
MSD_DEV uint32_t thread_max(const R& row) {
  float m = -INFINITY;
  row.template each<4>([&](int, int, const u32x4& u) { m = fmaxf(m, unit_max<R>(u)); });
  return key_of(m);
}

// ----------------------------------------------------------- a few first tokens ----

constexpr int FEW = 1024;      // tokens that are ranked,
constexpr int BUCKETS = 2048;  // among those of their bucket
struct FewLds : Lds {
  union {
    uint64_t hist[BINS];
    uint32_t base[BUCKETS + 1];
    uint64_t weights[LOGITS_TOP_MAX];
  };
  uint64_t list[FEW], other[FEW];
  uint64_t sorted[LOGITS_TOP_MAX];
};

// The bucket of a key at or below that of the row's largest: 32 to a factor of two of the
// distance between the keys.  It does not fall where the key does.
MSD_DEV int bucket_of(uint32_t most, uint32_t key) {
  return (int)((__float_as_uint((float)(most - key)) >> 18) - (most == key ? 0 : (126u << 5)));
}
static_assert(((127 + 32) << 5) - (126 << 5) < BUCKETS, "the largest distance");

// s.list[0 .. C) ranked: its first n in s.sorted.  most: the key of the row's largest.  A
// token is compared with those of its bucket only: of short lists no slower than all pairs
// (top 10 of a row of 32,000 8.0 us, by pairs 8.8; top 64 of 61 of them 10.3 and 10.7; top 20
// of 640 rows of 8,192 11.2 and 10.4), of long ones much faster (top 28 of one row of 304,
// which lists all of it, 9.7 and 40).
template <int LB>
MSD_DEV void rank(FewLds& s, int C, int n, uint32_t most, Group<LB / 64>& g) {
  constexpr int PER = FEW / LB, WIDE = BUCKETS / LB;
  for (int i = threadIdx.x; i <= BUCKETS; i += LB) s.base[i] = 0;
  lds_barrier();
  uint64_t mine[PER];
  int at[PER], bucket[PER];
#pragma unroll
  for (int q = 0; q < PER; ++q) {
    const int i = threadIdx.x + q * LB;
    if (i >= C) continue;
    mine[q] = s.list[i];
    bucket[q] = bucket_of(most, (uint32_t)(mine[q] >> 32));
    at[q] = (int)atomicAdd(&s.base[bucket[q]], 1u);
  }
  lds_barrier();
  uint32_t size[WIDE], sum = 0;
#pragma unroll
  for (int q = 0; q < WIDE; ++q) sum += size[q] = s.base[threadIdx.x * WIDE + q];
  uint64_t all;
  uint32_t run = (uint32_t)g.before(sum, &all);
#pragma unroll
  for (int q = 0; q < WIDE; ++q) {
    s.base[threadIdx.x * WIDE + q] = run;
    run += size[q];
  }
  if (threadIdx.x == LB - 1) s.base[BUCKETS] = run;
  lds_barrier();
#pragma unroll
  for (int q = 0; q < PER; ++q)
    if ((int)threadIdx.x + q * LB < C) s.other[s.base[bucket[q]] + at[q]] = mine[q];
  lds_barrier();
#pragma unroll
  for (int q = 0; q < PER; ++q) {
    if ((int)threadIdx.x + q * LB >= C) continue;
    const int from = s.base[bucket[q]], to = s.base[bucket[q] + 1];
    int above = from;
    if (above >= n) continue;
    for (int k = from; k < to; ++k) above += s.other[k] > mine[q];
    if (above < n) s.sorted[above] = mine[q];
  }
  lds_barrier();
}

// The first n (at most LOGITS_TOP_MAX and V) tokens of the row in order, in s.sorted:
// those that reach a bound that n at least do, ranked; with DEAD also those of -inf, if the
// others do not suffice.  Returns their number.
template <bool DEAD, class R>
MSD_DEV int first_tokens(const R& row, const Tops& t, int n, FewLds& s, Group<R::W>& g) {
  const float at_least = of_key(max(t.floor, KEY_NINF + 1));
  const Row<R::T, R::LB>& mem = row;
  uint64_t units = row.reach(at_least);
  for (; units; units &= units - 1) {
    const int j = __ffsll((unsigned long long)units) - 1;
    append(mem, mem.id(j), mem.load_tail(j), s.list, FEW, s,
           [&](float x, int) { return x >= at_least; });
  }
  lds_barrier();
  int C = s.count;
  if (C > FEW || (DEAD && C < n)) {  // very many equal ones, or the largest in few threads
    const Kept k = shortest(mem, nullptr, n, s.hist, g);
    clear_count(s);
    mem.template each<2>([&](int, int i, const u32x4& u) {
      append(mem, i, u, s.list, FEW, s, [&](float x, int id) {
        const uint32_t key = key_of(x);
        return key > k.key || (key == k.key && id <= k.id);
      });
    });
    lds_barrier();
    C = s.count;
  }
  n = min(n, C);
  rank<R::LB>(s, C, n, t.max, g);
  return n;
}

// The tokens that stay of a few at most (0 < top_k <= LOGITS_TOP_MAX): their number, in
// order in s.sorted, with their weights in s.weights and *all their sum.
template <class R>
MSD_DEV int choose_few(const R& row, const Tops& t, const Scale& sc, const LogitsChoice& how,
                       uint64_t* all, FewLds& s, Group<R::W>& g) {
  const int n = first_tokens<false>(row, t, min(how.top_k, row.V), s, g);
  uint32_t key = 0;
  uint64_t w = 0;
  if ((int)threadIdx.x < n) {
    key = (uint32_t)(s.sorted[threadIdx.x] >> 32);
    w = weight(of_key(key), sc);
    s.weights[threadIdx.x] = w;
  }
  uint64_t sum;
  const uint64_t before = g.before(w, &sum);
  bool stays = key > KEY_NINF;
  if (how.top_p < 1) {
    const uint64_t want = (uint64_t)ceil((double)sum * how.top_p);
    stays = stays && (before < want || threadIdx.x == 0);
  }
  if (how.min_d > -INFINITY) stays = stays && key >= min_key(sc.m, how.min_d);
  const int left = (int)g.sum((uint64_t)stays);
  *all = g.sum(stays ? w : 0);
  return left;
}

// ------------------------------------------------- any number of tokens that stay ----

// The pass that finds a row's largest counts its logits too, in COUNTS bins of T / 64
// around one of them (`ref`, the largest of its waves' first), HEAD bins above it, with
// the sums of their places in the bins.  Weights at the means of the bins are off by
// (1 / 64)^2 / 24 = 1e-5 at most, all nearly alike, so that they give the border of top-p
// to a few tokens.  The next pass computes the weights: those of all for their sum, those
// that surely stay, and it lists the tokens around the estimate, among which the border
// then has to lie.  Where it does not (rows of very many equal logits), the border is
// found digit by digit.  Sample by top_p of 512 x 152,064 f32: 355 us with every weight in
// a histogram of 64-bit sums -> 228 with the border estimated from counts -> 158 with the means.
//   Where it does not: values of 16 bits far from 0 lie so far apart that a flat row's border
// is among more equal ones than the list or `few` holds.  Of 512 x 152,064 normal logits at a
// mean of 12 and a deviation of 1, top_p 0.9: bf16 638 us, f16 481, f32 150.
constexpr double COUNTS_PER_T = 64;
constexpr int PLACE_BITS = 40;  // of a bin's sum of places, in 2^-20
constexpr int GROUP = 8;    // stretches of a wave that are summed together: a cell
constexpr int CELLS = 256;  // a row's, 16 to a wave
// Short rows take 31 KB for 76 KB, so that five share a CU and not two: sample of 3,136 x
// 300 f32 100 -> 45 us, filter of 3,000 x 5,000 bf16 119 -> 62.
template <int LB>
struct ManyLds : Lds {
  // a bin and 20 bits of a place in it are a word
  static constexpr int COUNTS = LB == 256 ? 2048 : 4096, HEAD = COUNTS / 4;
  static constexpr int LIST = LB == 256 ? 1024 : 4096;   // tokens around the estimate
  static constexpr int BORDER = LB == 256 ? 256 : 512;   // that share the border's bin of those
  static constexpr int LEVELS = 8 * (LIST + 2 * BORDER);
  union {
    uint64_t hist[BINS];
    uint64_t counts[COUNTS];
  };
  union {
    struct {
      uint64_t list[LIST];
      uint64_t few[BORDER], few_w[BORDER];
    };
    uint8_t levels[LEVELS];  // of the units, before there is a list
  };
  uint64_t cells[CELLS];
};

template <int LB>
struct Bins {
  static constexpr int COUNTS = ManyLds<LB>::COUNTS, HEAD = ManyLds<LB>::HEAD;
  float ref, scale;
  MSD_DEV Bins(float r, double c)
      : ref(r), scale((float)fmin(c * (COUNTS_PER_T / M_LOG2E), 1e30)) {}
  // A bin and the place in it, in 2^-20; 0 for what lies below, and for a NaN.
  MSD_DEV uint32_t at(float x) const {
    const float b = fmaf(x - ref, scale * 0x1p20f, (float)(COUNTS - HEAD) * 0x1p20f);
    return (uint32_t)fminf(fmaxf(b, 0.f), (float)COUNTS * (0x1p20f - 0x1p-4f));
  }
  MSD_DEV float edge(float b) const { return ref + (b - (float)(COUNTS - HEAD)) / scale; }
  // The weight there, of the row's largest at most; not rounded to a logit.
  MSD_DEV uint64_t weight_at(float b, const Scale& s) const {
    const double d = (double)ref - s.m64 + (double)(b - (float)(COUNTS - HEAD)) / (double)scale;
    return bits_at_distance(fmin(d, 0.0), s) - BITS_128;
  }
  // The coarse bin, of 256 at most; it does not fall where x rises.
  MSD_DEV uint32_t level(float x) const { return at(x) >> 24; }
};

// The row's largest, and with `count` its counts; with `levels` the level of each unit's
// largest too.  Where the row's largest is past the last bin (low temperatures, rows whose
// waves' first are masked) the row is counted again around that one.
template <class R>
MSD_DEV float largest(const R& row, double c, bool count, bool levels, float* ref, ManyLds<R::LB>& s,
                      Group<R::W>& g) {
  if (!count) return of_key(g.max(thread_max(row)));
  float m = row.full || row.part ? unit_max<R>(row.load_tail(0)) : -INFINITY;
#pragma unroll 1
  for (int round = 0;; ++round) {
    for (int i = threadIdx.x; i < s.COUNTS; i += R::LB) s.counts[i] = 0;
    *ref = of_key(g.max(key_of(m)));  // (its barrier: the counts are clear)
    const Bins<R::LB> bins(*ref, c);
    row.template each<4>([&](int j, int, const u32x4& u) {
      float most = -INFINITY;
#pragma unroll
      for (int e = 0; e < R::E; ++e) {
        const float x = from_bits<R::T>(lift<R::T>(u, e));
        most = fmaxf(most, x);
        const uint32_t b = bins.at(x);
        if (b)
          atomicAdd((unsigned long long*)&s.counts[b >> 20], 1ull << PLACE_BITS | (b & 0xFFFFFu));
      }
      m = fmaxf(m, most);
      if (levels) s.levels[j * R::LB + threadIdx.x] = (uint8_t)bins.level(most);
    });
    m = of_key(g.max(key_of(m)));
    if (round || !(fabsf(m) < INFINITY) || bins.at(m) >> 20 < (uint32_t)s.COUNTS - 1) return m;
    lds_barrier();  // before the counts are cleared
  }
}

// What is known before the weights: tokens that surely stay, and the least of the others
// that may (+inf: none, the choice is exact; else those that surely stay are all from a value on).
struct Plan {
  Kept above;
  float low;
};

// The estimate from the counts, bins from the last down.  least: the key that min_p asks for.
template <class R>
MSD_DEV Plan estimate(float ref, const Scale& sc, const LogitsChoice& how, uint32_t least,
                      ManyLds<R::LB>& s, Group<R::W>& g) {
  constexpr int COUNTS = ManyLds<R::LB>::COUNTS, PER = COUNTS / R::LB;
  const Bins<R::LB> bins(ref, sc.c);
  uint32_t n[PER];
  uint64_t w[PER], sum = 0, all;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int b = COUNTS - 1 - (threadIdx.x * PER + i);
    const uint64_t places = s.counts[b] & ((1ull << PLACE_BITS) - 1);
    n[i] = (uint32_t)(s.counts[b] >> PLACE_BITS);
    const float mean = (float)b + (float)places * 0x1p-20f / (float)n[i];
    sum += w[i] = n[i] ? n[i] * bins.weight_at(mean, sc) : 0;
  }
  if (least > KEY_NINF + 1) {
    // Does min_p end before top_p for certain?  Weights at the bins' edges, a hundredth
    // of a bin wider for the rounding of a place, bound those in them.
    const uint32_t at = bins.at(of_key(least));
    const float cut = at ? (float)(at >> 20) - 1.f : -1.f;
    uint64_t most = 0, whole = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const float b = (float)(COUNTS - 1 - (threadIdx.x * PER + i));
      whole += n[i] * bins.weight_at(b - 0.01f, sc);
      if (b >= cut) most += n[i] * bins.weight_at(b < COUNTS - 1 ? b + 1.01f : 2.f * COUNTS, sc);
    }
    most = g.sum(most);
    whole = g.sum(whole);
    if (cut >= 0.f && (double)most < (double)whole * how.top_p * (1 - 0x1p-20))
      return {{least, 0x7FFFFFFF}, INFINITY};
  }
  if (threadIdx.x == 0) {  // where no weight is to be seen
    s.bin = COUNTS - 1;
    s.count = 0;
    s.found[0] = 0;
  }
  uint64_t run = g.before(sum, &all);
  const uint64_t want = (uint64_t)((double)all * how.top_p);
  if (run <= want && want < run + sum) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (run <= want && want < run + w[i]) {
        s.bin = COUNTS - 1 - (threadIdx.x * PER + i);
        s.count = (int)n[i];
        s.found[0] = (uint64_t)((double)(want - run) / (double)w[i] * 0x1p20);
      }
      run += w[i];
    }
  }
  lds_barrier();
  // Around its place in the bin if the bin's tokens lay evenly: a few of their standard
  // deviations (of n in order, 1 / (2 sqrt(n)) at most), and no less than the bins beside
  // it where they are few.
  const float tokens = (float)s.count, down = (float)s.found[0] * 0x1p-20f;
  const float around = tokens > 100.f ? 0.1f + 3.f * rsqrtf(tokens) : 1.5f;
  const float at = (float)(s.bin + 1) - down;
  const float high = bins.edge(at + around);
  Plan p{{0xFF800000u, -1}, bins.edge(at - around)};
  if (at + around < (float)COUNTS && high < sc.m) p.above = {key_of(high), 0x7FFFFFFF};
  // (temperatures whose bins no float tells apart: nothing is listed)
  if (!(fabsf(p.low) < INFINITY) || !(p.low < high)) p = {{0xFF800000u, -1}, 3.402823466e38f};
  return p;
}

// The last token that stays by top-p, of which `want` of the weight is among the C listed;
// false where it is not, or where too many are alike.
template <int LB>
MSD_DEV bool border(ManyLds<LB>& s, int C, const Plan& p, uint64_t want, const Scale& sc, Kept* k,
                    Group<LB / 64>& g) {
  const float high = fminf(of_key(p.above.key), sc.m);
  const float width = high - p.low;
  const float c = width > 0 ? (float)BINS / width : 0.f;
  const auto bin_of = [&](float x) {
    return (int)fminf(fmaxf((high - x) * c, 0.f), (float)(BINS - 1));
  };
  clear_bins<LB / 64>(s.hist);
  if (threadIdx.x == 0) s.count = 0;
  for (int i = threadIdx.x; i < C; i += LB) {
    const float x = of_key((uint32_t)(s.list[i] >> 32));
    atomicAdd((unsigned long long*)&s.hist[bin_of(x)], weight(x, sc));
  }
  lds_barrier();
  uint64_t all;
  find_bin<LB / 64, false>(s.hist, want, &all, g);
  if (want < 1 || want > all) return false;
  const int bin = s.bin;
  want -= s.found[0];
  for (int i = threadIdx.x; i < C; i += LB) {
    const float x = of_key((uint32_t)(s.list[i] >> 32));
    if (bin_of(x) != bin) continue;
    const int at = atomicAdd(&s.count, 1);
    if (at < s.BORDER) {
      s.few[at] = s.list[i];
      s.few_w[at] = weight(x, sc);
    }
  }
  lds_barrier();
  const int n = s.count;
  if (n > s.BORDER) return false;
  for (int i = threadIdx.x; i < n; i += LB) {
    const uint64_t me = s.few[i];
    uint64_t before = 0;
    for (int j = 0; j < n; ++j) before += s.few[j] > me ? s.few_w[j] : 0;
    if (before < want && want <= before + s.few_w[i]) s.found[0] = me;
  }
  lds_barrier();
  *k = {(uint32_t)(s.found[0] >> 32), (int)~(uint32_t)s.found[0]};
  return true;
}

// What of a row's choice does not need its weights.
struct Start {
  static constexpr int LAST = 0x7FFFFFFF;
  Kept limit;      // of top_k; without one the least token above -inf, with id LAST
  uint32_t least;  // of min_p
  Plan plan;
  // (the id tells: the k-th token itself may be the least one)
  MSD_DEV bool limited() const { return limit.id != LAST; }
};
template <class R>
MSD_DEV Start start_many(const R& row, float ref, const Scale& sc, const LogitsChoice& how,
                         ManyLds<R::LB>& s, Group<R::W>& g) {
  const R& mem = row;
  constexpr int LAST = Start::LAST;
  Start st{{KEY_NINF + 1, LAST}, KEY_NINF + 1, {{0xFF800000u, -1}, 3.402823466e38f}};
  if (how.min_d > -INFINITY) st.least = min_key(sc.m, how.min_d);
  const bool limited = how.top_k > 0 && how.top_k < row.V;
  if (limited) {  // (the counts are gone then)
    const Kept f = shortest(mem, nullptr, how.top_k, s.hist, g);
    if (f.key > KEY_NINF) st.limit = f;
  }
  if (how.top_p == 1) {
    st.plan = {st.limit, INFINITY};
    if (st.least > st.limit.key) st.plan.above = {st.least, LAST};
  } else if (!sc.finite) {  // the infinite ones weigh alike
    const Keeps within(st.limit);
    uint64_t n = 0;
    mem.template each<2>([&](int, int i, const u32x4& u) {
#pragma unroll
      for (int e = 0; e < R::E; ++e) {
        const float x = from_bits<R::T>(lift<R::T>(u, e));
        n += x == INFINITY && within(x, i + e);
      }
    });
    n = g.sum(n);
    uint64_t want = (uint64_t)ceil((double)n * how.top_p);
    want = want < 1 ? 1 : want > n ? n : want;
    st.plan = {shortest(mem, nullptr, want, s.hist, g), INFINITY};
  } else if (!limited && fabsf(ref) < INFINITY) {
    st.plan = estimate<R>(ref, sc, how, st.least, s, g);
  }  // else nothing surely stays, and nothing is listed
  clear_count(s);
  return st;
}

// The pass that computes the weights of a row: the sums of all (with !EXACT) and of those
// that surely stay (with ALL: every token), by cells too.  Units that hold tokens that only
// may stay are marked and read again for the list, which they are few of.  f is called for
// each unit.
template <bool EXACT, bool ALL, class R, class F>
MSD_DEV void weigh(const R& row, const Scale& sc, const Start& st, uint64_t* all, uint64_t* above,
                   ManyLds<R::LB>& s, Group<R::W>& g, F f) {
  const Keeps stays(st.plan.above), within(st.limit);
  const float low = st.plan.low;
  const bool limited = !EXACT && st.limited();
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  uint64_t sum_all = 0, sum_above = 0, cell = 0, marked = 0;
  const int pairs = row.per_wave() > 64;  // a mark is of two units
  const auto close = [&](int j) {
    const uint64_t t = wave_scan(cell, (uint64_t)0, Sum());
    if (lane == 63) s.cells[wave * (CELLS / 16) + j / GROUP] = t;
    sum_above += cell;
    cell = 0;
  };
  row.template each<2>([&](int j, int i, const u32x4& u) {
    float x[R::E];
    bool in[R::E], any = false, may = false;
#pragma unroll
    for (int e = 0; e < R::E; ++e) x[e] = from_bits<R::T>(lift<R::T>(u, e));
    if (limited) {
#pragma unroll
      for (int e = 0; e < R::E; ++e)
        if (!within(x[e], i + e)) x[e] = -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < R::E; ++e) {
      in[e] = ALL || (EXACT ? stays(x[e], i + e) : x[e] >= stays.x);
      any |= in[e];
      if (!EXACT) may |= x[e] >= low && !in[e];
    }
    if (!EXACT) marked |= (uint64_t)may << (j >> pairs);
    if (ALL || !EXACT || __any(any)) {
      float z[R::E];
#pragma unroll
      for (int e = 0; e < R::E; ++e) z[e] = x[e];
      if (EXACT && !sc.finite) {
#pragma unroll
        for (int e = 0; e < R::E; ++e) z[e] = sc(x[e]);
      }
#pragma unroll
      for (int h = 0; h < R::E; h += 4) {  // in fours: registers for their arithmetic
        if (h) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int e = h; e < h + 4; ++e) {
          const uint64_t w = bits_of(z[e], sc);
          if (!EXACT) sum_all += w;
          cell += in[e] ? w : BITS_128;
        }
      }
      cell -= R::E * BITS_128;
      if (!EXACT) sum_all -= R::E * BITS_128;
    }
    if (j % GROUP == GROUP - 1) close(j);
    f(i, u, x, in);
  });
  const int n = row.full + row.part;
  if (n % GROUP) close(n - 1);
  if (!EXACT) {
    for (; marked; marked &= marked - 1) {
      const int j0 = (__ffsll((unsigned long long)marked) - 1) << pairs;
      for (int j = j0; j <= j0 + pairs && j < row.full + row.part; ++j)
        append(row, row.id(j), row.load_tail(j), s.list, s.LIST, s, [&](float v, int id) {
          return v >= low && !(v >= stays.x) && (!limited || within(v, id));
        });
    }
    *all = g.sum(sum_all);
  }
  *above = g.sum(sum_above);  // (its barrier: the list and the cells are whole)
}

// The last token that stays, after a plan's weights; false where it had to be looked for
// in passes of their own.
template <class R>
MSD_DEV bool decide(const R& row, const Scale& sc, const LogitsChoice& how, const Start& st,
                    uint64_t all, uint64_t above, int C, Kept* k, ManyLds<R::LB>& s, Group<R::W>& g) {
  uint64_t want = (uint64_t)ceil((double)all * how.top_p);
  want = want < 1 ? 1 : want > all ? all : want;
  const bool found = C <= s.LIST && want > above &&
                     border<R::LB>(s, C, st.plan, want - above, sc, k, g);
  if (!found) *k = shortest(row, &sc, want, s.hist, g);
  if (st.least > k->key) *k = {st.least, 0x7FFFFFFF};
  return found;
}

// ------------------------------------------------------------------- operators ----

// The row's logits that stay, -inf for the others; their number over the threads.
template <class R>
MSD_DEV uint32_t put_filtered(const R& row, char* o, Kept k) {
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
  return n;
}

// The row's first reading for a few first tokens: its largest and its threads', no weights.
template <class R>
MSD_DEV Tops read_tops(R& row, int n, Group<R::W>& g) {
  float mine = -INFINITY;
  row.read([&](const u32x4& u) {
    const float m = unit_max<R>(u);
    mine = fmaxf(mine, m);
    return m;
  });
  return tops(key_of(mine), (min(n, row.V) + R::W - 1) / R::W, g);
}

// Filter with a small top_k: one reading of the row, its writing, and the units with one of
// the tokens read again.  Bound by HBM: 488 x 152,064 f32, top_k 50, 594 MB in 122 us, 4.9
// TB/s, the rate of a large copy (133 -> 120 us against every unit read again).
template <class R>
__global__ __launch_bounds__(R::LB) void k_filter_few(const void* logits, size_t ld, int V,
                                                      LogitsChoice how, void* out, size_t ldo,
                                                      int* kept) {
  __shared__ FewLds s;
  Group<R::W> g{s};
  R row(logits, ld, V);
  char* const o = static_cast<char*>(out) + (size_t)blockIdx.x * ldo * Type<R::T>::SIZE;
  if (threadIdx.x == 0) s.count = 0;
  const Tops t = read_tops(row, how.top_k, g);
  Kept k{0xFF800000u, -1};  // nothing: +inf of no id
  int n = 0;
  if (t.max > KEY_NINF) {
    uint64_t all;
    n = choose_few(row, t, Scale(of_key(t.max), how.c), how, &all, s, g);
    const uint64_t last = s.sorted[n - 1];
    k = {(uint32_t)(last >> 32), (int)~(uint32_t)last};
  }
  // the few units with one of them are read again, and stored in their place
  const uint64_t units = row.reach(of_key(k.key));
  const Keeps stays(k);
  for (int j = 0; j < row.full + row.part; ++j) {
    u32x4 y = Type<R::T>::NINF;
    if (units >> j & 1) {
      const u32x4 u = row.load_tail(j);
#pragma unroll
      for (int e = 0; e < R::E; ++e)
        if (stays(from_bits<R::T>(lift<R::T>(u, e)), row.id(j) + e)) lower<R::T>(y, e, lift<R::T>(u, e));
    }
    row.store(o, row.id(j), y);
  }
  if (kept && threadIdx.x == 0) kept[blockIdx.x] = n;
}

// The same where the units' levels tell which of them to read: under min_p most hold no
// token that stays, so that the row is read once (filter of 488 x 152,064 f32, top_p 0.98 and
// min_p 0.02: 177 us with every unit read again -> 162 with levels).
template <class R>
MSD_DEV uint32_t put_leveled(const R& row, char* o, Kept k, const Bins<R::LB>& bins, const ManyLds<R::LB>& s) {
  constexpr int AHEAD = 4;
  const Keeps stays(k);
  const uint32_t level = bins.level(stays.x);
  const int units = row.full + row.part;
  uint32_t n = 0;
  for (int j0 = 0; j0 < units; j0 += AHEAD) {
    u32x4 u[AHEAD];
#pragma unroll
    for (int b = 0; b < AHEAD; ++b) {
      u[b] = Type<R::T>::NINF;
      if (j0 + b < units && s.levels[(j0 + b) * R::LB + threadIdx.x] >= level)
        u[b] = row.load_tail(j0 + b);
    }
#pragma unroll
    for (int b = 0; b < AHEAD; ++b) {
      if (j0 + b >= units) break;
      const int i = row.id(j0 + b);
#pragma unroll
      for (int e = 0; e < R::E; ++e) {
        const bool in = stays(from_bits<R::T>(lift<R::T>(u[b], e)), i + e);
        if (!in) lower<R::T>(u[b], e, Type<R::T>::NINF & (R::T == MX_F32 ? ~0u : 0xFFFFu));
        n += in;
      }
      row.store(o, i, u[b]);
    }
  }
  return n;
}

// Filter with any number of tokens that stay: a pass that counts, one that weighs and (where
// the output is not the input) writes all that may stay, and the few near the border masked
// in it.  Many rows are bound by HBM and by the weights' arithmetic, which the two rows of a
// CU overlap in part: 488 x 152,064 f32, min_p 0.02 and top_p 0.98, 164 us, 3.6 TB/s of what
// has to move (119 us at a copy's rate); 27 x 32,000 f32 25 us, of one CU's arithmetic on a
// row (at the instructions' rates 7 us of weights and 2 of counts) and a chain with 17
// barriers: 27 x 8,200 takes 17 us, and 1,000 more logits 0.4.
template <class R>
__global__ __launch_bounds__(R::LB) void k_filter_many(const void* logits, size_t ld, int V,
                                                       LogitsChoice how, void* out, size_t ldo,
                                                       int* kept) {
  __shared__ ManyLds<R::LB> s;
  Group<R::W> g{s};
  const R row(logits, ld, V);
  char* const o = static_cast<char*>(out) + (size_t)blockIdx.x * ldo * Type<R::T>::SIZE;
  float ref = 0.f;
  // min_p leaves few tokens, so that most units need not be read again
  const bool levels = how.min_d > -INFINITY && row.per_wave() * R::LB <= s.LEVELS;
  const float m = largest(row, how.c, how.top_p < 1 || levels, levels, &ref, s, g);
  Kept k{0xFF800000u, -1};  // nothing: +inf of no id
  bool known = false;
  if (m > -INFINITY) {
    const Scale sc(m, how.c);
    const Start st = start_many(row, ref, sc, how, s, g);
    k = st.plan.above;
    known = levels && fabsf(ref) < INFINITY && st.plan.low == INFINITY;
    if (st.plan.low < INFINITY) {
      // the pass writes as well, but in place, where the row may have to be read again
      const bool write = out != logits;
      uint64_t all, above;
      uint32_t n = 0;
      weigh<false, false>(
            row, sc, st, &all, &above, s, g,
            [&](int i, const u32x4& u, const float(&x)[R::E], const bool(&in)[R::E]) {
              if (!write) return;
              u32x4 y = u;
#pragma unroll
              for (int e = 0; e < R::E; ++e) {
                if (!(in[e] || x[e] >= st.plan.low))
                  lower<R::T>(y, e, Type<R::T>::NINF & (R::T == MX_F32 ? ~0u : 0xFFFFu));
                n += in[e];
              }
              row.store(o, i, y);
            });
      const int C = s.count;
      if (decide(row, sc, how, st, all, above, C, &k, s, g) && write &&
          (k.key < st.plan.above.key || (k.key == st.plan.above.key && k.id >= st.plan.above.id))) {
        // of those that may stay, the ones that do not
        const Keeps stays(k);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the row's stores are done
        __syncthreads();
        for (int i = threadIdx.x; i < C; i += R::LB) {
          const int id = (int)~(uint32_t)s.list[i];
          const bool in = stays(of_key((uint32_t)(s.list[i] >> 32)), id);
          if (!in) put_bits<R::T>(o, id, Type<R::T>::NINF);
          n += in;
        }
        const uint64_t total = g.sum((uint64_t)n);
        if (kept && threadIdx.x == 0) kept[blockIdx.x] = (int)total;
        return;
      }
    }
  }
  const uint64_t n = g.sum((uint64_t)(known ? put_leveled(row, o, k, Bins<R::LB>(ref, how.c), s)
                                            : put_filtered(row, o, k)));
  if (kept && threadIdx.x == 0) kept[blockIdx.x] = (int)n;
}

// The place of u in a whole of `all`.
MSD_DEV uint64_t drawn(float u, uint64_t all) {
  return u >= 1.f ? all - 1 : u > 0.f ? (uint64_t)((double)u * (double)all) : 0;
}
MSD_DEV void put_token(int id, float x, uint64_t all, const Scale& sc, int* tokens,
                       float* logprobs) {
  tokens[blockIdx.x] = id;
  if (logprobs)
    logprobs[blockIdx.x] = (float)((x == sc.m ? 0.0 : ((double)x - sc.m64) * sc.c * M_LN2) -
                                   log((double)all * (1 / ONE)));
}
MSD_DEV void put_no_token(int* tokens, float* logprobs, bool keep) {
  if (threadIdx.x) return;
  if (!keep) tokens[blockIdx.x] = -1;
  if (logprobs) logprobs[blockIdx.x] = -INFINITY;
}

// Sample with a small top_k: as the filter's, and the draw among the ranked tokens in the
// order of their ids.  One row on a CU takes the latency of its chain and what one CU reads:
// 64 x 152,064 bf16, top_k 50, 16 us for 304 KB a CU.
template <class R>
__global__ __launch_bounds__(R::LB) void k_sample_few(const void* logits, size_t ld, int V,
                                                      LogitsChoice how, const float* uniforms,
                                                      int* tokens, float* logprobs, bool keep) {
  __shared__ FewLds s;
  Group<R::W> g{s};
  const float u = uniforms[blockIdx.x];
  R row(logits, ld, V);
  if (threadIdx.x == 0) s.count = 0;
  const Tops t = read_tops(row, how.top_k, g);
  if (t.max <= KEY_NINF) return put_no_token(tokens, logprobs, keep);
  const Scale sc(of_key(t.max), how.c);
  uint64_t all;
  const int n = choose_few(row, t, sc, how, &all, s, g);
  if ((int)threadIdx.x >= n) return;
  // the running sum in the order of the ids, of which ~ makes the lower the greater
  const uint32_t me = (uint32_t)s.sorted[threadIdx.x];
  uint64_t before = 0;
  for (int i = 0; i < n; ++i) before += (uint32_t)s.sorted[i] > me ? s.weights[i] : 0;
  const uint64_t at = drawn(u, all);
  if (before <= at && at < before + s.weights[threadIdx.x])
    put_token((int)~me, of_key((uint32_t)(s.sorted[threadIdx.x] >> 32)), all, sc, tokens, logprobs);
}

// Sample with any number of tokens that stay: a pass that counts, one that weighs, and the
// sums of 2,048 or 4,096 neighbouring ids (a cell) tell where to read again for the draw;
// without top_p a pass for the largest and one for the weights.  Rows are in runs, not in
// tiles, so that a wave's cell is of neighbouring ids.  Bound by the arithmetic of the
// weights with the first pass's HBM time not hidden by it: 512 x 152,064 f32, top_p 0.95, 150
// us (62 us for its bytes once at a copy's rate, 44 at a read's; about 70 us for 78 million
// weights on 256 CUs at the instructions' rates).  A row alone: 1 x 32,000 f32 without a choice
// 13 to 15 us, by its inputs.
//   Few rows take one CU each all the same (8 x 152,064 f32, top_p: 71 us); a row over several
// workgroups would need memory of the caller's and two more launches or a grid's barrier.
template <class R>
__global__ __launch_bounds__(R::LB) void k_sample_many(const void* logits, size_t ld, int V,
                                                       LogitsChoice how, const float* uniforms,
                                                       int* tokens, float* logprobs, bool keep) {
  __shared__ ManyLds<R::LB> s;
  Group<R::W> g{s};
  const float u = uniforms[blockIdx.x];
  const R row(logits, ld, V);
  for (int i = threadIdx.x; i < CELLS; i += R::LB) s.cells[i] = 0;
  float ref = 0.f;
  const float m = largest(row, how.c, how.top_p < 1, false, &ref, s, g);
  if (!(m > -INFINITY)) return put_no_token(tokens, logprobs, keep);
  const Scale sc(m, how.c);
  const Start st = start_many(row, ref, sc, how, s, g);
  Kept k = st.plan.above;
  uint64_t all, above;
  const auto nothing = [](int, const u32x4&, const float(&)[R::E], const bool(&)[R::E]) {};
  const int w = threadIdx.x >> 6;
  bool exact = st.plan.low == INFINITY;
  if (!exact) {
    weigh<false, false>(row, sc, st, &all, &above, s, g, nothing);
    const int C = s.count;
    if (decide(row, sc, how, st, all, above, C, &k, s, g) && st.least <= st.plan.above.key) {
      const Keeps stays(k);
      for (int i = threadIdx.x; i < C; i += R::LB) {
        const float x = of_key((uint32_t)(s.list[i] >> 32));
        const int id = (int)~(uint32_t)s.list[i];
        const int q = id / R::STRETCH, wave = q / row.per_wave();
        const int cell = wave * (CELLS / 16) + (q - wave * row.per_wave()) / GROUP;
        if (stays(x, id)) atomicAdd((unsigned long long*)&s.cells[cell], weight(x, sc));
      }
    } else {
      exact = true;
    }
    lds_barrier();
  }
  if (exact) {
    for (int i = threadIdx.x; i < CELLS; i += R::LB) s.cells[i] = 0;
    lds_barrier();
    const Start chosen{{KEY_NINF + 1, Start::LAST}, KEY_NINF + 1, {k, INFINITY}};
    if (k.key == KEY_NINF + 1 && k.id >= V)
      weigh<true, true>(row, sc, chosen, &all, &above, s, g, nothing);
    else
      weigh<true, false>(row, sc, chosen, &all, &above, s, g, nothing);
  }
  // the cell that holds the place
  const uint64_t h = (int)threadIdx.x < CELLS ? s.cells[threadIdx.x] : 0;
  uint64_t run = g.before(h, &all);
  const uint64_t at = drawn(u, all);
  if (run <= at && at < run + h) {
    s.bin = threadIdx.x;
    s.found[0] = run;
  }
  lds_barrier();
  if (s.bin / (CELLS / 16) != w) return;
  const Keeps stays(k);
  run = s.found[0];
  const int from = __builtin_amdgcn_readfirstlane(s.bin % (CELLS / 16) * GROUP);
  for (int j = from; j < from + GROUP && run <= at; ++j) {
    const u32x4 un = row.load_tail(j);
    uint64_t ws[R::E], sum = 0;
#pragma unroll
    for (int e = 0; e < R::E; ++e) {
      const float x = from_bits<R::T>(lift<R::T>(un, e));
      ws[e] = stays(x, row.id(j) + e) ? weight(x, sc) : 0;
      sum += ws[e];
    }
    const uint64_t in = wave_scan(sum, (uint64_t)0, Sum());
    uint64_t before = run + in - sum;
#pragma unroll
    for (int e = 0; e < R::E; ++e) {
      if (before <= at && at < before + ws[e])
        put_token(row.id(j) + e, from_bits<R::T>(lift<R::T>(un, e)), all, sc, tokens, logprobs);
      before += ws[e];
    }
    run += __shfl((unsigned long long)in, 63);
  }
}

// The thread's largest logit, and its sum of e^((x - m) / T), c = log2(e) / T: a unit at a
// time, the sum brought to a new largest one when that comes.
struct Online {
  float m = -INFINITY, sum = 0.f;
};
MSD_DEV float exp_of(float x, float m, float c) { return __builtin_amdgcn_exp2f((x - m) * c); }
// Another unit; its largest.
template <bool NO_NAN, class R>
MSD_DEV float add_unit(Online& o, const u32x4& u, float c) {
  float x[R::E], top = -INFINITY;
#pragma unroll
  for (int e = 0; e < R::E; ++e) {
    x[e] = from_bits<R::T>(lift<R::T>(u, e));
    if (NO_NAN) x[e] = fmaxf(x[e], -INFINITY);
    top = fmaxf(top, x[e]);
  }
  const float m = fmaxf(o.m, top);
  const float from = m > -INFINITY ? m : 0.f;  // (no inf - inf where all are masked)
  float sum = o.sum * exp_of(o.m, from, c);
#pragma unroll
  for (int e = 0; e < R::E; ++e) sum += exp_of(x[e], from, c);
  o = {m, sum};
  return top;
}
// The same of the row, whose largest is m.
template <int W>
MSD_DEV double row_sum(const Online& o, float m, float c, Group<W>& g) {
  return g.sum(o.sum == 0.f ? 0.0 : (double)(o.sum * exp_of(o.m, m, c)));
}

// Top: one reading of the row, with its log-sum-exp (32-bit sums a thread, 64-bit over the
// row), and the ranking.  Many rows are bound by HBM: 1,151 x 152,064 bf16, k 128, 350 MB in
// 106 us, 3.3 TB/s, two rows to a CU (103 registers; fewer maxima a thread, for three, have
// not been tried), of which the ranking of one hides behind the reading of the other in part;
// 639 x 32,000 f32, k 64, 82 MB in 23 us, all rows resident, three to a CU at most: about 6 us
// of chain, then 4.3 TB/s (k 1 takes 1.5 us less).  Few rows by the chain: 61 x 50,021 f16, k
// 200, 15 us; 1 x 32,000 f32 8 us.
template <class R>
__global__ __launch_bounds__(R::LB) void k_top(const void* logits, size_t ld, int V, int n,
                                               float* values, int* ids, float* lse) {
  __shared__ FewLds s;
  Group<R::W> g{s};
  R row(logits, ld, V);
  if (threadIdx.x == 0) s.count = 0;
  constexpr float c = (float)M_LOG2E;
  Online on;
  row.read([&](const u32x4& u) { return add_unit<true, R>(on, u, c); });
  const Tops t = tops(key_of(on.m), (n + R::W - 1) / R::W, g);
  const float m = of_key(t.max);
  if (lse) {
    const double sum = row_sum(on, m, c, g);
    if (threadIdx.x == 0)
      lse[blockIdx.x] = fabsf(m) < INFINITY ? (float)((double)m + log(sum)) : m;
  }
  first_tokens<true>(row, t, n, s, g);
  if ((int)threadIdx.x < n) {
    const size_t o = (size_t)blockIdx.x * n + threadIdx.x;
    const uint64_t top = s.sorted[threadIdx.x];
    values[o] = of_key((uint32_t)(top >> 32));
    ids[o] = (int)~(uint32_t)top;
  }
}

// A row's teacher entry of this thread (id < 0: none).
struct Entry {
  int id;
  float value;
  double lq, q;
};

// q = softmax(t / T) over the row's entries, the first k threads'; all zero where none has
// a value above -inf, NaN where one is NaN or +inf.  Returns 1, 0 or NaN in these cases.
template <int W>
MSD_DEV double soften(Entry& e, int k, double inv_t, Group<W>& g) {
  const float top = of_key(g.max(key_of(e.value)));
  double d = 0, w = 0;
  if ((int)(threadIdx.x & ~63u) < k) {
    d = ((double)e.value - (double)top) * inv_t;
    w = e.value == -INFINITY ? 0 : exp(d);
  }
  const double sum = g.sum(w);
  e.lq = e.q = 0;
  if (w != 0) {
    e.lq = d - log(sum);
    e.q = w / sum;
  }
  return sum == 0 ? 0 : sum == sum ? 1 : sum;
}

// The entries as they meet the row's units: by the thread whose unit has their id, chained.
struct Chains {
  int id[LOGITS_TOP_MAX], next[LOGITS_TOP_MAX];
  double q[LOGITS_TOP_MAX];
  float gq[LOGITS_TOP_MAX];  // its part of the gradient
  int head[1024];
};

// Distillation, loss and gradient in one pass or either alone: the loss is
//   sum q (log q - log p) = sum q (log q - (x - m) / T + log sum e^((x - m) / T)),
// so it takes the row's sum and the entries' logits only; the gradient g / T (p - q) is p's
// for every column and q's at the entries, which the thread that writes their unit takes off
// before it rounds: no second write, no atomics on the output.  Sums and weights in 32 bits
// within a thread, in 64 over the row (a weight below 2^-126 of the largest is 0); the
// gradient recomputes its sum, since a row is held anyway.  Bound by HBM: 639 x 32,000 f32
// 164 MB in 43 us (3.8 TB/s: two rows to a CU, so 639 are 512 and a tail of 127), 1,151 x
// 152,064 bf16 700 MB in 183 us (3.8 TB/s: a row to a CU, whose registers it fills, 4.5
// rounds), the loss alone 66 us (5.3 TB/s).
template <class R>
__global__ __launch_bounds__(R::LB) void k_distill(const void* logits, size_t ld, int V,
                                                   LogitsTeacher t, float* loss, float* lse,
                                                   const float* grad, void* dx, size_t ldd) {
  __shared__ Lds s;
  __shared__ Chains ch;
  Group<R::W> g{s};
  Entry e{-1, -INFINITY, 0, 0};
  const int lane_k = threadIdx.x;
  if (lane_k < t.k) {
    const size_t o = (size_t)blockIdx.x * t.k + lane_k;
    e.id = t.ids[o];
    if (e.id < 0 || e.id >= V) e.id = -1;
    if (e.id >= 0) e.value = t.values[o];
  }
  const R row(logits, ld, V);
  const float zk = e.id >= 0 ? from_bits<R::T>(bits_at<R::T>(row.p, e.id)) : 0.f;
  const float gr = grad ? grad[blockIdx.x] : 0.f;
  const double mass = soften(e, t.k, t.inv_t, g);
  const float f = (float)(gr * t.inv_t * mass);
  ch.head[threadIdx.x] = -1;
  if (lane_k < t.k) {
    ch.id[lane_k] = e.id;
    ch.q[lane_k] = e.q;
  }
  lds_barrier();
  if (dx && e.id >= 0) {
    // the first entry of an id carries the others'
    double q = 0;
    bool first = true;
    for (int i = 0; i < t.k; ++i) {
      if (ch.id[i] != e.id) continue;
      first = first && i >= lane_k;
      q += ch.q[i];
    }
    if (first) {
      ch.gq[lane_k] = (float)(f * q);
      ch.next[lane_k] = atomicExch(&ch.head[e.id / R::E % R::LB], lane_k);
    }
  }
  const float c = (float)(t.inv_t * M_LOG2E);
  Online on;
  row.template each<4>([&](int, int, const u32x4& u) { add_unit<false, R>(on, u, c); });
  // the entries' logits are read before a gradient in their place is written
  asm volatile("" ::"v"(zk));
  // (a NaN is passed over here and found again by the sum)
  const float m = of_key(g.max(key_of(on.m)));
  const double sum = row_sum(on, m, c, g);
  if (dx) {
    char* const o = static_cast<char*>(dx) + (size_t)blockIdx.x * ldd * Type<R::T>::SIZE;
    const float fs = f / (float)sum;
    const int head = ch.head[threadIdx.x];
    row.template each<4>([&](int, int i, const u32x4& u) {
      float y[R::E];
#pragma unroll
      for (int q = 0; q < R::E; ++q) {
        y[q] = fs * exp_of(from_bits<R::T>(lift<R::T>(u, q)), m, c);
        if (mass == 0) y[q] = 0.f;
      }
      for (int k = head; k >= 0; k = ch.next[k]) {
        const int at = ch.id[k] - i;
        const float gq = ch.gq[k];
#pragma unroll
        for (int q = 0; q < R::E; ++q) y[q] -= at == q ? gq : 0.f;
      }
      row.store(o, i, pack<R::T>(y));
    });
  }
  if (!loss && !lse) return;
  const bool mine = (int)(threadIdx.x & ~63u) < t.k;
  double l = 0;
  const double ls = mine ? log(sum) : 0;
  if (mine && e.q != 0) l = e.q * (e.lq - (((double)zk - (double)m) * t.inv_t - ls));
  l = g.sum(l);
  if (threadIdx.x) return;
  if (loss) loss[blockIdx.x] = (float)l;
  if (lse) lse[blockIdx.x] = (float)(m * t.inv_t + ls);
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

template <class R>
struct Tag {
  using type = R;
};

// Rows of up to this many bytes take a workgroup of 256 threads: several share a CU, and a
// row has as few barriers' waits.  Against 1024 threads, us: top 64 of 3,000 x 1,000 f32 20
// (89) and of 3,000 x 8,192 32 (79), filter by top_p 41 (133) and 82 (180), sample by top_p
// of 3,000 x 1,000 47 (157), gradients 23 (109) and 43 (122).  Of 61 rows of 8,192, for which
// the rule is the same: top 8.9 (9.3), filter 18.4 (17.0), gradient 14.3 (12.6).
constexpr int SHORT_ROW = 256 * 8 * 16;

template <class R>
bool holds(int cols) {
  return cols / R::TILE <= R::UNITS;
}

// Calls f with the type for a row of `cols` that is held: by 256 threads if it is short; by
// 512, two rows to a CU, where there are more rows than CUs (639 x 32,000 f32 43 us, by 1024
// 49); by 1024; or read from memory in every pass, where no registers hold it.  A long row
// of 18 units that is read twice instead of held is no slower (1,151 x 152,064 bf16, 250 us
// for 248 in two calls) but reads half as much again.
template <int TYPE, class F>
void by_held(int rows, int cols, F f) {
  using Short = HeldRow<TYPE, 256, 8>;
  using Two = HeldRow<TYPE, 512, 16>;
  using One = HeldRow<TYPE, 1024, 8>;
  using LongOne = HeldRow<TYPE, 1024, 18>;
  if (cols * Type<TYPE>::SIZE <= SHORT_ROW) return f(Tag<Short>());
  if (rows > 256 && holds<Two>(cols)) return f(Tag<Two>());
  if (holds<One>(cols)) return f(Tag<One>());
  if (holds<LongOne>(cols)) return f(Tag<LongOne>());
  f(Tag<HeldRow<TYPE, 1024, 0>>());
}

// The same of rows that keep their units' largest.  512 threads against 1024 where there are
// more rows than CUs: 639 x 32,000 f32 23.5 us (29.8), 300 x 32,000 15.5 (19.3), 1,151 x
// 152,064 bf16 106 (114).
template <int TYPE, class F>
void by_tops(int rows, int cols, int k, F f) {
  constexpr int MOST = LOGITS_MAX_COLS / (1024 * Type<TYPE>::E);
  using Short = ToppedRow<TYPE, 256, 8, 8>;
  // rows that share a CU hide each other's reading; a row alone has all of it under way
  using Two = ToppedRow<TYPE, 512, 16, 8>;
  using LongTwo = ToppedRow<TYPE, 512, 38, 6>;
  using One = ToppedRow<TYPE, 1024, 8, 8>;
  using LongOne = ToppedRow<TYPE, 1024, 18, 18>;
  // (more than a quarter of the threads' largest bound too long a list: top 250 of 26 x
  // 15,400 bf16 takes 62 us with 256 threads, 14 with 1024)
  if (cols * Type<TYPE>::SIZE <= SHORT_ROW && k <= 64) return f(Tag<Short>());
  if (rows > 256 && holds<Two>(cols)) return f(Tag<Two>());
  if (rows > 256 && holds<LongTwo>(cols)) return f(Tag<LongTwo>());
  if (holds<One>(cols)) return f(Tag<One>());
  if (holds<LongOne>(cols)) return f(Tag<LongOne>());
  if constexpr (MOST > 38)
    if (holds<ToppedRow<TYPE, 1024, 38, 10>>(cols)) return f(Tag<ToppedRow<TYPE, 1024, 38, 10>>());
  f(Tag<ToppedRow<TYPE, 1024, MOST, MOST / 8, MOST / 32>>());
}

// The same of rows that take any number of tokens: 512 threads against 1024 where there are
// more rows than CUs: sample by top_p of 640 x 32,000 f32 70 us (94), of 512 x 152,064 152
// (168); filter by top_p of 640 x 32,000 66 (83), of 488 x 152,064 176 (193), by min_p 127
// (129), but by both, where levels spare a reading, 162 (151).
template <int TYPE, class F>
void by_runs(int rows, int cols, F f) {
  if (cols * Type<TYPE>::SIZE <= SHORT_ROW)
    f(Tag<Row<TYPE, 256, true>>());
  else if (rows > 256)
    f(Tag<Row<TYPE, 512, true>>());
  else
    f(Tag<Row<TYPE, 1024, true>>());
}

}  // namespace

void launch_logits_top(const void* x, int type, size_t ld, int rows, int cols, int k, float* values,
                       int* ids, float* lse, hipStream_t st) {
  if (rows <= 0) return;
  by_type(type, [&](auto t) {
    by_tops<t()>(rows, cols, k, [&](auto r) {
      using R = typename decltype(r)::type;
      k_top<R><<<rows, R::LB, 0, st>>>(x, ld, cols, k, values, ids, lse);
    });
  });
}

void launch_logits_sample(const void* x, int type, size_t ld, int rows, int cols,
                          const LogitsChoice& how, const float* uniforms, int* tokens,
                          float* logprobs, hipStream_t st, bool keep) {
  if (rows <= 0) return;
  const bool few = how.top_k > 0 && how.top_k <= LOGITS_TOP_MAX;
  by_type(type, [&](auto t) {
    if (few)
      by_tops<t()>(rows, cols, how.top_k, [&](auto r) {
        using R = typename decltype(r)::type;
        k_sample_few<R><<<rows, R::LB, 0, st>>>(x, ld, cols, how, uniforms, tokens, logprobs, keep);
      });
    else
      by_runs<t()>(rows, cols, [&](auto r) {
        using R = typename decltype(r)::type;
        k_sample_many<R><<<rows, R::LB, 0, st>>>(x, ld, cols, how, uniforms, tokens, logprobs, keep);
      });
  });
}

void launch_logits_filter(const void* x, int type, size_t ld, int rows, int cols,
                          const LogitsChoice& how, void* out, size_t ldo, int* kept,
                          hipStream_t st) {
  if (rows <= 0) return;
  const bool few = how.top_k > 0 && how.top_k <= LOGITS_TOP_MAX;
  by_type(type, [&](auto t) {
    if (few)
      by_tops<t()>(rows, cols, how.top_k, [&](auto r) {
        using R = typename decltype(r)::type;
        k_filter_few<R><<<rows, R::LB, 0, st>>>(x, ld, cols, how, out, ldo, kept);
      });
    else
      by_runs<t()>(rows, cols, [&](auto r) {
        using R = typename decltype(r)::type;
        k_filter_many<R><<<rows, R::LB, 0, st>>>(x, ld, cols, how, out, ldo, kept);
      });
  });
}

void launch_logits_distill(const void* x, int type, size_t ld, int rows, int cols,
                           const LogitsTeacher& t_, float* loss, float* lse, const float* grad,
                           void* dx, size_t ldd, hipStream_t st) {
  if (rows <= 0) return;
  by_type(type, [&](auto t) {
    const auto run = [&](auto r) {
      using R = typename decltype(r)::type;
      k_distill<R><<<rows, R::LB, 0, st>>>(x, ld, cols, t_, loss, lse, grad, dx, ldd);
    };
    // without a gradient a row is read once, and need not be held (1,151 x 152,064 bf16 66
    // us, with 1024 threads and held rows 104)
    if (!dx && rows > 256 && cols * Type<t()>::SIZE > SHORT_ROW)
      run(Tag<HeldRow<t(), 512, 0>>());
    else
      by_held<t()>(rows, cols, run);
  });
}

}  // namespace msd
