// One optimizer step over many tensors (AdamW, moments in 32 bits or in 8) and the 2-norm of their gradients.
//
//   g' = factor g,  m = beta1 m + (1 - beta1) g',  v = beta2 v + (1 - beta2) g'^2
//   p = p - lr decay p - (lr / c1) m / (sqrt(v / c2) + eps),   c = 1 - beta^step
//
// Every element is read once and written once and shares nothing with another, so the step is bound by memory.  The tensors'
// addresses and sizes travel in the launch's arguments: a captured graph holds them, and no copy has to arrive before the
// kernel may start.  Warps take units of up to eight blocks of 256 elements, one after the other over all tensors: what runs at a
// time then lies in a few pages (a run of its own for every CTA: 1465 instead of 955 us for the bare traffic of 492M bf16 weights with
// 8-bit moments).  Two CTAs on a multiprocessor are enough where every thread has 100 bytes and more on their way.
//
// Measured, of a plain copy's 6.5 TB/s: 246M fp16 weights with binary32 copies and moments 1105 us (0.95), 492M bf16 weights with
// 8-bit moments 934 to 993 us (0.76 to 0.81), where instruction issue (0.6, 44 instructions an element, a sixth of them the hash) and
// memory share the time: 865 us without the arithmetic, 950 us without the hash.  13M weights in tensors of any length 47 us (0.42).  8-bit moments
// of 246M weights beside binary32 copies 685 to 696 us (0.87), of binary32 weights 655 to 674 us (0.9), with binary32 gradients of bf16 weights without a
// copy 623 to 736 us (0.61 to 0.72): their rings hold one block a piece.
//
// Moments in 8 bits.  256 elements are a block with one scale per moment: the smallest power of two that keeps the
// block's largest magnitude in the format (m e4m3, up to 1.75 * 2^8; v e5m2, up to 1.75 * 2^15).  Powers of two, since scaling by them
// rounds nothing.  v changes by a thousandth of itself in a step, less than a hundredth of the distance between two values of
// e5m2: rounded to the nearest it would never move.  So roundings are random: the value goes to its upper neighbour where
// its place between the two and a random fraction add up to one, 16 bits each for m and v from a hash of the element's index and the step
// (two multiplications; a Weyl sequence over the steps is cheaper, but what v becomes depends on the sequence's past, and
// v then falls 13 percent too fast).  In the bits of a binary32 that is one addition below the last bit that is kept.
// This step's p goes by the m and v before they are rounded.  The products and sums of m and v are rounded one by one (no fused
// multiply-add), so that the stored codes are a matter of the formula and not of the compiler.  A block's values come through a ring in
// shared memory (loads ahead in registers are put off by the compiler until they are needed: 1080 us), and the scales of eight blocks
// leave as one sector (a scale at a time: 130 us more).

#include "aq_stage.h"
#include "aq_stage_device.cuh"

#include <type_traits>

namespace aq {
namespace {

constexpr int kAdamThreads = 256, kAdamWarps = kAdamThreads / 32;
constexpr int kAdamCtas = 2, kNormCtasPerSm = 4;    // CTAs on a multiprocessor
constexpr uint32_t kRoot3 = 0xBB67AE85u, kGolden = 0x9E3779B9u;   // fractions of the square root of 3 and of the golden ratio, times 2^32

template <int N> struct Table {
  AdamPart part[N];
  int first[N + 1];                           // units of the tensors before this one
  int n;
  uint32_t unit;                              // elements that a warp takes at a time, blocks of 256
};

// ---- eight elements of a lane: neighbours by one access of up to 32 bytes, or every 32nd element one by one ---------------

template <typename T> struct Eight {            // 16-bit types: two to a word
  static constexpr int W = 4;
  static __device__ void load(const T* p, uint32_t* w) {
    asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
  }
  static __device__ void store(T* p, const uint32_t* w) {
    asm volatile("st.global.L1::no_allocate.v4.b32 [%4], {%0, %1, %2, %3};" ::"r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "l"(p) : "memory");
  }
  static __device__ void load_one(const T* p, int j, uint32_t* w) { w[j / 2] |= (uint32_t)*reinterpret_cast<const uint16_t*>(p) << (16 * (j & 1)); }
  static __device__ void store_one(T* p, int j, const uint32_t* w) { *reinterpret_cast<uint16_t*>(p) = (uint16_t)(w[j / 2] >> (16 * (j & 1))); }
  static __device__ float2 open(const uint32_t* w, int i) { return Num<T>::open(w[i]); }
  static __device__ void close(uint32_t* w, int i, float2 f) { w[i] = Num<T>::close(f.x, f.y); }
};
template <> struct Eight<float> {
  static constexpr int W = 8;
  static __device__ void load(const float* p, uint32_t* w) {
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
  }
  static __device__ void store(float* p, const uint32_t* w) {
    asm volatile("st.global.L1::no_allocate.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                 ::"r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]), "l"(p) : "memory");
  }
  static __device__ void load_one(const float* p, int j, uint32_t* w) { w[j] = __float_as_uint(*p); }
  static __device__ void store_one(float* p, int j, const uint32_t* w) { *p = __uint_as_float(w[j]); }
  static __device__ float2 open(const uint32_t* w, int i) { return make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1])); }
  static __device__ void close(uint32_t* w, int i, float2 f) { w[2 * i] = __float_as_uint(f.x); w[2 * i + 1] = __float_as_uint(f.y); }
};
template <> struct Eight<uint8_t> {             // codes: four to a word
  static constexpr int W = 2;
  static __device__ void load(const uint8_t* p, uint32_t* w) { asm volatile("ld.global.L1::no_allocate.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p)); }
  static __device__ void store(uint8_t* p, const uint32_t* w) { asm volatile("st.global.L1::no_allocate.v2.b32 [%2], {%0, %1};" ::"r"(w[0]), "r"(w[1]), "l"(p) : "memory"); }
  static __device__ void load_one(const uint8_t* p, int j, uint32_t* w) { w[j / 4] |= (uint32_t)*p << (8 * (j & 3)); }
  static __device__ void store_one(uint8_t* p, int j, const uint32_t* w) { *p = (uint8_t)(w[j / 4] >> (8 * (j & 3))); }
};

// Every 32nd element of a tensor: those that a lane has.
struct Lane8 {
  uint32_t at, numel;                           // the first one
  __device__ bool has(int j) const { return at + 32 * j < numel; }
};
template <typename T> __device__ void take(const Lane8& l, const void* from, uint32_t* w) {
  const T* const p = static_cast<const T*>(from) + l.at;
#pragma unroll
  for (int i = 0; i < Eight<T>::W; ++i) w[i] = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (l.has(j)) Eight<T>::load_one(p + 32 * j, j, w);
}
template <typename T> __device__ void put(const Lane8& l, void* to, const uint32_t* w) {
  T* const p = static_cast<T*>(to) + l.at;
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (l.has(j)) Eight<T>::store_one(p + 32 * j, j, w);
}

// ---- eight elements to and from shared memory ---------------------------------------------------------------

// a warp's 256 values, 16 bytes a lane at a time
__device__ void copy_1k(uint32_t to, const char* from) { copy16(to, from); copy16(to + 512, from + 512); }
template <typename T> __device__ void copy_block(uint32_t to, const char* from) { if (sizeof(T) == 4) copy_1k(to, from); else copy16(to, from); }
__device__ void shared8(uint32_t from, uint32_t* w) { asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(from) : "memory"); }
__device__ void shared16(uint32_t from, uint32_t* w) { asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(from) : "memory"); }
__device__ void shared32(uint32_t from, uint32_t* w) { shared16(from, w); shared16(from + 16, w + 4); }
template <typename T> __device__ void shared_eight(uint32_t from, uint32_t* w) { if constexpr (sizeof(T) == 4) shared32(from, w); else shared16(from, w); }

// ---- arithmetic of the step -----------------------------------------------------------------------------------

// a + b, where both may be products that have been rounded: a packed product and sum become one fused operation in the assembler, rounding
// modes or not, and a factor of one that it does not know keeps them apart
__device__ float2 sum2(float2 a, float2 b, float one) { return fma2(a, both(one), b); }
// the largest magnitude; NaN if there is one
__device__ float largest3(float a, float b, float c) { float d; asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c)); return d; }
__device__ uint32_t largest_of_warp(float x) { return __reduce_max_sync(0xffffffffu, __float_as_uint(x) & 0x7fffffffu); }
// m / (root + eps); both approximations are within 2^-22, and a root below 1e-19 may come out as zero beside eps
__device__ float approximate_root(float x) { float y; asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ float approximate_inverse(float x) { float y; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// ---- moments in 8 bits ---------------------------------------------------------------------------------------

__device__ float2 half_pair(uint32_t u) { return __half22float2(*reinterpret_cast<const __half2*>(&u)); }
// values of codes 2i, 2i + 1 before the scale; every one is a binary16 number
__device__ float2 open_e4m3(const uint32_t* c, int i) {
  const uint16_t two = (uint16_t)(c[i / 2] >> (16 * (i & 1)));
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(two));
  return half_pair(h);
}
__device__ float2 open_e5m2(const uint32_t* c, int i) { return half_pair(__byte_perm(c[i / 2], 0, i & 1 ? 0x3424 : 0x1404)); }   // the upper byte of a binary16

// The exponent of a block's scale, 127 added to it, from the bits of its largest magnitude; top: the format's largest exponent.  The formats
// end at 1.75 * 2^top, so a magnitude above 1.75 of its octave counts to the next one.  At least 1: a binary32 of full precision.
__device__ int scale_exponent(uint32_t largest, int top) { return max((int)((largest + 0x1fffffu) >> 23) - top, 1); }
__device__ float power_of_two(int e) { return __uint_as_float((uint32_t)e << 23); }

// The random bits of an element at a step: for m the lower half, for v the upper.
__device__ uint32_t step_key(uint32_t step) {
  uint32_t k = step * kGolden;
  k = (k ^ (k >> 16)) * kRoot3;
  k = (k ^ (k >> 15)) * kGolden;
  return k ^ (k >> 16);
}
__device__ uint32_t random_bits(uint32_t scrambled) {           // of (element + key) * kRoot3
  const uint32_t u = (scrambled ^ (scrambled >> 15)) * kGolden;
  return u ^ (u >> 16);
}
// Codes of m[8] and v[8].  A moment is scaled so that the format's exponents are binary32's smallest, subnormal numbers among them; the
// format's last bit is then bit 20 or 21, the random number is added below it, and the bits above are the code.
template <int STRIDE>
__device__ __forceinline__ void store_codes(const float2* m, const float2* v, int em, int ev, uint32_t place, const uint32_t* wrap, uint32_t key, uint32_t* cm, uint32_t* cv) {
  float2 ym[4], yv[4];
  const float im = power_of_two(254 - em), iv = power_of_two(254 - ev);
  if (em <= 127 + 29 && ev <= 127 + 37) {                       // times 2^-120 and 2^-112 they still are binary32 numbers
    const float2 jm = both(im * 0x1p-120f), jv = both(iv * 0x1p-112f);
#pragma unroll
    for (int i = 0; i < 4; ++i) { ym[i] = mul2(m[i], jm); yv[i] = mul2(v[i], jv); }
  } else {                                                      // moments of 1e11 and more
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      ym[i] = mul2(mul2(m[i], both(im)), both(0x1p-120f));
      yv[i] = mul2(mul2(v[i], both(iv)), both(0x1p-112f));
    }
  }
  uint32_t tm[8], tv[8], least = 0xffffffffu;
  const uint32_t scrambled = (place + key) * kRoot3;
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    constexpr uint32_t kNext = (STRIDE ? STRIDE : 1) * kRoot3;
    const uint32_t u = random_bits(scrambled + (uint32_t)j * kNext + (STRIDE ? 0 : wrap[j])), w = random_bits(scrambled + (uint32_t)(j + 1) * kNext + (STRIDE ? 0 : wrap[j + 1]));
    tm[j] = __float_as_uint(ym[j / 2].x) + (u & 0xffffu) * 16;  // the sign stays in bit 31
    tm[j + 1] = __float_as_uint(ym[j / 2].y) + (w & 0xffffu) * 16;
    tv[j] = __float_as_uint(yv[j / 2].x) + (u >> 16) * 32;
    tv[j + 1] = __float_as_uint(yv[j / 2].y) + (w >> 16) * 32;
    least = __vimin3_u32(least, tv[j], tv[j + 1]);
  }
  if (least < 1u << 21) {                                       // a v above zero does not become zero
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if ((j & 1 ? v[j / 2].y : v[j / 2].x) > 0.0f) tv[j] = max(tv[j], 1u << 21);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t* const t = tm + 4 * i;                       // upper halves of two: sign, four zeros, seven bits of the code, four below
    const uint32_t a = __byte_perm(t[0], t[1], 0x7632), b = __byte_perm(t[2], t[3], 0x7632);
    cm[i] = __byte_perm((a >> 4 & 0x7f7f7f7fu) | (a >> 8 & 0x80808080u), (b >> 4 & 0x7f7f7f7fu) | (b >> 8 & 0x80808080u), 0x6420);
    const uint32_t* const s = tv + 4 * i;                       // three zeros, eight bits, five below
    cv[i] = __byte_perm(__byte_perm(s[0], s[1], 0x7632) >> 5, __byte_perm(s[2], s[3], 0x7632) >> 5, 0x6420);
  }
}

// ---- the step ------------------------------------------------------------------------------------------------

struct Clock { float step_size, root_c2, lr; uint32_t key; };

__device__ double power(double base, uint64_t n) {
  double p = 1.0;
  for (; n; n >>= 1) {
    if (n & 1) p *= base;
    base *= base;
  }
  return p;
}

// What a lane has read of its eight elements.  MIXED: some tensor has a binary32 gradient or a master beside 16-bit parameters.
template <typename T, int BITS, bool MIXED> struct Read {
  static constexpr int W = MIXED ? 8 : Eight<T>::W, S = BITS == 32 ? 8 : 2;
  uint32_t g[W], p[W], m[S], v[S];
  float sm, sv;
};
// ... and what becomes of them
template <typename T, int BITS> struct Written {
  uint32_t master[8], p[Eight<T>::W], m[BITS == 32 ? 8 : 2], v[BITS == 32 ? 8 : 2];
  float sm, sv;
};

struct Settings { float factor, beta1, rest1, beta2, rest2, one, eps, step_size, root_c2, decay; uint32_t key; };

// Eight elements of a lane, a block's 256 of a warp; place: of the lane's first one in its tensor, the others STRIDE apart.  STRIDE 0: one apart,
// and some of them 256 further on, which `wrap` has times kRoot3.
template <typename T, int BITS, bool MIXED, int STRIDE>
__device__ __forceinline__ void update(const Settings& a, const Read<T, BITS, MIXED>& r, bool grad32, bool master, uint32_t place, const uint32_t* wrap, Written<T, BITS>& o) {
  float2 m[4], v[4];
  float largest_m = 0.0f, largest_v = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 g = mul2(MIXED && grad32 ? Eight<float>::open(r.g, i) : Eight<T>::open(r.g, i), both(a.factor));
    if (BITS == 32) {
      m[i] = Eight<float>::open(r.m, i);
      v[i] = Eight<float>::open(r.v, i);
    } else {
      m[i] = mul2(open_e4m3(r.m, i), both(r.sm));
      v[i] = mul2(open_e5m2(r.v, i), both(r.sv));
    }
    m[i] = sum2(mul2(m[i], both(a.beta1)), mul2(g, both(a.rest1)), a.one);
    v[i] = sum2(mul2(v[i], both(a.beta2)), mul2(mul2(g, g), both(a.rest2)), a.one);
    if (BITS == 8) {
      largest_m = largest3(largest_m, m[i].x, m[i].y);
      largest_v = largest3(largest_v, v[i].x, v[i].y);
    }
    float2 root = make_float2(approximate_root(v[i].x), approximate_root(v[i].y));
    root = fma2(root, both(a.root_c2), both(a.eps));
    const float2 move = mul2(m[i], make_float2(approximate_inverse(root.x), approximate_inverse(root.y)));
    float2 p = MIXED && master ? Eight<float>::open(r.p, i) : Eight<T>::open(r.p, i);
    p = fma2(both(-a.step_size), move, fma2(both(-a.decay), p, p));
    if (MIXED) Eight<float>::close(o.master, i, p);
    Eight<T>::close(o.p, i, p);
    if (BITS == 32) {
      Eight<float>::close(o.m, i, m[i]);
      Eight<float>::close(o.v, i, v[i]);
    }
  }
  if (BITS == 8) {
    const uint32_t bits_m = largest_of_warp(largest_m), bits_v = largest_of_warp(largest_v);
    const int em = scale_exponent(bits_m, 8), ev = scale_exponent(bits_v, 15);
    store_codes<STRIDE>(m, v, em, ev, place, wrap, a.key, o.m, o.v);
    const float nan = __int_as_float(0x7fc00000);               // a block with an infinity or NaN is NaN from here on
    o.sm = bits_m < 0x7f800000u ? power_of_two(em) : nan;
    o.sv = bits_v < 0x7f800000u ? power_of_two(ev) : nan;
  }
}

// The tensor that has unit c, from t on.
template <int N> __device__ int tensor_of(const Table<N>& table, int c, int t) {
  if (c < table.first[t + 1]) return t;
  for (int hi = table.n; hi - t > 1;) {
    const int mid = (t + hi) / 2;
    if (table.first[mid] <= c) t = mid; else hi = mid;
  }
  return t;
}

// A warp's walk over the blocks of its units.
template <int N> struct Walk {
  int c, t, step;
  uint32_t at, left;                          // of the block: its first element in its tensor; blocks of the unit, this one among them
  __device__ Walk(const Table<N>& table, int first, int step) : c(first), t(0), step(step), at(0), left(0) { find(table); }
  __device__ bool here(const Table<N>& table) const { return c < table.first[table.n]; }
  __device__ void find(const Table<N>& table) {
    if (!here(table)) return;
    t = tensor_of(table, c, t);
    at = (uint32_t)(c - table.first[t]) * table.unit;
    left = min(table.unit, table.part[t].numel - at + 255) / 256;
  }
  __device__ void next(const Table<N>& table, uint32_t blocks) {
    at += 256 * blocks;
    left -= blocks;
    if (left) return;
    c += step;
    find(table);
  }
};

// Blocks that begin r elements behind a multiple of eight, in all operands: lane 0 has the block's first 8 - r elements and its last r, the
// other lanes have eight on the grid, which begins r elements before the block.  Of w words with PER elements each, bits of those below r.
template <int PER> __device__ uint32_t below(uint32_t r, int w) {
  const int n = min(max((int)r - PER * w, 0), PER) * (32 / PER);
  return n < 32 ? (1u << n) - 1 : 0xffffffffu;
}
template <int W> __device__ void merge(const uint32_t* mask, uint32_t* w, const uint32_t* low) {
#pragma unroll
  for (int i = 0; i < W; ++i) w[i] = (w[i] & ~mask[i]) | (low[i] & mask[i]);
}
// A lane's eight elements of such a block; `to`: the grid's.  `last`: lane 0's words of the block before, whose last r elements lie in its first
// eight of the grid here; without them (`open`) lane 0 stores only what is this block's.  mask: of the elements below r, in lane 0.
template <typename T> __device__ void put_shifted(T* to, uint32_t r, int lane, bool open, const uint32_t* mask, const uint32_t* w, uint32_t* last) {
  constexpr int W = Eight<T>::W;
  if (!open) {
    uint32_t now[W];
#pragma unroll
    for (int i = 0; i < W; ++i) now[i] = (w[i] & ~mask[i]) | (last[i] & mask[i]);
    Eight<T>::store(to, now);
  } else if (lane) {
    Eight<T>::store(to, w);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j >= r) Eight<T>::store_one(to + j, j, w);
  }
#pragma unroll
  for (int i = 0; i < W; ++i) last[i] = w[i];
}
// lane 0's last r elements of the last block
template <typename T> __device__ void put_last(T* to, uint32_t r, const uint32_t* last) {
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < r) Eight<T>::store_one(to + j, j, last);
}

// Shared memory of the 8-bit moments: every warp has two slots for a piece of P blocks each.  A block's gradients, parameters,
// codes of m and of v, and of a shifted block the eight elements of each behind the grid's first 256; behind the blocks their scales in pairs.
template <typename T, bool MIXED> struct Ring {
  static constexpr int kValues = 256 * (MIXED ? 4 : (int)sizeof(T)), P = kValues == 512 ? 4 : 1;
  static constexpr int kParam = kValues, kM = 2 * kValues, kV = kM + 256, kMore = kV + 256, kBlock = kMore + kValues / 16 + 16, kScales = P * kBlock, kSlot = kScales + (P * 8 + 15) / 16 * 16;
  static constexpr int kBytes = kAdamWarps * 2 * kSlot;
  static_assert(kBlock % 16 == 0 && kSlot % 16 == 0, "copies start on 16-byte boundaries");
};

template <typename T, int BITS, bool MIXED, int N>
__global__ void __launch_bounds__(kAdamThreads, kAdamCtas) adamw_kernel(const __grid_constant__ Table<N> table, const __grid_constant__ AdamScalars a) {
  using State = typename std::conditional<BITS == 32, float, uint8_t>::type;
  using Rg = Ring<T, MIXED>;
  constexpr uint32_t P = Rg::P;
  extern __shared__ __align__(16) uint8_t rings[];
  __shared__ Clock shared_clock;
  const int lane = threadIdx.x & 31, warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0);   // for the compiler to see that a warp goes one way
  uint32_t here = shared_address(rings) + warp * 2 * Rg::kSlot, there = here + Rg::kSlot;
  next_may_launch();
  wait_for_previous();
  Settings set{a.factor ? *a.factor : 1.0f, a.beta1, a.rest1, a.beta2, a.rest2, a.one, a.eps, 0, 0, 0, 0};
  if (!(fabsf(set.factor) < __int_as_float(0x7f800000))) return;   // a step that is to be left out

  // of a piece's blocks those from `first` to `end` lie on the grid of eight elements, or all as far behind it, with the grid's elements around
  // them in the same tensor
  struct Wide { uint32_t first, end, shift; };
  auto wide_blocks = [&](const Walk<N>& k) {
    const AdamPart& part = table.part[k.t];
    const uint32_t shift = BITS == 8 ? part.flags >> kPartShiftBit : 0, more = shift ? 8 - shift : 0, rest = part.numel - k.at;
    Wide w{shift && k.at == 0 ? 1u : 0u, part.flags & kPartWide && rest > more ? min(min(k.left, P), (rest - more) / 256) : 0u, shift};
    if (w.end < w.first) w.end = w.first = 0;
    return w;
  };
  auto ask = [&](const Walk<N>& k, uint32_t to) {
    const AdamPart& part = table.part[k.t];
    const Wide wide = wide_blocks(k);
    const uint32_t at = k.at - wide.shift, e = at + lane * 8;   // below 0 for the first block of a shifted tensor, which is left out
    const bool grad32 = MIXED && (part.flags & kPartGradF32), master = MIXED && part.master;
    const int gs = grad32 ? 4 : (int)sizeof(T), ps = master ? 4 : (int)sizeof(T);
    const char* const g = static_cast<const char*>(part.grad) + (long long)(int)at * gs + lane * 16;
    const char* const p = (master ? reinterpret_cast<const char*>(part.master) : static_cast<const char*>(part.param)) + (long long)(int)at * ps + lane * 16;
    const uint8_t *const m = static_cast<uint8_t*>(part.m) + (int)e, *const v = static_cast<uint8_t*>(part.v) + (int)e;
#pragma unroll
    for (uint32_t i = 0; i < P; ++i) {
      if (i >= wide.end) break;
      if (i < wide.first) continue;
      const uint32_t block = to + i * Rg::kBlock;
      if (grad32) copy_1k(block + lane * 16, g + i * 1024); else copy_block<T>(block + lane * 16, g + i * 256 * sizeof(T));
      if (master) copy_1k(block + Rg::kParam + lane * 16, p + i * 1024); else copy_block<T>(block + Rg::kParam + lane * 16, p + i * 256 * sizeof(T));
      copy8(block + Rg::kM + lane * 8, m + i * 256);
      copy8(block + Rg::kV + lane * 8, v + i * 256);
      if (wide.shift) {                                         // gs + ps lanes for gradients and parameters, one each for the codes
        const char* const from = lane < gs ? g + (i + 1) * 256 * gs - lane * 8 : lane < gs + ps ? p + (i + 1) * 256 * ps - gs * 8 - lane * 8
                                 : reinterpret_cast<const char*>(lane == gs + ps ? m : v) + (i + 1) * 256 - lane * 8;
        if (lane < gs + ps + 2) copy8(block + Rg::kMore + lane * 8, from);
      }
    }
    if ((lane & 15) >= wide.first && (lane & 15) < wide.end) copy4(to + Rg::kScales + (lane & 15) * 8 + (lane >> 4) * 4, (lane & 16 ? part.v_scale : part.m_scale) + k.at / 256 + (lane & 15));
  };
  Walk<N> k(table, blockIdx.x * kAdamWarps + warp, gridDim.x * kAdamWarps), ahead = k;
  if (BITS == 8) {
    if (ahead.here(table)) {
      ask(ahead, here);
      ahead.next(table, min(ahead.left, P));
    }
    copies_end();
  }

  if (threadIdx.x == 0) {
    const float lr = a.d_lr ? *a.d_lr : a.lr;
    float c1 = a.c1, c2 = a.c2;
    uint32_t step = a.step;
    if (a.d_step) {
      const int64_t n = max((long long)*a.d_step, 1ll);
      step = (uint32_t)n;
      c1 = (float)(1.0 - power(a.beta1_exact, (uint64_t)n));
      c2 = (float)(1.0 - power(a.beta2_exact, (uint64_t)n));
    }
    shared_clock = Clock{lr / c1, sqrtf(1.0f / c2), lr, step_key(step)};
  }
  __syncthreads();
  set.step_size = shared_clock.step_size;
  set.root_c2 = shared_clock.root_c2;
  set.key = shared_clock.key;
  const float lr = shared_clock.lr;

  float unit_sm = 0.0f, unit_sv = 0.0f;                         // lane i: scales of the unit's block i
  uint32_t in_unit = 0;
#pragma unroll 1
  while (k.here(table)) {
    const AdamPart& part = table.part[k.t];
    const bool grad32 = MIXED && (part.flags & kPartGradF32), master = MIXED && part.master;
    const uint32_t blocks = min(k.left, P);
    const Wide wide = wide_blocks(k);
    set.decay = lr * part.decay;
    if (BITS == 8) {                                            // the next piece goes where the whole warp has read the last one
      copies_wait<0>();
      __syncwarp();
      if (ahead.here(table)) {
        ask(ahead, there);
        ahead.next(table, min(ahead.left, P));
      }
      copies_end();
    }
    auto from_ring = [&](uint32_t i, Read<T, BITS, MIXED>& r) {
      const uint32_t block = here + i * Rg::kBlock;
      if (grad32) shared32(block + lane * 32, r.g); else shared_eight<T>(block + lane * 8 * sizeof(T), r.g);
      if (master) shared32(block + Rg::kParam + lane * 32, r.p); else shared_eight<T>(block + Rg::kParam + lane * 8 * sizeof(T), r.p);
      shared8(block + Rg::kM + lane * 8, r.m);
      shared8(block + Rg::kV + lane * 8, r.v);
      uint32_t scales[2];
      shared8(here + Rg::kScales + i * 8, scales);
      r.sm = __uint_as_float(scales[0]);
      r.sv = __uint_as_float(scales[1]);
    };
    const uint32_t e = k.at + lane * 8;
    if (BITS == 32 || !wide.shift) {
#pragma unroll 1
      for (uint32_t i = 0; i < wide.end; ++i) {
        Read<T, BITS, MIXED> r;
        const uint32_t to = e + i * 256;
        if (BITS == 8) {
          from_ring(i, r);
        } else {
          if (grad32) Eight<float>::load(static_cast<const float*>(part.grad) + to, r.g); else Eight<T>::load(static_cast<const T*>(part.grad) + to, r.g);
          if (master) Eight<float>::load(part.master + to, r.p); else Eight<T>::load(static_cast<const T*>(part.param) + to, r.p);
          Eight<State>::load(static_cast<const State*>(part.m) + to, r.m);
          Eight<State>::load(static_cast<const State*>(part.v) + to, r.v);
        }
        Written<T, BITS> o;
        update<T, BITS, MIXED, 1>(set, r, grad32, master, part.place + to, nullptr, o);
        if (master) Eight<float>::store(part.master + to, o.master);
        Eight<T>::store(static_cast<T*>(part.param) + to, o.p);
        Eight<State>::store(static_cast<State*>(part.m) + to, o.m);
        Eight<State>::store(static_cast<State*>(part.v) + to, o.v);
        if (BITS == 8 && lane == in_unit + i) { unit_sm = o.sm; unit_sv = o.sv; }
      }
    }
    if constexpr (BITS == 8) {
      if (wide.shift) {
        const uint32_t shift = wide.shift, wrapped = lane ? 0 : shift;
        uint32_t mask32[8], mask_t[Eight<T>::W], mask8[2], wrap[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          wrap[j] = j < wrapped ? 256 * kRoot3 : 0;
          mask32[j] = below<1>(wrapped, j);
          if (j < Eight<T>::W) mask_t[j] = below<8 / Eight<T>::W>(wrapped, j);
          if (j < 2) mask8[j] = below<4>(wrapped, j);
        }
        Written<T, BITS> last;
#pragma unroll 1
        for (uint32_t i = wide.first; i < wide.end; ++i) {
          Read<T, BITS, MIXED> r;
          from_ring(i, r);
          // lane 0's elements below `shift` come from behind the grid's 256
          const uint32_t more = here + i * Rg::kBlock + Rg::kMore, gs = grad32 ? 4 : sizeof(T), ps = master ? 4 : sizeof(T);
          uint32_t low[8];
          if (grad32) { shared32(more, low); merge<8>(mask32, r.g, low); } else { shared_eight<T>(more, low); merge<Eight<T>::W>(mask_t, r.g, low); }
          if (master) { shared32(more + gs * 8, low); merge<8>(mask32, r.p, low); } else { shared_eight<T>(more + gs * 8, low); merge<Eight<T>::W>(mask_t, r.p, low); }
          shared8(more + (gs + ps) * 8, low);
          merge<2>(mask8, r.m, low);
          shared8(more + (gs + ps) * 8 + 8, low);
          merge<2>(mask8, r.v, low);
          const uint32_t to = e - shift + i * 256;
          Written<T, BITS> o;
          update<T, BITS, MIXED, 0>(set, r, grad32, master, part.place + to, wrap, o);
          const bool open = i == wide.first;
          if (master) put_shifted(part.master + (int)to, shift, lane, open, mask32, o.master, last.master);
          put_shifted(static_cast<T*>(part.param) + (int)to, shift, lane, open, mask_t, o.p, last.p);
          put_shifted(static_cast<State*>(part.m) + (int)to, shift, lane, open, mask8, o.m, last.m);
          put_shifted(static_cast<State*>(part.v) + (int)to, shift, lane, open, mask8, o.v, last.v);
          if (lane == in_unit + i) { unit_sm = o.sm; unit_sv = o.sv; }
        }
        if (lane == 0 && wide.first < wide.end) {
          const uint32_t to = k.at - shift + wide.end * 256;
          if (master) put_last(part.master + to, shift, last.master);
          put_last(static_cast<T*>(part.param) + to, shift, last.p);
          put_last(static_cast<State*>(part.m) + to, shift, last.m);
          put_last(static_cast<State*>(part.v) + to, shift, last.v);
        }
      }
    }
#pragma unroll 1
    for (uint32_t n = blocks - (wide.end - wide.first), i = wide.first ? 0 : wide.end; n; --n, i = i + 1 == wide.first ? wide.end : i + 1) {
      // elements in turn, the last block's as far as they go
      const Lane8 l{k.at + i * 256 + lane, part.numel};
      Read<T, BITS, MIXED> r;
      if (grad32) take<float>(l, part.grad, r.g); else take<T>(l, part.grad, r.g);
      if (master) take<float>(l, part.master, r.p); else take<T>(l, part.param, r.p);
      take<State>(l, part.m, r.m);
      take<State>(l, part.v, r.v);
      if (BITS == 8) { r.sm = part.m_scale[k.at / 256 + i]; r.sv = part.v_scale[k.at / 256 + i]; }
      Written<T, BITS> o;
      update<T, BITS, MIXED, 32>(set, r, grad32, master, part.place + l.at, nullptr, o);
      if (master) put<float>(l, part.master, o.master);
      put<T>(l, part.param, o.p);
      put<State>(l, part.m, o.m);
      put<State>(l, part.v, o.v);
      if (BITS == 8 && lane == in_unit + i) { unit_sm = o.sm; unit_sv = o.sv; }
    }
    in_unit += blocks;
    if (BITS == 8) {                                            // the scales of a unit leave together: pieces of a sector cost as much as whole ones
      if (k.left == blocks) {
        if (lane < in_unit) {
          const uint32_t block = k.at / 256 + blocks - in_unit + lane;
          part.m_scale[block] = unit_sm;
          part.v_scale[block] = unit_sv;
        }
        in_unit = 0;
      }
      const uint32_t other = here;
      here = there;
      there = other;
    }
    k.next(table, blocks);
  }
}

// ---- 2-norm of the gradients ------------------------------------------------------------------------------------

// Squares of eight elements are added in binary32, then everything in binary64: a stage has up to billions of them.  Where binary32 cannot hold the
// sum of eight, they are rounded to it one by one, and the norm is infinite for an element whose own square is too large alone (no binary16 one's is).
template <typename G> __device__ double eight_squares(const uint32_t* w) {
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 g = Eight<G>::open(w, i);
    s = fmaf(g.x, g.x, fmaf(g.y, g.y, s));
  }
  if (!std::is_same<G, __half>::value && !(s < __int_as_float(0x7f800000))) {
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 g = Eight<G>::open(w, i);
      sum += (double)(g.x * g.x) + (double)(g.y * g.y);
    }
    return sum;
  }
  return (double)s;
}
// A warp's blocks of one tensor, from element `at` on.  Four blocks are on their way at a time: 492M fp16 gradients take 140 to 145 us, with one 206 us.
template <typename G> __device__ double squares(const AdamPart& part, uint32_t at, uint32_t blocks, int lane) {
  const G* const g = static_cast<const G*>(part.grad);
  double sum = 0.0;
  uint32_t i = 0;
  if (part.flags & kPartWide) {
    const uint32_t wide = min(blocks, (part.numel - at) / 256);
    const G* const from = g + at + lane * 8;
    for (; i + 4 <= wide; i += 4) {
      uint32_t w[4][Eight<G>::W];
#pragma unroll
      for (int j = 0; j < 4; ++j) Eight<G>::load(from + (i + j) * 256, w[j]);
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += eight_squares<G>(w[j]);
    }
    for (; i < wide; ++i) {
      uint32_t w[Eight<G>::W];
      Eight<G>::load(from + i * 256, w);
      sum += eight_squares<G>(w);
    }
  }
#pragma unroll 1
  for (; i < blocks; ++i) {
    uint32_t w[Eight<G>::W];
    take<G>(Lane8{at + i * 256 + lane, part.numel}, g, w);
    sum += eight_squares<G>(w);
  }
  return sum;
}

template <typename T, int N>
__global__ void __launch_bounds__(kAdamThreads, kNormCtasPerSm) grad_norm_kernel(const __grid_constant__ Table<N> table, const __grid_constant__ NormScalars a) {
  __shared__ double sums[kAdamWarps];
  __shared__ bool last_cta;
  const int lane = threadIdx.x & 31, warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0);
  next_may_launch();
  wait_for_previous();
  double sum = 0.0;
#pragma unroll 1
  for (Walk<N> k(table, blockIdx.x * kAdamWarps + warp, gridDim.x * kAdamWarps); k.here(table); k.next(table, k.left)) {
    const AdamPart& part = table.part[k.t];
    sum += part.flags & kPartGradF32 ? squares<float>(part, k.at, k.left, lane) : squares<T>(part, k.at, k.left, lane);
  }
  auto join = [&](double x) {                 // the CTA's sum, for thread 0
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if (lane == 0) sums[warp] = x;
    __syncthreads();
    x = 0.0;
    if (threadIdx.x == 0) {
#pragma unroll
      for (int i = 0; i < kAdamWarps; ++i) x += sums[i];
    }
    return x;
  };
  sum = join(sum);
  if (threadIdx.x == 0) {
    __stcg(a.partials + blockIdx.x, sum);
    __threadfence();
    last_cta = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last_cta) return;
  __threadfence();
  sum = 0.0;
  for (int i = threadIdx.x; i < (int)gridDim.x; i += kAdamThreads) sum += __ldcg(a.partials + i);
  sum = join(sum);
  if (threadIdx.x) return;
  *a.ticket = 0;
  double* const before = a.partials + kNormCtas;
  if (!a.first) sum += *before;
  if (!a.last) { *before = sum; return; }
  const double norm = sqrt(sum) * a.inv_scale;
  const bool fine = (float)norm < __int_as_float(0x7f800000);   // as it is returned; the factor is at most inv_scale then, a binary32 number
  if (a.norm) *a.norm = (float)norm;
  if (a.factor) *a.factor = fine ? (float)(a.inv_scale * fmin(1.0, a.max_norm / (norm + 1e-6))) : __int_as_float(0x7fc00000);
  if (a.step && fine) ++*a.step;
}

// Units of `unit` elements; how many there are.
template <int N> int fill(Table<N>& table, const AdamPart* parts, int n, uint32_t unit) {
  int units = 0;
  for (int i = 0; i < n; ++i) {
    table.part[i] = parts[i];
    table.first[i] = units;
    units += (int)((parts[i].numel + unit - 1) / unit);
  }
  for (int i = n; i <= N; ++i) table.first[i] = units;
  table.n = n;
  table.unit = unit;
  return units;
}

template <int N, typename Kernel, typename Scalars>
cudaError_t start(Kernel kernel, const AdamPart* parts, int n, const Scalars& a, int ctas, size_t shared, cudaStream_t s) {
  Table<N> table;
  // the longest units, up to eight blocks (whose scales fill a sector), with which every warp has four
  long long blocks = 0;
  for (int i = 0; i < n; ++i) blocks += (parts[i].numel + 255) / 256;
  uint32_t unit = 2048;
  while (unit > 256 && blocks * 256 < 4ll * unit * ctas * kAdamWarps) unit /= 2;
  const int units = fill(table, parts, n, unit), want = (units + kAdamWarps - 1) / kAdamWarps;
  return launch(kernel, dim3((unsigned)(want < 1 ? 1 : want < ctas ? want : ctas)), kAdamThreads, shared, s, table, a);
}

// Most calls of few tensors are short: a small table spares them 30 KB of arguments.
constexpr int kSmallTable = 24;

template <typename T, int BITS, bool MIXED, int N> cudaError_t run_table(const AdamPart* parts, int n, const AdamScalars& a, int sms, cudaStream_t s) {
  constexpr int kBytes = BITS == 8 ? Ring<T, MIXED>::kBytes : 0;
  const auto kernel = adamw_kernel<T, BITS, MIXED, N>;
  if (kBytes) {
    static std::atomic<uint64_t> allowed{0};
    const cudaError_t e = allow_shared(reinterpret_cast<const void*>(kernel), kBytes, allowed);
    if (e != cudaSuccess) return e;
  }
  return start<N>(kernel, parts, n, a, kAdamCtas * sms, kBytes, s);
}
template <typename T, int BITS, bool MIXED> cudaError_t run_mixed(const AdamPart* parts, int n, const AdamScalars& a, int sms, cudaStream_t s) {
  if (n <= kSmallTable) return run_table<T, BITS, MIXED, kSmallTable>(parts, n, a, sms, s);
  return run_table<T, BITS, MIXED, kAdamTable>(parts, n, a, sms, s);
}
template <typename T, int BITS> cudaError_t run_adamw(const AdamPart* parts, int n, const AdamScalars& a, int sms, cudaStream_t s) {
  bool mixed = false;
  for (int i = 0; i < n; ++i) mixed = mixed || parts[i].master || (parts[i].flags & kPartGradF32);
  if constexpr (!std::is_same<T, float>::value)
    if (mixed) return run_mixed<T, BITS, true>(parts, n, a, sms, s);
  return run_mixed<T, BITS, false>(parts, n, a, sms, s);
}

template <typename T> cudaError_t run_norm(const AdamPart* parts, int n, const NormScalars& a, int sms, cudaStream_t s) {
  const int most = kNormCtasPerSm * sms < kNormCtas ? kNormCtasPerSm * sms : kNormCtas;
  if (n <= kSmallTable) return start<kSmallTable>(grad_norm_kernel<T, kSmallTable>, parts, n, a, most, 0, s);
  return start<kAdamTable>(grad_norm_kernel<T, kAdamTable>, parts, n, a, most, 0, s);
}

}  // namespace

cudaError_t launch_adamw(int dtype, int state_bits, const AdamPart* parts, int n, const AdamScalars& a, int sms, cudaStream_t s) {
  if (n == 0) return cudaSuccess;
  if (state_bits == 8) {
    if (dtype == AQ_FP16) return run_adamw<__half, 8>(parts, n, a, sms, s);
    if (dtype == AQ_BF16) return run_adamw<__nv_bfloat16, 8>(parts, n, a, sms, s);
    return run_adamw<float, 8>(parts, n, a, sms, s);
  }
  if (dtype == AQ_FP16) return run_adamw<__half, 32>(parts, n, a, sms, s);
  if (dtype == AQ_BF16) return run_adamw<__nv_bfloat16, 32>(parts, n, a, sms, s);
  return run_adamw<float, 32>(parts, n, a, sms, s);
}

cudaError_t launch_grad_norm(int dtype, const AdamPart* parts, int n, const NormScalars& a, int sms, cudaStream_t s) {
  if (dtype == AQ_FP16) return run_norm<__half>(parts, n, a, sms, s);
  if (dtype == AQ_BF16) return run_norm<__nv_bfloat16>(parts, n, a, sms, s);
  return run_norm<float>(parts, n, a, sms, s);
}

}  // namespace aq
