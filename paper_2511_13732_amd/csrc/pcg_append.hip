// New tokens' keys and values into a paged cache, with the rotation of keys and queries on the way, and into and out of a cache of 4-bit
// codes (gfx950, wave64).
//
// A pair (x, y) of a head turned by an angle is (x cos - y sin, y cos + x sin).  It is formed in double, where products of two numbers of 24
// bits are exact, and so rounded once to float32, and from there to the type that it is stored in.  What 4 bits hold of a key is thereby the same
// whatever forms it: codes and scales are decided by float32 numbers that are fully rounded.
#include <math.h>

#include "pcg_cache.h"
#include "pcg_device.h"

namespace pcg {

namespace {

constexpr int kThreads = 256;

typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <typename T>
__device__ __forceinline__ float as_float(T x) {
  if constexpr (sizeof(T) == 2) return __uint_as_float((uint32_t) x << 16);
  else return x;
}
template <typename T>
__device__ __forceinline__ T as_type(float x) {
  if constexpr (sizeof(T) == 2) return __builtin_bit_cast(uint16_t, (__bf16) x);
  else return x;
}

// N elements, as float32; a multiple of 16 bytes in a row, aligned.
template <typename T, int N>
__device__ __forceinline__ void load(const T *p, float (&x)[N]) {
  constexpr int E = 16 / (int) sizeof(T);
#pragma unroll
  for (int i = 0; i < N; i += E) {
    const uint4 v = *reinterpret_cast<const uint4 *>(p + i);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if constexpr (sizeof(T) == 2) x[i + e] = __uint_as_float(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
      else x[i + e] = __uint_as_float(w[e]);
    }
  }
}
template <typename T, int N>
__device__ __forceinline__ void store(T *p, const float (&x)[N]) {
  constexpr int E = 16 / (int) sizeof(T);
#pragma unroll
  for (int i = 0; i < N; i += E) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(T) == 2)
        w[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2{x[i + 2 * e], x[i + 2 * e + 1]}), bf16x2));
      else
        w[e] = __float_as_uint(x[i + e]);
    }
    *reinterpret_cast<uint4 *>(p + i) = uint4{w[0], w[1], w[2], w[3]};
  }
}

// N / 2 numbers of a table's row.
template <int N>
__device__ __forceinline__ void load_half(const float *p, float (&x)[N]) {
  if constexpr (N == 8) {
    const float4 v = *reinterpret_cast<const float4 *>(p);
    x[0] = v.x;
    x[1] = v.y;
    x[2] = v.z;
    x[3] = v.w;
  } else {
    const float2 v = *reinterpret_cast<const float2 *>(p);
    x[0] = v.x;
    x[1] = v.y;
  }
}

__device__ __forceinline__ void turn(float &x, float &y, float cs, float sn) {
  const double a = x, b = y, c = cs, s = sn;
  x = (float) fma(-b, s, a * c);
  y = (float) fma(a, s, b * c);
}

// Where token t goes.  What it is made of is asked for ahead of anything that depends on it; a row of the rotation's table follows.
struct Place {
  int32_t number, position;
  __device__ __forceinline__ Place(const AppendArgs &a, int64_t t) : number(a.slots[t]), position(a.table ? a.positions[t] : 0) {}
  int64_t page, slot;
  const float *row;
  // false: nowhere
  __device__ __forceinline__ bool find(const AppendArgs &a) {
    if (number < 0) return false;
    page = number / a.page_size;
    slot = number - page * a.page_size;
    row = a.table ? a.table + (int64_t) position * a.table_stride : nullptr;
    return page < a.num_pages && (!a.table || (uint32_t) position < (uint32_t) a.places);
  }
};

// How a head is dealt to threads: `pairs` threads take E pairs each, or E elements with neighbours for pairs, then each takes E of
// the elements behind `rot`.  A thread owns what it reads, so that rows may be rotated in place.
template <typename T>
struct Deal {
  static constexpr int E = 16 / (int) sizeof(T);
  int32_t pairs, all;
  __host__ __device__ Deal(int32_t D, int32_t rot, bool interleaved) {
    pairs = interleaved ? 0 : (rot / 2 + E - 1) / E;
    all = interleaved ? D / E : pairs + (D - rot + E - 1) / E;
  }
};

// Part `i` of a head at x.  VEC: parts are whole and aligned, and so are those of the table.
template <typename T, bool VEC>
struct HeadPart {
  static constexpr int E = Deal<T>::E;
  const T *x;
  int32_t at, other;          // first elements, other < 0: of pairs that are neighbours or of none
  float u[E], v[E];
  __device__ __forceinline__ HeadPart(const AppendArgs &a, const Deal<T> &deal, int32_t i, const T *x_) : x(x_) {
    at = a.interleaved || i < deal.pairs ? i * E : a.rot + (i - deal.pairs) * E;
    other = !a.interleaved && i < deal.pairs ? a.rot / 2 + at : -1;
    if constexpr (VEC) {
      load<T, E>(x + at, u);
      if (other >= 0) load<T, E>(x + other, v);
    }
  }
  __device__ __forceinline__ void turn_to(const AppendArgs &a, const float *row, T *to) {
    const int32_t half = a.rot / 2;
    if constexpr (VEC) {
      float c[E], s[E];
      if (other >= 0) {
        load<float, E>(row + at, c);
        load<float, E>(row + half + at, s);
#pragma unroll
        for (int e = 0; e < E; ++e) turn(u[e], v[e], c[e], s[e]);
        store<T, E>(to + other, v);
      } else if (at < a.rot) {
        load_half<E>(row + at / 2, c);
        load_half<E>(row + half + at / 2, s);
#pragma unroll
        for (int e = 0; e < E; e += 2) turn(u[e], u[e + 1], c[e / 2], s[e / 2]);
      }
      store<T, E>(to + at, u);
    } else if (other >= 0) {
      for (int32_t e = at; e < min(at + E, half); ++e) {
        float y = as_float<T>(x[e]), z = as_float<T>(x[half + e]);
        turn(y, z, row[e], row[half + e]);
        to[e] = as_type<T>(y);
        to[half + e] = as_type<T>(z);
      }
    } else {
      for (int32_t e = at; e < min(at + E, a.D); ++e) {
        if (e >= a.rot) {
          to[e] = x[e];
          continue;
        }
        float y = as_float<T>(x[e]), z = as_float<T>(x[e + 1]);
        turn(y, z, row[e / 2], row[half + e / 2]);
        to[e++] = as_type<T>(y);
        to[e] = as_type<T>(z);
      }
    }
  }
};

struct Counts {
  int32_t token, part;                 // threads of a token, of a head
  uint32_t magic_token, magic_part;
};

// A part of a head a thread: queries (if any), keys, values.  Bound by memory: everything is read and written once, 16 bytes at a time, with
// nothing between but four products in double a pair.  16 prompts of up to 2048 tokens, 16 / 8 heads of 64, float32, take 34.9 us for 182 MB, 5.2
// TB/s; 24 of up to 3000, 32 / 8 heads of 128, bf16, 109 to 117 us for 605 MB, halves and neighbours alike; 576 rows of a step 5.3 us, the waits for a slot, the row and the table's row.
template <typename T, bool VEC>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a, Counts n, Deal<T> deal) {
  constexpr int E = Deal<T>::E;
  uint32_t t, i, head, part;
  split_by(blockIdx.x * kThreads + threadIdx.x, (uint32_t) n.token, n.magic_token, t, i);
  if (t >= a.T) return;
  Place p(a, t);
  const int64_t row = t;
  const int32_t with_q = a.q ? a.heads : 0;
  if ((int32_t) i < (with_q + a.kv_heads) * n.part) {
    split_by(i, (uint32_t) n.part, n.magic_part, head, part);
    const bool query = (int32_t) head < with_q;
    const int64_t h = query ? head : head - with_q;
    HeadPart<T, VEC> x(a, deal, (int32_t) part, query ? reinterpret_cast<const T *>(a.q) + row * a.q_tok + h * a.q_head
                                                      : reinterpret_cast<const T *>(a.k_new) + row * a.k_tok + h * a.k_head);
    if (!p.find(a)) return;
    x.turn_to(a, p.row, query ? reinterpret_cast<T *>(a.q_out) + row * a.o_tok + h * a.o_head
                              : reinterpret_cast<T *>(a.k) + p.page * a.page_stride + p.slot * a.slot_stride + h * a.head_stride);
    return;
  }
  i -= (with_q + a.kv_heads) * n.part;
  const int32_t parts = a.D / E;
  head = i / parts;
  const int64_t d = (int64_t) (i - head * parts) * E;
  const uint4 x = *reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(a.v_new) + row * a.v_tok + head * a.v_head + d);
  if (!p.find(a)) return;
  *reinterpret_cast<uint4 *>(reinterpret_cast<T *>(a.v) + p.page * a.page_stride + p.slot * a.slot_stride + head * a.head_stride + d) = x;
}

// The largest of N lanes, 8 or 16.
template <int N>
__device__ __forceinline__ uint32_t max_of(uint32_t x) {
  x = max(x, (uint32_t) __builtin_amdgcn_update_dpp(0, (int) x, 0xb1, 0xf, 0xf, false));        // neighbours
  x = max(x, (uint32_t) __builtin_amdgcn_update_dpp(0, (int) x, 0x4e, 0xf, 0xf, false));        // pairs of four
  x = max(x, (uint32_t) __builtin_amdgcn_update_dpp(0, (int) x, 0x141, 0xf, 0xf, false));       // eight the other way round
  if constexpr (N == 16) x = max(x, (uint32_t) __builtin_amdgcn_update_dpp(0, (int) x, 0x140, 0xf, 0xf, false));
  return x;
}

// The scale of numbers whose largest absolute value has these bits: a sixth of it in bfloat16, at most what 6 times is finite of.  Rounded to
// float32 and then to bfloat16 it would be rounded twice where it is subnormal: the quotient there may come to lie in the middle of two
// bfloat16 numbers.  A quotient that is not exact is therefore made the odd one of the two float32 numbers that it lies between (the rest of the
// division, which is exact, says on which side of the rounded one it lies), and an odd one is never such a middle.  NaN where a number is not
// finite: its bits are then at least those of infinity.
constexpr float kMostScale = 0x1.54p125f;
__device__ __forceinline__ uint16_t scale_of(uint32_t largest) {
  if (largest >= 0x7f800000u) return 0x7fc0;
  const float x = __uint_as_float(largest), nearest = x / 6.f, rest = fmaf(-6.f, nearest, x);
  const uint32_t below = __float_as_uint(nearest) - (rest < 0.f);
  return as_type<uint16_t>(fminf(__uint_as_float(below | (rest != 0.f)), kMostScale));
}

// Codes of eight numbers, the nearest to each quotient by the scale, ties to the even code: v_cvt_scalef32_pk_fp4_f32 of the float32
// quotient.  That is exact: a number of 24 bits and a border of two codes times a scale of 8 bits, if they differ, differ by more than half a
// float32 step of the quotient, and the product with a reciprocal in double, rounded to float32, is the rounded quotient there.
__device__ __forceinline__ uint32_t codes_of(const float (&x)[8], double inverse) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = (float) ((double) x[e] * inverse);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, r[0], r[1], 1.f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, r[2], r[3], 1.f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, r[4], r[5], 1.f, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, r[6], r[7], 1.f, 3);
}

// Eight elements of a key from element d on, and their partners.
template <typename T, bool VEC>
struct KeyEight {
  const T *x;
  int32_t d;
  bool upper;                 // the second ones of their pairs
  float v[8], u[8];
  __device__ __forceinline__ KeyEight(const AppendArgs &a, const T *x_, int32_t d_) : x(x_), d(d_) {
    load<T, 8>(x + d, v);
    upper = d >= a.rot / 2;
    if (VEC && !a.interleaved && d < a.rot) load<T, 8>(x + (upper ? d - a.rot / 2 : d + a.rot / 2), u);
  }
  __device__ __forceinline__ void turn_by(const AppendArgs &a, const float *row) {
    const int32_t half = a.rot / 2;
    if (a.interleaved) {
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const int32_t j = (d + e) / 2;
        if (j < half) turn(v[e], v[e + 1], row[j], row[half + j]);
      }
    } else if constexpr (VEC) {
      if (d >= a.rot) return;
      const int32_t j = upper ? d - half : d;
      float c[8], s[8];
      load<float, 8>(row + j, c);
      load<float, 8>(row + half + j, s);
      // the upper one of a pair is turned by the other sign
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (float) fma((double) u[e], (double) (upper ? s[e] : -s[e]), (double) v[e] * (double) c[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (d + e >= a.rot) continue;
        const bool second = d + e >= half;
        const int32_t j = second ? d + e - half : d + e;
        const float w = as_float<T>(x[second ? j : half + j]), s = row[half + j];
        v[e] = (float) fma((double) w, (double) (second ? s : -s), (double) v[e] * (double) row[j]);
      }
    }
  }
};

// Scale and codes of a head's elements, eight a lane (v of lanes behind the last: zeros).
template <int N>
__device__ __forceinline__ uint16_t quantise(const float (&v)[8], uint32_t &codes) {
  uint32_t largest = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) largest = max(largest, __float_as_uint(v[e]) & 0x7fffffffu);
  const uint16_t scale = scale_of(max_of<N>(largest));
  const float s = as_float<uint16_t>(scale);
  codes = s > 0.f ? codes_of(v, 1.0 / (double) s) : 0;          // all zero, or NaN
  return scale;
}

// Queries a part a thread in the first blocks; in the others N lanes a head of keys and values, eight elements of each a lane: a scale is the
// maximum of a head, which the lanes form among themselves, and a lane's eight codes are a word.  Bound by memory: 24 prompts, 24000
// tokens, 32 / 8 heads of 128, bf16 with queries, take 108 to 124 us for 531 MB, 4.3 to 4.9 TB/s, 12200 of float32 94 us for 519 MB; pairs that are
// neighbours, whose table is read number by number, 138 and 117; heads of 72, whose halves are no whole pieces, 245 us for 299 MB; a step's 576 rows
// 5.7 us, which are the waits for a slot, a row and a table's row one after the other.  Neighbours are the heads of a token, whose rows are read in a row; tokens of a head, which
// would be written in a row where the cache has a head's slots together, measure the same (138.4 us for 136.3, with the way back).
template <typename T, bool VEC, int N>
__global__ __launch_bounds__(kThreads) void append4_kernel(AppendArgs a, Counts n, Deal<T> deal, uint32_t q_blocks) {
  uint32_t t, i;
  if (blockIdx.x < q_blocks) {
    uint32_t head, part;
    split_by(blockIdx.x * kThreads + threadIdx.x, (uint32_t) n.token, n.magic_token, t, i);
    if (t >= a.T) return;
    Place p(a, t);
    split_by(i, (uint32_t) n.part, n.magic_part, head, part);
    HeadPart<T, VEC> x(a, deal, (int32_t) part, reinterpret_cast<const T *>(a.q) + (int64_t) t * a.q_tok + head * a.q_head);
    if (p.find(a)) x.turn_to(a, p.row, reinterpret_cast<T *>(a.q_out) + (int64_t) t * a.o_tok + head * a.o_head);
    return;
  }
  const uint32_t group = ((blockIdx.x - q_blocks) * kThreads + threadIdx.x) / N;
  const int32_t lane = threadIdx.x % N, d = 8 * lane;
  t = group / (uint32_t) a.kv_heads;
  i = group - t * (uint32_t) a.kv_heads;
  if (t >= a.T) return;                                 // all N lanes
  Place p(a, t);
  const int64_t head = i, in = d < a.D ? d : 0;
  KeyEight<T, VEC> key(a, reinterpret_cast<const T *>(a.k_new) + (int64_t) t * a.k_tok + head * a.k_head, in);
  float value[8];
  load<T, 8>(reinterpret_cast<const T *>(a.v_new) + (int64_t) t * a.v_tok + head * a.v_head + in, value);
  if (!p.find(a)) return;                               // all N lanes
  if (p.row) key.turn_by(a, p.row);
  if (d >= a.D) {
#pragma unroll
    for (int e = 0; e < 8; ++e) key.v[e] = value[e] = 0.f;
  }
  uint32_t codes[2];
  const uint32_t scales = (uint32_t) quantise<N>(key.v, codes[0]) | (uint32_t) quantise<N>(value, codes[1]) << 16;
  const int64_t at = p.page * a.page_stride + p.slot * a.slot_stride + head * a.head_stride + 4 * lane;
  if (d < (a.D + 31) / 32 * 32) {
    *reinterpret_cast<uint32_t *>(reinterpret_cast<uint8_t *>(a.k) + at) = codes[0];
    *reinterpret_cast<uint32_t *>(reinterpret_cast<uint8_t *>(a.v) + at) = codes[1];
  }
  if (lane == 0) reinterpret_cast<uint32_t *>(a.scales)[p.page * a.s_page + p.slot * a.s_slot + head * a.s_head] = scales;
}

// Eight elements of a key and of its value a thread.  Bound by memory: 24000 tokens of 8 heads of 128 into bf16, 124 MB, take 22.6 us, 5.5 TB/s.
template <typename T>
__global__ __launch_bounds__(kThreads) void cache4_read_kernel(ReadArgs r, Counts n) {
  uint32_t t, i, head, part;
  split_by(blockIdx.x * kThreads + threadIdx.x, (uint32_t) n.token, n.magic_token, t, i);
  if (t >= r.T) return;
  split_by(i, (uint32_t) n.part, n.magic_part, head, part);
  const int32_t slot = r.slots[t];
  if (slot < 0) return;
  const int64_t page = slot / r.page_size, at = slot - page * r.page_size;
  if (page >= r.num_pages) return;
  const int64_t from = page * r.page_stride + at * r.slot_stride + head * r.head_stride + 4 * part;
  const uint32_t codes[2] = {*reinterpret_cast<const uint32_t *>(r.k + from), *reinterpret_cast<const uint32_t *>(r.v + from)};
  const uint32_t scales = reinterpret_cast<const uint32_t *>(r.scales)[page * r.s_page + at * r.s_slot + head * r.s_head];
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float s = __uint_as_float(which ? scales & 0xffff0000u : scales << 16);
    s = fmaf(s, 0.f, s);               // what is not finite is NaN
    const floatx2 y[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[which], 1.f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[which], 1.f, 1),
                          __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[which], 1.f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[which], 1.f, 3)};
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = y[e / 2][e % 2] * s;
    T *to = which ? reinterpret_cast<T *>(r.v_out) + (int64_t) t * r.v_tok + head * r.v_head : reinterpret_cast<T *>(r.k_out) + (int64_t) t * r.k_tok + head * r.k_head;
    store<T, 8>(to + 8 * part, x);
  }
}

uint32_t magic(int32_t d) { return d > 1 ? (uint32_t) (((uint64_t) 1 << 32) / (uint32_t) d) : UINT32_MAX; }
uint32_t blocks(int64_t threads) { return (uint32_t) ((threads + kThreads - 1) / kThreads); }

template <typename T>
hipError_t go(const AppendArgs &a, hipStream_t stream) {
  constexpr int E = Deal<T>::E;
  const Deal<T> deal(a.D, a.rot, a.interleaved);
  // Parts of pairs and of the table in whole, aligned pieces of 16 bytes (eight elements where codes are formed); otherwise element by element,
  // at twice the time: prompts of float32 35 us in pieces and 67 by elements, into codes 138 and 365.
  const int32_t whole = a.scales ? 8 : E;
  const bool vec = a.rot / 2 % whole == 0 && a.table_stride % 4 == 0 && (uintptr_t) a.table % 16 == 0;
  Counts n;
  n.part = deal.all;
  n.magic_part = magic(n.part);
  if (a.scales) {
    n.token = a.q ? a.heads * deal.all : 1;
    n.magic_token = magic(n.token);
    // eight elements a lane: with 16 lanes for a head of 64 half of them would idle (prompts of 24 requests 74 us, 91 with 16)
    const int lanes = a.D <= 64 ? 8 : 16;
    const uint32_t q_blocks = a.q ? blocks(a.T * n.token) : 0, all = q_blocks + blocks(a.T * a.kv_heads * lanes);
    if (lanes == 8) {
      if (vec) append4_kernel<T, true, 8><<<all, kThreads, 0, stream>>>(a, n, deal, q_blocks);
      else append4_kernel<T, false, 8><<<all, kThreads, 0, stream>>>(a, n, deal, q_blocks);
    } else {
      if (vec) append4_kernel<T, true, 16><<<all, kThreads, 0, stream>>>(a, n, deal, q_blocks);
      else append4_kernel<T, false, 16><<<all, kThreads, 0, stream>>>(a, n, deal, q_blocks);
    }
  } else {
    n.token = ((a.q ? a.heads : 0) + a.kv_heads) * deal.all + a.kv_heads * (a.D / E);
    n.magic_token = magic(n.token);
    if (vec) append_kernel<T, true><<<blocks(a.T * n.token), kThreads, 0, stream>>>(a, n, deal);
    else append_kernel<T, false><<<blocks(a.T * n.token), kThreads, 0, stream>>>(a, n, deal);
  }
  return hipGetLastError();
}

}  // namespace

// A head takes at most a part more than it has pieces of 16 bytes, of float32, or 32 lanes of codes.
int64_t append_threads(int32_t heads, int32_t kv_heads, int32_t head_dim) {
  return (int64_t) (heads + 2 * kv_heads) * (head_dim / 4 + 2) + 32 * (int64_t) kv_heads + 2 * kThreads;
}

hipError_t launch_append(const AppendArgs &a, bool bf16, hipStream_t stream) { return bf16 ? go<uint16_t>(a, stream) : go<float>(a, stream); }

hipError_t launch_cache4_read(const ReadArgs &r, bool bf16, hipStream_t stream) {
  Counts n;
  n.part = r.D / 8;
  n.token = r.kv_heads * n.part;
  n.magic_part = magic(n.part);
  n.magic_token = magic(n.token);
  if (bf16) cache4_read_kernel<uint16_t><<<blocks(r.T * n.token), kThreads, 0, stream>>>(r, n);
  else cache4_read_kernel<float><<<blocks(r.T * n.token), kThreads, 0, stream>>>(r, n);
  return hipGetLastError();
}

}  // namespace pcg
