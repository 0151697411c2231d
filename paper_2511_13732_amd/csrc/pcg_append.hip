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

__device__ __forceinline__ void turn(float &x, float &y, float cs, float sn) {
  const double a = x, b = y, c = cs, s = sn;
  x = (float) fma(-b, s, a * c);
  y = (float) fma(a, s, b * c);
}

// Where token t goes; false: nowhere.
struct Place {
  int64_t page, slot;
  const float *row;           // of the rotation's table
};
__device__ __forceinline__ bool place_of(const AppendArgs &a, int64_t t, Place &p) {
  const int32_t slot = a.slots[t];
  if (slot < 0) return false;
  p.page = slot / a.page_size;
  p.slot = slot - p.page * a.page_size;
  p.row = nullptr;
  if (p.page >= a.num_pages) return false;
  if (a.table) {
    const int32_t at = a.positions[t];
    if (at < 0 || at >= a.places) return false;
    p.row = a.table + (int64_t) at * a.table_stride;
  }
  return true;
}

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

// Part `i` of a head, from `x` to `to`.  VEC: parts are whole and aligned, and so are those of the table.
template <typename T, bool VEC>
__device__ __forceinline__ void rotate_part(const AppendArgs &a, const Deal<T> &deal, int32_t i, const float *row, const T *x, T *to) {
  constexpr int E = Deal<T>::E;
  const int32_t half = a.rot / 2;
  if (a.interleaved) {
    const int32_t d = i * E;
    float v[E];
    load<T, E>(x + d, v);
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      const int32_t j = (d + e) / 2;
      if (j < half) turn(v[e], v[e + 1], row[j], row[half + j]);
    }
    store<T, E>(to + d, v);
    return;
  }
  if (i < deal.pairs) {
    const int32_t j = i * E;
    if constexpr (VEC) {
      float u[E], v[E], c[E], s[E];
      load<T, E>(x + j, u);
      load<T, E>(x + half + j, v);
      load<float, E>(row + j, c);
      load<float, E>(row + half + j, s);
#pragma unroll
      for (int e = 0; e < E; ++e) turn(u[e], v[e], c[e], s[e]);
      store<T, E>(to + j, u);
      store<T, E>(to + half + j, v);
    } else {
      for (int32_t e = j; e < min(j + E, half); ++e) {
        float u = as_float<T>(x[e]), v = as_float<T>(x[half + e]);
        turn(u, v, row[e], row[half + e]);
        to[e] = as_type<T>(u);
        to[half + e] = as_type<T>(v);
      }
    }
    return;
  }
  const int32_t j = a.rot + (i - deal.pairs) * E;
  if constexpr (VEC) {
    *reinterpret_cast<uint4 *>(to + j) = *reinterpret_cast<const uint4 *>(x + j);
  } else {
    for (int32_t e = j; e < min(j + E, a.D); ++e) to[e] = x[e];
  }
}

struct Counts {
  int32_t token, part;                 // threads of a token, of a head
  uint32_t magic_token, magic_part;
};

// A part of a head a thread: queries (if any), keys, values.
template <typename T, bool VEC>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a, Counts n, Deal<T> deal) {
  constexpr int E = Deal<T>::E;
  const uint32_t at = blockIdx.x * kThreads + threadIdx.x;
  uint32_t t, i, head, part;
  split_by(at, (uint32_t) n.token, n.magic_token, t, i);
  if (t >= a.T) return;
  Place p;
  if (!place_of(a, t, p)) return;
  const int64_t row = t;
  const int32_t with_q = a.q ? a.heads : 0;
  if ((int32_t) i < (with_q + a.kv_heads) * n.part) {
    split_by(i, (uint32_t) n.part, n.magic_part, head, part);
    if ((int32_t) head < with_q) {
      rotate_part<T, VEC>(a, deal, (int32_t) part, p.row, reinterpret_cast<const T *>(a.q) + row * a.q_tok + head * a.q_head,
                          reinterpret_cast<T *>(a.q_out) + row * a.o_tok + head * a.o_head);
    } else {
      head -= with_q;
      rotate_part<T, VEC>(a, deal, (int32_t) part, p.row, reinterpret_cast<const T *>(a.k_new) + row * a.k_tok + head * a.k_head,
                          reinterpret_cast<T *>(a.k) + p.page * a.page_stride + p.slot * a.slot_stride + head * a.head_stride);
    }
    return;
  }
  i -= (with_q + a.kv_heads) * n.part;
  const int32_t parts = a.D / E;
  head = i / parts;
  const int64_t d = (int64_t) (i - head * parts) * E;
  const T *from = reinterpret_cast<const T *>(a.v_new) + row * a.v_tok + head * a.v_head + d;
  T *to = reinterpret_cast<T *>(a.v) + p.page * a.page_stride + p.slot * a.slot_stride + head * a.head_stride + d;
  *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(from);
}

// The largest of 16 lanes.
__device__ __forceinline__ uint32_t max16(uint32_t x) {
  x = max(x, (uint32_t) __builtin_amdgcn_update_dpp(0, (int) x, 0x128, 0xf, 0xf, false));
  x = max(x, (uint32_t) __builtin_amdgcn_update_dpp(0, (int) x, 0x124, 0xf, 0xf, false));
  x = max(x, (uint32_t) __builtin_amdgcn_update_dpp(0, (int) x, 0x122, 0xf, 0xf, false));
  return max(x, (uint32_t) __builtin_amdgcn_update_dpp(0, (int) x, 0x121, 0xf, 0xf, false));
}

// The scale of numbers whose largest absolute value has these bits: a sixth of it in bfloat16, at most what 6 times is finite of.  (A
// float32 quotient by 6 never falls on the middle of two bfloat16 numbers unless the exact one does, so that rounding it again is
// rounding once.)  NaN where a number is not finite: its bits are then at least those of infinity.
constexpr float kMostScale = 0x1.54p125f;
__device__ __forceinline__ uint16_t scale_of(uint32_t largest) {
  if (largest >= 0x7f800000u) return 0x7fc0;
  return as_type<uint16_t>(fminf(__uint_as_float(largest) / 6.f, kMostScale));
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

// Eight rotated elements of a key from element d on.
template <typename T, bool VEC>
__device__ __forceinline__ void rotated_eight(const AppendArgs &a, const float *row, const T *x, int32_t d, float (&v)[8]) {
  load<T, 8>(x + d, v);
  const int32_t half = a.rot / 2;
  if (a.interleaved) {
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const int32_t j = (d + e) / 2;
      if (j < half) turn(v[e], v[e + 1], row[j], row[half + j]);
    }
  } else if constexpr (VEC) {
    if (d >= a.rot) return;
    const bool upper = d >= half;
    const int32_t j = upper ? d - half : d;
    float u[8], c[8], s[8];
    load<T, 8>(x + (upper ? j : half + j), u);
    load<float, 8>(row + j, c);
    load<float, 8>(row + half + j, s);
    // the upper one of a pair is turned by the other sign
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float) fma((double) u[e], (double) (upper ? s[e] : -s[e]), (double) v[e] * (double) c[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (d + e >= a.rot) continue;
      const bool upper = d + e >= half;
      const int32_t j = upper ? d + e - half : d + e;
      const float u = as_float<T>(x[upper ? j : half + j]), s = row[half + j];
      v[e] = (float) fma((double) u, (double) (upper ? s : -s), (double) v[e] * (double) row[j]);
    }
  }
}

// Queries a part a thread in the first blocks; keys and values 16 lanes a head, eight elements each, in the others.
template <typename T, bool VEC>
__global__ __launch_bounds__(kThreads) void append4_kernel(AppendArgs a, Counts n, Deal<T> deal, uint32_t q_blocks) {
  uint32_t t, i;
  Place p;
  if (blockIdx.x < q_blocks) {
    uint32_t head, part;
    split_by(blockIdx.x * kThreads + threadIdx.x, (uint32_t) n.token, n.magic_token, t, i);
    if (t >= a.T || !place_of(a, t, p)) return;
    split_by(i, (uint32_t) n.part, n.magic_part, head, part);
    rotate_part<T, VEC>(a, deal, (int32_t) part, p.row, reinterpret_cast<const T *>(a.q) + (int64_t) t * a.q_tok + head * a.q_head,
                        reinterpret_cast<T *>(a.q_out) + (int64_t) t * a.o_tok + head * a.o_head);
    return;
  }
  const uint32_t group = ((blockIdx.x - q_blocks) * kThreads + threadIdx.x) / 16;
  const int32_t lane = threadIdx.x & 15, d = 8 * lane;
  t = group / (2 * a.kv_heads);
  i = group - t * (2 * a.kv_heads);
  if (t >= a.T || !place_of(a, t, p)) return;           // all 16 lanes
  const bool value = (int32_t) i >= a.kv_heads;
  const int64_t head = value ? i - a.kv_heads : i;
  const T *x = value ? reinterpret_cast<const T *>(a.v_new) + (int64_t) t * a.v_tok + head * a.v_head
                     : reinterpret_cast<const T *>(a.k_new) + (int64_t) t * a.k_tok + head * a.k_head;
  float v[8] = {};
  if (d < a.D) {
    if (value || !p.row) load<T, 8>(x + d, v);
    else rotated_eight<T, VEC>(a, p.row, x, d, v);
  }
  uint32_t largest = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) largest = max(largest, __float_as_uint(v[e]) & 0x7fffffffu);
  const uint16_t scale = scale_of(max16(largest));
  const float s = as_float<uint16_t>(scale);
  const uint32_t codes = s > 0.f ? codes_of(v, 1.0 / (double) s) : 0;          // all zero, or NaN
  if (d < (a.D + 31) / 32 * 32) {
    uint8_t *to = reinterpret_cast<uint8_t *>(value ? a.v : a.k) + p.page * a.page_stride + p.slot * a.slot_stride + head * a.head_stride;
    *reinterpret_cast<uint32_t *>(to + 4 * lane) = codes;
  }
  if (lane == 0) a.scales[2 * (p.page * a.s_page + p.slot * a.s_slot + head * a.s_head) + (value ? 1 : 0)] = scale;
}

// Eight elements of a key or value a thread.
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
  const bool value = (int32_t) head >= r.kv_heads;
  const int64_t h = value ? head - r.kv_heads : head;
  const uint32_t w = *reinterpret_cast<const uint32_t *>((value ? r.v : r.k) + page * r.page_stride + at * r.slot_stride + h * r.head_stride +
                                                         4 * part);
  const uint16_t scale = r.scales[2 * (page * r.s_page + at * r.s_slot + h * r.s_head) + (value ? 1 : 0)];
  float s = as_float<uint16_t>(scale);
  s = fmaf(s, 0.f, s);                 // what is not finite is NaN
  float x[8];
  auto two = [&](floatx2 y, int e) {
    x[e] = y[0] * s;
    x[e + 1] = y[1] * s;
  };
  two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 0), 0);
  two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 1), 2);
  two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 2), 4);
  two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 3), 6);
  T *to = value ? reinterpret_cast<T *>(r.v_out) + (int64_t) t * r.v_tok + h * r.v_head : reinterpret_cast<T *>(r.k_out) + (int64_t) t * r.k_tok + h * r.k_head;
  store<T, 8>(to + 8 * part, x);
}

uint32_t magic(int32_t d) { return d > 1 ? (uint32_t) (((uint64_t) 1 << 32) / (uint32_t) d) : UINT32_MAX; }
uint32_t blocks(int64_t threads) { return (uint32_t) ((threads + kThreads - 1) / kThreads); }

template <typename T>
hipError_t go(const AppendArgs &a, hipStream_t stream) {
  constexpr int E = Deal<T>::E;
  const Deal<T> deal(a.D, a.rot, a.interleaved);
  // parts of pairs and of the table in whole, aligned pieces of 16 bytes (eight elements where codes are formed)
  const int32_t whole = a.scales ? 8 : E;
  const bool vec = a.rot / 2 % whole == 0 && a.table_stride % 4 == 0 && (uintptr_t) a.table % 16 == 0;
  Counts n;
  n.part = deal.all;
  n.magic_part = magic(n.part);
  if (a.scales) {
    n.token = a.q ? a.heads * deal.all : 1;
    n.magic_token = magic(n.token);
    const uint32_t q_blocks = a.q ? blocks(a.T * n.token) : 0, kv_blocks = blocks(a.T * a.kv_heads * 32);
    if (vec) append4_kernel<T, true><<<q_blocks + kv_blocks, kThreads, 0, stream>>>(a, n, deal, q_blocks);
    else append4_kernel<T, false><<<q_blocks + kv_blocks, kThreads, 0, stream>>>(a, n, deal, q_blocks);
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
  n.token = 2 * r.kv_heads * n.part;
  n.magic_part = magic(n.part);
  n.magic_token = magic(n.token);
  if (bf16) cache4_read_kernel<uint16_t><<<blocks(r.T * n.token), kThreads, 0, stream>>>(r, n);
  else cache4_read_kernel<float><<<blocks(r.T * n.token), kThreads, 0, stream>>>(r, n);
  return hipGetLastError();
}

}  // namespace pcg
