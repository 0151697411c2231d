// Attention of new tokens over a paged cache, and of packed prompts over themselves (gfx950, wave64).
//
// A query head reads the keys of its group's shared head, so the rows of one shared head are numbered
// r = t * G + g (t the new token, g the query head inside the group) and 32 of them make the columns of
// one wave's products:
//   S^T = K Q^T   keys x rows, 32 x 32 blocks; a lane holds one row's scores of half of the keys
//   O^T = V^T P^T d x rows; the scores' registers, exponentiated, are the operand as they stand
// so a row's maximum and sum stay in one lane pair, scaling a row is one multiplication per register, and
// the weights never pass through LDS.  One pass with the running maximum and sum of the softmax, in float32;
// products accumulate in float32.
#include <math.h>

#include "pcg_attend.h"
#include "pcg_device.h"
#include "pcg_kernels.h"

namespace pcg {

namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

constexpr int kAttendWaves = 4;
constexpr int kAttendThreads = kAttendWaves * kWave;
constexpr float kLag = 8.f;        // how far (in powers of two) a maximum may run ahead of the one in use

// What is read where there is nothing to read: keys behind the last, columns behind D.
__device__ const u32x4 kZeros = {0, 0, 0, 0};

// n / d and n % d for n < 2^32, magic = floor(2^32 / d), 2^32 - 1 for d = 1.
__device__ __forceinline__ void split_by(uint32_t n, uint32_t d, uint32_t magic, uint32_t &q, uint32_t &r) {
  q = __umulhi(n, magic);
  r = n - q * d;
  if (r >= d) { ++q; r -= d; }
}

__device__ __forceinline__ float other_half(float x) {           // the value of lane ^ 32
  return __shfl_xor(x, 32);
}

// One unit of work: 32 * WR rows of one shared head of one request.
struct Unit {
  int32_t first;       // token of the request's first row in the batch
  int32_t ctx;         // position of that token
  int32_t rows;        // rows of the request
  int32_t r0;          // first row of the unit
  int32_t b, head;
};

template <typename T, int DP, int WR>
struct Shape {
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int WK = kAttendWaves / WR;
  static constexpr int KB = WK == 1 && kBf16 ? 2 : 1;           // blocks of 32 keys a wave and tile
  static constexpr int TK = 32 * KB * WK;                       // keys a tile
  static constexpr int RB = DP * (int) sizeof(T);               // bytes of a key
  static constexpr int CH = RB / 16;
  static constexpr int NL = TK * CH / kAttendThreads;           // loads of a thread for keys, and for values
  static constexpr int NQ = RB / 32;                            // 16-byte parts of a row that a lane holds
  static constexpr int NO = DP / 32;
  static constexpr int kTileBytes = TK * RB;
  static constexpr int kPartBytes = WK > 1 ? WR * (DP + 2) * 32 * 4 : 0;       // a wave's rows on their way to another
  static constexpr int kLdsBytes = 2 * kTileBytes > kPartBytes ? 2 * kTileBytes : kPartBytes;
};

// Where 16-byte chunk `ch` of row `row` lies in a tile of keys or values.  A wave reads the same chunk of
// 16 consecutive keys at a time: they have to differ modulo 256 bytes.
template <int RB>
__device__ __forceinline__ int key_at(int row, int ch) {
  if constexpr (RB >= 256) return row * RB + ((ch ^ (row & 15)) << 4);
  else return row * RB + ((ch ^ ((row >> 1) & 7)) << 4);
}
// Values: bf16 reads 64 bytes of four consecutive keys at a time, float32 128 bytes of two keys that are four apart.
template <int RB, bool BF16>
__device__ __forceinline__ int value_at(int row, int ch) {
  if constexpr (!BF16) return row * RB + ((ch ^ (((row >> 2) & 1) << 3)) << 4);
  else if constexpr (RB >= 256) return row * RB + ((ch ^ ((row & 3) << 2)) << 4);
  else return row * RB + ((ch ^ (((row >> 1) & 1) << 2)) << 4);
}

template <bool BF16>
__device__ __forceinline__ bool not_finite(uint32_t x) {
  if constexpr (BF16) return (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u;
  else return (x & 0x7f800000u) == 0x7f800000u;
}

template <typename T>
__device__ __forceinline__ float lds_value(const unsigned char *p) {
  if constexpr (sizeof(T) == 2) return __uint_as_float((uint32_t) *reinterpret_cast<const uint16_t *>(p) << 16);
  else return *reinterpret_cast<const float *>(p);
}

// Rows of a unit over keys [k_lo, k_hi): O (not yet divided), the row's reference maximum (log2 units) and sum.
template <typename T, int DP, int WR, bool PAGED>
__device__ __forceinline__ void attend_keys(const AttendArgs &a, const Unit &u, int32_t k_lo, int32_t k_hi,
                                            unsigned char *lds, int *flag, const u32x4 (&qf)[Shape<T, DP, WR>::NQ],
                                            int32_t pos, int32_t min_hi, int32_t max_lo,
                                            floatx16 (&o)[Shape<T, DP, WR>::NO], float &ref, float &sum) {
  using S = Shape<T, DP, WR>;
  constexpr bool kBf16 = S::kBf16;
  constexpr int E = 16 / (int) sizeof(T);
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, half = lane >> 5, wk = wave / WR;
  unsigned char *lk = lds, *lv = lds + S::kTileBytes;
  const int ch = tid % S::CH, row0 = tid / S::CH;
  const bool in_d = ch * E < a.D;
  const char *kb = reinterpret_cast<const char *>(a.k) + ((int64_t) u.head * a.k_head + ch * E) * (int) sizeof(T);
  const char *vb = reinterpret_cast<const char *>(a.v) + ((int64_t) u.head * a.v_head + ch * E) * (int) sizeof(T);
  const int32_t *table = PAGED ? a.table + (int64_t) u.b * a.table_stride : nullptr;

  u32x4 rk[S::NL], rv[S::NL];
  auto fetch = [&](int32_t k0) {
#pragma unroll
    for (int i = 0; i < S::NL; ++i) {
      const int32_t key = k0 + row0 + i * (kAttendThreads / S::CH);
      bool there = key < k_hi && in_d;
      int64_t ok, ov;
      if constexpr (PAGED) {
        uint32_t block, slot;
        split_by((uint32_t) key, (uint32_t) a.page_size, a.magic_page, block, slot);
        there = there && block < (uint32_t) a.max_blocks;
        const int32_t page = there ? table[block] : 0;
        there = there && (uint32_t) page < (uint32_t) a.num_pages;
        ok = (int64_t) page * a.k_page + (int64_t) slot * a.k_tok;
        ov = (int64_t) page * a.v_page + (int64_t) slot * a.v_tok;
      } else {
        ok = (int64_t) (u.first + key) * a.k_tok;
        ov = (int64_t) (u.first + key) * a.v_tok;
      }
      const char *none = reinterpret_cast<const char *>(&kZeros);
      rk[i] = *reinterpret_cast<const u32x4 *>(there ? kb + ok * (int) sizeof(T) : none);
      rv[i] = *reinterpret_cast<const u32x4 *>(there ? vb + ov * (int) sizeof(T) : none);
    }
  };

  fetch(k_lo);
  for (int32_t k0 = k_lo; k0 < k_hi; k0 += S::TK) {
    // some row does not see all of the tile's keys
    const bool edge = k0 + S::TK > min_hi || k0 < max_lo;
    __syncthreads();
    if (edge) {
      bool odd = false;
#pragma unroll
      for (int i = 0; i < S::NL; ++i)
        odd = odd || not_finite<kBf16>(rv[i].x) || not_finite<kBf16>(rv[i].y) || not_finite<kBf16>(rv[i].z) ||
              not_finite<kBf16>(rv[i].w);
      if (tid == 0) *flag = 0;
      __syncthreads();
      if (odd) *flag = 1;
    }
#pragma unroll
    for (int i = 0; i < S::NL; ++i) {
      const int row = row0 + i * (kAttendThreads / S::CH);
      *reinterpret_cast<u32x4 *>(lk + key_at<S::RB>(row, ch)) = rk[i];
      *reinterpret_cast<u32x4 *>(lv + value_at<S::RB, kBf16>(row, ch)) = rv[i];
    }
    __syncthreads();
    if (k0 + S::TK < k_hi) fetch(k0 + S::TK);

    const int base = wk * 32 * S::KB;        // this wave's keys in the tile
    floatx16 s[S::KB];
#pragma unroll
    for (int kb2 = 0; kb2 < S::KB; ++kb2) {
      s[kb2] = floatx16{};
#pragma unroll
      for (int i = 0; i < S::NQ; ++i) {
        const u32x4 kf = *reinterpret_cast<const u32x4 *>(lk + key_at<S::RB>(base + kb2 * 32 + l32, 2 * i + half));
        if constexpr (kBf16) {
          s[kb2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf), __builtin_bit_cast(bf16x8, qf[i]),
                                                           s[kb2], 0, 0, 0);
        } else {
          s[kb2] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf.x), __uint_as_float(qf[i].x), s[kb2], 0, 0, 0);
          s[kb2] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf.y), __uint_as_float(qf[i].y), s[kb2], 0, 0, 0);
          s[kb2] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf.z), __uint_as_float(qf[i].z), s[kb2], 0, 0, 0);
          s[kb2] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf.w), __uint_as_float(qf[i].w), s[kb2], 0, 0, 0);
        }
      }
    }
    // register 4 j + i of block kb2 is key base + 32 kb2 + 8 j + 4 half + i
    if (edge) {
      const int32_t lo = a.window > 0 ? pos - a.window : -1;     // sees keys in (lo, pos]
#pragma unroll
      for (int kb2 = 0; kb2 < S::KB; ++kb2)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int32_t key = k0 + base + kb2 * 32 + (r >> 2) * 8 + half * 4 + (r & 3);
          if (key > pos || key <= lo) s[kb2][r] = -INFINITY;
        }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kb2 = 0; kb2 < S::KB; ++kb2)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[kb2][r]);
    mx = fmaxf(mx, other_half(mx)) * a.c;
    if (__builtin_amdgcn_ballot_w64(mx > ref + kLag) != 0) {
      const float now = fmaxf(ref, mx);
      const float f = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ref - now);
      ref = now;
      sum *= f;
#pragma unroll
      for (int n = 0; n < S::NO; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[n][r] *= f;
    }
    const float minus = ref == -INFINITY ? 0.f : -ref;
#pragma unroll
    for (int kb2 = 0; kb2 < S::KB; ++kb2)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[kb2][r] = __builtin_amdgcn_exp2f(fmaf(s[kb2][r], a.c, minus));
        sum += s[kb2][r];
      }
    if (edge && *flag) {
      // A value that is not finite stands in the tile, and not all rows see all keys: one key at a time, and only where its
      // weight is not zero (zero times such a value would be NaN).
#pragma unroll
      for (int kb2 = 0; kb2 < S::KB; ++kb2) {
#pragma nounroll
        for (int n = 0; n < 16; ++n) {
          const float mine = s[kb2][0], theirs = other_half(mine);
#pragma unroll
          for (int r = 0; r < 15; ++r) s[kb2][r] = s[kb2][r + 1];
#pragma unroll
          for (int hh = 0; hh < 2; ++hh) {
            const float w = hh == half ? mine : theirs;
            const int row = base + kb2 * 32 + (n >> 2) * 8 + hh * 4 + (n & 3);
#pragma unroll
            for (int m = 0; m < S::NO; ++m)
#pragma unroll
              for (int r = 0; r < 16; ++r) {
                const int d = m * 32 + (r >> 2) * 8 + half * 4 + (r & 3);
                const float x = lds_value<T>(lv + value_at<S::RB, kBf16>(row, d / E) + d % E * (int) sizeof(T));
                o[m][r] = w != 0.f ? fmaf(w, x, o[m][r]) : o[m][r];
              }
          }
        }
      }
    } else if constexpr (kBf16) {
      // The weights are rounded to bf16 here (half a step, at most 2^-8 of each): the products take bf16 operands, and the
      // values that they multiply carry the same step.  Their sum above is of the unrounded ones.
#pragma unroll
      for (int kb2 = 0; kb2 < S::KB; ++kb2)
#pragma unroll
        for (int c16 = 0; c16 < 2; ++c16) {
          uint32_t pw[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const floatx2 two = {s[kb2][c16 * 8 + 2 * e], s[kb2][c16 * 8 + 2 * e + 1]};
            pw[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(two, bf16x2));
          }
          const bf16x8 pf = __builtin_bit_cast(bf16x8, u32x4{pw[0], pw[1], pw[2], pw[3]});
          // lane 16 p + x of a half reads 4 elements of key x / 4, columns 16 p + 4 (x % 4), and gets back column
          // 16 p + x of the four keys
          const int row = base + kb2 * 32 + c16 * 16 + half * 4 + ((lane & 15) >> 2);
#pragma unroll
          for (int m = 0; m < S::NO; ++m) {
            const int d = m * 32 + ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
            typedef __attribute__((address_space(3))) shortx4 lds4;
            const shortx4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lds4 *) (lv + value_at<S::RB, true>(row, d >> 3) + (d & 4) * 2));
            const shortx4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lds4 *) (lv + value_at<S::RB, true>(row + 8, d >> 3) + (d & 4) * 2));
            typedef short shortx8 __attribute__((ext_vector_type(8)));
            const shortx8 vf = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
            o[m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf), pf, o[m], 0, 0, 0);
          }
        }
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int row = base + (r >> 2) * 8 + half * 4 + (r & 3);
#pragma unroll
        for (int m = 0; m < S::NO; ++m) {
          const int d = m * 32 + l32;
          const float x = *reinterpret_cast<const float *>(lv + value_at<S::RB, false>(row, d >> 2) + (d & 3) * 4);
          o[m] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, s[0][r], o[m], 0, 0, 0);
        }
      }
    }
  }
}

// Finds the unit that workgroup `index` works on: the requests' row blocks, one after the other.  False: none.
template <int R>
__device__ __forceinline__ bool find_unit(const AttendArgs &a, int32_t index, Unit &u) {
  const int lane = threadIdx.x & (kWave - 1);
  int32_t before = 0;
  for (int32_t b0 = 0; b0 < a.B; b0 += kWave) {
    const int32_t b = b0 + lane;
    int32_t first = 0, n = 0;
    if (b < a.B) {
      first = max(a.q_start[b], 0);
      n = max(min(a.q_start[b + 1], a.T) - first, 0);
    }
    const int32_t blocks = (int32_t) (((int64_t) n * a.G + R - 1) / R);
    int32_t upto = blocks;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
      const int32_t x = __shfl_up(upto, d);
      if (lane >= d) upto += x;
    }
    const uint64_t past = __builtin_amdgcn_ballot_w64(before + upto > index);
    if (past) {
      const int l = __ffsll((long long) past) - 1;
      u.b = b0 + l;
      u.first = __builtin_amdgcn_readlane(first, l);
      const int32_t nn = __builtin_amdgcn_readlane(n, l);
      u.rows = nn * a.G;
      u.r0 = (index - before - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(blocks, l))) * R;
      u.ctx = a.lens ? min(max(a.lens[u.b], 0), a.max_ctx) : 0;
      return true;
    }
    before += __builtin_amdgcn_readlane(upto, kWave - 1);
  }
  return false;
}

template <typename T, int DP, int WR, bool PAGED>
__global__ __launch_bounds__(kAttendThreads) void attend_kernel(AttendArgs a) {
  using S = Shape<T, DP, WR>;
  constexpr int R = 32 * WR;
  constexpr int E = 16 / (int) sizeof(T);
  __shared__ __align__(16) unsigned char lds[S::kLdsBytes];
  __shared__ int flag;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, half = lane >> 5, wr = wave % WR, wk = wave / WR;
  Unit u;
  if (!find_unit<R>(a, (int32_t) (blockIdx.x / (uint32_t) a.heads_kv), u)) return;
  u.head = (int32_t) (blockIdx.x % (uint32_t) a.heads_kv);

  const int32_t r = u.r0 + wr * 32 + l32;
  const bool mine = r < u.rows;
  uint32_t t, g;
  split_by((uint32_t) (mine ? r : 0), (uint32_t) a.G, a.magic_G, t, g);
  const int32_t pos = u.ctx + (int32_t) t;
  const int32_t head = u.head * a.G + (int32_t) g;
  u32x4 qf[S::NQ];
  {
    const T *q = reinterpret_cast<const T *>(a.q) + (int64_t) (u.first + (int32_t) t) * a.q_tok + (int64_t) head * a.q_head;
#pragma unroll
    for (int i = 0; i < S::NQ; ++i) {
      const int d = (2 * i + half) * E;
      qf[i] = *(mine && d < a.D ? reinterpret_cast<const u32x4 *>(q + d) : &kZeros);
    }
  }
  const int32_t t_first = u.r0 / a.G, t_last = (min(u.r0 + R, u.rows) - 1) / a.G;
  const int32_t k_hi = u.ctx + t_last + 1, min_hi = u.ctx + t_first + 1;
  const int32_t k_lo = a.window > 0 ? max(0, min_hi - a.window) : 0;
  const int32_t max_lo = a.window > 0 ? k_hi - a.window : 0;

  floatx16 o[S::NO];
#pragma unroll
  for (int n = 0; n < S::NO; ++n) o[n] = floatx16{};
  float ref = -INFINITY, sum = 0.f;
  attend_keys<T, DP, WR, PAGED>(a, u, k_lo, k_hi, lds, &flag, qf, pos, min_hi, max_lo, o, ref, sum);
  sum += other_half(sum);

  if constexpr (S::WK > 1) {
    // the waves that had the other keys of these rows, one after the other, through LDS
    float *part = reinterpret_cast<float *>(lds) + wr * (DP + 2) * 32;
#pragma unroll
    for (int w = 1; w < S::WK; ++w) {
      __syncthreads();
      if (wk == w) {
#pragma unroll
        for (int n = 0; n < S::NO; ++n)
#pragma unroll
          for (int i = 0; i < 16; ++i) part[(n * 32 + (i >> 2) * 8 + half * 4 + (i & 3)) * 32 + l32] = o[n][i];
        if (half == 0) {
          part[DP * 32 + l32] = ref;
          part[(DP + 1) * 32 + l32] = sum;
        }
      }
      __syncthreads();
      if (wk == 0) {
        const float theirs = part[DP * 32 + l32], now = fmaxf(ref, theirs);
        const float f0 = now == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref - now);
        const float f1 = now == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(theirs - now);
        ref = now;
        sum = sum * f0 + part[(DP + 1) * 32 + l32] * f1;
#pragma unroll
        for (int n = 0; n < S::NO; ++n)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            o[n][i] = o[n][i] * f0 + part[(n * 32 + (i >> 2) * 8 + half * 4 + (i & 3)) * 32 + l32] * f1;
      }
    }
    if (wk != 0) return;
  }
  if (!mine) return;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  T *out = reinterpret_cast<T *>(a.out) + (int64_t) (u.first + (int32_t) t) * a.o_tok + (int64_t) head * a.o_head;
#pragma unroll
  for (int n = 0; n < S::NO; ++n)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int d = n * 32 + j * 8 + half * 4;
      if (d >= a.D) continue;
      if constexpr (S::kBf16) {
        const floatx2 x = {o[n][4 * j] * inv, o[n][4 * j + 1] * inv}, y = {o[n][4 * j + 2] * inv, o[n][4 * j + 3] * inv};
        *reinterpret_cast<uint2 *>(out + d) = make_uint2(__builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2)),
                                                         __builtin_bit_cast(uint32_t, __builtin_convertvector(y, bf16x2)));
      } else {
        *reinterpret_cast<float4 *>(out + d) = make_float4(o[n][4 * j] * inv, o[n][4 * j + 1] * inv, o[n][4 * j + 2] * inv,
                                                           o[n][4 * j + 3] * inv);
      }
    }
}

template <typename T, int DP, int WR, bool PAGED>
hipError_t go(const AttendArgs &a, hipStream_t stream) {
  const int64_t units = (int64_t) a.T * a.G / (32 * WR) + a.B;
  attend_kernel<T, DP, WR, PAGED><<<dim3((uint32_t) (units * a.heads_kv)), kAttendThreads, 0, stream>>>(a);
  return hipGetLastError();
}

template <typename T, int DP>
hipError_t go_rows(const AttendArgs &a, int64_t longest, hipStream_t stream) {
  const int64_t rows = longest * a.G;
  if constexpr (DP * sizeof(T) <= 256) {
    if (rows <= 32) return a.table ? go<T, DP, 1, true>(a, stream) : go<T, DP, 1, false>(a, stream);
  }
  if (rows <= 64) return a.table ? go<T, DP, 2, true>(a, stream) : go<T, DP, 2, false>(a, stream);
  return a.table ? go<T, DP, 4, true>(a, stream) : go<T, DP, 4, false>(a, stream);
}

}  // namespace

size_t attend_workspace_bytes(int32_t, int32_t, int64_t) { return 256; }

hipError_t launch_attend(const AttendArgs &a, bool bf16, int64_t longest, hipStream_t stream) {
  if (bf16) return a.D <= 64 ? go_rows<uint16_t, 64>(a, longest, stream) : go_rows<uint16_t, 128>(a, longest, stream);
  return a.D <= 64 ? go_rows<float, 64>(a, longest, stream) : go_rows<float, 128>(a, longest, stream);
}

}  // namespace pcg
