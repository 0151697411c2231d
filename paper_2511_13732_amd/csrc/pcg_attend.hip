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
//
// Keys and values go from memory straight into LDS.  attend_thick_kernel (a cache) and attend_prompt_kernel (prompts beside their
// keys) let the four waves of a workgroup share tiles of keys: 128 rows, 32 a wave, or 64 rows, two waves on the two halves of a
// tile.  attend_thin_kernel: 32 rows of float32, each wave with keys of its own.  A cache's keys are split over the whole chip in
// runs of equal length (see Run), and attend_join_kernel joins the rows of what was split.
#include <math.h>

#include "pcg_attend.h"
#include "pcg_device.h"
#include "pcg_kernels.h"

namespace pcg {

namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef short shortx8 __attribute__((ext_vector_type(8)));

constexpr int kAttendWaves = 4;
constexpr int kAttendThreads = kAttendWaves * kWave;
constexpr int kThickRows = 32 * kAttendWaves;
constexpr int kCUs = 256;
// See Run.  kCost 0, 1, 2, 4: 64 sequences with 9 new tokens 82.5, 79.2, 76.9, 77.8 us, prompts by pieces 267, 262, 257, 258.
constexpr int kCost = 1, kThinLeast = 1;
constexpr int kJoinThreads = 256;
constexpr int kOrdered = 128;      // see find_place
constexpr float kLag = 8.f;        // how far (in powers of two) a maximum may run ahead of the one in use
constexpr float kFar = 16777216.f; // where half a step of a reference is a factor of two

// What is read where there is nothing to read: keys behind the last, columns behind D.
__device__ const u32x4 kZeros = {0, 0, 0, 0};

// n / d and n % d for n < 2^32, magic = floor(2^32 / d), 2^32 - 1 for d = 1.
__device__ __forceinline__ void split_by(uint32_t n, uint32_t d, uint32_t magic, uint32_t &q, uint32_t &r) {
  q = __umulhi(n, magic);
  r = n - q * d;
  if (r >= d) { ++q; r -= d; }
}

// Element i of an array that nothing writes while the kernel runs: by the scalar unit where i is the same in all lanes.
__device__ __forceinline__ int32_t fixed_at(const int32_t *p, int64_t i) {
  return ((const __attribute__((address_space(4))) int32_t *) p)[i];
}

// max and sum of a lane and lane ^ 32
__device__ __forceinline__ float pair_max(float x) {
  const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float pair_sum(float x) {
  const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// Waits until at most N of this wave's vector-memory operations are still in flight, and keeps reads of what they bring behind.
template <int N>
__device__ __forceinline__ void wait_vm() {
  static_assert(N < 64, "the counter has six bits");
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
  asm volatile("" ::: "memory");
}
// This wave's reads of LDS are through: what they read may be overwritten.
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// Meets the other waves without waiting for loads in flight.
__device__ __forceinline__ void bare_barrier() {
  wait_lds();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <typename T, int DP>
struct Shape {
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int E = 16 / (int) sizeof(T);                // elements of 16 bytes
  static constexpr int RB = DP * (int) sizeof(T);               // bytes of a key
  static constexpr int CH = RB / 16;
  static constexpr int RPI = kWave / CH;                        // keys that one load of a wave brings
  static constexpr int NQ = RB / 32;                            // 16-byte parts of a row that a lane holds
  static constexpr int NO = DP / 32;
};

// Which 16-byte chunk of key `row` lies at chunk position `pos` of its row in LDS (and the other way round).  A wave reads the
// same chunk of 16 consecutive keys at a time: they have to differ modulo 256 bytes.
template <int RB>
__device__ __forceinline__ int key_swap(int row, int pos) {
  if constexpr (RB >= 256) return pos ^ (row & 15);
  else return pos ^ ((row >> 1) & 7);
}
// Values: bf16 reads 64 bytes of four consecutive keys at a time, float32 128 bytes of two keys that are four apart.
template <int RB, bool BF16>
__device__ __forceinline__ int value_swap(int row, int pos) {
  if constexpr (!BF16) return pos ^ (((row >> 2) & 1) << 3);
  else if constexpr (RB >= 256) return pos ^ ((row & 3) << 2);
  else return pos ^ (((row >> 1) & 1) << 2);
}
template <int RB>
__device__ __forceinline__ int key_at(int row, int ch) { return row * RB + (key_swap<RB>(row, ch) << 4); }
template <int RB, bool BF16>
__device__ __forceinline__ int value_at(int row, int ch) { return row * RB + (value_swap<RB, BF16>(row, ch) << 4); }

template <bool BF16>
__device__ __forceinline__ bool not_finite(u32x4 x) {
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    odd = odd || (x[i] & 0x7f800000u) == 0x7f800000u;
    if constexpr (BF16) odd = odd || (x[i] & 0x7f80u) == 0x7f80u;
  }
  return odd;
}

// A block of rows of one shared head of one request.
struct Unit {
  int32_t b, head;
  int32_t first;       // token of the request's first row in the batch
  int32_t rows;        // rows of the request
  int32_t ctx;         // position of its first row's token
  int32_t r0;          // first row of the block
  int32_t k_lo, k_hi;  // keys that some row sees, from a multiple of 32
  int32_t min_hi;      // all rows see keys [max_lo, min_hi)
  int32_t max_lo;
};

// The same in all lanes: in scalar registers from here on.
__device__ __forceinline__ int32_t scalar(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t scalar(int64_t x) {
  return (int64_t) ((uint64_t) (uint32_t) scalar((int32_t) (x >> 32)) << 32 | (uint32_t) scalar((int32_t) x));
}
__device__ __forceinline__ Unit scalar(const Unit &u) {
  return Unit{scalar(u.b), scalar(u.head), scalar(u.first), scalar(u.rows), scalar(u.ctx),
              scalar(u.r0), scalar(u.k_lo), scalar(u.k_hi), scalar(u.min_hi), scalar(u.max_lo)};
}

template <int R>
__device__ __forceinline__ void unit_keys(const AttendArgs &a, Unit &u) {
  uint32_t t_first, t_last, g;
  split_by((uint32_t) u.r0, (uint32_t) a.G, a.magic_G, t_first, g);
  split_by((uint32_t) (min(u.r0 + R, u.rows) - 1), (uint32_t) a.G, a.magic_G, t_last, g);
  u.k_hi = u.ctx + (int32_t) t_last + 1;
  u.min_hi = u.ctx + (int32_t) t_first + 1;
  u.k_lo = a.window > 0 ? max(0, u.min_hi - a.window) & ~31 : 0;
  u.max_lo = a.window > 0 ? u.k_hi - a.window : 0;
}

// First row and tokens of request b.  Whatever q_start holds, nothing outside the batch is named.
__device__ __forceinline__ int32_t request_tokens(const AttendArgs &a, int32_t b, int32_t &first) {
  first = max(fixed_at(a.q_start, b), 0);
  return max(min(fixed_at(a.q_start, b + 1), a.T) - first, 0);
}
__device__ __forceinline__ int32_t request_ctx(const AttendArgs &a, int32_t b) {
  return a.lens ? min(max(fixed_at(a.lens, b), 0), a.max_ctx) : 0;
}

// 16 bytes a lane from memory to 1024 bytes of LDS in a row.  Written as instructions because the compiler waits for all such
// loads in flight ahead of a transposing read of LDS (ds_read_b64_tr_b16), whatever buffer they fill; the kernels wait themselves
// (wait_vm).  They bring nothing into registers, and what the compiler counts of its own loads stays right: it only waits longer.
// The place in LDS is handed over in m0 as an operand, so that the compiler knows what m0 holds.  It sees no load in these, though, and
// leaves no room ahead of one: a load may take an address from scalar registers five wait states after a vector instruction (a spilled
// scalar's way back is one) wrote them, and m0 after one.  Hence s_nop 4.
__device__ __forceinline__ uint32_t lds_address(const unsigned char *p) {
  return (uint32_t) (uintptr_t) (const __attribute__((address_space(3))) unsigned char *) p;
}
__device__ __forceinline__ void bring(const char *from, const unsigned char *to) {
  asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, off" :: "v"(from), "{m0}"(lds_address(to)) : "memory");
}
// N of them to N KB in a row, load i from base + offset[i] - kBias + 1024 i: what an instruction's own offset adds to the place in
// LDS it adds to the address as well.
constexpr uint32_t kBias = 3 * 1024;
// ONCE: what is read is not read again by others, and need not stay in the caches.  us with the hint and without: 32 sequences of
// 4000 keys with 9 new tokens 103 and 117, with 17 111 and 128; 2 of 120 000 with 9 158 and 178; 8 of 2000, which the caches would
// have kept from call to call, 30 and 29; prompts by pieces, whose keys others read too, 370 and 316.
#define PCG_BRING(HINT) \
  if constexpr (N == 4) { \
    asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, %4" HINT "\n\tglobal_load_lds_dwordx4 %1, %4 offset:0x400" HINT \
                 "\n\tglobal_load_lds_dwordx4 %2, %4 offset:0x800" HINT "\n\tglobal_load_lds_dwordx4 %3, %4 offset:0xc00" HINT \
                 :: "v"(offset[0]), "v"(offset[1]), "v"(offset[2]), "v"(offset[3]), "s"(base), "{m0}"(m) : "memory"); \
  } else if constexpr (N == 2) { \
    asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, %2" HINT "\n\tglobal_load_lds_dwordx4 %1, %2 offset:0x400" HINT \
                 :: "v"(offset[0]), "v"(offset[1]), "s"(base), "{m0}"(m) : "memory"); \
  } else { \
    asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" HINT :: "v"(offset[0]), "s"(base), "{m0}"(m) : "memory"); \
  }
template <int N, bool ONCE>
__device__ __forceinline__ void bring_some(const char *base, const uint32_t *offset, const unsigned char *to) {
  static_assert(N == 1 || N == 2 || N == 4, "");
  const uint32_t m = lds_address(to);
  base -= kBias;
  if constexpr (ONCE) {
    PCG_BRING(" nt")
  } else {
    PCG_BRING("")
  }
}
#undef PCG_BRING

// Brings ROWS keys or values of a unit, beginning at key k0, into LDS, dealt to NW waves: keys in a row to each, loads of
// 16 bytes a lane.  PAGES 0: the batch's own rows; 1: pages of a multiple of 16 slots, so that 16 keys in a row (k0 is a
// multiple of 32) share a page, which the scalar unit looks up; 2: pages of any size, looked up by each lane.  ONCE: no other
// workgroup reads them, see bring_some.  Columns behind D get the row's first ones: keys are cleared there once they are in, values
// make columns that nobody stores.
template <typename T, int DP, int ROWS, int NW, int PAGES, bool ONCE>
struct Loader {
  using S = Shape<T, DP>;
  static constexpr int kRows = ROWS / NW;                             // keys of a wave
  static constexpr int NI = kRows / S::RPI;                           // its loads
  static constexpr int NG = kRows > 16 ? kRows / 16 : 1;              // its groups of 16 keys, or what there are
  static constexpr int NL = NI / NG;                                  // loads of a group
  static constexpr int kAtOnce = NL < 4 ? NL : 4;
  const AttendArgs &a;
  const Unit &u;
  const int lane, wave;
  const int32_t *table;
  const char *kb, *vb;
  uint32_t koff[NL], voff[NL];       // of this lane from the first key of a group, see bring_some

  __device__ __forceinline__ int row_of(int i) const { return wave * kRows + i * S::RPI + lane / S::CH; }
  template <bool VALUES>
  __device__ __forceinline__ int chunk(int row) const {
    const int pos = lane % S::CH;
    const int ch = VALUES ? value_swap<S::RB, S::kBf16>(row, pos) : key_swap<S::RB>(row, pos);
    return ch * S::E < a.D ? ch : 0;
  }
  // Zeros in the columns behind D of the keys that this lane brought, once they are in.
  __device__ __forceinline__ void clear_keys(unsigned char *tile) const {
    if (a.D == DP) return;
#pragma unroll
    for (int i = 0; i < NI; ++i)
      if (key_swap<S::RB>(row_of(i), lane % S::CH) * S::E >= a.D)
        *reinterpret_cast<u32x4 *>(tile + (wave * NI + i) * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
  }
  __device__ __forceinline__ Loader(const AttendArgs &a_, const Unit &u_, int lane_, int wave_)
      : a(a_), u(u_), lane(lane_), wave(wave_), table(PAGES ? a_.table + (int64_t) u_.b * a_.table_stride : nullptr) {
    kb = reinterpret_cast<const char *>(a.k) + (int64_t) u.head * a.k_head * (int) sizeof(T);
    vb = reinterpret_cast<const char *>(a.v) + (int64_t) u.head * a.v_head * (int) sizeof(T);
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const uint32_t in = (uint32_t) (i * S::RPI + lane / S::CH), bias = kBias - (uint32_t) (i % kAtOnce) * 1024;
      koff[i] = (in * (uint32_t) a.k_tok + (uint32_t) (chunk<false>(row_of(i)) * S::E)) * (uint32_t) sizeof(T) + bias;
      voff[i] = (in * (uint32_t) a.v_tok + (uint32_t) (chunk<true>(row_of(i)) * S::E)) * (uint32_t) sizeof(T) + bias;
    }
  }

  // Pages of the keys from k0 on, asked for ahead of their use: of a group (PAGES 1), of each load of this lane (PAGES 2).
  static constexpr int NP = PAGES == 2 ? NI : NG;
  struct Pages {
    int32_t page[NP];
  };
  __device__ __forceinline__ int32_t key_of(int32_t k0, int i) const { return k0 + (PAGES == 2 ? row_of(i) : wave * kRows + 16 * i); }
  __device__ __forceinline__ Pages look_up(int32_t k0) const {
    Pages p;
#pragma unroll
    for (int i = 0; i < NP && PAGES; ++i) {
      uint32_t block, slot;
      split_by((uint32_t) key_of(k0, i), (uint32_t) a.page_size, a.magic_page, block, slot);
      p.page[i] = fixed_at(table, min(block, (uint32_t) a.max_blocks - 1));
    }
    return p;
  }

  template <bool VALUES>
  __device__ __forceinline__ void load(int32_t k0, const Pages &p, unsigned char *tile) const {
    const char *base = VALUES ? vb : kb;
    // of a cache keys and values have the same strides
    const int64_t tok = VALUES && !PAGES ? a.v_tok : a.k_tok;
    const char *from[NP];
    bool valid[NP], whole = PAGES < 2 && k0 + ROWS <= u.k_hi;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int32_t key = key_of(k0, i);
      valid[i] = key < u.k_hi;
      if constexpr (PAGES) {
        uint32_t block, slot;
        split_by((uint32_t) key, (uint32_t) a.page_size, a.magic_page, block, slot);
        valid[i] = valid[i] && block < (uint32_t) a.max_blocks && (uint32_t) p.page[i] < (uint32_t) a.num_pages;
        whole = whole && valid[i];
        from[i] = base + ((int64_t) p.page[i] * a.k_page + (int64_t) slot * tok) * (int) sizeof(T);
      } else {
        from[i] = base + (int64_t) (u.first + key) * tok * (int) sizeof(T);
      }
    }
    unsigned char *to = tile + wave * NI * 1024;
    if (whole) {
#pragma unroll
      for (int i = 0; i < NI; i += kAtOnce) bring_some<kAtOnce, ONCE>(from[i / NL % NP], (VALUES ? voff : koff) + i % NL, to + i * 1024);
    } else {
      // a unit's last tile, pages of odd sizes or outside the cache: zeros where there is no key
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const char *at;
        bool there;
        if constexpr (PAGES == 2) {
          there = valid[i];
          at = from[i] + chunk<VALUES>(row_of(i)) * 16;
        } else {
          there = valid[i / NL] && k0 + row_of(i) < u.k_hi;
          at = from[i / NL] + (int64_t) (VALUES ? voff : koff)[i % NL] - kBias + i % NL % kAtOnce * 1024;
        }
        bring(there ? at : reinterpret_cast<const char *>(&kZeros), to + i * 1024);
      }
    }
  }
};

template <bool BF16>
__device__ __forceinline__ void multiply(floatx16 &s, u32x4 x, u32x4 y) {
  if constexpr (BF16) {
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), s, 0, 0, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(x[e]), __uint_as_float(y[e]), s, 0, 0, 0);
  }
}

// Whether there is nothing to multiply from column d on.  Asked with float32 only, whose products take 64 cycles each and four a
// step; with bf16 the question would cost about what it saves.
template <typename T>
__device__ __forceinline__ bool beyond(int d, int32_t D) { return sizeof(T) == 4 && d > 0 && d >= D; }

// The 16-byte chunk of a key that a lane multiplies in step i: key `base` + lane % 32 of the tile.
template <int RB>
__device__ __forceinline__ u32x4 key_chunk(const unsigned char *lk, int base, int lane, int i) {
  return *reinterpret_cast<const u32x4 *>(lk + key_at<RB>(base + (lane & 31), 2 * i + (lane >> 5)));
}

// Scores of 32 keys: register 4 j + i is key 8 j + 4 half + i.
template <typename T, int DP>
__device__ __forceinline__ void scores(const unsigned char *lk, int lane, const u32x4 (&qf)[Shape<T, DP>::NQ], floatx16 (&s)[1],
                                       int32_t D) {
  using S = Shape<T, DP>;
  s[0] = floatx16{};
#pragma unroll
  for (int i = 0; i < S::NQ; ++i) {
    if (beyond<T>(i * 2 * S::E, D)) break;
    multiply<S::kBf16>(s[0], key_chunk<S::RB>(lk, 0, lane, i), qf[i]);
  }
}

// Keys that the row at position `pos` does not see: beyond it, or at `lo` and before.
__device__ __forceinline__ void hide(floatx16 &s, int32_t key0, int half, int32_t pos, int32_t lo) {
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int32_t key = key0 + (r >> 2) * 8 + half * 4 + (r & 3);
    if (key > pos || key <= lo) s[r] = -INFINITY;
  }
}

// The largest of a row's scores of KB blocks of keys, in log2 units.
template <int KB>
__device__ __forceinline__ float row_max(const floatx16 (&s)[KB], float c) {
  float m[2] = {s[0][0], s[0][1]};
#pragma unroll
  for (int k = 0; k < KB; ++k)
#pragma unroll
    for (int r = k ? 0 : 2; r < 16; ++r) m[r & 1] = fmaxf(m[r & 1], s[k][r]);
  return pair_max(fmaxf(m[0], m[1])) * c;
}

__device__ __forceinline__ float minus_ref(float ref) { return ref == -INFINITY ? 0.f : -ref; }

// The rows' reference maxima follow the maxima where one runs more than kLag ahead (weights stay below 2^kLag, and sums
// and outputs are rarely rescaled).  What the row's scores are to be multiplied by for the weights is returned: c, and the exponent
// c s - ref is then rounded once.  A reference is the rounded c m, though, half a step off, and beyond kFar that is a power of two of
// its own, 2^8 where c m is 2^32: there the scores are replaced by the rounded c s, as the reference is, and 1 is returned.
template <int NO, int KB>
__device__ __forceinline__ float follow(float mx, float &ref, float &sum, floatx16 (&o)[NO], floatx16 (&s)[KB], float c) {
  if (__builtin_amdgcn_ballot_w64(mx > ref + kLag || fabsf(minus_ref(ref)) > kFar) == 0) return c;
  const float now = fmaxf(ref, mx);
  const float f = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ref - now);
  ref = now;
  sum *= f;
#pragma unroll
  for (int n = 0; n < NO; ++n)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[n][r] *= f;
  const bool far = fabsf(minus_ref(ref)) > kFar;
  if (__builtin_amdgcn_ballot_w64(far) == 0) return c;
#pragma unroll
  for (int k = 0; k < KB; ++k)
#pragma unroll
    for (int r = 0; r < 16; ++r) s[k][r] *= far ? c : 1.f;
  return far ? 1.f : c;
}

// Scores to weights 2^(c s - ref), and their sum.
template <int KB>
__device__ __forceinline__ void to_weights(floatx16 (&s)[KB], float c, float minus, float &sum) {
  float z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < KB; ++k)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[k][r] = __builtin_amdgcn_exp2f(fmaf(s[k][r], c, minus));
      z[r & 3] += s[k][r];
    }
  sum += (z[0] + z[1]) + (z[2] + z[3]);
}

// Nothing moves across: the order of instructions around it is the one written.
__device__ __forceinline__ void pin() { __builtin_amdgcn_sched_barrier(0); }

// The same of KB blocks of 32 keys, in steps of one operand of keys that is read kAhead steps ahead.
template <typename T, int DP, int KB>
__device__ __forceinline__ void scores_in_steps(const unsigned char *lk, int lane, const u32x4 (&qf)[Shape<T, DP>::NQ], floatx16 (&s)[KB],
                                                int32_t D) {
  using S = Shape<T, DP>;
  constexpr int kAhead = 3, kSteps = KB * S::NQ;
  u32x4 kf[kAhead + 1];
  auto read = [&](int i) { kf[i % (kAhead + 1)] = key_chunk<S::RB>(lk, 32 * (i / S::NQ), lane, i % S::NQ); };
#pragma unroll
  for (int i = 0; i < kAhead && i < kSteps; ++i) read(i);
#pragma unroll
  for (int k = 0; k < KB; ++k) s[k] = floatx16{};
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    pin();
    if (i + kAhead < kSteps) read(i + kAhead);
    if (!beyond<T>(i % S::NQ * 2 * S::E, D)) multiply<S::kBf16>(s[i / S::NQ], kf[i % (kAhead + 1)], qf[i % S::NQ]);
  }
  pin();
}

// Operand of the product of weights and values: the weights of one 16 keys (bf16) or of two (float32) in a lane.
// The weights are rounded to bf16 here (half a step, at most 2^-8 of each): the products take bf16 operands, and the
// values that they multiply carry the same step.  Their sum is of the unrounded ones.
__device__ __forceinline__ bf16x8 weights_of(const floatx16 &p, int c16) {
  u32x4 pw;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const floatx2 two = {p[c16 * 8 + 2 * e], p[c16 * 8 + 2 * e + 1]};
    pw[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(two, bf16x2));
  }
  return __builtin_bit_cast(bf16x8, pw);
}
// Values of 16 keys, the first at row `base`, columns 32 m ..: lane x of 16 reads 4 elements of key x / 4, columns
// 4 (x % 4), and gets back column x of the four keys.
template <int RB>
__device__ __forceinline__ shortx8 values_of(const unsigned char *lv, int base, int lane, int m) {
  const int row = base + (lane >> 5) * 4 + ((lane & 15) >> 2);
  const int d = m * 32 + ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
  typedef __attribute__((address_space(3))) shortx4 lds4;
  const shortx4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *) (lv + value_at<RB, true>(row, d >> 3) + (d & 4) * 2));
  const shortx4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *) (lv + value_at<RB, true>(row + 8, d >> 3) + (d & 4) * 2));
  return __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
}
// Value of register r's key (of 32 from row `base`), column 32 m + lane % 32.
template <int RB>
__device__ __forceinline__ float value_of(const unsigned char *lv, int base, int lane, int r, int m) {
  const int row = base + (r >> 2) * 8 + (lane >> 5) * 4 + (r & 3), d = m * 32 + (lane & 31);
  return *reinterpret_cast<const float *>(lv + value_at<RB, false>(row, d >> 2) + (d & 3) * 4);
}

// Adds weights times values of 32 keys.
template <int DP>
__device__ __forceinline__ void add_values(const unsigned char *lv, int lane, const floatx16 &p, floatx16 (&o)[DP / 32], int32_t D) {
#pragma unroll
  for (int r = 0; r < 16; ++r)
#pragma unroll
    for (int m = 0; m < DP / 32; ++m) {
      if (beyond<float>(32 * m, D)) break;
      o[m] = __builtin_amdgcn_mfma_f32_32x32x2f32(value_of<DP * 4>(lv, 0, lane, r, m), p[r], o[m], 0, 0, 0);
    }
}

// The same of KB blocks of 32 keys, in steps with the operands read ahead.
template <typename T, int DP, int KB>
__device__ __forceinline__ void add_values_in_steps(const unsigned char *lv, int lane, const floatx16 (&p)[KB],
                                                    floatx16 (&o)[Shape<T, DP>::NO], int32_t D) {
  using S = Shape<T, DP>;
  if constexpr (S::kBf16) {
    constexpr int kAhead = 3, kSteps = KB * 2 * S::NO;
    shortx8 vf[kAhead + 1];
    bf16x8 pf[2];
    auto read = [&](int i) { vf[i % (kAhead + 1)] = values_of<S::RB>(lv, i / S::NO * 16, lane, i % S::NO); };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) read(i);
    pf[0] = weights_of(p[0], 0);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int c = i / S::NO, m = i % S::NO;
      pin();
      if (i + kAhead < kSteps) read(i + kAhead);
      if (m == 0 && c + 1 < 2 * KB) pf[(c + 1) & 1] = weights_of(p[(c + 1) / 2], (c + 1) & 1);
      o[m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[i % (kAhead + 1)]), pf[c & 1], o[m], 0, 0, 0);
    }
    pin();
  } else {
    constexpr int kSteps = KB * 16;
    float x[2][S::NO];
    auto read = [&](int i) {
#pragma unroll
      for (int m = 0; m < S::NO; ++m) x[i & 1][m] = value_of<S::RB>(lv, i / 16 * 32, lane, i % 16, m);
    };
    read(0);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      pin();
      if (i + 1 < kSteps) read(i + 1);
#pragma unroll
      for (int m = 0; m < S::NO; ++m)
        if (!beyond<T>(32 * m, D)) o[m] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i & 1][m], p[i / 16][i % 16], o[m], 0, 0, 0);
    }
    pin();
  }
}

// Zero times a value that is not finite would be NaN in the rows that do not see the value.  Where not all rows see all keys of a
// tile, such values are therefore taken out of it (`threads` threads, this one `index`, `bytes` of values) and, if there were
// any, put afterwards where they are seen (put_odd_values).
template <bool BF16>
__device__ __forceinline__ bool clear_odd_values(unsigned char *lv, int bytes, int index, int threads) {
  bool odd = false;
  for (int i = index * 16; i < bytes; i += threads * 16) {
    u32x4 x = *reinterpret_cast<const u32x4 *>(lv + i);
    if (!not_finite<BF16>(x)) continue;
    odd = true;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (BF16) {
        if ((x[e] & 0x7f80u) == 0x7f80u) x[e] &= 0xffff0000u;
        if ((x[e] & 0x7f800000u) == 0x7f800000u) x[e] &= 0xffffu;
      } else if ((x[e] & 0x7f800000u) == 0x7f800000u) {
        x[e] = 0;
      }
    }
    *reinterpret_cast<u32x4 *>(lv + i) = x;
  }
  return odd;
}

// Whether an element is infinite or NaN.
template <int NO>
__device__ __forceinline__ bool any_odd(const floatx16 (&o)[NO]) {
  float x = 0.f;                        // 0 * o is NaN then
#pragma unroll
  for (int n = 0; n < NO; ++n)
#pragma unroll
    for (int r = 0; r < 16; ++r) x = fmaf(o[n][r], 0.f, x);
  return x != 0.f;
}

// Elements of rows that see a value among keys [k0, k1) which is not finite: the sum of those that the row sees, whatever their
// weights, goes to put(column, sum).  By the formula every weight is positive; one that became zero, here or where a reference moved
// on, would make NaN of an infinity, and which ones do depends on the tiles.  A wave looks at 64 keys at a time, a key a lane, and ends
// where all is NaN.  Called when the rows are stored, so that it needs none of their registers.
template <typename T, int DP, bool PAGED, typename Put>
__device__ __forceinline__ void put_odd_values(const AttendArgs &a, const Unit &u, int32_t k0, int32_t k1, int lane, bool there, int32_t pos,
                                               int32_t lo, Put put) {
  using S = Shape<T, DP>;
  const int half = lane >> 5;
  auto find = [&](int32_t key) -> const T * {             // NULL: reads as zeros
    int64_t at = (int64_t) (u.first + key) * a.v_tok;
    if constexpr (PAGED) {
      uint32_t block, slot;
      split_by((uint32_t) key, (uint32_t) a.page_size, a.magic_page, block, slot);
      if (block >= (uint32_t) a.max_blocks) return nullptr;
      const int32_t page = a.table[(int64_t) u.b * a.table_stride + block];
      if ((uint32_t) page >= (uint32_t) a.num_pages) return nullptr;
      at = (int64_t) page * a.v_page + (int64_t) slot * a.v_tok;
    }
    return reinterpret_cast<const T *>(a.v) + at + (int64_t) u.head * a.v_head;
  };
  floatx16 odd[DP / 32];
#pragma unroll
  for (int m = 0; m < DP / 32; ++m) odd[m] = floatx16{};
#pragma nounroll
  for (; k0 < k1; k0 += kWave) {
    bool here = false;
    const T *v = k0 + lane < k1 ? find(k0 + lane) : nullptr;
    if (v) {
#pragma nounroll
      for (int d = 0; d < a.D; d += S::E) here = not_finite<S::kBf16>(*reinterpret_cast<const u32x4 *>(v + d)) || here;
    }
    uint64_t who = __builtin_amdgcn_ballot_w64(here);
    if (!who) continue;
#pragma nounroll
    for (; who; who &= who - 1) {
      const int32_t key = k0 + __ffsll((long long) who) - 1;
      const T *x = find(key);
      const bool seen = key <= pos && key > lo;
#pragma unroll
      for (int m = 0; m < DP / 32; ++m) {
        asm volatile("" ::: "memory");  // one block of columns after the other: there are no registers for all at a time
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int d = m * 32 + j * 8 + half * 4;
          if (d >= a.D) continue;
          floatx4 y;
          if constexpr (S::kBf16) {
            const u32x2 z = *reinterpret_cast<const u32x2 *>(x + d);
            y = floatx4{__uint_as_float(z[0] << 16), __uint_as_float(z[0] & 0xffff0000u), __uint_as_float(z[1] << 16),
                        __uint_as_float(z[1] & 0xffff0000u)};
          } else {
            y = *reinterpret_cast<const floatx4 *>(x + d);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (seen && !(fabsf(y[i]) < INFINITY)) odd[m][4 * j + i] += y[i];
        }
      }
    }
    bool open = false;
#pragma unroll
    for (int m = 0; m < DP / 32; ++m)
#pragma unroll
      for (int r = 0; r < 16; ++r) open = open || (m * 32 + (r >> 2) * 8 + half * 4 < a.D && odd[m][r] == odd[m][r]);
    if (__builtin_amdgcn_ballot_w64(open && there) == 0) break;
  }
#pragma unroll
  for (int m = 0; m < DP / 32; ++m)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (there && odd[m][r] != 0.f) put(m * 32 + (r >> 2) * 8 + half * 4 + (r & 3), odd[m][r]);
}

// Where a row's query and output are, and its position.
struct Row {
  bool there;
  int32_t pos;
  int64_t token, head;
};
__device__ __forceinline__ Row row_at(const AttendArgs &a, const Unit &u, int32_t r) {
  Row w;
  w.there = r < u.rows;
  uint32_t t, g;
  split_by((uint32_t) (w.there ? r : 0), (uint32_t) a.G, a.magic_G, t, g);
  w.pos = u.ctx + (int32_t) t;
  w.token = u.first + (int32_t) t;
  w.head = u.head * a.G + (int32_t) g;
  return w;
}

template <typename T, int DP>
__device__ __forceinline__ void load_query(const AttendArgs &a, const Row &w, int half, u32x4 (&qf)[Shape<T, DP>::NQ]) {
  using S = Shape<T, DP>;
  const T *q = reinterpret_cast<const T *>(a.q) + w.token * a.q_tok + w.head * a.q_head;
#pragma unroll
  for (int i = 0; i < S::NQ; ++i) {
    const int d = (2 * i + half) * S::E;
    qf[i] = *(w.there && d < a.D ? reinterpret_cast<const u32x4 *>(q + d) : &kZeros);
  }
}

// A row's output from its half in this lane: d = 32 n + 8 j + 4 half + i in register 4 j + i of o[n].  A row without a score above
// -infinity is zeros, also where a value was not finite and its product with the weight zero is NaN.
template <typename T, int DP>
__device__ __forceinline__ void store_row(const AttendArgs &a, const Row &w, int half, const floatx16 (&o)[Shape<T, DP>::NO],
                                          float sum) {
  using S = Shape<T, DP>;
  if (!w.there) return;
  const float inv = 1.f / sum;
  auto of = [&](float x) { return sum == 0.f ? 0.f : x * inv; };
  T *out = reinterpret_cast<T *>(a.out) + w.token * a.o_tok + w.head * a.o_head;
#pragma unroll
  for (int n = 0; n < S::NO; ++n)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int d = n * 32 + j * 8 + half * 4;
      if (d >= a.D) continue;
      if constexpr (S::kBf16) {
        const floatx2 x = {of(o[n][4 * j]), of(o[n][4 * j + 1])}, y = {of(o[n][4 * j + 2]), of(o[n][4 * j + 3])};
        *reinterpret_cast<u32x2 *>(out + d) = u32x2{__builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2)),
                                                    __builtin_bit_cast(uint32_t, __builtin_convertvector(y, bf16x2))};
      } else {
        *reinterpret_cast<floatx4 *>(out + d) = floatx4{of(o[n][4 * j]), of(o[n][4 * j + 1]), of(o[n][4 * j + 2]), of(o[n][4 * j + 3])};
      }
    }
}

// One element of it that is not finite.
template <typename T>
__device__ __forceinline__ void put_out(const AttendArgs &a, const Row &w, int d, float x) {
  T *out = reinterpret_cast<T *>(a.out) + w.token * a.o_tok + w.head * a.o_head;
  if constexpr (sizeof(T) == 2) out[d] = __builtin_bit_cast(uint16_t, (__bf16) x);
  else out[d] = x;
}

// Whether rows of this wave need put_odd_values: values were taken out of a tile, or an element is not finite.  (Of a row whose sum is NaN
// everything is.)
template <int NO>
__device__ __forceinline__ bool odd_rows(bool cleared, const floatx16 (&o)[NO], float sum) {
  return __builtin_amdgcn_ballot_w64((cleared || any_odd<NO>(o)) && sum == sum) != 0;
}

// ---- parts of a unit whose keys are split over workgroups ------------------------------------------------------------------

// Outputs (not divided), reference maxima and sums of R rows.
template <int DP, int R>
struct Part {
  float o[R][DP];
  float ref[R], sum[R];
};

// What attend_join_kernel finds at the workgroup that began a split unit: its parts are this workgroup's slot 1 and slot 0 of
// the parts - 1 that follow.
struct Join {
  int32_t parts, head, r0, rows, first;
};

template <int DP, int R>
__device__ __forceinline__ void store_part(Part<DP, R> *p, int row, int half, bool there, const floatx16 (&o)[DP / 32], float ref,
                                           float sum) {
  if (!there) return;
#pragma unroll
  for (int n = 0; n < DP / 32; ++n)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<floatx4 *>(&p->o[row][n * 32 + j * 8 + half * 4]) =
          floatx4{o[n][4 * j], o[n][4 * j + 1], o[n][4 * j + 2], o[n][4 * j + 3]};
  if (half == 0) {
    p->ref[row] = ref;
    p->sum[row] = sum;
  }
}

// Tiles of TK keys of the unit that begins at row r0.
template <int R, int TK>
__device__ __forceinline__ int32_t unit_tiles(const AttendArgs &a, Unit &u) {
  unit_keys<R>(a, u);
  return (u.k_hi - u.k_lo + TK - 1) / TK;
}

// All units (requests, their shared heads, their row blocks, in this order) in a row, kCost for what a unit costs beside its tiles
// and then 1 for each of them, are cut into `runs` runs of a length, one a workgroup; the first `longer` are one longer than `each`.
struct Run {
  int32_t runs, longer, index;
  int64_t each, left;
  __device__ __forceinline__ int64_t begin(int32_t i) const { return each * i + min(i, longer); }
  // the runs that begin ahead of x (which lies in one of them, or behind all)
  __device__ __forceinline__ int32_t ahead_of(int64_t x) const {
    int32_t lo = 0, hi = runs;
    while (lo < hi) {                   // first run that begins at x or behind it
      const int32_t mid = (lo + hi) >> 1;
      if (begin(mid) < x) lo = mid + 1;
      else hi = mid;
    }
    return lo;
  }
};

// Finds this workgroup's run, of `count` at most, LEAST long at least (but for the last): its first unit and how far into it.
// Every workgroup adds the requests up by itself, each wave its share of them, a request a lane or (with many row blocks) a row block
// a lane: for 64 requests that takes two microseconds, less than a launch ahead would.  Lengths are whole numbers below 2^53 in
// double, whose running sums go through DPP.
template <int R, int TK, int LEAST, int NW>
__device__ __forceinline__ Run find_run(const AttendArgs &a, int32_t count, unsigned char *lds, Unit &u, int64_t &into) {
  double *sums = reinterpret_cast<double *>(lds);
  int32_t *found = reinterpret_cast<int32_t *>(sums + NW);
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int32_t share = (a.B + NW - 1) / NW, b_lo = min(wave * share, a.B), b_hi = min(b_lo + share, a.B);
  // running sum of the lengths of requests b0 .. b0 + lane, all shared heads
  auto lengths = [&](int32_t b0, Unit &v, double &one) -> double {
    v.b = b0 + lane;
    v.rows = v.ctx = 0;
    if (v.b < b_hi) {
      v.rows = request_tokens(a, v.b, v.first) * a.G;
      v.ctx = request_ctx(a, v.b);
    }
    v.r0 = 0;
    one = v.rows > 0 && v.rows <= R ? unit_tiles<R, TK>(a, v) + kCost : 0;
    for (uint64_t many = __builtin_amdgcn_ballot_w64(v.rows > R); many; many &= many - 1) {
      const int l = __ffsll((long long) many) - 1;
      Unit x;
      x.rows = read_lane(v.rows, l);
      x.ctx = read_lane(v.ctx, l);
      double all = 0;
      for (int64_t r0 = (int64_t) lane * R; r0 < x.rows; r0 += kWave * R) {
        x.r0 = (int32_t) r0;
        all += unit_tiles<R, TK>(a, x) + kCost;
      }
      all = wave_sum(all);
      if (lane == l) one = all;
    }
    return wave_scan(one * a.heads_kv);
  };
  Unit v;
  double one, upto = 0, mine = 0;
  for (int32_t b0 = b_lo; b0 < b_hi; b0 += kWave) {
    upto = lengths(b0, v, one);
    mine += read_lane(upto, kWave - 1);
  }
  if (lane == 0) sums[wave] = mine;
  bare_barrier();
  Run run;
  double sum = 0, before = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const double x = sums[w];
    if (w < wave) before += x;
    sum += x;
  }
  const int64_t total = scalar((int64_t) sum);
  run.runs = (int32_t) min((int64_t) count, (total + LEAST - 1) / LEAST);
  // An XCD (every eighth workgroup) takes runs that follow each other: those of a shared head find its keys in its L2.
  const int32_t eighth = (run.runs + 7) / 8;
  run.index = (int32_t) blockIdx.x / 8 < eighth ? (int32_t) (blockIdx.x % 8) * eighth + (int32_t) blockIdx.x / 8 : run.runs;
  run.left = 0;
  if (run.index >= run.runs) return run;
  // a quotient of numbers below 2^53, off by one at most in double
  run.each = scalar((int64_t) ((double) total / (double) run.runs));
  if (run.each * run.runs > total) --run.each;
  if (total - run.each * run.runs >= run.runs) ++run.each;
  run.longer = (int32_t) (total - run.each * run.runs);
  const int64_t begin = run.begin(run.index);
  run.left = run.begin(run.index + 1) - begin;
  double ahead = (double) begin - before;
  if (0 <= ahead && ahead < mine) {
    for (int32_t b0 = b_lo; b0 < b_hi; b0 += kWave) {
      if (share > kWave) upto = lengths(b0, v, one);
      const uint64_t past = __builtin_amdgcn_ballot_w64(upto > ahead);
      if (!past) {
        ahead -= read_lane(upto, kWave - 1);
        continue;
      }
      const int l = __ffsll((long long) past) - 1;
      const double length = read_lane(one, l);
      ahead -= read_lane(upto, l) - length * a.heads_kv;
      int32_t head = (int32_t) (ahead / length);      // off by one at most
      if (head * length > ahead) --head;
      if (ahead - head * length >= length) ++head;
      ahead -= head * length;
      Unit x;
      x.b = b0 + l;
      x.rows = read_lane(v.rows, l);
      x.ctx = read_lane(v.ctx, l);
      x.first = read_lane(v.first, l);
      int32_t r0 = 0;
      for (int64_t c0 = 0; c0 < x.rows && x.rows > R; c0 += kWave * R) {
        const int64_t mine_r0 = c0 + (int64_t) lane * R;
        x.r0 = (int32_t) mine_r0;
        const double t = mine_r0 < x.rows ? unit_tiles<R, TK>(a, x) + kCost : 0, blocks = wave_scan(t);
        const uint64_t in = __builtin_amdgcn_ballot_w64(blocks > ahead);
        if (in) {
          const int k = __ffsll((long long) in) - 1;
          ahead -= read_lane(blocks - t, k);
          r0 = (int32_t) c0 + k * R;
          break;
        }
        ahead -= read_lane(blocks, kWave - 1);
      }
      if (lane == 0) {
        found[0] = x.b;
        found[1] = head;
        found[2] = r0;
        found[3] = (int32_t) ahead;
        found[4] = x.rows;
        found[5] = x.first;
        found[6] = x.ctx;
      }
      break;
    }
  }
  bare_barrier();
  u.b = found[0];
  u.head = found[1];
  u.r0 = found[2];
  into = scalar(found[3]);
  u.rows = found[4];
  u.first = found[5];
  u.ctx = found[6];
  bare_barrier();                       // the tiles of the first piece come here
  return run;
}

// The unit behind u.
template <int R>
__device__ __forceinline__ void next_unit(const AttendArgs &a, Unit &u) {
  u.r0 += R;
  if (u.r0 < u.rows) return;
  u.r0 = 0;
  if (++u.head < a.heads_kv) return;
  u.head = 0;
  do {
    if (++u.b >= a.B) return;
    u.rows = request_tokens(a, u.b, u.first) * a.G;
  } while (u.rows == 0);
  u.ctx = request_ctx(a, u.b);
}

// Calls work(unit, first tile, tiles, part) for every unit or piece of one in this workgroup's run; part: NULL where the unit is
// whole.  A workgroup has two places for parts: 1 for the unit that it begins and does not finish, 0 for one that another began.
template <int DP, int R, int TK, int LEAST, int NW, typename Work>
__device__ __forceinline__ void work_on_run(const AttendArgs &a, unsigned char *lds, Join *join, Part<DP, R> *parts, Work work) {
  Unit u;
  int64_t into = 0;
  Run run = find_run<R, TK, LEAST, NW>(a, (int32_t) gridDim.x, lds, u, into);
  Join j{0, 0, 0, 0, 0};
  // Where a head's keys are read by several row blocks, the end of a unit that another run began comes last: the runs of an XCD then
  // begin with units from their first key on, and those of one head read the same keys at the same time, out of its L2 (us with
  // and without: 1 sequence of 60 000 keys with 2048 new tokens 2004 and 2176, 4 of 8000 with 1024 579 and 612, prompts by pieces 262
  // and 278, 4 of 1000 with 200 51.3 and 51.8).
  int32_t rest_tile = 0, rest_tiles = 0, rest_b = 0, rest_head = 0, rest_r0 = 0;
  while (run.left > 0 || rest_tiles > 0) {
    int32_t tile, tiles;
    Part<DP, R> *part;
    if (run.left > 0) {
      u = scalar(u);
      const int32_t all = scalar(unit_tiles<R, TK>(a, u));
      const int64_t until = min((int64_t) all + kCost, into + run.left);       // in the unit's length
      tile = into > kCost ? (int32_t) into - kCost : 0;
      tiles = until > kCost ? (int32_t) until - kCost - tile : 0;
      run.left -= until - into;
      part = tiles == all ? nullptr : parts + 2 * (int64_t) run.index + (tile == 0);
      if (part && tile == 0 && tiles > 0) {
        // this run and those that begin ahead of the unit's end
        j.parts = run.ahead_of(run.begin(run.index + 1) - run.left + all + kCost - until) - run.index;
        j.head = u.head;
        j.r0 = u.r0;
        j.rows = u.rows;
        j.first = u.first;
      }
      if (R == kThickRows && tile > 0 && run.left > 0) {
        rest_tile = tile;
        rest_tiles = tiles;
        rest_b = u.b;
        rest_head = u.head;
        rest_r0 = u.r0;
        tiles = 0;
      }
    } else {
      tile = rest_tile;
      tiles = rest_tiles;
      rest_tiles = 0;
      u.b = rest_b;
      u.head = rest_head;
      u.r0 = rest_r0;
      u.rows = request_tokens(a, u.b, u.first) * a.G;
      u.ctx = request_ctx(a, u.b);
      u = scalar(u);
      (void) unit_tiles<R, TK>(a, u);
      u = scalar(u);
      part = parts + 2 * (int64_t) run.index;
    }
    if (tiles > 0) work(u, tile, tiles, part);
    into = 0;
    if (run.left > 0) next_unit<R>(a, u);
  }
  if (threadIdx.x != 0) return;
  if (run.index < run.runs) join[run.index] = j;
  if ((int32_t) blockIdx.x >= run.runs) join[blockIdx.x] = Join{0, 0, 0, 0, 0};
}

// ---- 128 rows a workgroup ----------------------------------------------------------------------------------------------

// Rows of a wave on their way to another through LDS: 32 rows' outputs (not divided), references and sums.
template <int DP>
constexpr int kRowsFloats = 32 * (DP + 2);

template <int DP>
__device__ __forceinline__ void give_rows(float *to, int lane, const floatx16 (&o)[DP / 32], float ref, float sum) {
  const int l32 = lane & 31, half = lane >> 5;
#pragma unroll
  for (int n = 0; n < DP / 32; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) to[(n * 32 + (i >> 2) * 8 + half * 4 + (i & 3)) * 32 + l32] = o[n][i];
  const float all = pair_sum(sum);
  if (half == 0) {
    to[DP * 32 + l32] = ref;
    to[(DP + 1) * 32 + l32] = all;
  }
}
template <int DP>
__device__ __forceinline__ void take_rows(const float *from, int lane, floatx16 (&o)[DP / 32], float &ref, float &sum) {
  const int l32 = lane & 31, half = lane >> 5;
  const float theirs = from[DP * 32 + l32], now = fmaxf(ref, theirs);
  const float f0 = now == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref - now);
  const float f1 = now == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(theirs - now);
  ref = now;
  sum = sum * f0 + (half == 0 ? from[(DP + 1) * 32 + l32] * f1 : 0.f);
#pragma unroll
  for (int n = 0; n < DP / 32; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[n][i] = o[n][i] * f0 + from[(n * 32 + (i >> 2) * 8 + half * 4 + (i & 3)) * 32 + l32] * f1;
}

// WK waves share 32 rows and take the keys of a tile in turn, KB blocks of 32 each: R rows a workgroup, tiles of 64 keys (fp32: 32
// where every wave has rows of its own), two in LDS, one in use while the other comes.  64 keys of 128 elements, twice, are 64 KB:
// two workgroups a CU, whose waves fill each other's waits (a third would not find registers: queries, outputs, scores
// and operands on their way take 200 to 224 a lane).  Four waves on 32 rows each bring a tile once for 128 rows; reading
// the operands then keeps LDS busy a quarter of the time.
template <typename T, int DP, int WK>
struct Thick {
  using S = Shape<T, DP>;
  static constexpr int R = kThickRows / WK;
  static constexpr int KB = S::kBf16 && WK == 1 ? 2 : 1;
  static constexpr int TK = 32 * KB * WK;
  static constexpr int kTile = TK * S::RB;
  static constexpr int kLds = 4 * kTile;            // keys and values, two of each
  static constexpr int kRuns = 2 * kLds < 160 * 1024 ? 512 : 256;        // two a CU (up to d = 64 three would fit) or one
  // See Run.  us with runs of 1, 2, 3 and 5 tiles at least, bf16, d = 128: 64 rows, 1 sequence of 1000 keys 13.6 14.5 18.1 20.6, of
  // 8000 27 27 25 24, 8 of 2000 24 24 24 24; 128 rows, 1 of 1000 18 18 21 24, of 8000 39 39 32 28, 4 of 4000 (d = 64) 27 27 27 27.
  static constexpr int kLeast = WK == 1 ? 5 : 1;
};

template <typename T, int DP, int WK, int PAGES, bool ONCE>
__device__ __forceinline__ void thick_piece(const AttendArgs &a, const Unit &u, int32_t tile, int32_t tiles, unsigned char *lds,
                                            int *odd, int turn, Part<DP, Thick<T, DP, WK>::R> *part) {
  using S = Shape<T, DP>;
  using W = Thick<T, DP, WK>;
  constexpr int WR = kAttendWaves / WK;
  int tid = threadIdx.x;
  asm("" : "+v"(tid));                  // what follows from it is formed here, not kept in registers from piece to piece
  const int lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, half = lane >> 5;
  const Loader<T, DP, W::TK, kAttendWaves, PAGES, ONCE> loader(a, u, lane, wave);
  int32_t k0 = u.k_lo + tile * W::TK;
  const int32_t end = min(u.k_hi, k0 + tiles * W::TK);
  unsigned char *cur = lds, *nxt = lds + 2 * W::kTile;
  auto pages = loader.look_up(k0);      // of the tile that is brought next
  auto load = [&](int32_t k, unsigned char *to) {
    loader.template load<false>(k, pages, to);
    loader.template load<true>(k, pages, to + W::kTile);
    pages = loader.look_up(k + W::TK);
  };
  bare_barrier();                       // nobody reads the piece before any more
  load(k0, cur);
  if (tid == 0) *odd = 0;               // read behind a barrier of the loop: a piece has a tile

  // A wave's number is its SIMD's, and the block's last rows see the most keys: they are turned round from workgroup to workgroup.
  const int32_t block = (wave + turn) % WR * 32, row = block + l32;
  const int32_t first_key = wave / WR * 32 * W::KB;       // this wave's in a tile
  const Row w = row_at(a, u, u.r0 + row);
  u32x4 qf[S::NQ];
  load_query<T, DP>(a, w, half, qf);
  // rows of this wave, and the positions of its first and last
  const int32_t last = min(u.r0 + block + 32, u.rows) - 1;
  const int32_t pos_first = u.ctx + (u.r0 + block) / a.G, pos_last = last >= u.r0 + block ? u.ctx + last / a.G : -1;
  const int32_t lo = a.window > 0 ? w.pos - a.window : -1;

  floatx16 o[S::NO];
#pragma unroll
  for (int n = 0; n < S::NO; ++n) o[n] = floatx16{};
  float ref = -INFINITY, sum = 0.f;
  const int32_t begin = k0;
  auto at_edge = [&](int32_t k) { return k + W::TK > u.min_hi || k < u.max_lo; };
  for (; k0 < end; k0 += W::TK) {
    wait_vm<0>();                       // this wave's part of the tile is in;
    loader.clear_keys(cur);
    bare_barrier();                     // now everyone's is, and nobody reads the tile before any more
    if (k0 + W::TK < end) load(k0 + W::TK, nxt);
    if (at_edge(k0)) {
      if (clear_odd_values<S::kBf16>(cur + W::kTile, W::kTile, tid, kAttendThreads)) *odd = 1;
      bare_barrier();
    }
    const int32_t k = k0 + first_key;
    if (k <= pos_last && k < end) {     // else no row of this wave sees anything of it
      const unsigned char *lk = cur + first_key * S::RB, *lv = lk + W::kTile;
      floatx16 s[W::KB];
      // The waves of a SIMD are then more often at different ends of their tiles, one in products while another forms weights
      // (bf16: 27 000 tokens of prompts 1312 -> 1271 us, prompts by pieces 372 -> 359).
      if constexpr (S::kBf16) __builtin_amdgcn_s_setprio(1);
      scores_in_steps<T, DP, W::KB>(lk, lane, qf, s, a.D);
      if constexpr (S::kBf16) __builtin_amdgcn_s_setprio(0);
      if (k + 32 * W::KB - 1 > pos_first || k < u.max_lo) {
#pragma unroll
        for (int i = 0; i < W::KB; ++i) hide(s[i], k + 32 * i, half, w.pos, lo);
      }
      const float c = follow<S::NO, W::KB>(row_max<W::KB>(s, a.c), ref, sum, o, s, a.c);
      to_weights<W::KB>(s, c, minus_ref(ref), sum);
      if constexpr (S::kBf16) __builtin_amdgcn_s_setprio(1);
      add_values_in_steps<T, DP, W::KB>(lv, lane, s, o, a.D);
      if constexpr (S::kBf16) __builtin_amdgcn_s_setprio(0);
    }
    unsigned char *x = cur;
    cur = nxt;
    nxt = x;
  }
  bare_barrier();
  const int cleared = *odd;
  if constexpr (WK > 1) {
    static_assert(WK == 2 && WR * kRowsFloats<DP> * 4 <= W::kLds, "the rows of the second half of the keys");
    float *room = reinterpret_cast<float *>(lds) + wave % WR * kRowsFloats<DP>;
    bare_barrier();
    if (wave >= WR) give_rows<DP>(room, lane, o, ref, sum);
    bare_barrier();
    if (wave >= WR) return;
    take_rows<DP>(room, lane, o, ref, sum);
  }
  sum = pair_sum(sum);
  const bool again = odd_rows<S::NO>(cleared, o, sum);
  if (part) store_part<DP, W::R>(part, row, half, w.there, o, ref, sum);
  else store_row<T, DP>(a, w, half, o, sum);
  if (__builtin_expect(again, 0)) {
    const bool put = w.there && (part || sum != 0.f);
    put_odd_values<T, DP, PAGES != 0>(a, u, begin, end, lane, put, w.pos, lo, [&](int d, float x) {
      if (part) part->o[row][d] = x;
      else put_out<T>(a, w, d, x);
    });
  }
}

// A cache's rows.  Few of them (WK 2): bound by memory, 32 sequences of 4000 keys with 9 new tokens 526 MB in 103 us, 5.1 TB/s, 2 of
// 120 000 keys 5.7 TB/s, more than a copy reaches because nothing is written; one token of one sequence of 1500 keys is two
// launches and the waits of one tile, 9.5 and 3.5 us.  Prompts by pieces (WK 1): 213 GFLOP in 257 to 278 us with the joining, 770 to
// 830 TFLOP/s; bound as attend_prompt_kernel is, with 60 MB of parts written and read between.
template <typename T, int DP, int WK, int PAGES, bool ONCE>
__global__ __launch_bounds__(kAttendThreads, (Thick<T, DP, WK>::kRuns / 256)) void attend_thick_kernel(AttendArgs a, Join *join,
                                                                                                       Part<DP, Thick<T, DP, WK>::R> *parts) {
  using W = Thick<T, DP, WK>;
  __shared__ __align__(16) unsigned char lds[W::kLds];
  __shared__ int odd;
  work_on_run<DP, W::R, W::TK, W::kLeast, kAttendWaves>(a, lds, join, parts, [&](const Unit &u, int32_t tile, int32_t tiles, Part<DP, W::R> *part) {
    thick_piece<T, DP, WK, PAGES, ONCE>(a, u, tile, tiles, lds, &odd, (int) blockIdx.x / kCUs, part);
  });
}

// Unit `rank` of all requests' row blocks, the ones furthest down their prompt first: they have the most keys, and what is
// begun last should be short.
template <int R>
__device__ __forceinline__ bool find_prompt_unit(const AttendArgs &a, int32_t rank, Unit &u) {
  const int lane = threadIdx.x & (kWave - 1);
  auto blocks_of = [&](int32_t b) -> int32_t {
    int32_t first;
    return b < a.B ? (request_tokens(a, b, first) * a.G + R - 1) / R : 0;
  };
  const int32_t here = blocks_of(lane);
  // units at block `level` (from 1) or further down
  auto at_least = [&](int32_t level) -> int32_t {
    int32_t n = max(0, here - level + 1);
    for (int32_t b = lane + kWave; b < a.B; b += kWave) n += max(0, blocks_of(b) - level + 1);
    return (int32_t) wave_sum((double) n);              // exact, through DPP
  };
  if (rank >= at_least(1)) return false;
  int32_t most = here;
  for (int32_t b = lane + kWave; b < a.B; b += kWave) most = max(most, blocks_of(b));
  // at_least(lo) > rank >= at_least(hi); a maximum in float32 may be rounded, up if need be
  int32_t lo = 1, hi = (int32_t) (wave_max((float) most) * 1.0000002f) + 2;
  while (hi - lo > 1) {
    const int32_t mid = (lo + hi) >> 1;
    if (at_least(mid) > rank) lo = mid;
    else hi = mid;
  }
  int32_t ahead = rank - at_least(lo + 1);
  for (int32_t b0 = 0; b0 < a.B; b0 += kWave) {
    const uint64_t who = __builtin_amdgcn_ballot_w64((b0 ? blocks_of(b0 + lane) : here) >= lo);
    const int32_t n = __popcll(who);
    if (ahead >= n) {
      ahead -= n;
      continue;
    }
    const uint64_t me = __builtin_amdgcn_ballot_w64(((who >> lane) & 1) && __popcll(who & (((uint64_t) 1 << lane) - 1)) == ahead);
    u.b = b0 + __ffsll((long long) me) - 1;
    break;
  }
  u.b = __builtin_amdgcn_readfirstlane(u.b);
  u.rows = request_tokens(a, u.b, u.first) * a.G;
  u.ctx = 0;
  u.r0 = (lo - 1) * R;
  return true;
}

// The same of more than kOrdered requests, in their order.  Places floor(first row / R) + b and on are request b's: as many as it has blocks of
// rows, or one more, so that a bisection finds whose a place is, where find_prompt_unit goes through all requests several times in
// every workgroup.  us there and here, 32 / 8 heads of 128, bf16: 64 prompts of 16 tokens 10.2 and 15.0, 256 40 and 36, 1024 279 and 137,
// 4096 2750 and 540; 512 of 200 tokens 1136 and 653.  fp32, d = 64, mixed lengths: 100 prompts 1847 and 2052, 512 2285 and 2166.
template <int R>
__device__ __forceinline__ bool find_place(const AttendArgs &a, int32_t place, Unit &u) {
  auto begin = [&](int32_t b) -> int32_t { return min(max(fixed_at(a.q_start, b), 0), a.T) * a.G / R + b; };
  int32_t lo = 0;
  for (int32_t n = a.B; n > 1; n -= n >> 1)
    if (begin(lo + (n >> 1)) <= place) lo += n >> 1;
  u.b = lo;
  u.rows = request_tokens(a, u.b, u.first) * a.G;
  u.ctx = 0;
  const int32_t back = place - begin(lo);       // the longest of a request first
  u.r0 = ((u.rows + R - 1) / R - 1 - back) * R;
  return back >= 0 && u.r0 >= 0;
}

// A unit a workgroup, no parts: there are enough of them.  Bound by the SIMDs' issue: products keep the matrix units busy 51 % of
// the time (bf16, d = 128; no LDS conflicts), exponentials, maxima, sums and rounding beside them are 7.4 vector instructions for
// every product.  27 000 tokens of prompts up to 8000, 32 heads: 1.23 PFLOP in 1255 us, 984 TFLOP/s (a library product of
// 8192 x 8192 reaches 1117 here).  Left out of it for a measurement: the exponential 1147, the loads 1095, the weights' product
// 924, the scores' 945 us.  Scores of the next tile beside the weights of this one (1382 us), 256 rows a workgroup by eight waves
// (1275 against 1262) or by four with two blocks of rows (2096) were not faster.  fp32, d = 64, 9 prompts of 1111 tokens: 80 TFLOP/s, 95 us, the
// matrix units busy half of the time too.
template <typename T, int DP, int WK>
__global__ __launch_bounds__(kAttendThreads, (Thick<T, DP, WK>::kRuns / 256)) void attend_prompt_kernel(AttendArgs a) {
  using W = Thick<T, DP, WK>;
  __shared__ __align__(16) unsigned char lds[W::kLds];
  __shared__ int odd;
  Unit u;
  u.b = 0;
  // Workgroups come in rounds of one a CU.  Every second round the other way round: where they all run at a time, the CU that began
  // with the longest unit then gets the shortest of the next round.
  const uint32_t round = blockIdx.x / kCUs, at = blockIdx.x % kCUs;
  const uint32_t rank = round % 2 && gridDim.x <= 4 * kCUs ? round * kCUs + kCUs - 1 - at : blockIdx.x;
  const int32_t place = (int32_t) (rank / (uint32_t) a.heads_kv);
  if (!(a.B > kOrdered ? find_place<W::R>(a, place, u) : find_prompt_unit<W::R>(a, place, u))) return;
  u.head = (int32_t) (rank % (uint32_t) a.heads_kv);
  const int32_t tiles = unit_tiles<W::R, W::TK>(a, u);
  thick_piece<T, DP, WK, 0, false>(a, scalar(u), 0, scalar(tiles), lds, &odd, (int) round, nullptr);
}

// ---- 32 rows of float32 a workgroup ------------------------------------------------------------------------------------

// Two waves of a workgroup where keys and values of four would fill the CU's shared memory: two workgroups then, less to join in each
// (four waves and two, d = 128: 64 sequences of 500 keys with 5 new tokens 88 and 74 us, 4 of 4000 with one 55 and 47, 32 of 4000
// with 8 240 and 244, 1 of 8000 with 8 40 and 43).
template <int DP>
struct Thin {
  static constexpr int NW = DP == 64 ? 4 : 2;
  static constexpr int R = 32, TK = 32 * NW;         // keys a turn of the waves takes
  static constexpr int kTile = 32 * DP * 4;
  static constexpr int kLds = NW * 2 * kTile;
  static_assert(NW / 2 * R * (DP + 2) * 4 <= kLds, "half of the waves' rows on their way to the others");
  static constexpr int kRuns = 2 * kLds <= 160 * 1024 ? 512 : 256;       // two a CU
};

template <int DP, int PAGES>
__device__ __forceinline__ void thin_piece(const AttendArgs &a, const Unit &u, int32_t tile, int32_t tiles, unsigned char *lds,
                                           int *odd, Part<DP, 32> *part) {
  using S = Shape<float, DP>;
  using W = Thin<DP>;
  int tid = threadIdx.x;
  asm("" : "+v"(tid));                  // what follows from it is formed here, not kept in registers from piece to piece
  const int lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, half = lane >> 5;
  const Loader<float, DP, 32, 1, PAGES, true> loader(a, u, lane, 0);
  constexpr int NI = decltype(loader)::NI;
  unsigned char *lk = lds + wave * 2 * W::kTile, *lv = lk + W::kTile;
  int32_t k0 = u.k_lo + tile * W::TK + wave * 32;
  const int32_t end = min(u.k_hi, u.k_lo + (tile + tiles) * W::TK);
  bare_barrier();                       // nobody uses the piece before any more
  const Row w = row_at(a, u, u.r0 + l32);
  const int32_t pos = w.pos;
  auto before = [&] { return a.window > 0 ? pos - a.window : -1; };
  u32x4 qf[S::NQ];
  load_query<float, DP>(a, w, half, qf);
  floatx16 o[S::NO];
#pragma unroll
  for (int n = 0; n < S::NO; ++n) o[n] = floatx16{};
  float ref = -INFINITY, sum = 0.f;
  auto at_edge = [&](int32_t k) { return k + 32 > u.min_hi || k < u.max_lo; };
  auto pages = loader.look_up(k0);      // of the keys that are brought next
  // A turn works on keys k0 - W::TK and brings keys k0 behind it: one place in the code for each load.
  for (bool now = false;; k0 += W::TK, now = true) {
    const bool more = k0 < end;
    if (!now && !more) break;
    const int32_t k = k0 - W::TK;
    floatx16 s[1];
    if (now) {
      wait_vm<NI>();                    // keys are in, values may be on their way
      loader.clear_keys(lk);
      scores<float, DP>(lk, lane, qf, s, a.D);
      wait_lds();
    }
    if (more) loader.template load<false>(k0, pages, lk);
    if (now) {
      const bool edge = at_edge(k);
      if (edge) hide(s[0], k, half, pos, before());
      const float c = follow<S::NO, 1>(row_max<1>(s, a.c), ref, sum, o, s, a.c);
      to_weights<1>(s, c, minus_ref(ref), sum);
      if (more) wait_vm<NI>();
      else wait_vm<0>();
      if (edge) {
        if (clear_odd_values<false>(lv, W::kTile, lane, kWave)) *odd = 1;
        wait_lds();
      }
      add_values<DP>(lv, lane, s[0], o, a.D);
      wait_lds();
    }
    if (!more) break;
    loader.template load<true>(k0, pages, lv);
    pages = loader.look_up(k0 + W::TK);
  }

  // The waves' sums: 2 to 0 and 3 to 1, then 1 to 0.
  float *room = reinterpret_cast<float *>(lds);
  bare_barrier();
#pragma unroll
  for (int n = W::NW / 2; n > 0; n /= 2) {
    if (wave >= n && wave < 2 * n) give_rows<DP>(room + (wave - n) * kRowsFloats<DP>, lane, o, ref, sum);
    bare_barrier();
    if (wave < n) take_rows<DP>(room + wave * kRowsFloats<DP>, lane, o, ref, sum);
    if (n > 1) bare_barrier();
  }
  if (wave > 0) return;
  sum = pair_sum(sum);
  int32_t r = l32;
  asm("" : "+v"(r));                    // formed here, not kept in registers since the beginning
  const Row out = row_at(a, u, u.r0 + r);
  const bool again = odd_rows<S::NO>(*odd, o, sum);
  *odd = 0;                             // for the next piece, which begins with a barrier
  if (part) store_part<DP, 32>(part, r, half, out.there, o, ref, sum);
  else store_row<float, DP>(a, out, half, o, sum);
  if (__builtin_expect(again, 0)) {
    const bool put = out.there && (part || sum != 0.f);
    put_odd_values<float, DP, PAGES != 0>(a, u, u.k_lo + tile * W::TK, end, lane, put, out.pos, a.window > 0 ? out.pos - a.window : -1,
                                          [&](int d, float x) {
      if (part) part->o[r][d] = x;
      else put_out<float>(a, out, d, x);
    });
  }
}

// 32 rows of float32 over a cache.  A product of 32 x 32 x 2 keeps a SIMD 64 cycles whether 32 rows are there or 4, so that the
// waves of a CU have to share the keys, 32 each, with the loads of a wave's next keys ahead of its products with these: 32
// sequences of 4000 keys, 8 new tokens of 4 heads a shared head, d = 128: 1053 MB in 231 to 245 us, 4.3 to 4.6 TB/s; 32 rows shared
// by two waves 391 us, by one 577.  A short window (12 sequences, 1000 keys, d = 80, 39 MB) takes 36 us: a run has a tile or two, whose
// waits (for the run's first unit, its pages, its keys, the other waves' sums) nothing fills.
template <int DP, int PAGES>
__global__ __launch_bounds__(Thin<DP>::NW * kWave, (Thin<DP>::kRuns * Thin<DP>::NW / 1024)) void attend_thin_kernel(AttendArgs a, Join *join,
                                                                                          Part<DP, 32> *parts) {
  __shared__ __align__(16) unsigned char lds[Thin<DP>::kLds];
  __shared__ int odd;
  if (threadIdx.x == 0) odd = 0;        // pieces come behind barriers
  work_on_run<DP, 32, Thin<DP>::TK, kThinLeast, Thin<DP>::NW>(a, lds, join, parts, [&](const Unit &u, int32_t tile, int32_t tiles, Part<DP, 32> *part) {
    thin_piece<DP, PAGES>(a, u, tile, tiles, lds, &odd, part);
  });
}

// ---- units in parts ----------------------------------------------------------------------------------------------------------

// Workgroups (i, y) join the parts of the unit that run i began and did not finish: outputs, references and sums of the parts are
// brought to the largest reference, added and divided.  A wave a row, every second part to each half of it.  Bound by trips to
// memory, a microsecond each: references, sums and first outputs are asked for together, 16 parts at a time, no more than there are.
// 64 sequences (two or three parts a unit) 8 us, prompts by pieces (60 MB of parts) 20 us, 2 x 120 000 tokens (33 parts) 8 us.  A
// kernel of its own because the next launch's start is the one meeting of all workgroups that a graph can hold.
template <typename T, int DP, int R>
__global__ __launch_bounds__(kJoinThreads) void attend_join_kernel(AttendArgs a, const Join *join, const Part<DP, R> *parts) {
  const Join j = join[blockIdx.x];
  if (j.parts < 2) return;
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l32 = lane & 31, half = lane >> 5;
  Unit u;
  u.head = j.head;
  u.rows = j.rows;
  u.first = j.first;
  u.ctx = 0;
  const Part<DP, R> *first = parts + 2 * (int64_t) blockIdx.x;
  auto part_at = [&](int32_t p) -> const Part<DP, R> & { return first[p ? 2 * p : 1]; };
  constexpr int kEach = DP / 32, kAtOnce = 8;
  typedef float vec __attribute__((ext_vector_type(kEach)));
  const int32_t rows = min(R, u.rows - j.r0);
  for (int row = blockIdx.y * (kJoinThreads / kWave) + wave; row < rows; row += gridDim.y * (kJoinThreads / kWave)) {
    const Row w = row_at(a, u, j.r0 + row);
    vec o = {};
    float sum = 0.f, top = -INFINITY;
    vec x[kAtOnce];
    // One, four or all eight (one by one: prompts by pieces 1 % faster, a single token's parts 2 % slower; always eight:
    // 5 % slower and the same).
    auto from = [](int32_t k) { return k < 1 ? 0 : k < 4 ? 2 : 8; };
    auto ask = [&](int32_t p0, int32_t i, int32_t n) {
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k)
        if (i + from(k) < n) x[k] = *reinterpret_cast<const vec *>(&part_at(p0 + min(i + 2 * k + half, n - 1)).o[row][l32 * kEach]);
    };
    for (int32_t p0 = 0; p0 < j.parts; p0 += kWave) {
      // references and sums of 64 parts, one a lane, and the first outputs beside them
      const int32_t n = min(j.parts - p0, kWave);
      const Part<DP, R> &mine = part_at(p0 + min(lane, n - 1));
      const float mine_ref = mine.ref[row], mine_sum = mine.sum[row];
      ask(p0, 0, n);
      const float ref = lane < n ? mine_ref : -INFINITY;
      const float now = fmaxf(top, wave_max(ref));
      const float before = now == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - now);
      const float f = now == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref - now);
      top = now;
      sum = sum * before + (lane < n ? f * mine_sum : 0.f);
      o *= before;
      for (int32_t i = 0; i < n; i += 2 * kAtOnce) {
        if (i) ask(p0, i, n);
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
          if (i + from(k) >= n) break;
          const int32_t p = i + 2 * k + half;
          const float fp = __shfl(f, min(p, n - 1));
#pragma unroll
          for (int e = 0; e < kEach; ++e) o[e] = p < n ? fmaf(fp, x[k][e], o[e]) : o[e];
        }
      }
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    const float inv = 1.f / sum;
    T *out = reinterpret_cast<T *>(a.out) + w.token * a.o_tok + w.head * a.o_head;
#pragma unroll
    for (int e = 0; e < kEach; ++e) o[e] = pair_sum(o[e]);
    float odd = 0.f;                    // NaN if an element is not finite
#pragma unroll
    for (int e = 0; e < kEach; ++e) odd = fmaf(o[e], 0.f, odd);
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(odd != 0.f) != 0, 0)) {
      // what is not finite in a part is so in the sum, also where its factor is zero, see put_odd_values
      vec all = {};
#pragma nounroll
      for (int32_t p = 0; p < j.parts; ++p) {
        const vec y = *reinterpret_cast<const vec *>(&part_at(p).o[row][l32 * kEach]);
#pragma unroll
        for (int e = 0; e < kEach; ++e)
          if (!(fabsf(y[e]) < INFINITY)) all[e] += y[e];
      }
#pragma unroll
      for (int e = 0; e < kEach; ++e)
        if (all[e] != 0.f) o[e] = all[e];
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) o[e] = sum == 0.f ? 0.f : o[e] * inv;        // see store_row
    const int d = l32 * kEach;
    if (half || d >= a.D) continue;
    if constexpr (sizeof(T) == 2) {
      uint32_t two[kEach / 2];
#pragma unroll
      for (int e = 0; e < kEach / 2; ++e)
        two[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2{o[2 * e], o[2 * e + 1]}), bf16x2));
#pragma unroll
      for (int e = 0; e < kEach / 2; ++e) reinterpret_cast<uint32_t *>(out + d)[e] = two[e];
    } else {
#pragma unroll
      for (int e = 0; e < kEach; ++e) out[d + e] = o[e];
    }
  }
}

// ---- launches ----------------------------------------------------------------------------------------------------------------

constexpr size_t join_bytes(int32_t runs) { return ((size_t) runs * sizeof(Join) + 255) / 256 * 256; }

template <typename T, int DP, int R>
size_t parts_bytes(int32_t runs) { return join_bytes(runs) + 2 * (size_t) runs * sizeof(Part<DP, R>); }

template <typename T, int DP, int R, typename Kernel>
hipError_t split_launch(Kernel kernel, int32_t runs, int threads, const AttendArgs &a, void *workspace, hipStream_t stream) {
  Join *join = reinterpret_cast<Join *>(workspace);
  Part<DP, R> *parts = reinterpret_cast<Part<DP, R> *>(reinterpret_cast<char *>(workspace) + join_bytes(runs));
  kernel<<<runs, threads, 0, stream>>>(a, join, parts);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  attend_join_kernel<T, DP, R><<<dim3(runs, R == 128 ? 8 : R / 4), kJoinThreads, 0, stream>>>(a, join, parts);
  return hipGetLastError();
}

template <int DP>
hipError_t go_thin(const AttendArgs &a, bool shared_pages, void *workspace, hipStream_t stream) {
  if (shared_pages) return split_launch<float, DP, 32>(attend_thin_kernel<DP, 1>, Thin<DP>::kRuns, Thin<DP>::NW * kWave, a, workspace, stream);
  return split_launch<float, DP, 32>(attend_thin_kernel<DP, 2>, Thin<DP>::kRuns, Thin<DP>::NW * kWave, a, workspace, stream);
}

template <typename T, int DP, int WK, bool ONCE>
hipError_t go_thick(const AttendArgs &a, bool shared_pages, void *workspace, hipStream_t stream) {
  using W = Thick<T, DP, WK>;
  if (shared_pages) return split_launch<T, DP, W::R>(attend_thick_kernel<T, DP, WK, 1, ONCE>, W::kRuns, kAttendThreads, a, workspace, stream);
  return split_launch<T, DP, W::R>(attend_thick_kernel<T, DP, WK, 2, ONCE>, W::kRuns, kAttendThreads, a, workspace, stream);
}

template <typename T, int DP>
hipError_t go_cache(const AttendArgs &a, int64_t longest, void *workspace, hipStream_t stream) {
  // 16 keys share a page, and lie within 32 bits of each other.  us with pages looked up for 16 keys and for each lane, bf16: 32
  // sequences of 4000 keys with 9 new tokens 121 and 133, 8 of 2000 35.2 and 37.1; fp32: 369 and 459, 76 and 91.
  const bool shared_pages = a.page_size % 16 == 0 && a.k_tok * 16 * (int64_t) sizeof(T) < (int64_t) 1 << 31;
  const int64_t rows = longest * a.G;
  // The keys are read as often as a request has blocks of rows: once, if they fit one.  In bf16 two waves on the keys of 64 rows
  // hide more of memory's delay than four on 128, most of which are not there, and than four with streams of their own; in fp32
  // the products bound, and a wave whose rows are not there does none.  us with 32, 64 and 128 rows a workgroup, d = 128:
  //   bf16, 4 rows:   1 sequence of 1000 keys 15 14 19;  8 of 2000 26 24 24;  32 of 4000 103 94 96
  //   bf16, 36 rows:  8 of 2000 37 29 29;  32 of 4000 141 103 107
  //   bf16, 68 rows:  8 of 2000 47 46 32;  32 of 4000 304 149 128
  //   fp32, 20 rows:  8 of 2000 54 67 88;  32 rows, 32 of 4000: 231 391 577
  //   fp32, 36 rows:  8 of 2000 81 69 93;  32 of 4000 452 393 579
  //   fp32, 68 rows:  8 of 2000 109 122 98;  32 of 4000 678 733 588
  if constexpr (sizeof(T) == 4) {
    if (rows <= 32) return go_thin<DP>(a, shared_pages, workspace, stream);
  }
  if (rows <= 64) return go_thick<T, DP, 2, true>(a, shared_pages, workspace, stream);
  // in fp32 the hint changes nothing here (586 and 588 us)
  if (sizeof(T) == 2 && rows <= kThickRows) return go_thick<T, DP, 1, sizeof(T) == 2>(a, shared_pages, workspace, stream);
  return go_thick<T, DP, 1, false>(a, shared_pages, workspace, stream);
}

template <typename T, int DP>
size_t cache_bytes(int64_t rows) {
  if (sizeof(T) == 4 && rows <= 32) return parts_bytes<T, DP, 32>(Thin<DP>::kRuns);
  if (rows <= 64) return parts_bytes<T, DP, 64>(Thick<T, DP, 2>::kRuns);
  return parts_bytes<T, DP, kThickRows>(Thick<T, DP, 1>::kRuns);
}

}  // namespace

size_t attend_workspace_bytes(int32_t G, int32_t D, int64_t longest) {
  const int64_t rows = longest * G;
  if (D <= 64) return max(cache_bytes<uint16_t, 64>(rows), cache_bytes<float, 64>(rows));
  return max(cache_bytes<uint16_t, 128>(rows), cache_bytes<float, 128>(rows));
}

hipError_t launch_cache_attend(const AttendArgs &a, bool bf16, int64_t longest, void *workspace, hipStream_t stream) {
  if (bf16) return a.D <= 64 ? go_cache<uint16_t, 64>(a, longest, workspace, stream) : go_cache<uint16_t, 128>(a, longest, workspace, stream);
  return a.D <= 64 ? go_cache<float, 64>(a, longest, workspace, stream) : go_cache<float, 128>(a, longest, workspace, stream);
}

namespace {
template <typename T, int DP, int WK>
hipError_t go_prompt(const AttendArgs &a, hipStream_t stream) {
  const int64_t units = ((int64_t) a.T * a.G / Thick<T, DP, WK>::R + a.B) * a.heads_kv;
  attend_prompt_kernel<T, DP, WK><<<(uint32_t) ((units + kCUs - 1) / kCUs * kCUs), kAttendThreads, 0, stream>>>(a);
  return hipGetLastError();
}

template <typename T, int DP>
hipError_t go_prompts(const AttendArgs &a, int64_t longest, hipStream_t stream) {
  // Keys that a workgroup place of the chip works through if all units fill it evenly, against those of the longest unit, which
  // nothing can overtake.  Two waves on the keys of the same rows halve the way, but every unit has its joining and half the rows for
  // the keys that it brings.  us with one wave and with two, at longest / even:
  //   bf16, d = 64:   0.57 64 and 82;  1.9 27 and 32;  2.1 40 and 35;  3.7 19 and 17;  8 14.5 and 13.3
  //   bf16, d = 128:  0.57 113 and 169;  2.1 57 and 66;  3.8 21 and 25;  7.6 15.4 and 13.6;  16 29 and 23
  //   fp32, d = 64:   0.57 297 and 369;  1.9 117 and 114;  2.8 124 and 98;  8 49 and 30
  //   fp32, d = 128:  0.57 601 and 914;  2.1 309 and 407;  3.7 123 and 124;  7.6 55 and 46;  16 158 and 93
  const double units = (double) a.T * a.G / kThickRows * a.heads_kv, even = units * (0.5 * a.T / a.B) / 512;
  if (longest > (DP == 64 ? 2 : 5) * even) return go_prompt<T, DP, 2>(a, stream);
  return go_prompt<T, DP, 1>(a, stream);
}
}  // namespace

hipError_t launch_prompt_attend(const AttendArgs &a, bool bf16, int64_t longest, hipStream_t stream) {
  if (bf16) return a.D <= 64 ? go_prompts<uint16_t, 64>(a, longest, stream) : go_prompts<uint16_t, 128>(a, longest, stream);
  return a.D <= 64 ? go_prompts<float, 64>(a, longest, stream) : go_prompts<float, 128>(a, longest, stream);
}

}  // namespace pcg
