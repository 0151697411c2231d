// What the attention kernels share (gfx950, wave64): requests and their units of work, runs of equal length over the whole chip and the
// parts that they leave, softmax references, rows on their way between waves and into memory.
#pragma once

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
constexpr int kCost = 1;
constexpr int kJoinThreads = 256;
constexpr float kLag = 8.f;        // how far (in powers of two) a maximum may run ahead of the one in use
constexpr float kFar = 16777216.f; // where half a step of a reference is a factor of two

// What is read where there is nothing to read: keys behind the last, columns behind D.
__device__ const u32x4 kZeros = {0, 0, 0, 0};

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

// Which shared heads a workgroup's runs are of (first, first + step, ..: `heads` of them, numbered from 0 in units), and how many workgroups
// there are for those, of which it is number `block`.
struct Heads {
  int32_t first, step, heads;
  uint32_t block;
  int32_t count;
};
// All workgroups are for all heads.
__device__ __forceinline__ Heads all_heads(const AttendArgs &a) {
  return Heads{0, 1, a.heads_kv, blockIdx.x, (int32_t) gridDim.x};
}

// All units (requests, their shared heads, their row blocks, in this order) in a row, COST for what a unit costs beside its tiles
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

// Finds this workgroup's run, of deal.count at most, LEAST long at least (but for the last): its first unit and how far into it.
// Every workgroup adds the requests up by itself, each wave its share of them, a request a lane or (with many row blocks) a row block
// a lane: for 64 requests that takes two microseconds, less than a launch ahead would.  Lengths are whole numbers below 2^53 in
// double, whose running sums go through DPP.
template <int R, int TK, int LEAST, int NW, int COST>
__device__ __forceinline__ Run find_run(const AttendArgs &a, const Heads &deal, unsigned char *lds, Unit &u, int64_t &into) {
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
    one = v.rows > 0 && v.rows <= R ? unit_tiles<R, TK>(a, v) + COST : 0;
    for (uint64_t many = __builtin_amdgcn_ballot_w64(v.rows > R); many; many &= many - 1) {
      const int l = __ffsll((long long) many) - 1;
      Unit x;
      x.rows = read_lane(v.rows, l);
      x.ctx = read_lane(v.ctx, l);
      double all = 0;
      for (int64_t r0 = (int64_t) lane * R; r0 < x.rows; r0 += kWave * R) {
        x.r0 = (int32_t) r0;
        all += unit_tiles<R, TK>(a, x) + COST;
      }
      all = wave_sum(all);
      if (lane == l) one = all;
    }
    return wave_scan(one * deal.heads);
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
  run.runs = (int32_t) min((int64_t) deal.count, (total + LEAST - 1) / LEAST);
  // An XCD (every eighth workgroup) takes runs that follow each other: those of a shared head find its keys in its L2.
  const int32_t eighth = (run.runs + 7) / 8;
  run.index = (int32_t) deal.block / 8 < eighth ? (int32_t) (deal.block % 8) * eighth + (int32_t) deal.block / 8 : run.runs;
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
      ahead -= read_lane(upto, l) - length * deal.heads;
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
        const double t = mine_r0 < x.rows ? unit_tiles<R, TK>(a, x) + COST : 0, blocks = wave_scan(t);
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
__device__ __forceinline__ void next_unit(const AttendArgs &a, int32_t heads, Unit &u) {
  u.r0 += R;
  if (u.r0 < u.rows) return;
  u.r0 = 0;
  if (++u.head < heads) return;
  u.head = 0;
  do {
    if (++u.b >= a.B) return;
    u.rows = request_tokens(a, u.b, u.first) * a.G;
  } while (u.rows == 0);
  u.ctx = request_ctx(a, u.b);
}

// Calls work(unit, first tile, tiles, part) for every unit or piece of one in this workgroup's run; part: NULL where the unit is
// whole.  A workgroup has two places for parts: 1 for the unit that it begins and does not finish, 0 for one that another began.
template <int DP, int R, int TK, int LEAST, int NW, int COST = kCost, typename Work>
__device__ __forceinline__ void work_on_run(const AttendArgs &a, const Heads &deal, unsigned char *lds, Join *join, Part<DP, R> *parts, Work work) {
  Unit u;
  int64_t into = 0;
  Run run = find_run<R, TK, LEAST, NW, COST>(a, deal, lds, u, into);
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
      const int64_t until = min((int64_t) all + COST, into + run.left);       // in the unit's length
      tile = into > COST ? (int32_t) into - COST : 0;
      tiles = until > COST ? (int32_t) until - COST - tile : 0;
      run.left -= until - into;
      part = tiles == all ? nullptr : parts + 2 * (int64_t) run.index + (tile == 0);
      if (part && tile == 0 && tiles > 0) {
        // this run and those that begin ahead of the unit's end
        j.parts = run.ahead_of(run.begin(run.index + 1) - run.left + all + COST - until) - run.index;
        j.head = deal.first + u.head * deal.step;
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
    if (run.left > 0) next_unit<R>(a, deal.heads, u);
  }
  if (threadIdx.x != 0) return;
  if (run.index < run.runs) join[run.index] = j;
  if ((int32_t) deal.block >= run.runs) join[deal.block] = Join{0, 0, 0, 0, 0};
}

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

// ---- units in parts ---------------------------------------------------------------------------------------------------------

// See attend_join_kernel.
template <typename T, int DP, int R>
__device__ __forceinline__ void join_parts(const AttendArgs &a, const Join *join, const Part<DP, R> *parts) {
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

constexpr size_t join_bytes(int32_t runs) { return ((size_t) runs * sizeof(Join) + 255) / 256 * 256; }

template <typename T, int DP, int R>
size_t parts_bytes(int32_t runs) { return join_bytes(runs) + 2 * (size_t) runs * sizeof(Part<DP, R>); }

}  // namespace

}  // namespace pcg
