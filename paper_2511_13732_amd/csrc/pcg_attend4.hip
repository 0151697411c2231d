// Attention of new tokens over a paged cache of 4-bit codes (gfx950, wave64).
//
// An element is scale * code, code one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives, one scale a token and shared head for its key
// and one for its value.  Codes are exact in bfloat16, so that the products of pcg_attend.hip are made of them as they stand,
//   S^T = C_k Q^T,  score = c s_k S        O^T = C_v^T (s_v P)^T
// and the scales meet scores and weights, one multiplication each, and never the elements.  float32 queries and weights are three
// bfloat16 numbers each, which hold all of their 24 bits (from 2^-110 on; the smallest bfloat16 is 2^-133): three products of the fast kind, exact
// in every term, where one of float32 takes sixteen times as long.
//
// The four waves of a workgroup have the same rows, one to three blocks of 16 that share decoded keys and values, and a stream of keys each, which
// a wave brings into its own part of LDS ahead of their use: nothing is shared in the loop, and no wave waits for another one in it.  The
// streams are joined at a piece's end.  Rows, units, runs and parts are those of pcg_attend.hip.
//
// What bounds it (bf16, 32 / 8 heads of 128; first kernel, then the joining of parts).  One block: memory, 128 requests of 3800 keys on average
// 112 to 117 + 5 us for 509 MB, 4.5 TB/s.  Three blocks: issue.  A stage of 64 keys is 96 products, 48 exponentials, 128 conversions of codes and
// about 300 other vector instructions, whose times one after the other are 1.55 us at 2.35 GHz, 2.2 at the 1.6 to 1.75 that the chip holds with all
// CUs busy; a SIMD's two waves take 4 a stage, so that not much of it overlaps.  (Some does: float32 with two blocks, three times the products and
// the cutting of their operands, takes 180 us where bfloat16 takes 108.  How much could was not measured.)  64 requests of 1260 keys with 9 tokens
// 43 to 44 + 6.7 us, 2 requests of 115000 69 + 9 (in a row 71 to 77 from one card to another), pieces of prompts, 2844 tokens, 317 to 326 + 10 one
// at a time and 289 to 298 in a row (715 to 735 TFLOP/s).  Windows of 1000 keys, bfloat16: 64 requests of 9 tokens 42, 128 of one token behind up
// to 6000 keys 40.5 for 137 MB, pieces of prompts 109.  Few keys: waits one after the other, the run, the pages, the first keys, the joining: 1 request of 1500 keys 8.1 + 3.4.
#include <algorithm>
#include <type_traits>

#include "pcg_attend_device.h"

namespace pcg {

namespace {

// 4 bytes a lane from memory to 256 bytes of LDS in a row; see bring.
__device__ __forceinline__ void bring_word(const char *from, const unsigned char *to) {
  asm volatile("s_nop 4\n\tglobal_load_lds_dword %0, off" :: "v"(from), "{m0}"(lds_address(to)) : "memory");
}
// Four of 16 bytes a lane to 4 KB in a row, load i from base[i] + offset[i] - kBias + 1024 i: what an instruction's own offset adds to the
// place in LDS it adds to the address as well.
constexpr uint32_t kBias = 3 * 1024;
__device__ __forceinline__ void bring_four(const char *const (&base)[4], const uint32_t (&offset)[4], const unsigned char *to) {
  asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, %4\n\tglobal_load_lds_dwordx4 %1, %5 offset:0x400"
               "\n\tglobal_load_lds_dwordx4 %2, %6 offset:0x800\n\tglobal_load_lds_dwordx4 %3, %7 offset:0xc00"
               :: "v"(offset[0]), "v"(offset[1]), "v"(offset[2]), "v"(offset[3]), "s"(base[0]), "s"(base[1]), "s"(base[2]), "s"(base[3]),
               "{m0}"(lds_address(to)) : "memory");
}

// The kernel's first argument as it lies in memory: what is read of it behind such a call is read there and not kept in scalar registers
// since the beginning, which the loop over stages has too few of (pieces of prompts 302 us with arguments kept, 295 with those of a piece's beginning
// and end read there, 290 with those of the loop apart as well).
__device__ __forceinline__ const Attend4Args &arguments() {
  typedef const Attend4Args __attribute__((address_space(4))) Args;
  Args *p = (Args *) __builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const Attend4Args *) p;
}

// A number on its own, not as the part of a group that it was loaded with.
template <typename X>
__device__ __forceinline__ X apart(X x) {
  asm("" : "+s"(x));
  return x;
}

template <int DP>
struct Codes {
  static constexpr int RB = DP / 2;                 // bytes of a key
  static constexpr int CH = RB / 16;
  static constexpr int RPI = kWave / CH;            // keys that one load of a wave brings
  static constexpr int KEYS = 64;                   // of a stage
  static constexpr int NI = KEYS / RPI;             // loads of their codes
  static constexpr int NG = KEYS / 16;              // groups of 16 keys
  static constexpr int kBytes = KEYS * RB;
  static constexpr int kStage = 2 * kBytes + 256;   // codes of keys, of values, scales
  static constexpr int kRest = 8 * KEYS + 256;      // the scales in use as float32, pages of stages to come
  static constexpr int NQ = DP / 32, NM = DP / 16;  // steps of the scores, blocks of 16 columns
};

// Which 16-byte chunk of key `row` lies at chunk position `pos` of its row in LDS, and the other way round: the keys that one read touches
// (four in a row of each 16 as scores, 16 in a row as values) should differ modulo 256 bytes.
template <int RB>
__device__ __forceinline__ int code_swap(int row, int pos) {
  if constexpr (RB == 64) return pos ^ (((row >> 2) ^ (row >> 4)) & 3);
  else return pos ^ (((row >> 3) ^ (row >> 4)) & 1);
}

__device__ __forceinline__ int64_t lane_value(int64_t x, int lane) {
  return (int64_t) ((uint64_t) (uint32_t) __shfl((int) (x >> 32), lane) << 32 | (uint32_t) __shfl((int) x, lane));
}

// Brings the keys, values and scales of a wave's stages into LDS, stages `step` keys from each other.  Where they lie is worked out for many
// stages at once: for 64 groups of 16 keys, one a lane, where such groups share a page (PAGES 1: pages of a multiple of 16 slots); for a stage's
// keys, one a lane, where they do not (PAGES 2).  The pages for the next time are brought into LDS too, like codes.  Chunks behind D are the
// row's first ones: queries are zero there, and the columns that values make there are not stored.
template <int DP, int PAGES>
struct Loader4 {
  using C = Codes<DP>;
  static constexpr int kEach = PAGES == 1 ? kWave / C::NG : 1;      // stages that are worked out at once
  const Attend4Args &a;
  const Unit &u;
  const int lane;
  const int32_t begin, step;
  unsigned char *const ids;
  const int32_t *table;
  const char *kb, *vb, *sb;
  uint32_t off[C::NI];        // of this lane from the first key of a group, see bring_four
  int64_t codes, scales;      // where this lane's group or key lies
  uint64_t there;             // lanes whose group or key there is
  int64_t next;               // scales of this lane's key of the next stage
  const uint32_t scale_off;   // from the first key of a group to this lane's

  __device__ __forceinline__ int row_of(int i) const { return i * C::RPI + lane / C::CH; }
  __device__ __forceinline__ int chunk(int row) const {
    const int ch = code_swap<C::RB>(row, lane % C::CH);
    return ch * 32 < a.D ? ch * 16 : 0;
  }
  __device__ __forceinline__ Loader4(const Attend4Args &a_, const Unit &u_, int lane_, int32_t begin_, int32_t step_, unsigned char *ids_)
      : a(a_), u(u_), lane(lane_), begin(begin_), step(step_), ids(ids_), table(a_.table + (int64_t) u_.b * a_.table_stride),
        scale_off((uint32_t) (lane_ & 15) * (uint32_t) a_.s_tok * 4) {
    kb = reinterpret_cast<const char *>(a.k) + (int64_t) u.head * a.k_head;
    vb = reinterpret_cast<const char *>(a.v) + (int64_t) u.head * a.k_head;
    sb = reinterpret_cast<const char *>(a.scales + (int64_t) u.head * a.s_head);
#pragma unroll
    for (int i = 0; i < C::NI; ++i)
      off[i] = (PAGES == 1 ? (uint32_t) (row_of(i) & 15) * (uint32_t) a.k_tok : 0) + (uint32_t) chunk(row_of(i)) + (kBias - i * 1024);
    place(0, table[block_of(key_of(0, lane))], lane);
  }

  // The key whose place lane `lane` works out with stages n and on.
  __device__ __forceinline__ int32_t key_of(int32_t n, int lane) const {
    // far behind the last key it may wrap, and is then past the table
    if constexpr (PAGES == 1) return (int32_t) ((uint32_t) begin + (uint32_t) (n + lane / C::NG) * (uint32_t) step + lane % C::NG * 16);
    else return (int32_t) ((uint32_t) begin + (uint32_t) n * (uint32_t) step + lane % C::KEYS);
  }
  __device__ __forceinline__ uint32_t block_of(int32_t key) const {
    uint32_t block, slot;
    split_by((uint32_t) key, (uint32_t) a.page_size, a.magic_page, block, slot);
    return min(block, (uint32_t) a.max_blocks - 1);
  }
  __device__ __forceinline__ void place(int32_t n, int32_t page, int lane) {
    const int32_t key = key_of(n, lane);
    uint32_t block, slot;
    split_by((uint32_t) key, (uint32_t) a.page_size, a.magic_page, block, slot);
    there = __builtin_amdgcn_ballot_w64(key < u.k_hi && block < (uint32_t) a.max_blocks && (uint32_t) page < (uint32_t) a.num_pages);
    codes = (int64_t) page * a.k_page + (int64_t) slot * a.k_tok;
    scales = ((int64_t) page * a.s_page + (int64_t) slot * a.s_tok) * 4;
    if constexpr (PAGES == 1) find_scales(0, lane);
    else next = scales;
  }
  __device__ __forceinline__ void ask(int32_t n, int lane) const {
    bring_word(reinterpret_cast<const char *>(table + block_of(key_of(n, lane))), ids);
  }

  // Those of the key lane of the stage whose groups begin with g0.
  __device__ __forceinline__ void find_scales(int g0, int lane) {
    next = lane_value(scales, g0 + lane / 16) + scale_off;
  }

  // Codes and scales of the keys of stage n (stages come in order), or afterwards the codes of its values.
  template <bool VALUES>
  __device__ __forceinline__ void load(int32_t n, unsigned char *to) {
    int lane = this->lane;
    asm("" : "+v"(lane));               // what follows from it is formed here, not kept in registers
    if (!VALUES && n > 0 && n % kEach == 0) {
      // asked for ahead of the keys of a stage before, which have been waited for
      place(n, reinterpret_cast<const int32_t *>(ids)[lane], lane);
      wait_lds();
      ask(n + kEach, lane);
    }
    const char *const base = (VALUES ? vb : kb) - kBias;
    unsigned char *const codes_to = VALUES ? to + C::kBytes : to, *const scales_to = to + 2 * C::kBytes;
    const char *const zeros = reinterpret_cast<const char *>(&kZeros);
    const int32_t k0 = begin + n * step;
    const int g0 = PAGES == 1 ? n % kEach * C::NG : 0;
    // of the group of key `row`, or of the key
    auto lane_of = [&](int row) { return PAGES == 1 ? g0 + row / 16 : row; };
    auto has = [&](int row) { return (there >> lane_of(row) & 1) && k0 + row < u.k_hi; };
    if (PAGES == 1 && k0 + C::KEYS <= u.k_hi && (~there >> g0 & ((1 << C::NG) - 1)) == 0) {
      if constexpr (C::NI == 4) {
        const char *from[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          from[i] = base + (int64_t) ((uint64_t) (uint32_t) read_lane((int32_t) (codes >> 32), g0 + i) << 32 | (uint32_t) read_lane((int32_t) codes, g0 + i));
        bring_four(from, off, codes_to);
      } else {
#pragma unroll
        for (int i = 0; i < C::NI; ++i) bring(base + lane_value(codes, g0 + 2 * i + lane / 32) + off[i] + i * 1024, codes_to + i * 1024);
      }
      if constexpr (!VALUES) bring_word(sb + next, scales_to);
    } else {
      // a unit's last keys, pages outside the cache, pages of any size: zeros where there is no key
#pragma unroll
      for (int i = 0; i < C::NI; ++i) {
        const int row = i * C::RPI + lane / C::CH;
        const int64_t at = lane_value(codes, lane_of(row));
        uint32_t from = off[i];
        asm("" : "+v"(from));
        bring(has(row) ? base + at + from + i * 1024 : zeros, codes_to + i * 1024);
      }
      if constexpr (!VALUES) bring_word(has(lane) ? sb + next : zeros, scales_to);
    }
    if constexpr (VALUES && PAGES == 1) find_scales(min(g0 + C::NG, kWave - C::NG), lane);
  }
};

// Eight codes as bfloat16.
__device__ __forceinline__ bf16x8 decoded(uint32_t w) {
  u32x4 x;
  x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 0));
  x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 1));
  x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 2));
  x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 3));
  return __builtin_bit_cast(bf16x8, x);
}

// x and y as the upper halves of one word, and what is left of them: three times takes all of a float32's 24 bits, 8 a time, cut off.  What
// is cut off an infinity is NaN unless `rest` asks for zero.
template <bool INF>
__device__ __forceinline__ uint32_t cut_two(float &x, float &y) {
  const uint32_t xb = __float_as_uint(x), yb = __float_as_uint(y);
  const float xt = __uint_as_float(xb & 0xffff0000u), yt = __uint_as_float(yb & 0xffff0000u);
  x = INF && fabsf(x) == INFINITY ? 0.f : x - xt;
  y = INF && fabsf(y) == INFINITY ? 0.f : y - yt;
  return __builtin_amdgcn_perm(yb, xb, 0x07060302);
}

// Eight numbers as NP operands of the products: rounded to bfloat16 (half a step, at most 2^-8 of each, as in pcg_attend.hip), or whole.
template <int NP, bool INF>
__device__ __forceinline__ void operands(const float (&x)[8], bf16x8 (&p)[NP]) {
  u32x4 w[NP];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float lo = x[2 * e], hi = x[2 * e + 1];
    if constexpr (NP == 1) {
      w[0][e] = __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2{lo, hi}), bf16x2));
    } else {
#pragma unroll
      for (int i = 0; i < NP; ++i) w[i][e] = cut_two<INF>(lo, hi);
    }
  }
#pragma unroll
  for (int i = 0; i < NP; ++i) p[i] = __builtin_bit_cast(bf16x8, w[i]);
}

__device__ __forceinline__ floatx4 product(bf16x8 x, bf16x8 y, floatx4 s) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, s, 0, 0, 0);
}

// max and sum of the lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float quad_max(float x) {
  const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return pair_max(fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1])));
}
__device__ __forceinline__ float quad_sum(float x) {
  const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return pair_sum(__uint_as_float(p[0]) + __uint_as_float(p[1]));
}

// NB blocks of 16 rows; every wave has all of them and a stream of keys.
template <typename T, int DP, int NB>
struct Work4 {
  static constexpr int NP = sizeof(T) == 2 ? 1 : 3; // bfloat16 numbers that make one of T
  static constexpr int R = 16 * NB, TK = Codes<DP>::KEYS * kAttendWaves;
  static constexpr int kWaveLds = Codes<DP>::kStage + Codes<DP>::kRest;
  static constexpr int kQueries = NB * Codes<DP>::NQ * NP * 1024;
  // passes of the streams' joining, what its outputs take, and with the references and sums
  static constexpr int kPasses = NB * DP > 192 ? 2 : 1, kRows = kAttendWaves * NB * DP / 16 / kPasses * 1024;
  static constexpr int kLds = std::max(kAttendWaves * kWaveLds + kQueries, kRows + kAttendWaves * R * 8);
  // Workgroups a CU.  Above one block of rows as many as find registers.  With one more runs mean more parts and more beginnings, fewer mean
  // less on its way from memory, and LDS has room for three of float32 and 128 elements.  us with 2, 3, 4, 5, at 128 requests of 4000 keys, 8
  // shared heads, 4 rows: bf16 of 64 elements 63, 64, 63, 67, of 128 106, 115, 107, 107 (32 requests 33, 36, 37, 37); float32 of 64 84, 80, 69, 76.
  static constexpr int kGroups = std::min(NB == 1 ? (DP == 64 ? 4 : NP == 1 ? 2 : 3) : NB == 2 && DP == 64 ? 3 : 2, 160 * 1024 / kLds);
  // What a unit's beginning and end cost, in tiles of 256 keys.  One block, us with 1, 3, 5: 32 requests of 3500 keys, 12 heads, float32, 26.7, 28.8,
  // 30.9; 128 of 6000, one token, 123.5, 126.3, 126.5.  More blocks, with 1, 2, 3, 4, 6: 64 requests of 2000 keys and 9 tokens 51.6, 48.9, 48.5, 48.5,
  // 47.4; with 2, 3, 4, 6: pieces of prompts 303, 306, 310, 321; requests of up to 1000, 2000 and 4000 keys (128, 8, 32), 64 rows a head 77.5, 81.1,
  // 82.7, 82.1, 21.9, 24.0, 24.3, 23.4 and 54.1, 55.7, 53.6, 56.6.
  static constexpr int kRuns = kGroups * kCUs, kLeast = 1, kCost = NB == 1 ? 1 : 2;
};

template <typename T, int DP, int NB, int PAGES>
__device__ __forceinline__ void codes_piece(const Attend4Args &a, const Unit &u, int32_t tile, int32_t tiles, unsigned char *lds,
                                            Part<DP, Work4<T, DP, NB>::R> *part) {
  using C = Codes<DP>;
  using W = Work4<T, DP, NB>;
  constexpr int NP = W::NP;
  int tid = threadIdx.x;
  asm("" : "+v"(tid));                  // what follows from it is formed here, not kept in registers from piece to piece
  const int lane = tid & (kWave - 1), stream = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, quarter = lane >> 4;
  unsigned char *const mine = lds + stream * W::kWaveLds;
  float *const scale = reinterpret_cast<float *>(mine + C::kStage);
  unsigned char *const queries = lds + kAttendWaves * W::kWaveLds + lane * 16;
  // the positions of the first and the last row, and the keys of this wave's stream that they see
  const int32_t last = min(u.r0 + W::R, u.rows) - 1;
  const int32_t pos_first = u.ctx + u.r0 / a.G, pos_last = u.ctx + last / a.G;
  const int32_t lo_last = a.window > 0 ? pos_last - a.window : -1;
  const int32_t begin = u.k_lo + tile * W::TK + stream * C::KEYS;
  const int32_t end = min(min(u.k_hi, u.k_lo + (tile + tiles) * W::TK), pos_last + 1);
  const int32_t stages = end > begin ? (end - begin + W::TK - 1) / W::TK : 0;

  // The rows' queries, asked for ahead of everything else: step i of the scores takes elements quarter * DP / 4 + 8 i and on of each quarter's
  // lanes, so that the codes of a key that lie in a row make all steps.
  int32_t pos[NB];
  u32x4 q[NB][C::NQ][sizeof(T) / 2];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const Row w = row_at(a, u, u.r0 + 16 * b + l16);
    pos[b] = w.pos;
    if (stream > 0) continue;
    const T *from = reinterpret_cast<const T *>(a.q) + w.token * a.q_tok + w.head * a.q_head;
#pragma unroll
    for (int i = 0; i < C::NQ; ++i) {
      const int d = quarter * (DP / 4) + 8 * i;
#pragma unroll
      for (int h = 0; h < (int) sizeof(T) / 2; ++h) q[b][i][h] = *(w.there && d < a.D ? reinterpret_cast<const u32x4 *>(from + d + 4 * h) : &kZeros);
    }
  }
  Loader4<DP, PAGES> loader(a, u, lane, begin, W::TK, mine + W::kWaveLds - 256);
  bare_barrier();                       // nobody uses the piece before any more
  loader.ask(loader.kEach, lane);
  if (stages > 0) {
    loader.template load<false>(0, mine);
    loader.template load<true>(0, mine);
  }
  if (stream == 0) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < C::NQ; ++i) {
        bf16x8 x[NP];
        if constexpr (NP == 1) {
          x[0] = __builtin_bit_cast(bf16x8, q[b][i][0]);
        } else {
          const floatx4 y = __builtin_bit_cast(floatx4, q[b][i][0]), z = __builtin_bit_cast(floatx4, q[b][i][1]);
          const float eight[8] = {y[0], y[1], y[2], y[3], z[0], z[1], z[2], z[3]};
          operands<NP, true>(eight, x);
        }
#pragma unroll
        for (int p = 0; p < NP; ++p) *reinterpret_cast<bf16x8 *>(queries + ((b * C::NQ + i) * NP + p) * 1024) = x[p];
      }
  }
  bare_barrier();

  // Scores of 64 keys are four products of 16; register i of product t is, in a lane of quarter g, key 16 g + 4 t + i: the operand of the lane's
  // weights and the codes of 16 keys that one transposing read brings then have the same order.
  const int key_row = (l16 >> 2) * 16 + (l16 & 3), value_row = lane;
  floatx4 o[NB][C::NM];
  float ref[NB], sum[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
#pragma unroll
    for (int m = 0; m < C::NM; ++m) o[b][m] = floatx4{};
    ref[b] = -INFINITY;
    sum[b] = 0.f;
  }
  // Arguments that the loop uses, each for itself: the arguments as a whole do not find scalar registers, and come back in groups of eight.
  const int32_t head_dim = apart(a.D), window = apart(a.window);
  const float score = apart(a.c);
  // compared where it is used: the results of all comparisons would be kept
  auto columns = [&] {
    int32_t d = head_dim;
    asm("" : "+s"(d));
    return d;
  };
#pragma nounroll
  for (int32_t n = 0; n < stages; ++n) {
    const bool more = n + 1 < stages;
    // A CU's two workgroups have precedence by turns, four stages each.  Without turns the older one always has it, and the younger one ends
    // alone, with half of the waves: after 59 and 80 us where 2 requests have 120000 keys.  With turns such a call takes 74 instead of 77 us, 8
    // prompts' pieces of up to 1024 tokens behind 8000 keys 305 instead of 317, 64 requests of 9 tokens and up to 2000 keys 48.5 instead of 49.8.
    // Turns of 2 to 16 stages measure within 2% of these.  One block of 16 rows, whose time is its codes', takes no turns: 127.3 for 126.0.
    if constexpr (NB > 1) {
      if ((n / 4 ^ (int) (blockIdx.x / kCUs)) & 1) __builtin_amdgcn_s_setprio(1);
      else __builtin_amdgcn_s_setprio(0);
    }
    // Loads come in in their order: pages for later stages (if any), a stage's keys, its scales, its values.  Keys, scales and the pages ahead of
    // them are in, the values may be on their way.
    wait_vm<C::NI>();
    const unsigned char *const kl = mine, *const vl = kl + C::kBytes;
    // All codes of keys into registers, so that those of another stage may come into their place.
    uint32_t kc[4][C::NQ];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int row = key_row + 4 * t;
      if constexpr (C::NQ == 4) {
        const u32x4 x = *reinterpret_cast<const u32x4 *>(kl + row * C::RB + (code_swap<C::RB>(row, quarter) << 4));
#pragma unroll
        for (int i = 0; i < 4; ++i) kc[t][i] = x[i];
      } else {
        const u32x2 x = *reinterpret_cast<const u32x2 *>(kl + row * C::RB + (code_swap<C::RB>(row, quarter >> 1) << 4) + (quarter & 1) * 8);
#pragma unroll
        for (int i = 0; i < 2; ++i) kc[t][i] = x[i];
      }
    }
    uint32_t both = reinterpret_cast<const uint32_t *>(kl + 2 * C::kBytes)[lane];
    bf16x8 qf[2][NB][NP];               // queries of a step and of the next
    auto ask = [&](int i) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int p = 0; p < NP; ++p) qf[i % 2][b][p] = *reinterpret_cast<const bf16x8 *>(queries + ((b * C::NQ + i) * NP + p) * 1024);
    };
    wait_lds();
    ask(0);
    if (more) loader.template load<false>(n + 1, mine);
    // scales as float32, those of keys with c; what is not finite is NaN, whatever the codes
    {
      const float x = __uint_as_float(both << 16), y = __uint_as_float(both & 0xffff0000u);
      scale[lane] = fmaf(x, 0.f, x) * score;
      scale[C::KEYS + lane] = fmaf(y, 0.f, y);
    }
    floatx4 s[NB][4];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int t = 0; t < 4; ++t) s[b][t] = floatx4{};
    floatx4 ks[4], vs[4];
#pragma unroll
    for (int i = 0; i < C::NQ; ++i) {
      pin();
      if (i + 1 < C::NQ) ask(i + 1);
      else
#pragma unroll
        for (int t = 0; t < 4; ++t) ks[t] = *reinterpret_cast<const floatx4 *>(scale + 16 * quarter + 4 * t);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const bf16x8 kf = decoded(kc[t][i]);
#pragma unroll
        for (int p = NP - 1; p >= 0; --p)
#pragma unroll
          for (int b = 0; b < NB; ++b) s[b][t] = product(kf, qf[i % 2][b][p], s[b][t]);
      }
    }
    pin();
    // Scores in log2 units: products with c s_k, rounded, so that those of one size have one weight wherever they stand.
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int b = 0; b < NB; ++b) s[b][t] *= ks[t];
    const int32_t k = begin + n * W::TK;
    const bool edge = k + C::KEYS - 1 > pos_first || k <= lo_last;
    // Numbers in place of those of keys that a row does not see.
    auto hide = [&](float x) {
      int l = lane;
      asm("" : "+v"(l));                // formed here, not kept in registers
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        // first <= 4 t + i <= to is seen; a window may be as long as numbers go
        const int32_t here = k + (l >> 4) * 16, to = pos[b] - here, first = window > 0 ? max(pos[b] - window, -1) + 1 - here : 0;
        const uint32_t count = (uint32_t) max(to - first + 1, 0);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          pin();                        // not all comparisons ahead of all moves
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if ((uint32_t) (4 * t + i - first) >= count) s[b][t][i] = x;
        }
      }
    };
    if (edge) hide(-INFINITY);
    float mx[NB];
    bool ahead = false;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      float m[2] = {s[b][0][0], s[b][0][1]};
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = t ? 0 : 2; i < 4; ++i) m[i & 1] = fmaxf(m[i & 1], s[b][t][i]);
      mx[b] = quad_max(fmaxf(m[0], m[1]));
      ahead = ahead || mx[b] > ref[b] + kLag;
    }
    // The rows' references follow the maxima where one runs more than kLag ahead, see follow in pcg_attend_device.h.
    if (__builtin_amdgcn_ballot_w64(ahead) != 0) {
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const float now = fmaxf(ref[b], mx[b]), f = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ref[b] - now);
        ref[b] = now;
        sum[b] *= f;
#pragma unroll
        for (int m = 0; m < C::NM; ++m) o[b][m] *= f;
      }
    }
    pin();
    if (more) wait_vm<C::NI + 1>();     // values are in, the next keys may be on their way
    else wait_vm<0>();
    // lane x of 16 reads 16 codes of key x, columns 16 m .., and gets back column x of the 16 keys
    typedef int intx2 __attribute__((ext_vector_type(2)));
    typedef __attribute__((address_space(3))) intx2 lds8;
    intx2 vc[C::NM];
#pragma unroll
    for (int m = 0; m < C::NM; ++m)
      vc[m] = __builtin_amdgcn_ds_read_tr4_b64_v2i32(
          (lds8 *) (vl + value_row * C::RB + (code_swap<C::RB>(value_row, m >> 1) << 4) + (m & 1) * 8));
#pragma unroll
    for (int t = 0; t < 4; ++t) vs[t] = *reinterpret_cast<const floatx4 *>(scale + C::KEYS + 16 * quarter + 4 * t);
    pin();
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const float minus = minus_ref(ref[b]);
      float z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[b][t][i] = __builtin_amdgcn_exp2f(s[b][t][i] + minus);
          z[i] += s[b][t][i];
        }
      sum[b] += (z[0] + z[1]) + (z[2] + z[3]);
      asm volatile("" : "+v"(sum[b]));  // formed here: weights that wait to be added take registers
    }
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int b = 0; b < NB; ++b) s[b][t] *= vs[t];
    if (edge) hide(0.f);                // a scale that is NaN stays out of rows that do not see its key
    bf16x8 pf[NB][2][NP];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const float eight[8] = {s[b][2 * c][0], s[b][2 * c][1], s[b][2 * c][2], s[b][2 * c][3], s[b][2 * c + 1][0], s[b][2 * c + 1][1],
                                s[b][2 * c + 1][2], s[b][2 * c + 1][3]};
        operands<NP, false>(eight, pf[b][c]);
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          u32x4 x = __builtin_bit_cast(u32x4, pf[b][c][p]);
          asm volatile("" : "+v"(x));   // formed here too
          pf[b][c][p] = __builtin_bit_cast(bf16x8, x);
        }
      }
    wait_lds();
    if (more) loader.template load<true>(n + 1, mine);
    // two blocks of columns at a time, so that products that add to the same sums do not follow each other
#pragma unroll
    for (int m = 0; m < C::NM; m += 2) {
      if (16 * m >= columns()) break;
      pin();
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const bf16x8 vf = decoded((uint32_t) vc[m + h][c]);
#pragma unroll
          for (int p = NP - 1; p >= 0; --p)
#pragma unroll
            for (int b = 0; b < NB; ++b) o[b][m + h] = product(vf, pf[b][c][p], o[b][m + h]);
        }
    }
  }

  const Attend4Args &e = arguments();
  // The streams' rows: outputs go to LDS in passes, and every wave joins and stores some columns of all of them.  They come where other
  // waves' stages and pages were: nothing may be on its way into LDS any more.  The loop ends with such a wait; a wave without a stage has not
  // been in it, and the pages that it asked for may not be in yet.
  wait_vm<0>();
  bare_barrier();
  constexpr int kColumns = C::NM / W::kPasses, kMine = kColumns / kAttendWaves;       // blocks of 16 of a pass, and of a wave
  static_assert(kMine >= 1, "");
  floatx4 *const room = reinterpret_cast<floatx4 *>(lds);
  floatx2 *const sums = reinterpret_cast<floatx2 *>(lds + W::kRows);
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const float all = quad_sum(sum[b]);
    if (quarter == 0) sums[(stream * NB + b) * 16 + l16] = floatx2{ref[b], all};
  }
  auto give = [&](int pass) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int m = 0; m < kColumns; ++m) room[((stream * NB + b) * kColumns + m) * kWave + lane] = o[b][pass * kColumns + m];
    bare_barrier();
  };
  give(0);
  // Where each row's outputs go, and what the streams' are to be multiplied by; a row without a score above -infinity is zeros, also where a value
  // was NaN.
  float f[NB][kAttendWaves];
  char *to[NB];
  bool there[NB], zero[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    int32_t r = 16 * b + l16;
    asm("" : "+v"(r));                  // formed here, not kept in registers since the beginning
    const Row w = row_at(e, u, u.r0 + r);
    there[b] = w.there;
    floatx2 of[kAttendWaves];
#pragma unroll
    for (int i = 0; i < kAttendWaves; ++i) of[i] = sums[(i * NB + b) * 16 + l16];
    float now = of[0][0], all = 0.f;
#pragma unroll
    for (int i = 1; i < kAttendWaves; ++i) now = fmaxf(now, of[i][0]);
#pragma unroll
    for (int i = 0; i < kAttendWaves; ++i) {
      f[b][i] = now == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(of[i][0] - now);
      all = fmaf(f[b][i], of[i][1], all);
    }
    zero[b] = !part && all == 0.f;
    if (part) {
      to[b] = reinterpret_cast<char *>(part->o[r] + 4 * quarter);
      if (quarter == 0 && stream == 0 && w.there) {
        part->ref[r] = now;
        part->sum[r] = all;
      }
    } else {
      to[b] = reinterpret_cast<char *>(reinterpret_cast<T *>(e.out) + w.token * e.o_tok + w.head * e.o_head + 4 * quarter);
      const float inv = 1.f / all;
#pragma unroll
      for (int i = 0; i < kAttendWaves; ++i) f[b][i] *= inv;
    }
  }
#pragma unroll
  for (int pass = 0; pass < W::kPasses; ++pass) {
    if (pass) {
      bare_barrier();
      give(pass);
    }
#pragma unroll
    for (int m = 0; m < kMine; ++m)
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int at = stream * kMine + m, d = 16 * (pass * kColumns + at);
        floatx4 x = floatx4{};
#pragma unroll
        for (int i = 0; i < kAttendWaves; ++i)
          x = __builtin_elementwise_fma(room[((i * NB + b) * kColumns + at) * kWave + lane], floatx4{f[b][i], f[b][i], f[b][i], f[b][i]}, x);
        if (zero[b]) x = floatx4{};
        if (!there[b] || (!part && d + 4 * quarter >= e.D)) continue;
        if (part || sizeof(T) == 4) {
          *reinterpret_cast<floatx4 *>(to[b] + d * 4) = x;
        } else {
          *reinterpret_cast<u32x2 *>(to[b] + d * 2) = u32x2{__builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2{x[0], x[1]}), bf16x2)),
                                                            __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2{x[2], x[3]}), bf16x2))};
        }
      }
  }
}

template <typename T, int DP, int NB, int PAGES>
__global__ __launch_bounds__(kAttendThreads, (Work4<T, DP, NB>::kGroups)) void attend4_kernel(Attend4Args a, Join *join,
                                                                                              Part<DP, Work4<T, DP, NB>::R> *parts) {
  using W = Work4<T, DP, NB>;
  __shared__ __align__(16) unsigned char lds[W::kLds];
  // Where heads lie closer together than a head's keys, two workgroups on one XCD (8 blocks apart) work through the keys of two neighbours at
  // the same time: memory is read in pieces of 128 bytes, or of 64 that are neighbours (128 requests of 3800 keys 118 us, 185 without).
  Heads deal = all_heads(a);
  if (a.pairs) {
    deal.first = (int32_t) (deal.block / 8 % 2);
    deal.step = 2;
    deal.heads /= 2;
    deal.block = deal.block / 16 * 8 + deal.block % 8;
    deal.count /= 2;
    join += deal.first * deal.count;
    parts += 2 * (int64_t) deal.first * deal.count;
  }
  work_on_run<DP, W::R, W::TK, W::kLeast, kAttendWaves, W::kCost>(a, deal, lds, join, parts,
                                                                  [&](const Unit &unit, int32_t tile, int32_t tiles, Part<DP, W::R> *part) {
    Unit u = unit;
    u.head = deal.first + u.head * deal.step;
    codes_piece<T, DP, NB, PAGES>(arguments(), u, tile, tiles, lds, part);
  });
}

// Joins the parts of units that runs cut: as many reads as there are parts, a few microseconds in a launch of its own (3.5 us where there is next
// to nothing, 6.7 for the parts of 512 runs of 36 rows, 19 MB).
template <typename T, int DP, int R>
__global__ __launch_bounds__(kJoinThreads) void attend4_join_kernel(AttendArgs a, const Join *join, const Part<DP, R> *parts) {
  join_parts<T, DP, R>(a, join, parts);
}

template <typename T, int DP, int NB>
hipError_t go(const Attend4Args &a, void *workspace, hipStream_t stream) {
  using W = Work4<T, DP, NB>;
  Join *join = reinterpret_cast<Join *>(workspace);
  Part<DP, W::R> *parts = reinterpret_cast<Part<DP, W::R> *>(reinterpret_cast<char *>(workspace) + join_bytes(W::kRuns));
  // Places by groups of 16 keys where these share a page and lie within 32 bits of each other: pieces of prompts 306 us, 338 with places key by
  // key; 2 requests of 115000 keys 77 and 84, 64 of 1260 48.6 and 50.2.
  if (a.page_size % 16 == 0 && a.k_tok < (int64_t) 1 << 27 && a.s_tok < (int64_t) 1 << 25)
    attend4_kernel<T, DP, NB, 1><<<W::kRuns, kAttendThreads, 0, stream>>>(a, join, parts);
  else attend4_kernel<T, DP, NB, 2><<<W::kRuns, kAttendThreads, 0, stream>>>(a, join, parts);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  attend4_join_kernel<T, DP, W::R><<<dim3(W::kRuns, W::R / 4), kJoinThreads, 0, stream>>>(a, join, parts);
  return hipGetLastError();
}

// Calls f(NB) as it fits `rows`: rows of a shared head of the longest request, of which there are `heads` in all requests.  bfloat16 takes the
// blocks of 16 that leave the fewest rows empty up to 48, and afterwards three unless two need no more passes over the keys.  32 requests of 4000
// keys, 8 shared heads of 128, NB = 1, 2, 3, us: 4 to 16 rows 36, 42, 54; 20 to 32 52, 44, 56; 36 to 48 80, 60, 58; 52 to 64 76, 63, 81; 68 to 96
// 119, 96, 79; 97 to 128 145, 108, 128; 132 195, 145, 129; 256 256, 208, 215.  float32 has no registers for three, and two are fewer workgroups: they
// pay where there is work for all.  NB = 1, 2, heads of 128, us: 32 requests of 4000 keys, 20 rows 68, 62, 48 rows 86, 96, 64 124, 98, 128 224, 180;
// 8 of 2000, 20 rows 24, 26, 64 28, 33, 256 70, 67, 1024 224, 203.
template <bool BF16, typename F>
auto by_rows(int64_t rows, int64_t heads, F f) {
  using std::integral_constant;
  if constexpr (BF16) {
    if (rows > 16 && (rows <= 32 || (rows > 48 && rows <= 64) || (rows > 96 && rows <= 128))) return f(integral_constant<int, 2>());
    if (rows > 32) return f(integral_constant<int, 3>());
  } else {
    if (rows > 16 && (rows <= 32 || rows > 48) && heads * ((rows + 15) / 16) >= 2 * kCUs) return f(integral_constant<int, 2>());
  }
  return f(integral_constant<int, 1>());
}

template <typename T, int DP, int NB>
size_t bytes() { return parts_bytes<T, DP, Work4<T, DP, NB>::R>(Work4<T, DP, NB>::kRuns); }
// What any call takes, so that what is enough for the longest chunks and the most requests is enough for others.
template <int DP>
size_t most() {
  return std::max({bytes<uint16_t, DP, 1>(), bytes<uint16_t, DP, 2>(), bytes<uint16_t, DP, 3>(), bytes<float, DP, 1>(), bytes<float, DP, 2>()});
}

template <typename T, int DP>
hipError_t go_rows(const Attend4Args &a, int64_t longest, void *workspace, hipStream_t stream) {
  return by_rows<sizeof(T) == 2>(longest * a.G, (int64_t) a.B * a.heads_kv, [&](auto nb) { return go<T, DP, decltype(nb)::value>(a, workspace, stream); });
}

}  // namespace

size_t attend4_workspace_bytes(int32_t D) { return D <= 64 ? most<64>() : most<128>(); }

hipError_t launch_cache4_attend(const Attend4Args &a, bool bf16, int64_t longest, void *workspace, hipStream_t stream) {
  if (bf16) return a.D <= 64 ? go_rows<uint16_t, 64>(a, longest, workspace, stream) : go_rows<uint16_t, 128>(a, longest, workspace, stream);
  return a.D <= 64 ? go_rows<float, 64>(a, longest, workspace, stream) : go_rows<float, 128>(a, longest, workspace, stream);
}

}  // namespace pcg
