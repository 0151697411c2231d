// Attention of new tokens over a paged cache of 4-bit codes (gfx950, wave64).
//
// An element is scale * code, code one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives, one scale a token and shared head for its key
// and one for its value.  Codes are exact in bfloat16, so that the products of pcg_attend.hip are made of them as they stand,
//   S^T = C_k Q^T,  score = c s_k S        O^T = C_v^T (s_v P)^T
// and the scales meet scores and weights, one multiplication each, and never the elements.  float32 queries and weights are three
// bfloat16 numbers each, which hold all of their 24 bits: three products of the fast kind, exact in every term, where one of float32
// takes sixteen times as long.
//
// Every wave has 32 rows and a stream of keys of its own, 32 at a time, which it brings into its own part of LDS several steps ahead: nothing is
// shared in the loop, and no wave waits for another one in it.  Rows, units, runs and parts are those of pcg_attend.hip.
#include "pcg_attend_device.h"

namespace pcg {

namespace {

// 4 bytes a lane from memory to 256 bytes of LDS in a row; see bring.
__device__ __forceinline__ void bring_word(const char *from, const unsigned char *to) {
  asm volatile("s_nop 4\n\tglobal_load_lds_dword %0, off" :: "v"(from), "{m0}"(lds_address(to)) : "memory");
}
// 16 bytes a lane from base + offset.
__device__ __forceinline__ void bring_from(const char *base, uint32_t offset, const unsigned char *to) {
  asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" :: "v"(offset), "s"(base), "{m0}"(lds_address(to)) : "memory");
}

template <int DP>
struct Codes {
  static constexpr int RB = DP / 2;                 // bytes of a key
  static constexpr int CH = RB / 16;
  static constexpr int RPI = kWave / CH;            // keys that one load of a wave brings
  static constexpr int NI = 32 / RPI;               // loads of 32 keys
  static constexpr int kBytes = 32 * RB;
  static constexpr int kStage = 2 * kBytes + 256;   // codes of keys, of values, scales
  static constexpr int kOps = 2 * NI + 1;           // loads of a stage
  static constexpr int kStages = 4;                 // one in use, three on their way
  static constexpr int kWaveLds = kStages * kStage + 256;     // and the scales in use, as float32
  static constexpr int NQ = DP / 16, NO = DP / 32;
};

// Which 16-byte chunk of key `row` lies at chunk position `pos` of its row in LDS, and the other way round: the keys that one read touches
// (0-3, 16-19, 4-7, 20-23 and so on as scores, 0-15 and 16-31 as values) have to differ modulo 256 bytes.
template <int RB>
__device__ __forceinline__ int code_swap(int row, int pos) {
  if constexpr (RB == 64) return pos ^ ((row >> 2) & 3) ^ ((row >> 4) << 1);
  else return pos ^ (((row >> 3) ^ (row >> 4)) & 1);
}

// Brings 32 keys, values and scales of a unit into LDS.  PAGES 1: pages of a multiple of 16 slots, so that 16 keys in a row share one, which the
// scalar unit looks up; 2: pages of any size, looked up by each lane.  Chunks behind D are the row's first ones: queries are zero
// there, and the columns that values make there are not stored.
template <int DP, int PAGES>
struct Loader4 {
  using C = Codes<DP>;
  const Attend4Args &a;
  const Unit &u;
  const int lane;
  const int32_t *table;
  const char *kb, *vb, *sb;
  uint32_t off[C::NI];        // of this lane from the first key of 16

  __device__ __forceinline__ int row_of(int i) const { return i * C::RPI + lane / C::CH; }
  __device__ __forceinline__ int chunk(int row) const {
    const int ch = code_swap<C::RB>(row, lane % C::CH);
    return ch * 32 < a.D ? ch * 16 : 0;
  }
  __device__ __forceinline__ Loader4(const Attend4Args &a_, const Unit &u_, int lane_)
      : a(a_), u(u_), lane(lane_), table(a_.table + (int64_t) u_.b * a_.table_stride) {
    kb = reinterpret_cast<const char *>(a.k) + (int64_t) u.head * a.k_head;
    vb = reinterpret_cast<const char *>(a.v) + (int64_t) u.head * a.k_head;
    sb = reinterpret_cast<const char *>(a.scales + (int64_t) u.head * a.s_head);
#pragma unroll
    for (int i = 0; i < C::NI; ++i) off[i] = (uint32_t) (row_of(i) & 15) * (uint32_t) a.k_tok + (uint32_t) chunk(row_of(i));
  }

  // Pages of the keys from k0 on: of 16 keys (PAGES 1); of each load's key of this lane, and of the key whose scales it brings.
  static constexpr int NP = PAGES == 1 ? 2 : C::NI + 1;
  struct Pages {
    int32_t page[NP];
  };
  __device__ __forceinline__ int32_t key_of(int32_t k0, int i) const {
    return k0 + (PAGES == 1 ? 16 * i : i < C::NI ? row_of(i) : lane & 31);
  }
  __device__ __forceinline__ Pages look_up(int32_t k0) const {
    Pages p;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      uint32_t block, slot;
      split_by((uint32_t) key_of(k0, i), (uint32_t) a.page_size, a.magic_page, block, slot);
      p.page[i] = fixed_at(table, min(block, (uint32_t) a.max_blocks - 1));
    }
    return p;
  }

  __device__ __forceinline__ void load(int32_t k0, const Pages &p, unsigned char *to) const {
    int64_t codes[NP], scales[NP];
    bool valid[NP], whole = PAGES == 1 && k0 + 32 <= u.k_hi;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      uint32_t block, slot;
      split_by((uint32_t) key_of(k0, i), (uint32_t) a.page_size, a.magic_page, block, slot);
      valid[i] = key_of(k0, i) < u.k_hi && block < (uint32_t) a.max_blocks && (uint32_t) p.page[i] < (uint32_t) a.num_pages;
      whole = whole && valid[i];
      codes[i] = (int64_t) p.page[i] * a.k_page + (int64_t) slot * a.k_tok;
      scales[i] = ((int64_t) p.page[i] * a.s_page + (int64_t) slot * a.s_tok) * 4;
    }
    unsigned char *const values = to + C::kBytes, *const both = to + 2 * C::kBytes;
    const char *const zeros = reinterpret_cast<const char *>(&kZeros);
    if constexpr (PAGES == 1) {
      const bool second = lane & 16;
      const char *at_scales = sb + (second ? scales[1] : scales[0]) + (int64_t) (lane & 15) * a.s_tok * 4;
      if (whole) {
#pragma unroll
        for (int i = 0; i < C::NI; ++i) {
          if constexpr (C::NI == 2) {
            bring_from(kb + codes[i], off[i], to + i * 1024);
            bring_from(vb + codes[i], off[i], values + i * 1024);
          } else {
            const int64_t at = (lane < 32 ? codes[0] : codes[1]) + off[0];
            bring(kb + at, to);
            bring(vb + at, values);
          }
        }
        bring_word(at_scales, both);
      } else {
        // a unit's last keys, pages outside the cache: zeros where there is no key
#pragma unroll
        for (int i = 0; i < C::NI; ++i) {
          const bool upper = row_of(i) & 16, there = (upper ? valid[1] : valid[0]) && k0 + row_of(i) < u.k_hi;
          const int64_t at = (upper ? codes[1] : codes[0]) + off[i];
          bring(there ? kb + at : zeros, to + i * 1024);
          bring(there ? vb + at : zeros, values + i * 1024);
        }
        bring_word((second ? valid[1] : valid[0]) && k0 + (lane & 31) < u.k_hi ? at_scales : zeros, both);
      }
    } else {
#pragma unroll
      for (int i = 0; i < C::NI; ++i) {
        const int64_t at = codes[i] + chunk(row_of(i));
        bring(valid[i] ? kb + at : zeros, to + i * 1024);
        bring(valid[i] ? vb + at : zeros, values + i * 1024);
      }
      bring_word(valid[C::NI] ? sb + scales[C::NI] : zeros, both);
    }
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

__device__ __forceinline__ floatx16 product(bf16x8 x, bf16x8 y, floatx16 s) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, s, 0, 0, 0);
}

// WK streams of keys, 4 / WK blocks of 32 rows.
template <int WK>
struct Work4 {
  static constexpr int WR = kAttendWaves / WK, R = 32 * WR, TK = 32 * WK;
  static constexpr int kRuns = 512, kLeast = 1;
};

template <typename T, int DP, int WK, int PAGES>
__device__ __forceinline__ void codes_piece(const Attend4Args &a, const Unit &u, int32_t tile, int32_t tiles, unsigned char *lds,
                                            Part<DP, Work4<WK>::R> *part) {
  using C = Codes<DP>;
  using W = Work4<WK>;
  constexpr int NP = sizeof(T) == 2 ? 1 : 3;
  int tid = threadIdx.x;
  asm("" : "+v"(tid));                  // what follows from it is formed here, not kept in registers from piece to piece
  const int lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, half = lane >> 5;
  const int block = wave % W::WR * 32, stream = wave / W::WR;
  const Loader4<DP, PAGES> loader(a, u, lane);
  unsigned char *const mine = lds + wave * C::kWaveLds;
  float *const scale = reinterpret_cast<float *>(mine + C::kStages * C::kStage);
  // rows of this wave, the positions of its first and last, and the keys that they see
  const Row w = row_at(a, u, u.r0 + block + l32);
  const int32_t last = min(u.r0 + block + 32, u.rows) - 1;
  const int32_t pos_first = u.ctx + (u.r0 + block) / a.G, pos_last = last >= u.r0 + block ? u.ctx + last / a.G : -1;
  const int32_t lo = a.window > 0 ? w.pos - a.window : -1, lo_last = a.window > 0 ? pos_last - a.window : -1;
  const int32_t begin = u.k_lo + tile * W::TK + stream * 32;
  const int32_t end = min(min(u.k_hi, u.k_lo + (tile + tiles) * W::TK), pos_last + 1);
  const int32_t stages = end > begin ? (end - begin + W::TK - 1) / W::TK : 0;

  bare_barrier();                       // nobody uses the piece before any more
  auto pages = loader.look_up(begin);   // of the stage that is brought next
  auto load = [&](int32_t n) {
    loader.load(begin + n * W::TK, pages, mine + n % C::kStages * C::kStage);
    pages = loader.look_up(begin + (n + 1) * W::TK);
  };
#pragma unroll
  for (int n = 0; n < C::kStages - 1; ++n)
    if (n < stages) load(n);

  // Step i of the scores takes elements half * DP / 2 + 8 i and on of each half's lanes: 16 bytes of codes in a row make four steps.
  bf16x8 qf[C::NQ][NP];
  {
    const T *q = reinterpret_cast<const T *>(a.q) + w.token * a.q_tok + w.head * a.q_head;
#pragma unroll
    for (int i = 0; i < C::NQ; ++i) {
      const int d = half * (DP / 2) + 8 * i;
      const bool there = w.there && d < a.D;
      if constexpr (NP == 1) {
        qf[i][0] = __builtin_bit_cast(bf16x8, *(there ? reinterpret_cast<const u32x4 *>(q + d) : &kZeros));
      } else {
        const floatx4 x = __builtin_bit_cast(floatx4, *(there ? reinterpret_cast<const u32x4 *>(q + d) : &kZeros));
        const floatx4 y = __builtin_bit_cast(floatx4, *(there ? reinterpret_cast<const u32x4 *>(q + d + 4) : &kZeros));
        const float eight[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
        operands<NP, true>(eight, qf[i]);
      }
    }
  }

  // The register r of a lane's scores is key 16 half + r: the operand of the lane's weights and the codes of 16 keys that one transposing
  // read brings then have the same order.  Lane l reads as key of the scores the one that comes out there.
  const int key_row = ((l32 >> 2) & 1) * 16 + (l32 >> 3) * 4 + (l32 & 3);
  const int value_row = half * 16 + (lane & 15);
  floatx16 o[C::NO];
#pragma unroll
  for (int n = 0; n < C::NO; ++n) o[n] = floatx16{};
  float ref = -INFINITY, sum = 0.f;
#pragma nounroll
  for (int32_t n = 0; n < stages; ++n) {
    wait_lds();                         // the stage before is read
    if (n + C::kStages - 1 < stages) load(n + C::kStages - 1);
    const int32_t ahead = stages - 1 - n;
    if (ahead >= 3) wait_vm<3 * C::kOps>();
    else if (ahead == 2) wait_vm<2 * C::kOps>();
    else if (ahead == 1) wait_vm<C::kOps>();
    else wait_vm<0>();
    const unsigned char *const codes = mine + n % C::kStages * C::kStage, *const values = codes + C::kBytes;
    // scales as float32, those of keys with c; what is not finite is NaN, whatever the codes
    {
      const uint32_t both = reinterpret_cast<const uint32_t *>(codes + 2 * C::kBytes)[l32];
      const float s = __uint_as_float(half ? both & 0xffff0000u : both << 16);
      scale[lane] = fmaf(s, 0.f, s) * (half ? 1.f : a.c);
    }
    u32x4 kc[C::NQ / 4];
#pragma unroll
    for (int j = 0; j < C::NQ / 4; ++j)
      kc[j] = *reinterpret_cast<const u32x4 *>(codes + key_row * C::RB + (code_swap<C::RB>(key_row, half * (C::NQ / 4) + j) << 4));
    floatx16 s[1] = {floatx16{}};
#pragma unroll
    for (int i = 0; i < C::NQ; ++i) {
      const bf16x8 kf = decoded(kc[i / 4][i % 4]);
#pragma unroll
      for (int p = NP - 1; p >= 0; --p) s[0] = product(kf, qf[i][p], s[0]);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) s[0][r] *= scale[16 * half + r];
    const int32_t k = begin + n * W::TK;
    const bool edge = k + 31 > pos_first || k <= lo_last;
    const int32_t from = lo - k - 16 * half, to = w.pos - k - 16 * half;      // registers that the row sees: from < r <= to
    if (edge) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (r > to || r <= from) s[0][r] = -INFINITY;
    }
    (void) follow<C::NO, 1>(row_max<1>(s, 1.f), ref, sum, o, s, 1.f);
    to_weights<1>(s, 1.f, minus_ref(ref), sum);
#pragma unroll
    for (int r = 0; r < 16; ++r) s[0][r] *= scale[32 + 16 * half + r];
    if (edge) {                         // a scale that is NaN stays out of rows that do not see its key
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (r > to || r <= from) s[0][r] = 0.f;
    }
    bf16x8 pf[2][NP];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      float eight[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) eight[e] = s[0][8 * c + e];
      operands<NP, false>(eight, pf[c]);
    }
#pragma unroll
    for (int m = 0; m < C::NO; ++m) {
      typedef int intx2 __attribute__((ext_vector_type(2)));
      typedef __attribute__((address_space(3))) intx2 lds8;
      // lane x of 16 reads 16 codes of key x, columns 16 .. of the block, and gets back column x of the 16 keys
      const intx2 vc = __builtin_amdgcn_ds_read_tr4_b64_v2i32(
          (lds8 *) (values + value_row * C::RB + (code_swap<C::RB>(value_row, m) << 4) + ((lane >> 4) & 1) * 8));
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const bf16x8 vf = decoded((uint32_t) vc[c]);
#pragma unroll
        for (int p = NP - 1; p >= 0; --p) o[m] = product(vf, pf[c][p], o[m]);
      }
    }
  }

  // the streams' rows: the upper half of them to the lower one, and again
  float *room = reinterpret_cast<float *>(lds);
  bare_barrier();
#pragma unroll
  for (int n = WK / 2; n > 0; n /= 2) {
    float *at = room + (stream % n * W::WR + wave % W::WR) * kRowsFloats<DP>;
    if (stream >= n && stream < 2 * n) give_rows<DP>(at, lane, o, ref, sum);
    bare_barrier();
    if (stream < n) take_rows<DP>(at, lane, o, ref, sum);
    if (n > 1) bare_barrier();
  }
  if (stream > 0) return;
  sum = pair_sum(sum);
  int32_t r = block + l32;
  asm("" : "+v"(r));                    // formed here, not kept in registers since the beginning
  const Row out = row_at(a, u, u.r0 + r);
  if (part) store_part<DP, W::R>(part, r, half, out.there, o, ref, sum);
  else store_row<T, DP>(a, out, half, o, sum);
}

template <typename T, int DP, int WK, int PAGES>
__global__ __launch_bounds__(kAttendThreads, 2) void attend4_kernel(Attend4Args a, Join *join, Part<DP, Work4<WK>::R> *parts) {
  using W = Work4<WK>;
  constexpr int kRoom = WK > 1 ? WK / 2 * W::WR * kRowsFloats<DP> * 4 : 0, kLds = kAttendWaves * Codes<DP>::kWaveLds;
  static_assert(kRoom <= kLds, "rows on their way between waves");
  __shared__ __align__(16) unsigned char lds[kLds];
  work_on_run<DP, W::R, W::TK, W::kLeast, kAttendWaves>(a, lds, join, parts, [&](const Unit &u, int32_t tile, int32_t tiles, Part<DP, W::R> *part) {
    codes_piece<T, DP, WK, PAGES>(a, u, tile, tiles, lds, part);
  });
}

template <typename T, int DP, int R>
__global__ __launch_bounds__(kJoinThreads) void attend4_join_kernel(AttendArgs a, const Join *join, const Part<DP, R> *parts) {
  join_parts<T, DP, R>(a, join, parts);
}

template <typename T, int DP, int WK>
hipError_t go(const Attend4Args &a, void *workspace, hipStream_t stream) {
  using W = Work4<WK>;
  Join *join = reinterpret_cast<Join *>(workspace);
  Part<DP, W::R> *parts = reinterpret_cast<Part<DP, W::R> *>(reinterpret_cast<char *>(workspace) + join_bytes(W::kRuns));
  // 16 keys share a page, and lie within 32 bits of each other
  if (a.page_size % 16 == 0 && a.k_tok < (int64_t) 1 << 27) attend4_kernel<T, DP, WK, 1><<<W::kRuns, kAttendThreads, 0, stream>>>(a, join, parts);
  else attend4_kernel<T, DP, WK, 2><<<W::kRuns, kAttendThreads, 0, stream>>>(a, join, parts);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  attend4_join_kernel<T, DP, W::R><<<dim3(W::kRuns, W::R == 128 ? 8 : W::R / 4), kJoinThreads, 0, stream>>>(a, join, parts);
  return hipGetLastError();
}

template <typename T, int DP>
hipError_t go_rows(const Attend4Args &a, int64_t longest, void *workspace, hipStream_t stream) {
  const int64_t rows = longest * a.G;
  if (rows <= 32) return go<T, DP, 4>(a, workspace, stream);
  if (rows <= 64) return go<T, DP, 2>(a, workspace, stream);
  return go<T, DP, 1>(a, workspace, stream);
}

template <int DP>
size_t bytes(int64_t rows) {
  if (rows <= 32) return parts_bytes<float, DP, 32>(Work4<4>::kRuns);
  if (rows <= 64) return parts_bytes<float, DP, 64>(Work4<2>::kRuns);
  return parts_bytes<float, DP, 128>(Work4<1>::kRuns);
}

}  // namespace

size_t attend4_workspace_bytes(int32_t G, int32_t D, int64_t longest) { return D <= 64 ? bytes<64>(longest * G) : bytes<128>(longest * G); }

hipError_t launch_cache4_attend(const Attend4Args &a, bool bf16, int64_t longest, void *workspace, hipStream_t stream) {
  if (bf16) return a.D <= 64 ? go_rows<uint16_t, 64>(a, longest, workspace, stream) : go_rows<uint16_t, 128>(a, longest, workspace, stream);
  return a.D <= 64 ? go_rows<float, 64>(a, longest, workspace, stream) : go_rows<float, 128>(a, longest, workspace, stream);
}

}  // namespace pcg
