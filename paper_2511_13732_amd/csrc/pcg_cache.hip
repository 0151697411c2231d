// Page table and slot map of a step's new tokens, and their keys and values into the paged cache (gfx950).
#include "pcg_cache.h"
#include "pcg_device.h"

namespace pcg {

namespace {

constexpr int kPagesThreads = 1024;
constexpr int kPagesWaves = kPagesThreads / kWave;
constexpr int kWriteThreads = 256;
constexpr int kFillAtOnce = 4;

// Inclusive running sum over the workgroup of WAVES waves, and the sum of all.  `part` holds a value per wave.
template <int WAVES, typename T>
__device__ __forceinline__ T block_scan(T v, T *part, T &total) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const T x = __shfl_up(v, d);
    if (lane >= d) v += x;
  }
  __syncthreads();
  if (lane == kWave - 1) part[wave] = v;
  __syncthreads();
  T before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    const T x = part[w];
    before += w < wave ? x : T(0);
    total += x;
  }
  return v + before;
}

// What request b holds and asks for.  The state is only trusted as far as memory is concerned: whatever it says, nothing
// outside the request's row of the table and the pool's stack is touched.
struct Request {
  int32_t len;         // tokens that stay
  int32_t held;        // pages
  int64_t want, need;  // new tokens, pages for both
  bool asks;
};

__device__ __forceinline__ Request request_at(const PagesArgs &p, int32_t b) {
  Request r;
  const int32_t room = p.max_blocks * p.page_size;        // below 2^31 (checked on the host)
  const int32_t len = min(max(p.state_in[b], 0), room);
  const int32_t chunk = min(max(p.state_in[2 * (int64_t) p.B + b], 0), room - len);
  r.held = min(max(p.state_in[p.B + b], 0), p.max_blocks);
  const int32_t add = p.add ? p.add[b] : p.add_all;
  int32_t kept = chunk;
  if (p.commit) {
    const int64_t c = (int64_t) p.commit[b] + p.commit_extra;
    kept = c < 0 ? 0 : c > chunk ? chunk : (int32_t) c;
  }
  r.len = add < 0 ? 0 : len + kept;
  r.asks = add > 0;
  r.want = add < 0 ? 0 : add;
  r.need = (int64_t) (((uint64_t) r.len + (uint64_t) r.want + (uint32_t) p.page_size - 1) / (uint32_t) p.page_size);
  return r;
}

// A run of pages that a request gives back or takes: upto[t] is the sum of the first t + 1 threads' counts.  Thread and place
// of page `i` of them all.
template <int THREADS>
__device__ __forceinline__ int run_of(const int32_t *upto, int32_t i) {
  int lo = 0, n = THREADS;
  while (n > 1) {                       // first t with upto[t] > i
    const int half = n >> 1;
    if (upto[lo + half - 1] <= i) lo += half;
    n -= half;
  }
  return lo;
}

// Slots and positions of N new tokens, `row` and then every `step`-th: their requests by bisection of the starts (in LDS where they
// fit), N beside each other because each is a chain of waits.
template <int N>
__device__ __forceinline__ void place_tokens(const PagesArgs &p, const int32_t *starts, const int32_t *lens, int32_t total,
                                             int64_t row, int32_t step) {
  int32_t lo[N], block[N], page[N], position[N];
#pragma unroll
  for (int i = 0; i < N; ++i) lo[i] = 0;
  for (int32_t n = p.B; n > 1; n -= n >> 1) {             // starts[lo] <= row, and row is ahead of starts[lo + n]
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (starts[lo[i] + (n >> 1)] <= row + (int64_t) i * step) lo[i] += n >> 1;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int64_t at = row + (int64_t) i * step;
    position[i] = page[i] = 0;
    if (at >= total) continue;
    position[i] = lens[lo[i]] + (int32_t) at - starts[lo[i]];
    block[i] = position[i] / p.page_size;
    page[i] = p.table[(int64_t) lo[i] * p.table_stride + block[i]];
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int64_t at = row + (int64_t) i * step;
    if (at >= p.max_tokens) continue;
    p.slots[at] = at < total ? page[i] * p.page_size + (position[i] - block[i] * p.page_size) : -1;
    if (p.positions) p.positions[at] = position[i];
  }
}

// New lengths, page counts, pages and first rows of all requests: running sums over the requests, of the tokens (who fits the batch)
// and of the pages given back and taken (who gets which).  One workgroup, because each sum needs all of the one before and a grid's
// meeting costs more than the work; as many threads as requests, or more, so that every request is read once and stays in registers.
// Bound by trips to memory one after the other (state, pages that come back, pages taken, the table for the slots): 3.4 us for a
// request, 4.4 for 64 with 9 tokens each, 7.4 for 300; the running sums are two where nobody is refused.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void pages_step_kernel(PagesArgs p, int32_t fill_rows) {
  constexpr int W = THREADS / kWave;
  __shared__ int64_t part64[W];
  __shared__ int32_t part[W];
  __shared__ int32_t upto_back[THREADS], upto_taken[THREADS], need[THREADS], held[THREADS], starts[THREADS + 1], lens[THREADS];
  const int tid = threadIdx.x, b = tid;
  const int32_t free_in = min(max(p.state_in[3 * (int64_t) p.B], 0), p.num_pages);
  Request r{0, 0, 0, 0, false};
  if (b < p.B) r = request_at(p, b);
  bool refuse = r.need > p.max_blocks;
  const int64_t want = refuse ? 0 : r.want;
  int64_t total;
  const int64_t sum = block_scan<W>(want, part64, total);
  refuse = refuse || (want > 0 && sum > p.max_tokens);
  const int32_t gives = !refuse && r.held > r.need ? r.held - (int32_t) r.need : 0;
  int32_t takes = !refuse && r.need > r.held ? (int32_t) r.need - r.held : 0;
  int64_t both;
  const int64_t moved = block_scan<W>((int64_t) gives << 32 | takes, part64, both);       // each sum is below 2^31
  const int32_t back = (int32_t) (both >> 32), top = min(free_in + back, p.num_pages);
  if (takes > 0 && (int32_t) moved > top) {
    refuse = true;
    takes = 0;
  }
  int32_t got = (int32_t) want, end = (int32_t) sum, given = (int32_t) both, all = (int32_t) total, refused = 0;
  if (__syncthreads_or(refuse)) {
    got = refuse ? 0 : got;
    end = block_scan<W>(got, part, all);
    (void) block_scan<W>(takes, part, given);
    (void) block_scan<W>(refuse && r.asks ? 1 : 0, part, refused);
  }
  upto_back[tid] = (int32_t) (moved >> 32);
  upto_taken[tid] = (int32_t) moved;
  need[tid] = (int32_t) r.need;
  held[tid] = r.held;
  starts[tid] = end - got;
  lens[tid] = r.len;
  if (tid == THREADS - 1) starts[THREADS] = all;
  __syncthreads();
  for (int32_t i = tid; i < back; i += THREADS) {
    const int t = run_of<THREADS>(upto_back, i);
    const int32_t at = free_in + i, block = need[t] + i - (t ? upto_back[t - 1] : 0);
    if (at < p.num_pages) p.free_pages[at] = p.table[(int64_t) t * p.table_stride + block];
  }
  if (back > 0) __syncthreads();         // what came back can be taken
  for (int32_t i = tid; i < given; i += THREADS) {
    const int t = run_of<THREADS>(upto_taken, i);
    p.table[(int64_t) t * p.table_stride + held[t] + i - (t ? upto_taken[t - 1] : 0)] = p.free_pages[top - 1 - i];
  }
  if (b < p.B) {
    p.state_out[b] = r.len;
    p.state_out[p.B + b] = refuse ? r.held : (int32_t) r.need;
    p.state_out[2 * (int64_t) p.B + b] = got;
    p.q_start[b] = end - got;
  }
  if (tid == 0) {
    p.state_out[3 * (int64_t) p.B] = top - given;
    p.q_start[p.B] = all;
    if (p.refused) *p.refused = refused;
  }
  if (!fill_rows) return;
  if (given > 0) __syncthreads();        // the table is whole
  for (int64_t row = tid; row < p.max_tokens; row += kFillAtOnce * THREADS) place_tokens<kFillAtOnce>(p, starts, lens, all, row, THREADS);
}

// More requests than threads: the same in two passes over them, because who gets pages depends on all that come back.  Requests of
// 4 tokens: 1025 in 19 us, 2600 in 27, 8192 in 61; 65 536 of one token in 432.
__global__ __launch_bounds__(kPagesThreads) void pages_step_large_kernel(PagesArgs p, int32_t fill_rows) {
  __shared__ int64_t part64[kPagesWaves];
  __shared__ int32_t part[kPagesWaves];
  __shared__ int32_t upto[kPagesThreads], first[kPagesThreads];
  // a request that the first pass refuses, one bit each
  __shared__ uint32_t no[kPagesMaxRequests / 32];
  const int tid = threadIdx.x;
  const int32_t free_in = min(max(p.state_in[3 * (int64_t) p.B], 0), p.num_pages);
  for (int i = tid; i < (p.B + 31) / 32; i += kPagesThreads) no[i] = 0;

  // First pass: who does not fit his row of the table or the batch, and the pages that come back.
  int64_t tokens = 0;
  int32_t top = free_in;
  for (int32_t b0 = 0; b0 < p.B; b0 += kPagesThreads) {
    const int32_t b = b0 + tid;
    Request r{0, 0, 0, 0, false};
    if (b < p.B) r = request_at(p, b);
    bool refuse = r.need > p.max_blocks;
    const int64_t want = refuse ? 0 : r.want;
    int64_t total;
    const int64_t sum = tokens + block_scan<kPagesWaves>(want, part64, total);
    tokens += total;
    refuse = refuse || (want > 0 && sum > p.max_tokens);
    if (refuse) atomicOr(&no[b >> 5], 1u << (b & 31));
    const int32_t gives = !refuse && r.held > r.need ? r.held - (int32_t) r.need : 0;
    int32_t back;
    upto[tid] = block_scan<kPagesWaves>(gives, part, back);
    first[tid] = (int32_t) r.need;
    __syncthreads();
    for (int32_t i = tid; i < back; i += kPagesThreads) {
      const int t = run_of<kPagesThreads>(upto, i);
      const int32_t at = top + i, block = first[t] + i - (t ? upto[t - 1] : 0);
      if (at < p.num_pages) p.free_pages[at] = p.table[(int64_t) (b0 + t) * p.table_stride + block];
    }
    top = min(top + back, p.num_pages);
    __syncthreads();
  }

  // Second pass: pages from the top of the stack, and where everybody's tokens are.
  int32_t asked = 0, taken = 0, starts = 0, refused = 0;
  for (int32_t b0 = 0; b0 < p.B; b0 += kPagesThreads) {
    const int32_t b = b0 + tid;
    Request r{0, 0, 0, 0, false};
    if (b < p.B) r = request_at(p, b);
    bool refuse = b < p.B && ((no[b >> 5] >> (b & 31)) & 1);
    int32_t takes = !refuse && r.need > r.held ? (int32_t) r.need - r.held : 0, total;
    const int32_t sum = asked + block_scan<kPagesWaves>(takes, part, total);
    const int32_t before = asked;        // nobody ahead of one who gets pages was refused for want of them
    asked += total;
    if (takes > 0 && sum > top) {
      refuse = true;
      takes = 0;
    }
    int32_t given;
    upto[tid] = block_scan<kPagesWaves>(takes, part, given);
    first[tid] = r.held;
    const int32_t got = refuse ? 0 : (int32_t) r.want;
    const int32_t end = starts + block_scan<kPagesWaves>(got, part, total);
    starts += total;
    (void) block_scan<kPagesWaves>(refuse && r.asks ? 1 : 0, part, total);
    refused += total;
    for (int32_t i = tid; i < given; i += kPagesThreads) {
      const int t = run_of<kPagesThreads>(upto, i);
      p.table[(int64_t) (b0 + t) * p.table_stride + first[t] + i - (t ? upto[t - 1] : 0)] = p.free_pages[top - 1 - before - i];
    }
    taken += given;
    if (b < p.B) {
      p.state_out[b] = r.len;
      p.state_out[p.B + b] = refuse ? r.held : (int32_t) r.need;
      p.state_out[2 * (int64_t) p.B + b] = got;
      p.q_start[b] = end - got;
    }
    __syncthreads();
  }
  if (tid == 0) {
    p.state_out[3 * (int64_t) p.B] = top - taken;
    p.q_start[p.B] = starts;
    if (p.refused) *p.refused = refused;
  }
  if (!fill_rows) return;
  __syncthreads();
  for (int64_t row = tid; row < p.max_tokens; row += kFillAtOnce * kPagesThreads)
    place_tokens<kFillAtOnce>(p, p.q_start, p.state_out, starts, row, kPagesThreads);
}

// A row a thread, where the rows are too many for the workgroup that knows the requests: 65 536 rows of 1024 requests in 9.9 us for
// both launches.
__global__ __launch_bounds__(256) void pages_slots_kernel(PagesArgs p) {
  const int32_t total = p.q_start[p.B];
  const int64_t row = (int64_t) blockIdx.x * 256 + threadIdx.x;
  if (row < p.max_tokens) place_tokens<1>(p, p.q_start, p.state_out, total, row, 0);
}

// One 16-byte part of a token's keys and of its values a thread.  Bound by memory, each part read and written once: 45 MB of float32
// prompts read and as many written in 15.1 us; a step of 576 rows, 2 x 2 KB each, 3.6 us, which a launch alone takes too.
__global__ __launch_bounds__(kWriteThreads) void cache_write_kernel(WriteArgs w) {
  const int64_t i = (int64_t) blockIdx.x * kWriteThreads + threadIdx.x;
  const int64_t row = i / w.parts;
  if (row >= w.T) return;
  const int32_t part = (int32_t) (i - row * w.parts), head = part / w.head_parts, ch = part - head * w.head_parts;
  const int32_t slot = w.slots[row];
  if (slot < 0) return;
  const int32_t page = slot / w.page_size;
  if (page >= w.num_pages) return;
  const int64_t at = slot - page * w.page_size;
  const int64_t e = w.part_elems;
  auto copy = [&](const void *from, int64_t tok, int64_t hd, void *to, int64_t pg, int64_t sl, int64_t hs) {
    const uint4 x = *reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(from) +
                                                     (row * tok + head * hd + ch * e) * w.elem);
    *reinterpret_cast<uint4 *>(reinterpret_cast<char *>(to) + (page * pg + at * sl + head * hs + ch * e) * w.elem) = x;
  };
  copy(w.k_new, w.k_tok, w.k_head, w.k, w.page_stride, w.slot_stride, w.head_stride);
  copy(w.v_new, w.v_tok, w.v_head, w.v, w.page_stride, w.slot_stride, w.head_stride);
}

}  // namespace

hipError_t launch_pages_step(const PagesArgs &p, hipStream_t stream) {
  // Fewer waves meet sooner, more move more pages at a time.  us with 256 and with 1024 threads: 1 request 3.4 and 5.1, 64 requests
  // 4.4 and 6.1; 64 requests that take 1024 pages 7.4 and 8.0, 4000 pages 11.7 and 9.4.
  const bool few = p.B <= 256 && p.max_tokens / p.page_size <= 2048;
  // One launch, or another one with as many threads as rows.  us with one and with two, of 256 threads: 4 rows 3.4 and 4.6, 576
  // 4.4 and 6.2, 2304 7.3 and 6.9, 4096 9.1 and 6.9; of 1024: 2700 7.4 and 8.7, 32 768 26.5 and 9.5.
  const bool fill = p.max_tokens <= (few ? 2048 : 4096);
  if (few) pages_step_kernel<256><<<1, 256, 0, stream>>>(p, fill);
  else if (p.B <= kPagesThreads) pages_step_kernel<kPagesThreads><<<1, kPagesThreads, 0, stream>>>(p, fill);
  else pages_step_large_kernel<<<1, kPagesThreads, 0, stream>>>(p, fill);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || fill) return e;
  pages_slots_kernel<<<(uint32_t) ((p.max_tokens + 255) / 256), 256, 0, stream>>>(p);
  return hipGetLastError();
}

hipError_t launch_cache_write(const WriteArgs &w, hipStream_t stream) {
  const int64_t n = w.T * w.parts;
  cache_write_kernel<<<(uint32_t) ((n + kWriteThreads - 1) / kWriteThreads), kWriteThreads, 0, stream>>>(w);
  return hipGetLastError();
}

}  // namespace pcg
