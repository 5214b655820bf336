// The paged 8-bit key/value cache: pages from the requests' lengths, tokens in,
// tokens out.
//
//  block_tables_kernel  pages of requests that end back onto the free stack,
//                       pages for new blocks off it, the new tokens' slots
//  spread_kernel        pages and slots of calls with many of them
//  kv_append_q8_kernel  new tokens into the pages their slots name
//  kv_fetch_q8_kernel   tokens of the cache back as bf16 or fp32
#include <climits>

#include "q8.h"
#include "sw_common.h"
#include "sw_internal.h"

namespace sw {

// ---------------------------------------------------------------------------
// block tables and slots
// ---------------------------------------------------------------------------

constexpr int kTabThreads = 1024;

// Exclusive prefixes over the workgroup of three numbers in [0, 2^31) per thread,
// and their sums, in 64 bits: scans of the lower 20 and the upper bits within
// each wavefront, then of the wavefronts' sums by every wavefront. One barrier.
struct TabSums {
  long long before[3], total[3];
};
__device__ __forceinline__ TabSums tab_scan(const int (&v)[3], int (*tmp)[kTabThreads / 64]) {
  constexpr int W = kTabThreads / 64;
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
  int part[6], own[6];
#pragma unroll
  for (int q = 0; q < 6; ++q) {
    part[q] = q & 1 ? v[q / 2] >> 20 : v[q / 2] & 0xfffff;
    own[q] = wave_inclusive_scan(part[q]);
    if (l == 63) tmp[q][w] = own[q];
  }
  __syncthreads();
  TabSums s;
#pragma unroll
  for (int q = 0; q < 6; ++q) {
    const int x = wave_inclusive_scan(l < W ? tmp[q][l] : 0);
    const int before = w > 0 ? __builtin_amdgcn_readlane(x, w - 1) : 0;
    const long long b = before + own[q] - part[q], t = __builtin_amdgcn_readlane(x, W - 1);
    s.before[q / 2] = q & 1 ? s.before[q / 2] + (b << 20) : b;
    s.total[q / 2] = q & 1 ? s.total[q / 2] + (t << 20) : t;
  }
  return s;
}

// The last i in [0, n) with pre[i] <= k (pre ascending, pre[0] <= k).
template <typename P>
__device__ __forceinline__ int last_at_most(P pre, int n, int k) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (pre[mid] <= k) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Slot of token p of a sequence, -1 on a page that the pool does not have.
__device__ __forceinline__ int slot_of(const int32_t* table, int p, int B, int n_pages) {
  const int j = p / B;
  const int page = table[j];
  return (unsigned)page < (unsigned)n_pages ? page * B + (p - j * B) : -1;
}

// What the workgroups of a spread call need of the plan: the pages that the
// sequences before each one give back and take, and the stack.
constexpr int kTabCheck = 32;                      // workgroups that look at the blocks given back
struct TabPlan {
  int32_t* rel;       // [n_seqs + 1]
  int32_t* alc;       // [n_seqs + 1]
  int32_t* head;      // [2]: whether the lengths can be served, height of the stack before the call
  int32_t* holes;     // [kTabCheck]: whether a block given back is without a page
};

// tokens >= 0 (in 32 bits: a 64-bit division is over a hundred instructions)
__device__ __forceinline__ int blocks_of(int tokens, int B) {
  return (int)(((uint32_t)tokens + (uint32_t)B - 1) / (uint32_t)B);
}

// Lengths that no call is served with.
__device__ __forceinline__ bool bad_lengths(int o, int w, long long top_len, int rows) {
  return o < 0 || o > top_len || w < 0 || w > top_len || (rows > 0 && (long long)w - o > rows);
}

// Whether a block that is given back is without a page, in any lane of the wavefront:
// `wave` of `waves` looks at sequences wave, wave + waves, ..., the first 64 blocks of
// four of them on their way at a time.
__device__ __forceinline__ bool without_page(int wave, int waves, int n_seqs, int B, int b_max, int rows,
                                             const int32_t* old_len, const int32_t* new_len,
                                             const int32_t* tables, int n_pages) {
  constexpr int N = 4;
  const int l = threadIdx.x & 63;
  uint32_t top = 0;                                // the entries as unsigned numbers
  for (long long base = wave; base < n_seqs; base += 64ll * waves) {
    const long long s = base + (long long)l * waves;
    const int o = s < n_seqs ? old_len[s] : 0, w = s < n_seqs ? new_len[s] : 0;
    const int first = blocks_of(w, B), end = blocks_of(o, B);
    uint64_t left = __ballot(!bad_lengths(o, w, (long long)b_max * B, rows) && first < end);
    while (left) {
      const int32_t* row[N];
      int size[N], who = 0;
      uint32_t page[N];
#pragma unroll
      for (int q = 0; q < N; ++q) {
        if (left) who = __builtin_ctzll(left);     // then the last one again
        left &= left - 1;
        const int a = __builtin_amdgcn_readlane(first, who);
        size[q] = __builtin_amdgcn_readlane(end, who) - a;
        row[q] = tables + (base + (long long)who * waves) * b_max + a;
        page[q] = (uint32_t)row[q][min(l, size[q] - 1)];
      }
#pragma unroll
      for (int q = 0; q < N; ++q) {
        top = max(top, page[q]);
#pragma unroll 4
        for (int j = 64 + l; j < size[q]; j += 64) top = max(top, (uint32_t)row[q][j]);
      }
    }
  }
  return __any(top >= (uint32_t)n_pages);
}

// One workgroup; a thread has the ceil(n / 1024) sequences from t times that on.
// Every length is checked and the pages to give back (R) and to take (A) and the
// new tokens are counted, with one scan. If the call can be served whole, the R
// released pages go onto the stack so that the first of them (sequences ascending,
// blocks ascending) is on top, and the A new blocks take pages from the top in the
// same order. Bounded by latency, three to five dependent loads and as many
// barriers: 4.6 us for one token more for each of 64 requests. PLAN: the prefixes
// alone, for spread_kernel (4.3 us for 512 requests): pages moved by one workgroup
// take 1.5 us per 1024, slots as much. A block given back has to have a page: the
// workgroup looks at them itself where there are any (64 requests, a step of one token and the
// same step back in turn: 4.6 -> 5.0 us a call); PLAN: kTabCheck workgroups beside it, and
// spread_kernel at what they found (512 requests, 8000 to 27000 blocks given back: 10.1 -> 11.1
// for the two launches; 14.9 with the check in the planning workgroup).
template <bool PLAN>
__global__ __launch_bounds__(kTabThreads) void block_tables_kernel(
    int n_seqs, int B, int b_max, const int32_t* __restrict__ old_len,
    const int32_t* __restrict__ new_len, int32_t* __restrict__ tables, int32_t* __restrict__ free_pages,
    int32_t* __restrict__ n_free, int n_pages, int rows, int n_slots, int32_t* __restrict__ slots,
    int32_t* __restrict__ cu, int32_t* __restrict__ pos, int32_t* __restrict__ status, TabPlan plan) {
  __shared__ int tmp[6][kTabThreads / 64];
  __shared__ int pre_r[PLAN ? 1 : kTabThreads], pre_a[PLAN ? 1 : kTabThreads];
  const int t = threadIdx.x;
  if (PLAN && blockIdx.x > 0) {
    const int x = blockIdx.x - 1;
    const bool hole = without_page(x * (kTabThreads / 64) + (t >> 6), kTabCheck * (kTabThreads / 64), n_seqs, B,
                                   b_max, rows, old_len, new_len, tables, n_pages);
    const bool any = __syncthreads_or(hole);
    if (t == 0) plan.holes[x] = any;
    return;
  }
  const int nf = *n_free;
  const long long top_len = (long long)b_max * B;
  const int each = (n_seqs + kTabThreads - 1) / kTabThreads;
  const int s0 = min(t * each, n_seqs), s1 = min(s0 + each, n_seqs);
  bool wrong = false;
  int sums[3];
  {
    long long v[3] = {0, 0, 0};
    for (int s = s0; s < s1; ++s) {
      const int o = old_len[s], w = new_len[s];
      const bool bad = bad_lengths(o, w, top_len, rows);
      wrong |= bad;
      if (bad) continue;
      const int has = blocks_of(o, B), need = blocks_of(w, B);
      v[0] += max(has - need, 0);
      v[1] += max(need - has, 0);
      v[2] += max(w - o, 0);
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      wrong |= v[q] > INT_MAX;
      sums[q] = (int)v[q];
    }
    if (wrong) sums[0] = sums[1] = sums[2] = 0;
  }
  wrong = __syncthreads_or(wrong);
  const TabSums sc = tab_scan(sums, tmp);
  const long long R = sc.total[0], A = sc.total[1];
  if (!PLAN && R > 0)
    wrong |= __syncthreads_or(without_page(t >> 6, kTabThreads / 64, n_seqs, B, b_max, rows, old_len, new_len,
                                           tables, n_pages));
  const bool valid = !wrong && nf >= 0 && nf + R <= n_pages && (rows > 0 || sc.total[2] <= n_slots);
  const bool ok = valid && A - R <= nf;
  const int top = nf + (int)R;                     // of the stack, after the releases
  if (t == 0) {
    *status = valid ? (ok ? 0 : 1) : 2;
    if (ok) *n_free = top - (int)A;
    cu[n_seqs] = ok ? (int)sc.total[2] : 0;
    if (PLAN) {
      plan.head[0] = ok;
      plan.head[1] = nf;
      plan.rel[n_seqs] = (int)R;
      plan.alc[n_seqs] = (int)A;
    }
  }
  // cumulative new tokens (and pages), positions of the last ones
  int r = (int)sc.before[0], a = (int)sc.before[1], g = (int)sc.before[2];
  if (!PLAN) {
    pre_r[t] = r;
    pre_a[t] = a;
  }
  for (int s = s0; s < s1; ++s) {
    const int o = old_len[s], w = new_len[s];
    cu[s] = ok ? g : 0;
    pos[s] = (ok ? w : o) - 1;
    if (!ok) continue;
    const int more = blocks_of(w, B) - blocks_of(o, B);
    if (PLAN) {
      plan.rel[s] = r;
      plan.alc[s] = a;
    }
    r += max(-more, 0);
    a += max(more, 0);
    g += max(w - o, 0);
  }
  if (PLAN) return;
  __syncthreads();                                 // the prefixes, and cu for the slots
  // the sequence of rank k among the blocks given back or taken, and k's number in it
  auto find = [&](const int* pre, int sign, int k, int* num) {
    const int i = last_at_most(pre, kTabThreads, k);
    int s = i * each, left = k - pre[i];
    for (;; ++s) {
      const int n = max(sign * (blocks_of(new_len[s], B) - blocks_of(old_len[s], B)), 0);
      if (left < n) break;
      left -= n;
    }
    *num = left;
    return s;
  };
  if (ok && R > 0) {
    for (int k = t; k < (int)R; k += kTabThreads) {
      int j;
      const int s = find(pre_r, -1, k, &j);
      int32_t* entry = tables + (long long)s * b_max + blocks_of(new_len[s], B) + j;
      free_pages[top - 1 - k] = *entry;
      *entry = -1;
    }
    __syncthreads();
  }
  if (ok && A > 0) {
    for (int k = t; k < (int)A; k += kTabThreads) {
      int j;
      const int s = find(pre_a, 1, k, &j);
      tables[(long long)s * b_max + blocks_of(old_len[s], B) + j] = free_pages[top - 1 - k];
    }
    __syncthreads();
  }
  const int total = ok ? (int)sc.total[2] : 0;
  for (int x = t; x < n_slots; x += kTabThreads) {
    int v = -1;
    if (rows > 0) {
      const int s = x / rows, i = x - s * rows;
      const int o = old_len[s];
      if (ok && i < new_len[s] - o) v = slot_of(tables + (long long)s * b_max, o + i, B, n_pages);
    } else if (x < total) {
      const int s = last_at_most(cu, n_seqs, x);
      v = slot_of(tables + (long long)s * b_max, old_len[s] + (x - cu[s]), B, n_pages);
    }
    slots[x] = v;
  }
}

constexpr int kSpreadLds = 1024;                   // sequences whose lengths and prefixes are kept in LDS

// Pages and slots of a planned call over many workgroups. 16 lanes take the page
// of rank k, from the k-th block given back, or off the stack where there is
// none, and put it into the k-th new block and that block's slots, or onto the
// stack where there is none: no workgroup reads what another one writes. Slots of
// the blocks that the sequences had before, and those that stay empty, are
// written per sequence and behind the last. 512 requests, a third of them prompts of
// 20000 tokens at most: 27000 pages and 1.7 million slots in 6.8 us, 52 with both by
// one workgroup and a search per slot. Eight workgroups per CU, as many as run at once
// (four: 7.9 us; sixteen: 7.2).
template <bool LDS>
__global__ __launch_bounds__(256) void spread_kernel(
    int n_seqs, int B, int b_max, const int32_t* __restrict__ old_len,
    const int32_t* __restrict__ new_len, int32_t* __restrict__ tables, int32_t* __restrict__ free_pages,
    int32_t* __restrict__ n_free, int n_pages, int rows, int n_slots, int32_t* __restrict__ slots,
    int32_t* __restrict__ cu, int32_t* __restrict__ pos, int32_t* __restrict__ status, TabPlan plan) {
  __shared__ int lds[4][LDS ? kSpreadLds : 1];
  const int t = threadIdx.x, lane = t & 15;
  const int unit0 = blockIdx.x * 16 + (t >> 4), units = gridDim.x * 16;
  const long long x0 = (long long)blockIdx.x * 256 + t, xs = (long long)gridDim.x * 256;
  const int ok = plan.head[0], nf = plan.head[1], R = plan.rel[n_seqs], A = plan.alc[n_seqs];
  const bool hole = __any(plan.holes[t % kTabCheck]);
  if constexpr (LDS) {
    for (int s = t; s < n_seqs; s += 256) {
      lds[0][s] = plan.rel[s];
      lds[1][s] = plan.alc[s];
      lds[2][s] = old_len[s];
      lds[3][s] = new_len[s];
    }
    __syncthreads();
  }
  auto array = [&](int which, const int32_t* from) {
    if constexpr (LDS) return static_cast<const int*>(lds[which]);
    else return from;
  };
  const auto rel = array(0, plan.rel), alc = array(1, plan.alc), len0 = array(2, old_len), len1 = array(3, new_len);
  if (!ok || hole) {
    for (long long x = x0; x < n_slots; x += xs) slots[x] = -1;
    if (!hole) return;
    // refused after the plan was made
    for (long long s = x0; s < n_seqs; s += xs) {
      cu[s] = 0;
      pos[s] = old_len[s] - 1;
    }
    if (x0 == 0) {
      cu[n_seqs] = 0;
      *n_free = nf;
      *status = 2;
    }
    return;
  }
  for (int k = unit0; k < max(R, A); k += units) {
    int page;
    if (k < R) {
      const int s = last_at_most(rel, n_seqs, k);
      int32_t* entry = tables + (long long)s * b_max + blocks_of(len1[s], B) + (k - rel[s]);
      page = *entry;
      // every lane has the page before one of them clears the entry
      page = __shfl(page, t & 48);
      if (lane == 0) *entry = -1;
    } else {
      page = free_pages[nf - 1 - (k - R)];
    }
    if (k >= A) {
      if (lane == 0) free_pages[nf + R - 1 - k] = page;
      continue;
    }
    const int s = last_at_most(alc, n_seqs, k);
    const int o = len0[s], w = len1[s];
    const int j = blocks_of(o, B) + (k - alc[s]);
    if (lane == 0) tables[(long long)s * b_max + j] = page;
    const bool have = (unsigned)page < (unsigned)n_pages;
    const long long out = (rows > 0 ? (long long)s * rows : cu[s]) + ((long long)j * B - o);
    const int n = min(B, w - j * B);
    for (int i = lane; i < n; i += 16) slots[out + i] = have ? page * B + i : -1;
  }
  for (int s = unit0; s < n_seqs; s += units) {
    const int o = len0[s], w = len1[s];
    const long long out = rows > 0 ? (long long)s * rows : cu[s];
    const int end = (int)min((long long)w, (long long)blocks_of(o, B) * B);   // of the block it had
    if (o < end) {
      const int j = o / B;
      const int page = tables[(long long)s * b_max + j];
      const bool have = (unsigned)page < (unsigned)n_pages;
      for (int p = o + lane; p < end; p += 16) slots[out + p - o] = have ? page * B + (p - j * B) : -1;
    }
    for (int i = max(w - o, 0) + lane; i < rows; i += 16) slots[out + i] = -1;
  }
  if (rows == 0)
    for (long long x = cu[n_seqs] + x0; x < n_slots; x += xs) slots[x] = -1;
}

// Calls with few slots are one launch. (Many pages given back by such a call are
// moved by its one workgroup.)
constexpr long long kTabOneLaunch = 4 * kTabThreads;

int64_t block_tables_workspace_bytes(int n_seqs, int64_t n_slots) {
  return n_slots <= kTabOneLaunch ? 0 : 8ll * (n_seqs + 2) + 4 * kTabCheck;
}

hipError_t launch_block_tables(int n_seqs, int B, int b_max, const int32_t* old_len,
                               const int32_t* new_len, int32_t* tables, int32_t* free_pages,
                               int32_t* n_free, int n_pages, int rows, int n_slots, int32_t* slots,
                               int32_t* cu, int32_t* pos, int32_t* status, int32_t* ws, hipStream_t st) {
  if (n_slots <= kTabOneLaunch) {
    hipLaunchKernelGGL(block_tables_kernel<false>, dim3(1), dim3(kTabThreads), 0, st, n_seqs, B, b_max,
                       old_len, new_len, tables, free_pages, n_free, n_pages, rows, n_slots, slots, cu,
                       pos, status, TabPlan{});
    return hipGetLastError();
  }
  int32_t* head = ws + 2 * (n_seqs + 1);
  const TabPlan plan{ws, ws + n_seqs + 1, head, head + 2};
  hipLaunchKernelGGL(block_tables_kernel<true>, dim3(1 + kTabCheck), dim3(kTabThreads), 0, st, n_seqs, B, b_max,
                     old_len, new_len, tables, free_pages, n_free, n_pages, rows, n_slots, slots, cu, pos,
                     status, plan);
#define SW_SPREAD(LDS)                                                                             \
  hipLaunchKernelGGL(spread_kernel<LDS>, dim3(2048), dim3(256), 0, st, n_seqs, B, b_max, old_len,  \
                     new_len, tables, free_pages, n_free, n_pages, rows, n_slots, slots, cu, pos, status, plan)
  if (n_seqs <= kSpreadLds) SW_SPREAD(true); else SW_SPREAD(false);
#undef SW_SPREAD
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// tokens into the cache
// ---------------------------------------------------------------------------

// The part of a sequence's tokens that lies in one block. Workgroup w of
// floor(N / B) + 2 n_seqs finds its own: sequence s has the workgroups from
// cu[s] / B + 2 s on, which is enough for its floor(n / B) + 2 blocks at most
// however it lies in them, so no prefix of block counts is needed. Every wavefront
// searches for itself, 64 sequences at a time (one load for up to 64, no
// barrier). Returns the block's number in the sequence's stretch; c0, c1 are the
// stretch's tokens.
__device__ __forceinline__ long long seq_of_wg(int w, int n_seqs, const int32_t* cu, int B, int N,
                                               int* s_out, int* c0, int* c1) {
  const int l = threadIdx.x & 63;
  int lo = 0, n = n_seqs, a, b;                    // the last one that starts at or before w
  do {
    const int step = (n + 63) / 64, s = lo + l * step;
    const int at = min(s, n_seqs - 1);
    const int x = cu[at], y = cu[at + 1];
    const uint64_t in = __ballot(s < lo + n && x / B + 2ll * s <= w);
    const int k = in ? 63 - __builtin_clzll(in) : 0;
    a = __builtin_amdgcn_readlane(x, k);
    b = __builtin_amdgcn_readlane(y, k);
    n = min(step, n - k * step);
    lo += k * step;
  } while (n > 1);
  *s_out = lo;
  *c0 = max(a, 0);
  *c1 = min(b, N);
  return w - (*c0 / B + 2ll * lo);
}

// Tokens of a block that an append workgroup holds in registers at a time: 64 KB,
// or the whole block if it is smaller. A multiple of 16.
__host__ __device__ constexpr int q8_part(int B, int d, int size) {
  const int most = 65536 / (d * size);
  return B < most ? B : most;
}

typedef unsigned int u32x4f __attribute__((ext_vector_type(4)));
typedef unsigned short u16x2q __attribute__((ext_vector_type(2)));
typedef short s16x2q __attribute__((ext_vector_type(2)));

// The elements of a word of two bf16 or one fp32 as magnitudes, by their bits
// (which order as the numbers do; infinity and NaN come last).
template <typename T>
struct Q8Word;
template <>
struct Q8Word<uint16_t> {
  static constexpr uint32_t kInf = 0x7f80u;
  u16x2q m = {0, 0};
  __device__ void add(uint32_t w) {
    m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2q, w & 0x7fff7fffu));
  }
  __device__ uint32_t largest() const { return m[0] > m[1] ? m[0] : m[1]; }
  __device__ static float value(uint32_t bits) { return __uint_as_float(bits << 16); }
  // finite elements only; infinities become NaN in w
  __device__ void add_finite(uint32_t& w) {
#pragma unroll
    for (int h = 0; h < 32; h += 16) {
      const uint32_t x = w >> h & 0x7fffu;
      if (x < kInf) add(x);
      else w |= 0x40u << h;
    }
  }
  // codes of the word's elements / scale in one half of `old`
  template <bool HI>
  __device__ static uint32_t codes(uint32_t old, uint32_t w, uint32_t, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(
        __builtin_bit_cast(s16x2q, old), __builtin_bit_cast(bf16x2q, w), scale, HI));
  }
};
template <>
struct Q8Word<float> {
  static constexpr uint32_t kInf = 0x7f800000u;
  uint32_t m = 0;
  __device__ void add(uint32_t w) { m = max(m, w & 0x7fffffffu); }
  __device__ uint32_t largest() const { return m; }
  __device__ static float value(uint32_t bits) { return __uint_as_float(bits); }
  __device__ void add_finite(uint32_t& w) {
    const uint32_t x = w & 0x7fffffffu;
    if (x < kInf) add(x);
    else w |= 0x400000u;
  }
  // codes of two words
  template <bool HI>
  __device__ static uint32_t codes(uint32_t old, uint32_t w, uint32_t w2, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(
        __builtin_bit_cast(s16x2q, old), __uint_as_float(w), __uint_as_float(w2), scale, HI));
  }
};

// One workgroup per (block with new tokens, head, keys or values). SEQ: the
// block's tokens are a stretch of one sequence's. Otherwise a workgroup per token
// collects all tokens of its page and leaves the work to the first of them.
//   amax    over the new tokens' finite values, by their bits: not finite is the
//           largest, and only a block that has such a value looks at each
//   scale   of those alone if the block's first token is among them, else the
//           larger of the block's own and theirs; in the latter case the
//           block's codes are rounded again if the scale grew
//   codes   keys row by row; values four tokens of a dimension at a time into
//           LDS and from there, 16 tokens of a dimension in one store where all
//           of them are new
// A thread takes 16 bytes of each of four consecutive rows and keeps them from the
// maximum to the codes (blocks over 64 KB are read twice), so the workgroup's
// size goes by the block's: 1024 threads at 64 KB (256 threads with four such
// pieces each need 250 registers, which halves the wavefronts).
// live (without SEQ, may be NULL): pos of each token that goes into the cache, -1 of
// the others.
template <typename T, int D, bool SEQ>
__global__ __launch_bounds__(1024) void kv_append_q8_kernel(
    const T* __restrict__ k, const T* __restrict__ v, TokenStrides sd, int N, int n_seqs,
    const int32_t* __restrict__ cu, const int32_t* __restrict__ slots, int n_pages, int h_kv, int B,
    uint8_t* __restrict__ Kp, uint8_t* __restrict__ Vp, uint8_t* __restrict__ ks,
    uint8_t* __restrict__ vs, const int32_t* __restrict__ pos, int32_t* __restrict__ live) {
  using W = Q8Word<T>;
  constexpr int V = 16 / (int)sizeof(T);           // elements of a 16-byte piece
  constexpr int PIECES = D / V;                    // of a row
  __shared__ __attribute__((aligned(16))) int map[SEQ ? 1 : 1024];   // token of each place, -1: none
  __shared__ uint32_t red[16];
  __shared__ int leader;
  extern __shared__ __attribute__((aligned(16))) uint8_t tile[];     // [D][part + 4]
  const int t = threadIdx.x, nt = blockDim.x;
  // Heads run fastest over the workgroups: a token's keys and values, often parts
  // of one row, are then read at about the same time and over all memory
  // channels (five fp32 prompts of 47662 tokens in rows of 4 KB, four heads: 69 us, with the
  // blocks fastest 78).
  const int wg = blockIdx.x / (2 * h_kv), hd = blockIdx.x - wg * 2 * h_kv;
  const bool val = hd >= h_kv;                     // values, else keys
  const int g = val ? hd - h_kv : hd;
  int page, o0 = 0, o1 = B;                        // places that may be written
  int i0 = 0;                                      // SEQ: token of place o0
  if constexpr (SEQ) {
    int s, c0, c1;
    const long long j = seq_of_wg(wg, n_seqs, cu, B, N, &s, &c0, &c1);
    if (c0 >= c1 || j < 0) return;
    // token j B of the stretch, or its last, lies in block j if any does
    const int begin = slots[c0], slot = slots[(int)min(c0 + j * B, (long long)c1 - 1)];
    if (begin < 0 || slot < 0) return;
    const long long row0 = c0 + j * B - begin % B;  // token of the block's first place
    i0 = (int)max((long long)c0, row0);
    const int i1 = (int)min((long long)c1, row0 + B);
    if (i0 >= i1) return;
    page = slot / B;
    o0 = (int)(i0 - row0);
    o1 = o0 + i1 - i0;
  } else {
    const int mine = t < N ? slots[t] : -1;        // beside the load of the workgroup's own
    const int i = wg, slot = slots[i];
    page = slot / B;
    if (live && hd == 0 && blockIdx.z == 0 && t == 0) live[i] = slot >= 0 && page < n_pages ? pos[i] : -1;
    if (slot < 0) return;
    const int base = page * B;
    for (int o = t; o < B; o += nt) map[o] = -1;
    if (t == 0) leader = 1;
    __syncthreads();
    for (int x = t; x < N; x += nt) {
      const int o = (int)((uint32_t)(x == t ? mine : slots[x]) - (uint32_t)base);
      if ((unsigned)o >= (unsigned)B) continue;
      if (x < i) leader = 0;
      else atomicMax(&map[o], x);
    }
    __syncthreads();
    if (!leader) return;
  }
  if (page >= n_pages) return;

  const int part = q8_part(B, D, sizeof(T));
  const long long layer = blockIdx.z;
  const long long at = (layer * n_pages + page) * h_kv + g;
  uint8_t* scale = (val ? vs : ks) + at;
  const int e_old = (int)*scale - 127;
  const T* src = (val ? v + g * sd.v_head : k + g * sd.k_head) + layer * sd.layer;
  const long long tok = val ? sd.v_tok : sd.k_tok;
  auto token = [&](int o) {                        // token of a place, -1: none
    if constexpr (SEQ) return o >= o0 && o < o1 ? i0 + o - o0 : -1;
    else return map[o];
  };
  uint32_t raw[4][4];
  // rows p0 + 4 (t / PIECES) .. of the part from place p0 on, piece t % PIECES
  const int pc = t % PIECES, o = t / PIECES * 4;
  auto load = [&](int p0) {
    const int rows = min(part, B - p0);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int r = o < rows ? token(p0 + o + q) : -1;
      uint4 w = make_uint4(0, 0, 0, 0);
      if (r >= 0) w = *reinterpret_cast<const uint4*>(src + r * tok + pc * V);
      raw[q][0] = w.x;
      raw[q][1] = w.y;
      raw[q][2] = w.z;
      raw[q][3] = w.w;
    }
  };
  auto each = [&](auto&& f) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int y = 0; y < 4; ++y) f(raw[q][y]);
  };
  auto over_all = [&](uint32_t a) {                // the workgroup's largest
    for (int off = 32; off > 0; off >>= 1) a = max(a, (uint32_t)__shfl_xor((int)a, off));
    if ((t & 63) == 0) red[t >> 6] = a;
    __syncthreads();
    for (int w = 0; w < nt / 64; ++w) a = max(a, red[w]);
    return a;
  };
  W m;
  for (int p0 = 0; p0 < B; p0 += part) {
    load(p0);
    each([&](uint32_t w) { m.add(w); });
  }
  uint32_t top = over_all(m.largest());
  const bool odd = top >= W::kInf;                 // infinity or NaN among them
  if (odd) {
    W f;
    for (int p0 = 0; p0 < B; p0 += part) {
      if (part < B) load(p0);
      each([&](uint32_t& w) { f.add_finite(w); });
    }
    __syncthreads();                               // before red is written again
    top = over_all(f.largest());
  }
  const bool fresh = token(0) >= 0;
  const int e_new = q8_exponent(W::value(top));
  const int e = fresh ? e_new : max(e_new, e_old);
  if (t == 0) *scale = (uint8_t)(e + 127);
  uint8_t* out = (val ? Vp : Kp) + at * B * D;
  if (!fresh && e > e_old) {
    const float f = ldexpf(1.0f, e_old - e);
    uint4* c = reinterpret_cast<uint4*>(out);
    for (int i = t; i < B * D / 16; i += nt) {
      uint4 w = c[i];
      w.x = q8_rescale4(w.x, f);
      w.y = q8_rescale4(w.y, f);
      w.z = q8_rescale4(w.z, f);
      w.w = q8_rescale4(w.w, f);
      c[i] = w;
    }
    __syncthreads();                               // before the new codes go over them
  }
  const float sc = ldexpf(1.0f, e);
  for (int p0 = 0; p0 < B; p0 += part) {
    if (part < B) {
      load(p0);
      if (odd) {
        W f;
        each([&](uint32_t& w) { f.add_finite(w); });
      }
    }
    const int rows = min(part, B - p0);
    const int stride = part + 4;
    if (o < rows && !val) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (token(p0 + o + q) < 0) continue;
        const uint32_t (&w)[4] = raw[q];
        uint8_t* dst = out + (long long)(p0 + o + q) * D + pc * V;
        if constexpr (V == 8) {
          const uint32_t lo = W::template codes<true>(W::template codes<false>(0, w[0], 0, sc), w[1], 0, sc);
          const uint32_t hi = W::template codes<true>(W::template codes<false>(0, w[2], 0, sc), w[3], 0, sc);
          *reinterpret_cast<uint2*>(dst) = make_uint2(lo, hi);
        } else {
          *reinterpret_cast<uint32_t*>(dst) =
              W::template codes<true>(W::template codes<false>(0, w[0], w[1], sc), w[2], w[3], sc);
        }
      }
    }
    if (o < rows && val) {
      // dims 2 y and 2 y + 1 of the four rows: bytes 0 and 1 of each half
#pragma unroll
      for (int y = 0; y < V / 2; ++y) {
        auto two = [&](int q) { return V == 8 ? raw[q][y] : raw[q][2 * y % 4]; };
        auto next = [&](int q) { return V == 8 ? 0u : raw[q][(2 * y + 1) % 4]; };
        const uint32_t a = W::template codes<true>(W::template codes<false>(0, two(0), next(0), sc), two(1), next(1), sc);
        const uint32_t b = W::template codes<true>(W::template codes<false>(0, two(2), next(2), sc), two(3), next(3), sc);
        uint8_t* dst = tile + (pc * V + 2 * y) * stride + o;
        *reinterpret_cast<uint32_t*>(dst) = __builtin_amdgcn_perm(b, a, 0x06040200u);
        *reinterpret_cast<uint32_t*>(dst + stride) = __builtin_amdgcn_perm(b, a, 0x07050301u);
      }
    }
    if (!val) continue;
    __syncthreads();
    const int chunks = rows / 16;
    for (int x = t; x < D * chunks; x += nt) {
      const int dim = x / chunks, c = (x - dim * chunks) * 16, p = p0 + c;
      const uint32_t* s4 = reinterpret_cast<const uint32_t*>(tile + dim * stride + c);
      uint8_t* dst = out + (long long)dim * B + p;
      bool all = SEQ && p >= o0 && p + 16 <= o1;
      if (!SEQ) {
        all = true;
        for (int q = 0; q < 16; ++q) all &= token(p + q) >= 0;
      }
      if (all) {
        *reinterpret_cast<uint4*>(dst) = make_uint4(s4[0], s4[1], s4[2], s4[3]);
      } else {
        for (int q = 0; q < 16; ++q)
          if (token(p + q) >= 0) dst[q] = reinterpret_cast<const uint8_t*>(s4)[q];
      }
    }
    __syncthreads();
  }
}

// 64 bytes a thread, whole wavefronts.
static int append_threads(int dtype, int d, int B) {
  const int size = dtype == SW_BF16 ? 2 : 4;
  return (q8_part(B, d, size) * d * size / 64 + 63) / 64 * 64;
}

long long kv_append_q8_threads(int dtype, int64_t N, int n_seqs, bool by_seq, int h_kv, int d, int B) {
  return (by_seq ? N / B + 2ll * n_seqs : N) * 2 * h_kv * append_threads(dtype, d, B);
}

hipError_t launch_kv_append_q8(int dtype, int layers, const void* k, const void* v,
                               const TokenStrides& sd, int N, int n_seqs, const int32_t* cu,
                               const int32_t* slots, int n_pages, int h_kv, int d, int B, void* Kp,
                               void* Vp, uint8_t* ks, uint8_t* vs, const int32_t* pos, int32_t* live,
                               hipStream_t st) {
  const long long wgs = cu ? (long long)N / B + 2ll * n_seqs : N;
  const dim3 grid((unsigned)(wgs * 2 * h_kv), 1, (unsigned)layers);
  uint8_t* kp = static_cast<uint8_t*>(Kp);
  uint8_t* vp = static_cast<uint8_t*>(Vp);
  const int part = q8_part(B, d, dtype == SW_BF16 ? 2 : 4);
  const int threads = append_threads(dtype, d, B);
#define SW_APPEND_(T, D, SEQ)                                                                      \
  hipLaunchKernelGGL((kv_append_q8_kernel<T, D, SEQ>), grid, dim3((unsigned)threads),              \
                     (unsigned)(D * (part + 4)), st, static_cast<const T*>(k),                     \
                     static_cast<const T*>(v), sd, N, n_seqs, cu, slots, n_pages, h_kv, B, kp, vp, ks, vs, \
                     pos, live)
#define SW_APPEND(T)                                             \
  do {                                                           \
    if (d == 128) {                                              \
      if (cu) SW_APPEND_(T, 128, true); else SW_APPEND_(T, 128, false); \
    } else {                                                     \
      if (cu) SW_APPEND_(T, 64, true); else SW_APPEND_(T, 64, false); \
    }                                                            \
  } while (0)
  if (dtype == SW_BF16) SW_APPEND(uint16_t); else SW_APPEND(float);
#undef SW_APPEND_
#undef SW_APPEND
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// tokens out of the cache
// ---------------------------------------------------------------------------

constexpr int kFetchTile = 64;                     // positions per workgroup, four chunks of 16
static_assert(kFetchTile == 1 << 6, "positions are shifted");
constexpr int kFetchStride = kFetchTile + 4;       // bytes from one dimension's row to the next in LDS

// One workgroup per (64 positions of a sequence, head): positions first[s] ..
// first[s] + cu[s + 1] - cu[s] - 1 go to rows cu[s] .. of K, V [h_kv][N][d]. The
// positions are taken in chunks of 16, each in its own block whatever the block
// size. Values are exact in both types. A position without a page reads as zero.
// All loads go out first; the values' 4 x 4 byte squares are transposed in
// registers between LDS and the rows.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv_fetch_q8_kernel(
    const uint8_t* __restrict__ Kp, const uint8_t* __restrict__ Vp, const uint8_t* __restrict__ ks,
    const uint8_t* __restrict__ vs, int n_pages, int h_kv, int B, int n_seqs, int b_max,
    const int32_t* __restrict__ tables, const int32_t* __restrict__ first,
    const int32_t* __restrict__ cu, int N, T* __restrict__ K, T* __restrict__ V) {
  constexpr int E = 16 / (int)sizeof(T);           // values of a 16-byte store
  constexpr int KP = D / E;                        // stores of a row
  constexpr int NK = kFetchTile * KP / 256;        // keys' stores of a thread
  constexpr int NV = D * 4 / 256;                  // its loads of 16 values' tokens
  constexpr int NS = (KP * kFetchTile / 4 + 255) / 256;   // its blocks of E dims by four tokens
  static_assert(NK * 256 == kFetchTile * KP && NV * 256 == D * 4, "whole pieces per thread");
  __shared__ __attribute__((aligned(16))) uint8_t tile[D * kFetchStride];
  __shared__ long long at4[4];
  __shared__ int off4[4];
  const int t = threadIdx.x, g = blockIdx.y;
  // Neighbouring tiles go to workgroups 8 apart, which run on one XCD: in blocks of
  // 128 and more they share the 128-byte lines of the values' rows.
  int wg = blockIdx.x;
  if (wg < (int)(gridDim.x & ~15u)) wg = (wg & ~15) + (wg & 7) * 2 + (wg >> 3 & 1);
  int s, c0, c1;
  const long long u = seq_of_wg(wg, n_seqs, cu, kFetchTile, N, &s, &c0, &c1);
  if (c0 >= c1 || u < 0) return;
  const int p0 = first ? first[s] : 0;
  const long long pt = ((p0 >> 6) + u) * kFetchTile;   // the tile's first position (p0 may be negative)
  // places lo .. hi - 1 of the tile are asked for; place o is row row0 + o
  const long long row0 = c0 + pt - p0;
  const int lo = (int)max(0ll, c0 - row0), hi = (int)min((long long)kFetchTile, c1 - row0);
  if (lo >= hi) return;
  // page and head of each chunk (-1 without a page) and its place in the page
  if (t < 4) {
    // a negative position is 2^31 or more here, behind every table
    const uint32_t p = (uint32_t)pt + 16 * t, j = p / (uint32_t)B;
    const int page = j < (uint32_t)b_max && pt < (1ll << 31) ? tables[(long long)s * b_max + j] : -1;
    at4[t] = (unsigned)page < (unsigned)n_pages ? (long long)page * h_kv + g : -1ll;
    off4[t] = (int)(p - j * B);
  }
  __syncthreads();
  uint32_t kr[NK][E / 4];
  float kf[NK];
#pragma unroll
  for (int i = 0; i < NK; ++i) {
    const int x = t + 256 * i, o = x / KP, pc = x % KP;
    const long long at = o >= lo && o < hi ? at4[o / 16] : -1;
    kf[i] = 0.0f;
    uint32_t w[2] = {0, 0};
    if (at >= 0) {
      const uint8_t* from = Kp + (at * B + off4[o / 16] + o % 16) * D + pc * E;
      if constexpr (E == 8) {
        const uint2 y = *reinterpret_cast<const uint2*>(from);
        w[0] = y.x;
        w[1] = y.y;
      } else {
        w[0] = *reinterpret_cast<const uint32_t*>(from);
      }
      kf[i] = q8_scale(ks[at]);
    }
#pragma unroll
    for (int e = 0; e < E / 4; ++e) kr[i][e] = w[e];
  }
  u32x4f vr[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int x = t + 256 * i, dim = x / 4, c = x % 4;
    const long long at = 16 * c < hi && 16 * c + 16 > lo ? at4[c] : -1;
    vr[i] = u32x4f{0, 0, 0, 0};
    if (at >= 0) vr[i] = *reinterpret_cast<const u32x4f*>(Vp + (at * D + dim) * B + off4[c]);
  }
  // scales of the values that this thread writes out below: dims E dq .., tokens
  // 4 (t / KP + 256 / KP i) ..
  const int dq = t % KP;
  float vf[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    const int o = (t / KP + 256 / KP * i) * 4;
    const long long at = o < hi && o + 4 > lo ? at4[o / 16] : -1;
    vf[i] = at >= 0 ? q8_scale(vs[at]) : 0.0f;
  }
  T* Kd = K + ((long long)g * N + row0) * D;
  T* Vd = V + ((long long)g * N + row0) * D;
  auto put = [&](T* dst, const uint32_t* w, float f) {   // E values
    f32x2q a[E / 2];
#pragma unroll
    for (int e = 0; e < E / 4; ++e) {
      a[2 * e] = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[e], false);
      a[2 * e + 1] = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[e], true);
    }
    // as a stream: written over the caches they would put out what is still to be
    // read (32768 tokens to bf16 44 -> 31 us, the pages then partly cached)
    u32x4f out;
    if constexpr (E == 8) {
#pragma unroll
      for (int e = 0; e < 4; ++e) out[e] = pack_bf16x2(a[e][0] * f, a[e][1] * f);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) out[e] = __float_as_uint(a[e / 2][e % 2] * f);
    }
    __builtin_nontemporal_store(out, reinterpret_cast<u32x4f*>(dst));
  };
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int x = t + 256 * i, dim = x / 4, o = x % 4 * 16;
    uint32_t* to = reinterpret_cast<uint32_t*>(tile + dim * kFetchStride + o);
#pragma unroll
    for (int e = 0; e < 4; ++e) to[e] = vr[i][e];
  }
#pragma unroll
  for (int i = 0; i < NK; ++i) {
    const int x = t + 256 * i, o = x / KP, pc = x % KP;
    if (o >= lo && o < hi) put(Kd + (long long)o * D + pc * E, kr[i], kf[i]);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    const int o = (t / KP + 256 / KP * i) * 4;
    if (o >= kFetchTile) break;
    uint32_t w[4][E / 4];                          // four tokens' codes
#pragma unroll
    for (int e = 0; e < E / 4; ++e) {
      uint32_t r[4];                               // dim E dq + 4 e + y, four tokens
#pragma unroll
      for (int y = 0; y < 4; ++y)
        r[y] = *reinterpret_cast<const uint32_t*>(tile + (E * dq + 4 * e + y) * kFetchStride + o);
      const uint32_t a0 = __builtin_amdgcn_perm(r[1], r[0], 0x05010400u);   // tokens 0 and 1 of dims 0, 1
      const uint32_t a1 = __builtin_amdgcn_perm(r[1], r[0], 0x07030602u);   // tokens 2 and 3
      const uint32_t b0 = __builtin_amdgcn_perm(r[3], r[2], 0x05010400u);
      const uint32_t b1 = __builtin_amdgcn_perm(r[3], r[2], 0x07030602u);
      w[0][e] = __builtin_amdgcn_perm(b0, a0, 0x05040100u);
      w[1][e] = __builtin_amdgcn_perm(b0, a0, 0x07060302u);
      w[2][e] = __builtin_amdgcn_perm(b1, a1, 0x05040100u);
      w[3][e] = __builtin_amdgcn_perm(b1, a1, 0x07060302u);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (o + q >= lo && o + q < hi) put(Vd + (long long)(o + q) * D + E * dq, w[q], vf[i]);
  }
}

hipError_t launch_kv_fetch_q8(int dtype, const void* Kp, const void* Vp, const uint8_t* ks,
                              const uint8_t* vs, int n_pages, int h_kv, int d, int B, int n_seqs,
                              int b_max, const int32_t* tables, const int32_t* first, const int32_t* cu,
                              int N, void* K, void* V, hipStream_t st) {
  const dim3 grid((unsigned)(N / kFetchTile + 2ll * n_seqs), (unsigned)h_kv);
  const uint8_t* kp = static_cast<const uint8_t*>(Kp);
  const uint8_t* vp = static_cast<const uint8_t*>(Vp);
#define SW_FETCH(T, D)                                                                          \
  hipLaunchKernelGGL((kv_fetch_q8_kernel<T, D>), grid, dim3(256), 0, st, kp, vp, ks, vs, n_pages, \
                     h_kv, B, n_seqs, b_max, tables, first, cu, N, static_cast<T*>(K), static_cast<T*>(V))
  if (dtype == SW_BF16) {
    if (d == 128) SW_FETCH(uint16_t, 128); else SW_FETCH(uint16_t, 64);
  } else {
    if (d == 128) SW_FETCH(float, 128); else SW_FETCH(float, 64);
  }
#undef SW_FETCH
  return hipGetLastError();
}

}  // namespace sw
