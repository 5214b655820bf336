// The paged 8-bit key/value cache: pages from the requests' lengths, tokens in,
// tokens out.
//
//  block_tables_kernel  pages of requests that end back onto the free stack,
//                       pages for new blocks off it, the new tokens' slots
//  slots_kernel         the slots alone, for calls with many of them
//  kv_append_q8_kernel  new tokens into the pages their slots name
//  kv_fetch_q8_kernel   tokens of the cache back as bf16 or fp32
#include <type_traits>

#include "q8.h"
#include "sw_common.h"
#include "sw_internal.h"

namespace sw {

// ---------------------------------------------------------------------------
// block tables and slots
// ---------------------------------------------------------------------------

constexpr int kTabThreads = 1024;

// Exclusive prefix of v over the workgroup, the sum in *total (two barriers).
__device__ __forceinline__ int tab_scan(int v, int* tmp, int* total) {
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  const int x = wave_inclusive_scan(v);
  if (lane == 63) tmp[w] = x;
  __syncthreads();
  int before = 0, sum = 0;
#pragma unroll
  for (int q = 0; q < kTabThreads / 64; ++q) {
    before += q < w ? tmp[q] : 0;
    sum += tmp[q];
  }
  *total = sum;
  __syncthreads();
  return before + x - v;
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

// One workgroup. In order: every length is checked and the pages to give back
// (R) and to take (A) are counted; then, if the call can be served whole, the
// R released pages go onto the stack so that the first of them (sequences
// ascending, blocks ascending) is on top, and the A new blocks take pages from
// the top in the same order. Bounded by latency: four dependent loads and a
// dozen barriers.
__global__ __launch_bounds__(kTabThreads) void block_tables_kernel(
    int n_seqs, int B, int b_max, const int32_t* __restrict__ old_len,
    const int32_t* __restrict__ new_len, int32_t* __restrict__ tables, int32_t* __restrict__ free_pages,
    int32_t* __restrict__ n_free, int n_pages, int rows, int n_slots, int slots_here,
    int32_t* __restrict__ slots, int32_t* __restrict__ cu, int32_t* __restrict__ pos,
    int32_t* __restrict__ status) {
  __shared__ int tmp[kTabThreads / 64];
  __shared__ int pre[kTabThreads], first[kTabThreads];
  __shared__ long long sums[3];
  __shared__ int bad;
  const int t = threadIdx.x;
  const long long top_len = (long long)b_max * B;
  if (t < 3) sums[t] = 0;
  if (t == 0) bad = 0;
  __syncthreads();
  const int nf = *n_free;
  {
    long long R = 0, A = 0, grow = 0;
    bool wrong = false;
    for (int s = t; s < n_seqs; s += kTabThreads) {
      const int o = old_len[s], w = new_len[s];
      wrong |= o < 0 || o > top_len || w < 0 || w > top_len;
      const int has = (int)((o + (long long)B - 1) / B), need = (int)((w + (long long)B - 1) / B);
      R += max(has - need, 0);
      A += max(need - has, 0);
      grow += max((long long)w - o, 0ll);
      wrong |= rows > 0 && (long long)w - o > rows;
    }
    if (wrong) bad = 1;
    if (R) atomicAdd((unsigned long long*)&sums[0], (unsigned long long)R);
    if (A) atomicAdd((unsigned long long*)&sums[1], (unsigned long long)A);
    if (grow) atomicAdd((unsigned long long*)&sums[2], (unsigned long long)grow);
  }
  __syncthreads();
  const long long R = sums[0], A = sums[1];
  const bool valid = !bad && nf >= 0 && nf + R <= n_pages && (rows > 0 || sums[2] <= n_slots);
  const bool ok = valid && A - R <= nf;
  const int top = nf + (int)R;                     // of the stack, after the releases
  if (t == 0) *status = valid ? (ok ? 0 : 1) : 2;

  int done_r = 0, done_a = 0, done_g = 0;
  for (int phase = 0; phase < 2 && ok; ++phase) {
    // 0: releases; 1: allocations
    if (phase == 0 ? R == 0 : A == 0) continue;
    for (int s0 = 0; s0 < n_seqs; s0 += kTabThreads) {
      const int s = s0 + t;
      int has = 0, need = 0;
      if (s < n_seqs) {
        has = (int)((old_len[s] + (long long)B - 1) / B);
        need = (int)((new_len[s] + (long long)B - 1) / B);
      }
      int total;
      const int k0 = tab_scan(phase == 0 ? max(has - need, 0) : max(need - has, 0), tmp, &total);
      pre[t] = k0;
      first[t] = phase == 0 ? need : has;
      __syncthreads();
      const int base = phase == 0 ? done_r : done_a;
      for (int k = t; k < total; k += kTabThreads) {
        const int i = last_at_most(pre, kTabThreads, k);
        int32_t* entry = tables + (long long)(s0 + i) * b_max + first[i] + (k - pre[i]);
        int32_t* item = free_pages + (top - 1 - (base + k));
        if (phase == 0) {
          *item = *entry;
          *entry = -1;
        } else {
          *entry = *item;
        }
      }
      if (phase == 0) done_r += total; else done_a += total;
      __syncthreads();
    }
  }
  if (t == 0 && ok) *n_free = top - (int)A;
  // cumulative new tokens, positions of the last ones
  for (int s0 = 0; s0 < n_seqs; s0 += kTabThreads) {
    const int s = s0 + t;
    const int o = s < n_seqs ? old_len[s] : 0, w = s < n_seqs ? new_len[s] : 0;
    int total;
    const int g0 = tab_scan(ok ? max(w - o, 0) : 0, tmp, &total);
    if (s < n_seqs) {
      cu[s] = done_g + g0;
      pos[s] = (ok ? w : o) - 1;
    }
    done_g += total;
  }
  if (t == 0) cu[n_seqs] = done_g;
  if (!slots_here) return;
  __syncthreads();                                 // tables and cu as written above
  for (int x = t; x < n_slots; x += kTabThreads) {
    int v = -1;
    if (rows > 0) {
      const int s = x / rows, i = x - s * rows;
      const int o = old_len[s];
      if (ok && i < new_len[s] - o) v = slot_of(tables + (long long)s * b_max, o + i, B, n_pages);
    } else if (x < done_g) {
      const int s = last_at_most(cu, n_seqs, x);
      v = slot_of(tables + (long long)s * b_max, old_len[s] + (x - cu[s]), B, n_pages);
    }
    slots[x] = v;
  }
}

// Slots of calls with many new tokens: thread x takes four of them.
__global__ __launch_bounds__(256) void slots_kernel(int n_seqs, int B, int b_max,
                                                    const int32_t* __restrict__ old_len,
                                                    const int32_t* __restrict__ new_len,
                                                    const int32_t* __restrict__ tables, int n_pages,
                                                    int rows, int n_slots, const int32_t* __restrict__ cu,
                                                    const int32_t* __restrict__ status,
                                                    int32_t* __restrict__ slots) {
  const bool ok = *status == 0;
  const int total = cu[n_seqs];
  for (int e = 0; e < 4; ++e) {
    const long long x = ((long long)blockIdx.x * 256 + threadIdx.x) * 4 + e;
    if (x >= n_slots) return;
    int v = -1;
    if (rows > 0) {
      const int s = (int)(x / rows), i = (int)(x - (long long)s * rows);
      const int o = old_len[s];
      if (ok && i < new_len[s] - o) v = slot_of(tables + (long long)s * b_max, o + i, B, n_pages);
    } else if (x < total) {
      const int s = last_at_most(cu, n_seqs, (int)x);
      v = slot_of(tables + (long long)s * b_max, old_len[s] + ((int)x - cu[s]), B, n_pages);
    }
    slots[x] = v;
  }
}

hipError_t launch_block_tables(int n_seqs, int B, int b_max, const int32_t* old_len,
                               const int32_t* new_len, int32_t* tables, int32_t* free_pages,
                               int32_t* n_free, int n_pages, int rows, int n_slots, int32_t* slots,
                               int32_t* cu, int32_t* pos, int32_t* status, hipStream_t st) {
  const int here = n_slots <= 8 * kTabThreads;
  hipLaunchKernelGGL(block_tables_kernel, dim3(1), dim3(kTabThreads), 0, st, n_seqs, B, b_max, old_len,
                     new_len, tables, free_pages, n_free, n_pages, rows, n_slots, here, slots, cu, pos,
                     status);
  if (!here)
    hipLaunchKernelGGL(slots_kernel, dim3((unsigned)((n_slots + 1023ll) / 1024)), dim3(256), 0, st,
                       n_seqs, B, b_max, old_len, new_len, tables, n_pages, rows, n_slots, cu, status,
                       slots);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// tokens into the cache
// ---------------------------------------------------------------------------

template <typename T>
__device__ __forceinline__ float q8_load(const T* p) {
  if constexpr (sizeof(T) == 2)
    return bf16_to_f32(*p);
  else
    return *p;
}

// The part of a sequence's tokens that lies in one block. Workgroup w of
// floor(N / B) + 2 n_seqs finds its own: sequence s has the workgroups from
// cu[s] / B + 2 s on, which is enough for its floor(n / B) + 2 blocks at most
// however it lies in them, so no prefix of block counts is needed.
__device__ __forceinline__ int seq_of_wg(int w, int n_seqs, const int32_t* cu, int B) {
  int count = 0;
  for (int s0 = 0; s0 < n_seqs; s0 += 256) {
    const int s = s0 + threadIdx.x;
    const int c = __syncthreads_count(s < n_seqs && (long long)cu[min(s, n_seqs)] / B + 2ll * s <= w);
    count += c;
    if (c < 256) break;
  }
  return max(count - 1, 0);
}

constexpr int kQ8Tile = 64;                        // tokens transposed at a time
constexpr int kQ8Stride = kQ8Tile + 4;             // bytes from one dimension's row to the next

// One workgroup per (block with new tokens, head). With cu the block's tokens
// are a stretch of one sequence's; without, a workgroup per token collects all
// tokens of its page and leaves the work to the first of them.
//   amax    over the new tokens' finite values, K and V apart
//   scale   of those alone if the block's first token is among them, else the
//           larger of the block's own and theirs; in the latter case the
//           block's codes are rounded again if the scale grew
//   codes   K rows as they are, V through LDS: 16 tokens of a dimension are one
//           16-byte store where all of them are new
template <typename T>
__global__ __launch_bounds__(256) void kv_append_q8_kernel(
    const T* __restrict__ k, const T* __restrict__ v, TokenStrides sd, int N, int n_seqs,
    const int32_t* __restrict__ cu, const int32_t* __restrict__ slots, int n_pages, int h_kv, int d,
    int B, uint8_t* __restrict__ Kp, uint8_t* __restrict__ Vp, uint8_t* __restrict__ ks,
    uint8_t* __restrict__ vs) {
  __shared__ int map[1024];                        // token of each place in the block, -1: none
  __shared__ float red[2][4];
  __shared__ __attribute__((aligned(16))) uint8_t tile[256 * kQ8Stride];
  __shared__ int leader;
  const int t = threadIdx.x, g = blockIdx.y;
  const long long layer = blockIdx.z;
  k += layer * sd.layer;
  v += layer * sd.layer;
  const long long pool = (long long)n_pages * h_kv;
  Kp += layer * pool * B * d;
  Vp += layer * pool * B * d;
  ks += layer * pool;
  vs += layer * pool;
  int i0, i1, slot;
  if (cu) {
    const int s = seq_of_wg(blockIdx.x, n_seqs, cu, B);
    const int c0 = max(cu[s], 0), c1 = min(cu[s + 1], N);
    if (c0 >= c1) return;
    const int begin = slots[c0];
    if (begin < 0) return;
    const long long j = blockIdx.x - (c0 / B + 2ll * s);
    const long long lo = c0 + j * B - begin % B;
    i0 = (int)max((long long)c0, lo);
    i1 = (int)min((long long)c1, lo + B);
    if (i0 >= i1) return;
    slot = slots[i0];
  } else {
    i0 = blockIdx.x;
    i1 = N;
    slot = slots[i0];
  }
  if (slot < 0) return;
  const int page = slot / B, base = page * B;
  if (page >= n_pages) return;
  for (int o = t; o < B; o += 256) map[o] = -1;
  if (t == 0) leader = 1;
  __syncthreads();
  if (!cu) {
    for (int i = t; i < i0; i += 256)
      if ((unsigned)(slots[i] - base) < (unsigned)B) leader = 0;
  }
  for (int i = i0 + t; i < i1; i += 256) {
    const int o = slots[i] - base;
    if ((unsigned)o < (unsigned)B) atomicMax(&map[o], i);
  }
  __syncthreads();
  if (!leader) return;

  constexpr int V = 16 / (int)sizeof(T);           // elements of a 16-byte piece
  const int pieces = d / V;                        // of a row
  const int per = 256 / pieces;                    // rows at a time
  const int pc = t % pieces, row0 = t / pieces;
  const T* kg = k + g * sd.k_head + pc * V;
  const T* vg = v + g * sd.v_head + pc * V;
  float ka = 0.0f, va = 0.0f;
  if (row0 < per)
    for (int o = row0; o < B; o += per) {
      const int i = map[o];
      if (i < 0) continue;
      const uint4 a = *reinterpret_cast<const uint4*>(kg + i * sd.k_tok);
      const uint4 b = *reinterpret_cast<const uint4*>(vg + i * sd.v_tok);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        ka = fmaxf(ka, q8_finite_abs(q8_load(reinterpret_cast<const T*>(&a) + e)));
        va = fmaxf(va, q8_finite_abs(q8_load(reinterpret_cast<const T*>(&b) + e)));
      }
    }
  for (int off = 32; off > 0; off >>= 1) {
    ka = fmaxf(ka, __shfl_xor(ka, off));
    va = fmaxf(va, __shfl_xor(va, off));
  }
  if ((t & 63) == 0) {
    red[0][t >> 6] = ka;
    red[1][t >> 6] = va;
  }
  __syncthreads();
  const long long at = (long long)page * h_kv + g;
  const bool fresh = map[0] >= 0;
  int e[2], grew[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const float m = fmaxf(fmaxf(red[x][0], red[x][1]), fmaxf(red[x][2], red[x][3]));
    const int e_old = (int)(x ? vs : ks)[at] - 127;
    const int e_new = q8_exponent(m);
    e[x] = fresh ? e_new : max(e_new, e_old);
    grew[x] = fresh ? 0 : e[x] - e_old;
  }
  __syncthreads();                                 // the old scales are read
  if (t == 0) {
    ks[at] = (uint8_t)(e[0] + 127);
    vs[at] = (uint8_t)(e[1] + 127);
  }
  uint8_t* Kb = Kp + at * B * d;
  uint8_t* Vb = Vp + at * B * d;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    if (grew[x] == 0) continue;
    const float m = ldexpf(1.0f, -grew[x]);
    uint4* c = reinterpret_cast<uint4*>(x ? Vb : Kb);
    for (int i = t; i < B * d / 16; i += 256) {
      uint4 w = c[i];
      w.x = q8_rescale4(w.x, m);
      w.y = q8_rescale4(w.y, m);
      w.z = q8_rescale4(w.z, m);
      w.w = q8_rescale4(w.w, m);
      c[i] = w;
    }
  }
  __syncthreads();                                 // before the new codes go over them
  const float ki = ldexpf(1.0f, -e[0]), vi = ldexpf(1.0f, -e[1]);
  for (int o0 = 0; o0 < B; o0 += kQ8Tile) {
    const int oe = min(o0 + kQ8Tile, B);
    if (row0 < per)
      for (int o = o0 + row0; o < oe; o += per) {
        const int i = map[o];
        if (i < 0) continue;
        const uint4 a = *reinterpret_cast<const uint4*>(kg + i * sd.k_tok);
        const uint4 b = *reinterpret_cast<const uint4*>(vg + i * sd.v_tok);
        const T* pa = reinterpret_cast<const T*>(&a);
        const T* pb = reinterpret_cast<const T*>(&b);
        uint32_t kw[V / 4];
#pragma unroll
        for (int x = 0; x < V; x += 4)
          kw[x / 4] = q8_pack2(q8_load(pa + x), q8_load(pa + x + 1), ki) |
                      q8_pack2(q8_load(pa + x + 2), q8_load(pa + x + 3), ki) << 16;
        uint32_t* kd = reinterpret_cast<uint32_t*>(Kb + (long long)o * d + pc * V);
#pragma unroll
        for (int x = 0; x < V / 4; ++x) kd[x] = kw[x];
#pragma unroll
        for (int x = 0; x < V; x += 2) {
          const uint32_t w = q8_pack2(q8_load(pb + x), q8_load(pb + x + 1), vi);
          tile[(pc * V + x) * kQ8Stride + o - o0] = (uint8_t)w;
          tile[(pc * V + x + 1) * kQ8Stride + o - o0] = (uint8_t)(w >> 8);
        }
      }
    __syncthreads();
    const int chunks = (oe - o0) / 16;             // B is a multiple of 16
    for (int x = t; x < d * chunks; x += 256) {
      const int dim = x / chunks, o = (x - dim * chunks) * 16;
      uint32_t have = 0;
      for (int q = 0; q < 16; ++q) have |= (uint32_t)(map[o0 + o + q] >= 0) << q;
      const uint8_t* src = tile + dim * kQ8Stride + o;
      uint8_t* dst = Vb + (long long)dim * B + o0 + o;
      if (have == 0xffffu) {
        const uint32_t* s4 = reinterpret_cast<const uint32_t*>(src);
        *reinterpret_cast<uint4*>(dst) = make_uint4(s4[0], s4[1], s4[2], s4[3]);
      } else if (have) {
        for (int q = 0; q < 16; ++q)
          if (have >> q & 1) dst[q] = src[q];
      }
    }
    __syncthreads();
  }
}

hipError_t launch_kv_append_q8(int dtype, int layers, const void* k, const void* v,
                               const TokenStrides& sd, int N, int n_seqs, const int32_t* cu,
                               const int32_t* slots, int n_pages, int h_kv, int d, int B, void* Kp,
                               void* Vp, uint8_t* ks, uint8_t* vs, hipStream_t st) {
  const long long wgs = cu ? (long long)N / B + 2ll * n_seqs : N;
  const dim3 grid((unsigned)wgs, (unsigned)h_kv, (unsigned)layers);
  if (dtype == SW_BF16)
    hipLaunchKernelGGL(kv_append_q8_kernel<uint16_t>, grid, dim3(256), 0, st,
                       static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v), sd, N, n_seqs,
                       cu, slots, n_pages, h_kv, d, B, static_cast<uint8_t*>(Kp),
                       static_cast<uint8_t*>(Vp), ks, vs);
  else
    hipLaunchKernelGGL(kv_append_q8_kernel<float>, grid, dim3(256), 0, st, static_cast<const float*>(k),
                       static_cast<const float*>(v), sd, N, n_seqs, cu, slots, n_pages, h_kv, d, B,
                       static_cast<uint8_t*>(Kp), static_cast<uint8_t*>(Vp), ks, vs);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// tokens out of the cache
// ---------------------------------------------------------------------------

// One workgroup per (block of a sequence's stretch, head): positions first[s]
// .. first[s] + cu[s + 1] - cu[s] - 1 go to rows cu[s] .. of K, V [h_kv][N][d].
// Values are exact in both types. A position without a page reads as zero.
template <typename T>
__global__ __launch_bounds__(256) void kv_fetch_q8_kernel(
    const uint8_t* __restrict__ Kp, const uint8_t* __restrict__ Vp, const uint8_t* __restrict__ ks,
    const uint8_t* __restrict__ vs, int n_pages, int h_kv, int d, int B, int n_seqs, int b_max,
    const int32_t* __restrict__ tables, const int32_t* __restrict__ first,
    const int32_t* __restrict__ cu, int N, T* __restrict__ K, T* __restrict__ V) {
  __shared__ __attribute__((aligned(16))) uint8_t tile[256 * kQ8Stride];
  const int t = threadIdx.x, g = blockIdx.y;
  const int s = seq_of_wg(blockIdx.x, n_seqs, cu, B);
  const int c0 = max(cu[s], 0), c1 = min(cu[s + 1], N);
  if (c0 >= c1) return;
  const int p0 = first ? max(first[s], 0) : 0;
  const long long j = blockIdx.x - (c0 / B + 2ll * s);
  const long long blk = p0 / B + j;
  // places lo .. hi - 1 of the block; place o is row row0 + o
  const long long row0 = c0 + blk * B - p0;
  const int lo = (int)max(0ll, c0 - row0), hi = (int)min((long long)B, c1 - row0);
  if (lo >= hi) return;
  const int page = blk < b_max ? tables[(long long)s * b_max + blk] : -1;
  const bool have = (unsigned)page < (unsigned)n_pages;
  const long long at = have ? (long long)page * h_kv + g : 0;
  const float kf = q8_scale(ks[at]), vf = q8_scale(vs[at]);
  const uint8_t* Kb = Kp + at * B * d;
  const uint8_t* Vb = Vp + at * B * d;
  T* Kd = K + ((long long)g * N + row0) * d;
  T* Vd = V + ((long long)g * N + row0) * d;
  auto put = [&](T* dst, uint32_t w, float f) {    // four values
    const f32x2q a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
    const f32x2q b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    if constexpr (sizeof(T) == 2)
      *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(a[0] * f, a[1] * f), pack_bf16x2(b[0] * f, b[1] * f));
    else
      *reinterpret_cast<float4*>(dst) = make_float4(a[0] * f, a[1] * f, b[0] * f, b[1] * f);
  };
  const int words = d / 4;                         // of a row
  for (int x = t; x < (hi - lo) * words; x += 256) {
    const int o = lo + x / words, c = x % words;
    const uint32_t w = have ? *reinterpret_cast<const uint32_t*>(Kb + (long long)o * d + 4 * c) : 0;
    put(Kd + (long long)o * d + 4 * c, w, kf);
  }
  for (int o0 = lo / kQ8Tile * kQ8Tile; o0 < hi; o0 += kQ8Tile) {
    const int chunks = (min(o0 + kQ8Tile, B) - o0) / 16;
    for (int x = t; x < d * chunks; x += 256) {
      const int dim = x / chunks, o = (x - dim * chunks) * 16;
      const uint4 w = have ? *reinterpret_cast<const uint4*>(Vb + (long long)dim * B + o0 + o)
                           : make_uint4(0, 0, 0, 0);
      uint32_t* to = reinterpret_cast<uint32_t*>(tile + dim * kQ8Stride + o);
      to[0] = w.x;
      to[1] = w.y;
      to[2] = w.z;
      to[3] = w.w;
    }
    __syncthreads();
    const int a = max(lo, o0), b = min(hi, o0 + kQ8Tile);
    for (int x = t; x < (b - a) * words; x += 256) {
      const int o = a + x / words, c = x % words;
      const uint8_t* from = tile + 4 * c * kQ8Stride + o - o0;
      const uint32_t w = from[0] | (uint32_t)from[kQ8Stride] << 8 | (uint32_t)from[2 * kQ8Stride] << 16 |
                         (uint32_t)from[3 * kQ8Stride] << 24;
      put(Vd + (long long)o * d + 4 * c, w, vf);
    }
    __syncthreads();
  }
}

hipError_t launch_kv_fetch_q8(int dtype, const void* Kp, const void* Vp, const uint8_t* ks,
                              const uint8_t* vs, int n_pages, int h_kv, int d, int B, int n_seqs,
                              int b_max, const int32_t* tables, const int32_t* first, const int32_t* cu,
                              int N, void* K, void* V, hipStream_t st) {
  const dim3 grid((unsigned)(N / B + 2ll * n_seqs), (unsigned)h_kv);
  const uint8_t* kp = static_cast<const uint8_t*>(Kp);
  const uint8_t* vp = static_cast<const uint8_t*>(Vp);
  if (dtype == SW_BF16)
    hipLaunchKernelGGL(kv_fetch_q8_kernel<uint16_t>, grid, dim3(256), 0, st, kp, vp, ks, vs, n_pages,
                       h_kv, d, B, n_seqs, b_max, tables, first, cu, N, static_cast<uint16_t*>(K),
                       static_cast<uint16_t*>(V));
  else
    hipLaunchKernelGGL(kv_fetch_q8_kernel<float>, grid, dim3(256), 0, st, kp, vp, ks, vs, n_pages, h_kv,
                       d, B, n_seqs, b_max, tables, first, cu, N, static_cast<float*>(K),
                       static_cast<float*>(V));
  return hipGetLastError();
}

}  // namespace sw
