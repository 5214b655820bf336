// Decode attention over the paged 8-bit cache (paper Alg. 2 step 7 with K and V
// as e4m3 codes): softmax attention of one token per sequence over the tokens
// of the selected key blocks, split-K over those tokens.
#include <climits>

#include "q8.h"
#include "sw_common.h"
#include "sw_internal.h"

namespace sw {

typedef __bf16 bf16x8q __attribute__((ext_vector_type(8)));
typedef float f32x4q __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4q __attribute__((ext_vector_type(4)));

constexpr float kLog2eQ = 1.4426950408889634f;

__device__ __forceinline__ float q8_xmax(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float q8_xsum(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Eight codes as the operand of a bf16 matrix instruction (exact).
__device__ __forceinline__ bf16x8q q8_bf16x8(uint32_t lo, uint32_t hi) {
  const bf16x2q a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
  const bf16x2q b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
  const bf16x2q c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
  const bf16x2q d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  return bf16x8q{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

constexpr int kQ8Chunks = 1024;                    // 16-token chunks listed at a time

// A listed chunk: byte offset of its (page, head) in the pools, its first token
// (INT_MAX: none of it counts), its place in the page, and the block's scales.
struct Q8Chunk {
  long long page;
  int t0, off;
  float ks, vs;
};

// Workgroup = (sequence, KV head, split), four wavefronts; a wavefront takes
// groups of 64 selected tokens, four chunks of 16, whichever blocks they are in.
//   S = K q^T      v_mfma_f32_16x16x32_bf16: row m of the x-th product is token
//                  4 x + m % 4 of chunk m / 4, so lane (n, lg) receives 16
//                  tokens of head n, all of chunk lg: its scale, its first token
//                  and its weights are the lane's own.
//   O^T += V^T P^T the same instruction: k = 8 lg + i of product y is token
//                  8 y + i of chunk lg, that is the lane's own weights as the B
//                  operand, and for the A operand 16 tokens of a dimension, one
//                  16-byte piece of the transposed page.
// fp32: q and the weights go in as sums of three bf16 numbers (24 bits).
template <typename T, int D>
__global__ __launch_bounds__(256) void attn_decode_q8_kernel(
    const T* __restrict__ q, const uint8_t* __restrict__ Kp, const uint8_t* __restrict__ Vp,
    const uint8_t* __restrict__ ks, const uint8_t* __restrict__ vs, int h_kv, int G, int n_pages,
    const int32_t* __restrict__ tables, int b_max, int B, const int32_t* __restrict__ pos,
    const int32_t* __restrict__ idx, const int32_t* __restrict__ cnt, int kmax, float sl2, int S,
    float* __restrict__ ws, DecodeQ8Steps ls) {
  const long long layer = blockIdx.y;
  q += layer * ls.q;
  Kp += layer * ls.pool * B * D;
  Vp += layer * ls.pool * B * D;
  ks += layer * ls.pool;
  vs += layer * ls.pool;
  idx += layer * ls.idx;
  cnt += layer * ls.cnt;
  ws += layer * ls.ws;
  constexpr int NP = sizeof(T) == 2 ? 1 : 3;       // bf16 parts of q and the weights
  constexpr int NK = D / 64;                       // 16-byte pieces of a key per lane
  constexpr int NT = D / 16;                       // tiles of 16 value dimensions
  __shared__ Q8Chunk list[kQ8Chunks];
  __shared__ float sm_o[4][16][D];
  __shared__ float sm_m[4][16], sm_l[4][16];
  const int sp = blockIdx.x % S;
  const int bg = blockIdx.x / S;
  const int bi = bg / h_kv;
  const int g = bg % h_kv;
  const int h_q = h_kv * G;
  const int tid = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63;
  const int ln = l & 15, lg = l >> 4;
  const int p = pos[bi], have = cnt[bi];
  const bool ok = p >= 0 && p / B < b_max;
  const int bc = ok ? p / B : 0;
  const int cpb = B / 16;
  const long long nch = ok ? (long long)max(0, min(have, kmax)) * cpb : 0;
  const long long ngroups = (nch + 3) / 4;
  const long long c_begin = ngroups * sp / S * 4;
  const long long c_end = min(ngroups * (sp + 1) / S * 4, nch);

  bf16x8q qf[NP][NK][2];
  {
    const bool hv = ln < G;
    const T* qp = q + ((long long)bi * h_q + g * G + (hv ? ln : 0)) * D + lg * 16;
#pragma unroll
    for (int c = 0; c < NK; ++c)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if constexpr (NP == 1) {
            const uint16_t raw = hv ? qp[64 * c + 8 * h + e] : (uint16_t)0;
            qf[0][c][h][e] = __builtin_bit_cast(__bf16, raw);
          } else {
            float x = hv ? qp[64 * c + 8 * h + e] : 0.0f;
#pragma unroll
            for (int n = 0; n < NP; ++n) {
              qf[n][c][h][e] = (__bf16)x;
              x -= (float)qf[n][c][h][e];
            }
          }
        }
  }
  f32x4q oacc[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) oacc[t] = f32x4q{0.f, 0.f, 0.f, 0.f};
  float mrun = -INFINITY, lrun = 0.0f;

  for (long long c0 = c_begin; c0 < c_end; c0 += kQ8Chunks) {
    const int n = (int)min((long long)kQ8Chunks, c_end - c0);
    if (c0 > c_begin) __syncthreads();             // the piece before is done with the list
    for (int x = tid; x < (n + 3) / 4 * 4; x += 256) {
      Q8Chunk c{0, INT_MAX, 0, 0.0f, 0.0f};
      if (x < n) {
        const long long e = (c0 + x) / cpb;
        const int off = (int)(c0 + x - e * cpb) * 16;
        const int j = idx[(long long)bi * kmax + e];
        if (j >= 0 && j <= bc && j * B + off <= p) {
          const int page = tables[(long long)bi * b_max + j];
          if ((unsigned)page < (unsigned)n_pages) {
            const long long at = (long long)page * h_kv + g;
            c.page = at * B * D;
            c.t0 = j * B + off;
            c.off = off;
            c.ks = q8_scale(ks[at]) * sl2;
            c.vs = q8_scale(vs[at]);
          }
        }
      }
      list[x] = c;
    }
    __syncthreads();
    for (int gi = w; gi * 4 < n; gi += 4) {
      const Q8Chunk ck = list[gi * 4 + (ln >> 2)];
      const Q8Chunk cv = list[gi * 4 + lg];
      u32x4q kr[4][NK], vr[NT];
      const uint8_t* kp = Kp + ck.page + (long long)(ck.off + (ln & 3)) * D + lg * 16;
      const uint8_t* vp = Vp + cv.page + (long long)ln * B + cv.off;
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int c = 0; c < NK; ++c)
          kr[x][c] = __builtin_nontemporal_load(reinterpret_cast<const u32x4q*>(kp + x * 4 * D + c * 64));
#pragma unroll
      for (int t = 0; t < NT; ++t)
        vr[t] = __builtin_nontemporal_load(reinterpret_cast<const u32x4q*>(vp + t * 16 * B));
      float sv[16];
      float mx = -INFINITY;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        f32x4q acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NK; ++c) {
          const bf16x8q a = q8_bf16x8(kr[x][c][0], kr[x][c][1]);
          const bf16x8q b = q8_bf16x8(kr[x][c][2], kr[x][c][3]);
#pragma unroll
          for (int i = NP - 1; i >= 0; --i) {
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[i][c][0], acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, qf[i][c][1], acc, 0, 0, 0);
          }
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const bool use = cv.t0 <= p - (4 * x + v);
          sv[4 * x + v] = use ? acc[v] * cv.ks : -INFINITY;
          mx = fmaxf(mx, sv[4 * x + v]);
        }
      }
      mx = fmaxf(mrun, q8_xmax(mx));
      // -infinity while no token counted: their weights are 0
      const float mnew = mx == -INFINITY ? 0.0f : mx;
      const float alpha = exp2f(mrun - mnew);
      mrun = mx;
      bf16x8q pf[NP][2];
      float ps = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float pv = exp2f(sv[i] - mnew);
        ps += pv;
        float x = pv * cv.vs;
#pragma unroll
        for (int n2 = 0; n2 < NP; ++n2) {
          pf[n2][i / 8][i % 8] = (__bf16)x;
          x -= (float)pf[n2][i / 8][i % 8];
        }
      }
      lrun = lrun * alpha + ps;
      // places that do not count may hold any code, NaN among them
      const int left = cv.t0 <= p ? min(p - cv.t0 + 1, 16) : 0;   // tokens of the chunk that count
      if (__any(left < 16)) {
        uint32_t mask[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int nb = max(0, min(left - 4 * i, 4));
          mask[i] = nb == 4 ? 0xffffffffu : (1u << (8 * nb)) - 1u;
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) vr[t][i] &= mask[i];
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        oacc[t] *= alpha;
        const bf16x8q a = q8_bf16x8(vr[t][0], vr[t][1]);
        const bf16x8q b = q8_bf16x8(vr[t][2], vr[t][3]);
#pragma unroll
        for (int i = NP - 1; i >= 0; --i) {
          oacc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pf[i][0], oacc[t], 0, 0, 0);
          oacc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, pf[i][1], oacc[t], 0, 0, 0);
        }
      }
    }
  }
  // per-wave partials: head ln; lane groups hold disjoint tokens (sum l) and
  // disjoint output dims
  const float lsum = q8_xsum(lrun);
  if (lg == 0) {
    sm_m[w][ln] = mrun;
    sm_l[w][ln] = lsum;
  }
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int v = 0; v < 4; ++v) sm_o[w][ln][t * 16 + 4 * lg + v] = oacc[t][v];
  __syncthreads();
  float* ws_ml = ws;
  float* ws_o = ws + (long long)gridDim.x / S * G * S * 2;
  for (int xx = tid; xx < G * D; xx += 256) {
    const int u = xx / D, dim = xx % D;
    float M = -INFINITY;
    for (int k = 0; k < 4; ++k) M = fmaxf(M, sm_m[k][u]);
    float Lsum = 0.0f, Osum = 0.0f;
    if (M != -INFINITY) {
      for (int k = 0; k < 4; ++k) {
        const float sc = exp2f(sm_m[k][u] - M);
        Lsum += sm_l[k][u] * sc;
        Osum += sm_o[k][u][dim] * sc;
      }
    }
    const long long hu = (long long)bi * h_q + g * G + u;
    ws_o[(hu * S + sp) * D + dim] = Osum;
    if (dim == 0) {
      ws_ml[(hu * S + sp) * 2 + 0] = M;
      ws_ml[(hu * S + sp) * 2 + 1] = Lsum;
    }
  }
}

hipError_t launch_attn_decode_q8(int dtype, int layers, const void* q, const void* Kp, const void* Vp,
                                 const uint8_t* ks, const uint8_t* vs, int batch, int h_q, int h_kv,
                                 int d, int n_pages, const int32_t* tables, int b_max, int B,
                                 const int32_t* pos, const int32_t* idx, const int32_t* cnt, int kmax,
                                 float scale, void* O, float* ws, hipStream_t st) {
  const int G = h_q / h_kv;
  const int S = decode_attn_splits(batch, h_kv);
  const dim3 grid((unsigned)(batch * h_kv * S), (unsigned)layers);
  const float sl2 = scale * kLog2eQ;
  DecodeQ8Steps ls;
  ls.q = (long long)batch * h_q * d;
  ls.pool = (long long)n_pages * h_kv;
  ls.idx = (long long)batch * kmax;
  ls.cnt = batch;
  ls.ws = (long long)batch * h_q * S * (d + 2);
  const uint8_t* kp = static_cast<const uint8_t*>(Kp);
  const uint8_t* vp = static_cast<const uint8_t*>(Vp);
#define SW_Q8(T, D)                                                                                  \
  hipLaunchKernelGGL((attn_decode_q8_kernel<T, D>), grid, dim3(256), 0, st, static_cast<const T*>(q), \
                     kp, vp, ks, vs, h_kv, G, n_pages, tables, b_max, B, pos, idx, cnt, kmax, sl2, S, \
                     ws, ls)
  if (dtype == SW_BF16) {
    if (d == 128) SW_Q8(uint16_t, 128); else SW_Q8(uint16_t, 64);
  } else {
    if (d == 128) SW_Q8(float, 128); else SW_Q8(float, 64);
  }
#undef SW_Q8
  return launch_attn_merge_q8(dtype, layers, batch, h_q, d, S, ws, O, st);
}

}  // namespace sw
