// Decode attention over the paged 8-bit cache (paper Alg. 2 step 7 with K and V
// as e4m3 codes): softmax attention of one token per sequence over the tokens
// of the selected key blocks, split-K over those tokens.
#include <climits>
#include <type_traits>

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

// 2^x; results below 2^-126 are 0.
__device__ __forceinline__ float q8_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Eight codes as the operand of a bf16 matrix instruction (exact).
__device__ __forceinline__ bf16x8q q8_bf16x8(uint32_t lo, uint32_t hi) {
  const bf16x2q a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
  const bf16x2q b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
  const bf16x2q c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
  const bf16x2q d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  return bf16x8q{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

constexpr int kQ8Wgs = 768;                        // shares of a call, at most
constexpr int kQ8Batch = 256;                      // sequences of such a call: four a lane
constexpr int kQ8Splits = 64;                      // workgroups per (sequence, KV head), at most

// Groups of 64 selected tokens of a sequence.
__device__ __forceinline__ int q8_groups(int p, int have, int kmax, int b_max, int B) {
  if (p < 0 || p / B >= b_max) return 0;
  return (int)(((long long)max(0, min(have, kmax)) * (B / 16) + 3) / 4);
}

// One sequence's part in a shared call.
struct Q8Part {
  int p, have;                                     // position and count
  int groups, splits;                              // per head; workgroups of each head
  int before;                                      // workgroups of the sequences before, per head
};

// How a call's groups are shared out, worked out by every wavefront for itself
// (no barrier): a workgroup takes a part of one (sequence, head), at most `per`
// groups, which is a `shares`th of all and at least one for each of its wavefronts.
// So sequences of different lengths keep all workgroups equally long, and a
// workgroup has one prologue and one epilogue. Shares: three workgroups per CU in
// bf16, two in fp32 (16 ragged sequences of up to 16000 tokens, bf16: 19.9 us with
// 512, 18.1 with 768, 20.7 with 1536; even ones of 65536 69.8, 70.1, 72.1; fp32 of
// head dimension 64 12.3, 12.5, 12.5).
struct Q8Plan {
  int lane_before, lane_splits, p[4], c[4], n[4], s[4];

  __device__ __forceinline__ void make(int batch, int h_kv, int kmax, int b_max, int B,
                                       const int32_t* pos, const int32_t* cnt, uint32_t shares) {
    const int l = threadIdx.x & 63;
    typedef int i32x4u __attribute__((ext_vector_type(4), aligned(4)));
    if (4 * l + 4 <= batch) {
      const i32x4u vp = *reinterpret_cast<const i32x4u*>(pos + 4 * l);
      const i32x4u vc = *reinterpret_cast<const i32x4u*>(cnt + 4 * l);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[i] = vp[i];
        c[i] = vc[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int b = 4 * l + i;
        p[i] = b < batch ? pos[b] : -1;
        c[i] = b < batch ? cnt[b] : 0;
      }
    }
    int sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += n[i] = q8_groups(p[i], c[i], kmax, b_max, B);
    const uint32_t T = (uint32_t)__builtin_amdgcn_readlane(wave_inclusive_scan(sum), 63) * h_kv;
    const uint32_t per = max(4u, (T + shares - 1) / shares);
    lane_splits = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s[i] = min(kQ8Splits, (int)(((uint32_t)n[i] + per - 1) / per));
      lane_splits += s[i];
    }
    lane_before = wave_inclusive_scan(lane_splits) - lane_splits;
  }
  // the part of sequence 4 lane + i (both the same in every lane)
  __device__ __forceinline__ Q8Part part(int lane, int i) const {
    Q8Part r{};
    int before = __builtin_amdgcn_readlane(lane_before, lane);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int sk = __builtin_amdgcn_readlane(s[k], lane);
      if (k == i) {
        r.p = __builtin_amdgcn_readlane(p[k], lane);
        r.have = __builtin_amdgcn_readlane(c[k], lane);
        r.groups = __builtin_amdgcn_readlane(n[k], lane);
        r.splits = sk;
        r.before = before;
      }
      before += sk;
    }
    return r;
  }
  // the sequence of workgroup x, -1 for none
  __device__ __forceinline__ int owner(int x, int h_kv) const {
    const uint64_t in = __ballot(lane_before * h_kv <= x && x < (lane_before + lane_splits) * h_kv);
    if (in == 0) return -1;
    const int lane = __builtin_ctzll(in);
    int before = __builtin_amdgcn_readlane(lane_before, lane), i = 0;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      before += __builtin_amdgcn_readlane(s[k], lane);
      if (x >= before * h_kv) i = k + 1;
    }
    return 4 * lane + i;
  }
};

// The output of a (sequence, head) whose largest logit is -infinity: 0 without a token
// (a sum of weights of 0), NaN otherwise.
__device__ __forceinline__ float q8_no_max(float l) { return l == 0.0f ? 0.0f : NAN; }

// The workspace of a layer, in floats: first workgroup and number of them of each
// (sequence, head); then of every workgroup its heads' maxima and sums of weights,
// and their outputs (16-byte aligned).
__host__ __device__ inline int64_t q8_ws_sums(int64_t pairs) { return 2 * pairs; }
__host__ __device__ inline int64_t q8_ws_outs(int64_t pairs, int G) {
  return (q8_ws_sums(pairs) + (kQ8Wgs + pairs) * G * 2 + 3) & ~3ll;
}

template <typename T>
__device__ __forceinline__ void q8_store(T* O, long long at, float v) {
  if constexpr (sizeof(T) == 2) O[at] = f32_to_bf16(v);
  else O[at] = v;
}

// Workgroup of four wavefronts over a part of a (sequence, head)'s groups of 64
// selected tokens, four chunks of 16, whichever blocks they are in; each wavefront
// takes every fourth group, so that the wavefronts together read 256 tokens of a
// value row at about the same time (a block of 128 has a 128-byte line of it in
// two groups; quarters of the range one after the other take 112 us where this takes
// 96). A lane holds the page and place of one chunk of 16 groups ahead,
// so that the loop has neither barriers nor index loads.
//   S = K q^T      v_mfma_f32_16x16x32_bf16: row m of the x-th product is token
//                  4 x + m % 4 of chunk m / 4, so lane (n, lg) receives 16
//                  tokens of head n, all of chunk lg: its scale, its first token
//                  and its weights are the lane's own.
//   O^T += V^T P^T the same instruction: k = 8 lg + i of product y is token
//                  8 y + i of chunk lg, that is the lane's own weights as the B
//                  operand, and for the A operand 16 tokens of a dimension, one
//                  16-byte piece of the transposed page.
// bf16: codes and q are bf16 numbers as they are; the weights go into the second product
// as sums of two bf16 numbers, at most 2^-16 of each off. One number (2^-8) would take half
// of that product's instructions and 0.3 to 2.5 % of a call's time (16 sequences of 65536
// tokens 80.2 us for 80.5, 16 ragged ones of head dimension 64 14.8 for 15.2), but moved
// the output by 0.0014 in the root mean square; with two it is that of 32-bit weights but for
// 6e-5, roundings at the end that fall the other way.
// fp32: q and the weights go in as sums of three bf16 numbers (24 bits).
// SHARE: the groups are shared out as Q8Plan does; a (sequence, head) of one
// workgroup is written out by it, others leave partial sums. Otherwise a
// workgroup per (sequence, head). STREAM: the values' loads, see below.
template <typename T, int D, bool SHARE, bool STREAM>
__global__ __launch_bounds__(256) void attn_decode_q8_kernel(
    const T* __restrict__ q, const uint8_t* __restrict__ Kp, const uint8_t* __restrict__ Vp,
    const uint8_t* __restrict__ ks, const uint8_t* __restrict__ vs, int batch, int h_kv, int G, int n_pages,
    const int32_t* __restrict__ tables, int b_max, int B, const int32_t* __restrict__ pos,
    const int32_t* __restrict__ idx, const int32_t* __restrict__ cnt, int kmax, float sl2,
    T* __restrict__ O, float* __restrict__ ws, DecodeQ8Steps ls) {
  const long long layer = blockIdx.y;
  q += layer * ls.q;
  O += layer * ls.q;
  Kp += layer * ls.pool * B * D;
  Vp += layer * ls.pool * B * D;
  ks += layer * ls.pool;
  vs += layer * ls.pool;
  idx += layer * ls.idx;
  cnt += layer * ls.cnt;
  ws += layer * ls.ws;
  constexpr int NP = sizeof(T) == 2 ? 1 : 3;       // bf16 parts of q
  constexpr int NW = sizeof(T) == 2 ? 2 : 3;       // of the weights
  constexpr int NK = D / 64;                       // 16-byte pieces of a key per lane
  constexpr int NT = D / 16;                       // tiles of 16 value dimensions
  __shared__ float sm_o[4][16][D];
  __shared__ float sm_m[4][16], sm_l[4][16];
  const int h_q = h_kv * G;
  const int tid = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63;
  const int ln = l & 15, lg = l >> 4;
  const int cpb = B / 16;

  int bi, g, ga, gb;                               // groups ga .. gb - 1 of (bi, g)
  Q8Part part;
  if constexpr (SHARE) {
    Q8Plan plan;
    plan.make(batch, h_kv, kmax, b_max, B, pos, cnt, sizeof(T) == 2 ? kQ8Wgs : kQ8Wgs * 2 / 3);
    // for the merge: first workgroup and number of them of each (sequence, head)
    const int b = blockIdx.x;
    if (b < batch && w == 0) {
      const Q8Part x = plan.part(b >> 2, b & 3);
      for (int h = l; h < h_kv; h += 64)
        reinterpret_cast<int2*>(ws)[b * h_kv + h] = make_int2(x.before * h_kv + h * x.splits, x.splits);
    }
    bi = plan.owner(blockIdx.x, h_kv);
    if (bi < 0) return;
    part = plan.part(bi >> 2, bi & 3);
    const int r = blockIdx.x - part.before * h_kv;
    g = r / part.splits;
    const int sp = r - g * part.splits, each = part.groups / part.splits, more = part.groups % part.splits;
    ga = sp * each + min(sp, more);
    gb = ga + each + (sp < more);
  } else {
    bi = blockIdx.x / h_kv;
    g = blockIdx.x - bi * h_kv;
    part.p = pos[bi];
    part.have = cnt[bi];
    part.splits = 1;
    ga = 0;
    gb = q8_groups(part.p, part.have, kmax, b_max, B);
  }
  const int p = part.p, bc = p / B;
  const int nch = max(0, min(part.have, kmax)) * cpb;   // chunks of the sequence
  bf16x8q qf[NP][NK][2];
  {
    const bool hv = ln < G;
    const T* qp = q + ((long long)bi * h_q + g * G + (hv ? ln : 0)) * D + lg * 16;
#pragma unroll
    for (int c = 0; c < NK; ++c)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if constexpr (NP == 1) {
          const uint4 v = *reinterpret_cast<const uint4*>(qp + 64 * c + 8 * h);
          qf[0][c][h] = __builtin_bit_cast(bf16x8q, hv ? v : make_uint4(0, 0, 0, 0));
        } else {
          const float4 v0 = *reinterpret_cast<const float4*>(qp + 64 * c + 8 * h);
          const float4 v1 = *reinterpret_cast<const float4*>(qp + 64 * c + 8 * h + 4);
          const float v[8] = {v0.x, v0.y, v0.z, v0.w, v1.x, v1.y, v1.z, v1.w};
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float x = hv ? v[e] : 0.0f;
#pragma unroll
            for (int n = 0; n < NP; ++n) {
              qf[n][c][h][e] = (__bf16)x;
              x -= (float)qf[n][c][h][e];
            }
          }
        }
      }
  }
  f32x4q oacc[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) oacc[t] = f32x4q{0.f, 0.f, 0.f, 0.f};
  float mrun = -INFINITY, lrun = 0.0f;
  bool seen = false;                               // a token that counts
  // the lane's chunk of the listed groups: page, first token (INT_MAX: none of it
  // counts), place in the page
  int c_page = 0, c_t0 = INT_MAX, c_off = 0;
  // The loads of a group. Its scales are loaded beside its codes. Whole
  // lines that are read once are loaded as a stream; of the values, blocks over 64
  // leave part of a line to another group (16 sequences of 65536 tokens, values as
  // a stream and not: 69.1 and 71.9 us at blocks of 64, 96 and 92 at 128, 114 and
  // 102 at 1024).
  struct Group {
    u32x4q k[4][NK], v[NT];
    uint32_t ks, vs;
    int t0;
  };
  // The i-th of the 16 listed groups.
  auto issue = [&](int i, Group& r) {
    const int fk = 4 * i + (ln >> 2), fv = 4 * i + lg;
    const long long at_k = (long long)__shfl(c_page, fk) * h_kv + g;
    const long long at_v = (long long)__shfl(c_page, fv) * h_kv + g;
    const uint8_t* kp = Kp + (at_k * B + __shfl(c_off, fk) + (ln & 3)) * D + lg * 16;
    const uint8_t* vp = Vp + (at_v * D + ln) * B + __shfl(c_off, fv);
    r.t0 = __shfl(c_t0, fv);
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int c = 0; c < NK; ++c)
        r.k[x][c] = __builtin_nontemporal_load(reinterpret_cast<const u32x4q*>(kp + x * 4 * D + c * 64));
    r.ks = ks[at_v];
    r.vs = vs[at_v];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const u32x4q* from = reinterpret_cast<const u32x4q*>(vp + t * 16 * B);
      if constexpr (STREAM) r.v[t] = __builtin_nontemporal_load(from);
      else r.v[t] = *from;
    }
    // all of them are out before the first is waited for (the scheduler
    // otherwise moves the values' loads behind the scores)
    __builtin_amdgcn_sched_barrier(0);
  };
  auto compute = [&](Group& r) {
    f32x4q acc[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      acc[x] = f32x4q{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NK; ++c) {
        const bf16x8q a = q8_bf16x8(r.k[x][c][0], r.k[x][c][1]);
        const bf16x8q b = q8_bf16x8(r.k[x][c][2], r.k[x][c][3]);
#pragma unroll
        for (int i = NP - 1; i >= 0; --i) {
          acc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[i][c][0], acc[x], 0, 0, 0);
          acc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, qf[i][c][1], acc[x], 0, 0, 0);
        }
      }
    }
    // a chunk that does not count has the scale of some page, maybe one never begun
    const float kf = q8_scale(r.ks) * sl2, vf = r.t0 <= p ? q8_scale(r.vs) : 0.0f;
    float sv[16];
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      sv[i] = r.t0 <= p - i ? acc[i / 4][i % 4] * kf : -INFINITY;
      mx = fmaxf(mx, sv[i]);
    }
    mx = fmaxf(mrun, q8_xmax(mx));
    // -infinity while no token counted: their weights are 0
    const float mnew = mx == -INFINITY ? 0.0f : mx;
    const float alpha = q8_exp2(mrun - mnew);
    mrun = mx;
    bf16x8q pf[NW][2];
    float ps = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float pv = q8_exp2(sv[i] - mnew);
      ps += pv;
      float x = pv * vf;
#pragma unroll
      for (int n2 = 0; n2 < NW; ++n2) {
        pf[n2][i / 8][i % 8] = (__bf16)x;
        x -= (float)pf[n2][i / 8][i % 8];
      }
    }
    lrun = lrun * alpha + ps;
    seen |= r.t0 <= p;
    // places that do not count may hold any code, NaN among them
    const int left = r.t0 <= p ? min(p - r.t0 + 1, 16) : 0;   // tokens of the chunk that count
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
        for (int i = 0; i < 4; ++i) r.v[t][i] &= mask[i];
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      oacc[t] *= alpha;
      const bf16x8q a = q8_bf16x8(r.v[t][0], r.v[t][1]);
      const bf16x8q b = q8_bf16x8(r.v[t][2], r.v[t][3]);
#pragma unroll
      for (int i = NW - 1; i >= 0; --i) {
        oacc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pf[i][0], oacc[t], 0, 0, 0);
        oacc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, pf[i][1], oacc[t], 0, 0, 0);
      }
    }
  };
  for (int g0 = ga + w; g0 < gb; g0 += 64) {
    c_page = c_off = 0;
    c_t0 = INT_MAX;
    const int gl = g0 + (l & ~3), ch = gl * 4 + (l & 3);
    if (gl < gb && ch < nch) {
      const int e = ch / cpb, off = (ch - e * cpb) * 16;
      const int j = idx[(long long)bi * kmax + e];
      if (j >= 0 && j <= bc && j * B + off <= p) {
        const int page = tables[(long long)bi * b_max + j];
        if ((unsigned)page < (unsigned)n_pages) {
          c_page = page;
          c_off = off;
          c_t0 = j * B + off;
        }
      }
    }
    for (int i = 0; i < 16 && g0 + 4 * i < gb; ++i) {
      Group r;
      issue(i, r);
      compute(r);
    }
  }
  // per-wave partials: head ln; lane groups hold disjoint tokens (sum l) and
  // disjoint output dims. A maximum of -infinity is that of no token, or of tokens
  // whose logits are all NaN or -infinity, for which the softmax has no value: a sum of
  // weights that is not 0 tells them apart (beside finite logits the latter weigh 0).
  const float lsum = q8_xsum(lrun);
  const float none = __any(seen) && mrun == -INFINITY ? 1.0f : 0.0f;
  if (ln < G) {
    if (lg == 0) {
      sm_m[w][ln] = mrun;
      sm_l[w][ln] = lsum + none;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
      *reinterpret_cast<f32x4q*>(&sm_o[w][ln][t * 16 + 4 * lg]) = oacc[t];
  }
  __syncthreads();
  const long long pairs = (long long)batch * h_kv, seg = blockIdx.x;
  float* ws_ml = ws + q8_ws_sums(pairs) + seg * G * 2;
  float* ws_o = ws + q8_ws_outs(pairs, G) + seg * G * D;
  for (int x = tid; x < G * D / 4; x += 256) {
    const int u = x / (D / 4), dim = x % (D / 4) * 4;
    float M = -INFINITY;
#pragma unroll
    for (int k = 0; k < 4; ++k) M = fmaxf(M, sm_m[k][u]);
    float Lsum = 0.0f;
    f32x4q Osum = {0.f, 0.f, 0.f, 0.f};
    if (M != -INFINITY) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float sc = q8_exp2(sm_m[k][u] - M);
        Lsum += sm_l[k][u] * sc;
        Osum += *reinterpret_cast<const f32x4q*>(&sm_o[k][u][dim]) * sc;
      }
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) Lsum += sm_l[k][u];
    }
    if (part.splits == 1) {
      const long long at = ((long long)bi * h_q + g * G + u) * D + dim;
      const float inv = M == -INFINITY ? q8_no_max(Lsum) : 1.0f / Lsum;
      if constexpr (sizeof(T) == 2)
        *reinterpret_cast<uint2*>(O + at) =
            make_uint2(pack_bf16x2(Osum[0] * inv, Osum[1] * inv), pack_bf16x2(Osum[2] * inv, Osum[3] * inv));
      else
        *reinterpret_cast<f32x4q*>(O + at) = Osum * inv;
    } else {
      *reinterpret_cast<f32x4q*>(ws_o + u * D + dim) = Osum;
      if (dim == 0) {
        ws_ml[2 * u] = M;
        ws_ml[2 * u + 1] = Lsum;
      }
    }
  }
}

// A value with that of the lane 1, 2, 4 and 8 further in its row of 16 lanes.
template <int BY>
__device__ __forceinline__ float q8_ror(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x120 + BY, 0xf, 0xf, true));
}
__device__ __forceinline__ float q8_wave_max(float v) {
  v = fmaxf(v, q8_ror<1>(v));
  v = fmaxf(v, q8_ror<2>(v));
  v = fmaxf(v, q8_ror<4>(v));
  return q8_xmax(fmaxf(v, q8_ror<8>(v)));
}
__device__ __forceinline__ float q8_wave_sum(float v) {
  v += q8_ror<1>(v);
  v += q8_ror<2>(v);
  v += q8_ror<4>(v);
  return q8_xsum(v + q8_ror<8>(v));
}

// Merge of the partial sums of one (sequence, query head): those of the
// workgroups that shared its groups, at most 64. Lane s of every wavefront holds
// the s-th one's maximum and sum; wavefront w adds the outputs of w, w + 4, ...,
// all on their way before the first is needed: two dependent loads, one barrier.
template <typename T, int D>
__global__ __launch_bounds__(256) void attn_merge_q8_kernel(const float* __restrict__ ws, int batch, int h_kv,
                                                            int G, T* __restrict__ O, DecodeQ8Steps ls) {
  static_assert(kQ8Splits <= 64, "one partial sum per lane");
  constexpr int V = D / 64;                        // output dims per lane
  typedef float vec __attribute__((ext_vector_type(V)));
  __shared__ float part[4][D];
  const long long layer = blockIdx.y;
  ws += layer * ls.ws;
  O += layer * ls.q;
  const int t = threadIdx.x, w = __builtin_amdgcn_readfirstlane(t >> 6), l = t & 63;
  const int pair = blockIdx.x / G, u = blockIdx.x - pair * G;
  const int2 info = reinterpret_cast<const int2*>(ws)[pair];
  const int S = info.y;
  const long long at = (long long)blockIdx.x * D;
  if (S == 0) {                                    // no token
    if (t < D) q8_store(O, at + t, 0.0f);
    return;
  }
  if (S == 1) return;                              // its workgroup wrote the output
  const long long pairs = (long long)batch * h_kv, seg = info.x;
  const float2 ml = *reinterpret_cast<const float2*>(ws + q8_ws_sums(pairs) + ((seg + min(l, S - 1)) * G + u) * 2);
  const float* o = ws + q8_ws_outs(pairs, G) + (seg * G + u) * D + l * V;
  vec acc = {};
  float top, Lsum;
  auto add = [&](auto n) {
    constexpr int N = decltype(n)::value;
    vec x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = *reinterpret_cast<const vec*>(o + (long long)min(w + 4 * i, S - 1) * G * D);
    const float m = l < S ? ml.x : -INFINITY;
    top = q8_wave_max(m);
    // without a maximum the outputs weigh 0, the sums of weights 1 (whether there is a token)
    const float sc = top != -INFINITY && l < S ? q8_exp2(m - top) : 0.0f;
    Lsum = q8_wave_sum(l < S ? ml.y * (top != -INFINITY ? sc : 1.0f) : 0.0f);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int s = w + 4 * i;
      if (s < S) acc += x[i] * __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(sc), s));
    }
  };
  if (S <= 16) add(std::integral_constant<int, 4>());
  else add(std::integral_constant<int, 16>());
#pragma unroll
  for (int e = 0; e < V; ++e) part[w][l * V + e] = acc[e];
  __syncthreads();
  if (t >= D) return;
  const float sum = ((part[0][t] + part[1][t]) + part[2][t]) + part[3][t];
  q8_store(O, at + t, top == -INFINITY ? q8_no_max(Lsum) : sum / Lsum);
}

int64_t attn_decode_q8_workspace_bytes(int batch, int h_q, int h_kv, int d) {
  if (batch > kQ8Batch) return 0;
  const int64_t pairs = (int64_t)batch * h_kv;
  return (q8_ws_outs(pairs, h_q / h_kv) + (kQ8Wgs + pairs) * (h_q / h_kv) * d) * 4;
}

hipError_t launch_attn_decode_q8(int dtype, int layers, const void* q, const void* Kp, const void* Vp,
                                 const uint8_t* ks, const uint8_t* vs, int batch, int h_q, int h_kv,
                                 int d, int n_pages, const int32_t* tables, int b_max, int B,
                                 const int32_t* pos, const int32_t* idx, const int32_t* cnt, int kmax,
                                 float scale, void* O, float* ws, hipStream_t st) {
  const int G = h_q / h_kv;
  const float sl2 = scale * kLog2eQ;
  const bool share = batch <= kQ8Batch;
  DecodeQ8Steps ls;
  ls.q = (long long)batch * h_q * d;
  ls.pool = (long long)n_pages * h_kv;
  ls.idx = (long long)batch * kmax;
  ls.cnt = batch;
  ls.ws = attn_decode_q8_workspace_bytes(batch, h_q, h_kv, d) / 4;
  const dim3 grid((unsigned)(batch * h_kv + (share ? kQ8Wgs : 0)), (unsigned)layers);
  const dim3 mgrid((unsigned)(batch * h_q), (unsigned)layers);
  const uint8_t* kp = static_cast<const uint8_t*>(Kp);
  const uint8_t* vp = static_cast<const uint8_t*>(Vp);
#define SW_Q8_(T, D, SHARE, STREAM)                                                                   \
  hipLaunchKernelGGL((attn_decode_q8_kernel<T, D, SHARE, STREAM>), grid, dim3(256), 0, st,            \
                     static_cast<const T*>(q), kp, vp, ks, vs, batch, h_kv, G, n_pages, tables, b_max, \
                     B, pos, idx, cnt, kmax, sl2, static_cast<T*>(O), ws, ls)
#define SW_Q8(T, D)                                                                                 \
  do {                                                                                              \
    if (share) {                                                                                    \
      if (B <= 64) SW_Q8_(T, D, true, true); else SW_Q8_(T, D, true, false);                        \
      hipLaunchKernelGGL((attn_merge_q8_kernel<T, D>), mgrid, dim3(256), 0, st, ws, batch, h_kv, G, \
                         static_cast<T*>(O), ls);                                                   \
    } else {                                                                                        \
      if (B <= 64) SW_Q8_(T, D, false, true); else SW_Q8_(T, D, false, false);                      \
    }                                                                                               \
  } while (0)
  if (dtype == SW_BF16) {
    if (d == 128) SW_Q8(uint16_t, 128); else SW_Q8(uint16_t, 64);
  } else {
    if (d == 128) SW_Q8(float, 128); else SW_Q8(float, 64);
  }
#undef SW_Q8
#undef SW_Q8_
  return hipGetLastError();
}

}  // namespace sw
