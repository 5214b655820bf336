// Launchers shared between the kernel translation units and the C ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sw_common.h"

namespace sw {

// Byte layout of one layer's decode state (every section 256-byte aligned):
//   double A_scale[batch]        score scale c frozen at its prefill value
//   int32  col0[batch]           first key block whose column decode fills
//   int32  cnt[batch][2][2]      token counts of the open query / key block,
//                                two copies selected by the position's parity
//   double bar[batch][2][2][d]   running means of the open query / key block,
//                                two copies selected by the position's parity
//   double qt[batch][r]          sketch of the current token's query
//   double Qs[batch][b_max][r]   sketch of every query-block representative
//   double Ks[batch][b_max][r]   sketch of every key-block representative
//   float  rowc[batch][b_max]    the open block's score row A[b_cur][:] and
//   float  colc[batch][b_max]    column A[:][b_cur] as the last step wrote
//                                them (contiguous copies of cache entries)
//   float  A[batch][lda/32][b_max][32]  block-score cache in strips of 32
//                                columns (entry (m, j) at cache_at(b_max, m, j)
//                                within a sequence), lda = b_max rounded up
//                                to a multiple of 32
// The step at position p reads the open-block means and counts of copy
// (p + 1) % 2 (written by the step at p - 1) and writes copy p % 2, so every
// workgroup of a step reads the previous values while one of them writes
// the new ones.
struct DecodeLayout {
  int64_t scale, col0, cnt, bar, qt, qs, ks, rowc, colc, a, total;
  int lda;
};

__host__ __device__ inline DecodeLayout decode_layout(int batch, int d, int r, int b_max) {
  auto al = [](int64_t x) { return (x + 255) / 256 * 256; };
  DecodeLayout L;
  L.lda = (b_max + 31) & ~31;
  int64_t o = 0;
  L.scale = o;  o = al(o + 8LL * batch);
  L.col0 = o;   o = al(o + 4LL * batch);
  L.cnt = o;    o = al(o + 16LL * batch);
  L.bar = o;    o = al(o + 32LL * batch * d);
  L.qt = o;     o = al(o + 8LL * batch * r);
  L.qs = o;     o = al(o + 8LL * batch * b_max * r);
  L.ks = o;     o = al(o + 8LL * batch * b_max * r);
  L.rowc = o;   o = al(o + 4LL * batch * b_max);
  L.colc = o;   o = al(o + 4LL * batch * b_max);
  L.a = o;      o = al(o + 4LL * batch * b_max * L.lda);
  L.total = o;
  return L;
}

// Offset (in floats) of score (m, j) within one sequence's cache: the cache
// is stored as strips of 32 columns, each strip's rows contiguous (128 bytes
// per row), so a walk over one strip's rows reads one contiguous range.
__host__ __device__ inline int cache_at(int b_max, int m, int j) {
  return ((j >> 5) * b_max + m) * 32 + (j & 31);
}

constexpr int kDecodeMaxSplits = 32;

// Bytes with which launch_sketch splits few block rows over more workgroups
// (0: it would not, whatever the type); without them (ws NULL) it does not split.
int64_t sketch_workspace_bytes(int h_q, int h_kv, int d, int B, int64_t nb);

hipError_t launch_sketch(int dtype, const void* Q, const void* K, int h_q, int h_kv, int d,
                         const SeqMeta& meta, int64_t nb, long long N, const int8_t* signs,
                         const int32_t* cols, int r, double* Qs, double* Ks, double* A,
                         double* A_scale, double* Qbar, double* Kbar, void* ws, hipStream_t st);

int64_t walk_workspace_bytes(int variant, int64_t nm);

hipError_t launch_walk(int variant, const double* A, const double* A_scale, int s_exp,
                       double logit_scale, const SeqMeta& meta, int64_t nb, const double* R_prev,
                       double* R_out, double* ws, hipStream_t st);

hipError_t launch_select(const double* R, const SeqMeta& meta, int64_t nb, int k, int pct,
                         uint32_t flags, int32_t* idx, int32_t* cnt, int kmax, hipStream_t st);

hipError_t launch_attn_prefill(int dtype, const void* Q, const void* K, const void* V, int h_q,
                               int h_kv, int d, long long N, const SeqMeta& meta, int64_t nb,
                               const int32_t* idx, const int32_t* cnt, int kmax, float scale,
                               void* O, float* lse, hipStream_t st);

hipError_t launch_decode_init(char* state, int batch, int d, int r, int b_max, int seq, int n, int B,
                              const double* Qs, const double* Ks, const double* A,
                              const double* A_scale, const double* Qbar, const double* Kbar,
                              hipStream_t st);

hipError_t launch_kv_append(int dtype, const void* k_new, const void* v_new, void* Kc, void* Vc,
                            int batch, int h_kv, int d, int T_max, const int32_t* pos,
                            hipStream_t st);

hipError_t launch_decode_sketch(int dtype, const void* q_new, const void* k_new, int batch, int h_q,
                                int h_kv, int d, int B, const int32_t* pos, const int8_t* signs,
                                const int32_t* cols, int r, int b_max, char* state,
                                hipStream_t st);

// Alg. 2 step 5 for the per-layer entry point: the walk row of every
// sequence, divided by its largest magnitude, into r_out [batch][b_max].
hipError_t launch_decode_walk(const char* state, int batch, int d, int r, int b_max, int B,
                              const int32_t* pos, int s_exp, bool relu, const double* r_prev,
                              double* r_out, hipStream_t st);

// Alg. 2 steps 1-6 of every layer for the one-call step: the incremental
// sketch with the KV append of all layers in one launch, then one launch per
// layer for the walk row with the selection of the layer before it, and a
// last one for the last layer's selection. Buffers are stacked over layers.
// Kc NULL: no append.
hipError_t launch_decode_layers(int dtype, int layers, const void* q_new, const void* k_new,
                                const void* v_new, void* Kc, void* Vc, int T_max, int batch, int h_q,
                                int h_kv, int d, int B, const int32_t* pos, const int8_t* signs,
                                const int32_t* cols, int r, int b_max, char* state, int s_exp,
                                bool relu, double* rows, int k, int pct, uint32_t flags, int32_t* idx,
                                int32_t* cnt, int kmax, hipStream_t st);

hipError_t launch_select_decode(const double* rows, int batch, int b_max, int B,
                                const int32_t* pos, int k, int pct, uint32_t flags, int32_t* idx,
                                int32_t* cnt, int kmax, hipStream_t st);

int decode_attn_splits(int batch, int h_kv);

// Device address of this device's fixed scratch array
// (SW_NOALLOC_SCRATCH_BYTES), looked up on the first call on each device.
hipError_t noalloc_scratch(void** out);

// Alg. 2 step 7 for `layers` layers in one launch (and one for the merge); all
// buffers stacked over the layers, ws too (decode_attn_workspace per layer).
hipError_t launch_attn_decode(int dtype, int layers, const void* q, const void* Kc, const void* Vc,
                              int batch, int h_q, int h_kv, int d, int T_max, int B,
                              const int32_t* pos, const int32_t* idx, const int32_t* cnt, int kmax,
                              float scale, void* O, float* ws, hipStream_t st);

// ---------------------------------------------------------------------------
// paged 8-bit cache
// ---------------------------------------------------------------------------

// Strides of the new tokens' keys and values in elements: from one head to the
// next, one token to the next, and one layer to the next of stacked buffers.
struct TokenStrides {
  long long k_head, k_tok, v_head, v_tok, layer;
};

// Elements from one layer to the next (pool: pages times heads).
struct DecodeQ8Steps {
  long long q, pool, idx, cnt, ws;
};

int64_t block_tables_workspace_bytes(int n_seqs, int64_t n_slots);

hipError_t launch_block_tables(int n_seqs, int B, int b_max, const int32_t* old_len,
                               const int32_t* new_len, int32_t* tables, int32_t* free_pages,
                               int32_t* n_free, int n_pages, int rows, int n_slots, int32_t* slots,
                               int32_t* cu, int32_t* pos, int32_t* status, int32_t* ws, hipStream_t st);

// Threads of an append's launch along its first dimension.
long long kv_append_q8_threads(int dtype, int64_t N, int n_seqs, bool by_seq, int h_kv, int d, int B);

// cu NULL: every token by its slot alone; live then receives pos of those that have
// a place, -1 of the others (both may be NULL).
hipError_t launch_kv_append_q8(int dtype, int layers, const void* k, const void* v,
                               const TokenStrides& sd, int N, int n_seqs, const int32_t* cu,
                               const int32_t* slots, int n_pages, int h_kv, int d, int B, void* Kp,
                               void* Vp, uint8_t* ks, uint8_t* vs, const int32_t* pos, int32_t* live,
                               hipStream_t st);

hipError_t launch_kv_fetch_q8(int dtype, const void* Kp, const void* Vp, const uint8_t* ks,
                              const uint8_t* vs, int n_pages, int h_kv, int d, int B, int n_seqs,
                              int b_max, const int32_t* tables, const int32_t* first, const int32_t* cu,
                              int N, void* K, void* V, hipStream_t st);

// Per layer; 0 for batches whose (sequence, KV head) pairs have a workgroup each.
int64_t attn_decode_q8_workspace_bytes(int batch, int h_q, int h_kv, int d);

hipError_t launch_attn_decode_q8(int dtype, int layers, const void* q, const void* Kp, const void* Vp,
                                 const uint8_t* ks, const uint8_t* vs, int batch, int h_q, int h_kv,
                                 int d, int n_pages, const int32_t* tables, int b_max, int B,
                                 const int32_t* pos, const int32_t* idx, const int32_t* cnt, int kmax,
                                 float scale, void* O, float* ws, hipStream_t st);

}  // namespace sw
