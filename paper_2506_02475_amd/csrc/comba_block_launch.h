// Internal interface between the host API (comba_block_api.cpp) and the kernels
// of a block's operators.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "comba_block.h"

namespace comba {

constexpr int DC_CH = 64;  // tokens of a chunk
constexpr int DC_BV = 32;  // value columns of a scan's workgroup

struct DecayArgs {
  bool bf16, g_f32, g_head;
  int S, Tseq, Ttot;  // S sequences
  const int32_t* cu_seqlens;
  int H, Hq, Hk, Hv, dk, dv;
  float scale;
  long q_row, k_row, v_row, g_row;
  const void *q, *k, *v, *g;
  const float* h0;
  void* o;
  float* ht;
  // states at every chunk's start, [chunk slot][H][state_bytes]: written,
  // read; a sequence's slots start at start / 64 + its number (fixed rows: at
  // its number times the row's chunks)
  void* kept;
  // step
  float* state;
  const int32_t* slots;
  int num_slots;
  // backward
  const void* dO;
  const float* dht;
  void *dq, *dk_, *dv_, *dg;
  float* dh0;
  void* dkept;  // gradients of the states at every chunk's end, laid out as `kept`
  float* met;  // [chunk slot][H][8 decay_splits] partial sums of both states' products
  float *pq, *pk, *pv;  // [tokens][H][d] gradients of shared heads before their sum, or NULL
  // sequences of more than seglen tokens run as segments of seglen (a multiple of 64)
  // side by side, each from its true state: per segment slot and head its end from
  // zero and its decay
  int seglen;
  float* segS;
  float* segG;  // log2
  hipStream_t stream;
};
// Slots of pieces of `unit` tokens.
inline long decay_slots(const DecayArgs& a, long unit) {
  const long per = (a.Tseq + unit - 1) / unit;
  return a.cu_seqlens ? a.Ttot / unit + a.S : a.S * (per > 1 ? per : 1);
}
// Padded size of the key dimension: of a scan's tiles.
inline int decay_dkp(int dk) { return dk <= 64 ? 64 : dk <= 128 ? 128 : 256; }
__host__ __device__ inline int decay_splits(int dv) { return (dv + DC_BV - 1) / DC_BV; }
// Bytes of a kept state: blocks of 16 rows (value columns), a scale for each, to 16.
__host__ __device__ inline long state_bytes(bool bf16, int dk, int dv) {
  const int cb = !bf16 || dk <= 64 ? 16 : 32;
  const long blocks = (long)((dv + 15) / 16) * ((dk + cb - 1) / cb);
  return blocks * 16 * cb * (bf16 ? 2 : 4) + (blocks * 4 + 15) / 16 * 16;
}
// Floats of one segment's end: every split's accumulators.
inline long decay_end_floats(const DecayArgs& a) {
  return (long)decay_splits(a.dv) * DC_BV * decay_dkp(a.dk);
}
hipError_t launch_decay_fwd(const DecayArgs& a);
hipError_t launch_decay_bwd(const DecayArgs& a);
hipError_t launch_decay_step(const DecayArgs& a);

struct BlockNormArgs {
  bool bf16, x_bf16;
  comba_activation act;
  long rows;
  int C;
  float eps;
  long y_row, z_row, x_row;
  const void *y, *x, *z;
  const float *w1, *sc, *w2;
  void *r, *n;
  const void *dr, *dn;
  void *dy, *dx, *dz;
  float *dw1, *dsc, *dw2;
  float* part;  // [blocks][3][C] partial sums of dw1, dsc, dw2
  int blocks;
  hipStream_t stream;
};
// Workgroups of the backward over the rows, which size its workspace.
int block_norm_bwd_blocks(const BlockNormArgs& a);
hipError_t launch_block_norm_fwd(const BlockNormArgs& a);
hipError_t launch_block_norm_bwd(const BlockNormArgs& a);

}  // namespace comba
