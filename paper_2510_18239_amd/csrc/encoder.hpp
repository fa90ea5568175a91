// Launcher interface of the history encoder's operators: norms and rotation of heads, attention over packed histories, the loss
// over a catalogue.
#pragma once

#include "common.hpp"

namespace lime {

// ----------------------------------------------------------------------------- attention over packed sequences
// User b's queries are rows q_offsets[b] .. of Q, the first q_lens[b] of its slot (NULL: all); its keys and values likewise.
struct SequenceAttention {
  const void *Q, *K, *V;                        // [q_rows][hq][dh], [k_rows][hk][dh] twice
  int64_t q_stride, k_stride, v_stride;         // elements from row to row
  const int32_t *q_offsets, *q_lens, *k_offsets, *k_lens;
  void* O;                                      // [q_rows][hq][dh]
  float* lse;                                   // [q_rows][hq], natural logarithm; nullable in the forward pass
  int64_t q_rows, k_rows;
  int B, max_q, max_k, hq, hk, dh;
  float scale;
  int causal, dtype;
  // the backward pass
  const void* dO;                               // [q_rows][hq][dh]
  void *dQ, *dK, *dV;
  int64_t dq_stride, dk_stride, dv_stride;
};
constexpr int kMaxSequenceHead = 128;
bool sequence_attention_fits(const SequenceAttention& a);  // the launches' sizes
size_t sequence_attention_workspace(const SequenceAttention& a);
hipError_t sequence_attention(const SequenceAttention& a, void* workspace, hipStream_t s);
bool sequence_attention_backward_fits(const SequenceAttention& a);
size_t sequence_attention_backward_workspace(const SequenceAttention& a);
hipError_t sequence_attention_backward(const SequenceAttention& a, void* workspace, hipStream_t s);

// ----------------------------------------------------------------------------- softmax cross entropy over a catalogue
struct CatalogueLoss {
  const void *X, *W;       // [rows][d], [items][d]
  const int32_t* targets;  // [rows]; outside [0, items): the row has no target
  float *loss, *lse;       // [rows]; lse: the backward pass's input
  const float* dloss;      // [rows]
  void *dX, *dW;           // nullable
  int64_t rows;
  int items, d, dtype;
  float scale;
};
constexpr int kMaxCatalogueWidth = 256;
bool catalogue_loss_fits(int64_t rows, int items);
size_t catalogue_loss_workspace(int64_t rows, int items, int d, int dtype, bool backward);
hipError_t catalogue_loss(const CatalogueLoss& a, void* workspace, hipStream_t s);
hipError_t catalogue_loss_backward(const CatalogueLoss& a, void* workspace, hipStream_t s);

// ----------------------------------------------------------------------------- norms and rotation of heads
// Queries and keys of the same rows: x[side][row][head][dh], heads of side 1 may be none.
struct NormRotary {
  const void* x[2];
  const void* dy[2];            // backward
  void* out[2];                 // forward: y; backward: dx
  const void* gamma[2];         // [dh], nullable = 1
  void* dgamma[2];              // [dh], nullable
  int64_t x_stride[2], dy_stride[2], out_stride[2];  // elements from row to row
  int heads[2];
  const int32_t* positions;     // [rows], nullable = no rotation
  int64_t rows;
  int dh, dtype;
  float base, eps;
};
constexpr int kMaxRotaryHead = 256;
bool norm_rotary_fits(const NormRotary& a);
hipError_t norm_rotary(const NormRotary& a, hipStream_t s);
size_t norm_rotary_backward_workspace(int64_t rows, int dh);
hipError_t norm_rotary_backward(const NormRotary& a, void* workspace, hipStream_t s);

}  // namespace lime
