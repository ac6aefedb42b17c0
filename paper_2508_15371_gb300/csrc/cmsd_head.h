// Internal declarations of the head's loss and of its 8-bit product, shared by
// their kernels and the C-ABI layer.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace cmsd {

// The head's loss and its gradients (cmsd_head_loss.cu).  Kept rows (those
// with a label) are packed to the front of a copy of the hidden states, so
// that ignored rows cost no products and their contents reach no sum.
constexpr int kHeadTile = 256;                  // rows of a packed block, columns of a vocabulary tile
constexpr int kHeadPart = 128;                  // vocabulary entries per partial statistic of the loss
constexpr int kFewParts = 152;                  // partial statistics at most where there are few rows
struct HeadLossArgs {
  const uint16_t* hidden;        // bf16 [R][d]
  const uint16_t* weight;        // bf16 [V][d]
  const int* labels;             // [R]
  int R, d, V, ignore;
  int Rp;                        // R rounded up to kHeadTile
  float* loss;                   // forward
  float* lse;
  const float* lse_in;           // backward
  const float* grad;
  uint16_t* d_hidden;
  uint16_t* d_weight;
  // workspace
  unsigned* err;
  int* n;                        // [1] kept rows
  int* pos;                      // [R] packed place of each row, -1: ignored
  int* lab;                      // [Rp] label of each packed row
  float* plse;                   // [Rp] lse and gradient of each packed row (backward)
  float* pgrad;
  uint16_t* packed;              // bf16 [Rp][d], zeros from row n to the next multiple of 64
  float* zlab;                   // [Rp] logit of the label (forward)
  float2* part;                  // [max(ceil(V / kHeadPart), kFewParts)][Rp] (maximum, sum) in base 2 (forward)
  int Vc;                        // vocabulary entries per piece, a multiple of kHeadTile (backward)
  int split;                     // parts that a piece's sum for d_hidden is cut into
  uint16_t* dz;                  // bf16 [Rp][Vc]
  float* dh;                     // [split][Rp][d]
};
int head_split(int Rp, int d, int Vc);
cudaError_t launch_head_loss(const HeadLossArgs& a, cudaStream_t s);
cudaError_t launch_head_loss_backward(const HeadLossArgs& a, cudaStream_t s);
cudaError_t take_head_loss_errors(unsigned* flags, cudaStream_t s);
cudaError_t launch_test_wait(unsigned* err, int arrive, cudaStream_t s);

// 8-bit rows and the product of the head in 8-bit integers (cmsd_head_i8.cu).
struct HeadI8Args {
  const int8_t* hidden;          // [R][d]
  const int8_t* weight;          // [V][d]
  const float* hidden_scale;
  const float* weight_scale;
  int R, d, V, dtype;
  void* logits;                  // dtype [R][V]
  unsigned* err;
  uint16_t* h16;                 // fp16 [R][d]: the hidden integers as the tensor cores take them
  int* mag;                      // [R] sum of each token's magnitudes
};
cudaError_t launch_quantize_rows(const void* x, int dtype, int R, int d, int8_t* q, float* scale, cudaStream_t s);
cudaError_t launch_head_i8(const HeadI8Args& a, cudaStream_t s);
cudaError_t take_head_i8_errors(unsigned* flags, cudaStream_t s);

}  // namespace cmsd
