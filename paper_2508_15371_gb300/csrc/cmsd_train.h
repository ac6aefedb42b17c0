// Internal declarations of what lies below the head in training -- embedding,
// layer norm, dropout -- shared by their kernels and the C-ABI layer.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace cmsd {

// Rows of the token table and their gradient (cmsd_embed.cu).
struct EmbedArgs {
  const int* tokens;             // [R]
  const void* table;             // [V][d] (forward)
  void* x;                       // [R][d] (forward)
  const void* d_x;               // [R][d] (backward)
  void* d_table;                 // [V][d] (backward)
  int dtype, R, d, V, ignore, add;
  float scale;
  int passes, bits, tile;        // radix passes, key bits of each, rows of a tile (backward)
  int slots;                     // rows of a tile of the sums
  size_t fill[6];                // borders of the bytes that each launch that orders rows fills with zeros
  // workspace (backward)
  unsigned* err;
  unsigned* key[2];              // [R] the rows' tokens in order (V: padding), where pass p writes: [p & 1]
  int* order[2];                 // [R] the rows
  int* count[4];                 // [tiles of rows][1 << bits] rows of each digit
  int2* state;                   // [tiles of the sums]
  float* head;                   // [tiles][d] pieces of sums that tiles' borders cut
  float* tail;
};
size_t embed_layout(EmbedArgs& a, char* w);
cudaError_t launch_embed(const EmbedArgs& a, cudaStream_t s);
cudaError_t launch_embed_backward(const EmbedArgs& a, cudaStream_t s);
cudaError_t take_embed_errors(unsigned* flags, cudaStream_t s);

// Layer norm and its gradients (cmsd_norm.cu).
struct NormArgs {
  const void* x;                 // [R][d]
  const void* weight;            // wdtype [d], null: ones
  const void* bias;              // wdtype [d], null: zeros
  int dtype, wdtype, R, d;
  float eps;
  void* y;                       // [R][d] (forward)
  float* mean;                   // [R], may be null (forward)
  float* rstd;
  const float* mean_in;          // backward
  const float* rstd_in;
  const void* d_y;               // [R][d]
  void* d_x;                     // [R][d], may be null
  void* d_weight;                // wdtype [d], may be null
  void* d_bias;
  // workspace (backward)
  float* part;
};
size_t norm_layout(NormArgs& a, char* w);
cudaError_t launch_norm(const NormArgs& a, cudaStream_t s);
cudaError_t launch_norm_backward(const NormArgs& a, cudaStream_t s);

// Dropout (cmsd_dropout.cu).
struct DropArgs {
  const void* x;                 // [n]
  const void* residual;          // [n], may be null
  void* y;                       // [n]
  int dtype;
  int64_t n;
  uint32_t drop;                 // an entry whose 16 bits are below is dropped
  float scale;                   // of the kept entries
  uint64_t seed;
  uint32_t iteration, site;
  const uint32_t* step;          // added to iteration, may be null
};
cudaError_t launch_dropout(const DropArgs& a, cudaStream_t s);

}  // namespace cmsd
