// Host-visible launch interface of the operators on a caller's matrices: products with 8-bit weights (f8.hip) and rules on logits
// (rules.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"

namespace onmt {

// Element types of a caller's matrices (ONMT_F32, ONMT_BF16, ONMT_F16).
enum { kF32 = 0, kBF16 = 1, kF16 = 2 };

// A matrix of e4m3 values with a power of two per row and block of 128 columns, in fragment blocks (f8.hip).
constexpr int kF8Block = 128;
constexpr int kF8Frag = 16 * kF8Block;         // bytes of a fragment block
struct F8Mat {
  char* data;
  int* exps;
  int rblocks, kblocks;
  __host__ __device__ int kquads() const { return (kblocks + 3) / 4; }
};
// Bytes of the fragment blocks and of the powers behind them.
inline size_t f8_data_bytes(int64_t rows, int cols) {
  return (size_t)((rows + 15) / 16) * ((cols + kF8Block - 1) / kF8Block) * kF8Frag;
}
inline size_t f8_exp_bytes(int64_t rows, int cols) {
  return (size_t)((rows + 15) / 16) * (((cols + kF8Block - 1) / kF8Block + 3) / 4) * 64;
}
inline F8Mat f8_mat(void* buf, int64_t rows, int cols) {
  return F8Mat{(char*)buf, (int*)((char*)buf + f8_data_bytes(rows, cols)), (int)((rows + 15) / 16), (cols + kF8Block - 1) / kF8Block};
}
hipError_t f8_pack(const void* x, int dtype, int64_t ld, int rows, int cols, const F8Mat& out, hipStream_t st);
hipError_t f8_unpack(const F8Mat& w, int rows, int cols, float* out, int64_t ld, hipStream_t st);
// The generator's partials of fp32 results: largest value and sum of exp per row and 128 columns, [M, ntiles].
struct F8Partials {
  float* max;
  float* sum;
  int ntiles;
};
// out [M, N] (row stride ld) = x w^T + bias (optional), x [M, cols] rounded to e4m3 in ws (f8_linear_ws bytes) first. part
// (optional): partials that are wanted too; its pointers are null afterwards if this product has not written them.
size_t f8_linear_ws(int M, int cols);
hipError_t f8_linear(const void* x, int dtype, int64_t ldx, int M, const F8Mat& w, int N, int cols, const float* bias, void* out,
                     int out_dtype, int64_t ld, void* ws, hipStream_t st, F8Partials* part = nullptr);

// Rules on logits (rules.hip); the pointers of rules that are off are null.
struct LogitRules {
  const int32_t* history;       // row r: history_len[r] ids from r * history_stride on
  const int32_t* history_len;
  int64_t history_stride;
  int max_history;
  const float* repetition;      // [N]
  const float* presence;
  const float* frequency;
  int ngram;
  const int32_t* bias_ids;      // row r: n_bias entries from r * bias_stride on
  const float* bias;
  int64_t bias_stride;
  int n_bias;
  const uint32_t* mask;         // n_masks rows of mask_stride words
  int64_t mask_stride;
  int n_masks;
  const int32_t* mask_row;
};
struct LogitMat {
  const void* x;
  int dtype;
  int64_t ld;
  int N, V;
};
// out [N, V] in the logits' own type.
hipError_t rules_logits(const LogitRules& r, const LogitMat& m, void* out, int64_t ld_out, hipStream_t st);
// Scratch of the calls below (K = 0: log-probabilities).
size_t rules_ws(int N, int V, int K);
// out, ids [N, K] = the K largest log-probabilities; lse optional.
hipError_t rules_top(const LogitRules& r, const LogitMat& m, int K, void* ws, float* out, int32_t* ids, float* lse,
                     hipStream_t st);
// logp [N, V]; lse optional.
hipError_t rules_log_probs(const LogitRules& r, const LogitMat& m, void* ws, float* logp, int64_t ld_out, float* lse,
                           hipStream_t st);

// The generator's partials (p.pmax, p.psum, with filters p.pfmax) of M rows of logits that another product left in p.logits.
hipError_t tile_partials(const GenParams& p, int M, hipStream_t st);

}  // namespace onmt
