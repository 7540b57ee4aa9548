// Launch interface of the operators between a hidden state and a committed token: 8-bit codes of rows (quant_i8.cu),
// products of such codes (gemm_i8.cu), the rules of constrained decoding on logits (logit_rules.cu).
#pragma once
#include "common.cuh"

namespace bs {

struct QuantI8Args {
  const void* x;          // [x_rows][ldx] bf16 or fp32
  long long ldx;
  int f32;
  const int* idx;         // nullable: row m of the output is row idx[m] of x
  int x_rows;
  const bf16* gain;       // nullable: RMS norm with this gain before the rounding
  float eps;
  int8_t* codes;          // [M][ldc]
  long long ldc;
  float* scale;           // [M]
  int M, K;
  int* error_flag;
};
cudaError_t launch_quant_i8(const QuantI8Args& a, cudaStream_t s);

struct GemmI8Args {
  const int8_t* A;        // [M][lda]
  long long lda;
  const float* sa;        // [M]
  const int8_t* W;        // [N][ldw]
  const int8_t* W2;       // mode 3
  long long ldw;
  const float* sw;        // [N]
  const float* sw2;       // mode 3
  void* C;
  long long ldc;
  int M, N, K, mode;
  int* error_flag;
};
constexpr int kGemmI8MaxK = 131071;   // codes reach -128: 131071 * 128 * 128 is the last sum below 2^31
cudaError_t launch_gemm_i8(const GemmI8Args& a, cudaStream_t s);

// The rules of constrained decoding; nullable members are absent rules.
struct RulesArgs {
  const void* logits;     // [n_rows][ld] fp32 or bf16
  long long ld;
  int bf16_logits;
  int n_rows, vocab, n_reqs, mask_id;
  const int* row_req;     // nullable: row r belongs to request r
  const int* ctx;
  long long ctx_total;
  const int *ctx_begin, *ctx_gen, *ctx_end;
  const float *repetition, *presence, *frequency;
  const int* bias_at;
  const int* bias_tok;
  const float* bias_val;
  long long bias_total;
  const unsigned* allowed;
  long long allowed_ld;
  int n_masks;
  const int* row_mask;    // nullable: row r has mask r
  int* error_flag;
};
constexpr int kRulesMaxVocab = 524288;
cudaError_t launch_logit_rules(const RulesArgs& a, void* out, long long out_ld, cudaStream_t s);
cudaError_t launch_rules_confidence(const RulesArgs& a, int* tok, float* conf, cudaStream_t s);

}  // namespace bs
