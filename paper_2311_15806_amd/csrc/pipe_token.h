// Shared by the calls with a scale for each token and the experts' calls (pipe_token.hip, pipe_token_gemm.hip).
#pragma once
#include "pipe_internal.h"

constexpr int PIPE_TOKEN_PITCH = 128;        // a row of codes is padded with zeros to a multiple of this
constexpr int PIPE_TOKEN_MAX_IN = 131072 - PIPE_TOKEN_PITCH;   // sums of products of codes stay below 2^31
constexpr int PIPE_EXPERTS_MAX = 1024, PIPE_TOP_K_MAX = 32;

int launch_token_quantize(const void* x, int type, int64_t rows, int in, int64_t row_stride, int pitch, int8_t* codes, float* scales,
                          hipStream_t st);

struct TokenProductArgs {
  const int8_t* qx;        // codes [n_x][pitch] and scales [n_x] of the inputs
  const float* sx;
  const int8_t* w;         // [E][rows][pitch], rows = out, or 2 out of a gated layer (gate rows first)
  const float* sw;         // [E][rows]
  const float* bias;       // [E][rows] or nullptr
  const int32_t* starts;   // [E + 1], rows of y by expert; nullptr: one layer, all rows
  const int32_t* order;    // [n]: row r of y is input order[r] / top_k (outside: zeros); nullptr: input r
  int64_t n_x, n;          // rows of the inputs and of y
  int top_k, E, pitch, out, act, type;
  void* y;                 // [n][out]
};
int launch_token_product(const TokenProductArgs& a, hipStream_t st);
extern int g_token_kernel;   // 0: by the sizes; 1 to 4: see pipe_set_token_kernel

struct ExpertRouteArgs {
  const void* logits;
  int type, T, E, top_k, renormalize;
  int64_t row_stride;
  int32_t* experts;
  float* weights;
};
int launch_expert_route(const ExpertRouteArgs& a, hipStream_t st);
int launch_expert_sort(const int32_t* experts, int n, int E, int32_t* starts, int32_t* order, int32_t* places, hipStream_t st);
int launch_expert_combine(const void* y, int type, int64_t n, int H, int64_t row_stride, const int32_t* places, const float* weights, int T,
                          int top_k, void* out, hipStream_t st);
