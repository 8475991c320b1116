// Shared by the calls with a scale for each token and the experts' calls (pipe_token.hip, pipe_token_gemm.hip).
#pragma once
#include "pipe_internal.h"

constexpr int PIPE_TOKEN_PITCH = 128;        // a row of codes is padded with zeros to a multiple of this
constexpr int PIPE_TOKEN_MAX_IN = 131072 - PIPE_TOKEN_PITCH;   // sums of products of codes stay below 2^31
constexpr int PIPE_EXPERTS_MAX = 1024, PIPE_TOP_K_MAX = 32;

int launch_token_quantize(const void* x, int type, int64_t rows, int in, int64_t row_stride, int pitch, int8_t* codes, float* scales,
                          hipStream_t st);

struct TokenProductArgs {
  const void* x;           // inputs [n_x], `in` values each
  int64_t x_stride;
  int in, x_wide;          // x_wide: rows can be read 16 bytes at a time
  const int8_t* qx;        // their codes [n_x][pitch] and scales [n_x], where a launch of their own made them
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
int launch_token_layer(TokenProductArgs& a, int8_t* codes, float* scales, hipStream_t st);   // (codes, scales: room for the inputs')
extern int g_token_kernel;   // 0: by the sizes; 1 to 4: see pipe_set_token_kernel

struct ExpertRouteArgs {
  const void* logits;
  int type, T, E, top_k, renormalize;
  int64_t row_stride;
  int32_t* experts;
  float* weights;
};
int64_t expert_sort_scratch(int T, int top_k, int E);      // bytes
int launch_expert_route(const ExpertRouteArgs& a, int32_t* starts, int32_t* order, int32_t* places, void* scratch, hipStream_t st);   // (T > 0)
int launch_expert_sort(const int32_t* experts, int T, int top_k, int E, int32_t* starts, int32_t* order, int32_t* places, void* scratch,
                       hipStream_t st);
int launch_expert_combine(const void* y, int type, int64_t n, int H, int64_t row_stride, const int32_t* places, const float* weights, int T,
                          int top_k, void* out, hipStream_t st);

#if defined(__HIPCC__)
#include "pipe_codes.h"
// the larger of m and |x|; +infinity from a NaN or an infinity on
__device__ __forceinline__ float raised(float m, float x) {
  const float v = fabsf(x);
  return v < INFINITY ? fmaxf(m, v) : INFINITY;
}
// The codes of a row whose largest magnitude is `top` (+infinity: it is not finite as a whole): s = top / 127, c = rint(x / s).
struct RowScale {
  float s;
  bool bad;
  Divisor d;
  __device__ __forceinline__ explicit RowScale(float top) : s(normal(__fdiv_rn(top, 127.f))), bad(!(top < INFINITY)), d(s > 0.f && !bad ? s : 1.f) {}
  static __device__ __forceinline__ float normal(float s) { return s < 0x1p-126f ? 0.f : s; }
  __device__ __forceinline__ float scale() const { return bad ? __uint_as_float(0x7fc00000u) : s; }
  __device__ __forceinline__ uint2 codes8(const float* x) const {
    int q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float r = d.fast ? d.quotient<true>(x[i]) : d.quotient<false>(x[i]);
      q[i] = s > 0.f && !bad ? (int)__builtin_amdgcn_fmed3f(rintf(r), -127.f, 127.f) : 0;
    }
    return make_uint2(pack4(q[0], q[1], q[2], q[3]), pack4(q[4], q[5], q[6], q[7]));
  }
};
#endif
