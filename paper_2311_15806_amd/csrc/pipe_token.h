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
int launch_token_layer(TokenProductArgs& a, int8_t* codes, float* scales, hipStream_t st);   // (codes, scales: room for the inputs', or nullptr)
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
// The larger of m and |x| as bit patterns, which order as the magnitudes do, an infinity and NaN behind all others.
__device__ __forceinline__ uint32_t raised(uint32_t m, float x) { return max(m, __float_as_uint(x) & 0x7fffffffu); }
// ... as a number, +infinity where the row is not finite as a whole
__device__ __forceinline__ float top_of(uint32_t m) { return __uint_as_float(min(m, 0x7f800000u)); }
// The codes of a row whose largest magnitude is `top`: s = top / 127, c = rint(x / s).  No quotient lies beyond 127 by more than its own rounding: nothing
// is bounded but by that.
struct RowScale {
  float s, y;
  bool live, bad, fast;
  __device__ __forceinline__ explicit RowScale(float top) {
    bad = !(top < INFINITY);
    s = __fdiv_rn(top, 127.f);
    if (s < 0x1p-126f) s = 0.f;
    live = s > 0.f && !bad;
    y = live ? __fdiv_rn(1.f, s) : 0.f;
    fast = s > 1e-27f && s < 1e27f;
  }
  __device__ __forceinline__ float scale() const { return bad ? __uint_as_float(0x7fc00000u) : s; }
  // (the correctly rounded quotient by two corrections, as Divisor's, within its range; sums are left apart whatever the file's contraction)
  template <bool FAST>
  __device__ __forceinline__ int code(float x) const {
    if (!FAST) return (int)rintf(__fdiv_rn(x, s));
    float q = __fmul_rn(x, y);
    q = __fmaf_rn(__fmaf_rn(-q, s, x), y, q);
    return (int)rintf(__fmaf_rn(__fmaf_rn(-q, s, x), y, q));
  }
  template <bool FAST>
  __device__ __forceinline__ uint2 eight(const float* x) const {
    return make_uint2(pack4(code<FAST>(x[0]), code<FAST>(x[1]), code<FAST>(x[2]), code<FAST>(x[3])),
                      pack4(code<FAST>(x[4]), code<FAST>(x[5]), code<FAST>(x[6]), code<FAST>(x[7])));
  }
  __device__ __forceinline__ uint2 codes8(const float* x) const {
    if (!live) return make_uint2(0, 0);
    return fast ? eight<true>(x) : eight<false>(x);
  }
};
#endif
