// Rows in 8 bits with a scale each; the router's choice, the order by expert, and the way back.
#include "pipe_attention.h"
#include "pipe_codes.h"
#include "pipe_token.h"

namespace {

// ------------------------------------------------------------------ rows to codes
// s = max|x| / 127, c = rint(x / s): NT threads a row, 8 values a thread and step, the first CH steps kept in registers between the maximum
// and the codes, the rest (rows of more than 8 NT CH values) read again.  A row with a NaN or an infinity has the maximum +infinity here.
template <typename T, int NT, int CH, bool WIDE>
__global__ __launch_bounds__(256) void token_quantize_kernel(const T* __restrict__ x, int64_t rows, int in, int64_t stride, int pitch,
                                                             int8_t* __restrict__ codes, float* __restrict__ scales) {
  constexpr int PER = 256 / NT;
  const int64_t row = (int64_t)blockIdx.x * PER + threadIdx.x / NT;
  const int tid = threadIdx.x % NT;
  if (PER > 1 && row >= rows) return;      // (a whole wave: no barrier follows)
  const T* xr = x + row * stride;
  const int n_chunk = (in + 7) >> 3;
  auto fetch = [&](int c, float* v) __attribute__((always_inline)) {
    if (c * 8 + 8 <= in) {
      load8<T, WIDE>(xr + c * 8, v);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = c * 8 + i < in ? to_f(xr[c * 8 + i]) : 0.f;
    }
  };
  float v[CH][8];
#pragma unroll
  for (int j = 0; j < CH; ++j) fetch(tid + j * NT, v[j]);
  float top = 0.f;
  auto raise = [&](const float* a) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) top = raised(top, a[i]);
  };
#pragma unroll
  for (int j = 0; j < CH; ++j) raise(v[j]);
  for (int c = tid + CH * NT; c < n_chunk; c += NT) {
    float a[8];
    fetch(c, a);
    raise(a);
  }
  top = NT == 64 ? wave_max(top) : block_max(top);
  const RowScale scale(top);
  if (tid == 0) scales[row] = scale.scale();
  uint2* dst = reinterpret_cast<uint2*>(codes + row * pitch);
  auto put = [&](int c, const float* a) __attribute__((always_inline)) {
    if (c * 8 < pitch) dst[c] = scale.codes8(a);
  };
#pragma unroll
  for (int j = 0; j < CH; ++j) put(tid + j * NT, v[j]);
  for (int c = tid + CH * NT; c * 8 < pitch; c += NT) {
    float a[8];
    fetch(c, a);
    put(c, a);
  }
}

template <typename T, bool WIDE>
int quantize_typed(const void* x, int64_t rows, int in, int64_t stride, int pitch, int8_t* codes, float* scales, hipStream_t st) {
  const T* p = (const T*)x;
  if (pitch <= 2048 && rows > 512)
    PIPE_KLAUNCH((token_quantize_kernel<T, 64, 4, WIDE>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, st, p, rows, in, stride, pitch, codes, scales);
  else
    PIPE_KLAUNCH((token_quantize_kernel<T, 256, 4, WIDE>), dim3((unsigned)rows), dim3(256), 0, st, p, rows, in, stride, pitch, codes, scales);
  PIPE_HIP(hipGetLastError());
  return PIPE_OK;
}

// ------------------------------------------------------------------ the choice of experts
// A wave a token, lane l its logits l, l + 64, ...; each of the top_k steps is a maximum over the wave and a ballot a register, which finds the
// lowest index that holds it.  A NaN equals nothing and is never chosen.
template <typename T, int EL>
__global__ __launch_bounds__(256) void expert_route_kernel(const ExpertRouteArgs a) {
  const int t = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (t >= a.T) return;
  const T* row = (const T*)a.logits + (int64_t)t * a.row_stride;
  float v[EL];
#pragma unroll
  for (int i = 0; i < EL; ++i) v[i] = i * 64 + lane < a.E ? to_f(row[i * 64 + lane]) : -INFINITY;
  float chosen = -INFINITY;      // lane j: the j-th largest logit
  int expert = -1;
  float first = 0.f, total = 0.f;
  for (int j = 0; j < a.top_k; ++j) {
    float m = v[0];
#pragma unroll
    for (int i = 1; i < EL; ++i) m = fmaxf(m, v[i]);
    m = wave_max(m);
    if (!(m > -INFINITY)) break;
    int at = -1;
#pragma unroll
    for (int i = 0; i < EL; ++i) {
      const unsigned long long b = __ballot(v[i] == m);
      if (at < 0 && b != 0) at = i * 64 + __ffsll(b) - 1;
    }
    if (j == 0) {
      first = m;
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < EL; ++i) sum += expf(v[i] - m);
      total = sum;
    }
    if (lane == j) { chosen = m; expert = at; }
#pragma unroll
    for (int i = 0; i < EL; ++i)
      if (i * 64 + lane == at) v[i] = -INFINITY;
  }
  const float e = chosen > -INFINITY ? expf(chosen - first) : 0.f;
  if (a.renormalize) total = e;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o, 64);
  if (lane < a.top_k) {
    a.experts[(int64_t)t * a.top_k + lane] = expert;
    a.weights[(int64_t)t * a.top_k + lane] = expert >= 0 ? e / total : 0.f;
  }
}

// ------------------------------------------------------------------ the order by expert
// A workgroup an expert, and one for the pairs without one: it counts the pairs of the experts before it, which gives its first row, and writes
// the rows of its own in order.  Nothing passes between workgroups.
constexpr int SORT_NT = 1024;
__global__ __launch_bounds__(SORT_NT) void expert_sort_kernel(const int32_t* __restrict__ experts, int n, int E, int32_t* __restrict__ starts,
                                                              int32_t* __restrict__ order, int32_t* __restrict__ places) {
  __shared__ int below[SORT_NT / 64], own[SORT_NT / 64];
  const int e = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;      // e == E: none
  const int share = (n + SORT_NT - 1) / SORT_NT * 64;       // pairs of a wave, whole rounds of 64
  const int lo = min(n, wave * share), hi = min(n, lo + share);
  auto key = [&](int i) {
    const int k = experts[i];
    return (unsigned)k < (unsigned)E ? k : E;
  };
  int b = 0, o = 0;
  for (int i = lo + lane; i < hi; i += 64) {
    const int k = key(i);
    b += k < e;
    o += k == e;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) { b += __shfl_xor(b, d, 64); o += __shfl_xor(o, d, 64); }
  if (lane == 0) { below[wave] = b; own[wave] = o; }
  __syncthreads();
  int row = 0;
  for (int w = 0; w < SORT_NT / 64; ++w) row += below[w] + (w < wave ? own[w] : 0);
  if (threadIdx.x == 0) starts[e] = row;
  for (int i = lo; i < hi; i += 64) {
    const bool mine = i + lane < hi && key(i + lane) == e;
    const unsigned long long all = __ballot(mine);
    const int at = row + __popcll(all & ((1ull << lane) - 1));
    if (mine) {
      order[at] = e < E ? i + lane : -1;
      places[i + lane] = e < E ? at : -1;
    }
    row += __popcll(all);
  }
}

// ------------------------------------------------------------------ back to the tokens
// 8 values of a token a thread, the rows of its experts summed in fp32 in the order of its choices.
template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void expert_combine_kernel(const T* __restrict__ y, int64_t n, int H, int64_t stride, const int32_t* __restrict__ places,
                                                             const float* __restrict__ weights, int64_t items, int top_k, T* __restrict__ out) {
  const int chunks = (H + 7) >> 3;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (id >= items) return;
  const int64_t t = id / chunks;
  const int c = (int)(id - t * chunks) * 8, have = min(8, H - c);
  float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int j = 0; j < top_k; ++j) {
    const int64_t p = places[t * top_k + j];
    if (p < 0 || p >= n) continue;
    const float w = weights[t * top_k + j];
    const T* src = y + p * stride + c;
    float v[8];
    if (have == 8) {
      load8<T, WIDE>(src, v);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < have ? to_f(src[i]) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = fmaf(w, v[i], sum[i]);
  }
  T* dst = out + t * H + c;
  if (WIDE && have == 8) {
    Vec8<T> r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = from_f<T>(sum[i]);
    uint4 w[sizeof(T) / 2];
    __builtin_memcpy(w, &r, sizeof r);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(dst)[i] = w[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < have) dst[i] = from_f<T>(sum[i]);
  }
}

template <typename T>
int route_typed(const ExpertRouteArgs& a, hipStream_t st) {
  const dim3 grid((a.T + 3) / 4), block(256);
  if (a.E <= 64) PIPE_KLAUNCH((expert_route_kernel<T, 1>), grid, block, 0, st, a);
  else if (a.E <= 128) PIPE_KLAUNCH((expert_route_kernel<T, 2>), grid, block, 0, st, a);
  else if (a.E <= 256) PIPE_KLAUNCH((expert_route_kernel<T, 4>), grid, block, 0, st, a);
  else if (a.E <= 512) PIPE_KLAUNCH((expert_route_kernel<T, 8>), grid, block, 0, st, a);
  else PIPE_KLAUNCH((expert_route_kernel<T, 16>), grid, block, 0, st, a);
  PIPE_HIP(hipGetLastError());
  return PIPE_OK;
}

template <typename T>
int combine_typed(const void* y, int64_t n, int H, int64_t stride, const int32_t* places, const float* weights, int T_, int top_k, void* out,
                  hipStream_t st) {
  const int64_t items = (int64_t)T_ * ((H + 7) / 8);
  const dim3 grid((unsigned)((items + 255) / 256));
  constexpr int V = 16 / (int)sizeof(T);
  const bool wide = ((reinterpret_cast<uintptr_t>(y) | reinterpret_cast<uintptr_t>(out)) & 15) == 0 && stride % V == 0 && H % V == 0;
  if (wide)
    PIPE_KLAUNCH((expert_combine_kernel<T, true>), grid, dim3(256), 0, st, (const T*)y, n, H, stride, places, weights, items, top_k, (T*)out);
  else
    PIPE_KLAUNCH((expert_combine_kernel<T, false>), grid, dim3(256), 0, st, (const T*)y, n, H, stride, places, weights, items, top_k, (T*)out);
  PIPE_HIP(hipGetLastError());
  return PIPE_OK;
}

}  // namespace

int launch_token_quantize(const void* x, int type, int64_t rows, int in, int64_t stride, int pitch, int8_t* codes, float* scales, hipStream_t st) {
  const int n = 16 / type_size(type);
  const bool wide = (reinterpret_cast<uintptr_t>(x) & 15) == 0 && stride % n == 0;
  if (type == PIPE_F32) return wide ? quantize_typed<float, true>(x, rows, in, stride, pitch, codes, scales, st) : quantize_typed<float, false>(x, rows, in, stride, pitch, codes, scales, st);
  if (type == PIPE_F16) return wide ? quantize_typed<f16, true>(x, rows, in, stride, pitch, codes, scales, st) : quantize_typed<f16, false>(x, rows, in, stride, pitch, codes, scales, st);
  return wide ? quantize_typed<bf16, true>(x, rows, in, stride, pitch, codes, scales, st) : quantize_typed<bf16, false>(x, rows, in, stride, pitch, codes, scales, st);
}

int launch_expert_route(const ExpertRouteArgs& a, hipStream_t st) {
  if (a.type == PIPE_F32) return route_typed<float>(a, st);
  return a.type == PIPE_F16 ? route_typed<f16>(a, st) : route_typed<bf16>(a, st);
}

int launch_expert_sort(const int32_t* experts, int n, int E, int32_t* starts, int32_t* order, int32_t* places, hipStream_t st) {
  PIPE_KLAUNCH(expert_sort_kernel, dim3(E + 1), dim3(SORT_NT), 0, st, experts, n, E, starts, order, places);
  PIPE_HIP(hipGetLastError());
  return PIPE_OK;
}

int launch_expert_combine(const void* y, int type, int64_t n, int H, int64_t stride, const int32_t* places, const float* weights, int T, int top_k,
                          void* out, hipStream_t st) {
  if (type == PIPE_F32) return combine_typed<float>(y, n, H, stride, places, weights, T, top_k, out, st);
  return type == PIPE_F16 ? combine_typed<f16>(y, n, H, stride, places, weights, T, top_k, out, st) : combine_typed<bf16>(y, n, H, stride, places, weights, T, top_k, out, st);
}
