// Attention over packed sequences.
#include "pipe_attention.h"

namespace {

// One wave per query row: 64 keys at a time, a lane per key for the scores, a lane per D/64 values for the output.
template <typename T, int D>
__global__ __launch_bounds__(64) void prompt_attn_kernel(PromptAttnArgs a) {
  __shared__ float sq[D], sp[64];
  const int t = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
  const int kvh = h / (a.Hq / a.Hkv);
  int b = -1;
  for (int i0 = 0; i0 < a.B; i0 += 64)
    b += __popcll(__ballot(i0 + lane < a.B && a.q_starts[min(i0 + lane, a.B)] <= t));
  const bool mine = b >= 0 && t < a.q_starts[a.B];
  int k0 = 0, seen = 0;
  if (mine) {
    k0 = max(0, min(a.k_starts[b], a.Tk));
    seen = min(a.k_starts[b + 1], a.Tk) - k0;
    if (a.causal) seen = min(seen, seen - (a.q_starts[b + 1] - t) + 1);
  }
  for (int i = lane; i < D; i += 64) sq[i] = to_f(((const T*)a.q)[(int64_t)t * a.qs.token + (int64_t)h * a.qs.head + i]);
  __syncthreads();
  float top = -INFINITY, sum = 0, o[D / 64] = {};
  for (int t0 = 0; t0 < seen; t0 += 64) {
    const int n = min(64, seen - t0);
    float S = -INFINITY;
    if (lane < n) {
      const T* kp = (const T*)a.k + (int64_t)(k0 + t0 + lane) * a.ks.token + (int64_t)kvh * a.ks.head;
      float dot = 0;
      for (int i = 0; i < D; ++i) dot = fmaf(sq[i], to_f(kp[i]), dot);
      S = dot * a.scale;
    }
    float mx = S;
    for (int d = 32; d; d >>= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
    const float ntop = fmaxf(top, mx);
    const float ref = ntop == -INFINITY ? 0.f : ntop, f = expf(top - ref);
    top = ntop;
    const float p = expf(S - ref);
    sum = sum * f + p;
    for (int i = 0; i < D / 64; ++i) o[i] *= f;
    sp[lane] = p;
    __syncthreads();
    for (int j = 0; j < n; ++j) {
      const T* vp = (const T*)a.v + (int64_t)(k0 + t0 + j) * a.vs.token + (int64_t)kvh * a.vs.head;
      for (int i = 0; i < D / 64; ++i) o[i] = fmaf(sp[j], to_f(vp[lane + 64 * i]), o[i]);
    }
    __syncthreads();
  }
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
  const bool none = top == -INFINITY && sum == 0.f;
  for (int i = 0; i < D / 64; ++i)
    ((T*)a.out)[((int64_t)t * a.Hq + h) * D + lane + 64 * i] = from_f<T>(none ? 0.f : o[i] / sum);
}

template <typename T>
int run(const PromptAttnArgs& a, hipStream_t st) {
  const dim3 grid(a.Tq, a.Hq);
  if (a.D == 64) PIPE_KLAUNCH((prompt_attn_kernel<T, 64>), grid, dim3(64), 0, st, a);
  else PIPE_KLAUNCH((prompt_attn_kernel<T, 128>), grid, dim3(64), 0, st, a);
  PIPE_HIP(hipGetLastError());
  return PIPE_OK;
}

}  // namespace

int launch_prompt_attention(const PromptAttnArgs& a, hipStream_t st) {
  if (a.Tq == 0) return PIPE_OK;
  return a.type == PIPE_F32 ? run<float>(a, st) : a.type == PIPE_F16 ? run<f16>(a, st) : run<bf16>(a, st);
}
