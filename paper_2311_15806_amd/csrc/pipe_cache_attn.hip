// Attention of fresh tokens over the 4-bit cache.
#include "pipe_attention.h"

namespace {

// One wave per query row: 64 cached tokens at a time, a lane per token for the scores, a lane per D/64 values for the output.
template <typename T, int D>
__global__ __launch_bounds__(64) void cache_attn_kernel(CacheAttnArgs a) {
  __shared__ float sq[D], sp[64], sps[64];
  __shared__ int srow[64];
  const int t = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
  const int kvh = h / (a.Hq / a.cache.Hkv);
  const int shift = a.cache.shift, P = 1 << shift;
  // the request of this token: the last one that starts at or before it
  int b = -1;
  for (int i0 = 0; i0 < a.B; i0 += 64) {
    const unsigned long long m = __ballot(i0 + lane < a.B && a.starts[min(i0 + lane, a.B)] <= t);
    b += __popcll(m);
  }
  const bool mine = b >= 0 && t < a.starts[a.B];
  int seen = 0;
  if (mine) seen = min(a.lengths[b], (int)min((int64_t)a.width << shift, (int64_t)0x7fffffff)) ;
  const int full = mine ? a.lengths[b] : 0;
  if (mine) seen = min(seen, full - (a.starts[b + 1] - t) + 1);
  float qsum = 0;
  for (int i = lane; i < D; i += 64) sq[i] = to_f(((const T*)a.q)[(int64_t)t * a.qs.token + (int64_t)h * a.qs.head + i]);
  __syncthreads();
  for (int i = 0; i < D; ++i) qsum += sq[i];
  float top = -INFINITY, sum = 0, o[D / 64] = {}, om = 0;
  const int64_t bytes = (int64_t)P * (D + 8);
  for (int t0 = 0; t0 < seen; t0 += 64) {
    const int tok = t0 + lane;
    float S = -INFINITY, vs = 0, vm = 0;
    int page = -1;
    const uint8_t* blk = nullptr;
    if (tok < seen) page = a.table[(int64_t)b * a.width + (tok >> shift)];
    const int off = tok & (P - 1);
    if (page >= 0 && page < a.cache.n_pages) {
      blk = a.cache.base + ((int64_t)page * a.cache.Hkv + kvh) * bytes;
      const uint32_t kw = *(const uint32_t*)(blk + P * D + 4 * off), vw = *(const uint32_t*)(blk + P * D + 4 * P + 4 * off);
      float dot = 0;
      for (int w = 0; w < D / 8; ++w) {
        const uint32_t x = ((const uint32_t*)(blk + off * (D / 2)))[w];
        for (int i = 0; i < 8; ++i) dot = fmaf(sq[8 * w + i], (float)((x >> (4 * i)) & 15u), dot);
      }
      S = (word_scale(kw) * dot + word_offset(kw) * qsum) * a.scale;
      vs = word_scale(vw);
      vm = word_offset(vw);
    }
    float mx = S;
    for (int d = 32; d; d >>= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
    const float ntop = fmaxf(top, mx);
    const float ref = ntop == -INFINITY ? 0.f : ntop, f = expf(top - ref);
    top = ntop;
    const float p = blk ? expf(S - ref) : 0.f;
    sum = sum * f + p;
    om = om * f + (blk ? p * vm : 0.f);
    for (int i = 0; i < D / 64; ++i) o[i] *= f;
    sps[lane] = blk ? p * vs : 0.f;
    srow[lane] = blk ? page : -1;
    __syncthreads();
    for (int j = 0; j < 64; ++j) {
      if (srow[j] < 0) continue;
      const uint8_t* vb = a.cache.base + ((int64_t)srow[j] * a.cache.Hkv + kvh) * bytes + P * D / 2 + ((t0 + j) & (P - 1)) * (D / 2);
      for (int i = 0; i < D / 64; ++i) {
        const int d = lane + 64 * i;
        o[i] = fmaf(sps[j], (float)((vb[d >> 1] >> (4 * (d & 1))) & 15), o[i]);
      }
    }
    __syncthreads();
  }
  for (int d = 32; d; d >>= 1) { sum += __shfl_xor(sum, d); om += __shfl_xor(om, d); }
  const bool none = top == -INFINITY && sum == 0.f;
  for (int i = 0; i < D / 64; ++i)
    ((T*)a.out)[((int64_t)t * a.Hq + h) * D + lane + 64 * i] = from_f<T>(none ? 0.f : (o[i] + om) / sum);
}

template <typename T>
int run(const CacheAttnArgs& a, hipStream_t st) {
  const dim3 grid(a.T, a.Hq);
  if (a.D == 64) PIPE_KLAUNCH((cache_attn_kernel<T, 64>), grid, dim3(64), 0, st, a);
  else PIPE_KLAUNCH((cache_attn_kernel<T, 128>), grid, dim3(64), 0, st, a);
  PIPE_HIP(hipGetLastError());
  return PIPE_OK;
}

}  // namespace

int launch_cache_attention(const CacheAttnArgs& a, hipStream_t st) {
  if (a.T == 0) return PIPE_OK;
  return a.type == PIPE_F32 ? run<float>(a, st) : a.type == PIPE_F16 ? run<f16>(a, st) : run<bf16>(a, st);
}
