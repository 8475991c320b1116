// Shared by the cache and attention kernels (pipe_cache.hip, pipe_cache_attn.hip, pipe_prompt_attn.hip).
#pragma once
#include "pipe_internal.h"

// The layout of a cache page is stated in pipe.h; a block is one head's part of one page.
constexpr int PIPE_PLAN_MAX_B = 4096;

struct CacheView {
  uint8_t* base;
  int n_pages, shift, Hkv;   // P = 1 << shift
};

// page sizes that exist, as the power of two; -1 otherwise
static inline int pipe_page_shift(int P) {
  for (int s = 4; s <= 8; ++s)
    if (P == 1 << s) return s;
  return -1;
}

struct HeadStrides {
  int64_t token, head;   // in elements
};
static inline int type_size(int type) { return type == PIPE_F32 ? 4 : 2; }
// whether every row of 8 values is 16-byte aligned
static inline bool rows_wide(const void* p, HeadStrides s, int type) {
  const int n = 16 / type_size(type);
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && s.token % n == 0 && s.head % n == 0;
}

int launch_cache_plan(const int32_t* cached, const int32_t* fresh, int B, int shift, const int32_t* free_list, int n_free,
                      const int32_t* used, int32_t* table, int width, int T, int32_t* lengths, int32_t* starts,
                      int32_t* slots, int32_t* positions, int32_t* counts, hipStream_t st);
int launch_cache_write(const void* k, const void* v, int type, int T, int D, HeadStrides ks, HeadStrides vs,
                       const int32_t* slots, CacheView c, hipStream_t st);
int launch_cache_read(CacheView c, const int32_t* slots, int T, int D, int type, void* k, void* v, hipStream_t st);

struct CacheAttnArgs {
  const void* q;
  HeadStrides qs;
  const int32_t *starts, *lengths, *table;
  CacheView cache;
  int type, T, Hq, D, B, width, max_length;
  float scale;
  void* out;
};
int launch_cache_attention(const CacheAttnArgs& a, hipStream_t st);

struct PromptAttnArgs {
  const void *q, *k, *v;
  HeadStrides qs, ks, vs;
  const int32_t *q_starts, *k_starts;
  int type, Tq, Tk, Hq, Hkv, D, B, causal;
  float scale;
  void* out;
};
int launch_prompt_attention(const PromptAttnArgs& a, hipStream_t st);

#if defined(__HIPCC__)
using bf16 = __bf16;
using f16 = _Float16;
__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(f16 x) { return (float)x; }
__device__ __forceinline__ float to_f(bf16 x) { return (float)x; }
template <typename T>
__device__ __forceinline__ T from_f(float x) { return (T)x; }
// 8 values from p; WIDE: p is 16-byte aligned
template <typename T>
struct Vec8 { T v[8]; };
template <typename T, bool WIDE>
__device__ __forceinline__ void load8(const T* p, float* x) {
  if constexpr (WIDE) {
    Vec8<T> r;
    uint4 w[sizeof(T) / 2];
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
    __builtin_memcpy(&r, w, sizeof r);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = to_f(r.v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = to_f(p[i]);
  }
}
// N values to p, which is aligned to their size (a power of two up to 32 bytes)
template <typename T, int N>
__device__ __forceinline__ void store_row(T* p, const float* x) {
  struct alignas(N * sizeof(T) < 16 ? N * sizeof(T) : 16) Row { T v[N]; } r;
#pragma unroll
  for (int i = 0; i < N; ++i) r.v[i] = from_f<T>(x[i]);
  *reinterpret_cast<Row*>(p) = r;
}
// minimum / maximum over the LANES (8 or 16) lanes of a row
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
template <int LANES, bool MAX>
__device__ __forceinline__ float row_reduce(float x) {
  auto op = [](float a, float b) { return MAX ? fmaxf(a, b) : fminf(a, b); };
  x = op(x, dpp<0xB1>(x));    // lane ^ 1
  x = op(x, dpp<0x4E>(x));    // lane ^ 2
  x = op(x, dpp<0x141>(x));   // 7 - lane within 8
  if (LANES == 16) x = op(x, dpp<0x140>(x));   // 15 - lane
  return x;
}
__device__ __forceinline__ float word_scale(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float word_offset(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
#endif
