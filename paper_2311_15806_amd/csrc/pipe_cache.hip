// The 4-bit key/value cache: tables of a step, writing rows, reading them back.
#include "pipe_attention.h"

namespace {

// ------------------------------------------------------------------ tables of a step
// Every workgroup scans the requests for itself (at most 4096 of them, 16 KiB from L2) and then makes its own share of the
// slots and of the new table entries: one launch, nothing passed between workgroups, no order of theirs in the result.
// Bound by latency, the scan's and three trips to memory: 64 requests of one token 5.6 us, 200 prompts of 192285 tokens 6.2 us (1.5 MB of
// slots and positions written; one search a slot in place of one for four: 17.2 us).
constexpr int PLAN_NT = 256;
constexpr int PLAN_EACH = 4;                      // consecutive slots of a thread: one search for their request
constexpr int PLAN_TOKENS = PLAN_EACH * PLAN_NT;  // slots of a workgroup

__device__ __forceinline__ uint32_t capped_add(uint32_t a, uint32_t b, uint32_t cap) {   // both <= cap < 2^31
  const uint32_t s = a + b;
  return s < cap ? s : cap;
}

// exclusive scan of one value per thread with addition capped at `cap` (associative for values >= 0); *total: the sum of all
__device__ uint32_t block_scan(uint32_t v, uint32_t cap, uint32_t* wave_sum, uint32_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t inc = v;
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_up(inc, d);
    if (lane >= d) inc = capped_add(inc, o, cap);
  }
  uint32_t exc = __shfl_up(inc, 1);
  if (lane == 0) exc = 0;
  __syncthreads();
  if (lane == 63) wave_sum[wave] = inc;
  __syncthreads();
  uint32_t before = 0, all = 0;
  for (int w = 0; w < PLAN_NT / 64; ++w) {
    if (w == wave) before = all;
    all = capped_add(all, wave_sum[w], cap);
  }
  *total = all;
  return capped_add(before, exc, cap);
}

// the last request whose first item is at or before i (items: tokens or new pages); first[n] holds the total
__device__ __forceinline__ int owner_of(const uint32_t* first, int n, uint32_t i) {
  int lo = 0, hi = n;   // first[lo] <= i, first[hi] > i
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= i) lo = mid; else hi = mid;
  }
  return lo;
}

__global__ __launch_bounds__(PLAN_NT) void cache_plan_kernel(
    const int32_t* __restrict__ cached, const int32_t* __restrict__ fresh, int B, int shift,
    const int32_t* __restrict__ free_list, int n_free, const int32_t* __restrict__ used, int32_t* table, int width, int T,
    int32_t* __restrict__ lengths, int32_t* __restrict__ starts, int32_t* __restrict__ slots,
    int32_t* __restrict__ positions, int32_t* __restrict__ counts) {
  __shared__ uint32_t tok0[PIPE_PLAN_MAX_B + 1], page0[PIPE_PLAN_MAX_B + 1], held[PIPE_PLAN_MAX_B];
  __shared__ uint32_t wave_sum[PLAN_NT / 64];
  const int per = (B + PLAN_NT - 1) / PLAN_NT;
  const int b0 = min(B, (int)threadIdx.x * per), b1 = min(B, b0 + per);
  const uint32_t cap = (uint32_t)T;
  // tokens: the fresh ones in the packed order, what exceeds T cut off
  uint32_t sum = 0;
  long long brought = 0;
  for (int b = b0; b < b1; ++b) {
    const uint32_t c = (uint32_t)max(0, cached[b]), n = min((uint32_t)max(0, fresh[b]), 0x7fffffffu - c);
    brought += n;
    sum = capped_add(sum, min(n, cap), cap);
  }
  uint32_t total;
  uint32_t at = block_scan(sum, cap, wave_sum, &total);
  uint32_t pages = 0, lost = 0;
  for (int b = b0; b < b1; ++b) {
    const uint32_t c = (uint32_t)max(0, cached[b]), n = min((uint32_t)max(0, fresh[b]), 0x7fffffffu - c);
    const uint32_t end = capped_add(at, min(n, cap), cap);
    const uint32_t len = c + (end - at);
    tok0[b] = at;
    held[b] = c;
    // pages: whole ones up to the cached end are there, those up to the new end are wanted
    const uint32_t P = 1u << shift;
    const uint32_t have = (c >> shift) + ((c & (P - 1)) != 0), need = (len >> shift) + ((len & (P - 1)) != 0);
    const uint32_t room = max(have, min(need, (uint32_t)width));
    page0[b] = room - have;
    pages += room - have;
    lost += need - room;
    if (blockIdx.x == 0) {
      lengths[b] = (int32_t)len;
      starts[b] = (int32_t)at;
    }
    at = end;
  }
  // (T + B new pages at most: no sum below wraps)
  uint32_t all_pages, all_lost, sum_hi, sum_lo;
  uint32_t pg = block_scan(pages, 0x7fffffffu, wave_sum, &all_pages);
  for (int b = b0; b < b1; ++b) {
    const uint32_t n = page0[b];
    page0[b] = pg;
    pg += n;
  }
  if (threadIdx.x == 0) { tok0[B] = total; page0[B] = all_pages; }
  const uint32_t first_free = (uint32_t)min(max(0, used[0]), n_free);
  if (blockIdx.x == 0) {
    block_scan(lost, 0x7fffffffu, wave_sum, &all_lost);
    // 43 bits of tokens brought, in two sums
    block_scan((uint32_t)(brought & 0xfffff), 0x7fffffffu, wave_sum, &sum_lo);
    block_scan((uint32_t)(brought >> 20), 0x7fffffffu, wave_sum, &sum_hi);
    if (threadIdx.x == 0) {
      starts[B] = (int32_t)total;
      const long long cut = ((long long)sum_hi << 20) + sum_lo - total;
      const uint32_t there = (uint32_t)n_free - first_free;
      counts[0] = (int32_t)(first_free + min(all_pages, there));
      counts[1] = (int32_t)min(all_lost + (all_pages > there ? all_pages - there : 0u), 0x7fffffffu);
      counts[2] = (int32_t)min(cut, 0x7fffffffll);
    }
  }
  __syncthreads();
  // new table entries
  for (uint32_t j = blockIdx.x * PLAN_NT + threadIdx.x; j < all_pages; j += gridDim.x * PLAN_NT) {
    const int b = owner_of(page0, B, j);
    const uint32_t c = held[b], P = 1u << shift;
    const uint32_t have = (c >> shift) + ((c & (P - 1)) != 0);
    const uint32_t f = first_free + j;
    table[(int64_t)b * width + have + (j - page0[b])] = f < (uint32_t)n_free ? free_list[f] : -1;
  }
  // slots and positions
  const uint32_t t0 = blockIdx.x * PLAN_TOKENS + threadIdx.x * PLAN_EACH, P = 1u << shift;
  int b = t0 < total ? owner_of(tok0, B, t0) : B;
#pragma unroll
  for (uint32_t u = 0; u < PLAN_EACH; ++u) {
    const uint32_t t = t0 + u;
    if (t >= (uint32_t)T) break;
    int32_t slot = -1, pos = -1;
    if (t < total) {
      while (t >= tok0[b + 1]) ++b;           // (tok0[B] is the total)
      const uint32_t c = held[b], p = c + (t - tok0[b]), col = p >> shift;
      const uint32_t have = (c >> shift) + ((c & (P - 1)) != 0);
      int32_t page = -1;
      if (col < have) {
        if (col < (uint32_t)width) page = table[(int64_t)b * width + col];   // an entry that no workgroup writes
      } else if (col - have < page0[b + 1] - page0[b]) {
        const uint32_t f = first_free + page0[b] + (col - have);
        if (f < (uint32_t)n_free) page = free_list[f];
      }
      pos = (int32_t)p;
      if (page >= 0 && page <= (0x7fffffff >> shift)) slot = (int32_t)(((uint32_t)page << shift) | (p & (P - 1)));
    }
    slots[t] = slot;
    positions[t] = pos;
  }
}

// ------------------------------------------------------------------ rows into the cache and back
// A row (one token's one head) of D values is D/8 lanes of 8 values; a lane's codes are one 32-bit word of the page, so that a
// row's words are one store of D/2 contiguous bytes.  Bound by the bytes, D values in, D/2 + 4 bytes out: 16384 tokens, 8 heads of 128,
// K and V in fp32, are written in 34 us (4.4 TB/s) and read back in 26 us (5.9 TB/s, stores that the cache behind L2 takes).  Small
// ones are a launch: 64 tokens 3 us each.  In 16 bits the instructions count too: 4999 tokens, 12 heads of 64, 8.2 us for 4.1 us of bytes, 369
// vector instructions a wave taking 4.6.  Two rows a thread were no faster.
// the bf16 value next to x below or equal / above or equal, as fp32
__device__ __forceinline__ float bf16_down(float x) {
  const uint32_t u = __float_as_uint(x);
  return __uint_as_float((u & 0xffff0000u) + (((u & 0xffffu) != 0 && (u >> 31) != 0) ? 0x10000u : 0u));
}
__device__ __forceinline__ float bf16_up_positive(float x) {
  const uint32_t u = __float_as_uint(x);
  return __uint_as_float((u + 0xffffu) & 0xffff0000u);
}

template <typename T, int D, bool WIDE>
__global__ __launch_bounds__(256) void cache_write_kernel(const T* __restrict__ k, const T* __restrict__ v, int n_rows, int Hkv,
                                                          HeadStrides ks, HeadStrides vs, const int32_t* __restrict__ slots,
                                                          CacheView c) {
  constexpr int LANES = D / 8;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int row = (int)(id / LANES), lane = (int)(id % LANES);
  const bool live = row < n_rows;
  const int t = live ? row / Hkv : 0, h = live ? row % Hkv : 0;
  const int32_t slot = live ? slots[t] : -1;
  const int page = slot >> c.shift;
  const bool put = slot >= 0 && page < c.n_pages;
  const int P = 1 << c.shift, off = slot & (P - 1);
  uint8_t* block = c.base + ((int64_t)page * Hkv + h) * ((int64_t)P * (D + 8));
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    const HeadStrides& st = side ? vs : ks;
    float x[8];
    load8<T, WIDE>((side ? v : k) + (int64_t)t * st.token + (int64_t)h * st.head + lane * 8, x);
    float lo = x[0], hi = x[0];
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      lo = fminf(lo, x[i]);
      hi = fmaxf(hi, x[i]);
      bad |= !(fabsf(x[i]) < INFINITY);
    }
    lo = row_reduce<LANES, false>(lo);
    hi = row_reduce<LANES, true>(hi);
    const float m = bf16_down(lo);
    float s = bf16_up_positive((hi - m) / 15.0f);
    if (s < 0x1p-126f) s = 0.f;
    const float r = s > 0.f ? 1.0f / s : 0.f;
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float q = __builtin_amdgcn_fmed3f(rintf((x[i] - m) * r), 0.f, 15.f);
      word |= (uint32_t)(int)q << (4 * i);
    }
    const unsigned long long any = __ballot(bad || !(s < INFINITY));
    const unsigned long long mine = ((1ull << LANES) - 1) << (threadIdx.x & 63 & ~(LANES - 1));
    if (put) {
      *reinterpret_cast<uint32_t*>(block + side * (P * D / 2) + off * (D / 2) + lane * 4) = word;
      if (lane == 0) {
        const uint32_t w = (__float_as_uint(m) & 0xffff0000u) | (__float_as_uint(s) >> 16);
        *reinterpret_cast<uint32_t*>(block + P * D + side * 4 * P + off * 4) = (any & mine) ? 0x7fc07fc0u : w;
      }
    }
  }
}

template <typename T, int D>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheView c, const int32_t* __restrict__ slots, int n_rows, int Hkv,
                                                         T* __restrict__ k, T* __restrict__ v) {
  constexpr int LANES = D / 8;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int row = (int)(id / LANES), lane = (int)(id % LANES);
  if (row >= n_rows) return;
  const int t = row / Hkv, h = row % Hkv;
  const int32_t slot = slots[t];
  const int page = slot >> c.shift;
  const bool there = slot >= 0 && page < c.n_pages;
  const int P = 1 << c.shift, off = slot & (P - 1);
  const uint8_t* block = c.base + ((int64_t)page * Hkv + h) * ((int64_t)P * (D + 8));
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    uint32_t word = 0, w = 0;
    if (there) {
      word = *reinterpret_cast<const uint32_t*>(block + side * (P * D / 2) + off * (D / 2) + lane * 4);
      w = *reinterpret_cast<const uint32_t*>(block + P * D + side * 4 * P + off * 4);
    }
    const float s = word_scale(w), m = word_offset(w);
    Vec8<T> r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = from_f<T>(fmaf(s, (float)((word >> (4 * i)) & 15u), m));   // (s * c is exact)
    T* dst = (side ? v : k) + (int64_t)row * D + lane * 8;
    uint4 o[sizeof(T) / 2];
    __builtin_memcpy(o, &r, sizeof r);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(dst)[i] = o[i];
  }
}

template <typename T, int D>
int write_typed(const void* k, const void* v, int T_, HeadStrides ks, HeadStrides vs, const int32_t* slots, CacheView c, bool wide, hipStream_t st) {
  const int rows = T_ * c.Hkv;
  const dim3 grid((unsigned)(((int64_t)rows * (D / 8) + 255) / 256));
  if (wide)
    PIPE_KLAUNCH((cache_write_kernel<T, D, true>), grid, dim3(256), 0, st, (const T*)k, (const T*)v, rows, c.Hkv, ks, vs, slots, c);
  else
    PIPE_KLAUNCH((cache_write_kernel<T, D, false>), grid, dim3(256), 0, st, (const T*)k, (const T*)v, rows, c.Hkv, ks, vs, slots, c);
  PIPE_HIP(hipGetLastError());
  return PIPE_OK;
}

template <typename T, int D>
int read_typed(CacheView c, const int32_t* slots, int T_, void* k, void* v, hipStream_t st) {
  const int rows = T_ * c.Hkv;
  PIPE_KLAUNCH((cache_read_kernel<T, D>), dim3((unsigned)(((int64_t)rows * (D / 8) + 255) / 256)), dim3(256), 0, st, c, slots, rows,
               c.Hkv, (T*)k, (T*)v);
  PIPE_HIP(hipGetLastError());
  return PIPE_OK;
}

}  // namespace

int launch_cache_plan(const int32_t* cached, const int32_t* fresh, int B, int shift, const int32_t* free_list, int n_free,
                      const int32_t* used, int32_t* table, int width, int T, int32_t* lengths, int32_t* starts,
                      int32_t* slots, int32_t* positions, int32_t* counts, hipStream_t st) {
  const int grid = T > 0 ? (T - 1) / PLAN_TOKENS + 1 : 1;
  PIPE_KLAUNCH(cache_plan_kernel, dim3(grid), dim3(PLAN_NT), 0, st, cached, fresh, B, shift, free_list, n_free, used, table, width, T,
               lengths, starts, slots, positions, counts);
  PIPE_HIP(hipGetLastError());
  return PIPE_OK;
}

int launch_cache_write(const void* k, const void* v, int type, int T, int D, HeadStrides ks, HeadStrides vs,
                       const int32_t* slots, CacheView c, hipStream_t st) {
  const bool wide = rows_wide(k, ks, type) && rows_wide(v, vs, type);
  if (type == PIPE_F32) return D == 64 ? write_typed<float, 64>(k, v, T, ks, vs, slots, c, wide, st) : write_typed<float, 128>(k, v, T, ks, vs, slots, c, wide, st);
  if (type == PIPE_F16) return D == 64 ? write_typed<f16, 64>(k, v, T, ks, vs, slots, c, wide, st) : write_typed<f16, 128>(k, v, T, ks, vs, slots, c, wide, st);
  return D == 64 ? write_typed<bf16, 64>(k, v, T, ks, vs, slots, c, wide, st) : write_typed<bf16, 128>(k, v, T, ks, vs, slots, c, wide, st);
}

int launch_cache_read(CacheView c, const int32_t* slots, int T, int D, int type, void* k, void* v, hipStream_t st) {
  if (type == PIPE_F32) return D == 64 ? read_typed<float, 64>(c, slots, T, k, v, st) : read_typed<float, 128>(c, slots, T, k, v, st);
  if (type == PIPE_F16) return D == 64 ? read_typed<f16, 64>(c, slots, T, k, v, st) : read_typed<f16, 128>(c, slots, T, k, v, st);
  return D == 64 ? read_typed<bf16, 64>(c, slots, T, k, v, st) : read_typed<bf16, 128>(c, slots, T, k, v, st);
}
