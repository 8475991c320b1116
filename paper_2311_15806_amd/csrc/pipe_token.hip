// Rows in 8 bits with a scale each; the router's choice, the order by expert, and the way back.
#include <algorithm>

#include "pipe_attention.h"
#include "pipe_codes.h"
#include "pipe_token.h"

namespace {

constexpr int64_t MOST_BLOCKS = 1 << 23;      // workgroups of 256 threads a launch

// ------------------------------------------------------------------ rows to codes
// Bound by the bytes: 4096 rows of 4096 in fp32 17.7 us, 4.7 TB/s.  In 16 bits (14.2 us for 50 MB) by neither: 17 vector instructions a value are 7.4 us of a
// SIMD's four waves, and a wave, whose loads, maximum and codes follow one another, waits 56 % of its time.  Few rows by latency, 2.3 to 3.4 us.
// s = max|x| / 127, c = rint(x / s): NT threads a row, 8 values a thread and step, the first CH steps kept in registers between the maximum
// and the codes, the rest (rows of more than 8 NT CH values) read again.  A row with a NaN or an infinity has the maximum +infinity here.
template <typename T, int NT, int CH, bool WIDE>
__global__ __launch_bounds__(256) void token_quantize_kernel(const T* __restrict__ x, int64_t rows, int in, int64_t stride, int pitch,
                                                             int8_t* __restrict__ codes, float* __restrict__ scales) {
  constexpr int PER = 256 / NT;
  const int tid = threadIdx.x % NT, n_chunk = (in + 7) >> 3;
  // (a launch holds fewer than 2^32 threads, rows are up to 2^30)
  for (int64_t row = (int64_t)blockIdx.x * PER + threadIdx.x / NT; row < rows; row += (int64_t)gridDim.x * PER) {
    const T* xr = x + row * stride;
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
    uint32_t bits = 0;
    auto raise = [&](const float* a) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) bits = raised(bits, a[i]);
    };
#pragma unroll
    for (int j = 0; j < CH; ++j) raise(v[j]);
    for (int c = tid + CH * NT; c < n_chunk; c += NT) {
      float a[8];
      fetch(c, a);
      raise(a);
    }
    const float top = top_of(bits);
    const RowScale scale(NT == 64 ? wave_max(top) : block_max(top));
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
}

template <typename T, bool WIDE>
int quantize_typed(const void* x, int64_t rows, int in, int64_t stride, int pitch, int8_t* codes, float* scales, hipStream_t st) {
  const T* p = (const T*)x;
  // a wave a row where there are many of up to 4096 values: no barrier (4096 rows of 4096: fp32 21.5 -> 19.0 us)
  const dim3 by_wave((unsigned)std::min<int64_t>((rows + 3) / 4, MOST_BLOCKS)), by_group((unsigned)std::min<int64_t>(rows, MOST_BLOCKS)), block(256);
  if (pitch <= 2048 && rows > 512) PIPE_KLAUNCH((token_quantize_kernel<T, 64, 4, WIDE>), by_wave, block, 0, st, p, rows, in, stride, pitch, codes, scales);
  else if (pitch <= 4096 && rows > 512) PIPE_KLAUNCH((token_quantize_kernel<T, 64, 8, WIDE>), by_wave, block, 0, st, p, rows, in, stride, pitch, codes, scales);
  else if (pitch <= 4096) PIPE_KLAUNCH((token_quantize_kernel<T, 256, 2, WIDE>), by_group, block, 0, st, p, rows, in, stride, pitch, codes, scales);
  else PIPE_KLAUNCH((token_quantize_kernel<T, 256, 4, WIDE>), by_group, block, 0, st, p, rows, in, stride, pitch, codes, scales);
  PIPE_HIP(hipGetLastError());
  return PIPE_OK;
}

// ------------------------------------------------------------------ the choice of experts, and the order by expert
// Pairs (token, choice) go by blocks of up to 512, whole tokens each, a pair a thread.  Where there is one block a single workgroup does all.  Otherwise a
// launch counts each block's pairs by expert (the router's beside its choice), and another has every workgroup sum the counts of the blocks
// before its own and of all (of many blocks and experts a third launch does), which gives its pairs' rows.  Nothing passes between the workgroups of a
// launch; no order of theirs is in the result.
// Bound by latency: 16384 tokens, eight of 128 experts, bf16, take 7 us for the choice (6 MB in and out), 8 to 10 for sums and rows (every workgroup
// reads the counts of all blocks); 48 tokens, six of 64, 5.4.
constexpr int PAIRS = 512;
__host__ __device__ constexpr int block_tokens(int top_k) { return PAIRS / top_k; }
static int block_count(int T, int top_k) { return (T + block_tokens(top_k) - 1) / block_tokens(top_k); }

struct SortArgs {
  int T, E, top_k, blocks;
  int32_t *starts, *order, *places;
  uint16_t* counts;     // [blocks][E + 1, rounded up to four], the last: pairs without an expert
  int32_t* before;      // their sums over the blocks before, and over all, [blocks + 1][likewise], or nullptr
};
__host__ __device__ constexpr int count_pitch(int E) { return (E + 4) / 4 * 4; }
// Whether a launch in between sums the counts, which every workgroup would else sum for itself.  One launch less is worth more than 2 us to a call, the
// work of the workgroups grows with the counts that each reads (a call, and one of a graph of calls, without and with: 136 blocks of 64 experts 18.3, 10.0
// and 21.9, 11.9 us; 256 of 128 18.3, 14.5 and 20.9, 14.0; 512 of 64 19.2, 17.9 and 21.1, 17.7; 384 of 128 21.6, 20.6 and 21.4, 18.1; 256 of 512 38 and 22).
static bool sums_apart(int64_t blocks, int E) { return blocks > 512 || blocks * count_pitch(E) > 36864; }

// lanes of the wave with the same key (of `bits` bits)
__device__ __forceinline__ unsigned long long same_key(int key, int bits) {
  unsigned long long m = ~0ull;
  for (int i = 0; i < bits; ++i) {
    const unsigned long long b = __ballot((key >> i) & 1);
    m &= (key >> i) & 1 ? b : ~b;
  }
  return m;
}

// The rows of block `b`'s pairs, `n` of them, a pair each of the first of NT threads: `key` is its expert (E: none; E + 1: behind the end).
template <int NT>
__device__ __forceinline__ void place(const SortArgs& a, int b, int n, int key, int* lds) {
  const int q = a.E + 1, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int *base = lds, *total = lds + q;                                // of each expert
  uint16_t* cnt = reinterpret_cast<uint16_t*>(lds + 2 * q);         // ... and of each wave's pairs
  __shared__ int wave_total[NT / 64];
  for (int i = threadIdx.x; i < PAIRS / 64 * q; i += NT) cnt[i] = 0;
  for (int e = threadIdx.x; e < q; e += NT) base[e] = total[e] = 0;
  __syncthreads();
  const bool mine = (int)threadIdx.x < n;
  const unsigned long long same = same_key(mine ? key : q, 32 - __clz(q));
  const int before = __popcll(same & ((1ull << lane) - 1));
  if (mine && before == 0) cnt[wave * q + key] = (uint16_t)__popcll(same);
  if (a.before != nullptr) {
    const int pitch = count_pitch(a.E);
    __syncthreads();
    for (int e = threadIdx.x; e < q; e += NT) {
      base[e] = a.before[(int64_t)b * pitch + e];
      total[e] = a.before[(int64_t)a.blocks * pitch + e];
    }
  } else if (a.blocks > 1) {
    const int quads = count_pitch(a.E) / 4, groups = max(1, NT / quads);      // four experts a thread, the blocks dealt to groups of threads
    for (int x = threadIdx.x; x < groups * quads; x += NT) {
      const int g = x / quads, e = (x - g * quads) * 4;
      int pre[4] = {0, 0, 0, 0}, all[4] = {0, 0, 0, 0};
#pragma unroll 8
      for (int r = g; r < a.blocks; r += groups) {
        const uint2 c = *reinterpret_cast<const uint2*>(a.counts + (int64_t)r * (4 * quads) + e);
        const int v[4] = {(int)(c.x & 0xffff), (int)(c.x >> 16), (int)(c.y & 0xffff), (int)(c.y >> 16)};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          all[i] += v[i];
          pre[i] += r < b ? v[i] : 0;
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (e + i < q) {
          atomicAdd(&base[e + i], pre[i]);
          atomicAdd(&total[e + i], all[i]);
        }
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < q; e += NT) {      // counts of the waves before
    int sum = 0;
#pragma unroll
    for (int w = 0; w < PAIRS / 64; ++w) {
      const int c = cnt[w * q + e];
      cnt[w * q + e] = (uint16_t)sum;
      sum += c;
    }
    if (a.blocks == 1) total[e] = sum;
  }
  __syncthreads();
  // first rows: all pairs of the experts before, `per` experts a thread
  const int per = (a.E + NT - 1) / NT, e0 = min((int)threadIdx.x * per, a.E), e1 = min(e0 + per, a.E);
  int own = 0;
  for (int e = e0; e < e1; ++e) own += total[e];
  int upto = own;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int v = __shfl_up(upto, d);
    if (lane >= d) upto += v;
  }
  if (lane == 63) wave_total[wave] = upto;
  __syncthreads();
  int first = upto - own;
  for (int w = 0; w < wave; ++w) first += wave_total[w];
  for (int e = e0; e < e1; ++e) {
    base[e] += first;
    if (b == 0) a.starts[e] = first;
    first += total[e];
    if (e == a.E - 1) {
      base[a.E] += first;
      if (b == 0) a.starts[a.E] = first;
    }
  }
  __syncthreads();
  if (!mine) return;
  const int pair = b * (block_tokens(a.top_k) * a.top_k) + threadIdx.x, row = base[key] + cnt[wave * q + key] + before;
  a.order[row] = key < a.E ? pair : -1;
  a.places[pair] = key < a.E ? row : -1;
}

// A workgroup four experts: the counts of all blocks summed up, a thread a share of the blocks.
constexpr int SUM_NT = 256;
__global__ __launch_bounds__(SUM_NT) void expert_sum_kernel(const SortArgs a) {
  __shared__ int wave_total[SUM_NT / 64][4];
  const int pitch = count_pitch(a.E), e = blockIdx.x * 4, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int share = (a.blocks + SUM_NT - 1) / SUM_NT, lo = min((int)threadIdx.x * share, a.blocks), hi = min(lo + share, a.blocks);
  auto counts_of = [&](int r, int* v) __attribute__((always_inline)) {
    const uint2 c = *reinterpret_cast<const uint2*>(a.counts + (int64_t)r * pitch + e);
    v[0] = (int)(c.x & 0xffff); v[1] = (int)(c.x >> 16); v[2] = (int)(c.y & 0xffff); v[3] = (int)(c.y >> 16);
  };
  int sum[4] = {0, 0, 0, 0}, v[4];
#pragma unroll 4
  for (int r = lo; r < hi; ++r) {
    counts_of(r, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] += v[i];
  }
  int at[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    int upto = sum[i];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(upto, d);
      if (lane >= d) upto += o;
    }
    at[i] = upto - sum[i];
    if (lane == 63) wave_total[wave][i] = upto;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i)
    for (int w = 0; w < wave; ++w) at[i] += wave_total[w][i];
#pragma unroll 4
  for (int r = lo; r < hi; ++r) {
    counts_of(r, v);
    *reinterpret_cast<int4*>(a.before + (int64_t)r * pitch + e) = make_int4(at[0], at[1], at[2], at[3]);
#pragma unroll
    for (int i = 0; i < 4; ++i) at[i] += v[i];
  }
  if (threadIdx.x == SUM_NT - 1) *reinterpret_cast<int4*>(a.before + (int64_t)a.blocks * pitch + e) = make_int4(at[0], at[1], at[2], at[3]);
}

// pairs of block b
__device__ __forceinline__ int pairs_of(const SortArgs& a, int b) {
  return min(block_tokens(a.top_k), a.T - b * block_tokens(a.top_k)) * a.top_k;
}
__device__ __forceinline__ int key_of(int expert, int E) { return (unsigned)expert < (unsigned)E ? expert : E; }
extern __shared__ int sort_lds[];
static size_t sort_lds_bytes(int E) { return (size_t)(E + 1) * (2 * sizeof(int) + PAIRS / 64 * sizeof(uint16_t)); }   // (24600 at most)

__global__ __launch_bounds__(PAIRS) void expert_place_kernel(const int32_t* __restrict__ experts, const SortArgs a) {
  const int b = blockIdx.x, n = pairs_of(a, b);
  const int key = (int)threadIdx.x < n ? key_of(experts[(int64_t)b * (block_tokens(a.top_k) * a.top_k) + threadIdx.x], a.E) : 0;
  place<PAIRS>(a, b, n, key, sort_lds);
}

// counts of a block by expert
template <int NT>
__device__ __forceinline__ void count_block(const SortArgs& a, int b, int n, int key, int* hist /* [E + 1] */) {
  const int q = a.E + 1;
  for (int e = threadIdx.x; e < q; e += NT) hist[e] = 0;
  __syncthreads();
  if ((int)threadIdx.x < n) atomicAdd(&hist[key], 1);
  __syncthreads();
  for (int e = threadIdx.x; e < q; e += NT) a.counts[(int64_t)b * count_pitch(a.E) + e] = (uint16_t)hist[e];
}
__global__ __launch_bounds__(PAIRS) void expert_count_kernel(const int32_t* __restrict__ experts, const SortArgs a) {
  const int b = blockIdx.x, n = pairs_of(a, b);
  const int key = (int)threadIdx.x < n ? key_of(experts[(int64_t)b * (block_tokens(a.top_k) * a.top_k) + threadIdx.x], a.E) : 0;
  count_block<PAIRS>(a, b, n, key, sort_lds);
}

// over the 16 lanes of a token
__device__ __forceinline__ float row_sum(float x) {
  x += dpp<0xB1>(x);
  x += dpp<0x4E>(x);
  x += dpp<0x141>(x);
  return x + dpp<0x140>(x);
}
template <int CTRL>
__device__ __forceinline__ int dpp_i(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xf, 0xf, true); }
__device__ __forceinline__ int row_min(int x) {
  x = min(x, dpp_i<0xB1>(x));
  x = min(x, dpp_i<0x4E>(x));
  x = min(x, dpp_i<0x141>(x));
  return min(x, dpp_i<0x140>(x));
}

__device__ __forceinline__ uint32_t row_max(uint32_t x) {
  x = max(x, (uint32_t)dpp_i<0xB1>((int)x));
  x = max(x, (uint32_t)dpp_i<0x4E>((int)x));
  x = max(x, (uint32_t)dpp_i<0x141>((int)x));
  return max(x, (uint32_t)dpp_i<0x140>((int)x));
}
// A 16-bit logit and its expert in one number: above others if the logit is larger, or the same (-0 as 0) and the expert lower.  0: not to be chosen.
template <typename T>
__device__ __forceinline__ uint32_t logit_key(T x, float v, int e) {
  const int u = v == 0.f ? 0 : __builtin_bit_cast(int16_t, x);      // in the upper half: a negative number's bits turned around, of another the sign
  const uint32_t key = (uint32_t)(u ^ (u >> 15 | 0x8000)) << 16 | (0xffffu - (uint32_t)e);
  return v > -INFINITY ? key : 0u;
}
template <typename T>
__device__ __forceinline__ float logit_of(uint32_t key) {
  const uint32_t u = key >> 16;
  return to_f(__builtin_bit_cast(T, (uint16_t)(u & 0x8000u ? u ^ 0x8000u : u ^ 0xffffu)));
}

// 16 lanes a token, lane l its logits l, l + 16, ...  In fp32 each of the top_k steps is a maximum and then the lowest index that holds it; a NaN equals
// nothing and is never chosen.  In 16 bits a logit and its index are one number k, no two alike, and a step is one maximum: with the last choice m the
// differences k - m, modulo 2^32, put all k below m over the others, in their order.  Bound by the instructions of a step (a wave a token: 12.7 us; 16 lanes
// by maximum and index 9.9, 1024 threads instead of 512 8.7; one number 6.8: 16384 tokens, eight of 128, bf16, with the counts of the blocks).
constexpr int route_threads(int EL) { return EL < 32 ? 1024 : 512; }      // (of 32 logits a lane the registers hold 512)
template <typename T, int EL>
__global__ __launch_bounds__(route_threads(EL)) void expert_route_kernel(const ExpertRouteArgs a, const SortArgs s) {
  constexpr int NT = route_threads(EL);
  __shared__ int keys[PAIRS];
  const int lane = threadIdx.x & 63, l = lane & 15, b = blockIdx.x;
  const int t0 = b * block_tokens(a.top_k), tokens = min(block_tokens(a.top_k), a.T - t0);
  for (int i0 = (threadIdx.x >> 6) * 4; i0 < tokens; i0 += NT / 16) {
    const int i = i0 + (lane >> 4), t = t0 + min(i, tokens - 1);
    const T* row = (const T*)a.logits + (int64_t)t * a.row_stride;
    float v[EL];
    uint32_t k[EL], last = 0;      // (16 bits)
#pragma unroll
    for (int c = 0; c < EL; c += 16) {      // (up to 16 loads at once, none behind a branch)
      constexpr int N = EL < 16 ? EL : 16;
      T x[N];
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = 2 * (c + i) < EL && EL > 1 ? row[(c + i) * 16 + l] : row[min((c + i) * 16 + l, a.E - 1)];      // (E > 8 EL there)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        v[c + i] = (c + i) * 16 + l < a.E ? to_f(x[i]) : -INFINITY;
        if constexpr (sizeof(T) == 2) k[c + i] = logit_key(x[i], v[c + i], (c + i) * 16 + l);
      }
      if (EL > 16) __builtin_amdgcn_sched_barrier(0);
    }
    float chosen[2] = {-INFINITY, -INFINITY};      // lane l: the l-th and the 16 + l-th largest
    int expert[2] = {-1, -1};
    uint32_t picked[2] = {0, 0};                   // (16 bits: both)
    float first = 0.f, total = 0.f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      for (int j = 0, steps = min(16, a.top_k - 16 * h); j < steps; ++j) {
        float m;
        int at = 0x7fffffff;
        if constexpr (sizeof(T) == 2) {
          uint32_t up = 0;
#pragma unroll
          for (int e = 0; e < EL; ++e) up = max(up, k[e] - last);
          const uint32_t next = row_max(up) + last;
          const bool there = next - 1u < last - 1u;      // 0 < next < last, or any but 0 at first; else no logit is left
          last = there ? next : last;
          picked[h] = l == j && there ? next : picked[h];
          m = there ? logit_of<T>(next) : -INFINITY;
        } else {
          m = v[0];
#pragma unroll
          for (int e = 1; e < EL; ++e) m = fmaxf(m, v[e]);
          m = row_reduce<16, true>(m);
#pragma unroll
          for (int e = EL - 1; e >= 0; --e) at = v[e] == m ? e * 16 + l : at;
          at = row_min(at);
          if (l == j && m > -INFINITY) {                 // (a maximum of NaNs is one, or -infinity)
            chosen[h] = m;
            expert[h] = at;
          }
        }
        if (h == 0 && j == 0) {
          first = m > -INFINITY ? m : 0.f;
          if (!a.renormalize) {
#pragma unroll
            for (int e = 0; e < EL; ++e) total += expf(v[e] - first);
          }
        }
        if constexpr (sizeof(T) == 4) {
#pragma unroll
          for (int e = 0; e < EL; ++e) v[e] = e * 16 + l == at ? -INFINITY : v[e];
        }
      }
      if constexpr (sizeof(T) == 2) {
        if (picked[h] != 0) {
          chosen[h] = logit_of<T>(picked[h]);
          expert[h] = 0xffff - (int)(picked[h] & 0xffffu);
        }
      }
    }
    float w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) w[h] = expert[h] >= 0 ? expf(chosen[h] - first) : 0.f;
    if (a.renormalize) total = w[0] + w[1];
    total = row_sum(total);
    if (i < tokens) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int j = h * 16 + l;
        if (j < a.top_k) {
          a.experts[(int64_t)t * a.top_k + j] = expert[h];
          a.weights[(int64_t)t * a.top_k + j] = expert[h] >= 0 ? w[h] / total : 0.f;
          keys[i * a.top_k + j] = key_of(expert[h], a.E);
        }
      }
    }
  }
  __syncthreads();
  const int n = tokens * a.top_k, key = (int)threadIdx.x < n ? keys[threadIdx.x] : 0;
  if (s.blocks == 1) place<NT>(s, b, n, key, sort_lds);
  else count_block<NT>(s, b, n, key, sort_lds);
}

// ------------------------------------------------------------------ back to the tokens
// 8 values of a token a thread, the rows of its experts summed in fp32 in the order of its choices.  Bound by the bytes: 8192 tokens, eight rows of 4096 each (a
// quarter of them left out), fp16, 100 us for 470 MB; 32 tokens of six rows of 2048 3.7 us.
template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void expert_combine_kernel(const T* __restrict__ y, int64_t n, int H, int64_t stride, const int32_t* __restrict__ places,
                                                             const float* __restrict__ weights, int64_t items, int top_k, T* __restrict__ out) {
  const int chunks = (H + 7) >> 3;
  for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < items; id += (int64_t)gridDim.x * 256) {
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
}

template <typename T>
int route_typed(const ExpertRouteArgs& a, const SortArgs& s, hipStream_t st) {
  const dim3 grid(s.blocks);
  const size_t lds = sort_lds_bytes(a.E);
  if (a.E <= 16) PIPE_KLAUNCH((expert_route_kernel<T, 1>), grid, dim3(route_threads(1)), lds, st, a, s);
  else if (a.E <= 32) PIPE_KLAUNCH((expert_route_kernel<T, 2>), grid, dim3(route_threads(2)), lds, st, a, s);
  else if (a.E <= 64) PIPE_KLAUNCH((expert_route_kernel<T, 4>), grid, dim3(route_threads(4)), lds, st, a, s);
  else if (a.E <= 128) PIPE_KLAUNCH((expert_route_kernel<T, 8>), grid, dim3(route_threads(8)), lds, st, a, s);
  else if (a.E <= 256) PIPE_KLAUNCH((expert_route_kernel<T, 16>), grid, dim3(route_threads(16)), lds, st, a, s);
  else if (a.E <= 512) PIPE_KLAUNCH((expert_route_kernel<T, 32>), grid, dim3(route_threads(32)), lds, st, a, s);
  else PIPE_KLAUNCH((expert_route_kernel<T, 64>), grid, dim3(route_threads(64)), lds, st, a, s);
  PIPE_HIP(hipGetLastError());
  return PIPE_OK;
}

template <typename T>
int combine_typed(const void* y, int64_t n, int H, int64_t stride, const int32_t* places, const float* weights, int T_, int top_k, void* out,
                  hipStream_t st) {
  const int64_t items = (int64_t)T_ * ((H + 7) / 8);
  const dim3 grid((unsigned)std::min<int64_t>((items + 255) / 256, MOST_BLOCKS));
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

int64_t expert_sort_scratch(int T, int top_k, int E) {
  const int64_t blocks = block_count(T, top_k), pitch = count_pitch(E);
  if (blocks <= 1) return 0;
  return round_up64(blocks * pitch * sizeof(uint16_t), 16) + (sums_apart(blocks, E) ? (blocks + 1) * pitch * (int64_t)sizeof(int32_t) : 0);
}
static SortArgs sort_args(int T, int E, int top_k, int32_t* starts, int32_t* order, int32_t* places, void* scratch) {
  const int blocks = std::max(1, block_count(T, top_k));
  SortArgs s{T, E, top_k, blocks, starts, order, places, (uint16_t*)scratch, nullptr};
  if (sums_apart(blocks, E)) s.before = (int32_t*)((char*)scratch + round_up64((int64_t)blocks * count_pitch(E) * sizeof(uint16_t), 16));
  return s;
}

static int launch_place(const int32_t* experts, const SortArgs& s, hipStream_t st) {
  if (s.before != nullptr) {
    PIPE_KLAUNCH(expert_sum_kernel, dim3(count_pitch(s.E) / 4), dim3(SUM_NT), 0, st, s);
    PIPE_HIP(hipGetLastError());
  }
  PIPE_KLAUNCH(expert_place_kernel, dim3(s.blocks), dim3(PAIRS), sort_lds_bytes(s.E), st, experts, s);
  PIPE_HIP(hipGetLastError());
  return PIPE_OK;
}

int launch_expert_route(const ExpertRouteArgs& a, int32_t* starts, int32_t* order, int32_t* places, void* scratch, hipStream_t st) {
  const SortArgs s = sort_args(a.T, a.E, a.top_k, starts, order, places, scratch);
  const int rc = a.type == PIPE_F32 ? route_typed<float>(a, s, st) : a.type == PIPE_F16 ? route_typed<f16>(a, s, st) : route_typed<bf16>(a, s, st);
  return rc || s.blocks == 1 ? rc : launch_place(a.experts, s, st);
}

int launch_expert_sort(const int32_t* experts, int T, int top_k, int E, int32_t* starts, int32_t* order, int32_t* places, void* scratch, hipStream_t st) {
  const SortArgs s = sort_args(T, E, top_k, starts, order, places, scratch);
  if (s.blocks > 1) {
    PIPE_KLAUNCH(expert_count_kernel, dim3(s.blocks), dim3(PAIRS), (E + 1) * sizeof(int), st, experts, s);
    PIPE_HIP(hipGetLastError());
  }
  return launch_place(experts, s, st);
}

int launch_expert_combine(const void* y, int type, int64_t n, int H, int64_t stride, const int32_t* places, const float* weights, int T, int top_k,
                          void* out, hipStream_t st) {
  if (type == PIPE_F32) return combine_typed<float>(y, n, H, stride, places, weights, T, top_k, out, st);
  return type == PIPE_F16 ? combine_typed<f16>(y, n, H, stride, places, weights, T, top_k, out, st) : combine_typed<bf16>(y, n, H, stride, places, weights, T, top_k, out, st);
}
