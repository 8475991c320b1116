// Products of 8-bit codes with a scale for each token and each channel, y = act(s_t s_o sum_i c_ti w_oi + b_o), of one layer or of a router's
// experts, whose rows lie one after the other in y.
//
// Sums are exact in 32 bits.  Both scales' exponents are kept apart from their mantissas until the end, so that no product of a sum and one of
// the scales leaves fp32's range where the whole does not.  Every kernel here computes an output by the same operations: which one serves a call
// changes no bit.
#include <type_traits>

#include "pipe_attention.h"
#include "pipe_tile.h"
#include "pipe_token.h"

int g_token_kernel = 0;

namespace {

// ------------------------------------------------------------------ what the kernels share
// A tile's rows of y: those of expert e from `row` on, n of them; e == E: rows without an expert.
struct Rows {
  int e, n;
  int64_t row;
};
// Tile `id`: expert e owns the ids from floor(starts[e] / BT) + e on, which are at least as many as its tiles; called by whole waves.
template <int BT>
__device__ __forceinline__ Rows find_rows(const TokenProductArgs& a, int id) {
  if (a.starts == nullptr) return Rows{0, (int)min((int64_t)BT, a.n - (int64_t)id * BT), (int64_t)id * BT};
  const int lane = threadIdx.x & 63, n = (int)a.n;
  auto start_of = [&](int e) { return e <= 0 ? 0 : min(max(a.starts[min(e, a.E)], 0), n); };
  int e = -1, start, end;
  if (a.E < 63) {      // a lane an expert: nothing is looked up twice
    const int s = start_of(lane);
    e = __popcll(__ballot(lane <= a.E && s / BT + lane <= id)) - 1;
    start = __builtin_amdgcn_readlane(s, e);
    end = e < a.E ? __builtin_amdgcn_readlane(s, e + 1) : n;
  } else {
    for (int i0 = 0; i0 <= a.E; i0 += 64) {
      const int i = i0 + lane;
      const int found = __popcll(__ballot(i <= a.E && start_of(i) / BT + i <= id));
      e += found;
      if (found < 64) break;
    }
    e = __builtin_amdgcn_readfirstlane(e);
    start = __builtin_amdgcn_readfirstlane(start_of(e));
    end = e < a.E ? __builtin_amdgcn_readfirstlane(start_of(e + 1)) : n;
  }
  const int skip = (id - start / BT - e) * BT;
  return Rows{e, skip < 0 ? 0 : min(BT, end - start - skip), (int64_t)start + skip};
}
template <int BT>
int64_t row_tiles(const TokenProductArgs& a) {
  return a.starts == nullptr ? (a.n + BT - 1) / BT : a.n / BT + a.E + 1;
}
// the input behind row i of a tile, -1: none
__device__ __forceinline__ int64_t input_of(const TokenProductArgs& a, const Rows& r, int i) {
  const int64_t row = r.row + min(i, r.n - 1);
  if (a.order == nullptr) return row < a.n_x ? row : -1;
  const int o = a.order[row];
  return o >= 0 && o < a.n_x * a.top_k ? o / a.top_k : -1;
}
__device__ __forceinline__ int w_rows_of(const TokenProductArgs& a, bool gated) { return gated ? 2 * a.out : a.out; }
// row of the weights behind row i of a tile from column o0 of y on; of a gated layer 16 of the gate, then 16 of the other half, and so on
template <bool GATED>
__device__ __forceinline__ int weight_of(const TokenProductArgs& a, int o0, int i) {
  if (!GATED) return min(o0 + i, a.out - 1);
  return ((i >> 4) & 1) * a.out + min(o0 + (i >> 5) * 16 + (i & 15), a.out - 1);
}

__device__ __forceinline__ float act_of(float z, int act) {
  if (act == PIPE_ACT_GELU) return gelu_erf(z);
  if (act == PIPE_ACT_RELU) return z < 0.f ? 0.f : z;
  return z;
}
__device__ __forceinline__ void act4(float* z, int act) {
  if (act == PIPE_ACT_NONE) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) z[i] = act_of(z[i], act);
}
// (the exponential's argument is one rounding off: 2^-24 |g| of the value, what the product g with anything may be off by as well)
__device__ __forceinline__ float silu(float g) { return g * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(g * -1.44269504f)); }

// Four channels' scales, as mantissa and exponent, and biases: z = (sum s_t) s_o + b
struct Channels {
  float m[4], b[4];
  int e[4];
  __device__ __forceinline__ void set(int i, float s, float bias) {
    m[i] = __builtin_amdgcn_frexp_mantf(s);
    e[i] = __builtin_amdgcn_frexp_expf(s);
    b[i] = bias;
  }
  __device__ __forceinline__ void values(const v4i& sum, float sx, bool with_bias, float* z) const {
    const float mx = __builtin_amdgcn_frexp_mantf(sx);
    const int ex = __builtin_amdgcn_frexp_expf(sx);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      z[i] = __builtin_amdgcn_ldexpf((float)sum[i] * mx * m[i], ex + e[i]);
      if (with_bias) z[i] += b[i];
    }
  }
};

// up to four values of a row of y
template <typename T>
__device__ __forceinline__ void put4_typed(T* p, const float* z, int have, bool wide) {
  if (wide && have >= 4) {
    store_row<T, 4>(p, z);
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < have) p[i] = from_f<T>(z[i]);
}
__device__ __forceinline__ void put4(void* y, int type, int64_t at, const float* z, int have, bool wide) {
  if (type == PIPE_F32) put4_typed((float*)y + at, z, have, wide);
  else if (type == PIPE_F16) put4_typed((f16*)y + at, z, have, wide);
  else put4_typed((bf16*)y + at, z, have, wide);
}
// zeros of the columns from o0 on, WIDTH of them, of a tile of rows without an expert
template <int WIDTH, int NT>
__device__ __forceinline__ void put_zeros(const TokenProductArgs& a, const Rows& r, int o0) {
  const float zero = 0.f;
  for (int i = threadIdx.x; i < r.n * WIDTH; i += NT) {
    const int t = i / WIDTH, o = o0 + i % WIDTH;
    if (o < a.out) put4(a.y, a.type, (r.row + t) * a.out + o, &zero, 1, false);
  }
}

// Scales and bias of a tile's BO rows of weights, scales of its BT tokens (negative: no input), by all NT threads.
template <int BO, int BT>
struct Side {
  float sw[BO], bias[BO], sx[BT];
  template <bool GATED, int NT>
  __device__ __forceinline__ void load(const TokenProductArgs& a, const Rows& r, int o0) {
    const int64_t w0 = (int64_t)r.e * w_rows_of(a, GATED);
    for (int i = threadIdx.x; i < BO; i += NT) {
      const int o = weight_of<GATED>(a, o0, i);
      sw[i] = a.sw[w0 + o];
      bias[i] = a.bias ? a.bias[w0 + o] : 0.f;
    }
    for (int i = threadIdx.x; i < BT; i += NT) {
      const int64_t in = input_of(a, r, i);
      sx[i] = in < 0 ? -1.f : a.sx[in];
    }
  }
};

// The outputs of a wave's FO x FT blocks of 16 rows x 16 tokens, which begin at the tile's row wo and token wt: 16 tokens after the other
// through LDS (`turn`, 16 x 4 FO pieces of four sums, in an order that differs by token), so that a store writes whole pieces of a row of y.
template <bool GATED, int FO, int FT, int BO, int BT>
__device__ __forceinline__ void finish(const TokenProductArgs& a, const Rows& r, int o0, int wo, int wt, const v4i (&acc)[FO][FT], v4i* turn,
                                       const Side<BO, BT>& side) {
  constexpr int PIECES = 4 * FO, LANES = GATED ? PIECES / 2 : PIECES;      // lanes of a token, 4 columns each
  constexpr int SH = PIECES == 32 ? 1 : 0, DOWN = PIECES == 8 ? 1 : 0;
  static_assert(PIECES == 8 || PIECES == 16 || PIECES == 32, "turn");
  const int lane = threadIdx.x & 63, n16 = lane & 15, k16 = lane >> 4;
  const int col = lane % LANES, first = lane / LANES;
  const int piece = GATED ? (col >> 2) * 8 + (col & 3) : col, i0 = wo + piece * 4;
  Channels c0, c1;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    c0.set(i, side.sw[i0 + i], side.bias[i0 + i]);
    if (GATED) c1.set(i, side.sw[i0 + 16 + i], side.bias[i0 + 16 + i]);
  }
  const int o = o0 + (GATED ? wo / 2 : wo) + col * 4;
  const bool wide = a.out % 4 == 0;
#pragma unroll 1
  for (int part = 0; part < FT; ++part) {
#pragma unroll
    for (int g = 0; g < FT; ++g)
      if (part == g) {
#pragma unroll
        for (int f = 0; f < FO; ++f) turn[n16 * PIECES + ((4 * f + k16) ^ (n16 << SH >> DOWN))] = acc[f][g];
      }
    __builtin_amdgcn_wave_barrier();              // a wave's own LDS accesses stay in order
    const int t0 = wt + part * 16;
#pragma unroll 2
    for (int t = first; t < 16; t += 64 / LANES) {
      const float sx = side.sx[t0 + t];
      const v4i* row = turn + t * PIECES;
      float z[4];
      c0.values(row[piece ^ (t << SH >> DOWN)], sx, a.bias != nullptr, z);
      if (GATED) {
        float u[4];
        c1.values(row[(piece + 4) ^ (t << SH >> DOWN)], sx, a.bias != nullptr, u);
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] = silu(z[i]) * u[i];
      } else {
        act4(z, a.act);
      }
      if (sx < 0.f) z[0] = z[1] = z[2] = z[3] = 0.f;
      if (t0 + t < r.n) put4(a.y, a.type, (r.row + t0 + t) * a.out + o, z, a.out - o, wide);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Where a wave's loads of 8 rows x 128 codes come from: row `first` + 8 p + (lane >> 3) of the tile's B rows of weights (first < B) or of its tokens.
// Addresses are a resource's base and 32 bits; of a gated layer 16 rows of the gate and of the other half in turn.
template <bool GATED, int B, int P>
struct Source {
  __amdgpu_buffer_rsrc_t from0, from1;
  unsigned off[P];
  __device__ __forceinline__ Source(const TokenProductArgs& a, const Rows& r, int o0, int first) {
    const int lane = threadIdx.x & 63;
    const bool weights = first < B;
    const int8_t *b0, *b1;
    if (weights) {
      b0 = a.w + ((int64_t)r.e * w_rows_of(a, GATED) + o0) * a.pitch;
      b1 = GATED ? b0 + (int64_t)a.out * a.pitch : b0;
    } else {
      b0 = b1 = a.qx + (a.order ? 0 : r.row) * a.pitch;
    }
    from0 = __builtin_amdgcn_make_buffer_rsrc((void*)b0, 0, 0xffffffffu, 0x00020000);
    from1 = __builtin_amdgcn_make_buffer_rsrc((void*)b1, 0, 0xffffffffu, 0x00020000);
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int row = first + p * 8 + (lane >> 3);
      int64_t at;
      if (weights) at = min(o0 + (GATED ? (row >> 5) * 16 + (row & 15) : row), a.out - 1) - o0;
      else at = max(input_of(a, r, row - B), (int64_t)0) - (a.order ? 0 : r.row);
      off[p] = (unsigned)(at * a.pitch);
    }
  }
  __device__ __forceinline__ const __amdgpu_buffer_rsrc_t& from(int p) const { return ((p >> 1) & 1) ? from1 : from0; }
};
// 16 bytes a lane from base + off + k to dst + 16 * lane
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t base, v4i* dst, unsigned off, int k) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(base, (__attribute__((address_space(3))) void*)dst, 16, off, k, 0, 0);
}
// whether 32 bits reach every input
static bool near(const TokenProductArgs& a) { return a.order == nullptr || a.n_x * a.pitch < (int64_t)0xffffffff; }

// Blocks b, b + 8, ... of a launch run on one XCD (one L2): neighbours there are HIGH tiles of tokens x some of weights.
template <int HIGH>
struct Order {
  int o_tiles, t_tiles, per_xcd;
  __device__ __forceinline__ bool tile(int block, int* ot, int* id) const {
    const int at = block >> 3;
    const int64_t place = (int64_t)(block & 7) * per_xcd + at;
    if (at >= per_xcd || place >= (int64_t)o_tiles * t_tiles) return false;
    const int band = (int)(place / (HIGH * (int64_t)o_tiles)), in_band = (int)(place - band * (HIGH * (int64_t)o_tiles));
    const int high = min(HIGH, t_tiles - band * HIGH);
    *ot = in_band / high;
    *id = band * HIGH + in_band - *ot * high;
    return true;
  }
};

// ------------------------------------------------------------------ few tokens
// Bound by the bytes of the weights.  16 rows (of the gate and of the other half as well) x 16 TB tokens a workgroup of eight waves, which take the
// steps of 64 codes in turn, straight from memory to operands; their sums meet in LDS.
template <bool GATED, int TB>
__global__ __launch_bounds__(512) void token_stream_kernel(const TokenProductArgs a, int o_tiles) {
  constexpr int NW = 8, G = GATED ? 2 : 1, U = 4;
  __shared__ v4i part[NW][G * TB][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int id = blockIdx.x / o_tiles, o0 = (blockIdx.x - id * o_tiles) * 16;
  const Rows r = find_rows<16 * TB>(a, id);
  if (r.n <= 0) return;
  if (r.e == a.E) {
    put_zeros<16, 512>(a, r, o0);
    return;
  }
  const int n16 = lane & 15, k16 = lane >> 4;
  const int64_t w0 = (int64_t)r.e * w_rows_of(a, GATED);
  // weights through a resource of the 16 rows, behind whose end a step beyond the last reads zeros; tokens at 64 bits
  __amdgpu_buffer_rsrc_t from[G];
#pragma unroll
  for (int h = 0; h < G; ++h)
    from[h] = __builtin_amdgcn_make_buffer_rsrc((void*)(a.w + (w0 + h * a.out + o0) * a.pitch), 0, (unsigned)(min(16, a.out - o0) * a.pitch), 0x00020000);
  const unsigned w_at = (unsigned)(min(n16, a.out - 1 - o0) * a.pitch + k16 * 16);
  const int8_t* xp[TB];
#pragma unroll
  for (int b = 0; b < TB; ++b) xp[b] = a.qx + max(input_of(a, r, 16 * b + n16), (int64_t)0) * a.pitch + k16 * 16;
  v4i acc[G][TB] = {};
  const int steps = a.pitch / 64;
  struct Set {
    v4i w[U][G], x[U][TB];
  } s0, s1;
  auto ask = [&](Set& q, int s) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = s + u * NW;
#pragma unroll
      for (int h = 0; h < G; ++h) q.w[u][h] = (v4i)__builtin_amdgcn_raw_buffer_load_b128(from[h], w_at + (k < steps ? k * 64u : 0x80000000u), 0, 0);
#pragma unroll
      for (int b = 0; b < TB; ++b) q.x[u][b] = (v4i)gload16(xp[b] + min(k, steps - 1) * 64);
    }
  };
  auto mul = [&](const Set& q) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < G; ++h)
#pragma unroll
        for (int b = 0; b < TB; ++b) acc[h][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(q.w[u][h], q.x[u][b], acc[h][b], 0, 0, 0);
  };
  int s = wave;
  ask(s0, s);
  while (true) {
    s += U * NW;
    if (s >= steps) { mul(s0); break; }
    ask(s1, s);
    mul(s0);
    s += U * NW;
    if (s >= steps) { mul(s1); break; }
    ask(s0, s);
    mul(s1);
  }
#pragma unroll
  for (int h = 0; h < G; ++h)
#pragma unroll
    for (int b = 0; b < TB; ++b) part[wave][h * TB + b][lane] = acc[h][b];
  __syncthreads();
  if (wave >= TB) return;
  const int b = wave, t = 16 * b + n16;
  v4i sum[G];
#pragma unroll
  for (int h = 0; h < G; ++h) {
    sum[h] = part[0][h * TB + b][lane];
#pragma unroll
    for (int q = 1; q < NW; ++q) sum[h] += part[q][h * TB + b][lane];
  }
  if (t >= r.n) return;
  const int64_t in = input_of(a, r, t);
  const float sx = in < 0 ? 0.f : a.sx[in];
  float z[2][4];
#pragma unroll
  for (int h = 0; h < G; ++h) {
    Channels c;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t o = w0 + weight_of<GATED>(a, o0, 16 * h + 4 * k16 + i);
      c.set(i, a.sw[o], a.bias ? a.bias[o] : 0.f);
    }
    c.values(sum[h], sx, a.bias != nullptr, z[h]);
  }
  if (GATED) {
#pragma unroll
    for (int i = 0; i < 4; ++i) z[0][i] = silu(z[0][i]) * z[1][i];
  } else {
    act4(z[0], a.act);
  }
  if (in < 0) z[0][0] = z[0][1] = z[0][2] = z[0][3] = 0.f;
  const int o = o0 + 4 * k16;
  put4(a.y, a.type, (r.row + t) * a.out + o, z[0], a.out - o, a.out % 4 == 0);
}

// ------------------------------------------------------------------ tiles
// B rows of weights x B tokens a workgroup of four waves, a quarter each.  A stage is 128 codes of every row, straight to LDS, one stage ahead; the
// eight pieces of 16 of a row lie in an order that differs by pairs of rows, so that the reads of 16 rows' same piece meet all banks.
template <bool GATED, int B>
__global__ __launch_bounds__(256, 2) void token_tile_kernel(const TokenProductArgs a, const Order<8> order) {
  constexpr int KB = 128, P = B / 16, F = B / 32, WIDTH = GATED ? B / 2 : B;
  __shared__ alignas(1024) v4i slot0[2 * B * KB / 16], slot1[2 * B * KB / 16];
  static_assert(sizeof(slot0) + sizeof(slot1) <= 65536, "loads to LDS reach the first 64 KiB");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int ot, id;
  if (!order.tile(blockIdx.x, &ot, &id)) return;
  const Rows r = find_rows<B>(a, id);
  if (r.n <= 0) return;
  const int o0 = ot * WIDTH;
  if (r.e == a.E) {
    put_zeros<WIDTH, 256>(a, r, o0);
    return;
  }
  Source<GATED, B, P> src(a, r, o0, wave * (B / 2));
  // the lane's piece of row (lane >> 3) of an even load; of an odd one it is 4 further
#pragma unroll
  for (int p = 0; p < P; ++p) src.off[p] += (((lane & 7) ^ (lane >> 4)) ^ ((p & 1) * 4)) * 16;
  int k = 0;
  auto ask = [&](v4i* slot) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < P; ++p)
      load_to_lds(src.from(p), slot + (wave * P + p) * 64, src.off[p], k);
    k += KB;
    __builtin_amdgcn_sched_barrier(0);      // requested before the stage that is there is read
  };
  const int wo = (wave & 1) * (B / 2), wt = (wave >> 1) * (B / 2), n16 = lane & 15, k16 = lane >> 4;
  const int at_w = (wo + n16) * 8 + (k16 ^ (n16 >> 1)), at_x = (B + wt + n16) * 8 + (k16 ^ (n16 >> 1));
  v4i acc[F][F] = {};
  auto mul = [&](const v4i* slot) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      v4i w[F], x[F];
#pragma unroll
      for (int f = 0; f < F; ++f) {
        w[f] = slot[(at_w ^ (4 * j)) + f * 128];
        x[f] = slot[(at_x ^ (4 * j)) + f * 128];
      }
#pragma unroll
      for (int f = 0; f < F; ++f)
#pragma unroll
        for (int g = 0; g < F; ++g) acc[f][g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[f], x[g], acc[f][g], 0, 0, 0);
    }
  };
  auto meet = [&]() __attribute__((always_inline)) { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
  const int stages = a.pitch / KB;
  ask(slot0);
  for (int i = 0; i + 2 < stages; i += 2) {
    meet();                       // slot 0 is there, slot 1 free
    ask(slot1);
    mul(slot0);
    meet();
    ask(slot0);
    mul(slot1);
  }
  meet();
  if (stages & 1) {
    mul(slot0);
  } else {
    ask(slot1);
    mul(slot0);
    meet();
    mul(slot1);
  }
  __syncthreads();
  auto& side = *reinterpret_cast<Side<B, B>*>(slot1);
  side.template load<GATED, 256>(a, r, o0);
  __syncthreads();
  static_assert(sizeof(slot0) >= 4 * 16 * 4 * F * sizeof(v4i) && sizeof(slot1) >= sizeof(side), "turn");
  finish<GATED>(a, r, o0, wo, wt, acc, slot0 + wave * (16 * 4 * F), side);
}

// ------------------------------------------------------------------ large tiles
// 256 rows of weights x 256 tokens a workgroup of eight waves, 128 x 64 a wave.
template <bool GATED>
__global__ __launch_bounds__(512, 2) void token_big_kernel(const TokenProductArgs a, const Order<8> order) {
  constexpr int N = 256, KB = 128, P = 8, WIDTH = GATED ? N / 2 : N;
  // rows of 128 codes: 256 of the weights, then 256 of the tokens; the eight pieces of 16 of a row in an order that differs by pairs of rows
  constexpr int SLOT = 2 * N * KB / 16;
  __shared__ alignas(1024) v4i slots[2 * SLOT];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int ot, id;
  if (!order.tile(blockIdx.x, &ot, &id)) return;
  const Rows r = find_rows<N>(a, id);
  if (r.n <= 0) return;
  const int o0 = ot * WIDTH;
  if (r.e == a.E) {
    put_zeros<WIDTH, 512>(a, r, o0);
    return;
  }
  Source<GATED, N, P> src(a, r, o0, wave * 64);
#pragma unroll
  for (int p = 0; p < P; ++p) src.off[p] += (lane & 7) * 16;
  v4i st[P];
  auto ask = [&](int p, int k) __attribute__((always_inline)) { st[p] = (v4i)__builtin_amdgcn_raw_buffer_load_b128(src.from(p), src.off[p], k, 0); };
  // row wave * 64 + p * 8 + (lane >> 3) has its pieces in the order (row >> 1) & 7
  const int put_at = wave * 512 + (lane >> 3) * 8, swz = lane >> 4;
  auto put = [&](int slot, int p) __attribute__((always_inline)) { slots[slot + put_at + p * 64 + ((lane & 7) ^ (swz + (p & 1) * 4))] = st[p]; };
  const int wo = (wave & 1) * 128, wt = (wave >> 1) * 64, n16 = lane & 15, k16 = lane >> 4;
  const int at_w = (wo + n16) * 8 + (k16 ^ (n16 >> 1)), at_x = (N + wt + n16) * 8 + (k16 ^ (n16 >> 1));
  auto read_w = [&](int slot, int j, int f) __attribute__((always_inline)) { return slots[slot + (at_w ^ (4 * j)) + f * 128]; };
  auto read_x = [&](int slot, int j, int f) __attribute__((always_inline)) { return slots[slot + (at_x ^ (4 * j)) + f * 128]; };
  v4i acc[8][4] = {};
  v4i w[3], x[4];
  // Half a stage, 64 codes: the four tokens' operands are in x, the first three of the weights' in w.  Each of its steps multiplies one of the weights' operands
  // with all of the tokens' and reads what a step three further on takes; `n`, `nj`: where the half after it lies.  MOVE: the next stage's codes go from
  // registers to slot n, the one's after it are requested.  Nothing is read or written in the last step, so that the wait behind it finds all done.
  constexpr int MFMA = 0x008, LOAD = 0x020, READ = 0x100, WRITE = 0x200;
  auto half = [&](int now, auto jj, int n, int to, int k) __attribute__((always_inline)) {
    constexpr int j = decltype(jj)::value, nj = 1 - j;
    constexpr bool MOVE = j == 0;
    constexpr int first[9] = {0, 0, 0, 2, 4, 6, 8, 8, 8};
    v4i ws[11], xn[4];
#pragma unroll
    for (int i = 0; i < 3; ++i) ws[i] = w[i];
#pragma unroll
    for (int f = 0; f < 8; ++f) {
      if (MOVE && f == 2) asm volatile("s_barrier" ::: "memory");      // every wave has read the stage before, whose slot is written from here on
      const int n_read = f < 5 ? 2 : f < 7, n_move = first[f + 1] - first[f];
      if (f < 5) ws[f + 3] = read_w(now, j, f + 3);
      if (f < 4) xn[f] = read_x(n, nj, f);
      else if (f < 7) ws[f + 4] = read_w(n, nj, f - 4);
      if (MOVE) {
#pragma unroll
        for (int p = first[f]; p < first[f + 1]; ++p) {
          put(to, p);
          ask(p, k);
        }
      }
#pragma unroll
      for (int g = 0; g < 4; ++g) acc[f][g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(ws[f], x[g], acc[f][g], 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        __builtin_amdgcn_sched_group_barrier(MFMA, 2, 0);
        if (i < n_read) __builtin_amdgcn_sched_group_barrier(READ, 1, 0);
        if (MOVE && i < n_move) __builtin_amdgcn_sched_group_barrier(WRITE, 1, 0);
        if (MOVE && i < n_move) __builtin_amdgcn_sched_group_barrier(LOAD, 1, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) w[i] = ws[8 + i];
#pragma unroll
    for (int g = 0; g < 4; ++g) x[g] = xn[g];
  };
  auto meet = [&]() __attribute__((always_inline)) { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
  const int last = a.pitch - KB;
#pragma unroll
  for (int p = 0; p < P; ++p) ask(p, 0);
#pragma unroll
  for (int p = 0; p < P; ++p) put(0, p);
#pragma unroll
  for (int p = 0; p < P; ++p) ask(p, min(KB, last));
  meet();
#pragma unroll
  for (int i = 0; i < 3; ++i) w[i] = read_w(0, 0, i);
#pragma unroll
  for (int g = 0; g < 4; ++g) x[g] = read_x(0, 0, g);
  // (the last two stages request the last one's codes again: one loop, whose sums stay where they are)
  int now = 0;
  if (wt < r.n) {
    for (int k = 0; k <= last; k += KB) {
      half(now, std::integral_constant<int, 0>{}, now, now ^ SLOT, min(k + 2 * KB, last));
      meet();
      half(now, std::integral_constant<int, 1>{}, now ^ SLOT, 0, 0);
      now ^= SLOT;
    }
  } else {      // no token of its own: it only loads, and leaves the matrix unit to the other wave (experts' last tiles)
    for (int k = 0; k <= last; k += KB) {
      asm volatile("s_barrier" ::: "memory");
      now ^= SLOT;
#pragma unroll
      for (int p = 0; p < P; ++p) {
        put(now, p);
        ask(p, min(k + 2 * KB, last));
      }
      meet();
    }
  }
  __syncthreads();
  auto& side = *reinterpret_cast<Side<N, N>*>(slots + SLOT);
  side.template load<GATED, 512>(a, r, o0);
  __syncthreads();
  finish<GATED>(a, r, o0, wo, wt, acc, slots + wave * (16 * 32), side);
}

// ------------------------------------------------------------------ launches
enum { AUTOMATIC = 0, STREAM = 1, TILES_64 = 2, TILES_128 = 3, TILES_256 = 4 };

template <int TB>
int launch_stream(const TokenProductArgs& a, bool gated, hipStream_t st) {
  const int o_tiles = (a.out + 15) / 16;
  const int64_t grid = (int64_t)o_tiles * row_tiles<16 * TB>(a);
  if (grid > 0x7fffffff) return PIPE_ESHAPE;
  if (gated) PIPE_KLAUNCH((token_stream_kernel<true, TB>), dim3((unsigned)grid), dim3(512), 0, st, a, o_tiles);
  else PIPE_KLAUNCH((token_stream_kernel<false, TB>), dim3((unsigned)grid), dim3(512), 0, st, a, o_tiles);
  PIPE_HIP(hipGetLastError());
  return PIPE_OK;
}

template <int B>
int launch_tiles(const TokenProductArgs& a, bool gated, hipStream_t st) {
  const int width = gated ? B / 2 : B;
  const int64_t o_tiles = (a.out + width - 1) / width, t_tiles = row_tiles<B>(a), per = (o_tiles * t_tiles + 7) / 8;
  if (per * 8 > 0x7fffffff) return PIPE_ESHAPE;
  const Order<8> order{(int)o_tiles, (int)t_tiles, (int)per};
  const dim3 grid((unsigned)(8 * per));
  if constexpr (B == 256) {
    if (gated) PIPE_KLAUNCH((token_big_kernel<true>), grid, dim3(512), 0, st, a, order);
    else PIPE_KLAUNCH((token_big_kernel<false>), grid, dim3(512), 0, st, a, order);
  } else {
    if (gated) PIPE_KLAUNCH((token_tile_kernel<true, B>), grid, dim3(256), 0, st, a, order);
    else PIPE_KLAUNCH((token_tile_kernel<false, B>), grid, dim3(256), 0, st, a, order);
  }
  PIPE_HIP(hipGetLastError());
  return PIPE_OK;
}

}  // namespace

int launch_token_product(const TokenProductArgs& a, hipStream_t st) {
  const bool gated = a.act == PIPE_ACT_SILU_GATED;
  const int64_t w_rows = gated ? 2 * (int64_t)a.out : a.out;
  int which = g_token_kernel;
  const int64_t each = a.n / a.E;       // tokens of an expert, about
  if (which == AUTOMATIC) {
    if (each <= 64) which = STREAM;
    else if ((w_rows + 255) / 256 * row_tiles<256>(a) >= 256) which = TILES_256;
    else if ((w_rows + 127) / 128 * row_tiles<128>(a) >= 256) which = TILES_128;
    else which = TILES_64;
  }
  if (!near(a)) which = STREAM;
  if (which == TILES_256) return launch_tiles<256>(a, gated, st);
  if (which == TILES_128) return launch_tiles<128>(a, gated, st);
  if (which == TILES_64) return launch_tiles<64>(a, gated, st);
  if (each <= 16) return launch_stream<1>(a, gated, st);
  if (each <= 32) return launch_stream<2>(a, gated, st);
  return launch_stream<4>(a, gated, st);
}
