// Products of 8-bit codes with a scale for each token and each channel, y = act(s_t s_o sum_i c_ti w_oi + b_o), of one layer or of a router's
// experts, whose rows lie one after the other in y.
//
// Sums are exact in 32 bits.  Both scales' exponents are kept apart from their mantissas until the end, so that no product of a sum and one of
// the scales leaves fp32's range where the whole does not.
#include "pipe_attention.h"
#include "pipe_tile.h"
#include "pipe_token.h"

namespace {

typedef int v16i __attribute__((ext_vector_type(16)));

// A tile's rows of y: those of expert e from `row` on, n of them; e == E: rows without an expert.
struct Rows {
  int e, n;
  int64_t row;
};
// Tile `id`: expert e owns the ids from floor(starts[e] / BT) + e on, which are at least as many as its tiles; whole waves.
template <int BT>
__device__ __forceinline__ Rows find_rows(const TokenProductArgs& a, int id) {
  if (a.starts == nullptr) return Rows{0, (int)min((int64_t)BT, a.n - (int64_t)id * BT), (int64_t)id * BT};
  const int lane = threadIdx.x & 63, n = (int)a.n;
  auto start_of = [&](int e) { return e <= 0 ? 0 : min(max(a.starts[min(e, a.E)], 0), n); };
  int e = -1;
  for (int i0 = 0; i0 <= a.E; i0 += 64) {
    const int i = i0 + lane;
    const int found = __popcll(__ballot(i <= a.E && start_of(i) / BT + i <= id));
    e += found;
    if (found < 64) break;
  }
  e = __builtin_amdgcn_readfirstlane(e);
  const int start = __builtin_amdgcn_readfirstlane(start_of(e)), end = e < a.E ? __builtin_amdgcn_readfirstlane(start_of(e + 1)) : n;
  const int skip = (id - start / BT - e) * BT;
  return Rows{e, skip < 0 ? 0 : min(BT, end - start - skip), (int64_t)start + skip};
}
template <int BT>
int row_tiles(const TokenProductArgs& a) {
  return a.starts == nullptr ? (int)((a.n + BT - 1) / BT) : (int)(a.n / BT) + a.E + 1;
}

__device__ __forceinline__ float act_of(float z, int act) {
  if (act == PIPE_ACT_GELU) return gelu_erf(z);
  if (act == PIPE_ACT_RELU) return z < 0.f ? 0.f : z;
  return z;
}
__device__ __forceinline__ float silu(float g) { return g / (1.f + expf(-g)); }

// up to four values of a row of y
__device__ __forceinline__ void put4(void* y, int type, int64_t at, const float* z, int have, bool wide) {
  if (type == PIPE_F32) {
    float* p = (float*)y + at;
    if (wide && have >= 4) { store_row<float, 4>(p, z); return; }
#pragma unroll
    for (int i = 0; i < 4; ++i) if (i < have) p[i] = z[i];
  } else if (type == PIPE_F16) {
    f16* p = (f16*)y + at;
    if (wide && have >= 4) { store_row<f16, 4>(p, z); return; }
#pragma unroll
    for (int i = 0; i < 4; ++i) if (i < have) p[i] = (f16)z[i];
  } else {
    bf16* p = (bf16*)y + at;
    if (wide && have >= 4) { store_row<bf16, 4>(p, z); return; }
#pragma unroll
    for (int i = 0; i < 4; ++i) if (i < have) p[i] = (bf16)z[i];
  }
}

// ------------------------------------------------------------------ tiles through LDS
// 64 rows of weights x 64 tokens a workgroup, 32 x 32 a wave.  A stage is 128 codes of every row, 16 bytes a lane straight to LDS; the eight pieces of 16 of
// a row lie in an order that differs by row, so that the reads of 16 rows' same piece meet all banks.
constexpr int BO = 64, BT = 64, BK = 128;
template <bool GATED>
__global__ __launch_bounds__(256) void token_tile_kernel(const TokenProductArgs a, int o_tiles) {
  __shared__ alignas(1024) v4i ws[BO * BK / 16], xs[BT * BK / 16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int id = blockIdx.x / o_tiles, ot = blockIdx.x - id * o_tiles;
  const Rows r = find_rows<BT>(a, id);
  if (r.n <= 0) return;
  constexpr int WIDTH = GATED ? BO / 2 : BO;      // columns of y
  const int o0 = ot * WIDTH;
  const bool wide = a.out % 4 == 0;
  if (r.e == a.E) {
    for (int i = threadIdx.x; i < r.n * WIDTH; i += 256) {
      const int t = i / WIDTH, o = o0 + i % WIDTH;
      const float zero = 0.f;
      if (o < a.out) put4(a.y, a.type, (r.row + t) * a.out + o, &zero, 1, false);
    }
    return;
  }
  const int w_rows = GATED ? 2 * a.out : a.out;
  // row of the weights behind row i of the tile: 16 of the gate, then 16 of the other half, and so on
  auto weight_row = [&](int i) {
    if (!GATED) return min(o0 + i, a.out - 1);
    return ((i >> 4) & 1) * a.out + min(o0 + (i >> 5) * 16 + (i & 15), a.out - 1);
  };
  auto input_row = [&](int i) -> int64_t {      // -1: none
    const int64_t row = r.row + min(i, r.n - 1);
    if (a.order == nullptr) return row < a.n_x ? row : -1;
    const int64_t o = a.order[row];
    return o >= 0 && o < a.n_x * a.top_k ? o / a.top_k : -1;
  };
  constexpr int PIECES = (BO + BT) / 8 / 4;       // a wave's loads of 8 rows a stage
  const int8_t* src[PIECES];
  v4i* dst[PIECES];
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    const int piece = wave * PIECES + p, row = (piece % (BO / 8)) * 8 + (lane >> 3);
    const int col = ((lane & 7) ^ (row & 7)) * 16;
    static_assert(BO == BT, "pieces");
    if (piece < BO / 8) src[p] = a.w + ((int64_t)r.e * w_rows + weight_row(row)) * a.pitch + col;
    else src[p] = a.qx + max(input_row(row), (int64_t)0) * a.pitch + col;
    dst[p] = (piece < BO / 8 ? ws : xs) + (piece % (BO / 8)) * 64;
  }
  v4i acc[2][2] = {};
  const int wo = (wave & 1) * 32, wt = (wave >> 1) * 32, n16 = lane & 15, k16 = lane >> 4;
  for (int k = 0; k < a.pitch; k += BK) {
    __syncthreads();
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src[p], (__attribute__((address_space(3))) void*)dst[p], 16, 0, 0);
      src[p] += BK;
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      v4i w[2], x[2];
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const int ro = wo + f * 16 + n16, rt = wt + f * 16 + n16;
        w[f] = ws[ro * 8 + ((j * 4 + k16) ^ (ro & 7))];
        x[f] = xs[rt * 8 + ((j * 4 + k16) ^ (rt & 7))];
      }
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int g = 0; g < 2; ++g) acc[f][g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[f], x[g], acc[f][g], 0, 0, 0);
    }
  }
  // a lane holds four channels of one token a block of 16 x 16
  const float* sw = a.sw + (int64_t)r.e * w_rows;
  const float* bias = a.bias ? a.bias + (int64_t)r.e * w_rows : nullptr;
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const int t = wt + g * 16 + n16;
    if (t >= r.n) continue;
    const int64_t in = input_row(t);
    const float sx = in < 0 ? 0.f : a.sx[in], mx = __builtin_amdgcn_frexp_mantf(sx);
    const int ex = __builtin_amdgcn_frexp_expf(sx);
    float z[2][4];
#pragma unroll
    for (int f = 0; f < 2; ++f)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int o = weight_row(wo + f * 16 + 4 * k16 + i);
        const float s = sw[o];
        z[f][i] = __builtin_amdgcn_ldexpf((float)acc[f][g][i] * mx * __builtin_amdgcn_frexp_mantf(s), ex + __builtin_amdgcn_frexp_expf(s));
        if (bias) z[f][i] += bias[o];
      }
    const int64_t at = (r.row + t) * a.out;
    if (GATED) {
      const int o = o0 + (wo >> 1) + 4 * k16;
#pragma unroll
      for (int i = 0; i < 4; ++i) z[0][i] = in < 0 ? 0.f : silu(z[0][i]) * z[1][i];
      put4(a.y, a.type, at + o, z[0], a.out - o, wide);
    } else {
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const int o = o0 + wo + f * 16 + 4 * k16;
#pragma unroll
        for (int i = 0; i < 4; ++i) z[f][i] = in < 0 ? 0.f : act_of(z[f][i], a.act);
        put4(a.y, a.type, at + o, z[f], a.out - o, wide);
      }
    }
  }
}

}  // namespace

int launch_token_product(const TokenProductArgs& a, hipStream_t st) {
  const bool gated = a.act == PIPE_ACT_SILU_GATED;
  const int width = gated ? BO / 2 : BO, o_tiles = (a.out + width - 1) / width;
  const int64_t grid = (int64_t)o_tiles * row_tiles<BT>(a);
  if (grid > 0x7fffffff) return PIPE_ESHAPE;
  if (gated) PIPE_KLAUNCH((token_tile_kernel<true>), dim3((unsigned)grid), dim3(256), 0, st, a, o_tiles);
  else PIPE_KLAUNCH((token_tile_kernel<false>), dim3((unsigned)grid), dim3(256), 0, st, a, o_tiles);
  PIPE_HIP(hipGetLastError());
  return PIPE_OK;
}
