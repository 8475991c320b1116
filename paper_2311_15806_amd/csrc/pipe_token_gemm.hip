// Products of 8-bit codes with a scale for each token and each channel, y = act(s_t s_o sum_i c_ti w_oi + b_o), of one layer or of a router's
// experts, whose rows lie one after the other in y.
//
// What bounds them: few tokens, the weights' bytes (32 tokens, six of 64 gated experts of 2048-1408, 370 MB: 69 us, 5.4 TB/s; 16 tokens of gated
// 4096-11008, 90 MB: 19 us); many, the matrix units at the clock that power leaves: 8192 tokens of 8192-8192 take 477 us, 39 of them the
// codes: 2510 TOP/s of the product, where the library's largest of that size reaches 2134 and multiplies alone, on random bytes, 3764.  Between them latency: a stage of 128 codes takes a tile of 64
// tokens that is alone on its unit 0.45 us, of 128 0.95, of 256 1.3.
//
// Sums are exact in 32 bits.  Both scales' exponents are kept apart from their mantissas until the end, so that no product of a sum and one of
// the scales leaves fp32's range where the whole does not.  Every kernel here computes an output by the same operations: which one serves a call
// changes no bit.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "pipe_attention.h"
#include "pipe_codes.h"
#include "pipe_tile.h"
#include "pipe_token.h"

int g_token_kernel = 0;

namespace {

// ------------------------------------------------------------------ what the kernels share
// A tile's rows of y: those of expert e from `row` on, n of them.
struct Rows {
  int e, n;
  int64_t row;
};
// sums over a wave's lanes up to and with each, by moves within the vector unit
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_add(int v) { return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int wave_sums(int v) {
  v = dpp_add<0x111, 0xf>(v);   // row_shr 1, 2, 4, 8
  v = dpp_add<0x112, 0xf>(v);
  v = dpp_add<0x114, 0xf>(v);
  v = dpp_add<0x118, 0xf>(v);
  v = dpp_add<0x142, 0xa>(v);   // row_bcast 15, 31
  return dpp_add<0x143, 0xc>(v);
}
// How many tiles of BT rows the experts have, one expert's after the other's.  Called by whole waves, a lane an expert; so is what follows.
template <int BT>
struct Experts {
  int start, end, tiles, upto;      // of the lane's expert: its rows, its tiles, all up to with them
  __device__ __forceinline__ Experts(const TokenProductArgs& a, int e0, int before) {
    const int e = e0 + (threadIdx.x & 63), n = (int)a.n;
    start = e > 0 ? min(max(a.starts[min(e, a.E)], 0), n) : 0;
    end = min(max(a.starts[min(e + 1, a.E)], 0), n);
    tiles = e < a.E && end > start ? (end - start + BT - 1) / BT : 0;
    upto = before + wave_sums(tiles);
  }
};
template <int BT>
__device__ __forceinline__ int live_tiles(const TokenProductArgs& a) {
  if (a.starts == nullptr) return (int)((a.n + BT - 1) / BT);
  int before = 0;
  for (int e0 = 0; e0 < a.E; e0 += 64) before = __builtin_amdgcn_readlane(Experts<BT>(a, e0, before).upto, 63);
  return before;
}
// Tile `id` of them; no rows: there is none.
template <int BT>
__device__ __forceinline__ Rows find_rows(const TokenProductArgs& a, int id) {
  if (a.starts == nullptr) return Rows{0, (int)min((int64_t)BT, a.n - (int64_t)id * BT), (int64_t)id * BT};
  int before = 0;
  for (int e0 = 0; e0 < a.E; e0 += 64) {
    const Experts<BT> x(a, e0, before);
    const int at = __popcll(__ballot(x.upto <= id));
    if (at < 64) {
      const int s = __builtin_amdgcn_readlane(x.start, at) + (id - __builtin_amdgcn_readlane(x.upto - x.tiles, at)) * BT;
      return Rows{e0 + at, min(BT, __builtin_amdgcn_readlane(x.end, at) - s), s};
    }
    before = __builtin_amdgcn_readlane(x.upto, 63);
  }
  return Rows{0, 0, 0};
}
// (never more tiles than this)
template <int BT>
int64_t row_tiles(const TokenProductArgs& a) {
  return a.starts == nullptr ? (a.n + BT - 1) / BT : a.n / BT + std::min<int64_t>(a.E, a.n);
}
// The rows of y behind the last expert's, zeros: a share for every workgroup of the launch.
template <int NT>
__device__ __forceinline__ void zero_rest(const TokenProductArgs& a) {
  if (a.starts == nullptr) return;
  const int64_t size = a.type == PIPE_F32 ? 4 : 2, first = (int64_t)min(max(a.starts[a.E], 0), (int)a.n) * a.out * size, end = a.n * a.out * size;
  const int64_t lo = (first + 15) / 16, hi = end / 16;      // whole pieces; what lies before and behind them is the first workgroup's
  char* y = (char*)a.y;
  for (int64_t i = lo + (int64_t)blockIdx.x * NT + threadIdx.x; i < hi; i += (int64_t)gridDim.x * NT) reinterpret_cast<uint4*>(y)[i] = make_uint4(0, 0, 0, 0);
  if (blockIdx.x == 0 && threadIdx.x < 16) {
    const int64_t before = first + threadIdx.x * 2, behind = max(hi * 16, first) + threadIdx.x * 2;
    if (before < min(lo * 16, end)) *reinterpret_cast<uint16_t*>(y + before) = 0;
    if (behind < end) *reinterpret_cast<uint16_t*>(y + behind) = 0;
  }
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
// SiLU(g) u of four channels.  (The exponential's argument is one rounding off: 2^-24 |g| of the value, what the product g with anything may be off by as well.)
// Beyond -87 the denominator's reciprocal is below fp32's normal numbers, where the instruction gives zero, beyond -88.7 the exponential above all of them, while
// SiLU is neither until -103: below -64 both are taken 2^32 smaller, beside which 1 is nothing, and the quotient brought back (4096 tokens, two of eight gated
// experts of 4096-11008: 4 to 5 of 770 us).
constexpr float SILU_FAR = -64.f;
__device__ __forceinline__ float silu(float g) { return g * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(g * -1.44269504f)); }
__device__ __forceinline__ float silu_far(float g) {
  return __builtin_amdgcn_ldexpf(g * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(__fmaf_rn(g, -1.44269504f, -32.f))), -32);
}
__device__ __forceinline__ void gate4(float* g, const float* u) {
  const float low = fminf(fminf(g[0], g[1]), fminf(g[2], g[3]));
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = silu(g[i]) * u[i];
  if (__builtin_expect(__any(low < SILU_FAR), 0)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = g[i] < SILU_FAR ? silu_far(g[i]) * u[i] : y[i];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) g[i] = y[i];
}

// Four channels' scales and biases: z = (sum s_t) s_o + b.  The product is made of the scales' mantissas and scaled by both exponents at once -- or, where
// these are so small (`plain`) that nothing on the way leaves fp32's normal range (a sum is below 2^31, each scale from 2^-49 up to below 2^48), of the
// scales as they are, which gives the same bits (4096 tokens of 4096-11008, fp32: 204 us, 199 so).
constexpr int PLAIN_EXPONENT = 48;
__device__ __forceinline__ bool plain_scale(float s) {
  const int e = __builtin_amdgcn_frexp_expf(s);
  return e <= PLAIN_EXPONENT && e >= -PLAIN_EXPONENT;
}
struct Channels {
  float s[4], b[4];
  __device__ __forceinline__ void set(int i, float scale, float bias) {
    s[i] = scale;
    b[i] = bias;
  }
  __device__ __forceinline__ bool plain() const { return plain_scale(s[0]) && plain_scale(s[1]) && plain_scale(s[2]) && plain_scale(s[3]); }
  template <bool PLAIN = false>
  __device__ __forceinline__ void values(const v4i& sum, float sx, bool with_bias, float* z) const {
    const float mx = __builtin_amdgcn_frexp_mantf(sx);
    const int ex = __builtin_amdgcn_frexp_expf(sx);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (PLAIN) z[i] = __fmul_rn(__fmul_rn((float)sum[i], sx), s[i]);
      else z[i] = __builtin_amdgcn_ldexpf(__fmul_rn(__fmul_rn((float)sum[i], mx), __builtin_amdgcn_frexp_mantf(s[i])), ex + __builtin_amdgcn_frexp_expf(s[i]));
      if (with_bias) z[i] = __fadd_rn(z[i], b[i]);
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
// PLAIN: no scale is far from 1 (see Channels) and every token has an input.
template <typename T, bool PLAIN, bool GATED, int FO, int FT, int BO, int BT>
__device__ __forceinline__ void finish_as(const TokenProductArgs& a, const Rows& r, int o0, int wo, int wt, const v4i (&acc)[FO][FT], v4i* turn,
                                          const Side<BO, BT>& side, const Channels& c0, const Channels& c1) {
  constexpr int PIECES = 4 * FO, LANES = GATED ? PIECES / 2 : PIECES;      // lanes of a token, 4 columns each
  constexpr int SH = PIECES == 32 ? 1 : 0, DOWN = PIECES == 8 ? 1 : 0, STEP = 64 / LANES;
  const int lane = threadIdx.x & 63, n16 = lane & 15, k16 = lane >> 4;
  const int col = lane % LANES, first = lane / LANES, piece = GATED ? (col >> 2) * 8 + (col & 3) : col;
  const int o = o0 + (GATED ? wo / 2 : wo) + col * 4, have = a.out - o;
  const bool wide = a.out % 4 == 0, with_bias = a.bias != nullptr;
  T* y = (T*)a.y + (r.row + wt + first) * a.out + o;
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
    for (int t = first; t < 16; t += STEP) {
      const float sx = side.sx[t0 + t];
      const v4i* row = turn + t * PIECES;
      float z[4];
      c0.template values<PLAIN>(row[piece ^ (t << SH >> DOWN)], sx, with_bias, z);
      if (GATED) {
        float u[4];
        c1.template values<PLAIN>(row[(piece + 4) ^ (t << SH >> DOWN)], sx, with_bias, u);
        gate4(z, u);
      } else {
        act4(z, a.act);
      }
      if (!PLAIN && sx < 0.f) z[0] = z[1] = z[2] = z[3] = 0.f;
      if (t0 + t < r.n) put4_typed(y, z, have, wide);
      y += (int64_t)STEP * a.out;
    }
    __builtin_amdgcn_wave_barrier();
  }
}
template <bool GATED, int FO, int FT, int BO, int BT>
__device__ __forceinline__ void finish(const TokenProductArgs& a, const Rows& r, int o0, int wo, int wt, const v4i (&acc)[FO][FT], v4i* turn,
                                       const Side<BO, BT>& side) {
  constexpr int PIECES = 4 * FO, LANES = GATED ? PIECES / 2 : PIECES;
  static_assert(PIECES == 8 || PIECES == 16 || PIECES == 32, "turn");
  static_assert(FT * 16 <= 64, "a lane a token");
  const int lane = threadIdx.x & 63, col = lane % LANES, i0 = wo + (GATED ? (col >> 2) * 8 + (col & 3) : col) * 4;
  Channels c0, c1;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    c0.set(i, side.sw[i0 + i], side.bias[i0 + i]);
    c1.set(i, side.sw[i0 + (GATED ? 16 : 0) + i], side.bias[i0 + (GATED ? 16 : 0) + i]);
  }
  const float sx = side.sx[wt + min(lane, FT * 16 - 1)];
  const bool plain = __all(c0.plain() && c1.plain() && plain_scale(sx) && !(sx < 0.f));
  if (a.type == PIPE_F32) {
    if (plain) finish_as<float, true, GATED>(a, r, o0, wo, wt, acc, turn, side, c0, c1);
    else finish_as<float, false, GATED>(a, r, o0, wo, wt, acc, turn, side, c0, c1);
  } else if (a.type == PIPE_F16) {
    if (plain) finish_as<f16, true, GATED>(a, r, o0, wo, wt, acc, turn, side, c0, c1);
    else finish_as<f16, false, GATED>(a, r, o0, wo, wt, acc, turn, side, c0, c1);
  } else {
    if (plain) finish_as<bf16, true, GATED>(a, r, o0, wo, wt, acc, turn, side, c0, c1);
    else finish_as<bf16, false, GATED>(a, r, o0, wo, wt, acc, turn, side, c0, c1);
  }
}

// an address that is the same in every lane, in scalar registers
__device__ __forceinline__ const int8_t* uniform(const int8_t* p) {
  const uint64_t u = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)u), hi = __builtin_amdgcn_readfirstlane((uint32_t)(u >> 32));
  return reinterpret_cast<const int8_t*>((uint64_t)hi << 32 | lo);
}
// Where a wave's loads of 8 rows x 128 codes come from: row `first` + 8 p + (lane >> 3) of the tile's B rows of weights (first < B) or of its tokens.
// Addresses are a resource's base and 32 bits, FAR: of tokens 64 bits; of a gated layer 16 rows of the gate and of the other half in turn.
template <bool GATED, int B, int P, bool FAR = false>
struct Source {
  const int8_t *b0, *b1;
  unsigned off[P];
  const int8_t* far[FAR ? P : 1];
  bool by_far;
  __device__ __forceinline__ Source(const TokenProductArgs& a, const Rows& r, int o0, int first) {
    const int lane = threadIdx.x & 63;
    const bool weights = first < B;
    if (weights) {
      b0 = a.w + ((int64_t)r.e * w_rows_of(a, GATED) + o0) * a.pitch;
      b1 = GATED ? b0 + (int64_t)a.out * a.pitch : b0;
    } else {
      b0 = b1 = a.qx + (a.order ? 0 : r.row) * a.pitch;
    }
    b0 = uniform(b0);
    b1 = uniform(b1);
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int row = first + p * 8 + (lane >> 3);
      int64_t at;
      if (weights) at = min(o0 + (GATED ? (row >> 5) * 16 + (row & 15) : row), a.out - 1) - o0;
      else at = max(input_of(a, r, row - B), (int64_t)0) - (a.order ? 0 : r.row);
      off[p] = (unsigned)(at * a.pitch) + (lane & 7) * 16;
      if (FAR) far[p] = b0 + at * a.pitch + (lane & 7) * 16;
    }
    by_far = FAR && !weights;
  }
  // load p of the codes from k on; zeros, without an access, where there are none
  __device__ __forceinline__ v4i load(int p, int k, int pitch) const {
    if (FAR && by_far) return (v4i)gload16(far[p] + min(k, pitch - 128));      // (behind the end the last codes again, for a slot that nobody reads)
    const __amdgpu_buffer_rsrc_t from =
        __builtin_amdgcn_make_buffer_rsrc((void*)uniform(((p >> 1) & 1) ? b1 : b0), 0, __builtin_amdgcn_readfirstlane(k < pitch ? 0xffffffffu : 0u), 0x00020000);
    return (v4i)__builtin_amdgcn_raw_buffer_load_b128(from, off[p], k, 0);
  }
};
// whether 32 bits reach every input
static bool near(const TokenProductArgs& a) { return a.order == nullptr || a.n_x * a.pitch < (int64_t)0xffffffff; }

// Which tile a workgroup takes, of o_tiles x t_tiles.  Blocks b, b + 8, ... of a launch run on one XCD (one L2), which takes an eighth of all tiles: 8 tiles of
// tokens x some of weights next to each other.  (Chunks of 8 x 4 tiles dealt to the XCDs in turn: 4096 tokens of 4096-11008 227 us for 217, eight
// gated experts 905 for 870.)
__device__ __forceinline__ bool place_of(int o_tiles, int t_tiles, int* ot, int* id) {
  const int all = o_tiles * t_tiles, per_xcd = (all + 7) / 8, at = blockIdx.x >> 3, place = (blockIdx.x & 7) * per_xcd + at;
  if (at >= per_xcd || place >= all) return false;
  const int band = place / (8 * o_tiles), in_band = place - band * 8 * o_tiles, high = min(8, t_tiles - band * 8);
  *ot = in_band / high;
  *id = band * 8 + in_band - *ot * high;
  return true;
}

// ------------------------------------------------------------------ few tokens
// the lane's four channels of token t of a tile
template <bool GATED>
__device__ __forceinline__ void outputs(const TokenProductArgs& a, const Rows& r, int o0, int t, const Channels* ch, const v4i* sum, float sx, bool none) {
  float z[2][4];
  ch[0].values(sum[0], sx, a.bias != nullptr, z[0]);
  if (GATED) {
    ch[GATED].values(sum[GATED], sx, a.bias != nullptr, z[1]);
    gate4(z[0], z[1]);
  } else {
    act4(z[0], a.act);
  }
  if (none) z[0][0] = z[0][1] = z[0][2] = z[0][3] = 0.f;
  const int o = o0 + 4 * ((threadIdx.x & 63) >> 4);
  put4(a.y, a.type, (r.row + t) * a.out + o, z[0], a.out - o, a.out % 4 == 0);
}
// The weights go straight from memory to operands.  A tile is 16 rows of weights (of the gate and of the other half as well) x
// 16 TB tokens; S of a workgroup's eight waves take its steps of 64 codes in turn and join their sums in LDS.
template <bool GATED, int TB, int S>
__global__ __launch_bounds__(512, 4) void token_stream_kernel(const TokenProductArgs a, int o_tiles, int tiles) {
  constexpr int G = GATED ? 2 : 1;
  constexpr int U = TB + G <= 2 ? 4 : TB + G == 3 ? 3 : 2;      // steps of a set of registers: two workgroups a unit
  __shared__ v4i part[S > 1 ? 8 : 1][G * TB][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), sub = wave % S;
  const int tile = blockIdx.x * (8 / S) + wave / S;
  const int id = tile / o_tiles, o0 = (tile - id * o_tiles) * 16;
  Rows r{0, 0, 0};
  if (tile < tiles) r = find_rows<16 * TB>(a, id);
  zero_rest<512>(a);
  const bool live = r.n > 0;
  if (S == 1 && !live) return;
  const int n16 = lane & 15, k16 = lane >> 4;
  v4i acc[G][TB] = {};
  // what the end takes is requested first: scales and biases of the lane's four channels, and of its token the wave's of the blocks it finishes
  Channels ch[G];
  float sx = 0.f;
  bool none = true;
  const int b_own = S > 1 ? min(sub, TB - 1) : 0;
  if (live) {
    const int64_t w0 = (int64_t)r.e * w_rows_of(a, GATED);
    // weights through a resource of the 16 rows, behind whose end a step beyond the last reads zeros; tokens at 64 bits
    __amdgpu_buffer_rsrc_t from[G];
#pragma unroll
    for (int h = 0; h < G; ++h)
      from[h] = __builtin_amdgcn_make_buffer_rsrc((void*)uniform(a.w + (w0 + h * a.out + o0) * a.pitch), 0, (unsigned)(min(16, a.out - o0) * a.pitch), 0x00020000);
    const unsigned w_at = (unsigned)(min(n16, a.out - 1 - o0) * a.pitch + k16 * 16);
    const int steps = a.pitch / 64;
    struct Set {
      v4i w[U][G], x[U][TB];
    } s0, s1;
    auto ask_w = [&](Set& q, int s) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int k = s + u * S;
#pragma unroll
        for (int h = 0; h < G; ++h) q.w[u][h] = (v4i)__builtin_amdgcn_raw_buffer_load_b128(from[h], w_at + (k < steps ? k * 64u : 0x80000000u), 0, 0);
      }
    };
    const int8_t* xp[TB];
    auto ask_x = [&](Set& q, int s) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int b = 0; b < TB; ++b) q.x[u][b] = (v4i)gload16(xp[b] + min(s + u * S, steps - 1) * 64);
    };
    auto mul = [&](const Set& q) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int h = 0; h < G; ++h)
#pragma unroll
          for (int b = 0; b < TB; ++b) acc[h][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(q.w[u][h], q.x[u][b], acc[h][b], 0, 0, 0);
    };
    int s = sub;
    ask_w(s0, s);
#pragma unroll
    for (int b = 0; b < TB; ++b) {
      const int64_t in = input_of(a, r, 16 * b + n16);
      xp[b] = a.qx + max(in, (int64_t)0) * a.pitch + k16 * 16;
      if (TB == 1 || (S > 1 && b == b_own)) { none = in < 0; sx = a.sx[max(in, (int64_t)0)]; }
    }
    ask_x(s0, s);
#pragma unroll
    for (int h = 0; h < G; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t o = w0 + weight_of<GATED>(a, o0, 16 * h + 4 * k16 + i);
        ch[h].set(i, a.sw[o], a.bias ? a.bias[o] : 0.f);
      }
    while (true) {
      s += U * S;
      if (s >= steps) { mul(s0); break; }
      ask_w(s1, s);
      ask_x(s1, s);
      mul(s0);
      s += U * S;
      if (s >= steps) { mul(s1); break; }
      ask_w(s0, s);
      ask_x(s0, s);
      mul(s1);
    }
  }
  if constexpr (S == 1) {
#pragma unroll
    for (int b = 0; b < TB; ++b) {
      if (TB > 1) {
        const int64_t in = input_of(a, r, 16 * b + n16);
        none = in < 0;
        sx = a.sx[max(in, (int64_t)0)];
      }
      v4i sum[G];
#pragma unroll
      for (int h = 0; h < G; ++h) sum[h] = acc[h][b];
      if (16 * b + n16 < r.n) outputs<GATED>(a, r, o0, 16 * b + n16, ch, sum, sx, none);
    }
  } else {
    static_assert(S >= TB, "a block of tokens a wave");
#pragma unroll
    for (int h = 0; h < G; ++h)
#pragma unroll
      for (int b = 0; b < TB; ++b) part[wave][h * TB + b][lane] = acc[h][b];
    __syncthreads();
    if (!live || sub >= TB) return;
    v4i sum[G];
#pragma unroll
    for (int h = 0; h < G; ++h) {
      sum[h] = part[wave - sub][h * TB + sub][lane];
#pragma unroll
      for (int q = 1; q < S; ++q) sum[h] += part[wave - sub + q][h * TB + sub][lane];
    }
    if (16 * sub + n16 < r.n) outputs<GATED>(a, r, o0, 16 * sub + n16, ch, sum, sx, none);
  }
}

// The same for a call of up to FUSED_CODES codes in one launch: every workgroup makes the codes of its tile's tokens itself, while its first weights are on
// their way.  (One token of 4096-4096 in bf16: 7.3 us a call, 5.4 on the device; two launches 13.0 and 7.2.)
constexpr int FUSED_CODES = 8192, FUSED_TILES = 1024;
template <bool GATED, typename T>
__global__ __launch_bounds__(512, 4) void token_stream_fused_kernel(const TokenProductArgs a, int o_tiles) {
  constexpr int G = GATED ? 2 : 1, U = 4, S = 8, EACH = FUSED_CODES / 8 / 512;
  __shared__ v4i part[8][G][64];
  __shared__ alignas(16) int8_t codes[FUSED_CODES];
  __shared__ uint32_t top[16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (threadIdx.x < 16) top[threadIdx.x] = 0;
  const int id = blockIdx.x / o_tiles, o0 = (blockIdx.x - id * o_tiles) * 16;
  const Rows r = find_rows<16>(a, id);
  zero_rest<512>(a);
  if (r.n <= 0) return;
  const int n16 = lane & 15, k16 = lane >> 4;
  const int64_t w0 = (int64_t)r.e * w_rows_of(a, GATED);
  __amdgpu_buffer_rsrc_t from[G];
#pragma unroll
  for (int h = 0; h < G; ++h)
    from[h] = __builtin_amdgcn_make_buffer_rsrc((void*)uniform(a.w + (w0 + h * a.out + o0) * a.pitch), 0, (unsigned)(min(16, a.out - o0) * a.pitch), 0x00020000);
  const unsigned w_at = (unsigned)(min(n16, a.out - 1 - o0) * a.pitch + k16 * 16);
  const int steps = a.pitch / 64;
  v4i w0s[U][G], w1s[U][G];
  auto ask = [&](v4i (&q)[U][G], int s) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = s + u * S;
#pragma unroll
      for (int h = 0; h < G; ++h) q[u][h] = (v4i)__builtin_amdgcn_raw_buffer_load_b128(from[h], w_at + (k < steps ? k * 64u : 0x80000000u), 0, 0);
    }
  };
  ask(w0s, wave);
  // 8 values a piece, pieces of the tile's tokens one after the other; 16 neighbouring lanes' are one token's
  const int per_row = a.pitch / 8, pieces = r.n * per_row;
  float v[EACH][8];
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    const int g = threadIdx.x + j * 512, row = g / per_row, c = (g - row * per_row) * 8;
    const int64_t in = g < pieces ? input_of(a, r, row) : -1;
    const T* x = (const T*)a.x + max(in, (int64_t)0) * a.x_stride + c;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[j][i] = 0.f;
    if (in >= 0) {
      if (a.x_wide && c + 8 <= a.in) {
        load8<T, true>(x, v[j]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (c + i < a.in) v[j][i] = to_f(x[i]);
      }
    }
  }
  ask(w1s, wave + U * S);
  const int64_t in = input_of(a, r, n16);
  Channels ch[G];
#pragma unroll
  for (int h = 0; h < G; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t o = w0 + weight_of<GATED>(a, o0, 16 * h + 4 * k16 + i);
      ch[h].set(i, a.sw[o], a.bias ? a.bias[o] : 0.f);
    }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    const int g = threadIdx.x + j * 512;
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) bits = raised(bits, v[j][i]);
    const float m = row_reduce<16, true>(top_of(bits));
    if (g < pieces && (lane & 15) == 0) atomicMax(&top[g / per_row], __float_as_uint(m));
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    const int g = threadIdx.x + j * 512;
    if (g < pieces) {
      const RowScale s(__uint_as_float(top[g / per_row]));
      *reinterpret_cast<uint2*>(codes + g * 8) = s.codes8(v[j]);
    }
  }
  __syncthreads();
  v4i acc[G] = {};
  const int x_at = min(n16, r.n - 1) * a.pitch + k16 * 16;
  auto mul = [&](const v4i (&q)[U][G], int s) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const v4i x = *reinterpret_cast<const v4i*>(codes + x_at + min(s + u * S, steps - 1) * 64);
#pragma unroll
      for (int h = 0; h < G; ++h) acc[h] = __builtin_amdgcn_mfma_i32_16x16x64_i8(q[u][h], x, acc[h], 0, 0, 0);
    }
  };
  // (two sets of U steps of eight waves hold 4096 codes of a row, a longer one takes two sets more)
  mul(w0s, wave);
  if (steps > 2 * U * S) ask(w0s, wave + 2 * U * S);
  mul(w1s, wave + U * S);
  if (steps > 2 * U * S) {
    ask(w1s, wave + 3 * U * S);
    mul(w0s, wave + 2 * U * S);
    mul(w1s, wave + 3 * U * S);
  }
  static_assert(FUSED_CODES == 4 * U * S * 64, "steps");
#pragma unroll
  for (int h = 0; h < G; ++h) part[wave][h][lane] = acc[h];
  __syncthreads();
  if (wave > 0 || n16 >= r.n) return;
  v4i sum[G];
#pragma unroll
  for (int h = 0; h < G; ++h) {
    sum[h] = part[0][h][lane];
#pragma unroll
    for (int q = 1; q < S; ++q) sum[h] += part[q][h][lane];
  }
  outputs<GATED>(a, r, o0, n16, ch, sum, RowScale(__uint_as_float(top[n16])).scale(), in < 0);
}

// ------------------------------------------------------------------ tiles
// B rows of weights x B tokens a workgroup of four waves, a quarter each.  A stage is 128 codes of every row; the eight pieces of 16 of a row lie in
// LDS in an order that differs by pairs of rows, so that the reads of 16 rows' same piece meet all banks.  One stage is in LDS ahead, D more are in
// registers or on their way there.
template <bool GATED, int B, int D, bool FAR>
__global__ __launch_bounds__(256, B == 128 ? 2 : 4) void token_tile_kernel(const TokenProductArgs a, int o_tiles) {
  constexpr int KB = 128, P = B / 16, F = B / 32, WIDTH = GATED ? B / 2 : B, SLOT = 2 * B * KB / 16;
  __shared__ alignas(1024) v4i slots[2 * SLOT];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int ot, id;
  zero_rest<256>(a);
  if (!place_of(o_tiles, live_tiles<B>(a), &ot, &id)) return;
  const Rows r = find_rows<B>(a, id);
  const int o0 = ot * WIDTH;
  const Source<GATED, B, P, FAR> src(a, r, o0, wave * (B / 2));
  v4i st[D][P];
  auto ask = [&](v4i (&q)[P], int k) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < P; ++p) q[p] = src.load(p, k, a.pitch);
    __builtin_amdgcn_sched_barrier(0);      // in this order, which the waits count on
  };
  const int put_at = wave * (P * 64) + (lane >> 3) * 8, swz = lane >> 4;
  auto put = [&](int slot, const v4i (&q)[P]) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < P; ++p) slots[slot + put_at + p * 64 + ((lane & 7) ^ (swz + (p & 1) * 4))] = q[p];
  };
  const int wo = (wave & 1) * (B / 2), wt = (wave >> 1) * (B / 2), n16 = lane & 15, k16 = lane >> 4;
  const int at_w = (wo + n16) * 8 + (k16 ^ (n16 >> 1)), at_x = (B + wt + n16) * 8 + (k16 ^ (n16 >> 1));
  v4i acc[F][F] = {};
  auto mul = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      v4i w[F], x[F];
#pragma unroll
      for (int f = 0; f < F; ++f) {
        w[f] = slots[slot + (at_w ^ (4 * j)) + f * 128];
        x[f] = slots[slot + (at_x ^ (4 * j)) + f * 128];
      }
#pragma unroll
      for (int f = 0; f < F; ++f)
#pragma unroll
        for (int g = 0; g < F; ++g) acc[f][g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[f], x[g], acc[f][g], 0, 0, 0);
    }
  };
  auto meet = [&]() __attribute__((always_inline)) { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
  // set i holds stages i, i + D, ...; in its turn a stage finds its codes in LDS and moves the next one's there, whose registers take the stage D later
#pragma unroll
  for (int i = 0; i < D; ++i) ask(st[i], i * KB);
  put(0, st[0]);
  ask(st[0], D * KB);
  meet();
  int now = 0, k = 0;
  for (; k + (D - 1) * KB < a.pitch; k += D * KB) {      // (one way through: with an exit in the middle every wait would be for all loads)
#pragma unroll
    for (int i = 0; i < D; ++i) {
      put(now ^ SLOT, st[(i + 1) % D]);
      ask(st[(i + 1) % D], k + (i + 1 + D) * KB);
      mul(now);
      meet();
      now ^= SLOT;
    }
  }
#pragma unroll
  for (int i = 0; i + 1 < D; ++i)
    if (k + i * KB < a.pitch) {
      if (i + 2 < D) put(now ^ SLOT, st[(i + 1) % D]);
      mul(now);
      meet();
      now ^= SLOT;
    }
  auto& side = *reinterpret_cast<Side<B, B>*>(slots + SLOT);
  side.template load<GATED, 256>(a, r, o0);
  __syncthreads();
  static_assert(SLOT >= 4 * 16 * 4 * F && SLOT * sizeof(v4i) >= sizeof(side), "turn");
  if (wt < r.n) finish<GATED>(a, r, o0, wo, wt, acc, slots + wave * (16 * 4 * F), side);
}

// ------------------------------------------------------------------ large tiles
// 256 rows of weights x 256 tokens a workgroup of eight waves, 128 x 64 a wave: 128 sums a lane, two waves a SIMD (four waves of 128 x 128 leave no register for
// what is on its way).  At 4096 tokens of 4096-11008 the matrix units are busy 46 % of the time: a stage takes 3100 cycles for 2048 of multiplies, the rest of a tile
// (first loads, outputs, whose stores all units send at once) 12 to 15 us beside 47, and 688 tiles make 2.7 rounds.  Loads straight to LDS, 64 codes a
// stage: 250 us for 200; lines of the stage after next requested ahead: 226 for 220.
template <bool GATED>
__global__ __launch_bounds__(512, 2) void token_big_kernel(const TokenProductArgs a, int o_tiles) {
  constexpr int N = 256, KB = 128, P = 8, WIDTH = GATED ? N / 2 : N;
  // rows of 128 codes: 256 of the weights, then 256 of the tokens; the eight pieces of 16 of a row in an order that differs by pairs of rows
  constexpr int SLOT = 2 * N * KB / 16;
  __shared__ alignas(1024) v4i slots[2 * SLOT];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int ot, id;
  zero_rest<512>(a);
  if (!place_of(o_tiles, live_tiles<N>(a), &ot, &id)) return;
  const Rows r = find_rows<N>(a, id);
  const int o0 = ot * WIDTH;
  const Source<GATED, N, P> src(a, r, o0, wave * 64);
  v4i st[P];
  auto ask = [&](int p, int k) __attribute__((always_inline)) { st[p] = src.load(p, k, a.pitch); };
  // row wave * 64 + p * 8 + (lane >> 3) has its pieces in the order (row >> 1) & 7
  const int put_at = wave * 512 + (lane >> 3) * 8, swz = lane >> 4;
  auto put = [&](int slot, int p) __attribute__((always_inline)) { slots[slot + put_at + p * 64 + ((lane & 7) ^ (swz + (p & 1) * 4))] = st[p]; };
  const int wo = (wave & 1) * 128, wt = (wave >> 1) * 64, n16 = lane & 15, k16 = lane >> 4;
  const int at_w = (wo + n16) * 8 + (k16 ^ (n16 >> 1)), at_x = (N + wt + n16) * 8 + (k16 ^ (n16 >> 1));
  auto read_w = [&](int slot, int j, int f) __attribute__((always_inline)) { return slots[slot + (at_w ^ (4 * j)) + f * 128]; };
  auto read_x = [&](int slot, int j, int f) __attribute__((always_inline)) { return slots[slot + (at_x ^ (4 * j)) + f * 128]; };
  v4i acc[8][4] = {};
  v4i w[3], x[4];
  // A stage in 16 steps, each of which multiplies one of the weights' operands with the four of the tokens': the first three of the weights' are in w, the
  // tokens' in x, a step reads what one three further on takes.  Beside them the next stage's codes go from registers to its slot, which nobody reads any
  // more, and the one's after it are requested.  The only barrier lies before step 14: behind it nobody reads this stage any more, the next one is there, and
  // its first operands are read (8192 tokens of 8192-8192 with their codes: 477 us; with one barrier near the begin and one
  // in the middle 504).
  constexpr int MFMA = 0x008, LOAD = 0x020, READ = 0x100, WRITE = 0x200;
  auto stage = [&](int now, int next, int k) __attribute__((always_inline)) {
    constexpr int move[16] = {0, 1, -1, 2, -1, 3, -1, 4, -1, 5, -1, 6, 7, -1, -1, -1};
    v4i ws[19], xb[4], xn[4];
#pragma unroll
    for (int i = 0; i < 3; ++i) ws[i] = w[i];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (i == 14) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (i < 13) ws[i + 3] = read_w(now, (i + 3) >> 3, (i + 3) & 7);
      if (i < 4) xb[i] = read_x(now, 1, i);
      if (i >= 14) {
        xn[2 * (i - 14)] = read_x(next, 0, 2 * (i - 14));
        xn[2 * (i - 14) + 1] = read_x(next, 0, 2 * (i - 14) + 1);
        ws[i + 2] = read_w(next, 0, i - 14);
        if (i == 15) ws[18] = read_w(next, 0, 2);
      }
      if (move[i] >= 0) {
        put(next, move[i]);
        ask(move[i], k);
      }
#pragma unroll
      for (int g = 0; g < 4; ++g) acc[i & 7][g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(ws[i], i < 8 ? x[g] : xb[g], acc[i & 7][g], 0, 0, 0);
      if (i < 14) {
        __builtin_amdgcn_sched_group_barrier(MFMA, 2, 0);
        if (i < 13) __builtin_amdgcn_sched_group_barrier(READ, 1, 0);
        if (move[i] >= 0) __builtin_amdgcn_sched_group_barrier(WRITE, 1, 0);
        __builtin_amdgcn_sched_group_barrier(MFMA, 2, 0);
        if (i < 4) __builtin_amdgcn_sched_group_barrier(READ, 1, 0);
        if (move[i] >= 0) __builtin_amdgcn_sched_group_barrier(LOAD, 1, 0);
      } else {
        __builtin_amdgcn_sched_group_barrier(READ, 3, 0);
        __builtin_amdgcn_sched_group_barrier(MFMA, 2, 0);
        __builtin_amdgcn_sched_group_barrier(READ, 1, 0);
        __builtin_amdgcn_sched_group_barrier(MFMA, 2, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) w[i] = ws[16 + i];
#pragma unroll
    for (int g = 0; g < 4; ++g) x[g] = xn[g];
  };
  auto meet = [&]() __attribute__((always_inline)) { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
  const int last = a.pitch - KB;
  {      // two stages requested together: the registers of the sums hold nothing yet
    v4i first[P];
#pragma unroll
    for (int p = 0; p < P; ++p) first[p] = src.load(p, 0, a.pitch);
#pragma unroll
    for (int p = 0; p < P; ++p) ask(p, KB);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int p = 0; p < P; ++p) slots[put_at + p * 64 + ((lane & 7) ^ (swz + (p & 1) * 4))] = first[p];
  }
  meet();
#pragma unroll
  for (int i = 0; i < 3; ++i) w[i] = read_w(0, 0, i);
#pragma unroll
  for (int g = 0; g < 4; ++g) x[g] = read_x(0, 0, g);
  // (what the last two stages request is none: one loop, whose sums stay where they are)
  int now = 0;
  if (wt < r.n) {
    for (int k = 0; k <= last; k += KB) {
      stage(now, now ^ SLOT, k + 2 * KB);
      now ^= SLOT;
    }
  } else {      // no token of its own: it only loads, and leaves the matrix unit to the other wave (experts' last tiles)
    for (int k = 0; k <= last; k += KB) {
      now ^= SLOT;
#pragma unroll
      for (int p = 0; p < P; ++p) {
        put(now, p);
        ask(p, k + 2 * KB);
      }
      meet();
    }
  }
  __syncthreads();
  auto& side = *reinterpret_cast<Side<N, N>*>(slots + SLOT);
  side.template load<GATED, 512>(a, r, o0);
  __syncthreads();
  if (wt < r.n) finish<GATED>(a, r, o0, wo, wt, acc, slots + wave * (16 * 32), side);
}

// ------------------------------------------------------------------ launches
enum { AUTOMATIC = 0, STREAM = 1, TILES_64 = 2, TILES_128 = 3, TILES_256 = 4, TILES_FAR = 5 };   // see pipe_set_token_kernel

template <int TB, int S>
int launch_stream_split(const TokenProductArgs& a, bool gated, int o_tiles, int tiles, hipStream_t st) {
  const dim3 grid((unsigned)((tiles + 8 / S - 1) / (8 / S)));
  if (gated) PIPE_KLAUNCH((token_stream_kernel<true, TB, S>), grid, dim3(512), 0, st, a, o_tiles, tiles);
  else PIPE_KLAUNCH((token_stream_kernel<false, TB, S>), grid, dim3(512), 0, st, a, o_tiles, tiles);
  PIPE_HIP(hipGetLastError());
  return PIPE_OK;
}
template <int TB>
int launch_stream(const TokenProductArgs& a, bool gated, hipStream_t st) {
  const int o_tiles = (a.out + 15) / 16;
  const int64_t tiles = (int64_t)o_tiles * row_tiles<16 * TB>(a);
  if (tiles >= (int64_t)1 << 23) return PIPE_ESHAPE;      // (a launch holds fewer than 2^32 threads)
  // as many waves a tile as keep about four a SIMD busy (us with one, two, four, eight waves: 8 tokens of 4096-11008 29, 18, 18, 16; nine, one of 16 experts of
  // 4096-4096, 42, 34, 34, 42; 32, six of 64 gated ones of 2048-1408, 72, 76, 77, 97)
  if (tiles <= 1024) return launch_stream_split<TB, 8>(a, gated, o_tiles, (int)tiles, st);
  if (tiles <= 2048) return launch_stream_split<TB, 4>(a, gated, o_tiles, (int)tiles, st);
  if (tiles <= 4096) return launch_stream_split<TB, 2>(a, gated, o_tiles, (int)tiles, st);
  return launch_stream_split<TB, 1>(a, gated, o_tiles, (int)tiles, st);
}

template <int B, bool FAR = false>
int launch_tiles(const TokenProductArgs& a, bool gated, hipStream_t st) {
  const int width = gated ? B / 2 : B;
  const int64_t o_tiles = (a.out + width - 1) / width, t_tiles = row_tiles<B>(a);
  if (o_tiles * t_tiles > ((int64_t)1 << 23) - 8) return PIPE_ESHAPE;
  const dim3 grid((unsigned)((o_tiles * t_tiles + 7) / 8 * 8));
  if constexpr (B == 256) {
    if (gated) PIPE_KLAUNCH((token_big_kernel<true>), grid, dim3(512), 0, st, a, (int)o_tiles);
    else PIPE_KLAUNCH((token_big_kernel<false>), grid, dim3(512), 0, st, a, (int)o_tiles);
  } else {
    if (gated) PIPE_KLAUNCH((token_tile_kernel<true, B, B == 128 ? 2 : 3, FAR>), grid, dim3(256), 0, st, a, (int)o_tiles);
    else PIPE_KLAUNCH((token_tile_kernel<false, B, B == 128 ? 2 : 3, FAR>), grid, dim3(256), 0, st, a, (int)o_tiles);
  }
  PIPE_HIP(hipGetLastError());
  return PIPE_OK;
}

}  // namespace

// whether a workgroup can make the codes of its tokens itself
static bool one_launch(const TokenProductArgs& a) {
  return a.n * a.pitch <= FUSED_CODES && (int64_t)((a.out + 15) / 16) * row_tiles<16>(a) <= FUSED_TILES;
}
static int kernel_of(const TokenProductArgs& a) {
  const bool gated = a.act == PIPE_ACT_SILU_GATED;
  int which = g_token_kernel;
  const int64_t each = a.n / a.E;       // tokens of an expert, about
  if (which == AUTOMATIC) {
    // Few tokens are streamed past: the weights' bytes are all that counts up to 32 tokens (4096-4096: 13 us, tiles 17; 48 tokens 17 both), longer where
    // that makes few tiles (136 tokens of 4096-704: 13 us, 17; 875 of 3136-128 16 and 19), not where they are many (16 of gated 4096-11008: 24 us, tiles
    // 23; 20 of 4096-32000 42 and 27; 8 of 4096-11008 16 and 17).  Experts' tokens are not spread evenly, a second tile reads the weights again: four each
    // (16 tokens, two of eight experts of 4096-4096: 28 us, tiles 29; 64 tokens: 60 and 30).
    const double w_rows = gated ? 2.0 * a.out : a.out;
    const int64_t streamed = (a.out + 15) / 16 * (each <= 16 ? row_tiles<16>(a) : row_tiles<32>(a));
    if (one_launch(a) || streamed <= 384 || (a.starts ? each <= 4 : a.n <= 32 && w_rows < 16384)) {
      which = STREAM;
    } else {
      // Microseconds of a launch: of a stage of 128 codes with few tiles and for each round of them that the chip holds (1024, 512 and 256; half a tile more
      // for each expert, one at least), and its ends, in stages.  Calls of 64, 128 and 256 tokens a tile: 512 tokens of 4096-4096 26, 35 and 53 us; 1000 42,
      // 40 and 56; 2048 75, 56 and 59; 4096 of 4096-11008 303, 223 and 173; 5227 of 3648-1730 84, 78 and 66; 512 tokens, six of 64 gated experts of
      // 2048-1408 96, 102 and 109; 1024, two of eight of 4096-4096 84, 77 and 60; 8192, two of 128 gated ones of 1024-1024 149, 127 and 146; 2069, two of
      // 110 of 3200-640 54, 80 and 99.  Off where rows are short: 2236 rows of five experts of 192-4096 25, 31 and 29, the rule's are of 128.
      const double stages = a.pitch / 128, n = (double)a.n;
      auto rounds = [&](int B, double held) {
        return std::ceil(w_rows / B) * (a.starts ? a.E * std::max(1.0, n / a.E / B + 0.5) : std::ceil(n / B)) / held;
      };
      const double r64 = rounds(64, 1024), r128 = rounds(128, 512), r256 = rounds(256, 256);
      const double t64 = (r64 <= 1 ? std::max(0.45, r64) : r64 + 0.3) * (stages + 4),
                   t128 = (r128 <= 1 ? std::max(0.95, 1.5 * r128) : 1.5 * r128 + 0.3) * (stages + 4), t256 = std::max(1.55, 1.6 * r256 + 0.1) * (stages + 10);
      which = t64 <= t128 && t64 <= t256 ? TILES_64 : t128 <= t256 ? TILES_128 : TILES_256;
    }
  }
  return near(a) || which == STREAM ? which : TILES_FAR;
}

template <bool GATED>
static int launch_fused(const TokenProductArgs& a, int o_tiles, hipStream_t st) {
  const dim3 grid((unsigned)(o_tiles * row_tiles<16>(a))), block(512);
  if (a.type == PIPE_F32) PIPE_KLAUNCH((token_stream_fused_kernel<GATED, float>), grid, block, 0, st, a, o_tiles);
  else if (a.type == PIPE_F16) PIPE_KLAUNCH((token_stream_fused_kernel<GATED, f16>), grid, block, 0, st, a, o_tiles);
  else PIPE_KLAUNCH((token_stream_fused_kernel<GATED, bf16>), grid, block, 0, st, a, o_tiles);
  PIPE_HIP(hipGetLastError());
  return PIPE_OK;
}

int launch_token_layer(TokenProductArgs& a, int8_t* codes, float* scales, hipStream_t st) {
  const bool gated = a.act == PIPE_ACT_SILU_GATED;
  const int which = kernel_of(a);
  const int n_wide = 16 / type_size(a.type), o_tiles = (a.out + 15) / 16;
  // (every workgroup reads x while others write y: not where these overlap)
  const char *x0 = (const char*)a.x, *y0 = (const char*)a.y;
  const int64_t size = type_size(a.type);
  const bool apart = x0 + ((a.n_x - 1) * a.x_stride + a.in) * size <= y0 || y0 + a.n * a.out * size <= x0;
  if (which == STREAM && apart && one_launch(a)) {
    a.x_wide = (reinterpret_cast<uintptr_t>(a.x) & 15) == 0 && a.x_stride % n_wide == 0;
    return gated ? launch_fused<true>(a, o_tiles, st) : launch_fused<false>(a, o_tiles, st);
  }
  if (codes == nullptr) return PIPE_EINVAL;
  a.qx = codes;
  a.sx = scales;
  const int rc = launch_token_quantize(a.x, a.type, a.n_x, a.in, a.x_stride, a.pitch, codes, scales, st);
  if (rc) return rc;
  const int64_t each = a.n / a.E;
  if (which == TILES_256) return launch_tiles<256>(a, gated, st);
  if (which == TILES_128) return launch_tiles<128>(a, gated, st);
  if (which == TILES_64) return launch_tiles<64>(a, gated, st);
  if (which == TILES_FAR) return launch_tiles<128, true>(a, gated, st);
  return each <= 16 ? launch_stream<1>(a, gated, st) : launch_stream<2>(a, gated, st);
}
