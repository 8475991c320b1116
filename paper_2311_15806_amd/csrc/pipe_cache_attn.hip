// Attention of fresh tokens over the 4-bit cache.
//
// For one key/value head of one request, the rows are its fresh tokens' query heads (row = token * G + head in the group), 16 of
// them a workgroup's tile; a wave walks 32 cached tokens at a time:
//   T[t][r] = s_t * (sum_d c_td q_rd) + m_t * (sum_d q_rd)          one MFMA tile per 16 tokens, codes as the A operand
//   P[t][r] = exp2(rs_r * (T - ref_r))                               ref_r: a row's running reference
//   O[d][r] += sum_t c'_td * (P * s'_t)                              codes of V as the A operand, P as the B operand
//   M[r]   += sum_t P * m'_t,  L[r] += sum_t P
// with T's accumulator layout (lane = row, 4 tokens in a lane's registers) being exactly the B operand's of the second product, once
// the tokens of a step are taken in the order 4*kg..+3 of one 16-block, then of the next: no shuffle between the products.
//
// Codes become fp16 without conversions: four bits at bit 4 of a half under the exponent of 64 are 64 + c; 7 instructions make
// 8 operand values.  The 64 is taken out of the sums again: from the scores by the accumulator's start, -64 sum q, from the
// outputs with one more product whose A operand is all ones, O = sum P' (64 + c) - 72 sum P'.  (Without the exponent the bits are
// the denormal c * 2^-24, two instructions less, but the sums then lose what lies 10 bits deeper: 2.5 times the error.)
// fp32 takes the codes as c - 8, subtracted in fp16 (exact), and q and P in two terms.
// The offsets' part of the output is P (m + 8 s), with m about -8 s: no large sums that cancel.
//
// Bound by the bytes of the codes as long as a tile holds all rows of the head: see the figures at the launch rules.
#include <algorithm>
#include <type_traits>

#include "pipe_attention.h"

namespace {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

#define GLOBAL __attribute__((address_space(1)))
typedef const GLOBAL uint8_t* GlobalBytes;
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(4))) int32_t ConstInt;   // memory that the kernel does not write

constexpr int WAVES = 4, ROWS = 16, STEP = 32;      // tokens of a wave's step
constexpr int AHEAD = 2;                            // steps whose loads are in flight while one is worked on
constexpr int CHUNK_UNIT = WAVES * STEP;            // a split's tokens are a multiple of this: every wave gets whole steps
constexpr int SPLIT_TILES = 768;
constexpr float REF_SLACK = 6.f;                    // log2: a row's reference rises only when a score exceeds it by this
constexpr float P_SCALE = 256.f;                    // 2^REF_SLACK * 2 * P_SCALE fits fp16

struct Kernel {
  CacheAttnArgs a;
  int G, n_split, chunk;
  bool wide;        // 16-byte loads of q
  float* part_o;    // [Hkv][T * G rows][split][D]
  float* part_ml;   // [Hkv][T * G rows][split][2]: log2 of the reference weight, sum of weights
};

struct Tile {
  int b, row0, n_rows, start;   // rows row0 .. row0 + n_rows - 1 of request b, whose tokens start at `start`
  int first_seen;               // cached tokens that the request's first fresh token sees (may be negative)
  int end;                      // cached tokens that any row of the tile sees
  int n_split, chunk;           // splits that have tokens (at least one), and theirs
};

// Tile `id` of the launch: request b (B: the rows behind the last request, which see nothing) owns the ids from
// floor(start_b * G / 16) + b on.
__device__ __forceinline__ Tile find_tile(const Kernel& k, int id) {
  const CacheAttnArgs& a = k.a;
  const int lane = threadIdx.x & 63;
  auto start_of = [&](int b) { return b > 0 ? min(max(a.starts[b], 0), a.T) : 0; };
  int b = -1;
  for (int i0 = 0; i0 <= a.B; i0 += 64) {
    const int i = i0 + lane;
    const bool le = i <= a.B && (int)(((int64_t)start_of(min(i, a.B)) * k.G) / ROWS) + i <= id;
    const int n = __popcll(__ballot(le));
    b += n;
    if (n < 64) break;
  }
  b = __builtin_amdgcn_readfirstlane(b);
  Tile t;
  t.b = b;
  t.start = start_of(b);
  const int n = (b < a.B ? start_of(b + 1) : a.T) - t.start;
  t.row0 = (id - ((int)(((int64_t)t.start * k.G) / ROWS) + b)) * ROWS;
  t.n_rows = t.row0 < 0 ? 0 : min(ROWS, max(0, n * k.G - t.row0));
  const int length = b < a.B ? max(0, a.lengths[b]) : 0;
  t.first_seen = length - n + 1;
  const int last_row = t.row0 + max(t.n_rows, 1) - 1;
  const int64_t table = (int64_t)a.width << a.cache.shift;
  t.end = (int)min((int64_t)max(0, t.first_seen + last_row / k.G), min(table, (int64_t)0x7ffff000));
  // (a request longer than the hint gets longer splits)
  const int per = (int)(((int64_t)t.end + k.n_split - 1) / k.n_split);
  t.chunk = max(k.chunk, (per + CHUNK_UNIT - 1) / CHUNK_UNIT * CHUNK_UNIT);
  t.n_split = max(1, (t.end + t.chunk - 1) / t.chunk);
  return t;
}

// the parts of row r of a tile, of the head of this workgroup
__device__ __forceinline__ int64_t part_row(const Kernel& k, const Tile& t, int r) {
  return ((int64_t)blockIdx.y * k.a.T * k.G + (int64_t)t.start * k.G + t.row0 + r) * k.n_split;
}

// what a part counts, beside the largest reference: nothing if it saw nothing (and NaN if it saw nothing but NaN)
__device__ __forceinline__ float part_weight(float lref, float sum, float top) {
  return lref == -INFINITY ? sum : __builtin_amdgcn_exp2f(lref - top);
}

// 8 codes of a word -> 4 registers of two fp16 values, nibbles (0,4) (1,5) (2,6) (3,7)
struct Bits {
  uint32_t mask, c64;   // in registers: with both as literals a code would take an `and` and an `or`, with neither one and_or
  __device__ __forceinline__ Bits() : mask(0x00f000f0u), c64(0x54005400u) { asm("" : "+v"(mask), "+v"(c64)); }
};
template <bool CENTRED>
__device__ __forceinline__ void expand(uint32_t x, const Bits& bits, uint32_t* o) {
  auto half = [&](uint32_t w) {   // nibble at bit 4: 64 + c, or less 72
    const uint32_t u = (w & bits.mask) | bits.c64;
    if constexpr (!CENTRED) return u;
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2, u) - (h2){(_Float16)72.f, (_Float16)72.f});
  };
  o[0] = half(x << 4); o[1] = half(x); o[2] = half(x >> 4); o[3] = half(x >> 8);
}

// Two values rounded to fp16, and what is left of them rounded likewise.  The first rounding is done once: the single and the packed
// conversion break ties differently, and a rest taken from the other's result is off by a unit.
__device__ __forceinline__ uint32_t half_pair(float x, float y) {
  uint32_t u = __builtin_bit_cast(uint32_t, (h2){(_Float16)x, (_Float16)y});
  asm volatile("" : "+v"(u));
  return u;
}
__device__ __forceinline__ uint32_t half_rest(float x, float y, uint32_t u) {
  const h2 v = __builtin_bit_cast(h2, u);
  return __builtin_bit_cast(uint32_t, (h2){(_Float16)(x - (float)v[0]), (_Float16)(y - (float)v[1])});
}

__device__ __forceinline__ float max_over_kg(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float sum_over_kg(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// A step's tokens.  NB page lookups serve them: 1 where a page holds 32 tokens or more, else one for every 16-block.
template <int NB>
struct Places {
  const uint8_t* blk[NB];   // the head's block of the page (any page where there is none)
  uint32_t off[NB];         // first token in it
  uint32_t there;           // lookups whose page exists
};
// The codes and words of a step's tokens, as a lane (l16, kg) holds them.
template <int D>
struct Tokens {
  uint32_t k[2][D / 32];    // [16-block]: of token l16 the D/32 words from kg * D/32 on
  uint32_t v[2][4];         // [16-block]: of token 4 kg + i the D/16 codes from l16 * D/16 on
  uint32_t w;               // the word of token 4 kg + l16 % 4 of 16-block l16 / 4 % 2: of K in lanes l16 < 8, of V in the others
  uint32_t there;           // lookups whose page exists
};
// what lane 4 j + i of a row of 16 lanes holds: the word of this lane's i-th token of 16-block j (folded into the operation that uses it)
template <int LANE>
__device__ __forceinline__ float from_lane(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x150 + LANE, 0xf, 0xf, true));
}
template <int N, typename F>
__device__ __forceinline__ void each(F&& f) {      // f(0) .. f(N - 1), with constants
  if constexpr (N > 1) each<N - 1>(f);
  f(std::integral_constant<int, N - 1>{});
}

template <int D, int NB>
struct Walk {
  const CacheAttnArgs& a;
  const Tile& t;
  int kvh;
  uint32_t at_k, at_v, at_w;   // a lane's place in a 16-block of codes of K, of V, and of words

  __device__ __forceinline__ Walk(const CacheAttnArgs& a_, const Tile& t_, int kvh_, int l16, int kg) : a(a_), t(t_), kvh(kvh_) {
    at_k = l16 * (D / 2) + kg * (D / 8);
    at_v = kg * (2 * D) + l16 * (D / 32);
    at_w = ((NB == 1 ? (l16 >> 2 & 1) * 16 : 0) + kg * 4 + (l16 & 3)) * 4 + (l16 >> 3) * (4u << a_.cache.shift);
  }
  // page entries of the tokens from tok on; -1 from `end` on
  __device__ __forceinline__ void pages_of(int32_t* pages, int tok, int end) const {
    // (scalar loads: among the vector loads, the wait for an entry would be one for all codes in flight)
    const ConstInt* row = (const ConstInt*)(uintptr_t)(a.table + (int64_t)t.b * a.width);
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int at = __builtin_amdgcn_readfirstlane(tok + 16 * j);
      pages[j] = at < end ? row[at >> a.cache.shift] : -1;
    }
  }
  __device__ __forceinline__ void find(Places<NB>& x, const int32_t* pages, int tok) const {
    const uint32_t P = 1u << a.cache.shift;
    const uint64_t block = (uint64_t)P * (D + 8), stride = block * (uint32_t)a.cache.Hkv;
    const uint8_t* head = a.cache.base + block * (uint32_t)kvh;
    x.there = 0;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const uint32_t page = (uint32_t)__builtin_amdgcn_readfirstlane(pages[j]);
      const bool there = page < (uint32_t)a.cache.n_pages;
      x.there |= there ? 1u << j : 0u;
      x.blk[j] = head + stride * (there ? page : 0u);
      x.off[j] = (uint32_t)(tok + 16 * j) & (P - 1);
    }
  }
  // kept whole in scalar registers: a load then needs one register of offset, not two of address that it has to add up first
  __device__ __forceinline__ static GlobalBytes base(const uint8_t* p) {
    GlobalBytes g = (GlobalBytes)(uintptr_t)p;
    asm("" : "+s"(g));
    return g;
  }
  __device__ __forceinline__ void load(Tokens<D>& x, const Places<NB>& p) const {
    const uint32_t P = 1u << a.cache.shift;
    uint32_t at_k = this->at_k, at_v = this->at_v, at_w = this->at_w;
    asm("" : "+v"(at_k), "+v"(at_v), "+v"(at_w));   // (32 bits here, not widened ahead of the loop)
    constexpr int INNER = NB == 1 ? 16 : 0;
    x.there = p.there;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int n = NB == 1 ? 0 : j;
      const GlobalBytes kp = base(p.blk[n] + p.off[n] * (D / 2)) + j * INNER * (D / 2);
      if constexpr (D == 128) {
        const u4 w = *(const GLOBAL u4*)(kp + at_k);
#pragma unroll
        for (int i = 0; i < 4; ++i) x.k[j][i] = w[i];
      } else {
        const u2 w = *(const GLOBAL u2*)(kp + at_k);
        x.k[j][0] = w.x; x.k[j][1] = w.y;
      }
    }
    GlobalBytes wp = base(p.blk[0] + P * D + p.off[0] * 4);
    if constexpr (NB == 2) {
      const GlobalBytes wq = base(p.blk[1] + P * D + p.off[1] * 4);
      wp = (threadIdx.x & 4) ? wq : wp;
    }
    x.w = *(const GLOBAL uint32_t*)(wp + at_w);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int n = NB == 1 ? 0 : j;
      const GlobalBytes vp = base(p.blk[n] + P * (D / 2) + p.off[n] * (D / 2)) + j * INNER * (D / 2);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (D == 128) x.v[j][i] = *(const GLOBAL uint32_t*)(vp + i * (D / 2) + at_v);
        else x.v[j][i] = *(const GLOBAL uint16_t*)(vp + i * (D / 2) + at_v);
      }
    }
  }
};

template <typename T, int D, int NB>
__global__ __launch_bounds__(WAVES * 64, 2) void cache_attn_kernel(const Kernel kr) {
  constexpr bool FINE = sizeof(T) == 4;                // fp32: centred codes, two terms
  constexpr int KS = D / 32, MT = D / 16, NT = FINE ? 2 : 1;
  __shared__ float s_o[WAVES][ROWS][D + 4];
  __shared__ float s_ref[WAVES][ROWS], s_sum[WAVES][ROWS];
  const CacheAttnArgs& a = kr.a;
  const Tile t = find_tile(kr, blockIdx.x);
  const int split = blockIdx.z;
  if (t.n_rows == 0 || split >= t.n_split) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, kg = lane >> 4;
  const Walk<D, NB> w(a, t, blockIdx.y, l16, kg);
  const Bits bits;

  // q: row l16, the values that meet the words kg * KS .. of a token
  const int row = t.row0 + l16;
  const bool real = l16 < t.n_rows;
  const int token = real ? row / kr.G : 0, head = real ? row % kr.G : 0;
  const int seen = real ? t.first_seen + token : 0;      // cached tokens this row sees
  const T* qp = (const T*)a.q + (int64_t)(t.start + token) * a.qs.token + (int64_t)(w.kvh * kr.G + head) * a.qs.head + kg * (KS * 8);
  float qv[KS * 8], qmax = 0, qsum = 0;
  if (kr.wide) {
#pragma unroll
    for (int i = 0; i < KS * 8; i += 8) load8<T, true>(qp + i, qv + i);
  } else {
#pragma unroll
    for (int i = 0; i < KS * 8; i += 8) load8<T, false>(qp + i, qv + i);
  }
#pragma unroll
  for (int i = 0; i < KS * 8; ++i) {
    qv[i] = real ? qv[i] : 0.f;
    qmax = fmaxf(qmax, fabsf(qv[i]));
  }
  qmax = max_over_kg(qmax);
  // a power of two that brings the row's largest value to 2^14 .. 2^15, and with it the sign of the scale
  const int qe = qmax > 0.f && qmax < INFINITY ? max(-80, min(100, 14 - ((int)(__float_as_uint(qmax) >> 23) - 127))) : 0;
  const float sgn = a.scale < 0.f ? -1.f : 1.f;
  h8 q[NT][KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    u4 hi, lo;
#pragma unroll
    for (int n = 0; n < 4; ++n) {                // nibbles n and n + 4 are a register of the operand
      const float x = a.scale == 0.f ? 0.f : sgn * ldexpf(qv[8 * s + n], qe), y = a.scale == 0.f ? 0.f : sgn * ldexpf(qv[8 * s + n + 4], qe);
      qsum += x + y;
      hi[n] = half_pair(x, y);
      lo[n] = half_rest(x, y, hi[n]);
    }
    q[0][s] = __builtin_bit_cast(h8, hi);
    if constexpr (FINE) q[1][s] = __builtin_bit_cast(h8, lo);
  }
  qsum = sum_over_kg(qsum);
  // scores in units of q * 2^qe; rs turns them into log2 of a weight
  const float rs = a.scale == 0.f ? 1.f : ldexpf(fabsf(a.scale) * 1.44269504f, -qe);
  const float acc0 = FINE ? 0.f : -64.f * qsum;

  f4 o[MT], ones = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < MT; ++i) o[i] = (f4){0.f, 0.f, 0.f, 0.f};
  // weights are exp2(rs * T + nref), nref = -rs * ref + log2(P_SCALE / sigma) with sigma a power of two, all scales of V under 2 sigma
  float ref = -INFINITY, nref = 0.f, lift = -INFINITY, sum = 0.f, osum = 0.f, sigma = 0x1p-100f;

  const int end = (int)min((int64_t)t.end, (int64_t)(split + 1) * t.chunk);
  const int full = max(0, t.first_seen + t.row0 / kr.G);   // tokens that every row sees
  int tok = split * t.chunk + wave * STEP, steps = 0;
  int32_t pages[NB];
  Tokens<D> r0, r1, r2;      // AHEAD + 1 of them, in turn
  auto fetch = [&](Tokens<D>& x, int from) {
    Places<NB> at;
    w.find(at, pages, from);
    w.load(x, at);
  };
  w.pages_of(pages, tok, end);
  if (tok < end) {
    fetch(r0, tok);
    w.pages_of(pages, tok + CHUNK_UNIT, end);
    fetch(r1, tok + CHUNK_UNIT);
    w.pages_of(pages, tok + AHEAD * CHUNK_UNIT, end);
  }
  // one step on `c`, while the next ones' loads fly, AHEAD steps on to `n`
  auto step = [&](const Tokens<D>& c, Tokens<D>& n) {
    // (behind the end they read page 0, which the caches hold: behind a branch, the wait for this step's would wait for all)
    fetch(n, tok + AHEAD * CHUNK_UNIT);
    w.pages_of(pages, tok + (AHEAD + 1) * CHUNK_UNIT, end);
    // scores
    float s[2][4];
    float ws = word_scale(c.w), wo = word_offset(c.w), wm = fmaf(8.f, ws, wo);      // scale, offset, and the offset of c - 8
    const float ko = FINE ? wm : wo;
    each<2>([&](auto J) {
      constexpr int j = J;
      f4 acc = {acc0, acc0, acc0, acc0};
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        uint32_t e[4];
        expand<FINE>(c.k[j][i], bits, e);
        const h8 op = __builtin_bit_cast(h8, (u4){e[0], e[1], e[2], e[3]});
#pragma unroll
        for (int m = 0; m < NT; ++m) acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(op, q[m][i], acc, 0, 0, 0);
      }
      each<4>([&](auto I) {
        constexpr int i = I;
        s[j][i] = fmaf(from_lane<4 * j + i>(ws), acc[i], from_lane<4 * j + i>(ko) * qsum);
      });
    });
    uint32_t vis = 0xffu;                                             // tokens that this row sees, bit 4 j + i
    const bool some = tok + STEP > full || tok + STEP > end || c.there != (1u << NB) - 1;      // some row does not see some token
    if (some) {
      const int lim = min(seen, end) - tok - 4 * kg;
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool yes = 16 * j + i < lim && ((c.there >> (NB == 1 ? 0 : j)) & 1u);
          s[j][i] = yes ? s[j][i] : -INFINITY;
          vis &= yes ? ~0u : ~(1u << (4 * j + i));
        }
      // words that nobody sees may hold anything
      const int j = l16 >> 2 & 1;
      const bool live = tok + 16 * j + 4 * kg + (l16 & 3) < end && ((c.there >> (NB == 1 ? 0 : j)) & 1u);
      ws = live ? ws : 0.f;
      wm = live ? wm : 0.f;
    }
    float smax = s[0][0];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) smax = fmaxf(smax, s[j][i]);
    const float vs = l16 < 8 ? 0.f : fabsf(ws);
    if (__any(smax > lift || vs > 2.f * sigma)) {
      const float nr = fmaxf(ref, max_over_kg(smax));
      float top = vs;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
      const float nsigma = fmaxf(sigma, __uint_as_float(__float_as_uint(top) & 0x7f800000u));
      const float f = (ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(rs * (ref - nr))) * (sigma / nsigma);
      sum *= f;
      osum *= f;
#pragma unroll
      for (int i = 0; i < MT; ++i) o[i] *= f;
      ones *= f;
      ref = nr;
      sigma = nsigma;
      nref = (nr == -INFINITY ? 0.f : -nr * rs) + __builtin_amdgcn_logf(P_SCALE / nsigma);
      lift = nr == -INFINITY ? -INFINITY : nr + REF_SLACK / rs;
    }
    // weights
    u4 p[NT];
    auto weights = [&](auto SOME) {
      each<2>([&](auto J) {
        each<2>([&](auto H) {
          constexpr int j = J, i = 2 * H;
          float y[2];
          each<2>([&](auto U) {
            constexpr int u = U, bit = 4 * j + i + u, lane_of = 8 + bit;
            const float e = __builtin_amdgcn_exp2f(fmaf(s[j][i + u], rs, nref));
            sum += e;
            if constexpr (SOME) {
              const bool yes = (vis >> bit) & 1u;
              const float m = from_lane<lane_of>(wm), g = from_lane<lane_of>(ws);
              osum = fmaf(e, yes ? m : 0.f, osum);
              y[u] = e * (yes ? g : 0.f);
            } else {
              osum = fmaf(from_lane<lane_of>(wm), e, osum);
              y[u] = from_lane<lane_of>(ws) * e;
            }
          });
          const uint32_t u = half_pair(y[0], y[1]);
          p[0][j * 2 + (i >> 1)] = u;
          if constexpr (FINE) p[1][j * 2 + (i >> 1)] = half_rest(y[0], y[1], u);
        });
      });
    };
    if (some) weights(std::true_type{});
    else weights(std::false_type{});
    if constexpr (!FINE) {
      // the 72s of the sums so far come out now and then: over thousands of tokens of equal weight they would cost fp32 its last digits
      if ((++steps & 7) == 0) {
#pragma unroll
        for (int i = 0; i < MT; ++i) o[i] = o[i] - 72.f * ones;
        ones = (f4){0.f, 0.f, 0.f, 0.f};
      }
    }
    // outputs
    constexpr int NH = D / 64;       // halves of a V word: 4 codes each
    uint32_t e[NH][4][4];            // [half][pair of tokens][nibble]
#pragma unroll
    for (int u = 0; u < 4; ++u) {    // tokens (0,1) (2,3) of one block, then of the other
      const uint32_t x0 = c.v[u >> 1][2 * (u & 1)], x1 = c.v[u >> 1][2 * (u & 1) + 1];
      expand<FINE>(__builtin_amdgcn_perm(x1, x0, 0x05040100u), bits, e[0][u]);
      if constexpr (NH == 2) expand<FINE>(__builtin_amdgcn_perm(x1, x0, 0x07060302u), bits, e[1][u]);
    }
#pragma unroll
    for (int m = 0; m < NT; ++m) {
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const int hf = i >> 2, nb = i & 3;
        const h8 op = __builtin_bit_cast(h8, (u4){e[hf][0][nb], e[hf][1][nb], e[hf][2][nb], e[hf][3][nb]});
        o[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(op, __builtin_bit_cast(h8, p[m]), o[i], 0, 0, 0);
      }
    }
    if constexpr (!FINE) {
      const h8 one = {1, 1, 1, 1, 1, 1, 1, 1};
      ones = __builtin_amdgcn_mfma_f32_16x16x32_f16(one, __builtin_bit_cast(h8, p[0]), ones, 0, 0, 0);
    }
    tok += CHUNK_UNIT;
  };
  while (tok < end) {
    step(r0, r2);
    if (tok >= end) break;
    step(r1, r0);
    if (tok >= end) break;
    step(r2, r1);
  }

  // a wave's outputs as they are, O[d][row] at d = MT * (4 kg + j) + i, over the reference weight
  sum = sum_over_kg(sum);
  osum = sum_over_kg(osum);
  const float lref = ref == -INFINITY ? -INFINITY : -nref;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      float y = o[i][j] + osum;
      if constexpr (!FINE) y = fmaf(-72.f, ones[j], y);
      s_o[wave][l16][MT * (4 * kg + j) + i] = y;
    }
  if (kg == 0) { s_ref[wave][l16] = lref; s_sum[wave][l16] = sum; }
  __syncthreads();
  // the waves' parts together: a thread has D/16 values of a row
  const int r = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * MT;
  if (r >= t.n_rows) return;
  float top = s_ref[0][r];
#pragma unroll
  for (int i = 1; i < WAVES; ++i) top = fmaxf(top, s_ref[i][r]);
  float y[MT] = {}, all = 0.f;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) {
    const float f = part_weight(s_ref[i][r], s_sum[i][r], top);
    all = fmaf(f, s_sum[i][r], all);
#pragma unroll
    for (int d = 0; d < MT; ++d) y[d] = fmaf(f, s_o[i][r][d0 + d], y[d]);
  }
  if (t.n_split == 1) {
    const float inv = top == -INFINITY && all == 0.f ? 0.f : 1.f / all;
    const int rr = t.row0 + r;
    T* out = (T*)a.out + ((int64_t)(t.start + rr / kr.G) * a.Hq + w.kvh * kr.G + rr % kr.G) * D + d0;
#pragma unroll
    for (int d = 0; d < MT; ++d) y[d] = inv == 0.f ? 0.f : y[d] * inv;
    store_row<T, MT>(out, y);
  } else {
    const int64_t at = part_row(kr, t, r) + split;
    store_row<float, MT>(kr.part_o + at * D + d0, y);
    if (d0 == 0) { kr.part_ml[at * 2] = top; kr.part_ml[at * 2 + 1] = all; }
  }
}

// The splits' parts of a tile together, in their order.
template <typename T, int D>
__global__ __launch_bounds__(256) void cache_attn_join_kernel(const Kernel kr) {
  constexpr int MT = D / 16;
  const CacheAttnArgs& a = kr.a;
  const Tile t = find_tile(kr, blockIdx.x);
  const int r = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * MT;
  if (r >= t.n_rows || t.n_split == 1) return;
  const int64_t at = part_row(kr, t, r);
  float top = -INFINITY;
  for (int s = 0; s < t.n_split; ++s) top = fmaxf(top, kr.part_ml[(at + s) * 2]);
  float y[MT] = {}, all = 0.f;
  for (int s = 0; s < t.n_split; ++s) {
    const int64_t i = at + s;
    const float lref = kr.part_ml[i * 2], sum = kr.part_ml[i * 2 + 1];
    const float f = part_weight(lref, sum, top);
    all = fmaf(f, sum, all);
#pragma unroll
    for (int d = 0; d < MT; ++d) y[d] = fmaf(f, kr.part_o[i * D + d0 + d], y[d]);
  }
  const float inv = top == -INFINITY && all == 0.f ? 0.f : 1.f / all;
  const int rr = t.row0 + r;
  T* out = (T*)a.out + ((int64_t)(t.start + rr / kr.G) * a.Hq + (int64_t)blockIdx.y * kr.G + rr % kr.G) * D + d0;
#pragma unroll
  for (int d = 0; d < MT; ++d) y[d] = inv == 0.f ? 0.f : y[d] * inv;
  store_row<T, MT>(out, y);
}

template <typename T, int D>
int run(Kernel& k, int tiles, hipStream_t st) {
  const dim3 grid(tiles, k.a.cache.Hkv, k.n_split);
  if (k.a.cache.shift >= 5) PIPE_KLAUNCH((cache_attn_kernel<T, D, 1>), grid, dim3(WAVES * 64), 0, st, k);
  else PIPE_KLAUNCH((cache_attn_kernel<T, D, 2>), grid, dim3(WAVES * 64), 0, st, k);
  PIPE_HIP(hipGetLastError());
  if (k.n_split > 1) {
    PIPE_KLAUNCH((cache_attn_join_kernel<T, D>), dim3(tiles, k.a.cache.Hkv), dim3(256), 0, st, k);
    PIPE_HIP(hipGetLastError());
  }
  return PIPE_OK;
}

}  // namespace

int launch_cache_attention(const CacheAttnArgs& a, hipStream_t st) {
  if (a.T == 0) return PIPE_OK;
  Kernel k{};
  k.a = a;
  k.G = a.Hq / a.cache.Hkv;
  k.wide = rows_wide(a.q, a.qs, a.type);
  const int64_t rows = (int64_t)a.T * k.G, tiles = rows / ROWS + a.B + 1;
  if (tiles > 0x3fffff) return PIPE_ESHAPE;
  const int64_t longest = std::min<int64_t>(a.max_length > 0 ? a.max_length : (int64_t)a.width << a.cache.shift, 1 << 30);
  // Splits: as many as bring the launch to SPLIT_TILES workgroups, each with 256 tokens at least.
  const int64_t base = std::max<int64_t>((rows + ROWS - 1) / ROWS, std::min(a.B, a.T)) * a.cache.Hkv;
  k.n_split = (int)std::max<int64_t>(1, std::min<int64_t>(SPLIT_TILES / base, (longest + CHUNK_UNIT - 1) / CHUNK_UNIT));
  k.chunk = (int)round_up64((longest + k.n_split - 1) / k.n_split, CHUNK_UNIT);
  if (k.n_split > 1) {
    // (T * Hq * n_split <= ROWS * SPLIT_TILES: one size serves every call)
    const size_t parts = (size_t)ROWS * SPLIT_TILES;
    k.part_o = (float*)pipe_ws_get(WS_ATTN, parts * (128 + 2) * sizeof(float));
    if (!k.part_o) return pipe_ws_error();
    k.part_ml = k.part_o + parts * 128;
  }
  if (a.type == PIPE_F32) return a.D == 64 ? run<float, 64>(k, (int)tiles, st) : run<float, 128>(k, (int)tiles, st);
  if (a.type == PIPE_F16) return a.D == 64 ? run<f16, 64>(k, (int)tiles, st) : run<f16, 128>(k, (int)tiles, st);
  return a.D == 64 ? run<bf16, 64>(k, (int)tiles, st) : run<bf16, 128>(k, (int)tiles, st);
}
