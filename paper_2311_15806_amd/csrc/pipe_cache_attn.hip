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
// Every byte of the cache is read once as long as a tile holds all rows of the head (tokens * G <= 16), and those bytes bound it:
// two requests of 131072 tokens, 8 heads of 128, take 62 us = 4.6 TB/s, 48 of 33 to 8000 tokens 51 us = 4.1 TB/s (a large copy: 4.8).
// To reach that: steps of 32 tokens with two in flight beside the one worked on, the table through scalar loads, a step's words in one
// register spread by DPP (the 131072s 86 us; 64 tokens and one in flight, words and addresses in each lane: 134); equal shares of all
// steps to as many workgroups as the chip holds (67); joined by whichever of a tile's shares ends last (one request of 777 tokens
// 10.8 us; in a second launch 13.3).  One request of 777 tokens is eight trips to memory in a row, 10 us.  fp32 is bound by its instructions: two terms of q
// and of the weights, made for 16 rows a tile whatever is real; 16 requests of 100 to 3000 tokens with 5 rows a tile, 32 heads of 64, take
// 27 us at 2.2 TB/s.  (Every instance keeps 13 to 33 scalar registers in lanes of vector ones.)
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
constexpr int UNIT = WAVES * STEP;                  // tokens of a workgroup's step: one step of every wave
constexpr int SHARES_128 = 512, SHARES_64 = 768;    // workgroups of a launch: as many as the chip holds at once (2 a unit at head_dim 128, 3 at 64)
constexpr size_t ATTN_COUNTS = 4096;                // bytes of the counts of parts
static_assert(SHARES_64 * sizeof(uint32_t) <= ATTN_COUNTS && SHARES_128 <= SHARES_64);
constexpr float REF_SLACK = 6.f;                    // log2: a row's reference rises only when a score exceeds it by this
constexpr float P_SCALE = 256.f;                    // 2^REF_SLACK * 2 * P_SCALE fits fp16
constexpr int K_LOG = 28;                           // a code's sums with q, up to 2^26, and q's, up to 2^22, meet K's scale and offset in units of 2^28: finite
constexpr float S_LEAST = 0x1p-116f;                // least unit of V's scales and offsets
constexpr float OFFSETS = 0x1p-8f;                  // an offset counts as a scale of so much of it: little beside a scale, which is 2^-12 of it or none
// log2 of a weight at the reference: weights times offsets stay well inside fp32's range, tiny ones and those next to its end.  (No more apart than
// that parts of different units are joined without losing a weight.)
__device__ __forceinline__ int level_of(float sigma) { return max(-32, min(16, 8 + 127 - (int)(__float_as_uint(sigma) >> 23))); }

struct Kernel {
  CacheAttnArgs a;
  int G;
  uint32_t n_share; // workgroups of a key/value head
  float load;       // of one of them on a compute unit, for each key/value head
  bool wide;        // 16-byte loads of q
  uint64_t* part_o;     // [Hkv][n_share][2][16 rows][D/32][16]: pairs of outputs
  uint64_t* part_ml;    // [Hkv][n_share][2][16 rows]: log2 of the reference weight, sum of weights
  uint32_t* arrived;    // [Hkv][n_share]: parts written of the tile that begins in the share; zero between calls
};

// The work of a key/value head is the tiles of all requests one after the other, a tile of request b counting the steps of UNIT tokens that
// its cache has.  A workgroup takes one of two kinds of share, whichever `locate` reckons to end first:
//   equal ones of all steps, wherever they begin and end: requests of any lengths keep all workgroups busy to the end.  A tile counts GAP steps
//   more ahead of its own, for the work of beginning it;
//   one tile, or one of the parts of `each` steps that a tile is cut into: no share then ends one tile and begins the next, which is a chain of
//   trips to memory of its own, and a tile in one piece needs no parts joined.
// Of a tile that several shares hold, each writes its part -- of its first tile to place 0, of its last to place 1 -- and whoever comes last
// sums them, in the shares' order.
struct Request {
  int b, start, n;              // its fresh tokens (b = B: the rows behind the last request and, after those, the ones before the first: they see nothing)
  int length, held;             // cached tokens, and those of them that its table has room for
  uint32_t tiles, steps;        // ... each of so many steps
};
__device__ __forceinline__ Request make_request(const Kernel& k, int b, int start, int n, int length) {
  Request r;
  r.b = b; r.start = start; r.n = n; r.length = length;
  r.held = (int)min((int64_t)length, min((int64_t)k.a.width << k.a.cache.shift, (int64_t)0x7ffff000));
  r.tiles = ((uint32_t)n * (uint32_t)k.G + ROWS - 1) / ROWS;
  r.steps = max(1u, ((uint32_t)r.held + UNIT - 1) / UNIT);
  return r;
}
__device__ __forceinline__ Request request(const Kernel& k, int b) {
  const CacheAttnArgs& a = k.a;
  auto start_of = [&](int i) { return min(max(a.starts[i], 0), a.T); };
  const int start = start_of(b), first = start_of(0);
  return make_request(k, b, start, max(0, (b < a.B ? start_of(b + 1) : a.T + min(first, start)) - start), b < a.B ? max(0, a.lengths[b]) : 0);
}
// Where a share begins.  (All steps of a head together are under 2^31: the launch sees to it.)
__device__ __forceinline__ uint32_t share_begin(uint32_t total, uint32_t n_share, uint32_t share) {
  return (uint32_t)((uint64_t)total * share / n_share);
}
// the share that holds a step: the last one that begins at or before it
__device__ __forceinline__ uint32_t share_of(uint32_t total, uint32_t n_share, uint32_t step) {
  return (uint32_t)(((uint64_t)(step + 1) * n_share - 1) / total);
}
struct Place {
  uint32_t total, at;           // steps of the head, and the first of the share, gaps included (`at`: equal shares only),
  uint32_t step, n;             // which is this step; the steps of the share
  uint32_t each;                // steps of a part, no gaps; 0: equal shares
  Request r;                    // of this request
};
template <typename T>
__device__ __forceinline__ T of_lane(T x, int lane) { return (T)__builtin_amdgcn_readlane((int)x, lane); }
// f over the lanes up to each one (the last lane: over all), f(0, x) = x
template <int CTRL, int ROWS_OF_16>
__device__ __forceinline__ uint32_t moved(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS_OF_16, 0xf, false); }
template <typename F>
__device__ __forceinline__ uint32_t wave_scan(uint32_t x, F f) {
  x = f(x, moved<0x111, 0xf>(x));      // from 1, 2, 4 and 8 lanes below within 16
  x = f(x, moved<0x112, 0xf>(x));
  x = f(x, moved<0x114, 0xf>(x));
  x = f(x, moved<0x118, 0xf>(x));
  x = f(x, moved<0x142, 0xa>(x));      // the last lane of the 16 below to every second 16
  return f(x, moved<0x143, 0xc>(x));   // lane 31 to the upper half
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  return wave_scan(x, [](uint32_t a, uint32_t b) { return a + b; });
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  return of_lane(wave_scan(x, [](uint32_t a, uint32_t b) { return max(a, b); }), 63);
}

// What the kinds of shares cost, in steps of a workgroup that has a compute unit to itself (0.7 us): LOAD steps' worth of every unit's time goes
// into each, the more of them at once the slower; JOIN for the trips of parts to memory and back, and a GAP a tile that equal shares begin.  16 requests of 750 tokens, 32 heads of 64 in bf16: whole 12.8 us, in equal shares 21.1; of 3000 tokens, 29 and 34; of 100 to 3000
// in fp32, 31 and 30; 8 heads of 128, 750 tokens: whole 11.2, in parts 13.0; 3000 tokens: 24 and 19.
constexpr int UNITS = 256;
constexpr float LOAD_64 = 0.67f, LOAD_128 = 1.f, JOIN = 4.f;
constexpr uint32_t GAP = 4;      // 48 requests of 33 to 8000 tokens: 54.8 us with 0, 53.6 with 2, 51.8 with 4, 53.0 with 6

// The first place of a share.  Up to 63 requests: every wave for itself, a lane a request.  More: the workgroup together, a thread sums
// every 256th part of them, and the one whose sum holds the place walks them again; those get equal shares only, because the search of one wave
// ends there, not because they were the better ones: 63 and 64 requests of 750 tokens in bf16, 32 heads over 8 of 64, take 12.8 and 15.8 us, of
// 3000 tokens 29.6 and 35.5; 16 heads over one of 128, 13.5 and 15.8, 16.3 and 18.3.
__device__ __forceinline__ Place locate(const Kernel& k, uint32_t share) {
  __shared__ uint32_t s_sum[4], s_step;
  __shared__ int s_b;
  const int B1 = k.a.B + 1, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Place p;
  if (B1 <= 64) {
    const Request r = request(k, min(lane, k.a.B));
    const uint32_t mine = lane < B1 ? r.tiles * r.steps : 0u, inc = wave_scan(mine);
    const uint32_t tiles = lane < B1 ? r.tiles : 0u, inc_t = wave_scan(tiles), all = of_lane(inc_t, 63);
    const uint32_t total = of_lane(inc, 63);
    p.total = total + GAP * all;
    if (k.n_share > 1) {
      const uint32_t longest = wave_max(tiles > 0 ? r.steps : 0u);
      if (all > 0 && all <= k.n_share) {
        // parts of as few steps as will do: of the average of a share, or if that makes too many of them, of so many that it cannot, a tile
        // of s steps having (s + cut - 1) / cut parts at most
        auto parts_of = [&](uint32_t cut) { return (r.steps + cut - 1) / cut; };
        uint32_t cut = (total + k.n_share - 1) / k.n_share;
        const uint32_t spare = k.n_share - all;
        if (of_lane(wave_scan(tiles * parts_of(cut)), 63) > k.n_share) cut = spare > 0 ? min(longest, (total - all + spare - 1) / spare) : longest;
        const float load = k.load;
        const float whole = longest * fmaxf(1.f, all * load);
        const float parts = cut * fmaxf(1.f, min(k.n_share, total / cut + all) * load) + JOIN;
        const float equal = (float)p.total / k.n_share * fmaxf(1.f, k.n_share * load) + JOIN;
        if (fminf(whole, parts) <= equal) {
          p.each = whole <= parts ? longest : cut;
          const uint32_t per = parts_of(p.each), n = tiles * per, inc_p = wave_scan(n);
          const unsigned long long behind = __ballot(inc_p > share);
          const int b = behind ? __builtin_ctzll(behind) : 0;
          p.r = make_request(k, b, of_lane(r.start, b), of_lane(r.n, b), of_lane(r.length, b));
          const uint32_t at = share - of_lane(inc_p - n, b), per_b = of_lane(per, b), cut_at = at % per_b * p.each;
          p.at = 0;
          p.step = at / per_b * p.r.steps + cut_at;
          p.n = behind ? min(p.each, p.r.steps - cut_at) : 0;
          return p;
        }
      }
    }
    p.each = 0;
    p.at = share_begin(p.total, k.n_share, share);
    p.n = share_begin(p.total, k.n_share, share + 1) - p.at;
    const uint32_t inc_w = inc + GAP * inc_t, before_w = inc_w - mine - GAP * tiles;
    const unsigned long long behind = __ballot(inc_w > p.at);
    const int b = behind ? __builtin_ctzll(behind) : 0;
    p.step = p.at - of_lane(before_w, b);
    p.r = make_request(k, b, of_lane(r.start, b), of_lane(r.n, b), of_lane(r.length, b));
    return p;
  }
  const int per = (B1 + 255) / 256;
  const int b0 = min(B1, (int)threadIdx.x * per), b1 = min(B1, b0 + per);
  uint32_t mine = 0;
  for (int b = b0; b < b1; ++b) {
    const Request r = request(k, b);
    mine += r.tiles * (r.steps + GAP);
  }
  const uint32_t inc = wave_scan(mine);
  if (lane == 63) s_sum[wave] = inc;
  if (threadIdx.x == 0) s_b = 0;
  __syncthreads();
  uint32_t before = inc - mine;
  p.total = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    before += w < wave ? s_sum[w] : 0;
    p.total += s_sum[w];
  }
  p.each = 0;
  p.at = share_begin(p.total, k.n_share, share);
  p.n = share_begin(p.total, k.n_share, share + 1) - p.at;
  if (before <= p.at && p.at < before + mine) {
    for (int b = b0; b < b1; ++b) {
      const Request r = request(k, b);
      const uint32_t c = r.tiles * (r.steps + GAP);
      if (p.at < before + c) {
        s_b = b;
        s_step = p.at - before;
        break;
      }
      before += c;
    }
  }
  __syncthreads();
  p.total = __builtin_amdgcn_readfirstlane(p.total);
  p.at = __builtin_amdgcn_readfirstlane(p.at);
  p.n = __builtin_amdgcn_readfirstlane(p.n);
  p.step = __builtin_amdgcn_readfirstlane(s_step);
  p.r = request(k, __builtin_amdgcn_readfirstlane(s_b));
  return p;
}

struct Tile {
  int b, row0, n_rows, start;   // rows row0 .. row0 + n_rows - 1 of request b, whose tokens start at `start`
  int first_seen;               // cached tokens that the request's first fresh token sees (may be negative)
  int end;                      // cached tokens that any row of the tile sees
  __device__ __forceinline__ Tile(const Kernel& k, const Request& r, uint32_t i) : b(r.b), start(r.start) {
    row0 = (int)(i * ROWS);
    n_rows = min(ROWS, r.n * k.G - row0);
    // (the table's width cuts a length short, not the places of the queries)
    first_seen = r.length - r.n + 1;
    end = min(r.held, max(0, first_seen + (row0 + n_rows - 1) / k.G));
  }
};

// its i-th token's row of q and of the output
__device__ __forceinline__ int token_row(const Kernel& k, const Tile& t, int i) {
  const int at = t.start + i;
  return at < k.a.T ? at : at - k.a.T;
}
template <typename T, int D>
__device__ __forceinline__ T* out_row(const Kernel& k, const Tile& t, int kvh, int r) {
  const int row = t.row0 + r;
  return (T*)k.a.out + ((int64_t)token_row(k, t, row / k.G) * k.a.Hq + (int64_t)kvh * k.G + row % k.G) * D;
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
  int b, kvh;
  uint32_t at_k, at_v, at_w;   // a lane's place in a 16-block of codes of K, of V, and of words

  __device__ __forceinline__ Walk(const CacheAttnArgs& a_, int b_, int kvh_, int l16, int kg) : a(a_), b(b_), kvh(kvh_) {
    at_k = l16 * (D / 2) + kg * (D / 8);
    at_v = kg * (2 * D) + l16 * (D / 32);
    at_w = ((NB == 1 ? (l16 >> 2 & 1) * 16 : 0) + kg * 4 + (l16 & 3)) * 4 + (l16 >> 3) * (4u << a_.cache.shift);
  }
  // page entries of the tokens from tok on; -1 from `end` on
  __device__ __forceinline__ void pages_of(int32_t* pages, int tok, int end) const {
    // (scalar loads: among the vector loads, the wait for an entry would be one for all codes in flight)
    const ConstInt* row = (const ConstInt*)(uintptr_t)(a.table + (int64_t)b * a.width);
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

// Two floats to and from memory at the scope of the device: the workgroups of a tile sit behind different L2 caches.
__device__ __forceinline__ void put_pair(uint64_t* p, float x, float y) {
  __hip_atomic_store(p, ((uint64_t)__float_as_uint(y) << 32) | __float_as_uint(x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get_pair(const uint64_t* p) {
  const uint64_t v = __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

// The parts of a tile together, in the shares' order: n_part shares from share p0 on.  Equal shares of `total` steps: the tile begins at t0,
// and empty shares may be among them; total = 0: a part a share.  scratch: 16 * 16 * (D/16 + 1) + 32 floats of LDS.
template <typename T, int D>
__device__ __forceinline__ void join(const Kernel& kr, const Tile& t, int kvh, uint32_t total, uint32_t t0, uint32_t p0, uint32_t n_part, float* scratch) {
  constexpr int MT = D / 16;
  float (*s_y)[16][MT + 1] = reinterpret_cast<float (*)[16][MT + 1]>(scratch);
  float* s_ref = scratch + 16 * 16 * (MT + 1);
  float* s_sum = s_ref + 16;
  // 16 threads have a row; where there are fewer rows than 16, the parts are dealt to several such groups
  const int rows = t.n_rows > 8 ? 16 : t.n_rows > 4 ? 8 : t.n_rows > 2 ? 4 : t.n_rows, groups = 16 / rows;
  const int slot = threadIdx.x >> 4, r = slot % rows, g = slot / rows, dl = threadIdx.x & 15;
  float top = -INFINITY, all = 0.f, y[MT] = {};
  if (r < t.n_rows) {
    constexpr int AT_ONCE = 4;
    for (uint32_t q = g; q < n_part; q += AT_ONCE * groups) {
      float lref[AT_ONCE], sum[AT_ONCE], x[AT_ONCE][MT];
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) {
        const uint32_t p = min(q + u * groups, n_part - 1) + p0;
        const uint32_t b0 = share_begin(total, kr.n_share, p);
        const bool there = q + u * groups < n_part && (total == 0 || b0 < share_begin(total, kr.n_share, p + 1));
        const int64_t at = (((int64_t)kvh * kr.n_share + p) * 2 + (total > 0 && b0 < t0 ? 1 : 0)) * ROWS + r;
        const float2 m = there ? get_pair(kr.part_ml + at) : make_float2(-INFINITY, 0.f);
        lref[u] = m.x;
        sum[u] = m.y;
#pragma unroll
        for (int d = 0; d < MT / 2; ++d) {
          const float2 v = there ? get_pair(kr.part_o + (at * (MT / 2) + d) * 16 + dl) : make_float2(0.f, 0.f);
          x[u][2 * d] = v.x;
          x[u][2 * d + 1] = v.y;
        }
      }
      float high = top;
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) high = fmaxf(high, lref[u]);
      const float f0 = part_weight(top, all, high);
      all *= f0;
#pragma unroll
      for (int d = 0; d < MT; ++d) y[d] *= f0;
      top = high;
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) {
        const float f = part_weight(lref[u], sum[u], high);
        all = fmaf(f, sum[u], all);
#pragma unroll
        for (int d = 0; d < MT; ++d) y[d] = fmaf(f, x[u][d], y[d]);
      }
    }
  }
#pragma unroll
  for (int d = 0; d < MT; ++d) s_y[slot][dl][d] = y[d];
  if (dl == 0) { s_ref[slot] = top; s_sum[slot] = all; }
  __syncthreads();
  if (g == 0 && r < t.n_rows) {
    float high = top;
    for (int i = 1; i < groups; ++i) high = fmaxf(high, s_ref[i * rows + r]);
    float sum = 0.f, z[MT] = {};
    for (int i = 0; i < groups; ++i) {
      const float f = part_weight(s_ref[i * rows + r], s_sum[i * rows + r], high);
      sum = fmaf(f, s_sum[i * rows + r], sum);
#pragma unroll
      for (int d = 0; d < MT; ++d) z[d] = fmaf(f, s_y[i * rows + r][dl][d], z[d]);
    }
    const float inv = high == -INFINITY && sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int d = 0; d < MT; ++d) z[d] = inv == 0.f ? 0.f : z[d] * inv;
    store_row<T, MT>(out_row<T, D>(kr, t, kvh, r) + dl * MT, z);
  }
}

template <typename T, int D, int NB>
__global__ __launch_bounds__(WAVES * 64, D == 64 ? 3 : 2) void cache_attn_kernel(const Kernel kr) {
  constexpr bool FINE = sizeof(T) == 4;                // fp32: centred codes, two terms
  constexpr int KS = D / 32, MT = D / 16, NT = FINE ? 2 : 1;
  __shared__ float s_o[WAVES][ROWS][D + 4];
  __shared__ float s_ref[WAVES][ROWS], s_sum[WAVES][ROWS];
  __shared__ bool s_last;
  const CacheAttnArgs& a = kr.a;
  const uint32_t share = blockIdx.x / a.cache.Hkv;
  const int kvh = blockIdx.x % a.cache.Hkv;
  const Place first = locate(kr, share);
  uint32_t pos = first.at, left = first.n;
  if (left == 0) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, kg = lane >> 4;
  const Bits bits;
  Request rq = first.r;
  const uint32_t gap = first.each > 0 ? 0 : GAP;
  uint32_t tile = first.step / (rq.steps + gap), at = first.step % (rq.steps + gap);

  for (int place = 0;; place = 1) {        // one tile's part after the other
    const uint32_t to = min(rq.steps + gap, at + left), step0 = max(at, gap) - gap, n_steps = max(to, gap) - gap - step0;
    if (n_steps == 0) break;               // (the share ends ahead of the tile's steps)
    const Tile t(kr, rq, tile);
    const Walk<D, NB> w(a, t.b, kvh, l16, kg);

    // q: row l16, the values that meet the words kg * KS .. of a token
    const int row = t.row0 + l16;
    const bool real = l16 < t.n_rows;
    const int token = real ? row / kr.G : 0, head = real ? row % kr.G : 0;
    const int seen = real ? t.first_seen + token : 0x7fffffff;      // cached tokens this row sees (one that is not there: as many as any)
    const T* qp = (const T*)a.q + (int64_t)token_row(kr, t, token) * a.qs.token + (int64_t)(kvh * kr.G + head) * a.qs.head + kg * (KS * 8);
    float qv[KS * 8], qmax = 0, qsum = 0;
    if (kr.wide) {
#pragma unroll
      for (int i = 0; i < KS * 8; i += 8) load8<T, true>(qp + i, qv + i);
    } else {
#pragma unroll
      for (int i = 0; i < KS * 8; i += 8) load8<T, false>(qp + i, qv + i);
    }
    // the first steps' loads fly while q is made ready
    const int end = (int)min((int64_t)t.end, (int64_t)(step0 + n_steps) * UNIT);
    const int full = max(0, t.first_seen + t.row0 / kr.G);   // tokens that every row sees
    int tok = (int)step0 * UNIT + wave * STEP, steps = 0;
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
      w.pages_of(pages, tok + UNIT, end);
      fetch(r1, tok + UNIT);
      w.pages_of(pages, tok + AHEAD * UNIT, end);
    }
#pragma unroll
    for (int i = 0; i < KS * 8; ++i) {
      qv[i] = real ? qv[i] : 0.f;
      qmax = fmaxf(qmax, fabsf(qv[i]));
    }
    qmax = max_over_kg(qmax);
    // a power of two that brings the row's largest value to 2^14 .. 2^15, and with it the sign of the scale
    const int qe = qmax > 0.f && qmax < INFINITY ? 14 - ((int)(__float_as_uint(qmax) >> 23) - 127) : 0;
    // scores are in units of 2^(K_LOG - qe), in which they are finite; rs turns them into log2 of a weight.  rs is finite, and where it would be 0 --
    // all scores are next to nothing then -- the scores are: 0 times an infinity, or a masked score times 0, would be NaN.
    const float rs0 = fminf(ldexpf(fabsf(a.scale) * 0.72134752f, 1 + K_LOG - qe), 0x1.fffffep127f), rs = rs0 > 0.f ? rs0 : 1.f;
    const float sgn = a.scale < 0.f ? -1.f : 1.f;
    h8 q[NT][KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      u4 hi, lo;
#pragma unroll
      for (int n = 0; n < 4; ++n) {                // nibbles n and n + 4 are a register of the operand
        const float x = rs0 == 0.f ? 0.f : sgn * ldexpf(qv[8 * s + n], qe), y = rs0 == 0.f ? 0.f : sgn * ldexpf(qv[8 * s + n + 4], qe);
        qsum += x + y;
        hi[n] = half_pair(x, y);
        lo[n] = half_rest(x, y, hi[n]);
      }
      q[0][s] = __builtin_bit_cast(h8, hi);
      if constexpr (FINE) q[1][s] = __builtin_bit_cast(h8, lo);
    }
    qsum = sum_over_kg(qsum);
    const float word_unit = l16 < 8 ? 1.f / (1 << K_LOG) : 1.f;      // (words of K in lanes l16 < 8, of V in the others)
    const float acc0 = FINE ? 0.f : -64.f * qsum;

    f4 o[MT], ones = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < MT; ++i) o[i] = (f4){0.f, 0.f, 0.f, 0.f};
    // weights are exp2(rs * T + nref), nref = -rs * ref + level_of(sigma), sigma a power of two: all scales of V that the row has seen are under
    // 2 sigma, all offsets under 2 sigma / OFFSETS.  The operand of the second product is a weight times a scale times `lev` = P_SCALE / sigma /
    // 2^level_of(sigma), under 2^15.  (Up to the tokens that every row sees all rows have one sigma.)
    float ref = -INFINITY, nref = 0.f, lift = -INFINITY, sum = 0.f, osum = 0.f, sigma = S_LEAST;
    auto lev_of = [](float sigma) { return ldexpf(P_SCALE / sigma, -level_of(sigma)); };
    float lev = lev_of(S_LEAST);

    // one step on `c`, while the next ones' loads fly, AHEAD steps on to `n`
    auto step = [&](const Tokens<D>& c, Tokens<D>& n) {
      // (behind the end they read page 0, which the caches hold: behind a branch, the wait for this step's would wait for all)
      fetch(n, tok + AHEAD * UNIT);
      w.pages_of(pages, tok + (AHEAD + 1) * UNIT, end);
      // scores
      float s[2][4];
      float ws = word_scale(c.w) * word_unit, wo = word_offset(c.w) * word_unit, wm = fmaf(8.f, ws, wo);      // scale, offset, and the offset of c - 8
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
        wo = live ? wo : 0.f;
        wm = live ? wm : 0.f;
      }
      float smax = s[0][0];
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) smax = fmaxf(smax, s[j][i]);
      // V's scales and offsets: of a token in each lane, or of the tokens that this row sees where the rows differ
      const float v_size = fmaf(fabsf(wo), OFFSETS, fabsf(ws));
      float vs = l16 < 8 ? 0.f : v_size;
      if (some) {
        vs = 0.f;
        each<8>([&](auto B) {
          constexpr int bit = B;
          const float g = from_lane<8 + bit>(v_size);
          vs = fmaxf(vs, (vis >> bit) & 1u ? g : 0.f);
        });
      }
      if (__any(smax > lift || vs > 2.f * sigma)) {
        const float nr = fmaxf(ref, max_over_kg(smax));
        float top = max_over_kg(vs);
        if (!some) {
#pragma unroll
          for (int d = 1; d < 16; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
        }
        const float nsigma = fmaxf(sigma, __uint_as_float(__float_as_uint(top) & 0x7f800000u));
        const float f = ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(rs * (ref - nr)), fo = f * (sigma / nsigma);
        const int down = level_of(nsigma) - level_of(sigma);
        sum = ldexpf(sum * f, down);
        osum = ldexpf(osum * f, down);
#pragma unroll
        for (int i = 0; i < MT; ++i) o[i] *= fo;
        ones *= fo;
        ref = nr;
        sigma = nsigma;
        lev = lev_of(nsigma);
        nref = (nr == -INFINITY ? 0.f : -nr * rs) + level_of(nsigma);
        lift = nr == -INFINITY ? -INFINITY : nr + REF_SLACK / rs;
      }
      // weights times V's scales: one fp16 value for outputs of 16 bits (2^-12 of each, at random, less than such an output's own rounding), two
      // for fp32; their sums take them unrounded
      if (!some) ws *= lev;
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
                y[u] = e * (yes ? g * lev : 0.f);
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
      tok += UNIT;
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
    const float lref = ref == -INFINITY ? -INFINITY : -nref, unit = ldexpf(sigma / P_SCALE, level_of(sigma));
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        float y = o[i][j];
        if constexpr (!FINE) y = fmaf(-72.f, ones[j], y);
        s_o[wave][l16][MT * (4 * kg + j) + i] = fmaf(y, unit, osum);
      }
    if (kg == 0) { s_ref[wave][l16] = lref; s_sum[wave][l16] = sum; }
    __syncthreads();
    // the waves' parts together: a thread has D/16 values of a row
    const int r = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * MT;
    if (r < t.n_rows) {
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
      if (n_steps == rq.steps) {
        const float inv = top == -INFINITY && all == 0.f ? 0.f : 1.f / all;
#pragma unroll
        for (int d = 0; d < MT; ++d) y[d] = inv == 0.f ? 0.f : y[d] * inv;
        store_row<T, MT>(out_row<T, D>(kr, t, kvh, r) + d0, y);
      } else {
        const int64_t at = (((int64_t)kvh * kr.n_share + share) * 2 + place) * ROWS + r;
#pragma unroll
        for (int d = 0; d < MT / 2; ++d) put_pair(kr.part_o + (at * (MT / 2) + d) * 16 + (threadIdx.x & 15), y[2 * d], y[2 * d + 1]);
        if (d0 == 0) put_pair(kr.part_ml + at, top, all);
      }
    }
    if (n_steps != rq.steps) {
      // Every wave's stores have reached the device's scope before the count says so.
      const uint32_t t0 = pos - at, t1 = t0 + gap + rq.steps;
      const bool cut = first.each > 0;
      const uint32_t p0 = cut ? share - step0 / first.each : share_of(first.total, kr.n_share, t0 + gap);
      const uint32_t n_part = cut ? (rq.steps + first.each - 1) / first.each : share_of(first.total, kr.n_share, t1 - 1) - p0 + 1;
      __builtin_amdgcn_s_waitcnt(0x0F70);    // vmcnt(0)
      __syncthreads();
      // (equal shares, fewer steps than them: as many parts as the tile has steps)
      uint32_t* count = kr.arrived + kvh * kr.n_share + p0;
      if (threadIdx.x == 0) s_last = atomicAdd(count, 1u) == (!cut && first.total < kr.n_share ? rq.steps : n_part) - 1;
      __syncthreads();
      if (s_last) {
        join<T, D>(kr, t, kvh, cut ? 0 : first.total, t0, p0, n_part, &s_o[0][0][0]);
        if (threadIdx.x == 0) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
    }
    pos += to - at;
    left -= to - at;
    if (left == 0) break;
    __syncthreads();                         // (the next part's outputs come to the same places)
    at = 0;
    if (++tile >= rq.tiles) {
      tile = 0;
      do rq = request(kr, rq.b + 1);         // (steps are left: there is a request)
      while (rq.tiles == 0);
    }
  }
}

template <typename T, int D>
int run(const Kernel& k, hipStream_t st) {
  const dim3 grid((unsigned)k.n_share * (unsigned)k.a.cache.Hkv);
  if (k.a.cache.shift >= 5) PIPE_KLAUNCH((cache_attn_kernel<T, D, 1>), grid, dim3(WAVES * 64), 0, st, k);
  else PIPE_KLAUNCH((cache_attn_kernel<T, D, 2>), grid, dim3(WAVES * 64), 0, st, k);
  PIPE_HIP(hipGetLastError());
  return PIPE_OK;
}

}  // namespace

int launch_cache_attention(const CacheAttnArgs& a, hipStream_t st) {
  if (a.T == 0) return PIPE_OK;
  Kernel k{};
  k.a = a;
  k.G = a.Hq / a.cache.Hkv;
  k.wide = rows_wide(a.q, a.qs, a.type);
  // No more shares than there are steps, as far as the longest request is known; tiles of up to 3 steps stay whole (300 tokens: 9.8 us a
  // call whole, 11.0 in parts; 777 tokens 12.5 and 11.1).
  const int64_t longest = a.max_length > 0 ? a.max_length : (int64_t)a.width << a.cache.shift;
  const int64_t tiles = ((int64_t)a.T * k.G + std::min<int64_t>((int64_t)a.B + 1, a.T) * (ROWS - 1)) / ROWS;      // at most: those of a request round up
  const int64_t most = (a.D == 64 ? SHARES_64 : SHARES_128) / a.cache.Hkv;
  const int64_t room = std::min<int64_t>((int64_t)a.width << a.cache.shift, 0x7ffff000);
  if ((((int64_t)a.T * k.G + ROWS - 1) / ROWS + a.B + 1) * (room / UNIT + 1 + GAP) > 0x7fffffff) return PIPE_ESHAPE;
  k.n_share = (uint32_t)std::max<int64_t>(1, std::min(most, tiles * (longest <= 3 * UNIT ? 1 : (longest + UNIT - 1) / UNIT)));
  k.load = (a.D == 64 ? LOAD_64 : LOAD_128) * a.cache.Hkv / UNITS;
  if (k.n_share > 1 || pipe_dry_run()) {
    const size_t parts = (size_t)SHARES_64 * 2 * ROWS;       // one size serves every call
    int rc = PIPE_OK;
    uint8_t* ws = (uint8_t*)pipe_ws_zeroed(WS_ATTN, ATTN_COUNTS + parts * (128 + 2) * sizeof(float), ATTN_COUNTS, &rc);
    if (!ws) return rc;
    k.arrived = (uint32_t*)ws;
    k.part_ml = (uint64_t*)(ws + ATTN_COUNTS);
    k.part_o = k.part_ml + parts;
  }
  if (a.type == PIPE_F32) return a.D == 64 ? run<float, 64>(k, st) : run<float, 128>(k, st);
  if (a.type == PIPE_F16) return a.D == 64 ? run<f16, 64>(k, st) : run<f16, 128>(k, st);
  return a.D == 64 ? run<bf16, 64>(k, st) : run<bf16, 128>(k, st);
}
