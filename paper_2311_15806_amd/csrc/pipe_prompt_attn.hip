// Attention over packed sequences: out = softmax(scale q K^T) V in one pass over the keys, with a running reference and sum a row.
//
// The rows of a key/value head of a sequence are its queries' heads (row = query * G + head in the group), so that every tile of keys
// serves the whole group.  A workgroup has 128 rows, 32 a wave, and walks its keys 64 at a time (fp32: 32):
//   S^T[key][row] = K q^T,  P = exp2(scale log2(e) (S - ref)),  O^T[d][row] += V^T P^T
// Both products are taken transposed: a lane then holds scores of one row only, maxima and sums need one exchange between two lanes, and the
// scores' accumulator layout is, up to the order of the keys, that of the second product's operand: weights never go through LDS.
//
// The floor is the products', 4 D operations a pair of query and key that sees it: 8192 tokens, 32 heads over 8 of 128, in bf16 take
// 0.53 to 0.55 ms = 1000 to 1035 TFLOP/s, where a matrix product of 8192^3 reaches 1182.  At that size the matrix units and the LDS reads
// are busy half of the time each and the softmax's instructions 45 %, between two waves a SIMD.  Seven packed prompts of 228 to 2500 tokens
// take 0.2 ms, 730 to 750 TFLOP/s, about 98 steps of 64 keys (2.05 us each) one after the other at every place of the chip: 69 are the pairs that
// are seen, 4 the causal edges of tiles, 15 the beginnings of tiles (3 steps each, of 15 on average), 10 an end that is not even.
// fp32, 4096 tokens, 32 heads over 8 of 128: 0.54 ms, 253 TFLOP/s counted once, three products each (at head_dim 128 150 registers a lane are
// spilled); 97 tokens 12 us, one workgroup's four tiles of keys in a row, where keys are not split between waves.
// The tallest tiles are launched first, so that the short ones fill the end; workgroups that follow each other have different heads of the
// same rows, which keeps the heads' keys in one XCD each where Hkv is 8.
#include <type_traits>

#include "pipe_attention.h"

namespace {

// ------------------------------------------------------------------ 16-bit types
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));

constexpr int WAVES = 4, WROWS = 32, QROWS = WAVES * WROWS, KEYS = 64;
constexpr float REF_SLACK = 8.f;   // log2: a row's reference rises only when a score exceeds it by this

__device__ __forceinline__ f16v mfma(u4 x, u4 y, f16v c, f16) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, x), __builtin_bit_cast(h8, y), c, 0, 0, 0);
}
__device__ __forceinline__ f16v mfma(u4 x, u4 y, f16v c, bf16) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, x), __builtin_bit_cast(b8, y), c, 0, 0, 0);
}
template <typename T>
__device__ __forceinline__ uint32_t pack(float x, float y) {      // (as a vector: one conversion for both)
  typedef T T2 __attribute__((ext_vector_type(2)));
  typedef float f2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2){x, y}, T2));
}

// Order of N products that read READS times each from LDS: the reads AHEAD of the products that wait for them.
template <int N, int READS, int AHEAD>
__device__ __forceinline__ void in_turn() {
  constexpr int DS_READ = 0x100, MFMA = 0x8, FIRST = AHEAD / READS;
  __builtin_amdgcn_sched_group_barrier(DS_READ, AHEAD, 0);
#pragma unroll
  for (int i = 0; i < N - FIRST; ++i) {
    __builtin_amdgcn_sched_group_barrier(MFMA, 1, 0);
    __builtin_amdgcn_sched_group_barrier(DS_READ, READS, 0);
  }
  __builtin_amdgcn_sched_group_barrier(MFMA, FIRST, 0);
}

struct Kernel {
  PromptAttnArgs a;
  int G, n_tiles;
  bool wide;       // 16-byte loads of q, k and v
};

struct Tile {
  int row0, n_rows, start;    // rows row0 .. of a sequence whose queries start at `start`; row = query * G + head in the group
  int k0, nk;                 // its keys
  int first_seen;             // keys that its first query sees (causal; may be negative)
  int none;                   // queries that see nothing ahead of them: the rows before the first sequence are counted to it
};

// Tile `id` of the launch: sequence b (B: the rows behind the last one, which see nothing) owns the ids from
// floor(start_b * G / QROWS) + b on.
__device__ __forceinline__ Tile find_tile(const Kernel& k, int place) {
  const PromptAttnArgs& a = k.a;
  const int id = k.n_tiles - 1 - place;       // (long tiles first: the last queries see most)
  const int lane = threadIdx.x & 63;
  const int none = min(max(a.q_starts[0], 0), a.Tq);
  auto start_of = [&](int i) { return i > 0 ? min(max(a.q_starts[min(i, a.B)], 0), a.Tq) : 0; };
  auto key_of = [&](int i) { return min(max(a.k_starts[min(i, a.B)], 0), a.Tk); };
  auto first_id = [&](int start, int i) { return (int)(((int64_t)start * k.G) / QROWS) + i; };
  int b, start, next, k0, k1;      // the sequence, its queries and its keys
  if (a.B < 64) {                  // a lane a sequence: nothing is looked up twice
    const int s = start_of(lane), key = key_of(lane);
    b = __popcll(__ballot(lane <= a.B && first_id(s, lane) <= id)) - 1;
    start = __builtin_amdgcn_readlane(s, b);
    next = b < a.B ? __builtin_amdgcn_readlane(s, b + 1 < 64 ? b + 1 : 63) : a.Tq;
    k0 = __builtin_amdgcn_readlane(key, b);
    k1 = b < a.B ? __builtin_amdgcn_readlane(key, b + 1 < 64 ? b + 1 : 63) : k0;
  } else {
    b = -1;
    for (int i0 = 0; i0 <= a.B; i0 += 64) {
      const int i = i0 + lane;
      const int n = __popcll(__ballot(i <= a.B && first_id(start_of(i), i) <= id));
      b += n;
      if (n < 64) break;
    }
    b = __builtin_amdgcn_readfirstlane(b);
    start = start_of(b);
    next = b < a.B ? start_of(b + 1) : a.Tq;
    k0 = key_of(b);
    k1 = b < a.B ? key_of(b + 1) : k0;
  }
  const int n = next - start;
  Tile t;
  t.start = start;
  t.row0 = (id - first_id(start, b)) * QROWS;
  t.n_rows = t.row0 < 0 ? 0 : min(QROWS, max(0, n * k.G - t.row0));
  t.k0 = k0;
  t.nk = max(0, k1 - k0);
  t.first_seen = t.nk - n + 1;
  t.none = b > 0 ? 0 : none;
  return t;
}

// A lane's row, and what its wave and its workgroup see.
template <typename T>
struct Row {
  bool real;
  const T* q;
  T* out;
  int seen;                   // keys this row sees
  int end, full;              // keys any row of the workgroup sees, and keys that all of them see
  int wave_end, wave_full;    // keys any row of the wave sees, and keys that all of them see
  __device__ __forceinline__ Row(const Kernel& k, const Tile& t, int wave, int n, int kvh) {
    const PromptAttnArgs& a = k.a;
    const int lrow = wave * WROWS + n;
    real = lrow < t.n_rows;
    const int row = t.row0 + (real ? lrow : 0);
    const int token = row / k.G, head = kvh * k.G + row % k.G;
    auto seen_by = [&](int query) { return query < t.none ? 0 : a.causal ? max(0, min(t.nk, t.first_seen + query)) : t.nk; };
    seen = real ? seen_by(token) : 0;
    q = (const T*)a.q + (int64_t)(t.start + token) * a.qs.token + (int64_t)head * a.qs.head;
    out = (T*)a.out + ((int64_t)(t.start + token) * a.Hq + head) * a.D;
    end = seen_by((t.row0 + t.n_rows - 1) / k.G);
    full = seen_by(t.row0 / k.G);
    const int rows = min(WROWS, t.n_rows - wave * WROWS);
    wave_end = rows > 0 ? seen_by((t.row0 + wave * WROWS + rows - 1) / k.G) : 0;
    wave_full = rows > 0 ? seen_by((t.row0 + wave * WROWS) / k.G) : 0;
  }
};

// Where chunk c (8 values) of key row r lies in its LDS row, as a chunk: the rows that one read of 16 lanes touches (16 rows' same chunk of K;
// 4 rows' 4 chunks of V) then lie in different banks.
template <int D>
__device__ __forceinline__ int swizzle(int r, int c) {
  if constexpr (D == 128) return c ^ (((r & 3) << 2) | ((r >> 2) & 3));
  return c ^ (((r & 2) << 1) | ((r >> 2) & 3));
}

template <typename T, int D, bool WIDE>
__global__ __launch_bounds__(WAVES * 64, 2) void prompt_mfma_kernel(const Kernel kr) {
  constexpr int CH = D / 8, KS = D / 16, DB = D / 32;    // chunks of a row, steps of the score product, blocks of the output's
  constexpr int LOADS = KEYS * CH / 256;                 // 16-byte loads a lane makes of a tile of K (and of V)
  // one array per slot: the compiler tells loads into one from reads of another by the array
  __shared__ alignas(1024) u4 k_a[KEYS * CH], k_b[KEYS * CH], v_a[KEYS * CH], v_b[KEYS * CH];
  const PromptAttnArgs& a = kr.a;
  const int id = blockIdx.x, kvh = id % a.Hkv;
  const Tile t = find_tile(kr, id / a.Hkv);
  if (t.n_rows == 0) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, h = lane >> 5;

  const Row<T> w(kr, t, wave, n, kvh);
  // ---- loads of a tile: LDS in the order of the lanes, so that a lane picks what belongs at its place
  auto fetch = [&](const void* src, const HeadStrides& st, u4* dst, int key0) {
    const T* base = (const T*)src + (int64_t)(t.k0 + key0) * st.token + (int64_t)kvh * st.head;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int at = (i * WAVES + wave) * 64 + lane, r = at / CH, c = swizzle<D>(r, at % CH);
      const int rr = min(r, t.nk - 1 - key0);              // (rows behind the last key: the last key again, which nobody sees there)
      if constexpr (WIDE) {
        const uint32_t off = (uint32_t)rr * (uint32_t)st.token * (uint32_t)sizeof(T) + c * 16;
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)((const char*)base + off),
                                         (__attribute__((address_space(3))) void*)(dst + (i * WAVES + wave) * 64), 16, 0, 0);
      } else {
        T v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = base[(int64_t)rr * st.token + c * 8 + e];
        u4 x;
        __builtin_memcpy(&x, v, 16);
        dst[at] = x;
      }
    }
  };

  auto first_tile = [&]() {
    if (w.end > 0) {
      fetch(a.k, a.ks, k_a, 0);
      fetch(a.v, a.vs, v_a, 0);
    }
  };
  first_tile();
  const T* qp = w.q + 8 * h;
  u4 q[KS];
  const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u, keep = w.real && a.scale != 0.f ? ~0u : 0u;
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    if constexpr (WIDE) {
      q[s] = *reinterpret_cast<const u4*>(qp + 16 * s);
    } else {
      T v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = qp[16 * s + i];
      __builtin_memcpy(&q[s], v, 16);
    }
  }
#pragma unroll
  for (int s = 0; s < KS; ++s)
#pragma unroll
    for (int i = 0; i < 4; ++i) q[s][i] = (q[s][i] ^ flip) & keep;
  // log2 of a weight per unit of a score
  const float rs = a.scale == 0.f ? 1.f : fminf(fabsf(a.scale) * 1.44269504f, 0x1.fffffep127f);    // (finite: 0 times it is 0)

  f16v o[DB];
  float ref, nref, lift, sum;
  bool careful = false;       // a second pass: some output of the first is not finite
  // log2 of a weight at the reference.  fp16: weights up to 2^15, so that small ones keep their digits.  bf16 has fp32's range, and sums over
  // values next to the end of it do not: weights up to 2^-24 in the second pass, for sums over 2^24 keys.
  auto p_log = [&]() { return std::is_same_v<T, f16> ? 7.f : careful ? -32.f : 0.f; };

  // Places in a tile, in bytes: of K the chunk h of row n -- chunk 2 j + h of row 32 b + n is j and b further, by an exclusive or and an
  // addition --, of V the piece that this lane brings to a transposed read: of every 16 lanes, lane i brings 4 columns from 4 (i % 4) on
  // of row i / 4, and gets column i of the 4 rows.
  const int vr = 4 * h + ((lane >> 2) & 3), vc = ((lane >> 4) & 1) * 2 + ((lane >> 1) & 1);
  int k_at = (n * CH + swizzle<D>(n, h)) * 16, v_at = (vr * CH + swizzle<D>(vr, vc)) * 16 + (lane & 1) * 8;
  // MASKED: some row may not see some key of the tile
  auto step = [&](auto MASKED, const u4* ks, const u4* vs, u4* kn, u4* vn, int key0) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");     // this tile is there, and the other slot free
    if (key0 + KEYS < w.end) {
      fetch(a.k, a.ks, kn, key0 + KEYS);
      fetch(a.v, a.vs, vn, key0 + KEYS);
    }
    if (MASKED && key0 >= w.wave_end) return;
    asm volatile("" : "+v"(k_at), "+v"(v_at));        // (the places are made here, not kept in 40 registers)
    __builtin_amdgcn_s_setprio(1);                    // (the products before the other waves' softmax)
    // scores, keys in the rows: lane (row n, h) holds keys 32 b + 8 (i / 4) + 4 h + i % 4
    f16v s[2];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
#pragma unroll
    for (int j = 0; j < KS; ++j)
#pragma unroll
      for (int b = 0; b < 2; ++b)
        s[b] = mfma(*reinterpret_cast<const u4*>(reinterpret_cast<const char*>(ks) + (k_at ^ (j << 5)) + b * 32 * CH * 16), q[j], s[b], T());
    in_turn<2 * KS, 1, 6>();
    __builtin_amdgcn_s_setprio(0);
    const bool some = MASKED && key0 + KEYS > w.wave_full;
    if (some) {
      const int lim = w.seen - key0 - 4 * h;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[b][i] = 32 * b + 8 * (i >> 2) + (i & 3) < lim ? s[b][i] : -INFINITY;
    }
    float smax = s[0][0];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) smax = fmaxf(smax, s[b][i]);
    if (__any(smax > lift)) {
      const float nr = fmaxf(ref, fmaxf(smax, __shfl_xor(smax, 32)));
      const float f = ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(rs * (ref - nr));
      sum *= f;
#pragma unroll
      for (int d = 0; d < DB; ++d) o[d] *= f;
      ref = nr;
      nref = p_log() - (nr == -INFINITY ? 0.f : nr * rs);
      lift = nr == -INFINITY ? -INFINITY : nr + REF_SLACK / rs;
    }
    // (weights are rounded to the inputs' type, the only one that the matrix unit multiplies with V's: 2^-12 or 2^-9 of each, at random; their
    // sum takes them unrounded)
    u4 p[2][2];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const float e0 = __builtin_amdgcn_exp2f(fmaf(s[b][i], rs, nref)), e1 = __builtin_amdgcn_exp2f(fmaf(s[b][i + 1], rs, nref));
        sum += e0 + e1;
        p[b][i >> 3][(i >> 1) & 3] = pack<T>(e0, e1);
      }
    asm volatile("" : "+v"(sum));                     // (summed here: 32 weights would live on into the next step)
    // V's operand: its column d = 32 e + n, keys 16 g + 8 u + 4 h + 0..3, read transposed
    auto column = [&](int g, int u, int e) {
      const char* at = reinterpret_cast<const char*>(vs) + (v_at ^ (e << 6) ^ (u << 5)) + (16 * g + 8 * u) * CH * 16;
      return __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)at));
    };
    if constexpr (MASKED) if (some && careful) {
      uint32_t big = 0;
#pragma unroll 1
      for (int g = 0; g < KEYS / 16; ++g)
#pragma unroll
        for (int e = 0; e < DB; ++e)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const u2 y = column(g, u, e);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const uint32_t x = y[i] & 0x7fff7fffu;
              big = max(big, max(x & 0xffffu, x >> 16));
            }
          }
      constexpr uint32_t INF_BITS = std::is_same_v<T, f16> ? 0x7c00u : 0x7f80u;
      if (__any(big >= INF_BITS)) {
        // such a tile is summed key by key, each row over the keys that it sees
#pragma unroll 1
        for (int k = 0; k < KEYS; ++k) {
          uint32_t pw = 0;
#pragma unroll
          for (int i = 0; i < 16; ++i) pw = (k & 31) / 8 * 2 + ((k & 31) % 4) / 2 + 8 * (k >> 5) == i ? p[i >> 3][(i >> 2) & 1][i & 3] : pw;
          pw = __shfl(pw, n + 32 * ((k >> 2) & 1));
          const uint16_t bits = (uint16_t)((k & 1) ? pw >> 16 : pw);
          const float pk = to_f(__builtin_bit_cast(T, bits));
          const bool yes = key0 + k < w.seen;
          const T* row_at = reinterpret_cast<const T*>(vs) + k * D;
#pragma unroll
          for (int e = 0; e < DB; ++e)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int d = 32 * e + 8 * (i >> 2) + 4 * h + (i & 3);
              const float v = to_f(row_at[swizzle<D>(k, d >> 3) * 8 + (d & 7)]);
              o[e][i] = yes ? fmaf(pk, v, o[e][i]) : o[e][i];
            }
        }
        return;
      }
    }
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int g = 0; g < KEYS / 16; ++g)
#pragma unroll
      for (int e = 0; e < DB; ++e) {
        const u2 x = column(g, 0, e), y = column(g, 1, e);
        o[e] = mfma((u4){x[0], x[1], y[0], y[1]}, p[g >> 1][g & 1], o[e], T());
      }
    in_turn<KEYS / 16 * DB, 2, 8>();
  };

  for (;;) {
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    ref = lift = -INFINITY;
    nref = sum = 0.f;
    int key0 = 0;
    for (; key0 + 2 * KEYS <= w.full; key0 += 2 * KEYS) {
      step(std::false_type{}, k_a, v_a, k_b, v_b, key0);
      step(std::false_type{}, k_b, v_b, k_a, v_a, key0 + KEYS);
    }
    for (; key0 < w.end; key0 += 2 * KEYS) {
      step(std::true_type{}, k_a, v_a, k_b, v_b, key0);
      if (key0 + KEYS >= w.end) break;
      step(std::true_type{}, k_b, v_b, k_a, v_a, key0 + KEYS);
    }
    // A row that does not see a key gives it the weight 0, and 0 times an infinity or a NaN of V would still reach it: where an output is
    // not finite, all is done once more, with care for such tiles (and in bf16 with smaller weights).
    if (careful) break;
    bool bad = false;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) bad |= !(fabsf(o[d][i]) < INFINITY);
    if (!__syncthreads_or(bad && w.seen > 0)) break;       // (a row that sees nothing gives zeros whatever it summed)
    careful = true;
    first_tile();
  }
  sum += __shfl_xor(sum, 32);
  const float inv = ref == -INFINITY && sum == 0.f ? 0.f : 1.f / sum;
  // 4 values of this lane's columns 8 g + 4 h and 4 of lane ^ 32's make 16 bytes: even groups go to the lower lanes, odd ones to the upper
#pragma unroll
  for (int e = 0; e < DB; ++e)
#pragma unroll
    for (int g = 0; g < 4; g += 2) {
      u4 y;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        auto value = [&](int j) { return inv == 0.f ? 0.f : o[e][j] * inv; };
        const uint32_t x = pack<T>(value(4 * g + 2 * i), value(4 * g + 2 * i + 1));
        const uint32_t x2 = pack<T>(value(4 * g + 4 + 2 * i), value(4 * g + 4 + 2 * i + 1));
        const auto z = __builtin_amdgcn_permlane32_swap(x, x2, false, false);
        y[i] = z[0];
        y[2 + i] = z[1];
      }
      if (w.real) *reinterpret_cast<u4*>(w.out + 32 * e + 8 * (g + h)) = y;
    }
}

// ------------------------------------------------------------------ fp32
// fp32 goes through the fp16 matrix instruction as two terms, x = 2^-e (hi + lo) with hi = fp16(2^e x) and lo = fp16(2^e x - hi): 22 bits of
// every value down to 2^-17 of the largest one of its row, for which e is chosen, and a b = hi hi + hi lo + lo hi, what is left out being
// 2^-22 of it.  Three instructions of 32 cycles for what the fp32 instruction does in 512: 4096 tokens of 32 heads 1.15 ms there, 0.54 here.  A key's
// factor of K goes back into its scores, that of V into its weight.  A tile of 32 keys is loaded one ahead into registers and split on its
// way into LDS, once for all waves.

// the exponent field of 2^e, for e that brings `largest` (finite, >= 0) to 2^14 .. 2^15
__device__ __forceinline__ int scale_of(float largest, int most = 253) { return min(most, 268 - (int)(__float_as_uint(largest) >> 23)); }
__device__ __forceinline__ float power_of(int scale) { return __uint_as_float((uint32_t)scale << 23); }

// f x and f y in two terms of fp16 each; the rest is taken from the rounded value itself, whichever way that fell.
__device__ __forceinline__ void two_terms(float x, float y, float f, uint32_t& hi, uint32_t& lo) {
  h2 a = {(f16)__builtin_fmaf(x, f, 0.f), (f16)__builtin_fmaf(y, f, 0.f)};
  hi = __builtin_bit_cast(uint32_t, a);
  asm volatile("" : "+v"(hi));
  a = __builtin_bit_cast(h2, hi);
  const h2 b = {(f16)__builtin_fmaf(x, f, -(float)a[0]), (f16)__builtin_fmaf(y, f, -(float)a[1])};
  lo = __builtin_bit_cast(uint32_t, b);
}
// the largest finite magnitude of 8 values
__device__ __forceinline__ float largest8(const float* x) {
  float m = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = __builtin_amdgcn_fmed3f(fabsf(x[e]), m, 0x1.fffffep127f);   // (NaN leaves m)
  if (__any(m == 0x1.fffffep127f)) {                    // an infinity, most likely: once more without
    m = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(x[e]) < INFINITY ? fabsf(x[e]) : 0.f);
  }
  return m;
}

template <int D, bool WIDE>
__global__ __launch_bounds__(WAVES * 64, 2) void prompt_f32_kernel(const Kernel kr) {
  constexpr int CH = D / 8, KS = D / 16, DB = D / 32, KEYS32 = 32;
  constexpr int LOADS = KEYS32 * CH / 256;               // chunks of 8 values a lane brings of a tile of K (and of V)
  __shared__ alignas(1024) u4 k_hi[KEYS32 * CH], k_lo[KEYS32 * CH], v_hi[KEYS32 * CH], v_lo[KEYS32 * CH];
  __shared__ u4 q_rest[D == 128 ? WAVES * KS * 64 : 1];      // the second terms of q, where registers do not hold them too
  __shared__ alignas(16) float k_unit[KEYS32], v_unit[KEYS32];     // what a key's scaled values are multiples of
  const PromptAttnArgs& a = kr.a;
  const int id = blockIdx.x, kvh = id % a.Hkv;
  const Tile t = find_tile(kr, id / a.Hkv);
  if (t.n_rows == 0) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, h = lane >> 5;
  const Row<float> w(kr, t, wave, n, kvh);

  float kx[LOADS][8], vx[LOADS][8];
  auto fetch = [&](int key0) {
    const float* kb = (const float*)a.k + (int64_t)(t.k0 + key0) * a.ks.token + (int64_t)kvh * a.ks.head;
    const float* vb = (const float*)a.v + (int64_t)(t.k0 + key0) * a.vs.token + (int64_t)kvh * a.vs.head;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int at = i * 256 + threadIdx.x, r = min(at / CH, t.nk - 1 - key0), c = at % CH;   // (rows behind the last key: the last key again)
      load8<float, WIDE>(kb + (int64_t)r * a.ks.token + c * 8, kx[i]);
      load8<float, WIDE>(vb + (int64_t)r * a.vs.token + c * 8, vx[i]);
    }
  };
  if (w.end > 0) fetch(0);

  // q: row n, in two terms
  float qv[KS][8], qmax = 0.f;
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    load8<float, WIDE>(w.q + 16 * s + 8 * h, qv[s]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      qv[s][i] = w.real && a.scale != 0.f ? qv[s][i] : 0.f;
      qmax = fmaxf(qmax, fabsf(qv[s][i]));
    }
  }
  qmax = fmaxf(qmax, __shfl_xor(qmax, 32));
  const int qe = qmax < INFINITY ? scale_of(qmax) : 127;
  // Scores are kept in multiples of 2^K_SHIFT: the sums of up to 2^37 times the unit of a key of up to 2^113 are finite then.  (Keys under 2^-88
  // are held to multiples of 2^-126.)
  constexpr int K_SHIFT = 24;
  // log2 of a weight per unit of a score, 2^(K_SHIFT - e) * |scale| * log2(e).  It is finite, and where it would be 0 -- all scores are next to nothing
  // then -- the scores are: 0 times an infinity, or a masked score times 0, would be NaN.
  const float rs0 = fminf(ldexpf(fabsf(a.scale) * 0.72134752f, 128 + K_SHIFT - qe), 0x1.fffffep127f), rs = rs0 > 0.f ? rs0 : 1.f;
  const float qf = rs0 > 0.f ? copysignf(power_of(qe), a.scale) : 0.f;
  u4 q_hi[KS], q_lo[D == 128 ? 1 : KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    u4 rest;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t hi, lo;
      two_terms(qv[s][2 * i], qv[s][2 * i + 1], qf, hi, lo);
      q_hi[s][i] = hi;
      rest[i] = lo;
    }
    if constexpr (D == 128) q_rest[(wave * KS + s) * 64 + lane] = rest;      // (read by this lane alone)
    else q_lo[s] = rest;
  }

  f16v o[DB];
  // weights exp2(rs * score + nref), outputs in units of sigma / P_SCALE: sigma a power of two, no unit of a key that this row sees above U_SLACK of it
  float ref, nref, lift, sum, sigma, per;
  bool careful = false;            // a second pass: some output of the first is not finite
  const int vr = 4 * h + ((lane >> 2) & 3), vc = ((lane >> 4) & 1) * 2 + ((lane >> 1) & 1);      // (places as in the 16-bit kernel)
  int k_at = (n * CH + swizzle<D>(n, h)) * 16, v_at = (vr * CH + swizzle<D>(vr, vc)) * 16 + (lane & 1) * 8;
  constexpr float U_SLACK = 8.f, P_SCALE = 16.f;        // 2^REF_SLACK * U_SLACK * P_SCALE fits fp16
  constexpr float U_LEAST = 0x1p-120f;                  // sigma at first: P_SCALE over it is finite, whatever V's units (of zeros: 2^-126)

  auto step = [&](auto MASKED, int key0) {
    // ---- the loaded tile's terms into LDS, once every wave is done with the tile before
    __syncthreads();
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int at = i * 256 + threadIdx.x, r = at / CH, c = at % CH, to = r * CH + swizzle<D>(r, c);
      const float km = largest8(kx[i]), vm = largest8(vx[i]);
      const int ke = scale_of(row_reduce<CH, true>(km), 253 - K_SHIFT), ve = scale_of(row_reduce<CH, true>(vm));
      if (c == 0) { k_unit[r] = power_of(254 - K_SHIFT - ke); v_unit[r] = power_of(254 - ve); }
      const float kf = power_of(ke), vf = power_of(ve);
      u4 kh, kl, vh, vl;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        uint32_t hi, lo;
        two_terms(kx[i][2 * e], kx[i][2 * e + 1], kf, hi, lo);
        kh[e] = hi; kl[e] = lo;
        two_terms(vx[i][2 * e], vx[i][2 * e + 1], vf, hi, lo);
        vh[e] = hi; vl[e] = lo;
      }
      if constexpr (MASKED) if (careful) {
        // an infinity of K becomes the second term, which only q's first one meets: the others would add infinities of either sign, or NaN
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t half = 0xffffu << 16 * (e & 1), x = kh[e >> 1] & half;
          const bool inf = (x & 0x7fff7fffu) == (0x7c007c00u & half);
          kl[e >> 1] = inf ? (kl[e >> 1] & ~half) | x : kl[e >> 1];
          kh[e >> 1] = inf ? kh[e >> 1] & ~half : kh[e >> 1];
        }
      }
      k_hi[to] = kh; k_lo[to] = kl; v_hi[to] = vh; v_lo[to] = vl;
    }
    if (key0 + KEYS32 < w.end) fetch(key0 + KEYS32);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");     // (the loads of the next tile fly on)
    if (MASKED && key0 >= w.wave_end) return;
    asm volatile("" : "+v"(k_at), "+v"(v_at));
    // ---- scores of 32 keys
    f16v s, s2;                                      // (two sums: products that wait for one another stand half as close)
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = s2[i] = 0.f;
#pragma unroll
    for (int j = 0; j < KS; ++j) {
      const u4 kh = *reinterpret_cast<const u4*>(reinterpret_cast<const char*>(k_hi) + (k_at ^ (j << 5)));
      const u4 kl = *reinterpret_cast<const u4*>(reinterpret_cast<const char*>(k_lo) + (k_at ^ (j << 5)));
      u4 ql;
      if constexpr (D == 128) ql = q_rest[(wave * KS + j) * 64 + lane];
      else ql = q_lo[j];
      s = mfma(kl, q_hi[j], s, f16());
      s2 = mfma(kh, q_hi[j], s2, f16());
      s = mfma(kh, ql, s, f16());
    }
    s += s2;
    float unit[16];
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const f4 ku = *reinterpret_cast<const f4*>(&k_unit[2 * i + 4 * h]), vu = *reinterpret_cast<const f4*>(&v_unit[2 * i + 4 * h]);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        s[i + u] *= ku[u];
        unit[i + u] = vu[u];
      }
    }
    const bool some = MASKED && key0 + KEYS32 > w.wave_full;
    if (some) {
      const int lim = w.seen - key0 - 4 * h;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const bool yes = 8 * (i >> 2) + (i & 3) < lim;
        s[i] = yes ? s[i] : -INFINITY;
        unit[i] = yes ? unit[i] : 0.f;
      }
    }
    float smax = s[0], umax = unit[0];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      smax = fmaxf(smax, s[i]);
      umax = fmaxf(umax, unit[i]);
    }
    smax *= rs;
    if (__any(smax > lift || umax > U_SLACK * sigma)) {
      const float nr = fmaxf(ref, fmaxf(smax, __shfl_xor(smax, 32))), ns = fmaxf(sigma, fmaxf(umax, __shfl_xor(umax, 32)));
      const float f = ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref - nr), fo = f * (sigma / ns);
      sum *= f;
#pragma unroll
      for (int d = 0; d < DB; ++d) o[d] *= fo;
      ref = nr;
      nref = nr == -INFINITY ? 0.f : -nr;
      lift = nr + REF_SLACK;
      sigma = ns;
      per = P_SCALE / ns;
    }
    u4 p_hi[2], p_lo[2];
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], rs, nref));
      s[i + 1] = __builtin_amdgcn_exp2f(fmaf(s[i + 1], rs, nref));
      sum += s[i] + s[i + 1];
      uint32_t hi, lo;
      two_terms(s[i] * unit[i], s[i + 1] * unit[i + 1], per, hi, lo);
      p_hi[i >> 3][(i >> 1) & 3] = hi;
      p_lo[i >> 3][(i >> 1) & 3] = lo;
    }
    if constexpr (MASKED) if (careful) {
      bool bad = false;
#pragma unroll 1
      for (int i = lane; i < KEYS32 * CH * 4; i += 64) {
        const uint32_t x = reinterpret_cast<const uint32_t*>(v_hi)[i];
        bad |= (x & 0x7c00u) == 0x7c00u || (x & 0x7c000000u) == 0x7c000000u;
      }
      if (__any(bad)) {
        // such a tile is summed key by key, each row over the keys that it sees
#pragma unroll 1
        for (int k = 0; k < KEYS32; ++k) {
          float p = 0.f;
#pragma unroll
          for (int i = 0; i < 16; ++i) p = k / 8 * 4 + k % 4 == i ? s[i] : p;
          p = __shfl(p, n + 32 * ((k >> 2) & 1)) * (v_unit[k] * per);
          const bool yes = key0 + k < w.seen;
          const f16* hi_at = reinterpret_cast<const f16*>(v_hi) + k * D;
          const f16* lo_at = reinterpret_cast<const f16*>(v_lo) + k * D;
#pragma unroll
          for (int e = 0; e < DB; ++e)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int d = 32 * e + 8 * (i >> 2) + 4 * h + (i & 3), at = swizzle<D>(k, d >> 3) * 8 + (d & 7);
              const float x = (float)hi_at[at], v = fabsf(x) < INFINITY ? x + (float)lo_at[at] : x;
              o[e][i] = yes ? fmaf(p, v, o[e][i]) : o[e][i];
            }
        }
        return;
      }
    }
    // ---- outputs
    auto column = [&](const u4* plane, int g, int u, int e) {
      const char* at = reinterpret_cast<const char*>(plane) + (v_at ^ (e << 6) ^ (u << 5)) + (16 * g + 8 * u) * CH * 16;
      return __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)at));
    };
#pragma unroll
    for (int g = 0; g < KEYS32 / 16; ++g)
#pragma unroll
      for (int e = 0; e < DB; ++e) {
        const u2 x = column(v_hi, g, 0, e), y = column(v_hi, g, 1, e), z = column(v_lo, g, 0, e), u = column(v_lo, g, 1, e);
        o[e] = mfma((u4){z[0], z[1], u[0], u[1]}, p_hi[g], o[e], f16());
        o[e] = mfma((u4){x[0], x[1], y[0], y[1]}, p_lo[g], o[e], f16());
        o[e] = mfma((u4){x[0], x[1], y[0], y[1]}, p_hi[g], o[e], f16());
      }
  };

  for (;;) {
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    ref = lift = -INFINITY;
    nref = sum = 0.f;
    sigma = U_LEAST;
    per = P_SCALE / U_LEAST;
    int key0 = 0;
    for (; !careful && key0 + KEYS32 <= w.full; key0 += KEYS32) step(std::false_type{}, key0);
    for (; key0 < w.end; key0 += KEYS32) step(std::true_type{}, key0);
    // A weight of 0 times an infinity or a NaN: see the 16-bit kernel.  Here an infinity of K or V that is seen needs the second pass too: its
    // second term is NaN.
    if (careful) break;
    bool bad = false;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) bad |= !(fabsf(o[d][i]) < INFINITY);
    if (!__syncthreads_or(bad && w.seen > 0)) break;       // (a row that sees nothing gives zeros whatever it summed)
    careful = true;
    fetch(0);
  }
  sum += __shfl_xor(sum, 32);
  if (!w.real) return;
  const bool none = ref == -INFINITY && sum == 0.f;
  const float inv = none ? 0.f : 1.f / sum, unit = sigma * (1.f / P_SCALE);
#pragma unroll
  for (int e = 0; e < DB; ++e)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      f4 y;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = none ? 0.f : o[e][4 * g + i] * inv * unit;
      *reinterpret_cast<f4*>(w.out + 32 * e + 8 * g + 4 * h) = y;
    }
}

template <int D>
int run_f32(const Kernel& k, hipStream_t st) {
  const dim3 grid((unsigned)(k.n_tiles * k.a.Hkv));
  if (k.wide) PIPE_KLAUNCH((prompt_f32_kernel<D, true>), grid, dim3(WAVES * 64), 0, st, k);
  else PIPE_KLAUNCH((prompt_f32_kernel<D, false>), grid, dim3(WAVES * 64), 0, st, k);
  PIPE_HIP(hipGetLastError());
  return PIPE_OK;
}

template <typename T, int D>
int run_mfma(const Kernel& k, hipStream_t st) {
  const dim3 grid((unsigned)(k.n_tiles * k.a.Hkv));
  if (k.wide) PIPE_KLAUNCH((prompt_mfma_kernel<T, D, true>), grid, dim3(WAVES * 64), 0, st, k);
  else PIPE_KLAUNCH((prompt_mfma_kernel<T, D, false>), grid, dim3(WAVES * 64), 0, st, k);
  PIPE_HIP(hipGetLastError());
  return PIPE_OK;
}

}  // namespace

int launch_prompt_attention(const PromptAttnArgs& a, hipStream_t st) {
  if (a.Tq == 0) return PIPE_OK;
  Kernel k{};
  k.a = a;
  k.G = a.Hq / a.Hkv;
  const int64_t tiles = (int64_t)a.Tq * k.G / QROWS + a.B + 1;
  if (tiles * a.Hkv > 0xffffff) return PIPE_ESHAPE;
  k.n_tiles = (int)tiles;
  // (a tile's rows are reached from its first by 32-bit offsets)
  k.wide = rows_wide(a.q, a.qs, a.type) && rows_wide(a.k, a.ks, a.type) && rows_wide(a.v, a.vs, a.type) && a.ks.token < (1 << 24) &&
           a.vs.token < (1 << 24);
  if (a.type == PIPE_F32) return a.D == 64 ? run_f32<64>(k, st) : run_f32<128>(k, st);
  if (a.type == PIPE_F16) return a.D == 64 ? run_mfma<f16, 64>(k, st) : run_mfma<f16, 128>(k, st);
  return a.D == 64 ? run_mfma<bf16, 64>(k, st) : run_mfma<bf16, 128>(k, st);
}
