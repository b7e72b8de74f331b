// Attention of the newest tokens of every sequence over a paged int8 cache.
//
// With s_j = scale * <q, K_j> over the visible keys j of a query, o = sum_j exp(s_j - m) V_j / sum_j exp(s_j - m), taken in one
// pass over the cache with the running maximum m and sum.  Codes are at most 127 in magnitude, so they are exact in half precision and
// both products run on v_mfma_f32_16x16x32_f16; the scales of the pages go into the float32 scores and weights.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "harp_serve.h"

namespace harp {
namespace {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));

typedef __attribute__((address_space(1))) const void gptr_t;
typedef __attribute__((address_space(3))) void lptr_t;

constexpr int kWaves = 4;

__device__ __forceinline__ f4 mfma_h(h8 a, h8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// Four codes as halves: the byte q + 128 under the exponent of 1024 is 1024 + 128 + q.
__device__ __forceinline__ void widen4(uint32_t x, h2 &lo, h2 &hi) {
  x ^= 0x80808080u;
  const h2 bias = {(_Float16)1152.f, (_Float16)1152.f};
  lo = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, x, 0x04010400u)) - bias;
  hi = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, x, 0x04030402u)) - bias;
}
__device__ __forceinline__ h8 widen8(uint32_t x, uint32_t y) {
  h2 a, b, c, d;
  widen4(x, a, b);
  widen4(y, c, d);
  return (h8){a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// Over the lanes n, n + 16, n + 32, n + 48.  A swap of two copies leaves each lane's own value and its partner's in the pair.
typedef uint32_t u2v __attribute__((ext_vector_type(2)));
__device__ __forceinline__ float over_groups_max(float x) {
  uint32_t u = __float_as_uint(x);
  u2v p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  u = __float_as_uint(fmaxf(__uint_as_float(p.x), __uint_as_float(p.y)));
  p = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(p.x), __uint_as_float(p.y));
}
__device__ __forceinline__ float over_groups_sum(float x) {
  uint32_t u = __float_as_uint(x);
  u2v p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  u = __float_as_uint(__uint_as_float(p.x) + __uint_as_float(p.y));
  p = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(p.x) + __uint_as_float(p.y);
}

// x as a value of the lane that the compiler knows nothing about, and does not compute ahead of its use
__device__ __forceinline__ int in_lane(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// 2^k as a float, k clamped to the normal numbers
__device__ __forceinline__ float pow2i(int k) {
  k = k < -126 ? -126 : (k > 127 ? 127 : k);
  return __uint_as_float((uint32_t)(k + 127) << 23);
}
__device__ __forceinline__ int exponent(float x) { return (int)((__float_as_uint(x) >> 23) & 0xffu) - 127; }

// Four neighbouring results; `wide`: their place is a multiple of four elements
__device__ __forceinline__ void put4(float *p, bool wide, f4 v) {
  if (wide) {
    *(f4 *)p = v;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = v[i];
  }
}
__device__ __forceinline__ void put4(uint16_t *p, bool wide, f4 v) {
  if (wide) {
    *(sv_u2 *)p = (sv_u2){sv_pack_bf16(v.x, v.y), sv_pack_bf16(v.z, v.w)};
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) sv_put(p + i, v[i]);
  }
}

// Pieces that a tile of rows has that sees `most` keys (more than one); the last goes on to the end.
__device__ __forceinline__ int used_pieces(int32_t most, int32_t piece, int32_t pieces) {
  const int used = (int)(((int64_t)most + piece - 1) / piece);
  return used < pieces ? used : pieces;
}

// Eight coordinates d0 .. d0 + 7 of a query, turned by its position.
template <typename T, int DH>
__device__ __forceinline__ void load_query(const T *q, int d0, bool wide, const RopeView &rope, int64_t pos, float (&x)[8]) {
#pragma clang fp contract(off)
  sv_load<8>(q + d0, wide, x);
  if (rope.cos == nullptr) return;
  const float *cp = rope.cos + pos * (DH / 2), *sp = rope.sin + pos * (DH / 2);
  if (rope.interleaved) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float a = x[2 * j], b = x[2 * j + 1], c = cp[d0 / 2 + j], s = sp[d0 / 2 + j];
      x[2 * j] = a * c - b * s;
      x[2 * j + 1] = b * c + a * s;
    }
  } else {
    float y[8];
    const bool low = d0 < DH / 2;
    sv_load<8>(q + (low ? d0 + DH / 2 : d0 - DH / 2), wide, y);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int i = (low ? d0 : d0 - DH / 2) + j;
      const float c = cp[i], s = sp[i];
      x[j] = low ? x[j] * c - y[j] * s : x[j] * c + y[j] * s;
    }
  }
}

// The running state of R tiles of 16 rows; a lane has row n of each.
// Weights are exp2(s - m + kWeightLog), m being the largest score or one that the largest has passed by less than kSlack: sums are rescaled
// only where it has passed by more.  They end below 2^15, and half precision at 2^-24, so one half has 2^-21 of the largest weight at full
// precision.  The sum of two halves keeps its 22 bits to 2^-17 of the largest weight times its value scale, which is what it is there for, so it
// rescales more often (2048 rows at the end of 8192 keys, float32: 448 us, with a slack of 8 438; few rows the same).
template <int DH, bool EXACT, int R>
struct Rows {
  static constexpr float kSlack = EXACT ? 1.f : 8.f, kWeightLog = 15.f - kSlack;
  static constexpr float kOut = 0x1p-15f;   // parts are joined as sums of weights up to 1: at 2^15 the sums of large values would pass the range
  h8 qh[R][DH / 32], ql[EXACT ? R : 1][DH / 32];   // queries over a power of two, as one half or the sum of two
  float row_scale[R];                              // not negative: what a product is a score's (base 2) of
  int32_t pos[R];                                  // keys 0 .. pos are visible
  float m[R], l[R], unit[R];                       // largest score, sum of weights; unit: power of two that the scales of the values seen are held against
  f4 acc[R][DH / 16];
  h8 wh[R][2], wl[EXACT ? R : 1][2];               // weights of this turn

  // Row r of the lane: 8 coordinates per step, from d0(step) on; the row's largest is brought to 2^13 .. 2^14.
  template <typename T, typename F>
  __device__ __forceinline__ void start(int r, const T *src, bool wide, const RopeView &rope, int32_t position, float scale_log2, F &&d0) {
    pos[r] = position, m[r] = -__builtin_inff(), l[r] = 0.f, unit[r] = 0x1p-100f;
#pragma unroll
    for (int v = 0; v < DH / 16; ++v) acc[r][v] = (f4){0.f, 0.f, 0.f, 0.f};
    float x[DH / 32][8], top = 0.f;
#pragma unroll
    for (int s = 0; s < DH / 32; ++s) {
      load_query<T, DH>(src, d0(s), wide, rope, position < 0 ? 0 : position, x[s]);
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(x[s][j]));
    }
    top = over_groups_max(top);
    int e = top > 0.f && sv_finite(top) ? 13 - exponent(top) : 0;
    e = e > 126 ? 126 : e;
    const float up = scale_log2 < 0.f ? -pow2i(e) : pow2i(e);
    // (an infinite query: every score is infinite or NaN, and scores of one sign only would leave weights of 0 and a sum of 0, as without a key)
    row_scale[r] = top == __builtin_inff() ? __uint_as_float(0x7fc00000u) : fabsf(scale_log2) * pow2i(-e);
#pragma unroll
    for (int s = 0; s < DH / 32; ++s)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float v = x[s][j] * up;
        qh[r][s][j] = (_Float16)v;
        if constexpr (EXACT) ql[r][s][j] = (_Float16)(v - (float)qh[r][s][j]);
      }
  }

  __device__ __forceinline__ void score(h8 keys, int s, int t, f4 (&sc)[R][4]) const {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      sc[r][t] = mfma_h(keys, qh[r][s], s == 0 ? (f4){0.f, 0.f, 0.f, 0.f} : sc[r][t]);
      if constexpr (EXACT) sc[r][t] = mfma_h(keys, ql[r][s], sc[r][t]);
    }
  }

  // Products of 64 keys to weights.  The lane's keys are key .. key + 15, ks and vs their scales.  hides: some of the 64 may be hidden (from `hi`
  // on, behind a row's position, or on no page: gone), and whatever their scores and scales are does not count.
  __device__ __forceinline__ void weigh(f4 (&sc)[R][4], bool hides, int32_t key, int32_t hi, bool gone, float ks, float vs) {
    // (gone: what was read is no scale; one below 0 would turn the hidden scores' sign, a large one pass the range over `unit`)
    ks = gone ? 0.f : ks, vs = gone ? 0.f : (sv_finite(vs) ? vs : __uint_as_float(0x7fc00000u));
    float f[R], top[R];
    int32_t end[R];   // the lane's keys from here on are hidden
    bool moves = false;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      f[r] = row_scale[r] * ks;
      end[r] = gone ? 0 : (pos[r] + 1 < hi ? pos[r] + 1 : hi) - key;
    }
    if (hides) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int32_t n = in_lane(end[r]);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) sc[r][t][i] = 4 * t + i < n ? sc[r][t][i] : -__builtin_inff();
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      top[r] = sc[r][0][0];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) top[r] = fmaxf(top[r], sc[r][t][i]);
      top[r] *= f[r];   // (f = 0 and nothing visible: NaN, which does not count)
      moves |= top[r] > m[r] + kSlack || (end[r] > 0 && vs > unit[r]);   // (a page that a row does not see has no say in how its weights are rounded)
    }
    // Rare: sums are rescaled only here.  (A lane's condition, though all lanes have the same: behind a scalar branch the sums were
    // copied to other registers in the turns that do not rescale.)
    if (in_lane(__ballot(moves) != 0 ? 1 : 0)) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float vtop = over_groups_max(end[r] > 0 && vs == vs ? vs : 0.f);
        int e = exponent(vtop) + 1;
        e = e > 126 ? 126 : e;
        const float unit_new = vtop > unit[r] ? pow2i(e) : unit[r], shrink = unit[r] * __uint_as_float((254u << 23) - __float_as_uint(unit_new));
        unit[r] = unit_new;
        const float m_new = fmaxf(m[r], over_groups_max(top[r]));
        const float alpha = m[r] == m_new ? 1.f : __builtin_amdgcn_exp2f(m[r] - m_new);
        l[r] *= alpha;
#pragma unroll
        for (int v = 0; v < DH / 16; ++v) acc[r][v] *= alpha * shrink;
        m[r] = m_new;
      }
    }
    float drop[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      // weights times rel; a page whose values are below 2^-60 units adds nothing to the result, but to the sum of weights
      float rel = vs * __uint_as_float((254u << 23) - __float_as_uint(unit[r]));
      rel = rel < 0x1p-60f ? 0x1p-60f : rel;
      drop[r] = __builtin_amdgcn_rcpf(rel);
      const float base = (m[r] == -__builtin_inff() ? 0.f : m[r]) - (__builtin_amdgcn_logf(rel) + kWeightLog);
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[r][t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[r][t][i], f[r], -base));
    }
    if (hides) {   // hidden: 0, also where a scale is NaN; a page whose values' scale is NaN makes its visible keys' weights NaN
      const bool bad = !(vs == vs);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int32_t n = in_lane(end[r]);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) sc[r][t][i] = 4 * t + i < n ? (bad ? vs : sc[r][t][i]) : 0.f;
        drop[r] = bad ? 1.f : drop[r];
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float part[4];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          part[i] = t == 0 ? sc[r][t][i] : part[i] + sc[r][t][i];
          float w = sc[r][t][i];
          if constexpr (EXACT) asm volatile("" : "+v"(w));
          const int j = 4 * (t & 1) + i;
          wh[r][t >> 1][j] = (_Float16)w;
          if constexpr (EXACT) wl[r][t >> 1][j] = (_Float16)(w - (float)wh[r][t >> 1][j]);
        }
      l[r] += ((part[0] + part[1]) + (part[2] + part[3])) * drop[r];
    }
  }

  __device__ __forceinline__ void add(h8 first, h8 second, int v) {   // values of the lane group's keys 0 .. 7 and 8 .. 15
#pragma unroll
    for (int r = 0; r < R; ++r) acc[r][v] = mfma_h(first, wh[r][0], acc[r][v]);
#pragma unroll
    for (int r = 0; r < R; ++r) acc[r][v] = mfma_h(second, wh[r][1], acc[r][v]);
    if constexpr (EXACT) {
#pragma unroll
      for (int r = 0; r < R; ++r) acc[r][v] = mfma_h(first, wl[r][0], acc[r][v]);
#pragma unroll
      for (int r = 0; r < R; ++r) acc[r][v] = mfma_h(second, wl[r][1], acc[r][v]);
    }
  }
};

// Few rows.  A workgroup: 16 rows (token, query head of the group) of one sequence and key head, and one piece of its keys, which its
// W waves take in turns of 64.  The scores are computed transposed (keys x rows), so a lane's scores belong to one row, and what it
// holds after the softmax is the second product's operand without an exchange between lanes: the key of element (tile t, row 4 g + r)
// is 16 g + 4 t + r, which makes the 16 weights of lane group g those of the 16 keys that one 16-byte piece of the value layout holds.
// Keys and values go from memory to registers, the next turn's keys while this turn is computed; nothing passes through LDS but the
// join of the W waves.
// Queries and weights are the sum of two halves, 22 bits, for bfloat16 callers too: what is then left between a result and the exact one is
// the result's own rounding.  One half of each took 3 % less time where the cache's bytes bound the kernel and up to 9 % less elsewhere (48
// ragged contexts of up to 8192 keys 98 us, 16 of 2000 keys 20.6), and moved one entry of six to the next bfloat16 number.
// Bound by the cache's bytes: 48 ragged contexts of up to 8192 keys (8 key heads of 128, 32 query heads) 101 us, 2 x 131072 keys 121 us (4.5 TB/s),
// 16 of 2000 keys 23 us, one of 700 keys 11.5 us.
template <typename T, int DH, int W>
__global__ __launch_bounds__(64 * W, 2) void harp_attention_few_kernel(KvView c, RopeView rope, const T *Q, int64_t q_row,
                                                                                  int64_t q_head, T *O, int64_t o_row, int64_t o_head,
                                                                                  int32_t q_heads, int32_t group, float scale_log2,
                                                                                  int32_t piece, int32_t pieces, float *ws, bool wide, bool wide_o) {
  constexpr int KS = DH / 32, VB = DH / 16, PITCH = DH + 4, TURN = 64 * W;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  int64_t nth;
  const Sequence q = find_sequence(c, c.slot0 + blockIdx.x, group, 4, 1, nth);
  const int64_t rows = (int64_t)q.count * group;
  const int64_t row0 = nth << 4;   // of token row0 / group
  if (nth < 0 || row0 >= rows) return;
  const int kvh = blockIdx.y;
  const int64_t last = row0 + 15 < rows ? row0 + 15 : rows - 1;
  const int32_t before = q.total - q.count;
  const int32_t most = before + (int32_t)(last / group) + 1;       // keys that some row sees
  const int32_t least = before + (int32_t)(row0 / group) + 1;      // keys that every row sees
  // this workgroup's keys; the last piece goes on to the end
  const int z = blockIdx.z;
  const int64_t lo = (int64_t)z * piece;
  int64_t hi = z + 1 == pieces ? (int64_t)most : lo + piece;
  if (hi > most) hi = most;
  if (z > 0 && lo >= most) return;

  const uint32_t head_bytes = (uint32_t)DH << c.page_log, page_bytes = head_bytes * (uint32_t)c.heads, mask = (1u << c.page_log) - 1;
  const int8_t *const k_head = c.k + (int64_t)kvh * head_bytes, *const v_head = c.v + (int64_t)kvh * head_bytes;
  const float *const k_scale = c.k_scale + kvh, *const v_scale = c.v_scale + kvh;
  const int32_t *table = c.table + (int64_t)q.b * c.ld_table;
  // pages of the keys that this lane loads (row n of the tiles), and of the 16 keys of its group
  struct Ids {
    int32_t k, v;
  };
  auto look = [&](int64_t t0) {
    const int64_t k16 = t0 + 16 * (n >> 2), v16 = t0 + 16 * g;
    Ids id = {-1, -1};
    if (k16 < hi) id.k = table[k16 >> c.page_log];
    if (v16 < hi) id.v = table[v16 >> c.page_log];
    return id;
  };
  auto there = [&](int32_t id) { return id >= 0 && id < c.pages; };
  struct Keys {
    sv_u4 code[4][KS / 2];
    float ks, vs;     // scales of the lane's group
    int32_t v;        // its page; -1: none
  };
  auto load_keys = [&](int64_t t0, Ids id, Keys &x) {
    const int8_t *kb = k_head + (uint64_t)(uint32_t)(there(id.k) ? id.k : 0) * page_bytes +
                       ((((uint32_t)t0 + 16 * (n >> 2)) & mask) + (n & 3)) * DH + 16 * g;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < KS / 2; ++i) x.code[t][i] = *(const sv_u4 *)(kb + 4 * t * DH + 64 * i);
    x.v = there(id.v) ? id.v : -1;
    const int64_t sa = (uint64_t)(uint32_t)(x.v < 0 ? 0 : x.v) * (uint32_t)c.heads;
    x.ks = k_scale[sa], x.vs = v_scale[sa];
  };

  const int64_t begin = lo + 64 * wave, open = least < hi ? least : hi;   // before `open` every row sees every key
  Keys ka, kb;
  Ids ahead = look(begin);
  load_keys(begin, ahead, ka);
  ahead = look(begin + TURN);

  Rows<DH, true, 1> st;
  {
    int64_t flat = row0 + n;
    flat = flat < rows ? flat : rows - 1;
    const int32_t tok = (int32_t)(flat / group);
    st.start(0, Q + (q.start + tok) * q_row + (kvh * group + (int)(flat % group)) * q_head, wide, rope, before + tok, scale_log2,
             [&](int s) { return 64 * (s >> 1) + 16 * g + 8 * (s & 1); });
  }
  auto turn = [&](int64_t t0, Keys &now, Keys &next) {
    const int32_t v16 = (int32_t)t0 + 16 * g;
    const bool gone = now.v < 0;
    sv_u4 vc[VB];
    const int8_t *vb = v_head + (uint64_t)(uint32_t)(gone ? 0 : now.v) * page_bytes + ((uint32_t)v16 & mask) * DH + 16 * n;
#pragma unroll
    for (int v = 0; v < VB; ++v) vc[v] = *(const sv_u4 *)(vb + v * 256);
    if (t0 + TURN < hi) {
      load_keys(t0 + TURN, ahead, next);
      ahead = look(t0 + 2 * TURN);
    }
    __builtin_amdgcn_sched_barrier(0);
    f4 sc[1][4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const sv_u4 w = now.code[t][s >> 1];
        st.score((s & 1) ? widen8(w.z, w.w) : widen8(w.x, w.y), s, t, sc);
      }
    st.weigh(sc, t0 + 64 > open || __ballot(gone) != 0, v16, (int32_t)hi, gone, now.ks, now.vs);
#pragma unroll
    for (int v = 0; v < VB; ++v) st.add(widen8(vc[v].x, vc[v].y), widen8(vc[v].z, vc[v].w), v);
  };
  for (int64_t t0 = begin; t0 < hi; t0 += 2 * TURN) {
    turn(t0, ka, kb);
    if (t0 + TURN >= hi) break;
    turn(t0 + TURN, kb, ka);
  }

  const bool whole = pieces == 1 || (piece >= most && z == 0);
  // join of the waves
  __shared__ __align__(16) float lds[W * 16 * PITCH];
  __shared__ float lds_m[W][16], lds_l[W][16];
  const float m = st.m[0], l = over_groups_sum(st.l[0]);
  if (g == 0) lds_m[wave][n] = m;
  __syncthreads();
  float top = lds_m[0][n];
#pragma unroll
  for (int w = 1; w < W; ++w) top = fmaxf(top, lds_m[w][n]);
  const float fac = __builtin_amdgcn_exp2f(m - (top == -__builtin_inff() ? 0.f : top)) * st.kOut;
  if (g == 0) lds_l[wave][n] = l * fac;
#pragma unroll
  for (int v = 0; v < VB; ++v) *(f4 *)&lds[(wave * 16 + n) * PITCH + 16 * v + 4 * g] = st.acc[0][v] * (fac * st.unit[0]);
  __syncthreads();
  for (int u = threadIdx.x; u < 16 * (DH / 4); u += 64 * W) {
    const int r = u / (DH / 4), d = 4 * (u % (DH / 4));
    const int64_t fr = row0 + r;
    if (fr >= rows) break;
    f4 sum = *(const f4 *)&lds[r * PITCH + d];
    float den = lds_l[0][r];
#pragma unroll
    for (int w = 1; w < W; ++w) sum += *(const f4 *)&lds[(w * 16 + r) * PITCH + d], den += lds_l[w][r];
    const int64_t row = q.start + fr / group;
    const int h = kvh * group + (int)(fr % group);
    if (whole) {
      const float inv = den == 0.f ? 0.f : 1.0f / den;
      put4(O + row * o_row + h * o_head + d, wide_o, den == 0.f ? (f4){0.f, 0.f, 0.f, 0.f} : sum * inv);
      if (pieces > 1 && d == 0) ws[(row * q_heads + h) * pieces * (DH + 4) + DH + 2] = __int_as_float(0);
    } else {
      float *part = ws + ((row * q_heads + h) * pieces + z) * (DH + 4);
      *(f4 *)(part + d) = sum;
      if (d == 0) {
        float mm = lds_m[0][r];
#pragma unroll
        for (int w = 1; w < W; ++w) mm = fmaxf(mm, lds_m[w][r]);
        part[DH] = mm;
        part[DH + 1] = den;
        part[DH + 2] = __int_as_float(used_pieces(most, piece, pieces));
      }
    }
  }
}

// Many rows: four waves of 32 rows each, of one sequence and key head, against 64 keys at a time that they share in LDS as halves: every
// code is widened once per workgroup.  Operands as above; a lane's 16 bytes of one product step are one piece of an LDS row, and the pieces
// of a row stand in an order that spreads the lanes of a read over all banks (keys: piece ^ row; values: the two pieces of a coordinate
// change places from 8 coordinates to the next).  The next turn's codes are loaded while this turn is computed, and widened behind it.
// EXACT (float32 callers): queries and weights as the sum of two halves, as above.  For bfloat16 callers they are one half each, an eighth of
// the result's own rounding: here the products and the weights' rounding are what takes the time (two chunks of up to 1500 rows behind up to
// 6000 keys 210 us, with both in two halves 303).
// Bound by vector instructions (the exponentials, the weights' rounding, the widening: 60 % of the cycles) and the matrix instructions (a third),
// which two waves per SIMD hardly overlap: 2048 rows at the end of 8192 keys, 32 query heads of 128, 289 us (0.83 PFLOP/s; float32 452), heads of
// 64 201 us; two chunks of up to 1500 rows behind up to 6000 keys 210 us (float32 323).
template <typename T, int DH, bool EXACT>
__global__ __launch_bounds__(256, 2) void harp_attention_many_kernel(KvView c, RopeView rope, const T *Q, int64_t q_row, int64_t q_head,
                                                                     T *O, int64_t o_row, int64_t o_head, int32_t q_heads, int32_t group,
                                                                     float scale_log2, int32_t piece, int32_t pieces, float *ws, bool wide, bool wide_o, uint32_t slots) {
  constexpr int R = 2, KS = DH / 32, VB = DH / 16, SLOT_LOG = 7, KC = DH / 16, CH = 64 * KC / 256;   // CH: pieces of 16 codes per thread
  __shared__ __align__(16) h8 lds_k[2][64 * DH / 8], lds_v[2][64 * DH / 8];
  __shared__ __align__(16) sv_u4 raw[kWaves][2][64 * CH];   // a wave's own part of the next turn's codes
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
  // Workgroups go to the eight XCDs in turn: each gets a run of slots of one or a few heads, whose keys and values its L2 then holds, the
  // slots with the longest contexts (a sequence's last ones) first.
  const uint32_t eighth = gridDim.x >> 3, rest = gridDim.x & 7, xcd = blockIdx.x & 7;
  const uint32_t idx = (xcd < rest ? xcd * (eighth + 1) : rest + xcd * eighth) + (blockIdx.x >> 3);
  const uint32_t slot = slots - 1 - idx % slots;
  const int kvh = idx / slots / pieces, z = idx / slots % pieces;
  int64_t nth;
  const Sequence q = find_sequence(c, slot, group, SLOT_LOG, 1, nth);
  const int64_t rows = (int64_t)q.count * group, slot0 = nth << SLOT_LOG;
  if (nth < 0 || slot0 >= rows) return;
  const int32_t before = q.total - q.count;
  auto seen = [&](int64_t row) { return before + (int32_t)((row < rows ? row : rows - 1) / group) + 1; };   // keys that a row sees
  const int64_t row0 = slot0 + wave * (16 * R);                 // this wave's first row
  const int64_t lo = (int64_t)z * piece;
  auto until = [&](int64_t most) { return z + 1 == pieces || lo + piece > most ? most : lo + piece; };
  const int64_t slot_most = seen(slot0 + 64 * R - 1), slot_hi = until(slot_most);
  if (z > 0 && lo >= slot_most) return;
  const int32_t most = seen(row0 + 16 * R - 1), least = seen(row0);
  const int64_t hi = row0 < rows ? until(most) : lo;            // this wave's keys end here

  const uint32_t head_bytes = (uint32_t)DH << c.page_log, page_bytes = head_bytes * (uint32_t)c.heads, mask = (1u << c.page_log) - 1;
  const int8_t *const k_head = c.k + (int64_t)kvh * head_bytes, *const v_head = c.v + (int64_t)kvh * head_bytes;
  const float *const k_scale = c.k_scale + kvh, *const v_scale = c.v_scale + kvh;
  const int32_t *table = c.table + (int64_t)q.b * c.ld_table;
  auto there = [&](int32_t id) { return id >= 0 && id < c.pages; };
  // page of the 16 keys of the lane's group
  auto look = [&](int64_t t0) {
    const int32_t k16 = (int32_t)t0 + 16 * g;
    int32_t id = -1;
    if (k16 < (int32_t)slot_hi) id = table[(uint32_t)k16 >> c.page_log];
    return there(id) ? id : -1;
  };
  // Wave w copies the keys and values of group w, one run of DH * 16 bytes each.
  float ks_next, vs_next;
  int32_t page_next;
  auto load = [&](int64_t t0, int32_t ids) {
    const int32_t page = __builtin_amdgcn_readlane(ids, 16 * wave);
    const uint64_t at = (uint64_t)(uint32_t)(page < 0 ? 0 : page) * page_bytes + (((uint32_t)t0 + 16 * wave) & mask) * DH;
    const int8_t *kb = k_head + at, *vb = v_head + at;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      __builtin_amdgcn_global_load_lds((gptr_t *)(kb + (uint32_t)(16 * lane + 1024 * i)), (lptr_t *)&raw[wave][0][64 * i], 16, 0, 0);
      __builtin_amdgcn_global_load_lds((gptr_t *)(vb + (uint32_t)(16 * lane + 1024 * i)), (lptr_t *)&raw[wave][1][64 * i], 16, 0, 0);
    }
    page_next = ids;
    const uint64_t sa = (uint64_t)(uint32_t)(ids < 0 ? 0 : ids) * (uint32_t)c.heads;
    ks_next = k_scale[sa], vs_next = v_scale[sa];
  };
  auto widen = [&](int half) {
    const int me = EXACT ? in_lane(lane) : lane;   // (float32: no registers are left to keep these places in)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (the wave's own copies: no barrier)
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int j = me + 64 * i, key = j / KC, row = 16 * (key >> 2) + 4 * wave + (key & 3), p = 2 * (j % KC);
      const int turn = DH == 128 ? row & 15 : (row >> 1) & 7, swap = (j >> 3) & 1;
      h8 *k = lds_k[half] + row * (DH / 8), *v = lds_v[half] + 2 * (DH * wave + j);
      const sv_u4 kc = raw[wave][0][j], vc = raw[wave][1][j];
      k[p ^ turn] = widen8(kc.x, kc.y);
      k[(p + 1) ^ turn] = widen8(kc.z, kc.w);
      v[swap] = widen8(vc.x, vc.y);
      v[swap ^ 1] = widen8(vc.z, vc.w);
    }
  };
  int32_t ids = look(lo);
  load(lo, ids);
  ids = look(lo + 64);

  Rows<DH, EXACT, R> st;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    int64_t flat = row0 + 16 * r + n;
    flat = flat < rows ? flat : rows - 1;
    const int32_t tok = (int32_t)(flat / group);
    st.start(r, Q + (q.start + tok) * q_row + (kvh * group + (int)(flat % group)) * q_head, wide, rope, before + tok, scale_log2,
             [&](int s) { return 32 * s + 8 * g; });
  }
  widen(0);
  int half = 0;
  const int64_t open = least < hi ? least : hi;   // before it every row sees every key
  for (int64_t t0 = lo; t0 < slot_hi; t0 += 64, half ^= 1) {
    const float ks = ks_next, vs = vs_next;
    const bool gone = page_next < 0;
    __syncthreads();
    load(t0 + 64, ids);   // (behind the last turn: page 0, and not used)
    ids = look(t0 + 128);
    __builtin_amdgcn_sched_barrier(0);
    const int k_turn = DH == 128 ? n : n >> 1, swap = (n >> 3) & 1;
    const h8 *kl = lds_k[half] + n * (DH / 8), *vl = lds_v[half] + (g * DH + n) * 2 + swap;
    // operands are read one tile of keys, or two of coordinates, ahead of the products
    h8 kf[2][KS], vf[2][4];
    auto read_keys = [&](int t) {
#pragma unroll
      for (int s = 0; s < KS; ++s) kf[t & 1][s] = kl[t * 16 * (DH / 8) + ((4 * s + g) ^ k_turn)];
    };
    auto read_values = [&](int p) {
#pragma unroll
      for (int i = 0; i < 2; ++i) vf[p & 1][2 * i] = vl[32 * (2 * p + i)], vf[p & 1][2 * i + 1] = vl[32 * (2 * p + i) + 1 - 2 * swap];
    };
    f4 sc[R][4];
    read_keys(0);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      if (t < 3) read_keys(t + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int s = 0; s < KS; ++s) st.score(kf[t & 1][s], s, t, sc);
      __builtin_amdgcn_sched_barrier(0);
    }
    st.weigh(sc, t0 + 64 > open || __ballot(gone) != 0, (int32_t)t0 + 16 * g, (int32_t)hi, gone, ks, vs);
    read_values(0);
#pragma unroll
    for (int p = 0; p < VB / 2; ++p) {
      if (p + 1 < VB / 2) read_values(p + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 2; ++i) st.add(vf[p & 1][2 * i], vf[p & 1][2 * i + 1], 2 * p + i);
      __builtin_amdgcn_sched_barrier(0);
    }
    widen(half ^ 1);
  }

  const bool whole = pieces == 1 || (piece >= slot_most && z == 0);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float den = over_groups_sum(st.l[r]);
    const int64_t flat = row0 + 16 * r + n;
    if (flat >= rows) continue;
    const int64_t row = q.start + flat / group;
    const int h = kvh * group + (int)(flat % group);
    if (whole) {
      T *dst = O + row * o_row + h * o_head + 4 * g;
      const float inv = den == 0.f ? 0.f : st.unit[r] / den;
#pragma unroll
      for (int v = 0; v < VB; ++v) put4(dst + 16 * v, wide_o, den == 0.f ? (f4){0.f, 0.f, 0.f, 0.f} : st.acc[r][v] * inv);
      if (pieces > 1 && g == 0) ws[(row * q_heads + h) * pieces * (DH + 4) + DH + 2] = __int_as_float(0);
    } else {
      float *part = ws + ((row * q_heads + h) * pieces + z) * (DH + 4);
#pragma unroll
      for (int v = 0; v < VB; ++v) *(f4 *)(part + 16 * v + 4 * g) = st.acc[r][v] * (st.kOut * st.unit[r]);
      if (g == 0) part[DH] = st.m[r], part[DH + 1] = st.kOut * den, part[DH + 2] = __int_as_float(used_pieces(slot_most, piece, pieces));
    }
  }
}

// Joins the pieces of (row, query head)s.  SPREAD: one of them per workgroup, whose groups of DH / 4 threads take its pieces in turns (many
// pieces); otherwise one per group of threads.  The first piece says how many there are; none: the result has been written.  Bound by
// its launch: 2 to 7 us.
template <typename T, int DH, bool SPREAD>
__global__ __launch_bounds__(256) void harp_attention_join_kernel(KvView c, T *O, int64_t o_row, int64_t o_head, int32_t q_heads,
                                                                  int32_t pieces, const float *ws, bool wide_o) {
  constexpr int TG = DH / 4, NG = 256 / TG, STEP = SPREAD ? NG : 1;
  const int d = threadIdx.x % TG, k = threadIdx.x / TG;
  const int64_t at = SPREAD ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * NG + k, row = at / q_heads;
  const int h = (int)(at % q_heads);
  const bool own = row >= c.row_start[0] && row < c.row_start[c.batch] && row < c.rows;   // (nobody's rows are left alone)
  const float *part = ws + (own ? at : 0) * pieces * (DH + 4);
  int used = own ? __float_as_int(part[DH + 2]) : 0;
  used = used > pieces ? pieces : used;
  if (SPREAD && used <= 0) return;
  float top = -__builtin_inff();
  if constexpr (SPREAD) {
    for (int z = threadIdx.x & 63; z < used; z += 64) top = fmaxf(top, part[z * (DH + 4) + DH]);
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) top = fmaxf(top, __shfl_xor(top, i));
  } else {
    for (int z = 0; z < used; ++z) top = fmaxf(top, part[z * (DH + 4) + DH]);
  }
  const float base = top == -__builtin_inff() ? 0.f : top;
  f4 sum = {0.f, 0.f, 0.f, 0.f};
  float den = 0.f;
#pragma unroll 4
  for (int z = SPREAD ? k : 0; z < used; z += STEP) {
    const float *p = part + z * (DH + 4);
    const float f = __builtin_amdgcn_exp2f(p[DH] - base);
    den += p[DH + 1] * f;
    sum += *(const f4 *)(p + 4 * d) * f;
  }
  if constexpr (SPREAD) {
    __shared__ __align__(16) f4 lds[NG][TG];
    __shared__ float lds_l[NG];
    lds[k][d] = sum;
    if (d == 0) lds_l[k] = den;
    __syncthreads();
    if (k != 0) return;
#pragma unroll
    for (int i = 1; i < NG; ++i) sum += lds[i][d], den += lds_l[i];
  }
  if (used <= 0) return;
  put4(O + row * o_row + h * o_head + 4 * d, wide_o, den == 0.f ? (f4){0.f, 0.f, 0.f, 0.f} : sum / den);
}

// Rows and keys of a workgroup, and how many pieces the longest context makes.
struct Split {
  int32_t slot, piece, pieces, waves;
};
// Many rows: from 128 rows of a key head and sequence in the mean on (contexts of 8192 keys, 8 key heads of 128, 4 sequences, with 64, 128 and
// 256 such rows each: few 64, 99, 158 us, many 63, 79, 95; float32 65, 99, 156 and 77, 103, 129), if that makes 112 workgroups or more: fewer
// leave more of the card idle than they save (128 rows behind 1000 keys, 8 workgroups: few 16 us, many 37; 1024 rows, 64: 24 and 37; 4 x 512
// rows, 128: 44 and 40; 256 rows behind 4000 keys, 112 in pieces: 38 and 33).  The mean is what the host knows: where few sequences have nearly
// all of the rows, the others' workgroups are the wrong ones (2048 rows at 4000 keys beside 31 sequences of one row, in many-row workgroups: 256 us,
// the two parts alone 138 and 68; beside 80, in few-row ones: 455, alone 138 and 147).
// Keys are cut into pieces of 512 or more until there are so many workgroups: 512 of the large ones (4 x 8192 keys, 2048 rows each: 316 us, with
// 1024 workgroups 341, and 512 rows each 100 and 121), 1536 of the small ones where a sequence has one tile of rows (48 ragged contexts of
// up to 8192 keys: 101 us, with 768 workgroups 106), 768 where it has more tiles and every piece costs their joining (16 x 2048
// keys, 32 rows each: 41 us, with 1536 workgroups 44).  All sequences have pieces of one length, from the longest that is announced: one of 131072 keys
// among 63 of 1000 takes 618 us, alone 72.  Few keys are one piece, since a second launch costs the host 5 us:
// up to 1024 (one sequence, kernels alone: 1024 keys 14.0 us; 1100 keys 11.2 in five pieces, 15.4 in one), up to 2048 with one tile
// of rows for each of 16 sequences and 8 heads or more (16 x 2000 keys 23 us, in four pieces 28; 64 ragged contexts of up to 2000 keys 48, in
// three 56; 64 x 2000 keys 72 and 70).  Where so short pieces still leave compute units idle, they have 256 keys, one turn of the four waves
// (one sequence of 2000 keys: 11.1 us, in pieces of 512 13.7).
// One piece of more than 512 keys and a compute unit for every workgroup: eight waves take it, since a turn of 64 keys per wave is 2.2 us of
// waiting for memory (kernel alone: one sequence of 700 keys 11.5 us, with four waves 12.9; 16 of 2000 keys 23 and 29; of 512 keys 10.2 both,
// 300 keys 10.4 and 9.8; 288 workgroups of up to 1900 keys, float32: 20.7 and 19.5).
// (Launches back to back in a graph, inputs of three calls in turn, the join of pieces included.)
Split choose_split(int64_t rows, int32_t batch, int32_t group, int32_t heads, int64_t max_kv) {
  const int64_t per = batch > 0 ? rows * group / batch : 0;
  for (bool many = per >= 128;; many = false) {
    const int64_t slot = many ? 128 : 16, slots = rows * group / slot > batch ? rows * group / slot : batch;
    int64_t want = (many ? 512 : per > 16 ? 768 : 1536) / (slots * heads > 0 ? slots * heads : 1);
    if (want < 1 || max_kv <= (per <= 16 && slots * heads >= 128 ? 2048 : 1024)) want = 1;
    int64_t piece = ((max_kv + want - 1) / want + 255) / 256 * 256;
    const int64_t least = !many && (max_kv + 255) / 256 * slots * heads <= 256 ? 256 : 512;
    if (piece < least) piece = least;
    const int64_t pieces = max_kv > piece ? (max_kv + piece - 1) / piece : 1;
    if (many && slots * heads * pieces < 112) continue;
    const bool eight = !many && pieces == 1 && max_kv > 512 && (rows * group / slot + batch) * heads <= 256;
    return {(int32_t)slot, (int32_t)(piece > 0x7fffff00 ? 0x7fffff00 : piece), (int32_t)pieces, eight ? 8 : 4};
  }
}

template <typename T, int DH>
harp_status_t attention_typed(const KvView &c, const RopeView &rope, const void *Q, int64_t q_row, int64_t q_head, void *O,
                              int64_t o_row, int64_t o_head, int32_t q_heads, float scale_log2, Split sp, float *ws, bool wide,
                              bool wide_o, hipStream_t stream) {
  const int32_t group = q_heads / c.heads;
  const int64_t slots = c.rows * group / sp.slot + c.batch;
  if (c.heads > 65535 || sp.pieces > 65535 || q_heads > 65535) return HARP_ERR_UNSUPPORTED;
  if (sp.slot == 16) {
    auto few = [&](auto kernel, int waves) {
      return for_slots(c, slots, [&](const KvView &part, unsigned count) {
        hipLaunchKernelGGL(kernel, dim3(count, (unsigned)c.heads, (unsigned)sp.pieces), dim3(64 * waves), 0, stream, part, rope, (const T *)Q, q_row,
                           q_head, (T *)O, o_row, o_head, q_heads, group, scale_log2, sp.piece, sp.pieces, ws, wide, wide_o);
      });
    };
    const harp_status_t st = sp.waves == 8 ? few(harp_attention_few_kernel<T, DH, 8>, 8) : few(harp_attention_few_kernel<T, DH, 4>, 4);
    if (st != HARP_OK) return st;
  } else {
    // (256 threads each; so many would have 2^31 results of 64 coordinates and more)
    if (slots * c.heads * sp.pieces >= 1 << 24) return HARP_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((harp_attention_many_kernel<T, DH, sizeof(T) == 4>), dim3((unsigned)(slots * c.heads * sp.pieces)), dim3(256), 0, stream, c,
                       rope, (const T *)Q, q_row, q_head, (T *)O, o_row, o_head, q_heads, group, scale_log2, sp.piece, sp.pieces, ws, wide,
                       wide_o, (uint32_t)slots);
    if (hipGetLastError() != hipSuccess) return HARP_ERR_DEVICE;
  }
  if (sp.pieces > 1) {
    const int64_t results = c.rows * q_heads;
    const bool spread = sp.pieces > 16 || (sp.pieces > 2 && results <= 2048);   // (few results: more threads for each)
    const int64_t groups = spread ? results : (results + 1024 / DH - 1) / (1024 / DH);
    if (groups > 0x7fffffff) return HARP_ERR_UNSUPPORTED;
    auto join = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(256), 0, stream, c, (T *)O, o_row, o_head, q_heads, sp.pieces, ws, wide_o);
    };
    if (spread)
      join(harp_attention_join_kernel<T, DH, true>);
    else
      join(harp_attention_join_kernel<T, DH, false>);
    if (hipGetLastError() != hipSuccess) return HARP_ERR_DEVICE;
  }
  return HARP_OK;
}

harp_status_t attention_args(const harp_kv_cache_t *cache, const harp_kv_batch_t *batch, int32_t q_heads, int64_t max_kv_len,
                             KvView *c, Split *sp, size_t *bytes) {
  harp_status_t st = kv_view(cache, batch, c);
  if (st != HARP_OK) return st;
  if (q_heads < 1 || q_heads % cache->kv_heads || max_kv_len < 0) return HARP_ERR_INVALID_ARG;
  if (max_kv_len > c->cap) max_kv_len = c->cap;
  *sp = choose_split(c->rows, c->batch, q_heads / c->heads, c->heads, max_kv_len);
  *bytes = sp->pieces > 1 ? (size_t)c->rows * q_heads * sp->pieces * (cache->head_dim + 4) * sizeof(float) : 0;
  return HARP_OK;
}

}  // namespace
}  // namespace harp

extern "C" {

harp_status_t harp_attention_int8_workspace_size(const harp_kv_cache_t *cache, const harp_kv_batch_t *batch, int32_t q_heads,
                                                 int64_t max_kv_len, size_t *bytes) {
  harp::KvView c;
  harp::Split sp;
  if (!bytes) return HARP_ERR_INVALID_ARG;
  size_t need = 0;
  const harp_status_t st = harp::attention_args(cache, batch, q_heads, max_kv_len, &c, &sp, &need);
  if (st == HARP_OK) *bytes = need;
  return st;
}

const char *harp_attention_int8_kernel_name(const harp_kv_cache_t *cache, const harp_kv_batch_t *batch, int32_t q_heads, int64_t max_kv_len) {
  harp::KvView c;
  harp::Split sp;
  size_t need = 0;
  if (harp::attention_args(cache, batch, q_heads, max_kv_len, &c, &sp, &need) != HARP_OK) return "none";
  return sp.slot == 16 ? (sp.pieces > 1 ? "few_rows_pieces" : "few_rows") : (sp.pieces > 1 ? "many_rows_pieces" : "many_rows");
}

harp_status_t harp_attention_int8(const harp_kv_cache_t *cache, const harp_kv_batch_t *batch, const void *Q, int64_t q_row,
                                  int64_t q_head, void *O, int64_t o_row, int64_t o_head, int32_t q_heads, harp_dtype_t dt,
                                  float scale, const harp_rope_t *rope, int64_t max_kv_len, void *workspace,
                                  size_t workspace_bytes, void *stream) {
  harp::KvView c;
  harp::RopeView r;
  harp::Split sp;
  size_t need = 0;
  harp_status_t st = harp::attention_args(cache, batch, q_heads, max_kv_len, &c, &sp, &need);
  if (st == HARP_OK) st = harp::rope_view(rope, c, &r);
  if (st != HARP_OK) return st;
  if ((dt != HARP_F32 && dt != HARP_BF16) || !(scale - scale == 0.f)) return HARP_ERR_INVALID_ARG;
  st = harp::check_heads(Q, q_row, q_head, c.rows, q_heads, cache->head_dim, false);
  if (st == HARP_OK) st = harp::check_heads(O, o_row, o_head, c.rows, q_heads, cache->head_dim, true);
  if (st != HARP_OK) return st;
  if (c.rows == 0 || c.batch == 0) return HARP_OK;
  if (need && (!workspace || workspace_bytes < need || (uintptr_t)workspace % 16)) return HARP_ERR_INVALID_ARG;
  const float scale_log2 = scale * 1.44269504088896340736f;
  const bool wide = harp::heads_aligned(Q, q_row, q_head, dt, 16);
  const bool wide_o = harp::heads_aligned(O, o_row, o_head, dt, dt == HARP_BF16 ? 8 : 16);
  float *ws = (float *)workspace;
  hipStream_t s = (hipStream_t)stream;
  if (dt == HARP_F32)
    return cache->head_dim == 64
               ? harp::attention_typed<float, 64>(c, r, Q, q_row, q_head, O, o_row, o_head, q_heads, scale_log2, sp, ws, wide, wide_o, s)
               : harp::attention_typed<float, 128>(c, r, Q, q_row, q_head, O, o_row, o_head, q_heads, scale_log2, sp, ws, wide, wide_o, s);
  return cache->head_dim == 64
             ? harp::attention_typed<uint16_t, 64>(c, r, Q, q_row, q_head, O, o_row, o_head, q_heads, scale_log2, sp, ws, wide, wide_o, s)
             : harp::attention_typed<uint16_t, 128>(c, r, Q, q_row, q_head, O, o_row, o_head, q_heads, scale_log2, sp, ws, wide, wide_o, s);
}

}  // extern "C"
