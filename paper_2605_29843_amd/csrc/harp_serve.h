// What the serving kernels share (harp_int8.hip, harp_kv.hip, harp_attn.hip): element types, the ragged batch of a
// paged cache, and checks of its arguments.
#ifndef HARP_SERVE_H_
#define HARP_SERVE_H_

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>

#include "harp.h"

namespace harp {

typedef float sv_f4 __attribute__((ext_vector_type(4)));
typedef uint32_t sv_u4 __attribute__((ext_vector_type(4)));
typedef uint32_t sv_u2 __attribute__((ext_vector_type(2)));

// A batch and its cache as the kernels take them (by value).
struct KvView {
  int8_t *k, *v;              // [pages, heads, page, dh]; [pages, heads, page / 16, dh, 16]
  float *k_scale, *v_scale;   // [pages, heads]
  int64_t pages;
  int32_t heads, page_log;
  const int32_t *table;       // [batch, max_pages], row pitch ld_table
  const int32_t *row_start;   // [batch + 1]
  const int32_t *kv_len;      // [batch]
  int64_t ld_table, rows;
  int32_t batch, cap;         // cap = max_pages * page
  int64_t slot0;              // the slot of a launch's first workgroup
};

// Slots of one launch: a launch has fewer than 2^32 threads in a dimension, and a slot up to 512.
constexpr int64_t kMostSlots = 1 << 22;

struct RopeView {
  const float *cos, *sin;   // [positions, dh / 2], or null
  int32_t interleaved;
};

// One sequence of a ragged batch; device data is clamped so that nothing derived from it leaves the arrays.
struct Sequence {
  int32_t b;
  int64_t start;   // its first row
  int32_t count;   // its rows
  int32_t total;   // its tokens, the rows being the last ones
};

#if defined(__HIPCC__)
__device__ __forceinline__ float sv_widen(uint16_t h) { return __uint_as_float((uint32_t)h << 16); }
__device__ __forceinline__ uint32_t sv_pack_bf16(float lo, float hi) {   // round to nearest, ties to even
  typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
  bf2 v;
  v.x = (__bf16)lo;
  v.y = (__bf16)hi;
  return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ float sv_get(const float *p) { return *p; }
__device__ __forceinline__ float sv_get(const uint16_t *p) { return sv_widen(*p); }
__device__ __forceinline__ void sv_put(float *p, float v) { *p = v; }
__device__ __forceinline__ void sv_put(uint16_t *p, float v) { *p = (uint16_t)sv_pack_bf16(v, v); }

// N consecutive elements; `wide`: they are aligned to 16 bytes (N * size where that is less)
template <int N>
__device__ __forceinline__ void sv_load(const float *p, bool wide, float (&x)[N]) {
  if (wide) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const sv_f4 v = *(const sv_f4 *)(p + i);
      x[i] = v.x, x[i + 1] = v.y, x[i + 2] = v.z, x[i + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = p[i];
  }
}
template <int N>
__device__ __forceinline__ void sv_load(const uint16_t *p, bool wide, float (&x)[N]) {
  if (wide) {
    uint32_t u[N / 2];
    if constexpr (N % 8 == 0) {
#pragma unroll
      for (int i = 0; i < N / 2; i += 4) {
        const sv_u4 v = *(const sv_u4 *)(p + 2 * i);
        u[i] = v.x, u[i + 1] = v.y, u[i + 2] = v.z, u[i + 3] = v.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < N / 2; i += 2) {
        const sv_u2 v = *(const sv_u2 *)(p + 2 * i);
        u[i] = v.x, u[i + 1] = v.y;
      }
    }
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = sv_widen(p[i]);
  }
}

// Codes of one scale, the same for the whole wave: rint of the float32 quotient x / scale, ties to even, within -127 .. 127.
// FAST: the division is a multiplication by the correctly rounded reciprocal and one residual step, t = x * (1 / s), r = x - t s (exact in an
// fma), t + r * (1 / s): 3 operations in place of the ten or so of a division; the quotient is the correctly rounded one.  It is not above
// 127 by more than a rounding, as |x| / 127 rounds to the scale at most, so it needs no bounds, and the integer next to it stands in the low
// byte of its sum with 1.5 * 2^23.  Scales near the ends of the exponent range take the division itself and its bounds; codes are 0 where
// `any` is false.
struct CodeScale {
  float scale, inv;
  bool fast, any;
  __device__ __forceinline__ CodeScale(float s, bool some) : scale(s) {
    any = some;
    fast = __builtin_amdgcn_readfirstlane(some && s > 0x1p-100f && s < 0x1p100f ? 1 : 0) != 0;
    inv = 1.0f / s;
  }
  template <bool FAST>
  __device__ __forceinline__ uint32_t code(float x) const {   // in the low byte
    if constexpr (FAST) {
      const float t = x * inv;
      return __float_as_uint(__builtin_fmaf(__builtin_fmaf(-t, scale, x), inv, t) + 0x1.8p23f);
    } else {
      const float t = __builtin_rintf(x / scale);
      return any ? (uint32_t)(int)(t > 127.f ? 127.f : (t < -127.f ? -127.f : t)) : 0u;
    }
  }
};
// the low bytes of four
__device__ __forceinline__ uint32_t sv_pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_amdgcn_perm(b, a, 0x0c0c0400u) | __builtin_amdgcn_perm(d, c, 0x04000c0cu);
}
// f(true_type) or f(false_type): one body for each, so that a wave's condition is tested once
template <typename F>
__device__ __forceinline__ void sv_either(bool yes, F &&f) {
  if (yes)
    f(std::true_type{});
  else
    f(std::false_type{});
}

// The largest finite value is the last one that a scale may have.
__device__ __forceinline__ bool sv_finite(float x) { return (__float_as_uint(x) & 0x7fffffffu) < 0x7f800000u; }

// Workgroups of a grid are handed to the sequences of a ragged batch without the host knowing their lengths: sequence b
// owns the slots from floor(row_start[b] * mul / 2^div_log) + extra * b on, which leaves it at least floor(rows_b * mul / 2^div_log) +
// extra of them.  A slot's sequence is the last whose first slot is not above it.  Up to 64 sequences are tested by a lane each, which has
// what there is to know of its own at hand (a kernel begins with one wait for memory less); more are searched, 64 places of what is left
// at a time.  nth: the slot's number in its sequence, below 0 where it has none.  There is a sequence (batch >= 1).
__device__ __forceinline__ Sequence find_sequence(const KvView &c, int64_t slot, int32_t mul, int32_t div_log, int32_t extra, int64_t &nth) {
  const int lane = threadIdx.x & 63;
  auto clamped = [&](int64_t row) { return row < 0 ? 0 : row > c.rows ? c.rows : row; };
  auto first = [&](int64_t row, int32_t b) { return ((clamped(row) * mul) >> div_log) + (int64_t)extra * b; };
  int32_t b = 0, begin, end, total;
  if (c.batch <= 64) {
    const int32_t mine = lane < c.batch ? lane : c.batch - 1;
    begin = c.row_start[mine], end = c.row_start[mine + 1], total = c.kv_len[mine];
    const unsigned long long m = __ballot(lane < c.batch && first(begin, lane) <= slot);
    b = m ? 63 - __builtin_clzll(m) : 0;
    begin = __builtin_amdgcn_readlane(begin, b), end = __builtin_amdgcn_readlane(end, b), total = __builtin_amdgcn_readlane(total, b);
  } else {
    for (int32_t left = c.batch;;) {
      const int32_t step = (left + 63) >> 6, at = lane * step;
      const unsigned long long m = __ballot(at < left && first(c.row_start[b + (at < left ? at : 0)], b + at) <= slot);
      const int32_t hit = m ? (63 - __builtin_clzll(m)) * step : 0;
      b += hit;
      if (step == 1) break;
      left = left - hit < step ? left - hit : step;
    }
    b = __builtin_amdgcn_readfirstlane(b);
    begin = c.row_start[b], end = c.row_start[b + 1], total = c.kv_len[b];
  }
  Sequence q;
  q.b = b;
  q.start = clamped(begin);
  const int64_t stop = end < q.start ? q.start : clamped(end);
  q.count = (int32_t)(stop - q.start);
  q.total = total < 0 ? 0 : (total > c.cap ? c.cap : total);
  nth = slot - first(begin, b);
  return q;
}
#endif

// Host side: launch(view, slots of it) for all slots, in launches that are not too large.
template <typename F>
harp_status_t for_slots(KvView c, int64_t slots, F &&launch) {
  for (c.slot0 = 0; c.slot0 < slots; c.slot0 += kMostSlots) {
    launch(c, (unsigned)(slots - c.slot0 < kMostSlots ? slots - c.slot0 : kMostSlots));
    if (hipGetLastError() != hipSuccess) return HARP_ERR_DEVICE;
  }
  return HARP_OK;
}

// Host side: HARP_OK and the kernels' view, or the error of the arguments.
harp_status_t kv_view(const harp_kv_cache_t *cache, const harp_kv_batch_t *batch, KvView *view);
harp_status_t rope_view(const harp_rope_t *rope, const KvView &kv, RopeView *view);
// rows x heads x dh elements with unit inner stride; `wide`: rows of every head may be read 16 bytes at a time
harp_status_t check_heads(const void *p, int64_t row, int64_t head, int64_t rows, int32_t heads, int32_t dh, bool written);
bool heads_aligned(const void *p, int64_t row, int64_t head, harp_dtype_t dt, int bytes);

}  // namespace harp
#endif  // HARP_SERVE_H_
