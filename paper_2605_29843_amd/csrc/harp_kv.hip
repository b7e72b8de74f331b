// The paged int8 cache: appending keys and values with the position rotation, and reading tokens back.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "harp_serve.h"

namespace harp {
namespace {

// Rescaling an older code: rint(q * ratio), ratio = s_old / s_new <= 1.
__device__ __forceinline__ uint32_t rescaled4(uint32_t x, float ratio) {
  uint32_t r = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) r |= ((uint32_t)(int)__builtin_rintf((float)(int8_t)(x >> (8 * i)) * ratio) & 0xffu) << (8 * i);
  return r;
}

// The largest of `top` and two magnitudes, as bit patterns
__device__ __forceinline__ uint32_t larger(uint32_t top, float a, float b) {
  const uint32_t x = __float_as_uint(a) & 0x7fffffffu, y = __float_as_uint(b) & 0x7fffffffu, m = x > y ? x : y;
  return m > top ? m : top;
}

// Threads that share one page of one head: 32 values each, but a wave at least and a workgroup at most.  A workgroup holds as many heads
// as fit.
constexpr int unit_threads(int page, int dh) { return page * dh / 32 < 64 ? 64 : page * dh / 32 > 256 ? 256 : page * dh / 32; }

// Largest |x| of a unit's TPU threads as its bit pattern: infinities and NaN stand above every number.
template <int TPU>
__device__ __forceinline__ uint32_t unit_top(uint32_t top, uint32_t *lds) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const uint32_t o = (uint32_t)__shfl_xor((int)top, m);
    top = top > o ? top : o;
  }
  if constexpr (TPU > 64) {
    constexpr int NW = TPU / 64;
    const int w = threadIdx.x >> 6, first = w / NW * NW;
    if ((threadIdx.x & 63) == 0) lds[w] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NW; ++i) top = top > lds[first + i] ? top : lds[first + i];
  }
  return top;
}

struct NewScale {
  float scale, ratio;   // ratio: what older codes are multiplied by; 1 where they stay
  bool codes;           // new codes are x / scale; otherwise 0
};
__device__ __forceinline__ NewScale grow(uint32_t top, bool older, float old) {
  NewScale s;
  const bool bad = top >= 0x7f800000u || (older && !(old >= 0.f && sv_finite(old)));
  const float a = __uint_as_float(top) / 127.0f;
  s.scale = older && old > a ? old : a;
  s.ratio = older && s.scale > old ? old / s.scale : 1.f;
  s.codes = !bad && s.scale > 0.f;
  if (bad) s.scale = __uint_as_float(0x7fc00000u), s.ratio = 1.f;
  return s;
}

// The page of a ragged batch that a workgroup works on.
struct PageWork {
  Sequence q;
  int32_t first;     // position of row 0; below 0: rows without a place
  int64_t page0;     // position of the page's token 0
  int32_t t0, t1;    // the batch's tokens t0 .. t1 - 1 of the page
  bool any;
};
template <int PAGE>
__device__ __forceinline__ PageWork page_work(const KvView &c, int64_t &nth) {
  PageWork w;
  w.q = find_sequence(c, c.slot0 + blockIdx.x, 1, c.page_log, 2, nth);
  w.first = w.q.total - w.q.count;
  const int32_t begin = w.first < 0 ? 0 : w.first;
  w.page0 = ((int64_t)begin / PAGE + nth) * PAGE;
  w.t0 = begin > w.page0 ? begin - (int32_t)w.page0 : 0;
  w.t1 = w.q.total - w.page0 < PAGE ? (int32_t)(w.q.total - w.page0) : PAGE;
  w.any = w.q.count > 0 && nth >= 0 && w.page0 < w.q.total && w.t1 > w.t0;
  return w;
}

// A unit of threads per sequence, touched page and head; blockIdx.z = 0: keys, 1: values.  It holds the page's new values in registers between
// the pass that finds the largest and the one that rounds them, so inputs are read once, and it alone writes this page's codes of
// this head.  A thread's piece is 8 values of one token for keys (4 pairs of the rotation), and 16 tokens of VP coordinates for values:
// those are the 16-byte groups that the value layout keeps together.  What a few tokens cost is the chain of loads that finds the page
// (rows, table, old scale), so the new values are asked for before the page is known: 64 tokens of 8 heads of 128, 6.3 us.  Many tokens: 8 x
// 2048 tokens 28 us in float32 with inputs and cache in the last-level cache (5.9 TB/s), 39 us with three of them in turn (4.3); bf16 takes
// as long (27 and 39 us) with 100 MB in place of 168, so not its bytes bound it but the steps from a value to its stored code, 16 loads of two
// coordinates for each piece of values among them.  (Launches back to back in a graph.)
template <typename T, int DH, int PAGE>
__global__ __launch_bounds__(256) void harp_kv_append_kernel(KvView c, RopeView rope, const T *K, int64_t k_row, int64_t k_head,
                                                             const T *V, int64_t v_row, int64_t v_head, bool k_wide, bool v_wide,
                                                             bool rope_wide) {
  constexpr int TPU = unit_threads(PAGE, DH), UNITS = 256 / TPU;
  __shared__ uint32_t lds[4];
  int64_t nth;
  const PageWork w = page_work<PAGE>(c, nth);
  if (!w.any) return;
  const int t0 = w.t0, t1 = w.t1, tid = threadIdx.x % TPU, slot = blockIdx.y * UNITS + threadIdx.x / TPU;
  const bool real = slot < c.heads;                               // (the last workgroup's spare units work on a copy of the last head)
  const int head = real ? slot : c.heads - 1;
  const int32_t entry = c.table[(int64_t)w.q.b * c.ld_table + (w.page0 >> c.page_log)];
  const int64_t row0 = w.q.start - w.first + w.page0;             // row of the page's token 0
  const bool older = t0 > 0;

  // `full`: every token of the page is new
  auto keys = [&](auto is_full) {
    constexpr bool FULL = decltype(is_full)::value;
    constexpr int UN = DH / 8, NU = PAGE * UN / TPU;              // pieces of a token, of a thread
    float x[NU][8];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int u = tid + TPU * i, t = t0 + u / UN, e = u % UN;
      if (FULL || t < t1) {
        const T *src = K + (row0 + t) * k_row + head * k_head;
        if (rope.cos == nullptr || rope.interleaved) {
          sv_load<8>(src + 8 * e, k_wide, x[i]);
        } else {   // pairs (j, j + DH / 2)
          float lo[4], hi[4];
          sv_load<4>(src + 4 * e, k_wide, lo);
          sv_load<4>(src + DH / 2 + 4 * e, k_wide, hi);
#pragma unroll
          for (int j = 0; j < 4; ++j) x[i][2 * j] = lo[j], x[i][2 * j + 1] = hi[j];
        }
        if (rope.cos != nullptr) {
#pragma clang fp contract(off)
          const int64_t at = (w.page0 + t) * (DH / 2) + 4 * e;
          float cp[4], sp[4];
          sv_load<4>(rope.cos + at, rope_wide, cp);
          sv_load<4>(rope.sin + at, rope_wide, sp);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float a = x[i][2 * j], b = x[i][2 * j + 1];
            x[i][2 * j] = a * cp[j] - b * sp[j];
            x[i][2 * j + 1] = b * cp[j] + a * sp[j];
          }
        }
#pragma unroll
        for (int j = 0; j < 8; j += 2) top = larger(top, x[i][j], x[i][j + 1]);
      }
    }
    const bool there = entry >= 0 && entry < c.pages;
    const int64_t ph = (there ? (int64_t)entry : 0) * c.heads + head;
    int8_t *codes = c.k + ph * (PAGE * DH);
    const float old = older ? c.k_scale[ph] : 0.f;
    top = unit_top<TPU>(top, lds);
    if (!there || !real) return;
    const NewScale s = grow(top, older, old);
    const CodeScale by(s.scale, s.codes);
    if (!FULL && s.ratio != 1.f) {
      for (int i = tid; i < t0 * (DH / 16); i += TPU) {
        sv_u4 o = *(sv_u4 *)(codes + 16 * i);
        o.x = rescaled4(o.x, s.ratio), o.y = rescaled4(o.y, s.ratio), o.z = rescaled4(o.z, s.ratio), o.w = rescaled4(o.w, s.ratio);
        *(sv_u4 *)(codes + 16 * i) = o;
      }
    }
    sv_either(by.fast, [&](auto fast) {
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        const int u = tid + TPU * i, t = t0 + u / UN, e = u % UN;
        if (FULL || t < t1) {
          uint32_t q[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) q[j] = by.code<decltype(fast)::value>(x[i][j]);
          int8_t *dst = codes + t * DH;
          if (rope.cos == nullptr || rope.interleaved) {
            *(sv_u2 *)(dst + 8 * e) = (sv_u2){sv_pack4(q[0], q[1], q[2], q[3]), sv_pack4(q[4], q[5], q[6], q[7])};
          } else {
            *(uint32_t *)(dst + 4 * e) = sv_pack4(q[0], q[2], q[4], q[6]);
            *(uint32_t *)(dst + DH / 2 + 4 * e) = sv_pack4(q[1], q[3], q[5], q[7]);
          }
        }
      }
    });
    if (tid == 0) c.k_scale[ph] = s.scale;
  };
  auto values = [&](auto is_full) {
    constexpr bool FULL = decltype(is_full)::value;
    constexpr int GR = PAGE / 16, VP = GR * DH / 2 >= TPU ? 2 : 1, NU = GR * DH / VP / TPU;   // groups of 16 tokens; pieces of a thread
    float x[NU][VP][16];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int u = tid + TPU * i, g = u / (DH / VP), e = u % (DH / VP);
#pragma unroll
      for (int t = 0; t < 16; ++t) {
#pragma unroll
        for (int h = 0; h < VP; ++h) x[i][h][t] = 0.f;
        if (FULL || (16 * g + t >= t0 && 16 * g + t < t1)) {
          const T *src = V + (row0 + 16 * g + t) * v_row + head * v_head + VP * e;
          if constexpr (VP == 2) {
            if (v_wide) {
              if constexpr (sizeof(T) == 2) {
                const uint32_t p = *(const uint32_t *)src;
                x[i][0][t] = __uint_as_float(p << 16), x[i][1][t] = __uint_as_float(p & 0xffff0000u);
              } else {
                const sv_u2 p = *(const sv_u2 *)src;
                x[i][0][t] = __uint_as_float(p.x), x[i][1][t] = __uint_as_float(p.y);
              }
            } else {
              x[i][0][t] = sv_get(src), x[i][1][t] = sv_get(src + 1);
            }
          } else {
            x[i][0][t] = sv_get(src);
          }
        }
      }
#pragma unroll
      for (int t = 0; t < 16; t += 2)
#pragma unroll
        for (int h = 0; h < VP; ++h) top = larger(top, x[i][h][t], x[i][h][t + 1]);
    }
    const bool there = entry >= 0 && entry < c.pages;
    const int64_t ph = (there ? (int64_t)entry : 0) * c.heads + head;
    int8_t *codes = c.v + ph * (PAGE * DH);
    const float old = older ? c.v_scale[ph] : 0.f;
    top = unit_top<TPU>(top, lds);
    if (!there || !real) return;
    const NewScale s = grow(top, older, old);
    const CodeScale by(s.scale, s.codes);
    sv_either(by.fast, [&](auto fast) {
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        const int u = tid + TPU * i, g = u / (DH / VP), e = u % (DH / VP);
        const bool has_new = 16 * g < t1 && 16 * g + 16 > t0, has_old = 16 * g < t0;
        if (!FULL && !(has_new || (has_old && s.ratio != 1.f))) continue;
#pragma unroll
        for (int h = 0; h < VP; ++h) {
          int8_t *dst = codes + ((int64_t)g * DH + VP * e + h) * 16;
          uint32_t q[4];
#pragma unroll
          for (int t = 0; t < 4; ++t)   // (a token that is not there has the value 0)
            q[t] = sv_pack4(by.code<decltype(fast)::value>(x[i][h][4 * t]), by.code<decltype(fast)::value>(x[i][h][4 * t + 1]),
                            by.code<decltype(fast)::value>(x[i][h][4 * t + 2]), by.code<decltype(fast)::value>(x[i][h][4 * t + 3]));
          if (!FULL && has_old) {
            const sv_u4 o = *(sv_u4 *)dst;
            const uint32_t was[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              const int n = t0 - 16 * g - 4 * t;   // older tokens among the four
              const uint32_t keep = n >= 4 ? ~0u : n <= 0 ? 0u : (1u << 8 * n) - 1;
              q[t] = (q[t] & ~keep) | ((s.ratio != 1.f ? rescaled4(was[t], s.ratio) : was[t]) & keep);
            }
          }
          *(sv_u4 *)dst = (sv_u4){q[0], q[1], q[2], q[3]};
        }
      }
    });
    if (tid == 0) c.v_scale[ph] = s.scale;
  };
  const bool full = t0 == 0 && t1 == PAGE;
  if (blockIdx.z == 0)
    sv_either(full, keys);
  else
    sv_either(full, values);
}

// The last rows of every sequence, code * scale; same workgroups and pieces as the append.  Bound by the bytes (8 x 2048 tokens of 8 heads of
// 128, bf16, 18 us behind the append that wrote them, 24 us with three caches in turn: 4.3 TB/s), few tokens by the same chain of loads (64
// tokens 4.0 us, 1848 tokens of 64 sequences 6.8).  Rows without a place, or on a page that the
// table does not name, are zeros.
template <typename T, int DH, int PAGE>
__global__ __launch_bounds__(256) void harp_kv_gather_kernel(KvView c, T *K, int64_t k_row, int64_t k_head, T *V, int64_t v_row,
                                                             int64_t v_head, bool k_wide, bool v_wide) {
  constexpr int TPU = unit_threads(PAGE, DH), UNITS = 256 / TPU;
  int64_t nth;
  const PageWork w = page_work<PAGE>(c, nth);
  const int tid = threadIdx.x % TPU, head = blockIdx.y * UNITS + threadIdx.x / TPU;
  if (w.q.count <= 0 || nth < 0 || head >= c.heads) return;
  T *out = blockIdx.z == 0 ? K + head * k_head : V + head * v_head;
  const int64_t pitch = blockIdx.z == 0 ? k_row : v_row;
  if (nth == 0 && w.first < 0) {
    const int64_t lost = w.q.count < -(int64_t)w.first ? w.q.count : -(int64_t)w.first;
    for (int64_t i = tid; i < lost * DH; i += TPU) sv_put(out + (w.q.start + i / DH) * pitch + i % DH, 0.f);
  }
  if (!w.any) return;
  const int t0 = w.t0, t1 = w.t1;
  const int32_t entry = c.table[(int64_t)w.q.b * c.ld_table + (w.page0 >> c.page_log)];
  const bool there = entry >= 0 && entry < c.pages;
  const int64_t ph = (there ? (int64_t)entry : 0) * c.heads + head;
  out += (w.q.start - w.first + w.page0) * pitch;
  if (blockIdx.z == 0) {
    constexpr int UN = DH / 8;
    const float s = c.k_scale[ph];
    const int8_t *codes = c.k + ph * (PAGE * DH);
#pragma unroll 4
    for (int u = tid; u < (t1 - t0) * UN; u += TPU) {
      const int t = t0 + u / UN, e = u % UN;
      const sv_u2 q = *(const sv_u2 *)(codes + t * DH + 8 * e);
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = there ? (float)(int8_t)((j < 4 ? q.x : q.y) >> (8 * (j % 4))) * s : 0.f;
      T *dst = out + t * pitch + 8 * e;
      if (k_wide) {
        if constexpr (sizeof(T) == 2) {
          *(sv_u4 *)dst = (sv_u4){sv_pack_bf16(x[0], x[1]), sv_pack_bf16(x[2], x[3]), sv_pack_bf16(x[4], x[5]), sv_pack_bf16(x[6], x[7])};
        } else {
          *(sv_f4 *)dst = (sv_f4){x[0], x[1], x[2], x[3]};
          *(sv_f4 *)(dst + 4) = (sv_f4){x[4], x[5], x[6], x[7]};
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) sv_put(dst + j, x[j]);
      }
    }
  } else {
    constexpr int GR = PAGE / 16, VP = GR * DH / 2 >= TPU ? 2 : 1;
    const float s = c.v_scale[ph];
    const int8_t *codes = c.v + ph * (PAGE * DH);
    for (int u = tid; u < GR * DH / VP; u += TPU) {
      const int g = u / (DH / VP), e = VP * (u % (DH / VP));
      if (16 * g >= t1 || 16 * g + 16 <= t0) continue;
      sv_u4 o[VP];
#pragma unroll
      for (int h = 0; h < VP; ++h) o[h] = *(const sv_u4 *)(codes + ((int64_t)g * DH + e + h) * 16);
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        if (16 * g + t < t0 || 16 * g + t >= t1) continue;
        float x[VP];
#pragma unroll
        for (int h = 0; h < VP; ++h) {
          const uint32_t q = t < 4 ? o[h].x : t < 8 ? o[h].y : t < 12 ? o[h].z : o[h].w;
          x[h] = there ? (float)(int8_t)(q >> (8 * (t % 4))) * s : 0.f;
        }
        T *dst = out + (16 * g + t) * pitch + e;
        if constexpr (VP == 2) {
          if (v_wide) {
            if constexpr (sizeof(T) == 2)
              *(uint32_t *)dst = sv_pack_bf16(x[0], x[1]);
            else
              *(sv_u2 *)dst = (sv_u2){__float_as_uint(x[0]), __float_as_uint(x[1])};
            continue;
          }
        }
#pragma unroll
        for (int h = 0; h < VP; ++h) sv_put(dst + h, x[h]);
      }
    }
  }
}

// How wide the arrays may be read and written: keys 16 bytes, values and tables 2 and 4 elements at a time.
struct Wide {
  bool k, v, rope;
};

template <typename T, int DH, int PAGE>
harp_status_t append_inst(const KvView &c, const RopeView &rope, const void *K, int64_t k_row, int64_t k_head, const void *V,
                          int64_t v_row, int64_t v_head, Wide wide, int64_t slots, hipStream_t stream) {
  constexpr int UNITS = 256 / unit_threads(PAGE, DH);
  return for_slots(c, slots, [&](const KvView &part, unsigned count) {
    hipLaunchKernelGGL((harp_kv_append_kernel<T, DH, PAGE>), dim3(count, (unsigned)((c.heads + UNITS - 1) / UNITS), 2), dim3(256), 0, stream,
                       part, rope, (const T *)K, k_row, k_head, (const T *)V, v_row, v_head, wide.k, wide.v, wide.rope);
  });
}
template <typename T, int DH, int PAGE>
harp_status_t gather_inst(const KvView &c, const RopeView &, const void *K, int64_t k_row, int64_t k_head, const void *V,
                          int64_t v_row, int64_t v_head, Wide wide, int64_t slots, hipStream_t stream) {
  constexpr int UNITS = 256 / unit_threads(PAGE, DH);
  return for_slots(c, slots, [&](const KvView &part, unsigned count) {
    hipLaunchKernelGGL((harp_kv_gather_kernel<T, DH, PAGE>), dim3(count, (unsigned)((c.heads + UNITS - 1) / UNITS), 2), dim3(256), 0, stream,
                       part, (T *)K, k_row, k_head, (T *)V, v_row, v_head, wide.k, wide.v);
  });
}

typedef harp_status_t (*KvLaunch)(const KvView &, const RopeView &, const void *, int64_t, int64_t, const void *, int64_t,
                                  int64_t, Wide, int64_t, hipStream_t);
// [append, gather][f32, bf16][dh 64, 128][page 16, 32, 64, 128]
#define HARP_KV_PAGES(f, T, D) {f<T, D, 16>, f<T, D, 32>, f<T, D, 64>, f<T, D, 128>}
#define HARP_KV_TYPES(f) {{HARP_KV_PAGES(f, float, 64), HARP_KV_PAGES(f, float, 128)}, {HARP_KV_PAGES(f, uint16_t, 64), HARP_KV_PAGES(f, uint16_t, 128)}}
const KvLaunch kLaunch[2][2][2][4] = {HARP_KV_TYPES(append_inst), HARP_KV_TYPES(gather_inst)};

harp_status_t run_kv(int op, const harp_kv_cache_t *cache, const harp_kv_batch_t *batch, const void *K, int64_t k_row,
                     int64_t k_head, const void *V, int64_t v_row, int64_t v_head, harp_dtype_t dt, const harp_rope_t *rope,
                     void *stream) {
  KvView c;
  RopeView r;
  harp_status_t st = kv_view(cache, batch, &c);
  if (st == HARP_OK) st = rope_view(rope, c, &r);
  if (st != HARP_OK) return st;
  if (dt != HARP_F32 && dt != HARP_BF16) return HARP_ERR_INVALID_ARG;
  st = check_heads(K, k_row, k_head, c.rows, c.heads, cache->head_dim, op == 1);
  if (st == HARP_OK) st = check_heads(V, v_row, v_head, c.rows, c.heads, cache->head_dim, op == 1);
  if (st != HARP_OK) return st;
  if (c.rows == 0 || c.batch == 0 || c.heads == 0) return HARP_OK;
  const int64_t slots = (c.rows >> c.page_log) + 2 * (int64_t)c.batch;
  if (c.heads > 65535) return HARP_ERR_UNSUPPORTED;
  const Wide wide = {heads_aligned(K, k_row, k_head, dt, 16), heads_aligned(V, v_row, v_head, dt, dt == HARP_BF16 ? 4 : 8),
                     ((uintptr_t)r.cos | (uintptr_t)r.sin) % 16 == 0};
  return kLaunch[op][dt == HARP_BF16][cache->head_dim == 128][c.page_log - 4](c, r, K, k_row, k_head, V, v_row, v_head, wide, slots,
                                                                             (hipStream_t)stream);
}

}  // namespace

harp_status_t kv_view(const harp_kv_cache_t *cache, const harp_kv_batch_t *batch, KvView *v) {
  if (!cache || !batch) return HARP_ERR_INVALID_ARG;
  if (cache->pages < 1 || cache->kv_heads < 1 || batch->batch < 0 || batch->rows < 0 || batch->max_pages < 0) return HARP_ERR_INVALID_ARG;
  if (!cache->k || !cache->v || !cache->k_scale || !cache->v_scale) return HARP_ERR_INVALID_ARG;
  if (((uintptr_t)cache->k | (uintptr_t)cache->v) % 16) return HARP_ERR_INVALID_ARG;
  if (cache->head_dim != 64 && cache->head_dim != 128) return HARP_ERR_UNSUPPORTED;
  int log = 4;
  while (log < 7 && (1 << log) != cache->page_size) ++log;
  if ((1 << log) != cache->page_size) return HARP_ERR_UNSUPPORTED;
  if (batch->batch > 0 && (!batch->row_start || !batch->kv_len)) return HARP_ERR_INVALID_ARG;
  if (batch->batch > 0 && batch->max_pages > 0 && (!batch->page_table || batch->ld_table < batch->max_pages)) return HARP_ERR_INVALID_ARG;
  if (batch->rows > 0x7fffffff || (int64_t)batch->max_pages * cache->page_size > (1 << 30)) return HARP_ERR_UNSUPPORTED;
  v->k = cache->k, v->v = cache->v, v->k_scale = cache->k_scale, v->v_scale = cache->v_scale;
  v->pages = cache->pages, v->heads = cache->kv_heads, v->page_log = log;
  v->table = batch->page_table, v->row_start = batch->row_start, v->kv_len = batch->kv_len;
  v->ld_table = batch->ld_table, v->rows = batch->rows, v->batch = batch->batch, v->cap = batch->max_pages * cache->page_size;
  v->slot0 = 0;
  return HARP_OK;
}

harp_status_t rope_view(const harp_rope_t *rope, const KvView &kv, RopeView *v) {
  *v = {nullptr, nullptr, 0};
  if (!rope) return HARP_OK;
  if (rope->positions < kv.cap || (rope->interleaved != 0 && rope->interleaved != 1)) return HARP_ERR_INVALID_ARG;
  if (kv.cap == 0) return HARP_OK;   // no position: the tables may be empty, and nothing is read from them
  if (!rope->cos || !rope->sin) return HARP_ERR_INVALID_ARG;
  *v = {rope->cos, rope->sin, rope->interleaved};
  return HARP_OK;
}

harp_status_t check_heads(const void *p, int64_t row, int64_t head, int64_t rows, int32_t heads, int32_t dh, bool written) {
  if (rows == 0) return HARP_OK;
  if (!p || row < 0 || head < 0) return HARP_ERR_INVALID_ARG;
  // results must not share places: one stride passes over all that the other one spans
  if (written && !((heads == 1 || head >= dh) && (rows == 1 || row >= dh) &&
                   (heads == 1 || rows == 1 || row >= head * (heads - 1) + dh || head >= row * (rows - 1) + dh)))
    return HARP_ERR_INVALID_ARG;
  return HARP_OK;
}

bool heads_aligned(const void *p, int64_t row, int64_t head, harp_dtype_t dt, int bytes) {
  const int64_t e = dt == HARP_BF16 ? 2 : 4;
  return (uintptr_t)p % bytes == 0 && row * e % bytes == 0 && head * e % bytes == 0;
}

}  // namespace harp

extern "C" {

harp_status_t harp_kv_append(const harp_kv_cache_t *cache, const harp_kv_batch_t *batch, const void *K, int64_t k_row,
                             int64_t k_head, const void *V, int64_t v_row, int64_t v_head, harp_dtype_t dt,
                             const harp_rope_t *rope, void *stream) {
  return harp::run_kv(0, cache, batch, K, k_row, k_head, V, v_row, v_head, dt, rope, stream);
}

harp_status_t harp_kv_gather(const harp_kv_cache_t *cache, const harp_kv_batch_t *batch, void *K, int64_t k_row, int64_t k_head,
                             void *V, int64_t v_row, int64_t v_head, harp_dtype_t dt, void *stream) {
  return harp::run_kv(1, cache, batch, K, k_row, k_head, V, v_row, v_head, dt, nullptr, stream);
}

}  // extern "C"
