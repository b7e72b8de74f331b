// Rows held in 8 bits, and their products.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "harp_serve.h"

namespace harp {
namespace {

typedef int32_t i4v __attribute__((ext_vector_type(4)));

// ---- one row per workgroup: s = max |x| / 127, q = rint(x / s)
// The row stays in registers between the two passes (NV pieces of 8 values per thread), so it is read once.  Bound by those bytes where there
// are many rows (16384 x 8192 bf16 74 us, 4096 x 28672 65 us: 5.4 TB/s; 2048 x 4096 6.8 us), by the way through one row where there are
// few (1 x 4096 2.3 us, 48 x 14336 3.3 us).  (Here and below: launches back to back in a graph, operands of three calls in turn, so that small
// ones stand in the last-level cache; traced launch by launch the shortest kernels take up to half as long again.)
template <typename T, int TH, int NV>
__global__ __launch_bounds__(TH) void harp_quantize_rows_kernel(const T *X, int64_t ldx, int64_t d, int8_t *codes, int64_t ldc,
                                                                 float *scales, bool wide_in, bool wide_out) {
  __shared__ uint32_t lds[TH / 64];
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x;
  const T *src = X + row * ldx;
  int8_t *dst = codes + row * ldc;
  float x[NV][8];
  uint32_t top = 0;
  auto load = [&](int64_t at, float(&v)[8]) {
    if (at + 8 <= d) {
      sv_load<8>(src + at, wide_in, v);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = at + j < d ? sv_get(src + at + j) : 0.f;
    }
  };
  auto see = [&](const float(&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t m = __float_as_uint(v[j]) & 0x7fffffffu;
      top = top > m ? top : m;
    }
  };
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int64_t at = 8 * (tid + TH * (int64_t)i);
    if (at < d) {
      load(at, x[i]);
      see(x[i]);
    }
  }
  for (int64_t at = 8 * (tid + TH * (int64_t)NV); at < d; at += 8 * TH) {   // rows longer than the registers
    float v[8];
    load(at, v);
    see(v);
  }
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const uint32_t o = (uint32_t)__shfl_xor((int)top, m);
    top = top > o ? top : o;
  }
  if ((tid & 63) == 0) lds[tid >> 6] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < TH / 64; ++i) top = top > lds[i] ? top : lds[i];
  const bool bad = top >= 0x7f800000u;   // an infinity or a NaN in the row
  const float scale = __uint_as_float(top) / 127.0f;
  const bool zero = bad || !(scale > 0.f);
  const CodeScale by(scale, !zero);
  if (tid == 0) scales[row] = bad ? __uint_as_float(0x7fc00000u) : scale;
  sv_either(by.fast, [&](auto fast) {
    auto store = [&](int64_t at, const float(&v)[8]) {
      uint32_t w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = by.code<decltype(fast)::value>(v[j]);
      if (wide_out && at + 8 <= d) {
        *(sv_u2 *)(dst + at) = (sv_u2){sv_pack4(w[0], w[1], w[2], w[3]), sv_pack4(w[4], w[5], w[6], w[7])};
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (at + j < d) dst[at + j] = (int8_t)w[j];
      }
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t at = 8 * (tid + TH * (int64_t)i);
      if (at < d) store(at, x[i]);
    }
    for (int64_t at = 8 * (tid + TH * (int64_t)NV); at < d; at += 8 * TH) {
      float v[8];
      load(at, v);
      store(at, v);
    }
  });
}

// ---- products.  v_mfma_i32_16x16x64_i8: the weight's channels are the rows of the result and the tokens its columns, so a
// lane holds four neighbouring channels of one token.
__device__ __forceinline__ i4v mfma_i8(sv_u4 a, sv_u4 b, i4v c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i4v, a), __builtin_bit_cast(i4v, b), c, 0, 0, 0);
}
__device__ __forceinline__ float scaled(int32_t sum, float sa, float sw) { return ((float)sum * sa) * sw; }

// 16 codes at any address
__device__ __forceinline__ sv_u4 load16(const int8_t *p) {
  sv_u4 v;
  __builtin_memcpy(&v, p, 16);
  return v;
}
// the first `count` (0 .. 15) of them; the others count as 0
__device__ __forceinline__ sv_u4 load_cut(const int8_t *p, int64_t count) {
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (i < count) w[i / 4] |= (uint32_t)(uint8_t)p[i] << (8 * (i % 4));
  return (sv_u4){w[0], w[1], w[2], w[3]};
}

// Any alignment and pitch: tiles of 64 channels x 64 tokens, steps of 128 codes through registers into LDS, the next step's loads in flight
// while this step is multiplied.  Copies straight into LDS, which the tiles below are made of, need aligned pieces.  Bound by the loads, which
// cross lines: 2048 x 4096 x 4096 at an odd address 135 us, aligned (in tiles) 37.
template <typename T>
__global__ __launch_bounds__(256) void harp_matmul_int8_any_kernel(const int8_t *A, int64_t lda, const float *sa, const int8_t *W,
                                                                   int64_t ldw, const float *sw, int64_t n, int64_t d_out,
                                                                   int64_t d_in, T *Y, int64_t ldy) {
  __shared__ __align__(16) int8_t lds[2][2][64][144];   // rows of 128 codes, 144 bytes apart
  const int64_t ch0 = (int64_t)blockIdx.x * 64, tok0 = (int64_t)blockIdx.y * 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, m = lane & 15, g = lane >> 4;
  const int row = tid >> 3, piece = tid & 7;            // and row + 32
  i4v acc[2][2] = {};
  sv_u4 next[2][2];
  auto fetch = [&](const int8_t *M, int64_t ld, int64_t r, int64_t rows, int64_t k) {
    if (r >= rows || k >= d_in) return (sv_u4){0, 0, 0, 0};
    const int8_t *p = M + r * ld + k;
    return k + 16 <= d_in ? load16(p) : load_cut(p, d_in - k);
  };
  auto load = [&](int64_t k) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      next[0][i] = fetch(W, ldw, ch0 + row + 32 * i, d_out, k + 16 * piece);
      next[1][i] = fetch(A, lda, tok0 + row + 32 * i, n, k + 16 * piece);
    }
  };
  auto store = [&](int half) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      *(sv_u4 *)&lds[half][0][row + 32 * i][16 * piece] = next[0][i];
      *(sv_u4 *)&lds[half][1][row + 32 * i][16 * piece] = next[1][i];
    }
  };
  load(0);
  store(0);
  int half = 0;
  for (int64_t k0 = 0; k0 < d_in; k0 += 128, half ^= 1) {
    __syncthreads();
    const bool more = k0 + 128 < d_in;
    if (more) load(k0 + 128);
#pragma unroll
    for (int kk = 0; kk < 128; kk += 64) {
      sv_u4 fw[2], fa[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        fw[i] = *(const sv_u4 *)&lds[half][0][(wave & 1) * 32 + 16 * i + m][kk + 16 * g];
        fa[i] = *(const sv_u4 *)&lds[half][1][(wave >> 1) * 32 + 16 * i + m][kk + 16 * g];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = mfma_i8(fw[i], fa[j], acc[i][j]);
    }
    if (more) store(half ^ 1);
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int64_t tok = tok0 + (wave >> 1) * 32 + 16 * j + m;
    if (tok >= n) continue;
    const float st = sa[tok];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int64_t ch = ch0 + (wave & 1) * 32 + 16 * i + 4 * g + r;
        if (ch < d_out) sv_put(Y + tok * ldy + ch, scaled(acc[i][j][r], st, sw[ch]));
      }
  }
}

// Large products: BM tokens x BN channels per workgroup, WT x WC waves, K in steps of 128 codes that are copied straight into LDS, the
// next step's copies in flight while this step's products run.  An LDS row holds its eight pieces of 16 codes in the order
// piece ^ (row & 7), so that the lanes that read one column of pieces spread over all banks (without it a read took twice as long); the
// copy puts lane i at place i, so it is the address that is exchanged.  A step is 128 codes because eight lanes then ask for one
// whole line of 128 bytes: with steps of 64 codes the same tiles took 10 to 25 % longer.  The rows of a tile of the weight are taken in the
// order that leaves 4 TN neighbouring channels of one token in a lane.
// Bound by power: 4096 x 8192 x 28672 takes 770 us (2500 TOP/s) on random codes and 684 on zeros.
typedef __attribute__((address_space(1))) const void gptr_t;
typedef __attribute__((address_space(3))) void lptr_t;

template <typename T, int BM, int BN, int WT, int WC>
__global__ __launch_bounds__(64 * WT * WC) void harp_matmul_int8_tile_kernel(const int8_t *A, int64_t lda, const float *sa,
                                                                             const int8_t *W, int64_t ldw, const float *sw, int64_t n,
                                                                             int64_t d_out, int64_t d_in, T *Y, int64_t ldy,
                                                                             int32_t tiles_m, int32_t tiles_n, bool wide_y, int32_t slice,
                                                                             int32_t *parts, int64_t ldp) {
  constexpr int NW = WT * WC, TM = BM / (16 * WT), TN = BN / (16 * WC), ROWS = BM + BN, CP = ROWS / 8 / NW;
  static_assert(ROWS % (8 * NW) == 0, "every wave copies the same number of rows");
  __shared__ __align__(16) int8_t lds[2][ROWS * 128];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // Workgroups go to the eight XCDs in turn: give each a run of neighbouring tiles, in columns of up to 8 token tiles, so that
  // its L2 sees few different rows at a time
  const uint32_t total = (uint32_t)tiles_m * tiles_n, xcd = blockIdx.x & 7, q = total >> 3, rem = total & 7;
  const uint32_t idx = (xcd < rem ? xcd * (q + 1) : rem * (q + 1) + (xcd - rem) * q) + (blockIdx.x >> 3);
  const uint32_t band = idx / (8u * tiles_n), in_band = idx % (8u * tiles_n);
  const uint32_t high = (uint32_t)tiles_m - 8 * band < 8 ? (uint32_t)tiles_m - 8 * band : 8;
  const int64_t tok0 = (int64_t)(8 * band + in_band % high) * BM, ch0 = (int64_t)(in_band / high) * BN;

  // rows 0 .. BN - 1 of LDS: channels, then tokens; this lane's part of the wave's CP copies of 8 rows, from the tile's first row
  const int8_t *const w0 = W + ch0 * ldw, *const a0 = A + tok0 * lda;
  uint32_t src[CP];
#pragma unroll
  for (int i = 0; i < CP; ++i) {
    const int r = (i * NW + wave) * 8 + (lane >> 3), piece = (lane & 7) ^ (r & 7);
    if (i * NW * 8 < BN) {
      int64_t ch = r / (16 * TN) * (16 * TN) + 4 * TN * ((r >> 2) & 3) + 4 * (r / 16 % TN) + (r & 3);
      ch = ch0 + ch < d_out ? ch : d_out - 1 - ch0;      // rows past an end are read from the last one and not stored
      src[i] = (uint32_t)(ch * ldw + 16 * piece);
    } else {
      int64_t tok = r - BN;
      tok = tok0 + tok < n ? tok : n - 1 - tok0;
      src[i] = (uint32_t)(tok * lda + 16 * piece);
    }
  }
  static_assert(TM % 2 == 0 && TN % 2 == 0, "tokens come in halves, and a lane stores 8 channels at a time");
  static_assert(BN % (8 * NW) == 0, "a copy is of channels in every wave, or of tokens");
  // this workgroup's slice of the sums: steps begin .. end - 1, and the cut one
  const int begin = blockIdx.y * slice, whole = (int)(d_in >> 7), end = begin + slice < whole ? begin + slice : whole;
  const bool cut = (d_in & 127) != 0 && begin <= whole && whole < begin + slice;
  auto copy_part = [&](int k, int i) {
    const int8_t *base = (i * NW * 8 < BN ? w0 : a0) + (int64_t)k * 128;
    __builtin_amdgcn_global_load_lds((gptr_t *)(base + src[i]), (lptr_t *)(lds[k & 1] + (i * NW + wave) * 1024), 16, 0, 0);
  };
  const int wt = wave % WT, wc = wave / WT, m = lane & 15, g = lane >> 4;
  i4v acc[TN][TM];
#pragma unroll
  for (int c = 0; c < TN; ++c)
#pragma unroll
    for (int t = 0; t < TM; ++t) acc[c][t] = (i4v){0, 0, 0, 0};
  // A step is multiplied in four quarters: two halves of its codes, each in two halves of the tokens.  What the next quarter needs is
  // read from LDS while one is multiplied.  The third quarter is the last that reads this step's half of LDS, so the one barrier of a step
  // stands behind it: the next step has arrived by then (a barrier alone does not wait for copies into LDS), its first operands are read
  // during the last quarter, and the step after it is copied during the last quarter and the next two, in parts: at once
  // the copies would stand in each other's way, and in the products'.
  constexpr int H = TM / 2;
  const int w_at = (wc * TN * 16 + m) * 128, a_at = (BN + wt * TM * 16 + m) * 128;
  const int slot[2] = {16 * (g ^ (m & 7)), 16 * ((4 + g) ^ (m & 7))};
  sv_u4 w[2][TN], f[2][H], b[2][H];
  auto read_front = [&](const int8_t *step, int kk) {
#pragma unroll
    for (int c = 0; c < TN; ++c) w[kk][c] = *(const sv_u4 *)(step + w_at + c * 16 * 128 + slot[kk]);
#pragma unroll
    for (int t = 0; t < H; ++t) f[kk][t] = *(const sv_u4 *)(step + a_at + t * 16 * 128 + slot[kk]);
  };
  auto read_back = [&](const int8_t *step, int kk) {
#pragma unroll
    for (int t = 0; t < H; ++t) b[kk][t] = *(const sv_u4 *)(step + a_at + (H + t) * 16 * 128 + slot[kk]);
  };
  auto nothing = [] {};
  auto quarter = [&](int kk, bool back, auto &&reads, int k, int part) {   // part: of 3 H, of the copies of step k
#pragma unroll
    for (int t = 0; t < H; ++t) {
#pragma unroll
      for (int c = 0; c < TN; ++c)
        acc[c][back ? H + t : t] = mfma_i8(w[kk][c], back ? b[kk][t] : f[kk][t], acc[c][back ? H + t : t]);
      __builtin_amdgcn_sched_barrier(0);
      if (t == 0) reads();
      if (part >= 0) {
        if (k < end) {
#pragma unroll
          for (int i = CP * (part + t) / (3 * H); i < CP * (part + t + 1) / (3 * H); ++i) copy_part(k, i);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  if (begin < end) {
#pragma unroll
    for (int i = 0; i < CP; ++i) copy_part(begin, i);
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    if (begin + 1 < end) {
#pragma unroll
      for (int i = 0; i < CP / 3; ++i) copy_part(begin + 1, i);
    }
    read_front(lds[begin & 1], 0);
    for (int k = begin; k < end; ++k) {
      const int8_t *step = lds[k & 1];
      quarter(0, false, [&] { read_back(step, 0); }, k + 1, H);
      quarter(0, true, [&] { read_front(step, 1); }, k + 1, 2 * H);
      quarter(1, false, [&] { read_back(step, 1); }, 0, -1);
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      quarter(1, true, [&] { read_front(lds[(k + 1) & 1], 0); }, k + 2, 0);   // (behind the last step: not used)
    }
  }
  if (cut) {   // the cut step goes through registers; codes past the end of a row are 0
    __syncthreads();
    const int64_t done = (int64_t)whole * 128;
#pragma unroll 1
    for (int i = 0; i < CP; ++i) {
      const int r = (i * NW + wave) * 8 + (lane >> 3);
      const int64_t at = done + 16 * ((lane & 7) ^ (r & 7));
      uint32_t w[4] = {0, 0, 0, 0};
      uint32_t from = src[0];
#pragma unroll
      for (int j = 1; j < CP; ++j) from = i == j ? src[j] : from;
      const int8_t *p = (i * NW * 8 < BN ? w0 : a0) + done + from;
#pragma unroll
      for (int b = 0; b < 16; ++b)
        if (at + b < d_in) w[b / 4] |= (uint32_t)(uint8_t)p[b] << (8 * (b % 4));
      *(sv_u4 *)(lds[0] + r * 128 + 16 * (lane & 7)) = (sv_u4){w[0], w[1], w[2], w[3]};
    }
    __syncthreads();
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      read_front(lds[0], kk);
      read_back(lds[0], kk);
      quarter(kk, false, nothing, 0, -1);
      quarter(kk, true, nothing, 0, -1);
    }
  }
  const int64_t ch = ch0 + wc * TN * 16 + 4 * TN * g;
  if (parts != nullptr) {   // (rows of ldp sums, which the channels of a tile do not pass)
#pragma unroll
    for (int t = 0; t < TM; ++t) {
      const int64_t tok = tok0 + (wt * TM + t) * 16 + m;
      if (tok >= n || ch >= ldp) continue;
      int32_t *dst = parts + ((int64_t)blockIdx.y * n + tok) * ldp + ch;
#pragma unroll
      for (int c = 0; c < TN; ++c) *(i4v *)(dst + 4 * c) = acc[c][t];
    }
    return;
  }
  float sc[4 * TN];
#pragma unroll
  for (int r = 0; r < 4 * TN; ++r) sc[r] = sw[ch + r < d_out ? ch + r : d_out - 1];
#pragma unroll
  for (int t = 0; t < TM; ++t) {
    const int64_t tok = tok0 + (wt * TM + t) * 16 + m;
    if (tok >= n) continue;
    const float st = sa[tok];
    float y[4 * TN];
#pragma unroll
    for (int c = 0; c < TN; ++c)
#pragma unroll
      for (int r = 0; r < 4; ++r) y[4 * c + r] = scaled(acc[c][t][r], st, sc[4 * c + r]);
    T *dst = Y + tok * ldy + ch;
    if (wide_y && ch + 4 * TN <= d_out) {
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int r = 0; r < 4 * TN; r += 8)
          *(sv_u4 *)(dst + r) = (sv_u4){sv_pack_bf16(y[r], y[r + 1]), sv_pack_bf16(y[r + 2], y[r + 3]), sv_pack_bf16(y[r + 4], y[r + 5]),
                                        sv_pack_bf16(y[r + 6], y[r + 7])};
      } else {
#pragma unroll
        for (int r = 0; r < 4 * TN; r += 4) *(sv_f4 *)(dst + r) = (sv_f4){y[r], y[r + 1], y[r + 2], y[r + 3]};
      }
    } else {
#pragma unroll
      for (int r = 0; r < 4 * TN; ++r)
        if (ch + r < d_out) sv_put(dst + r, y[r]);
    }
  }
}

// Few tokens: the weight is read once, straight into registers, by waves that share a tile of 16 channels x 16 RT tokens and divide its
// sums among them; their parts meet in LDS.  Any alignment.  Bound by the weight's bytes: 4096 x 14336, one row, 12.3 us (4.8 TB/s).  Up to 32 tokens; with
// more, every workgroup's own reading of all of them from L2 takes longer than the weight (32 rows: 22 us, tiles in slices 18 us).
template <typename T, int RT>
__global__ __launch_bounds__(512) void harp_matmul_int8_few_kernel(const int8_t *A, int64_t lda, const float *sa, const int8_t *W,
                                                                   int64_t ldw, const float *sw, int64_t n, int64_t d_out,
                                                                   int64_t d_in, T *Y, int64_t ldy) {
  constexpr int NW = 8, U = 4;
  __shared__ __align__(16) i4v lds[NW][RT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
  const int64_t ch0 = (int64_t)blockIdx.x * 16;
  const int64_t ch = ch0 + m < d_out ? ch0 + m : d_out - 1;      // rows past an end are read from the last one and not stored
  const int8_t *w = W + ch * ldw + 16 * g;
  const int8_t *a[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) a[t] = A + (16 * t + m < n ? 16 * t + m : n - 1) * lda + 16 * g;
  i4v acc[RT] = {};
  const int steps = (int)(d_in >> 6);
  int k = wave;
  for (; k + (U - 1) * NW < steps; k += U * NW) {
    sv_u4 fw[U], fa[U][RT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      fw[u] = load16(w + (int64_t)(k + u * NW) * 64);
#pragma unroll
      for (int t = 0; t < RT; ++t) fa[u][t] = load16(a[t] + (int64_t)(k + u * NW) * 64);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int t = 0; t < RT; ++t) acc[t] = mfma_i8(fw[u], fa[u][t], acc[t]);
  }
  for (; k < steps; k += NW) {
    const sv_u4 fw = load16(w + (int64_t)k * 64);
#pragma unroll
    for (int t = 0; t < RT; ++t) acc[t] = mfma_i8(fw, load16(a[t] + (int64_t)k * 64), acc[t]);
  }
  if ((d_in & 63) && wave == steps % NW) {   // the cut step; what lies past the end of a row counts as 0
    const int64_t done = (int64_t)steps * 64, left = d_in - done - 16 * g;
    auto fetch = [&](const int8_t *p) { return left >= 16 ? load16(p + done) : load_cut(p + done, left); };
    const sv_u4 fw = fetch(w);
#pragma unroll
    for (int t = 0; t < RT; ++t) acc[t] = mfma_i8(fw, fetch(a[t]), acc[t]);
  }
#pragma unroll
  for (int t = 0; t < RT; ++t) lds[wave][t][lane] = acc[t];
  __syncthreads();
  if (wave < RT) {
    const int t = wave;
    i4v sum = lds[0][t][lane];
#pragma unroll
    for (int i = 1; i < NW; ++i) sum += lds[i][t][lane];
    const int64_t tok = 16 * t + m;
    if (tok < n) {
      const float st = sa[tok];
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (ch0 + 4 * g + r < d_out) sv_put(Y + tok * ldy + ch0 + 4 * g + r, scaled(sum[r], st, sw[ch0 + 4 * g + r]));
    }
  }
}

// Y from the slices' sums: four channels of one token per thread.  Bound by the sums' bytes and its launch: 48 tokens x 4096 channels, twelve
// slices, 4.6 us.
template <typename T>
__global__ __launch_bounds__(256) void harp_matmul_int8_join_kernel(const int32_t *parts, int64_t ldp, int32_t slices, const float *sa,
                                                                    const float *sw, int64_t n, int64_t d_out, T *Y, int64_t ldy) {
  const int64_t ch = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x), tok = blockIdx.y;
  if (ch >= d_out) return;
  i4v sum = *(const i4v *)(parts + tok * ldp + ch);
  for (int z = 1; z < slices; ++z) sum += *(const i4v *)(parts + ((int64_t)z * n + tok) * ldp + ch);
  const float st = sa[tok];
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (ch + r < d_out) sv_put(Y + tok * ldy + ch + r, scaled(sum[r], st, sw[ch + r]));
}

// Rows of one launch: a launch has fewer than 2^32 threads in a dimension (rows of 1024 threads: fewer than 2^22 rows).
constexpr int64_t kMostRows = 1 << 21;

template <typename T>
harp_status_t quantize_typed(const T *X, int64_t ldx, int64_t n, int64_t d, int8_t *codes, int64_t ldc, float *scales,
                             bool wide_in, bool wide_out, hipStream_t stream) {
  auto go = [&](auto kernel, int threads) {
    for (int64_t i = 0; i < n; i += kMostRows) {
      const unsigned rows = (unsigned)(n - i < kMostRows ? n - i : kMostRows);
      hipLaunchKernelGGL(kernel, dim3(rows), dim3(threads), 0, stream, X + i * ldx, ldx, d, codes + i * ldc, ldc, scales + i, wide_in, wide_out);
      if (hipGetLastError() != hipSuccess) return HARP_ERR_DEVICE;
    }
    return HARP_OK;
  };
  // 1024 threads a row, up to one row per compute unit (48 rows of 14336: 3.3 us, with 256 threads 5.2) and for rows that 256 threads
  // would hold in too many registers.
  if ((n <= 256 && d > 8 * 256) || d > 8 * 1024) {
    const int64_t pieces = (d + 8 * 1024 - 1) / (8 * 1024);
    if (pieces <= 1) return go(harp_quantize_rows_kernel<T, 1024, 1>, 1024);
    if (pieces <= 2) return go(harp_quantize_rows_kernel<T, 1024, 2>, 1024);
    return go(harp_quantize_rows_kernel<T, 1024, 4>, 1024);
  }
  if (d <= 8 * 512) return go(harp_quantize_rows_kernel<T, 256, 2>, 256);
  return go(harp_quantize_rows_kernel<T, 256, 4>, 256);
}

enum MatmulKernel { kAny, kFew, k32x128, k64x64, k128x128, k192x256, k256x256 };   // (harp_matmul_int8_kernel_name names them in this order)
struct MatmulPlan {
  MatmulKernel kernel;
  int32_t slices;   // of the sums over k, joined by a second launch
};

// The kernel is the one whose estimated time is the least.  A tile kernel's time is its steps times what a step takes with p
// workgroups per compute unit, but no less than its bytes take: measured for n = 1 .. 2048 with weights of 2048 x 8192, 4096 x 4096,
// 4096 x 14336, 11008 x 4096 and 28672 x 8192; the choice is 7 % slower in the mean than the best of every kernel and number of
// slices, 61 % at most (400 rows of 11008 x 4096: 32 x 128 tiles 51 us, 128 x 128 31: five workgroups of the former do not fit a compute
// unit's LDS).  What it chooses between: 4096 x 14336, 48 rows: 64 x 64 tiles 68 us, 32 x 128 in twelve slices 19 us; 2048
// rows of 11008 x 4096: 192 x 256 tiles 95 us (two rounds of workgroups, nearly full), 256 x 256 108 us (two, one of them a third
// full), 128 x 128 108 us; 777 rows of 28672 x 8192: 256 x 256 211 us, 128 x 128 253 us; one row of 4096 x 14336: few 12.3 us, tiles 16.1 us.
struct TileCost {
  MatmulKernel kernel;
  int bm, bn;
};
const TileCost kTiles[] = {{k32x128, 32, 128}, {k64x64, 64, 64}, {k128x128, 128, 128}, {k192x256, 192, 256}, {k256x256, 256, 256}};

double step_us(MatmulKernel kernel, double p) {
  switch (kernel) {
    case k32x128: return p <= 5 ? .40 + .10 * p : .17 * p + .1;
    case k64x64: return p <= 4 ? .34 + .13 * p : .22 * p + .1;
    case k128x128: return p <= 1 ? .8 : p <= 2 ? 1.1 : .56 * p + .3;
    case k192x256: return 1.4 * p;
    default: return 1.62 * p;
  }
}

MatmulPlan choose_matmul(int64_t n, int64_t d_out, int64_t d_in) {
  MatmulPlan best = {k256x256, 1};
  const double weight = (double)d_out * d_in, steps = (double)((d_in + 127) / 128);
  double least = 1e300;
  if (n <= 32) {
    least = fmax(fmax(weight / 5.2e6, (weight + weight * n / 16) / 7.0e6), d_in * (2.4 / 4096));
    best = {kFew, 1};
  }
  static const int kSlices[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
  for (const TileCost &t : kTiles) {
    const double tiles = ceil((double)n / t.bm) * ceil((double)d_out / t.bn);
    for (int s : kSlices) {
      if (s > 1 && (steps < 2 * s || n > 65535)) break;
      const double p = ceil(tiles * s / 256);
      double us = (ceil(steps / s) + 1.5) * step_us(t.kernel, p);
      us = fmax(us, weight / (2.7e6 + .8e6 * fmin(p, 3)) + (double)n * d_in * ceil((double)d_out / t.bn) / 2.0e7);
      if (s > 1) us += 2.0 + (double)s * n * d_out * (8 / 4.5e6);
      if (us < least) least = us, best = {t.kernel, s};
    }
  }
  return best;
}
int64_t part_pitch(int64_t d_out) { return (d_out + 15) / 16 * 16; }
size_t parts_bytes(MatmulPlan plan, int64_t n, int64_t d_out) {
  return plan.slices > 1 ? (size_t)plan.slices * n * part_pitch(d_out) * sizeof(int32_t) : 0;
}

// One launch's part of a product (and the join of its slices)
template <typename T>
harp_status_t matmul_part(MatmulPlan plan, const int8_t *A, int64_t lda, const float *sa, const int8_t *W, int64_t ldw, const float *sw,
                           int64_t n, int64_t d_out, int64_t d_in, T *Y, int64_t ldy, int32_t *parts, hipStream_t stream) {
  auto status = [] { return hipGetLastError() == hipSuccess ? HARP_OK : HARP_ERR_DEVICE; };
  auto tiles = [&](auto kernel, int bm, int bn, int threads) {
    const int64_t tm = (n + bm - 1) / bm, tn = (d_out + bn - 1) / bn;
    const bool wide_y = (uintptr_t)Y % 16 == 0 && ldy * sizeof(T) % 16 == 0;
    const int32_t steps = (int32_t)((d_in + 127) / 128), slice = (steps + plan.slices - 1) / plan.slices;
    const int64_t ldp = part_pitch(d_out);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(tm * tn), (unsigned)plan.slices), dim3(threads), 0, stream, A, lda, sa, W, ldw, sw, n,
                       d_out, d_in, Y, ldy, (int32_t)tm, (int32_t)tn, wide_y, slice, plan.slices > 1 ? parts : nullptr, ldp);
    harp_status_t st = status();
    if (st == HARP_OK && plan.slices > 1) {
      hipLaunchKernelGGL(harp_matmul_int8_join_kernel<T>, dim3((unsigned)((d_out + 1023) / 1024), (unsigned)n), dim3(256), 0, stream,
                         parts, ldp, plan.slices, sa, sw, n, d_out, Y, ldy);
      st = status();
    }
    return st;
  };
  auto few = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)((d_out + 15) / 16)), dim3(512), 0, stream, A, lda, sa, W, ldw, sw, n, d_out, d_in, Y, ldy);
    return status();
  };
  switch (plan.kernel) {
    case kFew: return n <= 16 ? few(harp_matmul_int8_few_kernel<T, 1>) : few(harp_matmul_int8_few_kernel<T, 2>);
    case k32x128: return tiles(harp_matmul_int8_tile_kernel<T, 32, 128, 1, 4>, 32, 128, 256);
    case k64x64: return tiles(harp_matmul_int8_tile_kernel<T, 64, 64, 2, 2>, 64, 64, 256);
    case k128x128: return tiles(harp_matmul_int8_tile_kernel<T, 128, 128, 2, 4>, 128, 128, 512);
    case k192x256: return tiles(harp_matmul_int8_tile_kernel<T, 192, 256, 2, 4>, 192, 256, 512);
    case k256x256: return tiles(harp_matmul_int8_tile_kernel<T, 256, 256, 2, 4>, 256, 256, 512);
    case kAny: break;
  }
  hipLaunchKernelGGL(harp_matmul_int8_any_kernel<T>, dim3((unsigned)((d_out + 63) / 64), (unsigned)((n + 63) / 64)), dim3(256), 0, stream,
                     A, lda, sa, W, ldw, sw, n, d_out, d_in, Y, ldy);
  return status();
}

// A launch has fewer than 2^32 threads in x and fewer than 2^16 workgroups in y, so results are computed in parts of up to 2^24 channels and
// as many rows as make 2^34 results (every tile has 16 results a thread or more), 2^21 at most; rows are whole tiles of every size but in the
// last part.  Slices (n <= 65535) are joined before the next part's take their places.
template <typename T>
harp_status_t matmul_typed(MatmulPlan plan, const int8_t *A, int64_t lda, const float *sa, const int8_t *W, int64_t ldw, const float *sw,
                           int64_t n, int64_t d_out, int64_t d_in, T *Y, int64_t ldy, int32_t *parts, hipStream_t stream) {
  const int64_t most_ch = (int64_t)1 << 24, ch = d_out < most_ch ? d_out : most_ch, wide = ch < 256 ? 256 : ch;
  const int64_t fit = ((int64_t)1 << 34) / wide / 768 * 768, most_rows = fit < kMostRows / 768 * 768 ? fit : kMostRows / 768 * 768;
  for (int64_t j = 0; j < d_out; j += ch)
    for (int64_t i = 0; i < n; i += most_rows) {
      const harp_status_t st = matmul_part(plan, A + i * lda, lda, sa + i, W + j * ldw, ldw, sw + j, n - i < most_rows ? n - i : most_rows,
                                           d_out - j < ch ? d_out - j : ch, d_in, Y + i * ldy + j, ldy, parts, stream);
      if (st != HARP_OK) return st;
    }
  return HARP_OK;
}

// Tiles are addressed from their first row with 32 bits.
bool matmul_aligned(const int8_t *A, int64_t lda, const int8_t *W, int64_t ldw) {
  return ((uintptr_t)A | (uintptr_t)W | (uintptr_t)lda | (uintptr_t)ldw) % 16 == 0 && lda < (1 << 23) && ldw < (1 << 23);
}

}  // namespace
}  // namespace harp

extern "C" {

harp_status_t harp_quantize_rows(const void *X, int64_t ldx, int64_t n, int64_t d, harp_dtype_t dt, int8_t *codes, int64_t ldc,
                                 float *scales, void *stream) {
  if (n < 0 || d < 1 || ldx < d || ldc < d || (dt != HARP_F32 && dt != HARP_BF16)) return HARP_ERR_INVALID_ARG;
  if (n == 0) return HARP_OK;
  if (!X || !codes || !scales) return HARP_ERR_INVALID_ARG;
  if (n > 0x7fffffff) return HARP_ERR_UNSUPPORTED;
  const bool wide_out = ((uintptr_t)codes | (uintptr_t)ldc) % 8 == 0;
  if (dt == HARP_F32)
    return harp::quantize_typed((const float *)X, ldx, n, d, codes, ldc, scales, (uintptr_t)X % 16 == 0 && ldx % 4 == 0, wide_out,
                                (hipStream_t)stream);
  return harp::quantize_typed((const uint16_t *)X, ldx, n, d, codes, ldc, scales, (uintptr_t)X % 16 == 0 && ldx % 8 == 0, wide_out,
                              (hipStream_t)stream);
}

harp_status_t harp_matmul_int8_workspace_size(int64_t n, int64_t d_out, int64_t d_in, size_t *bytes) {
  if (n < 0 || d_out < 0 || d_in < 1 || !bytes) return HARP_ERR_INVALID_ARG;
  if (d_in > HARP_INT8_MAX_DEPTH) return HARP_ERR_UNSUPPORTED;
  *bytes = harp::parts_bytes(harp::choose_matmul(n, d_out, d_in), n, d_out);
  return HARP_OK;
}

const char *harp_matmul_int8_kernel_name(int64_t n, int64_t d_out, int64_t d_in) {
  if (n < 0 || d_out < 0 || d_in < 1 || d_in > HARP_INT8_MAX_DEPTH) return "none";
  static const char *const kNames[][2] = {{"any", nullptr}, {"few", nullptr}, {"tile_32x128", "tile_32x128_sliced"}, {"tile_64x64", "tile_64x64_sliced"},
                                          {"tile_128x128", "tile_128x128_sliced"}, {"tile_192x256", "tile_192x256_sliced"},
                                          {"tile_256x256", "tile_256x256_sliced"}};
  const harp::MatmulPlan plan = harp::choose_matmul(n, d_out, d_in);
  return kNames[plan.kernel][plan.slices > 1];
}

harp_status_t harp_matmul_int8(const int8_t *A, int64_t lda, const float *a_scales, const int8_t *W, int64_t ldw,
                               const float *w_scales, int64_t n, int64_t d_out, int64_t d_in, void *Y, int64_t ldy,
                               harp_dtype_t dt, void *workspace, size_t workspace_bytes, void *stream) {
  if (n < 0 || d_out < 0 || d_in < 1 || lda < d_in || ldw < d_in || ldy < d_out || (dt != HARP_F32 && dt != HARP_BF16))
    return HARP_ERR_INVALID_ARG;
  if (n == 0 || d_out == 0) return HARP_OK;
  if (!A || !a_scales || !W || !w_scales || !Y) return HARP_ERR_INVALID_ARG;
  if (d_in > HARP_INT8_MAX_DEPTH) return HARP_ERR_UNSUPPORTED;
  const harp::MatmulPlan plan = harp::matmul_aligned(A, lda, W, ldw) ? harp::choose_matmul(n, d_out, d_in)
                                                                     : harp::MatmulPlan{n <= 32 ? harp::kFew : harp::kAny, 1};
  const size_t need = harp::parts_bytes(plan, n, d_out);
  if (need && (!workspace || workspace_bytes < need || (uintptr_t)workspace % 16)) return HARP_ERR_INVALID_ARG;
  if (dt == HARP_F32)
    return harp::matmul_typed(plan, A, lda, a_scales, W, ldw, w_scales, n, d_out, d_in, (float *)Y, ldy, (int32_t *)workspace,
                              (hipStream_t)stream);
  return harp::matmul_typed(plan, A, lda, a_scales, W, ldw, w_scales, n, d_out, d_in, (uint16_t *)Y, ldy, (int32_t *)workspace,
                            (hipStream_t)stream);
}

}  // extern "C"
