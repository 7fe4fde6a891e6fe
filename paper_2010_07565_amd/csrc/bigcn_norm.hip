// Layer norm with its gradients, and activation checkpoints in 8 bits, on gfx950.
// C ABI entry points at the end of the file.
//
// All of it is bound by memory: 2-12 bytes and a few tens of vector instructions an
// element.  A row fits registers, so every kernel reads each input once and writes each
// output once.  On the card of the figures below a large copy reaches 4.8 TB/s and a
// fill 6.9.
#include <hip/hip_runtime.h>
#include <float.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "../../include/bigcn.h"
#include "bigcn_rows.h"

namespace {

using namespace bigcn;

constexpr int kB = 256;  // threads per block (4 waves)
constexpr int kW = kB / 64;

inline size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }
inline int64_t words(int64_t k) { return (k + 63) / 64; }
inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
inline bool dtype_ok(int t) {
  return t == BIGCN_DT_F32 || t == BIGCN_DT_F16 || t == BIGCN_DT_BF16;
}
inline size_t dtype_size(int t) { return t == BIGCN_DT_F32 ? 4 : 2; }

// Launches f with the storage type of a bigcn_dtype.
template <typename F>
inline void with_type(int t, F f) {
  if (t == BIGCN_DT_F16)
    f(F16());
  else if (t == BIGCN_DT_BF16)
    f(BF16());
  else
    f(F32());
}

struct NormOut {
  void* y;
  int64_t ldy;
  float *mean, *rstd;
  int8_t* codes;
  int64_t ldc;
  float* qscale;
  int64_t ldq;
  const int64_t* rowptr;
  int sym;
  uint64_t* bits;
  int64_t ldw;
  float* scale;
};

// The forward: the mean, then the mean square of the centred values (a second pass over
// the registers: nothing cancels), y, and from y what the caller asked for.
// 2449029 x 256 fp32: to y 873 us (5.7 TB/s), to signs, scales and checkpoint 629 (5.3);
// 232965 x 602 bf16: 110 (5.1) and 130 (3.5, by then bound by its instructions).
// Every row is read once and stays in registers; L lanes hold it (or W
// waves, one row a block), 64 / L rows a wave.  (Issuing the next rows' loads before
// this row's arithmetic measured no faster: other waves' loads fill the time.)
// Without NORM only the checkpoint is made.
template <typename T, int W, int L, int NV, bool TINY, bool NORM>
__global__ __launch_bounds__(64 * (W > 1 ? W : kW)) void k_norm(
    const typename T::elem* x, int64_t ldx, int64_t rows, int32_t cols,
    const float* __restrict__ gamma, const float* __restrict__ beta, float eps, NormOut o) {
  typedef RowMap<W, L, NV, TINY> Map;
  __shared__ float slots[3][W];
  const Map m(cols);
  constexpr int kRB = W > 1 ? 1 : kW * Map::kRows;  // rows a block holds at once
  const int sub = W > 1 ? 0 : (int)(threadIdx.x / L);
  f32x4 ga[NV], be[NV];
  if constexpr (NORM) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      ga[v] = gamma != nullptr ? m.template load<F32>(gamma + 4 * m.t, v)
                               : f32x4{1.f, 1.f, 1.f, 1.f};
      be[v] = beta != nullptr ? m.template load<F32>(beta + 4 * m.t, v)
                              : f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  const float inv_cols = 1.f / (float)cols;
  const int groups = (cols + kGroup - 1) / kGroup;
  uint32_t owned_bits = 0;  // of the last chunk's four
#pragma unroll
  for (int u = 0; u < 4; ++u) owned_bits |= m.owns(NV - 1, u) ? 1u << u : 0u;
  // the group of chunk v = l16 of the 16 lanes around this one
  const int l16 = m.t & 15, group16 = l16 * (Map::kLanes / 16) + (m.t >> 4);
  auto fetch = [&](int64_t i, typename T::raw (&v)[NV]) {
    const typename T::elem* p = x + (i < rows ? i : rows - 1) * ldx + 4 * m.t;
#pragma unroll
    for (int k = 0; k < NV; ++k) v[k] = m.template load<T>(p, k);
  };
  const int64_t stride = (int64_t)gridDim.x * kRB;
  int64_t i = (int64_t)blockIdx.x * kRB + sub;
  // (rows of a block start together: every lane takes the same number of turns)
  for (int64_t i0 = (int64_t)blockIdx.x * kRB; i0 < rows; i0 += stride, i += stride) {
    typename T::raw raw[NV];
    fetch(i, raw);
    f32x4 v[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) v[k] = m.owned(k, to_f32(raw[k]));
    const bool in = i < rows;
    if (!NORM || o.codes != nullptr) {
      int8_t* cr = o.codes + i * o.ldc + 4 * m.t;
      uint32_t tops[NV];
      Quant q[NV];
      float step = 0.f;
#pragma unroll
      for (int k = 0; k < NV; ++k) tops[k] = max16(magnitude_bits(v[k]));
      quants_of<NV>(tops, q);
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const uint32_t c = quantize4(v[k], q[k]);
        if (in) m.store_q8(cr, k, c);
        step = l16 == k ? q[k].step : step;
      }
      if (in && l16 < NV && group16 < groups) o.qscale[i * o.ldq + group16] = step;
    }
    if constexpr (!NORM) continue;
    // v less its mean, which is left in mean; returns the sum of its squares
    float mean;
    auto centre = [&] {
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < NV; ++k) s += (v[k][0] + v[k][1]) + (v[k][2] + v[k][3]);
      // (the quotient corrected by its remainder: the mean of equal elements is that
      // element)
      s = row_sum<W, L>(s, slots[0]);
      mean = s * inv_cols;
      mean = __builtin_fmaf(__builtin_fmaf(-mean, (float)cols, s), inv_cols, mean);
      float s2 = 0.f;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        v[k] -= mean;
        const f32x4 c = m.owned(k, v[k]);
        s2 += (c[0] * c[0] + c[1] * c[1]) + (c[2] * c[2] + c[3] * c[3]);
      }
      return row_sum<W, L>(s2, slots[1]);
    };
    float rstd = rsqrt1(centre() * inv_cols + eps), rstd_v = rstd;  // (of x and of v)
    // Finite elements whose sum or squares pass fp32's range (from about 1e17 on; rows that
    // hold an infinity or a NaN come here too): once more with the row read again times
    // 2^-80, whose largest is 2^-23 to 2^48 then.  Rows beside them get the same again.
    if constexpr (!std::is_same<T, F16>::value) {
      const bool over = !(rstd > 0.f);  // (0 * infinity of an infinite variance is NaN)
      if (__builtin_amdgcn_ballot_w64(over) != 0) {
        const float down = over ? 0x1p-80f : 1.f, up = over ? 0x1p80f : 1.f;
        int64_t j = i;  // (its addresses anew: the first ones held until here cost registers)
        if constexpr (W > 1)
          asm volatile("" : "+s"(j));
        else
          asm volatile("" : "+v"(j));
        fetch(j, raw);
#pragma unroll
        for (int k = 0; k < NV; ++k) v[k] = m.owned(k, to_f32(raw[k])) * down;
        const float var = centre() * inv_cols, whole = var * up * up + eps;
        mean *= up;
        // (finite where only sums passed the range; the limit: of a row of equal elements,
        // whose v is zero)
        const bool back = whole < INFINITY;
        const float r = over ? rsqrt1(back ? whole : var + eps * down * down) : rstd;
        rstd = back ? r : r * down;
        rstd_v = back ? fminf(r * up, FLT_MAX) : r;
      }
    }
    if (in && m.t == 0) {
      if (o.mean != nullptr) o.mean[i] = mean;
      if (o.rstd != nullptr) o.rstd[i] = rstd;
    }
    f32x4 y[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) y[k] = ga[k] * (v[k] * rstd_v) + be[k];
    if (o.bits != nullptr) {
      float l1 = 0.f;
      uint32_t lo = 0, hi = 0;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const f32x4 ay = m.owned(k, y[k]);
        l1 += (fabsf(ay[0]) + fabsf(ay[1])) + (fabsf(ay[2]) + fabsf(ay[3]));
        // the sign bits, element 3 first: a bit is set for y >= 0 (-0 too, a NaN not)
        uint32_t nib = 0;
#pragma unroll
        for (int u = 3; u >= 0; --u) nib = nib + nib + (y[k][u] >= 0.f ? 1u : 0u);
        if (k + 1 == NV) nib &= owned_bits;
        if (k + 1 == NV) nib >>= m.skip;
        uint32_t w = nib << (4 * (m.t & 7));
        w |= dpp_u32<kXor1>(w);
        w |= dpp_u32<kXor2>(w);
        w |= dpp_u32<kHalfMirror>(w);
        const uint32_t other = dpp_u32<kMirror>(w);  // the other 8 lanes' half of the word
        lo = l16 == k ? (l16 < 8 ? w : other) : lo;
        hi = l16 == k ? (l16 < 8 ? other : w) : hi;
      }
      l1 = row_sum<W, L>(l1, slots[2]);
      if (in) {
        if (l16 < NV && group16 < groups)
          o.bits[i * o.ldw + group16] = ((uint64_t)hi << 32) | lo;
        for (int64_t w = groups + m.t; w < o.ldw; w += Map::kLanes) o.bits[i * o.ldw + w] = 0;
        if (m.t == 0) {
          float sc = l1 * inv_cols;
          if (o.rowptr != nullptr && o.sym) {
            const int64_t dg = o.rowptr[i + 1] - o.rowptr[i];
            sc = sc * (dg > 0 ? rsqrt1((float)dg) : 0.f);
          }
          o.scale[i] = sc;
        }
      }
    }
    if (o.y != nullptr && in) {
      typename T::elem* yr = (typename T::elem*)o.y + i * o.ldy + 4 * m.t;
#pragma unroll
      for (int k = 0; k < NV; ++k) m.template store<T>(yr, k, y[k]);
    }
  }
}

// x of the norm's backward: the activations, or (Q8) their checkpoint.
template <typename T>
struct Kept {
  const typename T::elem* x;
  int64_t ldx;
  const int8_t* codes;
  int64_t ldc;
  const float* qscale;
  int64_t ldq;
};

// The backward: the row's two sums, dx and the terms of dgamma and dbeta in one pass over
// dy and x, or over dy and the 1.06 bytes an element of x's checkpoint.  2449029 x 256
// fp32: 1380 us from x (5.5 TB/s), 1020-1120 from the checkpoint (5.1-5.6); 169343 x 128
// fp32: 45-49 and 37; 232965 x 602 bf16: 158 and 135 (5.3).
// Each row is held in registers as in the forward, blocks taking rows in
// turn; dx is written, and each lane adds its columns' terms of dgamma and dbeta over
// the rows it sees in fp32, in runs of kRun turns, at whose end the block's lanes and
// waves are joined: a chain of at most 69 additions of fp32.  A block's runs are added up
// in fp64 in LDS and leave one part, rounded once: part[block][2][cols].  Where a row
// takes a block every run leaves a part of its own, part[run][block].  (Runs added to
// fp64 sums in memory instead cost 1-4 %: 300000 x 2048 bf16 721 -> 748 us.)
constexpr int kRun = 64;

template <typename T, bool Q8, int W, int L, int NV, bool TINY>
__global__ __launch_bounds__(64 * (W > 1 ? W : kW)) void k_norm_grad(
    const typename T::elem* dy, int64_t lddy, int64_t rows, int32_t cols, Kept<T> kept,
    const float* __restrict__ mean, const float* __restrict__ rstd,
    const float* __restrict__ gamma, int relu, typename T::elem* dx, int64_t lddx,
    float* __restrict__ part) {
  typedef RowMap<W, L, NV, TINY> Map;
  constexpr int kRB = W > 1 ? 1 : kW * Map::kRows;
  __shared__ float slots[2][2][W];
  __shared__ float red[W > 1 ? 1 : 2 * kW][W > 1 ? 1 : NV * Map::kStep];
  __shared__ double sums[2][W > 1 ? 1 : NV * Map::kStep];  // (column c: thread c mod kB alone)
  const Map m(cols);
  const int sub = W > 1 ? 0 : (int)(threadIdx.x / L);
  const int l16 = m.t & 15, group16 = l16 * (Map::kLanes / 16) + (m.t >> 4);
  const int groups = (cols + kGroup - 1) / kGroup;
  const int qat = min(group16, groups - 1);  // the scale this lane reads
  f32x4 ga[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v)
    ga[v] = gamma != nullptr ? m.template load<F32>(gamma + 4 * m.t, v) : f32x4{1.f, 1.f, 1.f, 1.f};
  const float inv_cols = 1.f / (float)cols;
  f32x4 dg[NV], db[NV];
  struct Row {
    typename T::raw d[NV], x[Q8 ? 1 : NV];
    uint32_t c[Q8 ? NV : 1];
    float q, mean, rstd;
  };
  auto fetch = [&](int64_t i, Row& r) {  // (past the last row: that one)
    const int64_t j = i < rows ? i : rows - 1;
    const typename T::elem* p = dy + j * lddy + 4 * m.t;
#pragma unroll
    for (int k = 0; k < NV; ++k) r.d[k] = m.template load<T>(p, k);
    if constexpr (Q8) {
      const int8_t* c = kept.codes + j * kept.ldc + 4 * m.t;
#pragma unroll
      for (int k = 0; k < NV; ++k) r.c[k] = m.load_q8(c, k);
      r.q = kept.qscale[j * kept.ldq + qat];
    } else {
      const typename T::elem* xr = kept.x + j * kept.ldx + 4 * m.t;
#pragma unroll
      for (int k = 0; k < NV; ++k) r.x[k] = m.template load<T>(xr, k);
    }
    r.mean = mean[j];
    r.rstd = rstd[j];
  };
  // One turn: the rows i of a block's lanes, held in r.  ALL: every row is in range
  // and dx is stored by every lane, also where its last chunk holds columns of another
  // lane (the same values twice).
  auto turn = [&](auto all, const Row& r, int64_t i, int32_t n) {
    constexpr bool ALL = decltype(all)::value;
    const bool in = ALL || i < rows;
    f32x4 xh[NV], d[NV];
    uint32_t neg = 0;  // bit 4k + u: a ReLU's output that is not positive
    if constexpr (Q8) {
      float q[NV];
      bcast_lanes<NV>(r.q, q);
      const float mr = r.mean * r.rstd;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const f32x4 c = codes_f32(r.c[k]);
        xh[k] = c * (q[k] * r.rstd) - mr;
        if (relu)
#pragma unroll
          for (int u = 0; u < 4; ++u) neg |= c[u] > 0.f ? 0u : 1u << (4 * k + u);
      }
    } else {
      // (halves: x - mean may be past fp32's range, its half is not)
      const float half_mean = 0.5f * r.mean, twice_rstd = 2.f * r.rstd;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const f32x4 x = to_f32(r.x[k]);
        xh[k] = (x * 0.5f - half_mean) * twice_rstd;
        if (relu)
#pragma unroll
          for (int u = 0; u < 4; ++u) neg |= x[u] > 0.f ? 0u : 1u << (4 * k + u);
      }
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) d[k] = to_f32(r.d[k]);
    if (!in)  // nothing of a row past the last
#pragma unroll
      for (int k = 0; k < NV; ++k) d[k] = xh[k] = f32x4{0.f, 0.f, 0.f, 0.f};
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const f32x4 dk = m.owned(k, d[k]), xk = m.owned(k, xh[k]);
      dg[k] += dk * xk;
      db[k] += dk;
      d[k] *= ga[k];
      const f32x4 g = dk * ga[k], t = g * xk;
      s1 += (g[0] + g[1]) + (g[2] + g[3]);
      s2 += (t[0] + t[1]) + (t[2] + t[3]);
    }
    if (!ALL && dx == nullptr) return;
    s1 = lanes_sum<L>(s1);
    s2 = lanes_sum<L>(s2);
    if constexpr (W > 1) {
      if ((threadIdx.x & 63) == 0) {
        slots[n & 1][0][threadIdx.x >> 6] = s1;
        slots[n & 1][1][threadIdx.x >> 6] = s2;
      }
      __syncthreads();
      s1 = slots[n & 1][0][0];
      s2 = slots[n & 1][1][0];
      for (int w = 1; w < W; ++w) {
        s1 += slots[n & 1][0][w];
        s2 += slots[n & 1][1][w];
      }
    }
    s1 *= inv_cols;
    s2 *= inv_cols;
    typename T::elem* out = dx + i * lddx + 4 * m.t;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      f32x4 g = r.rstd * ((d[k] - s1) - xh[k] * s2);
      if (relu)
#pragma unroll
        for (int u = 0; u < 4; ++u) g[u] = (neg >> (4 * k + u)) & 1u ? 0.f : g[u];
      if constexpr (ALL)
        store4<T>(out + m.offset(k), g);
      else if (in)
        m.template store<T>(out, k, g);
    }
  };
  // (a last group of 1-3 columns: a lane's other columns have another scale)
  const bool whole = !TINY && dx != nullptr && !(Q8 && (unsigned)(cols % kGroup - 1) < 3u);
  const int64_t stride = (int64_t)gridDim.x * kRB;
  const int wave = threadIdx.x >> 6;
  int64_t i0 = (int64_t)blockIdx.x * kRB;
  for (int64_t run = 0; i0 < rows; ++run) {
#pragma unroll
    for (int v = 0; v < NV; ++v) dg[v] = db[v] = f32x4{0.f, 0.f, 0.f, 0.f};
    int32_t n = 0;
    Row r;
    if (whole)
      for (; n < kRun && i0 + kRB <= rows; ++n, i0 += stride) {
        fetch(i0 + sub, r);
        __builtin_amdgcn_sched_barrier(0);
        turn(std::true_type(), r, i0 + sub, n);
      }
    for (; n < kRun && i0 < rows; ++n, i0 += stride) {
      fetch(i0 + sub, r);
      turn(std::false_type(), r, i0 + sub, n);
    }
    if (part == nullptr) continue;
    if constexpr (W > 1) {
      float* pg = part + (run * gridDim.x + blockIdx.x) * 2 * cols;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        m.template store<F32>(pg + 4 * m.t, k, dg[k]);
        m.template store<F32>(pg + cols + 4 * m.t, k, db[k]);
      }
    } else {
      // The wave's rows together, then chunk k of lane t at LDS column 4 (k L + t),
      // whatever row columns it is (those a lane holds for another are zero).
      if (run > 0) __syncthreads();
#pragma unroll
      for (int k = 0; k < NV; ++k) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          float g = dg[k][u], b = db[k][u];
          if constexpr (L < 64) {
            g = half_pair(g, Add());
            b = half_pair(b, Add());
          }
          if constexpr (L < 32) {
            g = row_pair(g, Add());
            b = row_pair(b, Add());
          }
          dg[k][u] = g;
          db[k][u] = b;
        }
        if ((threadIdx.x & 63) < L) {
          *reinterpret_cast<f32x4*>(&red[wave][k * Map::kStep + 4 * m.t]) = dg[k];
          *reinterpret_cast<f32x4*>(&red[kW + wave][k * Map::kStep + 4 * m.t]) = db[k];
        }
      }
      __syncthreads();
      float* pg = part + (int64_t)blockIdx.x * 2 * cols;
      for (int c = threadIdx.x; c < cols; c += kB) {
        // a lane that took the row's last four columns holds column c `back` places on
        const int back = !TINY && c >= (NV - 1) * Map::kStep && (c & ~3) + 4 > cols
                             ? 4 - (cols & 3) : 0;
        float g = 0.f, b = 0.f;
#pragma unroll
        for (int w = 0; w < kW; ++w) {
          g += red[w][c + back];
          b += red[kW + w][c + back];
        }
        if (run == 0 && i0 >= rows) {  // the only run
          pg[c] = g;
          pg[cols + c] = b;
          continue;
        }
        const double g1 = run == 0 ? (double)g : sums[0][c] + (double)g;
        const double b1 = run == 0 ? (double)b : sums[1][c] + (double)b;
        if (i0 < rows) {
          sums[0][c] = g1;
          sums[1][c] = b1;
        } else {
          pg[c] = (float)g1;
          pg[cols + c] = (float)b1;
        }
      }
    }
  }
}

// Sums of the blocks' partial sums, fp64: a block takes 16 of the 2 cols sums, and
// each of 64 groups of 4 lanes every 64th partial of them, then the groups' sums by
// a fixed tree.  Of 256-1536 parts a group adds 4-24, and the chain of dependent loads is
// its time: 4-5 us at up to 1433 columns, 14-25 with 8 groups of 32 lanes.  (Rows that
// take a block leave a part every 64 of them.)
__global__ __launch_bounds__(kB) void k_norm_sum(int32_t cols, int64_t chunks,
                                                 const float* __restrict__ part,
                                                 float* __restrict__ dgamma,
                                                 float* __restrict__ dbeta) {
  constexpr int kG = kB / 4;
  __shared__ double red[kG][16 + 1];
  const int l = threadIdx.x & 3, grp = threadIdx.x >> 2;
  const int idx = blockIdx.x * 16 + 4 * l;
  const int at = min(idx, max(0, 2 * cols - 4));  // (whole loads, inside the row)
  double acc[4] = {0.0, 0.0, 0.0, 0.0};
  auto add = [&](const f32x4 v) {
#pragma unroll
    for (int u = 0; u < 4; ++u) acc[u] += (double)v[u];
  };
  if (cols >= 2) {
    int64_t c = grp;
    for (; c + 7 * kG < chunks; c += 8 * kG) {
      f32x4 v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = load4<F32>(part + (c + u * kG) * 2 * cols + at);
#pragma unroll
      for (int u = 0; u < 8; ++u) add(v[u]);
    }
    for (; c < chunks; c += kG) add(load4<F32>(part + c * 2 * cols + at));
  } else {
    for (int64_t c = grp; c < chunks; c += kG)
      add(f32x4{part[2 * c], part[2 * c + 1], 0.f, 0.f});
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) red[grp][4 * l + u] = acc[u];
  __syncthreads();
  for (int off = kG / 2; off > 0; off >>= 1) {
    if (grp < off)
#pragma unroll
      for (int u = 0; u < 4; ++u) red[grp][4 * l + u] += red[grp + off][4 * l + u];
    __syncthreads();
  }
  if (grp != 0) return;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int k = at + u;  // (the sum this element is of; below idx: another lane's)
    if (k < idx || k >= 2 * cols) continue;
    float* out = k < cols ? dgamma : dbeta;
    if (out != nullptr) out[k < cols ? k : k - cols] = (float)red[0][4 * l + u];
  }
}

// Restoring: 16 lanes a group of 64 columns, kU groups a lane, whose loads are
// issued together: 2449029 x 256 fp32 543 us (5.8 TB/s), x 100 bf16 140-159 (4.7-5.4;
// the same row after row: 15 % more).  (A lane whose four columns reach past the row
// takes the row's last four, as in RowMap; TINY: rows of 1-3 columns.)
constexpr int kU = 4;

struct GroupWalk {  // (row, group) of slot t, then of every 16th slot after it
  int64_t i;
  int32_t g, groups, di, dg;
  __device__ GroupWalk(uint32_t t, int32_t groups_) : groups(groups_) {
    i = t / (uint32_t)groups;
    g = (int32_t)(t - (uint32_t)i * (uint32_t)groups);
    di = 16 / groups;
    dg = 16 - di * groups;
  }
  __device__ void next() {
    i += di;
    g += dg;
    if (g >= groups) {
      g -= groups;
      ++i;
    }
  }
};

template <bool TINY>
struct Quad {  // four columns of a row from `at`, the first `skip` another lane's
  int32_t at, skip, cols;
  __device__ Quad(int32_t c, int32_t cols_) : cols(cols_) {
    at = TINY ? c : min(c, cols - 4);
    skip = min(c - at, 4);
  }
  __device__ bool owns(int u) const { return TINY ? at + u < cols : u >= skip; }
};

template <typename T, bool TINY>
__global__ __launch_bounds__(kB) void k_restore(const int8_t* __restrict__ codes, int64_t ldc,
                                                const float* __restrict__ qscale, int64_t ldq,
                                                int64_t rows, int32_t cols, int32_t groups,
                                                typename T::elem* __restrict__ y, int64_t ldy) {
  const int l = threadIdx.x & 15;
  const GroupWalk start(blockIdx.x * 16 * kU + (threadIdx.x >> 4), groups);
  uint32_t c[kU];
  float step[kU];
  GroupWalk w = start;
#pragma unroll
  for (int n = 0; n < kU; ++n, w.next()) {
    const Quad<TINY> q(w.g * kGroup + 4 * l, cols);
    const int64_t i = w.i < rows ? w.i : rows - 1;
    const int8_t* p = codes + i * ldc + q.at;
    step[n] = qscale[i * ldq + w.g];
    if constexpr (TINY) {
      c[n] = 0;
      for (int u = 0; u < 3; ++u)
        if (q.owns(u)) c[n] |= (uint32_t)(uint8_t)p[u] << (8 * u);
    } else {
      c[n] = load_codes(p);
    }
  }
  w = start;
#pragma unroll
  for (int n = 0; n < kU; ++n, w.next()) {
    if (w.i >= rows) break;
    const Quad<TINY> q(w.g * kGroup + 4 * l, cols);
    const f32x4 x = codes_f32(c[n]) * step[n];
    typename T::elem* p = y + w.i * ldy + q.at;
    if (!TINY && q.skip == 0) {
      store4<T>(p, x);
    } else {
      for (int u = 0; u < 4; ++u)
        if (q.owns(u)) p[u] = (typename T::elem)x[u];
    }
  }
}

inline bigcn_status launched() {
  return hipGetLastError() == hipSuccess ? BIGCN_OK : BIGCN_EHIP;
}

// The layout of a row of `cols` columns: calls f with a RowMap type.  A row is within a
// wave up to 1536 columns, whose lanes hold up to 24 of its columns each: fewer lanes
// with more columns share a row's reductions and divisions among more rows (232965 x
// 602 bf16, 32 lanes of 20 columns against 64 of 12: forward with signs 140 -> 116 us,
// backward from the checkpoint 150 -> 134; 80000 x 1433 f16, 64 lanes of 24 against a
// block of two waves: 110 -> 99, 148 -> 117), but with 32 columns a lane the arrays
// cost more than that (200000 x 512 bf16: 78 -> 90, 98 -> 115), and the backward's with
// 24 where 12 do (300000 x 384 bf16: 125 -> 134).
template <bool GRAD, typename F>
void with_map(int32_t cols, F f) {
  if (cols < 4) return f(RowMap<1, 16, 1, true>(Shape{}));
  if (cols <= 64) return f(RowMap<1, 16, 1>(Shape{}));
  if (cols <= 128) return f(RowMap<1, 16, 2>(Shape{}));
  if (cols <= 192) return f(RowMap<1, 16, 3>(Shape{}));
  if (cols <= 256) return f(RowMap<1, 16, 4>(Shape{}));
  if (cols <= 320) return f(RowMap<1, 16, 5>(Shape{}));
  if (cols <= 384) return f(RowMap<1, 32, 3>(Shape{}));
  if (cols <= 512) return f(RowMap<1, 32, 4>(Shape{}));
  if (cols <= 640) return f(RowMap<1, 32, 5>(Shape{}));
  if constexpr (GRAD) {
    if (cols <= 768) return f(RowMap<1, 64, 3>(Shape{}));
  } else {
    if (cols <= 768) return f(RowMap<1, 32, 6>(Shape{}));
  }
  if (cols <= 1024) return f(RowMap<1, 64, 4>(Shape{}));
  if (cols <= 1280) return f(RowMap<1, 64, 5>(Shape{}));
  if (cols <= 1536) return f(RowMap<1, 64, 6>(Shape{}));
  if (cols <= 2048) return f(RowMap<2, 64, 4>(Shape{}));
  if (cols <= 3072) return f(RowMap<4, 64, 3>(Shape{}));
  if (cols <= 4096) return f(RowMap<4, 64, 4>(Shape{}));
  if (cols <= 6144) return f(RowMap<8, 64, 3>(Shape{}));
  return f(RowMap<8, 64, 4>(Shape{}));
}

// The backward's blocks and the sets of partial sums they leave.  What the card reads
// fastest is about 7 MB of loads at a time, in whole blocks a CU: more in flight spread
// over more of memory and cost bandwidth.  2449029 x 256 fp32 from the checkpoint,
// 21 KB of loads a turn: 1028 us with 256 blocks, 1075 with 512, 1107 with 768-2048 (and
// 1100-1150 where each block took a stretch of rows of its own); 900000 x 128 bf16,
// 8.2 KB: 230, 143, 131, 136, 151 with 256, 512, 768, 1024, 1536.  16-bit types have twice
// the arithmetic for their bytes and need two blocks a CU (80000 x 1433 f16: 155 us with
// 256 blocks, 135 with 512), waves that wait for one another some more loads (60000 x
// 2048 bf16 from the checkpoint, 6.1 KB: 171, 137, 123 with 768, 1024, 1536).
struct GradPlan {
  int64_t blocks, partials;
};
GradPlan grad_plan(int64_t rows, int32_t cols, int es, bool q8) {
  int64_t at_once = 1;  // rows a block holds
  with_map<true>(cols, [&](auto m) {
    typedef decltype(m) M;
    at_once = M::kWaves > 1 ? 1 : kW * M::kRows;
  });
  const int64_t turns = (rows + at_once - 1) / at_once;
  const int64_t bytes = at_once * cols * (q8 ? es + 1 : 2 * es);  // read in a turn of a block
  const int64_t per_cu = std::min<int64_t>(
      at_once > 1 ? 4 : 6,
      std::max<int64_t>(es == 2 ? 2 : 1,
                        ((at_once > 1 ? 7000000 : 9000000) / 256 + bytes / 2) / bytes));
  GradPlan p;
  p.blocks = std::min<int64_t>(turns, 256 * per_cu);
  // (where every run leaves sums: in the last ones only the blocks that have rows left)
  const int64_t runs = p.blocks == 0 ? 0 : turns / (kRun * p.blocks);
  p.partials = at_once > 1 ? p.blocks
                           : runs * p.blocks + std::min(p.blocks, turns - runs * kRun * p.blocks);
  return p;
}

constexpr int64_t kMaxRows = INT32_MAX;      // of the norm (its workspace grows with them)
constexpr int64_t kMaxThreads = UINT32_MAX;  // of a launch

template <typename T, bool NORM>
void launch_norm(const typename T::elem* x, int64_t ldx, int64_t rows, int32_t cols,
                 const float* gamma, const float* beta, float eps, const NormOut& o,
                 hipStream_t s) {
  with_map<false>(cols, [&](auto m) {
    typedef decltype(m) M;
    constexpr int kRB = M::kWaves > 1 ? 1 : kW * M::kRows;
    // A block takes turns until it has read kBytes, so most launch many more blocks than
    // run at once: on 2449029 x 256 fp32 blocks of one turn reach 5.4-5.9 TB/s, 2048
    // blocks of 75 turns 4.7; on 232965 x 602 bf16, 4.8 KB a turn, blocks of 4 turns 5.0
    // and of one 4.1 (each loads gamma and beta first: a whole row of both where a row
    // takes a block, hence twice the bytes).  But at least 1024 blocks while there are
    // rows: 2708 x 64, 4 KB a turn, takes 4.0 us in 170 blocks and 6.4 in 43.
    constexpr int64_t kBytes = M::kWaves > 1 ? 32768 : 16384;
    const int64_t turns = (rows + kRB - 1) / kRB, turn = (int64_t)kRB * cols * sizeof(*x);
    const int64_t each =
        std::max<int64_t>(1, std::min<int64_t>((kBytes + turn - 1) / turn, turns / 1024));
    constexpr int kThreads = 64 * (M::kWaves > 1 ? M::kWaves : kW);
    const int64_t blocks = std::min((turns + each - 1) / each, kMaxThreads / kThreads);
    hipLaunchKernelGGL((k_norm<T, M::kWaves, M::kL, M::kNV, M::kTiny, NORM>),
                       dim3((unsigned)blocks), dim3(kThreads), 0, s, x, ldx, rows, cols, gamma,
                       beta, eps, o);
  });
}

}  // namespace

extern "C" {

bigcn_status bigcn_checkpoint_q8(const void* x, bigcn_dtype xtype, int64_t rows, int32_t cols,
                                 int64_t ldx, int8_t* codes, int64_t ldc, float* qscale,
                                 int64_t ldq, void* stream) {
  if (!dtype_ok(xtype) || rows < 0 || cols < 1 || ldx < cols || ldc < cols ||
      ldq < words(cols))
    return BIGCN_EINVAL;
  if (rows > 0 && (x == nullptr || codes == nullptr || qscale == nullptr)) return BIGCN_EINVAL;
  if (!aligned(x, dtype_size(xtype)) || !aligned(qscale, 4)) return BIGCN_EALIGN;
  if (rows == 0) return BIGCN_OK;
  with_type(xtype, [&](auto t) {
    typedef decltype(t) T;
    // up to kMaxRowCols columns at a time (whole groups)
    for (int64_t c = 0; c < cols; c += kMaxRowCols) {
      const NormOut o = {nullptr, 0, nullptr, nullptr, codes + c, ldc, qscale + c / kGroup, ldq,
                         nullptr, 0, nullptr, 0, nullptr};
      launch_norm<T, false>((const typename T::elem*)x + c, ldx, rows,
                            (int32_t)std::min<int64_t>(cols - c, kMaxRowCols), nullptr, nullptr, 1.f, o,
                            (hipStream_t)stream);
    }
  });
  return launched();
}

bigcn_status bigcn_restore_q8(const int8_t* codes, int64_t ldc, const float* qscale,
                              int64_t ldq, int64_t rows, int32_t cols, void* y,
                              bigcn_dtype ytype, int64_t ldy, void* stream) {
  if (!dtype_ok(ytype) || rows < 0 || cols < 1 || ldy < cols || ldc < cols ||
      ldq < words(cols))
    return BIGCN_EINVAL;
  if (rows > 0 && (y == nullptr || codes == nullptr || qscale == nullptr)) return BIGCN_EINVAL;
  if (!aligned(y, dtype_size(ytype)) || !aligned(qscale, 4)) return BIGCN_EALIGN;
  with_type(ytype, [&](auto t) {
    typedef decltype(t) T;
    auto k = cols < 4 ? k_restore<T, true> : k_restore<T, false>;
    // as many rows at a time as one launch has threads for
    const int64_t groups = words(cols), most = kMaxThreads / kB * 16 * kU / groups;
    for (int64_t i = 0; i < rows; i += most) {
      const int64_t part = std::min(rows - i, most);
      hipLaunchKernelGGL(k, dim3((unsigned)((part * groups + 16 * kU - 1) / (16 * kU))), dim3(kB),
                         0, (hipStream_t)stream, codes + i * ldc, ldc, qscale + i * ldq, ldq, part,
                         cols, (int32_t)groups, (typename T::elem*)y + i * ldy, ldy);
    }
  });
  return launched();
}

bigcn_status bigcn_layernorm(const void* x, bigcn_dtype xtype, int64_t rows, int32_t cols,
                             int64_t ldx, const float* gamma, const float* beta, float eps,
                             void* y, int64_t ldy, float* mean, float* rstd, int8_t* codes,
                             int64_t ldc, float* qscale, int64_t ldq, const int64_t* rowptr,
                             bigcn_norm norm, uint64_t* bits, int64_t ldw, float* scale,
                             void* stream) {
  if (!dtype_ok(xtype) || rows < 0 || cols < 1 || ldx < cols) return BIGCN_EINVAL;
  if (norm != BIGCN_NORM_SYM && norm != BIGCN_NORM_MEAN) return BIGCN_EINVAL;
  if (!(eps >= FLT_MIN) || !isfinite(eps)) return BIGCN_EINVAL;
  if (rows > 0 && x == nullptr) return BIGCN_EINVAL;
  if ((codes == nullptr) != (qscale == nullptr) || (bits == nullptr) != (scale == nullptr))
    return BIGCN_EINVAL;
  if ((y != nullptr && ldy < cols) || (codes != nullptr && (ldc < cols || ldq < words(cols))) ||
      (bits != nullptr && ldw < words(cols)))
    return BIGCN_EINVAL;
  if (rows > 0 && y == nullptr && mean == nullptr && rstd == nullptr && codes == nullptr &&
      bits == nullptr)
    return BIGCN_EINVAL;
  if (y == x && y != nullptr && ldy != ldx) return BIGCN_EINVAL;
  if (!aligned(x, dtype_size(xtype)) || !aligned(y, dtype_size(xtype)) || !aligned(gamma, 4) ||
      !aligned(beta, 4) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(qscale, 4) ||
      !aligned(rowptr, 8) || !aligned(bits, 8) || !aligned(scale, 4))
    return BIGCN_EALIGN;
  if (cols > kMaxRowCols || rows > kMaxRows) return BIGCN_EUNSUPPORTED;
  if (rows == 0) return BIGCN_OK;
  const NormOut o = {y, ldy, mean, rstd, codes, ldc, qscale, ldq, rowptr,
                     norm == BIGCN_NORM_SYM, bits, ldw, scale};
  with_type(xtype, [&](auto t) {
    typedef decltype(t) T;
    launch_norm<T, true>((const typename T::elem*)x, ldx, rows, cols, gamma, beta, eps, o,
                         (hipStream_t)stream);
  });
  return launched();
}

size_t bigcn_layernorm_backward_workspace_bytes(int64_t rows, int32_t cols) {
  if (rows < 0 || rows > kMaxRows || cols < 1 || cols > kMaxRowCols) return 0;
  int64_t partials = 0;  // of any type and source
  for (int es : {2, 4})
    for (bool q8 : {false, true})
      partials = std::max(partials, grad_plan(rows, cols, es, q8).partials);
  return up256((size_t)partials * 2 * cols * 4);
}

bigcn_status bigcn_layernorm_backward(const void* dy, bigcn_dtype dtype, int64_t rows,
                                      int32_t cols, int64_t lddy, const void* x, int64_t ldx,
                                      const int8_t* codes, int64_t ldc, const float* qscale,
                                      int64_t ldq, const float* mean, const float* rstd,
                                      const float* gamma, bigcn_act act, void* dx,
                                      int64_t lddx, float* dgamma, float* dbeta,
                                      void* workspace, size_t ws_bytes, void* stream) {
  if (!dtype_ok(dtype) || rows < 0 || cols < 1 || lddy < cols) return BIGCN_EINVAL;
  if (act != BIGCN_ACT_NONE && act != BIGCN_ACT_RELU) return BIGCN_EINVAL;
  if (rows > 0 && (dy == nullptr || mean == nullptr || rstd == nullptr)) return BIGCN_EINVAL;
  if ((codes == nullptr) != (qscale == nullptr) || (x != nullptr && codes != nullptr) ||
      (rows > 0 && x == nullptr && codes == nullptr))
    return BIGCN_EINVAL;
  if ((x != nullptr && ldx < cols) || (codes != nullptr && (ldc < cols || ldq < words(cols))) ||
      (dx != nullptr && lddx < cols) || (dx == dy && dx != nullptr && lddx != lddy))
    return BIGCN_EINVAL;
  if (dx == nullptr && dgamma == nullptr && dbeta == nullptr) return BIGCN_EINVAL;
  const size_t es = dtype_size(dtype);
  if (!aligned(dy, es) || !aligned(x, es) || !aligned(dx, es) || !aligned(qscale, 4) ||
      !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(gamma, 4) || !aligned(dgamma, 4) ||
      !aligned(dbeta, 4))
    return BIGCN_EALIGN;
  if (cols > kMaxRowCols || rows > kMaxRows) return BIGCN_EUNSUPPORTED;
  const bool sums = dgamma != nullptr || dbeta != nullptr;
  if (sums && rows > 0) {
    if (workspace == nullptr || ws_bytes < bigcn_layernorm_backward_workspace_bytes(rows, cols))
      return BIGCN_EWORKSPACE;
    if (!aligned(workspace, 256)) return BIGCN_EALIGN;
  }
  hipStream_t s = (hipStream_t)stream;
  const GradPlan p = grad_plan(rows, cols, (int)es, codes != nullptr);
  float* part = sums ? (float*)workspace : nullptr;
  const int relu = act == BIGCN_ACT_RELU ? 1 : 0;
  if (rows > 0)
    with_type(dtype, [&](auto t) {
      typedef decltype(t) T;
      typedef typename T::elem E;
      const Kept<T> kept = {(const E*)x, ldx, codes, ldc, qscale, ldq};
      with_map<true>(cols, [&](auto m) {
        typedef decltype(m) M;
        const dim3 grid((unsigned)p.blocks), block(64 * (M::kWaves > 1 ? M::kWaves : kW));
        if (codes != nullptr)
          hipLaunchKernelGGL((k_norm_grad<T, true, M::kWaves, M::kL, M::kNV, M::kTiny>), grid, block,
                             0, s, (const E*)dy, lddy, rows, cols, kept, mean, rstd, gamma, relu,
                             (E*)dx, lddx, part);
        else
          hipLaunchKernelGGL((k_norm_grad<T, false, M::kWaves, M::kL, M::kNV, M::kTiny>), grid,
                             block, 0, s, (const E*)dy, lddy, rows, cols, kept, mean, rstd, gamma,
                             relu, (E*)dx, lddx, part);
      });
    });
  if (sums)
    hipLaunchKernelGGL(k_norm_sum, dim3((unsigned)((2 * cols + 15) / 16)), dim3(kB), 0, s, cols,
                       p.partials, part, dgamma, dbeta);
  return launched();
}

}  // extern "C"
