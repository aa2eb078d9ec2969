// The head's losses (include/vla_loss.h): cross entropy of tokens and distillation from a teacher's top logits, with their
// gradients.  Both are one thing: a row's target is a short sorted list of (id, probability), one entry for a token.
//
// Mathematics.  With z = h W^T / tau, a group of 64 columns of a row leaves m = max z and l = sum exp(z - m), the groups are joined
// in a fixed order, and
//     lse = m + log l,   loss = log l + (m - z_label)   (lists: sum p log p + (sum p) lse - sum p z).
// float32 carries t = l - 1, the sum without the largest, in place of l: a row that is sure of its token has nothing but t.
// The gradient forms z again, dz = q - r with q = exp(z - lse), and two products: grad_hidden = (g / tau) dz W, where a row's
// coefficient is applied at the end, and grad_head = dz^T (g h / tau), where it is applied to h.
//
// All products run on the half-precision kernel of gemm_tile.h.  Powers of two keep operands in the range of half precision: a
// row of h is scaled to a maximum in [2^13, 2^14) (exact for bfloat16), W by 2^8 (exact, as in the arena), dz, which lies in
// [-1, 1], by 2^15 for grad_hidden, whose rows take their g / tau at the end, and times g / tau over the row's scale as one tensor
// to a maximum of 2^15 for grad_head.  dz is rounded to half precision (2^-11 of its value at most, or 2^-40, for
// grad_head 2^-38 of the largest row's g h, where that is more: below the normal numbers); everything else is float32.
// float32 operands are carried as two terms hi + lo (22 bits); a product of two of them is three, hi hi + lo hi + hi lo,
// laid out as one contraction three times as long: [lo | hi | hi] against [hi | lo | hi], the small products first, so that their
// sums are rounded at their own size.
//
// What bounds them: the large calls by the matrix cores (2 T V d operations forward, 6 backward: 8192 rows of 32000 x 4096 1.36
// PFLOP/s forward in all, 1.31 backward, where a library's plain product of 8192^3 reaches 1.23), few rows by reading the head (once
// forward; twice and written once backward), the smallest by three to six launches of 4 to 10 us each.  The logits are never
// written: a tile's statistics, or its dz, are formed from the accumulators.  Keeping dz rather than forming z a second time for each
// product costs 2 T V bytes each way instead of 2 T V d operations.
#include "gemm_tile.h"
#include "../../include/vla_loss.h"

namespace vla {

constexpr float kDzScale = 32768.0f;
constexpr float kLog2e = 1.44269504088896341f;
constexpr int kGroup = 64;                 // columns of a group of partial statistics
constexpr int kMaxTop = 1024;

// ---- targets -------------------------------------------------------------------------------------------------
// What an epilogue needs to know of the rows.
struct RowTargets {
  const float* z_scale;        // [T] from accumulated products to z; 0: the row has no target
  const int32_t* label;        // [T] token, or nullptr: lists
  const int32_t* ids;          // [T][k] ascending, no two equal
  const float* p;              // [T][k]
  const unsigned short* first; // [T][groups + 1] entry that begins each group of columns
  int k, groups;
  // The entries of N - 1 groups of row m, from group g on, begin at at[0] .. (groups past the last have none).
  template <int N>
  __device__ __forceinline__ void entries(int m, int g, int (&at)[N]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) at[i] = first[(size_t)m * (groups + 1) + min(g + i, groups)];
  }
  // use(e, id, probability) of entries from .. to - 1 of row m, four requested at a time (one after the other each would wait for
  // its own loads, which use()'s stores keep behind them).
  template <class Use>
  __device__ __forceinline__ void each(int m, int from, int to, Use&& use) const {
    for (int e = from; e < to; e += 4) {
      int id[4];
      float pr[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const size_t at = (size_t)m * k + min(e + j, to - 1);
        id[j] = ids[at];
        pr[j] = p[at];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (e + j < to) use(e + j, id[j], pr[j]);
    }
  }
};

template <class T> struct Vec;
template <> struct Vec<float> { typedef f32x4 type; static constexpr int n = 4; };
template <> struct Vec<bf16> { typedef bf16x8 type; static constexpr int n = 8; };

// The exponent e for which |x| * 2^e lies in [2^13, 2^14), within [-60, 60]; 0 for 0 and what is not finite.
__device__ __forceinline__ int scale_exponent(float x) {
  if (!(x > 0.f) || x == INFINITY) return 0;
  int e;
  (void)frexpf(x, &e);                     // x = f 2^e, f in [1/2, 1)
  return max(-60, min(60, 14 - e));
}

// The largest of n values to the first of them (a launch of its own for what every wave of the products would have to read).
__global__ __launch_bounds__(256) void loss_max_kernel(float* __restrict__ v, int n) {
  __shared__ float red[4];
  float m = 0.f;
  for (int i = threadIdx.x; i < n; i += 256) m = fmaxf(m, v[i]);
  m = wave_max(m);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
  __syncthreads();
  if (threadIdx.x == 0) v[0] = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}
// 2^x that brings the largest of n values into [1/2, 1); the same in every wave.
__device__ __forceinline__ int max_exponent(const float* v, int n, int lane) {
  float m = 0.f;
  for (int i = lane; i < n; i += 64) m = fmaxf(m, v[i]);
  m = wave_max(m);
  if (!(m > 0.f)) return 0;
  int e;
  (void)frexpf(m, &e);
  return max(-120, min(120, -e));
}

// ---- operands in fragment order ---------------------------------------------------------------------------------
// What brings the sums of grad_head back.
__device__ __forceinline__ float head_scale(const float* dz_max, int n, int lane) {
  return ldexpf(1.0f / kDzScale, -max_exponent(dz_max, n, lane));
}

// The head where it is not read as it is: 64 x 64 elements of src [R, C] by 256 threads, as rows (F [Rp, Cp], contraction over
// the columns) and transposed (FT [Cp, Rp], or nullptr), zeros past R and C.  TERMS 3: [hi | lo | hi], a third of the contraction
// each.
template <class T>
struct HeadPack {
  const T* src;
  int64_t ld;
  int R, C, Rp, Cp;
  f16 *F, *FT;
};
template <class T, int TERMS>
__device__ __forceinline__ void pack_tile(const HeadPack<T>& h, int tile_id, int t, float (&tile)[64][65]) {
  const int across = h.Cp / 64, r0 = tile_id / across * 64, c0 = tile_id % across * 64;    // (r0 >= Rp: nothing)
  const int r = r0 + (t >> 2), c = c0 + (t & 3) * 16;
  float v[16];
#pragma unroll
  for (int i = 0; i < 16; i += Vec<T>::n) {
    typename Vec<T>::type x;
    const bool in = r < h.R && c + i < h.C;
    if (in) x = *(const typename Vec<T>::type*)(h.src + (size_t)r * h.ld + c + i);
#pragma unroll
    for (int j = 0; j < Vec<T>::n; ++j) v[i + j] = in ? (float)x[j] * kWeightScale : 0.f;
  }
  auto put = [&](f16* dst, int m, int kk, int third, const float* x) {      // 8 elements of a row, from k kk on
    f16x8 hi;
#pragma unroll
    for (int j = 0; j < 8; ++j) hi[j] = from_f32<f16>(x[j]);
    *(f16x8*)(dst + act_index(m, kk, TERMS * third)) = hi;
    if constexpr (TERMS == 3) {
      f16x8 lo;
#pragma unroll
      for (int j = 0; j < 8; ++j) lo[j] = from_f32<f16>(x[j] - (float)hi[j]);
      *(f16x8*)(dst + act_index(m, third + kk, 3 * third)) = lo;
      *(f16x8*)(dst + act_index(m, 2 * third + kk, 3 * third)) = hi;
    }
  };
  if (r < h.Rp) {
    put(h.F, r, c, h.Cp, v);
    put(h.F, r, c + 8, h.Cp, v + 8);
  }
  if (h.FT) {
#pragma unroll
    for (int j = 0; j < 16; ++j) tile[t >> 2][(t & 3) * 16 + j] = v[j];
    __syncthreads();
    const int col = t & 63, rr = (t >> 6) * 16;
    if (r0 + rr < h.Rp) {
      float x[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) x[j] = tile[rr + j][col];
      put(h.FT, c0 + col, r0 + rr, h.Rp, x);
      put(h.FT, c0 + col, r0 + rr + 8, h.Rp, x + 8);
    }
  }
}
template <class T, int TERMS>
__global__ __launch_bounds__(256) void loss_pack_kernel(HeadPack<T> head) {
  __shared__ float tile[64][65];
  pack_tile<T, TERMS>(head, blockIdx.x, threadIdx.x, tile);
}

struct RowsOut {
  float *z_scale, *coef, *dz_coef, *dz_max;    // [T], with a gradient also g / tau, that over the row's scale, [Tp / 8] maxima of it
  int32_t* label;                              // labels, -1 where there is no target
  int32_t* ids;                                // lists; sum p log p and sum p of a row
  float *p, *ent, *mass;
  unsigned short* first;
  f16 *F, *FT;                                 // h in fragment order: rows [Tp, dP], and transposed [dP, Tp] (or nullptr)
};

// Eight rows a workgroup, a wave each: the row's target and scale, then its h as operands; of few rows `splits` workgroups, which
// take the chunks of columns in turn (each finds the scale for itself: 448 rows of 4096 11.4 -> 8.8 us).  The workgroups behind
// those of the rows pack the head (two tiles each), where a call packs it in one piece: a launch less.  Bound by its chain of
// latencies (5 to 9 us), and of thousands of rows by what it moves (8192 x 4096 36 us, 3.7 TB/s); a head of 32000 x 4096 packed both
// ways 136 us with 2048 rows, 5.8 TB/s.
constexpr int kRowsChunk = 1024;               // columns at a time
constexpr int kRowsHeld = 4096;
template <class T, int TERMS>
__global__ __launch_bounds__(512) void loss_rows_kernel(const T* __restrict__ h, int64_t ld, int Tn, int d, int V, float inv_tau,
                                                        const int32_t* __restrict__ labels, const float* __restrict__ top_logits,
                                                        const int32_t* __restrict__ top_ids, int k, int groups,
                                                        const float* __restrict__ g, int Tp, int dP, int splits, RowsOut out,
                                                        HeadPack<T> head) {
  constexpr int PITCH = kRowsChunk + 8;
  __shared__ union {
    __attribute__((aligned(16))) f16 row[TERMS == 3 ? 2 : 1][8 * PITCH];
    float head[2][64][65];
  } s_tile;
  __shared__ float s_max[8];
  if ((int)blockIdx.x >= Tp / 8 * splits) {
    const int half = threadIdx.x >> 8;
    pack_tile<T, TERMS>(head, ((int)blockIdx.x - Tp / 8 * splits) * 2 + half, threadIdx.x & 255, s_tile.head[half]);
    return;
  }
  auto& tile = s_tile.row;
  extern __shared__ __attribute__((aligned(16))) int32_t lists[];     // [8 rows][ids | keys | p], kp entries each
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row0 = (int)blockIdx.x / splits * 8, row = row0 + wave, split = (int)blockIdx.x % splits;
  const bool first = split == 0;               // (what there is one of for a row)
  int32_t target = -1;                         // the label, or the lane's first entry
  float first_logit = 0.f;
  if (row < Tn) {
    if (labels) target = labels[row];
    else if (lane < k) target = top_ids[(size_t)row * k + lane], first_logit = top_logits[(size_t)row * k + lane];
  }
  // A row of up to kRowsHeld columns is requested at once and stays in registers.
  constexpr int N = Vec<T>::n, HELD = kRowsHeld / (64 * N);
  typedef typename Vec<T>::type X;
  const T* x = h + (size_t)row * ld;
  const bool held = d <= kRowsHeld;
  X xv[HELD] = {};
  if (held && row < Tn) {
#pragma unroll
    for (int u = 0; u < HELD; ++u)
      if ((u * 64 + lane) * N < d) xv[u] = *(const X*)(x + (u * 64 + lane) * N);
  }
  const float g_row = g && row < Tn ? g[row] : 0.f;
  bool live = row < Tn;
  if (!live) {
  } else if (labels) {
    live = target >= 0 && target < V;
    if (lane == 0 && first) out.label[row] = live ? target : -1;
  } else if (!first) {
    bool any = target >= 0 && target < V && first_logit != -INFINITY;
    for (int j = lane + 64; j < k; j += 64) {
      const int32_t id = top_ids[(size_t)row * k + j];
      any = any || (id >= 0 && id < V && top_logits[(size_t)row * k + j] != -INFINITY);
    }
    live = __any(any);
  } else {
    const int kp = (k + 3) & ~3;
    int32_t *s_id = lists + wave * 3 * kp, *s_key = s_id + kp;
    float* s_p = (float*)(s_key + kp);
    float m = -INFINITY;
    for (int j = lane; j < kp; j += 64) {
      int32_t id = -1;
      float l = 0.f;
      if (j < k) {
        id = j < 64 ? target : top_ids[(size_t)row * k + j];
        l = j < 64 ? first_logit : top_logits[(size_t)row * k + j];
        if (id < 0 || id >= V || l == -INFINITY) id = -1;
      }
      s_id[j] = id;
      s_p[j] = l;
      if (id >= 0) m = fmaxf(m, l);
    }
    m = wave_max(m);
    m = m == -INFINITY ? 0.f : m;                                    // (all NaN, or none)
    float sum = 0.f;
    for (int j = lane; j < kp; j += 64) {
      const float e = s_id[j] >= 0 ? expf((s_p[j] - m) * inv_tau) : 0.f;   // (the difference first: no logit overflows)
      s_p[j] = e;
      sum += e;
    }
    sum = wave_sum(sum);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __builtin_amdgcn_wave_barrier();
    // equal ids: the first of them stands for all, with its id as key; its place is the number of smaller keys
    typedef __attribute__((ext_vector_type(4))) int i32x4;
    constexpr int kNone = 0x7fffffff;
    for (int j = lane; j < kp; j += 64) {
      const int id = s_id[j];
      bool lead = id >= 0;
      for (int i = 0; i < kp; i += 4) {
        const i32x4 o = *(const i32x4*)(s_id + i);
#pragma unroll
        for (int u = 0; u < 4; ++u) lead = lead && !(o[u] == id && i + u < j);
      }
      s_key[j] = lead ? id : kNone;
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __builtin_amdgcn_wave_barrier();
    float ent = 0.f, mass = 0.f;
    int n = 0;
    for (int j = lane; j < kp; j += 64) {
      const int id = s_key[j];
      int at = 0;
      float p = 0.f;
      for (int i = 0; i < kp; i += 4) {
        const i32x4 o = *(const i32x4*)(s_id + i), ky = *(const i32x4*)(s_key + i);
        const f32x4 e = *(const f32x4*)(s_p + i);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          at += ky[u] < id;
          p += o[u] == id ? e[u] : 0.f;
        }
      }
      if (id != kNone) {
        p /= sum;
        out.ids[(size_t)row * k + at] = id;
        out.p[(size_t)row * k + at] = p;
        if (p != 0.f) ent += p * logf(p);
        mass += p;
        ++n;
      }
    }
    ent = wave_sum(ent);
    mass = wave_sum(mass);
    n = (int)wave_sum((float)n);
    live = n > 0;
    if (lane == 0) {
      out.ent[row] = ent;
      out.mass[row] = mass;
    }
    for (int b = lane; b <= groups; b += 64) {                       // first entry of id 64 b and more
      int at = 0;
      for (int i = 0; i < kp; i += 4) {
        const i32x4 ky = *(const i32x4*)(s_key + i);
#pragma unroll
        for (int u = 0; u < 4; ++u) at += ky[u] < b * kGroup;
      }
      out.first[(size_t)row * (groups + 1) + b] = (unsigned short)at;
    }
  }
  float mx = 0.f;
  auto max_of = [&](const X& v) {
#pragma unroll
    for (int j = 0; j < N; ++j) mx = fmaxf(mx, fabsf((float)v[j]));
  };
  if (live) {
    if (held) {
#pragma unroll
      for (int u = 0; u < HELD; ++u) max_of(xv[u]);
    } else {
      for (int i = lane * N; i < d; i += 64 * N) max_of(*(const X*)(x + i));
    }
  }
  mx = wave_max(mx);
  const int e = live ? scale_exponent(mx) : 0;
  const float scale = live ? ldexpf(1.0f, e) : 0.f;
  float top = 0.f;
  if (lane == 0 && row < Tn && first) {
    out.z_scale[row] = live ? ldexpf(inv_tau / kWeightScale, -e) : 0.f;
    if (g) {
      const float c = live ? g_row * inv_tau : 0.f, s = ldexpf(c, -e);
      out.coef[row] = c;
      out.dz_coef[row] = s;
      top = fabsf(s) < INFINITY ? fabsf(s) : 0.f;
    }
  }
  if (lane == 0) s_max[wave] = top;
  __syncthreads();
  if (g && threadIdx.x == 0 && first) {
    float t = s_max[0];
    for (int i = 1; i < 8; ++i) t = fmaxf(t, s_max[i]);
    out.dz_max[row0 / 8] = t;
  }
  bool again = false;
  auto chunk = [&](int c0, auto U) __attribute__((always_inline)) {
    constexpr int u0 = decltype(U)::value;                           // the chunk's first register, -1: read again
    const int n = min(kRowsChunk, dP - c0);
    if (again) __syncthreads();
    again = true;
#pragma unroll
    for (int u = 0; u < kRowsChunk / (64 * N); ++u) {
      const int i = (u * 64 + lane) * N;
      if (i >= n) break;
      X v{};
      if constexpr (u0 >= 0) v = xv[u0 + u];
      else if (live && c0 + i < d) v = *(const X*)(x + c0 + i);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float y = live ? (float)v[j] * scale : 0.f;
        const f16 hi = from_f32<f16>(y);
        tile[0][wave * PITCH + i + j] = hi;
        if constexpr (TERMS == 3) tile[1][wave * PITCH + i + j] = from_f32<f16>(y - (float)hi);
      }
    }
    __syncthreads();
    const int ldF = TERMS * dP, ldT = TERMS * Tp;
    for (int i = threadIdx.x; i < n; i += 512) {                     // rows: 8 of a chunk of 8 columns side by side
      const int r = i & 7, c = i & ~7;
      const f16x8 hi = *(const f16x8*)(&tile[0][r * PITCH + c]);
      *(f16x8*)(out.F + act_index(row0 + r, (TERMS - 1) * dP + c0 + c, ldF)) = hi;
      if constexpr (TERMS == 3) {
        *(f16x8*)(out.F + act_index(row0 + r, c0 + c, ldF)) = *(const f16x8*)(&tile[TERMS == 3][r * PITCH + c]);
        *(f16x8*)(out.F + act_index(row0 + r, dP + c0 + c, ldF)) = hi;
      }
    }
    if (out.FT)
      for (int i = threadIdx.x; i < n; i += 512) {                   // columns: their 8 rows
        f16x8 hi, lo;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          hi[r] = tile[0][r * PITCH + i];
          if constexpr (TERMS == 3) lo[r] = tile[TERMS == 3][r * PITCH + i];
        }
        *(f16x8*)(out.FT + act_index(c0 + i, row0, ldT)) = hi;
        if constexpr (TERMS == 3) {
          *(f16x8*)(out.FT + act_index(c0 + i, Tp + row0, ldT)) = lo;
          *(f16x8*)(out.FT + act_index(c0 + i, 2 * Tp + row0, ldT)) = hi;
        }
      }
  };
  if (held)
    static_for<kRowsHeld / kRowsChunk>([&](auto I) __attribute__((always_inline)) {
      constexpr int c0 = decltype(I)::value * kRowsChunk;
      if (c0 < dP && decltype(I)::value % splits == split) chunk(c0, std::integral_constant<int, c0 / (64 * N)>{});
    });
  else
    for (int c0 = split * kRowsChunk; c0 < dP; c0 += splits * kRowsChunk) chunk(c0, std::integral_constant<int, -1>{});
}

// ---- epilogues -----------------------------------------------------------------------------------------------
// Partial statistics of the groups of 64 columns.  ROWS rows of a group by 64 / ROWS lanes each; a group's sums are formed in
// the same order whatever the tile.  What rows hold does not reach the rows beside them (their number picks the tile and the
// slices, by which sums of products may be rounded otherwise).
// Bound by the matrix cores: 8192 x 32000 x 4096 1.5 ms, 1.43 PFLOP/s (256x256 tiles); with d 768 by this epilogue too (2301 rows 114
// us, 0.99); one row by reading the head as it is (40 us, 6.5 TB/s, a part of it from the last-level cache).
// EXACT (float32): t in place of l, from differences to the largest that are exact where they are small.
template <int RAW, bool EXACT>
struct EpiStats {
  static constexpr int kSpan = 64, kRaw = RAW;
  RowTargets tg;
  float *pm, *pl;            // [groups][T] m and l (t) of a group
  float* pa;                 // z of the label [T], or p z of the entries [T][k]
  int T, V, n_base;          // first column of the launch
  int64_t raw_ld;
  int raw_rows;
  template <int COLS, int PITCH, int ROWS>
  __device__ __forceinline__ void consume(const float* tile, int m_base, int nb, int lane, int M) const {
    constexpr int PARTS = 64 / ROWS, W = kGroup / PARTS;
    static_assert(COLS % kGroup == 0 && W % 16 == 0 && W <= 32, "whole groups, sums of 16 or of two of them a lane");
    const int r = lane % ROWS, part = lane / ROWS, m = m_base + r, mc = min(m, M - 1);
    const float zs = tg.z_scale[mc];
    const int label = tg.label ? tg.label[mc] : -1;
    int entry[COLS / kGroup + 1];                        // where the groups' entries begin
    if (!tg.label) tg.entries(mc, (n_base + nb) / kGroup, entry);
#pragma unroll
    for (int gg = 0; gg < COLS / kGroup; ++gg) {
      const int n0 = n_base + nb + gg * kGroup, c0 = gg * kGroup + part * W, left = V - n0 - part * W;
      float x[W];
#pragma unroll
      for (int i = 0; i < W; i += 4) *(f32x4*)(x + i) = *(const f32x4*)(tile + r * PITCH + c0 + i);
      // An infinite weight makes infinite products, which as -inf would count as probabilities of 0: a NaN then.
      float mn = INFINITY;
#pragma unroll
      for (int i = 0; i < W; ++i) mn = fminf(mn, x[i]);
      if (n0 + kGroup > V) {                             // (uniform) the last group
#pragma unroll
        for (int i = 0; i < W; ++i) x[i] = i < left ? x[i] : -INFINITY;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < W; ++i) mx = fmaxf(mx, x[i]);
      mx = lanes_max<ROWS, 32>(mx);
      const float z2 = zs * kLog2e, ref = mx == -INFINITY ? 0.f : mx, ref2 = -ref * z2;
      float l = 0.f;                                     // sums of 16 columns, joined in pairs
      int ties = 0;                                      // of the largest
#pragma unroll
      for (int h = 0; h < W / 16; ++h) {
        float s4[4] = {};
#pragma unroll
        for (int i = 16 * h; i < 16 * h + 16; ++i) {
          if constexpr (EXACT) {
            const float e = __builtin_amdgcn_exp2f((x[i] - ref) * z2);
            ties += x[i] == mx;
            s4[i & 3] += x[i] == mx ? 0.f : e;
          } else {
            s4[i & 3] += __builtin_amdgcn_exp2f(fmaf(x[i], z2, ref2));
          }
        }
        l += (s4[0] + s4[1]) + (s4[2] + s4[3]);
      }
      if (mn == -INFINITY) l = NAN;
      l = lanes_sum<ROWS, 32>(l);
      if constexpr (EXACT) l += lanes_sum<ROWS, 32>((float)ties) - 1.0f;
      if (part == 0 && m < M && n0 < V) {
        if (tg.label) {
          const int c = label - n0;
          if (c >= 0 && c < kGroup) pa[m] = tile[r * PITCH + gg * kGroup + c] * zs;
        } else {
          tg.each(m, entry[gg], entry[gg + 1], [&](int e, int id, float p) __attribute__((always_inline)) {
            pa[(size_t)m * tg.k + e] = p * (tile[r * PITCH + gg * kGroup + id - n0] * zs);
          });
        }
        const size_t at = (size_t)(n0 / kGroup) * T + m;
        pm[at] = mx == -INFINITY ? mx : mx * zs;
        pl[at] = l;
      }
    }
  }
};

// z - m with z rounded as it was for m: of the largest 0, which a fused multiply-subtract would miss by the rounding.
__device__ __forceinline__ float from_largest(float x, float z_scale, float m) {
#pragma clang fp contract(off)
  const float z = x * z_scale;
  return z - m;
}
// dz as the operand of both gradient products: rows (F, times 2^15) and transposed (FT, times the rows' coefficients and what
// brings them all to 2^15).  Rows T .. Tp and columns V .. are zeros.
// Bound by the matrix cores and by itself, for all tiles of a round store at the same time: 8192 x 32000 x 4096 1.78 ms, 1.21
// PFLOP/s; a round of 256x256 tiles ends with 16 us of this, 9 of statistics.  Four waves of 128x128 and loads that are not spread
// gained nothing, waves of 128x64 lost.
template <int RAW, int TERMS>
struct EpiDz {
  static constexpr int kSpan = 64, kRaw = RAW;
  RowTargets tg;
  const float* lse;          // float32: t of the row, with its m in ref
  const float* ref;
  const float *dz_coef, *dz_max;
  int n_max;
  f16 *F, *FT;
  int Tp, Np;                // Np: the launch's columns
  int V, n_base;
  int64_t raw_ld;
  int raw_rows;
  float ft_scale;
  __device__ __forceinline__ void begin(int lane) { ft_scale = ldexpf(1.0f, max_exponent(dz_max, n_max, lane)); }
  // 8 elements of an operand's row, and those of the second and third term (`third` halves on in a block of 32 rows).
  __device__ __forceinline__ void put(f16* dst, size_t third, const float (&x)[8]) const {
    f16x8 hi;
#pragma unroll
    for (int j = 0; j < 8; ++j) hi[j] = from_f32<f16>(x[j]);
    *(f16x8*)(dst + (TERMS - 1) * third) = hi;
    if constexpr (TERMS == 3) {
      f16x8 lo;
#pragma unroll
      for (int j = 0; j < 8; ++j) lo[j] = from_f32<f16>(x[j] - (float)hi[j]);
      *(f16x8*)dst = lo;
      *(f16x8*)(dst + third) = hi;
    }
  }
  template <int COLS, int PITCH, int ROWS>
  __device__ __forceinline__ void consume(const float* tile_in, int m_base, int nb, int lane, int M) const {
    float* tile = const_cast<float*>(tile_in);
    constexpr int PARTS = 64 / ROWS, CH = COLS / 8;
    const int r = lane % ROWS, part = lane / ROWS, m = m_base + r, mc = min(m, M - 1);
    // dz * 2^15; a row without target, and one past the last: zeros.  (A head that half precision does not hold has made lse a NaN.)
    const bool live = m < M && tg.z_scale[mc] != 0.f;
    // float32: q = exp(z - m) / (1 + t) from the statistics of these very logits; the largest one's distance from 1, which is all
    // there is of a row that is sure of its token, is -t / (1 + t).
    constexpr bool own = TERMS == 3;
    const float zs = live ? tg.z_scale[mc] : 0.f, z2 = zs * kLog2e, stat = lse[mc];
    const float ref2 = !live ? (own ? INFINITY : -INFINITY) : own ? ref[mc] : fmaf(-stat, kLog2e, 15.0f);
    const float scale = own && live ? kDzScale / (1.0f + stat) : 0.f, top = -stat * scale;
    const float ft = live ? dz_coef[mc] * ft_scale : 0.f;
    static_assert(kDzScale == 32768.0f, "2^15");
    const int label = tg.label ? tg.label[mc] : -1;
    int entry[COLS / kGroup + 1] = {};                   // the row's entries here: entry[0] to entry[COLS / kGroup]
    if (!tg.label) tg.entries(mc, (n_base + nb) / kGroup, entry);
    const bool edge = n_base + nb + COLS > V || m_base + ROWS > M;   // (uniform) columns or rows that are not there
    // Chunk `it` of a lane is 8 columns of its row; of the operand's blocks of 16 columns it is half `part` of block it, or (PARTS 4)
    // half part & 1 of block 2 it + part / 2.
    static_assert(PARTS == 2 || PARTS == 4, "as computed here");
    f16* const f_at = F + (F ? act_index(m, nb, TERMS * Np) : 0) + (part >> 1) * 512 + (part & 1) * 256;
    auto finish = [&](float* x, float (&v)[8], int it, int c) __attribute__((always_inline)) {
      if (edge) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = n_base + nb + c + j < V && m < M ? v[j] : 0.f;
      }
      if (FT) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = v[j] * ft;
      }
      if (F && m < Tp) put(f_at + it * (PARTS / 2) * 512, (size_t)32 * Np, v);
    };
#pragma unroll
    for (int it = 0; it < CH / PARTS; ++it) {
      const int c = (it * PARTS + part) * 8, n = n_base + nb + c;
      float* x = tile + r * PITCH + c;
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if constexpr (own) v[j] = __builtin_amdgcn_exp2f(from_largest(x[j], zs, ref2) * kLog2e) * scale;
        else v[j] = __builtin_amdgcn_exp2f(fmaf(x[j], z2, ref2));
      }
      if (tg.label) {
        if ((unsigned)(label - n) < 8u) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            if (n + j != label) continue;
            if constexpr (own) v[j] = v[j] == scale ? top : v[j] - kDzScale;
            else v[j] -= kDzScale;
          }
        }
        finish(x, v, it, c);
      } else {                                           // lists: the entries are taken off in the LDS
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = v[j];
      }
    }
    if (!tg.label) {
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
      __builtin_amdgcn_wave_barrier();
      if (part == 0 && live)
        tg.each(m, entry[0], entry[COLS / kGroup], [&](int, int id, float p) __attribute__((always_inline)) {
          float* x = &tile[r * PITCH + id - n_base - nb];
          if constexpr (own) *x = *x == scale ? fmaf(1.0f - p, kDzScale, top) : fmaf(p, -kDzScale, *x);
          else *x = fmaf(p, -kDzScale, *x);
        });
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int it = 0; it < CH / PARTS; ++it) {
        const int c = (it * PARTS + part) * 8;
        float* x = tile + r * PITCH + c;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = x[j];
        finish(x, v, it, c);
      }
    }
    if (FT) {
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
      __builtin_amdgcn_wave_barrier();
      // Eight rows (t) of a column (v) a lane: half lane / 32 of the blocks of 16 rows, of which there are RB, of 32 columns.
      constexpr int RB = ROWS / 16;
      const int rows0 = m_base + (lane >> 5) * 8;
      f16* const t_at = FT + act_index(nb, m_base, TERMS * Tp) + lane * 8;
#pragma unroll
      for (int it = 0; it < COLS / 32 * RB; ++it) {
        const int cb = it / RB, rb = it % RB;
        const float* x = tile + (rb * 16 + (lane >> 5) * 8) * PITCH + cb * 32 + (lane & 31);
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = x[j * PITCH];
        if (rows0 + rb * 16 < Tp) put(t_at + (size_t)cb * 32 * (TERMS * Tp) + rb * 512, (size_t)32 * Tp, v);
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
};

// Rounds four results to the storage type.
template <bool ONCE = false>
__device__ __forceinline__ void store_result(void* out, size_t at, bool f32, const f32x4& g) {
  if (f32) {
    if constexpr (ONCE) __builtin_nontemporal_store(g, (f32x4*)((float*)out + at));
    else *(f32x4*)((float*)out + at) = g;
  } else {
    bf16x4 o;
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = from_f32<bf16>(g[j]);
    if constexpr (ONCE) __builtin_nontemporal_store(__builtin_bit_cast(u32x2, o), (u32x2*)((bf16*)out + at));
    else *(bf16x4*)((bf16*)out + at) = o;
  }
}

// grad_hidden of one slice of the vocabulary: a plane of float32 sums, or, where there is only one, the result.
// 8192 x 4096 x 32000 1.45 ms, 1.48 PFLOP/s; 56 x 4096 x 32000 44 us, 6.0 TB/s of the head as it is.
template <int RAW>
struct EpiHidden {
  static constexpr int kSpan = 64, kRaw = RAW;
  static constexpr bool kSliced = true;
  int slices;
  float* planes;             // [slices][T][ld], or nullptr
  int add;                   // to what is there
  int T, ld;
  const float* coef;
  void* out;
  int out_f32, d;
  int64_t raw_ld;
  int raw_rows, raw_cols;
  __device__ __forceinline__ void slice(int kz) { if (planes) planes += (size_t)kz * T * ld; }
  template <int COLS, int PITCH, int ROWS>
  __device__ __forceinline__ void consume(const float* tile, int m_base, int nb, int lane, int M) const {
    constexpr int LPR = COLS / 4, RPI = 64 / LPR, IT = ROWS / RPI;
    const int r0 = lane / LPR, c4 = (lane % LPR) * 4;
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int r = it * RPI + r0, m = m_base + r;
      const f32x4 v = *(const f32x4*)(tile + r * PITCH + c4) * (1.0f / (kDzScale * kWeightScale));
      if (m >= M || nb + c4 >= d) continue;
      if (planes) {
        f32x4* p = (f32x4*)(planes + (size_t)m * ld + nb + c4);
        *p = add ? *p + v : v;
      } else {
        store_result(out, (size_t)m * d + nb + c4, out_f32, v * coef[m]);
      }
    }
  }
};
// ... and the planes in their order, times the rows' coefficients or (nullptr) what grad_head takes.  Bound by what it moves: two
// planes of 8192 x 4096 53 us, 6.3 TB/s.
__global__ __launch_bounds__(256) void loss_planes_kernel(const float* __restrict__ planes, int n, int plane_rows, int ld, int rows,
                                                          int d, const float* __restrict__ coef, const float* __restrict__ dz_max,
                                                          int n_max, void* __restrict__ out, int out_f32) {
  const int across = (d + 255) / 256, m = blockIdx.x / across * 4 + (threadIdx.x >> 6);
  const int c = (blockIdx.x % across * 64 + (threadIdx.x & 63)) * 4;
  const float scale = coef ? coef[min(m, rows - 1)] : head_scale(dz_max, n_max, threadIdx.x & 63);
  if (m >= rows || c >= d) return;
  const size_t plane = (size_t)plane_rows * ld;
  const float* p = planes + (size_t)m * ld + c;
  f32x4 v = *(const f32x4*)p;
  int i = 1;
  for (; i + 3 < n; i += 4) {
    f32x4 u[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) u[j] = *(const f32x4*)(p + (i + j) * plane);
#pragma unroll
    for (int j = 0; j < 4; ++j) v += u[j];
  }
  for (; i < n; ++i) v += *(const f32x4*)(p + i * plane);
  store_result(out, (size_t)m * d + c, out_f32, v * scale);
}

// Products of few tiles and a long contraction are sliced: planes of float32 sums, which this adds in their order and hands to the
// epilogue, a workgroup 32 rows of 64 columns.  448 rows of 256 bins over 4096: 28 tiles of 64x128 in four slices 6.0 us, this 5.8.
template <int RAW>
struct EpiPlanes {
  static constexpr int kSpan = 64, kRaw = RAW;
  static constexpr bool kSliced = true;
  int slices;
  float* planes;             // [slices][Tp][N]
  int Tp, N;
  int64_t raw_ld;
  int raw_rows;
  __device__ __forceinline__ void slice(int kz) { planes += (size_t)kz * Tp * N; }
  template <int COLS, int PITCH, int ROWS>
  __device__ __forceinline__ void consume(const float* tile, int m_base, int nb, int lane, int M) const {
    constexpr int LPR = COLS / 4, RPI = 64 / LPR;
    const int r0 = lane / LPR, c4 = (lane % LPR) * 4;
#pragma unroll
    for (int it = 0; it < ROWS / RPI; ++it) {
      const int r = it * RPI + r0, m = m_base + r;
      if (m < M) *(f32x4*)(planes + (size_t)m * N + nb + c4) = *(const f32x4*)(tile + r * PITCH + c4);
    }
  }
};
template <class Epi>
__global__ __launch_bounds__(256) void loss_slices_kernel(const float* __restrict__ planes, int slices, int Tp, int N, int M, Epi epi_in) {
  constexpr int PITCH = 68;
  __shared__ __attribute__((aligned(16))) float tile[32 * PITCH];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int across = N / 64, m0 = blockIdx.x / across * 32, n0 = blockIdx.x % across * 64;
  Epi epi = epi_in;
  const size_t plane = (size_t)Tp * N, row4 = (size_t)4 * N;
  const int r = wave * 8 + (lane >> 4), c4 = (lane & 15) * 4;        // eight rows a wave, in two halves
  const float* p = planes + (size_t)(m0 + r) * N + n0 + c4;
  f32x4 v[2] = {};
  for (int s = 0; s < slices; s += 8) {                              // eight slices at a time
    f32x4 u[8][2];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (s + j < slices) {
        u[j][0] = *(const f32x4*)(p + (s + j) * plane);
        u[j][1] = *(const f32x4*)(p + (s + j) * plane + row4);
      }
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (s + j < slices) {
        v[0] += u[j][0];
        v[1] += u[j][1];
      }
  }
  *(f32x4*)(tile + r * PITCH + c4) = v[0];
  *(f32x4*)(tile + (r + 4) * PITCH + c4) = v[1];
  if (wave < 2) {
    if constexpr (requires { epi.begin(lane); }) epi.begin(lane);
  }
  __syncthreads();
  if (wave < 2) epi.template consume<64, PITCH, 16>(tile + wave * 16 * PITCH, m0 + wave * 16, n0, lane, M);
}

// grad_head: rows of a piece of the vocabulary.  32000 x 4096 x 8192 1.65 ms, 1.30 PFLOP/s; 32003 x 768 x 1021 51 us (49 MB written).
struct EpiHead {
  static constexpr int kSpan = 64;
  static constexpr bool kSliced = true;                // (of the rows)
  int slices;
  float* planes;             // [slices][M][ld], or nullptr
  int plane, ld;             // rows of a plane
  void* out;                 // the piece's first row
  int out_f32, d, rows;
  const float* dz_max;
  int n_max;
  float scale;
  __device__ __forceinline__ void begin(int lane) { scale = planes ? 1.0f : head_scale(dz_max, n_max, lane); }
  __device__ __forceinline__ void slice(int kz) { if (planes) planes += (size_t)kz * plane * ld; }
  template <int COLS, int PITCH, int ROWS>
  __device__ __forceinline__ void consume(const float* tile, int m_base, int nb, int lane, int M) const {
    constexpr int LPR = COLS / 4, RPI = 64 / LPR, IT = ROWS / RPI;
    const int r0 = lane / LPR, c4 = (lane % LPR) * 4;
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int r = it * RPI + r0, m = m_base + r;
      const f32x4 g = *(const f32x4*)(tile + r * PITCH + c4) * scale;
      if (m >= rows || nb + c4 >= d) continue;
      if (planes) *(f32x4*)(planes + (size_t)m * ld + nb + c4) = g;
      else store_result<true>(out, (size_t)m * d + nb + c4, out_f32, g);
    }
  }
};

// grad_head of at most 128 rows (bfloat16), where it is bound by what it writes: 64 rows of the head by 64 columns at a time a
// wave, whose dz stays in registers while it walks `walk` columns, straight from the accumulators.  The products are transposed (a row
// of dz^T is a column here), and which columns of h a tile's rows are is chosen so that a lane holds eight in a row of each two
// tiles, and the four groups of lanes 64 bytes; lanes of rows 8 apart swap halves, so that a store covers 128.  32000 x 4096 of 56
// rows: 262 MB in 50 to 54 us, 5 TB/s (a large copy 4.8); by the products' tiles 81.
template <int KS>
__global__ __launch_bounds__(256) void loss_head_rows_kernel(const f16* __restrict__ dzT, const f16* __restrict__ hT, int Tp,
                                                             const float* __restrict__ dz_max, int n_max, bf16* __restrict__ out,
                                                             int rows, int d, int walk) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, i = lane & 15, across = (d + walk - 1) / walk, id = blockIdx.x * 4 + wave;
  const int v0 = id / across * 64, c_first = id % across * walk;
  if (v0 >= rows) return;                                            // (no barriers)
  const size_t k_at = (size_t)(g >> 1) * 512 + (g & 1) * 256;        // of a k-step of 32: group g has k 8 g ..
  f16x8 b[4][KS];
#pragma unroll
  for (int nt = 0; nt < 4; ++nt)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      b[nt][ks] = *(const f16x8*)(dzT + (size_t)(v0 / 32 + nt / 2) * 32 * Tp + ks * 1024 + k_at + ((nt & 1) * 16 + i) * 8);
  const float scale = head_scale(dz_max, n_max, lane);
  auto load = [&](f16x8 (&a)[4][KS], int c0) {
#pragma unroll
    for (int mt = 0; mt < 4; ++mt) {
      const int c = c0 + 32 * (mt >> 1) + 8 * (i >> 2) + 4 * (mt & 1) + (i & 3);    // (columns past d: zeros of the operand, dP of them)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) a[mt][ks] = *(const f16x8*)(hT + (size_t)(c >> 5) * 32 * Tp + ks * 1024 + k_at + (c & 31) * 8);
    }
  };
  const int c_end = min(c_first + walk, d);
  f16x8 a[2][4][KS];
  load(a[0], c_first);
  auto columns = [&](f16x8 (&now)[4][KS], f16x8 (&next)[4][KS], int c0) __attribute__((always_inline)) {
    if (c0 + 64 < c_end) load(next, c0 + 64);
    f32x4 acc[4][4];
#pragma unroll
    for (int mt = 0; mt < 4; ++mt)
#pragma unroll
      for (int nt = 0; nt < 4; ++nt) {
        acc[mt][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) acc[mt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(now[mt][ks], b[nt][ks], acc[mt][nt], 0, 0, 0);
      }
    // Lanes of rows 8 apart swap a half, so that a store covers 128 bytes of 8 rows.
    const bool up = i & 8;
    const int c = c0 + 8 * g + (up ? 32 : 0);
#pragma unroll
    for (int nt = 0; nt < 4; ++nt) {
      u32x4 o[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        bf16x8 e;
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = from_f32<bf16>(acc[2 * h + (j >> 2)][nt][j & 3] * scale);
        o[h] = __builtin_bit_cast(u32x4, e);
      }
      u32x4 s[2];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const unsigned other = __builtin_bit_cast(unsigned, dpp<0x128>(__builtin_bit_cast(float, up ? o[0][j] : o[1][j])));   // row_ror 8
        s[0][j] = up ? other : o[0][j];
        s[1][j] = up ? o[1][j] : other;
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int v = v0 + nt * 16 + h * 8 + (i & 7);
        if (v < rows && c < d) {
          __builtin_nontemporal_store(s[h], (u32x4*)(out + (size_t)v * d + c));
        }
      }
    }
  };
  for (int c0 = c_first; c0 < c_end; c0 += 128) {
    columns(a[0], a[1], c0);
    if (c0 + 64 < c_end) columns(a[1], a[0], c0 + 64);
  }
}

// Both gradients in one launch, where their tiles are the smallest ones: five microseconds less.
struct EpiGradients {
  static constexpr int kSpan = 64;
  static constexpr bool kSliced = true, kPair = true;
  EpiHidden<0> hidden;
  EpiHead head;
  unsigned split;
  const f16 *A, *Wp;         // of the second, grad_head
  int lda, M, K, tiles_m, tiles_n;
  bool second;
  __device__ __forceinline__ void begin(int lane) { if (second) head.begin(lane); }
  __device__ __forceinline__ void slice(int kz) {
    if (second) head.slice(kz);
    else hidden.slice(kz);
  }
  template <int COLS, int PITCH, int ROWS>
  __device__ __forceinline__ void consume(const float* tile, int m_base, int nb, int lane, int M) const {
    if (second) head.consume<COLS, PITCH, ROWS>(tile, m_base, nb, lane, M);
    else hidden.consume<COLS, PITCH, ROWS>(tile, m_base, nb, lane, M);
  }
};

static int round_up(int x, int n) { return (x + n - 1) / n * n; }
// Columns of a product: whole tiles of 256, or of 128 where that leaves more than an eighth less.
static int tile_up(int x) {
  const int a = round_up(x, 128), b = round_up(x, 256);
  return 8 * (b - a) > b ? a : b;
}

// ---- tiles and slices -----------------------------------------------------------------------------------------------
// Which tiles a product [M, N] over K takes, and into how many slices its contraction is split, goes by a model of its time: a
// round of 256 workgroups (two rounds' worth of the 64x128 tiles that share a compute unit) takes `fixed`, by what the epilogue
// does, and a time per 1024 k that grows from `few` on an empty chip to `full`.  Workgroups that fetch an operand from HBM take in
// 65 GB/s each at best.  Fitted to 552 launches (32 to 32000 rows and columns, K 64 to 32000): us a launch, the model's pick and
// others:
//   statistics, 4096 x 32000 x 4096 753 (256x256; 192x256 801, 128x256 883, 128x128 1106), x 768 190 (202, 215, 256);
//   1024 x 4096 x 4096 33 (128x128; 64x128 40, 256x256 73); 192 x 32000 x 4096 75 (128x256; 64x128 108); 64 x 4096 x 4096 18
//   (64x128; 128x128 25, 256x256 68);
//   grad_head 32000 x 4096 x 64 81 (192x256; 128x256 96, 128x128 128), x 4096 814 (256x256; 833, 903);
//   grad_hidden 2048 x 4096 x 32000 in one slice 407 (128x256; 192x256 467, 256x256 557 of 128 tiles), in two of 256x256 365.
// Unpacked weights cost 1.5 times the products on a full chip (re-encoding), twice on an empty one (the latency of pieces of 128
// bytes), and have no 256x256 tile (registers).
enum LossTile { L_64x128, L_64x128_PAIR, L_128x128, L_128x256, L_192x256, L_256x256, L_COUNT };
enum LossWork { L_STATS, L_DZ, L_STORE };
struct LossTileCost { int bm, bn, slots; float few, full, fixed[3]; };
constexpr LossTileCost kLossTiles[L_COUNT] = {
    {64, 128, 256, 3.5f, 5.8f, {0.7f, 5.0f, 2.6f}},    {64, 128, 512, 4.0f, 10.4f, {1.0f, 4.6f, 3.3f}},
    {128, 128, 256, 5.0f, 8.0f, {2.0f, 8.3f, 3.5f}},   {128, 256, 256, 8.1f, 12.9f, {3.8f, 12.5f, 5.2f}},
    {192, 256, 256, 11.5f, 17.0f, {6.0f, 15.0f, 6.3f}}, {256, 256, 256, 14.8f, 21.5f, {9.0f, 16.6f, 13.0f}}};
struct LossPick { int tile, slices; float us; };
static float launch_us(int t, LossWork work, int M, int N, int K, int slices, bool raw) {
  const LossTileCost& c = kLossTiles[t];
  const long long wgs = (long long)((M + c.bm - 1) / c.bm) * (N / c.bn) * slices;
  const float k = (float)round_up(K / slices, PK) / 1024.0f;
  float few = raw ? c.few * 2.0f : c.few, full = raw ? c.full * 1.5f : c.full;
  if ((long long)K * (M > N ? M : N) > 64'000'000) few = fmaxf(few, (float)(c.bm + c.bn) * 2048.0f / 65e3f), full = fmaxf(full, few);
  const float rounds = (float)(wgs / c.slots), rest = (float)(wgs % c.slots) / (float)c.slots;
  return 2.0f + rounds * (c.fixed[work] + full * k) + (rest > 0.f ? c.fixed[work] + (few + (full - few) * rest) * k : 0.f);
}
// most: slices at most (1: not sliced).  Slices cost a launch that joins them and their planes, written and read at 4 TB/s.
constexpr float kJoinUs[3] = {5.0f, 6.5f, 4.0f};
static LossPick pick_tiles(LossWork work, int M, int N, int K, int most, bool raw) {
  LossPick best{L_64x128, 1, 1e30f};
  for (int s = 1; s <= most; s += s < 8 ? 1 : s < 16 ? 2 : 4) {
    const float join = s > 1 ? kJoinUs[work] + (float)s * (float)M * (float)N * 2e-6f : 0.f;
    if (join > best.us) break;
    for (int t = 0; t < (raw ? L_256x256 : L_COUNT); ++t) {
      if (N % kLossTiles[t].bn) continue;
      const float us = launch_us(t, s > 1 ? L_STORE : work, M, N, K, s, raw) + join;
      if (us < best.us) best = LossPick{t, s, us};
    }
  }
  return best;
}

template <class Epi>
static void product(int tile, const f16* A, int lda, const void* W, int M, int N, int K, const Epi& epi, hipStream_t st) {
  const GemmF16 g{A, lda, (const f16*)W, M, N, K, K, nullptr};
  constexpr bool four = std::is_same_v<Epi, EpiHidden<0>> || std::is_same_v<Epi, EpiHead>;    // 128x128 waves, as residual adds
  switch (tile) {
    case L_64x128: launch<2, 4, 32, 32, 4, 4, 1, true, false, false>(g, epi, st); break;
    case L_64x128_PAIR: launch<2, 2, 32, 64, 3, 3, 2, false, false, false>(g, epi, st); break;
    case L_128x128: launch<4, 2, 32, 64, 4, 4, 1, false, false, false>(g, epi, st); break;
    case L_128x256: launch<2, 4, 64, 64, 3, 3, 1, false, false, false>(g, epi, st); break;
    case L_192x256: launch<2, 4, 96, 64, 2, 3, 1, false, false, false>(g, epi, st); break;
    default:
      if constexpr (raw_w<Epi>() != 0) launch<2, 4, 96, 64, 2, 3, 1, false, false, false>(g, epi, st);
      else if constexpr (four) launch<2, 2, 128, 128, 2, 3, 1, false, true, false>(g, epi, st);
      else launch<4, 2, 64, 128, 2, 3, 1, false, true, false>(g, epi, st);
  }
}

// Both gradients, dz [M, K] W [N, K] and the second's own product, in one launch of the smallest tiles.
static void gradients(const f16* A, int lda, const f16* W, int M, int N, int K, const EpiHidden<0>& hidden, const f16* A2, int lda2,
                      const f16* W2, int M2, int K2, const EpiHead& head, hipStream_t st) {
  auto up = [](int x) { return (x + 63) / 64; };
  const unsigned split = (unsigned)round_up(up(M) * (N / 128) * hidden.slices, 8);
  const EpiGradients both{hidden, head, split, A2, W2, lda2, M2, K2, up(M2), N / 128, false};
  launch<2, 4, 32, 32, 4, 4, 1, true, false, false>(GemmF16{A, lda, W, M, N, K, K, nullptr}, both, st);
}

// ---- joining the groups -------------------------------------------------------------------------------------------
// (EXACT as above.)  Bound by latency (3 to 5 us; 8192 rows of 500 groups 14).  16 rows a workgroup, 64 threads a row, which take every 64th group; their sums are joined in a tree.
template <bool EXACT>
__global__ __launch_bounds__(1024) void loss_join_kernel(const float* __restrict__ pm, const float* __restrict__ pl,
                                                         const float* __restrict__ pa, int T, int groups, RowTargets tg,
                                                         const float* __restrict__ ent, const float* __restrict__ mass,
                                                         float* __restrict__ loss, float* __restrict__ lse, float* __restrict__ ref_out) {
  __shared__ float sm[64][17], sl[64][17], sa[64][17];
  const int r = threadIdx.x & 15, part = threadIdx.x >> 4, row = blockIdx.x * 16 + r;
  const bool live = row < T && tg.z_scale[row] != 0.f;
  float m = -INFINITY, l = 0.f, a = 0.f;
  auto add = [](float& m, float& l, float m2, float l2) {            // (m, l) and another one to a common maximum
    if constexpr (EXACT) {
      if (m2 == -INFINITY) return;                                   // (a part without groups)
      if (m2 <= m) l += (1.0f + l2) * __builtin_amdgcn_exp2f((m2 - m) * kLog2e);
      else l = m == -INFINITY ? l2 : l2 + (1.0f + l) * __builtin_amdgcn_exp2f((m - m2) * kLog2e), m = m2;
    } else {
      const float mm = fmaxf(m, m2), ref = mm == -INFINITY ? 0.f : mm;
      l = l * __builtin_amdgcn_exp2f((m - ref) * kLog2e) + l2 * __builtin_amdgcn_exp2f((m2 - ref) * kLog2e);
      m = mm;
    }
  };
  if (live) {
    for (int g0 = part; g0 < groups; g0 += 256) {
      float um[4], ul[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const size_t at = (size_t)min(g0 + 64 * u, groups - 1) * T + row;
        um[u] = pm[at];
        ul[u] = pl[at];
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (g0 + 64 * u < groups) add(m, l, um[u], ul[u]);
    }
    if (!tg.label)
      for (int e = part, n = tg.first[(size_t)row * (groups + 1) + groups]; e < n; e += 64) a += pa[(size_t)row * tg.k + e];
  }
  sm[part][r] = m;
  sl[part][r] = l;
  sa[part][r] = a;
  for (int s = 32; s > 0; s >>= 1) {
    __syncthreads();
    if (part < s) {
      add(m, l, sm[part + s][r], sl[part + s][r]);
      a += sa[part + s][r];
      sm[part][r] = m;
      sl[part][r] = l;
      sa[part][r] = a;
    }
  }
  if (part == 0 && row < T) {
    const float ref = m == -INFINITY ? 0.f : m, lg = EXACT ? log1pf(l) : logf(l);
    if (ref_out) {                                                   // for a gradient: m and t
      ref_out[row] = live ? ref : 0.f;
      lse[row] = live ? l : 0.f;
    } else {                                                         // (the difference to the largest logit first: it is exact)
      lse[row] = live ? ref + lg : 0.f;
      loss[row] = !live ? 0.f : tg.label ? lg + (ref - pa[row]) : ent[row] + (mass[row] * lg + fmaf(mass[row], ref, -a));
    }
  }
}

// ---- host ------------------------------------------------------------------------------------------------------
namespace {

struct Plan {
  int T, d, V, k, terms, groups;
  int Tp, dP, Vp;              // padded sizes of operands: contractions in whole slabs, columns in whole tiles
  bool raw;                    // the head is read as it is
  int piece, pieces;           // columns of the vocabulary at a time (gradient)
  LossPick z, stats;           // the logits' products (stats: of float32 with a gradient, which has both)
  bool z_planes;               // they leave planes, for loss_slices_kernel
  LossPick hidden, head;
  int sets;                    // planes of grad_hidden: of each slice, of up to four pieces (later ones add to them)
  size_t z_scale, coef, dz_coef, dz_max, label, ids, p, ent, mass, first;
  size_t hF, hT, wF, wT, dzF, dzT, planes, head_planes, zp, pm, pl, pa, ref, sum, bytes;
};

Plan make_plan(const vla_head_rows& r, int k, bool grad) {
  Plan w{};
  w.T = r.n_rows, w.d = r.d_model, w.V = r.vocab, w.k = k;
  w.terms = r.dtype == VLA_F32 ? 3 : 1;
  w.Tp = round_up(w.T, 64), w.dP = tile_up(w.d), w.Vp = tile_up(w.V);
  w.groups = (w.V + kGroup - 1) / kGroup;
  const size_t half = 2 * (size_t)w.terms;
  w.piece = w.Vp, w.pieces = 1;
  if (grad) {
    // dz, both ways, is whole within 2 GB.  Otherwise it is formed in pieces: each reads and writes the planes of grad_hidden (8 d
    // bytes a row, against 8 a column of dz), so that a piece has 16 d columns, within 512 MB and 2 GB.  us, pieces within 512 MB,
    // 1 GB, 2 GB, and 4 GB of dz: 6171 x 28990 x 512 877, 673 (whole); 8192 x 32000 x 4096 4957, 4847 (whole); 32768 x 32000 x 768
    // 8020, 5697, 4794, 4684; 65536 x 32000 x 1024 30558, 18558, 13046, 11078; 20000 x 32000 x 4096 12782, 12171, 11882, 11770.
    // (Less than 512 MB is slower as well, although it would stay in the last-level cache.)
    const size_t column = 2 * half * w.Tp, low = (size_t)512 << 20, high = (size_t)2 << 30, by_d = 16 * column * w.dP;
    const size_t cols = ((column * w.Vp <= high || by_d > high ? high : by_d < low ? low : by_d) / column) & ~(size_t)255;
    const int most = cols < 256 ? 256 : cols > (size_t)w.Vp ? w.Vp : (int)cols;
    w.pieces = (w.Vp + most - 1) / most;
    if (w.pieces > 1) {                                             // (every piece whole tiles of any kind)
      w.Vp = round_up(w.V, 256);
      w.piece = round_up((w.Vp + w.pieces - 1) / w.pieces, 256);
      w.pieces = (w.Vp + w.piece - 1) / w.piece;
    }
  }
  // Slices: a slab at least in each (of four, but for the last piece's).
  const int Kz = w.terms * w.dP, Kh = w.terms * w.piece, Kw = w.terms * w.Tp;
  const int last = (w.V - (w.pieces - 1) * w.piece + PK - 1) / PK;
  auto most = [](int K) { return max(1, min(64, K / PK / 4)); };
  auto picks = [&](bool raw) {
    const int z_most = w.pieces > 1 ? 1 : raw ? most(w.d) : most(Kz);
    w.z = w.stats = pick_tiles(grad ? L_DZ : L_STATS, w.T, w.piece, raw ? w.d : Kz, z_most, raw);
    w.z_planes = w.z.slices > 1;
    if (w.terms == 3 && grad) {                  // two products, or one whose planes serve both (read twice)
      w.z = pick_tiles(L_DZ, w.T, w.piece, Kz, 1, false), w.stats = pick_tiles(L_STATS, w.T, w.piece, Kz, 1, false);
      float us = w.z.us + w.stats.us;
      w.z_planes = false;
      for (int s = 1; s <= z_most && w.pieces == 1; s += s < 8 ? 1 : s < 16 ? 2 : 4)
        for (int t = 0; t < L_COUNT; ++t) {
          if (w.piece % kLossTiles[t].bn) continue;
          const float both = launch_us(t, L_STORE, w.T, w.piece, Kz, s, false) + kJoinUs[L_STATS] + kJoinUs[L_DZ] +
                             (float)s * (float)w.T * (float)w.piece * 3e-6f;
          if (both < us) us = both, w.z = w.stats = LossPick{t, s, both}, w.z_planes = true;
        }
      w.z.us = us;
    }
    if (grad) w.hidden = pick_tiles(L_STORE, w.T, w.dP, Kh, min(most(Kh), last), raw);
    return (w.z.us + (grad ? w.hidden.us : 0.f)) * (float)w.pieces;
  };
  const float packed = picks(false);
  // A bfloat16 head is read as it is where packing it (5 TB/s of twice its bytes, three times with a gradient) costs more.  us, as
  // it is / packed, loss and gradient (with one form of grad_head): 32000 x 4096 56 rows 57 / 148, 238 / 365, 384 rows 112 / 185,
  // 425 / 525, 768 rows 202 / 258, 653 / 728, 1536 rows 404 / 391, 1196 / 1148; 32000 x 768 56 rows 21 / 34, 54 / 73, 256 rows 31 /
  // 39, 92 / 96, 512 rows 57 / 50, 160 / 133; 8000 x 2048 256 rows 30 / 31, 70 / 71, 384 rows 45 / 35, 101 / 84; 4000 x 1024 the
  // same within 5 % up to 384 rows.
  if (r.dtype == VLA_BF16 && w.d % PK == 0) {
    const float raw = picks(true);
    w.raw = raw < packed + (float)w.V * (float)w.d * (grad ? 6e-6f : 4e-6f) / 5.0f;
    if (!w.raw) picks(false);
  }
  if (grad) w.head = pick_tiles(L_STORE, w.Vp, w.dP, Kw, w.pieces > 1 ? 1 : most(Kw), false);
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t o = at; at += (bytes + 255) / 256 * 256; return o; };
  const size_t T = (size_t)w.T;
  w.z_scale = take(4 * T);
  if (k) {
    w.ids = take(4 * T * k), w.p = take(4 * T * k), w.ent = take(4 * T), w.mass = take(4 * T);
    w.first = take(2 * T * (w.groups + 1));
  } else {
    w.label = take(4 * T);
  }
  if (w.z_planes) w.zp = take(4 * (size_t)w.z.slices * w.Tp * w.Vp);
  w.hF = take((size_t)w.Tp * w.dP * half);
  if (!w.raw) w.wF = take((size_t)w.piece * w.dP * half);
  if (!grad || w.terms == 3) w.pm = take(4 * T * w.groups), w.pl = take(4 * T * w.groups), w.pa = take(4 * T * (k ? k : 1));
  if (grad) {
    w.coef = take(4 * T), w.dz_coef = take(4 * T), w.dz_max = take(w.Tp / 2);
    w.hT = take((size_t)w.Tp * w.dP * half);
    if (!w.raw) w.wT = take((size_t)w.piece * w.dP * half);
    w.dzF = take((size_t)w.Tp * w.piece * half), w.dzT = take((size_t)w.Tp * w.piece * half);
    w.sets = min(w.pieces, 4);
    if (w.sets * w.hidden.slices > 1) w.planes = take(4 * T * w.dP * w.sets * w.hidden.slices);
    if (w.head.slices > 1) w.head_planes = take(4 * (size_t)w.head.slices * w.Vp * w.dP);
    if (w.terms == 3) w.ref = take(4 * T), w.sum = take(4 * T);
  }
  w.bytes = at;
  return w;
}

// The last plans of this thread (some microseconds each), by the sizes that they depend on.
const Plan& plan_of(const vla_head_rows& r, int k, bool grad) {
  struct Kept { int T, d, V, dtype, k, grad; Plan plan; };
  static thread_local Kept kept[16] = {};
  static thread_local unsigned next = 0;
  for (const Kept& e : kept)
    if (e.T == r.n_rows && e.d == r.d_model && e.V == r.vocab && e.dtype == r.dtype && e.k == k && e.grad == (int)grad) return e.plan;
  Kept& e = kept[next++ % 16];
  e = Kept{r.n_rows, r.d_model, r.vocab, r.dtype, k, (int)grad, make_plan(r, k, grad)};
  return e.plan;
}

int check_rows(const vla_head_rows* r, bool pointers) {
  if (!r) return VLA_E_NULL;
  if (r->dtype != VLA_F32 && r->dtype != VLA_BF16) return VLA_E_CONFIG;
  const int unit = r->dtype == VLA_F32 ? 4 : 8;
  if (r->n_rows < 1 || r->n_rows > 1 << 18 || r->vocab < 1 || r->vocab > 1 << 20) return VLA_E_SHAPE;
  if (r->d_model < unit || r->d_model > 1 << 15 || r->d_model % unit) return VLA_E_SHAPE;
  if (r->temperature != 0.f && !(r->temperature >= 0x1p-40f && r->temperature <= 0x1p40f)) return VLA_E_SHAPE;
  if (!pointers) return VLA_OK;
  if (!r->hidden || !r->head) return VLA_E_NULL;
  if (r->ld_hidden < r->d_model || r->ld_head < r->d_model || r->ld_hidden > 1 << 22 || r->ld_head > 1 << 22 || r->ld_hidden % unit || r->ld_head % unit) return VLA_E_SHAPE;
  if (((uintptr_t)r->hidden | (uintptr_t)r->head) & 15) return VLA_E_SHAPE;
  return VLA_OK;
}

struct Targets {
  const int32_t* labels;       // or
  const float* top_logits;
  const int32_t* top_ids;
  int k;
};

int check_call(const vla_head_rows* r, const Targets& t, bool grad, void* work, size_t work_bytes, Plan* plan) {
  const int rc = check_rows(r, true);
  if (rc) return rc;
  if (!work || (t.k ? !t.top_logits || !t.top_ids : !t.labels)) return VLA_E_NULL;
  if ((uintptr_t)work & 255) return VLA_E_SHAPE;
  *plan = plan_of(*r, t.k, grad);
  return work_bytes < plan->bytes ? VLA_E_CAPACITY : VLA_OK;
}

template <class T>
HeadPack<T> head_pack(const Plan& w, const vla_head_rows& r, int n0, int N, bool transposed, char* work) {
  return HeadPack<T>{(const T*)r.head + (size_t)n0 * r.ld_head, r.ld_head, min(N, w.V - n0), w.d, N, w.dP, (f16*)(work + w.wF),
                     transposed ? (f16*)(work + w.wT) : nullptr};
}

// Rows and, if it is packed in one piece, the head.
template <class T>
RowTargets prepare(const Plan& w, const vla_head_rows& r, const Targets& t, const float* g, bool h_transposed, bool w_transposed,
                   char* work, hipStream_t st) {
  constexpr int TERMS = std::is_same_v<T, float> ? 3 : 1;
  auto f = [&](size_t o) { return (float*)(work + o); };
  const float tau = r.temperature > 0.f ? r.temperature : 1.0f;
  const RowsOut out{f(w.z_scale), f(w.coef), f(w.dz_coef), f(w.dz_max), (int32_t*)(work + w.label), (int32_t*)(work + w.ids), f(w.p),
                    f(w.ent), f(w.mass), (unsigned short*)(work + w.first), (f16*)(work + w.hF), h_transposed ? (f16*)(work + w.hT) : nullptr};
  auto kern = loss_rows_kernel<T, TERMS>;
  static bool attr_set = false;
  if (!attr_set) {
    (void)hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, 8 * 12 * kMaxTop);
    attr_set = true;
  }
  HeadPack<T> head{};
  const int chunks = (w.dP + kRowsChunk - 1) / kRowsChunk, splits = w.Tp / 8 * chunks <= 1024 ? chunks : 1;
  int wgs = w.Tp / 8 * splits;
  if (!w.raw && w.pieces == 1) {
    head = head_pack<T>(w, r, 0, w.Vp, w_transposed, work);
    wgs += (w.dP / 64) * (w.Vp / 64) / 2;                            // (columns in pairs of tiles: dP and Vp are multiples of 128)
  }
  hipLaunchKernelGGL(kern, dim3(wgs), dim3(512), (size_t)96 * ((w.k + 3) & ~3), st, (const T*)r.hidden, r.ld_hidden, w.T, w.d, w.V,
                     1.0f / tau, t.labels, t.top_logits, t.top_ids, w.k, w.groups, g, w.Tp, w.dP, splits, out, head);
  return RowTargets{out.z_scale, w.k ? nullptr : out.label, out.ids, out.p, out.first, w.k, w.groups};
}

template <class T>
void pack_piece(const Plan& w, const vla_head_rows& r, int n0, int N, bool transposed, char* work, hipStream_t st) {
  constexpr int TERMS = std::is_same_v<T, float> ? 3 : 1;
  hipLaunchKernelGGL((loss_pack_kernel<T, TERMS>), dim3((w.dP / 64) * (N / 64)), dim3(256), 0, st,
                     head_pack<T>(w, r, n0, N, transposed, work));
}

// The logits of columns n0 .. n0 + N, of which `rows` are there, to the epilogue.
template <class T, class Make>
void logits(const Plan& w, const LossPick& pick, const vla_head_rows& r, int n0, int N, int rows, bool have_planes, char* work, Make&& make, hipStream_t st) {
  const f16* hF = (const f16*)(work + w.hF);
  const int ld = w.terms * w.dP;
  const void* W = w.raw ? (const void*)((const T*)r.head + (size_t)n0 * r.ld_head) : (const void*)(work + w.wF);
  float* zp = (float*)(work + w.zp);
  auto run = [&](auto RAW, int K) {
    constexpr int raw = decltype(RAW)::value;
    const auto epi = make(RAW);
    if (!w.z_planes) return product(pick.tile, hF, ld, W, w.T, N, K, epi, st);
    if (!have_planes) product(pick.tile, hF, ld, W, w.T, N, K, EpiPlanes<raw>{pick.slices, zp, w.Tp, N, r.ld_head, rows}, st);
    hipLaunchKernelGGL((loss_slices_kernel<std::remove_const_t<decltype(epi)>>), dim3((w.Tp / 32) * (N / 64)), dim3(256), 0, st,
                       zp, pick.slices, w.Tp, N, w.T, epi);
  };
  if constexpr (std::is_same_v<T, bf16>) {
    if (w.raw) return run(std::integral_constant<int, 1>{}, w.d);
  }
  run(std::integral_constant<int, 0>{}, ld);
}

// Statistics of the whole vocabulary, and what they come to: loss and lse, or (ref) t and m.
template <class T>
void statistics(const Plan& w, const vla_head_rows& r, const RowTargets& tg, float* loss, float* lse, float* ref, char* work,
                hipStream_t st) {
  auto f = [&](size_t o) { return (float*)(work + o); };
  for (int i = 0; i < w.pieces; ++i) {
    const int n0 = i * w.piece, N = min(w.piece, w.Vp - n0), rows = min(N, w.V - n0);
    if (!w.raw && w.pieces > 1) pack_piece<T>(w, r, n0, N, false, work, st);
    logits<T>(w, w.stats, r, n0, N, rows, false, work, [&](auto RAW) {
      return EpiStats<decltype(RAW)::value, std::is_same_v<T, float>>{tg, f(w.pm), f(w.pl), f(w.pa), w.T, w.V, n0, r.ld_head, rows};
    }, st);
  }
  hipLaunchKernelGGL((loss_join_kernel<std::is_same_v<T, float>>), dim3((w.T + 15) / 16), dim3(1024), 0, st, f(w.pm), f(w.pl), f(w.pa), w.T, w.groups, tg,
                     f(w.ent), f(w.mass), loss, lse, ref);
}

template <class T>
int run_loss(const Plan& w, const vla_head_rows& r, const Targets& t, float* loss, float* lse, char* work, hipStream_t st) {
  const RowTargets tg = prepare<T>(w, r, t, nullptr, false, false, work, st);
  statistics<T>(w, r, tg, loss, lse, nullptr, work, st);
  return hipGetLastError() == hipSuccess ? VLA_OK : VLA_E_HIP;
}

template <class T>
int run_grad(const Plan& w, const vla_head_rows& r, const Targets& t, const float* lse, const float* g, void* gh, void* gw,
             char* work, hipStream_t st) {
  constexpr int TERMS = std::is_same_v<T, float> ? 3 : 1;
  constexpr bool f32 = TERMS == 3;
  const RowTargets tg = prepare<T>(w, r, t, g, gw != nullptr, gh != nullptr, work, st);
  auto f = [&](size_t o) { return (float*)(work + o); };
  auto h = [&](size_t o) { return (f16*)(work + o); };
  if (f32) {
    statistics<T>(w, r, tg, nullptr, f(w.sum), f(w.ref), work, st);
    lse = f(w.sum);
  }
  const bool have_planes = f32 && w.z_planes;                    // (of the logits, from their statistics)
  int n_max = w.Tp / 8;
  if (n_max > 2048) {
    hipLaunchKernelGGL(loss_max_kernel, dim3(1), dim3(256), 0, st, f(w.dz_max), n_max);
    n_max = 1;
  }
  float* planes = w.planes ? f(w.planes) : nullptr;
  for (int i = 0; i < w.pieces; ++i) {
    const int n0 = i * w.piece, N = min(w.piece, w.Vp - n0), rows = min(N, w.V - n0);
    float* set = planes ? planes + (size_t)(i % w.sets) * w.hidden.slices * w.T * w.dP : nullptr;
    const int add = i >= w.sets;
    f16 *dzF = gh ? h(w.dzF) : nullptr, *dzT = gw ? h(w.dzT) : nullptr;
    if (!w.raw && w.pieces > 1) pack_piece<T>(w, r, n0, N, gh != nullptr, work, st);
    logits<T>(w, w.z, r, n0, N, rows, have_planes, work, [&](auto RAW) {
      return EpiDz<decltype(RAW)::value, TERMS>{tg, lse, f(w.ref), f(w.dz_coef), f(w.dz_max), n_max, dzF, dzT, w.Tp, N, w.V, n0, r.ld_head, rows, 0.f};
    }, st);
    const EpiHead head{w.head.slices, w.head_planes ? f(w.head_planes) : nullptr, w.Vp, w.dP, (T*)gw + (size_t)n0 * w.d, f32, w.d, rows,
                       f(w.dz_max), n_max, 0.f};
    const EpiHidden<0> hidden{w.hidden.slices, set, add, w.T, w.dP, f(w.coef), gh, f32, w.d, 0, 0, 0};
    const int K = TERMS * N, K2 = TERMS * w.Tp;
    if (!w.raw && gh && gw && w.hidden.tile == L_64x128 && w.head.tile == L_64x128) {
      gradients(dzF, K, h(w.wT), w.T, w.dP, K, hidden, dzT, K2, h(w.hT), N, K2, head, st);
      continue;
    }
    if constexpr (!f32)
      if (w.raw && gh)
        product(w.hidden.tile, dzF, N, (const T*)r.head + (size_t)n0 * r.ld_head, w.T, w.dP, round_up(rows, PK),
                EpiHidden<2>{w.hidden.slices, set, add, w.T, w.dP, f(w.coef), gh, 0, w.d, r.ld_head, rows, w.d}, st);
    if (!w.raw && gh) product(w.hidden.tile, dzF, K, work + w.wT, w.T, w.dP, K, hidden, st);
    if (gw && !f32 && w.Tp <= 128) {
      int walk = 512;                                                // (1024 waves, if there are as many)
      while (walk > 64 && (long long)((rows + 63) / 64) * ((w.d + walk - 1) / walk) < 1024) walk /= 2;
      const dim3 grid((unsigned)(((rows + 63) / 64) * ((w.d + walk - 1) / walk) + 3) / 4);
      auto kern = w.Tp == 64 ? loss_head_rows_kernel<2> : loss_head_rows_kernel<4>;
      hipLaunchKernelGGL(kern, grid, dim3(256), 0, st, dzT, h(w.hT), w.Tp, f(w.dz_max), n_max, (bf16*)gw + (size_t)n0 * w.d, rows, w.d, walk);
      continue;
    }
    if (gw) product(w.head.tile, dzT, K2, h(w.hT), N, w.dP, K2, head, st);
  }
  auto join = [&](const float* from, int n, int plane_rows, int rows, const float* coef, void* out) {
    hipLaunchKernelGGL(loss_planes_kernel, dim3((w.d + 255) / 256 * ((rows + 3) / 4)), dim3(256), 0, st, from, n, plane_rows, w.dP, rows,
                       w.d, coef, f(w.dz_max), n_max, out, (int)f32);
  };
  if (gh && planes) join(planes, w.sets * w.hidden.slices, w.T, w.T, f(w.coef), gh);
  if (gw && w.head_planes) join(f(w.head_planes), w.head.slices, w.Vp, w.V, nullptr, gw);
  return hipGetLastError() == hipSuccess ? VLA_OK : VLA_E_HIP;
}

int loss_call(const vla_head_rows* r, const Targets& t, float* loss, float* lse, void* work, size_t bytes, void* stream) {
  Plan w;
  const int rc = check_call(r, t, false, work, bytes, &w);
  if (rc) return rc;
  if (!loss || !lse) return VLA_E_NULL;
  return r->dtype == VLA_F32 ? run_loss<float>(w, *r, t, loss, lse, (char*)work, (hipStream_t)stream)
                             : run_loss<bf16>(w, *r, t, loss, lse, (char*)work, (hipStream_t)stream);
}

int grad_call(const vla_head_rows* r, const Targets& t, const float* lse, const float* g, void* gh, void* gw, void* work, size_t bytes,
              void* stream) {
  Plan w;
  const int rc = check_call(r, t, true, work, bytes, &w);
  if (rc) return rc;
  if (!lse || !g || (!gh && !gw)) return VLA_E_NULL;
  if (((uintptr_t)gh | (uintptr_t)gw) & 15) return VLA_E_SHAPE;
  return r->dtype == VLA_F32 ? run_grad<float>(w, *r, t, lse, g, gh, gw, (char*)work, (hipStream_t)stream)
                             : run_grad<bf16>(w, *r, t, lse, g, gh, gw, (char*)work, (hipStream_t)stream);
}

}  // namespace
}  // namespace vla

extern "C" {

int vla_loss_workspace(const vla_head_rows* rows, int32_t n_top, int32_t grad, size_t* bytes) {
  const int rc = vla::check_rows(rows, false);
  if (rc) return rc;
  if (!bytes) return VLA_E_NULL;
  if (n_top < 0 || n_top > vla::kMaxTop) return VLA_E_SHAPE;
  *bytes = vla::make_plan(*rows, n_top, grad != 0).bytes;
  return VLA_OK;
}

int vla_token_loss(const vla_head_rows* rows, const int32_t* labels, float* loss_out, float* lse_out, void* work,
                   size_t work_bytes, void* hip_stream) {
  return vla::loss_call(rows, vla::Targets{labels, nullptr, nullptr, 0}, loss_out, lse_out, work, work_bytes, hip_stream);
}

int vla_distill_loss(const vla_head_rows* rows, const float* top_logits, const int32_t* top_ids, int32_t n_top, float* loss_out,
                     float* lse_out, void* work, size_t work_bytes, void* hip_stream) {
  if (n_top < 1 || n_top > vla::kMaxTop) return VLA_E_SHAPE;
  return vla::loss_call(rows, vla::Targets{nullptr, top_logits, top_ids, n_top}, loss_out, lse_out, work, work_bytes, hip_stream);
}

int vla_token_loss_grad(const vla_head_rows* rows, const int32_t* labels, const float* lse, const float* grad_loss,
                        void* grad_hidden, void* grad_head, void* work, size_t work_bytes, void* hip_stream) {
  return vla::grad_call(rows, vla::Targets{labels, nullptr, nullptr, 0}, lse, grad_loss, grad_hidden, grad_head, work, work_bytes,
                        hip_stream);
}

int vla_distill_loss_grad(const vla_head_rows* rows, const float* top_logits, const int32_t* top_ids, int32_t n_top,
                          const float* lse, const float* grad_loss, void* grad_hidden, void* grad_head, void* work,
                          size_t work_bytes, void* hip_stream) {
  if (n_top < 1 || n_top > vla::kMaxTop) return VLA_E_SHAPE;
  return vla::grad_call(rows, vla::Targets{nullptr, top_logits, top_ids, n_top}, lse, grad_loss, grad_hidden, grad_head, work,
                        work_bytes, hip_stream);
}

}  // extern "C"
