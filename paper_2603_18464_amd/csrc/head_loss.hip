// The head's losses (include/vla_loss.h): cross entropy of tokens and distillation from a teacher's top logits, with their
// gradients.  Both are one thing: a row's target is a short sorted list of (id, probability), one entry for a token.
//
// Mathematics.  With z = h W^T / tau in base-e logits, a group of 64 columns of a row leaves (m, l, a) = (max z, sum exp(z - m),
// sum over the row's entries in the group of p z); the groups are joined in their order to lse = m + log l, and
//     loss = sum p log p + (sum p) lse - sum p z        (a token: lse - z_label).
// The gradient forms z again, dz = q - r with q = exp(z - lse), and two products: grad_hidden = (g / tau) dz W, where a row's
// coefficient is applied at the end, and grad_head = dz^T (g h / tau), where it is applied to h.
//
// All products run on the half-precision kernel of gemm_tile.h, whose operands are in fragment order.  Powers of two keep them in
// the range of half precision: a row of h is scaled to a maximum in [2^13, 2^14) (exact for bfloat16), W by 2^8 (exact, as
// in the arena), dz, which lies in [-1, 1], by 2^15, and g h / tau as one tensor to a maximum in [2^13, 2^14).  dz is rounded to
// half precision (2^-11 of its value at most) and g h / tau likewise; everything else is float32.
// float32 operands are carried as two terms hi + lo (22 bits); a product of two of them is three, hi hi + lo hi + hi lo,
// laid out as one contraction three times as long: [hi | lo | hi] against [hi | hi | lo].
//
// What bounds them: the large calls by the matrix cores (2 T V d operations forward, 6 backward).
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
};

__device__ __forceinline__ float block_max(float v, float* red) {
  v = wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}
__device__ __forceinline__ float block_sum(float v, float* red) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

template <class T> struct Vec;
template <> struct Vec<float> { typedef f32x4 type; static constexpr int n = 4; };
template <> struct Vec<bf16> { typedef bf16x8 type; static constexpr int n = 8; };

// The exponent e for which |x| * 2^e lies in [2^13, 2^14), within what leaves 2^e and 2^-e finite; 0 for 0 and what is not finite.
__device__ __forceinline__ int scale_exponent(float x) {
  if (!(x > 0.f) || x == INFINITY) return 0;
  int e;
  (void)frexpf(x, &e);                     // x = f 2^e, f in [1/2, 1)
  return max(-100, min(100, 14 - e));
}

struct PrepOut {
  float *z_scale, *h_scale, *coef, *t_max;     // [T]; coef = g / tau and t_max = max |g h / tau| with a gradient only
  int32_t* label;
  int32_t* ids;
  float *p, *ent, *mass;                       // lists; sum p log p and sum p of a row
  unsigned short* first;
};

// One workgroup a row: its target, and the scales of its h.
template <class T>
__global__ __launch_bounds__(256) void loss_prep_kernel(const T* __restrict__ h, int64_t ld, int d, int V, float inv_tau,
                                                        const int32_t* __restrict__ labels, const float* __restrict__ top_logits,
                                                        const int32_t* __restrict__ top_ids, int k, int groups,
                                                        const float* __restrict__ g, PrepOut out) {
  __shared__ float red[4], s_p[kMaxTop];
  __shared__ int32_t s_id[kMaxTop], s_sorted[kMaxTop];
  __shared__ unsigned char s_lead[kMaxTop];
  __shared__ int s_n;
  const int row = blockIdx.x, t = threadIdx.x;
  bool live;
  if (labels) {
    const int32_t y = labels[row];
    live = y >= 0 && y < V;
    if (t == 0) out.label[row] = live ? y : -1;
  } else {
    if (t == 0) s_n = 0;
    float m = -INFINITY;
    for (int j = t; j < k; j += 256) {
      const int32_t id = top_ids[(size_t)row * k + j];
      const float l = top_logits[(size_t)row * k + j] * inv_tau;
      const bool in = id >= 0 && id < V && l != -INFINITY;
      s_id[j] = in ? id : -1;
      s_p[j] = l;
      if (in) m = fmaxf(m, l);
    }
    m = block_max(m, red);
    m = m == -INFINITY ? 0.f : m;                                    // (all NaN, or none)
    float sum = 0.f;
    for (int j = t; j < k; j += 256) {
      const float e = s_id[j] >= 0 ? expf(s_p[j] - m) : 0.f;
      s_p[j] = e;
      sum += e;
    }
    sum = block_sum(sum, red);                                       // (its barriers publish s_id and s_p)
    // equal ids: the first of them stands for all; its place is the number of smaller ids that stand
    for (int j = t; j < k; j += 256) {
      bool lead = s_id[j] >= 0;
      for (int i = 0; lead && i < j; ++i) lead = s_id[i] != s_id[j];
      s_lead[j] = lead;
    }
    __syncthreads();
    float ent = 0.f, mass = 0.f;
    int n = 0;
    for (int j = t; j < k; j += 256)
      if (s_lead[j]) {
        const int32_t id = s_id[j];
        int at = 0;
        float p = 0.f;
        for (int i = 0; i < k; ++i) {
          if (s_lead[i] && s_id[i] < id) ++at;
          if (s_id[i] == id) p += s_p[i];
        }
        p /= sum;
        s_sorted[at] = id;
        out.ids[(size_t)row * k + at] = id;
        out.p[(size_t)row * k + at] = p;
        if (p != 0.f) ent += p * logf(p);
        mass += p;
        ++n;
      }
    if (n) atomicAdd(&s_n, n);
    ent = block_sum(ent, red);
    mass = block_sum(mass, red);
    n = s_n;
    live = n > 0;
    if (t == 0) {
      out.ent[row] = ent;
      out.mass[row] = mass;
    }
    for (int j = t; j <= groups; j += 256) {                         // first entry of id 64 j and more
      int lo = 0, hi = n;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (s_sorted[mid] < j * kGroup) lo = mid + 1;
        else hi = mid;
      }
      out.first[(size_t)row * (groups + 1) + j] = (unsigned short)lo;
    }
  }
  float mx = 0.f;
  if (live) {
    const T* x = h + (size_t)row * ld;
    for (int i = t * Vec<T>::n; i < d; i += 256 * Vec<T>::n) {
      const typename Vec<T>::type v = *(const typename Vec<T>::type*)(x + i);
#pragma unroll
      for (int j = 0; j < Vec<T>::n; ++j) mx = fmaxf(mx, fabsf((float)v[j]));
    }
  }
  mx = block_max(mx, red);
  if (t == 0) {
    const int e = live ? scale_exponent(mx) : 0;
    out.h_scale[row] = live ? ldexpf(1.0f, e) : 0.f;
    out.z_scale[row] = live ? ldexpf(inv_tau / kWeightScale, -e) : 0.f;
    if (g) {
      const float c = live ? g[row] * inv_tau : 0.f;
      out.coef[row] = c;
      out.t_max[row] = fabsf(c) * mx;
    }
  }
}

// The power of two for g h / tau as one tensor: out[0], and its inverse times those of dz: out[1].
__global__ __launch_bounds__(256) void loss_scale_kernel(const float* __restrict__ t_max, int T, float* __restrict__ out) {
  __shared__ float red[4];
  float m = 0.f;
  for (int i = threadIdx.x; i < T; i += 256) m = t_max[i] < INFINITY ? fmaxf(m, t_max[i]) : m;
  m = block_max(m, red);
  if (threadIdx.x == 0) {
    const int e = scale_exponent(m);
    out[0] = ldexpf(1.0f, e);
    out[1] = ldexpf(1.0f / kDzScale, -e);
  }
}

// ---- operands in fragment order ---------------------------------------------------------------------------------
// 64 x 64 elements of src [R, C] a workgroup: as rows (F, ld halves a row, contraction over the columns) and / or transposed (FT,
// contraction over the rows), zeros past R and C up to Rp and Cp.  TERMS 3: [hi | lo | hi] (B: [hi | hi | lo]), a third of the
// contraction each.  f_scale, ft_scale: [R] or nullptr; rows of f_scale 0 are zero whatever they hold.
template <class T, int TERMS, bool B>
__global__ __launch_bounds__(256) void loss_pack_kernel(const T* __restrict__ src, int64_t ld_src, int R, int C, int Rp, int Cp,
                                                        float scale, const float* __restrict__ f_scale,
                                                        const float* __restrict__ ft_row, const float* __restrict__ ft_all,
                                                        f16* __restrict__ F, f16* __restrict__ FT) {
  __shared__ float tile[64][65];
  const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64, t = threadIdx.x;
  const int r = r0 + (t >> 2), c = c0 + (t & 3) * 16;
  float v[16];
  const float fs = f_scale ? (r < R ? f_scale[r] : 0.f) : scale;
  const bool live = r < R && fs != 0.f;
#pragma unroll
  for (int i = 0; i < 16; i += Vec<T>::n) {
    typename Vec<T>::type x;
    const bool in = live && c + i < C;
    if (in) x = *(const typename Vec<T>::type*)(src + (size_t)r * ld_src + c + i);
#pragma unroll
    for (int j = 0; j < Vec<T>::n; ++j) v[i + j] = in ? (float)x[j] : 0.f;
  }
  // 8 elements of a row, from k kk on.  What half precision does not hold becomes a NaN: an infinite head row would make a logit
  // of -inf, which a softmax takes for a probability of 0.
  auto put = [&](f16* dst, int m, int kk, int third, const float* x) {
    f16x8 hi;
#pragma unroll
    for (int j = 0; j < 8; ++j) hi[j] = fabsf(x[j]) <= 65504.0f ? from_f32<f16>(x[j]) : (f16)NAN;
    *(f16x8*)(dst + act_index(m, kk, TERMS * third)) = hi;
    if constexpr (TERMS == 3) {
      f16x8 lo;
#pragma unroll
      for (int j = 0; j < 8; ++j) lo[j] = from_f32<f16>(x[j] - (float)hi[j]);
      *(f16x8*)(dst + act_index(m, third + kk, 3 * third)) = B ? hi : lo;
      *(f16x8*)(dst + act_index(m, 2 * third + kk, 3 * third)) = B ? lo : hi;
    }
  };
  if (F && r < Rp && c < Cp) {
    float x[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) x[j] = v[j] * fs;
    put(F, r, c, Cp, x);
    put(F, r, c + 8, Cp, x + 8);
  }
  if (FT) {
    float s = scale;
    if (ft_row) s = r < R ? ft_row[r] : 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j) tile[t >> 2][(t & 3) * 16 + j] = live ? v[j] * s : 0.f;
    __syncthreads();
    const float all = ft_all ? ft_all[0] : 1.0f;
    const int col = t & 63, rr = (t >> 6) * 16;
    if (c0 + col < Cp && r0 + rr < Rp) {
      float x[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) x[j] = tile[rr + j][col] * all;
      put(FT, c0 + col, r0 + rr, Rp, x);
      put(FT, c0 + col, r0 + rr + 8, Rp, x + 8);
    }
  }
}

// ---- epilogues -----------------------------------------------------------------------------------------------
// Partial statistics of the groups of 64 columns.  ROWS rows of a group by 64 / ROWS lanes each; a group's sums are formed in
// the same order whatever the tile, so a row's loss does not depend on the rows beside it.
struct EpiStats {
  static constexpr int kSpan = 64;
  RowTargets tg;
  float *pm, *pl, *pa;       // [groups][T]
  int T, V, n_base;          // first column of the launch
  template <int COLS, int PITCH, int ROWS>
  __device__ __forceinline__ void consume(const float* tile, int m_base, int nb, int lane, int M) const {
    constexpr int PARTS = 64 / ROWS, W = kGroup / PARTS;
    static_assert(COLS % kGroup == 0 && W % 16 == 0 && W <= 32, "whole groups, sums of 16 or of two of them a lane");
    const int r = lane % ROWS, part = lane / ROWS, m = m_base + r, mc = min(m, M - 1);
    const float zs = tg.z_scale[mc];
#pragma unroll
    for (int gg = 0; gg < COLS / kGroup; ++gg) {
      const int n0 = n_base + nb + gg * kGroup, c0 = gg * kGroup + part * W;
      const float* x = tile + r * PITCH + c0;
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const float z = x[i] * zs;
        if (n0 + part * W + i < V) mx = fmaxf(mx, z);
      }
#pragma unroll
      for (int s = ROWS; s < 64; s *= 2) mx = fmaxf(mx, __shfl_xor(mx, s, 64));
      const float ref = mx == -INFINITY ? 0.f : mx;
      float l = 0.f;                                     // sums of 16 columns, joined in pairs
#pragma unroll
      for (int h = 0; h < W / 16; ++h) {
        float s4[4] = {};
#pragma unroll
        for (int i = 16 * h; i < 16 * h + 16; ++i) {
          const float e = __builtin_amdgcn_exp2f((x[i] * zs - ref) * kLog2e);
          s4[i & 3] += n0 + part * W + i < V ? e : 0.f;
        }
        l += (s4[0] + s4[1]) + (s4[2] + s4[3]);
      }
#pragma unroll
      for (int s = ROWS; s < 64; s *= 2) l += __shfl_xor(l, s, 64);
      if (part == 0 && m < M) {
        float a = 0.f;
        if (tg.label) {
          const int c = tg.label[m] - n0;
          if (c >= 0 && c < kGroup) a = tile[r * PITCH + gg * kGroup + c] * zs;
        } else {
          const unsigned short* f = tg.first + (size_t)m * (tg.groups + 1) + n0 / kGroup;
          for (int e = n0 < V ? f[0] : 0, end = n0 < V ? f[1] : 0; e < end; ++e)
            a += tg.p[(size_t)m * tg.k + e] * (tile[r * PITCH + gg * kGroup + tg.ids[(size_t)m * tg.k + e] - n0] * zs);
        }
        if (n0 < V) {
          const size_t at = (size_t)(n0 / kGroup) * T + m;
          pm[at] = mx;
          pl[at] = l;
          pa[at] = a;
        }
      }
    }
  }
};

// dz * 2^15 as the operand of both gradient products: rows (F) and transposed (FT).  Rows T .. Tp and columns V .. are zeros.
struct EpiDz {
  static constexpr int kSpan = 64;
  RowTargets tg;
  const float* lse;
  f16 *F, *FT;
  int Tp, Np, terms;         // Np: the launch's columns
  int V, n_base;
  __device__ __forceinline__ void put(f16* dst, int m, int k, int third, const float (&x)[8]) const {
    f16x8 hi;
#pragma unroll
    for (int j = 0; j < 8; ++j) hi[j] = from_f32<f16>(x[j]);
    *(f16x8*)(dst + act_index(m, k, terms * third)) = hi;
    if (terms == 3) {
      f16x8 lo;
#pragma unroll
      for (int j = 0; j < 8; ++j) lo[j] = from_f32<f16>(x[j] - (float)hi[j]);
      *(f16x8*)(dst + act_index(m, third + k, 3 * third)) = lo;
      *(f16x8*)(dst + act_index(m, 2 * third + k, 3 * third)) = hi;
    }
  }
  template <int COLS, int PITCH, int ROWS>
  __device__ __forceinline__ void consume(const float* tile_in, int m_base, int nb, int lane, int M) const {
    float* tile = const_cast<float*>(tile_in);
    constexpr int PARTS = 64 / ROWS, CH = COLS / 8;
    const int r = lane % ROWS, part = lane / ROWS, m = m_base + r, mc = min(m, M - 1);
    const float zs = m < M ? tg.z_scale[mc] : 0.f, ls = lse[mc];
    const int label = tg.label ? tg.label[mc] : -1;
#pragma unroll
    for (int it = 0; it < CH / PARTS; ++it) {
      const int c = (it * PARTS + part) * 8, n = n_base + nb + c;
      float* x = tile + r * PITCH + c;
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float q = __builtin_amdgcn_exp2f((x[j] * zs - ls) * kLog2e);
        if (n + j == label) q -= 1.0f;
        v[j] = q;
      }
      if (!tg.label && zs != 0.f && n < V) {
        const unsigned short* f = tg.first + (size_t)m * (tg.groups + 1) + n / kGroup;
        for (int e = f[0], end = f[1]; e < end; ++e) {
          const int id = tg.ids[(size_t)m * tg.k + e];
          const float p = tg.p[(size_t)m * tg.k + e];
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] -= n + j == id ? p : 0.f;
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[j] = zs != 0.f && n + j < V ? v[j] * kDzScale : 0.f;
        x[j] = v[j];
      }
      if (F && m < Tp) put(F, m, nb + c, Np, v);
    }
    if (FT) {
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      constexpr int RC = ROWS / 8;                       // chunks of 8 rows
#pragma unroll
      for (int it = 0; it < COLS * RC / 64; ++it) {
        const int i = (it * 64 + lane) >> 5, c = (i / RC) * 32 + (lane & 31), rc = i % RC;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = tile[(rc * 8 + j) * PITCH + c];
        if (m_base + rc * 8 < Tp) put(FT, nb + c, m_base + rc * 8, Tp, v);
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
};

// grad_hidden: the pieces' products summed in float32, the last one times g / tau and rounded.
struct EpiHidden {
  static constexpr int kSpan = 64;
  float* acc;                // [T][ld]
  int ld;
  int first, last;           // of the pieces
  const float* coef;
  void* out;
  int out_f32, d;
  template <int COLS, int PITCH, int ROWS>
  __device__ __forceinline__ void consume(const float* tile, int m_base, int nb, int lane, int M) const {
    constexpr int LPR = COLS / 4, RPI = 64 / LPR, IT = ROWS / RPI;
    const int r0 = lane / LPR, c4 = (lane % LPR) * 4;
    f32x4 v[IT];
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      v[it] = *(const f32x4*)(tile + (it * RPI + r0) * PITCH + c4) * (1.0f / (kDzScale * kWeightScale));
      if (!first) v[it] += *(const f32x4*)(acc + (size_t)min(m_base + it * RPI + r0, M - 1) * ld + nb + c4);
    }
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int m = m_base + it * RPI + r0;
      if (m >= M) continue;
      if (!last) {
        *(f32x4*)(acc + (size_t)m * ld + nb + c4) = v[it];
      } else if (nb + c4 < d) {
        const f32x4 g = v[it] * coef[m];
        const size_t at = (size_t)m * d + nb + c4;
        if (out_f32) {
          *(f32x4*)((float*)out + at) = g;
        } else {
          bf16x4 o;
#pragma unroll
          for (int j = 0; j < 4; ++j) o[j] = from_f32<bf16>(g[j]);
          *(bf16x4*)((bf16*)out + at) = o;
        }
      }
    }
  }
};

// grad_head: rows of a piece of the vocabulary.
struct EpiHead {
  static constexpr int kSpan = 64;
  void* out;                 // the piece's first row
  int out_f32, d, rows;
  const float* scale;        // [1]
  template <int COLS, int PITCH, int ROWS>
  __device__ __forceinline__ void consume(const float* tile, int m_base, int nb, int lane, int M) const {
    constexpr int LPR = COLS / 4, RPI = 64 / LPR, IT = ROWS / RPI;
    const int r0 = lane / LPR, c4 = (lane % LPR) * 4;
    const float s = scale[1];
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int r = it * RPI + r0, m = m_base + r;
      const f32x4 g = *(const f32x4*)(tile + r * PITCH + c4) * s;
      if (m >= rows || nb + c4 >= d) continue;
      const size_t at = (size_t)m * d + nb + c4;
      if (out_f32) {
        *(f32x4*)((float*)out + at) = g;
      } else {
        bf16x4 o;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = from_f32<bf16>(g[j]);
        *(bf16x4*)((bf16*)out + at) = o;
      }
    }
  }
};

// The tiles of gemm_f16_variant, of which those of 64x256, 160x256 and 224x256 are run as their neighbours: EpiDz writes whole
// blocks of 64 rows, and the difference does not pay for another instance each.
template <class Epi>
static void product(const f16* A, const f16* W, int M, int N, int K, const Epi& epi, hipStream_t st) {
  const GemmF16 g{A, K, W, M, N, K, K, nullptr};
  constexpr bool four = std::is_same_v<Epi, EpiHidden> || std::is_same_v<Epi, EpiHead>;    // 128x128 waves, as residual adds
  switch (gemm_f16_variant(M, N, K, K, false, Epi::kSpan)) {
    case V_64x128_8W: launch<2, 4, 32, 32, 4, 4, 1, true, false, false>(g, epi, st); break;
    case V_64x128: case V_64x128_ROUNDS: launch<2, 2, 32, 64, 3, 3, 2, false, false, false>(g, epi, st); break;
    case V_128x128: launch<4, 2, 32, 64, 4, 4, 1, false, false, false>(g, epi, st); break;
    case V_64x256: case V_128x256: launch<2, 4, 64, 64, 3, 3, 1, false, false, false>(g, epi, st); break;
    case V_160x256: case V_192x256: launch<2, 4, 96, 64, 2, 3, 1, false, false, false>(g, epi, st); break;
    default:
      if constexpr (four) launch<2, 2, 128, 128, 2, 3, 1, false, true, false>(g, epi, st);
      else launch<4, 2, 64, 128, 2, 3, 1, false, true, false>(g, epi, st);
  }
}

// ---- joining the groups -------------------------------------------------------------------------------------------
// 16 rows a workgroup, 16 lanes a row; a lane takes every 16th group, and the lanes are joined in their order.
__global__ __launch_bounds__(256) void loss_join_kernel(const float* __restrict__ pm, const float* __restrict__ pl,
                                                        const float* __restrict__ pa, int T, int groups, RowTargets tg,
                                                        const float* __restrict__ ent, const float* __restrict__ mass,
                                                        float* __restrict__ loss, float* __restrict__ lse) {
  __shared__ float sm[16][17], sl[16][17], sa[16][17];
  const int r = threadIdx.x & 15, part = threadIdx.x >> 4, row = blockIdx.x * 16 + r;
  float m = -INFINITY, l = 0.f, a = 0.f;
  if (row < T) {
    for (int g = part; g < groups; g += 16) m = fmaxf(m, pm[(size_t)g * T + row]);
    const float ref = m == -INFINITY ? 0.f : m;
    for (int g = part; g < groups; g += 16) {
      const size_t at = (size_t)g * T + row;
      l += pl[at] * __builtin_amdgcn_exp2f((pm[at] - ref) * kLog2e);
      a += pa[at];
    }
  }
  sm[part][r] = m;
  sl[part][r] = l;
  sa[part][r] = a;
  __syncthreads();
  if (part == 0 && row < T) {
    float mm = -INFINITY;
    for (int i = 0; i < 16; ++i) mm = fmaxf(mm, sm[i][r]);
    const float ref = mm == -INFINITY ? 0.f : mm;
    l = a = 0.f;
    for (int i = 0; i < 16; ++i) {
      const float mi = sm[i][r] == -INFINITY ? 0.f : sm[i][r];
      l += sl[i][r] * __builtin_amdgcn_exp2f((mi - ref) * kLog2e);
      a += sa[i][r];
    }
    const bool live = tg.z_scale[row] != 0.f;
    const float n = ref + logf(l);
    lse[row] = live ? n : 0.f;
    loss[row] = !live ? 0.f : tg.label ? n - a : ent[row] + mass[row] * n - a;
  }
}

// ---- host ------------------------------------------------------------------------------------------------------
namespace {

struct Plan {
  int T, d, V, k, terms, groups;
  int Tp, dP, Vp;              // padded sizes of operands: contractions in whole slabs, columns in whole tiles
  int piece;                   // columns of the vocabulary at a time (gradient)
  size_t z_scale, h_scale, coef, t_max, scales, label, ids, p, ent, mass, first;
  size_t hF, hT, wF, wT, dzF, dzT, acc, pm, pl, pa, bytes;
};

int round_up(int x, int n) { return (x + n - 1) / n * n; }
int tile_up(int x) { return x <= 128 ? 128 : round_up(x, 256); }        // columns of a product

Plan make_plan(const vla_head_rows& r, int k, bool grad) {
  Plan w{};
  w.T = r.n_rows, w.d = r.d_model, w.V = r.vocab, w.k = k;
  w.terms = r.dtype == VLA_F32 ? 3 : 1;
  w.Tp = round_up(w.T, 64), w.dP = tile_up(w.d), w.Vp = tile_up(w.V);
  w.groups = (w.V + kGroup - 1) / kGroup;
  const size_t half = 2 * (size_t)w.terms;
  w.piece = w.Vp;
  if (grad) {                                                       // dz, both ways, within 256 MB
    const size_t cols = (((size_t)256 << 20) / (2 * half * w.Tp)) & ~(size_t)255;
    const int most = cols < 256 ? 256 : cols > (size_t)w.Vp ? w.Vp : (int)cols;
    const int n = (w.Vp + most - 1) / most;
    w.piece = n == 1 ? w.Vp : round_up((w.Vp + n - 1) / n, 256);
  }
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t o = at; at += (bytes + 255) / 256 * 256; return o; };
  const size_t T = (size_t)w.T;
  w.z_scale = take(4 * T), w.h_scale = take(4 * T);
  if (k) {
    w.ids = take(4 * T * k), w.p = take(4 * T * k), w.ent = take(4 * T), w.mass = take(4 * T);
    w.first = take(2 * T * (w.groups + 1));
  } else {
    w.label = take(4 * T);
  }
  w.hF = take((size_t)w.Tp * w.dP * half);
  w.wF = take((size_t)w.piece * w.dP * half);
  if (grad) {
    w.coef = take(4 * T), w.t_max = take(4 * T), w.scales = take(8);
    w.hT = take((size_t)w.Tp * w.dP * half);
    w.wT = take((size_t)w.piece * w.dP * half);
    w.dzF = take((size_t)w.Tp * w.piece * half), w.dzT = take((size_t)w.Tp * w.piece * half);
    if (w.piece < w.Vp) w.acc = take(4 * T * w.dP);
  } else {
    w.pm = take(4 * T * w.groups), w.pl = take(4 * T * w.groups), w.pa = take(4 * T * w.groups);
  }
  w.bytes = at;
  return w;
}

int check_rows(const vla_head_rows* r, bool pointers) {
  if (!r) return VLA_E_NULL;
  if (r->dtype != VLA_F32 && r->dtype != VLA_BF16) return VLA_E_CONFIG;
  const int unit = r->dtype == VLA_F32 ? 4 : 8;
  if (r->n_rows < 1 || r->n_rows > 1 << 20 || r->vocab < 1 || r->vocab > 1 << 20) return VLA_E_SHAPE;
  if (r->d_model < unit || r->d_model > 1 << 15 || r->d_model % unit) return VLA_E_SHAPE;
  if (!(r->temperature >= 0.f) || r->temperature > 3e38f) return VLA_E_SHAPE;
  if (!pointers) return VLA_OK;
  if (!r->hidden || !r->head) return VLA_E_NULL;
  if (r->ld_hidden < r->d_model || r->ld_head < r->d_model || r->ld_hidden % unit || r->ld_head % unit) return VLA_E_SHAPE;
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
  *plan = make_plan(*r, t.k, grad);
  return work_bytes < plan->bytes ? VLA_E_CAPACITY : VLA_OK;
}

template <class T>
RowTargets prepare(const Plan& w, const vla_head_rows& r, const Targets& t, const float* g, char* work, hipStream_t st) {
  auto f = [&](size_t o) { return (float*)(work + o); };
  const float tau = r.temperature > 0.f ? r.temperature : 1.0f;
  const PrepOut out{f(w.z_scale), f(w.h_scale), g ? f(w.coef) : nullptr, g ? f(w.t_max) : nullptr, (int32_t*)(work + w.label),
                    (int32_t*)(work + w.ids), f(w.p), f(w.ent), f(w.mass), (unsigned short*)(work + w.first)};
  hipLaunchKernelGGL((loss_prep_kernel<T>), dim3(w.T), dim3(256), 0, st, (const T*)r.hidden, r.ld_hidden, w.d, w.V, 1.0f / tau,
                     t.labels, t.top_logits, t.top_ids, w.k, w.groups, g, out);
  return RowTargets{out.z_scale, w.k ? nullptr : out.label, out.ids, out.p, out.first, w.k, w.groups};
}

template <class T, bool B>
void pack(const T* src, int64_t ld, int R, int C, int Rp, int Cp, float scale, const float* f_scale, const float* ft_row,
          const float* ft_all, f16* F, f16* FT, hipStream_t st) {
  constexpr int TERMS = std::is_same_v<T, float> ? 3 : 1;
  hipLaunchKernelGGL((loss_pack_kernel<T, TERMS, B>), dim3((Cp + 63) / 64, (Rp + 63) / 64), dim3(256), 0, st, src, ld, R, C, Rp,
                     Cp, scale, f_scale, ft_row, ft_all, F, FT);
}

template <class T>
int run_loss(const Plan& w, const vla_head_rows& r, const Targets& t, float* loss, float* lse, char* work, hipStream_t st) {
  const RowTargets tg = prepare<T>(w, r, t, nullptr, work, st);
  auto f = [&](size_t o) { return (float*)(work + o); };
  f16 *hF = (f16*)(work + w.hF), *wF = (f16*)(work + w.wF);
  pack<T, false>((const T*)r.hidden, r.ld_hidden, w.T, w.d, w.Tp, w.dP, 1.0f, f(w.h_scale), nullptr, nullptr, hF, nullptr, st);
  pack<T, true>((const T*)r.head, r.ld_head, w.V, w.d, w.Vp, w.dP, kWeightScale, nullptr, nullptr, nullptr, wF, nullptr, st);
  product(hF, wF, w.T, w.Vp, w.terms * w.dP, EpiStats{tg, f(w.pm), f(w.pl), f(w.pa), w.T, w.V, 0}, st);
  hipLaunchKernelGGL(loss_join_kernel, dim3((w.T + 15) / 16), dim3(256), 0, st, f(w.pm), f(w.pl), f(w.pa), w.T, w.groups, tg,
                     w.k ? f(w.ent) : nullptr, w.k ? f(w.mass) : nullptr, loss, lse);
  return hipGetLastError() == hipSuccess ? VLA_OK : VLA_E_HIP;
}

template <class T>
int run_grad(const Plan& w, const vla_head_rows& r, const Targets& t, const float* lse, const float* g, void* gh, void* gw,
             char* work, hipStream_t st) {
  const RowTargets tg = prepare<T>(w, r, t, g, work, st);
  auto f = [&](size_t o) { return (float*)(work + o); };
  auto h = [&](size_t o) { return (f16*)(work + o); };
  const int out_f32 = std::is_same_v<T, float>;
  hipLaunchKernelGGL(loss_scale_kernel, dim3(1), dim3(256), 0, st, f(w.t_max), w.T, f(w.scales));
  pack<T, false>((const T*)r.hidden, r.ld_hidden, w.T, w.d, w.Tp, w.dP, 1.0f, f(w.h_scale), nullptr, nullptr, h(w.hF), nullptr, st);
  if (gw) pack<T, true>((const T*)r.hidden, r.ld_hidden, w.T, w.d, w.Tp, w.dP, 1.0f, f(w.h_scale), f(w.coef), f(w.scales), nullptr, h(w.hT), st);
  for (int n0 = 0; n0 < w.Vp; n0 += w.piece) {
    const int N = min(w.piece, w.Vp - n0), rows = min(N, w.V - n0);
    pack<T, true>((const T*)r.head + (size_t)n0 * r.ld_head, r.ld_head, rows, w.d, N, w.dP, kWeightScale, nullptr, nullptr, nullptr,
                  h(w.wF), gh ? h(w.wT) : nullptr, st);
    product(h(w.hF), h(w.wF), w.T, N, w.terms * w.dP,
            EpiDz{tg, lse, gh ? h(w.dzF) : nullptr, gw ? h(w.dzT) : nullptr, w.Tp, N, w.terms, w.V, n0}, st);
    if (gh)
      product(h(w.dzF), h(w.wT), w.T, w.dP, w.terms * N,
              EpiHidden{f(w.acc), w.dP, n0 == 0, n0 + N == w.Vp, f(w.coef), gh, out_f32, w.d}, st);
    if (gw)
      product(h(w.dzT), h(w.hT), N, w.dP, w.terms * w.Tp,
              EpiHead{(T*)gw + (size_t)n0 * w.d, out_f32, w.d, rows, f(w.scales)}, st);
  }
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
