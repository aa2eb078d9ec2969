// Row-wise and small kernels of the VLA policy path: prefix assembly, RMSNorm, the action head
// (final norm + slimmed LM head), token selection with log-probs and de-tokenisation, rotary
// tables, token maps.
#include "common.h"

namespace vla {

// ---- token maps ---------------------------------------------------------------------------------
// Packed prefix token t belongs to sequence b of the call with cu_seq[b] <= t < cu_seq[b+1], where
// cu_seq[b] = cu_patch[b] + cu_instr[b]; sequence b lives in cache slot slot_map[b] (b itself without a map).
// tok_src >= 0 is a row of patch_emb, tok_src < 0 is instruction id number -1 - tok_src.
__global__ void token_maps_kernel(const int32_t* __restrict__ cu_patch, const int32_t* __restrict__ cu_instr,
                                  const int32_t* __restrict__ slot_map, int B, int T, int32_t* tok_seq,
                                  int32_t* tok_pos, int32_t* tok_src, int32_t* last_row, int32_t* seq_len) {
  const int t = blockIdx.x * blockDim.x + threadIdx.x;
  if (t < B) {
    const int end = cu_patch[t + 1] + cu_instr[t + 1];
    last_row[t] = end - 1;
    seq_len[slot_map ? slot_map[t] : t] = end - (cu_patch[t] + cu_instr[t]);
  }
  if (t >= T) return;
  int lo = 0, hi = B;                       // find b with cu_seq[b] <= t < cu_seq[b+1]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu_patch[mid] + cu_instr[mid] <= t) lo = mid; else hi = mid;
  }
  const int b = lo;
  const int pos = t - (cu_patch[b] + cu_instr[b]);
  const int np = cu_patch[b + 1] - cu_patch[b];
  tok_seq[t] = slot_map ? slot_map[b] : b;
  tok_pos[t] = pos;
  tok_src[t] = pos < np ? cu_patch[b] + pos : -1 - (cu_instr[b] + pos - np);
}

void build_token_maps(const int32_t* cu_patch_dev, const int32_t* cu_instr_dev, const int32_t* slot_map, int B,
                      int T_tokens, int32_t* tok_seq, int32_t* tok_pos, int32_t* tok_src, int32_t* last_row,
                      int32_t* seq_len, hipStream_t st) {
  const int n = T_tokens > B ? T_tokens : B;
  hipLaunchKernelGGL(token_maps_kernel, dim3((n + 255) / 256), dim3(256), 0, st, cu_patch_dev, cu_instr_dev,
                     slot_map, B, T_tokens, tok_seq, tok_pos, tok_src, last_row, seq_len);
}

// ---- rotary table ---------------------------------------------------------------------------------
// cos/sin of pos * theta^(-2i/hd), evaluated in double so that the float32 path keeps 1e-4 logits.
__global__ void rope_table_kernel(float* cos_t, float* sin_t, int max_seq, int half, double theta) {
  const int idx = blockIdx.x * blockDim.x + threadIdx.x;
  if (idx >= max_seq * half) return;
  const int pos = idx / half, i = idx - pos * half;
  const double inv = pow(theta, -(double)i / (double)half);
  const double ang = (double)pos * inv;
  cos_t[idx] = (float)cos(ang);
  sin_t[idx] = (float)sin(ang);
}
void rope_table(float* cos_t, float* sin_t, int max_seq, int head_dim, float theta, hipStream_t st) {
  const int n = max_seq * (head_dim / 2);
  hipLaunchKernelGGL(rope_table_kernel, dim3((n + 255) / 256), dim3(256), 0, st, cos_t, sin_t, max_seq,
                     head_dim / 2, (double)theta);
}

// ---- copies ---------------------------------------------------------------------------------------
template <class T>
__global__ void convert_kernel(const T* src, float* dst, size_t n) {
  const size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) dst[i] = to_f32(src[i]);
}
template <class T>
void convert_copy(const T* src, float* dst, size_t n, hipStream_t st) {
  hipLaunchKernelGGL(convert_kernel<T>, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, src, dst, n);
}
template void convert_copy<float>(const float*, float*, size_t, hipStream_t);
template void convert_copy<bf16>(const bf16*, float*, size_t, hipStream_t);

template <class T>
__global__ void copy_kernel(const T* src, T* dst, size_t n) {
  size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
  const size_t stride = (size_t)gridDim.x * blockDim.x;
  for (; i < n; i += stride) dst[i] = src[i];
}
template <class T>
void plain_copy(const T* src, T* dst, size_t n, hipStream_t st) {
  size_t blocks = (n + 255) / 256;
  if (blocks > 65536) blocks = 65536;
  hipLaunchKernelGGL(copy_kernel<T>, dim3((unsigned)blocks), dim3(256), 0, st, src, dst, n);
}
template void plain_copy<float>(const float*, float*, size_t, hipStream_t);
template void plain_copy<bf16>(const bf16*, bf16*, size_t, hipStream_t);

// ---- prefix assembly ------------------------------------------------------------------------------
// x[t, :] = patch_emb[src] or embed[instr_ids[-1-src]], widened to the float32 residual stream.
template <class T>
__global__ void assemble_kernel(const T* __restrict__ patch_emb, const int32_t* __restrict__ instr_ids,
                                const T* __restrict__ embed, const int32_t* __restrict__ tok_src,
                                float* __restrict__ x, int d, int vocab) {
  const int t = blockIdx.x;
  const int src = tok_src[t];
  int id = src >= 0 ? 0 : instr_ids[-1 - src];
  id = id < 0 ? 0 : (id >= vocab ? vocab - 1 : id);   // ids come from device memory: stay in bounds
  const T* row = src >= 0 ? patch_emb + (size_t)src * d : embed + (size_t)id * d;
  float* out = x + (size_t)t * d;
  for (int i = threadIdx.x; i < d; i += blockDim.x) out[i] = to_f32(row[i]);
}
template <class T>
void assemble_prefix(const T* patch_emb, const int32_t* instr_ids, const T* embed, const int32_t* tok_src,
                     float* x, int T_tokens, int d, int vocab, hipStream_t st) {
  hipLaunchKernelGGL(assemble_kernel<T>, dim3(T_tokens), dim3(256), 0, st, patch_emb, instr_ids, embed,
                     tok_src, x, d, vocab);
}
template void assemble_prefix<float>(const float*, const int32_t*, const float*, const int32_t*, float*, int,
                                     int, int, hipStream_t);
template void assemble_prefix<bf16>(const bf16*, const int32_t*, const bf16*, const int32_t*, float*, int, int,
                                    int, hipStream_t);

// ---- last-layer tail: only the rows that feed the head go through the last O / feed-forward ------------
// Row i of the compact set is packed row need[i]: its attention output goes to fragment order
// [i/32][k/16][lane][8] (what the weight-streaming GEMMs read), its residual row to x_c[i].
__global__ __launch_bounds__(256) void gather_tail_kernel(const f16* __restrict__ att, int ld_att, int lo8,
                                                          const float* __restrict__ x,
                                                          const int32_t* __restrict__ need, int d,
                                                          f16* __restrict__ att_frag, f16* __restrict__ att_frag_lo,
                                                          float* __restrict__ x_c) {
  typedef __attribute__((ext_vector_type(2))) int i32x2;
  const int i = blockIdx.x, src = need[i];
  for (int k = threadIdx.x * 8; k < d; k += blockDim.x * 8) {
    const size_t to = act_index(i, k, d);
    *(u32x4*)(att_frag + to) = *(const u32x4*)(att + act_index(src, k, ld_att));
    if (att_frag_lo) {
      if (lo8) {                             // low terms as bytes: widened to half precision (exact)
        const i32x2 w = *(const i32x2*)((const unsigned char*)att + act_lo8_index(src, k, ld_att, d));
        f16x8 h;
        h[0] = (f16)unpack_lo8(w[0], 0); h[1] = (f16)unpack_lo8(w[0], 1); h[2] = (f16)unpack_lo8(w[0], 2); h[3] = (f16)unpack_lo8(w[0], 3);
        h[4] = (f16)unpack_lo8(w[1], 0); h[5] = (f16)unpack_lo8(w[1], 1); h[6] = (f16)unpack_lo8(w[1], 2); h[7] = (f16)unpack_lo8(w[1], 3);
        *(f16x8*)(att_frag_lo + to) = h;
      } else {
        *(u32x4*)(att_frag_lo + to) = *(const u32x4*)(att + act_index(src, d + k, ld_att));
      }
    }
  }
  const f32x4* xr = (const f32x4*)(x + (size_t)src * d);
  f32x4* xo = (f32x4*)(x_c + (size_t)i * d);
  for (int j = threadIdx.x; j < (d >> 2); j += blockDim.x) xo[j] = xr[j];
}
void gather_tail(const f16* att, int ld_att, bool lo8, const float* x, const int32_t* need, int n, int d,
                 f16* att_frag, f16* att_frag_lo, float* x_c, hipStream_t st) {
  hipLaunchKernelGGL(gather_tail_kernel, dim3(n), dim3(256), 0, st, att, ld_att, lo8 ? 1 : 0, x, need, d, att_frag,
                     att_frag_lo, x_c);
}
__global__ __launch_bounds__(256) void scatter_tail_kernel(const float* __restrict__ x_c,
                                                           const int32_t* __restrict__ need, int d,
                                                           float* __restrict__ x) {
  const int i = blockIdx.x;
  const f32x4* xr = (const f32x4*)(x_c + (size_t)i * d);
  f32x4* xo = (f32x4*)(x + (size_t)need[i] * d);
  for (int j = threadIdx.x; j < (d >> 2); j += blockDim.x) xo[j] = xr[j];
}
void scatter_tail(const float* x_c, const int32_t* need, int n, int d, float* x, hipStream_t st) {
  hipLaunchKernelGGL(scatter_tail_kernel, dim3(n), dim3(256), 0, st, x_c, need, d, x);
}

// ---- chunk pass: every sequence is [prefix ; n_tail fed tokens], logits wanted at its last n_tail + 1 rows ----
// cu2[b] = cu_instr[b] + b * n_tail are the offsets of the merged id stream.
__global__ void merge_tail_kernel(const int32_t* __restrict__ instr_ids, const int32_t* __restrict__ cu2,
                                  const int32_t* __restrict__ tail, int B, int n_tail, int total,
                                  int32_t* __restrict__ out) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= total) return;
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu2[mid] <= i) lo = mid; else hi = mid;
  }
  const int b = lo, j = i - cu2[b];
  const int li = cu2[b + 1] - cu2[b] - n_tail;
  out[i] = j < li ? instr_ids[cu2[b] - b * n_tail + j] : tail[b * n_tail + (j - li)];
}
void merge_tail_ids(const int32_t* instr_ids, const int32_t* cu2_dev, const int32_t* tail, int B, int n_tail,
                    int total, int32_t* out, hipStream_t st) {
  if (total <= 0) return;
  hipLaunchKernelGGL(merge_tail_kernel, dim3((total + 255) / 256), dim3(256), 0, st, instr_ids, cu2_dev, tail, B,
                     n_tail, total, out);
}

// tail[b, j] = placeholder (tokens == nullptr) or the vocabulary id of stored bin tokens[b, j], j < K - 1
__global__ void tail_ids_kernel(const int32_t* __restrict__ tokens, int B, int K, int id0, int A, int placeholder,
                                int32_t* __restrict__ tail) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= B * (K - 1)) return;
  const int b = i / (K - 1), j = i - b * (K - 1);
  if (tokens) {
    int t = tokens[b * K + j];
    t = t < 0 ? 0 : (t >= A ? A - 1 : t);
    tail[i] = id0 + t;
  } else {
    tail[i] = placeholder;
  }
}
void tail_ids(const int32_t* tokens, int B, int K, int id0, int A, int placeholder, int32_t* tail, hipStream_t st) {
  const int n = B * (K - 1);
  if (n <= 0) return;
  hipLaunchKernelGGL(tail_ids_kernel, dim3((n + 255) / 256), dim3(256), 0, st, tokens, B, K, id0, A, placeholder, tail);
}

// rows[b * K + k] = packed row that emits action token k of sequence b
__global__ void chunk_rows_kernel(const int32_t* __restrict__ last_row, int B, int K, int32_t* __restrict__ rows) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= B * K) return;
  const int b = i / K, k = i - b * K;
  rows[i] = last_row[b] - (K - 1) + k;
}
void chunk_rows(const int32_t* last_row, int B, int K, int32_t* rows, hipStream_t st) {
  hipLaunchKernelGGL(chunk_rows_kernel, dim3((B * K + 255) / 256), dim3(256), 0, st, last_row, B, K, rows);
}

// One wave per (sequence, token): log-prob of a given bin under log_softmax(logits / tau), and with the
// behaviour log-prob mu the importance ratio rho = exp(logp - mu) and rho * exp(-(log rho / sigma)^2 / 2).
__global__ __launch_bounds__(64) void score_kernel(const float* __restrict__ logits, int A, float temperature,
                                                   const int32_t* __restrict__ tokens,
                                                   const float* __restrict__ mu, float sigma,
                                                   float* __restrict__ logp_out, float* __restrict__ ratio_out,
                                                   float* __restrict__ weight_out) {
  const int r = blockIdx.x, lane = threadIdx.x;
  const float* z = logits + (size_t)r * A;
  const float inv_tau = temperature > 0.f ? 1.0f / temperature : 1.0f;
  float zmax = -INFINITY;
  for (int j = lane; j < A; j += 64) zmax = fmaxf(zmax, z[j] * inv_tau);
  zmax = wave_max(zmax);
  float se = 0.f;
  for (int j = lane; j < A; j += 64) se += expf(z[j] * inv_tau - zmax);
  se = wave_sum(se);
  if (lane == 0) {
    int t = tokens[r];
    t = t < 0 ? 0 : (t >= A ? A - 1 : t);
    const float logp = z[t] * inv_tau - zmax - logf(se);
    logp_out[r] = logp;
    if (mu) {
      const float lr = logp - mu[r];
      const float rho = expf(lr);
      const float q = lr / sigma;
      if (ratio_out) ratio_out[r] = rho;
      if (weight_out) weight_out[r] = rho * expf(-0.5f * q * q);
    }
  }
}
void score_rows(const float* logits, int rows, int A, float temperature, const int32_t* tokens, const float* mu,
                float sigma, float* logp_out, float* ratio_out, float* weight_out, hipStream_t st) {
  hipLaunchKernelGGL(score_kernel, dim3(rows), dim3(64), 0, st, logits, A, temperature, tokens, mu, sigma, logp_out,
                     ratio_out, weight_out);
}

// ---- RMSNorm ----------------------------------------------------------------------------------------
// out[r, :] = x[row, :] * gain / sqrt(mean(x^2) + eps), statistics in float32.
__device__ __forceinline__ float block_sum_256(float v, float* red) {
  v = wave_sum(v);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  __syncthreads();
  if (lane == 0) red[wave] = v;
  __syncthreads();
  return red[0] + red[1] + red[2] + red[3];
}

// A barrier that orders the LDS alone: __syncthreads() would wait for the stores to global memory as well.
__device__ __forceinline__ void lds_barrier() {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#endif
}
// The rows of a prefill, to fragment order: ROWS rows a workgroup, WPR waves each, HELD pieces of 256 elements a wave in registers
// between the two passes.  Bound by HBM, few rows by latency.  The 16-byte pieces of a row lie 512 bytes apart, those of the
// workgroup's rows side by side: the output goes through LDS, SPAN columns at a time, and leaves as segments of 16 * ROWS bytes, a
// block's 32 rows from one XCD, whose L2 puts the lines together.  One row a workgroup (few rows) leaves as it is, in the 8
// bytes of a lane.  ONCE: the rows outgrow the last-level cache and are read as data that does not come again, which leaves the
// lines in the L2 until they are whole.
template <int ROWS, int WPR, int HELD, bool ONCE>
__global__ __launch_bounds__(ROWS * WPR * 64) void rmsnorm_kernel(const float* __restrict__ x, const float* __restrict__ gain,
                                                                  f16* __restrict__ out, int rows, int d, float eps, int ldo, int lo_mode) {
  typedef __attribute__((ext_vector_type(4))) f16 f16x4;
  constexpr int SP = HELD < 4 ? HELD : 4, STEP = WPR * 256, SPAN = SP * STEP, NT = ROWS * WPR * 64;
  constexpr int PITCH = SPAN + 16;                         // (spreads the rows of a read over the banks)
  constexpr bool DIRECT = ROWS == 1;                       // a lane's four columns go out as they are
  __shared__ __attribute__((aligned(16))) f16 s_hi[DIRECT ? 1 : ROWS][DIRECT ? 8 : PITCH];
  __shared__ __attribute__((aligned(16))) f16 s_lo[DIRECT ? 1 : ROWS][DIRECT ? 8 : PITCH];     // or bytes, SPAN + 32 a row
  unsigned char* s_lo8 = (unsigned char*)s_lo;
  const int r0 = ((blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3)) * ROWS;
  if (r0 >= rows) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / WPR;
  const int c0 = (threadIdx.x % (WPR * 64)) * 4;
  const float* row = x + (size_t)min(r0 + wave, rows - 1) * d;
  f32x4 held[HELD];
#pragma unroll
  for (int it = 0; it < HELD; ++it) held[it] = c0 + it * STEP < d ? load_once<ONCE>((const f32x4*)(row + c0 + it * STEP)) : f32x4{0.f, 0.f, 0.f, 0.f};
  f32x4 g[SP];
  auto gains = [&](int k0) {                               // of the next span
#pragma unroll
    for (int i = 0; i < SP; ++i)
      if (k0 + c0 + i * STEP < d) g[i] = *(const f32x4*)(gain + k0 + c0 + i * STEP);
  };
  gains(0);
  // Whatever the form, the squares are added in one order: of a lane's pieces of 256 elements those of one number modulo four in a
  // sum, a butterfly over the lanes for each of the four, ((s0 + s1) + s2) + s3.
  static_assert(4 % WPR == 0 && HELD % (4 / WPR) == 0, "a wave has the pieces of 4 / WPR of the sums");
  constexpr int NS = 4 / WPR;
  float ss[NS] = {};
  auto squares = [&](const f32x4& v, int s) { ss[s] += fmaf(v[3], v[3], fmaf(v[2], v[2], fmaf(v[0], v[0], v[1] * v[1]))); };
#pragma unroll
  for (int it = 0; it < HELD; ++it) squares(held[it], it % NS);
  for (int k = c0 + HELD * STEP; k < d; k += NS * STEP)
#pragma unroll
    for (int s = 0; s < NS; ++s)
      if (k + s * STEP < d) squares(*(const f32x4*)(row + k + s * STEP), s);
#pragma unroll
  for (int s = 0; s < NS; ++s) ss[s] = wave_sum(ss[s]);
  float sum;
  if constexpr (WPR == 1) {
    sum = ((ss[0] + ss[1]) + ss[2]) + ss[3];
  } else {
    __shared__ float s_sum[ROWS][4];                       // (sum s is that of wave s % WPR)
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % WPR;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int s = 0; s < NS; ++s) s_sum[wave][s * WPR + w] = ss[s];
    }
    lds_barrier();
    sum = ((s_sum[wave][0] + s_sum[wave][1]) + s_sum[wave][2]) + s_sum[wave][3];
  }
  const float inv = 1.0f / sqrtf(sum / (float)d + eps);
  auto put = [&](int k0, int c, const f32x4& v, const f32x4& g) {      // columns c .. + 3 of the span at k0
    f16x4 q, qe;
    float e[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float h = v[j] * inv * g[j];
      q[j] = from_f32<f16>(h);
      e[j] = h - to_f32(q[j]);
      qe[j] = from_f32<f16>(e[j]);
    }
    if constexpr (DIRECT) {
      *(f16x4*)(out + act_index(r0, k0 + c, ldo)) = q;
      if (lo_mode == 1) *(f16x4*)(out + act_index(r0, d + k0 + c, ldo)) = qe;
      if (lo_mode == 2) *(int*)((unsigned char*)out + act_lo8_index(r0, k0 + c, ldo, d)) = pack_lo8(e[0], e[1], e[2], e[3]);
    } else {
      *(f16x4*)&s_hi[wave][c] = q;
      if (lo_mode == 1) *(f16x4*)&s_lo[wave][c] = qe;
      if (lo_mode == 2) *(int*)(s_lo8 + wave * (SPAN + 32) + c) = pack_lo8(e[0], e[1], e[2], e[3]);
    }
  };
  // the rows of a span, side by side; low terms of lo_mode 1 go to column d + k, of 2 as bytes behind the block's high terms
  auto leave = [&](int k0) {
    if constexpr (DIRECT) return;
    lds_barrier();
    const int n = min(d - k0, SPAN), m = r0 + threadIdx.x % ROWS;
    const f16 *hi = s_hi[threadIdx.x % ROWS], *lo = s_lo[threadIdx.x % ROWS];
    const unsigned char* lo8 = s_lo8 + threadIdx.x % ROWS * (SPAN + 32);
    if (m < rows) {
      for (int c = threadIdx.x / ROWS * 8; c < n; c += NT / ROWS * 8) {
        *(u32x4*)(out + act_index(m, k0 + c, ldo)) = *(const u32x4*)(hi + c);
        if (lo_mode == 1) *(u32x4*)(out + act_index(m, d + k0 + c, ldo)) = *(const u32x4*)(lo + c);
      }
      if (lo_mode == 2)
        for (int c = threadIdx.x / ROWS * 16; c < n; c += NT / ROWS * 16) *(u32x4*)((unsigned char*)out + act_lo8_index(m, k0 + c, ldo, d)) = *(const u32x4*)(lo8 + c);
    }
    lds_barrier();
  };
#pragma unroll
  for (int sp = 0; sp < HELD / SP; ++sp) {
    if (sp * SPAN < d) {                                   // (uniform)
#pragma unroll
      for (int i = 0; i < SP; ++i)
        if (sp * SPAN + c0 + i * STEP < d) put(sp * SPAN, c0 + i * STEP, held[sp * SP + i], g[i]);
      gains((sp + 1) * SPAN);
      leave(sp * SPAN);
    }
  }
  for (int k0 = HELD * STEP; k0 < d; k0 += SPAN) {
    for (int c = c0; c < SPAN && k0 + c < d; c += STEP) put(k0, c, *(const f32x4*)(row + k0 + c), *(const f32x4*)(gain + k0 + c));
    leave(k0);
  }
}
// us, rows of d by one workgroup a row / these forms (4096 columns in registers at most / these, where rows are wider):
//   d 768   288 rows 2.4 / 2.4, 580 2.5 / 2.5, 870 2.7 / 2.7, 1400 3.1 / 3.0, 2500 4.1 / 3.7, 9280 9.7 / 8.6; with low terms 580 rows
//           2.6 / 2.7, 870 2.8 / 2.9, 1400 3.3 / 3.2
//   d 4096  288 rows 3.2 / 3.5, 580 3.7 / 4.6, 1400 5.6 / 6.6, 2500 11.3 / 12.6, 9280 33.8 / 35.6, 18560 79 / 80 (93 without ONCE);
//           with low terms 288 3.5 / 4.1, 1400 6.9 / 8.8, 9280 39 to 41 / 41 to 46, 18560 92 / 91 (eight rows a workgroup, and one or two
//           waves a row of sixteen and eight pieces, are 3 to 40 % slower than these)
//   d 5120  288 rows 3.5 / 4.0 (4.5), 2000 10.8 / 12.7, 4640 22.6 / 25.0 (26.5), 18560 100 / 102 (100), with low terms 118 / 125 (152)
//   d 8192  288 rows 4.7 / 5.3 (6.1), 1400 12.8 / 14.2 (15.0), 4640 34 / 37 (45), 9280 84 / 83 (101), with low terms 99 / 100 (135)
// One row a workgroup wins while a compute unit has three or four of them (two where a row is four pieces a wave).
void rmsnorm(const float* x, const float* gain, f16* out, int rows, int d, float eps, int lo_mode, hipStream_t st) {
  const int ldo = lo_mode == 1 ? 2 * d : (lo_mode == 2 ? d + d / 2 : d);
  auto launch = [&](auto kern, int r, int wpr) {
    hipLaunchKernelGGL(kern, dim3(((rows + r - 1) / r + 7) / 8 * 8), dim3(r * wpr * 64), 0, st, x, gain, out, rows, d, eps, ldo, lo_mode);
  };
  const bool once = (size_t)rows * d * sizeof(float) > 245'000'000;
  if (d <= 1024) {
    if (rows <= 1000) launch(rmsnorm_kernel<1, 4, 1, false>, 1, 4);
    else if (rows <= 3500) launch(rmsnorm_kernel<2, 2, 2, false>, 2, 2);
    else launch(rmsnorm_kernel<4, 1, 4, false>, 4, 1);
  } else if (d > 4096 && rows <= 700) {
    launch(rmsnorm_kernel<1, 4, 8, false>, 1, 4);
  } else if (d > 6144 || (d > 4096 && rows > 3000)) {      // (up to there a second read of what is past 4096 costs less than wider spans)
    if (once) launch(rmsnorm_kernel<2, 4, 8, true>, 2, 4);
    else launch(rmsnorm_kernel<2, 4, 8, false>, 2, 4);
  } else {
    if (rows <= 500) launch(rmsnorm_kernel<1, 4, 4, false>, 1, 4);
    else if (rows <= 1400) launch(rmsnorm_kernel<2, 4, 4, false>, 2, 4);
    else if (once) launch(rmsnorm_kernel<4, 2, 8, true>, 4, 2);
    else launch(rmsnorm_kernel<4, 2, 8, false>, 4, 2);
  }
}

// ---- action head ------------------------------------------------------------------------------------
// Workgroup (b, h): final RMSNorm of a hidden row (float32, kept in LDS), then `rows` action rows of the slimmed head, one
// row per wave at a time, lanes striding over d with a wave reduction per output.  A few hidden rows are bound by latency:
// the action rows are then spread over more workgroups (4 a workgroup, one per wave; the norm is recomputed by each, 16 KiB
// from L2).  DEEP: eight loads of an action row in flight.  It takes a row long enough to fill them, the chip being full
// of waves otherwise.  The sum of an output does not depend on either.  256 bins, us, one load at a time / eight:
//   d 4096  1 hidden row 9.4 / 5.4, 64 rows 46 / 15, 1792 rows 345 / 230     d 2048  64 rows 25 / 10, 1792 rows 161 / 118
//   d 1536  64 rows 20 / 20, 256 rows 22 / 38, 1792 rows 118 / 160           d 768   256 rows 14 / 21, 1792 rows 69 / 96
// (Four hidden rows a workgroup, to share the reads of the head: 341, 164, 138 and 91 us at 1792 rows; its LDS leaves too
// few waves.)
__device__ __forceinline__ f32x4 load4_f32(const float* p) { return *(const f32x4*)p; }
__device__ __forceinline__ f32x4 load4_f32(const bf16* p) {
  const bf16x4 v = *(const bf16x4*)p;
  return f32x4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
}
template <class T, bool DEEP>
__global__ __launch_bounds__(256) void head_kernel(const float* __restrict__ x, const int32_t* __restrict__ row_index,
                                                   const float* __restrict__ gain, const T* __restrict__ w_head,
                                                   float* __restrict__ logits, int ld_logits, int d, int A, int rows,
                                                   float eps) {
  extern __shared__ __attribute__((aligned(16))) float hrow[];   // [d]
  __shared__ float red[4];
  const int b = blockIdx.x;
  const float* row = x + (size_t)(row_index ? row_index[b] : b) * d;
  float ss = 0.f;
  for (int i = threadIdx.x * 4; i < d; i += 1024) {
    const float4 v = *(const float4*)(row + i);
    ss += v.x * v.x + v.y * v.y + v.z * v.z + v.w * v.w;
  }
  ss = block_sum_256(ss, red);
  const float inv = 1.0f / sqrtf(ss / (float)d + eps);
  for (int i = threadIdx.x * 4; i < d; i += 1024) {
    const float4 v = *(const float4*)(row + i);
    const float4 g = *(const float4*)(gain + i);
    *(float4*)(hrow + i) = make_float4(v.x * inv * g.x, v.y * inv * g.y, v.z * inv * g.z, v.w * inv * g.w);
  }
  __syncthreads();
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int j0 = blockIdx.y * rows;
  for (int j = j0 + wave; j < min(j0 + rows, A); j += 4) {
    const T* w = w_head + (size_t)j * d;
    float acc = 0.f;
    auto columns = [&](int i) {
      const f32x4 wv = load4_f32(w + i), h = *(const f32x4*)(hrow + i);
      acc += wv[0] * h[0] + wv[1] * h[1] + wv[2] * h[2] + wv[3] * h[3];
    };
    if constexpr (DEEP) {
#pragma unroll 8
      for (int i = lane * 4; i < d; i += 256) columns(i);
    } else {
      for (int i = lane * 4; i < d; i += 256) columns(i);
    }
    acc = wave_sum(acc);
    if (lane == 0) logits[(size_t)b * ld_logits + j] = acc;
  }
}
template <class T, bool DEEP>
static void launch_head(const float* x, const int32_t* row_index, const float* gain, const T* w_head, float* logits,
                        int ld_logits, int B, int d, int A, int rows, float eps, hipStream_t st) {
  auto kern = head_kernel<T, DEEP>;
  static bool attr_set = false;
  if (!attr_set) {
    (void)hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, 64 * 1024);
    attr_set = true;
  }
  hipLaunchKernelGGL(kern, dim3(B, (A + rows - 1) / rows), dim3(256), (size_t)d * sizeof(float), st, x, row_index, gain,
                     w_head, logits, ld_logits, d, A, rows, eps);
}
template <class T>
void head_logits(const float* x, const int32_t* row_index, const float* gain, const T* w_head, float* logits,
                 int ld_logits, int B, int d, int A, float eps, hipStream_t st) {
  int rows = 32;                                            // at least about two workgroups per compute unit
  while (rows > 4 && (long long)B * ((A + rows - 1) / rows) < 512) rows >>= 1;
  if (d >= 2048) launch_head<T, true>(x, row_index, gain, w_head, logits, ld_logits, B, d, A, rows, eps, st);
  else launch_head<T, false>(x, row_index, gain, w_head, logits, ld_logits, B, d, A, rows, eps, st);
}
template void head_logits<float>(const float*, const int32_t*, const float*, const float*, float*, int, int, int,
                                 int, float, hipStream_t);
template void head_logits<bf16>(const float*, const int32_t*, const float*, const bf16*, float*, int, int, int,
                                int, float, hipStream_t);

// The rows that head_kernel multiplies, for a learner's losses: the same norm, rounded to the storage type.  A row a workgroup;
// bound by its launch (some hundred rows of 16 KB).
template <class T>
__global__ __launch_bounds__(256) void action_hidden_kernel(const float* __restrict__ x, const int32_t* __restrict__ row_index,
                                                            const float* __restrict__ gain, T* __restrict__ out, int d, float eps) {
  __shared__ float red[4];
  const float* row = x + (size_t)row_index[blockIdx.x] * d;
  float ss = 0.f;
  for (int i = threadIdx.x * 4; i < d; i += 1024) {
    const float4 v = *(const float4*)(row + i);
    ss += v.x * v.x + v.y * v.y + v.z * v.z + v.w * v.w;
  }
  ss = block_sum_256(ss, red);
  const float inv = 1.0f / sqrtf(ss / (float)d + eps);
  T* o = out + (size_t)blockIdx.x * d;
  for (int i = threadIdx.x * 4; i < d; i += 1024) {
    const float4 v = *(const float4*)(row + i);
    const float4 g = *(const float4*)(gain + i);
    o[i] = from_f32<T>(v.x * inv * g.x);
    o[i + 1] = from_f32<T>(v.y * inv * g.y);
    o[i + 2] = from_f32<T>(v.z * inv * g.z);
    o[i + 3] = from_f32<T>(v.w * inv * g.w);
  }
}
template <class T>
void action_hidden(const float* x, const int32_t* row_index, const float* gain, T* out, int rows, int d, float eps, hipStream_t st) {
  hipLaunchKernelGGL((action_hidden_kernel<T>), dim3(rows), dim3(256), 0, st, x, row_index, gain, out, d, eps);
}
template void action_hidden<float>(const float*, const int32_t*, const float*, float*, int, int, float, hipStream_t);
template void action_hidden<bf16>(const float*, const int32_t*, const float*, bf16*, int, int, float, hipStream_t);

// ---- value head ---------------------------------------------------------------------------------------
// Action-aware attention pooling over the K hidden rows that feed the action head, done online: after
// each head evaluation the row's score e = w_attn . h + b_attn updates a running softmax-weighted sum
// (m, l, z) per sequence, so no hidden state is stored.  h is the final-RMSNorm output in float32.
__global__ __launch_bounds__(256) void value_accumulate_kernel(const float* __restrict__ x,
                                                               const int32_t* __restrict__ row_index,
                                                               const float* __restrict__ gain, float eps,
                                                               const float* __restrict__ attn_w,
                                                               const float* __restrict__ attn_b, int d, int first,
                                                               float* __restrict__ vz, float* __restrict__ vml) {
  __shared__ float red[4];
  const int b = blockIdx.x;
  const float* row = x + (size_t)(row_index ? row_index[b] : b) * d;
  float ss = 0.f;
  for (int i = threadIdx.x; i < d; i += 256) ss += row[i] * row[i];
  ss = block_sum_256(ss, red);
  const float inv = 1.0f / sqrtf(ss / (float)d + eps);
  float e = 0.f;
  for (int i = threadIdx.x; i < d; i += 256) e += row[i] * inv * gain[i] * attn_w[i];
  e = block_sum_256(e, red) + attn_b[0];
  const float m_old = first ? -INFINITY : vml[2 * b], l_old = first ? 0.f : vml[2 * b + 1];
  const float m_new = fmaxf(m_old, e);
  const float scale = first ? 0.f : expf(m_old - m_new), p = expf(e - m_new);
  float* z = vz + (size_t)b * d;
  for (int i = threadIdx.x; i < d; i += 256) {
    const float h = row[i] * inv * gain[i];
    z[i] = (first ? 0.f : z[i] * scale) + p * h;
  }
  __syncthreads();                       // every thread has read the old statistics
  if (threadIdx.x == 0) {
    vml[2 * b] = m_new;
    vml[2 * b + 1] = l_old * scale + p;
  }
}
void value_accumulate(const float* x, const int32_t* row_index, const float* gain, float eps, const float* attn_w,
                      const float* attn_b, int B, int d, bool first, float* vz, float* vml, hipStream_t st) {
  hipLaunchKernelGGL(value_accumulate_kernel, dim3(B), dim3(256), 0, st, x, row_index, gain, eps, attn_w, attn_b, d,
                     first ? 1 : 0, vz, vml);
}

// u[b] = z[b] / l[b] + step_emb[step_t[b]]   (step clamped to the table)
template <class T>
__global__ __launch_bounds__(256) void value_pool_kernel(const float* __restrict__ vz, const float* __restrict__ vml,
                                                         const T* __restrict__ step_emb, int n_steps,
                                                         const int32_t* __restrict__ step_t, int d,
                                                         float* __restrict__ vu) {
  const int b = blockIdx.x;
  int t = step_t[b];
  t = t < 0 ? 0 : (t >= n_steps ? n_steps - 1 : t);
  const float inv_l = 1.0f / vml[2 * b + 1];
  for (int i = threadIdx.x; i < d; i += 256)
    vu[(size_t)b * d + i] = vz[(size_t)b * d + i] * inv_l + to_f32(step_emb[(size_t)t * d + i]);
}

// vh[b][j] = w2[j] * gelu(W1[j,:] . u[b] + b1[j]).  A workgroup keeps RB rows of u in LDS; each wave then walks
// jpw rows of W1, reading every weight once from memory for all RB rows.
template <class T, int RB>
__global__ __launch_bounds__(256) void value_mlp_kernel(const T* __restrict__ w1, const float* __restrict__ b1,
                                                        const float* __restrict__ w2, const float* __restrict__ vu,
                                                        int B, int d, int jpw, float* __restrict__ vh) {
  extern __shared__ float us[];                             // [RB][d]
  const int b0 = blockIdx.x * RB, nb = min(RB, B - b0);
  for (int i = threadIdx.x * 4; i < RB * d; i += 1024) {
    const int r = i / d, c = i - r * d;                     // d is a multiple of 4: a float4 stays inside a row
    *(f32x4*)(us + i) = r < nb ? *(const f32x4*)(vu + (size_t)(b0 + r) * d + c) : f32x4{0.f, 0.f, 0.f, 0.f};
  }
  __syncthreads();
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int jj = 0; jj < jpw; ++jj) {
    const int j = (blockIdx.y * 4 + wave) * jpw + jj;
    if (j >= d) break;                                      // uniform per wave
    const T* wr = w1 + (size_t)j * d;
    float acc[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) acc[r] = 0.f;
    for (int c = lane * 4; c < d; c += 256) {
      const f32x4 w = load4_f32(wr + c);
#pragma unroll
      for (int r = 0; r < RB; ++r) {
        const f32x4 u = *(const f32x4*)(us + r * d + c);
        acc[r] += w[0] * u[0] + w[1] * u[1] + w[2] * u[2] + w[3] * u[3];
      }
    }
#pragma unroll
    for (int r = 0; r < RB; ++r) acc[r] = wave_sum(acc[r]);
    if (lane == 0) {
      const float bj = b1[j], wj = w2[j];
#pragma unroll
      for (int r = 0; r < RB; ++r)
        if (r < nb) {
          const float t = acc[r] + bj;
          vh[(size_t)(b0 + r) * d + j] = wj * 0.5f * t * (1.0f + erff(t * 0.70710678118654752f));
        }
    }
  }
}
template <class T, int RB>
static void launch_value_mlp(const T* w1, const float* b1, const float* w2, const float* vu, int B, int d, float* vh,
                             hipStream_t st) {
  const size_t smem = (size_t)RB * d * sizeof(float);
  auto kern = value_mlp_kernel<T, RB>;
  static bool attr_set = false;
  if (!attr_set) {
    (void)hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
    attr_set = true;
  }
  // 16 rows a wave re-fill the LDS least; 4 where that would not be a workgroup per compute unit.  us with 4 / 16:
  //   d 4096: 8 pooled rows 39 / 132, 16 99 / 158, 24 144 / 160, 32 192 / 159, 40 234 / 314, 64 383 / 314, 256 1393 / 1233
  //   d 768 (12 workgroups for 8 pooled rows): 8 rows 12 / 37, 128 31 / 57, 256 53 / 75
  const int groups = (B + RB - 1) / RB, jpw = groups * ((d + 63) / 64) >= 256 ? 16 : 4;
  hipLaunchKernelGGL(kern, dim3(groups, (d + 4 * jpw - 1) / (4 * jpw)), dim3(256), smem, st, w1, b1, w2, vu, B, d, jpw, vh);
}

__global__ __launch_bounds__(256) void value_sum_kernel(const float* __restrict__ vh, const float* __restrict__ b2,
                                                        int d, float* __restrict__ values) {
  __shared__ float red[4];
  const int b = blockIdx.x;
  float s = 0.f;
  for (int i = threadIdx.x; i < d; i += 256) s += vh[(size_t)b * d + i];
  s = block_sum_256(s, red);
  if (threadIdx.x == 0) values[b] = s + b2[0];
}

template <class T>
void value_finish(const float* vz, const float* vml, const T* step_emb, int n_steps, const int32_t* step_t,
                  const T* w1, const float* b1, const float* w2, const float* b2, int B, int d, float* vu, float* vh,
                  float* values, hipStream_t st) {
  hipLaunchKernelGGL(value_pool_kernel<T>, dim3(B), dim3(256), 0, st, vz, vml, step_emb, n_steps, step_t, d, vu);
  if (d <= 5120) launch_value_mlp<T, 8>(w1, b1, w2, vu, B, d, vh, st);            // RB * d floats of LDS <= 160 KiB
  else if (d <= 10240) launch_value_mlp<T, 4>(w1, b1, w2, vu, B, d, vh, st);
  else launch_value_mlp<T, 2>(w1, b1, w2, vu, B, d, vh, st);
  hipLaunchKernelGGL(value_sum_kernel, dim3(B), dim3(256), 0, st, vh, b2, d, values);
}
template void value_finish<float>(const float*, const float*, const float*, int, const int32_t*, const float*,
                                  const float*, const float*, const float*, int, int, float*, float*, float*,
                                  hipStream_t);
template void value_finish<bf16>(const float*, const float*, const bf16*, int, const int32_t*, const bf16*,
                                 const float*, const float*, const float*, int, int, float*, float*, float*,
                                 hipStream_t);

// ---- practical ceilings, measured on request ------------------------------------------------------------
// MFMA-only loop with the instruction and the wave tile of the prefill GEMM (64 x 128 on 16x16x32): every wave loads four
// A and eight B fragments once (real weight bits, so the operands toggle like real data) and issues 32 independent MFMAs
// per iteration on them; nothing else runs.  Bound by power: 32x32x16 instructions sustain less (twice the accumulator
// traffic per product).
__global__ __launch_bounds__(256, 2) void probe_mfma_kernel(const f16* __restrict__ w, size_t n_frag, int iters,
                                                            float* __restrict__ sink) {
  constexpr int MT = 4, NT = 8;
  const int lane = threadIdx.x & 63;
  const size_t wave = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  f16x8 a[MT], b[NT];
#pragma unroll
  for (int i = 0; i < MT; ++i) a[i] = *(const f16x8*)(w + ((wave * (MT + NT) + i) % n_frag) * 512 + lane * 8);
#pragma unroll
  for (int j = 0; j < NT; ++j) b[j] = *(const f16x8*)(w + ((wave * (MT + NT) + MT + j) % n_frag) * 512 + lane * 8);
  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int it = 0; it < iters; ++it)
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[i], b[j], acc[i][j], 0, 0, 0);
  float t = 0.f;
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) t += acc[i][j][0];
  if (t == 123.456f) sink[0] = t;      // keeps the loop alive; never true in practice
}
double probe_mfma_flops(int n_wg, int iters) { return (double)n_wg * 4 * iters * 32 * (2.0 * 16 * 16 * 32); }
void probe_mfma(const f16* w, size_t n_frag, int n_wg, int iters, float* sink, hipStream_t st) {
  hipLaunchKernelGGL(probe_mfma_kernel, dim3(n_wg), dim3(256), 0, st, w, n_frag, iters, sink);
}
// Streaming read: 16 bytes per lane, grid-stride, four loads in flight per lane.
__global__ __launch_bounds__(256) void probe_stream_kernel(const u32x4* __restrict__ src, size_t n16,
                                                           unsigned* __restrict__ sink) {
  const size_t stride = (size_t)gridDim.x * 256;
  unsigned x = 0;
  size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  for (; i + 3 * stride < n16; i += 4 * stride) {
    const u32x4 a = src[i], b = src[i + stride], c = src[i + 2 * stride], d = src[i + 3 * stride];
    x ^= a[0] ^ b[1] ^ c[2] ^ d[3];
  }
  for (; i < n16; i += stride) x ^= src[i][0];
  if (x == 0x9e3779b9u) sink[0] = x;   // practically never
}
void probe_stream(const void* src, size_t bytes, int n_wg, unsigned* sink, hipStream_t st) {
  hipLaunchKernelGGL(probe_stream_kernel, dim3(n_wg), dim3(256), 0, st, (const u32x4*)src, bytes / 16, sink);
}

// ---- selection ----------------------------------------------------------------------------------------
// One wave per sequence: scores = logits / tau (+ Gumbel noise); token = lowest index among the
// maxima; log-prob = log_softmax(logits / tau)[token]; action = bin centre (optionally affine).
// Non-finite input: NaN scores never win the comparison, so the token is the best of the others; a row
// with no score above -inf (all NaN or all -inf) selects bin 0.  The log-prob of such rows is NaN.
__global__ __launch_bounds__(64) void select_kernel(const float* __restrict__ logits, int ld_logits, int A, float temperature,
                                                    const float* __restrict__ gumbel, int k, int n_tokens,
                                                    const float* __restrict__ act_scale,
                                                    const float* __restrict__ act_offset, int action_dim,
                                                    int32_t* tokens_out, float* logp_out, float* actions_out,
                                                    int out_stride, int32_t* next_ids, int id0) {
  const int b = blockIdx.x, lane = threadIdx.x;
  const float* z = logits + (size_t)b * ld_logits;
  const float inv_tau = temperature > 0.f ? 1.0f / temperature : 1.0f;
  const float* g = (gumbel && temperature > 0.f) ? gumbel + ((size_t)b * n_tokens + k) * A : nullptr;
  float best = -INFINITY, zmax = -INFINITY;
  int best_j = 0x7fffffff;
  for (int j = lane; j < A; j += 64) {
    const float y = z[j] * inv_tau;
    const float s = g ? y + g[j] : y;
    if (s > best) { best = s; best_j = j; }      // strict: keeps the lowest index within a lane
    zmax = fmaxf(zmax, y);
  }
  // the lowest index among the lanes at the maximum: indices up to 1023 are exact in float32
  const float top = wave_max(best);
  best_j = -(int)wave_max(best == top && best_j < A ? -(float)best_j : -(float)A);
  if (best_j >= A) best_j = 0;                     // no lane saw a score above -inf
  zmax = wave_max(zmax);
  float se = 0.f;
  for (int j = lane; j < A; j += 64) se += expf(z[j] * inv_tau - zmax);
  se = wave_sum(se);
  if (lane == 0) {
    const float logp = z[best_j] * inv_tau - zmax - logf(se);
    float a = -1.0f + (2.0f * (float)best_j + 1.0f) / (float)A;
    const int dim = action_dim > 0 ? k % action_dim : 0;
    if (act_scale) a *= act_scale[dim];
    if (act_offset) a += act_offset[dim];
    const size_t o = (size_t)b * out_stride + k;
    tokens_out[o] = best_j;
    logp_out[o] = logp;
    actions_out[o] = a;
    if (next_ids) next_ids[b] = id0 + best_j;
  }
}
void select_tokens(const float* logits, int ld_logits, int B, int A, float temperature, const float* gumbel, int k, int n_tokens,
                   const float* act_scale, const float* act_offset, int action_dim, int32_t* tokens_out,
                   float* logp_out, float* actions_out, int out_stride, int32_t* next_ids, int id0,
                   hipStream_t st) {
  hipLaunchKernelGGL(select_kernel, dim3(B), dim3(64), 0, st, logits, ld_logits, A, temperature, gumbel, k, n_tokens,
                     act_scale, act_offset, action_dim, tokens_out, logp_out, actions_out, out_stride, next_ids,
                     id0);
}

}  // namespace vla
