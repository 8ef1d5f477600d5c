// Causal grouped-query attention over the 8-bit cache.
//
// out = sum_j p_j v_j, p = softmax(q k_j / sqrt D) over rows j <= ctx + i; with mass,
// mass[j] += p_j summed over the KV head's query heads and the new tokens.
//
// One workgroup per (query head, token): 256 rows a step, a row per thread for the
// scores, then D threads over the values, with the running maximum and sum of the
// softmax in float32.  The log-sum-exp of every (token, head) goes to the workspace,
// from which a second kernel forms the weights again, row by row, and sums them.
#include "attn_kv8.hpp"

namespace tri {

constexpr float kLog2e = 1.4426950408889634f;

// q . (codes of row `at`), D values, q in LDS
template <int D, bool FP8>
__device__ __forceinline__ float dot_row(const uint8_t* codes, const float* q) {
  float s = 0.f;
#pragma unroll
  for (int d = 0; d < D; d += 16) {
    const u32x4 c = ldg16(codes + d);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x4 v = kv8_decode4<FP8>(c[j]);
#pragma unroll
      for (int e = 0; e < 4; ++e) s = fmaf(v[e], q[d + 4 * j + e], s);
    }
  }
  return s;
}

template <int D, bool FP8>
__global__ __launch_bounds__(256) void attn_kv8_kernel(BatchDev b, Kv8Dev c, int Hq, int Hkv,
                                                       const bf16* __restrict__ q, int64_t qs,
                                                       bf16* __restrict__ out,
                                                       float* __restrict__ lse, float scale_log2e) {
  __shared__ float qv[D], p[256], vscale[256], red[4];
  __shared__ int64_t vrow[256];
  const int t = blockIdx.x, hq = blockIdx.y, tid = threadIdx.x;
  int s = 0;
  while (s < b.n_seqs - 1 && b.cu_q[s + 1] <= t) ++s;
  int q0, n, ctx, sl;
  if (!kv8_seq(b, c, s, q0, n, ctx, sl) || t < q0 || t >= q0 + n || n == 1) return;
  const int h = hq / (Hq / Hkv), rows = ctx + (t - q0) + 1;
  if (tid < D) qv[tid] = bf2f(q[(int64_t)t * qs + (int64_t)hq * D + tid]);
  float m = -INFINITY, l = 0.f, acc = 0.f;
  for (int r0 = 0; r0 < rows; r0 += 256) {
    __syncthreads();
    const int r = r0 + tid;
    float sc = -INFINITY;
    vrow[tid] = -1;
    if (r < rows) {
      int prow;
      const int panel = kv_panel(c.kv, sl, r, prow);
      sc = 0.f;
      if (panel >= 0) {
        const int64_t at = kv8_row_at(c, Hkv, panel, h, prow), sa = kv8_scale_at(c, Hkv, panel, h, prow);
        sc = dot_row<D, FP8>(c.k + at * D, qv) * c.k_scale[sa] * scale_log2e;
        vrow[tid] = at;
        vscale[tid] = c.v_scale[sa];
      }
    }
    float mt = wave_max(sc);
    if ((tid & 63) == 0) red[tid >> 6] = mt;
    __syncthreads();
    const float mn = fmaxf(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])), m);
    const float a = exp2f(m - mn), w = exp2f(sc - mn);
    p[tid] = w;
    const float lt = wave_sum(w);
    __syncthreads();
    if ((tid & 63) == 0) red[tid >> 6] = lt;
    __syncthreads();
    l = l * a + (red[0] + red[1] + red[2] + red[3]);
    m = mn;
    if (tid < D) {
      acc *= a;
      for (int j = 0; j < min(256, rows - r0); ++j) {
        if (vrow[j] < 0) continue;
        const uint32_t word = c.v[vrow[j] * D + tid];
        acc = fmaf(p[j] * vscale[j], kv8_decode4<FP8>(word)[0], acc);
      }
    }
  }
  if (tid < D) out[((int64_t)t * Hq + hq) * D + tid] = f2bf(acc / l);
  if (lse && tid == 0) lse[(int64_t)t * Hq + hq] = m + log2f(l);
}

template <int D, bool FP8>
__global__ __launch_bounds__(256) void mass_kv8_kernel(BatchDev b, Kv8Dev c, int Hq, int Hkv,
                                                       const bf16* __restrict__ q, int64_t qs,
                                                       const float* __restrict__ lse,
                                                       float scale_log2e) {
  __shared__ float qv[D];
  const int s = blockIdx.z, h = blockIdx.y, tid = threadIdx.x;
  int q0, n, ctx, sl;
  if (!kv8_seq(b, c, s, q0, n, ctx, sl) || n <= 1) return;
  const int r = blockIdx.x * 256 + tid, G = Hq / Hkv;
  int prow, panel = -1;
  if (r < ctx + n) panel = kv_panel(c.kv, sl, r, prow);
  int64_t at = 0;
  float ks = 0.f, sum = 0.f;
  if (panel >= 0) {
    at = kv8_row_at(c, Hkv, panel, h, prow);
    ks = c.k_scale[kv8_scale_at(c, Hkv, panel, h, prow)] * scale_log2e;
  }
  for (int i = 0; i < n; ++i)
    for (int g = 0; g < G; ++g) {
      const int hq = h * G + g;
      __syncthreads();
      if (tid < D) qv[tid] = bf2f(q[(int64_t)(q0 + i) * qs + (int64_t)hq * D + tid]);
      __syncthreads();
      if (panel >= 0 && r <= ctx + i)
        sum += exp2f(dot_row<D, FP8>(c.k + at * D, qv) * ks - lse[(int64_t)(q0 + i) * Hq + hq]);
    }
  if (panel >= 0) c.mass[at] += sum;
}

size_t attn_kv8_workspace_bytes(const BatchDev& b, const Kv8Dev& c, int n_q_heads, int n_kv_heads,
                                int head_dim) {
  const size_t lse = c.mass ? (size_t)b.n_tokens * n_q_heads * sizeof(float) : 0;
  return (lse + 255) / 256 * 256 + attn_kv8_decode_bytes(b, c, n_q_heads, n_kv_heads, head_dim);
}

hipError_t launch_attn_kv8(const BatchDev& b, const Kv8Dev& c, bool fp8, int n_q_heads,
                           int n_kv_heads, int head_dim, const void* q, int64_t q_stride, void* out,
                           void* ws, hipStream_t s) {
  if (b.n_seqs == 0 || b.n_tokens == 0) return hipSuccess;
  const float scale_log2e = (float)(1.4426950408889634 / __builtin_sqrt((double)head_dim));
  float* lse = c.mass ? (float*)ws : nullptr;
  const size_t lse_bytes = c.mass ? (size_t)b.n_tokens * n_q_heads * sizeof(float) : 0;
  if (b.max_q_len == 1 || (int64_t)b.n_seqs * b.max_q_len != b.n_tokens) {
    const hipError_t e = launch_attn_kv8_decode(b, c, fp8, n_q_heads, n_kv_heads, head_dim, q, q_stride, out,
                                                (float*)((char*)ws + (lse_bytes + 255) / 256 * 256), s);
    if (e != hipSuccess || b.max_q_len == 1) return e;
  }
  auto go = [&](auto attend, auto weigh) {
    attend<<<dim3(b.n_tokens, n_q_heads), 256, 0, s>>>(b, c, n_q_heads, n_kv_heads, (const bf16*)q,
                                                       q_stride, (bf16*)out, lse, scale_log2e);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !lse) return e;
    const dim3 grid(cdiv(b.max_ctx_len + b.max_q_len, 256), n_kv_heads, b.n_seqs);
    weigh<<<grid, 256, 0, s>>>(b, c, n_q_heads, n_kv_heads, (const bf16*)q, q_stride, lse, scale_log2e);
    return hipGetLastError();
  };
  if (head_dim == 128)
    return fp8 ? go(attn_kv8_kernel<128, true>, mass_kv8_kernel<128, true>)
               : go(attn_kv8_kernel<128, false>, mass_kv8_kernel<128, false>);
  return fp8 ? go(attn_kv8_kernel<64, true>, mass_kv8_kernel<64, true>)
             : go(attn_kv8_kernel<64, false>, mass_kv8_kernel<64, false>);
}

}  // namespace tri
