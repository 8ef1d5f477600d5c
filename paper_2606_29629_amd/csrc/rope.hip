// Rotary positions of either pair layout over part of every head.
//
// Per pair: (a, b) -> m (a cos t - b sin t, b cos t + a sin t), t = pos f_i: 6
// flops on 4 to 8 bytes, so the kernel is a copy with the rotation under it, and a
// (cos, sin) pair serves every head of its token.  A workgroup takes a few tokens
// and forms their table in LDS first: the frequencies come from the host in turns
// per position (f / 2 pi), so u = pos f - rint(pos f) in double precision is the
// angle reduced exactly, and sin and cos of 2 pi u need single precision only.
// Then each thread turns items of V pairs: two 16-byte pieces, V values of pairs
// i .. i + V - 1 each (HALF: the same pairs' two halves; INTERLEAVED: adjacent).
// Where a 16-byte piece would straddle (addresses, strides or rotary_dim of other
// multiples), V = 1 moves single values.
#include "common.hpp"
#include "kernels.hpp"

namespace tri {

template <typename T, int V, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rope_kernel(tri_rope_table r, int n_heads, const T* x, int64_t xs, T* y,
                                                   int64_t ys, const int32_t* __restrict__ pos,
                                                   int n_tokens, int per_wg, int copy_tail) {
  extern __shared__ float2 table[];  // [per_wg][rot / 2]
  const int rot = r.rotary_dim, half = rot / 2;
  const int t0 = blockIdx.x * per_wg, nt = min(per_wg, n_tokens - t0);
  for (int i = threadIdx.x; i < nt * half; i += blockDim.x) {
    const int t = i / half;
    const double n = (double)pos[t0 + t] * r.turns[i - t * half];
    float s, c;
    sincospif((float)(2.0 * (n - rint(n))), &s, &c);
    table[i] = make_float2(c * r.magnitude, s * r.magnitude);
  }
  __syncthreads();
  typedef T Vec __attribute__((ext_vector_type(V)));
  // items of a head: `half / V` of pairs, then the unrotated rest in pieces of V
  const int pairs = half / V;
  const int per_head = pairs + (copy_tail ? (r.head_dim - rot) / V : 0);
  const int per_tok = per_head * n_heads;
  for (int i = threadIdx.x; i < nt * per_tok; i += blockDim.x) {
    const int t = i / per_tok, k = i - t * per_tok;
    const int h = k / per_head, j = k - h * per_head;
    const T* xp = x + (int64_t)(t0 + t) * xs + h * r.head_dim;
    T* yp = y + (int64_t)(t0 + t) * ys + h * r.head_dim;
    if (j >= pairs) {
      const int d = rot + (j - pairs) * V;
      *(Vec*)(yp + d) = *(const Vec*)(xp + d);
      continue;
    }
    const int ia = INTERLEAVED ? 2 * V * j : V * j;
    const int ib = INTERLEAVED ? ia + V : half + V * j;
    const Vec a = *(const Vec*)(xp + ia), b = *(const Vec*)(xp + ib);
    const float2* cs = table + t * half + V * j;
    Vec oa, ob;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      // pair e of the item: (a[e], b[e]), or values 2 e, 2 e + 1 of a | b
      const float2 w = cs[e];
      if constexpr (INTERLEAVED && V > 1) {
        const int p = 2 * e;
        const float u = p < V ? (float)a[p % V] : (float)b[p % V];
        const float v = p < V ? (float)a[(p + 1) % V] : (float)b[(p + 1) % V];
        const T o0 = (T)(u * w.x - v * w.y), o1 = (T)(v * w.x + u * w.y);
        if (p < V) {
          oa[p % V] = o0;
          oa[(p + 1) % V] = o1;
        } else {
          ob[p % V] = o0;
          ob[(p + 1) % V] = o1;
        }
      } else {
        const float u = (float)a[e], v = (float)b[e];
        oa[e] = (T)(u * w.x - v * w.y);
        ob[e] = (T)(v * w.x + u * w.y);
      }
    }
    *(Vec*)(yp + ia) = oa;
    *(Vec*)(yp + ib) = ob;
  }
}

template <typename T>
static hipError_t run_rope(const tri_rope_table& r, int n_heads, const void* x, int64_t xs, void* y,
                           int64_t ys, const int32_t* pos, int n_tokens, hipStream_t s) {
  constexpr int V = 16 / sizeof(T);
  const int rot = r.rotary_dim;
  const bool interleaved = r.layout == TRI_ROPE_INTERLEAVED;
  const bool wide = rot % (2 * V) == 0 && r.head_dim % V == 0 && xs % V == 0 && ys % V == 0 &&
                    ((uintptr_t)x | (uintptr_t)y) % 16 == 0;
  const int copy_tail = x != y && rot < r.head_dim;
  const int items = n_heads * (rot / 2 + (copy_tail ? r.head_dim - rot : 0)) / (wide ? V : 1);
  const int per_wg = std::max(1, std::min(8, 512 / std::max(1, items)));
  const size_t smem = (size_t)per_wg * (rot / 2) * sizeof(float2);
  auto go = [&](auto kernel) {
    kernel<<<cdiv(n_tokens, per_wg), 256, smem, s>>>(r, n_heads, (const T*)x, xs, (T*)y, ys, pos, n_tokens,
                                                     per_wg, copy_tail);
    return hipGetLastError();
  };
  if (wide) return interleaved ? go(rope_kernel<T, V, true>) : go(rope_kernel<T, V, false>);
  return interleaved ? go(rope_kernel<T, 1, true>) : go(rope_kernel<T, 1, false>);
}

hipError_t launch_rope(const tri_rope_table& r, int n_heads, const void* x, int64_t xs, void* y,
                       int64_t ys, const int32_t* pos, int n_tokens, bool f32, hipStream_t s) {
  return f32 ? run_rope<float>(r, n_heads, x, xs, y, ys, pos, n_tokens, s)
             : run_rope<bf16>(r, n_heads, x, xs, y, ys, pos, n_tokens, s);
}

}  // namespace tri
