// The 8-bit KV cache's append, and its eviction: which rows stay, and moving them.
#include "kv8.hpp"

namespace tri {

// Largest of the workgroup's values (every thread gets it).  `lds` holds one per wave.
template <int W>
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t* lds) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
  if constexpr (W == 1) return v;
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < W; ++w) v = max(v, lds[w]);
  return v;
}

// Append.  One workgroup per (scale block touched, head, sequence), keys and values:
// the largest magnitude of the block's new rows decides its scale, so a block is read
// (16 bf16 per thread and step), reduced and read again from cache to be written as
// codes.  Bytes bound it: two read and one written per value; the held rows of a
// block begun before are touched only where its scale grows.
template <int D, bool FP8, int W>
__global__ __launch_bounds__(64 * W) void kv8_append_kernel(BatchDev b, Kv8Dev c, int Hkv,
                                                            const bf16* __restrict__ kn,
                                                            const bf16* __restrict__ vn,
                                                            int64_t stride) {
  __shared__ uint32_t red[2][W];
  constexpr int CPR = D / 16;  // 16-value pieces of a row
  const int s = blockIdx.z, h = blockIdx.y, tid = threadIdx.x;
  int q0, n, ctx, sl;
  if (!kv8_seq(b, c, s, q0, n, ctx, sl)) return;
  const int R = 1 << c.scale_shift;
  const int blk0 = ((ctx >> c.scale_shift) + (int)blockIdx.x) << c.scale_shift;  // its first row
  const int lo = max(blk0, ctx), hi = min(blk0 + R, ctx + n);
  if (lo >= hi) return;
  int prow;
  const int panel = kv_panel(c.kv, sl, blk0, prow);
  if (panel < 0) return;
  const int64_t at = kv8_scale_at(c, Hkv, panel, h, prow);
  const int64_t row0 = kv8_row_at(c, Hkv, panel, h, prow);  // of blk0
  const int held = lo - blk0;
  const int items = (hi - lo) * CPR;
  const int64_t src0 = (int64_t)(q0 + lo - ctx) * stride + (int64_t)h * D;
  const bf16* in[2] = {kn + src0, vn + src0};
  uint8_t* codes[2] = {c.k + row0 * D, c.v + row0 * D};
  float* scale[2] = {c.k_scale + at, c.v_scale + at};
  float before[2];
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) before[kv] = held ? *scale[kv] : 0.f;
  float now[2];
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    uint32_t m = 0;
    for (int i = tid; i < items; i += 64 * W) {
      const int r = i / CPR, d = (i % CPR) * 16;
      const bf16* p = in[kv] + r * stride + d;
      const u32x4 a = ldg16(p), e = ldg16(p + 8);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        m = max(max(m, (a[j] << 16) & 0x7fffffffu), a[j] & 0x7fff0000u);
        m = max(max(m, (e[j] << 16) & 0x7fffffffu), e[j] & 0x7fff0000u);
      }
    }
    now[kv] = kv8_scale_of<FP8>(block_max<W>(m, red[kv]));
    if (held) now[kv] = kv8_scale_max(now[kv], before[kv]);
  }
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    const float inv = kv8_inverse(now[kv]);
    for (int i = tid; i < items; i += 64 * W) {
      const int r = i / CPR, d = (i % CPR) * 16;
      const bf16* p = in[kv] + r * stride + d;
      Pack8 x[2];
      x[0].u = ldg16(p);
      x[1].u = ldg16(p + 8);
      u32x4 o;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = inv > 0.f ? bf2f(x[j >> 1].e[4 * (j & 1) + e]) * inv : 0.f;
        o[j] = kv8_encode4<FP8>(v);
      }
      stg16(codes[kv] + (int64_t)(held + r) * D + d, o);
    }
    if (held && now[kv] != before[kv]) {  // grown (or NaN: all codes to 0)
      const float f = before[kv] == before[kv] ? before[kv] * inv : 0.f;
      for (int i = tid; i < held * CPR; i += 64 * W) {
        uint8_t* p = codes[kv] + (int64_t)i * 16;
        stg16(p, kv8_rescale16<FP8>(ldg16(p), f));
      }
    }
    if (tid == 0) *scale[kv] = now[kv];  // (every thread has read it: the reductions' barriers)
  }
  for (int r = tid; r < hi - lo; r += 64 * W) {
    if (c.mass) c.mass[row0 + held + r] = 0.f;
    if (c.stamp) c.stamp[row0 + held + r] = b.pos[q0 + lo - ctx + r];
  }
}

hipError_t launch_kv8_append(const BatchDev& b, const Kv8Dev& c, bool fp8, int n_kv_heads,
                             int head_dim, const void* k_new, const void* v_new, int64_t stride,
                             hipStream_t s) {
  if (b.n_seqs == 0 || b.max_q_len == 0) return hipSuccess;
  // blocks that max_q_len rows can touch, wherever they begin
  const int R = 1 << c.scale_shift;
  const dim3 grid((b.max_q_len + R - 2) / R + 1, n_kv_heads, b.n_seqs);
  const bool one = b.max_q_len * head_dim <= 2048;  // a wave has two pieces a thread at most
  auto go = [&](auto wide, auto narrow) {
    if (one) narrow<<<grid, 64, 0, s>>>(b, c, n_kv_heads, (const bf16*)k_new, (const bf16*)v_new, stride);
    else wide<<<grid, 256, 0, s>>>(b, c, n_kv_heads, (const bf16*)k_new, (const bf16*)v_new, stride);
    return hipGetLastError();
  };
  if (head_dim == 128)
    return fp8 ? go(kv8_append_kernel<128, true, 4>, kv8_append_kernel<128, true, 1>)
               : go(kv8_append_kernel<128, false, 4>, kv8_append_kernel<128, false, 1>);
  return fp8 ? go(kv8_append_kernel<64, true, 4>, kv8_append_kernel<64, true, 1>)
             : go(kv8_append_kernel<64, false, 4>, kv8_append_kernel<64, false, 1>);
}

// Select.  One workgroup per (head, sequence).  A row's key is its mass as an unsigned
// integer of the same order (protected rows above all, NaN below all); the budget-th
// largest key is found by three histograms of 11, 11 and 10 bits in LDS (integer
// counts: no order changes them), and one pass in row order then knows of every row,
// from the counts of greater and equal keys before it, whether it stays and, of rows
// evicted below budget and kept past it, the how-manieth it is.  The latter's rows are
// paired through a list in LDS, kSelList at a time.
constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;
constexpr int kSelBins = 2048, kSelList = 8192;

__global__ __launch_bounds__(kSelThreads) void kv8_select_kernel(BatchDev b, Kv8Dev c, int Hkv,
                                                                 int budget, int n_first,
                                                                 int n_recent,
                                                                 int32_t* __restrict__ plan,
                                                                 int32_t* __restrict__ new_len) {
  __shared__ uint32_t hist[kSelBins];
  __shared__ int list[kSelList];
  __shared__ uint32_t red[kSelWaves];
  __shared__ int wave_gt[kSelWaves], wave_eq[kSelWaves];
  __shared__ uint32_t found[2];
  const int s = blockIdx.y, h = blockIdx.x, tid = threadIdx.x;
  const int lane = tid & 63, wave = tid >> 6;
  int q0, nq, ctx, sl;
  const bool ok = kv8_seq(b, c, s, q0, nq, ctx, sl);
  const int n = ok ? ctx + nq : 0;
  int32_t* out = plan + ((int64_t)s * Hkv + h) * budget;
  if (h == 0 && tid == 0 && new_len) new_len[s] = min(n, budget);
  if (n <= budget) {
    for (int r = tid; r < budget; r += kSelThreads) out[r] = r < n ? r : -1;
    return;
  }
  auto place = [&](int r) {  // index of the row's mass and stamp; -1: no page
    int prow;
    const int panel = kv_panel(c.kv, sl, r, prow);
    return panel < 0 ? (int64_t)-1 : kv8_row_at(c, Hkv, panel, h, prow);
  };
  auto age = [&](int r, int64_t at) { return c.stamp && at >= 0 ? c.stamp[at] : r; };
  uint32_t newest = 0;  // (stamps as unsigned integers of the same order)
  for (int r = tid; r < n; r += kSelThreads)
    newest = max(newest, (uint32_t)age(r, place(r)) ^ 0x80000000u);
  newest = block_max<kSelWaves>(newest, red);
  const int64_t last_old = (int64_t)(int)(newest ^ 0x80000000u) - n_recent;  // stamps past it are recent
  auto key = [&](int r) -> uint32_t {
    const int64_t at = place(r);
    const int a = age(r, at);
    if (a < n_first || a > last_old) return 0xffffffffu;
    const float m = at >= 0 ? c.mass[at] + 0.f : 0.f;  // (-0 becomes 0)
    if (m != m) return 0u;
    const uint32_t u = __float_as_uint(m);
    return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
  };
  // The budget-th largest key T, and how many rows equal to T stay.
  uint32_t T = 0, mask = 0;
  int need = budget;
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0), bins = pass == 2 ? 1024 : 2048;
    for (int i = tid; i < bins; i += kSelThreads) hist[i] = 0;
    __syncthreads();
    for (int r = tid; r < n; r += kSelThreads) {
      const uint32_t k = key(r);
      if ((k & mask) == T) atomicAdd(&hist[(k >> shift) & (bins - 1)], 1u);
    }
    __syncthreads();
    // Rows in greater bins, by thread: bins per thread (descending), a scan over waves.
    const int per = bins / kSelThreads;
    uint32_t mine = 0;
    for (int i = 0; i < per; ++i) mine += hist[bins - 1 - (tid * per + i)];
    uint32_t upto = mine;
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t v = (uint32_t)__shfl_up((int)upto, o, 64);
      if (lane >= o) upto += v;
    }
    if (lane == 63) red[wave] = upto;
    __syncthreads();
    uint32_t above = upto - mine;
    for (int w = 0; w < wave; ++w) above += red[w];
    for (int i = 0; i < per; ++i) {
      const int bin = bins - 1 - (tid * per + i);
      const uint32_t cnt = hist[bin];
      if (above < (uint32_t)need && above + cnt >= (uint32_t)need) {
        found[0] = (uint32_t)bin;
        found[1] = above;
      }
      above += cnt;
    }
    __syncthreads();
    T |= found[0] << shift;
    mask |= (uint32_t)(bins - 1) << shift;
    need -= (int)found[1];
    __syncthreads();
  }
  // In row order: keys greater than and equal to T before each row.
  int gt0 = 0, eq0 = 0;  // before the tile
  auto scan = [&](bool gt, bool eq, int& ngt, int& neq) {
    const uint64_t bg = __builtin_amdgcn_ballot_w64(gt), be = __builtin_amdgcn_ballot_w64(eq);
    const uint64_t below = (1ull << lane) - 1;
    if (lane == 0) {
      wave_gt[wave] = __builtin_popcountll(bg);
      wave_eq[wave] = __builtin_popcountll(be);
    }
    __syncthreads();
    ngt = gt0 + __builtin_popcountll(bg & below);
    neq = eq0 + __builtin_popcountll(be & below);
    for (int w = 0; w < kSelWaves; ++w) {
      const int g = wave_gt[w], e = wave_eq[w];
      if (w < wave) { ngt += g; neq += e; }
      gt0 += g;
      eq0 += e;
    }
    __syncthreads();
  };
  for (int r0 = 0; r0 < budget; r0 += kSelThreads) {
    const int r = r0 + tid;
    const uint32_t k = r < budget ? key(r) : 0;
    const bool gt = r < budget && k > T, eq = r < budget && k == T;
    int ngt, neq;
    scan(gt, eq, ngt, neq);
    // kept before r: the greater ones and the first `need` equal ones
    if (r < budget) out[r] = gt || (eq && neq < need) ? r : -2 - (r - (ngt + min(neq, need)));
  }
  const int kept_low = gt0 + min(eq0, need), gt_low = gt0, eq_low = eq0;
  for (int base = 0; base < budget - kept_low; base += kSelList) {
    gt0 = gt_low;
    eq0 = eq_low;
    for (int r0 = budget; r0 < n; r0 += kSelThreads) {
      const int r = r0 + tid;
      const uint32_t k = r < n ? key(r) : 0;
      const bool gt = r < n && k > T, eq = r < n && k == T;
      int ngt, neq;
      scan(gt, eq, ngt, neq);
      const int j = ngt + min(neq, need) - kept_low - base;
      if ((gt || (eq && neq < need)) && j >= 0 && j < kSelList) list[j] = r;
    }
    __syncthreads();
    for (int r = tid; r < budget; r += kSelThreads) {  // (a thread reads what it wrote)
      const int v = out[r], j = -2 - v - base;
      if (v <= -2 && j >= 0 && j < kSelList) out[r] = list[j];
    }
    __syncthreads();
  }
}

hipError_t launch_kv8_select(const BatchDev& b, const Kv8Dev& c, int n_kv_heads, int budget,
                             int n_first, int n_recent, int32_t* plan, int32_t* new_len,
                             hipStream_t s) {
  if (b.n_seqs == 0) return hipSuccess;
  kv8_select_kernel<<<dim3(n_kv_heads, b.n_seqs), kSelThreads, 0, s>>>(b, c, n_kv_heads, budget,
                                                                      n_first, n_recent, plan, new_len);
  return hipGetLastError();
}

// Move.  One workgroup per (scale block below budget, head, sequence).  Rows come from
// at or past budget and go below it, so no workgroup reads what another writes.  Most
// blocks of a lightly trimmed cache change nothing and end at their plan entries.
template <int D, bool FP8>
__global__ __launch_bounds__(256) void kv8_move_kernel(BatchDev b, Kv8Dev c, int Hkv,
                                                       const int32_t* __restrict__ plan, int budget) {
  constexpr int CPR = D / 16, kMaxRows = 128;
  __shared__ int64_t src_row[kMaxRows];  // row index of the source, -1: leave the row
  __shared__ float src_scale[2][kMaxRows];
  __shared__ uint32_t red[2][4];
  const int s = blockIdx.z, h = blockIdx.y, tid = threadIdx.x;
  const int sl = b.slot[s];
  if (sl < 0 || sl >= c.kv.n_slots) return;
  const int R = 1 << c.scale_shift, r0 = blockIdx.x << c.scale_shift;
  int prow;
  const int panel = kv_panel(c.kv, sl, r0, prow);
  if (panel < 0) return;
  int src = -1;
  if (tid < R) {
    src = plan[((int64_t)s * Hkv + h) * budget + r0 + tid];
    if (src < 0 || src >= c.kv.max_seq) src = -1;
  }
  if (!__syncthreads_or(src >= 0 && src != r0 + tid)) return;
  const int64_t row0 = kv8_row_at(c, Hkv, panel, h, prow), at = kv8_scale_at(c, Hkv, panel, h, prow);
  uint32_t ks = 0, vs = 0;
  if (tid < R) {
    int64_t from = -1;
    if (src >= 0) {
      int p;
      const int sp = kv_panel(c.kv, sl, src, p);
      if (sp >= 0) {
        from = kv8_row_at(c, Hkv, sp, h, p);
        const int64_t sa = kv8_scale_at(c, Hkv, sp, h, p);
        src_scale[0][tid] = c.k_scale[sa];
        src_scale[1][tid] = c.v_scale[sa];
        ks = __float_as_uint(src_scale[0][tid]) & 0x7fffffffu;
        vs = __float_as_uint(src_scale[1][tid]) & 0x7fffffffu;
      }
    }
    src_row[tid] = from;
  }
  const float now[2] = {__uint_as_float(block_max<4>(ks, red[0])),
                        __uint_as_float(block_max<4>(vs, red[1]))};
  __syncthreads();
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    uint8_t* codes = kv ? c.v : c.k;
    const float inv = kv8_inverse(now[kv]);
    for (int i = tid; i < R * CPR; i += 256) {
      const int r = i / CPR, d = (i % CPR) * 16;
      const int64_t from = src_row[r], to = row0 + r;
      const float sc = src_scale[kv][r];
      if (from < 0 || (from == to && sc == now[kv])) continue;
      stg16(codes + to * D + d,
            kv8_rescale16<FP8>(ldg16(codes + from * D + d), sc == sc ? sc * inv : 0.f));
    }
    if (tid == 0) (kv ? c.v_scale : c.k_scale)[at] = now[kv];
  }
  if (tid < R && src_row[tid] >= 0 && src_row[tid] != row0 + tid) {
    if (c.mass) c.mass[row0 + tid] = c.mass[src_row[tid]];
    if (c.stamp) c.stamp[row0 + tid] = c.stamp[src_row[tid]];
  }
}

hipError_t launch_kv8_move(const BatchDev& b, const Kv8Dev& c, bool fp8, int n_kv_heads,
                           int head_dim, const int32_t* plan, int budget, hipStream_t s) {
  if (b.n_seqs == 0) return hipSuccess;
  const dim3 grid(budget >> c.scale_shift, n_kv_heads, b.n_seqs);
  auto go = [&](auto kernel) {
    kernel<<<grid, 256, 0, s>>>(b, c, n_kv_heads, plan, budget);
    return hipGetLastError();
  };
  if (head_dim == 128) return fp8 ? go(kv8_move_kernel<128, true>) : go(kv8_move_kernel<128, false>);
  return fp8 ? go(kv8_move_kernel<64, true>) : go(kv8_move_kernel<64, false>);
}

}  // namespace tri
