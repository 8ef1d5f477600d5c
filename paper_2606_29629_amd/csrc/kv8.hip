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

// Select.  A row's key is its mass as an unsigned integer of the same order (protected
// rows above all, NaN below all).  The budget-th largest key T of a (sequence, head) is
// found by histograms of its upper 11, next 11 and last 10 bits (integer counts: no order
// changes them); then of every row, from the counts of greater and equal keys before it,
// it is known whether it stays and, of rows evicted below budget and of rows kept past it,
// the how-manieth it is, which pairs them.  The work is a few operations a row, eight bytes
// read: a chain of short dependent steps bounds it, not bytes.
//
// Up to kSelOneRows rows one workgroup of 1024 threads does it all, K neighbouring rows a
// thread with their keys in registers (4352 rows: 64 x 4 heads in %SHORT%).
// Longer sequences take a workgroup per kSelChunk rows and one launch per step.
constexpr int kSelThreads = 1024;
constexpr int kSelOneRows = 16 * kSelThreads;
constexpr int kSelBins = 2048;
constexpr int kSelChunk = 2048;  // rows of a workgroup of 256, eight a thread
constexpr int kSelK = 8;

// The sequence's rows; 0 where it is skipped (also if past the batch's host fields, which
// the buffers are sized by).
__device__ __forceinline__ int select_rows(const BatchDev& b, const Kv8Dev& c, int s, int& sl) {
  int q0, nq, ctx;
  const bool ok = kv8_seq(b, c, s, q0, nq, ctx, sl);
  return ok && ctx <= b.max_ctx_len && nq <= b.max_q_len ? ctx + nq : 0;
}

// Mass and stamp of K neighbouring rows r .. (K divides the page; rows past n: 0).
template <int K>
__device__ __forceinline__ void select_load(const Kv8Dev& c, int Hkv, int h, int sl, int r, int n,
                                            float (&m)[K], int (&a)[K]) {
  int prow = 0;
  const int panel = r < n ? kv_panel(c.kv, sl, r, prow) : -1;
  const int64_t at = kv8_row_at(c, Hkv, max(panel, 0), h, prow);
#pragma unroll
  for (int i = 0; i < K; ++i) {
    const bool there = panel >= 0 && r + i < n;
    m[i] = there ? c.mass[at + i] : 0.f;
    a[i] = there && c.stamp ? c.stamp[at + i] : r + i;
  }
}

// A stamp as an unsigned integer of the same order.
__device__ __forceinline__ uint32_t stamp_key(int a) { return (uint32_t)a ^ 0x80000000u; }

__device__ __forceinline__ uint32_t select_key(float m, int age, uint32_t newest, int n_first,
                                               int n_recent) {
  const int64_t last_old = (int64_t)(int)(newest ^ 0x80000000u) - n_recent;
  if (age < n_first || age > last_old) return 0xffffffffu;
  if (m != m) return 0u;
  const uint32_t u = __float_as_uint(m + 0.f);  // (-0 becomes 0)
  return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}

constexpr int select_shift(int pass) { return pass == 0 ? 21 : (pass == 1 ? 10 : 0); }
constexpr int select_bins(int pass) { return pass == 2 ? 1024 : 2048; }
constexpr int kSelHist = 2048 + 2048 + 1024;  // the three histograms of a head
constexpr int select_hist_at(int pass) { return pass * 2048; }

// The bin in which the counts from the top reach `need`, and the count above it.  W waves;
// `red` holds W words, `found` two; every thread gets the answer.
template <int W>
__device__ __forceinline__ void select_bin(const uint32_t* hist, int bins, int need, uint32_t* red,
                                           uint32_t* found, int& bin, int& above) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = bins / (64 * W);
  uint32_t mine = 0;
  for (int i = 0; i < per; ++i) mine += hist[bins - 1 - (tid * per + i)];
  uint32_t upto = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t v = (uint32_t)__shfl_up((int)upto, o, 64);
    if (lane >= o) upto += v;
  }
  if (lane == 63) red[wave] = upto;
  __syncthreads();
  uint32_t over = upto - mine;
#pragma unroll
  for (int w = 0; w < W; ++w) over += w < wave ? red[w] : 0u;
  for (int i = 0; i < per; ++i) {
    const int at = bins - 1 - (tid * per + i);
    const uint32_t cnt = hist[at];
    if (over < (uint32_t)need && over + cnt >= (uint32_t)need) {
      found[0] = (uint32_t)at;
      found[1] = over;
    }
    over += cnt;
  }
  __syncthreads();
  bin = (int)found[0];
  above = (int)found[1];
}

// Exclusive prefixes of two counts over the workgroup, and their totals.
template <int W>
__device__ __forceinline__ void block_prefix2(int a, int e, int& pa, int& pe, int& ta, int& te,
                                              int (*red)[2]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int ua = a, ue = e;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(ua, o, 64), y = __shfl_up(ue, o, 64);
    if (lane >= o) {
      ua += x;
      ue += y;
    }
  }
  if (lane == 63) {
    red[wave][0] = ua;
    red[wave][1] = ue;
  }
  __syncthreads();
  pa = ua - a;
  pe = ue - e;
  ta = te = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const int x = red[w][0], y = red[w][1];
    if (w < wave) {
      pa += x;
      pe += y;
    }
    ta += x;
    te += y;
  }
}

template <int K>
__global__ __launch_bounds__(kSelThreads) void kv8_select_kernel(BatchDev b, Kv8Dev c, int Hkv,
                                                                 int budget, int n_first,
                                                                 int n_recent,
                                                                 int32_t* __restrict__ plan,
                                                                 int32_t* __restrict__ new_len) {
  constexpr int W = kSelThreads / 64;
  __shared__ uint32_t hist[kSelBins], red[W], found[2];
  __shared__ int sums[W][2], kept_low_at, list[K * kSelThreads / 2];  // (pairs: half of the rows at most)
  const int s = blockIdx.y, h = blockIdx.x, tid = threadIdx.x, r0 = tid * K;
  int sl;
  const int n = select_rows(b, c, s, sl);
  int32_t* out = plan + ((int64_t)s * Hkv + h) * budget;
  if (h == 0 && tid == 0 && new_len) new_len[s] = min(n, budget);
  if (n <= budget) {
    for (int r = tid; r < budget; r += kSelThreads) out[r] = r < n ? r : -1;
    return;
  }
  uint32_t key[K];
  {
    float m[K];
    int a[K];
    select_load<K>(c, Hkv, h, sl, r0, n, m, a);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < K; ++i) top = max(top, r0 + i < n ? stamp_key(a[i]) : 0u);
    top = block_max<W>(top, red);
#pragma unroll
    for (int i = 0; i < K; ++i) key[i] = select_key(m[i], a[i], top, n_first, n_recent);
  }
  uint32_t T = 0;
  int need = budget;
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = select_shift(pass), bins = select_bins(pass);
    const uint32_t mask = pass == 0 ? 0u : ~0u << select_shift(pass - 1);
    for (int i = tid; i < bins; i += kSelThreads) hist[i] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < K; ++i)
      if (r0 + i < n && (key[i] & mask) == T) atomicAdd(&hist[(key[i] >> shift) & (bins - 1)], 1u);
    __syncthreads();
    int bin, above;
    select_bin<W>(hist, bins, need, red, found, bin, above);
    T |= (uint32_t)bin << shift;
    need -= above;
  }
  // Kept before a row: the greater keys and the first `need` equal ones.
  int gt = 0, eq = 0;
#pragma unroll
  for (int i = 0; i < K; ++i) {
    gt += r0 + i < n && key[i] > T;
    eq += r0 + i < n && key[i] == T;
  }
  int ngt, neq, all_gt, all_eq;
  block_prefix2<W>(gt, eq, ngt, neq, all_gt, all_eq, sums);
  int place[K];  // kept rows before each row
  bool keep[K];
#pragma unroll
  for (int i = 0; i < K; ++i) {
    const bool there = r0 + i < n, more = there && key[i] > T, same = there && key[i] == T;
    place[i] = ngt + min(neq, need);
    keep[i] = more || (same && neq < need);
    if (r0 + i == budget) kept_low_at = place[i];
    ngt += more;
    neq += same;
  }
  __syncthreads();
  const int kept_low = kept_low_at;
#pragma unroll
  for (int i = 0; i < K; ++i)
    if (keep[i] && r0 + i >= budget) list[place[i] - kept_low] = r0 + i;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < K; ++i) {
    const int r = r0 + i;
    if (r < budget) out[r] = keep[i] ? r : list[r - place[i]];
  }
}

// The same in steps over chunks (grid: chunk, head, sequence).  Per (sequence, head) in the
// workspace: every row's key, the histograms, and of every chunk its newest stamp and its
// counts of greater and equal keys; the rows that move, in order.
struct SelectWs {
  uint32_t *key, *hist, *newest;
  int32_t *count, *list;
  int chunks, list_rows;
  __device__ uint32_t* keys_of(int64_t p) const { return key + p * chunks * kSelChunk; }
  __device__ uint32_t* hist_of(int64_t p, int pass) const { return hist + p * kSelHist + select_hist_at(pass); }
};

__global__ __launch_bounds__(256) void select_newest_kernel(BatchDev b, Kv8Dev c, int Hkv, int budget,
                                                            SelectWs w) {
  __shared__ uint32_t red[4];
  const int s = blockIdx.z, h = blockIdx.y, r0 = blockIdx.x * kSelChunk + (int)threadIdx.x * kSelK;
  const int64_t pair = (int64_t)s * Hkv + h;
  int sl;
  const int n = select_rows(b, c, s, sl);
  if (n <= budget) return;
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < kSelHist; i += 256) w.hist[pair * kSelHist + i] = 0;
  uint32_t top = 0;
  if (c.stamp) {
    float m[kSelK];
    int a[kSelK];
    select_load<kSelK>(c, Hkv, h, sl, r0, n, m, a);
#pragma unroll
    for (int i = 0; i < kSelK; ++i) top = max(top, r0 + i < n ? stamp_key(a[i]) : 0u);
    top = block_max<4>(top, red);
  } else {
    top = stamp_key(n - 1);
  }
  if (threadIdx.x == 0) w.newest[pair * w.chunks + blockIdx.x] = top;
}

// T's digits and the equal keys still needed after the first `passes` histograms.
template <int PASSES>
__device__ __forceinline__ uint32_t select_digits(const SelectWs& w, int64_t pair, int budget,
                                                  uint32_t* red, uint32_t* found, int& need) {
  uint32_t T = 0;
  need = budget;
#pragma unroll
  for (int pass = 0; pass < PASSES; ++pass) {
    int bin, above;
    __syncthreads();
    select_bin<4>(w.hist_of(pair, pass), select_bins(pass), need, red, found, bin, above);
    T |= (uint32_t)bin << select_shift(pass);
    need -= above;
  }
  return T;
}

template <int PASS>
__global__ __launch_bounds__(256) void select_hist_kernel(BatchDev b, Kv8Dev c, int Hkv, int budget,
                                                          int n_first, int n_recent, SelectWs w) {
  constexpr int BINS = select_bins(PASS), SHIFT = select_shift(PASS);
  __shared__ uint32_t hist[BINS], red[4], found[2];
  const int s = blockIdx.z, h = blockIdx.y, tid = threadIdx.x;
  const int r0 = blockIdx.x * kSelChunk + tid * kSelK;
  const int64_t pair = (int64_t)s * Hkv + h;
  int sl;
  const int n = select_rows(b, c, s, sl);
  if (n <= budget || (int)blockIdx.x * kSelChunk >= n) return;
  for (int i = tid; i < BINS; i += 256) hist[i] = 0;
  uint32_t key[kSelK];
  u32x4* kp = (u32x4*)(w.keys_of(pair) + r0);
  uint32_t T = 0, mask = 0;
  if constexpr (PASS == 0) {
    float m[kSelK];
    int a[kSelK];
    select_load<kSelK>(c, Hkv, h, sl, r0, n, m, a);
    uint32_t top = 0;
    for (int i = tid; i < cdiv(n, kSelChunk); i += 256) top = max(top, w.newest[pair * w.chunks + i]);
    top = block_max<4>(top, red);
#pragma unroll
    for (int i = 0; i < kSelK; ++i) key[i] = select_key(m[i], a[i], top, n_first, n_recent);
    kp[0] = u32x4{key[0], key[1], key[2], key[3]};
    kp[1] = u32x4{key[4], key[5], key[6], key[7]};
  } else {
    const u32x4 x = kp[0], y = kp[1];
#pragma unroll
    for (int i = 0; i < kSelK; ++i) key[i] = i < 4 ? x[i] : y[i - 4];
    int need;
    T = select_digits<PASS>(w, pair, budget, red, found, need);
    mask = ~0u << select_shift(PASS - 1);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSelK; ++i)
    if (r0 + i < n && (key[i] & mask) == T) atomicAdd(&hist[(key[i] >> SHIFT) & (BINS - 1)], 1u);
  __syncthreads();
  uint32_t* all = w.hist_of(pair, PASS);
  for (int i = tid; i < BINS; i += 256)
    if (hist[i]) atomicAdd(&all[i], hist[i]);
}

// ASSIGN false: the chunk's counts; true: what becomes of each of its rows.
template <bool ASSIGN>
__global__ __launch_bounds__(256) void select_place_kernel(BatchDev b, Kv8Dev c, int Hkv, int budget,
                                                           SelectWs w, int32_t* __restrict__ plan,
                                                           int32_t* __restrict__ new_len) {
  __shared__ uint32_t red[4], found[2];
  __shared__ int sums[4][2], total[2][4][2];
  const int s = blockIdx.z, h = blockIdx.y, tid = threadIdx.x, chunk = blockIdx.x;
  const int r0 = chunk * kSelChunk + tid * kSelK;
  const int64_t pair = (int64_t)s * Hkv + h;
  int sl;
  const int n = select_rows(b, c, s, sl);
  int32_t* out = plan + pair * budget;
  if (ASSIGN && h == 0 && chunk == 0 && tid == 0 && new_len) new_len[s] = min(n, budget);
  if (n <= budget) {
    if (ASSIGN)
      for (int r = chunk * kSelChunk + tid; r < min(budget, (chunk + 1) * kSelChunk); r += 256)
        out[r] = r < n ? r : -1;
    return;
  }
  if (chunk * kSelChunk >= n) return;
  const u32x4* kp = (const u32x4*)(w.keys_of(pair) + r0);
  const u32x4 x = kp[0], y = kp[1];
  int need;
  const uint32_t T = select_digits<3>(w, pair, budget, red, found, need);
  uint32_t key[kSelK];
  int gt = 0, eq = 0, gt_low = 0, eq_low = 0;  // (low: rows below budget)
#pragma unroll
  for (int i = 0; i < kSelK; ++i) {
    key[i] = i < 4 ? x[i] : y[i - 4];
    const int g = r0 + i < n && key[i] > T, e = r0 + i < n && key[i] == T;
    gt += g;
    eq += e;
    gt_low += r0 + i < budget ? g : 0;
    eq_low += r0 + i < budget ? e : 0;
  }
  int ngt, neq, all_gt, all_eq;
  block_prefix2<4>(gt, eq, ngt, neq, all_gt, all_eq, sums);
  int32_t* counts = w.count + pair * w.chunks * 4;
  if constexpr (!ASSIGN) {
    __syncthreads();
    int a, e, low_gt, low_eq;
    block_prefix2<4>(gt_low, eq_low, a, e, low_gt, low_eq, sums);
    if (tid == 0) *(int4*)(counts + 4 * chunk) = make_int4(all_gt, all_eq, low_gt, low_eq);
    return;
  } else {
    // counts of the chunks before this one, and of all rows below budget
    int before_gt = 0, before_eq = 0, low_gt = 0, low_eq = 0;
    for (int i = tid; i < cdiv(n, kSelChunk); i += 256) {
      const int4 v = *(const int4*)(counts + 4 * i);
      before_gt += i < chunk ? v.x : 0;
      before_eq += i < chunk ? v.y : 0;
      low_gt += v.z;
      low_eq += v.w;
    }
    int a, e, g0, e0, g1, e1;
    block_prefix2<4>(before_gt, before_eq, a, e, g0, e0, total[0]);
    block_prefix2<4>(low_gt, low_eq, a, e, g1, e1, total[1]);
    const int kept_low = g1 + min(e1, need);
    ngt += g0;
    neq += e0;
#pragma unroll
    for (int i = 0; i < kSelK; ++i) {
      const int r = r0 + i;
      const bool same = key[i] == T, keep = r < n && (key[i] > T || (same && neq < need));
      const int place = ngt + min(neq, need);
      ngt += key[i] > T;
      neq += same;
      if (r < budget) out[r] = keep ? r : -2 - (r - place);
      else if (keep) w.list[pair * w.list_rows + place - kept_low] = r;
    }
  }
}

__global__ __launch_bounds__(256) void select_pair_kernel(int budget, SelectWs w,
                                                          int32_t* __restrict__ plan) {
  const int64_t pair = (int64_t)blockIdx.z * gridDim.y + blockIdx.y;
  const int r = blockIdx.x * 256 + threadIdx.x;
  if (r >= budget) return;
  int32_t* out = plan + pair * budget + r;
  const int v = *out;
  if (v <= -2) *out = w.list[pair * w.list_rows + (-2 - v)];
}

static int select_most(const BatchDev& b) {
  return (int)std::min<int64_t>((int64_t)b.max_ctx_len + b.max_q_len, 0x7fffffff - kSelChunk);
}
size_t kv8_select_workspace_bytes(const BatchDev& b, int n_kv_heads, int budget) {
  const int most = select_most(b);
  if (most <= kSelOneRows || most <= budget) return 0;
  const size_t pairs = (size_t)b.n_seqs * n_kv_heads, chunks = cdiv(most, kSelChunk);
  const size_t list = std::min(budget, most - budget);
  return 4 * pairs * (chunks * kSelChunk + kSelHist + chunks * 5 + (list + 3) / 4 * 4) + 64;
}

hipError_t launch_kv8_select(const BatchDev& b, const Kv8Dev& c, int n_kv_heads, int budget,
                             int n_first, int n_recent, int32_t* plan, int32_t* new_len, void* ws,
                             hipStream_t s) {
  if (b.n_seqs == 0) return hipSuccess;
  const int most = select_most(b);
  if (most <= kSelOneRows || most <= budget) {
    auto go = [&](auto kernel) {
      kernel<<<dim3(n_kv_heads, b.n_seqs), kSelThreads, 0, s>>>(b, c, n_kv_heads, budget, n_first,
                                                               n_recent, plan, new_len);
      return hipGetLastError();
    };
    if (most <= 2 * kSelThreads || most <= budget) return go(kv8_select_kernel<2>);
    if (most <= 4 * kSelThreads) return go(kv8_select_kernel<4>);
    if (most <= 8 * kSelThreads) return go(kv8_select_kernel<8>);
    return go(kv8_select_kernel<16>);
  }
  SelectWs w{};
  const size_t pairs = (size_t)b.n_seqs * n_kv_heads;
  w.chunks = cdiv(most, kSelChunk);
  w.list_rows = std::min(budget, most - budget);
  w.key = (uint32_t*)ws;
  w.count = (int32_t*)(w.key + pairs * w.chunks * kSelChunk);
  w.hist = (uint32_t*)(w.count + pairs * w.chunks * 4);
  w.newest = w.hist + pairs * kSelHist;
  w.list = (int32_t*)(w.newest + pairs * w.chunks);
  const dim3 grid(w.chunks, n_kv_heads, b.n_seqs);
  select_newest_kernel<<<grid, 256, 0, s>>>(b, c, n_kv_heads, budget, w);
  select_hist_kernel<0><<<grid, 256, 0, s>>>(b, c, n_kv_heads, budget, n_first, n_recent, w);
  select_hist_kernel<1><<<grid, 256, 0, s>>>(b, c, n_kv_heads, budget, n_first, n_recent, w);
  select_hist_kernel<2><<<grid, 256, 0, s>>>(b, c, n_kv_heads, budget, n_first, n_recent, w);
  select_place_kernel<false><<<grid, 256, 0, s>>>(b, c, n_kv_heads, budget, w, plan, new_len);
  select_place_kernel<true><<<grid, 256, 0, s>>>(b, c, n_kv_heads, budget, w, plan, new_len);
  select_pair_kernel<<<dim3(cdiv(budget, 256), n_kv_heads, b.n_seqs), 256, 0, s>>>(budget, w, plan);
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
