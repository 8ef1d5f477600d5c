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
// thread with their keys in registers (4352 rows: 64 x 4 heads in 17.5 us).
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
template <int W, int BINS>
__device__ __forceinline__ void select_bin(const uint32_t* hist, int need, uint32_t* red,
                                           uint32_t* found, int& bin, int& above) {
  constexpr int PER = BINS / (64 * W);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t cnt[PER], mine = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    cnt[i] = hist[BINS - 1 - (tid * PER + i)];
    mine += cnt[i];
  }
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
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (over < (uint32_t)need && over + cnt[i] >= (uint32_t)need) {
      found[0] = (uint32_t)(BINS - 1 - (tid * PER + i));
      found[1] = over;
    }
    over += cnt[i];
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
  auto digit = [&](auto pass_) {
    constexpr int PASS = decltype(pass_)::value, SHIFT = select_shift(PASS), BINS = select_bins(PASS);
    constexpr uint32_t mask = PASS == 0 ? 0u : ~0u << (PASS == 1 ? 21 : 10);
    for (int i = tid; i < BINS; i += kSelThreads) hist[i] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < K; ++i)
      if (r0 + i < n && (key[i] & mask) == T) atomicAdd(&hist[(key[i] >> SHIFT) & (BINS - 1)], 1u);
    __syncthreads();
    int bin, above;
    select_bin<W, BINS>(hist, need, red, found, bin, above);
    T |= (uint32_t)bin << SHIFT;
    need -= above;
  };
  digit(Int<0>{});
  digit(Int<1>{});
  digit(Int<2>{});
  // Kept before a row: the greater keys and the first `need` equal ones.
  int gt = 0, eq = 0;
#pragma unroll
  for (int i = 0; i < K; ++i) {
    gt += r0 + i < n && key[i] > T;
    eq += r0 + i < n && key[i] == T;
  }
  int ngt, neq, all_gt, all_eq;
  block_prefix2<W>(gt, eq, ngt, neq, all_gt, all_eq, sums);
  int place[K];       // kept rows before each row
  uint32_t keep = 0;  // bit i: row i stays
#pragma unroll
  for (int i = 0; i < K; ++i) {
    const int more = r0 + i < n && key[i] > T, same = r0 + i < n && key[i] == T;
    place[i] = ngt + min(neq, need);
    keep |= (uint32_t)(more | (same & (int)(neq < need))) << i;
    if (r0 + i == budget) kept_low_at = place[i];
    ngt += more;
    neq += same;
  }
  __syncthreads();
  const int kept_low = kept_low_at;
#pragma unroll
  for (int i = 0; i < K; ++i)
    if ((keep >> i & 1) && r0 + i >= budget) list[place[i] - kept_low] = r0 + i;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < K; ++i) {
    const int r = r0 + i;
    if (r < budget) out[r] = (keep >> i & 1) ? r : list[r - place[i]];
  }
}

// The same in steps over chunks (grid: chunk, head, sequence).  Per (sequence, head) in the
// workspace: every row's key, the histograms, and of every chunk its newest stamp and its
// counts of greater and equal keys; the rows that move, in order.
struct SelectWs {
  uint32_t *key, *hist, *newest;
  int32_t *count, *list;
  uint2* state;  // T's digits so far, equal keys still needed (after pass 0 at 0, ...)
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

// T's digits and the equal keys still needed after histogram PASS: one scan on what the
// launch before had found, kept for the next one by the first chunk.
template <int PASS>
__device__ __forceinline__ uint32_t select_digit(const SelectWs& w, int64_t pair, int budget,
                                                 uint32_t* red, uint32_t* found, int& need) {
  uint2 st = PASS == 0 ? make_uint2(0u, (uint32_t)budget) : w.state[2 * pair + PASS - 1];
  int bin, above;
  select_bin<4, select_bins(PASS)>(w.hist_of(pair, PASS), (int)st.y, red, found, bin, above);
  st.x |= (uint32_t)bin << select_shift(PASS);
  st.y -= (uint32_t)above;
  if (PASS < 2 && blockIdx.x == 0 && threadIdx.x == 0) w.state[2 * pair + PASS] = st;
  need = (int)st.y;
  return st.x;
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
    T = select_digit<PASS - 1>(w, pair, budget, red, found, need);
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
  const uint32_t T = select_digit<2>(w, pair, budget, red, found, need);
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
  return 4 * pairs * (chunks * kSelChunk + kSelHist + chunks * 5 + 4 + list);
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
  w.state = (uint2*)(w.key + pairs * w.chunks * kSelChunk);
  w.count = (int32_t*)(w.state + 2 * pairs);
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

// Move.  One wave per (32 rows below budget, head, sequence), four to a workgroup.  Rows
// come from at or past budget and go below it, so no wave reads rows that another writes;
// the waves of one scale block (R = 32 WPB rows) each find its largest scale, and meet once
// before it is written.  A wave's rows are few and its loads depend on each other (plan,
// page, scales, codes), so the waves in flight bound it: sources stay in registers and all
// pieces of codes are in flight at once.  Blocks that nothing moves into end at their plan
// entries; a block whose scale grows is read and written whole.  (64 sequences of 4352 rows to
// 4096, 4 heads of 128, blocks of 32, a first eviction, in which nearly every block's scale
// grows: 44 us, 75 MB read and 71 written, 3.3 TB/s; the same plan once more, where only the
// rows that move are copied: 26 us, 25 and 20 MB.  One sequence of 131072 rows to 65536, blocks
// of 128: 20 us, 49 and 47 MB; once more 21, 39 and 37.)
template <int D, bool FP8, int WPB>
__global__ __launch_bounds__(256) void kv8_move_kernel(BatchDev b, Kv8Dev c, int Hkv, int blocks,
                                                       const int32_t* __restrict__ plan, int budget) {
  constexpr int CPR = D / 16, R = 32 * WPB, RPL = WPB == 4 ? 2 : 1, ITEMS = 32 * CPR / 64;
  const int s = blockIdx.z, h = blockIdx.y, lane = threadIdx.x & 63;
  const int wave = (int)(threadIdx.x >> 6), sub = wave % WPB;
  const int blk = blockIdx.x * (4 / WPB) + wave / WPB, r0 = blk * R;
  const int sl = b.slot[s];
  if (sl < 0 || sl >= c.kv.n_slots) return;
  int prow = 0;
  const int panel = blk < blocks ? kv_panel(c.kv, sl, r0, prow) : -1;
  // Lane j: rows j and (R = 128) j + 64 of the block.
  const int32_t* pl = plan + ((int64_t)s * Hkv + h) * budget + r0;
  int src[RPL];
  bool any = false;
#pragma unroll
  for (int j = 0; j < RPL; ++j) {
    const int r = lane + 64 * j;
    src[j] = panel >= 0 && r < R ? pl[r] : -1;
    if (src[j] >= c.kv.max_seq) src[j] = -1;
    any |= src[j] >= 0 && src[j] != r0 + r;
  }
  const bool live = __builtin_amdgcn_ballot_w64(any) != 0;
  const int64_t row0 = kv8_row_at(c, Hkv, max(panel, 0), h, prow);
  const int64_t at = kv8_scale_at(c, Hkv, max(panel, 0), h, prow);
  int64_t from[RPL];  // row index of the source, -1: no row
  float now[2], f[2][RPL];  // the block's scales; factor of each row's codes, 1: as they are
  if (live) {
    float scale[2][RPL];
    uint32_t top[2] = {0u, 0u};
#pragma unroll
    for (int j = 0; j < RPL; ++j) {
      from[j] = -1;
      scale[0][j] = scale[1][j] = 0.f;
      const int r = lane + 64 * j;
      if (r < R) {
        int p = 0;
        const int sp = src[j] >= 0 ? kv_panel(c.kv, sl, src[j], p) : -1;
        // (a row that is left out stays, under the block's scale as it comes out)
        from[j] = sp >= 0 ? kv8_row_at(c, Hkv, sp, h, p) : row0 + r;
        const int64_t sa = sp >= 0 ? kv8_scale_at(c, Hkv, sp, h, p) : at;
        scale[0][j] = c.k_scale[sa];
        scale[1][j] = c.v_scale[sa];
      }
      top[0] = max(top[0], __float_as_uint(scale[0][j]) & 0x7fffffffu);
      top[1] = max(top[1], __float_as_uint(scale[1][j]) & 0x7fffffffu);
    }
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      now[kv] = __uint_as_float(block_max<1>(top[kv], nullptr));
      const float inv = kv8_inverse(now[kv]);
#pragma unroll
      for (int j = 0; j < RPL; ++j) f[kv][j] = scale[kv][j] == scale[kv][j] ? scale[kv][j] * inv : 0.f;
    }
    // the wave's own rows 32 sub ..
    u32x4 x[2][ITEMS];
    float fac[2][ITEMS];
    uint32_t work = 0;
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      const int i = 64 * j + lane, r = 32 * sub + i / CPR, d = (i % CPR) * 16, l = r & 63;
      int64_t fr = __shfl(from[0], l, 64);
      fac[0][j] = __shfl(f[0][0], l, 64);
      fac[1][j] = __shfl(f[1][0], l, 64);
      if constexpr (RPL == 2) {
        const int64_t fr1 = __shfl(from[1], l, 64);
        const float a = __shfl(f[0][1], l, 64), e = __shfl(f[1][1], l, 64);
        fr = r >= 64 ? fr1 : fr;
        fac[0][j] = r >= 64 ? a : fac[0][j];
        fac[1][j] = r >= 64 ? e : fac[1][j];
      }
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        const bool go = fr >= 0 && !(fr == row0 + r && fac[kv][j] == 1.f);
        work |= (uint32_t)go << (2 * j + kv);
        if (go) x[kv][j] = ldg16((kv ? c.v : c.k) + fr * D + d);
      }
    }
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      const int i = 64 * j + lane, r = 32 * sub + i / CPR, d = (i % CPR) * 16;
#pragma unroll
      for (int kv = 0; kv < 2; ++kv)
        if (work >> (2 * j + kv) & 1) {
          if (fac[kv][j] != 1.f) x[kv][j] = kv8_rescale16<FP8>(x[kv][j], fac[kv][j]);
          stg16((kv ? c.v : c.k) + (row0 + r) * D + d, x[kv][j]);
        }
    }
#pragma unroll
    for (int j = 0; j < RPL; ++j) {
      const int r = lane + 64 * j;
      if (sub == 0 && from[j] >= 0 && from[j] != row0 + r) {
        if (c.mass) c.mass[row0 + r] = c.mass[from[j]];
        if (c.stamp) c.stamp[row0 + r] = c.stamp[from[j]];
      }
    }
  }
  if constexpr (WPB > 1) __syncthreads();  // every wave of the block has read its scales
  if (live && sub == 0 && lane == 0) {
    c.k_scale[at] = now[0];
    c.v_scale[at] = now[1];
  }
}

hipError_t launch_kv8_move(const BatchDev& b, const Kv8Dev& c, bool fp8, int n_kv_heads,
                           int head_dim, const int32_t* plan, int budget, hipStream_t s) {
  if (b.n_seqs == 0) return hipSuccess;
  const int blocks = budget >> c.scale_shift;
  const dim3 grid(cdiv(budget, 128), n_kv_heads, b.n_seqs);
  auto go = [&](auto one, auto two, auto four) {
    const auto kernel = c.scale_shift == 5 ? one : (c.scale_shift == 6 ? two : four);
    kernel<<<grid, 256, 0, s>>>(b, c, n_kv_heads, blocks, plan, budget);
    return hipGetLastError();
  };
  if (head_dim == 128)
    return fp8 ? go(kv8_move_kernel<128, true, 1>, kv8_move_kernel<128, true, 2>, kv8_move_kernel<128, true, 4>)
               : go(kv8_move_kernel<128, false, 1>, kv8_move_kernel<128, false, 2>, kv8_move_kernel<128, false, 4>);
  return fp8 ? go(kv8_move_kernel<64, true, 1>, kv8_move_kernel<64, true, 2>, kv8_move_kernel<64, true, 4>)
             : go(kv8_move_kernel<64, false, 1>, kv8_move_kernel<64, false, 2>, kv8_move_kernel<64, false, 4>);
}

}  // namespace tri
