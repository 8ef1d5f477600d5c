// Attention of single tokens over the 8-bit cache, and the merge of its splits with
// the sums of attention weights.
//
// A token reads its sequence's whole cache once, two flops a byte and query head, so
// bytes bound it: the kernel is a stream of the cache with the arithmetic under it.
// One wave per (split of the rows, KV head and 16 of its query heads, sequence), tiles
// of kTile8 rows, two in flight while one is used, ordered by the wave's own vmcnt.
//
// Codes become float16, which holds every one of them exactly (int8: a byte permute under
// the exponent of 1024 and a packed subtraction; e4m3: the conversion instruction), and
// both products run on v_mfma_f32_16x16x32_f16 with the query heads as columns.  q is
// bf16: a power of two per head brings its largest value to [2^14, 2^15), where its 8
// bits are exact in float16 down to 2^-28 of that largest value.  The contraction's order
// is free, so a lane's 16-byte load of K feeds two steps as it comes.  V goes through a
// wave-private LDS ring and is transposed by ds_read_b64_tr_b8.
//
// A block's value scale 2^e joins the exponent of the weights: with t = score + e (log2)
// and M its running maximum over rows, P' = 2^(t - M) multiplies the codes and the
// sum of weights takes P' 2^-e.  So P' is at most 2^8 (the maximum is raised lazily) and
// the largest contribution is near 1 whatever the scales: float16 rounds it to 11 bits.
#include "kv8.hpp"
#include "attn_kv8.hpp"

namespace tri {

constexpr int kTile8 = 64;       // rows per tile
constexpr int kStages8 = 3;      // LDS ring depth
constexpr int kMinSplit8 = 128;  // rows per split, at least
constexpr int kMaxSplit8 = 64 * 32;  // a lane keeps the scales of one 32-row group

static int waves_per_cu8(int head_dim) {
  const int by_lds = (160 * 1024) / (kStages8 * kTile8 * head_dim);
  return std::min(by_lds, 8);  // two waves per SIMD by registers
}

// Splits of max_kv rows: as many as make one round of resident waves, none under
// kMinSplit8 or over kMaxSplit8 rows.  `most`: a round's room or the sequences in shortest
// splits, whichever is less, or the sequences in longest splits.  (Not n_seqs times the
// splits of one: that product falls where the quotient for one sequence steps down.)
Kv8Splits kv8_splits(int n_seqs, int n_q_heads, int n_kv_heads, int head_dim, int max_kv) {
  const int64_t per_split = (int64_t)n_kv_heads * cdiv(n_q_heads / n_kv_heads, 16);  // waves
  const int64_t resident = (int64_t)waves_per_cu8(head_dim) * cu_count(), seqs = std::max(n_seqs, 1);
  const int64_t want = std::max<int64_t>(1, resident / (per_split * seqs));
  const int n = (int)std::min<int64_t>(want, cdiv(max_kv, kMinSplit8));
  const int rows = std::min(cdiv(cdiv(max_kv, n), kTile8) * kTile8, kMaxSplit8);
  const int64_t most = std::max(std::min(resident / per_split, seqs * cdiv(max_kv, kMinSplit8)),
                                seqs * cdiv(max_kv, kMaxSplit8));
  return Kv8Splits{cdiv(max_kv, rows), rows, most};
}

__device__ __forceinline__ uint32_t lds_offset(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)p;
}

// Eight transposing reads (within 16 lanes, lane j receives byte m = 0..7 from the byte
// at (address of lane 2 m + j / 8) + j % 8), then an LDS wait, in one block: outside the
// compiler's tracking of LDS fills, which the caller has waited for.
__device__ __forceinline__ void lds_read_tr8_x8(const uint32_t (&a)[8], u32x2 (&o)[8]) {
  asm volatile(
      "ds_read_b64_tr_b8 %0, %8\n\t"
      "ds_read_b64_tr_b8 %1, %9\n\t"
      "ds_read_b64_tr_b8 %2, %10\n\t"
      "ds_read_b64_tr_b8 %3, %11\n\t"
      "ds_read_b64_tr_b8 %4, %12\n\t"
      "ds_read_b64_tr_b8 %5, %13\n\t"
      "ds_read_b64_tr_b8 %6, %14\n\t"
      "ds_read_b64_tr_b8 %7, %15\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(o[0]), "=&v"(o[1]), "=&v"(o[2]), "=&v"(o[3]), "=&v"(o[4]), "=&v"(o[5]), "=&v"(o[6]),
        "=&v"(o[7])
      : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "v"(a[4]), "v"(a[5]), "v"(a[6]), "v"(a[7])
      : "memory");
}

// V tile in LDS: physical 16-byte chunk of logical chunk c in row r, so that the rows of
// a transposing read (r0 .. r0 + 7 and 16 more, one chunk) fall on different banks: D =
// 128 two rows per 256-byte window, D = 64 four.
template <int D>
__device__ __forceinline__ int v8_chunk(int c, int r) {
  if constexpr (D == 128) return c ^ (((r >> 1) & 3) | (((r >> 4) & 1) << 2));
  else return c ^ (((r >> 2) & 1) | (((r >> 4) & 1) << 1));
}

template <int D, bool FP8, bool PAGED>
__global__ __launch_bounds__(64, 2) void attn_kv8_decode_kernel(
    BatchDev b, Kv8Dev c, int Hq, int Hkv, const bf16* __restrict__ Q, int64_t qs,
    float* __restrict__ part, float* __restrict__ scores, int score_ld, int nsplit, int split_rows,
    float scale_log2e) {
  constexpr int CPR = D / 16;             // 16-byte chunks of a row
  constexpr int KB = kTile8 / 16;         // 16-row blocks of a tile
  constexpr int KJ = D / 64;              // K chunks of a lane and block
  constexpr int VL = kTile8 * D / 1024;   // 1 KB loads of a V tile
  constexpr int LPI = VL + KB * KJ;       // loads of a tile
  constexpr int DB = D / 16;              // 16-value blocks of the output
  __shared__ __align__(16) uint8_t vring[kStages8][kTile8 * D];

  const int s = blockIdx.z, sp = blockIdx.x, grp = Hq / Hkv, hblocks = cdiv(grp, 16);
  const int h = blockIdx.y / hblocks, hb = blockIdx.y - h * hblocks;
  int t, n, ctx, sl;
  if (!kv8_seq(b, c, s, t, n, ctx, sl) || n != 1) return;
  const int rows_seen = min(ctx, b.max_ctx_len) + 1;  // (the buffers' bound)
  const int k_begin = sp * split_rows, k_end = min(rows_seen, k_begin + split_rows);
  if (k_begin >= k_end) return;
  const int nt = cdiv(k_end - k_begin, kTile8);
  const int lane = threadIdx.x, r = lane & 15, g = lane >> 4;
  const int heads = min(16, grp - 16 * hb), head0 = h * grp + 16 * hb;
  const int prows = c.kv.panel_rows(), spp = c.scales_per_panel();

  // Lane j: the page of the split's 32-row group j (-1: none), its scales (rows past the
  // end keep 1: whatever is there reaches nothing).
  int panel_of = sl;
  float ksc = 1.f, vsc = 1.f;
  {
    const int row = k_begin + 32 * lane;
    if (row < k_end) {
      int prow;
      const int panel = kv_panel(c.kv, sl, row, prow);
      panel_of = panel;
      if (panel >= 0) {
        const int64_t at = ((int64_t)panel * Hkv + h) * spp + (prow >> c.scale_shift);
        ksc = c.k_scale[at];
        vsc = c.v_scale[at];
      }
    }
  }
  // The waves of one split index start at different tiles, so that the grid does not
  // read every sequence at the same offset at once.
  const int rot = (int)(((unsigned)s * 7u + blockIdx.y * 3u) % (unsigned)nt);
  auto phys = [&](int i) {
    const int j = i + rot;
    return i < nt ? (j >= nt ? j - nt : j) : i;
  };
  // Rows past the end, tiles past the split and pages outside the pool read as zero.
  auto tile_rsrc = [&](const uint8_t* base, int i) {
    const int key0 = k_begin + kTile8 * phys(i);
    int panel = sl, prow = key0, rows = 0;
    if (i < nt) {
      rows = min(kTile8, k_end - key0);
      if (PAGED) {
        panel = __builtin_amdgcn_readlane(panel_of, (key0 - k_begin) >> 5);
        prow = key0 % prows;
        if (panel < 0) rows = 0;
      }
    }
    if (rows == 0) panel = prow = 0;
    return __builtin_amdgcn_make_buffer_rsrc(
        (void*)(base + (((int64_t)panel * Hkv + h) * prows + prow) * D), (short)0, rows * D,
        0x00020000);
  };
  uint32_t v_off[VL];
#pragma unroll
  for (int j = 0; j < VL; ++j) {
    const int row = j * (64 / CPR) + lane / CPR;
    v_off[j] = (uint32_t)(row * D + v8_chunk<D>(lane % CPR, row) * 16);
  }
  auto issue_v = [&](int i) {
    const __amdgpu_buffer_rsrc_t rv = tile_rsrc(c.v, i);
#pragma unroll
    for (int j = 0; j < VL; ++j) buffer_load_lds16(rv, &vring[i % kStages8][j * 1024], v_off[j], 0);
  };
  // Lane (r, g): row 16 kb + r, chunks g and (D = 128) g + 4.
  u32x4 kreg[2][KB * KJ];
  auto issue_k = [&](auto slot, int i) {
    const __amdgpu_buffer_rsrc_t rk = tile_rsrc(c.k, i);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int j = 0; j < KJ; ++j)
        kreg[decltype(slot)::value][kb * KJ + j] = __builtin_bit_cast(
            u32x4, __builtin_amdgcn_raw_buffer_load_b128(rk, r * D + (g + 4 * j) * 16, kb * 16 * D, 0));
  };
  // q of head column r (columns past the group repeat its last head and are not
  // written): step 2 j + u takes values 16 (g + 4 j) + 8 u ...
  f16x8 qf[2 * KJ];
  float q_back;
  {
    const bf16* qp = Q + (int64_t)t * qs + (int64_t)(head0 + min(r, heads - 1)) * D;
    Pack8 x[2 * KJ];
#pragma unroll
    for (int j = 0; j < 2 * KJ; ++j) x[j].u = ldg16(qp + 16 * (g + 4 * (j >> 1)) + 8 * (j & 1));
    issue_v(0);
    issue_k(Int<0>{}, 0);
    issue_v(1);
    issue_k(Int<1>{}, 1);
    q_back = q_to_f16<48>(x, qf);
  }
  const float score_scale = q_back * scale_log2e;

  f32x4 oacc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) oacc[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = -INFINITY, l_run = 0.f;  // log2 units

  auto step = [&](auto slot, int i) {
    constexpr int ks = decltype(slot)::value;
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LPI) : "memory");  // tile i has landed
    issue_v(i + 2);  // into the stage of tile i - 1, whose reads are done
    const int tile = phys(i), key0 = k_begin + kTile8 * tile;
    // scores: element e of block kb is row key0 + 16 kb + 4 g + e, head column r
    f32x4 sc[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      sc[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < KJ; ++j) {
        const u32x4 k = kreg[ks][kb * KJ + j];
        sc[kb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_f16<FP8>(k[0], k[1]), qf[2 * j], sc[kb], 0, 0, 0);
        sc[kb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_f16<FP8>(k[2], k[3]), qf[2 * j + 1], sc[kb], 0, 0, 0);
      }
    }
    issue_k(slot, i + 2);  // the slot's codes have been read
    float kf[KB / 2], ve[KB / 2], vinv[KB / 2];
#pragma unroll
    for (int u = 0; u < KB / 2; ++u) {
      kf[u] = readlane_f(ksc, 2 * tile + u) * score_scale;
      const float v = readlane_f(vsc, 2 * tile + u);
      ve[u] = scale_log2(v);
      vinv[u] = scale_inverse(v);
    }
    if (scores && r < heads) {
      float* sp_ = scores + ((int64_t)s * Hq + head0 + r) * score_ld + key0 + 4 * g;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) *(f32x4*)(sp_ + 16 * kb) = sc[kb] * kf[kb / 2];
    }
    float mt = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = fmaf(sc[kb][e], kf[kb / 2], ve[kb / 2]);
        sc[kb][e] = key0 + 16 * kb + 4 * g + e < k_end ? x : -INFINITY;
        mt = fmaxf(mt, sc[kb][e]);
      }
    mt = fmaxf(mt, __shfl_xor(mt, 16, 64));
    mt = fmaxf(mt, __shfl_xor(mt, 32, 64));
    const bool raise = mt > m_run + kSoftmaxSlack;
    if (__builtin_amdgcn_ballot_w64(raise)) {
      const float m_new = raise ? mt : m_run;
      const float alpha = raise ? __builtin_amdgcn_exp2f(m_run - m_new) : 1.f;
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int d = 0; d < DB; ++d) oacc[d] *= alpha;
    }
    f16x8 p[KB / 2];
#pragma unroll
    for (int u = 0; u < KB / 2; ++u) {
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = __builtin_amdgcn_exp2f(sc[2 * u + (e >> 2)][e & 3] - m_run);
      l_run = fmaf(tree_sum8(w), vinv[u], l_run);
#pragma unroll
      for (int e = 0; e < 8; ++e) p[u][e] = (f16)w[e];
    }
    // O^T += V^T P'^T: slot e of lane group g is row 4 g + e (16 + 4 g + e - 4 for e >= 4)
    // of the 32 rows.
    const uint8_t* vt = vring[i % kStages8];
#pragma unroll
    for (int u = 0; u < KB / 2; ++u) {
      const int m = (lane & 15) >> 1;
      const int row = 32 * u + 4 * g + (m & 3) + 16 * (m >> 2);
#pragma unroll
      for (int d0 = 0; d0 < DB; d0 += (DB < 8 ? DB : 8)) {
        uint32_t a[8];
        u32x2 v[8];
#pragma unroll
        for (int d = 0; d < 8; ++d)
          a[d] = lds_offset(vt + row * D + v8_chunk<D>(d0 + d % DB, row) * 16 + 8 * (lane & 1));
        lds_read_tr8_x8(a, v);
#pragma unroll
        for (int d = 0; d < (DB < 8 ? DB : 8); ++d)
          oacc[d0 + d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_f16<FP8>(v[d][0], v[d][1]), p[u], oacc[d0 + d], 0, 0, 0);
      }
    }
  };
  int i = 0;
  for (; i + 1 < nt; i += 2) {
    step(Int<0>{}, i);
    step(Int<1>{}, i + 1);
  }
  if (i < nt) step(Int<0>{}, i);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no load may land after exit

  l_run += __shfl_xor(l_run, 16, 64);
  l_run += __shfl_xor(l_run, 32, 64);
  if (r >= heads) return;
  float* pp = part + (((int64_t)s * Hq + head0 + r) * nsplit + sp) * (D + 4);
#pragma unroll
  for (int d = 0; d < DB; ++d) *(f32x4*)(pp + 16 * d + 4 * g) = oacc[d];
  if (g == 0) *(f32x2*)(pp + D) = f32x2{m_run, l_run};
}

// The sums of a single token's attention weights, and the merge of its splits.
// Workgroups x < mass_wgs (the longer ones, first): kMassRows rows of a KV head, four
// neighbouring rows a thread; mass[row] += sum over the heads of 2^(score - M - log2 L).
// The others: query head x; M = max m_j, L = sum l_j 2^(m_j - M), out = sum O_j 2^(m_j -
// M) / L, TS threads' worth of splits side by side.
constexpr int kMassRows = 1024;

template <int D>
__global__ __launch_bounds__(256) void attn_kv8_merge_kernel(
    BatchDev b, Kv8Dev c, int Hq, int Hkv, const float* __restrict__ part, bf16* __restrict__ O,
    const float* __restrict__ scores, int score_ld, int nsplit, int split_rows, int mass_wgs) {
  constexpr int TD = D / 4, TS = 256 / TD;  // threads over d, and over splits
  __shared__ float red[TS][D];
  __shared__ float lse[32], ms[TS], ls[TS];
  const int s = blockIdx.y, tid = threadIdx.x;
  int t, n, ctx, sl;
  if (!kv8_seq(b, c, s, t, n, ctx, sl) || n != 1) return;
  const int rows_seen = min(ctx, b.max_ctx_len) + 1;
  const int ns = min(cdiv(rows_seen, split_rows), nsplit);
  if ((int)blockIdx.x < mass_wgs) {
    const int grp = Hq / Hkv, chunks = mass_wgs / Hkv;
    const int h = (int)blockIdx.x / chunks, row0 = ((int)blockIdx.x % chunks) * kMassRows;
    if (row0 >= rows_seen) return;
    // this thread's rows: their mass and the first heads' scores are under way while the
    // heads' log-sum-exps are formed, eight threads a head
    const int row = row0 + 4 * tid;
    int prow = 0;
    const int panel = row < rows_seen ? kv_panel(c.kv, sl, row, prow) : -1;
    const float* sp = scores + ((int64_t)s * Hq + h * grp) * score_ld + (panel < 0 ? row0 : row);
    float* mp = c.mass + kv8_row_at(c, Hkv, max(panel, 0), h, prow);
    float before[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) before[e] = panel >= 0 && row + e < rows_seen ? mp[e] : 0.f;
    f32x4 x[4];
    auto load = [&](int q0) {
#pragma unroll
      for (int q = 0; q < 4; ++q) x[q] = *(const f32x4*)(sp + (int64_t)min(q0 + q, grp - 1) * score_ld);
    };
    load(0);
    {
      const int q = tid >> 3;
      const float* pp = part + ((int64_t)s * Hq + h * grp + min(q, grp - 1)) * nsplit * (D + 4) + D;
      float M = -INFINITY, L = 0.f;
      for (int j = tid & 7; j < ns; j += 8) {
        const f32x2 ml = *(const f32x2*)(pp + (int64_t)j * (D + 4));
        const float Mn = fmaxf(M, ml[0]);
        L = (M == -INFINITY ? 0.f : L * exp2f(M - Mn)) + ml[1] * exp2f(ml[0] - Mn);
        M = Mn;
      }
      float top = M;
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
      L = (tid & 7) < ns ? L * exp2f(M - top) : 0.f;
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) L += __shfl_xor(L, o, 64);
      if ((tid & 7) == 0) lse[q] = top + log2f(L);
    }
    __syncthreads();
    if (panel < 0) return;
    f32x4 sum = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int q0 = 0; q0 < grp; q0 += 4) {
      if (q0 > 0) load(q0);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (q0 + q >= grp) break;
        const float off = lse[q0 + q];
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += __builtin_amdgcn_exp2f(x[q][e] - off);
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (row + e < rows_seen) mp[e] = before[e] + sum[e];
    return;
  }
  const int qh = (int)blockIdx.x - mass_wgs;
  const float* pp = part + ((int64_t)s * Hq + qh) * nsplit * (D + 4);
  const int d = 4 * (tid % TD), j0 = tid / TD;
  float M = -INFINITY, L = 0.f;
  f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int j = j0; j < ns; j += TS) {
    const float* q = pp + (int64_t)j * (D + 4);
    const f32x2 ml = *(const f32x2*)(q + D);
    const f32x4 a = *(const f32x4*)(q + d);
    const float Mn = fmaxf(M, ml[0]);
    const float x = M == -INFINITY ? 0.f : exp2f(M - Mn), w = exp2f(ml[0] - Mn);
    L = L * x + ml[1] * w;
    o = o * x + a * w;
    M = Mn;
  }
  // the TS threads of a d: through LDS in order, with the common maximum
  if (tid % TD == 0) ms[j0] = M;
  __syncthreads();
  float top = ms[0];
#pragma unroll
  for (int j = 1; j < TS; ++j) top = fmaxf(top, ms[j]);
  const float w = j0 < ns ? exp2f(M - top) : 0.f;
  if (tid % TD == 0) ls[j0] = j0 < ns ? L * w : 0.f;
  *(f32x4*)&red[j0][d] = j0 < ns ? o * w : f32x4{0.f, 0.f, 0.f, 0.f};
  __syncthreads();
  if (tid < D) {
    float sum = 0.f, l = 0.f;
#pragma unroll
    for (int j = 0; j < TS; ++j) {
      sum += red[j][tid];
      l += ls[j];
    }
    O[((int64_t)t * Hq + qh) * D + tid] = f2bf(sum / l);
  }
}

// Workspace: the splits' partials, then the scores where weights are summed.
static size_t score_bytes(const BatchDev& b, const Kv8Dev& c, int n_q_heads) {
  return c.mass ? (size_t)b.n_seqs * n_q_heads * cdiv(b.max_ctx_len + 1, kTile8) * kTile8 * 4 : 0;
}
size_t attn_kv8_decode_bytes(const BatchDev& b, const Kv8Dev& c, int n_q_heads, int n_kv_heads,
                             int head_dim) {
  const int64_t most = kv8_splits(b.n_seqs, n_q_heads, n_kv_heads, head_dim, b.max_ctx_len + 1).most;
  return (size_t)most * n_q_heads * (head_dim + 4) * 4 + score_bytes(b, c, n_q_heads);
}

template <int D, bool FP8>
static hipError_t run_decode8(const BatchDev& b, const Kv8Dev& c, int Hq, int Hkv, const void* q,
                              int64_t qs, void* out, float* part, hipStream_t s) {
  const int max_kv = b.max_ctx_len + 1;
  const Kv8Splits sp = kv8_splits(b.n_seqs, Hq, Hkv, D, max_kv);
  float* scores = c.mass ? part + (size_t)sp.most * Hq * (D + 4) : nullptr;
  const int ld = cdiv(max_kv, kTile8) * kTile8;
  const float scale_log2e = (float)(1.4426950408889634 / __builtin_sqrt((double)D));
  const dim3 grid(sp.n, Hkv * cdiv(Hq / Hkv, 16), b.n_seqs);
  auto go = [&](auto kernel) {
    kernel<<<grid, 64, 0, s>>>(b, c, Hq, Hkv, (const bf16*)q, qs, part, scores, ld, sp.n, sp.rows,
                               scale_log2e);
    return hipGetLastError();
  };
  hipError_t e = c.kv.table ? go(attn_kv8_decode_kernel<D, FP8, true>)
                            : go(attn_kv8_decode_kernel<D, FP8, false>);
  if (e != hipSuccess) return e;
  const int mass_wgs = c.mass ? Hkv * cdiv(max_kv, kMassRows) : 0;
  attn_kv8_merge_kernel<D><<<dim3(mass_wgs + Hq, b.n_seqs), 256, 0, s>>>(
      b, c, Hq, Hkv, part, (bf16*)out, scores, ld, sp.n, sp.rows, mass_wgs);
  return hipGetLastError();
}

hipError_t launch_attn_kv8_decode(const BatchDev& b, const Kv8Dev& c, bool fp8, int n_q_heads,
                                  int n_kv_heads, int head_dim, const void* q, int64_t q_stride,
                                  void* out, float* ws, hipStream_t s) {
  if (head_dim == 128)
    return fp8 ? run_decode8<128, true>(b, c, n_q_heads, n_kv_heads, q, q_stride, out, ws, s)
               : run_decode8<128, false>(b, c, n_q_heads, n_kv_heads, q, q_stride, out, ws, s);
  return fp8 ? run_decode8<64, true>(b, c, n_q_heads, n_kv_heads, q, q_stride, out, ws, s)
             : run_decode8<64, false>(b, c, n_q_heads, n_kv_heads, q, q_stride, out, ws, s);
}

}  // namespace tri
