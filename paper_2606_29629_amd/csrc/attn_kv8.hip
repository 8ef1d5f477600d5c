// Causal flash attention of chunks (sequences of two tokens or more) over the 8-bit
// cache, and the sums of their attention weights.
//
// The query rows of a KV head are its tokens times the group's G query heads, packed: row
// x is head x % G of token x / G.  So K and V are read and converted once for the whole
// group, a chunk of a few tokens fills a tile, and the causal edge crosses few rows of it.
// One workgroup = 128 rows, 4 waves of 32; 64 cache rows per tile.  Two products of 64 x
// 32 x D per wave and tile bound it (32 matrix instructions, 1024 cycles at D = 128);
// beside them 32 exponentials a lane and the tile's fragments out of LDS.
//
// A tile's codes go to registers two tiles ahead, are converted to float16 once per
// workgroup (exact: attn_kv8.hpp) and written to LDS one tile ahead, chunks swizzled by
// kv_chunk, double buffered, one barrier per tile.  S^T = K Q^T and O^T += V^T P'^T on
// v_mfma_f32_32x32x16_f16: a lane owns one query row and 32 of the tile's 64 keys, its
// weights are the second product's operand where they are, and V is transposed by
// ds_read_b64_tr_b16.  Value scales ride in the weights' exponent as in the single-token
// kernel, one float16 rounding (2^-11) per weight.
#include <type_traits>

#include "attn_kv8.hpp"
#include "side.hpp"

namespace tri {

constexpr int kRows8 = 128;    // packed query rows per workgroup
constexpr int kKeys8 = 64;     // cache rows per tile
constexpr int kMaxSplitF8 = 32;  // key-range splits of a row tile, at most

// Thread i of 256 (and 256 more for D = 128) moves 16 codes of a tile: row and chunk, rows
// ordered so that 16 neighbouring threads' float16 chunks fall on different banks (the
// swizzle of rows 4 apart differs in parity).
template <int D>
__device__ __forceinline__ void stage_place(int i, int& row, int& chunk) {
  if constexpr (D == 128) {
    const int r = i >> 3;
    chunk = i & 7;
    row = (r & ~7) | ((r & 1) << 2) | ((r & 7) >> 1);
  } else {
    const int r = i >> 2;
    chunk = i & 3;
    row = (r & ~7) | ((r & 2) << 1) | ((r & 4) >> 1) | (r & 1);
  }
}

// The sequences' pieces laid end to end (those of `least` tokens or more; `pieces` of the
// tokens and cached rows): the sequence of piece `item`, its fields, and which of its pieces
// it is, counted from the last if BACK; false past the end.  Every wave looks for itself, 64
// sequences at a time.  So the workgroups that have work come first: with a grid of the
// longest chunk's pieces for every sequence, those without held up the others, each for the
// time of its loads (8 prompts of 500 to 2048 tokens, 28/4 heads of 128: 243 us, 129 so; 512
// tokens beside 32 single ones, 14300 of 14800 without: 171 us, 141 so).
template <typename F>
__device__ __forceinline__ bool kv8_piece(const BatchDev& b, const Kv8Dev& c, int least, int item,
                                          F&& pieces, int& s, int& piece, int& count, int& q0, int& n,
                                          int& ctx, int& sl) {
  const int lane = threadIdx.x & 63;
  for (int j0 = 0; j0 < b.n_seqs; j0 += 64) {
    int lq, ln, lc, ls;
    const bool ok = kv8_seq(b, c, min(j0 + lane, b.n_seqs - 1), lq, ln, lc, ls) && ln >= least &&
                    j0 + lane < b.n_seqs;
    const int mine = ok ? pieces(ln, lc) : 0;
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(upto, o, 64);
      if (lane >= o) upto += v;
    }
    const uint64_t past = __builtin_amdgcn_ballot_w64(upto > item);
    if (past == 0) {
      item -= __builtin_amdgcn_readlane(upto, 63);
      continue;
    }
    const int at = __builtin_ctzll(past);
    s = j0 + at;
    count = __builtin_amdgcn_readlane(mine, at);
    piece = item - (__builtin_amdgcn_readlane(upto, at) - count);
    q0 = __builtin_amdgcn_readlane(lq, at);
    n = __builtin_amdgcn_readlane(ln, at);
    ctx = __builtin_amdgcn_readlane(lc, at);
    sl = __builtin_amdgcn_readlane(ls, at);
    return true;
  }
  return false;
}

template <int D, bool FP8, bool PAGED, bool SPLIT>
__global__ __launch_bounds__(256, 2) void attn_kv8_kernel(BatchDev b, Kv8Dev c, int Hq, int Hkv,
                                                          const bf16* __restrict__ Q, int64_t qs,
                                                          bf16* __restrict__ O,
                                                          float* __restrict__ lse,
                                                          float* __restrict__ part, int nsplit,
                                                          int least, float scale_log2e) {
  constexpr int DS = D / 16, DB = D / 32;
  constexpr int NL = D / 64;  // 16-code loads of a thread, operand and tile
  __shared__ __align__(16) f16 sk[2][kKeys8 * D], sv[2][kKeys8 * D];

  // Heads, then splits, then the row tiles, those with the most keys first: over all sequences
  // where they are equal chunks (least = 1; 8 of 2048 tokens: 292 us, in turn 308), else
  // sequence by sequence.
  const int per = Hkv * nsplit, h = (int)(blockIdx.x % per) % Hkv, sp = (int)(blockIdx.x % per) / Hkv;
  const int G = Hq / Hkv, item = (int)(blockIdx.x / per);
  int s, tile, tiles, q0, n, ctx, sl;
  if (least == 1) {
    s = item % b.n_seqs;
    tile = item / b.n_seqs;
    tiles = (int)(gridDim.x / per) / b.n_seqs;
    if (!kv8_seq(b, c, s, q0, n, ctx, sl) || n < 1) return;
  } else if (!kv8_piece(b, c, least, item, [&](int tokens, int) { return cdiv(tokens * G, kRows8); }, s,
                        tile, tiles, q0, n, ctx, sl)) {
    return;
  }
  const int rows = n * G, row0 = (tiles - 1 - tile) * kRows8;
  if (row0 >= rows) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, lg = lane >> 5;
  const int kv_len = ctx + (min(rows, row0 + kRows8) - 1) / G + 1;
  const int nkt = cdiv(kv_len, kKeys8);
  const int tps = SPLIT ? cdiv(nkt, nsplit) : nkt;
  const int kt_lo = sp * tps, kt_hi = min(nkt, kt_lo + tps);
  if (kt_lo >= kt_hi) return;  // (the merge skips an empty split)

  const int prows = c.kv.panel_rows(), spp = c.scales_per_panel();
  int st_row[NL], st_chunk[NL];
#pragma unroll
  for (int j = 0; j < NL; ++j) stage_place<D>(tid + 256 * j, st_row[j], st_chunk[j]);
  u32x4 kraw[NL], vraw[NL];
  float ks_next[2], vs_next[2];  // the scales of the tile in kraw, vraw
  // A tile's codes and scales: contiguous, at an offset from the head's first row; paged,
  // from its page.  Rows past the end (and tiles past the last) read as zero.
  auto rsrc = [&](const uint8_t* base, int panel, int rows) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)(base + ((int64_t)panel * Hkv + h) * prows * D), (short)0,
                                             rows * D, 0x00020000);
  };
  const auto rk0 = rsrc(c.k, sl, PAGED ? 0 : kv_len), rv0 = rsrc(c.v, sl, PAGED ? 0 : kv_len);
  const int64_t scale0 = ((int64_t)sl * Hkv + h) * spp;
  auto gload = [&](int kt) {
    auto rk = rk0, rv = rv0;
    int first = min(kt, nkt - 1) * kKeys8;  // row within the panel
    int64_t sa = scale0;
    const int live = kv_len - first;
    if constexpr (PAGED) {
      int panel = kv_panel(c.kv, sl, first, first);
      const int rows = panel < 0 ? 0 : min(prows, first + live);
      panel = max(panel, 0);
      rk = rsrc(c.k, panel, rows);
      rv = rsrc(c.v, panel, rows);
      sa = ((int64_t)panel * Hkv + h) * spp;
    }
#pragma unroll
    for (int j = 0; j < NL; ++j) {
      const int off = st_row[j] * D + st_chunk[j] * 16;
      kraw[j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rk, off, first * D, 0));
      vraw[j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rv, off, first * D, 0));
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {  // (a block wholly past the end takes the other's)
      const int64_t at = sa + ((first + (32 * u < live ? 32 * u : 0)) >> c.scale_shift);
      ks_next[u] = c.k_scale[at];
      vs_next[u] = c.v_scale[at];
    }
  };
  float ks[2], vs[2];
  // Eight codes of a thread's share of the tile in kraw, vraw into LDS: unit u of 4 NL.
  auto convert = [&](auto unit, int buf) {
    constexpr int j = decltype(unit)::value >> 2, is_v = (decltype(unit)::value >> 1) & 1,
                  half = decltype(unit)::value & 1;
    const int r = st_row[j];
    f16* dst = (is_v ? sv : sk)[buf] + r * D + kv_chunk<D>(2 * st_chunk[j] + half, r) * 8;
    const u32x4 x = is_v ? vraw[j] : kraw[j];
    *(f16x8*)dst = codes_to_f16<FP8>(x[2 * half], x[2 * half + 1]);
  };
  auto convert_all = [&](int buf) { each<4 * NL>([&](auto u) { convert(u, buf); }); };

  // This lane's query row (rows past the end repeat the last one and are not written).
  const int row = row0 + wave * 32 + lr, rc = min(row, rows - 1);
  const int tok = rc / G, hq = h * G + rc - tok * G;
  const int qpos = ctx + tok;
  const int wave_lo = ctx + min(row0 + wave * 32, rows - 1) / G;  // the wave's first token
  f16x8 qf[DS];
  float score_scale;
  gload(kt_lo);
  {
    Pack8 x[DS];
    const bf16* qp = Q + (int64_t)(q0 + tok) * qs + (int64_t)hq * D + 8 * lg;
#pragma unroll
    for (int t = 0; t < DS; ++t) x[t].u = ldg16(qp + 16 * t);
    score_scale = q_to_f16<32>(x, qf) * scale_log2e;
  }
  const int tr_key = 4 * lg + ((lane & 15) >> 2);
  const int tr_col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);

  f32x16 oacc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) oacc[d] = f32x16{0.f};
  float m_run = -INFINITY, l_run = 0.f;  // log2 units

  convert_all(0);
  ks[0] = ks_next[0], ks[1] = ks_next[1], vs[0] = vs_next[0], vs[1] = vs_next[1];
  gload(kt_lo + 1);

  // Key tile kt from buffer `buf`.  Both products have other work under them: the first the
  // conversion of the next tile, the second the weights of its next 16 keys.
  auto step = [&](int kt, auto buf) {
    constexpr int other = 1 - decltype(buf)::value;
    __syncthreads();  // tile kt is in LDS; every wave is done with tile kt - 1
    const f16* kb_lds = sk[decltype(buf)::value];
    const f16* vb = sv[decltype(buf)::value];
    const int key0 = kt * kKeys8;
    const float ks_after[2] = {ks_next[0], ks_next[1]}, vs_after[2] = {vs_next[0], vs_next[1]};
    constexpr int KLA = 3;
    f32x16 sacc[2] = {f32x16{0.f}, f32x16{0.f}};
    f16x8 kf[KLA + 1][2];
    auto kread = [&](int t, f16x8 (&dst)[2]) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const int key = kb * 32 + lr;
        dst[kb] = *(const f16x8*)&kb_lds[key * D + kv_chunk<D>(2 * t + lg, key) * 8];
      }
    };
#pragma unroll
    for (int t = 0; t < KLA && t < DS; ++t) kread(t, kf[t]);
    // (past the last tile the codes of the one before are converted again, for nobody)
    each<DS>([&](auto t_) {
      constexpr int t = decltype(t_)::value;
      if constexpr (t + KLA < DS) kread(t + KLA, kf[(t + KLA) % (KLA + 1)]);
      sacc[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[t % (KLA + 1)][0], qf[t], sacc[0], 0, 0, 0);
      convert(t_, other);
      sacc[1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[t % (KLA + 1)][1], qf[t], sacc[1], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    });
    gload(kt + 2);
    union VFrag {
      s16x4 s[2];
      f16x8 h;
    };
    VFrag vf[2][DB];
    auto vread = [&](int g16, VFrag (&dst)[DB]) {
      const int k1 = 16 * g16 + tr_key, k2 = k1 + 8;
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        const int col = 32 * d + tr_col;
        dst[d].s[0] = lds_read_tr16((const bf16*)(vb + k1 * D + kv_chunk<D>(col >> 3, k1) * 8 + (col & 7)));
        dst[d].s[1] = lds_read_tr16((const bf16*)(vb + k2 * D + kv_chunk<D>(col >> 3, k2) * 8 + (col & 7)));
      }
    };
    vread(0, vf[0]);
    // scores in log2 units: kf s + ve
    float kfac[2], ve[2], vinv[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const float f = ks[kb] * score_scale;
      kfac[kb] = f < 1.17549435e-38f ? 1.17549435e-38f : f;  // (not 0: -inf * 0)
      ve[kb] = scale_log2(vs[kb]);
      vinv[kb] = scale_inverse(vs[kb]);
    }
    if (key0 + kKeys8 - 1 > wave_lo) {  // the causal edge crosses this tile
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int key = key0 + 32 * kb + (e & 3) + 8 * (e >> 2) + 4 * lg;
          if (key > qpos) sacc[kb][e] = -INFINITY;
        }
        // a block past this row: none of its scales either (one may be NaN)
        const bool none = key0 + 32 * kb > qpos;
        kfac[kb] = none ? 1.f : kfac[kb];
        ve[kb] = none ? 0.f : ve[kb];
        vinv[kb] = none ? 1.f : vinv[kb];
      }
    }
    const float thr = m_run + kSoftmaxSlack;
    const float mh = fmaxf(fmaf(tree_max16(sacc[0]), kfac[0], ve[0]), fmaf(tree_max16(sacc[1]), kfac[1], ve[1]));
    if (__builtin_amdgcn_ballot_w64(mh > thr)) {
      const float mt = fmaxf(mh, __shfl_xor(mh, 32, 64));
      const bool raise = mt > thr;
      const float m_new = raise ? mt : m_run;
      const float alpha = raise ? __builtin_amdgcn_exp2f(m_run - m_new) : 1.f;
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int d = 0; d < DB; ++d) oacc[d] *= alpha;
    }
    // (a row that precedes every key so far has no maximum; its weights are 0)
    const float m_use = m_run == -INFINITY ? 0.f : m_run;
    const float off[2] = {ve[0] - m_use, ve[1] - m_use};
    f16x8 p[2];          // weights of the 16 keys at work and of the next 16
    float ls[4][2] = {};  // their sums, in pairs
    auto weights = [&](auto g_, auto pair_) {
      constexpr int g = decltype(g_)::value, i = decltype(pair_)::value, kb = g >> 1, e = 8 * (g & 1) + 2 * i;
      const float a = __builtin_amdgcn_exp2f(fmaf(sacc[kb][e], kfac[kb], off[kb]));
      const float c2 = __builtin_amdgcn_exp2f(fmaf(sacc[kb][e + 1], kfac[kb], off[kb]));
      ls[g][0] = i == 0 ? a : ls[g][0] + a;
      ls[g][1] = i == 0 ? c2 : ls[g][1] + c2;
      p[g & 1][2 * i] = (f16)a;
      p[g & 1][2 * i + 1] = (f16)c2;
    };
    each<4>([&](auto i) { weights(Int<0>{}, i); });
    each<4>([&](auto g_) {
      constexpr int g = decltype(g_)::value;
      if constexpr (g + 1 < 4) vread(g + 1, vf[(g + 1) & 1]);
      each<DB>([&](auto d_) {
        constexpr int d = decltype(d_)::value;
        oacc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[g & 1][d].h, p[g & 1], oacc[d], 0, 0, 0);
        if constexpr (g + 1 < 4)
          each<4 / DB>([&](auto j) { weights(Int<g + 1>{}, Int<d * (4 / DB) + decltype(j)::value>{}); });
      });
      __builtin_amdgcn_sched_barrier(0);
    });
    l_run = fmaf((ls[0][0] + ls[0][1]) + (ls[1][0] + ls[1][1]), vinv[0], l_run);
    l_run = fmaf((ls[2][0] + ls[2][1]) + (ls[3][0] + ls[3][1]), vinv[1], l_run);
    ks[0] = ks_after[0], ks[1] = ks_after[1], vs[0] = vs_after[0], vs[1] = vs_after[1];
  };
  for (int kt = kt_lo; kt < kt_hi; kt += 2) {
    step(kt, Int<0>{});
    if (kt + 1 < kt_hi) step(kt + 1, Int<1>{});
  }

  const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
  if (row >= rows) return;
  // packed rows of all sequences in order: q0 G + row
  const int64_t at = (int64_t)h * b.n_tokens * G + (int64_t)q0 * G + row;
  if constexpr (SPLIT) {
    float* pp = part + ((int64_t)sp * b.n_tokens * Hq + at) * (D + 4);
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
        *(f32x4*)(pp + 32 * d + 8 * r4 + 4 * lg) =
            f32x4{oacc[d][4 * r4], oacc[d][4 * r4 + 1], oacc[d][4 * r4 + 2], oacc[d][4 * r4 + 3]};
    if (lg == 0) *(f32x2*)(pp + D) = f32x2{m_run, l_tot};
    return;
  }
  const float inv = 1.0f / l_tot;
  bf16* op = O + ((int64_t)(q0 + tok) * Hq + hq) * D;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      bf16x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = f2bf(oacc[d][4 * r4 + e] * inv);
      *(bf16x4*)(op + 32 * d + 8 * r4 + 4 * lg) = o;
    }
  if (lse && lg == 0) lse[at] = m_run + log2f(l_tot);
}

// Merge of the key-range splits: a workgroup per token and KV head, D / 4 threads per
// query head, folded in split order.
template <int D>
__global__ __launch_bounds__(256) void attn_kv8_fold_kernel(BatchDev b, Kv8Dev c, int Hq, int Hkv,
                                                            const float* __restrict__ part,
                                                            bf16* __restrict__ O,
                                                            float* __restrict__ lse, int nsplit,
                                                            int least) {
  constexpr int TPR = D / 4;
  const int t = blockIdx.x, h = blockIdx.y, G = Hq / Hkv, lane = threadIdx.x & 63;
  // the token's sequence: as many ends lie at or before it
  int s = 0;
  for (int j0 = 0; j0 < b.n_seqs; j0 += 64) {
    const int end = b.cu_q[min(j0 + lane, b.n_seqs - 1) + 1];
    s += __builtin_popcountll(__builtin_amdgcn_ballot_w64(j0 + lane < b.n_seqs && end <= t));
  }
  int q0, n, ctx, sl;
  if (s >= b.n_seqs || !kv8_seq(b, c, s, q0, n, ctx, sl) || n < least || t < q0 || t >= q0 + n) return;
  const int64_t plane = (int64_t)b.n_tokens * Hq * (D + 4);
  const int d = 4 * ((int)threadIdx.x % TPR);
  for (int g = (int)threadIdx.x / TPR; g < G; g += 256 / TPR) {
    const int row = (t - q0) * G + g;
    const int last = min(n * G, (row / kRows8 + 1) * kRows8) - 1;  // of the flash kernel's tile
    const int nkt = cdiv(ctx + last / G + 1, kKeys8), ns = cdiv(nkt, cdiv(nkt, nsplit));
    const int64_t at = (int64_t)h * b.n_tokens * G + (int64_t)q0 * G + row;
    const float* pp = part + at * (D + 4);
    float M = -INFINITY, L = 0.f;
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int j0 = 0; j0 < ns; j0 += 4) {
      f32x2 ml[4];
      f32x4 a[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {  // (splits past the last are loaded again and dropped)
        const float* pj = pp + min(j0 + j, ns - 1) * plane;
        ml[j] = *(const f32x2*)(pj + D);
        a[j] = *(const f32x4*)(pj + d);
      }
      const float Mn = fmaxf(max3f(M, ml[0][0], ml[1][0]), fmaxf(ml[2][0], ml[3][0]));
      const float at_max = Mn == -INFINITY ? 0.f : Mn;  // (no key visible so far: all 0)
      const float x = __builtin_amdgcn_exp2f(M - at_max);
      M = Mn;
      L *= x;
      o *= x;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (j0 + j >= ns) continue;
        const float w = __builtin_amdgcn_exp2f(ml[j][0] - at_max);
        L = fmaf(ml[j][1], w, L);
        o += a[j] * w;
      }
    }
    bf16x4 o4;
#pragma unroll
    for (int e = 0; e < 4; ++e) o4[e] = f2bf(o[e] / L);
    *(bf16x4*)(O + ((int64_t)t * Hq + h * G + g) * D + d) = o4;
    if (lse && d == 0) lse[at] = M + log2f(L);
  }
}

// mass[key] += sum over the packed rows of 2^(score - lse): the scores once more, keys and
// rows the other way round.  A workgroup of eight waves has KG groups of 32 cache rows, their
// codes in registers as bf16 (exact too, and q needs no conversion); query rows come 32 RG =
// 256 / KG at a time through LDS by direct loads, 32 to each of a group's RG waves, so that a
// SIMD's two waves cover each other's waits.  Every sum has one order.  Fewer groups make
// more workgroups of fewer steps that read the queries more often: KG = 4 where that fills
// two thirds of the CUs, 2 down to a third, else 1 (whole calls with 4, 2 and 1: 4 chunks of
// 300 to 900 tokens, 2 KV heads of 64, 66 workgroups at 4: 88, 63, 52 us; 200 tokens at 2000
// beside single ones, 4 heads of 128, 144: 62, 55, 62; 8 x 1024, 256: 165, 195, 266).
//
// Workgroups: a grid of every sequence's most pieces, or, where that is more than 16 per CU,
// four per CU that go through the pieces there are (LIST): most of a large grid has no keys,
// and passes through the CUs that the others leave (512 tokens at 6144 beside 32 single ones:
// 138 us and 137, beside 128: 218 and 202; 256 at 1000 beside 256: 146 and 127; a grid of 9
// per CU: 54 and 55).
template <int D, bool FP8, int KG, bool LIST>
__global__ __launch_bounds__(512, 2) void attn_kv8_mass_kernel(BatchDev b, Kv8Dev c, int q_heads, int kv_heads,
                                                               const bf16* __restrict__ Q, int64_t q_stride,
                                                               const float* __restrict__ lse,
                                                               int least, float scale_log2e) {
  constexpr int DS = D / 16, DC = D / 8;
  constexpr int RPB = 64 / DC;             // rows of a 1 KB load
  constexpr int RG = 8 / KG, kMassKeys = 32 * KG, kMassQ = 32 * RG;
  constexpr int NL = kMassQ / RPB / 8;     // such loads of a wave and tile
  __shared__ __align__(16) bf16 sq0[kMassQ * D], sq1[kMassQ * D];
  __shared__ float sums[RG][KG][32];
  int item = blockIdx.x;
  do {
    // (formed anew for every item: what depends on these is not kept across items in registers)
    int Hq = q_heads, Hkv = kv_heads, tid = threadIdx.x;
    int64_t qs = q_stride;
    if constexpr (LIST) asm volatile("" : "+s"(Hq), "+s"(Hkv), "+s"(qs), "+v"(tid));
    int h, s, piece, q0, n, ctx, sl;
    if constexpr (LIST) {
      int pieces;
      h = item % Hkv;
      if (!kv8_piece(b, c, least, item / Hkv,
                     [&](int tokens, int held) { return cdiv(held + tokens, kMassKeys); }, s, piece, pieces, q0,
                     n, ctx, sl))
        return;
    } else {
      s = blockIdx.z, h = blockIdx.y, piece = blockIdx.x;
      if (!kv8_seq(b, c, s, q0, n, ctx, sl) || n < least || piece * kMassKeys >= ctx + n) return;
    }
    const int key0 = piece * kMassKeys;
    const int G = Hq / Hkv, rows = n * G;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lr = lane & 31, lg = lane >> 5;
    // codes of this wave's 32 keys: lane key lr, values 16 t + 8 lg ...
    const int kg = wave % KG, rg = wave / KG, wkey = key0 + 32 * kg;
    int prow = 0;
    const int panel = wkey < ctx + n ? kv_panel(c.kv, sl, wkey, prow) : -1;
    const int live = panel < 0 ? 0 : min(32, ctx + n - wkey);
    float kf = 0.f;
    bf16x8 kreg[DS];
    {
      const int64_t head = (int64_t)max(panel, 0) * Hkv + h;
      if (live > 0) kf = c.k_scale[head * c.scales_per_panel() + (prow >> c.scale_shift)] * scale_log2e;
      const auto rk = __builtin_amdgcn_make_buffer_rsrc(
          (void*)(c.k + (head * c.kv.panel_rows() + prow) * D), (short)0, live * D, 0x00020000);
#pragma unroll
      for (int t = 0; t < DS; ++t) {
        const auto w = __builtin_amdgcn_raw_buffer_load_b64(rk, lr * D + 16 * t + 8 * lg, 0, 0);
        const f32x4 lo = kv8_decode4<FP8>(w[0]), hi = kv8_decode4<FP8>(w[1]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          kreg[t][e] = f2bf(lo[e]);
          kreg[t][4 + e] = f2bf(hi[e]);
        }
      }
    }
    // (for the end, in vector registers)
    int64_t mass_at = kv8_row_at(c, Hkv, max(panel, 0), h, prow);
    int key_v = wkey, live_v = live, rg_v = rg, kg_v = kg, ctx_v = ctx, rows_v = rows;
    if constexpr (LIST) asm volatile("" : "+v"(mass_at), "+v"(key_v), "+v"(live_v), "+v"(rg_v), "+v"(kg_v), "+v"(ctx_v), "+v"(rows_v));
    // Row tiles from the first that sees key0.  A tile's first row is head `rem0` of token tok0;
    // both go on by a tile's rows, and a row's place in the tile takes one comparison.
    const int rt_lo = max(0, key0 - ctx) * G / kMassQ, rt_hi = cdiv(rows, kMassQ);
    const int tok_step = kMassQ / G, rem_step = kMassQ - tok_step * G;
    int tok0 = rt_lo * kMassQ / G, rem0 = rt_lo * kMassQ - tok0 * G;  // of the tile loaded next
    int head_of[NL];
    uint32_t place[NL];
#pragma unroll
    for (int j = 0; j < NL; ++j) {
      const int r = (wave + 8 * j) * RPB + lane / DC, t = r / G;
      head_of[j] = r - t * G;
      place[j] = (uint32_t)(t * (int)qs + head_of[j] * D + kv_chunk<D>(lane % DC, r) * 8) * 2;
    }
    auto gload = [&](auto buf) {
      bf16* dst = decltype(buf)::value ? sq1 : sq0;
      // (rows past the last read as zero)
      const int64_t bytes = ((int64_t)(n - 1 - tok0) * qs + G * D) * 2;
      const auto rq = __builtin_amdgcn_make_buffer_rsrc((void*)(Q + (int64_t)(q0 + tok0) * qs + (int64_t)h * G * D),
                                                        (short)0, (int)min(bytes, (int64_t)0x7fffffff), 0x00020000);
#pragma unroll
      for (int j = 0; j < NL; ++j) {
        const uint32_t off = place[j] + rem0 * D * 2 + (head_of[j] + rem0 >= G ? (uint32_t)((int)qs - G * D) * 2 : 0u);
        buffer_load_lds16(rq, dst + (wave + 8 * j) * 512, off, 0);
      }
      tok0 += tok_step;
      rem0 += rem_step;
      if (rem0 >= G) {
        rem0 -= G;
        ++tok0;
      }
    };
    float acc[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.f;
    const float* lp = lse + (int64_t)h * b.n_tokens * G + (int64_t)q0 * G;
    if constexpr (LIST) asm volatile("" : "+v"(lp));
    auto lse_of = [&](int rt) {
      const int row = rt * kMassQ + 32 * rg_v + lr;
      return row < rows_v ? lp[row] : INFINITY;
    };
    // Both matrix product and exponentials take most of a step: those of the tile before run
    // under the product of this one.  (rows past the end: 2^-inf)
    float off_next = lse_of(rt_lo), off_old = INFINITY;
    f32x16 old = f32x16{0.f};
    auto weigh = [&](auto e_) {
      constexpr int e = decltype(e_)::value;
      acc[e] += __builtin_amdgcn_exp2f(fmaf(old[e], kf, -off_old));
    };
    int tok_of = tok0;  // first token of the tile at work
    gload(Int<0>{});
    auto step = [&](int rt, auto buf) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      float off = off_next;
      const int first = tok_of;
      tok_of = tok0;
      if (rt + 1 < rt_hi) {
        off_next = lse_of(rt + 1);  // (before the rows: loads come back in order)
        gload(Int<1 - decltype(buf)::value>{});
      }
      const bf16* qb = decltype(buf)::value ? sq1 : sq0;
      const int r = 32 * rg_v + lr;
      constexpr int LA = 3;
      bf16x8 qf[LA + 1];
      auto qread = [&](int t) { return *(const bf16x8*)&qb[r * D + kv_chunk<D>(2 * t + lg, r) * 8]; };
#pragma unroll
      for (int t = 0; t < LA; ++t) qf[t] = qread(t);
      f32x16 sc = f32x16{0.f};
      each<DS>([&](auto t_) {
        constexpr int t = decltype(t_)::value, PER = 16 / DS;
        if constexpr (t + LA < DS) qf[(t + LA) % (LA + 1)] = qread(t + LA);
        sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kreg[t], qf[t % (LA + 1)], sc, 0, 0, 0);
        each<PER>([&](auto j) { weigh(Int<t * PER + decltype(j)::value>{}); });
        __builtin_amdgcn_sched_barrier(0);
      });
      if (key_v + 31 > ctx_v + first) {  // some row may not see some key
        const int qpos = ctx_v + min(rt * kMassQ + r, rows_v - 1) / G;
        // (a row without finite weights, lse NaN or -inf: NaN to what it sees, 0 to the rest)
        const bool bad = !(off > -INFINITY);
        off = bad ? 0.f : off;
#pragma unroll
        for (int e = 0; e < 16; ++e)
          sc[e] = key_v + (e & 3) + 8 * (e >> 2) + 4 * lg > qpos ? -INFINITY : (bad ? __builtin_nanf("") : sc[e]);
      }
      old = sc;
      off_old = off;
    };
    for (int rt = rt_lo; rt < rt_hi; rt += 2) {
      step(rt, Int<0>{});
      if (rt + 1 < rt_hi) step(rt + 1, Int<1>{});
    }
    each<16>(weigh);
    // the group's waves: their sums through LDS, added in order
    float* mp = c.mass + mass_at;
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = group_sum(acc[e], 32);
    if (lr == 0) {
#pragma unroll
      for (int e = 0; e < 16; ++e) sums[rg_v][kg_v][(e & 3) + 8 * (e >> 2) + 4 * lg] = acc[e];
    }
    __syncthreads();
    if (rg_v == 0 && lane < live_v) {
      float sum = 0.f;
#pragma unroll
      for (int r = 0; r < RG; ++r) sum += sums[r][kg_v][lane];
      mp[lane] += sum;
    }
    item += gridDim.x;
  } while (LIST);
}

// Key-range splits: doubled while the workgroups fit one to a CU and a split keeps 4 tiles of
// the longest range, or two to a CU and it keeps 8.  (512 tokens at 6144 beside 32 single
// ones, 28/4 heads of 128, 112 workgroups unsplit: 148 us with two splits, 141 with four, 176
// with eight; 40 tokens at 6000, 12: 35 us with eight, 31 with sixteen, 34 with 32; 500 at 1000
// beside single ones, 14/2 heads of 64, 60: 28 us with two, 24 with four, 28 with eight.)
static int kv8_key_splits(const BatchDev& b, int n_q_heads, int n_kv_heads) {
  const int64_t wgs = (int64_t)cdiv(b.n_tokens * (n_q_heads / n_kv_heads), kRows8) * n_kv_heads;
  const int tiles = cdiv(b.max_ctx_len + b.max_q_len, kKeys8), cus = cu_count();
  int sp = 1;
  while (sp < kMaxSplitF8 && ((wgs * sp * 2 <= cus && tiles >= 8 * sp) ||
                              (wgs * sp * 2 <= 2 * cus && tiles >= 16 * sp)))
    sp *= 2;
  return sp;
}

constexpr int64_t kForkBytes = (int64_t)192 << 20;  // codes that single tokens may read, for a side stream

static size_t round256(size_t v) { return (v + 255) / 256 * 256; }

// Workspace: log-sum-exps of the packed rows (with mass), the splits' partials, the
// single tokens' part.
static size_t lse_bytes(const BatchDev& b, const Kv8Dev& c, int n_q_heads) {
  return c.mass && b.max_q_len > 1 ? round256((size_t)b.n_tokens * n_q_heads * 4) : 0;
}
// (a bound that never falls as tokens are added: splits > 1 are at most two workgroups' rows
// per CU)
static size_t part8_bytes(const BatchDev& b, int n_q_heads, int n_kv_heads, int head_dim) {
  if (b.max_q_len < 2) return 0;
  const int64_t rows = std::min<int64_t>((int64_t)kMaxSplitF8 * b.n_tokens * n_q_heads,
                                         (int64_t)cu_count() * 2 * kRows8);
  return round256((size_t)rows * (head_dim + 4) * 4);
}
size_t attn_kv8_workspace_bytes(const BatchDev& b, const Kv8Dev& c, int n_q_heads, int n_kv_heads,
                                int head_dim) {
  return lse_bytes(b, c, n_q_heads) + part8_bytes(b, n_q_heads, n_kv_heads, head_dim) +
         attn_kv8_decode_bytes(b, c, n_q_heads, n_kv_heads, head_dim);
}

template <int D, bool FP8>
static hipError_t run_flash8(const BatchDev& b, const Kv8Dev& c, int Hq, int Hkv, const void* q,
                             int64_t qs, void* out, char* ws, int least, hipStream_t s) {
  const int sp = kv8_key_splits(b, Hq, Hkv), G = Hq / Hkv;
  float* lse = c.mass ? (float*)ws : nullptr;
  float* part = (float*)(ws + lse_bytes(b, c, Hq));
  const float scale_log2e = (float)(1.4426950408889634 / __builtin_sqrt((double)D));
  // row tiles: at most one of a sequence's is in part empty
  const int64_t chunks = std::min(b.n_seqs, b.n_tokens / least);
  const int64_t tiles = std::min(chunks * cdiv(b.max_q_len * G, kRows8),
                                 ((int64_t)b.n_tokens * G + chunks * (kRows8 - 1)) / kRows8);
  const int64_t wgs = (least == 1 ? (int64_t)b.n_seqs * cdiv(b.max_q_len * G, kRows8) : tiles) * Hkv * sp;
  if (wgs > 0x7fffffff) return hipErrorInvalidConfiguration;
  auto go = [&](auto kernel) {
    kernel<<<(unsigned)wgs, 256, 0, s>>>(b, c, Hq, Hkv, (const bf16*)q, qs, (bf16*)out, lse, part, sp,
                                         least, scale_log2e);
    return hipGetLastError();
  };
  hipError_t e;
  if (sp > 1) e = c.kv.table ? go(attn_kv8_kernel<D, FP8, true, true>) : go(attn_kv8_kernel<D, FP8, false, true>);
  else e = c.kv.table ? go(attn_kv8_kernel<D, FP8, true, false>) : go(attn_kv8_kernel<D, FP8, false, false>);
  if (e != hipSuccess) return e;
  if (sp > 1) {
    attn_kv8_fold_kernel<D><<<dim3(b.n_tokens, Hkv), 256, 0, s>>>(
        b, c, Hq, Hkv, part, (bf16*)out, lse, sp, least);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (c.mass) {
    // (as many chunks as the longest would make of the tokens)
    const int64_t wgs4 = (int64_t)cdiv(b.max_ctx_len + b.max_q_len, 128) * Hkv * cdiv(b.n_tokens, b.max_q_len);
    auto weigh = [&](auto kg, auto direct, auto listed) {
      const int rows = b.max_ctx_len + b.max_q_len, pieces = cdiv(rows, 32 * decltype(kg)::value);
      const int wgs = 4 * cu_count();
      if ((int64_t)pieces * Hkv * b.n_seqs > 4 * wgs)
        listed<<<wgs, 512, 0, s>>>(b, c, Hq, Hkv, (const bf16*)q, qs, lse, least, scale_log2e);
      else
        direct<<<dim3(pieces, Hkv, b.n_seqs), 512, 0, s>>>(b, c, Hq, Hkv, (const bf16*)q, qs, lse, least,
                                                           scale_log2e);
      return hipGetLastError();
    };
    const auto two = attn_kv8_mass_kernel<D, FP8, 2, true>;
    if (wgs4 * 3 >= 2 * cu_count())
      e = weigh(Int<4>{}, attn_kv8_mass_kernel<D, FP8, 4, false>, attn_kv8_mass_kernel<D, FP8, 4, true>);
    else if (wgs4 * 3 >= cu_count())
      e = weigh(Int<2>{}, attn_kv8_mass_kernel<D, FP8, 2, false>, two);
    else  // (one group of a listed workgroup would spill scalar registers)
      e = weigh(Int<1>{}, attn_kv8_mass_kernel<D, FP8, 1, false>, two);
  }
  return e;
}

hipError_t launch_attn_kv8(const BatchDev& b, const Kv8Dev& c, bool fp8, int n_q_heads,
                           int n_kv_heads, int head_dim, const void* q, int64_t q_stride, void* out,
                           void* ws, hipStream_t s) {
  if (b.n_seqs == 0 || b.n_tokens == 0) return hipSuccess;
  char* w = (char*)ws;
  float* own = (float*)(w + lse_bytes(b, c, n_q_heads) + part8_bytes(b, n_q_heads, n_kv_heads, head_dim));
  auto singles = [&](hipStream_t st) {
    return launch_attn_kv8_decode(b, c, fp8, n_q_heads, n_kv_heads, head_dim, q, q_stride, out, own, st);
  };
  if (b.max_q_len == 1) return singles(s);
  // Single tokens beside chunks, memory-bound beside compute-bound: on the side stream where
  // their stream is long enough (other output rows, other weights' rows, another part of the
  // workspace).  Fork and join cost about 20 us, so it pays from some 40 us of streaming:
  // 33 sequences up to 8192 rows (277 MB at most) take 139 us so and 171 in turn, up to 4000
  // rows (135 MB) 70 and 76 (on an idle GPU 98 and 91), 9 up to 600 47 and 25.
  // Chunks that fill n_tokens at max_q_len each leave no single token, unless some of the
  // tokens belong to no sequence: then one is a chunk of one.
  const int least = (int64_t)b.n_seqs * b.max_q_len == b.n_tokens ? 1 : 2;
  Fork fork;
  hipError_t e = hipSuccess;
  if (least == 2) {
    const int64_t bytes = (int64_t)b.n_seqs * (b.max_ctx_len + 1) * n_kv_heads * head_dim * 2;
    if (bytes >= kForkBytes) e = fork.begin(s);
    if (e == hipSuccess) e = singles(fork.stream ? fork.stream : s);
  }
  if (e == hipSuccess) {
    if (head_dim == 128)
      e = fp8 ? run_flash8<128, true>(b, c, n_q_heads, n_kv_heads, q, q_stride, out, w, least, s)
              : run_flash8<128, false>(b, c, n_q_heads, n_kv_heads, q, q_stride, out, w, least, s);
    else
      e = fp8 ? run_flash8<64, true>(b, c, n_q_heads, n_kv_heads, q, q_stride, out, w, least, s)
              : run_flash8<64, false>(b, c, n_q_heads, n_kv_heads, q, q_stride, out, w, least, s);
  }
  const hipError_t j = fork.end();
  return e != hipSuccess ? e : j;
}

}  // namespace tri
