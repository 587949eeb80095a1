// Windowed attention on an 8-bit K/V cache with block scales, bf16 queries, for any plan: the walk of the fp32 kernel
// over the plan's steps (32 keys x 16 queries, lane masks) with K and V rows gathered as codes.
//
// One workgroup = W waves = one query patch of one (batch, head); wave w takes the patch's steps w, w + W, ... and the
// partial results are merged through LDS.  Codes are whole numbers of 7 bits, which bf16 holds exactly, so the products
// run on them and the scales come afterwards in fp32:
//   S^T = Kc Q^T    (v_mfma_f32_16x16x32_bf16) the order of the head dimensions is free: lane (n, g4) takes the dimensions
//                   16 g4 .. + 15, one 16-byte load of key n's row; it receives the scores of query n with the keys
//                   16 t + 4 g4 + i, which are multiplied with their keys' scales;
//   O^T += Vc^T P^T the B operand is the lane's own probabilities times their keys' V scales, rounded to bf16 (one
//                   rounding; the row sum is of the probabilities in fp32); row n of dimension tile dt is dimension
//                   4 n + dt, so that the 4 x 4 bytes that a lane needs of four keys are four words, sixteen lanes to a row.
// Nothing of K or V is shared between waves or goes through LDS; the step's 32 pairs of scales do (a lane looks up one
// key, every lane reads the eight it owns).  Scales that are not finite reach the queries that keep their keys only:
// nothing is multiplied with a scale where the probability is zero.
//
// Bound: start-up (descriptor, tokens, rows, products one behind the other).  16 queries, 480 pairs 5.2 us in a graph; 25 queries
// 7.2 with one wave per patch, about 10 with four.  Every patch gathers and converts for itself: 36 / 64 queries 8.9 / 12.9 us, 5.8 / 7.9 in
// bf16 with keys shared through LDS.  Not for longer steps: 256 queries on 680 keys 80 us, 30 shared.
#include "attn_bf16_common.h"

namespace lv {

namespace {

// Four codes of a word as floats, exactly.
__device__ inline void unpack4(unsigned w, float (&x)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = (float)((int)(w << (24 - 8 * e)) >> 24);
}
}  // namespace

template <int W>
__global__ __launch_bounds__(W * 64) void k_attn_kv8(AttnArgs a, KV8Scales ks, int n_waves, float c) {
  int me, bh, wv, b, h;
  if (!xcd_item(a, n_waves, me, bh, wv)) return;
  divmod_by((uint32_t)bh, (uint32_t)a.H, a.H_magic, b, h);
  const int head_group = a.head_map ? ((const_i32_ptr)a.head_map)[h] : 0;   // (in the header's round trip)
  if (!plan_usable(a.hdr)) return;
  const const_u64_ptr wp = (const_u64_ptr)(a.waves + (wv + head_group * n_waves));
  uint64_t w0 = wp[0], w1 = wp[1], w2 = wp[2], w3 = wp[3];
  asm volatile("" : "+s"(w0), "+s"(w1), "+s"(w2), "+s"(w3));
  const uint64_t words[4] = {w0, w1, w2, w3};
  const WaveDesc wd = __builtin_bit_cast(WaveDesc, words);
  if (wd.ny == 0) return;
  const bool shared = a.cfg_share && a.cfg_share[h * a.n_scales + wd.kq];
  if (shared && b >= a.B / 2) return;

  __shared__ __align__(16) float2 step_scales[W][32];
  const int lane = threadIdx.x & 63, n = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int qrow = ((wd.valid >> n) & 1u) ? checked_index(a.hdr, wd.q_base + (n >> 2) * wd.sk + (n & 3), a.q_len) : -1;

  const int8_t* Kp = (const int8_t*)a.k + (int64_t)bh * a.kv_len * 64;
  const int8_t* Vp = (const int8_t*)a.v + (int64_t)bh * a.kv_len * 64;
  const float* Ks = ks.k + (int64_t)bh * ks.n_blocks;
  const float* Vs = ks.v + (int64_t)bh * ks.n_blocks;

  const int64_t S0 = wd.step_begin;
  const int n_steps = wd.n_steps;
  // the tokens of key `lane % 32`, of this lane's K rows (keys n and 16 + n) and V rows (keys 16 t + 4 g4 + i) of a step
  struct Tokens { int own, k[2]; int4 v[2]; };
  auto load_tokens = [&](int s) {
    const int32_t* t = a.step_tok + (S0 + min(s, n_steps - 1)) * kStepKeys;
    return Tokens{t[lane & 31], {t[n], t[16 + n]}, {*(const int4*)(t + 4 * g4), *(const int4*)(t + 16 + 4 * g4)}};
  };
  Tokens tok = load_tokens(wave);
  __builtin_amdgcn_sched_barrier(0);         // (the queries behind the tokens, for which the rows wait)
  bf16x8 qv[2];
  {
    const __bf16* Q = (const __bf16*)a.q + b * a.qs[0] + h * a.qs[1] + max(qrow, 0) * a.qs[2] + 16 * g4;
#pragma unroll
    for (int j = 0; j < 2; ++j) qv[j] = as_bf16x8(*(const uint4*)(Q + 8 * j));
  }
  f32x4 O[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) O[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;          // softmax reference of query n (the same in its four lanes), this lane's row sum

  // the rows of a step: scales of key `lane % 32`, codes of the keys above
  struct Rows { float2 sc; u32x4 kc[2]; unsigned vc[2][4]; };
  auto load_rows = [&](const Tokens& tok) {
    // (padding keys carry token -1; they read the row of the step's first key, which every step has)
    const int first = __builtin_amdgcn_readfirstlane(tok.own);
    auto row = [&](int t) -> int { return checked_index(a.hdr, t < 0 ? first : t, a.kv_len); };
    const int own = row(tok.own);
    int shift = 0;                           // 64 x block = token + shift, rounded down
    for (int j = 1; j <= wd.kq; ++j) shift = own >= ks.off[j] ? ks.shift[j] : shift;
    const int block = (own + shift) >> 6;
    Rows r;
    r.sc = make_float2(Ks[block], Vs[block]);
#pragma unroll
    for (int t = 0; t < 2; ++t) r.kc[t] = *(const u32x4*)(Kp + (int64_t)row(tok.k[t]) * 64 + 16 * g4);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int vt[4] = {tok.v[t].x, tok.v[t].y, tok.v[t].z, tok.v[t].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) r.vc[t][i] = *(const unsigned*)(Vp + (int64_t)row(vt[i]) * 64 + 4 * n);
    }
    return r;
  };
  auto absorb = [&](const Rows& r, int s) {
    const const_u64_ptr mk = (const_u64_ptr)(a.step_mask + (S0 + s) * 8);
    uint64_t keep[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) keep[e] = mk[e];
    if (lane < 32) step_scales[wave][lane] = make_float2(nan_unless_finite(r.sc.x), r.sc.y);
    asm volatile("" ::: "memory");           // (read by other lanes of the wave; LDS keeps a wave's order)

    f32x4 S[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      S[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_bf16(r.kc[t][0], r.kc[t][1]), qv[0], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
      S[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_bf16(r.kc[t][2], r.kc[t][3]), qv[1], S[t], 0, 0, 0);
    }
    float z[8], vs[8], mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float2 f = step_scales[wave][16 * (e >> 2) + 4 * g4 + (e & 3)];
      vs[e] = f.y;
      z[e] = mask_select(S[e >> 2][e & 3] * f.x, keep[e]);
      mx = fmaxf(mx, z[e]);
    }
    asm volatile("" ::: "memory");
    const float m_new = fmaxf(m, max_across_rows(mx));
    if (__builtin_amdgcn_ballot_w64(m_new > m) != 0) {
      const float alpha = m > -INFINITY ? __builtin_amdgcn_exp2f((m - m_new) * c) : 1.f;
      l *= alpha;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) O[dt] *= alpha;
      m = m_new;
    }
    const float ref = m > -INFINITY ? m : 0.f;           // (a query without a kept key so far: exp2(-inf) below)
    bf16x8 pb;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float p = __builtin_amdgcn_exp2f((z[e] - ref) * c);
      l += p;
      pb[e] = (__bf16)(p > 0.f ? p * vs[e] : 0.f);
    }
    float v[8][4];
#pragma unroll
    for (int e = 0; e < 8; ++e) unpack4(r.vc[e >> 2][e & 3], v[e]);
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) {
      bf16x8 vb;
#pragma unroll
      for (int e = 0; e < 8; ++e) vb[e] = (__bf16)v[e][dt];
      O[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb, pb, O[dt], 0, 0, 0);
    }
  };
  // A step's rows are requested ahead of the work on the step before it, their tokens one step earlier (64 queries, 480 pairs, five
  // steps to a patch 14.7 -> 14.1 us, 64 queries, 120 pairs 7.7 -> 7.1)
  if (wave < n_steps) {
    Rows even = load_rows(tok), odd;
    tok = load_tokens(wave + W);
    for (int s = wave;; s += 2 * W) {
      if (s + W >= n_steps) { absorb(even, s); break; }
      odd = load_rows(tok);
      tok = load_tokens(s + 2 * W);
      absorb(even, s);
      if (s + 2 * W >= n_steps) { absorb(odd, s + W); break; }
      even = load_rows(tok);
      tok = load_tokens(s + 3 * W);
      absorb(odd, s + W);
    }
  }

  // ---- O[dt][i]: dimension 16 g4 + 4 i + dt of query n.  Merged from the waves (wave w forms i = w), or its own ----
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  constexpr int kPieces = 4 / W;
  f32x4 acc[kPieces];
  float sum = 0.f;
  if constexpr (W > 1) {
    __shared__ __align__(16) f32x4 part_o[W][4][64];
    __shared__ float part_m[W][16], part_l[W][16];
#pragma unroll
    for (int i = 0; i < 4; ++i) part_o[wave][i][lane] = f32x4{O[0][i], O[1][i], O[2][i], O[3][i]};
    if (g4 == 0) { part_m[wave][n] = m; part_l[wave][n] = l; }
    __syncthreads();
    float m_all = part_m[0][n];
#pragma unroll
    for (int w = 1; w < W; ++w) m_all = fmaxf(m_all, part_m[w][n]);
#pragma unroll
    for (int p = 0; p < kPieces; ++p) acc[p] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = part_m[w][n] > -INFINITY ? __builtin_amdgcn_exp2f((part_m[w][n] - m_all) * c) : 0.f;
      sum = fmaf(part_l[w][n], f, sum);
#pragma unroll
      for (int p = 0; p < kPieces; ++p) acc[p] += part_o[w][kPieces * wave + p][lane] * f;
    }
  } else {
    sum = l;
#pragma unroll
    for (int p = 0; p < kPieces; ++p) acc[p] = f32x4{O[0][p], O[1][p], O[2][p], O[3][p]};
  }
  const float inv = 1.f / sum;
  float largest = 0.f;                         // magnitude of the row's results that this wave stores
#pragma unroll
  for (int p = 0; p < kPieces; ++p)
#pragma unroll
    for (int e = 0; e < 4; ++e) { acc[p][e] *= inv; largest = fmaxf(largest, fabsf(acc[p][e])); }
  if (qrow >= 0) {
    __bf16* o = (__bf16*)a.o + b * a.os[0] + h * a.os[1] + qrow * a.os[2] + 16 * g4 + 4 * kPieces * wave;
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      bf16x4 r;
#pragma unroll
      for (int e = 0; e < 4; ++e) r[e] = (__bf16)acc[p][e];
      *(bf16x4*)(o + 4 * p) = r;
      if (shared) *(bf16x4*)(o + 4 * p + (a.B / 2) * a.os[0]) = r;
    }
  }
  // Rows of very small values are formed again in fp32: products of weights and V scales below 2^-126 have lost bits as bf16
  const bool small = qrow >= 0 && largest > 0.f && largest < 0x1p-100f;
  uint64_t again = __builtin_amdgcn_ballot_w64(small);
  if (__builtin_expect(again != 0, 0)) {
    again = (again | (again >> 16) | (again >> 32) | (again >> 48)) & 0xffffull;
    for (; again != 0; again &= again - 1) {
      wait_vmcnt<0>();                         // (what is stored next goes to places that were just stored to)
      const int at = __builtin_ctzll(again), l0 = lane_of_wave();
      attend_row<false, true>(a, c, b, h, __builtin_amdgcn_readlane(qrow, at), shared, W == 1 || ((l0 >> 2) & 3) == wave,
                              PatchKeys{a, S0, n_steps, at}, ks);
    }
  }
}

litevar_status launch_attn_kv8(const litevar_plan* pl, const AttnArgs& args, const KV8Scales& scales, hipStream_t st) {
  AttnArgs a = args;
  // Four waves shorten the chain of a patch's steps; one wave per patch where patches have a single step, or where there are so
  // many that the chip is full of them.  (Patches, steps of one), us, one wave / four: (480, 1) 5.5 / 8.2; (480, 2) 6.1 / 5.8; (1920, 2)
  // 7.5 / 9.9; (1920, 5) 13.8 / 15.3; (1920, 7.5) 25.4 / 19.8; (4320, 5.9) 37.9 / 39.0; (27 360, 6.8) 147 / 195; two are nowhere better by
  // more than 8 %.
  const int64_t patches = (int64_t)pl->n_patches * pl->n_head_groups, all = (int64_t)a.B * a.H * pl->n_patches;
  const int W = pl->n_steps <= patches || all >= 4000 || (all >= 1500 && pl->n_steps <= 5 * patches) ? 1 : 4;
  const int64_t n_waves = (int64_t)pl->n_groups * pl->waves_per_group;
  const int64_t blocks = spread_over_xcds(a, n_waves, 64);
  if (blocks > 0x7fffffff) return fail(LITEVAR_E_UNSUPPORTED, "grid too large");
  const float c = a.sm_scale * 1.4426950408889634f;
  return launch_in_parts(blocks, W * 64, "8-bit cache attention launch", [&](int64_t first, unsigned n) {
    a.first_block = (uint32_t)first;
    if (W == 1) hipLaunchKernelGGL(k_attn_kv8<1>, dim3(n), dim3(64), 0, st, a, scales, (int)n_waves, c);
    else hipLaunchKernelGGL(k_attn_kv8<4>, dim3(n), dim3(256), 0, st, a, scales, (int)n_waves, c);
  });
}

}  // namespace lv
