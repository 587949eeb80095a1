// Cross attention for gfx950 (CDNA4): every query row sees the first len[b] of kv_len keys (an encoder's states),
//   O[b, h, i] = sum over t < len[b] of softmax_t(sm q_i . k_t) v_t,
// with K and V rows in bf16, in fp32, or as 8-bit codes with one scale per block of 64 tokens and kv head.  Query
// head h reads kv head h / (H / H_kv): the rows of one kv head are its G = H / H_kv query heads' rows, head after head.
//
// Two forms.  Few rows (k_cross_rows): one workgroup = four waves = 32 rows of one (batch, kv head) and one part of the
// key axis; the waves take the part's blocks of 64 keys (32 in fp32) in turn and join their results through LDS.  With
// several parts, each leaves its sums in the workspace and a second launch joins them (k_cross_join).  Many rows
// (k_cross_tiles, k_cross_tiles_f32): the waves of a workgroup have 32 rows each and share all keys, or those of a part of
// a long axis, through LDS.  shares_rows, shared_parts_of and parts_of choose, by measured cost.
//
// What a call cannot do without: Q, O and the valid keys' K and V once, 256 operations per row and key.  256 rows, 480 pairs of 77 to 512
// keys, bf16: 22.4 us for 73 MB (14.4 at the copy rate); 2240 rows, 32 pairs, fp32: 53 us for 4.2 GFLOP (27 at a large
// product's rate); four rows (one token, 4 query
// heads) on up to 30 011 keys in codes, 16 pairs: 17.5 us for 44 MB (8.7); 169 rows, 480 pairs of 51 to 333
// keys in codes: 17.7 us (7.0).
#include <algorithm>
#include <cmath>
#include <cstring>
#include <type_traits>

#include "attn_bf16_common.h"

namespace lv {
namespace {

constexpr int kRows = 32;                      // rows per workgroup: the columns of a 32 x 32 tile
constexpr int kWaves = 4;
constexpr int kBlock = LITEVAR_KV8_BLOCK;      // keys per turn
constexpr int kPitch = 68;                     // floats per row of the joining buffer
constexpr int kMaxParts = 512;                 // of the key axis

// An exponent that is added to a reference beyond this loses bits that show (codes: the V scales; see k_cross_tiles).
constexpr float kFarCodes = 0x1p12f;

enum Kind { kBf16 = 0, kF32 = 1, kCodes = 2 };

struct CrossArgs {
  const void* q; const void* k; const void* v; void* o;
  const float* k_scale; const float* v_scale;  // codes: [B][H_kv][blocks]
  int64_t qs[3], ks[3], os[3];                 // element strides of (B, head, token)
  const int32_t* len;                          // [B] or nullptr
  int B, H, Hkv, G, q_len, kv_len;
  int rows, tiles;                             // rows of a kv head, tiles of 32 of them
  int parts, shared_parts;                     // of the key axis; those of k_cross_tiles
  int scale_blocks;                            // of a (batch, kv head)
  float ks_least, ks_most;                     // K scales outside multiply the scores, not the softmax scale: see k_cross_tiles
  uint32_t q_magic, tiles_magic, hkv_magic, parts_magic, pairs_magic;   // see divmod_by
  uint32_t first_block, rows_magic;
  int groups, by_xcd, by_rank; uint32_t groups_magic;   // k_cross_tiles: workgroups of a pair, how they are laid out
  uint32_t prio_magic;                         // 2^18 / chunks of the longest axis, 0: no priorities
  float* part_o; float2* part_ml;              // [item][32][64] and [item][32] (largest score, sum), item = workgroup
};

struct Row { int h, i; };                      // query head, token

__device__ inline Row row_at(const CrossArgs& a, int j, int r) {
  int g, i;
  divmod_by((uint32_t)r, (uint32_t)a.q_len, a.q_magic, g, i);
  return Row{j * a.G + g, i};
}

__device__ inline int keys_of(const CrossArgs& a, int b) { return a.len ? min(max(a.len[b], 0), a.kv_len) : a.kv_len; }

// The batch row that is r-th in the order of lengths, longest first, and its number of keys: where workgroups follow others on
// a CU, those that run longest start first.  (By chunks of 64 keys, ties in the order of rows; every lane of a wave counts the rows
// ahead of its own.  288 pairs of 2240 rows on 149 to 512 keys: 86.0 -> 78.5 us in a graph.)
__device__ inline int batch_of_rank(const CrossArgs& a, int r, int& n_keys) {
  if (!a.by_rank) { n_keys = keys_of(a, r); return r; }
  const int lane = lane_of_wave(), keys = min(max(a.len[min(lane, a.B - 1)], 0), a.kv_len);
  const unsigned key = ((unsigned)keys + (kBlock - 1u)) / kBlock * 64u + (63u - (unsigned)lane);
  int rank = 0;
  for (int i = 0; i < a.B; ++i) rank += (unsigned)__builtin_amdgcn_readlane((int)key, i) > key;
  const int b = __builtin_ctzll(__builtin_amdgcn_ballot_w64(lane < a.B && rank == r));
  n_keys = __builtin_amdgcn_readlane(keys, b);
  return b;
}

// a value that is the same in all lanes, in a scalar register
__device__ inline float uniform(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }

// What a row without weights is multiplied with: zero where it has no key, NaN where all its scores are -inf in fp32.  (As
// bits, see not_finite.)
__device__ inline float without_weights(int n_keys) {
  unsigned u = n_keys > 0 ? 0x7fc00000u : 0u;
  asm volatile("" : "+v"(u));
  return __uint_as_float(u);
}

// log2 of a value >= 0 whatever its size (the instruction takes a subnormal value for 0)
__device__ inline float log2_of(float x) {
  return x < 0x1p-126f ? __builtin_amdgcn_logf(x * 0x1p24f) - 24.f : __builtin_amdgcn_logf(x);
}

// Writes eight output values of row r, dims 8 part .. + 7.
template <int KIND> __device__ inline void store_row(const CrossArgs& a, int b, int j, int r, int part, const float (&x)[8]) {
  const Row w = row_at(a, j, r);
  const int64_t at = b * a.os[0] + w.h * a.os[1] + w.i * a.os[2] + 8 * part;
  if constexpr (KIND == kF32) {
    float* p = (float*)a.o + at;
    *(float4*)p = make_float4(x[0], x[1], x[2], x[3]);
    *(float4*)(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    bf16x8 y;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = (__bf16)x[e];
    *(bf16x8*)((__bf16*)a.o + at) = y;
  }
}

// Joins `n` sums of 32 rows: sum s has its rows' (largest score, sum) at ml(s)[row] and its products at o(s)[row].
// Thread t forms dims 8 (t / 32) .. of row t % 32.  Returns the joined largest score and sum; x is not divided.
template <class Ml, class O>
__device__ inline float2 join(int n, float c, Ml ml, O o, float (&x)[8]) {
  float m = -INFINITY, l = 0.f;
  for (int s = 0; s < n; ++s) m = fmaxf(m, ml(s).x);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = 0.f;
  if (m == -INFINITY) return make_float2(m, 0.f);
  for (int s = 0; s < n; ++s) {
    const float2 p = ml(s);
    if (p.x == -INFINITY) continue;            // (no key: nothing was written)
    const float f = __builtin_amdgcn_exp2f((p.x - m) * c);
    l = fmaf(p.y, f, l);
    const float* y = o(s);
    const float4 lo = *(const float4*)y, hi = *(const float4*)(y + 4);
    x[0] = fmaf(lo.x, f, x[0]); x[1] = fmaf(lo.y, f, x[1]); x[2] = fmaf(lo.z, f, x[2]); x[3] = fmaf(lo.w, f, x[3]);
    x[4] = fmaf(hi.x, f, x[4]); x[5] = fmaf(hi.y, f, x[5]); x[6] = fmaf(hi.z, f, x[6]); x[7] = fmaf(hi.w, f, x[7]);
  }
  return make_float2(m, l);
}

}  // namespace

// S^T (32 keys x 32 rows) = K (A operand, straight from memory) . Q^T, so that a lane owns one row and 16 of 32 keys;
// O^T (64 dims x rows) += V^T . P^T.  The order of the head dimensions inside the first product is free: lane half hh
// takes dims 32 hh .. + 31, a lane's piece of a K row is then contiguous.  V^T is read from LDS by transposing reads
// (bf16, codes) or straight from memory (fp32, a value per lane).  Softmax with the running largest score as the reference,
// subtracted before the scale is applied, so that scores of any size keep their differences.
template <int KIND>
__global__ __launch_bounds__(kWaves * 64) __attribute__((amdgpu_waves_per_eu(KIND == kBf16 ? 4 : 3, KIND == kBf16 ? 4 : 3)))
void k_cross_rows(CrossArgs a, float c) {
  __shared__ __align__(16) unsigned char smem[kWaves * kRows * kPitch * 4 + kWaves * kRows * 8];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int n = lane & 31, hh = lane >> 5;
  int rest, tile, part, bj, b, j;
  const uint32_t item = a.first_block + blockIdx.x;
  divmod_by(item, (uint32_t)a.parts, a.parts_magic, rest, part);
  divmod_by((uint32_t)rest, (uint32_t)a.tiles, a.tiles_magic, bj, tile);
  divmod_by((uint32_t)bj, (uint32_t)a.Hkv, a.hkv_magic, b, j);
  const int n_keys = keys_of(a, b);
  const int row0 = tile * kRows;
  const int r = min(row0 + n, a.rows - 1);     // (a column without a row holds the last one; it is not stored)
  const Row qr = row_at(a, j, r);
  const int64_t q_at = b * a.qs[0] + qr.h * a.qs[1] + qr.i * a.qs[2] + 32 * hh, kv_at = b * a.ks[0] + j * a.ks[1];

  // this part's turns: blocks of kBlock keys
  const int blocks = (n_keys + kBlock - 1) / kBlock;
  const int begin = (int)((int64_t)blocks * part / a.parts), end = (int)((int64_t)blocks * (part + 1) / a.parts);

  float m = -INFINITY, L = 0.f;                // the row's reference; this lane's share of the sum
  f32x16 O[2] = {f32x16{}, f32x16{}};
  // scores of 32 keys -> probabilities, with the reference moved to their largest; returns what that multiplies sums by
  auto softmax = [&](f32x16& S, int key0) -> float {
    const int left = n_keys - key0 - 4 * hh;
    float mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      S[e] = 8 * (e >> 2) + (e & 3) < left ? S[e] : -INFINITY;
      mx = fmaxf(mx, S[e]);
    }
    mx = fmaxf(mx, other_half(mx));
    const float to = fmaxf(m, mx);
    float alpha = 1.f;
    if (__builtin_amdgcn_ballot_w64(to > m) != 0) {
      alpha = m > -INFINITY ? __builtin_amdgcn_exp2f((m - to) * c) : 1.f;
      m = to; L *= alpha;
#pragma unroll
      for (int e = 0; e < 16; ++e) { O[0][e] *= alpha; O[1][e] *= alpha; }
    }
    const float ref = m > -INFINITY ? m : 0.f;           // (only scores of -inf so far, or NaN, which stays)
#pragma unroll
    for (int e = 0; e < 16; ++e) S[e] = __builtin_amdgcn_exp2f((S[e] - ref) * c);
    return alpha;
  };

  if constexpr (KIND == kF32) {
    const float* q = (const float*)a.q + q_at;
    float qf[32];
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      const float4 x = *(const float4*)(q + 4 * t);
      qf[4 * t] = x.x; qf[4 * t + 1] = x.y; qf[4 * t + 2] = x.z; qf[4 * t + 3] = x.w;
    }
    const float* K = (const float*)a.k + kv_at + 32 * hh;
    const float* V = (const float*)a.v + kv_at + n;
    const int last = n_keys - 1, stop = min(n_keys, kBlock * end);
    // V of a step is requested ahead of its score products, K of the next step behind them: each has half a step (2048
    // cycles of the matrix pipe) to arrive.
    float kf[32];
    auto load_k = [&](int key0) {
      const float* kp = K + (int64_t)min(key0 + n, last) * a.ks[2];
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const float4 x = *(const float4*)(kp + 4 * t);
        kf[4 * t] = x.x; kf[4 * t + 1] = x.y; kf[4 * t + 2] = x.z; kf[4 * t + 3] = x.w;
      }
    };
    int key0 = kBlock * begin + 32 * wave;
    if (key0 < stop) load_k(key0);
    for (; key0 < stop; key0 += 32 * kWaves) {
      float vf[2][16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {           // (probability 0 where the key is clamped)
        const float* vp = V + (int64_t)min(key0 + 8 * (e >> 2) + 4 * hh + (e & 3), last) * a.ks[2];
        vf[0][e] = vp[0]; vf[1][e] = vp[32];
      }
      f32x16 S = f32x16{};
#pragma unroll
      for (int t = 0; t < 32; ++t) S = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[t], qf[t], S, 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      load_k(key0 + 32 * kWaves < stop ? key0 + 32 * kWaves : key0);
      __builtin_amdgcn_sched_barrier(0);
      softmax(S, key0);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        L += S[e];
        O[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf[0][e], S[e], O[0], 0, 0, 0);
        O[1] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf[1][e], S[e], O[1], 0, 0, 0);
      }
    }
  } else {
    constexpr bool CODES = KIND == kCodes;
    constexpr int kTurn = CODES ? 64 : 32;     // keys of a turn: 4 KiB of K and as much of V per wave
    constexpr int kPerBlock = kBlock / kTurn;
    const __bf16* q = (const __bf16*)a.q + q_at;
    bf16x8 qf[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) qf[t] = as_bf16x8(*(const uint4*)(q + 8 * t));
    unsigned char* const Vs = smem + wave * kTurn * kRow;          // this wave's V rows of a turn in bf16
    const int64_t scale_at = CODES ? (int64_t)bj * a.scale_blocks : 0;
    // A turn's K rows as the first product takes them, its V rows in coalesced pieces (a row behind the last key counts as the
    // last one, with probability 0), its scales.  The next turn's are requested before this one's are used.
    struct Turn { u32x4 k[4], v[4]; float ks, vs; };
    const int last = n_keys - 1, turns = min(end * kPerBlock, (n_keys + kTurn - 1) / kTurn);
    auto load = [&](int turn) -> Turn {
      Turn x;
      const int key0 = turn * kTurn;
      x.ks = x.vs = 1.f;
      if constexpr (CODES) {
        x.ks = a.k_scale[scale_at + turn]; x.vs = a.v_scale[scale_at + turn];
        const int8_t *K = (const int8_t*)a.k + kv_at + (int64_t)key0 * 64, *V = (const int8_t*)a.v + kv_at + (int64_t)key0 * 64;
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int i = 0; i < 2; ++i) x.k[2 * half + i] = *(const u32x4*)(K + min(32 * half + n, last - key0) * 64 + 32 * hh + 16 * i);
#pragma unroll
        for (int i = 0; i < 4; ++i) x.v[i] = *(const u32x4*)(V + min(16 * i + (lane >> 2), last - key0) * 64 + 16 * (lane & 3));
      } else {
        const __bf16* K = (const __bf16*)a.k + kv_at + (int64_t)min(key0 + n, last) * a.ks[2] + 32 * hh;
#pragma unroll
        for (int t = 0; t < 4; ++t) x.k[t] = *(const u32x4*)(K + 8 * t);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          x.v[i] = *(const u32x4*)((const __bf16*)a.v + kv_at + (int64_t)min(key0 + 8 * i + (lane >> 3), last) * a.ks[2] + 8 * (lane & 7));
      }
      return x;
    };
    int turn = begin * kPerBlock + wave;
    Turn next;
    if (turn < turns) next = load(turn);
    for (; turn < turns; turn += kWaves) {
      const Turn x = next;
      if (turn + kWaves < turns) next = load(turn + kWaves);
      if constexpr (CODES) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const unsigned row = 16u * i + ((unsigned)lane >> 2), p = 2u * ((unsigned)lane & 3u), sw = dense_swizzle(row);
          const unsigned w0 = x.v[i][0], w1 = x.v[i][1], w2 = x.v[i][2], w3 = x.v[i][3];
          *(bf16x8*)(Vs + row * kRow + ((p ^ sw) << 4)) = codes_to_bf16(w0, w1);
          *(bf16x8*)(Vs + row * kRow + (((p + 1u) ^ sw) << 4)) = codes_to_bf16(w2, w3);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const unsigned row = 8u * i + ((unsigned)lane >> 3);
          *(u32x4*)(Vs + row * kRow + ((((unsigned)lane & 7u) ^ dense_swizzle(row)) << 4)) = x.v[i];
        }
      }
      asm volatile("" ::: "memory");           // (the rows of V are read by other lanes than wrote them; LDS keeps a wave's order)
      [[maybe_unused]] const float ks = CODES ? nan_unless_finite(x.ks) : 1.f;
      f32x16 P[2];                             // codes: the turn's products with V, which the V scale multiplies
      if constexpr (CODES) { P[0] = f32x16{}; P[1] = f32x16{}; }
#pragma unroll
      for (int half = 0; half < kTurn / 32; ++half) {
        const int key0 = turn * kTurn + 32 * half;
        if (half > 0 && key0 > last) break;
        f32x16 S = f32x16{};
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          bf16x8 kf;
          if constexpr (CODES) {
            const unsigned lo = x.k[2 * half + (t >> 1)][2 * (t & 1)], hi = x.k[2 * half + (t >> 1)][2 * (t & 1) + 1];
            kf = codes_to_bf16(lo, hi);
          } else {
            kf = __builtin_bit_cast(bf16x8, x.k[t]);
          }
          S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[t], S, 0, 0, 0);
        }
        if constexpr (CODES) {
#pragma unroll
          for (int e = 0; e < 16; ++e) S[e] *= ks;
        }
        const float alpha = softmax(S, key0);
        if constexpr (CODES) {
          if (half > 0 && __builtin_amdgcn_ballot_w64(alpha != 1.f) != 0) {
#pragma unroll
            for (int e = 0; e < 16; ++e) { P[0][e] *= alpha; P[1][e] *= alpha; }
          }
        }
        bf16x8 pb[2];
        float sum = L;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
          for (int e = 0; e < 8; ++e) pb[t][e] = (__bf16)S[8 * t + e];
#pragma unroll
          for (int e = 0; e < 8; e += 2) sum = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{pb[t][e], pb[t][e + 1]}, kOnes, sum, false);
        }
        L = sum;
        f32x16 (&acc)[2] = CODES ? P : O;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int dt = 0; dt < 2; ++dt) {
            s16x8 v8;
#pragma unroll
            for (int jj = 0; jj < 2; ++jj) {
              const unsigned l16 = (unsigned)lane & 15u, row = 32u * half + 16u * t + 8u * jj + 4u * (unsigned)hh + (l16 >> 2);
              const unsigned piece = 4u * dt + 2u * (((unsigned)lane >> 4) & 1u) + ((l16 & 3u) >> 1);
              const s16x4 y = lds_read_tr16(Vs + row * kRow + ((piece ^ dense_swizzle(row)) << 4) + 8u * (l16 & 1u));
#pragma unroll
              for (int e = 0; e < 4; ++e) v8[4 * jj + e] = y[e];
            }
            acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v8), pb[t], acc[dt], 0, 0, 0);
          }
      }
      asm volatile("" ::: "memory");
      if constexpr (CODES) {
#pragma unroll
        for (int e = 0; e < 16; ++e) { O[0][e] = fmaf(P[0][e], x.vs, O[0][e]); O[1][e] = fmaf(P[1][e], x.vs, O[1][e]); }
      }
    }
  }

  // ---- join the waves ----
  L += other_half(L);
  if (not_finite(L)) m = 0.f;                  // (a NaN score enters no maximum: with m = -inf the row would count as one without keys)
  float2* const ML = (float2*)(smem + kWaves * kRows * kPitch * 4);
  __syncthreads();                             // (the rows of V are read)
  float* const mine = (float*)smem + (wave * kRows + n) * kPitch + 4 * hh;
#pragma unroll
  for (int dt = 0; dt < 2; ++dt)
#pragma unroll
    for (int t = 0; t < 4; ++t)
      *(float4*)(mine + 32 * dt + 8 * t) = make_float4(O[dt][4 * t], O[dt][4 * t + 1], O[dt][4 * t + 2], O[dt][4 * t + 3]);
  if (hh == 0) ML[wave * kRows + n] = make_float2(m, L);
  __syncthreads();
  const int row = tid & 31, dims = tid >> 5;
  float x[8];
  const float2 ml = join(kWaves, c, [&](int s) { return ML[s * kRows + row]; },
                         [&](int s) { return (const float*)smem + (s * kRows + row) * kPitch + 8 * dims; }, x);
  if (row0 + row >= a.rows) return;
  if (a.parts > 1) {
    if (dims == 0) a.part_ml[(int64_t)item * kRows + row] = ml;
    float* p = a.part_o + ((int64_t)item * kRows + row) * 64 + 8 * dims;
    *(float4*)p = make_float4(x[0], x[1], x[2], x[3]);
    *(float4*)(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
    return;
  }
  const float inv = ml.y > 0.f ? 1.f / ml.y : without_weights(n_keys);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] *= inv;
  store_row<KIND>(a, b, j, row0 + row, dims, x);
}

// One row, by all 64 lanes of a wave and behind its store: a score per lane, 64 keys at a time, then lane d dimension d.
// The largest score is subtracted before the scale is applied.
template <int KIND>
__device__ inline void row_again(const CrossArgs& a, float c, int b, int j, int bj, int n_keys, int row) {
  wait_vmcnt<0>();
  const int lane = lane_of_wave();
  const Row qr = row_at(a, j, row);
  using T = std::conditional_t<KIND == kF32, float, __bf16>;
  const T* q = (const T*)a.q + b * a.qs[0] + qr.h * a.qs[1] + qr.i * a.qs[2];
  const int64_t kv_at = b * a.ks[0] + j * a.ks[1];
  float m = -INFINITY, l = 0.f, o = 0.f;
  for (int key0 = 0; key0 < n_keys; key0 += 64) {
    const int64_t at = kv_at + min(key0 + lane, n_keys - 1) * a.ks[2];
    const int64_t scale_at = KIND == kCodes ? (int64_t)bj * a.scale_blocks + key0 / kBlock : 0;
    float s = 0.f;
#pragma unroll 1
    for (int d = 0; d < 64; d += 8) {
      float x[8];
      if constexpr (KIND == kF32) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = ((const float*)a.k)[at + d + e];
      } else {
        bf16x8 w;
        if constexpr (KIND == kCodes) {
          const uint2 u = *(const uint2*)((const int8_t*)a.k + at + d);
          w = codes_to_bf16(u.x, u.y);
        } else {
          w = as_bf16x8(*(const uint4*)((const __bf16*)a.k + at + d));
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)w[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(x[e], (float)q[d + e], s);
    }
    float vs = 1.f;
    if constexpr (KIND == kCodes) { s *= nan_unless_finite(a.k_scale[scale_at]); vs = a.v_scale[scale_at]; }
    s = key0 + lane < n_keys ? s : -INFINITY;
    float mx = s;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
    const float to = fmaxf(m, mx);
    const float alpha = m > -INFINITY ? __builtin_amdgcn_exp2f((m - to) * c) : 0.f;
    const float p = __builtin_amdgcn_exp2f((s - (to > -INFINITY ? to : 0.f)) * c);
    float sum = p;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    l = fmaf(l, alpha, sum); o *= alpha; m = to;
    for (int i = 0; i < min(64, n_keys - key0); ++i) {
      const int64_t v_at = kv_at + (int64_t)(key0 + i) * a.ks[2] + lane;
      const float v = KIND == kCodes ? (float)((const int8_t*)a.v)[v_at] * vs : (float)((const T*)a.v)[v_at];
      o = fmaf(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(p), i)), v, o);
    }
  }
  ((T*)a.o + b * a.os[0] + qr.h * a.os[1] + qr.i * a.os[2])[lane] = (T)(o * (1.f / l));
}

// A wave's 32 rows from row0 on: O times unit over the row sum, of which `part` is this lane's share (no key: zeros), as
// bf16.  Rows whose reference went too far (their lanes in `far`), and rows whose products with V overflowed under a sum that
// had been let grow (the reference has moved, or the sum is above one per key), are formed again behind the store.
template <int KIND>
__device__ inline void store_tile(const CrossArgs& a, float c, int b, int j, int bj, int n_keys, int row0, const f32x16 (&O)[2],
                                  float part, float unit, uint64_t far, uint64_t moved) {
  const float l = part + other_half(part), inv = l > 0.f ? 1.f / l : 0.f;
  unsigned r[2][8];
#pragma unroll
  for (int dt = 0; dt < 2; ++dt)
#pragma unroll
    for (int e = 0; e < 16; e += 2) {
      float x = O[dt][e] * inv, y = O[dt][e + 1] * inv;
      if constexpr (KIND == kCodes) { x *= unit; y *= unit; }
      r[dt][e / 2] = __builtin_bit_cast(unsigned, bf16x2{(__bf16)x, (__bf16)y});
    }
  const int row = row0 + (lane_of_wave() & 31);          // (formed anew: not worth registers through the loop)
  if (row < a.rows) {
    const Row qr = row_at(a, j, row);
    __bf16* op = (__bf16*)a.o + b * a.os[0] + qr.h * a.os[1] + qr.i * a.os[2] + 8 * (lane_of_wave() >> 5);
#pragma unroll
    for (int dt = 0; dt < 2; ++dt)
#pragma unroll
      for (int jj = 0; jj < 2; ++jj) {
        // dims 32 dt + 16 jj .. + 15 of the row: its lanes hold 4 of each 8; exchanged, 8 in a row
        const auto x0 = __builtin_amdgcn_permlane32_swap(r[dt][4 * jj], r[dt][4 * jj + 2], false, false);
        const auto x1 = __builtin_amdgcn_permlane32_swap(r[dt][4 * jj + 1], r[dt][4 * jj + 3], false, false);
        const u32x4 piece = {x0[0], x1[0], x0[1], x1[1]};
        *(u32x4*)(op + 32 * dt + 16 * jj) = piece;
      }
  }
  const uint64_t again = (far | moved | __builtin_amdgcn_ballot_w64(l > (float)n_keys)) & __builtin_amdgcn_ballot_w64(row < a.rows);
  if (__builtin_expect(again != 0, 0)) {
    float any = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) any = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, r[e >> 3][e & 7]), kOnes, any, false);
    uint64_t bad = (far | __builtin_amdgcn_ballot_w64(not_finite(any))) & again;
    bad = (bad | (bad >> 32)) & 0xffffffffull;
    for (; bad != 0; bad &= bad - 1) row_again<KIND>(a, c, b, j, bj, n_keys, row0 + __builtin_ctzll(bad));
  }
}

// What store_tile does for a part of the key axis: products (times unit), reference and sum of a wave's 32 rows for k_cross_join;
// a reference of +inf asks it to form the row again.
template <int KIND>
__device__ inline void keep_part(const CrossArgs& a, int bj, int part, int n_keys, int row0, const f32x16 (&O)[2], float share,
                                 float negm, float unit, uint64_t far, uint64_t moved) {
  const int lane = lane_of_wave(), n = lane & 31;
  const float l = share + other_half(share);
  const int64_t row = (((int64_t)bj * a.tiles + row0 / kRows) * a.parts + part) * kRows + n;
  float any = 0.f;
  float* o = a.part_o + row * 64 + 4 * (lane >> 5);
#pragma unroll
  for (int dt = 0; dt < 2; ++dt)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {          // dims 32 dt + 2 e + 4 (lane / 32) .. + 3
      float4 x = make_float4(O[dt][e], O[dt][e + 1], O[dt][e + 2], O[dt][e + 3]);
      if constexpr (KIND == kCodes) { x.x *= unit; x.y *= unit; x.z *= unit; x.w *= unit; }
      any += (x.x + x.y) + (x.z + x.w);
      *(float4*)(o + 32 * dt + 2 * e) = x;
    }
  uint64_t bad = far | (__builtin_amdgcn_ballot_w64(not_finite(any)) & (moved | __builtin_amdgcn_ballot_w64(l > (float)n_keys)));
  bad |= bad >> 32;
  if (lane < 32) a.part_ml[row] = make_float2(n_keys <= 0 ? -INFINITY : (bad >> n) & 1 ? INFINITY : not_finite(l) ? 0.f : -negm, l);
}

// Many rows: NWV waves of one (batch, kv head), each with 32 rows, share the K and V rows, which pass through LDS in chunks
// of 64 keys, three buffers: one read, one landing, one whose last readers may be behind, so that one barrier per chunk
// is enough.  All come by LDS-DMA.  The score products of a block of 32 keys are issued ahead of the exponentials of the
// block before it.
//
// Softmax in base 2: the reference is the largest score of the first block and moves (by whole powers of two) when a sum
// passes 2^40, so that no maximum is formed in the other blocks.  Rows whose reference went beyond kFarReference, where its
// rounding would show (on codes kFarCodes, for the V scale that joins it), and rows that overflowed are formed again behind the store.
//
// Codes come to a place behind the buffers and are converted (exactly) from there by the wave that brought them.  Two buffers
// do, 40 KiB with the codes, so that a CU holds four workgroups of four waves or two of eight; it costs the score products
// issued ahead across chunks.  480 pairs of 169 rows on 384 keys: three buffers, codes through registers, workgroups of four
// 24.5 us; three chunks of codes on their way instead of one 24.3 (nothing waits for memory); so 23.8; of eight, which convert a
// chunk once for six tiles, and a byte in one instruction, 21.0 (18.0 in bf16).
// A chunk is a block, its K scale joins the softmax scale.  Its V scale, relative to the largest of the
// keys that count, is added to the exponent, which costs nothing per score; the chunk's part of the row sum is divided by it
// again.  (Relative V scales are taken as at least 2^-96, so that no probability that counts is flushed to zero.)
//
// 288 pairs of 2240 rows on 149 to 512 keys: 88 to 92 us from card to card (650 to 624 TFLOP/s; on 2048 keys each 870).  What bounds it there is the vector issue,
// 54 instructions and 16 exponentials for 32 rows x 32 keys, about 300 more for a tile's start and end, and Q and O, 34 us
// at the copy rate, beside which a round of workgroups starts and ends with little else to do.  512 workgroups that stay, each with
// a run of five or six tiles whose rows of Q come under the tile before: 102 us (the runs are uneven).
template <int NWV, int KIND, bool PARTS>
__global__ __launch_bounds__(NWV * 64) __attribute__((amdgpu_waves_per_eu(NWV == 4 && KIND == kBf16 ? 3 : 4, NWV == 4 && KIND == kBf16 ? 3 : 4)))
void k_cross_tiles(CrossArgs a, float c) {
  constexpr bool CODES = KIND == kCodes;
  constexpr int kRowsPerWave = kBlock / NWV, kTransfers = kRowsPerWave / 8, kBuf = 2 * kBlock * kRow;
  __shared__ __align__(1024) unsigned char smem[CODES ? 2 * kBuf + 8192 : 3 * kBuf];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int n = lane & 31, hh = lane >> 5;
  // Workgroup i runs on XCD i % 8, each with an L2 of its own: the tiles of a pair follow one another on one XCD, or, with
  // few pairs, all pairs of one tile follow one another, which uses all XCDs.
  int tile, bj, b, j;
  const uint32_t block = a.first_block + blockIdx.x;
  if (a.by_xcd) {
    divmod_by(block >> 3, (uint32_t)a.groups, a.groups_magic, bj, tile);
    bj = 8 * bj + (int)(block & 7);
    if (bj >= a.B * a.Hkv) return;
  } else {
    divmod_by(block, (uint32_t)(a.B * a.Hkv), a.pairs_magic, tile, bj);
  }
  divmod_by((uint32_t)bj, (uint32_t)a.Hkv, a.hkv_magic, b, j);
  int n_keys;
  b = batch_of_rank(a, b, n_keys);
  bj = b * a.Hkv + j;
  // PARTS: the blocks of this part, the first of which counts as block 0 below
  [[maybe_unused]] int part = 0, first_block = 0;
  if constexpr (PARTS) {
    divmod_by((uint32_t)tile, (uint32_t)a.parts, a.parts_magic, tile, part);
    const int blocks = (n_keys + kBlock - 1) / kBlock;
    first_block = (int)((int64_t)blocks * part / a.parts);
    n_keys = min(n_keys, (int)((int64_t)blocks * (part + 1) / a.parts) * kBlock) - first_block * kBlock;
  }
  const int row0 = (tile * NWV + wave) * kRows;
  const bool working = row0 < a.rows;          // (uniform)
  bf16x8 qf[4];
  {
    const Row qr = row_at(a, j, min(row0 + n, a.rows - 1));    // (a column without a row holds the last one; it is not stored)
    const __bf16* qp = (const __bf16*)a.q + b * a.qs[0] + qr.h * a.qs[1] + qr.i * a.qs[2] + 8 * hh;
#pragma unroll
    for (int t = 0; t < 4; ++t) qf[t] = as_bf16x8(*(const uint4*)(qp + 16 * t));
  }
  const int n_chunks = (n_keys + kBlock - 1) / kBlock;
  __builtin_amdgcn_sched_barrier(0);           // (the loads of Q stay ahead of the transfers, which are counted below)

  // ---- loading duty ----
  const int64_t kv_at = b * a.ks[0] + j * a.ks[1] + (int64_t)first_block * kBlock * a.ks[2];
  const int lrow = lane >> 3;
  const unsigned piece_off = (((unsigned)lane & 7u) ^ dense_swizzle((unsigned)lrow)) << 4;
  [[maybe_unused]] const unsigned row_bytes = (unsigned)a.ks[2] * 2u;
  [[maybe_unused]] auto issue_chunk = [&](int chunk, int buf) {
#pragma unroll
    for (int i = 0; i < kTransfers; ++i) {
      // (a scalar base per chunk and 32-bit offsets inside it: 64 rows span less than 4 GiB, checked by the launch)
      const int r0 = kRowsPerWave * wave + 8 * i, key = min(r0 + lrow, n_keys - 1 - kBlock * chunk);
      const int64_t base = (kv_at + (int64_t)chunk * kBlock * a.ks[2]) * 2;
      const unsigned src = (unsigned)key * row_bytes + piece_off;
      unsigned char* dst = smem + buf * kBuf + r0 * kRow;
      __builtin_amdgcn_global_load_lds((global_void*)((const unsigned char*)a.k + base + src), (lds_void*)dst, 16, 0, 0);
      __builtin_amdgcn_global_load_lds((global_void*)((const unsigned char*)a.v + base + src), (lds_void*)(dst + kBlock * kRow), 16, 0, 0);
    }
  };
  // codes: a chunk is eight pieces of 16 K or V rows, 1 KiB each, which LDS-DMA leaves behind the buffers; the wave that
  // brought a piece converts it into a buffer
  constexpr int kPieces = 8 / NWV;
  [[maybe_unused]] unsigned char* const stage = smem + 2 * kBuf;
  [[maybe_unused]] auto issue_codes = [&](int chunk) {
    int lane = lane_of_wave();
    asm volatile("" : "+v"(lane));             // (addresses formed anew in every chunk: not worth registers through the loop)
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int piece = wave + NWV * i, key = min(16 * (piece & 3) + (lane >> 2), n_keys - 1 - kBlock * chunk);
      const int8_t* base = (const int8_t*)(piece < 4 ? a.k : a.v) + kv_at + (int64_t)chunk * (kBlock * 64);
      __builtin_amdgcn_global_load_lds((global_void*)(base + (unsigned)(key * 64 + 16 * (lane & 3))), (lds_void*)(stage + 1024 * piece), 16, 0, 0);
    }
  };
  [[maybe_unused]] auto commit_codes = [&](int buf_at) {
    int lane = lane_of_wave();
    asm volatile("" : "+v"(lane));
    wait_vmcnt<0>();
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int piece = wave + NWV * i, row = 16 * (piece & 3) + (lane >> 2);
      const u32x4 codes = *(const u32x4*)(stage + 1024 * piece + 16 * lane);
      const unsigned at = 2u * ((unsigned)lane & 3u), sw = dense_swizzle((unsigned)row);
      unsigned char* dst = smem + buf_at + (piece < 4 ? 0 : kBlock * kRow) + row * kRow;
      *(bf16x8*)(dst + ((at ^ sw) << 4)) = codes_to_bf16(codes[0], codes[1]);
      *(bf16x8*)(dst + (((at + 1u) ^ sw) << 4)) = codes_to_bf16(codes[2], codes[3]);
    }
  };
  // the scales of 64 chunks, one to a lane: K's, log2 of V's relative to the largest and its reciprocal
  [[maybe_unused]] float vmax = 0.f, log_vmax = 0.f, lane_ks = 1.f, lane_lv = 0.f, lane_iv = 1.f;
  [[maybe_unused]] auto scales_at = [&](int chunk) {
    int lane = lane_of_wave();
    asm volatile("" : "+v"(lane));             // (formed anew: not worth a register through the loop)
    return (int64_t)bj * a.scale_blocks + first_block + min(chunk + lane, n_chunks - 1);
  };
  [[maybe_unused]] auto set_scales = [&](float ks, float vs) {
    lane_ks = nan_unless_finite(ks);
    // (a scale of zero belongs to a block of zeros: any will do)
    // (one that is not finite makes NaN of its block's probabilities: it would enter no maximum and no product; as bits, see not_finite)
    unsigned lv = __float_as_uint(vs > 0.f ? fmaxf(log2_of(vs) - log_vmax, -96.f) : 0.f);
    lv = not_finite(vs) ? 0x7fc00000u : lv;
    asm volatile("" : "+v"(lv));
    lane_lv = __uint_as_float(lv);
    lane_iv = __builtin_amdgcn_exp2f(-lane_lv);
    asm volatile("" : "+v"(lane_ks));          // (its load is waited for here, not wherever the chunks go on)
  };
  [[maybe_unused]] auto scale_of = [](float x, int chunk) {
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), chunk & 63));
  };

  // LDS read offsets: K piece 2 t + hh of row n; V: 4 keys x 16 dims per 16 lanes
  unsigned k_off[4], v_off[2];
#pragma unroll
  for (int t = 0; t < 4; ++t)
    k_off[t] = lds_addr(smem) + (unsigned)n * kRow + ((((unsigned)(2 * t + hh)) ^ dense_swizzle((unsigned)n)) << 4);
#pragma unroll
  for (int dt = 0; dt < 2; ++dt) {
    const unsigned l16 = (unsigned)lane & 15u, r = 4u * (unsigned)hh + (l16 >> 2);
    const unsigned piece = 4u * dt + 2u * (((unsigned)lane >> 4) & 1u) + ((l16 & 3u) >> 1);
    v_off[dt] = lds_addr(smem) + r * kRow + ((piece ^ dense_swizzle(r)) << 4) + 8u * (l16 & 1u);
  }

  f32x16 O[2] = {f32x16{}, f32x16{}};
  float L[2] = {0.f, 0.f}, negm = 0.f;         // this lane's part of the row sum, one chain per slice; minus the reference (base 2)
  bool unset = true;
  uint64_t far = 0, moved = 0;                 // lanes whose reference has been beyond kFar, has moved

  auto is_beyond = [](float x) { return __builtin_amdgcn_ballot_w64(!(fabsf(x) < (CODES ? kFarCodes : kFarReference))); };
  auto scores = [&](u32x4 (&kr)[4]) -> f32x16 {
    lds_wait_k(kr[0], kr[1], kr[2], kr[3]);
    f32x16 S = f32x16{};
#pragma unroll
    for (int t = 0; t < 4; ++t)
      S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kr[t]), qf[t], S, 0, 0, 0);
    return S;
  };
  // of the block from key0 on, the scores of keys that do not exist
  auto mask = [&](f32x16& S, int key0) {
    if (key0 + 32 > n_keys) {                  // (uniform)
      const int left = n_keys - key0 - 4 * hh;
#pragma unroll
      for (int e = 0; e < 16; ++e) S[e] = 8 * (e >> 2) + (e & 3) < left ? S[e] : -INFINITY;
    }
  };
  // the rest of a block, its V rows requested; ks, lv, iv: of its chunk
  auto absorb = [&](f32x16& S, u32x2 (&va)[8], float ks, float lv, float iv) {
    if (CODES && (ks < a.ks_least || ks > a.ks_most)) {   // (scaled here: c ks would lose its bits, a block of zeros, or overflow)
#pragma unroll
      for (int e = 0; e < 16; ++e) S[e] = S[e] > -INFINITY ? S[e] * ks : S[e];
      ks = 1.f;
    }
    auto largest = [&]() {                     // of the row, over both of its lanes
      float mx = S[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = fmaxf(mx, S[e]);
      return fmaxf(mx, other_half(mx));
    };
    const float cb = CODES ? c * ks : c;
    if (unset) {
      negm = -largest() * cb; unset = false;
      far = is_beyond(negm);
    }
    bf16x8 pb[2];
    float sum[2];
    auto exponentials = [&]() {
      const float at = CODES ? negm + lv : negm;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        sum[t] = CODES ? 0.f : L[t];
#pragma unroll
        for (int e = 0; e < 8; ++e) pb[t][e] = (__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(S[8 * t + e], cb, at));
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const bf16x2 two = {pb[t][e], pb[t][e + 1]};
          sum[t] = __builtin_amdgcn_fdot2_f32_bf16(two, kOnes, sum[t], false);
        }
        if constexpr (CODES) sum[t] = __builtin_fmaf(sum[t], iv, L[t]);
      }
    };
    exponentials();
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(fmaxf(sum[0], sum[1]) > kMostSum) != 0, 0)) {
      auto both = [&](const float (&x)[2]) { const float y = x[0] + x[1]; return y + other_half(y); };   // slices, lanes
      const float now = both(sum), before = both(L);
      float to = __builtin_fmaf(largest(), cb, negm);
      if (before > 0.f) to = fmaxf(to, __builtin_amdgcn_logf(before));         // (base 2)
      const float shift = now > kMostSum ? rintf(to) : 0.f, alpha = __builtin_amdgcn_exp2f(-shift);
      negm -= shift; L[0] *= alpha; L[1] *= alpha;
      far |= is_beyond(negm);
      moved |= __builtin_amdgcn_ballot_w64(shift != 0.f);
#pragma unroll
      for (int e = 0; e < 16; ++e) { O[0][e] *= alpha; O[1][e] *= alpha; }
      exponentials();
    }
    L[0] = sum[0]; L[1] = sum[1];
    lds_wait_v_wide(va);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int dt = 0; dt < 2; ++dt) {
        const uint4 v8 = {va[4 * t + dt].x, va[4 * t + dt].y, va[4 * t + 2 + dt].x, va[4 * t + 2 + dt].y};
        O[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(v8), pb[t], O[dt], 0, 0, 0);
      }
  };

  // A wave's priority falls with the chunks that it still has: the scheduler prefers the oldest workgroup of a CU, and the
  // one after it would be left to work alone, at half the rate
  auto set_priority = [&](int chunk) {
    if (a.prio_magic == 0) return;
    switch (((uint32_t)(n_chunks - 1 - chunk) * a.prio_magic) >> 16) {
      case 0: __builtin_amdgcn_s_setprio(0); break;
      case 1: __builtin_amdgcn_s_setprio(1); break;
      case 2: __builtin_amdgcn_s_setprio(2); break;
      default: __builtin_amdgcn_s_setprio(3);
    }
  };
  if (n_chunks > 0) {
    if constexpr (CODES) {
      const float ks = a.k_scale[scales_at(0)], vs = a.v_scale[scales_at(0)];
      issue_codes(0);
      vmax = vs;
      for (int at = 64; at < n_chunks; at += 64) vmax = fmaxf(vmax, a.v_scale[scales_at(at)]);
      vmax = wave_max(vmax);
      log_vmax = uniform(log2_of(vmax));
      set_scales(ks, vs);
      commit_codes(0);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (n_chunks > 1) issue_codes(1);
      asm volatile("s_barrier" ::: "memory");
    } else {
      issue_chunk(0, 0);
      if (n_chunks > 1) { issue_chunk(1, 1); wait_vmcnt<2 * kTransfers>(); } else wait_vmcnt<0>();
      asm volatile("" : "+v"(qf[0]), "+v"(qf[1]), "+v"(qf[2]), "+v"(qf[3]));   // (older than the chunks: in)
      asm volatile("s_barrier" ::: "memory");
    }
    if constexpr (CODES) {
      // A chunk: the score products of both blocks, then their exponentials.  In between the next chunk is converted into
      // the other buffer, which nobody has read since the barrier that let this chunk begin.
      for (int chunk = 0, at = 0;; ++chunk, at = kBuf - at) {
        set_priority(chunk);
        const float ks = scale_of(lane_ks, chunk), lv = scale_of(lane_lv, chunk), iv = scale_of(lane_iv, chunk);
        const int key0 = chunk * kBlock;
        const bool more = chunk + 1 < n_chunks, second = key0 + 32 < n_keys;
        const unsigned v_at[2] = {v_off[0] + at, v_off[1] + at};
        f32x16 S1;
        asm volatile("" : "=v"(S1));             // (not set where there is no second block, and not used then)
        if (working) {
          const unsigned k_at[4] = {k_off[0] + at, k_off[1] + at, k_off[2] + at, k_off[3] + at};
          f32x16 S0;
          u32x2 va[8];
          {
            u32x4 kr[4];
            read_k<0>(k_at, kr);
            S0 = scores(kr);
          }
          if (second) {
            u32x4 kr[4];
            read_k<32 * kRow>(k_at, kr);
            S1 = scores(kr);
          }
          read_v<kBlock * kRow>(v_at, va);
          __builtin_amdgcn_sched_barrier(0);
          mask(S0, key0);
          absorb(S0, va, ks, lv, iv);
        }
        if (more) {
          commit_codes(kBuf - at);
          if (((chunk + 1) & 63) == 0) set_scales(a.k_scale[scales_at(chunk + 1)], a.v_scale[scales_at(chunk + 1)]);
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          if (chunk + 2 < n_chunks) issue_codes(chunk + 2);
        }
        if (working && second) {
          u32x2 va[8];
          read_v<(kBlock + 32) * kRow>(v_at, va);
          __builtin_amdgcn_sched_barrier(0);
          mask(S1, key0 + 32);
          absorb(S1, va, ks, lv, iv);
        }
        if (!more) break;
        asm volatile("s_barrier" ::: "memory");
      }
    } else {
      f32x16 S0 = f32x16{};                    // scores of the chunk's first block
      if (working) {
        u32x4 kr[4];
        read_k<0>(k_off, kr);
        S0 = scores(kr);
      }
      // A chunk: its two blocks, each with the next block's score products in front of its own exponentials.  Between the
      // blocks the next chunk is made sure of and the one after it requested, for the buffer that every wave has read to
      // its end by then.
      auto one = [&](int chunk, auto which) -> bool {
        constexpr int p = decltype(which)::value, AT = p * kBuf, NEXT = (p + 1) % 3 * kBuf;
        const int key0 = chunk * kBlock;
        const bool more = chunk + 1 < n_chunks, second = key0 + 32 < n_keys;
        set_priority(chunk);
        f32x16 S1;
        asm volatile("" : "=v"(S1));           // (not set where there is no second block, and not used then)
        if (working) {
          u32x2 va[8];
          if (second) {
            u32x4 kr[4];
            read_k<AT + 32 * kRow>(k_off, kr);
            S1 = scores(kr);
          }
          read_v<AT + kBlock * kRow>(v_off, va);
          __builtin_amdgcn_sched_barrier(0);
          mask(S0, key0);
          absorb(S0, va, 1.f, 0.f, 1.f);
        }
        if (more) {
          wait_vmcnt<0>();
          asm volatile("s_barrier" ::: "memory");
          if (chunk + 2 < n_chunks) issue_chunk(chunk + 2, (p + 2) % 3);
        }
        if (working && second) {
          u32x2 va[8];
          if (more) {
            u32x4 kr[4];
            read_k<NEXT>(k_off, kr);
            S0 = scores(kr);
          }
          read_v<AT + (kBlock + 32) * kRow>(v_off, va);
          __builtin_amdgcn_sched_barrier(0);
          mask(S1, key0 + 32);
          absorb(S1, va, 1.f, 0.f, 1.f);
        }
        return more;
      };
      for (int chunk = 0;; chunk += 3) {
        if (!one(chunk, std::integral_constant<int, 0>{})) break;
        if (!one(chunk + 1, std::integral_constant<int, 1>{})) break;
        if (!one(chunk + 2, std::integral_constant<int, 2>{})) break;
      }
    }
  }

  if (!working) return;
  if constexpr (PARTS) keep_part<KIND>(a, bj, part, n_keys, row0, O, L[0] + L[1], negm, CODES ? vmax : 1.f, far, moved);
  else store_tile<KIND>(a, c, b, j, bj, n_keys, row0, O, L[0] + L[1], CODES ? vmax : 1.f, far, moved);
}

// a lane's half of a K row of 256 bytes, eight pieces; issued only, a wait must precede the first use
template <int AT> __device__ inline void read_k_rows(unsigned k, u32x4 (&r)[8]) {
#pragma unroll
  for (int t = 0; t < 8; t += 4)
    asm volatile("ds_read_b128 %0, %4 offset:%8\n\tds_read_b128 %1, %5 offset:%8\n\t"
                 "ds_read_b128 %2, %6 offset:%8\n\tds_read_b128 %3, %7 offset:%8"
                 : "=&v"(r[t]), "=&v"(r[t + 1]), "=&v"(r[t + 2]), "=&v"(r[t + 3])
                 : "v"(k ^ (16u * t)), "v"(k ^ (16u * t + 16u)), "v"(k ^ (16u * t + 32u)), "v"(k ^ (16u * t + 48u)), "i"(AT) : "memory");
}

// Many rows in fp32: as k_cross_tiles, 32 keys to a chunk.  The matrix pipe bounds it: 64 instructions of 64 cycles for 32
// keys x 32 rows, beside which vector instructions of other waves do not run (two waves per SIMD take twice as long as one), so
// that each of these counts: no maximum, no mask but in the last chunk, one multiply-add and one addition per score.  K pieces are
// swizzled by row (sixteen rows put a piece into sixteen places); V rows are read whole, lane n dimensions 2 n and 2 n + 1.
// Four buffers: 64 KiB leave two workgroups to a CU, so that a launch of a few per CU is dealt out as they end (three to a CU, all
// resident at once: 2240 rows, 32 pairs of 301 and 153 keys 58.9 us, so 56.4).
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
void k_cross_tiles_f32(CrossArgs a, float c) {
  constexpr int NWV = 4, kKeys = 32, kRowF = 256, kBuf = 2 * kKeys * kRowF, kBufs = 4, kTransfers = kKeys / (4 * NWV);
  __shared__ __align__(1024) unsigned char smem[kBufs * kBuf];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int n = lane & 31, hh = lane >> 5;
  int tile, bj, b, j;
  const uint32_t block = a.first_block + blockIdx.x;
  if (a.by_xcd) {
    divmod_by(block >> 3, (uint32_t)a.groups, a.groups_magic, bj, tile);
    bj = 8 * bj + (int)(block & 7);
    if (bj >= a.B * a.Hkv) return;
  } else {
    divmod_by(block, (uint32_t)(a.B * a.Hkv), a.pairs_magic, tile, bj);
  }
  divmod_by((uint32_t)bj, (uint32_t)a.Hkv, a.hkv_magic, b, j);
  int n_keys;
  b = batch_of_rank(a, b, n_keys);
  bj = b * a.Hkv + j;
  const int row0 = (tile * NWV + wave) * kRows;
  const bool working = row0 < a.rows;          // (uniform)
  float qf[32];
  {
    const Row qr = row_at(a, j, min(row0 + n, a.rows - 1));
    const float* qp = (const float*)a.q + b * a.qs[0] + qr.h * a.qs[1] + qr.i * a.qs[2] + 32 * hh;
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      const float4 x = *(const float4*)(qp + 4 * t);
      qf[4 * t] = x.x; qf[4 * t + 1] = x.y; qf[4 * t + 2] = x.z; qf[4 * t + 3] = x.w;
    }
  }
  __builtin_amdgcn_sched_barrier(0);           // (the loads of Q stay ahead of the transfers, which are counted below)
  const int n_chunks = (n_keys + kKeys - 1) / kKeys;
  // a transfer: four rows, sixteen lanes each
  const int64_t kv_at = b * a.ks[0] + j * a.ks[1];
  const unsigned row_bytes = (unsigned)a.ks[2] * 4u;
  auto issue_chunk = [&](int chunk, int buf) {
    const int64_t base = (kv_at + (int64_t)chunk * kKeys * a.ks[2]) * 4;
#pragma unroll
    for (int i = 0; i < kTransfers; ++i) {
      const int r0 = 4 * (kTransfers * wave + i), r = r0 + (lane >> 4);
      const unsigned from = (unsigned)min(r, n_keys - 1 - kKeys * chunk) * row_bytes, piece = (unsigned)lane & 15u;
      unsigned char* dst = smem + buf * kBuf + r0 * kRowF;
      __builtin_amdgcn_global_load_lds((global_void*)((const unsigned char*)a.k + base + (from + ((piece ^ ((unsigned)r & 15u)) << 4))), (lds_void*)dst, 16, 0, 0);
      __builtin_amdgcn_global_load_lds((global_void*)((const unsigned char*)a.v + base + (from + (piece << 4))), (lds_void*)(dst + kKeys * kRowF), 16, 0, 0);
    }
  };
  const unsigned k_at = lds_addr(smem) + (unsigned)n * kRowF + (((8u * (unsigned)hh) ^ ((unsigned)n & 15u)) << 4);
  const unsigned v_at = lds_addr(smem) + kKeys * kRowF + 4u * (unsigned)hh * kRowF + 8u * (unsigned)n;

  f32x16 O[2] = {f32x16{}, f32x16{}};          // row m of tile dt: dimension 2 m + dt
  float negm = 0.f, L = 0.f;                   // minus the reference (base 2), this lane's part of the row sum
  uint64_t far = 0;                            // lanes whose reference has been beyond kFarReference
  if (n_chunks > 0) {
    issue_chunk(0, 0);
    if (n_chunks > 1) issue_chunk(1, 1);
    if (n_chunks > 2) { issue_chunk(2, 2); wait_vmcnt<4 * kTransfers>(); } else wait_vmcnt<0>();
    asm volatile("s_barrier" ::: "memory");
  }
  auto one = [&](int chunk, auto which) -> bool {
    constexpr int p = decltype(which)::value, AT = p * kBuf;
    const bool more = chunk + 1 < n_chunks;
    if (working) {
      u32x4 kr[8];
      u32x2 vr[16];
      read_k_rows<AT>(k_at, kr);
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        asm volatile("ds_read_b64 %0, %4 offset:%5\n\tds_read_b64 %1, %4 offset:%6\n\t"
                     "ds_read_b64 %2, %4 offset:%7\n\tds_read_b64 %3, %4 offset:%8"
                     : "=&v"(vr[e]), "=&v"(vr[e + 1]), "=&v"(vr[e + 2]), "=&v"(vr[e + 3])
                     : "v"(v_at), "i"(AT + 2 * e * kRowF), "i"(AT + (2 * e + 1) * kRowF), "i"(AT + (2 * e + 2) * kRowF),
                       "i"(AT + (2 * e + 3) * kRowF) : "memory");
      asm volatile("s_waitcnt lgkmcnt(0)"
                   : "+v"(kr[0]), "+v"(kr[1]), "+v"(kr[2]), "+v"(kr[3]), "+v"(kr[4]), "+v"(kr[5]), "+v"(kr[6]), "+v"(kr[7]) : : "memory");
      asm volatile("" : "+v"(vr[0]), "+v"(vr[1]), "+v"(vr[2]), "+v"(vr[3]), "+v"(vr[4]), "+v"(vr[5]), "+v"(vr[6]), "+v"(vr[7]),
                        "+v"(vr[8]), "+v"(vr[9]), "+v"(vr[10]), "+v"(vr[11]), "+v"(vr[12]), "+v"(vr[13]), "+v"(vr[14]), "+v"(vr[15]));
      f32x16 S = f32x16{};
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const u32x4 w = kr[t];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const unsigned u = w[e];
          S = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(u), qf[4 * t + e], S, 0, 0, 0);
        }
      }
      if (!more) {                             // (uniform; kept a branch)
        int left = n_keys - chunk * kKeys - 4 * hh;
        asm volatile("" : "+v"(left));
#pragma unroll
        for (int e = 0; e < 16; ++e) S[e] = 8 * (e >> 2) + (e & 3) < left ? S[e] : -INFINITY;
      }
      auto largest = [&]() {                   // of the row, over both of its lanes
        float mx = S[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mx = fmaxf(mx, S[e]);
        return fmaxf(mx, other_half(mx));
      };
      if (chunk == 0) {
        negm = -largest() * c;
        far = is_far(negm);
      }
      float P[16], sum;
      auto exponentials = [&]() {
        sum = L;
#pragma unroll
        for (int e = 0; e < 16; ++e) { P[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[e], c, negm)); sum += P[e]; }
      };
      exponentials();
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(sum > kMostSum) != 0, 0)) {
        const float now = sum + other_half(sum), before = L + other_half(L);
        float to = __builtin_fmaf(largest(), c, negm);
        if (before > 0.f) to = fmaxf(to, __builtin_amdgcn_logf(before));       // (base 2)
        const float shift = now > kMostSum ? rintf(to) : 0.f, alpha = __builtin_amdgcn_exp2f(-shift);
        negm -= shift; L *= alpha;
        far |= is_far(negm);
#pragma unroll
        for (int e = 0; e < 16; ++e) { O[0][e] *= alpha; O[1][e] *= alpha; }
        exponentials();
      }
      L = sum;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const unsigned u0 = vr[e][0], u1 = vr[e][1];
        O[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(u0), P[e], O[0], 0, 0, 0);
        O[1] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(u1), P[e], O[1], 0, 0, 0);
      }
    }
    if (!more) return false;
    if (chunk + 2 < n_chunks) wait_vmcnt<2 * kTransfers>(); else wait_vmcnt<0>();      // (the next chunk is in)
    asm volatile("s_barrier" ::: "memory");
    if (chunk + 3 < n_chunks) issue_chunk(chunk + 3, (p + 3) % kBufs);
    return true;
  };
  for (int chunk = 0; n_chunks > 0; chunk += kBufs) {
    if (!one(chunk, std::integral_constant<int, 0>{})) break;
    if (!one(chunk + 1, std::integral_constant<int, 1>{})) break;
    if (!one(chunk + 2, std::integral_constant<int, 2>{})) break;
    if (!one(chunk + 3, std::integral_constant<int, 3>{})) break;
  }
  if (!working) return;
  const float l = L + other_half(L), inv = l > 0.f ? 1.f / l : 0.f;            // (no key: zeros)
  const int row = row0 + (lane_of_wave() & 31);
  float any = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) { O[0][e] *= inv; O[1][e] *= inv; any += O[0][e] + O[1][e]; }
  if (row < a.rows) {
    const Row qr = row_at(a, j, row);
    // O[dt][e]: dimension 2 (8 (e / 4) + 4 hh + e % 4) + dt
    float* op = (float*)a.o + b * a.os[0] + qr.h * a.os[1] + qr.i * a.os[2] + 8 * (lane_of_wave() >> 5);
#pragma unroll
    for (int e = 0; e < 16; e += 2)
      *(float4*)(op + 16 * (e >> 2) + 2 * (e & 3)) = make_float4(O[0][e], O[1][e], O[0][e + 1], O[1][e + 1]);
  }
  // (rows formed again as in k_cross_tiles)
  uint64_t bad = (far | __builtin_amdgcn_ballot_w64(not_finite(any))) & __builtin_amdgcn_ballot_w64(row < a.rows);
  bad = (bad | (bad >> 32)) & 0xffffffffull;
  for (; __builtin_expect(bad != 0, 0); bad &= bad - 1) row_again<kF32>(a, c, b, j, bj, n_keys, row0 + __builtin_ctzll(bad));
}

// Joins the parts of a row (references times unit are in base 2): a workgroup per row, thread t dims 4 (t % 16) .. + 3 of the parts t / 16, + 16, ...
template <int KIND>
__global__ __launch_bounds__(256) void k_cross_join(CrossArgs a, float unit, float c) {
  __shared__ float weight[kMaxParts], wave_m[4], wave_l[4];
  __shared__ __align__(16) float4 sums[16][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int bj, r, b, j;
  divmod_by(a.first_block + blockIdx.x, (uint32_t)a.rows, a.rows_magic, bj, r);
  divmod_by((uint32_t)bj, (uint32_t)a.Hkv, a.hkv_magic, b, j);
  const int tile = r / kRows, row = r % kRows;
  const int64_t first = ((int64_t)bj * a.tiles + tile) * a.parts;
  float m = -INFINITY, own_m[kMaxParts / 256], own_l[kMaxParts / 256];
#pragma unroll
  for (int i = 0; i < kMaxParts / 256; ++i) {
    const int s = tid + 256 * i;
    const float2 ml = s < a.parts ? a.part_ml[(first + s) * kRows + row] : make_float2(-INFINITY, 0.f);
    own_m[i] = ml.x; own_l[i] = ml.y;
    m = fmaxf(m, ml.x);
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  if (lane == 0) wave_m[wave] = m;
  __syncthreads();
  m = fmaxf(fmaxf(wave_m[0], wave_m[1]), fmaxf(wave_m[2], wave_m[3]));
  if (m == INFINITY) {                         // (see keep_part)
    if (wave == 0) row_again<KIND>(a, c, b, j, bj, keys_of(a, b), r);
    return;
  }
  float l = 0.f;
#pragma unroll
  for (int i = 0; i < kMaxParts / 256; ++i) {
    // (a part without keys: its products were not written, and do not count)
    const float f = own_m[i] > -INFINITY ? __builtin_amdgcn_exp2f((own_m[i] - m) * unit) : 0.f;
    l = fmaf(own_l[i], f, l);
    weight[tid + 256 * i] = own_m[i] > -INFINITY ? f : -1.f;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) l += __shfl_xor(l, d);
  if (lane == 0) wave_l[wave] = l;
  __syncthreads();
  l = (wave_l[0] + wave_l[1]) + (wave_l[2] + wave_l[3]);
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int s = tid >> 4; s < a.parts; s += 16) {
    const float f = weight[s];
    const float4 y = *(const float4*)(a.part_o + ((first + s) * kRows + row) * 64 + 4 * (tid & 15));
    if (f >= 0.f) { x.x = fmaf(y.x, f, x.x); x.y = fmaf(y.y, f, x.y); x.z = fmaf(y.z, f, x.z); x.w = fmaf(y.w, f, x.w); }
  }
  sums[tid >> 4][tid & 15] = x;
  __syncthreads();
  if (wave != 0) return;
  float any = 0.f;
  if (tid < 8) {
    float out[8] = {};
    for (int s = 0; s < 16; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) out[e] += ((const float*)&sums[s][2 * tid])[e];
    const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) { out[e] *= inv; any += out[e]; }
    store_row<KIND>(a, b, j, r, tid, out);
  }
  // (as in store_tile: products that only overflowed under sums that had been let grow, those of all parts together; and rows whose
  // scores are all -inf in fp32, which become NaN there)
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(not_finite(any) || l == 0.f) != 0, 0)) {
    const int n_keys = keys_of(a, b);
    if (n_keys > 0 && (l == 0.f || l > (float)n_keys)) row_again<KIND>(a, c, b, j, bj, n_keys, r);
  }
}

namespace {

// Parts of the key axis for `tiles` tiles of 32 rows, `rows` rows in all.  A workgroup without parts needs 4.2 us and 0.36
// per block of 64 keys (bf16); parts divide that, and cost a second launch of 3.3 us and 0.27 ns per row and part for the sums that
// they leave.  That is least at sqrt(1355 blocks / rows) parts; with fewer than three, few blocks, or a tile for nearly every
// CU there is nothing to gain.  (Tiles, rows, blocks), bf16, us without / with as many parts as given here: (1, 1, 64) 26.2 / 8.7 (64);
// (8, 256, 64) 27.9 / 10.4 (18); (32, 1024, 64) 31.4 / 13.4 (9); (128, 4096, 64) 36.5 / 25.6 (4); (128, 4096, 256) 124 / 56 (4);
// (192, 4992, 165) 80 / 58 (5); (200, 6000, 125) 64 / 50 (5); (260, 5200, 94) 62 / 56 (3); (300, 9600, 125) 91 / 86 (3);
// declined (one rule for all types, which the size of the workspace knows nothing of: 225 to 256 tiles for fp32's sake): (256, 8192,
// 188) 118 / 100 (4), fp32 257 / 285; (220, 7040, 63) 35.6 / 38.1 (3); (400, 12800, 157) 117 / 155 (2); (64, 64, 4) 5.8 / 7.9 (4); (256, 256, 64) 40.2 / 46.2 (4); (256, 6400, 64) 39.7 / 41.4 (4).
int parts_of(int64_t tiles, int64_t rows, int64_t kv_len) {
  const int64_t blocks = (kv_len + kBlock - 1) / kBlock;
  const bool long_axis = blocks >= 80;
  if (tiles < 1 || tiles >= (long_axis ? 320 : 200) || (tiles > 224 && tiles <= 256) || blocks <= 8) return 1;
  int64_t most = blocks / 16 < 64 ? 64 : blocks / 16;
  if (most > kMaxParts) most = kMaxParts;
  if (most > blocks) most = blocks;
  const int64_t items = long_axis && tiles > 128 ? 1024 : 512;   // (workgroups)
  if (most > items / tiles) most = items / tiles;
  int64_t p = (int64_t)std::sqrt(1355.0 * (double)blocks / (double)rows);
  if (p > most) p = most;
  return p < 3 ? 1 : (int)p;
}

// Parts of a long key axis where rows share K and V through LDS in 16 and 8 bits: four workgroups of four waves to a CU, eight
// blocks to a part at least.  (Pairs, tiles of one, blocks), us, bf16 / codes, each tile its own, shared, and in parts: (3, 222, 192) 166 /
// 190, 181 / 249, 99 / 110; (12, 27, 314) 180 / 195, 294 / 401, 85 / 88; (10, 33, 101) 63 / 70, 97 / 131, 46 / 46; (16, 16, 125) 62 / 57, 119 / 160,
// 41 / 44; declined: (60, 8, 63) 45 / 49, 62 / 83, 46 / 48; (140, 5, 47) 49 / 54, 58 / 77, 54 / 61.
int shared_parts_of(int64_t pairs, int64_t tiles, int64_t kv_len) {
  const int64_t blocks = (kv_len + kBlock - 1) / kBlock, fours = pairs * ((tiles + 3) / 4);
  if (tiles < 4 || pairs * tiles < 200 || blocks < 80 || fours > 256) return 1;
  const int64_t p = std::min(1024 / fours, blocks / 8);
  return (int)std::min(p, (int64_t)kMaxParts);
}

// Whether rows share K and V through LDS (k_cross_tiles, k_cross_tiles_f32): from so many tiles of 32 rows on, and two or
// more of a pair.  (Tiles, keys), us, shared / each tile its own: bf16 (352, 1024) 17.9 / 16.6, (512, 1024) 18.2 / 24.0, (1024, 1024)
// 20.1 / 42.3; codes (512, 1024) 24.3 / 19.6, (640, 1024) 24.5 / 24.3, (960,
// 1024) 24.2 / 30.2, (1920, 1024) 31.4 / 50.6; fp32 (960, 1024) 131 / 97, (1408, 1024) 136 /
// 133, (2048, 1024) 139 / 181.
template <int KIND> bool shares_rows(const CrossArgs& a) {
  // (64 rows of K or V span less than 4 GiB, see issue_chunk)
  const int64_t least = KIND == kF32 ? 1800 : a.shared_parts > 1 ? 0 : KIND == kCodes ? 672 : 448;
  return (a.parts == 1 || (KIND != kF32 && a.shared_parts > 1)) && a.tiles > 1 && a.ks[2] < (1 << 23) && (int64_t)a.B * a.Hkv * a.tiles >= least;
}

uint32_t magic_of(int64_t n) { return (uint32_t)(((uint64_t)1 << 32) / (uint64_t)(n > 1 ? n : 1) - (n <= 1)); }

litevar_status check_shape(int32_t B, int32_t H, int32_t H_kv, int32_t q_len, int32_t kv_len) {
  if (B < 1 || H < 1 || H_kv < 1) return fail(LITEVAR_E_INVALID_ARG, "B, H and H_kv must be positive (got %d, %d, %d)", B, H, H_kv);
  if (H % H_kv) return fail(LITEVAR_E_INVALID_ARG, "H = %d is not a multiple of H_kv = %d", H, H_kv);
  if (q_len < 0 || kv_len < 0) return fail(LITEVAR_E_INVALID_ARG, "q_len and kv_len must not be negative (got %d, %d)", q_len, kv_len);
  if ((int64_t)B * H > (1 << 24)) return fail(LITEVAR_E_UNSUPPORTED, "B*H above 2^24");
  if ((int64_t)(H / H_kv) * q_len >= ((int64_t)1 << 31) - kRows || kv_len >= 0x7fffffff - 2 * kBlock)
    return fail(LITEVAR_E_UNSUPPORTED, "2^31 rows of a kv head, or 2^31 keys, or more");
  if ((int64_t)B * H_kv * (((int64_t)(H / H_kv) * q_len + kRows - 1) / kRows) >= 0x7fffffff)
    return fail(LITEVAR_E_UNSUPPORTED, "grid too large");
  return LITEVAR_OK;
}

int64_t tiles_of(int32_t B, int32_t H, int32_t H_kv, int32_t q_len) {
  return (int64_t)B * H_kv * (((int64_t)(H / H_kv) * q_len + kRows - 1) / kRows);
}

template <int KIND> litevar_status launch(CrossArgs& a, float c, hipStream_t st) {
  const int64_t tiles = (int64_t)a.B * a.Hkv * a.tiles;
  auto join_parts = [&](float unit) {
    return launch_in_parts((int64_t)a.B * a.Hkv * a.rows, 256, "cross attention join launch", [&](int64_t first, unsigned n) {
      a.first_block = (uint32_t)first;
      hipLaunchKernelGGL(k_cross_join<KIND>, dim3(n), dim3(256), 0, st, a, unit, c);
    });
  };
  if (shares_rows<KIND>(a)) {
    // Eight waves to a workgroup read K and V half as often; four waste less on few tiles and leave less of the chip idle:
    // (tiles of a pair, pairs), 1024 keys, eight / four: (8, 64) 21.4 / 18.2; (22, 64) 23.0 / 25.2; (8, 256) 25.9 / 27.8; (22, 480) 106 / 118.
    // On codes eight also convert them half as often: from more workgroups of four on than there are CUs, unless there are more of
    // eight than are resident at once and these idle more: (8, 120) 28.1 / 24.2, (8, 130) 28.2 / 29.9, (6, 480) 42.8 / 48.9, (9, 480) 78.4 / 66.8.
    const int64_t pairs = (int64_t)a.B * a.Hkv, fours = (a.tiles + 3) / 4, eights = (a.tiles + 7) / 8;
    const bool eight = KIND != kF32 && a.shared_parts > 1 ? fours == 2 * eights
                     : KIND == kBf16 ? a.tiles > 4 && pairs * eights >= 192
                                     : KIND == kCodes && pairs * fours > 256 && (pairs * eights <= 512 || fours == 2 * eights);
    const int nwv = eight ? 8 : 4;
    a.parts = KIND == kF32 ? 1 : a.shared_parts; a.parts_magic = magic_of(a.parts);
    a.part_ml = (float2*)((char*)a.part_o + (size_t)tiles * a.parts * kRows * 64 * 4);
    a.groups = (a.tiles + nwv - 1) / nwv * a.parts; a.groups_magic = magic_of(a.groups);
    a.by_xcd = 9 * pairs >= 8 * ((pairs + 7) / 8 * 8);         // (288 pairs of 2240 rows: 93.0 us pair by pair in turn, 91.7 so)
    const int64_t blocks = (a.by_xcd ? (pairs + 7) / 8 * 8 : pairs) * a.groups;
    if (blocks > 0x7fffffff) return fail(LITEVAR_E_UNSUPPORTED, "grid too large");
    // Workgroups that share a CU to their end: see set_priority.  (480 pairs of 256 rows on up to 512 keys 25.8 -> 25.0 us, 169 on up to 333
    // codes 19.6 -> 19.0; with more rounds new workgroups would hold up old ones: 288 pairs of 2240 rows 86.0 -> 90.2.)
    const int64_t chunks = (((int64_t)a.kv_len + kBlock - 1) / kBlock + a.parts - 1) / a.parts;
    const bool resident = blocks * nwv <= 256 * (KIND == kCodes || nwv == 8 ? 16 : KIND == kBf16 ? 12 : 8);
    a.prio_magic = KIND != kF32 && resident && chunks > 0 ? (uint32_t)((1 << 18) / chunks) : 0;
    a.by_rank = !resident && a.len && a.B > 1 && a.B <= 64;     // (a lane for each row)
    litevar_status s = launch_in_parts(blocks, nwv * 64, "cross attention launch", [&](int64_t first, unsigned n) {
      a.first_block = (uint32_t)first;
      if constexpr (KIND == kF32) {
        hipLaunchKernelGGL(k_cross_tiles_f32, dim3(n), dim3(256), 0, st, a, c);
      }
      else if (a.parts > 1) {
        if (nwv == 8) hipLaunchKernelGGL((k_cross_tiles<8, KIND, true>), dim3(n), dim3(512), 0, st, a, c);
        else hipLaunchKernelGGL((k_cross_tiles<4, KIND, true>), dim3(n), dim3(256), 0, st, a, c);
      }
      else if (nwv == 8) hipLaunchKernelGGL((k_cross_tiles<8, KIND, false>), dim3(n), dim3(512), 0, st, a, c);
      else hipLaunchKernelGGL((k_cross_tiles<4, KIND, false>), dim3(n), dim3(256), 0, st, a, c);
    });
    return s || a.parts == 1 ? s : join_parts(1.f);
  }
  if (litevar_status s = launch_in_parts(tiles * a.parts, kWaves * 64, "cross attention launch", [&](int64_t first, unsigned n) {
        a.first_block = (uint32_t)first;
        hipLaunchKernelGGL(k_cross_rows<KIND>, dim3(n), dim3(kWaves * 64), 0, st, a, c);
      })) return s;
  return a.parts == 1 ? LITEVAR_OK : join_parts(c);
}

// What both entry points check and fill; `kind` as in Kind.
litevar_status cross_attention(CrossArgs& a, Kind kind, int32_t B, int32_t H, int32_t H_kv, int32_t q_len, int32_t kv_len, int32_t D,
                               const int64_t* q_strides, const int64_t* kv_strides, const int64_t* o_strides, float sm_scale,
                               void* d_workspace, size_t workspace_bytes, void* stream) {
  if (litevar_status s = check_shape(B, H, H_kv, q_len, kv_len)) return s;
  if (D != 64) return fail(LITEVAR_E_UNSUPPORTED, "head dimension %d is not supported (only 64)", D);
  uint32_t bits;                               // (compared as bits: the build lets the compiler assume that no value is NaN)
  memcpy(&bits, &sm_scale, sizeof bits);
  if (bits == 0 || bits > 0x461c4000u)         // 1e4f; negative values, infinities and NaN are above it
    return fail(LITEVAR_E_INVALID_ARG, "sm_scale must be finite, positive and at most 1e4");
  if (litevar_status s = operand_strides(q_strides, B, H, q_len, D, a.qs)) return s;
  if (litevar_status s = operand_strides(kv_strides, B, H_kv, kv_len, D, a.ks)) return s;
  if (litevar_status s = operand_strides(o_strides, B, H, q_len, D, a.os)) return s;
  if (q_len == 0) return LITEVAR_OK;
  if (!a.q || !a.o || (kv_len > 0 && (!a.k || !a.v))) return fail(LITEVAR_E_INVALID_ARG, "q, k, v or o is NULL");
  if (a.o == a.q || (kv_len > 0 && (a.o == a.k || a.o == a.v))) return fail(LITEVAR_E_INVALID_ARG, "o aliases an input");
  if (((uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v | (uintptr_t)a.o) & 15)
    return fail(LITEVAR_E_INVALID_ARG, "q, k, v, o must be 16-byte aligned");
  if ((uintptr_t)a.len & 3) return fail(LITEVAR_E_INVALID_ARG, "lengths must be 4-byte aligned");
  size_t need = 0;
  if (litevar_status s = litevar_cross_attn_workspace_bytes(B, H, H_kv, q_len, kv_len, &need)) return s;
  if (need > 0 && !d_workspace) return fail(LITEVAR_E_INVALID_ARG, "d_workspace is NULL");
  if (workspace_bytes < need) return fail(LITEVAR_E_INVALID_ARG, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
  if (need > 0 && ((uintptr_t)d_workspace & 15)) return fail(LITEVAR_E_INVALID_ARG, "d_workspace must be 16-byte aligned");
  a.B = B; a.H = H; a.Hkv = H_kv; a.G = H / H_kv; a.q_len = q_len; a.kv_len = kv_len;
  a.rows = a.G * q_len; a.tiles = (a.rows + kRows - 1) / kRows;
  const int64_t tiles = tiles_of(B, H, H_kv, q_len);
  a.parts = parts_of(tiles, (int64_t)B * H * q_len, kv_len);
  a.shared_parts = shared_parts_of((int64_t)B * H_kv, a.tiles, kv_len);
  a.scale_blocks = (kv_len + kBlock - 1) / kBlock;
  a.q_magic = magic_of(q_len); a.tiles_magic = magic_of(a.tiles); a.hkv_magic = magic_of(H_kv); a.parts_magic = magic_of(a.parts);
  a.pairs_magic = magic_of((int64_t)B * H_kv); a.rows_magic = magic_of(a.rows);
  a.part_o = (float*)d_workspace;
  a.part_ml = (float2*)((char*)d_workspace + (size_t)tiles * a.parts * kRows * 64 * 4);
  const float c = sm_scale * 1.4426950408889634f;
  a.ks_least = std::max(0x1p-100f, 0x1p-120f / c); a.ks_most = 0x1p120f / c;   // (infinite for the smallest softmax scales)
  hipStream_t st = (hipStream_t)stream;
  if (kind == kF32) return launch<kF32>(a, c, st);
  if (kind == kCodes) return launch<kCodes>(a, c, st);
  return launch<kBf16>(a, c, st);
}

}  // namespace
}  // namespace lv

using namespace lv;

extern "C" {

litevar_status litevar_cross_attn_workspace_bytes(int32_t B, int32_t H, int32_t H_kv, int32_t q_len, int32_t kv_len,
                                                  size_t* out_bytes) {
  if (!out_bytes) return fail(LITEVAR_E_INVALID_ARG, "out_bytes is NULL");
  if (litevar_status s = check_shape(B, H, H_kv, q_len, kv_len)) return s;
  const int64_t pairs = (int64_t)B * H_kv, tiles = tiles_of(B, H, H_kv, q_len);
  const int64_t parts = std::max(parts_of(tiles, (int64_t)B * H * q_len, kv_len), shared_parts_of(pairs, tiles / pairs, kv_len));
  *out_bytes = parts > 1 ? (size_t)tiles * parts * kRows * (64 * 4 + 8) : 0;
  return LITEVAR_OK;
}

litevar_status litevar_cross_attn_fwd(const void* d_q, const void* d_k, const void* d_v, void* d_o, int32_t B, int32_t H,
                                      int32_t H_kv, int32_t q_len, int32_t kv_len, int32_t D, litevar_dtype dt,
                                      const int64_t* q_strides, const int64_t* kv_strides, const int64_t* o_strides,
                                      const int32_t* d_kv_len, float sm_scale, void* d_workspace, size_t workspace_bytes,
                                      void* stream) {
  if (dt != LITEVAR_BF16 && dt != LITEVAR_F32) return fail(LITEVAR_E_UNSUPPORTED, "unknown dtype %d", (int)dt);
  CrossArgs a{};
  a.q = d_q; a.k = d_k; a.v = d_v; a.o = d_o; a.len = d_kv_len;
  return cross_attention(a, dt == LITEVAR_F32 ? kF32 : kBf16, B, H, H_kv, q_len, kv_len, D, q_strides, kv_strides, o_strides,
                         sm_scale, d_workspace, workspace_bytes, stream);
}

litevar_status litevar_cross_attn_kv8_fwd(const void* d_q, const int8_t* d_k8, const float* d_k_scale, const int8_t* d_v8,
                                          const float* d_v_scale, void* d_o, int32_t B, int32_t H, int32_t H_kv, int32_t q_len,
                                          int32_t kv_len, int32_t D, const int64_t* q_strides, const int64_t* o_strides,
                                          const int32_t* d_kv_len, float sm_scale, void* d_workspace, size_t workspace_bytes,
                                          void* stream) {
  if (kv_len > 0 && (!d_k_scale || !d_v_scale)) return fail(LITEVAR_E_INVALID_ARG, "a scale pointer is NULL");
  if (((uintptr_t)d_k_scale | (uintptr_t)d_v_scale) & 3) return fail(LITEVAR_E_INVALID_ARG, "scales must be 4-byte aligned");
  CrossArgs a{};
  a.q = d_q; a.k = d_k8; a.v = d_v8; a.o = d_o; a.len = d_kv_len; a.k_scale = d_k_scale; a.v_scale = d_v_scale;
  return cross_attention(a, kCodes, B, H, H_kv, q_len, kv_len, D, q_strides, nullptr, o_strides, sm_scale, d_workspace,
                         workspace_bytes, stream);
}

}  // extern "C"
