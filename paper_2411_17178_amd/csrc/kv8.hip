// K and V rows in 8 bits with one scale per block of 64 tokens and head: storing, loading back, and the windowed
// attention that reads such a cache.
//   store   s = max |x| / 127 over a block's rows (64 x 64 values), code = rne(x / s) within +-127, s = 0 -> codes 0
//   load    bf16(s * code)
// A cache is cut into segments (the scales of a sequence) and a segment into blocks counted from its first token,
// so that no block spans two of them: what one generation step stores never changes what an earlier one has stored.
// Codes are decided in binary32: s and x / s are the correctly rounded quotients.
#include "attn_bf16_common.h"

namespace lv {
namespace {

constexpr int kBlock = LITEVAR_KV8_BLOCK;
constexpr int kWaves = 4;                      // per workgroup, each with a block of its own

struct Blocks {                                // the blocks that a launch visits, and where their rows are
  int B, H;
  int n_seg;                                   // segments visited
  int n_blocks, total_blocks;                  // blocks visited, of the whole cache
  int len;                                     // tokens of the whole cache
  uint32_t blocks_magic, H_magic;              // floor(2^32 / n), see divmod_by
  uint32_t first_block;                        // of this launch: see launch_in_parts
  int off[kMaxScales + 1];                     // first token of the i-th visited segment, end of the last
  int first[kMaxScales + 1];                   // its first block
};

struct StoreArgs {
  Blocks w;
  const void* x[2]; int64_t xs[3];             // K and V rows, strides (B, H, token) in elements
  int8_t* codes[2]; float* scale[2];
  const int32_t* valid;                        // [B] tokens that count, or nullptr
};

struct LoadArgs {
  Blocks w;
  const int8_t* codes[2]; const float* scale[2];
  unsigned short* out[2];
};

struct Block { int b, bh, h, index, token, rows; };

// Block of this wave: item = (pair x visited blocks + block) x 2 + tensor.  false: none.
__device__ inline bool my_block(const Blocks& w, int& tensor, Block& k) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t item = (w.first_block + blockIdx.x) * kWaves + wave;
  tensor = item & 1;
  int in_pair;
  divmod_by(item >> 1, (uint32_t)w.n_blocks, w.blocks_magic, k.bh, in_pair);
  if (k.bh >= w.B * w.H) return false;
  divmod_by((uint32_t)k.bh, (uint32_t)w.H, w.H_magic, k.b, k.h);
  // (lane i holds segment i's numbers and a ballot finds the segment)
  const int i = min(lane, kMaxScales), off = w.off[i], first = w.first[i];
  k.index = __builtin_amdgcn_readlane(first, 0) + in_pair;
  // (segments without tokens share their first block with the next one: the last that begins here or before)
  const int seg = __builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < w.n_seg && first <= k.index)) - 1;
  k.token = __builtin_amdgcn_readlane(off, seg) + kBlock * (k.index - __builtin_amdgcn_readlane(first, seg));
  k.rows = min(kBlock, __builtin_amdgcn_readlane(off, seg + 1) - k.token);
  return true;
}

// Eight values of a row as they lie in memory.
template <typename T> struct Eight;
template <> struct Eight<__bf16> {
  u32x4 w;
  __device__ void load(const __bf16* p) { w = *(const u32x4*)p; }
  __device__ float operator[](int e) const { return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16); }
};
template <> struct Eight<float> {
  u32x4 w[2];
  __device__ void load(const float* p) { w[0] = ((const u32x4*)p)[0]; w[1] = ((const u32x4*)p)[1]; }
  __device__ float operator[](int e) const { const unsigned u = w[e >> 2][e & 3]; return __uint_as_float(u); }
};

// The largest magnitude, as the bits of a float.  Magnitudes compare as integers, in which infinity and NaN are the largest.
template <typename T> struct Largest;
template <> struct Largest<__bf16> {
  typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
  u16x2 top = {0, 0};                          // (of the words' two halves)
  __device__ void add(const Eight<__bf16>& x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned m = x.w[i] & 0x7fff7fffu;
      top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, m));
    }
  }
  __device__ unsigned bits() const { return (unsigned)max(top.x, top.y) << 16; }
};
template <> struct Largest<float> {
  unsigned top = 0;
  __device__ void add(const Eight<float>& x) {
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
  }
  __device__ unsigned bits() const { return top; }
};

}  // namespace

// A wave per block and tensor: eight lanes per row, eight rows per load, all loads of the block in flight before the
// first is used; the largest magnitude goes across the wave in registers, so that nothing is read twice and no
// barrier is needed.  Bound: memory.  480 pairs x 256 bf16 rows 11.8 us (4.0 TB/s, start and tail of
// the launch included); x up to 333 fp32 rows 15.4 us (4.7 TB/s).
template <typename T>
__global__ __launch_bounds__(kWaves * 64) void k_kv8_store(StoreArgs a) {
  int tensor;
  Block k;
  if (!my_block(a.w, tensor, k)) return;
  const int lane = threadIdx.x & 63, row8 = lane >> 3, part = lane & 7;
  int rows = k.rows;
  if (a.valid) rows = min(rows, max(a.valid[k.b], 0) - k.token);   // (a difference that 32 bits hold)
  if (rows <= 0) return;                       // (rows behind the last valid one keep what they hold)
  const T* x = (const T*)(tensor ? a.x[1] : a.x[0]) + k.b * a.xs[0] + k.h * a.xs[1] + (k.token - a.w.off[0]) * a.xs[2] + 8 * part;
  Eight<T> v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (8 * i < rows) v[i].load(x + min(8 * i + row8, rows - 1) * a.xs[2]);
  Largest<T> largest;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (8 * i < rows) largest.add(v[i]);
  unsigned top = largest.bits();
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = max(top, (unsigned)__shfl_xor((int)top, d));
  constexpr unsigned kInf = 0x7f800000u;       // (a block that holds such a value or a NaN is left without codes)
  const float s = top < kInf ? __fdiv_rn(__uint_as_float(top), 127.0f) : 0.f;
  const int64_t row0 = (int64_t)k.bh * a.w.len + k.token;
  int8_t* out = (tensor ? a.codes[1] : a.codes[0]) + (row0 + row8) * 64 + 8 * part;
  // The correctly rounded quotient without a division: x / s by the reciprocal of s, corrected by its exact remainder
  // twice.  Holds while nothing overflows or loses bits, for which s is kept between 2^-100 and 2^100 (|x / s| <= 128; a
  // remainder that underflows belongs to a quotient that rounds to 0 either way).  Other blocks divide.
  const bool plain = s >= 0x1p-100f && s <= 0x1p100f;
  const float r = plain ? __fdiv_rn(1.0f, s) : 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (8 * i >= rows) break;
    unsigned word[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      unsigned u[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float d = v[i][4 * half + e];
        float q;
        if (plain) {
          q = __fmul_rn(d, r);
          q = __fmaf_rn(__fmaf_rn(-q, s, d), r, q);
          q = __fmaf_rn(__fmaf_rn(-q, s, d), r, q);
        } else {
          q = s > 0.f ? fminf(fmaxf(__fdiv_rn(d, s), -127.f), 127.f) : 0.f;
        }
        u[e] = __float_as_uint(__fadd_rn(q, 0x1.8p23f));   // rounds to the nearest even integer, its two's complement in the low bits
      }
      word[half] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(u[3], u[2], 0x0c0c0400u),
                                         __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u), 0x05040100u);
    }
    if (8 * i + row8 < rows) *(uint2*)(out + 8 * i * 64) = make_uint2(word[0], word[1]);
  }
  if (lane == 0)
    ((unsigned*)(tensor ? a.scale[1] : a.scale[0]))[(int64_t)k.bh * a.w.total_blocks + k.index] =
        top < kInf ? __float_as_uint(s) : top == kInf ? kInf : 0x7fc00000u;
}

// Codes -> rows [B][H][len][64] of bf16, or of f16 times the head's power of two (see HeadScales; every wave forms it
// from the scales of all visited blocks); a wave per block and tensor.  Bound: memory; 288 pairs x 2240 rows 41 us, the copy rate.
template <bool F16>
__global__ __launch_bounds__(kWaves * 64) void k_kv8_load(LoadArgs a) {
  int tensor;
  Block k;
  if (!my_block(a.w, tensor, k)) return;
  const int lane = threadIdx.x & 63, row8 = lane >> 3, part = lane & 7;
  const float* scales = (tensor ? a.scale[1] : a.scale[0]) + (int64_t)k.bh * a.w.total_blocks;
  const int64_t at = ((int64_t)k.bh * a.w.len + k.token) * 64 + 8 * part;
  const int8_t* codes = (tensor ? a.codes[1] : a.codes[0]) + at;
  unsigned short* out = (tensor ? a.out[1] : a.out[0]) + at;
  uint2 c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (8 * i < k.rows) c[i] = *(const uint2*)(codes + min(8 * i + row8, k.rows - 1) * 64);
  float s = scales[k.index];
  if constexpr (F16) {
    HeadScales head;
    for (int i = lane; i < a.w.n_blocks; i += 64) head.add(scales[a.w.first[0] + i]);
    head.join();
    s = ldexpf(nan_unless_finite(s), head.power());
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (8 * i >= k.rows) break;
    using T = std::conditional_t<F16, _Float16, __bf16>;
    typedef __attribute__((ext_vector_type(8))) T T8;
    T8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (T)(s * (float)((int)((e < 4 ? c[i].x : c[i].y) << (24 - 8 * (e & 3))) >> 24));
    if (8 * i + row8 < k.rows) *(T8*)(out + (8 * i + row8) * 64) = r;
  }
}

namespace {

// The segments' first tokens and blocks, [n + 1] each.
litevar_status segment_tables(const int32_t* len, int32_t n, int64_t (&off)[kMaxScales + 1], int64_t (&first)[kMaxScales + 1]) {
  if (!len) return fail(LITEVAR_E_INVALID_ARG, "segments is NULL");
  if (n < 1 || n > kMaxScales) return fail(LITEVAR_E_INVALID_ARG, "n_segments must be in 1..%d (got %d)", kMaxScales, n);
  off[0] = first[0] = 0;
  for (int i = 0; i < n; ++i) {
    if (len[i] < 0) return fail(LITEVAR_E_INVALID_ARG, "segments[%d] = %d is negative", i, len[i]);
    off[i + 1] = off[i] + len[i];
    first[i + 1] = first[i] + ((int64_t)len[i] + kBlock - 1) / kBlock;
  }
  if (off[n] >= ((int64_t)1 << 31) - kBlock) return fail(LITEVAR_E_UNSUPPORTED, "a cache of 2^31 tokens or more");
  return LITEVAR_OK;
}

// What the blocks of the segments [begin, end) need; w.n_blocks may come out as 0.
litevar_status make_blocks(const int32_t* segments, int32_t n, int32_t begin, int32_t end, int32_t B, int32_t H, Blocks& w) {
  int64_t off[kMaxScales + 1], first[kMaxScales + 1];
  if (litevar_status s = segment_tables(segments, n, off, first)) return s;
  if (begin < 0 || end > n || begin >= end)
    return fail(LITEVAR_E_INVALID_ARG, "segments [%d, %d) are not a range of the cache's %d", begin, end, n);
  if (B < 1 || H < 1) return fail(LITEVAR_E_INVALID_ARG, "B and H must be positive (got %d, %d)", B, H);
  if ((int64_t)B * H > (1 << 24)) return fail(LITEVAR_E_UNSUPPORTED, "B*H above 2^24");
  w = Blocks{};
  w.B = B; w.H = H; w.n_seg = end - begin;
  w.n_blocks = (int)(first[end] - first[begin]); w.total_blocks = (int)first[n]; w.len = (int)off[n];
  if ((int64_t)B * H * w.n_blocks * 2 >= ((int64_t)1 << 32) - 64) return fail(LITEVAR_E_UNSUPPORTED, "more than 2^32 blocks in a call");
  w.blocks_magic = (uint32_t)(((uint64_t)1 << 32) / (uint64_t)(w.n_blocks > 1 ? w.n_blocks : 1) - (w.n_blocks <= 1));
  w.H_magic = (uint32_t)(((uint64_t)1 << 32) / (uint64_t)H - (H <= 1));
  for (int i = 0; i <= kMaxScales; ++i) {
    const int at = begin + i < end ? begin + i : end;
    w.off[i] = (int)off[at]; w.first[i] = (int)first[at];
  }
  return LITEVAR_OK;
}

template <class Launch>
litevar_status launch_blocks(Blocks& w, const char* what, Launch launch) {
  if (w.n_blocks == 0) return LITEVAR_OK;
  const int64_t blocks = ((int64_t)w.B * w.H * w.n_blocks * 2 + kWaves - 1) / kWaves;
  return launch_in_parts(blocks, kWaves * 64, what, [&](int64_t first, unsigned n) {
    w.first_block = (uint32_t)first;
    launch(n);
  });
}

// How a plan's cache is read.  Plans whose bf16 calls run 32 queries per wave do so here too: with the codes converted in
// the attention kernel, once per group that streams a row, or from a copy that is converted once; plans of smaller groups,
// and handles that ask for sixteen waves, gather codes step by step.
// Rows streamed over rows seen, in the kernel / through a copy, us: 1.04 (480 pairs, 256 queries on 680) 28.9 / 54; 2.06 (288, 1024
// on 2240) 110.8 / 127.4; 2.74 (288, 2240, radius 1) 140.1 / 163.9; 3.01 (480, 680) 106.6 / 106.9; 3.17 (288, 2240, radius 2) 166.6 / 179.9;
// 3.57 (radius 3) 187.2 / 197.0; 4.06 (radius 4) 216.6 / 213.5, of 36 pairs 43.3 / 44.2; between 3 and 4 neither is ahead by more than 8 %.
enum Route { kGather, kInKernel, kCopy };
Route route_of(const litevar_plan* plan) {
  if (plan->waves_per_group != 16 || plan->patches_per_wave == 1 || (int64_t)plan->kv_len * 128 >= ((int64_t)1 << 31)) return kGather;
  int64_t seen = 0;
  for (int k = 0; k < plan->q_scale_end; ++k) seen += (int64_t)plan->scales[k] * plan->scales[k];
  const int64_t streamed = plan->n_union_keys / (plan->n_head_groups > 0 ? plan->n_head_groups : 1);
  return streamed <= 3 * seen ? kInKernel : kCopy;
}

}  // namespace

// (the stride of an axis with one entry is never used, and is what it is)
litevar_status operand_strides(const int64_t* s, int B, int heads, int64_t n, int D, int64_t (&out)[3]) {
  if (!s) { out[2] = D; out[1] = n * D; out[0] = heads * n * D; return LITEVAR_OK; }
  out[0] = B > 1 ? s[0] : 0; out[1] = heads > 1 ? s[1] : 0; out[2] = n > 1 ? s[2] : D;
  if (out[2] < D || out[2] % 8 || out[1] < 0 || out[0] < 0 || out[1] % 8 || out[0] % 8)
    return fail(LITEVAR_E_INVALID_ARG, "strides must be non-negative multiples of 8 with token stride >= D");
  return LITEVAR_OK;
}

}  // namespace lv

using namespace lv;

extern "C" {

litevar_status litevar_kv8_blocks(const int32_t* segments, int32_t n_segments, int64_t* out_first) {
  if (!out_first) return fail(LITEVAR_E_INVALID_ARG, "out_first is NULL");
  int64_t off[kMaxScales + 1], first[kMaxScales + 1];
  if (litevar_status s = segment_tables(segments, n_segments, off, first)) return s;
  for (int i = 0; i <= n_segments; ++i) out_first[i] = first[i];
  return LITEVAR_OK;
}

litevar_status litevar_kv8_store(const int32_t* segments, int32_t n_segments, int32_t segment_begin, int32_t segment_end,
                                 const void* d_k, const void* d_v, litevar_dtype dt, const int64_t* kv_strides, int32_t B,
                                 int32_t H, int32_t D, const int32_t* d_len, int8_t* d_k8, float* d_k_scale, int8_t* d_v8,
                                 float* d_v_scale, void* stream) {
  StoreArgs a{};
  if (D != 64) return fail(LITEVAR_E_UNSUPPORTED, "rows of %d values are not supported (only 64)", D);
  if (dt != LITEVAR_BF16 && dt != LITEVAR_F32) return fail(LITEVAR_E_UNSUPPORTED, "unknown dtype %d", (int)dt);
  if (litevar_status s = make_blocks(segments, n_segments, segment_begin, segment_end, B, H, a.w)) return s;
  const int64_t n = a.w.off[a.w.n_seg] - a.w.off[0];
  if (litevar_status s = operand_strides(kv_strides, B, H, n, D, a.xs)) return s;
  if (n == 0) return LITEVAR_OK;
  if (!d_k || !d_v || !d_k8 || !d_k_scale || !d_v8 || !d_v_scale) return fail(LITEVAR_E_INVALID_ARG, "a pointer is NULL");
  if (((uintptr_t)d_k | (uintptr_t)d_v | (uintptr_t)d_k8 | (uintptr_t)d_v8) & 15)
    return fail(LITEVAR_E_INVALID_ARG, "rows and codes must be 16-byte aligned");
  if (((uintptr_t)d_k_scale | (uintptr_t)d_v_scale | (uintptr_t)d_len) & 3)
    return fail(LITEVAR_E_INVALID_ARG, "scales and lengths must be 4-byte aligned");
  a.x[0] = d_k; a.x[1] = d_v; a.codes[0] = d_k8; a.codes[1] = d_v8; a.scale[0] = d_k_scale; a.scale[1] = d_v_scale;
  a.valid = d_len;
  return launch_blocks(a.w, "8-bit cache store", [&](unsigned n_wg) {
    if (dt == LITEVAR_BF16) hipLaunchKernelGGL(k_kv8_store<__bf16>, dim3(n_wg), dim3(kWaves * 64), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL(k_kv8_store<float>, dim3(n_wg), dim3(kWaves * 64), 0, (hipStream_t)stream, a);
  });
}

litevar_status litevar_kv8_load(const int32_t* segments, int32_t n_segments, int32_t segment_begin, int32_t segment_end,
                                const int8_t* d_k8, const float* d_k_scale, const int8_t* d_v8, const float* d_v_scale,
                                int32_t B, int32_t H, int32_t D, void* d_k_bf16, void* d_v_bf16, void* stream) {
  LoadArgs a{};
  if (D != 64) return fail(LITEVAR_E_UNSUPPORTED, "rows of %d values are not supported (only 64)", D);
  if (litevar_status s = make_blocks(segments, n_segments, segment_begin, segment_end, B, H, a.w)) return s;
  if (a.w.n_blocks == 0) return LITEVAR_OK;
  if (!d_k8 || !d_k_scale || !d_v8 || !d_v_scale || !d_k_bf16 || !d_v_bf16) return fail(LITEVAR_E_INVALID_ARG, "a pointer is NULL");
  if (((uintptr_t)d_k8 | (uintptr_t)d_v8 | (uintptr_t)d_k_bf16 | (uintptr_t)d_v_bf16) & 15)
    return fail(LITEVAR_E_INVALID_ARG, "rows and codes must be 16-byte aligned");
  if (((uintptr_t)d_k_scale | (uintptr_t)d_v_scale) & 3) return fail(LITEVAR_E_INVALID_ARG, "scales must be 4-byte aligned");
  a.codes[0] = d_k8; a.codes[1] = d_v8; a.scale[0] = d_k_scale; a.scale[1] = d_v_scale;
  a.out[0] = (unsigned short*)d_k_bf16; a.out[1] = (unsigned short*)d_v_bf16;
  return launch_blocks(a.w, "8-bit cache load", [&](unsigned n_wg) {
    hipLaunchKernelGGL(k_kv8_load<false>, dim3(n_wg), dim3(kWaves * 64), 0, (hipStream_t)stream, a);
  });
}

litevar_status litevar_windowed_attn_kv8_workspace_bytes(const litevar_plan* plan, int32_t B, int32_t H, size_t* out_bytes) {
  if (!plan || !out_bytes) return fail(LITEVAR_E_INVALID_ARG, "plan or out_bytes is NULL");
  if (B < 1 || H < 1) return fail(LITEVAR_E_INVALID_ARG, "B and H must be positive");
  *out_bytes = route_of(plan) == kCopy ? (size_t)B * H * 2 * (size_t)plan->kv_len * 64 * 2 : 0;
  return LITEVAR_OK;
}

litevar_status litevar_windowed_attn_kv8_fwd(const litevar_plan* plan, const void* d_q, const int8_t* d_k8, const float* d_k_scale,
                                             const int8_t* d_v8, const float* d_v_scale, void* d_o, int32_t B, int32_t H,
                                             int32_t D, const int64_t* q_strides, const int64_t* o_strides, float sm_scale,
                                             const uint8_t* d_cfg_share, uint32_t flags, void* d_workspace,
                                             size_t workspace_bytes, void* stream) {
  if (!d_q || !d_k8 || !d_k_scale || !d_v8 || !d_v_scale || !d_o) return fail(LITEVAR_E_INVALID_ARG, "a pointer is NULL");
  AttnArgs a;
  if (litevar_status s = make_attn_args(plan, B, H, D, sm_scale, d_cfg_share, flags, a)) return s;
  size_t need = 0;
  if (litevar_status s = litevar_windowed_attn_kv8_workspace_bytes(plan, B, H, &need)) return s;
  if (need > 0 && !d_workspace) return fail(LITEVAR_E_INVALID_ARG, "d_workspace is NULL");
  if (workspace_bytes < need) return fail(LITEVAR_E_INVALID_ARG, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
  if (need > 0 && ((uintptr_t)d_workspace & 255)) return fail(LITEVAR_E_INVALID_ARG, "d_workspace must be 256-byte aligned");
  if (litevar_status s = operand_strides(q_strides, B, H, plan->q_len, D, a.qs)) return s;
  if (litevar_status s = operand_strides(o_strides, B, H, plan->q_len, D, a.os)) return s;
  if (d_o == d_q) return fail(LITEVAR_E_INVALID_ARG, "o aliases an input");
  if (((uintptr_t)d_q | (uintptr_t)d_k8 | (uintptr_t)d_v8 | (uintptr_t)d_o) & 15)
    return fail(LITEVAR_E_INVALID_ARG, "q, o and the codes must be 16-byte aligned");
  if (((uintptr_t)d_k_scale | (uintptr_t)d_v_scale) & 3) return fail(LITEVAR_E_INVALID_ARG, "scales must be 4-byte aligned");
  a.q = d_q; a.k = d_k8; a.v = d_v8; a.o = d_o;
  a.ks[2] = 64; a.ks[1] = (int64_t)plan->kv_len * 64; a.ks[0] = a.ks[1] * H;
  KV8Scales scales{};
  scales.k = d_k_scale; scales.v = d_v_scale;
  int off = 0, first = 0;
  for (int k = 0; k <= kMaxScales; ++k) {
    scales.off[k] = off; scales.shift[k] = kBlock * first - off;
    const int n = k < plan->n_scales ? plan->scales[k] * plan->scales[k] : 0;
    off += n; first += (n + kBlock - 1) / kBlock;
  }
  scales.n_blocks = first;
  scales.n_seen = (scales.shift[plan->q_scale_end] + scales.off[plan->q_scale_end]) / kBlock;
  scales.k8 = d_k8; scales.v8 = d_v8;
  const Route route = route_of(plan);
  if (route == kGather) return launch_attn_kv8(plan, a, scales, (hipStream_t)stream);
  if (route == kInKernel) return launch_attn_kv8_pair(plan, a, scales, true, (hipStream_t)stream);
  int32_t seg[kMaxScales];
  for (int k = 0; k < plan->n_scales; ++k) seg[k] = plan->scales[k] * plan->scales[k];
  LoadArgs copy{};
  if (litevar_status s = make_blocks(seg, plan->n_scales, 0, plan->q_scale_end, B, H, copy.w)) return s;
  copy.codes[0] = d_k8; copy.codes[1] = d_v8; copy.scale[0] = d_k_scale; copy.scale[1] = d_v_scale;
  copy.out[0] = (unsigned short*)d_workspace; copy.out[1] = copy.out[0] + (int64_t)B * H * plan->kv_len * 64;
  if (litevar_status s = launch_blocks(copy.w, "8-bit cache copy", [&](unsigned n_wg) {
        hipLaunchKernelGGL(k_kv8_load<true>, dim3(n_wg), dim3(kWaves * 64), 0, (hipStream_t)stream, copy);
      })) return s;
  a.k = copy.out[0]; a.v = copy.out[1];
  return launch_attn_kv8_pair(plan, a, scales, false, (hipStream_t)stream);
}

}  // extern "C"
