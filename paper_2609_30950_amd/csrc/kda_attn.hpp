// Attention layers: launch interface, element types and the split of a
// ragged batch over its lengths (shared by the kernels and the C ABI).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/kda.h"
#include "kda_device.hpp"

namespace kda {

struct PlanArgs {
  kda_pages pg;
  int sh;                 // log2(page)
  int n_slots;
  const int32_t *lens, *newt, *n_free;
  int32_t *free_pages, *tables, *lens_out, *n_free_out, *cu, *slots, *ok;
};

struct AppendArgs {
  kda_pages pg;
  int sh, n, H, d, e4m3, f16;   // latent rows: H = 1, two parts of widths d and d2
  int d2;
  const void *a, *b;
  long long a_stride, b_stride;
  const int32_t* slots;
  const float *a_scale, *b_scale;
  void *a_cache, *b_cache;
};

struct AttnArgs {
  kda_pages pg;
  int sh, Hq, Hkv, g, mt;       // g query heads a key/value head in mt tiles of 16
  int f16, e4m3, d;
  int extra, lmin;              // split of the lengths (find_split)
  float scale2;                 // scale * log2(e)
  const void* q;
  long long q_stride;
  const void *kc, *vc;
  const int32_t *tables, *lens;
  const float *k_scale, *v_scale;
  void* o;
  float* lse;
  float *part_o, *part_ml;      // [items][Hq][d], [items][Hq][2]
  int32_t* reqs;                // [B][2]: first item and parts of a request, from the parts for the join
};

struct LatentArgs {
  kda_pages pg;
  int sh, H, dn, dr, dc, f16;
  int extra, lmin;
  float scale2;
  const void *qn, *qr;
  long long qn_stride, qn_head, qr_stride, qr_head;
  const void *w_uk, *w_uv, *cache;
  const int32_t *tables, *lens;
  void* o;
  void* qa;                     // [B][H][2 d_c + d_r]: q_n W_uk (hi, lo) and q_r
  float *part_o, *part_ml;      // [items][H][d_c], [items][H][2]
  // the split, written by the first launch: [B][2] first item and parts of a
  // request; [1 + items][4] number of items, then request, first and last + 1 token
  int32_t *reqs, *items;
};

struct LatentPrefillArgs {
  kda_pages pg;
  int sh, H, dn, dr, dc, f16, n;
  int max_kv;
  float scale2;
  const void *qn, *qr;
  long long qn_stride, qn_head, qr_stride, qr_head;
  const int32_t *cu, *tables, *lens;
  const void *w_uk, *w_uv, *cache;
  void* o;
  int kv_rows;                  // rows of the expanded arrays, a multiple of 256
  int32_t* src;                 // [kv_rows] cached row of each packed token, -1: no such page
  int32_t* lay;                 // off [B + 1], kvn [B], qoff [B + 1]
  int32_t* gone;                // [H][d_v / 32] bits of the value channels whose weights are not finite
  // f16: keys [H][kv_rows][d_n] (f16 elements: [2][H]..., hi and lo), shared parts [kv_rows][d_r], values [H][kv_rows / 8][d_v][8]
  void *ke, *re, *ve;
  int parts;                    // parts that a query tile's tokens are cut into
  // with several: [tiles][H][parts] sums of 128 rows (tiles in the launch's order), their maxima and sums of
  // weights, and [tiles][2] the rows of a tile
  float *part_o, *part_ml;
  int32_t* part_rows;
};

// Query tiles that n rows of B requests can have, and the longest request.
constexpr int PREFILL_ROWS = 128;
inline int prefill_tiles(const kda_pages& pg, int n) {
  const int requests = pg.B < n ? pg.B : n;   // sum of ceil(rows / 128) over so many requests
  return requests + (n - requests) / PREFILL_ROWS;
}
inline int prefill_longest(const kda_pages& pg, int max_kv) {
  const int64_t cap = (int64_t)pg.max_pages * pg.page;
  return cap < max_kv ? (int)cap : max_kv;
}

hipError_t launch_plan(const PlanArgs& a, hipStream_t st);
hipError_t launch_append(const AppendArgs& a, bool latent, hipStream_t st);
hipError_t launch_attn_step(const AttnArgs& a, hipStream_t st);
hipError_t launch_latent_step(const LatentArgs& a, hipStream_t st);
hipError_t launch_latent_prefill(const LatentPrefillArgs& a, hipStream_t st);

// Items a split into B + extra parts may have (find_split).
inline int split_extra(int per_item_blocks, int target) {
  const int e = (target + per_item_blocks - 1) / per_item_blocks;
  return e < 1 ? 1 : e;
}

// --------------------------------------------------------- element types ---
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

// Two floats as packed 16-bit values, round to nearest even.
template <int F16>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const f32x2_t x = {a, b};
  if constexpr (F16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, f16x2_t));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2_t));
}

template <int F16>
__device__ __forceinline__ float lo_f32(uint32_t w) {
  if constexpr (F16) return (float)__builtin_bit_cast(f16x2_t, w)[0];
  return __builtin_bit_cast(float, w << 16);
}
template <int F16>
__device__ __forceinline__ float hi_f32(uint32_t w) {
  if constexpr (F16) return (float)__builtin_bit_cast(f16x2_t, w)[1];
  return __builtin_bit_cast(float, w & 0xFFFF0000u);
}

// D += A B for 16x16 tiles, K = 32: lane l supplies row l % 16 of A and
// column l % 16 of B, each at k = 8 (l / 16) .. + 7; it receives rows
// 4 (l / 16) + r of column l % 16.
template <int F16>
__device__ __forceinline__ f32x4 mma16(uint4 a, uint4 b, f32x4 c) {
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a),
                                                  __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a),
                                                 __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// The same for 32x32 tiles, K = 16, in f16: lane l supplies row l % 32 of A and
// column l % 32 of B at k = 8 (l / 32) .. + 7; register 4 i + r of the result
// is row 8 i + 4 (l / 32) + r of column l % 32.
typedef float f32x16 __attribute__((ext_vector_type(16)));
__device__ __forceinline__ f32x16 mma32_f16(uint4 a, uint4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a),
                                                __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
}

// 16 bytes per lane from memory into LDS without passing registers; `to` is
// uniform over the wave, lane l's bytes land at to + 16 l.  A later read of
// that LDS waits for the wave's own copies only: wait_copies(), then a
// barrier.  Buffers that take turns are separate LDS variables, since the
// compiler makes a read wait for every copy in flight to the same variable.
__device__ __forceinline__ void copy16(const void* from, void* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                   (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}
__device__ __forceinline__ void wait_copies() { __builtin_amdgcn_s_waitcnt(0x0F70); }   // vmcnt(0)

// All but the wave's N latest requests (N < 16).
template <int N>
__device__ __forceinline__ void wait_copies_but() { __builtin_amdgcn_s_waitcnt(0x0F70 | N); }

// Barrier for what the waves exchange through LDS while copies into other LDS
// are in flight (__syncthreads would wait for those too).
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Wave-uniform load of an input that nothing writes meanwhile, through the
// scalar cache (the compiler takes that path by itself only for memory that
// it knows to be unwritten).
__device__ __forceinline__ int32_t load_uniform(const int32_t* p) {
  return *(const __attribute__((address_space(4))) int32_t*)p;
}

constexpr float NEG_INF = -__builtin_huge_valf();

__device__ __forceinline__ float exp2_f(float x) { return __builtin_amdgcn_exp2f(x); }

// Weight of a score d octaves below its reference.  Weights that meet the
// values in f16 are formed 2^15 too large, and with them the sums that divide
// the result: between 2^15 and f16's smallest number lie forty octaves instead
// of twenty-five, so that a great many small weights beside a large one keep
// their bits (relative 2^-11 down to 2^-29 of the largest, 2^-40 of it below).
template <int F16>
constexpr float STEP_SHIFT = F16 ? 15.f : 0.f;
template <int F16>
__device__ __forceinline__ float step_weight(float d) {
  if constexpr (F16) return exp2_f(d + STEP_SHIFT<F16>);
  return exp2_f(d);
}

// Maximum and sum over the four lanes l % 16 + 16 i (the token groups of a
// column of an MFMA result).
__device__ __forceinline__ float max_groups(float v) {
  uint32_t u = __builtin_bit_cast(uint32_t, v);
  auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  v = fmaxf(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]));
  u = __builtin_bit_cast(uint32_t, v);
  auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)b[0]), __builtin_bit_cast(float, (uint32_t)b[1]));
}
__device__ __forceinline__ float sum_groups(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// ------------------------------------------------- packed lists of requests ---
// Sums of counts saturate at 2^31 - 1: every count that matters is compared
// with less.
__device__ __forceinline__ int add_sat(int a, int b) { return __builtin_elementwise_add_sat(a, b); }

__device__ __forceinline__ int wave_incl_scan_sat(int v) {
  v = add_sat(v, dpp_add_src<0x111, 0xF>(v));
  v = add_sat(v, dpp_add_src<0x112, 0xF>(v));
  v = add_sat(v, dpp_add_src<0x114, 0xF>(v));
  v = add_sat(v, dpp_add_src<0x118, 0xF>(v));
  v = add_sat(v, dpp_add_src<0x142, 0xA>(v));
  v = add_sat(v, dpp_add_src<0x143, 0xC>(v));
  return v;
}

// Sum of the other threads' values before this one's, and the total; `part`
// has one slot per wave, used once.
template <int NT>
__device__ __forceinline__ int block_before(int v, int* part, int& total) {
  constexpr int NW = NT / WAVE;
  const int w = threadIdx.x / WAVE, lane = lane_id();
  const int upto = wave_incl_scan_sat(v);
  if (lane == WAVE - 1) part[w] = upto;
  const int left = __shfl_up(upto, 1);
  __syncthreads();
  int before = lane ? left : 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    if (i < w) before = add_sat(before, part[i]);
    total = add_sat(total, part[i]);
  }
  return before;
}

// Last index whose (not decreasing) offset is at most i[k]: the request that
// holds item i[k] of a packed list, whatever empty requests stand beside it.
// N bisections side by side, in ceil(log2 B) steps.
template <int N>
__device__ __forceinline__ void owners(const int* off, int B, const int (&i)[N], int (&at)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) at[k] = 0;
  for (int step = B > 1 ? 1 << (31 - __builtin_clz(B - 1)) : 0; step > 0; step >>= 1)
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int to = min(at[k] + step, B - 1);
      at[k] = off[to] <= i[k] ? max(at[k], to) : at[k];
    }
}
__device__ __forceinline__ int owner(const int* off, int B, int i) {
  const int x[1] = {i};
  int at[1];
  owners<1>(off, B, x, at);
  return at[0];
}

// ------------------------------------------------------ split of lengths ---
// A ragged batch is cut into items of at most L tokens, so that one long
// request does not hold the chip: L is a multiple of 64, at least lmin, with
// sum(ceil(len / 64)) 64 / L <= extra, which keeps the items within B + extra
// (the grid) whatever the lengths are.  A request without tokens is one item
// (it writes the zeros).  A wave finds an item by itself from the lengths:
// each lane holds ceil(B / 64) consecutive requests.  Lengths are below 2^26
// (SPLIT_MAX_LEN), which keeps the float32 quotients below exact after floor.
// These are a kernel's first instructions and come from a cold instruction
// cache, so they are few (the integer divisions and 64-bit sums of an earlier
// form took 9 600 cycles of a join's 21 000).
constexpr int SPLIT_MAX_LEN = 1 << 26;

struct Split {
  int b, s, ns, first, len, L;   // request, part, parts, its first item, tokens, tokens a part
};

__device__ __forceinline__ int cut_len(int x, int cap) { return x < 0 ? 0 : (x > cap ? cap : x); }

// Sum over the wave, the same in every wave (fixed order).
__device__ __forceinline__ float wave_sum_uniform(float v) {
  v += dpp_f<0xB1>(v);
  v += dpp_f<0x4E>(v);
  v += dpp_f<0x141>(v);
  v += dpp_f<0x140>(v);
  return (bcast_f(v, 0) + bcast_f(v, 16)) + (bcast_f(v, 32) + bcast_f(v, 48));
}

// Units of 64 tokens a part, from the sum of the requests' units.  Up to 2^20
// the sum and the rounded quotient's ceiling are exact; past that the margin
// covers the rounding of the sum.
__device__ __forceinline__ float split_units(float units, int extra, int lmin) {
  const float q = ceilf(units / (float)extra);
  float k = units > 1048576.f ? q + 1.f + floorf(q * (1.f / 1024.f)) : q;
  k = fminf(k, (float)(SPLIT_MAX_LEN / 64));
  return fmaxf(k, (float)(lmin / 64));
}
// Parts of a request of u units: ceil(u / k), at least one.  (u + k - 1/2) / k
// lies at least 1 / (2 k) from an integer, more than the quotient's error.
__device__ __forceinline__ int split_parts(float u, float k, float rk) {
  return (int)fmaxf(floorf((u + k - 0.5f) * rk), 1.f);
}
__device__ __forceinline__ float units_of(int len) { return (float)((len + 63) >> 6); }

// Requests of lane `lane` and their number of parts in a whole wave; f(b, len,
// parts, first item) is called for each request by its lane.
template <typename F>
__device__ __forceinline__ int split_all(const int32_t* lens, int B, int cap, int extra, int lmin, int& L, F f) {
  const int lane = lane_id(), R = (B + WAVE - 1) / WAVE;
  int len0 = 0;
  float units = 0.f;
  for (int r = 0; r < R; ++r) {
    const int b = lane * R + r;
    if (b < B) {
      len0 = cut_len(lens[b], cap);
      units += units_of(len0);
    }
  }
  const float k = split_units(wave_sum_uniform(units), extra, lmin);
  const float rk = 1.f / k;
  L = __builtin_amdgcn_readfirstlane(64 * (int)k);
  int first = 0;
  if (R == 1) {
    const int n = lane < B ? split_parts(units, k, rk) : 0, upto = wave_incl_scan(n);
    if (lane < B) f(lane, len0, n, upto - n);
    return __builtin_amdgcn_readlane(upto, WAVE - 1);
  }
  int sum = 0;
  for (int r = 0; r < R; ++r) {
    const int b = lane * R + r;
    if (b < B) sum += split_parts(units_of(cut_len(lens[b], cap)), k, rk);
  }
  const int upto = wave_incl_scan(sum);
  first = upto - sum;
  for (int r = 0; r < R; ++r) {
    const int b = lane * R + r;
    if (b < B) {
      const int len = cut_len(lens[b], cap), n = split_parts(units_of(len), k, rk);
      f(b, len, n, first);
      first += n;
    }
  }
  return __builtin_amdgcn_readlane(upto, WAVE - 1);
}

// The item `want`; false if there is no such item.  Called by whole waves with
// a uniform value.
__device__ __forceinline__ bool find_split(const int32_t* lens, int B, int cap, int extra, int lmin,
                                           int want, Split& out) {
  bool mine = false;
  int fb = 0, fs = 0, fn = 0, ff = 0, fl = 0, L;
  split_all(lens, B, cap, extra, lmin, L, [&](int b, int len, int n, int first) {
    if (want >= first && want < first + n) {
      mine = true;
      fb = b;
      fs = want - first;
      fn = n;
      ff = first;
      fl = len;
    }
  });
  const unsigned long long who = __ballot(mine);
  if (who == 0) return false;
  const int src = __ffsll((long long)who) - 1;
  out.b = __builtin_amdgcn_readlane(fb, src);
  out.s = __builtin_amdgcn_readlane(fs, src);
  out.ns = __builtin_amdgcn_readlane(fn, src);
  out.first = __builtin_amdgcn_readlane(ff, src);
  out.len = __builtin_amdgcn_readlane(fl, src);
  out.L = L;
  return true;
}

}  // namespace kda
