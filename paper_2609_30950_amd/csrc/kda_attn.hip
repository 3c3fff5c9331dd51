// Grouped-query attention of one new token per request over paged keys and
// values (kda_attn_step).
//
//   o_h = sum_t p_t v_t,  p = softmax(scale q_h k_t)
//
// Every cached row is read once and used by the g = H_q / H_kv query heads of
// its head, 4 g d operations for 4 d bytes (16-bit cache), so HBM bounds it
// for every g here as long as the products run on the matrix cores: one block
// per (part of a request, key/value head), four waves that take 32 tokens in
// turn.  Both products are formed transposed, S^T = K Q^T and O^T = V^T P^T,
// with the query heads as the 16 columns.  The rows of K in tile ti are the
// tokens 8 (m / 4) + 4 ti + m % 4, so that a lane's eight scores are those of
// eight consecutive tokens: exactly what it has to supply as the second
// operand of O^T.  With V stored eight tokens of a channel together, keys,
// probabilities and values all go from memory to the matrix cores in
// registers, without LDS.  The softmax is the running one (maximum and sum in
// float32, one pass); waves and parts are joined by their maxima and sums,
// which carry the factor of STEP_SHIFT with f16 elements.  The weights meet the
// values in 16 bits, their sum is float32.  As pairs hi + lo they would bring the
// error of 64 requests up to 8192 tokens in bf16 from 1.77e-3 to 1.66e-3, the
// output's own rounding; an infinite value, of which a lo part makes NaN, then
// needs a second pass over the part, and one request of 130000 tokens and a head
// takes 24 us for 20.3 (the batch 142.7 for 141.9).

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kda_attn.hpp"
#include "kda_profile.hpp"

namespace kda {

namespace {

// Eight elements of the cache as 16-bit operands.
template <int F16>
__device__ __forceinline__ uint4 widen(uint4 x) { return x; }
template <int F16>
__device__ __forceinline__ uint4 widen(uint2 x) {   // e4m3: exact in bf16 and f16
  uint4 r;
  if constexpr (F16) {
    r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)x.x, 1.f, false));
    r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)x.x, 1.f, true));
    r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)x.y, 1.f, false));
    r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)x.y, 1.f, true));
  } else {
    r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x.x, 1.f, false));
    r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x.x, 1.f, true));
    r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x.y, 1.f, false));
    r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x.y, 1.f, true));
  }
  return r;
}

template <bool E8>
struct Octet { typedef uint4 type; };
template <>
struct Octet<true> { typedef uint2 type; };

// First n (0..8) of eight packed 16-bit values, the rest zero.
__device__ __forceinline__ uint4 keep_first(uint4 v, int n) {
  const auto one = [&](uint32_t w, int at) { return n > at + 1 ? w : (n > at ? w & 0xFFFFu : 0u); };
  return make_uint4(one(v.x, 0), one(v.y, 2), one(v.z, 4), one(v.w, 6));
}

constexpr float LN2 = 0.69314718055994530942f;

}  // namespace

template <int F16, int E8, int D>
__global__ void __launch_bounds__(256) k_attn_part(AttnArgs p) {
  constexpr int KS = D / 32, NT = D / 16, EB = E8 ? 1 : 2;
  typedef typename Octet<E8 != 0>::type Oct;
  __shared__ __align__(16) float red[4][16][D + 4];
  __shared__ float rm[4][16], rl[4][16];
  const int t = threadIdx.x, lane = lane_id(), m = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(t / WAVE);
  // blocks of one (part, head) with several tiles of query heads share an XCD
  const int bi = blockIdx.x;
  const int pair = (bi / (8 * p.mt)) * 8 + bi % 8, tile = (bi / 8) % p.mt;
  const int item = pair / p.Hkv, hk = pair % p.Hkv;
  Split sp;
  if (!find_split(p.lens, p.pg.B, p.pg.max_pages << p.sh, p.extra, p.lmin, item, sp)) return;
  const int start = sp.s * sp.L, end = min(sp.len, start + sp.L);
  if (sp.s == 0 && hk == 0 && tile == 0 && t < 2) p.reqs[2 * sp.b + t] = t ? sp.ns : sp.first;
  const int mask = p.pg.page - 1;
  const int h16 = tile * 16 + m;              // query head within the group
  const int hq = hk * p.g + min(h16, p.g - 1);   // heads past the last repeat it and are not stored

  uint4 qf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
    qf[ks] = *(const uint4*)((const uint16_t*)p.q + sp.b * p.q_stride + (size_t)hq * D + 32 * ks + 8 * g);
  const float sc = p.scale2 * (E8 && p.k_scale ? p.k_scale[hk] : 1.f);

  f32x4 acc[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float mx = NEG_INF, ls = 0.f;
  const int32_t* row = p.tables + (size_t)sp.b * p.pg.max_pages;
  const size_t page_bytes = (size_t)p.pg.page * D * EB;
  const int koct = m >> 2;

  // the 32 tokens lie on one page or, with 16 tokens a page, on two; their
  // numbers are read one turn ahead
  const int last = max(end - 1, 0);
  int next0 = load_uniform(row + (min(start + 32 * w, last) >> p.sh));
  int next1 = load_uniform(row + (min(start + 32 * w + 16, last) >> p.sh));
  for (int t0 = start + 32 * w; t0 < end; t0 += 128) {
    int pid0 = next0, pid1 = next1;
    next0 = load_uniform(row + (min(t0 + 128, last) >> p.sh));
    next1 = load_uniform(row + (min(t0 + 144, last) >> p.sh));
    const bool ok0 = (unsigned)pid0 < (unsigned)p.pg.n_pages, ok1 = (unsigned)pid1 < (unsigned)p.pg.n_pages;
    pid0 = ok0 ? pid0 : 0;
    pid1 = ok1 ? pid1 : 0;
    const size_t at0 = ((size_t)pid0 * p.Hkv + hk) * page_bytes, at1 = ((size_t)pid1 * p.Hkv + hk) * page_bytes;
    const uint8_t* kp = (const uint8_t*)p.kc + (koct >= 2 ? at1 : at0);
    const uint8_t* vp = (const uint8_t*)p.vc + (g >= 2 ? at1 : at0) +
                        ((size_t)(((t0 + 8 * g) & mask) >> 3) * D + m) * 8 * EB;
    Oct kf[2][KS], vf[NT];
#pragma unroll
    for (int ti = 0; ti < 2; ++ti)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        kf[ti][ks] = *(const Oct*)(kp + ((size_t)((t0 + 8 * koct + 4 * ti + (m & 3)) & mask) * D + 32 * ks + 8 * g) * EB);
#pragma unroll
    for (int i = 0; i < NT; ++i) vf[i] = *(const Oct*)(vp + (size_t)i * 16 * 8 * EB);

    float x[8];
#pragma unroll
    for (int ti = 0; ti < 2; ++ti) {
      f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) s = mma16<F16>(widen<F16>(kf[ti][ks]), qf[ks], s);
#pragma unroll
      for (int r = 0; r < 4; ++r) x[4 * ti + r] = s[r] * sc;
    }
    const bool full = t0 + 32 <= end && ok0 && ok1;   // wave-uniform
    const int nv = full ? 8 : ((g >= 2 ? ok1 : ok0) ? min(max(end - (t0 + 8 * g), 0), 8) : 0);
    if (!full) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = e < nv ? x[e] : NEG_INF;
    }
    float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    top = fmaxf(max_groups(top), mx);
    const float ref = top == NEG_INF ? 0.f : top;
    if (__any(top != mx)) {
      const float a = exp2_f(mx - ref);
      ls *= a;
#pragma unroll
      for (int i = 0; i < NT; ++i) acc[i] *= a;
      mx = top;
    }
    float pr[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) pr[e] = step_weight<F16>(x[e] - ref);
    ls += ((pr[0] + pr[1]) + (pr[2] + pr[3])) + ((pr[4] + pr[5]) + (pr[6] + pr[7]));
    const uint4 pb = make_uint4(pack2<F16>(pr[0], pr[1]), pack2<F16>(pr[2], pr[3]),
                                pack2<F16>(pr[4], pr[5]), pack2<F16>(pr[6], pr[7]));
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      uint4 a = widen<F16>(vf[i]);
      if (!full) a = keep_first(a, nv);   // a zero weight does not hide Inf or NaN behind the end
      acc[i] = mma16<F16>(a, pb, acc[i]);
    }
  }
  ls = sum_groups(ls);

  // join the four waves: rows d = 16 i + 4 g + r of column m
#pragma unroll
  for (int i = 0; i < NT; ++i) *(f32x4*)&red[w][m][16 * i + 4 * g] = acc[i];
  if (g == 0) {
    rm[w][m] = mx;
    rl[w][m] = ls;
  }
  __syncthreads();
  const float vs = E8 && p.v_scale ? p.v_scale[hk] : 1.f;
  for (int e = t; e < 16 * D / 4; e += 256) {
    const int h = e / (D / 4), d4 = 4 * (e % (D / 4));
    if (tile * 16 + h >= p.g) break;
    const float top = fmaxf(fmaxf(rm[0][h], rm[1][h]), fmaxf(rm[2][h], rm[3][h]));
    const float ref = top == NEG_INF ? 0.f : top;
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float a = exp2_f(rm[u][h] - ref);
      l = __builtin_fmaf(a, rl[u][h], l);
      o += *(const f32x4*)&red[u][h][d4] * a;
    }
    const int q = hk * p.g + tile * 16 + h;
    if (sp.ns == 1) {
      const float inv = l == 0.f ? 0.f : vs / l;
      uint2 y;
      y.x = pack2<F16>(o[0] * inv, o[1] * inv);
      y.y = pack2<F16>(o[2] * inv, o[3] * inv);
      *(uint2*)((uint16_t*)p.o + ((size_t)sp.b * p.Hq + q) * D + d4) = y;
      if (p.lse && d4 == 0) p.lse[(size_t)sp.b * p.Hq + q] = (top + (log2f(l) - STEP_SHIFT<F16>)) * LN2;
    } else {
      const size_t at = (size_t)(sp.first + sp.s) * p.Hq + q;
      *(f32x4*)&p.part_o[at * D + d4] = o;
      if (d4 == 0) *(float2*)&p.part_ml[at * 2] = make_float2(top, l);
    }
  }
}

// Join of a request's parts for SL channels of one query head: weights
// 2^(m_s - max m) of the parts' unnormalised sums, 1024 / SL parts at once.
template <int F16, int SL>
__global__ void __launch_bounds__(256) k_attn_join(AttnArgs p) {
  constexpr int C4 = SL / 4, NG = 256 / C4;
  __shared__ __align__(16) float red[NG][SL + 4];
  const int slices = p.d / SL, q = blockIdx.x / slices, b = blockIdx.y, t = threadIdx.x, lane = lane_id();
  struct { int first, ns; } sp = {load_uniform(p.reqs + 2 * b), load_uniform(p.reqs + 2 * b + 1)};
  if (sp.ns == 1) return;
  const float2* ml = (const float2*)p.part_ml + (size_t)sp.first * p.Hq + q;
  const int gr = t / C4, d4 = SL * (blockIdx.x % slices) + 4 * (t % C4);
  const float* from = p.part_o + ((size_t)sp.first * p.Hq + q) * p.d + d4;
  const size_t step = (size_t)p.Hq * p.d;
  // the first parts are on their way while their weights are formed
  f32x4 ahead[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) ahead[i] = *(const f32x4*)(from + min(gr + NG * i, sp.ns - 1) * step);
  float top = NEG_INF;
  for (int s = lane; s < sp.ns; s += WAVE) top = fmaxf(top, ml[(size_t)s * p.Hq].x);
  top = wave_max_uniform(top);
  const float ref = top == NEG_INF ? 0.f : top;
  float l = 0.f;
  for (int s = lane; s < sp.ns; s += WAVE) {
    const float2 x = ml[(size_t)s * p.Hq];
    l = __builtin_fmaf(exp2_f(x.x - ref), x.y, l);
  }
  l = wave_sum_uniform(l);
  f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int s = gr + NG * i;
    if (s < sp.ns) o += ahead[i] * exp2_f(ml[(size_t)s * p.Hq].x - ref);
  }
  for (int s = gr + 4 * NG; s < sp.ns; s += NG)
    o += *(const f32x4*)(from + s * step) * exp2_f(ml[(size_t)s * p.Hq].x - ref);
  *(f32x4*)&red[gr][4 * (t % C4)] = o;
  __syncthreads();
  if (t < C4) {
#pragma unroll
    for (int u = 1; u < NG; ++u) o += *(const f32x4*)&red[u][4 * t];
    const float vs = p.e4m3 && p.v_scale ? p.v_scale[q / p.g] : 1.f;
    const float inv = l == 0.f ? 0.f : vs / l;
    uint2 y;
    y.x = pack2<F16>(o[0] * inv, o[1] * inv);
    y.y = pack2<F16>(o[2] * inv, o[3] * inv);
    *(uint2*)((uint16_t*)p.o + ((size_t)b * p.Hq + q) * p.d + d4) = y;
    if (p.lse && d4 == 0) p.lse[(size_t)b * p.Hq + q] = (top + (log2f(l) - STEP_SHIFT<F16>)) * LN2;
  }
}

namespace {

template <int F16, int D>
hipError_t launch_d(const AttnArgs& a, hipStream_t st) {
  const unsigned pairs = (unsigned)(a.pg.B + a.extra) * a.Hkv;
  const unsigned grid = (pairs + 7) / 8 * 8 * a.mt;
  const hipError_t e = a.e4m3 ? launch("attn", k_attn_part<F16, 1, D>, grid, 256, 0, st, a)
                              : launch("attn", k_attn_part<F16, 0, D>, grid, 256, 0, st, a);
  if (e != hipSuccess || ((long long)a.pg.max_pages << a.sh) <= a.lmin) return e;   // no request has two parts
  // few heads and requests (long contexts, many parts each): narrow slices, so
  // that the join has blocks enough (16 heads, 4 requests, d = 256, 256 parts:
  // 8.8 against 11.2 us; 32 heads, 64 requests, d = 128: 6.8 against 5.0)
  if (D > 64 && (long long)a.Hq * a.pg.B <= 256)
    return launch("attn_join", k_attn_join<F16, 64>, dim3((unsigned)a.Hq * (D / 64), (unsigned)a.pg.B), 256, 0, st, a);
  return launch("attn_join", k_attn_join<F16, D>, dim3((unsigned)a.Hq, (unsigned)a.pg.B), 256, 0, st, a);
}

template <int F16>
hipError_t launch_t(const AttnArgs& a, hipStream_t st) {
  if (a.d == 64) return launch_d<F16, 64>(a, st);
  if (a.d == 128) return launch_d<F16, 128>(a, st);
  return launch_d<F16, 256>(a, st);
}

}  // namespace

hipError_t launch_attn_step(const AttnArgs& a, hipStream_t st) {
  return a.f16 ? launch_t<1>(a, st) : launch_t<0>(a, st);
}

}  // namespace kda
