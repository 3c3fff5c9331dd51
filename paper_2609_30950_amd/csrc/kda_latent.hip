// Latent attention of one new token per request in the absorbed form
// (kda_latent_step).
//
//   s_t = scale ((q_n W_uk) c_t + q_r r_t),   o = W_uv sum_t softmax(s)_t c_t
//
// All heads share the cached rows [c_t, r_t], so a block that holds the
// absorbed queries of up to 32 heads reads a row once for all of them, and the
// blocks of further heads find it in the L2 that they share; with H heads a row of 2 (d_c + d_r) bytes costs 2 H (2 d_c + d_r) operations, which
// leaves HBM as the bound up to about a hundred heads.  Three launches: the
// queries through W_uk (k_latent_absorb), the attention over parts of the
// requests (k_latent_part), and the join of the parts through W_uv
// (k_latent_join).  The absorbed queries and the joined sums are 16-bit pairs
// hi + lo in the products (relative 2^-16 in bf16), since a single rounding of
// a query would shift every score of its head.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kda_attn.hpp"
#include "kda_profile.hpp"

namespace kda {

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// Transposing LDS read: each 16 lanes read four rows of 16 elements (lane i
// points at elements 4 (i % 4) .. + 3 of row i / 4), and lane i receives
// element i of the four rows.
__device__ __forceinline__ uint2 read_tr(const uint8_t* at) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at));
}
__device__ __forceinline__ uint4 join_tr(uint2 a, uint2 b) { return make_uint4(a.x, a.y, b.x, b.y); }

// A linear map of the row's four low bits that keeps banks apart both for the
// keys (16 rows of a chunk; eight of them and the next chunk of the other eight
// are served together) and for the transposed reads (32 bytes of rows 0 .. 3
// and 8 .. 11, then of the others): all sixteen values differ, and so do the
// upper three bits within each of those eights.
__device__ __forceinline__ int row_swizzle(int i) {
  return (i & 3) << 1 | (((i >> 2) ^ (i >> 3)) & 1) << 3 | ((i >> 3) & 1);
}

// Four floats as hi and lo 16-bit parts, the lo part times `up`.
template <int F16>
__device__ __forceinline__ void split4(const f32x4& x, uint2& hi, uint2& lo, float up = 1.f) {
  hi.x = pack2<F16>(x[0], x[1]);
  hi.y = pack2<F16>(x[2], x[3]);
  lo.x = pack2<F16>((x[0] - lo_f32<F16>(hi.x)) * up, (x[1] - hi_f32<F16>(hi.x)) * up);
  lo.y = pack2<F16>((x[2] - lo_f32<F16>(hi.y)) * up, (x[3] - hi_f32<F16>(hi.y)) * up);
}

// The joined sums are small where a token of large weight has a small latent
// vector.  Their lo part in f16 is formed 2^11 too large (the half step of
// 65504 still fits) and its product scaled down again: the pair then ends at
// 2^-36 instead of 2^-25.
template <int F16>
constexpr float LO_UP = F16 ? 2048.f : 1.f;

}  // namespace

// q_n W_uk for 64 channels of one head and 64 requests: the weights' tile is
// staged in LDS and read transposed (channels as rows of the product), each
// wave forms 16 requests.  Row 4 g + r of 16-row tile i is channel 16 g + 4 i
// + r, so that a lane's sixteen results lie side by side.  Writes the query
// rows {hi [d_c], lo [d_c], q_r [d_r]}.  One block more writes the split of
// the lengths for the launches that follow.
template <int F16, int DN>
__global__ void __launch_bounds__(256) k_latent_absorb(LatentArgs p) {
  constexpr int TS = 64 + 8;
  __shared__ __align__(16) uint16_t wt[DN * TS];
  const int t = threadIdx.x, lane = lane_id(), m = lane & 15, g = lane >> 4, w = t / WAVE;
  const int h = blockIdx.y, c0 = 64 * blockIdx.x, b0 = 64 * blockIdx.z;
  if (c0 == p.dc) {
    if (blockIdx.y | blockIdx.z | w) return;
    int L;
    int4* items = (int4*)p.items;
    const int cap = p.pg.max_pages << p.sh;
    const int B = p.pg.B, extra = p.extra, lmin = p.lmin;
    // every lane first notes its requests; their lengths a part are uniform
    const int n_all = split_all(p.lens, B, cap, extra, lmin, L, [&](int b, int len, int n, int first) {
      *(int2*)&p.reqs[2 * b] = make_int2(first, n);
      for (int s = 0; s < n; ++s) items[1 + first + s] = make_int4(b, s * L, min(len, s * L + L), 0);
    });
    if (lane == 0) items[0] = make_int4(n_all, 0, 0, 0);
    return;
  }
  const int qw = 2 * p.dc + p.dr;
  const int b = b0 + 16 * w + m, bc = min(b, p.pg.B - 1);
  uint4 q[DN / 32];
  {
    const uint16_t* from = (const uint16_t*)p.qn + bc * p.qn_stride + h * p.qn_head + 8 * g;
#pragma unroll
    for (int ks = 0; ks < DN / 32; ++ks) q[ks] = *(const uint4*)(from + 32 * ks);
  }
#pragma unroll
  for (int i = 0; i < DN * 8 / 256; ++i) {
    const int e = t + 256 * i, n = e / 8, c8 = e % 8;
    *(uint4*)&wt[n * TS + 8 * c8] = *(const uint4*)((const uint16_t*)p.w_uk + ((size_t)h * DN + n) * p.dc + c0 + 8 * c8);
  }
  uint16_t* qa = (uint16_t*)p.qa;
  if (blockIdx.x == 0) {
    const int r8 = p.dr / 8;
    for (int e = t; e < 64 * r8; e += 256) {
      const int y = b0 + e / r8, x = 8 * (e % r8);
      if (y < p.pg.B)
        *(uint4*)&qa[((size_t)y * p.H + h) * qw + 2 * p.dc + x] =
            *(const uint4*)((const uint16_t*)p.qr + y * p.qr_stride + h * p.qr_head + x);
    }
  }
  __syncthreads();
  if (b0 + 16 * w >= p.pg.B) return;
  f32x4 acc[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  // rows n 8 g .. of a step; columns 16 j .. + 3 of the four lanes that share a
  // row, channel 16 (m / 4) + 4 i + m % 4 for lane m
  const uint8_t* at = (const uint8_t*)&wt[(8 * g + (m >> 2)) * TS + 16 * (m & 3)];
#pragma unroll
  for (int ks = 0; ks < DN / 32; ++ks)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint8_t* x = at + 32 * ks * TS * 2 + 8 * i;
      acc[i] = mma16<F16>(join_tr(read_tr(x), read_tr(x + 4 * TS * 2)), q[ks], acc[i]);
    }
  if (b < p.pg.B) {
    uint4 hi[2], lo[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint2 h0, l0, h1, l1;
      split4<F16>(acc[2 * i], h0, l0);
      split4<F16>(acc[2 * i + 1], h1, l1);
      hi[i] = make_uint4(h0.x, h0.y, h1.x, h1.y);
      lo[i] = make_uint4(l0.x, l0.y, l1.x, l1.y);
    }
    uint4* to = (uint4*)&qa[((size_t)b * p.H + h) * qw + c0 + 16 * g];
    to[0] = hi[0];
    to[1] = hi[1];
    to += p.dc / 8;
    to[0] = lo[0];
    to[1] = lo[1];
  }
}

// One part of one request for up to 16 NH heads.  The latent vectors of 32
// tokens at a time are copied into LDS (two buffers, the next tile in flight)
// and serve as keys (channels along the product) and, read transposed, as
// values; the shared key parts r go straight to registers.  The waves of a
// group of 16 heads share the score product along the channels, KW waves a
// group, which keeps a wave's share of the absorbed queries (hi and lo) in 68
// registers at d_c = 512; they exchange their sums, each forms the weights of
// all 32 tokens, and every wave adds its share of the value channels for all
// heads.  The rows lie 2 d_c bytes apart and would share banks, so chunk c
// (16 bytes) of row i is stored at chunk c ^ row_swizzle(i).  Blocks of 64
// heads in eight waves read a row once less but load twice the queries before
// they begin (whole steps, 64 heads, with 512 blocks either way: 8 requests up
// to 8000 tokens 70 against 41 us, one of 4000 28 against 23).
// The weights meet the values in 16 bits, their sum is float32: as pairs hi + lo
// they would bring the error of 64 requests up to 8192 tokens in bf16 from
// 1.78e-3 to 1.65e-3, the output's own rounding, and the step from 75.5 to 79 us.
template <int F16, int DC, int DR, int NH>
__global__ void __launch_bounds__(256, 2) k_latent_part(LatentArgs p) {
  constexpr int NW = 4;                           // waves
  constexpr int KW = NW / NH;                     // waves of a group of heads
  constexpr int TT = 32;                          // tokens of a tile
  constexpr int CH = DC / 8;                      // 16-byte chunks of a latent vector
  constexpr int RB = (DC + DR) * 2;               // bytes of a cached row
  constexpr int NI = TT * CH / 64 / NW;           // wave-wide copies of a tile, per wave
  constexpr int KC = DC / 32 / KW, KR = DR / 32;  // k-steps over c (this wave's) and r (all)
  constexpr int KRW = (KR + KW - 1) / KW;
  constexpr int DT = DC / 16 / NW;                // 16-channel tiles of a wave
  constexpr int PS = TT + 8;
  __shared__ __align__(16) uint8_t tile0[TT * CH * 16], tile1[TT * CH * 16];
  __shared__ __align__(16) float xs[NW][2][WAVE][4];
  __shared__ __align__(16) uint16_t pt[NH * 16 * PS];
  __shared__ float sm[NH * 16], sl[NH * 16];
  const int t = threadIdx.x, lane = lane_id(), m = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(t / WAVE);
  const int hb_n = (p.H + 16 * NH - 1) / (16 * NH);
  // blocks of one part with several blocks of heads share an XCD
  const int bi = blockIdx.x;
  const int item = (bi / (8 * hb_n)) * 8 + bi % 8, h0 = (bi / 8) % hb_n * 16 * NH;
  const int rb = load_uniform(p.items + 4 + 4 * item), start = load_uniform(p.items + 4 + 4 * item + 1),
            end = load_uniform(p.items + 4 + 4 * item + 2);
  if (item >= load_uniform(p.items)) return;
  const int mask = p.pg.page - 1;
  const int32_t* row = p.tables + (size_t)rb * p.pg.max_pages;
  const int last = max(end - 1, 0);

  const int ht = w / KW, kw = w % KW;             // this wave's heads and k-steps kw + KW i
  uint4 qh[KC], ql[KC], qr[KRW];
  f32x4 acc[NH][DT];
#pragma unroll
  for (int n = 0; n < NH; ++n)
#pragma unroll
    for (int i = 0; i < DT; ++i) acc[n][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float mx[NH], own_l = 0.f;
#pragma unroll
  for (int n = 0; n < NH; ++n) mx[n] = NEG_INF;

  // pages of a tile's halves (with 16 tokens a page they differ), read a tile
  // ahead of their use; one that does not exist becomes -1 there
  const auto pages_of = [&](int t0, int& p0, int& p1) {
    p0 = load_uniform(row + (min(t0, last) >> p.sh));
    p1 = load_uniform(row + (min(t0 + 16, last) >> p.sh));
  };
  const auto checked = [&](int x) { return (unsigned)x < (unsigned)p.pg.n_pages ? x : -1; };
  const uint8_t* cache = (const uint8_t*)p.cache;
  const size_t page_bytes = (size_t)p.pg.page * RB;
  uint4 rk[2][KRW];                               // shared key parts of the tile in flight
  const auto copy_tile = [&](int t0, int p0, int p1, uint8_t* to) {
    const uint8_t* at0 = cache + (size_t)max(p0, 0) * page_bytes;
    const uint8_t* at1 = cache + (size_t)max(p1, 0) * page_bytes;
#pragma unroll
    for (int k = 0; k < NI; ++k) {
      const int id = 64 * (w + NW * k) + lane, r = id / CH, c = (id % CH) ^ row_swizzle(r);
      const uint8_t* from = (r >= 16 ? at1 : at0) + (unsigned)(((t0 + r) & mask) * RB + 16 * c);
      copy16(from, to + 1024 * (w + NW * k));
    }
#pragma unroll
    for (int ti = 0; ti < 2; ++ti)
#pragma unroll
      for (int i = 0; i < KRW; ++i)
        rk[ti][i] = *(const uint4*)((ti ? at1 : at0) + (unsigned)(((t0 + 16 * ti + m) & mask) * RB + 2 * DC +
                                                                  64 * min(kw + KW * i, KR - 1) + 16 * g));
  };

  int c0, c1, n0, n1;                             // pages of this tile and the next
  const auto work = [&](int t0, uint8_t* cur, uint8_t* next) {
    wait_copies();
    __syncthreads();
    const bool full = t0 + TT <= end && c0 >= 0 && c1 >= 0;
    if (!full) {   // rows without a token: zero, so that a zero weight hides them
      for (int e = t; e < TT * CH; e += NW * WAVE) {
        const int r = e / CH;
        if (t0 + r >= end || (r >= 16 ? c1 : c0) < 0) *(uint4*)(cur + 16 * e) = make_uint4(0u, 0u, 0u, 0u);
      }
      __syncthreads();
    }
    f32x4 s[2];
#pragma unroll
    for (int ti = 0; ti < 2; ++ti) {
      s[ti] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < KRW; ++i)
        if (kw + KW * i < KR) s[ti] = mma16<F16>(rk[ti][i], qr[i], s[ti]);
    }
    const int o0 = c0, o1 = c1;
    c0 = checked(n0);
    c1 = checked(n1);
    if (t0 + TT < end) copy_tile(t0 + TT, c0, c1, next);
    pages_of(t0 + 2 * TT, n0, n1);
#pragma unroll
    for (int i = 0; i < KC; ++i)
#pragma unroll
      for (int ti = 0; ti < 2; ++ti) {
        const uint4 a = *(const uint4*)(cur + (16 * ti + m) * CH * 16 + 16 * ((4 * (kw + KW * i) + g) ^ row_swizzle(m)));
        s[ti] = mma16<F16>(a, ql[i], s[ti]);
        s[ti] = mma16<F16>(a, qh[i], s[ti]);
      }
#pragma unroll
    for (int ti = 0; ti < 2; ++ti) *(f32x4*)&xs[w][ti][lane][0] = s[ti];
    lds_barrier();
    float x[8], top = NEG_INF;
#pragma unroll
    for (int ti = 0; ti < 2; ++ti) {
      f32x4 y = *(const f32x4*)&xs[ht * KW][ti][lane][0];
#pragma unroll
      for (int k = 1; k < KW; ++k) y += *(const f32x4*)&xs[ht * KW + k][ti][lane][0];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float v = y[r] * p.scale2;
        if (!full && (t0 + 16 * ti + 4 * g + r >= end || (ti ? o1 : o0) < 0)) v = NEG_INF;
        x[4 * ti + r] = v;
        top = fmaxf(top, v);
      }
    }
    top = max_groups(top);
#pragma unroll
    for (int n = 0; n < NH; ++n)
      if (n == ht) {
        top = fmaxf(top, mx[n]);
        own_l *= exp2_f(mx[n] - (top == NEG_INF ? 0.f : top));
      }
    const float ref = top == NEG_INF ? 0.f : top;
    // each wave writes its share of the group's weights
#pragma unroll
    for (int ti = 0; ti < 2; ++ti) {
      float pr[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) pr[r] = step_weight<F16>(x[4 * ti + r] - ref);
      own_l += (pr[0] + pr[1]) + (pr[2] + pr[3]);
      if (ti % KW == kw) {
        uint2 y;
        y.x = pack2<F16>(pr[0], pr[1]);
        y.y = pack2<F16>(pr[2], pr[3]);
        *(uint2*)&pt[(16 * ht + m) * PS + 16 * ti + 4 * g] = y;
      }
    }
    if (kw == 0 && g == 0) sm[16 * ht + m] = top;
    lds_barrier();
    uint4 pb[NH];
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      pb[n] = *(const uint4*)&pt[(16 * n + m) * PS + 8 * g];
      const float now = sm[16 * n + m];
      if (__any(now != mx[n])) {
        const float a = exp2_f(mx[n] - (now == NEG_INF ? 0.f : now));
#pragma unroll
        for (int i = 0; i < DT; ++i) acc[n][i] *= a;
        mx[n] = now;
      }
    }
    const int vr = 8 * g + (m >> 2);              // tokens 8 g .. + 3, then + 4 .. 7
    const uint8_t* v0 = cur + vr * CH * 16 + 8 * (m & 1);
    const int z0 = ((m & 3) >> 1) ^ row_swizzle(vr), z1 = ((m & 3) >> 1) ^ row_swizzle(vr + 4);
#pragma unroll
    for (int i = 0; i < DT; ++i) {
      const int ch = 2 * (w * DT + i);            // first chunk of the 16 channels
      const uint4 a = join_tr(read_tr(v0 + 16 * (ch ^ z0)), read_tr(v0 + 4 * CH * 16 + 16 * (ch ^ z1)));
#pragma unroll
      for (int n = 0; n < NH; ++n) acc[n][i] = mma16<F16>(a, pb[n], acc[n][i]);
    }
  };
  pages_of(start, c0, c1);
  c0 = checked(c0);
  c1 = checked(c1);
  if (start < end) copy_tile(start, c0, c1, tile0);
  pages_of(start + TT, n0, n1);
  // the queries behind the first tile's rows
  {
    const int h = min(h0 + 16 * ht + m, p.H - 1);   // heads past the last repeat it and are not stored
    const uint16_t* q = (const uint16_t*)p.qa + ((size_t)rb * p.H + h) * (2 * DC + DR) + 8 * g;
#pragma unroll
    for (int i = 0; i < KC; ++i) {
      qh[i] = *(const uint4*)(q + 32 * (kw + KW * i));
      ql[i] = *(const uint4*)(q + DC + 32 * (kw + KW * i));
    }
#pragma unroll
    for (int i = 0; i < KRW; ++i) qr[i] = *(const uint4*)(q + 2 * DC + 32 * min(kw + KW * i, KR - 1));
  }
  for (int t0 = start; t0 < end; t0 += 2 * TT) {
    work(t0, tile0, tile1);
    if (t0 + TT < end) work(t0 + TT, tile1, tile0);
  }
  own_l = sum_groups(own_l);
  if (kw == 0 && g == 0) {
    sl[16 * ht + m] = own_l;
    if (start >= end) sm[16 * ht + m] = NEG_INF;
  }
  __syncthreads();
  // the part's means, in float32 as every sum that is joined later
  const size_t at = (size_t)item * p.H;
#pragma unroll
  for (int n = 0; n < NH; ++n) {
    const int h = h0 + 16 * n + m;
    if (h >= p.H) continue;
    const float l = sl[16 * n + m], inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int i = 0; i < DT; ++i)
      *(f32x4*)&p.part_o[(at + h) * DC + 16 * (w * DT + i) + 4 * g] = acc[n][i] * inv;
  }
  for (int e = t; e < NH * 16; e += NW * WAVE)
    if (h0 + e < p.H) *(float2*)&p.part_ml[(at + h0 + e) * 2] = make_float2(sm[e], sl[e]);
}

// Join of the parts of up to rq requests for one head, and the product with NV
// rows of its W_uv: sixteen requests, the product's columns, or eight while
// those leave compute units without a block.  The block's
// sixteen waves share out the requests (16 / r waves each for r requests,
// which take the parts in turn), then the 16-value tiles and parts of d_c of
// the product.
template <int F16, int DC, int DV, int NV>
__global__ void __launch_bounds__(1024) k_latent_join(LatentArgs p, int rq) {
  constexpr int OS = DC + 8, PER = DC / WAVE / 4, VT = NV / 16, KP = 16 / VT;   // parts of d_c in the product
  __shared__ __align__(16) uint16_t mid[2][16 * OS];   // hi and lo
  __shared__ __align__(16) float sums[16][DC + 4];
  __shared__ float total[16];                          // a request's sum of weights
  const int t = threadIdx.x, lane = lane_id(), m = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(t / WAVE);
  const int h = blockIdx.x, b0 = rq * blockIdx.y, v0 = NV * blockIdx.z;
  const int nb = min(rq, p.pg.B - b0);
  const int wl = nb > 8 ? 0 : (nb > 4 ? 1 : (nb > 2 ? 2 : (nb > 1 ? 3 : 4)));   // log2 of a request's waves
  const int vt = w % VT, kp = w / VT;
  constexpr int KS = DC / 32 / KP;
  const uint16_t* wv = (const uint16_t*)p.w_uv + ((size_t)h * DV + v0 + 16 * vt + m) * DC + 32 * KS * kp + 8 * g;
  uint4 a[KS];
  f32x4 o[PER];
#pragma unroll
  for (int u = 0; u < PER; ++u) o[u] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int b = b0 + (w >> wl);
  if (b >= p.pg.B) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) a[ks] = *(const uint4*)(wv + 32 * ks);
  } else {
    struct { int first, ns; } sp = {load_uniform(p.reqs + 2 * b), load_uniform(p.reqs + 2 * b + 1)};
    const size_t at = (size_t)sp.first * p.H + h;
    const float2* ml = (const float2*)p.part_ml + at;
    const int s0 = w & ((1 << wl) - 1), ds = 1 << wl;
    const f32x4* from = (const f32x4*)p.part_o + at * (DC / 4) + lane;
    const auto part = [&](int s, int u) { return from[(size_t)s * p.H * (DC / 4) + 64 * u]; };
    // of part `lane`; the first parts are on their way while their weights are formed
    float2 mine = make_float2(NEG_INF, 0.f);
    if (lane < sp.ns) mine = ml[(size_t)lane * p.H];
    f32x4 ahead[4][PER];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int u = 0; u < PER; ++u) ahead[i][u] = part(min(s0 + ds * i, sp.ns - 1), u);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) a[ks] = *(const uint4*)(wv + 32 * ks);   // and the weights behind them
    float top = mine.x, l = 0.f;
    for (int s = lane + WAVE; s < sp.ns; s += WAVE) top = fmaxf(top, ml[(size_t)s * p.H].x);
    top = wave_max_uniform(top);
    const float ref = top == NEG_INF ? 0.f : top;
    mine.y *= exp2_f(mine.x - ref);
    if (sp.ns <= WAVE) {
      l = mine.y;
    } else {
      for (int s = lane; s < sp.ns; s += WAVE) {
        const float2 x = ml[(size_t)s * p.H];
        l = __builtin_fmaf(exp2_f(x.x - ref), x.y, l);
      }
    }
    l = wave_sum_uniform(l);
    if (s0 == 0 && lane == 0) total[w >> wl] = l;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const auto weight = [&](int s) {
      if (sp.ns <= WAVE) return bcast_f(mine.y, s) * inv;
      const float2 x = ml[(size_t)s * p.H];
      return exp2_f(x.x - ref) * x.y * inv;
    };
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int s = s0 + ds * i;
      if (s < sp.ns) {
        const float f = weight(s);
#pragma unroll
        for (int u = 0; u < PER; ++u) o[u] += ahead[i][u] * f;
      }
    }
    for (int s = s0 + 4 * ds; s < sp.ns; s += ds) {
      const float f = weight(s);
#pragma unroll
      for (int u = 0; u < PER; ++u) o[u] += part(s, u) * f;
    }
  }
#pragma unroll
  for (int u = 0; u < PER; ++u) *(f32x4*)&sums[w][256 * u + 4 * lane] = o[u];
  __syncthreads();
  for (int e = t; e < nb * DC / 4; e += 1024) {   // columns past the requests are not stored
    const int r = e / (DC / 4), c4 = 4 * (e % (DC / 4));
    f32x4 x = *(const f32x4*)&sums[r << wl][c4];
    for (int i = 1; i < 1 << wl; ++i) x += *(const f32x4*)&sums[(r << wl) + i][c4];
    uint2 hi, lo;
    split4<F16>(x, hi, lo, LO_UP<F16>);
    *(uint2*)&mid[0][r * OS + c4] = hi;
    *(uint2*)&mid[1][r * OS + c4] = lo;
  }
  __syncthreads();
  f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
  const int x0 = m * OS + 32 * KS * kp + 8 * g;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) acc = mma16<F16>(a[ks], *(const uint4*)&mid[1][x0 + 32 * ks], acc);
  if constexpr (F16) acc *= 1.f / LO_UP<F16>;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) acc = mma16<F16>(a[ks], *(const uint4*)&mid[0][x0 + 32 * ks], acc);
  *(f32x4*)&sums[w][4 * lane] = acc;   // the joined sums have been read
  __syncthreads();
  if (kp == 0 && m < nb) {
#pragma unroll
    for (int k = 1; k < KP; ++k) acc += *(const f32x4*)&sums[w + VT * k][4 * lane];
    if (total[m] == 0.f) acc = f32x4{0.f, 0.f, 0.f, 0.f};   // no tokens: zero whatever the weights are
    uint2 y;
    y.x = pack2<F16>(acc[0], acc[1]);
    y.y = pack2<F16>(acc[2], acc[3]);
    *(uint2*)((uint16_t*)p.o + ((size_t)(b0 + m) * p.H + h) * DV + v0 + 16 * vt + 4 * g) = y;
  }
}

namespace {

template <int F16, int DC, int DR>
hipError_t launch_part(const LatentArgs& a, hipStream_t st) {
  const int nh = a.H <= 16 ? 1 : 2;
  const unsigned hb = (unsigned)((a.H + 16 * nh - 1) / (16 * nh));
  const unsigned grid = (unsigned)(a.pg.B + a.extra + 7) / 8 * 8 * hb;
  if (nh == 1) return launch("latent", k_latent_part<F16, DC, DR, 1>, grid, 256, 0, st, a);
  return launch("latent", k_latent_part<F16, DC, DR, 2>, grid, 256, 0, st, a);
}

template <int F16, int DC, int DV>
hipError_t launch_join(const LatentArgs& a, hipStream_t st) {
  // few blocks would each draw a whole head's weights through one compute unit
  // (whole steps of one request, 32 heads: 22.6 us with a block a head, 19.8 with four)
  const dim3 grid((unsigned)a.H, (unsigned)((a.pg.B + 7) / 8));
  if (grid.x * grid.y < 256)
    return launch("latent_join", k_latent_join<F16, DC, DV, 32>, dim3(grid.x, grid.y, DV / 32), 1024, 0, st, a, 8);
  // two blocks a compute unit and more: half as many, which read the weights
  // half as often (whole steps, 64 requests up to 2000 tokens, 64 heads: 58.9
  // against 54.6 us; 128 requests up to 1000, 128 heads: 134 against 112)
  if (grid.x * grid.y >= 512)
    return launch("latent_join", k_latent_join<F16, DC, DV, DV>, dim3(grid.x, (unsigned)((a.pg.B + 15) / 16)), 1024, 0,
                  st, a, 16);
  return launch("latent_join", k_latent_join<F16, DC, DV, DV>, grid, 1024, 0, st, a, 8);
}

template <int F16, int DC>
hipError_t launch_dc(const LatentArgs& a, hipStream_t st) {
  const dim3 ga((unsigned)(DC / 64 + 1), (unsigned)a.H, (unsigned)((a.pg.B + 63) / 64));
  hipError_t e = a.dn == 64 ? launch("latent_absorb", k_latent_absorb<F16, 64>, ga, 256, 0, st, a)
                            : launch("latent_absorb", k_latent_absorb<F16, 128>, ga, 256, 0, st, a);
  if (e != hipSuccess) return e;
  e = a.dr == 32 ? launch_part<F16, DC, 32>(a, st) : launch_part<F16, DC, 64>(a, st);
  if (e != hipSuccess) return e;
  return a.dn == 64 ? launch_join<F16, DC, 64>(a, st) : launch_join<F16, DC, 128>(a, st);
}

}  // namespace

hipError_t launch_latent_step(const LatentArgs& a, hipStream_t st) {
  if (a.f16) return a.dc == 256 ? launch_dc<1, 256>(a, st) : launch_dc<1, 512>(a, st);
  return a.dc == 256 ? launch_dc<0, 256>(a, st) : launch_dc<0, 512>(a, st);
}

}  // namespace kda
