// Latent attention of prompts in the expanded form (kda_latent_prefill).
//
//   k_t = [W_uk c_t, r_t],  v_t = W_uv c_t,  causal softmax over them
//
// A prompt of n rows meets n (n + 1) / 2 tokens per head; with keys and values
// written out a pair costs 2 (d_n + d_r + d_v) operations instead of the
// 2 (2 d_c + d_r) of the absorbed form (640 against 2176 at the widths 128,
// 64, 512), for the price of forming them once per token.  k_latent_rows packs
// the requests that have rows, k_latent_expand is the product of the gathered
// latent rows with both weights, and k_latent_attend the attention.
// Keys, values, queries and probabilities are f16 in its products for both
// element types.  For bf16 elements that is three bits more than the type has,
// which a score, a sum over up to 192 such products, needs to stay within the
// rounding of the output.  For f16 elements keys and probabilities are pairs
// hi + lo instead, and the values' rounding is the only one beside the
// output's (single keys and probabilities gave twice the output's rounding;
// the pairs take twice the products).  Finite numbers are saturated at 65504.
//
// A product with the values meets all tokens of a tile, those that a row does
// not see with weight zero, which must not become NaN: the expanded values are
// finite whatever they are formed from.  A latent vector that is not has keys
// that are not either, in every head and channel; they are stored as NaN and
// reach the rows that see the token through its scores.  Weights W_uv that are
// not finite belong to a channel and not to a token: k_latent_rows notes those
// channels, which become NaN at the end.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kda_attn.hpp"
#include "kda_profile.hpp"

namespace kda {

namespace {

constexpr int QT = PREFILL_ROWS;   // query rows of a block
constexpr int KT = 64;    // tokens of a tile

// Weights are formed 2^SHIFT too large, and with them the sums that divide the
// result: up to 2^(SHIFT + LAG) they fit f16, whose smallest number is then
// 2^-35 of the largest weight, so that a great many small weights beside a
// large one keep their bits (4 M of them lose 2^-14 of the sum at most).  A
// longer lag rescales less often: long prompts 868 us with 4, 864 with 8.
constexpr float SHIFT = 11.f, LAG = 4.f;

__device__ __forceinline__ float sat16(float x) {   // infinities and NaN stay
  return __builtin_isfinite(x) ? __builtin_amdgcn_fmed3f(x, -65504.f, 65504.f) : x;
}
__device__ __forceinline__ float sat16_or_nan(float x) {
  return __builtin_isfinite(x) ? __builtin_amdgcn_fmed3f(x, -65504.f, 65504.f) : __builtin_nanf("");
}
__device__ __forceinline__ float sat16_or_0(float x) {
  return x != x ? 0.f : __builtin_amdgcn_fmed3f(x, -65504.f, 65504.f);
}

// Eight 16-bit elements as f16.
template <int F16>
__device__ __forceinline__ uint4 to_f16(uint4 v) {
  if constexpr (F16) return v;
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = pack2<1>(sat16(lo_f32<0>(w[i])), sat16(hi_f32<0>(w[i])));
  return make_uint4(r[0], r[1], r[2], r[3]);
}

// Rows of request b among the n given.
__device__ __forceinline__ void row_range(const LatentPrefillArgs& p, int b, int& first, int& last) {
  first = min(max(p.cu[b], 0), p.n);
  last = min(max(p.cu[b + 1], first), p.n);
}

}  // namespace

// Bit i: row i of 32 rows of dc (256 or 512) elements holds one that is not
// finite, the exponent's bits all set.  A load covers 512 elements.
template <int F16>
__device__ __forceinline__ uint32_t not_finite_rows(const uint16_t* from, int dc) {
  constexpr uint32_t EXP = F16 ? 0x7C007C00u : 0x7F807F80u, ONE = F16 ? 0x04000400u : 0x00800080u;
  const uint4* at = (const uint4*)from + lane_id();
  uint32_t bits = 0u;
  for (int i0 = 0; i0 < dc / 16; i0 += 16) {   // of the loads that the rows take, 16 or 32
    uint4 v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = at[WAVE * (i0 + i)];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint32_t all = ((v[i].x & EXP) + ONE) | ((v[i].y & EXP) + ONE) | ((v[i].z & EXP) + ONE) | ((v[i].w & EXP) + ONE);
      const unsigned long long who = __ballot((all & 0x80008000u) != 0u);
      if (dc == 512) bits |= (uint32_t)(who != 0) << (i0 + i);
      else bits |= (uint32_t)((uint32_t)who != 0u) << (2 * i) | (uint32_t)((who >> 32) != 0) << (2 * i + 1);
    }
  }
  return bits;
}

// Packs the requests that have rows: their tokens from multiples of 8 on
// (off), the tokens held (kvn; -1 where the sum of the lengths has passed
// max_kv) and their query tiles (qoff); and for every packed token its cached
// row (src; -1 on a page that does not exist) and its shared key part as f16.
// Each block forms the sums over the requests by itself (thread t holds the
// consecutive requests t R ..), which costs less than a launch before this one.
// The blocks from `row_blocks` on look for weights of the values that are not
// finite, a wave at 32 rows of W_uv (32 value channels of a head).
template <int F16, int R>
__global__ void __launch_bounds__(256) k_latent_rows(LatentPrefillArgs p, int row_blocks) {
  if ((int)blockIdx.x >= row_blocks) {
    const int word = __builtin_amdgcn_readfirstlane(4 * ((int)blockIdx.x - row_blocks) + (int)threadIdx.x / WAVE);
    if (word < p.H * p.dn / 32) p.gone[word] = not_finite_rows<F16>((const uint16_t*)p.w_uv + (size_t)word * 32 * p.dc, p.dc);
    return;
  }
  __shared__ int part[3][4], s_off[256 * R], s_kvn[256 * R];
  const int t = threadIdx.x, B = p.pg.B, cap = p.pg.max_pages << p.sh, most = p.max_kv + 1;
  int len[R], tiles[R], sum = 0;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int b = min(t * R + r, B - 1);
    int first, last;
    row_range(p, b, first, last);
    len[r] = cut_len(p.lens[b], cap);
    if (t * R + r >= B || first == last) len[r] = first = last = 0;
    tiles[r] = (last - first + QT - 1) / QT;
    sum = add_sat(sum, len[r]);
  }
  // the sum of the lengths decides who fits, the others count those who do
  int all, at = block_before<256>(sum, part[0], all), pads = 0, qts = 0;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    at = min(add_sat(at, len[r]), most);
    len[r] = at < most ? len[r] : -1;
    pads += len[r] > 0 ? (len[r] + 7) / 8 * 8 : 0;
    qts += tiles[r];
  }
  int off = block_before<256>(pads, part[1], all), qoff = block_before<256>(qts, part[2], all);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int b = t * R + r;
    s_off[b] = off;
    s_kvn[b] = len[r];
    if (blockIdx.x == 0 && b < B) {
      p.lay[b] = off;
      p.lay[B + 1 + b] = len[r];
      p.lay[2 * B + 1 + b] = qoff;
    }
    off += len[r] > 0 ? (len[r] + 7) / 8 * 8 : 0;
    qoff += tiles[r];
    if (t == 255 && r == R - 1) {
      part[0][0] = off;   // read before the sums that used it were formed
      if (blockIdx.x == 0) {
        p.lay[B] = off;
        p.lay[3 * B + 1] = qoff;
      }
    }
  }
  __syncthreads();
  const int total = part[0][0];
  const int r8 = p.dr / 8, sh8 = 31 - __builtin_clz(r8);   // 4 or 8
  const int e = blockIdx.x * 256 + t, r = e >> sh8, x = 8 * (e & (r8 - 1));
  if (r >= (total + KT + 255) / 256 * 256) return;
  int src = 0;   // rows that hold no token: any row, masked where it is read
  if (r < total) {
    const int b = owner(s_off, B, r), pos = r - s_off[b];
    if (pos < s_kvn[b]) {
      const int pid = p.tables[(size_t)b * p.pg.max_pages + (pos >> p.sh)];
      src = (unsigned)pid < (unsigned)p.pg.n_pages ? (pid << p.sh) + (pos & (p.pg.page - 1)) : -1;
    }
  }
  if (x == 0) p.src[r] = src;
  *(uint4*)((uint16_t*)p.re + (size_t)r * p.dr + x) =
      to_f16<F16>(*(const uint4*)((const uint16_t*)p.cache + (size_t)max(src, 0) * (p.dc + p.dr) + p.dc + x));
}

// Tiles of TX x TY of tokens times the columns of [W_uk; W_uv]: 32-wide steps
// over d_c, both operands copied into LDS with two steps in flight (a step
// takes a fraction of the latency of its copies).  Keys are formed with the
// columns as rows of the product and values with the tokens; row 4 g + r of
// 16-row tile i is row 16 g + 4 i + r of its 64, so that a lane's sixteen
// results of four tiles lie side by side in the layout that is read.  Blocks
// of four waves, two a compute unit with 128 x 64 a wave or, where a chip full
// of those is missing, three with 64 x 64.  10240 tokens, 8192 columns, d_c =
// 512: 122 us (0.71 PFLOP/s, 2.0 TB/s); 178 us with 64 x 64 throughout (bound by
// the L2's requests, 16 TB/s of them), 135 us with one block of 256 x 256,
// whose loads and stores nothing covers.  The small tiles with three steps in
// flight and two blocks: calls of few requests 2 to 5 % slower.
template <int F16, int DC, int DN, int TX>
__global__ void __launch_bounds__(256, TX == 128 ? 3 : 2) k_latent_expand(LatentPrefillArgs p) {
  constexpr int TY = 128, KB = 32, NS = DC / KB, OB = TX * KB * 2, YB = TY * KB * 2;
  constexpr int NG = TX / 128, XC = TX / 64, YC = TY / 64;   // 64-row groups of a wave; copies of a wave and step
  // rows of the product, then its columns
  __shared__ __align__(16) uint8_t s0[OB + YB], s1[OB + YB], s2[OB + YB];
  const int t = threadIdx.x, lane = lane_id(), m = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(t / WAVE);
  const int B = p.pg.B, total = p.lay[B];
  constexpr int cx = TX, cy = TY;
  const int cols = p.H * DN, nk = (cols + cx - 1) / cx, key_blocks = nk * (p.kv_rows / cy);
  const bool values = (int)blockIdx.x >= key_blocks;
  const int nc = values ? (cols + cy - 1) / cy : nk, bx = values ? blockIdx.x - key_blocks : blockIdx.x;
  const int r0 = bx / nc * (values ? cx : cy), n0 = bx % nc * (values ? cy : cx);   // first token and column
  if (r0 >= total + KT) return;
  const uint16_t* wsrc = (const uint16_t*)(values ? p.w_uv : p.w_uk);
  const uint16_t* cache = (const uint16_t*)p.cache;
  // Copies of 1 KB: 16 rows of 64 B each.  Chunk c of row r stands at
  // c ^ (-(r / 16) & 3) or, for the columns, c ^ (-(r / 4) & 3).  A 16-byte
  // read serves lanes 0-3, 12-15 and 20-27 together (and so on), whose places
  // that puts into different banks; c ^ (r / 16 & 3) had half the reads' cycles
  // in conflicts.
  const auto row_of = [&](bool tokens, int r) {
    return tokens ? cache + (size_t)max(p.src[r0 + r], 0) * (DC + p.dr) : wsrc + (size_t)min(n0 + r, cols - 1) * DC;
  };
  const uint16_t *xp[XC], *yp[YC];
#pragma unroll
  for (int i = 0; i < XC; ++i) {
    const int r = 16 * (XC * w + i) + lane / 4;
    xp[i] = row_of(values, r) + 8 * ((lane & 3) ^ (-(r >> 4) & 3));
  }
#pragma unroll
  for (int i = 0; i < YC; ++i) {
    const int r = 16 * (YC * w + i) + lane / 4;
    yp[i] = row_of(!values, r) + 8 * ((lane & 3) ^ (-(r >> 2) & 3));
  }
  const auto copy_step = [&](int s, uint8_t* to) {
#pragma unroll
    for (int i = 0; i < XC; ++i) copy16(xp[i] + KB * s, to + 1024 * (XC * w + i));
#pragma unroll
    for (int i = 0; i < YC; ++i) copy16(yp[i] + KB * s, to + OB + 1024 * (YC * w + i));
  };
  copy_step(0, s0);
  copy_step(1, s1);
  f32x4 acc[NG][4][4];
#pragma unroll
  for (int k = 0; k < NG; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[k][i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int rx = 64 * NG * (w & 1), ry = 64 * (w >> 1);   // this wave's rows and columns of the product
  const int xo = (rx + 16 * (m >> 2) + (m & 3)) * 64 + 16 * (g ^ (-(m >> 2) & 3));
  const int yo = OB + (ry + m) * 64 + 16 * (g ^ (-(m >> 2) & 3));
  const auto step = [&](int s, const uint8_t* cur, uint8_t* next) {
    // this step's copies are older than those of the step behind it
    if (s < NS - 1) wait_copies_but<XC + YC>();
    else wait_copies();
    lds_barrier();
    if (s + 2 < NS) copy_step(s + 2, next);
    uint4 fy[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) fy[j] = *(const uint4*)(cur + yo + 1024 * j);
#pragma unroll
    for (int k = 0; k < NG; ++k) {
      uint4 fx[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) fx[i] = *(const uint4*)(cur + xo + 4096 * k + 256 * i);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[k][i][j] = mma16<F16>(fx[i], fy[j], acc[k][i][j]);
    }
  };
#pragma unroll
  for (int s = 0; s < NS; ++s) {   // unrolled, so that each step names its buffers
    if (s % 3 == 0) step(s, s0, s2);
    else if (s % 3 == 1) step(s, s1, s0);
    else step(s, s2, s1);
  }
  uint16_t* out = (uint16_t*)(values ? p.ve : p.ke);
#pragma unroll
  for (int k = 0; k < NG; ++k)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int xr = rx + 64 * k + 16 * g, yc = ry + 16 * j + m;
      const int col = n0 + (values ? yc : xr), tok = r0 + (values ? xr : yc);
      uint32_t y[8];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float a = acc[k][i][j][2 * u], b = acc[k][i][j][2 * u + 1];
          y[2 * i + u] = values ? pack2<1>(sat16_or_0(a), sat16_or_0(b)) : pack2<1>(sat16_or_nan(a), sat16_or_nan(b));
        }
      if (col >= cols) continue;
      const size_t h = col / DN, d = col % DN;
      if (F16 && !values) {   // what the rounding left, behind the keys
        uint32_t z[8];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const uint32_t hi = y[2 * i + u];
            z[2 * i + u] = pack2<1>(sat16_or_0(acc[k][i][j][2 * u] - lo_f32<1>(hi)),
                                    sat16_or_0(acc[k][i][j][2 * u + 1] - hi_f32<1>(hi)));
          }
        uint4* to = (uint4*)(out + ((h + p.H) * p.kv_rows + tok) * DN + d);
        to[0] = make_uint4(z[0], z[1], z[2], z[3]);
        to[1] = make_uint4(z[4], z[5], z[6], z[7]);
      }
      uint16_t* to = values ? out + ((h * (p.kv_rows / 8) + tok / 8) * DN + d) * 8 : out + (h * p.kv_rows + tok) * DN + d;
      *(uint4*)to = make_uint4(y[0], y[1], y[2], y[3]);
      *(uint4*)(to + (values ? 8 * DN : 8)) = make_uint4(y[4], y[5], y[6], y[7]);
    }
}

// Place of a 16-byte chunk in row r of a tile of keys with NC chunks a row is
// chunk ^ key_swizzle(r): one chunk of sixteen neighbouring rows then fills
// the banks once.
template <int NC>
__device__ __forceinline__ int key_swizzle(int r) { return (r / (16 / NC)) & (NC - 1); }

// 128 rows of one request and head, 32 per wave; tiles of 64 tokens in LDS,
// two deep.  The products are transposed, S^T = K Q^T and O^T = V^T P^T, with
// the wave's 32 rows as columns: a row's softmax stays within two lanes.  Row
// 8 i + 4 h + r of a score tile is token 16 (i / 2) + 8 h + 4 (i % 2) + r, so
// that eight results of a lane in a row are eight consecutive tokens, the
// operand of the product with the values, which lie eight tokens of a channel
// together.  The scores of the next tile are formed beside the softmax of this
// one.  Bound by the clock, as if the chip's power were the limit: 36 M pairs of
// 32 heads take 1.36 to 1.39 M cycles with the matrix cores 52 % busy, which are
// 774 us at 1.8 GHz and 882 at 1.54 (0.94 and 0.83 PFLOP/s) in one run; before
// the two overlapped 44 % and 786 us at 1.9 GHz.
// With TS = 2 a block has two teams of four waves, which take the tiles in turn
// and join their sums through LDS at the end: while there are fewer blocks than
// the chip holds of the one-team form (512), it is the chain of a block's
// tiles that counts (whole calls, bf16, heads of 128: 128 rows behind 2000
// tokens, 16 heads, 78 against 67 us; 2048 rows, 16 heads, 75 against 66) until
// there are more blocks (2048 rows, 64 heads, 1088 blocks: 156 against 168 us)
// or every chain is short (128 tokens: 21 against 23 us).
// With fewer blocks than compute units the tokens of a query tile are cut into
// p.parts parts as well, whose sums k_latent_attend_join puts together.
template <int F16, int DN, int DR, int TS, int CUT>
__global__ void __launch_bounds__(256 * TS, F16 || TS == 2 ? 1 : 2) k_latent_attend(LatentPrefillArgs p) {
  constexpr int NK = DN / 8, NR = DR / 8;         // chunks of a row
  constexpr int KS = DN / 16, RS = DR / 16, NT = DN / 32;
  constexpr int KP = F16 ? 2 : 1;                 // keys as hi and lo
  constexpr int KBY = KT * DN * 2, RBY = KT * DR * 2, VBY = KT * DN * 2;
  constexpr int KEYS = KP * KBY + RBY, STEP = TS * KT;
  __shared__ __align__(16) uint8_t key0_all[TS * KEYS], key1_all[TS * KEYS], val0_all[TS * VBY], val1_all[TS * VBY];
  const int t = threadIdx.x, lane = lane_id(), c = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(t / WAVE), w = wave & 3, team = TS > 1 ? wave >> 2 : 0;
  uint8_t *key0 = key0_all + team * KEYS, *key1 = key1_all + team * KEYS;
  uint8_t *val0 = val0_all + team * VBY, *val1 = val1_all + team * VBY;
  const int B = p.pg.B, h = blockIdx.x;
  const int32_t *off = p.lay, *kvn = p.lay + B + 1, *qoff = p.lay + 2 * B + 1;
  const int tiles = qoff[B], qt = tiles - 1 - (int)blockIdx.y;   // late tiles, the long ones, first
  if (qt < 0) return;
  const int b = __builtin_amdgcn_readfirstlane(owner(qoff, B, qt));
  int first, last;
  row_range(p, b, first, last);
  const int q0 = first + (qt - qoff[b]) * QT;                 // first row of the block
  const int n_kv = kvn[b], cap = p.pg.max_pages << p.sh;
  const int len = cut_len(p.lens[b], cap), off_b = off[b];
  uint16_t* o = (uint16_t*)p.o;
  if (n_kv < 0) {
    if (CUT && blockIdx.z) return;
    if (CUT && h == 0 && t == 0) *(int2*)&p.part_rows[2 * blockIdx.y] = make_int2(q0, q0);   // nothing to join
    for (int e = t; e < QT * DN / 8; e += 256 * TS) {
      const int r = q0 + e / (DN / 8);
      const uint32_t nan2 = F16 ? 0x7E007E00u : 0x7FC07FC0u;
      if (r < last) *(uint4*)&o[((size_t)r * p.H + h) * DN + 8 * (e % (DN / 8))] = make_uint4(nan2, nan2, nan2, nan2);
    }
    return;
  }
  // position of a row: its request's last tokens
  const int shift = len - p.cu[b + 1];
  const int r = q0 + 32 * w + c;
  const int pos = r < last ? shift + r : -1;
  uint4 qf[KS + RS];
  {
    const int at = min(r, last - 1);   // rows past the last repeat it and are not stored
    const uint16_t* qn = (const uint16_t*)p.qn + at * p.qn_stride + h * p.qn_head + 8 * hh;
    const uint16_t* qr = (const uint16_t*)p.qr + at * p.qr_stride + h * p.qr_head + 8 * hh;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *(const uint4*)(qn + 16 * ks);
#pragma unroll
    for (int ks = 0; ks < RS; ++ks) qf[KS + ks] = *(const uint4*)(qr + 16 * ks);
  }
#pragma unroll
  for (int ks = 0; ks < KS + RS; ++ks) qf[ks] = to_f16<F16>(qf[ks]);
  // a factor below zero: its sign goes to the queries, so that the largest
  // product stays the largest score; a factor of zero is taken as 1e-30, which
  // leaves masked scores at -inf
  const float scale2 = fmaxf(fabsf(p.scale2), 1e-30f);
  if (p.scale2 < 0.f) {
#pragma unroll
    for (int ks = 0; ks < KS + RS; ++ks) {
      const uint4 v = qf[ks];
      qf[ks] = make_uint4(v.x ^ 0x80008000u, v.y ^ 0x80008000u, v.z ^ 0x80008000u, v.w ^ 0x80008000u);
    }
  }
  f32x16 acc[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[i][e] = 0.f;
  float mx = NEG_INF, ls = 0.f;

  // tokens the block meets: a part of those up to its last row, in whole tiles
  const int met = min(len, shift + min(q0 + QT, last)), met_tiles = (max(met, 0) + KT - 1) / KT;
  const int part = CUT ? blockIdx.z : 0, parts = CUT ? p.parts : 1, start = KT * (met_tiles * part / parts);
  const int n_end = min(met, KT * (met_tiles * (part + 1) / parts));
  const int low = shift + q0 + 1;                                 // all rows meet the tokens below it
  const uint8_t* kb = (const uint8_t*)p.ke + ((size_t)h * p.kv_rows + off_b) * DN * 2;
  const uint8_t* rb = (const uint8_t*)p.re + (size_t)off_b * DR * 2;
  const uint8_t* vb = (const uint8_t*)p.ve + ((size_t)h * p.kv_rows + off_b) * DN * 2;
  // copies of 1 KB, those of number w + 4 k by wave w
  const auto copy_keys = [&](int t0, uint8_t* to) {
#pragma unroll
    for (int k = 0; k < KBY / 4096; ++k) {
      const int id = 64 * (w + 4 * k) + lane, y = id / NK, x = (id % NK) ^ key_swizzle<NK>(y);
      copy16(kb + (size_t)t0 * DN * 2 + (unsigned)(y * DN * 2 + 16 * x), to + 1024 * (w + 4 * k));
      if constexpr (F16)
        copy16(kb + ((size_t)p.H * p.kv_rows + t0) * DN * 2 + (unsigned)(y * DN * 2 + 16 * x),
               to + KBY + RBY + 1024 * (w + 4 * k));
    }
#pragma unroll
    for (int k = 0; k < RBY / 4096; ++k) {
      const int id = 64 * (w + 4 * k) + lane, y = id / NR, x = (id % NR) ^ key_swizzle<NR>(y);
      copy16(rb + (size_t)t0 * DR * 2 + (unsigned)(y * DR * 2 + 16 * x), to + KBY + 1024 * (w + 4 * k));
    }
  };
  const auto copy_values = [&](int t0, uint8_t* to) {
#pragma unroll
    for (int k = 0; k < VBY / 4096; ++k)
      copy16(vb + (size_t)t0 * DN * 2 + (unsigned)(1024 * (w + 4 * k) + 16 * lane), to + 1024 * (w + 4 * k));
  };
  // LDS places of this lane's operands; both halves of a tile are constants away
  const int tr = 16 * (c >> 4) + 8 * ((c >> 2) & 1) + 4 * ((c >> 3) & 1) + (c & 3);   // its score row's token
  unsigned ka[KS], ra[RS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    ka[ks] = tr * DN * 2 + 16 * ((2 * ks + hh) ^ key_swizzle<NK>(tr));
    asm volatile("" : "+v"(ka[ks]));
  }
#pragma unroll
  for (int ks = 0; ks < RS; ++ks) {
    ra[ks] = tr * DR * 2 + 16 * ((2 * ks + hh) ^ key_swizzle<NR>(tr));
    asm volatile("" : "+v"(ra[ks]));
  }
  unsigned va = (hh * DN + c) * 16;
  asm volatile("" : "+v"(va));

  // tokens of the tile that lie on pages that do not exist, looked up a tile ahead
  const int32_t* src = p.src + off_b + lane;
  int next_src = 0;
  // scores of a tile: x[hf][8 s + e] of token t0 + 32 hf + 16 s + 8 hh + e
  const auto scores = [&](const uint8_t* lk, f32x16* x) {
    const uint8_t* lr = lk + KBY;
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int e = 0; e < 16; ++e) x[hf][e] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
      {
        if constexpr (F16)
          x[hf] = mma32_f16(*(const uint4*)(lk + KBY + RBY + ka[ks] + 32 * hf * DN * 2), qf[ks], x[hf]);
        x[hf] = mma32_f16(*(const uint4*)(lk + ka[ks] + 32 * hf * DN * 2), qf[ks], x[hf]);
      }
#pragma unroll
    for (int ks = 0; ks < RS; ++ks)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
        x[hf] = mma32_f16(*(const uint4*)(lr + ra[ks] + 32 * hf * DR * 2), qf[KS + ks], x[hf]);
  };
  // One turn: the weights of tile t0 from its scores x while the matrix cores
  // form the next tile's scores y, then the product with the tile's values.
  // Keys two tiles ahead and values one ahead are copied meanwhile, into the
  // buffers that the turn before has read.
  const auto turn = [&](int t0, f32x16* x, f32x16* y, uint8_t* k_free, const uint8_t* k_next, const uint8_t* lv,
                        uint8_t* v_free) {
    wait_copies();
    __syncthreads();
    if (TS > 1 && t0 >= n_end) return;
    if (t0 + 2 * STEP < n_end) copy_keys(t0 + 2 * STEP, k_free);
    if (t0 + STEP < n_end) copy_values(t0 + STEP, v_free);
    const unsigned long long bad = __ballot(next_src < 0);
    next_src = t0 + STEP < n_end ? src[t0 + STEP] : 0;
    if (t0 + KT > low) {
      const int left = pos - t0 - 8 * hh;   // of the lane's tokens, which are 16 s + e
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (32 * hf + 16 * (e >> 3) + (e & 7) > left) x[hf][e] = NEG_INF;
    }
    if (bad) {
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        const uint32_t gone = (uint32_t)(bad >> (32 * hf)) >> (8 * hh);
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (gone >> (16 * (e >> 3) + (e & 7)) & 1) x[hf][e] = NEG_INF;
      }
    }
    float top = fmaxf(x[0][0], x[1][0]);
#pragma unroll
    for (int e = 1; e < 16; ++e) top = fmaxf(fmaxf(top, x[0][e]), x[1][e]);
    {
      const uint32_t u = __builtin_bit_cast(uint32_t, top);
      auto z = __builtin_amdgcn_permlane32_swap(u, u, false, false);
      top = fmaxf(__builtin_bit_cast(float, (uint32_t)z[0]), __builtin_bit_cast(float, (uint32_t)z[1])) * scale2;
    }
    // the reference follows the maximum only when that has grown by 2^LAG:
    // larger weights are as exact in f16, and few tiles rescale
    if (__any(top > mx + LAG)) {
      const float ref = fmaxf(top, mx);
      const float a = exp2_f(mx - (ref == NEG_INF ? 0.f : ref));
      ls *= a;
#pragma unroll
      for (int i = 0; i < NT; ++i) acc[i] *= a;
      mx = ref;
    }
    const float sub = mx == NEG_INF ? 0.f : mx;
    scores(k_next, y);   // past the last tile: of what the buffer holds, not used
    uint4 pb[2][2], pl[2][2];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        x[hf][e] = exp2_f(__builtin_fmaf(x[hf][e], scale2, SHIFT - sub));
        sum += x[hf][e];
      }
      ls += sum;
#pragma unroll
      for (int s = 0; s < 2; ++s)
      {
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float a = x[hf][8 * s + 2 * i], b = x[hf][8 * s + 2 * i + 1];
          hi[i] = pack2<1>(a, b);
          if constexpr (F16) lo[i] = pack2<1>(a - lo_f32<1>(hi[i]), b - hi_f32<1>(hi[i]));
        }
        pb[hf][s] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        if constexpr (F16) pl[hf][s] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
      }
    }
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          const uint4 a = *(const uint4*)(lv + va + ((4 * hf + 2 * s) * DN + 32 * i) * 16);
          if constexpr (F16) acc[i] = mma32_f16(a, pl[hf][s], acc[i]);
          acc[i] = mma32_f16(a, pb[hf][s], acc[i]);
        }
  };
  f32x16 xa[2], xb[2];
  const int mine = start + KT * team;   // this team's first tile; every wave passes the barriers of the first team's
  if (start < n_end) {
    if (mine < n_end) {
      next_src = src[mine];
      copy_keys(mine, key0);
      copy_values(mine, val0);
    }
    wait_copies();
    __syncthreads();
    if (mine + STEP < n_end) copy_keys(mine + STEP, key1);
    if (mine < n_end) scores(key0, xa);
  }
  for (int t0 = start; t0 < n_end; t0 += 2 * STEP) {
    turn(t0 + KT * team, xa, xb, key0, key1, val0, val1);
    if (t0 + STEP < n_end) turn(t0 + STEP + KT * team, xb, xa, key1, key0, val1, val0);
  }
  if constexpr (TS > 1) {   // the second team's sums to the first, through the keys' LDS
    constexpr int HALF = NT / 2;
    static_assert(4 * HALF * 4096 <= TS * KEYS && 2048 <= TS * VBY);
    f32x4 *lo = (f32x4*)key0_all, *hi = (f32x4*)key1_all;
    float2* ml = (float2*)val0_all;
    __syncthreads();
    if (team) {
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          (i < HALF ? lo : hi)[((w * HALF + i % HALF) * 4 + k) * WAVE + lane] =
              f32x4{acc[i][4 * k], acc[i][4 * k + 1], acc[i][4 * k + 2], acc[i][4 * k + 3]};
      ml[WAVE * w + lane] = make_float2(mx, ls);
    }
    __syncthreads();
    if (team) return;
    const float2 other = ml[WAVE * w + lane];
    const float top = fmaxf(mx, other.x), ref = top == NEG_INF ? 0.f : top;
    const float a = exp2_f(mx - ref), b2 = exp2_f(other.x - ref);
    ls = __builtin_fmaf(other.y, b2, ls * a);
    mx = top;
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const f32x4 y = (i < HALF ? lo : hi)[((w * HALF + i % HALF) * 4 + k) * WAVE + lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][4 * k + e] = __builtin_fmaf(y[e], b2, acc[i][4 * k + e] * a);
      }
  }
  const float l = ls + __shfl_xor(ls, 32), inv = l == 0.f ? 0.f : 1.f / l;
  if constexpr (CUT) {
    const size_t block = ((size_t)blockIdx.y * p.H + h) * p.parts + part;
    f32x4* to = (f32x4*)p.part_o + block * (QT * DN / 4) + w * (32 * DN / 4) + lane;
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        to[(i * 4 + k) * WAVE] = f32x4{acc[i][4 * k], acc[i][4 * k + 1], acc[i][4 * k + 2], acc[i][4 * k + 3]};
    if (hh == 0) ((float2*)p.part_ml)[block * QT + 32 * w + c] = make_float2(mx, l);
    if (h == 0 && part == 0 && t == 0) *(int2*)&p.part_rows[2 * blockIdx.y] = make_int2(q0, last);
    return;
  }
  if (r < last) {
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const uint32_t gone = load_uniform(p.gone + h * NT + i);
      if (gone != 0 && l != 0.f) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (gone >> (8 * (e >> 2) + 4 * hh + (e & 3)) & 1) acc[i][e] = __builtin_nanf("");
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint2 y;
        y.x = pack2<F16>(acc[i][4 * k] * inv, acc[i][4 * k + 1] * inv);
        y.y = pack2<F16>(acc[i][4 * k + 2] * inv, acc[i][4 * k + 3] * inv);
        *(uint2*)&o[((size_t)r * p.H + h) * DN + 32 * i + 8 * k + 4 * hh] = y;
      }
    }
  }
}

// Join of a query tile's parts for 32 rows and 32 channels of one head, lanes
// and registers as the parts wrote them.  The four waves share the parts, so
// that sixteen parts take one round of loads, then the four groups of channels.
template <int F16, int DN>
__global__ void __launch_bounds__(256) k_latent_attend_join(LatentPrefillArgs p) {
  constexpr int NT = DN / 32;
  __shared__ __align__(16) f32x4 red[4][4][WAVE];
  __shared__ float rl[4][WAVE];
  const int t = threadIdx.x, lane = lane_id(), c = lane & 31, hh = lane >> 5, v = t / WAVE;
  const int h = blockIdx.x, y = blockIdx.y, i = blockIdx.z % NT, w = blockIdx.z / NT;
  const int tiles = load_uniform(p.lay + 3 * p.pg.B + 1);
  const int q0 = load_uniform(p.part_rows + 2 * y), last = load_uniform(p.part_rows + 2 * y + 1);
  if (y >= tiles || q0 + 32 * w >= last) return;
  const size_t block = ((size_t)y * p.H + h) * p.parts;
  const float2* ml = (const float2*)p.part_ml + block * QT + 32 * w + c;
  const f32x4* from = (const f32x4*)p.part_o + block * (QT * DN / 4) + (w * NT + i) * 4 * WAVE + lane;
  float top = NEG_INF;
#pragma unroll 8
  for (int s = 0; s < p.parts; ++s) top = fmaxf(top, ml[s * QT].x);
  const float ref = top == NEG_INF ? 0.f : top;
  f32x4 o[4];
  float l = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) o[k] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = v; s < p.parts; s += 4) {
    const float2 x = ml[s * QT];
    const float a = exp2_f(x.x - ref);
    l = __builtin_fmaf(x.y, a, l);
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] += from[(size_t)s * (QT * DN / 4) + k * WAVE] * a;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) red[v][k][lane] = o[k];
  rl[v][lane] = l;
  __syncthreads();
  l = (rl[0][lane] + rl[1][lane]) + (rl[2][lane] + rl[3][lane]);
  f32x4 x = (red[0][v][lane] + red[1][v][lane]) + (red[2][v][lane] + red[3][v][lane]);
  const uint32_t gone = load_uniform(p.gone + h * NT + i);
  if (gone != 0 && l != 0.f) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (gone >> (8 * v + 4 * hh + e) & 1) x[e] = __builtin_nanf("");
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int r = q0 + 32 * w + c;
  if (r >= last) return;
  uint2 u;
  u.x = pack2<F16>(x[0] * inv, x[1] * inv);
  u.y = pack2<F16>(x[2] * inv, x[3] * inv);
  *(uint2*)&((uint16_t*)p.o)[((size_t)r * p.H + h) * DN + 32 * i + 8 * v + 4 * hh] = u;
}

namespace {

template <int F16, int DC, int DN>
hipError_t launch_expand(const LatentPrefillArgs& a, hipStream_t st) {
  const auto grid = [&](int tx) {
    const unsigned cols = (unsigned)a.H * DN, rows = (unsigned)a.kv_rows;
    return (cols + tx - 1) / tx * (rows / 128) + (cols + 127) / 128 * (rows / tx);
  };
  if (grid(256) >= 1024)   // two rounds of two blocks a compute unit
    return launch("latent_expand", k_latent_expand<F16, DC, DN, 256>, grid(256), 256, 0, st, a);
  return launch("latent_expand", k_latent_expand<F16, DC, DN, 128>, grid(128), 256, 0, st, a);
}

template <int F16, int DN, int DR>
hipError_t launch_attend(const LatentPrefillArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)a.H, (unsigned)prefill_tiles(a.pg, a.n), (unsigned)a.parts);
  const int longest = prefill_longest(a.pg, a.max_kv);
  constexpr int TEAMS = F16 && DN == 128 ? 1 : 2;   // there the second team's tiles do not fit the LDS
  const bool few = (long long)grid.x * grid.y < 512 && longest > 4 * KT;
  if (a.parts == 1)
    return few ? launch("latent_attend", k_latent_attend<F16, DN, DR, TEAMS, 0>, grid, 256 * TEAMS, 0, st, a)
               : launch("latent_attend", k_latent_attend<F16, DN, DR, 1, 0>, grid, 256, 0, st, a);
  const hipError_t e = launch("latent_attend", k_latent_attend<F16, DN, DR, TEAMS, 1>, grid, 256 * TEAMS, 0, st, a);
  if (e != hipSuccess) return e;
  return launch("latent_attend_join", k_latent_attend_join<F16, DN>, dim3(grid.x, grid.y, DN / 8), 256, 0, st, a);
}

template <int F16>
hipError_t launch_prefill_t(const LatentPrefillArgs& a, hipStream_t st) {
  const unsigned row_blocks = ((unsigned)a.kv_rows * (a.dr / 8) + 255) / 256;
  const unsigned grid = row_blocks + ((unsigned)a.H * a.dn / 32 + 3) / 4;
  hipError_t e = a.pg.B <= 256 ? launch("latent_rows", k_latent_rows<F16, 1>, grid, 256, 0, st, a, (int)row_blocks)
                               : launch("latent_rows", k_latent_rows<F16, 16>, grid, 256, 0, st, a, (int)row_blocks);
  if (e != hipSuccess) return e;
  if (a.dn == 64)
    e = a.dc == 256 ? launch_expand<F16, 256, 64>(a, st) : launch_expand<F16, 512, 64>(a, st);
  else
    e = a.dc == 256 ? launch_expand<F16, 256, 128>(a, st) : launch_expand<F16, 512, 128>(a, st);
  if (e != hipSuccess) return e;
  if (a.dn == 64) return a.dr == 32 ? launch_attend<F16, 64, 32>(a, st) : launch_attend<F16, 64, 64>(a, st);
  return a.dr == 32 ? launch_attend<F16, 128, 32>(a, st) : launch_attend<F16, 128, 64>(a, st);
}

}  // namespace

hipError_t launch_latent_prefill(const LatentPrefillArgs& a, hipStream_t st) {
  return a.f16 ? launch_prefill_t<1>(a, st) : launch_prefill_t<0>(a, st);
}

}  // namespace kda
