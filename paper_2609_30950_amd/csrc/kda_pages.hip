// Block tables and slot maps of a serving step, and the writes of new tokens
// into paged caches (kda_pages_plan, kda_attn_append, kda_latent_append).

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kda_attn.hpp"
#include "kda_profile.hpp"

namespace kda {

namespace {

constexpr int PLAN_MAX_B = 4096;
constexpr int PLAN_SLOTS = 4096;   // slots the planning block writes itself

__device__ __forceinline__ int place(const PlanArgs& p, int pid, int pos) {
  return (unsigned)pid < (unsigned)p.pg.n_pages ? (pid << p.sh) + (pos & (p.pg.page - 1)) : -1;
}

// The step's bookkeeping is a chain of three prefix sums over at most 4096
// requests (rows, pages returned, pages taken) and packed lists of page moves,
// so one block does it: thread t holds the consecutive requests t R .., and
// item i of a list finds its request by bisection of the offsets in LDS.  A
// page taken is read where it comes from (a returned page from its old table
// row), so that no move waits for another's write.  Bound by latency: two
// rounds of loads, the barriers, and instructions that come from a cold cache
// (hence a form of its own for the usual R = 1).
template <int NT, int R>
__global__ void __launch_bounds__(NT) k_plan(PlanArgs p) {
  __shared__ int part[3][NT / WAVE];
  __shared__ int s_row[NT * R], s_back[NT * R], s_grow[NT * R], s_len[NT * R];   // length, -1: refused
  __shared__ int s_taken;
  const int t = threadIdx.x, B = p.pg.B;
  const int cap = p.pg.max_pages << p.sh, mask = p.pg.page - 1;
  if (t == 0) s_taken = 0;
  int len[R], nw[R], have[R], rows = 0, back = 0;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int b = min(t * R + r, B - 1);
    len[r] = p.lens[b];
    nw[r] = p.newt[b];
  }
  const int n0 = min(max(p.n_free[0], 0), p.pg.n_pages);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (t * R + r >= B) nw[r] = 0;
    have[r] = len[r] >= 0 && len[r] <= cap ? (len[r] + mask) >> p.sh : 0;
    rows = add_sat(rows, max(nw[r], 0));
    if (nw[r] < 0) back = add_sat(back, have[r]);
  }
  int rows_all, back_all, grow_all;
  int row0 = block_before<NT>(rows, part[0], rows_all);
  int back0 = block_before<NT>(back, part[1], back_all);
  const int returned = min(back_all, p.pg.n_pages - n0), n1 = n0 + returned;
  int grow[R], grows = 0;
  bool fits[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int b = t * R + r, add = max(nw[r], 0);
    s_row[b] = row0;
    s_back[b] = back0;
    if (b < B) p.cu[b] = row0;
    row0 = add_sat(row0, add);
    if (nw[r] < 0) back0 = add_sat(back0, have[r]);
    fits[r] = b < B && nw[r] >= 0 && len[r] >= 0 && len[r] <= cap && add <= cap - len[r] && row0 <= p.n_slots;
    grow[r] = fits[r] ? ((len[r] + add + mask) >> p.sh) - have[r] : 0;
    grows = add_sat(grows, grow[r]);
  }
  int grow0 = block_before<NT>(grows, part[2], grow_all);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int b = t * R + r;
    s_grow[b] = grow0;
    grow0 = add_sat(grow0, grow[r]);
    const bool ok = fits[r] && (grow[r] == 0 || grow0 <= n1);
    if (ok && grow[r] > 0) atomicMax(&s_taken, grow0);
    s_len[b] = ok ? len[r] : -1;
    if (b < B) {
      p.ok[b] = ok || nw[r] < 0;
      p.lens_out[b] = nw[r] < 0 ? 0 : (ok ? len[r] + nw[r] : len[r]);
    }
  }
  if (t == 0) p.cu[B] = rows_all;
  __syncthreads();
  const int taken = s_taken;
  if (t == 0) p.n_free_out[0] = n1 - taken;

  const auto returned_page = [&](int i) {
    const int b = owner(s_back, B, i);
    return p.tables[(size_t)b * p.pg.max_pages + (i - s_back[b])];
  };
  const auto taken_page = [&](int i) {
    const int at = n1 - 1 - i;
    return at >= n0 ? returned_page(at - n0) : p.free_pages[at];
  };
  for (int i0 = t; i0 < returned; i0 += 4 * NT) {   // four moves at once: ended requests may hold many pages
    int i[4], b[4], pid[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) i[k] = min(i0 + k * NT, returned - 1);
    owners<4>(s_back, B, i, b);
#pragma unroll
    for (int k = 0; k < 4; ++k) pid[k] = p.tables[(size_t)b[k] * p.pg.max_pages + (i[k] - s_back[b[k]])];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i0 + k * NT < returned) p.free_pages[n0 + i[k]] = pid[k];
  }
  for (int i = t; i < taken; i += NT) {
    const int b = owner(s_grow, B, i), held = (s_len[b] + mask) >> p.sh;
    p.tables[(size_t)b * p.pg.max_pages + held + (i - s_grow[b])] = taken_page(i);
  }
  if (p.n_slots > PLAN_SLOTS) return;   // k_slots writes them
  for (int i = t; i < p.n_slots; i += NT) {
    int slot = -1;
    if (i < rows_all) {
      const int b = owner(s_row, B, i), n = s_len[b];
      if (n >= 0) {
        const int pos = n + (i - s_row[b]), idx = pos >> p.sh, held = (n + mask) >> p.sh;
        slot = place(p, idx < held ? p.tables[(size_t)b * p.pg.max_pages + idx] : taken_page(s_grow[b] + idx - held), pos);
      }
    }
    p.slots[i] = slot;
  }
}

// Slots of a step with many rows, spread over the chip: a row finds its
// request in cu and its token from the end of the request.
__global__ void __launch_bounds__(256) k_slots(PlanArgs p) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= p.n_slots) return;
  int slot = -1;
  if (i < p.cu[p.pg.B]) {
    const int b = owner(p.cu, p.pg.B, i);
    if (p.ok[b]) {
      const int pos = p.lens_out[b] - (p.cu[b + 1] - i);
      slot = place(p, p.tables[(size_t)b * p.pg.max_pages + (pos >> p.sh)], pos);
    }
  }
  p.slots[i] = slot;
}

// ------------------------------------------------------------- appends ---

// Division by a head's scale s = m 2^e, correctly rounded: with y = x 2^-e, r =
// fl(1 / m) and q = fl(y r), fl(q + r (y - q m)) is fl(x / s), since the
// remainder is exact in a fused multiply-add.  Where y leaves the normal range,
// so does the quotient (m lies in [1/2, 1)): it saturates or rounds to zero.
// Quotients that saturate skip the correction, whose remainder may overflow,
// and so do scales that are zero or not finite.  (The compiler's division
// takes a dozen instructions an element and came to half the kernel's time.)
struct Scale {
  float m, r;
  int e;
  bool fix;
  __device__ __forceinline__ explicit Scale(float s)
      : m(__builtin_amdgcn_frexp_mantf(s)), r(1.f / m), e(-__builtin_amdgcn_frexp_expf(s)),
        fix(s != 0.f && __builtin_isfinite(s)) {}
  __device__ __forceinline__ float operator()(float x) const {   // saturated; NaN stays NaN
    const float y = __builtin_amdgcn_ldexpf(x, e), q = y * r;
    const float c = __builtin_fmaf(__builtin_fmaf(-q, m, y), r, q);
    const float z = fix && fabsf(q) < 1024.f ? c : q;
    return z != z ? z : __builtin_amdgcn_fmed3f(z, -448.f, 448.f);
  }
};

__device__ __forceinline__ uint32_t word(const uint4& v, int i) {
  return i == 0 ? v.x : (i == 1 ? v.y : (i == 2 ? v.z : v.w));
}
template <int F16>
__device__ __forceinline__ float element(const uint4& v, int i) {
  return i & 1 ? hi_f32<F16>(word(v, i / 2)) : lo_f32<F16>(word(v, i / 2));
}
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}

// Rows of keys and values, eight channels of a head per thread.  Eight tokens
// of a value channel lie together: where the eight rows of such a group come
// one after the other (a prompt's rows do), the threads of the one whose number
// divides by eight write all of them, 16 or 8 bytes a channel (v_blocks
// blocks).  The other rows have threads of their own, which write an element
// per channel (the first blocks); since a prompt leaves those nothing but the
// look at the slots, they then take all heads of a row one after the other.
// Keys are copied as rows (the last blocks).  A block is one head's and a
// thread one key row's: two or four rows a thread, or the heads of a row side
// by side, took 24 and 32 us instead of 17 (8191 rows of 8 heads, d = 128, 16
// bits), and looking at several rows a thread 25.
struct Group {
  int row, slot;   // the first row's
  bool whole;
};
__device__ __forceinline__ Group group_of(const AppendArgs& p, int row, int slot) {
  Group g = {row - (slot & 7), slot & ~7, false};
  g.whole = slot >= 0 && g.row >= 0 && g.row + 7 < p.n && (slot >> p.sh) < p.pg.n_pages;
  if (g.whole) {
    bool same = true;
#pragma unroll
    for (int j = 0; j < 8; ++j) same = same && p.slots[g.row + j] == g.slot + j;
    g.whole = same;
  }
  return g;
}

template <int F16>
__device__ __forceinline__ uint2 e4m3x8(const Scale& f, const uint4& v) {
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = f(element<F16>(v, i));
  return make_uint2(e4m3x4(x[0], x[1], x[2], x[3]), e4m3x4(x[4], x[5], x[6], x[7]));
}

template <int F16, int E8>
__device__ __forceinline__ void append_single(const AppendArgs& p, int row, int c8, int h0, int h1) {
  const int slot = p.slots[row];
  const int pid = slot >> p.sh, off = slot & (p.pg.page - 1);
  if (slot < 0 || pid >= p.pg.n_pages || group_of(p, row, slot).whole) return;
  for (int h = h0; h < h1; ++h) {
    const uint4 v = *(const uint4*)((const uint16_t*)p.b + row * p.b_stride + (size_t)h * p.d + 8 * c8);
    const size_t to = ((size_t)pid * p.H + h) * p.pg.page * p.d + ((size_t)(off >> 3) * p.d + 8 * c8) * 8 + (off & 7);
    if constexpr (E8) {
      const uint2 q = e4m3x8<F16>(Scale(p.b_scale ? p.b_scale[h] : 1.f), v);
      uint8_t* out = (uint8_t*)p.b_cache + to;
#pragma unroll
      for (int i = 0; i < 8; ++i) out[8 * i] = (uint8_t)((i < 4 ? q.x : q.y) >> (8 * (i & 3)));
    } else {
      uint16_t* out = (uint16_t*)p.b_cache + to;
#pragma unroll
      for (int i = 0; i < 8; ++i) out[8 * i] = (uint16_t)(word(v, i / 2) >> (16 * (i & 1)));
    }
  }
}

template <int F16, int E8>
__global__ void __launch_bounds__(256) k_append_kv(AppendArgs p, int s_blocks, int v_blocks, int all_heads) {
  const int d8 = p.d / 8, sh8 = 31 - __builtin_clz(d8);   // 8, 16 or 32
  const int bx = blockIdx.x, h = blockIdx.y;
  if (bx < s_blocks) {
    const int e = bx * 256 + threadIdx.x, row = e >> sh8;
    if (row < p.n && (!all_heads || h == 0))
      append_single<F16, E8>(p, row, e & (d8 - 1), h, all_heads ? p.H : h + 1);
    return;
  }
  const bool keys = bx >= s_blocks + v_blocks;
  const int e = (bx - s_blocks - (keys ? v_blocks : 0)) * 256 + threadIdx.x, c8 = e & (d8 - 1);
  const int row = (e >> sh8) * (keys ? 1 : 8);
  if (row >= p.n) return;
  const int slot = p.slots[row];
  const int pid = slot >> p.sh, off = slot & (p.pg.page - 1);
  const size_t in_head = (size_t)h * p.d + 8 * c8;
  if (keys) {
    const uint4 k = *(const uint4*)((const uint16_t*)p.a + row * p.a_stride + in_head);
    if (slot < 0 || pid >= p.pg.n_pages) return;
    const size_t to = (((size_t)pid * p.H + h) * p.pg.page + off) * p.d + 8 * c8;
    if constexpr (E8)
      *(uint2*)((uint8_t*)p.a_cache + to) = e4m3x8<F16>(Scale(p.a_scale ? p.a_scale[h] : 1.f), k);
    else
      *(uint4*)((uint16_t*)p.a_cache + to) = k;
    return;
  }
  const Group grp = group_of(p, row, slot);
  if (!grp.whole) return;
  const uint16_t* from = (const uint16_t*)p.b + grp.row * p.b_stride + in_head;
  const size_t to = ((size_t)pid * p.H + h) * p.pg.page * p.d + ((size_t)(off >> 3) * p.d + 8 * c8) * 8;
  uint4 v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = *(const uint4*)(from + j * p.b_stride);
  if constexpr (E8) {
    const Scale f(p.b_scale ? p.b_scale[h] : 1.f);
    // row by row, the bytes shifted into their channels: a short loop over
    // rows that move down the registers, as every launch fetches its
    // instructions anew
    uint32_t lo[8], hi[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) lo[i] = hi[i] = 0u;
#pragma unroll 1
    for (int j = 0; j < 8; ++j) {
      const uint2 q = e4m3x8<F16>(f, v[0]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        lo[i] = (lo[i] >> 8) | (hi[i] << 24);
        hi[i] = (hi[i] >> 8) | ((i < 4 ? q.x >> (8 * i) : q.y >> (8 * (i - 4))) << 24);
      }
#pragma unroll
      for (int u = 0; u < 7; ++u) v[u] = v[u + 1];
    }
    uint4* out = (uint4*)((uint8_t*)p.b_cache + to);
#pragma unroll
    for (int i = 0; i < 8; i += 2) out[i / 2] = make_uint4(lo[i], hi[i], lo[i + 1], hi[i + 1]);
  } else {
    uint4* out = (uint4*)((uint16_t*)p.b_cache + to);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const auto two = [&](int j) {   // channel i of tokens j and j + 1
        const uint32_t a = word(v[j], i / 2), b = word(v[j + 1], i / 2);
        return i & 1 ? (a >> 16) | (b & 0xFFFF0000u) : (a & 0xFFFFu) | (b << 16);
      };
      out[i] = make_uint4(two(0), two(2), two(4), two(6));
    }
  }
}

// Latent rows: c and r side by side, 16 bytes per thread.
__global__ void __launch_bounds__(256) k_append_latent(AppendArgs p) {
  const int per = (p.d + p.d2) / 8;
  const int e = blockIdx.x * 256 + threadIdx.x;
  const int row = e / per, c8 = e % per;
  if (row >= p.n) return;
  const int slot = p.slots[row];
  if (slot < 0 || (slot >> p.sh) >= p.pg.n_pages) return;
  const int x = 8 * c8;
  const uint16_t* from = x < p.d ? (const uint16_t*)p.a + row * p.a_stride + x
                                 : (const uint16_t*)p.b + row * p.b_stride + (x - p.d);
  *(uint4*)((uint16_t*)p.a_cache + (size_t)slot * (p.d + p.d2) + x) = *(const uint4*)from;
}

}  // namespace

hipError_t launch_plan(const PlanArgs& a, hipStream_t st) {
  const int B = a.pg.B;
  const hipError_t e = B <= 256 && a.n_slots <= 1024 ? launch("plan", k_plan<256, 1>, 1, 256, 0, st, a)
                       : B <= 1024                    ? launch("plan", k_plan<1024, 1>, 1, 1024, 0, st, a)
                                   : launch("plan", k_plan<1024, PLAN_MAX_B / 1024>, 1, 1024, 0, st, a);
  if (e != hipSuccess || a.n_slots <= PLAN_SLOTS) return e;
  return launch("plan", k_slots, (unsigned)((a.n_slots + 255) / 256), 256, 0, st, a);
}

hipError_t launch_append(const AppendArgs& a, bool latent, hipStream_t st) {
  if (latent) {
    const long long th = (long long)a.n * ((a.d + a.d2) / 8);
    return launch("append", k_append_latent, (unsigned)((th + 255) / 256), 256, 0, st, a);
  }
  const long long rows = (long long)a.n * (a.d / 8);   // threads for the rows of a head
  const auto blocks = [](long long threads) { return (int)((threads + 255) / 256); };
  const int blocks1 = blocks(rows), v_blocks = a.n < 8 ? 0 : blocks((a.n + 7LL) / 8 * (a.d / 8));
  const int all_heads = rows * a.H >= 1 << 18;   // fewer rows: a thread per row and head
  const dim3 grid((unsigned)(2 * blocks1 + v_blocks), (unsigned)a.H);
  if (a.e4m3)
    return a.f16 ? launch("append", k_append_kv<1, 1>, grid, 256, 0, st, a, blocks1, v_blocks, all_heads)
                 : launch("append", k_append_kv<0, 1>, grid, 256, 0, st, a, blocks1, v_blocks, all_heads);
  return launch("append", k_append_kv<0, 0>, grid, 256, 0, st, a, blocks1, v_blocks, all_heads);
}

}  // namespace kda
