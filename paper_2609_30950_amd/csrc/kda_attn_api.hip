// C ABI of the attention layers: argument validation, workspace layout and
// launches.  Declarations and argument contracts: include/kda.h.

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>

#include "../../include/kda.h"
#include "kda_attn.hpp"

namespace {

constexpr double LOG2E = 1.4426950408889634;
constexpr int MAX_ROWS = 1 << 24;   // rows of one append, slots of one plan (32-bit thread indexes)

size_t up256(size_t x) { return (x + 255) / 256 * 256; }
bool aligned(const void* ptr, uintptr_t a) { return ((uintptr_t)ptr & (a - 1)) == 0; }
int hip_status(hipError_t e) { return e == hipSuccess ? KDA_OK : KDA_ERR_HIP; }

int log2_of(int x) {
  int s = 0;
  while ((1 << s) < x) ++s;
  return s;
}

int check_pages(const kda_pages* pg) {
  if (pg->B < 1 || pg->n_pages < 1 || pg->max_pages < 1) return KDA_ERR_SHAPE;
  if (pg->B > 4096) return KDA_ERR_UNSUPPORTED;
  if (pg->page != 16 && pg->page != 32 && pg->page != 64 && pg->page != 128 && pg->page != 256)
    return KDA_ERR_UNSUPPORTED;
  if ((int64_t)pg->n_pages * pg->page > INT32_MAX) return KDA_ERR_SHAPE;
  if ((int64_t)pg->max_pages * pg->page >= kda::SPLIT_MAX_LEN) return KDA_ERR_UNSUPPORTED;
  return KDA_OK;
}

// A factor of the scores that float32 holds together with log2(e).
bool bad_scale(double scale) { return !std::isfinite((float)(scale * LOG2E)); }

int check_attn(const kda_attn_config* cfg) {
  if (cfg == nullptr) return KDA_ERR_ARG;
  const int st = check_pages(&cfg->pg);
  if (st != KDA_OK) return st;
  if (cfg->H_kv < 1 || cfg->H_q < cfg->H_kv || cfg->H_q % cfg->H_kv != 0) return KDA_ERR_SHAPE;
  if (cfg->H_q > 1024) return KDA_ERR_UNSUPPORTED;
  if (cfg->d != 64 && cfg->d != 128 && cfg->d != 256) return KDA_ERR_UNSUPPORTED;
  if (cfg->dtype != KDA_BF16 && cfg->dtype != KDA_F16) return KDA_ERR_ARG;
  if (cfg->cache_dtype != cfg->dtype && cfg->cache_dtype != KDA_E4M3) return KDA_ERR_ARG;
  if (bad_scale(cfg->scale)) return KDA_ERR_ARG;
  return KDA_OK;
}

// Parts are cut so that about this many blocks run: some rounds of the two
// (d = 256, by its LDS) or three and more that a compute unit holds.  Longer
// lists even out the end of ragged batches (64 requests up to 8192 tokens, 8
// heads, d = 128: 139 us with 2048 blocks, 144 with 1024) but give the join
// more parts (4 requests up to 131000 tokens, 2 heads, d = 256 in 8 bits: 58 +
// 15 us with 2048, 53 + 9 with 1024).  No part is cut below ATTN_LMIN tokens.
int attn_blocks(int d) { return d == 256 ? 1024 : 2048; }
constexpr int ATTN_LMIN = 128;
// Few requests are not ragged, and their join grows with the parts: so many a
// request on average (one request, d = 128: 130000 tokens, 1 head 44 us without
// the limit and 20 with it, 60000 tokens, 8 heads 56 and 52).
constexpr int ATTN_PARTS = 128;

struct AttnWs {
  size_t o_off, ml_off, req_off, total;
};

int attn_extra(const kda_attn_config* cfg) {
  const int mt = (cfg->H_q / cfg->H_kv + 15) / 16;
  const int extra = kda::split_extra(cfg->H_kv * mt, attn_blocks(cfg->d)), most = ATTN_PARTS * cfg->pg.B;
  return extra < most ? extra : most;
}

AttnWs attn_ws(const kda_attn_config* cfg) {
  const size_t rows = (size_t)(cfg->pg.B + attn_extra(cfg)) * cfg->H_q;
  AttnWs w;
  w.o_off = 0;
  w.ml_off = up256(rows * cfg->d * sizeof(float));
  w.req_off = up256(w.ml_off + rows * 2 * sizeof(float));
  w.total = up256(w.req_off + (size_t)cfg->pg.B * 2 * sizeof(int32_t));
  return w;
}

int check_latent(const kda_latent_config* cfg) {
  if (cfg == nullptr) return KDA_ERR_ARG;
  const int st = check_pages(&cfg->pg);
  if (st != KDA_OK) return st;
  if (cfg->H < 1) return KDA_ERR_SHAPE;
  if (cfg->H > 256) return KDA_ERR_UNSUPPORTED;
  if ((cfg->d_n != 64 && cfg->d_n != 128) || cfg->d_v != cfg->d_n) return KDA_ERR_UNSUPPORTED;
  if (cfg->d_r != 32 && cfg->d_r != 64) return KDA_ERR_UNSUPPORTED;
  if (cfg->d_c != 256 && cfg->d_c != 512) return KDA_ERR_UNSUPPORTED;
  if (cfg->dtype != KDA_BF16 && cfg->dtype != KDA_F16) return KDA_ERR_ARG;
  if (bad_scale(cfg->scale)) return KDA_ERR_ARG;
  return KDA_OK;
}

// The chip holds 512 blocks at once, two a compute unit.  With up to 32 heads a
// part is a block, and the parts of a large batch are cut so that they fit that
// (whole steps, 32 heads, bf16: 128 requests up to 4000 tokens 80 us, 93 with
// 512 parts besides one a request and 86 with 256; 64 requests up to 8192: 74,
// 75 and 86).  With more heads a part has a block per 32 of them, which read
// the same rows; as many blocks are then past the 512, and still this is the
// faster cut: 512 less a batch's B ceil(H / 32) blocks takes 135 us against 109
// (128 requests up to 4000, 64 heads), 223 against 187 (64 up to 8000, 128
// heads).  A block a compute unit does for few requests, which are not ragged
// and whose join grows with the parts (32 heads, 8 requests up to 16000 tokens:
// 43 us, with 512 blocks 64; 1 of 60000: 51 and 73).  No part below 64 tokens:
// with 32 the join pays what the parts gain (one request of 2001 tokens: 19.4
// and 19.6 us), with 128 there are too few (23.1 against 19.8 us).
int latent_blocks(int B) {
  const int few = 16 * B > 256 ? 16 * B : 256, many = B < 256 ? 512 - B : 256;
  return few < many ? few : many;
}
constexpr int LATENT_LMIN = 64;
constexpr int MAX_PROMPT = 1 << 22;   // rows and cached tokens of one prompt call (grid dimensions)

struct LatentWs {
  size_t qa_off, o_off, ml_off, req_off, item_off, total;
};

int latent_extra(const kda_latent_config* cfg) {
  return kda::split_extra((cfg->H + 31) / 32, latent_blocks(cfg->pg.B));
}

LatentWs latent_ws(const kda_latent_config* cfg) {
  const size_t rows = (size_t)(cfg->pg.B + latent_extra(cfg)) * cfg->H;
  LatentWs w;
  w.qa_off = 0;
  w.o_off = up256((size_t)cfg->pg.B * cfg->H * (2 * cfg->d_c + cfg->d_r) * 2);
  w.ml_off = up256(w.o_off + rows * cfg->d_c * sizeof(float));
  w.req_off = up256(w.ml_off + rows * 2 * sizeof(float));
  w.item_off = up256(w.req_off + (size_t)cfg->pg.B * 2 * sizeof(int32_t));
  // the grid is rounded up to whole groups of eight parts
  w.total = up256(w.item_off + ((size_t)cfg->pg.B + latent_extra(cfg) + 1 + 8) * 4 * sizeof(int32_t));
  return w;
}

// The tokens of a prompt's query tiles are cut so that up to PREFILL_BLOCKS
// blocks run, one a compute unit, into parts of PREFILL_LMIN tokens at least.
// Whole calls, bf16, heads of 128: 128 rows behind 16000 tokens, 8 heads 314 ->
// 88 us (512 blocks allowed: the same), 16 rows behind 4000, 32 heads 117 -> 74
// (with parts of 1024 tokens 81), 512 rows behind 8000, 16 heads 197 -> 118
// (512 blocks 130), 1024 rows alone, 16 heads 41.8 -> 42.6.
constexpr int PREFILL_BLOCKS = 256;
constexpr int PREFILL_LMIN = 512;

int prefill_parts(const kda_latent_config* cfg, int n, int max_kv) {
  const int64_t blocks = (int64_t)cfg->H * kda::prefill_tiles(cfg->pg, n);
  const int64_t fit = PREFILL_BLOCKS / blocks, most = kda::prefill_longest(cfg->pg, max_kv) / PREFILL_LMIN;
  const int64_t parts = fit < most ? fit : most;
  return parts < 1 ? 1 : (int)parts;
}

struct PrefillWs {
  int kv_rows;
  size_t lay_off, gone_off, src_off, k_off, r_off, v_off, o_off, ml_off, rows_off, total;
};

// Requests start at multiples of 8 tokens, tiles of 64 tokens may read past
// the last one, and the expansion works on up to 256 tokens at a time.
PrefillWs prefill_ws(const kda_latent_config* cfg, int max_kv) {
  const int parts = cfg->pg.B < max_kv ? cfg->pg.B : max_kv;
  PrefillWs w;
  w.kv_rows = (max_kv + 7 * parts + 64 + 255) / 256 * 256;
  const size_t rows = (size_t)w.kv_rows;
  w.lay_off = 0;
  w.gone_off = up256((size_t)(3 * cfg->pg.B + 2) * sizeof(int32_t));
  w.src_off = up256(w.gone_off + (size_t)cfg->H * cfg->d_v / 32 * sizeof(int32_t));
  w.k_off = up256(w.src_off + rows * sizeof(int32_t));
  w.r_off = up256(w.k_off + rows * cfg->H * cfg->d_n * 2 * (cfg->dtype == KDA_F16 ? 2 : 1));   // hi (and lo) keys
  w.v_off = up256(w.r_off + rows * cfg->d_r * 2);
  w.o_off = up256(w.v_off + rows * cfg->H * cfg->d_v * 2);
  // any number of rows may come, but only these blocks if tokens are cut
  const bool cut = kda::prefill_longest(cfg->pg, max_kv) >= 2 * PREFILL_LMIN;
  const size_t part_rows = cut ? (size_t)PREFILL_BLOCKS * kda::PREFILL_ROWS : 0;
  w.ml_off = up256(w.o_off + part_rows * cfg->d_v * sizeof(float));
  w.rows_off = up256(w.ml_off + part_rows * 2 * sizeof(float));
  w.total = up256(w.rows_off + (cut ? (size_t)PREFILL_BLOCKS * 2 * sizeof(int32_t) : 0));
  return w;
}

// Rows of `len` elements at `stride`.
bool bad_rows(const void* ptr, int64_t stride, int64_t len) {
  return !aligned(ptr, 16) || stride < len || stride % 8 != 0;
}

// Scales belong to an 8-bit cache.
bool bad_scales(const kda_attn_config* cfg, const float* k_scale, const float* v_scale) {
  if (cfg->cache_dtype != KDA_E4M3) return k_scale != nullptr || v_scale != nullptr;
  return !aligned(k_scale, 4) || !aligned(v_scale, 4);
}

// Rows of H vectors of d elements, `head` apart.
bool bad_heads(const void* ptr, int64_t stride, int64_t head, int H, int d) {
  return head < d || head % 8 != 0 || bad_rows(ptr, stride, (int64_t)(H - 1) * head + d);
}

}  // namespace

extern "C" {

int kda_pages_plan(const kda_pages* pg, int32_t n_slots, const int32_t* lens,
                   const int32_t* new_tokens, const int32_t* n_free, int32_t* free_pages,
                   int32_t* tables, int32_t* lens_out, int32_t* n_free_out, int32_t* cu,
                   int32_t* slots, int32_t* ok, void* stream) {
  if (pg == nullptr) return KDA_ERR_ARG;
  const int st = check_pages(pg);
  if (st != KDA_OK) return st;
  if (n_slots < 1) return KDA_ERR_ARG;
  if (n_slots > MAX_ROWS) return KDA_ERR_UNSUPPORTED;
  const void* all[] = {lens, new_tokens, n_free, free_pages, tables, lens_out, n_free_out, cu, slots, ok};
  for (const void* x : all)
    if (x == nullptr || !aligned(x, 4)) return KDA_ERR_ARG;
  kda::PlanArgs a;
  a.pg = *pg;
  a.sh = log2_of(pg->page);
  a.n_slots = n_slots;
  a.lens = lens;
  a.newt = new_tokens;
  a.n_free = n_free;
  a.free_pages = free_pages;
  a.tables = tables;
  a.lens_out = lens_out;
  a.n_free_out = n_free_out;
  a.cu = cu;
  a.slots = slots;
  a.ok = ok;
  return hip_status(kda::launch_plan(a, (hipStream_t)stream));
}

int kda_attn_append(const kda_attn_config* cfg, int32_t n, const void* k, int64_t k_stride,
                    const void* v, int64_t v_stride, const int32_t* slots, const float* k_scale,
                    const float* v_scale, void* k_cache, void* v_cache, void* stream) {
  const int st = check_attn(cfg);
  if (st != KDA_OK) return st;
  if (n < 1) return KDA_ERR_ARG;
  if (n > MAX_ROWS) return KDA_ERR_UNSUPPORTED;
  if (!k || !v || !slots || !k_cache || !v_cache) return KDA_ERR_ARG;
  const int64_t len = (int64_t)cfg->H_kv * cfg->d;
  if (bad_rows(k, k_stride, len) || bad_rows(v, v_stride, len)) return KDA_ERR_ARG;
  if (!aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(slots, 4)) return KDA_ERR_ARG;
  if (bad_scales(cfg, k_scale, v_scale)) return KDA_ERR_ARG;
  kda::AppendArgs a;
  std::memset(&a, 0, sizeof(a));
  a.pg = cfg->pg;
  a.sh = log2_of(cfg->pg.page);
  a.n = n;
  a.H = cfg->H_kv;
  a.d = cfg->d;
  a.e4m3 = cfg->cache_dtype == KDA_E4M3;
  a.f16 = cfg->dtype == KDA_F16;
  a.a = k;
  a.b = v;
  a.a_stride = k_stride;
  a.b_stride = v_stride;
  a.slots = slots;
  a.a_scale = k_scale;
  a.b_scale = v_scale;
  a.a_cache = k_cache;
  a.b_cache = v_cache;
  return hip_status(kda::launch_append(a, false, (hipStream_t)stream));
}

size_t kda_attn_workspace_bytes(const kda_attn_config* cfg) {
  return check_attn(cfg) == KDA_OK ? attn_ws(cfg).total : 0;
}

int kda_attn_step(const kda_attn_config* cfg, const void* q, int64_t q_stride,
                  const void* k_cache, const void* v_cache, const int32_t* tables,
                  const int32_t* lens, const float* k_scale, const float* v_scale, void* o,
                  float* lse, void* ws, void* stream) {
  const int st = check_attn(cfg);
  if (st != KDA_OK) return st;
  if (!q || !k_cache || !v_cache || !tables || !lens || !o) return KDA_ERR_ARG;
  if (!ws) return KDA_ERR_WORKSPACE;
  if (bad_rows(q, q_stride, (int64_t)cfg->H_q * cfg->d)) return KDA_ERR_ARG;
  if (!aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(o, 16) || !aligned(ws, 16) ||
      !aligned(tables, 4) || !aligned(lens, 4) || !aligned(lse, 4) || bad_scales(cfg, k_scale, v_scale))
    return KDA_ERR_ARG;
  kda::AttnArgs a;
  std::memset(&a, 0, sizeof(a));
  a.pg = cfg->pg;
  a.sh = log2_of(cfg->pg.page);
  a.Hq = cfg->H_q;
  a.Hkv = cfg->H_kv;
  a.g = cfg->H_q / cfg->H_kv;
  a.mt = (a.g + 15) / 16;
  a.f16 = cfg->dtype == KDA_F16;
  a.e4m3 = cfg->cache_dtype == KDA_E4M3;
  a.d = cfg->d;
  a.extra = attn_extra(cfg);
  a.lmin = ATTN_LMIN;
  a.scale2 = (float)(cfg->scale * LOG2E);
  a.q = q;
  a.q_stride = q_stride;
  a.kc = k_cache;
  a.vc = v_cache;
  a.tables = tables;
  a.lens = lens;
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.o = o;
  a.lse = lse;
  const AttnWs w = attn_ws(cfg);
  a.part_o = (float*)((uint8_t*)ws + w.o_off);
  a.part_ml = (float*)((uint8_t*)ws + w.ml_off);
  a.reqs = (int32_t*)((uint8_t*)ws + w.req_off);
  return hip_status(kda::launch_attn_step(a, (hipStream_t)stream));
}

int kda_latent_append(const kda_latent_config* cfg, int32_t n, const void* c, int64_t c_stride,
                      const void* r, int64_t r_stride, const int32_t* slots, void* cache,
                      void* stream) {
  const int st = check_latent(cfg);
  if (st != KDA_OK) return st;
  if (n < 1) return KDA_ERR_ARG;
  if (n > MAX_ROWS) return KDA_ERR_UNSUPPORTED;
  if (!c || !r || !slots || !cache) return KDA_ERR_ARG;
  if (bad_rows(c, c_stride, cfg->d_c) || bad_rows(r, r_stride, cfg->d_r)) return KDA_ERR_ARG;
  if (!aligned(cache, 16) || !aligned(slots, 4)) return KDA_ERR_ARG;
  kda::AppendArgs a;
  std::memset(&a, 0, sizeof(a));
  a.pg = cfg->pg;
  a.sh = log2_of(cfg->pg.page);
  a.n = n;
  a.H = 1;
  a.d = cfg->d_c;
  a.d2 = cfg->d_r;
  a.a = c;
  a.b = r;
  a.a_stride = c_stride;
  a.b_stride = r_stride;
  a.slots = slots;
  a.a_cache = cache;
  return hip_status(kda::launch_append(a, true, (hipStream_t)stream));
}

size_t kda_latent_workspace_bytes(const kda_latent_config* cfg) {
  return check_latent(cfg) == KDA_OK ? latent_ws(cfg).total : 0;
}

int kda_latent_step(const kda_latent_config* cfg, const void* q_n, int64_t q_n_stride,
                    int64_t q_n_head, const void* q_r, int64_t q_r_stride, int64_t q_r_head,
                    const void* w_uk, const void* w_uv, const void* cache, const int32_t* tables,
                    const int32_t* lens, void* o, void* ws, void* stream) {
  const int st = check_latent(cfg);
  if (st != KDA_OK) return st;
  if (!q_n || !q_r || !w_uk || !w_uv || !cache || !tables || !lens || !o) return KDA_ERR_ARG;
  if (!ws) return KDA_ERR_WORKSPACE;
  if (bad_heads(q_n, q_n_stride, q_n_head, cfg->H, cfg->d_n) ||
      bad_heads(q_r, q_r_stride, q_r_head, cfg->H, cfg->d_r))
    return KDA_ERR_ARG;
  if (!aligned(w_uk, 16) || !aligned(w_uv, 16) || !aligned(cache, 16) || !aligned(o, 16) ||
      !aligned(ws, 16) || !aligned(tables, 4) || !aligned(lens, 4))
    return KDA_ERR_ARG;
  kda::LatentArgs a;
  std::memset(&a, 0, sizeof(a));
  a.pg = cfg->pg;
  a.sh = log2_of(cfg->pg.page);
  a.H = cfg->H;
  a.dn = cfg->d_n;
  a.dr = cfg->d_r;
  a.dc = cfg->d_c;
  a.f16 = cfg->dtype == KDA_F16;
  a.extra = latent_extra(cfg);
  a.lmin = LATENT_LMIN;
  a.scale2 = (float)(cfg->scale * LOG2E);
  a.qn = q_n;
  a.qr = q_r;
  a.qn_stride = q_n_stride;
  a.qn_head = q_n_head;
  a.qr_stride = q_r_stride;
  a.qr_head = q_r_head;
  a.w_uk = w_uk;
  a.w_uv = w_uv;
  a.cache = cache;
  a.tables = tables;
  a.lens = lens;
  a.o = o;
  const LatentWs w = latent_ws(cfg);
  a.qa = (uint8_t*)ws + w.qa_off;
  a.part_o = (float*)((uint8_t*)ws + w.o_off);
  a.part_ml = (float*)((uint8_t*)ws + w.ml_off);
  a.reqs = (int32_t*)((uint8_t*)ws + w.req_off);
  a.items = (int32_t*)((uint8_t*)ws + w.item_off);
  return hip_status(kda::launch_latent_step(a, (hipStream_t)stream));
}

size_t kda_latent_prefill_workspace_bytes(const kda_latent_config* cfg, int32_t max_kv) {
  if (check_latent(cfg) != KDA_OK || max_kv < 1 || max_kv > MAX_PROMPT) return 0;
  return prefill_ws(cfg, max_kv).total;
}

int kda_latent_prefill(const kda_latent_config* cfg, int32_t n, int32_t max_kv, const void* q_n,
                       int64_t q_n_stride, int64_t q_n_head, const void* q_r, int64_t q_r_stride,
                       int64_t q_r_head, const int32_t* cu, const void* w_uk, const void* w_uv,
                       const void* cache, const int32_t* tables, const int32_t* lens, void* o,
                       void* ws, void* stream) {
  const int st = check_latent(cfg);
  if (st != KDA_OK) return st;
  if (n < 1 || max_kv < 1) return KDA_ERR_ARG;
  if (n > MAX_PROMPT || max_kv > MAX_PROMPT) return KDA_ERR_UNSUPPORTED;
  if (!q_n || !q_r || !cu || !w_uk || !w_uv || !cache || !tables || !lens || !o) return KDA_ERR_ARG;
  if (!ws) return KDA_ERR_WORKSPACE;
  if (bad_heads(q_n, q_n_stride, q_n_head, cfg->H, cfg->d_n) ||
      bad_heads(q_r, q_r_stride, q_r_head, cfg->H, cfg->d_r))
    return KDA_ERR_ARG;
  if (!aligned(w_uk, 16) || !aligned(w_uv, 16) || !aligned(cache, 16) || !aligned(o, 16) ||
      !aligned(ws, 16) || !aligned(cu, 4) || !aligned(tables, 4) || !aligned(lens, 4))
    return KDA_ERR_ARG;
  kda::LatentPrefillArgs a;
  std::memset(&a, 0, sizeof(a));
  a.pg = cfg->pg;
  a.sh = log2_of(cfg->pg.page);
  a.H = cfg->H;
  a.dn = cfg->d_n;
  a.dr = cfg->d_r;
  a.dc = cfg->d_c;
  a.f16 = cfg->dtype == KDA_F16;
  a.n = n;
  a.max_kv = max_kv;
  a.scale2 = (float)(cfg->scale * LOG2E);
  a.qn = q_n;
  a.qr = q_r;
  a.qn_stride = q_n_stride;
  a.qn_head = q_n_head;
  a.qr_stride = q_r_stride;
  a.qr_head = q_r_head;
  a.cu = cu;
  a.tables = tables;
  a.lens = lens;
  a.w_uk = w_uk;
  a.w_uv = w_uv;
  a.cache = cache;
  a.o = o;
  const PrefillWs w = prefill_ws(cfg, max_kv);
  a.kv_rows = w.kv_rows;
  a.lay = (int32_t*)((uint8_t*)ws + w.lay_off);
  a.gone = (int32_t*)((uint8_t*)ws + w.gone_off);
  a.src = (int32_t*)((uint8_t*)ws + w.src_off);
  a.ke = (uint8_t*)ws + w.k_off;
  a.re = (uint8_t*)ws + w.r_off;
  a.ve = (uint8_t*)ws + w.v_off;
  a.parts = prefill_parts(cfg, n, max_kv);
  a.part_o = (float*)((uint8_t*)ws + w.o_off);
  a.part_ml = (float*)((uint8_t*)ws + w.ml_off);
  a.part_rows = (int32_t*)((uint8_t*)ws + w.rows_off);
  return hip_status(kda::launch_latent_prefill(a, (hipStream_t)stream));
}

}  // extern "C"
