// Host side of the operators around the paged 8-bit cache: argument validation and the C ABI entry points.
// Every check runs before any HIP call so that invalid input never reaches a kernel.
#include <hip/hip_runtime.h>

#include "fluxbin_quant_checks.h"
#include "fluxbin_serve_internal.h"

namespace fluxbin {

namespace {

// A strided tensor of rows whose extent is `row` elements of 2 bytes.
struct Rows {
  const uint16_t* p;
  int64_t ts, hs, rows, row;
  Range range;
};

// Whether two of them have no byte in common: apart as a whole, or side by side in rows of one stride.
bool apart(const Rows& a, const Rows& b) {
  if (!any_overlap({a.range}, {b.range})) return true;
  if (a.ts != b.ts || a.row > a.ts || b.row > b.ts) return false;
  const int64_t d = (int64_t(reinterpret_cast<uintptr_t>(b.p)) - int64_t(reinterpret_cast<uintptr_t>(a.p))) / 2;
  if ((reinterpret_cast<uintptr_t>(b.p) ^ reinterpret_cast<uintptr_t>(a.p)) & 1) return false;
  const int64_t at = ((d % a.ts) + a.ts) % a.ts;   // where b's rows start in a's
  return at >= a.row && at + b.row <= a.ts;
}

bool same(const Rows& a, const Rows& b) { return a.p == b.p && a.ts == b.ts && a.hs == b.hs; }

fluxbin_status check_rows(const char* name, const uint16_t* p, int64_t rows, int32_t heads, int32_t D, int64_t ts, int64_t hs,
                          bool written, Rows* r) {
  const fluxbin_status st = check_strided(name, p, rows, heads, D, ts, hs, written, &r->range);
  if (st != FLUXBIN_OK) return st;
  r->p = p;
  r->ts = ts;
  r->hs = hs;
  r->rows = rows;
  r->row = int64_t(heads - 1) * hs + D;
  return FLUXBIN_OK;
}

fluxbin_status check_pool(const fluxbin_page_pool* p, PoolArgs* a) {
  if (!p) return fail(FLUXBIN_ERR_INVALID_ARG, "pool is NULL");
  const fluxbin_status st = check_kv8_sizes(p->pages, p->page_size, 1, 64);
  if (st != FLUXBIN_OK) return st;
  if (!p->d_state || misaligned(p->d_state, 16))
    return fail(FLUXBIN_ERR_INVALID_ARG, "the pool's state is NULL or not 16-byte aligned");
  a->state = p->d_state;
  a->pages = int32_t(p->pages);
  a->pshift = 0;
  while ((1 << a->pshift) < p->page_size) ++a->pshift;
  return FLUXBIN_OK;
}

Range state_range(const fluxbin_page_pool& p) { return {p.d_state, (uint64_t(p.pages) + 4) * 4}; }

fluxbin_status check_table(const char* name, const int32_t* t, int32_t rows, int32_t blocks, int64_t stride, Range* r) {
  if (rows < 1 || rows > 65535) return fail(FLUXBIN_ERR_INVALID_ARG, "%s: %d rows, out of range [1, 65535]", name, rows);
  if (blocks < 1 || blocks > (1 << 24))
    return fail(FLUXBIN_ERR_INVALID_ARG, "%s: %d columns, out of range [1, 2^24]", name, blocks);
  if (stride < blocks || stride > (int64_t(1) << 40))
    return fail(FLUXBIN_ERR_INVALID_ARG, "%s: row stride %lld < its columns", name, (long long)stride);
  if (!t || misaligned(t, 4)) return fail(FLUXBIN_ERR_INVALID_ARG, "%s is NULL or not aligned to its elements", name);
  *r = {t, (uint64_t(rows - 1) * uint64_t(stride) + uint64_t(blocks)) * 4};
  return FLUXBIN_OK;
}

}  // namespace

extern "C" {

fluxbin_status fluxbin_qk_rotate(const fluxbin_rotary* rotary, int64_t rows, const int32_t* d_positions, int32_t q_heads,
                                 const uint16_t* d_q, int64_t q_token_stride, int64_t q_head_stride, uint16_t* d_q_out,
                                 int64_t q_out_token_stride, int64_t q_out_head_stride, int32_t k_heads,
                                 const uint16_t* d_k, int64_t k_token_stride, int64_t k_head_stride, uint16_t* d_k_out,
                                 int64_t k_out_token_stride, int64_t k_out_head_stride, hipStream_t stream) {
  clear_error();
  if (!rotary) return fail(FLUXBIN_ERR_INVALID_ARG, "rotary is NULL");
  const int32_t D = rotary->head_dim, R = rotary->rotary_dim;
  if (D < 1) return fail(FLUXBIN_ERR_INVALID_ARG, "head_dim = %d must be >= 1", D);
  if (D != 64 && D != 128 && D != 256)
    return fail(FLUXBIN_ERR_UNSUPPORTED, "head_dim = %d: supported are 64, 128, 256", D);
  if (R < 0 || R > D) return fail(FLUXBIN_ERR_INVALID_ARG, "rotary_dim = %d out of range [0, head_dim]", R);
  if (R % 16 != 0) return fail(FLUXBIN_ERR_UNSUPPORTED, "rotary_dim = %d: supported are multiples of 16", R);
  if (rotary->interleaved != 0 && rotary->interleaved != 1)
    return fail(FLUXBIN_ERR_INVALID_ARG, "interleaved must be 0 or 1");
  if (!(rotary->eps >= 0.f && rotary->eps < 1e30f)) return fail(FLUXBIN_ERR_INVALID_ARG, "eps must be a number >= 0");
  if (!(rotary->magnitude > -1e30f && rotary->magnitude < 1e30f))
    return fail(FLUXBIN_ERR_INVALID_ARG, "magnitude must be a finite number");
  if (R > 0 && !rotary->d_frequencies) return fail(FLUXBIN_ERR_INVALID_ARG, "frequencies are NULL");
  if (misaligned(rotary->d_frequencies, 4) || misaligned(rotary->d_q_weight, 4) || misaligned(rotary->d_k_weight, 4))
    return fail(FLUXBIN_ERR_INVALID_ARG, "frequencies or weights are not aligned to their elements");
  if (rows < 0 || rows > (int64_t(1) << 22))
    return fail(FLUXBIN_ERR_INVALID_ARG, "rows = %lld out of range [0, 2^22]", (long long)rows);
  if (q_heads < 1 || q_heads > 1024) return fail(FLUXBIN_ERR_INVALID_ARG, "q_heads = %d out of range [1, 1024]", q_heads);
  if (k_heads < 0 || k_heads > 1024) return fail(FLUXBIN_ERR_INVALID_ARG, "k_heads = %d out of range [0, 1024]", k_heads);
  if (rows * (q_heads + k_heads) * D > (int64_t(1) << 35))   // the kernel's grid has fewer than 2^32 threads
    return fail(FLUXBIN_ERR_UNSUPPORTED, "rows * heads * head_dim exceeds 2^35");
  if (rows > 0 && R > 0 && (!d_positions || misaligned(d_positions, 4)))
    return fail(FLUXBIN_ERR_INVALID_ARG, "positions are NULL or not aligned to their elements");
  Rows q, qo, k{}, ko{};
  fluxbin_status st = check_rows("q", d_q, rows, q_heads, D, q_token_stride, q_head_stride, false, &q);
  if (st != FLUXBIN_OK) return st;
  st = check_rows("q_out", d_q_out, rows, q_heads, D, q_out_token_stride, q_out_head_stride, true, &qo);
  if (st != FLUXBIN_OK) return st;
  if (k_heads > 0) {
    st = check_rows("k", d_k, rows, k_heads, D, k_token_stride, k_head_stride, false, &k);
    if (st != FLUXBIN_OK) return st;
    st = check_rows("k_out", d_k_out, rows, k_heads, D, k_out_token_stride, k_out_head_stride, true, &ko);
    if (st != FLUXBIN_OK) return st;
  }
  bool clear = (same(q, qo) || apart(q, qo));
  if (k_heads > 0) clear = clear && (same(k, ko) || apart(k, ko)) && apart(qo, k) && apart(qo, ko) && apart(ko, q);
  const Range pos{R > 0 ? d_positions : nullptr, uint64_t(rows) * 4}, freq{rotary->d_frequencies, uint64_t(R) * 2};
  const Range wq{rotary->d_q_weight, uint64_t(D) * 4}, wk{k_heads > 0 ? rotary->d_k_weight : nullptr, uint64_t(D) * 4};
  if (!clear || any_overlap({qo.range}, {pos, freq, wq, wk}) || any_overlap({ko.range}, {pos, freq, wq, wk}))
    return fail(FLUXBIN_ERR_INVALID_ARG, "the outputs overlap each other or the inputs");
  if (rows == 0) return FLUXBIN_OK;
  RotateArgs a{};
  a.side[0] = {d_q, d_q_out, rotary->d_q_weight, q_token_stride, q_head_stride, q_out_token_stride, q_out_head_stride};
  a.side[1] = {d_k, d_k_out, k_heads > 0 ? rotary->d_k_weight : nullptr, k_token_stride, k_head_stride, k_out_token_stride,
               k_out_head_stride};
  a.positions = d_positions;
  a.freq = rotary->d_frequencies;
  a.rows = rows;
  a.Hq = q_heads;
  a.H = q_heads + k_heads;
  a.R = R;
  a.eps = rotary->eps;
  a.magnitude = rotary->magnitude;
  return launch_qk_rotate(a, D, rotary->interleaved, stream);
}

fluxbin_status fluxbin_tree_masks(int64_t rows, int32_t sequences, const int32_t* d_offsets, const int32_t* d_context,
                                  const int32_t* d_parents, int32_t words, uint64_t* d_masks, int32_t* d_positions,
                                  hipStream_t stream) {
  clear_error();
  const fluxbin_status st = check_kv8_rows(rows, sequences);
  if (st != FLUXBIN_OK) return st;
  if (words < 1) return fail(FLUXBIN_ERR_INVALID_ARG, "words = %d must be >= 1", words);
  if (words > kTreeMaxWords) return fail(FLUXBIN_ERR_UNSUPPORTED, "words = %d: supported are up to %d", words, kTreeMaxWords);
  if (!d_offsets || !d_context) return fail(FLUXBIN_ERR_INVALID_ARG, "offsets or context is NULL");
  if (rows > 0 && (!d_parents || !d_masks)) return fail(FLUXBIN_ERR_INVALID_ARG, "parents or masks are NULL");
  if (misaligned(d_offsets, 4) || misaligned(d_context, 4) || misaligned(d_parents, 4) || misaligned(d_positions, 4) ||
      misaligned(d_masks, 8))
    return fail(FLUXBIN_ERR_INVALID_ARG, "an array is not aligned to its elements");
  if (any_overlap({{d_masks, uint64_t(rows) * uint64_t(words) * 8}, {d_positions, uint64_t(rows) * 4}},
                  {{d_offsets, (uint64_t(sequences) + 1) * 4}, {d_context, uint64_t(sequences) * 4},
                   {d_parents, uint64_t(rows) * 4}}))
    return fail(FLUXBIN_ERR_INVALID_ARG, "masks, positions and the inputs overlap");
  if (rows == 0) return FLUXBIN_OK;
  MasksArgs a{d_offsets, d_context, d_parents, d_masks, d_positions, int32_t(rows), sequences, words};
  return launch_tree_masks(a, stream);
}

fluxbin_status fluxbin_kv8_tree_workspace_query(const fluxbin_kv8_cache* cache, int64_t rows, int32_t sequences,
                                                int32_t q_heads, size_t* bytes) {
  clear_error();
  fluxbin_status st = check_kv8_cache(cache);
  if (st != FLUXBIN_OK) return st;
  st = check_kv8_rows(rows, sequences);
  if (st != FLUXBIN_OK) return st;
  if (q_heads < 1 || q_heads > 1024 || q_heads % cache->kv_heads != 0)
    return fail(FLUXBIN_ERR_INVALID_ARG, "q_heads = %d must be a multiple of kv_heads, up to 1024", q_heads);
  if (!bytes) return fail(FLUXBIN_ERR_INVALID_ARG, "bytes is NULL");
  const int cus = device_cu_count();
  if (cus < 1) return fail(FLUXBIN_ERR_HIP, "reading the device's CU count failed");
  *bytes = size_t(kv8_tree_workspace(cache->head_dim, cus));
  return FLUXBIN_OK;
}

fluxbin_status fluxbin_kv8_tree_attention(const fluxbin_kv8_cache* cache, const fluxbin_kv8_batch* batch, int32_t q_heads,
                                          const uint16_t* d_q, int64_t q_token_stride, int64_t q_head_stride,
                                          uint16_t* d_out, int64_t out_token_stride, int64_t out_head_stride,
                                          float softmax_scale, const uint64_t* d_masks, int32_t words, int32_t window,
                                          void* d_workspace, size_t workspace_bytes, hipStream_t stream) {
  clear_error();
  Kv8AttnArgs a{};
  fluxbin_status st = check_kv8_call(cache, batch, &a.c);
  if (st != FLUXBIN_OK) return st;
  const int32_t H = cache->kv_heads, D = cache->head_dim;
  if (q_heads < 1 || q_heads > 1024 || q_heads % H != 0)
    return fail(FLUXBIN_ERR_INVALID_ARG, "q_heads = %d must be a multiple of kv_heads, up to 1024", q_heads);
  if (batch->rows * (q_heads / H) > (int64_t(1) << 30))   // rows times heads of a group are 32-bit numbers
    return fail(FLUXBIN_ERR_UNSUPPORTED, "rows * (q_heads / kv_heads) exceeds 2^30");
  if (!(softmax_scale > -1e30f && softmax_scale < 1e30f))
    return fail(FLUXBIN_ERR_INVALID_ARG, "softmax_scale must be a finite number");
  if (words < 1) return fail(FLUXBIN_ERR_INVALID_ARG, "words = %d must be >= 1", words);
  if (words > kTreeMaxWords) return fail(FLUXBIN_ERR_UNSUPPORTED, "words = %d: supported are up to %d", words, kTreeMaxWords);
  if (window < 0) return fail(FLUXBIN_ERR_INVALID_ARG, "window = %d must be >= 0", window);
  if (batch->rows > 0 && (!d_masks || misaligned(d_masks, 8)))
    return fail(FLUXBIN_ERR_INVALID_ARG, "masks are NULL or not aligned to their elements");
  Range q, out;
  st = check_strided("q", d_q, batch->rows, q_heads, D, q_token_stride, q_head_stride, false, &q);
  if (st != FLUXBIN_OK) return st;
  st = check_strided("out", d_out, batch->rows, q_heads, D, out_token_stride, out_head_stride, true, &out);
  if (st != FLUXBIN_OK) return st;
  const int cus = device_cu_count();
  if (cus < 1) return fail(FLUXBIN_ERR_HIP, "reading the device's CU count failed");
  const uint64_t need = kv8_tree_workspace(D, cus);
  if (workspace_bytes < need)
    return fail(FLUXBIN_ERR_BUFFER_TOO_SMALL, "workspace has %zu bytes, needs %llu", workspace_bytes,
                (unsigned long long)need);
  if (!d_workspace || misaligned(d_workspace, 16))
    return fail(FLUXBIN_ERR_INVALID_ARG, "workspace is NULL or not 16-byte aligned");
  if (any_overlap({out, {d_workspace, need}},
                  {q, {cache->d_base, cache->bytes}, table_range(*batch), offsets_range(*batch), context_range(*batch),
                   {d_masks, uint64_t(batch->rows) * uint64_t(words) * 8}}))
    return fail(FLUXBIN_ERR_INVALID_ARG, "out, the workspace and the inputs overlap");
  if (batch->rows == 0) return FLUXBIN_OK;
  a.q = d_q;
  a.out = d_out;
  a.part = static_cast<float*>(d_workspace);
  a.qts = q_token_stride;
  a.qhs = q_head_stride;
  a.ots = out_token_stride;
  a.ohs = out_head_stride;
  a.G = q_heads / H;
  a.window = window;
  a.masks = d_masks;
  a.words = words;
  a.scale2 = softmax_scale * 1.4426950408889634f;
  return launch_kv8_tree_attention(a, D, cus, stream);
}

fluxbin_status fluxbin_kv8_keep(const fluxbin_kv8_cache* cache, const fluxbin_kv8_batch* batch, const int32_t* d_keep,
                                const int32_t* d_kept, hipStream_t stream) {
  clear_error();
  Kv8KeepArgs a{};
  const fluxbin_status st = check_kv8_call(cache, batch, &a.c);
  if (st != FLUXBIN_OK) return st;
  if (!d_kept || (batch->rows > 0 && !d_keep)) return fail(FLUXBIN_ERR_INVALID_ARG, "keep or kept is NULL");
  if (misaligned(d_keep, 4) || misaligned(d_kept, 4))
    return fail(FLUXBIN_ERR_INVALID_ARG, "keep or kept is not aligned to its elements");
  if (any_overlap({{cache->d_base, cache->bytes}},
                  {{d_keep, uint64_t(batch->rows) * 4}, {d_kept, uint64_t(batch->sequences) * 4}, table_range(*batch),
                   offsets_range(*batch), context_range(*batch)}))
    return fail(FLUXBIN_ERR_INVALID_ARG, "the cache overlaps an input");
  if (batch->rows == 0) return FLUXBIN_OK;
  const int cus = device_cu_count();
  if (cus < 1) return fail(FLUXBIN_ERR_HIP, "reading the device's CU count failed");
  a.keep = d_keep;
  a.kept = d_kept;
  return launch_kv8_keep(a, cache->head_dim, cus, stream);
}

fluxbin_status fluxbin_pages_resize(const fluxbin_page_pool* pool, int32_t sequences, int32_t max_blocks,
                                    int32_t* d_block_table, int64_t block_table_stride, const int32_t* d_tokens,
                                    hipStream_t stream) {
  clear_error();
  ResizeArgs a{};
  fluxbin_status st = check_pool(pool, &a.pool);
  if (st != FLUXBIN_OK) return st;
  Range table;
  st = check_table("block table", d_block_table, sequences, max_blocks, block_table_stride, &table);
  if (st != FLUXBIN_OK) return st;
  if (!d_tokens || misaligned(d_tokens, 4))
    return fail(FLUXBIN_ERR_INVALID_ARG, "tokens are NULL or not aligned to their elements");
  if (any_overlap({table, state_range(*pool)}, {{d_tokens, uint64_t(sequences) * 4}}))
    return fail(FLUXBIN_ERR_INVALID_ARG, "the block table, the pool's state and the tokens overlap");
  a.table = d_block_table;
  a.stride = block_table_stride;
  a.tokens = d_tokens;
  a.B = sequences;
  a.max_blocks = max_blocks;
  return launch_pages_resize(a, stream);
}

fluxbin_status fluxbin_pages_fork(const fluxbin_page_pool* pool, int32_t sequences, int32_t max_blocks,
                                  const int32_t* d_block_table, int64_t block_table_stride, const int32_t* d_context,
                                  int32_t children, int32_t child_blocks, int32_t* d_child_table,
                                  int64_t child_table_stride, const int32_t* d_source, int32_t* d_copies,
                                  hipStream_t stream) {
  clear_error();
  ForkArgs a{};
  fluxbin_status st = check_pool(pool, &a.pool);
  if (st != FLUXBIN_OK) return st;
  Range table, child;
  st = check_table("block table", d_block_table, sequences, max_blocks, block_table_stride, &table);
  if (st != FLUXBIN_OK) return st;
  st = check_table("child table", d_child_table, children, child_blocks, child_table_stride, &child);
  if (st != FLUXBIN_OK) return st;
  if (!d_context || !d_source || !d_copies)
    return fail(FLUXBIN_ERR_INVALID_ARG, "context, source or copies is NULL");
  if (misaligned(d_context, 4) || misaligned(d_source, 4) || misaligned(d_copies, 8))
    return fail(FLUXBIN_ERR_INVALID_ARG, "context or source is not aligned to its elements, or copies not to 8 bytes");
  if (any_overlap({child, state_range(*pool), {d_copies, uint64_t(children) * 8}},
                  {table, {d_context, uint64_t(sequences) * 4}, {d_source, uint64_t(children) * 4}}))
    return fail(FLUXBIN_ERR_INVALID_ARG, "the child table, copies, the pool's state and the inputs overlap");
  a.table = d_block_table;
  a.stride = block_table_stride;
  a.context = d_context;
  a.child = d_child_table;
  a.child_stride = child_table_stride;
  a.source = d_source;
  a.copies = d_copies;
  a.B = sequences;
  a.max_blocks = max_blocks;
  a.C = children;
  a.child_blocks = child_blocks;
  return launch_pages_fork(a, stream);
}

fluxbin_status fluxbin_kv8_copy_pages(const fluxbin_kv8_cache* to, const fluxbin_kv8_cache* from, int64_t copies,
                                      const int32_t* d_copies, hipStream_t stream) {
  clear_error();
  fluxbin_status st = check_kv8_cache(to);
  if (st != FLUXBIN_OK) return st;
  st = check_kv8_cache(from);
  if (st != FLUXBIN_OK) return st;
  if (to->page_size != from->page_size || to->kv_heads != from->kv_heads || to->head_dim != from->head_dim)
    return fail(FLUXBIN_ERR_INVALID_ARG, "the caches differ in page_size, kv_heads or head_dim");
  const bool one = to->d_base == from->d_base && to->pages == from->pages;
  if (copies < 0 || copies > (int64_t(1) << 22))
    return fail(FLUXBIN_ERR_INVALID_ARG, "copies = %lld out of range [0, 2^22]", (long long)copies);
  if (copies > 0 && (!d_copies || misaligned(d_copies, 8)))
    return fail(FLUXBIN_ERR_INVALID_ARG, "copies are NULL or not aligned to 8 bytes");
  const Range pairs{d_copies, uint64_t(copies) * 8};
  if (any_overlap({{to->d_base, to->bytes}}, {pairs}) ||
      (!one && any_overlap({{to->d_base, to->bytes}}, {{from->d_base, from->bytes}})))
    return fail(FLUXBIN_ERR_INVALID_ARG, "the caches and the list of copies overlap");
  if (copies == 0) return FLUXBIN_OK;
  const fluxbin_kv8_cache* c[2] = {from, to};
  CopyArgs a{};
  for (int i = 0; i < 2; ++i) {
    const Kv8Derived d = kv8_derive(c[i]->pages, c[i]->page_size, c[i]->kv_heads, c[i]->head_dim);
    uint8_t* base = static_cast<uint8_t*>(c[i]->d_base);
    float* scales[2] = {reinterpret_cast<float*>(base + d.off_ks), reinterpret_cast<float*>(base + d.off_vs)};
    for (int side = 0; side < 2; ++side) {
      uint8_t* codes = base + (side ? d.off_v : 0);
      if (i == 0) {
        a.from[side] = codes;
        a.from_scales[side] = scales[side];
      } else {
        a.to[side] = codes;
        a.to_scales[side] = scales[side];
      }
    }
  }
  a.copies = d_copies;
  a.n = copies;
  a.page_bytes = int64_t(to->kv_heads) * to->page_size * to->head_dim;
  a.Hkv = to->kv_heads;
  a.from_pages = int32_t(from->pages);
  a.to_pages = int32_t(to->pages);
  return launch_kv8_copy_pages(a, stream);
}

}  // extern "C"

}  // namespace fluxbin
