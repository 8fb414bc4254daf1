// pp_serve.cpp -- host side of the prefix cache: the two host layouts, the
// argument checks of the device operators and their C entries.  The
// operators allocate nothing and wait for nothing.

#include "pp_internal.h"
#include "pp_serve.h"

#include <cmath>
#include <new>
#include <vector>

using namespace pp;

namespace {

bool pow2_page(int32_t ps) { return ps >= 16 && ps <= 1024 && (ps & (ps - 1)) == 0; }

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Rows whose starts are 16-byte aligned, whatever their numbers.
bool row_layout(const void* p, int64_t size, int64_t s0, int64_t s1, int64_t s2 = 0) {
  auto ok = [](int64_t s) { return s >= 0 && s < (int64_t)1 << 48; };   // bytes stay within 64 bits
  return aligned16(p) && ok(s0) && ok(s1) && ok(s2) && s0 * size % 16 == 0 &&
         s1 * size % 16 == 0 && s2 * size % 16 == 0;
}

// Rows that are written: those next to each other in a dimension of `count` do not overlap.
bool apart(int64_t count, int64_t stride, int32_t dim) { return count < 2 || stride >= dim; }

int64_t size_of(int32_t dtype) { return dtype == PP_E4M3 ? 1 : 2; }

bool row_type(int32_t t) { return t == PP_BF16 || t == PP_F16; }

int check_pages(const pp_kv_pages* p, int32_t dtype) {
  if (!p || !p->k || !p->v) return report(PP_E_ARG, "null pages");
  if (!row_type(dtype)) return report(PP_E_ARG, "rows are PP_BF16 or PP_F16");
  if (p->dtype != dtype && p->dtype != PP_E4M3)
    return report(PP_E_ARG, "pages hold the rows' type or PP_E4M3");
  if (p->dtype != PP_E4M3 && (p->k_scale || p->v_scale))
    return report(PP_E_ARG, "only PP_E4M3 pages have scales");
  if (p->n_pages < 1 || p->heads < 1) return report(PP_E_ARG, "need n_pages >= 1 and heads >= 1");
  if (!pow2_page(p->page_size))
    return report(PP_E_UNSUPPORTED, "page_size is a power of two from 16 to 1,024");
  if (p->dim != 64 && p->dim != 128 && p->dim != 256)
    return report(PP_E_UNSUPPORTED, "dim is 64, 128 or 256");
  const int64_t size = size_of(p->dtype);
  if (!row_layout(p->k, size, p->page_stride, p->head_stride, p->token_stride) ||
      !row_layout(p->v, size, p->page_stride, p->head_stride, p->token_stride))
    return report(PP_E_ARG, "page rows start at 16-byte boundaries, at strides >= 0");
  // kernels keep offsets inside a page in 32 bits
  if (((__int128)(p->heads - 1) * p->head_stride + (__int128)(p->page_size - 1) * p->token_stride +
       p->dim) * size > (int64_t)1 << 31)
    return report(PP_E_UNSUPPORTED, "one page spans more than 2 GiB");
  return PP_OK;
}

int check_attention(const pp_kv_pages* p, const pp_attention_args* a) {
  if (!a) return report(PP_E_ARG, "null arguments");
  const int rc = check_pages(p, a->dtype);
  if (rc != PP_OK) return rc;
  if (a->requests < 0 || a->requests > 65536 || a->tokens < 0 || a->max_new < 0 ||
      a->max_len < 0 || a->max_blocks < 0 || a->window < 0 || a->row_stride < 0)
    return report(PP_E_ARG, "negative size, or more than 65,536 requests");
  if (a->q_heads < 1 || a->q_heads % p->heads != 0)
    return report(PP_E_ARG, "q_heads is a multiple of the pages' heads");
  if ((int64_t)a->tokens * a->q_heads > INT32_MAX)
    return report(PP_E_UNSUPPORTED, "tokens * q_heads exceeds 2^31 - 1");
  if ((int64_t)a->max_blocks * p->page_size > INT32_MAX)
    return report(PP_E_UNSUPPORTED, "max_blocks * page_size exceeds 2^31 - 1");
  if (!std::isfinite(a->scale)) return report(PP_E_ARG, "scale is not finite");
  return PP_OK;
}

// Nothing to do: no rows.
bool empty(const pp_attention_args& a) { return a.requests == 0 || a.tokens == 0 || a.max_new == 0; }

int launched(hipError_t e) {
  return e == hipSuccess ? PP_OK : report(PP_E_DEVICE, hipGetErrorString(e));
}

}  // namespace

extern "C" {

int pp_prefix_table(int32_t n, const int32_t* parent, int32_t* table) {
  report(PP_OK, "");
  if (n < 1 || !parent || !table) return report(PP_E_ARG, "bad arguments to pp_prefix_table");
  for (int32_t v = 0; v < n; ++v)
    if (parent[v] < -1 || parent[v] >= n || parent[v] == v)
      return report(PP_E_TREE, "a parent is out of range or the node itself");
  try {
    // depths from the root down: unwinding each path up to what is known
    std::vector<int32_t> depth(n, -1), path;
    for (int32_t v = 0; v < n; ++v) {
      int32_t u = v;
      path.clear();
      while (u >= 0 && depth[u] < 0) {
        if ((int64_t)path.size() >= n) return report(PP_E_TREE, "the parents have a cycle");
        path.push_back(u);
        u = parent[u];
      }
      int32_t d = u < 0 ? -1 : depth[u];
      for (auto it = path.rbegin(); it != path.rend(); ++it) depth[*it] = ++d;
    }
    for (int32_t v = 0; v < n; ++v) {
      int32_t* line = table + (int64_t)v * kLine;
      int32_t u = v;
      for (int j = 0; j < kLine - 1; ++j) {
        line[j] = u;
        if (u >= 0) u = parent[u];
      }
      line[kLine - 1] = depth[v];
    }
  } catch (const std::bad_alloc&) {
    return report(PP_E_NOMEM, "host allocation failed");
  }
  return PP_OK;
}

int pp_cache_slots(int32_t n, const uint8_t* target, const int32_t* held, int32_t n_slots,
                   int32_t* slot, int32_t* n_new) {
  report(PP_OK, "");
  if (n < 1 || n_slots < 0 || !target || !slot)
    return report(PP_E_ARG, "bad arguments to pp_cache_slots");
  int64_t want = 0;
  for (int32_t v = 0; v < n; ++v) want += target[v] != 0;
  if (want > n_slots) return report(PP_E_RANGE, "the target has more chunks than slots");
  try {
    std::vector<uint8_t> used(n_slots, 0), seen(n_slots, 0);
    if (held)
      for (int32_t v = 0; v < n; ++v) {
        const int32_t s = held[v];
        if (s < 0) continue;
        if (s >= n_slots || seen[s])
          return report(PP_E_RANGE, "held names a slot out of range or twice");
        seen[s] = 1;
        if (target[v]) used[s] = 1;
      }
    int32_t next = 0, fresh = 0;
    for (int32_t v = 0; v < n; ++v) {
      const int32_t s = held ? held[v] : -1;
      if (!target[v]) {
        slot[v] = -1;
      } else if (s >= 0) {
        slot[v] = s;
      } else {
        while (used[next]) ++next;
        slot[v] = next++;
        ++fresh;
      }
    }
    if (n_new) *n_new = fresh;
  } catch (const std::bad_alloc&) {
    return report(PP_E_NOMEM, "host allocation failed");
  }
  return PP_OK;
}

int pp_block_tables(const pp_block_args* a, void* hip_stream) {
  report(PP_OK, "");
  if (!a) return report(PP_E_ARG, "null arguments");
  if (a->requests < 0 || a->requests > 65536 || a->n < 0 || a->n_slots < 0 || a->n_free < 0 ||
      a->max_blocks < 0 || a->max_tokens < 0 || a->max_new < 0 || a->row_stride < 0)
    return report(PP_E_ARG, "negative size, or more than 65,536 requests");
  if (!pow2_page(a->page_size))
    return report(PP_E_UNSUPPORTED, "page_size is a power of two from 16 to 1,024");
  if (a->chunk_tokens < a->page_size || a->chunk_tokens % a->page_size != 0)
    return report(PP_E_ARG, "chunk_tokens is a multiple of page_size");
  if ((int64_t)a->n_slots * (a->chunk_tokens / a->page_size) > INT32_MAX ||
      (int64_t)a->max_blocks * a->page_size > INT32_MAX)
    return report(PP_E_UNSUPPORTED, "page numbers or tokens of a row exceed 2^31 - 1");
  if (!a->query_start || !a->taken ||
      (a->requests && (!a->leaf || !a->length || !a->cached || !a->start || !a->end)) ||
      (a->requests && a->max_blocks && !a->block_table) ||
      (a->n && (!a->prefix_table || !a->slot)) || (a->n_free && !a->free_pages) ||
      (a->max_tokens && (!a->slot_map || !a->position)))
    return report(PP_E_ARG, "null pointer");
  if (!aligned16(a->prefix_table)) return report(PP_E_ARG, "prefix_table is 16-byte aligned");
  if (a->requests > 1 && a->row_stride < a->max_blocks)
    return report(PP_E_ARG, "rows of block_table overlap");   // they are written
  return launched(launch_block_tables(*a, (hipStream_t)hip_stream));
}

int pp_kv_write(const pp_kv_pages* pages, int32_t tokens, int32_t dtype, const void* k,
                int64_t k_token_stride, int64_t k_head_stride, const void* v,
                int64_t v_token_stride, int64_t v_head_stride, const int64_t* slot_map,
                void* hip_stream) {
  report(PP_OK, "");
  const int rc = check_pages(pages, dtype);
  if (rc != PP_OK) return rc;
  if (tokens < 0) return report(PP_E_ARG, "negative size");
  if (tokens == 0) return PP_OK;
  if (!apart(pages->n_pages, pages->page_stride, pages->dim) ||
      !apart(pages->heads, pages->head_stride, pages->dim) ||
      !apart(pages->page_size, pages->token_stride, pages->dim))
    return report(PP_E_ARG, "rows of the pages overlap");
  if (!k || !v || !slot_map) return report(PP_E_ARG, "null pointer");
  if (!row_layout(k, 2, k_token_stride, k_head_stride) ||
      !row_layout(v, 2, v_token_stride, v_head_stride))
    return report(PP_E_ARG, "rows start at 16-byte boundaries, at strides >= 0");
  return launched(launch_kv_write(*pages, tokens, dtype, k, k_token_stride, k_head_stride, v,
                                  v_token_stride, v_head_stride, slot_map,
                                  (hipStream_t)hip_stream));
}

int64_t pp_attention_workspace(const pp_kv_pages* pages, const pp_attention_args* args) {
  report(PP_OK, "");
  const int rc = check_attention(pages, args);
  if (rc != PP_OK) return rc;
  return empty(*args) ? 0 : attention_workspace(*pages, *args);
}

int pp_paged_attention(const pp_kv_pages* pages, const pp_attention_args* a, void* hip_stream) {
  report(PP_OK, "");
  const int rc = check_attention(pages, a);
  if (rc != PP_OK) return rc;
  if (empty(*a)) return PP_OK;
  if (!a->q || !a->out || !a->query_start || !a->length || (a->max_blocks && !a->block_table))
    return report(PP_E_ARG, "null pointer");
  if (!row_layout(a->q, 2, a->q_token_stride, a->q_head_stride) ||
      !row_layout(a->out, 2, a->out_token_stride, a->out_head_stride))
    return report(PP_E_ARG, "rows start at 16-byte boundaries, at strides >= 0");
  if (!apart(a->tokens, a->out_token_stride, pages->dim) || !apart(a->q_heads, a->out_head_stride, pages->dim))
    return report(PP_E_ARG, "rows of out overlap");
  const int64_t need = attention_workspace(*pages, *a);
  if (need && (!a->workspace || ((uintptr_t)a->workspace & 255) || a->workspace_bytes < need))
    return report(PP_E_ARG, "workspace too small or not 256-byte aligned");
  return launched(launch_attention(*pages, *a, (hipStream_t)hip_stream));
}

}  // extern "C"
