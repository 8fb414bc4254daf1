// pp_serve.cpp -- host side of the prefix cache: the two host layouts, the
// argument checks of the device operators and their C entries.  The
// operators allocate nothing and wait for nothing.

#include "pp_internal.h"
#include "pp_serve.h"

#include <algorithm>
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

// Pages of keys and values, or with `alone` of one kind of rows only; any dim.
int check_layout(const pp_kv_pages* p, int32_t dtype, bool alone) {
  if (!p || !p->k || (!p->v && !alone)) return report(PP_E_ARG, "null pages");
  if (!row_type(dtype)) return report(PP_E_ARG, "rows are PP_BF16 or PP_F16");
  if (p->dtype != dtype && p->dtype != PP_E4M3)
    return report(PP_E_ARG, "pages hold the rows' type or PP_E4M3");
  if (p->dtype != PP_E4M3 && (p->k_scale || p->v_scale))
    return report(PP_E_ARG, "only PP_E4M3 pages have scales");
  if (p->n_pages < 1 || p->heads < 1) return report(PP_E_ARG, "need n_pages >= 1 and heads >= 1");
  if (!pow2_page(p->page_size))
    return report(PP_E_UNSUPPORTED, "page_size is a power of two from 16 to 1,024");
  return PP_OK;
}

// Strides of pages whose dim has been checked.
int check_strides(const pp_kv_pages* p) {
  const int64_t size = size_of(p->dtype);
  if (!row_layout(p->k, size, p->page_stride, p->head_stride, p->token_stride) ||
      (p->v && !row_layout(p->v, size, p->page_stride, p->head_stride, p->token_stride)))
    return report(PP_E_ARG, "page rows start at 16-byte boundaries, at strides >= 0");
  // kernels keep offsets inside a page in 32 bits
  if (((__int128)(p->heads - 1) * p->head_stride + (__int128)(p->page_size - 1) * p->token_stride +
       p->dim) * size > (int64_t)1 << 31)
    return report(PP_E_UNSUPPORTED, "one page spans more than 2 GiB");
  return PP_OK;
}

int check_pages(const pp_kv_pages* p, int32_t dtype) {
  const int rc = check_layout(p, dtype, false);
  if (rc != PP_OK) return rc;
  if (p->dim != 64 && p->dim != 128 && p->dim != 256)
    return report(PP_E_UNSUPPORTED, "dim is 64, 128 or 256");
  return check_strides(p);
}

// Rows of `dim` elements in up to three dimensions, one inside the other: no two of them overlap.
struct Dimension {
  int64_t count, stride;
};
bool nested(int32_t dim, Dimension a, Dimension b, Dimension c = {1, 0}) {
  Dimension d[3] = {a, b, c};
  std::sort(d, d + 3, [](const Dimension& x, const Dimension& y) { return x.stride < y.stride; });
  __int128 extent = dim;
  for (const Dimension& x : d) {
    if (x.count < 2) continue;
    if (x.stride < extent) return false;
    extent += (__int128)(x.count - 1) * x.stride;
  }
  return true;
}

int check_batch(const pp_kv_pages* p, const pp_attention_args* a) {
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

int check_attention(const pp_kv_pages* p, const pp_attention_args* a) {
  if (!a) return report(PP_E_ARG, "null arguments");
  const int rc = check_pages(p, a->dtype);
  return rc != PP_OK ? rc : check_batch(p, a);
}

int check_latent(const pp_kv_pages* p, int32_t value_dim, const pp_attention_args* a) {
  if (!a) return report(PP_E_ARG, "null arguments");
  int rc = check_layout(p, a->dtype, true);
  if (rc != PP_OK) return rc;
  if (p->v || p->v_scale) return report(PP_E_ARG, "pages of latent rows have no v");
  if (p->heads != 1) return report(PP_E_UNSUPPORTED, "pages of latent rows have one head");
  if ((value_dim != 256 && value_dim != 512) || p->dim != value_dim + 64)
    return report(PP_E_UNSUPPORTED, "value_dim is 256 or 512, dim 64 more");
  rc = check_strides(p);
  return rc != PP_OK ? rc : check_batch(p, a);
}

// Pointers, rows and workspace of a call that has rows; `out_dim` elements an output row.
int check_call(const pp_attention_args* a, int32_t out_dim, int64_t need) {
  if (!a->q || !a->out || !a->query_start || !a->length || (a->max_blocks && !a->block_table))
    return report(PP_E_ARG, "null pointer");
  if (!row_layout(a->q, 2, a->q_token_stride, a->q_head_stride) ||
      !row_layout(a->out, 2, a->out_token_stride, a->out_head_stride))
    return report(PP_E_ARG, "rows start at 16-byte boundaries, at strides >= 0");
  if (!apart(a->tokens, a->out_token_stride, out_dim) || !apart(a->q_heads, a->out_head_stride, out_dim))
    return report(PP_E_ARG, "rows of out overlap");
  if (need && (!a->workspace || ((uintptr_t)a->workspace & 255) || a->workspace_bytes < need))
    return report(PP_E_ARG, "workspace too small or not 256-byte aligned");
  return PP_OK;
}

// One kind of rows of pp_rotary_write; `weight` where norm is not 0.
int check_rotary_rows(int32_t tokens, int32_t heads, int32_t dim, int32_t first, int32_t norm, int32_t rot,
                      const void* in, int64_t token, int64_t head, const void* out, int64_t out_token,
                      int64_t out_head, const void* weight, bool to_out) {
  if (dim < 8 || dim > 1024 || dim % 8 || first < 0 || first % 8 || norm < 0 || norm % 8 || norm > dim ||
      (int64_t)first + rot > dim)
    return report(PP_E_UNSUPPORTED, "dims, firsts and norms are multiples of 8 within a dim of 1,024 at most");
  if (!in || (to_out && !out) || (norm && !weight)) return report(PP_E_ARG, "null pointer");
  if (!row_layout(in, 2, token, head) || (to_out && !row_layout(out, 2, out_token, out_head)) ||
      (norm && !aligned16(weight)))
    return report(PP_E_ARG, "rows and weights start at 16-byte boundaries, at strides >= 0");
  if (to_out && !nested(dim, {tokens, out_token}, {heads, out_head}))
    return report(PP_E_ARG, "rows of an output overlap");
  if (to_out && in == out && (token != out_token || head != out_head))
    return report(PP_E_ARG, "an output that is its input has its strides");
  return PP_OK;
}

// Whether rows of out_table and of block_table have entries in common.  Rows of one may lie between the other's.
bool tables_meet(const pp_fork_args& a) {
  const __int128 n = (__int128)4 * a.max_blocks, in_step = (__int128)4 * a.row_stride, out_step = (__int128)4 * a.out_row_stride;
  const __int128 first = (__int128)(uintptr_t)a.out_table - (uintptr_t)a.block_table, last = in_step * (a.parents - 1);
  if (first >= last + n || first + out_step * (a.rows - 1) + n <= 0) return false;
  if (in_step == out_step && in_step) {                      // all rows alike, so one tells
    const __int128 at = (first % in_step + in_step) % in_step;
    if (at >= n && at + n <= in_step) return false;
  }
  for (int32_t r = 0; r < a.rows; ++r) {
    const __int128 at = first + out_step * r;               // from the first row of block_table
    const __int128 below = at <= 0 || in_step == 0 ? 0 : at >= last ? last : at / in_step * in_step;   // the nearest rows
    const __int128 above = below + in_step < last ? below + in_step : last;
    if ((at > below - n && at < below + n) || (at > above - n && at < above + n)) return true;
  }
  return false;
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
  const int bad = check_call(a, pages->dim, attention_workspace(*pages, *a));
  if (bad != PP_OK) return bad;
  return launched(launch_attention(*pages, *a, (hipStream_t)hip_stream));
}

int pp_turns(int32_t n, const double* radians, uint64_t* turns) {
  report(PP_OK, "");
  if (n < 0 || (n && (!radians || !turns))) return report(PP_E_ARG, "bad arguments to pp_turns");
  for (int32_t i = 0; i < n; ++i)
    if (!std::isfinite(radians[i])) return report(PP_E_RANGE, "a frequency is not finite");
  for (int32_t i = 0; i < n; ++i) {
    const long double x = (long double)radians[i] / (2 * 3.14159265358979323846264338327950288L);
    const long double part = x - std::floor(x);       // 0 <= part <= 1, as it is rounded
    turns[i] = part >= 1 ? 0 : (uint64_t)std::rint(std::ldexp(part, 64));   // below 2^64: 64 bits hold it
  }
  return PP_OK;
}

int pp_rotary_turns(int32_t dim, double base, double factor, double original, double slow, double fast,
                    double* radians, uint64_t* turns) {
  report(PP_OK, "");
  if (dim < 0 || dim % 2) return report(PP_E_ARG, "dim is even");
  if (!(base > 1) || !(factor >= 1) || !(original >= 0) || !std::isfinite(base) || !std::isfinite(factor) ||
      !std::isfinite(original) || !(slow >= 0) || !(fast > slow) || !std::isfinite(fast))
    return report(PP_E_RANGE, "need base > 1, factor >= 1, original >= 0 and fast > slow >= 0");
  for (int32_t i = 0; i < dim / 2; ++i) {
    double w = std::pow(base, -2.0 * i / dim);
    if (factor != 1) {
      double keep = original > 0 ? (original * w / (2 * M_PI) - slow) / (fast - slow) : 0;
      keep = keep < 0 ? 0 : keep > 1 ? 1 : keep;
      w = keep * w + (1 - keep) * w / factor;
    }
    if (radians) radians[i] = w;
    if (turns) {
      const int rc = pp_turns(1, &w, turns + i);
      if (rc != PP_OK) return rc;
    }
  }
  return PP_OK;
}

int pp_rotary_write(const pp_rotary_args* a, const pp_kv_pages* pages, void* hip_stream) {
  report(PP_OK, "");
  if (!a) return report(PP_E_ARG, "null arguments");
  if (a->tokens < 0 || a->q_heads < 0 || a->k_heads < 0) return report(PP_E_ARG, "negative size");
  if (!row_type(a->dtype)) return report(PP_E_ARG, "rows are PP_BF16 or PP_F16");
  if (a->rot_dim < 0 || a->rot_dim % 16 || a->rot_dim > 1024)
    return report(PP_E_UNSUPPORTED, "rot_dim is a multiple of 16, 1,024 at most");
  if (!std::isfinite(a->amplitude) || !(a->eps >= 0) || !std::isfinite(a->eps))
    return report(PP_E_ARG, "amplitude is not finite, or eps not finite and >= 0");
  if (!a->k_heads && (pages || a->v)) return report(PP_E_ARG, "pages or values without keys");
  if (a->k_heads && !pages && a->v) return report(PP_E_ARG, "values go to pages only");
  if (pages) {
    int rc = check_layout(pages, a->dtype, true);
    if (rc != PP_OK) return rc;
    if ((pages->v != nullptr) != (a->v != nullptr)) return report(PP_E_ARG, "values and their pages go together");
    if (!pages->v && pages->v_scale) return report(PP_E_ARG, "a scale of no values");
    if (pages->heads != a->k_heads || pages->dim != a->k_dim)
      return report(PP_E_ARG, "pages have the keys' heads and dim");
    rc = check_strides(pages);
    if (rc != PP_OK) return rc;
    if (!nested(pages->dim, {pages->n_pages, pages->page_stride}, {pages->heads, pages->head_stride},
                {pages->page_size, pages->token_stride}))
      return report(PP_E_ARG, "rows of the pages overlap");
  }
  if (a->tokens == 0 || (a->q_heads == 0 && a->k_heads == 0)) return PP_OK;
  if ((int64_t)a->tokens * a->q_heads > INT32_MAX || (int64_t)a->tokens * a->k_heads > INT32_MAX)
    return report(PP_E_UNSUPPORTED, "tokens * heads exceeds 2^31 - 1");
  if (a->q_heads) {
    const int rc = check_rotary_rows(a->tokens, a->q_heads, a->q_dim, a->q_first, a->q_norm, a->rot_dim, a->q,
                                     a->q_token_stride, a->q_head_stride, a->q_out, a->q_out_token_stride,
                                     a->q_out_head_stride, a->q_weight, true);
    if (rc != PP_OK) return rc;
  }
  if (a->k_heads) {
    const int rc = check_rotary_rows(a->tokens, a->k_heads, a->k_dim, a->k_first, a->k_norm, a->rot_dim, a->k,
                                     a->k_token_stride, a->k_head_stride, a->k_out, a->k_out_token_stride,
                                     a->k_out_head_stride, a->k_weight, !pages);
    if (rc != PP_OK) return rc;
  }
  if (a->v && !row_layout(a->v, 2, a->v_token_stride, a->v_head_stride))
    return report(PP_E_ARG, "rows start at 16-byte boundaries, at strides >= 0");
  if (a->rot_dim && (!a->position || !a->turns || !aligned16(a->turns)))
    return report(PP_E_ARG, "null position or turns, or turns not 16-byte aligned");
  if (pages && !a->slot_map) return report(PP_E_ARG, "null pointer");
  return launched(launch_rotary(*a, pages, (hipStream_t)hip_stream));
}

int64_t pp_latent_workspace(const pp_kv_pages* pages, int32_t value_dim, const pp_attention_args* args) {
  report(PP_OK, "");
  const int rc = check_latent(pages, value_dim, args);
  if (rc != PP_OK) return rc;
  return empty(*args) ? 0 : latent_workspace(*pages, value_dim, *args);
}

int pp_latent_attention(const pp_kv_pages* pages, int32_t value_dim, const pp_attention_args* a,
                        void* hip_stream) {
  report(PP_OK, "");
  const int rc = check_latent(pages, value_dim, a);
  if (rc != PP_OK) return rc;
  if (empty(*a)) return PP_OK;
  if (!nested(value_dim, {a->tokens, a->out_token_stride}, {a->q_heads, a->out_head_stride}))
    return report(PP_E_ARG, "rows of out overlap");
  const int bad = check_call(a, value_dim, latent_workspace(*pages, value_dim, *a));
  if (bad != PP_OK) return bad;
  return launched(launch_latent(*pages, value_dim, *a, (hipStream_t)hip_stream));
}

int pp_page_copy(const pp_copy_args* a, void* hip_stream) {
  report(PP_OK, "");
  if (!a) return report(PP_E_ARG, "null arguments");
  if (a->moves < 0 || a->n_pools < 0) return report(PP_E_ARG, "negative size");
  if (!row_type(a->dtype) && a->dtype != PP_E4M3) return report(PP_E_ARG, "no pages of this type");
  if (a->n_pages < 1 || a->heads < 1 || a->dim < 1) return report(PP_E_ARG, "need n_pages, heads and dim >= 1");
  if (!pow2_page(a->page_size)) return report(PP_E_UNSUPPORTED, "page_size is a power of two from 16 to 1,024");
  const int64_t size = size_of(a->dtype);
  if (a->dim * size % 16) return report(PP_E_UNSUPPORTED, "rows of pages are multiples of 16 bytes");
  if ((__int128)a->heads * a->page_size * a->dim * size > (int64_t)1 << 31)
    return report(PP_E_UNSUPPORTED, "one page has more than 2 GiB");
  if (a->moves == 0 || a->n_pools == 0) return PP_OK;
  if (!a->pools || !a->source || !a->target) return report(PP_E_ARG, "null pointer");
  for (int32_t i = 0; i < a->n_pools; ++i)
    if (!a->pools[i] || !row_layout(a->pools[i], size, a->page_stride, a->head_stride, a->token_stride))
      return report(PP_E_ARG, "page rows start at 16-byte boundaries, at strides >= 0");
  if (!nested(a->dim, {a->n_pages, a->page_stride}, {a->heads, a->head_stride}, {a->page_size, a->token_stride}))
    return report(PP_E_ARG, "rows of the pages overlap");
  return launched(launch_page_copy(*a, (hipStream_t)hip_stream));
}

int pp_fork_tables(const pp_fork_args* a, void* hip_stream) {
  report(PP_OK, "");
  if (!a) return report(PP_E_ARG, "null arguments");
  if (a->rows < 0 || a->rows > 65536 || a->parents < 0 || a->parents > 65536 || a->n_free < 0 ||
      a->max_blocks < 0 || a->row_stride < 0 || a->out_row_stride < 0)
    return report(PP_E_ARG, "negative size, or more than 65,536 rows");
  if (!pow2_page(a->page_size)) return report(PP_E_UNSUPPORTED, "page_size is a power of two from 16 to 1,024");
  if ((int64_t)a->max_blocks * a->page_size > INT32_MAX)
    return report(PP_E_UNSUPPORTED, "tokens of a row exceed 2^31 - 1");
  if (!a->taken || (a->rows && (!a->parent || !a->out_length || !a->source || !a->target || !a->tokens)) ||
      (a->parents && !a->length) || (a->parents && a->max_blocks && !a->block_table) ||
      (a->rows && a->max_blocks && !a->out_table) || (a->n_free && !a->free_pages))
    return report(PP_E_ARG, "null pointer");
  if (a->rows > 1 && a->out_row_stride < a->max_blocks)
    return report(PP_E_ARG, "rows of out_table overlap");
  if (a->rows && a->parents && tables_meet(*a)) return report(PP_E_ARG, "out_table overlaps block_table");
  return launched(launch_fork_tables(*a, (hipStream_t)hip_stream));
}

int pp_free_pages(const pp_free_args* a, void* hip_stream) {
  report(PP_OK, "");
  if (!a) return report(PP_E_ARG, "null arguments");
  if (a->requests < 0 || a->requests > 65536 || a->max_blocks < 0 || a->n_pages < 0 || a->first < 0 ||
      a->first > a->n_pages || a->room < 0 || a->row_stride < 0)
    return report(PP_E_ARG, "negative size, first past n_pages, or more than 65,536 requests");
  if (a->n_pages > 1 << 24) return report(PP_E_UNSUPPORTED, "more than 16,777,216 pages");
  if (!pow2_page(a->page_size)) return report(PP_E_UNSUPPORTED, "page_size is a power of two from 16 to 1,024");
  if ((int64_t)a->max_blocks * a->page_size > INT32_MAX)
    return report(PP_E_UNSUPPORTED, "tokens of a row exceed 2^31 - 1");
  if (!a->count || (a->requests && !a->length) || (a->requests && a->max_blocks && !a->block_table) ||
      (a->room && !a->free_pages) || (a->n_pages && !a->marks))
    return report(PP_E_ARG, "null pointer");
  if ((uintptr_t)a->marks & 7) return report(PP_E_ARG, "marks are 8-byte aligned");
  return launched(launch_free_pages(*a, (hipStream_t)hip_stream));
}

}  // extern "C"
