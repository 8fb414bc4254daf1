// pp_pages.hip -- copies, forks and the free list of pages (gfx950).

#include "pp_serve.h"

namespace pp {

namespace {

constexpr int kWave = 64;
typedef __attribute__((__vector_size__(16))) int i32x4;

// ------------------------------------------------------------------ copies ---

constexpr int kPools = 128;      // base pointers a launch takes as arguments

struct Copy {
  const int32_t *source, *target, *tokens;
  int64_t page, outer, inner;    // strides in bytes
  int32_t moves, n_pages, page_size;
  int32_t outers, inners, units; // a page's rows, and 16-byte units of a row
  int32_t tokens_inner;          // the inner rows are the tokens
  int32_t dense;                 // a whole page is one run of bytes
  int32_t blocks;                // a page's blocks
  char* pools[kPools];
};

// A block copies kCopyUnits units (32 KB) of one page in one pool, four at a time a thread.  Bound by memory: 512
// chunks of pages in all layers' pools, 537 MB read and written, 204 us, 5.3 TB/s, as a large copy.  29 open
// pages take 3.4 us, two reads one after the other, and 8.5 with the call.
constexpr int kCopyUnits = 2048;

__global__ void __launch_bounds__(256) k_copy(Copy c) {
  const int32_t part = blockIdx.x % c.blocks;
  const int32_t move = blockIdx.x / c.blocks % c.moves;
  char* const pool = c.pools[blockIdx.x / c.blocks / c.moves];
  const int32_t from = c.source[move], to = c.target[move];
  if (from < 0 || from >= c.n_pages || to < 0 || to >= c.n_pages || from == to) return;
  int32_t n = c.tokens ? c.tokens[move] : c.page_size;
  if (n <= 0) return;
  if (n > c.page_size) n = c.page_size;
  const char* a = pool + from * c.page;
  char* b = pool + to * c.page;
  const int32_t outers = c.tokens_inner ? c.outers : n, inners = c.tokens_inner ? n : c.inners;
  const int32_t run = inners * c.units, all = outers * run;
  const bool dense = c.dense && (n == c.page_size || !c.tokens_inner || c.outers == 1);
  const int32_t end = (part + 1) * kCopyUnits < all ? (part + 1) * kCopyUnits : all;
  auto at = [&](int32_t u) {
    if (dense) return (int64_t)u * 16;
    const int32_t o = u / run, r = u - o * run, i = r / c.units;
    return o * c.outer + i * c.inner + (int64_t)(r - i * c.units) * 16;
  };
  for (int32_t u = part * kCopyUnits + threadIdx.x; u < end; u += 1024) {
    i32x4 x[4];
    int64_t off[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      off[j] = at(u + 256 * j);
      if (u + 256 * j < end) x[j] = *(const i32x4*)(a + off[j]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (u + 256 * j < end) *(i32x4*)(b + off[j]) = x[j];
  }
}

// ------------------------------------------------------------------- forks ---

constexpr int kForkRows = 16;    // new rows of a block, one wave each
constexpr int kForkMost = 65536;

__device__ __forceinline__ int32_t blocks_of(int32_t length, int shift) {
  return length > 0 ? (int32_t)(((int64_t)length + (1 << shift) - 1) >> shift) : 0;
}

// Parent of a new row, -1 = none, and whether its last page is open (so that only one row can keep it).
__device__ __forceinline__ int32_t parent_of(const pp_fork_args& a, int32_t r) {
  const int32_t p = a.parent[r];
  return p >= 0 && p < a.parents ? p : -1;
}

__device__ __forceinline__ bool is_open(const pp_fork_args& a, int32_t n) {
  return n > 0 && (n & (a.page_size - 1)) && n / a.page_size < a.max_blocks;
}

// Rows need as many pages as rows before them have an open parent, less the different ones of
// those parents.  Every block counts both for itself, with a bit for each parent seen, so that one launch
// does.  Bound by the chain of its reads (parents, their lengths, rows): 64 new rows 4.4 us, 4,096 of up to 512
// blocks 9.5 us, 9.5 MB; 8.6 and 9.2 us a call among others.  The counting grows with the square of the rows and
// shows from 8,192 on: 15 us, 16,384 43, 65,536 444.
__global__ void __launch_bounds__(1024) k_fork(pp_fork_args a, int shift) {
  __shared__ uint32_t seen[kForkMost / 32];
  __shared__ int32_t sums[16];
  __shared__ int32_t parent_s[kForkRows], length_s[kForkRows], page_s[kForkRows], fresh_s[kForkRows];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int32_t first = blockIdx.x * kForkRows;
  const int words = (a.parents + 31) / 32;
  for (int i = tid; i < words; i += 1024) seen[i] = 0;
  __syncthreads();
  int32_t count = 0;
  for (int32_t r = tid; r < first; r += 1024) {
    const int32_t p = parent_of(a, r);
    if (p >= 0 && is_open(a, a.length[p])) {
      const uint32_t bit = 1u << (p % 32);
      if (!(atomicOr(&seen[p / 32], bit) & bit)) --count;
      ++count;
    }
  }
  for (int o = kWave / 2; o; o >>= 1) count += __shfl_xor(count, o);
  if (lane == 0) sums[wave] = count;
  __syncthreads();
  if (wave == 0) {
    int32_t before = lane < 16 ? sums[lane] : 0;
    for (int o = kWave / 2; o; o >>= 1) before += __shfl_xor(before, o);
    const int32_t r = first + lane;
    const bool mine = lane < kForkRows && r < a.rows;
    const int32_t p = mine ? parent_of(a, r) : -1;
    const int32_t n = p >= 0 ? a.length[p] : 0;
    const bool open = p >= 0 && is_open(a, n);
    bool kept = open && (seen[p / 32] >> (p % 32) & 1);
    for (int j = 0; j < kForkRows - 1; ++j) {
      const int32_t other = __shfl(p, j);
      if (j < lane && other == p) kept = kept || open;
    }
    const uint64_t need = __ballot(kept);
    const int32_t rank = before + __popcll(need & ((1ull << lane) - 1));
    if (mine) {
      const int32_t fresh = kept && rank < a.n_free ? a.free_pages[rank] : -1;
      parent_s[lane] = p;
      length_s[lane] = n > 0 ? n : 0;
      page_s[lane] = kept ? n >> shift : -1;
      fresh_s[lane] = fresh;
      a.out_length[r] = n > 0 ? n : 0;
      a.source[r] = kept ? a.block_table[p * a.row_stride + (n >> shift)] : -1;
      a.target[r] = fresh;
      a.tokens[r] = kept ? n & (a.page_size - 1) : 0;
    }
    if (blockIdx.x == gridDim.x - 1 && lane == 0) a.taken[0] = before + __popcll(need);
  }
  __syncthreads();
  const int32_t r = first + wave;
  if (r >= a.rows) return;
  const int32_t p = parent_s[wave], own = page_s[wave];
  if (p < 0) return;
  int32_t blocks = blocks_of(length_s[wave], shift);
  if (blocks > a.max_blocks) blocks = a.max_blocks;
  const int32_t* from = a.block_table + p * a.row_stride;
  int32_t* to = a.out_table + r * a.out_row_stride;
  for (int32_t b = lane; b < blocks; b += kWave * 4) {
    int32_t x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (b + j * kWave < blocks) x[j] = b + j * kWave == own ? fresh_s[wave] : from[b + j * kWave];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (b + j * kWave < blocks) to[b + j * kWave] = x[j];
  }
}

__global__ void k_fork_none(int32_t* taken) { taken[0] = 0; }

// --------------------------------------------------------------- free pages ---

// Calls f(page) for the pages in range that row r names, its blocks `at`, at + step and so on.
template <class F>
__device__ __forceinline__ void pages_of(const pp_free_args& a, int shift, int32_t r, int32_t at, int32_t step, F&& f) {
  int32_t blocks = blocks_of(a.length[r], shift);
  if (blocks > a.max_blocks) blocks = a.max_blocks;
  const int32_t* row = a.block_table + r * a.row_stride;
  for (int32_t b = at; b < blocks; b += step * 4) {
    int32_t page[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) page[j] = (int64_t)b + j * step < blocks ? row[b + j * step] : -1;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (page[j] >= a.first && page[j] < a.n_pages) f(page[j]);
  }
}

// Sum of x over the block's 1,024 threads before this one, and over all of them.
__device__ __forceinline__ int32_t before(int32_t x, int32_t& all, int32_t* sums) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int32_t up = x;
  for (int o = 1; o < kWave; o <<= 1) {
    const int32_t y = __shfl_up(up, o);
    if (lane >= o) up += y;
  }
  if (lane == kWave - 1) sums[wave] = up;
  __syncthreads();
  int32_t base = 0;
  all = 0;
  for (int w = 0; w < 16; ++w) {
    if (w < wave) base += sums[w];
    all += sums[w];
  }
  return base + up - x;
}

// The whole of it in one block, with a bit a page in LDS, for few rows: 16 waves take two rows at a time each.  64
// rows of up to 512 blocks 7.2 us (7.4 a call among others); 128 of 512 10.8 us and 256 of 256 13.4, where the
// four launches below take 12.5.
constexpr int kFreeWords = 32768;     // pages / 32
constexpr int kFewRows = 256;
constexpr int kFewEntries = 65536;

__global__ void __launch_bounds__(1024) k_free_few(pp_free_args a, int shift) {
  extern __shared__ uint32_t named[];
  __shared__ int32_t sums[16];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int32_t pages = a.n_pages - a.first, words = (pages + 31) / 32;
  // the blocks of this wave's rows, one a lane
  int32_t blocks = wave + 16 * lane < a.requests ? blocks_of(a.length[wave + 16 * lane], shift) : 0;
  if (blocks > a.max_blocks) blocks = a.max_blocks;
  for (int i = tid; i < words; i += 1024) named[i] = i == words - 1 && pages % 32 ? ~0u << (pages % 32) : 0;
  __syncthreads();
  constexpr int kRows = 2, kTurn = 4;
  for (int i = 0; wave + 16 * i < a.requests; i += kRows) {
    int32_t n[kRows], most = 0;
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      n[j] = __builtin_amdgcn_readlane(blocks, i + j);      // rows past the last have none
      most = n[j] > most ? n[j] : most;
    }
    for (int32_t b = lane; b < most; b += kWave * kTurn) {
      int32_t page[kRows][kTurn];
#pragma unroll
      for (int j = 0; j < kRows; ++j)
#pragma unroll
        for (int k = 0; k < kTurn; ++k)
          page[j][k] = b + k * kWave < n[j] ? a.block_table[(wave + 16 * (i + j)) * a.row_stride + b + k * kWave] : -1;
#pragma unroll
      for (int j = 0; j < kRows; ++j)
#pragma unroll
        for (int k = 0; k < kTurn; ++k) {
          const uint32_t p = (uint32_t)page[j][k] - (uint32_t)a.first;     // past the last where it is before the first
          if (p < (uint32_t)pages) atomicOr(&named[p / 32], 1u << (p % 32));
        }
    }
  }
  __syncthreads();
  const int32_t each = (words + 1023) / 1024, w0 = tid * each < words ? tid * each : words;
  const int32_t w1 = w0 + each < words ? w0 + each : words;
  int32_t count = 0, all;
  for (int32_t i = w0; i < w1; ++i) count += __popc(~named[i]);
  int32_t at = before(count, all, sums);
  for (int32_t i = w0; i < w1; ++i)
    for (uint32_t x = ~named[i]; x; x &= x - 1, ++at)
      if (at < a.room) a.free_pages[at] = a.first + i * 32 + __builtin_ctz(x);
  if (tid == 0) a.count[0] = all;
}

// Byte p of `marks` says whether page p is named: bytes because waves store them without waiting for each
// other, where bits would take an atomic each.  4,096 rows that name 1.2 million pages take 18.9 us: k_clear 2.2, k_mark 9.7
// (scattered bytes), k_count 1.9, k_list 3.7, each a launch behind the other.
__global__ void __launch_bounds__(256) k_clear(uint8_t* marks, int32_t n_pages) {
  const int32_t whole = n_pages / 8, at = blockIdx.x * 256 + threadIdx.x;
  for (int64_t i = at; i < whole; i += (int64_t)gridDim.x * 256) ((uint64_t*)marks)[i] = 0;
  if (at < n_pages % 8) marks[whole * 8 + at] = 0;
}

__global__ void __launch_bounds__(256) k_mark(pp_free_args a, int shift) {
  const int32_t r = blockIdx.x * 4 + threadIdx.x / kWave;
  if (r >= a.requests) return;
  pages_of(a, shift, r, threadIdx.x % kWave, kWave, [&](int32_t p) { a.marks[p] = 1; });
}

// Free pages of word i of the marks: bit 0 of a byte, 0 for bytes before `first` and from n_pages on.
__device__ __forceinline__ uint64_t free_of(const pp_free_args& a, int32_t i) {
  const int32_t words = (a.n_pages + 7) / 8;
  if (i >= words) return 0;
  uint64_t x = 0;
  if (i * 8 + 8 <= a.n_pages) {
    x = ((const uint64_t*)a.marks)[i];
  } else {
    for (int j = 0; i * 8 + j < a.n_pages; ++j) x |= (uint64_t)a.marks[i * 8 + j] << (8 * j);
  }
  x = (x & 0x0101010101010101ull) ^ 0x0101010101010101ull;
  if (i == a.first / 8) x &= ~0ull << (a.first % 8 * 8);
  if (i * 8 + 8 > a.n_pages) x &= ~0ull >> ((i * 8 + 8 - a.n_pages) * 8);
  return x;
}

// The marks are taken in groups of 1,024 words.  k_count leaves a group's number of free pages in the upper bits of its first
// word's bytes, two bits in each, so that k_list needs no more memory and reads one word a group before its own:
// 106,000 pages' marks added up by every block took 60 us.  (The last group's is nobody's, and its first word may
// be short.)
__global__ void __launch_bounds__(1024) k_count(pp_free_args a) {
  __shared__ int32_t sums[16];
  const int32_t i = a.first / 8 + blockIdx.x * 1024 + threadIdx.x;
  const uint64_t x = free_of(a, i);
  int32_t all;
  before(__popcll(x), all, sums);
  if (threadIdx.x == 0 && blockIdx.x + 1 < gridDim.x) {
    uint64_t n = 0;
    for (int j = 0; j < 8; ++j) n |= (uint64_t)(all >> (2 * j) & 3) << (8 * j + 1);
    ((uint64_t*)a.marks)[i] = (((uint64_t*)a.marks)[i] & 0x0101010101010101ull) | n;
  }
}

__global__ void __launch_bounds__(1024) k_list(pp_free_args a) {
  __shared__ int32_t sums[16], sums2[16];
  const int tid = threadIdx.x;
  const int32_t begin = a.first / 8 + blockIdx.x * 1024;
  int32_t sum = 0, all, total;
  for (int32_t g = tid; g < (int32_t)blockIdx.x; g += 1024) {
    const uint64_t n = ((const uint64_t*)a.marks)[a.first / 8 + g * 1024];
    for (int j = 0; j < 8; ++j) sum += (int32_t)(n >> (8 * j + 1) & 3) << (2 * j);
  }
  const uint64_t x = free_of(a, begin + tid);
  before(sum, all, sums);
  int32_t at = all + before(__popcll(x), total, sums2);
  for (uint64_t y = x; y; y &= y - 1, ++at)
    if (at < a.room) a.free_pages[at] = (begin + tid) * 8 + __builtin_ctzll(y) / 8;
  if (blockIdx.x == gridDim.x - 1 && tid == 0) a.count[0] = all + total;
}

}  // namespace

hipError_t launch_page_copy(const pp_copy_args& a, hipStream_t st) {
  const int32_t size = a.dtype == PP_E4M3 ? 1 : 2;
  Copy c{};
  c.page = a.page_stride * size;
  c.n_pages = a.n_pages;
  c.page_size = a.page_size;
  c.units = a.dim * size / 16;
  // the rows nearer to each other go first
  c.tokens_inner = a.heads == 1 || a.token_stride <= a.head_stride;
  c.outers = c.tokens_inner ? a.heads : a.page_size;
  c.inners = c.tokens_inner ? a.page_size : a.heads;
  c.outer = (c.tokens_inner ? a.head_stride : a.token_stride) * size;
  c.inner = (c.tokens_inner ? a.token_stride : a.head_stride) * size;
  c.dense = (c.inners == 1 || c.inner == c.units * 16) && (c.outers == 1 || c.outer == (int64_t)c.inners * c.units * 16);
  const int64_t all = (int64_t)c.outers * c.inners * c.units;
  c.blocks = (int32_t)((all + kCopyUnits - 1) / kCopyUnits);
  // as many moves, and then pools, at a time as a launch takes (a page has 2^16 blocks at most)
  const int64_t most = most_blocks(256) / c.blocks;
  for (int64_t move = 0; move < a.moves; move += most) {
    c.moves = (int32_t)(a.moves - move < most ? a.moves - move : most);
    c.source = a.source + move;
    c.target = a.target + move;
    c.tokens = a.tokens ? a.tokens + move : nullptr;
    const int32_t turn = most / c.moves < kPools ? (int32_t)(most / c.moves) : kPools;
    for (int32_t at = 0; at < a.n_pools; at += turn) {
      const int32_t n = a.n_pools - at < turn ? a.n_pools - at : turn;
      for (int32_t i = 0; i < n; ++i) c.pools[i] = (char*)a.pools[at + i];
      k_copy<<<(unsigned)((int64_t)c.blocks * c.moves * n), 256, 0, st>>>(c);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

hipError_t launch_fork_tables(const pp_fork_args& a, hipStream_t st) {
  if (a.rows == 0)
    k_fork_none<<<1, 1, 0, st>>>(a.taken);
  else
    k_fork<<<(a.rows + kForkRows - 1) / kForkRows, 1024, 0, st>>>(a, __builtin_ctz(a.page_size));
  return hipGetLastError();
}

hipError_t launch_free_pages(const pp_free_args& a, hipStream_t st) {
  const int shift = __builtin_ctz(a.page_size);
  const int64_t words = ((int64_t)a.n_pages - a.first + 31) / 32;
  if (a.requests <= kFewRows && (int64_t)a.requests * a.max_blocks <= kFewEntries && words <= kFreeWords) {
    const int lds = (int)(words * 4);
    if (lds > 65536 - 256) {
      static OnEachGpu once;
      int gpu;
      hipError_t e = hipGetDevice(&gpu);
      if (e == hipSuccess)
        e = once(gpu, [] {
          return hipFuncSetAttribute((const void*)&k_free_few, hipFuncAttributeMaxDynamicSharedMemorySize, kFreeWords * 4);
        });
      if (e != hipSuccess) return e;
    }
    k_free_few<<<1, 1024, lds, st>>>(a, shift);
    return hipGetLastError();
  }
  const int64_t whole = a.n_pages / 8;
  k_clear<<<(unsigned)(whole / 256 < 1024 ? whole / 256 + 1 : 1024), 256, 0, st>>>(a.marks, a.n_pages);
  if (a.requests && a.max_blocks) k_mark<<<(a.requests + 3) / 4, 256, 0, st>>>(a, shift);
  const int32_t left = (a.n_pages + 7) / 8 - a.first / 8, groups = left > 0 ? (left + 1023) / 1024 : 1;
  if (groups > 1) k_count<<<groups, 1024, 0, st>>>(a);
  k_list<<<groups, 1024, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace pp
