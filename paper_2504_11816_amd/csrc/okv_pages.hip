// Pages of a paged KV cache (include/okv_pages.h), for gfx950.
//
// Two kinds of kernels.  What is decided -- which ids are free, who gets which, what moves where -- is prefix sums over a few thousand
// integers: one workgroup of 1024 threads, a launch of 3 to 5 us.  What is moved is bound by HBM, twice its bytes: a workgroup takes 16 KiB,
// four 16-byte loads of every thread in flight before the first store; loads through the caches (several forks read one page), stores past
// them.  Measured, us: 48 forks of 256 KiB pages in 32 layers 120 (403 MB written, 354 of the 403 MB read past L2), 592 pages of 256 KiB in 4
// layers and 200 gathered 310 (5.4 TB/s, read and written); with 32 KiB a workgroup 200 and 471, with loads past the caches 158 and 314, stores
// through them 144 and 337.
#include "okv_pages.h"
#include "okv_report.h"

#include <hip/hip_runtime.h>

#include <algorithm>

#include "okv.h"

namespace okv {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 1024, kMoveThreads = 256, kInFlight = 4;
constexpr int kSmallPage = 2048;         // bytes of a page in an array that is moved together with another's piece
constexpr int kMoveBlocks = 8192;        // of launches that may have more work than workgroups

struct Lists {                           // in the workspace
  int32_t *count;                        // pages to move (compact), or whether the fork is carried out
  int32_t *from, *to;                    // pages (compact); page that fork i copies and the one it has taken, -1: none
  int32_t *place;                        // compact: where page p is now; fork: tokens of src[i] (its row may be the dst of another fork)
};

struct State {
  int32_t *table, *lens, *refs, *status;
  int32_t max_seqs, width, log2_T, n_pages;
};

__device__ __forceinline__ bool is_row(const State &s, int r) { return r >= 0 && r < s.max_seqs; }
__device__ __forceinline__ int length_of(const State &s, int r) { return min(max(s.lens[r], 0), s.width << s.log2_T); }
__device__ __forceinline__ int pages_of(const State &s, int n) { return (n + (1 << s.log2_T) - 1) >> s.log2_T; }
__device__ __forceinline__ void blame(const State &s, int code) { if (s.status[0] == 0) s.status[0] = code; }

// x + y, numbers that are not negative, at most 2^31 - 1
__device__ __forceinline__ int add_up(const int x, const int y) { return (int)min((uint32_t)x + (uint32_t)y, 0x7fffffffu); }

// Exclusive prefix sum over the workgroup; `total` is everybody's.  Sums that pass 2^31 - 1 stay there (and the prefixes mean nothing)
__device__ __forceinline__ int scan(const int x, int &total, int *sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int upto = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int other = __shfl_up(upto, o);
    if (lane >= o) upto = add_up(upto, other);
  }
  __syncthreads();                       // sums may still be read from the last time
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int before = upto - x;
  total = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < wave) before = add_up(before, sums[w]);
    total = add_up(total, sums[w]);
  }
  return before;
}

// give(rank, page) for the first `need` free pages, lowest id first; returns how many there were
template <class Give>
__device__ __forceinline__ int take_free(const State &s, const int need, int *sums, const Give &give) {
  constexpr int kEach = 4;
  int found = 0;
  for (int p0 = 0; p0 < s.n_pages && found < need; p0 += kThreads * kEach) {
    const int p = p0 + threadIdx.x * kEach;
    int free_ones = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) free_ones |= (p + i < s.n_pages && s.refs[p + i] == 0 ? 1 : 0) << i;
    int total, rank = found + scan(__popc(free_ones), total, sums);
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (free_ones >> i & 1) {
        if (rank < need) give(rank, p + i);
        ++rank;
      }
    found += total;
  }
  return min(found, need);
}

constexpr int kEachSeq = OKV_PAGES_MAX_SEQS / kThreads;

__global__ void __launch_bounds__(kThreads) extend_kernel(State s, const int32_t *seqs, const int32_t *n_new, int n, int32_t *fresh) {
  __shared__ int sums[kThreads / 64], first[OKV_PAGES_MAX_SEQS + 1], bad;
  // After one that was refused nothing grows until the caller has seen it: with this one's outcome in its place, the steps over the other's
  // sequences would write.  (Nobody writes status before the barriers of `scan`.)
  if (s.status[0] != 0 && s.status[3] != 0) return;
  if (threadIdx.x == 0) bad = 0;
  __syncthreads();
  const int each = (n + kThreads - 1) / kThreads;
  int more[kEachSeq], need = 0;
#pragma unroll
  for (int i = 0; i < kEachSeq; ++i) {
    const int j = threadIdx.x * each + i, row = i < each && j < n ? seqs ? seqs[j] : j : -1;
    more[i] = 0;
    if (!is_row(s, row)) continue;
    const int len = length_of(s, row), add = n_new ? max(n_new[j], 0) : 1;
    if (add > (s.width << s.log2_T) - len) bad = 1;
    else more[i] = pages_of(s, len + add) - pages_of(s, len);
    need = add_up(need, more[i]);
  }
  int total, at = scan(need, total, sums);
#pragma unroll
  for (int i = 0; i < kEachSeq; ++i) {
    if (i < each) first[threadIdx.x * each + i] = at;
    at = add_up(at, more[i]);
  }
  if (threadIdx.x == kThreads - 1) first[kThreads * each] = at;
  __syncthreads();
  const bool lacks = bad || total > s.n_pages || take_free(s, total, sums, [&](int rank, int page) { fresh[rank] = page; }) < total;
  if (threadIdx.x == 0) s.status[3] = lacks ? OKV_ENOSPC : 0;
  if (lacks) {
    if (threadIdx.x == 0) blame(s, OKV_ENOSPC);
    return;
  }
  __threadfence_block();
  __syncthreads();
  for (int k = threadIdx.x; k < total; k += kThreads) {
    int lo = 0, hi = n;                  // first[lo] <= k < first[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      (first[mid] <= k ? lo : hi) = mid;
    }
    const int row = seqs ? seqs[lo] : lo, page = fresh[k];
    s.table[(int64_t)row * s.width + pages_of(s, length_of(s, row)) + k - first[lo]] = page;
    s.refs[page] = 1;
  }
  __syncthreads();                       // the lengths are read above
  for (int j = threadIdx.x; j < n; j += kThreads) {
    const int row = seqs ? seqs[j] : j;
    if (is_row(s, row)) s.lens[row] = length_of(s, row) + (n_new ? max(n_new[j], 0) : 1);
  }
}

__global__ void __launch_bounds__(kThreads) fork_plan_kernel(State s, const int32_t *src, const int32_t *dst, int n, Lists l) {
  __shared__ int sums[kThreads / 64], bad, holes[OKV_PAGES_MAX_SEQS];
  if (threadIdx.x == 0) bad = 0;
  __syncthreads();
  const int each = (n + kThreads - 1) / kThreads;
  int row[kEachSeq], len[kEachSeq], need = 0;
  const int within = (1 << s.log2_T) - 1;
#pragma unroll
  for (int i = 0; i < kEachSeq; ++i) {
    const int j = threadIdx.x * each + i;
    row[i] = len[i] = 0;
    if (i >= each || j >= n) continue;
    const int a = src[j], b = dst[j];
    if (!is_row(s, a) || !is_row(s, b) || a == b) {
      bad = 1;
      continue;
    }
    row[i] = a;
    len[i] = length_of(s, a);
    if (s.lens[b] != 0) bad = 1;
    need += len[i] & within ? 1 : 0;
  }
  int total, at = scan(need, total, sums);         // (its barriers: `bad` is everybody's)
  const int found = bad ? 0 : take_free(s, total, sums, [&](int rank, int page) { holes[rank] = page; });
  __syncthreads();
  const bool go = !bad && found == total;
  if (threadIdx.x == 0) {
    l.count[0] = go;
    if (!go) blame(s, bad ? OKV_ESTATE : OKV_ENOSPC);
  }
  if (!go) return;
#pragma unroll
  for (int i = 0; i < kEachSeq; ++i) {
    const int j = threadIdx.x * each + i;
    if (i >= each || j >= n) continue;
    int from = -1, to = -1;
    if (len[i] & within) {
      to = holes[at++];
      from = s.table[(int64_t)row[i] * s.width + (len[i] >> s.log2_T)];
      s.refs[to] = 1;
    }
    l.from[j] = from;
    l.to[j] = to;
    l.place[j] = len[i];
  }
}

// A page array as kernels see it; pieces of 16 KiB (4 KiB where it is moved by 4 bytes)
struct Moved {
  char *base, *to;
  int64_t page_bytes, layer_stride, to_layer_stride, unit_bytes;
  int32_t log2_units_tokens, whole_units, wide, pieces;      // pieces 0: a small array, moved with the page's first piece
};
struct MovedRows {
  char *base;
  int64_t layer_stride;
  int32_t groups, rows, row_bytes, wide, pieces;
};
struct Moves {
  Moved arrays[OKV_PAGES_MAX_ARRAYS];
  MovedRows rows[OKV_PAGES_MAX_ROWS];
  int32_t n_arrays, n_rows, pieces, row_pieces;      // pieces of a page over all arrays, of a sequence's rows over all row arrays
};

// The first `bytes` bytes of what begins at piece `piece` of a page
template <class T>
__device__ __forceinline__ void move_piece(char *to, const char *from, const int piece, const int64_t bytes) {
  const int64_t first = (int64_t)piece * kMoveThreads * kInFlight, n = bytes / (int64_t)sizeof(T) - first;
  const T *f = reinterpret_cast<const T *>(from) + first;
  T *t = reinterpret_cast<T *>(to) + first;
  T x[kInFlight];
#pragma unroll
  for (int i = 0; i < kInFlight; ++i)
    if ((int64_t)i * kMoveThreads + threadIdx.x < n) x[i] = f[i * kMoveThreads + threadIdx.x];
#pragma unroll
  for (int i = 0; i < kInFlight; ++i)
    if ((int64_t)i * kMoveThreads + threadIdx.x < n) __builtin_nontemporal_store(x[i], t + i * kMoveThreads + threadIdx.x);
}
__device__ __forceinline__ void move_page(const Moves &m, int piece, const int layer, const int64_t from, const int64_t to, const int used) {
  const bool small_ones = piece == 0;
#pragma unroll
  for (int i = 0; i < OKV_PAGES_MAX_ARRAYS; ++i) {
    if (i >= m.n_arrays) return;
    const Moved &a = m.arrays[i];
    const bool mine = piece >= 0 && piece < a.pieces;
    if (mine || (a.pieces == 0 && small_ones)) {
      const char *f = a.base + layer * a.layer_stride + from * a.page_bytes;
      char *t = a.to + layer * a.to_layer_stride + to * a.page_bytes;
      const int units = used < 0 ? 0 : (used + (a.whole_units ? 0 : (1 << a.log2_units_tokens) - 1)) >> a.log2_units_tokens;
      const int64_t bytes = used < 0 ? a.page_bytes : units * a.unit_bytes;
      if (a.wide) move_piece<u32x4>(t, f, mine ? piece : 0, bytes);
      else move_piece<uint32_t>(t, f, mine ? piece : 0, bytes);
    }
    piece -= a.pieces;
  }
}
// Piece `piece` of the first n rows of every group
template <class T>
__device__ __forceinline__ void move_rows(char *to, const char *from, const MovedRows &r, const int n, const int piece) {
  const int per_row = r.row_bytes / (int)sizeof(T), per_group = n * per_row, all = r.groups * per_group, stride = r.rows * per_row;
  const int first = piece * kMoveThreads * kInFlight + threadIdx.x;
  int at[kInFlight];
  T x[kInFlight];
#pragma unroll
  for (int i = 0; i < kInFlight; ++i) {
    const int j = first + i * kMoveThreads, g = j / per_group;
    at[i] = g * stride + j - g * per_group;
    if (j < all) x[i] = reinterpret_cast<const T *>(from)[at[i]];
  }
#pragma unroll
  for (int i = 0; i < kInFlight; ++i)
    if (first + i * kMoveThreads < all) reinterpret_cast<T *>(to)[at[i]] = x[i];
}

// Block (piece, layer, fork): a piece of the fork's last page, behind these a piece of its rows, and behind those its row of the table (layer 0)
__global__ void __launch_bounds__(kMoveThreads) fork_move_kernel(State s, const int32_t *src, const int32_t *dst, Lists l, Moves m) {
  const int i = blockIdx.z, layer = blockIdx.y, piece = blockIdx.x;
  if (!l.count[0]) return;
  const int a = src[i], b = dst[i], len = l.place[i], from = l.from[i], to = l.to[i];
  if (piece < m.pieces) {
    if (to >= 0 && from >= 0 && from < s.n_pages) move_page(m, piece, layer, from, to, len & ((1 << s.log2_T) - 1));
    return;
  }
  int of_rows = piece - m.pieces;
#pragma unroll
  for (int k = 0; k < OKV_PAGES_MAX_ROWS; ++k) {
    if (k >= m.n_rows) break;
    const MovedRows &r = m.rows[k];
    if (of_rows >= 0 && of_rows < r.pieces) {
      const int64_t bytes = (int64_t)r.groups * r.rows * r.row_bytes;
      const int n = len % r.rows;
      if (n == 0) return;
      char *base = r.base + layer * r.layer_stride;
      if (r.wide) move_rows<u32x4>(base + b * bytes, base + a * bytes, r, n, of_rows);
      else move_rows<uint32_t>(base + b * bytes, base + a * bytes, r, n, of_rows);
      return;
    }
    of_rows -= r.pieces;
  }
  if (layer) return;
  const int full = len >> s.log2_T;
  for (int p = threadIdx.x; p < s.width; p += kMoveThreads) {
    int page = -1;
    if (p < full) {
      page = s.table[(int64_t)a * s.width + p];
      if (page >= 0 && page < s.n_pages) atomicAdd(s.refs + page, 1);
    } else if (p == full) {
      page = to;
    }
    s.table[(int64_t)b * s.width + p] = page;
  }
  if (threadIdx.x == 0) s.lens[b] = len;
}

__global__ void __launch_bounds__(kMoveThreads) free_kernel(State s, const int32_t *seqs) {
  const int row = seqs[blockIdx.x];
  if (!is_row(s, row)) return;
  for (int p = threadIdx.x; p < s.width; p += kMoveThreads) {
    const int page = atomicExch(s.table + (int64_t)row * s.width + p, -1);     // one call takes it, if the sequence is named twice
    if (page >= 0 && page < s.n_pages) atomicSub(s.refs + page, 1);
  }
  if (threadIdx.x == 0) s.lens[row] = 0;
}

__global__ void __launch_bounds__(kThreads) compact_plan_kernel(State s, Lists l) {
  __shared__ int sums[kThreads / 64];
  const int each = (s.n_pages + kThreads - 1) / kThreads, p0 = min((int)threadIdx.x * each, s.n_pages), p1 = min(p0 + each, s.n_pages);
  int mine = 0, live, moving;
  for (int p = p0; p < p1; ++p) mine += s.refs[p] > 0;
  scan(mine, live, sums);
  int holes = 0, movers = 0;
  for (int p = p0; p < p1; ++p) {
    const bool used = s.refs[p] > 0;
    holes += !used && p < live;
    movers += used && p >= live;
  }
  int hole = scan(holes, moving, sums), mover = scan(movers, moving, sums);
  for (int p = p0; p < p1; ++p) {
    const bool used = s.refs[p] > 0;
    if (!used && p < live) l.to[hole++] = p;
    if (used && p >= live) l.from[mover++] = p;
    else l.place[p] = p;
  }
  __threadfence_block();
  __syncthreads();
  for (int k = threadIdx.x; k < moving; k += kThreads) {
    const int from = l.from[k], to = l.to[k];
    l.place[from] = to;
    s.refs[to] = s.refs[from];
    s.refs[from] = 0;
  }
  if (threadIdx.x == 0) l.count[0] = moving, s.status[1] = live, s.status[2] = moving;
}

__global__ void __launch_bounds__(kMoveThreads) compact_move_kernel(State s, Lists l, Moves m, int n_layers) {
  const int64_t entries = (int64_t)s.max_seqs * s.width, all = (int64_t)l.count[0] * n_layers * m.pieces;
  for (int64_t i = (int64_t)blockIdx.x * kMoveThreads + threadIdx.x; i < entries; i += (int64_t)gridDim.x * kMoveThreads) {
    const int page = s.table[i];
    if (page >= 0 && page < s.n_pages) s.table[i] = l.place[page];
  }
  for (int64_t i = blockIdx.x; i < all; i += gridDim.x) {
    const int64_t move = i / m.pieces, k = move / n_layers;
    move_page(m, (int)(i - move * m.pieces), (int)(move - k * n_layers), l.from[k], l.to[k], -1);
  }
}

__global__ void __launch_bounds__(kMoveThreads) copy_pages_kernel(const int32_t *src, const int32_t *dst, Moves m, int n_layers, int64_t all, int n_pages,
                                                                  int to_pages) {
  for (int64_t i = blockIdx.x; i < all; i += gridDim.x) {
    const int64_t move = i / m.pieces, k = move / n_layers;
    const int from = src[k], to = dst[k];
    if (from < 0 || from >= n_pages || to < 0 || to >= to_pages) continue;
    move_page(m, (int)(i - move * m.pieces), (int)(move - k * n_layers), from, to, -1);
  }
}

// ---- host -------------------------------------------------------------------------------------------

bool multiple(int64_t x, int64_t of) { return x % of == 0; }
bool multiple(const void *p, int64_t of) { return reinterpret_cast<uintptr_t>(p) % of == 0; }

const char *problem(const okv_pages *p) {
  if (!p) return "pages is NULL";
  if (p->n_layers < 1 || p->n_layers > 65535) return "n_layers must be in [1, 65535]";
  if (p->page_tokens < 1 || p->page_tokens > 1024 || (p->page_tokens & (p->page_tokens - 1))) return "page_tokens must be a power of two in [1, 1024]";
  if (p->max_seqs < 1 || p->max_pages_per_seq < 1 || p->n_pages < 1) return "max_seqs, max_pages_per_seq and n_pages must be at least 1";
  if ((int64_t)p->max_pages_per_seq * p->page_tokens > 0x7fffffff) return "max_pages_per_seq * page_tokens must be below 2^31";
  if (p->n_arrays < 0 || p->n_arrays > OKV_PAGES_MAX_ARRAYS || p->n_rows < 0 || p->n_rows > OKV_PAGES_MAX_ROWS) return "too many arrays";
  if (!p->table || !p->lens || !p->refs || !p->status || !p->workspace) return "NULL pointer";
  if (!multiple(p->workspace, 16) || p->workspace_bytes < okv_pages_workspace_bytes(p->n_pages)) return "the workspace is too small or misaligned";
  for (int i = 0; i < p->n_arrays; ++i) {
    const okv_page_array &a = p->arrays[i];
    if (!a.base || a.page_bytes < 4) return "an array is NULL or its pages are empty";
    if (a.unit_tokens < 1 || p->page_tokens % a.unit_tokens || (a.unit_tokens & (a.unit_tokens - 1))) return "unit_tokens must be a power of two that divides page_tokens";
    const int64_t units = p->page_tokens / a.unit_tokens;
    if (!multiple(a.page_bytes, 4 * units) || !multiple(a.layer_stride, 4) || !multiple(a.base, 4)) return "an array's addresses and sizes must be multiples of 4";
    if (a.page_bytes > (int64_t)1 << 30) return "a page of an array must be at most 2^30 bytes";
  }
  for (int i = 0; i < p->n_rows; ++i) {
    const okv_row_array &r = p->rows[i];
    if (!r.base || r.groups < 1 || r.rows < 1 || r.row_bytes < 4) return "a row array is NULL or empty";
    if (!multiple(r.row_bytes, 4) || !multiple(r.layer_stride, 4) || !multiple(r.base, 4)) return "a row array's addresses and sizes must be multiples of 4";
    if ((int64_t)r.groups * r.rows * r.row_bytes > (int64_t)1 << 30) return "a sequence's rows must be at most 2^30 bytes";
  }
  return nullptr;
}

int log2_of(int32_t x) { return 31 - __builtin_clz((unsigned)x); }

State state_of(const okv_pages *p) {
  return {p->table, p->lens, p->refs, p->status, p->max_seqs, p->max_pages_per_seq, log2_of(p->page_tokens), p->n_pages};
}
Lists lists_of(const okv_pages *p) {
  int32_t *w = static_cast<int32_t *>(p->workspace);
  const int64_t n = std::max<int64_t>(p->n_pages, OKV_PAGES_MAX_SEQS);
  return {w, w + 16, w + 16 + n, w + 16 + 2 * n};
}
Moves moves_of(const okv_pages *p, const okv_page_array *to) {
  Moves m;
  m.n_arrays = p->n_arrays, m.n_rows = p->n_rows, m.pieces = m.row_pieces = 0;
  for (int i = 0; i < p->n_arrays; ++i) {
    const okv_page_array &a = p->arrays[i], &t = to ? to[i] : a;
    Moved &k = m.arrays[i];
    k.base = static_cast<char *>(a.base), k.to = static_cast<char *>(t.base);
    k.page_bytes = a.page_bytes, k.layer_stride = a.layer_stride, k.to_layer_stride = t.layer_stride;
    k.unit_bytes = a.page_bytes / (p->page_tokens / a.unit_tokens);
    k.log2_units_tokens = log2_of(a.unit_tokens), k.whole_units = a.whole_units != 0;
    k.wide = multiple(a.base, 16) && multiple(t.base, 16) && multiple(k.unit_bytes, 16) && multiple(a.layer_stride, 16) && multiple(t.layer_stride, 16);
    const int64_t piece = (int64_t)kMoveThreads * kInFlight * (k.wide ? 16 : 4);
    k.pieces = a.page_bytes <= kSmallPage ? 0 : (int32_t)((a.page_bytes + piece - 1) / piece);
    m.pieces += k.pieces;
  }
  if (p->n_arrays && m.pieces == 0) m.pieces = 1;
  for (int i = 0; i < p->n_rows; ++i) {
    const okv_row_array &r = p->rows[i];
    const bool wide = multiple(r.base, 16) && multiple(r.row_bytes, 16) && multiple(r.layer_stride, 16);
    const int64_t piece = (int64_t)kMoveThreads * kInFlight * (wide ? 16 : 4), bytes = (int64_t)r.groups * r.rows * r.row_bytes;
    m.rows[i] = {static_cast<char *>(r.base), r.layer_stride, r.groups, r.rows, r.row_bytes, wide, (int32_t)((bytes + piece - 1) / piece)};
    m.row_pieces += m.rows[i].pieces;
  }
  return m;
}

int check(const char *who, const okv_pages *p, int32_t n, int32_t most) {
  if (const char *why = problem(p)) return report(OKV_EINVAL, "%s: %s", who, why);
  if (n < 0 || n > most) return report(OKV_EINVAL, "%s: n must be in [0, %d]", who, most);
  return OKV_OK;
}
int hip_result(const char *who) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? OKV_OK : report(OKV_EHIP, "%s: %s", who, hipGetErrorString(e));
}

}  // namespace

}  // namespace okv

using namespace okv;

extern "C" {

int64_t okv_pages_workspace_bytes(int32_t n_pages) {
  if (n_pages < 1) return report(OKV_EINVAL, "okv_pages_workspace_bytes: n_pages must be at least 1");
  return 4 * (16 + 3 * std::max<int64_t>(n_pages, OKV_PAGES_MAX_SEQS));
}

int okv_pages_extend(const okv_pages *p, int32_t n, const int32_t *seqs, const int32_t *n_new, void *stream) {
  if (const int rc = check("okv_pages_extend", p, n, OKV_PAGES_MAX_SEQS)) return rc;
  if (n == 0) return OKV_OK;
  if (!seqs && n > p->max_seqs) return report(OKV_EINVAL, "okv_pages_extend: more sequences than the table has rows");
  hipLaunchKernelGGL(extend_kernel, dim3(1), dim3(kThreads), 0, static_cast<hipStream_t>(stream), state_of(p), seqs, n_new, n, lists_of(p).from);
  return hip_result("okv_pages_extend");
}

int okv_pages_fork(const okv_pages *p, int32_t n, const int32_t *src, const int32_t *dst, void *stream) {
  if (const int rc = check("okv_pages_fork", p, n, OKV_PAGES_MAX_SEQS)) return rc;
  if (n == 0) return OKV_OK;
  if (!src || !dst) return report(OKV_EINVAL, "okv_pages_fork: NULL pointer");
  const Lists l = lists_of(p);
  const Moves m = moves_of(p, nullptr);
  const State s = state_of(p);
  hipLaunchKernelGGL(fork_plan_kernel, dim3(1), dim3(kThreads), 0, static_cast<hipStream_t>(stream), s, src, dst, n, l);
  hipLaunchKernelGGL(fork_move_kernel, dim3((unsigned)(m.pieces + m.row_pieces + 1), (unsigned)p->n_layers, (unsigned)n), dim3(kMoveThreads), 0,
                     static_cast<hipStream_t>(stream), s, src, dst, l, m);
  return hip_result("okv_pages_fork");
}

int okv_pages_free(const okv_pages *p, int32_t n, const int32_t *seqs, void *stream) {
  if (const int rc = check("okv_pages_free", p, n, OKV_PAGES_MAX_SEQS)) return rc;
  if (n == 0) return OKV_OK;
  if (!seqs) return report(OKV_EINVAL, "okv_pages_free: NULL pointer");
  hipLaunchKernelGGL(free_kernel, dim3((unsigned)n), dim3(kMoveThreads), 0, static_cast<hipStream_t>(stream), state_of(p), seqs);
  return hip_result("okv_pages_free");
}

int okv_pages_compact(const okv_pages *p, void *stream) {
  if (const int rc = check("okv_pages_compact", p, 0, 0)) return rc;
  const Lists l = lists_of(p);
  hipLaunchKernelGGL(compact_plan_kernel, dim3(1), dim3(kThreads), 0, static_cast<hipStream_t>(stream), state_of(p), l);
  const Moves m = moves_of(p, nullptr);            // at most every other page is moved
  const int64_t entries = ((int64_t)p->max_seqs * p->max_pages_per_seq + kMoveThreads - 1) / kMoveThreads;
  const int64_t blocks = std::min<int64_t>(kMoveBlocks, std::max(entries, (int64_t)(p->n_pages / 2) * p->n_layers * m.pieces));
  hipLaunchKernelGGL(compact_move_kernel, dim3((unsigned)blocks), dim3(kMoveThreads), 0, static_cast<hipStream_t>(stream), state_of(p), l, m, p->n_layers);
  return hip_result("okv_pages_compact");
}

int okv_pages_copy(const okv_pages *p, int32_t n, const int32_t *src_ids, const int32_t *dst_ids, const okv_page_array *to, int32_t to_pages, void *stream) {
  if (const int rc = check("okv_pages_copy", p, n, 0x7fffffff)) return rc;
  if (n == 0 || p->n_arrays == 0) return OKV_OK;
  if (!src_ids || !dst_ids || !to) return report(OKV_EINVAL, "okv_pages_copy: NULL pointer");
  if (to_pages < 1) return report(OKV_EINVAL, "okv_pages_copy: to_pages must be at least 1");
  for (int i = 0; i < p->n_arrays; ++i) {
    if (!to[i].base || to[i].page_bytes != p->arrays[i].page_bytes) return report(OKV_EINVAL, "okv_pages_copy: an array is NULL or its pages have another size");
    if (!multiple(to[i].base, 4) || !multiple(to[i].layer_stride, 4)) return report(OKV_EINVAL, "okv_pages_copy: addresses and strides must be multiples of 4");
  }
  const Moves m = moves_of(p, to);
  const int64_t all = (int64_t)n * p->n_layers * m.pieces;
  hipLaunchKernelGGL(copy_pages_kernel, dim3((unsigned)std::min<int64_t>(all, kMoveBlocks)), dim3(kMoveThreads), 0, static_cast<hipStream_t>(stream), src_ids,
                     dst_ids, m, p->n_layers, all, p->n_pages, to_pages);
  return hip_result("okv_pages_copy");
}

}  // extern "C"
