// Page tables of a cache along the beam: rows continue others, shared pages that are written next are copied, free
// pages given out; and the used pages packed into another cache.  Which pages are free follows from the tables alone.
#include "mt_mha.h"

namespace mt {

namespace {

constexpr int kRowChunk = 256, kPageChunk = 4096;

// Workspace: per page its references, those by rows that go on writing it, and the last such row + 1; per row its needs
// and where they begin; per chunk of rows and of pages their sums; the free (packed: used) pages in order
struct Space {
  int *refs, *growers, *last;  // [n_pages]
  int *list;                   // [n_pages]
  int *begin, *need;           // [M] pages that the rows before a row take, and its own
  int *row_sum, *page_sum;     // per chunk
  int *flags;                  // [4]: too long a row; pages needed; pages free (packed: used)
};

__host__ __device__ inline int chunks(int n, int c) { return (n + c - 1) / c; }

Space space(void *ws, int M, int n_pages) {
  Space s;
  int *p = (int *)ws;
  s.flags = p; p += 4;
  s.refs = p; p += n_pages;
  s.growers = p; p += n_pages;
  s.last = p; p += n_pages;
  s.list = p; p += n_pages;
  s.begin = p; p += M;
  s.need = p; p += M;
  s.row_sum = p; p += chunks(M, kRowChunk);
  s.page_sum = p;
  return s;
}

// A row's source, length and growth, as the arguments say and clamped; out of range is reported where tell is set
struct Row {
  int src, len, blocks, add;  // src < 0: an empty row
};
__device__ __forceinline__ Row row_of(const PagesArgs &a, int m, bool tell) {
  Row r;
  int bad = 0;
  r.src = a.row ? a.row[m] : m;
  if (r.src >= a.M_in) {
    r.src = a.M_in - 1;
    bad |= kErrRow;
  }
  const int cap = a.n_blocks << a.page_log2;
  r.len = 0;
  if (r.src >= 0) {
    const int l = a.len_in[r.src];
    r.len = min(max(l, 0), cap);
    if (l != r.len) bad |= kErrLen;
  }
  r.blocks = (r.len + (1 << a.page_log2) - 1) >> a.page_log2;
  const int add = a.add ? a.add[m] : 1;
  r.add = max(add, 0);
  if (add < 0) bad |= kErrLen;
  if (tell && bad) atomicOr(a.err, bad);
  return r;
}

__device__ __forceinline__ int page_of(const PagesArgs &a, const Row &r, int j, bool tell) {
  int p = a.table_in[(long long)r.src * a.n_blocks + j];
  if ((unsigned)p >= (unsigned)a.n_pages) {
    if (tell) atomicOr(a.err, kErrPage);
    p = p < 0 ? 0 : a.n_pages - 1;
  }
  return p;
}

__global__ void __launch_bounds__(256) clear_kernel(int *p, long long n) {
  for (long long i = blockIdx.x * 256ll + threadIdx.x; i < n; i += gridDim.x * 256ll) p[i] = 0;
}

// Copies the tables and counts the references.  GROW: and those by rows that go on writing their last page.
template <bool GROW>
__global__ void __launch_bounds__(256) count_kernel(PagesArgs a, Space s) {
  const long long n = (long long)a.M * a.n_blocks;
  for (long long e = blockIdx.x * 256ll + threadIdx.x; e < n; e += gridDim.x * 256ll) {
    const int m = (int)(e / a.n_blocks), j = (int)(e - (long long)m * a.n_blocks);
    const Row r = row_of(a, m, j == 0);
    int p = -1;
    if (j < r.blocks) {
      p = page_of(a, r, j, true);
      if (GROW) {
        atomicAdd(&s.refs[p], 1);
        if (j == r.blocks - 1 && r.add > 0 && (r.len & ((1 << a.page_log2) - 1))) {
          atomicAdd(&s.growers[p], 1);
          atomicMax(&s.last[p], m + 1);
        }
      } else {
        s.refs[p] = 1;  // whoever writes it
      }
    }
    if (GROW) a.table_out[e] = p;
  }
}

// whether row m takes a copy of the page that it goes on writing
__device__ __forceinline__ bool copies(const PagesArgs &a, const Space &s, const Row &r, int m) {
  if (r.add == 0 || !(r.len & ((1 << a.page_log2) - 1))) return false;
  const int p = page_of(a, r, r.blocks - 1, false);
  return s.refs[p] > 1 && !(s.last[p] == m + 1 && s.growers[p] == s.refs[p]);
}

__device__ __forceinline__ int blocks_after(const PagesArgs &a, const Row &r) {  // both addends are below 2^31
  return (int)(((long long)r.len + r.add + (1 << a.page_log2) - 1) >> a.page_log2);
}

// sum over a workgroup of 256 threads, and the sum of the threads before this one
__device__ __forceinline__ int block_scan(int v, int &total) {
  __shared__ int w[4];
  const int incl = wave_incl_scan(v);
  if ((threadIdx.x & 63) == 63) w[threadIdx.x >> 6] = incl;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (i < (int)(threadIdx.x >> 6)) before += w[i];
    total += w[i];
  }
  __syncthreads();
  return before + incl - v;
}

// sum of n values before a chunk, over the workgroup
__device__ __forceinline__ int sum_before(const int *v, int n) {
  int x = 0, total;
  for (int i = threadIdx.x; i < n; i += 256) x += v[i];
  block_scan(x, total);
  return total;
}

// The first workgroups: the needs of a chunk of rows; the others: the free (used) pages of a chunk of pages.
template <bool GROW>
__global__ void __launch_bounds__(256) need_kernel(PagesArgs a, Space s, int row_chunks) {
  int total;
  if ((int)blockIdx.x < row_chunks) {
    const int m = blockIdx.x * kRowChunk + threadIdx.x;
    int need = 0;
    if (m < a.M) {
      const Row r = row_of(a, m, false);
      const int after = blocks_after(a, r);
      if (after > a.n_blocks)
        s.flags[0] = 1;
      else  // fewer than 2^30 blocks a table: their sum fits
        need = after - r.blocks + (copies(a, s, r, m) ? 1 : 0);
    }
    const int before = block_scan(need, total);
    if (m < a.M) {
      s.begin[m] = before;
      s.need[m] = need;
    }
    if (threadIdx.x == 0) s.row_sum[blockIdx.x] = total;
    return;
  }
  const int c = blockIdx.x - row_chunks, p0 = c * kPageChunk;
  int n = 0;
  for (int i = threadIdx.x; i < kPageChunk; i += 256)
    if (p0 + i < a.n_pages) n += GROW ? s.refs[p0 + i] == 0 : s.refs[p0 + i] != 0;
  block_scan(n, total);
  if (threadIdx.x == 0) s.page_sum[c] = total;
}

// The free pages in order; PACK: every used page's number in the order too.  The last workgroups: where the rows' needs begin.
template <bool PACK>
__global__ void __launch_bounds__(256) list_kernel(PagesArgs a, Space s, int row_chunks, int page_chunks) {
  if ((int)blockIdx.x >= page_chunks) {
    const int c = blockIdx.x - page_chunks, m = c * kRowChunk + threadIdx.x, before = sum_before(s.row_sum, c);
    if (m < a.M) s.begin[m] += before;
    if (c == row_chunks - 1 && threadIdx.x == 0) s.flags[1] = before + s.row_sum[c];
    return;
  }
  const int p0 = blockIdx.x * kPageChunk;
  int at = sum_before(s.page_sum, blockIdx.x);
  if ((int)blockIdx.x == page_chunks - 1 && threadIdx.x == 0) s.flags[2] = at + s.page_sum[blockIdx.x];
  constexpr int PER = kPageChunk / 256;  // a thread's pages are neighbours
  const int first = p0 + threadIdx.x * PER;
  int n = 0, total;
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (first + i < a.n_pages) n += (s.refs[first + i] == 0) != PACK;
  at += block_scan(n, total);
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (first + i < a.n_pages && (s.refs[first + i] == 0) != PACK) {
      s.list[at] = first + i;
      if (PACK) s.growers[first + i] = at;
      ++at;
    }
}

// All of the above by one workgroup, the counts in LDS, for tables and pools of moderate size: 768 rows of 3900 pages 38 -> 22 (7 of them here: rows, table, counts and ranks wait for each other).
constexpr int kSmallPages = 8192, kSmallRows = 2048, kSmallEntries = 1 << 15;

template <bool GROW>
__global__ void __launch_bounds__(1024) small_kernel(PagesArgs a, Space s) {
  __shared__ int refs[kSmallPages], growers[GROW ? kSmallPages : 1], last[GROW ? kSmallPages : 1];
  __shared__ int src[kSmallRows], len[kSmallRows], add[GROW ? kSmallRows : 1], end[GROW ? kSmallRows : 1];  // of the rows; end: their last page
  __shared__ int sums[16], too_long;
  for (int p = threadIdx.x; p < a.n_pages; p += 1024) {
    refs[p] = 0;
    if (GROW) growers[p] = last[p] = 0;
  }
  if (threadIdx.x == 0) too_long = 0;
  __syncthreads();
  const int n = a.M * a.n_blocks, pmask = (1 << a.page_log2) - 1;
  for (int m = threadIdx.x; m < a.M; m += 1024) {
    const Row r = row_of(a, m, true);
    src[m] = r.src;
    len[m] = r.len;
    if (GROW) add[m] = r.add;
  }
  __syncthreads();
  auto row = [&](int m) {
    Row r;
    r.src = src[m];
    r.len = len[m];
    r.blocks = (r.len + pmask) >> a.page_log2;
    r.add = GROW ? add[m] : 0;
    return r;
  };
  constexpr int U = 4;  // entries of a thread on their way at a time
  for (int e0 = threadIdx.x; e0 < n; e0 += U * 1024) {
    int page[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = min(e0 + u * 1024, n - 1), m = e / a.n_blocks, j = e - m * a.n_blocks;
      // an entry that is not the row's is not used: any entry's address will do
      page[u] = a.table_in[(long long)max(src[m], 0) * a.n_blocks + j];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = e0 + u * 1024, m = min(e, n - 1) / a.n_blocks, j = e - m * a.n_blocks;
      if (e >= n) continue;
      const Row r = row(m);
      int p = -1;
      if (j < r.blocks) {
        p = page[u];
        if ((unsigned)p >= (unsigned)a.n_pages) {
          atomicOr(a.err, kErrPage);
          p = p < 0 ? 0 : a.n_pages - 1;
        }
        if (GROW) {
          atomicAdd(&refs[p], 1);
          if (j == r.blocks - 1) {
            end[m] = p;
            if (r.add > 0 && (r.len & pmask)) {
              atomicAdd(&growers[p], 1);
              atomicMax(&last[p], m + 1);
            }
          }
        } else {
          refs[p] = 1;
        }
      }
      if (GROW) a.table_out[e] = p;
    }
  }
  __syncthreads();
  // sum over the workgroup, and of the threads before this one
  auto scan = [&](int v, int &total) {
    const int incl = wave_incl_scan(v), w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 63) sums[w] = incl;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (i < w) before += sums[i];
      total += sums[i];
    }
    __syncthreads();
    return before + incl - v;
  };
  int total, need_all = 0;
  if (GROW) {
    for (int m0 = 0; m0 < a.M; m0 += 1024) {
      const int m = m0 + threadIdx.x;
      int need = 0;
      if (m < a.M) {
        const Row r = row(m);
        const int after = blocks_after(a, r);
        if (after > a.n_blocks) {
          too_long = 1;
        } else {
          need = after - r.blocks;
          if (r.add > 0 && (r.len & pmask)) {
            const int p = end[m];
            need += refs[p] > 1 && !(last[p] == m + 1 && growers[p] == refs[p]);
          }
        }
      }
      const int before = scan(need, total);
      if (m < a.M) {
        s.begin[m] = need_all + before;
        s.need[m] = need;
      }
      need_all += total;
    }
  }
  const int per = (a.n_pages + 1023) / 1024, first = threadIdx.x * per;  // a thread's pages are neighbours
  int mine = 0;
  for (int i = 0; i < per; ++i)
    if (first + i < a.n_pages) mine += (refs[first + i] == 0) == GROW;
  int at = scan(mine, total);
  for (int i = 0; i < per; ++i)
    if (first + i < a.n_pages && (refs[first + i] == 0) == GROW) {
      s.list[at] = first + i;
      if (!GROW) refs[first + i] = at;
      ++at;
    }
  if (!GROW) {  // the tables renumbered
    __syncthreads();
    const bool fails = total > a.n_pages_out;
    for (int e = threadIdx.x; e < n; e += 1024) {
      const int m = e / a.n_blocks, j = e - m * a.n_blocks;
      const Row r = row(m);
      a.table_out[e] = !fails && j < r.blocks ? refs[page_of(a, r, j, false)] : -1;
      if (j == 0) a.len_out[m] = fails ? 0 : r.len;
    }
    if (threadIdx.x == 0) {
      if (a.free_out) *a.free_out = fails ? 0 : total;
      if (fails) atomicOr(a.err, kErrRoom);
    }
  }
  if (threadIdx.x == 0) {
    s.flags[0] = too_long;
    s.flags[1] = need_all;
    s.flags[2] = total;
  }
}

// bytes of one page of one layer's keys or values
__device__ __forceinline__ long long page_size(const PagesArgs &a) { return (a.head_bytes << a.page_log2) * a.Hk; }

// n chunks of 16 bytes by the workgroup, four of a thread on their way at a time; where(i): chunk i's offset.  Named registers:
// an array of them is moved to LDS (53 small pages 19 us, so 6.5).  363 pages of 131 KB in eight slices: 152 us, 5.0 TB/s.
template <typename F>
__device__ __forceinline__ void copy_chunks(char *dst, const char *src, int n, F where) {
  typedef int v4 __attribute__((ext_vector_type(4)));
  int i = threadIdx.x;
  for (; i - (int)threadIdx.x + 1024 <= n; i += 1024) {
    const long long a0 = where(i), a1 = where(i + 256), a2 = where(i + 512), a3 = where(i + 768);
    const v4 v0 = *(const v4 *)(src + a0), v1 = *(const v4 *)(src + a1), v2 = *(const v4 *)(src + a2), v3 = *(const v4 *)(src + a3);
    *(v4 *)(dst + a0) = v0;
    *(v4 *)(dst + a1) = v1;
    *(v4 *)(dst + a2) = v2;
    *(v4 *)(dst + a3) = v3;
  }
  for (; i < n; i += 256) {
    const long long at = where(i);
    *(v4 *)(dst + at) = *(const v4 *)(src + at);
  }
}

// The page that row r goes on writing, copied to another one in slice blockIdx.y: its positions so far, a run of every head
__device__ __forceinline__ void copy_begun(const PagesArgs &a, const Row &r, int from, int to) {
  const long long size = page_size(a), base = (long long)(blockIdx.y >> 1) * a.n_pages * size;
  char *const cache = (char *)(blockIdx.y & 1 ? a.v_out : a.k_out) + base;
  const int run = (int)((r.len & ((1 << a.page_log2) - 1)) * a.head_bytes / 16), head = (int)(a.head_bytes << a.page_log2);
  auto where = [&](int i) __attribute__((always_inline)) -> long long {
    const int h = i / run;
    return h * head + (i - h * run) * 16;
  };
  copy_chunks(cache + to * size, cache + from * size, run * a.Hk, where);
}

// Row m: its table and length, and (blockIdx.y: a layer's keys or values) the copy of its shared page.
__global__ void __launch_bounds__(256) assign_kernel(PagesArgs a, Space s) {
  const int m = blockIdx.x;
  const int need_all = s.flags[1], free_all = s.flags[2], begin = s.begin[m], need = s.need[m];
  int *const row = a.table_out + (long long)m * a.n_blocks;
  const Row r = row_of(a, m, false);
  if (s.flags[0] || need_all > free_all) {
    if (blockIdx.y) return;
    for (int j = threadIdx.x; j < a.n_blocks; j += 256) row[j] = -1;
    if (threadIdx.x == 0) {
      a.len_out[m] = 0;
      if (m == 0) {
        if (a.free_out) *a.free_out = a.n_pages;
        atomicOr(a.err, kErrRoom);
      }
    }
    return;
  }
  const int after = blocks_after(a, r), cow = need - (after - r.blocks);
  if (blockIdx.y == 0) {
    for (int j = threadIdx.x; j < after - r.blocks; j += 256) row[r.blocks + j] = s.list[begin + cow + j];
    if (threadIdx.x == 0) {
      a.len_out[m] = r.len + r.add;
      if (cow) row[r.blocks - 1] = s.list[begin];
      if (m == 0 && a.free_out) *a.free_out = free_all - need_all;
    }
  }
  if (cow) copy_begun(a, r, page_of(a, r, r.blocks - 1, false), s.list[begin]);
}

// Pages list[0 .. used) of slice y, a layer's keys or values, to the front of the other cache
__device__ __forceinline__ void move_pages(const PagesArgs &a, const int *list, int used, int y) {
  const long long size = page_size(a), layer = y >> 1;
  const char *in = (const char *)(y & 1 ? a.v_in : a.k_in) + layer * a.n_pages * size;
  char *out = (char *)(y & 1 ? a.v_out : a.k_out) + layer * a.n_pages_out * size;
  for (int i = blockIdx.x; i < used; i += gridDim.x)
    copy_chunks(out + i * size, in + list[i] * size, (int)(size / 16), [](int c) __attribute__((always_inline)) { return c * 16ll; });
}

// Pack: the pages, each slice blockIdx.y a layer's keys or values; TABLES: in front of them a slice that renumbers the tables
template <bool TABLES>
__global__ void __launch_bounds__(256) move_kernel(PagesArgs a, Space s) {
  const int used = s.flags[2];
  const bool fails = used > a.n_pages_out;
  if (TABLES && blockIdx.y == 0) {
    if (blockIdx.x == 0 && threadIdx.x == 0) {
      if (a.free_out) *a.free_out = fails ? 0 : used;
      if (fails) atomicOr(a.err, kErrRoom);
    }
    const long long n = (long long)a.M * a.n_blocks;
    for (long long e = blockIdx.x * 256ll + threadIdx.x; e < n; e += gridDim.x * 256ll) {
      const int m = (int)(e / a.n_blocks), j = (int)(e - (long long)m * a.n_blocks);
      const Row r = row_of(a, m, false);
      a.table_out[e] = !fails && j < r.blocks ? s.growers[page_of(a, r, j, false)] : -1;
      if (j == 0) a.len_out[m] = fails ? 0 : r.len;
    }
    return;
  }
  if (!fails) move_pages(a, s.list, used, blockIdx.y - TABLES);
}

// A call on small tables and pools in one launch: every workgroup makes the plan for itself, in LDS, instead of waiting for
// one that does: 5 rows of a pool of 21 pages 6.9 -> 4.1 us (the call 10.0 -> 7.2), 120 rows of 445 pages through six layers
// 9.3 -> 7.6; 240 rows of 866 pages through six 11.9 -> 15.4, so not where many workgroups would plan for many entries.  Packed,
// whose plan is shorter: 106 pages through three layers 6.0 -> 3.3 us, 558 through six 21.9 -> 21.2.  Grid as assign_kernel's or
// move_kernel<false>'s.
constexpr int kTinyPages = 1024, kTinyRows = 256, kTinyEntries = 2048;

template <bool GROW>
__global__ void __launch_bounds__(256) tiny_kernel(PagesArgs a) {
  __shared__ int refs[kTinyPages], list[kTinyPages], growers[GROW ? kTinyPages : 1], last[GROW ? kTinyPages : 1];
  __shared__ int src[kTinyRows], len[kTinyRows], add[GROW ? kTinyRows : 1], end[GROW ? kTinyRows : 1];  // of the rows; end: their last page
  __shared__ int too_long, mine[2];  // pages that the rows before this workgroup's take, and its own
  const int t = threadIdx.x, pmask = (1 << a.page_log2) - 1, n = a.M * a.n_blocks;
  const bool one = blockIdx.x == 0 && blockIdx.y == 0;  // reports, and writes what is there once
  for (int p = t; p < a.n_pages; p += 256) {
    refs[p] = 0;
    if (GROW) growers[p] = last[p] = 0;
  }
  if (t == 0) too_long = 0;
  if (t < a.M) {
    const Row r = row_of(a, t, one);
    src[t] = r.src;
    len[t] = r.len;
    if (GROW) add[t] = r.add;
  }
  __syncthreads();
  auto row = [&](int m) {
    Row r;
    r.src = src[m];
    r.len = len[m];
    r.blocks = (r.len + pmask) >> a.page_log2;
    r.add = GROW ? add[m] : 0;
    return r;
  };
  for (int e = t; e < n; e += 256) {
    const int m = e / a.n_blocks, j = e - m * a.n_blocks;
    const Row r = row(m);
    if (j >= r.blocks) continue;
    const int p = page_of(a, r, j, one);
    if (!GROW) {
      refs[p] = 1;
      continue;
    }
    atomicAdd(&refs[p], 1);
    if (j == r.blocks - 1) {
      end[m] = p;
      if (r.add > 0 && (r.len & pmask)) {
        atomicAdd(&growers[p], 1);
        atomicMax(&last[p], m + 1);
      }
    }
  }
  __syncthreads();
  int need_all = 0, total;
  if (GROW) {
    int need = 0;
    if (t < a.M) {
      const Row r = row(t);
      const int after = blocks_after(a, r);
      if (after > a.n_blocks) {
        too_long = 1;
      } else {
        need = after - r.blocks;
        if (r.add > 0 && (r.len & pmask)) {
          const int p = end[t];
          need += refs[p] > 1 && !(last[p] == t + 1 && growers[p] == refs[p]);
        }
      }
    }
    const int before = block_scan(need, need_all);
    if (t == (int)blockIdx.x) mine[0] = before, mine[1] = need;
  }
  const int per = (a.n_pages + 255) / 256, first = t * per;  // a thread's pages are neighbours
  int count = 0;
  for (int i = 0; i < per; ++i)
    if (first + i < a.n_pages) count += (refs[first + i] == 0) == GROW;
  int at = block_scan(count, total);
  for (int i = 0; i < per; ++i)
    if (first + i < a.n_pages && (refs[first + i] == 0) == GROW) {
      list[at] = first + i;
      if (!GROW) refs[first + i] = at;
      ++at;
    }
  __syncthreads();
  const bool fails = GROW ? too_long || need_all > total : total > a.n_pages_out;
  if (one && t == 0) {
    if (a.free_out) *a.free_out = GROW ? (fails ? a.n_pages : total - need_all) : fails ? 0 : total;
    if (fails) atomicOr(a.err, kErrRoom);
  }
  if (!GROW) {
    if (one) {
      for (int e = t; e < n; e += 256) {
        const int m = e / a.n_blocks, j = e - m * a.n_blocks;
        const Row r = row(m);
        a.table_out[e] = !fails && j < r.blocks ? refs[page_of(a, r, j, false)] : -1;
        if (j == 0) a.len_out[m] = fails ? 0 : r.len;
      }
    }
    if (!fails) move_pages(a, list, total, blockIdx.y);
    return;
  }
  const int m = blockIdx.x;
  const Row r = row(m);
  const int begin = mine[0], after = fails ? 0 : blocks_after(a, r), cow = fails ? 0 : mine[1] - (after - r.blocks);
  if (blockIdx.y == 0) {
    for (int j = t; j < a.n_blocks; j += 256) {
      int p = -1;
      if (!fails && j < r.blocks)
        p = cow && j == r.blocks - 1 ? list[begin] : page_of(a, r, j, false);
      else if (j < after)
        p = list[begin + cow + j - r.blocks];
      a.table_out[(long long)m * a.n_blocks + j] = p;
    }
    if (t == 0) a.len_out[m] = fails ? 0 : r.len + r.add;
  }
  if (cow) copy_begun(a, r, end[m], list[begin]);
}

// wgs: workgroups of the launch
bool tiny(const PagesArgs &a, long long wgs, long long most) {
  const long long n = (long long)a.M * a.n_blocks;
  return a.n_pages <= kTinyPages && a.M <= kTinyRows && n <= kTinyEntries && wgs * n <= most;
}

}  // namespace

size_t pages_workspace_bytes(int M, int n_pages) {
  const long long n = 4 + 4ll * n_pages + 2ll * M + chunks(M, kRowChunk) + chunks(n_pages, kPageChunk);
  return (size_t)((n * 4 + 255) / 256 * 256);
}

namespace {

// The plan of a call: what every row needs, and the free (used) pages in order.  Whether one workgroup made it.
template <bool GROW>
bool plan(const PagesArgs &a, const Space &s, hipStream_t st) {
  const long long n = (long long)a.M * a.n_blocks;
  if (a.n_pages <= kSmallPages && a.M <= kSmallRows && n <= kSmallEntries) {
    hipLaunchKernelGGL(small_kernel<GROW>, dim3(1), dim3(1024), 0, st, a, s);
    return true;
  }
  const int rc = GROW ? chunks(a.M, kRowChunk) : 0, pc = chunks(a.n_pages, kPageChunk);
  const long long clear = 4 + (GROW ? 3ll : 1ll) * a.n_pages;
  auto blocks = [](long long k) { return dim3((unsigned)(k < 256 * 4096 ? (k + 255) / 256 : 4096)); };
  hipLaunchKernelGGL(clear_kernel, blocks(clear), dim3(256), 0, st, s.flags, clear);
  hipLaunchKernelGGL(count_kernel<GROW>, blocks(n), dim3(256), 0, st, a, s);
  hipLaunchKernelGGL(need_kernel<GROW>, dim3(rc + pc), dim3(256), 0, st, a, s, rc);
  hipLaunchKernelGGL(list_kernel<!GROW>, dim3(rc + pc), dim3(256), 0, st, a, s, rc, pc);
  return false;
}

}  // namespace

hipError_t launch_advance(const PagesArgs &a, hipStream_t st) {
  if (tiny(a, 2ll * a.M * a.layers, 1 << 21)) {
    hipLaunchKernelGGL(tiny_kernel<true>, dim3(a.M, 2 * a.layers), dim3(256), 0, st, a);
    return hipGetLastError();
  }
  const Space s = space(a.ws, a.M, a.n_pages);
  plan<true>(a, s, st);
  hipLaunchKernelGGL(assign_kernel, dim3(a.M, 2 * a.layers), dim3(256), 0, st, a, s);
  return hipGetLastError();
}

hipError_t launch_pack(const PagesArgs &a, hipStream_t st) {
  const int most = a.n_pages < a.n_pages_out ? a.n_pages : a.n_pages_out, x = most < 65536 ? most : 65536;
  if (tiny(a, 2ll * x * a.layers, 1 << 23)) {
    hipLaunchKernelGGL(tiny_kernel<false>, dim3(x, 2 * a.layers), dim3(256), 0, st, a);
    return hipGetLastError();
  }
  const Space s = space(a.ws, a.M, a.n_pages);
  if (plan<false>(a, s, st))
    hipLaunchKernelGGL(move_kernel<false>, dim3(x, 2 * a.layers), dim3(256), 0, st, a, s);
  else
    hipLaunchKernelGGL(move_kernel<true>, dim3(x, 2 * a.layers + 1), dim3(256), 0, st, a, s);
  return hipGetLastError();
}

}  // namespace mt
