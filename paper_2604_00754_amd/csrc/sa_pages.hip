// The page tables of the caches in 4 bits (include/sa.h): dealing sequences anew, giving pages back, making room with copy on write,
// moving the pages in use to the front.  Tables are small and what is decided about them hangs together: one workgroup
// decides, in a fixed order, and leaves a list; a second launch moves the bytes, at the rate of a copy.  No
// result depends on the order of anything: counts change by integer atomics, pages are dealt by prefix sums.
#include "sa_cache4.h"
#include "sa_device.h"

namespace sa {
namespace {

struct Tables {
  int B, max_pages, pages, rows_log2;   // rows_log2: of a page
  int capacity;
};

__device__ __forceinline__ bool is_page(const Tables& t, int x) { return (unsigned)x < (unsigned)t.pages; }
// pages of the first `rows` rows (clamped to 0..capacity)
__device__ __forceinline__ int pages_of(const Tables& t, int rows) {
  const int r = min(max(rows, 0), t.capacity);
  return (r + (1 << t.rows_log2) - 1) >> t.rows_log2;  // (the capacity is at most 2^30)
}

__global__ __launch_bounds__(256) void copy_ints_kernel(const int32_t* from, int32_t* to, int n) {
  for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) to[i] = from[i];
}

__device__ __forceinline__ void fork_sequence(const Tables& t, int b, int lane, int lanes, const int32_t* parents, const int32_t* table,
                                              const int32_t* lens, int32_t* table_out, int32_t* lens_out, int32_t* refs) {
  const int p = parents[b];
  const bool named = (unsigned)p < (unsigned)t.B;
  const int32_t* old = table + (size_t)b * t.max_pages;
  const int32_t* from = table + (size_t)(named ? p : b) * t.max_pages;
  const int len = named ? lens[p] : 0;
  const int held = p == b ? t.max_pages : named ? pages_of(t, len) : 0;
  for (int e = lane; e < t.max_pages; e += lanes) {
    int x = e < held ? from[e] : -1;
    if (p != b) {
      const int o = old[e];
      if (is_page(t, o)) atomicAdd(refs + o, -1);
      if (is_page(t, x)) atomicAdd(refs + x, 1);
      else x = -1;
    }
    table_out[(size_t)b * t.max_pages + e] = x;
  }
  if (lane == 0) lens_out[b] = len;
}

// One workgroup per sequence; the counts are there.
__global__ __launch_bounds__(256) void pages_fork_kernel(Tables t, const int32_t* parents, const int32_t* table, const int32_t* lens,
                                                         int32_t* table_out, int32_t* lens_out, int32_t* refs) {
  fork_sequence(t, blockIdx.x, threadIdx.x, 256, parents, table, lens, table_out, lens_out, refs);
}

// Small tables whose counts go elsewhere: one workgroup, counts copied first, then a wave a sequence.
constexpr int kDecide = 1024;          // threads of a workgroup that works alone
constexpr int kDecideWaves = kDecide / 64;
__global__ __launch_bounds__(kDecide) void pages_fork_small_kernel(Tables t, const int32_t* parents, const int32_t* table, const int32_t* lens,
                                                                   const int32_t* refs, int32_t* table_out, int32_t* lens_out, int32_t* refs_out) {
  for (int i = threadIdx.x; i < t.pages; i += kDecide) refs_out[i] = refs[i];
  __syncthreads();
  for (int b = threadIdx.x >> 6; b < t.B; b += kDecideWaves)
    fork_sequence(t, b, threadIdx.x & 63, 64, parents, table, lens, table_out, lens_out, refs_out);
}

__global__ __launch_bounds__(256) void pages_free_kernel(Tables t, const int32_t* keep, int32_t* table, int32_t* refs) {
  const int b = blockIdx.x;
  int32_t* row = table + (size_t)b * t.max_pages;
  for (int e = pages_of(t, keep[b]) + threadIdx.x; e < t.max_pages; e += 256) {
    const int x = row[e];
    if (is_page(t, x)) atomicAdd(refs + x, -1);
    row[e] = -1;
  }
}

// Sum of v over the threads before this one, and over all of them.  Two barriers; `area` holds kDecideWaves ints.
__device__ __forceinline__ int scan_before(int v, int* area, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int s = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(s, d);
    if (lane >= d) s += o;
  }
  if (lane == 63) area[wave] = s;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kDecideWaves; ++w) {
    const int x = area[w];
    before += w < wave ? x : 0;
    all += x;
  }
  __syncthreads();
  *total = all;
  return before + s - v;
}

// Pages are looked through kLook at a time, kLookEach of them a lane: position at + 256 wave + 64 i + lane of the order.
constexpr int kLookEach = 4, kLook = kDecide * kLookEach;
__device__ __forceinline__ unsigned look_place(int i) { return (threadIdx.x >> 6) * (64 * kLookEach) + 64 * i + (threadIdx.x & 63); }
// Bit i: the lane's page number i of those from position `at` on, upwards from lo or downwards from hi - 1, is free (FREE) or in use.
template <bool UP, bool FREE>
__device__ __forceinline__ int look(const int32_t* refs, int lo, int hi, unsigned at) {
  int n[kLookEach], flags = 0;
#pragma unroll
  for (int i = 0; i < kLookEach; ++i) {
    const unsigned k = at + look_place(i);
    n[i] = k < (unsigned)(hi - lo) ? refs[UP ? lo + k : hi - 1 - k] : (FREE ? 1 : 0);
  }
#pragma unroll
  for (int i = 0; i < kLookEach; ++i) flags |= (n[i] <= 0) == FREE ? 1 << i : 0;
  return flags;
}

// Ids of the first `want` pages of the asked kind into list[0..]; all threads return how many there are up to `want`.  flags: look() from the
// first position.
template <bool UP, bool FREE>
__device__ __forceinline__ int collect(const int32_t* refs, int lo, int hi, int want, int flags, int32_t* list, int* area) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int found = 0;
  for (unsigned at = 0; at < (unsigned)(hi - lo) && found < want; at += kLook) {
    if (at > 0) flags = look<UP, FREE>(refs, lo, hi, at);
    int mine = 0;
#pragma unroll
    for (int i = 0; i < kLookEach; ++i) mine += __popcll(__ballot(flags >> i & 1));
    if (lane == 0) area[wave] = mine;
    __syncthreads();
    int k = found, all = 0;
#pragma unroll
    for (int w = 0; w < kDecideWaves; ++w) {
      const int x = area[w];
      k += w < wave ? x : 0;
      all += x;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kLookEach; ++i) {
      const unsigned long long who = __ballot(flags >> i & 1);
      if (flags >> i & 1) {
        const int at_list = k + __popcll(who & ((1ull << lane) - 1));
        const unsigned j = at + look_place(i);
        if (at_list < want) list[at_list] = UP ? lo + j : hi - 1 - j;
      }
      k += __popcll(who);
    }
    found += all;
  }
  return min(found, want);
}

struct ExtendArgs {
  Tables t;
  const int32_t* lens;
  const int32_t* add;
  int32_t* table;
  int32_t* refs;
  int32_t* info;
  int32_t* need;     // [B]: entries that need a page, then those of the sequences before
  int32_t* copies;   // [B][2]: page to copy and where to, or -1
  int32_t* pages;    // [pages]: the pages dealt
  int32_t* left;     // [pages]: the shared page that each replaces, or -1
};

struct Touched { int first, last, begun; };  // entries first..last-1; the first holds rows already
__device__ __forceinline__ Touched touched(const Tables& t, int len, int add) {
  const int a = min(max(len, 0), t.capacity);
  const int b = a + min(max(add, 0), t.capacity - a);
  Touched x;
  x.first = a >> t.rows_log2;
  x.last = b > a ? pages_of(t, b) : x.first;
  x.begun = (a & ((1 << t.rows_log2) - 1)) != 0;
  return x;
}

constexpr int kGroup = 16;      // lanes that look through the entries of a sequence
constexpr int kGroups = kDecide / kGroup;
constexpr int kNear = 2048;     // numbers of sequences and of pages dealt that are kept in LDS

struct Entry { bool need; int old; };  // old: the shared page that lies there, or -1
__device__ __forceinline__ Entry look_at(const ExtendArgs& a, int b, int e, int last) {
  Entry x = {false, -1};
  if (e < last) {
    const int page = a.table[(size_t)b * a.t.max_pages + e];
    const bool there = is_page(a.t, page), shared = there && a.refs[page] > 1;
    x.need = shared || !there;
    x.old = shared ? page : -1;
  }
  return x;
}

// Three round trips to memory in the usual call (at most 64 sequences and 16 entries of each, few pages): lengths, entries, counts.
__global__ __launch_bounds__(kDecide) void pages_extend_kernel(ExtendArgs a) {
  __shared__ int area[kDecideWaves], near_need[kNear], near_pages[kNear], near_left[kNear];
  const int group = threadIdx.x / kGroup, sub = threadIdx.x & (kGroup - 1), shift = (threadIdx.x & 63) & ~(kGroup - 1);
  int* need = a.t.B <= kNear ? near_need : a.need;
  const auto needed = [&](bool mine) { return (uint32_t)(__ballot(mine) >> shift) & 0xffffu; };
  const int free_pages = look<true, true>(a.refs, 0, a.t.pages, 0);
  // what the lanes of a group saw of its first sequence's first entries is kept
  Touched first = {0, 0, false};
  Entry seen = {false, -1};
  for (int b = group; b < a.t.B; b += kGroups) {
    const Touched x = touched(a.t, a.lens[b], a.add[b]);
    int n = 0;
    for (int e0 = x.first; e0 < x.last; e0 += kGroup) {
      const Entry v = look_at(a, b, e0 + sub, x.last);
      if (b == group && e0 == x.first) seen = v;
      n += __popc(needed(v.need));
    }
    if (b == group) first = x;
    if (sub == 0) {
      need[b] = n;
      a.copies[2 * b] = -1;
    }
  }
  __syncthreads();
  int total = 0;
  for (int b0 = 0; b0 < a.t.B; b0 += kDecide) {
    const int b = b0 + threadIdx.x;
    int all;
    const int before = scan_before(b < a.t.B ? need[b] : 0, area, &all);
    if (b < a.t.B) need[b] = total + before;
    total += all;
  }
  int* pages = total <= kNear ? near_pages : a.pages;
  int* left = total <= kNear ? near_left : a.left;
  const int found = total ? collect<true, true>(a.refs, 0, a.t.pages, total, free_pages, pages, area) : 0;
  if (threadIdx.x == 0) {
    a.info[0] = found < total ? 0 : total;
    a.info[1] = total - found;
  }
  if (found < total) return;
  __syncthreads();
  for (int b = group; b < a.t.B; b += kGroups) {
    const Touched x = b == group ? first : touched(a.t, a.lens[b], a.add[b]);
    int k = need[b];
    for (int e0 = x.first; e0 < x.last; e0 += kGroup) {
      const int e = e0 + sub;
      const Entry v = b == group && e0 == x.first ? seen : look_at(a, b, e, x.last);
      const uint32_t who = needed(v.need);
      if (v.need) {
        const int mine = k + __popc(who & ((1u << sub) - 1u)), page = pages[mine];
        a.table[(size_t)b * a.t.max_pages + e] = page;
        left[mine] = v.old;
        if (v.old >= 0 && e == x.first && x.begun) {
          a.copies[2 * b] = v.old;
          a.copies[2 * b + 1] = page;
        }
      }
      k += __popc(who);
    }
  }
  __syncthreads();  // counts change once every entry has been judged by those before
  for (int k = threadIdx.x; k < total; k += kDecide) {
    a.refs[pages[k]] = 1;
    if (left[k] >= 0) atomicAdd(a.refs + left[k], -1);
  }
}

constexpr int kPiece = 16384;  // bytes that a workgroup copies at a time at most
// n bytes, a multiple of 16
__device__ __forceinline__ void copy_piece(const unsigned char* from, unsigned char* to, int n) {
  const u32x4* s = reinterpret_cast<const u32x4*>(from);
  u32x4* d = reinterpret_cast<u32x4*>(to);
  constexpr int U = kPiece / (256 * 16);
  u32x4 x[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = threadIdx.x + 256 * u;
    if (i < n / 16) x[u] = s[i];
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = threadIdx.x + 256 * u;
    if (i < n / 16) d[i] = x[u];
  }
}

// blockIdx = (piece, layer, entry of the list)
__global__ __launch_bounds__(256) void pages_copy_kernel(const int32_t* copies, unsigned char* pool, size_t layer_bytes, int page_bytes) {
  const int from = copies[2 * blockIdx.z], to = copies[2 * blockIdx.z + 1];
  if (from < 0) return;
  unsigned char* layer = pool + blockIdx.y * layer_bytes;
  const int at = blockIdx.x * kPiece;
  copy_piece(layer + (size_t)from * page_bytes + at, layer + (size_t)to * page_bytes + at, min(kPiece, page_bytes - at));
}

struct CompactArgs {
  Tables t;
  int max_moves;
  const int32_t* table;
  const int32_t* refs;
  int32_t* table_out;
  int32_t* refs_out;
  int32_t* info;
  int32_t* holes;   // [pages]
  int32_t* movers;  // [pages]
  int32_t* to;      // [pages]: where a page at or above U goes
};

constexpr int kNearRefs = 16384;  // counts that are kept in LDS

__global__ __launch_bounds__(kDecide) void pages_compact_kernel(CompactArgs a) {
  __shared__ int area[kDecideWaves], near_refs[kNearRefs];
  const bool near = a.t.pages <= kNearRefs;
  int mine = 0, used;
  for (int i = threadIdx.x; i < a.t.pages; i += kDecide) {
    const int n = a.refs[i];
    mine += n > 0 ? 1 : 0;
    if (near) near_refs[i] = n;
    if (a.refs_out != a.refs) a.refs_out[i] = n;
  }
  scan_before(mine, area, &used);
  const int32_t* refs = near ? near_refs : a.refs;
  const int holes = collect<true, true>(refs, 0, used, a.max_moves, look<true, true>(refs, 0, used, 0), a.holes, area);
  const int moves = holes ? collect<false, false>(refs, used, a.t.pages, holes, look<false, false>(refs, used, a.t.pages, 0), a.movers, area) : 0;  // as many
  for (int i = used + threadIdx.x; i < a.t.pages; i += kDecide) a.to[i] = i;
  __syncthreads();
  for (int k = threadIdx.x; k < moves; k += kDecide) {
    const int from = a.movers[k], to = a.holes[k];
    a.to[from] = to;
    a.refs_out[to] = refs[from];
    a.refs_out[from] = 0;
  }
  if (threadIdx.x == 0) {
    a.info[0] = used;
    a.info[1] = moves;
  }
}

// All workgroups share the moves in steps of 4 KB of a page, two of them in flight (sources at or above U, destinations below: nothing is
// read that is written), then the table.  Bound: HBM.  What moves is not used again soon and passes the caches: 619 pages of 69 KB in
// four layers 69 -> 58 us (5.9 TB/s); pieces of 16 KB with what is left of a page behind them 73 us.
constexpr int kStep = 4096, kMoveGroups = 4096;
__global__ __launch_bounds__(256) void pages_move_kernel(CompactArgs a, unsigned char* pool, size_t layer_bytes, int page_bytes, int layers, int steps) {
  const int used = a.info[0], moves = a.info[1];
  const long total = (long)moves * layers * steps;
  constexpr int U = 2;
  for (long w0 = blockIdx.x; w0 < total; w0 += (long)gridDim.x * U) {
    u32x4 x[U];
    unsigned char* to[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long w = w0 + (long)gridDim.x * u;
      to[u] = nullptr;
      const unsigned rest = (unsigned)((w < total ? w : w0) / steps);
      const int at = (int)((w < total ? w : w0) - (long)rest * steps) * kStep + 16 * threadIdx.x;
      const int layer = rest / moves, k = rest % moves;
      if (w < total && at < page_bytes) {
        unsigned char* base = pool + layer * layer_bytes + at;
        to[u] = base + (size_t)a.holes[k] * page_bytes;
        x[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(base + (size_t)a.movers[k] * page_bytes));
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (to[u]) __builtin_nontemporal_store(x[u], reinterpret_cast<u32x4*>(to[u]));
  }
  const int entries = a.t.B * a.t.max_pages;
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < entries; i += (long)gridDim.x * 256) {
    const int x = a.table[i];
    a.table_out[i] = is_page(a.t, x) && x >= used ? a.to[x] : x;
  }
}

int log2_of(int v) { int k = 0; while ((1 << k) < v) ++k; return k; }

Tables tables_of(const sa_cache4_desc* c) { return Tables{c->B, c->max_pages, c->pages, log2_of(c->page_rows), c->max_pages * c->page_rows}; }
int page_bytes_of(const sa_cache4_desc* c) { return c->Hkv * (c->page_rows / 32) * 34 * c->d; }
size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

// Numbers that one workgroup goes through in less time than a second launch takes (528: 2.1 us, 10340: 10.9 against 5.4).
constexpr long kForkAlone = 2048;

size_t pages_extend_workspace_bytes(const sa_cache4_desc* c) {
  return align256((size_t)c->B * 12) + 2 * align256((size_t)c->pages * 4);
}
size_t pages_compact_workspace_bytes(const sa_cache4_desc* c) { return 3 * align256((size_t)c->pages * 4); }

hipError_t launch_pages_fork(const sa_cache4_desc* c, const int32_t* parents, const int32_t* table, const int32_t* lens, const int32_t* refs,
                             int32_t* table_out, int32_t* lens_out, int32_t* refs_out, hipStream_t st) {
  if (refs_out != refs && (long)c->B * c->max_pages + c->pages <= kForkAlone) {
    pages_fork_small_kernel<<<1, kDecide, 0, st>>>(tables_of(c), parents, table, lens, refs, table_out, lens_out, refs_out);
    return hipGetLastError();
  }
  if (refs_out != refs) {
    const int blocks = (c->pages + 255) / 256;
    copy_ints_kernel<<<blocks < 1024 ? blocks : 1024, 256, 0, st>>>(refs, refs_out, c->pages);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  pages_fork_kernel<<<c->B, 256, 0, st>>>(tables_of(c), parents, table, lens, table_out, lens_out, refs_out);
  return hipGetLastError();
}

hipError_t launch_pages_free(const sa_cache4_desc* c, const int32_t* keep, int32_t* table, int32_t* refs, hipStream_t st) {
  pages_free_kernel<<<c->B, 256, 0, st>>>(tables_of(c), keep, table, refs);
  return hipGetLastError();
}

hipError_t launch_pages_extend(const sa_cache4_desc* c, const int32_t* lens, const int32_t* add, int32_t* table, int32_t* refs, void* pool,
                               int32_t* info, void* ws, hipStream_t st) {
  ExtendArgs a;
  a.t = tables_of(c);
  a.lens = lens; a.add = add; a.table = table; a.refs = refs; a.info = info;
  char* base = reinterpret_cast<char*>(ws);
  a.need = reinterpret_cast<int32_t*>(base);
  a.copies = a.need + c->B;
  a.pages = reinterpret_cast<int32_t*>(base + align256((size_t)c->B * 12));
  a.left = reinterpret_cast<int32_t*>(base + align256((size_t)c->B * 12) + align256((size_t)c->pages * 4));
  pages_extend_kernel<<<1, kDecide, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int page_bytes = page_bytes_of(c);
  const dim3 grid((page_bytes + kPiece - 1) / kPiece, c->layers, c->B);
  pages_copy_kernel<<<grid, 256, 0, st>>>(a.copies, reinterpret_cast<unsigned char*>(pool), (size_t)c->pages * page_bytes, page_bytes);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const sa_cache4_desc* c, int max_moves, const int32_t* table, const int32_t* refs, int32_t* table_out,
                                int32_t* refs_out, void* pool, int32_t* info, void* ws, hipStream_t st) {
  CompactArgs a;
  a.t = tables_of(c);
  a.max_moves = max_moves;
  a.table = table; a.refs = refs; a.table_out = table_out; a.refs_out = refs_out; a.info = info;
  char* base = reinterpret_cast<char*>(ws);
  const size_t step = align256((size_t)c->pages * 4);
  a.holes = reinterpret_cast<int32_t*>(base);
  a.movers = reinterpret_cast<int32_t*>(base + step);
  a.to = reinterpret_cast<int32_t*>(base + 2 * step);
  pages_compact_kernel<<<1, kDecide, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int page_bytes = page_bytes_of(c);
  pages_move_kernel<<<kMoveGroups, 256, 0, st>>>(a, reinterpret_cast<unsigned char*>(pool), (size_t)c->pages * page_bytes, page_bytes, c->layers, (page_bytes + kStep - 1) / kStep);
  return hipGetLastError();
}

}  // namespace sa
