// Attention of a batch over a paged KV cache (BaseRT Sec. 3.2: the KV cache;
// Sec. 3.4: attention over key tiles with the running maximum and sum of each
// row), prompts and single tokens together, with the pages of a prefix that all
// requests share read once for all of them.
//
// Token j of request i (of t_i new ones, kv_i cached with them) attends to the
// first n = kv_i - t_i + j + 1 keys of its request:
//   o = sum_{p < n} w_p v_p,  w = softmax(scale q . k_p).
// Keys p < S (the shared prefix) lie in the prefix pages, the others in the
// request's own.  The sum splits at S and at any further place, since
//   o = (sum_s 2^(m_s - M) a_s) / (sum_s 2^(m_s - M) l_s),  M = max m_s,
// over the parts s with their maxima m_s (base 2), sums l_s and sums of values
// a_s, so every part is computed by its own workgroup and the parts of a row
// are joined by a second launch, in a fixed order.
//
// The rows of one KV head are the batch's (token, query head of the group)
// pairs, token-major.  An item is a tile of rows with all the keys that it needs:
//   prefix items:  a tile of rows of any requests  x  the prefix keys,
//   own items:     a tile of one request's rows    x  its own keys.
// Items of more than 16 rows are the work of a workgroup (128 rows, 32 per
// wavefront, keys shared through LDS), bound by MFMA and softmax; the others, a single
// token's group of heads, of a wavefront by itself, bound by HBM.  The items of
// each kind and KV head, laid end to end and each as long as it costs, are cut into
// equal lengths, one for each workgroup (or wavefront) that the CUs hold at once:
// all have the same to do whatever the lengths of the requests, and at most the
// first and the last item of each are parts that have to be joined.  Half of the
// workgroups take their length of the wide items first and half that of the narrow
// ones, so that MFMA and HBM are busy together.  Which items there are follows from
// the offsets and lengths on the device; every workgroup works it out by itself with
// sums over the requests, so the call needs no host copy of the lengths, no plan
// made before it, and can be replayed from a graph while the lengths move on.
#include "lds_dma.h"
#include "qm_internal.h"
#include "wave_scan.h"

#include <algorithm>
#include <cfloat>
#include <cstdio>

namespace qm {
namespace {

typedef _Float16 half4v __attribute__((ext_vector_type(4)));
typedef short short4v __attribute__((ext_vector_type(4)));

// Rows of a tile: 16 where a request (or the whole batch, for the prefix) has no
// more, else 128.  The four wavefronts of a workgroup share the rows of the first
// and split its keys, and split the rows of the second and share its keys.
constexpr int kNarrow = 16, kWide = 128;
__host__ __device__ __forceinline__ int tile_rows(int rows) { return rows <= kNarrow ? kNarrow : kWide; }
// A row's maximum moves only when it grows by more than 2^8, so that the sums are
// rarely rescaled.  Weights go to the second product in fp16, rounded to nearest, as 2^7 w
// relative to it: the largest is 2^15, and they keep 11 bits down to 2^-21.  Sums of
// values and of (rounded) weights carry the same factor, in fp32.  Against 64 bits the
// norm of the error is 2.4 .. 2.9e-4 of the output's with it, 2.07e-4 from the output's own
// rounding to fp16.  A second fp16 term for what the rounding leaves takes that back for
// twice the products: single tokens alone took 3 % (48 of 200 to 20,000 keys, 161 -> 166 us) to
// 9 % (16 of 1,000, 22.1 -> 24.1) longer, and tiles are bound by their products already.
constexpr float kWeightBits = 7.0f, kMaxSlack = 8.0f;

// ------------------------------------------------------------ work units

// Offsets and lengths of the requests, in LDS, within their limits whatever the
// arrays hold.
struct Requests {
  int off[kKvMaxRequests + 1];
  int kv[kKvMaxRequests];
};

__device__ __forceinline__ void load_requests(Requests& r, const PagedAttnArgs& a) {
  const int most = static_cast<int>(min<int64_t>(static_cast<int64_t>(a.max_pages) << a.page_log2, INT32_MAX));
  for (int i = threadIdx.x; i <= a.n_req; i += blockDim.x) {
    r.off[i] = min(max(a.offsets[i], 0), a.tokens);
    if (i < a.n_req) r.kv[i] = min(max(a.kv_lens[i], 0), most);
  }
  __syncthreads();
}

// The request of a token (the last one that starts at or before it).
__device__ __forceinline__ int request_of(const Requests& r, int n, int token) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (r.off[mid] <= token) lo = mid; else hi = mid - 1;
  }
  return lo;
}


// The inclusive sum over the lanes of 0 <= v < 2^49, in two halves.
__device__ __forceinline__ int64_t wave_scan64(int64_t v) {
  const int lo = wave_scan(static_cast<int>(v & 0xFFFFFF)), hi = wave_scan(static_cast<int>(v >> 24));
  return (static_cast<int64_t>(hi) << 24) + lo;
}
__device__ __forceinline__ int64_t lane_value(int64_t v, int lane) {
  const uint32_t lo = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), lane));
  return (static_cast<int64_t>(__builtin_amdgcn_readlane(static_cast<int>(v >> 32), lane)) << 32) | lo;
}

// The two kinds of item: rows of a tile, keys of a block, cost of an item beside
// its keys in blocks (fetching the page ids and the queries, writing the result),
// the fewest blocks of a part.
enum Kind { kNarrowItem = 0, kWideItem = 1 };
template <Kind K> constexpr int kRows = K == kWideItem ? kWide : kNarrow;
template <Kind K> constexpr int kKeys = K == kWideItem ? 64 : 32;
template <Kind K> __device__ __forceinline__ int blocks_of(int keys) { return max((keys + kKeys<K> - 1) / kKeys<K>, 1); }

// The items of one kind of one request (or of the prefix).
struct Items {
  int rows, tiles;
  int64_t base;   // cost of a tile without the keys that its own rows bring
  int slope;      // those: blocks per tile, times 256
  // Cost of the first j tiles.  Later tiles of a prompt see more keys.
  __device__ __forceinline__ int64_t cost(int j) const {
    return j * base + ((static_cast<int64_t>(slope) * j * (j + 1)) >> 9);
  }
};

template <Kind K>
__device__ __forceinline__ Items items_of(const Requests& r, const PagedAttnArgs& a, int i) {
  Items t;
  const int tokens = max(r.off[i + 1] - r.off[i], 0), own = r.kv[i] - (a.prefix_pages << a.page_log2);
  t.rows = tokens * a.group;
  t.tiles = tile_rows(t.rows) == kRows<K> ? (t.rows + kRows<K> - 1) / kRows<K> : 0;
  t.base = a.item_cost[K] + (K == kWideItem ? max(own - tokens, 0) / kKeys<K> : blocks_of<K>(own));
  t.slope = K == kWideItem ? 256 * kWide / (kKeys<K> * a.group) : 0;
  return t;
}

template <Kind K>
__device__ __forceinline__ Items prefix_items(const Requests& r, const PagedAttnArgs& a) {
  Items t{a.prefix_pages ? r.off[a.n_req] * a.group : 0, 0, 0, 0};
  t.tiles = tile_rows(t.rows) == kRows<K> ? (t.rows + kRows<K> - 1) / kRows<K> : 0;
  t.base = a.item_cost[K] + blocks_of<K>(a.prefix_pages << a.page_log2);
  return t;
}

// The line of one kind.  Every lane of a wavefront has `per` consecutive requests;
// before: the cost of everything ahead of them; chunk: the length that a worker takes.
struct Line {
  int per;
  int64_t before, total, chunk;
};

template <Kind K>
__device__ __forceinline__ Line make_line(const Requests& r, const PagedAttnArgs& a) {
  const int lane = threadIdx.x & 63;
  Line n;
  n.per = (a.n_req + 63) / 64;
  const Items shared = prefix_items<K>(r, a);
  const int64_t prefix = shared.cost(shared.tiles);
  int64_t cost = 0;
  for (int i = lane * n.per; i < min((lane + 1) * n.per, a.n_req); ++i) {
    const Items t = items_of<K>(r, a, i);
    cost += t.cost(t.tiles);
  }
  const int64_t upto = wave_scan64(cost);
  n.before = prefix + upto - cost;
  n.total = prefix + lane_value(upto, 63);
  n.chunk = max<int64_t>(static_cast<int64_t>(static_cast<double>(n.total) * a.per_worker[K]) + 1, a.min_chunk[K]);
  if (shared.tiles > 1 && n.chunk < shared.base && shared.base < INT32_MAX) {
    // Tiles of the prefix cut at the same keys are read at the same time, once from
    // HBM for all of them: lengths up to 1/8 longer are taken for that.
    const int whole = static_cast<int>(shared.base), pieces = whole / static_cast<int>(n.chunk);
    const int64_t even = (whole + pieces - 1) / pieces;
    if (8 * (even - n.chunk) <= n.chunk) n.chunk = even;
  }
  return n;
}

// A place on the line: an item and where it starts.
struct Walk {
  int i, tile;                 // request (-1: the prefix), tile
  int64_t start, req_start;
  Items it;
};

template <Kind K>
__device__ __forceinline__ Walk item_at(const Requests& r, const PagedAttnArgs& a, const Line& line, int64_t x) {
  Walk w{-1, 0, 0, 0, prefix_items<K>(r, a)};
  if (x >= w.it.cost(w.it.tiles)) {
    const uint64_t at = __builtin_amdgcn_ballot_w64(line.before <= x);
    const int owner = 63 - __builtin_clzll(at);
    w.req_start = lane_value(line.before, owner);
    w.i = owner * line.per;
    w.it = items_of<K>(r, a, w.i);
    while (w.req_start + w.it.cost(w.it.tiles) <= x && w.i + 1 < a.n_req) {
      w.req_start += w.it.cost(w.it.tiles);
      w.it = items_of<K>(r, a, ++w.i);
    }
  }
  int hi = w.it.tiles - 1;
  while (w.tile < hi) {
    const int mid = (w.tile + hi + 1) >> 1;
    if (w.req_start + w.it.cost(mid) <= x) w.tile = mid; else hi = mid - 1;
  }
  w.start = w.req_start + w.it.cost(w.tile);
  return w;
}

// The next item; there has to be one.
template <Kind K>
__device__ __forceinline__ void next_item(const Requests& r, const PagedAttnArgs& a, Walk& w) {
  if (++w.tile < w.it.tiles) {
    w.start = w.req_start + w.it.cost(w.tile);
    return;
  }
  w.req_start += w.it.cost(w.it.tiles);
  w.start = w.req_start;
  w.tile = 0;
  do {
    w.it = items_of<K>(r, a, ++w.i);
  } while (w.it.tiles == 0 && w.i + 1 < a.n_req);
}

// What the launches that join the parts have to know, at the start of the
// workspace.  Workers of a KV head: its W workgroups for the wide items, its 4 W
// wavefronts for the narrow ones.  Without a prefix: for each worker, wide ones
// first, the item that it has begun and the next `parts` ones go on with.  With
// one, where every row has parts: for each token, for each tile (at the token of its
// first row) and for each prefix tile the workers w0 .. w0 + n - 1 that go on with it.
struct CutItem { int row, rows, parts, blind; };   // rows of the batch; the first `blind` see no key
struct TokenInfo { int j, t, kv, pad; };           // token j of t new ones, kv keys
struct TileParts { int w0, n; };
// Their bytes ahead of the records, a multiple of 16.
__host__ __device__ __forceinline__ int64_t prefix_tiles_most(int64_t tokens, int64_t group) {
  return (tokens * group + kWide - 1) / kWide;
}
__host__ __device__ __forceinline__ int64_t header_bytes(int workgroups, int64_t tokens, int64_t group, bool prefix) {
  return prefix ? (tokens * static_cast<int64_t>(sizeof(TokenInfo) + sizeof(TileParts)) +
                   prefix_tiles_most(tokens, group) * static_cast<int64_t>(sizeof(TileParts)) + 15) / 16 * 16
                : 5 * workgroups * static_cast<int64_t>(sizeof(CutItem));
}
// Rows of records that the workers of one KV head have.
__host__ __device__ __forceinline__ int64_t worker_rows(int workgroups) { return workgroups * (kWide + 4 * kNarrow); }

// Records, (D + 4) floats a row: D sums, maximum, sum of weights, 2 unused.  For each
// worker and KV head the rows of a tile that goes on from the worker before; then as
// many for one that the next goes on with, or, with a prefix, a row per (token,
// query head) for the first part of the own keys and one for that of the prefix.
struct Space {
  CutItem* cut;
  TokenInfo* tokens;
  TileParts* tiles;
  TileParts* prefix_tiles;
  float* records;
};
__device__ __forceinline__ Space space_of(const PagedAttnArgs& a) {
  Space s;
  s.cut = reinterpret_cast<CutItem*>(a.ws);
  s.tokens = reinterpret_cast<TokenInfo*>(a.ws);
  s.tiles = reinterpret_cast<TileParts*>(s.tokens + a.tokens);
  s.prefix_tiles = s.tiles + a.tokens;
  s.records = a.ws + header_bytes(a.workgroups, a.tokens, a.group, a.prefix_pages > 0) / 4;
  return s;
}
template <int D, Kind K>
__device__ __forceinline__ float* going_on(const Space& s, const PagedAttnArgs& a, int w, int head, int row) {
  const int64_t first = K == kWideItem ? 0 : static_cast<int64_t>(a.workgroups) * a.hkv * kWide;
  return s.records + (first + (static_cast<int64_t>(w) * a.hkv + head) * kRows<K> + row) * (D + 4);
}
template <int D, Kind K>
__device__ __forceinline__ float* begun(const Space& s, const PagedAttnArgs& a, int w, int head, int row) {
  return going_on<D, K>(s, a, w, head, row) + worker_rows(a.workgroups) * a.hkv * (D + 4);
}
// at: (token, query head) as an element of [tokens][heads].
template <int D>
__device__ __forceinline__ float* own_row(const Space& s, const PagedAttnArgs& a, int64_t at) {
  return s.records + (worker_rows(a.workgroups) * a.hkv + at) * (D + 4);
}
template <int D>
__device__ __forceinline__ float* prefix_row(const Space& s, const PagedAttnArgs& a, int64_t at) {
  return own_row<D>(s, a, static_cast<int64_t>(a.tokens) * a.hkv * a.group + at);
}

// ---------------------------------------------------- one part of one tile

// The thread's index as the compiler may not know it: what depends on it is worked
// out again for every item instead of being kept in registers across both kinds.
__device__ __forceinline__ int fresh_thread() {
  int t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

// A range of keys behind a page table.
struct Keys {
  const int32_t* pages;   // page ids of positions 0, page, 2 page, ...
  int lo, hi;             // this part's keys: positions [lo, hi); lo is a multiple of 16
};

// An fp16 fragment with its infinities and NaNs as 0; seen is set if there were any.
__device__ __forceinline__ half8v finite_part(half8v v, bool& seen) {
  uint4 w = __builtin_bit_cast(uint4, v);
  uint32_t* x = reinterpret_cast<uint32_t*>(&w);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool lo = (x[i] & 0x7C00u) == 0x7C00u, hi = (x[i] & 0x7C000000u) == 0x7C000000u;
    seen |= lo || hi;
    x[i] = (lo ? 0u : x[i] & 0xFFFFu) | (hi ? 0u : x[i] & 0xFFFF0000u);
  }
  return __builtin_bit_cast(half8v, w);
}

// Sum of the weights of a pair, as rounded, on top of l.  (v_dot2_f32_f16 would be one
// instruction for it, but waits until no MFMA of any wavefront of the SIMD is under
// way: beside MFMAs it takes its time on top of theirs, these two run with them.)
__device__ __forceinline__ float add_pair(half8v w, int i, float l) {
  const uint32_t pair = __builtin_bit_cast(uint32_t, half2v{w[i], w[i + 1]});
  asm("v_fma_mix_f32 %0, %1, 1.0, %0 op_sel_hi:[1,0,0]" : "+v"(l) : "v"(pair));
  asm("v_fma_mix_f32 %0, %1, 1.0, %0 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "+v"(l) : "v"(pair));
  return l;
}

__device__ __forceinline__ half4v read_tr(const _Float16* p) {
  typedef __attribute__((address_space(3))) short4v* lds_ptr;
  return __builtin_bit_cast(half4v, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                        (lds_ptr)(const_cast<short4v*>(reinterpret_cast<const short4v*>(p)))));
}

// K and V in LDS: rows of D halves, the 16-byte chunk c of row r at chunk
// c ^ swizzle(r), so that the 256 bytes that are read at once fall on different banks:
// of K 16 bytes of 16 rows one after the other; of V, transposed, 32 bytes of eight rows
// (narrow tiles) or 64 bytes of four (wide ones).
template <int D>
__device__ __forceinline__ constexpr int k_swizzle(int row) { return D == 64 ? (row >> 1) & 7 : row & 15; }
template <int D, Kind K>
__device__ __forceinline__ constexpr int v_swizzle(int row) {
  return K == kWideItem ? (D == 64 ? 2 * row & 7 : 4 * row & 15) : (D == 64 ? row & 6 : 2 * row & 15);
}
template <int D, Kind K>
__device__ __forceinline__ int v_at(int row, int dim) {
  return row * D + (((dim >> 3) ^ v_swizzle<D, K>(row)) << 3) + (dim & 7);
}

constexpr int kBlock = kKeys<kWideItem>;
template <int D>
struct WideLds {
  _Float16 k[2][kBlock * D], v[2][kBlock * D];   // two blocks: one read, one on its way
  int bad;
};
template <int D>
struct NarrowLds {
  _Float16 v[4][kKeys<kNarrowItem> * D];                 // a block of V per wavefront
};
template <int D>
union TileLds {
  NarrowLds<D> narrow;
  WideLds<D> wide;
};

// One tile of 16 rows against the keys [k.lo, k.hi) of one KV head, by one
// wavefront, 32 keys at a time, the next ones on their way meanwhile:
//   S^T = K Q^T   16 keys x 16 rows, K fragments straight from their pages,
//   O^T += V^T W^T, V^T read transposed out of LDS; its k slots are relabelled to
//   the keys that a lane holds weights of, so the weights never leave their lane.
// limit: keys visible to this lane's row (lane & 15), 0 for rows that do not
// exist.  acc[b][r]: dimension 16 b + 4 (lane / 16) + r of the row; m, l: its maximum
// and sum of weights.  Bound by HBM: 48 single tokens after 200 to 20,000 keys, 870 MB
// of keys in 155 us (16 / 8 heads of 128); one after 32,000, 131 MB in 33 with the join.
template <int D>
__device__ __forceinline__ void narrow_part(const PagedAttnArgs& a, _Float16* vl, const uint16_t* q_row, int limit,
                                            int head, const Keys& k, float4v (&acc)[D / 16], float& m, float& l) {
  constexpr int KS = D / 32, DB = D / 16, VL = D / 16;   // k steps of S, dimension tiles, V loads per lane
  const int lane = fresh_thread() & 63, col = lane & 15, g = lane >> 4;
  const int page_rows = 1 << a.page_log2;
  int most = limit, least = limit > 0 ? limit : INT32_MAX;
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) {
    most = max(most, __shfl_xor(most, o));
    least = min(least, __shfl_xor(least, o));
  }
  const int hi = __builtin_amdgcn_readfirstlane(min(k.hi, most));
  const int all = __builtin_amdgcn_readfirstlane(least);            // keys below are visible to every row
  half8v qf[KS];
#pragma unroll
  for (int c = 0; c < KS; ++c) qf[c] = *reinterpret_cast<const half8v*>(q_row + 32 * c + 8 * g);

  bool bad = false;                                                 // a page id that is none
  // The page ids of 64 times 16 keys are fetched at once, a lane each.
  const int end = (hi - 1) & ~15;
  int ids = 0;
  auto fetch_ids = [&](int key) __attribute__((always_inline)) {
    ids = k.pages[min(key + 16 * lane, end) >> a.page_log2];
    if (static_cast<uint32_t>(ids) >= static_cast<uint32_t>(a.n_pages)) {
      bad = true;
      ids = 0;
    }
  };
  // Row of the pools of the first of 16 keys (past the end: the last ones).
  auto row_of = [&](int key) __attribute__((always_inline)) {
    const int id = __builtin_amdgcn_readlane(ids, (key - k.lo) >> 4 & 63);
    return ((static_cast<int64_t>(id) * a.hkv + head) << a.page_log2) + (min(key, end) & (page_rows - 1));
  };
  struct Blk { half8v k[2][KS], v[VL]; };
  auto load = [&](int kb) __attribute__((always_inline)) {
    Blk b;
    int64_t row[2];
    if (((kb - k.lo) >> 4 & 63) == 0) fetch_ids(kb);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      row[t] = row_of(kb + 16 * t);
#pragma unroll
      for (int c = 0; c < KS; ++c)
        b.k[t][c] = *reinterpret_cast<const half8v*>(a.k_pages + (row[t] + col) * D + 32 * c + 8 * g);
    }
#pragma unroll
    for (int j = 0; j < VL; ++j) {
      const int piece = lane + 64 * j, r = piece / (D / 8);
      b.v[j] = *reinterpret_cast<const half8v*>(a.v_pages + (row[j >= VL / 2] + (r & 15)) * D + piece % (D / 8) * 8);
    }
    return b;
  };
#pragma unroll
  for (int b = 0; b < DB; ++b) acc[b] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
  m = -FLT_MAX;
  l = 0.0f;

  Blk cur;
  if (k.lo < hi) cur = load(k.lo);
  for (int kb = k.lo; kb < hi; kb += 32) {
    const Blk x = cur;
    if (kb + 32 < hi) cur = load(kb + 32);
#pragma unroll
    for (int j = 0; j < VL; ++j) {
      const int piece = lane + 64 * j;
      *reinterpret_cast<half8v*>(&vl[v_at<D, kNarrowItem>(piece / (D / 8), piece % (D / 8) * 8)]) = x.v[j];
    }
    float4v st[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      st[t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < KS; ++c) st[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x.k[t][c], qf[c], st[t], 0, 0, 0);
    }
    // Lane: row col, keys kb + 16 t + 4 g + r.
    const bool masked = kb + 32 > min(all, hi);
    if (masked) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          st[t][r] = kb + 16 * t + 4 * g + r < min(limit, hi) ? st[t][r] : -INFINITY;
    }
    float bm = fmaxf(fmaxf(fmaxf(st[0][0], st[0][1]), fmaxf(st[0][2], st[0][3])),
                     fmaxf(fmaxf(st[1][0], st[1][1]), fmaxf(st[1][2], st[1][3])));
    bm = fmaxf(bm, __shfl_xor(bm, 16));
    bm = fmaxf(bm, __shfl_xor(bm, 32));
    const float mn = bm * a.scale_log2 > m + kMaxSlack ? bm * a.scale_log2 : m;
    const float alpha = __builtin_amdgcn_exp2f(m - mn);
    m = mn;
    half8v w;
    l *= alpha;                                             // of this lane's keys; joined at the end
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; r += 2) {
        const float w0 = __builtin_amdgcn_exp2f(fmaf(st[t][r], a.scale_log2, kWeightBits - mn));
        const float w1 = __builtin_amdgcn_exp2f(fmaf(st[t][r + 1], a.scale_log2, kWeightBits - mn));
        w[4 * t + r] = static_cast<_Float16>(w0);           // to nearest: errors of the weights average out
        w[4 * t + r + 1] = static_cast<_Float16>(w1);
        l = add_pair(w, 4 * t + r, l);
      }
    if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
      for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[b][r] *= alpha;
    }
    // k slot (g, j) of the second product: key 16 (j / 4) + 4 g + j % 4.
    auto value = [&](int b) __attribute__((always_inline)) {
      const half4v lo = read_tr(&vl[v_at<D, kNarrowItem>(4 * g + (col >> 2), 16 * b + 4 * (col & 3))]);
      const half4v up = read_tr(&vl[v_at<D, kNarrowItem>(16 + 4 * g + (col >> 2), 16 * b + 4 * (col & 3))]);
      return half8v{lo[0], lo[1], lo[2], lo[3], up[0], up[1], up[2], up[3]};
    };
    if (!masked) {
#pragma unroll
      for (int b = 0; b < DB; ++b) acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(value(b), w, acc[b], 0, 0, 0);
    } else {
      // Some row does not see some key of the block: 0 x infinity must not reach
      // it.  Infinities and NaNs leave the product and are added to the rows that
      // see them.
      bool odd = false;
#pragma unroll
      for (int b = 0; b < DB; ++b)
        acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(finite_part(value(b), odd), w, acc[b], 0, 0, 0);
      if (__builtin_amdgcn_ballot_w64(odd) != 0) {
        for (int key = 0; key < 32; ++key) {
          if (kb + key < min(limit, hi)) {
#pragma unroll
            for (int b = 0; b < DB; ++b)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const float x = static_cast<float>(vl[v_at<D, kNarrowItem>(key, 16 * b + 4 * g + r)]);
                acc[b][r] += __builtin_fabsf(x) < INFINITY ? 0.0f : x;
              }
          }
        }
      }
    }
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (__builtin_amdgcn_ballot_w64(bad) != 0) l = __builtin_nanf("");
}

// One tile of 128 rows against the keys [k.lo, hi) of one KV head: wavefront w has
// rows 32 w .. 32 w + 31, and all share the blocks of 64 keys that come into LDS by
// DMA, each wavefront copying 16 keys of K and V, while the block before is worked on.
//   S^T = K Q^T   32 keys x 32 rows at a time, K fragments out of LDS,
//   O^T += V^T W^T as in narrow_part.
// limit: keys visible to this lane's row (lane & 31).  acc[b][r]: dimension
// 32 b + 8 (r / 4) + 4 (lane / 32) + r % 4 of the row; m, l: its maximum and this
// lane's share of the sum of weights.  Per block a wavefront takes 512 cycles of MFMA and
// 860 of VALU with heads of 64, 1,024 and 990 with heads of 128, which overlap between
// wavefronts in part: a prompt of 1,024 tokens after 16,384 at 752 and 884 TFLOP/s (32 / 8
// heads), 1,000 tokens after 16,384 shared ones at 734 (24 / 8 heads of 128).
// Blocks that every row sees have a loop of their own: with a branch for the others in
// it the compiler copied all sums twice a block (that and the reads of fragments eight
// at a time: 345 -> 326 us for this prompt with heads of 128).
template <int D>
__device__ __forceinline__ void wide_part(const PagedAttnArgs& a, WideLds<D>& s, const uint16_t* q_row, int limit,
                                          int head, const Keys& k, float16v (&acc)[D / 32], float& m, float& l) {
  constexpr int KS = D / 16, DB = D / 32, C = D / 8, PIECES = D / 32;   // PIECES: KiB of 16 keys
  // Fragments of V read before the softmax (heads of 64: no more fit in registers).
  constexpr int AHEAD = D == 64 ? 6 : 8;
  const int thread = fresh_thread(), lane = thread & 63, col = lane & 31, lh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(thread >> 6);
  const int page_rows = 1 << a.page_log2, hi = k.hi;
  int most = limit, least = limit > 0 ? limit : INT32_MAX;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    most = max(most, __shfl_xor(most, o));
    least = min(least, __shfl_xor(least, o));
  }
  most = __builtin_amdgcn_readfirstlane(min(most, hi));             // nothing for this wavefront from here on
  // Keys below are visible to every row.  None where the wavefront has no row that sees any: it copies its
  // share of the blocks and multiplies nothing (64 requests of 5 tokens after 4,000, 32 / 8 heads of 64, three
  // of four wavefronts without rows: 122 us with their products, 109 without).
  const int all = __builtin_amdgcn_readfirstlane(min(least, most));
  half8v qf[KS];
#pragma unroll
  for (int c = 0; c < KS; ++c) qf[c] = *reinterpret_cast<const half8v*>(q_row + 16 * c + 8 * lh);
  if (thread == 0) s.bad = 0;
#pragma unroll
  for (int b = 0; b < DB; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[b][r] = 0.0f;
  m = -FLT_MAX;
  l = 0.0f;

  // This wavefront's 16 keys of a block (keys past the end: the last ones).  The page
  // ids of 64 blocks are fetched at once, a lane each: a load in the loop would wait
  // for the copies under way.
  const int last = (hi - 1) & ~15;
  bool bad = false;
  int ids = 0;
  auto fetch_ids = [&](int kb) __attribute__((always_inline)) {
    ids = k.pages[min(kb + kBlock * lane + 16 * wave, last) >> a.page_log2];
    if (static_cast<uint32_t>(ids) >= static_cast<uint32_t>(a.n_pages)) {
      bad = true;
      ids = 0;
    }
  };
  // Of a piece: 64 / C rows of C chunks; byte offsets from the first row.
  uint32_t k_off[PIECES], v_off[PIECES];
#pragma unroll
  for (int j = 0; j < PIECES; ++j) {
    const int r = j * (64 / C) + lane / C;
    k_off[j] = 2 * (r * D + (((lane % C) ^ k_swizzle<D>(r)) << 3));
    v_off[j] = 2 * (r * D + (((lane % C) ^ v_swizzle<D, kWideItem>(r)) << 3));
  }
  auto copy = [&](int buf, int kb) __attribute__((always_inline)) {
    const int n = (kb - k.lo) / kBlock & 63;
    if (n == 0) fetch_ids(kb);
    const int id = __builtin_amdgcn_readlane(ids, n);
    const int t = min(kb + 16 * wave, last) & (page_rows - 1);
    const int64_t row = ((static_cast<int64_t>(id) * a.hkv + head) << a.page_log2) + t;
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
      qg::lds_dma16(a.k_pages + row * D, k_off[j], &s.k[buf][16 * wave * D + 512 * j]);
      qg::lds_dma16(a.v_pages + row * D, v_off[j], &s.v[buf][16 * wave * D + 512 * j]);
    }
  };
  auto compute = [&]<bool MASKED>(int buf, int kb) __attribute__((always_inline)) {
    const _Float16* const kl = s.k[buf];
    const _Float16* const vl = s.v[buf];
    float16v st[2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) st[t][r] = 0.0f;
    // Fragments in groups of eight, read ahead of their use (left to itself the compiler
    // reads one, waits for it and multiplies).
    auto key_at = [&](int c, int t) __attribute__((always_inline)) {
      return *reinterpret_cast<const half8v*>(&kl[(32 * t + col) * D + (((2 * c + lh) ^ k_swizzle<D>(col)) << 3)]);
    };
    half8v kf[2 * KS];
    float bm = -INFINITY;
#pragma unroll
    for (int x = 0; x < 8; ++x) kf[x] = key_at(x % KS, x / KS);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int c = 0; c < KS; ++c) {
      st[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[c], qf[c], st[0], 0, 0, 0);
      if (KS > 4) {
        kf[KS + c] = key_at(c, 1);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    // (the first keys' maxima while the second ones' products are on their way)
#pragma unroll
    for (int c = 0; c < KS; ++c) {
      st[1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[KS + c], qf[c], st[1], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (!MASKED) {
#pragma unroll
        for (int r = c * 16 / KS; r < (c + 1) * 16 / KS; ++r) bm = fmaxf(bm, st[0][r]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    // k slot (lh, j) of step kk: key 16 kk + 8 (j / 4) + 4 lh + j % 4.
    auto value = [&](int kk, int b) __attribute__((always_inline)) {
      const int row = 16 * kk + 4 * lh + ((lane & 15) >> 2), dim = 32 * b + (col & 16) + 4 * (lane & 3);
      const half4v lo = read_tr(&vl[v_at<D, kWideItem>(row, dim)]);
      const half4v up = read_tr(&vl[v_at<D, kWideItem>(row + 8, dim)]);
      return half8v{lo[0], lo[1], lo[2], lo[3], up[0], up[1], up[2], up[3]};
    };
    half8v vf[4 * DB];
    if constexpr (!MASKED) {
#pragma unroll
      for (int x = 0; x < AHEAD; ++x) vf[x] = value(x / DB, x % DB);
      __builtin_amdgcn_sched_barrier(0);
    }
    // Lane: row col, keys kb + 32 t + 8 (r / 4) + 4 lh + r % 4.
    if constexpr (MASKED) {
      const int seen = min(limit, hi) - kb - 4 * lh;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) st[t][r] = 32 * t + 8 * (r >> 2) + (r & 3) < seen ? st[t][r] : -INFINITY;
    }
#pragma unroll
    for (int t = MASKED ? 0 : 1; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) bm = fmaxf(bm, st[t][r]);
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(bm), __float_as_uint(bm), false, false);
    bm = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * a.scale_log2;
    const float mn = bm > m + kMaxSlack ? bm : m;
    if (__builtin_amdgcn_ballot_w64(mn != m) != 0) {
      const float alpha = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= alpha;
#pragma unroll
      for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[b][r] *= alpha;
    }
    const float shift = kWeightBits - m;
    half8v w[4];
    auto weights = [&](int p) __attribute__((always_inline)) {   // pair p of 16
      const int t = p / 8, r = 2 * (p % 8);
      half8v& x = w[2 * t + (r >> 3)];
      x[r & 7] = static_cast<_Float16>(__builtin_amdgcn_exp2f(fmaf(st[t][r], a.scale_log2, shift)));
      x[(r & 7) + 1] = static_cast<_Float16>(__builtin_amdgcn_exp2f(fmaf(st[t][r + 1], a.scale_log2, shift)));
      l = add_pair(x, r & 7, l);
    };
#pragma unroll
    for (int p = 0; p < 8; ++p) weights(p);
    if constexpr (!MASKED) {
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int x = AHEAD; x < 4 * DB; ++x) vf[x] = value(x / DB, x % DB);
      __builtin_amdgcn_sched_barrier(0);
      auto product = [&](int x) __attribute__((always_inline)) {
        acc[x % DB] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[x], w[x / DB], acc[x % DB], 0, 0, 0);
      };
      // (the second keys' weights between the first ones' products)
#pragma unroll
      for (int p = 0; p < 4; ++p) {
#pragma unroll
        for (int x = p * DB / 2; x < (p + 1) * DB / 2; ++x) product(x);
        weights(8 + 2 * p);
        weights(9 + 2 * p);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int x = 2 * DB; x < 4 * DB; ++x) product(x);
    } else {                                                // as in narrow_part
#pragma unroll
      for (int p = 8; p < 16; ++p) weights(p);
      bool odd = false;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
#pragma unroll
        for (int b = 0; b < DB; ++b)
          acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(finite_part(value(kk, b), odd), w[kk], acc[b], 0, 0, 0);
      if (__builtin_amdgcn_ballot_w64(odd) != 0) {
        for (int key = 0; key < kBlock; ++key) {
          if (kb + key < min(limit, hi)) {
#pragma unroll
            for (int b = 0; b < DB; ++b)
#pragma unroll
              for (int r = 0; r < 16; ++r) {
                const float x = static_cast<float>(vl[v_at<D, kWideItem>(key, 32 * b + 8 * (r >> 2) + 4 * lh + (r & 3))]);
                acc[b][r] += __builtin_fabsf(x) < INFINITY ? 0.0f : x;
              }
          }
        }
      }
    }
  };
  // A block that this wavefront has copied is there and its reads of the other one are
  // done; after the barrier so are everybody's.
  auto step = [&](int buf, int kb) __attribute__((always_inline)) {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);                     // lgkmcnt(0)
    qg::vm_wait<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (kb + kBlock < hi) copy(buf ^ 1, kb + kBlock);
  };
  if (k.lo < hi) {
    copy(0, k.lo);
    int buf = 0, kb = k.lo;
    for (; kb + kBlock <= all; kb += kBlock, buf ^= 1) {
      step(buf, kb);
      compute.template operator()<false>(buf, kb);
    }
    for (; kb < hi; kb += kBlock, buf ^= 1) {
      step(buf, kb);
      if (kb < most) compute.template operator()<true>(buf, kb);
    }
  }
  __syncthreads();
  if (bad) s.bad = 1;                                       // (any lane: an id outside the pool among those fetched)
  __syncthreads();
  const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
  l = __uint_as_float(both[0]) + __uint_as_float(both[1]);
  if (s.bad) l = __builtin_nanf("");
}

// Four dimensions of a row's result: the output, or a part's record.
template <int D>
__device__ __forceinline__ void write4(uint16_t* out, float* rec, int dim, float4v v, float inv, bool none) {
  if (out) {
    half4v h;
#pragma unroll
    for (int c = 0; c < 4; ++c) h[c] = static_cast<_Float16>(none ? 0.0f : v[c] * inv);
    *reinterpret_cast<half4v*>(out + dim) = h;
  } else {
    *reinterpret_cast<float4v*>(rec + dim) = v;
  }
}

// Worker w's length of the line of kind K.
template <int D, Kind K, class Lds>
__device__ __forceinline__ void work_line(const PagedAttnArgs& a, const Requests& req, const Line& line, Lds& s, int w,
                                          int head) {
  const Space space = space_of(a);
  const int prefix_len = a.prefix_pages << a.page_log2;
  const int64_t hq = static_cast<int64_t>(a.hkv) * a.group;
  const int64_t x0 = w * line.chunk, x1 = min(x0 + line.chunk, line.total);
  CutItem* const cut = space.cut + (K == kWideItem ? w : a.workgroups + w);
  const bool teller = head == 0 && (K == kWideItem ? threadIdx.x == 0 : (threadIdx.x & 63) == 0);
  bool begins = false;                                      // an item that the next worker goes on with
  if (x0 < line.total) {
    Walk at = item_at<K>(req, a, line, x0);
    for (;;) {
      const bool shared = at.i < 0;
      const int i = at.i;
      const int64_t end = at.req_start + at.it.cost(at.tile + 1);
      const int row0 = at.tile * kRows<K>, last = min(row0 + kRows<K>, at.it.rows) - 1;
      const int t = shared ? 0 : at.it.rows / a.group;
      const int seen = shared ? prefix_len : min(req.kv[i], req.kv[i] - t + last / a.group + 1);   // keys of the last row
      const int first_key = shared ? 0 : prefix_len;
      const int blocks = blocks_of<K>(seen - first_key), least = a.min_part[K];
      // Blocks of the item ahead of a place on the line; what would be a very short
      // part goes to its neighbour.
      auto ahead = [&](int64_t x) __attribute__((always_inline)) {
        const int64_t b = x - at.start - a.item_cost[K];
        return x >= end ? blocks : b < 0 ? 0 : b > blocks - least ? blocks : b < least ? 0 : static_cast<int>(b);
      };
      const int from = ahead(x0), to = ahead(x1);
      if (from < to) {
        const int thread = fresh_thread(), lane = thread & 63, group_thread = K == kWideItem ? thread : lane;
        if (from == 0 && head == 0) {
          // Workers w + 1 .. w + n go on with the item: those whose length begins
          // `least` blocks or more before its end.
          const int64_t left = min(at.start + a.item_cost[K] + blocks - least, end - 1) - (w + 1) * line.chunk;
          const int n = to == blocks ? 0 : static_cast<int>(left / line.chunk) + 1;
          if (!a.prefix_pages) {
            // The rows of the batch, those of them that see no key.
            if (n && group_thread == 0)
              *cut = CutItem{req.off[i] * a.group + row0, last + 1 - row0, n,
                             min(max((t - req.kv[i]) * a.group - row0, 0), kWide)};
            begins = begins || n;
          } else if (shared) {
            if (group_thread == 0) space.prefix_tiles[at.tile] = TileParts{w + 1, n};
          } else {
            if (group_thread == 0) space.tiles[req.off[i] + row0 / a.group] = TileParts{w + 1, n};
            // The tokens whose first row is in this tile.
            for (int j = (row0 + a.group - 1) / a.group + group_thread; j * a.group <= last; j += K == kWideItem ? 256 : 64)
              space.tokens[req.off[i] + j] = TokenInfo{j, t, req.kv[i], 0};
          }
        }
        const bool whole = !a.prefix_pages && from == 0 && to == blocks;
        Keys k;
        k.pages = shared ? a.prefix : a.tables + static_cast<int64_t>(i) * a.max_pages;
        k.lo = first_key + from * kKeys<K>;
        k.hi = min(seen, first_key + to * kKeys<K>);
        // This lane's row of the tile.
        const int col = K == kWideItem ? (thread >> 6) * 32 + (lane & 31) : lane & 15;
        const int row = min(row0 + col, last);
        int token = row / a.group;
        const int gq = row - token * a.group;
        const int r = shared ? request_of(req, a.n_req, token) : i;
        if (!shared) token += req.off[i];
        const int sees = max(min(req.kv[r], req.kv[r] - max(req.off[r + 1] - token, 0) + 1), 0);
        const int limit = row0 + col > last ? 0 : shared ? min(sees, prefix_len) : sees;
        const int64_t el = token * hq + head * a.group + gq;  // of q and out
        float m, l;
        float16v wide[D / 32];
        float4v narrow[D / 16];
        if constexpr (K == kWideItem) wide_part<D>(a, s, a.q + el * D, limit, head, k, wide, m, l);
        else narrow_part<D>(a, s.v[__builtin_amdgcn_readfirstlane(thread >> 6)], a.q + el * D, limit, head, k, narrow, m, l);
        if (row0 + col <= last) {
          uint16_t* const out = whole ? a.out + el * D : nullptr;
          float* const rec = from ? going_on<D, K>(space, a, w, head, col)
                             : !a.prefix_pages ? begun<D, K>(space, a, w, head, col)
                             : shared ? prefix_row<D>(space, a, el) : own_row<D>(space, a, el);
          const float inv = 1.0f / l;
          if constexpr (K == kWideItem) {
            const int lh = lane >> 5;
#pragma unroll
            for (int b = 0; b < D / 32; ++b)
#pragma unroll
              for (int q = 0; q < 16; q += 4)
                write4<D>(out, rec, 32 * b + 2 * q + 4 * lh,
                          float4v{wide[b][q], wide[b][q + 1], wide[b][q + 2], wide[b][q + 3]}, inv, sees == 0);
          } else {
#pragma unroll
            for (int b = 0; b < D / 16; ++b) write4<D>(out, rec, 16 * b + 4 * (lane >> 4), narrow[b], inv, sees == 0);
          }
          if (!whole && lane < (K == kWideItem ? 32 : 16)) {
            rec[D] = m;
            rec[D + 1] = l;
          }
        }
        if (K == kWideItem) __syncthreads();                // the tile's LDS is free
      }
      if (end >= x1) break;
      next_item<K>(req, a, at);
    }
  }
  if (!a.prefix_pages && !begins && teller) cut->parts = 0;
}

// Workgroups that a CU holds at once, by registers and LDS.
template <int D>
constexpr int kResident = D == 64 ? 3 : 2;

template <int D>
__global__ __launch_bounds__(256, kResident<D>) void paged_attn_kernel(PagedAttnArgs a) {
  __shared__ Requests req;
  __shared__ __attribute__((aligned(1024))) TileLds<D> s;
  load_requests(req, a);
  const int head = static_cast<int>(blockIdx.x % a.hkv), wg = static_cast<int>(blockIdx.x / a.hkv);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // A CU holds workgroups of both halves of the grid.  Where there are fewer narrow
  // lengths than wavefronts, they go to the last workgroups, the wide ones to the first.
  const int narrow_first = 2 * blockIdx.x >= gridDim.x;
  for (int phase = 0; phase < 2; ++phase) {
    if (phase == narrow_first) {
      const Line line = make_line<kWideItem>(req, a);
      work_line<D, kWideItem>(a, req, line, s.wide, wg, head);
    } else {
      const Line line = make_line<kNarrowItem>(req, a);
      work_line<D, kNarrowItem>(a, req, line, s.narrow, 4 * (a.workgroups - 1 - wg) + wave, head);
      __syncthreads();                                      // the wide tiles' LDS is free
    }
  }
}

// The same where all items are narrow: less LDS to wait for, nothing of the wide ones.
template <int D>
__global__ __launch_bounds__(256, kResident<D>) void paged_attn_narrow_kernel(PagedAttnArgs a) {
  __shared__ Requests req;
  __shared__ __attribute__((aligned(1024))) NarrowLds<D> s;
  load_requests(req, a);
  const int head = static_cast<int>(blockIdx.x % a.hkv), wg = static_cast<int>(blockIdx.x / a.hkv);
  work_line<D, kNarrowItem>(a, req, make_line<kNarrowItem>(req, a), s,
                            4 * wg + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), head);
}

// Parts s0, s0 + step, ... of a row, each with its weight relative to the largest
// maximum so far; rec(s): the record of part s, d4: this thread's four dimensions.
struct Joined { float4v o; float m, l; };
template <int D, int BATCH, class Rec>                      // BATCH: records on their way at once
__device__ __forceinline__ void join_batch(Joined& r, int s0, int step, int parts, int d4, Rec rec) {
  float4v v[BATCH];
  float ms[BATCH], ls[BATCH];
#pragma unroll
  for (int b = 0; b < BATCH; ++b) {
    const float* p = rec(min(s0 + b * step, parts - 1));
    v[b] = *reinterpret_cast<const float4v*>(p + 4 * d4);
    ms[b] = p[D];
    ls[b] = p[D + 1];
  }
  float mn = r.m;
#pragma unroll
  for (int b = 0; b < BATCH; ++b) mn = fmaxf(mn, ms[b]);
  const float f0 = __builtin_amdgcn_exp2f(r.m - mn);
  r.m = mn;
  r.l *= f0;
#pragma unroll
  for (int c = 0; c < 4; ++c) r.o[c] *= f0;
#pragma unroll
  for (int b = 0; b < BATCH; ++b) {
    if (s0 + b * step >= parts) continue;
    const float f = __builtin_amdgcn_exp2f(ms[b] - mn);
    r.l = fmaf(ls[b], f, r.l);
#pragma unroll
    for (int c = 0; c < 4; ++c) r.o[c] = fmaf(v[b][c], f, r.o[c]);
  }
}
template <int D, class Rec>
__device__ __forceinline__ Joined join_parts(int s0, int step, int parts, int d4, Rec rec) {
  Joined r{float4v{0.0f, 0.0f, 0.0f, 0.0f}, -FLT_MAX, 0.0f};
  for (; parts - s0 > 4 * step; s0 += 12 * step) join_batch<D, 12>(r, s0, step, parts, d4, rec);
  if (s0 < parts) join_batch<D, 4>(r, s0, step, parts, d4, rec);
  return r;
}

// The groups of `width` threads of a workgroup joined in order; whole workgroup.
__device__ __forceinline__ Joined join_groups(Joined r, int groups, int width) {
  __shared__ float4v part[256];
  __shared__ float2 stat[256];
  const int th = threadIdx.x % width;
  part[threadIdx.x] = r.o;
  stat[threadIdx.x] = make_float2(r.m, r.l);
  __syncthreads();
  r = Joined{float4v{0.0f, 0.0f, 0.0f, 0.0f}, -FLT_MAX, 0.0f};
  for (int x = 0; x < groups; ++x) r.m = fmaxf(r.m, stat[x * width + th].x);
  for (int x = 0; x < groups; ++x) {
    const float2 st = stat[x * width + th];
    const float f = __builtin_amdgcn_exp2f(st.x - r.m);
    r.l = fmaf(st.y, f, r.l);
#pragma unroll
    for (int c = 0; c < 4; ++c) r.o[c] = fmaf(part[x * width + th][c], f, r.o[c]);
  }
  return r;
}

template <int D>
__device__ __forceinline__ void write_joined(const PagedAttnArgs& a, int64_t at, int d4, const Joined& r, bool none) {
  half4v h;
#pragma unroll
  for (int c = 0; c < 4; ++c) h[c] = static_cast<_Float16>(none ? 0.0f : r.o[c] / r.l);
  *reinterpret_cast<half4v*>(a.out + at * D + 4 * d4) = h;
}

// Element of [tokens][heads] of a row of the batch.
__device__ __forceinline__ int64_t element_of(const PagedAttnArgs& a, int row, int head) {
  const int token = row / a.group;
  return static_cast<int64_t>(token) * a.hkv * a.group + head * a.group + (row - token * a.group);
}

// Without a prefix: the items that are cut.  A row has D / 4 threads, four dimensions
// each.  A workgroup takes the narrow items that four workers have begun, a wavefront
// each, or all threads for one that has many parts, groups of them sharing the parts;
// or 32 rows of a wide item.  (A workgroup for every possible item and few rows left
// thousands without work: 9.4 us against 4.7 for 16 sequences of 1,000 keys, 16 / 8
// heads of 128.)  QUARTERS: 4 where the batch has 16 rows at most and so few items,
// of many parts: four workgroups for each, a quarter of the dimensions each (one
// sequence of 32,000 keys, 250 parts: 11.4 -> 8.0 us).
constexpr int kManyParts = 8, kJoinRows = 32;

template <int D, int QUARTERS>
__global__ __launch_bounds__(256) void paged_attn_join_kernel(PagedAttnArgs a) {
  constexpr int C4 = D / 4;
  const Space space = space_of(a);
  const int head = static_cast<int>(blockIdx.x % a.hkv), x = static_cast<int>(blockIdx.x / a.hkv);
  if (x < QUARTERS * a.workgroups) {
    const int wg = x % a.workgroups, quarter = x / a.workgroups;
    CutItem its[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) its[i] = space.cut[a.workgroups + 4 * wg + i];
    auto rec_of = [&](int w, int row) __attribute__((always_inline)) {
      return [&space, &a, w, head, row](int part) __attribute__((always_inline)) {
        return part == 0 ? begun<D, kNarrowItem>(space, a, w, head, row)
                         : going_on<D, kNarrowItem>(space, a, min(w + part, 4 * a.workgroups - 1), head, row);
      };
    };
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const CutItem it = its[i];
      if (it.parts <= kManyParts) continue;
      constexpr int Q4 = C4 / QUARTERS;
      int groups = 1;
      while (2 * groups * it.rows * Q4 <= 256) groups *= 2;
      const int width = 256 / groups, grp = threadIdx.x / width;
      for (int e0 = 0; e0 < it.rows * Q4; e0 += width) {    // (once where there are several groups)
        const int e = e0 + threadIdx.x % width, row = min(e / Q4, it.rows - 1), d4 = quarter * Q4 + e % Q4;
        Joined r = join_parts<D>(grp, groups, it.parts + 1, d4, rec_of(4 * wg + i, row));
        if (groups > 1) r = join_groups(r, groups, width);
        if (grp == 0 && e < it.rows * Q4) write_joined<D>(a, element_of(a, it.row + row, head), d4, r, row < it.blind);
      }
      __syncthreads();                                      // (the next item's groups)
    }
    if (quarter) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const CutItem it = space.cut[a.workgroups + 4 * wg + wave];
    if (it.parts == 0 || it.parts > kManyParts) return;
    for (int e = threadIdx.x & 63; e < it.rows * C4; e += 64) {
      const int row = e / C4, d4 = e % C4;
      write_joined<D>(a, element_of(a, it.row + row, head), d4,
                      join_parts<D>(0, 1, it.parts + 1, d4, rec_of(4 * wg + wave, row)), row < it.blind);
    }
  } else {
    const int w = x % a.workgroups, row0 = (x / a.workgroups - QUARTERS) * kJoinRows;
    const CutItem it = space.cut[w];
    if (it.parts == 0) return;
    for (int e = threadIdx.x; e < min(it.rows - row0, kJoinRows) * C4; e += 256) {
      const int row = row0 + e / C4, d4 = e % C4;
      auto rec = [&](int part) __attribute__((always_inline)) {
        return part == 0 ? begun<D, kWideItem>(space, a, w, head, row)
                         : going_on<D, kWideItem>(space, a, min(w + part, a.workgroups - 1), head, row);
      };
      write_joined<D>(a, element_of(a, it.row + row, head), d4, join_parts<D>(0, 1, it.parts + 1, d4, rec), row < it.blind);
    }
  }
}

// With a prefix every row has parts: a workgroup of `groups` groups takes
// 256 / groups / (D / 4) rows of the batch.
template <int D>
__global__ __launch_bounds__(256) void paged_attn_join_rows_kernel(PagedAttnArgs a, int groups) {
  constexpr int C4 = D / 4;
  const Space space = space_of(a);
  const int head = static_cast<int>(blockIdx.x % a.hkv);
  const int tokens = min(max(a.offsets[a.n_req], 0), a.tokens), rows = tokens * a.group;
  const int width = 256 / groups, grp = threadIdx.x / width, th = threadIdx.x % width;
  const int row = static_cast<int>(blockIdx.x / a.hkv) * (width / C4) + th / C4, d4 = th % C4;
  if (row - th / C4 >= rows) return;                        // whole workgroup
  const int prow = min(row, rows - 1), token = prow / a.group, gq = prow - token * a.group;
  const TokenInfo tp = space.tokens[token];
  // (The test holds whatever lies there for a token of no request, where offsets do not rise.)
  const bool there = row < rows && tp.j >= 0 && tp.j <= token && tp.t > tp.j && tp.t <= a.tokens;
  const int own = there ? tp.j * a.group + gq : 0;          // row of the request
  const int per = tile_rows(there ? tp.t * a.group : 0), prefix_per = tile_rows(rows);
  const TileParts op = space.tiles[there ? token - tp.j + own / per * per / a.group : 0];
  const TileParts pp = space.prefix_tiles[prow / prefix_per];
  const int64_t at = element_of(a, prow, head);
  const int own_at = min(max(pp.n, 0), 4 * a.workgroups) + 1;   // parts of the prefix
  const int parts = own_at + 1 + min(max(op.n, 0), 4 * a.workgroups);
  auto on = [&](int w, int rows_per, int r) __attribute__((always_inline)) {
    return rows_per == kWide ? going_on<D, kWideItem>(space, a, min(max(w, 0), a.workgroups - 1), head, r % kWide)
                             : going_on<D, kNarrowItem>(space, a, min(max(w, 0), 4 * a.workgroups - 1), head, r % kNarrow);
  };
  auto rec = [&](int x) __attribute__((always_inline)) {
    if (x == 0) return prefix_row<D>(space, a, at);
    if (x < own_at) return on(pp.w0 + x - 1, prefix_per, prow);
    if (x == own_at) return own_row<D>(space, a, at);
    return on(op.w0 + x - own_at - 1, per, own);
  };
  Joined r = join_parts<D>(grp, groups, there ? parts : 0, d4, rec);
  if (groups > 1) r = join_groups(r, groups, width);
  if (grp == 0 && there) write_joined<D>(a, at, d4, r, tp.kv - tp.t + tp.j + 1 <= 0);
}

// Workgroups per KV head: those that the CUs hold at once.
int workgroups_of(int hkv, int d, int cu_count) {
  return std::max(1, (d == 64 ? kResident<64> : kResident<128>) * cu_count / hkv);
}

}  // namespace

size_t attn_paged_workspace_bytes(int32_t hq, int32_t hkv, int32_t d, int64_t tokens, bool prefix, int cu_count) {
  const int workgroups = workgroups_of(hkv, d, cu_count);
  const int64_t slots = worker_rows(workgroups) * hkv;
  const int64_t records = prefix ? slots + 2 * tokens * hq : 2 * slots;
  return static_cast<size_t>(header_bytes(workgroups, tokens, hq / hkv, prefix)) +
         static_cast<size_t>(records) * (d + 4) * sizeof(float);
}

namespace {

template <int D>
hipError_t launch_paged(const PagedAttnArgs& a, hipStream_t st) {
  const bool narrow = static_cast<int64_t>(a.tokens) * a.group <= kNarrow;
  const unsigned workgroups = static_cast<unsigned>(a.workgroups * a.hkv);
  if (narrow) hipLaunchKernelGGL(paged_attn_narrow_kernel<D>, dim3(workgroups), dim3(256), 0, st, a);
  else hipLaunchKernelGGL(paged_attn_kernel<D>, dim3(workgroups), dim3(256), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (!a.prefix_pages) {
    if (narrow) hipLaunchKernelGGL((paged_attn_join_kernel<D, 4>), dim3(workgroups * 4), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((paged_attn_join_kernel<D, 1>), dim3(workgroups * (1 + kWide / kJoinRows)), dim3(256), 0, st, a);
    return hipGetLastError();
  }
  // More groups a row while that leaves at most about 1,024 workgroups.
  const int64_t rows = static_cast<int64_t>(a.tokens) * a.group;
  int groups = 1;
  auto blocks = [&](int g) { return (rows + 256 / g / (D / 4) - 1) / (256 / g / (D / 4)) * a.hkv; };
  while (2 * groups * (D / 4) <= 256 && blocks(2 * groups) <= 1024) groups *= 2;
  hipLaunchKernelGGL(paged_attn_join_rows_kernel<D>, dim3(static_cast<unsigned>(blocks(groups))), dim3(256), 0, st, a, groups);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_paged(PagedAttnArgs a, int32_t d, int cu_count, hipStream_t st) {
  if (a.tokens == 0) return hipSuccess;
  a.item_cost[kNarrowItem] = 1;
  a.item_cost[kWideItem] = 2;
  a.min_chunk[kNarrowItem] = 2;
  a.min_chunk[kWideItem] = 4;
  a.min_part[kNarrowItem] = 1;
  a.min_part[kWideItem] = 3;
  if (const char* e = tuning_override("QM_PAGED_PLAN"))
    std::sscanf(e, "%d,%d,%d,%d,%d,%d", &a.item_cost[0], &a.item_cost[1], &a.min_chunk[0], &a.min_chunk[1], &a.min_part[0],
                &a.min_part[1]);
  // No more workgroups than the page tables leave work for.
  const int64_t most_keys = static_cast<int64_t>(a.max_pages) << a.page_log2;
  const int64_t narrow = std::min(a.n_req, a.tokens) * (a.item_cost[kNarrowItem] + (most_keys + 31) / 32) / a.min_chunk[kNarrowItem];
  const int64_t wide = static_cast<int64_t>(a.tokens) * a.group <= kNarrow
                           ? 0
                           : 2 * (static_cast<int64_t>(a.tokens) * a.group / kWide + a.n_req + 1) *
                                 (a.item_cost[kWideItem] + (most_keys + 63) / 64) / a.min_chunk[kWideItem];
  a.workgroups = static_cast<int>(std::min<int64_t>(workgroups_of(a.hkv, d, cu_count), std::max((narrow + 3) / 4, wide) + 2));
  a.per_worker[kWideItem] = 1.0 / a.workgroups;
  a.per_worker[kNarrowItem] = 0.25 / a.workgroups;
  return d == 64 ? launch_paged<64>(a, st) : launch_paged<128>(a, st);
}

}  // namespace qm
