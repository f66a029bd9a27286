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
// The items of a KV head, laid end to end and each as long as it costs, are cut
// into equal lengths, one for each workgroup that the CUs hold at once: every
// workgroup has the same to do whatever the lengths of the requests, and at most
// its first and its last item are parts that have to be joined.  Which items there
// are follows from the offsets and lengths on the device; every workgroup works it
// out by itself with two sums over the requests, so the call needs no host copy of
// the lengths, no plan made before it, and can be replayed from a graph while the
// lengths move on.
#include "lds_dma.h"
#include "qm_internal.h"

#include <algorithm>
#include <cfloat>
#include <cstdio>

namespace qm {
namespace {

typedef _Float16 half4v __attribute__((ext_vector_type(4)));
typedef short short4v __attribute__((ext_vector_type(4)));

constexpr int kBlockKeys = 64;      // keys are cut in multiples of this
// Rows of a tile: 16 where a request (or the whole batch, for the prefix) has no
// more, else 128.  The four wavefronts of a workgroup share the rows of the first
// and split its keys, and split the rows of the second and share its keys.
constexpr int kNarrow = 16, kWide = 128;
__host__ __device__ __forceinline__ int tile_rows(int rows) { return rows <= kNarrow ? kNarrow : kWide; }
// A row's maximum moves only when it grows by more than 2^8, so that the sums are
// rarely rescaled.  Weights go to fp16 as 2^7 w relative to it: the largest is
// 2^15, and they keep 11 bits down to 2^-21.  Sums of values and of (rounded)
// weights carry the same factor.
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

__device__ __forceinline__ int blocks_of(int keys) { return max((keys + kBlockKeys - 1) / kBlockKeys, 1); }

// Inclusive sum over the lanes of a wavefront.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);   // row_shr:1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);   // row_bcast:15, 31
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);
  return v;
}
// The same for 0 <= v < 2^49, in two halves.
__device__ __forceinline__ int64_t wave_scan(int64_t v) {
  const int lo = wave_scan(static_cast<int>(v & 0xFFFFFF)), hi = wave_scan(static_cast<int>(v >> 24));
  return (static_cast<int64_t>(hi) << 24) + lo;
}
__device__ __forceinline__ int64_t lane_value(int64_t v, int lane) {
  const uint32_t lo = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), lane));
  return (static_cast<int64_t>(__builtin_amdgcn_readlane(static_cast<int>(v >> 32), lane)) << 32) | lo;
}

// Costs of an item beside its keys and of a block of 64 keys, for the two kinds of
// tile, in what a block of the narrow kind costs.
struct Cost { int item, block; };
__device__ __forceinline__ Cost cost_of(const PagedAttnArgs& a, int per) {
  return per == kWide ? Cost{a.wide_item, a.wide_block} : Cost{a.narrow_item, 1};
}

// The items of one request.
struct Items {
  int rows, per, tiles;
  int64_t base;   // cost of a tile without the keys that its own rows bring
  int slope;      // those: cost of a tile's, times 256
  // Cost of the first j tiles.  Later tiles of a prompt see more keys.
  __device__ int64_t cost(int j) const { return j * base + ((static_cast<int64_t>(slope) * j * (j + 1)) >> 9); }
};

__device__ __forceinline__ Items items_of(const Requests& r, const PagedAttnArgs& a, int i) {
  Items t;
  const int tokens = max(r.off[i + 1] - r.off[i], 0), own = r.kv[i] - (a.prefix_pages << a.page_log2);
  t.rows = tokens * a.group;
  t.per = tile_rows(t.rows);
  t.tiles = (t.rows + t.per - 1) / t.per;
  const bool wide = t.per == kWide;
  const Cost c = cost_of(a, t.per);
  t.base = c.item + static_cast<int64_t>(c.block) * (wide ? max(own - tokens, 0) / kBlockKeys : blocks_of(own));
  t.slope = wide ? c.block * 256 * kWide / (kBlockKeys * a.group) : 0;
  return t;
}

// Where the items lie on the line.  Every lane of a wavefront has `per` consecutive
// requests; before: the cost of everything ahead of them.
struct Line {
  int per, prefix_rows, prefix_tile, prefix_tiles, prefix_cost;
  int64_t before, total, chunk;
};

__device__ __forceinline__ Line make_line(const Requests& r, const PagedAttnArgs& a) {
  const int lane = threadIdx.x & 63;
  Line n;
  n.per = (a.n_req + 63) / 64;
  n.prefix_rows = a.prefix_pages ? r.off[a.n_req] * a.group : 0;
  n.prefix_tile = tile_rows(n.prefix_rows);
  n.prefix_tiles = (n.prefix_rows + n.prefix_tile - 1) / n.prefix_tile;
  const Cost c = cost_of(a, n.prefix_tile);
  n.prefix_cost = c.item + c.block * blocks_of(a.prefix_pages << a.page_log2);
  int64_t cost = 0;
  for (int i = lane * n.per; i < min((lane + 1) * n.per, a.n_req); ++i) {
    const Items t = items_of(r, a, i);
    cost += t.cost(t.tiles);
  }
  const int64_t upto = wave_scan(cost), prefix = static_cast<int64_t>(n.prefix_tiles) * n.prefix_cost;
  n.before = prefix + upto - cost;
  n.total = prefix + lane_value(upto, 63);
  n.chunk = max<int64_t>(static_cast<int64_t>(static_cast<double>(n.total) * a.per_workgroup) + 1, a.min_chunk);
  return n;
}

// What the launches that join the parts have to know, at the start of the
// workspace.  Without a prefix: the item that workgroup w has begun and the next
// `parts` ones go on with.  With one, where every row has parts: for each token,
// for each tile (at the token of its first row) and for each prefix tile the
// workgroups w0 .. w0 + n - 1 that go on with it.
struct CutItem { int row, rows, parts, blind; };   // rows of the batch; the first `blind` see no key
struct TokenInfo { int j, t, kv, per; };           // token j of t new ones, kv keys, rows of its request's tiles
struct TileParts { int w0, n; };
struct Space {
  CutItem* cut;
  TokenInfo* tokens;
  TileParts* tiles;
  TileParts* prefix_tiles;
  float* records;
  int workgroups, hq;
};
// Their bytes ahead of the records, a multiple of 16.
__host__ __device__ __forceinline__ int64_t prefix_tiles_most(int64_t tokens, int64_t group) {
  return (tokens * group + kWide - 1) / kWide;
}
__host__ __device__ __forceinline__ int64_t header_bytes(int workgroups, int64_t tokens, int64_t group, bool prefix) {
  return prefix ? (tokens * static_cast<int64_t>(sizeof(TokenInfo) + sizeof(TileParts)) +
                   prefix_tiles_most(tokens, group) * static_cast<int64_t>(sizeof(TileParts)) + 15) / 16 * 16
                : workgroups * static_cast<int64_t>(sizeof(CutItem));
}

// Records, (D + 4) floats a row (D sums, maximum, sum of weights, 2 unused):
// 128 rows per workgroup and KV head for a part that goes on from the workgroup
// before, then as many for one that the next goes on with; with a prefix, in place
// of those, one per row for the first part of the own keys and one for the prefix.
template <int D>
__device__ __forceinline__ float* row_record(const Space& s, int64_t row) { return s.records + row * (D + 4); }
template <int D>
__device__ __forceinline__ float* going_on(const Space& s, const PagedAttnArgs& a, int w, int head, int row) {
  return row_record<D>(s, (static_cast<int64_t>(w) * a.hkv + head) * kWide + row);
}
template <int D>
__device__ __forceinline__ float* begun(const Space& s, const PagedAttnArgs& a, int w, int head, int row) {
  return going_on<D>(s, a, s.workgroups + w, head, row);
}
// at: (token, query head) as an element of [tokens][heads].
template <int D>
__device__ __forceinline__ float* own_row(const Space& s, const PagedAttnArgs& a, int64_t at) {
  return row_record<D>(s, static_cast<int64_t>(s.workgroups) * a.hkv * kWide + at);
}
template <int D>
__device__ __forceinline__ float* prefix_row(const Space& s, const PagedAttnArgs& a, int64_t at) {
  return own_row<D>(s, a, static_cast<int64_t>(a.tokens) * s.hq + at);
}

__device__ __forceinline__ Space space_of(const PagedAttnArgs& a) {
  Space s;
  s.cut = reinterpret_cast<CutItem*>(a.ws);
  s.tokens = reinterpret_cast<TokenInfo*>(a.ws);
  s.tiles = reinterpret_cast<TileParts*>(s.tokens + a.tokens);
  s.prefix_tiles = s.tiles + a.tokens;
  s.records = a.ws + header_bytes(a.workgroups, a.tokens, a.group, a.prefix_pages > 0) / 4;
  s.workgroups = a.workgroups;
  s.hq = a.hkv * a.group;
  return s;
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

// Sum of the weights of a pair, as rounded, on top of l.
__device__ __forceinline__ float add_pair(half8v w, int i, float l) {
  const half2v one = {static_cast<_Float16>(1.0f), static_cast<_Float16>(1.0f)};
  return __builtin_amdgcn_fdot2(half2v{w[i], w[i + 1]}, one, l, false);
}

__device__ __forceinline__ half4v read_tr(const _Float16* p) {
  typedef __attribute__((address_space(3))) short4v* lds_ptr;
  return __builtin_bit_cast(half4v, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                        (lds_ptr)(const_cast<short4v*>(reinterpret_cast<const short4v*>(p)))));
}

// K and V in LDS: rows of D halves, the 16-byte chunk c of row r at chunk
// c ^ swizzle(r).  K is read as 16 bytes of 32 rows at once: eight lanes, on rows
// one after the other, fall on different banks.  V is read transposed, four rows x
// 32 bytes by 16 lanes: they do with twice the row.
template <int D>
__device__ __forceinline__ constexpr int k_swizzle(int row) { return row & (D / 8 - 1); }
template <int D>
__device__ __forceinline__ constexpr int v_swizzle(int row) { return (2 * row) & (D / 8 - 1); }
template <int D>
__device__ __forceinline__ int v_at(int row, int dim) {
  return row * D + (((dim >> 3) ^ v_swizzle<D>(row)) << 3) + (dim & 7);
}

template <int D>
struct NarrowLds {
  union {
    _Float16 v[4][32 * D];          // a block of V per wavefront
    float acc[4][16][D + 4];        // the wavefronts' parts
  };
  float m[4][16], l[4][16];
};
template <int D>
struct WideLds {
  _Float16 k[2][kBlockKeys * D], v[2][kBlockKeys * D];   // two blocks: one read, one on its way
  int bad;
};
template <int D>
union TileLds {
  NarrowLds<D> n;
  WideLds<D> w;
};

// One tile of 16 rows against the keys [k.lo, k.hi) of one KV head: the four
// wavefronts take blocks of 32 keys in turn.
//   S^T = K Q^T   16 keys x 16 rows, K fragments straight from their pages,
//   O^T += V^T W^T, V^T read transposed out of LDS; its k slots are relabelled to
//   the keys that a lane holds weights of, so the weights never leave their lane.
// limit: keys visible to this lane's row (lane & 15), 0 for rows that do not
// exist.  Leaves the joined sums in s.acc[0], maxima in s.m[0], sums in s.l[0].
template <int D>
__device__ __forceinline__ void narrow_part(const PagedAttnArgs& a, NarrowLds<D>& s, const uint16_t* q_row, int limit,
                                            int head, const Keys& k) {
  constexpr int KS = D / 32, DB = D / 16, VL = D / 16;   // k steps of S, dimension tiles, V loads per lane
  const int thread = fresh_thread(), lane = thread & 63, col = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(thread >> 6);
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
  // Row 0 of the page of 16 keys (keys past the end: the last ones), in rows of the pool.
  auto row_of = [&](int key) __attribute__((always_inline)) {
    const int t = min(key, (hi - 1) & ~15);
    int id = k.pages[t >> a.page_log2];
    if (static_cast<uint32_t>(id) >= static_cast<uint32_t>(a.n_pages)) {
      bad = true;
      id = 0;
    }
    return ((static_cast<int64_t>(id) * a.hkv + head) << a.page_log2) + (t & (page_rows - 1));
  };
  struct Blk { half8v k[2][KS], v[VL]; };
  auto load = [&](int kb) __attribute__((always_inline)) {
    Blk b;
    int64_t row[2];
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
  float4v acc[DB];
#pragma unroll
  for (int b = 0; b < DB; ++b) acc[b] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
  float m = -FLT_MAX, l = 0.0f;

  _Float16* const vl = s.v[wave];
  const int first = k.lo + 32 * wave;
  Blk cur;
  if (first < hi) cur = load(first);
  for (int kb = first; kb < hi; kb += 128) {
    const Blk x = cur;
    if (kb + 128 < hi) cur = load(kb + 128);
#pragma unroll
    for (int j = 0; j < VL; ++j) {
      const int piece = lane + 64 * j;
      *reinterpret_cast<half8v*>(&vl[v_at<D>(piece / (D / 8), piece % (D / 8) * 8)]) = x.v[j];
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
      const half4v lo = read_tr(&vl[v_at<D>(4 * g + (col >> 2), 16 * b + 4 * (col & 3))]);
      const half4v up = read_tr(&vl[v_at<D>(16 + 4 * g + (col >> 2), 16 * b + 4 * (col & 3))]);
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
                const float x = static_cast<float>(vl[v_at<D>(key, 16 * b + 4 * g + r)]);
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
  __syncthreads();                                          // V has been read by every wavefront
#pragma unroll
  for (int b = 0; b < DB; ++b) *reinterpret_cast<float4v*>(&s.acc[wave][col][16 * b + 4 * g]) = acc[b];
  if (g == 0) {
    s.m[wave][col] = m;
    s.l[wave][col] = l;
  }
  __syncthreads();
}

// One tile of 128 rows against the keys [k.lo, hi) of one KV head: wavefront w has
// rows 32 w .. 32 w + 31, and all share the blocks of 64 keys that come into LDS by
// DMA, each wavefront copying 16 keys of K and V, while the block before is worked on.
//   S^T = K Q^T   32 keys x 32 rows at a time, K fragments out of LDS,
//   O^T += V^T W^T as in narrow_part.
// limit: keys visible to this lane's row (lane & 31).  acc[b][r]: dimension
// 32 b + 8 (r / 4) + 4 (lane / 32) + r % 4 of the row; m, l: its maximum and this
// lane's share of the sum of weights.
template <int D>
__device__ __forceinline__ void wide_part(const PagedAttnArgs& a, WideLds<D>& s, const uint16_t* q_row, int limit,
                                          int head, const Keys& k, float16v (&acc)[D / 32], float& m, float& l) {
  constexpr int KS = D / 16, DB = D / 32, C = D / 8, PIECES = D / 32;   // PIECES: KiB of 16 keys
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
  const int all = __builtin_amdgcn_readfirstlane(min(least, hi));   // keys below are visible to every row
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

  // This wavefront's 16 keys of the block at kb (keys past the end: the last ones).
  const int last = (hi - 1) & ~15;
  bool bad = false;
  auto page_of = [&](int kb) __attribute__((always_inline)) {
    return __builtin_amdgcn_readfirstlane(k.pages[min(kb + 16 * wave, last) >> a.page_log2]);
  };
  const int lrow = lane / C, chunk = lane % C;            // of a piece: 64 / C rows of C chunks
  auto copy = [&](int buf, int kb, int id) __attribute__((always_inline)) {
    if (static_cast<uint32_t>(id) >= static_cast<uint32_t>(a.n_pages)) {
      bad = true;
      id = 0;
    }
    const int t = min(kb + 16 * wave, last) & (page_rows - 1);
    const int64_t row = ((static_cast<int64_t>(id) * a.hkv + head) << a.page_log2) + t;
    const uint16_t* kr = a.k_pages + row * D;
    const uint16_t* vr = a.v_pages + row * D;
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
      const int r = j * (64 / C) + lrow;
      qg::lds_dma16(kr + r * D + ((chunk ^ k_swizzle<D>(r)) << 3), &s.k[buf][16 * wave * D + 512 * j]);
      qg::lds_dma16(vr + r * D + ((chunk ^ v_swizzle<D>(r)) << 3), &s.v[buf][16 * wave * D + 512 * j]);
    }
  };
  auto compute = [&](int buf, int kb) __attribute__((always_inline)) {
    const _Float16* const kl = s.k[buf];
    const _Float16* const vl = s.v[buf];
    float16v st[2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) st[t][r] = 0.0f;
#pragma unroll
    for (int c = 0; c < KS; ++c)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const half8v f =
            *reinterpret_cast<const half8v*>(&kl[(32 * t + col) * D + (((2 * c + lh) ^ k_swizzle<D>(col)) << 3)]);
        st[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f, qf[c], st[t], 0, 0, 0);
      }
    // Lane: row col, keys kb + 32 t + 8 (r / 4) + 4 lh + r % 4.
    const bool masked = kb + kBlockKeys > all;
    if (masked) {
      const int seen = min(limit, hi) - kb - 4 * lh;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) st[t][r] = 32 * t + 8 * (r >> 2) + (r & 3) < seen ? st[t][r] : -INFINITY;
    }
    float bm = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
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
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        half8v& x = w[2 * t + (r >> 3)];
        x[r & 7] = static_cast<_Float16>(__builtin_amdgcn_exp2f(fmaf(st[t][r], a.scale_log2, shift)));
        x[(r & 7) + 1] = static_cast<_Float16>(__builtin_amdgcn_exp2f(fmaf(st[t][r + 1], a.scale_log2, shift)));
        l = add_pair(x, r & 7, l);
      }
    // k slot (lh, j) of step kk: key 16 kk + 8 (j / 4) + 4 lh + j % 4.
    auto value = [&](int kk, int b) __attribute__((always_inline)) {
      const int row = 16 * kk + 4 * lh + ((lane & 15) >> 2), dim = 32 * b + (col & 16) + 4 * (lane & 3);
      const half4v lo = read_tr(&vl[v_at<D>(row, dim)]);
      const half4v up = read_tr(&vl[v_at<D>(row + 8, dim)]);
      return half8v{lo[0], lo[1], lo[2], lo[3], up[0], up[1], up[2], up[3]};
    };
    if (!masked) {
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
#pragma unroll
        for (int b = 0; b < DB; ++b)
          acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(value(kk, b), w[kk], acc[b], 0, 0, 0);
    } else {                                                // as in narrow_part
      bool odd = false;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
#pragma unroll
        for (int b = 0; b < DB; ++b)
          acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(finite_part(value(kk, b), odd), w[kk], acc[b], 0, 0, 0);
      if (__builtin_amdgcn_ballot_w64(odd) != 0) {
        for (int key = 0; key < kBlockKeys; ++key) {
          if (kb + key < min(limit, hi)) {
#pragma unroll
            for (int b = 0; b < DB; ++b)
#pragma unroll
              for (int r = 0; r < 16; ++r) {
                const float x = static_cast<float>(vl[v_at<D>(key, 32 * b + 8 * (r >> 2) + 4 * lh + (r & 3))]);
                acc[b][r] += __builtin_fabsf(x) < INFINITY ? 0.0f : x;
              }
          }
        }
      }
    }
  };
  if (k.lo < hi) {
    copy(0, k.lo, page_of(k.lo));
    int id = page_of(k.lo + kBlockKeys);
    int buf = 0;
    for (int kb = k.lo; kb < hi; kb += kBlockKeys, buf ^= 1) {
      // This wavefront's copies have landed and its reads of the other block are
      // done; after the barrier so are everybody's.
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(0xC07F);                   // lgkmcnt(0)
      qg::vm_wait<0>();
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      if (kb + kBlockKeys < hi) {
        copy(buf ^ 1, kb + kBlockKeys, id);
        id = page_of(kb + 2 * kBlockKeys);
      }
      if (kb < most) compute(buf, kb);
    }
  }
  __syncthreads();
  if (bad) s.bad = 1;
  __syncthreads();
  const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
  l = __uint_as_float(both[0]) + __uint_as_float(both[1]);
  if (s.bad) l = __builtin_nanf("");
}

// Workgroups that a CU holds at once, by registers and LDS.
template <int D>
constexpr int kResident = D == 64 ? 3 : 2;

template <int D>
__global__ __launch_bounds__(256, kResident<D>) void paged_attn_kernel(PagedAttnArgs a) {
  __shared__ Requests req;
  __shared__ __attribute__((aligned(1024))) TileLds<D> s;
  load_requests(req, a);
  const Line line = make_line(req, a);
  const Space space = space_of(a);
  const int head = static_cast<int>(blockIdx.x % a.hkv), wg = static_cast<int>(blockIdx.x / a.hkv);
  const int64_t x0 = wg * line.chunk, x1 = min(x0 + line.chunk, line.total);   // this workgroup's length of the line
  bool begins = false;                                      // an item that the next workgroup goes on with
  if (x0 >= line.total) {
    if (!a.prefix_pages && head == 0 && threadIdx.x == 0) space.cut[wg].parts = 0;
    return;
  }
  const int prefix_len = a.prefix_pages << a.page_log2;
  const int64_t hq = space.hq;
  // The item at x0: a prefix tile, or a request and a tile of it; it starts at `start`.
  const int64_t prefix_end = static_cast<int64_t>(line.prefix_tiles) * line.prefix_cost;
  int i = -1, tile = 0;                                     // request (-1: the prefix), tile
  int64_t start = 0, req_start = prefix_end;
  Items it{line.prefix_rows, line.prefix_tile, line.prefix_tiles, line.prefix_cost, 0};
  if (x0 < prefix_end) {
    tile = static_cast<int>(static_cast<double>(x0) / line.prefix_cost);
    tile -= it.cost(tile) > x0;
    tile += it.cost(tile + 1) <= x0;
    start = it.cost(tile);
  } else {
    const uint64_t at = __builtin_amdgcn_ballot_w64(line.before <= x0);
    const int owner = 63 - __builtin_clzll(at);
    req_start = lane_value(line.before, owner);
    i = owner * line.per;
    it = items_of(req, a, i);
    while (req_start + it.cost(it.tiles) <= x0 && i + 1 < a.n_req) {
      req_start += it.cost(it.tiles);
      it = items_of(req, a, ++i);
    }
    int hi = it.tiles - 1;
    while (tile < hi) {
      const int mid = (tile + hi + 1) >> 1;
      if (req_start + it.cost(mid) <= x0) tile = mid; else hi = mid - 1;
    }
    start = req_start + it.cost(tile);
  }
  for (;;) {
    const bool shared = i < 0;
    const int64_t end = (shared ? 0 : req_start) + it.cost(tile + 1);
    const int row0 = tile * it.per, rows = it.rows, per = it.per;
    const int last = min(row0 + per, rows) - 1, t = shared ? 0 : rows / a.group;
    const int seen = shared ? prefix_len : min(req.kv[i], req.kv[i] - t + last / a.group + 1);   // keys of the last row
    const int first_key = shared ? 0 : prefix_len;
    const int blocks = blocks_of(seen - first_key);
    // Blocks of the item ahead of a place on the line; what would be a very short
    // part goes to its neighbour.
    const Cost cost = cost_of(a, per);
    const int min_part = per == kWide ? a.wide_part : a.narrow_part;
    auto ahead = [&](int64_t x) __attribute__((always_inline)) {
      const int64_t keys = max<int64_t>(min<int64_t>(x - start - cost.item, INT32_MAX), -1);
      const int b = static_cast<int>(keys) / cost.block;
      return x >= end ? blocks : keys < 0 ? 0 : b > blocks - min_part ? blocks : b < min_part ? 0 : b;
    };
    const int from = ahead(x0), to = ahead(x1);
    if (from < to) {
      const int thread = fresh_thread(), lane = thread & 63;
      if (from == 0 && head == 0) {
        // Workgroups wg + 1 .. wg + n go on with the item: those whose length begins
        // at the block blocks - min_part or before.
        const int64_t left =
            min(start + cost.item + static_cast<int64_t>(blocks - min_part + 1) * cost.block, end) - 1 - (wg + 1) * line.chunk;
        const int n = to == blocks ? 0 : static_cast<int>(left / line.chunk) + 1;
        if (!a.prefix_pages) {
          // The rows of the batch, those of them that see no key.
          if (n && thread == 0)
            space.cut[wg] = CutItem{req.off[i] * a.group + row0, last + 1 - row0, n,
                                    min(max((t - req.kv[i]) * a.group - row0, 0), kWide)};
          begins = begins || n;
        } else if (shared) {
          if (thread == 0) space.prefix_tiles[tile] = TileParts{wg + 1, n};
        } else {
          if (thread == 0) space.tiles[req.off[i] + row0 / a.group] = TileParts{wg + 1, n};
          // The tokens whose first row is in this tile.
          for (int j = (row0 + a.group - 1) / a.group + thread; j * a.group <= last; j += 256)
            space.tokens[req.off[i] + j] = TokenInfo{j, t, req.kv[i], per};
        }
      }
      const bool whole = !a.prefix_pages && from == 0 && to == blocks;
      Keys k;
      k.pages = shared ? a.prefix : a.tables + static_cast<int64_t>(i) * a.max_pages;
      k.lo = first_key + from * kBlockKeys;
      k.hi = min(seen, first_key + to * kBlockKeys);
      // This lane's row of the tile.
      const bool narrow = per == kNarrow;
      const int col = narrow ? lane & 15 : (thread >> 6) * 32 + (lane & 31);
      const int row = min(row0 + col, last);
      int token = row / a.group;
      const int gq = row % a.group;
      const int r = shared ? request_of(req, a.n_req, token) : i;
      if (!shared) token += req.off[i];
      const int sees = max(min(req.kv[r], req.kv[r] - max(req.off[r + 1] - token, 0) + 1), 0);
      const int limit = row0 + col > last ? 0 : shared ? min(sees, prefix_len) : sees;
      const int64_t at = token * hq + head * a.group + gq;  // of q and out
      if (!narrow) {
        float16v acc[D / 32];
        float m, l;
        wide_part<D>(a, s.w, a.q + at * D, limit, head, k, acc, m, l);
        const int lh = lane >> 5;
        if (row0 + col <= last) {
          if (whole) {
            const float inv = sees ? 1.0f / l : 0.0f;
            uint16_t* o = a.out + at * D;
#pragma unroll
            for (int b = 0; b < D / 32; ++b)
#pragma unroll
              for (int q = 0; q < 16; q += 4) {
                half4v h;
#pragma unroll
                for (int c = 0; c < 4; ++c) h[c] = static_cast<_Float16>(sees ? acc[b][q + c] * inv : 0.0f);
                *reinterpret_cast<half4v*>(o + 32 * b + 2 * q + 4 * lh) = h;
              }
          } else {
            float* rec = from ? going_on<D>(space, a, wg, head, col)
                         : !a.prefix_pages ? begun<D>(space, a, wg, head, col)
                         : shared ? prefix_row<D>(space, a, at) : own_row<D>(space, a, at);
#pragma unroll
            for (int b = 0; b < D / 32; ++b)
#pragma unroll
              for (int q = 0; q < 16; q += 4)
                *reinterpret_cast<float4v*>(rec + 32 * b + 2 * q + 4 * lh) =
                    float4v{acc[b][q], acc[b][q + 1], acc[b][q + 2], acc[b][q + 3]};
            if (lh == 0) {
              rec[D] = m;
              rec[D + 1] = l;
            }
          }
        }
      } else {
        narrow_part<D>(a, s.n, a.q + at * D, limit, head, k);
        // The four wavefronts' sums, joined; thread: row, 4 dimensions.
        for (int e = thread; e < 16 * (D / 4); e += 256) {
          const int x = e / (D / 4), d4 = e % (D / 4);
          if (row0 + x > last) continue;
          const float mx = fmaxf(fmaxf(s.n.m[0][x], s.n.m[1][x]), fmaxf(s.n.m[2][x], s.n.m[3][x]));
          float4v o{0.0f, 0.0f, 0.0f, 0.0f};
          float l = 0.0f;
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const float f = __builtin_amdgcn_exp2f(s.n.m[w][x] - mx);
            l = fmaf(s.n.l[w][x], f, l);
            const float4v v = *reinterpret_cast<const float4v*>(&s.n.acc[w][x][4 * d4]);
#pragma unroll
            for (int c = 0; c < 4; ++c) o[c] = fmaf(v[c], f, o[c]);
          }
          const int tk = (row0 + x) / a.group;              // of the request or the batch
          const int64_t xat = ((shared ? 0 : req.off[i]) + tk) * hq + head * a.group + (row0 + x) % a.group;
          if (whole) {
            const bool none = req.kv[i] - t + tk + 1 <= 0;
            half4v h;
#pragma unroll
            for (int c = 0; c < 4; ++c) h[c] = static_cast<_Float16>(none ? 0.0f : o[c] / l);
            *reinterpret_cast<half4v*>(a.out + xat * D + 4 * d4) = h;
          } else {
            float* rec = from ? going_on<D>(space, a, wg, head, x)
                         : !a.prefix_pages ? begun<D>(space, a, wg, head, x)
                         : shared ? prefix_row<D>(space, a, xat) : own_row<D>(space, a, xat);
            *reinterpret_cast<float4v*>(rec + 4 * d4) = o;
            if (d4 == 0) {
              rec[D] = mx;
              rec[D + 1] = l;
            }
          }
        }
      }
      __syncthreads();                                      // the tile's LDS is free
    }
    if (end >= x1) break;
    start = end;
    if (++tile == it.tiles) {
      req_start = end;
      tile = 0;
      do {                                                  // (there is one: end < x1 <= total)
        it = items_of(req, a, ++i);
      } while (it.tiles == 0 && i + 1 < a.n_req);
    }
  }
  if (!a.prefix_pages && !begins && head == 0 && threadIdx.x == 0) space.cut[wg].parts = 0;
}

// Parts s0, s0 + step, ... of a row, each with its weight relative to the largest
// maximum so far; rec(s): the record of part s, d4: this thread's four dimensions.
struct Joined { float4v o; float m, l; };
template <int D, class Rec>
__device__ __forceinline__ Joined join_parts(int s0, int step, int parts, int d4, Rec rec) {
  constexpr int BATCH = 8;                                  // loads in flight
  Joined r{float4v{0.0f, 0.0f, 0.0f, 0.0f}, -FLT_MAX, 0.0f};
  for (; s0 < parts; s0 += BATCH * step) {
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

// Without a prefix: the items that are cut, a workgroup for 16 rows of each.  A row
// has D / 4 threads, four dimensions each; with few rows several groups of threads
// share its parts.
template <int D>
__global__ __launch_bounds__(256) void paged_attn_join_kernel(PagedAttnArgs a) {
  constexpr int C4 = D / 4;
  const Space space = space_of(a);
  const int head = static_cast<int>(blockIdx.x % a.hkv), rest = static_cast<int>(blockIdx.x / a.hkv);
  const int w = rest % a.workgroups, row0 = rest / a.workgroups * 16;
  const CutItem it = space.cut[w];
  const int rows = min(it.rows - row0, 16);
  if (it.parts == 0 || rows <= 0) return;
  int groups = 1;
  while (2 * groups * rows * C4 <= 256 && 2 * groups <= it.parts) groups *= 2;
  const int width = 256 / groups, grp = threadIdx.x / width;
  for (int e = threadIdx.x % width; e < rows * C4 || groups > 1; e += width) {   // (once where there are several groups)
    const int row = row0 + min(e / C4, rows - 1), d4 = e % C4;
    auto rec = [&](int x) __attribute__((always_inline)) {
      return x == 0 ? begun<D>(space, a, w, head, row) : going_on<D>(space, a, min(w + x, a.workgroups - 1), head, row);
    };
    Joined r = join_parts<D>(grp, groups, it.parts + 1, d4, rec);
    if (groups > 1) r = join_groups(r, groups, width);
    if (grp == 0 && e < rows * C4) write_joined<D>(a, element_of(a, it.row + row, head), d4, r, row < it.blind);
    if (groups > 1) break;
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
  const int token = min(row, rows - 1) / a.group, gq = min(row, rows - 1) - token * a.group;
  const TokenInfo tp = space.tokens[token];
  // (The test holds whatever lies there for a token of no request, where offsets do not rise.)
  const bool there = row < rows && (tp.per == kNarrow || tp.per == kWide) && tp.j >= 0 && tp.j <= token;
  const int per = there ? tp.per : kNarrow, own_row_at = there ? tp.j * a.group + gq : 0;   // row of the request
  const int tile = own_row_at / per, prefix_tile = tile_rows(rows), prow = token * a.group + gq;
  const TileParts own = space.tiles[there ? token - tp.j + tile * per / a.group : 0];
  const TileParts pre = space.prefix_tiles[prow / prefix_tile];
  const int64_t at = element_of(a, prow, head);
  const int own_at = min(max(pre.n, 0), a.workgroups) + 1;  // parts of the prefix
  const int parts = own_at + 1 + min(max(own.n, 0), a.workgroups);
  auto rec = [&](int x) __attribute__((always_inline)) {
    auto held = [&](int w) __attribute__((always_inline)) { return min(max(w, 0), a.workgroups - 1); };
    if (x == 0) return prefix_row<D>(space, a, at);
    if (x < own_at) return going_on<D>(space, a, held(pre.w0 + x - 1), head, prow % prefix_tile);
    if (x == own_at) return own_row<D>(space, a, at);
    return going_on<D>(space, a, held(own.w0 + x - own_at - 1), head, own_row_at % per);
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
  const int64_t slots = static_cast<int64_t>(workgroups) * hkv * kWide;
  const int64_t records = prefix ? slots + 2 * tokens * hq : 2 * slots;
  return static_cast<size_t>(header_bytes(workgroups, tokens, hq / hkv, prefix)) +
         static_cast<size_t>(records) * (d + 4) * sizeof(float);
}

namespace {

template <int D>
hipError_t launch_paged(const PagedAttnArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(paged_attn_kernel<D>, dim3(static_cast<unsigned>(a.workgroups * a.hkv)), dim3(256), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (!a.prefix_pages) {
    hipLaunchKernelGGL(paged_attn_join_kernel<D>, dim3(static_cast<unsigned>(a.workgroups * a.hkv * (kWide / 16))), dim3(256),
                       0, st, a);
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
  a.workgroups = workgroups_of(a.hkv, d, cu_count);
  a.per_workgroup = 1.0 / a.workgroups;
  a.narrow_item = 1;
  a.wide_item = 4;
  a.wide_block = 2;
  a.min_chunk = 4;
  a.narrow_part = 2;
  a.wide_part = 4;
  if (const char* e = tuning_override("QM_PAGED_PLAN"))
    std::sscanf(e, "%d,%d,%d,%d,%d,%d", &a.narrow_item, &a.wide_item, &a.wide_block, &a.min_chunk, &a.narrow_part, &a.wide_part);
  return d == 64 ? launch_paged<64>(a, st) : launch_paged<128>(a, st);
}

}  // namespace qm
