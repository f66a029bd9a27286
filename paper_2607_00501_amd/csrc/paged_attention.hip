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
// pairs, token-major.  Work units, one workgroup each per KV head:
//   prefix part:  a tile of rows of any requests  x  a range of prefix keys,
//   own part:     a tile of one request's rows    x  a range of its own keys.
// Which units there are follows from the offsets and lengths on the device;
// every workgroup works it out by itself with two sums over the requests, so
// the call needs no host copy of the lengths, no plan made before it, and can be
// replayed from a graph while the lengths move on.
#include "lds_dma.h"
#include "qm_internal.h"

#include <algorithm>
#include <cfloat>

namespace qm {
namespace {

typedef _Float16 half4v __attribute__((ext_vector_type(4)));
typedef short short4v __attribute__((ext_vector_type(4)));

constexpr int kBlockKeys = 64;      // keys are split in multiples of this
constexpr int kMinBlocks = 2;       // fewest blocks of a split
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

struct Share {
  int rows, tiles, blocks, splits;
  int granules;   // of 16 rows, that a tile leaves in the workspace; 0: its only part writes the output itself
};

__device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }

// c: blocks per split (0: not known yet).
__device__ __forceinline__ Share share_of(const Requests& r, const PagedAttnArgs& a, int i, int c) {
  const int own = r.kv[i] - (a.prefix_pages << a.page_log2);
  Share s;
  s.rows = max(r.off[i + 1] - r.off[i], 0) * a.group;
  const int per = tile_rows(s.rows);
  s.tiles = (s.rows + per - 1) / per;
  s.blocks = own > 0 ? (own + kBlockKeys - 1) / kBlockKeys : 1;
  s.splits = c ? ceil_div(s.blocks, c) : 1;
  s.granules = s.splits > 1 || a.prefix_pages ? per / 16 : 0;
  return s;
}

// Every lane of a wavefront takes `per` consecutive requests; units_before and
// granules_before are the sums over the earlier lanes' requests.
struct Units {
  int c, per, prefix_tile, prefix_tiles, prefix_splits, units_before, granules_before, total;
};

template <class T>
__device__ __forceinline__ T wave_scan(T v) {   // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const T o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}

__device__ __forceinline__ Units make_units(const Requests& r, const PagedAttnArgs& a) {
  const int lane = threadIdx.x & 63;
  Units u;
  u.per = (a.n_req + 63) / 64;
  const int lo = lane * u.per, hi = min(lo + u.per, a.n_req);
  int64_t work = 0;
  for (int i = lo; i < hi; ++i) {
    const Share s = share_of(r, a, i, 0);
    work += static_cast<int64_t>(s.tiles) * s.blocks;
  }
  work = __shfl(wave_scan(work), 63);
  const int prefix_blocks = ((a.prefix_pages << a.page_log2) + kBlockKeys - 1) / kBlockKeys;
  const int rows = r.off[a.n_req] * a.group;
  u.prefix_tile = tile_rows(rows);
  u.prefix_tiles = a.prefix_pages ? ceil_div(rows, u.prefix_tile) : 0;
  work += static_cast<int64_t>(u.prefix_tiles) * prefix_blocks;
  // Splits of c blocks: sum tiles ceil(blocks / c) <= tiles + target.
  u.c = static_cast<int>(max<int64_t>(kMinBlocks, (work + a.target - 1) / a.target));
  u.prefix_splits = a.prefix_pages ? ceil_div(prefix_blocks, u.c) : 0;
  int units = 0, granules = 0;
  for (int i = lo; i < hi; ++i) {
    const Share s = share_of(r, a, i, u.c);
    units += s.tiles * s.splits;
    granules += s.tiles * s.splits * s.granules;
  }
  const int units_to = wave_scan(units), granules_to = wave_scan(granules);
  const int p = u.prefix_tiles * u.prefix_splits;
  u.units_before = p + units_to - units;
  u.granules_before = p * (u.prefix_tile / 16) + granules_to - granules;
  u.total = p + __shfl(units_to, 63);
  return u;
}

// ---------------------------------------------------- one part of one tile

// A range of keys behind a page table.
struct Keys {
  const int32_t* pages;   // page ids of positions 0, page, 2 page, ...
  int lo, hi;             // this part's keys: positions [lo, hi); lo is a multiple of 16
};

// Record of a row in a part: D sums, maximum, sum of weights, 2 pad floats.
__device__ __forceinline__ float* record(const PagedAttnArgs& a, int d, int granule, int head, int granules_per_head,
                                         int row) {
  return a.ws + ((static_cast<int64_t>(granule) * a.hkv + static_cast<int64_t>(head) * granules_per_head) * 16 + row) *
                    (d + 4);
}

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
  const int lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
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
  const int lane = threadIdx.x & 63, col = lane & 31, lh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
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
  if (threadIdx.x == 0) s.bad = 0;
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

template <int D>
__global__ __launch_bounds__(256, 2) void paged_attn_kernel(PagedAttnArgs a) {
  __shared__ Requests req;
  __shared__ __attribute__((aligned(1024))) TileLds<D> s;
  load_requests(req, a);
  const Units u = make_units(req, a);
  const int head = static_cast<int>(blockIdx.x % a.hkv);
  const int unit = static_cast<int>(blockIdx.x / a.hkv);
  if (unit >= u.total) return;
  const int prefix_len = a.prefix_pages << a.page_log2;
  const int lane = threadIdx.x & 63;
  int row0, rows, per, granule, i = 0;                      // tile: first row, counted over the batch or the request
  Keys k;
  bool direct = false;
  const bool shared = unit < u.prefix_tiles * u.prefix_splits;
  // Parts of the same keys follow each other: they share what the L2 holds.
  if (shared) {
    per = u.prefix_tile;
    row0 = unit % u.prefix_tiles * per;
    rows = req.off[a.n_req] * a.group;
    const int part = unit / u.prefix_tiles;
    granule = unit * (per / 16);
    k = Keys{a.prefix, part * u.c * kBlockKeys, min(prefix_len, (part + 1) * u.c * kBlockKeys)};
  } else {
    // The lane whose requests hold the unit, then the request.
    const uint64_t before = __builtin_amdgcn_ballot_w64(u.units_before <= unit);
    const int owner = 63 - __builtin_clzll(before);
    int at = __builtin_amdgcn_readlane(u.units_before, owner);
    granule = __builtin_amdgcn_readlane(u.granules_before, owner);
    i = owner * u.per;
    const int end = min(i + u.per, a.n_req);
    Share sh = share_of(req, a, i, u.c);
    while (at + sh.tiles * sh.splits <= unit && i + 1 < end) {
      at += sh.tiles * sh.splits;
      granule += sh.tiles * sh.splits * sh.granules;
      sh = share_of(req, a, ++i, u.c);
    }
    rows = sh.rows;
    per = tile_rows(rows);
    row0 = (unit - at) % sh.tiles * per;
    const int part = (unit - at) / sh.tiles;
    granule += (unit - at) * sh.granules;
    direct = sh.granules == 0;
    // Splits past the keys that the tile's last row sees have nothing to do
    // (the first is always there, so that every row is written).
    const int last = min(row0 + per, rows) - 1;
    const int seen = req.kv[i] - rows / a.group + last / a.group + 1;
    const int64_t lo = prefix_len + static_cast<int64_t>(part) * u.c * kBlockKeys;
    if (part > 0 && lo >= seen) return;
    k = Keys{a.tables + static_cast<int64_t>(i) * a.max_pages, static_cast<int>(lo),
             static_cast<int>(min<int64_t>(min(req.kv[i], seen), lo + static_cast<int64_t>(u.c) * kBlockKeys))};
  }
  if (!direct && granule + per / 16 > a.granules) return;   // (the workspace covers every batch of these limits)
  // This lane's row of the tile.
  const bool narrow = per == kNarrow;
  const int col = narrow ? lane & 15 : static_cast<int>(threadIdx.x >> 6) * 32 + (lane & 31);
  const int row = min(row0 + col, rows - 1);
  int token = row / a.group;
  const int gq = row % a.group;
  if (shared) i = request_of(req, a.n_req, token);
  else token += req.off[i];
  const int j = token - req.off[i], t = max(req.off[i + 1] - req.off[i], 0);
  const int sees = max(min(req.kv[i] - t + j + 1, req.kv[i]), 0);
  const int limit = row0 + col >= rows ? 0 : shared ? min(sees, prefix_len) : sees;
  const int64_t hq = static_cast<int64_t>(a.hkv) * a.group;
  const int64_t at_row = static_cast<int64_t>(token) * hq + head * a.group + gq;   // of q and out
  if (!narrow) {
    float16v acc[D / 32];
    float m, l;
    wide_part<D>(a, s.w, a.q + at_row * D, limit, head, k, acc, m, l);
    if (row0 + col >= rows) return;
    const int lh = lane >> 5;
    if (direct) {
      const float inv = sees ? 1.0f / l : 0.0f;
      uint16_t* o = a.out + at_row * D;
#pragma unroll
      for (int b = 0; b < D / 32; ++b)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          half4v h;
#pragma unroll
          for (int c = 0; c < 4; ++c) h[c] = static_cast<_Float16>(sees ? acc[b][r + c] * inv : 0.0f);
          *reinterpret_cast<half4v*>(o + 32 * b + 2 * r + 4 * lh) = h;
        }
    } else {
      float* rec = record(a, D, granule, head, kWide / 16, col);
#pragma unroll
      for (int b = 0; b < D / 32; ++b)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
          *reinterpret_cast<float4v*>(rec + 32 * b + 2 * r + 4 * lh) =
              float4v{acc[b][r], acc[b][r + 1], acc[b][r + 2], acc[b][r + 3]};
      if (lh == 0) {
        rec[D] = m;
        rec[D + 1] = l;
      }
    }
    return;
  }
  narrow_part<D>(a, s.n, a.q + at_row * D, limit, head, k);
  // The four wavefronts' sums, joined; thread: row, 4 dimensions.
  for (int e = threadIdx.x; e < 16 * (D / 4); e += 256) {
    const int r = e / (D / 4), d4 = e % (D / 4);
    if (row0 + r >= rows) continue;
    const float mx = fmaxf(fmaxf(s.n.m[0][r], s.n.m[1][r]), fmaxf(s.n.m[2][r], s.n.m[3][r]));
    float4v o{0.0f, 0.0f, 0.0f, 0.0f};
    float l = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = __builtin_amdgcn_exp2f(s.n.m[w][r] - mx);
      l = fmaf(s.n.l[w][r], f, l);
      const float4v v = *reinterpret_cast<const float4v*>(&s.n.acc[w][r][4 * d4]);
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c] = fmaf(v[c], f, o[c]);
    }
    if (direct) {
      const int rr = row0 + r, tk = req.off[i] + rr / a.group;
      const bool none = req.kv[i] - t + rr / a.group + 1 <= 0;
      half4v h;
#pragma unroll
      for (int c = 0; c < 4; ++c) h[c] = static_cast<_Float16>(none ? 0.0f : o[c] / l);
      *reinterpret_cast<half4v*>(a.out + (static_cast<int64_t>(tk) * hq + head * a.group + rr % a.group) * D + 4 * d4) = h;
    } else {
      float* rec = record(a, D, granule, head, kNarrow / 16, r);
      *reinterpret_cast<float4v*>(rec + 4 * d4) = o;
      if (d4 == 0) {
        rec[D] = mx;
        rec[D + 1] = l;
      }
    }
  }
}

// The parts of the rows of one token and KV head, joined: prefix parts first, then
// the request's own, each with its weight relative to the largest maximum so far.
// A workgroup takes `steps` tokens in turn, since each works out the units first.
template <int D>
__global__ __launch_bounds__(256) void paged_attn_join_kernel(PagedAttnArgs a, int steps) {
  __shared__ Requests req;
  load_requests(req, a);
  const int head = static_cast<int>(blockIdx.x % a.hkv);
  const Units u = make_units(req, a);
  const int prefix_len = a.prefix_pages << a.page_log2;
  const int64_t hq = static_cast<int64_t>(a.hkv) * a.group;
  const int first = static_cast<int>(blockIdx.x / a.hkv) * steps;
  const int end = min(first + steps, req.off[a.n_req]);
  for (int token = first; token < end; ++token) {
    const int i = __builtin_amdgcn_readfirstlane(request_of(req, a.n_req, token));
    const Share sh = share_of(req, a, i, u.c);
    const int j = token - req.off[i], t = max(req.off[i + 1] - req.off[i], 0);
    if (sh.granules == 0 || j < 0 || j >= t) continue;      // written by its only part (or offsets that do not rise)
    const int owner = i / u.per;
    int base = __builtin_amdgcn_readlane(u.granules_before, owner);
    for (int x = owner * u.per; x < i; ++x) {
      const Share before = share_of(req, a, x, u.c);
      base += before.tiles * before.splits * before.granules;
    }
    const bool none = req.kv[i] - t + j + 1 <= 0;
    const int per = tile_rows(sh.rows);
    for (int e = threadIdx.x; e < a.group * (D / 4); e += 256) {
      const int gq = e / (D / 4), d4 = e % (D / 4);
      const int row = j * a.group + gq, tile = row / per;   // of the request
      const int last = min((tile + 1) * per, sh.rows) - 1;
      const int seen = req.kv[i] - t + last / a.group + 1 - prefix_len;
      const int blocks = seen > 0 ? (seen + kBlockKeys - 1) / kBlockKeys : 1;
      const int own = ceil_div(blocks, u.c), parts = u.prefix_splits + own;
      const int prow = token * a.group + gq;                // of the batch
      auto rec = [&](int s) __attribute__((always_inline)) {
        const bool pre = s < u.prefix_splits;
        const int g = pre ? u.prefix_tile / 16 : sh.granules;
        const int granule = pre ? (s * u.prefix_tiles + prow / u.prefix_tile) * g
                                : base + ((s - u.prefix_splits) * sh.tiles + tile) * g;
        return record(a, D, min(granule, a.granules - g), head, g, pre ? prow % u.prefix_tile : row % per);
      };
      float mx = -FLT_MAX, l = 0.0f;
      float4v o{0.0f, 0.0f, 0.0f, 0.0f};
      constexpr int BATCH = 8;
      for (int s0 = 0; s0 < parts; s0 += BATCH) {
        float4v v[BATCH];
        float ms[BATCH], ls[BATCH];
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
          const float* p = rec(min(s0 + b, parts - 1));
          v[b] = *reinterpret_cast<const float4v*>(p + 4 * d4);
          ms[b] = p[D];
          ls[b] = p[D + 1];
        }
        float mn = mx;
#pragma unroll
        for (int b = 0; b < BATCH; ++b) mn = fmaxf(mn, ms[b]);
        const float f0 = __builtin_amdgcn_exp2f(mx - mn);
        mx = mn;
        l *= f0;
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] *= f0;
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
          if (s0 + b >= parts) continue;
          const float f = __builtin_amdgcn_exp2f(ms[b] - mx);
          l = fmaf(ls[b], f, l);
#pragma unroll
          for (int c = 0; c < 4; ++c) o[c] = fmaf(v[b][c], f, o[c]);
        }
      }
      half4v h;
#pragma unroll
      for (int c = 0; c < 4; ++c) h[c] = static_cast<_Float16>(none ? 0.0f : o[c] / l);
      *reinterpret_cast<half4v*>(a.out + (static_cast<int64_t>(token) * hq + head * a.group + gq) * D + 4 * d4) = h;
    }
  }
}

// Workgroups per KV head that the keys are split for: about two per CU.
int target_of(int hkv, int cu_count) { return std::max(1, (2 * cu_count + hkv - 1) / hkv); }

// Most tiles of the requests: narrow ones, one per request with tokens at most, and
// wide ones, whole ones and one begun per request of more than 16 rows.
int64_t wide_tiles(int64_t n_req, int64_t tokens, int64_t group) {
  return tokens * group / kWide + std::min(n_req, tokens * group / (kNarrow + 1));
}
int64_t most_tiles(int64_t n_req, int64_t tokens, int64_t group) {
  return wide_tiles(n_req, tokens, group) + std::min(n_req, tokens);
}
int64_t prefix_tiles(int64_t tokens, int64_t group) { return (tokens * group + kWide - 1) / kWide; }

}  // namespace

size_t attn_paged_workspace_bytes(int32_t hq, int32_t hkv, int32_t d, int64_t n_req, int64_t tokens, bool prefix,
                                  int cu_count) {
  const int64_t target = target_of(hkv, cu_count), group = hq / hkv;
  // Splits of c blocks: sum tiles ceil(blocks / c) <= tiles + target, and 2 target
  // over the tiles with two or more, which alone leave parts where there is no prefix.
  const int64_t granules =
      prefix ? std::min(n_req, tokens) +
                   (wide_tiles(n_req, tokens, group) + prefix_tiles(tokens, group) + target) * (kWide / 16)
             : 2 * target * (kWide / 16);
  return static_cast<size_t>(granules) * hkv * 16 * (d + 4) * sizeof(float);
}

hipError_t launch_attn_paged(PagedAttnArgs a, int32_t d, size_t ws_bytes, int cu_count, hipStream_t st) {
  if (a.tokens == 0) return hipSuccess;
  a.target = target_of(a.hkv, cu_count);
  a.granules = static_cast<int>(
      std::min<size_t>(ws_bytes / (static_cast<size_t>(a.hkv) * 16 * (d + 4) * sizeof(float)), INT32_MAX));
  const int64_t units = most_tiles(a.n_req, a.tokens, a.group) + a.target +
                        (a.prefix_pages ? prefix_tiles(a.tokens, a.group) : 0);
  // About 2,048 workgroups join the parts.
  const int steps = static_cast<int>((static_cast<int64_t>(a.tokens) * a.hkv + 2047) / 2048);
  const dim3 grid(static_cast<unsigned>(units * a.hkv)), join(static_cast<unsigned>((a.tokens + steps - 1) / steps * a.hkv));
  if (d == 64) {
    hipLaunchKernelGGL(paged_attn_kernel<64>, grid, dim3(256), 0, st, a);
    hipLaunchKernelGGL(paged_attn_join_kernel<64>, join, dim3(256), 0, st, a, steps);
  } else {
    hipLaunchKernelGGL(paged_attn_kernel<128>, grid, dim3(256), 0, st, a);
    hipLaunchKernelGGL(paged_attn_join_kernel<128>, join, dim3(256), 0, st, a, steps);
  }
  return hipGetLastError();
}

}  // namespace qm
