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
#include "qm_internal.h"

#include <algorithm>
#include <cfloat>

namespace qm {
namespace {

typedef _Float16 half4v __attribute__((ext_vector_type(4)));
typedef short short4v __attribute__((ext_vector_type(4)));

constexpr int kBlockKeys = 64;      // keys are split in multiples of this
constexpr int kMinBlocks = 2;       // fewest blocks of a split
constexpr int kTile = 16;           // rows of a tile
// Weights go to fp16 as 2^15 w: the largest is 32,768, and relative to it weights
// keep 11 bits down to 2^-29 (2^-14 unscaled).  Sums of weights carry the same factor.
constexpr float kWeightBits = 15.0f;

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

struct Share { int tiles, blocks, splits, granules; };   // of one request: granules per split of a tile

__device__ __forceinline__ int rows_of(const Requests& r, const PagedAttnArgs& a, int i) {
  return max(r.off[i + 1] - r.off[i], 0) * a.group;
}

__device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }

// c: blocks per split (0: not known yet).
__device__ __forceinline__ Share share_of(const Requests& r, const PagedAttnArgs& a, int i, int c) {
  const int rows = rows_of(r, a, i), own = r.kv[i] - (a.prefix_pages << a.page_log2);
  Share s;
  s.tiles = (rows + kTile - 1) / kTile;
  s.blocks = own > 0 ? (own + kBlockKeys - 1) / kBlockKeys : 1;
  s.splits = c ? ceil_div(s.blocks, c) : 1;
  s.granules = s.splits > 1 || a.prefix_pages ? kTile / 16 : 0;   // a lone part writes the output itself
  return s;
}

// Every lane of a wavefront takes `per` consecutive requests; units_before and
// granules_before are the sums over the earlier lanes' requests.
struct Units {
  int c, per, prefix_tiles, prefix_blocks, prefix_splits, units_before, granules_before, total;
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
  u.prefix_blocks = ((a.prefix_pages << a.page_log2) + kBlockKeys - 1) / kBlockKeys;
  u.prefix_tiles = a.prefix_pages ? (r.off[a.n_req] * a.group + kTile - 1) / kTile : 0;
  work += static_cast<int64_t>(u.prefix_tiles) * u.prefix_blocks;
  // Splits of c blocks: sum tiles ceil(blocks / c) <= tiles + target.
  u.c = static_cast<int>(max<int64_t>(kMinBlocks, (work + a.target - 1) / a.target));
  u.prefix_splits = a.prefix_pages ? ceil_div(u.prefix_blocks, u.c) : 0;
  int units = 0, granules = 0;
  for (int i = lo; i < hi; ++i) {
    const Share s = share_of(r, a, i, u.c);
    units += s.tiles * s.splits;
    granules += s.tiles * s.splits * s.granules;
  }
  const int units_to = wave_scan(units), granules_to = wave_scan(granules);
  const int p = u.prefix_tiles * u.prefix_splits;
  u.units_before = p + units_to - units;
  u.granules_before = p * (kTile / 16) + granules_to - granules;
  u.total = p + __shfl(units_to, 63);
  return u;
}

// ---------------------------------------------------- one part of one tile

// Sixteen consecutive keys of a page table: where they lie.
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

__device__ __forceinline__ half4v read_tr(const _Float16* p) {
  typedef __attribute__((address_space(3))) short4v* lds_ptr;
  return __builtin_bit_cast(half4v, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                        (lds_ptr)(const_cast<short4v*>(reinterpret_cast<const short4v*>(p)))));
}

// V in LDS: rows of D halves, the 16-byte chunk c of row r at chunk c ^ swizzle(r):
// the four rows x 32 bytes that a group of 16 lanes reads transposed fall on
// different banks.
template <int D>
__device__ __forceinline__ int v_at(int row, int dim) {
  constexpr int C = D / 8;
  return row * D + (((dim >> 3) ^ ((2 * row) & (C - 1))) << 3) + (dim & 7);
}

template <int D>
struct TileLds {
  union {
    _Float16 v[4][32 * D];          // a block of V per wavefront
    float acc[4][16][D + 4];        // the wavefronts' parts
  };
  float m[4][16], l[4][16];
};

// One tile of 16 rows against the keys [k.lo, k.hi) of one KV head: the four
// wavefronts take blocks of 32 keys in turn.
//   S^T = K Q^T   16 keys x 16 rows, K fragments straight from their pages,
//   O^T += V^T W^T, V^T read transposed out of LDS; its k slots are relabelled to
//   the keys that a lane holds weights of, so the weights never leave their lane.
// limit: keys visible to this lane's row (lane & 15), 0 for rows that do not
// exist.  Leaves the joined sums in s.acc[0], maxima in s.m[0], sums in s.l[0].
template <int D>
__device__ __forceinline__ void tile_part(const PagedAttnArgs& a, TileLds<D>& s, const uint16_t* q_row, int limit,
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
    const float mn = fmaxf(m, bm * a.scale_log2);
    const float alpha = __builtin_amdgcn_exp2f(m - mn);
    m = mn;
    half8v w;
    float sum = 0.0f;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; r += 2) {
        const float w0 = __builtin_amdgcn_exp2f(fmaf(st[t][r], a.scale_log2, kWeightBits - mn));
        const float w1 = __builtin_amdgcn_exp2f(fmaf(st[t][r + 1], a.scale_log2, kWeightBits - mn));
        sum += w0 + w1;
        w[4 * t + r] = static_cast<_Float16>(w0);           // to nearest: errors of the weights average out
        w[4 * t + r + 1] = static_cast<_Float16>(w1);
      }
    l = fmaf(l, alpha, sum);                                // of this lane's keys; joined at the end
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

template <int D>
__global__ __launch_bounds__(256, 2) void paged_attn_kernel(PagedAttnArgs a) {
  __shared__ Requests req;
  __shared__ TileLds<D> s;
  load_requests(req, a);
  const Units u = make_units(req, a);
  const int head = static_cast<int>(blockIdx.x % a.hkv);
  const int unit = static_cast<int>(blockIdx.x / a.hkv);
  if (unit >= u.total) return;
  const int prefix_len = a.prefix_pages << a.page_log2;
  const int lane = threadIdx.x & 63, col = lane & 15;
  int row0, rows, part, granule, i = 0;                     // first row of the tile, counted over the batch or the request
  Keys k;
  bool direct = false;
  const int p = u.prefix_tiles * u.prefix_splits;
  if (unit < p) {
    row0 = unit / u.prefix_splits * kTile;
    rows = req.off[a.n_req] * a.group;
    part = unit % u.prefix_splits;
    granule = unit * (kTile / 16);
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
    const int tile = (unit - at) / sh.splits;
    part = (unit - at) % sh.splits;
    granule += (unit - at) * sh.granules;
    direct = sh.granules == 0;
    row0 = tile * kTile;
    rows = rows_of(req, a, i);
    // Splits past the keys that the tile's last row sees have nothing to do
    // (the first is always there, so that every row is written).
    const int last = min(row0 + kTile, rows) - 1;
    const int seen = req.kv[i] - rows / a.group + last / a.group + 1 - prefix_len;
    if (part > 0 && part * u.c * kBlockKeys >= seen) return;
    const int64_t lo = prefix_len + static_cast<int64_t>(part) * u.c * kBlockKeys;
    k = Keys{a.tables + static_cast<int64_t>(i) * a.max_pages, static_cast<int>(lo),
             static_cast<int>(min<int64_t>(req.kv[i], lo + static_cast<int64_t>(u.c) * kBlockKeys))};
  }
  if (!direct && granule + kTile / 16 > a.granules) return;   // (the workspace covers every batch of these limits)
  // This lane's row.
  const int row = min(row0 + col, rows - 1);
  int token = row / a.group;
  const int gq = row % a.group;
  if (unit < p) i = request_of(req, a.n_req, token);
  else token += req.off[i];
  const int j = token - req.off[i], t = max(req.off[i + 1] - req.off[i], 0);
  int limit = max(min(req.kv[i] - t + j + 1, req.kv[i]), 0);
  if (unit < p) limit = min(limit, prefix_len);
  if (row0 + col >= rows) limit = 0;
  const int64_t hq = static_cast<int64_t>(a.hkv) * a.group;
  const uint16_t* q_row = a.q + (static_cast<int64_t>(token) * hq + head * a.group + gq) * D;
  tile_part<D>(a, s, q_row, limit, head, k);
  // The four wavefronts' sums, joined; thread: row, 4 dimensions.
  for (int e = threadIdx.x; e < 16 * (D / 4); e += 256) {
    const int r = e / (D / 4), d4 = e % (D / 4);
    if (row0 + r >= rows) continue;
    const float mx = fmaxf(fmaxf(s.m[0][r], s.m[1][r]), fmaxf(s.m[2][r], s.m[3][r]));
    float4v o{0.0f, 0.0f, 0.0f, 0.0f};
    float l = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = __builtin_amdgcn_exp2f(s.m[w][r] - mx);
      l = fmaf(s.l[w][r], f, l);
      const float4v v = *reinterpret_cast<const float4v*>(&s.acc[w][r][4 * d4]);
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
      float* rec = record(a, D, granule, head, kTile / 16, r);
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
template <int D>
__global__ __launch_bounds__(256) void paged_attn_join_kernel(PagedAttnArgs a) {
  __shared__ Requests req;
  load_requests(req, a);
  const int token = static_cast<int>(blockIdx.x / a.hkv), head = static_cast<int>(blockIdx.x % a.hkv);
  if (token >= req.off[a.n_req]) return;
  const Units u = make_units(req, a);
  const int i = __builtin_amdgcn_readfirstlane(request_of(req, a.n_req, token));
  const int owner = i / u.per;
  int base = __builtin_amdgcn_readlane(u.granules_before, owner);
  for (int x = owner * u.per; x < i; ++x) {
    const Share sh = share_of(req, a, x, u.c);
    base += sh.tiles * sh.splits * sh.granules;
  }
  const Share sh = share_of(req, a, i, u.c);
  if (sh.granules == 0) return;                             // written by its only part
  const int prefix_len = a.prefix_pages << a.page_log2;
  const int j = token - req.off[i], t = max(req.off[i + 1] - req.off[i], 0);
  if (j < 0 || j >= t) return;                              // (offsets that do not rise)
  const bool none = req.kv[i] - t + j + 1 <= 0;
  const int64_t hq = static_cast<int64_t>(a.hkv) * a.group;
  for (int e = threadIdx.x; e < a.group * (D / 4); e += 256) {
    const int gq = e / (D / 4), d4 = e % (D / 4);
    const int row = j * a.group + gq, tile = row / kTile;   // of the request
    const int last = min((tile + 1) * kTile, t * a.group) - 1;
    const int seen = req.kv[i] - t + last / a.group + 1 - prefix_len;
    const int blocks = seen > 0 ? (seen + kBlockKeys - 1) / kBlockKeys : 1;
    const int own = ceil_div(blocks, u.c), parts = u.prefix_splits + own;
    const int prow = token * a.group + gq;                  // of the batch
    auto rec = [&](int s) __attribute__((always_inline)) {
      const bool pre = s < u.prefix_splits;
      const int granule = pre ? prow / kTile * u.prefix_splits * (kTile / 16) + s * (kTile / 16)
                              : base + (tile * sh.splits + s - u.prefix_splits) * sh.granules;
      return record(a, D, min(granule, a.granules - kTile / 16), head, kTile / 16, (pre ? prow : row) % kTile);
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

// Workgroups per KV head that the keys are split for: about two per CU.
int target_of(int hkv, int cu_count) { return std::max(1, (2 * cu_count + hkv - 1) / hkv); }

// Tiles of the requests (and as many again of the prefix part at most): whole ones
// and one begun per request with tokens.
int64_t most_tiles(int64_t n_req, int64_t tokens, int64_t group) {
  return tokens * group / kTile + std::min(n_req, tokens);
}
int64_t prefix_tiles(int64_t tokens, int64_t group) { return (tokens * group + kTile - 1) / kTile; }

}  // namespace

size_t attn_paged_workspace_bytes(int32_t hq, int32_t hkv, int32_t d, int64_t n_req, int64_t tokens, bool prefix,
                                  int cu_count) {
  const int64_t target = target_of(hkv, cu_count), group = hq / hkv;
  // Without a prefix only tiles of two or more splits leave parts: ceil(b / c) <= 2 b / c there.
  const int64_t units = prefix ? most_tiles(n_req, tokens, group) + prefix_tiles(tokens, group) + target : 2 * target;
  return static_cast<size_t>(units * (kTile / 16)) * hkv * 16 * (d + 4) * sizeof(float);
}

hipError_t launch_attn_paged(PagedAttnArgs a, int32_t d, size_t ws_bytes, int cu_count, hipStream_t st) {
  if (a.tokens == 0) return hipSuccess;
  a.target = target_of(a.hkv, cu_count);
  a.granules = static_cast<int>(
      std::min<size_t>(ws_bytes / (static_cast<size_t>(a.hkv) * 16 * (d + 4) * sizeof(float)), INT32_MAX));
  const int64_t units = most_tiles(a.n_req, a.tokens, a.group) + a.target +
                        (a.prefix_pages ? prefix_tiles(a.tokens, a.group) : 0);
  const dim3 grid(static_cast<unsigned>(units * a.hkv)), join(static_cast<unsigned>(static_cast<int64_t>(a.tokens) * a.hkv));
  if (d == 64) {
    hipLaunchKernelGGL(paged_attn_kernel<64>, grid, dim3(256), 0, st, a);
    hipLaunchKernelGGL(paged_attn_join_kernel<64>, join, dim3(256), 0, st, a);
  } else {
    hipLaunchKernelGGL(paged_attn_kernel<128>, grid, dim3(256), 0, st, a);
    hipLaunchKernelGGL(paged_attn_join_kernel<128>, join, dim3(256), 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace qm
