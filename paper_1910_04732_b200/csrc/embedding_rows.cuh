// Embedding lookup with a scale, Y[t] = scale E[ids[t]], and the table's gradient, dE[v] = scale sum over {t: ids[t] = v} of dY[t].
// Words outside the table are padding: a row of zeros, no gradient.
//
// The gradient sorts the tokens by word (stably: a word's tokens stay in the order of the batch) and adds up runs of equal words.  Every
// sum is taken in fp32 in an order that depends on the sizes only, every row is written once, and there are no atomics.
//   sort_kernel   : one thread-block cluster sorts (word, token) pairs, least significant digit first; the blocks behind it clear dE
//                   meanwhile, because most rows of a large table stay empty
//   runs_kernel   : the sorted tokens in chunks of equal length, whatever the words: a word that fills half of a batch is
//                   as well spread over the machine as a batch of rare ones.  A run that lies within a chunk is written to dE; what a chunk holds of
//                   a run that crosses its border goes to the workspace
//   joints_kernel : adds up the parts of the runs that cross borders, in order
#pragma once
#include <cooperative_groups.h>

#include "rows8.cuh"

namespace flop {
namespace emb {

// ---------------------------------------------------------------- lookup
struct LookupArgs {
  const int32_t* ids; int64_t T;
  const void* E; int64_t lde; int64_t V;
  void* Y; int64_t ldy;
  float scale;
  int d, groups;
  int64_t total, step_rows; int step_groups;   // groups of all rows; the grid's stride in rows and groups
  int vec;
};

template <typename T>
__global__ void __launch_bounds__(256)
lookup_kernel(const LookupArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, t = i / a.groups;
  int g = (int)(i - t * a.groups);
  for (; i < a.total; i += (int64_t)gridDim.x * blockDim.x) {
    const int n = a.d - g * 8;
    const int64_t id = a.ids[t];
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (id >= 0 && id < a.V) {
      unpack8(load8((const T*)a.E + id * a.lde + g * 8, n, a.vec, id + 1 < a.V), n, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= a.scale;
    }
    store8((T*)a.Y + t * a.ldy + g * 8, pack8<T>(v), n, a.vec);
    t += a.step_rows;
    g += a.step_groups;
    if (g >= a.groups) { g -= a.groups; ++t; }
  }
}

// ---------------------------------------------------------------- sort
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32, kMaxDigitBits = 9;

struct SortArgs {
  const int32_t* ids; int64_t T;
  uint32_t V;
  int passes, bits;                 // digits of a word, bits of a digit
  uint2* order[2];                  // (word, token) pairs, written in turn; the last pass writes order[0]
  int cluster;                      // blocks of the cluster that sorts
  unsigned char* dE; int64_t row_bytes, pitch, rows;   // what the other blocks clear (rows 0: nothing)
  int vec;
};
// Counters of every warp, then the block's and the cluster's sums.
inline size_t sort_smem(int bits) { return ((size_t)kSortWarps + 2) * (1u << bits) * 4; }

// Rows of zeros, 16 bytes at a time where rows start on 16 bytes; the last piece of a row by its elements (2 bytes divide both types).
__device__ __forceinline__ void clear_rows(const SortArgs& a, int64_t first, int64_t step) {
  const int64_t pieces = a.vec ? (a.row_bytes + 15) / 16 : a.row_bytes / 2, total = a.rows * pieces;
  int64_t i = first, row = i / pieces, piece = i - row * pieces;
  const int64_t step_rows = step / pieces, step_pieces = step - step_rows * pieces;
  for (; i < total; i += step) {
    unsigned char* p = a.dE + row * a.pitch;
    if (!a.vec) {
      *reinterpret_cast<uint16_t*>(p + piece * 2) = 0;
    } else if ((piece + 1) * 16 <= a.row_bytes) {
      *reinterpret_cast<uint4*>(p + piece * 16) = make_uint4(0, 0, 0, 0);
    } else {
      for (int64_t k = piece * 16; k < a.row_bytes; k += 2) *reinterpret_cast<uint16_t*>(p + k) = 0;
    }
    row += step_rows;
    piece += step_pieces;
    if (piece >= pieces) { piece -= pieces; ++row; }
  }
}

// A pass of a cluster of C blocks of 32 warps: warp w of block c owns the (c 32 + w)-th run of consecutive pairs.  It counts its digits;
// the block turns the counts into positions (digit by digit, over its warps; the blocks' sums over distributed shared memory); the warp
// then walks its run again and moves every pair behind the ones of the same digit before it.  Within a group of 32 the equal
// digits are found with one match instruction, so the order among them is that of the lanes.
__global__ void __launch_bounds__(kSortThreads)
sort_kernel(const SortArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  if ((int)blockIdx.x >= a.cluster) {
    clear_rows(a, (int64_t)(blockIdx.x - a.cluster) * kSortThreads + threadIdx.x, (int64_t)(gridDim.x - a.cluster) * kSortThreads);
    return;
  }
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  extern __shared__ uint32_t sm[];
  __shared__ int scan[33];
  const int bins = 1 << a.bits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rank = (int)cluster.block_rank(), C = (int)cluster.num_blocks();
  uint32_t* mine = sm + warp * bins;                     // this warp's counters
  uint32_t* total = sm + kSortWarps * bins;              // the block's counts, read by the other blocks
  uint32_t* base = total + bins;                         // where the block's pairs of a digit begin
  const int64_t per = ((a.T + (int64_t)C * kSortWarps * 32 - 1) / ((int64_t)C * kSortWarps * 32)) * 32;
  const int64_t lo = min(a.T, ((int64_t)rank * kSortWarps + warp) * per), hi = min(a.T, lo + per);
  for (int pass = 0; pass < a.passes; ++pass) {
    const bool even = ((a.passes - pass) & 1) == 0;
    const uint2* from = even ? a.order[0] : a.order[1];
    uint2* to = even ? a.order[1] : a.order[0];
    const int shift = pass * a.bits;
    auto pair = [&](int64_t i) {
      if (pass) return from[i];
      const int32_t id = a.ids[i];
      return make_uint2(min((uint32_t)id, a.V), (uint32_t)i);       // padding sorts behind every word
    };
    for (int b = lane; b < bins; b += 32) mine[b] = 0;
    __syncwarp();
    for (int64_t i = lo; i < hi; i += 32) {
      const bool on = i + lane < hi;
      const uint32_t digit = on ? (pair(i + lane).x >> shift) & (bins - 1) : bins;
      const uint32_t same = __match_any_sync(0xffffffffu, digit);
      if (on && (same >> lane) == 1u) mine[digit] += __popc(same);  // the highest lane of each digit
      __syncwarp();
    }
    __syncthreads();
    // counts of a digit, warp by warp, to the number of pairs before the warp's
    for (int b = threadIdx.x; b < bins; b += kSortThreads) {
      uint32_t s = 0;
      for (int w = 0; w < kSortWarps; ++w) {
        const uint32_t c = sm[w * bins + b];
        sm[w * bins + b] = s;
        s += c;
      }
      total[b] = s;
    }
    cluster.sync();
    int before = 0, all = 0;
    const int b = threadIdx.x;                           // bins <= threads
    if (b < bins) {
      for (int c = 0; c < C; ++c) {
        const int v = (int)*cluster.map_shared_rank(total + b, c);
        all += v;
        if (c < rank) before += v;
      }
    }
    int sum;
    const int start = block_exclusive_scan(all, scan, &sum);
    if (b < bins) base[b] = (uint32_t)(start + before);
    __syncthreads();
    for (int d = lane; d < bins; d += 32) mine[d] += base[d];
    __syncwarp();
    for (int64_t i = lo; i < hi; i += 32) {
      const bool on = i + lane < hi;
      uint2 p = make_uint2(0, 0);
      if (on) p = pair(i + lane);
      const uint32_t digit = on ? (p.x >> shift) & (bins - 1) : bins;
      const uint32_t same = __match_any_sync(0xffffffffu, digit), at = on ? mine[digit] : 0;
      __syncwarp();
      if (on) {
        to[at + __popc(same & ((1u << lane) - 1))] = p;
        if ((same >> lane) == 1u) mine[digit] = at + __popc(same);
      }
      __syncwarp();
    }
    cluster.sync();                                      // the pairs are in place and `total` has been read
  }
}

// ---------------------------------------------------------------- runs of equal words
struct RunArgs {
  const uint2* order; int64_t T;
  uint32_t V;
  const void* dY; int64_t lddy;
  void* dE; int64_t ldde;
  float* part; int64_t part_ld;     // [chunks][2][part_ld]: a chunk's share of the run that comes from before it, of the run that goes on behind it
  int64_t chunks; int chunk;        // tokens of a chunk, a multiple of 8
  float scale;
  int d, slices;                    // slices of LPT * 8 columns
  int accumulate, vec, vec_out;
};

// scale v (+)= into dE's row
template <typename TW>
__device__ __forceinline__ void write_row8(const RunArgs& a, uint32_t word, int k, int n, const float (&v)[8]) {
  TW* p = (TW*)a.dE + (int64_t)word * a.ldde + k;
  float s[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) s[j] = a.scale * v[j];
  if (a.accumulate) {
    float old[8];
    unpack8(load8((const TW*)p, n, a.vec_out, false), n, old);
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] += old[j];
  }
  store8(p, pack8<TW>(s), n, a.vec_out);
}

// LPT lanes take a chunk's slice of columns, eight columns each; rows in batches of U in flight.
template <typename T, typename TW, int LPT, int U>
__global__ void __launch_bounds__(256)
runs_kernel(const RunArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  const int64_t unit = (int64_t)blockIdx.x * (256 / LPT) + threadIdx.x / LPT;
  const int64_t c = unit / a.slices;
  if (c >= a.chunks) return;
  const int k = ((int)(unit - c * a.slices) * LPT + threadIdx.x % LPT) * 8, n = a.d - k;
  if (n <= 0) return;
  const int64_t lo = c * a.chunk, hi = min(a.T, lo + a.chunk);
  const uint32_t none = 0xFFFFFFFFu;                     // no word: words are below 2^31
  uint2 next = a.order[lo];
  bool open = lo > 0 && a.order[lo - 1].x == next.x;     // the run comes from before the chunk
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int64_t i = lo; i < hi; i += U) {
    uint2 e[U + 1];
    e[0] = next;
#pragma unroll
    for (int u = 1; u <= U; ++u) e[u] = i + u < a.T ? a.order[i + u] : make_uint2(none, 0);
    next = e[U];
    if (e[0].x >= a.V) return;                           // padding: nothing but padding follows
    Raw8<T> raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u < hi && e[u].x < a.V) raw[u] = load8((const T*)a.dY + (int64_t)e[u].y * a.lddy + k, n, a.vec, (int64_t)e[u].y + 1 < a.T);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u < hi && e[u].x < a.V) {
        float v[8];
        unpack8(raw[u], n, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += v[j];
        const bool ends = e[u + 1].x != e[u].x, last = i + u + 1 == hi;
        if (ends && !open) {
          write_row8<TW>(a, e[u].x, k, n, acc);
        } else if (ends || last) {
          float* p = a.part + ((int64_t)c * 2 + (open ? 0 : 1)) * a.part_ld + k;
          *reinterpret_cast<float4*>(p) = make_float4(acc[0], acc[1], acc[2], acc[3]);
          *reinterpret_cast<float4*>(p + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
        }
        if (ends) {
          open = false;
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[j] = 0.f;
        }
      }
    }
  }
}

// Block c: the run that begins in chunk c and crosses its end, if there is one.  Its parts in the chunks behind are dealt out to the eight
// warps as runs of consecutive chunks; the warps' sums are added in order.  A warp covers 256 columns, blockIdx.y the rest.
template <typename TW>
__global__ void __launch_bounds__(256)
joints_kernel(const RunArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  __shared__ float red[8][32][8];
  const int64_t c = blockIdx.x, lo = c * a.chunk, hi = lo + a.chunk;
  if (hi >= a.T) return;
  const uint32_t word = a.order[hi - 1].x;
  if (word >= a.V || a.order[hi].x != word) return;
  if (a.order[lo].x == word && lo > 0 && a.order[lo - 1].x == word) return;       // it began before
  // chunks behind that begin with the word: 32 candidates at a time, each warp for itself
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t m = 0;
  for (;;) {
    const int64_t at = (c + 1 + m + lane) * a.chunk;
    const unsigned on = __ballot_sync(0xffffffffu, at < a.T && a.order[at < a.T ? at : 0].x == word);
    if (on == 0xffffffffu) { m += 32; continue; }
    m += __ffs(~on) - 1;
    break;
  }
  const int k = (blockIdx.y * 32 + lane) * 8, n = a.d - k;
  const int64_t per = (m + 7) / 8, p0 = warp * per, p1 = min(m, p0 + per);
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  auto add = [&](int64_t chunk, int slot) {
    const float4* p = reinterpret_cast<const float4*>(a.part + (chunk * 2 + slot) * a.part_ld + k);
    const float4 u = p[0], v = p[1];
    acc[0] += u.x; acc[1] += u.y; acc[2] += u.z; acc[3] += u.w;
    acc[4] += v.x; acc[5] += v.y; acc[6] += v.z; acc[7] += v.w;
  };
  if (n > 0) {
    if (warp == 0) add(c, 1);
#pragma unroll 4
    for (int64_t p = p0; p < p1; ++p) add(c + 1 + p, 0);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) red[warp][lane][j] = acc[j];
  __syncthreads();
  if (warp == 0 && n > 0) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      acc[j] = 0.f;
#pragma unroll
      for (int w = 0; w < 8; ++w) acc[j] += red[w][lane][j];
    }
    write_row8<TW>(a, word, k, n, acc);
  }
}

}  // namespace emb
}  // namespace flop
