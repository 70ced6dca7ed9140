// C ABI of the operators on token rows in front of and between the factorised matrices (see include/flop.h): embedding lookup and
// its gradient, dropout, layer norm.  Argument checks, workspace planning and launches; the kernels are in embedding_rows.cuh, dropout.cuh
// and layer_norm.cuh.
#include <math.h>
#include <string.h>

#include "host.cuh"
#include "embedding_rows.cuh"
#include "layer_norm.cuh"
#include "rows_ws.h"

using namespace flop;
typedef __nv_bfloat16 bf16;

namespace {

constexpr int64_t kMaxCols = 1 << 23;      // a launch has at most 65535 segments of a row, of 256 columns or more

// Kernels read and write whole values: an address between them would fault.
bool on_values(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }         // fp32, int32
bool on_pairs(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 7) == 0; }          // the generator's counter, (mean, rstd)

// A matrix that an operator reads or writes: where it lies, and whether the kernels can take it.
struct RowsArg {
  const void* p; int64_t ld; int dt;
  bool given() const { return p != nullptr; }
  bool fits(int64_t d) const { return ld >= d; }
  bool placed() const { return dt == FLOP_BF16 ? bf16_ok(p, ld) : on_values(p); }           // the library's rule for bf16; whole values
  bool vec() const { return aligned16(p) && (ld * (int64_t)elt(dt)) % 16 == 0; }            // rows start on 16 bytes
  Span span(int64_t T, int64_t d) const { return Span(p, T, d, ld, elt(dt)); }
  // Whether this matrix, of T rows, and another one of To rows share a byte.  Rows of the same pitch may lie side by side: then neither's columns reach the other's, to the right or,
  // in the next row, to the left.
  bool meets(const RowsArg& o, int64_t T, int64_t To, int64_t d) const {
    if (!span(T, d).meets(o.span(To, d))) return false;
    const uint64_t pitch = (uint64_t)ld * elt(dt), mine = (uint64_t)d * elt(dt), theirs = (uint64_t)d * elt(o.dt);
    if (pitch != (uint64_t)o.ld * elt(o.dt)) return true;
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(o.p);
    const uint64_t right = a <= b ? (b - a) % pitch : (pitch - (a - b) % pitch) % pitch;      // from a row's start to that of the other's next one
    return right < mine || pitch - right < theirs;
  }
};
// Every row is read before it is written, element by element by the same thread, so an output may be an input; half of it may not.
bool in_place_or_apart(const RowsArg& out, const RowsArg& in, int64_t T, int64_t d) {
  return !out.given() || !in.given() || (out.p == in.p && out.ld == in.ld && out.dt == in.dt) || !out.meets(in, T, T, d);
}
bool apart(const RowsArg& a, const RowsArg& b, int64_t T, int64_t d) { return !a.given() || !b.given() || !a.meets(b, T, T, d); }

int64_t groups_of(int64_t d) { return (d + 7) / 8; }
int64_t units_of(int64_t d, int dt) { return (d * (int64_t)elt(dt) + 15) / 16; }

template <typename T> constexpr int kType = sizeof(T) == 2 ? FLOP_BF16 : FLOP_F32;

bool valid_p(float p) { return p >= 0.f && p < 1.f; }
Drop make_drop(float p, uint64_t seed, uint64_t offset, const uint64_t* offset_dev) {
  Drop d{};
  d.key = make_uint2((uint32_t)seed, (uint32_t)(seed >> 32));
  d.offset = offset; d.offset_dev = offset_dev;
  d.threshold = std::min<uint32_t>((uint32_t)floor((double)p * 65536.0 + 0.5), 65535u);
  d.scale = (float)(65536.0 / (65536.0 - (double)d.threshold));
  return d;
}

int launched() {
  count_launch();
  FLOP_CUDA(cudaGetLastError());
  return FLOP_OK;
}

// ---------------------------------------------------------------- embedding
template <typename T, int LANES, int NG>
int launch_lookup_as(const emb::LookupArgs& a, int64_t units, cudaStream_t st) {
  constexpr int RB = 4, rows = 256 / LANES * RB;
  // a row for each set of threads where four would leave the machine without a round of blocks
  const int64_t segments = (units + LANES * NG - 1) / (LANES * NG);
  if ((a.T + rows - 1) / rows * segments < num_sms()) {
    launch_k(emb::lookup_kernel<T, LANES, NG, 1>, dim3((unsigned)((a.T + rows / RB - 1) / (rows / RB)), (unsigned)segments), dim3(256), (size_t)0, st, a);
  } else {
    launch_k(emb::lookup_kernel<T, LANES, NG, RB>, dim3((unsigned)((a.T + rows - 1) / rows), (unsigned)segments), dim3(256), (size_t)0, st, a);
  }
  return launched();
}
template <typename T>
int launch_lookup(const emb::LookupArgs& a, int64_t units, cudaStream_t st) {
  if (units <= 4) return launch_lookup_as<T, 4, 1>(a, units, st);
  if (units <= 8) return launch_lookup_as<T, 8, 1>(a, units, st);
  if (units <= 16) return launch_lookup_as<T, 16, 1>(a, units, st);
  if (units <= 32) return launch_lookup_as<T, 32, 1>(a, units, st);
  if (units <= 64) return launch_lookup_as<T, 32, 2>(a, units, st);
  if (units <= 96) return launch_lookup_as<T, 32, 3>(a, units, st);
  return launch_lookup_as<T, 64, 2>(a, units, st);
}

struct RunPlan { int lanes, slices, chunk; int64_t chunks; };
// Chunks so long that there are about 16 warps for an SM, which is what the rings leave room for (with 24 and shorter rings 16384 tokens of 205 words take the same time, a batch
// of one word 38 us instead of 35).  A long batch of narrow rows has longer ones, up to 256 tokens, so that a frequent word has not too many parts: 4219 of 135000 tokens of 16 columns, 16384
// of 4 Mi.
constexpr int kRunWarps = 16, kRunAhead = 6, kLeastChunk = 16, kMostChunk = 256;
RunPlan plan_runs(int64_t T, int64_t d) {
  RunPlan p;
  p.lanes = d <= 64 ? 8 : d <= 128 ? 16 : 32;
  p.slices = (int)((d + p.lanes * 8 - 1) / (p.lanes * 8));
  const int64_t warps = (int64_t)num_sms() * kRunWarps, by_work = (T * p.slices * p.lanes + 32 * warps - 1) / (32 * warps), by_parts = T / 4096;
  p.chunk = (int)round_up(std::min<int64_t>(std::max<int64_t>({kLeastChunk, by_work, by_parts}), kMostChunk), 4);
  p.chunks = (T + p.chunk - 1) / p.chunk;
  return p;
}
// Room for the parts: the most chunks of any batch of up to T tokens, so that a workspace for a batch serves the smaller ones (their chunks are shorter, and there may be more of
// them).  Chunks that are not of the greatest length are at least the work of a warp long.
int64_t most_chunks(int64_t T, int64_t d) {
  const RunPlan p = plan_runs(T, d);
  const int64_t warps = (int64_t)num_sms() * kRunWarps, share = (int64_t)p.slices * p.lanes;
  return std::min<int64_t>((T + kLeastChunk - 1) / kLeastChunk, std::max<int64_t>((warps * 32 + share - 1) / share, (T + kMostChunk - 1) / kMostChunk));
}
struct EmbWs { uint2* order[2]; uint32_t* counts; float* part; int64_t part_ld; size_t bytes; };
EmbWs plan_emb_ws(Arena& ar, int64_t T, int64_t d) {
  EmbWs w{};
  if (T == 0 || d == 0) return w;
  for (auto& o : w.order) o = (uint2*)ar.take((size_t)(T + emb::kBehind) * sizeof(uint2));
  w.counts = (uint32_t*)ar.take((size_t)emb::kSortBlocks * (1u << emb::kMaxDigitBits) * 4);
  w.part_ld = round_up(d, 8);
  w.part = (float*)ar.take((size_t)most_chunks(T, d) * 2 * w.part_ld * 4);
  w.bytes = ar.used;
  return w;
}

// Batches of up to 8 x 2048 tokens by one cluster; longer ones by two launches a digit.
constexpr int kSortCluster = 8;
int launch_sort(const emb::SortArgs& a, int beside, cudaStream_t st) {
  static OncePerDevice configured;
  FLOP_TRY(allow_smem(configured, emb::sort_smem(emb::kMaxDigitBits), emb::sort_kernel, emb::sort_count_kernel, emb::sort_move_kernel));
  const size_t smem = emb::sort_smem(a.bits);
  if (a.blocks > kSortCluster) {
    for (int pass = 0; pass < a.passes; ++pass) {
      launch_k(emb::sort_count_kernel, dim3((unsigned)(a.blocks + (pass == 0 ? beside : 0))), dim3(emb::kSortThreads), smem, st, a, pass);
      FLOP_TRY(launched());
      launch_k(emb::sort_move_kernel, dim3((unsigned)a.blocks), dim3(emb::kSortThreads), smem, st, a, pass);
      FLOP_TRY(launched());
    }
    return FLOP_OK;
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(a.blocks + beside / a.blocks * a.blocks));
  cfg.blockDim = dim3(emb::kSortThreads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)a.blocks; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl_on() ? 2 : 1;
  FLOP_CUDA(cudaLaunchKernelEx(&cfg, emb::sort_kernel, a));
  count_launch();
  return FLOP_OK;
}

template <typename T, typename TW, int LPT>
int launch_runs_as(const emb::RunArgs& a, cudaStream_t st) {
  constexpr int AHEAD = kRunAhead / (sizeof(T) / 2);     // the same bytes
  constexpr size_t ring = (size_t)AHEAD * emb::kStep * (sizeof(T) / 2) * 256 * 16;
  auto kern = emb::runs_kernel<T, TW, LPT, AHEAD>;
  static OncePerDevice configured;
  FLOP_TRY(allow_smem(configured, ring, kern));
  launch_k(kern, dim3((unsigned)((a.chunks * a.slices + 256 / LPT - 1) / (256 / LPT))), dim3(256), ring, st, a);
  FLOP_TRY(launched());
  if (a.chunks > 1) {
    launch_k(emb::joints_kernel<TW, LPT>, dim3((unsigned)((a.chunks + 7) / 8), (unsigned)a.slices), dim3(256), (size_t)0, st, a);
    FLOP_TRY(launched());
  }
  return FLOP_OK;
}
template <typename T, typename TW>
int launch_runs(const emb::RunArgs& a, int lanes, cudaStream_t st) {
  return lanes == 8 ? launch_runs_as<T, TW, 8>(a, st) : lanes == 16 ? launch_runs_as<T, TW, 16>(a, st) : launch_runs_as<T, TW, 32>(a, st);
}

// One launch, in which every token looks through all words for every 256 columns (at most 12 Mi looks), against a sort and two more launches.  us in one launch / sorted: 32000 words, 768 columns, 256
// tokens 16.6 / 25.9, 1024 19.9 / 28.0, 1500 23.0 / 28.5, 2048 26.8 / 29.1; 205 words, 2048 columns, 1024 tokens 12.5 / 15.1, 1500 17.6 / 14.2; 50000 words, 4096 columns, 1024
// tokens 77.6 / 71, 1500 94 / 72.  A batch of one word is the worst for it, and the rule does not see it: 512 tokens, 2048 columns 13.1 / 11.1, 1024 22.5 / 12.4.
bool few_tokens(int64_t T, int64_t d) { return T <= emb::kFewTokens && T * T * ((d + 255) / 256) <= 12 << 20; }
template <typename T, typename TW>
int launch_few(emb::RunArgs a, cudaStream_t st) {
  a.slices = (a.d + 255) / 256;
  a.token_blocks = (int)((a.T + 7) / 8) * a.slices;
  a.clear_rows = (int)std::max<int64_t>(1, std::min<int64_t>(emb::kFewRows, 65536 / std::max<int64_t>(a.clear.row_bytes, 1)));
  const int64_t clear_blocks = (a.clear.rows + a.clear_rows - 1) / a.clear_rows;
  const dim3 grid((unsigned)(a.token_blocks + clear_blocks));
  // lists of 2048 tokens in every block: 1000 tokens of 50001 x 410 fp32 25.1 us, lists of 1024 24.4
  if (a.T <= 1024) launch_k(emb::few_kernel<T, TW, 1>, grid, dim3(256), (size_t)0, st, a);
  else launch_k(emb::few_kernel<T, TW, 2>, grid, dim3(256), (size_t)0, st, a);
  return launched();
}

// ---------------------------------------------------------------- layer norm
// How a row is held: by `lanes` threads with `ng` units of 16 bytes each, in blocks of `threads`; lanes 0: rows too wide for that, which are walked.
struct NormPlan { int lanes, ng, threads; };
NormPlan plan_norm(int64_t units, int dt) {
  if (units <= 8) return {8, 1, 128};
  if (units <= 16) return {16, 1, 128};
  if (units <= 32) return {32, 1, 128};
  if (units <= 64) return {32, 2, 128};
  if (units <= 96) return {32, 3, 128};
  if (units <= 128) return {64, 2, 64};
  if (units <= 256) return {128, 2, 128};
  if (units <= 384) return {128, 3, 128};
  if (units <= 512) return {256, 2, 256};
  if (units <= 768) return {256, 3, 256};
  if (units <= 1024) return {512, 2, 512};
  if (units <= 1536) return {512, 3, 512};
  if (units <= 2048) return {512, 4, 512};
  // a thread's units of fp32 take half the registers: 1024 x 16384 forward and backward 81 us, 118 walked
  if (dt == FLOP_F32 && units <= 3 * 1024) return {1024, 3, 1024};
  if (dt == FLOP_F32 && units <= 4096) return {1024, 4, 1024};
  return {0, 0, 0};
}
#define FLOP_HELD_PLANS(X) X(8, 1, 128) X(16, 1, 128) X(32, 1, 128) X(32, 2, 128) X(32, 3, 128) X(64, 2, 64) X(128, 2, 128) X(128, 3, 128) X(256, 2, 256) X(256, 3, 256) \
  X(512, 2, 512) X(512, 3, 512) X(512, 4, 512)
constexpr int between(int lo, int v, int hi) { return v < lo ? lo : v > hi ? hi : v; }
constexpr int kRing = 220 * 1024;                     // shared memory of an SM that the rings of its blocks may take
// Rows that a set of threads works on at once, blocks of an SM and batches copied ahead: 512 threads of an SM (dropout, with fewer registers, 768: 9000 x 410 with
// residual 6.6 us, 8.5 with 512).
struct NormShape { int rb, blocks, stages; };
constexpr NormShape fwd_shape(int ng, int threads, int tensors, int per_sm = 512) {
  const int rb = between(1, 4 / (ng * tensors), 4), blocks = between(1, per_sm / threads, 16);
  return {rb, blocks, between(1, kRing / (tensors * rb * ng * threads * 16 * blocks), 4)};
}
// One block on an SM, so that there are few parts of the column sums to add up: 512 threads, or, because a thread's three units of bf16 take more than 128
// registers, 384 (4096 x 768 bf16 15.0 us, 16.7 with 512 threads that spill; 32 lanes still spill 8 bytes).  It goes by the units, not by the type: three of fp32 take 118.  Four units of
// bf16 (12289 to 16384 columns) keep 512 threads, and spill 196 bytes a thread here and 120 in the forward pass with sums; so do four of fp32 on 1024 threads (64 and 128).
constexpr int bwd_threads(int lanes, int ng) { return lanes > 512 ? lanes : ng < 3 || lanes == 512 ? 512 : 384 / lanes > 0 ? 384 / lanes * lanes : lanes; }
// Two rows at once for every barrier among the warps that share one (16384 x 2048 bf16: 43.0 us, 44.5 one by one); fp32 rows are twice the bytes.
constexpr NormShape bwd_shape(int lanes, int ng, int dt) {
  const int rb = between(1, (lanes > 32 && dt == FLOP_BF16 ? 4 : 2) / ng, 4);
  return {rb, 1, between(1, kRing / (3 * rb * ng * bwd_threads(lanes, ng) * 16), 4)};
}
// No more blocks than an equal share of the batches needs: 333 batches on 148 places are three each for 111 blocks.
int64_t norm_blocks(int lanes, int threads, int64_t T, const NormShape& s) {
  const int64_t rows = (int64_t)(threads / lanes) * s.rb, batches = (T + rows - 1) / rows, most = (int64_t)num_sms() * s.blocks;
  const int64_t each = (batches + most - 1) / most;
  return (batches + each - 1) / each;
}
// Parts of the column sums: one for each block that holds rows; where rows are walked, enough blocks for the machine, 64 rows each at least.
int64_t norm_parts(int64_t T, int64_t d, int dt) {
  const NormPlan p = plan_norm(units_of(d, dt), dt);
  if (p.lanes) return norm_blocks(p.lanes, bwd_threads(p.lanes, p.ng), T, bwd_shape(p.lanes, p.ng, dt));
  const int64_t slabs = std::max<int64_t>((groups_of(d) + 31) / 32, 1);
  return std::max<int64_t>(1, std::min<int64_t>((T + 63) / 64, std::max<int64_t>(1, (int64_t)num_sms() * 4 / slabs)));
}
// Room for the parts: the most of any batch of up to T rows (equal shares may leave a larger batch fewer blocks than a smaller one), so that a workspace for a batch serves the
// smaller ones.
int64_t most_parts(int64_t T, int64_t d, int dt) {
  const NormPlan p = plan_norm(units_of(d, dt), dt);
  if (!p.lanes) return norm_parts(T, d, dt);
  const NormShape s = bwd_shape(p.lanes, p.ng, dt);
  const int64_t rows = (int64_t)(bwd_threads(p.lanes, p.ng) / p.lanes) * s.rb;
  return std::min<int64_t>((T + rows - 1) / rows, (int64_t)num_sms() * s.blocks);
}
struct NormWs { float* part; int64_t part_ld, n_part; size_t bytes; };
NormWs plan_norm_ws(Arena& ar, int64_t T, int64_t d, int dt) {
  NormWs w{};
  if (T == 0 || d == 0) return w;
  w.part_ld = round_up(d, 8);
  w.n_part = norm_parts(T, d, dt);
  w.part = (float*)ar.take((size_t)most_parts(T, d, dt) * 2 * w.part_ld * 4);
  w.bytes = ar.used;
  return w;
}

int walk_threads(int groups) { return std::min(512, (groups + 31) / 32 * 32); }

template <typename T, int MODE, int LANES, int NG, int THREADS>
int launch_fwd_held(const norm::FwdArgs& a, unsigned segments, cudaStream_t st) {
  constexpr int TENSORS = norm::kTensors<MODE>;
  constexpr NormShape s = fwd_shape(NG, THREADS, TENSORS, norm::kNorm<MODE> ? 512 : 768);
  constexpr size_t smem = (size_t)s.stages * TENSORS * s.rb * NG * THREADS * 16;
  auto kern = norm::fwd_kernel<T, MODE, LANES, NG, s.rb, s.stages, THREADS, s.blocks>;
  static OncePerDevice configured;
  FLOP_TRY(allow_smem(configured, smem, kern));
  const int64_t blocks = norm_blocks(LANES, THREADS, a.T, s);
  launch_k(kern, dim3((unsigned)(segments == 1 ? blocks : (blocks + segments - 1) / segments), segments), dim3(THREADS), smem, st, a);
  return launched();
}
// Dropout by itself: rows of more than 256 units in segments of 256.
template <typename T, int MODE>
int launch_dropout(const norm::FwdArgs& a, cudaStream_t st) {
  const int64_t units = units_of(a.d, kType<T>);
  if (units <= 8) return launch_fwd_held<T, MODE, 8, 1, 128>(a, 1, st);
  if (units <= 16) return launch_fwd_held<T, MODE, 16, 1, 128>(a, 1, st);
  if (units <= 32) return launch_fwd_held<T, MODE, 32, 1, 128>(a, 1, st);
  if (units <= 64) return launch_fwd_held<T, MODE, 32, 2, 128>(a, 1, st);
  if (units <= 96) return launch_fwd_held<T, MODE, 32, 3, 128>(a, 1, st);
  if (units <= 128) return launch_fwd_held<T, MODE, 64, 2, 128>(a, 1, st);
  return launch_fwd_held<T, MODE, 128, 2, 128>(a, (unsigned)((units + 255) / 256), st);
}
template <typename T, bool SUM>
int launch_norm_fwd(const norm::FwdArgs& a, cudaStream_t st) {
  const NormPlan p = plan_norm(units_of(a.d, kType<T>), kType<T>);
#define FLOP_HELD(L, N, B) if (p.lanes == L && p.ng == N) return launch_fwd_held<T, SUM ? norm::SUMMED : norm::WHOLE, L, N, B>(a, 1, st);
  FLOP_HELD_PLANS(FLOP_HELD)
  if constexpr (sizeof(T) == 4) { FLOP_HELD(1024, 3, 1024) FLOP_HELD(1024, 4, 1024) }
#undef FLOP_HELD
  launch_k(norm::fwd_walk_kernel<T, SUM>, dim3((unsigned)a.T), dim3(walk_threads(a.groups)), (size_t)0, st, a);
  return launched();
}

template <typename T, int LANES, int NG>
int launch_norm_bwd_held(const norm::BwdArgs& a, cudaStream_t st) {
  constexpr int THREADS = bwd_threads(LANES, NG);
  constexpr NormShape s = bwd_shape(LANES, NG, kType<T>);
  auto kern = norm::bwd_kernel<T, LANES, NG, s.rb, s.stages, THREADS, s.blocks>;
  constexpr size_t tensor = (size_t)s.stages * s.rb * NG * THREADS * 16;
  static OncePerDevice configured;
  FLOP_TRY(allow_smem(configured, 3 * tensor, kern));
  launch_k(kern, dim3((unsigned)norm_blocks(LANES, THREADS, a.T, s)), dim3(THREADS), (a.dS ? 3 : 2) * tensor, st, a);
  return launched();
}
template <typename T>
int launch_norm_bwd_rows(const norm::BwdArgs& a, cudaStream_t st) {
  const NormPlan p = plan_norm(units_of(a.d, kType<T>), kType<T>);
#define FLOP_HELD(L, N, B) if (p.lanes == L && p.ng == N) return launch_norm_bwd_held<T, L, N>(a, st);
  FLOP_HELD_PLANS(FLOP_HELD)
  if constexpr (sizeof(T) == 4) { FLOP_HELD(1024, 3, 1024) FLOP_HELD(1024, 4, 1024) }
#undef FLOP_HELD
  if (a.n_part) {     // before the rows, whose outputs may take the place of what the sums read
    launch_k(norm::bwd_columns_kernel<T>, dim3((unsigned)((a.groups + 31) / 32), (unsigned)a.n_part), dim3(256), (size_t)0, st, a);
    FLOP_TRY(launched());
  }
  if (a.dX || a.dR) {
    launch_k(norm::bwd_walk_kernel<T>, dim3((unsigned)a.T), dim3(walk_threads(a.groups)), (size_t)0, st, a);
    FLOP_TRY(launched());
  }
  return FLOP_OK;
}
template <typename T>
int launch_norm_bwd(const norm::BwdArgs& a, cudaStream_t st) {
  if (a.n_part || a.dX || a.dR) FLOP_TRY(launch_norm_bwd_rows<T>(a, st));
  const bool held = plan_norm(units_of(a.d, kType<T>), kType<T>).lanes > 0;
  if (a.n_part > 1 || (a.n_part && !held)) {       // a single block that holds rows has written the sums itself
    launch_k(norm::bwd_finish_kernel, dim3((unsigned)((a.d + 31) / 32), 2), dim3(32 * norm::kFinishWarps), (size_t)0, st, (const float*)a.part, a.part_ld, a.n_part, a.d, a.dweight,
             a.dbias, a.accumulate);
    FLOP_TRY(launched());
  }
  return FLOP_OK;
}

}  // namespace

namespace flop {
size_t embedding_rows_ws_bytes(int64_t T, int64_t d) {
  Arena ar{nullptr, 0, 0};
  return plan_emb_ws(ar, T, d).bytes;
}
size_t layer_norm_ws_bytes(int64_t T, int64_t d, int dt) {
  Arena ar{nullptr, 0, 0};
  return plan_norm_ws(ar, T, d, dt).bytes;
}
}  // namespace flop

extern "C" {

int flop_embedding_fwd(const int32_t* ids, int64_t T, const void* E, int64_t lde, int64_t n_rows, float scale, void* Y, int64_t ldy, int64_t d, int dt,
                       void* stream) {
  if (T < 0 || n_rows < 0 || d < 0 || !valid_dt(dt)) return FLOP_ERR_INVALID_ARG;
  if (T == 0 || d == 0) return FLOP_OK;
  const RowsArg e{E, lde, dt}, y{Y, ldy, dt};
  if (!ids || !y.given() || !y.fits(d) || (n_rows > 0 && (!e.given() || !e.fits(d)))) return FLOP_ERR_INVALID_ARG;
  if (T > INT32_MAX || n_rows > INT32_MAX || d > kMaxCols || !y.placed() || (n_rows > 0 && !e.placed()) || !on_values(ids)) return FLOP_ERR_UNSUPPORTED;
  if (e.meets(y, n_rows, T, d) || Span(ids, 1, T, T, 4).meets(y.span(T, d))) return FLOP_ERR_INVALID_ARG;
  emb::LookupArgs a{};
  a.ids = ids; a.T = T; a.E = E; a.lde = lde; a.V = n_rows; a.Y = Y; a.ldy = ldy; a.scale = scale; a.d = (int)d;
  a.vec = y.vec() && (n_rows == 0 || e.vec());
  return dt == FLOP_BF16 ? launch_lookup<bf16>(a, units_of(d, dt), (cudaStream_t)stream) : launch_lookup<float>(a, units_of(d, dt), (cudaStream_t)stream);
}

int flop_embedding_bwd(const void* dY, int64_t lddy, const int32_t* ids, int64_t T, int64_t n_rows, float scale, void* dE, int64_t ldde, int accumulate,
                       int64_t d, int dt, int wgrad_dt, void* ws, size_t ws_bytes, void* stream) {
  if (T < 0 || n_rows < 0 || d < 0 || !valid_dt(dt) || !valid_dt(wgrad_dt)) return FLOP_ERR_INVALID_ARG;
  if (n_rows == 0 || d == 0 || (T == 0 && accumulate)) return FLOP_OK;
  const RowsArg dy{dY, lddy, dt}, de{dE, ldde, wgrad_dt};
  if (!de.given() || !de.fits(d) || (T > 0 && (!ids || !dy.given() || !dy.fits(d)))) return FLOP_ERR_INVALID_ARG;
  if (T > INT32_MAX || n_rows > INT32_MAX || d > kMaxCols || lddy > INT32_MAX || !de.placed() || (T > 0 && (!dy.placed() || !on_values(ids)))) return FLOP_ERR_UNSUPPORTED;
  const Span out = de.span(n_rows, d);
  if (T > 0 && (de.meets(dy, n_rows, T, d) || out.meets(Span(ids, 1, T, T, 4)))) return FLOP_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  Arena ar{(unsigned char*)ws, ws_bytes, 0};
  const EmbWs w = plan_emb_ws(ar, T, d);
  FLOP_TRY(check_ws(ws, ws_bytes, w.bytes));
  const RunPlan p = plan_runs(T, d);
  emb::RunArgs a{};
  a.order = w.order[0]; a.ids = ids; a.T = T; a.V = (uint32_t)n_rows; a.dY = dY; a.lddy = lddy; a.dE = dE; a.ldde = ldde; a.part = w.part; a.part_ld = w.part_ld;
  a.chunks = p.chunks; a.chunk = p.chunk; a.scale = scale; a.d = (int)d; a.slices = p.slices; a.accumulate = accumulate; a.vec = dy.vec(); a.vec_out = de.vec();
  emb::ClearArgs& z = a.clear;
  if (!accumulate) {
    z.p = (unsigned char*)dE; z.rows = n_rows; z.row_bytes = d * (int64_t)elt(wgrad_dt); z.pitch = ldde * (int64_t)elt(wgrad_dt); z.vec = de.vec();
  }
  auto typed = [&](auto go) {
    if (dt == FLOP_BF16) return wgrad_dt == FLOP_BF16 ? go(bf16{}, bf16{}) : go(bf16{}, float{});
    return wgrad_dt == FLOP_BF16 ? go(float{}, bf16{}) : go(float{}, float{});
  };
  if (few_tokens(T, d)) return typed([&](auto t, auto tw) { return launch_few<decltype(t), decltype(tw)>(a, st); });
  emb::SortArgs s{};
  s.ids = ids; s.T = T; s.V = (uint32_t)n_rows; s.clear = z;
  s.order[0] = w.order[0]; s.order[1] = w.order[1];
  int word_bits = 1;
  while ((uint64_t)n_rows >> word_bits) ++word_bits;          // n_rows itself stands for padding
  s.passes = (word_bits + emb::kMaxDigitBits - 1) / emb::kMaxDigitBits;
  s.bits = (word_bits + s.passes - 1) / s.passes;
  s.counts = w.counts;
  const int64_t blocks = (T + emb::kSortBlock - 1) / emb::kSortBlock;
  s.blocks = 1;
  while (s.blocks < kSortCluster && s.blocks < blocks) s.blocks *= 2;
  if (blocks > kSortCluster) s.blocks = (int)std::min<int64_t>(blocks, emb::kSortBlocks);
  // Blocks that clear dE beside the sort, a tile for each, up to 32 for an SM.  (Asking for rows of dY ahead of time there as well made the sort slower by more than the rows
  // then came sooner: 16384 tokens of 205 words, 2048 columns 38 us, 27 without; clearing a part of the rows beside the joints instead, 4096 tokens of 32000 words, 768 columns 33 us, 31 without.)
  const int64_t tiles = (z.rows * ((z.row_bytes + 15) / 16) + 4 * emb::kSortThreads - 1) / (4 * emb::kSortThreads);
  const int beside = (int)std::min<int64_t>(round_up(tiles, s.blocks), (int64_t)num_sms() * 32);
  FLOP_TRY(launch_sort(s, beside, st));
  return typed([&](auto t, auto tw) { return launch_runs<decltype(t), decltype(tw)>(a, p.lanes, st); });
}

static int dropout_impl(const void* X, int64_t ldx, const void* R, int64_t ldr, float p, uint64_t seed, uint64_t offset, const uint64_t* offset_dev, void* Y,
                        int64_t ldy, int64_t T, int64_t d, int dt, void* stream) {
  if (T < 0 || d < 0 || !valid_dt(dt) || !valid_p(p)) return FLOP_ERR_INVALID_ARG;
  if (T == 0 || d == 0) return FLOP_OK;
  const RowsArg x{X, ldx, dt}, r{R, ldr, dt}, y{Y, ldy, dt};
  if (!x.given() || !x.fits(d) || !y.given() || !y.fits(d) || (r.given() && !r.fits(d))) return FLOP_ERR_INVALID_ARG;
  if (T > INT32_MAX || d > kMaxCols || !x.placed() || !y.placed() || (r.given() && !r.placed()) || !on_pairs(offset_dev)) return FLOP_ERR_UNSUPPORTED;
  if (!in_place_or_apart(y, x, T, d) || !in_place_or_apart(y, r, T, d)) return FLOP_ERR_INVALID_ARG;
  norm::FwdArgs a{};
  a.X = X; a.ldx = ldx; a.R = R; a.ldr = ldr; a.S = Y; a.lds = ldy; a.T = T; a.d = (int)d; a.groups = (int)groups_of(d);
  a.vec = x.vec() && y.vec() && (!r.given() || r.vec());
  a.drop = make_drop(p, seed, offset, offset_dev);
  cudaStream_t st = (cudaStream_t)stream;
  if (dt == FLOP_BF16) return R ? launch_dropout<bf16, norm::ADDED>(a, st) : launch_dropout<bf16, norm::DROPPED>(a, st);
  return R ? launch_dropout<float, norm::ADDED>(a, st) : launch_dropout<float, norm::DROPPED>(a, st);
}

int flop_dropout_fwd(const void* X, int64_t ldx, const void* R, int64_t ldr, float p, uint64_t seed, uint64_t offset, const uint64_t* offset_dev, void* Y,
                     int64_t ldy, int64_t T, int64_t d, int dt, void* stream) {
  return dropout_impl(X, ldx, R, ldr, p, seed, offset, offset_dev, Y, ldy, T, d, dt, stream);
}
int flop_dropout_bwd(const void* dY, int64_t lddy, float p, uint64_t seed, uint64_t offset, const uint64_t* offset_dev, void* dX, int64_t lddx, int64_t T,
                     int64_t d, int dt, void* stream) {
  return dropout_impl(dY, lddy, nullptr, 0, p, seed, offset, offset_dev, dX, lddx, T, d, dt, stream);
}

int flop_layer_norm_fwd(const void* X, int64_t ldx, const void* R, int64_t ldr, float p, uint64_t seed, uint64_t offset, const uint64_t* offset_dev,
                        const float* weight, const float* bias, float eps, void* S, int64_t lds, void* Y, int64_t ldy, float* stats, int64_t T, int64_t d,
                        int dt, void* stream) {
  if (T < 0 || d < 0 || !valid_dt(dt) || !valid_p(p) || !(eps >= 0.f) || !(eps < INFINITY)) return FLOP_ERR_INVALID_ARG;
  if (T == 0 || d == 0) return FLOP_OK;
  const RowsArg x{X, ldx, dt}, r{R, ldr, dt}, s{S, lds, dt}, y{Y, ldy, dt};
  if (!x.given() || !x.fits(d) || !y.given() || !y.fits(d) || (r.given() && !r.fits(d)) || (s.given() && !s.fits(d))) return FLOP_ERR_INVALID_ARG;
  if (T > INT32_MAX || d > kMaxCols || !x.placed() || !y.placed() || (r.given() && !r.placed()) || (s.given() && !s.placed()) ||
      !on_pairs(stats) || !on_pairs(offset_dev) || !on_values(weight) || !on_values(bias))
    return FLOP_ERR_UNSUPPORTED;
  if (!in_place_or_apart(s, x, T, d) || !in_place_or_apart(s, r, T, d) || !in_place_or_apart(y, x, T, d) || !in_place_or_apart(y, r, T, d) || !apart(s, y, T, d))
    return FLOP_ERR_INVALID_ARG;
  const Span rs(stats, 1, 2 * T, 2 * T, 4);
  for (const Span& v : {rs, Span(weight, 1, d, d, 4), Span(bias, 1, d, d, 4)})
    if (y.span(T, d).meets(v) || (s.given() && s.span(T, d).meets(v))) return FLOP_ERR_INVALID_ARG;
  if (rs.meets(x.span(T, d)) || (r.given() && rs.meets(r.span(T, d))) || rs.meets(Span(weight, 1, d, d, 4)) || rs.meets(Span(bias, 1, d, d, 4))) return FLOP_ERR_INVALID_ARG;
  norm::FwdArgs a{};
  a.X = X; a.ldx = ldx; a.R = R; a.ldr = ldr; a.S = S; a.lds = lds; a.Y = Y; a.ldy = ldy; a.w = weight; a.b = bias; a.stats = (float2*)stats; a.eps = eps; a.inv_d = 1. / (double)d;
  a.T = T; a.d = (int)d; a.groups = (int)groups_of(d);
  a.vec = x.vec() && y.vec() && (!r.given() || r.vec()) && (!s.given() || s.vec());
  a.wvec = aligned16(weight) && aligned16(bias);
  a.drop = make_drop(p, seed, offset, offset_dev);
  const bool sum = R || S || a.drop.threshold;
  cudaStream_t st = (cudaStream_t)stream;
  if (dt == FLOP_BF16) return sum ? launch_norm_fwd<bf16, true>(a, st) : launch_norm_fwd<bf16, false>(a, st);
  return sum ? launch_norm_fwd<float, true>(a, st) : launch_norm_fwd<float, false>(a, st);
}

int flop_layer_norm_bwd(const void* dY, int64_t lddy, const void* S, int64_t lds, const float* stats, const float* weight, const void* dS, int64_t ldds,
                        float p, uint64_t seed, uint64_t offset, const uint64_t* offset_dev, void* dX, int64_t lddx, void* dR, int64_t lddr,
                        float* dweight, float* dbias, int accumulate, int64_t T, int64_t d, int dt, void* ws, size_t ws_bytes, void* stream) {
  if (T < 0 || d < 0 || !valid_dt(dt) || !valid_p(p)) return FLOP_ERR_INVALID_ARG;
  if (d == 0) return FLOP_OK;
  cudaStream_t st = (cudaStream_t)stream;
  if (d > kMaxCols || T > INT32_MAX || !on_values(dweight) || !on_values(dbias)) return FLOP_ERR_UNSUPPORTED;
  if (T == 0) {                          // sums over no rows
    if (accumulate || (!dweight && !dbias)) return FLOP_OK;
    launch_k(norm::bwd_finish_kernel, dim3((unsigned)((d + 31) / 32), 2), dim3(32 * norm::kFinishWarps), (size_t)0, st, (const float*)nullptr, (int64_t)0, 0, (int)d, dweight, dbias, 0);
    return launched();
  }
  const RowsArg dy{dY, lddy, dt}, s{S, lds, dt}, ds{dS, ldds, dt}, dx{dX, lddx, dt}, dr{dR, lddr, dt};
  if (!dy.given() || !dy.fits(d) || !s.given() || !s.fits(d) || !stats || (ds.given() && !ds.fits(d)) || (dx.given() && !dx.fits(d)) || (dr.given() && !dr.fits(d)))
    return FLOP_ERR_INVALID_ARG;
  if (!dy.placed() || !s.placed() || (ds.given() && !ds.placed()) || (dx.given() && !dx.placed()) || (dr.given() && !dr.placed()) ||
      !on_pairs(stats) || !on_pairs(offset_dev) || !on_values(weight))
    return FLOP_ERR_UNSUPPORTED;
  for (const RowsArg* out : {&dx, &dr})
    for (const RowsArg* in : {&dy, &s, &ds})
      if (!in_place_or_apart(*out, *in, T, d)) return FLOP_ERR_INVALID_ARG;
  if (!apart(dx, dr, T, d)) return FLOP_ERR_INVALID_ARG;
  const Span gw(dweight, 1, d, d, 4), gb(dbias, 1, d, d, 4), rs(stats, 1, 2 * T, 2 * T, 4), wv(weight, 1, d, d, 4);
  for (const RowsArg* out : {&dx, &dr}) {
    const Span o = out->given() ? out->span(T, d) : Span();
    if (o.meets(gw) || o.meets(gb) || o.meets(rs) || o.meets(wv)) return FLOP_ERR_INVALID_ARG;
  }
  for (const RowsArg* in : {&dy, &s, &ds})
    if (in->given() && (in->span(T, d).meets(gw) || in->span(T, d).meets(gb))) return FLOP_ERR_INVALID_ARG;
  if (gw.meets(gb) || gw.meets(rs) || gb.meets(rs) || gw.meets(wv) || gb.meets(wv)) return FLOP_ERR_INVALID_ARG;
  norm::BwdArgs a{};
  if (dweight || dbias) {
    Arena ar{(unsigned char*)ws, ws_bytes, 0};
    const NormWs w = plan_norm_ws(ar, T, d, dt);
    FLOP_TRY(check_ws(ws, ws_bytes, w.bytes));
    a.part = w.part; a.part_ld = w.part_ld; a.n_part = (int)w.n_part;
  }
  a.dweight = dweight; a.dbias = dbias; a.accumulate = accumulate;
  a.dY = dY; a.lddy = lddy; a.S = S; a.lds = lds; a.stats = (const float2*)stats; a.w = weight; a.dS = dS; a.ldds = ldds; a.dX = dX; a.lddx = lddx; a.dR = dR;
  a.lddr = lddr; a.T = T; a.d = (int)d; a.groups = (int)groups_of(d);
  a.vec = dy.vec() && s.vec() && (!ds.given() || ds.vec()) && (!dx.given() || dx.vec()) && (!dr.given() || dr.vec());
  a.wvec = aligned16(weight);
  a.drop = make_drop(p, seed, offset, offset_dev);
  return dt == FLOP_BF16 ? launch_norm_bwd<bf16>(a, st) : launch_norm_bwd<float>(a, st);
}

}  // extern "C"
