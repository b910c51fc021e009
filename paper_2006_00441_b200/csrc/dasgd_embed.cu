// Embedding lookup of K replicas and the table's gradient by sorted tokens.
//
//   lookup      out[k][t] = scale * E_k[token[k][t]]
//   gradient    dE_k[v] (+)= scale * sum_{t : token[k][t] = v} dy[k][t]
//
// Both move each byte once and do one multiply or add per element: HBM bandwidth bounds them at training sizes,
// launch latency at a token or two.  The gradient avoids floating-point atomics (whose order, and so whose result,
// changes from run to run) by sorting the tokens: the sorted order fixes the order of every sum.
#include "dasgd.h"

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <string>

namespace cg = cooperative_groups;

// defined with the contexts: stores the message that dasgd_last_error(NULL) returns
extern "C" __attribute__((visibility("hidden"))) dasgd_status dasgd_internal_fail(dasgd_ctx *ctx, dasgd_status st, const char *msg);

namespace {

constexpr int kThreads = 256;
constexpr int kSortThreads = 512, kSortWarps = kSortThreads / 32, kMaxRadixBits = 9, kMaxRadix = 1 << kMaxRadixBits;

// ---------------------------------------------------------------- loads and stores of VEC elements

template <typename T, int VEC>
__device__ __forceinline__ void load(const T *p, float (&x)[VEC]) {
  if constexpr (VEC == 1) {
    x[0] = static_cast<float>(__ldg(p));
  } else if constexpr (sizeof(T) == 4) {
    static_assert(VEC % 4 == 0, "16-byte accesses");
#pragma unroll
    for (int i = 0; i < VEC / 4; ++i) {
      const float4 v = __ldg(reinterpret_cast<const float4 *>(p) + i);
      x[4 * i] = v.x, x[4 * i + 1] = v.y, x[4 * i + 2] = v.z, x[4 * i + 3] = v.w;
    }
  } else {
    static_assert(VEC == 8, "16-byte accesses");
    const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p));
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
}

__device__ __forceinline__ uint32_t pack(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t *>(&v);
}

template <typename T, int VEC>
__device__ __forceinline__ void store(T *p, const float (&x)[VEC]) {  // streaming: nothing here is read again
  if constexpr (VEC == 1) {
    if constexpr (sizeof(T) == 4) *p = x[0];
    else *p = __float2bfloat16_rn(x[0]);
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < VEC / 4; ++i)
      __stcs(reinterpret_cast<float4 *>(p) + i, make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]));
  } else {
    __stcs(reinterpret_cast<uint4 *>(p), make_uint4(pack(x[0], x[1]), pack(x[2], x[3]), pack(x[4], x[5]), pack(x[6], x[7])));
  }
}

// ---------------------------------------------------------------- lookup

struct LookupArgs {
  const void *table;   // already moved to the table's first element
  const void *tokens;
  void *out;
  long long ld, T;
  int V, D, token_bits;
  float scale;
  int xs;              // log2 of the threads of a CTA that share a row
};

__device__ __forceinline__ long long token_at(const void *tokens, int bits, long long i) {
  return bits == 64 ? __ldg(static_cast<const long long *>(tokens) + i) : (long long)__ldg(static_cast<const int *>(tokens) + i);
}

// A CTA is 2^xs threads across a row (units of VEC elements) by 256 >> xs rows; each thread takes kRows rows at once so
// that kRows independent row reads are in flight.
template <typename W, typename O, int VEC>
__global__ void __launch_bounds__(kThreads) k_embed_lookup(const LookupArgs a) {
  constexpr int kRows = 4;
  const int X = 1 << a.xs, Y = kThreads >> a.xs;
  const int tx = threadIdx.x & (X - 1), ty = threadIdx.x >> a.xs;
  const long long k = blockIdx.y, t0 = (long long)blockIdx.x * (Y * kRows) + ty;
  const W *table = static_cast<const W *>(a.table) + k * a.ld;
  O *out = static_cast<O *>(a.out) + k * a.T * a.D;
  const W *src[kRows];
  bool live[kRows], hit[kRows];
#pragma unroll
  for (int j = 0; j < kRows; ++j) {
    const long long t = t0 + (long long)j * Y;
    live[j] = t < a.T;
    const long long tok = live[j] ? token_at(a.tokens, a.token_bits, k * a.T + t) : -1;
    hit[j] = tok >= 0 && tok < a.V;
    src[j] = table + (hit[j] ? tok : 0) * a.D;
  }
  for (int c = tx * VEC; c < a.D; c += X * VEC) {
    float x[kRows][VEC];
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      if (hit[j]) {
        load<W, VEC>(src[j] + c, x[j]);
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) x[j][i] = 0.f;
      }
    }
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      if (!live[j]) continue;
#pragma unroll
      for (int i = 0; i < VEC; ++i) x[j][i] = hit[j] ? __fmul_rn(x[j][i], a.scale) : 0.f;
      store<O, VEC>(out + (t0 + (long long)j * Y) * a.D + c, x[j]);
    }
  }
}

// ---------------------------------------------------------------- sorting the tokens of a replica

struct SortArgs {
  const void *tokens;
  uint32_t *key[2], *pos[2];  // [K][T] each; the sorted result is in [passes & 1]
  uint8_t *met;               // [K][V]: 1 where the table's row is selected by some token
  long long T;
  int V, token_bits, passes, radix_bits;
};

// One cluster sorts one replica's tokens: a stable radix sort from the lowest digit up, `passes` digits of `radix_bits`
// bits.  Every CTA owns a contiguous part of the sequence and every warp a contiguous part of that, so the order within
// a digit is (CTA, warp, round, lane) = the order of the sequence.  Tokens outside the table get the key V and sort to
// the end.  All passes run in one launch: the digit counts cross CTAs through distributed shared memory, the keys
// through L2, and a cluster barrier (a fraction of a microsecond) stands where a launch boundary would.
__global__ void __launch_bounds__(kSortThreads) k_sort_tokens(const SortArgs a) {
  __shared__ uint32_t hist[kSortWarps][kMaxRadix];
  __shared__ uint32_t total[kMaxRadix];
  __shared__ uint32_t scan[kSortThreads / 32];
  cg::cluster_group cluster = cg::this_cluster();
  const int nC = cluster.num_blocks(), rank = cluster.block_rank();
  const long long k = blockIdx.x / nC;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int R = 1 << a.radix_bits;
  const uint32_t none = (uint32_t)a.V;
  const long long per = (a.T + nC - 1) / nC;                            // positions of a CTA
  const long long seg = ((per + kSortWarps - 1) / kSortWarps + 31) / 32 * 32;  // positions of a warp
  const long long lo = min(a.T, rank * per), hi = min(a.T, lo + per);
  const long long w0 = min(hi, lo + warp * seg), w1 = min(hi, w0 + seg);
  uint8_t *met = a.met + k * a.V;
  for (long long v = rank * (long long)kSortThreads + tid; v < a.V; v += (long long)nC * kSortThreads) met[v] = 0;

  for (int pass = 0; pass < a.passes; ++pass) {
    const uint32_t *kin = a.key[pass & 1] + k * a.T, *pin = a.pos[pass & 1] + k * a.T;
    uint32_t *kout = a.key[(pass & 1) ^ 1] + k * a.T, *pout = a.pos[(pass & 1) ^ 1] + k * a.T;
    const int shift = pass * a.radix_bits;
    auto key_at = [&](long long i) -> uint32_t {
      if (pass) return __ldcg(kin + i);
      const long long t = token_at(a.tokens, a.token_bits, k * a.T + i);
      return t >= 0 && t < a.V ? (uint32_t)t : none;
    };
    for (int d = lane; d < R; d += 32) hist[warp][d] = 0;
    __syncwarp();
    for (long long i = w0 + lane; i - lane < w1; i += 32) {
      const bool in = i < w1;
      const uint32_t d = in ? (key_at(i) >> shift) & (R - 1) : (uint32_t)R;
      const unsigned same = __match_any_sync(0xffffffffu, d);
      if (in && lane == __ffs(same) - 1) hist[warp][d] += __popc(same);
      __syncwarp();
    }
    __syncthreads();
    if (tid < R) {  // counts of the warps -> exclusive prefix over the warps, and the CTA's total
      uint32_t s = 0;
#pragma unroll
      for (int w = 0; w < kSortWarps; ++w) {
        const uint32_t c = hist[w][tid];
        hist[w][tid] = s;
        s += c;
      }
      total[tid] = s;
    }
    cluster.sync();
    uint32_t before = 0, all = 0;
    if (tid < R) {
      for (int c = 0; c < nC; ++c) {
        const uint32_t n = *cluster.map_shared_rank(&total[tid], c);
        all += n;
        if (c < rank) before += n;
      }
    }
    uint32_t incl = all;  // exclusive scan of `all` over the digits (threads beyond R hold 0)
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t n = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += n;
    }
    if (lane == 31) scan[warp] = incl;
    __syncthreads();
    uint32_t base = incl - all + before;
    for (int w = 0; w < warp; ++w) base += scan[w];
    if (tid < R)
#pragma unroll
      for (int w = 0; w < kSortWarps; ++w) hist[w][tid] += base;
    __syncthreads();
    for (long long i = w0 + lane; i - lane < w1; i += 32) {
      const bool in = i < w1;
      const uint32_t key = in ? key_at(i) : 0;
      const uint32_t d = in ? (key >> shift) & (R - 1) : (uint32_t)R;
      const unsigned same = __match_any_sync(0xffffffffu, d);
      if (in) {
        const uint32_t at = hist[warp][d] + __popc(same & ((1u << lane) - 1));
        kout[at] = key;
        pout[at] = pass ? __ldcg(pin + i) : (uint32_t)i;
      }
      __syncwarp();
      if (in && lane == __ffs(same) - 1) hist[warp][d] += __popc(same);
      __syncwarp();
    }
    cluster.sync();  // the next pass reads what other CTAs wrote, and `total` may be overwritten
  }
  const uint32_t *key = a.key[a.passes & 1] + k * a.T;
  for (long long i = lo + tid; i < hi; i += kSortThreads) {
    const uint32_t v = __ldcg(key + i);
    if (v != none && (i == 0 || __ldcg(key + i - 1) != v)) met[v] = 1;
  }
}

// ---------------------------------------------------------------- sums over the sorted tokens

struct GradArgs {
  const void *dy;             // [K][T][D]
  void *grad;                 // already moved to the table's first element
  const uint32_t *key, *pos;  // [K][T], sorted
  const uint8_t *met;         // [K][V]
  float *part;                // [K][blocks][2][D]: sums of runs that cross the borders of a block
  long long ld, T;
  int V, D, K;
  int blk;                    // sorted positions of a block, a multiple of 32
  int blocks, slices;         // blocks of a replica; column slices of a row
  long long sum_ctas;         // CTAs of the launch that sum; the ones after them write rows of zeros
  float scale;
  int accumulate;
};

template <typename G, int VEC>
__device__ __forceinline__ void write_row(const GradArgs &a, G *p, float (&x)[VEC]) {
  if (a.accumulate) {
    float old[VEC];
    load<G, VEC>(p, old);
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = fmaf(a.scale, x[i], old[i]);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = __fmul_rn(a.scale, x[i]);
  }
  store<G, VEC>(p, x);
}

constexpr int kSliceCols = 256;  // columns that a warp carries: 8 per lane
constexpr int kSumWarps = 4, kAhead = 4, kZeroRows = 32;

// A warp walks one block of the sorted tokens over one slice of columns, kAhead rows of dy in flight, and ends a sum
// wherever the token changes.  A run inside the block goes straight to the gradient; one that crosses a border leaves
// its sum in `part`: slot 0 when it began in an earlier block, slot 1 when it begins here and goes on.
template <typename Y, typename G, int VEC>
__device__ void sum_block(const GradArgs &a, long long task) {
  constexpr int NV = 8 / VEC;
  const int lane = threadIdx.x & 31;
  const int s = (int)(task % a.slices);
  const long long kb = task / a.slices;
  const int b = (int)(kb % a.blocks);
  const long long k = kb / a.blocks;
  const uint32_t none = (uint32_t)a.V;
  const uint32_t *key = a.key + k * a.T, *pos = a.pos + k * a.T;
  const Y *dy = static_cast<const Y *>(a.dy) + k * a.T * a.D;
  G *grad = static_cast<G *>(a.grad) + k * a.ld;
  float *part = a.part + (k * a.blocks + b) * 2 * a.D;
  const long long e0 = (long long)b * a.blk, e1 = min(a.T, e0 + a.blk);
  if (key[e0] == none) return;
  const uint32_t prev = e0 ? key[e0 - 1] : none, next = e1 < a.T ? key[e1] : none;
  const int c0 = s * kSliceCols + lane * VEC;
  bool col[NV];
#pragma unroll
  for (int u = 0; u < NV; ++u) col[u] = c0 + u * 32 * VEC < a.D;

  float acc[NV][VEC] = {};
  bool head = prev == key[e0];  // the first run of the block began earlier
  for (long long e = e0; e < e1; e += 32) {
    const int n = (int)min(32LL, e1 - e);
    const uint32_t kl = lane < n ? key[e + lane] : none, pl = lane < n ? pos[e + lane] : 0;
    uint32_t after = e + 32 < e1 ? key[e + 32] : none;  // the key that follows lane 31 inside the block
    for (int j0 = 0; j0 < n; j0 += kAhead) {
      float x[kAhead][NV][VEC];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const uint32_t kj = __shfl_sync(0xffffffffu, kl, j0 + j), pj = __shfl_sync(0xffffffffu, pl, j0 + j);
        const Y *row = dy + (long long)pj * a.D + c0;
#pragma unroll
        for (int u = 0; u < NV; ++u)
          if (kj != none && col[u]) load<Y, VEC>(row + u * 32 * VEC, x[j][u]);
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const uint32_t kj = __shfl_sync(0xffffffffu, kl, j0 + j);
        const uint32_t kn = __shfl_sync(0xffffffffu, kl, (j0 + j + 1) & 31);
        if (kj == none) continue;  // also the lanes past the end
#pragma unroll
        for (int u = 0; u < NV; ++u)
#pragma unroll
          for (int i = 0; i < VEC; ++i) acc[u][i] = __fadd_rn(acc[u][i], x[j][u][i]);
        const bool last = e + j0 + j == e1 - 1;
        const uint32_t follows = last ? none : (j0 + j == 31 ? after : kn);
        if (follows == kj) continue;
        const bool tail = last && next == kj;
#pragma unroll
        for (int u = 0; u < NV; ++u) {
          if (!col[u]) continue;
          const int c = c0 + u * 32 * VEC;
          if (head) store<float, VEC>(part + c, acc[u]);
          else if (tail) store<float, VEC>(part + a.D + c, acc[u]);
          else write_row<G, VEC>(a, grad + (long long)kj * a.D + c, acc[u]);
#pragma unroll
          for (int i = 0; i < VEC; ++i) acc[u][i] = 0.f;
        }
        head = false;
      }
    }
  }
}

template <typename Y, typename G, int VEC>
__global__ void __launch_bounds__(kSumWarps * 32) k_embed_sum(const GradArgs a) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (blockIdx.x < a.sum_ctas) {
    const long long task = (long long)blockIdx.x * kSumWarps + warp;
    if (task < (long long)a.K * a.blocks * a.slices) sum_block<Y, G, VEC>(a, task);
    return;
  }
  // rows that no token selects become zero
  const long long z = blockIdx.x - a.sum_ctas, per = (a.V + kZeroRows - 1) / kZeroRows;
  const long long k = z / per;
  const int v0 = (int)(z % per) * kZeroRows;
  const float zero[VEC] = {};
  for (int v = v0 + warp; v < min(a.V, v0 + kZeroRows); v += kSumWarps) {
    if (a.met[k * a.V + v]) continue;
    G *row = static_cast<G *>(a.grad) + k * a.ld + (long long)v * a.D;
    for (int c = lane * VEC; c < a.D; c += 32 * VEC) store<G, VEC>(row + c, zero);
  }
}

// The runs that cross blocks: one CTA for each block in which such a run begins, and 128 columns.  Its warps take every
// eighth partial sum, the eight sums are added in the order of the warps.
constexpr int kJoinWarps = 8, kJoinCols = 128;

template <typename G>
__global__ void __launch_bounds__(kJoinWarps * 32) k_embed_join(const GradArgs a) {
  __shared__ float sums[kJoinWarps][kJoinCols];
  const int b = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long k = blockIdx.z;
  const uint32_t *key = a.key + k * a.T;
  const long long e0 = (long long)b * a.blk, e1 = e0 + a.blk;
  if (e1 >= a.T) return;
  const uint32_t v = key[e1 - 1];
  if (v == (uint32_t)a.V || key[e1] != v || (key[e0] == v && e0 && key[e0 - 1] == v)) return;
  int n = 1;  // blocks after this one whose first run is this run; b + n is looked at next
  for (;; n += 32) {
    const long long e = (long long)(b + n + lane) * a.blk;
    const unsigned more = __ballot_sync(0xffffffffu, e < a.T && key[min(e, a.T - 1)] == v);
    if (more != 0xffffffffu) {
      n += __ffs(~more) - 1;
      break;
    }
  }
  const float *part = a.part + (k * a.blocks + b) * 2 * a.D;  // part 0: slot 1 of block b; part i: slot 0 of block b + i
  const int c = blockIdx.y * kJoinCols + lane;
  float acc[kJoinCols / 32] = {};
#pragma unroll 4
  for (int i = warp; i < n; i += kJoinWarps) {
    const float *p = part + (i ? (long long)i * 2 * a.D : (long long)a.D);
#pragma unroll
    for (int u = 0; u < kJoinCols / 32; ++u)
      if (c + 32 * u < a.D) acc[u] = __fadd_rn(acc[u], __ldg(p + c + 32 * u));
  }
#pragma unroll
  for (int u = 0; u < kJoinCols / 32; ++u) sums[warp][lane + 32 * u] = acc[u];
  __syncthreads();
  const int cc = blockIdx.y * kJoinCols + threadIdx.x;
  if (threadIdx.x < kJoinCols && cc < a.D) {
    float x[1] = {0.f};
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) x[0] = __fadd_rn(x[0], sums[w][threadIdx.x]);
    write_row<G, 1>(a, static_cast<G *>(a.grad) + k * a.ld + (long long)v * a.D + cc, x);
  }
}

// ---------------------------------------------------------------- host side

dasgd_status bad(const std::string &m) { return dasgd_internal_fail(nullptr, DASGD_ERR_INVALID_ARG, m.c_str()); }

dasgd_status check(const dasgd_embed_config *c, const char *who) {
  const std::string at = std::string(who) + ": ";
  if (!c) return bad(at + "cfg is NULL");
  if (c->K < 1 || c->K > 65535) return bad(at + "K must be in [1, 65535]");
  if (c->V < 1 || c->V == INT32_MAX) return bad(at + "V must be in [1, 2^31 - 2]");
  if (c->D < 1 || c->D > (1 << 22)) return bad(at + "D must be in [1, 2^22]");
  if (c->T < 0 || c->T >= (1LL << 31)) return bad(at + "T must be in [0, 2^31)");
  if (c->offset < 0 || c->ld < 1 || c->offset > c->ld || (int64_t)c->V * c->D > c->ld - c->offset)
    return bad(at + "the table must lie inside a row: offset >= 0, offset + V*D <= ld");
  if (c->token_bits != 32 && c->token_bits != 64) return bad(at + "token_bits must be 32 or 64");
  if ((c->table_elem | 1) != 1 || (c->rows_elem | 1) != 1) return bad(at + "unknown element type");
  if (c->device < 0) return bad(at + "device must be >= 0");
  return DASGD_OK;
}

size_t size_of(int elem) { return elem == DASGD_ELEM_BF16 ? 2 : 4; }
bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

struct OnDevice {
  int prev = -1;
  cudaError_t e;
  bool switched = false;
  explicit OnDevice(int dev) {
    e = cudaGetDevice(&prev);
    if (e == cudaSuccess && prev != dev) {
      e = cudaSetDevice(dev);
      switched = e == cudaSuccess;
    }
  }
  ~OnDevice() {
    if (switched) cudaSetDevice(prev);
  }
};

dasgd_status cuda_fail(cudaError_t e, const char *what) {
  return dasgd_internal_fail(nullptr, DASGD_ERR_CUDA, (std::string(what) + ": " + cudaGetErrorString(e)).c_str());
}

// units of 8 elements where every row of both arrays starts on a 16-byte boundary, single elements otherwise
bool wide(const dasgd_embed_config &c, const void *array, const void *rows) {
  return c.D % 8 == 0 && c.ld % 8 == 0 && c.offset % 8 == 0 && aligned(array, 16) && aligned(rows, 16);
}

struct Plan {  // of the gradient's workspace
  int blk, blocks, slices, passes, radix_bits, cluster;
  size_t key[2], pos[2], met, part, bytes;
};

constexpr int kBlkMax = 128, kBlkMin = 32, kEnoughWarps = 4096;

Plan plan(const dasgd_embed_config &c) {
  Plan p;
  p.slices = (c.D + kSliceCols - 1) / kSliceCols;
  auto blocks_of = [&](long long blk) { return (c.T + blk - 1) / blk; };
  p.blk = kBlkMax;
  while (p.blk > kBlkMin && c.K * blocks_of(p.blk) * p.slices < kEnoughWarps) p.blk /= 2;
  p.blocks = (int)blocks_of(p.blk);
  // the most blocks that c.T tokens or fewer can give: a block is shorter than kBlkMax only while blocks of twice its
  // length are fewer than kEnoughWarps / (K * slices)
  const long long few = (kEnoughWarps + (long long)c.K * p.slices - 1) / ((long long)c.K * p.slices);
  const long long most = std::max(blocks_of(kBlkMax), std::min(blocks_of(kBlkMin), 2 * few));
  int bits = 1;
  while (bits < 31 && (1LL << bits) <= c.V) ++bits;  // keys 0..V
  p.passes = (bits + kMaxRadixBits - 1) / kMaxRadixBits;
  p.radix_bits = (bits + p.passes - 1) / p.passes;
  p.cluster = c.T <= 1024 ? 1 : c.T <= 2048 ? 2 : c.T <= 4096 ? 4 : 8;
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t o = at;
    at += (n + 255) / 256 * 256;
    return o;
  };
  const size_t list = (size_t)c.K * c.T * 4;
  for (int i = 0; i < 2; ++i) p.key[i] = take(list), p.pos[i] = take(list);
  p.met = take((size_t)c.K * c.V);
  p.part = take((size_t)c.K * most * 2 * c.D * 4);
  p.bytes = at;
  return p;
}

template <typename W, typename O>
void launch_lookup(const dasgd_embed_config &c, LookupArgs a, bool vec, cudaStream_t s) {
  const int units = vec ? c.D / 8 : c.D;
  a.xs = 0;
  while (a.xs < 8 && (1 << a.xs) < units) ++a.xs;
  const int rows = (kThreads >> a.xs) * 4;
  const dim3 grid((unsigned)((c.T + rows - 1) / rows), (unsigned)c.K);
  if (vec) k_embed_lookup<W, O, 8><<<grid, kThreads, 0, s>>>(a);
  else k_embed_lookup<W, O, 1><<<grid, kThreads, 0, s>>>(a);
}

template <typename Y, typename G>
void launch_sum(const GradArgs &a, bool vec, long long ctas, cudaStream_t s) {
  if (vec) k_embed_sum<Y, G, 8><<<(unsigned)ctas, kSumWarps * 32, 0, s>>>(a);
  else k_embed_sum<Y, G, 1><<<(unsigned)ctas, kSumWarps * 32, 0, s>>>(a);
}

}  // namespace

extern "C" {

dasgd_status dasgd_embed_lookup(const dasgd_embed_config *cfg, const void *table_array, const void *tokens, void *out,
                                void *stream) {
  const dasgd_status st = check(cfg, "embed_lookup");
  if (st != DASGD_OK) return st;
  const dasgd_embed_config &c = *cfg;
  if (c.T == 0) return DASGD_OK;
  if (!table_array || !tokens || !out) return bad("embed_lookup: table_array, tokens and out must not be NULL");
  if (!aligned(table_array, size_of(c.table_elem)) || !aligned(out, size_of(c.rows_elem)) || !aligned(tokens, c.token_bits / 8))
    return bad("embed_lookup: buffers must be aligned to their elements");
  OnDevice dev(c.device);
  if (dev.e != cudaSuccess) return cuda_fail(dev.e, "embed_lookup");
  LookupArgs a{};
  a.table = static_cast<const char *>(table_array) + c.offset * size_of(c.table_elem);
  a.tokens = tokens;
  a.out = out;
  a.ld = c.ld, a.T = c.T, a.V = c.V, a.D = c.D, a.token_bits = c.token_bits, a.scale = c.scale;
  const bool vec = wide(c, table_array, out);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (c.table_elem == DASGD_ELEM_F32) {
    if (c.rows_elem == DASGD_ELEM_F32) launch_lookup<float, float>(c, a, vec, s);
    else launch_lookup<float, __nv_bfloat16>(c, a, vec, s);
  } else {
    if (c.rows_elem == DASGD_ELEM_F32) launch_lookup<__nv_bfloat16, float>(c, a, vec, s);
    else launch_lookup<__nv_bfloat16, __nv_bfloat16>(c, a, vec, s);
  }
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? DASGD_OK : cuda_fail(e, "embed_lookup");
}

dasgd_status dasgd_embed_workspace(const dasgd_embed_config *cfg, int64_t *bytes) {
  const dasgd_status st = check(cfg, "embed_workspace");
  if (st != DASGD_OK) return st;
  if (!bytes) return bad("embed_workspace: bytes is NULL");
  *bytes = (int64_t)plan(*cfg).bytes;
  return DASGD_OK;
}

dasgd_status dasgd_embed_gradient(const dasgd_embed_config *cfg, const void *dy, const void *tokens, void *grad_array,
                                  void *workspace, int64_t workspace_bytes, void *stream) {
  dasgd_status st = check(cfg, "embed_gradient");
  if (st != DASGD_OK) return st;
  const dasgd_embed_config &c = *cfg;
  const Plan p = plan(c);
  if (c.T == 0 && c.accumulate) return DASGD_OK;
  if (!grad_array || (c.T && (!dy || !tokens))) return bad("embed_gradient: dy, tokens and grad_array must not be NULL");
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < (int64_t)p.bytes)
    return bad("embed_gradient: needs a 256-byte aligned workspace of " + std::to_string(p.bytes) + " bytes");
  if (!aligned(grad_array, size_of(c.table_elem)) || !aligned(dy, size_of(c.rows_elem)) || !aligned(tokens, c.token_bits / 8))
    return bad("embed_gradient: buffers must be aligned to their elements");
  const long long zero_ctas = c.accumulate ? 0 : (long long)c.K * ((c.V + kZeroRows - 1) / kZeroRows);
  const long long sum_ctas = ((long long)c.K * p.blocks * p.slices + kSumWarps - 1) / kSumWarps;
  if (sum_ctas + zero_ctas > INT32_MAX || p.blocks > INT32_MAX / 2)
    return dasgd_internal_fail(nullptr, DASGD_ERR_UNSUPPORTED, "embed_gradient: K*V or K*T*D too large for one launch");
  OnDevice dev(c.device);
  if (dev.e != cudaSuccess) return cuda_fail(dev.e, "embed_gradient");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  char *ws = static_cast<char *>(workspace);

  SortArgs so{};
  so.tokens = tokens;
  for (int i = 0; i < 2; ++i) {
    so.key[i] = reinterpret_cast<uint32_t *>(ws + p.key[i]);
    so.pos[i] = reinterpret_cast<uint32_t *>(ws + p.pos[i]);
  }
  so.met = reinterpret_cast<uint8_t *>(ws + p.met);
  so.T = c.T, so.V = c.V, so.token_bits = c.token_bits, so.passes = p.passes, so.radix_bits = p.radix_bits;
  cudaLaunchConfig_t lc{};
  lc.gridDim = dim3((unsigned)(c.K * p.cluster));
  lc.blockDim = dim3(kSortThreads);
  lc.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = p.cluster, attr[0].val.clusterDim.y = 1, attr[0].val.clusterDim.z = 1;
  lc.attrs = attr, lc.numAttrs = 1;
  cudaError_t e = cudaLaunchKernelEx(&lc, k_sort_tokens, so);
  if (e != cudaSuccess) return cuda_fail(e, "embed_gradient: sort");

  GradArgs a{};
  a.dy = dy;
  a.grad = static_cast<char *>(grad_array) + c.offset * size_of(c.table_elem);
  a.key = so.key[p.passes & 1], a.pos = so.pos[p.passes & 1], a.met = so.met;
  a.part = reinterpret_cast<float *>(ws + p.part);
  a.ld = c.ld, a.T = c.T, a.V = c.V, a.D = c.D, a.K = c.K, a.blk = p.blk, a.blocks = p.blocks, a.slices = p.slices;
  a.sum_ctas = sum_ctas, a.scale = c.scale, a.accumulate = c.accumulate != 0;
  const bool vec = wide(c, grad_array, dy);
  const bool y32 = c.rows_elem == DASGD_ELEM_F32, g32 = c.table_elem == DASGD_ELEM_F32;
  if (y32 && g32) launch_sum<float, float>(a, vec, sum_ctas + zero_ctas, s);
  else if (y32) launch_sum<float, __nv_bfloat16>(a, vec, sum_ctas + zero_ctas, s);
  else if (g32) launch_sum<__nv_bfloat16, float>(a, vec, sum_ctas + zero_ctas, s);
  else launch_sum<__nv_bfloat16, __nv_bfloat16>(a, vec, sum_ctas + zero_ctas, s);
  if (p.blocks > 1) {
    const dim3 grid((unsigned)(p.blocks - 1), (unsigned)((c.D + kJoinCols - 1) / kJoinCols), (unsigned)c.K);
    if (g32) k_embed_join<float><<<grid, kJoinWarps * 32, 0, s>>>(a);
    else k_embed_join<__nv_bfloat16><<<grid, kJoinWarps * 32, 0, s>>>(a);
  }
  e = cudaGetLastError();
  return e == cudaSuccess ? DASGD_OK : cuda_fail(e, "embed_gradient");
}

}  // extern "C"
