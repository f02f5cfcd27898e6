// Tokens sorted by expert and back: the plan (a stable counting sort of the choices), the dispatch of rows, the weighted
// combine and its gradient.  All of it moves memory: the floor of each call is its bytes at the copy rate.
#include "internal.h"

#include <limits.h>

namespace ecmoe {

namespace {

// ---- the plan ----------------------------------------------------------------------------------------------
// A counting sort.  The flat choices are cut into one contiguous piece per CTA and those into one per warp; a choice's row is
//   offsets[e] + (choices of e in earlier pieces) + (in earlier warps of this piece) + (earlier in this warp),
// all of them plain counts, so the order is the stable one and unique.  A warp ranks 32 choices at a time: the lanes with the
// same expert find each other by one vote per bit of its number (a match instruction takes three times as long), the lowest of them
// adds their number to the warp's own row of counters in shared memory.
// Up to kOnePiece choices one CTA does it all, up to kClusterMost the eight of a cluster, which read each other's counts in shared
// memory; beyond, a first launch leaves each piece's counts and, in `place`, ranks inside the piece, and in a second each CTA sums what it
// needs of the counts (148 x 256 at most, 148 KiB out of L2) and adds.
// Latency bounds it, its bytes being a few microseconds' at most: 128 choices 2.7 us, 2048 4.4, 16384 5.2 (two launches 6.4, one CTA 11), 32768 7.1
// (a cluster 7.5), 524288 of 256 experts 16.
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32, kMaxExperts = 256, kClusterCtas = 8;
constexpr int64_t kOnePiece = 2048, kClusterMost = 24576;
constexpr int kMaxPieces = 148;
constexpr int kHeld = 4;                              // rounds of 32 choices whose ranks a warp keeps in registers
enum { ONE_CTA, ONE_CLUSTER, TWO_LAUNCHES };

struct SortArgs {
  const int32_t* choice; int32_t* offsets; int32_t* order; int32_t* place; int* status; int* counts;   // counts [pieces, E]
  int64_t total, per_cta;                                                                  // flat choices; per_cta a multiple of 1024
  int E, bits, pieces;                                                                     // bits: of an expert's number
};

// One round: the number of earlier choices of the same expert in the warp's stretch, counters moved on.
__device__ __forceinline__ int rank_round(int e, bool in, int bits, int* mine, int lane) {
  unsigned peers = __ballot_sync(0xffffffffu, in);
  for (int b = 0; b < bits; ++b) {
    const bool one = (e >> b) & 1;
    const unsigned with = __ballot_sync(0xffffffffu, one);
    peers &= one ? with : ~with;
  }
  const int before = __popc(peers & ((1u << lane) - 1));
  const int at = in ? mine[e] + before : -1;
  __syncwarp();
  if (in && before == 0) mine[e] += __popc(peers);
  __syncwarp();
  return at;
}

// Exclusive sums of v over the 256 threads with part = 0 (in order of e); every thread of the CTA calls it.
__device__ __forceinline__ int scan_experts(int v, int part, int warp, int lane, int* warp_sum) {
  int incl = v;
#pragma unroll
  for (int o = 1; o < 32; o *= 2) { const int u = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += u; }
  if (part == 0 && lane == 31) warp_sum[warp] = incl;
  __syncthreads();
  int first = incl - v;
  if (part == 0) for (int w = 0; w < warp; ++w) first += warp_sum[w];
  return first;
}

template <int HOW>
__global__ void __launch_bounds__(kSortThreads) sort_rank_kernel(const SortArgs a) {
  __shared__ int counters[kSortWarps][kMaxExperts];
  __shared__ int parts[4][kMaxExperts], earlier[4][kMaxExperts];         // per expert: of eight warps each; of the cluster's pieces in four parts
  __shared__ int own[kMaxExperts], start[kMaxExperts], warp_sum[kMaxExperts / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, E = a.E;
  for (int e = lane; e < E; e += 32) counters[warp][e] = 0;
  __syncwarp();
  chain_enter();
  if (blockIdx.x == 0 && threadIdx.x == kSortThreads - 1) begin_status(a.status);
  const int32_t* choice = after_enter(a.choice);
  const int64_t per_warp = a.per_cta / kSortWarps, lo = blockIdx.x * a.per_cta + warp * per_warp, hi = min(lo + per_warp, a.total);
  int* mine = counters[warp];
  int held_e[kHeld], held[kHeld];
#pragma unroll
  for (int u = 0; u < kHeld; ++u) { const int64_t at = lo + 32 * u + lane; held_e[u] = at < hi ? __ldg(choice + at) : -1; }
#pragma unroll
  for (int u = 0; u < kHeld; ++u) if (lo + 32 * u < hi) held[u] = rank_round(held_e[u], (unsigned)held_e[u] < (unsigned)E, a.bits, mine, lane);
  for (int64_t i = lo + 32 * kHeld; i < hi; i += 32 * kHeld) {           // the ranks of later rounds wait in `place`
    int e[kHeld];
#pragma unroll
    for (int u = 0; u < kHeld; ++u) { const int64_t at = i + 32 * u + lane; e[u] = at < hi ? __ldg(choice + at) : -1; }
#pragma unroll
    for (int u = 0; u < kHeld; ++u) {
      if (i + 32 * u >= hi) break;
      const int64_t at = i + 32 * u + lane;
      const int r = rank_round(e[u], (unsigned)e[u] < (unsigned)E, a.bits, mine, lane);
      if (at < hi) a.place[at] = r;
    }
  }
  __syncthreads();
  // per expert, exclusive sums over the warps, eight to a thread
  const int e = threadIdx.x & (kMaxExperts - 1), part = threadIdx.x / kMaxExperts;
  int c[8], sum = 0;
  if (e < E)
#pragma unroll
    for (int w = 0; w < 8; ++w) { c[w] = counters[part * 8 + w][e]; sum += c[w]; }
  parts[part][e] = sum;
  __syncthreads();
  int piece = 0, base = 0;                            // of the whole piece; of the parts before
#pragma unroll
  for (int q = 0; q < 4; ++q) { piece += parts[q][e]; if (q < part) base += parts[q][e]; }
  if (HOW == TWO_LAUNCHES && part == 0 && e < E) a.counts[(int64_t)blockIdx.x * E + e] = piece;
  int first = 0;                                      // part 0: the expert's first row in this piece
  if constexpr (HOW == ONE_CLUSTER) {
    if (part == 0) own[e] = piece;
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
    int before = 0, all = 0;
#pragma unroll
    for (int q = 0; q < kClusterCtas / 4; ++q) {
      const int p = part + 4 * q;
      uint32_t there;
      int n;
      asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"((uint32_t)__cvta_generic_to_shared(own + e)), "r"(p));
      asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(n) : "r"(there) : "memory");
      all += n;
      if (p < (int)blockIdx.x) before += n;
    }
    // nobody leaves while its counts are read: arrived here, waited for at the end
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    earlier[part][e] = before;
    __syncthreads();                                  // parts has been read
    parts[part][e] = all;
    __syncthreads();
    if (part == 0) { all = parts[0][e] + parts[1][e] + parts[2][e] + parts[3][e]; before = earlier[0][e] + earlier[1][e] + earlier[2][e] + earlier[3][e]; }
    first = scan_experts(all, part, warp, lane, warp_sum);
    if (part == 0) {
      if (blockIdx.x == 0 && e < E) { a.offsets[e] = first; if (e == E - 1) a.offsets[E] = first + all; }
      start[e] = first + before;
    }
  } else if constexpr (HOW == ONE_CTA) {
    first = scan_experts(piece, part, warp, lane, warp_sum);
    if (part == 0) {
      if (e < E) { a.offsets[e] = first; if (e == E - 1) a.offsets[E] = first + piece; }
      start[e] = first;
    }
  } else {
    if (part == 0) start[e] = 0;
  }
  __syncthreads();
  if (e < E) {
    base += start[e];
#pragma unroll
    for (int w = 0; w < 8; ++w) { counters[part * 8 + w][e] = base; base += c[w]; }
  }
  __syncthreads();
  auto put = [&](int64_t at, int x, int r) {
    if (at >= hi) return;
    const int row = r < 0 ? -1 : r + mine[x];
    a.place[at] = row;
    if (HOW != TWO_LAUNCHES && row >= 0) a.order[row] = (int)at;
  };
#pragma unroll
  for (int u = 0; u < kHeld; ++u) if (lo + 32 * u < hi) put(lo + 32 * u + lane, held_e[u], held[u]);
  for (int64_t i = lo + 32 * kHeld; i < hi; i += 32 * kHeld) {
    int x[kHeld], r[kHeld];
#pragma unroll
    for (int u = 0; u < kHeld; ++u) { const int64_t at = i + 32 * u + lane; if (at < hi) { x[u] = __ldg(choice + at); r[u] = a.place[at]; } }
#pragma unroll
    for (int u = 0; u < kHeld; ++u) put(i + 32 * u + lane, x[u], r[u]);
  }
  if constexpr (HOW == ONE_CLUSTER) {
    __syncwarp();                                     // the lanes took different ways through put(); .aligned wants the warp together
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
}

__global__ void __launch_bounds__(kSortThreads) sort_shift_kernel(const SortArgs a) {
  __shared__ int before[4][kMaxExperts], all[4][kMaxExperts];            // of the pieces, in four parts
  __shared__ int start[kMaxExperts], warp_sum[kMaxExperts / 32];
  chain_enter();
  const int32_t* choice = after_enter(a.choice);
  const int* counts = after_enter((const int*)a.counts);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, E = a.E, e = threadIdx.x & (kMaxExperts - 1), part = threadIdx.x / kMaxExperts;
  int b = 0, t = 0;
  if (e < E)
#pragma unroll 16
    for (int p = part; p < a.pieces; p += 4) { const int c = __ldg(counts + (int64_t)p * E + e); t += c; if (p < (int)blockIdx.x) b += c; }
  before[part][e] = b; all[part][e] = t;
  __syncthreads();
  int total = 0;
  if (part == 0) { total = all[0][e] + all[1][e] + all[2][e] + all[3][e]; b = before[0][e] + before[1][e] + before[2][e] + before[3][e]; }
  const int first = scan_experts(total, part, warp, lane, warp_sum);
  if (part == 0) {
    if (blockIdx.x == 0 && e < E) { a.offsets[e] = first; if (e == E - 1) a.offsets[E] = first + total; }
    start[e] = first + b;
  }
  __syncthreads();
  const int64_t lo = blockIdx.x * a.per_cta, hi = min(lo + a.per_cta, a.total);
  constexpr int U = 4;
  for (int64_t i = lo + threadIdx.x; i < hi; i += kSortThreads * U) {
    int x[U], r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) { const int64_t at = i + kSortThreads * u; if (at < hi) { x[u] = __ldg(choice + at); r[u] = a.place[at]; } }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = i + kSortThreads * u;
      if (at >= hi || r[u] < 0) continue;             // without an expert: -1 already
      const int row = r[u] + start[x[u]];
      a.place[at] = row;
      a.order[row] = (int)at;
    }
  }
}

// ---- rows ------------------------------------------------------------------------------------------------
// A work item is a token's stretch of kPieces 16-byte pieces per lane, by a group of G lanes (8, 16 or 32: narrow rows share a
// warp), so a few long rows occupy the card as well as many short ones.  Every piece of X is read once, by the token's item,
// whatever the number of its rows.  Memory bounds it: 16384 x 4096 bf16, two rows per token, 62 us, 6.5 TB/s (99 % of the copy rate);
// 65536 x 1024, eight rows, 190 us, 97 %; 8192 x 768 fp32 12.9 us.
template <int G, int kPieces>
__global__ void __launch_bounds__(256) dispatch_kernel(const uint4* X, const int32_t* place, uint4* X_s, int64_t items, int stretches, int pieces, int K,
                                                       int64_t rows) {
  chain_enter();
  const uint4* x = after_enter(X);
  const int32_t* pl = after_enter(place);
  const int lane = threadIdx.x % G;
  for (int64_t it = ((int64_t)blockIdx.x * 256 + threadIdx.x) / G; it < items; it += (int64_t)gridDim.x * 256 / G) {
    const int64_t t = it / stretches;
    const int p0 = (int)(it - t * stretches) * (G * kPieces) + lane;
    uint4 v[kPieces];
#pragma unroll
    for (int u = 0; u < kPieces; ++u) if (p0 + u * G < pieces) v[u] = __ldg(x + t * pieces + p0 + u * G);
#pragma unroll 4
    for (int j = 0; j < K; ++j) {
      const int r = __ldg(pl + t * K + j);
      if ((unsigned)r >= (unsigned)rows) continue;
      uint4* out = X_s + (int64_t)r * pieces;
#pragma unroll
      for (int u = 0; u < kPieces; ++u) if (p0 + u * G < pieces) out[p0 + u * G] = v[u];
    }
  }
}

// A 16-byte piece of Y is V values; the same V values of X_out or dX_out are 16 bytes, or 8 where Y is fp32 and they are bf16.
template <typename T> struct Vec { static constexpr int V = 16 / sizeof(T); };
template <typename T, int V> struct Pack;
template <> struct Pack<float, 4> { using type = uint4; };
template <> struct Pack<bf16, 8> { using type = uint4; };
template <> struct Pack<bf16, 4> { using type = uint2; };

__device__ __forceinline__ void unpack_word(unsigned w, float& a, float& b) { a = __uint_as_float(w << 16); b = __uint_as_float(w & 0xFFFF0000u); }
template <typename T, int V> __device__ __forceinline__ void unpack(const typename Pack<T, V>::type& p, float* f) {
  const unsigned* w = reinterpret_cast<const unsigned*>(&p);
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = __uint_as_float(w[i]);
  } else {
#pragma unroll
    for (int i = 0; i < V / 2; ++i) unpack_word(w[i], f[2 * i], f[2 * i + 1]);
  }
}
template <typename T, int V> __device__ __forceinline__ typename Pack<T, V>::type pack(const float* f) {
  typename Pack<T, V>::type p;
  unsigned* w = reinterpret_cast<unsigned*>(&p);
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < V; ++i) w[i] = __float_as_uint(f[i]);
  } else {
#pragma unroll
    for (int i = 0; i < V / 2; ++i) { __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]); w[i] = *reinterpret_cast<unsigned*>(&h); }
  }
  return p;
}

// KB rows of a token are on their way at a time, kPieces pieces of each; the sum runs over j in ascending order, in fp32, and is rounded once.
// Memory bounds it, short rows the latency of place -> row: 16384 x 4096 bf16, two rows, 68 us (91 % of the copy rate); 65536 x 1024,
// eight rows, 194 us (95 %); 8192 x 768 fp32 13.7 us (84 %); 6079 x 1000, three rows, 13.1 us (57 %); 262144 x 64, two, 24 us (64 %; with
// room for four rows, whose registers hold up to a third of the warps, 31).
template <typename T, typename TY, int G, int kPieces, int KB>
__global__ void __launch_bounds__(256, G < 32 && KB == 2 ? 6 : 0) combine_rows_kernel(const uint4* Y, const float* weights, const int32_t* place, void* X_out, int64_t items,
                                                           int stretches, int pieces, int K, int64_t rows) {
  constexpr int V = Vec<TY>::V;
  using Out = typename Pack<T, V>::type;
  chain_enter();
  const uint4* y = after_enter(Y);
  const float* ws = after_enter(weights);
  const int32_t* pl = after_enter(place);
  const int lane = threadIdx.x % G;
  for (int64_t it = ((int64_t)blockIdx.x * 256 + threadIdx.x) / G; it < items; it += (int64_t)gridDim.x * 256 / G) {
    const int64_t t = it / stretches;
    const int p0 = (int)(it - t * stretches) * (G * kPieces) + lane;
    float acc[kPieces][V];
#pragma unroll
    for (int u = 0; u < kPieces; ++u)
#pragma unroll
      for (int i = 0; i < V; ++i) acc[u][i] = 0.f;
    for (int j0 = 0; j0 < K; j0 += KB) {
      int r[KB]; float w[KB]; uint4 v[KB][kPieces];
#pragma unroll
      for (int j = 0; j < KB; ++j) {
        r[j] = j0 + j < K ? __ldg(pl + t * K + j0 + j) : -1;
        w[j] = j0 + j < K && ws != nullptr ? __ldg(ws + t * K + j0 + j) : 1.f;
      }
#pragma unroll
      for (int j = 0; j < KB; ++j)
#pragma unroll
        for (int u = 0; u < kPieces; ++u)
          if ((unsigned)r[j] < (unsigned)rows && p0 + u * G < pieces) v[j][u] = __ldg(y + (int64_t)r[j] * pieces + p0 + u * G);
#pragma unroll
      for (int j = 0; j < KB; ++j) {
        if ((unsigned)r[j] >= (unsigned)rows) continue;
#pragma unroll
        for (int u = 0; u < kPieces; ++u) {
          float f[V];
          unpack<TY, V>(v[j][u], f);
#pragma unroll
          for (int i = 0; i < V; ++i) acc[u][i] = fmaf(w[j], f[i], acc[u][i]);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kPieces; ++u) if (p0 + u * G < pieces) ((Out*)X_out)[t * pieces + p0 + u * G] = pack<T, V>(acc[u]);
  }
}

// A token is the work of G lanes, or of WPT warps of a CTA (G = 32): they share its pieces, so that dX_out is read once for KB of the
// token's rows, and the dot products' parts are joined in a fixed order: lanes by halves, then the warps in turn.  One pass gives dY and
// the weights' gradient.  Memory bounds it, with eight to twelve loads on their way per lane: 16384 x 4096 bf16, two rows, 103 us (99 % of the
// copy rate; with half as many loads 137); 65536 x 1024, eight rows, 358 us (97 %; 470); 262144 x 64 34 us (with a warp per token 141).
template <typename T, typename TY, int G, int WPT, int KB, int U>
__global__ void __launch_bounds__(256) combine_backward_kernel(const void* dX_out, const uint4* Y, const float* weights, const int32_t* place, uint4* dY,
                                                               float* dweights, int64_t n, int pieces, int K, int64_t rows) {
  static_assert(G == 32 || WPT == 1, "lanes of a warp, or warps");
  constexpr int V = Vec<TY>::V, kLanes = G * WPT, kTokens = 256 / kLanes;
  using In = typename Pack<T, V>::type;
  __shared__ float parts[8][KB];
  chain_enter();
  const In* g = after_enter((const In*)dX_out);
  const uint4* y = after_enter(Y);
  const float* ws = after_enter(weights);
  const int32_t* pl = after_enter(place);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x % G, sub = threadIdx.x % kLanes;
  for (int64_t t0 = (int64_t)blockIdx.x * kTokens; t0 < n; t0 += (int64_t)gridDim.x * kTokens) {       // the same for the whole CTA
    const int64_t t = t0 + threadIdx.x / kLanes;
    const bool live = t < n;
    for (int j0 = 0; j0 < K; j0 += KB) {
      int r[KB]; float w[KB], dot[KB];
#pragma unroll
      for (int j = 0; j < KB; ++j) {
        r[j] = live && j0 + j < K ? __ldg(pl + t * K + j0 + j) : -1;
        w[j] = live && j0 + j < K ? __ldg(ws + t * K + j0 + j) : 0.f;
        if ((unsigned)r[j] >= (unsigned)rows) r[j] = -1;
        dot[j] = 0.f;
      }
      if (live) {
        for (int p0 = sub; p0 < pieces; p0 += kLanes * U) {
          In gp[U]; uint4 v[U][KB];
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int p = p0 + u * kLanes;
            if (p >= pieces) continue;
            gp[u] = __ldg(g + t * pieces + p);
#pragma unroll
            for (int j = 0; j < KB; ++j) if (r[j] >= 0) v[u][j] = __ldg(y + (int64_t)r[j] * pieces + p);
          }
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int p = p0 + u * kLanes;
            if (p >= pieces) continue;
            float a[V];
            unpack<T, V>(gp[u], a);
#pragma unroll
            for (int j = 0; j < KB; ++j) {
              if (r[j] < 0) continue;
              float f[V], o[V];
              unpack<TY, V>(v[u][j], f);
#pragma unroll
              for (int i = 0; i < V; ++i) { dot[j] = fmaf(a[i], f[i], dot[j]); o[i] = w[j] * a[i]; }
              dY[(int64_t)r[j] * pieces + p] = pack<TY, V>(o);
            }
          }
        }
      }
#pragma unroll
      for (int j = 0; j < KB; ++j)
#pragma unroll
        for (int o = G / 2; o > 0; o >>= 1) dot[j] += __shfl_xor_sync(0xffffffffu, dot[j], o);
      if constexpr (WPT == 1) {
#pragma unroll
        for (int j = 0; j < KB; ++j) if (live && lane == j && j0 + j < K) dweights[t * K + j0 + j] = dot[j];
      } else {
        if (lane == 0)
#pragma unroll
          for (int j = 0; j < KB; ++j) parts[warp][j] = dot[j];
        __syncthreads();
        if (live && sub < KB && j0 + sub < K) {
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < WPT; ++i) sum += parts[warp + i][sub];
          dweights[t * K + j0 + sub] = sum;
        }
        __syncthreads();
      }
    }
  }
}

int device_sms() {
  int dev = 0, sms = 148;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return sms;
}

// Lanes per stretch: a warp for rows of 32 pieces and more
int group_of(int pieces) { return pieces > 16 ? 32 : pieces > 8 ? 16 : 8; }
unsigned item_grid(int64_t items, int group, int sms) {
  const int64_t ctas = (items * group + 255) / 256, most = (int64_t)sms * 64;
  return (unsigned)(ctas < most ? ctas : most);
}

template <int G>
cudaError_t dispatch_with(const void* X, const int32_t* place, void* X_s, int64_t n, int pieces, int K, int sms, cudaStream_t st) {
  constexpr int kPieces = 4;
  const int stretches = (pieces + G * kPieces - 1) / (G * kPieces);
  const int64_t items = n * stretches;
  return launch_chained(dispatch_kernel<G, kPieces>, dim3(item_grid(items, G, sms)), dim3(256), 0, st, (const uint4*)X, place, (uint4*)X_s, items, stretches,
                        pieces, K, n * K);
}

template <typename T, typename TY, int G, int kPieces, int KB>
cudaError_t combine_with(const void* Y, const float* w, const int32_t* place, void* X_out, int64_t n, int pieces, int K, cudaStream_t st) {
  const int stretches = (pieces + G * kPieces - 1) / (G * kPieces);
  const int64_t items = n * stretches;
  return launch_chained(combine_rows_kernel<T, TY, G, kPieces, KB>, dim3(item_grid(items, G, device_sms())), dim3(256), 0, st, (const uint4*)Y, w, place, X_out,
                        items, stretches, pieces, K, n * K);
}
// Four 16-byte loads on their way per lane: the pieces of one row, of two, or one piece of four (measured against twice as many, which
// cost the registers of a third of the warps: 16384 x 4096 bf16, two rows per token, 68 us and 77; 65536 x 1024, eight rows, 194 and 209;
// 4096 x 8192, one row, four pieces 25.6, two 33.6).
template <typename T, typename TY>
cudaError_t combine_of(const void* Y, const float* w, const int32_t* place, void* X_out, int64_t n, int d, int K, cudaStream_t st) {
  const int pieces = d / Vec<TY>::V;
  // narrow rows, two to a token: 65536 x 120 bf16 12.9 us by twos, 16.5 by fours; three: 65536 x 64 fp32 16.7 and 15.0; four: 262144 x 64 35.4 and 35.7
  switch (group_of(pieces)) {
    case 8: return K <= 2 ? combine_with<T, TY, 8, 1, 2>(Y, w, place, X_out, n, pieces, K, st) : combine_with<T, TY, 8, 1, 4>(Y, w, place, X_out, n, pieces, K, st);
    case 16: return K <= 2 ? combine_with<T, TY, 16, 1, 2>(Y, w, place, X_out, n, pieces, K, st) : combine_with<T, TY, 16, 1, 4>(Y, w, place, X_out, n, pieces, K, st);
  }
  if (K == 1) return combine_with<T, TY, 32, 4, 1>(Y, w, place, X_out, n, pieces, K, st);
  return K == 2 ? combine_with<T, TY, 32, 2, 2>(Y, w, place, X_out, n, pieces, K, st) : combine_with<T, TY, 32, 1, 4>(Y, w, place, X_out, n, pieces, K, st);
}

template <typename T, typename TY, int G, int WPT, int KB, int U>
cudaError_t backward_with(const void* dX_out, const void* Y, const float* w, const int32_t* place, void* dY, float* dw, int64_t n, int pieces, int K,
                          cudaStream_t st) {
  const int64_t ctas = (n * G * WPT + 255) / 256, most = (int64_t)device_sms() * 8;
  return launch_chained(combine_backward_kernel<T, TY, G, WPT, KB, U>, dim3((unsigned)(ctas < most ? ctas : most)), dim3(256), 0, st, dX_out, (const uint4*)Y, w,
                        place, (uint4*)dY, dw, n, pieces, K, n * K);
}
template <typename T, typename TY, int KB, int U>
cudaError_t backward_rows(const void* dX_out, const void* Y, const float* w, const int32_t* place, void* dY, float* dw, int64_t n, int pieces, int K,
                          cudaStream_t st) {
  switch (group_of(pieces)) {
    case 8: return backward_with<T, TY, 8, 1, KB, 1>(dX_out, Y, w, place, dY, dw, n, pieces, K, st);
    case 16: return backward_with<T, TY, 16, 1, KB, 1>(dX_out, Y, w, place, dY, dw, n, pieces, K, st);
  }
  if (pieces <= 64) return backward_with<T, TY, 32, 1, KB, U>(dX_out, Y, w, place, dY, dw, n, pieces, K, st);
  if (pieces <= 256) return backward_with<T, TY, 32, 2, KB, U>(dX_out, Y, w, place, dY, dw, n, pieces, K, st);
  return backward_with<T, TY, 32, 4, KB, U>(dX_out, Y, w, place, dY, dw, n, pieces, K, st);
}
template <typename T, typename TY>
cudaError_t backward_of(const void* dX_out, const void* Y, const float* w, const int32_t* place, void* dY, float* dw, int64_t n, int d, int K, cudaStream_t st) {
  const int pieces = d / Vec<TY>::V;
  return K <= 2 ? backward_rows<T, TY, 2, 4>(dX_out, Y, w, place, dY, dw, n, pieces, K, st) : backward_rows<T, TY, 4, 2>(dX_out, Y, w, place, dY, dw, n, pieces, K, st);
}

}  // namespace

size_t sort_scratch_bytes(int E) { return sizeof(StatusWord) + (size_t)kMaxPieces * E * 4; }

cudaError_t launch_sort_tokens(const int32_t* choice, int64_t total, int E, int32_t* offsets, int32_t* order, int32_t* place, void* scratch, cudaStream_t st) {
  SortArgs a{choice, offsets, order, place, (int*)scratch, (int*)((char*)scratch + sizeof(StatusWord)), total, 0, E, 0, 1};
  while ((1 << a.bits) < E) ++a.bits;
  auto cut = [&](int ctas) { a.per_cta = ((total + ctas - 1) / ctas + 1023) / 1024 * 1024; };
  if (total <= kOnePiece) {
    cut(1);
    return launch_chained(sort_rank_kernel<ONE_CTA>, dim3(1), dim3(kSortThreads), 0, st, a);
  }
  if (total <= kClusterMost) {                        // the last CTAs may have no choices
    cut(kClusterCtas);
    return launch_chained_cluster(kClusterCtas, sort_rank_kernel<ONE_CLUSTER>, dim3(kClusterCtas), dim3(kSortThreads), 0, st, a);
  }
  cut(kMaxPieces);
  a.pieces = (int)((total + a.per_cta - 1) / a.per_cta);
  const cudaError_t e = launch_chained(sort_rank_kernel<TWO_LAUNCHES>, dim3(a.pieces), dim3(kSortThreads), 0, st, a);
  return e != cudaSuccess ? e : launch_chained(sort_shift_kernel, dim3(a.pieces), dim3(kSortThreads), 0, st, a);
}

cudaError_t launch_dispatch(const void* X, const int32_t* place, void* X_s, int64_t n, int64_t row_bytes, int K, cudaStream_t st) {
  const int pieces = (int)(row_bytes / 16), sms = device_sms();
  switch (group_of(pieces)) {
    case 32: return dispatch_with<32>(X, place, X_s, n, pieces, K, sms, st);
    case 16: return dispatch_with<16>(X, place, X_s, n, pieces, K, sms, st);
    default: return dispatch_with<8>(X, place, X_s, n, pieces, K, sms, st);
  }
}

cudaError_t launch_combine_rows(int dtype, int y_dtype, const void* Y, const float* weights, const int32_t* place, void* X_out, int64_t n, int d, int K,
                                cudaStream_t st) {
  if (dtype == 0) return combine_of<float, float>(Y, weights, place, X_out, n, d, K, st);
  return y_dtype == 0 ? combine_of<bf16, float>(Y, weights, place, X_out, n, d, K, st) : combine_of<bf16, bf16>(Y, weights, place, X_out, n, d, K, st);
}

cudaError_t launch_combine_backward(int dtype, int y_dtype, const void* dX_out, const void* Y, const float* weights, const int32_t* place, void* dY,
                                    float* dweights, int64_t n, int d, int K, cudaStream_t st) {
  if (dtype == 0) return backward_of<float, float>(dX_out, Y, weights, place, dY, dweights, n, d, K, st);
  return y_dtype == 0 ? backward_of<bf16, float>(dX_out, Y, weights, place, dY, dweights, n, d, K, st)
                      : backward_of<bf16, bf16>(dX_out, Y, weights, place, dY, dweights, n, d, K, st);
}

}  // namespace ecmoe
