// What the two decode kernels share: how the rows of all heads are spread over CTAs and how partial results are joined.
//
// The heads of a compressed cache have different lengths, known only on the device.  Every item (sequence, KV head,
// chunk of its query heads) is cut into tiles of TILE rows; the tiles of all items in order are one long list, and CTA
// i of n takes the i-th n-th of it: equal work whatever the lengths are.  A range may end in the middle of an item, so
// a CTA has at most two incomplete items: the one its range begins inside (partial slot 0) and the one that begins in
// the range and goes on behind it (slot 1).  Their unnormalised sums with the running maximum and sum go to the
// workspace; decode_join_kernel adds them up in CTA order, so equal inputs give equal bits.
//
// Items of few tiles (by the size of the page table) are instead given to a CTA each or, where they are few, to a team of
// CTAs each, a thread-block cluster whose parts meet in distributed shared memory: one launch instead of two.
#pragma once
#include <cuda_bf16.h>

#include <atomic>

#include "launch_early.cuh"
#include "paged_common.cuh"

namespace ckv {

constexpr int kDecodeThreads = 128;
constexpr int kDecodeWarps = kDecodeThreads / 32;
constexpr int kDecodeMaxCtas = 592;      // four a multiprocessor on 148
constexpr int kJoinThreads = 256, kLongJoinThreads = 1024;
constexpr int kLongJoinParts = 16;       // CTAs an item from which the long join is taken
constexpr int kMaxTeam = 16;             // CTAs that share an item where items have teams, at most

struct DecodeArgs {
  Pages c;
  const char* q;
  long long qs[2];             // byte strides: sequence, head
  const int32_t* lens;
  char* out;                   // [nseq, Hq, dh] dense
  float* lse;                  // [nseq, Hq] or null
  float* part;                 // [CTA][2][rows of an item][dh + 2]: sums, maximum (base 2), sum of weights
  int2* join;                  // [CTA]: item that ends in this CTA and began in an earlier one (or -1), its first CTA
  int items, Hq, G;            // G = Hq / Hkv
  int chunks, chunk_rows;      // query heads of a KV head: chunks of at most chunk_rows
  int part_rows;               // the most query heads an item has
  int team;                    // item i is the cluster's of CTAs i * team ..., or a CTA's (1); 0: all items are one list
  int allow_cluster;           // host: whether a team may be chosen
  float scale_log2, scale_rest;   // scale * log2(e), and what its rounding to a float left out
  int* status;                 // CKV_FLAG_DEBUG_CHECKS: where a violated bound is reported; null otherwise
  int* timeout;                // where a wait that ran out is reported
};

struct ItemRows {   // the query heads of an item
  int s, head, rows, kv;       // sequence, first query head, number of heads, sequence * Hkv + KV head
};
__device__ __forceinline__ ItemRows item_rows(const DecodeArgs& p, int kv, int chunk) {
  ItemRows r;
  r.kv = kv;
  r.s = kv / p.c.Hkv;
  r.head = (kv - r.s * p.c.Hkv) * p.G + chunk * p.chunk_rows;
  r.rows = min(p.chunk_rows, p.G - chunk * p.chunk_rows);
  return r;
}
// sequence * Hkv + KV head of an item; most calls have one chunk, and a division is twenty instructions
__device__ __forceinline__ int kv_of(const DecodeArgs& p, int item) { return p.chunks == 1 ? item : item / p.chunks; }
__device__ __forceinline__ ItemRows item_rows(const DecodeArgs& p, int item) {
  const int kv = kv_of(p, item);
  return item_rows(p, kv, item - kv * p.chunks);
}
__device__ __forceinline__ int item_len(const DecodeArgs& p, int kv) {
  return (int)min(max((long long)p.lens[kv], 0LL), p.c.capacity);
}

__device__ __forceinline__ float* part_slot(const DecodeArgs& p, int dh, int cta, int slot) {
  return p.part + ((long long)cta * 2 + slot) * p.part_rows * (dh + 2);
}

// weight of a partial sum with maximum m against the joint maximum (m == -inf: nothing was visible there)
__device__ __forceinline__ float rescale(float m, float top) { return m == -INFINITY ? 0.f : exp2f(m - top); }

template <typename T> __device__ __forceinline__ void put2(char* at, float a, float b);
template <> __device__ __forceinline__ void put2<float>(char* at, float a, float b) {
  *reinterpret_cast<float2*>(at) = make_float2(a, b);
}
template <> __device__ __forceinline__ void put2<__nv_bfloat16>(char* at, float a, float b) {
  *reinterpret_cast<__nv_bfloat162*>(at) = __floats2bfloat162_rn(a, b);
}

// Elements 2*pair, 2*pair+1 of row r of an item, and its lse (written by pair 0).  An item without rows gives zeros.
template <typename T, int DH>
__device__ __forceinline__ void put_out(const DecodeArgs& p, const ItemRows& it, int r, int pair, float a, float b, float m,
                                        float l, bool empty) {
  const long long row = (long long)it.s * p.Hq + it.head + r;
  // l == 0 with rows present (every logit -inf) is 0 / 0, as in the formula
  const float inv = empty ? 0.f : 1.f / l;
  put2<T>(p.out + (row * DH + 2 * pair) * sizeof(T), a * inv, b * inv);
  if (pair == 0 && p.lse != nullptr) p.lse[row] = empty ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

// A CTA's range of the tile list, and the walk over the items in it.
struct Walk {
  int begin, end;              // tiles (the host has checked that they fit)
  int item;                    // first item
  int first;                   // its first tile in the list
  int total;
  int ctas;                    // CTAs that have work (all others have an empty range)
};

// Fills the walk (all threads get the same values).  Items without rows are written here, spread over the CTAs.
template <typename T, int DH, int TILE>
__device__ __forceinline__ Walk plan(const DecodeArgs& p) {
  __shared__ int upto[kDecodeThreads];                     // tiles of all items up to a thread's last (the host has
  __shared__ int warp_sums[kDecodeWarps];                  // checked that they fit)
  const int tid = threadIdx.x;
  const int per = (p.items + kDecodeThreads - 1) / kDecodeThreads;
  const int lo = min(tid * per, p.items), hi = min(lo + per, p.items);
  int incl = 0;
  bool bad = false, empty = false;
#pragma unroll 4
  for (int j = lo; j < hi; ++j) {
    const int given = p.lens[kv_of(p, j)];
    const int len = (int)min(max((long long)given, 0LL), p.c.capacity);
    bad = bad || len != given;
    empty = empty || len == 0;
    incl += (len + TILE - 1) / TILE;
  }
  if (bad && p.status != nullptr) atomicExch(p.status, (int)CKV_EBOUNDS);
  if (empty) {
    for (int j = lo; j < hi; ++j)
      if (item_len(p, kv_of(p, j)) == 0 && j % gridDim.x == blockIdx.x) {
        const ItemRows it = item_rows(p, j);
        for (int r = 0; r < it.rows; ++r)
          for (int k = 0; k < DH / 2; ++k) put_out<T, DH>(p, it, r, k, 0.f, 0.f, 0.f, 0.f, true);
      }
  }
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, incl, o);
    if ((tid & 31) >= o) incl += v;
  }
  if ((tid & 31) == 31) warp_sums[tid >> 5] = incl;
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int w = 0; w < kDecodeWarps; ++w) {
    if (w < (tid >> 5)) incl += warp_sums[w];
    total += warp_sums[w];
  }
  upto[tid] = incl;
  __syncthreads();
  Walk w;
  w.total = total;
  w.ctas = min((int)gridDim.x, total);
  w.begin = w.end = 0;
  w.item = 0;
  w.first = 0;
  if ((int)blockIdx.x < w.ctas) {
    w.begin = (int)((long long)total * blockIdx.x / w.ctas);
    w.end = (int)((long long)total * (blockIdx.x + 1) / w.ctas);
    int a = 0, b = kDecodeThreads - 1;     // first thread whose items reach behind tile `begin`
    while (a < b) {
      const int mid = (a + b) / 2;
      if (upto[mid] > w.begin) b = mid; else a = mid + 1;
    }
    w.first = a ? upto[a - 1] : 0;
    w.item = a * per;
  }
  return w;
}

// The walk of a CTA of a team: its share of the team's one item.
template <typename T, int DH, int TILE>
__device__ __forceinline__ Walk team_walk(const DecodeArgs& p) {
  Walk w;
  const int rank = blockIdx.x % p.team;
  w.item = blockIdx.x / p.team;
  const int kv = kv_of(p, w.item), len = item_len(p, kv);
  w.total = (len + TILE - 1) / TILE;
  w.first = 0;
  w.ctas = p.team;
  w.begin = w.total * rank / p.team;       // few tiles: decode_team
  w.end = w.total * (rank + 1) / p.team;
  if (rank == 0) {
    if (threadIdx.x == 0 && len != p.lens[kv] && p.status != nullptr) atomicExch(p.status, (int)CKV_EBOUNDS);
    if (len == 0) {
      const ItemRows it = item_rows(p, w.item);
      for (int i = threadIdx.x; i < it.rows * (DH / 2); i += kDecodeThreads)
        put_out<T, DH>(p, it, i / (DH / 2), i % (DH / 2), 0.f, 0.f, 0.f, 0.f, true);
    }
  }
  return w;
}

// A team's parts: every CTA of it calls this, also those without a tile.  parts [row][DH + 2] of the CTA: sums, maximum,
// sum of weights, filled where the CTA had tiles but not all of them; otherwise the sum of weights is 0.  The results are
// spread over the team's threads; each adds up the parts in order.
__device__ __forceinline__ float2 load_of_team(const float* mine, int rank) {
  uint32_t at;
  float2 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(mine)), "r"(rank));
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void team_barrier() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
template <typename T, int DH>
__device__ __forceinline__ void join_team(const DecodeArgs& p, const Walk& w, const float* parts) {
  if (p.team == 1) return;                 // has written the result
  team_barrier();
  if (w.total > 1) {                       // a single tile was one CTA's, which has written the result
    const ItemRows it = item_rows(p, w.item);
    for (int i = blockIdx.x % p.team * kDecodeThreads + threadIdx.x; i < it.rows * (DH / 2); i += p.team * kDecodeThreads) {
      const int r = i / (DH / 2), pair = i % (DH / 2);
      const float* row = parts + r * (DH + 2);
      float2 ml[kMaxTeam], v[kMaxTeam];
#pragma unroll
      for (int c = 0; c < kMaxTeam; ++c) {
        ml[c] = v[c] = make_float2(-INFINITY, 0.f);
        if (c < p.team) {
          ml[c] = load_of_team(row + DH, c);
          v[c] = load_of_team(row + 2 * pair, c);
        }
      }
      float top = -INFINITY, a = 0.f, b = 0.f, l = 0.f;
#pragma unroll
      for (int c = 0; c < kMaxTeam; ++c) top = fmaxf(top, ml[c].x);
#pragma unroll
      for (int c = 0; c < kMaxTeam; ++c)
        if (ml[c].y != 0.f) {              // else nothing was visible there, and its sums may not have been written
          const float f = rescale(ml[c].x, top);
          a += f * v[c].x;
          b += f * v[c].y;
          l += f * ml[c].y;
        }
      put_out<T, DH>(p, it, r, pair, a, b, top, l, false);
    }
  }
  team_barrier();                          // nobody leaves while its parts are read
}

// CTA whose range holds a tile: the largest i with total * i / ctas <= tile.
__device__ __forceinline__ int cta_of(const Walk& w, int tile) { return (int)(((tile + 1LL) * w.ctas - 1) / w.total); }

// Joins the warps' results of one group of NR rows and hands them on: to the output when the CTA did the whole item,
// else to its part.  o_s [warp][NR][DH] unnormalised sums, m_s, l_s [warp][NR].  All threads call it, and the
// buffers may be reused behind the barrier that the caller places.
template <typename T, int DH, int NR>
__device__ __forceinline__ void finish(const DecodeArgs& p, const ItemRows& it, const float* o_s, const float* m_s,
                                       const float* l_s, int row0, bool whole, float* parts) {
  constexpr int PAIRS = DH / 2;
  for (int i = threadIdx.x; i < NR * PAIRS; i += kDecodeThreads) {
    const int r = i / PAIRS, k = i % PAIRS;
    if (row0 + r >= it.rows) break;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kDecodeWarps; ++w) top = fmaxf(top, m_s[w * NR + r]);
    float a = 0.f, b = 0.f, l = 0.f;
#pragma unroll
    for (int w = 0; w < kDecodeWarps; ++w) {
      const float f = rescale(m_s[w * NR + r], top);
      const float2 v = *reinterpret_cast<const float2*>(o_s + (w * NR + r) * DH + 2 * k);
      // a warp that saw no finite logit has weight 0; its sums are 0 as well
      a += f * v.x;
      b += f * v.y;
      l += f * l_s[w * NR + r];
    }
    if (whole) {
      put_out<T, DH>(p, it, row0 + r, k, a, b, top, l, false);
    } else {
      float* part = parts + (row0 + r) * (DH + 2);
      *reinterpret_cast<float2*>(part + 2 * k) = make_float2(a, b);
      if (k == 0) *reinterpret_cast<float2*>(part + DH) = make_float2(top, l);
    }
  }
}

// Adds up a row's parts of CTAs c, c + step, ... <= c1 of an item that began in CTA c0 (in slot 1 there): four parts'
// loads are in flight before the first is looked at, for most calls all there are.
template <int DH>
__device__ __forceinline__ void add_parts(const DecodeArgs& p, int r, int c0, int c1, int c, int step, float& m, float& l,
                                          float2 (&acc)[DH / 64]) {
  constexpr int FLY = 4, E = DH / 64;
  m = -INFINITY;
  l = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = make_float2(0.f, 0.f);
  for (; c <= c1; c += FLY * step) {
    float2 ml[FLY], v[FLY][E];
#pragma unroll
    for (int i = 0; i < FLY; ++i) {
      const int ci = c + i * step;
      ml[i] = make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int e = 0; e < E; ++e) v[i][e] = make_float2(0.f, 0.f);
      if (ci <= c1) {
        const float* part = part_slot(p, DH, ci, ci == c0 ? 1 : 0) + r * (DH + 2);
        ml[i] = *reinterpret_cast<const float2*>(part + DH);
#pragma unroll
        for (int e = 0; e < E; ++e) v[i][e] = *reinterpret_cast<const float2*>(part + 2 * (threadIdx.x % 32 + 32 * e));
      }
    }
    float top = m;
#pragma unroll
    for (int i = 0; i < FLY; ++i) top = fmaxf(top, ml[i].x);
    const float f = rescale(m, top);
    m = top;
    l *= f;
#pragma unroll
    for (int e = 0; e < E; ++e) { acc[e].x *= f; acc[e].y *= f; }
#pragma unroll
    for (int i = 0; i < FLY; ++i) {
      const float g = rescale(ml[i].x, top);
      l += ml[i].y * g;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        acc[e].x += v[i][e].x * g;
        acc[e].y += v[i][e].y * g;
      }
    }
  }
}

// A row of an item of the parts of CTAs c0 ... c1: the warps take the parts in turn and meet in shared memory.
template <typename T, int DH, int THREADS>
__device__ __forceinline__ void join_row(const DecodeArgs& p, const ItemRows& it, int r, int c0, int c1) {
  constexpr int WARPS = THREADS / 32, E = DH / 64;        // pairs of elements a lane
  __shared__ __align__(8) float o_s[WARPS][DH];
  __shared__ float m_s[WARPS], l_s[WARPS];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  float m, l;
  float2 acc[E];
  add_parts<DH>(p, r, c0, c1, c0 + warp, WARPS, m, l, acc);
#pragma unroll
  for (int e = 0; e < E; ++e) *reinterpret_cast<float2*>(&o_s[warp][2 * (lane + 32 * e)]) = acc[e];
  if (lane == 0) { m_s[warp] = m; l_s[warp] = l; }
  __syncthreads();
  if (threadIdx.x < DH / 2) {
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) top = fmaxf(top, m_s[w]);
    float a = 0.f, b = 0.f;
    l = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float f = rescale(m_s[w], top);
      a += f * o_s[w][2 * threadIdx.x];
      b += f * o_s[w][2 * threadIdx.x + 1];
      l += f * l_s[w];
    }
    put_out<T, DH>(p, it, r, threadIdx.x, a, b, top, l, false);
  }
}

// CTAs (i, y): the item that ends in CTA i of the decode kernel, if it began in an earlier one.  Up to eight parts: y = 0
// does it all, a warp a row.  More: y is the row, whose parts the warps take in turn before they meet in shared memory.
// A fixed order of additions either way.
template <typename T, int DH>
__global__ void __launch_bounds__(kJoinThreads) decode_join_kernel(DecodeArgs p) {
  constexpr int WARPS = kJoinThreads / 32, E = DH / 64;   // pairs of elements a lane
  wait_for_previous_kernel();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, r = blockIdx.y;
  const int2 what = p.join[blockIdx.x];
  if (what.x < 0) return;
  const ItemRows it = item_rows(p, what.x);
  if ((int)blockIdx.x - what.y < 8) {
    if (r > 0) return;
    float m, l;
    float2 acc[E];
    for (int row = warp; row < it.rows; row += WARPS) {
      add_parts<DH>(p, row, what.y, blockIdx.x, what.y, 1, m, l, acc);
#pragma unroll
      for (int e = 0; e < E; ++e) put_out<T, DH>(p, it, row, lane + 32 * e, acc[e].x, acc[e].y, m, l, false);
    }
    return;
  }
  if (r >= it.rows) return;
  join_row<T, DH, kJoinThreads>(p, it, r, what.y, blockIdx.x);
}

// The same for few items of many parts: a CTA a row of an item (y: the row), which looks for the item's last CTA.
template <typename T, int DH>
__global__ void __launch_bounds__(kLongJoinThreads) decode_join_long_kernel(DecodeArgs p, int ctas) {
  __shared__ int2 found;                                   // last CTA, first CTA
  const int item = blockIdx.x, r = blockIdx.y;
  if (threadIdx.x == 0) found = make_int2(-1, 0);
  wait_for_previous_kernel();
  const ItemRows it = item_rows(p, item);
  if (r >= it.rows) return;
  __syncthreads();
  for (int c = threadIdx.x; c < ctas; c += kLongJoinThreads) {
    const int2 what = p.join[c];
    if (what.x == item) found = make_int2(c, what.y);      // one at most
  }
  __syncthreads();
  const int2 to = found;
  if (to.x >= 0) join_row<T, DH, kLongJoinThreads>(p, it, r, to.y, to.x);
}

// ---- host side ----------------------------------------------------------------------------------------------------
inline DecodeArgs decode_args(const CacheDims& d, const DecodeCall& call, int chunk_rows, int* status_word) {
  const int es = d.dtype == CKV_F32 ? 4 : 2;
  DecodeArgs p;
  p.c = pages_of(d);
  p.q = (const char*)call.q;
  p.qs[0] = call.q_stride[0] * es;
  p.qs[1] = call.q_stride[1] * es;
  p.lens = call.lens;
  p.out = (char*)call.out;
  p.lse = call.lse;
  p.join = (int2*)call.ws;
  p.part = (float*)((char*)call.ws + kDecodeMaxCtas * sizeof(int2));
  p.Hq = d.Hq;
  p.G = d.Hq / d.Hkv;
  p.chunk_rows = chunk_rows;
  p.chunks = (p.G + chunk_rows - 1) / chunk_rows;
  p.part_rows = p.G < chunk_rows ? p.G : chunk_rows;
  p.items = d.nseq * d.Hkv * p.chunks;
  p.scale_log2 = (float)(d.scale * 1.4426950408889634);
  p.scale_rest = (float)(d.scale * 1.4426950408889634 - (double)p.scale_log2);
  p.status = d.debug_checks ? status_word : nullptr;
  p.timeout = status_word;
  p.team = 0;
  p.allow_cluster = d.allow_cluster;
  return p;
}

// What a kernel needs to know once per device (asked for on its first launch there): CTAs an SM holds, and clusters of 2, 4,
// 8 and 16 that can run at once.
struct LaunchSetup {
  static constexpr int kDevices = 64;
  struct Fit {
    std::atomic<int> per_sm{0};
    std::atomic<int> clusters[4] = {};
  } fit[kDevices];
  template <typename K> const Fit* of(K kernel, int device, int smem) {
    if (device >= kDevices) return nullptr;
    Fit& f = fit[device];
    if (f.per_sm.load(std::memory_order_acquire) > 0) return &f;
    if (smem > 48 * 1024 - 2048 &&
        cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess)
      return nullptr;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return nullptr;
    for (int i = 0; i < 4; ++i) {
      cudaLaunchConfig_t cfg = {};
      cudaLaunchAttribute attr;
      attr.id = cudaLaunchAttributeClusterDimension;
      attr.val.clusterDim.x = 2u << i;
      attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
      cfg.gridDim = dim3((unsigned)(kMaxTeam * 64));
      cfg.blockDim = dim3(kDecodeThreads);
      cfg.dynamicSmemBytes = (size_t)smem;
      cfg.attrs = &attr;
      cfg.numAttrs = 1;
      int n = 0;
      if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) {
        n = 0;
        cudaGetLastError();
      }
      f.clusters[i].store(n, std::memory_order_relaxed);
    }
    int n = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, kDecodeThreads, smem) != cudaSuccess || n < 1) return nullptr;
    f.per_sm.store(n, std::memory_order_release);
    return &f;
  }
};

// CTAs an item's team has; 0: no teams, the even split and its join.
// A CTA alone (team 1) needs neither the split's scan of all lengths nor a join; a larger team costs 1 to 2 us for the
// cluster's launch and barriers, more the more of them there are (hence small ones first, on half the GPU), and saves 1 us per 64-row
// tile of bf16 rows of 128; the even split costs 3 us more than a CTA alone and a second launch.  Tiles are counted by the
// table's size, the lengths are not known here; where they are very uneven a CTA has at most seven tiles behind the split.
// Device times in us with 1, 2, 4, 8, 16 CTAs, and of the even split, 8 KV heads of 128, bf16 rows with a spread of 30 %
// (a call is 2.3 us shorter with teams where the host bounds it):
//   1 sequence  x   60 rows:  5.6   6.5   6.4   6.3   6.6, 7.3      18 x  60:  5.9   7.8 ...      , 8.3
//   1 sequence  x  400 rows:   -    9.6   7.6   6.7   7.6, 8.1      18 x 200:  8.7  10.0 ...      , 11.6
//   1 sequence  x  819 rows:   -   13.9  10.2   8.6   8.1, 8.1      37 x 200: 10.5  18.6 ...      , 14.1
//   6 sequences x  400 rows:   -   10.3   8.5   8.6  22.3, 9.9      128 x 60: 16.4  33.1 ...      , 19.0
// In between the choice is up to 17 % off on the device (14 sequences of 400 e4m3 rows 12.4, split 10.6), which is what the
// second launch costs a call.  A cache whose table has room for much more than its heads hold takes the split, too (1
// sequence x 819 bf16 rows in a table for 16384: 8.6 us instead of 8.0 on the device, 12.2 instead of 9.7 a call).
inline int decode_team(const DecodeArgs& p, const LaunchSetup::Fit& fit, int sm_count, int tile) {
  const long long tiles = (p.c.capacity + tile - 1) / tile, resident = (long long)fit.per_sm.load() * sm_count;
  auto fit_at_once = [&](int i) { return p.allow_cluster && p.items <= fit.clusters[i].load(std::memory_order_relaxed); };
  if (tiles <= 3 && p.items <= 3 * resident) return 1;
  for (int most = 1; most <= 2; ++most)                    // tiles a CTA
    for (int i = 0; i < 4; ++i)
      if (tiles <= most * (2 << i) && fit_at_once(i) && p.items * (4LL << i) <= resident) return 2 << i;
  if (tiles <= 7 && p.items <= resident && 4LL * p.items > resident) return 1;
  for (int i = 3; i >= 0; --i)
    if (tiles <= (i >= 2 ? 3 : 4) * (2 << i) && fit_at_once(i)) return 2 << i;
  return 0;
}

// One CTA per resident slot, fewer when even full heads have fewer tiles than that.
inline int decode_grid(const DecodeArgs& p, int resident, int tile) {
  const long long tiles = (p.c.capacity + tile - 1) / tile * p.items;
  long long grid = resident < kDecodeMaxCtas ? resident : kDecodeMaxCtas;
  if (grid > tiles) grid = tiles;
  return grid < 1 ? 1 : (int)grid;
}

template <typename T, int DH> cudaError_t launch_decode_join(const DecodeArgs& p, int grid, cudaStream_t st) {
  // many parts an item: device times of the whole call in us, this join and the other, heads of 128: 1 KV head of 48936 rows
  // (444 parts) 16.0 and 21.5, 8 of 6553 (55 parts) 11.7 and 12.2, 32 (14 parts) 24.3 and 24.7, 56 (8 parts) 40.2 and 38.0
  if (grid >= kLongJoinParts * p.items)
    return launch_early<DecodeArgs, int>(decode_join_long_kernel<T, DH>, dim3((unsigned)p.items, (unsigned)p.part_rows),
                                         kLongJoinThreads, 0, st, p, grid);
  return launch_early<DecodeArgs>(decode_join_kernel<T, DH>, dim3((unsigned)grid, (unsigned)p.part_rows), kJoinThreads, 0, st, p);
}

}  // namespace ckv
