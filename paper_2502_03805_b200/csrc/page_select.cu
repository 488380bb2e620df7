// Which pages of a long cache a new token looks at: summaries of pages, their scores against the queries, and the choice.
//
// Summary of a page: per channel the largest and the smallest of its keys (of what the pages stand for), as 8-bit codes with
// one float32 scale, rounded outwards.  Score of a page for a query: sum over the channels of the larger of query * largest
// and query * smallest, which no logit of the page exceeds but for the roundings of the codes; with the query in 8-bit codes
// too it is the sum of products of its positive codes with the largest and of its negative ones with the smallest: whole
// numbers, so the matrix instructions' order of additions does not matter and equal inputs choose equal pages anywhere.
//
// summarise reads every key once and is bound by HBM.  select reads 2 dh + 4 bytes a page: a (sequence, KV head) is a
// cluster's of 1 to 8 CTAs whose warps score 16 pages at a time (pages on the 16-row side of mma.sync, 8 queries on the
// other) and leave the scores in the shared memory of the cluster's first CTA, which looks for the smallest chosen one in a
// histogram and writes the chosen pages in order: one launch, and the table that it writes is one that decode reads.
//
// Measured, 8 KV heads of 128: summaries of 131072 bf16 rows 44.6 us, 6.1 TB/s (0.94 of the copy bandwidth; with conversions to
// float32 66.9), of e4m3 rows 43 (no unit full: ALU 62 %, DRAM 38 %; what holds it was not found); the choice of 64 of 2048 pages for 4 queries a head 8.0 us, a chain of
// latencies (length, page, summary, two cluster barriers, histogram; 11.9 with a bisection of the keys), 32 sequences of 512
// pages 13.4 us.
#include "launch_early.cuh"
#include "paged_codes.cuh"

namespace ckv {
namespace {

// ---- summaries -------------------------------------------------------------------------------------------------------
constexpr int kThreads = 128;

struct SummaryArgs {
  Pages c;
  const int32_t* start;            // null: all pages
  const int32_t* lens;
  int8_t* codes;                   // [num_pages, 2, dh]
  float* scales;                   // [num_pages]
  int workers;                     // CTAs or warps a head
  int* status;
};

// Eight consecutive elements of a stored row: as they lie in memory, and as floats.
template <typename T, int FMT> struct Eight {
  static constexpr int V = Piece<T>::V;
  uint4 raw[FMT == CKV_CACHE_PLAIN ? 8 / V : 1];       // 8-bit and 4-bit codes: x, y
  float scale;
  uint32_t group;
  __device__ __forceinline__ void load(const Pages& c, long long page, int in_page, int dh, int e) {
    const char* base = c.page[0] + page * c.page_stride;
    if constexpr (FMT == CKV_CACHE_PLAIN) {
#pragma unroll
      for (int i = 0; i < 8 / V; ++i) raw[i] = *reinterpret_cast<const uint4*>(base + (in_page * dh + e + V * i) * (int)sizeof(T));
    } else {
      const long long slot = (page << c.page_shift) + in_page;
      if constexpr (FMT == CKV_CACHE_E2M1) {
        raw[0].x = *reinterpret_cast<const uint32_t*>(base + (in_page * dh + e) / 2);
        group = c.group[0][slot * (dh / 16) + e / 16];
      } else {
        const uint2 code = *reinterpret_cast<const uint2*>(base + in_page * dh + e);
        raw[0].x = code.x;
        raw[0].y = code.y;
      }
      scale = c.scale[0][slot];
    }
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    if constexpr (FMT == CKV_CACHE_PLAIN) {
#pragma unroll
      for (int i = 0; i < 8 / V; ++i) {
        float y[V];
        Piece<T>::get(raw[i], y);
#pragma unroll
        for (int j = 0; j < V; ++j) x[V * i + j] = y[j];
      }
    } else if constexpr (FMT == CKV_CACHE_E2M1) {
      decode8_e2m1(raw[0].x, group, x);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] *= scale;
    } else {
      float y[2][4];
      decode4<FMT>(raw[0].x, y[0]);
      decode4<FMT>(raw[0].y, y[1]);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = y[i / 4][i % 4] * scale;
    }
  }
};

// Maximum and minimum that are NaN where either is one: a page with an infinity or a NaN is then seen by its extremes alone.
__device__ __forceinline__ float nan_max(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ float nan_min(float a, float b, float c) {
  float d;
  asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ float nan_max(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ float nan_min(float a, float b) {
  float d;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}

// Largest and smallest of the rows `sub`, `sub` + step, ... of a page, several in flight (the last row again behind the end).
template <typename T, int FMT>
__device__ __forceinline__ void reduce_rows(const Pages& c, long long page, int rows, int dh, int e, int sub, int step, float (&hi)[8],
                                            float (&lo)[8]) {
  if constexpr (FMT == CKV_CACHE_PLAIN && sizeof(T) == 2) {
    // two elements an instruction, as they are stored
    constexpr int FLY = 8;
    const char* base = c.page[0] + page * c.page_stride + e * 2;
    __nv_bfloat162 up[4], down[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      up[j] = __floats2bfloat162_rn(-INFINITY, -INFINITY);
      down[j] = __floats2bfloat162_rn(INFINITY, INFINITY);
    }
    for (int r = sub; r < rows; r += FLY * step) {
      uint4 raw[FLY];
#pragma unroll
      for (int i = 0; i < FLY; ++i) raw[i] = *reinterpret_cast<const uint4*>(base + min(r + i * step, rows - 1) * dh * 2);
#pragma unroll
      for (int i = 0; i < FLY; ++i) {
        const uint32_t x[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const __nv_bfloat162 y = *reinterpret_cast<const __nv_bfloat162*>(&x[j]);
          up[j] = __hmax2_nan(up[j], y);
          down[j] = __hmin2_nan(down[j], y);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 a = __bfloat1622float2(up[j]), b = __bfloat1622float2(down[j]);
      hi[2 * j] = a.x; hi[2 * j + 1] = a.y;
      lo[2 * j] = b.x; lo[2 * j + 1] = b.y;
    }
  } else {
    constexpr int FLY = FMT == CKV_CACHE_PLAIN ? 4 : 8;
#pragma unroll
    for (int j = 0; j < 8; ++j) { hi[j] = -INFINITY; lo[j] = INFINITY; }
    for (int r = sub; r < rows; r += FLY * step) {
      Eight<T, FMT> row[FLY];
#pragma unroll
      for (int i = 0; i < FLY; ++i) row[i].load(c, page, min(r + i * step, rows - 1), dh, e);
#pragma unroll
      for (int i = 0; i < FLY; i += 2) {
        float x[2][8];
        row[i].get(x[0]);
        row[i + 1].get(x[1]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          hi[j] = nan_max(hi[j], x[0][j], x[1][j]);
          lo[j] = nan_min(lo[j], x[0][j], x[1][j]);
        }
      }
    }
  }
}

// WARPS warps share a page: one where there are many, four where there are few.
template <typename T, int FMT, int DH, int WARPS> __global__ void __launch_bounds__(kThreads) summarise_kernel(SummaryArgs p) {
  wait_for_previous_kernel();
  constexpr int LANES = DH / 8, ROWS = 32 / LANES;        // lanes a row, rows a warp takes at a time
  constexpr int TEAMS = 4 / WARPS;                        // pages a CTA works on
  __shared__ float part[2][4][DH];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int item = blockIdx.x / p.workers, worker = blockIdx.x % p.workers * TEAMS + warp / WARPS;
  const int given = p.lens[item];
  const long long len = min(max((long long)given, 0LL), p.c.capacity);
  long long from = 0;
  bool bad = len != given;
  if (p.start != nullptr) {
    const int at = p.start[item];
    from = min(max((long long)at, 0LL), len);
    bad = bad || from != at;
  }
  if (bad && worker == 0 && lane == 0 && p.status != nullptr) atomicExch(p.status, (int)CKV_EBOUNDS);
  const int e = lane % LANES * 8;
  const int size = 1 << p.c.page_shift;
  // all warps of a team take the same turns
  for (long long n = (from >> p.c.page_shift) + worker; (n << p.c.page_shift) < len && from < len; n += (long long)p.workers * TEAMS) {
    const int page = p.c.table[(long long)item * p.c.max_pages + n];
    if (page < 0 || page >= p.c.num_pages) {
      if (p.status != nullptr && lane == 0) atomicExch(p.status, (int)CKV_EBOUNDS);
      continue;
    }
    const int rows = (int)min(len - (n << p.c.page_shift), (long long)size);
    float hi[8], lo[8];
    reduce_rows<T, FMT>(p.c, page, rows, DH, e, warp % WARPS * ROWS + lane / LANES, WARPS * ROWS, hi, lo);
#pragma unroll
    for (int o = LANES; o < 32; o <<= 1)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        hi[j] = nan_max(hi[j], __shfl_xor_sync(0xffffffffu, hi[j], o));
        lo[j] = nan_min(lo[j], __shfl_xor_sync(0xffffffffu, lo[j], o));
      }
    if (WARPS > 1) {
      __syncthreads();                                    // the page before has been joined
      if (lane < LANES) {
#pragma unroll
        for (int j = 0; j < 8; ++j) { part[0][warp][e + j] = hi[j]; part[1][warp][e + j] = lo[j]; }
      }
      __syncthreads();
      if (warp > 0) continue;
#pragma unroll
      for (int w = 1; w < 4; ++w) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          hi[j] = nan_max(hi[j], part[0][w][e + j]);
          lo[j] = nan_min(lo[j], part[1][w][e + j]);
        }
      }
    }
    uint32_t top = 0;                                     // the order of the bits puts NaN above infinity
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, max(__float_as_uint(hi[j]) & 0x7fffffffu, __float_as_uint(lo[j]) & 0x7fffffffu));
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    const bool finite = top < 0x7f800000u;
    float scale = __fdiv_rn(__uint_as_float(top), 127.f);
    if (scale < kLeastScale) scale = kLeastScale;
    const float r = __frcp_rn(scale);
    if (lane < LANES) {
      uint32_t code[2][2] = {{0, 0}, {0, 0}};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int up = min(max(__float2int_ru(__fmul_rn(hi[j], r)), -127), 127);
        const int down = min(max(__float2int_rd(__fmul_rn(lo[j], r)), -127), 127);
        code[0][j / 4] |= ((uint32_t)(finite ? up : 0) & 0xffu) << (8 * (j % 4));
        code[1][j / 4] |= ((uint32_t)(finite ? down : 0) & 0xffu) << (8 * (j % 4));
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
        *reinterpret_cast<uint2*>(p.codes + ((long long)page * 2 + h) * DH + e) = make_uint2(code[h][0], code[h][1]);
    }
    if (lane == 0) p.scales[page] = scale;
  }
}

// ---- choice ----------------------------------------------------------------------------------------------------------
constexpr int kSelectThreads = 512, kSelectWarps = kSelectThreads / 32;
constexpr int kBins = 1024, kShort = 1024;       // of the histogram of keys; pages that share the last bin and are ranked one by one
constexpr uint32_t kForced = 0xffffffffu;        // key of a page that is always chosen

// Bytes from query to query in shared memory, half of what the banks span more than a multiple of it: the eight lanes of a read, four
// on each of two queries, are on different banks.
constexpr int query_bytes(int dh) { return dh % 128 == 64 ? dh : dh + 64; }

struct SelectArgs {
  Pages c;
  const char* q;
  long long qs[2];                 // byte strides: sequence, head
  const int32_t* lens;
  const int8_t* codes;
  const float* scales;
  int G, Hq;
  int count, first, last;
  int32_t* table_out;              // [items, count]
  int32_t* lens_out;               // [items]
  int32_t* chosen;                 // [items, count] or null
  int cluster;
  int* status;
};

__device__ __forceinline__ void mma_s8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Order of scores: larger is better, a NaN better than any number, 0 for a page that does not exist.
__device__ __forceinline__ uint32_t key_of(float score) {
  const uint32_t b = __float_as_uint(__fadd_rn(score, 0.f));       // -0 becomes 0
  if ((b & 0x7fffffffu) > 0x7f800000u) return kForced - 1;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

// Sum over the threads in front of this one; `total`: over all of them.
__device__ __forceinline__ uint32_t sum_before(uint32_t x, uint32_t (&sums)[kSelectWarps], uint32_t& total) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  uint32_t incl = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += v;
  }
  __syncthreads();                               // the sums of the call before have been read
  if (lane == 31) sums[warp] = incl;
  __syncthreads();
  total = 0;
  uint32_t before = incl - x;
#pragma unroll
  for (int w = 0; w < kSelectWarps; ++w) {
    if (w < warp) before += sums[w];
    total += sums[w];
  }
  return before;
}

// What the first CTA of a cluster looks for the smallest chosen key with.
struct Search {
  uint32_t bins[kBins];
  uint32_t keys[kShort];                         // of the pages in the last bin
  uint32_t sums[kSelectWarps], low, high, bin, above, listed, least, ties;
};

// The smallest chosen key of n and how many of the pages that have it are chosen: `count` in all, n > count.  Every thread
// gets them.  Keys are spread over bins by their distance from the smallest, the bin that holds the border is listed, and
// every listed page counts those above it; a bin that is too full (equal scores) is halved until it is not.
__device__ __forceinline__ void find_least(const uint32_t* keys, int n, uint32_t count, Search& f) {
  uint32_t low = kForced, high = 0, forced = 0;
  for (int j = threadIdx.x; j < n; j += kSelectThreads) {
    const uint32_t k = keys[j];
    if (k == kForced) { forced += 1; continue; }
    low = min(low, k);
    high = max(high, k);
  }
  low = __reduce_min_sync(0xffffffffu, low);
  high = __reduce_max_sync(0xffffffffu, high);
  forced = __reduce_add_sync(0xffffffffu, forced);
  if (threadIdx.x % 32 == 0) {                   // set up before the scores
    atomicMin(&f.low, low);
    atomicMax(&f.high, high);
    atomicAdd(&f.above, forced);
  }
  __syncthreads();
  low = f.low;
  high = f.high;
  uint32_t above = f.above;                      // keys above `high`
  if (above >= count) {                          // (equal: the forced ones are all)
    if (threadIdx.x == 0) { f.least = kForced; f.ties = count; }
    __syncthreads();
    return;
  }
  while (true) {
    // the border is among the keys of low ... high, `above` keys are above them
    const int shift = max(0, 32 - __clz(high - low) - 10);
    for (int b = threadIdx.x; b < kBins; b += kSelectThreads) f.bins[b] = 0;
    if (threadIdx.x == 0) f.listed = 0;
    __syncthreads();
    for (int j = threadIdx.x; j < n; j += kSelectThreads) {
      const uint32_t k = keys[j];
      if (k >= low && k <= high) atomicAdd(&f.bins[kBins - 1 - ((k - low) >> shift)], 1u);   // the largest first
    }
    __syncthreads();
    static_assert(kBins == 2 * kSelectThreads, "two bins a thread");
    const uint32_t b0 = f.bins[2 * threadIdx.x], b1 = f.bins[2 * threadIdx.x + 1];
    uint32_t total, before = above + sum_before(b0 + b1, f.sums, total);
    if (before < count && before + b0 + b1 >= count) {
      const bool second = before + b0 < count;
      f.bin = 2 * threadIdx.x + second;
      f.above = before + (second ? b0 : 0);
    }
    __syncthreads();
    const uint32_t at = low + ((uint32_t)(kBins - 1 - f.bin) << shift);       // smallest key of the bin
    const uint32_t held = f.bins[f.bin];
    above = f.above;
    if (shift == 0) {                            // one key a bin
      if (threadIdx.x == 0) { f.least = at; f.ties = count - above; }
      __syncthreads();
      return;
    }
    low = at;
    high = at + min(high - at, (1u << shift) - 1u);
    if (held <= kShort) {
      for (int j = threadIdx.x; j < n; j += kSelectThreads) {
        const uint32_t k = keys[j];
        if (k >= low && k <= high) f.keys[atomicAdd(&f.listed, 1u)] = k;
      }
      __syncthreads();
      for (uint32_t i = threadIdx.x; i < held; i += kSelectThreads) {
        const uint32_t k = f.keys[i];
        uint32_t larger = above, equal = 0;
        for (uint32_t o = 0; o < held; ++o) {
          larger += f.keys[o] > k;
          equal += f.keys[o] == k;
        }
        if (larger < count && larger + equal >= count) { f.least = k; f.ties = count - larger; }   // the same of equal ones
      }
      __syncthreads();
      return;
    }
    __syncthreads();                             // all have read the bin
  }
}

template <typename T, int DH> __global__ void __launch_bounds__(kSelectThreads, 2) select_pages_kernel(SelectArgs p) {
  wait_for_previous_kernel();
  constexpr int Q = query_bytes(DH);
  static_assert(Q % 128 == 64, "two queries a turn of the banks");
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ Search found;
  const int heads8 = (p.G + 7) / 8 * 8;
  unsigned char* q_pos = smem;                   // [heads8][Q] positive codes, then negative ones
  unsigned char* q_neg = smem + heads8 * Q;
  float* q_scale = reinterpret_cast<float*>(smem + 2 * heads8 * Q);
  uint32_t* keys = reinterpret_cast<uint32_t*>(q_scale + heads8);   // of all pages, in the cluster's first CTA
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, r = lane >> 2, c = lane & 3;
  const int item = blockIdx.x / p.cluster, rank = blockIdx.x % p.cluster;
  const int s = item / p.c.Hkv, head0 = (item - s * p.c.Hkv) * p.G;
  if (threadIdx.x == 0) { found.low = kForced; found.high = 0; found.above = 0; }
  if (p.cluster > 1) cluster_arrive();           // the others may write to this CTA's shared memory
  // what the first tile needs is on its way before the length is known
  const int given = p.lens[item];
  const int32_t* pages = p.c.table + (long long)item * p.c.max_pages;
  int tile = rank * kSelectWarps + warp, page[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) page[h] = tile * 16 + r + 8 * h < p.c.max_pages ? pages[tile * 16 + r + 8 * h] : -1;
  // ---- queries as 8-bit codes
  for (int h = warp; h < heads8; h += kSelectWarps) {
    constexpr int E = DH / 32;
    float x[E];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      x[i] = h < p.G ? (float)reinterpret_cast<const T*>(p.q + s * p.qs[0] + (head0 + h) * p.qs[1])[E * lane + i] : 0.f;
      top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    }
    top = __reduce_max_sync(0xffffffffu, top);
    float scale = __fdiv_rn(__uint_as_float(top), 127.f);
    if (scale < kLeastScale) scale = kLeastScale;
    const float inv = __frcp_rn(scale);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int code = top < 0x7f800000u ? min(max(__float2int_rn(__fmul_rn(x[i], inv)), -127), 127) : 0;
      q_pos[h * Q + E * lane + i] = (unsigned char)max(code, 0);
      q_neg[h * Q + E * lane + i] = (unsigned char)min(code, 0);
    }
    if (lane == 0) q_scale[h] = scale;
  }
  const long long len = min(max((long long)given, 0LL), p.c.capacity);
  if (len != given && rank == 0 && threadIdx.x == 0 && p.status != nullptr) atomicExch(p.status, (int)CKV_EBOUNDS);
  const int size = 1 << p.c.page_shift;
  const int held = (int)((len + size - 1) >> p.c.page_shift);       // pages of the head
  const bool all = held <= p.count;
  __syncthreads();
  bool arrived = p.cluster == 1;
  uint32_t keys_at;                              // of the first CTA
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(keys_at) : "r"((uint32_t)__cvta_generic_to_shared(keys)), "r"(0));
  // ---- scores of 16 pages at a time
  const int tiles = all ? 0 : (held + 15) / 16;
  while (tile < tiles) {
    const int row[2] = {tile * 16 + r, tile * 16 + r + 8};
    uint4 a[2][2][DH / 64];                      // [page][largest, smallest][16 bytes of 64]
    float scale[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool there = row[h] < held && page[h] >= 0 && page[h] < p.c.num_pages;
      if (!there && row[h] < held && p.status != nullptr && c == 0) atomicExch(p.status, (int)CKV_EBOUNDS);
      if (!there) page[h] = -1;
      const int8_t* at = p.codes + (long long)(there ? page[h] : 0) * 2 * DH + c * 16;
      scale[h] = there ? p.scales[page[h]] : 0.f;
#pragma unroll
      for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int j = 0; j < DH / 64; ++j)
          a[h][w][j] = there ? *reinterpret_cast<const uint4*>(at + w * DH + 64 * j) : make_uint4(0, 0, 0, 0);
    }
    tile += p.cluster * kSelectWarps;
    int next[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) next[h] = tile * 16 + r + 8 * h < held ? pages[tile * 16 + r + 8 * h] : -1;
    uint32_t best[2] = {0, 0};
    for (int h0 = 0; h0 < p.G; h0 += 8) {
      int d[4] = {0, 0, 0, 0};
#pragma unroll
      for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int j = 0; j < DH / 64; ++j) {
          const uint4 b = *reinterpret_cast<const uint4*>((w ? q_neg : q_pos) + (h0 + r) * Q + c * 16 + 64 * j);
          mma_s8(d, a[0][w][j].x, a[1][w][j].x, a[0][w][j].y, a[1][w][j].y, b.x, b.y);
          mma_s8(d, a[0][w][j].z, a[1][w][j].z, a[0][w][j].w, a[1][w][j].w, b.z, b.w);
        }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int h = h0 + 2 * c + x;
        if (h < p.G) {
          const float qs = q_scale[h];
#pragma unroll
          for (int y = 0; y < 2; ++y)
            best[y] = max(best[y], key_of(__fmul_rn(__fmul_rn((float)d[2 * y + x], qs), scale[y])));
        }
      }
    }
    if (!arrived) {                              // the first CTA is there
      cluster_wait();
      arrived = true;
    }
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      best[y] = max(best[y], __shfl_xor_sync(0xffffffffu, best[y], 1));
      best[y] = max(best[y], __shfl_xor_sync(0xffffffffu, best[y], 2));
      if (c == 0 && row[y] < held) {
        uint32_t key = page[y] < 0 ? 0u : best[y];
        if (row[y] < p.first || row[y] >= held - p.last) key = kForced;
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(keys_at + 4 * row[y]), "r"(key) : "memory");
      }
    }
    page[0] = next[0];
    page[1] = next[1];
  }
  if (p.cluster > 1) {
    if (!arrived) cluster_wait();
    cluster_arrive();
    cluster_wait();
  } else {
    __syncthreads();
  }
  if (rank != 0) return;

  uint32_t least = 0, ties = 0;
  if (!all) {
    find_least(keys, held, (uint32_t)p.count, found);
    least = found.least;
    ties = found.ties;
  }
  // ---- the chosen pages in order: every thread has consecutive ones; first their numbers (where the bins were, if there is
  // room), then their ids
  const int per = (held + kSelectThreads - 1) / kSelectThreads, at = min((int)threadIdx.x * per, held), to = min(at + per, held);
  uint32_t mine = 0;                             // low half: keys above, high half: keys equal to `least`
  for (int j = at; j < to; ++j) mine += all ? 1u : keys[j] > least ? 1u : keys[j] == least ? 0x10000u : 0u;
  uint32_t total;
  const uint32_t before = sum_before(mine, found.sums, total);
  uint32_t above = before & 0xffffu, equal = before >> 16;
  int32_t* table = p.table_out + (long long)item * p.count;
  int32_t* chosen = p.chosen != nullptr ? p.chosen + (long long)item * p.count : nullptr;
  int32_t* numbers = p.count <= kBins ? reinterpret_cast<int32_t*>(found.bins) : table;
  for (int j = at; j < to; ++j) {
    const uint32_t key = all ? kForced : keys[j];
    const bool is = key > least || all, tie = !is && key == least;
    const uint32_t place = above + min(equal, ties);
    if ((is || (tie && equal < ties)) && place < (uint32_t)p.count) numbers[place] = j;
    above += is;
    equal += tie;
  }
  const int n = (int)((total & 0xffffu) + min(total >> 16, ties));
  if (at < held && to == held) {
    // the last page may not be full; it is the last of the chosen ones where it is chosen
    const uint32_t key = all ? kForced : keys[held - 1];
    const bool tail = all || key > least || (key == least && equal - 1 < ties);
    p.lens_out[item] = n * size - (tail ? (int)(((long long)held << p.c.page_shift) - len) : 0);
  } else if (held == 0 && threadIdx.x == 0) {
    p.lens_out[item] = 0;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < p.count; i += kSelectThreads) {
    const int j = i < n ? numbers[i] : -1;
    table[i] = j >= 0 ? pages[j] : -1;
    if (chosen != nullptr) chosen[i] = j;
  }
}

template <typename F> void by_type(const CacheDims& d, F&& f) {
  auto dims = [&](auto t, auto fmt) {
    if (d.dh == 64) f(t, fmt, std::integral_constant<int, 64>());
    else f(t, fmt, std::integral_constant<int, 128>());
  };
  auto formats = [&](auto t) {
    if (d.format == CKV_CACHE_PLAIN) dims(t, std::integral_constant<int, CKV_CACHE_PLAIN>());
    else if (d.format == CKV_CACHE_E4M3) dims(t, std::integral_constant<int, CKV_CACHE_E4M3>());
    else if (d.format == CKV_CACHE_E2M1) dims(t, std::integral_constant<int, CKV_CACHE_E2M1>());
    else dims(t, std::integral_constant<int, CKV_CACHE_INT8>());
  };
  if (d.dtype == CKV_F32) formats(float());
  else formats(__nv_bfloat16());
}

}  // namespace

cudaError_t launch_summarise(const CacheDims& d, const int32_t* start, const int32_t* lens, int8_t* codes, float* scales,
                             int sm_count, int* status_word, cudaStream_t st, int* launches) {
  const long long items = (long long)d.nseq * d.Hkv;
  SummaryArgs p;
  p.c = pages_of(d);
  p.start = start; p.lens = lens; p.codes = codes; p.scales = scales;
  p.status = d.debug_checks ? status_word : nullptr;
  // the lengths are not known here: workers for as many pages as the table has, up to what the GPU holds
  const bool few = items * d.max_pages <= 16LL * sm_count || start != nullptr;
  const int teams = few ? 1 : 4;
  long long workers = (16LL * sm_count + items - 1) / items;
  if (workers > (d.max_pages + teams - 1) / teams) workers = (d.max_pages + teams - 1) / teams;
  const long long most = 0x7fffffffLL / items;
  if (workers > most) workers = most;
  p.workers = workers < 1 ? 1 : (int)workers;
  cudaError_t e = cudaSuccess;
  by_type(d, [&](auto t, auto fmt, auto dh) {
    using T = decltype(t);
    constexpr int FMT = decltype(fmt)::value, DH = decltype(dh)::value;
    e = launch_early<SummaryArgs>(few ? summarise_kernel<T, FMT, DH, 4> : summarise_kernel<T, FMT, DH, 1>,
                                  dim3((unsigned)(items * p.workers)), kThreads, 0, st, p);
  });
  *launches += 1;
  return e;
}

constexpr size_t select_pages_smem(int group, int dh, int max_pages) {
  return (size_t)(group + 7) / 8 * 8 * (2 * query_bytes(dh) + 4) + 4 * (size_t)max_pages;
}

cudaError_t launch_select_pages(const CacheDims& d, const SelectPagesCall& call, int sm_count, int* status_word, cudaStream_t st,
                                int* launches) {
  const int es = d.dtype == CKV_F32 ? 4 : 2;
  const long long items = (long long)d.nseq * d.Hkv;
  SelectArgs p;
  p.c = pages_of(d);
  p.q = (const char*)call.q;
  p.qs[0] = call.q_stride[0] * es; p.qs[1] = call.q_stride[1] * es;
  p.lens = call.lens; p.codes = call.codes; p.scales = call.scales;
  p.G = d.Hq / d.Hkv; p.Hq = d.Hq;
  p.count = call.count; p.first = call.first; p.last = call.last;
  p.table_out = call.table_out; p.lens_out = call.lens_out; p.chosen = call.chosen;
  p.status = d.debug_checks ? status_word : nullptr;
  const int smem = (int)select_pages_smem(d.Hq / d.Hkv, d.dh, d.max_pages);
  // a cluster as large as its pages keep busy and as leaves every head one at the same time
  const int tiles = (d.max_pages + 15) / 16;
  p.cluster = 1;
  while (d.allow_cluster && p.cluster < 8 && p.cluster * kSelectWarps < tiles && 2 * p.cluster * items <= 2LL * sm_count) p.cluster *= 2;
  const auto kernel = d.dtype == CKV_F32 ? (d.dh == 64 ? select_pages_kernel<float, 64> : select_pages_kernel<float, 128>)
                                         : (d.dh == 64 ? select_pages_kernel<__nv_bfloat16, 64> : select_pages_kernel<__nv_bfloat16, 128>);
  if (smem > 48 * 1024 - (int)sizeof(Search)) {
    // the same number for every call: host threads with handles of their own set it for one another
    constexpr int most = (int)select_pages_smem(kSelectMostGroup, 128, kSelectMostPages);
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    if (e != cudaSuccess) return e;
  }
  *launches += 1;
  return launch_early_in_clusters<SelectArgs>(kernel, dim3((unsigned)(items * p.cluster)), kSelectThreads, smem, p.cluster, st, p);
}

}  // namespace ckv
