// Rows into and out of the paged cache.  Both kernels read and write every row once and are bound by HBM.
//
// Store: a row is handled by the fewest lanes that keep its 16-byte pieces coalesced (64 bytes of the row each), because
// the scale's division and reciprocal are paid once per lane.  A thread has 64 bytes of K and of V in flight, 32 warps
// an SM, and follows the chain row index -> page id of its next row while it rounds and writes this one.  8 x 8 heads,
// 6553 of 32768 rows of 128 bf16 each to e4m3: 58 us, 5.6 TB/s (101 us with 16 bytes a lane, 87 us with 16 warps an SM).
// Load: 16 bytes of output a lane, four rows of K and V in flight.  8 x 8 heads of 6553 e4m3 rows of 128 to bf16: 55 us,
// 6.0 TB/s.
#include <cuda_bf16.h>

#include "launch_early.cuh"
#include "paged_common.cuh"

namespace ckv {
namespace {

constexpr int kThreads = 256;     // load
constexpr int kStoreThreads = 128, kStoreCtas = 8;
constexpr int kRows = 4;          // load: rows of K and V in flight per thread
constexpr int kPieces = 4;        // store: 16-byte pieces of a row per lane

// (a, b) rounded to two e4m3 codes, a in the low byte.
__device__ __forceinline__ uint32_t e4m3x2(float a, float b) {
  uint16_t v;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(v) : "f"(b), "f"(a));
  return v;
}

// 16 bytes of a source row as floats.
template <typename T> struct Piece;
template <> struct Piece<float> {
  static constexpr int V = 4;
  static __device__ __forceinline__ void get(const uint4& r, float (&x)[4]) {
    x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y); x[2] = __uint_as_float(r.z); x[3] = __uint_as_float(r.w);
  }
  static __device__ __forceinline__ uint4 put(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};
__device__ __forceinline__ uint32_t bf16x2(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <> struct Piece<__nv_bfloat16> {
  static constexpr int V = 8;
  static __device__ __forceinline__ void get(const uint4& r, float (&x)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 put(const float (&x)[8]) {
    return make_uint4(bf16x2(x[0], x[1]), bf16x2(x[2], x[3]), bf16x2(x[4], x[5]), bf16x2(x[6], x[7]));
  }
};

// Scale and codes of a row piece (criticalkv.h states the rule).  The row's largest magnitude is found on the bit
// patterns, whose order puts NaN above infinity, so a row with a NaN gets a NaN scale.
template <int FMT, int LANES, int N>
__device__ __forceinline__ float quantise(const float (&x)[N], uint32_t (&code)[N / 4]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  constexpr float kTop = FMT == CKV_CACHE_E4M3 ? 448.f : 127.f;
  float scale = __fdiv_rn(__uint_as_float(top), kTop);
  if (scale < kLeastScale) scale = kLeastScale;
  // a row that reaches the largest float must not read back as infinity because the quotient was rounded up
  if (top < 0x7f800000u && __fmul_rn(scale, kTop) == INFINITY) scale = __uint_as_float(__float_as_uint(scale) - 1);
  const float r = __frcp_rn(scale);
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    float y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = __fmul_rn(x[4 * i + j], r);
    if (FMT == CKV_CACHE_E4M3) {
      code[i] = e4m3x2(y[0], y[1]) | (e4m3x2(y[2], y[3]) << 16);
    } else {
      code[i] = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        code[i] |= ((uint32_t)min(max(__float2int_rn(y[j]), -127), 127) & 0xffu) << (8 * j);   // NaN becomes 0
    }
  }
  return scale;
}

struct StoreArgs {
  Pages c;
  const char* src[2];          // K, V
  long long ss[3];             // source byte strides: sequence, head, row
  int n;
  const int32_t* idx;
  const int32_t* offsets;
  long long idx_rows;
  const int32_t* counts;
  const int32_t* start;
  int32_t* lens_out;           // null: nothing to write, or left to the kernel that follows
  int chunks;                  // CTAs a head
  int* status;
};

// Rows of head `item` that the call writes, and where its part of idx begins.
__device__ __forceinline__ int rows_of(const StoreArgs& p, int s, int g, long long& first, bool& bad) {
  first = 0;
  if (p.idx != nullptr) {
    const long long lo = p.offsets[(long long)s * (p.c.Hkv + 1) + g], hi = p.offsets[(long long)s * (p.c.Hkv + 1) + g + 1];
    first = min(max(lo, 0LL), p.idx_rows);
    const long long last = min(max(hi, first), p.idx_rows);
    bad = lo != first || hi != last;
    return (int)(last - first);
  }
  if (p.counts == nullptr) return p.n;
  const int c = p.counts[s];
  bad = c < 0 || c > p.n;
  return min(max(c, 0), p.n);
}

__device__ __forceinline__ int32_t new_length(const StoreArgs& p, int item, int rows) {
  const long long m = (long long)p.start[item] + rows;
  return (int32_t)min(max(m, 0LL), p.c.capacity);
}

// Lanes that share a row in the store kernel.
constexpr int store_lanes(int row_bytes) { return row_bytes / (16 * kPieces); }

template <typename T, int FMT, int DH>
__global__ void __launch_bounds__(kStoreThreads, kStoreCtas) store_kernel(StoreArgs p) {
  wait_for_previous_kernel();
  constexpr int V = Piece<T>::V, LANES = store_lanes(DH * (int)sizeof(T)), ROWS = kStoreThreads / LANES;   // rows a pass
  const int item = blockIdx.x / p.chunks, chunk = blockIdx.x % p.chunks;
  const int s = item / p.c.Hkv, g = item % p.c.Hkv;
  const int lane = threadIdx.x % LANES, sub = threadIdx.x / LANES;
  long long first;
  bool bad = false;
  const int rows = rows_of(p, s, g, first, bad);
  const long long start = p.start[item];
  if (p.lens_out != nullptr) {
    __syncthreads();                      // lens_out may be start itself: every thread has read it
    if (chunk == 0 && threadIdx.x == 0) p.lens_out[item] = new_length(p, item, rows);
  }
  const int32_t* pages = p.c.table + (long long)item * p.c.max_pages;
  // where row r goes (page * page_size + row in it, -1: nowhere) and comes from
  auto find = [&](long long r, long long& slot, int& from) {
    slot = -1;
    from = 0;
    if (r >= rows) return;
    from = p.idx != nullptr ? p.idx[(long long)s * p.idx_rows + first + r] : (int)r;
    const long long to = start + r;
    if (to >= 0 && to < p.c.capacity && from >= 0 && from < p.n) {
      const int page = pages[to >> p.c.page_shift];
      if (page >= 0 && page < p.c.num_pages)
        slot = ((long long)page << p.c.page_shift) + (to & ((1 << p.c.page_shift) - 1));
    }
    bad = bad || slot < 0;
  };
  const int step = p.chunks * ROWS;
  long long base = (long long)chunk * ROWS, slot;
  int from;
  find(base + sub, slot, from);
  while (base < rows) {
    uint4 raw[2][kPieces];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const char* src = p.src[w] + s * p.ss[0] + g * p.ss[1] + from * p.ss[2] + lane * 16;
#pragma unroll
      for (int j = 0; j < kPieces; ++j) {
        raw[w][j] = make_uint4(0, 0, 0, 0);
        if (slot >= 0) raw[w][j] = *reinterpret_cast<const uint4*>(src + j * LANES * 16);
      }
    }
    base += step;
    long long slot_next;
    int from_next;
    find(base + sub, slot_next, from_next);               // in flight while this row is rounded and written
    const long long page_at = (slot >> p.c.page_shift) * p.c.page_stride;
    const int in_page = (int)(slot & ((1 << p.c.page_shift) - 1));
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      if constexpr (FMT == CKV_CACHE_PLAIN) {
        char* to = p.c.page[w] + page_at + in_page * (DH * (int)sizeof(T)) + lane * 16;
#pragma unroll
        for (int j = 0; j < kPieces; ++j)
          if (slot >= 0) *reinterpret_cast<uint4*>(to + j * LANES * 16) = raw[w][j];
      } else {
        float x[kPieces * V];
        uint32_t code[kPieces * V / 4];
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
          float piece[V];
          Piece<T>::get(raw[w][j], piece);
#pragma unroll
          for (int i = 0; i < V; ++i) x[V * j + i] = piece[i];
        }
        const float scale = quantise<FMT, LANES>(x, code);
        char* to = p.c.page[w] + page_at + in_page * DH + lane * V;
        if (slot >= 0) {
#pragma unroll
          for (int j = 0; j < kPieces; ++j) {
            if constexpr (V == 8)
              *reinterpret_cast<uint2*>(to + j * LANES * V) = make_uint2(code[2 * j], code[2 * j + 1]);
            else
              *reinterpret_cast<uint32_t*>(to + j * LANES * V) = code[j];
          }
          if (lane == 0) p.c.scale[w][slot] = scale;
        }
      }
    }
    slot = slot_next;
    from = from_next;
  }
  if (bad && p.status != nullptr) atomicExch(p.status, (int)CKV_EBOUNDS);
}

// lens_out = start + rows where several CTAs read start and lens_out is start itself.
__global__ void store_lengths_kernel(StoreArgs p, int items) {
  wait_for_previous_kernel();
  const int item = blockIdx.x * blockDim.x + threadIdx.x;
  if (item >= items) return;
  long long first;
  bool bad = false;
  const int rows = rows_of(p, item / p.c.Hkv, item % p.c.Hkv, first, bad);
  p.lens_out[item] = new_length(p, item, rows);
}

struct LoadArgs {
  Pages c;
  const int32_t* lens;
  char* dst[2];
  long long ds[3];             // destination byte strides: sequence, head, row
  int n;
  int align_right;
  int chunks;
  int* status;
};

template <typename T, int FMT, int DH>
__global__ void __launch_bounds__(kThreads) load_kernel(LoadArgs p) {
  wait_for_previous_kernel();
  constexpr int V = Piece<T>::V, LANES = DH / V, RPP = kThreads / LANES;
  const int item = blockIdx.x / p.chunks, chunk = blockIdx.x % p.chunks;
  const int s = item / p.c.Hkv, g = item % p.c.Hkv;
  const int lane = threadIdx.x % LANES, sub = threadIdx.x / LANES;
  const int given = p.lens[item];
  const int len = (int)min(max((long long)given, 0LL), p.c.capacity);
  bool bad = len != given;
  const int rows = min(len, p.n);
  const int from = p.align_right ? len - rows : 0;       // first row read
  const int at = p.align_right ? p.n - rows : 0;         // and where it goes
  const int32_t* pages = p.c.table + (long long)item * p.c.max_pages;
  const int step = RPP * kRows;
  for (long long base = (long long)chunk * step; base < rows; base += (long long)p.chunks * step) {
    long long slot[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const long long r = base + u * RPP + sub;
      slot[u] = -1;
      if (r < rows) {
        const int row = from + (int)r;
        const int page = pages[row >> p.c.page_shift];
        if (page >= 0 && page < p.c.num_pages)
          slot[u] = ((long long)page << p.c.page_shift) + (row & ((1 << p.c.page_shift) - 1));
        bad = bad || slot[u] < 0;
      }
    }
    if constexpr (FMT == CKV_CACHE_PLAIN) {
      uint4 raw[kRows][2];
#pragma unroll
      for (int u = 0; u < kRows; ++u)
#pragma unroll
        for (int w = 0; w < 2; ++w)
          if (slot[u] >= 0)
            raw[u][w] = *reinterpret_cast<const uint4*>(p.c.page[w] + (slot[u] >> p.c.page_shift) * p.c.page_stride +
                                                        (slot[u] & ((1 << p.c.page_shift) - 1)) * (DH * (int)sizeof(T)) +
                                                        lane * 16);
#pragma unroll
      for (int u = 0; u < kRows; ++u)
#pragma unroll
        for (int w = 0; w < 2; ++w)
          if (slot[u] >= 0)
            *reinterpret_cast<uint4*>(p.dst[w] + s * p.ds[0] + g * p.ds[1] + (at + base + u * RPP + sub) * p.ds[2] +
                                      lane * 16) = raw[u][w];
    } else {
      uint32_t code[kRows][2][V / 4];
      float scale[kRows][2];
#pragma unroll
      for (int u = 0; u < kRows; ++u)
#pragma unroll
        for (int w = 0; w < 2; ++w)
          if (slot[u] >= 0) {
            const char* row = p.c.page[w] + (slot[u] >> p.c.page_shift) * p.c.page_stride +
                              (slot[u] & ((1 << p.c.page_shift) - 1)) * DH + lane * V;
            if constexpr (V == 8) {
              const uint2 v = *reinterpret_cast<const uint2*>(row);
              code[u][w][0] = v.x;
              code[u][w][V / 4 - 1] = v.y;
            } else {
              code[u][w][0] = *reinterpret_cast<const uint32_t*>(row);
            }
            scale[u][w] = p.c.scale[w][slot[u]];
          }
#pragma unroll
      for (int u = 0; u < kRows; ++u)
#pragma unroll
        for (int w = 0; w < 2; ++w)
          if (slot[u] >= 0) {
            float x[V];
#pragma unroll
            for (int i = 0; i < V / 4; ++i) {
              float y[4];
              decode4<FMT>(code[u][w][i], y);
#pragma unroll
              for (int j = 0; j < 4; ++j) x[4 * i + j] = y[j] * scale[u][w];
            }
            *reinterpret_cast<uint4*>(p.dst[w] + s * p.ds[0] + g * p.ds[1] + (at + base + u * RPP + sub) * p.ds[2] +
                                      lane * 16) = Piece<T>::put(x);
          }
    }
  }
  if (bad && p.status != nullptr) atomicExch(p.status, (int)CKV_EBOUNDS);
}

// Calls f with the element type, the page format and the head dim as compile-time constants.
template <typename F> void by_type(const CacheDims& d, F&& f) {
  auto dims = [&](auto t, auto fmt) {
    if (d.dh == 64) f(t, fmt, std::integral_constant<int, 64>());
    else f(t, fmt, std::integral_constant<int, 128>());
  };
  auto formats = [&](auto t) {
    if (d.format == CKV_CACHE_PLAIN) dims(t, std::integral_constant<int, CKV_CACHE_PLAIN>());
    else if (d.format == CKV_CACHE_E4M3) dims(t, std::integral_constant<int, CKV_CACHE_E4M3>());
    else dims(t, std::integral_constant<int, CKV_CACHE_INT8>());
  };
  if (d.dtype == CKV_F32) formats(float());
  else formats(__nv_bfloat16());
}

// CTAs a head: one pass of `step` rows each for a head of `rows` rows (a longer head loops), bounded for the grid.
int chunks_for(long long rows, int step, long long items) {
  long long c = (rows + step - 1) / step;
  const long long most = 0x7fffffffLL / items;
  if (c > 4096) c = 4096;
  if (c > most) c = most;
  return c < 1 ? 1 : (int)c;
}

}  // namespace

cudaError_t launch_cache_store(const CacheDims& d, const void* K, const void* V, int n, const long long* stride,
                               const int32_t* idx, const int32_t* offsets, long long idx_rows, const int32_t* counts,
                               const int32_t* start, int32_t* lens_out, int sm_count, int* status_word,
                               cudaStream_t st, int* launches) {
  const int es = d.dtype == CKV_F32 ? 4 : 2;
  const long long items = (long long)d.nseq * d.Hkv;
  StoreArgs p;
  p.c = pages_of(d);
  p.src[0] = (const char*)K; p.src[1] = (const char*)V;
  for (int i = 0; i < 3; ++i) p.ss[i] = stride[i] * es;
  p.n = n; p.idx = idx; p.offsets = offsets; p.idx_rows = idx_rows; p.counts = counts; p.start = start;
  p.status = d.debug_checks ? status_word : nullptr;
  const int step = kStoreThreads / store_lanes(d.dh * es);
  p.chunks = chunks_for(idx ? (idx_rows + d.Hkv - 1) / d.Hkv : n, step, items);
  // three rounds of resident CTAs: enough to even out heads of different lengths, and every CTA but the last has a next
  // row to look up while it writes one (one, two, three, four rounds: 64.1, 60.6, 58.5, 58.4 us)
  const long long most = 3LL * sm_count * kStoreCtas / items;
  if (p.chunks > most) p.chunks = most < 1 ? 1 : (int)most;
  const bool later = lens_out == start && lens_out != nullptr && p.chunks > 1;
  p.lens_out = later ? nullptr : lens_out;
  cudaError_t e = cudaSuccess;
  by_type(d, [&](auto t, auto fmt, auto dh) {
    e = launch_early<StoreArgs>(store_kernel<decltype(t), decltype(fmt)::value, decltype(dh)::value>,
                                dim3((unsigned)(items * p.chunks)), kStoreThreads, 0, st, p);
  });
  *launches += 1;
  if (e != cudaSuccess || !later) return e;
  p.lens_out = lens_out;
  *launches += 1;
  return launch_early<StoreArgs, int>(store_lengths_kernel, dim3((unsigned)((items + 127) / 128)), 128, 0, st, p, (int)items);
}

cudaError_t launch_cache_load(const CacheDims& d, const int32_t* lens, int n, const long long* stride, int align_right,
                              void* K_out, void* V_out, int* status_word, cudaStream_t st, int* launches) {
  const int es = d.dtype == CKV_F32 ? 4 : 2;
  const long long items = (long long)d.nseq * d.Hkv;
  LoadArgs p;
  p.c = pages_of(d);
  p.lens = lens;
  p.dst[0] = (char*)K_out; p.dst[1] = (char*)V_out;
  for (int i = 0; i < 3; ++i) p.ds[i] = stride[i] * es;
  p.n = n; p.align_right = align_right;
  p.status = d.debug_checks ? status_word : nullptr;
  const int step = kThreads / (d.dh * es / 16) * kRows;
  p.chunks = chunks_for(n, step, items);
  cudaError_t e = cudaSuccess;
  by_type(d, [&](auto t, auto fmt, auto dh) {
    e = launch_early<LoadArgs>(load_kernel<decltype(t), decltype(fmt)::value, decltype(dh)::value>,
                               dim3((unsigned)(items * p.chunks)), kThreads, 0, st, p);
  });
  *launches += 1;
  return e;
}

}  // namespace ckv
