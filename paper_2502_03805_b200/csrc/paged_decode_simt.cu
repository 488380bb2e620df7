// Decode attention on CUDA cores: float32 queries (whose products tensor cores would round), and CKV_FLAG_FORCE_SIMT.
//
// A warp takes 16 rows of a 64-row tile.  Logits: the four lanes of a quad share rows r and r + 8, each with a quarter
// of the elements, the queries come from shared memory (one 16-byte read per 8 products).  Softmax: lane = (query row,
// four cache rows), running maximum and sum in float32.  Values: a lane owns four elements and keeps the sums of all
// eight query rows, the weights come from shared memory.  Products, weights and sums are float32 throughout.
#include <cuda_bf16.h>

#include "paged_decode.cuh"

namespace ckv {
namespace {

constexpr int kTile = 64, kWarpRows = kTile / kDecodeWarps, kQ = 8;   // cache rows a tile and a warp, query rows a chunk

// Four consecutive elements of a stored row, at element offset e.
template <typename T, int FMT> struct Four {
  uint32_t w[FMT == CKV_CACHE_PLAIN ? sizeof(T) : 1];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (unsigned i = 0; i < sizeof(w) / 4; ++i) w[i] = 0;
  }
  __device__ __forceinline__ void load(const char* row, int e) {
    if constexpr (FMT != CKV_CACHE_PLAIN) {
      w[0] = *reinterpret_cast<const uint32_t*>(row + e);
    } else if constexpr (sizeof(T) == 2) {
      const uint2 v = *reinterpret_cast<const uint2*>(row + e * 2);
      w[0] = v.x; w[1] = v.y;
    } else {
      const uint4 v = *reinterpret_cast<const uint4*>(row + e * 4);
      w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    }
  }
  __device__ __forceinline__ void get(float (&x)[4]) const {
    if constexpr (FMT != CKV_CACHE_PLAIN) {
      decode4<FMT>(w[0], x);
    } else if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
    }
  }
};

template <typename T, int FMT, int DH> struct Shared {
  float q[kQ][DH];
  float s[kDecodeWarps][kQ][kWarpRows + 4];     // logits
  float w[kDecodeWarps][kWarpRows][kQ];         // weights
  float f[kDecodeWarps][kQ];                    // rescaling of the sums
  float o[kDecodeWarps][kQ][DH];
  float m[kDecodeWarps][kQ], l[kDecodeWarps][kQ];
};

template <typename T, int FMT, int DH>
__global__ void __launch_bounds__(kDecodeThreads) decode_simt_kernel(DecodeArgs p) {
  constexpr int ROW_BYTES = DH * (FMT == CKV_CACHE_PLAIN ? (int)sizeof(T) : 1);
  constexpr int PIECES = DH / 16;               // pieces of four elements a quad lane has of a row
  constexpr int LPR = DH / 4, KPI = 32 / LPR;   // values: lanes a row, rows at a time
  __shared__ __align__(16) Shared<T, FMT, DH> sh;      // read and written 16 bytes at a time
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  wait_for_previous_kernel();
  const Walk walk = plan<T, DH, kTile>(p);
  int2 join = make_int2(-1, 0);
  long long first = walk.first, t = walk.begin;
  for (int item = walk.item; t < walk.end; ++item) {
    const ItemRows it = item_rows(p, item);
    const int len = item_len(p, it.kv);
    const int tiles = (len + kTile - 1) / kTile;
    if (first + tiles <= t) { first += tiles; continue; }
    const int t0 = (int)(t - first), t1 = (int)min((long long)tiles, walk.end - first);

    __syncthreads();
    for (int i = threadIdx.x; i < kQ * DH; i += kDecodeThreads) {
      const int r = i / DH, e = i % DH;
      float v = 0.f;
      if (r < it.rows) v = (float)reinterpret_cast<const T*>(p.q + it.s * p.qs[0] + (it.head + r) * p.qs[1])[e];
      sh.q[r][e] = v;
    }
    __syncthreads();

    const int row = lane >> 2, c = lane & 3;
    float m = -INFINITY, l = 0.f;               // of query row `row`; l holds this lane's share of the sum
    float acc[kQ][4];
#pragma unroll
    for (int r = 0; r < kQ; ++r)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[r][e] = 0.f;

    for (int tile = t0; tile < t1; ++tile) {
      const int base = tile * kTile + warp * kWarpRows;
      int here = min(len - base, kWarpRows);    // page_size is a multiple of 16: the rows lie in one page
      if (here <= 0) break;
      const int page = p.c.table[(long long)it.kv * p.c.max_pages + (base >> p.c.page_shift)];
      if (page < 0 || page >= p.c.num_pages) {
        if (p.status != nullptr) atomicExch(p.status, (int)CKV_EBOUNDS);
        continue;
      }
      const int in_page = base & ((1 << p.c.page_shift) - 1);
      const long long off = page * p.c.page_stride + (long long)in_page * ROW_BYTES;
      const long long slot = ((long long)page << p.c.page_shift) + in_page;
      const char* K = p.c.page[0] + off;
      const char* V = p.c.page[1] + off;

      // ---- logits
      Four<T, FMT> k[2][PIECES];
      float ks[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int i = row + 8 * h;
        ks[h] = (FMT != CKV_CACHE_PLAIN && i < here) ? p.c.scale[0][slot + i] : 1.f;
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
          if (i < here) k[h][j].load(K + i * ROW_BYTES, 4 * c + 16 * j);
          else k[h][j].clear();
        }
      }
      float s[kQ][2];
#pragma unroll
      for (int r = 0; r < kQ; ++r) s[r][0] = s[r][1] = 0.f;
#pragma unroll
      for (int j = 0; j < PIECES; ++j) {
        float x[2][4];
        k[0][j].get(x[0]);
        k[1][j].get(x[1]);
#pragma unroll
        for (int r = 0; r < kQ; ++r) {
          const float4 q = *reinterpret_cast<const float4*>(&sh.q[r][4 * c + 16 * j]);
#pragma unroll
          for (int h = 0; h < 2; ++h)
            s[r][h] += q.x * x[h][0] + q.y * x[h][1] + q.z * x[h][2] + q.w * x[h][3];
        }
      }
#pragma unroll
      for (int r = 0; r < kQ; ++r)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float v = s[r][h];
          v += __shfl_xor_sync(0xffffffffu, v, 1);
          v += __shfl_xor_sync(0xffffffffu, v, 2);
          if ((r >> 1) == c) sh.s[warp][r][row + 8 * h] = row + 8 * h < here ? v * ks[h] * p.scale_log2 : -INFINITY;
        }
      __syncwarp();

      // ---- weights: lane = (query row `row`, cache rows 4c..4c+3)
      const float4 sv = *reinterpret_cast<const float4*>(&sh.s[warp][row][4 * c]);
      const float ls[4] = {sv.x, sv.y, sv.z, sv.w};
      float top = fmaxf(fmaxf(ls[0], ls[1]), fmaxf(ls[2], ls[3]));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      top = fmaxf(top, m);
      const float f = rescale(m, top);
      m = top;
      l *= f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float w = ls[j] == -INFINITY ? 0.f : exp2f(ls[j] - top);
        l += w;
        float vs = 1.f;
        if (FMT != CKV_CACHE_PLAIN && 4 * c + j < here) vs = p.c.scale[1][slot + 4 * c + j];
        sh.w[warp][4 * c + j][row] = w * vs;
      }
      if (c == 0) sh.f[warp][row] = f;
      __syncwarp();

      // ---- values
#pragma unroll
      for (int r = 0; r < kQ; ++r) {
        const float g = sh.f[warp][r];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[r][e] *= g;
      }
#pragma unroll
      for (int b = 0; b < kWarpRows; b += 8) {
        Four<T, FMT> v[8 / KPI];
#pragma unroll
        for (int j = 0; j < 8 / KPI; ++j) {
          const int i = b + j * KPI + lane / LPR;
          if (i < here) v[j].load(V + i * ROW_BYTES, 4 * (lane % LPR));
          else v[j].clear();
        }
#pragma unroll
        for (int j = 0; j < 8 / KPI; ++j) {
          const int i = b + j * KPI + lane / LPR;
          const float4 w0 = *reinterpret_cast<const float4*>(&sh.w[warp][i][0]);
          const float4 w1 = *reinterpret_cast<const float4*>(&sh.w[warp][i][4]);
          const float w[kQ] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
          float x[4];
          v[j].get(x);
#pragma unroll
          for (int r = 0; r < kQ; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[r][e] += w[r] * x[e];
        }
      }
      __syncwarp();
    }

    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
    if (c == 0) { sh.m[warp][row] = m; sh.l[warp][row] = l; }
#pragma unroll
    for (int r = 0; r < kQ; ++r) {
      if (KPI == 2) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[r][e] += __shfl_xor_sync(0xffffffffu, acc[r][e], 16);
      }
      if (lane < LPR)
        *reinterpret_cast<float4*>(&sh.o[warp][r][4 * lane]) = make_float4(acc[r][0], acc[r][1], acc[r][2], acc[r][3]);
    }
    __syncthreads();
    finish<T, DH, kQ>(p, it, &sh.o[0][0][0], &sh.m[0][0], &sh.l[0][0], 0, t0 == 0 && t1 == tiles, t0 > 0 ? 0 : 1);
    if (t0 > 0 && t1 == tiles) join = make_int2(item, cta_of(walk, first));
    t = first + t1;
    first += tiles;
  }
  if (threadIdx.x == 0) p.join[blockIdx.x] = join;
}

template <typename T, int FMT, int DH> cudaError_t launch(DecodeArgs p, int device, int sm_count, cudaStream_t st) {
  static LaunchSetup setup;
  const int per_sm = setup.resident(decode_simt_kernel<T, FMT, DH>, device, 0);
  if (per_sm < 1) return cudaErrorInvalidDeviceFunction;
  cudaError_t e;
  const int grid = decode_grid(p, per_sm * sm_count, kTile);
  e = launch_early<DecodeArgs>(decode_simt_kernel<T, FMT, DH>, dim3(grid), kDecodeThreads, 0, st, p);
  if (e != cudaSuccess) return e;
  return launch_decode_join<T, DH>(p, grid, st);
}

template <typename T> cudaError_t by_format(const DecodeArgs& p, int format, int dh, int device, int sm_count, cudaStream_t st) {
  if (format == CKV_CACHE_PLAIN)
    return dh == 64 ? launch<T, CKV_CACHE_PLAIN, 64>(p, device, sm_count, st) : launch<T, CKV_CACHE_PLAIN, 128>(p, device, sm_count, st);
  if (format == CKV_CACHE_E4M3)
    return dh == 64 ? launch<T, CKV_CACHE_E4M3, 64>(p, device, sm_count, st) : launch<T, CKV_CACHE_E4M3, 128>(p, device, sm_count, st);
  return dh == 64 ? launch<T, CKV_CACHE_INT8, 64>(p, device, sm_count, st) : launch<T, CKV_CACHE_INT8, 128>(p, device, sm_count, st);
}

}  // namespace

size_t decode_workspace_bytes(const CacheDims& d) {
  const int G = d.Hq / d.Hkv;
  const size_t rows = G < 16 ? G : 16;                   // the most an item of either kernel has
  return (kDecodeMaxCtas * (sizeof(int2) + 2 * rows * (d.dh + 2) * sizeof(float)) + 255) / 256 * 256;
}

cudaError_t launch_decode_simt(const CacheDims& d, const DecodeCall& call, int device, int sm_count, int* status_word, cudaStream_t st,
                               int* launches) {
  const DecodeArgs p = decode_args(d, call, kQ, status_word);
  *launches += 2;
  return d.dtype == CKV_F32 ? by_format<float>(p, d.format, d.dh, device, sm_count, st)
                            : by_format<__nv_bfloat16>(p, d.format, d.dh, device, sm_count, st);
}

}  // namespace ckv
