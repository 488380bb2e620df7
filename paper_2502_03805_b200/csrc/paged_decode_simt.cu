// Decode attention on CUDA cores: float32 queries (whose products tensor cores would round), and CKV_FLAG_FORCE_SIMT.
//
// A warp takes 16 rows of a 64-row tile.  Logits: the four lanes of a quad share rows r and r + 8, each with a quarter
// of the elements, the queries come from shared memory (one 16-byte read per 8 products).  Softmax: lane = (query row,
// two or four cache rows), running maximum and sum in float32.  Values: a lane owns four elements and keeps the sums of
// all query rows of the item (four, or eight where the group is larger: half the products of a group of four would be of
// rows that do not exist), the weights come from shared memory.  Products, weights and sums are float32 throughout; the
// scale enters with the rest of its rounding, and only the difference of a logit to the maximum is rounded.
// Half of the values and the page of the next rows are loaded before the logits.
//
// Measured (8 x 6553 rows a head, 8 KV heads): float32 rows of 128, four queries a head, 79 us, 5.5 TB/s (0.85 of the copy
// bandwidth; 119 us without the early loads and with items of eight); e4m3 rows 62 us (floor 17).  That is latency, not
// products: 2.2 instructions a cycle and SM, and most of a warp's stalls wait for its 4-byte loads and the shared-memory
// round trips of logits and weights, with 15 warps an SM to hide them.
#include <cuda_bf16.h>

#include "paged_decode.cuh"

namespace ckv {
namespace {

constexpr int kTile = 64, kWarpRows = kTile / kDecodeWarps;   // cache rows a tile and a warp

// Four consecutive elements of a stored row, at element offset e.
template <typename T, int FMT> struct Four {
  uint32_t w[FMT == CKV_CACHE_PLAIN ? sizeof(T) : 1];
  uint32_t g;                                   // e2m1: scale of the group
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (unsigned i = 0; i < sizeof(w) / 4; ++i) w[i] = 0;
    g = 0;
  }
  __device__ __forceinline__ void load(const char* row, const uint8_t* groups, int e) {
    if constexpr (FMT == CKV_CACHE_E2M1) {
      w[0] = *reinterpret_cast<const uint16_t*>(row + e / 2);
      g = groups[e / 16];
    } else if constexpr (FMT != CKV_CACHE_PLAIN) {
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
      if constexpr (FMT == CKV_CACHE_E2M1) {
        const float s = e4m3_to_float(g);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] *= s;
      }
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

template <int DH, int kQ> struct Shared {   // kQ: query rows an item
  float q[kQ][DH];
  float s[kDecodeWarps][kQ][kWarpRows + 4];     // logits before the scale
  float w[kDecodeWarps][kWarpRows][kQ];         // weights
  float f[kDecodeWarps][kQ];                    // rescaling of the sums
  float o[kDecodeWarps][kQ][DH];
  float m[kDecodeWarps][kQ], l[kDecodeWarps][kQ];
  alignas(8) float parts[kQ][DH + 2];           // of a CTA of a team
};

// CTAs an SM: four where the sums of four query rows leave the registers for it, three with eight (two to four measured)
template <typename T, int FMT, int DH, int kQ>
__global__ void __launch_bounds__(kDecodeThreads, kQ == 4 ? 4 : 3) decode_simt_kernel(DecodeArgs p) {
  constexpr int ROW_BYTES = FMT == CKV_CACHE_PLAIN ? DH * (int)sizeof(T) : FMT == CKV_CACHE_E2M1 ? DH / 2 : DH;
  constexpr int PIECES = DH / 16;               // pieces of four elements a quad lane has of a row
  constexpr int LPR = DH / 4, KPI = 32 / LPR;   // values: lanes a row, rows at a time
  constexpr int WL = 32 / kQ, WR = kWarpRows / WL;   // weights: lanes a query row, cache rows a lane
  __shared__ __align__(16) Shared<DH, kQ> sh;      // read and written 16 bytes at a time
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  wait_for_previous_kernel();
  const Walk walk = p.team ? team_walk<T, DH, kTile>(p) : plan<T, DH, kTile>(p);
  if (threadIdx.x < kQ) *reinterpret_cast<float2*>(&sh.parts[threadIdx.x][DH]) = make_float2(-INFINITY, 0.f);
  int2 join = make_int2(-1, 0);
  int first = walk.first, t = walk.begin;
  for (int item = walk.item; t < walk.end; ++item) {
    const ItemRows it = item_rows(p, item);
    const int len = item_len(p, it.kv);
    const int tiles = (len + kTile - 1) / kTile;
    if (first + tiles <= t) { first += tiles; continue; }
    const int t0 = t - first, t1 = min(tiles, walk.end - first);

    __syncthreads();
    for (int i = threadIdx.x; i < kQ * DH; i += kDecodeThreads) {
      const int r = i / DH, e = i % DH;
      float v = 0.f;
      if (r < it.rows) v = (float)reinterpret_cast<const T*>(p.q + it.s * p.qs[0] + (it.head + r) * p.qs[1])[e];
      sh.q[r][e] = v;
    }
    __syncthreads();

    const int row = lane >> 2, c = lane & 3;    // logits: cache rows row, row + 8
    const int wq = lane / WL, wr = lane % WL * WR;   // weights: query row wq, cache rows wr...
    float m = -INFINITY, l = 0.f;               // of query row wq; l holds this lane's share of the sum
    float acc[kQ][4];
#pragma unroll
    for (int r = 0; r < kQ; ++r)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[r][e] = 0.f;

    const int32_t* pages = p.c.table + (long long)it.kv * p.c.max_pages;
    const auto page_of = [&](int tile) {        // page_size is a multiple of 16: a warp's rows lie in one page
      const int base = tile * kTile + warp * kWarpRows;
      return tile < t1 && base < len ? pages[base >> p.c.page_shift] : 0;
    };
    int page = page_of(t0);
    for (int tile = t0; tile < t1; ++tile) {
      const int base = tile * kTile + warp * kWarpRows;
      const int here = min(len - base, kWarpRows);
      if (here <= 0) break;
      const int at_page = page;
      page = page_of(tile + 1);
      if (at_page < 0 || at_page >= p.c.num_pages) {
        if (p.status != nullptr) atomicExch(p.status, (int)CKV_EBOUNDS);
        continue;
      }
      const int in_page = base & ((1 << p.c.page_shift) - 1);
      const long long off = at_page * p.c.page_stride + (long long)in_page * ROW_BYTES;
      const long long slot = ((long long)at_page << p.c.page_shift) + in_page;
      const char* K = p.c.page[0] + off;
      const char* V = p.c.page[1] + off;
      const uint8_t* gk = FMT == CKV_CACHE_E2M1 ? p.c.group[0] + slot * (DH / 16) : nullptr;
      const uint8_t* gv = FMT == CKV_CACHE_E2M1 ? p.c.group[1] + slot * (DH / 16) : nullptr;

      // ---- logits
      Four<T, FMT> k[2][PIECES];
      float ks[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int i = row + 8 * h;
        ks[h] = (FMT != CKV_CACHE_PLAIN && i < here) ? p.c.scale[0][slot + i] : 1.f;
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
          if (i < here) k[h][j].load(K + i * ROW_BYTES, gk + i * (DH / 16), 4 * c + 16 * j);
          else k[h][j].clear();
        }
      }
      Four<T, FMT> v[8 / KPI];
      const auto load_v = [&](int b) {
#pragma unroll
        for (int j = 0; j < 8 / KPI; ++j) {
          const int i = b + j * KPI + lane / LPR;
          if (i < here) v[j].load(V + i * ROW_BYTES, gv + i * (DH / 16), 4 * (lane % LPR));
          else v[j].clear();
        }
      };
      load_v(0);
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
          if ((r >> 1) == c) sh.s[warp][r][row + 8 * h] = row + 8 * h < here ? v * ks[h] : -INFINITY;
        }
      __syncwarp();

      // ---- weights
      float ls[WR];
#pragma unroll
      for (int j = 0; j < WR; ++j) ls[j] = sh.s[warp][wq][wr + j];
      float top = ls[0];
#pragma unroll
      for (int j = 1; j < WR; ++j) top = fmaxf(top, ls[j]);
#pragma unroll
      for (int o = 1; o < WL; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      top = fmaxf(top * p.scale_log2, m);
      const float f = rescale(m, top);
      m = top;
      l *= f;
#pragma unroll
      for (int j = 0; j < WR; ++j) {
        // the difference to the maximum is rounded, not the logit: fma, and both parts of the factor
        const float w = ls[j] == -INFINITY ? 0.f : exp2f(fmaf(ls[j], p.scale_log2, -top) + ls[j] * p.scale_rest);
        l += w;
        float vs = 1.f;
        if (FMT != CKV_CACHE_PLAIN && wr + j < here) vs = p.c.scale[1][slot + wr + j];
        sh.w[warp][wr + j][wq] = w * vs;
      }
      if (wr == 0) sh.f[warp][wq] = f;
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
        if (b > 0) load_v(b);
#pragma unroll
        for (int j = 0; j < 8 / KPI; ++j) {
          const int i = b + j * KPI + lane / LPR;
          float w[kQ];
#pragma unroll
          for (int r = 0; r < kQ; r += 4) {
            const float4 w4 = *reinterpret_cast<const float4*>(&sh.w[warp][i][r]);
            w[r] = w4.x; w[r + 1] = w4.y; w[r + 2] = w4.z; w[r + 3] = w4.w;
          }
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

#pragma unroll
    for (int o = 1; o < WL; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    if (wr == 0) { sh.m[warp][wq] = m; sh.l[warp][wq] = l; }
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
    finish<T, DH, kQ>(p, it, &sh.o[0][0][0], &sh.m[0][0], &sh.l[0][0], 0, t0 == 0 && t1 == tiles,
                      p.team ? &sh.parts[0][0] : part_slot(p, DH, blockIdx.x, t0 > 0 ? 0 : 1));
    if (t0 > 0 && t1 == tiles) join = make_int2(item, cta_of(walk, first));
    t = first + t1;
    first += tiles;
  }
  if (p.team) join_team<T, DH>(p, walk, &sh.parts[0][0]);
  else if (threadIdx.x == 0) p.join[blockIdx.x] = join;
}

template <typename T, int FMT, int DH, int kQ> cudaError_t launch_rows(DecodeArgs p, int device, int sm_count, cudaStream_t st,
                                                                               int* launches) {
  const auto kernel = decode_simt_kernel<T, FMT, DH, kQ>;
  static LaunchSetup setup;
  const LaunchSetup::Fit* fit = setup.of(kernel, device, 0);
  if (!fit) return cudaErrorInvalidDeviceFunction;
  p.team = decode_team(p, *fit, sm_count, kTile);
  const int grid = p.team ? p.items * p.team : decode_grid(p, fit->per_sm * sm_count, kTile);
  *launches += 1;
  const cudaError_t e = launch_early_in_clusters<DecodeArgs>(kernel, dim3(grid), kDecodeThreads, 0, p.team, st, p);
  if (e != cudaSuccess || p.team) return e;
  *launches += 1;
  return launch_decode_join<T, DH>(p, grid, st);
}

template <typename T, int FMT, int DH> cudaError_t launch(const DecodeArgs& p, int device, int sm_count, cudaStream_t st, int* launches) {
  return p.chunk_rows == 4 ? launch_rows<T, FMT, DH, 4>(p, device, sm_count, st, launches)
                           : launch_rows<T, FMT, DH, 8>(p, device, sm_count, st, launches);
}

template <typename T> cudaError_t by_format(const DecodeArgs& p, int format, int dh, int device, int sm_count, cudaStream_t st,
                                             int* launches) {
  if (format == CKV_CACHE_PLAIN)
    return dh == 64 ? launch<T, CKV_CACHE_PLAIN, 64>(p, device, sm_count, st, launches) : launch<T, CKV_CACHE_PLAIN, 128>(p, device, sm_count, st, launches);
  if (format == CKV_CACHE_E4M3)
    return dh == 64 ? launch<T, CKV_CACHE_E4M3, 64>(p, device, sm_count, st, launches) : launch<T, CKV_CACHE_E4M3, 128>(p, device, sm_count, st, launches);
  if (format == CKV_CACHE_E2M1)
    return dh == 64 ? launch<T, CKV_CACHE_E2M1, 64>(p, device, sm_count, st, launches) : launch<T, CKV_CACHE_E2M1, 128>(p, device, sm_count, st, launches);
  return dh == 64 ? launch<T, CKV_CACHE_INT8, 64>(p, device, sm_count, st, launches) : launch<T, CKV_CACHE_INT8, 128>(p, device, sm_count, st, launches);
}

}  // namespace

size_t decode_workspace_bytes(const CacheDims& d) {
  const int G = d.Hq / d.Hkv;
  const size_t rows = G < 16 ? G : 16;                   // the most an item of either kernel has
  return (kDecodeMaxCtas * (sizeof(int2) + 2 * rows * (d.dh + 2) * sizeof(float)) + 255) / 256 * 256;
}

cudaError_t launch_decode_simt(const CacheDims& d, const DecodeCall& call, int device, int sm_count, int* status_word, cudaStream_t st,
                               int* launches) {
  const DecodeArgs p = decode_args(d, call, d.Hq / d.Hkv <= 4 ? 4 : 8, status_word);
  return d.dtype == CKV_F32 ? by_format<float>(p, d.format, d.dh, device, sm_count, st, launches)
                            : by_format<__nv_bfloat16>(p, d.format, d.dh, device, sm_count, st, launches);
}

}  // namespace ckv
