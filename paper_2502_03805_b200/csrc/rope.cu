// Rotary positions of query and key rows, both in one launch.
// Pair i of a row is turned by pos * freq[i]: (a, b) -> factor * (a cos - b sin, b cos + a sin).
//
// The angle is reduced to a fraction of a turn in float64 (pos * freq loses up to pos * 2^-24 radians in float32: 0.008
// at position 131072) and only then goes to sincospif.  All heads of a token share its rot/2 angles, so a CTA works on
// a tile of tokens, puts their cosines and sines into shared memory once and then streams the tokens' rows of every
// head: 16 bytes of a pair's first and second elements per thread, four such units in flight.  Bound by HBM (every
// row is read and written once).
#include <cuda_bf16.h>

#include "ckv_internal.h"

namespace ckv {
namespace {

constexpr int kThreads = 256;
constexpr int kUnits = 4;        // units in flight per thread

struct RopeArgs {
  const char* x[2];              // q, k
  char* y[2];
  long long xs[2][3], ys[2][3];  // byte strides: sequence, head, token
  const int32_t* pos;
  const double* freq;
  float factor;
  int T, Hq, H, dh, rot;         // H = Hq + Hk
  int tile, tiles;               // tokens a CTA, CTAs along the tokens of a sequence
  int heads;                     // heads a CTA
};

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

template <typename T> union Vec16 {
  uint4 raw;
  T e[16 / sizeof(T)];
};

// What one unit of a row covers: VEC units move 16-byte vectors, the others single elements (row parts that do not
// divide into vectors).
template <typename T, bool VEC, bool HALF>
__global__ void __launch_bounds__(kThreads) rope_kernel(RopeArgs p) {
  extern __shared__ float table[];              // cos [tile][rot/2], sin [tile][rot/2], both times factor
  constexpr int V = VEC ? 16 / (int)sizeof(T) : 1;
  const int pairs = p.rot / 2;
  const int s = blockIdx.x / p.tiles, t0 = (blockIdx.x % p.tiles) * p.tile;
  const int nt = min(p.tile, p.T - t0);
  const int h0 = blockIdx.y * p.heads, nh = min(p.heads, p.H - h0);
  float* cosine = table;
  float* sine = table + p.tile * pairs;

  // units of a row: first the rotated ones, then the copied ones
  const unsigned turned = (HALF || !VEC) ? pairs / V : p.rot / V;
  const unsigned units = turned + (p.dh - p.rot) / V;
  const unsigned total = (unsigned)nh * nt * units;

  auto locate = [&](unsigned i, const char*& src, char*& dst, unsigned& u, int& t) {
    u = i % units;
    const unsigned j = i / units;
    t = (int)(j % (unsigned)nt);
    int h = h0 + (int)(j / (unsigned)nt);
    const int which = h >= p.Hq;
    if (which) h -= p.Hq;
    src = p.x[which] + s * p.xs[which][0] + h * p.xs[which][1] + (long long)(t0 + t) * p.xs[which][2];
    dst = p.y[which] + s * p.ys[which][0] + h * p.ys[which][1] + (long long)(t0 + t) * p.ys[which][2];
  };

  for (int i = threadIdx.x; i < nt * pairs; i += kThreads) {
    const int t = i / pairs, f = i - t * pairs;
    const double turns = (double)p.pos[(long long)s * p.T + t0 + t] * (p.freq[f] * 0.15915494309189533577);
    float sn, cs;
    sincospif(2.f * (float)(turns - rint(turns)), &sn, &cs);
    cosine[t * pairs + f] = cs * p.factor;
    sine[t * pairs + f] = sn * p.factor;
  }
  __syncthreads();

  for (unsigned base = threadIdx.x; base < total; base += kThreads * kUnits) {
    if constexpr (VEC) {
      Vec16<T> a[kUnits], b[kUnits];
#pragma unroll
      for (int k = 0; k < kUnits; ++k) {
        const unsigned i = base + k * kThreads;
        if (i >= total) break;
        const char* src; char* dst; unsigned u; int t;
        locate(i, src, dst, u, t);
        if (HALF && u < turned) {
          a[k].raw = *reinterpret_cast<const uint4*>(src + u * 16);
          b[k].raw = *reinterpret_cast<const uint4*>(src + u * 16 + pairs * sizeof(T));
        } else {   // copied vectors of the half layout lie behind twice the rotated units
          a[k].raw = *reinterpret_cast<const uint4*>(src + (HALF ? u + turned : u) * 16);
        }
      }
#pragma unroll
      for (int k = 0; k < kUnits; ++k) {
        const unsigned i = base + k * kThreads;
        if (i >= total) break;
        const char* src; char* dst; unsigned u; int t;
        locate(i, src, dst, u, t);
        if (u >= turned) {
          *reinterpret_cast<uint4*>(dst + (HALF ? u + turned : u) * 16) = a[k].raw;
        } else if (HALF) {
          const float* cs = cosine + t * pairs + u * V;
          const float* sn = sine + t * pairs + u * V;
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float x = to_f32<T>(a[k].e[e]), y = to_f32<T>(b[k].e[e]);
            a[k].e[e] = from_f32<T>(x * cs[e] - y * sn[e]);
            b[k].e[e] = from_f32<T>(y * cs[e] + x * sn[e]);
          }
          *reinterpret_cast<uint4*>(dst + u * 16) = a[k].raw;
          *reinterpret_cast<uint4*>(dst + u * 16 + pairs * sizeof(T)) = b[k].raw;
        } else {
          const float* cs = cosine + t * pairs + u * (V / 2);
          const float* sn = sine + t * pairs + u * (V / 2);
#pragma unroll
          for (int e = 0; e < V / 2; ++e) {
            const float x = to_f32<T>(a[k].e[2 * e]), y = to_f32<T>(a[k].e[2 * e + 1]);
            a[k].e[2 * e] = from_f32<T>(x * cs[e] - y * sn[e]);
            a[k].e[2 * e + 1] = from_f32<T>(y * cs[e] + x * sn[e]);
          }
          *reinterpret_cast<uint4*>(dst + u * 16) = a[k].raw;
        }
      }
    } else {
      for (int k = 0; k < kUnits; ++k) {
        const unsigned i = base + k * kThreads;
        if (i >= total) break;
        const char* src; char* dst; unsigned u; int t;
        locate(i, src, dst, u, t);
        const T* xr = reinterpret_cast<const T*>(src);
        T* yr = reinterpret_cast<T*>(dst);
        if (u < turned) {
          const int ia = HALF ? u : 2 * u, ib = HALF ? u + pairs : 2 * u + 1;
          const float x = to_f32<T>(xr[ia]), y = to_f32<T>(xr[ib]);
          const float cs = cosine[t * pairs + u], sn = sine[t * pairs + u];
          yr[ia] = from_f32<T>(x * cs - y * sn);
          yr[ib] = from_f32<T>(y * cs + x * sn);
        } else {
          yr[p.rot + (u - turned)] = xr[p.rot + (u - turned)];
        }
      }
    }
  }
}

template <typename T>
cudaError_t launch_typed(const RopeArgs& p, int layout, dim3 grid, size_t smem, cudaStream_t st) {
  constexpr int V = 16 / (int)sizeof(T);
  // whole vectors only where the rotated part (each half of it in the half layout) divides into them
  const bool half = layout == CKV_ROPE_HALF;
  const bool vec = (half ? p.rot / 2 : p.rot) % V == 0;
  if (half) {
    if (vec) rope_kernel<T, true, true><<<grid, kThreads, smem, st>>>(p);
    else rope_kernel<T, false, true><<<grid, kThreads, smem, st>>>(p);
  } else {
    if (vec) rope_kernel<T, true, false><<<grid, kThreads, smem, st>>>(p);
    else rope_kernel<T, false, false><<<grid, kThreads, smem, st>>>(p);
  }
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_rope(const RopeDims& d, const void* q, const void* k, const int32_t* pos, const double* freq,
                        void* q_out, void* k_out, int sm_count, cudaStream_t st, int* launches) {
  const int es = d.dtype == CKV_F32 ? 4 : 2;
  RopeArgs p;
  p.x[0] = (const char*)q; p.x[1] = (const char*)k;
  p.y[0] = (char*)q_out; p.y[1] = (char*)k_out;
  for (int i = 0; i < 3; ++i) {
    p.xs[0][i] = d.qs[i] * es; p.xs[1][i] = d.ks[i] * es;
    p.ys[0][i] = d.qos[i] * es; p.ys[1][i] = d.kos[i] * es;
  }
  p.pos = pos; p.freq = freq; p.factor = d.factor;
  p.T = d.T; p.Hq = d.Hq; p.H = d.Hq + d.Hk; p.dh = d.dh; p.rot = d.rot;
  p.tile = d.T < 16 ? d.T : 16;
  p.tiles = (d.T + p.tile - 1) / p.tile;
  const long long ctas = (long long)p.tiles * d.nseq;
  if (ctas > 0x7fffffffLL) return cudaErrorInvalidValue;
  // few tokens: the heads are spread over CTAs too (each then computes the tile's angles again)
  long long split = (2LL * sm_count + ctas - 1) / ctas;
  const int most = (p.H + 3) / 4;       // at least four heads a CTA
  if (split > most) split = most;
  p.heads = (int)((p.H + split - 1) / split);
  const dim3 grid((unsigned)ctas, (unsigned)((p.H + p.heads - 1) / p.heads));
  const size_t smem = (size_t)p.tile * p.rot * sizeof(float);
  const cudaError_t e = d.dtype == CKV_F32 ? launch_typed<float>(p, d.layout, grid, smem, st)
                                           : launch_typed<__nv_bfloat16>(p, d.layout, grid, smem, st);
  *launches += 1;
  return e;
}

}  // namespace ckv
