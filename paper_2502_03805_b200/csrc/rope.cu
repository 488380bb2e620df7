// Rotary positions of query and key rows, both in one launch.
// Pair i of a row is turned by pos * freq[i]: (a, b) -> factor * (a cos - b sin, b cos + a sin).
//
// The angle is reduced to a fraction of a turn in float64 (pos * freq loses up to pos * 2^-24 radians in float32: 0.008
// at position 131072) and only then rounded, to within 2 pi 2^-26 radians, for sincospif; cosine and sine times `factor`
// and the products are float32.  All heads of a token share its rot/2 angles, so a thread owns
// one unit of one token's rows (half layout: 16 bytes of a pair's first elements and 16 of its second; interleaved: 16
// bytes), keeps the unit's cosines and sines in registers and walks over the heads, 64 bytes in flight, 32 warps an SM.
// Elements that are only copied form units of the same size.  Bound by HBM: every row is read and written once (32768
// tokens of 40 heads of 128 bf16: 106 us, 6.3 TB/s; four rows in flight on 16 warps: 153 us; a quarter of the elements
// turned: within 1 % of all of them, 22 % slower while copied units were 16 bytes).
#include <cuda_bf16.h>

#include "ckv_internal.h"
#include "launch_early.cuh"
#include "rotate.cuh"

namespace ckv {
namespace {

constexpr int kThreads = 256;

struct RopeArgs {
  const char* x[2];              // q, k
  char* y[2];
  long long xs[2][3], ys[2][3];  // byte strides: sequence, head, token
  const int32_t* pos;
  const double* freq;
  float factor;
  int T, heads[2], dh, rot;
  int units, tile, tiles;        // units a row; tokens a CTA, CTAs along the tokens of a sequence
  int groups;                    // threads that share a unit of a token and take turns at the heads
  int splits;                    // CTAs that share a tile of tokens and take turns at the heads
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

// Rows in flight per thread: 32 bytes of each (half layout, two rows), 16 bytes (interleaved, four), or an element or two.
constexpr int rows_in_flight(bool vec, bool half) { return vec && half ? 2 : 4; }

// VEC units move 16-byte vectors, the others single elements (row parts that do not divide into vectors).
template <typename T, bool VEC, bool HALF>
__global__ void __launch_bounds__(kThreads, 4) rope_kernel(RopeArgs p) {
  wait_for_previous_kernel();
  constexpr int V = VEC ? 16 / (int)sizeof(T) : 1;
  constexpr int P = (HALF || !VEC) ? V : V / 2;                // pairs a unit
  constexpr int kRows = rows_in_flight(VEC, HALF);
  const int pairs = p.rot / 2;
  const int turned = pairs / P;                                // units that are turned; the others are copied
  const int u = threadIdx.x % p.units, rest = threadIdx.x / p.units;
  const int tok = rest % p.tile, group = rest / p.tile;
  const int s = blockIdx.x / p.tiles, t = (blockIdx.x % p.tiles) * p.tile + tok;
  if (group >= p.groups || t >= p.T) return;
  const bool turn = u < turned;
  // element offsets of the unit's two parts; the copied vectors of the half layout go by two as well
  int ea, eb;
  bool two = turn;
  if (VEC && HALF) {
    const int copied = (p.dh - p.rot) / V, i = u - turned;
    ea = turn ? u * V : p.rot + i * V;
    eb = turn ? ea + pairs : ea + (copied + 1) / 2 * V;
    two = eb < p.dh;
  } else if (VEC) {
    ea = eb = u * V;
    two = false;
  } else {
    ea = turn ? (HALF ? u : 2 * u) : p.rot + u - turned;
    eb = HALF ? u + pairs : 2 * u + 1;
  }
  float cs[P], sn[P];
  bool ready = false;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const char* x = p.x[which] + s * p.xs[which][0] + (long long)t * p.xs[which][2];
    char* y = p.y[which] + s * p.ys[which][0] + (long long)t * p.ys[which][2];
    const int step = p.groups * p.splits;
    for (int h = blockIdx.y * p.groups + group; h < p.heads[which]; h += step * kRows) {
      Vec16<T> a[kRows], b[kRows];
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        const int hk = h + k * step;
        if (hk < p.heads[which]) {
          const T* row = reinterpret_cast<const T*>(x + hk * p.xs[which][1]);
          if (VEC) {
            a[k].raw = *reinterpret_cast<const uint4*>(row + ea);
            if (HALF && two) b[k].raw = *reinterpret_cast<const uint4*>(row + eb);
          } else {
            a[k].e[0] = row[ea];
            if (turn) b[k].e[0] = row[eb];
          }
        }
      }
      if (!ready) {                                            // behind the first loads
        ready = true;
        if (turn) {
          const double pos = (double)p.pos[(long long)s * p.T + t] * 0.15915494309189533577;
#pragma unroll
          for (int i = 0; i < P; ++i) {
            const double turns = pos * p.freq[u * P + i];
            sincospif(2.f * (float)(turns - rint(turns)), &sn[i], &cs[i]);
            cs[i] *= p.factor;
            sn[i] *= p.factor;
          }
        }
      }
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        const int hk = h + k * step;
        if (hk < p.heads[which]) {
          T* row = reinterpret_cast<T*>(y + hk * p.ys[which][1]);
          if (turn) {
#pragma unroll
            for (int i = 0; i < P; ++i) {
              T& ta = (VEC && !HALF) ? a[k].e[(2 * i) % (16 / (int)sizeof(T))] : a[k].e[i];
              T& tb = (VEC && !HALF) ? a[k].e[(2 * i + 1) % (16 / (int)sizeof(T))] : b[k].e[i];
              const float va = to_f32<T>(ta), vb = to_f32<T>(tb);
              ta = from_f32<T>(turned_first(va, vb, cs[i], sn[i]));
              tb = from_f32<T>(turned_second(va, vb, cs[i], sn[i], VEC && sizeof(T) == 2));
            }
          }
          if (VEC) {
            *reinterpret_cast<uint4*>(row + ea) = a[k].raw;
            if (HALF && two) *reinterpret_cast<uint4*>(row + eb) = b[k].raw;
          } else {
            row[ea] = a[k].e[0];
            if (turn) row[eb] = b[k].e[0];
          }
        }
      }
    }
  }
}

template <typename T>
cudaError_t launch_typed(RopeArgs p, int layout, int nseq, int sm_count, cudaStream_t st) {
  constexpr int V = 16 / (int)sizeof(T);
  // whole vectors only where the rotated part (each half of it in the half layout) divides into them
  const bool half = layout == CKV_ROPE_HALF;
  const bool vec = (half ? p.rot / 2 : p.rot) % V == 0;
  p.units = !vec ? p.rot / 2 + p.dh - p.rot                                     // at most 256
            : half ? p.rot / 2 / V + ((p.dh - p.rot) / V + 1) / 2 : p.dh / V;
  p.tile = kThreads / p.units < p.T ? kThreads / p.units : p.T;
  p.tiles = (p.T + p.tile - 1) / p.tile;
  p.groups = kThreads / (p.units * p.tile);
  const int most = p.heads[0] > p.heads[1] ? p.heads[0] : p.heads[1];
  if (p.groups > most) p.groups = most;
  const long long ctas = (long long)p.tiles * nseq;
  if (ctas > 0x7fffffffLL) return cudaErrorInvalidValue;
  // heads are spread over CTAs as well until every SM has eight (each of them computes the tile's angles again), but
  // not below the rows a thread has in flight
  const int per_turn = p.groups * rows_in_flight(vec, half), turns = (most + per_turn - 1) / per_turn;
  p.splits = (int)((8LL * sm_count + ctas - 1) / ctas);
  if (p.splits > turns) p.splits = turns;
  const dim3 grid((unsigned)ctas, (unsigned)p.splits);
  const auto kernel = half ? (vec ? rope_kernel<T, true, true> : rope_kernel<T, false, true>)
                           : (vec ? rope_kernel<T, true, false> : rope_kernel<T, false, false>);
  return launch_early<RopeArgs>(kernel, grid, kThreads, 0, st, p);
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
  p.T = d.T; p.heads[0] = d.Hq; p.heads[1] = d.Hk; p.dh = d.dh; p.rot = d.rot;
  const cudaError_t e = d.dtype == CKV_F32 ? launch_typed<float>(p, d.layout, d.nseq, sm_count, st)
                                           : launch_typed<__nv_bfloat16>(p, d.layout, d.nseq, sm_count, st);
  *launches += 1;
  return e;
}

}  // namespace ckv
