// New tokens on their way into the paged cache, in one launch: queries and keys rotated, keys and values written (quantised
// where the pages are) behind the rows that their heads hold.
//
// The rotation is that of rope.cu (angles reduced in float64; cosine and sine in float32; rotate.cuh), the rounding of a rotated row
// to the model's type and the scales and codes are those of rope and store one behind the other: the pages get the same bits,
// but the keys do not travel through memory in between.  A thread owns 16 elements of a row: eight of a half-layout pair's
// first elements and the eight second ones, or 16 neighbours, so that rotation needs no other lane; it keeps their angles in
// registers and walks over the rows of its token, two at a time: two query rows, or the key and the value row of a head.
// Bound by HBM: every row is read and written once.  32768 tokens of 32 + 8 heads of 128 bf16 into plain pages: 130 us, 6.2 TB/s
// (rope and store one behind the other: 107 + 45 us); into 4-bit pages 143 us (floor 109; no unit is full: ALU 41 %, 22 warps an
// SM on 80 registers).  One token: 2.7 us, a chain of latencies.
// Turned parts that are no multiple of 16 take a kernel of 16 angles a thread that reads a pair's other element by itself, with
// up to 344 bytes spilled: slower than rope and store, whose kernels move whole vectors for some of these (32768 tokens, plain bf16,
// 20 elements turned 455 us, rope and store 374; 24 interleaved 447 and 150, into 4-bit pages 503 and 141; float32, 24 in the half
// layout 644 and 289; one token 5.9 and 3.6, 36 in the half layout 6.8 and 3.6).
#include "launch_early.cuh"
#include "paged_codes.cuh"
#include "rotate.cuh"

namespace ckv {
namespace {

constexpr int kThreads = 256;
constexpr int kOwn = 16;           // elements of a row a thread owns, in two pieces of eight

struct AppendArgs {
  Pages c;
  const char* x[3];                // q, k, v
  long long xs[3][3];              // byte strides: sequence, head, token
  char* q_out;
  long long qos[3];
  const int32_t* pos;
  const double* freq;
  float factor;
  const int32_t* counts;
  const int32_t* start;
  int32_t* lens_out;               // null: nothing to write, or left to the kernel that follows
  int T, Hq, rot, layout;
  int lanes;                       // threads a row
  int tile, tiles;                 // tokens a CTA, CTAs along the tokens of a sequence
  int groups, splits;              // threads of a CTA that share a piece of a token and take turns at its rows; CTAs that do
  int q_jobs, jobs;                // pairs of query rows; and heads of K and V
  int* status;
};

enum { kHalf, kInterleaved, kAnyPair };   // the last: pairs that do not divide into pieces of eight

// Eight elements as floats, and back.
template <typename T> struct Eight {
  static constexpr int N = 8 / Piece<T>::V;
  uint4 raw[N];
  __device__ __forceinline__ void load(const char* at) {
#pragma unroll
    for (int i = 0; i < N; ++i) raw[i] = *reinterpret_cast<const uint4*>(at + 16 * i);
  }
  __device__ __forceinline__ void store(char* at) const {
#pragma unroll
    for (int i = 0; i < N; ++i) *reinterpret_cast<uint4*>(at + 16 * i) = raw[i];
  }
  __device__ __forceinline__ void get(float* x) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float y[Piece<T>::V];
      Piece<T>::get(raw[i], y);
#pragma unroll
      for (int j = 0; j < Piece<T>::V; ++j) x[Piece<T>::V * i + j] = y[j];
    }
  }
  __device__ __forceinline__ void put(const float* x) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float y[Piece<T>::V];
#pragma unroll
      for (int j = 0; j < Piece<T>::V; ++j) y[j] = x[Piece<T>::V * i + j];
      raw[i] = Piece<T>::put(y);
    }
  }
  // The elements from the even number `turned` on as they were in `was`: through a float and back a NaN of a bf16 becomes another.
  __device__ __forceinline__ void keep(const Eight& was, int turned) {
    if constexpr (sizeof(T) == 2) {
      if (turned <= 0) raw[0].x = was.raw[0].x;
      if (turned <= 2) raw[0].y = was.raw[0].y;
      if (turned <= 4) raw[0].z = was.raw[0].z;
      if (turned <= 6) raw[0].w = was.raw[0].w;
    }
  }
};

__device__ __forceinline__ float element(const char* row, int e, float) { return reinterpret_cast<const float*>(row)[e]; }
__device__ __forceinline__ float element(const char* row, int e, __nv_bfloat16) {
  return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(row)[e]);
}

__device__ __forceinline__ int32_t new_length(const AppendArgs& p, int item, int rows) {
  return (int32_t)min(max((long long)p.start[item] + rows, 0LL), p.c.capacity);
}
// Tokens of a sequence.
__device__ __forceinline__ int tokens_of(const AppendArgs& p, int s, bool& bad) {
  if (p.counts == nullptr) return p.T;
  const int n = p.counts[s];
  bad = bad || n < 0 || n > p.T;
  return min(max(n, 0), p.T);
}

// Pair of the turned element e.
__device__ __forceinline__ int pair_of(const AppendArgs& p, int e) {
  return p.layout == CKV_ROPE_INTERLEAVED ? e / 2 : e < p.rot / 2 ? e : e - p.rot / 2;
}
__device__ __forceinline__ uint32_t top_of_eight(const float* x) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  return top;
}

template <typename T, int FMT, int MODE>
__global__ void __launch_bounds__(kThreads, 3) append_kernel(AppendArgs p) {
  wait_for_previous_kernel();
  constexpr int P = MODE == kAnyPair ? kOwn : kOwn / 2;        // angles a thread needs
  const int u = threadIdx.x % p.lanes, rest = threadIdx.x / p.lanes;
  const int tok = rest % p.tile, group = rest / p.tile;
  const int s = blockIdx.x / p.tiles, t = (blockIdx.x % p.tiles) * p.tile + tok;
  const int dh = p.lanes * kOwn, pairs = p.rot / 2;
  const unsigned mask = ((1u << p.lanes) - 1) << (threadIdx.x % 32 / p.lanes * p.lanes);   // the threads of this row
  bool bad = false;
  const int count = tokens_of(p, s, bad);
  // pieces of the row: eight elements from ea, eight from eb
  const bool turn = kOwn * u < p.rot, split = MODE == kHalf && turn;
  const int ea = split ? 8 * u : kOwn * u, eb = split ? pairs + 8 * u : kOwn * u + 8;
  float cs[P], sn[P];
  bool ready = false;
  const int step = p.groups * p.splits;
  for (int j = blockIdx.y * p.groups + group; j < p.jobs && group < p.groups && t < count; j += step) {
    const bool is_q = j < p.q_jobs;
    const int head = is_q ? 2 * j : j - p.q_jobs;
    const char* row[2];
    bool there[2] = {true, true};
    if (is_q) {
      there[1] = head + 1 < p.Hq;
      row[0] = p.x[0] + s * p.xs[0][0] + head * p.xs[0][1] + t * p.xs[0][2];
      row[1] = row[0] + p.xs[0][1];
    } else {
#pragma unroll
      for (int w = 0; w < 2; ++w) row[w] = p.x[1 + w] + s * p.xs[1 + w][0] + head * p.xs[1 + w][1] + t * p.xs[1 + w][2];
    }
    Eight<T> a[2], b[2];
#pragma unroll
    for (int w = 0; w < 2; ++w)
      if (there[w]) {
        a[w].load(row[w] + ea * (int)sizeof(T));
        b[w].load(row[w] + eb * (int)sizeof(T));
      }
    long long slot = -1;                                       // page * page_size + row in it
    if (!is_q) {
      const long long to = (long long)p.start[(long long)s * p.c.Hkv + head] + t;
      if (to >= 0 && to < p.c.capacity) {
        const int page = p.c.table[((long long)s * p.c.Hkv + head) * p.c.max_pages + (to >> p.c.page_shift)];
        if (page >= 0 && page < p.c.num_pages)
          slot = ((long long)page << p.c.page_shift) + (to & ((1 << p.c.page_shift) - 1));
      }
      bad = bad || slot < 0;
    }
    if (!ready && turn) {                                      // behind the first loads
      const double pos = (double)p.pos[(long long)s * p.T + t] * 0.15915494309189533577;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const int pair = MODE == kAnyPair ? min(pair_of(p, kOwn * u + i), pairs - 1) : 8 * u + i;
        const double turns = pos * p.freq[pair];
        sincospif(2.f * (float)(turns - rint(turns)), &sn[i], &cs[i]);
        cs[i] *= p.factor;
        sn[i] *= p.factor;
      }
    }
    ready = true;
    float x[2][kOwn];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      if (!there[w]) continue;
      a[w].get(x[w]);
      b[w].get(x[w] + 8);
      if (!turn || (!is_q && w == 1)) continue;
      if (MODE == kAnyPair) {
        const bool vectors = sizeof(T) == 2 && p.layout == CKV_ROPE_INTERLEAVED && p.rot % 8 == 0;
        float other[kOwn];
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
          const int e = kOwn * u + i;
          other[i] = e < p.rot ? element(row[w], p.layout == CKV_ROPE_INTERLEAVED ? e ^ 1 : e < pairs ? e + pairs : e - pairs, T()) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
          const int e = kOwn * u + i;
          const bool first = p.layout == CKV_ROPE_INTERLEAVED ? e % 2 == 0 : e < pairs;
          const float v = x[w][i];
          if (e < p.rot) x[w][i] = first ? turned_first(v, other[i], cs[i % P], sn[i % P]) : turned_second(other[i], v, cs[i % P], sn[i % P], vectors);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float& xa = MODE == kHalf ? x[w][i] : x[w][2 * i];
          float& xb = MODE == kHalf ? x[w][8 + i] : x[w][2 * i + 1];
          const float va = xa, vb = xb;
          xa = turned_first(va, vb, cs[i], sn[i]);
          xb = turned_second(va, vb, cs[i], sn[i], sizeof(T) == 2);
        }
      }
      const Eight<T> was[2] = {a[w], b[w]};
      a[w].put(x[w]);                                          // rounded to the model's type
      b[w].put(x[w] + 8);
      if (MODE == kAnyPair) {                                  // the last thread that turns has elements that are copied
        a[w].keep(was[0], p.rot - kOwn * u);
        b[w].keep(was[1], p.rot - kOwn * u - 8);
      }
    }
    if (MODE == kAnyPair) __syncwarp(mask);                    // the outputs may be the rows that others read pairs from
    if (is_q) {
      char* to = p.q_out + s * p.qos[0] + head * p.qos[1] + t * p.qos[2];
#pragma unroll
      for (int w = 0; w < 2; ++w)
        if (there[w]) {
          a[w].store(to + w * p.qos[1] + ea * (int)sizeof(T));
          b[w].store(to + w * p.qos[1] + eb * (int)sizeof(T));
        }
      continue;
    }
    const long long page_at = (slot >> p.c.page_shift) * p.c.page_stride;
    const int in_page = (int)(slot & ((1 << p.c.page_shift) - 1));
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      if constexpr (FMT == CKV_CACHE_PLAIN) {
        char* to = p.c.page[w] + page_at + in_page * dh * (int)sizeof(T);
        if (slot >= 0) {
          a[w].store(to + ea * (int)sizeof(T));
          b[w].store(to + eb * (int)sizeof(T));
        }
      } else {
        a[w].get(x[w]);
        b[w].get(x[w] + 8);
        uint32_t of[2] = {top_of_eight(x[w]), top_of_eight(x[w] + 8)};
        uint32_t top = max(of[0], of[1]);
        for (int o = p.lanes / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(mask, top, o));
        const float scale = row_scale<FMT>(top), r = __frcp_rn(scale);
        if constexpr (FMT == CKV_CACHE_E2M1) {
          // the group of 16 of each piece: both pieces of this thread, or one of it and one of a neighbour
          if (MODE == kHalf) {
            const int chunks = p.rot / 16;                     // pieces of first elements, and as many of second ones
            uint32_t with[2] = {of[1], of[0]};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int other = (h * chunks + u) ^ 1;          // both are even or odd ones of an even number
              const int from = split ? (other < chunks ? other : other - chunks) : u;
              const uint32_t m0 = __shfl_sync(mask, of[0], from, p.lanes), m1 = __shfl_sync(mask, of[1], from, p.lanes);
              if (split) with[h] = other < chunks ? m0 : m1;
            }
            of[0] = max(of[0], with[0]);
            of[1] = max(of[1], with[1]);
          } else {
            of[0] = of[1] = max(of[0], of[1]);
          }
          char* to = p.c.page[w] + page_at + in_page * (dh / 2);
          uint8_t* groups = p.c.group[w] + slot * (dh / 16);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int e = h ? eb : ea;
            float factor;
            const uint32_t g = group_scale(__uint_as_float(of[h]), r, top < 0x7f800000u, factor);
            const uint32_t code = encode8_e2m1(x[w] + 8 * h, factor);
            if (slot >= 0) {
              *reinterpret_cast<uint32_t*>(to + e / 2) = code;
              if (e % 16 == 0) groups[e / 16] = (uint8_t)g;
            }
          }
        } else {
          char* to = p.c.page[w] + page_at + in_page * dh;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint2 code = make_uint2(encode4<FMT>(x[w] + 8 * h, r), encode4<FMT>(x[w] + 8 * h + 4, r));
            if (slot >= 0) *reinterpret_cast<uint2*>(to + (h ? eb : ea)) = code;
          }
        }
        if (slot >= 0 && u == 0) p.c.scale[w][slot] = scale;
      }
    }
  }
  if (bad && p.status != nullptr) atomicExch(p.status, (int)CKV_EBOUNDS);
  if (p.lens_out != nullptr) {
    // lens_out may be start itself where a sequence has one tile: a head's start is then read by one CTA, above
    __syncthreads();
    if (blockIdx.x % p.tiles == 0)
      for (int g = threadIdx.x; g < p.c.Hkv; g += kThreads)
        if ((p.q_jobs + g) / p.groups % p.splits == (int)blockIdx.y)
          p.lens_out[(long long)s * p.c.Hkv + g] = new_length(p, s * p.c.Hkv + g, count);
  }
}

// lens_out = start + tokens where several CTAs read start and lens_out is start itself.
__global__ void append_lengths_kernel(AppendArgs p, int items) {
  wait_for_previous_kernel();
  const int item = blockIdx.x * blockDim.x + threadIdx.x;
  if (item >= items) return;
  bool bad = false;
  p.lens_out[item] = new_length(p, item, tokens_of(p, item / p.c.Hkv, bad));
}

template <typename T, int FMT>
cudaError_t launch_mode(const AppendArgs& p, dim3 grid, cudaStream_t st) {
  const auto kernel = p.rot % 16 ? append_kernel<T, FMT, kAnyPair>
                      : p.layout == CKV_ROPE_HALF ? append_kernel<T, FMT, kHalf> : append_kernel<T, FMT, kInterleaved>;
  return launch_early<AppendArgs>(kernel, grid, kThreads, 0, st, p);
}
template <typename T> cudaError_t launch_format(const AppendArgs& p, int format, dim3 grid, cudaStream_t st) {
  if (format == CKV_CACHE_PLAIN) return launch_mode<T, CKV_CACHE_PLAIN>(p, grid, st);
  if (format == CKV_CACHE_E4M3) return launch_mode<T, CKV_CACHE_E4M3>(p, grid, st);
  if (format == CKV_CACHE_E2M1) return launch_mode<T, CKV_CACHE_E2M1>(p, grid, st);
  return launch_mode<T, CKV_CACHE_INT8>(p, grid, st);
}

}  // namespace

cudaError_t launch_append(const CacheDims& d, const AppendCall& call, int sm_count, int* status_word, cudaStream_t st,
                          int* launches) {
  const int es = d.dtype == CKV_F32 ? 4 : 2;
  AppendArgs p;
  p.c = pages_of(d);
  const void* x[3] = {call.q, call.k, call.v};
  const long long* xs[3] = {call.qs, call.ks, call.vs};
  for (int w = 0; w < 3; ++w) {
    p.x[w] = (const char*)x[w];
    for (int i = 0; i < 3; ++i) p.xs[w][i] = xs[w][i] * es;
  }
  p.q_out = (char*)call.q_out;
  for (int i = 0; i < 3; ++i) p.qos[i] = call.qos[i] * es;
  p.pos = call.pos; p.freq = call.freq; p.factor = call.factor; p.counts = call.counts; p.start = call.start;
  p.T = call.T; p.Hq = d.Hq; p.rot = call.rot; p.layout = call.layout;
  p.status = d.debug_checks ? status_word : nullptr;
  p.lanes = d.dh / kOwn;
  p.tile = kThreads / p.lanes < p.T ? kThreads / p.lanes : p.T;
  if (p.tile < 1) p.tile = 1;                                  // no tokens: the lengths are written all the same
  p.tiles = p.T > 0 ? (p.T + p.tile - 1) / p.tile : 1;
  p.q_jobs = (d.Hq + 1) / 2;
  p.jobs = p.q_jobs + d.Hkv;
  p.groups = kThreads / (p.lanes * p.tile);
  if (p.groups > p.jobs) p.groups = p.jobs;
  const long long ctas = (long long)p.tiles * d.nseq;
  if (ctas > 0x7fffffffLL) return cudaErrorInvalidValue;
  const int turns = (p.jobs + p.groups - 1) / p.groups;
  // CTAs that share a tile's rows, of up to eight an SM in all: as many as end first, where they run three an SM in rounds and
  // each takes its turns and, for the angles, about one more (7000 tokens of 32 + 8 heads of 128: 438 CTAs of 12 turns 30.0 us,
  // 1314 of 4 31.1; 2500 tokens: 395 of 5 9.4 us, 1185 of 2 12.3; 25534 of heads of 64: 399 of 24 54.4 us, 1197 of 8 57.1)
  const long long most = (8LL * sm_count + ctas - 1) / ctas, slots = 3LL * sm_count;
  p.splits = 1;
  for (long long s = 1, least = 0; s <= most && s <= turns; ++s) {
    const long long time = (ctas * s + slots - 1) / slots * (1 + (turns + s - 1) / s);
    if (s > 1 && time >= least) continue;
    least = time;
    p.splits = (int)s;
  }
  const bool later = call.lens_out == call.start && call.lens_out != nullptr && p.tiles > 1;
  p.lens_out = later ? nullptr : call.lens_out;
  const dim3 grid((unsigned)ctas, (unsigned)p.splits);
  cudaError_t e = d.dtype == CKV_F32 ? launch_format<float>(p, d.format, grid, st) : launch_format<__nv_bfloat16>(p, d.format, grid, st);
  *launches += 1;
  if (e != cudaSuccess || !later) return e;
  p.lens_out = call.lens_out;
  const int items = d.nseq * d.Hkv;
  *launches += 1;
  return launch_early<AppendArgs, int>(append_lengths_kernel, dim3((unsigned)((items + 127) / 128)), 128, 0, st, p, items);
}

}  // namespace ckv
