// Decode attention for bf16 queries on tensor cores.
//
// A decode step multiplies every stored row with only the G = Hq/Hkv queries of its KV head: it is bound by the stream
// of K and V from HBM, and CUDA cores cannot keep up with that stream (at G = 4 and 8-bit pages the CUDA-core kernel
// reached a quarter of it).  The matrix instruction is mma.sync with the CACHE ROWS on its 16-row side and 8 queries on
// the other: a query tile of tcgen05.mma would be 64 or 128 rows of which G are used, its operands would have to lie in
// shared memory in the format of the instruction (8-bit pages converted and written back), and this kernel keeps the tensor
// pipe busy for 13 to 31 % of its time.
//
//   S^T = K Q^T   A = 16 rows of K.  Lane (r, c) = (lane / 4, lane % 4) reads 16 bytes of two rows; which of a row's
//                 elements those are is free, as long as the query fragments are loaded in the same order.
//   O^T = V^T P^T A = V^T: the lane needs two cache rows of one element in a register.  It reads 16 bytes of four rows
//                 and interleaves them with byte permutes; which elements form a 16-row tile is free again.  P^T is
//                 the accumulator of the first product with rows and columns exchanged (movmatrix).
//
// Every warp streams on its own: it works through 16 to 64 rows at a time (Shape::kSub), which one lane fetches with TMA
// (16 rows of a page are contiguous) into the warp's own slots, K of the next step as soon as K Q^T of this one is done, V
// likewise after V^T P^T, also across the end of an item: 8 KB a warp are on their way (16 with two query tiles on 128-byte
// rows), on 12 warps an SM with one query tile and 8 with two.  The 128-byte swizzle and the order of the rows (row_of)
// keep both reads free of bank conflicts.
// Softmax statistics are float32; the running maximum is only reduced over the warp (and the sums only rescaled) in
// steps in which some lane sees a larger logit.  The weights enter the second product as the sum of two 16-bit numbers:
// for bf16 pages two bf16 (16 bits); for 8-bit pages, whose codes are exact halves, two halves (22 bits) of weight * scale
// of the row * 2^15 / the largest such product so far.  What is below 2^-40 of that largest product is lost, so rows of very
// different norms and long tails of small weights keep theirs.  The queries of 8-bit pages become halves after a scaling
// by a power of two (at most 2^100) that puts the largest of a row at 2^14: exact but for elements 2^-29 below it or below
// 2^-114, which are rounded to multiples of 2^-38 of it or of 2^-124.  The factor of a logit, scale * log2(e), is one float
// and the exponential is ex2.approx (2^-22); the CUDA-core kernel keeps the rest of the factor as well.
//
// Measured: 2 x 131072 bf16 rows a head, 40 query heads on 8, 168 us, 6.4 TB/s (0.98 of the copy bandwidth); 32 x 6553
// e4m3 rows a head, 32 query heads on 8, 86 us, 5.2 TB/s (0.81; 82 us with weights of 11 bits, whose error is seen where
// values cancel), bound by instruction latency: 168 registers (60 bytes spilled) leave three CTAs an SM; four, with 128 and
// 400 bytes spilled, take 99 us.  1 x 819 bf16 rows: 8.0 us, a chain of latencies.
#include "paged_decode.cuh"
#include "sm100_ptx.cuh"
#include "tma_host.h"

namespace ckv {
namespace {

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 8 x 8 matrix of 16-bit elements, rows on lane / 4, two columns a register: rows and columns exchanged.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// Four 8-bit codes as two pairs of halves, exact.  int8: 0x64uu is the half 1024 + u, and u = code + 128 after a flip of
// the sign bit, so subtracting 1152 gives the code.
template <int FMT> __device__ __forceinline__ void codes_to_halves(uint32_t four, uint32_t& low, uint32_t& high) {
  if (FMT == CKV_CACHE_E4M3) {
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\t"
        "cvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
        : "=r"(low), "=r"(high)
        : "r"(four));
  } else {
    const uint32_t u = four ^ 0x80808080u, a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
    const __half2 bias = __half2half2(__ushort_as_half(0x6480));
    const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&a), bias), y = __hsub2(*reinterpret_cast<const __half2*>(&b), bias);
    low = *reinterpret_cast<const uint32_t*>(&x);
    high = *reinterpret_cast<const uint32_t*>(&y);
  }
}

// The largest product of a weight and a row's scale so far, as a half (8-bit pages): the top of the range, so that a long
// tail of small weights keeps its part of the sums.
constexpr float kTopWeight = 32768.f;
constexpr float kLeastTop = 3.851859888774472e-34f;   // 2^-111: kTopWeight over it and it over kTopWeight are normal floats

template <int FMT, int DH, int NT> struct Shape {
  static constexpr bool kPlain = FMT == CKV_CACHE_PLAIN;
  static constexpr int kRowBytes = kPlain ? DH * 2 : DH;
  // 16-row groups a warp takes at a time.  4 KB of K and of V; 8 KB for two query tiles on 128-byte rows, where the work
  // per step that does not depend on the rows weighs more (16 queries on e4m3 rows of 128: 144 -> 123 us; with one
  // query tile 86.0 and 85.3 us, int8 95 and 101 us).
  static constexpr int kSub = kRowBytes >= 256 ? 1 : kRowBytes == 128 ? 2 * NT : 4;
  static constexpr int kTile = kDecodeWarps * 16 * kSub;           // cache rows a CTA takes at a time
  static constexpr int kChunks = kRowBytes / 64;                   // 16-byte pieces of a K row per lane
  static constexpr int kQWords = kPlain ? 4 : 8;                   // registers of query elements per piece
  static constexpr int kVBytes = kRowBytes >= 128 ? 16 : 8;        // piece of a V row per lane
  static constexpr int kVPieces = kRowBytes / (8 * kVBytes);
  static constexpr int kElems = DH / 8;                            // V elements a lane has of a row
  static constexpr int kVWords = kVPieces * kVBytes / 4;           // registers they take
  static constexpr int kMTiles = kElems / 2;                       // 16-row tiles of V^T
  static constexpr int kGroupBytes = 16 * kRowBytes;               // a 16-row group of K or V in shared memory
  static constexpr int kSpan = kRowBytes >= 128 ? 128 : 64;        // bytes of a row that the swizzle keeps together
  // 16-byte chunk `chunk` of a row (half = which span of it) in a group as TMA writes it
  static __device__ __forceinline__ int at(int half, int row, int chunk) {
    return half * 16 * kSpan + row * kSpan + ((chunk ^ (kSpan == 128 ? row & 7 : (row >> 1) & 3)) * 16);
  }
};

// Cache row that row i of the matrix instruction stands for (i + 8: 8 further).  In the K read the eight lanes that
// are served together hold two neighbouring i and all c: their rows must differ in bit 2; in the V read they hold rows
// row_of(0, 2, 4, 6) or (1, 3, 5, 7): those must differ in bits 1-2.
__device__ __forceinline__ int row_of(int i) { return (0x37156240 >> (4 * i)) & 7; }   // 0 4 2 6 5 1 7 3

template <int FMT, int DH, int NT> struct alignas(1024) Slots {   // of a warp
  using S = Shape<FMT, DH, NT>;
  unsigned char k[S::kSub][S::kGroupBytes];
  unsigned char v[S::kSub][S::kGroupBytes];
};
template <int FMT, int DH, int NT> struct Scales {   // of a warp; quantised pages only
  float k[Shape<FMT, DH, NT>::kSub][16], v[Shape<FMT, DH, NT>::kSub][16];
};
template <int FMT, int DH, int NT> struct Shared {
  Slots<FMT, DH, NT> slots[kDecodeWarps];
  Scales<FMT, DH, NT> scales[kDecodeWarps];
  float o[kDecodeWarps][4][DH];                            // four queries at a time
  float m[kDecodeWarps][16], l[kDecodeWarps][16], top[16];
  alignas(8) float parts[8 * NT][DH + 2];                  // of a CTA of a team
  uint64_t full[kDecodeWarps][2];                          // K and V of a warp have arrived
  uint32_t late;                                           // a copy did not arrive in time: the other waits give up too
};

// The rows of one step of a warp: 16 * SUB of them, `here` of which exist.  They lie in one page, or in several where
// pages are shorter than a step: page[u] is the page of the 16-row groups u, u + 1, ..., -1: no rows.
template <int SUB> struct Step {
  int page[SUB];
  int in_page;
  int here;
};

// A CTA's part of an item: tiles [t0, t1) of it.
struct Segment {
  int item, kv, len, tiles, t0, t1;
  int first;                                               // the item's first tile in the list of all tiles
};

template <int FMT, int DH, int NT>
__global__ void __launch_bounds__(kDecodeThreads, NT == 1 ? 3 : 2)
    decode_mma_kernel(const __grid_constant__ DecodeArgs p, const __grid_constant__ CUtensorMap k_map,
                      const __grid_constant__ CUtensorMap v_map) {
  using S = Shape<FMT, DH, NT>;
  constexpr int SUB = S::kSub;
  using T = __nv_bfloat16;
  extern __shared__ unsigned char smem_raw[];
  Shared<FMT, DH, NT>& sh = *reinterpret_cast<Shared<FMT, DH, NT>*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32, r = lane >> 2, c = lane & 3;
  const uint32_t k_full = ptx::smem_addr(&sh.full[warp][0]), v_full = ptx::smem_addr(&sh.full[warp][1]);
  if (threadIdx.x < kDecodeWarps * 2) ptx::mbar_init(ptx::smem_addr(&sh.full[0][0] + threadIdx.x), 1);
  if (threadIdx.x == 0) {
    sh.late = 0;
    ptx::prefetch_tensormap(&k_map);
    ptx::prefetch_tensormap(&v_map);
  }
  ptx::fence_barrier_init();
  wait_for_previous_kernel();
  const Walk walk = p.team ? team_walk<T, DH, S::kTile>(p) : plan<T, DH, S::kTile>(p);
  if (threadIdx.x < 8 * NT) *reinterpret_cast<float2*>(&sh.parts[threadIdx.x][DH]) = make_float2(-INFINITY, 0.f);
  __syncthreads();                                         // the mbarriers are visible

  // The segment behind `g` (its item, first and tiles), or one with t0 == t1.
  auto following = [&](Segment g) {
    while (true) {
      g.first += g.tiles;
      g.item += 1;
      g.t0 = g.t1 = 0;
      if (g.first >= walk.end) return g;
      g.kv = kv_of(p, g.item);
      g.len = item_len(p, g.kv);
      g.tiles = (g.len + S::kTile - 1) / S::kTile;
      g.t0 = max(walk.begin - g.first, 0);
      g.t1 = min(g.tiles, walk.end - g.first);
      if (g.t1 > g.t0) return g;
    }
  };
  bool ok = true;                                          // no wait of this lane has run out
  // Looks up the pages of a step (without looking at what it finds: the loads stay in flight).
  const int page_mask = (1 << p.c.page_shift) - 1;
  const int together = SUB > 1 ? min(SUB, 1 << (p.c.page_shift - 4)) : 1;     // groups of a step in one page
  auto look_up = [&](const int32_t* pages, int len, int base, Step<SUB>& w) {
    w.here = min(len - base, 16 * SUB);
    w.in_page = base & page_mask;
#pragma unroll
    for (int u = 0; u < SUB; ++u) {
      w.page[u] = -1;
      if (u == 0 || (together < SUB && u % together == 0)) {
        if (w.here > 16 * u) w.page[u] = pages[(base + 16 * u) >> p.c.page_shift];
      }
    }
  };
  auto check = [&](Step<SUB>& w) {
#pragma unroll
    for (int u = 0; u < SUB; ++u)
      if ((u == 0 || (together < SUB && u % together == 0)) && (unsigned)w.page[u] >= (unsigned)p.c.num_pages) {
        if (w.here > 16 * u && p.status != nullptr && lane == 0) atomicExch(p.status, (int)CKV_EBOUNDS);
        w.page[u] = -1;
      }
  };
  // Rows of group u that exist, 0..16.
  auto rows = [&](const Step<SUB>& w, int u) {
    int page = w.page[0];
#pragma unroll
    for (int i = 1; i < SUB; ++i)
      if (i <= u && i % together == 0) page = w.page[i];
    return page < 0 ? 0 : max(0, min(w.here - 16 * u, 16));
  };
  // One phase of the barrier per step, also when there is nothing to fetch.  The scales come with K.
  auto fetch = [&](const Step<SUB>& w, bool is_k) {
    __syncwarp();                                          // every lane has read what the slot held
    if (lane == 0 && ok) {
      const uint32_t full = is_k ? k_full : v_full;
      const uint32_t slot = ptx::smem_addr(is_k ? sh.slots[warp].k[0] : sh.slots[warp].v[0]);
      const int count = 16 * together, bytes = count * (S::kRowBytes + (is_k && !S::kPlain ? 8 : 0));
      int n = w.page[0] >= 0;
      if (together < SUB) {
#pragma unroll
        for (int u = 1; u < SUB; ++u) n += u % together == 0 && w.page[u] >= 0;
      }
      ptx::mbar_arrive_expect_tx(full, n * bytes);
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        if ((u == 0 || (together < SUB && u % together == 0)) && w.page[u] >= 0) {
          const int in_page = u == 0 ? w.in_page : 0;
          ptx::tma_load_4d(slot + u * S::kGroupBytes, is_k ? &k_map : &v_map, 0, in_page, 0, w.page[u], full);
          if (is_k && !S::kPlain) {
            const long long at = ((long long)w.page[u] << p.c.page_shift) + in_page;
            ptx::bulk_load(ptx::smem_addr(sh.scales[warp].k[u]), p.c.scale[0] + at, count * 4, full);
            ptx::bulk_load(ptx::smem_addr(sh.scales[warp].v[u]), p.c.scale[1] + at, count * 4, full);
          }
        }
      }
    }
  };
  auto wait_for = [&](uint32_t full, uint32_t phase) {
    if (!ptx::mbar_wait_bounded(full, phase, &sh.late)) {
      ok = false;
      *(volatile uint32_t*)&sh.late = 1;
    }
  };
  const int k_row = row_of(r);
  // The queries of an item as they are stored, in the element order of the K pieces.
  uint32_t q[NT][S::kChunks][S::kQWords];
  auto load_queries = [&](const Segment& g) {
    const ItemRows it = item_rows(p, g.kv, g.item - g.kv * p.chunks);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int row = 8 * n + r;
      const char* src = p.q + it.s * p.qs[0] + (it.head + row) * p.qs[1] + c * 8 * S::kQWords / 2;
#pragma unroll
      for (int j = 0; j < S::kChunks; ++j)
#pragma unroll
        for (int h = 0; h < S::kQWords / 4; ++h) {
          uint4 v = make_uint4(0, 0, 0, 0);
          if (row < it.rows) v = *reinterpret_cast<const uint4*>(src + 16 * S::kQWords * j + 16 * h);
          q[n][j][4 * h] = v.x; q[n][j][4 * h + 1] = v.y; q[n][j][4 * h + 2] = v.z; q[n][j][4 * h + 3] = v.w;
        }
    }
  };

  int2 join = make_int2(-1, 0);
  Segment seg;
  seg.item = walk.item - 1;
  seg.kv = seg.len = 0;
  seg.first = walk.first;
  seg.tiles = 0;
  seg.t0 = seg.t1 = 0;
  if (walk.begin < walk.end) seg = following(seg);
  // Two steps ahead of the arithmetic: `ahead` has its pages being looked up, `next` is about to be fetched.
  Segment front = seg;
  int front_left = seg.t1 - seg.t0;                        // steps of `front` not looked up yet
  int front_base = (seg.t0 * kDecodeWarps + warp) * 16 * SUB;
  const int32_t* front_pages = p.c.table + (long long)seg.kv * p.c.max_pages;
  auto advance = [&](Step<SUB>& w) {
    if (front_left == 0) {
      if (front.t0 < front.t1) front = following(front);
      front_left = front.t1 - front.t0;
      front_base = (front.t0 * kDecodeWarps + warp) * 16 * SUB;
      front_pages = p.c.table + (long long)front.kv * p.c.max_pages;
    }
    look_up(front_pages, front_left > 0 ? front.len : 0, front_base, w);
    front_left -= front_left > 0;
    front_base += S::kTile;
  };
  Step<SUB> cur, next;
  uint32_t phase = 0;
  if (seg.t0 < seg.t1) {
    advance(cur);
    advance(next);
    load_queries(seg);
    check(cur);
    fetch(cur, true);
    fetch(cur, false);
  }
  while (seg.t0 < seg.t1 && ok) {
    const ItemRows it = item_rows(p, seg.kv, seg.item - seg.kv * p.chunks);
    float to_log2[NT][2];                      // factor of the products for query columns 2c, 2c+1
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      to_log2[n][0] = to_log2[n][1] = p.scale_log2;
      if (!S::kPlain) {
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < S::kChunks; ++j)
#pragma unroll
          for (int i = 0; i < S::kQWords; ++i) top = max(top, max(q[n][j][i] & 0x7fffu, (q[n][j][i] >> 16) & 0x7fffu));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // exponent of the largest element minus 14, so that both powers are normal floats (rows below 2^-86 in all
        // elements stay smaller than 2^14); 0 for rows of zeros, infinities or NaN
        int e = 0;
        if (top != 0 && top < 0x7f80u) e = max((int)(top >> 7) - 127 - 14, -100);
        const float down = __int_as_float((127 - e) << 23);
#pragma unroll
        for (int j = 0; j < S::kChunks; ++j)
#pragma unroll
          for (int i = 0; i < S::kQWords; ++i) {
            const uint32_t w = q[n][j][i];
            q[n][j][i] = pack_half(__uint_as_float(w << 16) * down, __uint_as_float(w & 0xffff0000u) * down);
          }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int ec = __shfl_sync(0xffffffffu, e, 8 * c + 4 * h);       // of query 8n + 2c + h
          to_log2[n][h] *= __int_as_float((127 + ec) << 23);
        }
      }
    }

    float o[NT][S::kMTiles][4];
    // running maximum, this lane's share of the sum, largest weight * scale so far and kTopWeight / that
    float m[NT][2], l[NT][2], big[NT][2], inv[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int i = 0; i < S::kMTiles; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][i][e] = 0.f;
#pragma unroll
      for (int h = 0; h < 2; ++h) { m[n][h] = -INFINITY; l[n][h] = 0.f; big[n][h] = 0.f; inv[n][h] = 0.f; }
    }

    const Segment after = following(seg);
    for (int tile = seg.t0; tile < seg.t1; ++tile) {
      Step<SUB> ahead;
      advance(ahead);
      check(next);
      wait_for(k_full, phase);

      // ---- logits
      float s[NT][SUB][4];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[n][u][e] = 0.f;
#pragma unroll
      for (int u = 0; u < SUB; ++u)
#pragma unroll
        for (int j = 0; j < S::kChunks; ++j) {
          const unsigned char* src = sh.slots[warp].k[u] + S::at(j / 2, k_row, c + 4 * (j % 2));
          const uint4 k0 = *reinterpret_cast<const uint4*>(src), k1 = *reinterpret_cast<const uint4*>(src + 8 * S::kSpan);
          const uint32_t a[4] = {k0.x, k0.y, k0.z, k0.w};
          const uint32_t b[4] = {k1.x, k1.y, k1.z, k1.w};
          if (S::kPlain) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int n = 0; n < NT; ++n)
                mma_bf16(s[n][u], a[2 * i], b[2 * i], a[2 * i + 1], b[2 * i + 1], q[n][j][2 * i], q[n][j][2 * i + 1]);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t a0, a1, a2, a3;
              codes_to_halves<FMT>(a[i], a0, a2);
              codes_to_halves<FMT>(b[i], a1, a3);
#pragma unroll
              for (int n = 0; n < NT; ++n)
                mma_f16(s[n][u], a0, a1, a2, a3, q[n][j][(2 * i) % S::kQWords], q[n][j][(2 * i + 1) % S::kQWords]);
            }
          }
        }
      float ks[SUB][2], vs[SUB][2];
      if constexpr (!S::kPlain) {
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            ks[u][h] = sh.scales[warp].k[u][k_row + 8 * h];
            vs[u][h] = sh.scales[warp].v[u][k_row + 8 * h];
          }
      }
      fetch(next, true);
      // rows that do not exist: no weight, and no value or scale that could be NaN
      bool whole_step = cur.here == 16 * SUB && cur.page[0] >= 0;
      if (together < SUB) {
#pragma unroll
        for (int u = 1; u < SUB; ++u) whole_step = whole_step && (u % together != 0 || cur.page[u] >= 0);
      }
      if (tile + 1 == seg.t1 && after.t0 < after.t1) load_queries(after);

      // ---- weights.  s[n][u][2h + x]: cache row k_row + 8h of group u, query 8n + 2c + x
      if (!whole_step) {
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (k_row + 8 * h >= rows(cur, u)) {
              if (!S::kPlain) ks[u][h] = vs[u][h] = 1.f;
#pragma unroll
              for (int n = 0; n < NT; ++n) s[n][u][2 * h] = s[n][u][2 * h + 1] = -INFINITY;
            }
      }
      uint32_t w_hi[NT][SUB][2], w_lo[NT][SUB][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float top[2] = {m[n][0], m[n][1]};
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              float& z = s[n][u][2 * h + x];
              // the two scales first: a product of codes and normalised queries, up to 2^31, times a large row scale alone
              // would overflow where tiny queries make up for it
              z *= S::kPlain ? to_log2[n][x] : ks[u][h] * to_log2[n][x];
              top[x] = fmaxf(top[x], z);
            }
        float f[2] = {1.f, 1.f};                                     // what the sums so far are multiplied by
        bool moved = false;
        if (__any_sync(0xffffffffu, top[0] > m[n][0] || top[1] > m[n][1])) {
          moved = true;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], 4));
            top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], 8));
            top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], 16));
            f[x] = m[n][x] == top[x] ? 1.f : ptx::ex2_approx(m[n][x] - top[x]);   // equal infinities included
            m[n][x] = top[x];
            l[n][x] *= f[x];
            big[n][x] *= f[x];
          }
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const float ref = m[n][x] == -INFINITY ? 0.f : m[n][x];    // nothing visible yet: all weights are 0
#pragma unroll
          for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float& z = s[n][u][2 * h + x];
              z = ptx::ex2_approx(z - ref);
              l[n][x] += z;
            }
        }
        if (S::kPlain) {
#pragma unroll
          for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float a = s[n][u][2 * h], b = s[n][u][2 * h + 1];
              const uint32_t hi = pack_bf16(a, b);
              w_hi[n][u][h] = transpose8(hi);
              w_lo[n][u][h] = transpose8(pack_bf16(a - __uint_as_float(hi << 16), b - __uint_as_float(hi & 0xffff0000u)));
            }
        } else {
          float most[2] = {big[n][0], big[n][1]};
#pragma unroll
          for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int x = 0; x < 2; ++x) {
                float& z = s[n][u][2 * h + x];
                z *= vs[u][h];
                most[x] = fmaxf(most[x], z);
              }
          if (moved || __any_sync(0xffffffffu, most[0] > big[n][0] || most[1] > big[n][1])) {
            moved = true;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              most[x] = fmaxf(most[x], __shfl_xor_sync(0xffffffffu, most[x], 4));
              most[x] = fmaxf(most[x], __shfl_xor_sync(0xffffffffu, most[x], 8));
              most[x] = fmaxf(most[x], __shfl_xor_sync(0xffffffffu, most[x], 16));
              most[x] = fmaxf(most[x], kLeastTop);
              const float one = __frcp_rn(most[x]);
              f[x] = big[n][x] * one;
              big[n][x] = most[x];
              inv[n][x] = one * kTopWeight;
            }
          }
#pragma unroll
          for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
            {
              const float a = s[n][u][2 * h] * inv[n][0], b = s[n][u][2 * h + 1] * inv[n][1];
              const __half2 hi = __floats2half2_rn(a, b);
              const float2 back = __half22float2(hi);
              w_hi[n][u][h] = transpose8(*reinterpret_cast<const uint32_t*>(&hi));
              w_lo[n][u][h] = transpose8(pack_half(a - back.x, b - back.y));
            }
        }
        if (moved) {
#pragma unroll
          for (int i = 0; i < S::kMTiles; ++i) {
            o[n][i][0] *= f[0]; o[n][i][1] *= f[1];
            o[n][i][2] *= f[0]; o[n][i][3] *= f[1];
          }
        }
      }
      wait_for(v_full, phase);

      // ---- O^T += V^T P^T
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        uint32_t v[4][S::kVWords];             // of cache rows row_of(2c), row_of(2c + 1) and 8 further
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          const int row = row_of(2 * c + (h & 1)) + 8 * (h >> 1);
#pragma unroll
          for (int j = 0; j < S::kVPieces; ++j) {
            if constexpr (S::kVBytes == 16) {
              const uint4 x = *reinterpret_cast<const uint4*>(sh.slots[warp].v[u] + S::at(j, row, r));
              v[h][4 * j] = x.x; v[h][4 * j + 1] = x.y; v[h][4 * j + 2] = x.z; v[h][4 * j + 3] = x.w;
            } else {
              const uint2 x = *reinterpret_cast<const uint2*>(sh.slots[warp].v[u] + S::at(0, row, r / 2) + 8 * (r % 2));
              v[h][2 * j] = x.x; v[h][2 * j + 1] = x.y;
            }
          }
          if (!whole_step && row >= rows(cur, u)) {
#pragma unroll
            for (int w = 0; w < S::kVWords; ++w) v[h][w] = 0;
          }
        }
        if (S::kPlain) {
#pragma unroll
          for (int i = 0; i < S::kMTiles; ++i) {
            const int e0 = i, e1 = i + S::kMTiles;
            const uint32_t p0 = e0 & 1 ? 0x7632 : 0x5410, p1 = e1 & 1 ? 0x7632 : 0x5410;
            const uint32_t a0 = __byte_perm(v[0][e0 / 2], v[1][e0 / 2], p0), a1 = __byte_perm(v[0][e1 / 2], v[1][e1 / 2], p1);
            const uint32_t a2 = __byte_perm(v[2][e0 / 2], v[3][e0 / 2], p0), a3 = __byte_perm(v[2][e1 / 2], v[3][e1 / 2], p1);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              mma_bf16(o[n][i], a0, a1, a2, a3, w_hi[n][u][0], w_hi[n][u][1]);
              mma_bf16(o[n][i], a0, a1, a2, a3, w_lo[n][u][0], w_lo[n][u][1]);
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < S::kMTiles; i += 2) {       // two tiles: elements i, i+1 and kMTiles further
            uint32_t a[2][4];
#pragma unroll
            for (int g = 0; g < 2; ++g) {                 // g: rows 0, 1 or 2, 3 of v
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const int at = i + e * S::kMTiles;
                codes_to_halves<FMT>(__byte_perm(v[2 * g][at / 4], v[2 * g + 1][at / 4], at & 2 ? 0x7362 : 0x5140),
                                     a[0][2 * g + e], a[1][2 * g + e]);
              }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
              for (int e = 0; e < 2; ++e)
                mma_f16(o[n][i + e], a[e][0], a[e][1], a[e][2], a[e][3], w_hi[n][u][0], w_hi[n][u][1]);
#pragma unroll
              for (int e = 0; e < 2; ++e)
                mma_f16(o[n][i + e], a[e][0], a[e][1], a[e][2], a[e][3], w_lo[n][u][0], w_lo[n][u][1]);
            }
          }
        }
      }
      fetch(next, false);
      phase ^= 1;
      cur = next;
      next = ahead;
    }
    // ---- the warps meet in shared memory: maxima first, then the sums rescaled to the joint maximum, four queries at a
    // time
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int x = 0; x < 2; ++x)
        if (r == 0) sh.m[warp][8 * n + 2 * c + x] = m[n][x];
    ok = !__syncthreads_or(!ok);               // also: everything of the previous item has been read
    if (!ok) break;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int row = 8 * n + 2 * c + x;
        float top = sh.m[0][row];
#pragma unroll
        for (int w = 1; w < kDecodeWarps; ++w) top = fmaxf(top, sh.m[w][row]);
        const float f = m[n][x] == -INFINITY ? 0.f : ptx::ex2_approx(m[n][x] - top);
        float sum = l[n][x];
        sum += __shfl_xor_sync(0xffffffffu, sum, 4);
        sum += __shfl_xor_sync(0xffffffffu, sum, 8);
        sum += __shfl_xor_sync(0xffffffffu, sum, 16);
        if (r == 0) {
          sh.l[warp][row] = sum * f;
          if (warp == 0) sh.top[row] = top;
        }
        big[n][x] = S::kPlain ? f : f * (big[n][x] * (1.f / kTopWeight));   // factor of the sums
      }
    const bool whole = seg.t0 == 0 && seg.t1 == seg.tiles;
#pragma unroll
    for (int g = 0; g < 2 * NT; ++g) {
      if (4 * g < it.rows) {
        if (g > 0) __syncthreads();
        if (c / 2 == g % 2) {
          const int n = g / 2;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            float* dst = sh.o[warp][2 * (c % 2) + x];
            const float f = big[n][x];
            // element e of the lane's piece: o[n][e % kMTiles][2 * (e / kMTiles) + x]
#pragma unroll
            for (int e = 0; e < S::kElems; e += 4) {
              const int half = e / S::kMTiles, i = e % S::kMTiles;
              const int at = (S::kVPieces == 2) ? 8 * r + 64 * half + i : S::kElems * r + e;
              *reinterpret_cast<float4*>(dst + at) = make_float4(o[n][i][2 * half + x] * f, o[n][i + 1][2 * half + x] * f,
                                                                 o[n][i + 2][2 * half + x] * f, o[n][i + 3][2 * half + x] * f);
            }
          }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 4 * (DH / 2); i += kDecodeThreads) {
          const int row = 4 * g + i / (DH / 2), pair = i % (DH / 2);
          if (row >= it.rows) break;
          float2 sum = make_float2(0.f, 0.f);
          float total = 0.f;
#pragma unroll
          for (int w = 0; w < kDecodeWarps; ++w) {
            const float2 v = *reinterpret_cast<const float2*>(&sh.o[w][i / (DH / 2)][2 * pair]);
            sum.x += v.x;
            sum.y += v.y;
            total += sh.l[w][row];
          }
          if (whole) {
            put_out<T, DH>(p, it, row, pair, sum.x, sum.y, sh.top[row], total, false);
          } else {
            float* part = p.team ? sh.parts[row] : part_slot(p, DH, blockIdx.x, seg.t0 > 0 ? 0 : 1) + row * (DH + 2);
            *reinterpret_cast<float2*>(part + 2 * pair) = sum;
            if (pair == 0) *reinterpret_cast<float2*>(part + DH) = make_float2(sh.top[row], total);
          }
        }
      }
    }
    if (seg.t0 > 0 && seg.t1 == seg.tiles) join = make_int2(seg.item, cta_of(walk, seg.first));
    seg = after;
  }
  if (!ok) {
    // a copy did not arrive in time: report it, and give what is still on its way a last chance before the CTA (and
    // with it the shared memory the copies write) goes away
    if (threadIdx.x == 0) atomicExch(p.timeout, (int)CKV_ETIMEOUT);
    volatile uint32_t zero = 0;
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_wait_bounded(k_full, phase ^ i, &zero, 200000000ull);
      ptx::mbar_wait_bounded(v_full, phase ^ i, &zero, 200000000ull);
    }
  }
  if (p.team) join_team<T, DH>(p, walk, &sh.parts[0][0]);
  else if (threadIdx.x == 0) p.join[blockIdx.x] = join;
}

// Pages as TMA sees them: bytes in spans of 128 (or 64) x spans of a row x rows of a page x pages.
template <typename S> bool page_map(CUtensorMap* m, const DecodeArgs& p, int which, int box_rows) {
  EncodeTiledFn fn = tma_encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[4] = {(cuuint64_t)S::kSpan, (cuuint64_t)1 << p.c.page_shift, (cuuint64_t)(S::kRowBytes / S::kSpan),
                              (cuuint64_t)p.c.num_pages};
  const cuuint64_t strides[3] = {(cuuint64_t)S::kRowBytes, (cuuint64_t)S::kSpan, (cuuint64_t)p.c.page_stride};
  const cuuint32_t box[4] = {(cuuint32_t)S::kSpan, (cuuint32_t)box_rows, (cuuint32_t)(S::kRowBytes / S::kSpan), 1}, ones[4] = {1, 1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, p.c.page[which], dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
            S::kSpan == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int FMT, int DH, int NT>
cudaError_t launch(DecodeArgs p, int device, int sm_count, cudaStream_t st, int* launches) {
  const auto kernel = decode_mma_kernel<FMT, DH, NT>;
  constexpr int smem = (int)sizeof(Shared<FMT, DH, NT>) + 1024;   // the slots start on a multiple of 1024
  static LaunchSetup setup;
  const LaunchSetup::Fit* fit = setup.of(kernel, device, smem);
  if (!fit) return cudaErrorInvalidDeviceFunction;
  CUtensorMap maps[2];
  for (int i = 0; i < 2; ++i)
    if (!page_map<Shape<FMT, DH, NT>>(&maps[i], p, i, min(1 << p.c.page_shift, 16 * Shape<FMT, DH, NT>::kSub))) return cudaErrorInvalidValue;
  p.team = decode_team(p, *fit, sm_count, Shape<FMT, DH, NT>::kTile);
  const int grid = p.team ? p.items * p.team : decode_grid(p, fit->per_sm * sm_count, Shape<FMT, DH, NT>::kTile);
  *launches += 1;
  const cudaError_t e = launch_early_in_clusters<DecodeArgs, CUtensorMap, CUtensorMap>(kernel, dim3(grid), kDecodeThreads, smem,
                                                                                       p.team, st, p, maps[0], maps[1]);
  if (e != cudaSuccess || p.team) return e;
  *launches += 1;
  return launch_decode_join<__nv_bfloat16, DH>(p, grid, st);
}

template <int FMT> cudaError_t by_shape(const DecodeArgs& p, int dh, int device, int sm_count, cudaStream_t st, int* launches) {
  if (p.chunk_rows == 8) return dh == 64 ? launch<FMT, 64, 1>(p, device, sm_count, st, launches) : launch<FMT, 128, 1>(p, device, sm_count, st, launches);
  return dh == 64 ? launch<FMT, 64, 2>(p, device, sm_count, st, launches) : launch<FMT, 128, 2>(p, device, sm_count, st, launches);
}

}  // namespace

cudaError_t launch_decode_mma(const CacheDims& d, const DecodeCall& call, int device, int sm_count, int* status_word, cudaStream_t st,
                              int* launches) {
  // queries of a KV head: 8 or 16 an item; more than 16 read the cache once per 16
  const DecodeArgs p = decode_args(d, call, d.Hq / d.Hkv <= 8 ? 8 : 16, status_word);
  if (d.format == CKV_CACHE_PLAIN) return by_shape<CKV_CACHE_PLAIN>(p, d.dh, device, sm_count, st, launches);
  if (d.format == CKV_CACHE_E4M3) return by_shape<CKV_CACHE_E4M3>(p, d.dh, device, sm_count, st, launches);
  return by_shape<CKV_CACHE_INT8>(p, d.dh, device, sm_count, st, launches);
}

}  // namespace ckv
