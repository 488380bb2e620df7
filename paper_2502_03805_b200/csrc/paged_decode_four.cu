// Decode attention over pages in 4 bits a value, on tensor cores.
//
// The products are those of paged_decode_mma.cu: the cache rows on the 16-row side of mma.sync, 8 queries on the other,
// S^T = K Q^T, then O^T = V^T P^T.  A row of 128 elements is 76 bytes, for which the instructions that turn codes into halves are
// many, so everything else is kept short.
//
//   codes      cvt takes two codes of a byte to two halves; code times group scale is exact in a half (2 and 4 significant
//              bits), one instruction for two elements.  K: a byte is two elements of a row.  V: the matrix instruction wants two
//              rows of an element in a register, so the half bytes of two rows are mixed first, two instructions for four
//              registers.
//   queries    halves after a scaling by a power of two that puts the largest element at 2^14, as for 8-bit pages; a float32
//              query is the sum of two halves (an error of 2^-23 of an element, or 2^-39 of the largest), two products each.
//   softmax    a warp's logits are taken relative to a maximum that is moved only when one is 2^10 times above it, and its
//              weights (times the row scales) relative to a largest one that is moved only when one is 16 times above it: sums
//              are rescaled a few times a head instead of in most steps.  A weight enters the second product as two halves
//              (22 bits, no finer than 2^-36 of the largest such product).  Float pairs go through the packed instructions.
//   queries    up to four of a KV head leave half of the matrix instruction's columns free: they hold the second halves of the
//              weights, and the lanes of those columns work on the other of two tiles.
//   copies     a warp has a ring of steps of 32 rows, filled by asynchronous copies of 16 bytes a lane: a step is ten of them.
//              (Bulk copies take their operands from uniform registers, which made each of six to nine a step some fifteen
//              instructions.)
//
// Measured: 32 x 6553 rows a head, 32 query heads on 8 of 128, 66 to 67 us (73 on another B200), 3.9 TB/s (0.60 of the copy
// bandwidth; as 4-bit pages in paged_decode_mma.cu 88.8, with bulk copies and masks as selections 76 to 82).  348 instructions for
// 16 rows (codes and products 165, copies 48), which at four a cycle and SM would be 31 us.  No unit is full: 2.0 a cycle, 2.4 in the
// loop, ALU 42 %, tensor pipe 19 %, DRAM 40 %.  What holds it are the 12 warps an SM that 163 registers leave, whose most frequent
// stall is the fixed latency of the instruction before, and CTAs that end 49 to 66 us after the start with equal shares; 16 warps,
// with up to 270 bytes spilled, take 69 us, a ring of three steps 68.  float32 queries 75.5 us, with 8 query heads a KV head 90.5 (in
// one chain of cut-off sums 85.8).  1 x 819 rows: 8.4 us, a chain of latencies.
#include <stddef.h>

#include "paged_decode.cuh"
#include "sm100_ptx.cuh"

namespace ckv {
namespace {

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
__device__ __forceinline__ uint32_t bits(__half2 x) { return *reinterpret_cast<const uint32_t*>(&x); }
__device__ __forceinline__ __half2 halves(uint32_t x) { return *reinterpret_cast<const __half2*>(&x); }

// Two float32 operations in one instruction.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("mul.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<unsigned long long&>(d))
      : "l"(reinterpret_cast<const unsigned long long&>(a)), "l"(reinterpret_cast<const unsigned long long&>(b)));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("add.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<unsigned long long&>(d))
      : "l"(reinterpret_cast<const unsigned long long&>(a)), "l"(reinterpret_cast<const unsigned long long&>(b)));
  return d;
}
__device__ __forceinline__ void add4(float (&a)[4], const float (&b)[4]) {
#pragma unroll
  for (int i = 0; i < 4; i += 2) {
    const float2 x = add2(make_float2(a[i], a[i + 1]), make_float2(b[i], b[i + 1]));
    a[i] = x.x;
    a[i + 1] = x.y;
  }
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

constexpr float kTop = 2048.f;         // where the largest product of a weight and a row scale is put ...
constexpr float kMost = 32768.f;       // ... and what a later one may reach before it is moved
constexpr float kAhead = 10.f;         // log2 of what a weight may reach before the maximum is moved
constexpr float kLeastTop = 3.851859888774472e-34f;   // 2^-111: kTop over it and it over kTop are normal floats
// In place of minus the reference where no logit has been seen: any logit is far above it, and -infinity has weight 0.
constexpr float kNoReference = 3.4028234e38f;

constexpr int kWarpRows = 32, kTiles = kWarpRows / 16;          // rows of a step of a warp, in tiles of the matrix instruction
constexpr int kRows = kDecodeWarps * kWarpRows;                 // rows of a step of all warps

template <int DH> struct Row {
  static constexpr int kBytes = DH / 2, kGroups = DH / 16, kWords = DH / 32;   // of codes; scales; words of codes a quad lane has
  // V lies in chunks of eight rows that are 32 bytes apart, so that the rows of the four lanes c below are on different banks.
  static constexpr int kChunk = 8 * kBytes + 32;
};

// Row i of tile u of a warp is row 8 * (i / 2 % 4) + 4u + 2 * (i / 8) + i % 2: of the lanes (r, c), c has rows 2c, 2c + 1, 2c + 8 and
// 2c + 9 of V^T P^T in one chunk, and neighbouring rows of K Q^T are neighbours in memory.
__device__ __forceinline__ int row_of(int u, int i) { return 8 * (i >> 1 & 3) + 4 * u + 2 * (i >> 3) + (i & 1); }

template <int DH> struct alignas(16) Step {        // the rows of a step of a warp in shared memory
  unsigned char k[kWarpRows * Row<DH>::kBytes], v[4 * Row<DH>::kChunk];
  uint8_t kg[kWarpRows][Row<DH>::kGroups], vg[kWarpRows][Row<DH>::kGroups];
  float ks[kWarpRows], vs[kWarpRows];
};

__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}

template <int DH, int NT, int RING> struct Shared {
  Step<DH> ring[kDecodeWarps][RING];
  float o[kDecodeWarps][4][DH];                    // four queries at a time
  float m[kDecodeWarps][8 * NT], l[kDecodeWarps][8 * NT], top[8 * NT];
  alignas(8) float parts[8 * NT][DH + 2];          // of a CTA of a team
};

// A CTA's part of an item: tiles [t0, t1) of it, a tile being a step of every warp.
struct Segment {
  int item, kv, len, tiles, t0, t1;
  int first;                                       // the item's first tile in the list of all tiles
};

// QUAD: no KV head has more than four queries (NT is 1).
template <typename T, int DH, int NT, bool QUAD, int RING, int CTAS>
__global__ void __launch_bounds__(kDecodeThreads, CTAS) decode_four_kernel(const __grid_constant__ DecodeArgs p) {
  using R = Row<DH>;
  constexpr int kParts = sizeof(T) == 4 ? 2 : 1;   // halves a query element is the sum of
  constexpr int kQ = DH / 8;                       // registers of a query's elements
  constexpr int kM = DH / 16;                      // 16-row tiles of V^T
  constexpr int kUnits = QUAD ? 1 : kTiles;        // tiles whose weights a lane works on
  extern __shared__ __align__(16) unsigned char smem_raw[];
  Shared<DH, NT, RING>& sh = *reinterpret_cast<Shared<DH, NT, RING>*>(smem_raw);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32, r = lane >> 2, c = lane & 3;
  const int cc = QUAD ? c & 1 : c;                 // the lane's pair of query columns
  wait_for_previous_kernel();
  const Walk walk = p.team ? team_walk<T, DH, kRows>(p) : plan<T, DH, kRows>(p);
  if (threadIdx.x < 8 * NT) *reinterpret_cast<float2*>(&sh.parts[threadIdx.x][DH]) = make_float2(-INFINITY, 0.f);

  // The segment behind `g` (its item, first and tiles), or one with t0 == t1.
  auto following = [&](Segment g) {
    while (true) {
      g.first += g.tiles;
      g.item += 1;
      g.t0 = g.t1 = 0;
      if (g.first >= walk.end) return g;
      g.kv = kv_of(p, g.item);
      g.len = item_len(p, g.kv);
      g.tiles = (g.len + kRows - 1) / kRows;
      g.t0 = max(walk.begin - g.first, 0);
      g.t1 = min(g.tiles, walk.end - g.first);
      if (g.t1 > g.t0) return g;
    }
  };
  // ---- copies.  A step is two halves of 16 rows, each of one page.
  Segment front;                                   // the step that is looked up next: front_left of this segment are left
  int front_left, front_row;
  struct Next {                                    // a step to be fetched: its pages, rows, first row in its page
    int page[2], here, in_page;
  };
  uint32_t present = 0;                            // four bits a step of the ring: whether rows 8i ... 8i + 7 are there
  const uint32_t ring = ptx::smem_addr(&sh.ring[warp][0]);
  auto enter = [&]() {
    front_left = front.t1 - front.t0;
    front_row = (front.t0 * kDecodeWarps + warp) * kWarpRows;
  };
  auto look_up = [&](Next& n) {
    if (front_left == 0) {
      if (front.t0 < front.t1) front = following(front);
      enter();
    }
    n.here = front_left > 0 ? front.len - front_row : 0;
    n.in_page = front_row & ((1 << p.c.page_shift) - 1);
    const int32_t* pages = p.c.table + (long long)front.kv * p.c.max_pages + (front_row >> p.c.page_shift);
    n.page[0] = n.here > 0 ? pages[0] : 0;
    n.page[1] = n.page[0];
    if (p.c.page_shift == 4 && n.here > 16) n.page[1] = pages[1];
    front_left -= front_left > 0;
    front_row += kRows;
  };
  // scales are copied by lanes 0 to 15 (those of K) and 16 to 31 (of V)
  const int w = lane >> 4, l = lane & 15;
  auto fetch = [&](int stage, const Next& n) {
    using S = Step<DH>;
    constexpr int kCopy = 512 / R::kBytes;         // rows that the lanes copy at once: 8 or 16
    const uint32_t to = ring + stage * (uint32_t)sizeof(S), to_codes = to + lane * 16;
    const uint32_t to_v = DH == 128 ? to_codes : to + lane / 16 * R::kChunk + lane % 16 * 16;
    const uint32_t to_groups = to + l * 16 + (w ? offsetof(S, vg) : offsetof(S, kg));
    const uint32_t to_scales = to + (l & 7) * 16 + (w ? offsetof(S, vs) : offsetof(S, ks));
    const bool groups = DH == 128 || l < 8, scales = DH == 128 ? l < 8 : l >= 8;
    present &= ~(15u << (4 * stage));
    __syncwarp();                                  // every lane has read what the step held
    if (n.here >= kWarpRows && p.c.page_shift > 4 && (unsigned)n.page[0] < (unsigned)p.c.num_pages) {
      present |= 15u << (4 * stage);
      const long long at = n.page[0] * p.c.page_stride + n.in_page * R::kBytes + lane * 16;
      const long long slot = ((long long)n.page[0] << p.c.page_shift) + n.in_page;
      const char *k = p.c.page[0] + at, *v = p.c.page[1] + at;
#pragma unroll
      for (int i = 0; i < kWarpRows / kCopy; ++i) {
        copy16(to_codes + offsetof(S, k) + 512 * i, k + 512 * i);
        copy16(to_v + offsetof(S, v) + kCopy / 8 * R::kChunk * i, v + 512 * i);
      }
      if (groups) copy16(to_groups, p.c.group[w] + slot * R::kGroups + l * 16);
      if (scales) copy16(to_scales, p.c.scale[w] + slot + (l & 7) * 4);
    } else {                                       // the same by halves of 16 rows, which are of a page each and may be absent
#pragma unroll 1
      for (int h = 0; h < 2; ++h) {
        if (n.here <= 16 * h) break;
        const int of = h ? n.page[1] : n.page[0];
        if ((unsigned)of >= (unsigned)p.c.num_pages) {
          if (p.status != nullptr && lane == 0) atomicExch(p.status, (int)CKV_EBOUNDS);
          continue;
        }
        present |= (n.here > 16 * h + 8 ? 3u : 1u) << (4 * stage + 2 * h);
        const int first = n.in_page + (p.c.page_shift == 4 ? 0 : 16 * h);
        const long long at = of * p.c.page_stride + first * R::kBytes + lane * 16;
        const long long slot = ((long long)of << p.c.page_shift) + first - 16 * h;
#pragma unroll
        for (int i = 0; i < 16 / kCopy; ++i) {
          copy16(to_codes + offsetof(S, k) + 16 * h * R::kBytes + 512 * i, p.c.page[0] + at + 512 * i);
          copy16(to_v + offsetof(S, v) + 2 * h * R::kChunk + kCopy / 8 * R::kChunk * i, p.c.page[1] + at + 512 * i);
        }
        // the lanes of this half's rows
        if (groups && (DH == 128 ? l >> 3 : l >> 2) == h) copy16(to_groups, p.c.group[w] + slot * R::kGroups + l * 16);
        if (scales && (l >> 2 & 1) == h) copy16(to_scales, p.c.scale[w] + slot + (l & 7) * 4);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };

  // The queries of an item, in the element order of the K pieces: lane c of a quad has elements DH/4 * c ...
  uint32_t q[NT][kParts][kQ];
  float2 to_log2[NT];                              // factor of the products for query columns 2cc, 2cc + 1
  auto load_queries = [&](const Segment& g) {
    const ItemRows it = item_rows(p, g.kv, g.item - g.kv * p.chunks);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int row = 8 * n + r;
      const char* src = p.q + it.s * p.qs[0] + (it.head + row) * p.qs[1] + c * (DH / 4) * (int)sizeof(T);
      float x[2 * kQ];
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 2 * kQ; i += 16 / (int)sizeof(T)) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (row < it.rows) v = *reinterpret_cast<const uint4*>(src + i * (int)sizeof(T));
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (sizeof(T) == 4) {
            x[i + j] = __uint_as_float(w[j]);
          } else {
            x[i + 2 * j] = __uint_as_float(w[j] << 16);
            x[i + 2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 2 * kQ; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      // exponent of the largest element minus 14, so that both powers are normal floats (rows below 2^-86 in all elements
      // stay smaller than 2^14); 0 for rows of zeros, infinities or NaN
      int e = 0;
      if (top != 0 && top < 0x7f800000u) e = max((int)(top >> 23) - 127 - 14, -100);
      const float down = __int_as_float((127 - e) << 23);
#pragma unroll
      for (int i = 0; i < kQ; ++i) {
        const float a = x[2 * i] * down, b = x[2 * i + 1] * down;
        const __half2 hi = __floats2half2_rn(a, b);
        q[n][0][i] = bits(hi);
        if (kParts == 2) {
          const float2 back = __half22float2(hi);
          q[n][kParts - 1][i] = bits(__floats2half2_rn(a - back.x, b - back.y));
        }
      }
      float up[2];                                 // (the scale as one float: 2^-24 of a logit, as its other roundings)
#pragma unroll
      for (int y = 0; y < 2; ++y)
        up[y] = p.scale_log2 * __int_as_float((127 + __shfl_sync(0xffffffffu, e, 8 * cc + 4 * y)) << 23);   // of query 8n + 2cc + y
      to_log2[n] = make_float2(up[0], up[1]);
    }
  };
  // Largest over the lanes that have the same query columns.
  auto top_of_columns = [&](float x) {
    if (QUAD) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
    return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
  };

  int2 join = make_int2(-1, 0);
  Segment seg;
  seg.item = walk.item - 1;
  seg.kv = seg.len = 0;
  seg.first = walk.first;
  seg.tiles = 0;
  seg.t0 = seg.t1 = 0;
  if (walk.begin < walk.end) seg = following(seg);
  front = seg;
  enter();
  int stage = 0;
  Next next = {};
  if (seg.t0 < seg.t1) {
    Next first[RING];                              // the pages of all of them before the first is needed
#pragma unroll
    for (int i = 0; i < RING; ++i) look_up(first[i]);
    look_up(next);
#pragma unroll
    for (int i = 0; i < RING; ++i) fetch(i, first[i]);
  }
  while (seg.t0 < seg.t1) {
    const ItemRows it = item_rows(p, seg.kv, seg.item - seg.kv * p.chunks);
    load_queries(seg);
    float o[NT][kM][4];                            // [tile of V^T][even, odd element; columns 2c, 2c + 1]
    float2 m[NT], l[NT], big[NT], inv[NT];         // reference of the logits, sums, largest product, kTop over it
    float2 less[NT];                               // minus the reference
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int i = 0; i < kM; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][i][e] = 0.f;
      m[n] = both(-INFINITY);
      l[n] = big[n] = inv[n] = both(0.f);
      less[n] = both(kNoReference);
    }

    for (int tile = seg.t0; tile < seg.t1; ++tile) {
      const Step<DH>& step = sh.ring[warp][stage];
      asm volatile("cp.async.wait_group %0;" ::"n"(RING - 1) : "memory");
      __syncwarp();
      const int rows = seg.len - (tile * kDecodeWarps + warp) * kWarpRows;      // that exist, where their pages do
      const uint32_t chunks = present >> (4 * stage) & 15u;
      const bool whole_step = rows >= kWarpRows && chunks == 15u;
      const auto absent = [&](int row) { return row >= rows || !(chunks >> (row >> 3) & 1u); };
      if (!whole_step && chunks) {
        // what is left in the places of absent rows may be no number
        if (absent(lane)) {
          Step<DH>& own = sh.ring[warp][stage];
#pragma unroll 1
          for (int i = 0; i < R::kBytes / 16; ++i) {
            *reinterpret_cast<uint4*>(own.k + lane * R::kBytes + 16 * i) = make_uint4(0, 0, 0, 0);
            *reinterpret_cast<uint4*>(own.v + (lane >> 3) * R::kChunk + (lane & 7) * R::kBytes + 16 * i) = make_uint4(0, 0, 0, 0);
          }
#pragma unroll 1
          for (int i = 0; i < R::kGroups; ++i) own.kg[lane][i] = own.vg[lane][i] = 0;
          own.ks[lane] = own.vs[lane] = 0.f;
        }
        __syncwarp();
      }
      if (chunks) {
        // ---- logits
        float s[NT][kTiles][4];
#pragma unroll
        for (int u = 0; u < kTiles; ++u) {
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][u][e] = 0.f;
          // The matrix instructions cut their sums off instead of rounding them.  For float32 queries two of them at a time
          // begin anew, and the products of the second halves have a sum of their own: outputs of 1 to 5 queries a head over
          // 1101 to 11297 rows were 5e-7 to 3e-6 off in one chain, 3e-7 to 6e-7 so (32 x 6553 rows 74.2 -> 75 us)
          float small[4] = {0.f, 0.f, 0.f, 0.f};
          uint32_t x[2][R::kWords];
          __half2 g[2][DH / 64];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int row = row_of(u, r) + 2 * h;
            const uint8_t* group = step.kg[row] + c * (DH / 64);
            if constexpr (DH == 128) {
              const uint4 v = *reinterpret_cast<const uint4*>(step.k + row * R::kBytes + 16 * c);
              x[h][0] = v.x; x[h][1] = v.y; x[h][R::kWords - 2] = v.z; x[h][R::kWords - 1] = v.w;
              const __half2 pair = halves(e4m3x2_to_half2(*reinterpret_cast<const uint16_t*>(group)));
              g[h][0] = __low2half2(pair);
              g[h][DH / 64 - 1] = __high2half2(pair);
            } else {
              const uint2 v = *reinterpret_cast<const uint2*>(step.k + row * R::kBytes + 8 * c);
              x[h][0] = v.x; x[h][1] = v.y;
              g[h][0] = halves(e4m3x2_to_half2(*group * 0x101u));
            }
          }
#pragma unroll
          for (int w = 0; w < R::kWords; ++w) {
            uint32_t a[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              e2m1x8_to_half2(x[h][w], a[h]);
#pragma unroll
              for (int i = 0; i < 4; ++i) a[h][i] = bits(__hmul2(halves(a[h][i]), g[h][w / 2]));
            }
            if constexpr (kParts == 2) {
              float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int i = 0; i < 4; i += 2) {
                mma_f16(d, a[0][i], a[1][i], a[0][i + 1], a[1][i + 1], q[0][0][4 * w + i], q[0][0][4 * w + i + 1]);
                mma_f16(small, a[0][i], a[1][i], a[0][i + 1], a[1][i + 1], q[0][kParts - 1][4 * w + i], q[0][kParts - 1][4 * w + i + 1]);
              }
              add4(s[0][u], d);
            } else {
#pragma unroll
              for (int i = 0; i < 4; i += 2)
#pragma unroll
                for (int n = 0; n < NT; ++n)
                  mma_f16(s[n][u], a[0][i], a[1][i], a[0][i + 1], a[1][i + 1], q[n][0][4 * w + i], q[n][0][4 * w + i + 1]);
            }
          }
          if (kParts == 2) add4(s[0][u], small);
        }
        // ---- weights.  Pair h of unit u: row `row` of the warp's, query columns 2cc and 2cc + 1
        float2 z[NT][kUnits][2];
        float vs[kUnits][2];
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int row = row_of(QUAD ? c >> 1 : u, r) + 2 * h;
            const float ks = step.ks[row];
            vs[u][h] = step.vs[row];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              float2 x = make_float2(s[n][u][2 * h], s[n][u][2 * h + 1]);
              if (QUAD) {                          // the upper lanes take the second tile
                const float a = __shfl_xor_sync(0xffffffffu, s[n][kTiles - 1][2 * h], 2);
                const float b = __shfl_xor_sync(0xffffffffu, s[n][kTiles - 1][2 * h + 1], 2);
                if (c >= 2) x = make_float2(a, b);
              }
              // the two scales first: a product of codes and normalised queries times a large row scale alone would overflow
              // where tiny queries make up for it
              z[n][u][h] = mul2(x, mul2(both(ks), to_log2[n]));
            }
          }
        if (!whole_step) {
          asm volatile("" ::: "memory");           // a branch: as selections it was a tenth of a step
#pragma unroll
          for (int u = 0; u < kUnits; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              if (absent(row_of(QUAD ? c >> 1 : u, r) + 2 * h)) {
#pragma unroll
                for (int n = 0; n < NT; ++n) z[n][u][h] = both(-INFINITY);
              }
        }
        float2 wt[NT][kUnits][2];                  // weights, then times the value's scale
        float2 sum[NT];
        bool far = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float ahead = 0.f, most = 0.f;
          sum[n] = both(0.f);
#pragma unroll
          for (int u = 0; u < kUnits; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float2 d = add2(z[n][u][h], less[n]);
              ahead = fmaxf(ahead, fmaxf(d.x, d.y));
              wt[n][u][h] = make_float2(ptx::ex2_approx(d.x), ptx::ex2_approx(d.y));
              sum[n] = add2(sum[n], wt[n][u][h]);
              wt[n][u][h] = mul2(mul2(wt[n][u][h], both(vs[u][h])), inv[n]);
              most = fmaxf(most, fmaxf(wt[n][u][h].x, wt[n][u][h].y));
            }
          far = far || ahead > kAhead || most > kMost;
        }
        if (__any_sync(0xffffffffu, far)) {
          // ---- the references move: sums so far are rescaled, the weights of this step taken again
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            float top[2] = {m[n].x, m[n].y}, most[2];
#pragma unroll
            for (int u = 0; u < kUnits; ++u)
#pragma unroll
              for (int h = 0; h < 2; ++h) { top[0] = fmaxf(top[0], z[n][u][h].x); top[1] = fmaxf(top[1], z[n][u][h].y); }
            float f[2], old[2] = {m[n].x, m[n].y}, was[2] = {big[n].x, big[n].y};
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              top[x] = top_of_columns(top[x]);
              f[x] = old[x] == top[x] ? 1.f : ptx::ex2_approx(old[x] - top[x]);   // equal infinities included
              most[x] = was[x] * f[x];
            }
            m[n] = make_float2(top[0], top[1]);
            less[n] = make_float2(top[0] == -INFINITY ? kNoReference : -top[0], top[1] == -INFINITY ? kNoReference : -top[1]);
            l[n] = mul2(l[n], make_float2(f[0], f[1]));
            sum[n] = both(0.f);
#pragma unroll
            for (int u = 0; u < kUnits; ++u)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const float2 d = add2(z[n][u][h], less[n]);
                wt[n][u][h] = make_float2(ptx::ex2_approx(d.x), ptx::ex2_approx(d.y));
                sum[n] = add2(sum[n], wt[n][u][h]);
                wt[n][u][h] = mul2(wt[n][u][h], both(vs[u][h]));
                most[0] = fmaxf(most[0], wt[n][u][h].x);
                most[1] = fmaxf(most[1], wt[n][u][h].y);
              }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              most[x] = fmaxf(top_of_columns(most[x]), kLeastTop);
              f[x] *= was[x] * __frcp_rn(most[x]);
            }
            big[n] = make_float2(most[0], most[1]);
            inv[n] = make_float2(kTop * __frcp_rn(most[0]), kTop * __frcp_rn(most[1]));
#pragma unroll
            for (int u = 0; u < kUnits; ++u)
#pragma unroll
              for (int h = 0; h < 2; ++h) wt[n][u][h] = mul2(wt[n][u][h], inv[n]);
#pragma unroll
            for (int i = 0; i < kM; ++i) {
              o[n][i][0] *= f[0]; o[n][i][1] *= f[1];
              o[n][i][2] *= f[0]; o[n][i][3] *= f[1];
            }
          }
        }
        // P^T: first and second halves of the weights, of a tile in one matrix (QUAD) or in two
        constexpr int kB = QUAD ? 1 : 2;
        uint32_t weight[NT][kTiles][kB][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          l[n] = add2(l[n], sum[n]);
#pragma unroll
          for (int u = 0; u < kUnits; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const __half2 hi = __floats2half2_rn(wt[n][u][h].x, wt[n][u][h].y);
              const float2 back = __half22float2(hi);
              const uint32_t first = bits(hi), second = bits(__floats2half2_rn(wt[n][u][h].x - back.x, wt[n][u][h].y - back.y));
              if (QUAD) {
                // lower lanes have the first tile and give its second halves, upper lanes the second tile and its first ones
                const uint32_t got = __shfl_xor_sync(0xffffffffu, c < 2 ? second : first, 2);
                weight[n][0][0][h] = transpose8(c < 2 ? first : got);
                weight[n][kTiles - 1][0][h] = transpose8(c < 2 ? got : second);
              } else {
                weight[n][u][0][h] = transpose8(first);
                weight[n][u][kB - 1][h] = transpose8(second);
              }
            }
        }
        // ---- O^T += V^T P^T.  Lane r has elements DH/8 * r ... of four rows; elements 2i and 2i + 1 are its rows of tile i
#pragma unroll
        for (int u = 0; u < kTiles; ++u) {
          uint32_t x[4][DH / 64], g[4];
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            const int in_chunk = 4 * u + 2 * (h >> 1) + (h & 1), row = 8 * c + in_chunk;
            const unsigned char* at = step.v + c * R::kChunk + in_chunk * R::kBytes + r * (R::kBytes / 8);
            if constexpr (DH == 128) {
              const uint2 v = *reinterpret_cast<const uint2*>(at);
              x[h][0] = v.x;
              x[h][DH / 64 - 1] = v.y;
            } else {
              x[h][0] = *reinterpret_cast<const uint32_t*>(at);
            }
            g[h] = step.vg[row][r * (DH / 64) / 2];
          }
          __half2 scale[2];
#pragma unroll
          for (int t = 0; t < 2; ++t) scale[t] = halves(e4m3x2_to_half2(g[2 * t] | (g[2 * t + 1] << 8)));
#pragma unroll
          for (int y = 0; y < DH / 64; ++y) {
            uint32_t even[2][4], odd[2][4];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              const uint32_t a = x[2 * t][y], b = x[2 * t + 1][y];
              e2m1x8_to_half2((a & 0x0f0f0f0fu) | ((b << 4) & 0xf0f0f0f0u), even[t]);
              e2m1x8_to_half2(((a >> 4) & 0x0f0f0f0fu) | (b & 0xf0f0f0f0u), odd[t]);
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                even[t][i] = bits(__hmul2(halves(even[t][i]), scale[t]));
                odd[t][i] = bits(__hmul2(halves(odd[t][i]), scale[t]));
              }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                // Cut-off sums again: a chain over all rows of a warp ends up to half a step a tile low.  For float32 queries
                // each tile begins anew and is added with a rounding (448 heads of 100000 rows with values of one sign:
                // 8.5e-5 off on the average in one chain)
                float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int b = 0; b < kB; ++b)
                  mma_f16(kParts == 2 ? d : o[n][4 * y + i], even[0][i], odd[0][i], even[1][i], odd[1][i], weight[n][u][b][0],
                          weight[n][u][b][1]);
                if (kParts == 2) add4(o[n][4 * y + i], d);
              }
          }
        }
      }
      fetch(stage, next);
      look_up(next);
      if (++stage == RING) stage = 0;
    }
    // ---- the warps meet in shared memory: references first, then the sums rescaled to the largest, four queries at a time
#pragma unroll
    for (int n = 0; n < NT; ++n)
      if (r == 0 && c == cc) *reinterpret_cast<float2*>(&sh.m[warp][8 * n + 2 * cc]) = m[n];
    __syncthreads();                               // also: everything of the previous item has been read
    float2 factor[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float own[2] = {m[n].x, m[n].y}, sums[2] = {l[n].x, l[n].y}, bigs[2] = {big[n].x, big[n].y};
      float fs[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int row = 8 * n + 2 * cc + x;
        float top = sh.m[0][row];
#pragma unroll
        for (int w = 1; w < kDecodeWarps; ++w) top = fmaxf(top, sh.m[w][row]);
        const float f = own[x] == -INFINITY ? 0.f : ptx::ex2_approx(own[x] - top);
        float sum = sums[x];
        if (QUAD) sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        sum += __shfl_xor_sync(0xffffffffu, sum, 4);
        sum += __shfl_xor_sync(0xffffffffu, sum, 8);
        sum += __shfl_xor_sync(0xffffffffu, sum, 16);
        if (r == 0 && c == cc) {
          sh.l[warp][row] = sum * f;
          if (warp == 0) sh.top[row] = top;
        }
        fs[x] = f * (bigs[x] * (1.f / kTop));
      }
      factor[n] = make_float2(fs[0], fs[1]);
    }
    if (QUAD) {                                    // what the second halves of the weights came to
#pragma unroll
      for (int i = 0; i < kM; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[0][i][e] += __shfl_xor_sync(0xffffffffu, o[0][i][e], 2);
    }
    const bool whole = seg.t0 == 0 && seg.t1 == seg.tiles;
#pragma unroll
    for (int g = 0; g < (QUAD ? 1 : 2 * NT); ++g) {
      if (4 * g < it.rows) {
        if (g > 0) __syncthreads();
        if (c / 2 == g % 2) {
          constexpr int E = DH / 8;                // elements of a lane
          const int n = g / 2;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            float* dst = sh.o[warp][2 * (c % 2) + x] + E * r;
            const float f = x ? factor[n].y : factor[n].x;
#pragma unroll
            for (int e = 0; e < E; e += 4)
              *reinterpret_cast<float4*>(dst + e) = make_float4(o[n][e / 2][x] * f, o[n][e / 2][2 + x] * f, o[n][e / 2 + 1][x] * f,
                                                                o[n][e / 2 + 1][2 + x] * f);
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
    seg = following(seg);
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  if (p.team) join_team<T, DH>(p, walk, &sh.parts[0][0]);
  else if (threadIdx.x == 0) p.join[blockIdx.x] = join;
}

template <typename T, int DH, int NT, bool QUAD> cudaError_t launch(DecodeArgs p, int device, int sm_count, cudaStream_t st, int* launches) {
  constexpr int RING = NT == 1 ? 2 : 3, CTAS = NT == 1 ? 3 : 2;
  const auto kernel = decode_four_kernel<T, DH, NT, QUAD, RING, CTAS>;
  constexpr int smem = (int)sizeof(Shared<DH, NT, RING>);
  static LaunchSetup setup;
  const LaunchSetup::Fit* fit = setup.of(kernel, device, smem);
  if (!fit) return cudaErrorInvalidDeviceFunction;
  p.team = decode_team(p, *fit, sm_count, kRows);
  const int grid = p.team ? p.items * p.team : decode_grid(p, fit->per_sm * sm_count, kRows);
  *launches += 1;
  const cudaError_t e = launch_early_in_clusters<DecodeArgs>(kernel, dim3(grid), kDecodeThreads, smem, p.team, st, p);
  if (e != cudaSuccess || p.team) return e;
  *launches += 1;
  return launch_decode_join<T, DH>(p, grid, st);
}

template <typename T, int DH> cudaError_t by_queries(const DecodeArgs& p, int device, int sm_count, cudaStream_t st, int* launches) {
  if (p.part_rows <= 4) return launch<T, DH, 1, true>(p, device, sm_count, st, launches);
  if constexpr (sizeof(T) == 2) {
    if (p.chunk_rows == 16) return launch<T, DH, 2, false>(p, device, sm_count, st, launches);
  }
  return launch<T, DH, 1, false>(p, device, sm_count, st, launches);
}
template <typename T> cudaError_t by_shape(const DecodeArgs& p, int dh, int device, int sm_count, cudaStream_t st, int* launches) {
  return dh == 64 ? by_queries<T, 64>(p, device, sm_count, st, launches) : by_queries<T, 128>(p, device, sm_count, st, launches);
}

}  // namespace

cudaError_t launch_decode_four(const CacheDims& d, const DecodeCall& call, int device, int sm_count, int* status_word, cudaStream_t st,
                               int* launches) {
  // queries of a KV head: 8 or 16 an item, as paged_decode_mma.cu (float32 queries, of two halves, have registers for 8)
  const DecodeArgs p = decode_args(d, call, d.Hq / d.Hkv <= 8 || d.dtype == CKV_F32 ? 8 : 16, status_word);
  return d.dtype == CKV_F32 ? by_shape<float>(p, d.dh, device, sm_count, st, launches)
                            : by_shape<__nv_bfloat16>(p, d.dh, device, sm_count, st, launches);
}

}  // namespace ckv
