// Decode attention over pages in 4 bits a value, on tensor cores.
//
// The products are those of paged_decode_mma.cu: the cache rows on the 16-row side of mma.sync, 8 queries on the other,
// S^T = K Q^T, then O^T = V^T P^T.  A row of 128 elements is 76 bytes, so the kernel is bound by the instructions that turn
// codes into halves, and everything else is kept short.
//
//   codes      cvt takes two codes of a byte to two halves; code times group scale is exact in a half (2 and 4 significant
//              bits), one instruction for two elements.  K: a byte is two elements of a row.  V: the matrix instruction wants two
//              rows of an element in a register, so the half bytes of two rows are mixed first, two instructions for four
//              registers.
//   queries    halves after a scaling by a power of two that puts the largest element at 2^14, as for 8-bit pages; a float32
//              query is the sum of two halves (an error of 2^-24 of an element, or 2^-39 of the largest), two products each.
//   softmax    a warp's logits are taken relative to a maximum that is moved only when one is 2^10 times above it, and its
//              weights (times the row scales) relative to a largest one that is moved only when one is 16 times above it: sums
//              are rescaled a few times a head instead of in most steps.  A weight enters the second product as two halves
//              (22 bits, no finer than 2^-36 of the largest such product).  Float pairs go through the packed instructions.
//   copies     a warp has a ring of steps of 32 rows, filled by TMA: codes, group scales and row scales of K and of V, each
//              copy issued by a lane of its own, one barrier a step.
#include "paged_decode.cuh"
#include "sm100_ptx.cuh"
#include "tma_host.h"

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
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 negative(float2 x) { return make_float2(-x.x, -x.y); }

constexpr float kTop = 2048.f;         // where the largest product of a weight and a row scale is put ...
constexpr float kMost = 32768.f;       // ... and what a later one may reach before it is moved
constexpr float kAhead = 10.f;         // log2 of what a weight may reach before the maximum is moved
constexpr float kLeastTop = 3.851859888774472e-34f;   // 2^-111: kTop over it and it over kTop are normal floats

// In place of minus the reference where no logit has been seen: any logit is far above it, and -infinity has weight 0.
constexpr float kNoReference = 3.4028234e38f;

constexpr int kRows = 32, kTiles = kRows / 16;   // rows of a step, in tiles of the matrix instruction

template <int DH> struct Row {
  static constexpr int kBytes = DH / 2, kGroups = DH / 16, kWords = DH / 32;   // of codes; scales; words of codes a quad lane has
  // 16-byte piece `chunk` of a row as TMA writes it (64-byte rows: 64-byte swizzle, 32-byte rows: none)
  static __device__ __forceinline__ int at(int row, int chunk) {
    return row * kBytes + ((DH == 128 ? chunk ^ ((row >> 1) & 3) : chunk) * 16);
  }
  // Cache row of a tile that row i of the matrix instruction stands for (i + 8: 8 further), so that neither read has bank
  // conflicts.  64 bytes: neighbours differ in bit 0, rows 0, 2, 4, 6 (and 1, 3, 5, 7) in bits 0 and 2; 32 bytes: four
  // neighbours, and those rows, in bits 0 and 1.
  static __device__ __forceinline__ int of(int i) {
    constexpr uint32_t order = DH == 128 ? 0x65742130u    // 0 3 1 2 4 7 5 6
                                         : 0x67453210u;   // 0 1 2 3 5 4 7 6
    return (order >> (4 * i)) & 7;
  }
};

template <int DH> struct alignas(1024) Step {      // the rows of a step in shared memory
  unsigned char k[kRows * Row<DH>::kBytes], v[kRows * Row<DH>::kBytes];
  uint8_t kg[kRows][Row<DH>::kGroups], vg[kRows][Row<DH>::kGroups];
  float ks[kRows], vs[kRows];
  int here[2];                                     // rows that exist in either half (a page may end between them)
};

template <int DH, int NT, int RING> struct Shared {
  Step<DH> ring[kDecodeWarps][RING];
  float o[kDecodeWarps][4][DH];                    // four queries at a time
  float m[kDecodeWarps][8 * NT], l[kDecodeWarps][8 * NT], top[8 * NT];
  alignas(8) float parts[8 * NT][DH + 2];          // of a CTA of a team
  uint64_t full[kDecodeWarps][RING];
  uint32_t late;                                   // a copy did not arrive in time: the other waits give up too
};

// A CTA's part of an item: tiles [t0, t1) of it, a tile being a step of every warp.
struct Segment {
  int item, kv, len, tiles, t0, t1;
  int first;                                       // the item's first tile in the list of all tiles
};

template <typename T, int DH, int NT, int RING, int CTAS>
__global__ void __launch_bounds__(kDecodeThreads, CTAS)
    decode_four_kernel(const __grid_constant__ DecodeArgs p, const __grid_constant__ CUtensorMap k_map,
                       const __grid_constant__ CUtensorMap v_map) {
  using R = Row<DH>;
  constexpr int kTile = kDecodeWarps * kRows;
  constexpr int kParts = sizeof(T) == 4 ? 2 : 1;   // halves a query element is the sum of
  constexpr int kQ = DH / 8;                       // registers of a query's elements
  constexpr int kM = DH / 16;                      // 16-row tiles of V^T
  extern __shared__ unsigned char smem_raw[];
  Shared<DH, NT, RING>& sh = *reinterpret_cast<Shared<DH, NT, RING>*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32, r = lane >> 2, c = lane & 3;
  if (threadIdx.x < kDecodeWarps * RING) ptx::mbar_init(ptx::smem_addr(&sh.full[0][0] + threadIdx.x), 1);
  if (threadIdx.x == 0) {
    sh.late = 0;
    ptx::prefetch_tensormap(&k_map);
    ptx::prefetch_tensormap(&v_map);
  }
  ptx::fence_barrier_init();
  wait_for_previous_kernel();
  const Walk walk = p.team ? team_walk<T, DH, kTile>(p) : plan<T, DH, kTile>(p);
  if (threadIdx.x < 8 * NT) *reinterpret_cast<float2*>(&sh.parts[threadIdx.x][DH]) = make_float2(-INFINITY, 0.f);
  __syncthreads();                                 // the mbarriers are visible

  // The segment behind `g` (its item, first and tiles), or one with t0 == t1.
  auto following = [&](Segment g) {
    while (true) {
      g.first += g.tiles;
      g.item += 1;
      g.t0 = g.t1 = 0;
      if (g.first >= walk.end) return g;
      g.kv = kv_of(p, g.item);
      g.len = item_len(p, g.kv);
      g.tiles = (g.len + kTile - 1) / kTile;
      g.t0 = max(walk.begin - g.first, 0);
      g.t1 = min(g.tiles, walk.end - g.first);
      if (g.t1 > g.t0) return g;
    }
  };

  // ---- copies.  Lane 8h + kind of a warp fetches one of the six arrays, of all rows of a step (h = 0) or, where a page has
  // 16 rows, of its half h.
  const bool halved = p.c.page_shift == 4;
  const int kind = lane & 7, half = lane >> 3 & 1;
  const bool copies = kind < 6 && lane < (halved ? 16 : 8);
  const int count = halved ? 16 : 32;              // rows of a copy
  Segment front;                                   // what is looked up next
  int front_left, front_base;                      // steps of `front` left, first row of the next one
  int page = -1, here = 0, in_page = 0;            // of this lane's copy in the step that is fetched next
  auto look_up = [&]() {
    here = 0;
    page = -1;
    if (front_left == 0) {
      if (front.t0 < front.t1) front = following(front);
      front_left = front.t1 - front.t0;
      front_base = (front.t0 * kDecodeWarps + warp) * kRows;
    }
    if (front_left > 0) {
      const int base = front_base + (halved ? 16 * half : 0);
      here = max(0, min(front.len - base, count));
      in_page = base & ((1 << p.c.page_shift) - 1);
      if (here > 0) page = p.c.table[(long long)front.kv * p.c.max_pages + (base >> p.c.page_shift)];
      front_left -= 1;
      front_base += kTile;
    }
  };
  auto fetch = [&](int stage) {
    Step<DH>& to = sh.ring[warp][stage];
    if (here > 0 && (unsigned)page >= (unsigned)p.c.num_pages) {
      if (p.status != nullptr && copies) atomicExch(p.status, (int)CKV_EBOUNDS);
      here = 0;
    }
    const uint32_t full = ptx::smem_addr(&sh.full[warp][stage]);
    const bool go = here > 0;
    const int n = go + (halved ? (int)__shfl_xor_sync(0xffffffffu, (int)go, 8) : 0);
    __syncwarp();                                  // every lane has read what the slot held
    if (kind == 0 && lane < 16) {
      if (halved) to.here[half] = here;
      else to.here[half] = max(0, min(here - 16 * half, 16));
    }
    if (lane == 0) ptx::mbar_arrive_expect_tx(full, n * count * 2 * (R::kBytes + R::kGroups + 4));
    __syncwarp();
    if (copies && go) {
      const int row = halved ? 16 * half : 0;
      if (kind < 2) {
        ptx::tma_load_4d(ptx::smem_addr(kind == 0 ? to.k : to.v) + row * R::kBytes, kind == 0 ? &k_map : &v_map, 0, in_page, 0, page, full);
      } else {
        const long long slot = ((long long)page << p.c.page_shift) + in_page;
        const int w = kind & 1;
        if (kind < 4)
          ptx::bulk_load(ptx::smem_addr(w ? to.vg[row] : to.kg[row]), p.c.group[w] + slot * R::kGroups, count * R::kGroups, full);
        else
          ptx::bulk_load(ptx::smem_addr(w ? to.vs + row : to.ks + row), p.c.scale[w] + slot, count * 4, full);
      }
    }
  };

  const int k_row = R::of(r);
  // The queries of an item, in the element order of the K pieces: lane c of a quad has elements DH/4 * c ...
  uint32_t q[NT][kParts][kQ];
  float2 to_log2[NT];                              // factor of the products for query columns 2c, 2c + 1
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
      float up[2];
#pragma unroll
      for (int x2 = 0; x2 < 2; ++x2)
        up[x2] = p.scale_log2 * __int_as_float((127 + __shfl_sync(0xffffffffu, e, 8 * c + 4 * x2)) << 23);   // of query 8n + 2c + x2
      to_log2[n] = make_float2(up[0], up[1]);
    }
  };

  bool ok = true;                                  // no wait of this lane has run out
  int2 join = make_int2(-1, 0);
  Segment seg;
  seg.item = walk.item - 1;
  seg.kv = seg.len = 0;
  seg.first = walk.first;
  seg.tiles = 0;
  seg.t0 = seg.t1 = 0;
  if (walk.begin < walk.end) seg = following(seg);
  front = seg;
  front_left = seg.t1 - seg.t0;
  front_base = (seg.t0 * kDecodeWarps + warp) * kRows;
  int stage = 0;
  uint32_t phase = 0;
  if (seg.t0 < seg.t1) {
    look_up();
    for (int i = 0; i < RING; ++i) {
      fetch(i);
      look_up();
    }
  }
  while (seg.t0 < seg.t1 && ok) {
    const ItemRows it = item_rows(p, seg.kv, seg.item - seg.kv * p.chunks);
    load_queries(seg);
    float o[NT][kM][4];                            // [tile of V^T][even, odd element; query columns 2c, 2c + 1]
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
      if (!ptx::mbar_wait_bounded(ptx::smem_addr(&sh.full[warp][stage]), phase, &sh.late)) {
        ok = false;
        *(volatile uint32_t*)&sh.late = 1;
      }
      if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
      const int rows0 = step.here[0], rows1 = step.here[1];
      const bool whole_step = rows0 + rows1 == kRows;
      if (rows0 + rows1 > 0) {
        // ---- logits
        float s[NT][kTiles][4];
#pragma unroll
        for (int u = 0; u < kTiles; ++u) {
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][u][e] = 0.f;
          uint32_t x[2][R::kWords];
          __half2 g[2][DH / 64];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int row = 16 * u + 8 * h + k_row;
            const uint8_t* group = step.kg[row] + c * (DH / 64);
            if constexpr (DH == 128) {
              const uint4 v = *reinterpret_cast<const uint4*>(step.k + R::at(row, c));
              x[h][0] = v.x; x[h][1] = v.y; x[h][R::kWords - 2] = v.z; x[h][R::kWords - 1] = v.w;
              const __half2 pair = halves(e4m3x2_to_half2(*reinterpret_cast<const uint16_t*>(group)));
              g[h][0] = __low2half2(pair);
              g[h][DH / 64 - 1] = __high2half2(pair);
            } else {
              const uint2 v = *reinterpret_cast<const uint2*>(step.k + R::at(row, c / 2) + 8 * (c % 2));
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
#pragma unroll
            for (int i = 0; i < 4; i += 2)
#pragma unroll
              for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int part = 0; part < kParts; ++part)
                  mma_f16(s[n][u], a[0][i], a[1][i], a[0][i + 1], a[1][i + 1], q[n][part][4 * w + i], q[n][part][4 * w + i + 1]);
          }
        }
        // ---- weights.  Pair h of a tile: row k_row + 8h, query columns 2c and 2c + 1
        float2 z[NT][kTiles][2];
        float vs[kTiles][2];
#pragma unroll
        for (int u = 0; u < kTiles; ++u)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int row = 16 * u + 8 * h + k_row;
            const float ks = step.ks[row];
            vs[u][h] = step.vs[row];
            // the two scales first: a product of codes and normalised queries times a large row scale alone would overflow
            // where tiny queries make up for it
#pragma unroll
            for (int n = 0; n < NT; ++n)
              z[n][u][h] = mul2(make_float2(s[n][u][2 * h], s[n][u][2 * h + 1]), mul2(both(ks), to_log2[n]));
          }
        if (!whole_step) {
#pragma unroll
          for (int u = 0; u < kTiles; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              if (8 * h + k_row >= (u ? rows1 : rows0)) {
                vs[u][h] = 1.f;
#pragma unroll
                for (int n = 0; n < NT; ++n) z[n][u][h] = both(-INFINITY);
              }
        }
        float2 w[NT][kTiles][2];                   // weights, then times the value's scale
        float2 sum[NT];
        bool far = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float ahead = 0.f, most = 0.f;
#pragma unroll
          for (int u = 0; u < kTiles; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float2 d = add2(z[n][u][h], less[n]);
              ahead = fmaxf(ahead, fmaxf(d.x, d.y));
              const float2 e = make_float2(ptx::ex2_approx(d.x), ptx::ex2_approx(d.y));
              w[n][u][h] = e;
            }
          far = far || ahead > kAhead;
          sum[n] = both(0.f);
#pragma unroll
          for (int u = 0; u < kTiles; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              sum[n] = add2(sum[n], w[n][u][h]);
              w[n][u][h] = mul2(mul2(w[n][u][h], both(vs[u][h])), inv[n]);
              most = fmaxf(most, fmaxf(w[n][u][h].x, w[n][u][h].y));
            }
          far = far || most > kMost;
        }
        if (__any_sync(0xffffffffu, far)) {
          // ---- the references move: sums so far are rescaled, the weights of this step taken again
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            float top[2] = {m[n].x, m[n].y}, most[2];
#pragma unroll
            for (int u = 0; u < kTiles; ++u)
#pragma unroll
              for (int h = 0; h < 2; ++h) { top[0] = fmaxf(top[0], z[n][u][h].x); top[1] = fmaxf(top[1], z[n][u][h].y); }
            float f[2], old[2] = {m[n].x, m[n].y}, was[2] = {big[n].x, big[n].y};
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], 4));
              top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], 8));
              top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], 16));
              f[x] = old[x] == top[x] ? 1.f : ptx::ex2_approx(old[x] - top[x]);   // equal infinities included
              most[x] = was[x] * f[x];
            }
            m[n] = make_float2(top[0], top[1]);
            less[n] = make_float2(top[0] == -INFINITY ? kNoReference : -top[0], top[1] == -INFINITY ? kNoReference : -top[1]);
            l[n] = mul2(l[n], make_float2(f[0], f[1]));
            sum[n] = both(0.f);
#pragma unroll
            for (int u = 0; u < kTiles; ++u)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const float2 d = add2(z[n][u][h], less[n]);
                w[n][u][h] = make_float2(ptx::ex2_approx(d.x), ptx::ex2_approx(d.y));
                sum[n] = add2(sum[n], w[n][u][h]);
                w[n][u][h] = mul2(w[n][u][h], both(vs[u][h]));
                most[0] = fmaxf(most[0], w[n][u][h].x);
                most[1] = fmaxf(most[1], w[n][u][h].y);
              }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              most[x] = fmaxf(most[x], __shfl_xor_sync(0xffffffffu, most[x], 4));
              most[x] = fmaxf(most[x], __shfl_xor_sync(0xffffffffu, most[x], 8));
              most[x] = fmaxf(most[x], __shfl_xor_sync(0xffffffffu, most[x], 16));
              most[x] = fmaxf(most[x], kLeastTop);
              f[x] *= was[x] * __frcp_rn(most[x]);
            }
            big[n] = make_float2(most[0], most[1]);
            inv[n] = make_float2(kTop * __frcp_rn(most[0]), kTop * __frcp_rn(most[1]));
#pragma unroll
            for (int u = 0; u < kTiles; ++u)
#pragma unroll
              for (int h = 0; h < 2; ++h) w[n][u][h] = mul2(w[n][u][h], inv[n]);
#pragma unroll
            for (int i = 0; i < kM; ++i) {
              o[n][i][0] *= f[0]; o[n][i][1] *= f[1];
              o[n][i][2] *= f[0]; o[n][i][3] *= f[1];
            }
          }
        }
        uint32_t w_hi[NT][kTiles][2], w_lo[NT][kTiles][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          l[n] = add2(l[n], sum[n]);
#pragma unroll
          for (int u = 0; u < kTiles; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const __half2 hi = __floats2half2_rn(w[n][u][h].x, w[n][u][h].y);
              const float2 rest = add2(w[n][u][h], negative(__half22float2(hi)));
              w_hi[n][u][h] = transpose8(bits(hi));
              w_lo[n][u][h] = transpose8(bits(__floats2half2_rn(rest.x, rest.y)));
            }
        }
        // ---- O^T += V^T P^T.  Lane r has elements DH/8 * r ... of four rows; elements 2i and 2i + 1 are its rows of tile i
#pragma unroll
        for (int u = 0; u < kTiles; ++u) {
          uint32_t x[4][DH / 64], g[4];
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            const int in_tile = R::of(2 * c + (h & 1)) + 8 * (h >> 1), row = 16 * u + in_tile;
            if constexpr (DH == 128) {
              const uint2 v = *reinterpret_cast<const uint2*>(step.v + R::at(row, r / 2) + 8 * (r % 2));
              x[h][0] = v.x;
              x[h][DH / 64 - 1] = v.y;
            } else {
              x[h][0] = *reinterpret_cast<const uint32_t*>(step.v + R::at(row, r / 4) + 4 * (r % 4));
            }
            g[h] = step.vg[row][r * (DH / 64) / 2];
            if (!whole_step && in_tile >= (u ? rows1 : rows0)) {       // what is left there may be no number
              x[h][0] = x[h][DH / 64 - 1] = 0;
              g[h] = 0;
            }
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
                mma_f16(o[n][4 * y + i], even[0][i], odd[0][i], even[1][i], odd[1][i], w_hi[n][u][0], w_hi[n][u][1]);
                mma_f16(o[n][4 * y + i], even[0][i], odd[0][i], even[1][i], odd[1][i], w_lo[n][u][0], w_lo[n][u][1]);
              }
          }
        }
      }
      fetch(stage);
      look_up();
      if (++stage == RING) { stage = 0; phase ^= 1; }
    }
    // ---- the warps meet in shared memory: references first, then the sums rescaled to the largest, four queries at a time
#pragma unroll
    for (int n = 0; n < NT; ++n)
      if (r == 0) *reinterpret_cast<float2*>(&sh.m[warp][8 * n + 2 * c]) = m[n];
    ok = !__syncthreads_or(!ok);                   // also: everything of the previous item has been read
    if (!ok) break;
    float2 factor[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float own[2] = {m[n].x, m[n].y}, sums[2] = {l[n].x, l[n].y}, bigs[2] = {big[n].x, big[n].y};
      float fs[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int row = 8 * n + 2 * c + x;
        float top = sh.m[0][row];
#pragma unroll
        for (int w = 1; w < kDecodeWarps; ++w) top = fmaxf(top, sh.m[w][row]);
        const float f = own[x] == -INFINITY ? 0.f : ptx::ex2_approx(own[x] - top);
        float sum = sums[x];
        sum += __shfl_xor_sync(0xffffffffu, sum, 4);
        sum += __shfl_xor_sync(0xffffffffu, sum, 8);
        sum += __shfl_xor_sync(0xffffffffu, sum, 16);
        if (r == 0) {
          sh.l[warp][row] = sum * f;
          if (warp == 0) sh.top[row] = top;
        }
        fs[x] = f * (bigs[x] * (1.f / kTop));
      }
      factor[n] = make_float2(fs[0], fs[1]);
    }
    const bool whole = seg.t0 == 0 && seg.t1 == seg.tiles;
#pragma unroll
    for (int g = 0; g < 2 * NT; ++g) {
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
  if (!ok) {
    // a copy did not arrive in time: report it, and give what is still on its way a last chance before the CTA (and with
    // it the shared memory the copies write) goes away
    if (threadIdx.x == 0) atomicExch(p.timeout, (int)CKV_ETIMEOUT);
    volatile uint32_t zero = 0;
    for (int i = 0; i < RING; ++i)
      for (int x = 0; x < 2; ++x) ptx::mbar_wait_bounded(ptx::smem_addr(&sh.full[warp][i]), phase ^ x, &zero, 100000000ull);
  }
  if (p.team) join_team<T, DH>(p, walk, &sh.parts[0][0]);
  else if (threadIdx.x == 0) p.join[blockIdx.x] = join;
}

// Pages as TMA sees them: bytes of a row x rows of a page x 1 x pages.
template <int DH> bool page_map(CUtensorMap* m, const DecodeArgs& p, int which) {
  EncodeTiledFn fn = tma_encode_fn();
  if (!fn) return false;
  using R = Row<DH>;
  const int box_rows = p.c.page_shift == 4 ? 16 : kRows;
  const cuuint64_t dims[4] = {(cuuint64_t)R::kBytes, (cuuint64_t)1 << p.c.page_shift, 1, (cuuint64_t)p.c.num_pages};
  const cuuint64_t strides[3] = {(cuuint64_t)R::kBytes, (cuuint64_t)p.c.page_stride, (cuuint64_t)p.c.page_stride};
  const cuuint32_t box[4] = {(cuuint32_t)R::kBytes, (cuuint32_t)box_rows, 1, 1}, ones[4] = {1, 1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, p.c.page[which], dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
            DH == 128 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int DH, int NT> cudaError_t launch(DecodeArgs p, int device, int sm_count, cudaStream_t st, int* launches) {
  constexpr int RING = 3, CTAS = NT == 1 ? 3 : 2;
  const auto kernel = decode_four_kernel<T, DH, NT, RING, CTAS>;
  constexpr int smem = (int)sizeof(Shared<DH, NT, RING>) + 1024;   // the steps start on a multiple of 1024
  constexpr int tile = kDecodeWarps * kRows;
  static LaunchSetup setup;
  const LaunchSetup::Fit* fit = setup.of(kernel, device, smem);
  if (!fit) return cudaErrorInvalidDeviceFunction;
  CUtensorMap maps[2];
  for (int i = 0; i < 2; ++i)
    if (!page_map<DH>(&maps[i], p, i)) return cudaErrorInvalidValue;
  p.team = decode_team(p, *fit, sm_count, tile);
  const int grid = p.team ? p.items * p.team : decode_grid(p, fit->per_sm * sm_count, tile);
  *launches += 1;
  const cudaError_t e = launch_early_in_clusters<DecodeArgs, CUtensorMap, CUtensorMap>(kernel, dim3(grid), kDecodeThreads, smem,
                                                                                       p.team, st, p, maps[0], maps[1]);
  if (e != cudaSuccess || p.team) return e;
  *launches += 1;
  return launch_decode_join<T, DH>(p, grid, st);
}

template <typename T> cudaError_t by_shape(const DecodeArgs& p, int dh, int device, int sm_count, cudaStream_t st, int* launches) {
  if (p.chunk_rows == 8) return dh == 64 ? launch<T, 64, 1>(p, device, sm_count, st, launches) : launch<T, 128, 1>(p, device, sm_count, st, launches);
  return dh == 64 ? launch<T, 64, 2>(p, device, sm_count, st, launches) : launch<T, 128, 2>(p, device, sm_count, st, launches);
}

}  // namespace

cudaError_t launch_decode_four(const CacheDims& d, const DecodeCall& call, int device, int sm_count, int* status_word, cudaStream_t st,
                               int* launches) {
  // queries of a KV head: 8 or 16 an item, as paged_decode_mma.cu (float32 queries, of two halves, have registers for 8)
  const DecodeArgs p = decode_args(d, call, d.Hq / d.Hkv <= 8 || d.dtype == CKV_F32 ? 8 : 16, status_word);
  return d.dtype == CKV_F32 ? (d.dh == 64 ? launch<float, 64, 1>(p, device, sm_count, st, launches)
                                          : launch<float, 128, 1>(p, device, sm_count, st, launches))
                            : by_shape<__nv_bfloat16>(p, d.dh, device, sm_count, st, launches);
}

}  // namespace ckv
