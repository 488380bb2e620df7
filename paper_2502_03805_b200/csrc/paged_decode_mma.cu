// Decode attention for bf16 queries on tensor cores.
//
// A decode step multiplies every stored row with only the G = Hq/Hkv queries of its KV head: it is bound by the stream
// of K and V from HBM, and CUDA cores cannot keep up with that stream (at G = 4 and 8-bit pages the CUDA-core kernel
// reaches a quarter of it).  The matrix instruction is mma.sync with the CACHE ROWS on its 16-row side and 8 queries on
// the other: a query tile of tcgen05.mma would be 64 or 128 rows of which G are used, its operands would have to go
// through shared memory in the format of the instruction (8-bit pages converted on the way), and this kernel needs
// about a tenth of the mma.sync rate.  So every stored byte goes from global memory straight into the registers of the
// lane that feeds it to the matrix instruction, once:
//
//   S^T = K Q^T   A = 16 rows of K.  Lane (r, c) = (lane / 4, lane % 4) loads 16 bytes of rows r and r + 8; which of the
//                 row's elements those are is free, as long as the query fragments are loaded in the same order.
//   O^T = V^T P^T A = V^T: the lane needs two cache rows of one element in a register.  It loads 16 bytes of rows 2c,
//                 2c+1, 2c+8, 2c+9 and interleaves them with byte permutes; which elements form a 16-row tile is free
//                 again.  P^T is the accumulator of the first product with rows and columns exchanged (movmatrix).
//
// A warp works through 16 or 32 rows at a time: the V loads of a step are issued before its K Q^T, the K loads of the
// next step right after it, so 4 to 8 KB per warp are in flight all the time.  Softmax statistics are float32.
// The weights enter the second product as the sum of two bf16 numbers (16 bits) for bf16 pages; for 8-bit pages, whose
// codes are exact halves, as halves (11 bits) of weight * scale of the row / the largest such product so far, so that
// rows of very different norms keep their precision.  The queries of 8-bit pages become halves after a scaling by a
// power of two that puts the largest of a row at 2^14: exact but for elements 2^-29 below it.
#include "paged_decode.cuh"

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
// Two 8-bit codes, in the low 16 bits of `two` (int8: with the sign bit flipped), as two halves.  int8: 0x64uu is the
// half 1024 + u, so 1024 + 128 + code - 1152 is exact.
template <int FMT, bool HIGH> __device__ __forceinline__ uint32_t codes_to_half2(uint32_t four) {
  if (FMT == CKV_CACHE_E4M3) return e4m3x2_to_half2(HIGH ? four >> 16 : four);
  const uint32_t biased = __byte_perm(four, 0x64646464u, HIGH ? 0x4342 : 0x4140);
  const __half2 v = __hsub2(*reinterpret_cast<const __half2*>(&biased), __half2half2(__ushort_as_half(0x6480)));
  return *reinterpret_cast<const uint32_t*>(&v);
}

template <int FMT, int DH> struct Shape {
  static constexpr bool kPlain = FMT == CKV_CACHE_PLAIN;
  static constexpr int kRowBytes = kPlain ? DH * 2 : DH;
  static constexpr int kSub = kRowBytes >= 256 ? 1 : 2;            // 16-row groups a warp takes at a time
  static constexpr int kTile = kDecodeWarps * 16 * kSub;           // cache rows a CTA takes at a time
  static constexpr int kChunks = kRowBytes / 64;                   // 16-byte pieces of a K row per lane
  static constexpr int kQWords = kPlain ? 4 : 8;                   // registers of query elements per piece
  static constexpr int kVBytes = kRowBytes >= 128 ? 16 : 8;        // piece of a V row per lane
  static constexpr int kVPieces = kRowBytes / (8 * kVBytes);
  static constexpr int kElems = DH / 8;                            // V elements a lane has of a row
  static constexpr int kVWords = kVPieces * kVBytes / 4;           // registers they take
  static constexpr int kMTiles = kElems / 2;                       // 16-row tiles of V^T
};

// Where the 16 * SUB rows of a warp's step lie.
template <int SUB> struct Where {
  long long row[SUB];      // slot number of the first row: page * page_size + row in the page
  long long off[SUB];      // its byte offset in k_pages / v_pages
  int here[SUB];           // rows that exist, 0..16
};

template <int FMT, int DH, int NT>
__global__ void __launch_bounds__(kDecodeThreads, 3) decode_mma_kernel(DecodeArgs p) {
  using S = Shape<FMT, DH>;
  constexpr int SUB = S::kSub;
  using T = __nv_bfloat16;
  __shared__ float o_s[kDecodeWarps][8][DH];
  __shared__ float m_s[kDecodeWarps][8], l_s[kDecodeWarps][8];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, r = lane >> 2, c = lane & 3;
  const Walk walk = plan<T, DH, S::kTile>(p);
  asm volatile("griddepcontrol.launch_dependents;");
  int2 join = make_int2(-1, 0);
  long long first = walk.first, t = walk.begin;
  for (int item = walk.item; t < walk.end; ++item) {
    const ItemRows it = item_rows(p, item);
    const int len = item_len(p, it.kv);
    const int tiles = (len + S::kTile - 1) / S::kTile;
    if (first + tiles <= t) { first += tiles; continue; }
    const int t0 = (int)(t - first), t1 = (int)min((long long)tiles, walk.end - first);
    const int32_t* pages = p.c.table + (long long)it.kv * p.c.max_pages;

    auto locate = [&](int tile, Where<SUB>& w) {
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        const int base = tile * S::kTile + (warp * SUB + u) * 16;   // page_size is a multiple of 16: one page
        w.here[u] = max(0, min(len - base, 16));
        w.row[u] = w.off[u] = 0;
        if (w.here[u] > 0) {
          const int page = pages[base >> p.c.page_shift];
          if (page < 0 || page >= p.c.num_pages) {
            w.here[u] = 0;
            if (p.status != nullptr) atomicExch(p.status, (int)CKV_EBOUNDS);
          } else {
            const int in_page = base & ((1 << p.c.page_shift) - 1);
            w.row[u] = ((long long)page << p.c.page_shift) + in_page;
            w.off[u] = page * p.c.page_stride + (long long)in_page * S::kRowBytes;
          }
        }
      }
    };
    uint4 k[SUB][2][S::kChunks];
    float ks[SUB][2], vs[SUB][2];
    auto load_k = [&](const Where<SUB>& w) {
#pragma unroll
      for (int u = 0; u < SUB; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int i = r + 8 * h;
          const char* row = p.c.page[0] + w.off[u] + i * S::kRowBytes + c * 16;
#pragma unroll
          for (int j = 0; j < S::kChunks; ++j) {
            k[u][h][j] = make_uint4(0, 0, 0, 0);
            if (i < w.here[u]) k[u][h][j] = __ldg(reinterpret_cast<const uint4*>(row + 64 * j));
          }
        }
    };
    auto load_scales = [&](const Where<SUB>& w, float (&a)[SUB][2], float (&b)[SUB][2]) {
#pragma unroll
      for (int u = 0; u < SUB; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          a[u][h] = b[u][h] = 1.f;
          if (!S::kPlain && r + 8 * h < w.here[u]) {
            a[u][h] = __ldg(p.c.scale[0] + w.row[u] + r + 8 * h);
            b[u][h] = __ldg(p.c.scale[1] + w.row[u] + r + 8 * h);
          }
        }
    };

    // ---- queries, in the element order of the K pieces
    uint32_t q[NT][S::kChunks][S::kQWords];
    float scale_a[NT][2], scale_b[NT][2];      // logit = (S * ks * scale_a) * scale_b, for query columns 2c, 2c+1
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int row = 8 * n + r;
      const char* src = p.q + it.s * p.qs[0] + (it.head + row) * p.qs[1];
      if (S::kPlain) {
#pragma unroll
        for (int j = 0; j < S::kChunks; ++j) {
          uint4 v = make_uint4(0, 0, 0, 0);
          if (row < it.rows) v = *reinterpret_cast<const uint4*>(src + c * 16 + 64 * j);
          q[n][j][0] = v.x; q[n][j][1] = v.y; q[n][j][2] = v.z; q[n][j][3] = v.w;
        }
        scale_a[n][0] = scale_a[n][1] = 1.f;
        scale_b[n][0] = scale_b[n][1] = p.scale_log2;
      } else {
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < S::kChunks; ++j)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (row < it.rows) v = *reinterpret_cast<const uint4*>(src + (c + 4 * j) * 32 + 16 * h);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              q[n][j][(4 * h + i) % S::kQWords] = w[i];
              top = max(top, max((w[i] & 0x7fffu), (w[i] >> 16) & 0x7fffu));
            }
          }
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // exponent of the largest element minus 14; 0 for rows of zeros, infinities or NaN
        int e = 0;
        if (top != 0 && top < 0x7f80u) e = max((int)(top >> 7), 1) - 127 - 14;
        // 2^-e in two factors, both normal floats
        const float down_a = __int_as_float((127 - e / 2) << 23), down_b = __int_as_float((127 - (e - e / 2)) << 23);
#pragma unroll
        for (int j = 0; j < S::kChunks; ++j)
#pragma unroll
          for (int i = 0; i < S::kQWords; ++i) {
            const uint32_t w = q[n][j][i];
            q[n][j][i] = pack_half(__uint_as_float(w << 16) * down_a * down_b, __uint_as_float(w & 0xffff0000u) * down_a * down_b);
          }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int ec = __shfl_sync(0xffffffffu, e, 8 * c + 4 * h);       // of query 8n + 2c + h
          scale_a[n][h] = __int_as_float((127 + ec / 2) << 23);
          scale_b[n][h] = __int_as_float((127 + ec - ec / 2) << 23) * p.scale_log2;
        }
      }
    }

    float o[NT][S::kMTiles][4];
    float m[NT][2], l[NT][2], big[NT][2];       // running maximum, this lane's share of the sum, largest weight * scale
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int i = 0; i < S::kMTiles; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][i][e] = 0.f;
#pragma unroll
      for (int h = 0; h < 2; ++h) { m[n][h] = -INFINITY; l[n][h] = 0.f; big[n][h] = 0.f; }
    }

    Where<SUB> cur, next;
    locate(t0, cur);
    load_k(cur);
    load_scales(cur, ks, vs);
    for (int tile = t0; tile < t1; ++tile) {
      if (tile * S::kTile + warp * SUB * 16 >= len) break;           // the last tile: no rows for this warp
      if (tile + 1 < t1) {
        locate(tile + 1, next);
      } else {
#pragma unroll
        for (int u = 0; u < SUB; ++u) { next.here[u] = 0; next.row[u] = next.off[u] = 0; }
      }

      // ---- V rows 2c, 2c+1, 2c+8, 2c+9 of each group
      uint32_t v[SUB][4][S::kVWords];
#pragma unroll
      for (int u = 0; u < SUB; ++u)
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          const int i = 2 * c + (h & 1) + 8 * (h >> 1);
          const char* row = p.c.page[1] + cur.off[u] + i * S::kRowBytes + r * S::kVBytes;
#pragma unroll
          for (int w = 0; w < S::kVWords; ++w) v[u][h][w] = 0;
          if (i < cur.here[u]) {
#pragma unroll
            for (int j = 0; j < S::kVPieces; ++j) {
              if constexpr (S::kVBytes == 16) {
                const uint4 x = __ldg(reinterpret_cast<const uint4*>(row + j * 8 * S::kVBytes));
                v[u][h][4 * j] = x.x; v[u][h][4 * j + 1] = x.y; v[u][h][4 * j + 2] = x.z; v[u][h][4 * j + 3] = x.w;
              } else {
                const uint2 x = __ldg(reinterpret_cast<const uint2*>(row + j * 8 * S::kVBytes));
                v[u][h][2 * j] = x.x; v[u][h][2 * j + 1] = x.y;
              }
            }
          }
        }

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
          const uint32_t a[4] = {k[u][0][j].x, k[u][0][j].y, k[u][0][j].z, k[u][0][j].w};
          const uint32_t b[4] = {k[u][1][j].x, k[u][1][j].y, k[u][1][j].z, k[u][1][j].w};
          if (S::kPlain) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int n = 0; n < NT; ++n)
                mma_bf16(s[n][u], a[2 * i], b[2 * i], a[2 * i + 1], b[2 * i + 1], q[n][j][2 * i], q[n][j][2 * i + 1]);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t flip = FMT == CKV_CACHE_INT8 ? 0x80808080u : 0u;
              const uint32_t x = a[i] ^ flip, y = b[i] ^ flip;
              const uint32_t a0 = codes_to_half2<FMT, false>(x), a2 = codes_to_half2<FMT, true>(x);
              const uint32_t a1 = codes_to_half2<FMT, false>(y), a3 = codes_to_half2<FMT, true>(y);
#pragma unroll
              for (int n = 0; n < NT; ++n)
                mma_f16(s[n][u], a0, a1, a2, a3, q[n][j][(2 * i) % S::kQWords], q[n][j][(2 * i + 1) % S::kQWords]);
            }
          }
        }
      load_k(next);
      float ks_next[SUB][2], vs_next[SUB][2];
      load_scales(next, ks_next, vs_next);

      // ---- weights.  s[n][u][2h + x]: cache row r + 8h of group u, query 8n + 2c + x
      uint32_t w_hi[NT][SUB][2], w_lo[NT][SUB][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              float& z = s[n][u][2 * h + x];
              z = r + 8 * h < cur.here[u] ? (S::kPlain ? z : z * ks[u][h] * scale_a[n][x]) * scale_b[n][x] : -INFINITY;
              top[x] = fmaxf(top[x], z);
            }
        float f[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], 4));
          top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], 8));
          top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], 16));
          top[x] = fmaxf(top[x], m[n][x]);
          const float ref = top[x] == -INFINITY ? 0.f : top[x];      // nothing visible yet: all weights are 0
          f[x] = exp2f(m[n][x] - ref);
          m[n][x] = top[x];
          l[n][x] *= f[x];
#pragma unroll
          for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float& z = s[n][u][2 * h + x];
              z = exp2f(z - ref);
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
          float inv[2];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            float most = 0.f;
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                float& z = s[n][u][2 * h + x];
                z *= vs[u][h];
                most = fmaxf(most, z);
              }
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 4));
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 8));
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 16));
            const float old = big[n][x] * f[x];
            most = fmaxf(most, old);
            big[n][x] = most;
            inv[x] = most > 0.f ? __frcp_rn(most) : 0.f;
            f[x] = old * inv[x];
          }
#pragma unroll
          for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              w_hi[n][u][h] = transpose8(pack_half(s[n][u][2 * h] * inv[0], s[n][u][2 * h + 1] * inv[1]));
        }
#pragma unroll
        for (int i = 0; i < S::kMTiles; ++i) {
          o[n][i][0] *= f[0]; o[n][i][1] *= f[1];
          o[n][i][2] *= f[0]; o[n][i][3] *= f[1];
        }
      }

      // ---- O^T += V^T P^T
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        if (S::kPlain) {
#pragma unroll
          for (int i = 0; i < S::kMTiles; ++i) {
            const int e0 = i, e1 = i + S::kMTiles;
            const uint32_t p0 = e0 & 1 ? 0x7632 : 0x5410, p1 = e1 & 1 ? 0x7632 : 0x5410;
            const uint32_t a0 = __byte_perm(v[u][0][e0 / 2], v[u][1][e0 / 2], p0), a1 = __byte_perm(v[u][0][e1 / 2], v[u][1][e1 / 2], p1);
            const uint32_t a2 = __byte_perm(v[u][2][e0 / 2], v[u][3][e0 / 2], p0), a3 = __byte_perm(v[u][2][e1 / 2], v[u][3][e1 / 2], p1);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              mma_bf16(o[n][i], a0, a1, a2, a3, w_hi[n][u][0], w_hi[n][u][1]);
              mma_bf16(o[n][i], a0, a1, a2, a3, w_lo[n][u][0], w_lo[n][u][1]);
            }
          }
        } else {
          const uint32_t flip = FMT == CKV_CACHE_INT8 ? 0x80808080u : 0u;
#pragma unroll
          for (int i = 0; i < S::kMTiles; i += 2) {       // two tiles: elements i, i+1 and kMTiles further
            uint32_t a[2][4];
#pragma unroll
            for (int g = 0; g < 2; ++g) {                 // g: rows 2c, 2c+1 or 2c+8, 2c+9
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const int at = i + e * S::kMTiles;
                const uint32_t four = __byte_perm(v[u][2 * g][at / 4], v[u][2 * g + 1][at / 4], at & 2 ? 0x7362 : 0x5140) ^ flip;
                a[0][2 * g + e] = codes_to_half2<FMT, false>(four);
                a[1][2 * g + e] = codes_to_half2<FMT, true>(four);
              }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int e = 0; e < 2; ++e)
                mma_f16(o[n][i + e], a[e][0], a[e][1], a[e][2], a[e][3], w_hi[n][u][0], w_hi[n][u][1]);
          }
        }
      }
      cur = next;
#pragma unroll
      for (int u = 0; u < SUB; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) { ks[u][h] = ks_next[u][h]; vs[u][h] = vs_next[u][h]; }
    }

    // ---- the warps meet in shared memory, eight queries at a time
    const bool whole = t0 == 0 && t1 == tiles;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (8 * n < it.rows) {
        __syncthreads();                                   // the buffers of the previous group are free
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          float sum = l[n][x];
          sum += __shfl_xor_sync(0xffffffffu, sum, 4);
          sum += __shfl_xor_sync(0xffffffffu, sum, 8);
          sum += __shfl_xor_sync(0xffffffffu, sum, 16);
          if (r == 0) { m_s[warp][2 * c + x] = m[n][x]; l_s[warp][2 * c + x] = sum; }
          const float unit = S::kPlain ? 1.f : big[n][x];
          float* dst = o_s[warp][2 * c + x];
          // element e of the lane's piece: o[n][e % kMTiles][2 * (e / kMTiles) + x]
#pragma unroll
          for (int e = 0; e < S::kElems; e += 4) {
            const int half = e / S::kMTiles, i = e % S::kMTiles;
            const int at = (S::kVPieces == 2) ? 8 * r + 64 * half + i : S::kElems * r + e;
            *reinterpret_cast<float4*>(dst + at) =
                make_float4(o[n][i][2 * half + x] * unit, o[n][i + 1][2 * half + x] * unit,
                            o[n][i + 2][2 * half + x] * unit, o[n][i + 3][2 * half + x] * unit);
          }
        }
        __syncthreads();
        finish<T, DH, 8>(p, it, &o_s[0][0][0], &m_s[0][0], &l_s[0][0], 8 * n, whole, t0 > 0 ? 0 : 1);
      }
    }
    if (t0 > 0 && t1 == tiles) join = make_int2(item, cta_of(walk, first));
    t = first + t1;
    first += tiles;
  }
  if (threadIdx.x == 0) p.join[blockIdx.x] = join;
}

template <int FMT, int DH, int NT> cudaError_t launch(const DecodeArgs& p, int sm_count, cudaStream_t st) {
  int per_sm = 0;
  cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, decode_mma_kernel<FMT, DH, NT>, kDecodeThreads, 0);
  if (e != cudaSuccess) return e;
  const int grid = decode_grid(p, per_sm * sm_count, Shape<FMT, DH>::kTile);
  decode_mma_kernel<FMT, DH, NT><<<grid, kDecodeThreads, 0, st>>>(p);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;
  return launch_decode_join<__nv_bfloat16, DH>(p, grid, st);
}

template <int FMT> cudaError_t by_shape(const DecodeArgs& p, int dh, int sm_count, cudaStream_t st) {
  if (p.chunk_rows == 8) return dh == 64 ? launch<FMT, 64, 1>(p, sm_count, st) : launch<FMT, 128, 1>(p, sm_count, st);
  return dh == 64 ? launch<FMT, 64, 2>(p, sm_count, st) : launch<FMT, 128, 2>(p, sm_count, st);
}

}  // namespace

cudaError_t launch_decode_mma(const CacheDims& d, const DecodeCall& call, int sm_count, int* status_word, cudaStream_t st,
                              int* launches) {
  // queries of a KV head: 8 or 16 an item; more than 16 read the cache once per 16
  const DecodeArgs p = decode_args(d, call, d.Hq / d.Hkv <= 8 ? 8 : 16, status_word);
  *launches += 2;
  if (d.format == CKV_CACHE_PLAIN) return by_shape<CKV_CACHE_PLAIN>(p, d.dh, sm_count, st);
  if (d.format == CKV_CACHE_E4M3) return by_shape<CKV_CACHE_E4M3>(p, d.dh, sm_count, st);
  return by_shape<CKV_CACHE_INT8>(p, d.dh, sm_count, st);
}

}  // namespace ckv
