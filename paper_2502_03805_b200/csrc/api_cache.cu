// C ABI of rotary positions, the paged cache and decode attention: argument validation and dispatch.
// All checks run on the host before the first launch; nothing here synchronises or allocates.
#include <math.h>

#include "handle.h"

namespace {

using ckv::CacheDims;
using ckv::DeviceGuard;
using ckv::aligned16;
using ckv::record_cuda;
using ckv::stored_bytes;

inline bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Whether two arrays of int32 share memory.
inline bool overlap(const int32_t* a, long long na, const int32_t* b, long long nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && x < y + 4 * (uintptr_t)nb && y < x + 4 * (uintptr_t)na;
}

int resolve_cache(const criticalkv_cache* c, CacheDims* o) {
  if (!c) return CKV_EINVAL;
  if (c->nseq < 0 || c->Hq < 1 || c->Hkv < 1 || c->Hq % c->Hkv != 0) return CKV_EINVAL;
  if (c->Hkv > 64) return CKV_ENOTSUP;
  if (c->Hq > 65536) return CKV_ENOTSUP;
  if (c->dh != 64 && c->dh != 128) return CKV_ENOTSUP;
  if (c->dtype != CKV_F32 && c->dtype != CKV_BF16) return CKV_EINVAL;
  if (c->format < CKV_CACHE_PLAIN || c->format > CKV_CACHE_E2M1) return CKV_EINVAL;
  int shift = 0;
  switch (c->page_size) {
    case 16: shift = 4; break;
    case 32: shift = 5; break;
    case 64: shift = 6; break;
    case 128: shift = 7; break;
    case 256: shift = 8; break;
    default: return CKV_ENOTSUP;
  }
  if (c->num_pages < 1 || c->max_pages < 1) return CKV_EINVAL;
  if (c->flags & ~(uint32_t)(CKV_FLAG_FORCE_SIMT | CKV_FLAG_DEBUG_CHECKS | CKV_FLAG_SELECT_NO_CLUSTER)) return CKV_EINVAL;
  if (c->reserved != 0 || !isfinite(c->scale)) return CKV_EINVAL;
  const long long capacity = (long long)c->max_pages << shift;
  // row numbers are 32-bit, and so is the number of a call's (sequence, query head) pairs
  if (capacity > 0x7fffffffLL - 256 || (long long)c->nseq * c->Hq > 0x7fffffffLL) return CKV_ENOTSUP;
  const long long dense = (long long)c->page_size * c->dh;
  o->page_stride = c->page_stride ? c->page_stride : dense;
  if (o->page_stride < dense) return CKV_EINVAL;
  if (o->page_stride >= (1LL << 38)) return CKV_ENOTSUP;   // a tensor map holds strides below 2^40 bytes
  if (o->page_stride % 2 || stored_bytes(c->format, c->dtype, o->page_stride) % 16) return CKV_EALIGN;
  if (!c->k_pages || !c->v_pages || (c->nseq && !c->page_table)) return CKV_EINVAL;
  if (c->format != CKV_CACHE_PLAIN && (!c->k_scale || !c->v_scale)) return CKV_EINVAL;
  if (!aligned16(c->k_pages) || !aligned16(c->v_pages) || !aligned_to(c->page_table, 4)) return CKV_EALIGN;
  if (c->format != CKV_CACHE_PLAIN && (!aligned16(c->k_scale) || !aligned16(c->v_scale))) return CKV_EALIGN;
  if (c->format == CKV_CACHE_E2M1) {
    if (!c->k_group_scale || !c->v_group_scale) return CKV_EINVAL;
    if (!aligned16(c->k_group_scale) || !aligned16(c->v_group_scale)) return CKV_EALIGN;
    o->k_group = c->k_group_scale; o->v_group = c->v_group_scale;
  } else {
    o->k_group = o->v_group = nullptr;
  }
  o->nseq = c->nseq; o->Hq = c->Hq; o->Hkv = c->Hkv; o->dh = c->dh; o->dtype = c->dtype; o->format = c->format;
  o->page_shift = shift; o->num_pages = c->num_pages; o->max_pages = c->max_pages;
  o->capacity = capacity;
  o->scale = c->scale > 0.f ? (double)c->scale : 1.0 / sqrt((double)c->dh);
  o->debug_checks = (c->flags & CKV_FLAG_DEBUG_CHECKS) ? 1 : 0;
  o->allow_cluster = (c->flags & CKV_FLAG_SELECT_NO_CLUSTER) ? 0 : 1;
  o->k_pages = c->k_pages; o->v_pages = c->v_pages;
  o->k_scale = c->k_scale; o->v_scale = c->v_scale;
  o->page_table = c->page_table;
  return CKV_OK;
}

// Element strides of a [nseq, H, rows, dh] array: the caller's, or the dense default where they are 0.
int resolve_stride(const int64_t* given, long long heads, long long rows, int dh, int dtype, long long* out) {
  const long long dense[3] = {heads * rows * dh, rows * dh, dh};
  const int vec = dtype == CKV_F32 ? 4 : 8;
  for (int i = 0; i < 3; ++i) {
    out[i] = given && given[i] ? given[i] : dense[i];
    if (out[i] < 0) return CKV_EINVAL;
    if (out[i] % vec) return CKV_EALIGN;
  }
  return out[2] < dh ? CKV_EINVAL : CKV_OK;
}

}  // namespace

extern "C" {

int criticalkv_rope(criticalkv_handle h, const criticalkv_rope_desc* d, const void* q, const void* k,
                    const int32_t* pos, const double* freq, void* q_out, void* k_out, void* stream) {
  if (!h || !d) return CKV_EINVAL;
  if (d->nseq < 0 || d->T < 0 || d->Hq < 1 || d->Hk < 0 || d->reserved != 0) return CKV_EINVAL;
  if (d->Hq > 4096 || d->Hk > 4096) return CKV_ENOTSUP;
  if (d->dh < 8 || d->dh % 8) return CKV_EINVAL;
  if (d->dh > 256) return CKV_ENOTSUP;
  if (d->rot < 2 || d->rot % 2 || d->rot > d->dh) return CKV_EINVAL;
  if (d->dtype != CKV_F32 && d->dtype != CKV_BF16) return CKV_EINVAL;
  if (d->layout != CKV_ROPE_HALF && d->layout != CKV_ROPE_INTERLEAVED) return CKV_EINVAL;
  if (!isfinite(d->factor)) return CKV_EINVAL;
  ckv::RopeDims o;
  o.nseq = d->nseq; o.T = d->T; o.Hq = d->Hq; o.Hk = d->Hk; o.dh = d->dh; o.rot = d->rot; o.dtype = d->dtype;
  o.layout = d->layout; o.factor = d->factor;
  int rc;
  if ((rc = resolve_stride(d->q_stride, d->Hq, d->T, d->dh, d->dtype, o.qs)) != CKV_OK ||
      (rc = resolve_stride(d->k_stride, d->Hk, d->T, d->dh, d->dtype, o.ks)) != CKV_OK ||
      (rc = resolve_stride(d->q_out_stride, d->Hq, d->T, d->dh, d->dtype, o.qos)) != CKV_OK ||
      (rc = resolve_stride(d->k_out_stride, d->Hk, d->T, d->dh, d->dtype, o.kos)) != CKV_OK)
    return rc;
  // tokens are numbered in 32 bits, up to a whole tile of them behind the last
  if ((long long)d->nseq * d->T > 0x7fffffffLL - 256) return CKV_ENOTSUP;
  if (d->nseq == 0 || d->T == 0) return CKV_OK;
  if (!q || !q_out || !pos || !freq || (d->Hk && (!k || !k_out))) return CKV_EINVAL;
  if (!aligned16(q) || !aligned16(q_out) || (d->Hk && (!aligned16(k) || !aligned16(k_out))) || !aligned_to(pos, 4) ||
      !aligned_to(freq, 8))
    return CKV_EALIGN;
  DeviceGuard guard(h->device);
  if (!guard.ok) return CKV_ECUDA;
  int launches = 0;
  const cudaError_t e = ckv::launch_rope(o, q, k, pos, freq, q_out, k_out, h->sm_count, (cudaStream_t)stream, &launches);
  h->launches += launches;
  return record_cuda(h, e);
}

int criticalkv_cache_store(criticalkv_handle h, const criticalkv_cache* c, const void* K, const void* V, int32_t n,
                           const int64_t* stride, const int32_t* idx, const int32_t* offsets, int64_t idx_rows,
                           const int32_t* counts, const int32_t* start, int32_t* lens_out, void* stream) {
  if (!h) return CKV_EINVAL;
  CacheDims d;
  int rc = resolve_cache(c, &d);
  if (rc != CKV_OK) return rc;
  if (n < 0 || idx_rows < 0 || (idx && (!offsets || counts)) || (!idx && offsets)) return CKV_EINVAL;
  if (idx_rows > 0x7fffffffLL) return CKV_ENOTSUP;
  long long ss[3];
  if ((rc = resolve_stride(stride, d.Hkv, n, d.dh, d.dtype, ss)) != CKV_OK) return rc;
  if (d.nseq == 0) return CKV_OK;
  if (!start || (n && (!K || !V))) return CKV_EINVAL;
  if (!aligned16(K) || !aligned16(V) || !aligned_to(idx, 4) || !aligned_to(offsets, 4) || !aligned_to(counts, 4) ||
      !aligned_to(start, 4) || !aligned_to(lens_out, 4))
    return CKV_EALIGN;
  // lens_out is start itself or an array apart from everything that the kernel reads while it is written
  const long long heads = (long long)d.nseq * d.Hkv;
  if (lens_out && ((lens_out != start && overlap(lens_out, heads, start, heads)) || overlap(lens_out, heads, counts, d.nseq) ||
                   overlap(lens_out, heads, offsets, heads + d.nseq) || overlap(lens_out, heads, idx, d.nseq * (long long)idx_rows) ||
                   overlap(lens_out, heads, d.page_table, heads * d.max_pages)))
    return CKV_EINVAL;
  DeviceGuard guard(h->device);
  if (!guard.ok) return CKV_ECUDA;
  int launches = 0;
  const cudaError_t e = ckv::launch_cache_store(d, K, V, n, ss, idx, offsets, idx_rows, counts, start, lens_out,
                                                h->sm_count, h->status_word, (cudaStream_t)stream, &launches);
  h->launches += launches;
  return record_cuda(h, e);
}

int criticalkv_cache_append(criticalkv_handle h, const criticalkv_cache* c, const criticalkv_rope_desc* r, const void* q,
                            const void* k, const void* v, const int64_t* v_stride, const int32_t* pos, const double* freq,
                            const int32_t* counts, const int32_t* start, void* q_out, int32_t* lens_out, void* stream) {
  if (!h || !r) return CKV_EINVAL;
  CacheDims d;
  int rc = resolve_cache(c, &d);
  if (rc != CKV_OK) return rc;
  if (r->T < 0 || r->nseq != d.nseq || r->Hq != d.Hq || r->Hk != d.Hkv || r->dh != d.dh || r->dtype != d.dtype || r->reserved != 0)
    return CKV_EINVAL;
  if (r->rot < 2 || r->rot % 2 || r->rot > r->dh) return CKV_EINVAL;
  if (r->layout != CKV_ROPE_HALF && r->layout != CKV_ROPE_INTERLEAVED) return CKV_EINVAL;
  if (!isfinite(r->factor)) return CKV_EINVAL;
  if (r->k_out_stride[0] || r->k_out_stride[1] || r->k_out_stride[2]) return CKV_EINVAL;
  ckv::AppendCall a;
  if ((rc = resolve_stride(r->q_stride, d.Hq, r->T, d.dh, d.dtype, a.qs)) != CKV_OK ||
      (rc = resolve_stride(r->k_stride, d.Hkv, r->T, d.dh, d.dtype, a.ks)) != CKV_OK ||
      (rc = resolve_stride(v_stride, d.Hkv, r->T, d.dh, d.dtype, a.vs)) != CKV_OK ||
      (rc = resolve_stride(r->q_out_stride, d.Hq, r->T, d.dh, d.dtype, a.qos)) != CKV_OK)
    return rc;
  // tokens are numbered in 32 bits, up to a whole tile of them behind the last
  if ((long long)d.nseq * r->T > 0x7fffffffLL - 256) return CKV_ENOTSUP;
  if (d.nseq == 0) return CKV_OK;
  if (!start || (r->T && (!q || !k || !v || !q_out || !pos || !freq))) return CKV_EINVAL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned_to(pos, 4) || !aligned_to(freq, 8) ||
      !aligned_to(counts, 4) || !aligned_to(start, 4) || !aligned_to(lens_out, 4))
    return CKV_EALIGN;
  const long long heads = (long long)d.nseq * d.Hkv;
  if (lens_out && ((lens_out != start && overlap(lens_out, heads, start, heads)) || overlap(lens_out, heads, counts, d.nseq) ||
                   overlap(lens_out, heads, pos, (long long)d.nseq * r->T) ||
                   overlap(lens_out, heads, (const int32_t*)freq, r->rot) ||
                   overlap(lens_out, heads, d.page_table, heads * d.max_pages)))
    return CKV_EINVAL;
  a.q = q; a.k = k; a.v = v; a.T = r->T; a.rot = r->rot; a.layout = r->layout; a.factor = r->factor;
  a.pos = pos; a.freq = freq; a.counts = counts; a.start = start; a.q_out = q_out; a.lens_out = lens_out;
  DeviceGuard guard(h->device);
  if (!guard.ok) return CKV_ECUDA;
  int launches = 0;
  const cudaError_t e = ckv::launch_append(d, a, h->sm_count, h->status_word, (cudaStream_t)stream, &launches);
  h->launches += launches;
  return record_cuda(h, e);
}

int criticalkv_cache_load(criticalkv_handle h, const criticalkv_cache* c, const int32_t* lens, int32_t n,
                          const int64_t* stride, int32_t align_right, void* K_out, void* V_out, void* stream) {
  if (!h) return CKV_EINVAL;
  CacheDims d;
  int rc = resolve_cache(c, &d);
  if (rc != CKV_OK) return rc;
  const int clear = align_right & CKV_LOAD_CLEAR;
  align_right &= ~CKV_LOAD_CLEAR;
  if (n < 0 || (align_right != 0 && align_right != 1)) return CKV_EINVAL;
  long long ds[3];
  if ((rc = resolve_stride(stride, d.Hkv, n, d.dh, d.dtype, ds)) != CKV_OK) return rc;
  if (d.nseq == 0 || n == 0) return CKV_OK;
  if (!lens || !K_out || !V_out) return CKV_EINVAL;
  if (!aligned16(K_out) || !aligned16(V_out) || !aligned_to(lens, 4)) return CKV_EALIGN;
  DeviceGuard guard(h->device);
  if (!guard.ok) return CKV_ECUDA;
  int launches = 0;
  const cudaError_t e = ckv::launch_cache_load(d, lens, n, ds, align_right, clear, K_out, V_out, h->status_word,
                                               (cudaStream_t)stream, &launches);
  h->launches += launches;
  return record_cuda(h, e);
}

int criticalkv_summarise_pages(criticalkv_handle h, const criticalkv_cache* c, const int32_t* start, const int32_t* lens,
                               int8_t* codes, float* scales, void* stream) {
  if (!h) return CKV_EINVAL;
  CacheDims d;
  const int rc = resolve_cache(c, &d);
  if (rc != CKV_OK) return rc;
  if (d.nseq == 0) return CKV_OK;
  if (!lens || !codes || !scales) return CKV_EINVAL;
  if (!aligned16(codes) || !aligned_to(scales, 4) || !aligned_to(lens, 4) || !aligned_to(start, 4)) return CKV_EALIGN;
  DeviceGuard guard(h->device);
  if (!guard.ok) return CKV_ECUDA;
  int launches = 0;
  const cudaError_t e = ckv::launch_summarise(d, start, lens, codes, scales, h->sm_count, h->status_word, (cudaStream_t)stream, &launches);
  h->launches += launches;
  return record_cuda(h, e);
}

int criticalkv_select_pages(criticalkv_handle h, const criticalkv_cache* c, const void* q, const int64_t* q_stride,
                            const int32_t* lens, const int8_t* codes, const float* scales, int32_t count, int32_t first,
                            int32_t last, int32_t* table_out, int32_t* lens_out, int32_t* chosen, void* stream) {
  if (!h) return CKV_EINVAL;
  CacheDims d;
  const int rc = resolve_cache(c, &d);
  if (rc != CKV_OK) return rc;
  if (count < 1 || first < 0 || last < 0 || first > count || last > count - first) return CKV_EINVAL;
  ckv::SelectPagesCall a;
  const int vec = d.dtype == CKV_F32 ? 4 : 8;
  const long long dense[2] = {(long long)d.Hq * d.dh, d.dh};
  for (int i = 0; i < 2; ++i) {
    a.q_stride[i] = q_stride && q_stride[i] ? q_stride[i] : dense[i];
    if (a.q_stride[i] < 0) return CKV_EINVAL;
    if (a.q_stride[i] % vec) return CKV_EALIGN;
  }
  const long long heads = (long long)d.nseq * d.Hkv;
  if (d.Hq / d.Hkv > ckv::kSelectMostGroup || d.max_pages > ckv::kSelectMostPages || heads > (1LL << 26)) return CKV_ENOTSUP;
  // rows are numbered in 32 bits in the chosen table too
  if ((long long)count << d.page_shift > 0x7fffffffLL - 256) return CKV_ENOTSUP;
  if (d.nseq == 0) return CKV_OK;
  if (!q || !lens || !codes || !scales || !table_out || !lens_out) return CKV_EINVAL;
  if (!aligned16(q) || !aligned16(codes) || !aligned_to(scales, 4) || !aligned_to(lens, 4) || !aligned_to(table_out, 4) ||
      !aligned_to(lens_out, 4) || !aligned_to(chosen, 4))
    return CKV_EALIGN;
  // the outputs lie apart from what is read and from each other
  const long long in = heads * d.max_pages, out = heads * count;
  if (overlap(table_out, out, d.page_table, in) || overlap(table_out, out, lens, heads) || overlap(lens_out, heads, lens, heads) ||
      overlap(lens_out, heads, d.page_table, in) || overlap(table_out, out, lens_out, heads) || overlap(chosen, out, d.page_table, in) ||
      overlap(chosen, out, lens, heads) || overlap(chosen, out, lens_out, heads) || overlap(chosen, out, table_out, out))
    return CKV_EINVAL;
  a.q = q; a.lens = lens; a.codes = codes; a.scales = scales; a.count = count; a.first = first; a.last = last;
  a.table_out = table_out; a.lens_out = lens_out; a.chosen = chosen;
  DeviceGuard guard(h->device);
  if (!guard.ok) return CKV_ECUDA;
  int launches = 0;
  const cudaError_t e = ckv::launch_select_pages(d, a, h->sm_count, h->status_word, (cudaStream_t)stream, &launches);
  h->launches += launches;
  return record_cuda(h, e);
}

int criticalkv_decode_workspace_bytes(const criticalkv_cache* c, size_t* bytes) {
  if (!bytes) return CKV_EINVAL;
  CacheDims d;
  const int rc = resolve_cache(c, &d);
  if (rc != CKV_OK) return rc;
  *bytes = ckv::decode_workspace_bytes(d);
  return CKV_OK;
}

int criticalkv_decode(criticalkv_handle h, const criticalkv_cache* c, const void* q, const int64_t* q_stride,
                      const int32_t* lens, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  if (!h) return CKV_EINVAL;
  CacheDims d;
  int rc = resolve_cache(c, &d);
  if (rc != CKV_OK) return rc;
  ckv::DecodeCall call;
  const int vec = d.dtype == CKV_F32 ? 4 : 8;
  const long long dense[2] = {(long long)d.Hq * d.dh, d.dh};
  for (int i = 0; i < 2; ++i) {
    call.q_stride[i] = q_stride && q_stride[i] ? q_stride[i] : dense[i];
    if (call.q_stride[i] < 0) return CKV_EINVAL;
    if (call.q_stride[i] % vec) return CKV_EALIGN;
  }
  // the list of 64-row tiles of all heads is counted in 32 bits, and so are the heads a thread further and sixteen times them
  const long long items = (long long)d.nseq * d.Hkv * ((d.Hq / d.Hkv + 7) / 8);
  if (items > 0x7fffffffLL / ((d.capacity + 63) / 64) || items > (1LL << 26)) return CKV_ENOTSUP;
  if (d.nseq == 0) return CKV_OK;
  if (!q || !lens || !out || !ws) return CKV_EINVAL;
  if (!aligned16(q) || !aligned16(out) || !aligned_to(lens, 4) || !aligned_to(lse, 4) || !aligned_to(ws, 256))
    return CKV_EALIGN;
  if (ws_bytes < ckv::decode_workspace_bytes(d)) return CKV_EWORKSPACE;
  call.q = q; call.lens = lens; call.out = out; call.lse = lse; call.ws = ws;
  DeviceGuard guard(h->device);
  if (!guard.ok) return CKV_ECUDA;
  int launches = 0;
  // tensor cores would round float32 queries (on 4-bit pages they enter as two halves); CKV_FLAG_FORCE_SIMT asks for the
  // CUDA-core kernel
  const bool four = d.format == CKV_CACHE_E2M1, mma = (d.dtype == CKV_BF16 || four) && !(c->flags & CKV_FLAG_FORCE_SIMT);
  const cudaError_t e = (!mma ? ckv::launch_decode_simt : four ? ckv::launch_decode_four : ckv::launch_decode_mma)(d, call, h->device, h->sm_count, h->status_word,
                                                                                 (cudaStream_t)stream, &launches);
  h->last_decode = mma ? 1 : 2;
  h->launches += launches;
  return record_cuda(h, e);
}

}  // extern "C"
