// The paged key/value cache: its handle, writing a batch's new tokens into it (with the per-head
// norms, the rotation and the quantisation), and reading sequences back.
//
// Both kernels move every byte once and are bound by memory at many tokens, by one chain of loads
// (sequence, page, row) at few.
#include <cudaTypedefs.h>

#include <new>

#include "qtea_kv_internal.h"

namespace qtea {
namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

struct AppendParams {
  KvView kv;
  KvBatchView b;
  const void* q;
  const void* k;
  const void* v;
  long long q_ld, k_ld, v_ld;
  int q_heads, n_positions;
  const float* cos;
  const float* sin;
  const __half* q_norm;
  const __half* k_norm;
  float eps;
  __half* q_out;
};

constexpr int kAppendWarps = 8;

template <int TYPE, int P>
__device__ __forceinline__ void load_pairs(const void* row, int i, float* v) {
  if (P == 2) {
    // element-aligned rows only: two scalar loads that the coalescer joins
    if (TYPE == QTEA_TYPE_F32) {
      const float* p = static_cast<const float*>(row) + i;
      v[0] = p[0], v[1] = p[1];
    } else {
      const __half* p = static_cast<const __half*>(row) + i;
      v[0] = __half2float(p[0]), v[1] = __half2float(p[1]);
    }
  } else {
    v[0] = TYPE == QTEA_TYPE_F32 ? static_cast<const float*>(row)[i]
                                 : __half2float(static_cast<const __half*>(row)[i]);
  }
}

__device__ __forceinline__ float saturate_f16(float x) {  // NaN stays NaN
  return x > 65504.f ? 65504.f : x < -65504.f ? -65504.f : x;
}

// One warp per (token, head): lane l holds P = D/64 elements of each half of the head's row, l * P
// of the first half and the same of the second, the two that a rotation joins. Blocks of 32
// elements are then 32 / P neighbouring lanes of one half.
template <int TYPE, int FMT, int D>
__global__ void __launch_bounds__(kAppendWarps * 32) qtea_kv_append_kernel(const AppendParams p) {
  constexpr int P = D / 64;
  const int lane = threadIdx.x & 31, heads = p.q_heads + 2 * p.kv.heads;
  const long long job = (long long)blockIdx.x * kAppendWarps + (threadIdx.x >> 5);
  const int t = (int)(job / heads), head = (int)(job % heads);
  if (t >= p.b.n_tokens) return;

  // which of the three this head is of, and its row
  const bool is_q = head < p.q_heads, is_k = !is_q && head < p.q_heads + p.kv.heads;
  const int h = is_q ? head : is_k ? head - p.q_heads : head - p.q_heads - p.kv.heads;
  const long long first = is_q ? t * p.q_ld : is_k ? t * p.k_ld : t * p.v_ld;
  const char* row = static_cast<const char*>(is_q ? p.q : is_k ? p.k : p.v) +
                    (first + (long long)h * D) * (TYPE == QTEA_TYPE_F32 ? 4 : 2);
  float a[P], b[P];
  load_pairs<TYPE, P>(row, lane * P, a);
  load_pairs<TYPE, P>(row, D / 2 + lane * P, b);

  const int s = kv_find_sequence(p.b.q_start, p.b.n_seqs, t);
  if (s < 0) return;
  const int q0 = __ldg(p.b.q_start + s), i = t - q0;
  const int n = min(__ldg(p.b.q_start + s + 1), p.b.n_tokens) - q0;
  if (i >= p.b.max_q) return;
  // a batch longer than max_q counts its first max_q tokens, at the positions the lengths give
  const int pos = kv_context(p.b, p.kv, s) - n + i;

  const __half* weight = is_q ? p.q_norm : is_k ? p.k_norm : nullptr;
  if (weight) {
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < P; ++e) ss = fmaf(a[e], a[e], fmaf(b[e], b[e], ss));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    const float f = rsqrtf(ss * (1.f / D) + p.eps);
#pragma unroll
    for (int e = 0; e < P; ++e) {
      a[e] = a[e] * f * __half2float(weight[lane * P + e]);
      b[e] = b[e] * f * __half2float(weight[D / 2 + lane * P + e]);
    }
  }
  if (p.cos && (is_q || is_k)) {
    const long long at = (long long)min(max(pos, 0), p.n_positions - 1) * (D / 2) + lane * P;
#pragma unroll
    for (int e = 0; e < P; ++e) {
      const float c = __ldg(p.cos + at + e), d = __ldg(p.sin + at + e);
      const float x = __fsub_rn(__fmul_rn(a[e], c), __fmul_rn(b[e], d));
      b[e] = __fadd_rn(__fmul_rn(b[e], c), __fmul_rn(a[e], d));
      a[e] = x;
    }
  }
  if (is_q) {
    __half* o = p.q_out + ((long long)t * p.q_heads + h) * D;
    if (P == 2) {
      reinterpret_cast<__half2*>(o)[lane] = __floats2half2_rn(a[0], a[P - 1]);
      reinterpret_cast<__half2*>(o)[32 + lane] = __floats2half2_rn(b[0], b[P - 1]);
    } else {
      o[lane] = __float2half_rn(a[0]);
      o[32 + lane] = __float2half_rn(b[0]);
    }
    return;
  }
  if (pos < 0) return;
  const int page = __ldg(p.b.pages + (long long)s * p.b.max_pages + (pos >> p.kv.page_shift));
  if ((unsigned)page >= (unsigned)p.kv.n_pages) return;
  const long long slot = ((long long)page * p.kv.heads + h) * p.kv.page_size + (pos & (p.kv.page_size - 1));
  uint8_t* dst = (is_k ? p.kv.k : p.kv.v) + slot * kv_row_bytes(FMT, D);
  if (FMT == QTEA_KV_F16) {
    __half* o = reinterpret_cast<__half*>(dst);
    if (P == 2) {
      reinterpret_cast<__half2*>(o)[lane] = __floats2half2_rn(saturate_f16(a[0]), saturate_f16(a[P - 1]));
      reinterpret_cast<__half2*>(o)[32 + lane] = __floats2half2_rn(saturate_f16(b[0]), saturate_f16(b[P - 1]));
    } else {
      o[lane] = __float2half_rn(saturate_f16(a[0]));
      o[32 + lane] = __float2half_rn(saturate_f16(b[0]));
    }
    return;
  }
  // the largest magnitude of each block (maxima skip NaN), then its power of two
  float ta = fabsf(a[0]), tb = fabsf(b[0]);
  if (P == 2) ta = fmaxf(ta, fabsf(a[P - 1])), tb = fmaxf(tb, fabsf(b[P - 1]));
#pragma unroll
  for (int o = 16 / P; o > 0; o >>= 1) {
    ta = fmaxf(ta, __shfl_xor_sync(0xffffffffu, ta, o));
    tb = fmaxf(tb, __shfl_xor_sync(0xffffffffu, tb, o));
  }
  if (P == 1) {  // D = 64: a block is a whole half
    ta = fmaxf(ta, __shfl_xor_sync(0xffffffffu, ta, 16));
    tb = fmaxf(tb, __shfl_xor_sync(0xffffffffu, tb, 16));
  }
  constexpr int F = FMT == QTEA_KV_F16 ? QTEA_KV_FP8 : FMT;
  const int ea = kv_exponent<F>(ta), eb = kv_exponent<F>(tb);
  const float fa = exp2i(-ea), fb = exp2i(-eb);
  uint8_t* scales = (is_k ? p.kv.ks : p.kv.vs) + slot * (D / kKvBlock);
  if (P == 2) {
    if ((lane & 15) == 0) {
      scales[lane >> 4] = (uint8_t)(ea + 127);
      scales[2 + (lane >> 4)] = (uint8_t)(eb + 127);
    }
  } else if (lane == 0) {
    scales[0] = (uint8_t)(ea + 127);
    scales[1] = (uint8_t)(eb + 127);
  }
#pragma unroll
  for (int e = 0; e < P; ++e) a[e] *= fa, b[e] *= fb;
  if (FMT == QTEA_KV_FP8) {
    if (P == 2) {
      reinterpret_cast<uint16_t*>(dst)[lane] = (uint16_t)to_e4m3x2(a[0], a[P - 1]);
      reinterpret_cast<uint16_t*>(dst)[32 + lane] = (uint16_t)to_e4m3x2(b[0], b[P - 1]);
    } else {
      const uint32_t c = to_e4m3x2(a[0], b[0]);
      dst[lane] = (uint8_t)c;
      dst[32 + lane] = (uint8_t)(c >> 8);
    }
  } else {
    if (P == 2) {
      dst[lane] = (uint8_t)to_e2m1x2(a[0], a[P - 1]);
      dst[32 + lane] = (uint8_t)to_e2m1x2(b[0], b[P - 1]);
    } else {  // a lane holds one element of each half: even lanes write their byte and the next lane's
      const float an = __shfl_down_sync(0xffffffffu, a[0], 1), bn = __shfl_down_sync(0xffffffffu, b[0], 1);
      if ((lane & 1) == 0) {
        dst[lane >> 1] = (uint8_t)to_e2m1x2(a[0], an);
        dst[16 + (lane >> 1)] = (uint8_t)to_e2m1x2(b[0], bn);
      }
    }
  }
}

// ------------------------------------------------------------------------------------ reading back

struct ReadParams {
  KvView kv;
  KvBatchView b;
  const int32_t* row_start;
  int n_rows;
  uint4* k_out;
  uint4* v_out;
};

constexpr int kReadThreads = 256;
constexpr int kReadRows = 16;  // output rows of a CTA

// A CTA takes kReadRows consecutive output rows: its first threads find each row's place in the
// cache, then every thread converts 16 elements at a time, so that a warp's stores are one run of
// memory. 16 elements are 32, 16 or 8 bytes of codes, one load each.
template <int FMT, int D>
__global__ void __launch_bounds__(kReadThreads) qtea_kv_read_kernel(const ReadParams p) {
  __shared__ long long where[kReadRows];  // slot of head 0, -1: zeros, -2: no sequence's row
  const int r0 = blockIdx.x * kReadRows;
  if (threadIdx.x < kReadRows) {
    const int r = r0 + threadIdx.x;
    long long at = -2;
    if (r < p.n_rows && r >= __ldg(p.row_start) && r < __ldg(p.row_start + p.b.n_seqs)) {
      int lo = 0, hi = p.b.n_seqs;  // the last sequence that starts at or before r, and is not empty
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (__ldg(p.row_start + mid) <= r) lo = mid;
        else hi = mid;
      }
      const int pos = r - __ldg(p.row_start + lo);
      at = -1;
      if (pos < kv_context(p.b, p.kv, lo)) {
        const int page = __ldg(p.b.pages + (long long)lo * p.b.max_pages + (pos >> p.kv.page_shift));
        if ((unsigned)page < (unsigned)p.kv.n_pages)
          at = (long long)page * p.kv.heads * p.kv.page_size + (pos & (p.kv.page_size - 1));
      }
    }
    where[threadIdx.x] = at;
  }
  __syncthreads();
  constexpr int kChunks = D / 16;  // of 16 elements
  const int per_row = p.kv.heads * kChunks;
  constexpr int kBytes = FMT == QTEA_KV_F16 ? 32 : FMT == QTEA_KV_FP8 ? 16 : 8;
  const int all = kReadRows * per_row;
#pragma unroll 2
  for (int u = threadIdx.x; u < all; u += kReadThreads) {
    const int r = u / per_row, w = u - r * per_row, head = w / kChunks, c = w - head * kChunks;
    const long long base = where[r];
    if (base == -2) continue;
    const long long slot = base + (long long)head * p.kv.page_size;
    const long long to = ((long long)(r0 + r) * per_row + w) * 2;
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      uint4* out = side == 0 ? p.k_out : p.v_out;
      if (!out) continue;
      uint32_t o[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (base >= 0) {
        const uint8_t* src = (side == 0 ? p.kv.k : p.kv.v) + slot * kv_row_bytes(FMT, D) + c * kBytes;
        if (FMT == QTEA_KV_F16) {
          const uint4 x = __ldcs(reinterpret_cast<const uint4*>(src)), y = __ldcs(reinterpret_cast<const uint4*>(src) + 1);
          o[0] = x.x, o[1] = x.y, o[2] = x.z, o[3] = x.w, o[4] = y.x, o[5] = y.y, o[6] = y.z, o[7] = y.w;
        } else {
          const uint32_t f = scale_bits(__ldg((side == 0 ? p.kv.ks : p.kv.vs) + slot * (D / kKvBlock) + c / 2)) * 0x10001u;
          if (FMT == QTEA_KV_FP8) {
            const uint4 x = __ldcs(reinterpret_cast<const uint4*>(src));
            const uint32_t v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              o[2 * i] = hmul2(from_e4m3x2(v[i]), f);
              o[2 * i + 1] = hmul2(from_e4m3x2_hi(v[i]), f);
            }
          } else {
            const uint2 x = __ldcs(reinterpret_cast<const uint2*>(src));
            from_e2m1x8(x.x, o);
            from_e2m1x8(x.y, o + 4);
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = hmul2(o[i], f);
          }
        }
      }
      __stcs(out + to, make_uint4(o[0], o[1], o[2], o[3]));
      __stcs(out + to + 1, make_uint4(o[4], o[5], o[6], o[7]));
    }
  }
}

template <int TYPE, int FMT>
void launch_append(const AppendParams& p, int grid, cudaStream_t st) {
  if (p.kv.dim == 128) qtea_kv_append_kernel<TYPE, FMT, 128><<<grid, kAppendWarps * 32, 0, st>>>(p);
  else qtea_kv_append_kernel<TYPE, FMT, 64><<<grid, kAppendWarps * 32, 0, st>>>(p);
}

template <int FMT>
void launch_read(const ReadParams& p, int grid, cudaStream_t st) {
  if (p.kv.dim == 128) qtea_kv_read_kernel<FMT, 128><<<grid, kReadThreads, 0, st>>>(p);
  else qtea_kv_read_kernel<FMT, 64><<<grid, kReadThreads, 0, st>>>(p);
}

}  // namespace

// The batch's host-side checks; `queries`: the call looks at q_start, n_tokens and max_q_len.
int check_batch(const qtea_kv* kv, const qtea_kv_batch* b, bool queries, KvBatchView* out) {
  if (!kv || !b || b->n_seqs < 0 || b->n_seqs > kKvMaxSeqs || b->max_pages < 1) return QTEA_ERR_INVALID_ARG;
  if ((long long)b->max_pages * kv->view.page_size > 0x7fffffffLL) return QTEA_ERR_INVALID_ARG;
  if (b->n_seqs > 0 && (!b->ctx_len || !b->pages || !aligned(b->ctx_len, 4) || !aligned(b->pages, 4)))
    return QTEA_ERR_INVALID_ARG;
  if (queries && (b->n_tokens < 0 || b->max_q_len < 1 ||
                  (b->n_seqs > 0 && (!b->q_start || !aligned(b->q_start, 4)))))
    return QTEA_ERR_INVALID_ARG;
  *out = KvBatchView{b->q_start, b->ctx_len, b->pages, b->n_seqs, b->max_pages, b->n_tokens, b->max_q_len};
  return QTEA_OK;
}

}  // namespace qtea

using namespace qtea;

extern "C" {

int qtea_kv_create(void* k_pages, void* v_pages, void* k_scales, void* v_scales, int n_pages, int page_size,
                   int n_kv_heads, int head_dim, int format, qtea_kv** out) {
  if (!out) return QTEA_ERR_INVALID_ARG;
  *out = nullptr;
  if (!k_pages || !v_pages || !aligned(k_pages, 16) || !aligned(v_pages, 16)) return QTEA_ERR_INVALID_ARG;
  if (format != QTEA_KV_F16 && format != QTEA_KV_FP8 && format != QTEA_KV_FP4) return QTEA_ERR_INVALID_ARG;
  if (format != QTEA_KV_F16 && (!k_scales || !v_scales || !aligned(k_scales, 16) || !aligned(v_scales, 16)))
    return QTEA_ERR_INVALID_ARG;
  if (n_pages < 1 || n_kv_heads < 1 || n_kv_heads > 1024 || page_size < 1 || head_dim < 1) return QTEA_ERR_INVALID_ARG;
  int shift = 0;
  while (shift < 9 && (1 << shift) != page_size) ++shift;
  if (shift < 4 || shift > 8 || (head_dim != 64 && head_dim != 128)) return QTEA_ERR_UNSUPPORTED;
  if ((long long)n_pages * n_kv_heads * page_size > 0x7fffffffLL) return QTEA_ERR_INVALID_ARG;

  int dev = 0, sms = 0;
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult found;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
      cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess ||
      found != cudaDriverEntryPointSuccess) {
    cudaGetLastError();
    return QTEA_ERR_CUDA;
  }
  qtea_kv* kv = new (std::nothrow) qtea_kv();
  if (!kv) return QTEA_ERR_ALLOC;
  kv->view = KvView{static_cast<uint8_t*>(k_pages), static_cast<uint8_t*>(v_pages), static_cast<uint8_t*>(k_scales),
                    static_cast<uint8_t*>(v_scales), n_pages, page_size, n_kv_heads, head_dim, format, shift};
  kv->device = dev;
  kv->sm_count = sms;
  kv->encode = fn;
  // A box's row is swizzled over its whole length: reading 8 rows at one place of the row, as the
  // fragment loads do, touches every bank once. A box lies within a page; the larger the box, the
  // fewer copies: boxes of 16 tokens throughout held the fp4 kernel to one copy per 18 ns.
  const int row = kv_row_bytes(format, head_dim), wide = row < 128 ? row : 128;
  cuuint64_t dims[2] = {(cuuint64_t)row, (cuuint64_t)n_pages * n_kv_heads * page_size};
  cuuint64_t strides[1] = {(cuuint64_t)row};
  cuuint32_t step[2] = {1, 1};
  const CUtensorMapSwizzle swizzle = wide == 128  ? CU_TENSOR_MAP_SWIZZLE_128B
                                     : wide == 64 ? CU_TENSOR_MAP_SWIZZLE_64B
                                                  : CU_TENSOR_MAP_SWIZZLE_32B;
  auto encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
  auto make = [&](CUtensorMap* map, void* pages, int most) {
    cuuint32_t box[2] = {(cuuint32_t)wide, (cuuint32_t)(page_size < most ? page_size : most)};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, pages, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  };
  const int unit = 1 << kv_unit_shift(format);
  bool made = make(&kv->map_k, k_pages, unit) && make(&kv->map_v, v_pages, unit);
  if (format == QTEA_KV_F16) made = made && make(&kv->wide_k, k_pages, 128) && make(&kv->wide_v, v_pages, 128);
  if (!made) {
    delete kv;
    return QTEA_ERR_CUDA;
  }
  *out = kv;
  return QTEA_OK;
}

void qtea_kv_free(qtea_kv* kv) { delete kv; }

int qtea_kv_append(const qtea_kv* kv, const qtea_kv_batch* batch, const qtea_kv_append_args* a, qtea_stream_t stream) {
  if (!kv || !a) return QTEA_ERR_INVALID_ARG;
  AppendParams p;
  int rc = check_batch(kv, batch, true, &p.b);
  if (rc) return rc;
  const int size = a->type == QTEA_TYPE_F32 ? 4 : 2;
  if (a->type != QTEA_TYPE_F32 && a->type != QTEA_TYPE_F16) return QTEA_ERR_INVALID_ARG;
  if (p.b.n_seqs == 0 || p.b.n_tokens == 0) return QTEA_OK;
  const long long kv_row = (long long)kv->view.heads * kv->view.dim;
  if (!a->k || !a->v || a->k_ld < kv_row || a->v_ld < kv_row || !aligned(a->k, size) || !aligned(a->v, size))
    return QTEA_ERR_INVALID_ARG;
  if (a->q && (a->n_q_heads < 1 || a->n_q_heads > (1 << 16) || a->q_ld < (long long)a->n_q_heads * kv->view.dim ||
               !a->q_out || !aligned(a->q, size) || !aligned(a->q_out, 4)))
    return QTEA_ERR_INVALID_ARG;
  if ((a->cos == nullptr) != (a->sin == nullptr) ||
      (a->cos && (a->n_positions < 1 || !aligned(a->cos, 4) || !aligned(a->sin, 4))))
    return QTEA_ERR_INVALID_ARG;
  if (!aligned(a->q_norm, 2) || !aligned(a->k_norm, 2)) return QTEA_ERR_INVALID_ARG;
  p.kv = kv->view;
  p.q = a->q, p.k = a->k, p.v = a->v;
  p.q_ld = a->q_ld, p.k_ld = a->k_ld, p.v_ld = a->v_ld;
  p.q_heads = a->q ? a->n_q_heads : 0;
  p.n_positions = a->n_positions;
  p.cos = a->cos, p.sin = a->sin;
  p.q_norm = reinterpret_cast<const __half*>(a->q_norm);
  p.k_norm = reinterpret_cast<const __half*>(a->k_norm);
  p.eps = a->eps;
  p.q_out = reinterpret_cast<__half*>(a->q_out);
  const long long jobs = (long long)p.b.n_tokens * (p.q_heads + 2 * p.kv.heads);
  const long long grid = (jobs + kAppendWarps - 1) / kAppendWarps;
  if (grid > 0x7fffffffLL) return QTEA_ERR_INVALID_ARG;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const bool f32 = a->type == QTEA_TYPE_F32;
  if (p.kv.format == QTEA_KV_F16) {
    if (f32) launch_append<QTEA_TYPE_F32, QTEA_KV_F16>(p, (int)grid, st);
    else launch_append<QTEA_TYPE_F16, QTEA_KV_F16>(p, (int)grid, st);
  } else if (p.kv.format == QTEA_KV_FP8) {
    if (f32) launch_append<QTEA_TYPE_F32, QTEA_KV_FP8>(p, (int)grid, st);
    else launch_append<QTEA_TYPE_F16, QTEA_KV_FP8>(p, (int)grid, st);
  } else {
    if (f32) launch_append<QTEA_TYPE_F32, QTEA_KV_FP4>(p, (int)grid, st);
    else launch_append<QTEA_TYPE_F16, QTEA_KV_FP4>(p, (int)grid, st);
  }
  return cudaGetLastError() == cudaSuccess ? QTEA_OK : QTEA_ERR_CUDA;
}

int qtea_kv_read(const qtea_kv* kv, const qtea_kv_batch* batch, const int32_t* row_start, int n_rows, uint16_t* k_out,
                 uint16_t* v_out, qtea_stream_t stream) {
  ReadParams p;
  int rc = check_batch(kv, batch, false, &p.b);
  if (rc) return rc;
  if (n_rows < 0 || !aligned(k_out, 16) || !aligned(v_out, 16)) return QTEA_ERR_INVALID_ARG;
  if (p.b.n_seqs == 0 || n_rows == 0 || (!k_out && !v_out)) return QTEA_OK;
  if (!row_start || !aligned(row_start, 4)) return QTEA_ERR_INVALID_ARG;
  p.kv = kv->view;
  p.row_start = row_start;
  p.n_rows = n_rows;
  p.k_out = reinterpret_cast<uint4*>(k_out);
  p.v_out = reinterpret_cast<uint4*>(v_out);
  const int grid = (int)(((long long)n_rows + kReadRows - 1) / kReadRows);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (p.kv.format == QTEA_KV_F16) launch_read<QTEA_KV_F16>(p, grid, st);
  else if (p.kv.format == QTEA_KV_FP8) launch_read<QTEA_KV_FP8>(p, grid, st);
  else launch_read<QTEA_KV_FP4>(p, grid, st);
  return cudaGetLastError() == cudaSuccess ? QTEA_OK : QTEA_ERR_CUDA;
}

}  // extern "C"
