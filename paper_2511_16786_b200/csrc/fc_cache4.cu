// Rows of a cache into 4 bits and back (layout: fc_cache4.cuh).
//
// Per half row: min and max, scale = (max - min) / 15 rounded up to the cache's type, so that 15 steps reach the maximum and
// no value is more than half a step off; code = (x - min) / scale to the nearest whole number, the even one of two equally
// near.  Both are decided exactly, whatever the rounding of the arithmetic on the way: the scale by comparing 15 times a
// candidate with the range, the code by the sign of what is left over beside a tie, in 64 bits where it is close.
// Every row is read once and written once: bound by HBM.  A lane holds 8 consecutive channels (16 bytes), 16 or 8 lanes a
// row of K and the same row of V; the nibbles change lanes in registers, and every lane writes one aligned word of codes.
#include "fc_cache4.cuh"

namespace {

constexpr int kQThreads = 256;

template <typename T> struct Num;
template <> struct Num<__half> {
  using T2 = __half2;
  static __device__ float to(__half x) { return __half2float(x); }
  static __device__ __half from(float x) { return __float2half_rn(x); }
  static __device__ __half up(float x) { return __float2half_ru(x); }
  static __device__ __half bits(unsigned short b) { return __ushort_as_half(b); }
  static __device__ unsigned short bits(__half x) { return __half_as_ushort(x); }
  static __device__ float2 both(unsigned w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }
  static __device__ unsigned pack(float a, float b) { const __half2 v = __floats2half2_rn(a, b); return *reinterpret_cast<const unsigned *>(&v); }
  static constexpr unsigned kNan = 0x7e00u;
};
template <> struct Num<__nv_bfloat16> {
  using T2 = __nv_bfloat162;
  static __device__ float to(__nv_bfloat16 x) { return __bfloat162float(x); }
  static __device__ __nv_bfloat16 from(float x) { return __float2bfloat16_rn(x); }
  static __device__ __nv_bfloat16 up(float x) { return __float2bfloat16_ru(x); }
  static __device__ __nv_bfloat16 bits(unsigned short b) { return __ushort_as_bfloat16(b); }
  static __device__ unsigned short bits(__nv_bfloat16 x) { return __bfloat16_as_ushort(x); }
  static __device__ float2 both(unsigned w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
  static __device__ unsigned pack(float a, float b) { const __nv_bfloat162 v = __floats2bfloat162_rn(a, b); return *reinterpret_cast<const unsigned *>(&v); }
  static constexpr unsigned kNan = 0x7fc0u;
};

struct CacheParams {
  const char *k, *v;              // rows (quantising); bytes between tokens and heads
  long long token, head;
  char *out_k, *out_v;            // rows (the values back), dense [row][head][d]
  unsigned char *ck, *cv;
  char *pk, *pv;
  long long cap, rows;
  const long long *used, *out_rows;
  int *status;
  int H;
};

// The smallest number of the type whose 15-fold reaches hi - lo: a first guess in 32 bits, moved by what 15 times it lacks.
template <typename T>
__device__ __forceinline__ float scale_up(float lo, float hi) {
  const float d = hi - lo;
  if (!(d > 0.f)) return 0.f;
  const float z = d - hi;                            // two-sum: hi - lo = d + e
  const float e = (hi - (d - z)) + (-lo - z);
  auto lacks = [&](float s) { return fmaf(15.f, s, -d) - e; };       // >= 0: enough (15 s and d are multiples of ulp(d) > |e|)
  T s = Num<T>::up(d * (1.f / 15.f));
  if (lacks(Num<T>::to(s)) < 0.f) s = Num<T>::bits((unsigned short)(Num<T>::bits(s) + 1));
  const T below = Num<T>::bits((unsigned short)(Num<T>::bits(s) - (Num<T>::bits(s) ? 1 : 0)));
  if (lacks(Num<T>::to(below)) >= 0.f) s = below;
  return Num<T>::to(s);
}

// Nearest whole number of steps, ties to even.
__device__ __forceinline__ unsigned code_of(float x, float lo, float s, float up, float inv) {
  const float dx = (x - lo) * up, su = s * up;
  const float m = fmaf(dx, inv, 12582912.f);         // 1.5 * 2^23: the sum's last bits are the whole number
  float k = m - 12582912.f;
  const float r = fmaf(-k, su, dx);
  if (fabsf(r) >= 0.49999f * su) {                  // beside a tie, or past it: decided by the exact remainder
    const double left = (double)x - (double)lo;
    const double h = floor(left / (double)s);
    const double over = left - (h + 0.5) * (double)s;
    k = (float)h + ((over > 0.0 || (over == 0.0 && ((int)h & 1))) ? 1.f : 0.f);
  }
  return (unsigned)(int)k & 15u;
}

// One matrix's row of one head: LANES lanes with 8 channels each.
template <typename T, int D, bool VALUES>
__device__ __forceinline__ void quantize_row(uint4 raw, int u, unsigned char *codes, char *params, bool write) {
  constexpr int LANES = D / 8, HALF = LANES / 2;
  const unsigned w[4] = {raw.x, raw.y, raw.z, raw.w};
  float x[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) { const float2 f = Num<T>::both(w[i]); x[2 * i] = f.x; x[2 * i + 1] = f.y; }
  float lo = x[0], hi = x[0], odd = 0.f;             // odd: not 0 (NaN) once a value is not finite
#pragma unroll
  for (int i = 0; i < 8; ++i) { lo = fminf(lo, x[i]); hi = fmaxf(hi, x[i]); odd = fmaf(x[i], 0.f, odd); }
#pragma unroll
  for (int o = 1; o < HALF; o <<= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    odd += __shfl_xor_sync(0xffffffffu, odd, o);
  }
  const bool finite = odd == 0.f && hi - lo < INFINITY;
  const float s = finite ? scale_up<T>(lo, hi) : 0.f;
  const float up = s < 1e-35f ? 1099511627776.f : 1.f;                  // 2^40: keeps the reciprocal finite
  const float inv = s > 0.f ? 1.f / (s * up) : 0.f;
  unsigned word = 0;                                 // code i of the lane at nibble i
  if (s > 0.f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) word |= code_of(x[i], lo, s, up, inv) << (4 * i);
  }
  if (VALUES) {
    // nibble i of lane n -> nibble n of lane i, 8 lanes at a time: exchanges of nibbles, bytes, half-words
    unsigned o = __shfl_xor_sync(0xffffffffu, word, 1);
    word = (u & 1) ? ((word & 0xf0f0f0f0u) | ((o >> 4) & 0x0f0f0f0fu)) : ((word & 0x0f0f0f0fu) | ((o << 4) & 0xf0f0f0f0u));
    o = __shfl_xor_sync(0xffffffffu, word, 2);
    word = (u & 2) ? ((word & 0xff00ff00u) | ((o >> 8) & 0x00ff00ffu)) : ((word & 0x00ff00ffu) | ((o << 8) & 0xff00ff00u));
    o = __shfl_xor_sync(0xffffffffu, word, 4);
    word = (u & 4) ? ((word & 0xffff0000u) | (o >> 16)) : ((word & 0x0000ffffu) | (o << 16));
    if (write) *reinterpret_cast<unsigned *>(codes + (u & 7) * (D / 16) + (u >> 3) * 4) = word;
  } else {
    // two quads of one slice, of runs t and t + 1, t = 2 (u & 1); the lane that has the other slice of the words is u ^ 2
    const int odd_slice = (u >> 1) & 1;
    auto spread = [&](unsigned q) {                  // i = 0..3 -> nibbles 0, 4, 1, 5 (odd slices: 2 more)
      const unsigned v = (q & 0xfu) | ((q & 0xf0u) << 12) | ((q & 0xf00u) >> 4) | ((q & 0xf000u) << 8);
      return v << (8 * odd_slice);
    };
    const unsigned q0 = spread(word & 0xffffu), q1 = spread(word >> 16);
    const unsigned got = __shfl_xor_sync(0xffffffffu, odd_slice ? q0 : q1, 2);
    word = (odd_slice ? q1 : q0) | got;
    const int t = 2 * (u & 1) + odd_slice;
    if (write) *reinterpret_cast<unsigned *>(codes + t * (D / 8) + (u >> 2) * 4) = word;
  }
  if (write && (u & (HALF - 1)) == 0) {
    const unsigned ms = Num<T>::bits(Num<T>::from(s)), ml = finite ? (unsigned)Num<T>::bits(Num<T>::from(lo)) : Num<T>::kNan;
    reinterpret_cast<unsigned *>(params)[u / HALF] = ms | (ml << 16);
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(kQThreads)
k_quantize(const CacheParams P) {
  constexpr int LANES = D / 8;
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  long long n = P.rows;
  if (P.used && *P.used < n) n = *P.used < 0 ? 0 : *P.used;
  const int u = threadIdx.x % LANES;
  const long long units = n * P.H, step = (long long)gridDim.x * (kQThreads / LANES);
  // a warp's lanes stay together: the bound is that of its first unit
  for (long long i0 = ((long long)blockIdx.x * kQThreads + (threadIdx.x & ~31)) / LANES; i0 < units; i0 += step) {
    const long long i = i0 + (threadIdx.x & 31) / LANES;
    const bool have = i < units;
    const long long t = have ? i / P.H : 0;
    const int h = have ? (int)(i - t * P.H) : 0;
    const uint4 rk = __ldcs(reinterpret_cast<const uint4 *>(P.k + t * P.token + h * P.head) + u);
    const uint4 rv = __ldcs(reinterpret_cast<const uint4 *>(P.v + t * P.token + h * P.head) + u);
    const long long row = P.out_rows ? P.out_rows[t] : t;
    if (have && row >= P.cap && u == 0) atomicOr(P.status, FC_DEV_FLAG_INTERNAL);
    const bool write = have && row >= 0 && row < P.cap;
    const long long at = (long long)h * P.cap + (write ? row : 0);
    quantize_row<T, D, false>(rk, u, P.ck + at * (D / 2), P.pk + at * cache4::kParamBytes, write);
    quantize_row<T, D, true>(rv, u, P.cv + at * (D / 2), P.pv + at * cache4::kParamBytes, write);
  }
}

template <typename T, int D, bool VALUES>
__device__ __forceinline__ uint4 values_row(const unsigned char *codes, const char *params, int u) {
  constexpr int HALF = D / 16;
  unsigned word;                                     // code i of the lane at nibble i: the steps above backwards
  if (VALUES) {
    word = *reinterpret_cast<const unsigned *>(codes + (u & 7) * (D / 16) + (u >> 3) * 4);
    unsigned o = __shfl_xor_sync(0xffffffffu, word, 4);
    word = (u & 4) ? ((word & 0xffff0000u) | (o >> 16)) : ((word & 0x0000ffffu) | (o << 16));
    o = __shfl_xor_sync(0xffffffffu, word, 2);
    word = (u & 2) ? ((word & 0xff00ff00u) | ((o >> 8) & 0x00ff00ffu)) : ((word & 0x00ff00ffu) | ((o << 8) & 0xff00ff00u));
    o = __shfl_xor_sync(0xffffffffu, word, 1);
    word = (u & 1) ? ((word & 0xf0f0f0f0u) | ((o >> 4) & 0x0f0f0f0fu)) : ((word & 0x0f0f0f0fu) | ((o << 4) & 0xf0f0f0f0u));
  } else {
    const int odd_slice = (u >> 1) & 1, t = 2 * (u & 1) + odd_slice;
    word = *reinterpret_cast<const unsigned *>(codes + t * (D / 8) + (u >> 2) * 4);
    const unsigned mine = (word >> (8 * odd_slice)) & 0x00ff00ffu, theirs = (word >> (8 - 8 * odd_slice)) & 0x00ff00ffu;
    const unsigned got = __shfl_xor_sync(0xffffffffu, theirs, 2);
    auto gather = [](unsigned v) {                   // nibbles 0, 4, 1, 5 -> 0, 1, 2, 3
      return (v & 0xfu) | ((v >> 12) & 0xf0u) | ((v << 4) & 0xf00u) | ((v >> 8) & 0xf000u);
    };
    const unsigned a = gather(mine), b = gather(got);
    word = odd_slice ? (b | (a << 16)) : (a | (b << 16));
  }
  const float2 sl = Num<T>::both(reinterpret_cast<const unsigned *>(params)[u / HALF]);
  unsigned r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    r[i] = Num<T>::pack(fmaf(sl.x, (float)((word >> (8 * i)) & 15u), sl.y), fmaf(sl.x, (float)((word >> (8 * i + 4)) & 15u), sl.y));
  return make_uint4(r[0], r[1], r[2], r[3]);
}

template <typename T, int D>
__global__ void __launch_bounds__(kQThreads)
k_dequantize(const CacheParams P) {
  constexpr int LANES = D / 8;
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  long long n = P.rows;
  if (P.used && *P.used < n) n = *P.used < 0 ? 0 : *P.used;
  const int u = threadIdx.x % LANES;
  const long long units = n * P.H, step = (long long)gridDim.x * (kQThreads / LANES);
  for (long long i0 = ((long long)blockIdx.x * kQThreads + (threadIdx.x & ~31)) / LANES; i0 < units; i0 += step) {
    const long long i = i0 + (threadIdx.x & 31) / LANES;
    const bool have = i < units;
    const long long t = have ? i / P.H : 0;
    const int h = have ? (int)(i - t * P.H) : 0;
    const long long at = (long long)h * P.cap + t;
    const uint4 k = values_row<T, D, false>(P.ck + at * (D / 2), P.pk + at * cache4::kParamBytes, u);
    const uint4 v = values_row<T, D, true>(P.cv + at * (D / 2), P.pv + at * cache4::kParamBytes, u);
    if (have) {
      const size_t o = ((size_t)t * P.H + h) * (D / 8) + u;
      reinterpret_cast<uint4 *>(P.out_k)[o] = k;
      reinterpret_cast<uint4 *>(P.out_v)[o] = v;
    }
  }
}

template <typename K>
fc_status launch_rows(fc_handle *h, K kern, const CacheParams &P, int D, cudaStream_t st) {
  const long long units_per_block = kQThreads / (D / 8), blocks = (P.rows * P.H + units_per_block - 1) / units_per_block;
  const long long most = (long long)h->num_sms * 8;                     // what fits at once: a block then walks on
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3((unsigned)(blocks < most ? blocks : most));
  lc.blockDim = dim3(kQThreads);
  lc.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  lc.attrs = at;
  lc.numAttrs = 1;
  if (cudaLaunchKernelEx(&lc, kern, P) != cudaSuccess) {
    cudaGetLastError();
    return FC_ERR_CUDA;
  }
  return fc_after_launch(h);
}

CacheParams params_of(const fc_handle *h, const fc_cache4 *c) {
  CacheParams P = {};
  P.ck = static_cast<unsigned char *>(c->codes_k);
  P.cv = static_cast<unsigned char *>(c->codes_v);
  P.pk = static_cast<char *>(c->params_k);
  P.pv = static_cast<char *>(c->params_v);
  P.cap = c->capacity_rows;
  P.status = h->status_word;
  P.H = c->num_heads;
  return P;
}

}  // namespace

extern "C" fc_status fc_quantize_cache(fc_handle *h, const fc_kv_view *kv, const fc_cache4 *cache, const int64_t *used,
                                       const int64_t *out_rows, fc_stream stream) {
  if (!h || !kv || !kv->k || !kv->v || !kv->cu_seqlens || kv->batch < 1) return FC_ERR_INVALID_ARG;
  fc_status s = cache4::check(cache);
  if (s != FC_OK) return s;
  if (kv->dtype != cache->dtype || kv->num_heads != cache->num_heads || kv->head_dim != cache->head_dim) return FC_ERR_INVALID_ARG;
  if (((uintptr_t)kv->k & 15) || ((uintptr_t)kv->v & 15) || (kv->stride_token * 2) % 16 != 0 || (kv->stride_head * 2) % 16 != 0)
    return FC_ERR_INVALID_ARG;
  const int64_t rows = kv->cu_seqlens[kv->batch];
  if (rows < 0 || (!out_rows && rows > cache->capacity_rows)) return FC_ERR_INVALID_ARG;
  if (rows == 0) return FC_OK;
  CacheParams P = params_of(h, cache);
  P.k = static_cast<const char *>(kv->k);
  P.v = static_cast<const char *>(kv->v);
  P.token = kv->stride_token * 2;
  P.head = kv->stride_head * 2;
  P.rows = rows;
  P.used = reinterpret_cast<const long long *>(used);
  P.out_rows = reinterpret_cast<const long long *>(out_rows);
  FcDeviceGuard on(h->device);
  if (!on.ok) return FC_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if ((s = fc_flush_pending(h, st)) != FC_OK) return s;
  const bool wide = cache->head_dim == 128;
  if (cache->dtype == FC_F16) return launch_rows(h, wide ? k_quantize<__half, 128> : k_quantize<__half, 64>, P, cache->head_dim, st);
  return launch_rows(h, wide ? k_quantize<__nv_bfloat16, 128> : k_quantize<__nv_bfloat16, 64>, P, cache->head_dim, st);
}

extern "C" fc_status fc_dequantize_cache(fc_handle *h, const fc_cache4 *cache, void *out_k, void *out_v, int64_t rows,
                                         const int64_t *used, fc_stream stream) {
  if (!h || !out_k || !out_v || rows < 0) return FC_ERR_INVALID_ARG;
  fc_status s = cache4::check(cache);
  if (s != FC_OK) return s;
  if (rows > cache->capacity_rows || ((uintptr_t)out_k & 15) || ((uintptr_t)out_v & 15)) return FC_ERR_INVALID_ARG;
  if (rows == 0) return FC_OK;
  CacheParams P = params_of(h, cache);
  P.out_k = static_cast<char *>(out_k);
  P.out_v = static_cast<char *>(out_v);
  P.rows = rows;
  P.used = reinterpret_cast<const long long *>(used);
  FcDeviceGuard on(h->device);
  if (!on.ok) return FC_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if ((s = fc_flush_pending(h, st)) != FC_OK) return s;
  const bool wide = cache->head_dim == 128;
  if (cache->dtype == FC_F16) return launch_rows(h, wide ? k_dequantize<__half, 128> : k_dequantize<__half, 64>, P, cache->head_dim, st);
  return launch_rows(h, wide ? k_dequantize<__nv_bfloat16, 128> : k_dequantize<__nv_bfloat16, 64>, P, cache->head_dim, st);
}
