// Rotary positions of a layer's queries and keys, and the append of a step's keys and values to the cache.
//
// A pair of channels (a, b) of a token at position p is turned by the angle p * f of its pair:
//     a' = a c - b s,  b' = b c + a s,  c = scale * cos(p f),  s = scale * sin(p f)   (inverse: s -> -s).
// The path reads and writes every row once and computes next to nothing: it is bound by HBM (or, for a step's few rows, by
// one launch).  So a block takes whole tokens: the angles of a token are computed once, by one thread per pair, and all
// heads use them from shared memory; every thread then moves 32 bytes of a row (16 of either member of its pairs).
// 32768 tokens of 28 + 4 heads of 128 (bf16): 86.5 us, 6.2 TB/s, 0.95 of a plain copy; a step's 8 tokens 2.6 us.
// Angles: p f in turns, in 64 bits and the remainder of the frequency's rounding, reduced by whole turns before anything is
// rounded to 32 (at p = 10^6 a product in 32 bits is off by 0.06 radians); sine and cosine of the remainder by sincospif.
#include "fc_common.cuh"

#include <math.h>
#include <string.h>

namespace {

constexpr int kRotThreads = 256;
constexpr int kRotMaxPairs = 128;

struct RotParams {
  const char *q, *k, *v;
  char *oq, *ok, *ov;
  long long q_token, q_head, oq_token, oq_head;      // bytes
  long long k_token, k_head, ok_token, ok_head;
  const long long *rows, *pos;
  long long cap, pos_axis, T;
  int *status;
  int Hq, H, Hv, d, R;
  int end1, end2;                                    // pairs below end1 turn by axis 0, below end2 by axis 1, else 2
  float scale, sign;
  double turns[kRotMaxPairs], more[kRotMaxPairs];    // f / (2 pi), and what its rounding to 64 bits left over
};

template <typename T> __device__ __forceinline__ float rot_load(T x);
template <> __device__ __forceinline__ float rot_load(float x) { return x; }
template <> __device__ __forceinline__ float rot_load(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float rot_load(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T rot_store(float x);
template <> __device__ __forceinline__ float rot_store(float x) { return x; }
template <> __device__ __forceinline__ __half rot_store(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 rot_store(float x) { return __float2bfloat16_rn(x); }

template <typename T, int V> struct alignas(sizeof(T) * V) RotVec { T x[V]; };

// V channels of either member per thread: 16 bytes where the rotated part splits into them, else one channel.
template <typename T, int V, bool INTER>
__global__ void __launch_bounds__(kRotThreads)
k_rotary(const __grid_constant__ RotParams P, int tokens_per_block) {
  // [token][pair], the pairs of a thread 16 bytes at a time beside those of its neighbours (94.7 -> 90.6 us: in a run of its own each
  // thread's pairs meet its neighbours' in the same banks; the rest of the way to 86.5 are divisions)
  extern __shared__ __align__(16) float2 cs[];
  using Vec = RotVec<T, V>;
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  const long long t0 = (long long)blockIdx.x * tokens_per_block;
  const int nt = P.T - t0 < tokens_per_block ? (int)(P.T - t0) : tokens_per_block;
  const int pairs = P.R / 2;
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  for (int i = threadIdx.x; i < nt * pairs; i += kRotThreads) {
    const int t = (int)((unsigned)i / (unsigned)pairs), j = i - t * pairs;
    const int axis = j < P.end1 ? 0 : (j < P.end2 ? 1 : 2);
    const double p = (double)P.pos[axis * P.pos_axis + t0 + t];
    double turn = fma(p, P.turns[j], -rint(p * P.turns[j])) + p * P.more[j];
    turn -= rint(turn);
    float s, c;
    sincospif(2.f * (float)turn, &s, &c);
    const int at = V == 1 ? j : 2 * ((j % V) / 2 * (pairs / V) + j / V) + (j & 1);
    cs[t * pairs + at] = make_float2(c * P.scale, s * P.scale * P.sign);
  }
  __syncthreads();
  // r / per_head is the high word of r * over: exact, r * per_head stays below 2^32 (12288 heads of 512)
  const unsigned over = 0xffffffffu / (unsigned)(P.d / (2 * V)) + 1u;
  const int per_head = P.d / (2 * V), per_token = (P.Hq + P.H + P.Hv) * per_head, turned = pairs / V;
  for (int i = threadIdx.x; i < nt * per_token; i += kRotThreads) {
    int t = 0, r = i;
    while (r >= per_token) { r -= per_token; ++t; }  // a token or two
    int h = (int)__umulhi((unsigned)r, over);
    const int e = r - h * per_head;
    const char *src;
    char *dst;
    bool copy = e >= turned;
    if (h < P.Hq) {
      src = P.q + (t0 + t) * P.q_token + h * P.q_head;
      dst = P.oq + (t0 + t) * P.oq_token + h * P.oq_head;
    } else {
      h -= P.Hq;
      const bool value = h >= P.H;
      if (value) { h -= P.H; copy = true; }
      src = (value ? P.v : P.k) + (t0 + t) * P.k_token + h * P.k_head;
      long long row = t0 + t;
      if (P.rows) {
        row = P.rows[t0 + t];
        if (row >= P.cap) {                          // would lie behind the cache: left out and said
          if (e == 0) atomicOr(P.status, FC_DEV_FLAG_INTERNAL);
          continue;
        }
        if (row < 0) continue;                       // a padded token
      }
      dst = (value ? P.ov : P.ok) + row * P.ok_token + h * P.ok_head;
    }
    // channels of the two vectors: the members of V pairs, or 2 V channels as they are
    const int c0 = e < turned ? (INTER ? 2 * V * e : V * e) : 2 * V * e;
    const int c1 = e < turned ? (INTER ? c0 + V : c0 + pairs) : c0 + V;
    const Vec a = *reinterpret_cast<const Vec *>(src + c0 * sizeof(T)), b = *reinterpret_cast<const Vec *>(src + c1 * sizeof(T));
    Vec x = a, y = b;
    if (!copy) {
      float2 w[V];
      if constexpr (V == 1) w[0] = cs[t * pairs + e];
      else {
#pragma unroll
        for (int j = 0; j < V; j += 2) {
          const float4 two = reinterpret_cast<const float4 *>(cs + t * pairs)[j / 2 * turned + e];
          w[j] = make_float2(two.x, two.y);
          w[j + 1] = make_float2(two.z, two.w);
        }
      }
      if (INTER) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float m = rot_load(2 * j < V ? a.x[(2 * j) % V] : b.x[(2 * j) % V]);
          const float n = rot_load(2 * j + 1 < V ? a.x[(2 * j + 1) % V] : b.x[(2 * j + 1) % V]);
          const float2 u = w[j];
          (2 * j < V ? x : y).x[(2 * j) % V] = rot_store<T>(m * u.x - n * u.y);
          (2 * j + 1 < V ? x : y).x[(2 * j + 1) % V] = rot_store<T>(n * u.x + m * u.y);
        }
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float m = rot_load(a.x[j]), n = rot_load(b.x[j]);
          const float2 u = w[j];
          x.x[j] = rot_store<T>(m * u.x - n * u.y);
          y.x[j] = rot_store<T>(n * u.x + m * u.y);
        }
      }
    }
    *reinterpret_cast<Vec *>(dst + c0 * sizeof(T)) = x;
    *reinterpret_cast<Vec *>(dst + c1 * sizeof(T)) = y;
  }
}

template <typename T>
fc_status launch_rotary(fc_handle *h, const RotParams &P, bool inter, cudaStream_t st) {
  constexpr int W = 16 / (int)sizeof(T);
  const bool wide = P.R % (2 * W) == 0;
  // Two tokens to a block where the blocks come in many waves (32768 tokens of 32 heads 94 -> 86 us, 4 tokens 87), else one (5001
  // tokens of 64 heads 27.4 us; 29 and 32 with 2 and 4: fewer blocks fill the last wave worse).
  const int tb = P.T > 64ll * h->num_sms ? 2 : 1;
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3((unsigned)((P.T + tb - 1) / tb));
  lc.blockDim = dim3(kRotThreads);
  lc.dynamicSmemBytes = (size_t)tb * (P.R / 2) * sizeof(float2);
  lc.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  lc.attrs = at;
  lc.numAttrs = 1;
  auto kern = wide ? (inter ? k_rotary<T, W, true> : k_rotary<T, W, false>) : (inter ? k_rotary<T, 1, true> : k_rotary<T, 1, false>);
  if (cudaLaunchKernelEx(&lc, kern, P, tb) != cudaSuccess) {
    cudaGetLastError();
    return FC_ERR_CUDA;
  }
  return fc_after_launch(h);
}

bool rows16(const void *p, int64_t a, int64_t b, size_t elem) {
  return !((uintptr_t)p & 15) && (a * (int64_t)elem) % 16 == 0 && (b * (int64_t)elem) % 16 == 0;
}

}  // namespace

extern "C" fc_status fc_rotary_frequencies(int32_t rotary_dim, double base, const fc_rope_scaling *sc, double *freq, double *scale) {
  if (!freq || !scale || rotary_dim < 2 || rotary_dim > 2 * kRotMaxPairs || (rotary_dim & 1) || !(base > 1.0) || isinf(base))
    return FC_ERR_INVALID_ARG;
  const int kind = sc ? sc->kind : FC_ROPE_PLAIN;
  const double f = sc ? sc->factor : 1.0, r = rotary_dim, two_pi = 6.283185307179586476925;
  if (kind < FC_ROPE_PLAIN || kind > FC_ROPE_BANDS) return FC_ERR_INVALID_ARG;
  if (kind != FC_ROPE_PLAIN && (!(f >= 1.0) || isinf(f))) return FC_ERR_INVALID_ARG;
  if ((kind == FC_ROPE_YARN || kind == FC_ROPE_BANDS) &&
      (sc->original_len < 1 || !(sc->low > 0.0) || !(sc->high > sc->low) || isinf(sc->high)))
    return FC_ERR_INVALID_ARG;
  if (kind == FC_ROPE_NTK && rotary_dim < 4) return FC_ERR_INVALID_ARG;
  if (kind == FC_ROPE_NTK) base *= pow(f, r / (r - 2.0));
  *scale = 1.0;
  double lo = 0.0, hi = 1.0;
  if (kind == FC_ROPE_YARN) {
    // pairs that make more than `high` turns over the original length stay, those of fewer than `low` are stretched by the
    // factor, with a line in between; the pairs where that happens are rounded outwards to whole ones
    auto pair_of = [&](double turns) { return r * log((double)sc->original_len / (turns * two_pi)) / (2.0 * log(base)); };
    lo = floor(pair_of(sc->high));
    hi = ceil(pair_of(sc->low));
    lo = lo > 0.0 ? lo : 0.0;
    hi = hi < r - 1.0 ? hi : r - 1.0;
    if (!(hi > lo)) hi = lo + 0.001;
    *scale = 0.1 * log(f) + 1.0;
  }
  for (int j = 0; j < rotary_dim / 2; ++j) {
    const double x = pow(base, -2.0 * j / r);
    double y = x;
    if (kind == FC_ROPE_LINEAR) y = x / f;
    if (kind == FC_ROPE_YARN) {
      double m = (j - lo) / (hi - lo);
      m = m < 0.0 ? 0.0 : (m > 1.0 ? 1.0 : m);
      y = x * (1.0 - m) + x / f * m;
    }
    if (kind == FC_ROPE_BANDS) {                     // by the turns of the pair itself
      double m = (sc->original_len * x / two_pi - sc->low) / (sc->high - sc->low);
      m = m < 0.0 ? 0.0 : (m > 1.0 ? 1.0 : m);
      y = x * m + x / f * (1.0 - m);
    }
    freq[j] = y;
  }
  return FC_OK;
}

extern "C" fc_status fc_rotary(fc_handle *h, const fc_rotary_args *a, fc_stream stream) {
  if (!h || !a || !a->positions || !a->freq || a->tokens < 0) return FC_ERR_INVALID_ARG;
  if (!a->q && !a->k) return FC_ERR_INVALID_ARG;
  if ((a->q && (!a->out_q || a->num_q_heads < 1)) || (a->k && (!a->out_k || a->num_heads < 1))) return FC_ERR_INVALID_ARG;
  if ((a->v != nullptr) != (a->out_v != nullptr) || (a->v && !a->k)) return FC_ERR_INVALID_ARG;
  if (a->out_rows && (!a->k || a->out_capacity_rows < 0)) return FC_ERR_INVALID_ARG;
  if (a->dtype != FC_F32 && a->dtype != FC_F16 && a->dtype != FC_BF16) return FC_ERR_UNSUPPORTED;
  if (a->head_dim < 64 || a->head_dim % 64 != 0 || a->head_dim > 1024) return FC_ERR_UNSUPPORTED;
  if (a->rotary_dim < 2 || (a->rotary_dim & 1) || a->rotary_dim > a->head_dim) return FC_ERR_INVALID_ARG;
  if (a->rotary_dim > 2 * kRotMaxPairs) return FC_ERR_UNSUPPORTED;
  if ((a->q ? a->num_q_heads : 0) > 4096 || (a->k ? a->num_heads : 0) > 4096 || a->tokens > 0x7fffffffll) return FC_ERR_UNSUPPORTED;
  const size_t es = a->dtype == FC_F32 ? 4 : 2;
  if (a->q && (!rows16(a->q, a->q_stride_token, a->q_stride_head, es) || !rows16(a->out_q, a->out_q_stride_token, a->out_q_stride_head, es)))
    return FC_ERR_INVALID_ARG;
  if (a->k && (!rows16(a->k, a->k_stride_token, a->k_stride_head, es) || !rows16(a->out_k, a->out_k_stride_token, a->out_k_stride_head, es)))
    return FC_ERR_INVALID_ARG;
  if (((uintptr_t)a->v & 15) || ((uintptr_t)a->out_v & 15)) return FC_ERR_INVALID_ARG;
  const int pairs = a->rotary_dim / 2;
  int sec[3] = {a->sections[0], a->sections[1], a->sections[2]};
  if (sec[0] == 0 && sec[1] == 0 && sec[2] == 0) sec[0] = pairs;      // one axis
  if (sec[0] < 0 || sec[1] < 0 || sec[2] < 0 || (int64_t)sec[0] + sec[1] + sec[2] != pairs) return FC_ERR_INVALID_ARG;
  for (int j = 0; j < pairs; ++j)
    if (!isfinite(a->freq[j])) return FC_ERR_INVALID_ARG;
  if (!isfinite(a->scale)) return FC_ERR_INVALID_ARG;
  if (a->tokens == 0) return FC_OK;
  RotParams P;
  memset(&P, 0, sizeof(P));
  const long long b = (long long)es;
  P.q = static_cast<const char *>(a->q);
  P.k = static_cast<const char *>(a->k);
  P.v = static_cast<const char *>(a->v);
  P.oq = static_cast<char *>(a->out_q);
  P.ok = static_cast<char *>(a->out_k);
  P.ov = static_cast<char *>(a->out_v);
  P.q_token = a->q_stride_token * b; P.q_head = a->q_stride_head * b;
  P.oq_token = a->out_q_stride_token * b; P.oq_head = a->out_q_stride_head * b;
  P.k_token = a->k_stride_token * b; P.k_head = a->k_stride_head * b;
  P.ok_token = a->out_k_stride_token * b; P.ok_head = a->out_k_stride_head * b;
  P.rows = reinterpret_cast<const long long *>(a->out_rows);
  P.pos = reinterpret_cast<const long long *>(a->positions);
  P.cap = a->out_capacity_rows;
  P.pos_axis = a->position_stride;
  P.T = a->tokens;
  P.status = h->status_word;
  P.Hq = a->q ? a->num_q_heads : 0;
  P.H = a->k ? a->num_heads : 0;
  P.Hv = a->v ? a->num_heads : 0;
  P.d = a->head_dim;
  P.R = a->rotary_dim;
  P.end1 = sec[0];
  P.end2 = sec[0] + sec[1];
  P.scale = (float)a->scale;
  P.sign = a->inverse ? -1.f : 1.f;
  const double per_turn = 0.15915494309189535, per_turn_more = -9.839338337591243e-18;      // 1 / (2 pi) to 106 bits
  for (int j = 0; j < pairs; ++j) {
    P.turns[j] = a->freq[j] * per_turn;
    P.more[j] = fma(a->freq[j], per_turn, -P.turns[j]) + a->freq[j] * per_turn_more;
  }
  FcDeviceGuard on(h->device);
  if (!on.ok) return FC_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  fc_status s = fc_flush_pending(h, st);
  if (s != FC_OK) return s;
  if (a->dtype == FC_F32) return launch_rotary<float>(h, P, a->interleaved != 0, st);
  if (a->dtype == FC_F16) return launch_rotary<__half>(h, P, a->interleaved != 0, st);
  return launch_rotary<__nv_bfloat16>(h, P, a->interleaved != 0, st);
}
