// Rows of a cache into 4 bits and back (layout: fc_cache4.cuh).
//
// Per half row: min and max, scale = (max - min) / 15 rounded up to the cache's type, so that 15 steps reach the maximum and
// no value is more than half a step off; code = (x - min) / scale to the nearest whole number, the even one of two equally
// near.  Both are decided exactly, whatever the rounding of the arithmetic on the way: the scale by comparing 15 times a
// candidate with the range, the code by the sign of what is left over beside a tie, in 64 bits where it is close.
// Every row is read once and written once.  A lane holds 16 consecutive channels (32 bytes), 8 or 4 lanes a row of K and the same
// row of V; the nibbles change lanes in registers, and every lane writes 8 bytes of codes.  16384 rows of 32 heads: 82 us, 4.2 TB/s,
// bound by the instructions (about 16 a value; 8 channels to a lane 131 us); back 70 us, 4.9 TB/s.
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
  static constexpr unsigned kNan = 0x7e00u, kUnits = 0x6400u;        // 1024
};
template <> struct Num<__nv_bfloat16> {
  using T2 = __nv_bfloat162;
  static __device__ float to(__nv_bfloat16 x) { return __bfloat162float(x); }
  static __device__ __nv_bfloat16 from(float x) { return __float2bfloat16_rn(x); }
  static __device__ __nv_bfloat16 up(float x) { return __float2bfloat16_ru(x); }
  static __device__ __nv_bfloat16 bits(unsigned short b) { return __ushort_as_bfloat16(b); }
  static __device__ unsigned short bits(__nv_bfloat16 x) { return __bfloat16_as_ushort(x); }
  static __device__ float2 both(unsigned w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
  static constexpr unsigned kNan = 0x7fc0u, kUnits = 0x4300u;        // 128
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

// What a lane needs of its half row, and its 8 codes, code i at nibble i, where the short way below cannot be sure: exact
// throughout, and 0 with scale 0 for a half that is all one value or not finite.
struct Quantized { float scale; unsigned word; };

template <typename T>
__device__ __noinline__ Quantized quantize_exactly(uint4 raw, float lo, float hi) {
  Quantized q = {0.f, 0u};
  const float d = hi - lo;
  if (!(d > 0.f && d < INFINITY)) return q;          // also: NaN, an infinity, a range past fp32
  // the smallest number of the type whose 15-fold reaches hi - lo: a guess, moved by what 15 times it lacks
  const float z = d - hi;                            // two-sum: hi - lo = d + e
  const float e = (hi - (d - z)) + (-lo - z);
  auto lacks = [&](float s) { return fmaf(15.f, s, -d) - e; };       // >= 0: enough (15 s and d are multiples of ulp(d) > |e|)
  T s = Num<T>::up(d * (1.f / 15.f));
  if (lacks(Num<T>::to(s)) < 0.f) s = Num<T>::bits((unsigned short)(Num<T>::bits(s) + 1));
  const T below = Num<T>::bits((unsigned short)(Num<T>::bits(s) - (Num<T>::bits(s) ? 1 : 0)));
  if (lacks(Num<T>::to(below)) >= 0.f) s = below;
  q.scale = Num<T>::to(s);
  for (int i = 0; i < 8; ++i) {
    const unsigned two = i < 4 ? (i < 2 ? raw.x : raw.y) : (i < 6 ? raw.z : raw.w);
    const float2 both = Num<T>::both(two);
    const float x = i & 1 ? both.y : both.x, left = x - lo;
    unsigned k;
    if (q.scale > 1e-30f && left + lo == x && x - left == lo) {
      // the difference is exact, and so is the sign of what is left beside the tie above k (a quotient rounded up to a whole
      // number is that number's, and what is left then is below the tie)
      k = (unsigned)__float2int_rd(left / q.scale);
      const float r = fmaf(-((float)k + 0.5f), q.scale, left);
      if (r > 0.f || (r == 0.f && (k & 1u))) k += 1u;
    } else {
      const double wide = (double)x - (double)lo, h = floor(wide / (double)q.scale);
      const double over = wide - (h + 0.5) * (double)q.scale;
      k = (unsigned)((int)h + ((over > 0.0 || (over == 0.0 && ((int)h & 1))) ? 1 : 0));
    }
    q.word |= (k & 15u) << (4 * i);
  }
  return q;
}

// The short way.  Scale: a fifteenth of the range in 32 bits is off by less than 2^-21 of it, so it is one of the numbers of the type
// that both ends of that round up to.  Codes: whole numbers in the last bits of 1.5 * 2^23 + (x - lo) / scale, with a
// quotient that is too small by up to 3e-5: they can only be one too low, at a tie or past it by that much, and what they
// leave over (exact as long as x - lo is) tells, next to being odd at a tie itself.  Where x - lo may not be exact, because its
// parts are 2^12 apart, and some rest is near a tie, it all goes the long way.
template <typename T>
__device__ __forceinline__ float quantize_lane(const uint4 (&raw)[2], float lo, float hi, unsigned (&word)[2]) {
  using T2 = typename Num<T>::T2;
  const float d = hi - lo, v = d * (1.f / 15.f);
  const float above = Num<T>::to(Num<T>::up(fmaf(v, 0x1p-21f, v))), least = Num<T>::to(Num<T>::up(fmaf(v, -0x1p-21f, v)));
  const float z = d - hi, e = (hi - (d - z)) + (-lo - z);            // two-sum: hi - lo = d + e
  float s = fmaf(15.f, least, -d) - e >= 0.f ? least : above;        // is the smaller one enough (a range is often 15 steps sharp)?
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
  inv = fmaf(inv, -0x1p-20f, inv);
  const float2 lo2 = make_float2(-lo, -lo), inv2 = make_float2(inv, inv), s2 = make_float2(-s, -s), two = make_float2(2.f, 2.f);
  const float2 big = make_float2(12582912.f, 12582912.f), gib = make_float2(-12582912.f, -12582912.f);
  float most = -INFINITY;
  float2 past[8];                                    // twice the rest, less a step
  T2 tiny2;
#pragma unroll
  for (int a = 0; a < 2; ++a) {
    const unsigned *w = reinterpret_cast<const unsigned *>(&raw[a]);
    const T2 *h = reinterpret_cast<const T2 *>(&raw[a]);
    word[a] = 0u - 0x3f400000u;                      // what the bits of 1.5 * 2^23, shifted to the nibbles, add up to
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 x = __fadd2_rn(Num<T>::both(w[i]), lo2);
      const float2 m = __ffma2_rn(x, inv2, big);
      const float2 p = past[4 * a + i] = __ffma2_rn(__ffma2_rn(__fadd2_rn(m, gib), s2, x), two, s2);
      word[a] += __float_as_uint(m.x) << (8 * i);
      word[a] += __float_as_uint(m.y) << (8 * i + 4);
      most = fmaxf(fmaxf(most, p.x), p.y);
    }
    const T2 t = __hmin2(__hmin2(__habs2(h[0]), __habs2(h[1])), __hmin2(__habs2(h[2]), __habs2(h[3])));
    tiny2 = a ? __hmin2(tiny2, t) : t;
  }
  // v past 1e-30: neither d nor 1 / s is out of the numbers (so nothing above was NaN)
  const bool plain = v > 1e-30f && v < 1e30f;
  if (!plain || most > -1e-4f * s) {
    const float tiny = fminf(fminf(Num<T>::to(tiny2.x), Num<T>::to(tiny2.y)), fabsf(lo));
    if (!plain || tiny < 0x1p-12f * fmaxf(fabsf(lo), fabsf(hi))) {
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        const Quantized q = quantize_exactly<T>(raw[a], lo, hi);
        word[a] = q.word;
        s = q.scale;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int p = __float_as_int(i & 1 ? past[i / 2].y : past[i / 2].x);
        const unsigned odd = (word[i / 8] >> (4 * (i % 8))) & 1u;
        if (p + (int)odd > 0) word[i / 8] += 1u << (4 * (i % 8));    // > 0, or 0 at an odd one
      }
    }
  }
  return s;
}

// Eight rows of bytes in eight lanes (four in four: MANY false), first and last four of a row in a and b: columns in the lanes'
// place, by exchanges over one bit of the lane at a time.  Twice is nothing.
template <bool MANY>
__device__ __forceinline__ void turn_bytes(int u, unsigned &a, unsigned &b) {
  if (MANY) {
    const unsigned got = __shfl_xor_sync(0xffffffffu, u & 4 ? a : b, 4);
    if (u & 4) a = got; else b = got;
  }
  unsigned got = __shfl_xor_sync(0xffffffffu, __byte_perm(a, b, u & 2 ? 0x5410 : 0x7632), 2);
  a = __byte_perm(a, got, u & 2 ? 0x3254 : 0x5410);
  b = __byte_perm(b, got, u & 2 ? 0x3276 : 0x7610);
  got = __shfl_xor_sync(0xffffffffu, __byte_perm(a, b, u & 1 ? 0x6420 : 0x7531), 1);
  a = __byte_perm(a, got, u & 1 ? 0x3514 : 0x5240);
  b = __byte_perm(b, got, u & 1 ? 0x3716 : 0x7260);
}
// Nibbles of two words: the even ones of both in the first, the odd ones in the second.  Twice is nothing.
__device__ __forceinline__ void turn_nibbles(unsigned &a, unsigned &b) {
  const unsigned even = (a & 0x0f0f0f0fu) | ((b & 0x0f0f0f0fu) << 4), odd = ((a >> 4) & 0x0f0f0f0fu) | (b & 0xf0f0f0f0u);
  a = even;
  b = odd;
}
// Where lane u keeps its 8 bytes of a row of values: after the exchange it has run u of the even ones, then of the odd ones.
template <int D>
__device__ __forceinline__ int value_bytes(int u) { return D == 128 ? (u < 4 ? 2 * u : 2 * u - 7) * 8 : 8 * u; }

// One matrix's row of one head: LANES lanes with 16 channels each.
template <typename T, int D, bool VALUES>
__device__ __forceinline__ void quantize_row(const uint4 (&raw)[2], int u, unsigned char *codes, char *params, bool write) {
  constexpr int LANES = D / 16, HALF = LANES / 2;
  using T2 = typename Num<T>::T2;
  const T2 *w = reinterpret_cast<const T2 *>(&raw[0]);
  // minimum, and minus the maximum, of the half: two 16-bit numbers in one exchange; NaN stays
  T2 a = __hmin2_nan(__hmin2_nan(__hmin2_nan(w[0], w[1]), __hmin2_nan(w[2], w[3])), __hmin2_nan(__hmin2_nan(w[4], w[5]), __hmin2_nan(w[6], w[7])));
  T2 b = __hmax2_nan(__hmax2_nan(__hmax2_nan(w[0], w[1]), __hmax2_nan(w[2], w[3])), __hmax2_nan(__hmax2_nan(w[4], w[5]), __hmax2_nan(w[6], w[7])));
  T2 both;
  both.x = __hmin_nan(a.x, a.y);
  both.y = __hneg(__hmax_nan(b.x, b.y));
#pragma unroll
  for (int o = 1; o < HALF; o <<= 1) {
    const unsigned other = __shfl_xor_sync(0xffffffffu, *reinterpret_cast<const unsigned *>(&both), o);
    both = __hmin2_nan(both, *reinterpret_cast<const T2 *>(&other));
  }
  const float lo = Num<T>::to(both.x), hi = -Num<T>::to(both.y);
  unsigned word[2];
  const float s = quantize_lane<T>(raw, lo, hi, word);
  __syncwarp();
  const bool finite = hi - lo < INFINITY;            // not so with NaN, an infinity, or a range past fp32
  if (VALUES) {
    turn_nibbles(word[0], word[1]);
    turn_bytes<D == 128>(u, word[0], word[1]);
    if (write) *reinterpret_cast<uint2 *>(codes + value_bytes<D>(u)) = make_uint2(word[0], word[1]);
  } else {
    // the lane's slice has a quad for each run; the neighbour has the other slice of the words.  An even lane makes the words of
    // runs 0 and 1, an odd one of 2 and 3.
    const bool odd = u & 1;
    const unsigned got = __shfl_xor_sync(0xffffffffu, odd ? word[0] : word[1], 1), mine = odd ? word[1] : word[0];
    const unsigned first = odd ? got : mine, second = odd ? mine : got;                      // of the even slice, of the odd one
    auto spread = [](unsigned q) {                   // i = 0..3 -> nibbles 0, 4, 1, 5
      return (q & 0xfu) | ((q & 0xf0u) << 12) | ((q & 0xf00u) >> 4) | ((q & 0xf000u) << 8);
    };
    if (write) {
      unsigned char *at = codes + 2 * odd * (D / 8) + (u >> 1) * 4;
      *reinterpret_cast<unsigned *>(at) = spread(first) | (spread(second) << 8);
      *reinterpret_cast<unsigned *>(at + D / 8) = spread(first >> 16) | (spread(second >> 16) << 8);
    }
  }
  if (write && (u & (HALF - 1)) == 0) {
    const unsigned ms = Num<T>::bits(Num<T>::from(s)), ml = finite ? (unsigned)Num<T>::bits(both.x) : Num<T>::kNan;
    reinterpret_cast<unsigned *>(params)[u / HALF] = ms | (ml << 16);
  }
}

// A block does one head's rows, 256 / LANES at a time: its reads are whole rows, its writes runs of rows.
template <typename T, int D>
__global__ void __launch_bounds__(kQThreads, 3)
k_quantize(const CacheParams P, int rounds) {
  constexpr int LANES = D / 16, ROWS = kQThreads / LANES;
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  const unsigned h = blockIdx.x % (unsigned)P.H;
  const int u = threadIdx.x % LANES;
  int t = (int)(blockIdx.x / (unsigned)P.H) * rounds * ROWS + threadIdx.x / LANES;
  const int warp_row = t - (threadIdx.x & 31) / LANES;                // of the warp's first lane: a warp stays together
  const char *k = P.k + h * P.head + t * P.token + 32 * u, *v = P.v + h * P.head + t * P.token + 32 * u;
  const long long step = ROWS * P.token;
  const size_t head = (size_t)h * P.cap;
  unsigned char *ck = P.ck + head * (D / 2), *cv = P.cv + head * (D / 2);
  char *pk = P.pk + head * cache4::kParamBytes, *pv = P.pv + head * cache4::kParamBytes;
  uint4 rk[2] = {}, rv[2] = {};
  auto fetch = [&]() {
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      rk[a] = __ldcs(reinterpret_cast<const uint4 *>(k) + a);
      rv[a] = __ldcs(reinterpret_cast<const uint4 *>(v) + a);
    }
  };
  if (t < (int)P.rows) fetch();                                       // fewer than 2^31; beside the look at how many are used
  int rows = (int)P.rows;
  if (P.used) { const long long m = *P.used; rows = m < rows ? (int)(m < 0 ? 0 : m) : rows; }
#pragma unroll 1
  for (int i = 0; i < rounds && warp_row + i * ROWS < rows; ++i, t += ROWS) {
    const uint4 now_k[2] = {rk[0], rk[1]}, now_v[2] = {rv[0], rv[1]};
    if (i + 1 < rounds && t + ROWS < rows) {                          // the next rows, while these are worked on
      k += step;
      v += step;
      fetch();
    }
    const bool have = t < rows;
    long long row = t;
    if (P.out_rows) {
      row = have ? P.out_rows[t] : 0;
      if (have && row >= P.cap && u == 0) atomicOr(P.status, FC_DEV_FLAG_INTERNAL);
    }
    const bool write = have && row >= 0 && row < P.cap;
    const unsigned r = write ? (unsigned)row : 0u;
    quantize_row<T, D, false>(now_k, u, ck + (size_t)r * (D / 2), pk + (size_t)r * cache4::kParamBytes, write);
    quantize_row<T, D, true>(now_v, u, cv + (size_t)r * (D / 2), pv + (size_t)r * cache4::kParamBytes, write);
  }
}

template <typename T, int D, bool VALUES>
__device__ __forceinline__ void values_row(const unsigned char *codes, const char *params, int u, uint4 (&out)[2]) {
  constexpr int HALF = D / 32;
  unsigned word[2];                                  // code i of the lane at nibble i: the steps above backwards
  if (VALUES) {
    const uint2 x = __ldcs(reinterpret_cast<const uint2 *>(codes + value_bytes<D>(u)));
    word[0] = x.x;
    word[1] = x.y;
    turn_bytes<D == 128>(u, word[0], word[1]);
    turn_nibbles(word[0], word[1]);
  } else {
    const bool odd = u & 1;
    const unsigned char *at = codes + 2 * odd * (D / 8) + (u >> 1) * 4;
    const unsigned a = *reinterpret_cast<const unsigned *>(at), b = *reinterpret_cast<const unsigned *>(at + D / 8);
    auto gather = [](unsigned v) {                   // nibbles 0, 4, 1, 5 -> 0, 1, 2, 3
      return (v & 0xfu) | ((v >> 12) & 0xf0u) | ((v << 4) & 0xf00u) | ((v >> 8) & 0xf000u);
    };
    const unsigned first = gather(a) | (gather(b) << 16), second = gather(a >> 8) | (gather(b >> 8) << 16);
    const unsigned got = __shfl_xor_sync(0xffffffffu, odd ? first : second, 1);
    word[0] = odd ? got : first;
    word[1] = odd ? second : got;
  }
  // Two neighbours at a time: their nibbles under the exponent of the first number whose last bit is 1, less that number, are the
  // codes; what they stand for is one fused operation, and so rounded once.
  using T2 = typename Num<T>::T2;
  const T2 sl = reinterpret_cast<const T2 *>(params)[u / HALF];
  const unsigned one = Num<T>::kUnits | (Num<T>::kUnits << 16);
  T2 scale, low, units;
  scale.x = scale.y = sl.x;
  low.x = low.y = sl.y;
  units = *reinterpret_cast<const T2 *>(&one);
#pragma unroll
  for (int a = 0; a < 2; ++a) {
    unsigned r[4];
    const unsigned next = word[a] >> 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned x = (__byte_perm(word[a], next, i | ((4 + i) << 8)) & 0x000f000fu) | one;
      const T2 y = __hfma2(__hsub2(*reinterpret_cast<const T2 *>(&x), units), scale, low);
      r[i] = *reinterpret_cast<const unsigned *>(&y);
    }
    out[a] = make_uint4(r[0], r[1], r[2], r[3]);
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(kQThreads, 8)
k_dequantize(const CacheParams P, int rounds) {
  constexpr int LANES = D / 16, ROWS = kQThreads / LANES;
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  int rows = (int)P.rows;                            // fewer than 2^31
  if (P.used) { const long long m = *P.used; rows = m < rows ? (int)(m < 0 ? 0 : m) : rows; }
  const unsigned h = blockIdx.x % (unsigned)P.H;
  const int u = threadIdx.x % LANES;
  int t = (int)(blockIdx.x / (unsigned)P.H) * rounds * ROWS + threadIdx.x / LANES;
  const int warp_row = t - (threadIdx.x & 31) / LANES;
  const size_t head = (size_t)h * P.cap;
  const unsigned char *ck = P.ck + head * (D / 2), *cv = P.cv + head * (D / 2);
  const char *pk = P.pk + head * cache4::kParamBytes, *pv = P.pv + head * cache4::kParamBytes;
  uint4 *ok = reinterpret_cast<uint4 *>(P.out_k) + h * (D / 8) + 2 * u, *ov = reinterpret_cast<uint4 *>(P.out_v) + h * (D / 8) + 2 * u;
  const size_t pitch = (size_t)P.H * (D / 8);
#pragma unroll 1
  for (int i = 0; i < rounds && warp_row + i * ROWS < rows; ++i, t += ROWS) {
    const bool have = t < rows;
    const unsigned r = have ? (unsigned)t : 0u;
    uint4 k[2], v[2];
    values_row<T, D, false>(ck + (size_t)r * (D / 2), pk + (size_t)r * cache4::kParamBytes, u, k);
    values_row<T, D, true>(cv + (size_t)r * (D / 2), pv + (size_t)r * cache4::kParamBytes, u, v);
    if (have) {
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        __stcs(ok + r * pitch + a, k[a]);                           // not read again soon
        __stcs(ov + r * pitch + a, v[a]);
      }
    }
  }
}

// most: rounds of a block, once every SM has its blocks many times over.  Forth the next round's loads are under way beside the
// arithmetic (16384 rows of 32 heads: 107, 91, 84, 81, 81 and 95 us with 1, 2, 4, 8, 16 and 32); back there is little to hide and many
// short blocks spread the writes better (71, 70, 72, 77, 89 and 149 us).
template <typename K>
fc_status launch_rows(fc_handle *h, K kern, const CacheParams &P, int D, int most, cudaStream_t st) {
  const long long rows_per_round = kQThreads / (D / 16), rounds_all = (P.rows + rows_per_round - 1) / rows_per_round;
  const int rounds = rounds_all * P.H >= 4ll * most * h->num_sms ? most : (rounds_all * P.H >= 4ll * 2 * h->num_sms ? 2 : 1);
  const long long blocks = (rounds_all + rounds - 1) / rounds * P.H;
  if (blocks > 0x7fffffffll) return FC_ERR_UNSUPPORTED;
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3((unsigned)blocks);
  lc.blockDim = dim3(kQThreads);
  lc.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  lc.attrs = at;
  lc.numAttrs = 1;
  if (cudaLaunchKernelEx(&lc, kern, P, rounds) != cudaSuccess) {
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
  if (rows > 0x7fffffffll - 4096) return FC_ERR_UNSUPPORTED;        // row numbers past the last, in whole blocks, are ints too
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
  if (cache->dtype == FC_F16) return launch_rows(h, wide ? k_quantize<__half, 128> : k_quantize<__half, 64>, P, cache->head_dim, 8, st);
  return launch_rows(h, wide ? k_quantize<__nv_bfloat16, 128> : k_quantize<__nv_bfloat16, 64>, P, cache->head_dim, 8, st);
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
  if (cache->dtype == FC_F16) return launch_rows(h, wide ? k_dequantize<__half, 128> : k_dequantize<__half, 64>, P, cache->head_dim, 2, st);
  return launch_rows(h, wide ? k_dequantize<__nv_bfloat16, 128> : k_dequantize<__nv_bfloat16, 64>, P, cache->head_dim, 2, st);
}
