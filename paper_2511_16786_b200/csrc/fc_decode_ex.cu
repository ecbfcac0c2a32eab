// Decoding step over rows held in 4 bits or in 16, with or without a window and sinks (fc_decode_attention_ex).
//
// For every sequence and query head  out = sum_j w_j v_j / sum_j w_j,  w_j = exp(q k_j / sqrt d)  over the visible rows j: kept
// rows, then the 16-bit tail.  A step reads every visible row once; the frame is that of fc_decode.cu: the tiles of all
// sequences and heads form one line, one block per SM takes an equal share of it, a warp keeps a ring of tiles in flight, the
// other warps only ever wait for the tile they use, blocks that share a sequence meet in a second kernel.
// 189810 rows of 4 heads (4 bits, 7 query heads each, d = 128): 34.4 us, 3.2 TB/s; 41770 rows of 32 heads 50.1 us, 3.9 TB/s: some
// 7 us for two launches, the first tile and the joins, the rest bound by the instructions (0.54 a cycle and scheduler, over the
// whole kernel; a 4-bit row has 3.6 times the arithmetic per byte of a 16-bit one).  A step over 820 rows takes 7.4 us.
//
//  * A row of 4 bits is 72 bytes of K or V at d = 128 instead of 256.  Nothing is expanded in memory or to fp32:
//    - codes are masked out of the loaded words and are the tensor cores' operands as they stand, as subnormal half numbers
//      (code * 2^-24, exact; the second nibble of a word is 16 times that, which the queries or the output rows undo);
//    - a half row's scale multiplies sums of d/2 products (keys) or the weights (values), never a code;
//    - its minimum goes with the sum of the query's channels (keys) or with a sum of weights (values), both in fp32.
//    Rows of the cache are the rows of the first product and queries its columns, channels the rows of the second: the scores,
//    turned round in registers (8 x 8 blocks, one instruction each), are the second product's right operand, what a lane keeps
//    of a query stays with it, and eight columns are enough for 8 query heads (queries as rows: 43 and 61 us).
//  * Four warps share a tile of 128 rows, 32 each, and three such teams take the tiles by turns (two: 43 and 66 us, queries as rows).
//  * Queries are brought to 2^14 .. 2^15 by a power of two before they become half numbers (exact but for channels 2^-25 of the
//    largest).  Weight * scale becomes one at a power of two of its own, which a query has for either half of its output and which
//    follows the largest such product, not the largest weight or the largest scale: the rounding (11 bits, or 2^-33 of that product)
//    neither overflows nor loses rows beside one whose scale is large and whose weight is not, whatever the range of the cache's
//    type.  (With one power for all, of the largest scale met: 48.7 instead of 50.1 us over the 41770 rows, 33.4 instead of 36.5
//    over 100000 rows of 4 heads with 12 query heads each, but a row lost bits from 2^25 times its scale on.)
//  * Kept rows of 16 bits and tails come in tiles of 32 rows (two warps each, 16 KB at d = 128, about what 128 rows of 4 bits take),
//    so every tile of the line costs about the same.
//  * A window makes of a sequence's tiles the first few and the last ones; rows of them that are not visible get no weight.
#include "fc_cache4.cuh"
#include "fc_line.cuh"
#include "fc_mbar.cuh"
#include "fc_tile.cuh"

namespace {

using namespace tile;
using line::Share;

constexpr int kTeam = 4;                       // warps on one tile
constexpr int kTeams = 3;                      // that take the tiles of a block by turns
constexpr int kWarps = kTeam * kTeams;         // consumer warps; the first of four more loads
constexpr int kConsumers = 32 * kWarps;
constexpr int kThreads = kConsumers + 128;
// Registers of a thread: 128 at launch, moved from the loading warps to the others (with 152 instead of 160 a step over 41770
// rows of 32 heads takes 52 us instead of 49).
constexpr int kRegsLaunch = 128, kRegsLoad = 32, kRegsRows = 160;
static_assert(kRegsLoad + kTeams * kRegsRows <= kRegsLaunch * (kTeams + 1), "a register split has to come out of what was launched");
constexpr int kRows4 = 32 * kTeam;             // rows of a 4-bit tile
constexpr int kRows16 = 32;                    // rows of a 16-bit tile
constexpr int kMaxBlocks = 256;                // blocks of a launch, at most
// Weights are 2^(score - reference).  A reference moves up, so that the largest weight is 2^kReset, where one passes 2^kTop: in 16 bits
// none overflows then, and weights down to 2^-24 of the largest keep all bits.
constexpr float kTop = 14.f, kReset = 10.f;
// Beside 4-bit tiles weights stay in fp32 and are 2^kDown smaller, so that sums of weight * minimum over up to 2^18 rows do not
// overflow, whatever the values are.  There weight * scale is kept to these bounds, by a power of two of its own, kMostUp at most.
constexpr float kDown = 34.f, kMostUp = 126.f;
constexpr float kDownPower = 0x1p34f, kMostUpPower = 0x1p126f;
constexpr float kNothing = -3e38f;             // reference of a query that has seen nothing yet

struct ExParams {
  const void *q;
  void *out;
  const long long *offsets;
  const int *tail_len;
  float *part_o;                               // [slot][query heads of a KV head][D]
  float2 *part_ml;                             // [slot][query heads of a KV head]: (reference, sum)
  int2 *span;                                  // [H][batch]: first and last block with tiles of the sequence (first > last: none)
  int *status;
  int B, H, Hq, G, nb, tail_cap, has_tail, window, sinks;
  float scale_log2;                            // log2(e) / sqrt(D)
  long long cache_rows;
  const unsigned char *ck, *cv, *pk, *pv;      // a 4-bit cache
};

struct ExMaps {
  CUtensorMap k, v, tk, tv;                    // k, v: only of 16-bit rows
};

// A sequence's tiles: of the kept rows [0, a) and [b, c), then of the tail [ta, tb) and [tc, td) (tile numbers).
struct SeqTiles {
  long long off0, start;                       // first row; where its tiles start (even in a 4-bit cache: copies are in 16 bytes)
  int n_main, n_tail;
  int low, high;                               // visible: rows < low and rows >= high
  int a, b, main, ta, tb, tiles;               // main: tiles of kept rows in the list; ta, tb as a, b
};

// Where a sequence's rows are: in the cache [r0, r1), in the tail nt.
struct Rows {
  long long r0, r1;
  int nt;
  __device__ __forceinline__ bool operator==(const Rows &o) const { return r0 == o.r0 && r1 == o.r1 && nt == o.nt; }
};
__device__ __forceinline__ Rows rows_of(const ExParams &P, int i) {
  return {__ldcg(P.offsets + i), __ldcg(P.offsets + i + 1), P.has_tail ? __ldcg(P.tail_len + i) : 0};
}

template <bool Q4>
__device__ __forceinline__ SeqTiles seq_tiles(const ExParams &P, const Rows &rows) {
  constexpr int M = Q4 ? kRows4 : kRows16;
  SeqTiles s;
  long long r0 = rows.r0, r1 = rows.r1;
  const int nt = rows.nt;
  r1 = r1 > P.cache_rows ? P.cache_rows : r1;  // rows that the cache does not have are none
  r0 = r0 < 0 ? 0 : r0;
  s.off0 = r0;
  s.n_main = r1 > r0 ? (int)(r1 - r0) : 0;
  s.n_tail = nt < 0 ? 0 : (nt > P.tail_cap ? P.tail_cap : nt);
  const int n = s.n_main + s.n_tail, skew = Q4 ? (int)(r0 & 1) : 0;
  s.start = r0 - skew;
  s.low = n;
  s.high = n;
  if (P.window > 0 && n > P.window && n - P.window > P.sinks) {
    s.low = P.sinks;
    s.high = n - P.window;
  }
  auto up = [](int x, int m) { return (x + m - 1) / m; };
  const int all = s.n_main ? up(s.n_main + skew, M) : 0;
  s.a = s.n_main ? up((s.low < s.n_main ? s.low : s.n_main) + (s.low ? skew : 0), M) : 0;
  s.b = s.high < s.n_main ? (s.high + skew) / M : all;
  s.b = s.b < s.a ? s.a : s.b;
  s.main = s.a + all - s.b;
  const int tall = up(s.n_tail, kRows16), tlow = s.low - s.n_main, thigh = s.high - s.n_main;
  s.ta = up(tlow < 0 ? 0 : (tlow < s.n_tail ? tlow : s.n_tail), kRows16);
  s.tb = (thigh < 0 ? 0 : (thigh < s.n_tail ? thigh : s.n_tail)) / kRows16;
  if (thigh >= s.n_tail) s.tb = tall;
  s.tb = s.tb < s.ta ? s.ta : s.tb;
  s.tiles = s.main + s.ta + tall - s.tb;
  return s;
}
// local tile lt -> is it of the tail, its number there, the row (of the sequence) it starts at
struct TileAt {
  bool tail;
  int number, row;
};
template <bool Q4>
__device__ __forceinline__ TileAt tile_at(const SeqTiles &s, int lt) {
  TileAt t;
  t.tail = lt >= s.main;
  if (!t.tail) {
    t.number = lt < s.a ? lt : lt - s.a + s.b;
    t.row = t.number * (Q4 ? kRows4 : kRows16) - (Q4 ? (int)(s.off0 - s.start) : 0);
  } else {
    lt -= s.main;
    t.number = lt < s.ta ? lt : lt - s.ta + s.tb;
    t.row = s.n_main + t.number * kRows16;
  }
  return t;
}

__device__ __forceinline__ unsigned bits_below(int n) { return n <= 0 ? 0u : (n >= 32 ? 0xffffffffu : (1u << n) - 1u); }

__device__ __forceinline__ void load_bytes(void *dst, const void *src, unsigned bytes, unsigned long long *bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n"
               ::"r"(mbar::address(dst)), "l"(__cvta_generic_to_global(src)), "r"(bytes), "r"(mbar::address(bar)) : "memory");
}

__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, %0;\n" ::"n"(kConsumers) : "memory"); }

// Sizes in shared memory.  A stage holds a 4-bit tile (codes of K, of V, parameters of K, of V) or a 16-bit one (K, V as boxes of 64 channels).
template <int D, bool Q4, int NQ>
struct Geo {
  static constexpr int kCode = D / 2, kParam = cache4::kParamBytes;
  static constexpr int kBytes4 = kRows4 * 2 * (kCode + kParam);
  static constexpr int kBox = kRows16 * 128, kBytes16 = 2 * (D / 64) * kBox;
  static constexpr int kStage = ((Q4 && kBytes4 > kBytes16 ? kBytes4 : kBytes16) + 1023) / 1024 * 1024;
  static constexpr int kStride = D + 4;        // floats per row of a warp's output in the merge buffer
  static constexpr int kMerge = kWarps * 8 * NQ * (kStride + 4) * (int)sizeof(float);    // output, (reference, sum), two sums of minima
  static constexpr int kRoom = 226 * 1024 - 1024 - 256 - kMerge;
  static constexpr int kFit = kRoom / kStage > 12 ? 12 : kRoom / kStage;
  static constexpr int kStages = kFit / kTeams * kTeams;                               // a stage is always the same team's
  static constexpr size_t kSmem = (size_t)kStages * kStage + kMerge + 1024;
};

// The first product of a sum: nothing is there yet.
template <typename T>
__device__ __forceinline__ void mma_first(float (&d)[4], const unsigned (&a)[4], unsigned b0, unsigned b1) {
  if (std::is_same<T, __half>::value)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};\n"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};\n"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
// An 8 x 8 block of 16-bit numbers, a row over four lanes, turned round.
__device__ __forceinline__ unsigned transposed(unsigned x) {
  unsigned y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(y) : "r"(x));
  return y;
}
// Shared memory by its own address: one register, offsets in the instruction.
__device__ __forceinline__ uint4 lds128(unsigned a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ uint2 lds64(unsigned a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];\n" : "=r"(v.x), "=r"(v.y) : "r"(a));
  return v;
}
__device__ __forceinline__ unsigned lds32(unsigned a) {
  unsigned v;
  asm volatile("ld.shared.u32 %0, [%1];\n" : "=r"(v) : "r"(a));
  return v;
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <typename T> __device__ __forceinline__ float2 two(unsigned w);
template <> __device__ __forceinline__ float2 two<__half>(unsigned w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }
template <> __device__ __forceinline__ float2 two<__nv_bfloat16>(unsigned w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

template <typename T, int D, bool Q4, int NQ>
__global__ void __launch_bounds__(kThreads, 1)
k_decode_ex(const __grid_constant__ ExParams P, const __grid_constant__ ExMaps M) {
  using S = Geo<D, Q4, NQ>;
  constexpr int kStages = S::kStages, kHeads = 8 * NQ, MT = D / 16;
  extern __shared__ unsigned char smem_raw[];
  unsigned char *smem = reinterpret_cast<unsigned char *>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  float *mbuf = reinterpret_cast<float *>(smem + kStages * S::kStage);
  __shared__ unsigned long long full[kStages], empty[kStages];
  const int blk = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), g = lane >> 2, t = lane & 3;
  const int team = warp / kTeam;

  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) { mbar::init(&full[i], 1u); mbar::init(&empty[i], kTeam); }
    mbar::init_done();
  }
  if (tid == kConsumers) {
    if (!Q4) { prefetch_map(&M.k); prefetch_map(&M.v); }
    if (P.has_tail) { prefetch_map(&M.tk); prefetch_map(&M.tv); }
  }
  __syncthreads();
  // While the kernels in front still run, the share is worked out from the lengths as they are now.  It is kept if they are
  // the same once those kernels are done, as they are but for the first step after a selection.
  const bool few = P.B <= 32;                  // a sequence per lane
  Rows mine = few && lane < P.B ? rows_of(P, lane) : Rows{};
  auto share = [&]() {
    return line::find_share(P.B, P.H, P.nb, blk, lane, [&](int i) { return seq_tiles<Q4>(P, few ? mine : rows_of(P, i)).tiles; });
  };
  Share sr;
  if (few) sr = share();
  asm volatile("griddepcontrol.wait;\n" ::: "memory");       // what the kernels before this one wrote is visible from here
  const Rows now = few && lane < P.B ? rows_of(P, lane) : Rows{};
  if (!few || !__all_sync(0xffffffffu, now == mine)) {
    mine = now;
    sr = share();
  }
  const long long lo = sr.lo, hi = sr.hi, line_len = sr.line_len;
  const int nb = sr.nb;
  int h = sr.h, b = sr.b;
  long long at = sr.line;
  if (blk == 0)                                // sequences without rows
    for (int i = tid; i < P.B; i += kThreads)
      if (seq_tiles<Q4>(P, rows_of(P, i)).tiles == 0) {
        for (int hh = 0; hh < P.H; ++hh) P.span[(size_t)hh * P.B + i] = make_int2(0, -1);
        for (int c = 0; c < P.Hq * D / 8; ++c)
          reinterpret_cast<uint4 *>(static_cast<T *>(P.out) + (size_t)i * P.Hq * D)[c] = make_uint4(0u, 0u, 0u, 0u);
      }
  if (lo >= hi) return;
  SeqTiles s = seq_tiles<Q4>(P, rows_of(P, b));
  auto advance = [&](long long ti) {           // on to the sequence and head that tile ti belongs to
    while (ti >= at + s.tiles) {
      at += s.tiles;
      if (++b == P.B) { b = 0; ++h; }
      s = seq_tiles<Q4>(P, rows_of(P, b));
    }
  };

  if (warp >= kWarps) {
    // producer
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(kRegsLoad));
    if (warp == kWarps && lane == 0) {
      int n = 0;
      bool ok = true;
      for (long long ti = lo; ti < hi; ++ti, ++n) {
        advance(ti);
        const int st = n % kStages;
        if (n >= kStages && !mbar::wait(&empty[st], (unsigned)(n / kStages - 1) & 1u)) { ok = false; break; }
        unsigned char *dst = smem + st * S::kStage;
        const TileAt ta = tile_at<Q4>(s, (int)(ti - at));
        if (Q4 && !ta.tail) {
          const long long row = s.start + (long long)ta.number * kRows4;            // even, and even many: runs of 16 bytes
          const long long end = s.off0 + s.n_main - row;
          const unsigned rows = (unsigned)(end < kRows4 ? end + (end & 1) : kRows4);
          mbar::expect_tx(&full[st], rows * 2u * (S::kCode + S::kParam));
          const size_t r = (size_t)h * P.cache_rows + row;
          load_bytes(dst, P.ck + r * S::kCode, rows * S::kCode, &full[st]);
          load_bytes(dst + 2 * kRows4 * S::kCode, P.pk + r * S::kParam, rows * S::kParam, &full[st]);
          load_bytes(dst + kRows4 * S::kCode, P.cv + r * S::kCode, rows * S::kCode, &full[st]);
          load_bytes(dst + kRows4 * (2 * S::kCode + S::kParam), P.pv + r * S::kParam, rows * S::kParam, &full[st]);
        } else {
          mbar::expect_tx(&full[st], (unsigned)S::kBytes16);
#pragma unroll
          for (int c = 0; c < D / 64; ++c) {
            if (!ta.tail) {
              const int r = (int)(s.off0 + (long long)ta.number * kRows16);
              tma_load_3d(dst + c * S::kBox, &M.k, 64 * c, h, r, &full[st]);
              tma_load_3d(dst + (D / 64 + c) * S::kBox, &M.v, 64 * c, h, r, &full[st]);
            } else {
              tma_load_4d(dst + c * S::kBox, &M.tk, 64 * c, h, ta.number * kRows16, b, &full[st]);
              tma_load_4d(dst + (D / 64 + c) * S::kBox, &M.tv, 64 * c, h, ta.number * kRows16, b, &full[st]);
            }
          }
        }
      }
      if (!mbar::drain(full, n)) ok = false;   // no block ends under its own loads
      if (!ok) atomicOr(P.status, FC_DEV_FLAG_TIMEOUT);
    }
    return;
  }

  // consumers
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" ::"n"(kRegsRows));
  const unsigned sbase = mbar::address(smem);
  float *mo = mbuf;                                                        // [warp][kHeads][kStride]
  float2 *mml = reinterpret_cast<float2 *>(mo + kWarps * kHeads * S::kStride);   // [warp][kHeads]
  float2 *mmin = mml + kWarps * kHeads;                                    // [warp][kHeads]: weights times minima, either half
  // a number that lanes (g, .) have for query g, as that of the queries 2t and 2t + 1
  auto of_columns = [&](float x) { return make_float2(__shfl_sync(0xffffffffu, x, 8 * t), __shfl_sync(0xffffffffu, x, 8 * t + 4)); };
  bool failed = false;
  int n = 0;
  for (long long ti = lo; ti < hi;) {
    advance(ti);
    const long long ti0 = ti, seg_end = at + s.tiles < hi ? at + s.tiles : hi;
    const T *qb = static_cast<const T *>(P.q) + ((long long)b * P.Hq + (long long)h * P.G) * D;
    // The query heads of this KV head as columns of the right operand: query g (+ 8 r), depth as the left operand's channels.
    // Scores then have rows (of the cache) as rows and queries as columns, like the output has channels and queries: what a lane
    // keeps of a query (reference, sums) is of its columns 2t, 2t+1 (+ 8 r) throughout.
    unsigned qf[MT][NQ][2];
    float2 qsum[NQ][2] = {}, qback[NQ] = {};   // of a 4-bit tile: log2(e)/sqrt(d) times the halves' sums; what undoes the power of two
    auto load_q4 = [&]() {
#pragma unroll
      for (int r = 0; r < NQ; ++r) {
        const bool mine = g + 8 * r < P.G;
        const T *row = qb + (g + 8 * r) * D;
        float top = 0.f, sum[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < MT; ++i) {         // channels 16 i + 4 t ..
          const uint2 w = mine ? *reinterpret_cast<const uint2 *>(row + 16 * i + 4 * t) : make_uint2(0u, 0u);
          const float2 x = two<T>(w.x), y = two<T>(w.y);
          top = fmaxf(top, fmaxf(fmaxf(fabsf(x.x), fabsf(x.y)), fmaxf(fabsf(y.x), fabsf(y.y))));
          sum[i / (MT / 2)] += (x.x + x.y) + (y.x + y.y);
        }
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
          sum[0] += __shfl_xor_sync(0xffffffffu, sum[0], o);
          sum[1] += __shfl_xor_sync(0xffffffffu, sum[1], o);
        }
        int e = (int)(__float_as_uint(top) >> 23);                         // biased exponent of the largest
        e = e < 16 ? 16 : (e > 254 ? 254 : e);
        const float f = __uint_as_float((unsigned)(268 - e) << 23);        // 2^(14 - (e - 127))
        // a sum of codes * 2^-24 times queries * f, times this: the score's part in log2 units
        const float back = P.scale_log2 * 16777216.f * __uint_as_float((unsigned)(e - 14) << 23);
        qback[r] = of_columns(back);
        qsum[r][0] = of_columns(sum[0] * P.scale_log2);
        qsum[r][1] = of_columns(sum[1] * P.scale_log2);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          const uint2 w = mine ? *reinterpret_cast<const uint2 *>(row + 16 * i + 4 * t) : make_uint2(0u, 0u);
          const float2 x = two<T>(w.x), y = two<T>(w.y);
          qf[i][r][0] = Mma<__half>::pack(x.x * f, x.y * f);
          qf[i][r][1] = Mma<__half>::pack(y.x * f * 0.0625f, y.y * f * 0.0625f);        // meets 16 times the code
        }
      }
    };
    auto load_q16 = [&]() {
#pragma unroll
      for (int r = 0; r < NQ; ++r)
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          const T *row = qb + (g + 8 * r) * D + 16 * i + 2 * t;
          qf[i][r][0] = g + 8 * r < P.G ? *reinterpret_cast<const unsigned *>(row) : 0u;
          qf[i][r][1] = g + 8 * r < P.G ? *reinterpret_cast<const unsigned *>(row + 8) : 0u;
        }
    };
    // output: rows (channels) g and g + 8 of 16, columns (queries) 2t, 2t+1 of 8.  Beside 4-bit tiles rows g are in units of
    // 2^-24 and rows g + 8 of 2^-20.
    float oacc[MT][NQ][4];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int r = 0; r < NQ; ++r) oacc[i][r][0] = oacc[i][r][1] = oacc[i][r][2] = oacc[i][r][3] = 0.f;
    float2 omin[NQ][2] = {};                   // sums of weight * minimum over this lane's rows, for its two queries (+8)
    float2 m[NQ], l[NQ] = {};                  // reference of the weights (log2), and their sum over this lane's rows
    float2 up[NQ][2];                          // the power of two that the output of either half is held times, beside 4-bit tiles
#pragma unroll
    for (int r = 0; r < NQ; ++r) {
      m[r] = make_float2(kNothing, kNothing);
      up[r][0] = up[r][1] = make_float2(kMostUpPower, kMostUpPower);
    }
    bool in4 = false, have_q = false;
    auto to_one = [&](float more) {            // from the units of 4-bit tiles to 1; more: of what the weights are taken times
#pragma unroll
      for (int r = 0; r < NQ; ++r) {
        l[r].x *= more; l[r].y *= more;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          omin[r][u].x *= more; omin[r][u].y *= more;
          const float d0 = __uint_as_float(0x7f000000u - __float_as_uint(up[r][u].x)) * more;      // more / up
          const float d1 = __uint_as_float(0x7f000000u - __float_as_uint(up[r][u].y)) * more;
#pragma unroll
          for (int i = u * (MT / 2); i < (u + 1) * (MT / 2); ++i) {
            oacc[i][r][0] = oacc[i][r][0] * 16777216.f * d0; oacc[i][r][1] = oacc[i][r][1] * 16777216.f * d1;
            oacc[i][r][2] = oacc[i][r][2] * 1048576.f * d0; oacc[i][r][3] = oacc[i][r][3] * 1048576.f * d1;
          }
        }
      }
    };
    auto over_rows = [&](float x) {            // the lanes that have the same columns
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
      return x;
    };
    // Scores beside 16-bit rows, the lane's largest of either column: the references move where any lane needs it.
    auto refer = [&](const float2 (&x)[NQ]) {
      bool move = false;
#pragma unroll
      for (int r = 0; r < NQ; ++r) move |= x[r].x > m[r].x + kTop || x[r].y > m[r].y + kTop;
      if (__any_sync(0xffffffffu, move)) {
#pragma unroll
        for (int r = 0; r < NQ; ++r) {
          const float n0 = over_rows(x[r].x), n1 = over_rows(x[r].y);
          const float t0 = n0 > m[r].x + kTop ? n0 - kReset : m[r].x, t1 = n1 > m[r].y + kTop ? n1 - kReset : m[r].y;
          const float c0 = exp2f(m[r].x - t0), c1 = exp2f(m[r].y - t1);
          m[r] = make_float2(t0, t1);
          l[r].x *= c0; l[r].y *= c1;
          omin[r][0].x *= c0; omin[r][0].y *= c1;
          omin[r][1].x *= c0; omin[r][1].y *= c1;
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            oacc[i][r][0] *= c0; oacc[i][r][1] *= c1;
            oacc[i][r][2] *= c0; oacc[i][r][3] *= c1;
          }
        }
      }
    };
    // The same beside 4-bit rows, 8 N of them: a query's reference follows its largest score, and the power of two of a half of its output
    // the largest weight * scale of that half, each for itself: a row with a large scale but no weight holds nothing down, nor does
    // the other half.  The largest weight is a power of two then, and its product exact, which where few rows have most of the
    // weight is most of the accuracy (references that moved in whole steps: errors of 820 rows five times as large).
    constexpr int JJ = NQ == 1 ? 2 : 1, N = 2 * JJ;
    auto refer4 = [&](int r, const float2 (&x)[N], const unsigned (&vp)[N][2]) {
      float2 n = x[0];
#pragma unroll
      for (int b8 = 1; b8 < N; ++b8) n = make_float2(fmaxf(n.x, x[b8].x), fmaxf(n.y, x[b8].y));
      auto moved = [&](float top, float was) { return top > was + (kTop - kDown) ? top - (kReset - kDown) : was; };
      const float2 to = make_float2(moved(over_rows(n.x), m[r].x), moved(over_rows(n.y), m[r].y));
      const float2 by = make_float2(to.x - m[r].x, to.y - m[r].y), c = make_float2(exp2f(-by.x), exp2f(-by.y));
      m[r] = to;
      l[r].x *= c.x; l[r].y *= c.y;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        omin[r][u].x *= c.x; omin[r][u].y *= c.y;
        float2 z = make_float2(-INFINITY, -INFINITY);                    // weight * scale < 2^z
#pragma unroll
        for (int b8 = 0; b8 < N; ++b8) {
          const float e = (float)((int)((__float_as_uint(two<T>(vp[b8][u]).x) >> 23) & 255u) - 126);
          z = make_float2(fmaxf(z.x, x[b8].x - to.x + e), fmaxf(z.y, x[b8].y - to.y + e));
        }
        // `was`: the exponent of `up` if the output so far stayed as it is
        auto held = [&](float most, float was) { was = fminf(was, kMostUp); return floorf(most + was > kTop ? kReset - most : was); };
        auto exponent = [](float x) { return (float)((int)(__float_as_uint(x) >> 23) - 127); };
        auto power = [](float e) { return __uint_as_float((unsigned)((int)e + 127) << 23); };
        const float2 was = make_float2(exponent(up[r][u].x) + by.x, exponent(up[r][u].y) + by.y);
        const float2 e = make_float2(held(over_rows(z.x), was.x), held(over_rows(z.y), was.y));
        const float2 f = make_float2(exp2f(e.x - was.x), exp2f(e.y - was.y));
        up[r][u] = make_float2(power(e.x), power(e.y));
#pragma unroll
        for (int i = u * (MT / 2); i < (u + 1) * (MT / 2); ++i) {
          oacc[i][r][0] *= f.x; oacc[i][r][1] *= f.y;
          oacc[i][r][2] *= f.x; oacc[i][r][3] *= f.y;
        }
      }
    };
    // 16 JJ rows of a 4-bit tile at shared address `tile_p`, from its row `first` on.
    // (With 16 query heads the registers are enough for 16 rows at a time.)
    // `visible`: a bit for each of them.
    auto rows4 = [&](unsigned tile_p, int first, unsigned visible) {
      // operand row g of 8 is row `mine` of the tile's 8, so that the values' lanes (rows t and 7 - t) meet fewer bank conflicts
      const int mine = (g & 1) ? 7 - (g >> 1) : (g >> 1);
      const unsigned kc = tile_p + (unsigned)((first + mine) * S::kCode + t * (D / 8));
      const unsigned kpar = tile_p + (unsigned)(2 * kRows4 * S::kCode + (first + mine) * S::kParam);
      float2 sc[NQ][N];                                                         // [8 rows]: the lane's row, its two queries
      unsigned vp[N][2];                                                        // (scale, minimum) of its values, [half]
#pragma unroll
      for (int jj = 0; jj < JJ; ++jj) {                                     // 16 rows: operand rows g and g + 8
        unsigned w[2][D / 32];
        uint2 kp[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const unsigned off = (unsigned)(16 * jj + 8 * c);
          if (D == 128) {
            const uint4 x = lds128(kc + off * S::kCode);
            w[c][0] = x.x; w[c][1] = x.y; w[c][D / 32 - 2] = x.z; w[c][D / 32 - 1] = x.w;
          } else {
            const uint2 x = lds64(kc + off * S::kCode);
            w[c][0] = x.x; w[c][1] = x.y;
          }
          kp[c] = lds64(kpar + off * S::kParam);
          const uint2 v = lds64(kpar + (kRows4 + off) * S::kParam);
          vp[2 * jj + c][0] = v.x; vp[2 * jj + c][1] = v.y;
        }
        float acc[2][NQ][4];
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
          for (int o = 0; o < 2; ++o) {
            const unsigned x = o ? w[0][i] >> 8 : w[0][i], y = o ? w[1][i] >> 8 : w[1][i];
            const unsigned a[4] = {x & 0x000f000fu, y & 0x000f000fu, x & 0x00f000f0u, y & 0x00f000f0u};
            const int sl = 2 * i + o, u = i / (D / 64);
#pragma unroll
            for (int r = 0; r < NQ; ++r) {
              if (o == 0 && i % (D / 64) == 0) mma_first<__half>(acc[u][r], a, qf[sl][r][0], qf[sl][r][1]);
              else Mma<__half>::run(acc[u][r], a, qf[sl][r][0], qf[sl][r][1]);
            }
          }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int b8 = 2 * jj + c;
          const float2 k0 = two<T>(kp[c].x), k1 = two<T>(kp[c].y);
#pragma unroll
          for (int r = 0; r < NQ; ++r) {
            float2 x;
            x.x = fmaf(fmaf(k1.x, acc[1][r][2 * c], k0.x * acc[0][r][2 * c]), qback[r].x, fmaf(k1.y, qsum[r][1].x, k0.y * qsum[r][0].x));
            x.y = fmaf(fmaf(k1.x, acc[1][r][2 * c + 1], k0.x * acc[0][r][2 * c + 1]), qback[r].y, fmaf(k1.y, qsum[r][1].y, k0.y * qsum[r][0].y));
            sc[r][b8] = x;
          }
        }
      }
      if (visible != (JJ == 2 ? 0xffffffffu : 0xffffu)) {                  // seldom: an end of the rows or of the window
#pragma unroll
        for (int b8 = 0; b8 < 2 * JJ; ++b8)
          if (!((visible >> (8 * b8 + mine)) & 1u)) {
            vp[b8][0] = vp[b8][1] = 0u;
#pragma unroll
            for (int r = 0; r < NQ; ++r) sc[r][b8] = make_float2(-INFINITY, -INFINITY);
          }
      }
      // Weights by the references as they are.  That none passes its bound shows in their sums and products; only where one does is the
      // largest looked for.
      unsigned pw[NQ][2][N];                                                    // [half][8 rows]: weight * scale as the right operand
#pragma unroll
      for (int r = 0; r < NQ; ++r) {
        float2 sum, with_min[2];
        auto weigh = [&]() {                                               // -> did a sum or a product pass
          sum = make_float2(0.f, 0.f);
          with_min[0] = omin[r][0];
          with_min[1] = omin[r][1];
          unsigned most = 0u;                                              // largest products of both queries, by their bits (a NaN's are larger)
#pragma unroll
          for (int b8 = 0; b8 < N; ++b8) {
            const float2 x = __fadd2_rn(sc[r][b8], make_float2(-m[r].x, -m[r].y));
            const float2 p = make_float2(exp2_fast(x.x), exp2_fast(x.y));
            sum = __fadd2_rn(sum, p);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const float2 v = two<T>(vp[b8][u]), w = __fmul2_rn(p, up[r][u]);
              pw[r][u][b8] = Mma<__half>::pack(w.x * v.x, w.y * v.x);
              with_min[u].x = fmaf(p.x, v.y, with_min[u].x);
              with_min[u].y = fmaf(p.y, v.y, with_min[u].y);
            }
            most = __vimax3_u16x2(most, pw[r][0][b8], pw[r][1][b8]);
          }
          // 2^14 as a half number; eight weights that no reference has to move for sum to no more than 2^-17
          return !(sum.x + sum.y <= 0x1p-16f) || (most & 0xffffu) > 0x7400u || (most >> 16) > 0x7400u;
        };
        if (__any_sync(0xffffffffu, weigh())) {
          refer4(r, sc[r], vp);
          weigh();
        }
        l[r] = __fadd2_rn(l[r], sum);
        omin[r][0] = with_min[0];
        omin[r][1] = with_min[1];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int b8 = 0; b8 < N; ++b8) pw[r][u][b8] = transposed(pw[r][u][b8]);
      }
      // values: run g of the rows t and 7 - t of every 8; nibble n of a run is channel 8 n + g
      const unsigned va = tile_p + (unsigned)((kRows4 + first) * S::kCode + g * (D / 16));
      const unsigned v0 = va + (unsigned)(t * S::kCode), v1 = va + (unsigned)((7 - t) * S::kCode);
#pragma unroll
      for (int jj = 0; jj < JJ; ++jj) {
        unsigned w[2][2][D / 64];                                          // [8 rows][column][word]
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const unsigned p = (c ? v1 : v0) + (unsigned)((16 * jj + 8 * j) * S::kCode);
            if (D == 128) {
              const uint2 x = lds64(p);
              w[j][c][0] = x.x; w[j][c][D / 64 - 1] = x.y;
            } else {
              w[j][c][0] = lds32(p);
            }
          }
#pragma unroll
        for (int i = 0; i < D / 64; ++i)
#pragma unroll
          for (int hw = 0; hw < 2; ++hw) {                                 // nibbles 0..3, 4..7 of the word, of two rows side by side
            unsigned x = __byte_perm(w[0][0][i], w[0][1][i], hw ? 0x7632 : 0x5410);
            unsigned y = __byte_perm(w[1][0][i], w[1][1][i], hw ? 0x7632 : 0x5410);
#pragma unroll
            for (int o = 0; o < 2; ++o) {
              const int mt = 4 * i + 2 * hw + o, u = mt / (MT / 2);
              const unsigned a[4] = {x & 0x000f000fu, x & 0x00f000f0u, y & 0x000f000fu, y & 0x00f000f0u};
#pragma unroll
              for (int r = 0; r < NQ; ++r) Mma<__half>::run(oacc[mt][r], a, pw[r][u][2 * jj], pw[r][u][2 * jj + 1]);
              x >>= 8;
              y >>= 8;
            }
          }
      }
    };
    // 16 rows of a 16-bit tile
    auto rows16 = [&](unsigned sb, int first, int row0, int end) {
      const bool whole = row0 >= 0 && row0 + 16 <= end && (row0 + 16 <= s.low || row0 >= s.high);
      auto sees = [&](int row) { return whole || (row < end && (row < s.low || row >= s.high)); };
      float acc[NQ][4];
      const int mi = lane >> 3;
      // 16-byte chunk c of row r, as the swizzled boxes of 64 channels leave it
      auto chunk_at = [&](int r, int c) { return (unsigned)((c >> 3) * S::kBox + r * 128 + (((c & 7) ^ (r & 7)) << 4)); };
#pragma unroll
      for (int kk = 0; kk < MT; ++kk) {
        unsigned a[4];
        ldmatrix_x4(sb + chunk_at(first + (mi & 1) * 8 + (lane & 7), 2 * kk + (mi >> 1)), a);
#pragma unroll
        for (int r = 0; r < NQ; ++r) {
          if (kk == 0) mma_first<T>(acc[r], a, qf[kk][r][0], qf[kk][r][1]);
          else Mma<T>::run(acc[r], a, qf[kk][r][0], qf[kk][r][1]);
        }
      }
      float2 sc[NQ][2], top[NQ];
      unsigned keep[2] = {0xffffffffu, 0xffffffffu};                       // bits of the rows 2t, 2t+1 (+ 8) that have weight
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (!sees(row0 + 8 * j + 2 * t)) keep[j] &= 0xffff0000u;
        if (!sees(row0 + 8 * j + 2 * t + 1)) keep[j] &= 0x0000ffffu;
        const bool vis = sees(row0 + 8 * j + g);
#pragma unroll
        for (int r = 0; r < NQ; ++r)
          sc[r][j] = vis ? make_float2(acc[r][2 * j] * P.scale_log2, acc[r][2 * j + 1] * P.scale_log2) : make_float2(-INFINITY, -INFINITY);
      }
#pragma unroll
      for (int r = 0; r < NQ; ++r) top[r] = make_float2(fmaxf(sc[r][0].x, sc[r][1].x), fmaxf(sc[r][0].y, sc[r][1].y));
      refer(top);
      unsigned pw[NQ][2];
#pragma unroll
      for (int r = 0; r < NQ; ++r) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float2 x = __fadd2_rn(sc[r][j], make_float2(-m[r].x, -m[r].y));
          const float2 p = make_float2(exp2_fast(x.x), exp2_fast(x.y));
          l[r] = __fadd2_rn(l[r], p);
          pw[r][j] = transposed(Mma<T>::pack(p.x, p.y));
        }
      }
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        unsigned v[4];
        ldmatrix_x4_trans(sb + (D / 64) * S::kBox + chunk_at(first + (mi >> 1) * 8 + (lane & 7), 2 * i + (mi & 1)), v);
        // rows without weight may hold anything, and 0 x NaN is NaN
        const unsigned a[4] = {v[0] & keep[0], v[1] & keep[0], v[2] & keep[1], v[3] & keep[1]};
#pragma unroll
        for (int r = 0; r < NQ; ++r) Mma<T>::run(oacc[i][r], a, pw[r][0], pw[r][1]);
      }
    };

    const int lt0 = (int)(ti - at), cnt = (int)(seg_end - ti), team0 = n % kTeams;
    int i = (team + kTeams - team0) % kTeams;
    if (i < cnt) {                             // the queries, while the first tile is on its way
      if (Q4 && lt0 + i < s.main) { load_q4(); in4 = true; }
      else { load_q16(); have_q = true; }
    }
    for (; i < cnt && !failed; i += kTeams) {
      const int st = (n + i) % kStages;
      if (!mbar::wait_warp(&full[st], (unsigned)((n + i) / kStages) & 1u)) {
        // a load did not arrive in time (for any lane): say so and report an empty share
        failed = true;
        if (lane == 0) atomicOr(P.status, FC_DEV_FLAG_TIMEOUT);
        break;
      }
      const TileAt ta = tile_at<Q4>(s, lt0 + i);
      const int end = ta.tail ? s.n_main + s.n_tail : s.n_main;
      if (Q4 && !ta.tail) {
        if constexpr (Q4) {
#pragma unroll
          for (int part = 0; part < 2; part += JJ) {
            const int first = 32 * (warp % kTeam) + 16 * part, row0 = ta.row + first;
            const unsigned there = bits_below(end - row0) & ~bits_below(-row0);
            const unsigned visible = there & (bits_below(s.low - row0) | ~bits_below(s.high - row0)) & (JJ == 2 ? 0xffffffffu : 0xffffu);
            if (visible) rows4(sbase + (unsigned)(st * S::kStage), first, visible);
          }
        }
      } else {
        // two of the team's four warps, the others on its next tile
        const int first = 16 * (warp & 1), row0 = ta.row + first;
        if ((((warp % kTeam) >> 1) == (((n + i) / kTeams) & 1)) && row0 < end && (row0 < s.low || row0 + 15 >= s.high)) {
          if (!have_q) {                                                   // kept rows come before the tail: never back
            load_q16();
            to_one(kDownPower);
#pragma unroll
            for (int r = 0; r < NQ; ++r) m[r] = make_float2(m[r].x - kDown, m[r].y - kDown);
            have_q = true;
            in4 = false;
          }
          rows16(sbase + (unsigned)(st * S::kStage), first, row0, end);
        }
      }
      __syncwarp();
      if (lane == 0) mbar::arrive(&empty[st]);                             // this warp is through with the stage
    }
    n += cnt;
    ti = seg_end;
    if (in4) to_one(1.f);
    if (failed) {
#pragma unroll
      for (int r = 0; r < NQ; ++r) {
        m[r] = make_float2(kNothing, kNothing);
        l[r] = omin[r][0] = omin[r][1] = make_float2(0.f, 0.f);
      }
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int r = 0; r < NQ; ++r) oacc[i][r][0] = oacc[i][r][1] = oacc[i][r][2] = oacc[i][r][3] = 0.f;
    }

    // Only now: blocks of the second kernel that wait on this one's SM take issue slots from it (the step over 189810 rows of 4
    // heads 35 -> 32 us).
    if (seg_end >= hi) asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    // merge the warps of the teams that had a tile: `parts` of them, from warp `warp0` on
    const int parts = kTeam * (cnt < kTeams ? cnt : kTeams), warp0 = kTeam * team0;
    const bool part = (warp + kWarps - warp0) % kWarps < parts;
    if (ti0 > lo) consumers_sync();                                        // the merge buffer is free again
#pragma unroll
    for (int r = 0; r < NQ; ++r) {
      if (!part) break;
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {
        l[r].x += __shfl_xor_sync(0xffffffffu, l[r].x, o);
        l[r].y += __shfl_xor_sync(0xffffffffu, l[r].y, o);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          omin[r][u].x += __shfl_xor_sync(0xffffffffu, omin[r][u].x, o);
          omin[r][u].y += __shfl_xor_sync(0xffffffffu, omin[r][u].y, o);
        }
      }
      float *w = mo + ((size_t)warp * kHeads + 8 * r) * S::kStride;
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        w[(2 * t) * S::kStride + 16 * i + g] = oacc[i][r][0];
        w[(2 * t + 1) * S::kStride + 16 * i + g] = oacc[i][r][1];
        w[(2 * t) * S::kStride + 16 * i + 8 + g] = oacc[i][r][2];
        w[(2 * t + 1) * S::kStride + 16 * i + 8 + g] = oacc[i][r][3];
      }
      if (g == 0) {
        const int q = warp * kHeads + 8 * r + 2 * t;
        mml[q] = make_float2(m[r].x, l[r].x);
        mml[q + 1] = make_float2(m[r].y, l[r].y);
        mmin[q] = make_float2(omin[r][0].x, omin[r][1].x);
        mmin[q + 1] = make_float2(omin[r][0].y, omin[r][1].y);
      }
    }
    consumers_sync();
    const int i0 = line::share_of(at, line_len, nb), i1 = line::share_of(at + s.tiles - 1, line_len, nb);
    const size_t slot = ((size_t)blk + (size_t)h * P.B + b) * P.G;
    constexpr int C = D / 32;                                              // channels per lane
    for (int r = warp; r < P.G; r += kWarps) {                             // a warp per query head
      float mm = kNothing, ll = 0.f, o[C];
      for (int k = 0, w = warp0; k < parts; ++k, w = w + 1 == kWarps ? 0 : w + 1) mm = fmaxf(mm, mml[w * kHeads + r].x);
#pragma unroll
      for (int c = 0; c < C; ++c) o[c] = 0.f;
#pragma unroll 4
      for (int k = 0, w = warp0; k < parts; ++k, w = w + 1 == kWarps ? 0 : w + 1) {
        const float2 ml = mml[w * kHeads + r], mn = mmin[w * kHeads + r];
        const float f = exp2f(ml.x - mm), add = lane < 16 ? mn.x : mn.y;
        const float *src = mo + ((size_t)w * kHeads + r) * S::kStride + C * lane;
#pragma unroll
        for (int c = 0; c < C; ++c) o[c] = fmaf(src[c] + add, f, o[c]);
        ll = fmaf(ml.y, f, ll);
      }
      if (i0 == i1) {
        const float inv = 1.f / ll;                                        // 0 only of scores that are all minus infinity: 0 / 0
        T *out = static_cast<T *>(P.out) + ((size_t)b * P.Hq + (size_t)h * P.G + r) * D + C * lane;
#pragma unroll
        for (int c = 0; c < C; c += 2) *reinterpret_cast<unsigned *>(out + c) = Mma<T>::pack(o[c] * inv, o[c + 1] * inv);
      } else {
        float *dst = P.part_o + (slot + r) * D + C * lane;
#pragma unroll
        for (int c = 0; c < C; c += 2) *reinterpret_cast<float2 *>(dst + c) = make_float2(o[c], o[c + 1]);
        if (lane == 0) P.part_ml[slot + r] = make_float2(mm, ll);
      }
    }
    if (blk == i0 && tid == 0) P.span[(size_t)h * P.B + b] = make_int2(i0, i1);
  }
}

// out of a sequence that several blocks share: their results rescaled to the common reference and divided by the common sum.
// Block i's result of sequence (h, b) is in slot i + h*B + b (both only ever advance along the line, so slots do not collide).
// A block does `width` channels of a query head, all of them or, where there are few heads, a part; a thread does one, of every
// (128 / width)th result: 16 of them are on their way at once, next to the references and sums, which every thread of the block
// loads one or two of.
template <typename T, int D>
__global__ void __launch_bounds__(128)
k_decode_ex_combine(const __grid_constant__ ExParams P, int width) {
  constexpr int kThreadsC = 128, kAhead = 16;
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  __shared__ float weight[2 * kThreadsC], part[kThreadsC], top[4], sum[4];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int b = blockIdx.x / P.Hq, hq = blockIdx.x - b * P.Hq, h = hq / P.G, r = hq - h * P.G;
  const int c = tid & (width - 1), first = tid / width, groups = kThreadsC / width;
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  const int2 span = __ldcg(P.span + (size_t)h * P.B + b);
  if (span.y <= span.x) return;                                            // no rows, or finished by its only block
  const int cnt = span.y - span.x + 1;
  const size_t slot0 = ((size_t)span.x + (size_t)h * P.B + b) * P.G + r;
  const float *src = P.part_o + slot0 * D + blockIdx.y * width + c;
  const unsigned step = (unsigned)(P.G * D);
  float v[kAhead];
#pragma unroll
  for (int a = 0; a < kAhead; ++a) v[a] = first + groups * a < cnt ? __ldcg(src + (unsigned)(first + groups * a) * step) : 0.f;
  float2 ml[2];
#pragma unroll
  for (int e = 0; e < 2; ++e)
    ml[e] = tid + kThreadsC * e < cnt ? __ldcg(P.part_ml + slot0 + (unsigned)(tid + kThreadsC * e) * (unsigned)P.G) : make_float2(kNothing, 0.f);
  float m = fmaxf(ml[0].x, ml[1].x);
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (lane == 0) top[warp] = m;
  __syncthreads();
  m = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
  float l = 0.f;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const float f = exp2_fast(ml[e].x - m);
    weight[tid + kThreadsC * e] = f;
    l = fmaf(f, ml[e].y, l);
  }
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
  if (lane == 0) sum[warp] = l;
  __syncthreads();
  float acc = 0.f;
#pragma unroll 1
  for (int i = first;;) {
#pragma unroll
    for (int a = 0; a < kAhead; ++a)
      if (i + groups * a < cnt) acc = fmaf(v[a], weight[i + groups * a], acc);
    i += groups * kAhead;
    if (i >= cnt) break;
#pragma unroll
    for (int a = 0; a < kAhead; ++a) v[a] = i + groups * a < cnt ? __ldcg(src + (unsigned)(i + groups * a) * step) : 0.f;
  }
  part[tid] = acc;
  __syncthreads();
  if (first != 0) return;
  for (int k = 1; k < groups; ++k) acc += part[tid + k * width];
  l = (sum[0] + sum[1]) + (sum[2] + sum[3]);
  const float inv = 1.f / l;
  static_cast<T *>(P.out)[((size_t)b * P.Hq + hq) * D + blockIdx.y * width + c] = Mma<T>::from_float(acc * inv);
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
// Tiles of 32 rows x 64 channels of one head, rows 128 bytes wide in shared memory, 128-byte swizzle.
fc_status encode_rows(CUtensorMap *m, CUtensorMapDataType dt, int rank, const void *base, const cuuint64_t *dims, const cuuint64_t *strides) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return FC_ERR_CUDA;
  const cuuint32_t box[4] = {64, 1, (cuuint32_t)kRows16, 1}, ones[4] = {1, 1, 1, 1};
  return fn(m, dt, (cuuint32_t)rank, const_cast<void *>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? FC_OK : FC_ERR_INTERNAL;
}

fc_status check_ex(const fc_handle *h, const fc_decode_args *a, const fc_decode_options *o) {
  if (!h || !a || !o || !a->q || !a->offsets) return FC_ERR_INVALID_ARG;
  if (a->batch < 1 || a->num_heads < 1 || a->num_q_heads < 1 || a->max_rows < 0 || o->window < 0 || o->sinks < 0) return FC_ERR_INVALID_ARG;
  if (a->dtype != FC_F16 && a->dtype != FC_BF16) return FC_ERR_UNSUPPORTED;
  if (a->head_dim != 64 && a->head_dim != 128) return FC_ERR_UNSUPPORTED;
  if (a->num_q_heads % a->num_heads != 0 || a->num_q_heads / a->num_heads > 16) return FC_ERR_UNSUPPORTED;
  if (o->cache4) {
    const fc_status s = cache4::check(o->cache4);
    if (s != FC_OK) return s;
    if (o->cache4->dtype != a->dtype || o->cache4->num_heads != a->num_heads || o->cache4->head_dim != a->head_dim) return FC_ERR_INVALID_ARG;
  } else {
    if (!a->cache_k || !a->cache_v || a->cache_rows < 1) return FC_ERR_INVALID_ARG;
    if (((uintptr_t)a->cache_k & 15) || ((uintptr_t)a->cache_v & 15)) return FC_ERR_INVALID_ARG;
    if (a->cache_rows > 0x7fffffffll - 4096) return FC_ERR_UNSUPPORTED;
  }
  if (a->max_rows > 0x7fffffffll - 4096 || a->batch > 65535 || a->num_heads > 65535 ||
      (int64_t)a->batch * a->num_q_heads > 0x7fffffffll)
    return FC_ERR_UNSUPPORTED;
  if ((uintptr_t)a->q & 15) return FC_ERR_INVALID_ARG;
  if (a->tail_k || a->tail_v || a->tail_len) {
    if (!a->tail_k || !a->tail_v || !a->tail_len || a->tail_capacity < 1) return FC_ERR_INVALID_ARG;
    if (((uintptr_t)a->tail_k & 15) || ((uintptr_t)a->tail_v & 15)) return FC_ERR_INVALID_ARG;
    // a sequence's rows, kept ones and tail, are counted in 32 bits
    if ((o->cache4 ? o->cache4->capacity_rows : a->cache_rows) + a->tail_capacity > 0x7fffffffll - 4096) return FC_ERR_UNSUPPORTED;
  }
  return FC_OK;
}

struct ExPlan {
  int nb;
  size_t off_ml, off_span, total;
};

ExPlan plan_ex(const fc_handle *h, const fc_decode_args *a, const fc_decode_options *o) {
  ExPlan p;
  // one block per SM (the ring takes most of its shared memory), or as many as there can be tiles: of what a sequence of
  // max_rows rows shows, however it splits into kept rows, tail, sinks and window (each part's ends may cut a tile)
  const long long size = o->cache4 ? kRows4 : kRows16;
  long long rows = a->max_rows;
  if (o->window > 0 && (long long)o->window + o->sinks < rows) rows = (long long)o->window + o->sinks;
  const long long per = (rows + size - 1) / size + 3 + (a->tail_k ? (a->tail_capacity < rows ? a->tail_capacity : rows) / kRows16 + 3 : 0);
  const long long units = (long long)a->batch * a->num_heads, tiles = units * per;
  p.nb = h->num_sms < kMaxBlocks ? h->num_sms : kMaxBlocks;
  if (tiles < p.nb) p.nb = (int)tiles;
  const size_t slots = (size_t)(p.nb + units) * (size_t)(a->num_q_heads / a->num_heads);
  p.off_ml = (slots * a->head_dim * sizeof(float) + 255) & ~(size_t)255;
  p.off_span = p.off_ml + ((slots * sizeof(float2) + 255) & ~(size_t)255);
  p.total = p.off_span + (((size_t)units * sizeof(int2) + 255) & ~(size_t)255);
  return p;
}

template <typename T, int D, bool Q4, int NQ>
fc_status launch_ex(fc_handle *h, const ExParams &P, const ExMaps &M, cudaStream_t st) {
  using S = Geo<D, Q4, NQ>;
  static_assert(S::kStages >= 4 && S::kSmem <= 227 * 1024 - 512, "shared memory");
  constexpr unsigned bit = 1u << ((std::is_same<T, __half>::value ? 1 : 0) + (D == 128 ? 2 : 0) + (Q4 ? 4 : 0) + (NQ == 2 ? 8 : 0));
  if (!(h->forms_ready & bit)) {           // once per handle
    FC_CUDA_TRY(cudaFuncSetAttribute(k_decode_ex<T, D, Q4, NQ>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmem));
    h->forms_ready |= bit;
  }
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3(P.nb);
  lc.blockDim = dim3(kThreads);
  lc.dynamicSmemBytes = S::kSmem;
  lc.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  lc.attrs = at;
  lc.numAttrs = 1;
  if (cudaLaunchKernelEx(&lc, k_decode_ex<T, D, Q4, NQ>, P, M) != cudaSuccess) {
    cudaGetLastError();
    return FC_ERR_CUDA;
  }
  fc_status s = fc_after_launch(h);
  if (s != FC_OK) return s;
  static_assert(kMaxBlocks <= 256, "the second kernel's threads take two results each");
  // a head's channels in parts as long as there is an SM for each
  int width = D;
  while (width > 32 && 2ll * P.B * P.Hq * (D / width) <= h->num_sms) width /= 2;
  lc.gridDim = dim3((unsigned)(P.B * P.Hq), (unsigned)(D / width));
  lc.blockDim = dim3(128);
  lc.dynamicSmemBytes = 0;
  if (cudaLaunchKernelEx(&lc, k_decode_ex_combine<T, D>, P, width) != cudaSuccess) {
    cudaGetLastError();
    return FC_ERR_CUDA;
  }
  return fc_after_launch(h);
}

template <typename T, int D>
fc_status launch_of(fc_handle *h, const ExParams &P, const ExMaps &M, bool q4, cudaStream_t st) {
  if (q4) return P.G <= 8 ? launch_ex<T, D, true, 1>(h, P, M, st) : launch_ex<T, D, true, 2>(h, P, M, st);
  return P.G <= 8 ? launch_ex<T, D, false, 1>(h, P, M, st) : launch_ex<T, D, false, 2>(h, P, M, st);
}

}  // namespace

extern "C" size_t fc_decode_workspace_bytes_ex(const fc_handle *h, const fc_decode_args *a, const fc_decode_options *opt) {
  if (!opt) return fc_decode_workspace_bytes(h, a);
  if (check_ex(h, a, opt) != FC_OK) return 0;
  return plan_ex(h, a, opt).total;
}

extern "C" fc_status fc_decode_attention_ex(fc_handle *h, const fc_decode_args *a, const fc_decode_options *opt, void *out,
                                            void *workspace, size_t workspace_bytes, fc_stream stream) {
  if (!opt) return fc_decode_attention(h, a, out, workspace, workspace_bytes, stream);
  fc_status s = check_ex(h, a, opt);
  if (s != FC_OK) return s;
  if (!out || ((uintptr_t)out & 15)) return FC_ERR_INVALID_ARG;
  const ExPlan pl = plan_ex(h, a, opt);
  if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < pl.total) return FC_ERR_WORKSPACE;
  FcDeviceGuard on(h->device);
  if (!on.ok) return FC_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if ((s = fc_flush_pending(h, st)) != FC_OK) return s;
  const int D = a->head_dim;
  const CUtensorMapDataType dt = a->dtype == FC_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  const cuuint64_t head_b = (cuuint64_t)D * 2, row_b = (cuuint64_t)a->num_heads * head_b;
  ExMaps M = {};
  if (!opt->cache4) {
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)a->num_heads, (cuuint64_t)a->cache_rows}, str[2] = {head_b, row_b};
    if ((s = encode_rows(&M.k, dt, 3, a->cache_k, dims, str)) != FC_OK) return s;
    if ((s = encode_rows(&M.v, dt, 3, a->cache_v, dims, str)) != FC_OK) return s;
  }
  if (a->tail_k) {
    const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)a->num_heads, (cuuint64_t)a->tail_capacity, (cuuint64_t)a->batch};
    const cuuint64_t str[3] = {head_b, row_b, row_b * (cuuint64_t)a->tail_capacity};
    if ((s = encode_rows(&M.tk, dt, 4, a->tail_k, dims, str)) != FC_OK) return s;
    if ((s = encode_rows(&M.tv, dt, 4, a->tail_v, dims, str)) != FC_OK) return s;
  }
  char *ws = static_cast<char *>(workspace);
  ExParams P = {};
  P.q = a->q;
  P.out = out;
  P.offsets = reinterpret_cast<const long long *>(a->offsets);
  P.tail_len = a->tail_len;
  P.part_o = reinterpret_cast<float *>(ws);
  P.part_ml = reinterpret_cast<float2 *>(ws + pl.off_ml);
  P.span = reinterpret_cast<int2 *>(ws + pl.off_span);
  P.status = h->status_word;
  P.B = a->batch;
  P.H = a->num_heads;
  P.Hq = a->num_q_heads;
  P.G = a->num_q_heads / a->num_heads;
  P.nb = pl.nb;
  P.tail_cap = a->tail_k ? a->tail_capacity : 0;
  P.has_tail = a->tail_k ? 1 : 0;
  P.window = opt->window;
  P.sinks = opt->sinks;
  P.scale_log2 = (float)(1.4426950408889634 / sqrt((double)D));
  P.cache_rows = opt->cache4 ? opt->cache4->capacity_rows : a->cache_rows;
  if (opt->cache4) {
    P.ck = static_cast<const unsigned char *>(opt->cache4->codes_k);
    P.cv = static_cast<const unsigned char *>(opt->cache4->codes_v);
    P.pk = static_cast<const unsigned char *>(opt->cache4->params_k);
    P.pv = static_cast<const unsigned char *>(opt->cache4->params_v);
  }
  const bool q4 = opt->cache4 != nullptr;
  if (a->dtype == FC_F16) return D == 128 ? launch_of<__half, 128>(h, P, M, q4, st) : launch_of<__half, 64>(h, P, M, q4, st);
  return D == 128 ? launch_of<__nv_bfloat16, 128>(h, P, M, q4, st) : launch_of<__nv_bfloat16, 64>(h, P, M, q4, st);
}
