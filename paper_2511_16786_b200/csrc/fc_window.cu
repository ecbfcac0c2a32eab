// Attention of a prefill with a sliding window and sinks (fc_window_attention).
//
// Query i of a sequence stands at p = n_k - n_q + i and sees the keys j <= p with j > p - window or j < sinks;
//     out = sum_j w_j v_j / sum_j w_j,   w_j = 2^(c s_j - m),  s = q k,  c = log2(e) / sqrt(d),  m a reference near max c s.
// 4 d operations per visible pair and query head.  The floor is the tensor cores' time; what bounds the kernel is the way of one
// tile's scores through it (128 keys at d = 128, in cycles: 2000 from scores to weights, of them 770 + 880 for exponentials, sums and
// rounding, the rest loads, stores and barriers; 1050 for the products that use them and make the next scores): two such tiles
// take turns, and the tensor cores have work for 2050 of some 3100 cycles.  32768 tokens of 28 heads over 4 (d = 128, bf16, window
// 4096): 1.77 ms back to back, where the GPU runs at its power limit, 1.58 ms alone (1020 and 1145 TFLOP/s).
//
//  * Queries are taken in tiles of 128 rows, two to a block (one at d = 64) that share one stream of key tiles (128 keys).  A row is a query of one
//    head; the query heads that share a KV head lie side by side in a tile (128 / G queries each), so keys are read once for
//    all of them and a tile spans few positions: little of a short window is masked away.
//  * Both products run on tcgen05: scores S = Q K^T from shared memory, outputs O += P V with the weights P (16 bits, written over
//    the scores they came from) out of tensor memory.  Two times (128 + d) columns hold S and O of both tiles.  Products are issued
//    in steps of 16 keys; those that no row of the tile sees are left out.
//  * Four warps per tile turn scores into weights, a thread a row (two threads a row: 1930 us, the barriers between them cost more
//    than the shorter way gains); one warp loads (TMA, a ring of key and value tiles), one issues the products, in an order
//    that works on one tile's products while the other tile's weights are made.  O += P V starts on the first 64 keys' weights.
//  * A quarter of the exponentials (an eighth at d = 64) are polynomials: the special-function units give 16 a cycle and SM, so a
//    128 x 128 tile would take 1024 cycles, as long as its two products at d = 128 (1770 us; an eighth 1797, three eighths 1807; at
//    d = 64 a ragged batch 41.3 us with an eighth, 42.4 with a quarter).
//  * The reference m moves only when a score passes it by 15 (fp16) or 24 (bf16), so the outputs are rarely rescaled, and weights stay
//    finite.  At d = 128 that none did is read off the sums of the weights; the largest score is only looked for where one did,
//    in a row's first tile and in tiles seen in part (1807 -> 1773 us; the polynomial's upper end, which that needs, takes 11 of them
//    back; at d = 64, where most tiles are such, 42 -> 46 us).
//  * Values that are not finite: a product takes 0 x NaN from keys that a row does not see.  Tiles that some row sees in part
//    are looked through by two more warps, which clear what is not finite and note the keys; rows that see such a key then
//    add weight x value by themselves.  (Tiles seen by every row need nothing; nor do keys, whose scores are masked.)
//  * Few blocks (a short chunk against a long cache): the key tiles of a block are split over several, whose outputs, maxima and
//    sums meet in a second kernel.
#include "fc_mbar.cuh"
#include "fc_tcgen05.cuh"
#include "fc_tile.cuh"

#include <math.h>

namespace {

using namespace tile;
using umma::after_sync;
using umma::before_sync;

constexpr int kTileRows = 128;                 // query rows, and keys, of a tile
constexpr int kSeqs = 64;                      // sequences described per launch (kernel-argument table)
constexpr int kValues = 4;                     // value tiles in the ring, at most
constexpr int kSplitMin = 4;                   // key tiles that a part of a split has at least
// How far, in powers of two, a score may pass its row's reference before that moves (and the outputs are rescaled), and how far it
// is above it then: a row's largest weight is 2^7..2^15 in fp16, 1..2^24 in bf16.  A half number below 2^-14 has fewer bits and one of
// 2^-25 is none, so a row loses 2^-32 of its largest weight at most for every key; with the largest at 1, 2^17 keys of 2^-25.5 each
// would be missing in the output but not in the sum.  (16384 tokens of 28 heads, fp16, d = 128, window 4096: 738 us with 1 and with
// 2^7, 747 with 2^8; with queries four times as long, whose references move more often, 900, 937 and 960.)  bf16 has fp32's exponents.
template <typename T> constexpr float kSlack = std::is_same<T, __half>::value ? 15.f : 24.f;
template <typename T> constexpr float kAbove = std::is_same<T, __half>::value ? 7.f : 0.f;
// What a sum may come to that shows none of its weights to have passed what the type holds.
template <typename T> constexpr float kMost = std::is_same<T, __half>::value ? 65504.f : 0x1p24f;

struct WinSeq { int q0, nq, k0, nk, item; };   // item: first of the sequence's, in blocks before splitting

struct WinParams {
  void *out;
  float *part_o;                               // [item][split][tile][128][D]
  float2 *part_ml;                             // [item][split][tile][128]
  int *status;
  const char *v;
  long long v_token, v_head;                   // bytes
  int seqs, H, Hq, G, per, tiles;              // per: queries of a tile; tiles: of a block
  int window, sinks, splits;
  float scale_log2;
  WinSeq seq[kSeqs];
};

struct WinMaps { CUtensorMap q, k, v; };

// NT query tiles to a block: two where they share what they read (128 channels); one, and two blocks to an SM, where there is room
// for it (64): a block's beginning and end then have another's products beside them (a ragged batch of 64 channels 47 -> 43 us).
template <int D>
struct WinShape {
  static constexpr int NT = D == 128 ? 2 : 1;
  static constexpr int kBox = 128 * 128;       // 128 rows of 64 channels
  static constexpr int kTileBytes = D / 64 * kBox;
  static constexpr int kSlots = 5;
  static constexpr size_t kSmem = (size_t)(NT + kSlots) * kTileBytes + 1024;
  static constexpr int kThreads = 128 * NT + 128;                  // weights; then four warps: loads, products, values, values
  // registers of a thread at launch, of the weights' and of the other threads
  static constexpr int kRegs = NT == 2 ? 168 : 128, kRegsRows = NT == 2 ? 208 : 200, kRegsRest = NT == 2 ? 88 : 56;
  static_assert(NT * kRegsRows + kRegsRest <= (NT + 1) * kRegs, "a register split has to come out of what was launched");
  static constexpr int kColumns = NT == 2 ? 512 : 256;             // tensor memory: S of tile q at 128 q, O behind them
};

template <int SLOTS>
struct WinShared {
  unsigned long long qfull, full[SLOTS], empty[SLOTS], scores[2], weights[2][2], halved[2], done[2];      // weights: of the first and the last 64 keys
  // by value tile, not by slot (an odd ring holds keys and values by turns in one slot): no more than kValues of them are in it
  unsigned long long clean[kValues];
  unsigned bad[kValues][4];                    // keys of the value tile with something not finite
  unsigned tmem;
};

// ---------------------------------------------------------------------------------------------------- tensor memory, 32 columns at a time
__device__ __forceinline__ void tm_ld32(unsigned addr, float *v) {
  unsigned *r = reinterpret_cast<unsigned *>(v);
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
               "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                 "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
                 "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
                 "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
               : "r"(addr));
}
__device__ __forceinline__ void tm_st32(unsigned addr, const unsigned *r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
               "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};\n"
               ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                 "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
                 "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
                 "r"(r[30]), "r"(r[31]) : "memory");
}
__device__ __forceinline__ void tm_st16(unsigned addr, const unsigned *r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};\n"
               ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                 "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tm_ld1(unsigned addr, unsigned &r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\n" : "=r"(r) : "r"(addr));
}
__device__ __forceinline__ void tm_st1(unsigned addr, unsigned r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};\n" ::"r"(addr), "r"(r) : "memory");
}
// Nothing that uses the registers is moved in front of the wait: it, and what follows it, names them.
__device__ __forceinline__ void tm_tie32(float *v) {
  asm volatile("" : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]),
                    "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), "+f"(v[16]), "+f"(v[17]), "+f"(v[18]),
                    "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]), "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]),
                    "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31]));
}
template <int N>
__device__ __forceinline__ void tm_wait_ld(float (&v)[N]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; i += 32) tm_tie32(v + i);
}
__device__ __forceinline__ void tm_wait_ld1(unsigned &r) { asm volatile("tcgen05.wait::ld.sync.aligned;\n" : "+r"(r)::"memory"); }
__device__ __forceinline__ void tm_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory"); }

// The left operand out of tensor memory.
__device__ __forceinline__ void mma_ts(unsigned lead, unsigned d, unsigned a, unsigned blo, unsigned bhi, unsigned idesc, unsigned add) {
  asm volatile("{\n .reg .pred p, q;\n .reg .b64 b;\n setp.ne.u32 q, %0, 0;\n setp.ne.u32 p, %6, 0;\n mov.b64 b, {%3, %4};\n"
               " @q tcgen05.mma.cta_group::1.kind::f16 [%1], [%2], b, %5, p;\n}\n"
               ::"r"(lead), "r"(d), "r"(a), "r"(blo), "r"(bhi), "r"(idesc), "r"(add) : "memory");
}

// The largest; NaN if any is.
__device__ __forceinline__ float max_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

__device__ __forceinline__ float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// Two powers of two without the special-function units, which give 16 a cycle and SM and are what the weights wait for: the
// nearest whole number into the exponent, the rest (at most half) by the polynomial of degree 4 with the smallest largest relative
// error on [-1/2, 1/2] (2.7e-6, found by linear programming over 4001 points).  From -126 on down it stays at 2^-126, so it is
// for tiles without masked scores; NaN becomes something above 2^127.  UP: from 127 on it stays at 2^127.  Without, x is below 128: the
// exponent would run into the sign, and what comes out be small or negative.
template <bool UP>
__device__ __forceinline__ float2 exp2_poly(float2 x) {
  x = make_float2(max_nan(x.x, -126.f), max_nan(x.y, -126.f));
  if (UP) x = make_float2(min_nan(x.x, 127.f), min_nan(x.y, 127.f));
  const float2 r = __fadd2_rn(x, make_float2(12582912.f, 12582912.f));                     // 1.5 * 2^23: the last bits are the number
  const float2 n = __fadd2_rn(r, make_float2(-12582912.f, -12582912.f));
  const float2 f = __ffma2_rn(n, make_float2(-1.f, -1.f), x);
  float2 p = make_float2(0.009569705463945866f, 0.009569705463945866f);
  p = __ffma2_rn(p, f, make_float2(0.05591819807887077f, 0.05591819807887077f));
  p = __ffma2_rn(p, f, make_float2(0.24024765193462372f, 0.24024765193462372f));
  p = __ffma2_rn(p, f, make_float2(0.6931217312812805f, 0.6931217312812805f));
  p = __ffma2_rn(p, f, make_float2(0.9999992251396179f, 0.9999992251396179f));
  return make_float2(__uint_as_float(__float_as_uint(p.x) + (__float_as_uint(r.x) << 23)),
                     __uint_as_float(__float_as_uint(p.y) + (__float_as_uint(r.y) << 23)));
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// ---------------------------------------------------------------------------------------------------- what a block works on
struct Span { int a, b; };                     // positions of a tile's first and last query (b < 0 or b < a: it sees nothing)
struct WinItem {
  WinSeq s;
  int h, first, item, split;                   // first: the block's first query; item: unsplit number
  Span at[2];
  int sink_tiles, win0, u0, u1;                // list of key tiles: [0, sink_tiles), then from win0 on; this block's part [u0, u1) of it
  __device__ __forceinline__ int key_tile(int u) const { return u < sink_tiles ? u : win0 + (u - sink_tiles); }
};

__device__ __forceinline__ WinItem find_item(const WinParams &P, int blk) {
  WinItem w;
  w.split = blk % P.splits;
  w.item = blk / P.splits;
  int i = 0;
  while (i + 1 < P.seqs && P.seq[i + 1].item <= w.item) ++i;
  w.s = P.seq[i];
  const int in = w.item - w.s.item, pairs = (w.s.nq + P.tiles * P.per - 1) / (P.tiles * P.per);
  w.h = in % P.H;
  w.first = (pairs - 1 - in / P.H) * P.tiles * P.per;                    // the ones that see most first
  const int p0 = w.s.nk - w.s.nq;
  for (int q = 0; q < 2; ++q) {
    const int f = w.first + q * P.per, l = (f + P.per < w.s.nq ? f + P.per : w.s.nq) - 1;
    w.at[q].a = p0 + f;
    w.at[q].b = f < w.s.nq ? p0 + l : -1;
    if (f >= w.s.nq || q >= P.tiles) w.at[q] = {0, -1};
  }
  const int hi = w.at[1].b > w.at[0].b ? w.at[1].b : w.at[0].b;
  int n = 0;
  w.sink_tiles = w.win0 = 0;
  if (hi >= 0) {
    const int last = hi / kTileRows + 1;
    const int lo = w.at[0].a < 0 ? 0 : w.at[0].a, start = lo - P.window + 1;
    w.win0 = start > 0 ? start / kTileRows : 0;
    const int sinks = (P.sinks + kTileRows - 1) / kTileRows;
    w.sink_tiles = sinks < last ? sinks : last;
    if (w.sink_tiles > w.win0) w.win0 = w.sink_tiles;
    n = w.sink_tiles + last - w.win0;
  }
  const int each = n / P.splits, more = n % P.splits;
  w.u0 = w.split * each + (w.split < more ? w.split : more);
  w.u1 = w.u0 + each + (w.split < more ? 1 : 0);
  return w;
}
// does any row of the tile see any key of it; does every row see every key
__device__ __forceinline__ bool sees_some(const WinParams &P, const Span &s, int kt) {
  const int k = kt * kTileRows;
  return k <= s.b && (k + kTileRows - 1 > (s.a < 0 ? 0 : s.a) - P.window || k < P.sinks);
}
__device__ __forceinline__ bool sees_all(const WinParams &P, const Span &s, int kt) {
  const int k = kt * kTileRows;
  return k + kTileRows - 1 <= s.a && (k > s.b - P.window || k + kTileRows <= P.sinks);
}
__device__ __forceinline__ bool seen_in_part(const WinParams &P, const WinItem &w, int kt) {
  bool part = false;
#pragma unroll
  for (int q = 0; q < 2; ++q) part |= sees_some(P, w.at[q], kt) && !sees_all(P, w.at[q], kt);
  return part;
}
// 16 keys at a time: which of the tile's eight steps any row sees
__device__ __forceinline__ unsigned seen_steps(const WinParams &P, const Span &s, int kt) {
  const int k = kt * kTileRows, lo = (s.a < 0 ? 0 : s.a) - P.window + 1 - k, hi = s.b - k;
  const unsigned to = hi < 0 ? 0u : (hi >= 127 ? 255u : (2u << (hi >> 4)) - 1u), from = lo <= 0 ? 0u : (lo >= 128 ? 255u : (1u << (lo >> 4)) - 1u);
  const int sinks = P.sinks - k;
  return to & (~from | (sinks <= 0 ? 0u : (sinks >= 128 ? 255u : (2u << ((sinks - 1) >> 4)) - 1u)));
}
__device__ __forceinline__ unsigned low_bits(int n) { return n <= 0 ? 0u : (n >= 32 ? 0xffffffffu : (1u << n) - 1u); }
// keys 32 i .. of the tile that the query at position p sees (p < 0: none)
__device__ __forceinline__ unsigned seen_bits(const WinParams &P, int p, int kt, int i) {
  const int base = kt * kTileRows + 32 * i;
  return low_bits(p - base + 1) & (~low_bits(p - P.window + 1 - base) | low_bits(P.sinks - base));
}

template <typename T> struct Zero2;
template <> struct Zero2<__half> {
  static __device__ __forceinline__ unsigned fma0(unsigned x, unsigned acc) {
    const __half2 r = __hfma2(*reinterpret_cast<__half2 *>(&x), __float2half2_rn(0.f), *reinterpret_cast<__half2 *>(&acc));
    return *reinterpret_cast<const unsigned *>(&r);
  }
  static constexpr unsigned kExp = 0x7c00u;
  static __device__ __forceinline__ float value(unsigned short b) { return __half2float(__ushort_as_half(b)); }
};
template <> struct Zero2<__nv_bfloat16> {
  static __device__ __forceinline__ unsigned fma0(unsigned x, unsigned acc) {
    const __nv_bfloat162 r = __hfma2(*reinterpret_cast<__nv_bfloat162 *>(&x), __float2bfloat162_rn(0.f), *reinterpret_cast<__nv_bfloat162 *>(&acc));
    return *reinterpret_cast<const unsigned *>(&r);
  }
  static constexpr unsigned kExp = 0x7f80u;
  static __device__ __forceinline__ float value(unsigned short b) { return __uint_as_float((unsigned)b << 16); }
};

template <typename T, int D>
__global__ void __launch_bounds__(WinShape<D>::kThreads, WinShape<D>::NT == 1 ? 2 : 1)
k_window(const __grid_constant__ WinParams P, const __grid_constant__ WinMaps M) {
  using S = WinShape<D>;
  constexpr int kSlots = S::kSlots, NT = S::NT, kLoads = 4 * NT;          // kLoads: the first warp behind the weights'
  extern __shared__ unsigned char smem_raw[];
  unsigned char *smem = reinterpret_cast<unsigned char *>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  unsigned char *ring = smem + NT * S::kTileBytes;
  __shared__ WinShared<kSlots> sh;
  __shared__ WinItem item;                                         // found by one thread while others set up
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);

  if (tid == 0) {
    mbar::init(&sh.qfull, 1u);
    for (int i = 0; i < kSlots; ++i) { mbar::init(&sh.full[i], 1u); mbar::init(&sh.empty[i], 1u); }
    for (int i = 0; i < kValues; ++i) mbar::init(&sh.clean[i], 2u);
    for (int q = 0; q < 2; ++q) { mbar::init(&sh.scores[q], 1u); mbar::init(&sh.halved[q], 1u); mbar::init(&sh.weights[q][0], 4u); mbar::init(&sh.weights[q][1], 4u); mbar::init(&sh.done[q], 1u); }
    mbar::init_done();
  }
  if (warp == kLoads && lane == 0) { prefetch_map(&M.q); prefetch_map(&M.k); prefetch_map(&M.v); }
  if (warp == kLoads + 1) umma::tmem_alloc(&sh.tmem, S::kColumns);
  if (tid == 32) item = find_item(P, blockIdx.x);
  before_sync();
  __syncthreads();
  after_sync();
  // Not before this block has its tensor memory: a block of the next kernel that took it would wait for this one to end.
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  asm volatile("griddepcontrol.wait;\n" ::: "memory");             // what the kernels before this one wrote is visible from here
  const unsigned tmem = sh.tmem;                                   // S of tile q at 128 q, O at 128 (NT + q)
  const WinItem &w = item;
  const int n = w.u1 - w.u0;
  // key tile u of the list is item 2 (u - u0) of the ring, its values the next one
  bool ok = true;

  if (warp >= kLoads) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(S::kRegsRest));
    if (warp == kLoads) {
      if (lane == 0) {
        const int tiles_q = NT == 2 && w.first + P.per < w.s.nq ? 2 : 1;
        const unsigned q_bytes = (unsigned)(P.per * P.G * 128 * (D / 64));
        int items = 0;
        if (n > 0) {
          mbar::expect_tx(&sh.qfull, q_bytes * tiles_q);
          for (int q = 0; q < tiles_q; ++q)
            for (int c = 0; c < D / 64; ++c)
              tma_load_3d(smem + q * S::kTileBytes + c * S::kBox, &M.q, 64 * c, w.h * P.G, w.s.q0 + w.first + q * P.per, &sh.qfull);
          for (; items < 2 * n; ++items) {
            const int st = items % kSlots, kt = w.key_tile(w.u0 + items / 2);
            if (items >= kSlots && !mbar::wait(&sh.empty[st], (unsigned)(items / kSlots - 1) & 1u)) { ok = false; break; }
            mbar::expect_tx(&sh.full[st], (unsigned)S::kTileBytes);
            for (int c = 0; c < D / 64; ++c)
              tma_load_3d(ring + st * S::kTileBytes + c * S::kBox, items & 1 ? &M.v : &M.k, 64 * c, w.h, w.s.k0 + kt * kTileRows, &sh.full[st]);
          }
          ok &= mbar::wait(&sh.qfull, 0u);
          ok &= mbar::drain(sh.full, items);                       // no block ends under its own loads
        }
        if (!ok) atomicOr(P.status, FC_DEV_FLAG_TIMEOUT);
      }
      __syncwarp();
    } else if (warp == kLoads + 1) {
      constexpr bool kF16 = std::is_same<T, __half>::value;
      constexpr unsigned s_desc = umma::instruction(kF16, false, kTileRows), o_desc = umma::instruction(kF16, false, D) | (1u << 16);
      constexpr unsigned hi = umma::operand_hi(1024, 2);           // 8 rows of 128 bytes each, 128-byte swizzle
      const unsigned lead = umma::elect();
      const unsigned qb = (umma::smem_addr(smem) >> 4) | umma::operand_lo(16);
      const unsigned kb = (umma::smem_addr(ring) >> 4) | umma::operand_lo(16), vb = (umma::smem_addr(ring) >> 4) | umma::operand_lo(S::kBox);
      unsigned turn[2] = {0u, 0u};
      const WinItem w = item;                                      // in registers
      auto scores = [&](int q, int i) {                            // S of tile q with keys i of the ring
        const unsigned k = kb + (unsigned)((2 * i) % kSlots) * (S::kTileBytes / 16), a = qb + (unsigned)q * (S::kTileBytes / 16);
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
          const unsigned off = (unsigned)(c >> 2) * (S::kBox / 16) + (unsigned)(c & 3) * 2u;
          umma::mma(lead, tmem + 128u * q, a + off, hi, k + off, hi, s_desc, c ? 1u : 0u);
        }
        umma::commit(lead, &sh.scores[q]);
      };
      if (n > 0) {
        ok = mbar::wait_warp(&sh.qfull, 0u) && mbar::wait_warp(&sh.full[0], 0u);
        if (ok) {
          after_sync();
          for (int q = 0; q < NT; ++q)
            if (sees_some(P, w.at[q], w.key_tile(w.u0))) scores(q, 0);
          umma::commit(lead, &sh.empty[0]);
        }
      }
      for (int i = 0; i < n && ok; ++i) {
        const int kt = w.key_tile(w.u0 + i), vi = 2 * i + 1, vs = vi % kSlots, ki = vi + 1;
        const bool next = i + 1 < n;
        const int kn = next ? w.key_tile(w.u0 + i + 1) : 0;
        if (!mbar::wait_warp(&sh.full[vs], (unsigned)(vi / kSlots) & 1u) ||
            (next && !mbar::wait_warp(&sh.full[ki % kSlots], (unsigned)(ki / kSlots) & 1u))) { ok = false; break; }
#pragma unroll
        for (int q = 0; q < NT && ok; ++q) {
          if (q == NT - 1 && !mbar::wait_warp(&sh.clean[i % kValues], (unsigned)(i / kValues) & 1u)) { ok = false; break; }
          if (sees_some(P, w.at[q], kt)) {
            const unsigned steps = seen_steps(P, w.at[q], kt);
#pragma unroll
            for (int half = 0; half < 2 && ok; ++half) {
              if (!mbar::wait_warp(&sh.weights[q][half], turn[q] & 1u)) { ok = false; break; }
              after_sync();
#pragma unroll
              for (int c = 4 * half; c < 4 * half + 4; ++c)
                if ((steps >> c) & 1u) mma_ts(lead, tmem + 128u * (NT + q), tmem + 128u * q + 8u * c, vb + (unsigned)vs * (S::kTileBytes / 16) + 128u * c, hi, o_desc, 1u);
              if (D == 128 && half == 0) umma::commit(lead, &sh.halved[q]);          // for rows that go on with a reference that moved
            }
            if (!ok) break;
            ++turn[q];
          }
          if (q == NT - 1) umma::commit(lead, &sh.empty[vs]);
          if (next) {
            if (sees_some(P, w.at[q], kn)) scores(q, i + 1);
            if (q == NT - 1) umma::commit(lead, &sh.empty[ki % kSlots]);
          }
        }
      }
      // nothing is left running when the block ends, and the rows' warps may take the outputs
      umma::commit(lead, &sh.done[0]);
      umma::commit(lead, &sh.done[1]);
      ok &= mbar::wait_warp(&sh.done[0], 0u) && mbar::wait_warp(&sh.done[1], 0u);
      if (!ok && lane == 0) atomicOr(P.status, FC_DEV_FLAG_TIMEOUT);
    } else {
      // values: clears what is not finite, and what lies past the sequence, in tiles that some row sees in part
      for (int i = 0; i < n; ++i) {
        const int kt = w.key_tile(w.u0 + i), vi = 2 * i + 1, vs = vi % kSlots;
        if (!mbar::wait_warp(&sh.full[vs], (unsigned)(vi / kSlots) & 1u)) { ok = false; break; }
        if (seen_in_part(P, w, kt)) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int r = 64 * (warp - kLoads - 2) + 32 * e + lane;
            unsigned char *row = ring + vs * S::kTileBytes + r * 128;
            const bool past = kt * kTileRows + r >= w.s.nk;
            unsigned acc = 0u;
            if (!past) {
#pragma unroll
              for (int c = 0; c < D / 8; ++c) {
                const uint4 x = *reinterpret_cast<const uint4 *>(row + (c >> 3) * S::kBox + (((c + r) & 7) << 4));
                acc = Zero2<T>::fma0(x.x, Zero2<T>::fma0(x.y, Zero2<T>::fma0(x.z, Zero2<T>::fma0(x.w, acc))));
              }
            }
            const bool odd = (acc & 0x7fff7fffu) != 0u;            // 0 as long as everything is finite
            if (past || odd) {
              for (int c = 0; c < D / 8; ++c) {
                unsigned *x = reinterpret_cast<unsigned *>(row + (c >> 3) * S::kBox + ((c & 7) << 4));
                for (int j = 0; j < 4; ++j) {
                  unsigned v = x[j];
                  if (past || (v & Zero2<T>::kExp) == Zero2<T>::kExp) v &= 0xffff0000u;
                  if (past || ((v >> 16) & Zero2<T>::kExp) == Zero2<T>::kExp) v &= 0x0000ffffu;
                  x[j] = v;
                }
              }
              asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
            }
            const unsigned which = __ballot_sync(0xffffffffu, odd);
            if (lane == 0) sh.bad[i % kValues][2 * (warp - kLoads - 2) + e] = which;
          }
        }
        __syncwarp();
        if (lane == 0) mbar::arrive(&sh.clean[i % kValues]);
      }
      if (!ok && lane == 0) atomicOr(P.status, FC_DEV_FLAG_TIMEOUT);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" ::"n"(S::kRegsRows));
    const int q = warp >> 2, r = (warp & 3) * 32 + lane;
    const unsigned rows = (unsigned)((warp & 3) * 32) << 16;       // this warp's lanes of tensor memory
    const unsigned s_at = tmem + rows + 128u * q, o_at = tmem + rows + 128u * (NT + q);
    const int qi = w.first + q * P.per + r / P.G, head = w.h * P.G + r % P.G;
    const bool have = r < P.per * P.G && qi < w.s.nq;
    const int p = have ? w.s.nk - w.s.nq + qi : -1;
    float m = -INFINITY, l = 0.f;
    {
      unsigned zero[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) zero[i] = 0u;
#pragma unroll
      for (int c = 0; c < D; c += 32) tm_st32(o_at + c, zero);
      tm_wait_st();
    }
    unsigned turn = 0u;
    const float2 scale = make_float2(P.scale_log2, P.scale_log2);
    for (int i = 0; i < n; ++i) {
      const int kt = w.key_tile(w.u0 + i);
      if (!sees_some(P, w.at[q], kt)) continue;
      const bool all = sees_all(P, w.at[q], kt), looked = seen_in_part(P, w, kt);
      if (!mbar::wait_warp(&sh.scores[q], turn & 1u)) { ok = false; break; }
      ++turn;
      after_sync();
      float s[128];
#pragma unroll
      for (int c = 0; c < 128; c += 32) tm_ld32(s_at + c, s + c);
      tm_wait_ld(s);
      float2 sum;
      unsigned pk[32];
      // Weights of the keys c .. c + 63, all seen by all.  any: their scores may be any distance above the reference.
      auto weights = [&](int c, float ref, auto any) {
        const float2 minus = make_float2(-ref, -ref);
        sum = make_float2(0.f, 0.f);
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          const float2 x = __ffma2_rn(make_float2(s[c + 2 * j], s[c + 2 * j + 1]), scale, minus);
          const float2 y = (j & (D == 128 ? 3 : 7)) == 3 ? exp2_poly<decltype(any)::value>(x) : make_float2(exp2_fast(x.x), exp2_fast(x.y));
          sum = __fadd2_rn(sum, y);
          pk[j] = Mma<T>::pack(y.x, y.y);
        }
      };
      auto ready = [&](int half) {
        before_sync();
        __syncwarp();
        if (lane == 0) mbar::arrive(&sh.weights[q][half]);
      };
      auto give = [&](int half) {
        tm_st32(s_at + 32 * half, pk);
        tm_wait_st();
        ready(half);
        l += sum.x + sum.y;
      };
      // As a rule the reference stays as it is, and that it may shows in the sums: a weight that passes its bound makes a sum that does
      // (so does NaN): none is negative, and one that no number holds is infinite or 2^127.  No largest score is looked for then.
      const bool quick = D == 128 && !looked && turn > 1u && !__any_sync(0xffffffffu, have && m == -INFINITY);
      bool begun = false;                                          // the first half is the product's already
      if (quick) {
        const float ref = m == -INFINITY ? 0.f : m;
        auto fits = [&]() { return !__any_sync(0xffffffffu, have && !(sum.x + sum.y <= kMost<T>)); };
        weights(0, ref, std::true_type());
        if (fits()) {
          give(0);
          weights(64, ref, std::true_type());
          if (fits()) {
            give(1);
            continue;
          }
          begun = true;
          if (ok) ok = mbar::wait_warp(&sh.halved[q], (turn - 1u) & 1u);
          if (!ok) break;
          after_sync();
        }
      }
      unsigned chunks = 0u;                                        // of a tile seen in part: 32 keys at a time, those that a row of the warp sees
      float top;                                                   // NaN if any score is
      if (all) {
        float tops[4] = {s[0], s[1], s[2], s[3]};                  // chains of their own
#pragma unroll
        for (int c = 4; c < 124; c += 8)
#pragma unroll
          for (int k = 0; k < 4; ++k) tops[k] = max_nan(tops[k], s[c + 2 * k], s[c + 2 * k + 1]);
        top = max_nan(max_nan(tops[0], s[124], s[125]), max_nan(tops[1], s[126], s[127]), max_nan(tops[2], tops[3], tops[3]));
      } else {
        top = -INFINITY;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const unsigned bits = seen_bits(P, p, kt, c);
          if (!__any_sync(0xffffffffu, bits != 0u)) continue;
          chunks |= 1u << c;
          float t[2] = {-INFINITY, -INFINITY};
#pragma unroll
          for (int j = 0; j < 32; j += 4) {
#pragma unroll
            for (int k = 0; k < 4; ++k) s[32 * c + j + k] = (bits >> (j + k)) & 1u ? s[32 * c + j + k] : -INFINITY;
            t[0] = max_nan(t[0], s[32 * c + j], s[32 * c + j + 1]);
            t[1] = max_nan(t[1], s[32 * c + j + 2], s[32 * c + j + 3]);
          }
          top = max_nan(top, t[0], t[1]);
        }
      }
      top *= P.scale_log2;
      const bool move = top > m + (quick ? kSlack<T> - 7.f : kSlack<T>);          // a sum of 64 has passed it
      if (__any_sync(0xffffffffu, move)) {
        const float to = move ? top - kAbove<T> : m, f = m == to ? 1.f : exp2f(m - to);
        m = to;
        l *= f;
        if (turn > 1u) {                                           // the products so far are done: the scores came after them
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            float o[32];
            tm_ld32(o_at + c, o);
            tm_wait_ld(o);
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] *= f;
            tm_st32(o_at + c, reinterpret_cast<const unsigned *>(o));
          }
        }
      }
      const float ref = top != top ? top : (m == -INFINITY ? 0.f : m);                       // a NaN among the scores: all weights
      if (!looked) {                                               // the product starts on half of them
        if (!begun) {
          weights(0, ref, std::false_type());
          give(0);
        }
        weights(64, ref, std::false_type());
        give(1);
      } else {
        const float2 minus = make_float2(-ref, -ref);
        sum = make_float2(0.f, 0.f);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          unsigned pk[16];
          if (all || ((chunks >> c) & 1u)) {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const float2 x = __ffma2_rn(make_float2(s[32 * c + 2 * j], s[32 * c + 2 * j + 1]), scale, minus);
              const float2 y = make_float2(exp2_fast(x.x), exp2_fast(x.y));
              sum = __fadd2_rn(sum, y);
              pk[j] = Mma<T>::pack(y.x, y.y);
            }
          } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) pk[j] = 0u;
          }
          tm_st16(s_at + 16 * c, pk);
        }
        tm_wait_st();
        if (!mbar::wait_warp(&sh.clean[i % kValues], (unsigned)(i / kValues) & 1u)) { ok = false; break; }
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          const unsigned mine = all ? 0xffffffffu : seen_bits(P, p, kt, c);
          for (unsigned left = sh.bad[i % kValues][c]; left; left &= left - 1u) {
            const int key = 32 * c + __ffs(left) - 1;
            unsigned pair;
            tm_ld1(s_at + key / 2, pair);
            tm_wait_ld1(pair);
            const float weight = Zero2<T>::value((unsigned short)(key & 1 ? pair >> 16 : pair));
            const unsigned short *row = reinterpret_cast<const unsigned short *>(P.v + (w.s.k0 + kt * kTileRows + key) * P.v_token + w.h * P.v_head);
            for (int j = 0; j < D; ++j) {
              const unsigned short v = row[j];
              if ((v & Zero2<T>::kExp) != Zero2<T>::kExp) continue;
              unsigned o;
              tm_ld1(o_at + j, o);
              tm_wait_ld1(o);
              if ((mine >> (key & 31)) & 1u) o = __float_as_uint(fmaf(weight, Zero2<T>::value(v), __uint_as_float(o)));
              tm_st1(o_at + j, o);
              tm_wait_st();
            }
          }
        }
        ready(0);
        ready(1);
        l += sum.x + sum.y;
      }
    }
    if (ok) ok = mbar::wait_warp(&sh.done[q], 0u);
    if (!ok && lane == 0) atomicOr(P.status, FC_DEV_FLAG_TIMEOUT);
    after_sync();
    // nothing seen: 0; only scores of minus infinity: 0 / 0 (their weights by polynomial are not 0)
    const float inv = p < 0 ? 0.f : (m == -INFINITY ? __int_as_float(0x7fffffff) : 1.f / l);
    const size_t slot = (((size_t)w.item * P.splits + w.split) * NT + q) * kTileRows + r;
#pragma unroll 1
    for (int c = 0; c < D; c += 32) {
      float o[32];
      tm_ld32(o_at + c, o);
      tm_wait_ld(o);
      if (!have || !ok) continue;
      if (P.splits > 1) {
        float4 *dst = reinterpret_cast<float4 *>(P.part_o + slot * D + c);
#pragma unroll
        for (int j = 0; j < 8; ++j) dst[j] = make_float4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
        if (c == 0) P.part_ml[slot] = make_float2(m, l);
      } else {
        uint4 *dst = reinterpret_cast<uint4 *>(static_cast<T *>(P.out) + ((size_t)(w.s.q0 + qi) * P.Hq + head) * D + c);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          dst[j] = make_uint4(Mma<T>::pack(o[8 * j] * inv, o[8 * j + 1] * inv), Mma<T>::pack(o[8 * j + 2] * inv, o[8 * j + 3] * inv),
                              Mma<T>::pack(o[8 * j + 4] * inv, o[8 * j + 5] * inv), Mma<T>::pack(o[8 * j + 6] * inv, o[8 * j + 7] * inv));
      }
    }
  }
  before_sync();
  __syncthreads();
  after_sync();
  if (warp == kLoads + 1) umma::tmem_free(tmem, S::kColumns);
}

// Joins the parts of split blocks: a warp per row, D / 32 channels per lane.
template <typename T, int D>
__global__ void __launch_bounds__(128)
k_window_join(const __grid_constant__ WinParams P) {
  constexpr int C = D / 32;
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  const int lane = threadIdx.x & 31, r = blockIdx.y * 4 + (threadIdx.x >> 5), q = blockIdx.z;
  const WinItem w = find_item(P, blockIdx.x * P.splits);
  const int qi = w.first + q * P.per + r / P.G;
  if (r >= P.per * P.G || qi >= w.s.nq) return;
  const size_t step = P.tiles * kTileRows, slot0 = (size_t)w.item * P.splits * step + q * kTileRows + r;
  float m = -INFINITY;
  for (int i = 0; i < P.splits; ++i) m = fmaxf(m, __ldcg(P.part_ml + slot0 + i * step).x);
  const float ref = m == -INFINITY ? 0.f : m;
  float acc[C], l = 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c) acc[c] = 0.f;
  for (int i = 0; i < P.splits; ++i) {
    const size_t slot = slot0 + i * step;
    const float2 ml = __ldcg(P.part_ml + slot);
    const float f = exp2f(ml.x - ref);
    l = fmaf(ml.y, f, l);
#pragma unroll
    for (int c = 0; c < C; c += 2) {
      const float2 x = __ldcg(reinterpret_cast<const float2 *>(P.part_o + slot * D + C * lane + c));
      acc[c] = fmaf(x.x, f, acc[c]);
      acc[c + 1] = fmaf(x.y, f, acc[c + 1]);
    }
  }
  const float inv = w.s.nk - w.s.nq + qi < 0 ? 0.f : 1.f / l;     // 0 / 0 of scores that are all minus infinity
  T *out = static_cast<T *>(P.out) + ((size_t)(w.s.q0 + qi) * P.Hq + w.h * P.G + r % P.G) * D + C * lane;
#pragma unroll
  for (int c = 0; c < C; c += 2) *reinterpret_cast<unsigned *>(out + c) = Mma<T>::pack(acc[c] * inv, acc[c + 1] * inv);
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
fc_status encode_heads(CUtensorMap *m, CUtensorMapDataType dt, const void *base, int d, int heads, int64_t tokens, int64_t stride_token,
                       int64_t stride_head, int box_heads, int box_tokens) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return FC_ERR_CUDA;
  const cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)heads, (cuuint64_t)tokens};
  const cuuint64_t str[2] = {(cuuint64_t)stride_head * 2, (cuuint64_t)stride_token * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_tokens}, ones[3] = {1, 1, 1};
  return fn(m, dt, 3, const_cast<void *>(base), dims, str, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS ? FC_OK : FC_ERR_INTERNAL;
}

bool lengths_ok(const int32_t *cu, int batch) {
  if (!cu || cu[0] != 0) return false;
  for (int b = 0; b < batch; ++b)
    if (cu[b + 1] < cu[b]) return false;
  return cu[batch] <= (1 << 30);
}

fc_status check_window(const fc_handle *h, const fc_window_args *a) {
  if (!h || !a || !a->kv || !a->q || !a->kv->k || !a->kv->v) return FC_ERR_INVALID_ARG;
  const fc_kv_view *kv = a->kv;
  if (kv->batch < 1 || kv->num_heads < 1 || a->num_q_heads < 1 || a->window < 1 || a->sinks < 0) return FC_ERR_INVALID_ARG;
  if (kv->dtype != FC_F16 && kv->dtype != FC_BF16) return FC_ERR_UNSUPPORTED;
  if (kv->head_dim != 64 && kv->head_dim != 128) return FC_ERR_UNSUPPORTED;
  if (a->num_q_heads % kv->num_heads != 0 || a->num_q_heads / kv->num_heads > 64) return FC_ERR_UNSUPPORTED;
  if (!lengths_ok(kv->cu_seqlens, kv->batch) || !lengths_ok(a->cu_seqlens_q, kv->batch)) return FC_ERR_INVALID_ARG;
  if (((uintptr_t)a->q & 15) || ((uintptr_t)kv->k & 15) || ((uintptr_t)kv->v & 15)) return FC_ERR_INVALID_ARG;
  const int64_t str[4] = {a->q_stride_token, a->q_stride_head, kv->stride_token, kv->stride_head};
  for (int i = 0; i < 4; ++i)
    if (str[i] < 8 || str[i] % 8 != 0 || str[i] >= (1ll << 38)) return FC_ERR_INVALID_ARG;
  return FC_OK;
}

int tiles_of(int d) { return d == 128 ? WinShape<128>::NT : WinShape<64>::NT; }

// One launch: sequences [b0, b1), those without queries left out.
struct WinLaunch { int b1, items, splits, seqs; };

WinLaunch plan_launch(const fc_handle *h, const fc_window_args *a, int b0, WinSeq *seq) {
  const fc_kv_view *kv = a->kv;
  const int G = a->num_q_heads / kv->num_heads, per = kTileRows / G, rows = tiles_of(kv->head_dim) * per;       // queries of a block
  WinLaunch l = {b0, 0, 1, 0};
  long long items = 0, most = 0;
  for (; l.b1 < kv->batch && l.seqs < kSeqs; ++l.b1) {
    const int b = l.b1, nq = a->cu_seqlens_q[b + 1] - a->cu_seqlens_q[b], nk = kv->cu_seqlens[b + 1] - kv->cu_seqlens[b];
    if (nq == 0) continue;
    const long long mine = (long long)((nq + rows - 1) / rows) * kv->num_heads;
    if (items > 0 && items + mine > (1 << 24)) break;
    if (seq) seq[l.seqs] = {a->cu_seqlens_q[b], nq, kv->cu_seqlens[b], nk, (int)items};
    ++l.seqs;
    items += mine;
    long long span = (long long)a->window + rows + a->sinks;    // keys a block may see
    if (span > nk) span = nk;
    if (span > most) most = span;
  }
  l.items = (int)items;
  // Fewer blocks than SMs: the key tiles of each are split so that all SMs have a part, of kSplitMin tiles at least.
  const int room = h->num_sms * (tiles_of(kv->head_dim) == 1 ? 2 : 1);
  if (items > 0 && 2 * items <= room) {
    const long long tiles = most / kTileRows + 1, by_sm = room / items, by_len = tiles / kSplitMin;
    l.splits = (int)(by_sm < by_len ? by_sm : by_len);
    if (l.splits < 1) l.splits = 1;
  }
  return l;
}

size_t part_bytes(const WinLaunch &l, int D) { return l.splits > 1 ? (size_t)l.items * l.splits * tiles_of(D) * kTileRows * (D + 2) * sizeof(float) : 0; }

template <typename T, int D>
fc_status launch_window(fc_handle *h, const WinParams &P, const WinMaps &M, int items, cudaStream_t st) {
  using S = WinShape<D>;
  static_assert(S::kSlots <= 2 * kValues, "a value tile's turn comes again after the one before it has gone");
  static_assert((S::kSmem + sizeof(WinShared<S::kSlots>) + sizeof(WinItem) + 1024) * (S::NT == 1 ? 2 : 1) <= 228 * 1024, "shared memory");
  constexpr unsigned bit = 1u << (16 + (std::is_same<T, __half>::value ? 1 : 0) + (D == 128 ? 2 : 0));
  if (!(h->forms_ready & bit)) {           // once per handle
    FC_CUDA_TRY(cudaFuncSetAttribute(k_window<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmem));
    h->forms_ready |= bit;
  }
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3((unsigned)(items * P.splits));
  lc.blockDim = dim3(S::kThreads);
  lc.dynamicSmemBytes = S::kSmem;
  lc.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  lc.attrs = at;
  lc.numAttrs = 1;
  if (cudaLaunchKernelEx(&lc, k_window<T, D>, P, M) != cudaSuccess) {
    cudaGetLastError();
    return FC_ERR_CUDA;
  }
  fc_status s = fc_after_launch(h);
  if (s != FC_OK || P.splits == 1) return s;
  lc.gridDim = dim3((unsigned)items, (unsigned)((P.per * P.G + 3) / 4), (unsigned)S::NT);
  lc.blockDim = dim3(128);
  lc.dynamicSmemBytes = 0;
  if (cudaLaunchKernelEx(&lc, k_window_join<T, D>, P) != cudaSuccess) {
    cudaGetLastError();
    return FC_ERR_CUDA;
  }
  return fc_after_launch(h);
}

}  // namespace

extern "C" size_t fc_window_workspace_bytes(const fc_handle *h, const fc_window_args *a) {
  if (check_window(h, a) != FC_OK) return 0;
  size_t most = 0;
  for (int b = 0; b < a->kv->batch;) {
    const WinLaunch l = plan_launch(h, a, b, nullptr);
    const size_t n = part_bytes(l, a->kv->head_dim);
    most = n > most ? n : most;
    b = l.b1;
  }
  return most + 256;                           // never 0 for arguments that are in order
}

extern "C" fc_status fc_window_attention(fc_handle *h, const fc_window_args *a, void *out, void *workspace, size_t workspace_bytes,
                                         fc_stream stream) {
  fc_status s = check_window(h, a);
  if (s != FC_OK) return s;
  if (!out || ((uintptr_t)out & 15)) return FC_ERR_INVALID_ARG;
  if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < fc_window_workspace_bytes(h, a)) return FC_ERR_WORKSPACE;
  const fc_kv_view *kv = a->kv;
  const int64_t Tq = a->cu_seqlens_q[kv->batch], Tk = kv->cu_seqlens[kv->batch];
  if (Tq == 0) return FC_OK;
  const int D = kv->head_dim;
  FcDeviceGuard on(h->device);
  if (!on.ok) return FC_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if ((s = fc_flush_pending(h, st)) != FC_OK) return s;
  WinParams P = {};
  P.out = out;
  P.status = h->status_word;
  P.v = static_cast<const char *>(kv->v);
  P.v_token = kv->stride_token * 2;
  P.v_head = kv->stride_head * 2;
  P.H = kv->num_heads;
  P.Hq = a->num_q_heads;
  P.G = P.Hq / P.H;
  P.per = kTileRows / P.G;
  P.tiles = tiles_of(D);
  P.window = a->window < (1 << 30) ? a->window : (1 << 30);
  P.sinks = a->sinks < (1 << 30) ? a->sinks : (1 << 30);
  P.scale_log2 = (float)(1.4426950408889634 / sqrt((double)D));
  const CUtensorMapDataType dt = kv->dtype == FC_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  WinMaps M = {};
  if ((s = encode_heads(&M.q, dt, a->q, D, P.Hq, Tq, a->q_stride_token, a->q_stride_head, P.G, P.per)) != FC_OK) return s;
  // without any key nothing is loaded, but a map wants a row
  if ((s = encode_heads(&M.k, dt, kv->k, D, P.H, Tk < 1 ? 1 : Tk, kv->stride_token, kv->stride_head, 1, kTileRows)) != FC_OK) return s;
  if ((s = encode_heads(&M.v, dt, kv->v, D, P.H, Tk < 1 ? 1 : Tk, kv->stride_token, kv->stride_head, 1, kTileRows)) != FC_OK) return s;
  for (int b = 0; b < kv->batch;) {
    const WinLaunch l = plan_launch(h, a, b, P.seq);
    b = l.b1;
    if (l.items == 0) continue;
    P.seqs = l.seqs;
    P.splits = l.splits;
    P.part_o = static_cast<float *>(workspace);
    P.part_ml = reinterpret_cast<float2 *>(P.part_o + (size_t)l.items * l.splits * P.tiles * kTileRows * D);
    if (kv->dtype == FC_F16) s = D == 128 ? launch_window<__half, 128>(h, P, M, l.items, st) : launch_window<__half, 64>(h, P, M, l.items, st);
    else s = D == 128 ? launch_window<__nv_bfloat16, 128>(h, P, M, l.items, st) : launch_window<__nv_bfloat16, 64>(h, P, M, l.items, st);
    if (s != FC_OK) return s;
  }
  return FC_OK;
}
