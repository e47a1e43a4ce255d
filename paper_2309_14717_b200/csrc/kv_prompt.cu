// Attention of many new tokens over the 8-bit key/value cache (a prompt, or the next piece of one) on
// the 5th-generation tensor cores, and the weights that its cached tokens gather.
#define QALORA_TU 14
#include <cooperative_groups.h>

#include "kv.cuh"
#include "kv_ptx.cuh"

namespace cg = cooperative_groups;

namespace qalora {

namespace {

constexpr int PT_CONV = 8;                     // conversion warps
constexpr int PT_THREADS = 256 + PT_CONV * 32 + 128;   // 2 x 128 softmax, conversion, 2 issuing warps, the look-ups (and one idle warp)
constexpr int PT_ISSUE = 8 + PT_CONV;          // first issuing warp
constexpr int PT_TOK = 128, PT_ROWS = 128;    // a tile: tokens x rows (new tokens x heads of a group)
constexpr int PT_HALF = 64;                   // tokens of a step: half a tile
constexpr int PS_MAX_CLUSTER = 8;             // thread blocks that share a token tile's row tiles
constexpr int PT_RING = 8;                    // tiles whose blocks and scales are kept
constexpr int PT_RING_FLOATS = 48;            // ks[8], log2 of vs / ref [8], ref / vs [8], {ref_before / ref, ref, all there, largest ks},
                                              // blocks of keys [8] at 32 and of values [8] at 40
constexpr float kLargeFactor = 0x1p-9f;       // of S, which allows scores beyond 2^20 (|S| <= 2^29)
constexpr float kMostGathered = 0x1p24f;      // largest score with which a row takes part in the gathered weights
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNoMax = -3.40282347e38f;
constexpr float kGrow = 6.f, kLift = 8.f;     // as in the few-row kernel: weights at most 2^14 in fp16
constexpr float kTiny = 1e-37f;               // stands for a smaller factor of a score (|score| < 2^30): keeps 0 * -inf away
constexpr float kLeastExponent = -80.f, kLeastValueScale = 0x1p-80f;   // of the largest one met so far: below it a block's values count as 0
constexpr float kMostSum = 64.f;              // a change of reference lets a row's sum grow to 2^64, and the weights after it by 2^80 each

struct PromptArgs {
  KvShape sh;
  KvBatch kb;
  KvAttention at;
  int splits;
  long long slots;
  float2* part_ml;       // [splits][kv_heads * slots * 128]
  float* part_o;         // [splits][kv_heads * slots * 128][D]
  uint8_t* q_image;      // [kv_heads * slots][128 * D * 2]
  float* rows;           // [kv_heads * slots][2][128]: the factor of a row's scores (not 0, see kTiny); minus log2 of its sum
  int* status;
};

// Slot of the first row tile of sequence b (of every kv head): rows of 128 that no other sequence uses.
__device__ __forceinline__ long long first_slot(const KvShape& sh, const KvSeq& s, int b) {
  return (long long)s.row0 * sh.group / PT_ROWS + b;
}

template <int D>
struct PtSmem {
  static constexpr int TILE = 128 * D * 2;                    // bytes of an fp16 tile
  static constexpr int OFF_Q = 0;                             // two row tiles
  static constexpr int OFF_K = 2 * TILE, OFF_V = 4 * TILE;    // two stages each
  static constexpr int STAGED = 128 * D;                      // bytes of a tile of codes
  static constexpr int OFF_STAGED = 6 * TILE;                 // keys, values
  static constexpr int OFF_RING = OFF_STAGED + 2 * STAGED;
  static constexpr int OFF_BARS = OFF_RING + PT_RING * PT_RING_FLOATS * 4;
  static constexpr int NBARS = 1 + 4 * 2 + 6 * 2 + PT_RING + 4 + 2;
  static constexpr int OFF_SLOT = OFF_BARS + NBARS * 8 + 8;
  static constexpr int TOTAL = OFF_SLOT + 16 + 1024;
};

// 16 codes to fp16 and into row `row`, 16-byte chunks 2 * piece and 2 * piece + 1, of a tile of [128][64]
// blocks with 128-byte swizzle.
__device__ __forceinline__ void store_codes(uint8_t* tile, int row, int piece, const uint4& c) {
  uint4 lo, hi;
  kvp::codes_to_half(c.x, lo.x, lo.y);
  kvp::codes_to_half(c.y, lo.z, lo.w);
  kvp::codes_to_half(c.z, hi.x, hi.y);
  kvp::codes_to_half(c.w, hi.z, hi.w);
  const int chunk = (2 * piece) & 7;
  uint8_t* base = tile + (piece >> 2) * 16384 + row * 128;
  *reinterpret_cast<uint4*>(base + ((chunk ^ (row & 7)) << 4)) = lo;
  *reinterpret_cast<uint4*>(base + (((chunk + 1) ^ (row & 7)) << 4)) = hi;
}

// Which 16 codes of pass p over a tile thread t of `THREADS` takes.  Eight neighbouring lanes read the eight pieces of a
// 128-byte row (or the four of two 64-byte rows): different banks.  With 128 channels the lanes of the second half take
// the neighbouring row, so that the swizzled chunks that the eight of them store lie in different banks too.
template <int D, int THREADS>
struct TileMap {
  static constexpr int PIECES = D / 16, ROWS = THREADS / PIECES, PASSES = 128 / ROWS;
  int piece, row0;
  __device__ __forceinline__ explicit TileMap(int t) : piece(t % PIECES), row0(D == 128 ? (t / PIECES) ^ ((t >> 2) & 1) : t / PIECES) {}
};

// A staged tile of codes, rows of D bytes, to an fp16 tile.  Unless all of it is there, rows from `rows` on and those of
// blocks that are not there (`ids`: the blocks of the tile's groups of 16 tokens) become zeros.
template <int D>
__device__ __forceinline__ void convert_tile(const uint8_t* staged, uint8_t* tile, bool all, const int* ids, int rows, int t) {
  using Map = TileMap<D, PT_CONV * 32>;
  const Map map(t);
#pragma unroll
  for (int p = 0; p < Map::PASSES; ++p) {
    const int row = p * Map::ROWS + map.row0;
    uint4 c = *reinterpret_cast<const uint4*>(staged + row * D + map.piece * 16);
    if (!all && (row >= rows || ids[row >> 4] < 0)) c = make_uint4(0, 0, 0, 0);
    store_codes(tile, row, map.piece, c);
  }
}

// A softmax thread's row.
struct SoftmaxRow {
  float factor;            // softmax_scale * log2(e) / (the row's power of two)
  float m, l;              // running maximum of score + log2 of the relative value scale, in powers of two; sum of 2^(score - m)
  float ref;               // value scale that the outputs are relative to
};

// A step's scores in a thread's registers: the columns (tokens) beyond `seen` masked.  c, off: the factor of a score and log2 of the value scale,
// of 16 tokens each.  Returns the step's maximum.
__device__ __forceinline__ float softmax_top(float (&x)[PT_HALF], const float4 c, const float4 off, bool edge, int seen) {
  if (edge) {
#pragma unroll
    for (int t = 0; t < PT_HALF; ++t) if (t > seen) x[t] = -INFINITY;
  }
  const float cs[4] = {c.x, c.y, c.z, c.w}, os[4] = {off.x, off.y, off.z, off.w};
  float top = -INFINITY;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const float* v = x + 16 * g;
    float a = fmaxf(v[0], v[1]), b = fmaxf(v[2], v[3]);
#pragma unroll
    for (int t = 4; t < 16; t += 4) {
      a = kvp::max3(a, v[t], v[t + 1]);
      b = kvp::max3(b, v[t + 2], v[t + 3]);
    }
    top = fmaxf(top, fmaf(fmaxf(a, b), cs[g], os[g]));
  }
  return top;
}

// The step's weights to P, over its own columns of S; inv: the inverse of the relative value scale; m: what the scores are
// relative to.
template <int q>
__device__ __forceinline__ void softmax_exp(SoftmaxRow& w, float m, const float (&x)[PT_HALF], const float4 c, const float4 off, const float4 inv, uint32_t t_s) {
  const float cs[4] = {c.x, c.y, c.z, c.w}, os[4] = {off.x, off.y, off.z, off.w}, is[4] = {inv.x, inv.y, inv.z, inv.w};
  const float base = kLift - m;
  {
    uint32_t pk[16];
#pragma unroll
    for (int g2 = 0; g2 < 2; ++g2) {
      const int g = 2 * q + g2;
      const float2 cc = make_float2(cs[g], cs[g]), oo = make_float2(os[g] + base, os[g] + base);
      float2 sum = make_float2(0.f, 0.f);
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        float2 y = ptx::ffma2(make_float2(x[16 * g + 2 * t], x[16 * g + 2 * t + 1]), cc, oo);
        y.x = kvp::exp2_fast(y.x);
        y.y = kvp::exp2_fast(y.y);
        sum = ptx::fadd2(sum, y);
        pk[8 * g2 + t] = kvp::pack_half2(y.x, y.y);
      }
      w.l = fmaf(sum.x + sum.y, is[g], w.l);
    }
    ptx::tmem_st16(t_s + 16 * q, pk);
  }
}

// What a row whose sum is NaN leaves for the gathered weights: a query of NaN, which spoils the weights of the tokens it sees, and
// (in `rows`) minus infinity, as NaN there would reach the masked tokens too.
template <int D>
__device__ __forceinline__ void spoil_row(uint8_t* q_image, long long slot, int row) {
  *reinterpret_cast<uint16_t*>(q_image + slot * PtSmem<D>::TILE + row * 128 + ((row & 7) << 4)) = 0x7fff;
}
// (A score here and the row's logarithm are rounded apart: with scores beyond 2^24 their difference is no longer a weight's
// exponent, and the row is left out.)
__device__ __forceinline__ float minus_log2_sum(float m, float l) { return l > 0.f && fabsf(m) <= kMostGathered ? kLift - m - log2f(l) : -INFINITY; }

// Two tiles of 128 rows of one kv head against a range of its sequence's tokens, in tiles of 128 and steps of 64:
//   look-up warp      blocks and scales of a tile, bulk copies of its codes;
//   conversion warps  codes of a tile -> fp16 keys (K-major) and values (MN-major) in shared memory;
//   issuing warps     one per row tile: S = Q K^T of a step into one of two places in tensor memory, O += P V with P in
//                     tensor memory;
//   softmax threads   one per row: S from tensor memory, P back over its columns.
// S of the next step is there while a step's softmax runs: a row tile's softmax never waits for its products.  (Steps of
// 128 tokens, for whose S there is one place only, left softmax and products of a row tile to alternate: 189 us for a
// 4096-token prompt of 32 heads of 128, against 185.)  S of the next step but one
// lies where P of a step was, so it waits for the arrival that tells that P V of the step is done: tcgen05 products of
// one thread are ordered among themselves only where accumulator and shape are the same, and these two differ in
// both.  (Relying on the order of issue: 179.2 us for that prompt against 179.9 with the wait; two pieces of up to 700 tokens,
// 32 heads of 64, with the weights gathered 356.0 against 359.6.)
// What bounds it: the softmax warps.  A step takes about 2200 cycles, of which the exponential unit is busy for 1024 (64 x 128
// exponentials of either row tile at 16 a cycle), the tensor core for 1024 to 1280 (S with 64 columns reads Q again for
// every half tile) and the four issue slots for about 1150; the two softmax warps of a scheduler run in step, so that the
// unit rests while both look for their maxima.  Taking turns (by mbarriers, by named barriers), half a step's offset at the start,
// S fetched in the middle of the step before, a share of the exponentials on the FMA pipe and two places of registers
// for S were each measured and none was faster.  A block's beginning and end cost another 15 000 cycles, most of them
// waits for instructions that no block has run for a while: hence the rolled loops there, 172 us against 176.  (One block to
// a multiprocessor that takes over the work of blocks not yet started, with rows and tiles of the next piece brought in
// during the last: 175 against 176.)
template <int D>
__global__ void __launch_bounds__(PT_THREADS, 1)
kv_prompt_kernel(const __grid_constant__ PromptArgs a, int pairs_max, int* dbg) {
  using S = PtSmem<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (ptx::smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t sbase = ptx::smem_u32(smem), bars = sbase + S::OFF_BARS;
  float* ring = reinterpret_cast<float*>(smem + S::OFF_RING);
  const uint32_t q_full = bars;
  auto k_full = [&](int s) { return bars + 8 + 8 * s; };
  auto k_empty = [&](int s) { return bars + 24 + 8 * s; };
  auto v_full = [&](int s) { return bars + 40 + 8 * s; };
  auto v_empty = [&](int s) { return bars + 56 + 8 * s; };
  auto s_full = [&](int i, int step) { return bars + 72 + 16 * i + 8 * (step & 1); };
  auto p_full = [&](int i, int step) { return bars + 104 + 16 * i + 8 * (step & 1); };
  // P V of a step is done.  (Two: a wait tells a barrier's phase from the next but not from the next but one, and a softmax
  // thread that holds S of a step knows only that P V of the step two before is done.)
  auto o_done = [&](int i, int step) { return bars + 136 + 16 * i + 8 * (step & 1); };
  auto r_used = [&](int x) { return bars + 168 + 8 * x; };              // the codes of a tile have been converted
  auto c_full = [&](int w) { return bars + 168 + 8 * (PT_RING + w); };  // codes of keys (0) or values (1) are staged
  auto c_empty = [&](int w) { return bars + 168 + 8 * (PT_RING + 2 + w); };
  auto given_up = [&](int i) { return bars + 168 + 8 * (PT_RING + 4 + i); };    // products issued before a wait ran out are done
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + S::OFF_SLOT);
  volatile int* flag = reinterpret_cast<volatile int*>(smem + S::OFF_SLOT + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const KvShape& sh = a.sh;

  kv_begin();
  // the work of this block, the longest row tiles of the batch first
  const int per_pair = sh.kv_heads * a.kb.batch * a.splits;
  const int pair = pairs_max - 1 - (int)(blockIdx.x / per_pair), rest = blockIdx.x % per_pair;
  const int split = rest % a.splits, h = (rest / a.splits) % sh.kv_heads, b = rest / (a.splits * sh.kv_heads);
  const KvSeq s = kv_seq(a.kb, b);
  const int rows = s.n * sh.group;                               // of this kv head
  if (pair * 2 * PT_ROWS >= rows) return;
  int steps[2];                                                   // steps that the rows of each row tile can see
  for (int i = 0; i < 2; ++i) {
    const int r0 = (pair * 2 + i) * PT_ROWS, last = (r0 + PT_ROWS < rows ? r0 + PT_ROWS : rows) - 1;
    const int lim = r0 < rows ? s.first + last / sh.group : -1;
    steps[i] = lim < 0 ? 0 : lim / PT_HALF + 1;
  }
  const int most = ((steps[0] > steps[1] ? steps[0] : steps[1]) + 1) >> 1, per_split = (most + a.splits - 1) / a.splits;
  const int first = split * per_split;                            // tiles first ... of this part
  const int stop = first + per_split < most ? first + per_split : most, count = stop > first ? stop - first : 0;
  int mine_of[2];                                                 // its steps that each row tile sees
  for (int i = 0; i < 2; ++i) {
    const int n = (steps[i] < 2 * stop ? steps[i] : 2 * stop) - 2 * first;
    mine_of[i] = count > 0 && n > 0 ? n : 0;
  }

  if (threadIdx.x == 0) {
    *flag = 0;
    ptx::mbar_init(q_full, 8);
    for (int x = 0; x < 2; ++x) {
      ptx::mbar_init(k_full(x), PT_CONV);
      ptx::mbar_init(k_empty(x), 2);
      ptx::mbar_init(v_full(x), PT_CONV);
      ptx::mbar_init(v_empty(x), 2);
      for (int y = 0; y < 2; ++y) { ptx::mbar_init(s_full(x, y), 1); ptx::mbar_init(p_full(x, y), 4); ptx::mbar_init(o_done(x, y), 1); }
    }
    for (int x = 0; x < PT_RING; ++x) ptx::mbar_init(r_used(x), PT_CONV);
    for (int x = 0; x < 2; ++x) { ptx::mbar_init(c_full(x), 1); ptx::mbar_init(c_empty(x), PT_CONV); ptx::mbar_init(given_up(x), 1); }
    ptx::fence_mbar_init();
  }
  if (warp == PT_ISSUE) {
    __syncwarp();
    ptx::tmem_alloc(ptx::smem_u32(tmem_slot), 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  constexpr uint32_t COL_O = 256;                                // S (and P) of row tile i at columns 128 i and 128 i + 64, O at 256 + 128 i

  if (warp < 8) {
    // ------------------------------------------------------------------------------ softmax ----
    kvp::more_registers<176>();
    const int i = warp >> 2, quarter = warp & 3, row = quarter * 32 + lane;
    const int r = (pair * 2 + i) * PT_ROWS + row;
    const bool there = r < rows;
    const int tok = s.row0 + (there ? r / sh.group : 0), head = h * sh.group + (there ? r % sh.group : 0);
    const int limit = there ? s.first + r / sh.group : -1;
    const int limit_lo = __reduce_min_sync(0xffffffffu, limit);
    const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
    const uint32_t t_s = tmem + lane_base + 128 * i, t_o = tmem + lane_base + COL_O + 128 * i;
    const long long slot = ((long long)h * a.slots + first_slot(sh, s, b) + pair * 2 + i);
    const bool tile_there = (pair * 2 + i) * PT_ROWS < rows;
    // A warp moves its 32 rows of Q and of the output LANES lanes to a row, so that an access covers whole rows: a thread
    // to a row would touch 32 lines at a time, 64 times the 256-byte rows' share of the load unit.
    constexpr int LANES = D / 8, AT_ONCE = 32 / LANES, MOVES = 32 / AT_ONCE;
    const int part = lane / LANES, piece = lane % LANES;
    const long long out_row = there ? (long long)tok * sh.heads + head : -1;
    float factor;                                                // softmax_scale * log2(e) / (the row's power of two)
    {
      const long long q_row = there && QALORA_CHECK(dbg, tok, a.kb.m) ? (long long)tok * a.at.q_stride + (long long)head * D : -1;
      uint8_t* tile = smem + S::OFF_Q + i * S::TILE;
#pragma unroll 4
      for (int x = 0; x < MOVES; ++x) {
        const int at_row = x * AT_ONCE + part, tile_row = quarter * 32 + at_row;
        const long long from = __shfl_sync(0xffffffffu, q_row, at_row);
        uint8_t* to = tile + (piece >> 3) * 16384 + tile_row * 128 + (((piece & 7) ^ (tile_row & 7)) << 4);
        if (from >= 0) kvp::copy16_async(ptx::smem_u32(to), reinterpret_cast<const uint4*>(a.at.q + from) + piece);
        else *reinterpret_cast<uint4*>(to) = make_uint4(0, 0, 0, 0);
      }
      kvp::copies_done();
      __syncwarp();
      // each row's largest element is brought to 2^14 .. 2^15: exact in fp16 down to 2^-28 of it
      uint8_t* mine = tile + row * 128;
      uint32_t mx = 0;
#pragma unroll 4
      for (int c = 0; c < D / 8; ++c) {
        const uint4 v = *reinterpret_cast<const uint4*>(mine + (c >> 3) * 16384 + (((c & 7) ^ (row & 7)) << 4));
        mx = __vmaxu2(mx, __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu)));
      }
      mx = max(mx & 0xffffu, mx >> 16);
      int e = 268 - (int)(mx >> 7);
      e = e > 254 ? 254 : (e < 1 ? 1 : e);
      const float f = __uint_as_float((uint32_t)e << 23);
      factor = a.at.softmax_scale * kLog2e * (e == 254 ? 0x1p-127f : __uint_as_float((uint32_t)(254 - e) << 23));
#pragma unroll 4
      for (int c = 0; c < D / 8; ++c) {
        uint4* at = reinterpret_cast<uint4*>(mine + (c >> 3) * 16384 + (((c & 7) ^ (row & 7)) << 4));
        const uint4 v = *at;
        const uint32_t in[4] = {v.x, v.y, v.z, v.w};
        uint32_t to[4];
#pragma unroll
        for (int y = 0; y < 4; ++y)
          to[y] = kvp::pack_half2(__uint_as_float(in[y] << 16) * f, __uint_as_float(in[y] & 0xffff0000u) * f);
        *at = make_uint4(to[0], to[1], to[2], to[3]);
      }
      ptx::fence_proxy_async();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(q_full);
      if (a.q_image != nullptr && tile_there && split == 0 && QALORA_CHECK(dbg, slot, a.slots * sh.kv_heads)) {
#pragma unroll 4
        for (int x = 0; x < D / 8; ++x) {
          const int of = (x >> 3) * 16384 + quarter * 4096 + (x & 7) * 512 + lane * 16;
          *reinterpret_cast<uint4*>(a.q_image + slot * S::TILE + of) = *reinterpret_cast<const uint4*>(tile + of);
        }
      }
    }
    SoftmaxRow w{factor, kNoMax, 0.f, 0.f};
    bool ok = true;
    const int n_steps = mine_of[i];
    const bool some = n_steps > 0;
    // S of a step, asked for while the one before is worked on
    float x[PT_HALF];
    auto ask = [&](int step) {
      if (step >= n_steps) return true;
      if (!__all_sync(0xffffffffu, ptx::mbar_wait(s_full(i, step), (step >> 1) & 1, flag))) return false;
      ptx::tc_fence_after();
      ptx::tmem_ld32(t_s + PT_HALF * (step & 1), reinterpret_cast<uint32_t*>(x));
      return true;
    };
    auto ask_rest = [&](int step) { if (step < n_steps) ptx::tmem_ld32(t_s + PT_HALF * (step & 1) + 32, reinterpret_cast<uint32_t*>(x + 32)); };
    auto work = [&](int step) {
      const uint32_t t_mine = t_s + PT_HALF * (step & 1);
      const float4* rg = reinterpret_cast<const float4*>(ring + ((step >> 1) % PT_RING) * PT_RING_FLOATS) + (step & 1);
      const float4 k = rg[0], off = rg[2], inv = rg[4];
      float4 c = make_float4(fmaxf(factor * k.x, kTiny), fmaxf(factor * k.y, kTiny), fmaxf(factor * k.z, kTiny), fmaxf(factor * k.w, kTiny));
      const float4 refs = rg[6 - (step & 1)];                    // {reference before the tile / in it, in it, -, largest scale of keys}
      const bool large = factor * refs.w > kLargeFactor;
      const float ref_ratio = (step & 1) == 0 ? refs.x : 1.f;
      w.ref = refs.y;
      const int t0 = (2 * first + step) * PT_HALF;
      ptx::tmem_wait_ld();
      const float most = softmax_top(x, c, off, t0 + PT_HALF - 1 > limit_lo, limit - t0);
      float m = w.m;
      if (__any_sync(0xffffffffu, most > m + kGrow || large) || ref_ratio != 1.f) {
        // Rare: the maximum and the outputs are brought up to date.  With a larger reference the logarithms of all relative
        // scales fall, and the maximum with them; else the weights of values like the earlier ones would sink into fp16's
        // subnormals.  The sum, which no scale enters, grows in turn, so that the fall is limited.
        float fall = 0.f;
        if (ref_ratio != 1.f) fall = fmaxf(fmaxf(log2f(ref_ratio), kLeastExponent), fminf(log2f(w.l) - kMostSum, 0.f));
        const float top = fmaxf(w.m + fall, most), by = exp2f(w.m - top), scale = by * ref_ratio;
        m = w.m = top;
        w.l *= by;
        if (step > 0) {
          if (!__all_sync(0xffffffffu, ptx::mbar_wait(o_done(i, step - 1), ((step - 1) >> 1) & 1, flag))) return false;
          ptx::tc_fence_after();
#pragma unroll 1
          for (int q = 0; q < D / 16; ++q) {
            uint32_t o[16];
            kvp::tmem_ld16(t_o + 16 * q, o);
            ptx::tmem_wait_ld();
#pragma unroll
            for (int t = 0; t < 16; ++t) o[t] = __float_as_uint(__uint_as_float(o[t]) * scale);
            ptx::tmem_st16(t_o + 16 * q, o);
          }
        }
        if (large) {
          // The weights' exponents are a fused product minus a rounded maximum, which of scores beyond 2^27 may be any number.
          // So the product is rounded too, and its difference from the maximum bounded.  (That such scores are looked for at all:
          // 178.1 us and 179.2 for a 4096-token prompt of 32 heads of 128.)
          const float cs[4] = {c.x, c.y, c.z, c.w}, os[4] = {off.x, off.y, off.z, off.w};
#pragma unroll
          for (int t = 0; t < PT_HALF; ++t)
            x[t] = kvp::min_nan(__fadd_rn(__fmul_rn(x[t], cs[t >> 4]), -m), kGrow - os[t >> 4]);
          c = make_float4(1.f, 1.f, 1.f, 1.f);
          m = 0.f;
        }
      }
      softmax_exp<0>(w, m, x, c, off, inv, t_mine);
      softmax_exp<1>(w, m, x, c, off, inv, t_mine);
      ptx::tmem_wait_st();
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(p_full(i, step));
      if (!ask(step + 1)) return false;
      ask_rest(step + 1);
      return true;
    };
    if ((pair * 2 + i) * PT_ROWS + quarter * 32 < rows) {
      ok = ask(0);
      ask_rest(0);
#pragma unroll 1
      for (int step = 0; step < n_steps && ok; ++step) ok = work(step);
    } else {
      // none of the warp's rows is there: whatever its part of P holds reaches only its own rows of O, which nobody reads
      // (four drafted tokens of 31 sequences of up to 23 159 tokens, 16 heads on 2 of 64, weights gathered: 324 us -> 300)
#pragma unroll 1
      for (int step = 0; step < n_steps && ok; ++step) {
        ok = __all_sync(0xffffffffu, ptx::mbar_wait(s_full(i, step), (step >> 1) & 1, flag));
        if (ok && lane == 0) ptx::mbar_arrive(p_full(i, step));
      }
    }
    if (some && ok) ok = __all_sync(0xffffffffu, ptx::mbar_wait(o_done(i, n_steps - 1), ((n_steps - 1) >> 1) & 1, flag));
    ptx::tc_fence_after();
    const float m = w.m, l = w.l, ref = w.ref;
    const bool partial = a.splits > 1;
    const long long prow = slot * PT_ROWS + row;
    if (a.rows != nullptr && tile_there && split == 0 && QALORA_CHECK(dbg, slot, a.slots * sh.kv_heads)) {
      a.rows[slot * 2 * PT_ROWS + row] = fmaxf(factor, kTiny);
      a.rows[slot * 2 * PT_ROWS + PT_ROWS + row] = !partial && there ? minus_log2_sum(m, l) : -INFINITY;
      if (!partial && there && l != l) spoil_row<D>(a.q_image, slot, row);
    }
    if (partial && tile_there) {
      const long long at = (long long)split * a.slots * sh.kv_heads * PT_ROWS + prow;
      if (QALORA_CHECK(dbg, slot, a.slots * sh.kv_heads)) a.part_ml[at] = make_float2(m, l);
    }
    const float by = l == 0.f ? 0.f : __fdiv_rn(1.f, l);         // (not ref / l: the reference may be the least number there is)
    // through a quarter of the tile of Q, CHUNKS pieces of 16 bytes of a row at a time in an order that keeps both sides
    // free of bank conflicts.  With 128 channels that quarter holds rows of Q that other warps of the row tile fetched.
    // o_done says that the products are done with them; where there is no product, in a part of the tokens that the row tile does
    // not see, the four warps meet instead, so that nobody's rows are still on their way.
    if (!some) { if (i == 0) ptx::named_barrier(1, 128); else ptx::named_barrier(2, 128); }
    constexpr int CHUNKS = D / 8;
    uint8_t* stage = smem + S::OFF_Q + i * S::TILE + quarter * (S::TILE / 4);
    auto place = [&](int of, int c) { return stage + of * (16 * CHUNKS) + ((c ^ (of & 7)) << 4); };
    const int channels = partial ? 4 * CHUNKS : 8 * CHUNKS;      // of a pass
    const bool store = tile_there && QALORA_CHECK(dbg, slot, a.slots * sh.kv_heads);
    const long long at = there && QALORA_CHECK(dbg, out_row, (long long)a.kb.m * sh.heads) ? out_row : -1;
#pragma unroll 1
    for (int q = 0; q < D; q += channels) {
#pragma unroll 1
      for (int c = 0; c < channels; c += 16) {
        uint32_t o[16];
        if (some && ok) {
          kvp::tmem_ld16(t_o + q + c, o);
          ptx::tmem_wait_ld();
        }
        float f[16];
#pragma unroll
        for (int t = 0; t < 16; ++t) f[t] = !some || !ok || l == 0.f ? 0.f : __uint_as_float(o[t]) * by * ref;
        if (partial) {
#pragma unroll
          for (int t = 0; t < 4; ++t) *reinterpret_cast<float4*>(place(lane, (c >> 2) + t)) = make_float4(f[4 * t], f[4 * t + 1], f[4 * t + 2], f[4 * t + 3]);
        } else {
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            uint32_t v[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const __nv_bfloat162 two = __floats2bfloat162_rn(f[8 * t + 2 * y], f[8 * t + 2 * y + 1]);
              v[y] = *reinterpret_cast<const uint32_t*>(&two);
            }
            *reinterpret_cast<uint4*>(place(lane, (c >> 3) + t)) = make_uint4(v[0], v[1], v[2], v[3]);
          }
        }
      }
      __syncwarp();
#pragma unroll 4
      for (int x = 0; x < MOVES; ++x) {
        const int from = x * AT_ONCE + part;
        const uint4 v = *reinterpret_cast<const uint4*>(place(from, piece));
        const long long to = __shfl_sync(0xffffffffu, at, from);
        if (partial) {
          if (store) *reinterpret_cast<uint4*>(a.part_o + ((long long)split * a.slots * sh.kv_heads * PT_ROWS + slot * PT_ROWS + quarter * 32 + from) * D + q + 4 * piece) = v;
        } else if (to >= 0) {
          *reinterpret_cast<uint4*>(a.at.out + to * D + 8 * piece) = v;
        }
      }
      __syncwarp();
    }
    if (!partial && there) kvp::store_lse(a.at.lse, out_row, nullptr, 0, m, l, kLift);
  } else if (warp < PT_ISSUE) {
    // --------------------------------------------------------------------------- conversion ----
    kvp::fewer_registers<40>();
    const int t = threadIdx.x - 256;
    auto wait = [&](uint32_t bar, int phase) { return __all_sync(0xffffffffu, ptx::mbar_wait(bar, phase & 1, flag)); };
    bool ok = true;
#pragma unroll 1
    for (int it = 0; it < count && ok; ++it) {
      const int st = it & 1, rows_here = s.len - (first + it) * PT_TOK;
      const int* ids = reinterpret_cast<const int*>(ring + (it % PT_RING) * PT_RING_FLOATS) + 32;
#pragma unroll 1
      for (int w = 0; w < 2; ++w) {                              // keys, values
        if (!(ok = wait(c_full(w), it))) break;
        if (it >= 2 && !(ok = wait(w == 0 ? k_empty(st) : v_empty(st), (it >> 1) - 1))) break;
        convert_tile<D>(smem + S::OFF_STAGED + w * S::STAGED, smem + (w == 0 ? S::OFF_K : S::OFF_V) + st * S::TILE, ids[-6] != 0, ids + 8 * w, rows_here, t);
        ptx::fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
          ptx::mbar_arrive(c_empty(w));
          ptx::mbar_arrive(w == 0 ? k_full(st) : v_full(st));
          if (w == 1) ptx::mbar_arrive(r_used(it % PT_RING));
        }
      }
    }
  } else {
    // --------------------------------------------------------------------------- MMA issuers ----
    kvp::fewer_registers<40>();
    const int i = __shfl_sync(0xffffffffu, warp, 0) - PT_ISSUE;
    if (i < 2) {
      const uint32_t leader = kvp::elect_one();
      constexpr uint32_t IDESC_S = kvp::idesc_f16(128, PT_HALF, false, false), IDESC_O = kvp::idesc_f16(128, D, false, true);
      const uint32_t t_s = tmem + 128 * i, t_o = tmem + COL_O + 128 * i;
      const uint64_t q_desc = ptx::smem_desc(sbase + S::OFF_Q + i * S::TILE, 16, 1024);
      auto wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, ptx::mbar_wait(bar, parity, flag)); };
      bool ok = count == 0 || wait(q_full, 0);
      const int n_steps = mine_of[i];
      auto scores = [&](int step) {                              // S of a step
        const int it = step >> 1, st = it & 1;
        if ((step & 1) == 0 && !wait(k_full(st), (it >> 1) & 1)) return false;
        if (step < n_steps) {
          if (step >= 2 && !wait(o_done(i, step), ((step >> 1) - 1) & 1)) return false;      // P V of the step two before
          ptx::tc_fence_after();
          const uint64_t k_desc = ptx::smem_desc(sbase + S::OFF_K + st * S::TILE, 16, 1024) + (uint64_t)((step & 1) * 512);
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint64_t at = (uint64_t)((k >> 2) * 1024 + (k & 3) * 2);      // 16 channels; 64 to a block of 16 KiB
            kvp::mma_ss(leader, t_s + PT_HALF * (step & 1), q_desc + at, k_desc + at, IDESC_S, k > 0 ? 1u : 0u);
          }
          kvp::mma_commit(leader, s_full(i, step));
        }
        if ((step & 1) == 1) {                                   // the keys of the tile are done with
          if (step - 1 < n_steps) kvp::mma_commit(leader, k_empty(st));
          else if (leader) ptx::mbar_arrive(k_empty(st));
        }
        __syncwarp();
        return true;
      };
      ok = ok && (count == 0 || (scores(0) && scores(1)));
      for (int step = 0; step < 2 * count && ok; ++step) {
        const int it = step >> 1, st = it & 1;
        if ((step & 1) == 0 && !(ok = wait(v_full(st), (it >> 1) & 1))) break;
        if (step < n_steps) {
          if (!(ok = wait(p_full(i, step), it & 1))) break;
          ptx::tc_fence_after();
          const uint64_t v_desc = ptx::smem_desc(sbase + S::OFF_V + st * S::TILE, 16384, 1024) + (uint64_t)((step & 1) * 512);
#pragma unroll
          for (int k = 0; k < PT_HALF / 16; ++k)
            kvp::mma_ts(leader, t_o, t_s + PT_HALF * (step & 1) + 8 * k, v_desc + (uint64_t)(k * 128), IDESC_O, step > 0 || k > 0 ? 1u : 0u);
          kvp::mma_commit(leader, o_done(i, step));
        }
        if ((step & 1) == 1) {                                   // and its values
          if (step - 1 < n_steps) kvp::mma_commit(leader, v_empty(st));
          else if (leader) ptx::mbar_arrive(v_empty(st));
        }
        __syncwarp();
        if (step + 2 < 2 * count) ok = scores(step + 2);
      }
      if (!ok) {                                                 // (the limit of a wait holds here too)
        kvp::mma_commit(leader, given_up(i));
        wait(given_up(i), 0);
      }
    } else if (i == 2) {
      // ------------------------------------------------------------------------- look-ups ----
      // lane l < 8: block and scales of tokens 16 l ... of a tile, each step of the chain table -> scales asked for one
      // tile before it is needed
      auto entry = [&](int it) {
        const int t0 = (first + it) * PT_TOK + lane * 16;
        return lane < 8 && it < count && t0 < s.len ? a.kb.table[(size_t)b * a.kb.max_blocks + (t0 >> sh.log_block)] : -1;
      };
      struct Look { int id; float ks, vs; };
      auto look = [&](int raw) {
        const int id = raw >= 0 && raw < sh.num_blocks ? raw : -1;
        const long long plane = ((long long)(id < 0 ? 0 : id) * 2) * sh.kv_heads + h;
        return Look{id, a.at.scales[plane], a.at.scales[plane + sh.kv_heads]};
      };
      Look next = look(entry(0));
      int after = entry(1);
      float ref = 0.f;
      int sent[2] = {0, 0};                                      // tiles of keys, of values
      for (int it = 0; it < count; ++it) {
        const Look cur = next;
        next = look(after);
        after = entry(it + 2);
        // value scales relative to the largest one so far; blocks far below it (or of zeros) count as zeros
        const float ks = cur.id >= 0 ? cur.ks : 0.f, vs = cur.id >= 0 ? cur.vs : 0.f;
        float top = vs, k_top = ks;
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) {
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
          k_top = fmaxf(k_top, __shfl_xor_sync(0xffffffffu, k_top, o));
        }
        k_top = __shfl_sync(0xffffffffu, k_top, 0);
        top = fmaxf(ref, __shfl_sync(0xffffffffu, top, 0));
        const float ratio = ref == top ? 1.f : ref / top;
        const float rel = top > 0.f ? vs / top : 0.f, least = fmaxf(rel, kLeastValueScale);
        const int v_id = rel >= kLeastValueScale ? cur.id : -1;
        const bool all = __all_sync(0xffffffffu, lane >= 8 || v_id >= 0) && (first + it + 1) * PT_TOK <= s.len;
        ref = top;
        // The ring's entry is free once tile it - 4 has been converted: its values waited for P V of tile it - 6, hence
        // for that tile's softmax, which came after the one that read this entry (tile it - 8).
        if (it >= PT_RING && !__all_sync(0xffffffffu, ptx::mbar_wait(r_used((it - 4) % PT_RING), ((it - 4) / PT_RING) & 1, flag))) break;
        float* rg = ring + (it % PT_RING) * PT_RING_FLOATS;
        if (lane < 8) {
          rg[lane] = ks;
          const float off = log2f(least);
          rg[8 + lane] = off;
          rg[16 + lane] = exp2f(-off);             // (of the rounded logarithm: its error leaves the softmax's sum alone)
          reinterpret_cast<int*>(rg)[32 + lane] = cur.id;
          reinterpret_cast<int*>(rg)[40 + lane] = v_id;
        }
        if (lane == 8) { rg[24] = ratio; rg[25] = ref; reinterpret_cast<int*>(rg)[26] = all ? 1 : 0; rg[27] = k_top; }
        __syncwarp();
        // the codes of the blocks that are there, one copy each (a copy starts on a 16-byte boundary: blocks are multiples
        // of 1 KiB); lane 16-token group l stands for the block that begins with it
        const int groups = sh.block >> 4;
        const bool begins = lane < 8 && lane % groups == 0;
        bool ok = true;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const int id = w == 0 ? cur.id : v_id;
          const bool copies = begins && id >= 0;
          const int n = __popc(__ballot_sync(0xffffffffu, copies));
          if (it >= 1 && !(ok = __all_sync(0xffffffffu, ptx::mbar_wait(c_empty(w), (it - 1) & 1, flag)))) break;
          if (lane == 0) ptx::mbar_arrive_expect_tx(c_full(w), (uint32_t)(n * sh.block * D));
          __syncwarp();
          if (copies)
            ptx::bulk_load(sbase + S::OFF_STAGED + w * S::STAGED + lane * 16 * D,
                           a.at.codes + (((long long)id * 2 + w) * sh.kv_heads + h) * sh.block * D, (uint32_t)(sh.block * D), c_full(w));
          ++sent[w];
        }
        if (!ok) break;
      }
      // nothing is on its way to shared memory when the block ends, also where a wait ran out
#pragma unroll
      for (int w = 0; w < 2; ++w) if (sent[w] > 0) ptx::mbar_wait(c_full(w), (sent[w] - 1) & 1, flag);
    }
    __syncwarp();
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *flag != 0) *a.status = 1;
  if (warp == PT_ISSUE) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, 512);
  }
}

// Joins the parts of each row, in the order of the tokens: D / 4 threads per row.
template <int D>
__global__ void __launch_bounds__(256)
kv_prompt_join_kernel(const __grid_constant__ PromptArgs a, int row_blocks, int* dbg) {
  constexpr int PER_ROW = D / 4, ROWS = 256 / PER_ROW;
  kv_begin();
  const KvShape& sh = a.sh;
  const int b = blockIdx.y, h = blockIdx.x / row_blocks;
  const KvSeq s = kv_seq(a.kb, b);
  const int r = (blockIdx.x % row_blocks) * ROWS + threadIdx.x / PER_ROW, d = (threadIdx.x % PER_ROW) * 4;
  if (r >= s.n * sh.group) return;
  const long long prow = ((long long)h * a.slots + first_slot(sh, s, b)) * PT_ROWS + r, plane = a.slots * sh.kv_heads * PT_ROWS;
  if (!QALORA_CHECK(dbg, prow, plane)) return;
  float m = kNoMax, l = 0.f;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p = 0; p < a.splits; ++p) {
    const float2 v = a.part_ml[p * plane + prow];
    const float top = fmaxf(m, v.x);
    l = l * exp2f(m - top) + v.y * exp2f(v.x - top);
    m = top;
  }
  const float by = l == 0.f ? 0.f : __fdiv_rn(1.f, l);
  for (int p = 0; p < a.splits; ++p) {                            // (each part's output is its own weighted mean)
    const float2 v = a.part_ml[p * plane + prow];
    const float4 y = *reinterpret_cast<const float4*>(a.part_o + (p * plane + prow) * D + d);
    const float share = v.y * exp2f(v.x - m) * by;
    x.x = fmaf(y.x, share, x.x); x.y = fmaf(y.y, share, x.y); x.z = fmaf(y.z, share, x.z); x.w = fmaf(y.w, share, x.w);
  }
  const long long at = (long long)(s.row0 + r / sh.group) * sh.heads + h * sh.group + r % sh.group;
  kvp::store_row4(a.at.out + at * D + d, x);
  if (d == 0) {
    kvp::store_lse(a.at.lse, at, nullptr, 0, m, l, kLift);
    if (a.rows != nullptr) {
      a.rows[(prow / PT_ROWS * 2 + 1) * PT_ROWS + prow % PT_ROWS] = minus_log2_sum(m, l);
      if (l != l) spoil_row<D>(a.q_image, prow / PT_ROWS, (int)(prow % PT_ROWS));
    }
  }
}

template <int D>
struct PsSmem {
  static constexpr int TILE = 128 * D * 2, STAGES = 2;
  static constexpr int OFF_K = 0, OFF_Q = TILE;
  static constexpr int OFF_ROWS = OFF_Q + STAGES * TILE;         // [NROWS][2][128]: read after the tile itself is free
  static constexpr int NROWS = 4;
  static constexpr int OFF_SUM = OFF_ROWS + NROWS * 128 * 8;     // [2][128] sums of the second half; of the block
  static constexpr int OFF_BARS = OFF_SUM + 1024;
  static constexpr int NBARS = 1 + 2 * STAGES + 2 * 2 + 1;
  static constexpr int OFF_SLOT = OFF_BARS + NBARS * 8 + 8;
  static constexpr int TOTAL = OFF_SLOT + 16 + 1024;
};

// 2^y of two values on the FMA pipe: y = n + r with |r| <= 1/2 by adding 1.5 * 2^23, 2^r by its minimax polynomial
// of degree 5 (Remez exchange on the relative error: 7.5e-8, 2.2e-7 = 2^-22.1 with the roundings of its evaluation, as the
// exponential unit's), times 2^n.  y <= 126; a y of -126.5 or less gives 0 (its 2^n has no bits
// left), NaN gives NaN.
__device__ __forceinline__ float2 exp2_fma(float2 y) {
  y.x = kvp::max_nan(y.x, -127.f);
  y.y = kvp::max_nan(y.y, -127.f);
  const float2 n = ptx::fadd2(y, make_float2(12582912.f, 12582912.f));
  const float2 r = ptx::ffma2(ptx::fadd2(n, make_float2(-12582912.f, -12582912.f)), make_float2(-1.f, -1.f), y);
  float2 p = make_float2(0.00132764725f, 0.00132764725f);
  p = ptx::ffma2(p, r, make_float2(0.00967554096f, 0.00967554096f));
  p = ptx::ffma2(p, r, make_float2(0.0555071309f, 0.0555071309f));
  p = ptx::ffma2(p, r, make_float2(0.240221202f, 0.240221202f));
  p = ptx::ffma2(p, r, make_float2(0.693146944f, 0.693146944f));
  p = ptx::ffma2(p, r, make_float2(1.00000012f, 1.00000012f));
  return ptx::fmul2(p, make_float2(__uint_as_float((__float_as_uint(n.x) << 23) + 0x3f800000u),
                                   __uint_as_float((__float_as_uint(n.y) << 23) + 0x3f800000u)));
}

// The weights that 128 tokens of one kv head gather: S^T = K Q^T with the tokens as the rows of the product, so
// that a thread owns a token and adds up exp2(S * factor - lse) over the rows without any exchange.
// The row tiles come as the images that kv_prompt_kernel left; where there are few token tiles, a cluster of blocks
// shares a tile's row tiles and adds its sums, in the order of the blocks, through distributed shared memory.  Two
// groups of 128 threads, each with its accumulator, take the row tiles in turn, and two blocks share a multiprocessor,
// so that one's tile of keys is fetched and its products run while the other's exponentials do.  Those bound it: two
// pieces of up to 700 tokens, 32 heads of 64, against up to 12345 cached ones 180 us with one block of four
// accumulators, 138 with two blocks (the exponential unit busy for 71 % of the time), 128 with a quarter of the
// exponentials on the FMA pipe (an eighth 133, three eighths 135, half 145).  The unit is then busy for 56 % of the time and
// the issue slots for 52 %, so that neither is a limit by itself.
// COLS: groups of 32 rows of a row tile that may be there (one where a sequence has 32 rows at most).
template <int D, int COLS>
__global__ void __launch_bounds__(320, 2)
kv_prompt_score_kernel(const __grid_constant__ PromptArgs a, int* dbg) {
  using S = PsSmem<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (ptx::smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t sbase = ptx::smem_u32(smem), bars = sbase + S::OFF_BARS;
  const uint32_t k_full = bars;
  auto q_full = [&](int x) { return bars + 8 + 8 * x; };
  auto q_empty = [&](int x) { return bars + 8 + 8 * (S::STAGES + x); };
  auto s_full = [&](int x) { return bars + 8 + 8 * (2 * S::STAGES + x); };
  auto s_empty = [&](int x) { return bars + 8 + 8 * (2 * S::STAGES + 2 + x); };
  const uint32_t given_up = bars + 8 + 8 * (2 * S::STAGES + 4);                 // as in kv_prompt_kernel
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + S::OFF_SLOT);
  volatile int* flag = reinterpret_cast<volatile int*>(smem + S::OFF_SLOT + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  kv_begin();
  const KvShape& sh = a.sh;
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), unit = blockIdx.x / C;
  const int b = blockIdx.y, h = unit % sh.kv_heads, j = unit / sh.kv_heads, t0 = j * PT_TOK;
  const KvSeq s = kv_seq(a.kb, b);
  if (s.n == 0 || t0 >= s.len) return;                           // (the same for the whole cluster)
  const int rows = s.n * sh.group, row_tiles = (rows + PT_ROWS - 1) / PT_ROWS;
  const int seen = t0 > s.first ? (int)(((long long)(t0 - s.first) * sh.group) / PT_ROWS) : 0;   // the first that sees a token of the tile
  const int share = (row_tiles - seen + C - 1) / C, rt0 = seen + rank * share;                   // this block's row tiles
  const int count = rt0 >= row_tiles ? 0 : (rt0 + share < row_tiles ? share : row_tiles - rt0);
  const long long slot0 = (long long)h * a.slots + first_slot(sh, s, b) + rt0;

  if (threadIdx.x == 0) {
    *flag = 0;
    ptx::mbar_init(k_full, 8);
    for (int x = 0; x < S::STAGES; ++x) { ptx::mbar_init(q_full(x), 1); ptx::mbar_init(q_empty(x), 1); }
    for (int x = 0; x < 2; ++x) { ptx::mbar_init(s_full(x), 1); ptx::mbar_init(s_empty(x), 4); }
    ptx::mbar_init(given_up, 1);
    ptx::fence_mbar_init();
  }
  if (warp == 8) {
    __syncwarp();
    ptx::tmem_alloc(ptx::smem_u32(tmem_slot), 256);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  float* sums = reinterpret_cast<float*>(smem + S::OFF_SUM);
  int id = -1;                                                   // block of the thread's token
  float before = 0.f;                                            // what the token had gathered

  if (warp < 8) {
    const int half = warp >> 2, quarter = warp & 3, token = quarter * 32 + lane;
    {
      using Map = TileMap<D, 256>;
      const Map map(threadIdx.x);
#pragma unroll
      for (int p = 0; p < Map::PASSES; ++p) {
        const int row = p * Map::ROWS + map.row0, t = t0 + row;
        uint4 c = make_uint4(0, 0, 0, 0);
        if (t < s.len) {
          const int from = kv_block(a.kb.table, a.kb.max_blocks, sh.num_blocks, b, t >> sh.log_block);
          if (from >= 0)
            c = *reinterpret_cast<const uint4*>(a.at.codes + ((((long long)from * 2) * sh.kv_heads + h) * sh.block + (t & (sh.block - 1))) * D + map.piece * 16);
        }
        store_codes(smem + S::OFF_K, row, map.piece, c);
      }
      ptx::fence_proxy_async();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(k_full);
    }
    const int t = t0 + token;
    if (t < s.len) id = kv_block(a.kb.table, a.kb.max_blocks, sh.num_blocks, b, t >> sh.log_block);
    const float ks = id >= 0 ? a.at.scales[((long long)id * 2) * sh.kv_heads + h] : 0.f;
    const long long own = ((long long)id * sh.kv_heads + h) * sh.block + (t & (sh.block - 1));
    if (half == 0 && rank == 0 && id >= 0 && a.at.score_in != nullptr) before = a.at.score_in[own];
    // the first row of this tile's first row tile that sees the token (rows before it are masked)
    const long long sees = t > s.first ? (long long)(t - s.first) * sh.group - (long long)rt0 * PT_ROWS : 0;
    const float2 kk = make_float2(fmaxf(ks, kTiny), fmaxf(ks, kTiny));
    float sum = 0.f;
    bool ok = true;
#pragma unroll 1
    for (int it = half; it < count; it += 2) {
      if (!(ok = __all_sync(0xffffffffu, ptx::mbar_wait(s_full(half), (it >> 1) & 1, flag)))) break;
      ptx::tc_fence_after();
      const float4* rw = reinterpret_cast<const float4*>(smem + S::OFF_ROWS) + (it % S::NROWS) * 64;
      const int skip = sees > (long long)it * PT_ROWS ? (int)(sees - (long long)it * PT_ROWS < 128 ? sees - (long long)it * PT_ROWS : 128) : 0;
      const bool edge = __any_sync(0xffffffffu, skip > 0);
      float2 part[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
      for (int q = 0; q < COLS; ++q) {
        float v[32];
        ptx::tmem_ld32(tmem + ((uint32_t)(quarter * 32) << 16) + 128 * half + 32 * q, reinterpret_cast<uint32_t*>(v));
        ptx::tmem_wait_ld();
        if (edge) {
#pragma unroll
          for (int x = 0; x < 32; ++x) if (32 * q + x < skip) v[x] = -INFINITY;
        }
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const float4 f = rw[8 * q + x], g = rw[32 + 8 * q + x];           // factors and -log2 of the sums of four rows
          float2 e0 = ptx::ffma2(ptx::fmul2(make_float2(v[4 * x], v[4 * x + 1]), kk), make_float2(f.x, f.y), make_float2(g.x, g.y));
          float2 e1 = ptx::ffma2(ptx::fmul2(make_float2(v[4 * x + 2], v[4 * x + 3]), kk), make_float2(f.z, f.w), make_float2(g.z, g.w));
          e0.x = kvp::exp2_fast(e0.x); e0.y = kvp::exp2_fast(e0.y);
          if (x % 2 == 1) {                                      // a quarter of them
            e1 = exp2_fma(e1);
          } else {
            e1.x = kvp::exp2_fast(e1.x);
            e1.y = kvp::exp2_fast(e1.y);
          }
          part[0] = ptx::fadd2(part[0], e0);
          part[1] = ptx::fadd2(part[1], e1);
        }
      }
      part[0] = ptx::fadd2(part[0], part[1]);
      sum += part[0].x + part[0].y;
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(s_empty(half));
    }
    if (half == 1) sums[token] = sum;
    ptx::named_barrier(1, 256);
    if (half == 0) sums[128 + token] = sum + sums[token];
  } else if (warp == 8) {
    if (lane == 0) {
      constexpr uint32_t IDESC = kvp::idesc_f16(128, 128, false, false);
      const uint64_t k_desc = ptx::smem_desc(sbase + S::OFF_K, 16, 1024);
      bool ok = ptx::mbar_wait(k_full, 0, flag);
      for (int it = 0; it < count && ok; ++it) {
        const int st = it % S::STAGES, buf = it & 1;
        if (!(ok = ptx::mbar_wait(q_full(st), (it / S::STAGES) & 1, flag))) break;
        if (it >= 2 && !(ok = ptx::mbar_wait(s_empty(buf), ((it >> 1) - 1) & 1, flag))) break;
        ptx::tc_fence_after();
        const uint64_t q_desc = ptx::smem_desc(sbase + S::OFF_Q + st * S::TILE, 16, 1024);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint64_t step = (uint64_t)((k >> 2) * 1024 + (k & 3) * 2);
          ptx::mma_ss(tmem + 128 * buf, k_desc + step, q_desc + step, IDESC, k > 0 ? 1u : 0u);
        }
        ptx::mma_commit(s_full(buf));
        ptx::mma_commit(q_empty(st));
      }
      if (!ok) {
        ptx::mma_commit(given_up);
        ptx::mbar_wait(given_up, 0, flag);
      }
    }
    __syncwarp();
  } else {
    if (lane == 0) {
      int it = 0;
      for (; it < count; ++it) {
        const int st = it % S::STAGES;
        if (it >= S::STAGES && !ptx::mbar_wait(q_empty(st), ((it / S::STAGES) - 1) & 1, flag)) break;
        // (the rows' entry was last read for the tile four before, whose accumulator has since been handed back: the
        // product of the tile two before, which is done, went there)
        if (!QALORA_CHECK(dbg, slot0 + it, a.slots * sh.kv_heads)) break;
        ptx::mbar_arrive_expect_tx(q_full(st), S::TILE + 1024);
        ptx::bulk_load(sbase + S::OFF_Q + st * S::TILE, a.q_image + (slot0 + it) * S::TILE, S::TILE, q_full(st));
        ptx::bulk_load(sbase + S::OFF_ROWS + (it % S::NROWS) * 1024, a.rows + (slot0 + it) * 2 * PT_ROWS, 1024, q_full(st));
      }
      for (int i = it < S::STAGES ? 0 : it - S::STAGES; i < it; ++i) ptx::mbar_wait(q_full(i % S::STAGES), (i / S::STAGES) & 1, flag);
    }
    __syncwarp();
  }
  ptx::tc_fence_before();
  if (C == 1) __syncthreads(); else cluster.sync();
  if (threadIdx.x < 128 && rank == 0 && id >= 0) {
    float sum = 0.f;
    for (int r = 0; r < C; ++r) sum += cluster.map_shared_rank(sums, r)[128 + threadIdx.x];
    const long long at = ((long long)id * sh.kv_heads + h) * sh.block + ((t0 + threadIdx.x) & (sh.block - 1));
    if (QALORA_CHECK(dbg, at, (long long)sh.num_blocks * sh.kv_heads * sh.block))
      a.at.score_out[at] = before + sum;
  }
  if (threadIdx.x == 0 && *flag != 0) *a.status = 1;
  if (warp == 8) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, 256);
  }
  if (C > 1) cluster.sync();                                     // (a block's sums are read by its cluster until here)
}

template <int D>
int prompt(const PromptArgs& a, cudaStream_t st) {
  static PerDeviceOnce once, once_score;
  int ok = once.run([] {
    return cudaFuncSetAttribute(kv_prompt_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, PtSmem<D>::TOTAL);
  });
  if (ok != QALORA_OK) return ok;
  const KvShape& sh = a.sh;
  const long long rows_max = (long long)a.kb.max_new * sh.group;
  const int pairs = (int)((rows_max + 2 * PT_ROWS - 1) / (2 * PT_ROWS));
  const long long blocks = (long long)pairs * sh.kv_heads * a.kb.batch * a.splits;
  if (blocks > 0x7fffffffll) return QALORA_ERR_UNSUPPORTED_SHAPE;
  {
    MainKernelProbe probe("kv_prompt_kernel", st);
    ok = kv_launch(kv_prompt_kernel<D>, dim3((unsigned)blocks), PT_THREADS, (size_t)PtSmem<D>::TOTAL, st, a, pairs, debug_words());
  }
  if (ok != QALORA_OK) return ok;
  if (a.splits > 1) {
    constexpr int ROWS = 256 / (D / 4);
    const int row_blocks = (int)((rows_max + ROWS - 1) / ROWS);
    if ((long long)row_blocks * sh.kv_heads > 0x7fffffffll) return QALORA_ERR_UNSUPPORTED_SHAPE;
    ok = kv_launch(kv_prompt_join_kernel<D>, dim3((unsigned)(row_blocks * sh.kv_heads), (unsigned)a.kb.batch), 256, 0, st, a, row_blocks, debug_words());
    if (ok != QALORA_OK) return ok;
  }
  if (a.at.score_out != nullptr && a.kb.max_len > 0) {
    ok = once_score.run([] {
      const cudaError_t e = cudaFuncSetAttribute(kv_prompt_score_kernel<D, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, PsSmem<D>::TOTAL);
      return e != cudaSuccess ? e : cudaFuncSetAttribute(kv_prompt_score_kernel<D, 4>, cudaFuncAttributeMaxDynamicSharedMemorySize, PsSmem<D>::TOTAL);
    });
    if (ok != QALORA_OK) return ok;
    const int tiles = (a.kb.max_len + PT_TOK - 1) / PT_TOK;
    const long long units = (long long)tiles * sh.kv_heads, row_tiles = (rows_max + PT_ROWS - 1) / PT_ROWS;
    // Thread blocks per token tile, a cluster that shares its row tiles: while they all run at once, and each has two row
    // tiles at least.  (Both kernels, one and up to eight blocks: 2500 tokens of a sequence of 6000, 8 heads on one of 128,
    // 231 us and 144; a prompt of 1000 tokens, 16 heads on 2, 90 and 45; 700 tokens, 32 heads on 8, 50 and 39; 60 new
    // ones of 3000, 8 heads on one of 64, 26.8 and 26.1.)
    int C = 1;
    while (C < PS_MAX_CLUSTER && units * a.kb.batch * C * 2 <= 2ll * device_sm_count() && row_tiles >= 4 * C) C *= 2;
    if (units * C > 0x7fffffffll) return QALORA_ERR_UNSUPPORTED_SHAPE;
    // (a few drafted tokens of a large group of heads: four of 31 sequences of up to 23 159 tokens, 16 heads on 2 of 64, both
    // kernels 300 us with all four groups of rows, 284 with one)
    return kv_launch_clusters(rows_max <= 32 ? kv_prompt_score_kernel<D, 1> : kv_prompt_score_kernel<D, 4>, dim3((unsigned)(units * C), (unsigned)a.kb.batch), C, 320,
                              (size_t)PsSmem<D>::TOTAL, st, a, debug_words());
  }
  return QALORA_OK;
}

}  // namespace

KvPromptScratch kv_prompt_scratch(const KvShape& sh, int batch, int64_t m, int max_len, bool with_score) {
  KvPromptScratch s{};
  s.slots = (long long)m * sh.group / PT_ROWS + batch;
  // A row tile's tokens are cut into as many parts as make the grid's last wave end first: a part costs about ten tiles' time
  // beyond its own, its rows go through memory in float32, and it has two tiles at least.  (Two pieces of up to
  // 700 tokens, 32 heads on 8 of 64, against 12345 cached ones, weights gathered: 404 us uncut, 349 cut; a prompt of 1000
  // tokens with 8 heads of 128: 31 and 23.)
  const long long blocks = sh.kv_heads * ((long long)m * sh.group / (2 * PT_ROWS) + batch), tiles = ((long long)max_len + PT_TOK - 1) / PT_TOK;
  const long long sms = device_sm_count(), most = tiles / 2 < 2 * sms ? tiles / 2 : 2 * sms;
  long long splits = 1, least = 0;
  for (long long n = 1; n <= most || n == 1; ++n) {
    const long long cost = (blocks * n + sms - 1) / sms * ((tiles + n - 1) / n + 10) + (n > 1 ? 2 : 0);
    if (n == 1 || cost < least) { least = cost; splits = n; }
  }
  s.splits = (int)splits;
  const size_t rows = (size_t)s.slots * sh.kv_heads * PT_ROWS;
  s.part_ml = s.splits > 1 ? rows * s.splits * sizeof(float2) : 0;
  s.part_o = s.splits > 1 ? rows * s.splits * sh.dim * 4 : 0;
  s.q_image = with_score ? rows * sh.dim * 2 : 0;
  s.rows = with_score ? rows * sizeof(float2) : 0;
  return s;
}

int launch_kv_prompt(const KvShape& sh, const KvBatch& b, const KvAttention& at, const KvPromptScratch& s, float2* part_ml,
                     float* part_o, uint8_t* q_image, float* rows, int* status, cudaStream_t st) {
  const bool scores = at.score_out != nullptr;
  PromptArgs a{sh, b, at, s.splits, s.slots, part_ml, part_o, scores ? q_image : nullptr, scores ? rows : nullptr, status};
  return sh.dim == 128 ? prompt<128>(a, st) : prompt<64>(a, st);
}

}  // namespace qalora
