// Attention of a few new tokens over the 8-bit key/value cache (the generating step of a served
// model), bound by HBM: every cached code is read once per kv head.
#define QALORA_TU 12
#include <cuda_fp16.h>

#include "kv_ptx.cuh"
#include "kv.cuh"
#include "tc_host.cuh"

namespace qalora {

namespace {

constexpr int AT_WARPS = 4;                       // consumer warps; one more warp brings the tiles in
constexpr int AT_THREADS = (AT_WARPS + 1) * 32;
constexpr int AT_MAX_BATCH = 512;                 // sequences of one launch (their rows, lengths and units lie in shared memory)
constexpr int JOIN_TOKENS = 512;                  // whose gathered weights a block of the second kernel adds up
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNoMax = -3.40282347e38f;         // running maximum of a row that has met no token
constexpr float kGrow = 6.f;                      // a row is rescaled when its maximum has grown by 2^6 or more
constexpr float kLift = 8.f;                      // weighted value scales are kept times 2^8: below 2^15 in fp16, and 2^-22 of the
                                                  // largest still is an ordinary fp16 number
constexpr float kNoScale = -1000.f;               // exponent of a value scale of 0

struct AttnArgs {
  KvShape sh;
  KvBatch kb;
  KvAttention at;
  int* status;
  uint32_t* plan;        // [batch + 2]: first unit of each sequence, their number, units per thread block
  float* parts;          // partial results, two slots per thread block (see part_slot)
  float* lse2;           // [sequence][n_hi][heads] log2 of the row's sum, for the gathered weights
  float* logits;         // [sequence][n_hi][heads][logit_stride] scaled scores in powers of two, or NULL
  long long logit_stride;
  int batch0;            // first sequence of this launch
  int units_grid;        // thread blocks of the first kernel
  int whole;             // each of them takes all units of one (sequence, kv head)
};

// Work is cut into units of TOK tokens of one (sequence, kv head), in this order; every thread block takes the same number
// of consecutive units, whatever the sequences' lengths.
template <int TOK>
__device__ __forceinline__ int seq_tiles(const KvSeq& s) {
  return s.n == 0 ? 0 : (s.len > 0 ? (s.len + TOK - 1) / TOK : 1);       // (rows without tokens: one empty unit writes zeros)
}

struct UnitPlace {
  int b, h, tile, tiles;
};
template <int TOK>
__device__ __forceinline__ UnitPlace find_unit(const uint32_t* prefix, const KvSeq* seqs, int batch, uint32_t u) {
  int lo = 0, hi = batch;                                      // last b with prefix[b] <= u (its successor's is larger)
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (prefix[mid] <= u) lo = mid; else hi = mid;
  }
  UnitPlace p;
  p.b = lo;
  p.tiles = seq_tiles<TOK>(seqs[lo]);
  const uint32_t r = u - prefix[lo];
  p.h = (int)(r / p.tiles);
  p.tile = (int)(r % p.tiles);
  return p;
}

template <int D, int NT, int SUB>
struct AtSmem {
  static constexpr int ROWS = 8 * NT, TOK = 16 * AT_WARPS * SUB, SUBS = TOK / 16;
  static constexpr int TILE = TOK * D;                          // bytes of keys (or values) of a unit
  static constexpr int STAGES = NT == 1 ? 3 : 4;
  static constexpr int BLOCKS = NT == 1 ? 3 : 2;                // thread blocks per multiprocessor
  static constexpr int MERGE = AT_WARPS * ROWS * D * 4;
  static constexpr int OFF_MERGE = STAGES * 2 * TILE;
  static constexpr int OFF_SCALES = OFF_MERGE + MERGE;                        // [STAGES][3][SUBS]
  static constexpr int OFF_ML = OFF_SCALES + STAGES * 3 * SUBS * 4;           // [AT_WARPS][ROWS]
  static constexpr int OFF_BARS = OFF_ML + AT_WARPS * ROWS * 16;
  static constexpr int OFF_FLAG = OFF_BARS + STAGES * 2 * 8;
  static constexpr int OFF_SEQS = OFF_FLAG + 16;                              // [batch] KvSeq, then the plan
  static int total(int batch) { return OFF_SEQS + batch * (int)sizeof(KvSeq) + (batch + 2) * 4 + 1024; }   // (the window starts on a 1 KiB boundary)
};

// Partial result `slot` = 2 * block + (0: the rows' units began in an earlier block, 1: they began here):
// [ROWS] of {maximum, sum, maximum of weighted value scales relative to it, -}, then [ROWS][D] sums of weighted values relative to the latter.
template <int D, int ROWS>
__host__ __device__ constexpr long long part_floats() { return (long long)ROWS * (D + 4); }

// A value scale as v.x * 2^v.y, v.x in 1 .. 2.
__device__ __forceinline__ float2 split_scale(float s) {
  const bool tiny = s < 0x1p-126f;
  const uint32_t u = __float_as_uint(tiny ? s * 0x1p64f : s);
  if (!(s > 0.f && s < INFINITY)) return make_float2(s, s == 0.f ? kNoScale : 0.f);
  return make_float2(__uint_as_float((u & 0x007fffffu) | 0x3f800000u), (float)((int)(u >> 23) - (tiny ? 127 + 64 : 127)));
}

// x brought from weighted value scales relative to 2^v to values: times 2^v / l, the power in two halves, since with scales
// near either end of float32 it would leave the range of one.
struct RowScale {
  float by, again;
  __device__ __forceinline__ RowScale(float v, float l) {
    const float half = exp2f(0.5f * (v - kLift));
    by = l == 0.f ? 0.f : __fdiv_rn(half, l);
    again = l == 0.f ? 0.f : half;
  }
  __device__ __forceinline__ float4 operator()(float4 x) const {
    return make_float4(x.x * by * again, x.y * by * again, x.z * by * again, x.w * by * again);
  }
};

// D: head width; NT: tiles of 8 rows (new tokens x heads of a group); SUB: 16-token steps per warp and unit.
// Both products have the tokens or channels as the 16 rows of m16n8k16 and the few query rows as its 8 columns:
//   S^T = K Q^T   ldmatrix hands a lane four consecutive codes of one token, which are two A registers of a 16-channel
//                 step if the same permutation of the channels is applied to the query;
//   O^T = V^T P^T the transposing ldmatrix, whose 16-bit elements are pairs of channels, gives the even and the odd
//                 channels as rows 0-7 and 8-15 of A; P^T is S^T's result through movmatrix.
// (With the query rows as the 16 rows of the product, most of them padding, the same work took twice the products and
// 450 instead of 250 instructions per 16 tokens: 32 conversations of up to 4096 tokens 181 us, against 115 to 122 from GPU
// to GPU: 5.0 to 5.3 TB/s.)
// Codes turn into fp16 exactly (1024 + 128 + c by byte permutation, minus 1152), the query is fp16 after a
// power-of-two scaling per row (bf16 has fewer bits), so the scores are sums of exact products in float32.
// Every warp keeps maximum, sum and output of its own tokens; the warps meet only at the end of a row tile.
// Value scales go into the weights, as the channels' sums run over blocks of different scales, and the weights into fp16: a
// scale is split into 2^e and a factor of 1 .. 2, and the weights of the values are relative to the row's largest score + e
// (held as a difference from the largest score, which would swallow e where scores are large), those of the softmax's sum
// to its largest score.  So both keep their bits wherever the scales lie in float32, for
// a second exponential.  (Against weights relative to the score alone, times the scale relative to the largest one: 32
// conversations of up to 4096 tokens 121.9 us and 121.4, two documents of up to 100 003 tokens with eight heads to a key
// head and gathered weights 78.5 and 77.3, four new tokens of 16 sequences, 32 heads on 8: of up to 4000 tokens with
// heads of 128 43.8 and 45.3, of 6000 with heads of 64 33.0 and 31.8.)
template <int D, int NT, int SUB>
__global__ void __launch_bounds__(AT_THREADS, AtSmem<D, NT, SUB>::BLOCKS)
kv_attend_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ AttnArgs a, int* dbg) {
  using S = AtSmem<D, NT, SUB>;
  constexpr int ROWS = S::ROWS, TOK = S::TOK, SUBS = S::SUBS, STAGES = S::STAGES;
  constexpr int KSTEPS = D / 16;
  extern __shared__ uint8_t raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t sbase = ptx::smem_u32(smem);
  float* scale_ring = reinterpret_cast<float*>(smem + S::OFF_SCALES);
  float4* ml = reinterpret_cast<float4*>(smem + S::OFF_ML);
  float* merge = reinterpret_cast<float*>(smem + S::OFF_MERGE);
  volatile int* flag = reinterpret_cast<volatile int*>(smem + S::OFF_FLAG);
  KvSeq* seqs = reinterpret_cast<KvSeq*>(smem + S::OFF_SEQS);
  uint32_t* prefix = reinterpret_cast<uint32_t*>(seqs + a.kb.batch);
  const uint32_t bars = sbase + S::OFF_BARS;
  auto full = [&](int s) { return bars + s * 16; };
  auto empty = [&](int s) { return bars + s * 16 + 8; };
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const KvShape& sh = a.sh;

  if (tid == 0) {
    *flag = 0;
    for (int s = 0; s < STAGES; ++s) { ptx::mbar_init(full(s), 1); ptx::mbar_init(empty(s), AT_WARPS); }
    ptx::fence_mbar_init();
  }
  kv_begin();
  if (tid == 0 && blockIdx.x == 0 && a.batch0 == 0) *a.status = 0;
  // the plan: an exclusive sum over the sequences' units, by one warp
  if (warp == AT_WARPS) {
    ptx::prefetch_tensormap(&map);
    uint32_t run = 0;
    for (int b0 = 0; b0 < a.kb.batch; b0 += 32) {
      uint32_t n = 0;
      if (b0 + lane < a.kb.batch) {
        const KvSeq s = kv_seq(a.kb, b0 + lane);
        seqs[b0 + lane] = s;
        n = (uint32_t)sh.kv_heads * seq_tiles<TOK>(s);
      }
      uint32_t sum = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t up = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += up;
      }
      if (b0 + lane < a.kb.batch) prefix[b0 + lane] = run + sum - n;
      run += __shfl_sync(0xffffffffu, sum, 31);
    }
    const uint32_t per_block = a.whole ? (run > 0 ? run : 1u) : (run + gridDim.x - 1) / gridDim.x;
    if (lane == 0) { prefix[a.kb.batch] = run; prefix[a.kb.batch + 1] = per_block; }
    __syncwarp();
    if (blockIdx.x == 0)
      for (int i = lane; i < a.kb.batch + 2; i += 32) a.plan[i] = prefix[i];
  }
  __syncthreads();
  uint32_t u0, u1;
  if (a.whole) {
    const int b = blockIdx.x / sh.kv_heads, tiles = seq_tiles<TOK>(seqs[b]);
    u0 = prefix[b] + (uint32_t)(blockIdx.x % sh.kv_heads) * tiles;
    u1 = u0 + tiles;
  } else {
    const uint32_t total = prefix[a.kb.batch], per_block = prefix[a.kb.batch + 1];
    u0 = blockIdx.x * per_block;
    u1 = u0 + per_block < total ? u0 + per_block : total;
  }
  if (u0 >= u1) return;

  if (warp == AT_WARPS) {
    // ---- producer: the lanes look up the blocks and scales of 32 / SUBS units ahead, then issue their copies
    constexpr int AHEAD = 32 / SUBS;
    const int sub = lane % SUBS, box = sh.block < TOK ? sh.block : TOK;
    struct Look { int k_row, v_row; float ks, vs; };
    // (no branch hangs on what is loaded: nothing waits here)
    auto look = [&](uint32_t u) {
      const UnitPlace p = find_unit<TOK>(prefix, seqs, a.kb.batch, u < u1 ? u : u1 - 1);
      const int t = p.tile * TOK + sub * 16;
      const bool in = u < u1 && t < seqs[p.b].len;
      const int entry = in ? a.kb.table[(size_t)p.b * a.kb.max_blocks + (t >> sh.log_block)] : -1;
      const bool valid = entry >= 0 && entry < sh.num_blocks;
      const long long k_plane = ((long long)(valid ? entry : 0) * 2) * sh.kv_heads + p.h, v_plane = k_plane + sh.kv_heads;
      const float ks = a.at.scales[k_plane], vs = a.at.scales[v_plane];
      const int at = t & (sh.block - 1);
      return Look{valid ? (int)(k_plane * sh.block + at) : -1, (int)(v_plane * sh.block + at), valid ? ks : 0.f, valid ? vs : 0.f};
    };
    Look cur = look(u0 + lane / SUBS), next = cur;
    uint32_t it = 0;
    bool ok = true;
    for (uint32_t base = u0; base < u1 && ok; base += AHEAD) {
      for (int i = 0; i < AHEAD && base + i < u1; ++i, ++it) {
        const int st = it % STAGES;
        if (i == (STAGES < AHEAD ? STAGES : AHEAD) - 1) next = look(base + AHEAD + lane / SUBS);   // (not before the first copies are out)
        if (it >= STAGES) ok = __all_sync(0xffffffffu, ptx::mbar_wait(empty(st), ((it / STAGES) - 1) & 1, flag));
        if (!ok) break;
        // the copies first: they need only the block, the scales may still be on their way
        const bool mine = lane / SUBS == i, issues = mine && cur.k_row >= 0 && (sub * 16) % box == 0;
        const int boxes = __popc(__ballot_sync(0xffffffffu, issues));
        if (issues) {
          const uint32_t at = sbase + st * 2 * S::TILE + sub * 16 * D;
          ptx::tma_load_2d(at, &map, 0, cur.k_row, full(st));
          ptx::tma_load_2d(at + S::TILE, &map, 0, cur.v_row, full(st));
        }
        if (mine) {
          const float2 v = split_scale(cur.vs);
          float* ring = scale_ring + st * 3 * SUBS + sub;
          ring[0] = cur.ks;
          ring[SUBS] = v.x;
          ring[2 * SUBS] = v.y;
        }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive_expect_tx(full(st), (uint32_t)(boxes * 2 * box * D));
        __syncwarp();
      }
      cur = next;
    }
    // nothing is on its way to shared memory when the block ends, also where a wait ran out (the limit holds here too)
    for (uint32_t i = it < (uint32_t)STAGES ? 0 : it - STAGES; i < it; ++i) ptx::mbar_wait(full(i % STAGES), (i / STAGES) & 1, flag);
  } else {
    // ---- consumers
    const int g8 = lane >> 2, q4 = lane & 3;          // token (or channel pair) within 8, quad lane: rows 2 q4 and 2 q4 + 1
    uint32_t qf[NT][KSTEPS][2];
    float q_scale[NT][2];                              // softmax_scale * log2(e) / (the row's power of two)
    int limit[NT][2];                                  // last token the row sees, -1: none
    float mrow[NT][2], vrow[NT][2], lrow[NT][2], o[NT][KSTEPS][4];       // running maxima of score, and of score - that one + e; sum; output
    float* logit_row[NT][2];
    UnitPlace p{};
    KvSeq s{};
    bool fresh = true, ok = true;
    int rows = 0;
    for (uint32_t u = u0, it = 0; u < u1; ++u, ++it) {
      if (fresh) {
        p = find_unit<TOK>(prefix, seqs, a.kb.batch, u);
        s = seqs[p.b];
        rows = s.n * sh.group;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          // this lane's part of row g8 of the tile, as the B operand
          const int r = nt * 8 + g8, i = r / sh.group, g = r % sh.group;
          const bool load = r < rows && QALORA_CHECK(dbg, s.row0 + i, a.kb.m);
          const __nv_bfloat16* src = a.at.q + (long long)(s.row0 + i) * a.at.q_stride + (long long)(p.h * sh.group + g) * D;
          uint2 w[KSTEPS];
          uint32_t mx = 0;
#pragma unroll
          for (int k = 0; k < KSTEPS; ++k) w[k] = load ? *reinterpret_cast<const uint2*>(src + k * 16 + q4 * 4) : make_uint2(0, 0);
#pragma unroll
          for (int k = 0; k < KSTEPS; ++k) mx = __vmaxu2(__vmaxu2(mx, w[k].x & 0x7fff7fffu), w[k].y & 0x7fff7fffu);
          mx = max(mx & 0xffffu, mx >> 16);
          mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
          mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
          // times a power of two that brings the row's largest element to 2^14 .. 2^15: exact in fp16
          // down to 2^-28 of it
          int e = 268 - (int)(mx >> 7);
          e = e > 254 ? 254 : (e < 1 ? 1 : e);
          const float f = __uint_as_float((uint32_t)e << 23);
          const float back = a.at.softmax_scale * kLog2e * (e == 254 ? 0x1p-127f : __uint_as_float((uint32_t)(254 - e) << 23));
#pragma unroll
          for (int k = 0; k < KSTEPS; ++k) {
            qf[nt][k][0] = kvp::pack_half2(__uint_as_float(w[k].x << 16) * f, __uint_as_float(w[k].x & 0xffff0000u) * f);
            qf[nt][k][1] = kvp::pack_half2(__uint_as_float(w[k].y << 16) * f, __uint_as_float(w[k].y & 0xffff0000u) * f);
          }
          // and what belongs to the rows 2 q4, 2 q4 + 1 whose scores this lane holds
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const int own = nt * 8 + q4 * 2 + c, io = own / sh.group;
            q_scale[nt][c] = __shfl_sync(0xffffffffu, back, (q4 * 2 + c) * 4);
            limit[nt][c] = own < rows ? s.first + io : -1;
            mrow[nt][c] = vrow[nt][c] = kNoMax;
            lrow[nt][c] = 0.f;
            logit_row[nt][c] = a.logits != nullptr && own < rows
                                   ? a.logits + ((long long)((a.batch0 + p.b) * a.kb.n_hi + io) * sh.heads + p.h * sh.group + own % sh.group) *
                                                    a.logit_stride
                                   : nullptr;
          }
#pragma unroll
          for (int k = 0; k < KSTEPS; ++k)
#pragma unroll
            for (int c = 0; c < 4; ++c) o[nt][k][c] = 0.f;
        }
        fresh = false;
      }
      const int st = it % STAGES;
      ok = ok && ptx::mbar_wait(full(st), (it / STAGES) & 1, flag);
      ok = __all_sync(0xffffffffu, ok);
      const uint32_t k_base = sbase + st * 2 * S::TILE, v_base = k_base + S::TILE;
      const int sub0 = warp * SUB, t0 = p.tile * TOK + sub0 * 16;        // this warp's SUB * 16 tokens of the unit
      if (t0 < s.len && ok) {
        float ks[SUB], vs[SUB], ve[SUB], sc[SUB][NT][4];
#pragma unroll
        for (int g = 0; g < SUB; ++g) {                // (a group behind the sequence's end has scales of 0 and is masked)
          const float* ring = scale_ring + st * 3 * SUBS + sub0 + g;
          ks[g] = ring[0];
          vs[g] = ring[SUBS];
          ve[g] = ring[2 * SUBS];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 4; ++c) sc[g][nt][c] = 0.f;
        }
        // scores: rows of the product are tokens g8 and g8 + 8 of a group
        const int tok = sub0 * 16 + (lane & 15);       // ldmatrix: lanes 0-15 the tokens of one chunk, 16-31 of the next
#pragma unroll
        for (int c2 = 0; c2 < D / 32; ++c2)
#pragma unroll
          for (int g = 0; g < SUB; ++g) {
            uint32_t r[4];
            kvp::ldmatrix_x4(r, k_base + kvp::swizzled<D>(tok + g * 16, c2 * 2 + (lane >> 4)));
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              uint32_t f[4];                           // {token g8, +8} x {channels 0-1, 2-3 of the lane's four}
              kvp::codes_to_half(r[2 * x], f[0], f[2]);
              kvp::codes_to_half(r[2 * x + 1], f[1], f[3]);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) kvp::mma16816(sc[g][nt], f, qf[nt][c2 * 2 + x][0], qf[nt][c2 * 2 + x][1]);
            }
          }
        // scaled scores in powers of two, masked
        const bool edge = t0 + SUB * 16 - 1 > s.first || rows < ROWS;    // (the first row sees the least)
        bool grow = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int g = 0; g < SUB; ++g) {
              const float f = q_scale[nt][c] * ks[g];
              const int t = t0 + g * 16 + g8;
              float &x0 = sc[g][nt][c], &x1 = sc[g][nt][2 + c];
              x0 *= f;
              x1 *= f;
              if (edge) {
                if (t > limit[nt][c]) x0 = -INFINITY;
                if (t + 8 > limit[nt][c]) x1 = -INFINITY;
              }
              const float over = fmaxf(x0, x1) - mrow[nt][c];
              grow |= over > kGrow || over + ve[g] > vrow[nt][c] + kGrow;
              if (logit_row[nt][c] != nullptr && QALORA_CHECK(dbg, t + 8, a.logit_stride)) {
                logit_row[nt][c][t] = x0;
                logit_row[nt][c][t + 8] = x1;
              }
            }
        if (__any_sync(0xffffffffu, grow)) {
          // rare: bring the rows to their new maxima
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float by[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              float mx = mrow[nt][c];
#pragma unroll
              for (int g = 0; g < SUB; ++g) mx = fmaxf(mx, fmaxf(sc[g][nt][c], sc[g][nt][2 + c]));
#pragma unroll
              for (int w = 4; w < 32; w <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
              const float before = vrow[nt][c] + (mrow[nt][c] - mx);        // in terms of the new maximum
              float vx = before;
#pragma unroll
              for (int g = 0; g < SUB; ++g) vx = fmaxf(vx, fmaxf(sc[g][nt][c], sc[g][nt][2 + c]) - mx + ve[g]);
#pragma unroll
              for (int w = 4; w < 32; w <<= 1) vx = fmaxf(vx, __shfl_xor_sync(0xffffffffu, vx, w));
              lrow[nt][c] *= exp2f(mrow[nt][c] - mx);
              by[c] = exp2f(before - vx);
              mrow[nt][c] = mx;
              vrow[nt][c] = vx;
            }
#pragma unroll
            for (int k = 0; k < KSTEPS; ++k) {
              o[nt][k][0] *= by[0]; o[nt][k][1] *= by[1];
              o[nt][k][2] *= by[0]; o[nt][k][3] *= by[1];
            }
          }
        }
        uint32_t pf[SUB][NT][2];                       // P^T as the B operand: tokens 0-7 and 8-15 of a group
#pragma unroll
        for (int g = 0; g < SUB; ++g)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float x[4], e[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) x[c] = sc[g][nt][c] - mrow[nt][c & 1];
            lrow[nt][0] += kvp::exp2_fast(x[0]) + kvp::exp2_fast(x[2]);
            lrow[nt][1] += kvp::exp2_fast(x[1]) + kvp::exp2_fast(x[3]);
#pragma unroll
            for (int c = 0; c < 4; ++c) e[c] = kvp::exp2_fast(x[c] + (ve[g] + (kLift - vrow[nt][c & 1]))) * vs[g];
            pf[g][nt][0] = kvp::movmatrix(kvp::pack_half2(e[0], e[1]));
            pf[g][nt][1] = kvp::movmatrix(kvp::pack_half2(e[2], e[3]));
          }
#pragma unroll
        for (int g = 0; g < SUB; ++g)
#pragma unroll
          for (int c2 = 0; c2 < D / 32; ++c2) {
            uint32_t r[4];
            kvp::ldmatrix_x4_trans(r, v_base + kvp::swizzled<D>(tok + g * 16, c2 * 2 + (lane >> 4)));
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              uint32_t f[4];                           // {even, odd channels} x {tokens 0-7, 8-15}
              kvp::pairs_to_half(r[2 * x], f[0], f[1]);
              kvp::pairs_to_half(r[2 * x + 1], f[2], f[3]);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) kvp::mma16816(o[nt][c2 * 2 + x], f, pf[g][nt][0], pf[g][nt][1]);
            }
          }
      }
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(empty(st));

      if (++p.tile == p.tiles || u + 1 == u1) {
        // ---- the rows' tokens end here, or go on in the next block: the warps' shares are added up
        const uint32_t first_unit = u + 1 - p.tile;          // their unit of tile 0
        const bool whole = first_unit >= u0 && p.tile == p.tiles;
        const int slot = 2 * (int)blockIdx.x + (first_unit < u0 ? 0 : 1);
        float* part = a.parts + slot * part_floats<D, ROWS>();
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float l = lrow[nt][c];
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) l += __shfl_xor_sync(0xffffffffu, l, w);
            const int r = nt * 8 + q4 * 2 + c;
            if (g8 == 0) ml[warp * ROWS + r] = make_float4(mrow[nt][c], l, vrow[nt][c], 0.f);
            if (r < rows) {
#pragma unroll
              for (int k = 0; k < KSTEPS; ++k)
                *reinterpret_cast<float2*>(merge + (warp * ROWS + r) * D + k * 16 + g8 * 2) = make_float2(o[nt][k][c], o[nt][k][2 + c]);
            }
          }
        ptx::named_barrier(1, AT_WARPS * 32);
        for (int i = tid; i < rows * (D / 4); i += AT_WARPS * 32) {
          const int r = i / (D / 4), d = (i % (D / 4)) * 4;
          float mx = kNoMax, vx = kNoMax, l = 0.f;
#pragma unroll
          for (int w = 0; w < AT_WARPS; ++w) mx = fmaxf(mx, ml[w * ROWS + r].x);
#pragma unroll
          for (int w = 0; w < AT_WARPS; ++w) vx = fmaxf(vx, ml[w * ROWS + r].z + (ml[w * ROWS + r].x - mx));
          float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int w = 0; w < AT_WARPS; ++w) {
            const float4 of = ml[w * ROWS + r];
            const float by = exp2f(of.z + (of.x - mx) - vx);
            const float4 y = *reinterpret_cast<const float4*>(merge + (w * ROWS + r) * D + d);
            l = fmaf(exp2f(of.x - mx), of.y, l);
            x.x = fmaf(by, y.x, x.x); x.y = fmaf(by, y.y, x.y); x.z = fmaf(by, y.z, x.z); x.w = fmaf(by, y.w, x.w);
          }
          if (whole) {
            const int i_new = r / sh.group, head = p.h * sh.group + r % sh.group;
            const long long at = (long long)(s.row0 + i_new) * sh.heads + head;
            if (!QALORA_CHECK(dbg, at, (long long)a.kb.m * sh.heads)) continue;
            kvp::store_row4(a.at.out + at * D + d, RowScale(vx, l)(x));
            if (d == 0) {
              const long long own = (long long)((a.batch0 + p.b) * a.kb.n_hi + i_new) * sh.heads + head;
              kvp::store_lse(a.at.lse, at, a.lse2, own, mx, l, 0.f);
            }
          } else if (QALORA_CHECK(dbg, slot, 2 * a.units_grid)) {
            *reinterpret_cast<float4*>(part + 4 * ROWS + r * D + d) = x;
            if (d == 0) *reinterpret_cast<float4*>(part + 4 * r) = make_float4(mx, l, vx, 0.f);
          }
        }
        ptx::named_barrier(1, AT_WARPS * 32);
        fresh = true;
      }
    }
  }
  if (*flag != 0 && lane == 0) *a.status = 1;
}

// Joins the partial results of rows that several blocks shared (first blocks of the grid, one per row: the tokens of a
// long sequence lie in up to some hundred parts), and adds up the gathered weights from the stored scores (the
// other blocks, JOIN_TOKENS tokens of one kv head each).
template <int D, int ROWS, int TOK>
__global__ void __launch_bounds__(128, 12)
kv_join_kernel(const __grid_constant__ AttnArgs a, int row_blocks, int* dbg) {
  __shared__ float row_lse[ROWS];
  __shared__ float4 share[4][32];
  kv_begin();
  const KvShape& sh = a.sh;
  const int b = blockIdx.y, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const bool scores = (int)blockIdx.x >= row_blocks;
  const int x = scores ? (int)blockIdx.x - row_blocks : (int)blockIdx.x, h = x % sh.kv_heads;
  const int t0 = scores ? x / sh.kv_heads * JOIN_TOKENS : 0, row = scores ? 0 : x / sh.kv_heads;
  const KvSeq s = kv_seq(a.kb, b);
  const int rows = s.n * sh.group;
  if (row >= rows) return;                                      // (also: no rows)
  const uint32_t per_block = a.plan[a.kb.batch + 1];
  const int tiles = seq_tiles<TOK>(s);
  const uint32_t f = a.plan[b] + (uint32_t)h * tiles, c0 = f / per_block, c1 = (f + tiles - 1) / per_block;
  if (scores ? t0 >= s.len : c0 == c1) return;                  // (c0 == c1: one block had all of it)
  auto part_of = [&](uint32_t c) { return a.parts + (2ll * c + (f < c * per_block ? 0 : 1)) * part_floats<D, ROWS>(); };
  // maxima and sum of row r over the parts, by one warp
  auto stats = [&](int r, float& mx, float& l, float& vx) {
    mx = vx = kNoMax;
    l = 0.f;
    for (uint32_t c = c0 + lane; c <= c1; c += 32) {
      const float4 v = *reinterpret_cast<const float4*>(part_of(c) + 4 * r);
      const float top = fmaxf(mx, v.x);
      l = l * exp2f(mx - top) + v.y * exp2f(v.x - top);
      vx = fmaxf(vx + (mx - top), v.z + (v.x - top));
      mx = top;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const float m2 = __shfl_xor_sync(0xffffffffu, mx, o), l2 = __shfl_xor_sync(0xffffffffu, l, o), top = fmaxf(mx, m2);
      l = l * exp2f(mx - top) + l2 * exp2f(m2 - top);
      vx = fmaxf(vx + (mx - top), __shfl_xor_sync(0xffffffffu, vx, o) + (m2 - top));
      mx = top;
    }
  };
  if (!scores) {
    constexpr int LANES = D / 4, SHARES = 128 / LANES;          // lanes of a row's output; shares of its parts
    float mx, l, vx;
    stats(row, mx, l, vx);
    const int who = tid / LANES, d = (tid % LANES) * 4;
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (uint32_t c = c0 + who; c <= c1; c += SHARES) {
      const float* part = part_of(c);
      const float by = exp2f(part[4 * row + 2] + (part[4 * row] - mx) - vx);
      const float4 v = *reinterpret_cast<const float4*>(part + 4 * ROWS + row * D + d);
      y.x = fmaf(v.x, by, y.x); y.y = fmaf(v.y, by, y.y); y.z = fmaf(v.z, by, y.z); y.w = fmaf(v.w, by, y.w);
    }
    share[warp][lane] = y;
    __syncthreads();
    if (tid >= LANES) return;
    y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < SHARES; ++i) {
      const float4 v = (&share[0][0])[i * LANES + tid];
      y.x += v.x; y.y += v.y; y.z += v.z; y.w += v.w;
    }
    const long long at = (long long)(s.row0 + row / sh.group) * sh.heads + h * sh.group + row % sh.group;
    if (!QALORA_CHECK(dbg, at, (long long)a.kb.m * sh.heads)) return;
    kvp::store_row4(a.at.out + at * D + d, RowScale(vx, l)(y));
    if (d == 0) kvp::store_lse(a.at.lse, at, nullptr, 0, mx, l, 0.f);
    return;
  }
  // Four tokens per thread; the scores of the first four rows are asked for before the rows' sums, whose parts take two
  // trips to memory.  Both kernels, 48 conversations of up to 3001 tokens, four heads to a key head: 37.2 us -> 35.2; two
  // documents of up to 100 003 tokens, eight heads to a key head: 74.4 -> 75.5, as 40 registers leave room for twelve
  // blocks.  (Eight rows early 81 there; two rows 73.8 and 36.9.)
  const float* logits = a.logits + ((long long)(a.batch0 + b) * a.kb.n_hi * sh.heads + h * sh.group) * a.logit_stride;
  const int t = t0 + tid * 4;
  constexpr int EARLY = 4;
  const long long skip = (long long)(sh.heads - sh.group) * a.logit_stride;      // from one new token's last head to the next one's first
  const float* at_row = logits + t;
  int g = 0;
  auto next_row = [&] {
    const float4 v = __ldcs(reinterpret_cast<const float4*>(at_row));
    at_row += a.logit_stride;
    if (++g == sh.group) { g = 0; at_row += skip; }
    return v;
  };
  float4 early[EARLY];
  int id = -1;
  if (t < s.len) {
    id = kv_block(a.kb.table, a.kb.max_blocks, sh.num_blocks, b, t >> sh.log_block);
#pragma unroll
    for (int r = 0; r < EARLY; ++r) if (r < rows) early[r] = next_row();
  }
  if (c0 != c1) {
    for (int r = warp; r < rows; r += 4) {
      float mx, l, vx;
      stats(r, mx, l, vx);
      if (lane == 0) row_lse[r] = l == 0.f ? INFINITY : mx + log2f(l);
    }
  } else if (tid < rows) {
    row_lse[tid] = a.lse2[(long long)((a.batch0 + b) * a.kb.n_hi + tid / sh.group) * sh.heads + h * sh.group + tid % sh.group];
  }
  __syncthreads();
  if (id < 0) return;
  float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](const float4 v, float n) {
    if (n != n) {                                               // a row of NaN spoils the tokens it sees (the others' scores are -infinity)
      w.x += v.x == -INFINITY ? 0.f : n; w.y += v.y == -INFINITY ? 0.f : n;
      w.z += v.z == -INFINITY ? 0.f : n; w.w += v.w == -INFINITY ? 0.f : n;
      return;
    }
    w.x += kvp::exp2_fast(v.x - n); w.y += kvp::exp2_fast(v.y - n);
    w.z += kvp::exp2_fast(v.z - n); w.w += kvp::exp2_fast(v.w - n);
  };
#pragma unroll
  for (int r = 0; r < EARLY; ++r)
    if (r < rows) add(early[r], row_lse[r]);
#pragma unroll 4
  for (int r = EARLY; r < rows; ++r) add(next_row(), row_lse[r]);
  const long long at = ((long long)id * sh.kv_heads + h) * sh.block + (t & (sh.block - 1));
  if (t + 4 <= s.len) {
    if (a.at.score_in != nullptr) {
      const float4 v = *reinterpret_cast<const float4*>(a.at.score_in + at);
      w.x += v.x; w.y += v.y; w.z += v.z; w.w += v.w;
    }
    *reinterpret_cast<float4*>(a.at.score_out + at) = w;
  } else {                                                      // the sequence ends inside
    const float got[4] = {w.x, w.y, w.z, w.w};
    for (int c = 0; t + c < s.len; ++c) a.at.score_out[at + c] = (a.at.score_in != nullptr ? a.at.score_in[at + c] : 0.f) + got[c];
  }
}

// keys and values as one matrix of rows of `dim` bytes; a box is the part of a block that a unit takes
bool make_cache_map(CUtensorMap* map, const int8_t* codes, const KvShape& sh, int box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (fn == nullptr) return false;
  cuuint64_t dims[2] = {(cuuint64_t)sh.dim, (cuuint64_t)sh.num_blocks * 2 * sh.kv_heads * sh.block};
  cuuint64_t strides[1] = {(cuuint64_t)sh.dim};
  cuuint32_t box[2] = {(cuuint32_t)sh.dim, (cuuint32_t)box_rows};
  cuuint32_t estr[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t*>(codes), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, sh.dim == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int NT, int SUB>
int attend(const AttnArgs& a, cudaStream_t st) {
  using S = AtSmem<D, NT, SUB>;
  CUtensorMap map;
  if (!make_cache_map(&map, a.at.codes, a.sh, a.sh.block < S::TOK ? a.sh.block : S::TOK)) return QALORA_ERR_CUDA;
  static PerDeviceOnce once;
  const int ok = once.run([] {
    return cudaFuncSetAttribute(kv_attend_kernel<D, NT, SUB>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::total(AT_MAX_BATCH));
  });
  if (ok != QALORA_OK) return ok;
  int r;
  {
    MainKernelProbe probe("kv_attend_kernel", st);
    r = kv_launch(kv_attend_kernel<D, NT, SUB>, dim3((unsigned)a.units_grid), AT_THREADS, (size_t)S::total(a.kb.batch), st, map, a, debug_words());
  }
  if (r != QALORA_OK) return r;
  const int row_blocks = a.whole ? 0 : a.sh.kv_heads * a.kb.max_new * a.sh.group;
  const int score_blocks = a.logits != nullptr ? a.sh.kv_heads * ((a.kb.max_len + JOIN_TOKENS - 1) / JOIN_TOKENS) : 0;
  if (row_blocks + score_blocks == 0) return QALORA_OK;
  return kv_launch(kv_join_kernel<D, S::ROWS, S::TOK>, dim3((unsigned)(row_blocks + score_blocks), (unsigned)a.kb.batch), 128, 0, st, a,
                   row_blocks, debug_words());
}

struct AttnLayout {
  size_t status, plan, parts, lse2, logits, pr_ml, pr_o, pr_q, pr_rows, total;
  int few, many_lo;      // new rows per sequence up to which the kernels of this file take it, from which the prompt kernel does
  bool any_few, any_many;
  KvPromptScratch prompt;
};

// Rows (new tokens x heads of a group) of one kv head up to which a sequence is taken here; with more, its
// products fill the tensor core's tiles of 128 rows.
constexpr int kFewRows = 16;

// Whether every thread block takes one whole (sequence, kv head): nothing is left to join, but the blocks are as uneven as
// the sequences, and fewer than could run.  Even shares need the second kernel, about 3 us, and pairs / most of them
// less units each; a unit takes about 0.6 us with one tile of rows, 1 us with two.  So `allowed` units are given up for the
// second kernel, half of them where it runs anyway for the gathered weights.  Measured, 32 heads of 128, microseconds whole
// / even shares: one conversation of 333 tokens 7.6 / 8.4, of 700 10.9 / 9.0; 12 of up to 1000 20.3 / 25.8; 32 of 1000
// tokens with four new ones and 8 kv heads 28.8 / 40.0.  kWholeUnits bounds what uneven sequences cost: 12 of up to 2000
// tokens 33.1 / 33.0, of 2000 each 36.9 / 42.7, 13 of up to 4000 62.9 / 52.1.
constexpr int kWholeUnits = 16;
bool whole_sequences(long long units, long long pairs, long long most, int nt, bool scores) {
  const long long allowed = (nt == 1 ? 8 : 5) >> (scores ? 1 : 0);
  return units <= kWholeUnits && pairs <= most && units * (most - pairs) <= allowed * most;
}

int column_tiles(const KvShape& sh, int max_new) { return max_new * sh.group <= 8 ? 1 : 2; }     // NT

AttnLayout attention_layout(const KvShape& sh, int batch, int64_t m, int max_new, int max_len, bool with_score, Workspace* guards) {
  AttnLayout w{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += round_up(bytes, 256);
    if (kDebugBuild) { if (guards != nullptr) guards->guard[guards->n_guard++] = off; off += kGuardBytes; }
    return at;
  };
  const int most_few = kFewRows / sh.group;
  w.few = max_new < most_few ? max_new : most_few;
  w.any_many = max_new > w.few;
  // Which kernels run.  m bounds the rows, so nothing follows from it about a sequence's own; the rule only guesses.  If
  // the rows were exactly m, a sequence with few of them would need the others to be near their bound: where even
  // that leaves many, this looks like prompts alone, and the prompt kernel takes every sequence (many_lo), a short one
  // in a tile of 128 rows.
  w.any_few = w.few > 0 && (!w.any_many || m - (int64_t)(batch - 1) * max_new <= w.few);
  w.many_lo = w.any_few ? w.few + 1 : 1;
  const int rows = 8 * column_tiles(sh, w.few);
  const size_t few_rows = w.any_few ? (size_t)batch * w.few * sh.heads : 0;
  w.status = take(256);
  w.plan = take((size_t)((batch < AT_MAX_BATCH ? batch : AT_MAX_BATCH) + 2) * 4);
  w.parts = take(w.any_few ? (size_t)device_sm_count() * 3 * 2 * rows * (sh.dim + 4) * 4 : 0);   // (two for each of up to three blocks)
  w.lse2 = take(with_score ? few_rows * 4 : 0);
  w.logits = take(with_score ? few_rows * round_up((size_t)max_len, 128) * 4 : 0);
  if (w.any_many) w.prompt = kv_prompt_scratch(sh, batch, m, max_len, with_score);
  w.pr_ml = take(w.prompt.part_ml);
  w.pr_o = take(w.prompt.part_o);
  w.pr_q = take(w.prompt.q_image);
  w.pr_rows = take(w.prompt.rows);
  w.total = off;
  return w;
}

int launch_few(const KvShape& sh, const KvBatch& b, const KvAttention& at, const AttnLayout& L, char* base, int max_len, cudaStream_t st) {
  AttnArgs a{};
  a.sh = sh;
  a.kb = b;
  a.kb.max_new = a.kb.n_hi = L.few;
  a.at = at;
  a.status = reinterpret_cast<int*>(base + L.status);
  a.plan = reinterpret_cast<uint32_t*>(base + L.plan);
  a.parts = reinterpret_cast<float*>(base + L.parts);
  a.lse2 = at.score_out != nullptr ? reinterpret_cast<float*>(base + L.lse2) : nullptr;
  a.logits = at.score_out != nullptr ? reinterpret_cast<float*>(base + L.logits) : nullptr;
  a.logit_stride = (long long)round_up((size_t)max_len, 128);
  const int nt = column_tiles(sh, L.few), tok = sh.dim == 128 ? 64 : 128;
  const long long tiles = b.max_len > 0 ? (b.max_len + tok - 1) / tok : 1;
  const long long per_seq = tiles * sh.kv_heads;
  if (per_seq > 0x7fffffffll) return QALORA_ERR_UNSUPPORTED_SHAPE;
  // sequences of one launch: their plan fits shared memory and their units 31 bits
  const long long fit = 0x7fffffffll / per_seq;
  const int chunk = (int)(fit < AT_MAX_BATCH ? fit : AT_MAX_BATCH);
  for (int b0 = 0; b0 < b.batch; b0 += chunk) {
    a.batch0 = b0;
    a.kb.batch = b.batch - b0 < chunk ? b.batch - b0 : chunk;
    a.kb.starts = b.starts + b0;
    a.kb.lens = b.lens + b0;
    a.kb.table = b.table + (size_t)b0 * b.max_blocks;
    const long long units = per_seq * a.kb.batch, most = (nt == 1 ? 3ll : 2ll) * device_sm_count();
    a.units_grid = (int)(units < most ? units : most);
    const long long pairs = (long long)a.kb.batch * sh.kv_heads;
    a.whole = whole_sequences(tiles, pairs, most, nt, at.score_out != nullptr);
    if (a.whole) a.units_grid = (int)pairs;
    int r;
    if (sh.dim == 128) r = nt == 1 ? attend<128, 1, 1>(a, st) : attend<128, 2, 1>(a, st);
    else r = nt == 1 ? attend<64, 1, 2>(a, st) : attend<64, 2, 2>(a, st);
    if (r != QALORA_OK) return r;
  }
  return QALORA_OK;
}

}  // namespace

size_t kv_attention_workspace(const KvShape& sh, int batch, int64_t m, int max_new, int max_len, bool with_score, Workspace* guards) {
  return attention_layout(sh, batch, m, max_new, max_len, with_score, guards).total;
}

int launch_kv_attention(const KvShape& sh, const KvBatch& b, const KvAttention& at, void* workspace, int max_len, cudaStream_t st) {
  const AttnLayout L = attention_layout(sh, b.batch, b.m, b.max_new, max_len, at.score_out != nullptr, nullptr);
  char* base = static_cast<char*>(workspace);
  if (!L.any_few && cudaMemsetAsync(base + L.status, 0, sizeof(int), st) != cudaSuccess) return QALORA_ERR_CUDA;
  int r = L.any_few ? launch_few(sh, b, at, L, base, max_len, st) : QALORA_OK;
  if (r != QALORA_OK || !L.any_many) return r;
  KvBatch many = b;
  many.n_lo = L.many_lo;
  return launch_kv_prompt(sh, many, at, L.prompt, reinterpret_cast<float2*>(base + L.pr_ml), reinterpret_cast<float*>(base + L.pr_o),
                          reinterpret_cast<uint8_t*>(base + L.pr_q), reinterpret_cast<float*>(base + L.pr_rows),
                          reinterpret_cast<int*>(base + L.status), st);
}

}  // namespace qalora
