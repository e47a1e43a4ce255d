// Eviction from the key/value cache by accumulated attention weight: for every sequence and kv
// head the places of the tokens to keep (select), then their move to new blocks (gather).
#define QALORA_TU 11
#include <cooperative_groups.h>

#include "kv.cuh"

namespace cg = cooperative_groups;

namespace qalora {

namespace {

constexpr int SEL_BINS = 2048;                  // 11 bits of the key per pass: 11 + 11 + 10
constexpr int SEL_COARSE = SEL_BINS / 32;
constexpr int SEL_MAX_CLUSTER = 8;
constexpr int SEL_CACHED_KEYS = 49152;          // keys of one thread block that fit its shared memory (192 KiB)

// Order-preserving key of a score: larger score, larger key; -0 equals +0; NaN is the largest.
__device__ __forceinline__ uint32_t score_key(float x) {
  if (x != x) return 0xffffffffu;
  const uint32_t u = __float_as_uint(x + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

struct SelectArgs {
  const float* score;
  int32_t* dst_lens;
  int32_t* kept;
  int budget, recent;
  int cached;                                   // keys of a thread block that its shared memory holds, 0: they are read again
};

// One cluster per (sequence, kv head); its thread blocks share the candidates (all tokens but the
// last `recent`) as consecutive ranges.  A radix select of the (budget - recent)-th largest key:
// three passes of 11, 11 and 10 bits, each a histogram per thread block that the cluster adds up
// through distributed shared memory.  The keys stay in shared memory between the passes, so
// the scores are read once.  Then every warp counts its range, one scan turns the counts into
// offsets, and the places come out in order.
template <int SEL_THREADS>
__global__ void __launch_bounds__(SEL_THREADS)
kv_select_kernel(KvShape sh, KvBatch kb, SelectArgs a, int* dbg) {
  constexpr int SEL_WARPS = SEL_THREADS / 32;
  extern __shared__ __align__(16) uint32_t keys[];   // [cached] when the keys fit
  __shared__ uint32_t hist[SEL_BINS];
  __shared__ uint32_t coarse[SEL_COARSE], warp_gt[SEL_WARPS], warp_eq[SEL_WARPS];
  __shared__ uint32_t found[2];                 // bin, keys above it
  __shared__ uint32_t share[2];                 // this block's keys above / at the threshold, read by its cluster
  kv_begin();
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int pair = blockIdx.x / C, b = pair / sh.kv_heads, h = pair % sh.kv_heads;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  int len = kb.lens[b];
  len = len < 0 ? 0 : (len > kb.max_len ? kb.max_len : len);
  const int count = len < a.budget ? len : a.budget;
  int32_t* kept = a.kept + ((long long)b * sh.kv_heads + h) * a.budget;
  if (h == 0 && rank == 0 && tid == 0) a.dst_lens[b] = count;
  for (int i = count + rank * SEL_THREADS + tid; i < a.budget; i += C * SEL_THREADS) kept[i] = -1;
  if (len <= a.budget) {                        // (the same for the whole cluster)
    for (int i = rank * SEL_THREADS + tid; i < len; i += C * SEL_THREADS) kept[i] = i;
    return;
  }
  const int cand = len - a.recent, want = a.budget - a.recent;          // cand > want >= 0
  for (int i = rank * SEL_THREADS + tid; i < a.recent; i += C * SEL_THREADS)
    if (QALORA_CHECK(dbg, want + i, a.budget)) kept[want + i] = cand + i;
  if (want == 0) return;
  const int per = ((cand + C - 1) / C + 3) & ~3, begin = rank * per, end = begin + per < cand ? begin + per : cand;
  auto meet = [&] { if (C == 1) __syncthreads(); else cluster.sync(); };
  auto fetch = [&](int t) -> uint32_t {
    const int id = kv_block(kb.table, kb.max_blocks, sh.num_blocks, b, t >> sh.log_block);
    return id < 0 ? 0u : score_key(a.score[((long long)id * sh.kv_heads + h) * sh.block + (t & (sh.block - 1))]);
  };
  if (a.cached) {                               // four neighbouring tokens, which lie in one block, at a time
#pragma unroll 4
    for (int t = begin + tid * 4; t < end; t += SEL_THREADS * 4) {
      const int id = kv_block(kb.table, kb.max_blocks, sh.num_blocks, b, t >> sh.log_block);
      const float4 x = *reinterpret_cast<const float4*>(a.score + ((long long)(id < 0 ? 0 : id) * sh.kv_heads + h) * sh.block + (t & (sh.block - 1)));
      const uint4 k = make_uint4(score_key(x.x), score_key(x.y), score_key(x.z), score_key(x.w));
      if (QALORA_CHECK(dbg, t - begin + 3, a.cached)) *reinterpret_cast<uint4*>(keys + (t - begin)) = id < 0 ? make_uint4(0, 0, 0, 0) : k;
    }
    __syncthreads();
  }
  auto key_at = [&](int t) -> uint32_t { return a.cached ? keys[t - begin] : fetch(t); };

  uint32_t prefix = 0, mask = 0, left = (uint32_t)want;                 // keys still wanted among those that match prefix
  constexpr int SHIFT[3] = {21, 10, 0}, BITS[3] = {11, 11, 10};
#pragma unroll 1
  for (int p = 0; p < 3; ++p) {
    for (int i = tid; i < SEL_BINS; i += SEL_THREADS) hist[i] = 0;
    __syncthreads();
    const uint32_t digit_mask = (1u << BITS[p]) - 1;
    for (int t = begin + tid; t < end; t += SEL_THREADS) {
      const uint32_t key = key_at(t);
      if ((key & mask) == prefix) atomicAdd(&hist[(key >> SHIFT[p]) & digit_mask], 1u);
    }
    __syncthreads();
    // sums of 32 neighbouring bins, so that the cluster reads few words of each other's: 64 sums, then the 32 bins of one
    for (int i = warp; i < SEL_COARSE; i += SEL_WARPS) {
      const uint32_t n = __reduce_add_sync(0xffffffffu, hist[i * 32 + lane]);
      if (lane == 0) coarse[i] = n;
    }
    meet();
    if (warp == 0) {
      // from the largest key down: the lane's bins are hi and hi - 1 of the sums, then one of the 32
      auto total = [&](uint32_t* mine, int at) {
        uint32_t part[SEL_MAX_CLUSTER], n = 0;                          // (all loads first: each takes some hundred cycles)
#pragma unroll
        for (int r = 0; r < SEL_MAX_CLUSTER; ++r) part[r] = r < C ? cluster.map_shared_rank(mine, r)[at] : 0u;
#pragma unroll
        for (int r = 0; r < SEL_MAX_CLUSTER; ++r) n += part[r];
        return n;
      };
      auto inclusive = [&](uint32_t n) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t up = __shfl_up_sync(0xffffffffu, n, o);
          if (lane >= o) n += up;
        }
        return n;
      };
      const int hi = SEL_COARSE - 1 - 2 * lane;
      const uint32_t n0 = total(coarse, hi), n1 = total(coarse, hi - 1), above = inclusive(n0 + n1) - n0 - n1;
      const bool first = above < left && left <= above + n0, second = above + n0 < left && left <= above + n0 + n1;
      const uint32_t who = __ballot_sync(0xffffffffu, first || second);       // one lane: `left` keys at least match the prefix
      const int from = __ffs(who) - 1;
      const int group = __shfl_sync(0xffffffffu, first ? hi : hi - 1, from);
      const uint32_t before = __shfl_sync(0xffffffffu, first ? above : above + n0, from);
      const int bin = group * 32 + 31 - lane;
      const uint32_t n = total(hist, bin), over = before + inclusive(n) - n;
      if (over < left && left <= over + n) { found[0] = bin; found[1] = over; }
    }
    meet();                                                             // (also: nobody reads this histogram any more)
    prefix |= found[0] << SHIFT[p];
    mask |= digit_mask << SHIFT[p];
    left -= found[1];
  }
  // prefix is the want-th largest key; `left` of the keys equal to it are taken, the earliest ones
  const int span = ((per + SEL_WARPS - 1) / SEL_WARPS + 31) & ~31;
  const int w0 = begin + warp * span, w1 = w0 + span < end ? w0 + span : end;
  uint32_t gt = 0, eq = 0;
  for (int t = w0 + lane; t < w1; t += 32) {
    const uint32_t key = key_at(t);
    gt += key > prefix;
    eq += key == prefix;
  }
  gt = __reduce_add_sync(0xffffffffu, gt);
  eq = __reduce_add_sync(0xffffffffu, eq);
  if (lane == 0) { warp_gt[warp] = gt; warp_eq[warp] = eq; }
  __syncthreads();
  uint32_t gt0 = __reduce_add_sync(0xffffffffu, lane < warp ? warp_gt[lane] : 0u);
  uint32_t eq0 = __reduce_add_sync(0xffffffffu, lane < warp ? warp_eq[lane] : 0u);
  if (warp == SEL_WARPS - 1 && lane == 0) { share[0] = gt0 + gt; share[1] = eq0 + eq; }
  meet();
  for (int r = 0; r < rank; ++r) {
    const uint32_t* other = cluster.map_shared_rank(share, r);
    gt0 += other[0];
    eq0 += other[1];
  }
  for (int t0 = w0; t0 < w1; t0 += 32) {
    const int t = t0 + lane;
    const uint32_t key = t < w1 ? key_at(t) : 0u;
    const bool is_gt = t < w1 && key > prefix, is_eq = t < w1 && key == prefix;
    const uint32_t below = (1u << lane) - 1, bg = __ballot_sync(0xffffffffu, is_gt), be = __ballot_sync(0xffffffffu, is_eq);
    const uint32_t my_eq = eq0 + __popc(be & below);
    if (is_gt || (is_eq && my_eq < left)) {
      const uint32_t at = gt0 + __popc(bg & below) + (my_eq < left ? my_eq : left);
      if (QALORA_CHECK(dbg, at, a.budget)) kept[at] = t;
    }
    gt0 += __popc(bg);
    eq0 += __popc(be);
  }
  meet();                                       // a block's shared memory is read by its cluster until here
}

// One thread block per (destination block, kv head, sequence): T threads move the keys and T the values, up to four times 16
// codes each, which stay in registers between the maximum and the rounding; T follows the block's size, so that
// its threads are all busy, and 1536 threads a multiprocessor cover the look-ups (place -> block -> codes and scale):
// 1024 leave it at 98 us for eight conversations of 2048 kept tokens, 32 heads of 128, against 87.  It is bound by the instructions
// of the correctly rounded quotients more than by the 38 us of its bytes.  (Blocks of 16 x 64 elements with T = 128 took
// 68 us where T = 32 takes 41.)
template <int D, int PASSES, int T>
__global__ void __launch_bounds__(2 * T, PASSES == 4 && T == 32 ? 20 : 768 / T)
kv_gather_kernel(KvShape sh, KvBatch kb, int budget, const int32_t* __restrict__ kept, int8_t* codes, float* scales, float* score,
                 const int32_t* __restrict__ dst_table, int dst_max_blocks, int* dbg) {
  constexpr int CHUNKS = D / 16, ROWS = T / CHUNKS, WARPS = T / 32;
  __shared__ float warp_max[2 * WARPS];
  kv_begin();
  const int b = blockIdx.y, h = blockIdx.x % sh.kv_heads, j = blockIdx.x / sh.kv_heads;
  int len = kb.lens[b];
  len = len < 0 ? 0 : (len > kb.max_len ? kb.max_len : len);
  int count = len < budget ? len : budget;
  const int base = j * sh.block;
  if (base >= count || j >= dst_max_blocks) return;
  const int n = count - base < sh.block ? count - base : sh.block;
  const int dst_id = kv_block(dst_table, dst_max_blocks, sh.num_blocks, b, j);
  if (dst_id < 0) return;
  const int32_t* from = kept + ((long long)b * sh.kv_heads + h) * budget + base;
  const int which = threadIdx.x / T, t = threadIdx.x % T, chunk = t % CHUNKS, row = t / CHUNKS;
  uint4 x[PASSES];
  float s[PASSES], mx = 0.f;
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int slot = p * ROWS + row;
    x[p] = make_uint4(0, 0, 0, 0);
    s[p] = 0.f;
    if (slot < n) {
      const int pos = from[slot];
      const int id = QALORA_CHECK(dbg, pos, len) ? kv_block(kb.table, kb.max_blocks, sh.num_blocks, b, pos >> sh.log_block) : -1;
      if (id >= 0) {
        const long long plane = ((long long)id * 2 + which) * sh.kv_heads + h;
        s[p] = scales[plane];
        x[p] = *reinterpret_cast<const uint4*>(codes + (plane * sh.block + (pos & (sh.block - 1))) * D + chunk * 16);
      }
    }
  }
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    // largest magnitude of 16 codes, two at a time as signed 16-bit numbers
    const uint32_t w[4] = {x[p].x, x[p].y, x[p].z, x[p].w};
    uint32_t hi = 0, lo = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t a = signed_pair<0>(w[q]), c = signed_pair<1>(w[q]);
      hi = max_s16x2(max_s16x2(hi, a), c);
      lo = min_s16x2(min_s16x2(lo, a), c);
    }
    const int top = max((int)(int16_t)(hi & 0xffffu), (int)(int16_t)(hi >> 16)), low = min((int)(int16_t)(lo & 0xffffu), (int)(int16_t)(lo >> 16));
    const float m = (float)max(top, -low);
    mx = fmaxf(mx, __fmul_rn(m, s[p]));                 // (the rounded product grows with the code)
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
  if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = mx;
  __syncthreads();
  mx = warp_max[which * WARPS];
#pragma unroll
  for (int y = 1; y < WARPS; ++y) mx = fmaxf(mx, warp_max[which * WARPS + y]);
  const float scale = __fdiv_rn(mx, 127.f);
  const long long plane = ((long long)dst_id * 2 + which) * sh.kv_heads + h;
  if (t == 0 && QALORA_CHECK(dbg, plane, (long long)sh.num_blocks * 2 * sh.kv_heads)) scales[plane] = scale;
  const bool exact = !kv_fast_scale(scale);
  const float inv = exact ? 0.f : __fdiv_rn(1.f, scale);
  int8_t* dst = codes + plane * sh.block * D;
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int slot = p * ROWS + row;
    if (slot >= n || !QALORA_CHECK(dbg, slot, sh.block)) continue;
    const uint32_t w[4] = {x[p].x, x[p].y, x[p].z, x[p].w};
    const float2 ss = make_float2(s[p], s[p]);
    uint2 o[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      float2 f[4];
      kv_floats4(w[2 * q], f[0], f[1]);
      kv_floats4(w[2 * q + 1], f[2], f[3]);
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = ptx::fmul2(f[e], ss);
      o[q] = kv_codes8(f, scale, inv);
      if (exact) {
        o[q].x = kv_codes4_any(f[0].x, f[0].y, f[1].x, f[1].y, scale);
        o[q].y = kv_codes4_any(f[2].x, f[2].y, f[3].x, f[3].y, scale);
      }
    }
    *reinterpret_cast<uint4*>(dst + slot * D + chunk * 16) = make_uint4(o[0].x, o[0].y, o[1].x, o[1].y);
  }
  for (int slot = threadIdx.x; slot < n; slot += 2 * T) {
    const int pos = from[slot];
    const int id = QALORA_CHECK(dbg, pos, len) ? kv_block(kb.table, kb.max_blocks, sh.num_blocks, b, pos >> sh.log_block) : -1;
    const float moved = id < 0 ? 0.f : score[((long long)id * sh.kv_heads + h) * sh.block + (pos & (sh.block - 1))];
    score[((long long)dst_id * sh.kv_heads + h) * sh.block + slot] = moved;
  }
}

template <int D>
int gather_passes(const KvShape& sh, const KvBatch& b, dim3 grid, int budget, const int32_t* kept, int8_t* codes, float* scales,
                  float* score, const int32_t* dst_table, int dst_max_blocks, cudaStream_t st) {
#define QALORA_KV_GATHER(P, T)                                                                                               \
    return kv_launch(kv_gather_kernel<D, P, T>, grid, 2 * T, 0, st, sh, b, budget, kept, codes, scales, score, dst_table,    \
                     dst_max_blocks, debug_words());
  // (twice the threads where all blocks run at once all the same: seven sequences of 411 tokens, 40 heads of 64,
  // cut to 149 in 14.6 us against 17.5)
  const bool wide = (long long)grid.x * grid.y * sh.block * (D / 16) <= 2ll * 768 * device_sm_count();
  switch (sh.block * (D / 16)) {                                 // pieces of 16 codes
    case 64: QALORA_KV_GATHER(2, 32)
    case 128: if (wide) QALORA_KV_GATHER(2, 64) QALORA_KV_GATHER(4, 32)
    case 256: if (wide) QALORA_KV_GATHER(2, 128) QALORA_KV_GATHER(4, 64)
    case 512: if (wide) QALORA_KV_GATHER(2, 256) QALORA_KV_GATHER(4, 128)
    case 1024: if (wide) QALORA_KV_GATHER(2, 512) QALORA_KV_GATHER(4, 256)
    default: return QALORA_ERR_UNSUPPORTED_SHAPE;
  }
#undef QALORA_KV_GATHER
}

}  // namespace

int launch_kv_evict(const KvShape& sh, const KvBatch& b, int budget, int recent, int8_t* codes, float* scales, float* score,
                    const int32_t* dst_table, int dst_max_blocks, int32_t* dst_lens, int32_t* kept, cudaStream_t st) {
  // Thread blocks per cluster: enough to hold every key in shared memory, and more while the
  // grid leaves multiprocessors free and each still has some thousand keys.
  const long long pairs = (long long)b.batch * sh.kv_heads;
  int C = 1;
  while (C < SEL_MAX_CLUSTER && ((b.max_len + C - 1) / C > SEL_CACHED_KEYS / 2 ||
                                 (pairs * C * 2 <= device_sm_count() && b.max_len / C >= 4096)))
    C *= 2;
  const int per = ((b.max_len + C - 1) / C + 3) & ~3;
  if (pairs * C > 0x7fffffffll) return QALORA_ERR_UNSUPPORTED_SHAPE;
  SelectArgs a{score, dst_lens, kept, budget, recent, per <= SEL_CACHED_KEYS ? per : 0};
  // Few keys to a block: eight blocks of 256 threads to a multiprocessor instead of two, and cheaper meetings (480 pairs of
  // 337 tokens 38.9 -> 29.8 us with their move; 256 of 8000 107 -> 104).  With fewer pairs than multiprocessors
  // the many threads of one block read faster (128 pairs of 8000: 57 us against 64).
  const int threads = per <= (pairs * C > device_sm_count() ? 8192 : 2048) ? 256 : 1024;
  const auto kernel = threads == 256 ? kv_select_kernel<256> : kv_select_kernel<1024>;
  static PerDeviceOnce once;
  const int ok = once.run([] {
    const cudaError_t e = cudaFuncSetAttribute(kv_select_kernel<256>, cudaFuncAttributeMaxDynamicSharedMemorySize, SEL_CACHED_KEYS * 4);
    return e != cudaSuccess ? e : cudaFuncSetAttribute(kv_select_kernel<1024>, cudaFuncAttributeMaxDynamicSharedMemorySize, SEL_CACHED_KEYS * 4);
  });
  if (ok != QALORA_OK) return ok;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(pairs * C));
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = (size_t)a.cached * 4;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)C;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  if (cudaLaunchKernelEx(&cfg, kernel, sh, b, a, debug_words()) != cudaSuccess) return QALORA_ERR_CUDA;
  count_launch();
  const int most = b.max_len < budget ? b.max_len : budget, blocks = (most + sh.block - 1) / sh.block;
  if (blocks == 0) return cuda_status(cudaGetLastError());
  if ((long long)blocks * sh.kv_heads > 0x7fffffffll) return QALORA_ERR_UNSUPPORTED_SHAPE;
  const dim3 grid((unsigned)(blocks * sh.kv_heads), (unsigned)b.batch);
  return sh.dim == 128 ? gather_passes<128>(sh, b, grid, budget, kept, codes, scales, score, dst_table, dst_max_blocks, st)
                       : gather_passes<64>(sh, b, grid, budget, kept, codes, scales, score, dst_table, dst_max_blocks, st);
}

}  // namespace qalora
