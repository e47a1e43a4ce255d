// Key/value cache in 8 bits: storing new tokens (append) and reading tokens back (read).
// Both are bound by HBM: append reads 2 B and writes 1 B per element, read the reverse.
#define QALORA_TU 10
#include "kv.cuh"

namespace qalora {

namespace {

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t max_abs2(uint32_t m, uint32_t w) { return max_u16x2(m, w & 0x7fff7fffu); }

// One thread block per (block of tokens that new rows enter, kv head, sequence): the new rows of
// that block stay in registers between the maximum and the rounding, so each element is read once.
// T threads for keys and T for values, PASSES * T * 8 = block * D elements: T follows the block's size, so that its threads
// are all busy, mostly with eight pieces each (three prompts of up to 4093 tokens, 32 heads: blocks of 16 x 128 elements 79 us with
// T = 128, 52 with 32; of 16 x 64 57 and 35).
template <int D, int PASSES, int T>
__global__ void __launch_bounds__(2 * T, (PASSES <= 8 ? 512 : 256) / T)
kv_append_kernel(KvShape sh, KvBatch kb, const __nv_bfloat16* __restrict__ k, long long k_stride,
                 const __nv_bfloat16* __restrict__ v, long long v_stride, int8_t* __restrict__ codes, float* __restrict__ scales,
                 float* __restrict__ score, int32_t* __restrict__ dev_status, int* dbg) {
  constexpr int CHUNKS = D / 8, ROWS = T / CHUNKS, WARPS = T / 32;
  __shared__ uint32_t warp_max[2 * WARPS];
  kv_begin();
  const int b = blockIdx.y, h = blockIdx.x % sh.kv_heads, j = blockIdx.x / sh.kv_heads;
  const KvSeq s = kv_seq(kb, b);
  if (s.n == 0) return;
  const int lo = s.first > 0 ? s.first : 0;
  const int jb = (lo >> sh.log_block) + j;
  if (jb > (s.len - 1) >> sh.log_block) return;        // (compared as blocks: a position behind the last one may pass 2^31)
  const int base = jb * sh.block;
  const int s0 = lo > base ? lo - base : 0;                                       // slots s0 .. s1 - 1 are new
  const int s1 = s.len - base < sh.block ? s.len - base : sh.block;
  const int raw = kb.table[(size_t)b * kb.max_blocks + jb];
  const int which = threadIdx.x / T, t = threadIdx.x % T, chunk = t % CHUNKS, row = t / CHUNKS;
  const __nv_bfloat16* src = which == 0 ? k : v;
  const long long stride = which == 0 ? k_stride : v_stride;

  const __nv_bfloat16* from = src + ((long long)s.row0 + (base + row - s.first)) * stride + (long long)h * D + chunk * 8;
  const long long step = ROWS * stride;
  uint4 x[PASSES];
  uint32_t mx = 0;
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int slot = p * ROWS + row;
    x[p] = make_uint4(0, 0, 0, 0);
    if ((uint32_t)(slot - s0) < (uint32_t)(s1 - s0) && QALORA_CHECK(dbg, (long long)s.row0 + (base + slot - s.first), kb.m))
      x[p] = __ldcs(reinterpret_cast<const uint4*>(from + p * step));
  }
  const int id = raw >= 0 && raw < sh.num_blocks ? raw : -1;      // (looked up while the rows are on their way)
  if (id < 0) return;
  const long long plane = ((long long)id * 2 + which) * sh.kv_heads + h;
  int8_t* dst = codes + plane * sh.block * D;
  const float before = scales[plane];
#pragma unroll
  for (int p = 0; p < PASSES; ++p) mx = max_abs2(max_abs2(max_abs2(max_abs2(mx, x[p].x), x[p].y), x[p].z), x[p].w);
  mx = max(mx & 0xffffu, mx >> 16);
  mx = __reduce_max_sync(0xffffffffu, mx);
  if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = mx;
  auto of_plane = [&] {
    uint32_t most = warp_max[which * WARPS];
#pragma unroll
    for (int w = 1; w < WARPS; ++w) most = max(most, warp_max[which * WARPS + w]);
    return most;
  };
  __syncthreads();
  mx = of_plane();
  const bool odd = mx >= 0x7f80u;                      // an infinity or a NaN among the new elements
  if (__syncthreads_or(odd)) {                         // (both halves take part in the barriers)
    uint32_t fin = 0;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const uint32_t w[4] = {x[p].x, x[p].y, x[p].z, x[p].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t a = w[i] & 0x7fffu, c = (w[i] >> 16) & 0x7fffu;
        if (a < 0x7f80u) fin = max(fin, a);
        if (c < 0x7f80u) fin = max(fin, c);
      }
    }
    fin = __reduce_max_sync(0xffffffffu, fin);
    if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = fin;
    __syncthreads();
    mx = of_plane();
    if (odd && t == 0 && dev_status != nullptr) atomicOr(dev_status, 1);
  }
  const float need = __fdiv_rn(__uint_as_float(mx << 16), 127.f);
  const float scale = s0 > 0 ? fmaxf(before, need) : need;
  if (t == 0 && QALORA_CHECK(dbg, plane, (long long)sh.num_blocks * 2 * sh.kv_heads)) scales[plane] = scale;

  if (s0 > 0 && scale > before) {                      // the block's earlier codes under the larger scale
    const float ratio = __fdiv_rn(before, scale);
    for (int i = t; i < s0 * (D / 16); i += T) {
      uint4 c = reinterpret_cast<uint4*>(dst)[i];
      uint32_t* w = reinterpret_cast<uint32_t*>(&c);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float2 f0, f1;
        kv_floats4(w[q], f0, f1);
        // (scalar operations: of a packed product and sum ptxas makes one rounding)
        const float p[4] = {f0.x, f0.y, f1.x, f1.y};
        uint32_t r[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = __float_as_uint(__fadd_rn(__fmul_rn(p[e], ratio), 12582912.f));
        w[q] = kv_pack4(r[0], r[1], r[2], r[3]);
      }
      if (QALORA_CHECK(dbg, i, sh.block * (D / 16))) reinterpret_cast<uint4*>(dst)[i] = c;
    }
  }
  const bool exact = odd || !kv_fast_scale(scale);
  const float inv = exact ? 0.f : __fdiv_rn(1.f, scale);
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int slot = p * ROWS + row;
    if ((uint32_t)(slot - s0) >= (uint32_t)(s1 - s0) || !QALORA_CHECK(dbg, slot, sh.block)) continue;
    const float2 e[4] = {make_float2(bf16_lo(x[p].x), bf16_hi(x[p].x)), make_float2(bf16_lo(x[p].y), bf16_hi(x[p].y)),
                         make_float2(bf16_lo(x[p].z), bf16_hi(x[p].z)), make_float2(bf16_lo(x[p].w), bf16_hi(x[p].w))};
    uint2 out = kv_codes8(e, scale, inv);
    if (exact) {
      out.x = kv_codes4_any(e[0].x, e[0].y, e[1].x, e[1].y, scale);
      out.y = kv_codes4_any(e[2].x, e[2].y, e[3].x, e[3].y, scale);
    }
    *reinterpret_cast<uint2*>(dst + slot * D + chunk * 8) = out;
  }
  if (score != nullptr)
    for (int slot = s0 + threadIdx.x; slot < s1; slot += 2 * T)
      score[((long long)id * sh.kv_heads + h) * sh.block + slot] = 0.f;
}

// One thread block per (block of tokens that is read from, kv head, sequence), half of it for keys and half for
// values: one look-up and one scale each, 16 codes per thread and pass.
template <int D, int PASSES, int T, bool BF16>
__global__ void __launch_bounds__(2 * T, (PASSES == 8 ? 384 : 640) / T)
kv_read_kernel(KvShape sh, KvBatch kb, const int8_t* __restrict__ codes, const float* __restrict__ scales,
               void* __restrict__ k, void* __restrict__ v, int* dbg) {
  constexpr int CHUNKS = D / 16, ROWS = T / CHUNKS;
  kv_begin();
  const int b = blockIdx.y, h = blockIdx.x % sh.kv_heads, j = blockIdx.x / sh.kv_heads;
  const int r0 = kb.starts[b], r1 = kb.starts[b + 1], first = kb.lens[b];         // (lens: position of the first token read)
  if (r0 < 0 || r1 < r0 || r1 > kb.m || r1 - r0 > kb.max_new) return;
  const long long stop = (long long)first + (r1 - r0);
  const int lo = first > 0 ? first : 0, hi = (int)(stop < kb.max_len ? stop : kb.max_len);   // positions read: lo .. hi - 1
  const int jb = (lo >> sh.log_block) + j;
  if (lo >= hi || jb > (hi - 1) >> sh.log_block) return;   // (first may be any number: jb * block may pass 2^31)
  const int base = jb * sh.block;
  const int s0 = lo > base ? lo - base : 0, s1 = hi - base < sh.block ? hi - base : sh.block;
  const int which = threadIdx.x / T, t = threadIdx.x % T, chunk = t % CHUNKS, row = t / CHUNKS;
  void* out = which == 0 ? k : v;
  const int id = kv_block(kb.table, kb.max_blocks, sh.num_blocks, b, jb);
  if (id < 0 || out == nullptr) return;
  const long long plane = ((long long)id * 2 + which) * sh.kv_heads + h;
  const int8_t* src = codes + plane * sh.block * D + chunk * 16;
  const float s = scales[plane];
  uint4 c[PASSES];
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int slot = p * ROWS + row;
    c[p] = make_uint4(0, 0, 0, 0);
    if (slot >= s0 && slot < s1) c[p] = __ldcs(reinterpret_cast<const uint4*>(src + slot * D));
  }
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int slot = p * ROWS + row;
    const long long out_row = (long long)r0 + (base + slot - first);
    if (slot < s0 || slot >= s1 || !QALORA_CHECK(dbg, out_row, kb.m)) continue;
    const uint32_t w[4] = {c[p].x, c[p].y, c[p].z, c[p].w};
    const long long at = (out_row * sh.kv_heads + h) * D + chunk * 16;
    float2 f[8];
    const float2 ss = make_float2(s, s);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      kv_floats4(w[e], f[2 * e], f[2 * e + 1]);
      f[2 * e] = ptx::fmul2(f[2 * e], ss);
      f[2 * e + 1] = ptx::fmul2(f[2 * e + 1], ss);
    }
    if (BF16) {
      uint32_t o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const __nv_bfloat162 two = __floats2bfloat162_rn(f[e].x, f[e].y);
        o[e] = *reinterpret_cast<const uint32_t*>(&two);
      }
      uint4* dst = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(out) + at);
      __stcs(dst, make_uint4(o[0], o[1], o[2], o[3]));
      __stcs(dst + 1, make_uint4(o[4], o[5], o[6], o[7]));
    } else {
      float4* dst = reinterpret_cast<float4*>(static_cast<float*>(out) + at);
#pragma unroll
      for (int e = 0; e < 4; ++e) __stcs(dst + e, make_float4(f[2 * e].x, f[2 * e].y, f[2 * e + 1].x, f[2 * e + 1].y));
    }
  }
}

template <int D, bool BF16>
int read_passes(const KvShape& sh, const KvBatch& b, dim3 grid, const int8_t* codes, const float* scales, void* k, void* v, cudaStream_t st) {
#define QALORA_KV_READ(P, T) return kv_launch(kv_read_kernel<D, P, T, BF16>, grid, 2 * T, 0, st, sh, b, codes, scales, k, v, debug_words());
  switch (sh.block * (D / 16)) {                                 // pieces of 16 codes
    case 64: QALORA_KV_READ(2, 32)
    case 128: QALORA_KV_READ(2, 64)
    case 256: QALORA_KV_READ(2, 128)
    case 512: QALORA_KV_READ(4, 128)
    case 1024: QALORA_KV_READ(8, 128)
    default: return QALORA_ERR_UNSUPPORTED_SHAPE;
  }
#undef QALORA_KV_READ
}

template <int D>
int append_passes(const KvShape& sh, const KvBatch& b, dim3 grid, const __nv_bfloat16* k, int64_t k_stride, const __nv_bfloat16* v,
                  int64_t v_stride, int8_t* codes, float* scales, float* score, int32_t* dev_status, cudaStream_t st) {
#define QALORA_KV_APPEND(P, T)                                                                                             \
    return kv_launch(kv_append_kernel<D, P, T>, grid, 2 * T, 0, st, sh, b, k, (long long)k_stride, v, (long long)v_stride, codes, \
                     scales, score, dev_status, debug_words());
  switch (sh.block * (D / 8)) {                                  // pieces of 8 elements
    case 128: QALORA_KV_APPEND(4, 32)
    case 256: QALORA_KV_APPEND(8, 32)
    case 512: QALORA_KV_APPEND(8, 64)
    case 1024: QALORA_KV_APPEND(8, 128)
    case 2048: QALORA_KV_APPEND(16, 128)
    default: return QALORA_ERR_UNSUPPORTED_SHAPE;
  }
#undef QALORA_KV_APPEND
}

}  // namespace

// Blocks that `n` consecutive tokens can lie in, wherever the first one lies in its block.
static int touched_blocks(const KvShape& sh, const KvBatch& b, int n) {
  const int touched = (n + sh.block - 2) / sh.block + 1;
  return touched < b.max_blocks ? touched : b.max_blocks;
}

int launch_kv_append(const KvShape& sh, const KvBatch& b, const __nv_bfloat16* k, int64_t k_stride, const __nv_bfloat16* v,
                     int64_t v_stride, int8_t* codes, float* scales, float* score, int32_t* dev_status, cudaStream_t st) {
  const int bound = touched_blocks(sh, b, b.max_new);
  if ((long long)bound * sh.kv_heads > 0x7fffffffll) return QALORA_ERR_UNSUPPORTED_SHAPE;
  const dim3 grid((unsigned)(bound * sh.kv_heads), (unsigned)b.batch);
  return sh.dim == 128 ? append_passes<128>(sh, b, grid, k, k_stride, v, v_stride, codes, scales, score, dev_status, st)
                       : append_passes<64>(sh, b, grid, k, k_stride, v, v_stride, codes, scales, score, dev_status, st);
}

int launch_kv_read(const KvShape& sh, const KvBatch& b, const int8_t* codes, const float* scales, void* k, void* v, bool bf16,
                   cudaStream_t st) {
  const int bound = touched_blocks(sh, b, b.max_new);
  if ((long long)bound * sh.kv_heads > 0x7fffffffll) return QALORA_ERR_UNSUPPORTED_SHAPE;
  const dim3 grid((unsigned)(bound * sh.kv_heads), (unsigned)b.batch);
  if (sh.dim == 128)
    return bf16 ? read_passes<128, true>(sh, b, grid, codes, scales, k, v, st) : read_passes<128, false>(sh, b, grid, codes, scales, k, v, st);
  return bf16 ? read_passes<64, true>(sh, b, grid, codes, scales, k, v, st) : read_passes<64, false>(sh, b, grid, codes, scales, k, v, st);
}

}  // namespace qalora
