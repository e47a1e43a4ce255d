// Key/value cache in 8 bits: storing new tokens (append) and reading tokens back (read).
// Both are bound by HBM: append reads 2 B and writes 1 B per element, read the reverse.
#define QALORA_TU 10
#include "kv.cuh"

namespace qalora {

namespace {

constexpr int KV_THREADS = 256;            // 128 threads for keys, 128 for values

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t max_abs2(uint32_t m, uint32_t w) { return __vmaxu2(m, w & 0x7fff7fffu); }

// One thread block per (block of tokens that new rows enter, kv head, sequence): the new rows of
// that block stay in registers between the maximum and the rounding, so each element is read once.
// PASSES rows of D elements per 128 / (D / 8) rows in flight: PASSES * 128 * 8 = block * D elements.
template <int D, int PASSES>
__global__ void __launch_bounds__(KV_THREADS)
kv_append_kernel(KvShape sh, KvBatch kb, const __nv_bfloat16* __restrict__ k, long long k_stride,
                 const __nv_bfloat16* __restrict__ v, long long v_stride, int8_t* __restrict__ codes, float* __restrict__ scales,
                 float* __restrict__ score, int32_t* __restrict__ dev_status, int* dbg) {
  constexpr int CHUNKS = D / 8, ROWS = 128 / CHUNKS;
  __shared__ uint32_t warp_max[8];
  const int b = blockIdx.y, h = blockIdx.x % sh.kv_heads, j = blockIdx.x / sh.kv_heads;
  const KvSeq s = kv_seq(kb, b);
  if (s.n == 0) return;
  const int lo = s.first > 0 ? s.first : 0;
  const int jb = lo / sh.block + j, base = jb * sh.block;
  if (base >= s.len) return;
  const int s0 = lo > base ? lo - base : 0;                                       // slots s0 .. s1 - 1 are new
  const int s1 = s.len - base < sh.block ? s.len - base : sh.block;
  const int id = kv_block(kb.table, kb.max_blocks, sh.num_blocks, b, jb);
  if (id < 0) return;
  const int which = threadIdx.x >> 7, t = threadIdx.x & 127, chunk = t % CHUNKS, row = t / CHUNKS;
  const __nv_bfloat16* src = which == 0 ? k : v;
  const long long stride = which == 0 ? k_stride : v_stride;
  const long long plane = ((long long)id * 2 + which) * sh.kv_heads + h;
  int8_t* dst = codes + plane * sh.block * D;
  const float before = scales[plane];

  uint4 x[PASSES];
  uint32_t mx = 0;
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int slot = p * ROWS + row;
    x[p] = make_uint4(0, 0, 0, 0);
    if (slot >= s0 && slot < s1) {
      const long long r = (long long)s.row0 + (base + slot - s.first);
      if (QALORA_CHECK(dbg, r, kb.m))
        x[p] = __ldcs(reinterpret_cast<const uint4*>(src + r * stride + (long long)h * D + chunk * 8));
    }
  }
#pragma unroll
  for (int p = 0; p < PASSES; ++p) mx = max_abs2(max_abs2(max_abs2(max_abs2(mx, x[p].x), x[p].y), x[p].z), x[p].w);
  mx = max(mx & 0xffffu, mx >> 16);
  mx = __reduce_max_sync(0xffffffffu, mx);
  if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = mx;
  __syncthreads();
  mx = max(max(warp_max[which * 4], warp_max[which * 4 + 1]), max(warp_max[which * 4 + 2], warp_max[which * 4 + 3]));
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
    mx = max(max(warp_max[which * 4], warp_max[which * 4 + 1]), max(warp_max[which * 4 + 2], warp_max[which * 4 + 3]));
    if (odd && t == 0 && dev_status != nullptr) atomicOr(dev_status, 1);
  }
  const float need = __fdiv_rn(__uint_as_float(mx << 16), 127.f);
  const float scale = s0 > 0 ? fmaxf(before, need) : need;
  if (t == 0 && QALORA_CHECK(dbg, plane, (long long)sh.num_blocks * 2 * sh.kv_heads)) scales[plane] = scale;

  if (s0 > 0 && scale > before) {                      // the block's earlier codes under the larger scale
    const float ratio = __fdiv_rn(before, scale);
    for (int i = t; i < s0 * (D / 16); i += 128) {
      uint4 c = reinterpret_cast<uint4*>(dst)[i];
      uint32_t* w = reinterpret_cast<uint32_t*>(&c);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t r[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          r[e] = __float_as_uint(__fadd_rn(__fmul_rn((float)(int8_t)(w[q] >> (8 * e)), ratio), 12582912.f));
        w[q] = kv_pack4(r[0], r[1], r[2], r[3]);
      }
      if (QALORA_CHECK(dbg, i, sh.block * (D / 16))) reinterpret_cast<uint4*>(dst)[i] = c;
    }
  }
  const bool fast = !odd && kv_fast_scale(scale);
  const float inv = fast ? __fdiv_rn(1.f, scale) : 0.f;
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int slot = p * ROWS + row;
    if (slot < s0 || slot >= s1 || !QALORA_CHECK(dbg, slot, sh.block)) continue;
    const float a[4] = {bf16_lo(x[p].x), bf16_hi(x[p].x), bf16_lo(x[p].y), bf16_hi(x[p].y)};
    const float c[4] = {bf16_lo(x[p].z), bf16_hi(x[p].z), bf16_lo(x[p].w), bf16_hi(x[p].w)};
    uint2 out;
    if (fast) { out.x = kv_codes4(a, scale, inv); out.y = kv_codes4(c, scale, inv); }
    else { out.x = kv_codes4_any(a, scale); out.y = kv_codes4_any(c, scale); }
    *reinterpret_cast<uint2*>(dst + slot * D + chunk * 8) = out;
  }
  if (score != nullptr)
    for (int slot = s0 + threadIdx.x; slot < s1; slot += KV_THREADS)
      score[((long long)id * sh.kv_heads + h) * sh.block + slot] = 0.f;
}

// READ_ROWS tokens of one sequence per thread block; a thread converts 16 codes at a time.
constexpr int READ_ROWS = 8;

template <bool BF16>
__global__ void __launch_bounds__(KV_THREADS)
kv_read_kernel(KvShape sh, KvBatch kb, const int8_t* __restrict__ codes, const float* __restrict__ scales,
               void* __restrict__ k, void* __restrict__ v, int* dbg) {
  const int b = blockIdx.y;
  const int r0 = kb.starts[b], r1 = kb.starts[b + 1];
  if (r0 < 0 || r1 < r0 || r1 > kb.m || r1 - r0 > kb.max_new) return;
  const int row0 = blockIdx.x * READ_ROWS;
  const int rows = r1 - r0 - row0 < READ_ROWS ? r1 - r0 - row0 : READ_ROWS;
  if (rows <= 0) return;
  const long long pos0 = (long long)kb.lens[b] + row0;          // (lens: position of the first token read)
  const int per_head = sh.dim / 16, per_plane = sh.kv_heads * per_head, per_row = 2 * per_plane;
  for (int i = threadIdx.x; i < rows * per_row; i += KV_THREADS) {
    const int row = i / per_row, rest = i % per_row, which = rest / per_plane, col = rest % per_plane;
    void* out = which == 0 ? k : v;
    const long long pos = pos0 + row;
    if (out == nullptr || pos < 0 || pos >= (long long)kb.max_blocks * sh.block) continue;
    const int h = col / per_head, part = col % per_head, slot = (int)(pos % sh.block);
    const int id = kv_block(kb.table, kb.max_blocks, sh.num_blocks, b, (int)(pos / sh.block));
    if (id < 0) continue;
    const long long plane = ((long long)id * 2 + which) * sh.kv_heads + h;
    if (!QALORA_CHECK(dbg, plane, (long long)sh.num_blocks * 2 * sh.kv_heads)) continue;
    const float s = scales[plane];
    const uint4 c = __ldcs(reinterpret_cast<const uint4*>(codes + (plane * sh.block + slot) * sh.dim + part * 16));
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    const long long at = ((long long)(r0 + row0 + row) * sh.kv_heads + h) * sh.dim + part * 16;
    float f[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) f[e] = __fmul_rn((float)(int8_t)(w[e >> 2] >> (8 * (e & 3))), s);
    if (BF16) {
      uint32_t o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const __nv_bfloat162 two = __floats2bfloat162_rn(f[2 * e], f[2 * e + 1]);
        o[e] = *reinterpret_cast<const uint32_t*>(&two);
      }
      uint4* dst = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(out) + at);
      __stcs(dst, make_uint4(o[0], o[1], o[2], o[3]));
      __stcs(dst + 1, make_uint4(o[4], o[5], o[6], o[7]));
    } else {
      float4* dst = reinterpret_cast<float4*>(static_cast<float*>(out) + at);
#pragma unroll
      for (int e = 0; e < 4; ++e) __stcs(dst + e, make_float4(f[4 * e], f[4 * e + 1], f[4 * e + 2], f[4 * e + 3]));
    }
  }
}

template <int D>
int append_passes(const KvShape& sh, const KvBatch& b, dim3 grid, const __nv_bfloat16* k, int64_t k_stride, const __nv_bfloat16* v,
                  int64_t v_stride, int8_t* codes, float* scales, float* score, int32_t* dev_status, cudaStream_t st) {
  const int passes = sh.block * D / 1024;
#define QALORA_KV_APPEND(P)                                                                                              \
  case P:                                                                                                                \
    kv_append_kernel<D, P><<<grid, KV_THREADS, 0, st>>>(sh, b, k, k_stride, v, v_stride, codes, scales, score, dev_status, \
                                                        debug_words());                                                  \
    break;
  switch (passes) {
    QALORA_KV_APPEND(1) QALORA_KV_APPEND(2) QALORA_KV_APPEND(4) QALORA_KV_APPEND(8) QALORA_KV_APPEND(16)
    default: return QALORA_ERR_UNSUPPORTED_SHAPE;
  }
#undef QALORA_KV_APPEND
  count_launch();
  return cuda_status(cudaGetLastError());
}

}  // namespace

int launch_kv_append(const KvShape& sh, const KvBatch& b, const __nv_bfloat16* k, int64_t k_stride, const __nv_bfloat16* v,
                     int64_t v_stride, int8_t* codes, float* scales, float* score, int32_t* dev_status, cudaStream_t st) {
  // blocks that max_new consecutive tokens can enter, wherever the first one lies in its block
  const int touched = (b.max_new + sh.block - 2) / sh.block + 1;
  const int bound = touched < b.max_blocks ? touched : b.max_blocks;
  if ((long long)bound * sh.kv_heads > 0x7fffffffll) return QALORA_ERR_UNSUPPORTED_SHAPE;
  const dim3 grid((unsigned)(bound * sh.kv_heads), (unsigned)b.batch);
  return sh.dim == 128 ? append_passes<128>(sh, b, grid, k, k_stride, v, v_stride, codes, scales, score, dev_status, st)
                       : append_passes<64>(sh, b, grid, k, k_stride, v, v_stride, codes, scales, score, dev_status, st);
}

int launch_kv_read(const KvShape& sh, const KvBatch& b, const int8_t* codes, const float* scales, void* k, void* v, bool bf16,
                   cudaStream_t st) {
  const dim3 grid((unsigned)((b.max_new + READ_ROWS - 1) / READ_ROWS), (unsigned)b.batch);
  if (bf16) kv_read_kernel<true><<<grid, KV_THREADS, 0, st>>>(sh, b, codes, scales, k, v, debug_words());
  else kv_read_kernel<false><<<grid, KV_THREADS, 0, st>>>(sh, b, codes, scales, k, v, debug_words());
  count_launch();
  return cuda_status(cudaGetLastError());
}

}  // namespace qalora
