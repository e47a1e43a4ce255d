// Shared helpers of the key/value cache kernels: the description of a batch, the checks of its
// device-side entries, and conversions between values and 8-bit codes.
#pragma once
#include "common.cuh"
#include "ptx.cuh"

namespace qalora {

struct KvShape {
  int heads, kv_heads, group, dim, block, log_block, num_blocks;
};

// A batch as the kernels see it.
struct KvBatch {
  const int32_t* starts;   // [batch + 1]
  const int32_t* lens;     // [batch]
  const int32_t* table;    // [batch][max_blocks]
  int batch, max_blocks;
  int m, max_new;          // rows in all / of one sequence
  int max_len;             // tokens of one sequence that a kernel may visit: min(max_len, max_blocks * block)
  int n_lo, n_hi;          // sequences with fewer or more new rows are another kernel's
};

int check_kv_desc(const qalora_kv_desc* desc, KvShape* sh);

int launch_kv_append(const KvShape& sh, const KvBatch& b, const __nv_bfloat16* k, int64_t k_stride, const __nv_bfloat16* v,
                     int64_t v_stride, int8_t* codes, float* scales, float* score, int32_t* dev_status, cudaStream_t st);
int launch_kv_read(const KvShape& sh, const KvBatch& b, const int8_t* codes, const float* scales, void* k, void* v, bool bf16,
                   cudaStream_t st);

struct KvAttention {
  const __nv_bfloat16* q;
  int64_t q_stride;
  const int8_t* codes;
  const float* scales;
  float softmax_scale;
  __nv_bfloat16* out;
  float* lse;
  const float* score_in;
  float* score_out;
};
size_t kv_attention_workspace(const KvShape& sh, int batch, int64_t m, int max_new, int max_len, bool with_score, Workspace* guards);
int launch_kv_attention(const KvShape& sh, const KvBatch& b, const KvAttention& a, void* workspace, int max_len, cudaStream_t st);

// Many new rows per sequence (kv_prompt.cu): tensor-core tiles of 128 rows x 128 tokens.
struct KvPromptScratch {
  int splits;              // parts of a row tile's tokens
  long long slots;         // tiles of 128 rows of one kv head, at most
  size_t part_ml, part_o;  // bytes: {maximum, sum} and output of each part's rows (splits > 1)
  size_t q_image, rows;    // bytes: the queries' tiles as the tensor core reads them, {scale, lse} of their rows (gathered weights)
};
KvPromptScratch kv_prompt_scratch(const KvShape& sh, int batch, int64_t m, int max_len, bool with_score);
int launch_kv_prompt(const KvShape& sh, const KvBatch& b, const KvAttention& a, const KvPromptScratch& s, float2* part_ml,
                     float* part_o, uint8_t* q_image, float* rows, int* status, cudaStream_t st);

int launch_kv_evict(const KvShape& sh, const KvBatch& b, int budget, int recent, int8_t* codes, float* scales, float* score,
                    const int32_t* dst_table, int dst_max_blocks, int32_t* dst_lens, int32_t* kept, cudaStream_t st);

#ifdef __CUDACC__
// Launches a kernel of the cache so that its blocks may be set up while the kernel before it in the stream ends
// (programmatic dependent launch); kv_begin() is the first thing such a kernel does that touches memory.
template <class... P, class... A>
inline int kv_launch_clusters(void (*kernel)(P...), dim3 grid, int cluster, int threads, size_t smem, cudaStream_t st, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  if (cudaLaunchKernelEx(&cfg, kernel, args...) != cudaSuccess) return QALORA_ERR_CUDA;
  count_launch();
  return QALORA_OK;
}
template <class... P, class... A>
inline int kv_launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, A... args) {
  return kv_launch_clusters(kernel, grid, 1, threads, smem, st, args...);
}
// Waits for the kernel before, and only then lets the one after be set up: it can never run beside one before this.
__device__ __forceinline__ void kv_begin() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
}

// Rows and tokens of sequence b; n == 0 where the entries break the call's bounds.
struct KvSeq {
  int row0, n;     // its rows are row0 .. row0 + n - 1
  int len;         // tokens to visit, 0 .. max_len
  int first;       // position of row row0 (negative: that row is not there)
};
__device__ __forceinline__ KvSeq kv_seq(const KvBatch& kb, int b) {
  KvSeq s;
  const int r0 = kb.starts[b], r1 = kb.starts[b + 1], len = kb.lens[b];
  s.row0 = r0;
  s.n = (r0 >= 0 && r1 >= r0 && r1 <= kb.m && r1 - r0 <= kb.n_hi && r1 - r0 >= kb.n_lo) ? r1 - r0 : 0;
  s.len = len < 0 ? 0 : (len > kb.max_len ? kb.max_len : len);
  s.first = s.len - s.n;
  return s;
}

// Block that holds token t (0 <= t < max_blocks * block) of sequence b, or -1 when the entry is outside the pool.
__device__ __forceinline__ int kv_block(const int32_t* table, int max_blocks, int num_blocks, int b, int j) {
  const int id = table[(size_t)b * max_blocks + j];
  return (id >= 0 && id < num_blocks) ? id : -1;
}

// Code of v under scale s > 0: clamp(rint(v / s), -127, 127) with the IEEE quotient.
__device__ __forceinline__ float kv_code_div(float v, float s) {
  const float t = __fdiv_rn(v, s);
  return fminf(fmaxf(rintf(t), -127.f), 127.f);
}
__device__ __forceinline__ bool kv_fast_scale(float s) { return s > 1e-30f && s < 1e30f; }

__device__ __forceinline__ uint32_t kv_pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {   // the low byte of each
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}

// Four codes as floats: 2^23 + (c + 128) by byte permutation (its last place is 1), minus 2^23 + 128.  (The
// conversion unit runs at a quarter of the rate.)
__device__ __forceinline__ void kv_floats4(uint32_t w, float2& a, float2& b) {
  const uint32_t u = w ^ 0x80808080u;
  const float2 k = make_float2(8388736.f, 8388736.f);
  a = ptx::fsub2(make_float2(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7540)), __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7541))), k);
  b = ptx::fsub2(make_float2(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7542)), __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7543))), k);
}

// Four codes by division, for scales whose inverse is not an ordinary number and elements that may not be finite.  A
// call, not inlined: unrolled into every pass it made the kernels wait for instructions.
static __device__ __noinline__ uint32_t kv_codes4_any(float v0, float v1, float v2, float v3, float s) {
  const float v[4] = {v0, v1, v2, v3};
  uint32_t c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) c[i] = (s > 0.f && v[i] == v[i]) ? (uint32_t)(int)kv_code_div(v[i], s) : 0u;
  return kv_pack4(c[0], c[1], c[2], c[3]);
}
// Eight elements under scale s, 1 / s correctly rounded in inv, to their codes.  The quotient is q = x * inv with two
// corrections q += (x - q * s) * inv: the first brings q within a unit of its last place, and from there one
// correction yields the correctly rounded quotient (P. Markstein, "Computation of elementary functions on the IBM
// RISC System/6000 processor", 1990: the residual is exact, and inv is the correctly rounded reciprocal).  A check
// whether x * inv lies near a tie, with a division where it does, took a third of the kernels' instructions: elements of
// 8 significant bits over a scale of their own meet exact ties every few hundred elements.  The low byte of
// q + 1.5 * 2^23 is the rounded quotient in two's complement: no float-to-integer conversion.
__device__ __forceinline__ uint2 kv_codes8(const float2 (&x)[4], float s, float inv) {
  const float2 ii = make_float2(inv, inv), ms = make_float2(-s, -s), up = make_float2(12582912.f, 12582912.f);
  float2 u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float2 q = ptx::fmul2(x[i], ii);
    q = ptx::ffma2(ptx::ffma2(q, ms, x[i]), ii, q);
    q = ptx::ffma2(ptx::ffma2(q, ms, x[i]), ii, q);
    u[i] = ptx::fadd2(q, up);
  }
  return make_uint2(kv_pack4(__float_as_uint(u[0].x), __float_as_uint(u[0].y), __float_as_uint(u[1].x), __float_as_uint(u[1].y)),
                    kv_pack4(__float_as_uint(u[2].x), __float_as_uint(u[2].y), __float_as_uint(u[3].x), __float_as_uint(u[3].y)));
}

// Packed 16-bit maxima and minima in one instruction each.
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.u16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t max_s16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.s16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t min_s16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("min.s16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// Bytes 2 p and 2 p + 1 of w as signed 16-bit numbers (prmt's selector bit 3 repeats a byte's sign).
template <int P>
__device__ __forceinline__ uint32_t signed_pair(uint32_t w) {
  uint32_t d;
  asm("prmt.b32 %0, %1, 0, %2;" : "=r"(d) : "r"(w), "n"(P == 0 ? 0x9180 : 0xb3a2));
  return d;
}
#endif

}  // namespace qalora
