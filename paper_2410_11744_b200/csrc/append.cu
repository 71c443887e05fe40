// New tokens into the paged KV cache, rotated by their positions on the way (rotary position embedding), and
// their queries rotated with them.  Token j of request r has position context[r] + j, or context[r] + depth[j]
// when it is a node of a draft tree, and with half-split pairs (i, i + rot / 2), or neighbouring ones (2 i, 2 i + 1),
//   (a, b) -> (a cos - b sin, b cos + a sin),   cos / sin = columns i and rot / 2 + i of the position's table row,
// in fp32, rounded once to bf16 (half a step: 2^-8 relative).  V, and columns behind `rot`,
// are copied bit for bit.
//
// Bound by bytes: every value is read once and written once.  The unit of work is 32 bytes of one head, the two
// 16-byte chunks that hold whole pairs (chunk u and chunk u + rot / 16, or two neighbours), so a pair never leaves its
// thread and Q may be rotated in place.  A head has D / 16 units, a power of two, so a thread meets the same unit of
// every head that it works on: its 16 cosines and sines stay in registers.  A thread asks for its chunks before it knows
// where they go; the chain in front of the writes (request of the token, context, page) runs under those loads.
// A token is worked on by a group of 32 to 256 threads, as many as leave each about kBatch units.  64 registers, four CTAs per
// SM: 14891 tokens of 80 heads of 128 (618 MB) 100.4 us call after call, 6.2 TB/s, against 102.6 with three CTAs of 80 registers.
#include "common.cuh"

namespace dyspec {

namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 3;      // units in flight per thread: 64 + 8 + 8 heads of 128 are 640 units

struct AppendParams {
  const uint4 *q, *k, *v;                 // rows of 16-byte chunks
  uint4 *q_out, *k_cache, *v_cache;
  int64_t q_stride, k_stride, v_stride, q_out_stride;   // chunks between tokens
  const int32_t *offsets, *context, *depths;
  const int64_t* tree_row_offset;
  const int32_t* page_table;
  const float* rope;
  int32_t* status;
  int64_t cache_rows;
  int n_req, n_tokens, pages_per_req, page_shift, n_positions, rot, interleaved, hq, hkv;
  int log2_group;                         // threads per token
};

// The request that owns `token`: how many requests end at or before it (n_req: none, the token is padding).  Whole
// warp; two rounds of 32 probes settle 1024 requests.
__device__ __forceinline__ int find_request(const int32_t* offsets, int n_req, int token, int lane) {
  int lo = 0, hi = n_req;                 // the count lies in [lo, hi]
  while (hi > lo) {
    const int step = (hi - lo + 31) >> 5;
    const int at = lo + (lane + 1) * step;                        // the lane's probe: does request at - 1 end at or before it?
    const unsigned ends = __ballot_sync(0xffffffffu, at <= hi && __ldg(offsets + min(at, hi)) <= token);
    const int done = __popc(ends);
    if (step == 1) return lo + done;
    lo += done * step;
    hi = min(hi, lo + step - 1);          // (request lo + step - 1 does not end before the token)
  }
  return lo;
}

__device__ __forceinline__ float2 bf16x2_to_f32(uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }

template <int D>
__global__ void __launch_bounds__(kThreads, 4) append_kv_kernel(const AppendParams p) {
  constexpr int P = D / 16;               // units per head
  constexpr int C = D / 8;                // 16-byte chunks per head
  const int group = 1 << p.log2_group, in_group = int(threadIdx.x) & (group - 1);
  const int64_t token64 = int64_t(blockIdx.x) * (kThreads >> p.log2_group) + (threadIdx.x >> p.log2_group);
  if (token64 >= p.n_tokens) return;      // (a group is whole warps)
  const int token = int(token64);
  const int lane = threadIdx.x & 31;
  const int pair_units = p.rot >> 4;
  const int u = threadIdx.x % P;          // the same unit of every head (kThreads is a multiple of P)
  const bool turned = u < pair_units;
  const int c0 = turned && !p.interleaved ? u : 2 * u;
  const int c1 = turned && !p.interleaved ? u + pair_units : 2 * u + 1;
  const int n_heads = p.hq + 2 * p.hkv;
  const int head0 = blockIdx.y * (group / P) + in_group / P, head_step = gridDim.y * (group / P);

  uint4 a[kBatch], b[kBatch];
  auto fetch = [&](int i, int head) {
    if (head >= n_heads) return;
    const uint4* row = head < p.hq ? p.q + int64_t(token) * p.q_stride + int64_t(head) * C
                       : head < p.hq + p.hkv ? p.k + int64_t(token) * p.k_stride + int64_t(head - p.hq) * C
                                             : p.v + int64_t(token) * p.v_stride + int64_t(head - p.hq - p.hkv) * C;
    a[i] = row[c0];
    b[i] = row[c1];
  };
#pragma unroll
  for (int i = 0; i < kBatch; ++i) fetch(i, head0 + i * head_step);

  const int r = find_request(p.offsets, p.n_req, token, lane);
  if (r >= p.n_req) return;               // behind the last request
  const int j = token - __ldg(p.offsets + r);
  const int64_t context = __ldg(p.context + r);
  const int64_t position = context + (p.depths ? __ldg(p.depths + token) : j);
  const int64_t tree0 = p.tree_row_offset ? __ldg(p.tree_row_offset + r) : 0;
  int64_t row = -1;
  if (p.tree_row_offset) {
    row = tree0 < 0 || tree0 >= p.cache_rows ? -1 : tree0 + j;    // (no sum that could pass 63 bits)
  } else if (context >= 0) {
    const int64_t t = context + j, pi = t >> p.page_shift;
    const int page = pi < p.pages_per_req ? __ldg(p.page_table + int64_t(r) * p.pages_per_req + pi) : -1;
    if (page >= 0) row = (int64_t(page) << p.page_shift) + (t & ((int64_t(1) << p.page_shift) - 1));
  }
  // a token without a row or a rotation is left out whole (the checks hold for every thread of the token alike)
  if (j < 0 || row < 0 || row >= p.cache_rows || (p.rot > 0 && (position < 0 || position >= p.n_positions))) {
    if (p.status && in_group == 0 && blockIdx.y == 0) atomicCAS(p.status, 0, DYSPEC_ERR_INVALID_ARG);
    return;
  }
  float cs[8], sn[8];
  if (turned) {
    const float4* cos_at = reinterpret_cast<const float4*>(p.rope + position * p.rot + 8 * u);
    const float4* sin_at = reinterpret_cast<const float4*>(p.rope + position * p.rot + p.rot / 2 + 8 * u);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float4 x = __ldg(cos_at + h), y = __ldg(sin_at + h);
      cs[4 * h] = x.x; cs[4 * h + 1] = x.y; cs[4 * h + 2] = x.z; cs[4 * h + 3] = x.w;
      sn[4 * h] = y.x; sn[4 * h + 1] = y.y; sn[4 * h + 2] = y.z; sn[4 * h + 3] = y.w;
    }
  }

  for (int first = head0; first < n_heads; first += kBatch * head_step) {
    if (first != head0) {
#pragma unroll
      for (int i = 0; i < kBatch; ++i) fetch(i, first + i * head_step);
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int head = first + i * head_step;
      if (head >= n_heads) break;
      uint32_t* x = reinterpret_cast<uint32_t*>(&a[i]);
      uint32_t* y = reinterpret_cast<uint32_t*>(&b[i]);
      if (turned && head < p.hq + p.hkv) {
        if (p.interleaved) {              // word w of the 8 words holds pair w of the unit
#pragma unroll
          for (int w = 0; w < 8; ++w) {
            uint32_t& word = w < 4 ? x[w] : y[w - 4];
            const float2 z = bf16x2_to_f32(word);
            word = pack_bf16x2(z.x * cs[w] - z.y * sn[w], z.y * cs[w] + z.x * sn[w]);
          }
        } else {                          // value e of chunk c0 pairs with value e of chunk c1
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const float2 z0 = bf16x2_to_f32(x[w]), z1 = bf16x2_to_f32(y[w]);
            x[w] = pack_bf16x2(z0.x * cs[2 * w] - z1.x * sn[2 * w], z0.y * cs[2 * w + 1] - z1.y * sn[2 * w + 1]);
            y[w] = pack_bf16x2(z1.x * cs[2 * w] + z0.x * sn[2 * w], z1.y * cs[2 * w + 1] + z0.y * sn[2 * w + 1]);
          }
        }
      }
      uint4* dst = head < p.hq ? p.q_out + int64_t(token) * p.q_out_stride + int64_t(head) * C
                   : head < p.hq + p.hkv ? p.k_cache + (row * p.hkv + (head - p.hq)) * C
                                         : p.v_cache + (row * p.hkv + (head - p.hq - p.hkv)) * C;
      dst[c0] = a[i];
      dst[c1] = b[i];
    }
  }
}

}  // namespace

cudaError_t launch_append_kv_paged(const dyspec_append_t& a, int page_shift, cudaStream_t stream) {
  AppendParams p{};
  p.q = static_cast<const uint4*>(a.q); p.k = static_cast<const uint4*>(a.k_new); p.v = static_cast<const uint4*>(a.v_new);
  p.q_out = static_cast<uint4*>(a.q_out); p.k_cache = static_cast<uint4*>(a.k_cache); p.v_cache = static_cast<uint4*>(a.v_cache);
  p.q_stride = a.q_stride / 8; p.k_stride = a.k_stride / 8; p.v_stride = a.v_stride / 8; p.q_out_stride = a.q_out_stride / 8;
  p.offsets = a.token_offsets; p.context = a.context_len; p.depths = a.depths; p.tree_row_offset = a.tree_row_offset;
  p.page_table = a.page_table; p.rope = a.rope_table; p.status = a.status; p.cache_rows = a.kv_total_rows;
  p.n_req = a.n_req; p.n_tokens = a.n_tokens; p.pages_per_req = a.pages_per_req; p.page_shift = page_shift;
  p.n_positions = a.n_positions; p.rot = a.rotary_dim; p.interleaved = a.interleaved != 0; p.hq = a.n_q_heads; p.hkv = a.n_kv_heads;
  // Few tokens (less than a wave of CTAs): 256 threads each and more than one CTA, one unit a thread.  Else the smallest group
  // that needs one batch.
  const int units = (a.n_q_heads + 2 * a.n_kv_heads) * (a.head_dim / 16);
  const bool few = a.n_tokens <= kDefaultSMs;
  p.log2_group = 5;
  while (p.log2_group < 8 && (few || units > (kBatch << p.log2_group))) ++p.log2_group;
  const int per_cta = kThreads >> p.log2_group;
  const dim3 grid(unsigned((int64_t(a.n_tokens) + per_cta - 1) / per_cta), unsigned(few ? (units + kThreads - 1) / kThreads : 1));
  if (a.head_dim == 128) append_kv_kernel<128><<<grid, kThreads, 0, stream>>>(p);
  else append_kv_kernel<64><<<grid, kThreads, 0, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace dyspec
