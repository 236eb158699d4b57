// The gradient of the merge coefficients.  For the additive operator M_A = M_0 + sum_i alpha_i A_i Delta_i
// (Prop. 2; one alpha per expert, or one per expert and tensor) and a loss L of the merged weights,
//
//   dL / dalpha_{i,t} = sum over the blocks b of tensor t with A_{i,b} = 1 of
//                       sum_j G[j] * (M_i[j] - M_0[j]),      G = dL / dM_A.
//
// Bound by memory: G and the base are read once for all experts of a block, an expert's block only where
// the mask has it, and blocks that no expert is read from not at all.  An item is one or four rounds of a
// CTA's 16-byte vectors of one block; a thread keeps its vectors of G and of the base while the experts of the mask stream
// past, the next expert's loads in flight.  Differences and products are fp32 sums of 64 elements
// per thread, then trees over lanes and warps; the items' sums are added in fp64 in a fixed order.
#include <algorithm>

#include "layer.cuh"

namespace mp {

namespace {

constexpr int kThreads = 256;
constexpr int kVecs = 2;                              // vectors a thread keeps at a time
constexpr uint32_t kRounds = 4;                       // rounds of those in an item, where items are plenty

// element e of a 16-byte vector as fp32
template <typename T>
__device__ __forceinline__ float elem_of(const uint4& q, int e);
template <>
__device__ __forceinline__ float elem_of<float>(const uint4& q, int e) {
  return __uint_as_float(e == 0 ? q.x : e == 1 ? q.y : e == 2 ? q.z : q.w);
}
template <>
__device__ __forceinline__ float elem_of<__nv_bfloat16>(const uint4& q, int e) {
  const uint32_t w = e < 2 ? q.x : e < 4 ? q.y : e < 6 ? q.z : q.w;
  return __uint_as_float(e & 1 ? w & 0xFFFF0000u : w << 16);
}

// vector v of the n elements at p; past the end zeros, in a last partial vector element by element
template <typename T>
__device__ __forceinline__ uint4 load_vec(const T* p, uint32_t v, uint32_t n) {
  constexpr int V = Elem<T>::kVec;
  const uint32_t at = v * V;
  if (at + V <= n) return __ldcs(reinterpret_cast<const uint4*>(p + at));
  uint32_t w[4] = {};
#pragma unroll
  for (int e = 0; e < V; ++e)
    if (at + e < n) {
      if constexpr (sizeof(T) == 2)
        w[e / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[at + e] << (16 * (e % 2));
      else
        w[e] = reinterpret_cast<const uint32_t*>(p)[at + e];
    }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 4) coef_kernel(const CoefLaunch p, float* part, uint32_t per_block, uint32_t item) {
  kernel_begin();
  constexpr int V = Elem<T>::kVec;
  __shared__ float sum[kThreads / 32][kMaxK];
  const uint64_t n_items = gridDim.x, b = blockIdx.x / per_block;
  const uint32_t at = blockIdx.x % per_block * item;  // item: elements of one
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  const uint32_t len = p.blk_len[b];
  uint32_t mask = at < len ? p.mask[b] : 0u;
  const uint64_t off = p.blk_off[b] + at;
  const uint32_t n = at < len ? min(len - at, item) : 0u;
  if (kChecked && mask != 0u && !chunk_in_bounds(b, 0, p.n_blocks, p.blk_off[b], len, off, n, mask, p.K, sizeof(T), 0, p.ext)) {
    if (threadIdx.x == 0) atomicOr_system(p.err, kErrBounds);
    mask = 0u;
  }
  if (lane < p.K) sum[warp][lane] = 0.0f;
  __syncwarp();
  if (mask) {
    const T* base = static_cast<const T*>(p.base) + off;
    const T* grad = static_cast<const T*>(p.grad) + off;
#pragma unroll 1
    for (uint32_t r0 = 0; r0 * V < n; r0 += kThreads * kVecs) {  // the same rounds for every thread
      const uint32_t v0 = r0 + threadIdx.x;
      uint4 g[kVecs], m[kVecs], x[kVecs];
      uint32_t left = mask;
      uint32_t i = __ffs(left) - 1;
      left &= left - 1;
#pragma unroll
      for (int k = 0; k < kVecs; ++k) {
        g[k] = load_vec(grad, v0 + k * kThreads, n);
        m[k] = load_vec(base, v0 + k * kThreads, n);
      }
#pragma unroll
      for (int k = 0; k < kVecs; ++k) x[k] = load_vec(static_cast<const T*>(p.experts.p[i]) + off, v0 + k * kThreads, n);
      while (true) {
        uint4 y[kVecs];
        uint32_t next = 0;
        if (left) {
          next = __ffs(left) - 1;
#pragma unroll
          for (int k = 0; k < kVecs; ++k)
            y[k] = load_vec(static_cast<const T*>(p.experts.p[next]) + off, v0 + k * kThreads, n);
        }
        float a[kVecs] = {};
#pragma unroll
        for (int k = 0; k < kVecs; ++k)
#pragma unroll
          for (int e = 0; e < V; ++e)
            a[k] = fmaf(elem_of<T>(g[k], e), elem_of<T>(x[k], e) - elem_of<T>(m[k], e), a[k]);
        float s = a[0] + a[1];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
        if (lane == 0) sum[warp][i] += s;
        if (!left) break;
        left &= left - 1;
        i = next;
#pragma unroll
        for (int k = 0; k < kVecs; ++k) x[k] = y[k];
      }
    }
  }
  __syncthreads();
  if (threadIdx.x < p.K) {
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) s += sum[w][threadIdx.x];
    part[threadIdx.x * n_items + blockIdx.x] = s;
  }
}

// out[i][t] = the sum of tensor t's items of expert i, in fp64: every thread a strided run, then a tree over lanes and
// one over warps
__global__ void __launch_bounds__(kThreads) coef_sum_kernel(const float* part, uint64_t n_items, uint32_t per_block,
                                                            const uint32_t* t_blk0, uint32_t n_tensors, float* out) {
  kernel_begin();
  __shared__ double red[kThreads / 32];
  const uint32_t t = blockIdx.x, i = blockIdx.y, lane = threadIdx.x & 31u;
  const float* src = part + (uint64_t)i * n_items;
  double s = 0.0;
  for (uint64_t q = (uint64_t)t_blk0[t] * per_block + threadIdx.x; q < (uint64_t)t_blk0[t + 1] * per_block; q += kThreads)
    s += (double)src[q];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  if (lane == 0) red[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x < 32) {
    s = lane < kThreads / 32 ? red[lane] : 0.0;
#pragma unroll
    for (int o = kThreads / 64; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    if (lane == 0) out[(uint64_t)i * n_tensors + t] = (float)s;
  }
}

// Elements of an item: four rounds of a CTA; one where four-round items would not give each of 1,024 CTAs (four to an SM and
// a second lot) one of its own: a CTA's experts stream past one after the other, so that 16 of them over 1.8M elements in
// blocks of 65,536 took 51 us with four rounds, 26 with one.
uint32_t item_elems(const CoefLaunch& p) {
  const uint32_t round = kThreads * kVecs * (p.dtype == MP_BF16 ? 8u : 4u), item = round * kRounds;
  return p.n_blocks * ((p.block_elems + item - 1) / item) < 1024 ? round : item;
}
uint32_t items_per_block(const CoefLaunch& p) { return (p.block_elems + item_elems(p) - 1) / item_elems(p); }

}  // namespace

size_t coef_scratch(const CoefLaunch& p) { return (size_t)p.n_blocks * items_per_block(p) * p.K * sizeof(float); }

cudaError_t launch_coef(const CoefLaunch& p, float* part, cudaStream_t st) {
  const uint32_t per_block = items_per_block(p);
  const uint64_t items = p.n_blocks * per_block;
  if (items > 0x7FFFFFFFull) return cudaErrorInvalidValue;
  const dim3 grid((unsigned)items);
  cudaError_t e = p.dtype == MP_BF16
                      ? launch_kernel(true, coef_kernel<__nv_bfloat16>, grid, kThreads, 0, st, p, part, per_block, item_elems(p))
                      : launch_kernel(true, coef_kernel<float>, grid, kThreads, 0, st, p, part, per_block, item_elems(p));
  if (e != cudaSuccess) return e;
  return launch_kernel(true, coef_sum_kernel, dim3(p.n_tensors, p.K), kThreads, 0, st, (const float*)part, items,
                       per_block, p.t_blk0, p.n_tensors, p.out);
}

}  // namespace mp
