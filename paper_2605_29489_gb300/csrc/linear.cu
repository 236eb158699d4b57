// Products of a linear layer and its gradients, with what follows them in the epilogue:
//
//   forward       z = x w^T + b,  y = act(z) * m + r,  pre = z
//   backward      dz = dy * m * act'(z),  dm = dy * act(z),  db = column sums of dz   (dz_kernel)
//                 dx = dz w + add,  dw = dz^T x + add
//
// bf16 operands go to the tensor cores (tcgen05), accumulated in fp32 in tensor memory: TMA brings the
// tiles, whichever way the operand is stored (the three products need x and w both along and across
// their rows), one thread issues the products, four warps take the sums through the epilogue.
// What lies past an edge is read as zeros and not written.  Two kernels:
//
//   gemm_kernel   tiles of 256 x 256 by pairs of CTAs, persistent: while the epilogue of one tile runs, the
//                 products of the next fill the other half of tensor memory.  Bound by the tensor cores.
//   split_kernel  tiles of 128 features x up to 128 rows, the inner dimension split over the CTAs of a
//                 cluster, whose sums are added over distributed shared memory in the order of the CTAs (no
//                 scratch, no atomics, one launch).  For few rows, where the weights' bytes are the work
//                 and all SMs have to stream them, and for products too small to fill the GPU with tiles of 256.
//
// fp32 operands are multiplied in fp32 (fma) by a tiled kernel of the ordinary cores: a checkpoint kept
// in fp32 is kept so for its accuracy, and splitting into tensor-core types does not hold it over long sums.
#include <dlfcn.h>

#include <algorithm>

#include "layer.cuh"
#include "umma.cuh"

namespace mp {

namespace {

// ---- the epilogue -------------------------------------------------------------------------------

// act(z).  FAST: bf16 results, where the fast exponential's 2 ulp do not show.
template <bool FAST>
__device__ __forceinline__ float sigmoid(float z) {
  return FAST ? __fdividef(1.0f, 1.0f + __expf(-z)) : 1.0f / (1.0f + expf(-z));
}
constexpr float kRootHalf = 0.70710678118654752f, kRoot2Pi = 0.79788456080286536f, kInvRoot2Pi = 0.39894228040143268f;
constexpr float kTanhCubic = 0.044715f;

template <int ACT, bool FAST>
__device__ __forceinline__ float act_of(float z) {
  if constexpr (ACT == MP_ACT_RELU) return z > 0.0f ? z : (z == z ? 0.0f : z);
  if constexpr (ACT == MP_ACT_SILU) return z * sigmoid<FAST>(z);
  if constexpr (ACT == MP_ACT_GELU) return 0.5f * z * (1.0f + erff(z * kRootHalf));
  if constexpr (ACT == MP_ACT_GELU_TANH) return 0.5f * z * (1.0f + tanhf(kRoot2Pi * fmaf(kTanhCubic * z * z, z, z)));
  return z;
}
// act(z) in a and act'(z) in g: they share what costs most
template <int ACT, bool FAST>
__device__ __forceinline__ void act_both(float z, float& a, float& g) {
  a = z;
  g = 1.0f;
  if constexpr (ACT == MP_ACT_RELU) {
    a = act_of<ACT, FAST>(z);
    g = z > 0.0f ? 1.0f : 0.0f;
  }
  if constexpr (ACT == MP_ACT_SILU) {
    const float s = sigmoid<FAST>(z);
    a = z * s;
    g = s * fmaf(z, 1.0f - s, 1.0f);
  }
  if constexpr (ACT == MP_ACT_GELU) {
    const float s = 0.5f * (1.0f + erff(z * kRootHalf));
    a = z * s;
    g = fmaf(z, kInvRoot2Pi * expf(-0.5f * z * z), s);
  }
  if constexpr (ACT == MP_ACT_GELU_TANH) {
    const float t = tanhf(kRoot2Pi * fmaf(kTanhCubic * z * z, z, z)), s = 0.5f * (1.0f + t);
    const float c = fminf(fmaxf(z, -16.0f), 16.0f);  // t is +-1 from there on: no 0 * infinity
    a = z * s;
    g = fmaf(0.5f * c * (1.0f - t * t), kRoot2Pi * fmaf(3.0f * kTanhCubic * c, c, 1.0f), s);
  }
}

template <bool FAST, int N>
__device__ __forceinline__ void act_all(int act, float* v) {
  switch (act) {
    case MP_ACT_RELU:
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = act_of<MP_ACT_RELU, FAST>(v[j]);
      break;
    case MP_ACT_SILU:
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = act_of<MP_ACT_SILU, FAST>(v[j]);
      break;
    case MP_ACT_GELU:
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = act_of<MP_ACT_GELU, FAST>(v[j]);
      break;
    case MP_ACT_GELU_TANH:
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = act_of<MP_ACT_GELU_TANH, FAST>(v[j]);
      break;
    default: break;
  }
}

// the epilogue as the kernels take it: strides in elements, vec: every row of every matrix in whole vectors of 16 bytes
template <typename T>
struct Epi {
  uint32_t rows, cols;
  int act;
  const T *bias, *mul, *res;
  uint64_t ldmul, ldres, ldy, ldpre;
  T *y, *pre;
  uint32_t vec, quad;  // quad: in whole vectors of four elements
};

template <typename T>
__device__ __forceinline__ float epi_bias(const Epi<T>& e, uint32_t c) {
  return e.bias ? Elem<T>::load(e.bias[c]) : 0.0f;
}

// one element: z = acc + bias
template <typename T>
__device__ __forceinline__ void epi_one(const Epi<T>& e, uint32_t r, uint32_t c, float z) {
  constexpr bool FAST = sizeof(T) == 2;
  if (e.pre) e.pre[r * e.ldpre + c] = Elem<T>::store(z);
  act_all<FAST, 1>(e.act, &z);
  if (e.mul) z *= Elem<T>::load(e.mul[r * e.ldmul + c]);
  if (e.res) z += Elem<T>::load(e.res[r * e.ldres + c]);
  e.y[r * e.ldy + c] = Elem<T>::store(z);
}

// four consecutive columns of a row, of which those below e.cols exist; quad: they are whole vectors of every matrix
template <typename T>
__device__ __forceinline__ void epi_quad(const Epi<T>& e, uint32_t r, uint32_t c, float* v, bool quad) {
  constexpr bool FAST = sizeof(T) == 2;
  if (!quad) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (c + k < e.cols) epi_one(e, r, c + k, v[k]);
    return;
  }
  Pack<T, 4> m, s;
  if (e.mul) m = *reinterpret_cast<const Pack<T, 4>*>(e.mul + r * e.ldmul + c);
  if (e.res) s = *reinterpret_cast<const Pack<T, 4>*>(e.res + r * e.ldres + c);
  if (e.pre) *reinterpret_cast<Pack<T, 4>*>(e.pre + r * e.ldpre + c) = pack<T, 4>(v);
  act_all<FAST, 4>(e.act, v);
  float u[4];
  if (e.mul) {
    unpack(m, u);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] *= u[k];
  }
  if (e.res) {
    unpack(s, u);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] += u[k];
  }
  *reinterpret_cast<Pack<T, 4>*>(e.y + r * e.ldy + c) = pack<T, 4>(v);
}

// N consecutive columns of a row, from c on (a multiple of N), of which those below e.cols exist
template <typename T, int N>
__device__ __forceinline__ void epi_run(const Epi<T>& e, uint32_t r, uint32_t c, float* v) {
  constexpr int V = Elem<T>::kVec;
  constexpr bool FAST = sizeof(T) == 2;
  if (r >= e.rows || c >= e.cols) return;
  if (!e.vec || c + N > e.cols) {
    for (int j = 0; j < N; ++j)
      if (c + j < e.cols) {
        // v[j] without indexing registers by a variable
        float z = v[0];
#pragma unroll
        for (int k = 1; k < N; ++k) z = k == j ? v[k] : z;
        epi_one(e, r, c + j, z + epi_bias(e, c + j));
      }
    return;
  }
  float u[V];
  if (e.bias) {
#pragma unroll
    for (int j = 0; j < N; j += V) {
      unpack(load_pack<T, V>(e.bias + c + j), u);
#pragma unroll
      for (int k = 0; k < V; ++k) v[j + k] += u[k];
    }
  }
  if (e.pre) {
#pragma unroll
    for (int j = 0; j < N; j += V) store_pack<T, V>(e.pre + r * e.ldpre + c + j, pack<T, V>(v + j));
  }
  act_all<FAST, N>(e.act, v);
  if (e.mul) {
#pragma unroll
    for (int j = 0; j < N; j += V) {
      unpack(load_pack<T, V>(e.mul + r * e.ldmul + c + j), u);
#pragma unroll
      for (int k = 0; k < V; ++k) v[j + k] *= u[k];
    }
  }
  if (e.res) {
#pragma unroll
    for (int j = 0; j < N; j += V) {
      unpack(load_pack<T, V>(e.res + r * e.ldres + c + j), u);
#pragma unroll
      for (int k = 0; k < V; ++k) v[j + k] += u[k];
    }
  }
#pragma unroll
  for (int j = 0; j < N; j += V) store_pack<T, V>(e.y + r * e.ldy + c + j, pack<T, V>(v + j));
}

// ---- tensor-core products -----------------------------------------------------------------------

constexpr int kBK = 64;                 // inner elements of a stage: one 128-byte swizzle span of bf16
constexpr uint32_t kBoxT = 8192;        // bytes of an mn-major box: 64 k x 64 mn
constexpr uint32_t kWarps = 6;
constexpr int kGemmThreads = 32 * kWarps;       // a TMA warp, a warp that issues products, four epilogue warps

using bf16 = __nv_bfloat16;

struct Wait {
  uint32_t* err;   // the host's error word
  uint32_t limit;  // rounds of a wait
  uint32_t stall;  // test hook: the first stage is never filled
};

// loads ROWS rows (m or n, from r0 on) x 64 k (from k0 on) of an operand
template <int CG, int ROWS, bool T>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, int32_t r0, int32_t k0, uint32_t bar) {
  if constexpr (T) {
#pragma unroll
    for (int q = 0; q < ROWS / 64; ++q) tma_load_2d<CG>(dst + q * kBoxT, map, r0 + q * 64, k0, bar);
  } else {
    tma_load_2d<CG>(dst, map, k0, r0, bar);
  }
}

__device__ __forceinline__ void give_up(volatile int* abort, const Wait& w) {
  *abort = 1;
  atomicOr_system(w.err, kErrTimeout);
}

// a warp's bounded wait on an mbarrier that threads of another CTA arrive on
__device__ __forceinline__ bool warp_wait_cluster(uint64_t* bar, uint32_t parity, volatile int* abort, uint32_t limit) {
  uint32_t ok = 0;
  for (uint32_t k = 0; k < limit; ++k) {
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, "
        "p;\n}\n"
        : "=r"(ok)
        : "r"(su32(bar)), "r"(parity)
        : "memory");
    if (ok || ((k & 15u) == 15u && *abort)) break;
  }
  return __all_sync(0xFFFFFFFFu, ok != 0);
}

// Few rows.  out[r, c]: c (features, the lanes of tensor memory) from operand a, r from operand b.  A cluster makes one
// tile of 128 c x BN r; its CTA q has the q-th part of the inner dimension.  Tiles with the same features are neighbours.
template <int BN, bool AT, bool BT>
__global__ void __launch_bounds__(kGemmThreads) split_kernel(const __grid_constant__ CUtensorMap ma,
                                                             const __grid_constant__ CUtensorMap mb, const Epi<bf16> e,
                                                             uint32_t kb_all, uint32_t tiles_r, int stages, const Wait w) {
  constexpr int kMaxStages = 12;
  constexpr uint32_t kA = 128 * 128, kB = BN * 128, kStage = kA + kB;
  constexpr uint32_t kCols = BN < 32 ? 32 : BN;
  extern __shared__ uint8_t raw[];
  __shared__ uint64_t full[kMaxStages], empty[kMaxStages], done;
  __shared__ uint32_t tmem_at;
  __shared__ volatile int abort;
  const uint32_t smem = (su32(raw) + 1023u) & ~1023u;
  const uint32_t warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31u;
  uint32_t split, rank = cluster_rank();
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(split));
  const uint32_t tile = blockIdx.x / split;
  const int32_t r0 = (int32_t)(tile % tiles_r) * BN, c0 = (int32_t)(tile / tiles_r) * 128;
  const uint32_t k0 = (uint32_t)((uint64_t)kb_all * rank / split), k1 = (uint32_t)((uint64_t)kb_all * (rank + 1) / split);
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    mbar_init(&done, 1);
    mbar_fence_init();
    abort = 0;
    prefetch_map(&ma);
    prefetch_map(&mb);
  }
  kernel_wait();  // what the kernel ahead wrote is read from here on
  if (warp == 1) tmem_alloc<1>(&tmem_at, kCols);
  umma_fence_before();
  __syncthreads();
  umma_fence_after();
  kernel_release();
  const uint32_t tmem = tmem_at;
  if (warp == 0) {
    uint32_t it = 0;
    for (uint32_t kb = k0; kb < k1; ++kb, ++it) {
      const uint32_t s = it % stages;
      if (it >= (uint32_t)stages && !warp_wait(&empty[s], ((it / stages) - 1) & 1u, &abort, w.limit)) {
        give_up(&abort, w);
        break;
      }
      if (!(w.stall && it == 0) && elect_one()) {
        mbar_arrive_expect_tx(&full[s], kStage);
        load_tile<1, 128, AT>(smem + s * kStage, &ma, c0, (int32_t)kb * kBK, su32(&full[s]));
        load_tile<1, BN, BT>(smem + s * kStage + kA, &mb, r0, (int32_t)kb * kBK, su32(&full[s]));
      }
      __syncwarp();
    }
    // the stages still on their way, when something gave up: their copies end before the CTA does
    if (abort)
      for (uint32_t q = it > (uint32_t)stages ? it - stages : 0u; q < it; ++q)
        if (!(w.stall && q == 0)) mbar_wait_drain(&full[q % stages], (q / stages) & 1u);
  } else if (warp == 1) {
    uint32_t it = 0;
    for (uint32_t kb = k0; kb < k1; ++kb, ++it) {
      const uint32_t s = it % stages;
      if (!warp_wait(&full[s], (it / stages) & 1u, &abort, w.limit)) {
        give_up(&abort, w);
        break;
      }
      umma_fence_after();
      const uint64_t da = umma_desc<AT>(smem + s * kStage), db = umma_desc<BT>(smem + s * kStage + kA);
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < kBK / 16; ++k)
          umma<1>(tmem, da + k * (umma_k_step<AT>() >> 4), db + k * (umma_k_step<BT>() >> 4), umma_idesc<128, BN, AT, BT>(),
                  it > 0 || k > 0);
        umma_commit<1>(&empty[s]);
      }
      __syncwarp();
    }
    if (elect_one()) umma_commit<1>(&done);
    mbar_wait_drain(&done, 0);
  }
  __syncwarp();
  const bool ok = warp < 2 || warp_wait(&done, 0, &abort, w.limit);
  if (!ok && lane == 0) give_up(&abort, w);
  __syncthreads();  // all copies and products are over, or have been waited for
  umma_fence_after();
  // the CTA's sums to shared memory, [rows][128] (the stages are over), then every warp takes whole rows: a lane's
  // four features from each CTA in turn, several rows' loads in flight
  const uint32_t n_r = min((uint32_t)BN, e.rows - (uint32_t)r0);
  if (warp >= 2) {
    const uint32_t quarter = warp & 3u, row = quarter * 32u + lane;  // this thread's lane of tensor memory
#pragma unroll 1
    for (uint32_t j0 = 0; j0 < n_r; j0 += 16) {
      float v[16];
      tmem_load16(tmem + ((quarter * 32u) << 16) + j0, v);
#pragma unroll
      for (int j = 0; j < 16; ++j)
        asm volatile("st.shared.f32 [%0], %1;" ::"r"(smem + ((j0 + j) * 128u + row) * 4u), "f"(v[j]) : "memory");
    }
  }
  if (split > 1)
    cluster_sync();
  else
    __syncthreads();
  const uint32_t c = (uint32_t)c0 + lane * 4u;
  if (!abort && c < e.cols) {
    float bias[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) bias[k] = c + k < e.cols ? epi_bias(e, c + k) : 0.0f;
    const bool whole = e.quad && c + 4 <= e.cols;
    const uint32_t j1 = n_r * (rank + 1) / split;
    constexpr int kAhead = 4;
    for (uint32_t j = n_r * rank / split + warp; j < j1; j += kWarps * kAhead) {
      float4 z[kAhead];
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        z[a] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        const uint32_t at = smem + (min(j + a * kWarps, j1 - 1) * 128u + lane * 4u) * 4u;
        if (split == 1) {
          z[a] = cluster_load4(at);
        } else {
          for (uint32_t q = 0; q < split; q += 2) {
            const float4 u = cluster_load4(cluster_map(at, q)), v = cluster_load4(cluster_map(at, q + 1));
            z[a].x = (z[a].x + u.x) + v.x;
            z[a].y = (z[a].y + u.y) + v.y;
            z[a].z = (z[a].z + u.z) + v.z;
            z[a].w = (z[a].w + u.w) + v.w;
          }
        }
      }
#pragma unroll
      for (int a = 0; a < kAhead; ++a)
        if (j + a * kWarps < j1) {
          float v[4] = {z[a].x + bias[0], z[a].y + bias[1], z[a].z + bias[2], z[a].w + bias[3]};
          epi_quad(e, (uint32_t)r0 + j + a * kWarps, c, v, whole);
        }
    }
  }
  if (split > 1) cluster_sync();  // nothing of this CTA is read any more
  umma_fence_before();
  __syncthreads();
  if (warp == 1) tmem_free<1>(tmem, kCols);
}

// Many rows: tiles of CG * 128 rows x 256 columns, the next tile's products during this one's epilogue.  a: the rows'
// operand, b: the columns'.
template <int CG, bool AT, bool BT>
__global__ void __launch_bounds__(kGemmThreads) gemm_kernel(const __grid_constant__ CUtensorMap ma,
                                                            const __grid_constant__ CUtensorMap mb, const Epi<bf16> e,
                                                            uint32_t kb_all, uint32_t tiles_r, uint32_t tiles_c,
                                                            const Wait w) {
  constexpr int kBN = 256, kBNs = kBN / CG;  // columns of a tile, and those whose operand this CTA holds
  constexpr uint32_t kA = 128 * 128, kB = kBNs * 128, kStage = kA + kB;
  constexpr int kStages = CG == 2 ? 6 : 4;
  constexpr uint32_t kGroup = 8;  // row tiles that go down the columns together: what they read stays in L2
  extern __shared__ uint8_t raw[];
  __shared__ uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2];
  __shared__ uint32_t tmem_at;
  __shared__ volatile int abort;
  const uint32_t smem = (su32(raw) + 1023u) & ~1023u;
  const uint32_t warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31u;
  const uint32_t rank = CG == 2 ? cluster_rank() : 0u;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&acc_full[s], 1);
      mbar_init(&acc_empty[s], CG * 4);
    }
    mbar_fence_init();
    abort = 0;
    prefetch_map(&ma);
    prefetch_map(&mb);
  }
  kernel_wait();
  if (warp == 1) tmem_alloc<CG>(&tmem_at, 512);
  umma_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync();  // the other CTA's barriers are there
  umma_fence_after();
  kernel_release();
  const uint32_t tmem = tmem_at;
  const uint32_t n_tiles = tiles_r * tiles_c;
  auto place = [&](uint32_t t, int32_t& r0, int32_t& c0) {
    const uint32_t per = kGroup * tiles_c, g = t / per, in = t % per;
    const uint32_t high = min(kGroup, tiles_r - g * kGroup);
    r0 = (int32_t)((g * kGroup + in % high) * (128u * CG));
    c0 = (int32_t)((in / high) * kBN);
  };
  const uint32_t first = blockIdx.x / CG, step = gridDim.x / CG;
  if (warp == 0) {
    uint32_t it = 0;
    bool ok = true;
    for (uint32_t t = first; t < n_tiles && ok; t += step) {
      int32_t r0, c0;
      place(t, r0, c0);
      for (uint32_t kb = 0; kb < kb_all; ++kb, ++it) {
        const uint32_t s = it % kStages;
        if (it >= kStages && !warp_wait(&empty[s], ((it / kStages) - 1) & 1u, &abort, w.limit)) {
          give_up(&abort, w);
          ok = false;
          break;
        }
        if (!(w.stall && it == 0) && elect_one()) {
          uint32_t bar = su32(&full[s]);
          if (rank == 0) mbar_arrive_expect_tx(&full[s], CG * kStage);
          if (CG == 2) bar = cluster_map(bar, 0);
          load_tile<CG, 128, AT>(smem + s * kStage, &ma, r0 + (int32_t)rank * 128, (int32_t)kb * kBK, bar);
          load_tile<CG, kBNs, BT>(smem + s * kStage + kA, &mb, c0 + (int32_t)rank * kBNs, (int32_t)kb * kBK, bar);
        }
        __syncwarp();
      }
    }
    // after a wait that gave up: the copies still on their way end before the CTAs do.  Those of the second CTA
    // count on the first one's barriers, which only that one can wait for: it stays a millisecond, a
    // thousand times what a copy takes
    if (abort && rank != 0)
      for (int q = 0; q < 1000; ++q) __nanosleep(1000);
    if (abort && rank == 0)
      for (uint32_t q = it > kStages ? it - kStages : 0u; q < it; ++q)
        if (!(w.stall && q == 0)) mbar_wait_drain(&full[q % kStages], (q / kStages) & 1u);
  } else if (warp == 1 && rank == 0) {
    uint32_t it = 0, n = 0;
    bool ok = true;
    for (uint32_t t = first; t < n_tiles && ok; t += step, ++n) {
      const uint32_t half = n & 1u;
      if (n >= 2 && !warp_wait_cluster(&acc_empty[half], ((n >> 1) - 1) & 1u, &abort, w.limit)) {
        give_up(&abort, w);
        break;
      }
      umma_fence_after();
      for (uint32_t kb = 0; kb < kb_all; ++kb, ++it) {
        const uint32_t s = it % kStages;
        if (!warp_wait(&full[s], (it / kStages) & 1u, &abort, w.limit)) {
          give_up(&abort, w);
          ok = false;
          break;
        }
        umma_fence_after();
        const uint64_t da = umma_desc<AT>(smem + s * kStage), db = umma_desc<BT>(smem + s * kStage + kA);
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < kBK / 16; ++k)
            umma<CG>(tmem + half * kBN, da + k * (umma_k_step<AT>() >> 4), db + k * (umma_k_step<BT>() >> 4),
                     umma_idesc<128 * CG, kBN, AT, BT>(), kb > 0 || k > 0);
          umma_commit<CG>(&empty[s]);
        }
        __syncwarp();
      }
      if (ok && elect_one()) umma_commit<CG>(&acc_full[half]);
    }
    if (!ok) {  // products still running end before their memory goes
      if (elect_one()) umma_commit<CG>(&acc_full[n & 1u]);
      mbar_wait_drain(&acc_full[n & 1u], (n >> 1) & 1u);
    }
  } else if (warp >= 2) {
    const uint32_t quad = warp & 3u, row = quad * 32u + lane;
    uint32_t n = 0;
    for (uint32_t t = first; t < n_tiles; t += step, ++n) {
      const uint32_t half = n & 1u;
      int32_t r0, c0;
      place(t, r0, c0);
      if (!warp_wait(&acc_full[half], (n >> 1) & 1u, &abort, w.limit) || abort) {
        if (lane == 0) give_up(&abort, w);
        break;
      }
      umma_fence_after();
#pragma unroll 1
      for (int j0 = 0; j0 < kBN; j0 += 16) {
        float v[16];
        tmem_load16(tmem + ((quad * 32u) << 16) + half * kBN + j0, v);
        epi_run<bf16, 16>(e, (uint32_t)r0 + rank * 128u + row, (uint32_t)(c0 + j0), v);
      }
      umma_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (CG == 2)
          cluster_arrive(cluster_map(su32(&acc_empty[half]), 0));
        else
          mbar_arrive(&acc_empty[half]);
      }
    }
  }
  __syncwarp();
  umma_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync();
  umma_fence_after();
  if (warp == 1) tmem_free<CG>(tmem, 512);
}

// ---- fp32 products --------------------------------------------------------------------------------

// out[r, c] = sum over k of a(r, k) b(c, k), element (r, k) at a + r * ar + k * ak: tiles of 64 R x 64 R, BK k at a time,
// 4 R x 4 R sums a thread.  The next step's elements are on their way while this one's are multiplied.  With R = 1 the
// inner dimension may be split over a cluster, whose sums are added over distributed shared memory in the CTAs'
// order: a product of 512 x 512 x 512 is a chain of steps of about 1 us on 64 CTAs, a quarter of it on 256.
template <int R, int BK>
__global__ void __launch_bounds__(256, R == 1 ? 2 : 1) gemm_f32_kernel(const float* a, uint64_t ar, uint64_t ak, const float* b, uint64_t br,
                                                       uint64_t bk, uint32_t inner, uint32_t k_each, const Epi<float> e) {
  kernel_begin();
  constexpr uint32_t kTile = 64 * R, kPitch = kTile + 4;
  constexpr int kLoads = kTile * BK / 256;
  __shared__ alignas(16) float stage[2][2][BK][kPitch];  // [turn][operand]
  const uint32_t rank = R == 1 ? cluster_rank() : 0u;
  uint32_t split = 1;
  if (R == 1) asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(split));
  const uint32_t tiles_c = (e.cols + kTile - 1) / kTile, tile = blockIdx.x / split;
  const uint32_t r0 = tile / tiles_c * kTile, c0 = tile % tiles_c * kTile;
  const uint32_t first = rank * k_each, last = min(inner, first + k_each);
  const uint32_t t = threadIdx.x, tr = t / 16u, tc = t % 16u;
  // element q of this thread's share of a tile: along k first where k is contiguous, else along the rows
  auto spot = [&](uint64_t sk, int q, uint32_t& row, uint32_t& k) {
    if (sk == 1) {
      k = t % BK;
      row = t / BK + (256u / BK) * q;
    } else {
      row = t % kTile;
      k = t / kTile + (256u / kTile) * q;
    }
  };
  float ra[kLoads], rb[kLoads];
  auto fetch = [&](uint32_t k0) {
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
      uint32_t row, k;
      spot(ak, q, row, k);
      ra[q] = r0 + row < e.rows && k0 + k < last ? a[(r0 + row) * ar + (k0 + k) * ak] : 0.0f;
      spot(bk, q, row, k);
      rb[q] = c0 + row < e.cols && k0 + k < last ? b[(c0 + row) * br + (k0 + k) * bk] : 0.0f;
    }
  };
  auto put = [&](int s) {
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
      uint32_t row, k;
      spot(ak, q, row, k);
      stage[s][0][k][row] = ra[q];
      spot(bk, q, row, k);
      stage[s][1][k][row] = rb[q];
    }
  };
  float acc[4 * R][4 * R] = {};
  fetch(first);
  put(0);
  __syncthreads();
  int s = 0;
  for (uint32_t k0 = first; k0 < last; k0 += BK, s ^= 1) {
    const bool more = k0 + BK < last;
    if (more) fetch(k0 + BK);
#pragma unroll
    for (int k = 0; k < BK; ++k) {
      float x[4 * R], y[4 * R];
#pragma unroll
      for (int h = 0; h < R; ++h) {
        *reinterpret_cast<float4*>(x + 4 * h) = *reinterpret_cast<const float4*>(&stage[s][0][k][h * 64 + tr * 4u]);
        *reinterpret_cast<float4*>(y + 4 * h) = *reinterpret_cast<const float4*>(&stage[s][1][k][h * 64 + tc * 4u]);
      }
#pragma unroll
      for (int i = 0; i < 4 * R; ++i)
#pragma unroll
        for (int j = 0; j < 4 * R; ++j) acc[i][j] = fmaf(x[i], y[j], acc[i][j]);
    }
    if (more) put(s ^ 1);
    __syncthreads();
  }
  if constexpr (R == 1) {
    if (split > 1) {
      float* sum = &stage[0][0][0][0];  // [64][64]
      static_assert(sizeof(stage) >= 64 * 64 * 4, "the sums fit the stages");
#pragma unroll
      for (int i = 0; i < 4; ++i) *reinterpret_cast<float4*>(sum + (tr * 4u + i) * 64u + tc * 4u) = *reinterpret_cast<float4*>(acc[i]);
      cluster_sync();
      for (uint32_t r = 64u * rank / split + tr; r < 64u * (rank + 1) / split; r += 16u) {
        float v[4] = {};
        const uint32_t at = su32(sum + r * 64u + tc * 4u);
        for (uint32_t q = 0; q < split; ++q) {
          const float4 u = cluster_load4(cluster_map(at, q));
          v[0] += u.x;
          v[1] += u.y;
          v[2] += u.z;
          v[3] += u.w;
        }
        epi_run<float, 4>(e, r0 + r, c0 + tc * 4u, v);
      }
      cluster_sync();
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < 4 * R; ++i)
#pragma unroll
    for (int h = 0; h < R; ++h)
      epi_run<float, 4>(e, r0 + (i / 4) * 64u + tr * 4u + i % 4, c0 + h * 64u + tc * 4u, acc[i] + 4 * h);
}

// ---- elementwise and layout kernels ---------------------------------------------------------------

template <typename T>
struct DzArgs {
  uint64_t rows, rows_each, lddy, ldpre, ldmul, lddz, lddmul;
  uint32_t cols;
  const T *dy, *pre, *mul;
  T *dz, *dmul;
  float* part;  // [gridDim.y][cols] column sums, or null
};

// 32 threads x V columns and a run of rows to a CTA, the rows dealt out to its eight warps; the warps' column sums are
// added in order
template <typename T, int V, int ACT>
__global__ void __launch_bounds__(256) dz_kernel(const DzArgs<T> p) {
  kernel_begin();
  constexpr bool FAST = sizeof(T) == 2;
  __shared__ float sum[8][32 * V + 1];
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  const uint32_t c = (blockIdx.x * 32u + lane) * V;
  const uint64_t q0 = blockIdx.y * p.rows_each, q1 = q0 + p.rows_each < p.rows ? q0 + p.rows_each : p.rows;
  float s[V] = {};
  if (c < p.cols) {
#pragma unroll 2
    for (uint64_t r = q0 + warp; r < q1; r += 8) {
      const Pack<T, V> dq = load_pack<T, V>(p.dy + r * p.lddy + c);
      Pack<T, V> zq, mq;
      if (p.pre) zq = load_pack<T, V>(p.pre + r * p.ldpre + c);
      if (p.mul) mq = load_pack<T, V>(p.mul + r * p.ldmul + c);
      float d[V], z[V] = {}, m[V], om[V];
      unpack(dq, d);
      if (p.pre) unpack(zq, z);
      if (p.mul) unpack(mq, m);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        float a, g;
        act_both<ACT, FAST>(z[k], a, g);
        om[k] = d[k] * a;
        if (ACT != MP_ACT_NONE) d[k] *= g;
        if (p.mul) d[k] *= m[k];
        s[k] += d[k];
      }
      if (p.dz) store_pack<T, V>(p.dz + r * p.lddz + c, pack<T, V>(d));
      if (p.dmul) store_pack<T, V>(p.dmul + r * p.lddmul + c, pack<T, V>(om));
    }
  }
  if (!p.part) return;
#pragma unroll
  for (int k = 0; k < V; ++k) sum[warp][lane * V + k] = s[k];
  __syncthreads();
  for (uint32_t k = threadIdx.x; k < 32u * V; k += 256u) {
    const uint32_t cc = blockIdx.x * 32u * V + k;
    if (cc < p.cols) {
      float v = 0.0f;
#pragma unroll
      for (int q = 0; q < 8; ++q) v += sum[q][k];
      p.part[(uint64_t)blockIdx.y * p.cols + cc] = v;
    }
  }
}

// copies (or zeros: no source) of up to two matrices, blockIdx.y saying which
template <typename T>
struct CopyArgs {
  const T* src;
  T* dst;
  uint64_t lds, ldd, rows;
  uint32_t cols;
};
template <typename T>
__global__ void __launch_bounds__(256) copy_kernel(const CopyArgs<T> a, const CopyArgs<T> b) {
  kernel_begin();
  const CopyArgs<T>& m = blockIdx.y ? b : a;
  // a warp to a row, four elements of a lane in flight
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  for (uint64_t r = blockIdx.x * 8ull + warp; r < m.rows; r += gridDim.x * 8ull)
    for (uint32_t c = lane; c < m.cols; c += 128u) {
      T v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = m.src && c + 32u * k < m.cols ? m.src[r * m.lds + c + 32u * k] : T(0.0f);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (c + 32u * k < m.cols) m.dst[r * m.ldd + c + 32u * k] = v[k];
    }
}

// ---- launches -------------------------------------------------------------------------------------

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// the driver's encoder, found in the driver's library at the first use (the library itself links no driver)
EncodeTiled encode_tiled() {
  static const EncodeTiled f = [] {
    void* so = dlopen("libcuda.so.1", RTLD_NOW);
    return reinterpret_cast<EncodeTiled>(so ? dlsym(so, "cuTensorMapEncodeTiled") : nullptr);
  }();
  return f;
}

// the map of an operand of n rows (m or n) with `inner` k; box: rows of a k-major tile
mp_status make_map(CUtensorMap* map, const Mat& m, bool t, uint64_t n, uint64_t inner, uint32_t box) {
  const EncodeTiled f = encode_tiled();
  if (!f) {
    set_static_error("the driver's tensor-map encoder is not available");
    return MP_ERR_CUDA;
  }
  const cuuint64_t dims[2] = {t ? n : inner, t ? inner : n};
  const cuuint64_t stride[1] = {m.ld * 2u};
  const cuuint32_t boxes[2] = {64u, t ? 64u : box}, ones[2] = {1u, 1u};
  const CUresult r = f(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(m.p), dims, stride, boxes, ones,
                       CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                       CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) {
    set_static_error("the driver refused a matrix (cuTensorMapEncodeTiled)");
    return MP_ERR_CUDA;
  }
  return MP_OK;
}

template <typename T>
Epi<T> epi_of(const Epilogue& e) {
  const size_t es = sizeof(T);
  size_t unit = 16;
  auto ok = [&](const void* p, uint64_t ld) { return !p || (reinterpret_cast<uintptr_t>(p) % unit == 0 && ld * es % unit == 0); };
  auto all = [&] { return ok(e.bias, 0) && ok(e.mul.p, e.mul.ld) && ok(e.res.p, e.res.ld) && ok(e.y, e.ldy) && ok(e.pre, e.ldpre); };
  Epi<T> q;
  q.rows = (uint32_t)e.rows;
  q.cols = (uint32_t)e.cols;
  q.act = e.act;
  q.bias = static_cast<const T*>(e.bias);
  q.mul = static_cast<const T*>(e.mul.p);
  q.res = static_cast<const T*>(e.res.p);
  q.ldmul = e.mul.ld;
  q.ldres = e.res.ld;
  q.y = static_cast<T*>(e.y);
  q.pre = static_cast<T*>(e.pre);
  q.ldy = e.ldy;
  q.ldpre = e.ldpre;
  q.vec = all();
  unit = 4 * es;
  q.quad = all();
  return q;
}

int device_sms() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
    cudaGetLastError();
    return 152;
  }
  return n;
}

template <typename... P, typename... A>
cudaError_t launch_cluster(void (*k)(P...), unsigned grid, unsigned threads, unsigned cluster, size_t smem, cudaStream_t st,
                           const A&... a) {
  if (smem > 0) {
    const cudaError_t e =
        cudaFuncSetAttribute(reinterpret_cast<const void*>(k), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = cluster;
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  count_launches(1);
  return cudaLaunchKernelEx(&cfg, k, P(a)...);
}

template <int BN, bool AT, bool BT>
cudaError_t launch_split(const CUtensorMap& ma, const CUtensorMap& mb, const Epi<bf16>& e, uint32_t kb, unsigned split,
                         int stages, const Wait& w, cudaStream_t st) {
  const uint32_t tiles_r = (e.rows + BN - 1) / BN, tiles_c = (e.cols + 127u) / 128u;
  // the stages, and in their place the sums at the end ([BN][128] fp32)
  const size_t smem = std::max((size_t)stages * (128 * 128 + BN * 128), (size_t)BN * 512) + 1024;
  return launch_cluster(split_kernel<BN, AT, BT>, tiles_r * tiles_c * split, kGemmThreads, split, smem, st, ma, mb, e, kb, tiles_r,
                        stages, w);
}

template <bool AT, bool BT>
cudaError_t launch_split_of(int bn, const CUtensorMap& ma, const CUtensorMap& mb, const Epi<bf16>& e, uint32_t kb,
                            unsigned split, int stages, const Wait& w, cudaStream_t st) {
  if constexpr (!BT) {
    if (bn == 16) return launch_split<16, AT, BT>(ma, mb, e, kb, split, stages, w, st);
    if (bn == 32) return launch_split<32, AT, BT>(ma, mb, e, kb, split, stages, w, st);
    if (bn == 64) return launch_split<64, AT, BT>(ma, mb, e, kb, split, stages, w, st);
  }
  return launch_split<128, AT, BT>(ma, mb, e, kb, split, stages, w, st);
}

template <int CG, bool AT, bool BT>
cudaError_t launch_big(const CUtensorMap& ma, const CUtensorMap& mb, const Epi<bf16>& e, uint32_t kb,
                       const Wait& w, cudaStream_t st) {
  const uint32_t tiles_r = (e.rows + 128u * CG - 1) / (128u * CG), tiles_c = (e.cols + 255u) / 256u;
  const uint64_t tiles = (uint64_t)tiles_r * tiles_c;
  const unsigned groups = (unsigned)std::min<uint64_t>(tiles, (uint64_t)device_sms() / CG);
  const size_t smem = CG == 2 ? 6 * 32768 + 1024 : 4 * 49152 + 1024;
  return launch_cluster(gemm_kernel<CG, AT, BT>, groups * CG, kGemmThreads, CG, smem, st, ma, mb, e, kb, tiles_r, tiles_c, w);
}

mp_status gemm_bf16(const GemmLaunch& g, cudaStream_t st) {
  const Epi<bf16> e = epi_of<bf16>(g.e);
  const uint64_t kb64 = (g.inner + kBK - 1) / kBK;
  const uint32_t kb = (uint32_t)kb64;
  const uint64_t sms = (uint64_t)device_sms();
  const uint64_t big_tiles = ((g.e.rows + 255) / 256) * ((g.e.cols + 255) / 256);
  const bool big = g.e.rows > 128 && big_tiles * 2 >= sms / 2;
  // split: rows of a tile, and the CTAs that share it
  int bn = 128;
  if (!g.a_t) bn = g.e.rows <= 16 ? 16 : g.e.rows <= 32 ? 32 : g.e.rows <= 64 ? 64 : 128;
  CUtensorMap ma, mb;  // of the rows' operand and of the columns'
  mp_status s;
  if ((s = make_map(&ma, g.a, g.a_t, g.e.rows, g.inner, big ? 128u : (uint32_t)bn)) != MP_OK) return s;
  if ((s = make_map(&mb, g.b, g.b_t, g.e.cols, g.inner, 128u)) != MP_OK) return s;
  const Wait w = {g.err, g.wait_limit ? g.wait_limit : kWaitLimit, g.stall};
  cudaError_t r;
  if (big) {
    r = g.a_t ? launch_big<2, true, true>(ma, mb, e, kb, w, st)
        : g.b_t ? launch_big<2, false, true>(ma, mb, e, kb, w, st)
                : launch_big<2, false, false>(ma, mb, e, kb, w, st);
  } else {
    const uint64_t tiles = ((g.e.rows + bn - 1) / bn) * ((g.e.cols + 127) / 128);
    // As many CTAs as share a tile while three to an SM hold them all and each has two stages at least, and as many
    // stages as shared memory holds then (with a tenth of the SMs' places to spare: clusters do not fill every one).
    // One row, 4096 -> 14336, 112 tiles: 26.8 us unsplit, 23.0 with two CTAs of 5 stages, 21.9 with four of 3, 29 with
    // four of 4 stages, which do not all fit; 24 rows, 14336 -> 4096, 32 tiles: 83 us unsplit, 25.1 with eight of 5.
    const int stage = 128 * 128 + bn * 128;
    auto stages_with = [&](uint64_t ctas) {
      const uint64_t per_sm = std::max<uint64_t>(1, std::min<uint64_t>(4, (ctas * 11 + sms * 10 - 1) / (sms * 10)));
      return (int)std::min<uint64_t>(6, (228 * 1024 / per_sm - 2560) / stage);
    };
    unsigned split = 1;
    while (split < 8 && tiles * split * 2 <= sms * 3 && kb >= 4 * split && stages_with(tiles * split * 2) >= 2) split *= 2;
    const int stages = std::max(2, stages_with(tiles * split));
    r = g.a_t ? launch_split_of<true, true>(bn, mb, ma, e, kb, split, stages, w, st)
        : g.b_t ? launch_split_of<true, false>(bn, mb, ma, e, kb, split, stages, w, st)
                : launch_split_of<false, false>(bn, mb, ma, e, kb, split, stages, w, st);
  }
  return r == cudaSuccess ? MP_OK : cuda_fail(r, "linear kernel");
}

mp_status gemm_f32(const GemmLaunch& g, cudaStream_t st) {
  const Epi<float> e = epi_of<float>(g.e);
  auto tiles_of = [&](uint64_t n) { return ((g.e.rows + n - 1) / n) * ((g.e.cols + n - 1) / n); };
  const uint64_t sms = (uint64_t)device_sms(), one = 1;
  const bool large = tiles_of(128) >= sms;  // tiles of 128 fill the GPU
  const uint64_t tiles = tiles_of(large ? 128 : 64);
  if (tiles > 0x7FFFFFFFull) {
    set_static_error("the output has too many tiles");
    return MP_ERR_UNSUPPORTED;
  }
  unsigned split = 1;
  while (!large && split < 8 && tiles * split * 2 <= sms * 2 && g.inner >= 128ull * split) split *= 2;
  const uint32_t inner = (uint32_t)g.inner, each = (uint32_t)(((g.inner + split - 1) / split + 31) / 32 * 32);
  const float *a = static_cast<const float*>(g.a.p), *b = static_cast<const float*>(g.b.p);
  const uint64_t ar = g.a_t ? one : g.a.ld, ak = g.a_t ? g.a.ld : one, br = g.b_t ? one : g.b.ld, bk = g.b_t ? g.b.ld : one;
  const cudaError_t r =
      large ? launch_kernel(true, gemm_f32_kernel<2, 16>, dim3((unsigned)tiles), 256, 0, st, a, ar, ak, b, br, bk, inner, inner, e)
            : launch_cluster(gemm_f32_kernel<1, 32>, (unsigned)tiles * split, 256, split, 0, st, a, ar, ak, b, br, bk, inner, each, e);
  return r == cudaSuccess ? MP_OK : cuda_fail(r, "linear kernel");
}

template <typename T, int V, int ACT>
cudaError_t dz_launch(const DzArgs<T>& a, dim3 grid, cudaStream_t st) {
  return launch_kernel(true, dz_kernel<T, V, ACT>, grid, 256, 0, st, a);
}

constexpr uint32_t kDzParts = 64;  // runs of rows at most: their column sums are read again

uint32_t dz_parts(const DzLaunch& p, int v) {
  const uint64_t across = (p.cols + 32u * v - 1) / (32u * v);
  const uint64_t want = std::max<uint64_t>(1, 8ull * device_sms() / across);
  return (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>({want, (uint64_t)kDzParts, (p.rows + 15) / 16}));
}

bool dz_vectors(const DzLaunch& p) {
  const size_t es = p.dtype == MP_BF16 ? 2 : 4;
  auto ok = [&](const void* q, uint64_t ld) { return !q || (reinterpret_cast<uintptr_t>(q) % 16 == 0 && ld * es % 16 == 0); };
  return p.cols * es % 16 == 0 && ok(p.dy.p, p.dy.ld) && ok(p.pre.p, p.pre.ld) && ok(p.mul.p, p.mul.ld) && ok(p.dz, p.lddz) &&
         ok(p.dmul, p.lddmul);
}

template <typename T, int V>
cudaError_t dz_of(const DzLaunch& p, float* part, cudaStream_t st) {
  DzArgs<T> a;
  a.rows = p.rows;
  a.cols = (uint32_t)p.cols;
  a.dy = static_cast<const T*>(p.dy.p);
  a.lddy = p.dy.ld;
  a.pre = static_cast<const T*>(p.pre.p);
  a.ldpre = p.pre.ld;
  a.mul = static_cast<const T*>(p.mul.p);
  a.ldmul = p.mul.ld;
  a.dz = static_cast<T*>(p.dz);
  a.lddz = p.lddz;
  a.dmul = static_cast<T*>(p.dmul);
  a.lddmul = p.lddmul;
  a.part = p.db ? part : nullptr;
  const uint32_t parts = dz_parts(p, V);
  a.rows_each = (p.rows + parts - 1) / parts;
  const dim3 grid((unsigned)((p.cols + 32u * V - 1) / (32u * V)), parts);
  cudaError_t e;
  switch (p.act) {
    case MP_ACT_RELU: e = dz_launch<T, V, MP_ACT_RELU>(a, grid, st); break;
    case MP_ACT_SILU: e = dz_launch<T, V, MP_ACT_SILU>(a, grid, st); break;
    case MP_ACT_GELU: e = dz_launch<T, V, MP_ACT_GELU>(a, grid, st); break;
    case MP_ACT_GELU_TANH: e = dz_launch<T, V, MP_ACT_GELU_TANH>(a, grid, st); break;
    default: e = dz_launch<T, V, MP_ACT_NONE>(a, grid, st); break;
  }
  if (e != cudaSuccess || !p.db) return e;
  return launch_column_sums(p.dtype, part, parts, (uint32_t)p.cols, p.db, st);
}

}  // namespace

bool gemm_operand_ok(mp_dtype dtype, const Mat& m) {
  return dtype != MP_BF16 || (reinterpret_cast<uintptr_t>(m.p) % 16 == 0 && m.ld % 8 == 0);
}

mp_status launch_gemm(const GemmLaunch& g, cudaStream_t st) {
  if (g.dtype == MP_BF16) return gemm_bf16(g, st);
  return gemm_f32(g, st);
}

size_t dz_scratch(const DzLaunch& p) {
  return p.db ? (size_t)kDzParts * p.cols * sizeof(float) : 0;
}

cudaError_t launch_dz(const DzLaunch& p, float* scratch, cudaStream_t st) {
  const bool vec = dz_vectors(p);
  if (p.dtype == MP_BF16) return vec ? dz_of<bf16, 8>(p, scratch, st) : dz_of<bf16, 1>(p, scratch, st);
  return vec ? dz_of<float, 4>(p, scratch, st) : dz_of<float, 1>(p, scratch, st);
}

template <typename T>
cudaError_t copy_of(const Copy* m, int n, cudaStream_t st) {
  CopyArgs<T> a[2] = {};
  uint64_t rows = 0;
  for (int k = 0; k < n; ++k) {
    a[k] = CopyArgs<T>{static_cast<const T*>(m[k].src.p), static_cast<T*>(m[k].dst), m[k].src.ld, m[k].ldd, m[k].rows,
                       (uint32_t)m[k].cols};
    rows = std::max(rows, m[k].rows);
  }
  const dim3 grid((unsigned)std::min<uint64_t>((rows + 7) / 8, 8ull * device_sms()), n);
  return launch_kernel(true, copy_kernel<T>, grid, 256, 0, st, a[0], a[1]);
}

cudaError_t launch_copies(mp_dtype dtype, const Copy* m, int n, cudaStream_t st) {
  return dtype == MP_BF16 ? copy_of<bf16>(m, n, st) : copy_of<float>(m, n, st);
}

}  // namespace mp
