// tokens_embed.hip -- rows of a token table and their gradient.
//
// Lookup: out_m = round(scale * W[t_m]), one pass, bound by HBM: each thread
// carries four rows' worth of one 16-byte column.
//
// Gradient: dW_v = round(scale * sum over the positions of v of G_m).
//   1. sort       positions by token, stable
//   2. zero       rows of dW (tokens without a position stay zero)
//   3. sums       one wave per slice of consecutive sorted positions and block of
//                 columns adds each token's rows in fp32 in that order; a run that
//                 a slice end cuts leaves its part in `carry`
//   4. cut runs   the slice where a run starts adds its parts in slice order
// No atomics on floating-point values: the same bits on every run.
#include <algorithm>
#include <type_traits>

#include "fkm_device.h"
#include "tokens_internal.h"

namespace fkm {

namespace {

// E elements of a row as fp32: 16 bytes where the row's start is aligned to them
// (VEC), else element by element with the row's end checked.
template <int DT> struct Tok {
  static constexpr int E = DT == DT_F32 ? 4 : 8;  // elements in 16 bytes
  using T = std::conditional_t<DT == DT_F32, float, uint16_t>;
  __device__ static float widen(T v) {
    if constexpr (DT == DT_F32) return v;
    else return Elem<DT>::widen(v);
  }
  __device__ static T narrow(float v) {
    if constexpr (DT == DT_F32) return v;
    else return Elem<DT>::narrow(v);
  }
};

template <int DT, bool VEC>
__device__ __forceinline__ void load_e(const typename Tok<DT>::T* row, int d, int D,
                                       float (&v)[Tok<DT>::E]) {
  constexpr int E = Tok<DT>::E;
  alignas(16) typename Tok<DT>::T x[E];
  if constexpr (VEC) {
    *reinterpret_cast<uint4*>(x) = *reinterpret_cast<const uint4*>(row + d);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = d + e < D ? row[d + e] : typename Tok<DT>::T(0);
  }
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = Tok<DT>::widen(x[e]);
}

// E elements (of type WT, which may hold them in 32 bytes) to a row.
template <int WT, int E, bool VEC>
__device__ __forceinline__ void store_e(typename Tok<WT>::T* row, int d, int D,
                                        const float (&v)[E]) {
  using T = typename Tok<WT>::T;
  alignas(16) T x[E];
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = Tok<WT>::narrow(v[e]);
  if constexpr (VEC) {
#pragma unroll
    for (int e = 0; e < E; e += 16 / (int)sizeof(T))
      *reinterpret_cast<uint4*>(row + d + e) = *reinterpret_cast<const uint4*>(x + e);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (d + e < D) row[d + e] = x[e];
  }
}

constexpr int EMB_U = 4;  // rows per thread
constexpr int64_t MAX_BLOCKS = 1 << 22;  // of 256 threads: a grid holds fewer than 2^32 threads

// tpr threads (a power of two) share a row.
template <int DT, bool VEC>
__global__ __launch_bounds__(256) void embed_kernel(const typename Tok<DT>::T* __restrict__ W,
                                                    const int32_t* __restrict__ idx, int64_t rows,
                                                    int64_t M, int V, int D, float scale, int tpr,
                                                    typename Tok<DT>::T* __restrict__ out) {
  constexpr int E = Tok<DT>::E;
  const int t = threadIdx.x, rpb = 256 / tpr;
  for (int64_t r0 = (int64_t)blockIdx.x * rpb * EMB_U + t / tpr; r0 < rows;
       r0 += (int64_t)gridDim.x * rpb * EMB_U) {
  int64_t src[EMB_U];
#pragma unroll
  for (int u = 0; u < EMB_U; ++u) {
    const int64_t r = r0 + u * rpb;
    const int id = r < rows ? idx[r] : -1;
    src[u] = (unsigned)id < (unsigned)V ? (r / M) * V + id : -1;
  }
  for (int d = (t % tpr) * E; d < D; d += tpr * E) {
    float v[EMB_U][E];
#pragma unroll
    for (int u = 0; u < EMB_U; ++u) {
      if (src[u] >= 0) {
        load_e<DT, VEC>(W + src[u] * D, d, D, v[u]);
#pragma unroll
        for (int e = 0; e < E; ++e) v[u][e] *= scale;
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[u][e] = 0.f;
      }
    }
#pragma unroll
    for (int u = 0; u < EMB_U; ++u)
      if (r0 + u * rpb < rows) store_e<DT, E, VEC>(out + (r0 + u * rpb) * D, d, D, v[u]);
  }
  }
}

template <int DT>
hipError_t launch_embed_dt(const void* W, const int32_t* idx, int64_t B, int64_t M, int64_t V,
                           int64_t D, float scale, void* out, hipStream_t s) {
  using T = typename Tok<DT>::T;
  constexpr int E = Tok<DT>::E;
  int tpr = 1;
  while (tpr < 256 && tpr * E < D) tpr *= 2;
  const int64_t rows = B * M, per = 256 / tpr * EMB_U;
  const dim3 grid((unsigned)std::min<int64_t>((rows + per - 1) / per, MAX_BLOCKS));
  if (D % E == 0)
    embed_kernel<DT, true><<<grid, 256, 0, s>>>((const T*)W, idx, rows, M, (int)V, (int)D, scale,
                                                tpr, (T*)out);
  else
    embed_kernel<DT, false><<<grid, 256, 0, s>>>((const T*)W, idx, rows, M, (int)V, (int)D, scale,
                                                 tpr, (T*)out);
  return hipGetLastError();
}

// ---- gradient ------------------------------------------------------------------
constexpr int64_t SUM_SLICE = 32;  // sorted positions per wave

__global__ __launch_bounds__(256) void zero_kernel(char* __restrict__ p, int64_t bytes) {
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 16; i < bytes;
       i += (int64_t)gridDim.x * 4096) {
    if (i + 16 <= bytes) {
      *reinterpret_cast<uint4*>(p + i) = make_uint4(0, 0, 0, 0);
    } else {
      for (int64_t j = i; j < bytes; ++j) p[j] = 0;
    }
  }
}

// The row of token v gets `acc` (times scale; added to what it holds).
template <int WT, int E, bool VEC>
__device__ __forceinline__ void put_row(typename Tok<WT>::T* row, int d, int D, float (&acc)[E],
                                        float scale, bool accumulate) {
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] *= scale;
  if (accumulate) {
    using T = typename Tok<WT>::T;
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (VEC || d + e < D) acc[e] += Tok<WT>::widen((T)row[d + e]);
  }
  store_e<WT, E, VEC>(row, d, D, acc);
}

// One wave per slice and block of LPR column chunks; 64 / LPR rows in a step,
// added up at each run's end in a fixed order.
template <int DT, int WT, bool VEC>
__global__ __launch_bounds__(256) void embed_sums_kernel(
    const typename Tok<DT>::T* __restrict__ G, const int32_t* __restrict__ keys,
    const int32_t* __restrict__ perm, const int32_t* __restrict__ total, int64_t M, int V, int D,
    int lpr, int nslices, float scale, int accumulate, typename Tok<WT>::T* __restrict__ dW,
    float* __restrict__ carry) {
  constexpr int E = Tok<DT>::E, U = 4;
  const int lane = threadIdx.x & 63;
  const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t b = blockIdx.z;
  const int64_t n = total[b], j0 = w * SUM_SLICE;
  if (j0 >= n) return;
  const int cnt = (int)min<int64_t>(n - j0, SUM_SLICE);
  keys += b * M + j0;
  perm += b * M + j0;
  G += b * M * D;
  dW += b * V * D;
  // the slice's entries, one a lane; `starts`: the lanes where a run begins
  const int kl = lane < cnt ? keys[lane] : -1, pl = lane < cnt ? perm[lane] : 0;
  const int before = j0 > 0 ? keys[-1] : -1, after = j0 + cnt < n ? keys[cnt] : -1;
  const int kprev = __shfl_up(kl, 1);
  const uint64_t starts = __ballot(lane < cnt && (lane == 0 || kl != kprev));
  const int d = (blockIdx.y * lpr + lane % lpr) * E, r = lane / lpr, rpw = 64 / lpr;
  int pos = 0;
  while (pos < cnt) {
    const int key = __shfl(kl, pos);
    const uint64_t rest = (starts >> pos) >> 1;
    const int end = rest ? pos + 1 + (int)__builtin_ctzll(rest) : cnt;
    float acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
    for (int j = pos; j < end; j += U * rpw) {
      float v[U][E];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int jj = j + u * rpw + r;
        const int64_t p = __shfl(pl, jj & 63);
        if (jj < end && d < D) {
          load_e<DT, VEC>(G + p * D, d, D, v[u]);
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) v[u][e] = 0.f;
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += v[u][e];
    }
    for (int m = lpr; m < 64; m <<= 1)
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += __shfl_xor(acc[e], m);
    const bool head = pos == 0 && before == key;  // began in an earlier slice
    const bool tail = end == cnt && after == key;  // goes on in the next
    if (r == 0 && d < D) {
      if (head || tail) {
        float* c = carry + ((b * nslices + w) * 2 + (head ? 0 : 1)) * D;
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (VEC || d + e < D) c[d + e] = acc[e];
      } else {
        put_row<WT, E, VEC>(dW + (int64_t)key * D, d, D, acc, scale, accumulate);
      }
    }
    pos = end;
  }
}

// The slice in which a cut run starts adds the run's parts in slice order.
template <int WT, int E, bool VEC>
__global__ __launch_bounds__(256) void embed_cut_kernel(
    const int32_t* __restrict__ keys, const int32_t* __restrict__ total, int64_t M, int V, int D,
    int nslices, float scale, int accumulate, const float* __restrict__ carry,
    typename Tok<WT>::T* __restrict__ dW) {
  const int64_t w = blockIdx.x, b = blockIdx.z;
  const int64_t n = total[b], j0 = w * SUM_SLICE, j1 = j0 + SUM_SLICE;
  if (j1 >= n) return;  // nothing after this slice
  keys += b * M;
  const int key = keys[j1 - 1];
  if (keys[j1] != key || (j0 > 0 && keys[j0 - 1] == key)) return;  // not cut, or began earlier
  const int d = (blockIdx.y * 256 + threadIdx.x) * E;
  if (d >= D) return;
  const float* c = carry + (b * nslices + w) * 2 * D;
  float acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = VEC || d + e < D ? c[D + d + e] : 0.f;
  for (int64_t j = j1; j < n && keys[j] == key; j += SUM_SLICE) {
    c += 2 * D;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] += VEC || d + e < D ? c[d + e] : 0.f;
  }
  put_row<WT, E, VEC>(dW + (b * V + key) * D, d, D, acc, scale, accumulate);
}

template <int DT, int WT, bool VEC>
hipError_t launch_sums_dt(const void* G, int64_t B, int64_t M, int64_t V, int64_t D, float scale,
                          bool accumulate, void* dW, const EmbedGradWs& w, hipStream_t s) {
  constexpr int E = Tok<DT>::E;
  const int64_t chunks = (D + E - 1) / E, nslices = (M + SUM_SLICE - 1) / SUM_SLICE;
  int lpr = 1;
  while (lpr < 64 && lpr < chunks) lpr *= 2;
  using T = typename Tok<WT>::T;
  embed_sums_kernel<DT, WT, VEC>
      <<<dim3((unsigned)((nslices + 3) / 4), (unsigned)((chunks + lpr - 1) / lpr), (unsigned)B), 256,
         0, s>>>((const typename Tok<DT>::T*)G, w.sort.keys[0], w.sort.vals[0], w.sort.total, M,
                 (int)V, (int)D, lpr, (int)nslices, scale, accumulate, (T*)dW, w.carry);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  embed_cut_kernel<WT, E, VEC>
      <<<dim3((unsigned)nslices, (unsigned)((chunks + 255) / 256), (unsigned)B), 256, 0, s>>>(
          w.sort.keys[0], w.sort.total, M, (int)V, (int)D, (int)nslices, scale, accumulate, w.carry,
          (T*)dW);
  return hipGetLastError();
}

template <int DT, int WT>
hipError_t launch_sums_wt(const void* G, int64_t B, int64_t M, int64_t V, int64_t D, float scale,
                          bool accumulate, void* dW, const EmbedGradWs& w, hipStream_t s) {
  return D % Tok<DT>::E == 0
             ? launch_sums_dt<DT, WT, true>(G, B, M, V, D, scale, accumulate, dW, w, s)
             : launch_sums_dt<DT, WT, false>(G, B, M, V, D, scale, accumulate, dW, w, s);
}

}  // namespace

hipError_t launch_embed(const void* W, int dt, const int32_t* idx, int64_t B, int64_t M, int64_t V,
                        int64_t D, float scale, void* out, hipStream_t s) {
  if (dt == DT_BF16) return launch_embed_dt<DT_BF16>(W, idx, B, M, V, D, scale, out, s);
  if (dt == DT_F16) return launch_embed_dt<DT_F16>(W, idx, B, M, V, D, scale, out, s);
  return launch_embed_dt<DT_F32>(W, idx, B, M, V, D, scale, out, s);
}

EmbedGradWs embed_grad_carve(void* base, int64_t B, int64_t M, int64_t V, int64_t D) {
  EmbedGradWs w{};
  char* p = (char*)base;
  size_t o = 0;
  auto take = [&](size_t bytes) {
    char* r = p ? p + o : nullptr;
    o = (o + bytes + 255) & ~size_t(255);
    return r;
  };
  const int64_t chunks = (M + RADIX_CHUNK - 1) / RADIX_CHUNK;
  const int64_t nslices = (M + SUM_SLICE - 1) / SUM_SLICE;
  for (int i = 0; i < 2; ++i) {
    w.sort.keys[i] = (int32_t*)take((size_t)(B * M) * 4);
    w.sort.vals[i] = (int32_t*)take((size_t)(B * M) * 4);
  }
  w.sort.hist = (int32_t*)take((size_t)(B * RADIX_MAX_R * chunks) * 4);
  w.sort.bins = (int32_t*)take((size_t)(B * RADIX_MAX_R) * 4);
  w.sort.total = (int32_t*)take((size_t)B * 4);
  w.carry = (float*)take((size_t)(B * nslices * 2 * D) * 4);
  w.total = o;
  return w;
}

hipError_t launch_embed_grad(const void* G, int gdt, const int32_t* idx, int64_t B, int64_t M,
                             int64_t V, int64_t D, float scale, bool accumulate, void* dW, int wdt,
                             const EmbedGradWs& w, hipStream_t s) {
  hipError_t e = launch_token_sort(idx, B, M, V, w.sort, s);
  if (e != hipSuccess) return e;
  if (!accumulate) {
    const int64_t bytes = B * V * D * dt_bytes(wdt);
    zero_kernel<<<dim3((unsigned)std::min<int64_t>((bytes + 4095) / 4096, MAX_BLOCKS)), 256, 0, s>>>((char*)dW, bytes);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (gdt == DT_F32)
    return launch_sums_wt<DT_F32, DT_F32>(G, B, M, V, D, scale, accumulate, dW, w, s);
  if (gdt == DT_BF16)
    return wdt == DT_F32
               ? launch_sums_wt<DT_BF16, DT_F32>(G, B, M, V, D, scale, accumulate, dW, w, s)
               : launch_sums_wt<DT_BF16, DT_BF16>(G, B, M, V, D, scale, accumulate, dW, w, s);
  return wdt == DT_F32
             ? launch_sums_wt<DT_F16, DT_F32>(G, B, M, V, D, scale, accumulate, dW, w, s)
             : launch_sums_wt<DT_F16, DT_F16>(G, B, M, V, D, scale, accumulate, dW, w, s);
}

}  // namespace fkm
