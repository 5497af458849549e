// Joining the records of the gradient kernels: a user's history is worked on in pieces (the segments of the split-L
// schedule), each leaving its rows' statistics and its share of the queries' gradient in a record of its own.  They
// are joined in a fixed order -- ascending, or in interleaved ascending runs where users hold many -- so equal
// calls give equal bits.  Bound by latency: a few megabytes of records at most.
#include "common.hpp"
#include "grad.hpp"

namespace vista {
namespace {

struct Slots { int64_t first, count; };
// The records of user b.  Any offsets keep them inside [0, G + B).
__device__ __forceinline__ Slots slots_of(const GradRows& r, int64_t b) {
  int64_t begin = r.offsets[b], end = r.offsets[b + 1];
  begin = begin < 0 ? 0 : begin > r.N ? r.N : begin;
  end = end < 0 ? 0 : end > r.N ? r.N : end;
  if (end <= begin) return {0, 0};
  const int64_t g0 = segment_of(begin, r.seg), g1 = segment_of(end - 1, r.seg);
  return {g0 + b, g1 - g0 + 1};
}

// LPR lanes a row (1, 8 or 64): lane k joins every LPR-th record from its k-th on, and takes every LPR-th channel of the own key's
// products.  (One thread a row: 20 us instead of 5 where 9600 rows have a key of
// their own; eight: 50 instead of 9 for a million rows of one record each and none.)
template <typename T, int LPR>
__global__ __launch_bounds__(256) void join_stats_kernel(GradRows r, const float* __restrict__ stats, int rows,
                                                         float* __restrict__ lse, float* __restrict__ delta, const T* Q,
                                                         const T* dO, const float* Ks, const float* Vs, float* own_p,
                                                         float* own_ds) {
  if (blockIdx.x == 0) publish_status(r.offsets, r.B, r.check, r.status);
  const int64_t total = int64_t(r.B) * r.H * r.S, stride = int64_t(gridDim.x) * (256 / LPR);
  const int k = threadIdx.x % LPR, dh = r.d / r.H;
  for (int64_t at = (int64_t(blockIdx.x) * 256 + threadIdx.x) / LPR; at < total; at += stride) {
    const int64_t b = at / (r.H * r.S);
    const int rest = int(at % (r.H * r.S)), h = rest / r.S, i = rest % r.S;
    const Slots sl = slots_of(r, b);
    float m = kLowest, l = 0.f, e = 0.f;
    for (int64_t n = k; n < sl.count; n += LPR) {
      const float* s = stats + (((sl.first + n) * r.H + h) * rows + i) * 3;
      join_stats(m, l, e, s[0], s[1], s[2]);
    }
    float own_s = 0.f, own_t = 0.f;
    if (Ks && sl.count) {
      const T* q = Q + b * r.q_user_stride + int64_t(i) * r.d + h * dh;
      const T* o = dO + (b * r.S + i) * r.d + h * dh;
      const int64_t own = ((r.q_user_stride ? b * r.S : 0) + i) * r.d + h * dh;
      for (int c = k; c < dh; c += LPR) {
        own_s = fmaf(to_f32(q[c]), Ks[own + c], own_s);
        own_t = fmaf(to_f32(o[c]), Vs[own + c], own_t);
      }
    }
#pragma unroll
    for (int o = 1; o < LPR; o *= 2) {
      const float m2 = __shfl_xor(m, o, 64), l2 = __shfl_xor(l, o, 64), e2 = __shfl_xor(e, o, 64);
      join_stats(m, l, e, m2, l2, e2);
      own_s += __shfl_xor(own_s, o, 64);
      own_t += __shfl_xor(own_t, o, 64);
    }
    if (k != 0) continue;
    own_s *= r.scale_log2;
    if (Ks && sl.count) join_stats(m, l, e, own_s, 1.f, own_t);
    const float ls = sl.count ? m + __builtin_amdgcn_logf(l) : 0.f, dl = sl.count ? e / l : 0.f;
    lse[at] = ls;
    delta[at] = dl;
    if (Ks) {
      const float p = sl.count ? exp2_fast(own_s - ls) : 0.f;
      own_p[at] = p;
      own_ds[at] = p * (own_t - dl);
    }
  }
}

template <typename T, int V>
__device__ __forceinline__ void store_grads(T* p, const float (&v)[V]) {
  if constexpr (V == 1) {
    store_grad(p, v[0]);
  } else if constexpr (sizeof(T) == 2) {
    struct __attribute__((packed, aligned(2))) Raw { uint32_t v[V / 2]; } r;
#pragma unroll
    for (int e = 0; e < V / 2; ++e) r.v[e] = pair_to_bf16(v[2 * e], v[2 * e + 1]);
    *reinterpret_cast<Raw*>(p) = r;
  } else {
    struct __attribute__((packed, aligned(4))) Raw { float v[V]; } r;
#pragma unroll
    for (int e = 0; e < V; ++e) r.v[e] = v[e];
    *reinterpret_cast<Raw*>(p) = r;
  }
}

// V columns a thread (4 where they divide the head's width: a quarter of the index arithmetic, which is most of this kernel; 18 us
// with single columns for 64 users of 256 x 128).  RUNS threads for the same columns (1 or 8), each an interleaved ascending
// run, added in ascending order.
template <typename T, int RUNS, int V>
__global__ __launch_bounds__(256) void join_queries_kernel(GradRows r, const float* __restrict__ records, int rows, float factor,
                                                           const T* Q, const T* dO, const float* Ks, const float* own_p,
                                                           const float* own_ds, T* d_queries, T* d_self_keys, T* d_self_values) {
  constexpr int kCols = 256 / RUNS;
  struct alignas(4 * V) Chunk { float v[V]; };
  __shared__ Chunk part[RUNS][kCols];
  const int64_t total = int64_t(r.B) * r.S * r.d / V;
  const int c = threadIdx.x % kCols, k = threadIdx.x / kCols, dh = r.d / r.H;
  for (int64_t base = int64_t(blockIdx.x) * kCols; base < total; base += int64_t(gridDim.x) * kCols) {
    const bool in = base + c < total;
    const int64_t at = (base + c) * V, row = in ? at / r.d : 0, b = row / r.S;
    const int i = int(row - b * r.S), col = in ? int(at - row * r.d) : 0, h = col / dh;
    const Slots sl = slots_of(r, b);
    Chunk sum = {};
    if (in) {
      const float* rec = records + ((sl.first * r.H + h) * rows + i) * dh + (col - h * dh);
      const int64_t step = int64_t(r.H) * rows * dh;
#pragma unroll 4
      for (int64_t n = k; n < sl.count; n += RUNS) {
        const Chunk one = *reinterpret_cast<const Chunk*>(rec + n * step);
#pragma unroll
        for (int e = 0; e < V; ++e) sum.v[e] += one.v[e];
      }
    }
    if (RUNS > 1) {
      __syncthreads();
      part[k][c] = sum;
      __syncthreads();
      if (k == 0)
#pragma unroll
        for (int n = 1; n < RUNS; ++n)
#pragma unroll
          for (int e = 0; e < V; ++e) sum.v[e] += part[n][c].v[e];
    }
    if (!in || k != 0) continue;
#pragma unroll
    for (int e = 0; e < V; ++e) sum.v[e] *= factor;
    if (Ks) {
      const int64_t stat = (b * r.H + h) * r.S + i, own = ((r.q_user_stride ? b * r.S : 0) + i) * r.d + col;
      const bool any = sl.count != 0;
      const float ds = any ? own_ds[stat] * r.scale : 0.f, p = any ? own_p[stat] : 0.f;
      float dk[V], dv[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        if (any) sum.v[e] = fmaf(ds, Ks[own + e], sum.v[e]);
        dk[e] = any ? ds * to_f32(Q[b * r.q_user_stride + int64_t(i) * r.d + col + e]) : 0.f;
        dv[e] = any ? p * to_f32(dO[at + e]) : 0.f;
      }
      store_grads<T, V>(d_self_keys + at, dk);
      store_grads<T, V>(d_self_values + at, dv);
    }
    store_grads<T, V>(d_queries + at, sum.v);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void join_shares_kernel(const float* __restrict__ records, int shares, int64_t total, int S,
                                                          int d, int H, T* d_summ) {
  const int dh = d / H;
  for (int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x; at < total; at += int64_t(gridDim.x) * 256) {
    const int64_t row = at / d, b = row / S;
    const int i = int(row % S), col = int(at % d);
    const float* rec = records + ((b * H + col / dh) * S + i) * dh + col % dh;
    float sum = 0.f;
#pragma unroll 8
    for (int n = 0; n < shares; ++n) sum += rec[n * total];
    store_grad(d_summ + at, sum);
  }
}

unsigned blocks_for(int64_t threads) {
  const int64_t n = (threads + 255) / 256;
  return unsigned(n < (1 << 20) ? n : 1 << 20);
}

template <typename T>
hipError_t join_stats_t(const GradRows& r, const float* stats, int rows, float* lse, float* delta, const void* Q, const void* dO,
                        const float* Ks, const float* Vs, float* own_p, float* own_ds, hipStream_t s) {
  const int64_t total = int64_t(r.B) * r.H * r.S;
  // a lane a row where users hold less than two records and have no key of their own, a wave once they hold eight or more
  if (r.G < r.B && !Ks)
    return launch(join_stats_kernel<T, 1>, dim3(blocks_for(total)), dim3(256), 0, s, r, stats, rows, lse, delta,
                  static_cast<const T*>(Q), static_cast<const T*>(dO), Ks, Vs, own_p, own_ds);
  if (r.G >= 7 * int64_t(r.B))
    return launch(join_stats_kernel<T, 64>, dim3(blocks_for(total * 64)), dim3(256), 0, s, r, stats, rows, lse, delta,
                  static_cast<const T*>(Q), static_cast<const T*>(dO), Ks, Vs, own_p, own_ds);
  return launch(join_stats_kernel<T, 8>, dim3(blocks_for(total * 8)), dim3(256), 0, s, r, stats, rows, lse, delta,
                static_cast<const T*>(Q), static_cast<const T*>(dO), Ks, Vs, own_p, own_ds);
}

template <typename T>
hipError_t join_queries_t(const GradRows& r, const float* records, int rows, float factor, const void* Q, const void* dO,
                          const float* Ks, const float* own_p, const float* own_ds, void* dq, void* dks, void* dvs,
                          hipStream_t s) {
  auto run = [&](auto* kernel, int runs, int columns) {
    const int64_t threads = int64_t(r.B) * r.S * r.d / columns * runs;
    return launch(kernel, dim3(blocks_for(threads)), dim3(256), 0, s, r, records, rows, factor, static_cast<const T*>(Q),
                  static_cast<const T*>(dO), Ks, own_p, own_ds, static_cast<T*>(dq), static_cast<T*>(dks), static_cast<T*>(dvs));
  };
  const bool many = r.G >= 7 * int64_t(r.B);
  if (r.d / r.H % 4 == 0) return many ? run(join_queries_kernel<T, 8, 4>, 8, 4) : run(join_queries_kernel<T, 1, 4>, 1, 4);
  return many ? run(join_queries_kernel<T, 8, 1>, 8, 1) : run(join_queries_kernel<T, 1, 1>, 1, 1);
}

}  // namespace

hipError_t grad_join_stats(const GradRows& r, int dtype, const float* stats, int rows, float* lse, float* delta, const void* Q,
                           const void* dO, const float* Ks, const float* Vs, float* own_p, float* own_ds, hipStream_t s) {
  return dtype == VISTA_BF16 ? join_stats_t<bf16_t>(r, stats, rows, lse, delta, Q, dO, Ks, Vs, own_p, own_ds, s)
                             : join_stats_t<float>(r, stats, rows, lse, delta, Q, dO, Ks, Vs, own_p, own_ds, s);
}

hipError_t grad_join_queries(const GradRows& r, int dtype, const float* records, int rows, float factor, const void* Q,
                             const void* dO, const float* Ks, const float* own_p, const float* own_ds, void* d_queries,
                             void* d_self_keys, void* d_self_values, hipStream_t s) {
  return dtype == VISTA_BF16
             ? join_queries_t<bf16_t>(r, records, rows, factor, Q, dO, Ks, own_p, own_ds, d_queries, d_self_keys, d_self_values, s)
             : join_queries_t<float>(r, records, rows, factor, Q, dO, Ks, own_p, own_ds, d_queries, d_self_keys, d_self_values, s);
}

hipError_t grad_join_shares(int dtype, const float* records, int shares, int64_t B, int S, int d, int H, void* d_summ,
                            hipStream_t s) {
  const int64_t total = B * S * d;
  if (dtype == VISTA_BF16)
    return launch(join_shares_kernel<bf16_t>, dim3(blocks_for(total)), dim3(256), 0, s, records, shares, total, S, d, H,
                  static_cast<bf16_t*>(d_summ));
  return launch(join_shares_kernel<float>, dim3(blocks_for(total)), dim3(256), 0, s, records, shares, total, S, d, H,
                static_cast<float*>(d_summ));
}

}  // namespace vista
