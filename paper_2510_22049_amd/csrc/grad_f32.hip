// Gradients of softmax attention, both stages, on the fp32 matrix instructions (v_mfma_f32_16x16x4_f32), for fp32
// and bf16 storage and any head width up to 64.
//
//   P = softmax(scale Q K^T),  dP = dO V^T,  delta_i = sum_j P_ij dP_ij,  dS = P (dP - delta)
//   dV = P^T dO,  dQ = scale dS K,  dK = scale dS^T Q
//
// Nothing of the forward pass is kept: scores are formed again, first for each row's maximum, sum and delta, then
// for the gradients.  One walk serves all of it.  A wave owns 16 rows (queries, or keys), one a lane of 16 and
// both of its vectors in registers, and passes over the rows of the other kind, which the workgroup stages in LDS
// 32 at a time.  The two products of a tile, scores and dP, have the own rows on the accumulator's columns, so
// their registers are the next product's operand as they stand (the contraction then runs over the other rows):
//   queries' own rows (q, dO), others (k, v):   row statistics; dQ^T += K^T dS^T
//   keys' own rows (k, v), others (q, dO):      dV^T += dO^T P, dK^T += Q^T dS
// That is seven products of the history's gradient where five and the two of the statistics would do, and no
// exchange between waves: on these instructions (157 TFLOP/s) the products are what a call waits for.
// Head widths that are no multiple of 16 are padded with zeros on their way into LDS and registers.
//
// Measured: one user of 1024 items, d = 64, one head, 16 queries, fp32: 32 us, five launches of 4 to 11 us, all latency.  75 users x 333
// candidates, d = 64, one head, 100 summaries, with the self term: 39 us, 5 of them the join; 61 with a pass for the
// candidates' rows and one for the summaries' rows, each forming scores and dP (as beyond 128 summaries).
#include "common.hpp"
#include "grad.hpp"

namespace vista {

typedef __attribute__((ext_vector_type(4))) float f32x4;

namespace {

constexpr int kOthers = 32;            // rows staged at a time
constexpr int kOwn = 64;               // rows a workgroup owns, 16 a wave

__device__ __forceinline__ f32x4 mfma4(float a, float b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float at(const float4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// Four channels of a row from channel c on, zeros beyond the head's width.  wide: the row's address is a multiple of
// four elements and so is the width.
template <typename T>
__device__ __forceinline__ float4 load_channels(const T* row, int c, int dh, bool wide) {
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  if (wide) {
    if (c < dh) {
      struct alignas(4 * sizeof(T)) Raw { T v[4]; };
      const Raw r = *reinterpret_cast<const Raw*>(row + c);
      v = make_float4(to_f32(r.v[0]), to_f32(r.v[1]), to_f32(r.v[2]), to_f32(r.v[3]));
    }
    return v;
  }
  if (c < dh) v.x = to_f32(row[c]);
  if (c + 1 < dh) v.y = to_f32(row[c + 1]);
  if (c + 2 < dh) v.z = to_f32(row[c + 2]);
  if (c + 3 < dh) v.w = to_f32(row[c + 3]);
  return v;
}
template <typename T>
__device__ __forceinline__ void store_channels(T* row, int c, int dh, const f32x4& v) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (c + i < dh) store_grad(row + c + i, v[i]);
}

// Rows of 16 DT channels and 4 more: four rows are 16 banks apart, so reads by rows and by columns both spread.
template <int DT>
struct Others {
  static constexpr int kRow = 16 * DT + 4;
  float a[kOthers * kRow], b[kOthers * kRow];
  float lse[kOthers], delta[kOthers];
};

template <int DT>
struct Fetched {
  static constexpr int kChunks = kOthers * 4 * DT, kEach = (kChunks + 255) / 256;
  float4 a[kEach], b[kEach];
  float lse, delta;
};

// rows: how many of the 32 there are; the others come as zeros with lse = inf, whose weight 2^(s - lse) is 0.
template <int DT, bool STATS, typename TA, typename TB>
__device__ __forceinline__ void fetch(Fetched<DT>& f, const TA* a, const TB* b, const float* lse, const float* delta,
                                      int d, int rows, int dh, bool wide) {
#pragma unroll
  for (int e = 0; e < Fetched<DT>::kEach; ++e) {
    const int i = threadIdx.x + 256 * e, r = i / (4 * DT), c = i % (4 * DT) * 4;
    f.a[e] = f.b[e] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (i < Fetched<DT>::kChunks && r < rows) {
      f.a[e] = load_channels(a + int64_t(r) * d, c, dh, wide);
      f.b[e] = load_channels(b + int64_t(r) * d, c, dh, wide);
    }
  }
  if (STATS && threadIdx.x < kOthers) {
    const bool in = int(threadIdx.x) < rows;
    f.lse = in ? lse[threadIdx.x] : __builtin_inff();
    f.delta = in ? delta[threadIdx.x] : 0.f;
  }
}
template <int DT, bool STATS>
__device__ __forceinline__ void put(Others<DT>& o, const Fetched<DT>& f) {
#pragma unroll
  for (int e = 0; e < Fetched<DT>::kEach; ++e) {
    const int i = threadIdx.x + 256 * e, r = i / (4 * DT), c = i % (4 * DT) * 4;
    if (i < Fetched<DT>::kChunks) {
      *reinterpret_cast<float4*>(o.a + r * Others<DT>::kRow + c) = f.a[e];
      *reinterpret_cast<float4*>(o.b + r * Others<DT>::kRow + c) = f.b[e];
    }
  }
  if (STATS && threadIdx.x < kOthers) {
    o.lse[threadIdx.x] = f.lse;
    o.delta[threadIdx.x] = f.delta;
  }
}

// Passes over n rows of the other kind, the next 32 requested while a tile is worked on; every thread of the workgroup
// calls it.  tile(first row of the 16 in LDS, rows left from there).
template <int DT, bool STATS, typename TA, typename TB, typename Tile>
__device__ __forceinline__ void sweep(Others<DT>& o, const TA* a, const TB* b, const float* lse, const float* delta, int d,
                                      int64_t n, int dh, bool wide, Tile tile) {
  Fetched<DT> f;
  auto left = [&](int64_t t) { return n - t < kOthers ? int(n - t) : kOthers; };
  if (n > 0) fetch<DT, STATS>(f, a, b, lse, delta, d, left(0), dh, wide);
  for (int64_t t = 0; t < n; t += kOthers) {
    __syncthreads();
    put<DT, STATS>(o, f);
    __syncthreads();
    const int64_t u = t + kOthers;
    if (u < n) fetch<DT, STATS>(f, a + u * d, b + u * d, lse + u, delta + u, d, left(u), dh, wide);
    const int rows = left(t);
    tile(0, rows);
    if (rows > 16) tile(16, rows - 16);
  }
}

// 16 of the staged rows times the own row of each lane's column: register r of lane 16 g + c is row 4 g + r, own row c.
template <int DT>
__device__ __forceinline__ f32x4 products(const float* rows, const float4 (&own)[DT]) {
  const int g = (threadIdx.x & 63) >> 4, c = threadIdx.x & 15;
  f32x4 s = {0.f, 0.f, 0.f, 0.f}, t = s;       // two chains: half the latency
#pragma unroll
  for (int n = 0; n < DT; ++n) {
    const float4 x = *reinterpret_cast<const float4*>(rows + c * Others<DT>::kRow + 16 * n + 4 * g);
    s = mfma4(x.x, own[n].x, s);
    t = mfma4(x.y, own[n].y, t);
    s = mfma4(x.z, own[n].z, s);
    t = mfma4(x.w, own[n].w, t);
  }
  return s + t;
}
// acc^T[channel][own] += sum over the 16 rows of row[channel] w[row][own]
template <int DT>
__device__ __forceinline__ void add_weighted(f32x4 (&acc)[DT], const float* rows, const f32x4& w) {
  const int g = (threadIdx.x & 63) >> 4, c = threadIdx.x & 15;
#pragma unroll
  for (int n = 0; n < DT; ++n)
#pragma unroll
    for (int r = 0; r < 4; ++r) acc[n] = mfma4(rows[(4 * g + r) * Others<DT>::kRow + 16 * n + c], w[r], acc[n]);
}

template <int DT, typename T>
__device__ __forceinline__ void load_own(float4 (&own)[DT], const T* row, bool in, int dh, bool wide, float times = 1.f) {
  const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int n = 0; n < DT; ++n) {
    own[n] = in ? load_channels(row, 16 * n + 4 * g, dh, wide) : make_float4(0.f, 0.f, 0.f, 0.f);
    own[n].x *= times; own[n].y *= times; own[n].z *= times; own[n].w *= times;
  }
}
template <int DT>
__device__ __forceinline__ void clear(f32x4 (&acc)[DT]) {
#pragma unroll
  for (int n = 0; n < DT; ++n) acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
}

// A query's statistics over the keys a lane has seen: those at rows 4 g + r of every tile.  The four lanes of a query
// keep maxima of their own and are joined at the end.
struct Stats {
  float m, l, e;       // maximum (base 2), sum of 2^(s - m), sum of 2^(s - m) dP
  __device__ __forceinline__ void reset() { m = kLowest; l = e = 0.f; }
  __device__ __forceinline__ void add(f32x4 s, const f32x4& t, int rows) {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int r = 0; r < 4; ++r) s[r] = 4 * g + r < rows ? s[r] : -__builtin_inff();
    const float top = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), m);
    const float f = exp2_fast(m - top);
    l *= f;
    e *= f;
    m = top;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float p = exp2_fast(s[r] - m);
      l += p;
      e = fmaf(p, t[r], e);
    }
  }
  __device__ __forceinline__ void join() {
#pragma unroll
    for (int o = 16; o < 64; o *= 2) {
      const float m2 = __shfl_xor(m, o, 64), l2 = __shfl_xor(l, o, 64), e2 = __shfl_xor(e, o, 64);
      join_stats(m, l, e, m2, l2, e2);
    }
  }
};

// ------------------------------------------------------------------------------------------------ projections
// K = X W_k, V = X W_v in fp32, 64 rows x 64 columns of [K | V] a workgroup.
template <typename T>
__global__ __launch_bounds__(256) void grad_project_kernel(const T* __restrict__ X, const T* __restrict__ Wk,
                                                           const T* __restrict__ Wv, float* __restrict__ K,
                                                           float* __restrict__ V, int64_t N, int d, int64_t row_blocks,
                                                           int col_blocks, bool wide) {
  __shared__ __align__(16) float xs[64 * 36], ws[32 * 68];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, c = lane & 15;
  for (int64_t item = blockIdx.x; item < row_blocks * col_blocks; item += gridDim.x) {
    const int64_t r0 = item / col_blocks * 64;
    const int c0 = int(item % col_blocks) * 64;             // of 2 d columns
    f32x4 acc[4];
    clear(acc);
    for (int k0 = 0; k0 < d; k0 += 32) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int i = threadIdx.x + 256 * e, r = i / 8, k = i % 8 * 4;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r0 + r < N) v = load_channels(X + (r0 + r) * d + k0, k, d - k0, wide);
        *reinterpret_cast<float4*>(xs + r * 36 + k) = v;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int i = threadIdx.x + 256 * e, k = i / 64, n = c0 + i % 64;
        float v = 0.f;
        if (k0 + k < d && n < 2 * d) v = to_f32(n < d ? Wk[int64_t(k0 + k) * d + n] : Wv[int64_t(k0 + k) * d + n - d]);
        ws[k * 68 + i % 64] = v;
      }
      __syncthreads();
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        const float4 x = *reinterpret_cast<const float4*>(xs + (16 * wave + c) * 36 + 16 * a + 4 * g);
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[n] = mfma4(at(x, i), ws[(16 * a + 4 * g + i) * 68 + 16 * n + c], acc[n]);
      }
    }
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int64_t row = r0 + 16 * wave + 4 * g + r;
        const int col = c0 + 16 * n + c;
        if (row < N && col < 2 * d) (col < d ? K : V)[row * d + (col < d ? col : col - d)] = acc[n][r];
      }
  }
}

// ------------------------------------------------------------------------------------------------ stage 1
struct HistoryGrad {
  const void* Q;
  const void* dO;
  const float* K;
  const float* V;
  const int64_t* offsets;
  float* stats;          // [slot][H][S][3]
  const float* lse;      // [B][H][S]
  const float* delta;    // [B][H][S]
  float* records;        // [slot][H][S][dh]: dS K, base of dQ
  void* dK;
  void* dV;
  int64_t q_user_stride, N, G;
  int B, S, d, H, seg, groups;   // groups of 64 queries
  float scale, scale_log2;
  bool wide;             // Q and dO by four elements
  bool wide_kv;          // K, V likewise
};

// Queries' rows over one segment: the statistics of every piece, or (GRAD) its share of dQ.
template <typename T, int DT, bool GRAD>
__device__ __forceinline__ void history_queries(const HistoryGrad& p, Others<DT>& o, int64_t block, int64_t blocks) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, c = lane & 15;
  const int dh = p.d / p.H;
  for (int64_t item = block; item < p.G * p.H * p.groups; item += blocks) {
    const int64_t segment = item / (p.H * p.groups);
    const int rest = int(item % (p.H * p.groups)), h = rest / p.groups;
    const int i = rest % p.groups * kOwn + 16 * wave + c;
    const bool in = i < p.S;
    const int64_t begin = segment * p.seg, end = begin + p.seg < p.N ? begin + p.seg : p.N;
    int user = find_user_wave(p.offsets, p.B, begin);
    int64_t pos = begin;
    Piece pc;
    while (next_piece(p.offsets, p.B, end, user, pos, pc)) {
      const int64_t q_row = int64_t(pc.user) * p.q_user_stride + int64_t(i) * p.d + h * dh;
      const int64_t do_row = (int64_t(pc.user) * p.S + i) * p.d + h * dh;
      const int64_t stat = (int64_t(pc.user) * p.H + h) * p.S + i;
      const int64_t slot = ((segment + pc.user) * p.H + h) * p.S + i;
      float4 q[DT], w[DT];
      load_own<DT>(q, static_cast<const T*>(p.Q) + q_row, in, dh, p.wide, p.scale_log2);
      load_own<DT>(w, static_cast<const T*>(p.dO) + do_row, in, dh, p.wide);
      const float* K = p.K + pc.begin * p.d + h * dh;
      const float* V = p.V + pc.begin * p.d + h * dh;
      if constexpr (!GRAD) {
        Stats st;
        st.reset();
        sweep<DT, false>(o, K, V, nullptr, nullptr, p.d, pc.end - pc.begin, dh, p.wide_kv, [&](int r0, int rows) {
          const f32x4 s = products<DT>(o.a + r0 * Others<DT>::kRow, q), t = products<DT>(o.b + r0 * Others<DT>::kRow, w);
          st.add(s, t, rows);
        });
        st.join();
        if (in && g == 0) {
          p.stats[3 * slot] = st.m;
          p.stats[3 * slot + 1] = st.l;
          p.stats[3 * slot + 2] = st.e;
        }
      } else {
        const float lse = in ? p.lse[stat] : __builtin_inff(), delta = in ? p.delta[stat] : 0.f;
        f32x4 acc[DT];
        clear(acc);
        sweep<DT, false>(o, K, V, nullptr, nullptr, p.d, pc.end - pc.begin, dh, p.wide_kv, [&](int r0, int rows) {
          const f32x4 s = products<DT>(o.a + r0 * Others<DT>::kRow, q), t = products<DT>(o.b + r0 * Others<DT>::kRow, w);
          f32x4 ds;
#pragma unroll
          for (int r = 0; r < 4; ++r) ds[r] = 4 * g + r < rows ? exp2_fast(s[r] - lse) * (t[r] - delta) : 0.f;
          add_weighted<DT>(acc, o.a + r0 * Others<DT>::kRow, ds);
        });
        if (in) {
#pragma unroll
          for (int n = 0; n < DT; ++n) store_channels(p.records + slot * dh, 16 * n + 4 * g, dh, acc[n]);
        }
      }
    }
  }
}

// Items' rows, 64 a workgroup: dK and dV over all seeds of their user.  A block of rows that several users share is passed once
// for each of them, with accumulators of its own, so that nothing of one user reaches another's rows.  K and V may be the
// memory of dK and dV: a wave reads its own rows before it stores them, and nobody else reads them.
template <typename T, int DT>
__device__ __forceinline__ void history_items(const HistoryGrad& p, Others<DT>& o, int64_t block, int64_t blocks) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, c = lane & 15;
  const int dh = p.d / p.H;
  const int64_t row_blocks = (p.N + kOwn - 1) / kOwn;
  for (int64_t item = block; item < row_blocks * p.H; item += blocks) {
    const int64_t begin = item / p.H * kOwn, end = begin + kOwn < p.N ? begin + kOwn : p.N;
    const int h = int(item % p.H);
    const int64_t row = begin + 16 * wave + c;
    const bool in = row < end;
    float4 k[DT], v[DT];
    load_own<DT>(k, p.K + row * p.d + h * dh, in, dh, p.wide_kv, p.scale_log2);
    load_own<DT>(v, p.V + row * p.d + h * dh, in, dh, p.wide_kv);
    int user = find_user_wave(p.offsets, p.B, begin);
    int64_t pos = begin;
    Piece pc;
    while (next_piece(p.offsets, p.B, end, user, pos, pc)) {
      const T* Q = static_cast<const T*>(p.Q) + int64_t(pc.user) * p.q_user_stride + h * dh;
      const T* dO = static_cast<const T*>(p.dO) + int64_t(pc.user) * p.S * p.d + h * dh;
      const int64_t stat = (int64_t(pc.user) * p.H + h) * p.S;
      f32x4 dk[DT], dv[DT];
      clear(dk);
      clear(dv);
      sweep<DT, true>(o, Q, dO, p.lse + stat, p.delta + stat, p.d, p.S, dh, p.wide, [&](int r0, int) {
        const f32x4 s = products<DT>(o.a + r0 * Others<DT>::kRow, k), t = products<DT>(o.b + r0 * Others<DT>::kRow, v);
        f32x4 w, ds;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          w[r] = exp2_fast(s[r] - o.lse[r0 + 4 * g + r]);
          ds[r] = w[r] * (t[r] - o.delta[r0 + 4 * g + r]);
        }
        add_weighted<DT>(dv, o.b + r0 * Others<DT>::kRow, w);
        add_weighted<DT>(dk, o.a + r0 * Others<DT>::kRow, ds);
      });
      if (row >= pc.begin && row < pc.end) {
#pragma unroll
        for (int n = 0; n < DT; ++n) {
          store_channels(static_cast<T*>(p.dK) + row * p.d + h * dh, 16 * n + 4 * g, dh, dk[n] * p.scale);
          store_channels(static_cast<T*>(p.dV) + row * p.d + h * dh, 16 * n + 4 * g, dh, dv[n]);
        }
      }
    }
  }
}

template <typename T, int DT>
__global__ __launch_bounds__(256) void history_stats_kernel(HistoryGrad p) {
  __shared__ __align__(16) Others<DT> o;
  history_queries<T, DT, false>(p, o, blockIdx.x, gridDim.x);
}
// The first `queries` workgroups form dQ, the others dK and dV; with none of one kind it is the other's launch alone.
template <typename T, int DT>
__global__ __launch_bounds__(256) void history_grads_kernel(HistoryGrad p, unsigned queries) {
  __shared__ __align__(16) Others<DT> o;
  if (blockIdx.x < queries)
    history_queries<T, DT, true>(p, o, blockIdx.x, queries);
  else
    history_items<T, DT>(p, o, blockIdx.x - queries, gridDim.x - queries);
}

// ------------------------------------------------------------------------------------------------ stage 2
struct CandidateGrad {
  const void* cand;
  const void* summ;
  const void* dO;
  void* d_cand;
  void* d_summ;
  float* lse;            // [B][H][C]
  float* delta;          // [B][H][C]
  float* records;        // [share][B][H][S][dh], where candidates are shared out
  int64_t B;
  int C, S, d, H, shares, rows_each;   // candidates of a share
  float scale, scale_log2;
  bool self_term, wide;
};

// Sum over the four lanes of an own row of the products of its channels.
template <int DT>
__device__ __forceinline__ float own_dot(const float4 (&a)[DT], const float4 (&b)[DT]) {
  float s = 0.f;
#pragma unroll
  for (int n = 0; n < DT; ++n) s = fmaf(a[n].x, b[n].x, fmaf(a[n].y, b[n].y, fmaf(a[n].z, b[n].z, fmaf(a[n].w, b[n].w, s))));
  s += __shfl_xor(s, 16, 64);
  s += __shfl_xor(s, 32, 64);
  return s;
}

// Candidates' rows, 64 a workgroup: statistics, then dQ, over the user's summaries.
template <typename T, int DT>
__global__ __launch_bounds__(256) void candidate_rows_kernel(CandidateGrad p) {
  __shared__ __align__(16) Others<DT> o;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, c = lane & 15;
  const int dh = p.d / p.H;
  const int64_t groups = (int64_t(p.C) + kOwn - 1) / kOwn, per = p.H * groups;
  for (int64_t item = blockIdx.x; item < p.B * per; item += gridDim.x) {
    const int64_t b = item / per;
    const int h = int(item % per / groups);
    const int64_t i = item % groups * kOwn + 16 * wave + c;
    const bool in = i < p.C;
    const int64_t row = (b * p.C + i) * p.d + h * dh;
    const T* Y = static_cast<const T*>(p.summ) + b * p.S * p.d + h * dh;
    float4 q[DT], w[DT];
    load_own<DT>(q, static_cast<const T*>(p.cand) + row, in, dh, p.wide);
    load_own<DT>(w, static_cast<const T*>(p.dO) + row, in, dh, p.wide);
    float own_s = 0.f, own_t = 0.f;
    if (p.self_term) {
      own_s = own_dot<DT>(q, q) * p.scale_log2;
      own_t = own_dot<DT>(w, q);
    }
    Stats st;
    st.reset();
    auto scores = [&](int r0) { return products<DT>(o.a + r0 * Others<DT>::kRow, q) * p.scale_log2; };
    sweep<DT, false>(o, Y, Y, nullptr, nullptr, p.d, p.S, dh, p.wide, [&](int r0, int rows) {
      st.add(scores(r0), products<DT>(o.a + r0 * Others<DT>::kRow, w), rows);
    });
    st.join();
    if (p.self_term) join_stats(st.m, st.l, st.e, own_s, 1.f, own_t);
    const float lse = st.m + __builtin_amdgcn_logf(st.l), delta = st.e / st.l;
    f32x4 acc[DT];
    clear(acc);
    sweep<DT, false>(o, Y, Y, nullptr, nullptr, p.d, p.S, dh, p.wide, [&](int r0, int rows) {
      const f32x4 s = scores(r0), t = products<DT>(o.a + r0 * Others<DT>::kRow, w);
      f32x4 ds;
#pragma unroll
      for (int r = 0; r < 4; ++r) ds[r] = 4 * g + r < rows ? exp2_fast(s[r] - lse) * (t[r] - delta) : 0.f;
      add_weighted<DT>(acc, o.a + r0 * Others<DT>::kRow, ds);
    });
    if (in) {
      const float pw = p.self_term ? exp2_fast(own_s - lse) : 0.f, ds = 2.f * p.scale * pw * (own_t - delta);
#pragma unroll
      for (int n = 0; n < DT; ++n) {
        f32x4 r = acc[n] * p.scale;
        if (p.self_term) {
#pragma unroll
          for (int e = 0; e < 4; ++e) r[e] += fmaf(ds, at(q[n], e), pw * at(w[n], e));
        }
        store_channels(static_cast<T*>(p.d_cand) + row, 16 * n + 4 * g, dh, r);
      }
      if (g == 0) {
        p.lse[(b * p.H + h) * p.C + i] = lse;
        p.delta[(b * p.H + h) * p.C + i] = delta;
      }
    }
  }
}

// Both gradients where there are at most 128 summaries: their rows fit LDS together, and a wave keeps scores and dP of its 16
// candidates (64 registers), so that each product is formed once.  A workgroup takes a share of one user's head, 64 candidates at a
// time; dY of 64 candidates is formed from dS, then P, of all four waves, which take the summaries' rows dY (accumulators for the
// whole share) lies in turn by 16.  The weights pass through LDS where the summaries' rows were.
constexpr int kShort = 128;
template <typename T, int DT>
__global__ __launch_bounds__(256, 2) void candidates_short_kernel(CandidateGrad p) {
  constexpr int kRow = Others<DT>::kRow, kTiles = kShort / 16, kWeights = kOwn + 4;
  __shared__ __align__(16) float y[kShort * kWeights];            // summaries' rows, then weights [summary][candidate]
  __shared__ __align__(16) float rows[2][kOwn * kRow];            // candidates, d_out
  static_assert(kRow <= kWeights, "summaries' rows fit the weights' place");
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, c = lane & 15;
  const int dh = p.d / p.H, tiles = (p.S + 15) / 16;
  const int64_t per = int64_t(p.H) * p.shares;
  for (int64_t item = blockIdx.x; item < p.B * per; item += gridDim.x) {
    const int64_t b = item / per;
    const int share = int(item % per) / p.H, h = int(item % per) % p.H;
    const int64_t begin = int64_t(share) * p.rows_each, end = begin + p.rows_each < p.C ? begin + p.rows_each : p.C;
    const T* Y = static_cast<const T*>(p.summ) + b * p.S * p.d + h * dh;
    f32x4 dy[2][DT];
    clear(dy[0]);
    clear(dy[1]);
    for (int64_t first = begin; first < end; first += kOwn) {
      const int64_t i = first + 16 * wave + c;
      const bool in = i < end;
      const int64_t row = (b * p.C + i) * p.d + h * dh;
      float4 q[DT], w[DT];
      load_own<DT>(q, static_cast<const T*>(p.cand) + row, in, dh, p.wide);      // zeros beyond the share: nothing for dY
      load_own<DT>(w, static_cast<const T*>(p.dO) + row, in, dh, p.wide);
      __syncthreads();                   // the candidates before have been read
#pragma unroll 4
      for (int n = threadIdx.x; n < tiles * 16 * 4 * DT; n += 256) {
        const int r = n / (4 * DT), ch = n % (4 * DT) * 4;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r < p.S) v = load_channels(Y + int64_t(r) * p.d, ch, dh, p.wide);
        *reinterpret_cast<float4*>(y + r * kRow + ch) = v;
      }
#pragma unroll
      for (int n = 0; n < DT; ++n) {
        *reinterpret_cast<float4*>(rows[0] + (16 * wave + c) * kRow + 16 * n + 4 * g) = q[n];
        *reinterpret_cast<float4*>(rows[1] + (16 * wave + c) * kRow + 16 * n + 4 * g) = w[n];
      }
      float own_s = 0.f, own_t = 0.f;
      if (p.self_term) {
        own_s = own_dot<DT>(q, q) * p.scale_log2;
        own_t = own_dot<DT>(w, q);
      }
      __syncthreads();
      f32x4 s[kTiles], t[kTiles];
      float m = kLowest;
      int left = p.S - 4 * g;
      asm volatile("" : "+v"(left));     // compared here, not once before the loop: 32 masks do not fit the scalar registers
#pragma unroll
      for (int k = 0; k < kTiles; ++k) {
        if (k >= tiles) break;
        s[k] = products<DT>(y + 16 * k * kRow, q) * p.scale_log2;
        t[k] = products<DT>(y + 16 * k * kRow, w);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[k][r] = 16 * k + r < left ? s[k][r] : -__builtin_inff();
          m = fmaxf(m, s[k][r]);
        }
      }
      m = fmaxf(m, __shfl_xor(m, 16, 64));
      m = fmaxf(m, __shfl_xor(m, 32, 64));
      if (p.self_term) m = fmaxf(m, own_s);
      float l = 0.f, e = 0.f;
#pragma unroll
      for (int k = 0; k < kTiles; ++k) {
        if (k >= tiles) break;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[k][r] = exp2_fast(s[k][r] - m);
          l += s[k][r];
          e = fmaf(s[k][r], t[k][r], e);
        }
      }
#pragma unroll
      for (int o = 16; o < 64; o *= 2) {
        l += __shfl_xor(l, o, 64);
        e += __shfl_xor(e, o, 64);
      }
      const float own_w = p.self_term ? exp2_fast(own_s - m) : 0.f;
      l += own_w;
      e = fmaf(own_w, own_t, e);
      const float over = 1.f / l, delta = e * over;
      f32x4 acc[DT];
      clear(acc);
#pragma unroll
      for (int k = 0; k < kTiles; ++k) {
        if (k >= tiles) break;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[k][r] *= over;                // 0 beyond S, and dP there is 0 as well
          t[k][r] = s[k][r] * (t[k][r] - delta) * p.scale;
        }
        add_weighted<DT>(acc, y + 16 * k * kRow, t[k]);
      }
      if (in) {
        const float pw = own_w * over, ds = 2.f * p.scale * pw * (own_t - delta);
#pragma unroll
        for (int n = 0; n < DT; ++n) {
          f32x4 r = acc[n];
          if (p.self_term) {
#pragma unroll
            for (int k = 0; k < 4; ++k) r[k] += fmaf(ds, at(q[n], k), pw * at(w[n], k));
          }
          store_channels(static_cast<T*>(p.d_cand) + row, 16 * n + 4 * g, dh, r);
        }
      }
      // dY[summary][channel] += weights[summary][candidate] rows[candidate][channel]
      auto add = [&](const f32x4 (&v)[kTiles], const float* of) __attribute__((always_inline)) {
        __syncthreads();                 // what lies there has been read
#pragma unroll
        for (int k = 0; k < kTiles; ++k) {
          if (k >= tiles) break;
#pragma unroll
          for (int r = 0; r < 4; ++r) y[(16 * k + 4 * g + r) * kWeights + 16 * wave + c] = v[k][r];
        }
        __syncthreads();
        if (wave >= tiles) return;
        const bool both = wave + 4 < tiles;
        const float* mine = y + (16 * wave + c) * kWeights + 4 * g;
#pragma unroll
        for (int j = 0; j < kOwn / 16; ++j) {
          const float4 a = *reinterpret_cast<const float4*>(mine + 16 * j);
          float4 a2 = a;
          if (both) a2 = *reinterpret_cast<const float4*>(mine + 64 * kWeights + 16 * j);
#pragma unroll
          for (int n = 0; n < DT; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float x = of[(16 * j + 4 * g + r) * kRow + 16 * n + c];
              dy[0][n] = mfma4(at(a, r), x, dy[0][n]);
              if (both) dy[1][n] = mfma4(at(a2, r), x, dy[1][n]);
            }
        }
      };
      add(t, rows[0]);
      add(s, rows[1]);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int n = 0; n < DT; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int i = 16 * (wave + 4 * k) + 4 * g + r, ch = 16 * n + c;
          if (i >= p.S || ch >= dh) continue;
          if (p.shares == 1)
            store_grad(static_cast<T*>(p.d_summ) + (b * p.S + i) * p.d + h * dh + ch, dy[k][n][r]);
          else
            p.records[(((int64_t(share) * p.B + b) * p.H + h) * p.S + i) * dh + ch] = dy[k][n][r];
        }
  }
}

// Summaries' rows, 64 a workgroup, over one share of the user's candidates.  Summaries are keys and values: both parts of
// their gradient go to one accumulator.
template <typename T, int DT>
__global__ __launch_bounds__(256) void summary_rows_kernel(CandidateGrad p) {
  __shared__ __align__(16) Others<DT> o;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, c = lane & 15;
  const int dh = p.d / p.H, groups = (p.S + kOwn - 1) / kOwn;
  const int64_t per = int64_t(p.shares) * p.H * groups;
  for (int64_t item = blockIdx.x; item < p.B * per; item += gridDim.x) {
    const int64_t b = item / per;
    const int64_t rest = item % per;
    const int share = int(rest / (int64_t(p.H) * groups)), h = int(rest / groups % p.H);
    const int i = int(rest % groups) * kOwn + 16 * wave + c;
    const bool in = i < p.S;
    const int64_t first = int64_t(share) * p.rows_each, n = p.C - first < p.rows_each ? p.C - first : p.rows_each;
    const int64_t cand = (b * p.C + first) * p.d + h * dh, stat = (b * p.H + h) * p.C + first;
    const int64_t row = (b * p.S + i) * p.d + h * dh;
    float4 y[DT];
    load_own<DT>(y, static_cast<const T*>(p.summ) + row, in, dh, p.wide);
    f32x4 acc[DT];
    clear(acc);
    sweep<DT, true>(o, static_cast<const T*>(p.cand) + cand, static_cast<const T*>(p.dO) + cand, p.lse + stat, p.delta + stat,
                    p.d, n, dh, p.wide, [&](int r0, int) {
      const f32x4 s = products<DT>(o.a + r0 * Others<DT>::kRow, y) * p.scale_log2;
      const f32x4 t = products<DT>(o.b + r0 * Others<DT>::kRow, y);
      f32x4 w, ds;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        w[r] = exp2_fast(s[r] - o.lse[r0 + 4 * g + r]);
        ds[r] = w[r] * (t[r] - o.delta[r0 + 4 * g + r]) * p.scale;
      }
      add_weighted<DT>(acc, o.b + r0 * Others<DT>::kRow, w);
      add_weighted<DT>(acc, o.a + r0 * Others<DT>::kRow, ds);
    });
    if (in) {
#pragma unroll
      for (int k = 0; k < DT; ++k) {
        if (p.shares == 1)
          store_channels(static_cast<T*>(p.d_summ) + row, 16 * k + 4 * g, dh, acc[k]);
        else
          store_channels(p.records + (((int64_t(share) * p.B + b) * p.H + h) * p.S + i) * dh, 16 * k + 4 * g, dh, acc[k]);
      }
    }
  }
}

constexpr int64_t kMostBlocks = 1 << 20;
unsigned grid_of(int64_t items) { return unsigned(items < kMostBlocks ? items : kMostBlocks); }

bool aligned_to(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// The launches of stage 1: statistics, both gradients together (the projections lie apart from the outputs), dQ alone, dK and dV
// alone.
enum class Step { kStats, kBoth, kQueries, kItems };
template <typename T, int DT>
hipError_t run_history(const HistoryGrad& p, Step step, hipStream_t s) {
  const unsigned queries = grid_of(p.G * p.H * p.groups), items = grid_of((p.N + kOwn - 1) / kOwn * p.H);
  const dim3 block(256);
  switch (step) {
    case Step::kStats: return launch(history_stats_kernel<T, DT>, dim3(queries), block, 0, s, p);
    case Step::kBoth: return launch(history_grads_kernel<T, DT>, dim3(queries + items), block, 0, s, p, queries);
    case Step::kQueries: return launch(history_grads_kernel<T, DT>, dim3(queries), block, 0, s, p, queries);
    default: return launch(history_grads_kernel<T, DT>, dim3(items), block, 0, s, p, 0u);
  }
}
template <typename T>
hipError_t history_step(const HistoryGrad& p, Step step, hipStream_t s) {
  switch ((p.d / p.H + 15) / 16) {
    case 1: return run_history<T, 1>(p, step, s);
    case 2: return run_history<T, 2>(p, step, s);
    case 3: return run_history<T, 3>(p, step, s);
    default: return run_history<T, 4>(p, step, s);
  }
}

template <typename T, int DT>
hipError_t run_candidates(const CandidateGrad& p, int step, hipStream_t s) {
  const int64_t rows = p.B * p.H * ((int64_t(p.C) + kOwn - 1) / kOwn), summ = p.B * p.H * p.shares * ((p.S + kOwn - 1) / kOwn);
  if (p.S <= kShort)
    return step == 0 ? launch(candidates_short_kernel<T, DT>, dim3(grid_of(p.B * p.H * p.shares)), dim3(256), 0, s, p) : hipSuccess;
  if (step == 0) return launch(candidate_rows_kernel<T, DT>, dim3(grid_of(rows)), dim3(256), 0, s, p);
  return launch(summary_rows_kernel<T, DT>, dim3(grid_of(summ)), dim3(256), 0, s, p);
}
template <typename T>
hipError_t candidates_step(const CandidateGrad& p, int step, hipStream_t s) {
  switch ((p.d / p.H + 15) / 16) {
    case 1: return run_candidates<T, 1>(p, step, s);
    case 2: return run_candidates<T, 2>(p, step, s);
    case 3: return run_candidates<T, 3>(p, step, s);
    default: return run_candidates<T, 4>(p, step, s);
  }
}

size_t align256(size_t v) { return (v + 255) & ~size_t(255); }

// Shares of a user's candidates in the summaries' pass: so many that some 1024 workgroups have work, or the 512 that run at a time
// where one pass does everything, 64 candidates or more each.
int candidate_shares(const vista_attend_desc& d) {
  const bool one = d.S <= kShort;
  const int64_t base = int64_t(d.B) * d.H * (one ? 1 : (d.S + kOwn - 1) / kOwn), most = (int64_t(d.C) + kOwn - 1) / kOwn;
  const int64_t want = ((one ? 512 : 1024) + base - 1) / base;
  return int(want < most ? want : most);
}

}  // namespace

// ------------------------------------------------------------------------------------------------ stage 1, host side

// Segments of the queries' passes where the caller leaves their size open: some 1024 workgroups of (segment, head, 64 queries),
// 64 to 4096 items each.
int f32_grad_segment(const vista_summarize_desc& d) {
  if (d.segment_items > 0) return d.segment_items;
  const int64_t each = int64_t(d.H) * ((d.S + kOwn - 1) / kOwn), want = (1024 + each - 1) / each;
  int64_t seg = ((d.total_items + want - 1) / want + 31) / 32 * 32;
  return int(seg < 64 ? 64 : seg > 4096 ? 4096 : seg);
}

namespace {
// The fp32 projections of the items: in the workspace, so that dQ and dK, dV are one launch (a small call is all latency), or, for
// fp32 histories of more than 64 MiB of keys, in the memory of the outputs until the items' pass overwrites them.
bool projections_apart(const vista_summarize_desc& d) {
  return d.dtype != VISTA_F32 || d.total_items * d.d <= (int64_t(64) << 20) / 4;
}
struct HistoryLayout {
  size_t stats, records, rows, self, K, V, Ks, total;   // byte offsets into the workspace
};
HistoryLayout history_layout(const vista_summarize_desc& d) {
  const int64_t seg = f32_grad_segment(d), G = (d.total_items + seg - 1) / seg;
  const size_t slots = size_t(G + d.B) * d.H * d.S, rows = size_t(d.B) * d.H * d.S;
  const size_t kv = projections_apart(d) ? align256(size_t(d.total_items) * d.d * sizeof(float)) : 0;
  HistoryLayout l;
  l.stats = kHeaderBytes;
  l.records = l.stats + align256(slots * 3 * sizeof(float));
  l.rows = l.records + align256(slots * (d.d / d.H) * sizeof(float));
  l.self = l.rows + 2 * align256(rows * sizeof(float));
  l.K = l.self + ((d.flags & VISTA_FLAG_SELF_TERM) ? 2 * align256(rows * sizeof(float)) : 0);
  l.V = l.K + kv;
  l.Ks = l.V + kv;
  l.total = l.Ks + 2 * self_kv_bytes(d);
  return l;
}
}  // namespace

size_t f32_summarize_backward_workspace(const vista_summarize_desc& d) { return history_layout(d).total; }

vista_status f32_summarize_backward(const SummarizeArgs& a, const void* d_out, void* d_queries, void* d_keys, void* d_values,
                                    void* d_self_keys, void* d_self_values) {
  const vista_summarize_desc& d = a.desc;
  const HistoryLayout l = history_layout(d);
  const size_t e = d.dtype == VISTA_F32 ? 4 : 2;
  const int dh = d.d / d.H;
  const size_t rows = size_t(d.B) * d.H * d.S;
  auto floats = [&](size_t off) { return reinterpret_cast<float*>(a.workspace + off); };
  HistoryGrad p;
  p.Q = a.Q;
  p.dO = d_out;
  const bool apart = projections_apart(d);
  float* K = apart ? floats(l.K) : static_cast<float*>(d_keys);
  float* V = apart ? floats(l.V) : static_cast<float*>(d_values);
  p.K = K;
  p.V = V;
  p.offsets = a.offsets;
  p.stats = floats(l.stats);
  float* lse = floats(l.rows);
  float* delta = lse + align256(rows * sizeof(float)) / sizeof(float);
  p.lse = lse;
  p.delta = delta;
  p.records = floats(l.records);
  p.dK = d_keys;
  p.dV = d_values;
  p.q_user_stride = d.q_user_stride;
  p.N = d.total_items;
  p.G = a.G;
  p.B = d.B;
  p.S = d.S;
  p.d = d.d;
  p.H = d.H;
  p.seg = a.seg;
  p.groups = (d.S + kOwn - 1) / kOwn;
  p.scale = a.scale_plain;
  p.scale_log2 = a.scale_log2;
  p.wide = dh % 4 == 0 && aligned_to(a.Q, 4 * e) && aligned_to(d_out, 4 * e);
  p.wide_kv = dh % 4 == 0 && aligned_to(K, 16) && aligned_to(V, 16);
  const bool bf16 = d.dtype == VISTA_BF16;
  auto step = [&](Step n) { return bf16 ? history_step<bf16_t>(p, n, a.stream) : history_step<float>(p, n, a.stream); };

  float *Ks = nullptr, *Vs = nullptr, *own_p = nullptr, *own_ds = nullptr;
  if (d.flags & VISTA_FLAG_SELF_TERM) {
    Ks = floats(l.Ks);
    Vs = Ks + self_kv_bytes(d) / sizeof(float);
    own_p = floats(l.self);
    own_ds = own_p + align256(rows * sizeof(float)) / sizeof(float);
    if (launch_self_kv(d, a.Q, a.Wk, a.Wv, Ks, Vs, a.stream) != hipSuccess) return VISTA_ERR_HIP;
  }
  if (p.N > 0) {
    const int64_t row_blocks = (p.N + 63) / 64;
    const int col_blocks = (2 * d.d + 63) / 64;
    const unsigned grid = grid_of(row_blocks * col_blocks);
    const bool wide = d.d % 4 == 0 && aligned_to(a.X, 4 * e);
    if (bf16)
      VISTA_LAUNCH(grad_project_kernel<bf16_t>, dim3(grid), dim3(256), 0, a.stream, static_cast<const bf16_t*>(a.X),
                   static_cast<const bf16_t*>(a.Wk), static_cast<const bf16_t*>(a.Wv), K, V, p.N, d.d, row_blocks, col_blocks,
                   wide);
    else
      VISTA_LAUNCH(grad_project_kernel<float>, dim3(grid), dim3(256), 0, a.stream, static_cast<const float*>(a.X),
                   static_cast<const float*>(a.Wk), static_cast<const float*>(a.Wv), K, V, p.N, d.d, row_blocks, col_blocks,
                   wide);
    if (step(Step::kStats) != hipSuccess) return VISTA_ERR_HIP;
  }
  const GradRows r = {a.offsets, d.B, d.S, d.d, d.H, a.seg, d.total_items, a.G, a.scale_plain, a.scale_log2, d.q_user_stride,
                      a.offsets_checked ? -1 : d.total_items, reinterpret_cast<int*>(a.workspace)};
  if (grad_join_stats(r, d.dtype, p.stats, d.S, lse, delta, a.Q, d_out, Ks, Vs, own_p, own_ds, a.stream) != hipSuccess)
    return VISTA_ERR_HIP;
  if (p.N > 0 && (apart ? step(Step::kBoth) != hipSuccess
                        : step(Step::kQueries) != hipSuccess || step(Step::kItems) != hipSuccess))
    return VISTA_ERR_HIP;
  if (grad_join_queries(r, d.dtype, p.records, d.S, a.scale_plain, a.Q, d_out, Ks, own_p, own_ds, d_queries, d_self_keys, d_self_values,
                        a.stream) != hipSuccess)
    return VISTA_ERR_HIP;
  return VISTA_OK;
}

// ------------------------------------------------------------------------------------------------ stage 2, host side

size_t f32_attend_backward_workspace(const vista_attend_desc& d) {
  const size_t shares = candidate_shares(d), rows = d.S <= kShort ? 1 : size_t(d.B) * d.H * d.C;
  return 2 * align256(rows * sizeof(float)) + (shares > 1 ? align256(shares * d.B * d.S * d.d * sizeof(float)) : 0);
}

vista_status f32_attend_backward(const vista_attend_desc& d, float scale, const void* cand, const void* summ, const void* d_out,
                                 void* d_cand, void* d_summ, void* workspace, hipStream_t s) {
  const size_t e = d.dtype == VISTA_F32 ? 4 : 2, rows = d.S <= kShort ? 1 : size_t(d.B) * d.H * d.C;
  const int dh = d.d / d.H, unit = d.S <= kShort ? kOwn : kOthers;
  CandidateGrad p;
  p.cand = cand;
  p.summ = summ;
  p.dO = d_out;
  p.d_cand = d_cand;
  p.d_summ = d_summ;
  p.lse = static_cast<float*>(workspace);
  p.delta = p.lse + align256(rows * sizeof(float)) / sizeof(float);
  p.records = p.delta + align256(rows * sizeof(float)) / sizeof(float);
  p.B = d.B;
  p.C = d.C;
  p.S = d.S;
  p.d = d.d;
  p.H = d.H;
  p.shares = candidate_shares(d);
  p.rows_each = int(((int64_t(d.C) + p.shares - 1) / p.shares + unit - 1) / unit * unit);
  p.shares = int((int64_t(d.C) + p.rows_each - 1) / p.rows_each);
  p.scale = scale;
  p.scale_log2 = scale * kLog2e;
  p.self_term = (d.flags & VISTA_FLAG_SELF_TERM) != 0;
  p.wide = dh % 4 == 0 && aligned_to(cand, 4 * e) && aligned_to(summ, 4 * e) && aligned_to(d_out, 4 * e);
  const bool bf16 = d.dtype == VISTA_BF16;
  for (int n = 0; n < 2; ++n)
    if ((bf16 ? candidates_step<bf16_t>(p, n, s) : candidates_step<float>(p, n, s)) != hipSuccess) return VISTA_ERR_HIP;
  if (p.shares > 1 && grad_join_shares(d.dtype, p.records, p.shares, int64_t(d.B), d.S, d.d, d.H, d_summ, s) != hipSuccess)
    return VISTA_ERR_HIP;
  return VISTA_OK;
}

}  // namespace vista
