// Layer norm of rows and its gradients, gfx950.
//
//   z = (x - mean) r,  r = 1 / sqrt(mean((x - mean)^2) + eps),  y = z w + b
//   g = dy w,  dx = r (g - mean(g) - z mean(g z)),  dw = sum over rows dy z,  db = sum over rows dy
//
// Both directions read every row once and keep it in registers: the mean, then the squared deviations
// from it (two passes over registers, so a large common offset costs no digits), all in fp32; the
// gradients form mean and r again from the row they read anyway, so nothing is saved between the two.
// A row is held by a group of lanes, a chunk of up to 16 bytes a lane (a row of 128 bf16 by 16 lanes, four
// rows a wave), so that every load of a wave is one run of memory.  Bound by HBM:
// 768597 x 128 bf16 in 72.9 us forward (5.4 TB/s) and 111.6 backward (5.3 TB/s); a copy of 2 GiB reaches 4.9 TB/s.  Rows that are not
// whole aligned chunks: 450875 x 211 in 80 and 129 us (4.8 and 4.5 TB/s).
// The weight's and bias's gradients are added up in the lanes that own their channels, over all rows of a
// workgroup, which writes one partial row of each; a second kernel adds these in a fixed order.
#include "common.hpp"
#include "grad.hpp"

namespace vista {
namespace {

constexpr int kNormThreads = 256;
constexpr int kNormWaves = kNormThreads / 64;
constexpr int kNormGroups = 1024;      // most partial rows of the gradients: four workgroups a compute unit

// A chunk as one load or store of 16 bytes (of one element where VEC is 1).  ALIGN is what the address is a multiple of:
// global memory takes any multiple of the element.
template <typename T, int VEC, int ALIGN>
__device__ __forceinline__ void load_chunk(const T* p, float (&out)[VEC]) {
  struct __attribute__((packed, aligned(ALIGN))) Raw { T v[VEC]; };
  const Raw r = *reinterpret_cast<const Raw*>(p);
#pragma unroll
  for (int e = 0; e < VEC; ++e) out[e] = to_f32(r.v[e]);
}
template <int VEC, int ALIGN>
__device__ __forceinline__ void store_chunk(float* p, const float (&v)[VEC]) {
  struct __attribute__((packed, aligned(ALIGN))) Raw { float v[VEC]; } r;
#pragma unroll
  for (int e = 0; e < VEC; ++e) r.v[e] = v[e];
  *reinterpret_cast<Raw*>(p) = r;
}
template <int VEC, int ALIGN>
__device__ __forceinline__ void store_chunk(bf16_t* p, const float (&v)[VEC]) {
  if constexpr (VEC == 1) {
    p->bits = uint16_t(pair_to_bf16(v[0], 0.f));
  } else {
    struct __attribute__((packed, aligned(ALIGN))) Raw { uint32_t v[VEC / 2]; } r;
#pragma unroll
    for (int e = 0; e < VEC / 2; ++e) r.v[e] = pair_to_bf16(v[2 * e], v[2 * e + 1]);
    *reinterpret_cast<Raw*>(p) = r;
  }
}

// Sum over the LPR lanes of a group, in every lane of it: within 16 lanes by data-parallel moves (a
// vector instruction each), beyond by a read across lanes.
template <int CTRL>
__device__ __forceinline__ float moved(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, false));
}
template <int LPR>
__device__ __forceinline__ float group_sum(float v) {
  if (LPR > 1) v += moved<0xB1>(v);      // quad_perm [1, 0, 3, 2]
  if (LPR > 2) v += moved<0x4E>(v);      // quad_perm [2, 3, 0, 1]
  if (LPR > 4) v += moved<0x141>(v);     // the half row mirrored
  if (LPR > 8) v += moved<0x140>(v);     // the row mirrored
  if (LPR > 16) v += __shfl_xor(v, 16, 64);
  if (LPR > 32) v += __shfl_xor(v, 32, 64);
  return v;
}

// LPR lanes a row, CPL chunks of VEC elements a lane: chunk lane + LPR j of the row, j < CPL.  WHOLE: rows are whole chunks at
// aligned addresses.  Otherwise the row's last chunk is its last VEC elements; those that the chunk before holds as well count
// once in sums and are stored twice, alike.
template <typename T, int VEC, int LPR, int CPL, bool WHOLE>
struct Row {
  static constexpr int kAlign = WHOLE ? VEC * sizeof(T) : sizeof(T);
  float v[CPL][VEC];
  static __device__ __forceinline__ bool in(int at, int j, int d) { return (at + LPR * j) * VEC < d; }
  static __device__ __forceinline__ int first(int at, int j, int d) {
    const int c = (at + LPR * j) * VEC;
    return WHOLE || c + VEC <= d ? c : d - VEC;
  }
  // whether element e of a chunk that is in the row is its own
  static __device__ __forceinline__ bool own(int at, int j, int e, int d) {
    return WHOLE || first(at, j, d) + e >= (at + LPR * j) * VEC;
  }
  __device__ __forceinline__ void load(const T* row, int at, int d) {
#pragma unroll
    for (int j = 0; j < CPL; ++j) {
      if (in(at, j, d)) {
        load_chunk<T, VEC, kAlign>(row + first(at, j, d), v[j]);
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[j][e] = 0.f;
      }
    }
  }
  __device__ __forceinline__ void store(T* row, int at, int d) const {
#pragma unroll
    for (int j = 0; j < CPL; ++j)
      if (in(at, j, d)) store_chunk<VEC, kAlign>(row + first(at, j, d), v[j]);
  }
  // v -> z; returns r.  Lanes beyond the row's end hold zeros before and after.
  __device__ __forceinline__ float normalise(int at, int d, float inv_d, float eps) {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < CPL; ++j)
#pragma unroll
      for (int e = 0; e < VEC; ++e) s += own(at, j, e, d) ? v[j][e] : 0.f;
    const float mean = group_sum<LPR>(s) * inv_d;
    float q = 0.f;
#pragma unroll
    for (int j = 0; j < CPL; ++j) {
      const bool inside = in(at, j, d);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        v[j][e] = inside ? v[j][e] - mean : 0.f;
        const float x = own(at, j, e, d) ? v[j][e] : 0.f;
        q = fmaf(x, x, q);
      }
    }
    // v_rsq_f32 is within one unit of the last place
    const float r = __builtin_amdgcn_rsqf(fmaf(group_sum<LPR>(q), inv_d, eps));
#pragma unroll
    for (int j = 0; j < CPL; ++j)
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[j][e] *= r;
    return r;
  }
};

struct NormParams {
  const void* x;
  const void* w;
  const void* b;
  const void* dy;
  void* out;            // y, or dx
  float* partials;      // [groups][2][d], null: no gradients of weight and bias wanted
  int64_t rows;
  int d;
  float eps;
};

template <typename T, int VEC, int LPR, int CPL, bool WHOLE>
__global__ __launch_bounds__(kNormThreads) void norm_kernel(NormParams p) {
  constexpr int kRows = 64 / LPR;        // rows a wave holds
  const int lane = threadIdx.x & 63, at = lane % LPR, sub = lane / LPR;
  const T* X = static_cast<const T*>(p.x);
  T* Y = static_cast<T*>(p.out);
  const float inv_d = 1.f / float(p.d);
  using R = Row<T, VEC, LPR, CPL, WHOLE>;
  R w, b;
  if (p.w) w.load(static_cast<const T*>(p.w), at, p.d);
  if (p.b) b.load(static_cast<const T*>(p.b), at, p.d);
  const int64_t stride = int64_t(gridDim.x) * kNormWaves * kRows;
  for (int64_t r = (int64_t(blockIdx.x) * kNormWaves + (threadIdx.x >> 6)) * kRows + sub; r < p.rows; r += stride) {
    R x;
    x.load(X + r * p.d, at, p.d);
    x.normalise(at, p.d, inv_d, p.eps);
#pragma unroll
    for (int j = 0; j < CPL; ++j)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        float y = x.v[j][e];
        if (p.w) y *= w.v[j][e];
        if (p.b) y += b.v[j][e];
        x.v[j][e] = y;
      }
    x.store(Y + r * p.d, at, p.d);
  }
}

template <typename T, int VEC, int LPR, int CPL, bool WHOLE>
__global__ __launch_bounds__(kNormThreads) void norm_backward_kernel(NormParams p) {
  constexpr int kRows = 64 / LPR;
  const int lane = threadIdx.x & 63, at = lane % LPR, sub = lane / LPR;
  const int wave = threadIdx.x >> 6;
  const T* X = static_cast<const T*>(p.x);
  const T* DY = static_cast<const T*>(p.dy);
  T* DX = static_cast<T*>(p.out);
  const float inv_d = 1.f / float(p.d);
  using R = Row<T, VEC, LPR, CPL, WHOLE>;
  R w;
  if (p.w) w.load(static_cast<const T*>(p.w), at, p.d);
  float dw[CPL][VEC] = {}, db[CPL][VEC] = {};
  const int64_t stride = int64_t(gridDim.x) * kNormWaves * kRows;
  for (int64_t r = (int64_t(blockIdx.x) * kNormWaves + wave) * kRows + sub; r < p.rows; r += stride) {
    R x, g;
    x.load(X + r * p.d, at, p.d);
    g.load(DY + r * p.d, at, p.d);
    const float rs = x.normalise(at, p.d, inv_d, p.eps);
    float s = 0.f, t = 0.f;
#pragma unroll
    for (int j = 0; j < CPL; ++j)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        dw[j][e] = fmaf(g.v[j][e], x.v[j][e], dw[j][e]);
        db[j][e] += g.v[j][e];
        if (p.w) g.v[j][e] *= w.v[j][e];
        const float u = R::own(at, j, e, p.d) ? g.v[j][e] : 0.f;
        s += u;
        t = fmaf(u, x.v[j][e], t);
      }
    s = group_sum<LPR>(s) * inv_d;
    t = group_sum<LPR>(t) * inv_d;
#pragma unroll
    for (int j = 0; j < CPL; ++j)
#pragma unroll
      for (int e = 0; e < VEC; ++e) g.v[j][e] = rs * (g.v[j][e] - fmaf(x.v[j][e], t, s));
    g.store(DX + r * p.d, at, p.d);
  }
  if (!p.partials) return;
  // the rows of a wave, then its waves in ascending order
  __shared__ float sums[kNormWaves][2][LPR * CPL * VEC];
#pragma unroll
  for (int j = 0; j < CPL; ++j)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
#pragma unroll
      for (int o = LPR; o < 64; o *= 2) {
        dw[j][e] += __shfl_xor(dw[j][e], o, 64);
        db[j][e] += __shfl_xor(db[j][e], o, 64);
      }
      if (sub == 0 && R::in(at, j, p.d) && R::own(at, j, e, p.d)) {
        sums[wave][0][R::first(at, j, p.d) + e] = dw[j][e];
        sums[wave][1][R::first(at, j, p.d) + e] = db[j][e];
      }
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * p.d; i += kNormThreads) {
    const int which = i >= p.d, c = i - which * p.d;
    float v = sums[0][which][c];
#pragma unroll
    for (int k = 1; k < kNormWaves; ++k) v += sums[k][which][c];
    p.partials[int64_t(blockIdx.x) * 2 * p.d + i] = v;
  }
}

// Columns of the partial rows: 16 columns a workgroup, 64 threads a column, each an ascending run of every 64th row, the runs
// added in ascending order.  (16 threads a column: 7.8 us for 1024 rows of 512 columns, 64: 4.9; latency.)
constexpr int kRuns = 64;
template <typename T>
__global__ __launch_bounds__(16 * kRuns) void norm_columns_kernel(const float* __restrict__ partials, int groups, int d,
                                                                 T* __restrict__ d_weight, T* __restrict__ d_bias) {
  __shared__ float part[kRuns][17];
  const int c = threadIdx.x & 15, k = threadIdx.x >> 4;
  const int col = blockIdx.x * 16 + c;
  float s = 0.f;
  if (col < 2 * d) {
#pragma unroll 8
    for (int g = k; g < groups; g += kRuns) s += partials[int64_t(g) * 2 * d + col];
  }
  part[k][c] = s;
  __syncthreads();
  if (k == 0 && col < 2 * d) {
#pragma unroll 16
    for (int i = 1; i < kRuns; ++i) s += part[i][c];
    T* out = col < d ? d_weight : d_bias;
    if (out) store_chunk<1, sizeof(T)>(out + (col < d ? col : col - d), {s});
  }
}

// Whether a row is whole chunks of 16 bytes at addresses that are multiples of 16.
bool norm_whole(int dtype, int d, const void* const (&ptrs)[4]) {
  uintptr_t low = 0;
  for (const void* q : ptrs) low |= reinterpret_cast<uintptr_t>(q);
  return d * (dtype == VISTA_BF16 ? 2 : 4) % 16 == 0 && (low & 15) == 0;
}
// Elements of a chunk: 16 bytes, unless the row has fewer.
int norm_vector(int dtype, int d) {
  const int vec = dtype == VISTA_BF16 ? 8 : 4;
  return d < vec ? 1 : vec;
}

int norm_lanes(int d, int vec) {
  const int chunks = (d + vec - 1) / vec;
  return chunks <= 8 ? 8 : chunks <= 16 ? 16 : chunks <= 32 ? 32 : 64;
}

unsigned norm_grid(int64_t rows, int lanes, int most) {
  const int64_t per = kNormWaves * (64 / lanes);
  const int64_t need = (rows + per - 1) / per;
  return unsigned(need < most ? need : most);
}

template <typename T, int VEC, int LPR, int CPL, bool WHOLE>
hipError_t run_norm(const NormParams& p, bool backward, unsigned grid, hipStream_t s) {
  return backward ? launch(norm_backward_kernel<T, VEC, LPR, CPL, WHOLE>, dim3(grid), dim3(kNormThreads), 0, s, p)
                  : launch(norm_kernel<T, VEC, LPR, CPL, WHOLE>, dim3(grid), dim3(kNormThreads), 0, s, p);
}

// CPL for widths up to kNormMaxWidth = 1024: 128 chunks of bf16, 256 of fp32
template <typename T, int VEC, bool WHOLE>
hipError_t pick_norm(const NormParams& p, bool backward, unsigned grid, int lanes, hipStream_t s) {
  const int chunks = (p.d + VEC - 1) / VEC;
  if (lanes == 8) return run_norm<T, VEC, 8, 1, WHOLE>(p, backward, grid, s);
  if (lanes == 16) return run_norm<T, VEC, 16, 1, WHOLE>(p, backward, grid, s);
  if (lanes == 32) return run_norm<T, VEC, 32, 1, WHOLE>(p, backward, grid, s);
  if (chunks <= 64) return run_norm<T, VEC, 64, 1, WHOLE>(p, backward, grid, s);
  if (chunks <= 128) return run_norm<T, VEC, 64, 2, WHOLE>(p, backward, grid, s);
  if constexpr (VEC == 4) {
    if (chunks <= 256) return run_norm<T, VEC, 64, 4, WHOLE>(p, backward, grid, s);
  }
  return hipErrorInvalidValue;
}

template <typename T>
hipError_t dispatch_norm(const NormParams& p, int vec, bool whole, bool backward, unsigned grid, int lanes, hipStream_t s) {
  constexpr int kVec = 16 / sizeof(T);
  return vec == 1 ? run_norm<T, 1, 8, 1, true>(p, backward, grid, s)
         : whole  ? pick_norm<T, kVec, true>(p, backward, grid, lanes, s)
                  : pick_norm<T, kVec, false>(p, backward, grid, lanes, s);
}

}  // namespace

vista_status layer_norm(const vista_norm_desc& d, float eps, const void* x, const void* w, const void* b, void* y,
                        hipStream_t s) {
  if (d.rows == 0) return VISTA_OK;
  const int vec = norm_vector(d.dtype, d.d), lanes = norm_lanes(d.d, vec);
  const bool whole = norm_whole(d.dtype, d.d, {x, w, b, y});
  const NormParams p = {x, w, b, nullptr, y, nullptr, d.rows, d.d, eps};
  const unsigned grid = norm_grid(d.rows, lanes, 8 * 256);
  const hipError_t e = d.dtype == VISTA_BF16 ? dispatch_norm<bf16_t>(p, vec, whole, false, grid, lanes, s)
                                             : dispatch_norm<float>(p, vec, whole, false, grid, lanes, s);
  return e == hipSuccess ? VISTA_OK : VISTA_ERR_HIP;
}

size_t layer_norm_backward_workspace(const vista_norm_desc& d) {
  return size_t(kNormGroups) * 2 * d.d * sizeof(float);
}

vista_status layer_norm_backward(const vista_norm_desc& d, float eps, const void* x, const void* w, const void* dy,
                                 void* dx, void* dw, void* db, void* workspace, hipStream_t s) {
  const int vec = norm_vector(d.dtype, d.d), lanes = norm_lanes(d.d, vec);
  const bool whole = norm_whole(d.dtype, d.d, {x, w, dy, dx});
  const bool sums = dw || db;
  const NormParams p = {x, w, nullptr, dy, dx, sums ? static_cast<float*>(workspace) : nullptr, d.rows, d.d, eps};
  const unsigned grid = norm_grid(d.rows, lanes, kNormGroups);
  if (grid) {
    const hipError_t e = d.dtype == VISTA_BF16 ? dispatch_norm<bf16_t>(p, vec, whole, true, grid, lanes, s)
                                               : dispatch_norm<float>(p, vec, whole, true, grid, lanes, s);
    if (e != hipSuccess) return VISTA_ERR_HIP;
  }
  if (!sums) return VISTA_OK;
  const dim3 blocks((2 * d.d + 15) / 16);
  if (d.dtype == VISTA_BF16)
    VISTA_LAUNCH(norm_columns_kernel<bf16_t>, blocks, dim3(16 * kRuns), 0, s, p.partials, int(grid), d.d,
                 static_cast<bf16_t*>(dw), static_cast<bf16_t*>(db));
  else
    VISTA_LAUNCH(norm_columns_kernel<float>, blocks, dim3(16 * kRuns), 0, s, p.partials, int(grid), d.d, static_cast<float*>(dw),
                 static_cast<float*>(db));
  return VISTA_OK;
}

}  // namespace vista
