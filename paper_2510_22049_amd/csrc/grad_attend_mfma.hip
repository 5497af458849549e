// Gradients of candidate attention on the matrix cores (bf16 MFMA, fp32 accumulate), gfx950: heads of width 32, up to 512
// summaries, which are keys and values at once.
//
//   P = softmax(scale Q Y^T),  dP = dO Y^T,  dS = P (dP - delta),  delta = rowsum(P dP)
//   dQ = scale dS Y,           dY = scale dS^T Q + P^T dO
//
// A workgroup is one wave and takes one user's head and a share of its candidates, 32 at a time, on the lanes of every
// accumulator, against all summaries, whose rows stay in LDS.  Nothing is exchanged between waves; with four to a workgroup,
// the loads at its start and the sum of four dY at its end took a quarter of the time.
//   S^T = Y Q^T, dP^T = Y dO^T      one operand of Y for both; a candidate's statistics are sums within its lane
//   first walk over the summaries: sum of 2^S and of 2^S dP; second walk, scores formed again with -lse and -delta as the
//   accumulators' start:
//   dQ^T += Y^T dS                  contracted over the summaries: dS as it stands; complete at the end of the walk
//   dY^T += Q^T dS^T + dO^T P^T     contracted over the candidates, which are on lanes: P and dS are turned through LDS; its
//                                   accumulators, 16 registers for 32 summaries, stay with the wave to the end
// One wave a SIMD from S = 65 on (dY's accumulators), so a wave's vector work runs beside its own products: scores of block n,
// vector work of block n - 1 and gradients of block n - 2 share a step.
//
// Roundings.  scale log2(e) Q is taken as two bf16 terms (one would move a score s by 2^-9 s); P and dS are rounded to
// bf16 once each, their errors independent; everything else is exact or fp32.  Against fp64, 2-norm: 2.3e-3 to 2.4e-3, of which
// 1.7e-3 is the output's rounding.
//
// Measured, 1024 users x 512 candidates, d = 128, H = 4, S = 256: 385 us a call in a stream, 206 GFLOP of the definition, at 2.05 GHz;
// 18 products of 32x32x16 a unit of 32 candidates x 32 summaries, 12 of them the definition's, are 144 us of the matrix pipe, and
// 32 exponentials and some 90 plain vector instructions a lane and unit nearly as much of the vector unit; the rest is what a wave
// alone on its SIMD waits for: a tile's start and its statistics between the walks.  With a mask on every block instead of the last
// few: 459.  Two users x 100 candidates: 14 us, one tile a wave, of which most is code that is walked once.
#include "grad_mfma.hpp"

namespace vista {
namespace {

constexpr float kBounded = 60.f;

struct AttendGradParams {
  const uint16_t* cand;
  const uint16_t* summ;
  const uint16_t* dO;
  uint16_t* d_cand;
  uint16_t* d_summ;
  float* records;          // [share][B][H][S][32], where candidates are shared out
  int64_t B;
  int C, S, d, H, shares, rows_each;
  float scale;
  bool self_term;
};

// Candidates of a tile on their way: 8 bytes for each half slice of the operand order, of q and of dO.
struct CandidateTile {
  Pack8 q[2], o[2];
  __device__ __forceinline__ void request(const uint16_t* Q, const uint16_t* dO, int64_t first, int64_t end, int d, int lane) {
    int64_t row = first + (lane & 31);
    row = row < end ? row : end - 1;
    const uint16_t *a = Q + row * d + 4 * (lane >> 5), *b = dO + row * d + 4 * (lane >> 5);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        q[t].d[k] = *reinterpret_cast<const u32x2*>(a + 16 * t + 8 * k);
        o[t].d[k] = *reinterpret_cast<const u32x2*>(b + 16 * t + 8 * k);
      }
  }
  __device__ __forceinline__ void clear_unless(bool in) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        q[t].w[i] = in ? q[t].w[i] : 0u;
        o[t].w[i] = in ? o[t].w[i] : 0u;
      }
  }
};
__device__ __forceinline__ float element(const Pack8& p, int j) {
  const uint32_t w = p.w[j / 2];
  return __uint_as_float(j % 2 ? w & 0xFFFF0000u : w << 16);
}
// Sum over a candidate's channels of a b; both halves get it.
__device__ __forceinline__ float dot(const Pack8 (&a)[2], const Pack8 (&b)[2]) {
  float s = 0.f;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fmaf(element(a[t], j), element(b[t], j), s);
  return s + __shfl_xor(s, 32, 64);
}

// NKB blocks of 32 summaries; those from FULL on may hold rows beyond S.
template <int NKB, int FULL>
__global__ __launch_bounds__(64, 1) void attend_grad_kernel(AttendGradParams p) {
  __shared__ __align__(16) char rows[NKB * kBlockBytes];
  __shared__ __align__(16) float beyond[NKB * 32];              // 0, minus infinity from S on
  __shared__ __align__(16) char patches[2 * kBlockBytes];       // dS and P of a block: reads of one precede writes of the next
  const int lane = threadIdx.x, l32 = lane & 31, hf = lane >> 5;
  // the heads and shares of a user, which read the same lines, run on one XCD one after another
  const int64_t unit = int64_t(blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
  const int per = p.H * p.shares, h = int(unit % per) % p.H, share = int(unit % per) / p.H;
  const int64_t b = unit / per;
  if (b >= p.B) return;
  const int64_t begin = int64_t(share) * p.rows_each, end = begin + p.rows_each < p.C ? begin + p.rows_each : p.C;
  const uint16_t* Y = p.summ + b * p.S * p.d + 32 * h;
  const uint16_t* Q = p.cand + b * p.C * p.d + 32 * h;
  const uint16_t* dO = p.dO + b * p.C * p.d + 32 * h;
  const int tiles = int((end - begin + 31) / 32);
  CandidateTile next;
  next.request(Q, dO, begin, end, p.d, lane);

  // summaries into LDS, and the square of their largest norm
  float top = 0.f;
  // loads under way at a time, two a block of summaries; rows beyond S read the last one, since a load behind a condition waits for
  // the one before (1024 x 512 candidates: 444 us instead of 424; 833 x 10, S = 490: 134 instead of 113)
  constexpr int kBatch = NKB % 4 == 0 ? 8 : NKB % 2 == 0 ? 4 : 2;
  for (int from = 0; from < 2 * NKB; from += kBatch) {
    u32x4 raw[kBatch];
#pragma unroll
    for (int n = 0; n < kBatch; ++n) {
      const int row = 16 * (from + n) + lane / 4, cn = lane % 4;
      raw[n] = *reinterpret_cast<const u32x4*>(Y + int64_t(row < p.S ? row : p.S - 1) * p.d + 8 * cn);
    }
#pragma unroll
    for (int n = 0; n < kBatch; ++n) {
      const int row = 16 * (from + n) + lane / 4, cn = lane % 4;
      Pack8 v;
      v.u = row < p.S ? raw[n] : u32x4{0, 0, 0, 0};
      put_row_chunk(rows, row, cn, v.u);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) sum = fmaf(element(v, j), element(v, j), sum);
      sum += __shfl_xor(sum, 1, 64);     // four lanes a row
      sum += __shfl_xor(sum, 2, 64);
      top = sum > top || sum != sum ? sum : top;   // NaN stays: no tile is then bounded
    }
  }
  for (int i = lane; i < NKB * 32; i += 64) beyond[i] = i < p.S ? 0.f : -__builtin_inff();
#pragma unroll
  for (int o = 4; o < 64; o *= 2) {
    const float n = __shfl_xor(top, o, 64);
    top = n > top || n != n ? n : top;
  }
  __syncthreads();
  const float c = p.scale * kLog2e, limit = kBounded * kBounded / (top * c * c);   // of |q|^2

  const RowReader rd(rows, lane);
  const Patch patch(patches, lane);
  const uint32_t beyond_at = kept(lds_address(beyond) + 16 * hf);
  auto masked = [&](int qb) __attribute__((always_inline)) {   // 0 or minus infinity for the accumulator's rows
    f32x16 v;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 a = lds_read<f32x4>(beyond_at + 128 * qb + 32 * g);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * g + i] = a[i];
    }
    return v;
  };
  f32x16 dy[NKB];
#pragma unroll
  for (int kb = 0; kb < NKB; ++kb) dy[kb] = f32x16{0};

  for (int t = 0; t < tiles; ++t) {
    const int64_t first = begin + int64_t(t) * 32;
    CandidateTile tile = next;
    if (first + 32 > end) tile.clear_unless(first + l32 < end);   // zeros: no weight in any gradient
    if (t + 1 < tiles) next.request(Q, dO, first + 32, end, p.d, lane);
    bf16x8 qh[2], ql[2], o[2] = {tile.o[0].v, tile.o[1].v}, qt[2], ot[2];
    {
      f32x16 s;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = element(tile.q[i / 8], i % 8) * c;
      pack2(s, qh, ql);
      const bf16x8 q[2] = {tile.q[0].v, tile.q[1].v};
      patch.put(0, q);
      patch.put(kBlockBytes, o);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        qt[k] = patch.get(0, k);
        ot[k] = patch.get(kBlockBytes, k);
      }
    }
    const float n2 = dot(tile.q, tile.q);
    // a candidate that is not finite has no result that a bound could spoil
    const bool bounded = __builtin_amdgcn_ballot_w64(!(n2 <= limit) && n2 - n2 == 0.f) == 0;
    float m = 0.f, l = 0.f, e = 0.f;
    if (bounded) {
      bf16x8 y[2];
      f32x16 s[2], dp[2];
      auto request_block = [&](auto block) __attribute__((always_inline)) {
        constexpr int kb = decltype(block)::value;
#pragma unroll
        for (int k = 0; k < 2; ++k) y[k] = rd.rows(kBlockBytes * kb, k);
      };
      request_block(Int<0>{});
      each<NKB + 1>([&](auto step) __attribute__((always_inline)) {
        constexpr int n = decltype(step)::value;              // products of block n, vector work of block n - 1
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (n < NKB) {
          f32x16 a = {0};
          if constexpr (n >= FULL) a = masked(n);
          a = mfma(y[0], ql[0], a);
          f32x16 d = mfma(y[0], o[0], f32x16{0});
          a = mfma(y[1], ql[1], a);
          dp[n % 2] = mfma(y[1], o[1], d);
          a = mfma(y[0], qh[0], a);
          s[n % 2] = mfma(y[1], qh[1], a);
        }
        if constexpr (n + 1 < NKB) request_block(Int<n + 1>{});
        if constexpr (n >= 1) {
          constexpr int i = (n - 1) % 2;
          float l2 = 0.f, e2 = 0.f;
#pragma unroll
          for (int k = 0; k < 16; k += 2) {
            const float w0 = exp2_fast(s[i][k]), w1 = exp2_fast(s[i][k + 1]);
            l += w0;
            e = fmaf(w0, dp[i][k], e);
            l2 += w1;
            e2 = fmaf(w1, dp[i][k + 1], e2);
          }
          l += l2;
          e += e2;
        }
        if constexpr (n >= 1 && n < NKB) {
#pragma unroll
          for (int i = 0; i < 6; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x400, 3, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 6, 0);
            if (i == 3) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
          }
        }
      });
    } else {
      m = kLowest;
      each<NKB>([&](auto block) __attribute__((always_inline)) {
        constexpr int kb = decltype(block)::value;
        __builtin_amdgcn_sched_barrier(0);
        f32x16 s = masked(kb), dp = {0};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const bf16x8 y = rd.rows(kBlockBytes * kb, k);
          s = mfma(y, ql[k], s);
          s = mfma(y, qh[k], s);
          dp = mfma(y, o[k], dp);
        }
        float best = m;
#pragma unroll
        for (int k = 0; k < 16; ++k) best = fmaxf(best, s[k]);
        const float f = exp2_fast(m - best);
        l *= f;
        e *= f;
        m = best;
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const float w = exp2_fast(s[k] - m);
          l += w;
          e = fmaf(w, dp[k], e);
        }
        asm volatile("" : "+v"(l), "+v"(e));
      });
    }
    {
      const float m2 = __shfl_xor(m, 32, 64), l2 = __shfl_xor(l, 32, 64), e2 = __shfl_xor(e, 32, 64);
      join_stats(m, l, e, m2, l2, e2);
    }
    float own_s = 0.f, own_t = 0.f;
    if (p.self_term) {
      own_s = n2 * c;
      own_t = dot(tile.o, tile.q);
      join_stats(m, l, e, own_s, 1.f, own_t);
    }
    const float lse = m + __builtin_amdgcn_logf(l), delta = e / l;

    f32x16 dq;
    {
      bf16x8 y[2], yt[2], w[2][2], dsp[2][2];
      f32x16 s[2], ds[2], cs, cd;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        cs[i] = -lse;
        cd[i] = -delta;
      }
      auto request_block = [&](auto block) __attribute__((always_inline)) {
        constexpr int kb = decltype(block)::value;
#pragma unroll
        for (int k = 0; k < 2; ++k) y[k] = rd.rows(kBlockBytes * kb, k);
      };
      request_block(Int<0>{});
      each<NKB + 2>([&](auto step) __attribute__((always_inline)) {
        constexpr int n = decltype(step)::value;
        constexpr bool scores = n < NKB, vector = n >= 1 && n <= NKB, products = n >= 2;
        __builtin_amdgcn_sched_barrier(0);
        bf16x8 dst[2], pt[2];
        if constexpr (products) {
          constexpr int kb = n - 2;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            dst[k] = patch.get(0, k);
            pt[k] = patch.get(kBlockBytes, k);
            yt[k] = rd.columns(kBlockBytes * kb, k);
          }
        }
        if constexpr (scores) {
          f32x16 a = mfma(y[0], ql[0], cs), d = mfma(y[0], o[0], cd);
          a = mfma(y[1], ql[1], a);
          ds[n % 2] = mfma(y[1], o[1], d);
          a = mfma(y[0], qh[0], a);
          s[n % 2] = mfma(y[1], qh[1], a);
        }
        if constexpr (n + 1 < NKB) request_block(Int<n + 1>{});
        if constexpr (vector) {
          constexpr int kb = n - 1, i = kb % 2;
          if constexpr (kb >= FULL) s[i] += masked(kb);
#pragma unroll
          for (int k = 0; k < 16; ++k) s[i][k] = exp2_fast(s[i][k]);
          ds[i] *= s[i];
          ds[i] *= p.scale;
          pack(s[i], w[i]);
          pack(ds[i], dsp[i]);
          patch.put(0, dsp[i]);
          patch.put(kBlockBytes, w[i]);
        }
        if constexpr (products) {
          constexpr int kb = n - 2, i = kb % 2;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            dq = mfma(yt[k], dsp[i][k], kb == 0 && k == 0 ? f32x16{0} : dq);
            dy[kb] = mfma(qt[k], dst[k], dy[kb]);
            dy[kb] = mfma(ot[k], pt[k], dy[kb]);
          }
        }
        if constexpr (scores && vector && products) {
#pragma unroll
          for (int i = 0; i < 6; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x400, 3, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
          }
#pragma unroll
          for (int i = 0; i < 6; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (i == 0) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 7, 0);
            if (i == 4) __builtin_amdgcn_sched_group_barrier(0x200, 4, 0);
          }
          __builtin_amdgcn_sched_group_barrier(0x200, 4, 0);
        }
      });
    }
    // registers 0..7 of a lane are channels 8 hf on, 8..15 channels 16 + 8 hf on
    if (p.self_term) {
      const float pw = exp2_fast(own_s - lse), ds = 2.f * p.scale * pw * (own_t - delta);
      int64_t row = first + l32;
      row = row < end ? row : end - 1;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        Pack8 q, g;
        q.u = *reinterpret_cast<const u32x4*>(Q + row * p.d + 16 * k + 8 * hf);
        g.u = *reinterpret_cast<const u32x4*>(dO + row * p.d + 16 * k + 8 * hf);
#pragma unroll
        for (int j = 0; j < 8; ++j) dq[8 * k + j] += fmaf(ds, element(q, j), pw * element(g, j));
      }
    }
    bf16x8 out[2];
    pack(dq, out);
    if (first + l32 < end) {
      uint16_t* to = p.d_cand + (b * p.C + first + l32) * p.d + 32 * h + 8 * hf;
#pragma unroll
      for (int k = 0; k < 2; ++k) *reinterpret_cast<bf16x8*>(to + 16 * k) = out[k];
    }
  }

  // dY: a lane has 4 channels of one summary in every four registers
  each<NKB>([&](auto block) __attribute__((always_inline)) {
    constexpr int kb = decltype(block)::value;
    const int i = 32 * kb + l32;
    if (i < p.S) {
      if (p.shares == 1) {
        uint16_t* to = p.d_summ + (b * p.S + i) * p.d + 32 * h + 4 * hf;
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<u32x2*>(to + 8 * g) =
              u32x2{pair_to_bf16(dy[kb][4 * g], dy[kb][4 * g + 1]), pair_to_bf16(dy[kb][4 * g + 2], dy[kb][4 * g + 3])};
      } else {
        float* to = p.records + (((int64_t(share) * p.B + b) * p.H + h) * p.S + i) * 32 + 4 * hf;
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<f32x4*>(to + 8 * g) = f32x4{dy[kb][4 * g], dy[kb][4 * g + 1], dy[kb][4 * g + 2], dy[kb][4 * g + 3]};
      }
    }
  });
}

// Shares of a user's candidates: the count with the shortest time, the smallest of equals.  Waves are all alike, 1024 run at a
// time, and a wave takes about as long as two tiles before its first and after its last, a tile 0.75 us for 32 summaries.  More
// shares than one are joined, which takes 4 us and their records' way to memory and back at 4 TB/s.
int shares_of(const vista_attend_desc& d) {
  const int64_t base = int64_t(d.B) * d.H, tiles = (int64_t(d.C) + 31) / 32;
  int64_t best = 1;
  float time = __builtin_inff();
  for (int64_t n = 1; n <= tiles && n <= 256 && (n == 1 || base * (n - 1) < 4096); ++n) {
    const int64_t steps = (base * n + 1023) / 1024 * ((tiles + n - 1) / n + 2);
    const float join = n == 1 ? 0.f : 4.f + float(n) * float(d.B) * float(d.S) * float(d.d) * 2e-6f;
    const float t = float(steps) * 0.75f * float((d.S + 31) / 32) + join;
    if (t < time) {
      time = t;
      best = n;
    }
  }
  return int(best);
}

template <int NKB, int FULL>
hipError_t run(const AttendGradParams& p, hipStream_t s) {
  const dim3 grid(unsigned((p.B * p.H * p.shares + 7) / 8 * 8));
  return p.S == 32 * NKB ? launch(attend_grad_kernel<NKB, NKB>, grid, dim3(64), 0, s, p)
                         : launch(attend_grad_kernel<NKB, FULL>, grid, dim3(64), 0, s, p);
}

}  // namespace

bool mfma_attend_backward_supported(const vista_attend_desc& d) {
  return d.dtype == VISTA_BF16 && d.d == 32 * d.H && (int64_t(d.B) + 8) * d.H * shares_of(d) < (1 << 25);
}

size_t mfma_attend_backward_workspace(const vista_attend_desc& d) {
  const size_t shares = shares_of(d);
  return shares > 1 ? shares * d.B * d.S * d.d * sizeof(float) : 256;
}

vista_status mfma_attend_backward(const vista_attend_desc& d, float scale, const void* cand, const void* summ, const void* d_out,
                                  void* d_cand, void* d_summ, void* workspace, hipStream_t s) {
  AttendGradParams p;
  p.cand = static_cast<const uint16_t*>(cand);
  p.summ = static_cast<const uint16_t*>(summ);
  p.dO = static_cast<const uint16_t*>(d_out);
  p.d_cand = static_cast<uint16_t*>(d_cand);
  p.d_summ = static_cast<uint16_t*>(d_summ);
  p.records = static_cast<float*>(workspace);
  p.B = d.B;
  p.C = d.C;
  p.S = d.S;
  p.d = d.d;
  p.H = d.H;
  p.shares = shares_of(d);
  p.rows_each = int(((int64_t(d.C) + p.shares - 1) / p.shares + 31) / 32 * 32);
  p.shares = int((int64_t(d.C) + p.rows_each - 1) / p.rows_each);
  p.scale = scale;
  p.self_term = (d.flags & VISTA_FLAG_SELF_TERM) != 0;
  const int blocks = (d.S + 31) / 32;
  const hipError_t e = blocks <= 1    ? run<1, 0>(p, s)
                       : blocks <= 2  ? run<2, 1>(p, s)
                       : blocks <= 3  ? run<3, 2>(p, s)
                       : blocks <= 4  ? run<4, 3>(p, s)
                       : blocks <= 6  ? run<6, 4>(p, s)
                       : blocks <= 8  ? run<8, 6>(p, s)
                       : blocks <= 10 ? run<10, 8>(p, s)
                       : blocks <= 12 ? run<12, 10>(p, s)
                                      : run<16, 12>(p, s);
  if (e != hipSuccess) return VISTA_ERR_HIP;
  if (p.shares > 1 && grad_join_shares(d.dtype, p.records, p.shares, int64_t(d.B), d.S, d.d, d.H, d_summ, s) != hipSuccess)
    return VISTA_ERR_HIP;
  return VISTA_OK;
}

}  // namespace vista
