// Gradients of softmax summarization on the matrix cores (bf16 MFMA, fp32 accumulate), gfx950: heads of width 32 in a
// model of width 64, 128 or 256.
//
//   P = softmax(scale Q K^T),  dP = dO V^T,  delta_i = sum_j P_ij dP_ij,  dS = P (dP - delta)
//   dV = P^T dO,  dQ = scale dS K,  dK = scale dS^T Q,       K = X W_k, V = X W_v of the user's items
//
// Two passes over the history, each forming the projections again from X (2 D bytes an item, against 4 D for K and V):
// the statistics of every query's row (maximum, sum, sum of P dP), then, joined, the gradients.  A workgroup takes one
// segment for one head; its waves take the tiles of a piece in turn and nothing is exchanged between them in the loop.
//
// Layouts.  A lane of a 32x32 accumulator holds 16 values of one column, rows 8 (r / 4) + 4 hf + r % 4 (hf = lane / 32);
// an operand holds 8 values of one row (A) or column (B) for each slice of 16 of the contraction, and any order of these
// is fine as long as both operands use it.  So an accumulator, rounded and packed, is an operand over its rows:
//   K^T, V^T = W^T X^T           items on lanes, channels in registers: operands of S and dP as they stand
//   S = Q K^T, dP = dO V^T       queries in registers, items on lanes; -lse and -delta are the accumulators' start
//   dV^T += dO^T P, dK^T += Q^T dS   contracted over the queries: P and dS as they stand; an item stays on its lane, so dK and
//                                dV are complete when the wave has passed over all queries, and go straight to memory
//   dQ^T += K^T dS^T             contracted over the items, which are on lanes: dS is turned through LDS (written as [item][query],
//                                read back by ds_read_b64_tr_b16); its accumulators, 16 registers for 32 queries, stay with the
//                                wave for the whole piece
// Q and dO are kept in LDS once, as rows; the same transposing read gives Q^T and dO^T.
//
// Roundings.  K and V are formed in fp32 and enter every product that forms a score or dP as two bf16 terms (16 bits): one
// term would move a score of size s by 2^-9 s, and P and dS with it.  P and dS are rounded to bf16 once each (their errors are
// independent from item to item and do not add up), and so is the output.  Measured against fp64, 2-norm: dQ, dK and dV 1.7e-3
// to 2.4e-3, of which 1.7e-3 is the output's rounding.
//
// Measured, 64 users with 768597 items, d = 128, H = 4, S = 256: 703 us, of it 300 the statistics, 385 the gradients (as parts of a
// stream of calls; by themselves 310 and 500, at a lower clock), 15 the joins.  22 products of 32x32x16 a unit of 32 queries x 32
// items, 10 of them the definition's, are 310 us of the matrix pipe at the 1.7 GHz that the gradients' kernel runs at; the rest
// is what a wave alone on its SIMD cannot hide: two exponentials' worth of vector work beside a product, and a tile's start
// (projections, packing, turning K).  Without the low terms the call takes 612 us, and its scores are off by 2^-9 of their size.
#include "grad_mfma.hpp"

namespace vista {
namespace {

struct HistoryGradParams {
  const uint16_t* X;
  const uint16_t* Wk;
  const uint16_t* Wv;
  const uint16_t* Q;
  const uint16_t* dO;
  const int64_t* offsets;
  float* stats;            // [slot][H][S][3]
  const float* lse;        // [B][H][S]
  const float* delta;
  float* records;          // [slot][H][32 NQB][32]: sum of dS K scale log2(e)
  uint16_t* dK;
  uint16_t* dV;
  int64_t q_user_stride, N, G;
  int B, S, H, seg, rows;  // rows: 32 ceil(S / 32), those of a record
  float scale, scale_log2;
};

// Which (segment, head) a block takes: the heads of a segment, which read the same rows of X, run on one XCD one after
// another.  false: past the end.
__device__ __forceinline__ bool segment_and_head(int64_t G, int H, int64_t& segment, int& h) {
  const int64_t r = blockIdx.x >> 3;
  h = int(r % H);
  segment = r / H * 8 + (blockIdx.x & 7);
  return segment < G;
}
unsigned segment_blocks(int64_t G, int H) { return unsigned((G + 7) / 8 * 8 * H); }

// Projection weights of a head as operands: element j of slice ks of lane (hf, channel) is W[16 ks + 8 hf + j][channel].
template <int D, int THREADS>
__device__ __forceinline__ void put_weights(uint4* dst, const uint16_t* W, int h) {
  uint16_t* out = reinterpret_cast<uint16_t*>(dst);
  for (int i = threadIdx.x; i < D * 32; i += THREADS) {
    const int k = i / 32, c = i % 32;
    out[((k / 16) * 64 + (k / 8 % 2) * 32 + c) * 8 + k % 8] = W[k * D + 32 * h + c];
  }
}

// Q and dO of a user and head.  Rows beyond S are zeros.
template <int D, int THREADS>
__device__ __forceinline__ void put_queries(char* q, char* o, const HistoryGradParams& p, int user, int h, int rows) {
  const uint16_t* Q = p.Q + int64_t(user) * p.q_user_stride + 32 * h;
  const uint16_t* dO = p.dO + int64_t(user) * p.S * D + 32 * h;
  for (int i = threadIdx.x; i < rows * 4; i += THREADS) {
    const int row = i / 4, cn = i % 4;
    u32x4 a = {0, 0, 0, 0}, b = a;
    if (row < p.S) {
      a = *reinterpret_cast<const u32x4*>(Q + row * D + 8 * cn);
      b = *reinterpret_cast<const u32x4*>(dO + row * D + 8 * cn);
    }
    put_row_chunk(q, row, cn, a);
    put_row_chunk(o, row, cn, b);
  }
}

// 32 items of one wave: their rows in LDS, as operands ([slice][lane], 16 bytes each), put there by direct loads that need
// no registers while they are under way.  At width 256 the second half of a row does not fit: it is loaded into registers,
// which are free while a tile begins.
template <int D>
struct Items {
  static constexpr int KS = D / 16, kAhead = KS < 8 ? KS : 8, kRest = KS - kAhead;
  static constexpr int kBytes = kAhead * 1024;
  uint32_t x_at, w_at;       // this lane's operand of the first slice, of the rows and of the weights (W_k; W_v follows)
  __device__ __forceinline__ Items(const void* buffer, const void* weights, int lane)
      : x_at(kept(lds_address(buffer) + 16 * lane)), w_at(kept(lds_address(weights) + 16 * lane)) {}
  // Rows first .. first + 31; those from end on repeat the last.  Written as assembly so that the wait is the explicit
  // one below, not a conservative one of the compiler's before the next read of LDS.
  __device__ __forceinline__ void request(const uint16_t* X, int64_t first, int64_t end, int lane) const {
    const uint16_t* base = X + first * D;
    const uint32_t from = offset(first, end, lane);
    const uint32_t to = __builtin_amdgcn_readfirstlane(x_at);        // lane 0's: lane i lands 16 i bytes on
#pragma unroll
    for (int ks = 0; ks < kAhead; ++ks)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                   :
                   : "s"(to + 1024 * ks), "v"(from + 32 * ks), "s"(base)
                   : "memory", "m0");
  }
  static __device__ __forceinline__ uint32_t offset(int64_t first, int64_t end, int lane) {
    const int last = int(end - first < 32 ? end - first : 32) - 1, l32 = lane & 31;
    return (l32 < last ? l32 : last) * (2 * D) + 16 * (lane >> 5);
  }
  // Every request of this wave has landed.  AFTER: what the wave has sent to memory since then, counted down in order.
  template <int AFTER>
  __device__ __forceinline__ void wait() const {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(AFTER) : "memory");
  }
  // K^T, V^T of the items, channels in registers, items on lanes
  __device__ __forceinline__ void project(const uint16_t* X, int64_t first, int64_t end, int lane, f32x16& k, f32x16& v) const {
    Pack8 rest[kRest > 0 ? kRest : 1];
    if constexpr (kRest > 0) {
      const char* src = reinterpret_cast<const char*>(X + first * D) + offset(first, end, lane) + 32 * kAhead;
#pragma unroll
      for (int i = 0; i < kRest; ++i) rest[i].u = *reinterpret_cast<const u32x4*>(src + 32 * i);
    }
    k = v = f32x16{0};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      Pack8 a, b, x;
      a.u = lds_read<u32x4>(w_at + 1024 * ks);
      b.u = lds_read<u32x4>(w_at + 1024 * (KS + ks));
      if (ks < kAhead) x.u = lds_read<u32x4>(x_at + 1024 * ks); else x.u = rest[ks < kAhead ? 0 : ks - kAhead].u;
      k = mfma(a.v, x.v, k);
      v = mfma(b.v, x.v, v);
    }
  }
};

// ------------------------------------------------------------------------------------------------ statistics
// S^T = K Q^T and dP^T = V dO^T with the queries on lanes: a lane keeps its query's reference m, sum of 2^(s - m) and sum
// of 2^(s - m) dP over the rows of its half.  While every |q| |k| of a tile is at most 60 (base 2; Cauchy-Schwarz on the
// tile's key norms) and nothing else was met in the piece, the reference is 0: no maximum, nothing to subtract, and the
// vector work of one block of queries runs beside the products of the next.  Any other tile, and one that is not full, takes
// the general way: m is the first tile's maximum, raised where a score exceeds it by 2^20.
constexpr float kBounded = 60.f;
constexpr int kStatsWaves = 8;         // two a SIMD

template <int D, int NQB>
__global__ __launch_bounds__(64 * kStatsWaves, 2) void history_stats_kernel(HistoryGradParams p) {
  constexpr int NT = 64 * kStatsWaves, KS = D / 16;
  __shared__ __align__(16) char rows[2 * NQB * kBlockBytes];      // Q, dO
  constexpr uint32_t kGrad = NQB * kBlockBytes;                   // where dO begins
  __shared__ uint4 ws[2][KS * 64];
  __shared__ __align__(16) char xs[kStatsWaves][Items<D>::kBytes];
  const int lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int64_t segment;
  int h;
  if (!segment_and_head(p.G, p.H, segment, h)) return;
  const int64_t begin = segment * p.seg, end = begin + p.seg < p.N ? begin + p.seg : p.N;
  put_weights<D, NT>(ws[0], p.Wk, h);
  put_weights<D, NT>(ws[1], p.Wv, h);
  const Items<D> it(xs[wave], ws[0], lane);
  const RowReader rd(rows, lane);
  int user = find_user_wave(p.offsets, p.B, begin);
  int64_t pos = begin;
  Piece pc;
  while (next_piece(p.offsets, p.B, end, user, pos, pc)) {
    const int tiles = int((pc.end - pc.begin + 31) / 32);
    __syncthreads();                     // the piece before has been read
    int t = wave;
    if (t < tiles) it.request(p.X, pc.begin + int64_t(t) * 32, pc.end, lane);
    put_queries<D, NT>(rows, rows + kGrad, p, pc.user, h, NQB * 32);
    __syncthreads();
    float m[NQB], l[NQB], e[NQB], limit = 0.f;
    each<NQB>([&](auto block) __attribute__((always_inline)) {
      constexpr int qb = decltype(block)::value;
      m[qb] = l[qb] = e[qb] = 0.f;
      float n = 0.f;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        Pack8 q;
        q.v = rd.rows(kBlockBytes * qb, k);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float a = __uint_as_float(q.w[i] << 16), b = __uint_as_float(q.w[i] & 0xFFFF0000u);
          n = fmaf(a, a, fmaf(b, b, n));
        }
      }
      n += __shfl_xor(n, 32, 64);
      limit = n > limit || n != n ? n : limit;       // NaN stays: no tile is then bounded
    });
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const float n = __shfl_xor(limit, o, 64);
      limit = n > limit || n != n ? n : limit;
    }
    limit = kBounded * kBounded / limit;             // of |k|^2
    bool fresh = true, plain = true;
    for (; t < tiles; t += kStatsWaves) {
      const int64_t first = pc.begin + int64_t(t) * 32;
      const int left = pc.end - first < 32 ? int(pc.end - first) : 32;
      bf16x8 kh[2], kl[2], vh[2], vl[2];
      bool bounded;
      {
        f32x16 k, v;
        it.template wait<0>();
        it.project(p.X, first, pc.end, lane, k, v);
        k *= p.scale_log2;
        float n = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) n = fmaf(k[r], k[r], n);
        n += __shfl_xor(n, 32, 64);
        bounded = __builtin_amdgcn_ballot_w64(!(n <= limit)) == 0;
        pack2(k, kh, kl);
        pack2(v, vh, vl);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // the rows have been read
      if (t + kStatsWaves < tiles) it.request(p.X, first + int64_t(kStatsWaves) * 32, pc.end, lane);
      if (bounded && plain && left == 32) {
        bf16x8 q[2], o[2];
        f32x16 s[2], dp[2];
        auto request_block = [&](auto block) __attribute__((always_inline)) {
          constexpr int qb = decltype(block)::value;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            q[k] = rd.rows(kBlockBytes * qb, k);
            o[k] = rd.rows(kGrad + kBlockBytes * qb, k);
          }
        };
        request_block(Int<0>{});
        each<NQB + 1>([&](auto step) __attribute__((always_inline)) {
          constexpr int n = decltype(step)::value;            // products of block n, vector work of block n - 1
          __builtin_amdgcn_sched_barrier(0);
          if constexpr (n < NQB) {
            f32x16 a = mfma(kl[0], q[0], f32x16{0}), b = mfma(vl[0], o[0], f32x16{0});
            a = mfma(kl[1], q[1], a);
            b = mfma(vl[1], o[1], b);
            a = mfma(kh[0], q[0], a);
            b = mfma(vh[0], o[0], b);
            s[n % 2] = mfma(kh[1], q[1], a);
            dp[n % 2] = mfma(vh[1], o[1], b);
          }
          if constexpr (n + 1 < NQB) request_block(Int<n + 1>{});
          if constexpr (n >= 1) {
            constexpr int qb = n - 1, i = qb % 2;
            float l2 = 0.f, e2 = 0.f;                          // chains of their own: half the latency
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
              const float w0 = exp2_fast(s[i][r]), w1 = exp2_fast(s[i][r + 1]);
              l[qb] += w0;
              e[qb] = fmaf(w0, dp[i][r], e[qb]);
              l2 += w1;
              e2 = fmaf(w1, dp[i][r + 1], e2);
            }
            l[qb] += l2;
            e[qb] += e2;
            asm volatile("" : "+v"(l[qb]), "+v"(e[qb]));       // formed here, not after the last block
          }
          if constexpr (n >= 1 && n < NQB) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
              __builtin_amdgcn_sched_group_barrier(0x400, 2, 0);
              __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
            }
          }
        });
        fresh = false;
        continue;
      }
      each<NQB>([&](auto block) __attribute__((always_inline)) {
        constexpr int qb = decltype(block)::value;
        __builtin_amdgcn_sched_barrier(0);
        f32x16 s, dp = {0};
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = -m[qb];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const bf16x8 q = rd.rows(kBlockBytes * qb, k), o = rd.rows(kGrad + kBlockBytes * qb, k);
          s = mfma(kl[k], q, s);
          dp = mfma(vl[k], o, dp);
          s = mfma(kh[k], q, s);
          dp = mfma(vh[k], o, dp);
        }
        float top = kLowest;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const bool in = 8 * (r / 4) + 4 * hf + r % 4 < left;
          s[r] = in ? s[r] : -__builtin_inff();
          dp[r] = in ? dp[r] : 0.f;
          top = fmaxf(top, s[r]);
        }
        if (fresh || __builtin_amdgcn_ballot_w64(top > 20.f) != 0) {
          const float up = fresh ? top : fmaxf(top, 0.f), f = exp2_fast(-up);
          m[qb] = fresh ? up : m[qb] + up;
          l[qb] = fresh ? 0.f : l[qb] * f;
          e[qb] = fresh ? 0.f : e[qb] * f;
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] -= up;
          plain = false;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float w = exp2_fast(s[r]);
          l[qb] += w;
          e[qb] = fmaf(w, dp[r], e[qb]);
        }
        asm volatile("" : "+v"(l[qb]), "+v"(e[qb]));
      });
      fresh = false;
    }
    // the two halves of a query, then the waves that had a tile in ascending order, eight blocks at a time through the memory of the
    // items' rows
    constexpr int kAtOnce = NQB < 8 ? NQB : 8;
    static_assert(kAtOnce * 32 * 3 * sizeof(float) <= Items<D>::kBytes, "a wave's statistics fit its rows' place");
    const int64_t slot = (segment + pc.user) * p.H + h;
    const int active = tiles < kStatsWaves ? tiles : kStatsWaves;
    auto joined = [&](int w, int i) { return reinterpret_cast<float*>(xs[w]) + 3 * i; };
    each<(NQB + kAtOnce - 1) / kAtOnce>([&](auto part) __attribute__((always_inline)) {
      constexpr int from = decltype(part)::value * kAtOnce, count = NQB - from < kAtOnce ? NQB - from : kAtOnce;
      if (from > 0) __syncthreads();
      if (wave < active)
        each<count>([&](auto block) __attribute__((always_inline)) {
          constexpr int n = decltype(block)::value, qb = from + n;
          const float m2 = __shfl_xor(m[qb], 32, 64), l2 = __shfl_xor(l[qb], 32, 64), e2 = __shfl_xor(e[qb], 32, 64);
          join_stats(m[qb], l[qb], e[qb], m2, l2, e2);
          if (hf == 0) {
            float* at = joined(wave, 32 * n + l32);
            at[0] = m[qb];
            at[1] = l[qb];
            at[2] = e[qb];
          }
        });
      __syncthreads();
      for (int n = threadIdx.x; n < 32 * count && 32 * from + n < p.S; n += NT) {
        const float* first = joined(0, n);
        float jm = first[0], jl = first[1], je = first[2];
        for (int w = 1; w < active; ++w) {
          const float* at = joined(w, n);
          join_stats(jm, jl, je, at[0], at[1], at[2]);
        }
        float* out = p.stats + (slot * p.S + 32 * from + n) * 3;
        out[0] = jm;
        out[1] = jl;
        out[2] = je;
      }
    });
  }
}

// ------------------------------------------------------------------------------------------------ gradients
// LOW: the keys' low terms are in dQ's product too.  The keys' roundings are independent and average out of the sum over a
// long history's items, while the gradient's own part grows with it: dQ is off by 2.9e-3 of its norm at 16 items, 2.3e-3 at
// 4 d, 1.9e-3 at 16 d, of which 1.7e-3 is its rounding to bf16.  With the low terms it is 2.4e-3 at 16 items; they cost
// 750 us a call instead of 707 (768597 items of 64 users, d = 128, H = 4, S = 256).  So they are there for average histories
// of less than 4 d items.
constexpr int kGradWaves = 4;          // one a SIMD: dQ alone is 16 registers for 32 queries
constexpr int kLongHistory = 4;        // times d

template <int D, int NQB, bool LOW>
__global__ __launch_bounds__(64 * kGradWaves, 1) void history_grad_kernel(HistoryGradParams p) {
  constexpr int NT = 64 * kGradWaves, KS = D / 16;
  __shared__ __align__(16) char rows[2 * NQB * kBlockBytes];      // Q, dO
  constexpr uint32_t kGrad = NQB * kBlockBytes;                   // where dO begins
  __shared__ __align__(16) float starts[2][NQB * 32];          // -lse, -delta
  __shared__ uint4 ws[2][KS * 64];
  __shared__ __align__(16) char xs[kGradWaves][Items<D>::kBytes];
  __shared__ __align__(16) char patches[kGradWaves][4096];           // dS of two units; K once a tile; dQ at the end of a piece
  const int lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int64_t segment;
  int h;
  if (!segment_and_head(p.G, p.H, segment, h)) return;
  const int64_t begin = segment * p.seg, end = begin + p.seg < p.N ? begin + p.seg : p.N;
  put_weights<D, NT>(ws[0], p.Wk, h);
  put_weights<D, NT>(ws[1], p.Wv, h);
  const Items<D> it(xs[wave], ws[0], lane);
  const RowReader rd(rows, lane);
  const Patch patch(patches[wave], lane);
  const uint32_t starts_at = kept(lds_address(starts) + 16 * hf);
  int user = find_user_wave(p.offsets, p.B, begin);
  int64_t pos = begin;
  Piece pc;
  while (next_piece(p.offsets, p.B, end, user, pos, pc)) {
    const int tiles = int((pc.end - pc.begin + 31) / 32);
    int t = wave;
    if (t < tiles) it.request(p.X, pc.begin + int64_t(t) * 32, pc.end, lane);
    __syncthreads();                     // the piece before has been read
    put_queries<D, NT>(rows, rows + kGrad, p, pc.user, h, NQB * 32);
    const int64_t stat = (int64_t(pc.user) * p.H + h) * p.S;
    for (int i = threadIdx.x; i < NQB * 32; i += NT) {
      starts[0][i] = i < p.S ? -p.lse[stat + i] : -__builtin_inff();    // no weight beyond S
      starts[1][i] = i < p.S ? -p.delta[stat + i] : 0.f;
    }
    __syncthreads();
    f32x16 dq[NQB];
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) dq[qb] = f32x16{0};
    for (; t < tiles; t += kGradWaves) {
      const int64_t first = pc.begin + int64_t(t) * 32;
      const int left = pc.end - first < 32 ? int(pc.end - first) : 32;
      bf16x8 kh[2], kl[2], vh[2], vl[2], kt[2], kt_low[2];
      {
        f32x16 k, v;
        // the four stores of the last tile's gradients, which followed the request, may still be under way
        if (t == wave) it.template wait<0>(); else it.template wait<4>();
        it.project(p.X, first, pc.end, lane, k, v);
        pack2(k * p.scale_log2, kh, kl);
        // Items past the piece are copies of its last: finite where it is, never stored, and with zeros for keys here they
        // add nothing to dQ.
        auto turn = [&](const bf16x8 (&from)[2], uint32_t offset, bf16x8 (&to)[2]) __attribute__((always_inline)) {
          bf16x8 masked[2];
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            Pack8 m;
            m.v = from[n];
#pragma unroll
            for (int i = 0; i < 4; ++i) m.w[i] = l32 < left ? m.w[i] : 0u;
            masked[n] = m.v;
          }
          patch.put(offset, masked);
#pragma unroll
          for (int n = 0; n < 2; ++n) to[n] = patch.get(offset, n);
        };
        turn(kh, 0, kt);
        if constexpr (LOW) turn(kl, kBlockBytes, kt_low);
        pack2(v, vh, vl);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // the rows have been read
      if (t + kGradWaves < tiles) it.request(p.X, first + int64_t(kGradWaves) * 32, pc.end, lane);
      f32x16 dk, dv;
      // Units of 32 queries x 32 items, three under way at a time: in one step scores and dP of unit n, the vector work of
      // unit n - 1, the gradients' products of unit n - 2.  What is carried from step to step goes by the unit's parity;
      // operands are read out of LDS a step, or half a step, before they are used.
      bf16x8 q[2], o[2], qt[2], ot[2], w[2][2], dsp[2][2];
      f32x16 cs, cd, s[2], ds[2];
      auto request_block = [&](auto block) __attribute__((always_inline)) {
        constexpr int qb = decltype(block)::value;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          q[k] = rd.rows(kBlockBytes * qb, k);
          o[k] = rd.rows(kGrad + kBlockBytes * qb, k);
        }
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 a = lds_read<f32x4>(starts_at + 128 * qb + 32 * g);
          const f32x4 b = lds_read<f32x4>(starts_at + 128 * (NQB + qb) + 32 * g);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            cs[4 * g + i] = a[i];
            cd[4 * g + i] = b[i];
          }
        }
      };
      request_block(Int<0>{});
      each<NQB + 2>([&](auto step) __attribute__((always_inline)) {
        constexpr int n = decltype(step)::value;
        constexpr bool scores = n < NQB, vector = n >= 1 && n <= NQB, products = n >= 2;
        __builtin_amdgcn_sched_barrier(0);
        bf16x8 turned[2];
        if constexpr (products) {
          constexpr int qb = n - 2;
#pragma unroll
          for (int k = 0; k < 2; ++k) turned[k] = patch.get(kBlockBytes * (qb % 2), k);
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            ot[k] = rd.columns(kGrad + kBlockBytes * qb, k);
            qt[k] = rd.columns(kBlockBytes * qb, k);
          }
        }
        if constexpr (scores) {
          f32x16 a = mfma(q[0], kl[0], cs), b = mfma(o[0], vl[0], cd);
          a = mfma(q[1], kl[1], a);
          b = mfma(o[1], vl[1], b);
          a = mfma(q[0], kh[0], a);
          b = mfma(o[0], vh[0], b);
          s[n % 2] = mfma(q[1], kh[1], a);
          ds[n % 2] = mfma(o[1], vh[1], b);
        }
        if constexpr (n + 1 < NQB) request_block(Int<n + 1>{});
        if constexpr (vector) {
          constexpr int i = (n - 1) % 2;
#pragma unroll
          for (int r = 0; r < 16; ++r) s[i][r] = exp2_fast(s[i][r]);
          ds[i] *= s[i];
          pack(s[i], w[i]);
          pack(ds[i], dsp[i]);
          patch.put(kBlockBytes * i, dsp[i]);
        }
        if constexpr (products) {
          constexpr int qb = n - 2, i = qb % 2;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            dv = mfma(ot[k], w[i][k], qb == 0 && k == 0 ? f32x16{0} : dv);
            dk = mfma(qt[k], dsp[i][k], qb == 0 && k == 0 ? f32x16{0} : dk);
            if constexpr (LOW) dq[qb] = mfma(kt_low[k], turned[k], dq[qb]);
            dq[qb] = mfma(kt[k], turned[k], dq[qb]);
          }
        }
        // the order: reads for the products, then every product with its share of the vector work beside it
        if constexpr (scores && vector && products) {
          __builtin_amdgcn_sched_group_barrier(0x100, 12, 0);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x400, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);
          }
          __builtin_amdgcn_sched_group_barrier(0x100, 12, 0);
#pragma unroll
          for (int i = 0; i < (LOW ? 8 : 6); ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, LOW ? 4 : 5, 0);
          }
          __builtin_amdgcn_sched_group_barrier(0x200, 4, 0);
        }
      });
      bf16x8 k8[2], v8[2];
      pack(dk * p.scale, k8);
      pack(dv, v8);
      if (l32 < left) {
        const int64_t at = (first + l32) * D + 32 * h + 8 * hf;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          *reinterpret_cast<bf16x8*>(p.dK + at + 16 * k) = k8[k];
          *reinterpret_cast<bf16x8*>(p.dV + at + 16 * k) = v8[k];
        }
      }
    }
    // dQ of the piece: 32 queries at a time every wave that had a tile lays its sums down, [query][channel] in fp32, and a part of
    // each wave's threads adds them up in ascending order
    const int active = tiles < kGradWaves ? tiles : kGradWaves;
    // One wave's sums need no adding up: straight to memory (not beside 16 blocks, whose registers are spilled for it: 804 us instead
    // of 745 for 200003 items, d = 256, S = 512).  1024 users of 50 items each, S = 256, d = 128: 235 -> 213 us of this kernel.
    float* rec = p.records + ((segment + pc.user) * p.H + h) * int64_t(p.rows) * 32;
    if (NQB < 16 && active == 1) {
      if (wave == 0)
        each<NQB>([&](auto block) __attribute__((always_inline)) {
          constexpr int qb = decltype(block)::value;
          if (32 * qb < p.rows)
#pragma unroll
            for (int g = 0; g < 4; ++g)
              *reinterpret_cast<float4*>(rec + (32 * qb + l32) * 32 + 8 * g + 4 * hf) =
                  make_float4(dq[qb][4 * g], dq[qb][4 * g + 1], dq[qb][4 * g + 2], dq[qb][4 * g + 3]);
        });
      continue;
    }
    each<NQB>([&](auto block) __attribute__((always_inline)) {
      constexpr int qb = decltype(block)::value;
      __syncthreads();
      if (wave < active)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int c = 2 * g + hf;      // 16-byte chunk of the query's row: channels 8 g + 4 hf on
          *reinterpret_cast<float4*>(patches[wave] + l32 * 128 + ((c ^ (l32 & 7)) << 4)) =
              make_float4(dq[qb][4 * g], dq[qb][4 * g + 1], dq[qb][4 * g + 2], dq[qb][4 * g + 3]);
        }
      __syncthreads();
      for (int i = threadIdx.x; i < 256 && 32 * qb < p.rows; i += NT) {
        const int row = i / 8, c = i % 8;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int w = 0; w < active; ++w) {
          const float4 v = *reinterpret_cast<const float4*>(patches[w] + row * 128 + ((c ^ (row & 7)) << 4));
          sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
        }
        *reinterpret_cast<float4*>(rec + (32 * qb + row) * 32 + 4 * c) = sum;
      }
    });
    __syncthreads();
  }
}

template <int D, int NQB>
hipError_t run_blocks(const HistoryGradParams& p, bool grad, hipStream_t s) {
  const dim3 grid(segment_blocks(p.G, p.H));
  if (!grad) return launch(history_stats_kernel<D, NQB>, grid, dim3(64 * kStatsWaves), 0, s, p);
  return p.N < int64_t(kLongHistory) * D * p.B ? launch(history_grad_kernel<D, NQB, true>, grid, dim3(64 * kGradWaves), 0, s, p)
                                               : launch(history_grad_kernel<D, NQB, false>, grid, dim3(64 * kGradWaves), 0, s, p);
}
// The kernels know how many blocks of 32 queries there are; a call takes the next larger count that is built.
template <int D>
hipError_t run(const HistoryGradParams& p, bool grad, hipStream_t s) {
  const int blocks = p.rows / 32;
  return blocks <= 1   ? run_blocks<D, 1>(p, grad, s)
         : blocks <= 2  ? run_blocks<D, 2>(p, grad, s)
         : blocks <= 3  ? run_blocks<D, 3>(p, grad, s)
         : blocks <= 4  ? run_blocks<D, 4>(p, grad, s)
         : blocks <= 6  ? run_blocks<D, 6>(p, grad, s)
         : blocks <= 8  ? run_blocks<D, 8>(p, grad, s)
         : blocks <= 10 ? run_blocks<D, 10>(p, grad, s)
         : blocks <= 12 ? run_blocks<D, 12>(p, grad, s)
                        : run_blocks<D, 16>(p, grad, s);
}

size_t align256(size_t v) { return (v + 255) & ~size_t(255); }

struct Layout {
  size_t stats, records, rows, self, Ks, total;
};
Layout layout(const vista_summarize_desc& d) {
  const int64_t seg = mfma_grad_segment(d), G = (d.total_items + seg - 1) / seg;
  const size_t slots = size_t(G + d.B) * d.H, rows = size_t(d.B) * d.H * d.S;
  Layout l;
  l.stats = kHeaderBytes;
  l.records = l.stats + align256(slots * d.S * 3 * sizeof(float));
  l.rows = l.records + align256(slots * ((d.S + 31) / 32 * 32) * 32 * sizeof(float));
  l.self = l.rows + 2 * align256(rows * sizeof(float));
  l.Ks = l.self + ((d.flags & VISTA_FLAG_SELF_TERM) ? 2 * align256(rows * sizeof(float)) : 0);
  l.total = l.Ks + 2 * self_kv_bytes(d);
  return l;
}

}  // namespace

bool mfma_summarize_backward_supported(const vista_summarize_desc& d) {
  return d.dtype == VISTA_BF16 && d.attn == VISTA_ATTN_SOFTMAX && d.d == 32 * d.H && (d.d == 64 || d.d == 128 || d.d == 256);
}

// A workgroup is one (segment, head); one fits a compute unit.  Segments that make one round of 256 workgroups, at most 32768 items
// and at least 128, a tile for every wave, or, where users have fewer items than that and a segment's pieces cost more than its
// tiles, 32.  (98 users of 539 items together, S = 512, d = 256: 400 us instead of 1400.)
int mfma_grad_segment(const vista_summarize_desc& d) {
  if (d.segment_items > 0) return d.segment_items;
  const int64_t each = 256 / d.H, k = (d.total_items + each * 32768 - 1) / (each * 32768);
  const int64_t parts = each * (k > 0 ? k : 1);
  const int64_t seg = ((d.total_items + parts - 1) / parts + 31) / 32 * 32;
  const int64_t least = d.total_items < 128 * int64_t(d.B) ? 32 : 128;
  return int(seg < least ? least : seg);
}

size_t mfma_summarize_backward_workspace(const vista_summarize_desc& d) { return layout(d).total; }

vista_status mfma_summarize_backward(const SummarizeArgs& a, const void* d_out, void* d_queries, void* d_keys, void* d_values,
                                     void* d_self_keys, void* d_self_values) {
  const vista_summarize_desc& d = a.desc;
  const Layout l = layout(d);
  const size_t rows = size_t(d.B) * d.H * d.S;
  auto floats = [&](size_t off) { return reinterpret_cast<float*>(a.workspace + off); };
  float* lse = floats(l.rows);
  float* delta = lse + align256(rows * sizeof(float)) / sizeof(float);
  HistoryGradParams p;
  p.X = static_cast<const uint16_t*>(a.X);
  p.Wk = static_cast<const uint16_t*>(a.Wk);
  p.Wv = static_cast<const uint16_t*>(a.Wv);
  p.Q = static_cast<const uint16_t*>(a.Q);
  p.dO = static_cast<const uint16_t*>(d_out);
  p.offsets = a.offsets;
  p.stats = floats(l.stats);
  p.lse = lse;
  p.delta = delta;
  p.records = floats(l.records);
  p.dK = static_cast<uint16_t*>(d_keys);
  p.dV = static_cast<uint16_t*>(d_values);
  p.q_user_stride = d.q_user_stride;
  p.N = d.total_items;
  p.G = a.G;
  p.B = d.B;
  p.S = d.S;
  p.H = d.H;
  p.seg = a.seg;
  p.rows = (d.S + 31) / 32 * 32;
  p.scale = a.scale_plain;
  p.scale_log2 = a.scale_log2;
  float *Ks = nullptr, *Vs = nullptr, *own_p = nullptr, *own_ds = nullptr;
  if (d.flags & VISTA_FLAG_SELF_TERM) {
    Ks = floats(l.Ks);
    Vs = Ks + self_kv_bytes(d) / sizeof(float);
    own_p = floats(l.self);
    own_ds = own_p + align256(rows * sizeof(float)) / sizeof(float);
    if (launch_self_kv(d, a.Q, a.Wk, a.Wv, Ks, Vs, a.stream) != hipSuccess) return VISTA_ERR_HIP;
  }
  auto step = [&](bool grad) {
    if (p.N == 0) return hipSuccess;
    return d.d == 64 ? run<64>(p, grad, a.stream) : d.d == 128 ? run<128>(p, grad, a.stream) : run<256>(p, grad, a.stream);
  };
  const GradRows r = {a.offsets, d.B, d.S, d.d, d.H, a.seg, d.total_items, a.G, a.scale_plain, a.scale_log2, d.q_user_stride,
                      a.offsets_checked ? -1 : d.total_items, reinterpret_cast<int*>(a.workspace)};
  if (step(false) != hipSuccess) return VISTA_ERR_HIP;
  if (grad_join_stats(r, d.dtype, p.stats, d.S, lse, delta, a.Q, d_out, Ks, Vs, own_p, own_ds, a.stream) != hipSuccess)
    return VISTA_ERR_HIP;
  if (step(true) != hipSuccess) return VISTA_ERR_HIP;
  if (grad_join_queries(r, d.dtype, p.records, p.rows, 1.f / kLog2e, a.Q, d_out, Ks, own_p, own_ds, d_queries, d_self_keys,
                        d_self_values, a.stream) != hipSuccess)
    return VISTA_ERR_HIP;
  return VISTA_OK;
}

}  // namespace vista
