// logprobs.h -- scores of rows against a whole token table and what follows from
// them (include/flashtokens.h): log-softmax, entropy, the best alternatives, and
// the gradients.  Instantiated per storage type in logprobs_bf16.hip and
// logprobs_f16.hip.
//
// One tiled product carries it all, P[a, b] = sum_c A[a, c] B[b, c] with both
// operands' contraction contiguous: 256 (or 128) rows of A by 256 rows of B to a
// workgroup of eight waves, each 2 (or 1) x 4 tiles of 32 x 32 x 16 MFMAs.  Stages of
// 64 elements of both operands go from L2 straight into one of two LDS buffers, a whole
// 128-byte line of a row at a time, while the MFMAs read the other conflict-free from
// swizzled rows.  A's rows lie in a lane's registers and B's across the lanes, so
// with the table as A a lane holds 32 scores of one position and the softmax's
// running maximum, sum and weighted sum stay in that lane until the last block.
#pragma once

#include <algorithm>

#include "fkm_device.h"
#include "tokens_internal.h"

namespace fkm {

namespace {

constexpr int NT_T = 512;  // threads of a workgroup
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;
constexpr float NEG_INF = -__builtin_inff();

__device__ const uint4 nt_zero = {0, 0, 0, 0};

// L2 -> LDS copies of 16 bytes a lane into the wave's slots at `lds`, issued
// by inline assembly so that only the explicit waits below govern them; M0 (the LDS
// base) is set in the same statement, one wait state before the load reads it.  From
// a scalar base and 32-bit offsets, or from 64-bit addresses.
__device__ __forceinline__ uint32_t nt_lds(char* lds) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)(lds);
}
// A pointer that all lanes share, in scalar registers.
__device__ __forceinline__ const char* nt_uniform(const char* p) {
  const uint64_t v = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((int)(uint32_t)v);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((int)(uint32_t)(v >> 32));
  return (const char*)(((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ void nt_dma16(const char* base, uint32_t off, char* lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :
               : "v"(off), "s"(base), "s"(nt_lds(lds))
               : "memory");
}
__device__ __forceinline__ void nt_dma16(const void* src, char* lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
               :
               : "v"(src), "s"(nt_lds(lds))
               : "memory");
}

// Until at most n of this wave's vector memory operations are in flight and its LDS
// reads are done, then a barrier that leaves the later loads in flight.
template <int n>
__device__ __forceinline__ void nt_wait_and_sync() {
  __builtin_amdgcn_s_waitcnt((n & 0xF) | ((n >> 4) << 14) | (7 << 4));
  asm volatile("s_barrier" ::: "memory");
}

// Row r of a stage keeps its eight 16-byte chunks in slots c ^ nt_swz(r): 16 rows' reads
// of one chunk then meet all 64 banks.
__device__ __forceinline__ int nt_swz(int r) { return (r >> 1) & 7; }

template <typename T>
__device__ __forceinline__ T& nt_at(char* base, int off) {
  return *reinterpret_cast<T*>(base + off);
}

constexpr int TCW = 2;  // tiles of 32 of A's rows that a wave has
struct NtSize {
  static constexpr int BA = 128 * TCW;      // rows of A in a block
  static constexpr int AB = BA * 128;       // bytes of A in a stage
  static constexpr int STAGE = AB + LP_BB * 128;
  static constexpr int LA = BA * 8 / NT_T, LB = LP_BB * 8 / NT_T;  // loads of a thread in a stage
  static constexpr int LOADS = LA + LB;
  static constexpr int SMEM = 2 * STAGE;
};

// The operands of a workgroup: rows a0 .. of A (nblk blocks) by rows b0 .. of B,
// chunks [c0, c1) of the contraction.  Rows past the last one are read as the last
// one (their results are dropped), chunks past c1 as zeros.
struct NtIn {
  const char *A, *B;
  int64_t lda, ldb;   // bytes of a row
  int nA, nB, a0, b0, c0, c1, nblk;
};

struct NtFrag {
  uint4 a[TCW], b[4];
};

template <int DT>
struct NtLoop {
  using Z = NtSize;
  NtIn in;
  // the stage to load next: block iblk, stage id of it; each operand's first row and
  // chunk of that stage, and the thread's offsets from it (rows clamped)
  const char *ab, *bb;
  uint32_t ao[Z::LA], bo[Z::LB];
  int tid, wave, cc, iblk, id, nds;
  int lo, wp, wc;
  char* smem;

  __device__ __forceinline__ void block_rows(int blk) {
    const int a0 = in.a0 + blk * Z::BA, last = in.nA - 1 - a0;
    ab = nt_uniform(in.A + (int64_t)a0 * in.lda + in.c0 * 16);
#pragma unroll
    for (int u = 0; u < Z::LA; ++u)
      ao[u] = (uint32_t)max(min((tid >> 3) + 64 * u, last), 0) * (uint32_t)in.lda + cc * 16;
  }

  __device__ __forceinline__ void init(const NtIn& i, char* sm) {
    in = i;
    smem = sm;
    tid = threadIdx.x;
    wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lane = tid & 63, n = lane & 31, h = lane >> 5;
    cc = (tid & 7) ^ nt_swz(tid >> 3);
    nds = (in.c1 - in.c0 + 7) / 8;
    iblk = id = 0;
    bb = nt_uniform(in.B + (int64_t)in.b0 * in.ldb + in.c0 * 16);
#pragma unroll
    for (int u = 0; u < Z::LB; ++u)
      bo[u] = (uint32_t)min((tid >> 3) + 64 * u, in.nB - 1 - in.b0) * (uint32_t)in.ldb + cc * 16;
    block_rows(0);
    // lane 32 h + n reads row (tile base + n), chunk 2 step + h
    lo = n * 128 + (h ^ nt_swz(n)) * 16;
    wp = wave & 1;   // half of B's rows
    wc = wave >> 1;  // quarter of A's rows
  }

  // Start the loads of the next stage.
  __device__ __forceinline__ void issue(char* buf) {
    char* dst = buf + wave * 1024;
    if (in.c0 + id * 8 + 8 <= in.c1) {
#pragma unroll
      for (int u = 0; u < Z::LA; ++u) nt_dma16(ab, ao[u], dst + u * (NT_T * 16));
#pragma unroll
      for (int u = 0; u < Z::LB; ++u) nt_dma16(bb + id * 128, bo[u], dst + Z::AB + u * (NT_T * 16));
    } else {  // the last stage of a contraction that is no whole number of them
      const bool have = in.c0 + id * 8 + cc < in.c1;
#pragma unroll
      for (int u = 0; u < Z::LA; ++u)
        nt_dma16(have ? ab + ao[u] : (const char*)&nt_zero, dst + u * (NT_T * 16));
#pragma unroll
      for (int u = 0; u < Z::LB; ++u)
        nt_dma16(have ? bb + id * 128 + bo[u] : (const char*)&nt_zero, dst + Z::AB + u * (NT_T * 16));
    }
    ab += 128;
    if (++id == nds) {
      id = 0;
      block_rows(++iblk);
    }
  }

  __device__ __forceinline__ void read(NtFrag& f, char* buf, int i) {  // i-th fragment
    if (i < TCW) f.a[i < TCW ? i : 0] = nt_at<uint4>(buf, (wc * TCW + i) * 4096);
    else f.b[i < TCW ? 0 : i - TCW] = nt_at<uint4>(buf, Z::AB + (wp * 4 + i - TCW) * 4096);
  }
  // Step k (16 elements) of a stage's buffer, at this lane's row.
  __device__ __forceinline__ char* step_at(char* buf, int k) { return buf + (lo ^ (k * 32)); }

  // The MFMAs of one 16-element step on `f`, in a fixed order with everything else that
  // the wave has to issue between them: the next step's fragments into `g` from `buf`,
  // then (if `load`) the loads of a later stage into `ahead`.  The matrix cores take 32
  // cycles an MFMA, so what stands between two of them is free; in a block of its own,
  // after the barrier and before the MFMAs, it cost both waves of a SIMD the same idle
  // cycles.
  __device__ __forceinline__ void step(f32x16 (&acc)[4][TCW], const NtFrag& f, NtFrag& g,
                                       char* buf, char* ahead, bool load) {
    constexpr int N = 4 * TCW, R = TCW + 4;
#pragma unroll
    for (int m = 0; m < N; ++m) {
      const int tp = m / TCW, tc = m % TCW;
      acc[tp][tc] = mfma32_chunk<DT>(f.a[tc], f.b[tp], acc[tp][tc]);
      __builtin_amdgcn_sched_barrier(0);
      // two reads after each of the first MFMAs (a step has at least 4)
      if (2 * m < R) read(g, buf, 2 * m);
      if (2 * m + 1 < R) read(g, buf, 2 * m + 1);
      if (m == N / 2 && load) issue(ahead);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // Stage s, whose first step's fragments are in f0.  Three steps read the next one's
  // fragments; then every wave has read the stage's buffer, and after a barrier, for
  // which stage s + 1 has to be there, the last step goes with the first fragments of
  // stage s + 1 and the loads of stage s + 2 (`load`) into this stage's buffer.  Past the
  // last stage the reads bring values that nobody uses; one path for all stages keeps
  // the accumulators in their registers.
  __device__ __forceinline__ void stage(int s, bool load, f32x16 (&acc)[4][TCW], NtFrag& f0,
                                        NtFrag& f1) {
    char *cur = at(s), *nxt = at(s + 1);
    step(acc, f0, f1, step_at(cur, 1), nullptr, false);
    step(acc, f1, f0, step_at(cur, 2), nullptr, false);
    step(acc, f0, f1, step_at(cur, 3), nullptr, false);
    nt_wait_and_sync<0>();
    step(acc, f1, f0, step_at(nxt, 0), cur, load);
  }
  __device__ __forceinline__ char* at(int s) { return smem + (s & 1) * Z::STAGE; }

  // epi(acc, block, scratch) after each block.  SCRATCH: the loads of the stage after the
  // next, into the buffer of the block's last stage, are put off until the wave is
  // through with its epilogue, which meanwhile has the parts of that buffer that these
  // loads of its own will fill: rows of 128 bytes, eight consecutive ones every 8 KiB
  // (scratch_row).
  template <bool SCRATCH, class Epi>
  __device__ __forceinline__ void run(Epi&& epi) {
    const int S = in.nblk * nds;
    issue(at(0));
    if (1 < S) issue(at(1));
    if (1 < S) nt_wait_and_sync<Z::LOADS>();
    else nt_wait_and_sync<0>();
    NtFrag f0, f1;
#pragma unroll
    for (int i = 0; i < TCW + 4; ++i) read(f0, step_at(at(0), 0), i);
    f32x16 acc[4][TCW];
    int s = 0;
    for (int g = 0; g < in.nblk; ++g) {
#pragma unroll
      for (int tp = 0; tp < 4; ++tp)
#pragma unroll
        for (int tc = 0; tc < TCW; ++tc)
#pragma unroll
          for (int j = 0; j < 16; ++j) acc[tp][tc][j] = 0.f;
      for (const int end = s + nds; s < end; ++s)
        stage(s, s + 2 < S && !(SCRATCH && s == end - 1), acc, f0, f1);
      epi(acc, g, at(s - 1) + wave * 1024);
      if (SCRATCH && s + 1 < S) issue(at(s - 1));
    }
  }
};
// Byte of row r (0 .. 31) of a wave's scratch.
__device__ __forceinline__ int scratch_row(int r) { return (r >> 3) * (NT_T * 16) + (r & 7) * 128; }

// The offsets of the wave's 64 columns from v0 on, one a lane (0 past the last).
__device__ __forceinline__ float bias_lane(const float* bias, int v0, int V) {
  const int v = v0 + (threadIdx.x & 63);
  return v < V ? bias[v] : 0.f;
}
// Those of columns at .. at + 3 (a multiple of 4, different between the half-waves).
__device__ __forceinline__ f32x4 bias_quad(float lane_bias, int at) {
  f32x4 x;
#pragma unroll
  for (int r = 0; r < 4; ++r)
    x[r] = __int_as_float(__builtin_amdgcn_ds_bpermute((at + r) * 4, __float_as_int(lane_bias)));
  return x;
}

// ---- softmax statistics ----------------------------------------------------------
// Of some scores z: m = max (at least -FLT_MAX), s = sum exp(z - m), t = sum
// exp(z - m) (z - m).  -inf scores add nothing.
struct Stat {
  float m, s, t;
};
__device__ __forceinline__ Stat stat_none() { return {-__FLT_MAX__, 0.f, 0.f}; }
// The same about a larger maximum m.
__device__ __forceinline__ void stat_raise(Stat& a, float m) {
  const float d = __builtin_fmaxf(a.m - m, -1e30f);
  const float f = __builtin_amdgcn_exp2f(d * LOG2E);
  a.t = f * __builtin_fmaf(d, a.s, a.t);
  a.s *= f;
  a.m = m;
}
__device__ __forceinline__ Stat stat_merge(Stat a, Stat b) {
  const float m = __builtin_fmaxf(a.m, b.m);
  stat_raise(a, m);
  stat_raise(b, m);
  return {m, a.s + b.s, a.t + b.t};
}

// ---- scores --------------------------------------------------------------------
// Share `sp` of n blocks among k: the first block past it, in a scalar register (the
// division runs on the vector ALU, whose results the compiler takes for different).
__device__ __forceinline__ int share_end(int n, int sp, int k) {
  return __builtin_amdgcn_readfirstlane((int)((int64_t)n * sp / k));
}

// Workgroup `id`: its blocks of A and B and instance; false past the last one.
__device__ __forceinline__ bool raster_place(const Raster& r, int id, int& a, int& b, int64_t& inst) {
  const int xcd = id & 7, j = id >> 3, size = r.ga * r.gb;
  const int64_t sup = (int64_t)(j / size) * 8 + xcd;
  const int nsa = (r.na + r.ga - 1) / r.ga, nsb = (r.nb + r.gb - 1) / r.gb, in = j % size;
  const int i = __builtin_amdgcn_readfirstlane((int)(sup / (nsa * nsb)));
  const int at = (int)(sup - (int64_t)i * (nsa * nsb));
  inst = i;
  a = __builtin_amdgcn_readfirstlane(at / nsb * r.ga + in / r.gb);
  b = __builtin_amdgcn_readfirstlane(at % nsb * r.gb + in % r.gb);
  return sup < r.supers && a < r.na && b < r.nb;
}

// (by value: a conditional between array elements puts the array into memory)
__device__ __forceinline__ float pick(bool c, float a, float b) { return c ? a : b; }

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t half2_bits(float a, float b) {
  return __builtin_bit_cast(uint32_t, half2_t{(_Float16)a, (_Float16)b});  // to nearest even
}
__device__ __forceinline__ uint32_t half2_mul(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2_t, a) * __builtin_bit_cast(half2_t, b));
}

// One workgroup: 256 rows of X by a share of the column blocks (all shares within one
// block of a size).
struct ScoreArgs {
  const char *X, *W;
  const float* bias;
  const int32_t* target;
  int64_t xs, ws, ts;    // instance strides: bytes, bytes, positions
  int64_t rows;          // rows of this block of rows
  int64_t ld;            // bytes of a row
  int V, chunks;         // 16-byte chunks of a row
  float scale;
  int vb0, nvb;          // the column blocks of this launch
  Raster grid;           // shares of them by row blocks
  int share0, shares;    // the first one's place among all of a row's
  float4* part;          // [B, shares, rows]
  float* zt;             // [B, rows]
  float *z, *gmax;       // [B, rows, ldz], [B, rows, groups]
  const float* bound;    // [B, rows] groups whose best does not exceed it are not stored; NULL: all are
  int64_t ldz, groups;
};

template <int DT, bool BIAS, bool TOPK>
__global__ __launch_bounds__(NT_T, 1) void score_kernel(ScoreArgs a) {
  using Z = NtSize;
  __shared__ __attribute__((aligned(16))) char smem[Z::SMEM];
  int mb, sp;
  int64_t b;
  if (!raster_place(a.grid, blockIdx.x, sp, mb, b)) return;
  const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
  const int blk0 = a.vb0 + share_end(a.nvb, sp, a.grid.na);
  const int blk1 = a.vb0 + share_end(a.nvb, sp + 1, a.grid.na);
  NtIn in;
  in.A = a.W + b * a.ws;
  in.B = a.X + b * a.xs;
  in.lda = in.ldb = a.ld;
  in.nA = a.V;
  in.nB = (int)a.rows;
  in.a0 = blk0 * 256;
  in.b0 = mb * LP_BB;
  in.c0 = 0;
  in.c1 = a.chunks;
  in.nblk = blk1 - blk0;
  NtLoop<DT> loop;
  loop.init(in, smem);
  const int wp = loop.wp, wc = loop.wc;
  // per row: the target, its score, the bound (in LDS: registers are short)
  __shared__ int tgt_s[LP_BB];
  __shared__ float zt_s[LP_BB], bound_s[TOPK ? LP_BB : 1];
  for (int r = threadIdx.x; r < LP_BB; r += NT_T) {
    const int64_t row = in.b0 + r;
    tgt_s[r] = a.target && row < a.rows ? a.target[b * a.ts + row] : -1;
    if (TOPK) bound_s[r] = a.bound && row < a.rows ? a.bound[b * a.rows + row] : NEG_INF;
  }
  Stat st[4];
#pragma unroll
  for (int tp = 0; tp < 4; ++tp) st[tp] = stat_none();
  __syncthreads();
  const float c2 = a.scale * LOG2E;
  auto epi = [&](f32x16(&acc)[4][2], int g, char* scratch) {
    const int v0 = in.a0 + g * 256 + wc * 64;  // the wave's 64 columns
    const float bl = BIAS ? bias_lane(a.bias + b * a.V, v0, a.V) : 0.f;
    const bool edge = v0 + 64 > a.V;
    if (BIAS || edge) {  // the scores themselves, with the offsets, into acc
#pragma unroll
      for (int tc = 0; tc < 2; ++tc)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          f32x4 x = {0, 0, 0, 0};
          const int at = tc * 32 + 8 * q + 4 * h;
          if constexpr (BIAS) x = bias_quad(bl, at);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            // a forbidden token's score is -inf, whatever its row holds
            const bool off = (BIAS && x[r] == NEG_INF) || v0 + at + r >= a.V;
#pragma unroll
            for (int tp = 0; tp < 4; ++tp) {
              const float z = __builtin_fmaf(acc[tp][tc][4 * q + r], a.scale, x[r]);
              acc[tp][tc][4 * q + r] = off ? NEG_INF : z;
            }
            __builtin_amdgcn_sched_barrier(0);  // one mask at a time: 32 of them spill
          }
        }
    }
    const float zs = BIAS || edge ? 1.f : a.scale;  // acc to scores
#pragma unroll
    for (int tp = 0; tp < 4; ++tp) {
      float lm, es = 0.f, et = 0.f;
      if (zs >= 0.f) {
        float x = acc[tp][0][0];
#pragma unroll
        for (int i = 1; i < 32; ++i) x = __builtin_fmaxf(x, acc[tp][i >> 4][i & 15]);
        lm = x * zs;
      } else {
        float x = acc[tp][0][0];
#pragma unroll
        for (int i = 1; i < 32; ++i) x = __builtin_fminf(x, acc[tp][i >> 4][i & 15]);
        lm = x * zs;
      }
      if (lm > st[tp].m) stat_raise(st[tp], lm);
      if (BIAS || edge) {  // in natural units: an offset may be the type's lowest value
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          const float u = acc[tp][i >> 4][i & 15] - st[tp].m;
          const float e = __builtin_amdgcn_exp2f(u * LOG2E);
          es += e;
          et = __builtin_fmaf(e, __builtin_fmaxf(u, -1e30f), et);  // 0 for -inf
        }
      } else {
        // in units of log 2, one fma: the vector ALU bounds this part, an exponential's
        // four cycles for each of the others' one.  The maximum's product rounds by
        // 2^-24 of it, as the scores themselves do.
        const float m2 = st[tp].m * LOG2E;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          const float u = __builtin_fmaf(acc[tp][i >> 4][i & 15], c2, -m2);
          const float e = __builtin_amdgcn_exp2f(u);
          es += e;
          et = __builtin_fmaf(e, u, et);
        }
        et *= LN2;
      }
      st[tp].s += es;
      st[tp].t += et;
      // the target, if it is among this lane's 32 columns
      const int rl = wp * 128 + tp * 32 + n, rel = tgt_s[rl] - v0;
      const bool hit = (unsigned)rel < 64u && ((rel >> 2) & 1) == h;
      if (__ballot(hit)) {  // halves of its 32 scores by the bits of its place among them
        float x[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) x[j] = pick(rel & 32, acc[tp][1][j], acc[tp][0][j]);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = pick(rel & 16, x[j + 8], x[j]);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = pick(rel & 8, x[j + 4], x[j]);
#pragma unroll
        for (int j = 0; j < 2; ++j) x[j] = pick(rel & 2, x[j + 2], x[j]);
        if (hit) zt_s[rl] = pick(rel & 1, x[1], x[0]) * zs;
      }
      if constexpr (TOPK) {
        const int64_t row = in.b0 + rl;
        const float gm = __builtin_fmaxf(lm, __shfl_xor(lm, 32));
        const bool keep = !a.bound || gm > bound_s[rl];
        if (row < a.rows && h == 0 && v0 < a.V)
          a.gmax[(b * a.rows + row) * a.groups + v0 / LP_GROUP] = keep ? gm : NEG_INF;
        // 32 x 32 scores at a time through the wave's part of the finished stage's
        // buffer (row n's 16-byte unit c at c ^ (n & 7)), so that whole lines are written:
        // straight from the lanes, 32 bytes of each of 32 rows, they took 2.5 times as long
        const uint64_t kept = __ballot(row < a.rows && keep);
        if (kept) {
          float* zr = a.z + (b * a.rows + in.b0 + wp * 128 + tp * 32) * a.ldz + v0;
#pragma unroll
          for (int tc = 0; tc < 2; ++tc) {
            const f32x16& x = acc[tp][tc];
#pragma unroll
            for (int q = 0; q < 4; ++q)
              nt_at<f32x4>(scratch, scratch_row(n) + (((2 * q + h) ^ (n & 7)) << 4)) =
                  f32x4{x[4 * q] * zs, x[4 * q + 1] * zs, x[4 * q + 2] * zs, x[4 * q + 3] * zs};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int r = 8 * i + (lane >> 3), c = lane & 7;
              const f32x4 y = nt_at<f32x4>(scratch, scratch_row(r) + ((c ^ (r & 7)) << 4));
              if (kept >> r & 1) *reinterpret_cast<f32x4*>(zr + r * a.ldz + tc * 32 + 4 * c) = y;
            }
          }
        }
      }
    }
  };
  loop.template run<TOPK>(epi);

  // the two lanes of a row, then the four waves that share it, in a fixed order
  __syncthreads();
  Stat* sh = reinterpret_cast<Stat*>(smem);  // [4][256]
#pragma unroll
  for (int tp = 0; tp < 4; ++tp) {
    const int rl = wp * 128 + tp * 32 + n;
    Stat o = {__shfl_xor(st[tp].m, 32), __shfl_xor(st[tp].s, 32), __shfl_xor(st[tp].t, 32)};
    o = stat_merge(h ? o : st[tp], h ? st[tp] : o);
    if (h == 0) sh[wc * LP_BB + rl] = o;
  }
  __syncthreads();
  for (int r = threadIdx.x; r < LP_BB; r += NT_T) {
    // a target among this share's columns has its score
    const int rel = tgt_s[r] - in.a0;
    if ((unsigned)tgt_s[r] < (unsigned)a.V && (unsigned)rel < (unsigned)(in.nblk * 256))
      a.zt[b * a.rows + in.b0 + r] = zt_s[r];
    Stat o = sh[r];
#pragma unroll
    for (int q = 1; q < 4; ++q) o = stat_merge(o, sh[q * LP_BB + r]);
    if (in.b0 + r < a.rows)
      a.part[(b * a.shares + a.share0 + sp) * a.rows + in.b0 + r] = make_float4(o.m, o.s, o.t, 0.f);
  }
}

// ---- few rows --------------------------------------------------------------------
// Up to 64 rows (a decoding step): the table streams through once, bound by HBM.  A
// workgroup owns 64 table rows and up to 64 positions (more positions with a small table,
// which then comes from L2 again, where tiles of 256 x 256 would leave the chip idle:
// 256 x 5,000 x 1,024: 52 -> 24 us); its four waves split the contraction
// in units of 64 elements (whole 128-byte lines of each row), each wave holding 4 x CB
// 16 x 16 x 32 MFMA tiles and loading the fragments of both operands straight into
// registers, two units ahead, without LDS or barriers.  The waves' sums meet in LDS,
// where each wave then has the 64 scores of a position in its lanes.  131,072 x 4,096
// bf16: one row 264 -> 187 us (5.7 TB/s), against the tiles of 256 positions.
struct FewArgs {
  const char *X, *W;
  const float* bias;
  const int32_t* target;
  int M, V, chunks;
  int64_t ld;  // bytes of a row
  float scale;
  float4* part;  // [B, blocks, M]
  float* zt;     // [B, M]
  float *z, *gmax;
  int64_t ldz, groups;
};

// ONCE: the table is read past the caches, for ones beyond the 256 MiB of the last cache
// (131,072 x 4,096: 214 -> 204 us; but 205 MB: 60 -> 62).
constexpr int FEW_LD = 68;  // floats from position to position: 64 scores and 4 of padding
template <int DT, int CB, bool ONCE>
__device__ __forceinline__ void few_products(const FewArgs& a, float (&red)[4][16 * CB * FEW_LD]) {
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, q4 = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t b = blockIdx.y;
  const int v0 = blockIdx.x * 64, m0 = blockIdx.z * (16 * CB);
  const char *pa[4], *pb[CB];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    pa[i] = a.W + (b * a.V + min(v0 + 16 * i + r16, a.V - 1)) * a.ld + q4 * 16;
#pragma unroll
  for (int i = 0; i < CB; ++i) pb[i] = a.X + (b * a.M + min(m0 + 16 * i + r16, a.M - 1)) * a.ld + q4 * 16;
  struct Unit {
    uint4 a[2][4], b[2][CB];
  };
  auto fetch = [&](Unit& f, int u) {
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      if constexpr (ONCE) {  // a table that no cache will hold until the next call
#pragma unroll
        for (int i = 0; i < 4; ++i)
          f.a[st][i] = __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(
                                                     pa[i] + (int64_t)u * 128 + st * 64)));
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          f.a[st][i] = *reinterpret_cast<const uint4*>(pa[i] + (int64_t)u * 128 + st * 64);
      }
#pragma unroll
      for (int i = 0; i < CB; ++i)
        f.b[st][i] = *reinterpret_cast<const uint4*>(pb[i] + (int64_t)u * 128 + st * 64);
    }
  };
  f32x4 acc[4][CB];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < CB; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
  auto mfma = [&](const Unit& f) {
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < CB; ++j) acc[i][j] = mfma_chunk<DT>(f.a[st][i], f.b[st][j], acc[i][j]);
  };
  const int full = a.chunks / 8;  // whole units; then one with what is left
  Unit f0, f1;
  int u = w;
  if (u < full) fetch(f0, u);
  if (u + 4 < full) fetch(f1, u + 4);
  for (; u + 4 < full; u += 8) {
    mfma(f0);
    if (u + 8 < full) fetch(f0, u + 8);
    mfma(f1);
    if (u + 12 < full) fetch(f1, u + 12);
  }
  if (u < full) mfma(f0);
  if (full * 8 < a.chunks && w == full % 4) {
    Unit f;
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      const bool in = full * 8 + st * 4 + q4 < a.chunks;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        f.a[st][i] = in ? *reinterpret_cast<const uint4*>(pa[i] + (int64_t)full * 128 + st * 64)
                        : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < CB; ++i)
        f.b[st][i] = in ? *reinterpret_cast<const uint4*>(pb[i] + (int64_t)full * 128 + st * 64)
                        : make_uint4(0, 0, 0, 0);
    }
    mfma(f);
  }
  // lane 16 q + c holds rows 4 q .. 4 q + 3 of column c
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < CB; ++j)
      *reinterpret_cast<f32x4*>(&red[w][(16 * j + r16) * FEW_LD + 16 * i + 4 * q4]) = acc[i][j];
  __syncthreads();
}

template <int DT, int CB, bool BIAS, bool TOPK, bool ONCE>
__global__ __launch_bounds__(256, CB <= 2 ? 3 : 2) void few_kernel(FewArgs a) {
  __shared__ __attribute__((aligned(16))) float red[4][16 * CB * FEW_LD];
  few_products<DT, CB, ONCE>(a, red);
  const int tid = threadIdx.x;
  const int64_t b = blockIdx.y;
  const int v0 = blockIdx.x * 64, m0 = blockIdx.z * (16 * CB);
  // 16 / CB lanes a position, 4 CB columns each
  constexpr int TPM = 16 / CB, VPT = 4 * CB;
  const int ml = tid / TPM, part = tid % TPM, m = m0 + ml;
  const int vb = v0 + part * VPT;
  float z[VPT], lm = NEG_INF;
#pragma unroll
  for (int j = 0; j < VPT; j += 4) {
    const int at = ml * FEW_LD + part * VPT + j;
    f32x4 x = (*reinterpret_cast<const f32x4*>(&red[0][at]) + *reinterpret_cast<const f32x4*>(&red[1][at])) +
              (*reinterpret_cast<const f32x4*>(&red[2][at]) + *reinterpret_cast<const f32x4*>(&red[3][at]));
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int v = vb + j + r;
      const float bz = BIAS && v < a.V ? a.bias[b * a.V + v] : 0.f;
      const bool off = v >= a.V || (BIAS && bz == NEG_INF);
      z[j + r] = off ? NEG_INF : __builtin_fmaf(x[r], a.scale, bz);
      lm = __builtin_fmaxf(lm, z[j + r]);
    }
  }
#pragma unroll
  for (int d = 1; d < TPM; d <<= 1) lm = __builtin_fmaxf(lm, __shfl_xor(lm, d));
  const float mx = __builtin_fmaxf(lm, -__FLT_MAX__);
  float s = 0.f, t = 0.f;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const float un = z[j] - mx, e = __builtin_amdgcn_exp2f(un * LOG2E);
    s += e;
    t = __builtin_fmaf(e, __builtin_fmaxf(un, -1e30f), t);
  }
#pragma unroll
  for (int d = 1; d < TPM; d <<= 1) {
    s += __shfl_xor(s, d);
    t += __shfl_xor(t, d);
  }
  if (m >= a.M) return;
  if (part == 0) a.part[(b * gridDim.x + blockIdx.x) * a.M + m] = make_float4(mx, s, t, 0.f);
  if (a.target) {
    const int rel = a.target[b * a.M + m] - vb;
#pragma unroll
    for (int j = 0; j < VPT; ++j)
      if (rel == j && vb + j < a.V) a.zt[b * a.M + m] = z[j];
  }
  if constexpr (TOPK) {
    if (part == 0) a.gmax[(b * a.M + m) * a.groups + blockIdx.x] = lm;
    float* zr = a.z + (b * a.M + m) * a.ldz + vb;
#pragma unroll
    for (int j = 0; j < VPT; j += 4)
      *reinterpret_cast<f32x4*>(zr + j) = f32x4{z[j], z[j + 1], z[j + 2], z[j + 3]};
  }
}

// ---- results of a row --------------------------------------------------------------
// Scores as integers in the same order (-0 as +0).
__device__ __forceinline__ uint32_t score_key(float v) {
  const uint32_t u = __float_as_uint(v + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_score(uint32_t u) {
  return __uint_as_float((u & 0x80000000u) ? (u & 0x7fffffffu) : ~u);
}

// The k-th largest of a wave's 256 keys, or something below it that exactly k reach.
__device__ __forceinline__ uint32_t wave_kth(const uint32_t (&x)[4], int k) {
  uint32_t kth = 0;
  for (int bit = 31; bit >= 0; --bit) {
    const uint32_t c = kth | (1u << bit);
    int cnt = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) cnt += __popcll(__ballot(x[i] >= c));
    if (cnt >= k) kth = c;
    if (cnt == k) break;
  }
  return kth;
}

// A bound for the columns still to come, one wave per row: at least k of the first
// `groups` groups' bests reach it, so a later group is among a row's k best only if its
// own best exceeds it (at an equal score the earlier column is the better).
__global__ __launch_bounds__(256) void bound_kernel(const float* __restrict__ gmax, int64_t rows,
                                                    int64_t stride, int groups, int k,
                                                    float* __restrict__ bound) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= rows) return;
  uint32_t x[4] = {0, 0, 0, 0};
  for (int i = lane; i < groups; i += 256)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + 64 * j < groups) x[j] = max(x[j], score_key(gmax[row * stride + i + 64 * j]));
  const uint32_t kth = wave_kth(x, k);
  if (lane == 0) bound[row] = key_score(kth);
}

struct FinishArgs {
  const float4* part;
  const float* zt;
  const float *z, *gmax;
  const int32_t* target;
  int64_t rows, ts, ldz, groups;
  int splits, V, k;
  bool all;                        // every score is stored, not those that a bound keeps
  float *logprob, *entropy, *lse;  // of this block of rows; ts positions an instance
  int32_t* top_idx;
  float* top_logprob;
};

__device__ __forceinline__ void finish_row(const FinishArgs& a, int64_t b, int64_t row, const Stat& st,
                                           float logs) {
  const bool none = st.s == 0.f;  // every token is forbidden
  const int64_t o = b * a.ts + row;
  a.lse[o] = none ? NEG_INF : st.m + logs;
  if (a.entropy) a.entropy[o] = none ? 0.f : logs - st.t / st.s;
  if (a.target) {
    const int t = a.target[o];
    a.logprob[o] = (unsigned)t >= (unsigned)a.V ? 0.f
                   : none ? NEG_INF : (a.zt[b * a.rows + row] - st.m) - logs;
  }
}

// One thread per row: a few shares' statistics merged in order.
__global__ __launch_bounds__(256) void finish_rows_kernel(FinishArgs a) {
  const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x, b = blockIdx.y;
  if (row >= a.rows) return;
  Stat st = stat_none();
  for (int s0 = 0; s0 < a.splits; s0 += 8) {  // eight on their way at a time
    float4 p[8];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      p[u] = a.part[(b * a.splits + min(s0 + u, a.splits - 1)) * a.rows + row];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (s0 + u < a.splits) st = stat_merge(st, Stat{p[u].x, p[u].y, p[u].z});
  }
  finish_row(a, b, row, st, logf(st.s));
}

// One workgroup per row: many shares, and the k best.
//
// The k best lie in groups whose best score is among the k largest of those (ties to the
// lowest group): each of these groups has an entry as good as anything elsewhere.  Every
// thread keeps the best of its groups; the k-th largest of the 256 thread bests is a
// bound that k groups reach, few others do, and nothing below it is among the k best.
// The entries that reach it, gathered from those groups, are ranked against each other.
// Where too many reach it (equal scores, a large table's best tokens in one thread), the
// bound is raised to the k-th largest group best, which the lowest groups that reach it
// settle exactly, and the entries are taken one by one.
constexpr int TOP_GROUPS = 64, TOP_ENTRIES = 256;

template <bool TOPK>
__global__ __launch_bounds__(256) void finish_top_kernel(FinishArgs a) {
  const int64_t row = blockIdx.x, b = blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  __shared__ Stat sh[4];
  Stat st = stat_none();
  for (int s0 = tid; s0 < a.splits; s0 += 4 * 256) {  // four on their way at a time
    float4 p[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      p[u] = a.part[(b * a.splits + min(s0 + 256 * u, a.splits - 1)) * a.rows + row];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (s0 + 256 * u < a.splits) st = stat_merge(st, Stat{p[u].x, p[u].y, p[u].z});
  }
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const Stat o = {__shfl_xor(st.m, m), __shfl_xor(st.s, m), __shfl_xor(st.t, m)};
    st = stat_merge(lane & m ? o : st, lane & m ? st : o);
  }
  if (lane == 0) sh[w] = st;
  __syncthreads();
  st = stat_merge(stat_merge(sh[0], sh[1]), stat_merge(sh[2], sh[3]));
  const float logs = logf(st.s);
  if (tid == 0) finish_row(a, b, row, st, logs);
  if constexpr (TOPK) {
    __shared__ uint32_t best[256], ekey[TOP_ENTRIES];
    __shared__ int eidx[TOP_ENTRIES], sel[TOP_GROUPS];
    __shared__ uint32_t bound_s;
    __shared__ int ngroups, nentries, cnt_s[4];
    const float* gm = a.gmax + (b * a.rows + row) * a.groups;
    const float* zr = a.z + (b * a.rows + row) * a.ldz;
    const int G = (int)a.groups, k = a.k, kg = min(k, G);
    int32_t* ti = a.top_idx + (b * a.ts + row) * k;
    float* tl = a.top_logprob + (b * a.ts + row) * k;
    const bool none = st.s == 0.f;
    // a group with this best holds nothing (and its scores may not be stored)
    const uint32_t nothing = score_key(NEG_INF);
    auto put = [&](int j, uint32_t key, int v) {  // forbidden tokens are no alternatives
      const bool have = key > nothing && v < a.V && !none;
      ti[j] = have ? v : -1;
      tl[j] = have ? (key_score(key) - st.m) - logs : NEG_INF;
    };
    // with few groups (a table of up to 4,096 rows) the entries themselves, if all are stored
    const bool direct = a.all && G <= TOP_GROUPS;
    uint32_t mine = 0;
    const float* src = direct ? zr : gm;
    const int nsrc = direct ? a.V : G;
    for (int i0 = tid; i0 < nsrc; i0 += 8 * 256) {
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = src[min(i0 + 256 * u, nsrc - 1)];  // the last one again
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (i0 + 256 * u < nsrc) mine = max(mine, score_key(x[u]));
    }
    best[tid] = mine;
    if (tid == 0) ngroups = nentries = 0;
    __syncthreads();
    if (w == 0) {  // the k-th largest of the thread bests
      uint32_t x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = best[lane + 64 * i];
      const uint32_t kth = wave_kth(x, k);
      if (lane == 0) bound_s = kth;
    }
    __syncthreads();
    const uint32_t bound = bound_s;
    auto entry = [&](float z, int v) {
      const uint32_t key = score_key(z);
      if (key >= bound) {
        const int at = atomicAdd(&nentries, 1);
        if (at < TOP_ENTRIES) ekey[at] = key, eidx[at] = v;
      }
    };
    for (int i0 = tid; i0 < nsrc; i0 += 8 * 256) {
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = src[min(i0 + 256 * u, nsrc - 1)];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int i = i0 + 256 * u;
        if (i >= nsrc) continue;
        if (direct) {
          entry(x[u], i);
        } else if (score_key(x[u]) >= max(bound, nothing + 1)) {
          const int at = atomicAdd(&ngroups, 1);
          if (at < TOP_GROUPS) sel[at] = i;
        }
      }
    }
    if (!direct) {
      __syncthreads();
      const int ng = ngroups;
      if (ng > TOP_GROUPS) {
        if (tid == 0) nentries = TOP_ENTRIES + 1;
      } else {
        for (int i0 = w; i0 < ng; i0 += 4 * 8) {
          float x[8];
#pragma unroll
          for (int u = 0; u < 8; ++u) x[u] = zr[sel[min(i0 + 4 * u, ng - 1)] * LP_GROUP + lane];
#pragma unroll
          for (int u = 0; u < 8; ++u)
            if (i0 + 4 * u < ng) entry(x[u], sel[i0 + 4 * u] * LP_GROUP + lane);
        }
      }
    }
    __syncthreads();
    const int n = nentries;
    if (n <= TOP_ENTRIES) {
      if (tid >= n && tid < k) put(tid, 0u, -1);  // fewer than k are allowed

      // each entry's rank: whichever way they were gathered, the order is the same
      if (tid < n) {
        const uint32_t key = ekey[tid];
        const int v = eidx[tid];
        int rank = 0;
        for (int i = 0; i < n; ++i) {
          const uint32_t o = ekey[i];
          rank += o > key || (o == key && eidx[i] < v) ? 1 : 0;
        }
        if (rank < k) put(rank, key, v);
      }
      return;
    }
    // exactly: the kg-th largest group best, then the lowest groups that reach it
    auto count = [&](uint32_t c, bool over) {  // groups whose best reaches (exceeds) c
      int n = 0;
      for (int i = tid; i < G; i += 256) {
        const uint32_t key = score_key(gm[i]);
        n += over ? key > c : key >= c;
      }
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) n += __shfl_xor(n, m);
      __syncthreads();
      if (lane == 0) cnt_s[w] = n;
      __syncthreads();
      return cnt_s[0] + cnt_s[1] + cnt_s[2] + cnt_s[3];
    };
    uint32_t kth = 0;
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t c = kth | (1u << bit);
      if (count(c, false) >= kg) kth = c;
    }
    int ties = kg - count(kth, true), got = 0;
    __syncthreads();
    if (w != 0) return;
    for (int i0 = 0; i0 < G && got < kg; i0 += 64) {
      const uint32_t key = i0 + lane < G ? score_key(gm[i0 + lane]) : 0u;
      const bool in = i0 + lane < G, tie = in && key == kth;
      const uint64_t tm = __ballot(tie), below = (1ull << lane) - 1;
      const bool take = (in && key > kth) || (tie && __popcll(tm & below) < ties);
      const uint64_t km = __ballot(take);
      if (take) sel[got + __popcll(km & below)] = i0 + lane;
      got += __popcll(km);
      ties -= min(ties, (int)__popcll(tm));
    }
    __builtin_amdgcn_wave_barrier();
    uint32_t key[TOK_MAX_K];  // entry `lane` of each chosen group; groups in ascending order
#pragma unroll
    for (int i = 0; i < TOK_MAX_K; ++i)
      key[i] = i < kg && score_key(gm[sel[i]]) > nothing
                   ? score_key(zr[(int64_t)sel[i] * LP_GROUP + lane]) : 0u;
    for (int j = 0; j < k; ++j) {
      uint32_t top = 0;
      int at = -1;
#pragma unroll
      for (int i = 0; i < TOK_MAX_K; ++i)
        if (key[i] > top) top = key[i], at = i;
      const int v = at >= 0 ? sel[at] * LP_GROUP + lane : 0x7fffffff;
      uint32_t wb = top;
      int wv = v;
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) {
        const uint32_t ob = __shfl_xor(wb, m);
        const int ov = __shfl_xor(wv, m);
        if (ob > wb || (ob == wb && ov < wv)) wb = ob, wv = ov;
      }
      if (at >= 0 && v == wv) {
#pragma unroll
        for (int i = 0; i < TOK_MAX_K; ++i)
          if (i == at) key[i] = 0u;
      }
      if (lane == 0) put(j, wb, wv);
    }
  }
}

// Eight products more.
template <int DT>
__device__ __forceinline__ float dot_chunk(const uint4& x, const uint4& y, float z) {
  const uint32_t a[4] = {x.x, x.y, x.z, x.w}, b[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    z = __builtin_fmaf(Elem<DT>::widen((uint16_t)a[i]), Elem<DT>::widen((uint16_t)b[i]), z);
    z = __builtin_fmaf(Elem<DT>::widen((uint16_t)(a[i] >> 16)), Elem<DT>::widen((uint16_t)(b[i] >> 16)), z);
  }
  return z;
}

// ---- gradient ------------------------------------------------------------------
// dz and the copies of X and W that the two products read are fp16 for both storage
// types: 11 significant bits against bf16's 8 make dz's rounding an eighth, below that
// of the results (bf16 dz: dX and dW off by 2.4e-3 of their norm, 1.7e-3 being their own
// rounding; fp16: 1.7e-3).  All three are kept in range: each row's dz is stored over gs
// and DZ_UP times larger; X and W times the power of two that brings their largest value
// just below 2^15, where fp16 holds every bf16 or fp16 value down to 2^-29 of that
// exactly.  gs is a power of two at or above max(|g|, |h|).  dW sums over rows of
// different gs: X's copy is times gs over the largest gs, but for what dz's transpose
// takes of that (faint_part).
// dz's rounding is then, with fp16 results, as large as theirs, and one relative error of
// a row wherever one dz, the target's, makes most of it: over many rows 1.4 times the
// results' own rounding, over few up to 2.3 times (1 position, 8 x 8,931 x 586: 3.5e-4).
// So for up to LP_EXACT fp16 positions gs is dz of the target wherever that is the
// largest: it has no rounding then, and X's copies, rounded each for itself, bring less
// into dW (the same: 2.2e-4, 2.1e-4 being the results' own rounding).
constexpr float DZ_UP = 2048.f;

// Of a row whose gs is 2^-k of the largest, the factor that dz's transpose takes: nothing
// down to 2^-12, then half of the exponent up to 14, so that with the rest in X's copy
// either stays in fp16's normal range down to 2^-40 (all of it in X's copy: to 2^-25 or so,
// and at 2^-36 a third of the row's dW was left).
__device__ __forceinline__ float faint_part(float gs, float top) {
  int a, b;
  (void)frexpf(top, &a);
  (void)frexpf(gs, &b);
  return ldexpf(1.f, -min(max((a - b - 12) / 2, 0), 14));
}

// fp32 holds an lse far from 0 to half a step only: from FAR on, where that is 2^-12 and
// more of p (an offset of -2^20 that all of a row's tokens share: 6%; of the type's lowest
// value: p = 1 for each of them), a row's maximum and sum are taken again and kept apart.
constexpr float FAR = 4096.f;

// Both of up to 16 rows by a workgroup of 512 threads: a wave takes every eighth 16 table
// rows against all of them in 16 x 16 x 32 MFMAs, fragments straight from memory (x: of
// the lane's row, lane % 16).  sh: 8 x 16 values; the results in the first 16.  Bound by
// latency: one row or 16 of 65,536 x 1,024 take their workgroup 4.6 ms, 4,096 of them the
// call 9.3 ms instead of 2.0 (one row at a time 79).
constexpr int FAR_R = 16;
template <int DT>
__device__ __forceinline__ void far_stats(const uint16_t* x, const uint16_t* W, const float* bias,
                                          float scale, int V, int D, Stat* sh) {
  constexpr int U = 8;
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, q4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), ch = D / 8;
  const uint4* xc = reinterpret_cast<const uint4*>(x) + q4;
  Stat st = stat_none();
  for (int v0 = wave * 16; v0 < V; v0 += 128) {
    const uint4* wc = reinterpret_cast<const uint4*>(W + (int64_t)min(v0 + r16, V - 1) * D) + q4;
    f32x4 acc = {0, 0, 0, 0};
    for (int c = 0; c < ch; c += 4 * U) {  // U on their way at a time, zeros past the last
      uint4 a[U], b[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool in = c + 4 * u + q4 < ch;
        a[u] = in ? wc[c + 4 * u] : make_uint4(0, 0, 0, 0);
        b[u] = in ? xc[c + 4 * u] : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) acc = mfma_chunk<DT>(a[u], b[u], acc);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {  // table row v0 + 4 q4 + r, the lane's row
      const int v = v0 + 4 * q4 + r;
      const float bz = v < V ? bias[v] : NEG_INF;
      if (bz == NEG_INF) continue;
      const float z = __builtin_fmaf(acc[r], scale, bz);
      if (z > st.m) stat_raise(st, z);
      st.s += __builtin_amdgcn_exp2f((z - st.m) * LOG2E);
    }
  }
#pragma unroll
  for (int m = 16; m < 64; m <<= 1) {
    const Stat o = {__shfl_xor(st.m, m), __shfl_xor(st.s, m), 0.f};
    st = stat_merge(lane & m ? o : st, lane & m ? st : o);
  }
  __syncthreads();
  if (q4 == 0) sh[wave * FAR_R + r16] = st;
  __syncthreads();
  if (tid < FAR_R) {
    for (int i = 1; i < 8; ++i) sh[tid] = stat_merge(sh[tid], sh[i * FAR_R + tid]);
  }
}

// What each position's gradient needs, and the largest gs and magnitudes: X's of the
// rows that take part, W's of the tokens that do.  A workgroup goes over blocks of `rbx`
// rows (about 64 KiB; with offsets fewer, as far ones may follow) of X, or past the first
// `nx` workgroups of `rbw` of W: first a thread per row, then all threads through the rows' 16-byte chunks.
template <int DT, bool BIAS>
__global__ __launch_bounds__(512) void grad_rows_kernel(
    const uint16_t* __restrict__ X, const uint16_t* __restrict__ W, const int32_t* __restrict__ target,
    const float* __restrict__ lse, const float* __restrict__ ent, const float* __restrict__ g,
    const float* __restrict__ h, const float* __restrict__ bias, float scale, bool exact, int64_t M,
    int V, int D, int rbx, int rbw, int nx, RowGrad* __restrict__ out, float4* __restrict__ stats) {
  __shared__ float sh[8][2];
  __shared__ bool part[512];
  __shared__ float zt_s[DT == DT_F16 ? 512 : 1];
  __shared__ float lse_s[BIAS ? 512 : 1], more_s[BIAS ? 512 : 1];
  __shared__ Stat far_s[BIAS ? 8 * FAR_R : 1];
  __shared__ int16_t far_q[BIAS ? 512 + FAR_R : 1];
  __shared__ int far_n;
  const int64_t b = blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const bool is_x = (int)blockIdx.x < nx;
  const int rb = is_x ? rbx : rbw;
  const int64_t rows = is_x ? M : V, nblk = is_x ? nx : gridDim.x - nx;
  const uint16_t* in = (is_x ? X : W) + b * rows * D;
  float gsmax = 0.f;
  uint32_t mag = 0;  // the largest magnitude's bits, which order as the values do
  constexpr uint32_t FIN = DT == DT_BF16 ? 0x7f7f : 0x7bff;  // the largest finite one
  auto one = [&](uint32_t v) {
    v &= 0x7fffu;
    return v > FIN ? 0u : v;
  };
  for (int64_t r0 = (is_x ? blockIdx.x : blockIdx.x - nx) * (int64_t)rb; r0 < rows; r0 += nblk * rb) {
    const int nr = (int)min<int64_t>(rb, rows - r0);
    if (BIAS && is_x) {
      bool far = false;
      if (tid < nr) {
        const int64_t i = b * M + r0 + tid;
        const float l = lse[i];
        far = __builtin_fabsf(l) >= FAR && l != NEG_INF && (g[i] != 0.f || (h && h[i] != 0.f));
        lse_s[tid] = l;
        more_s[tid] = 0.f;
        part[tid] = far;
      }
      if (__syncthreads_or(far)) {
        if (tid == 0) {  // the far rows, the last of them once more to a whole group
          int n = 0;
          for (int q = 0; q < nr; ++q)
            if (part[q]) far_q[n++] = q;
          for (int e = 0; e < FAR_R; ++e) far_q[n + e] = far_q[n - 1];
          far_n = n;
        }
        __syncthreads();
        for (int i = 0; i < far_n; i += FAR_R) {
          far_stats<DT>(in + (r0 + far_q[i + (tid & 15)]) * D, W + b * V * D, bias + b * V, scale, V, D,
                        far_s);
          if (tid < FAR_R && i + tid < far_n) {
            lse_s[far_q[i + tid]] = far_s[tid].m;
            more_s[far_q[i + tid]] = log2f(far_s[tid].s);
          }
        }
        __syncthreads();
      }
    }
    if (DT == DT_F16 && exact) {
      if (is_x) {
        // the targets' scores: `lpr` lanes a row, four rows of each at a time
        const int ch = D / 8, lpr = ch > 32 ? 64 : ch > 16 ? 32 : ch > 8 ? 16 : 8;
        const int step = 512 / lpr, l = tid % lpr;
        for (int q0 = tid / lpr; q0 < nr; q0 += 4 * step) {
          int t[4];
          float z[4] = {0, 0, 0, 0};
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            t[u] = target[b * M + r0 + min(q0 + u * step, nr - 1)];
            if ((unsigned)t[u] >= (unsigned)V) t[u] = 0;  // (not used)
          }
          for (int c = l; c < ch; c += lpr) {
            uint4 x[4], y[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              x[u] = reinterpret_cast<const uint4*>(in + (r0 + min(q0 + u * step, nr - 1)) * D)[c];
              y[u] = reinterpret_cast<const uint4*>(W + (b * V + t[u]) * D)[c];
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) z[u] = dot_chunk<DT>(x[u], y[u], z[u]);
          }
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            for (int m = 1; m < lpr; m <<= 1) z[u] += __shfl_xor(z[u], m);
            if (l == 0 && q0 + u * step < nr) zt_s[q0 + u * step] = scale * z[u];
          }
        }
      }
      __syncthreads();
    }
    if (tid < nr) {
      if (is_x) {
        const int64_t i = b * M + r0 + tid;
        RowGrad r;
        const int t = target[i];
        const bool ok = (unsigned)t < (unsigned)V;
        r.target = ok && (!BIAS || bias[b * V + (ok ? t : 0)] != NEG_INF) ? t : -1;
        r.lse = BIAS ? lse_s[tid] : lse[i];
        const float more = BIAS ? more_s[tid] : 0.f;  // (see RowGrad)
        r.part = 1.f;
        r.g = r.target >= 0 ? g[i] : 0.f;
        float rh = h ? h[i] : 0.f;
        const float re = h ? ent[i] : 0.f;
        r.active = r.lse != NEG_INF && (r.g != 0.f || rh != 0.f);
        r.gs = 1.f;
        const float big = __builtin_fmaxf(__builtin_fabsf(r.g), __builtin_fabsf(rh));
        float u = 0.f;  // dz of the target, where it is the row's largest
        if (DT == DT_F16 && exact) {
          if (r.active && r.target >= 0) {
            const float z = zt_s[tid] + (BIAS ? bias[b * V + r.target] : 0.f);
            const float lp = __builtin_fminf((z - r.lse) - more * LN2, 0.f), p = __expf(lp);
            if (rh == 0.f) {
              u = r.g * __builtin_fmaxf(1.f - p, 0x1p-8f);
            } else {
              u = r.g * (1.f - p) - (p > 0.f ? rh * p * (lp + re) : 0.f);
              if (__builtin_fabsf(u) < 0.25f * big) u = 0.f;
            }
            const float a = __builtin_fabsf(u);
            if (!(a > 0x1p-100f && a < 0x1p100f && big < 0x1p100f)) u = 0.f;
          }
        }
        if (u != 0.f) {
          r.gs = u;
          r.g /= u;
          rh /= u;
        } else if (r.active && big <= __FLT_MAX__) {
          int e;
          (void)frexpf(big, &e);
          e = min(max(e, -120), 120);
          r.gs = copysignf(ldexpf(1.f, e), r.g);
          r.g *= copysignf(ldexpf(1.f, -e), r.g);
          rh *= 1.f / r.gs;
        }
        r.c0 = -DZ_UP * __builtin_fmaf(rh, re, r.g);
        r.c1 = -DZ_UP * LN2 * rh;
        r.g *= DZ_UP;
        if (BIAS) {
          const float f = __builtin_amdgcn_exp2f(-more);
          r.c0 = f * __builtin_fmaf(-more, r.c1, r.c0);
          r.c1 *= f;
        } else {
          r.lse *= LOG2E;
        }
        out[i] = r;
        part[tid] = r.active;
        if (r.active) gsmax = __builtin_fmaxf(gsmax, __builtin_fabsf(r.gs));
      } else {
        part[tid] = !BIAS || bias[b * V + r0 + tid] != NEG_INF;
      }
    }
    __syncthreads();
    const uint16_t* p = in + r0 * D;
    const int rc = D / 8, n = nr * rc;  // (D: the padded rows')
    for (int i0 = tid; i0 < n; i0 += 4 * 512) {
      uint4 q[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        q[u] = *reinterpret_cast<const uint4*>(p + (int64_t)min(i0 + u * 512, n - 1) * 8);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint32_t x[4] = {q[u].x, q[u].y, q[u].z, q[u].w};
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) m = max(m, max(one(x[e]), one(x[e] >> 16)));
        mag = max(mag, part[min(i0 + u * 512, n - 1) / rc] ? m : 0u);
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    mag = max(mag, (uint32_t)__shfl_xor((int)mag, d));
    gsmax = __builtin_fmaxf(gsmax, __shfl_xor(gsmax, d));
  }
  if (lane == 0) {
    sh[w][0] = gsmax;
    sh[w][1] = Elem<DT>::widen((uint16_t)mag);
  }
  __syncthreads();
  if (tid == 0) {
    float gm = 0.f, m = 0.f;
    for (int i = 0; i < 8; ++i) {
      gm = __builtin_fmaxf(gm, sh[i][0]);
      m = __builtin_fmaxf(m, sh[i][1]);
    }
    stats[b * gridDim.x + blockIdx.x] = make_float4(gm, is_x ? m : 0.f, is_x ? 0.f : m, 0.f);
  }
}

// The power of two that brings values of magnitude up to m below 2^15.
__device__ __forceinline__ float up_to_2_15(float m) {
  if (!(m > 0.f)) return 1.f;
  int e;
  (void)frexpf(m, &e);
  return ldexpf(1.f, min(15 - e, 126));
}
// (largest gs, factor of X, factor of W) from n statistics, by 256 threads.
__device__ __forceinline__ float4 grad_scales(const float4* stats, int n, float4* sh) {
  float4 o = make_float4(0, 0, 0, 0);
  auto take = [&](const float4& s) {
    o.x = __builtin_fmaxf(o.x, s.x);
    o.y = __builtin_fmaxf(o.y, s.y);
    o.z = __builtin_fmaxf(o.z, s.z);
  };
  for (int i = threadIdx.x; i < n; i += 256) take(stats[i]);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1)
    take(make_float4(__shfl_xor(o.x, d), __shfl_xor(o.y, d), __shfl_xor(o.z, d), 0.f));
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = o;
  __syncthreads();
  for (int i = 0; i < 4; ++i) take(sh[i]);
  return make_float4(o.x > 0.f ? o.x : 1.f, up_to_2_15(o.y), up_to_2_15(o.z), 0.f);
}

// Transposed fp16 copies: in [nb, R, ld] rows r0 .. r0 + nr - 1 of each instance, times a
// factor, -> out [nb, C, ldo] (C of their ld elements), zeros up to np.  Rows that take no
// part become zeros: of X those without a gradient (the others times gs over the largest
// too, but for faint_part, which the rows' constants for dW get), of W the forbidden
// tokens.  64 x 64 values at a time: a thread reads 8 columns of two rows and stores them
// in LDS as pairs of rows, and writes 8 rows of two columns.
struct CopyJob {
  const uint16_t* in;
  int64_t R, r0, nr, np, ldo;
  RowGrad* rows;      // of X, whose `part` is set
  const float* bias;  // of W
  uint16_t* out;
  int tiles;  // np / 64; 0: no such job
  bool mixed; // columns 16 t + 8 h + i hold rows 16 t + 8 (i / 4) + 4 h + i % 4
};
template <int DT>
__global__ __launch_bounds__(256) void copy_kernel(CopyJob x, CopyJob w, int C, int ld,
                                                   const float4* __restrict__ stats, int nstats,
                                                   float4* __restrict__ scales) {
  __shared__ float4 sh[4];
  constexpr int LD = 33;  // pairs from column to column: no conflicts on writes
  __shared__ uint32_t tile[64 * LD];
  const bool is_x = (int)blockIdx.x < x.tiles;
  const CopyJob j = is_x ? x : w;
  const int64_t b = blockIdx.z, rt = (int64_t)((int)blockIdx.x - (is_x ? 0 : x.tiles)) * 64;
  const int ct = blockIdx.y * 64, t = threadIdx.x;
  const float4 sc = grad_scales(stats + b * nstats, nstats, sh);
  if (blockIdx.x == 0 && blockIdx.y == 0 && t == 0) scales[b] = sc;  // for the products
  {
    const int c8 = t % 8, rp = t / 8;  // 8 columns of rows 2 rp, 2 rp + 1
    uint16_t v[2][8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t r = rt + 2 * rp + i;
      float f = 0.f;
      if (r < j.nr) {
        const int64_t ri = b * j.R + j.r0 + r;
        if (is_x) {
          const float gs = j.rows[ri].gs, part = faint_part(gs, sc.x);
          f = j.rows[ri].active ? gs / sc.x * sc.y / part : 0.f;
          if (blockIdx.y == 0 && c8 == 0) {
            j.rows[ri].g *= part;
            j.rows[ri].c0 *= part;
            j.rows[ri].c1 *= part;
            j.rows[ri].part = part;
          }
        } else f = j.bias && j.bias[ri] == NEG_INF ? 0.f : sc.z;
      }
      alignas(16) uint16_t x8[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      const int c = ct + 8 * c8;
      if (f != 0.f && c < C) {
        *reinterpret_cast<uint4*>(x8) =
            *reinterpret_cast<const uint4*>(j.in + (b * j.R + j.r0 + r) * ld + c);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e)
        v[i][e] = f != 0.f ? Elem<DT_F16>::narrow(Elem<DT>::widen(x8[e]) * f) : (uint16_t)0;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      tile[(8 * c8 + e) * LD + rp] = v[0][e] | ((uint32_t)v[1][e] << 16);
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int r8 = t % 8, cl = t / 8 + 32 * u, c = ct + cl;
    const int64_t r = rt + 8 * r8;
    const uint32_t* q = tile + cl * LD + (j.mixed ? 8 * (r8 >> 1) + 2 * (r8 & 1) : 4 * r8);
    const int up = j.mixed ? 4 : 2;  // pairs to the second half
    if (c < C && r < j.np)
      *reinterpret_cast<uint4*>(j.out + (b * C + c) * j.ldo + r) = make_uint4(q[0], q[1], q[up], q[up + 1]);
  }
}

struct DzArgs {
  const char *X, *W;
  const float* bias;
  const RowGrad* rows;
  int64_t xs, ws;   // instance strides in bytes
  int64_t M, ld;
  int V, v0, nv;    // all table rows; the block of them
  int chunks;
  float scale;
  uint16_t *dz, *dzt;  // [nb, M, lv], [nb, Vp, lm], zeros up to Vp and Mp
  int64_t Vp, Mp, lv, lm;
  Raster grid;         // shares of the block's 256-column blocks by row blocks
};

// dz of 256 positions by a share of the column blocks, in fp16, and its transpose.  The
// scores come as in score_kernel.  32 x 64 values at a time go through the wave's part of the
// finished stage's buffer, so that lines of both results are written whole.
template <int DT, bool BIAS, bool ENT>
__global__ __launch_bounds__(NT_T, 1) void dz_kernel(DzArgs a) {
  using Z = NtSize;
  __shared__ __attribute__((aligned(16))) char smem[Z::SMEM];
  __shared__ float4 row_s[LP_BB];  // c0, c1, lse, g
  __shared__ int tgt_s[LP_BB];     // -1: none; -2: the row takes no part
  __shared__ __attribute__((aligned(16))) uint32_t part_s[LP_BB];  // `part` twice
  __shared__ uint64_t faint_s[LP_BB / 64];  // the rows with one
  int sp, bb;
  int64_t b;
  if (!raster_place(a.grid, blockIdx.x, sp, bb, b)) return;
  const int nvb = (a.nv + 255) / 256;
  const int blk0 = share_end(nvb, sp, a.grid.na), blk1 = share_end(nvb, sp + 1, a.grid.na);
  NtIn in;
  in.A = a.W + b * a.ws;
  in.B = a.X + b * a.xs;
  in.lda = in.ldb = a.ld;
  in.nA = a.v0 + a.nv;
  in.nB = (int)a.M;
  in.a0 = a.v0 + blk0 * 256;
  in.b0 = bb * LP_BB;
  in.c0 = 0;
  in.c1 = a.chunks;
  in.nblk = blk1 - blk0;
  for (int r = threadIdx.x; r < LP_BB; r += NT_T) {
    RowGrad rg;
    rg.active = 0;
    if (in.b0 + r < a.M) rg = a.rows[b * a.M + in.b0 + r];
    tgt_s[r] = rg.active ? rg.target : -2;
    const float f = rg.active ? rg.part : 1.f, up = 1.f / f;
    row_s[r] = make_float4(rg.c0 * up, rg.c1 * up, rg.lse, rg.g * up);
    part_s[r] = half2_bits(f, f);
    const uint64_t faint = __ballot(f != 1.f);
    if ((r & 63) == 0) faint_s[r / 64] = faint;
  }
  __syncthreads();
  NtLoop<DT> loop;
  loop.init(in, smem);
  const int wp = loop.wp, wc = loop.wc;
  const float c2 = a.scale * LOG2E;
  uint16_t* dz = a.dz + b * a.M * a.lv;
  uint16_t* dzt = a.dzt + b * a.Vp * a.lm;
  auto epi = [&](f32x16(&acc)[4][2], int g, char* scratch) {
    // the lane as a new value, or the addresses below stay in registers through the loop
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    const int n = lane & 31, h = lane >> 5;
    const int v0 = in.a0 + g * 256 + wc * 64;  // the wave's 64 columns
    const float bl = BIAS ? bias_lane(a.bias + b * a.V, v0, a.V) : 0.f;
    const bool edge = v0 + 64 > in.nA;
    char* sq = scratch;
    // unit u (8 bytes: 4 columns) of row r at u ^ (r & 15)
    auto at = [&](int r, int u) { return scratch_row(r) + ((u ^ (r & 15)) << 3); };
#pragma unroll
    for (int tp = 0; tp < 4; ++tp) {
      const int rl = wp * 128 + tp * 32 + n;
      const float4 rc = row_s[rl];
      const int tgt = tgt_s[rl], rel = tgt - v0 - 4 * h;
      const uint32_t keep = tgt == -2 ? 0u : ~0u;
      const bool hit = (unsigned)(tgt - v0) < 64u && (((tgt - v0) >> 2) & 1) == h;
      const bool hits = __ballot(hit) != 0;
#pragma unroll
      for (int tc = 0; tc < 2; ++tc)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          f32x4 bz = {0, 0, 0, 0};
          if constexpr (BIAS) bz = bias_quad(bl, tc * 32 + 8 * q + 4 * h);
          float y[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float x = acc[tp][tc][4 * q + r];
            float l;
            if constexpr (BIAS)  // in natural units: an offset may be the type's lowest value
              l = (__builtin_fmaf(x, a.scale, bz[r]) - rc.z) * LOG2E;
            else
              l = __builtin_fmaf(x, c2, -rc.z);
            const float p = __builtin_amdgcn_exp2f(l);
            if constexpr (ENT)
              y[r] = p * __builtin_fmaf(BIAS ? __builtin_fmaxf(l, -1e30f) : l, rc.y, rc.x);
            else
              y[r] = p * rc.x;
          }
          if (hits) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (rel == tc * 32 + 8 * q + r) y[r] += rc.w;
          }
          if (BIAS || edge) {  // forbidden tokens and columns past the last
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if ((BIAS && bz[r] == NEG_INF) || v0 + 4 * h + tc * 32 + 8 * q + r >= in.nA) y[r] = 0.f;
          }
          nt_at<uint2>(sq, at(n, tc * 8 + 2 * q + h)) =
              make_uint2(half2_bits(y[0], y[1]) & keep, half2_bits(y[2], y[3]) & keep);
        }
      __builtin_amdgcn_sched_barrier(0);
      const int64_t m0 = in.b0 + wp * 128 + tp * 32;
      const int vb = v0 - a.v0;  // within the block of table rows
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 8 * i + (lane >> 3), c = lane & 7;  // 8 columns of row r
        const uint2 lo = nt_at<uint2>(sq, at(r, 2 * c)), hi = nt_at<uint2>(sq, at(r, 2 * c + 1));
        if (m0 + r < a.M && vb + 8 * c < a.Vp)
          *reinterpret_cast<uint4*>(dz + (m0 + r) * a.lv + vb + 8 * c) = make_uint4(lo.x, lo.y, hi.x, hi.y);
      }
      // columns 2 n, 2 n + 1 of 16 rows
      uint32_t x[16];
#pragma unroll
      for (int i = 0; i < 16; ++i)
        x[i] = nt_at<uint32_t>(sq, at(16 * h + i, n >> 1) + (n & 1) * 4);
      if (faint_s[wp * 2 + tp / 2]) {
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const uint4 f = *reinterpret_cast<const uint4*>(&part_s[wp * 128 + tp * 32 + 16 * h + i]);
          x[i] = half2_mul(x[i], f.x);
          x[i + 1] = half2_mul(x[i + 1], f.y);
          x[i + 2] = half2_mul(x[i + 2], f.z);
          x[i + 3] = half2_mul(x[i + 3], f.w);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      if (vb + 2 * n < a.Vp) {
#pragma unroll
        for (int o = 0; o < 2; ++o) {
          if (m0 + 16 * h + 8 * o >= a.Mp) continue;
          uint32_t lo[4], hi[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            lo[e] = (x[8 * o + 2 * e] & 0xffffu) | (x[8 * o + 2 * e + 1] << 16);
            hi[e] = (x[8 * o + 2 * e] >> 16) | (x[8 * o + 2 * e + 1] & 0xffff0000u);
          }
          uint16_t* t = dzt + (int64_t)(vb + 2 * n) * a.lm + m0 + 16 * h + 8 * o;
          *reinterpret_cast<uint4*>(t) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
          *reinterpret_cast<uint4*>(t + a.lm) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  loop.template run<true>(epi);
}

// The same of few rows (see few_kernel, whose products these are): a lane has 4 CB
// columns of a position, and the transpose goes through LDS to whole lines.  2 x 3,178 x
// 1,472: the call 96 -> 42 us.
template <int DT, int CB, bool BIAS, bool ENT>
__global__ __launch_bounds__(256, CB <= 2 ? 3 : 2) void few_dz_kernel(
    FewArgs a, const RowGrad* __restrict__ rows, uint16_t* __restrict__ dz, uint16_t* __restrict__ dzt,
    int64_t lv, int64_t Vp, int64_t lm) {
  __shared__ __attribute__((aligned(16))) float red[4][16 * CB * FEW_LD];
  few_products<DT, CB, false>(a, red);
  constexpr int TPM = 16 / CB, VPT = 4 * CB, LT = 72;  // LT: elements from column to column
  const int tid = threadIdx.x, ml = tid / TPM, part = tid % TPM;
  const int64_t b = blockIdx.y;
  const int v0 = blockIdx.x * 64, m0 = blockIdx.z * (16 * CB), m = m0 + ml, vb = v0 + part * VPT;
  RowGrad rg;
  rg.active = 0;
  if (m < a.M) rg = rows[b * a.M + m];
  const float c2 = a.scale * LOG2E, fp = rg.active ? rg.part : 1.f;
  const float c0 = rg.c0 / fp, c1 = rg.c1 / fp, g = rg.g / fp;
  uint32_t y2[VPT / 2];
#pragma unroll
  for (int j = 0; j < VPT; j += 4) {
    const int at = ml * FEW_LD + part * VPT + j;
    const f32x4 x =
        (*reinterpret_cast<const f32x4*>(&red[0][at]) + *reinterpret_cast<const f32x4*>(&red[1][at])) +
        (*reinterpret_cast<const f32x4*>(&red[2][at]) + *reinterpret_cast<const f32x4*>(&red[3][at]));
    float y[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int v = vb + j + r;
      const float bz = BIAS && v < a.V ? a.bias[b * a.V + v] : 0.f;
      float l;
      if constexpr (BIAS)
        l = (__builtin_fmaf(x[r], a.scale, bz) - rg.lse) * LOG2E;
      else
        l = __builtin_fmaf(x[r], c2, -rg.lse);
      const float p = __builtin_amdgcn_exp2f(l);
      y[r] = ENT ? p * __builtin_fmaf(__builtin_fmaxf(l, -1e30f), c1, c0) : p * c0;
      if (v == rg.target) y[r] += g;
      if (!rg.active || v >= a.V || bz == NEG_INF) y[r] = 0.f;
    }
    y2[j / 2] = half2_bits(y[0], y[1]);
    y2[j / 2 + 1] = half2_bits(y[2], y[3]);
  }
  if (m < a.M) {
    uint16_t* o = dz + (b * a.M + m) * lv + vb;
#pragma unroll
    for (int j = 0; j < VPT / 2; j += 2) *reinterpret_cast<uint2*>(o + 2 * j) = make_uint2(y2[j], y2[j + 1]);
  }
#pragma unroll
  for (int j = 0; j < VPT / 2; ++j) y2[j] = half2_mul(y2[j], half2_bits(fp, fp));
  __syncthreads();
  uint16_t* tile = reinterpret_cast<uint16_t*>(&red[0][0]);
#pragma unroll
  for (int j = 0; j < VPT; ++j)
    tile[(part * VPT + j) * LT + ml] = (uint16_t)(y2[j / 2] >> (j % 2 * 16));
  __syncthreads();
#pragma unroll
  for (int u = 0; u < 2; ++u) {  // eight positions of a column a thread, zeros past the last
    const int at = u * 256 + tid, r = at / 8, c = at % 8;
    uint4 x = make_uint4(0, 0, 0, 0);
    if (8 * c < 16 * CB) x = *reinterpret_cast<const uint4*>(&tile[r * LT + 8 * c]);
    *reinterpret_cast<uint4*>(dzt + (b * Vp + v0 + r) * lm + m0 + 8 * c) = x;
  }
}

// ---- the two products of the gradient ----------------------------------------------
// out[r, d] = sum over c of At[d, c] Br[r, c]: At a transposed copy (D rows), Br dz or
// its transpose.  Shares of the contraction go to `part` in fp32; whole ones are
// written in 16 bits, or added to `acc` (dX over several blocks of table rows).
enum OutMode { OUT_16 = 0, OUT_PART = 1, OUT_FIRST = 2, OUT_ADD = 3 };
struct OutArgs {
  const char *At, *Br;
  int64_t as, bs;      // instance strides in bytes
  int64_t ld;          // bytes of a row of either
  int64_t R, os;       // rows, rows between instances of the output
  int D, chunks, per;  // chunks of the contraction, stages of a share
  int ldf;
  int splits, mode, lanes;
  float factor;
  const RowGrad* rows;   // dX: times gs of the row, over W's factor
  const float4* scales;  // dW (rows NULL): times the largest gs, over X's factor
  const float* bias;     // dW: offsets of its rows; NULL: none
  uint16_t* out;
  float* f32;          // part [nb, splits, R, ldf] or acc [R, ldf]
  Raster grid;         // instances: the shares of each
};

// An instance's factor, but for dX's rows' gs: once for all results, as a load and a
// division each time cost more than writing them (one position, 131,072 x 1,024: the
// call 425 -> 406 us).
__device__ __forceinline__ float out_factor(const OutArgs& a, int64_t b) {
  const float4 s = a.scales[b];
  return a.rows ? a.factor / s.z : a.factor / s.y * s.x;
}

// Eight consecutive results of a row (those below D) from `v`; zeros for rows that take no
// part, whose sums of zeros times a NaN of another row are none.  Rows of fp32 sums are
// ldf (D's multiple of 8) elements apart.  16-bit rows of other widths begin at any
// element (an instance's first one too): three aligned pairs and the two elements that
// are left (65 x 43,047 x 1,331: one by one 372 -> 305 us).
template <int DT>
__device__ __forceinline__ void out_store(const OutArgs& a, float f, int64_t b, int sp, int64_t r, int d,
                                          float (&v)[8]) {
  if (a.mode == OUT_16) {
    bool keep = true;
    if (a.rows) {
      f *= a.rows[b * a.os + r].gs;
      keep = a.rows[b * a.os + r].active;
    } else if (a.bias) {
      keep = a.bias[b * a.os + r] != NEG_INF;
    }
    uint16_t* o = a.out + (b * a.os + r) * a.D + d;
    alignas(16) uint16_t x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = keep ? Elem<DT>::narrow(v[e] * f) : (uint16_t)0;
    if (a.D % 8 == 0) {
      *reinterpret_cast<uint4*>(o) = *reinterpret_cast<const uint4*>(x);
    } else if (d + 8 <= a.D) {
      const bool odd = (uintptr_t)o & 2;
#pragma unroll
      for (int e = 0; e < 3; ++e) {
        const uint32_t even2 = x[2 * e] | (uint32_t)x[2 * e + 1] << 16;
        const uint32_t odd2 = x[2 * e + 1] | (uint32_t)x[2 * e + 2] << 16;
        *reinterpret_cast<uint32_t*>(o + 2 * e + (odd ? 1 : 0)) = odd ? odd2 : even2;
      }
      o[odd ? 0 : 6] = odd ? x[0] : x[6];
      o[7] = x[7];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (d + e < a.D) o[e] = x[e];
    }
  } else {
    float* p = a.mode == OUT_PART ? a.f32 + ((b * a.splits + sp) * a.R + r) * a.ldf + d
                                  : a.f32 + r * a.ldf + d;
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      f32x4 x = {v[e], v[e + 1], v[e + 2], v[e + 3]};
      if (a.mode == OUT_ADD) x += *reinterpret_cast<const f32x4*>(p + e);
      *reinterpret_cast<f32x4*>(p + e) = x;
    }
  }
}

// (Both products in one launch: the workgroups past the first np are q's.)
template <int DT>
__global__ __launch_bounds__(NT_T, 1) void out_kernel(OutArgs p, OutArgs q, int np) {
  using Z = NtSize;
  __shared__ __attribute__((aligned(16))) char smem[Z::SMEM];
  const bool is_p = (int)blockIdx.x < np;
  const OutArgs a = is_p ? p : q;
  int ab, bb;
  int64_t inst;
  if (!raster_place(a.grid, blockIdx.x - (is_p ? 0 : np), ab, bb, inst)) return;
  const int b = __builtin_amdgcn_readfirstlane((int)inst / a.splits);
  const int sp = (int)inst - b * a.splits;
  const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
  NtIn in;
  in.A = a.At + b * a.as;
  in.B = a.Br + b * a.bs;
  in.lda = in.ldb = a.ld;
  in.nA = a.D;
  in.nB = (int)a.R;
  in.a0 = ab * Z::BA;
  in.b0 = bb * LP_BB;
  in.c0 = sp * a.per * 8;
  in.c1 = min(a.chunks, in.c0 + a.per * 8);
  in.nblk = 1;
  NtLoop<DT_F16> loop;
  loop.init(in, smem);
  const int wp = loop.wp, wc = loop.wc;
  auto epi = [&](f32x16(&acc)[4][TCW], int, char*) {
    // 32 rows by 32 TCW columns at a time through the wave's own LDS, so that lines are
    // written whole: row n's 16-byte unit c at c ^ (n & 7)
    __syncthreads();  // every wave has read its last stage
    const float f = out_factor(a, b);
    char* sq = smem + loop.wave * (4096 * TCW);
    constexpr int LPR = 4 * TCW, RPI = 64 / LPR;  // lanes a row, rows a step
    const int d = in.a0 + wc * 32 * TCW + 8 * (lane % LPR);
#pragma unroll
    for (int tp = 0; tp < 4; ++tp) {
#pragma unroll
      for (int tc = 0; tc < TCW; ++tc)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          nt_at<f32x4>(sq, n * (128 * TCW) + (((8 * tc + 2 * q + h) ^ (n & 7)) << 4)) =
              f32x4{acc[tp][tc][4 * q], acc[tp][tc][4 * q + 1], acc[tp][tc][4 * q + 2],
                    acc[tp][tc][4 * q + 3]};
#pragma unroll 1
      for (int i = 0; i < 32; i += RPI) {
        const int rl = i + lane / LPR;
        const int64_t r = in.b0 + wp * 128 + tp * 32 + rl;
        float v[8];
#pragma unroll
        for (int e = 0; e < 2; ++e)
          *reinterpret_cast<f32x4*>(v + 4 * e) =
              nt_at<f32x4>(sq, rl * (128 * TCW) + (((2 * (lane % LPR) + e) ^ (rl & 7)) << 4));
        if (r < a.R && d < a.D) out_store<DT>(a, f, b, sp, r, d, v);
      }
    }
  };
  loop.template run<false>(epi);
}

// out[b, r, d] = the sum over the shares of part[b, s, r, d], times its factor: eight
// results by `lanes` threads, each with every lanes-th share in order, then a tree.
template <int DT>
__global__ __launch_bounds__(256) void out_reduce_kernel(OutArgs p, OutArgs q, int np, int64_t nb) {
  const bool is_p = (int)blockIdx.x < np;
  const OutArgs a = is_p ? p : q;
  const int dc = (a.D + 7) / 8, l = threadIdx.x % a.lanes, per = 256 / a.lanes;
  const int64_t n = nb * a.R * dc;
  const int64_t i = (int64_t)(blockIdx.x - (is_p ? 0 : np)) * per + threadIdx.x / a.lanes;
  OutArgs o = a;
  o.mode = OUT_16;
  const int64_t br = min(i, n - 1) / dc, b = br / a.R, r = br % a.R;
  const int d = (int)(min(i, n - 1) % dc) * 8;
  const float* from = a.f32 + (b * a.splits * a.R + r) * a.ldf + d;
  float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int s = l; s < a.splits; s += a.lanes) {
    const float* x = from + s * (a.R * a.ldf);
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      const f32x4 y = *reinterpret_cast<const f32x4*>(x + e);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[e + k] += y[k];
    }
  }
  for (int m = 1; m < a.lanes; m <<= 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += __shfl_xor(v[e], m);
  }
  if (l == 0 && i < n) out_store<DT>(o, out_factor(o, b), b, 0, r, d, v);
}

#include "logprobs_narrow.h"

// ---- launchers -------------------------------------------------------------------
template <int DT, int CB, bool ONCE>
hipError_t launch_few_once(const FewArgs& q, const LogprobsArgs& a, dim3 grid, hipStream_t s) {
  if (a.bias) {
    if (a.k) few_kernel<DT, CB, true, true, ONCE><<<grid, 256, 0, s>>>(q);
    else few_kernel<DT, CB, true, false, ONCE><<<grid, 256, 0, s>>>(q);
  } else {
    if (a.k) few_kernel<DT, CB, false, true, ONCE><<<grid, 256, 0, s>>>(q);
    else few_kernel<DT, CB, false, false, ONCE><<<grid, 256, 0, s>>>(q);
  }
  return hipGetLastError();
}
template <int DT, int CB>
hipError_t launch_few(const FewArgs& q, const LogprobsArgs& a, const LogprobsWs& w, hipStream_t s) {
  const dim3 grid((unsigned)w.plan.splits, (unsigned)a.B, (unsigned)((a.M + 16 * CB - 1) / (16 * CB)));
  return a.M <= LP_FEW_M && a.B * a.V * w.Dk * 2 > (256 << 20)
             ? launch_few_once<DT, CB, true>(q, a, grid, s)
             : launch_few_once<DT, CB, false>(q, a, grid, s);
}

template <int DT>
hipError_t launch_score(const ScoreArgs& q, const LogprobsArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)q.grid.blocks());
  if (a.bias) {
    if (a.k) score_kernel<DT, true, true><<<grid, NT_T, 0, s>>>(q);
    else score_kernel<DT, true, false><<<grid, NT_T, 0, s>>>(q);
  } else {
    if (a.k) score_kernel<DT, false, true><<<grid, NT_T, 0, s>>>(q);
    else score_kernel<DT, false, false><<<grid, NT_T, 0, s>>>(q);
  }
  return hipGetLastError();
}

template <int DT>
hipError_t launch_logprobs_dt(const LogprobsArgs& a, const LogprobsWs& w, hipStream_t s) {
  hipError_t e;
  const char *X = (const char*)a.X, *W = (const char*)a.W;
  if (w.Dk != a.D) {
    if ((e = launch_pad_both(X, a.B * a.M, w.xpad, W, a.B * a.V, w.wpad, a.D, s)) != hipSuccess)
      return e;
    X = (const char*)w.xpad;
    W = (const char*)w.wpad;
  }
  for (int64_t m0 = 0; m0 < a.M; m0 += w.plan.rows) {
    const int64_t rows = std::min(w.plan.rows, a.M - m0);
    if (w.plan.few) {
      const FewArgs q{X, W, a.bias, a.target, (int)a.M, (int)a.V, (int)(w.Dk / 8), w.Dk * 2, a.scale,
                      w.part, w.zt, w.z, w.gmax, w.ldz, w.groups};
      const int cb = (int)((a.M + 15) / 16);
      e = cb == 1 ? launch_few<DT, 1>(q, a, w, s) : cb == 2 ? launch_few<DT, 2>(q, a, w, s)
                                                            : launch_few<DT, 4>(q, a, w, s);
    } else {
      ScoreArgs q;
      q.X = X + m0 * w.Dk * 2;
      q.W = W;
      q.bias = a.bias;
      q.target = a.target ? a.target + m0 : nullptr;
      q.xs = a.M * w.Dk * 2;
      q.ws = a.V * w.Dk * 2;
      q.ts = a.M;
      q.rows = rows;
      q.ld = w.Dk * 2;
      q.V = (int)a.V;
      q.chunks = (int)(w.Dk / 8);
      q.scale = a.scale;
      q.shares = w.plan.head_splits + w.plan.splits;
      q.part = w.part;
      q.zt = w.zt;
      q.z = w.z;
      q.gmax = w.gmax;
      q.ldz = w.ldz;
      q.groups = w.groups;
      q.bound = nullptr;
      const int64_t nmb = (rows + LP_BB - 1) / LP_BB;
      q.vb0 = q.share0 = 0;
      if (w.plan.head) {
        q.nvb = w.plan.head;
        q.grid = make_raster(w.plan.head_splits, nmb, a.B);
        if ((e = launch_score<DT>(q, a, s)) != hipSuccess) return e;
        bound_kernel<<<dim3((unsigned)((a.B * rows + 3) / 4)), 256, 0, s>>>(
            w.gmax, a.B * rows, w.groups, w.plan.head * 4, a.k, w.bound);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        q.bound = w.bound;
        q.vb0 = w.plan.head;
        q.share0 = w.plan.head_splits;
      }
      q.nvb = (int)(w.ldz / 256) - q.vb0;
      q.grid = make_raster(w.plan.splits, nmb, a.B);
      e = launch_score<DT>(q, a, s);
    }
    if (e != hipSuccess) return e;
    FinishArgs f;
    f.part = w.part;
    f.zt = w.zt;
    f.z = w.z;
    f.gmax = w.gmax;
    f.target = a.target ? a.target + m0 : nullptr;
    f.rows = rows;
    f.ts = a.M;
    f.ldz = w.ldz;
    f.groups = w.groups;
    f.splits = w.plan.head_splits + w.plan.splits;
    f.V = (int)a.V;
    f.k = a.k;
    f.all = w.plan.head == 0;
    f.logprob = a.logprob + m0;
    f.entropy = a.entropy ? a.entropy + m0 : nullptr;
    f.lse = a.lse + m0;
    f.top_idx = a.top_idx + m0 * a.k;
    f.top_logprob = a.top_logprob + m0 * a.k;
    // a thread merges a few shares in a row; a workgroup many
    if (a.k) finish_top_kernel<true><<<dim3((unsigned)rows, (unsigned)a.B), 256, 0, s>>>(f);
    else if (f.splits > 32)
      finish_top_kernel<false><<<dim3((unsigned)rows, (unsigned)a.B), 256, 0, s>>>(f);
    else
      finish_rows_kernel<<<dim3((unsigned)((rows + 255) / 256), (unsigned)a.B), 256, 0, s>>>(f);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int DT>
hipError_t launch_reduce(OutArgs& p, OutArgs& q, int64_t nb, hipStream_t s) {
  // more threads to a result while there are few results: many shares of few rows would
  // be as many latencies one after another (one position, 131,072 x 1,024: the call
  // 519 -> 460 us)
  auto blocks = [&](OutArgs& a) -> int64_t {
    if (a.mode != OUT_PART) return 0;
    const int64_t n = nb * a.R * ((a.D + 7) / 8);
    a.lanes = 1;
    while (a.lanes < 64 && a.lanes * 4 <= a.splits && n * a.lanes < 65536) a.lanes *= 2;
    return (n * a.lanes + 255) / 256;
  };
  const int64_t np = blocks(p), nq = blocks(q);
  if (np + nq == 0) return hipSuccess;
  out_reduce_kernel<DT><<<dim3((unsigned)(np + nq)), 256, 0, s>>>(p, q, (int)np, nb);
  return hipGetLastError();
}

// Both products over nb instances: p's and q's contractions in `sp` and `sq` shares.
// `hold`: p's shares are joined later.
template <int DT>
hipError_t launch_out(OutArgs& p, int sp, OutArgs& q, int sq, int64_t nb, bool hold, hipStream_t s) {
  auto plan = [&](OutArgs& a, int splits) {
    const int nst = (a.chunks + 7) / 8;
    a.per = (nst + splits - 1) / splits;
    a.splits = (nst + a.per - 1) / a.per;
    a.grid = make_raster((a.D + 255) / 256,
                         (a.R + LP_BB - 1) / LP_BB, nb * a.splits);
    return a.grid.blocks();
  };
  const int64_t np = plan(p, sp), nq = plan(q, sq);
  const dim3 grid((unsigned)(np + nq));
  out_kernel<DT><<<grid, NT_T, 0, s>>>(p, q, (int)np);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  OutArgs none{};
  return launch_reduce<DT>(hold ? none : p, q, nb, s);
}

template <int DT, int DD>
hipError_t launch_narrow_dd(const GradArgs& a, const NarrowArgs& x, const NarrowArgs& w,
                            hipStream_t s) {
  const int64_t nx = x.out.grid.blocks();
  const dim3 grid((unsigned)(nx + w.out.grid.blocks()));
  if (a.bias) {
    if (a.h) narrow_kernel<DT, DD, true, true><<<grid, 256, 0, s>>>(x, w, (int)nx);
    else narrow_kernel<DT, DD, true, false><<<grid, 256, 0, s>>>(x, w, (int)nx);
  } else {
    if (a.h) narrow_kernel<DT, DD, false, true><<<grid, 256, 0, s>>>(x, w, (int)nx);
    else narrow_kernel<DT, DD, false, false><<<grid, 256, 0, s>>>(x, w, (int)nx);
  }
  return hipGetLastError();
}
template <int DT>
hipError_t launch_narrow(const GradArgs& a, const GradWs& g, const char* X, const char* W,
                         const float4* scales, int64_t lm, int64_t lv, hipStream_t s) {
  NarrowArgs x{};
  x.ld = g.Dk * 2;
  x.chunks = (int)(g.Dk / 8);
  x.V = (int)a.V;
  x.M = a.M;
  x.bias = a.bias;
  x.rows = g.rows;
  x.scale = a.scale;
  x.out.D = (int)a.D;
  x.out.ldf = (int)g.Dk;
  x.out.factor = (a.h ? a.scale : -a.scale) / DZ_UP;  // (see dz_of)
  x.out.scales = scales;
  NarrowArgs w = x;
  auto side = [&](NarrowArgs& n, const char* own, int64_t nown, const char* stream, int64_t nstream,
                  const void* t, int64_t ldt, int splits, void* out, float* part) {
    n.own = own;
    n.stream = stream;
    n.os = nown * n.ld;
    n.ss = nstream * n.ld;
    n.nown = (int)nown;
    n.nstream = (int)nstream;
    n.t = (const char*)t;
    n.ldt = ldt * 2;
    n.ts = a.D * n.ldt;
    const int64_t stages = (nstream + 63) / 64;
    n.per = (int)((stages + splits - 1) / splits);
    n.out.splits = (int)((stages + n.per - 1) / n.per);
    n.out.mode = n.out.splits > 1 ? OUT_PART : OUT_16;
    n.out.R = n.out.os = nown;
    n.out.out = (uint16_t*)out;
    n.out.f32 = part;
    n.out.grid = make_raster(n.out.splits, (nown + 127) / 128, a.B);
  };
  side(x, X, a.M, W, a.V, g.wt, lv, g.sx, a.dX, g.part);
  x.out.rows = g.rows;
  w.out.bias = a.bias;
  side(w, W, a.V, X, a.M, g.xt, lm, g.sw, a.dW,
       g.part + (x.out.mode == OUT_PART ? a.B * g.sx * a.M * g.Dk : 0));
  const hipError_t e = a.D <= 64 ? launch_narrow_dd<DT, 64>(a, x, w, s)
                       : a.D <= 128 ? launch_narrow_dd<DT, 128>(a, x, w, s)
                                    : launch_narrow_dd<DT, 256>(a, x, w, s);
  return e != hipSuccess ? e : launch_reduce<DT>(x.out, w.out, a.B, s);
}

template <int DT, int CB>
hipError_t launch_few_dz(const DzArgs& d, int64_t nb, bool ent, hipStream_t s) {
  FewArgs q{};
  q.X = d.X;
  q.W = d.W;
  q.bias = d.bias;
  q.M = (int)d.M;
  q.V = d.V;
  q.chunks = d.chunks;
  q.ld = d.ld;
  q.scale = d.scale;
  const dim3 grid((unsigned)(d.Vp / 64), (unsigned)nb, (unsigned)((d.M + 16 * CB - 1) / (16 * CB)));
  if (d.bias) {
    if (ent) few_dz_kernel<DT, CB, true, true><<<grid, 256, 0, s>>>(q, d.rows, d.dz, d.dzt, d.lv, d.Vp, d.lm);
    else few_dz_kernel<DT, CB, true, false><<<grid, 256, 0, s>>>(q, d.rows, d.dz, d.dzt, d.lv, d.Vp, d.lm);
  } else {
    if (ent) few_dz_kernel<DT, CB, false, true><<<grid, 256, 0, s>>>(q, d.rows, d.dz, d.dzt, d.lv, d.Vp, d.lm);
    else few_dz_kernel<DT, CB, false, false><<<grid, 256, 0, s>>>(q, d.rows, d.dz, d.dzt, d.lv, d.Vp, d.lm);
  }
  return hipGetLastError();
}

template <int DT>
hipError_t launch_grad_dt(const GradArgs& a, const GradWs& w, hipStream_t s) {
  hipError_t e;
  const char *X = (const char*)a.X, *W = (const char*)a.W;
  if (w.Dk != a.D) {
    if ((e = launch_pad_both(X, a.B * a.M, w.xpad, W, a.B * a.V, w.wpad, a.D, s)) != hipSuccess)
      return e;
    X = (const char*)w.xpad;
    W = (const char*)w.wpad;
  }
  const int64_t lm = grad_ld(w.Mp);
  // blocks of about 64 KiB of rows, at most STATS_WGS / 2 workgroups for each of X and W;
  // smaller ones for the few rows that wait for their targets' scores
  const bool exact = DT == DT_F16 && a.B * a.M <= LP_EXACT;
  const int64_t full = std::max<int64_t>(1, std::min<int64_t>(512, 32768 / w.Dk));
  const int64_t rb = exact ? std::min(full, std::max<int64_t>(16, a.V / 256)) : full;
  // with offsets one to a CU, if there are fewer: a far row takes its workgroup a table's worth
  const int64_t rbx = a.bias ? std::min(rb, std::max<int64_t>(1, a.B * a.M / 256)) : rb;
  const int64_t nx = std::min<int64_t>((a.M + rbx - 1) / rbx, STATS_WGS / 2);
  const int64_t wgs = nx + std::min<int64_t>((a.V + rb - 1) / rb, STATS_WGS / 2);
  auto grad_rows = a.bias ? grad_rows_kernel<DT, true> : grad_rows_kernel<DT, false>;
  grad_rows<<<dim3((unsigned)wgs, (unsigned)a.B), 512, 0, s>>>(
      (const uint16_t*)X, (const uint16_t*)W, a.target, a.lse, a.entropy, a.g, a.h, a.bias,
      a.scale, exact, a.M, (int)a.V, (int)w.Dk, (int)rbx, (int)rb, (int)nx, w.rows, w.stats);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  for (int64_t b0 = 0; b0 < a.B; b0 += w.nb) {
    const int64_t nb = std::min<int64_t>(w.nb, a.B - b0);
    RowGrad* rg = w.rows + b0 * a.M;
    float4* scales = w.scales + b0;
    const float* bias = a.bias ? a.bias + b0 * a.V : nullptr;
    int64_t shares = 0;  // of dX over the blocks of table rows
    for (int64_t v0 = 0; v0 < a.V; v0 += w.Vc) {
      const int64_t nv = std::min(w.Vc, a.V - v0), vp = (nv + 63) / 64 * 64, lv = grad_ld(vp);
      const CopyJob jx{(const uint16_t*)X + b0 * a.M * w.Dk, a.M, 0, a.M, w.Mp, lm, rg, nullptr,
                       (uint16_t*)w.xt, v0 ? 0 : (int)(w.Mp / 64), w.narrow};
      const CopyJob jw{(const uint16_t*)W + b0 * a.V * w.Dk, a.V, v0, nv, vp, lv, nullptr, bias,
                       (uint16_t*)w.wt, (int)(vp / 64), w.narrow};
      copy_kernel<DT><<<dim3((unsigned)(jx.tiles + jw.tiles), (unsigned)((a.D + 63) / 64), (unsigned)nb),
                        256, 0, s>>>(jx, jw, (int)a.D, (int)w.Dk, w.stats + b0 * wgs, (int)wgs, scales);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      if (w.narrow) {  // all instances and table rows at once
        if ((e = launch_narrow<DT>(a, w, X, W, scales, lm, lv, s)) != hipSuccess) return e;
        break;
      }
      DzArgs d;
      d.X = X + b0 * a.M * w.Dk * 2;
      d.W = W + b0 * a.V * w.Dk * 2;
      d.bias = bias;
      d.rows = rg;
      d.xs = a.M * w.Dk * 2;
      d.ws = a.V * w.Dk * 2;
      d.M = a.M;
      d.ld = w.Dk * 2;
      d.V = (int)a.V;
      d.v0 = (int)v0;
      d.nv = (int)nv;
      d.chunks = (int)(w.Dk / 8);
      d.scale = a.scale;
      d.dz = (uint16_t*)w.dz;
      d.dzt = (uint16_t*)w.dzt;
      d.Vp = vp;
      d.Mp = w.Mp;
      d.lv = lv;
      d.lm = lm;
      if (nv == a.V && score_few(nb, a.M, a.V, w.Dk)) {
        e = a.M <= 16 ? launch_few_dz<DT, 1>(d, nb, a.h, s) : a.M <= 32 ? launch_few_dz<DT, 2>(d, nb, a.h, s)
                                                                      : launch_few_dz<DT, 4>(d, nb, a.h, s);
        if (e != hipSuccess) return e;
      } else {
        const int64_t nmb = (a.M + LP_BB - 1) / LP_BB, nvb = (nv + 255) / 256;
        d.grid = make_raster(score_splits(nmb, nb, nvb, (w.Dk + LP_DC - 1) / LP_DC), nmb, nb);
        const dim3 grid((unsigned)d.grid.blocks());
        if (a.bias) {
          if (a.h) dz_kernel<DT, true, true><<<grid, NT_T, 0, s>>>(d);
          else dz_kernel<DT, true, false><<<grid, NT_T, 0, s>>>(d);
        } else {
          if (a.h) dz_kernel<DT, false, true><<<grid, NT_T, 0, s>>>(d);
          else dz_kernel<DT, false, false><<<grid, NT_T, 0, s>>>(d);
        }
        if ((e = hipGetLastError()) != hipSuccess) return e;
      }

      const bool whole = w.Vc >= a.V;  // one block of table rows
      OutArgs x{};
      x.D = (int)a.D;
      x.ldf = (int)w.Dk;
      x.factor = a.scale / DZ_UP;
      x.scales = scales;
      OutArgs q = x;
      // dX: positions by D, over the table rows of this block
      x.At = (const char*)w.wt;
      x.Br = (const char*)w.dz;
      x.ld = lv * 2;
      x.as = a.D * x.ld;
      x.bs = a.M * x.ld;
      x.R = x.os = a.M;
      x.chunks = (int)(vp / 8);
      x.rows = rg;
      x.out = (uint16_t*)a.dX + b0 * a.M * a.D;
      x.mode = w.sx > 1 ? OUT_PART : whole ? OUT_16 : v0 ? OUT_ADD : OUT_FIRST;
      x.f32 = whole ? w.part : w.accx + shares * a.M * w.Dk;
      // dW: the block's table rows by D, over the positions
      q.At = (const char*)w.xt;
      q.Br = (const char*)w.dzt;
      q.ld = lm * 2;
      q.as = a.D * q.ld;
      q.bs = vp * q.ld;
      q.R = nv;
      q.os = a.V;
      q.bias = bias ? bias + v0 : nullptr;
      q.chunks = (int)(w.Mp / 8);
      q.out = (uint16_t*)a.dW + (b0 * a.V + v0) * a.D;
      q.mode = w.sw > 1 ? OUT_PART : OUT_16;
      q.f32 = w.part + (whole && w.sx > 1 ? nb * w.sx * a.M * w.Dk : 0);
      if ((e = launch_out<DT>(x, w.sx, q, w.sw, nb, !whole, s)) != hipSuccess) return e;
      shares += w.sx > 1 ? x.splits : 0;
    }
    if (w.Vc < a.V) {  // dX from its fp32 sums
      OutArgs x{}, none{};
      x.D = (int)a.D;
      x.ldf = (int)w.Dk;
      x.R = x.os = a.M;
      x.splits = (int)std::max<int64_t>(1, shares);
      x.mode = OUT_PART;
      x.factor = a.scale / DZ_UP;
      x.rows = rg;
      x.scales = scales;
      x.out = (uint16_t*)a.dX + b0 * a.M * a.D;
      x.f32 = w.accx;
      if ((e = launch_reduce<DT>(x, none, 1, s)) != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

}  // namespace

}  // namespace fkm
