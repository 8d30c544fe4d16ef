// logprobs_narrow.h -- the gradient of log probabilities for rows of up to 256 elements
// (part of logprobs.h).  dz is never stored: one kernel computes a block of scores again,
// turns it into dz in registers and multiplies that on, once with the positions as its
// own rows (dX) and once with the table rows (dW).  Four products instead of three, but
// none of the 8 bytes a score that writing and reading dz twice costs, which bound rows
// this short: 16,384 x 16,384 bf16 of 64 / 256 elements 627 / 841 -> 249 / 666 us, 8 x
// 4,096 x 1,024 x 128 104 -> 78 us.
//
// A wave owns 32 rows, which stay in registers as the columns (B) of 32 x 32 x 16 MFMAs;
// the other side's rows stream through LDS in stages of 64.  Per tile of 32:
//   S    A: 32 streamed rows, B: the own rows            -> 16 scores a lane, of its column
//   dz   in registers; lane 32 h + n has streamed rows 8 q + 4 h + r of column n, which
//        are eight consecutive places of a contraction over the streamed rows if place
//        16 t + 8 h + i stands for row 16 t + 8 (i / 4) + 4 h + i % 4: so dz, rounded to
//        fp16, is at once the B operand of
//   P    A: the streamed side's transposed copy, its columns in that order -> own rows' sums
// The vector ALU (dz) takes about as long as the matrix cores (S and P) at 128 elements,
// and the two only overlap within a wave: a phase has the next tile's S, the last tile's P
// and this tile's dz side by side.  S of tile t + 1 and P of tile t - 1 need S operands
// one stage ahead of P's, so the two are loaded apart, each a whole stage ahead, with one
// barrier a stage.

template <int DD>
struct NarrowSize {
  static constexpr int CH = DD / 8;      // 16-byte chunks of a row
  static constexpr int SB = 64 * DD * 2; // a stage's streamed rows
  static constexpr int TB = DD * 128;    // their transposed copy
  static constexpr int LS = 64 * CH / 256, LT = DD * 8 / 256;  // loads of a thread
  static constexpr int SMEM = 2 * (SB + TB);
  __device__ static int fs(int r) { return CH == 8 ? (r >> 1) & 7 : r & 15; }  // slots c ^ fs(row)
  __device__ static int ft(int d) { return (d >> 1) & 7; }
};

struct NarrowArgs {
  const char *own, *stream;  // rows
  const char* t;             // the streamed side's copy, [D, ldt]
  int64_t os, ss, ts;        // instance strides in bytes
  int64_t ld, ldt;           // bytes of a row
  int nown, nstream, chunks, V;
  int64_t M;
  const float* bias;
  const RowGrad* rows;
  float scale;
  int per;                   // stages of a share
  OutArgs out;               // its raster: shares by blocks of 128 own rows
};

template <int DT, int DD, bool IS_X, bool BIAS, bool ENT>
__device__ __forceinline__ void narrow_run(const NarrowArgs& a, int id, char* smem) {
  using Z = NarrowSize<DD>;
  // per streamed row, three stages' worth: dX: the offset; dW: c0, c1, lse in units of
  // log 2, g (see dz_kernel) and the target
  __shared__ __attribute__((aligned(16))) float con_s[3][IS_X ? 1 : 4][64];
  __shared__ __attribute__((aligned(16))) int tgt_s[IS_X ? 1 : 3][64];
  __shared__ __attribute__((aligned(16))) uint16_t keep_s[3][64];  // all ones: takes part
  __shared__ int hit_s[3][4];  // dW: whether a target of the stage is among a wave's rows
  int sp, ob;
  int64_t b;
  if (!raster_place(a.out.grid, id, sp, ob, b)) return;
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int stages = (a.nstream + 63) / 64;
  const int s0 = sp * a.per, ns = min(a.per, stages - s0);
  const int own0 = ob * 128 + wave * 32, own = own0 + n;  // the lane's own row
  const char* stream = nt_uniform(a.stream + b * a.ss + (int64_t)s0 * 64 * a.ld);
  const char* tsrc = nt_uniform(a.t + b * a.ts + (int64_t)s0 * 128);
  const bool whole = a.chunks == Z::CH;

  // stage s (of this share): 64 rows into S buffer s & 1
  auto issue_s = [&](int s) {
    const int last = a.nstream - 1 - (s0 + s) * 64;
    char* dst = smem + (s & 1) * Z::SB + wave * 1024;
    const char* base = stream + (int64_t)s * 64 * a.ld;
#pragma unroll
    for (int u = 0; u < Z::LS; ++u) {
      const int at = u * 256 + tid, r = at / Z::CH, c = (at % Z::CH) ^ Z::fs(r);
      const uint32_t off = (uint32_t)min(r, last) * (uint32_t)a.ld + c * 16;
      if (whole) nt_dma16(base, off, dst + u * 4096);
      else nt_dma16(c < a.chunks ? base + off : (const char*)&nt_zero, dst + u * 4096);
    }
  };
  auto issue_t = [&](int s) {
    char* dst = smem + 2 * Z::SB + (s & 1) * Z::TB + wave * 1024;
    const char* base = tsrc + (int64_t)s * 128;
#pragma unroll
    for (int u = 0; u < Z::LT; ++u) {
      const int d = u * 32 + tid / 8, c = (tid % 8) ^ Z::ft(d);
      nt_dma16(base, (uint32_t)min(d, a.out.D - 1) * (uint32_t)a.ldt + c * 16, dst + u * 4096);
    }
  };
  // a streamed row's constants: fetched by one thread each, stored before the barrier
  // that the stage's first use lies behind
  struct Con {
    float4 f;
    int t;
    bool keep;
  } con;
  auto fetch_con = [&](int s) {
    const int i = (s0 + s) * 64 + tid;
    con.f = make_float4(0, 0, 0, 0);
    con.t = -1;
    con.keep = false;
    if (tid >= 64 || i >= a.nstream) return;
    if constexpr (IS_X) {
      if (BIAS) con.f.x = a.bias[b * a.V + i];
      con.keep = !BIAS || con.f.x != NEG_INF;
    } else {
      const RowGrad r = a.rows[b * a.M + i];
      con.f = make_float4(-DZ_UP * __builtin_fmaf(r.h, r.ent, r.g), -DZ_UP * LN2 * r.h,
                          r.lse * LOG2E, DZ_UP * r.g);
      con.keep = r.active;
      con.t = r.active ? r.target : -1;
    }
  };
  auto store_con = [&](int s) {
    const int k = s % 3;
    if (tid < 64) {
      con_s[k][0][tid] = con.f.x;
      if constexpr (!IS_X) {
        con_s[k][1][tid] = con.f.y;
        con_s[k][2][tid] = con.f.z;
        con_s[k][3][tid] = con.f.w;
        tgt_s[k][tid] = con.t;
        // (the wave that stores: all of the stage's targets at once)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint64_t m = __ballot((unsigned)(con.t - ob * 128 - 32 * w) < 32u);
          if (tid == 0) hit_s[k][w] = m != 0;
        }
      }
      keep_s[k][tid] = con.keep ? 0xffff : 0;
    }
  };

  // the own rows, and what the lane's own row needs
  uint4 b_own[DD / 16];
  {
    const char* row = a.own + b * a.os + (int64_t)min(own, a.nown - 1) * a.ld;
#pragma unroll
    for (int k = 0; k < DD / 16; ++k) {
      const int c = 2 * k + h;
      b_own[k] = c < a.chunks ? *reinterpret_cast<const uint4*>(row + c * 16) : make_uint4(0, 0, 0, 0);
    }
  }
  float c0 = 0.f, c1 = 0.f, lse2 = 0.f, gt = 0.f, bz = 0.f;
  int tgt = -1;
  uint32_t keep = 0;
  if (own < a.nown) {
    if constexpr (IS_X) {
      const RowGrad r = a.rows[b * a.M + own];
      c0 = -DZ_UP * __builtin_fmaf(r.h, r.ent, r.g);
      c1 = -DZ_UP * LN2 * r.h;
      lse2 = r.lse * LOG2E;
      gt = DZ_UP * r.g;
      tgt = r.active ? r.target : -1;
      keep = r.active ? ~0u : 0u;
    } else {
      if (BIAS) bz = a.bias[b * a.V + own];
      keep = BIAS && bz == NEG_INF ? 0u : ~0u;
    }
  }
  const float c2 = a.scale * LOG2E;

  const int ls = n * (DD * 2), lt = n * 128;
  auto s_prod = [&](f32x16& acc, int buf, int tile) {
    char* p = smem + buf * Z::SB + tile * (32 * DD * 2);
#pragma unroll
    for (int j = 0; j < 16; ++j) acc[j] = 0.f;
#pragma unroll
    for (int k = 0; k < DD / 16; ++k)
      acc = mfma32_chunk<DT>(nt_at<uint4>(p, ls + (((2 * k + h) ^ Z::fs(n)) << 4)), b_own[k], acc);
  };
  f32x16 acc2[DD / 32];
#pragma unroll
  for (int i = 0; i < DD / 32; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) acc2[i][j] = 0.f;
  auto p_prod = [&](const uint4 (&dz)[2], int buf, int tile) {
    char* p = smem + 2 * Z::SB + buf * Z::TB;
#pragma unroll
    for (int i = 0; i < DD / 32; ++i)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        acc2[i] = mfma32_chunk<DT_F16>(
            nt_at<uint4>(p, i * 4096 + lt + (((tile * 4 + 2 * t + h) ^ Z::ft(n)) << 4)), dz[t], acc2[i]);
  };
  // scores of tile `tile` of stage s -> dz in fp32
  auto dz_of = [&](f32x16& x, int s, int tile) {
    const int k = s % 3, at = tile * 32 + 4 * h;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      f32x4 f0, f1, fl, fb;
      if constexpr (IS_X) {
        if (BIAS) fb = *reinterpret_cast<const f32x4*>(&con_s[k][0][at + 8 * q]);
      } else {
        f0 = *reinterpret_cast<const f32x4*>(&con_s[k][0][at + 8 * q]);
        if (ENT) f1 = *reinterpret_cast<const f32x4*>(&con_s[k][1][at + 8 * q]);
        fl = *reinterpret_cast<const f32x4*>(&con_s[k][2][at + 8 * q]);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float z = x[4 * q + r], lz = IS_X ? lse2 : fl[r];
        float l;
        if constexpr (BIAS)  // in natural units: an offset may be the type's lowest value
          l = __builtin_fmaf(__builtin_fmaf(z, a.scale, IS_X ? fb[r] : bz), LOG2E, -lz);
        else
          l = __builtin_fmaf(z, c2, -lz);
        const float p = __builtin_amdgcn_exp2f(l), d0 = IS_X ? c0 : f0[r];
        if constexpr (ENT)
          x[4 * q + r] = p * __builtin_fmaf(BIAS ? __builtin_fmaxf(l, -1e30f) : l, IS_X ? c1 : f1[r], d0);
        else
          x[4 * q + r] = p * d0;
      }
    }
  };
  // g more at the targets, then fp16 (nothing from rows and tokens that take no part)
  auto pack = [&](f32x16& y, uint4 (&dz)[2], int s, int tile) {
    const int k = s % 3, at = tile * 32 + 4 * h;
    if constexpr (IS_X) {
      const int rel = tgt - ((s0 + s) * 64 + tile * 32) - 4 * h;
      if (__ballot((unsigned)(rel + 4 * h) < 32u)) {
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (rel == 8 * (j >> 2) + (j & 3)) y[j] += gt;
      }
    } else {
      if (__builtin_amdgcn_readfirstlane(hit_s[k][wave])) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int4 t = *reinterpret_cast<const int4*>(&tgt_s[k][at + 8 * q]);
          const f32x4 g = *reinterpret_cast<const f32x4*>(&con_s[k][3][at + 8 * q]);
          if (t.x == own) y[4 * q] += g[0];
          if (t.y == own) y[4 * q + 1] += g[1];
          if (t.z == own) y[4 * q + 2] += g[2];
          if (t.w == own) y[4 * q + 3] += g[3];
        }
      }
    }
    uint32_t w[8];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint2 m = *reinterpret_cast<const uint2*>(&keep_s[k][at + 8 * q]);
      w[2 * q] = half2_bits(y[4 * q], y[4 * q + 1]) & m.x & keep;
      w[2 * q + 1] = half2_bits(y[4 * q + 2], y[4 * q + 3]) & m.y & keep;
    }
    dz[0] = make_uint4(w[0], w[1], w[2], w[3]);
    dz[1] = make_uint4(w[4], w[5], w[6], w[7]);
  };

  issue_s(0);
  fetch_con(0);
  store_con(0);
  if (1 < ns) issue_s(1);
  issue_t(0);
  fetch_con(1);
  store_con(1);
  nt_wait_and_sync<0>();
  f32x16 x0, x1;
  uint4 dz0[2] = {}, dz1[2] = {};  // of the stage's tiles 0 and 1
  s_prod(x0, 0, 0);
  for (int s = 0; s < ns; ++s) {
    // tile 0's dz; the last stage's tile 1 multiplied on (nothing before the first)
    s_prod(x1, s & 1, 1);
    p_prod(dz1, s ? (s - 1) & 1 : 0, 1);
    dz_of(x0, s, 0);
    pack(x0, dz0, s, 0);
    nt_wait_and_sync<0>();  // S of stage s + 1, P's operand of stage s
    if (s + 2 < ns) issue_s(s + 2);
    if (s + 1 < ns) issue_t(s + 1);
    fetch_con(s + 2);
    s_prod(x0, (s + 1) & 1, 0);
    p_prod(dz0, s & 1, 0);
    dz_of(x1, s, 1);
    pack(x1, dz1, s, 1);
    store_con(s + 2);
  }
  p_prod(dz1, (ns - 1) & 1, 1);

  // 32 rows by 64 columns at a time through LDS, whole lines out, as in out_kernel
  __syncthreads();
  char* sq = smem + wave * 8192;
#pragma unroll
  for (int i = 0; i < DD / 64; ++i) {
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x16& y = acc2[2 * i + c];
        nt_at<f32x4>(sq, n * 256 + (((8 * c + 2 * q + h) ^ (n & 7)) << 4)) =
            f32x4{y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]};
      }
    const int d = 64 * i + 8 * (lane & 7);
#pragma unroll 1
    for (int j = 0; j < 32; j += 8) {
      const int rl = j + (lane >> 3);
      float v[8];
#pragma unroll
      for (int e = 0; e < 2; ++e)
        *reinterpret_cast<f32x4*>(v + 4 * e) =
            nt_at<f32x4>(sq, rl * 256 + (((2 * (lane & 7) + e) ^ (rl & 7)) << 4));
      if (own0 + rl < a.nown && d < a.out.D) out_store<DT>(a.out, b, sp, own0 + rl, d, v);
    }
  }
}

// Both sides in one launch: the workgroups past the first nx are dW's.
template <int DT, int DD, bool BIAS, bool ENT>
__global__ __launch_bounds__(256, DD <= 128 ? 2 : 1) void narrow_kernel(NarrowArgs x, NarrowArgs w,
                                                                        int nx) {
  __shared__ __attribute__((aligned(16))) char smem[NarrowSize<DD>::SMEM];
  if ((int)blockIdx.x < nx) narrow_run<DT, DD, true, BIAS, ENT>(x, blockIdx.x, smem);
  else narrow_run<DT, DD, false, BIAS, ENT>(w, blockIdx.x - nx, smem);
}
