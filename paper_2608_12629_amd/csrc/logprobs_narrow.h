// logprobs_narrow.h -- the gradient of log probabilities for rows of up to 256 elements
// (part of logprobs.h).  dz is never stored: one kernel computes a block of scores again,
// turns it into dz in registers and multiplies that on, once with the positions as its
// own rows (dX) and once with the table rows (dW).  Four products instead of three, but
// none of the 8 bytes a score that writing and reading dz twice costs, which bound rows
// this short: 16,384 x 16,384 bf16 of 64 / 128 / 256 elements 627 / 703 / 848 -> 209 /
// 332 / 672 us, 8 x 4,096 x 1,024 x 128 104 -> 74 us.
//
// A wave owns 32 rows, which stay in registers as the columns (B) of 32 x 32 x 16 MFMAs;
// the other side's rows stream through LDS in stages of 64.  Per tile of 32:
//   S    A: 32 streamed rows, B: the own rows            -> 16 scores a lane, of its column
//   dz   in registers; lane 32 h + n has streamed rows 8 q + 4 h + r of column n, which
//        are eight consecutive places of a contraction over the streamed rows if place
//        16 t + 8 h + i stands for row 16 t + 8 (i / 4) + 4 h + i % 4: so dz, rounded to
//        fp16, is at once the B operand of
//   P    A: the streamed side's transposed copy, its columns in that order -> own rows' sums
// A phase has the next tile's S, the last tile's P and this tile's dz side by side, none
// of which waits for another.  S of tile t + 1 and P of tile t - 1 need S operands one
// stage ahead of P's, so the two are loaded apart, each a whole stage ahead, with one
// barrier a stage.  Latency bounds it: at 128 elements the matrix cores are busy for 44%
// of the time; without any of the loads, the LDS reads or the exponentials it takes 0-10%
// less.

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
  // per streamed row, three stages' worth (dX: the offset; dW: lz, g, then c0, c1 or l0; see dz_of)
  constexpr bool L0 = BIAS && !ENT;
  constexpr int NC = IS_X ? 1 : ENT ? 4 : L0 ? 3 : 2;
  __shared__ __attribute__((aligned(16))) float con_s[3][NC][64];
  __shared__ __attribute__((aligned(16))) int tgt_s[3][64];
  __shared__ __attribute__((aligned(16))) uint16_t keep_s[3][64];  // all ones: takes part
  // by wave; bits 0, 1: a target of tile 0, 1 is among its rows; 2: rows that take no part
  __shared__ int odd_s[3][4];
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
  uint32_t off_s[Z::LS], off_t[Z::LT];
#pragma unroll
  for (int u = 0; u < Z::LS; ++u) {
    const int at = u * 256 + tid, r = at / Z::CH, c = (at % Z::CH) ^ Z::fs(r);
    off_s[u] = (uint32_t)r * (uint32_t)a.ld + c * 16;
  }
#pragma unroll
  for (int u = 0; u < Z::LT; ++u) {
    const int d = u * 32 + tid / 8, c = (tid % 8) ^ Z::ft(d);
    off_t[u] = (uint32_t)min(d, a.out.D - 1) * (uint32_t)a.ldt + c * 16;
  }
  auto issue_s = [&](int s) {
    const int last = a.nstream - 1 - (s0 + s) * 64;
    char* dst = smem + (s & 1) * Z::SB + wave * 1024;
    const char* base = stream + (int64_t)s * 64 * a.ld;
    if (whole && last >= 63) {
#pragma unroll
      for (int u = 0; u < Z::LS; ++u) nt_dma16(base, off_s[u], dst + u * 4096);
    } else {  // the last row again after the last; zeros after a row's last chunk
#pragma unroll
      for (int u = 0; u < Z::LS; ++u) {
        const int at = u * 256 + tid, r = at / Z::CH, c = (at % Z::CH) ^ Z::fs(r);
        const uint32_t off = (uint32_t)min(r, last) * (uint32_t)a.ld + c * 16;
        nt_dma16(c < a.chunks ? base + off : (const char*)&nt_zero, dst + u * 4096);
      }
    }
  };
  auto issue_t = [&](int s) {
    char* dst = smem + 2 * Z::SB + (s & 1) * Z::TB + wave * 1024;
    const char* base = tsrc + (int64_t)s * 128;
#pragma unroll
    for (int u = 0; u < Z::LT; ++u) nt_dma16(base, off_t[u], dst + u * 4096);
  };
  // a streamed row's constants: fetched by one thread each, and stored a stage later when
  // the wait for the tiles has covered their loads too (a wait of their own would be one
  // for every load on its way)
  constexpr bool CON = !IS_X || BIAS;
  struct Con {
    float lz, l0, c0, c1, g;
    int t;
    bool keep;
  } con;
  auto row_con = [&](const RowGrad& r) {
    const float f = IS_X ? 1.f / r.part : 1.f;
    con.lz = r.lse;
    con.g = r.g * f;
    if constexpr (ENT) {
      con.c0 = r.c0 * f;
      con.c1 = r.c1 * f;
    } else {
      const float l0 = __builtin_log2f(-r.c0 * f);
      if constexpr (L0) con.l0 = l0;
      else con.lz -= l0;
      con.g = -con.g;
    }
    con.keep = r.active;
    con.t = r.active ? r.target : -1;
  };
  auto fetch_con = [&](int s) {
    const int i = (s0 + s) * 64 + tid;
    con = {0, 0, 0, 0, 0, -1, false};
    if (!CON || tid >= 64 || i >= a.nstream) return;
    if constexpr (IS_X) {
      con.lz = a.bias[b * a.V + i];
      con.keep = con.lz != NEG_INF;
    } else {
      row_con(a.rows[b * a.M + i]);
    }
  };
  auto store_con = [&](int s) {
    if (!CON || tid >= 64) return;
    const int k = s % 3;
    con_s[k][0][tid] = con.lz;
    if constexpr (!IS_X) {
      con_s[k][1][tid] = con.g;
      if constexpr (ENT) {
        con_s[k][2][tid] = con.c0;
        con_s[k][3][tid] = con.c1;
      }
      if constexpr (L0) con_s[k][2][tid] = con.l0;
      tgt_s[k][tid] = con.t;
    }
    keep_s[k][tid] = con.keep ? 0xffff : 0;
    const int out = __ballot(!con.keep) ? 4 : 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint64_t hit = IS_X ? 0 : __ballot((unsigned)(con.t - ob * 128 - 32 * w) < 32u);
      if (tid == 0) odd_s[k][w] = out | ((uint32_t)hit ? 1 : 0) | (hit >> 32 ? 2 : 0);
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
  float bz = 0.f;
  bool mine = false;  // the own row takes part
  con = {0, 0, 0, 0, 0, -1, false};
  if (own < a.nown) {
    if constexpr (IS_X) {
      row_con(a.rows[b * a.M + own]);
      mine = con.keep;
    } else {
      if (BIAS) bz = a.bias[b * a.V + own];
      mine = !BIAS || bz != NEG_INF;
    }
  }
  const Con o = con;
  const float c2 = a.scale * LOG2E;

  // where a lane's chunks of S and T lie, in the buffers of the next products: kept and
  // moved from buffer to buffer, as computing them again costs as much as dz does
  uint32_t at_s[DD / 16], at_t[4];
#pragma unroll
  for (int k = 0; k < DD / 16; ++k) at_s[k] = n * (DD * 2) + (((2 * k + h) ^ Z::fs(n)) << 4);
#pragma unroll
  for (int k = 0; k < 4; ++k) at_t[k] = 2 * Z::SB + n * 128 + (((2 * k + h) ^ Z::ft(n)) << 4);
  auto move = [](auto& at, uint32_t d) {
#pragma unroll
    for (auto& x : at) {
      x += d;
      asm volatile("" : "+v"(x));
    }
  };
  move(at_s, 0);
  move(at_t, 0);
  auto s_prod = [&](f32x16& acc, int tile) {
#pragma unroll
    for (int j = 0; j < 16; ++j) acc[j] = 0.f;
#pragma unroll
    for (int k = 0; k < DD / 16; ++k)
      acc = mfma32_chunk<DT>(nt_at<uint4>(smem, at_s[k] + tile * (32 * DD * 2)), b_own[k], acc);
  };
  f32x16 acc2[DD / 32];
#pragma unroll
  for (int i = 0; i < DD / 32; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) acc2[i][j] = 0.f;
  auto p_prod = [&](const uint4 (&dz)[2], int tile) {
#pragma unroll
    for (int i = 0; i < DD / 32; ++i)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        acc2[i] = mfma32_chunk<DT_F16>(nt_at<uint4>(smem, at_t[2 * tile + t] + i * 4096), dz[t], acc2[i]);
  };
  // Scores of tile `tile` of stage s -> dz in fp32, DZ_UP times larger.  With gradients
  // of entropies as in dz_kernel; without, -dz = p g is one exponential (g >= 0, its
  // sign is in gs): 2^(z - lz), lz the lse less log2 g.  With offsets lz is the lse itself
  // (see RowGrad), and l0 = log2 g, less `more`.
  auto dz_of = [&](f32x16& x, int s, int tile) {
    const int k = s % 3, at = tile * 32 + 4 * h;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      f32x4 f, f0, f1, fl;
      if constexpr (CON) f = *reinterpret_cast<const f32x4*>(&con_s[k][0][at + 8 * q]);
      if constexpr (!IS_X && ENT) {
        f0 = *reinterpret_cast<const f32x4*>(&con_s[k][2][at + 8 * q]);
        f1 = *reinterpret_cast<const f32x4*>(&con_s[k][3][at + 8 * q]);
      }
      if constexpr (!IS_X && L0) fl = *reinterpret_cast<const f32x4*>(&con_s[k][2][at + 8 * q]);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float z = x[4 * q + r], lz = IS_X ? o.lz : f[r];
        float l;
        if constexpr (BIAS)  // in natural units: an offset may be the type's lowest value
          l = __builtin_fmaf(__builtin_fmaf(z, a.scale, IS_X ? f[r] : bz) - lz, LOG2E,
                             ENT ? 0.f : IS_X ? o.l0 : fl[r]);
        else
          l = __builtin_fmaf(z, c2, -lz);
        x[4 * q + r] = __builtin_amdgcn_exp2f(l);
        if constexpr (ENT)
          x[4 * q + r] *= __builtin_fmaf(BIAS ? __builtin_fmaxf(l, -1e30f) : l, IS_X ? o.c1 : f1[r],
                                         IS_X ? o.c0 : f0[r]);
      }
    }
  };
  // g more at the targets, then fp16 (nothing from rows and tokens that take no part)
  auto pack = [&](f32x16& y, uint4 (&dz)[2], int s, int tile, int odd) {
    const int k = s % 3, at = tile * 32 + 4 * h;
    if constexpr (IS_X) {
      const int rel = o.t - ((s0 + s) * 64 + tile * 32) - 4 * h;
      if (__ballot((unsigned)(rel + 4 * h) < 32u)) {
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (rel == 8 * (j >> 2) + (j & 3)) y[j] += o.g;
      }
      // the last row again after the last: p g of a target may be past fp16 without that
      const int left = a.nstream - ((s0 + s) * 64 + tile * 32) - 4 * h;
      if (left + 4 * h < 32) {
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (8 * (j >> 2) + (j & 3) >= left) y[j] = 0.f;
      }
    } else if (odd & (1 << tile)) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int4 t = *reinterpret_cast<const int4*>(&tgt_s[k][at + 8 * q]);
        const f32x4 g = *reinterpret_cast<const f32x4*>(&con_s[k][1][at + 8 * q]);
        if (t.x == own) y[4 * q] += g[0];
        if (t.y == own) y[4 * q + 1] += g[1];
        if (t.z == own) y[4 * q + 2] += g[2];
        if (t.w == own) y[4 * q + 3] += g[3];
      }
    }
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = half2_bits(y[2 * j], y[2 * j + 1]);
    if (odd & 4) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint2 m = *reinterpret_cast<const uint2*>(&keep_s[k][at + 8 * q]);
        w[2 * q] &= m.x;
        w[2 * q + 1] &= m.y;
      }
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
  fetch_con(2);
  nt_wait_and_sync<0>();
  f32x16 x0, x1;
  uint4 dz0[2] = {}, dz1[2] = {};  // of the stage's tiles 0 and 1
  s_prod(x0, 0);
  int next = CON ? odd_s[0][wave] : 0;
  for (int s = 0; s < ns; ++s) {
    const uint32_t up = s & 1;  // which buffer stage s is in
    const int odd = __builtin_amdgcn_readfirstlane(next);
    // tile 0's dz; the last stage's tile 1 multiplied on (nothing before the first)
    s_prod(x1, 1);
    p_prod(dz1, 1);
    dz_of(x0, s, 0);
    pack(x0, dz0, s, 0, odd);
    nt_wait_and_sync<0>();  // S of stage s + 1, P's operand of stage s, constants
    if (CON) next = odd_s[(s + 1) % 3][wave];
    store_con(s + 2);
    fetch_con(s + 3);
    if (s + 2 < ns) issue_s(s + 2);
    if (s + 1 < ns) issue_t(s + 1);
    move(at_s, up ? -Z::SB : Z::SB);
    if (s) move(at_t, up ? Z::TB : -Z::TB);
    s_prod(x0, 0);
    p_prod(dz0, 0);
    dz_of(x1, s, 1);
    pack(x1, dz1, s, 1, odd);
  }
  p_prod(dz1, 1);

  // 32 rows by 64 columns at a time through LDS, whole lines out, as in out_kernel
  __syncthreads();
  char* sq = smem + wave * 8192;
  const float f = out_factor(a.out, b);
#pragma unroll
  for (int i = 0; i < DD / 64; ++i) {
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x16& y = acc2[2 * i + c];
        nt_at<f32x4>(sq, n * 256 + (((8 * c + 2 * q + h) ^ (n & 7)) << 4)) =
            mine ? f32x4{y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]} : f32x4{0, 0, 0, 0};
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
      if (own0 + rl < a.nown && d < a.out.D) out_store<DT>(a.out, f, b, sp, own0 + rl, d, v);
    }
  }
}

// Both sides in one launch: the workgroups past the first nx are dW's.
template <int DT, int DD, bool BIAS, bool ENT>
__global__ __launch_bounds__(256, DD <= 64 ? 3 : DD <= 128 ? 2 : 1) void narrow_kernel(NarrowArgs x, NarrowArgs w,
                                                                        int nx) {
  __shared__ __attribute__((aligned(16))) char smem[NarrowSize<DD>::SMEM];
  if ((int)blockIdx.x < nx) narrow_run<DT, DD, true, BIAS, ENT>(x, blockIdx.x, smem);
  else narrow_run<DT, DD, false, BIAS, ENT>(w, blockIdx.x - nx, smem);
}
