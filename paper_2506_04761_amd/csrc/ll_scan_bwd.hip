// Selective state space scan, backward.  With g_t the gradient of the state h_t (all later tokens included),
//   g_t = C_t dy_t + a_(t+1) g_(t+1),   q_t = a_t h_(t-1) g_t,
//   dx_t = D_t sum_n B_tn g_tn + skip dy_t,   dD_t = x_t sum_n B_tn g_tn + sum_n A_n q_tn,
//   dA_n = sum_t D_t q_tn,   dB_tn = sum_d g_tdn D_td x_td,   dC_tn = sum_d dy_td h_tdn,
// where dy is the gradient before the gate: d_y silu(z).
//
// The layout of lanes, and the split of the length into segments, are the forward's: k_scan_rev runs every
// segment backwards by itself (carry G = a g, from zero), k_scan_bwd starts each from the carries of the
// segments after it.  It needs the states too: from the state saved before every chunk it first runs the
// chunk forwards, keeping the state before each tile of 8 tokens in LDS, then takes the tiles last to first,
// forming a tile's rates and states again in registers.  A wave holds two blocks of 16 channels, so that
// the sums over channels (dB, dC) are half added before lanes are; the four waves of a workgroup are added
// in LDS, workgroups by k_scan_bc.
#include "ll_layer.hpp"
#include "ll_layer_device.hpp"

namespace ll {

namespace {

constexpr int kTile = 8;          // tokens of a tile
constexpr int kWaves = 4;
constexpr int kCG = 2;            // blocks of 16 channels of a wave
constexpr int kWaveCh = 16 * kCG;
constexpr int kBlock = kWaveCh * kWaves;
constexpr int kRevTile = 16;
constexpr float kLn2 = 0.6931471805599453f;

struct BwdDev {
  Rows x, dt, z, Bm, Cm;
  const float *A, *skip, *dt_bias, *states, *dh_final;
  const int32_t* lengths;
  const void* dy;
  void *dx, *ddt, *dz, *dB, *dC;
  float *seg_g, *seg_d, *part_bc, *part, *dh0;
  int64_t T, D, chunks, T4, len;  // T4: groups of four tokens, padded to whole tiles
  int N, G, Dg, blocks, cblocks, rev_blocks, rev_cblocks, S, B;
  int softplus, vec;
};

__device__ inline int64_t rec(int64_t b, int64_t s, int64_t S, int64_t D, int64_t ch, int NP) {
  return ((b * S + s) * D + ch) * NP;
}

__device__ inline int64_t live_tokens(const int32_t* lengths, int64_t b, int64_t T) {
  if (!lengths) return T;
  const int64_t n = lengths[b];
  return n < 0 ? 0 : (n > T ? T : n);
}

template <int... I, typename F>
__device__ inline void unrolled(std::integer_sequence<int, I...>, F&& f) {
  (f(std::integral_constant<int, I>{}), ...);
}

// A segment backwards by itself: lanes and staging as in the forward kernel.
template <typename T, int NB, bool GATED>
__global__ __launch_bounds__(256) void k_scan_rev(BwdDev p) {
  constexpr int NP = 16 * NB;
  typedef typename VecN<T, 4>::type V4;
  __shared__ float2 s_dy[kWaves][kRevTile][16];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane >> 4, c = lane & 15;
  int64_t id = blockIdx.x;
  const int cb = int(id % p.rev_cblocks);
  id /= p.rev_cblocks;
  const int seg = 1 + int(id % (p.S - 1)), b = int(id / (p.S - 1));  // nothing comes before segment 0
  const int g = cb / p.rev_blocks, c0 = (cb % p.rev_blocks) * 64 + wave * 16;
  if (c0 >= p.Dg) return;
  const int nch = p.Dg - c0 < 16 ? p.Dg - c0 : 16;
  const int64_t ch0 = int64_t(g) * p.Dg + c0, ch = ch0 + (c < nch ? c : nch - 1);
  float A2[NB][4], G[NB][4];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = nb * 16 + 4 * r + i;
      A2[nb][i] = n < p.N ? p.A[ch * p.N + n] * kLog2e : 0.0f;
      G[nb][i] = seg == p.S - 1 && p.dh_final && n < p.N ? p.dh_final[(int64_t(b) * p.D + ch) * p.N + n] : 0.0f;
    }
  const int64_t t_begin = int64_t(seg) * p.len, t_end = t_begin + p.len < p.T ? t_begin + p.len : p.T;
  const int64_t live = live_tokens(p.lengths, b, p.T), end = live < t_end ? live : t_end;
  const int ts = lane >> 2, cs = 4 * (lane & 3);
  const int mine = nch - cs < 0 ? 0 : (nch - cs > 4 ? 4 : nch - cs);
  const T* dp = static_cast<const T*>(p.dt.p) + b * p.dt.sb + ch0;
  const T* zp = static_cast<const T*>(p.z.p) + b * p.z.sb + ch0;
  const T* gp = static_cast<const T*>(p.dy) + int64_t(b) * p.T * p.D + ch0;
  const T* Cp = static_cast<const T*>(p.Cm.p) + b * p.Cm.sb + int64_t(g) * p.N;
  float bias[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) bias[i] = p.dt_bias && i < mine ? p.dt_bias[ch0 + cs + i] : 0.0f;
  V4 dr = {}, zr = {}, gr = {};
  T cr[NB][4];
  auto fetch = [&](int64_t t0) {
    const int left = end - t0 < kRevTile ? int(end - t0) : kRevTile;
    if (left <= 0) return;
    const int row = ts < left ? ts : left - 1;
    dr = load_row4<T>(dp + t0 * p.dt.st, row, p.dt.st, cs, nch, p.vec);
    gr = load_row4<T>(gp + t0 * p.D, row, p.D, cs, nch, p.vec);
    if (GATED) zr = load_row4<T>(zp + t0 * p.z.st, row, p.z.st, cs, nch, p.vec);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int rj = 4 * j + (c >> 2) < left ? 4 * j + (c >> 2) : left - 1;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int n = nb * 16 + 4 * r + (c & 3) < p.N ? nb * 16 + 4 * r + (c & 3) : 0;
        cr[nb][j] = load_at<T>(Cp + t0 * p.Cm.st, rj, p.Cm.st, n);
      }
    }
  };
  float dsum = 0.0f;
  const int64_t last = t_begin + (t_end - 1 - t_begin) / kRevTile * kRevTile;
  fetch(last);
  for (int64_t t0 = last; t0 >= t_begin; t0 -= kRevTile) {
    {
      const bool in = ts < end - t0;
      float2 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float d = to_f32(T(dr[i])) + bias[i], e = to_f32(T(gr[i]));
        if (p.softplus) d = softplusf(d);
        if (GATED) e *= silu(to_f32(T(zr[i])));
        v[i] = make_float2(in ? d : 0.0f, in ? e : 0.0f);
      }
      wave_sync();
      float4* q = reinterpret_cast<float4*>(&s_dy[wave][ts][cs]);
      q[0] = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
      q[1] = make_float4(v[2].x, v[2].y, v[3].x, v[3].y);
      wave_sync();
    }
    float Cv[NB][4];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool ok = 4 * j + (c >> 2) < end - t0 && nb * 16 + 4 * r + (c & 3) < p.N;
        Cv[nb][j] = ok ? to_f32(cr[nb][j]) : 0.0f;
      }
    if (t0 > t_begin) fetch(t0 - kRevTile);
#pragma unroll
    for (int j = 3; j >= 0; --j)
      unrolled(std::make_integer_sequence<int, 4>{}, [&](auto K) {
        constexpr int k = 3 - decltype(K)::value;
        const float2 v = s_dy[wave][4 * j + k][c];
        dsum += v.x;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          axpy4_bcast<4 * k>(G[nb], Cv[nb][j], v.y);
#pragma unroll
          for (int i = 0; i < 4; ++i) G[nb][i] *= fast_exp2(v.x * A2[nb][i]);
        }
      });
  }
  if (c < nch) {
    float* q = p.seg_g + rec(b, seg, p.S, p.D, ch, NP) + 4 * r;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
      *reinterpret_cast<f32x4*>(q + 16 * nb) = f32x4{G[nb][0], G[nb][1], G[nb][2], G[nb][3]};
    if (r == 0) p.seg_d[(int64_t(b) * p.S + seg) * p.D + ch] = dsum;
  }
}

template <typename T, int NB, bool GATED>
__global__ __launch_bounds__(256, 2) void k_scan_bwd(BwdDev p) {
  constexpr int NP = 16 * NB;
  constexpr int CH = 64 / NB;          // tokens of a chunk
  constexpr int TILES = CH / kTile;
  constexpr bool OVER = NB == 1;       // a tile's sums may take the place of its staged inputs
  typedef typename VecN<T, 4>::type V4;
  __shared__ f32x4 s_h[kWaves][TILES - 1][kCG][NB][64];   // states before tiles 1, 2, ..
  __shared__ float2 s_du[kWaves][kTile][kWaveCh];         // step size, step size times input
  __shared__ float s_dy[kWaves][kTile][kWaveCh];
  __shared__ float2 s_sum[OVER ? 1 : kWaves][kTile][kWaveCh];
  __shared__ float s_out[OVER ? 1 : kWaves][kTile][kWaveCh];
  __shared__ float s_bc[2][kWaves][4][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane >> 4, c = lane & 15;

  int64_t id = blockIdx.x;
  const int cb = int(id % p.cblocks);
  id /= p.cblocks;
  const int seg = int(id % p.S), b = int(id / p.S);
  const int grp = cb / p.blocks, c0 = (cb % p.blocks) * kBlock + wave * kWaveCh;
  const int nch = p.Dg - c0 < 0 ? 0 : (p.Dg - c0 > kWaveCh ? kWaveCh : p.Dg - c0);  // may be none: the wave only meets barriers
  const int64_t ch0 = int64_t(grp) * p.Dg + c0;

  // Spare lanes and states have rate, state and gradient zero, so that they add nothing to any sum.
  float A2[kCG][NB][4], g[kCG][NB][4], dA[kCG][NB][4];
#pragma unroll
  for (int k = 0; k < kCG; ++k)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int n = nb * 16 + 4 * r + i, cc = 16 * k + c;
        const bool ok = cc < nch && n < p.N;
        A2[k][nb][i] = ok ? p.A[(ch0 + cc) * p.N + n] * kLog2e : 0.0f;
        g[k][nb][i] = ok && seg == p.S - 1 && p.dh_final ? p.dh_final[(int64_t(b) * p.D + ch0 + cc) * p.N + n] : 0.0f;
        dA[k][nb][i] = 0.0f;
      }
  for (int s = p.S - 1; s > seg; --s)
#pragma unroll
    for (int k = 0; k < kCG; ++k)
      if (16 * k + c < nch) {
        const int64_t ch = ch0 + 16 * k + c;
        const float d = p.seg_d[(int64_t(b) * p.S + s) * p.D + ch];
        const float* q = p.seg_g + rec(b, s, p.S, p.D, ch, NP) + 4 * r;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const f32x4 v = *reinterpret_cast<const f32x4*>(q + 16 * nb);
#pragma unroll
          for (int i = 0; i < 4; ++i) g[k][nb][i] = fmaf(fast_exp2(A2[k][nb][i] * d), g[k][nb][i], v[i]);
        }
      }

  const int64_t t_begin = int64_t(seg) * p.len, t_end = t_begin + p.len < p.T ? t_begin + p.len : p.T;
  const int64_t live = live_tokens(p.lengths, b, p.T), end = live < t_end ? live : t_end;
  // staging: lane = token lane / 8 of the tile, channels 4 (lane % 8) .. + 3
  const int ts = lane >> 3, cs = 4 * (lane & 7);
  const int mine = nch - cs < 0 ? 0 : (nch - cs > 4 ? 4 : nch - cs);
  const int64_t base = int64_t(b) * p.T * p.D + ch0;
  const T* xp = static_cast<const T*>(p.x.p) + b * p.x.sb + ch0;
  const T* dp = static_cast<const T*>(p.dt.p) + b * p.dt.sb + ch0;
  const T* zp = static_cast<const T*>(p.z.p) + b * p.z.sb + ch0;
  const T* gp = static_cast<const T*>(p.dy) + base;
  const T* Bp = static_cast<const T*>(p.Bm.p) + b * p.Bm.sb + int64_t(grp) * p.N;
  const T* Cp = static_cast<const T*>(p.Cm.p) + b * p.Cm.sb + int64_t(grp) * p.N;
  float bias[4], skip[4], dskip[4], dbias[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    bias[i] = p.dt_bias && i < mine ? p.dt_bias[ch0 + cs + i] : 0.0f;
    skip[i] = p.skip && i < mine ? p.skip[ch0 + cs + i] : 0.0f;
    dskip[i] = dbias[i] = 0.0f;
  }
  V4 xr = {}, dr = {}, zr = {}, gr = {};
  T br[NB][2], cr[NB][2];
  // A tile's inputs; `all`: those of the backward too.  Rows from the end of the sequence on repeat its last
  // and are masked when used.
  auto fetch = [&](int64_t t0, bool all) {
    const int left = end - t0 < kTile ? int(end - t0) : kTile;
    if (left <= 0 || nch == 0) return;
    const int row = ts < left ? ts : left - 1;
    xr = load_row4<T>(xp + t0 * p.x.st, row, p.x.st, cs, nch, p.vec);
    dr = load_row4<T>(dp + t0 * p.dt.st, row, p.dt.st, cs, nch, p.vec);
    if (all) {
      gr = load_row4<T>(gp + t0 * p.D, row, p.D, cs, nch, p.vec);
      if (GATED) zr = load_row4<T>(zp + t0 * p.z.st, row, p.z.st, cs, nch, p.vec);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int rj = 4 * j + (c >> 2) < left ? 4 * j + (c >> 2) : left - 1;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int n = nb * 16 + 4 * r + (c & 3) < p.N ? nb * 16 + 4 * r + (c & 3) : 0;
        br[nb][j] = load_at<T>(Bp + t0 * p.Bm.st, rj, p.Bm.st, n);
        if (all) cr[nb][j] = load_at<T>(Cp + t0 * p.Cm.st, rj, p.Cm.st, n);
      }
    }
  };
  // whether this lane's entry of B and C (token 4 j + c / 4 of the tile, state nb 16 + 4 r + c % 4) is an input
  auto used = [&](int64_t t0, int nb, int j) { return 4 * j + (c >> 2) < end - t0 && nb * 16 + 4 * r + (c & 3) < p.N; };
  auto step_size = [&](float v) { return p.softplus ? softplusf(v) : v; };
  auto stage_du = [&](bool in, float* delta) {
    float u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool ok = in && i < mine;
      delta[i] = ok ? step_size(to_f32(T(dr[i])) + bias[i]) : 0.0f;
      u[i] = ok ? delta[i] * to_f32(T(xr[i])) : 0.0f;
    }
    float4* q = reinterpret_cast<float4*>(&s_du[wave][ts][cs]);
    q[0] = make_float4(delta[0], u[0], delta[1], u[1]);
    q[1] = make_float4(delta[2], u[2], delta[3], u[3]);
  };
  auto load_states = [&](int64_t chunk, int k, int nb) {
    const int cc = 16 * k + c;
    return cc < nch ? *reinterpret_cast<const f32x4*>(p.states + rec(b, chunk, p.chunks, p.D, ch0 + cc, NP) + 16 * nb + 4 * r)
                    : f32x4{0, 0, 0, 0};
  };

  int buf = 0;
  const int64_t last_chunk = (t_end - 1) / CH, first_chunk = t_begin / CH;
  fetch(last_chunk * CH, false);
  for (int64_t chunk = last_chunk; chunk >= first_chunk; --chunk) {
    const int64_t tc = chunk * CH;
    const int tiles = int((t_end - tc < CH ? t_end - tc : CH) + kTile - 1) / kTile;
    f32x4 h0[kCG][NB];
#pragma unroll
    for (int k = 0; k < kCG; ++k)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) h0[k][nb] = load_states(chunk, k, nb);
    // forwards: the states before tiles 1, 2, ..
    for (int tile = 0; tile + 1 < tiles; ++tile) {
      const int64_t t0 = tc + tile * kTile;
      float delta[4], Bv[NB][2];
      wave_sync();
      stage_du(ts < end - t0, delta);
      wave_sync();
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int j = 0; j < 2; ++j) Bv[nb][j] = used(t0, nb, j) ? to_f32(br[nb][j]) : 0.0f;
      fetch(t0 + kTile, tile + 2 == tiles);
      if (nch > 0) {
#pragma unroll
        for (int k = 0; k < kCG; ++k)
          unrolled(std::make_integer_sequence<int, kTile>{}, [&](auto K) {
            constexpr int t = decltype(K)::value;
            const float2 du = s_du[wave][t][16 * k + c];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
              unrolled(std::make_integer_sequence<int, 4>{}, [&](auto I) {
                constexpr int i = decltype(I)::value;
                h0[k][nb][i] = fmaf(fast_exp2(du.x * A2[k][nb][i]), h0[k][nb][i],
                                    row_bcast<4 * (t & 3) + i>(Bv[nb][t >> 2]) * du.y);
              });
          });
#pragma unroll
        for (int k = 0; k < kCG; ++k)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) s_h[wave][tile][k][nb][lane] = h0[k][nb];
      }
    }
    if (tiles == 1) fetch(tc, true);
    // backwards
    for (int tile = tiles - 1; tile >= 0; --tile) {
      const int64_t t0 = tc + tile * kTile;
      const bool in = ts < end - t0;
      float delta[4], dyg[4];
      const V4 xk = xr, dk = dr, zk = zr, gk = gr;
      wave_sync();
      stage_du(in, delta);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        dyg[i] = to_f32(T(gk[i]));
        if (GATED) dyg[i] *= silu(to_f32(T(zk[i])));
        dyg[i] = in && i < mine ? dyg[i] : 0.0f;
      }
      *reinterpret_cast<float4*>(&s_dy[wave][ts][cs]) = make_float4(dyg[0], dyg[1], dyg[2], dyg[3]);
      wave_sync();
      float Bv[NB][2], Cv[NB][2];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          Bv[nb][j] = used(t0, nb, j) ? to_f32(br[nb][j]) : 0.0f;
          Cv[nb][j] = used(t0, nb, j) ? to_f32(cr[nb][j]) : 0.0f;
        }
      if (tile > 0) fetch(t0 - kTile, true);
      else if (chunk > first_chunk) fetch(tc - CH, false);

#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float db[2][16], dc[2][16];
        if (nch > 0) {
          unrolled(std::make_integer_sequence<int, kCG>{}, [&](auto KK) {
            constexpr int k = decltype(KK)::value;
            __builtin_amdgcn_sched_barrier(0);
            float a[kTile][4], h[kTile + 1][4];
            const f32x4 hs = tile > 0 ? s_h[wave][tile > 0 ? tile - 1 : 0][k][nb][lane] : load_states(chunk, k, nb);
#pragma unroll
            for (int i = 0; i < 4; ++i) h[0][i] = hs[i];
            unrolled(std::make_integer_sequence<int, kTile>{}, [&](auto K) {
              constexpr int t = decltype(K)::value;
              const float2 du = s_du[wave][t][16 * k + c];
              unrolled(std::make_integer_sequence<int, 4>{}, [&](auto I) {
                constexpr int i = decltype(I)::value;
                a[t][i] = fast_exp2(du.x * A2[k][nb][i]);
                h[t + 1][i] = fmaf(a[t][i], h[t][i], row_bcast<4 * (t & 3) + i>(Bv[nb][t >> 2]) * du.y);
              });
            });
#pragma unroll
            for (int j = 1; j >= 0; --j) {
              __builtin_amdgcn_sched_barrier(0);  // no work of another half tile in flight: registers are full
              float sx[4], sq[4], sy[4];
              unrolled(std::make_integer_sequence<int, 4>{}, [&](auto K) {
                constexpr int m = 3 - decltype(K)::value;
                const int t = 4 * j + m;
                const float2 du = s_du[wave][t][16 * k + c];
                const float dy = s_dy[wave][t][16 * k + c];
                axpy4_bcast<4 * m>(g[k][nb], Cv[nb][j], dy);
                sx[m] = dot4_bcast<4 * m>(0.0f, Bv[nb][j], g[k][nb]);
                sy[m] = GATED ? dot4_bcast<4 * m>(0.0f, Cv[nb][j], h[t + 1]) : 0.0f;
                float q = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  db[j][4 * m + i] = k == 0 ? du.y * g[k][nb][i] : fmaf(du.y, g[k][nb][i], db[j][4 * m + i]);
                  dc[j][4 * m + i] = k == 0 ? dy * h[t + 1][i] : fmaf(dy, h[t + 1][i], dc[j][4 * m + i]);
                  g[k][nb][i] *= a[t][i];
                  const float gh = g[k][nb][i] * h[t][i];
                  dA[k][nb][i] = fmaf(du.x, gh, dA[k][nb][i]);
                  q = fmaf(A2[k][nb][i], gh, q);
                }
                sq[m] = q;
              });
              // the four tokens' inputs have been read: their sums may stand there
              float2 v = make_float2(sum_rows4(sx[0], sx[1], sx[2], sx[3]), sum_rows4(sq[0], sq[1], sq[2], sq[3]));
              float y = GATED ? sum_rows4(sy[0], sy[1], sy[2], sy[3]) : 0.0f;
              if (OVER) {
                wave_sync();
                s_du[wave][4 * j + r][16 * k + c] = v;
                s_dy[wave][4 * j + r][16 * k + c] = y;
              } else {
                if (nb > 0) {
                  const float2 o = s_sum[OVER ? 0 : wave][4 * j + r][16 * k + c];
                  v.x += o.x, v.y += o.y;
                  y += s_out[OVER ? 0 : wave][4 * j + r][16 * k + c];
                }
                s_sum[OVER ? 0 : wave][4 * j + r][16 * k + c] = v;
                s_out[OVER ? 0 : wave][4 * j + r][16 * k + c] = y;
              }
            }
          });
        }
        __builtin_amdgcn_sched_barrier(0);
        // sums over the channels: lanes of a row, then the waves
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          s_bc[buf][wave][j][lane] = nch > 0 ? sum_lanes16(db[j]) : 0.0f;
          s_bc[buf][wave][2 + j][lane] = nch > 0 ? sum_lanes16(dc[j]) : 0.0f;
        }
        __syncthreads();  // the other buffer is free: all waves have passed the barrier after its sums were read
        {
          const float v = (s_bc[buf][0][wave][lane] + s_bc[buf][1][wave][lane]) +
                          (s_bc[buf][2][wave][lane] + s_bc[buf][3][wave][lane]);
          const int64_t t4 = t0 / 4 + (wave & 1);
          p.part_bc[((((int64_t(wave >> 1) * p.B + b) * p.cblocks + cb) * p.T4 + t4) * NB + nb) * 64 + lane] = v;
        }
        buf ^= 1;
      }
      // outputs, four channels of a token to a lane
      wave_sync();
      if (mine > 0 && ts < t_end - t0) {
        const float4 w0 = *reinterpret_cast<const float4*>(OVER ? &s_du[wave][ts][cs] : &s_sum[OVER ? 0 : wave][ts][cs]);
        const float4 w1 = *reinterpret_cast<const float4*>(OVER ? &s_du[wave][ts][cs + 2] : &s_sum[OVER ? 0 : wave][ts][cs + 2]);
        const float4 w2 = *reinterpret_cast<const float4*>(OVER ? &s_dy[wave][ts][cs] : &s_out[OVER ? 0 : wave][ts][cs]);
        const float sx[4] = {w0.x, w0.z, w1.x, w1.z}, sq[4] = {w0.y, w0.w, w1.y, w1.w}, sy[4] = {w2.x, w2.y, w2.z, w2.w};
        float ox[4], od[4], oz[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = to_f32(T(xk[i])), zf = GATED ? to_f32(T(zk[i])) : 0.0f;
          ox[i] = in ? fmaf(delta[i], sx[i], skip[i] * dyg[i]) : 0.0f;
          float dd = fmaf(x, sx[i], kLn2 * sq[i]);
          if (p.softplus) dd *= sigmoidf(to_f32(T(dk[i])) + bias[i]);
          od[i] = in ? dd : 0.0f;
          if (GATED) oz[i] = in ? to_f32(T(gk[i])) * fmaf(skip[i], x, sy[i]) * silu_grad(zf, sigmoidf(zf)) : 0.0f;
          dskip[i] += in ? dyg[i] * x : 0.0f;
          dbias[i] += od[i];
        }
        const int64_t at = base + t0 * p.D;
        store_row4<T>(static_cast<T*>(p.dx) + at, ts, p.D, cs, ox, mine, p.vec);
        store_row4<T>(static_cast<T*>(p.ddt) + at, ts, p.D, cs, od, mine, p.vec);
        if (GATED) store_row4<T>(static_cast<T*>(p.dz) + at, ts, p.D, cs, oz, mine, p.vec);
      }
    }
  }

  // the segment's sums over tokens: dA, dskip, dbias; and before token 0 the state's gradient
  float* row = p.part + (int64_t(b) * p.S + seg) * p.D * (NP + 2);
#pragma unroll
  for (int k = 0; k < kCG; ++k)
    if (16 * k + c < nch) {
      const int64_t ch = ch0 + 16 * k + c;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int n = nb * 16 + 4 * r + i;
          row[ch * NP + n] = dA[k][nb][i];
          if (seg == 0 && p.dh0 && n < p.N) p.dh0[(int64_t(b) * p.D + ch) * p.N + n] = g[k][nb][i];
        }
    }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int m = 8; m < 64; m <<= 1) {
      dskip[i] += __shfl_xor(dskip[i], m);
      dbias[i] += __shfl_xor(dbias[i], m);
    }
    if (ts == 0 && i < mine) {
      row[p.D * NP + ch0 + cs + i] = dskip[i];
      row[p.D * (NP + 1) + ch0 + cs + i] = dbias[i];
    }
  }
}

// dB and dC from the workgroups' sums over channels: a lane adds a group's workgroups.
template <typename T, int NB>
__global__ __launch_bounds__(256) void k_scan_bc(BwdDev p, int64_t total) {
  const int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x;  // [dB or dC][b][group][t4][nb][64]
  if (id >= total) return;
  const int lane = int(id & 63), r = lane >> 4, m = lane & 15;
  int64_t q = id >> 6;
  const int nb = int(q % NB);
  q /= NB;
  const int64_t t4 = q % p.T4;
  q /= p.T4;
  const int g = int(q % p.G);
  q /= p.G;
  const int64_t b = q % p.B, which = q / p.B;
  const int64_t t = 4 * t4 + (m >> 2);
  const int n = nb * 16 + 4 * r + (m & 3);
  if (t >= p.T || n >= p.N) return;
  const bool live = t < live_tokens(p.lengths, b, p.T);
  const float* in = p.part_bc + (((which * p.B + b) * p.cblocks + int64_t(g) * p.blocks) * p.T4 + t4) * NB * 64 + nb * 64 + lane;
  float v = 0.0f;
#pragma unroll 4
  for (int k = 0; k < p.blocks; ++k) v += in[int64_t(k) * p.T4 * NB * 64];
  T* out = static_cast<T*>(which ? p.dC : p.dB);
  out[((b * p.T + t) * p.G + g) * p.N + n] = from_f32<T>(live ? v : 0.0f);
}

int elem(int dtype) { return dtype == 1 ? 2 : 4; }
int64_t align256(int64_t v) { return (v + 255) / 256 * 256; }

// Segments: two workgroups on every compute unit.
struct BwdLayout {
  int64_t S, len, T4, seg_g, seg_d, bc, part, total;
};
BwdLayout layout(int64_t B, int64_t T, int64_t D, int64_t N, int64_t G) {
  BwdLayout l;
  const int64_t NP = 16 * scan_state_blocks(N), wgs = B * G * ceil_div(D / G, kBlock);
  int64_t want = ceil_div(512, wgs);
  const int64_t most = ceil_div(T, 64);
  if (want > most) want = most;
  l.len = ceil_div(ceil_div(T, want), 64) * 64;
  l.S = ceil_div(T, l.len);
  l.T4 = ceil_div(T, kTile) * (kTile / 4);
  l.seg_g = 0;
  l.seg_d = l.seg_g + (l.S > 1 ? align256(B * l.S * D * NP * 4) : 0);
  l.bc = l.seg_d + (l.S > 1 ? align256(B * l.S * D * 4) : 0);
  l.part = l.bc + align256(2 * wgs * l.T4 * NP * 4 * 4);
  l.total = l.part + align256(B * l.S * D * (NP + 2) * 4);
  return l;
}

template <typename T, int NB, bool GATED>
void go_main(const BwdDev& p, hipStream_t st) {
  if (p.S > 1)
    k_scan_rev<T, NB, GATED><<<dim3(unsigned(int64_t(p.rev_cblocks) * p.B * (p.S - 1))), 256, 0, st>>>(p);
  k_scan_bwd<T, NB, GATED><<<dim3(unsigned(int64_t(p.cblocks) * p.B * p.S)), 256, 0, st>>>(p);
}

template <typename T, int NB>
hipError_t go(const BwdDev& p, hipStream_t st) {
  if (p.z.p) go_main<T, NB, true>(p, st);
  else go_main<T, NB, false>(p, st);
  const int64_t total = 2 * int64_t(p.B) * p.G * p.T4 * NB * 64;
  k_scan_bc<T, NB><<<dim3(unsigned(ceil_div(total, 256))), 256, 0, st>>>(p, total);
  return hipGetLastError();
}

}  // namespace

int64_t scan_bwd_workspace(int64_t B, int64_t T, int64_t D, int64_t N, int64_t G) { return layout(B, T, D, N, G).total; }

hipError_t launch_scan_bwd(const ScanArgs& a, const ScanGrads& g, hipStream_t st) {
  const int nb = scan_state_blocks(a.N), e = elem(a.dtype);
  const BwdLayout l = layout(a.B, a.T, a.D, a.N, a.G);
  BwdDev p = {};
  p.x = a.x, p.dt = a.dt, p.z = a.z, p.Bm = a.Bm, p.Cm = a.Cm;
  p.A = a.A, p.skip = a.skip, p.dt_bias = a.dt_bias, p.states = a.states, p.dh_final = g.dh_final;
  p.lengths = a.lengths, p.dy = g.dy;
  p.dx = g.dx, p.ddt = g.ddt, p.dz = g.dz, p.dB = g.dB, p.dC = g.dC, p.dh0 = g.dh0;
  char* ws = static_cast<char*>(a.workspace);
  p.seg_g = reinterpret_cast<float*>(ws + l.seg_g), p.seg_d = reinterpret_cast<float*>(ws + l.seg_d);
  p.part_bc = reinterpret_cast<float*>(ws + l.bc), p.part = reinterpret_cast<float*>(ws + l.part);
  p.T = a.T, p.D = a.D, p.chunks = ceil_div(a.T, scan_chunk(a.N)), p.T4 = l.T4, p.len = l.len;
  p.N = int(a.N), p.G = int(a.G), p.Dg = int(a.D / a.G);
  p.blocks = int(ceil_div(p.Dg, kBlock)), p.cblocks = int(p.blocks * a.G);
  p.rev_blocks = int(ceil_div(p.Dg, 64)), p.rev_cblocks = int(p.rev_blocks * a.G);
  p.S = int(l.S), p.B = int(a.B), p.softplus = a.softplus;
  const Rows flat[4] = {{g.dy, 0, a.D}, {g.dx, 0, a.D}, {g.ddt, 0, a.D}, {g.dz, 0, a.D}};
  p.vec = p.Dg % 4 == 0 && rows_aligned(a.x, e, 4) && rows_aligned(a.dt, e, 4) && (!a.z.p || rows_aligned(a.z, e, 4));
  for (const Rows& r : flat) p.vec = p.vec && rows_aligned(r, e, 4);
  hipError_t err;
  if (a.dtype == 1) err = nb == 1 ? go<__bf16, 1>(p, st) : (nb == 2 ? go<__bf16, 2>(p, st) : go<__bf16, 4>(p, st));
  else err = nb == 1 ? go<float, 1>(p, st) : (nb == 2 ? go<float, 2>(p, st) : go<float, 4>(p, st));
  if (err != hipSuccess) return err;
  const int64_t NP = 16 * nb;
  ColSum s = {};
  s.part = p.part, s.rows = a.B * l.S, s.stride = a.D * (NP + 2);
  s.out[s.n++] = {0, a.D * NP, g.dA, NP, a.N, a.N, 1};
  if (g.dskip) s.out[s.n++] = {a.D * NP, a.D, g.dskip, a.D, a.D, 0, 1};
  if (g.dbias) s.out[s.n++] = {a.D * (NP + 1), a.D, g.dbias, a.D, a.D, 0, 1};
  return launch_colsum(s, st);
}

}  // namespace ll
