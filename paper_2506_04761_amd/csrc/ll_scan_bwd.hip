// Selective state space scan, backward.  With g_t the gradient of the state h_t (all later tokens included),
//   g_t = C_t dy_t + a_(t+1) g_(t+1),   q_t = a_t h_(t-1) g_t,
//   dx_t = D_t sum_n B_tn g_tn + skip dy_t,   dD_t = x_t sum_n B_tn g_tn + sum_n A_n q_tn,
//   dA_n = sum_t D_t q_tn,   dB_tn = sum_d g_tdn D_td x_td,   dC_tn = sum_d dy_td h_tdn,
// where dy is the gradient before the gate: d_y silu(z).
//
// The split of the length into segments is the forward's: k_scan_rev runs every segment backwards by itself (carry
// G = a g, from zero; lanes and staging as in k_scan_fwd), k_scan_join turns these into the carries that segments
// start from, and k_scan_bwd runs them from there.
//
// k_scan_bwd has to add over channels as well as over states, so it spreads both over lanes: lane (r, c) =
// (lane / 16, lane % 16) holds states 4r .. 4r+3 of channel c, for two blocks of 16 channels one after the other, so
// that the sums over channels (dB, dC) are half added before lanes are.  B and C are the same for all channels: one
// register per 4 tokens holds them with lane (r, m) = token m / 4, state 4r + m % 4, and a product takes its factor
// as a row-broadcast (DPP) operand.  Step sizes, inputs and dy pass through LDS, 16 tokens x 32 channels to a wave,
// eight channels of a token to a lane, and the sums over states come back the same way.  A chunk of 16 tokens starts
// from the state that the forward saved before it: it is run once for the states before its tiles of 4 tokens, then
// the tiles are taken last to first, forming rates and states again in registers.  The waves of a workgroup are added
// in LDS, workgroups by k_scan_bc.
//
// Bound by the vector ALU: two waves a SIMD up to 16 states (256 registers: rates, states and gradients of 4 tokens x 2
// blocks, the sums over channels; the gated float32 instance has 17 more in scratch), one beyond (registers, and 101 and
// 109 KiB of LDS), about 3200 instructions per 16 tokens x 32 channels x 16 states, the ALU busy 81 % of the time.
// bf16, 2 x 4032 tokens of 2048 channels, 16 states: k_scan_bwd 250 us, k_scan_rev 69, the join 10, k_scan_bc 6.5, the
// parameters' sums 5.  One block of 16 channels instead of two, at three and four waves a SIMD: 291 and 383 us.
// A training step of those tokens, forward and backward: 8 states 433 us, 16 466, 24 875, 32 932, 64 1963 (8 and 24 work
// as 16 and 32 here).
#include "ll_layer.hpp"
#include "ll_layer_device.hpp"

namespace ll {

namespace {

constexpr int kChunk = kScanChunk;
constexpr int kTile = 4;          // tokens whose rates and states are in registers
constexpr int kWaves = 4;
constexpr int kCG = 2;            // blocks of 16 channels of a wave
constexpr int kWaveCh = 16 * kCG;
constexpr int kStep = 4;          // tokens that k_scan_rev loads together
constexpr int kRows = 8;          // tokens, times the waves, whose C it stages together
constexpr float kLn2 = 0.6931471805599453f;

struct BwdDev {
  Rows x, dt, z, Bm, Cm;
  const float *A, *skip, *dt_bias, *states, *dh_final;
  const int32_t* lengths;
  const void* dy;
  void *dx, *ddt, *dz, *dB, *dC;
  float *seg_g, *seg_d, *part_bc, *part, *dh0;
  int64_t T, D, chunks, T4, len, flen;  // T4: groups of four tokens, padded to whole chunks; tokens of a (fine) segment
  int N, G, Dg, blocks, cblocks, waves, rev_blocks, rev_cblocks, rev_waves, S, F, R, B;  // segments, fine segments, R fine ones to a segment
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

// A fine segment backwards by itself.
template <typename T, int NB, bool GATED>
__global__ __launch_bounds__(256, NB == 1 ? 4 : (NB == 2 ? 2 : 1)) void k_scan_rev(BwdDev p) {
  constexpr int NP = 16 * NB, STAGE = kRows * NP / 64;
  __shared__ float s_row[2][kRows * kWaves][NP];
  const int threads = 64 * p.rev_waves, tile = kRows * p.rev_waves;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  int64_t id = blockIdx.x;
  const int cb = int(id % p.rev_cblocks);
  id /= p.rev_cblocks;
  const int seg = 1 + int(id % (p.F - 1)), b = int(id / (p.F - 1));  // nothing comes before segment 0
  const int g = cb / p.rev_blocks, c0 = (cb % p.rev_blocks * p.rev_waves + wave) * 64;
  const bool mine = c0 + lane < p.Dg;         // spare lanes repeat the group's last channel and store nothing
  const int c = mine ? lane : p.Dg - 1 - c0;  // may be negative: a spare wave, which only helps to stage
  const int64_t ch0 = int64_t(g) * p.Dg + c0, ch = ch0 + c;
  float A2[NP], G[NP];
#pragma unroll
  for (int n = 0; n < NP; ++n) {
    A2[n] = n < p.N ? p.A[ch * p.N + n] * kLog2e : 0.0f;
    G[n] = seg == p.F - 1 && p.dh_final && n < p.N ? p.dh_final[(int64_t(b) * p.D + ch) * p.N + n] : 0.0f;
  }
  const float bias = p.dt_bias ? p.dt_bias[ch] : 0.0f;
  const int64_t t_begin = int64_t(seg) * p.flen, t_end = t_begin + p.flen < p.T ? t_begin + p.flen : p.T;
  const int64_t live = live_tokens(p.lengths, b, p.T), end = live < t_end ? live : t_end;
  const int count = __builtin_amdgcn_readfirstlane(end > t_begin ? int(end - t_begin) : 0);
  // token i, counted from the end
  const T* dp = static_cast<const T*>(p.dt.p) + b * p.dt.sb + (end - 1) * p.dt.st + ch0;
  const T* zp = static_cast<const T*>(p.z.p) + b * p.z.sb + (end - 1) * p.z.st + ch0;
  const T* gp = static_cast<const T*>(p.dy) + (int64_t(b) * p.T + end - 1) * p.D + ch0;
  const T* Cp = static_cast<const T*>(p.Cm.p) + b * p.Cm.sb + (end - 1) * p.Cm.st + int64_t(g) * p.N;
  T stage[STAGE];
  auto fetch_rows = [&](int i0) {
#pragma unroll
    for (int k = 0; k < STAGE; ++k) {
      const int e = threadIdx.x + threads * k, i = i0 + e / NP, n = e % NP;
      stage[k] = i < count && n < p.N ? (Cp - int64_t(i) * p.Cm.st)[n] : from_f32<T>(0.0f);
    }
  };
  T dr[kStep], zr[kStep], gr[kStep];
  int ahead = 0;  // tokens fetched; before the first that one is fetched again, and masked when used
  auto fetch = [&] {
#pragma unroll
    for (int k = 0; k < kStep; ++k) {
      dr[k] = load_at<T>(dp, 0, 0, c);
      gr[k] = load_at<T>(gp, 0, 0, c);
      if (GATED) zr[k] = load_at<T>(zp, 0, 0, c);
      const bool more = ++ahead < count;
      dp -= more ? p.dt.st : 0;
      gp -= more ? p.D : 0;
      if (GATED) zp -= more ? p.z.st : 0;
    }
  };
  float dsum = 0.0f;
  auto run = [&](const float (*rows)[NP], int i0) {
    float d[kStep], e[kStep];
#pragma unroll
    for (int k = 0; k < kStep; ++k) {
      d[k] = to_f32(dr[k]) + bias;
      e[k] = to_f32(gr[k]);
      if (GATED) e[k] *= silu(to_f32(zr[k]));
    }
    if (i0 + kStep < count) fetch();
    if (p.softplus) {
#pragma unroll
      for (int k = 0; k < kStep; ++k) d[k] = softplusf(d[k]);
    }
#pragma unroll
    for (int k = 0; k < kStep; ++k)
      if (i0 + k >= count) d[k] = e[k] = 0.0f;
    f32x4 now = *reinterpret_cast<const f32x4*>(&rows[0][0]), next = now;
#pragma unroll
    for (int k = 0; k < kStep; ++k) {
      dsum += d[k];
#pragma unroll
      for (int q = 0; q < NP; q += 4) {
        if (k * NP + q + 4 < kStep * NP) next = *reinterpret_cast<const f32x4*>(&rows[0][0] + k * NP + q + 4);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 4; ++i) G[q + i] = fmaf(now[i], e[k], G[q + i]) * fast_exp2(d[k] * A2[q + i]);
        now = next;
      }
    }
  };
  const bool works = c0 < p.Dg;
  fetch_rows(0);
  if (works && count > 0) fetch();
  int buf = 0;
  for (int i0 = 0; i0 < count; i0 += tile, buf ^= 1) {
    float(*rows)[NP] = s_row[buf];
#pragma unroll
    for (int k = 0; k < STAGE; ++k) (&rows[0][0])[threadIdx.x + threads * k] = to_f32(stage[k]);
    __syncthreads();
    if (i0 + tile < count) fetch_rows(i0 + tile);
    if (!works) continue;
    const int n = count - i0 < tile ? count - i0 : tile;
    for (int i = 0; i < n; i += kStep) run(rows + i, i0 + i);
  }
  if (mine) {
    float* q = p.seg_g + rec(b, seg, p.F, p.D, ch, NP);
#pragma unroll
    for (int n = 0; n < NP; n += 4) *reinterpret_cast<f32x4*>(q + n) = f32x4{G[n], G[n + 1], G[n + 2], G[n + 3]};
    p.seg_d[(int64_t(b) * p.F + seg) * p.D + ch] = dsum;
  }
}

template <typename T, int NB, bool GATED>
__global__ __launch_bounds__(256, 2) void k_scan_bwd(BwdDev p) {
  constexpr int NP = 16 * NB;
  constexpr int TILES = kChunk / kTile;
  constexpr bool OVER = NB == 1;  // a tile's sums may take the place of its staged inputs
  typedef typename VecN<T, 8>::type V8;
  // rows padded for lanes that write one token each
  __shared__ float2 s_du[kWaves][kChunk][kWaveCh + 2];  // step size, step size times input; then sums of B g, of A2 q
  __shared__ float s_dy[kWaves][kChunk][kWaveCh + 4];   // dy; then sums of C h
  __shared__ float2 s_sum[OVER ? 1 : kWaves][kChunk][kWaveCh + 2];
  __shared__ float s_out[OVER ? 1 : kWaves][kChunk][kWaveCh + 4];
  __shared__ float s_row[2][2][kChunk][NP];             // B and C of a chunk
  __shared__ f32x4 s_h[kWaves][TILES - 1][kCG][64];  // states before tiles 1, 2, ..
  __shared__ float s_bc[2][kWaves][2 * TILES][64];
  __shared__ float s_par[kWaves][2][kWaveCh];        // bias, skip
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane >> 4, c = lane & 15;

  int64_t id = blockIdx.x;
  const int cb = int(id % p.cblocks);
  id /= p.cblocks;
  const int seg = int(id % p.S), b = int(id / p.S);
  const int grp = cb / p.blocks, c0 = (cb % p.blocks * p.waves + wave) * kWaveCh;
  const int nch = p.Dg - c0 < 0 ? 0 : (p.Dg - c0 > kWaveCh ? kWaveCh : p.Dg - c0);  // may be none: the wave adds zeros
  const int64_t ch0 = int64_t(grp) * p.Dg + c0;

  const int fine = (seg + 1) * p.R < p.F ? (seg + 1) * p.R - 1 : p.F - 1;  // the segment's last fine one
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
        g[k][nb][i] = 0.0f;
        if (ok && p.F > 1) g[k][nb][i] = p.seg_g[rec(b, fine, p.F, p.D, ch0 + cc, NP) + n];
        else if (ok && p.dh_final) g[k][nb][i] = p.dh_final[(int64_t(b) * p.D + ch0 + cc) * p.N + n];
        dA[k][nb][i] = 0.0f;
      }

  const int64_t t_begin = int64_t(seg) * p.len, t_end = t_begin + p.len < p.T ? t_begin + p.len : p.T;
  const int64_t live = live_tokens(p.lengths, b, p.T), end = live < t_end ? live : t_end;
  // staging: lane (r, c) = channels 8 r .. 8 r + 7 of token c of the chunk
  const int ts = c, cs = 8 * r;
  const int own = nch - cs < 0 ? 0 : (nch - cs > 8 ? 8 : nch - cs);
  const int64_t base = int64_t(b) * p.T * p.D + ch0;
  const T* xp = static_cast<const T*>(p.x.p) + b * p.x.sb + ch0;
  const T* dp = static_cast<const T*>(p.dt.p) + b * p.dt.sb + ch0;
  const T* zp = static_cast<const T*>(p.z.p) + b * p.z.sb + ch0;
  const T* gp = static_cast<const T*>(p.dy) + base;
  const T* Bp = static_cast<const T*>(p.Bm.p) + b * p.Bm.sb + int64_t(grp) * p.N;
  const T* Cp = static_cast<const T*>(p.Cm.p) + b * p.Cm.sb + int64_t(grp) * p.N;
  if (lane < kWaveCh) {
    s_par[wave][0][lane] = p.dt_bias && lane < nch ? p.dt_bias[ch0 + lane] : 0.0f;
    s_par[wave][1][lane] = p.skip && lane < nch ? p.skip[ch0 + lane] : 0.0f;
  }
  float dparam = 0.0f;  // lane (r, m): the sum of dskip (m < 8) or dbias of channel 8 r + m % 8
  // p.vec: the rows' channels are whole vectors of eight, at their alignment; own is 0 or 8
  auto load8 = [&](const T* q, int row, int64_t stride) {
    const char* at = reinterpret_cast<const char*>(q) + (unsigned(row) * unsigned(stride) + unsigned(cs)) * unsigned(sizeof(T));
    return load_n<T, 8>(reinterpret_cast<const T*>(at), own, p.vec);
  };
  auto store8 = [&](void* q, int64_t t0, const float* f) {
    char* at = reinterpret_cast<char*>(static_cast<T*>(q) + base + t0 * p.D) +
               (unsigned(ts) * unsigned(p.D) + unsigned(cs)) * unsigned(sizeof(T));
    store_n<T, 8>(reinterpret_cast<T*>(at), f, own, p.vec);
  };

  V8 xr = {}, dr = {}, zr = {}, gr = {};
  // the workgroup's B and C of a chunk, [B or C][token][state]: thread i holds values i, i + threads, .. (a workgroup of
  // fewer waves loads the rest when it stages them)
  T bc[2 * NB];
  const int threads = 64 * p.waves;
  f32x4 hr[kCG][NB];
#pragma unroll
  for (int k = 0; k < kCG; ++k)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) hr[k][nb] = f32x4{0, 0, 0, 0};  // what a wave without channels works on
  // A chunk's inputs and the states before it.  Rows from the end of the sequence on repeat its last and are
  // masked when used.
  auto row_value = [&](int64_t chunk, int e) {
    const int64_t t0 = chunk * kChunk;
    const int t = e / NP % kChunk, n = e % NP;
    const bool is_c = e >= kChunk * NP;
    return t < end - t0 && n < p.N ? load_at<T>((is_c ? Cp : Bp) + t0 * (is_c ? p.Cm.st : p.Bm.st), t, is_c ? p.Cm.st : p.Bm.st, n)
                                   : from_f32<T>(0.0f);
  };
  auto fetch = [&](int64_t chunk) {
    const int64_t t0 = chunk * kChunk;
    const int left = end - t0 < kChunk ? int(end - t0) : kChunk;
#pragma unroll
    for (int i = 0; i < 2 * NB; ++i) bc[i] = row_value(chunk, threadIdx.x + threads * i);
    if (nch == 0) return;
    const float* hp = p.states + rec(b, chunk, p.chunks, p.D, ch0, NP);
#pragma unroll
    for (int k = 0; k < kCG; ++k)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
        if (16 * k + c < nch) hr[k][nb] = *reinterpret_cast<const f32x4*>(reinterpret_cast<const char*>(hp) + unsigned((16 * k + c) * NP + 16 * nb + 4 * r) * 4);
    if (left <= 0) return;
    const int row = ts < left ? ts : left - 1;
    xr = load8(xp + t0 * p.x.st, row, p.x.st);
    dr = load8(dp + t0 * p.dt.st, row, p.dt.st);
    gr = load8(gp + t0 * p.D, row, p.D);
    if (GATED) zr = load8(zp + t0 * p.z.st, row, p.z.st);
  };
  auto stage_rows = [&](int64_t chunk, int buf) {
#pragma unroll
    for (int i = 0; i < 2 * NB; ++i) (&s_row[buf][0][0][0])[threadIdx.x + threads * i] = to_f32(bc[i]);
    for (int e = threadIdx.x + 2 * NB * threads; e < 2 * kChunk * NP; e += threads)
      (&s_row[buf][0][0][0])[e] = to_f32(row_value(chunk, e));
  };

  int buf = 0;
  const int64_t last_chunk = (t_end - 1) / kChunk, first_chunk = t_begin / kChunk;
  fetch(last_chunk);
  stage_rows(last_chunk, 0);
  __syncthreads();
  for (int64_t chunk = last_chunk; chunk >= first_chunk; --chunk) {
    const int64_t t0 = chunk * kChunk;
    const bool in = ts < end - t0;
    const V8 xk = xr, dk = dr, zk = zr, gk = gr;
    wave_sync();
    float delta[8];
    const bool all = own == 8 && in;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      float u[2], e[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float d = to_f32(T(dk[i + j])) + s_par[wave][0][cs + i + j];
        if (p.softplus) d = softplusf(d);
        e[j] = to_f32(T(gk[i + j]));
        if (GATED) e[j] *= silu(to_f32(T(zk[i + j])));
        u[j] = d * to_f32(T(xk[i + j]));
        delta[i + j] = d;
        if (!all) {
          const bool ok = in && i + j < own;
          u[j] = ok ? u[j] : 0.0f;
          delta[i + j] = ok ? d : 0.0f;
          e[j] = ok ? e[j] : 0.0f;
        }
      }
      *reinterpret_cast<float4*>(&s_du[wave][ts][cs + i]) = make_float4(delta[i], u[0], delta[i + 1], u[1]);
      *reinterpret_cast<float2*>(&s_dy[wave][ts][cs + i]) = make_float2(e[0], e[1]);
    }
    wave_sync();
    f32x4 first[kCG][NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int k = 0; k < kCG; ++k) first[k][nb] = hr[k][nb];
    const int rb = int(last_chunk - chunk) & 1;
    // lane (r, m)'s B or C of a tile: token m / 4, state 4 r + m % 4
    auto row4 = [&](int which, int tile, int nb) { return s_row[rb][which][4 * tile + (c >> 2)][16 * nb + 4 * r + (c & 3)]; };
    if (chunk > first_chunk) fetch(chunk - 1);

#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      // forwards through all tiles but the last, for the states between them
      {
#pragma unroll
        for (int k = 0; k < kCG; ++k) {
          f32x4 h = first[k][nb];
#pragma unroll
          for (int tile = 0; tile + 1 < TILES; ++tile) {
            const float Bv = row4(0, tile, nb);
            float2 du[kTile];
#pragma unroll
            for (int t = 0; t < kTile; ++t) du[t] = s_du[wave][kTile * tile + t][16 * k + c];
            unrolled(std::make_integer_sequence<int, kTile>{}, [&](auto K) {
              constexpr int t = decltype(K)::value;
              unrolled(std::make_integer_sequence<int, 4>{}, [&](auto I) {
                constexpr int i = decltype(I)::value;
                h[i] = fmaf(fast_exp2(du[t].x * A2[k][nb][i]), h[i], row_bcast<4 * t + i>(Bv) * du[t].y);
              });
            });
            s_h[wave][tile][k][lane] = h;
          }
        }
      }
      // backwards, tile by tile
#pragma unroll
      for (int tile = TILES - 1; tile >= 0; --tile) {
        const float Bv = row4(0, tile, nb), Cv = row4(1, tile, nb);
        float db[16], dc[16];
        {
          unrolled(std::make_integer_sequence<int, kCG>{}, [&](auto KK) {
            constexpr int k = decltype(KK)::value;
            __builtin_amdgcn_sched_barrier(0);
            float a[kTile][4], h[kTile + 1][4], dy[kTile];
            float2 du[kTile];
            const f32x4 hs = tile > 0 ? s_h[wave][tile > 0 ? tile - 1 : 0][k][lane] : first[k][nb];
#pragma unroll
            for (int t = 0; t < kTile; ++t) {
              du[t] = s_du[wave][kTile * tile + t][16 * k + c];
              dy[t] = s_dy[wave][kTile * tile + t][16 * k + c];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) h[0][i] = hs[i];
            unrolled(std::make_integer_sequence<int, kTile>{}, [&](auto K) {
              constexpr int t = decltype(K)::value;
              unrolled(std::make_integer_sequence<int, 4>{}, [&](auto I) {
                constexpr int i = decltype(I)::value;
                a[t][i] = fast_exp2(du[t].x * A2[k][nb][i]);
                h[t + 1][i] = fmaf(a[t][i], h[t][i], row_bcast<4 * t + i>(Bv) * du[t].y);
              });
            });
            __builtin_amdgcn_sched_barrier(0);
            float sx[4], sq[4], sy[4];
            unrolled(std::make_integer_sequence<int, 4>{}, [&](auto K) {
              constexpr int t = 3 - decltype(K)::value;
              grad_token<4 * t, GATED>(g[k][nb], Bv, Cv, dy[t], h[t + 1], sx[t], sy[t]);
              float q;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                db[4 * t + i] = k == 0 ? du[t].y * g[k][nb][i] : fmaf(du[t].y, g[k][nb][i], db[4 * t + i]);
                dc[4 * t + i] = k == 0 ? dy[t] * h[t + 1][i] : fmaf(dy[t], h[t + 1][i], dc[4 * t + i]);
                g[k][nb][i] *= a[t][i];
                const float gh = g[k][nb][i] * h[t][i];
                dA[k][nb][i] = fmaf(du[t].x, gh, dA[k][nb][i]);
                q = i == 0 ? A2[k][nb][i] * gh : fmaf(A2[k][nb][i], gh, q);
              }
              sq[t] = q;
            });
            // formed here, not where they are used (the compiler would keep all their terms until then)
#pragma unroll
            for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(dA[k][nb][i]));
#pragma unroll
            for (int i = 0; i < 16; ++i) asm volatile("" : "+v"(db[i]), "+v"(dc[i]));
            // row r of the sums is token r of the tile
            float2 v = make_float2(sum_rows4(sx[0], sx[1], sx[2], sx[3]), sum_rows4(sq[0], sq[1], sq[2], sq[3]));
            float y = GATED ? sum_rows4(sy[0], sy[1], sy[2], sy[3]) : 0.0f;
            const int t = kTile * tile + r;
            if (OVER) {  // the wave has read the tile's inputs
              wave_sync();
              s_du[wave][t][16 * k + c] = v;
              s_dy[wave][t][16 * k + c] = y;
            } else {
              if (nb > 0) {
                const float2 o = s_sum[OVER ? 0 : wave][t][16 * k + c];
                v.x += o.x, v.y += o.y;
                y += s_out[OVER ? 0 : wave][t][16 * k + c];
              }
              s_sum[OVER ? 0 : wave][t][16 * k + c] = v;
              s_out[OVER ? 0 : wave][t][16 * k + c] = y;
            }
          });
          __builtin_amdgcn_sched_barrier(0);
        }
        // the sums over this wave's channels, lane (r, m): token m / 4 of the tile, state 4 r + m % 4
        s_bc[buf][wave][tile][lane] = sum_lanes16(db);
        s_bc[buf][wave][TILES + tile][lane] = sum_lanes16(dc);
      }
      if (nb == NB - 1 && chunk > first_chunk) stage_rows(chunk - 1, rb ^ 1);
      __syncthreads();  // the other buffers are free: all waves have passed this barrier after they were read
      for (int e = wave; e < 2 * TILES; e += p.waves) {
        const int which = e / TILES, tile = e % TILES;
        float v = s_bc[buf][0][e][lane];
        for (int w = 1; w < p.waves; ++w) v += s_bc[buf][w][e][lane];
        (p.part_bc + ((((int64_t(which) * p.B + b) * p.cblocks + cb) * p.T4 + t0 / 4 + tile) * NB + nb) * 64)[lane] = v;
      }
      buf ^= 1;
    }
    // outputs, eight channels of a token to a lane
    wave_sync();
    float sums[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) sums[i] = 0.0f;
    if (own > 0 && ts < t_end - t0) {
      float ox[8], od[8], oz[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 s = OVER ? s_du[wave][ts][cs + i] : s_sum[OVER ? 0 : wave][ts][cs + i];
        const float sy = OVER ? s_dy[wave][ts][cs + i] : s_out[OVER ? 0 : wave][ts][cs + i];
        const float x = to_f32(T(xk[i])), v = to_f32(T(dk[i])) + s_par[wave][0][cs + i], skip = s_par[wave][1][cs + i];
        const float dout = to_f32(T(gk[i])), z = GATED ? to_f32(T(zk[i])) : 0.0f, sg = GATED ? sigmoidf(z) : 1.0f;
        const float dy = GATED ? dout * (z * sg) : dout;
        const float grad = p.softplus ? sigmoidf(v) : 1.0f;
        ox[i] = in ? fmaf(delta[i], s.x, skip * dy) : 0.0f;
        od[i] = in ? fmaf(x, s.x, kLn2 * s.y) * grad : 0.0f;
        if (GATED) oz[i] = in ? dout * fmaf(skip, x, sy) * silu_grad(z, sg) : 0.0f;
        sums[i] = in ? dy * x : 0.0f;
        sums[8 + i] = od[i];
      }
      store8(p.dx, t0, ox);
      store8(p.ddt, t0, od);
      if (GATED) store8(p.dz, t0, oz);
    }
    dparam += sum_lanes16(sums);
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
          // where no token was, a state or gradient that is not finite has left its product with zero
          row[ch * NP + n] = end > t_begin ? dA[k][nb][i] : 0.0f;
          if (seg == 0 && p.dh0 && n < p.N) p.dh0[(int64_t(b) * p.D + ch) * p.N + n] = g[k][nb][i];
        }
    }
  if ((c & 7) < own) row[p.D * (NP + (c >> 3)) + ch0 + cs + (c & 7)] = dparam;
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

// Segments: two workgroups of k_scan_bwd on every compute unit (beyond 16 states one is resident: they take two
// rounds); split further for k_scan_rev, to four waves on
// every SIMD.
struct BwdLayout {
  int64_t S, len, F, flen, R, T4, seg_g, seg_d, bc, part, total;
};
BwdLayout layout(int64_t B, int64_t T, int64_t D, int64_t N, int64_t G) {
  BwdLayout l;
  const int64_t NP = 16 * scan_state_blocks(N), wgs = B * G * ceil_div(D / G, kWaveCh * kWaves), most = ceil_div(T, kChunk);
  const int64_t rev = B * G * ceil_div(D / G, 64);
  // workgroups of fewer waves: more of them
  const int64_t w = ceil_div(D / G, kWaveCh), per = ceil_div(w, ceil_div(w, kWaves));
  int64_t want = ceil_div(512 * kWaves / per, wgs), fine = ceil_div(4096, rev);
  want = want > most ? most : want;
  fine = fine > most ? most : fine;
  fine = fine < want ? want : fine;
  l.flen = ceil_div(ceil_div(T, fine), kChunk) * kChunk;
  l.R = ceil_div(ceil_div(T, want), l.flen);
  l.len = l.R * l.flen;
  l.S = ceil_div(T, l.len);
  l.F = ceil_div(T, l.flen);
  l.T4 = ceil_div(T, kChunk) * (kChunk / 4);
  l.seg_g = 0;
  l.seg_d = l.seg_g + (l.F > 1 ? align256(B * l.F * D * NP * 4) : 0);
  l.bc = l.seg_d + (l.F > 1 ? align256(B * l.F * D * 4) : 0);
  l.part = l.bc + align256(2 * wgs * l.T4 * NP * 4 * 4);
  l.total = l.part + align256(B * l.S * D * (NP + 2) * 4);
  return l;
}

int64_t bc_threads(int64_t B, int64_t G, int64_t T4, int64_t NP) { return 2 * B * G * T4 * NP * 4; }

template <typename T, int NB, bool GATED>
hipError_t go_main(const BwdDev& p, hipStream_t st) {
  if (p.F > 1) {
    k_scan_rev<T, NB, GATED><<<dim3(unsigned(int64_t(p.rev_cblocks) * p.B * (p.F - 1))), 64 * p.rev_waves, 0, st>>>(p);
    const hipError_t e = launch_scan_join({p.A, p.dh_final, p.seg_g, p.seg_d, p.B, p.F, p.D, p.N, 16 * NB, true}, st);
    if (e != hipSuccess) return e;
  }
  k_scan_bwd<T, NB, GATED><<<dim3(unsigned(int64_t(p.cblocks) * p.B * p.S)), 64 * p.waves, 0, st>>>(p);
  return hipGetLastError();
}

template <typename T, int NB>
hipError_t go(const BwdDev& p, hipStream_t st) {
  const hipError_t e = p.z.p ? go_main<T, NB, true>(p, st) : go_main<T, NB, false>(p, st);
  if (e != hipSuccess) return e;
  const int64_t total = bc_threads(p.B, p.G, p.T4, 16 * NB);
  k_scan_bc<T, NB><<<dim3(unsigned(ceil_div(total, 256))), 256, 0, st>>>(p, total);
  return hipGetLastError();
}

}  // namespace

int64_t scan_bwd_workspace(int64_t B, int64_t T, int64_t D, int64_t N, int64_t G) {
  const int64_t own = layout(B, T, D, N, G).total, fwd = scan_fwd_workspace(B, T, D, N, G);
  return own > fwd ? own : fwd;  // one workspace serves both
}

bool scan_bwd_launchable(const ScanArgs& a) {
  const BwdLayout l = layout(a.B, a.T, a.D, a.N, a.G);
  const int64_t NP = 16 * scan_state_blocks(a.N), BG = a.B * a.G;
  const int64_t waves = ceil_div(a.D / a.G, kWaveCh), blocks = ceil_div(waves, kWaves);
  const int64_t rev = ceil_div(a.D / a.G, 64), rev_blocks = ceil_div(rev, kWaves);
  return launchable(BG * blocks * l.S, int(64 * ceil_div(waves, blocks))) &&
         launchable(BG * rev_blocks * (l.F - 1), int(64 * ceil_div(rev, rev_blocks))) &&
         (l.F == 1 || launchable(scan_join_workgroups(a.B, a.D, NP), 64)) &&
         launchable(ceil_div(bc_threads(a.B, a.G, l.T4, NP), 256), 256) &&
         launchable(ceil_div(a.D * NP, 64) + 2 * ceil_div(a.D, 64), 1024);
}

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
  p.T = a.T, p.D = a.D, p.chunks = ceil_div(a.T, kScanChunk), p.T4 = l.T4, p.len = l.len, p.flen = l.flen;
  p.N = int(a.N), p.G = int(a.G), p.Dg = int(a.D / a.G);
  const int64_t waves = ceil_div(p.Dg, kWaveCh);  // of a group: as few workgroups as hold them, of equal size
  p.blocks = int(ceil_div(waves, kWaves)), p.waves = int(ceil_div(waves, p.blocks)), p.cblocks = int(p.blocks * a.G);
  const int64_t rev = ceil_div(p.Dg, 64);
  p.rev_blocks = int(ceil_div(rev, kWaves)), p.rev_waves = int(ceil_div(rev, p.rev_blocks));
  p.rev_cblocks = int(p.rev_blocks * a.G);
  p.S = int(l.S), p.F = int(l.F), p.R = int(l.R), p.B = int(a.B), p.softplus = a.softplus;
  const Rows flat[4] = {{g.dy, 0, a.D}, {g.dx, 0, a.D}, {g.ddt, 0, a.D}, {g.dz, 0, a.D}};
  p.vec = p.Dg % 8 == 0 && rows_aligned(a.x, e, 16 / e) && rows_aligned(a.dt, e, 16 / e) && (!a.z.p || rows_aligned(a.z, e, 16 / e));
  for (const Rows& r : flat) p.vec = p.vec && rows_aligned(r, e, 16 / e);
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
