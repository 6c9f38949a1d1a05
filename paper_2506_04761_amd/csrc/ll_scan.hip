// Selective state space scan (a decay per channel and state), forward and single token:
//
//   D_td = softplus(dt_td + bias_d),  a_tdn = exp(D_td A_dn),  h_tdn = a_tdn h_(t-1)dn + D_td x_td B_tn,
//   y_td = (sum_n C_tn h_tdn + skip_d x_td) silu(z_td).
//
// Layout of a wave: 16 channels x 16 states (per block of 16 states).  Lane (r, c) = (lane / 16, lane % 16)
// holds states 4r .. 4r+3 of channel c.  B and C are the same for all channels, so one register per
// 4 tokens holds them with lane (r, m) = token m / 4, state 4r + m % 4, and a product takes its factor
// as a row-broadcast operand (DPP) without an instruction for it.  Step sizes, inputs, gates and outputs
// go through a wave's own LDS rows: loaded and finished as 16 tokens x 16 channels, four channels to
// a lane, so that softplus and the gate are computed once for a token and channel.
//
// Bound by the vector ALU: per token, channel and state one exp, the rate's product, the input's
// product and two FMAs.  The states of a channel are a chain over tokens, and channels x sequences alone
// rarely fill the card, so the length is split into S segments: a first kernel runs every segment but the
// last by itself (the first from the initial state, the others from zero) without outputs, the second starts
// each from the segments before it,
//   h = exp(A sum D) h + (segment by itself),
// and runs it with the outputs.  The second kernel's first segment starts from the first kernel's copy of the
// initial state, so that the final state may be written over it.
#include "ll_layer.hpp"
#include "ll_layer_device.hpp"

namespace ll {

namespace {

constexpr int kTile = 16;      // tokens a wave stages at a time
constexpr int kWaves = 4;      // waves of a workgroup: neighbouring blocks of 16 channels share cache lines
constexpr int kBlock = 16 * kWaves;

struct ScanDev {
  Rows x, dt, z, Bm, Cm;
  const float *A, *skip, *dt_bias, *h0;
  const int32_t* lengths;
  float *h_final, *states, *seg_h, *seg_d;
  void* y;
  int64_t T, D, chunks;
  int N, Dg, blocks, cblocks;  // states; channels of a group; workgroups of a group and of a sequence
  int S, B;
  int64_t len;            // tokens of a segment
  int softplus, vec;      // vec: x, dt, z and y rows may be accessed four channels at a time
};

// Start of [.., segment or chunk, channel, padded state] records.
__device__ inline int64_t rec(int64_t b, int64_t s, int64_t S, int64_t D, int64_t ch, int NP) {
  return ((b * S + s) * D + ch) * NP;
}

template <typename T, int NB, bool OUT, bool GATED>
__global__ __launch_bounds__(64 * kWaves) void k_scan_fwd(ScanDev p) {
  constexpr int NP = 16 * NB;
  typedef typename VecN<T, 4>::type V4;
  __shared__ float2 s_du[kWaves][kTile][16];
  __shared__ float s_y[kWaves][kTile][16];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane >> 4, c = lane & 15;

  int64_t id = blockIdx.x;
  const int cb = int(id % p.cblocks);
  id /= p.cblocks;
  const int segs = OUT ? p.S : p.S - 1;  // nothing follows the last segment
  const int seg = int(id % segs), b = int(id / segs);
  const int g = cb / p.blocks, c0 = (cb % p.blocks) * kBlock + wave * 16;
  if (c0 >= p.Dg) return;
  const int nch = p.Dg - c0 < 16 ? p.Dg - c0 : 16;       // channels of this wave
  const int64_t ch0 = int64_t(g) * p.Dg + c0;
  const int64_t ch = ch0 + (c < nch ? c : nch - 1);      // spare lanes repeat the last channel

  float A2[NB][4], h[NB][4];
  auto save = [&](float* base, int s) {
    float* q = base + rec(b, s, p.S, p.D, ch, NP) + 4 * r;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
      *reinterpret_cast<f32x4*>(q + 16 * nb) = f32x4{h[nb][0], h[nb][1], h[nb][2], h[nb][3]};
  };
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = nb * 16 + 4 * r + i;
      A2[nb][i] = n < p.N ? p.A[ch * p.N + n] * kLog2e : 0.0f;
      h[nb][i] = p.h0 && seg == 0 && (!OUT || p.S == 1) && n < p.N ? p.h0[(int64_t(b) * p.D + ch) * p.N + n] : 0.0f;
    }
  if (!OUT && seg == 0 && p.h0 && c < nch) save(p.seg_h, p.S - 1);
  if (OUT && seg == 0 && p.S > 1 && p.h0) {
    const float* q = p.seg_h + rec(b, p.S - 1, p.S, p.D, ch, NP) + 4 * r;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int i = 0; i < 4; ++i) h[nb][i] = q[16 * nb + i];
  }
  if (OUT) {
#pragma unroll 4
    for (int s = 0; s < seg; ++s) {
      const float d = p.seg_d[(int64_t(b) * p.S + s) * p.D + ch];
      const float* q = p.seg_h + rec(b, s, p.S, p.D, ch, NP) + 4 * r;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(q + 16 * nb);
#pragma unroll
        for (int i = 0; i < 4; ++i) h[nb][i] = fmaf(fast_exp2(A2[nb][i] * d), h[nb][i], v[i]);
      }
    }
  }

  const int64_t t_begin = int64_t(seg) * p.len, t_end = t_begin + p.len < p.T ? t_begin + p.len : p.T;
  int64_t live = p.T;  // tokens from here on are no inputs
  if (p.lengths) {
    live = p.lengths[b];
    live = live < 0 ? 0 : (live > p.T ? p.T : live);
  }
  // staging: lane = token lane / 4 of the tile, channels 4 (lane % 4) .. + 3
  const int ts = lane >> 2, cs = 4 * (lane & 3);
  const int mine = nch - cs < 0 ? 0 : (nch - cs > 4 ? 4 : nch - cs);
  const T* xp = static_cast<const T*>(p.x.p) + b * p.x.sb + ch0;
  const T* dp = static_cast<const T*>(p.dt.p) + b * p.dt.sb + ch0;
  const T* zp = static_cast<const T*>(p.z.p) + b * p.z.sb + ch0;
  constexpr bool gated = OUT && GATED;
  T* yp = static_cast<T*>(p.y) + int64_t(b) * p.T * p.D + ch0;
  const T* Bp = static_cast<const T*>(p.Bm.p) + b * p.Bm.sb + int64_t(g) * p.N;
  const T* Cp = static_cast<const T*>(p.Cm.p) + b * p.Cm.sb + int64_t(g) * p.N;
  float bias[4], skip[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    bias[i] = p.dt_bias && i < mine ? p.dt_bias[ch0 + cs + i] : 0.0f;
    skip[i] = OUT && p.skip && i < mine ? p.skip[ch0 + cs + i] : 0.0f;
  }

  V4 xr = {}, dr = {}, zr = {};
  T br[NB][4], cr[NB][4];
  const int64_t end = live < t_end ? live : t_end;
  // The inputs of a tile; rows from the end of the sequence on repeat its last and are masked when used.
  auto fetch = [&](int64_t t0) {
    const int left = end - t0 < kTile ? int(end - t0) : kTile;
    if (left <= 0) return;
    const int row = ts < left ? ts : left - 1;
    xr = load_row4<T>(xp + t0 * p.x.st, row, p.x.st, cs, nch, p.vec);
    dr = load_row4<T>(dp + t0 * p.dt.st, row, p.dt.st, cs, nch, p.vec);
    if (gated) zr = load_row4<T>(zp + t0 * p.z.st, row, p.z.st, cs, nch, p.vec);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int rj = 4 * j + (c >> 2) < left ? 4 * j + (c >> 2) : left - 1;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int n = nb * 16 + 4 * r + (c & 3) < p.N ? nb * 16 + 4 * r + (c & 3) : 0;
        br[nb][j] = load_at<T>(Bp + t0 * p.Bm.st, rj, p.Bm.st, n);
        if (OUT) cr[nb][j] = load_at<T>(Cp + t0 * p.Cm.st, rj, p.Cm.st, n);
      }
    }
  };

  float dsum = 0.0f;
  if (t_begin < t_end) fetch(t_begin);
  for (int64_t t0 = t_begin; t0 < t_end; t0 += kTile) {
    if (OUT && p.states && (t0 - t_begin) % (64 / NB) == 0 && c < nch) {
      float* q = p.states + rec(b, t0 / (64 / NB), p.chunks, p.D, ch, NP) + 4 * r;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
        *reinterpret_cast<f32x4*>(q + 16 * nb) = f32x4{h[nb][0], h[nb][1], h[nb][2], h[nb][3]};
    }
    const V4 xk = xr, zk = zr;
    const bool in = ts < end - t0;
    {
      float2 du[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float d = to_f32(T(dr[i])) + bias[i];
        if (p.softplus) d = softplusf(d);
        d = in ? d : 0.0f;  // a token that is no input leaves the states as they are
        du[i] = make_float2(d, in ? d * to_f32(T(xk[i])) : 0.0f);
      }
      wave_sync();
      float4* q = reinterpret_cast<float4*>(&s_du[wave][ts][cs]);
      q[0] = make_float4(du[0].x, du[0].y, du[1].x, du[1].y);
      q[1] = make_float4(du[2].x, du[2].y, du[3].x, du[3].y);
      wave_sync();
    }
    float Bv[NB][4], Cv[NB][4];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool ok = 4 * j + (c >> 2) < end - t0 && nb * 16 + 4 * r + (c & 3) < p.N;
        Bv[nb][j] = ok ? to_f32(br[nb][j]) : 0.0f;
        if (OUT) Cv[nb][j] = ok ? to_f32(cr[nb][j]) : 0.0f;
      }
    if (t0 + kTile < t_end) fetch(t0 + kTile);

#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float yt[4];
      auto step = [&](auto K) {
        constexpr int k = decltype(K)::value;
        const float2 du = s_du[wave][4 * j + k][c];
        if (!OUT) dsum += du.x;
        float y = 0.0f;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          auto state = [&](auto I) {
            constexpr int i = decltype(I)::value;
            const float a = fast_exp2(du.x * A2[nb][i]);
            h[nb][i] = fmaf(a, h[nb][i], row_bcast<4 * k + i>(Bv[nb][j]) * du.y);
          };
          state(std::integral_constant<int, 0>{});
          state(std::integral_constant<int, 1>{});
          state(std::integral_constant<int, 2>{});
          state(std::integral_constant<int, 3>{});
          if (OUT) y = dot4_bcast<4 * k>(y, Cv[nb][j], h[nb]);
        }
        yt[k] = y;
      };
      step(std::integral_constant<int, 0>{});
      step(std::integral_constant<int, 1>{});
      step(std::integral_constant<int, 2>{});
      step(std::integral_constant<int, 3>{});
      if (OUT) s_y[wave][4 * j + r][c] = sum_rows4(yt[0], yt[1], yt[2], yt[3]);
    }
    if (OUT) {
      wave_sync();
      const float4 v = *reinterpret_cast<const float4*>(&s_y[wave][ts][cs]);
      float o[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        o[i] = fmaf(skip[i], to_f32(T(xk[i])), o[i]);
        if (gated) o[i] *= silu(to_f32(T(zk[i])));
        o[i] = in ? o[i] : 0.0f;
      }
      store_row4<T>(yp + t0 * p.D, ts, p.D, cs, o, ts < t_end - t0 ? mine : 0, p.vec);
    }
  }

  if (OUT) {
    if (seg == p.S - 1 && p.h_final && c < nch) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int n = nb * 16 + 4 * r + i;
          if (n < p.N) p.h_final[(int64_t(b) * p.D + ch) * p.N + n] = h[nb][i];
        }
    }
  } else if (c < nch) {
    save(p.seg_h, seg);
    if (r == 0) p.seg_d[(int64_t(b) * p.S + seg) * p.D + ch] = dsum;
  }
}

// One token: four lanes to a channel, lane q of them states 4q .. 4q+3, 16 + 4q .. and so on, so that a
// wave reads 1 KiB of adjacent state.  Bound by the state's read and write.
struct StepDev {
  Rows x, dt, z, Bm, Cm;
  const float *A, *skip, *dt_bias, *h0;
  float* h1;
  void* y;
  int64_t D, total;  // total: sequences x channels
  int N, Dg, softplus, vec;  // vec: N is a multiple of 4 and A and the states are 16-byte aligned
};

template <typename T>
__global__ __launch_bounds__(256) void k_scan_step(StepDev p) {
  const int64_t id = int64_t(blockIdx.x) * 64 + (threadIdx.x >> 2);
  if (id >= p.total) return;  // all four lanes of a channel together
  const int q = threadIdx.x & 3;
  const int64_t b = id / p.D, ch = id - b * p.D;
  const float x = to_f32(static_cast<const T*>(p.x.p)[b * p.x.sb + ch]);
  float d = to_f32(static_cast<const T*>(p.dt.p)[b * p.dt.sb + ch]) + (p.dt_bias ? p.dt_bias[ch] : 0.0f);
  const float z = p.z.p ? to_f32(static_cast<const T*>(p.z.p)[b * p.z.sb + ch]) : 0.0f;
  const int g = int(ch / p.Dg);
  const T* Bp = static_cast<const T*>(p.Bm.p) + b * p.Bm.sb + int64_t(g) * p.N;
  const T* Cp = static_cast<const T*>(p.Cm.p) + b * p.Cm.sb + int64_t(g) * p.N;
  const float* hp = p.h0 ? p.h0 + id * p.N : nullptr;
  const float* Ap = p.A + ch * p.N;
  float* op = p.h1 + id * p.N;
  if (p.softplus) d = softplusf(d);
  const float u = d * x;
  float y = 0.0f;
  for (int n = 4 * q; n < p.N; n += 16) {
    const int m = p.N - n < 4 ? p.N - n : 4;
    const f32x4 hv = hp ? load_n<float, 4>(hp + n, m, p.vec) : f32x4{0, 0, 0, 0};
    const f32x4 av = load_n<float, 4>(Ap + n, m, p.vec);
    const typename VecN<T, 4>::type bv = load_n<T, 4>(Bp + n, m, false), cv = load_n<T, 4>(Cp + n, m, false);
    float o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[i] = fmaf(fast_exp2(d * (av[i] * kLog2e)), hv[i], to_f32(T(bv[i])) * u);
      if (i < m) y = fmaf(to_f32(T(cv[i])), o[i], y);
    }
    store_n<float, 4>(op + n, o, m, p.vec);
  }
  y += dpp_mov<0xB1>(y);  // quad_perm 1,0,3,2
  y += dpp_mov<0x4E>(y);  // quad_perm 2,3,0,1
  if (q == 0) {
    if (p.skip) y = fmaf(p.skip[ch], x, y);
    if (p.z.p) y *= silu(z);
    static_cast<T*>(p.y)[id] = from_f32<T>(y);
  }
}

int elem(int dtype) { return dtype == 1 ? 2 : 4; }

// Segments: enough waves to hold two on every SIMD, in segments of 256 tokens and more.
ScanSplit split(int64_t B, int64_t T, int64_t D, int64_t G) {
  const int64_t waves = B * G * ceil_div(D / G, kBlock) * kWaves;
  ScanSplit s;
  int64_t want = waves >= 1024 ? 1 : ceil_div(2048, waves);
  const int64_t most = ceil_div(T, 256);
  if (want > most) want = most;
  s.len = ceil_div(ceil_div(T, want), 64) * 64;
  s.S = ceil_div(T, s.len);
  return s;
}

int64_t align256(int64_t v) { return (v + 255) / 256 * 256; }

}  // namespace

int scan_state_blocks(int64_t N) { return N <= 16 ? 1 : (N <= 32 ? 2 : 4); }
int64_t scan_chunk(int64_t N) { return 64 / scan_state_blocks(N); }
int64_t scan_states_bytes(int64_t B, int64_t T, int64_t D, int64_t N) {
  return B * ceil_div(T, scan_chunk(N)) * D * 16 * scan_state_blocks(N) * 4;
}
int64_t scan_fwd_workspace(int64_t B, int64_t T, int64_t D, int64_t N, int64_t G) {
  const ScanSplit s = split(B, T, D, G);
  if (s.S == 1) return 0;
  return align256(B * s.S * D * 16 * scan_state_blocks(N) * 4) + align256(B * s.S * D * 4);
}

template <typename T>
static hipError_t run_fwd(const ScanDev& p, int nb, hipStream_t st) {
  const int64_t per = int64_t(p.cblocks) * p.B;
  const dim3 first(unsigned(per * (p.S - 1))), second(unsigned(per * p.S)), threads(64 * kWaves);
  if (p.S > 1) {
    if (nb == 1) k_scan_fwd<T, 1, false, false><<<first, threads, 0, st>>>(p);
    else if (nb == 2) k_scan_fwd<T, 2, false, false><<<first, threads, 0, st>>>(p);
    else k_scan_fwd<T, 4, false, false><<<first, threads, 0, st>>>(p);
  }
  if (p.z.p) {
    if (nb == 1) k_scan_fwd<T, 1, true, true><<<second, threads, 0, st>>>(p);
    else if (nb == 2) k_scan_fwd<T, 2, true, true><<<second, threads, 0, st>>>(p);
    else k_scan_fwd<T, 4, true, true><<<second, threads, 0, st>>>(p);
  } else {
    if (nb == 1) k_scan_fwd<T, 1, true, false><<<second, threads, 0, st>>>(p);
    else if (nb == 2) k_scan_fwd<T, 2, true, false><<<second, threads, 0, st>>>(p);
    else k_scan_fwd<T, 4, true, false><<<second, threads, 0, st>>>(p);
  }
  return hipGetLastError();
}

hipError_t launch_scan_fwd(const ScanArgs& a, hipStream_t st) {
  const int nb = scan_state_blocks(a.N), e = elem(a.dtype);
  const ScanSplit s = split(a.B, a.T, a.D, a.G);
  ScanDev p = {};
  p.x = a.x, p.dt = a.dt, p.z = a.z, p.Bm = a.Bm, p.Cm = a.Cm;
  p.A = a.A, p.skip = a.skip, p.dt_bias = a.dt_bias, p.h0 = a.h0, p.lengths = a.lengths;
  p.h_final = a.h_final, p.states = a.states, p.y = a.y;
  p.T = a.T, p.D = a.D, p.chunks = ceil_div(a.T, scan_chunk(a.N));
  p.N = int(a.N), p.Dg = int(a.D / a.G);
  p.blocks = int(ceil_div(p.Dg, kBlock)), p.cblocks = int(p.blocks * a.G);
  p.S = int(s.S), p.B = int(a.B), p.len = s.len;
  p.softplus = a.softplus;
  p.vec = p.Dg % 4 == 0 && rows_aligned(a.x, e, 4) && rows_aligned(a.dt, e, 4) &&
          (!a.z.p || rows_aligned(a.z, e, 4)) && rows_aligned(Rows{a.y, a.T * a.D, a.D}, e, 4);
  if (s.S > 1) {
    p.seg_h = static_cast<float*>(a.workspace);
    p.seg_d = reinterpret_cast<float*>(static_cast<char*>(a.workspace) + align256(a.B * s.S * a.D * 16 * nb * 4));
  }
  return a.dtype == 1 ? run_fwd<__bf16>(p, nb, st) : run_fwd<float>(p, nb, st);
}

hipError_t launch_scan_step(const ScanArgs& a, hipStream_t st) {
  StepDev p = {};
  p.x = a.x, p.dt = a.dt, p.z = a.z, p.Bm = a.Bm, p.Cm = a.Cm;
  p.A = a.A, p.skip = a.skip, p.dt_bias = a.dt_bias, p.h0 = a.h0, p.h1 = a.h_final, p.y = a.y;
  p.D = a.D, p.total = a.B * a.D, p.N = int(a.N), p.Dg = int(a.D / a.G), p.softplus = a.softplus;
  const uintptr_t at = reinterpret_cast<uintptr_t>(a.h0) | reinterpret_cast<uintptr_t>(a.h_final) |
                       reinterpret_cast<uintptr_t>(a.A);
  p.vec = a.N % 4 == 0 && at % 16 == 0;
  const dim3 grid(unsigned(ceil_div(p.total, 64)));
  if (a.dtype == 1) k_scan_step<__bf16><<<grid, 256, 0, st>>>(p);
  else k_scan_step<float><<<grid, 256, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace ll
