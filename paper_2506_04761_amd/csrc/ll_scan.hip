// Selective state space scan (a decay per channel and state), forward and single token:
//
//   D_td = softplus(dt_td + bias_d),  a_tdn = exp(D_td A_dn),  h_tdn = a_tdn h_(t-1)dn + D_td x_td B_tn,
//   y_td = (sum_n C_tn h_tdn + skip_d x_td) silu(z_td).
//
// Layout: a lane holds one channel and all its states in registers, so that no sum crosses lanes.  x, dt, z and y
// are one element a lane and token, 64 adjacent channels to a wave, any alignment.  B and C, the same for all
// channels of a group, are staged in LDS as fp32 rows of padded length and read at one address by all lanes (as
// scalar operands they would halve the rate of the products that take them).
//
// Bound by the vector ALU: per token, channel and state one exp (8 cycles of a wave), and the rate's product, the
// input's product, the state's and the output's FMA (3 to 4 cycles each beside the exp, with four waves on a SIMD; a
// lone wave issues one in 8), and about 27 instructions per token and channel.  bf16, 16 states, 4 x 8192 tokens of
// 2048 channels: the two passes below take 190 and 245 us, in which counters see the ALU busy for 96 and 95 % of the
// cycles, and the joining of segments between them 17; the bytes alone would take 104.
//
// The states of a channel are a chain over tokens, and channels x sequences alone rarely make four waves a SIMD, so the
// length is split into S segments, run twice: k_scan_fwd<OUT = false> runs every segment but the last by itself (the
// first from the initial state, the others from zero) for its final state and its sum of step sizes, k_scan_join turns
// these into the states that segments start from,
//   h = exp(A sum D) h + (segment by itself),
// and k_scan_fwd<OUT = true> runs them from there with the outputs.
#include "ll_layer.hpp"
#include "ll_layer_device.hpp"

namespace ll {

namespace {

constexpr int kWaves = 4;            // waves of a workgroup at most: neighbouring channels of the same tokens
constexpr int kStep = 4;             // tokens that are loaded together

constexpr int kQ = 4;                // states whose B and C are read from LDS together
constexpr int kRows = 8;             // tokens, times the waves, whose B and C are staged together

struct ScanDev {
  Rows x, dt, z, Bm, Cm;
  const float *A, *skip, *dt_bias, *h0;
  const int32_t* lengths;
  float *h_final, *states, *seg_h, *seg_d;
  void* y;
  int64_t T, D, chunks;
  int N, G, Dg, blocks, cblocks;  // states; groups; channels of a group; workgroups of a group and of a sequence
  int waves;                      // of a workgroup
  int S, B, softplus;
  int64_t len;                    // tokens of a segment
};

// Start of [.., segment or chunk, channel, padded state] records.
__device__ inline int64_t rec(int64_t b, int64_t s, int64_t S, int64_t D, int64_t ch, int NP) {
  return ((b * S + s) * D + ch) * NP;
}

__device__ inline int64_t live_tokens(const int32_t* lengths, int64_t b, int64_t T) {
  if (!lengths) return T;
  const int64_t n = lengths[b];
  return n < 0 ? 0 : (n > T ? T : n);
}

template <int NP>
__device__ inline void load_state(const float* q, float* h) {
#pragma unroll
  for (int n = 0; n < NP; n += 4) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(q + n);
#pragma unroll
    for (int i = 0; i < 4; ++i) h[n + i] = v[i];
  }
}
template <int NP>
__device__ inline void save_state(float* q, const float* h) {
#pragma unroll
  for (int n = 0; n < NP; n += 4) *reinterpret_cast<f32x4*>(q + n) = f32x4{h[n], h[n + 1], h[n + 2], h[n + 3]};
}

// NP: states of a lane, N rounded up to one of a few sizes.
template <typename T, int NP, bool OUT, bool GATED>
__global__ __launch_bounds__(64 * kWaves, NP <= 16 ? 4 : (NP <= 24 ? 3 : (NP <= 32 ? 2 : 1))) void k_scan_fwd(ScanDev p) {
  constexpr int CH = kScanChunk, RP = (NP + 15) / 16 * 16;  // states of a saved record
  constexpr int W = OUT ? 2 * NP : NP, STAGE = kRows * W / 64;  // values of a token's row; of a tile and thread
  __shared__ float s_row[2][kRows * kWaves][W];
  const int threads = 64 * p.waves, tile = kRows * p.waves;  // of this launch: tokens staged together
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  int64_t id = blockIdx.x;
  const int cb = int(id % p.cblocks);
  id /= p.cblocks;
  const int segs = OUT ? p.S : p.S - 1;  // nothing follows the last segment
  const int seg = int(id % segs), b = int(id / segs);
  const int g = cb / p.blocks, c0 = (cb % p.blocks * p.waves + wave) * 64;
  const bool mine = c0 + lane < p.Dg;  // spare lanes repeat the group's last channel and store nothing
  const int c = mine ? lane : p.Dg - 1 - c0;  // may be negative: a spare wave
  const int64_t ch0 = int64_t(g) * p.Dg + c0, ch = ch0 + c;

  float A2[NP], h[NP];
#pragma unroll
  for (int n = 0; n < NP; ++n) {
    A2[n] = n < p.N ? p.A[ch * p.N + n] * kLog2e : 0.0f;
    h[n] = 0.0f;
  }
  if (OUT && p.S > 1) {
    load_state<NP>(p.seg_h + rec(b, seg, p.S, p.D, ch, NP), h);
  } else if (seg == 0 && p.h0) {
#pragma unroll
    for (int n = 0; n < NP; ++n) h[n] = n < p.N ? p.h0[(int64_t(b) * p.D + ch) * p.N + n] : 0.0f;
  }
  const float bias = p.dt_bias ? p.dt_bias[ch] : 0.0f, skip = OUT && p.skip ? p.skip[ch] : 0.0f;

  const int64_t t_begin = int64_t(seg) * p.len, t_end = t_begin + p.len < p.T ? t_begin + p.len : p.T;
  const int64_t live = live_tokens(p.lengths, b, p.T), end = live < t_end ? live : t_end;
  // uniform addresses of the next token to be fetched, to be run; a lane adds its channel
  const T* xp = static_cast<const T*>(p.x.p) + b * p.x.sb + t_begin * p.x.st + ch0;
  const T* dp = static_cast<const T*>(p.dt.p) + b * p.dt.sb + t_begin * p.dt.st + ch0;
  const T* zp = static_cast<const T*>(p.z.p) + b * p.z.sb + t_begin * p.z.st + ch0;
  T* yp = static_cast<T*>(p.y) + (int64_t(b) * p.T + t_begin) * p.D + ch0;
  const int count = __builtin_amdgcn_readfirstlane(end > t_begin ? int(end - t_begin) : 0);  // tokens to run

  // a tile's rows: thread i of the workgroup holds values i, i + threads, ..
  T stage[STAGE];
  const T* Bp = static_cast<const T*>(p.Bm.p) + b * p.Bm.sb + t_begin * p.Bm.st + int64_t(g) * p.N;
  const T* Cp = static_cast<const T*>(p.Cm.p) + b * p.Cm.sb + t_begin * p.Cm.st + int64_t(g) * p.N;
  auto fetch_rows = [&](int t0) {
#pragma unroll
    for (int k = 0; k < STAGE; ++k) {
      const int e = threadIdx.x + threads * k, t = t0 + e / W, n = e % NP;
      const bool is_c = OUT && e % W >= NP;
      const T* q = is_c ? Cp : Bp;
      stage[k] = t < count && n < p.N ? q[int64_t(t) * (is_c ? p.Cm.st : p.Bm.st) + n] : from_f32<T>(0.0f);
    }
  };

  T xr[kStep], dr[kStep], zr[kStep];
  int ahead = 0;  // tokens fetched; behind the end the last one is fetched again, and masked when used
  auto fetch = [&] {
#pragma unroll
    for (int k = 0; k < kStep; ++k) {
      xr[k] = load_at<T>(xp, 0, 0, c);
      dr[k] = load_at<T>(dp, 0, 0, c);
      if (GATED) zr[k] = load_at<T>(zp, 0, 0, c);
      const bool more = ++ahead < count;
      xp += more ? p.x.st : 0;
      dp += more ? p.dt.st : 0;
      if (GATED) zp += more ? p.z.st : 0;
    }
  };
  float dsum = 0.0f;
  // kStep tokens from t on, whose rows are at `rows`.  A step size of zero leaves the states as they are, and rows
  // behind the end are zeros.
  auto run = [&](const float (*rows)[W], int t) {
    float x[kStep], d[kStep], gate[kStep], y[kStep];
#pragma unroll
    for (int k = 0; k < kStep; ++k) {
      x[k] = to_f32(xr[k]);
      d[k] = to_f32(dr[k]) + bias;
      gate[k] = GATED ? to_f32(zr[k]) : 0.0f;
    }
    if (t + kStep < count) fetch();
    if (p.softplus) {
#pragma unroll
      for (int k = 0; k < kStep; ++k) d[k] = softplusf(d[k]);
    }
#pragma unroll
    for (int k = 0; k < kStep; ++k)
      if (t + k >= count) d[k] = x[k] = 0.0f;
    // kQ states at a time, the next ones' B and C on their way (registers are for the states: no more are)
    auto read = [&](int i, f32x4 (*v)[2]) {
#pragma unroll
      for (int j = 0; j < kQ / 4; ++j) {
        v[j][0] = *reinterpret_cast<const f32x4*>(&rows[0][0] + i / NP * W + i % NP + 4 * j);
        if (OUT) v[j][1] = *reinterpret_cast<const f32x4*>(&rows[0][0] + i / NP * W + NP + i % NP + 4 * j);
      }
    };
    f32x4 now[kQ / 4][2], next[kQ / 4][2];
    read(0, now);
#pragma unroll
    for (int k = 0; k < kStep; ++k) {
      const float u = d[k] * x[k];
      if (!OUT) dsum += d[k];
      y[k] = skip * x[k];
#pragma unroll
      for (int q = 0; q < NP; q += kQ) {
        if (k * NP + q + kQ < kStep * NP) read(k * NP + q + kQ, next);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < kQ; ++i) {
          h[q + i] = fmaf(fast_exp2(d[k] * A2[q + i]), h[q + i], now[i / 4][0][i % 4] * u);
          if (OUT) y[k] = fmaf(now[i / 4][1][i % 4], h[q + i], y[k]);
        }
#pragma unroll
        for (int j = 0; j < kQ / 4; ++j) now[j][0] = next[j][0], now[j][1] = next[j][1];
      }
      if (GATED) y[k] *= silu(gate[k]);
      asm volatile("" : "+v"(y[k]));  // the sums are formed here, not where they are stored: every state would stay alive
    }
    if (OUT && mine) {
#pragma unroll
      for (int k = 0; k < kStep; ++k)
        if (t + k < count) (yp + k * p.D)[c] = from_f32<T>(y[k]);
    }
    yp += kStep * p.D;
  };
  auto save = [&](int64_t t) {
    if (OUT && p.states && t % CH == 0 && mine) {
      float* q = p.states + rec(b, t / CH, p.chunks, p.D, ch, RP);
      save_state<NP>(q, h);
#pragma unroll
      for (int n = NP; n < RP; n += 4) *reinterpret_cast<f32x4*>(q + n) = f32x4{0, 0, 0, 0};
    }
  };
  const bool works = c0 < p.Dg;  // a spare wave only helps to stage
  fetch_rows(0);
  if (works && count > 0) fetch();
  int buf = 0;
  for (int t0 = 0; t0 < count; t0 += tile, buf ^= 1) {
    float(*rows)[W] = s_row[buf];
#pragma unroll
    for (int k = 0; k < STAGE; ++k) (&rows[0][0])[threadIdx.x + threads * k] = to_f32(stage[k]);
    __syncthreads();  // the rows are there; and every wave has left the other buffer, which is written next
    if (t0 + tile < count) fetch_rows(t0 + tile);
    if (!works) continue;
    const int n = count - t0 < tile ? count - t0 : tile;
    for (int t = 0; t < n; t += kStep) {
      save(t_begin + t0 + t);
      run(rows + t, t0 + t);
    }
  }
  if (OUT) {
    yp = static_cast<T*>(p.y) + int64_t(b) * p.T * p.D + ch0;
    if (mine)
      for (int64_t t = t_begin + count; t < t_end; ++t) {
        yp[t * p.D + c] = from_f32<T>(0.0f);
        save(t);
      }
    if (seg == p.S - 1 && p.h_final && mine) {
#pragma unroll
      for (int n = 0; n < NP; ++n)
        if (n < p.N) p.h_final[(int64_t(b) * p.D + ch) * p.N + n] = h[n];
    }
  } else if (mine) {
    save_state<NP>(p.seg_h + rec(b, seg, p.S, p.D, ch, NP), h);
    p.seg_d[(int64_t(b) * p.S + seg) * p.D + ch] = dsum;
  }
}

// In place: the records of segments (what each leaves by itself) become what each starts from,
//   start_0 = init, start_1 = own_0 (the first ran from init), start_(s+1) = exp(A d_s) start_s + own_s.
// A workgroup takes 64 adjacent (channel, state) chains; its RUNS rows of 64 threads take a run of segments each: first
// a run's decay and own end, then, from the runs before it, its segments' starts.  Bound by reading and writing the
// records.  RUNS = 1 reads them once and is for few segments or more workgroups than are resident at a time (131072
// chains of 63 segments 17 us, RUNS = 16 28; 65536 chains of 63 segments 10.4 and 14.4).  RUNS = 16 has 16 times the
// loads in flight (1152 chains of 1308 segments 23 us, RUNS = 1 83; 32768 chains of 255 segments 22 and 24.5; 8192
// chains of 39 segments 5.2 and 6.1).
template <int RUNS>
__global__ __launch_bounds__(64 * RUNS) void k_scan_join(ScanJoin p) {
  constexpr int AHEAD = RUNS == 1 ? 32 : 8;  // segments whose loads are in flight together
  __shared__ float s_f[RUNS][64], s_v[RUNS][64];
  const int run = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t per = p.D * p.NP, chains = (per + 63) / 64, b = blockIdx.x / chains, e = blockIdx.x % chains * 64 + lane;
  const bool on = e < per;
  const int64_t ch = on ? e / p.NP : 0;
  const int n = on ? int(e - ch * p.NP) : 0;
  const float A2 = on && n < p.N ? p.A[ch * p.N + n] * kLog2e : 0.0f;
  const float init = on && p.init && n < p.N ? p.init[(b * p.D + ch) * p.N + n] : 0.0f;
  const int len = (p.S + RUNS - 1) / RUNS, s0 = run * len, s1 = s0 + len < p.S ? s0 + len : p.S;
  // Addresses step through the records: a product of 64 bits for each would be most of the work.
  const int64_t h_step = p.reverse ? -per : per, d_step = p.reverse ? -p.D : p.D, first = p.reverse ? p.S - 1 - s0 : s0;
  float* const q0 = p.h + (b * p.S + first) * per + (on ? e : 0);
  const float* const d0 = p.d + (b * p.S + first) * p.D + ch;
  // Nothing follows the last segment: it has no record of its own.  Loads do not depend on conditions (a branch between
  // them would wait), so what is behind the last repeats it and is masked when used.
  const int known = s1 < p.S ? s1 : p.S - 1;
  float own[AHEAD], step[AHEAD];
  const float *q = q0, *d = d0;
  auto fetch = [&](int s) {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      own[k] = *q;
      step[k] = *d;
      const bool more = s + k + 1 < known;
      q += more ? h_step : 0;
      d += more ? d_step : 0;
    }
    __builtin_amdgcn_sched_barrier(0);  // all on their way before the first is used
  };
  float f = 1.0f, v = 0.0f;
  for (int s = s0; RUNS > 1 && s < known; s += AHEAD) {
    fetch(s);
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const bool in = s + k < known;
      const float a = s + k == 0 ? 0.0f : fast_exp2(A2 * step[k]);
      const float next = s + k == 0 ? own[k] : fmaf(a, v, own[k]);
      v = in ? next : v;
      f *= in ? a : 1.0f;
    }
  }
  s_f[run][lane] = f, s_v[run][lane] = v;
  __syncthreads();
  float h = init;
  for (int i = 0; i < run; ++i) h = i == 0 && s_f[0][lane] == 0.0f ? s_v[0][lane] : fmaf(s_f[i][lane], h, s_v[i][lane]);
  float* out = q0;
  q = q0, d = d0;
  for (int s = s0; s < s1; s += AHEAD) {
    if (s < known) fetch(s);
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (s + k < s1) {
        if (on) *out = h;
        out += h_step;
      }
      h = s + k == 0 ? own[k] : fmaf(fast_exp2(A2 * step[k]), h, own[k]);
    }
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

// Bound by reading and writing the states: 64 sequences of 2048 channels and 16 states 7 us, 18 MB.
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

// Segments: enough waves for four on every SIMD, of 8 tokens and more (16 for T > 4096: 128 channels of 18292 tokens
// would have 2287 segments to join, and a long chain of them takes as long as it saves); for eight where segments stay
// longer than 128 tokens (439 against 447 us at T = 8192, 4 x 2048 channels, 835 against 864 at T = 65536, 2048
// channels; the states of segments are written and read twice, which costs short ones more than it gives).
ScanSplit split(int64_t B, int64_t T, int64_t D, int64_t G) {
  const int64_t waves = B * G * ceil_div(D / G, 64);
  ScanSplit s;
  int64_t want = waves >= 4096 ? 1 : ceil_div(4096, waves);
  if (want > 1 && T / want >= 256) want = ceil_div(8192, waves);
  const int64_t most = ceil_div(T, T > 4096 ? 16 : 8);
  if (want > most) want = most;
  s.len = ceil_div(ceil_div(T, want), kStep) * kStep;
  s.S = ceil_div(T, s.len);
  return s;
}

int64_t align256(int64_t v) { return (v + 255) / 256 * 256; }

}  // namespace

int64_t scan_join_workgroups(int64_t B, int64_t D, int64_t NP) { return B * ceil_div(D * NP, 64); }

hipError_t launch_scan_join(const ScanJoin& p, hipStream_t st) {
  const int64_t wgs = scan_join_workgroups(p.B, p.D, p.NP);
  if (p.S > 16 && wgs <= 512) k_scan_join<16><<<dim3(unsigned(wgs)), 1024, 0, st>>>(p);
  else k_scan_join<1><<<dim3(unsigned(wgs)), 64, 0, st>>>(p);
  return hipGetLastError();
}

int scan_state_blocks(int64_t N) { return N <= 16 ? 1 : (N <= 32 ? 2 : 4); }
int64_t scan_states_bytes(int64_t B, int64_t T, int64_t D, int64_t N) {
  return B * ceil_div(T, kScanChunk) * D * 16 * scan_state_blocks(N) * 4;
}
namespace {
int lane_states(int64_t N) { return N <= 8 ? 8 : (N <= 16 ? 16 : (N <= 24 ? 24 : (N <= 32 ? 32 : 64))); }

struct FwdLayout {
  ScanSplit split;
  int64_t seg_d, total;  // the segments' states come first
};
FwdLayout layout(int64_t B, int64_t T, int64_t D, int64_t N, int64_t G) {
  const int64_t NP = lane_states(N);
  FwdLayout l;
  l.split = split(B, T, D, G);
  l.seg_d = l.split.S > 1 ? align256(B * l.split.S * D * NP * 4) : 0;
  l.total = l.seg_d + (l.split.S > 1 ? align256(B * l.split.S * D * 4) : 0);
  return l;
}

template <typename T, int NP>
hipError_t run_fwd(const ScanDev& p, hipStream_t st) {
  const int64_t per = int64_t(p.cblocks) * p.B;
  if (p.S > 1) {
    k_scan_fwd<T, NP, false, false><<<dim3(unsigned(per * (p.S - 1))), 64 * p.waves, 0, st>>>(p);
    const hipError_t e = launch_scan_join({p.A, p.h0, p.seg_h, p.seg_d, p.B, p.S, p.D, p.N, NP, false}, st);
    if (e != hipSuccess) return e;
  }
  const dim3 grid(unsigned(per * p.S));
  if (p.z.p) k_scan_fwd<T, NP, true, true><<<grid, 64 * p.waves, 0, st>>>(p);
  else k_scan_fwd<T, NP, true, false><<<grid, 64 * p.waves, 0, st>>>(p);
  return hipGetLastError();
}

template <typename T>
hipError_t run_fwd(const ScanDev& p, hipStream_t st) {
  switch (lane_states(p.N)) {
    case 8: return run_fwd<T, 8>(p, st);
    case 16: return run_fwd<T, 16>(p, st);
    case 24: return run_fwd<T, 24>(p, st);
    case 32: return run_fwd<T, 32>(p, st);
    default: return run_fwd<T, 64>(p, st);
  }
}
}  // namespace

int64_t scan_fwd_workspace(int64_t B, int64_t T, int64_t D, int64_t N, int64_t G) { return layout(B, T, D, N, G).total; }

bool scan_fwd_launchable(const ScanArgs& a) {
  const FwdLayout l = layout(a.B, a.T, a.D, a.N, a.G);
  const int64_t waves = ceil_div(a.D / a.G, 64), blocks = ceil_div(waves, kWaves);
  return launchable(a.B * a.G * blocks * l.split.S, int(64 * ceil_div(waves, blocks))) &&
         (l.split.S == 1 || launchable(scan_join_workgroups(a.B, a.D, lane_states(a.N)), 64));
}

bool scan_step_launchable(const ScanArgs& a) { return launchable(ceil_div(a.B * a.D, 64), 256); }

hipError_t launch_scan_fwd(const ScanArgs& a, hipStream_t st) {
  const FwdLayout l = layout(a.B, a.T, a.D, a.N, a.G);
  ScanDev p = {};
  p.x = a.x, p.dt = a.dt, p.z = a.z, p.Bm = a.Bm, p.Cm = a.Cm;
  p.A = a.A, p.skip = a.skip, p.dt_bias = a.dt_bias, p.h0 = a.h0, p.lengths = a.lengths;
  p.h_final = a.h_final, p.states = a.states, p.y = a.y;
  p.T = a.T, p.D = a.D, p.chunks = ceil_div(a.T, kScanChunk);
  p.N = int(a.N), p.G = int(a.G), p.Dg = int(a.D / a.G);
  const int64_t waves = ceil_div(p.Dg, 64);  // of a group: as few workgroups as hold them, of equal size
  p.blocks = int(ceil_div(waves, kWaves)), p.waves = int(ceil_div(waves, p.blocks)), p.cblocks = int(p.blocks * a.G);
  p.S = int(l.split.S), p.B = int(a.B), p.len = l.split.len;
  p.softplus = a.softplus;
  char* ws = static_cast<char*>(a.workspace);
  p.seg_h = reinterpret_cast<float*>(ws), p.seg_d = reinterpret_cast<float*>(ws + l.seg_d);
  return a.dtype == 1 ? run_fwd<__bf16>(p, st) : run_fwd<float>(p, st);
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
