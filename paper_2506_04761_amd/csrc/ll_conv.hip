// Short causal convolution over the tokens of each channel, with its activation:
//   v_td = b_d + sum_{j < W} w_dj e_(t+j)d,  e = (the W - 1 tokens before the first, x),  y = act(v).
//
// Bound by memory: a token and channel are read and written once (backward: x and dy read, dx written).
// A lane owns 8 bytes of adjacent channels and walks a run of tokens with the W - 1 tokens before it in
// registers, so that a token is read again only by the run after it.  16 bytes to a lane took 76 us where 8 take 60
// (the taps alone are then 32 registers).  bf16, W = 4: 32768 tokens of 2048 channels 51 us, 5.2 TB/s, the rate of a
// copy; forward of 8064 tokens 18 us (3.7 TB/s: a single round of waves), backward 29 us (3.4 TB/s).  One token for 64
// sequences 3.5 us, a launch's latency.  float32, 32768 tokens of 2048 channels 110 us, 4.9 TB/s.  Channels that are not
// whole vectors: 118 us for 2047 in bf16, 142 in float32, where each of the forward's loads and stores goes through the
// test for a short vector as well.
#include "ll_layer.hpp"
#include "ll_layer_device.hpp"

namespace ll {

namespace {

constexpr int kVecBytes = 8;   // of adjacent channels to a lane

struct ConvDev {
  Rows x;
  const float *weight, *bias;
  const void* state;
  void* new_state;
  const int32_t* lengths;
  void* y;
  // backward
  const void *dy, *dfinal;
  void *dx, *dinit;
  float* part;
  int64_t T, D, total;  // total: threads that have work
  int64_t ncv, runs;    // channel vectors; runs of tokens of a sequence
  int run;              // tokens of a run
  int act, vec, pvec;   // pvec: a lane's taps and biases are 16-byte aligned
};

__device__ inline int64_t live_tokens(const int32_t* lengths, int64_t b, int64_t T) {
  if (!lengths) return T;
  const int64_t n = lengths[b];
  return n < 0 ? 0 : (n > T ? T : n);
}

template <int W, int V>
__device__ inline void load_taps(const ConvDev& p, int64_t d0, int n, float (&w)[W][V], float (&bias)[V]) {
  float t[V * W];
  load_params<V * W>(p.weight + d0 * W, n * W, 0.0f, p.pvec, t);
  load_params<V>(p.bias ? p.bias + d0 : nullptr, n, 0.0f, p.pvec, bias);
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int j = 0; j < W; ++j) w[j][i] = t[i * W + j];
}

// Token t of sequence b as V floats; t < 0 comes from the state, t >= live and spare channels are zero.
template <typename T, int W, int V>
__device__ inline void token(const ConvDev& p, int64_t b, int64_t t, int64_t live, int64_t d0, int n, float* f) {
  typename VecN<T, V>::type v = {};
  if (t >= 0) {
    if (t < live) v = load_n<T, V>(static_cast<const T*>(p.x.p) + b * p.x.sb + t * p.x.st + d0, n, p.vec);
  } else if (p.state) {
    v = load_n<T, V>(static_cast<const T*>(p.state) + (b * (W - 1) + (t + W - 1)) * p.D + d0, n, p.vec);
  }
#pragma unroll
  for (int i = 0; i < V; ++i) f[i] = to_f32(T(v[i]));
}

template <typename T, int W>
__global__ __launch_bounds__(256) void k_conv_fwd(ConvDev p) {
  constexpr int V = kVecBytes / sizeof(T), U = 4;
  const int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (id >= p.total) return;
  const int64_t cv = id % p.ncv, run = id / p.ncv % p.runs, b = id / p.ncv / p.runs;
  const int64_t d0 = cv * V;
  const int n = p.D - d0 < V ? int(p.D - d0) : V;
  const int64_t t0 = run * p.run, t1 = t0 + p.run < p.T ? t0 + p.run : p.T;
  const int64_t live = live_tokens(p.lengths, b, p.T);
  float w[W][V], bias[V];
  load_taps<W, V>(p, d0, n, w, bias);
  float e[W - 1 + U][V];
#pragma unroll
  for (int j = 0; j < W - 1; ++j) token<T, W, V>(p, b, t0 - (W - 1) + j, live, d0, n, e[j]);

  if (p.new_state && run == 0) {  // the tokens before position `live`; the old state is in e by now
    T* out = static_cast<T*>(p.new_state) + b * (W - 1) * p.D + d0;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
      const int64_t t = live + j - (W - 1);
      float f[V];
      if (t >= 0) {
        token<T, W, V>(p, b, t, live, d0, n, f);
      } else {
#pragma unroll
        for (int k = 0; k < W - 1; ++k)
          if (k == t + (W - 1)) {
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = e[k][i];
          }
      }
      store_n<T, V>(out + j * p.D, f, n, p.vec);
    }
  }

  T* y = static_cast<T*>(p.y) + b * p.T * p.D + d0;
  const T* xp = static_cast<const T*>(p.x.p) + b * p.x.sb + d0;
  typename VecN<T, V>::type raw[U];
  auto fetch = [&](int64_t t) {
#pragma unroll
    for (int k = 0; k < U; ++k)
      raw[k] = load_n<T, V>(xp + (t + k) * p.x.st, t + k < live && t + k < t1 ? n : 0, p.vec);
  };
  fetch(t0);
  for (int64_t t = t0; t < t1; t += U) {
#pragma unroll
    for (int k = 0; k < U; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) e[W - 1 + k][i] = to_f32(T(raw[k][i]));
    if (t + U < t1) fetch(t + U);
#pragma unroll
    for (int k = 0; k < U; ++k) {
      float o[V];
      const bool in = t + k < live;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float v = bias[i];
#pragma unroll
        for (int j = 0; j < W; ++j) v = fmaf(w[j][i], e[k + j][i], v);
        if (p.act) v = silu(v);
        o[i] = in ? v : 0.0f;
      }
      store_n<T, V>(y + (t + k) * p.D, o, t + k < t1 ? n : 0, p.vec);
    }
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) e[j][i] = e[j + U][i];
  }
}

template <typename T, int W>
__global__ __launch_bounds__(256) void k_conv_step(ConvDev p) {
  constexpr int V = kVecBytes / sizeof(T);
  const int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (id >= p.total) return;
  const int64_t cv = id % p.ncv, b = id / p.ncv, d0 = cv * V;
  const int n = p.D - d0 < V ? int(p.D - d0) : V;
  float w[W][V], bias[V], e[W][V], o[V];
#pragma unroll
  for (int j = 0; j < W; ++j) token<T, W, V>(p, b, j - (W - 1), 1, d0, n, e[j]);
  load_taps<W, V>(p, d0, n, w, bias);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float v = bias[i];
#pragma unroll
    for (int j = 0; j < W; ++j) v = fmaf(w[j][i], e[j][i], v);
    o[i] = p.act ? silu(v) : v;
  }
  store_n<T, V>(static_cast<T*>(p.y) + b * p.D + d0, o, n, p.vec);
#pragma unroll
  for (int j = 0; j < W - 1; ++j)
    store_n<T, V>(static_cast<T*>(p.new_state) + (b * (W - 1) + j) * p.D + d0, e[j + 1], n, p.vec);
}

// Backward: dv_t = dy_t act'(v_t), dx_s = sum_j w_j dv_(s+W-1-j), dw_j = sum_t dv_t e_(t+j), db = sum_t dv_t.
// A lane walks its run and the W - 1 tokens after it (whose dv reach back into the run) and keeps the run's
// sums; the workgroup's four runs are added in LDS, and k_colsum adds the workgroups (4.7 us of 8064 tokens' 33).
// Registers (126 of the 128 that four waves a SIMD leave, and for bf16 with W = 4 four in scratch): taps, their sums, W
// tokens of x and of dv, loads ahead.
template <typename T, int W>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 4 : 5) void k_conv_bwd(ConvDev p) {
  constexpr int V = kVecBytes / sizeof(T);
  __shared__ float s_sum[4][64][V + 1];
  const int lane = threadIdx.x & 63, strip = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int64_t id = blockIdx.x;
  const int64_t cblocks = (p.ncv + 63) / 64, groups = (p.runs + 3) / 4;
  const int64_t cv = id % cblocks * 64 + lane;
  id /= cblocks;
  const int64_t run = id % groups * 4 + strip, b = id / groups;
  const int64_t d0 = cv * V;
  const int n = cv >= p.ncv || run >= p.runs ? 0 : (p.D - d0 < V ? int(p.D - d0) : V);
  float dw[W][V], db[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    db[i] = 0.0f;
#pragma unroll
    for (int j = 0; j < W; ++j) dw[j][i] = 0.0f;
  }
  if (n > 0) {
    const int64_t t0 = run * p.run, t1 = t0 + p.run < p.T ? t0 + p.run : p.T;
    const int64_t live = live_tokens(p.lengths, b, p.T);
    float w[W][V], bias[V], e[W][V], dv[W][V];
    load_taps<W, V>(p, d0, n, w, bias);
#pragma unroll
    for (int j = 0; j < W; ++j) {
      // a sequence without tokens has a part in no sum, whatever its state holds
      if (j > 0) token<T, W, V>(p, b, t0 - W + j, live, d0, live > 0 ? n : 0, e[j]);
#pragma unroll
      for (int i = 0; i < V; ++i) dv[j][i] = 0.0f;
    }
    const T* dyp = static_cast<const T*>(p.dy) + b * p.T * p.D + d0;
    const T* xp = static_cast<const T*>(p.x.p) + b * p.x.sb + d0;
    const T* dfp = p.dfinal ? static_cast<const T*>(p.dfinal) + b * (W - 1) * p.D + d0 : nullptr;
    T* dxp = static_cast<T*>(p.dx) + b * p.T * p.D + d0;
    typedef typename VecN<T, V>::type Vec;
    typedef typename VecN<T, V>::loose Loose;
    constexpr int U = 4;
    Vec xr[U], gr[U];
    const int64_t last = t1 + W - 1;  // one past the last dv that the run needs
    // Token t's dv (zero where !in), its share of the run's sums (where own), and o = dx of token t - (W - 1).
    auto step = [&](const Vec& xv, const Vec& gv, bool in, bool own, float* o) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
#pragma unroll
        for (int j = 0; j + 1 < W; ++j) e[j][i] = e[j + 1][i], dv[j][i] = dv[j + 1][i];
        e[W - 1][i] = to_f32(T(xv[i]));
        float g = to_f32(T(gv[i]));
        if (p.act) {
          float v = bias[i];
#pragma unroll
          for (int j = 0; j < W; ++j) v = fmaf(w[j][i], e[j][i], v);
          g *= silu_grad(v, sigmoidf(v));
        }
        g = in ? g : 0.0f;
        dv[W - 1][i] = g;  // dv[j] = dv of token t - (W - 1) + j
        const float own_g = own ? g : 0.0f;
        db[i] += own_g;
        float a = 0.0f;
#pragma unroll
        for (int j = 0; j < W; ++j) {
          dw[j][i] = fmaf(own_g, e[j][i], dw[j][i]);
          a = fmaf(w[j][i], dv[W - 1 - j][i], a);
        }
        o[i] = a;
      }
    };
    // A run of whole vectors and whole groups of U tokens, with as many live tokens after it as it needs: no load or
    // store depends on a condition, so that waiting for a load does not wait for what was issued after it.
    if (n == V && t1 - t0 == p.run && last + (U - W + 1) <= live && !(run == 0 && p.dinit)) {
      auto fetch = [&](int64_t t) {
#pragma unroll
        for (int k = 0; k < U; ++k) {
          xr[k] = *reinterpret_cast<const Loose*>(xp + (t + k) * p.x.st);
          gr[k] = *reinterpret_cast<const Loose*>(dyp + (t + k) * p.D);
        }
      };
      Vec xk[U], gk[U];
      auto next = [&] {
#pragma unroll
        for (int k = 0; k < U; ++k) xk[k] = xr[k], gk[k] = gr[k];
      };
      auto put = [&](int64_t s, const float* o) { store_n<T, V>(dxp + s * p.D, o, V, false); };
      float o[V];
      fetch(t0);
      next();
      fetch(t0 + U);
#pragma unroll
      for (int k = 0; k < U; ++k) {
        step(xk[k], gk[k], true, true, o);
        if (k >= W - 1) put(t0 + k - (W - 1), o);
      }
      for (int64_t t = t0 + U; t < t1; t += U) {
        next();
        fetch(t + U);
#pragma unroll
        for (int k = 0; k < U; ++k) {
          step(xk[k], gk[k], true, true, o);
          put(t + k - (W - 1), o);
        }
      }
#pragma unroll
      for (int k = 0; k < W - 1; ++k) {
        step(xr[k], gr[k], true, false, o);
        put(t1 + k - (W - 1), o);
      }
    } else {
      auto fetch = [&](int64_t t) {
#pragma unroll
        for (int k = 0; k < U; ++k) {
          const int m = t + k < live && t + k < last ? n : 0;
          xr[k] = load_n<T, V>(xp + (t + k) * p.x.st, m, p.vec);
          gr[k] = load_n<T, V>(dyp + (t + k) * p.D, m, p.vec);
        }
      };
      for (int64_t t = t0; t < last; t += U) {
        fetch(t);
#pragma unroll
        for (int k = 0; k < U; ++k) {
          const int64_t tk = t + k, s = tk - (W - 1);
          float o[V];
          step(xr[k], gr[k], tk < live && tk < last, tk < t1, o);
          if (dfp && s < live && s >= live - (W - 1)) {
            const Vec f = load_n<T, V>(dfp + (s - live + W - 1) * p.D, n, p.vec);
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] += to_f32(T(f[i]));
          }
          if (s >= t0 && s < t1) {
            store_n<T, V>(dxp + s * p.D, o, n, p.vec);
          } else if (s < 0 && run == 0 && p.dinit) {
            store_n<T, V>(static_cast<T*>(p.dinit) + (b * (W - 1) + s + W - 1) * p.D + d0, o, n, p.vec);
          }
        }
      }
    }
  }
  // sums of the four strips, one tap at a time
  float* part = p.part + blockIdx.x / cblocks * (W + 1) * p.D;
#pragma unroll
  for (int j = 0; j <= W; ++j) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) s_sum[strip][lane][i] = j < W ? dw[j < W ? j : 0][i] : db[i];
    __syncthreads();
    for (int q = threadIdx.x; q < 64 * V; q += 256) {
      const int l = q / V, i = q % V;
      const int64_t d = (cv - lane + l) * V + i;
      if (d < p.D) part[j * p.D + d] = (s_sum[0][l][i] + s_sum[1][l][i]) + (s_sum[2][l][i] + s_sum[3][l][i]);
    }
  }
}

// out[c] = sum over rows of part[row][col0 + c], 64 columns and 16 strips of rows to a workgroup.
__global__ __launch_bounds__(1024) void k_colsum(ColSum p) {
  __shared__ float s[16][64];
  const int lane = threadIdx.x & 63, strip = threadIdx.x >> 6;
  int64_t blk = blockIdx.x;
  int k = 0;
  while (blk >= (p.out[k].cols + 63) / 64) blk -= (p.out[k++].cols + 63) / 64;
  const ColSum::Out o = p.out[k];
  const int64_t c = blk * 64 + lane;
  float a = 0.0f;
  if (c < o.cols) {
    const float* q = p.part + o.col0 + c;
#pragma unroll 8
    for (int64_t r = strip; r < p.rows; r += 16) a += q[r * p.stride];
  }
  s[strip][lane] = a;
  __syncthreads();
  if (strip == 0 && c < o.cols) {
    float v = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) v += s[i][lane];
    const int64_t major = c / o.in_cols, minor = c % o.in_cols;
    if (minor < o.out_cols) o.out[major * o.major + minor * o.minor] = v;
  }
}

int elem(int dtype) { return dtype == 1 ? 2 : 4; }

// Tokens of a run: long enough that the W - 1 tokens read twice are few, short enough for 2^18 lanes, four waves on
// every SIMD at once (8064 tokens of 2048 channels, backward: runs of 16 28.8 us, of 12, which end in a part of a round,
// 31.8).
int run_length(int64_t B, int64_t T, int64_t ncv, int most) {
  int64_t r = B * T * ncv / (int64_t(1) << 18);
  r = r < 4 ? 4 : (r > most ? most : r);
  return int((r + 3) / 4 * 4);
}

bool conv_vec(const ConvArgs& a) {
  const int e = elem(a.dtype), V = kVecBytes / e;
  auto flat = [&](const void* q) { return !q || reinterpret_cast<uintptr_t>(q) % kVecBytes == 0; };
  return a.D % V == 0 && rows_aligned(a.x, e, V) && flat(a.y) && flat(a.state) && flat(a.new_state);
}

ConvDev conv_dev(const ConvArgs& a, int most) {
  ConvDev p = {};
  p.x = a.x, p.weight = a.weight, p.bias = a.bias, p.state = a.state, p.new_state = a.new_state;
  p.lengths = a.lengths, p.y = a.y, p.T = a.T, p.D = a.D, p.act = a.act, p.vec = conv_vec(a);
  p.pvec = p.vec && reinterpret_cast<uintptr_t>(a.weight) % 16 == 0 && reinterpret_cast<uintptr_t>(a.bias) % 16 == 0;
  p.ncv = ceil_div(a.D, kVecBytes / elem(a.dtype));
  p.run = run_length(a.B, a.T, p.ncv, most);
  p.runs = ceil_div(a.T, p.run);
  p.total = p.ncv * p.runs * a.B;
  return p;
}

constexpr int kFwdRun = 32, kBwdRun = 32;

template <typename T>
void go_fwd(const ConvDev& p, int W, hipStream_t st) {
  const dim3 grid(unsigned(ceil_div(p.total, 256)));
  if (W == 2) k_conv_fwd<T, 2><<<grid, 256, 0, st>>>(p);
  else if (W == 3) k_conv_fwd<T, 3><<<grid, 256, 0, st>>>(p);
  else k_conv_fwd<T, 4><<<grid, 256, 0, st>>>(p);
}

template <typename T>
void go_step(const ConvDev& p, int W, hipStream_t st) {
  const dim3 grid(unsigned(ceil_div(p.total, 256)));
  if (W == 2) k_conv_step<T, 2><<<grid, 256, 0, st>>>(p);
  else if (W == 3) k_conv_step<T, 3><<<grid, 256, 0, st>>>(p);
  else k_conv_step<T, 4><<<grid, 256, 0, st>>>(p);
}

template <typename T>
void go_bwd(const ConvDev& p, int W, unsigned grid, hipStream_t st) {
  if (W == 2) k_conv_bwd<T, 2><<<grid, 256, 0, st>>>(p);
  else if (W == 3) k_conv_bwd<T, 3><<<grid, 256, 0, st>>>(p);
  else k_conv_bwd<T, 4><<<grid, 256, 0, st>>>(p);
}

}  // namespace

int64_t conv_bwd_workspace(int64_t B, int64_t T, int64_t D, int64_t W, int dtype) {
  const int64_t runs = ceil_div(T, run_length(B, T, ceil_div(D, kVecBytes / elem(dtype)), kBwdRun));
  return B * ceil_div(runs, 4) * (W + 1) * D * 4;
}

hipError_t launch_colsum(const ColSum& p, hipStream_t st) {
  int64_t blocks = 0;
  for (int k = 0; k < p.n; ++k) blocks += ceil_div(p.out[k].cols, 64);
  k_colsum<<<dim3(unsigned(blocks)), 1024, 0, st>>>(p);
  return hipGetLastError();
}

// The sums of columns hold at most 5 x 2^24 / 64 workgroups.
bool conv_launchable(const ConvArgs& a, bool backward) {
  const ConvDev p = conv_dev(a, backward ? kBwdRun : kFwdRun);
  return launchable(backward ? ceil_div(p.ncv, 64) * a.B * ceil_div(p.runs, 4) : ceil_div(p.total, 256), 256);
}

hipError_t launch_conv_fwd(const ConvArgs& a, hipStream_t st) {
  const ConvDev p = conv_dev(a, kFwdRun);
  if (a.dtype == 1) go_fwd<__bf16>(p, int(a.W), st);
  else go_fwd<float>(p, int(a.W), st);
  return hipGetLastError();
}

hipError_t launch_conv_step(const ConvArgs& a, hipStream_t st) {
  const ConvDev p = conv_dev(a, kFwdRun);
  if (a.dtype == 1) go_step<__bf16>(p, int(a.W), st);
  else go_step<float>(p, int(a.W), st);
  return hipGetLastError();
}

hipError_t launch_conv_bwd(const ConvArgs& a, const ConvGrads& g, hipStream_t st) {
  ConvDev p = conv_dev(a, kBwdRun);
  auto flat = [&](const void* q) { return !q || reinterpret_cast<uintptr_t>(q) % kVecBytes == 0; };
  p.vec = p.vec && flat(g.dy) && flat(g.dfinal) && flat(g.dx) && flat(g.dinit);
  p.dy = g.dy, p.dfinal = g.dfinal, p.dx = g.dx, p.dinit = g.dinit, p.part = static_cast<float*>(g.workspace);
  const int64_t rows = a.B * ceil_div(p.runs, 4);
  const unsigned grid = unsigned(ceil_div(p.ncv, 64) * rows);
  if (a.dtype == 1) go_bwd<__bf16>(p, int(a.W), grid, st);
  else go_bwd<float>(p, int(a.W), grid, st);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  ColSum c = {};
  c.part = p.part, c.rows = rows, c.stride = (a.W + 1) * a.D;
  c.out[c.n++] = {0, a.W * a.D, g.dw, a.D, a.D, 1, a.W};  // [W][D] -> [D][W]
  if (g.db) c.out[c.n++] = {a.W * a.D, a.D, g.db, a.D, a.D, 0, 1};
  return launch_colsum(c, st);
}

}  // namespace ll
