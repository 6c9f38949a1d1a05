// Group norm over channels-last rows, with its activation and an optional gate:
//   u = (x - mean) rstd w + b,  y = act(u), or u act(z) with a gate z;
// mean and variance over the S tokens and C / G channels of a group.
//
// Bound by memory.  bf16: rows form, 65536 tokens of 16 groups of 128 channels with a gate 147 us, 5.5 TB/s (a copy
// reaches 5.2); backward of 8064 such tokens 33 us, 5.0 TB/s, and 5 for the sums of dw and db.  Slab form, 4 x 8192
// tokens of 32 groups of 32 channels: statistics 14 us (4.7 TB/s), their combination 5, output 24 us (5.5 TB/s).
// Two forms:
//   rows  (S = 1, the norm of every token by itself): a group's values stay in the registers of up to 64
//         lanes, or of a workgroup, between the statistics and the output; one pass over the data.
//   slab  (statistics over tokens too): partial statistics of runs of tokens, their combination, and a
//         second pass (a sequence's rows do not fit on a compute unit; short ones, which would, go the same way).
//         Partial statistics are means and centred sums of squares, merged pairwise, so that a large mean costs no
//         precision.  One workgroup to a sequence and group combines them, so that few groups in all take long: one
//         sequence of 65536 tokens of 1024 bf16 channels in one group 313 us, its training step 2112 us.
#include "ll_layer.hpp"
#include "ll_layer_device.hpp"

namespace ll {

namespace {

struct NormDev {
  Rows x, z;
  const float *weight, *bias;
  void* y;
  float* stats;        // [N, G, 2]; may be null in the rows form
  const void* dy;
  void *dx, *dz;
  float* part;         // backward: [rows, 2, C] partial sums of du xh and du; slab forward: [N, chunks, ncv, 2]
  float* coef;         // slab backward: [N, G, 2]
  int64_t N, S, C, per, chunks, ncv;  // per: rows form, workgroups over the rows; slab, tokens of a chunk
  int G, cg, act, vec, pvec;  // pvec: a lane's weights and biases are 16-byte aligned
  int nvg, lanes;       // slab: channel vectors of a group (the last may be short), of a workgroup
  int slots, bpr, rpw;  // rows form: lanes of a row, workgroups of a row, rows of a workgroup
  float eps;
};

__device__ inline float act_of(float v, int act) { return act ? silu(v) : v; }
__device__ inline float act_grad(float v, int act) { return act ? silu_grad(v, sigmoidf(v)) : 1.0f; }

// Sum over LG adjacent lanes (LG = 256: a strip of the workgroup), in every lane.
template <int LG>
__device__ inline float group_sum(float v, float* s) {
  if (LG > 1) v += dpp_mov<0xB1>(v);   // quad_perm 1,0,3,2
  if (LG > 2) v += dpp_mov<0x4E>(v);   // quad_perm 2,3,0,1
  if (LG > 4) v += dpp_mov<0x141>(v);  // row_half_mirror
  if (LG > 8) v += dpp_mov<0x140>(v);  // row_mirror
  if (LG > 16) {
    const auto p = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    v = __builtin_bit_cast(float, (unsigned)p[0]) + __builtin_bit_cast(float, (unsigned)p[1]);
  }
  if (LG > 32) {
    const auto p = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    v = __builtin_bit_cast(float, (unsigned)p[0]) + __builtin_bit_cast(float, (unsigned)p[1]);
  }
  if (LG > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    s += threadIdx.x >> 8 << 2;
    v = (s[0] + s[1]) + (s[2] + s[3]);
  }
  return v;
}

// A lane's V channels of a group: the group's last vector, where it would be short, is moved back over the one before
// (both lanes then store the same outputs), so that all loads and stores are whole vectors; what it takes part with in
// sums is channels lo .. n - 1 of the vector.  Groups of less than a vector: channels 0 .. n - 1.
struct Place {
  int c = 0, lo = 0, n = 0;  // c: the first channel, within the group; n = 0: none
  __device__ Place() {}
  __device__ Place(int at, int cg, int V) {
    if (at >= cg) return;
    c = at, n = cg - at < V ? cg - at : V;
    if (n < V && cg >= V) c = cg - V, lo = V - n, n = V;
  }
  __device__ bool has(int i) const { return i >= lo && i < n; }
};

// out[i] = v[i] for the channels that count.
template <int V>
__device__ inline void store_sums(float* out, const Place& at, const float* v) {
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (at.has(i)) out[i] = v[i];
}

// What a thread of the rows form works on: vectors lane, lane + LG, .. of one group, in rows first, first + step, ..
// A workgroup is `strips` strips of 256 threads, each a row of its own (or rpw small ones).
struct RowPlan {
  int g, lane, strip;
  int64_t part, first, step;
  bool on;
  __device__ RowPlan(const NormDev& p, int LG, int strips) {
    strip = threadIdx.x >> 8;
    int slot = threadIdx.x & 255, row = 0;
    if (p.bpr > 1) {
      slot += int(blockIdx.x % p.bpr) * 256;
    } else {
      row = slot / p.slots;
      slot -= row * p.slots;
    }
    const int64_t blk = blockIdx.x / p.bpr;
    on = row < p.rpw && slot < p.slots;
    g = on ? slot / LG : 0;
    lane = slot % LG;
    part = blk * p.rpw + row;
    first = (blk * strips + strip) * p.rpw + row;
    step = p.per * strips * p.rpw;
  }
};

template <typename T, int V, int LG, int PV>
__global__ __launch_bounds__(256) void k_norm_rows(NormDev p) {
  typedef typename VecN<T, V>::type Vec;
  __shared__ float s[4];
  const RowPlan q(p, LG, 1);
  if (LG <= 64 && !q.on) return;
  float w[PV][V], bi[PV][V];
  int off[PV], n[PV];
  Place at[PV];
#pragma unroll
  for (int k = 0; k < PV; ++k) {
    at[k] = Place((q.lane + k * LG) * V, p.cg, V);
    n[k] = at[k].n;
    off[k] = q.g * p.cg + at[k].c;
    load_params<V>(p.weight ? p.weight + off[k] : nullptr, n[k], 1.0f, p.pvec, w[k]);
    load_params<V>(p.bias ? p.bias + off[k] : nullptr, n[k], 0.0f, p.pvec, bi[k]);
  }
  const float inv = 1.0f / float(p.cg);
  const bool gated = p.z.p;
  Vec xr[PV], zr[PV];
  auto fetch = [&](int64_t r) {
#pragma unroll
    for (int k = 0; k < PV; ++k) {
      const int m = r < p.N ? n[k] : 0;
      xr[k] = load_n<T, V>(static_cast<const T*>(p.x.p) + r * p.x.sb + off[k], m, p.vec);
      if (gated) zr[k] = load_n<T, V>(static_cast<const T*>(p.z.p) + r * p.z.sb + off[k], m, p.vec);
    }
  };
  fetch(q.first);
  for (int64_t r = q.first; r < p.N; r += q.step) {
    float x[PV][V], z[PV][V], sum = 0.0f;
#pragma unroll
    for (int k = 0; k < PV; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        x[k][i] = to_f32(T(xr[k][i]));
        if (gated) z[k][i] = to_f32(T(zr[k][i]));
        sum += at[k].has(i) ? x[k][i] : 0.0f;
      }
    fetch(r + q.step);
    const float mean = group_sum<LG>(sum, s) * inv;
    float sq = 0.0f;
#pragma unroll
    for (int k = 0; k < PV; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        x[k][i] -= mean;
        sq += at[k].has(i) ? x[k][i] * x[k][i] : 0.0f;
      }
    const float rstd = 1.0f / sqrtf(fmaf(group_sum<LG>(sq, s), inv, p.eps));
    if (p.stats && q.lane == 0) {
      p.stats[(r * p.G + q.g) * 2] = mean;
      p.stats[(r * p.G + q.g) * 2 + 1] = rstd;
    }
#pragma unroll
    for (int k = 0; k < PV; ++k) {
      float o[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float u = fmaf(x[k][i] * rstd, w[k][i], bi[k][i]);
        o[i] = gated ? u * act_of(z[k][i], p.act) : act_of(u, p.act);
      }
      store_n<T, V>(static_cast<T*>(p.y) + r * p.C + off[k], o, n[k], p.vec);
    }
  }
}

// Gradients of one vector: x centred and scaled to xh in place; returns du (in place of dy if asked) and, with a
// gate, dz.
template <int V>
__device__ inline void norm_du(const NormDev& p, bool gated, float mean, float rstd, const float* w, const float* b,
                               const float* dy, const float* z, float* xh, float* du, float* dz) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    xh[i] = (xh[i] - mean) * rstd;
    const float u = fmaf(xh[i], w[i], b[i]), d = dy[i];
    if (gated) {
      const float sg = p.act ? sigmoidf(z[i]) : 1.0f;
      du[i] = d * (p.act ? z[i] * sg : z[i]);
      dz[i] = d * u * (p.act ? silu_grad(z[i], sg) : 1.0f);
    } else {
      du[i] = d * act_grad(u, p.act);
    }
  }
}

// The product that both a group's mean and its elements' differences from that mean are formed of: rounded by itself
// in both, so that a group of one element has no gradient.
__device__ inline float rounded_mul(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}

// Strips of a backward workgroup: four of one vector a lane, fewer of more (registers).
template <int PV>
constexpr int kBwdStrips = 4 / PV;

// The next row's loads are on their way while a row is worked on.  `gated` is a template parameter because a wait for
// loads behind a store that may not have been issued waits for the store too (8064 rows of 2048 bf16 channels with a
// gate: 33 us, with a test in the loop 43).
template <typename T, int V, int LG, int PV, bool gated>
__global__ __launch_bounds__(256 * kBwdStrips<PV>) void k_norm_rows_bwd(NormDev p) {
  typedef typename VecN<T, V>::type Vec;
  constexpr int STRIPS = kBwdStrips<PV>;
  __shared__ float s[4 * STRIPS];
  __shared__ float s_sum[STRIPS > 1 ? STRIPS - 1 : 1][V][256];
  const RowPlan q(p, LG, STRIPS);
  float w[PV][V], bi[PV][V], dw[PV][V], db[PV][V];
  int off[PV], n[PV];
  Place at[PV];
#pragma unroll
  for (int k = 0; k < PV; ++k) {
    if (q.on) at[k] = Place((q.lane + k * LG) * V, p.cg, V);
    n[k] = at[k].n;
    off[k] = q.g * p.cg + at[k].c;
    load_params<V>(p.weight ? p.weight + off[k] : nullptr, n[k], 1.0f, p.pvec, w[k]);
    load_params<V>(p.bias ? p.bias + off[k] : nullptr, n[k], 0.0f, p.pvec, bi[k]);
#pragma unroll
    for (int i = 0; i < V; ++i) dw[k][i] = db[k][i] = 0.0f;
  }
  const float inv = 1.0f / float(p.cg);
  Vec xr[PV], zr[PV], gr[PV];
  float2 st = make_float2(0.0f, 0.0f);
  auto fetch = [&](int64_t r) {
    if (r < p.N) st = *reinterpret_cast<const float2*>(p.stats + (r * p.G + q.g) * 2);
#pragma unroll
    for (int k = 0; k < PV; ++k) {
      const int m = r < p.N ? n[k] : 0;
      xr[k] = load_n<T, V>(static_cast<const T*>(p.x.p) + r * p.x.sb + off[k], m, p.vec);
      gr[k] = load_n<T, V>(static_cast<const T*>(p.dy) + r * p.C + off[k], m, p.vec);
      if (gated) zr[k] = load_n<T, V>(static_cast<const T*>(p.z.p) + r * p.z.sb + off[k], m, p.vec);
    }
  };
  fetch(q.first);
  const int64_t rounds = (p.N + q.step - 1) / q.step;  // the same for all threads: sums over strips meet barriers
  for (int64_t i0 = 0; i0 < rounds; ++i0) {
    const int64_t r = q.first + i0 * q.step;
    const bool row = r < p.N;
    float x[PV][V], du[PV][V], z[PV][V], s1 = 0.0f, s2 = 0.0f;
    const float mean = st.x, rstd = st.y;
#pragma unroll
    for (int k = 0; k < PV; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        x[k][i] = to_f32(T(xr[k][i]));
        du[k][i] = to_f32(T(gr[k][i]));
        z[k][i] = gated ? to_f32(T(zr[k][i])) : 0.0f;
      }
    fetch(r + q.step);
#pragma unroll
    for (int k = 0; k < PV; ++k) {
      float dz[V];
      norm_du<V>(p, gated, mean, rstd, w[k], bi[k], du[k], z[k], x[k], du[k], dz);
      if (gated) store_n<T, V>(static_cast<T*>(p.dz) + r * p.C + off[k], dz, row ? n[k] : 0, p.vec);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const bool on = row && at[k].has(i);
        const float d = on ? du[k][i] : 0.0f;
        if (!row) x[k][i] = 0.0f;
        db[k][i] += d;
        dw[k][i] = fmaf(d, x[k][i], dw[k][i]);
        du[k][i] = rounded_mul(du[k][i], w[k][i]);
        const float dg = on ? du[k][i] : 0.0f;
        s1 += dg;
        s2 = fmaf(dg, x[k][i], s2);
      }
    }
    s1 = group_sum<LG>(s1, s) * inv;
    s2 = group_sum<LG>(s2, s) * inv;
#pragma unroll
    for (int k = 0; k < PV; ++k) {
      float o[V];
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] = rstd * ((du[k][i] - s1) - x[k][i] * s2);
      store_n<T, V>(static_cast<T*>(p.dx) + r * p.C + off[k], o, row ? n[k] : 0, p.vec);
    }
  }
  if (!p.part) return;
  // one row of partial sums for the workgroup's strips
  float* out = p.part + q.part * 2 * p.C;
  const int slot = threadIdx.x & 255;
#pragma unroll
  for (int k = 0; k < 2 * PV; ++k) {
    float(&v)[V] = k < PV ? dw[k % PV] : db[k % PV];
    __syncthreads();
    if (q.strip > 0) {
#pragma unroll
      for (int i = 0; i < V; ++i) s_sum[q.strip > 0 ? q.strip - 1 : 0][i][slot] = v[i];
    }
    __syncthreads();
    if (q.strip == 0) {
#pragma unroll
      for (int j = 0; j < STRIPS - 1; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] += s_sum[j][i][slot];
      store_sums<V>(out + (k < PV ? 0 : p.C) + off[k % PV], at[k % PV], v);
    }
  }
}

// ---- statistics over tokens

// Merges (n2, mean2, M2_2) into (n1, mean1, M2_1): counts, means and centred sums of squares.  The square of the means'
// difference is not formed by itself: beside nothing (n1 = 0) it is that of a mean, which may be beyond float32.
__device__ inline void merge(float& n1, float& m1, float& q1, float n2, float m2, float q2) {
  const float n = n1 + n2, d = m2 - m1;
  if (n2 == 0.0f) return;
  const float f = n2 / n;
  m1 = fmaf(d, f, m1);
  q1 += q2 + (d * n1) * (d * f);
  n1 = n;
}

// Threads of the slab kernels: `lanes` channel vectors x 256 / lanes strips of tokens.
template <int V>
struct SlabPlan {
  int lanes, strip, strips;
  int64_t cv, n, t0, t1, chunk;
  int g, width;  // the vector's group; its channels
  Place at;
  int64_t d0;    // its first channel
  __device__ SlabPlan(const NormDev& p) {
    lanes = p.lanes;
    strips = 256 / lanes;
    strip = threadIdx.x / lanes;
    const int64_t cblocks = (p.ncv + lanes - 1) / lanes;
    int64_t id = blockIdx.x;
    cv = id % cblocks * lanes + threadIdx.x % lanes;
    id /= cblocks;
    chunk = id % p.chunks;
    n = id / p.chunks;
    t0 = chunk * p.per;
    t1 = t0 + p.per < p.S ? t0 + p.per : p.S;
    g = int(cv / p.nvg);
    at = Place(int(cv - int64_t(g) * p.nvg) * V, p.cg, V);
    width = at.n;
    d0 = int64_t(g) * p.cg + at.c;
  }
  __device__ bool on(const NormDev& p) const { return strip < strips && cv < p.ncv; }
};

template <typename T, int V>
__global__ __launch_bounds__(256) void k_norm_slab_stats(NormDev p) {
  constexpr int U = 8;
  __shared__ float s[256][3];
  const SlabPlan<V> q(p);
  float cnt = 0.0f, mean = 0.0f, sq = 0.0f;
  if (q.on(p)) {
    const T* xp = static_cast<const T*>(p.x.p) + q.n * p.x.sb + q.d0;
    for (int64_t t = q.t0 + q.strip; t < q.t1; t += U * q.strips) {
      typename VecN<T, V>::type v[U];
#pragma unroll
      for (int k = 0; k < U; ++k) v[k] = load_n<T, V>(xp + (t + k * q.strips) * p.x.st, t + k * q.strips < q.t1 ? q.width : 0, p.vec);
      float a = 0.0f, b = 0.0f, m = 0.0f;
#pragma unroll
      for (int k = 0; k < U; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) a += q.at.has(i) ? to_f32(T(v[k][i])) : 0.0f;
#pragma unroll
      for (int k = 0; k < U; ++k) m += t + k * q.strips < q.t1 ? float(q.width - q.at.lo) : 0.0f;
      a /= m;
#pragma unroll
      for (int k = 0; k < U; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float d = to_f32(T(v[k][i])) - a;
          b += t + k * q.strips < q.t1 && q.at.has(i) ? d * d : 0.0f;
        }
      merge(cnt, mean, sq, m, a, b);
    }
  }
  s[threadIdx.x][0] = cnt, s[threadIdx.x][1] = mean, s[threadIdx.x][2] = sq;
  __syncthreads();
  if (q.strip == 0 && q.on(p)) {
    for (int k = 1; k < q.strips; ++k) {
      const float* o = s[threadIdx.x + k * q.lanes];
      merge(cnt, mean, sq, o[0], o[1], o[2]);
    }
    float* out = p.part + ((q.n * p.chunks + q.chunk) * p.ncv + q.cv) * 2;
    out[0] = mean, out[1] = sq;
  }
}

// One workgroup to a sequence and group: the chunks' and channel vectors' partial statistics.
__global__ __launch_bounds__(256) void k_norm_slab_join(NormDev p, int V) {
  __shared__ float s[256][3];
  const int64_t n = blockIdx.x / p.G;
  const int g = int(blockIdx.x % p.G), nv = p.nvg;
  float cnt = 0.0f, mean = 0.0f, sq = 0.0f;
  for (int64_t e = threadIdx.x; e < p.chunks * nv; e += 256) {
    const int64_t chunk = e / nv, cv = int64_t(g) * nv + e % nv;
    const float* o = p.part + ((n * p.chunks + chunk) * p.ncv + cv) * 2;
    const int64_t t = p.S - chunk * p.per < p.per ? p.S - chunk * p.per : p.per;
    const int last = p.cg - (nv - 1) * V, width = e % nv == nv - 1 ? last : V;
    merge(cnt, mean, sq, float(t) * float(width), o[0], o[1]);
  }
  for (int half = 128; half > 0; half >>= 1) {
    s[threadIdx.x][0] = cnt, s[threadIdx.x][1] = mean, s[threadIdx.x][2] = sq;
    __syncthreads();
    if (int(threadIdx.x) < half) {
      const float* o = s[threadIdx.x + half];
      merge(cnt, mean, sq, o[0], o[1], o[2]);
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    p.stats[blockIdx.x * int64_t(2)] = mean;
    p.stats[blockIdx.x * int64_t(2) + 1] = 1.0f / sqrtf(sq / cnt + p.eps);
  }
}

template <int V>
__device__ inline void slab_params(const NormDev& p, const SlabPlan<V>& q, float* w, float* b) {
  load_params<V>(p.weight ? p.weight + q.d0 : nullptr, q.width, 1.0f, p.pvec, w);
  load_params<V>(p.bias ? p.bias + q.d0 : nullptr, q.width, 0.0f, p.pvec, b);
}

template <typename T, int V>
__global__ __launch_bounds__(256) void k_norm_slab_out(NormDev p) {
  constexpr int U = 4;
  const SlabPlan<V> q(p);
  if (!q.on(p)) return;
  float w[V], b[V];
  slab_params<V>(p, q, w, b);
  const float* st = p.stats + (q.n * p.G + q.g) * 2;
  const float mean = st[0], rstd = st[1];
  const bool gated = p.z.p;
  const T* xp = static_cast<const T*>(p.x.p) + q.n * p.x.sb + q.d0;
  const T* zp = static_cast<const T*>(p.z.p) + q.n * p.z.sb + q.d0;
  T* yp = static_cast<T*>(p.y) + q.n * p.S * p.C + q.d0;
  for (int64_t t = q.t0 + q.strip; t < q.t1; t += U * q.strips) {
    typename VecN<T, V>::type x[U], z[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int64_t tk = t + k * q.strips;
      x[k] = load_n<T, V>(xp + tk * p.x.st, tk < q.t1 ? q.width : 0, p.vec);
      if (gated) z[k] = load_n<T, V>(zp + tk * p.z.st, tk < q.t1 ? q.width : 0, p.vec);
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      float o[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float u = fmaf((to_f32(T(x[k][i])) - mean) * rstd, w[i], b[i]);
        o[i] = gated ? u * act_of(to_f32(T(z[k][i])), p.act) : act_of(u, p.act);
      }
      const int64_t tk = t + k * q.strips;
      store_n<T, V>(yp + tk * p.C, o, tk < q.t1 ? q.width : 0, p.vec);
    }
  }
}

// Slab backward, first pass (OUT = false): a chunk's sums of du xh and du for every channel, from which come
// dw, db and, weighted, the two group sums that dx needs; with a gate, dz.  Second pass (OUT = true): dx.
template <typename T, int V, bool OUT, bool gated>
__global__ __launch_bounds__(256) void k_norm_slab_bwd(NormDev p) {
  constexpr int U = 2;
  __shared__ float s[OUT ? 1 : 256 * (2 * V + 1)];
  const SlabPlan<V> q(p);
  const bool on = q.on(p);
  float dw[V], db[V];
#pragma unroll
  for (int i = 0; i < V; ++i) dw[i] = db[i] = 0.0f;
  if (on) {
    float w[V], b[V];
    slab_params<V>(p, q, w, b);
    const int64_t grp = q.n * p.G + q.g;
    const float mean = p.stats[grp * 2], rstd = p.stats[grp * 2 + 1];
    const float s1 = OUT ? p.coef[grp * 2] : 0.0f, s2 = OUT ? p.coef[grp * 2 + 1] : 0.0f;
    const T* xp = static_cast<const T*>(p.x.p) + q.n * p.x.sb + q.d0;
    const T* zp = static_cast<const T*>(p.z.p) + q.n * p.z.sb + q.d0;
    const int64_t base = q.n * p.S * p.C + q.d0;
    for (int64_t t = q.t0 + q.strip; t < q.t1; t += U * q.strips) {
      typename VecN<T, V>::type x[U], z[U], g[U];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int64_t tk = t + k * q.strips;
        const int m = tk < q.t1 ? q.width : 0;
        x[k] = load_n<T, V>(xp + tk * p.x.st, m, p.vec);
        g[k] = load_n<T, V>(static_cast<const T*>(p.dy) + base + tk * p.C, m, p.vec);
        if (gated) z[k] = load_n<T, V>(zp + tk * p.z.st, m, p.vec);
      }
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int64_t tk = t + k * q.strips;
        float xf[V], dy[V], zf[V], du[V], dz[V], o[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          xf[i] = to_f32(T(x[k][i]));
          dy[i] = to_f32(T(g[k][i]));
          zf[i] = gated ? to_f32(T(z[k][i])) : 0.0f;
        }
        norm_du<V>(p, gated, mean, rstd, w, b, dy, zf, xf, du, dz);
        if (OUT) {
#pragma unroll
          for (int i = 0; i < V; ++i) o[i] = rstd * (fmaf(du[i], w[i], -s1) - xf[i] * s2);
          store_n<T, V>(static_cast<T*>(p.dx) + base + tk * p.C, o, tk < q.t1 ? q.width : 0, p.vec);
        } else if (tk < q.t1) {
          if (gated) store_n<T, V>(static_cast<T*>(p.dz) + base + tk * p.C, dz, q.width, p.vec);
#pragma unroll
          for (int i = 0; i < V; ++i) {
            db[i] += du[i];
            dw[i] = fmaf(du[i], xf[i], dw[i]);
          }
        }
      }
    }
  }
  if (!OUT) {
    float* mine = s + threadIdx.x * (2 * V + 1);
#pragma unroll
    for (int i = 0; i < V; ++i) mine[i] = dw[i], mine[V + i] = db[i];
    __syncthreads();
    if (q.strip == 0 && on) {
      for (int k = 1; k < q.strips; ++k) {
        const float* o = s + (threadIdx.x + k * q.lanes) * (2 * V + 1);
#pragma unroll
        for (int i = 0; i < V; ++i) dw[i] += o[i], db[i] += o[V + i];
      }
      float* out = p.part + (q.n * p.chunks + q.chunk) * 2 * p.C + q.d0;
      store_sums<V>(out, q.at, dw);
      store_sums<V>(out + p.C, q.at, db);
    }
  }
}

// coef = means over the group of g and g xh (g = du w), from the chunks' sums.
__global__ __launch_bounds__(256) void k_norm_slab_coef(NormDev p) {
  __shared__ float s[4];
  const int64_t n = blockIdx.x / p.G;
  const int g = int(blockIdx.x % p.G);
  float a = 0.0f, b = 0.0f;
  for (int64_t e = threadIdx.x; e < p.chunks * p.cg; e += 256) {
    const int64_t chunk = e / p.cg, c = int64_t(g) * p.cg + e % p.cg;
    const float* o = p.part + (n * p.chunks + chunk) * 2 * p.C + c;
    const float w = p.weight ? p.weight[c] : 1.0f;
    a = fmaf(w, o[p.C], a);
    b = fmaf(w, o[0], b);
  }
  const float inv = 1.0f / (float(p.S) * float(p.cg));
  a = group_sum<256>(a, s) * inv;
  b = group_sum<256>(b, s) * inv;
  if (threadIdx.x == 0) {
    p.coef[blockIdx.x * int64_t(2)] = a;
    p.coef[blockIdx.x * int64_t(2) + 1] = b;
  }
}

int elem(int dtype) { return dtype == 1 ? 2 : 4; }
int64_t align256(int64_t v) { return (v + 255) / 256 * 256; }

constexpr int kMaxPV = 4;  // vectors of a lane in the rows form

// The rows form: lanes of a group (a power of two up to 64, or a workgroup) and vectors of a lane.
struct RowShape {
  int V = 1, LG = 0, PV = 0;  // LG = 0: the group does not fit
};
RowShape row_shape(int64_t cg, int V) {
  RowShape r;
  r.V = V;
  const int64_t nv = ceil_div(cg, V);
  if (nv > 256 * kMaxPV) return r;
  if (nv > 64 * kMaxPV) {
    r.LG = 256;
  } else {
    r.LG = 1;
    while (r.LG < 64 && r.LG < nv) r.LG *= 2;
  }
  r.PV = 1;
  while (int64_t(r.LG) * r.PV < nv) r.PV *= 2;
  return r;
}

// Workgroups over the rows.  Forward: up to 16384, of two rows and more (65536 rows of 2048 bf16 with a gate: 146 us,
// 4096 workgroups 165, 2048, which end in a part of a round, 185).  Backward: 512 workgroups (of four strips where a
// lane has one vector); each leaves a row of sums.
int64_t row_blocks(int64_t rows, int rpw, int bpr, int most, int least) {
  const int64_t all = ceil_div(rows, rpw * least), want = ceil_div(most, bpr);
  return all < want ? all : want;
}

// Channel vectors of a slab workgroup, the other threads taking other tokens: all of them up to 256 (130 vectors: 49 us
// together, 55 in blocks of 64), beyond that the block of 256, 128 or 64 that leaves the fewest threads without work
// (training step of 64 x 512 fp32 tokens of 280 vectors: 374 us in blocks of 64, 467 in blocks of 256).
int64_t slab_lanes(int64_t ncv) {
  if (ncv <= 256) return ncv;
  int64_t best = 256;
  for (int64_t lanes = 128; lanes >= 64; lanes /= 2)
    if (ceil_div(ncv, lanes) * lanes < ceil_div(ncv, best) * best) best = lanes;
  return best;
}

// Tokens of a chunk of the slab form, for about 1024 workgroups.
int64_t slab_chunk(int64_t N, int64_t S, int64_t ncv) {
  const int64_t lanes = slab_lanes(ncv), strips = 256 / lanes, cblocks = ceil_div(ncv, lanes);
  int64_t chunks = ceil_div(1024, N * cblocks);
  const int64_t least = 8 * strips;
  int64_t per = ceil_div(S, chunks);
  return per < least ? least : per;
}

bool norm_vec(const NormArgs& a, const NormGrads* g) {
  const int e = elem(a.dtype), V = 16 / e;
  auto flat = [&](const void* q) { return !q || reinterpret_cast<uintptr_t>(q) % 16 == 0; };
  return (a.C / a.G) % V == 0 && rows_aligned(a.x, e, V) && (!a.z.p || rows_aligned(a.z, e, V)) && flat(a.y) &&
         (!g || (flat(g->dy) && flat(g->dx) && flat(g->dz)));
}

template <typename T, int V, int LG, int PV>
void go_rows_bwd(const NormDev& p, unsigned grid, hipStream_t st) {
  if (p.z.p) k_norm_rows_bwd<T, V, LG, PV, true><<<grid, 256 * kBwdStrips<PV>, 0, st>>>(p);
  else k_norm_rows_bwd<T, V, LG, PV, false><<<grid, 256 * kBwdStrips<PV>, 0, st>>>(p);
}

// The half vectors are the backward's, which takes whole ones only for groups that fit no other way.  A lane has one
// vector below 64 lanes, one, two or four at 64, two or four at 256.
template <typename T, int V, int LG>
void go_rows(const NormDev& p, int PV, unsigned grid, bool bwd, hipStream_t st) {
  constexpr bool kHalf = V * sizeof(T) == 8;
  constexpr int P1 = LG == 256 ? 2 : 1, P2 = LG >= 64 ? 2 : 1, P4 = LG >= 64 ? 4 : 1;
  if (!bwd) {
    if constexpr (!kHalf) {
      if (PV == 1) k_norm_rows<T, V, LG, P1><<<grid, 256, 0, st>>>(p);
      else if (PV == 2) k_norm_rows<T, V, LG, P2><<<grid, 256, 0, st>>>(p);
      else k_norm_rows<T, V, LG, P4><<<grid, 256, 0, st>>>(p);
    }
  } else if constexpr (!kHalf) {
    if constexpr (LG == 256) go_rows_bwd<T, V, LG, kMaxPV>(p, grid, st);
  } else {
    if (PV == 1) go_rows_bwd<T, V, LG, P1>(p, grid, st);
    else if (PV == 2) go_rows_bwd<T, V, LG, P2>(p, grid, st);
    else go_rows_bwd<T, V, LG, P4>(p, grid, st);
  }
}

template <typename T, int V>
void go_rows_lanes(const NormDev& p, const RowShape& r, unsigned grid, bool bwd, hipStream_t st) {
  switch (r.LG) {
    case 1: return go_rows<T, V, 1>(p, r.PV, grid, bwd, st);
    case 2: return go_rows<T, V, 2>(p, r.PV, grid, bwd, st);
    case 4: return go_rows<T, V, 4>(p, r.PV, grid, bwd, st);
    case 8: return go_rows<T, V, 8>(p, r.PV, grid, bwd, st);
    case 16: return go_rows<T, V, 16>(p, r.PV, grid, bwd, st);
    case 32: return go_rows<T, V, 32>(p, r.PV, grid, bwd, st);
    case 64: return go_rows<T, V, 64>(p, r.PV, grid, bwd, st);
    default: return go_rows<T, V, 256>(p, r.PV, grid, bwd, st);
  }
}

template <typename T>
void go_rows_form(const NormDev& p, const RowShape& r, unsigned grid, bool bwd, hipStream_t st) {
  constexpr int V = 16 / sizeof(T);
  if (r.V == V) go_rows_lanes<T, V>(p, r, grid, bwd, st);
  else go_rows_lanes<T, V / 2>(p, r, grid, bwd, st);
}

template <typename T>
void go_slab(const NormDev& p, unsigned grid, bool bwd, hipStream_t st) {
  constexpr int V = 16 / sizeof(T);
  const unsigned groups = unsigned(p.N * p.G);
  if (!bwd) {
    k_norm_slab_stats<T, V><<<grid, 256, 0, st>>>(p);
    k_norm_slab_join<<<groups, 256, 0, st>>>(p, V);
    k_norm_slab_out<T, V><<<grid, 256, 0, st>>>(p);
  } else if (p.z.p) {
    k_norm_slab_bwd<T, V, false, true><<<grid, 256, 0, st>>>(p);
    k_norm_slab_coef<<<groups, 256, 0, st>>>(p);
    k_norm_slab_bwd<T, V, true, true><<<grid, 256, 0, st>>>(p);
  } else {
    k_norm_slab_bwd<T, V, false, false><<<grid, 256, 0, st>>>(p);
    k_norm_slab_coef<<<groups, 256, 0, st>>>(p);
    k_norm_slab_bwd<T, V, true, false><<<grid, 256, 0, st>>>(p);
  }
}

// How a call is laid out and what it needs of the workspace.
struct NormPlan {
  RowShape rows;
  int bpr = 1, rpw = 1, slots = 0;
  int64_t per = 0, chunks = 0, ncv = 0, nvg = 0, part = 0, coef = 0, stats = 0, total = 0;
};
NormPlan plan(int64_t N, int64_t S, int64_t C, int64_t G, int dtype, bool bwd) {
  NormPlan q;
  const int V = 16 / elem(dtype);
  const int64_t cg = C / G;
  // A backward lane keeps its channels' parameters and sums too: half the vector (43 us instead of 57 for 8064 rows
  // of 2048 bf16 channels with a gate), where the group fits that way.
  if (S == 1) q.rows = row_shape(cg, bwd ? V / 2 : V);
  if (S == 1 && bwd && !q.rows.LG) q.rows = row_shape(cg, V);
  if (q.rows.LG) {
    const int64_t slots = G * q.rows.LG;
    q.slots = int(slots);
    q.bpr = int(slots > 256 ? ceil_div(slots, 256) : 1);
    q.rpw = int(slots > 256 ? 1 : 256 / slots);
    q.per = row_blocks(N, bwd ? q.rpw * (4 / q.rows.PV) : q.rpw, q.bpr, bwd ? 512 * q.rows.PV : 16384, bwd ? 1 : 2);
    q.total = bwd ? q.per * q.rpw * 2 * C * 4 : 0;
    return q;
  }
  q.nvg = ceil_div(cg, V);
  q.ncv = G * q.nvg;
  q.per = slab_chunk(N, S, q.ncv);
  q.chunks = ceil_div(S, q.per);
  q.part = align256(N * q.chunks * (bwd ? 2 * C : 2 * q.ncv) * 4);
  q.total = q.part + align256(N * G * 2 * 4);  // the group sums of a backward, a forward's statistics
  return q;
}

hipError_t launch(const NormArgs& a, const NormGrads* g, hipStream_t st) {
  NormDev p = {};
  p.vec = norm_vec(a, g);
  const NormPlan q = plan(a.N, a.S, a.C, a.G, a.dtype, g != nullptr);
  p.pvec = a.C / a.G % 4 == 0 && reinterpret_cast<uintptr_t>(a.weight) % 16 == 0 && reinterpret_cast<uintptr_t>(a.bias) % 16 == 0;
  p.x = a.x, p.z = a.z, p.weight = a.weight, p.bias = a.bias, p.y = a.y, p.stats = a.stats;
  p.N = a.N, p.S = a.S, p.C = a.C, p.G = int(a.G), p.cg = int(a.C / a.G), p.act = a.act, p.eps = a.eps;
  p.per = q.per, p.chunks = q.chunks, p.ncv = q.ncv, p.nvg = int(q.nvg), p.slots = q.slots, p.bpr = q.bpr, p.rpw = q.rpw;
  char* ws = static_cast<char*>(a.workspace);
  const bool bwd = g != nullptr, sums = bwd && (g->dw || g->db);
  if (bwd) p.dy = g->dy, p.dx = g->dx, p.dz = g->dz;
  int64_t rows;
  if (q.rows.LG) {
    p.part = sums ? reinterpret_cast<float*>(ws) : nullptr;
    rows = q.per * q.rpw;
    const unsigned grid = unsigned(q.per * q.bpr);
    if (a.dtype == 1) go_rows_form<__bf16>(p, q.rows, grid, bwd, st);
    else go_rows_form<float>(p, q.rows, grid, bwd, st);
  } else {
    p.part = reinterpret_cast<float*>(ws);
    p.coef = reinterpret_cast<float*>(ws + q.part);
    if (!bwd && !p.stats) p.stats = p.coef;
    rows = a.N * q.chunks;
    p.lanes = int(slab_lanes(q.ncv));
    const unsigned grid = unsigned(ceil_div(q.ncv, p.lanes) * rows);
    if (a.dtype == 1) go_slab<__bf16>(p, grid, bwd, st);
    else go_slab<float>(p, grid, bwd, st);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !sums) return e;
  ColSum c = {};
  c.part = p.part, c.rows = rows, c.stride = 2 * a.C;
  if (g->dw) c.out[c.n++] = {0, a.C, g->dw, a.C, a.C, 0, 1};
  if (g->db) c.out[c.n++] = {a.C, a.C, g->db, a.C, a.C, 0, 1};
  return launch_colsum(c, st);
}

}  // namespace

int64_t norm_workspace(int64_t N, int64_t S, int64_t C, int64_t G, int dtype, bool backward) {
  return plan(N, S, C, G, dtype, backward).total;
}

// The sums of columns hold at most 2^25 / 64 workgroups.
bool norm_launchable(const NormArgs& a, bool backward) {
  const NormPlan q = plan(a.N, a.S, a.C, a.G, a.dtype, backward);
  if (q.rows.LG) return launchable(q.per * q.bpr, 256 * (backward ? 4 / q.rows.PV : 1));
  return launchable(ceil_div(q.ncv, slab_lanes(q.ncv)) * a.N * q.chunks, 256) && launchable(a.N * a.G, 256);
}

hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t st) { return launch(a, nullptr, st); }
hipError_t launch_norm_bwd(const NormArgs& a, const NormGrads& g, hipStream_t st) { return launch(a, &g, st); }

}  // namespace ll
