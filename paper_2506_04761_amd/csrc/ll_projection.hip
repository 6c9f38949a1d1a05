// Projections: u = x W^T + bias, y = act(u) + residual, x [M, K], W [N, K], and their gradients
//   du = dy act'(u), dx = du W, dW = du^T x, dbias = sum over the rows of du.
//
// One kernel serves the three products.  Each is out[m, n] = sum_k a(n, k) b(m, k); an operand lies in memory
// "along" the reduction (x and W in the forward: rows of k) or "down" it (W in dx, du and x in dW: every row is one
// k).  A stage of 128 bytes of k of both operands is copied to LDS as it lies, and the fragments of the matrix
// instructions are read from there along or down the rows, so that nothing is transposed in memory.
//
// bf16: 32768 x 1024 to 4096 299 us, 919 TFLOP/s (the library's product 254); training step of 8064 x 2048 to 1024 143 us, 710
// TFLOP/s (in a kernel trace 41 the forward, 40 dx, 51 dW in four splits, 12 dbias).  The matrix cores are busy 42 % of the time, LDS 16 to 32 %:
// what bounds the products is the turn of a stage, its wait, barrier and first reads.
#include "ll_layer.hpp"
#include "ll_layer_device.hpp"

namespace ll {

namespace {

// A fragment is 16 bytes of k of each of 16 outputs: lane (g = lane / 16, i = lane % 16) holds k = KF / 4 * g + {0 ..}
// of output i.
template <typename T>
struct Op;
template <>
struct Op<__bf16> {
  static constexpr int KF = 32;
  typedef bf16x8 Frag;
  __device__ static inline f32x4 mma(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Op<float> {
  static constexpr int KF = 16;
  typedef f32x4 Frag;
  __device__ static inline f32x4 mma(Frag a, Frag b, f32x4 c) {
#pragma unroll
    for (int r = 0; r < 4; ++r) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[r], b[r], c, 0, 0, 0);
    return c;
  }
};

// Outputs are taken in pairs of 16: output i of fragment t is 32 (t / 2) + 8 (i / 4) + 4 (t % 2) + i % 4, so that the four
// results that a lane holds of each of a pair are eight adjacent ones.
__device__ inline int output_of(int t, int i) { return 32 * (t >> 1) + 8 * (i >> 2) + 4 * (t & 1) + (i & 3); }

constexpr int kStageBytes = 128;  // of k

// The LDS tile of TD outputs' stage: 16-byte chunks, chunk c of a row at c ^ key(row).  A read serves 256 bytes at a time,
// 16 lanes of 16 bytes or 32 of 8; with these keys it finds them in different banks: along, a chunk of the 16 rows
// output_of(t, 0 .. 15); down, two chunks of 8 rows (0 - 3 and 8 - 11) or in fp32 four chunks of four rows 4 apart.
// PAIRED: outputs in the order of output_of, else 16 t + i (down in bf16 half of a chunk each is read of a pair, so that
// the banks serve it at half their rate).
template <typename T, int TD, bool DOWN, bool PAIRED>
struct Tile {
  static constexpr int E = 16 / sizeof(T);
  static constexpr int BK = kStageBytes / sizeof(T);
  static constexpr int CH = DOWN ? TD / E : 8;  // chunks of a row
  __device__ static inline int key(int row) {
    const int b1 = (row >> 1) & 1, b3 = (row >> 3) & 1;
    if (!DOWN) return b1 | b3 << 1 | ((row >> 4) & 1) << 2;
    if (sizeof(T) == 4) return ((row >> 2) & 1) | (row & 8);
    return CH == 8 ? b1 << 1 | b3 << 2 : (row & 1) << 1 | b1 << 2 | b3 << 3;
  }
  __device__ static inline int output(int t, int i) { return PAIRED ? output_of(t, i) : 16 * t + i; }
  // Fragment t of k step ks of the outputs from d0 on.
  __device__ static inline typename Op<T>::Frag frag(const T* s, int d0, int t, int ks, int lane) {
    const int g = lane >> 4, i = lane & 15;
    if constexpr (!DOWN) {
      const int row = d0 + output(t, i);
      return *reinterpret_cast<const typename Op<T>::Frag*>(s + (row * CH + ((4 * ks + g) ^ key(row))) * E);
    } else if constexpr (sizeof(T) == 2) {
      // lane 4 j + c of 16 supplies four outputs of row j, see lds_read_tr
      const int row = 32 * ks + 8 * g + (i >> 2), d = d0 + output(t, 4 * (i & 3));
      const int at = (d >> 3) ^ key(row);
      const bf16x4 lo = lds_read_tr(s + (row * CH + at) * E + (d & 7));
      const bf16x4 hi = lds_read_tr(s + ((row + 4) * CH + at) * E + (d & 7));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      const int row = 16 * ks + 4 * g, d = d0 + output(t, i);
      const int at = (d >> 2) ^ key(row);
      f32x4 f;
#pragma unroll
      for (int r = 0; r < 4; ++r) f[r] = s[((row + r) * CH + at) * E + (d & 3)];
      return f;
    }
  }
};

// An operand: `n` outputs, rows of memory `stride` elements apart.
struct Side {
  const void* p;
  int64_t stride, n;
};

__device__ const uint4 kZeros = {0, 0, 0, 0};  // the k beyond the last

// Copies stages of an operand to LDS, 16 bytes a thread at a time: straight there (DIRECT: rows of whole, aligned
// chunks), or through registers (any rows; the last, short vector of a row is read moved back over the one before and
// shifted).  A stage's address is the same for all lanes, a lane's offset from it (at most
// 64 rows of less than 2^24 elements) the same for all stages.
template <typename T, typename Tl, int TD, bool DOWN, bool DIRECT, int NT>
struct Copy {
  typedef typename VecN<T, Tl::E>::type Vec;
  typedef typename VecN<T, Tl::E>::loose Loose;
  static constexpr int E = Tl::E, CH = Tl::CH, ITS = TD * 8 / NT, ROWS = NT / CH;
  const char* base;  // of the next stage
  int64_t turn, jump;  // bytes between stages, between a lane's rows
  unsigned off[ITS];
  int64_t n;         // outputs from the tile's first on
  Vec held[DIRECT ? 1 : ITS];
  int back[DIRECT ? 1 : ITS];  // elements that a short vector was moved back by
  bool movable;                // vectors lie before a short one

  __device__ inline void start(const Side& s, int64_t d0, int64_t k0, int64_t K) {
    n = s.n - d0;
    movable = (DOWN ? s.n : K) >= E;
    base = static_cast<const char*>(s.p) + (DOWN ? k0 * s.stride + d0 : d0 * s.stride + k0) * int64_t(sizeof(T));
    turn = (DOWN ? Tl::BK * s.stride : Tl::BK) * int64_t(sizeof(T));
    jump = ROWS * s.stride * int64_t(sizeof(T));
#pragma unroll
    for (int it = 0; it < ITS; ++it) {
      const int row0 = threadIdx.x / CH;
      off[it] = (unsigned(row0) * unsigned(s.stride) + chunk(row0 + it * ROWS) * E) * unsigned(sizeof(T));
    }
  }
  __device__ static inline int chunk(int row) { return (threadIdx.x % CH) ^ Tl::key(row); }
  // Begins the copy of the next stage, of which `left` k are inputs.
  __device__ inline void load(T* lds, int64_t left) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (left >= Tl::BK && n >= TD) {
#pragma unroll
      for (int it = 0; it < ITS; ++it) {
        if constexpr (DIRECT) copy16_to_lds(lds_address(lds + (it * NT + wave * 64) * E), base + it * jump, off[it]);
        else held[it] = *reinterpret_cast<const Loose*>(base + it * jump + off[it]), back[it] = 0;
      }
    } else {
#pragma unroll
      for (int it = 0; it < ITS; ++it) {
        const int row = threadIdx.x / CH + it * ROWS, c = chunk(row);
        const int64_t k = left - (DOWN ? row : c * E), d = n - (DOWN ? c * E : row);  // what is left from here on
        const char* src = base + it * jump + off[it];
        if constexpr (DIRECT) {
          copy16_to_lds(lds_address(lds + (it * NT + wave * 64) * E), k > 0 && d > 0 ? static_cast<const void*>(src) : &kZeros);
        } else {
          const int64_t whole = k <= 0 || d <= 0 ? 0 : (DOWN ? d : k);
          const int m = whole < E ? int(whole) : E;
          back[it] = movable && m > 0 ? E - m : 0;
          if (movable) held[it] = *static_cast<const Loose*>(m > 0 ? static_cast<const void*>(src - back[it] * int(sizeof(T))) : &kZeros);
          else held[it] = load_n<T, E>(reinterpret_cast<const T*>(src), m, false);
        }
      }
    }
    base += turn;
  }
  // Through registers: ends the copy.
  __device__ inline void store(T* lds) {
    if constexpr (!DIRECT) {
#pragma unroll
      for (int it = 0; it < ITS; ++it) {
        if (back[it]) held[it] = __builtin_bit_cast(Vec, __builtin_bit_cast(unsigned __int128, held[it]) >> (back[it] * int(sizeof(T)) * 8));
        *reinterpret_cast<Vec*>(lds + (it * NT + threadIdx.x) * E) = held[it];
      }
    }
  }
};

// What becomes of a product's sums.
struct Finish {
  void* out;           // [M, N]
  const float* bias;   // may be null
  const void* res;     // may be null
  int64_t res_stride;
  float* pre;          // may be null
  int64_t M, N;
  int act;
};

// V adjacent sums of row m from column n on.
template <typename T, int V>
__device__ inline void finish(const Finish& f, float* v, int64_t m, int64_t n) {
  if (m >= f.M || n >= f.N) return;
  const int count = f.N - n < V ? int(f.N - n) : V;
  if (f.bias) {
    float b[V];
    load_params<V>(f.bias + n, count, 0.0f, false, b);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] += b[i];
  }
  if (f.pre) store_n<float, V>(f.pre + m * f.N + n, v, count, false);
  if (f.act) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = silu(v[i]);
  }
  if (f.res) {
    const auto r = load_n<T, V>(static_cast<const T*>(f.res) + m * f.res_stride + n, count, false);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] += to_f32(T(r[i]));
  }
  store_n<T, V>(static_cast<T*>(f.out) + m * f.N + n, v, count, false);
}

struct GemmDev {
  Side a, b;               // outputs n, outputs m
  const void* low;         // TWO: what b's rounding leaves, laid out as b
  int64_t K, span;         // span: k of a split, whole stages
  int64_t m_tiles, n_tiles, splits;
  float* part;             // several splits: [splits, M, N] partial sums
  Finish f;
};

// TWO: the products of b's second part come after those of the first, into the same sums.
template <typename T, int TM, int TN, int WM, int WN, bool DOWN_M, bool DOWN_N, bool DIRECT, bool TWO = false>
__global__ __launch_bounds__(64 * WM * WN, 2) void k_gemm(GemmDev p) {
  constexpr int NT = 64 * WM * WN, FM = TM / WM / 16, FN = TN / WN / 16;
  typedef Tile<T, TM, DOWN_M, !(DOWN_M && sizeof(T) == 2)> TlM;
  typedef Tile<T, TN, DOWN_N, true> TlN;
  constexpr int BK = TlM::BK, KS = BK / Op<T>::KF;
  constexpr int kStage = (TM + TN) * BK;
  __shared__ __attribute__((aligned(1024))) T s[2 * kStage];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WN * (TM / WM), wn = wave % WN * (TN / WN);

  // an XCD takes adjacent tiles, eight rows of tiles at a time, so that its L2 serves both operands
  const unsigned m_tiles = unsigned(p.m_tiles), n_tiles = unsigned(p.n_tiles), tiles = m_tiles * n_tiles;
  unsigned id = unsigned(xcd_remap(blockIdx.x, int64_t(tiles) * p.splits));
  const unsigned split = id / tiles;
  id %= tiles;
  const unsigned strip = id / (8 * n_tiles), rows = m_tiles - 8 * strip < 8 ? m_tiles - 8 * strip : 8;
  id %= 8 * n_tiles;
  const int64_t m0 = int64_t(8 * strip + id % rows) * TM, n0 = int64_t(id / rows) * TN;

  const int64_t k0 = split * p.span;
  const int64_t own = p.K - k0 < p.span ? p.K - k0 : p.span;
  int64_t left = own;
  Copy<T, TlM, TM, DOWN_M, DIRECT, NT> cm;
  Copy<T, TlN, TN, DOWN_N, DIRECT, NT> cn;
  cm.start(p.b, m0, k0, p.K);
  cn.start(p.a, n0, k0, p.K);
  f32x4 acc[FM][FN] = {};
  cm.load(s, left);
  cn.load(s + TM * BK, left);
  cm.store(s);
  cn.store(s + TM * BK);
  const int stages = int((left + BK - 1) / BK);
  for (int st = 0; st < (TWO ? 2 : 1) * stages; ++st) {
    T* now = s + (st & 1) * kStage;
    T* next = s + (~st & 1) * kStage;
    if (DIRECT) copies_done();
    __syncthreads();
    left -= BK;
    if (TWO && st + 1 == stages) {
      cm.start({p.low, p.b.stride, p.b.n}, m0, k0, p.K);
      cn.start(p.a, n0, k0, p.K);
      left = own;
    }
    if (left > 0) {
      cm.load(next, left);
      cn.load(next + TM * BK, left);
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      typename Op<T>::Frag a[FN], b[FM];
#pragma unroll
      for (int j = 0; j < FN; ++j) a[j] = TlN::frag(now + TM * BK, wn, j, ks, lane);
#pragma unroll
      for (int i = 0; i < FM; ++i) b[i] = TlM::frag(now, wm, i, ks, lane);
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = Op<T>::mma(a[j], b[i], acc[i][j]);
    }
    if (left > 0) {
      cm.store(next);
      cn.store(next + TM * BK);
    }
  }
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    const int64_t m = m0 + wm + TlM::output(i, lane & 15);
#pragma unroll
    for (int j = 0; j < FN; j += 2) {
      const int64_t n = n0 + wn + 16 * j + 8 * (lane >> 4);
      float v[8];
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] = acc[i][j][r], v[4 + r] = acc[i][j + 1][r];
      if (p.part) {
        if (m < p.f.M && n < p.f.N)
          store_n<float, 8>(p.part + (split * p.f.M + m) * p.f.N + n, v, p.f.N - n < 8 ? int(p.f.N - n) : 8, false);
      } else {
        finish<T, 8>(p.f, v, m, n);
      }
    }
  }
}

// The splits' partial sums, added in their order, and what becomes of them.
template <typename T>
__global__ __launch_bounds__(256) void k_gemm_join(GemmDev p) {
  constexpr int V = 4;
  const int64_t per_row = (p.f.N + V - 1) / V, id = int64_t(blockIdx.x) * 256 + threadIdx.x;
  const int64_t m = id / per_row, n = id % per_row * V;
  if (m >= p.f.M) return;
  const int count = p.f.N - n < V ? int(p.f.N - n) : V;
  float v[V] = {};
#pragma unroll 4
  for (int64_t s = 0; s < p.splits; ++s) {
    const auto w = load_n<float, V>(p.part + (s * p.f.M + m) * p.f.N + n, count, false);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] += w[i];
  }
  finish<T, V>(p.f, v, m, n);
}

// A few rows (up to 16 MT): 16 outputs n to a workgroup, whose waves take 128 bytes of k each in turn, straight from
// memory, and are added at the end in their order.  Bound by the loads in flight: those of U turns are issued together
// (one row of 8192 x 8192 in bf16: 44 us one turn at a time, 29 with eight, 4.6 TB/s).
constexpr int kFewWaves = 8;
template <typename T, int MT, bool VEC>
__global__ __launch_bounds__(64 * kFewWaves) void k_few_rows(GemmDev p) {
  constexpr int E = 16 / sizeof(T), KF = Op<T>::KF, U = 8 / MT;
  typedef typename Op<T>::Frag Frag;
  __shared__ f32x4 s[kFewWaves][MT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, i = lane & 15;
  const int64_t n0 = int64_t(blockIdx.x) * 16;
  const int64_t arow = n0 + i < p.a.n ? n0 + i : p.a.n - 1;
  const T* a = static_cast<const T*>(p.a.p) + arow * p.a.stride + E * g;
  const T* b[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) b[t] = static_cast<const T*>(p.b.p) + (16 * t + i < p.b.n ? 16 * t + i : p.b.n - 1) * p.b.stride + E * g;
  f32x4 acc[MT] = {};
  constexpr int64_t kTurn = kFewWaves * 2 * KF;
  // `n` turns from k0 on; `whole`: all their k are inputs
  auto turns = [&](int64_t k0, auto n, auto whole) {
    constexpr int H = 2 * decltype(n)::value;
    Frag fa[H], fb[H][MT];
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const int64_t k = k0 + h / 2 * kTurn + h % 2 * KF;
      const int64_t left = p.K - k - E * g;
      const int m = whole.value || left >= E ? E : (left > 0 ? int(left) : 0);
      fa[h] = load_n<T, E>(a + k, m, VEC);
#pragma unroll
      for (int t = 0; t < MT; ++t) fb[h][t] = load_n<T, E>(b[t] + k, m, VEC);
    }
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int t = 0; t < MT; ++t) acc[t] = Op<T>::mma(fa[h], fb[h][t], acc[t]);
  };
  int64_t k0 = wave * 2 * KF;
  for (; k0 + (U - 1) * kTurn + 2 * KF <= p.K; k0 += U * kTurn) turns(k0, std::integral_constant<int, U>{}, std::true_type{});
  for (; k0 + kTurn + 2 * KF <= p.K; k0 += 2 * kTurn) turns(k0, std::integral_constant<int, 2>{}, std::true_type{});
  for (; k0 < p.K; k0 += kTurn) turns(k0, std::integral_constant<int, 1>{}, std::false_type{});
#pragma unroll
  for (int t = 0; t < MT; ++t) s[wave][t][lane] = acc[t];
  __syncthreads();
  for (int t = wave; t < MT; t += kFewWaves) {
    float v[4] = {};
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w)
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] += s[w][t][lane][r];
    finish<T, 4>(p.f, v, 16 * t + i, n0 + 4 * g);
  }
}

// du = dy act'(pre), rounded to the storage type for the two products that read it, and its sums over strips of rows,
// which take it as it is.  64 lanes of E columns and four rows at a time to a workgroup.
struct DuDev {
  const void* dy;
  const float* pre;  // null: du = dy, only the sums
  void* du;
  void* low;         // what du's rounding leaves; may be null
  float* part;       // [strips, N]; may be null
  int64_t M, N, rows, cols;  // rows of a strip, workgroups over the columns
};
template <typename T>
__global__ __launch_bounds__(256) void k_du(DuDev p) {
  constexpr int E = 16 / sizeof(T);
  __shared__ float s[4][64][E + 1];
  const int lane = threadIdx.x & 63, sub = threadIdx.x >> 6;
  const int64_t strip = blockIdx.x / p.cols, n = (blockIdx.x % p.cols * 64 + lane) * E;
  const int count = n >= p.N ? 0 : (p.N - n < E ? int(p.N - n) : E);
  // a row's last, short vector is moved back over the one before: it does again what that does, and counts its own
  const int64_t at = count > 0 && count < E && p.N >= E ? p.N - E : n;
  const int64_t end = (strip + 1) * p.rows < p.M ? (strip + 1) * p.rows : p.M;
  float sum[E] = {};
  auto row = [&](int64_t m, int c) {
    const auto g = load_n<T, E>(static_cast<const T*>(p.dy) + m * p.N + at, c, false);
    float d[E];
#pragma unroll
    for (int i = 0; i < E; ++i) d[i] = to_f32(T(g[i]));
    if (p.pre) {
      const auto u = load_n<float, E>(p.pre + m * p.N + at, c, false);
#pragma unroll
      for (int i = 0; i < E; ++i) d[i] *= silu_grad(u[i], sigmoidf(u[i]));
      store_n<T, E>(static_cast<T*>(p.du) + m * p.N + at, d, c, false);
      if (p.low) {
        float left[E];
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const float held = to_f32(from_f32<T>(d[i]));
          left[i] = d[i] == held ? 0.0f : d[i] - held;  // nothing of infinities
        }
        store_n<T, E>(static_cast<T*>(p.low) + m * p.N + at, left, c, false);
      }
    }
#pragma unroll
    for (int i = 0; i < E; ++i) sum[i] += d[i];
  };
  if (count > 0) {
    if (p.N >= E) {
#pragma unroll 4
      for (int64_t m = strip * p.rows + sub; m < end; m += 4) row(m, E);
    } else {
      for (int64_t m = strip * p.rows + sub; m < end; m += 4) row(m, count);
    }
  }
  if (!p.part) return;
  const int own = int(n - at);  // of the vector's elements, those before are the one before's
#pragma unroll
  for (int i = 0; i < E; ++i)
    if (i >= own) s[sub][lane][i - own] = sum[i];
  __syncthreads();
  for (int c = threadIdx.x; c < 64 * E; c += 256) {
    const int64_t col = blockIdx.x % p.cols * 64 * E + c;
    if (col < p.N) p.part[strip * p.N + col] = s[0][c / E][c % E] + s[1][c / E][c % E] + s[2][c / E][c % E] + s[3][c / E][c % E];
  }
}

// ------------------------------------------------------------------------------------ plans

int elem(int dtype) { return dtype == 1 ? 2 : 4; }

enum Product { kForward, kDx, kDw };

struct GemmPlan {
  int few = 0;             // fragments of 16 rows, or 0
  int tile = 0;            // outputs of a tile's sides
  int64_t m_tiles = 0, n_tiles = 0, splits = 1, span = 0;
  int64_t workgroups = 0;
  int64_t bytes = 0;       // of partial sums
};

// What a stage takes on a compute unit that holds n workgroups (at most `most`) of a tile, and a workgroup's results, in
// us: fitted to products of 128 to 65536 rows in 1 to 32 splits.  Of 69 measured ones the choice is within 5 % of the best of
// tiles and splits in 53, within 15 % in 61; the worst are 1001 x 1000 over 1501 in fp32, one side in unaligned rows (65 us,
// 47 in three splits), and 1000 x 4104 over 700 in bf16 (19.4, in tiles of 128 15.6).
struct TileCost {
  int tile, most;
  double stage, each, results;
};
constexpr TileCost kCosts[2][3] = {{{64, 5, 0.1, 0.6, 1.0}, {128, 2, 0.2, 2.1, 1.5}, {0, 0, 0, 0, 0}},
                                   {{64, 5, 0.35, 0.09, 1.0}, {128, 2, 0.39, 0.35, 1.5}, {256, 1, 0, 1.65, 5.0}}};

// out [M, N] over K: the tile and the splits of K that take the least time by those costs.  Larger tiles read less from
// LDS (8192 x 1024 over 8192 in bf16: tiles of 64 202 us, of 128 152, of 256 in two splits 133), smaller ones and splits
// fill more compute units (1024 x 1024 over 1024: 11.6, 15.2 and 26.6 us; 1024 x 2048 over 8064: 128 without splits 68, in
// four 49).
GemmPlan plan(int64_t M, int64_t N, int64_t K, int dtype, Product what, int largest = 256) {
  GemmPlan q;
  const int64_t BK = kStageBytes / elem(dtype), stages = ceil_div(K, BK);
  // what is read, at the rate of a copy; tiles' stages overlap with about half of it
  const double read = double(M + N) * K * elem(dtype) / 4.6e6;
  double best = 0;
  if (what == kForward && M <= 64) {
    // a workgroup's time is its K's, two on a compute unit take twice that (8192 x 8192: 16 rows 39 us, 32 54, 64 82)
    q.few = M <= 16 ? 1 : M <= 32 ? 2 : 4;
    q.workgroups = ceil_div(N, 16);
    const double units = q.workgroups > 256 ? q.workgroups / 256.0 : 1;
    best = K * units * 1e-3 * (M <= 4 ? 1.5 : M <= 16 ? 2.0 : M <= 32 ? 2.5 : 4.4) * (dtype == 1 ? 1 : 2.4);
    if (dtype == 1 && K % 8) best *= 1.8;  // unaligned rows (64 rows of 2047 x 4001 36 us, in tiles 17)
    best = best > read ? best : read;
    if (best <= 4) return q;  // less than tiles and their join take at all
  }
  for (const TileCost& c : kCosts[dtype]) {
    if (!c.tile || c.tile > largest) continue;
    const int64_t m_tiles = ceil_div(M, c.tile), n_tiles = ceil_div(N, c.tile);
    for (const int64_t want : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
      const int64_t each = ceil_div(stages, want), splits = ceil_div(stages, each);
      if (want > 1 && (want > stages / 2 || m_tiles * n_tiles * want > 2304)) break;
      const int64_t a_unit = ceil_div(m_tiles * n_tiles * splits, 256), rounds = a_unit / c.most, rest = a_unit % c.most;
      auto round = [&](int64_t n) { return n ? each * (c.stage + n * c.each) + c.results : 0.0; };
      const double join = splits > 1 ? 3 + double(splits) * M * N * 8 / 7e6 : 0;
      const double us = rounds * round(c.most) + round(rest) + read / 2 + join;
      if ((q.tile || q.few) && us >= best) continue;
      best = us;
      q.few = 0, q.tile = c.tile, q.m_tiles = m_tiles, q.n_tiles = n_tiles, q.splits = splits, q.span = each * BK;
    }
  }
  if (q.few) return q;
  q.workgroups = q.m_tiles * q.n_tiles * q.splits;
  q.bytes = q.splits > 1 ? q.splits * M * N * 4 : 0;
  return q;
}

int64_t up256(int64_t n) { return (n + 255) / 256 * 256; }

struct DuPlan {
  int64_t cols, rows, strips;
};
DuPlan du_plan(int64_t M, int64_t N, int dtype) {
  DuPlan q;
  q.cols = ceil_div(N, 64 * (16 / elem(dtype)));
  q.rows = ceil_div(M * q.cols, 512);
  q.rows = ceil_div(q.rows < 16 ? 16 : q.rows, 4) * 4;
  q.strips = ceil_div(M, q.rows);
  return q;
}

struct BwdPlan {
  GemmPlan dx, dw;
  DuPlan du;
  bool two = false;  // du in two bf16 parts, tiles of 64
  int64_t o_du = 0, o_low = 0, o_part = 0, total = 0;  // du; its second part; partial sums of whichever kernel runs
};
BwdPlan bwd_plan(int64_t M, int64_t K, int64_t N, int dtype, bool act) {
  BwdPlan q;
  // The roundings of few values of du do not average out (256 values: the gradient of the weight off by up to 1.55 times what
  // its own rounding takes, with 1024 by 1.48 as with many), and few are cheap to take twice: 1 x 2048 to 64 13.6 us either
  // way, 1 x 8192 to 1023 20.0 and 26.4.  Many are not: twice the products of 4096 x 1024 to 2816, 83 us.
  q.two = act && dtype == 1 && M * N < 1024;
  q.dx = plan(M, K, N, dtype, kDx, q.two ? 64 : 256);
  q.dw = plan(N, K, M, dtype, kDw, q.two ? 64 : 256);
  q.du = du_plan(M, N, dtype);
  q.o_low = act ? up256(M * N * elem(dtype)) : 0;
  q.o_part = q.two ? 2 * q.o_low : q.o_low;
  int64_t part = q.du.strips * N * 4;
  part = part < q.dx.bytes ? q.dx.bytes : part;
  part = part < q.dw.bytes ? q.dw.bytes : part;
  q.total = q.o_part + up256(part);
  return q;
}

bool direct(const Side& s, bool down, int64_t K, int esize) {
  const int e = 16 / esize;
  return reinterpret_cast<uintptr_t>(s.p) % 16 == 0 && s.stride % e == 0 && (down ? s.n : K) % e == 0;
}

template <typename T, int TILE, bool DM, bool DN, bool DIRECT, bool TWO = false>
void launch_tiles(const GemmDev& p, int64_t workgroups, hipStream_t st) {
  constexpr int WM = 2, WN = TILE == 256 ? 4 : 2;
  k_gemm<T, TILE, TILE, WM, WN, DM, DN, DIRECT, TWO><<<dim3(uint32_t(workgroups)), dim3(64 * WM * WN), 0, st>>>(p);
}

template <typename T, bool DM, bool DN>
void launch_tile(const GemmDev& p, const GemmPlan& q, hipStream_t st) {
  const bool dir = direct(p.b, DM, p.K, sizeof(T)) && direct(p.a, DN, p.K, sizeof(T));
  if constexpr (sizeof(T) == 2) {
    if constexpr (DN) {
      if (p.low) return dir ? launch_tiles<T, 64, DM, DN, true, true>(p, q.workgroups, st) : launch_tiles<T, 64, DM, DN, false, true>(p, q.workgroups, st);
    }
    if (q.tile == 256) dir ? launch_tiles<T, 256, DM, DN, true>(p, q.workgroups, st) : launch_tiles<T, 256, DM, DN, false>(p, q.workgroups, st);
  }
  if (q.tile == 128) dir ? launch_tiles<T, 128, DM, DN, true>(p, q.workgroups, st) : launch_tiles<T, 128, DM, DN, false>(p, q.workgroups, st);
  else if (q.tile == 64) dir ? launch_tiles<T, 64, DM, DN, true>(p, q.workgroups, st) : launch_tiles<T, 64, DM, DN, false>(p, q.workgroups, st);
}

// A product by its plan.
template <typename T, bool DM, bool DN>
hipError_t launch_product(GemmDev p, const GemmPlan& q, float* part, hipStream_t st) {
  p.m_tiles = q.m_tiles, p.n_tiles = q.n_tiles, p.splits = q.splits, p.span = q.span;
  p.part = q.bytes ? part : nullptr;
  launch_tile<T, DM, DN>(p, q, st);
  if (q.bytes) k_gemm_join<T><<<dim3(uint32_t(ceil_div(p.f.M * ceil_div(p.f.N, 4), 256))), dim3(256), 0, st>>>(p);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_few(const GemmDev& p, const GemmPlan& q, hipStream_t st) {
  const bool vec = direct(p.a, false, p.K, sizeof(T)) && direct(p.b, false, p.K, sizeof(T));
  const dim3 grid(uint32_t(q.workgroups)), block(64 * kFewWaves);
  if (q.few == 1) vec ? k_few_rows<T, 1, true><<<grid, block, 0, st>>>(p) : k_few_rows<T, 1, false><<<grid, block, 0, st>>>(p);
  else if (q.few == 2) vec ? k_few_rows<T, 2, true><<<grid, block, 0, st>>>(p) : k_few_rows<T, 2, false><<<grid, block, 0, st>>>(p);
  else vec ? k_few_rows<T, 4, true><<<grid, block, 0, st>>>(p) : k_few_rows<T, 4, false><<<grid, block, 0, st>>>(p);
  return hipGetLastError();
}

template <typename T>
hipError_t fwd(const ProjArgs& a, hipStream_t st) {
  const GemmPlan q = plan(a.M, a.N, a.K, a.dtype, kForward);
  GemmDev p = {};
  p.a = {a.weight, a.K, a.N}, p.b = {a.x, a.x_stride, a.M}, p.K = a.K;
  p.f = {a.y, a.bias, a.residual, a.residual_stride, a.pre, a.M, a.N, a.act};
  if (q.few) return launch_few<T>(p, q, st);
  return launch_product<T, false, false>(p, q, static_cast<float*>(a.workspace), st);
}

template <typename T>
hipError_t bwd(const ProjArgs& a, const ProjGrads& g, hipStream_t st) {
  const BwdPlan q = bwd_plan(a.M, a.K, a.N, a.dtype, a.act != 0);
  char* ws = static_cast<char*>(a.workspace);
  float* part = reinterpret_cast<float*>(ws + q.o_part);
  const void* du = a.act ? ws + q.o_du : g.dy;
  void* const low = q.two ? ws + q.o_low : nullptr;  // may be null
  hipError_t e = hipSuccess;
  if (a.act || g.dbias) {
    const DuDev d = {g.dy, a.act ? a.pre : nullptr, ws + q.o_du, low, g.dbias ? part : nullptr,
                      a.M, a.N, q.du.rows, q.du.cols};
    k_du<T><<<dim3(uint32_t(q.du.cols * q.du.strips)), dim3(256), 0, st>>>(d);
    e = hipGetLastError();
    if (e == hipSuccess && g.dbias) {
      ColSum c;
      c.part = part, c.rows = q.du.strips, c.stride = a.N, c.n = 1;
      c.out[0] = {0, a.N, g.dbias, a.N, a.N, 0, 1};
      e = launch_colsum(c, st);
    }
  }
  if (e == hipSuccess && g.dx) {
    GemmDev p = {};
    p.a = {a.weight, a.K, a.K}, p.b = {du, a.N, a.M}, p.low = low, p.K = a.N;
    p.f = {g.dx, nullptr, nullptr, 0, nullptr, a.M, a.K, 0};
    e = launch_product<T, false, true>(p, q.dx, part, st);
  }
  if (e == hipSuccess && g.dweight) {
    GemmDev p = {};
    p.a = {a.x, a.x_stride, a.K}, p.b = {du, a.N, a.N}, p.low = low, p.K = a.M;
    p.f = {g.dweight, nullptr, nullptr, 0, nullptr, a.N, a.K, 0};
    e = launch_product<T, true, true>(p, q.dw, part, st);
  }
  return e;
}

}  // namespace

int64_t projection_workspace(int64_t M, int64_t K, int64_t N, int act, int dtype, bool backward) {
  const int64_t f = up256(plan(M, N, K, dtype, kForward).bytes);
  if (!backward) return f;
  const int64_t b = bwd_plan(M, K, N, dtype, act != 0).total;
  return b > f ? b : f;
}

bool projection_launchable(int64_t M, int64_t K, int64_t N, int act, int dtype, bool backward) {
  auto ok = [](const GemmPlan& q, int64_t m, int64_t n) {
    return launchable(q.workgroups, 64 * kFewWaves) && (!q.bytes || launchable(ceil_div(m * ceil_div(n, 4), 256), 256));
  };
  if (!backward) return ok(plan(M, N, K, dtype, kForward), M, N);
  const BwdPlan q = bwd_plan(M, K, N, dtype, act != 0);
  return ok(q.dx, M, K) && ok(q.dw, N, K) && launchable(q.du.cols * q.du.strips, 256);
}

hipError_t launch_projection_fwd(const ProjArgs& a, hipStream_t st) { return a.dtype == 1 ? fwd<__bf16>(a, st) : fwd<float>(a, st); }
hipError_t launch_projection_bwd(const ProjArgs& a, const ProjGrads& g, hipStream_t st) {
  return a.dtype == 1 ? bwd<__bf16>(a, g, st) : bwd<float>(a, g, st);
}

}  // namespace ll
