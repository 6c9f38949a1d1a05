// Linear attention with a fixed decay g_h for each head, over a state of d_k x d_v a head:
//   S_t = g S_(t-1) + k_t v_t^T,   o_t = scale S_t^T q_t.
// Chunks of C tokens from the state S before them, with i, j the tokens of a chunk:
//   o_i = scale (g^(i+1) S^T q_i + sum_{j <= i} g^(i-j) (q_i . k_j) v_j),   S' = g^C S + sum_j g^(C-1-j) k_j v_j^T.
// The gradients are the same sums of other operands: with D_t = dL/dS_t,
//   dq_t = scale S_t do_t                                  queries do, keys v, values k, over the transposed states
//   dk_t = D_t v_t,  dv_t = D_t^T k_t                      in reversed time: queries v, keys do, values q, and k, q, do
//   D_t = g D_(t+1) + scale q_t do_t^T                     the gradient of the final state enters without a decay
// so one kernel, k_attend, serves all.  The length is split into segments where batch and heads are few: their own sums
// come first (k_attend with STATE), are joined in order (k_join), and every segment starts from its state.
//
// Everything is computed transposed: P^T = K Q^T, O^T = S^T Q^T + V^T P^T, S += K^T V.  A result of one matrix instruction
// then is an operand of the next as the lanes hold it (P^T through LDS, where other waves read it; S in place), since a
// contraction only needs both operands to agree on which k a slot stands for.
//
// bf16: 65536 tokens of 16 heads of 128 x 128 386 us a call, 4.5 TB/s over the 1.75 GB that are moved; 4 x 8192 tokens of 32
// heads of 128 x 64 with states in and out 274 us, 4.4 TB/s; a copy reaches 5.0.  (In a kernel trace, which runs one launch
// at a time and slower: sums of 32 segments 137, their join 16, results 268; and 79, 12, 206.)  Bound by memory there, by a
// chunk's way through the waves (7 to 9 us with two workgroups on a compute unit) where segments are short.
#include "ll_layer.hpp"
#include "ll_layer_device.hpp"

namespace ll {

namespace {

// Fragments of 16 bytes: lane (g, i) holds KF / 4 contracted values from KF / 4 * g on, of row i.
template <typename T>
struct Op;
template <>
struct Op<__bf16> {
  static constexpr int KF = 32, C = 64;
  typedef bf16x8 Frag;
  __device__ static inline f32x4 mma(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Op<float> {
  static constexpr int KF = 16, C = 32;
  typedef f32x4 Frag;
  __device__ static inline f32x4 mma(Frag a, Frag b, f32x4 c) {
#pragma unroll
    for (int r = 0; r < 4; ++r) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[r], b[r], c, 0, 0, 0);
    return c;
  }
};

// Row i of result t that becomes an operand: results (two of bf16, one of fp32) fill a fragment's slots, so that those of
// lane group g are KF / 4 adjacent rows.
template <typename T>
__device__ inline int row_of(int t, int i) {
  return sizeof(T) == 2 ? 32 * (t >> 1) + 8 * (i >> 2) + 4 * (t & 1) + (i & 3) : 16 * t + i;
}

// An LDS tile of rows of W elements: chunk c of 16 bytes at c ^ key(row).  A read serves 256 bytes at a time, 16 lanes of
// 16 bytes or 32 of 8, which the keys spread over all banks: one chunk of 16 rows (0 - 15, or 0 - 3, 8 - 11, 16 - 19 and
// 24 - 27), two chunks of 8 rows (0 - 3 and 8 - 11), and in fp32 16 columns of four rows 4 apart.  The values of paired
// columns (NV = 2) are read in halves of four chunks of 8 rows, which the banks serve at half their rate.  All in all 39 % of
// the cycles of LDS reads and copies in k_attend's results of 128 x 128 are conflicts (LDS is active a third of the time).
template <typename T, int W>
struct Tile {
  static constexpr int E = 16 / sizeof(T), CH = W / E;
  __device__ static inline constexpr int key(int row) {
    if (sizeof(T) == 4) return row & 15;
    const int b = ((row >> 2) ^ (row >> 4)) & 1, b1 = (row >> 1) & 1, b3 = (row >> 3) & 1;
    return CH == 8 ? b | b1 << 1 | b3 << 2 : b | (row & 1) << 1 | b1 << 2 | b3 << 3;
  }
  __device__ static inline int at(int row, int c) { return (row * CH + (c ^ key(row))) * E; }
  // Addresses of fragments in LDS: a lane's of the first, which the others' differ from by exclusive ors and sums of
  // constants.  (Their keys differ by the constant rows' own, as no sum of a row carries, and a tile begins at a multiple
  // of 1024.)
  __device__ static inline unsigned address(const T* s) { return unsigned(reinterpret_cast<uintptr_t>(s)); }
  template <typename V>
  __device__ static inline V read(unsigned at, int offset) {
    return *reinterpret_cast<const __attribute__((address_space(3))) V*>((__attribute__((address_space(3))) const char*)(uintptr_t(at)) + offset);
  }
  // Chunk 4 ks + g of the lane's row and of those `row` further on.
  __device__ static inline unsigned along0(const T* s, int row, int lane) { return address(s) + at(row, lane >> 4) * unsigned(sizeof(T)); }
  __device__ static inline typename Op<T>::Frag along(unsigned at0, int ks, int row) {
    return read<typename Op<T>::Frag>(at0 ^ (64 * ks) ^ (16 * key(row)), row * CH * 16);
  }
  // The same of a bf16 row with the slots of two stacked results: elements 4 g .. and 16 + 4 g .. of a step's 32.
  __device__ static inline unsigned stacked0(const T* s, int row, int lane) {
    const int g = lane >> 4;
    return sizeof(T) == 2 ? address(s) + at(row, g >> 1) * 2 + 8 * (g & 1) : along0(s, row, lane);
  }
  __device__ static inline typename Op<T>::Frag stacked(unsigned at0, int ks, int row) {
    if constexpr (sizeof(T) == 2) {
      const unsigned lo = at0 ^ (64 * ks) ^ (16 * key(row));
      return __builtin_shufflevector(read<bf16x4>(lo, row * CH * 16), read<bf16x4>(lo ^ 32, row * CH * 16), 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      return along(at0, ks, row);
    }
  }
  // Down the rows KF u .., 16 columns from 16 t on.
  __device__ static inline unsigned down0(const T* s, int lane) {
    const int g = lane >> 4, i = lane & 15;
    if (sizeof(T) == 2) return address(s) + at(8 * g + (i >> 2), (i & 3) >> 1) * 2 + 8 * (i & 1);
    return address(s) + (at(4 * g, i >> 2) + (i & 3)) * 4;
  }
  __device__ static inline typename Op<T>::Frag down(unsigned at0, int t, int u) {
    if constexpr (sizeof(T) == 2) {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) char* Lds;
      const unsigned lo = at0 ^ (32 * t), hi = lo ^ (16 * key(4));
      const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)((Lds)(uintptr_t(lo)) + 32 * u * CH * 16));
      const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)((Lds)(uintptr_t(hi)) + (32 * u + 4) * CH * 16));
      return __builtin_shufflevector(__builtin_bit_cast(bf16x4, x), __builtin_bit_cast(bf16x4, y), 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      f32x4 f;
#pragma unroll
      for (int r = 0; r < 4; ++r) f[r] = read<float>(at0 ^ (64 * t) ^ (16 * key(r)), (16 * u + r) * CH * 16);
      return f;
    }
  }
  // Down the rows in any order of columns: `col` is the first of lane i & 3's four for bf16, the lane's own for fp32.
  __device__ static inline typename Op<T>::Frag down_at(const T* s, int u, int col, int lane) {
    const int g = lane >> 4, i = lane & 15;
    if constexpr (sizeof(T) == 2) {
      const int row = 32 * u + 8 * g + (i >> 2);
      const bf16x4 lo = lds_read_tr(s + at(row, col >> 3) + (col & 7));
      const bf16x4 hi = lds_read_tr(s + at(row + 4, col >> 3) + (col & 7));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      f32x4 f;
#pragma unroll
      for (int r = 0; r < 4; ++r) f[r] = s[at(16 * u + 4 * g + r, col >> 2) + (col & 3)];
      return f;
    }
  }
};

// A tensor [B, T, heads, width] whose heads are adjacent: `group` heads of the call share one of it.
struct Heads {
  const void* p;
  int64_t sb, st;
  int width, group;
  bool vec;  // rows of whole, aligned 16-byte vectors
};

struct DecayDev {
  Heads a, b, c;         // queries and keys of d1 elements, values of d2
  void* out;             // [B, T, H, d2] in the storage type, or fp32 (wide)
  const float* first;    // states at the segments' starts, [B, H, S, rows, cols]; may be null: zeros
  float* last;           // STATE: as first; else the final state [B, H, rows, cols]; may be null
  const float* log_decay;
  const int32_t* lengths;
  int64_t T, L;          // L: tokens of a segment
  int H, S, blocks;      // blocks: workgroups over d2
  int64_t groups;        // workgroups
  float in_scale, out_scale;  // of keys times values, of results
  bool transposed;       // states are [d2, d1]
  bool reversed, wide, vec_out;
};

__device__ inline int64_t live_tokens(const int32_t* lengths, int64_t b, int64_t T) {
  if (!lengths) return T;
  const int64_t n = lengths[b];
  return n < 0 ? 0 : (n < T ? n : T);
}
// A value that all lanes share, for the compiler to know.
__device__ inline int64_t uniform64(int64_t v) {
  const unsigned lo = __builtin_amdgcn_readfirstlane(int(v)), hi = __builtin_amdgcn_readfirstlane(int(v >> 32));
  return int64_t(uint64_t(hi) << 32 | lo);
}
// log2 of a head's decay, finite so that its zeroth power is 1.
__device__ inline float log2_decay(const float* log_decay, int h) {
  const float v = log_decay[h] * kLog2e;
  return v < -1e30f ? -1e30f : v;
}

__device__ const uint4 kZeros = {0, 0, 0, 0};  // rows before the first token, elements beyond the width

// g^n for the state's way over n tokens, and what fp32 leaves of it: its error would be taken to the power of the chunks (a
// state after 14758 tokens: off by 1.1e-6 with v_exp_f32's power, 6e-7 so).  `hi` is the float towards zero and `lo` not
// zero where g^n is not: an infinite state stays one (0 or a negative rest times it would make NaN of it).
struct Carry {
  float hi, lo;
  __device__ inline Carry(const float* log_decay, int h, double n) {
    const double w = exp(double(log_decay[h]) * n);
    hi = float(w);
    if (hi > w) hi = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, hi) - 1);
    const double rest = w - hi, least = w * 0x1p-60;
    lo = float(rest > least ? rest : least);
  }
  __device__ inline float times_plus(float v, float u) const { return fmaf(hi, v, fmaf(lo, v, u)); }  // g^n v + u
};

// Copies chunks of C rows of up to W elements to LDS, 16 bytes a thread at a time: straight there (VEC: rows of whole,
// aligned vectors), or through registers, where a row's last, short vector is read moved back over the one before and
// shifted (101 and 143 elements, 4 x 24115 tokens of 8 heads: element by element 2027 us).  A chunk's address is the same for
// all lanes, a lane's offset from it (fewer than 64 rows of less than 2^24 elements) the same for all chunks.
template <typename T, int W, bool VEC>
struct Stage {
  typedef Tile<T, W> Tl;
  typedef typename VecN<T, Tl::E>::type Vec;
  typedef typename VecN<T, Tl::E>::loose Loose;
  static constexpr int E = Tl::E, CH = Tl::CH, C = Op<T>::C, ITS = C * CH / 256, ROWS = 256 / CH;
  const char* base;  // of the next chunk: its row with the lowest address
  int64_t turn;      // bytes between chunks
  unsigned off[ITS];
  int left;          // elements of a row
  Vec held[VEC ? 1 : ITS];
  // `p`: element 0 of the first chunk's row 0, tokens `stride` elements apart, later ones lower where `reversed`
  __device__ inline void start(const T* p, int64_t stride, bool reversed, int left_) {
    left = left_;
    base = reinterpret_cast<const char*>(p - (reversed ? (C - 1) * stride : 0));
    turn = (reversed ? -C : C) * stride * int64_t(sizeof(T));
#pragma unroll
    for (int it = 0; it < ITS; ++it) {
      const int row = threadIdx.x / CH + it * ROWS, c = (threadIdx.x % CH) ^ Tl::key(row);
      off[it] = (unsigned(reversed ? C - 1 - row : row) * unsigned(stride) + c * E) * unsigned(sizeof(T));
    }
  }
  // Begins the copy of the next chunk, of which rows before `first` are zeros: to `s` (VEC), or to registers.
  __device__ inline void load(T* s, int first) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    auto copy = [&](auto edge) {
#pragma unroll
      for (int it = 0; it < ITS; ++it) {
        const int row = threadIdx.x / CH + it * ROWS, c = (threadIdx.x % CH) ^ Tl::key(row);
        const int k = row < first ? 0 : left - c * E;
        if constexpr (VEC) {
          const unsigned to = lds_address(s + (it * 256 + wave * 64) * E);
          if (edge.value) copy16_to_lds(to, k > 0 ? static_cast<const void*>(base + off[it]) : &kZeros);
          else copy16_to_lds(to, base, off[it]);
        } else if (left >= E) {
          const int back = k < E ? E - k : 0;
          const void* src = k > 0 ? static_cast<const void*>(base + off[it] - back * int(sizeof(T))) : &kZeros;
          held[it] = *static_cast<const Loose*>(src);
        } else {
          held[it] = load_n<T, E>(reinterpret_cast<const T*>(base + off[it]), k <= 0 ? 0 : (k < E ? k : E), false);
        }
      }
    };
    if (!VEC || first > 0 || left < W) copy(std::true_type{});
    else copy(std::false_type{});
    base += turn;
  }
  // Through registers: ends the copy.
  __device__ inline void store(T* s) {
    if constexpr (!VEC) {
#pragma unroll
      for (int it = 0; it < ITS; ++it) {
        const int row = threadIdx.x / CH + it * ROWS, c = (threadIdx.x % CH) ^ Tl::key(row), k = left - c * E;
        if (left >= E && k > 0 && k < E) {
          const int shift = (E - k) * int(sizeof(T)) * 8;
          held[it] = __builtin_bit_cast(Vec, __builtin_bit_cast(unsigned __int128, held[it]) >> shift);
        }
        reinterpret_cast<Vec*>(s)[it * 256 + threadIdx.x] = held[it];
      }
    }
  }
};

template <typename T>
__device__ inline typename Op<T>::Frag pack(const f32x4* v);
template <>
__device__ inline bf16x8 pack<__bf16>(const f32x4* v) {
  bf16x8 f;
#pragma unroll
  for (int r = 0; r < 4; ++r) f[r] = static_cast<__bf16>(v[0][r]), f[4 + r] = static_cast<__bf16>(v[1][r]);
  return f;
}
template <>
__device__ inline f32x4 pack<float>(const f32x4* v) {
  return v[0];
}

// One of two parts of values that are not -0.  The upper one is formed again for the rest: kept, those of a state spill.
__device__ inline f32x4 part_of(f32x4 v, int part) {
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    if (part) asm volatile("" : "+v"(v[r]));
    const float hi = upper_part(v[r]);
    v[r] = part ? v[r] - hi : hi;
  }
  return v;
}

// v w of a fragment's slots as N bf16 parts, upper ones but for the third: three are off by 2^-24 of a product, two by 2^-14.
// fp32: the product.
template <int N>
__device__ inline void weighted(bf16x8 v, const float* w, bf16x8* part) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int x = 0; x < 8; x += 2) {
    float a = product(to_f32(__bf16(v[x])), w[x]), b = product(to_f32(__bf16(v[x + 1])), w[x + 1]);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      bf16x2 y = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
      if (k < 2) {
        const float ha = upper_part(a), hb = upper_part(b);
        y = __builtin_bit_cast(bf16x2, __builtin_amdgcn_perm(__builtin_bit_cast(unsigned, hb), __builtin_bit_cast(unsigned, ha), 0x07060302u));
        a -= ha, b -= hb;
      }
      part[k][x] = y[0], part[k][x + 1] = y[1];
    }
  }
}
template <int N>
__device__ inline void weighted(f32x4 v, const float* w, f32x4* part) {
#pragma unroll
  for (int x = 0; x < 4; ++x) part[0][x] = v[x] * w[x];
}

// Whether the next chunk's keys (STATE: and values) have LDS of their own to arrive in while this one's are in use.
constexpr bool keys_ahead(int dk) { return dk <= 128; }

// One segment of one head, 64 NV values a workgroup: a wave holds the state's rows of its 16 NV columns.  d1 <= DK.
// Chunks end with the segment: the first may begin with rows of zeros, and powers of the decay are the same in all others.
// FEW: bf16 sequences of one chunk take scores and states in two parts: with few of them their roundings do not average out
// (28 sequences of one token: results off by 0.0032, 0.0017 so; of more than 64 tokens 0.0025 at most).  512 sequences of 64
// tokens, 16 heads of 128 x 128: 597 us, 626 so.
template <typename T, int DK, int NV, bool STATE, bool VEC, bool FEW, typename Keys, typename Values, typename Queries, typename Scores>
__device__ __attribute__((always_inline)) inline void attend_segment(const DecayDev& p, int64_t b, int h, int seg, int blk, int64_t live,
                                                                     Keys& sk, Values& sv, Queries& sq, Scores& sp, float* sw) {
  constexpr int KF = Op<T>::KF, C = Op<T>::C, R = KF / 16, QT = C / 16, US = C / KF, KS = DK / KF, DT = DK / 16;
  constexpr int NW = 4, DV = 16 * NW * NV, NU = QT * US / NW;  // NU: fragments of P^T that a wave forms
  constexpr bool AHEAD = keys_ahead(DK);
  constexpr int PARTS = FEW ? 2 : 1;
  typedef typename Op<T>::Frag Frag;
  typedef Tile<T, DK> TlK;
  typedef Tile<T, DV> TlV;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, i = lane & 15;
  const int d1 = p.a.width, d2 = p.c.width, col0 = blk * DV;
  const int64_t t0 = seg * p.L;
  int64_t n = live - t0 < p.L ? live - t0 : p.L;  // tokens of this segment
  n = n < 0 ? 0 : n;
  const int64_t chunks = (n + C - 1) / C;
  int first = int(chunks * C - n);  // rows of zeros
  // the segment whose state a caller may get
  const bool ends = STATE || seg == (live > 0 ? (live - 1) / p.L : 0);
  const float lg = log2_decay(p.log_decay, h);
  const int rho = p.reversed ? 1 : 0;

  // tokens by their order in time: that of the first chunk's row 0, and the step between two
  const int64_t tok = p.reversed ? live - 1 - (t0 - first) : t0 - first, dir = p.reversed ? -1 : 1;
  Stage<T, DK, VEC> lk, lq;
  Stage<T, DV, VEC> lv;
  lk.start(static_cast<const T*>(p.b.p) + b * p.b.sb + tok * p.b.st + (h / p.b.group) * d1, p.b.st, p.reversed, d1);
  lv.start(static_cast<const T*>(p.c.p) + b * p.c.sb + tok * p.c.st + (h / p.c.group) * d2 + col0, p.c.st, p.reversed, d2 - col0);
  if (!STATE) lq.start(static_cast<const T*>(p.a.p) + b * p.a.sb + tok * p.a.st + (h / p.a.group) * d1, p.a.st, p.reversed, d1);
  if (n > 0) {
    lk.load(sk[0], first), lk.store(sk[0]);
    if (!STATE) lq.load(sq, first), lq.store(sq);
    lv.load(sv[0], first), lv.store(sv[0]);
  }
  const Carry chunk(p.log_decay, h, double(C));
  Carry begin = chunk;
  if (first > 0) begin = Carry(p.log_decay, h, double(C - first));
  float over = 0.0f;
  if (threadIdx.x < C) sw[threadIdx.x] = p.in_scale * fast_exp2(lg * float(C - 1 - int(threadIdx.x) + rho));

  // columns: those of tile v that lane i holds; two tiles interleaved in fours, so that a lane's results are adjacent
  const int wcol = 16 * NV * wave;
  auto vcol = [&](int v, int x) { return wcol + (NV == 2 ? 8 * (x >> 2) + 4 * v + (x & 3) : x); };
  auto element = [&](int row, int col) { return p.transposed ? col * d1 + row : row * d2 + col; };
  f32x4 S[DT][NV] = {};
  if (!STATE && p.first && (n > 0 || ends)) {
    const float* f = p.first + ((b * p.H + h) * p.S + seg) * int64_t(d1) * d2;
#pragma unroll
    for (int t = 0; t < DT; ++t) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 16 * t + 4 * g + r, col = col0 + vcol(v, i);
          if (row < d1 && col < d2) S[t][v][r] = f[element(row, col)];
        }
      if (t % 2) __builtin_amdgcn_sched_barrier(0);  // few addresses at a time: registers
    }
  }
  // g^(i-j) of the wave's scores, nothing where j > i, with both scales
  float pw[NU][R][4];
#pragma unroll
  for (int x = 0; x < NU; ++x)
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int item = wave + x * NW, gap = 16 * (item % QT) + i - row_of<T>(R * (item / QT) + r, 4 * g + e);
        pw[x][r][e] = gap >= 0 ? p.in_scale * p.out_scale * fast_exp2(lg * float(gap)) : 0.0f;
      }
  const int ocol = col0 + wcol + 4 * NV * g, ocount = d2 - ocol < 4 * NV ? d2 - ocol : 4 * NV;
  int64_t orow = ((b * p.T + tok + dir * i) * p.H + h) * d2 + ocol;
  const int64_t ostep = dir * p.H * d2;

  for (int64_t ch = 0; ch < chunks; ++ch) {
    const T* k_now = sk[AHEAD ? ch & 1 : 0];
    const T* v_now = sv[AHEAD && STATE ? ch & 1 : 0];
    const bool more = ch + 1 < chunks;
    // opaque at every use: the addresses that depend on it would all be formed, and spilled, before the loop
    auto opaque = [&] {
      int ln = lane;
      asm volatile("" : "+v"(ln));
      return ln;
    };
    auto x4 = [](int ln) { return sizeof(T) == 2 ? 4 * (ln & 3) : ln & 15; };  // a lane's column of those read down
    if (VEC) copies_done();
    __syncthreads();
    T* const k_next = sk[AHEAD ? ~ch & 1 : 0];
    T* const v_next = sv[AHEAD && STATE ? ~ch & 1 : 0];
    if (more && (AHEAD || !VEC)) {
      lk.load(k_next, 0);
      if (STATE) lv.load(v_next, 0);
    }
    if (more && !STATE && !VEC) lq.load(sq, 0), lv.load(v_next, 0);
    Frag vf[NV][US];
    auto values = [&] {
      const int ln = opaque();
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int u = 0; u < US; ++u) vf[v][u] = TlV::down_at(v_now, u, vcol(v, x4(ln)), ln);
    };
    if (STATE) values();

    if constexpr (!STATE) {
      f32x4 o[QT][NV] = {};
#pragma unroll
      for (int part = 0; part < PARTS; ++part) {
        if (part) __syncthreads();  // the first part's scores are read; queries and keys are there: no chunk comes after
        // P^T of 16 queries and the keys up to them
#pragma unroll
        for (int x = 0; x < NU; ++x) {
          const int qt = (wave + x * NW) % QT, u = (wave + x * NW) / QT;
          if (u * KF > 16 * qt + 15) continue;
          f32x4 pt[R] = {};
          const int ln = opaque();
          const unsigned qa = TlK::along0(sq, 16 * qt + (ln & 15), ln), ka = TlK::along0(k_now, KF * u + row_of<T>(0, ln & 15), ln);
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            const Frag q = TlK::along(qa, ks, 0);
#pragma unroll
            for (int r = 0; r < R; ++r) pt[r] = Op<T>::mma(TlK::along(ka, ks, row_of<T>(r, 0)), q, pt[r]);
          }
#pragma unroll
          for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) pt[r][e] = FEW ? product(pt[r][e], pw[x][r][e]) : pt[r][e] * pw[x][r][e];
          if (FEW) {
#pragma unroll
            for (int r = 0; r < R; ++r) pt[r] = part_of(pt[r], part);
          }
          sp[qt][u][lane] = pack<T>(pt);
        }
        if (part == 0) {
#pragma unroll
          for (int low = 0; low < PARTS; ++low) {
            const int ln = opaque();
            const unsigned qa = TlK::stacked0(sq, ln & 15, ln);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
              Frag s[NV];
#pragma unroll
              for (int v = 0; v < NV; ++v) {
                f32x4 x[R];
#pragma unroll
                for (int r = 0; r < R; ++r) {
                  if (FEW && !low) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) S[R * ks + r][v][e] = positive(S[R * ks + r][v][e]);
                  }
                  x[r] = S[R * ks + r][v];
                  if (FEW) x[r] = part_of(x[r], low);
                }
                s[v] = pack<T>(x);
              }
#pragma unroll
              for (int qt = 0; qt < QT; ++qt) {
                const Frag q = TlK::stacked(qa, ks, 16 * qt);
#pragma unroll
                for (int v = 0; v < NV; ++v) o[qt][v] = Op<T>::mma(s[v], q, o[qt][v]);
              }
            }
          }
          values();
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) {
            const int after = 16 * qt + i + 1 - rho - first;
            const float w = p.out_scale * fast_exp2(lg * float(after > 0 ? after : 0));
#pragma unroll
            for (int v = 0; v < NV; ++v) o[qt][v] *= w;
          }
        }
        __syncthreads();
        if (PARTS == 1 && more) {
          if (VEC) lq.load(sq, 0), lv.load(v_next, 0);
          lq.store(sq), lv.store(v_next);
        }
#pragma unroll
        for (int qt = 0; qt < QT; ++qt)
#pragma unroll
          for (int u = 0; u < US; ++u) {
            if (u * KF > 16 * qt + 15) continue;
            const Frag pf = sp[qt][u][lane];
#pragma unroll
            for (int v = 0; v < NV; ++v) o[qt][v] = Op<T>::mma(vf[v][u], pf, o[qt][v]);
          }
      }
      if (ocount > 0) {
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          float f[4 * NV];
#pragma unroll
          for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int r = 0; r < 4; ++r) f[4 * v + r] = o[qt][v][r];
          const int64_t e = orow + 16 * qt * ostep;
          const bool in = 16 * qt + i >= first;
          if (!in) continue;
          if (p.wide) store_n<float, 4 * NV>(static_cast<float*>(p.out) + e, f, VEC ? 4 * NV : ocount, VEC);
          else store_n<T, 4 * NV>(static_cast<T*>(p.out) + e, f, VEC ? 4 * NV : ocount, VEC);
        }
      }
      orow += C * ostep;
    }

    // the state after the chunk; values times powers of the decay in bf16 parts, three where fp32's bits are wanted and two
    // where only rounded results come of it (the state itself is rounded to 8 bits there, an operand of the next chunk)
    // what the factors leave out of exact ones is carried over, so that their product over the chunks is off by a rounding
    over += ch ? chunk.lo : begin.lo;
    const float carry = (ch ? chunk.hi : begin.hi) + over;
    over -= carry - (ch ? chunk.hi : begin.hi);
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int v = 0; v < NV; ++v) S[t][v] *= carry;
#pragma unroll
    for (int u = 0; u < US; ++u) {
      float w[KF / 4];
#pragma unroll
      for (int x = 0; x < KF / 4; x += 4) {
        const f32x4 y = *reinterpret_cast<const f32x4*>(sw + KF * u + KF / 4 * g + x);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[x + e] = y[e];
      }
      // adds the parts from `from` on to the state
      auto add = [&](auto from, auto to) {
        constexpr int P0 = decltype(from)::value, P1 = decltype(to)::value;
        if (P0 && DK <= 64 && NV == 2) {  // formed again: kept from the parts before, they take the registers of a third workgroup
#pragma unroll
          for (int x = 0; x < KF / 4; ++x) asm volatile("" : "+v"(w[x]));
        }
        Frag part[NV][P1];
#pragma unroll
        for (int v = 0; v < NV; ++v) weighted<P1>(vf[v][u], w, part[v]);
        const unsigned ka = TlK::down0(k_now, opaque());
        // two tiles at a time, so that a product does not wait for the one before, and the next two are on their way
        Frag k[2][2];
#pragma unroll
        for (int x = 0; x < 2; ++x) k[0][x] = TlK::down(ka, x, u);
#pragma unroll
        for (int t = 0; t < DT; t += 2) {
          if (t + 2 < DT) {
#pragma unroll
            for (int x = 0; x < 2; ++x) k[(t / 2 + 1) & 1][x] = TlK::down(ka, t + 2 + x, u);
          }
#pragma unroll
          for (int y = P0; y < P1; ++y)
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
              for (int v = 0; v < NV; ++v) S[t + x][v] = Op<T>::mma(k[t / 2 & 1][x], part[v][y], S[t + x][v]);
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      typedef std::integral_constant<int, 0> None;
      if constexpr (sizeof(T) == 4) {
        add(None{}, std::integral_constant<int, 1>{});
      } else if constexpr (STATE) {
        add(None{}, std::integral_constant<int, 3>{});
      } else {
        add(None{}, std::integral_constant<int, 2>{});
        if (ends) add(std::integral_constant<int, 2>{}, std::integral_constant<int, 3>{});
      }
    }
    if (!AHEAD) __syncthreads();
    if (more) {
      if (VEC && !AHEAD) {
        lk.load(k_next, 0);
        if (STATE) lv.load(v_next, 0);
      }
      lk.store(k_next);
      if (STATE) lv.store(v_next);
    }
    first = 0;
  }

  // STATE: this segment's own sums, where the next one starts.  Else the final state, of the segment that ends there.
  float* to = nullptr;
  if (STATE) to = p.last + ((b * p.H + h) * p.S + seg + 1) * int64_t(d1) * d2;
  else if (p.last && ends) to = p.last + (b * p.H + h) * int64_t(d1) * d2;
  if (to) {
#pragma unroll
    for (int t = 0; t < DT; ++t) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 16 * t + 4 * g + r, col = col0 + vcol(v, i);
          if (row < d1 && col < d2) to[element(row, col)] = S[t][v][r];
        }
      if (t % 2) __builtin_amdgcn_sched_barrier(0);
    }
  }
  // rows after the sequence's end
  if (!STATE) {
    const int64_t end = t0 + p.L < p.T ? t0 + p.L : p.T, from = live > t0 ? live : t0;
    const int cols = d2 - col0 < DV ? d2 - col0 : DV;
    for (int64_t t = from + wave; t < end; t += NW) {
      const int64_t e = ((b * p.T + t) * p.H + h) * d2 + col0;
      for (int c = lane; c < cols; c += 64) {
        if (p.wide) static_cast<float*>(p.out)[e + c] = 0.0f;
        else static_cast<T*>(p.out)[e + c] = from_f32<T>(0.0f);
      }
    }
  }
}

// SHORT: there may be sequences of one chunk, which take the FEW way whatever stands beside them in the batch.  (A launch of
// its own for them: 32 sequences of up to 512 tokens, 16 heads of 128 x 128, 74 -> 95 us, 75 so.  Without the instances that
// lack it: 320 tokens, 8 heads of 64 x 64, 17.0 -> 17.8.)
template <typename T, int DK, int NV, bool STATE, bool VEC, bool SHORT = false>
__global__ __launch_bounds__(256, 2) void k_attend(DecayDev p) {
  constexpr int KF = Op<T>::KF, C = Op<T>::C, DV = 64 * NV;
  constexpr bool AHEAD = keys_ahead(DK);
  __shared__ __attribute__((aligned(1024))) T sk[AHEAD ? 2 : 1][C * DK];
  __shared__ __attribute__((aligned(1024))) T sv[AHEAD && STATE ? 2 : 1][C * DV];
  __shared__ __attribute__((aligned(1024))) T sq[STATE ? 8 : C * DK];
  __shared__ typename Op<T>::Frag sp[STATE ? 1 : C / 16][C / KF][64];
  __shared__ __attribute__((aligned(16))) float sw[C];  // what a token's product counts in the state after the chunk
  // the sums of segments go through the input in one order, the results in the other: what was read last is still cached
  unsigned id = unsigned(xcd_remap(blockIdx.x, p.groups));
  if (!STATE && p.S > 1) id = unsigned(p.groups) - 1 - id;
  const unsigned segs = STATE ? p.S - 1 : p.S;
  const int blk = int(id % unsigned(p.blocks));
  id /= unsigned(p.blocks);
  const int seg = int(id % segs);
  id /= segs;
  const int h = int(id % unsigned(p.H));
  const int64_t b = id / unsigned(p.H);
  const int64_t live = uniform64(live_tokens(p.lengths, b, p.T));
  if constexpr (SHORT) {
    if (live <= C) return attend_segment<T, DK, NV, STATE, VEC, true>(p, b, h, seg, blk, live, sk, sv, sq, sp, sw);
  }
  attend_segment<T, DK, NV, STATE, VEC, false>(p, b, h, seg, blk, live, sk, sv, sq, sp, sw);
}

// The states at the segments' starts, in place of the segments' own sums: h_0 = first, h_(s+1) = g^(n_s) h_s + u_s.
__global__ __launch_bounds__(256) void k_join(float* h, const float* first, const float* log_decay, const int32_t* lengths,
                                              int64_t T, int64_t L, int H, int S, int64_t size, int64_t total) {
  const int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (id >= total) return;
  const int64_t bh = id / size, e = id % size;
  const int64_t live = live_tokens(lengths, bh / H, T);
  const int used = live > 0 ? int((live - 1) / L) + 1 : 1;  // segments that hold tokens
  float* p = h + bh * S * size + e;
  float v = first ? first[id] : 0.0f;
  p[0] = v;
  const Carry w(log_decay, int(bh % H), double(L));  // a segment with one after it is whole
  constexpr int U = 8;  // loads ahead of the stores
  for (int s = 1; s < used; s += U) {
    float u[U];
#pragma unroll
    for (int k = 0; k < U; ++k) u[k] = s + k < used ? p[(s + k) * size] : 0.0f;
#pragma unroll
    for (int k = 0; k < U; ++k) {
      v = w.times_plus(v, u[k]);
      if (s + k < used) p[(s + k) * size] = v;
    }
  }
}

// Bound by memory: 64 sequences of 16 heads of 128 x 128 32 us, 4.2 TB/s of states in and out.
// One token of 256 / LV rows at a time: o = scale (g S + k v^T)^T q, the state passed through.
// g with what its rounding leaves, as the prompts' kernels have it: g in fp32 alone moves a state by up to 2^-25 a token, all
// to one side (4096 tokens of 1 - g = 2^-12.5: by 7e-5).
struct StepDev {
  Heads q, k, v;
  const float* state;
  float* next;
  void* out;
  const float* log_decay;
  int H, dk, dv;
  float scale;
  bool vec;
};
template <typename T, int LV>
__global__ __launch_bounds__(256) void k_decay_step(StepDev p) {
  constexpr int RS = 256 / LV;
  __shared__ float s[RS][LV][5];
  const int c = threadIdx.x % LV, r0 = threadIdx.x / LV;
  const int64_t bh = blockIdx.x, b = bh / p.H;
  const int h = int(bh % p.H);
  const int col = 4 * c, count = p.dv - col < 4 ? (p.dv > col ? p.dv - col : 0) : 4;
  const T* q = static_cast<const T*>(p.q.p) + b * p.q.sb + (h / p.q.group) * p.dk;
  const T* k = static_cast<const T*>(p.k.p) + b * p.k.sb + (h / p.k.group) * p.dk;
  const T* v = static_cast<const T*>(p.v.p) + b * p.v.sb + h * p.dv + col;
  const Carry decay(p.log_decay, h, 1.0);
  const auto vr = load_n<T, 4>(v, count, false);
  float vf[4], o[4] = {};
#pragma unroll
  for (int i = 0; i < 4; ++i) vf[i] = to_f32(T(vr[i]));
  const int64_t base = bh * p.dk * p.dv + col;
  if (count > 0) {
    // rows are loaded ahead of the stores, which could be the same memory
    constexpr int U = 8;
    for (int r = r0; r < p.dk; r += U * RS) {
      typename VecN<float, 4>::type st[U];
      float kr[U], qr[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int at = r + u * RS, n = at < p.dk ? count : 0;
        st[u] = load_n<float, 4>(p.state + base + int64_t(at) * p.dv, n, p.vec);
        kr[u] = n ? to_f32(k[at]) : 0.0f, qr[u] = n ? to_f32(q[at]) : 0.0f;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = decay.times_plus(st[u][i], kr[u] * vf[i]);
          o[i] = fmaf(qr[u], x[i], o[i]);
        }
        store_n<float, 4>(p.next + base + int64_t(r + u * RS) * p.dv, x, r + u * RS < p.dk ? count : 0, p.vec);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) s[r0][c][i] = o[i];
  __syncthreads();
  for (int e = threadIdx.x; e < p.dv; e += 256) {
    float sum = 0.0f;
#pragma unroll
    for (int r = 0; r < RS; ++r) sum += s[r][e / 4][e % 4];
    static_cast<T*>(p.out)[bh * p.dv + e] = from_f32<T>(p.scale * sum);
  }
}

// Gradients of shared heads: the sum of each group's, in their order.
template <typename T>
__global__ __launch_bounds__(256) void k_group_sum(const float* x, void* out, int group, int width, int64_t total) {
  const int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (id >= total) return;
  const float* q = x + id / width * group * width + id % width;
  float v = 0.0f;
#pragma unroll 4
  for (int i = 0; i < group; ++i) v += q[int64_t(i) * width];
  static_cast<T*>(out)[id] = from_f32<T>(v);
}

// ------------------------------------------------------------------------------------ plans

int64_t up256(int64_t n) { return (n + 255) / 256 * 256; }

// Tiles of 16 values that a wave holds: two where it has registers for them.
int value_tiles(int64_t d1, int64_t d2) { return d1 <= 128 && d2 > 64 ? 2 : 1; }

struct Split {
  int64_t L, S;
};
// Segments of whole chunks: as many as the card holds workgroups at once (three to a compute unit of keys up to 64
// elements, two up to 128, else one; one more segment begins a second round: 2 x 4096 tokens, 24 heads of 128 x 128, 10
// segments 90 us, 12 109), of 128 tokens at least, and none below 512 tokens, where the two launches more take longer.  One
// segment of 4 x 8192 tokens, 32 heads of 64 x 64 takes 301 us, two 222, six 181.
Split split_of(int64_t B, int64_t T, int64_t H, int64_t dk, int64_t dv) {
  const int64_t held = dk <= 64 ? 768 : dk <= 128 ? 512 : 256;
  int64_t S = held / (B * H * ceil_div(dv, 64 * value_tiles(dk, dv)));
  S = S < T / 128 ? S : T / 128;
  if (S < 1 || T < 512) S = 1;
  Split q;
  q.L = ceil_div(ceil_div(T, S), 64) * 64;
  q.S = ceil_div(T, q.L);
  return q;
}

Heads heads_of(const Rows& r, int64_t heads, int64_t H, int64_t width, int esize) {
  const int n = 16 / esize;
  return {r.p, r.sb, r.st, int(width), int(H / heads), rows_aligned(r, esize, n) && width % n == 0};
}

template <typename T, int DK, int NV>
hipError_t launch_attend(const DecayDev& p, bool state, hipStream_t st) {
  const dim3 grid(uint32_t(p.groups)), block(256);
  const bool vec = p.b.vec && p.c.vec && (state || (p.a.vec && p.vec_out));
  if constexpr (sizeof(T) == 2) {
    if (!state && (p.T <= Op<T>::C || p.lengths)) {
      vec ? k_attend<T, DK, NV, false, true, true><<<grid, block, 0, st>>>(p) : k_attend<T, DK, NV, false, false, true><<<grid, block, 0, st>>>(p);
      return hipGetLastError();
    }
  }
  if (state) vec ? k_attend<T, DK, NV, true, true><<<grid, block, 0, st>>>(p) : k_attend<T, DK, NV, true, false><<<grid, block, 0, st>>>(p);
  else vec ? k_attend<T, DK, NV, false, true><<<grid, block, 0, st>>>(p) : k_attend<T, DK, NV, false, false><<<grid, block, 0, st>>>(p);
  return hipGetLastError();
}

template <typename T>
hipError_t attend(DecayDev p, int64_t B, bool state, hipStream_t st) {
  const int nv = value_tiles(p.a.width, p.c.width);
  p.blocks = int(ceil_div(p.c.width, 64 * nv));
  p.groups = B * p.H * p.blocks * (state ? p.S - 1 : p.S);
  p.vec_out = reinterpret_cast<uintptr_t>(p.out) % 16 == 0 && p.c.width % 8 == 0;  // rows of whole vectors of 4 NV
  if (p.a.width <= 64) return nv == 2 ? launch_attend<T, 64, 2>(p, state, st) : launch_attend<T, 64, 1>(p, state, st);
  if (p.a.width <= 128) return nv == 2 ? launch_attend<T, 128, 2>(p, state, st) : launch_attend<T, 128, 1>(p, state, st);
  return launch_attend<T, 256, 1>(p, state, st);
}

// The states at the segments' starts into `h`: the segments' own sums, then their join.
template <typename T>
hipError_t states(DecayDev p, int64_t B, float* h, const float* first, hipStream_t st) {
  hipError_t e = hipSuccess;
  p.last = h, p.first = nullptr;
  if (p.S > 1) e = attend<T>(p, B, true, st);
  if (e != hipSuccess) return e;
  const int64_t size = int64_t(p.a.width) * p.c.width, total = B * p.H * size;
  k_join<<<dim3(uint32_t(ceil_div(total, 256))), dim3(256), 0, st>>>(h, first, p.log_decay, p.lengths, p.T, p.L, p.H, p.S,
                                                                     size, total);
  return hipGetLastError();
}

DecayDev common(const DecayArgs& a, const Split& s) {
  DecayDev p = {};
  p.log_decay = a.log_decay, p.lengths = a.lengths, p.T = a.T, p.L = s.L, p.H = int(a.H), p.S = int(s.S);
  p.in_scale = 1.0f, p.out_scale = 1.0f;
  return p;
}

template <typename T>
hipError_t fwd(const DecayArgs& a, hipStream_t st) {
  const Split s = split_of(a.B, a.T, a.H, a.dk, a.dv);
  DecayDev p = common(a, s);
  p.a = heads_of(a.q, a.Hqk, a.H, a.dk, sizeof(T)), p.b = heads_of(a.k, a.Hqk, a.H, a.dk, sizeof(T));
  p.c = heads_of(a.v, a.H, a.H, a.dv, sizeof(T));
  p.out = a.o, p.out_scale = a.scale;
  const float* first = a.initial;
  if (a.states || s.S > 1) {
    float* h = a.states ? a.states : static_cast<float*>(a.workspace);
    const hipError_t e = states<T>(p, a.B, h, a.initial, st);
    if (e != hipSuccess) return e;
    first = h;
  }
  p.first = first, p.last = a.final_state;
  return attend<T>(p, a.B, false, st);
}

struct BwdPlan {
  Split s;
  int64_t o_states = 0, o_wide = 0, total = 0;  // reversed states; fp32 gradients of shared heads
};
BwdPlan bwd_plan(int64_t B, int64_t T, int64_t H, int64_t Hqk, int64_t dk, int64_t dv) {
  BwdPlan q;
  q.s = split_of(B, T, H, dk, dv);
  q.o_wide = q.s.S > 1 ? up256(B * H * dk * dv * 4 * q.s.S) : 0;
  q.total = q.o_wide + (Hqk < H ? up256(B * T * H * dk * 4) : 0);
  return q;
}

template <typename T>
hipError_t bwd(const DecayArgs& a, const DecayGrads& g, hipStream_t st) {
  const BwdPlan q = bwd_plan(a.B, a.T, a.H, a.Hqk, a.dk, a.dv);
  char* ws = static_cast<char*>(a.workspace);
  const bool shared = a.Hqk < a.H;
  void* wide = ws + q.o_wide;
  const Rows dout = {g.d_o, a.T * a.H * a.dv, a.H * a.dv};
  const Heads hq = heads_of(a.q, a.Hqk, a.H, a.dk, sizeof(T)), hk = heads_of(a.k, a.Hqk, a.H, a.dk, sizeof(T));
  const Heads hv = heads_of(a.v, a.H, a.H, a.dv, sizeof(T)), hd = heads_of(dout, a.H, a.H, a.dv, sizeof(T));
  const int64_t n = a.B * a.T * a.Hqk * a.dk;
  auto group_sum = [&](void* out) {
    k_group_sum<T><<<dim3(uint32_t(ceil_div(n, 256))), dim3(256), 0, st>>>(static_cast<const float*>(wide), out, int(a.H / a.Hqk),
                                                                           int(a.dk), n);
    return hipGetLastError();
  };
  const DecayDev base = common(a, q.s);
  hipError_t e = hipSuccess;
  {
    DecayDev p = base;
    p.a = hd, p.b = hv, p.c = hk, p.first = a.states, p.transposed = true, p.out_scale = a.scale;
    p.out = shared ? wide : g.dq, p.wide = shared;
    e = attend<T>(p, a.B, false, st);
    if (e == hipSuccess && shared) e = group_sum(g.dq);
  }
  DecayDev p = base;  // dv, with the state D
  p.a = hk, p.b = hq, p.c = hd, p.in_scale = a.scale, p.reversed = true;
  const float* first = g.d_final;
  if (e == hipSuccess && q.s.S > 1) {
    float* h = reinterpret_cast<float*>(ws + q.o_states);
    e = states<T>(p, a.B, h, g.d_final, st);
    first = h;
  }
  if (e == hipSuccess) {
    p.first = first, p.last = nullptr, p.out = g.dv;
    e = attend<T>(p, a.B, false, st);
  }
  if (e == hipSuccess) {  // dk, with its transpose
    p.a = hv, p.b = hd, p.c = hq, p.transposed = true;
    p.last = g.d_initial, p.out = shared ? wide : g.dk, p.wide = shared;
    e = attend<T>(p, a.B, false, st);
    if (e == hipSuccess && shared) e = group_sum(g.dk);
  }
  return e;
}

template <typename T>
hipError_t step(const DecayArgs& a, hipStream_t st) {
  StepDev p = {};
  p.q = heads_of(a.q, a.Hqk, a.H, a.dk, sizeof(T)), p.k = heads_of(a.k, a.Hqk, a.H, a.dk, sizeof(T));
  p.v = heads_of(a.v, a.H, a.H, a.dv, sizeof(T));
  p.state = a.initial, p.next = a.final_state, p.out = a.o, p.log_decay = a.log_decay;
  p.H = int(a.H), p.dk = int(a.dk), p.dv = int(a.dv), p.scale = a.scale;
  p.vec = a.dv % 4 == 0 && reinterpret_cast<uintptr_t>(a.initial) % 16 == 0 && reinterpret_cast<uintptr_t>(a.final_state) % 16 == 0;
  const dim3 grid(uint32_t(a.B * a.H)), block(256);
  if (a.dv <= 64) k_decay_step<T, 16><<<grid, block, 0, st>>>(p);
  else if (a.dv <= 128) k_decay_step<T, 32><<<grid, block, 0, st>>>(p);
  else k_decay_step<T, 64><<<grid, block, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace

int64_t decay_states_bytes(int64_t B, int64_t T, int64_t H, int64_t dk, int64_t dv) {
  return B * H * dk * dv * 4 * split_of(B, T, H, dk, dv).S;
}
int64_t decay_workspace(int64_t B, int64_t T, int64_t H, int64_t Hqk, int64_t dk, int64_t dv, bool backward) {
  const int64_t S = split_of(B, T, H, dk, dv).S, f = S > 1 ? up256(B * H * dk * dv * 4 * S) : 0;
  if (!backward) return f;
  const int64_t b = bwd_plan(B, T, H, Hqk, dk, dv).total;
  return b > f ? b : f;
}
bool decay_launchable(const DecayArgs& a, bool backward) {
  const int64_t S = split_of(a.B, a.T, a.H, a.dk, a.dv).S, heads = a.B * a.H;
  auto attends = [&](int64_t d2) { return launchable(heads * S * ceil_div(d2, 64), 256); };
  if (!attends(a.dv) || !launchable(ceil_div(heads * a.dk * a.dv, 256), 256)) return false;
  if (!backward) return true;
  return attends(a.dk) &&
         (a.Hqk == a.H || launchable(ceil_div(a.B * a.T * a.Hqk * a.dk, 256), 256));
}
bool decay_step_launchable(const DecayArgs& a) { return launchable(a.B * a.H, 256); }

hipError_t launch_decay_fwd(const DecayArgs& a, hipStream_t st) { return a.dtype == 1 ? fwd<__bf16>(a, st) : fwd<float>(a, st); }
hipError_t launch_decay_bwd(const DecayArgs& a, const DecayGrads& g, hipStream_t st) {
  return a.dtype == 1 ? bwd<__bf16>(a, g, st) : bwd<float>(a, g, st);
}
hipError_t launch_decay_step(const DecayArgs& a, hipStream_t st) { return a.dtype == 1 ? step<__bf16>(a, st) : step<float>(a, st); }

}  // namespace ll
