// Host-side argument bundles of the operators around a token mixer (short causal convolution,
// selective state space scan, group norm), shared by their C ABI (ll_layer_api.hip) and kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace ll {

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// A launch holds fewer than 2^32 threads.
inline bool launchable(int64_t workgroups, int threads) { return workgroups <= int64_t(0xffffffff) / threads; }

// A [B, T, D] tensor whose channels are adjacent: strides of a sequence and of a token in elements.
struct Rows {
  const void* p = nullptr;
  int64_t sb = 0, st = 0;
};

// Whether rows of `width` elements of `esize` bytes may be read `n` elements at a time.
inline bool rows_aligned(const Rows& r, int esize, int n) {
  return reinterpret_cast<uintptr_t>(r.p) % (uintptr_t(esize) * n) == 0 && r.sb % n == 0 && r.st % n == 0;
}

// ---- selective scan
struct ScanArgs {
  Rows x, dt, z, Bm, Cm;  // z.p may be null
  const float* A;
  const float* skip;      // may be null
  const float* dt_bias;   // may be null
  const int32_t* lengths; // may be null
  int64_t B, T, D, N, G;
  int softplus, dtype;
  const float* h0;        // may be null: zeros
  float* h_final;         // may be null
  float* states;          // forward: may be null; backward: the forward's
  void* y;
  void* workspace;
};

struct ScanGrads {
  const void* dy;
  const float* dh_final;  // may be null: zeros
  void* dx;
  void* ddt;
  void* dz;               // null without a gate
  float* dA;
  void* dB;
  void* dC;
  float* dskip;           // may be null
  float* dbias;           // may be null
  float* dh0;             // may be null
};

constexpr int kScanMaxN = 64;

// How a scan is split over its length: S segments of `len` tokens (a multiple of 4: one of fewer than 16 may hold no
// saved state).
struct ScanSplit {
  int64_t S = 1, len = 0;
};
// The segments' records of one split scan, joined in place (see k_scan_join); `reverse`: from the last segment on.
struct ScanJoin {
  const float *A, *init;  // init [B, D, N], may be null: zeros
  float* h;               // [B, S, D, NP]
  const float* d;         // [B, S, D] sums of step sizes
  int64_t B;
  int S;
  int64_t D;
  int N, NP;
  bool reverse;
};
int64_t scan_join_workgroups(int64_t B, int64_t D, int64_t NP);  // of 64 threads, or at most 512 of 1024
hipError_t launch_scan_join(const ScanJoin& p, hipStream_t st);
int scan_state_blocks(int64_t N);            // blocks of 16 states a lane group holds: 1, 2 or 4
constexpr int kScanChunk = 16;               // tokens between two saved states
int64_t scan_states_bytes(int64_t B, int64_t T, int64_t D, int64_t N);
int64_t scan_fwd_workspace(int64_t B, int64_t T, int64_t D, int64_t N, int64_t G);
int64_t scan_bwd_workspace(int64_t B, int64_t T, int64_t D, int64_t N, int64_t G);
// The *_launchable: whether each launch of a call on these sizes holds few enough threads.
bool scan_fwd_launchable(const ScanArgs& a);
bool scan_bwd_launchable(const ScanArgs& a);
bool scan_step_launchable(const ScanArgs& a);
hipError_t launch_scan_fwd(const ScanArgs& a, hipStream_t st);
hipError_t launch_scan_bwd(const ScanArgs& a, const ScanGrads& g, hipStream_t st);
hipError_t launch_scan_step(const ScanArgs& a, hipStream_t st);  // h0 -> h_final, one token

// ---- causal convolution
struct ConvArgs {
  Rows x;
  const float* weight;
  const float* bias;       // may be null
  const void* state;       // [B, W-1, D], may be null: zeros
  void* new_state;         // may be null
  const int32_t* lengths;  // may be null
  void* y;
  int64_t B, T, D, W;
  int act, dtype;
};
struct ConvGrads {
  const void* dy;
  const void* dfinal;      // may be null
  void* dx;
  float* dw;
  float* db;               // may be null
  void* dinit;             // may be null
  void* workspace;
};
int64_t conv_bwd_workspace(int64_t B, int64_t T, int64_t D, int64_t W, int dtype);
bool conv_launchable(const ConvArgs& a, bool backward);
hipError_t launch_conv_fwd(const ConvArgs& a, hipStream_t st);
hipError_t launch_conv_bwd(const ConvArgs& a, const ConvGrads& g, hipStream_t st);
hipError_t launch_conv_step(const ConvArgs& a, hipStream_t st);

// ---- group norm
struct NormArgs {
  Rows x, z;               // [N, S, C]; z.p may be null
  const float* weight;     // may be null: ones
  const float* bias;       // may be null: zeros
  void* y;
  float* stats;            // [N, G, 2] mean and 1/std; forward: may be null
  int64_t N, S, C, G;
  float eps;
  int act, dtype;
  void* workspace;
};
struct NormGrads {
  const void* dy;
  void* dx;
  void* dz;                // null without a gate
  float* dw;               // may be null
  float* db;               // may be null
};
int64_t norm_workspace(int64_t N, int64_t S, int64_t C, int64_t G, int dtype, bool backward);
bool norm_launchable(const NormArgs& a, bool backward);
hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t st);
hipError_t launch_norm_bwd(const NormArgs& a, const NormGrads& g, hipStream_t st);

// Column sums of an fp32 matrix of partial sums, rows added in an order that the sizes alone fix.  Output k
// takes columns col0 .. col0 + cols - 1; column c goes to out[(c / in_cols) * major + (c % in_cols) * minor],
// those with c % in_cols >= out_cols (padding) nowhere.
struct ColSum {
  struct Out {
    int64_t col0, cols;
    float* out;
    int64_t in_cols, out_cols, major, minor;
  };
  const float* part = nullptr;
  int64_t rows = 0, stride = 0;
  Out out[3] = {};
  int n = 0;
};
hipError_t launch_colsum(const ColSum& p, hipStream_t st);

}  // namespace ll
