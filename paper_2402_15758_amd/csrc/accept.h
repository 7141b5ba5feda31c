// Verification of drafted tokens by their probabilities (kernels_accept.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

// A tree of up to 64 nodes by value, a byte a parent (the root's: 0), as words that
// scalar loads bring whole.
struct AcceptTree {
  uint32_t parent[16];
  void set(int u, int p) { parent[u / 4] |= (uint32_t)(u == 0 ? 0 : p) << (8 * (u % 4)); }
};

// A row's largest logit and its sum of exp((z - largest) / temperature).
struct RowSum {
  double m, s;
};
// Where a sequence's walk ended.
struct Walk {
  int node, depth;          // node -1: an empty place
  bool ok;                  // the last row has a distribution
  uint64_t path, rejected;  // nodes on the path; rejected children of the last one
  RowSum p, q;              // of the last row
};

struct AcceptArgs {
  const void* logits;       // [B N][ld]
  int64_t ld;
  const void* draft;        // [B N][ldd], nullptr: the tokens were chosen
  int64_t ldd;
  const int* tokens;        // [B][N]
  const double* u;          // [B][N]
  int B, N, V, K;           // K: the tree's depth
  double scale;             // 32 / (temperature ln 2)
  int* new_tokens;          // [B][K + 1]
  int* n_new;               // [B]
  int* path;                // [B][K + 1], nullptr: not wanted
  int parts;                // of a row
  // scratch: each part's maximum and sum of exp((z - maximum) / temperature), target rows
  // then draft rows; the residual's parts; the walks
  float* part_m;            // [2][B N][parts]
  double* part_s;
  double* resid;            // [B][parts]
  Walk* walks;              // [B]
  uint64_t inner;           // nodes with children
  int none;                 // what stands for a token where a row has no distribution
  AcceptTree tree;
};
constexpr int ACCEPT_PART = 1024;  // entries of a part: 16 a lane
inline double accept_scale(float temperature) { return 32.0 / ((double)temperature * 0.69314718055994530942); }
int64_t accept_bytes(int B, int N, int V, bool drawn);
void accept_carve(AcceptArgs& a, void* ws);
void launch_accept(int dtype, const AcceptArgs& a, hipStream_t st);
// Random numbers of a step: u[b][i] of sequence b and node i at its committed length
// n_b[b], the top 53 bits of SplitMix64(SplitMix64(SplitMix64(SplitMix64(seed) ^ b) ^ n)
// ^ i).
void launch_accept_uniforms(const int* n_b, int B, int N, unsigned long long seed, double* u, hipStream_t st);
// The same for prompts that end in a prefill chunk, i = 64; tokens[j] = 0.
struct PrefillEnds;
void launch_accept_first(const PrefillEnds& e, unsigned long long seed, double* u, int* tokens, hipStream_t st);
