// The status and state block at the head of a loss's workspace.
#pragma once

namespace kdkl {

constexpr int KDKL_MAGIC = 0x4b444b4c;  // "KDKL"
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;

// Head of the workspace (256 bytes). Written by forward, read by backward.
struct WsHeader {
  int status;        // 0 or the first device-detected error code
  int where;         // detail for the error (wait site, row, ...)
  int magic;         // KDKL_MAGIC once forward has completed its last kernel
  int go;            // backward gate: 1 when the state matches the call, else 0
  long long T, H, V;
  int K;
  int n_bad_idx;     // teacher indices >= V seen by prep (ignored entries)
  long long n_tokens;  // number of counted tokens (mask = 1)
  float denom;       // divisor of the mean actually used
  float tau;
  double loss_sum;   // sum of counted per-token losses
  long long chunk;   // tokens per chunk of the forward call that filled the workspace
  int g_state;       // what the [chunk, V] buffer holds after forward: G_NONE, G_EXPONENTIALS (option
                     // stored_exponentials: backward converts them once), G_CONSUMED (they have been converted)
  int neg_grad;      // 1 when the upstream gradient of the backward call in flight is negative (the recompute
                     // GEMM carries |a_t| in the exponent and needs the sign separately)
};

}  // namespace kdkl
