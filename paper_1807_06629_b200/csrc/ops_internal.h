// Host entries that the context's own local step shares with the stand-alone operators.
#pragma once
#include "kernels_ortho.cuh"

namespace prsgd {

struct NsPlan {                    // one orthogonalisation of a batch, arguments already checked
  NsShape shape;
  NsSource src; int g_type;
  NsDest dst;
  int steps; float a, b, c, eps;
  int precision;
  DeviceStatus* status;            // a context's status words, or nullptr: the workspace's
};
int ns_prepare();                  // what the first call on a device needs to find out, outside a stream capture

size_t ns_workspace_bytes(const NsShape& sh, int precision);
// Enqueues the whole chain; returns a PRSGD_ code and counts its launches.
int ns_run(const NsPlan& p, void* d_work, cudaStream_t st, int64_t* launches);

}  // namespace prsgd
