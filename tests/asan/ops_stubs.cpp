// The linear and differential attention's launchers as host stubs, for the
// sanitizer build of their validation layer: each writes one byte through every
// pointer that it is handed for a result, so that a wrong one is found.
#include "sol_ops.h"

namespace sol {

size_t lin_states_bytes(int64_t slabs, int N, int) { return N > 10000 ? (size_t)slabs * kStateElems * 4 : 0; }
size_t diff_fwd_bytes(const DiffShape& s) { return s.M > 1000 ? (size_t)s.N * 1024 : 0; }
size_t diff_bwd_bytes(const DiffShape& s, DiffBwd*) { return (size_t)s.H * 1024; }

static void touch(void* p) {
  if (p) *static_cast<volatile char*>(p) = 0;
}
hipError_t launch_lin_fwd(const LinFwd& a, hipStream_t) {
  touch(a.out.p);
  touch(a.state_out);
  touch(a.states);
  return hipSuccess;
}
hipError_t launch_lin_bwd(const LinBwd& a, hipStream_t) {
  touch(a.dq.p);
  touch(a.dk.p);
  touch(a.dv.p);
  touch(a.dstate_out);
  touch(a.partial);
  return hipSuccess;
}
hipError_t launch_lin_step(const LinStep& a, hipStream_t) {
  touch(a.out.p);
  touch(a.state);
  return hipSuccess;
}
hipError_t launch_diff_fwd(const DiffFwd& a, hipStream_t) {
  touch(a.out.p);
  touch(a.out2);
  touch(a.lse);
  return hipSuccess;
}
hipError_t launch_diff_bwd(const DiffBwd& a, hipStream_t) {
  touch(a.dq.p);
  touch(a.dk.p);
  touch(a.dv.p);
  touch(a.dlambda);
  touch(a.stats);
  return hipSuccess;
}

}  // namespace sol
