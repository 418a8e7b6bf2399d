// The launchers of the norm and rotation at given positions and of cross attention
// as host stubs, for the sanitizer build of their validation layer: each writes one
// byte through every pointer that it is handed for a result, so that a wrong one is
// found.
#include "sol_cross.h"

namespace sol {

size_t norm_rope_bwd_bytes(int64_t, int heads) { return (size_t)heads * 1024; }
size_t cross_fwd_bytes(const CrossShape& s, CrossFwd* a, void* ws) {
  if (a) a->ws = static_cast<float*>(ws);
  if ((int64_t)s.B * s.H * s.N > 1 << 27) return kTooLarge;
  return s.M > 1000 || (s.mask && s.N > 1000) ? (size_t)s.N * 1024 : 0;
}
size_t cross_bwd_bytes(const CrossShape& s, CrossBwd* a, void* ws) {
  if (a) a->stats = static_cast<float*>(ws);
  return (int64_t)s.B * s.H * s.N > 1 << 27 ? kTooLarge : (size_t)s.H * 1024;
}

static void touch(void* p) {
  if (p) *static_cast<volatile char*>(p) = 0;
}
hipError_t launch_norm_rope_fwd(const NormRopeFwd& a, hipStream_t) {
  touch(a.q_out.p);
  touch(a.k_out.p);
  return hipSuccess;
}
hipError_t launch_norm_rope_bwd(const NormRopeBwd& a, hipStream_t) {
  touch(a.dq.p);
  touch(a.dk.p);
  touch(a.dq_gamma);
  touch(a.dk_gamma);
  touch(a.partial);
  return hipSuccess;
}
hipError_t launch_cross_fwd(const CrossFwd& a, hipStream_t) {
  touch(a.out.p);
  touch(a.left);
  touch(a.lse);
  touch(a.ws);
  return hipSuccess;
}
hipError_t launch_cross_bwd(const CrossBwd& a, hipStream_t) {
  touch(a.dq.p);
  touch(a.dk.p);
  touch(a.dv.p);
  touch(a.stats);
  return hipSuccess;
}

}  // namespace sol
