// The gated delta rule's kernels for blr_gdr_fwd and blr_gdr_bwd: f32.
#include "blr_gdr_launch.cuh"

namespace blr {
namespace gdr {

blr_status fwd_f32(const Problem& p, const FwdCall& c) { return fwd<float, 3, 3>(p, c); }
blr_status bwd_f32(const Problem& p, const BwdCall& c) { return bwd<float, 3, 3>(p, c); }

}  // namespace gdr
}  // namespace blr
