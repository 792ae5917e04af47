// The absorbed decode over the joint cache at rank 256.
#include "joint_attend.h"

namespace dckv {

hipError_t launch_joint_attend_256(const dckv_joint_desc& d, int row_waves, const JointAttend& a, hipStream_t stream) {
  return joint::launch<256>(d, row_waves, a, stream);
}

}  // namespace dckv
