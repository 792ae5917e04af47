#include "joint.h"
namespace dckv {
JointPrompt joint_prompt(const dckv_joint_desc& d, int32_t batch, int32_t n_rows, int32_t max_context,
                         int64_t total_context) { return JointPrompt{}; }
hipError_t launch_joint_prefill(const JointPrompt& s, const void* q, const int32_t* row_start,
                                const void* pool, int64_t num_pages, const int32_t* page_table,
                                int32_t max_pages, const int32_t* seq_lens, const void* W_keys,
                                const void* W_values, void* out, void* workspace, hipStream_t stream) { return hipErrorInvalidValue; }
}
