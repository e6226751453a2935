#include "serve_common.cuh"
namespace stream {
bool prompt_tc_supported(const PromptGeom &, int, const void *, const void *, const void *) { return false; }
stream_status launch_prompt_tc(const PromptGeom &, const void *, const void *, const void *, cudaStream_t) { return STREAM_ERR_UNSUPPORTED; }
}  // namespace stream
