// Launch stubs of the ragged-batch and query/key calls for the host-only sanitizer
// build: a launch aborts unless it is expected, and leaves its arguments here then.
#include "serve_stubs.hpp"

#include <cstdio>
#include <cstdlib>

namespace sf {
ServeRecord *serve_record = nullptr;
static ServeRecord &record(const char *what) {
    if (!serve_record) {
        std::fprintf(stderr, "unexpected launch: %s\n", what);
        std::abort();
    }
    return *serve_record;
}
hipError_t launch_gdn_tokens(const GdnRaggedArgs &a, hipStream_t, hipEvent_t, hipEvent_t) {
    record("launch_gdn_tokens").gdn.push_back(a);
    return hipSuccess;
}
hipError_t launch_gdn_chunk_prep(const GdnRaggedArgs &a, hipStream_t, hipEvent_t, hipEvent_t) {
    record("launch_gdn_chunk_prep").prep.push_back(a);
    return hipSuccess;
}
hipError_t launch_gdn_chunk_walk(const GdnRaggedArgs &a, hipStream_t, hipEvent_t, hipEvent_t) {
    record("launch_gdn_chunk_walk").walk.push_back(a);
    return hipSuccess;
}
hipError_t launch_conv_ragged(const ConvRaggedArgs &a, hipStream_t, hipEvent_t, hipEvent_t) {
    record("launch_conv_ragged").conv.push_back(a);
    return hipSuccess;
}
hipError_t launch_qk(bool bwd, const QkArgs &a, hipStream_t, hipEvent_t, hipEvent_t) {
    record("launch_qk").qk.push_back({bwd, a});
    return hipSuccess;
}
}  // namespace sf
