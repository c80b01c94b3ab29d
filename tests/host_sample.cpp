// csrc/sample.hip on the host (stub_wavefronts): SAMPLE_SOURCE is its text with launches as calls and the two lines of assembly as what
// they compute.
#include SAMPLE_SOURCE

extern "C" size_t host_sample_workspace(int M, int V) { return evospec::sample_workspace(M, V); }
// NULL, or what went wrong
extern "C" const char* host_sample(unsigned order, const void* logits, long long stride, int type, int M, int V, const float* u,
                           const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p, const int32_t* ids,
                           int32_t* out_ids, float* out_logprob, void* workspace) {
    wavefronts::order = order;
    wavefronts::lines.clear();
    const evospec::SampleArgs a{logits, stride, M, V, u, temperature, top_k, top_p, min_p, ids, out_ids, out_logprob};
    static wavefronts::Error error;
    try {
        evospec::launch_sample(a, type, workspace, nullptr);
    } catch (const wavefronts::Error& e) {
        error = e;
        return error.text;
    }
    return nullptr;
}
// Barriers of the last call: lines of SAMPLE_SOURCE.
extern "C" int host_barriers(const int** lines) {
    *lines = wavefronts::lines.data();
    return (int)wavefronts::lines.size();
}
