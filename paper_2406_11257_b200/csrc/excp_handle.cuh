// The handle behind excp_handle and the small helpers that every C entry point uses.
#pragma once
#include <vector>

#include "../../include/excp.h"
#include "excp_common.cuh"
#include "score.cuh"

namespace excp {
// Launch counter and optional CUDA-event timing of the stages of one call.
struct Profiler {
    bool enabled = false;
    std::vector<cudaEvent_t> ev;
    std::vector<int> stage;
    size_t used = 0;
    double ms[ST_COUNT] = {};
    unsigned long long launches = 0;
    void begin(cudaStream_t s) {
        used = 0;
        launches = 0;
        for (double& m : ms) m = 0.0;
        if (enabled && !ev.empty()) cudaEventRecord(ev[0], s);
    }
    void finish() {   // after the stream has been synchronised
        if (!enabled) return;
        for (size_t i = 1; i <= used; ++i) {
            float t = 0.f;
            if (cudaEventElapsedTime(&t, ev[i - 1], ev[i]) == cudaSuccess) ms[stage[i]] += t;
        }
    }
};
}  // namespace excp

struct excp_handle_s {
    int device = 0;
    int sms = 0;
    size_t cap_tiles = 0;
    excp::Workspace ws{};
    excp::KmArrays km{};
    excp::TensorState* d_state = nullptr;      // MAX_GROUP_TENSORS
    excp::DecState* d_dstate = nullptr;        // MAX_GROUP_TENSORS
    excp::CallState* d_call = nullptr;
    void* d_desc = nullptr;              // TensorDesc[] or DecDesc[] of the whole call
    excp::TensorResult* d_results = nullptr;
    void* h_desc = nullptr;              // pinned
    excp::TensorResult* h_results = nullptr;   // pinned
    excp::CallState* h_call = nullptr;         // pinned
    size_t tensor_cap = 0;               // entries the per-call arrays hold
    int last_cuda_error = 0;
    int km_margin = 1;                   // see excp_set_kmeans_margin
    unsigned long long wait_limit_ns = 2000000000ull;   // see excp_set_wait_limit
    bool report_sse = false;             // see excp_set_report_sse
    excp::Profiler prof;
    // host-buffer path: two staging slots (inputs + records), its own copy streams
    float* stage[2][4] = {};
    unsigned char* stage_blob[2] = {};
    size_t stage_blob_bytes = 0;
    int stage_bits = 0;                  // code width the record staging is sized for
    cudaStream_t s_h2d = nullptr, s_d2h = nullptr;
    cudaEvent_t ev_h2d[2] = {}, ev_compute[2] = {}, ev_d2h[2] = {};
    excp::ScoreWorkspace score;                // operators that score a restored checkpoint (score_api.cu)
};

struct DeviceGuard {
    int prev = -1;
    bool ok = true;
    explicit DeviceGuard(int dev) {
        if (cudaGetDevice(&prev) != cudaSuccess) prev = -1;
        if (prev != dev) ok = cudaSetDevice(dev) == cudaSuccess;
    }
    ~DeviceGuard() {
        int now = -1;
        if (prev >= 0 && cudaGetDevice(&now) == cudaSuccess && now != prev) cudaSetDevice(prev);
    }
};

inline bool check(excp_handle h, cudaError_t e) {
    if (e == cudaSuccess) return true;
    h->last_cuda_error = (int)e;
    return false;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
