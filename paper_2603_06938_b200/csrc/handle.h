// The library's handle and what every entry point does with it: error text, alignment, device.
#pragma once
#include <cstdio>

#include "internal.h"
#include "tc05.cuh"

using namespace swimba;

struct swimba_handle {
    swimba_config cfg;
    int device;
    int sm_count;
    int *d_status;          // device status word
    cudaStream_t last_stream;
    int last_launches;
    Profiler prof;
    TmapCache tmaps;        // tensor maps encoded so far (same buffers call after call: encoded once)
    // host-buffer entry point: copy streams and events of its batch-slice pipeline
    cudaStream_t s_in, s_out;
    cudaEvent_t ev_start, ev_out, ev_in[32], ev_done[32];
    char err[256];
};

namespace {

constexpr size_t kAlign = 256;
inline size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }
inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t elt_size(int dtype) { return dtype == SWIMBA_DTYPE_FP32 ? 4 : 2; }

inline int fail(swimba_handle *h, int code, const char *msg)
{
    if (h) snprintf(h->err, sizeof(h->err), "%s", msg);
    return code;
}

inline int set_device(swimba_handle *h)
{
    int cur = -1;
    if (cudaGetDevice(&cur) != cudaSuccess) return fail(h, SWIMBA_ERR_CUDA, "cudaGetDevice failed");
    if (cur != h->device) return fail(h, SWIMBA_ERR_CUDA, "handle used on a different device than it was created on");
    return SWIMBA_OK;
}

}  // namespace
