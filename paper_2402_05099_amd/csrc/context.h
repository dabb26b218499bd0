// What a context holds (host side), for the translation units with entry points.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>

struct hg_ctx {
    int device;
    hipStream_t stream;
    unsigned char* ws;
    size_t ws_bytes;
    int opt_prefix_splits;
    int opt_suffix_chunk;
    int opt_overlap;
    int opt_naive_chunk;
    int opt_prefix_kernel;
    int opt_wide_slots;
    int opt_nq;            // queries per sequence (1 = decode)
    int opt_suffix_kernel; // 0 automatic, 1 vector-ALU kernel, 2 matrix-core kernel wherever it applies
    int opt_suffix_ipw;    // matrix-core suffix kernel: work items per wavefront (0 automatic)
    int opt_suffix_tile;   // matrix-core suffix kernel: query rows per tile (0 automatic, 16, 32)
    int opt_fused_kernel;  // fused call: 0 automatic, 1 separate kernels, 2 single launch whenever it applies
    unsigned* counters;    // kContextCounters device counters, zero between calls (null: none left)
    int counter_slot;      // (-1: none, or not to be given back)
    bool counters_used, counters_in_graph;
    hipStream_t counter_stream;      // the stream that used them last
    hipStream_t aux;       // second stream for the overlap option
    hipEvent_t ev_fork, ev_join;
    // stage timing ring: slot = call % HG_TIMING_RING, 2 events (begin, end) per stage
    int opt_timing;
    hipEvent_t* tev;       // [HG_TIMING_RING][HG_MAX_STAGES][2], created when timing is first enabled
    unsigned char* tused;  // [HG_TIMING_RING][HG_MAX_STAGES]
    long long tcalls;      // fused calls recorded since timing was enabled
};
