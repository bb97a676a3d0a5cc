// The context behind the C ABI's handle; shared by the files that implement its entry points.
#pragma once
#include "../../include/lasad.h"
#include "lasad_common.cuh"

struct lasad_ctx {
    int device;
    int* d_status;        // device status word
    int last_cuda_error;
    uint64_t launches;
    int opt_prefill_impl; // LASAD_OPT_PREFILL_IMPL: 0 auto, 1..5 as listed in lasad.h
    int opt_prefill_chunk;
    int opt_decode_tpu;
    int opt_window_impl;  // LASAD_OPT_WINDOW_IMPL: 0 auto, 1 CUDA cores, 2 tensor cores
    unsigned wait_limit;
    int sm_count;
    // state relay of the task-streaming prefill (see lasad_prefill_tc_stream.cu)
    void* d_relay;                // [relay_cap] slots of kTcRelaySlotBytes
    int64_t relay_cap;
    uint64_t epoch;               // launches of the task-streaming prefill so far
    int stream_max_ctas;
    // states at the cuts when the CTA-per-chain prefill splits few, long chains into segments
    float* d_segstate;            // [2 x SMs][dk * dv], then [2 x SMs] counters
    // per-chain flags of the gated tensor-core prefill: chains it left to the CUDA-core kernel
    int* d_redo;                  // [redo_cap]
    int64_t redo_cap;
    // state slots and flags at the cuts of the balanced tensor-core prefill (one per SM)
    void* d_pair;
    // host-buffer pipeline of lasad_forward_host: two staging slots (q | k | v | o of one batch
    // element each), a decay and a state buffer, copy streams and the events that order them
    void* d_stage[2];
    size_t stage_bytes;
    float* d_host_decay;
    int64_t host_decay_cap;
    float* d_host_state;
    size_t host_state_bytes;
    cudaStream_t s_in, s_out;
    cudaEvent_t ev_start, ev_in[2], ev_comp[2], ev_out[2];
    bool pipeline_ready;
};
