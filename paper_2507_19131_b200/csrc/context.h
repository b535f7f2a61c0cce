// The library's context and the helpers of every host entry point: error texts, checks of launches, per-kernel timing.
#pragma once
#include <nvtx3/nvToolsExt.h>
#include "../../include/mixaq.h"
#include "graph_cache.h"
#include "kernels.h"
#include <cstdio>
#include <mutex>
#include <vector>

struct ProfRec { int cat; cudaEvent_t e0, e1; };
constexpr size_t MAX_BACKBONE_GRAPHS = 16, MAX_BLOCK_GRAPHS = 8;     // kept, and calls remembered (see graph_cache.h)
struct mixaq_ctx {
  int device;
  int* d_status;
  int launches;
  char err[256];
  bool profiling;
  bool graph_cache;                    // replay backbone forwards as CUDA graphs (see mixaq_set_graph_cache)
  bool reverse_selection;              // backbone: worst-case selection order (Table 4) in every block
  bool prof_capture;                   // the profiled call is being captured: event records become graph nodes
  std::vector<cudaGraphExec_t> prof_execs;   // graphs of profiled forwards, destroyed when the profiling ends
  bool guards;                         // fill the guard zones of the workspace before a forward, compare them after it
  bool nvtx;                           // name every kernel family, stage and block with an NVTX range (host side)
  bool allow_elevation;                // backbone: every pair uses its own ratios even if an earlier pair of the stage had larger ones
  cudaStream_t capture_stream;         // calls are recorded here, not on the caller's stream (see replay_record_or_run)
  cudaStream_t side_stream; cudaEvent_t fork, join;   // output norms run beside the next stage inside a captured forward
  std::mutex graph_lock;               // for what follows and the two streams above
  mixaq::GraphCache<cudaGraphExec_t> graphs{MAX_BACKBONE_GRAPHS, MAX_BACKBONE_GRAPHS};      // of backbone forwards
  mixaq::GraphCache<cudaGraphExec_t> block_graphs{MAX_BLOCK_GRAPHS, MAX_BLOCK_GRAPHS};
  std::vector<ProfRec> prof;          // event pairs recorded since mixaq_profile_begin
  std::vector<cudaEvent_t> pool;      // events ready for reuse
};

enum ProfCat { PC_ENERGY = 0, PC_SELECT, PC_LN1, PC_QKV, PC_ATTN, PC_PROJ, PC_LN2, PC_FC1, PC_FC2, PC_COPY,
               PC_MERGE_GATHER, PC_MERGE_GEMM, PC_STEM, PC_OUT_NORM, PC_BRACKET, PC_FP8_QUANT, PC_FP8_MATMUL, PC_RES_NORM, PC_COUNT };
static const char* const kProfNames[PC_COUNT] = {"energy", "select", "gather_ln1_quant", "gemm_qkv", "attention",
                                           "gemm_proj", "ln2_quant", "gemm_fc1_gelu", "gemm_fc2_scatter",
                                           "copy_pruned", "merge_gather_ln_quant", "gemm_merge", "patch_embed",
                                           "stage_output_norm", "empty_event_bracket", "fp8_quantize", "fp8_matmul",
                                           "residual_norm"};

namespace {

inline bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline mixaq_status fail(mixaq_ctx* ctx, mixaq_status s, const char* msg) {
  if (ctx) snprintf(ctx->err, sizeof(ctx->err), "%s", msg);
  return s;
}

inline mixaq_status check_cuda(mixaq_ctx* ctx, const char* where) {
  cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess) return MIXAQ_OK;
  if (ctx) snprintf(ctx->err, sizeof(ctx->err), "%s: %s", where, cudaGetErrorString(e));
  return MIXAQ_CUDA_ERROR;
}

// Per-kernel CUDA-event timing (only while profiling is on; the events sit on the launching stream).
struct ProfScope {
  mixaq_ctx* ctx; cudaStream_t st; cudaEvent_t e1; bool on, range;
  ProfScope(mixaq_ctx* c, int cat, cudaStream_t s) : ctx(c), st(s), e1(nullptr), on(c && c->profiling), range(c && c->nvtx) {
    if (range) nvtxRangePushA(kProfNames[cat]);
    if (!on) return;
    cudaEvent_t ev[2];
    for (int i = 0; i < 2; ++i) {
      if (!ctx->pool.empty()) { ev[i] = ctx->pool.back(); ctx->pool.pop_back(); }
      else if (cudaEventCreate(&ev[i]) != cudaSuccess) { on = false; return; }
    }
    record(ev[0]);
    e1 = ev[1];
    ctx->prof.push_back({cat, ev[0], ev[1]});
  }
  // inside a stream capture the record becomes a graph node of its own (an "external" event keeps its timestamp)
  void record(cudaEvent_t e) {
    if (ctx->prof_capture) cudaEventRecordWithFlags(e, st, cudaEventRecordExternal);
    else cudaEventRecord(e, st);
  }
  ~ProfScope() { if (on) record(e1); if (range) nvtxRangePop(); }
};

}  // namespace
