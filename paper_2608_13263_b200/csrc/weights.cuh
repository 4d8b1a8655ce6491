// What the two kernels of vtoken_token_weights share.
#pragma once
#include "attention.cuh"

struct VtkWeightsArgs {
    VtkAttnArgs at;                      // (values, outputs and parts are not used)
    const float *lse_in;
    vtk_arr<const float> prev;           // null: there is none
    vtk_arr<float> scores;
    float decay;
};

// host: launcher of weights_prompt.cu, and its part of the workspace
int vtk_launch_weights_prompt(vtoken_ctx *ctx, const vtoken_heads *heads, const VtkWeightsArgs &w, void *workspace, cudaStream_t st);
int64_t vtk_weights_prompt_workspace(const vtoken_ctx *ctx, const vtoken_heads *heads, int32_t max_query_tokens);
