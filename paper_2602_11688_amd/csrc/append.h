// What the host side of gorgo_kv_append and gorgo_rotate_heads (append.cpp) hands to their kernel (append.hip).
#pragma once
#include "attention.h"

namespace gorgo {

struct RotationArgs {
    const double* frequencies;           // null: no rotation, and no pairs
    const int32_t* positions;            // [axes][tokens], or null: places in the sequences
    int64_t axis_stride;
    double magnitude;
    uint64_t axis_low, axis_high;        // bit i: of pair i's axis
    int32_t pairs, neighbours;
};

struct NormArgs {
    const float* weight;                 // null: ones
    int64_t head_stride;
    float eps;                           // 0: no norm
};

struct AppendArgs {
    CacheArgs cache;                     // (rows alone: only d)
    BatchArgs batch;
    RotationArgs rotation;
    NormArgs q_norm, k_norm;
    RowsArgs q, q_out, k, v;
    Divider q_heads, kv_heads;           // divisor 0: none of them
    float one_over_d;
    int32_t pair_bits;                   // least power of two that holds all pairs
    int32_t block, parts;                // tokens of a workgroup, and workgroups that share them
};

constexpr int APPEND_THREADS = 256;
constexpr int MOST_BLOCK = 8;            // tokens of a workgroup at most
constexpr int MOST_PAIRS = MAX_HEAD / 2;

// append.hip
int launch_append(const AppendArgs& a, int type, void* stream);

}  // namespace gorgo
