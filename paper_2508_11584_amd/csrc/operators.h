// Operators on packed rows of many requests (vpe_attention, vpe_block_norm, vpe_adapter_linear): what their launchers take.  The entry points
// in operators.hip have checked it.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "vpe.h"

namespace vpe {

// Launch plan of an attention call: a function of its sizes alone, so that workspace and grid agree whatever the arrays hold.
struct SeqAttnPlan {
    int rows;            // rows of a workgroup: 128, 64 or 32
    int blocks;          // row blocks of the longest possible sequence, or of all sequences together (`packed`); -1: too many for a launch
    int packed;          // 1: a workgroup looks its sequence up among the row blocks of all of them
    int splits;          // parts of the keys, joined by a launch of their own if there are several
    int per_split;       // keys of a part (a multiple of the key tile)
    int64_t sets;        // key sets that row blocks read: key heads, sequences (unless packed), parts
    int chunk;           // row blocks of a set that follow one another on an XCD
    uint32_t grid;
    uint64_t workspace;
};
SeqAttnPlan plan_seq_attention(const vpe_attention_args& a);
hipError_t launch_seq_attention(const vpe_attention_args& a, const SeqAttnPlan& plan, hipStream_t s);

hipError_t launch_block_norm(const vpe_block_norm_args& a, hipStream_t s);

uint64_t adapter_linear_workspace(const vpe_adapter_linear_args& a);
hipError_t launch_adapter_linear(const vpe_adapter_linear_args& a, hipStream_t s);

// Leaves the message that vpe_last_error(NULL) gives on this thread, returns `code` (engine.hip).
int call_error(int code, const char* message) noexcept;

}  // namespace vpe
