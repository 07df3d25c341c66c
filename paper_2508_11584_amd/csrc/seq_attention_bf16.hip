// Instantiations of the attention over packed sequences, bf16.
#include "seq_attention.h"

namespace vpe {
namespace {

template <bool CAP, int DIST>
SeqShape of(int head_dim, int rows) {
    // (with these 64 keys at a time take a register or more too many)
    constexpr int K64 = CAP || DIST == DIST_LINE ? 32 : 64, K128 = CAP && DIST == DIST_GRID ? 32 : 64;
    if (head_dim == 64) return rows == 128 ? seq_shape<bf16, 64, K64, 4, 1, CAP, DIST, 3>() : rows == 64 ? seq_shape<bf16, 64, 32, 2, 2, CAP, DIST, 3>() : seq_shape<bf16, 64, 32, 1, 4, CAP, DIST, 2>();
    return rows == 128 ? seq_shape<bf16, 128, K128, 4, 1, CAP, DIST, 2>() : rows == 64 ? seq_shape<bf16, 128, 32, 2, 2, CAP, DIST, 2>() : seq_shape<bf16, 128, 32, 1, 4, CAP, DIST, 1>();
}

}  // namespace

SeqShape seq_shape_bf16(bool cap, int dist, int head_dim, int rows) {
    if (cap) return dist == DIST_GRID ? of<true, DIST_GRID>(head_dim, rows) : dist == DIST_LINE ? of<true, DIST_LINE>(head_dim, rows) : of<true, DIST_NONE>(head_dim, rows);
    return dist == DIST_GRID ? of<false, DIST_GRID>(head_dim, rows) : dist == DIST_LINE ? of<false, DIST_LINE>(head_dim, rows) : of<false, DIST_NONE>(head_dim, rows);
}

}  // namespace vpe
