// Launches and workspace of the experts: host arithmetic, apart from the kernels for the CPU tests.  Not part of the
// public ABI.
#pragma once

#include <stddef.h>

namespace ffn {

constexpr int kMoePieces = 8;  // of an expert's neurons, at most

// Groups of workgroups of k_moe_hidden and k_moe_down: a place's expert each, or an expert each.
int moe_slots(int T, int E, int k);
// Elements of a hidden row in the workspace.
int moe_ldz(int d_ff);
// Pieces of the neurons in k_moe_down, and room for what they leave, rows of d: pieces T k or more, and no less for more tokens.
int moe_pieces(bool f32, int T, int d, int d_ff, int E, int k);
size_t moe_part_rows(bool f32, int T, int d, int d_ff, int E, int k);

}  // namespace ffn
