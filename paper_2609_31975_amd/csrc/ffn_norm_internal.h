// Launches of the norms: host arithmetic, apart from the kernels for the CPU tests.  Not part of the public ABI.
#pragma once

namespace ffn {

// Threads to a row and elements to a thread.
struct NormPlan {
  int tpr, ept;
};
NormPlan norm_forward_plan(int d);
NormPlan norm_backward_plan(int d);
// Workgroups of the forward call, each of which takes every so many'th row (four of them with 64 threads to a row).
int norm_blocks(int T, int d);
// Groups of threads of the backward call, each of which takes every so many'th row, and rows of its partial sums.
int norm_groups(int T, int d);

}  // namespace ffn
