"""B200-native DropCompute threshold-sweep simulator.

``paper_2306_10598_b200.api`` is the thin binding over the C-ABI library (it raises if the CUDA
library is missing); ``paper_2306_10598_b200.workloads`` holds the seeded synthetic inputs;
``paper_2306_10598_b200.build`` compiles the library in-tree.  ``api`` also binds the training operators;
``paper_2306_10598_b200.autograd`` has them as differentiable functions and ``drop_train`` runs them in Algorithm 1's loop.
"""
__all__ = ["api", "workloads", "build", "autograd", "drop_train"]
