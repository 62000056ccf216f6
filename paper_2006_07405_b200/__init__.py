"""B200-native A2SGD per-worker gradient path (two-level gradient averaging).

``binding`` wraps the C-ABI CUDA library (``liba2sgd.so``, built in-tree from
``csrc/``): the gradient path, and the training operators beside it (AdamW,
layer norm, the gated feed-forward block, windowed attention, rotary positions,
the residual connection with its norms); ``workloads`` holds the seeded synthetic input generators.  There
is no CPU fallback: calling the binding without the built library raises.
"""
