"""MI355X-native scaled-Muon optimizer step (hand-written HIP behind a C ABI), and the operators in front of it that make its
largest gradients.

``binding`` exposes the C entry points; ``losses`` and ``experts`` are the head's losses and the mixture's dispatch on torch
tensors; ``workloads`` holds the seeded synthetic inputs; ``build`` compiles the library in-tree for gfx950.
"""
__all__ = ["binding", "workloads", "build", "losses", "experts"]
