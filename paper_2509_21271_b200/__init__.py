"""B200-native bucketized speculative AdamW (SuperOffload's optimizer hot path),
and the memory-bound operators of the training step around it
(:mod:`paper_2509_21271_b200.operators`), with AdamW over a list of tensors
(:mod:`paper_2509_21271_b200.tensor_adamw`).

The CUDA library is reached through :mod:`paper_2509_21271_b200.binding`
(loaded on first use; it raises if the compiled library is missing).
"""
__all__ = ["binding", "workloads", "build", "operators", "tensor_adamw"]
