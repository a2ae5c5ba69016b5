"""MI355X-native batched simulation of distributed training strategies
(DistIR's simulator, Santhanam et al., MLSys 2022).

The simulation runs in the HIP kernels of ``libdsim.so`` behind the C ABI in
``include/dsim.h``; ``paper_2111_05426_amd.dsim`` is its Python binding,
``paper_2111_05426_amd.workloads`` holds the synthetic workload shapes,
``paper_2111_05426_amd.frontend`` binds the library's front end, which
turns programs written op by op into op tables (mixed abstract/concrete
interpretation, host C++), ``paper_2111_05426_amd.programs``
writes example programs for it, ``paper_2111_05426_amd.ops`` binds the
operators of a single-token step (``include/dsim_ops.h``: paged cache append,
paged attention, logit adjustment) and of a step of several tokens
(``include/dsim_multi_ops.h``: attention of prompts and drafted trees, the
append on several axes, the cache's pages), and ``paper_2111_05426_amd.calibrate`` fits
the empirical costs on the GPU it runs on.
"""
__all__ = ["dsim", "workloads", "frontend", "programs", "ops", "calibrate"]
