"""MI355X-native detect-and-aggregate step of Aspis (MLSys 2022).

The product is libaspis.so (include/aspis.h): HIP kernels for gfx950 plus
the host steps of the method.  This package only binds it (aspis.py) and
builds it (build.py).
"""
from . import aspis  # noqa: F401
from .aspis import (AspisError, DetectBuffers, NormBuffers, TensorList,  # noqa: F401
                    aggregate, assign, clip_grads, clip_rows, clipped_adamw, clipped_sgd,
                    clique, detect, detect_aggregate, grad_norm, norm_workspace, num_files,
                    read_probe, row_norms, row_workspace)
