"""Quantized Adam with error feedback: one parameter-server step on a B200, and the
training step around it (AdamW, gradient norm, embedding rows and their gradient, layer norm, products in 8 bits).

Thin Python binding over the C interface of include/qadam.h (libqadam.so, built
from csrc/ by build.py).  Every step of the method runs in the library's CUDA
kernels; this package only marshals arguments and uses PyTorch for device
memory and streams.  There is no CPU fallback: importing the binding without
the built library, or calling it without a CUDA device, raises.
"""
from .binding import (  # noqa: F401
    PLACE_SERVER, PLACE_WORKER, GRID_POW2, GRID_UNIFORM, GRID_STOCHASTIC,
    ST_NONFINITE, ST_TIMEOUT, ST_INDEX,
    QAdamError, QAdamConfig, QAdamBuffers, QAdamOptions, QAdam,
    SERVER_AUTO, SERVER_PLAIN, WORKER_AUTO, WORKER_STREAMING, HANDOVER_AUTO, HANDOVER_COUNTERS,
    qadam_create_ex, qadam_server_step_range, qadam_finish_step, qadam_shard_cuts,
    library_path, load_library, exported_symbols,
    qadam_query_sizes, qadam_grad_code_bits, qadam_weight_code_bits,
    qadam_create, qadam_worker_compress, qadam_server_step, qadam_step_host,
    qadam_worker_scales_static, STATIC_MAX_ELEMENTS, STATIC_MAX_WORKERS,
    qadam_worker_pass_model, qadam_set_moment_rates, qadam_set_regularization,
    qadam_poll_status, qadam_profile_enable, qadam_profile_read, KERNEL_NAMES, qadam_launch_count, qadam_destroy, qadam_strerror,
)
from .adamw import AdamW, GradNorm  # noqa: F401
from .embedding import embedding_grad, embedding_lookup, held_lookup  # noqa: F401
from .norm import Normed, layer_norm, layer_norm_grad  # noqa: F401
from .int8 import Int8Rows, held_matmul, held_rows, int8_matmul, quantize_columns, quantize_rows  # noqa: F401
