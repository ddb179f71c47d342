"""B200-native PTS W8A8 linear layer (PTQ4VM, arXiv 2412.20386, Sec. 5.1).

The product is the C-ABI library declared in ``include/ptq_linear.h``; this
package holds its CUDA sources (``csrc/``), the build step (``build.py``), a thin
ctypes binding with the same entry points (``binding.py``) and the seeded
synthetic inputs (``workloads.py``).  The shared library is loaded on first use
and the binding raises if it is missing: there is no CPU fallback.

``block.py`` holds the operators between a block's linears (``include/ptq_block.h``), ``heads.py`` the recurrence of blocks with heads
(``include/ptq_heads.h``), ``fp8.py`` linears in block-scaled 8-bit floating point (``include/ptq_fp8.h``).
"""
from . import workloads  # noqa: F401
from .binding import (PtqError, PtqLinear, calibrate, calibrate_asym, calibrate_w4a4, search_act_step, library_path, load_library,  # noqa: F401
                      FLAG_FUSED_PROLOGUE, FLAG_CTA_PAIR)
from .block import (block_norm, block_norm_backward, gated_scan, gated_scan_backward, gated_scan_step, scan_history, short_conv,  # noqa: F401
                    short_conv_backward)
from .fp8 import fp8_device_status, fp8_linear, fp8_matmul, fp8_quantize, fp8_quantize_weight  # noqa: F401
from .heads import head_scan, head_scan_backward, head_scan_history, head_scan_step  # noqa: F401
