"""MI355X (gfx950) kernels for the memory-budgeted CNN training step of
SuperNeurons (arXiv 1801.04380): convolution forward / backward with an explicit
workspace budget (Sec. 3.5), the planner that picks the fastest algorithm that
fits, the cheap layers recomputation replays (Sec. 3.4), and layers along token
sequences (include/sn_seq.h: short causal convolution, norm of heads with the
position rotation, selective state space scan).

This package is a thin binding over the C ABI in include/sn.h and include/sn_seq.h: every function
here only marshals arguments; all arithmetic runs in the HIP library.
"""
from .api import *  # noqa: F401,F403
from .seq import *  # noqa: F401,F403
from .api import __all__ as _api_all
from .seq import __all__ as _seq_all

__all__ = _api_all + _seq_all
