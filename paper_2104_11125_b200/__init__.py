"""B200-native CLT-k compression step of ScaleCom (Algorithm 1): C-ABI CUDA library + thin binding.

`Context` is the compression step; `Operators` are the computations on either side of it for transformer learners."""
from .binding import Context, ScaleComError, lib, strerror  # noqa: F401
from .operators import Operators  # noqa: F401
from . import binding, operators, workloads  # noqa: F401
