"""Rules of the feed-forward kernels that no result shows, checked on their sources."""
from test_kernel_sources import _code

FILES = ("rms_norm.cu", "gated_ffn.cu", "lora.cu", "tile_gemm.cuh", "skinny_gemm.cuh")


def test_no_read_only_loads_in_chained_kernels():
    """A chained kernel runs while the launch before it writes what it will read: a load through the read-only path may be moved above
    the wait, and asks for memory that nobody writes while the kernel runs."""
    for name in FILES:
        code = _code(name)
        assert "__ldg" not in code and "ld.global.nc" not in code and "__restrict__" not in code, name
