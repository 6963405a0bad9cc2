"""B200-native FP64 GEMM ``C += A @ B`` (row-major) behind the C ABI of ``libdgemm``.

The Python layer only marshals arguments; every step of the computation runs in the CUDA
kernels of ``csrc/``. The library is loaded lazily on first use and its absence is an error.
"""
from .binding import (  # noqa: F401
    DGEMM_OK,
    DGEMM_OP_N,
    DGEMM_OP_T,
    DGEMM_VARIANT_AUTO,
    DGEMM_VARIANT_GENERIC,
    DGEMM_VARIANT_NAIVE,
    DGEMM_VARIANT_TMA,
    DGEMM_VARIANT_TMA_WS,
    DGEMM_VARIANT_GENERIC_WS,
    DGEMM_VARIANT_TMA_CLUSTER,
    DGEMM_VARIANT_GENERIC_CLUSTER,
    DGEMM_VARIANT_SMEM,
    DGEMM_VARIANT_TMA_DFMA,
    DGEMM_VARIANT_GENERIC_DFMA,
    DGEMM_VARIANT_TMA_WS_BULK,
    DGEMM_ERR_VARIANT,
    DGEMM_TEST_NO_C_PREFETCH,
    DGEMM_TEST_NO_BLOCKED_B,
    DGEMM_TEST_TALL_TILES,
    DGEMM_TEST_SMALL_WARP_TILES,
    DGEMM_TEST_NO_PACKING,
    DGEMM_TEST_WS_TWO_CTAS,
    DGEMM_TEST_NO_CLUSTER,
    DGEMM_TEST_DROP_LOADS,
    DgemmError,
    dgemm_f64,
    dgemm_f64_ex,
    dgemm_f64_host,
    dgemm_f64_raw,
    dgemm_f64_static_ws,
    dgemm_fp64_fma_probe,
    dgemm_fp64_peak_probe,
    dgemm_last_device_status,
    dgemm_launch_count,
    dgemm_plan,
    dgemm_release_scratch,
    dgemm_selftest_wait_timeout,
    dgemm_set_split_k,
    dgemm_set_test_flags,
    dgemm_set_test_wait_limit,
    dgemm_set_variant,
    dgemm_strerror,
    dgemm_version,
    HGEMM_ACT_GELU,
    HGEMM_ACT_GELU_TANH,
    HGEMM_ACT_NONE,
    HGEMM_ACT_RELU,
    HGEMM_ACT_SILU,
    HGEMM_TYPE_BF16,
    HGEMM_TYPE_F16,
    HGEMM_TYPE_F32,
    hgemm_last_device_status,
    hgemm_plan,
    hgemm_set_test_drop_loads,
    lib_path,
    load_library,
    sgemm_f32,
    sgemm_last_device_status,
)


def __getattr__(name):
    """hgemm_epilogue, qgemm_epilogue, layernorm_fwd, rmsnorm_fwd, dropout_fwd and the like: loaded on first use."""
    from . import binding
    if name in binding.MARSHALLED:
        value = globals()[name] = getattr(binding, name)
        return value
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
