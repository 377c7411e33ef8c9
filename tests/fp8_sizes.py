"""Products that between them launch every kernel of zs_fp8_gemm and zs_fp8_gemm_bf16 on 256 compute units: (M, N, K, bytes of
workspace), the kernel's tile (tokens, features; none for the kernel of few tokens) and whether K is split.  Ragged on every side."""
WORKSPACE = 32 << 20
PRODUCTS = [((1, 200, 300, 0), None, False),
            ((16, 500, 1030, WORKSPACE), None, False),
            ((40, 300, 1000, 0), (64, 128), False),
            ((70, 130, 3000, WORKSPACE), (64, 128), True),
            ((700, 1030, 390, WORKSPACE), (64, 128), False),
            ((1030, 2050, 130, WORKSPACE), (128, 128), False),
            ((200, 4090, 4200, WORKSPACE), (128, 128), True),
            ((2050, 2050, 1000, 0), (256, 128), False),
            ((1030, 2050, 4200, WORKSPACE), (256, 128), True)]
