/*
 * Host-only driver for the sanitizer build of the argument validation of the
 * products in 4 bits and of the heads' norms (tests/test_sanitizers_mx4.py builds
 * tcu_mx4_abi.cpp, tcu_heads_abi.cpp and tcu_abi.cpp with AddressSanitizer and
 * UndefinedBehaviorSanitizer and links them here).
 *
 * Every call uses fake, never-dereferenced device addresses and is built to be
 * rejected by validation, except the calls marked "valid", which reach the device
 * query and must report TCU_ERR_NO_DEVICE: the driver runs only on a machine with
 * no GPU.  Exit status 0 when every status is the expected one.
 */
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include "tcu.h"

static int failures = 0;

static void expect(const char *what, long long got, long long want)
{
    if (got != want) {
        fprintf(stderr, "%s: got %lld, want %lld\n", what, got, want);
        ++failures;
    }
}

#define P(i) ((void *)(uintptr_t)(0x100000000u + ((uint64_t)(i) << 42)))
#define BIG ((int64_t)1 << 62)
#define DIM TCU_MAX_MX4_DIM

/* (the macro is for sizes in range) */
static int64_t row(int64_t n)
{
    return n >= 0 && n <= DIM ? TCU_MX4_ROW_BYTES(n) : 64;
}

static int quant(int64_t rows, int64_t cols, int64_t ldx, int64_t ldq, int64_t lds)
{
    return tcu_mx4_quant(P(0), ldx, P(1), ldq, P(2), lds, P(3), row(rows), P(4), cols,
                         rows, cols, TCU_ELEM_BF16, 0);
}

static int dequant(int64_t rows, int64_t cols, int64_t ldq, int64_t ldy)
{
    return tcu_mx4_dequant(P(0), ldq, P(1), rows, P(2), ldy, rows, cols, TCU_ELEM_F32, 0);
}

static int gemm(int64_t M, int64_t K, int64_t N, int64_t lda, int64_t ldas, int64_t ldc)
{
    return tcu_mx4_gemm(P(0), lda, P(1), ldas, P(2), row(K), P(3), N, P(4), ldc, P(5),
                        M, K, N, 0, TCU_ELEM_F32, 0);
}

static int linear(int64_t M, int64_t K, int64_t N, int64_t ldx)
{
    return tcu_mx4_linear(P(0), ldx, P(2), row(K), P(3), N, P(4), N, P(5), M, K, N,
                          TCU_ACCUMULATE, TCU_ELEM_F16, TCU_ELEM_F16, 0);
}

static int heads(int64_t T, int64_t hq, int64_t hk, int64_t dim, int64_t rot, int64_t ld, int64_t hd,
                 float eps)
{
    return tcu_qk_norm(P(0), ld, hd, P(1), ld, hd, P(2), P(3), P(4), P(5), P(6), ld, hd, P(7), ld,
                       hd, T, hq, hk, dim, rot, eps, 0, TCU_ELEM_BF16, 0);
}

static int heads_grad(int64_t T, int64_t hq, int64_t hk, int64_t dim, int64_t ld, int64_t hd)
{
    return tcu_qk_norm_grad(P(0), ld, hd, P(1), ld, hd, P(2), ld, hd, P(3), ld, hd, P(4), P(5), P(6),
                            P(7), P(8), ld, hd, P(9), ld, hd, P(10), P(11), P(12), T, hq, hk, dim,
                            0, 1e-5f, 0, TCU_ELEM_F32, 0);
}

int main(void)
{
    const int64_t odd[] = {-1, -BIG, BIG, INT64_MAX, INT64_MIN, DIM + 1};
    const int n = sizeof odd / sizeof odd[0];

    expect("quant valid", quant(10, 200, 200, 128, 10), TCU_ERR_NO_DEVICE);
    expect("quant largest", quant(DIM, 200, 200, 128, DIM), TCU_ERR_NO_DEVICE);
    expect("quant too many", quant(DIM, DIM, DIM, DIM / 2, DIM), TCU_ERR_SHAPE);
    expect("quant none", quant(0, 200, 200, 128, 10), TCU_OK);
    expect("dequant valid", dequant(10, 200, 128, 200), TCU_ERR_NO_DEVICE);
    expect("gemm valid", gemm(10, 200, 30, 128, 10, 30), TCU_ERR_NO_DEVICE);
    expect("gemm far scales", gemm(10, 200, 30, 128, (int64_t)1 << 36, 30), TCU_ERR_NO_DEVICE);
    expect("gemm largest", gemm(DIM, 128, 64, 64, DIM, 64), TCU_ERR_NO_DEVICE);
    expect("gemm too long", gemm(DIM, DIM, 1, DIM / 2, DIM, 1), TCU_ERR_SHAPE);
    expect("gemm too large", gemm(DIM, 128, DIM, 64, DIM, DIM), TCU_ERR_SHAPE);
    expect("linear valid", linear(10, 200, 30, 200), TCU_ERR_NO_DEVICE);
    expect("heads valid", heads(7, 4, 2, 64, 64, 256, 64, 0.f), TCU_ERR_NO_DEVICE);
    expect("heads by head", heads(7, 4, 2, 64, 64, 64, 448, 0.f), TCU_ERR_NO_DEVICE);
    expect("heads most", heads(TCU_MAX_RECT_DIM, 4, 4, 64, 2, 256, 64, 1.f), TCU_ERR_NO_DEVICE);
    expect("heads too many", heads(TCU_MAX_RECT_DIM, TCU_MAX_HEADS, 1, 1024, 0, 1 << 26, 1024, 1.f),
           TCU_ERR_SHAPE);
    expect("heads far apart", heads(TCU_MAX_RECT_DIM, 65536, 2, 64, 0, 64, (int64_t)1 << 39, 1.f),
           TCU_ERR_SHAPE);
    expect("heads eps", heads(7, 4, 2, 64, 64, 256, 64, NAN), TCU_ERR_SHAPE);
    expect("grad valid", heads_grad(7, 4, 2, 64, 256, 64), TCU_ERR_NO_DEVICE);
    expect("grad of nothing", heads_grad(0, 4, 2, 64, 256, 64), TCU_ERR_NO_DEVICE);
    expect("work", tcu_mx4_work(DIM, DIM, DIM), -1);
    for (int i = 0; i < n; ++i) {
        const int64_t v = odd[i];
        expect("quant rows", quant(v, 200, 200, 128, 10), TCU_ERR_SHAPE);
        expect("quant cols", quant(10, v, 200, 128, 10), TCU_ERR_SHAPE);
        expect("dequant rows", dequant(v, 200, 128, 200), TCU_ERR_SHAPE);
        expect("dequant cols", dequant(10, v, 128, 200), TCU_ERR_SHAPE);
        expect("gemm M", gemm(v, 200, 30, 128, 10, 30), TCU_ERR_SHAPE);
        expect("gemm K", gemm(10, v, 30, 128, 10, 30), TCU_ERR_SHAPE);
        expect("gemm N", gemm(10, 200, v, 128, 10, 30), TCU_ERR_SHAPE);
        expect("linear M", linear(v, 200, 30, 200), TCU_ERR_SHAPE);
        expect("linear K", linear(10, v, 30, 200), TCU_ERR_SHAPE);
        expect("linear N", linear(10, 200, v, 200), TCU_ERR_SHAPE);
        expect("work M", tcu_mx4_work(v, 1, 1), -1);
        expect("work K", tcu_mx4_work(1, v, 1), -1);
        expect("work N", tcu_mx4_work(1, 1, v), -1);
        expect("heads hq", heads(7, v, 2, 64, 64, 256, 64, 0.f), TCU_ERR_SHAPE);
        expect("heads dim", heads(7, 4, 2, v, 64, 256, 64, 0.f), TCU_ERR_SHAPE);
        expect("heads rot", heads(7, 4, 2, 64, v, 256, 64, 0.f), TCU_ERR_SHAPE);
        expect("grad hk", heads_grad(7, 4, v, 64, 256, 64), TCU_ERR_SHAPE);
        expect("grad work", tcu_qk_norm_grad_work(7, v, 2, 64), -1);
        if (v == DIM + 1) continue;   /* fine as pitches and tokens */
        expect("quant ldx", quant(10, 200, v, 128, 10), TCU_ERR_SHAPE);
        expect("quant ldq", quant(10, 200, 200, v, 10), TCU_ERR_SHAPE);
        expect("quant lds", quant(10, 200, 200, 128, v), TCU_ERR_SHAPE);
        expect("dequant ldy", dequant(10, 200, 128, v), TCU_ERR_SHAPE);
        expect("gemm lda", gemm(10, 200, 30, v, 10, 30), TCU_ERR_SHAPE);
        expect("gemm ldas", gemm(10, 200, 30, 128, v, 30), TCU_ERR_SHAPE);
        expect("gemm ldc", gemm(10, 200, 30, 128, 10, v), TCU_ERR_SHAPE);
        expect("linear ldx", linear(10, 200, 30, v), TCU_ERR_SHAPE);
        expect("heads tokens", heads(v, 4, 2, 64, 64, 256, 64, 0.f), TCU_ERR_SHAPE);
        expect("heads ld", heads(7, 4, 2, 64, 64, v, 64, 0.f), TCU_ERR_SHAPE);
        expect("heads hd", heads(7, 4, 2, 64, 64, 256, v, 0.f), TCU_ERR_SHAPE);
        expect("grad ld", heads_grad(7, 4, 2, 64, v, 64), TCU_ERR_SHAPE);
        expect("grad hd", heads_grad(7, 4, 2, 64, 256, v), TCU_ERR_SHAPE);
    }
    printf("%d failures\n", failures);
    return failures != 0;
}
