/*
 * Host-only driver for the sanitizer build of the layer operators' argument
 * validation (tests/test_sanitizers_layer.py builds tcu_layer_abi.cpp and
 * tcu_abi.cpp with AddressSanitizer and UndefinedBehaviorSanitizer and links
 * them here).
 *
 * Every call uses fake, never-dereferenced device addresses and is built to
 * be rejected by validation, except the calls marked "valid", which reach the
 * device query and must report TCU_ERR_NO_DEVICE: the driver runs only on a
 * machine with no GPU.  Exit status 0 when every status is the expected one.
 */
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

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
#define ROWS TCU_MAX_RECT_DIM
#define DIM TCU_MAX_ADAPTED_DIM

static int norm(int64_t rows, int64_t cols, int64_t ld, float eps, int elem, void *h, int64_t ldh)
{
    return tcu_rms_norm(P(0), ld, P(1), ld, P(2), h, ldh, P(4), ld, P(5), ld, P(6), rows, cols, eps,
                        elem, 0);
}

static int norm_grad(int64_t rows, int64_t cols, int64_t ld, void *dx, void *work)
{
    return tcu_rms_norm_grad(P(0), ld, P(1), ld, P(2), P(3), ld, dx, ld, P(5), work, rows, cols,
                             1e-5f, TCU_ELEM_BF16, 0);
}

static int adapter(int64_t M, int64_t K, int64_t N, int64_t r, int64_t G)
{
    return tcu_adapter_gemm(P(0), K, P(1), N, P(2), P(3), P(4), P(5), P(6), N, P(7), M, K, N, r, G,
                            TCU_BF16_BF16, 0);
}

static int adapter_q8(int64_t M, int64_t K, int64_t N, int64_t r, int64_t G, int64_t ldwq)
{
    return tcu_adapter_gemm_q8(P(8), K, P(9), P(1), ldwq, P(10), P(0), K, P(2), P(3), P(4), P(5),
                               P(6), N, P(7), M, K, N, r, G, 0);
}

static int adapter_grad(int64_t M, int64_t K, int64_t N, int64_t r, int64_t G, void *dB)
{
    return tcu_adapter_grad(P(0), K, P(1), N, P(2), P(3), P(4), P(5), P(6), dB, P(8), M, K, N, r, G,
                            TCU_ELEM_F16, 0);
}

static int input_grad(int64_t M, int64_t K, int64_t N, int64_t r, int64_t G)
{
    return tcu_adapter_input_grad(P(0), N, P(1), K, P(2), P(3), P(4), P(5), P(6), K, P(7), M, K, N,
                                  r, G, TCU_F16_F32, 0);
}

int main(void)
{
    /* norm: sizes and pitches near the limits, views of one array */
    expect("norm valid", norm(10, 64, 64, 1e-5f, 2, P(3), 64), TCU_ERR_NO_DEVICE);
    expect("norm in place", norm(10, 64, 64, 0.f, 2, P(0), 64), TCU_ERR_NO_DEVICE);
    expect("norm other pitch", norm(10, 64, 64, 0.f, 2, P(0), 72), TCU_ERR_OVERLAP);
    expect("norm interleaved", norm(10, 32, 64, 0.f, 2, (char *)P(0) + 64, 64),
           TCU_ERR_NO_DEVICE);
    expect("norm rows", norm(-BIG, 64, 64, 0.f, 2, P(3), 64), TCU_ERR_SHAPE);
    expect("norm cols", norm(10, BIG, BIG, 0.f, 2, P(3), BIG), TCU_ERR_SHAPE);
    expect("norm extent", norm(ROWS, ROWS, ROWS, 0.f, 0, P(3), ROWS), TCU_ERR_SHAPE);
    expect("norm pitch", norm(ROWS, 64, ((int64_t)1 << 40) - 1, 0.f, 0, P(3), 64), TCU_ERR_SHAPE);
    expect("norm eps", norm(10, 64, 64, NAN, 2, P(3), 64), TCU_ERR_SHAPE);
    expect("norm elem", norm(10, 64, 64, 0.f, 0x7fffffff, P(3), 64), TCU_ERR_UNSUPPORTED);
    expect("norm empty", norm(0, 64, 64, 0.f, 1, P(3), 64), TCU_OK);
    expect("norm grad valid", norm_grad(10, 64, 64, P(4), P(6)), TCU_ERR_NO_DEVICE);
    expect("norm grad in place", norm_grad(10, 64, 64, P(0), P(6)), TCU_ERR_NO_DEVICE);
    expect("norm grad long", norm_grad(4, ROWS, ROWS, P(4), P(6)), TCU_ERR_NO_DEVICE);
    expect("norm grad work", norm_grad(10, 64, 64, P(4), (char *)P(4) + 16), TCU_ERR_OVERLAP);
    expect("norm grad align", norm_grad(10, 64, 64, P(4), (char *)P(6) + 4), TCU_ERR_ALIGN);
    expect("norm grad size", tcu_rms_norm_grad_work(ROWS, ROWS), 512 * ROWS * 4);
    expect("norm grad size -", tcu_rms_norm_grad_work(-BIG, 4), -1);

    /* adapters: every size at its limit */
    expect("adapter valid", adapter(10, 64, 96, 16, 3), TCU_ERR_NO_DEVICE);
    expect("adapter long", adapter(1, DIM, DIM, 128, 1), TCU_ERR_SHAPE);   /* W is 2^49 bytes */
    expect("adapter tall", adapter(ROWS, 256, 256, 16, 1), TCU_ERR_NO_DEVICE);
    expect("adapter none", adapter(0, 64, 96, 16, 3), TCU_OK);
    expect("q8 valid", adapter_q8(10, 64, 96, 16, 3, 96), TCU_ERR_NO_DEVICE);
    expect("q8 2^17", adapter_q8(10, 1 << 17, 96, 16, 3, 96), TCU_ERR_SHAPE);
    expect("q8 pitch", adapter_q8(10, 64, 96, 16, 3, BIG), TCU_ERR_SHAPE);
    expect("grad valid", adapter_grad(10, 64, 96, 16, 3, P(7)), TCU_ERR_NO_DEVICE);
    expect("grad overlap", adapter_grad(10, 64, 96, 16, 3, (char *)P(6) + 64), TCU_ERR_OVERLAP);
    expect("grad no adapters", adapter_grad(10, 64, 96, 16, 0, P(7)), TCU_OK);
    expect("input grad valid", input_grad(10, 64, 96, 16, 3), TCU_ERR_NO_DEVICE);
    {
        const int64_t sizes[][5] = {
            {ROWS, 1 << 18, 1 << 18, 16, 4}, {ROWS, DIM, DIM, 16, 0}, {ROWS, DIM, DIM, 128, 65536},
            {BIG, 64, 64, 16, 1}, {-BIG, 64, 64, 16, 1}, {64, -BIG, 64, 16, 1},
            {64, 64, BIG, 16, 1}, {64, 64, 64, BIG, 1}, {64, 64, 64, -BIG, 1},
            {64, 64, 64, 16, BIG}, {64, 64, 64, 16, -BIG}, {1, DIM, 1, 128, 65536}};
        for (size_t i = 0; i < sizeof(sizes) / sizeof(sizes[0]); ++i) {
            const int64_t *s = sizes[i];
            expect("work size", tcu_adapter_work(s[0], s[1], s[2], s[3], s[4]), -1);
            expect("adapter size", adapter(s[0], s[1], s[2], s[3], s[4]), TCU_ERR_SHAPE);
            expect("q8 size", adapter_q8(s[0], s[1], s[2], s[3], s[4], s[2]), TCU_ERR_SHAPE);
            expect("grad size", adapter_grad(s[0], s[1], s[2], s[3], s[4], P(7)), TCU_ERR_SHAPE);
            expect("input grad size", input_grad(s[0], s[1], s[2], s[3], s[4]), TCU_ERR_SHAPE);
        }
    }

    /* clipping: the ranges' table with many tensors, out of order */
    {
        enum { T = 1000 };
        const void **g = malloc(T * sizeof(*g));
        void **o = malloc(T * sizeof(*o));
        int64_t *n = malloc(T * sizeof(*n));
        int32_t *e = malloc(T * sizeof(*e));
        for (int i = 0; i < T; ++i) {
            const int at = (i * 7919) % T;
            g[i] = (const char *)P(0) + (int64_t)at * 4096;
            o[i] = i % 3 ? (void *)((char *)P(1) + (int64_t)at * 4096) : (void *)g[i];
            n[i] = i % 5 == 4 ? 0 : 1 + i;
            e[i] = i % 3;
        }
        expect("clip valid", tcu_clip_grads(g, o, n, e, T, 1.f, P(2), P(3), 0), TCU_ERR_NO_DEVICE);
        n[1] = 4096;
        expect("clip overlap", tcu_clip_grads(g, o, n, e, T, 1.f, P(2), P(3), 0), TCU_ERR_OVERLAP);
        n[1] = BIG;
        expect("clip count", tcu_clip_grads(g, o, n, e, T, 1.f, P(2), P(3), 0), TCU_ERR_SHAPE);
        n[1] = 2;
        e[T - 1] = 3;
        expect("clip elem", tcu_clip_grads(g, o, n, e, T, 1.f, P(2), P(3), 0), TCU_ERR_UNSUPPORTED);
        expect("clip tensors", tcu_clip_grads(g, o, n, e, -BIG, 1.f, P(2), P(3), 0), TCU_ERR_SHAPE);
        expect("clip tensors", tcu_clip_grads(g, o, n, e, BIG, 1.f, P(2), P(3), 0), TCU_ERR_SHAPE);
        expect("clip max", tcu_clip_grads(g, o, n, e, 1, NAN, P(2), P(3), 0), TCU_ERR_SHAPE);
        expect("clip none", tcu_clip_grads(0, 0, 0, 0, 0, 1.f, P(2), P(3), 0), TCU_ERR_NO_DEVICE);
        free(g);
        free(o);
        free(n);
        free(e);
    }

    printf("%d failures\n", failures);
    return failures != 0;
}
