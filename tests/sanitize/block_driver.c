/* The host side of qvggt_heads_norm_rope, qvggt_attention and qvggt_residual_norm under sanitizers, as abi_driver.c has the other entry points': sizes at the ends of their ranges, which are answered before
 * the first HIP call; the "device" pointers are never dereferenced. */
#include <limits.h>
#include <stdint.h>
#include <stdio.h>
#include "qvggt.h"

static int failures = 0;
static void expect(int got, int want, int line)
{
    if (got != want) {
        fprintf(stderr, "line %d: %d (%s), expected %d\n", line, got, qvggt_status_string(got), want);
        ++failures;
    }
}
#define EXPECT(call, want) expect(call, want, __LINE__)

int main(void)
{
    void *dev = (void *)(uintptr_t)0x7f0000000000ull, *other = (char *)dev + 4096;
    const int n[] = {INT_MIN, -1, 0, 1, 31, 32, 33, 128, 65535, 65536, 1 << 23, 1 << 30, INT_MAX};
    const unsigned many = sizeof n / sizeof *n;
    size_t sink = 0;
    for (unsigned a = 0; a < many; ++a)
        for (unsigned b = 0; b < many; ++b)
            for (unsigned c = 0; c < many; ++c) {
                for (unsigned e = 0; e < many; e += 3) {
                    sink += qvggt_attention_workspace_bytes(n[c], n[a], n[b], n[c], n[e], n[e], 64);
                    sink += qvggt_attention_workspace_bytes(4, n[a], n[b], n[c], n[e], 1, 128);
                }
                /* null operands: whatever the sizes, nothing is launched */
                int s = qvggt_attention(NULL, dev, dev, QVGGT_BF16, n[a], n[b], 64, 64, 64, 1, 1, 64, 1.0f, 1, dev, dev, NULL, n[c], n[c], n[b], dev, dev, SIZE_MAX, NULL);
                if (s != QVGGT_OK && s != QVGGT_ERR_SHAPE && s != QVGGT_ERR_NULL) expect(s, QVGGT_ERR_NULL, __LINE__);
                s = qvggt_heads_norm_rope(NULL, dev, QVGGT_F32, n[a], LLONG_MAX - 3, LLONG_MAX - 3, n[b], n[c], 128, QVGGT_NORM_RMS, 0.0f, NULL, NULL, NULL, NULL, dev, n[b], 128, 64, NULL, 4, NULL, dev, dev,
                                          LLONG_MAX - 3, LLONG_MAX - 3, NULL);
                if (s != QVGGT_OK && s != QVGGT_ERR_SHAPE && s != QVGGT_ERR_NULL) expect(s, QVGGT_ERR_NULL, __LINE__);
                s = qvggt_residual_norm(NULL, QVGGT_BF16, dev, QVGGT_F32, n[a], n[b], QVGGT_NORM_NONE, NULL, NULL, NULL, dev, QVGGT_NORM_LAYER, NULL, NULL, NULL, NULL, QVGGT_F32, n[c], LLONG_MAX - 3, NULL,
                                        1e-6f, other, NULL, QVGGT_BF16, NULL);
                if (s != QVGGT_OK && s != QVGGT_ERR_SHAPE && s != QVGGT_ERR_NULL) expect(s, QVGGT_ERR_NULL, __LINE__);
            }
    EXPECT(qvggt_attention(dev, dev, dev, QVGGT_F32, 4, 4, 64, 64, 64, 1, 1, 64, 1.0f, 1, dev, dev, NULL, 1, 4, 4, dev, dev, 0, NULL), QVGGT_ERR_DTYPE);
    EXPECT(qvggt_attention(dev, dev, dev, QVGGT_BF16, 1, 1 << 20, 64, 64, 64, 1, 1, 64, 1.0f, 1, dev, dev, NULL, 1, 1, 1 << 20, other, dev, 15, NULL), QVGGT_ERR_WORKSPACE);
    EXPECT(qvggt_residual_norm(dev, QVGGT_BF16, dev, QVGGT_BF16, 4, 64, 0, NULL, NULL, NULL, NULL, 0, NULL, NULL, NULL, NULL, 0, 0, 0, NULL, 0.0f, other, other, QVGGT_BF16, NULL), QVGGT_ERR_ARG);
    printf("%d mismatches (%zu)\n", failures, sink & 1);
    return failures != 0;
}
