/* Plain C99 translation unit against cnr_lm.h: the header is valid C, every entry point links, and what can be
 * refused without a GPU is.  Built and run by tests/test_language_host.py. */
#include <stdio.h>
#include <string.h>

#include "cnr_lm.h"

int main(void) {
    typedef void (*fn)(void);
    const fn exports[] = {(fn)cnr_block_row_bytes, (fn)cnr_block_scale_stride, (fn)cnr_block_scale_count, (fn)cnr_quantize_blocks,
                          (fn)cnr_block_product_workspace_bytes, (fn)cnr_block_product, (fn)cnr_count_tokens, (fn)cnr_adjust_logits};
    size_t i, n_exports = sizeof(exports) / sizeof(exports[0]);
    cnr_adjustments none;
    for (i = 0; i < n_exports; ++i)
        if (!exports[i]) return 10;
    memset(&none, 0, sizeof none);
    if (cnr_block_row_bytes(0) != 0 || cnr_block_row_bytes(1) != 128 || cnr_block_row_bytes(129) != 256) return 11;
    if (cnr_block_scale_stride(129, CNR_BLOCK_ROW) != 256 || cnr_block_scale_stride(129, CNR_BLOCK_TILE) != 2) return 12;
    if (cnr_block_scale_count(5000000000u, 300, CNR_BLOCK_ROW) != 3u * 5000000000u) return 13;
    if (cnr_quantize_blocks(NULL, NULL, CNR_FLOAT_F32, 0, 0, 0, CNR_BLOCK_ROW, CNR_SCALE_E8M0, NULL, NULL, NULL, NULL, NULL) != CNR_E_INVALID) return 14;
    if (cnr_block_product(NULL, NULL, NULL, CNR_BLOCK_ROW, 0, NULL, NULL, CNR_BLOCK_ROW, 0, 0, CNR_SCALE_E8M0, NULL, CNR_FLOAT_F32, 0, 0, NULL, NULL) != CNR_E_INVALID) return 15;
    if (cnr_count_tokens(NULL, NULL, NULL, 0, 0, NULL, 0, CNR_IDX_I64, NULL, NULL, 0, 0, 0, NULL) != CNR_E_INVALID) return 16;
    if (cnr_adjust_logits(NULL, NULL, 0, NULL, 0, CNR_FLOAT_F32, 0, 0, &none, NULL) != CNR_E_INVALID) return 17;
    printf("abi ok: %u exports\n", (unsigned)n_exports);
    return 0;
}
