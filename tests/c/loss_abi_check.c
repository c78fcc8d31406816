/* Plain C99 translation unit against cnr_loss.h: the header is valid C, every entry point links, and what can be
 * refused without a GPU is.  Built and run by tests/test_losses_host.py. */
#include <stdio.h>
#include <string.h>

#include "cnr_loss.h"

int main(void) {
    typedef void (*fn)(void);
    const fn exports[] = {(fn)cnr_loss_state_floats, (fn)cnr_loss_workspace_bytes, (fn)cnr_vocabulary_loss, (fn)cnr_vocabulary_loss_backward, (fn)cnr_top_logits};
    size_t i, n_exports = sizeof(exports) / sizeof(exports[0]);
    cnr_vocabulary v;
    cnr_targets t;
    for (i = 0; i < n_exports; ++i)
        if (!exports[i]) return 10;
    memset(&v, 0, sizeof v);
    memset(&t, 0, sizeof t);
    t.top = t.token_stride = 1;
    if (cnr_loss_state_floats(10, 3) != 100 || cnr_loss_state_floats(0, 1) != 0) return 11;
    if (cnr_loss_workspace_bytes(0, 10, 10, CNR_FLOAT_F32, 1, CNR_FLOAT_F32) != 0) return 12;
    if (cnr_vocabulary_loss(NULL, &v, &t, NULL, NULL, NULL, 0, NULL) != CNR_E_INVALID) return 13;
    if (cnr_vocabulary_loss_backward(NULL, &v, &t, NULL, NULL, NULL, 0, NULL, CNR_FLOAT_F32, 0, 0, NULL, 0, NULL) != CNR_E_INVALID) return 14;
    if (cnr_top_logits(NULL, NULL, 0, CNR_FLOAT_F32, 0, 0, 0, NULL, NULL, NULL, NULL) != CNR_E_INVALID) return 15;
    printf("abi ok: %u exports\n", (unsigned)n_exports);
    return 0;
}
