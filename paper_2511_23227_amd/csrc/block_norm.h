// Arguments of the kernels between two blocks of a residual network (block_norm.hip), checked by the entry points; not part of the C ABI.
#pragma once

#include "pcpp_internal.h"

namespace pcpp {

struct ActOut { int8_t *q; uint8_t *e; };                         // 8-bit rows to write (q NULL: none)
struct ActIn { const int8_t *q; const uint8_t *e; };

struct BlockNormFwd {
    const void *x, *f, *gate;
    const float *w_post, *w_pre;
    void *r, *h;
    ActOut f_codes, h_codes;
    int64_t n, ld_f, ld_gate;
    int c, gate_cols, post, pre;
    float scale, eps, inv_c;
};

struct BlockNormBwd {
    const void *dr, *dh, *r, *f, *gate;
    ActIn f_codes;
    const float *w_post, *w_pre;
    void *dx, *df, *dgate;
    float *dw_post, *dw_pre, *part;
    int64_t n, ld_f, ld_gate;
    int c, gate_cols, post, pre;
    float scale, eps, inv_c;
};

int block_norm_fwd(const BlockNormFwd &a, int stream_dtype, int dtype, hipStream_t stream);
size_t block_norm_bwd_workspace_bytes(int64_t n, int c);
int block_norm_bwd(const BlockNormBwd &a, int stream_dtype, int dtype, hipStream_t stream);

}  // namespace pcpp
