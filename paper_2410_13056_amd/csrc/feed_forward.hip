// A gated feed-forward part in 8 bits: the norm, the gated projections and the output projection one after the other, what passes
// between them in the caller's workspace.  Four launches (three for one or two tokens) for one call, since the host bounds a small
// part: 13 tokens of 102, 2 x 2491 take 17.7 us, as three calls from Python 29.6.
#include "int8_rows.h"

namespace {

struct Parts {
    cmpq_norm_job norm;
    cmpq_int8_job gated, down;
    void *ws;          // of the last product
    size_t ws_bytes, bytes;
};

Parts parts_of(const cmpq_int8_feed_forward_job &j, void *ws) {
    Parts p = {};
    WsCarver c(ws);
    const size_t m = (size_t)j.m, stream = j.add.ptr ? m * (size_t)j.d * dtype_bytes(j.X.dtype) : 0;
    int8_t *codes = c.take<int8_t>(cmpq_int8_weight_bytes(j.m, j.d));
    float *scale = c.take<float>(m);
    char *sum = c.take<char>(stream), *hidden = c.take<char>(m * (size_t)j.d_ff * dtype_bytes(j.hidden_dtype));
    p.ws = c.take<char>(0);
    p.ws_bytes = cmpq_ws_int8_product(j.d_ff, j.m);
    c.take<char>(p.ws_bytes);
    p.bytes = c.need();
    p.norm = {j.X, j.add, j.gain, {}, {}, codes, scale, j.m, j.d, j.eps, j.status};
    if (j.add.ptr) p.norm.S = {sum, j.d, j.X.dtype};
    const cmpq_rows residual = j.add.ptr ? p.norm.S : j.X;
    p.gated.x_codes = codes, p.gated.x_scale = scale, p.gated.m = j.m, p.gated.d_in = j.d, p.gated.d_out = j.d_ff, p.gated.gated = 1;
    p.gated.codes = j.gate_up_codes, p.gated.scale = j.gate_up_scale, p.gated.activation = j.activation;
    p.gated.Y = hidden, p.gated.y_dtype = j.hidden_dtype, p.gated.ldy = j.d_ff;
    p.down.X = hidden, p.down.x_dtype = j.hidden_dtype, p.down.m = j.m, p.down.d_in = j.d_ff, p.down.ldx = j.d_ff, p.down.d_out = j.d;
    p.down.codes = j.down_codes, p.down.scale = j.down_scale, p.down.status = j.status;
    p.down.residual = residual.ptr, p.down.r_dtype = residual.dtype, p.down.ldr = residual.ld;
    p.down.Y = j.Y.ptr, p.down.y_dtype = j.Y.dtype, p.down.ldy = j.Y.ld;
    return p;
}

// The largest sizes that the parts are asked for stay within size_t.
int check_sizes(const cmpq_int8_feed_forward_job *j) {
    if (!j || j->m < 0 || j->d < 1 || j->d_ff < 1 || !serving_dtype(j->X.dtype) || !serving_dtype(j->hidden_dtype)) return CMPQ_EINVAL;
    return j->m < (1 << 24) && j->d <= kMostDepth && j->d_ff <= kMostDepth ? CMPQ_OK : CMPQ_ESHAPE;
}

}  // namespace

extern "C" size_t cmpq_int8_feed_forward_workspace(const cmpq_int8_feed_forward_job *j) {
    return check_sizes(j) ? 0 : parts_of(*j, nullptr).bytes;
}

extern "C" int cmpq_int8_feed_forward(const cmpq_int8_feed_forward_job *j, void *ws, size_t ws_bytes, void *stream) {
    if (int rc = check_sizes(j)) return rc;
    Parts p = parts_of(*j, reinterpret_cast<void *>(256));  // with a workspace's place, whether there is one or not
    if (int rc = cmpq_check_rms_norm(&p.norm)) return rc;
    if (int rc = cmpq_check_int8_product(&p.gated)) return rc;
    if (int rc = cmpq_check_int8_product(&p.down)) return rc;
    if (j->m == 0) return CMPQ_OK;
    if (!ws || reinterpret_cast<uintptr_t>(ws) % 256 || ws_bytes < p.bytes) return CMPQ_EWORKSPACE;
    p = parts_of(*j, ws);
    if (int rc = cmpq_rms_norm(&p.norm, stream)) return rc;
    if (int rc = cmpq_int8_product_job(&p.gated, nullptr, 0, stream)) return rc;
    return cmpq_int8_product_job(&p.down, p.ws, p.ws_bytes, stream);
}
