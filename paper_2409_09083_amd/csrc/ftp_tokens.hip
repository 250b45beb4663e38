// C ABI of the token block's operators: checks of the arguments, then the launches.
#include "ftp_tokens.h"

#include <cmath>

using namespace ftp;

namespace {

bool is_type(int32_t dtype) { return dtype == FTP_F32 || dtype == FTP_BF16; }

// FTP_OK if there is something to do; *nothing: an empty call, which is no error.  Strides are those that the pass uses: x and y, or x (not from a checkpoint: held), dy and dx.
int check(const ftp_norm_shape* s, bool back, bool held, bool* nothing)
{
    *nothing = false;
    if (!s || !is_type(s->dtype) || s->outer < 0 || s->inner < 0 || s->channels < 1 || !(s->eps >= 0)) return FTP_EINVAL;
    const int64_t* used[] = {held ? s->dy_stride : s->x_stride, back ? s->dy_stride : s->y_stride, back ? s->dx_stride : s->y_stride};
    bool rows = true;
    for (const int64_t* t : used) {
        if (t[0] < 0 || t[1] < 0 || t[2] < 0) return FTP_EINVAL;
        rows = rows && (t[2] == 1 || s->channels == 1);
    }
    if (s->outer == 0 || s->inner == 0) { *nothing = true; return FTP_OK; }
    if (s->outer > 0x7FFFFFFFll || s->inner > 0x7FFFFFFFll || s->outer * s->inner > 0x7FFFFFFFll) return FTP_EUNSUPPORTED;
    return rows || s->channels <= kNormMapChannels ? FTP_OK : FTP_EUNSUPPORTED;
}

int check(const ftp_checkpoint_shape* s)
{
    if (!s || !is_type(s->dtype) || s->rows < 0 || s->cols < 1 || s->stride < s->cols) return FTP_EINVAL;
    if (s->block != 32 && s->block != 64 && s->block != 128 && s->block != 256) return FTP_EUNSUPPORTED;
    if (s->cols > (1ll << 30)) return FTP_EUNSUPPORTED;
    return FTP_OK;
}

int check(const ftp_attention_shape* s)
{
    if (!s || !is_type(s->dtype) || s->batch < 0 || s->heads < 1 || s->kv_heads < 1 || s->heads % s->kv_heads || s->q_len < 0 || s->kv_len < 0 ||
        s->head_dim < 1 || !std::isfinite(s->scale)) return FTP_EINVAL;
    if (s->head_dim > 128) return FTP_EUNSUPPORTED;
    // rows and keys, with a block's overhang, are 32-bit numbers
    if ((double)s->q_len * (s->heads / s->kv_heads) > 2e9 || s->kv_len > 2000000000 || (double)s->batch * s->kv_heads > 2e9 || !attention_fits(*s)) return FTP_EUNSUPPORTED;
    return FTP_OK;
}

bool negative(const int64_t (&stride)[3]) { return stride[0] < 0 || stride[1] < 0 || stride[2] < 0; }

// ... and the strides that a pass uses (rows of a tile are fetched at offsets from its first one, where a negative one means no row).
int check(const ftp_attention_shape* s, bool back)
{
    const int rc = check(s);
    if (rc != FTP_OK) return rc;
    if (negative(s->q_stride) || negative(s->k_stride) || negative(s->v_stride) || negative(s->out_stride)) return FTP_EINVAL;
    if (back && (negative(s->dout_stride) || negative(s->dq_stride) || negative(s->dk_stride) || negative(s->dv_stride))) return FTP_EINVAL;
    return FTP_OK;
}

bool is_act(int32_t act) { return act >= FTP_ACT_NONE && act <= FTP_ACT_SILU; }

}  // namespace

extern "C" {

int ftp_norm_forward(const ftp_norm_shape* shape, const void* x, const void* gamma, const void* beta, void* y, float* mean, float* rstd, void* stream)
{
    bool nothing;
    const int rc = check(shape, false, false, &nothing);
    if (rc != FTP_OK || nothing) return rc;
    if (!x || !y) return FTP_EINVAL;
    norm_forward(*shape, x, gamma, beta, y, mean, rstd, (hipStream_t)stream);
    return launched();
}

int ftp_norm_workspace(const ftp_norm_shape* shape, size_t* bytes)
{
    if (!shape || shape->channels < 1 || !bytes) return FTP_EINVAL;
    *bytes = norm_workspace(*shape);
    return FTP_OK;
}

int ftp_norm_backward(const ftp_norm_shape* shape, const void* dy, const void* x, const int8_t* codes, const int8_t* exponents, int32_t block,
                      const void* gamma, const float* mean, const float* rstd, void* dx, float* dgamma, float* dbeta, void* workspace, void* stream)
{
    bool nothing;
    const int rc = check(shape, true, codes != nullptr, &nothing);
    if (rc != FTP_OK) return rc;
    if (!dgamma != !dbeta || !codes != !exponents || (x && codes)) return FTP_EINVAL;
    if (codes) {
        if (block != 32 && block != 64 && block != 128 && block != 256) return FTP_EUNSUPPORTED;
        if (shape->channels > 1 && (shape->dx_stride[2] != 1 || shape->dy_stride[2] != 1)) return FTP_EUNSUPPORTED;
    }
    if (dgamma && !workspace) return FTP_EINVAL;
    if (!nothing && (!dy || (!x && !codes) || !mean || !rstd || !dx)) return FTP_EINVAL;
    norm_backward(*shape, dy, x, codes, exponents, block, gamma, mean, rstd, dx, dgamma, dbeta, (float*)workspace, (hipStream_t)stream);
    return launched();
}

int ftp_checkpoint_pack(const ftp_checkpoint_shape* shape, const void* x, int8_t* codes, int8_t* exponents, void* stream)
{
    const int rc = check(shape);
    if (rc != FTP_OK || shape->rows == 0) return rc;
    if (!x || !codes || !exponents) return FTP_EINVAL;
    held_pack(*shape, x, codes, exponents, (hipStream_t)stream);
    return launched();
}

int ftp_checkpoint_unpack(const ftp_checkpoint_shape* shape, const int8_t* codes, const int8_t* exponents, int32_t act, float slope, void* out, void* stream)
{
    const int rc = check(shape);
    if (rc != FTP_OK) return rc;
    if (!is_act(act)) return FTP_EINVAL;
    if (shape->rows == 0) return FTP_OK;
    if (!codes || !exponents || !out) return FTP_EINVAL;
    held_unpack(*shape, codes, exponents, act, slope, out, (hipStream_t)stream);
    return launched();
}

int ftp_checkpoint_act_backward(const ftp_checkpoint_shape* shape, const int8_t* codes, const int8_t* exponents, int32_t act, float slope, const void* dy,
                                void* dx, void* stream)
{
    const int rc = check(shape);
    if (rc != FTP_OK) return rc;
    if (!is_act(act)) return FTP_EINVAL;
    if (shape->rows == 0) return FTP_OK;
    if (!codes || !exponents || !dy || !dx) return FTP_EINVAL;
    held_act_backward(*shape, codes, exponents, act, slope, dy, dx, (hipStream_t)stream);
    return launched();
}

int ftp_checkpoint_workspace(const ftp_checkpoint_shape* shape, int32_t outputs, size_t* bytes)
{
    const int rc = check(shape);
    if (rc != FTP_OK) return rc;
    if (outputs < 1 || !bytes) return FTP_EINVAL;
    *bytes = held_wgrad_workspace(*shape, outputs);
    return FTP_OK;
}

int ftp_checkpoint_wgrad(const ftp_checkpoint_shape* shape, const int8_t* codes, const int8_t* exponents, const void* dy, int64_t dy_stride, int32_t outputs,
                         float* dw, void* workspace, void* stream)
{
    const int rc = check(shape);
    if (rc != FTP_OK) return rc;
    if (outputs < 1 || dy_stride < outputs || !dw || (shape->rows && (!codes || !exponents || !dy))) return FTP_EINVAL;
    if (ceil_div(outputs, 128) * ceil_div(shape->cols, 128) > kMostGroups) return FTP_EUNSUPPORTED;
    if (!workspace && held_wgrad_workspace(*shape, outputs)) return FTP_EINVAL;
    held_wgrad(*shape, codes, exponents, dy, dy_stride, outputs, dw, (float*)workspace, (hipStream_t)stream);
    return launched();
}

int ftp_attention_workspace(const ftp_attention_shape* shape, size_t* forward_bytes, size_t* backward_bytes)
{
    const int rc = check(shape);
    if (rc != FTP_OK) return rc;
    if (forward_bytes) *forward_bytes = attention_forward_workspace(*shape);
    if (backward_bytes) *backward_bytes = attention_backward_workspace(*shape);
    return FTP_OK;
}

int ftp_attention_forward(const ftp_attention_shape* shape, const void* q, const void* k, const void* v, const int32_t* q_lens, const int32_t* kv_lens,
                          void* out, float* lse, void* workspace, void* stream)
{
    const int rc = check(shape, false);
    if (rc != FTP_OK || shape->batch == 0 || shape->q_len == 0) return rc;
    if (!q || !out || (shape->kv_len && (!k || !v)) || (!workspace && attention_forward_workspace(*shape))) return FTP_EINVAL;
    attention_forward(*shape, q, k, v, q_lens, kv_lens, out, lse, (float*)workspace, (hipStream_t)stream);
    return launched();
}

int ftp_attention_backward(const ftp_attention_shape* shape, const void* dout, const void* q, const void* k, const void* v, const int32_t* q_lens,
                           const int32_t* kv_lens, const void* out, const float* lse, void* dq, void* dk, void* dv, void* workspace, void* stream)
{
    const int rc = check(shape, true);
    if (rc != FTP_OK || shape->batch == 0) return rc;
    if (shape->q_len && (!dout || !q || !out || !lse || !dq || !workspace)) return FTP_EINVAL;
    if (shape->kv_len && (!k || !v || !dk || !dv)) return FTP_EINVAL;
    attention_backward(*shape, dout, q, k, v, q_lens, kv_lens, out, lse, dq, dk, dv, (float*)workspace, (hipStream_t)stream);
    return launched();
}

}  // extern "C"
