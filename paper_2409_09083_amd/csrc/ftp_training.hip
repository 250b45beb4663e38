// C ABI of the training operators (embedding, loss over a vocabulary, orthogonal updates): checks of the arguments, then the launches.
#include "ftp_training.h"

#include <cmath>

using namespace ftp;

namespace {

bool is_type(int32_t dtype) { return dtype == FTP_F32 || dtype == FTP_BF16; }
bool is_id(int32_t type) { return type == FTP_I32 || type == FTP_I64; }

int check(const ftp_embedding_shape* s)
{
    if (!s || !is_type(s->dtype) || !is_id(s->id_type) || s->rows < 0 || s->vocab < 1 || s->channels < 1 || !std::isfinite(s->scale)) return FTP_EINVAL;
    if (s->table_stride < 0 || s->row_stride < 0) return FTP_EINVAL;
    if (s->rows > (1ll << 26) || s->vocab > (1 << 26) || s->channels > (1 << 20)) return FTP_EUNSUPPORTED;
    return FTP_OK;
}

int check(const ftp_token_loss_shape* s)
{
    if (!s || !is_type(s->dtype) || !is_id(s->id_type) || s->rows < 0 || s->vocab < 1 || s->channels < 1 || !(std::fabs(s->scale) <= 1e38f)) return FTP_EINVAL;
    if (s->x_stride < 0 || s->w_stride < 0 || s->dx_stride < 0 || s->dw_stride < 0) return FTP_EINVAL;
    return token_loss_fits(*s) ? FTP_OK : FTP_EUNSUPPORTED;
}

int check(const ftp_orthogonal_shape* s)
{
    if (!s || !is_type(s->dtype) || s->count < 0 || s->rows < 1 || s->cols < 1 || s->steps < 1 || !(s->eps >= 0) || !std::isfinite(s->eps)) return FTP_EINVAL;
    if (!std::isfinite(s->a) || !std::isfinite(s->b) || !std::isfinite(s->c) || s->matrix_stride < 0 || s->row_stride < 0) return FTP_EINVAL;
    return orthogonal_fits(*s) ? FTP_OK : FTP_EUNSUPPORTED;
}

}  // namespace

extern "C" {

int ftp_embedding_forward(const ftp_embedding_shape* shape, const void* ids, const void* table, void* out, void* stream)
{
    const int rc = check(shape);
    if (rc != FTP_OK || shape->rows == 0) return rc;
    if (!ids || !table || !out || (shape->rows > 1 && shape->row_stride < shape->channels)) return FTP_EINVAL;
    embedding_forward(*shape, ids, table, out, (hipStream_t)stream);
    return launched();
}

int ftp_embedding_workspace(const ftp_embedding_shape* shape, size_t* bytes)
{
    const int rc = check(shape);
    if (rc != FTP_OK) return rc;
    if (!embedding_backward_fits(*shape)) return FTP_EUNSUPPORTED;
    if (!bytes) return FTP_EINVAL;
    *bytes = embedding_workspace(*shape);
    return FTP_OK;
}

int ftp_embedding_backward(const ftp_embedding_shape* shape, const void* ids, const void* dy, float* dtable, void* workspace, void* stream)
{
    const int rc = check(shape);
    if (rc != FTP_OK) return rc;
    if (!embedding_backward_fits(*shape)) return FTP_EUNSUPPORTED;
    if (!dtable || (shape->rows && (!ids || !dy || !workspace))) return FTP_EINVAL;
    embedding_backward(*shape, ids, dy, dtable, workspace, (hipStream_t)stream);
    return launched();
}

int ftp_token_loss_workspace(const ftp_token_loss_shape* shape, size_t* forward_bytes, size_t* backward_bytes)
{
    const int rc = check(shape);
    if (rc != FTP_OK) return rc;
    if (forward_bytes) *forward_bytes = token_loss_forward_workspace(*shape);
    if (backward_bytes) *backward_bytes = token_loss_backward_workspace(*shape);
    return FTP_OK;
}

int ftp_token_loss_forward(const ftp_token_loss_shape* shape, const void* x, const void* weight, const void* labels, float* loss, float* lse, float* mean,
                           void* workspace, void* stream)
{
    const int rc = check(shape);
    if (rc != FTP_OK) return rc;
    if (!weight || !workspace || (shape->rows && (!x || !labels))) return FTP_EINVAL;
    token_loss_forward(*shape, x, weight, labels, loss, lse, mean, (char*)workspace, (hipStream_t)stream);
    return launched();
}

int ftp_token_loss_backward(const ftp_token_loss_shape* shape, const void* x, const void* weight, const void* labels, const float* lse, const float* dloss,
                            void* dx, void* dweight, void* workspace, void* stream)
{
    const int rc = check(shape);
    if (rc != FTP_OK) return rc;
    if (!weight || !workspace || (shape->rows && (!x || !labels || !lse))) return FTP_EINVAL;
    if (dx && shape->rows > 1 && shape->dx_stride < shape->channels) return FTP_EINVAL;
    if (dweight && shape->vocab > 1 && shape->dw_stride < shape->channels) return FTP_EINVAL;
    token_loss_backward(*shape, x, weight, labels, lse, dloss, dx, dweight, (char*)workspace, (hipStream_t)stream);
    return launched();
}

int ftp_orthogonal_workspace(const ftp_orthogonal_shape* shape, size_t* bytes)
{
    const int rc = check(shape);
    if (rc != FTP_OK) return rc;
    if (!bytes) return FTP_EINVAL;
    *bytes = orthogonal_workspace(*shape);
    return FTP_OK;
}

int ftp_orthogonal(const ftp_orthogonal_shape* shape, const void* x, void* out, void* workspace, void* stream)
{
    const int rc = check(shape);
    if (rc != FTP_OK || shape->count == 0) return rc;
    if (!x || !out || !workspace) return FTP_EINVAL;
    orthogonal(*shape, x, out, (char*)workspace, (hipStream_t)stream);
    return launched();
}

}  // extern "C"
