// Launchers of the training operators (embedding, loss over a vocabulary, orthogonal updates); arguments have been checked by the callers in ftp_training.hip.
#pragma once
#include "ftp_tokens.h"

namespace ftp {

void embedding_forward(const ftp_embedding_shape& s, const void* ids, const void* table, void* out, hipStream_t st);
bool embedding_backward_fits(const ftp_embedding_shape& s);
size_t embedding_workspace(const ftp_embedding_shape& s);
void embedding_backward(const ftp_embedding_shape& s, const void* ids, const void* dy, float* dtable, void* ws, hipStream_t st);

bool token_loss_fits(const ftp_token_loss_shape& s);
size_t token_loss_forward_workspace(const ftp_token_loss_shape& s);
size_t token_loss_backward_workspace(const ftp_token_loss_shape& s);
void token_loss_forward(const ftp_token_loss_shape& s, const void* x, const void* w, const void* labels, float* loss, float* lse, float* mean, char* ws, hipStream_t st);
void token_loss_backward(const ftp_token_loss_shape& s, const void* x, const void* w, const void* labels, const float* lse, const float* dloss, void* dx, void* dw, char* ws,
                         hipStream_t st);

bool orthogonal_fits(const ftp_orthogonal_shape& s);
size_t orthogonal_workspace(const ftp_orthogonal_shape& s);
void orthogonal(const ftp_orthogonal_shape& s, const void* x, void* out, char* ws, hipStream_t st);

// The id of a row as a number from 0 to count - 1, or -1 where there is none.
__device__ __forceinline__ int id_of(const void* ids, int wide, long long row, int count)
{
    if (wide) {
        const long long v = ((const long long*)ids)[row];
        return v >= 0 && v < count ? (int)v : -1;
    }
    const int v = ((const int*)ids)[row];
    return v >= 0 && v < count ? v : -1;
}

// Parts of a caller's scratch, one after the other, 256-byte aligned.
struct Parts {
    char* base;
    size_t used = 0;
    explicit Parts(void* p) : base((char*)p) {}
    template <typename T>
    T* take(size_t n)
    {
        T* p = (T*)(base + used);
        used += (n * sizeof(T) + 255) & ~(size_t)255;
        return p;
    }
};

}  // namespace ftp
