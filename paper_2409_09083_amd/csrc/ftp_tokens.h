// Launchers of the token block's operators (layer norm, 8-bit checkpoints, attention), and what their kernels share.
// Arguments have been checked by the callers in ftp_tokens.hip.
#pragma once
#include <hip/hip_runtime.h>
#include "ftp.h"
#include "ftp_device.h"
#include "ftp_split.h"

namespace ftp {

// FTP_OK, or FTP_EHIP with the error of the launches so far kept for ftp_last_hip_error (ftp_api.hip).
int launched();

size_t norm_workspace(const ftp_norm_shape& s);
void norm_forward(const ftp_norm_shape& s, const void* x, const void* gamma, const void* beta, void* y, float* mean, float* rstd, hipStream_t st);
void norm_backward(const ftp_norm_shape& s, const void* dy, const void* x, const int8_t* codes, const int8_t* exponents, int block, const void* gamma,
                   const float* mean, const float* rstd, void* dx, float* dgamma, float* dbeta, float* partial, hipStream_t st);
constexpr int kNormMapChannels = 4096;              // most channels of a tensor that is not made of rows

void held_pack(const ftp_checkpoint_shape& s, const void* x, int8_t* codes, int8_t* exponents, hipStream_t st);
void held_unpack(const ftp_checkpoint_shape& s, const int8_t* codes, const int8_t* exponents, int act, float slope, void* out, hipStream_t st);
void held_act_backward(const ftp_checkpoint_shape& s, const int8_t* codes, const int8_t* exponents, int act, float slope, const void* dy, void* dx, hipStream_t st);
size_t held_wgrad_workspace(const ftp_checkpoint_shape& s, int outputs);
void held_wgrad(const ftp_checkpoint_shape& s, const int8_t* codes, const int8_t* exponents, const void* dy, long long dy_stride, int outputs, float* dw,
                float* partial, hipStream_t st);

// A launch has less than 2^32 threads.
constexpr long long kMostGroups = (1ll << 24) - 1;  // ... in workgroups of 256
bool attention_fits(const ftp_attention_shape& s);  // (of shapes whose rows, keys and heads are 32-bit numbers)
size_t attention_forward_workspace(const ftp_attention_shape& s);
size_t attention_backward_workspace(const ftp_attention_shape& s);
void attention_forward(const ftp_attention_shape& s, const void* q, const void* k, const void* v, const int* q_lens, const int* kv_lens, void* out, float* lse,
                       float* ws, hipStream_t st);
void attention_backward(const ftp_attention_shape& s, const void* dout, const void* q, const void* k, const void* v, const int* q_lens, const int* kv_lens,
                        const void* out, const float* lse, void* dq, void* dk, void* dv, float* ws, hipStream_t st);

inline bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
inline long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// VEC neighbouring elements as they lie in memory, loaded and stored at once.
template <int BYTES> struct RawOf;
template <> struct RawOf<1> { typedef uint8_t type; };
template <> struct RawOf<2> { typedef uint16_t type; };
template <> struct RawOf<4> { typedef uint32_t type; };
template <> struct RawOf<8> { typedef uint32_t type __attribute__((ext_vector_type(2))); };
template <> struct RawOf<16> { typedef uint32_t type __attribute__((ext_vector_type(4))); };
template <typename T, int VEC>
struct Pack {
    static constexpr int kWords = (VEC * (int)sizeof(T) + 15) / 16, kBytes = VEC * (int)sizeof(T) / kWords;
    typedef typename RawOf<kBytes>::type Raw;
    Raw w[kWords];
    __device__ __forceinline__ void load(const T* p)
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = ((const Raw*)p)[i];
    }
    __device__ __forceinline__ void store(T* p) const
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i) ((Raw*)p)[i] = w[i];
    }
    // ... from and to any address: the hardware takes unaligned vectors from global memory
    __device__ __forceinline__ void load_any(const T* p) { __builtin_memcpy(w, p, sizeof(w)); }
    __device__ __forceinline__ void store_any(T* p) const { __builtin_memcpy(p, w, sizeof(w)); }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = (Raw)0;
    }
    __device__ __forceinline__ float get(int i) const
    {
        if constexpr (sizeof(T) == 4) {
            return __uint_as_float(word(i));
        } else if constexpr (sizeof(T) == 2) {
            if constexpr (VEC == 1) return __uint_as_float((uint32_t)w[0] << 16);
            else return __uint_as_float((i & 1) ? (word(i / 2) & 0xFFFF0000u) : (word(i / 2) << 16));
        } else {
            if constexpr (VEC < 4) return (float)(int8_t)((uint32_t)w[0] >> (8 * i));
            else return (float)(int8_t)(word(i / 4) >> (8 * (i & 3)));
        }
    }
    __device__ __forceinline__ void put(const float (&v)[VEC])
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) set_word(i, __float_as_uint(v[i]));
        } else if constexpr (VEC == 1) {
            w[0] = (Raw)bf16_bits(v[0]);
        } else {
#pragma unroll
            for (int i = 0; i < VEC / 2; ++i) set_word(i, pack_bf16(v[2 * i], v[2 * i + 1]));
        }
    }
private:
    __device__ __forceinline__ uint32_t word(int i) const
    {
        if constexpr (kBytes == 4) return w[i];
        else return w[i / (kBytes / 4)][i % (kBytes / 4)];
    }
    __device__ __forceinline__ void set_word(int i, uint32_t v)
    {
        if constexpr (kBytes == 4) w[i] = v;
        else w[i / (kBytes / 4)][i % (kBytes / 4)] = v;
    }
};

// 2^e of a checkpoint's exponent -126 .. 122; NaN for the 127 of a block that held an infinity or a NaN.
__device__ __forceinline__ float held_scale(int e) { return __uint_as_float(e == 127 ? 0x7FC00000u : (uint32_t)(e + 127) << 23); }

}  // namespace ftp
