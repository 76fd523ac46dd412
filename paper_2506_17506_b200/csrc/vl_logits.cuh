// What the kernels over rows of logits share: element types, tokens, and which entries of a row are open.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "vl_internal.cuh"

namespace {

// A checked vl_logits in the form the kernels take.
struct LogitRows {
    const void *x;
    uint64_t n_rows, stride;     // elements from row to row
    uint32_t V, W;               // entries of a row, words of a mask
    uint32_t token_bytes;
    const void *tokens;
    const uint32_t *occupied;
    uint64_t n_masks;
    const int32_t *mask_rows;
    const uint8_t *widths;
    float scale;
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_f32(float &d, float x) { d = x; }
__device__ __forceinline__ void from_f32(__half &d, float x) { d = __float2half_rn(x); }
__device__ __forceinline__ void from_f32(__nv_bfloat16 &d, float x) { d = __float2bfloat16_rn(x); }

// Token of row r, or -1 where the row is left out (no entry of that number).  Without tokens every row counts, with entry V:
// one that no index reaches.
__device__ __forceinline__ int64_t row_token(const LogitRows &q, uint64_t r)
{
    if (!q.tokens) return q.V;
    int64_t t;
    if (q.token_bytes == 2) t = static_cast<const uint16_t *>(q.tokens)[r];
    else if (q.token_bytes == 4) t = static_cast<const int32_t *>(q.tokens)[r];
    else t = static_cast<const int64_t *>(q.tokens)[r];
    return t >= 0 && t < (int64_t)q.V ? t : -1;
}

// The mask of a row and the width of its tuple: entry i is closed if one of the entries i .. i + width - 1 is occupied or lies
// behind the last one.
struct RowMask {
    const uint32_t *words;  // null: nothing is occupied
    uint32_t V, W, width;
    __device__ __forceinline__ bool any() const { return words != nullptr || width > 1; }
    __device__ __forceinline__ uint32_t taken(uint32_t w) const
    {
        if (w >= W) return 0xFFFFFFFFu;
        uint32_t m = words ? __ldg(words + w) : 0u;
        if (w == W - 1 && (V & 31)) m |= 0xFFFFFFFFu << (V & 31);
        return m;
    }
    // Closed entries among 32 w .. 32 w + 31.
    __device__ __forceinline__ uint32_t closed(uint32_t w) const
    {
        const uint32_t own = taken(w);
        if (width <= 1) return own;
        if (width <= 32) {  // every bit to the width - 1 places below it, doubling the reach
            unsigned long long y = own | ((unsigned long long)taken(w + 1) << 32);
            for (uint32_t n = 1; n < width;) {
                const uint32_t s = min(n, width - n);
                y |= y >> s;
                n += s;
            }
            return (uint32_t)y;
        }
        // the next taken entry behind this word closes the width - 1 entries in front of it; one inside closes all below it
        uint32_t m = own ? 0xFFFFFFFFu >> __clz(own) : 0u;
        for (uint32_t j = 1; j * 32 < width + 31; ++j) {
            const uint32_t next = taken(w + j);
            if (!next) continue;
            const int from = (int)(32 * j + __ffs(next) - 1) - (int)(width - 1);  // first entry that it closes
            if (from < 32) m |= from <= 0 ? 0xFFFFFFFFu : 0xFFFFFFFFu << from;
            break;
        }
        return m;
    }
    __device__ __forceinline__ bool is_closed(uint32_t i) const { return (closed(i >> 5) >> (i & 31)) & 1; }
};
__device__ __forceinline__ RowMask row_mask(const LogitRows &q, uint64_t r)
{
    RowMask m;
    m.V = q.V;
    m.W = q.W;
    m.width = q.widths ? q.widths[r] : 1u;
    m.words = nullptr;
    if (q.occupied) {
        const uint64_t j = q.mask_rows ? (uint64_t)(int64_t)q.mask_rows[r] : r;  // (a negative one is a large one)
        if (j < q.n_masks) m.words = q.occupied + j * q.W;
    }
    return m;
}

}  // namespace

// Checks a descriptor: VL_OK and the kernels' form of it, or an error.
int vl_logit_rows(const vl_logits *x, LogitRows *out);

// Makes `device` current and puts the caller's device back at the end of the call.
struct DeviceScope {
    int before = -1;
    cudaError_t error;
    explicit DeviceScope(int device)
    {
        error = cudaGetDevice(&before);
        if (error == cudaSuccess && before != device) error = cudaSetDevice(device);
        else before = -1;
    }
    ~DeviceScope() { if (before >= 0) cudaSetDevice(before); }
};
