// The global norm of a model's gradients, and clipping: what the gradient of the loss over verdicts (Section 6) goes through before a step.
//
//   norm = scale sqrt(sum x^2),   factor = max_norm / norm where the norm is above max_norm, else 1,   out = scale factor x
//
// What bounds it: bytes.  Every element is read once for the norm and, if there is a result, read again and written.  The second
// pass takes the tensors from the end on: what the first one read last is still in L2.
//
// Tensors are cut into chunks of 8 or 16 vectors of 16 bytes a thread; block b takes the chunks b, b + blocks, ...  Its sum of squares, in 64
// bits, is a number of its own in the working memory, and whoever needs the norm adds these up in their order: no atomics, the same result
// on every run.
#include <math.h>

#include <algorithm>
#include <new>

#include "vl_logits.cuh"

namespace {

constexpr uint32_t CL_THREADS = 256, CL_WARPS = CL_THREADS / 32;
constexpr uint32_t CL_PARTS = 1024;   // blocks of a launch, at most
constexpr uint32_t CL_FEW = 64, CL_MANY = 960;  // tensors of a launch: they travel as kernel arguments (2 KB, or 31 KB which the host has to copy)

// Blocks of a multiprocessor by the vectors that a thread has in flight: what their registers leave room for.
constexpr uint32_t per_sm(uint32_t V) { return V == 16 ? 2 : 4; }

struct Piece {
    const char *x;
    char *out;
    uint64_t n;
    uint32_t first, dtype;  // its first chunk
};
template <uint32_t N>
struct Pieces {
    uint32_t n, chunks;
    Piece p[N];
};

// A tensor as 16-byte vectors of memory: vector v holds the elements first(v) .. first(v) + EPV - 1, of which the first and the last one
// may lack some.
template <typename T>
struct Vectors {
    const T *x;
    uint64_t n, count;
    uint32_t lead;
    __device__ __forceinline__ explicit Vectors(const Piece &p)
        : x(reinterpret_cast<const T *>(p.x)), n(p.n), lead((uint32_t)((uintptr_t)p.x & 15) / (uint32_t)sizeof(T))
    {
        count = (lead + n + EPV<T> - 1) / EPV<T>;
    }
    __device__ __forceinline__ bool whole(uint64_t v) const { return (v > 0 || lead == 0) && (v + 1) * EPV<T> <= lead + n; }
    __device__ __forceinline__ const uint4 *at(uint64_t v) const
    {
        return reinterpret_cast<const uint4 *>(reinterpret_cast<uintptr_t>(x) & ~(uintptr_t)15) + v;
    }
    __device__ __forceinline__ bool has(uint64_t v, int j) const { return v * EPV<T> + j >= lead && v * EPV<T> + j - lead < n; }
    __device__ __forceinline__ uint64_t place(uint64_t v, int j) const { return v * EPV<T> + j - lead; }
    __device__ __forceinline__ uint4 part(uint64_t v) const  // 0 elsewhere
    {
        T e[EPV<T>];
#pragma unroll
        for (int j = 0; j < EPV<T>; ++j) {
            from_f32(e[j], 0.0f);
            if (has(v, j)) e[j] = x[place(v, j)];
        }
        uint4 r;
        memcpy(&r, e, 16);
        return r;
    }
    template <uint32_t V>
    __device__ __forceinline__ void fetch(uint4 (&raw)[V], uint64_t v0) const  // of the chunk that begins at v0
    {
#pragma unroll
        for (uint32_t j = 0; j < V; ++j) {
            const uint64_t v = v0 + j * CL_THREADS + threadIdx.x;
            raw[j] = make_uint4(0, 0, 0, 0);
            if (whole(v)) raw[j] = *at(v);
            else if (v < count) raw[j] = part(v);
        }
    }
};

// Sum of the squares of eight of a thread's vectors.  In 32 bits, eight sums of eight (or four) squares; where these leave the range in which what they
// lose is nothing next to them (squares from 2^-150 on; a sum of 64), in 64 bits, 0 aside.
template <typename T>
__device__ __forceinline__ double squares(const uint4 *raw)
{
    f32x2 s[4] = {0ull, 0ull, 0ull, 0ull};
    uint32_t any = 0;
#pragma unroll
    for (uint32_t u = 0; u < 8; ++u) {
        float x[EPV<T>];
        unpack(raw[u], x, T{});
        any |= raw[u].x | raw[u].y | raw[u].z | raw[u].w;
#pragma unroll
        for (int j = 0; j < EPV<T>; j += 2) {
            const f32x2 y = both(x[j], x[j + 1]);
            s[(j / 2 + u * (EPV<T> / 2)) % 4] = fma2(y, y, s[(j / 2 + u * (EPV<T> / 2)) % 4]);
        }
    }
    float a, b;
    apart(add2(add2(s[0], s[1]), add2(s[2], s[3])), a, b);
    const float sum = a + b;
    if (std::is_same_v<T, __half>) return (double)sum;  // (halves: no square is below 2^-48 or above 2^32)
    const uint32_t value = sizeof(T) == 4 ? 0x7FFFFFFFu : 0x7FFF7FFFu;
    if ((sum >= 7.9e-31f && sum < __int_as_float(0x7f800000)) || !(any & value)) return (double)sum;
    double d = 0.0;
#pragma unroll
    for (uint32_t u = 0; u < 8; ++u) {
        float x[EPV<T>];
        unpack(raw[u], x, T{});
#pragma unroll
        for (int j = 0; j < EPV<T>; ++j) d = fma((double)x[j], (double)x[j], d);
    }
    return d;
}

// The piece of a chunk: the last one that begins at or in front of it (pieces have a chunk at least).
template <uint32_t N>
__device__ __forceinline__ uint32_t piece_of(const Pieces<N> &q, uint32_t chunk)
{
    uint32_t a = 0, b = q.n;
    while (b - a > 1) {
        const uint32_t mid = (a + b) / 2;
        if (q.p[mid].first <= chunk) a = mid; else b = mid;
    }
    return a;
}

// Sum over the block in a fixed order, in every thread.
__device__ __forceinline__ double block_total(double v, double *s)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0;
    for (uint32_t w = 0; w < CL_WARPS; ++w) v += s[w];
    return v;
}

template <uint32_t N, uint32_t V>
__global__ void __launch_bounds__(CL_THREADS, per_sm(V)) k_grad_squares(const __grid_constant__ Pieces<N> q, double *part)
{
    __shared__ double s[CL_WARPS];
    pdl_go();
    double sum = 0.0;
    for (uint32_t chunk = blockIdx.x; chunk < q.chunks; chunk += gridDim.x) {
        const Piece &p = q.p[piece_of(q, chunk)];
        const uint64_t v0 = (uint64_t)(chunk - p.first) * (CL_THREADS * V);
        uint4 raw[V];
        auto add = [&](auto t) {
            Vectors<decltype(t)>(p).template fetch<V>(raw, v0);
#pragma unroll
            for (uint32_t j = 0; j < V; j += 8) sum += squares<decltype(t)>(raw + j);
        };
        if (p.dtype == VL_F32) add(float{});
        else if (p.dtype == VL_F16) add(__half{});
        else add(__nv_bfloat16{});
    }
    sum = block_total(sum, s);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

// Where the sum of squares comes from: parts of it, or a number that was given (and has the scale in it already).
struct Total {
    const double *part;
    uint32_t n;
    double scale;
    int given;
};
// scale^2 times the sum, in every thread.
__device__ __forceinline__ double sum_squares(const Total &t, double *s)
{
    if (t.given) return t.part[0];
    double v = 0.0;
    for (uint32_t i = threadIdx.x; i < t.n; i += CL_THREADS) v += t.part[i];
    return block_total(v, s) * t.scale * t.scale;
}

__global__ void __launch_bounds__(CL_THREADS) k_grad_norm(const Total t, float *norm, double *squares)
{
    __shared__ double s[CL_WARPS];
    pdl_wait();
    const double v = sum_squares(t, s);
    if (threadIdx.x == 0) {
        if (norm) *norm = (float)sqrt(v);
        if (squares) *squares = v;
    }
}

// by = scale * factor in two parts, so that a product is rounded once; where a part of 32 bits does not hold it, in 64.
struct By {
    float hi, lo;
    double all;
    bool wide;
    __device__ __forceinline__ explicit By(double b) : hi((float)b), lo((float)(b - (double)(float)b)), all(b), wide(!(b > 1e-25 && b < 1e25)) {}
    __device__ __forceinline__ float times(float x) const
    {
        const float r = fmaf(x, hi, x * lo);
        return fabsf(x) < __int_as_float(0x7f800000) ? r : x * hi;  // (an infinite x may have a lo of 0, or of another sign)
    }
    __device__ __forceinline__ float times_wide(float x) const { return (float)((double)x * all); }
};

template <typename T, uint32_t V>
__device__ __forceinline__ void scale_chunk(const Piece &p, uint64_t v0, const By &by)
{
    const Vectors<T> x(p);
    T *const out = reinterpret_cast<T *>(p.out);
    const bool aligned = (((uintptr_t)p.out ^ (uintptr_t)p.x) & 15) == 0;
    uint4 raw[V];
    if (by.all == 0.0) {
#pragma unroll
        for (uint32_t j = 0; j < V; ++j) raw[j] = make_uint4(0, 0, 0, 0);
    } else {
        x.template fetch<V>(raw, v0);
    }
#pragma unroll
    for (uint32_t j = 0; j < V; ++j) {
        const uint64_t v = v0 + j * CL_THREADS + threadIdx.x;
        float e[EPV<T>];
        unpack(raw[j], e, T{});
#pragma unroll
        for (int i = 0; i < EPV<T>; ++i) e[i] = by.all == 0.0 ? 0.0f : by.wide ? by.times_wide(e[i]) : by.times(e[i]);
        if (aligned && x.whole(v)) {
            *reinterpret_cast<uint4 *>(out + x.place(v, 0)) = pack(e, T{});
        } else if (v < x.count) {
#pragma unroll
            for (int i = 0; i < EPV<T>; ++i)
                if (x.has(v, i)) from_f32(out[x.place(v, i)], e[i]);
        }
    }
}

template <uint32_t N, uint32_t V>
__global__ void __launch_bounds__(CL_THREADS, per_sm(V)) k_grad_clip(const __grid_constant__ Pieces<N> q, const Total t, double max_norm,
                                                                     float *norm_out, float *factor_out)
{
    __shared__ double s[CL_WARPS];
    pdl_wait();
    const double norm = sqrt(sum_squares(t, s));
    const double factor = !(norm <= 1.7976931348623157e308) ? 0.0 : norm > max_norm ? max_norm / norm : 1.0;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        if (norm_out) *norm_out = (float)norm;
        if (factor_out) *factor_out = (float)factor;
    }
    const By by(t.scale * factor);
    for (uint32_t i = blockIdx.x; i < q.chunks; i += gridDim.x) {
        const uint32_t chunk = q.chunks - 1 - i;
        const Piece &p = q.p[piece_of(q, chunk)];
        const uint64_t v0 = (uint64_t)(chunk - p.first) * (CL_THREADS * V);
        if (by.all == 1.0 && p.out == p.x) continue;  // (it is there already)
        if (p.dtype == VL_F32) scale_chunk<float, V>(p, v0, by);
        else if (p.dtype == VL_F16) scale_chunk<__half, V>(p, v0, by);
        else scale_chunk<__nv_bfloat16, V>(p, v0, by);
    }
}

uint32_t size_of(int dtype) { return dtype == VL_F32 ? 4 : 2; }

// Whether every result is its own tensor, or memory that no other result and no tensor has a byte in.
bool results_apart(uint32_t n, const vl_gradient *t, bool *failed)
{
    struct Range {
        uintptr_t a, b;
    };
    Range few[CL_FEW], *out = n <= CL_FEW ? few : new (std::nothrow) Range[n];
    *failed = !out;
    if (!out) return false;
    uint32_t m = 0;
    for (uint32_t j = 0; j < n; ++j)
        if (t[j].n) out[m++] = Range{(uintptr_t)t[j].out, (uintptr_t)t[j].out + t[j].n * size_of(t[j].dtype)};
    std::sort(out, out + m, [](const Range &x, const Range &y) { return x.a < y.a; });
    bool apart = true;
    for (uint32_t j = 1; j < m && apart; ++j) apart = out[j].a >= out[j - 1].b;
    for (uint32_t j = 0; j < n && apart; ++j) {
        if (!t[j].n || t[j].x == t[j].out) continue;
        const uintptr_t a = (uintptr_t)t[j].x, b = a + t[j].n * size_of(t[j].dtype);
        const Range *const next = std::lower_bound(out, out + m, b, [](const Range &r, uintptr_t v) { return r.a < v; });  // begins at b or later
        apart = next == out || (next - 1)->b <= a;
    }
    if (out != few) delete[] out;
    return apart;
}

int check(uint32_t n, const vl_gradient *t, bool out, double scale, const void *work, uint64_t work_bytes)
{
    if ((n && !t) || !(scale >= 1e-18 && scale <= 1e18)) return VL_ERR_INVALID_ARG;
    if (!work || ((uintptr_t)work & 15) || work_bytes < vl_grad_work(n)) return VL_ERR_INVALID_ARG;
    for (uint32_t j = 0; j < n; ++j) {
        if (t[j].dtype != VL_F32 && t[j].dtype != VL_F16 && t[j].dtype != VL_BF16) return VL_ERR_INVALID_ARG;
        if (t[j].n > (1ull << 40) || (t[j].n && (!t[j].x || (out && !t[j].out)))) return VL_ERR_INVALID_ARG;
        if (((uintptr_t)t[j].x | (out ? (uintptr_t)t[j].out : 0)) % size_of(t[j].dtype)) return VL_ERR_INVALID_ARG;
    }
    return VL_OK;
}

// The next tensors of a launch, from j on; tensors without elements are passed over.
template <uint32_t N>
void gather(Pieces<N> &q, uint32_t n, const vl_gradient *t, uint32_t &j, uint32_t V)
{
    q.n = q.chunks = 0;
    for (; j < n && q.n < N; ++j) {
        if (!t[j].n) continue;
        const uint32_t size = size_of(t[j].dtype), per = 16 / size;
        const uint64_t vectors = ((uintptr_t)t[j].x % 16 / size + t[j].n + per - 1) / per;
        const uint64_t chunks = (vectors + CL_THREADS * V - 1) / (CL_THREADS * V);
        if (q.chunks + chunks > 0xF0000000ull) break;
        q.p[q.n++] = Piece{static_cast<const char *>(t[j].x), static_cast<char *>(t[j].out), t[j].n, q.chunks, (uint32_t)t[j].dtype};
        q.chunks += (uint32_t)chunks;
    }
}

uint32_t blocks_of(uint32_t chunks, uint32_t V, int device)
{
    const uint32_t resident = per_sm(V) * (uint32_t)vl_device_sm_count(device), most = resident < CL_PARTS ? resident : CL_PARTS;
    return chunks < most ? chunks : most;
}

// The sums of squares of the tensors, as parts in the working memory.
template <uint32_t N, uint32_t V>
cudaError_t add_squares(uint32_t n, const vl_gradient *t, double *part, uint32_t *parts, int device, cudaStream_t st)
{
    Pieces<N> q;
    for (uint32_t j = 0; j < n;) {
        gather(q, n, t, j, V);
        if (!q.n) break;
        const uint32_t blocks = blocks_of(q.chunks, V, device);
        const cudaError_t e = launch_overlap(k_grad_squares<N, V>, dim3(blocks), CL_THREADS, 0, st, false, q, part + *parts);
        if (e != cudaSuccess) return e;
        *parts += blocks;
    }
    return cudaSuccess;
}
template <uint32_t N, uint32_t V>
cudaError_t clip(uint32_t n, const vl_gradient *t, const Total &total, bool overlap, double max_norm, float *norm, float *factor, int device,
                 cudaStream_t st)
{
    Pieces<N> q;
    uint32_t j = 0;
    do {
        gather(q, n, t, j, V);
        const uint32_t blocks = blocks_of(q.chunks, V, device);
        const cudaError_t e = launch_overlap(k_grad_clip<N, V>, dim3(blocks ? blocks : 1), CL_THREADS, 0, st, overlap, q, total, max_norm, norm, factor);
        if (e != cudaSuccess) return e;
        norm = factor = nullptr;
        overlap = false;
    } while (j < n && q.n);
    return cudaSuccess;
}

// Sixteen vectors of a thread in flight where there are some rounds of them for every block; eight where that would leave blocks idle.
// us with 8 and 16, 40 tensors of bf16: norm of 25, 100, 200, 400 MB 7.7, 7.2; 23, 17; 45, 35; 88, 63 (and of 0.5 MB 3.7, 4.0); clipping these to as many
// bytes elsewhere 21, 27; 63, 84; 118, 140; 228, 249; 1.2 GB of fp32 599, 580.
bool large(uint32_t n, const vl_gradient *t)
{
    uint64_t bytes = 0;
    for (uint32_t j = 0; j < n; ++j) bytes += t[j].n * size_of(t[j].dtype);
    return bytes >= 100000000;
}
auto adds(uint32_t n, const vl_gradient *t)
{
    if (large(n, t)) return n <= CL_FEW ? add_squares<CL_FEW, 16> : add_squares<CL_MANY, 16>;
    return n <= CL_FEW ? add_squares<CL_FEW, 8> : add_squares<CL_MANY, 8>;
}

}  // namespace

extern "C" uint64_t vl_grad_work(uint32_t n) { return ((uint64_t)n / CL_MANY + 2) * CL_PARTS * 8; }

extern "C" int vl_grad_norm(int device, uint32_t n, const vl_gradient *tensors, double scale, float *d_norm, double *d_sum_squares, void *d_work,
                            uint64_t work_bytes, void *stream)
{
    const int rc = check(n, tensors, false, scale, d_work, work_bytes);
    if (rc != VL_OK) return rc;
    if (((uintptr_t)d_norm & 3) || ((uintptr_t)d_sum_squares & 7)) return VL_ERR_INVALID_ARG;
    const DeviceScope scope(device);
    if (scope.error != cudaSuccess) return VL_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)stream;
    double *const part = static_cast<double *>(d_work);
    uint32_t parts = 0;
    if (adds(n, tensors)(n, tensors, part, &parts, device, st) != cudaSuccess) return VL_ERR_CUDA;
    const Total t{part, parts, scale, 0};
    return launch_overlap(k_grad_norm, dim3(1), CL_THREADS, 0, st, parts != 0, t, d_norm, d_sum_squares) == cudaSuccess ? VL_OK : VL_ERR_CUDA;
}

extern "C" int vl_clip_grads(int device, uint32_t n, const vl_gradient *tensors, double scale, double max_norm, const double *d_given,
                             float *d_norm, float *d_factor, void *d_work, uint64_t work_bytes, void *stream)
{
    const int rc = check(n, tensors, true, scale, d_work, work_bytes);
    if (rc != VL_OK) return rc;
    bool failed = false;
    if (!results_apart(n, tensors, &failed)) return failed ? VL_ERR_UNSUPPORTED : VL_ERR_INVALID_ARG;
    if (!(max_norm >= 0.0) || (((uintptr_t)d_norm | (uintptr_t)d_factor) & 3) || ((uintptr_t)d_given & 7)) return VL_ERR_INVALID_ARG;
    const DeviceScope scope(device);
    if (scope.error != cudaSuccess) return VL_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)stream;
    double *const part = static_cast<double *>(d_work);
    uint32_t parts = 0;
    if (!d_given && adds(n, tensors)(n, tensors, part, &parts, device, st) != cudaSuccess) return VL_ERR_CUDA;
    const Total t{d_given ? d_given : part, parts, scale, d_given != nullptr};
    const auto out = large(n, tensors) ? (n <= CL_FEW ? clip<CL_FEW, 16> : clip<CL_MANY, 16>) : (n <= CL_FEW ? clip<CL_FEW, 8> : clip<CL_MANY, 8>);
    return out(n, tensors, t, parts != 0, max_norm, d_norm, d_factor, device, st) == cudaSuccess ? VL_OK : VL_ERR_CUDA;
}
