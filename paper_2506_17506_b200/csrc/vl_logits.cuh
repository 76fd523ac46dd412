// What the kernels over rows of logits share: element types, tokens, and which entries of a row are open.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "vl_internal.cuh"

// A checked vl_logits in the form the kernels take.
struct LogitRows {
    const void *x;
    uint64_t n_rows, stride;     // elements from row to row
    uint32_t V, W;               // entries of a row, words of a mask
    uint32_t token_bytes;
    const void *tokens;
    const uint32_t *occupied;
    uint32_t n_masks;            // that mask_rows can name: at most 2^31
    const int32_t *mask_rows;
    const uint8_t *widths;
    float scale;
};
// Where the scores go; what is null is not wanted.
struct ScoreOut {
    float *logprob, *entropy, *stats;
    uint32_t top;
    int32_t *ids;
    float *lps;
};
cudaError_t vl_scores_f32(const LogitRows &q, const ScoreOut &o, int device, cudaStream_t st);
cudaError_t vl_scores_f16(const LogitRows &q, const ScoreOut &o, int device, cudaStream_t st);
cudaError_t vl_scores_bf16(const LogitRows &q, const ScoreOut &o, int device, cudaStream_t st);

// Checks a descriptor: VL_OK and the kernels' form of it, or an error.
int vl_logit_rows(const vl_logits *x, LogitRows *out);

namespace {

template <typename T> __device__ __forceinline__ T lowest_bits();  // minus infinity
template <> __device__ __forceinline__ float lowest_bits<float>() { return __int_as_float(0xFF800000); }
template <> __device__ __forceinline__ __half lowest_bits<__half>() { return __ushort_as_half(0xFC00); }
template <> __device__ __forceinline__ __nv_bfloat16 lowest_bits<__nv_bfloat16>() { return __ushort_as_bfloat16(0xFF80); }
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_f32(float &d, float x) { d = x; }
__device__ __forceinline__ void from_f32(__half &d, float x) { d = __float2half_rn(x); }
__device__ __forceinline__ void from_f32(__nv_bfloat16 &d, float x) { d = __float2bfloat16_rn(x); }

template <typename T> constexpr int EPV = 16 / (int)sizeof(T);  // elements of a 16-byte vector
template <typename T> constexpr uint32_t MINUS_INF2 = sizeof(T) == 4 ? 0xFF800000u : 0u;
template <> constexpr uint32_t MINUS_INF2<__half> = 0xFC00FC00u;
template <> constexpr uint32_t MINUS_INF2<__nv_bfloat16> = 0xFF80FF80u;

__device__ __forceinline__ void unpack(const uint4 &r, float (&x)[4], float)
{
    x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y); x[2] = __uint_as_float(r.z); x[3] = __uint_as_float(r.w);
}
__device__ __forceinline__ void unpack(const uint4 &r, float (&x)[8], __nv_bfloat16)
{
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) { x[2 * j] = __uint_as_float(w[j] << 16); x[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u); }
}
__device__ __forceinline__ void unpack(const uint4 &r, float (&x)[8], __half)
{
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        __half2 h;
        memcpy(&h, &w[j], 4);
        const float2 f = __half22float2(h);
        x[2 * j] = f.x; x[2 * j + 1] = f.y;
    }
}
__device__ __forceinline__ uint32_t pack2(float a, float b, __half)
{
    const __half2 h = __floats2half2_rn(a, b);
    uint32_t w;
    memcpy(&w, &h, 4);
    return w;
}
__device__ __forceinline__ uint32_t pack2(float a, float b, __nv_bfloat16)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    uint32_t w;
    memcpy(&w, &h, 4);
    return w;
}
__device__ __forceinline__ uint4 pack(const float (&x)[4], float)
{
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
template <typename T>
__device__ __forceinline__ uint4 pack(const float (&x)[8], T t)
{
    return make_uint4(pack2(x[0], x[1], t), pack2(x[2], x[3], t), pack2(x[4], x[5], t), pack2(x[6], x[7], t));
}
// The largest of a vector's elements, of those that are numbers.
__device__ __forceinline__ float vector_max(const uint4 &r, float)
{
    return fmaxf(fmaxf(__uint_as_float(r.x), __uint_as_float(r.y)), fmaxf(__uint_as_float(r.z), __uint_as_float(r.w)));
}
__device__ __forceinline__ float vector_max(const uint4 &r, __half)
{
    __half2 h[4];
    memcpy(h, &r, 16);
    const __half2 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    return fmaxf(__low2float(m), __high2float(m));
}
__device__ __forceinline__ float vector_max(const uint4 &r, __nv_bfloat16)
{
    __nv_bfloat162 h[4];
    memcpy(h, &r, 16);
    const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    return fmaxf(__low2float(m), __high2float(m));
}

// The largest of several vectors' elements.
template <int N>
__device__ __forceinline__ float vectors_max(const uint4 (&r)[N], float t)
{
    float m = vector_max(r[0], t);
#pragma unroll
    for (int j = 1; j < N; ++j) m = fmaxf(m, vector_max(r[j], t));
    return m;
}
template <typename P, int N>
__device__ __forceinline__ P halves_max(const uint4 (&r)[N])
{
    P m[4];
    memcpy(m, &r[0], 16);
#pragma unroll
    for (int j = 1; j < N; ++j) {
        P h[4];
        memcpy(h, &r[j], 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) m[i] = __hmax2(m[i], h[i]);
    }
    return __hmax2(__hmax2(m[0], m[1]), __hmax2(m[2], m[3]));
}
template <int N>
__device__ __forceinline__ float vectors_max(const uint4 (&r)[N], __half)
{
    const __half2 m = halves_max<__half2>(r);
    return fmaxf(__low2float(m), __high2float(m));
}
template <int N>
__device__ __forceinline__ float vectors_max(const uint4 (&r)[N], __nv_bfloat16)
{
    const __nv_bfloat162 m = halves_max<__nv_bfloat162>(r);
    return fmaxf(__low2float(m), __high2float(m));
}

// bf16 entries no lower than -1e30 (what is no number stays none): two at once, so that no product with them leaves the range of numbers.
// The other types are bounded after the product.
template <typename T> constexpr bool BOUNDED = false;
template <> constexpr bool BOUNDED<__nv_bfloat16> = true;
template <typename T>
__device__ __forceinline__ uint4 above(const uint4 &r)
{
    if constexpr (BOUNDED<T>) {
        const __nv_bfloat162 low = __floats2bfloat162_rn(-1e30f, -1e30f);
        __nv_bfloat162 h[4];
        memcpy(h, &r, 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) h[j] = __hmax2_nan(h[j], low);
        uint4 o;
        memcpy(&o, h, 16);
        return o;
    } else {
        return r;
    }
}

constexpr float LOWEST = -3.402823466e38f;
constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;
// Up to here the rounded product of a logit with scale log2 e is off by at most 1/8 of a power of two.  Beyond it, it may be off by many
// powers of two (by 440 at 1e10): there differences of logits are multiplied, which costs two instructions an entry for one.
constexpr float FAR_OUT = 4194304.0f;  // 2^22
__device__ __forceinline__ bool far_out(float m, float c) { return !(fabsf(__fmul_rn(m, c)) < FAR_OUT); }

// A row as 16-byte vectors: vector v holds the entries first(v) .. first(v) + EPV - 1; the first and the last vector may hold
// entries of no row, which are read one by one around them.
template <typename T>
struct RowVectors {
    const T *row;
    uint32_t V, lead, n;  // entries; entries of the first vector in front of the row; vectors
    __device__ __forceinline__ RowVectors(const T *x, uint32_t entries)
        : row(x), V(entries), lead((uint32_t)((uintptr_t)x & 15) / (uint32_t)sizeof(T)), n((lead + entries + EPV<T> - 1) / EPV<T>) {}
    __device__ __forceinline__ int first(uint32_t v) const { return (int)(v * EPV<T>) - (int)lead; }
    __device__ __forceinline__ bool whole(uint32_t v) const { return (v > 0 || lead == 0) && (v + 1) * EPV<T> <= lead + V; }
    __device__ __forceinline__ const uint4 *at(uint32_t v) const
    {
        return reinterpret_cast<const uint4 *>(reinterpret_cast<uintptr_t>(row) & ~(uintptr_t)15) + v;
    }
    // Entries that are in the row; minus infinity elsewhere.
    __device__ __forceinline__ uint4 part(uint32_t v) const
    {
        T e[EPV<T>];
#pragma unroll
        for (int j = 0; j < EPV<T>; ++j) {
            const int i = first(v) + j;
            e[j] = (uint32_t)i < V ? row[i] : lowest_bits<T>();
        }
        uint4 r;
        memcpy(&r, e, 16);
        return r;
    }
};

// Blocks of 256 threads of a multiprocessor for short rows, by the vectors of a lane: what hides the loads are warps (200,000 rows of 256 bf16
// logits in us for 2, 3, 4, 5, 6 blocks of 122, 77, 64, 48, 40 registers a thread: 27.5, 21.8, 19.3, 24.5, 32).  Kernels with alternatives, for which this was
// not measured, spill at 64.
constexpr int short_blocks(int NV) { return NV <= 8 ? 4 : 2; }

// Short rows: groups of G lanes, a row each; lane g of a group holds the vectors g, g + G, ... and the closed entries of the words g,
// g + G, ...
// Entries whose bit is set to minus infinity.  Halves: a byte permutation takes their bytes from the one or the other word; the selectors
// of four entries are made at once, a bit spread to a byte of 0x44 (14 instructions a vector, 28 with a mask per pair).
template <typename T>
__device__ __forceinline__ void close_entries(uint4 &r, uint32_t bits)
{
    if constexpr (sizeof(T) == 4) {
        if (bits & 1) r.x = MINUS_INF2<T>;
        if (bits & 2) r.y = MINUS_INF2<T>;
        if (bits & 4) r.z = MINUS_INF2<T>;
        if (bits & 8) r.w = MINUS_INF2<T>;
    } else {
        const uint32_t a = (((bits & 15u) * 0x00204081u) & 0x01010101u) * 0x44u + 0x32103210u;
        const uint32_t b = (((bits >> 4) * 0x00204081u) & 0x01010101u) * 0x44u + 0x32103210u;
        r.x = __byte_perm(r.x, MINUS_INF2<T>, a);
        r.y = __byte_perm(r.y, MINUS_INF2<T>, a >> 16);
        r.z = __byte_perm(r.z, MINUS_INF2<T>, b);
        r.w = __byte_perm(r.w, MINUS_INF2<T>, b >> 16);
    }
}

// ALIGNED: rows start and end on vectors.  Else, with `around`, the vectors that reach into the rows in front and behind are read whole; without
// it (what lies there is not the matrix, or another thread's to write) their entries of the row alone.
template <typename T, int G, int NV, bool ALIGNED>
__device__ __forceinline__ void fetch_row(uint4 (&raw)[NV], const RowVectors<T> &x, uint32_t g, bool around)
{
    const uint4 *at = x.at(g);
    if (ALIGNED && x.n == G * NV) {
#pragma unroll
        for (int j = 0; j < NV; ++j) raw[j] = at[G * j];
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const uint32_t v = g + G * j;
            raw[j] = make_uint4(MINUS_INF2<T>, MINUS_INF2<T>, MINUS_INF2<T>, MINUS_INF2<T>);
            if (ALIGNED || around ? v < x.n : x.whole(v)) raw[j] = at[G * j];
        }
    }
    if (ALIGNED) return;
    const uint32_t last = x.n - 1, over = x.n * EPV<T> - x.lead - x.V;
    uint4 begin, end;
    if (!around) {
        if (g == 0) begin = x.part(0);
        if (g == last % G) end = x.part(last);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const uint32_t v = g + G * j;
        if (v == last || (j == 0 && g == 0)) {
            if (around) close_entries<T>(raw[j], ((v == 0 ? (1u << x.lead) - 1 : 0u) | (v == last ? 0xFFu << (EPV<T> - over) : 0u)) & ((1u << EPV<T>) - 1));
            else raw[j] = v == 0 ? begin : end;
        }
    }
}

// Two 32-bit numbers side by side: one instruction works on both.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 both(float a, float b)
{
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void apart(f32x2 r, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r)); }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c)
{
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// max and min that keep what is no number
__device__ __forceinline__ float min_nan(float a, float b)
{
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

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
    // Closed entries among i .. i + n - 1 (n <= 8; i may be negative: those in front of the row are closed), as the low bits.
    __device__ __forceinline__ uint32_t closed_from(int i, int n) const
    {
        const int w = i >> 5, s = i & 31;
        const uint32_t a = w < 0 ? 0xFFFFFFFFu : closed((uint32_t)w);
        const uint32_t b = s + n > 32 ? closed((uint32_t)(w + 1)) : 0u;
        return __funnelshift_r(a, b, s) & ((1u << n) - 1);
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
    if (q.mask_rows) {
        const uint32_t j = (uint32_t)q.mask_rows[r];  // (a negative one is a large one)
        if (j < q.n_masks) m.words = q.occupied + (uint64_t)j * q.W;
    } else if (q.occupied) {
        m.words = q.occupied + r * q.W;
    }
    return m;
}

// Sets the closed entries of a group's rows to minus infinity.  Each word of a mask is worked out by one lane and handed to those that
// hold its entries.  Every lane of the warp calls it; the result says whether entry tok is closed (true for what is no entry).
template <typename T, int G, int NV, bool ALIGNED>
__device__ __forceinline__ bool close_row(uint4 (&raw)[NV], const RowVectors<T> &x, const RowMask &mask, uint32_t g, int64_t tok)
{
    // words of a lane (rows that are not aligned have no more than one a lane to hand out, short_shape)
    constexpr int WL = NV * EPV<T> <= 32 ? 1 : (NV * EPV<T> + (ALIGNED ? 31 : 0)) / 32;
    constexpr bool WORDS = ALIGNED || WL == 1;
    static_assert(!ALIGNED || (NV - 1) * EPV<T> / 32 < WL, "every vector's word is one of the lane's");
    uint32_t word[WL];
    if (WORDS) {
#pragma unroll
        for (int k = 0; k < WL; ++k) word[k] = mask.closed(g + G * k);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        uint32_t bits;
        if (ALIGNED) {
            const uint32_t first = (g + G * j) * EPV<T>;
            bits = __shfl_sync(0xffffffffu, word[j * EPV<T> / 32], (first >> 5) & (G - 1), G) >> (first & 31);
        } else if (WORDS) {
            const int first = x.first(g + G * j), w = first >> 5;
            const uint32_t a = __shfl_sync(0xffffffffu, word[0], w & (G - 1), G), b = __shfl_sync(0xffffffffu, word[0], (w + 1) & (G - 1), G);
            bits = __funnelshift_r(a, b, first & 31);
        } else {
            bits = g + G * j < x.n ? mask.closed_from(x.first(g + G * j), EPV<T>) : 0u;
        }
        close_entries<T>(raw[j], bits & ((1u << EPV<T>) - 1));
    }
    const uint32_t t = tok < 0 ? 0u : (uint32_t)tok;
    if (!WORDS) return tok < 0 || mask.is_closed(t);
    uint32_t at = 0;
#pragma unroll
    for (int k = 0; k < WL; ++k) {
        const uint32_t w = __shfl_sync(0xffffffffu, word[k], (t >> 5) & (G - 1), G);
        if ((int)((t >> 5) / G) == k) at = w;
    }
    return (at >> (t & 31)) & 1;
}

// The kernel of rows of at most n vectors and W words of a mask: calls f with the lanes of a group and the vectors of a lane; false if the
// rows are long.  A group has a lane for every word (where a lane holds at most 32 entries it has one anyway).  Rows that are not aligned
// have a vector more than their entries fill: a fifth one a lane takes it in.
template <bool WARP, bool ALIGNED, typename F>
bool short_shape(uint32_t n, uint32_t W, F &&f)
{
    using std::integral_constant;
    auto with = [&](auto g, auto v) { f(g, v); return true; };
    constexpr integral_constant<int, 4> g4;
    constexpr integral_constant<int, 8> g8;
    constexpr integral_constant<int, 16> g16;
    constexpr integral_constant<int, 32> g32;
    constexpr integral_constant<int, 1> v1;
    constexpr integral_constant<int, 5> v5;
    if constexpr (WARP) {  // the whole warp at a row
        if (n <= 32) return with(g32, v1);
        if (n <= 160 && W <= 32) return with(g32, v5);
    } else if constexpr (ALIGNED) {
        if (n <= 4) return with(g4, v1);
        if (n <= 16) return with(g4, g4);
        if (n <= 32) return with(g4, g8);
        if (n <= 64) return with(g8, g8);
        if (n <= 128) return with(g16, g8);
    } else {
        if (n <= 4) return with(g4, v1);
        if (n <= 20 && W <= 4) return with(g4, v5);
        if (n <= 40 && W <= 8) return with(g8, v5);
        if (n <= 80 && W <= 16) return with(g16, v5);
        if (n <= 160 && W <= 32) return with(g32, v5);
    }
    if (n <= 256) return with(g32, g8);
    return false;
}

}  // namespace

// Largest number of 16-byte vectors that a row of the descriptor spans, and whether rows start and end on them.
static inline uint32_t row_vectors(const LogitRows &q, uint32_t size, bool *aligned)
{
    const uint32_t n = 16 / size;
    const bool starts = ((uintptr_t)q.x & 15) == 0 && (q.n_rows <= 1 || q.stride % n == 0);
    *aligned = starts && q.V % n == 0;
    return starts ? (q.V + n - 1) / n : (q.V + 2 * (n - 1)) / n;
}

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
