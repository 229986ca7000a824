// The norm over all gradients of a step, and the gradients scaled to it (include/dmmv_layer.h).
//
// Both passes are bound by memory.  The tensors' places come with the kernel's arguments, LIST of them a launch, so a call copies nothing to the
// device and can be captured.  A tensor is cut into chunks of 8192 numbers, 2048 where there are few (rows with gaps into pieces of a row), and
// a workgroup has a run of consecutive chunks.  Short rows with gaps come several to a chunk, number by number.  Squares are summed in 64 bits: those of all 32-bit numbers are there, and no order of summing matters to 32 bits.
#include <algorithm>
#include <new>

#include "dmmv_layer_common.h"

namespace dmmv {

constexpr int LIST = 64, GROUPS = 1024;              // tensors a launch, most partial sums a launch
constexpr int SHORT = 512;                           // columns of rows that come several to a chunk
constexpr int PIECE = 2048;                          // numbers that 256 threads take at a time; a chunk is one of them, or four

struct TensorPlace {
    const void* in;
    void* out;
    int64_t cols, ld, ldo;               // one row, if the rows have no gaps
    uint32_t rows, many;                 // rows a chunk, 0: a chunk is a piece of a row
    uint32_t first;                      // chunks of the tensors before
    uint16_t in_bf16, out_bf16;
};
struct TensorList {
    TensorPlace t[LIST];
    int32_t count;
    uint32_t chunks;
};
static_assert(sizeof(TensorList) <= 3600, "with the other arguments below 4 KB");

// The workgroup's chunks of CHUNK numbers, in order or from the last: piece(tensor, row, first column, columns of the chunk), or for short rows
// one(tensor, row, column) for each of this thread's numbers
template <int CHUNK, bool BACK, class F, class G>
__device__ __forceinline__ void for_chunks(const TensorList& l, F piece, G one) {
    const uint32_t a = (uint32_t)((uint64_t)l.chunks * blockIdx.x / gridDim.x), b = (uint32_t)((uint64_t)l.chunks * (blockIdx.x + 1) / gridDim.x);
    if (a >= b) return;
    int at = 0, hi = l.count - 1;                            // the last tensor that begins at or before the first chunk to take
    while (at < hi) {
        const int mid = (at + hi + 1) >> 1;
        if (l.t[mid].first <= (BACK ? b - 1 : a)) at = mid;
        else hi = mid - 1;
    }
    for (uint32_t n = 0; n < b - a; ++n) {
        const uint32_t c = BACK ? b - 1 - n : a + n;
        if constexpr (BACK) {
            while (l.t[at].first > c) --at;
        } else {
            while (at + 1 < l.count && l.t[at + 1].first <= c) ++at;
        }
        const TensorPlace& t = l.t[at];
        const uint32_t i = c - t.first;
        if (t.many) {
            const uint32_t row0 = i * t.many, cols = (uint32_t)t.cols, numbers = min(t.many, t.rows - row0) * cols;
            for (uint32_t k = threadIdx.x; k < numbers; k += 256) {
                const uint32_t r = k / cols;
                one(t, (int64_t)(row0 + r), k - r * cols);
            }
        } else {
            const uint32_t pieces = (uint32_t)((t.cols + CHUNK - 1) / CHUNK), row = i / pieces;
            const int64_t col = (int64_t)(i - row * pieces) * CHUNK;
            piece(t, (int64_t)row, col, (int)min((int64_t)CHUNK, t.cols - col));
        }
    }
}

// sum over the 256 threads of the workgroup in a fixed order, in every thread
__device__ __forceinline__ double group_sum(double v, double (&sh)[4]) {
    v += dpp_mov<DPP_QUAD_XOR1>(v);
    v += dpp_mov<DPP_QUAD_XOR2>(v);
    v += dpp_mov<DPP_ROW_HALF_MIRROR>(v);
    v += dpp_mov<DPP_ROW_MIRROR>(v);
    v = (read_lane(v, 0) + read_lane(v, 16)) + (read_lane(v, 32) + read_lane(v, 48));
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    return (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

template <int CHUNK, class T>
__device__ __forceinline__ void add_squares(const T* __restrict__ p, int n, double (&s)[2]) {
#pragma unroll
    for (int i = 0; i < CHUNK / PIECE; ++i) {
        float v[8];
        load8(p, i * PIECE + threadIdx.x * 8, n, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e & 1] = __builtin_fma((double)v[e], (double)v[e], s[e & 1]);
    }
}

__device__ __forceinline__ float value_at(const TensorPlace& t, int64_t at) {
    return t.in_bf16 ? value_of(static_cast<const bf16_t*>(t.in)[at]) : static_cast<const float*>(t.in)[at];
}

// part[workgroup] = sum of the squares of its chunks.  360 M numbers in 32 bits: 243 us, 5.9 TB/s.
template <int CHUNK>
__global__ __launch_bounds__(256, 4) void k_gradient_squares(TensorList l, double* __restrict__ part) {
    __shared__ double sh[4];
    double s[2] = {0.0, 0.0};
    for_chunks<CHUNK, false>(l, [&](const TensorPlace& t, int64_t row, int64_t col, int n) {
        if (t.in_bf16) add_squares<CHUNK>(static_cast<const bf16_t*>(t.in) + row * t.ld + col, n, s);
        else add_squares<CHUNK>(static_cast<const float*>(t.in) + row * t.ld + col, n, s);
    }, [&](const TensorPlace& t, int64_t row, uint32_t col) {
        const double v = value_at(t, row * t.ld + col);
        s[0] = __builtin_fma(v, v, s[0]);
    });
    const double v = group_sum(s[0] + s[1], sh);
    if (threadIdx.x == 0) part[blockIdx.x] = v;
}

// the norm of all parts, the same in every workgroup that asks
__device__ __forceinline__ double norm_of(const double* __restrict__ part, int32_t parts, double (&sh)[4]) {
    double s = 0.0;
    for (int32_t i = threadIdx.x; i < parts; i += 256) s += part[i];
    return __builtin_sqrt(group_sum(s, sh));
}

__global__ __launch_bounds__(256) void k_gradient_norm(const double* __restrict__ part, int32_t parts, float* __restrict__ norm) {
    __shared__ double sh[4];
    const double v = norm_of(part, parts, sh);
    if (threadIdx.x == 0) *norm = (float)v;
}

// part[0] = the sum of all parts, in the order of norm_of: once for all launches of the scaling where there are more than two launches' parts, or their
// reading would grow with the square of the launches.  Clipping of 1024 tensors of 262144 numbers (16384 parts) 770 us, 996 with every workgroup adding
// up all of them, 4096 such 3060 and 7070; up to 2048 parts the launch costs as much as it saves (128 such 84 and 84, 256 of 8192 93 and 88).
__global__ __launch_bounds__(256) void k_gradient_total(double* part, int32_t parts) {
    __shared__ double sh[4];
    double s = 0.0;
    for (int32_t i = threadIdx.x; i < parts; i += 256) s += part[i];
    s = group_sum(s, sh);                            // (its barrier comes after all parts have been read)
    if (threadIdx.x == 0) part[0] = s;
}

// W consecutive numbers of which `left` are there, and back: past the caches, where what the sum of squares has read stays.  A wavefront's store
// fills whole lines, 16 bytes a lane.  Norm and scaling of 34 M numbers in 32 bits 70 us, 84 by ordinary stores; of 360 M 817 and 839, and 899 past the
// caches with 32 bytes a lane.
template <int W>
__device__ __forceinline__ void take(const float* p, int left, float (&v)[W]) {
    if (left >= W) {
#pragma unroll
        for (int k = 0; k < W; k += 4) {
            const piece16 a = *reinterpret_cast<const piece16_any*>(p + k);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[k + i] = __uint_as_float(a[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = i < left ? p[i] : 0.0f;
    }
}
template <int W>
__device__ __forceinline__ void take(const bf16_t* p, int left, float (&v)[W]) {
    if (left >= W) {
        uint32_t a[W / 2];
        if constexpr (W == 8) {
            const piece16 r = *reinterpret_cast<const piece16_any*>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) a[i] = r[i];
        } else {
            const piece8 r = *reinterpret_cast<const piece8_any*>(p);
            a[0] = r[0];
            a[1] = r[1];
        }
#pragma unroll
        for (int i = 0; i < W / 2; ++i) { v[2 * i] = bf16_value(a[i] & 0xFFFFu); v[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u); }
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = i < left ? bf16_value(p[i].u) : 0.0f;
    }
}
template <int W>
__device__ __forceinline__ void give(float* p, int left, const float (&v)[W]) {
    static_assert(W == 4, "16 bytes");
    if (left >= W) {
        const piece16 a = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
        __builtin_nontemporal_store(a, reinterpret_cast<piece16_any*>(p));
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i)
            if (i < left) p[i] = v[i];
    }
}
template <int W>
__device__ __forceinline__ void give(bf16_t* p, int left, const float (&v)[W]) {
    if (left >= W) {
        if constexpr (W == 8)
            __builtin_nontemporal_store(piece16{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])}, reinterpret_cast<piece16_any*>(p));
        else
            __builtin_nontemporal_store(piece8{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])}, reinterpret_cast<piece8_any*>(p));
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i)
            if (i < left) p[i].u = (uint16_t)bf16_bits(v[i]);
    }
}

template <int CHUNK, class T, class U>
__device__ __forceinline__ void scale_chunk(const T* in, U* out, int n, float c, float rest) {      // (out may be in)
    constexpr int W = sizeof(T) + sizeof(U) == 4 ? 8 : 4, N = CHUNK / (256 * W);
    float v[N][W];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int at = (i * 256 + (int)threadIdx.x) * W;
        take<W>(in + at, n - at, v[i]);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int at = (i * 256 + (int)threadIdx.x) * W;
#pragma unroll
        for (int e = 0; e < W; ++e) v[i][e] = v[i][e] * c * rest;
        give<W>(out + at, n - at, v[i]);
    }
}

// out = c in, with c = max_norm / (norm + eps) where that is below 1.  Tensors that stay where they are are not touched if c is 1.  Every workgroup
// adds up the parts for itself, which costs less than a launch between where there are few (k_gradient_total).  360 M numbers in 32 bits: 570 us, 5.0 TB/s of reading and writing.
template <int CHUNK>
__global__ __launch_bounds__(256) void k_gradient_scale(TensorList l, const double* __restrict__ part, int32_t parts, const float* __restrict__ given,
                                                        float max_norm, float eps, int32_t in_place, float* __restrict__ norm) {
    __shared__ double sh[4];
    const double v = given ? (double)*given : norm_of(part, parts, sh);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)v;
    const double sum = v + (double)eps;
    const double d = sum <= (double)max_norm ? 1.0 : (double)max_norm / sum;
    if (d == 1.0 && in_place) return;
    // a factor near the least normal number would lose bits that its product with a large number has
    const float rest = d < 0x1p-64 ? 0x1p-64f : 1.0f, c = (float)(d < 0x1p-64 ? d * 0x1p64 : d);
    // (from the last: what the sum of squares has read last is in the chip's cache still)
    for_chunks<CHUNK, true>(l, [&](const TensorPlace& t, int64_t row, int64_t col, int n) {
        const float* f = static_cast<const float*>(t.in) + row * t.ld + col;
        const bf16_t* b = static_cast<const bf16_t*>(t.in) + row * t.ld + col;
        float* fo = static_cast<float*>(t.out) + row * t.ldo + col;
        bf16_t* bo = static_cast<bf16_t*>(t.out) + row * t.ldo + col;
        if (t.in_bf16) t.out_bf16 ? scale_chunk<CHUNK>(b, bo, n, c, rest) : scale_chunk<CHUNK>(b, fo, n, c, rest);
        else t.out_bf16 ? scale_chunk<CHUNK>(f, bo, n, c, rest) : scale_chunk<CHUNK>(f, fo, n, c, rest);
    }, [&](const TensorPlace& t, int64_t row, uint32_t col) {
        const float v = value_at(t, row * t.ld + col) * c * rest;
        if (t.out_bf16) put_y(static_cast<bf16_t*>(t.out) + row * t.ldo + col, v);
        else put_y(static_cast<float*>(t.out) + row * t.ldo + col, v);
    });
}

// ---- host ---------------------------------------------------------------------------------------
static bool nothing(const dmmv_gradient& g) { return g.rows == 0 || g.cols == 0; }
static bool no_gaps(const dmmv_gradient& g) { return g.rows == 1 || g.ld == g.cols; }

static dmmv_status check_gradients(int64_t count, const dmmv_gradient* g, const char* what) {
    if (count < 0 || count > 1 << 20) return fail(DMMV_ERR_SHAPE, "%s: count out of range", what);
    if (count > 0 && !g) return fail(DMMV_ERR_NULL, "%s is NULL", what);
    for (int64_t i = 0; i < count; ++i) {
        DMMV_TRY(layer_check_dtype(g[i].dtype));
        if (g[i].rows < 0 || g[i].cols < 0) return fail(DMMV_ERR_SHAPE, "%s: negative size", what);
        if (g[i].rows > INT32_MAX || (g[i].rows > 0 && g[i].cols > ((int64_t)1 << 42) / g[i].rows)) return fail(DMMV_ERR_SHAPE, "%s: size out of range", what);
        DMMV_TRY(layer_check_array(g[i].data, g[i].rows, g[i].cols, g[i].ld, layer_width(g[i].dtype), what));
    }
    return DMMV_OK;
}

struct Extent {
    uintptr_t from, to;
    int64_t i;
};
static Extent extent_of(const dmmv_gradient& g, int64_t i) {
    const uintptr_t p = (uintptr_t)g.data;
    return {p, p + ((uintptr_t)((g.rows - 1) * (g.rows > 1 ? g.ld : 0)) + (uintptr_t)g.cols) * layer_width(g.dtype), i};
}
static bool same_place(const dmmv_gradient& a, const dmmv_gradient& b) {
    return a.data == b.data && a.dtype == b.dtype && a.rows == b.rows && a.cols == b.cols && (a.ld == b.ld || a.rows == 1);
}
// Whether two matrices whose extents (from the first number to the last) meet may share a number: parts of one matrix, of one type, row stride and more rows
// than one, need not.  Others in the gaps of a matrix are not looked for: gradients are whole tensors or parts of one.
static bool share(const dmmv_gradient& a, const dmmv_gradient& b) {      // a begins first
    const uintptr_t w = layer_width(a.dtype), ld = (uintptr_t)a.ld * w;
    if (a.dtype != b.dtype || no_gaps(a) || a.ld != b.ld || b.rows == 1) return true;
    const uintptr_t off = ((uintptr_t)b.data - (uintptr_t)a.data) % ld;
    return off < (uintptr_t)a.cols * w || off + (uintptr_t)b.cols * w > ld;
}
constexpr int64_t PAIRS = 1 << 27;                   // most that are compared: 0.5 to 0.7 s of the host, in every call
// What is written, the `to` of each gradient, shares memory neither with what else is written nor with another gradient that is read (from NULL:
// the gradients are their own place).  A gradient that is scaled where it is counts once.
static dmmv_status check_apart(int64_t count, const dmmv_gradient* to, const dmmv_gradient* from) {
    Extent* e = new (std::nothrow) Extent[count > 0 ? 2 * count : 1];
    if (!e) return fail(DMMV_ERR_WORKSPACE, "no host memory for %lld places", (long long)(2 * count));
    Extent* const r = e + count;
    int64_t n = 0, m = 0;
    for (int64_t i = 0; i < count; ++i)
        if (!nothing(to[i])) {
            e[n++] = extent_of(to[i], i);
            if (from && !same_place(from[i], to[i])) r[m++] = extent_of(from[i], i);
        }
    const auto before = [](const Extent& a, const Extent& b) { return a.from != b.from ? a.from < b.from : a.i < b.i; };
    std::sort(e, e + n, before);
    std::sort(r, r + m, before);
    // in the order of their first numbers; those before `first` end before what comes next
    struct Side {
        const Extent* e;
        const dmmv_gradient* g;
        int64_t n, first, at;
        uintptr_t most;
    };
    Side out = {e, to, n, 0, 0, 0}, in = {r, from, m, 0, 0, 0};
    int64_t pairs = 0;
    const Extent *bad = nullptr, *other = nullptr;
    bool read = false;                               // one of the two is read
    auto against = [&](Side& s, const dmmv_gradient& g, const Extent& x, bool reads) {
        if (x.from >= s.most) s.first = s.at;
        else if ((pairs += s.at - s.first) <= PAIRS)
            for (int64_t j = s.at - 1; j >= s.first && !bad; --j)
                if (s.e[j].to > x.from && share(s.g[s.e[j].i], g)) bad = &x, other = s.e + j, read = reads;
    };
    while (out.at + in.at < n + m && !bad && pairs <= PAIRS) {
        const bool write = in.at == m || (out.at < n && e[out.at].from <= r[in.at].from);
        Side& s = write ? out : in;
        const Extent& x = s.e[s.at];
        against(out, s.g[x.i], x, !write);
        if (write) against(in, s.g[x.i], x, true);
        else if (x.from >= in.most) in.first = in.at;
        s.most = std::max(s.most, x.to);
        ++s.at;
    }
    const int64_t a = bad ? std::min(bad->i, other->i) : 0, b = bad ? std::max(bad->i, other->i) : 0;
    delete[] e;
    if (pairs > PAIRS) return fail(DMMV_ERR_SHAPE, "gradients: too many parts of one matrix");
    if (!bad) return DMMV_OK;
    return read ? fail(DMMV_ERR_SHAPE, "gradients %lld and %lld: what one is written to may share memory with what the other is read from: their extents meet", (long long)a, (long long)b)
                : fail(DMMV_ERR_SHAPE, "gradients %lld and %lld may share memory: their extents meet", (long long)a, (long long)b);
}
// a norm is no number of tensors that are written, or that are read while it is
static dmmv_status check_norm_apart(const float* p, int64_t count, const dmmv_gradient* g, const char* what) {
    const uintptr_t at = (uintptr_t)p;
    for (int64_t i = 0; p && i < count; ++i)
        if (!nothing(g[i])) {
            const Extent e = extent_of(g[i], i);
            if (at + 4 > e.from && at < e.to) {
                const uintptr_t w = layer_width(g[i].dtype), ld = (uintptr_t)(g[i].rows > 1 ? g[i].ld : g[i].cols) * w, off = at > e.from ? (at - e.from) % ld : 0;
                if (off < (uintptr_t)g[i].cols * w || off + 4 > ld) return fail(DMMV_ERR_SHAPE, "%s is a number of gradient %lld", what, (long long)i);
            }
        }
    return DMMV_OK;
}

// Numbers a chunk: PIECE while chunks of four would be fewer than the workgroups of a launch (norm and scaling of 1.3 M numbers: 8.4 us, 12 with four).
static int chunk_of(int64_t count, const dmmv_gradient* g) {
    double n = 0.0;
    for (int64_t i = 0; i < count; ++i) n += (double)g[i].rows * (double)g[i].cols;
    return n < (double)GROUPS * 4 * PIECE ? PIECE : 4 * PIECE;
}

// lists of at most LIST tensors that hold something: f(list, its number)
template <class F>
static dmmv_status for_lists(int64_t count, const dmmv_gradient* g, const dmmv_gradient* out, int chunk, F f) {
    TensorList l;
    l.count = 0;
    l.chunks = 0;
    int32_t k = 0;
    for (int64_t i = 0; i < count; ++i) {
        if (nothing(g[i])) continue;
        const bool whole = no_gaps(g[i]) && (!out || no_gaps(out[i]));
        const int64_t rows = whole ? 1 : g[i].rows, cols = whole ? g[i].rows * g[i].cols : g[i].cols;
        const int64_t many = !whole && cols <= SHORT ? PIECE / cols : 0;
        const int64_t chunks = many ? ceil_div(rows, many) : rows * ceil_div(cols, chunk);
        if (chunks > INT32_MAX) return fail(DMMV_ERR_SHAPE, "gradient %lld: more pieces than a launch takes", (long long)i);
        if (l.count == LIST || l.chunks + (uint64_t)chunks > INT32_MAX) {
            DMMV_TRY(f(l, k++));
            l.count = 0;
            l.chunks = 0;
        }
        TensorPlace& t = l.t[l.count++];
        t.in = g[i].data;
        t.out = out ? out[i].data : nullptr;
        t.cols = cols;
        t.ld = whole ? cols : g[i].ld;
        t.ldo = whole ? cols : out ? out[i].ld : 0;
        t.rows = (uint32_t)rows;
        t.many = (uint32_t)many;
        t.first = l.chunks;
        t.in_bf16 = g[i].dtype == DMMV_BF16;
        t.out_bf16 = out && out[i].dtype == DMMV_BF16;
        l.chunks += (uint32_t)chunks;
    }
    return l.count ? f(l, k) : DMMV_OK;
}

// parts[n] of the lists, one after the other
static dmmv_status squares(int64_t count, const dmmv_gradient* g, double* part, int32_t& parts, hipStream_t s) {
    parts = 0;
    const int chunk = chunk_of(count, g);
    return for_lists(count, g, nullptr, chunk, [&](const TensorList& l, int32_t) -> dmmv_status {
        const int32_t n = (int32_t)std::min<uint32_t>(l.chunks, GROUPS);
        hipLaunchKernelGGL(chunk == PIECE ? k_gradient_squares<PIECE> : k_gradient_squares<4 * PIECE>, dim3((unsigned)n), dim3(256), 0, s, l, part + parts);
        DMMV_LAUNCH_CHECK();
        parts += n;
        return DMMV_OK;
    });
}

static dmmv_status gradient_workspace(int64_t count, const dmmv_gradient* g, size_t& bytes) {
    bytes = 0;
    return for_lists(count, g, nullptr, chunk_of(count, g), [&](const TensorList& l, int32_t) -> dmmv_status {
        bytes += std::min<uint32_t>(l.chunks, GROUPS) * sizeof(double);
        return DMMV_OK;
    });
}

}  // namespace dmmv

using namespace dmmv;

extern "C" size_t dmmv_gradient_workspace_bytes(int64_t count, const dmmv_gradient* gradients) {
    size_t bytes = 0;
    return check_gradients(count, gradients, "gradients") == DMMV_OK && gradient_workspace(count, gradients, bytes) == DMMV_OK ? bytes : 0;
}

extern "C" dmmv_status dmmv_gradient_norm(int64_t count, const dmmv_gradient* gradients, float* norm, void* workspace, size_t workspace_bytes, void* hip_stream) {
    DMMV_TRY(check_gradients(count, gradients, "gradients"));
    DMMV_TRY(layer_check_vector(norm, true, "norm"));
    size_t need = 0;
    DMMV_TRY(gradient_workspace(count, gradients, need));
    DMMV_TRY(layer_check_workspace(workspace, workspace_bytes, need));
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    int32_t parts = 0;
    DMMV_TRY(squares(count, gradients, static_cast<double*>(workspace), parts, s));
    hipLaunchKernelGGL(k_gradient_norm, dim3(1), dim3(256), 0, s, static_cast<const double*>(workspace), parts, norm);
    DMMV_LAUNCH_CHECK();
    return DMMV_OK;
}

extern "C" dmmv_status dmmv_gradient_clip(int64_t count, const dmmv_gradient* gradients, const dmmv_gradient* out, float max_norm, float eps,
                                          const float* given, float* norm, void* workspace, size_t workspace_bytes, void* hip_stream) {
    DMMV_TRY(check_gradients(count, gradients, "gradients"));
    if (out) {
        DMMV_TRY(check_gradients(count, out, "out"));
        for (int64_t i = 0; i < count; ++i)
            if (out[i].rows != gradients[i].rows || out[i].cols != gradients[i].cols)
                return fail(DMMV_ERR_SHAPE, "out: gradient %lld is %lld x %lld, expected %lld x %lld", (long long)i, (long long)out[i].rows, (long long)out[i].cols,
                            (long long)gradients[i].rows, (long long)gradients[i].cols);
    }
    if (!(max_norm >= 0.0f && max_norm <= 3.4e38f)) return fail(DMMV_ERR_DOMAIN, "max_norm must be finite and not negative");
    if (!(eps >= 0.0f && eps <= 3.4e38f)) return fail(DMMV_ERR_DOMAIN, "eps must be finite and not negative");
    DMMV_TRY(layer_check_vector(given, false, "given"));
    DMMV_TRY(layer_check_vector(norm, false, "norm"));
    DMMV_TRY(check_apart(count, out ? out : gradients, out ? gradients : nullptr));
    size_t need = 0;
    DMMV_TRY(gradient_workspace(count, gradients, need));                // (refuses what the launches would)
    if (!given) DMMV_TRY(layer_check_workspace(workspace, workspace_bytes, need));
    DMMV_TRY(check_norm_apart(given, count, out ? out : gradients, "given"));
    DMMV_TRY(check_norm_apart(norm, count, gradients, "norm"));
    if (out) DMMV_TRY(check_norm_apart(norm, count, out, "norm"));
    const int chunk = chunk_of(count, gradients);
    if (out) DMMV_TRY(for_lists(count, gradients, out, chunk, [](const TensorList&, int32_t) -> dmmv_status { return DMMV_OK; }));
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    double* part = static_cast<double*>(workspace);
    int32_t parts = 0, lists = 0;
    if (!given) DMMV_TRY(squares(count, gradients, part, parts, s));
    if (parts > 2 * GROUPS) {
        hipLaunchKernelGGL(k_gradient_total, dim3(1), dim3(256), 0, s, part, parts);
        DMMV_LAUNCH_CHECK();
        parts = 1;
    }
    DMMV_TRY(for_lists(count, gradients, out ? out : gradients, chunk, [&](const TensorList& l, int32_t k) -> dmmv_status {
        hipLaunchKernelGGL(chunk == PIECE ? k_gradient_scale<PIECE> : k_gradient_scale<4 * PIECE>, dim3((unsigned)std::min<uint32_t>(l.chunks, GROUPS)), dim3(256), 0, s, l, part, parts, given, max_norm, eps,
                           (int32_t)!out, k == 0 ? norm : nullptr);
        DMMV_LAUNCH_CHECK();
        lists = k + 1;
        return DMMV_OK;
    }));
    if (lists == 0 && norm) {                  // nothing to scale
        TensorList none;
        none.count = 0;
        none.chunks = 0;
        hipLaunchKernelGGL(k_gradient_scale<PIECE>, dim3(1), dim3(256), 0, s, none, part, 0, given, max_norm, eps, 1, norm);
        DMMV_LAUNCH_CHECK();
    }
    return DMMV_OK;
}
