// The global norm of many gradients, and clipping by it.
//
// A list is cut into chunks of about 32 KB at its creation; a table of them on the device gives a block all it needs to know of a chunk with one
// read, so that any number of tensors of any sizes is one launch.  Squares and their sums are held in 64 bits: no gradient over- or underflows them,
// and the sums' order is fixed by the list and the number of compute units.
//
// Both passes are bound by memory.  The first reads at 6.1 TB/s (1.2e8 f32, 82 us); what the last-level cache can keep is read through it, the
// rest past it.  The second begins with what was read last, and writes past the caches: 3.7e8 f16 into f32 in 563 us with both, 6e7 f32
// into f32 in 120 (148 with stores through the caches).  Short lists are bound by two launches and their chains of reads: 5 to 7 us; one
// block of 1024 threads that did such a list in one launch took 5 to 12.
#include "icq_overlap.h"
#include "icq_types.h"

#include <math.h>

#include <algorithm>
#include <vector>

namespace {

constexpr int THREADS = 256;
constexpr int64_t CHUNK = 1 << 15;                     // bytes of a chunk's wider side
constexpr int64_t CACHED = 192 << 20;                  // of the last-level cache's 256 MB

// Rows of `cols` values, ld apart (one row: a stretch of a tensor without gaps).
struct Chunk {
    const void *g;
    void *out;
    int64_t ld, ld_out;
    uint32_t rows, cols;
    int type, out_type;
};

}  // namespace

struct icq_grad_list {
    Chunk *chunks;             // device; nullptr where there are none
    int count, blocks;         // chunks; blocks of the first pass, whose partial sums the workspace holds
    int clip_blocks, keep;     // blocks of the second; the chunks from keep on are those that the last-level cache holds
    int device;
};

namespace {

// Values that a thread takes at a time: 16 bytes of the narrower of its types, or 8 beside 16 of the wider, so that a wavefront's loads and stores are
// whole stretches (eight 16-bit values beside eight of 32 bits, 32 bytes a lane in two stores: 3.2 TB/s).
template <int FROM, int TO>
constexpr int at_once() { return FROM == ICQ_F32 || TO == ICQ_F32 ? 4 : 8; }

template <int TYPE, int N>
struct Values { uint32_t w[N * (TYPE == ICQ_F32 ? 4 : 2) / 4]; };

template <int TYPE, int N>
__device__ __forceinline__ void unpack(const Values<TYPE, N> &v, float *x) {
    if constexpr (TYPE == ICQ_F32) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = __uint_as_float(v.w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) IcqElem<TYPE>::unpack2(v.w[i], x + 2 * i);
    }
}

template <int TYPE, int N>
__device__ __forceinline__ Values<TYPE, N> pack(const float *x) {
    Values<TYPE, N> v;
    if constexpr (TYPE == ICQ_F32) {
#pragma unroll
        for (int i = 0; i < N; ++i) v.w[i] = __float_as_uint(x[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) v.w[i] = IcqElem<TYPE>::pack2(x[2 * i], x[2 * i + 1]);
    }
    return v;
}

// A thread's 8 or 16 bytes from or to any address, past the caches: what is used once should not put out what is used again.
template <int BYTES> struct Stretch;
template <> struct Stretch<16> { typedef uint32_t T __attribute__((ext_vector_type(4), aligned(2))); };
template <> struct Stretch<8> { typedef uint32_t T __attribute__((ext_vector_type(2), aligned(2))); };

template <bool PAST, typename V>
__device__ __forceinline__ void read(V &v, const void *from) {
    typedef typename Stretch<sizeof(V)>::T T;
    T t;
    if constexpr (PAST) t = __builtin_nontemporal_load(static_cast<const T *>(from));
    else t = *static_cast<const T *>(from);
    __builtin_memcpy(&v, &t, sizeof v);
}

template <typename V>
__device__ __forceinline__ void write(void *to, const V &v) {
    typedef typename Stretch<sizeof(V)>::T T;
    T t;
    __builtin_memcpy(&t, &v, sizeof v);
    __builtin_nontemporal_store(t, static_cast<T *>(to));
}

// Visits a chunk's values: take(place in g, place in out, its raw values) for N neighbours at a time, LOADS of them requested before the first is taken, and one(place in g,
// place in out) for what is left.
template <int TYPE, int N, int LOADS, bool PAST, typename F, typename G>
__device__ __forceinline__ void visit(const Chunk &c, F take, G one) {
    typedef typename IcqElem<TYPE>::raw raw;
    const raw *g = static_cast<const raw *>(c.g);
    if (c.rows == 1) {
        constexpr uint32_t STEP = THREADS * N;
        const uint32_t groups = c.cols / N;                                   // whole ones
        uint32_t i = threadIdx.x;
        for (; i + (LOADS - 1) * THREADS < groups; i += LOADS * THREADS) {
            Values<TYPE, N> v[LOADS];
#pragma unroll
            for (int k = 0; k < LOADS; ++k) read<PAST>(v[k], g + (size_t)i * N + k * STEP);
#pragma unroll
            for (int k = 0; k < LOADS; ++k) take((int64_t)i * N + k * STEP, (int64_t)i * N + k * STEP, v[k]);
        }
        for (; i < groups; i += THREADS) {
            Values<TYPE, N> v;
            read<PAST>(v, g + (size_t)i * N);
            take((int64_t)i * N, (int64_t)i * N, v);
        }
        const uint32_t rest = groups * N + threadIdx.x;
        if (rest < c.cols) one(rest, rest);
    } else {
        const uint32_t groups = c.cols / N, rest = c.cols % N;
        for (uint32_t i = threadIdx.x; i < c.rows * groups; i += THREADS) {
            const uint32_t r = i / groups, k = i % groups * N;
            Values<TYPE, N> v;
            read<PAST>(v, g + (int64_t)r * c.ld + k);
            take((int64_t)r * c.ld + k, (int64_t)r * c.ld_out + k, v);
        }
        for (uint32_t i = threadIdx.x; i < c.rows * rest; i += THREADS) {
            const uint32_t r = i / rest, k = groups * N + i % rest;
            one((int64_t)r * c.ld + k, (int64_t)r * c.ld_out + k);
        }
    }
}

// The block's sum of x, in all threads; s: one value for each wavefront.
__device__ __forceinline__ double block_sum(double x, double *s) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d, 64);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) x += s[w];
    return x;
}

template <int TYPE, bool PAST>
__device__ __forceinline__ double squares(const Chunk &c) {
    constexpr int N = TYPE == ICQ_F32 ? 4 : 8;
    double sum = 0.0;
    visit<TYPE, N, 4, PAST>(c,
        [&](int64_t, int64_t, const Values<TYPE, N> &v) {
            float x[N];
            unpack<TYPE, N>(v, x);
#pragma unroll
            for (int i = 0; i < N; ++i) sum = fma((double)x[i], (double)x[i], sum);
        },
        [&](int64_t at, int64_t) {
            const double x = (double)IcqElem<TYPE>::get(static_cast<const typename IcqElem<TYPE>::raw *>(c.g)[at]);
            sum = fma(x, x, sum);
        });
    return sum;
}

// Chunks from `keep` on are read through the caches, for a second pass that begins with the last.
__global__ __launch_bounds__(THREADS) void grad_squares_kernel(const Chunk *__restrict__ chunks, int count, int keep, double *part) {
    __shared__ double s[THREADS / 64];
    double sum = 0.0;
    for (int k = blockIdx.x; k < count; k += gridDim.x) {
        const Chunk c = chunks[k];
        if (k < keep) ICQ_FOR_TYPE(c.type, sum += (squares<TYPE, true>(c)))
        else ICQ_FOR_TYPE(c.type, sum += (squares<TYPE, false>(c)))
    }
    sum = block_sum(sum, s);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

// The norm from the blocks' sums, in all threads.
__device__ __forceinline__ float join(const double *part, int n, float scale, double *s) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < n; i += THREADS) sum += part[i];
    return (float)(sqrt(block_sum(sum, s)) * (double)scale);
}

__global__ __launch_bounds__(THREADS) void grad_norm_kernel(const double *part, int n, float scale, float *norm) {
    __shared__ double s[THREADS / 64];
    const float x = join(part, n, scale, s);
    if (threadIdx.x == 0) *norm = x;
}

template <int FROM, int TO>
__device__ __forceinline__ void scale_chunk(const Chunk &c, float factor) {
    constexpr int N = at_once<FROM, TO>();
    typedef typename IcqElem<TO>::raw raw;
    raw *out = static_cast<raw *>(c.out);
    visit<FROM, N, 4, false>(c,
        [&](int64_t, int64_t to, const Values<FROM, N> &v) {
            float x[N];
            unpack<FROM, N>(v, x);
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] *= factor;
            const Values<TO, N> w = pack<TO, N>(x);
            write(out + to, w);
        },
        [&](int64_t at, int64_t to) { out[to] = IcqElem<TO>::put(IcqElem<FROM>::get(static_cast<const typename IcqElem<FROM>::raw *>(c.g)[at]) * factor); });
}

// part: the blocks' sums of the squares, from which the norm comes (block 0 writes it); nullptr: it is there.  The chunks in the reverse of the order in
// which their squares were summed: the last ones are still in the caches.
__global__ __launch_bounds__(THREADS) void grad_clip_kernel(const Chunk *__restrict__ chunks, int count, const double *part, int parts, float scale, float max_norm, float *norm) {
    __shared__ double s[THREADS / 64];
    float x;
    if (part) {
        x = join(part, parts, scale, s);
        if (blockIdx.x == 0 && threadIdx.x == 0) *norm = x;
    } else {
        x = *norm;
    }
    const float factor = x <= max_norm ? scale : scale * (max_norm / x);
    for (int k = count - 1 - blockIdx.x; k >= 0; k -= gridDim.x) {
        const Chunk c = chunks[k];
        if (factor == 1.0f && c.g == c.out) continue;
        ICQ_FOR_TYPE(c.type, constexpr int FROM = TYPE; ICQ_FOR_TYPE(c.out_type, scale_chunk<FROM, TYPE>(c, factor)))
    }
}

bool usable(const icq_grad_list *list) {
    int dev = 0;
    return list && hipGetDevice(&dev) == hipSuccess && dev == list->device;
}

bool workspace_ok(const icq_grad_list *list, const void *workspace, size_t bytes) {
    return workspace && (uintptr_t)workspace % ICQ_ALIGN == 0 && bytes >= (size_t)list->blocks * sizeof(double);
}

void sum_squares(const icq_grad_list *list, int keep, double *part, hipStream_t s) {
    hipLaunchKernelGGL(grad_squares_kernel, dim3((uint32_t)list->blocks), dim3(THREADS), 0, s, list->chunks, list->count, keep, part);
}

// A matrix's place as it is read or written.
struct Place {
    icq_extent at;
    int matrix;
    bool written;
};

// Whether some matrix that is written shares memory with another, or with what it is itself read from elsewhere than in its place.
bool overlap(std::vector<Place> &places, const std::vector<bool> &in_place) {
    std::sort(places.begin(), places.end(), [](const Place &x, const Place &y) { return x.at.from < y.at.from; });
    std::vector<const Place *> open;                                          // those that may reach beyond the present start
    for (const Place &x : places) {
        size_t kept = 0;
        for (const Place *y : open) {
            if ((__int128)y->at.from + (__int128)(y->at.rows - 1) * y->at.ld + y->at.len <= (__int128)x.at.from) continue;
            open[kept++] = y;
            if ((!x.written && !y->written) || (x.matrix == y->matrix && in_place[x.matrix])) continue;
            if (icq_extents_overlap(x.at, y->at)) return true;
        }
        open.resize(kept);
        open.push_back(&x);
    }
    return false;
}

}  // namespace

ICQ_EXPORT int icq_grad_list_create(icq_grad_list **out, const void *const *grads, const int *types, const int64_t *rows, const int64_t *cols,
                                    const int64_t *ld, void *const *outs, const int *out_types, const int64_t *ld_outs, int count, void *stream) {
    if (!out) return ICQ_ERR_ARG;
    *out = nullptr;
    if (count < 0 || (count > 0 && (!grads || !types || !rows || !cols || !ld)) || (outs && (!out_types || !ld_outs))) return ICQ_ERR_ARG;
    try {
        std::vector<Place> places;
        std::vector<bool> in_place(count);
        std::vector<Chunk> chunks;
        __int128 total = 0;
        for (int i = 0; i < count; ++i) {
            const int type = types[i], to_type = outs ? out_types[i] : type, size = icq_type_bytes(type), to_size = icq_type_bytes(to_type);
            if (size == 0 || to_size == 0 || rows[i] < 0 || cols[i] < 0 || rows[i] > ((int64_t)1 << 48) || cols[i] > ((int64_t)1 << 48)) return ICQ_ERR_ARG;
            if (rows[i] == 0 || cols[i] == 0) continue;
            const int64_t to_ld = outs ? ld_outs[i] : ld[i];
            const uintptr_t g = (uintptr_t)grads[i], to = outs ? (uintptr_t)outs[i] : g;
            if (!g || !to || g % size != 0 || to % to_size != 0 || (rows[i] > 1 && (ld[i] < cols[i] || to_ld < cols[i]))) return ICQ_ERR_ARG;
            if ((__int128)(rows[i] - 1) * std::max(ld[i], to_ld) + cols[i] > (__int128)1 << 48) return ICQ_ERR_ARG;
            total += (__int128)rows[i] * cols[i];
            in_place[i] = g == to && type == to_type && (rows[i] == 1 || ld[i] == to_ld);
            if (!in_place[i]) places.push_back({{g, rows[i], (rows[i] > 1 ? ld[i] : cols[i]) * size, cols[i] * size}, i, false});
            places.push_back({{to, rows[i], (rows[i] > 1 ? to_ld : cols[i]) * to_size, cols[i] * to_size}, i, true});
        }
        if (total > (__int128)1 << 40 || overlap(places, in_place)) return ICQ_ERR_ARG;
        int64_t longer = 1;                                                    // (a table of 2^19 chunks and one for each matrix at most: rows longer than half a chunk fill it by halves)
        while (total / (CHUNK / 4 * longer) > (1 << 18)) longer *= 2;
        for (int i = 0; i < count; ++i) {
            const int type = types[i], to_type = outs ? out_types[i] : type;
            const int64_t to_ld = outs ? ld_outs[i] : ld[i], size = CHUNK * longer / std::max(icq_type_bytes(type), icq_type_bytes(to_type));
            const auto add = [&](int64_t r, int64_t c, int64_t nr, int64_t nc) {
                Chunk k;
                k.ld = ld[i]; k.ld_out = to_ld; k.rows = (uint32_t)nr; k.cols = (uint32_t)nc; k.type = type; k.out_type = to_type;
                k.g = static_cast<const char *>(grads[i]) + (r * ld[i] + c) * icq_type_bytes(type);
                k.out = outs ? static_cast<char *>(outs[i]) + (r * to_ld + c) * icq_type_bytes(to_type) : const_cast<void *>(k.g);
                chunks.push_back(k);
            };
            if (cols[i] == 0) continue;
            const int64_t high = std::max<int64_t>(1, size / cols[i]);
            for (int64_t r = 0; r < rows[i]; r += high)
                for (int64_t c = 0; c < cols[i]; c += size) add(r, c, std::min(high, rows[i] - r), std::min(size, cols[i] - c));
        }
        if (chunks.size() > 0x7fffffff) return ICQ_ERR_ARG;
        const int cu = icq_num_cu();
        int dev = 0;
        if (cu <= 0 || hipGetDevice(&dev) != hipSuccess) return ICQ_ERR_HIP;
        icq_grad_list *list = new icq_grad_list;
        list->chunks = nullptr;
        list->count = (int)chunks.size();
        list->blocks = std::max(1, std::min(list->count, cu * 4));
        list->clip_blocks = std::max(1, std::min(list->count, cu * 2));
        int64_t kept = 0;
        for (list->keep = list->count; list->keep > 0; --list->keep) {
            const Chunk &k = chunks[list->keep - 1];
            if ((kept += (int64_t)k.rows * k.cols * icq_type_bytes(k.type)) > CACHED) break;
        }
        list->device = dev;
        if (!chunks.empty()) {
            hipStream_t s = static_cast<hipStream_t>(stream);
            const size_t bytes = chunks.size() * sizeof(Chunk);
            if (hipMalloc(reinterpret_cast<void **>(&list->chunks), bytes) != hipSuccess ||
                hipMemcpyAsync(list->chunks, chunks.data(), bytes, hipMemcpyHostToDevice, s) != hipSuccess || hipStreamSynchronize(s) != hipSuccess) {
                icq_grad_list_destroy(list);
                (void)hipGetLastError();                                       // (told here, not by the next launch's check)
                return ICQ_ERR_HIP;
            }
        }
        *out = list;
        return ICQ_OK;
    } catch (...) {                                                           // (no memory for the tables)
        return ICQ_ERR_HIP;
    }
}

ICQ_EXPORT void icq_grad_list_destroy(icq_grad_list *list) {
    if (!list) return;
    if (list->chunks) (void)hipFree(list->chunks);
    delete list;
}

ICQ_EXPORT int icq_grad_workspace_bytes(const icq_grad_list *list, size_t *out) {
    if (!list || !out) return ICQ_ERR_ARG;
    *out = icq_align_up((size_t)list->blocks * sizeof(double), ICQ_ALIGN);
    return ICQ_OK;
}

ICQ_EXPORT int icq_grad_norm(const icq_grad_list *list, float scale, float *norm, void *workspace, size_t workspace_bytes, void *stream) {
    if (!(scale >= 0.0f) || isinf(scale) || !norm || !usable(list)) return ICQ_ERR_ARG;
    if (!workspace_ok(list, workspace, workspace_bytes)) return ICQ_ERR_WORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    double *part = static_cast<double *>(workspace);
    sum_squares(list, list->count, part, s);
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(THREADS), 0, s, part, list->blocks, scale, norm);
    return icq_check_launch();
}

ICQ_EXPORT int icq_grad_clip(const icq_grad_list *list, float scale, float max_norm, const float *norm, void *stream) {
    if (!(scale >= 0.0f) || isinf(scale) || !(max_norm >= 0.0f) || !norm || !usable(list)) return ICQ_ERR_ARG;
    if (list->count == 0) return ICQ_OK;
    hipLaunchKernelGGL(grad_clip_kernel, dim3((uint32_t)list->clip_blocks), dim3(THREADS), 0, static_cast<hipStream_t>(stream), list->chunks, list->count, nullptr, 0, scale, max_norm,
                       const_cast<float *>(norm));
    return icq_check_launch();
}

ICQ_EXPORT int icq_grad_norm_clip(const icq_grad_list *list, float scale, float max_norm, float *norm, void *workspace, size_t workspace_bytes, void *stream) {
    if (!(scale >= 0.0f) || isinf(scale) || !(max_norm >= 0.0f) || !norm || !usable(list)) return ICQ_ERR_ARG;
    if (!workspace_ok(list, workspace, workspace_bytes)) return ICQ_ERR_WORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    double *part = static_cast<double *>(workspace);
    sum_squares(list, list->keep, part, s);
    hipLaunchKernelGGL(grad_clip_kernel, dim3((uint32_t)list->clip_blocks), dim3(THREADS), 0, s, list->chunks, list->count, part, list->blocks, scale, max_norm, norm);
    return icq_check_launch();
}
