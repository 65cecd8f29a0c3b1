// Distillation of a scoring head from lists of a teacher's nearest items.
//
// Row r has student logits x_v over V items, s_v = scale * x_v, q = softmax(s), and a list of ids with teacher scores
// z_j = teacher_scale * value_j; entries are those with an id below V and a score above -inf (an id listed twice counts once,
// with the sum of its probabilities).  p_j = exp(z_j - L), L = logsumexp of the list, or the caller's logsumexp over everything
// the teacher scored; then the remaining mass p_r = max(0, 1 - sum p) faces the student's mass off the list, q_r.
//     loss = sum_j p_j (log p_j - log q_j)  [+ p_r (log p_r - log q_r)]
//     d loss / d x_v = scale (q_v - p_v) on the list, scale c q_v off it, c = 1 [1 - p_r / q_r].
// Statistics and sums are held in 32 bits.  The mass off the list is summed directly (the listed items are marked bit by bit), not as
// one minus the listed mass: a student that has learnt its list leaves little there.
//
// A row is a one-pass reduction (running maximum, sum rescaled when it moves) and one more pass for the gradient.  Few rows are cut
// into slices whose partial results a second launch joins; the order of every sum is fixed, so a call gives the same bits each time.
#include "icq_types.h"

#include <float.h>

namespace {

constexpr int T = 256;
constexpr int CHUNK = 65536;       // elements marked at a time
constexpr float LOG2E = 1.44269504088896340736f;

struct Distill {
    const void *x;
    int64_t R, V, ld;
    float scale, a2;               // a2 = scale * log2(e)
    const uint32_t *ids;
    const float *values;
    int topk, slots;               // slots: size of the duplicate table, a power of two >= 2 * topk
    float teacher_scale;
    const float *teacher_lse;
    float *loss;
    float4 *stats;                 // [R] maximum of x, sum of exp, c, 1 if the row counts
    const float *grad_loss;
    void *grad;
    int64_t ld_grad;
    int splits;
    float4 *part;                  // [R][splits] maximum, sum, sum off the list
};

__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ float block_sum(float v, float *red) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
    for (int w = 1; w < (int)blockDim.x / 64; ++w) v += red[w];
    return v;
}

__device__ __forceinline__ float block_max(float v, float *red) {      // NaN does not count
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d, 64));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
    for (int w = 1; w < (int)blockDim.x / 64; ++w) v = fmaxf(v, red[w]);
    return v;
}

// The row's list in LDS.  id[j] = ICQ_PAD_ID where position j holds no entry of its own.
struct List {
    uint32_t id[ICQ_MAX_TOPK];
    float p[ICQ_MAX_TOPK], log_p[ICQ_MAX_TOPK];
    uint32_t slot_id[2 * ICQ_MAX_TOPK];                 // the ids, by hash
    float red[16];
    uint32_t twice;
};

// Fills the list; returns the number of entries (distinct ids) and the sum of their probabilities.  All threads of the block.
__device__ int load_list(const Distill &a, int64_t row, List &l, float &sum_p) {
    const int tid = threadIdx.x, n = blockDim.x;
    for (int i = tid; i < a.slots; i += n) l.slot_id[i] = ICQ_PAD_ID;
    if (tid == 0) l.twice = 0;
    float top = -INFINITY;
    for (int j = tid; j < a.topk; j += n) {
        const uint32_t id = a.ids[row * a.topk + j];
        const float z = a.teacher_scale * a.values[row * a.topk + j];
        const bool entry = (int64_t)id < a.V && !(z == -INFINITY);
        l.id[j] = entry ? id : ICQ_PAD_ID;
        l.p[j] = entry ? z : -INFINITY;
        if (entry) top = fmaxf(top, z);
    }
    top = block_max(top, l.red);                       // (its barriers also cover the tables)
    float lse = 0.0f, ref = 0.0f;
    if (a.teacher_lse) {
        ref = a.teacher_lse[row];
    } else if (top > -INFINITY) {
        ref = top;
        float s = 0.0f;
        for (int j = tid; j < a.topk; j += n)
            if (l.id[j] != ICQ_PAD_ID) s += expf(l.p[j] - top);
        lse = logf(block_sum(s, l.red));
    }
    for (int j = tid; j < a.topk; j += n) {
        const uint32_t id = l.id[j];
        if (id == ICQ_PAD_ID) { l.p[j] = 0.0f; continue; }
        const float lp = (l.p[j] - ref) - lse;
        l.log_p[j] = lp;
        l.p[j] = expf(lp);
        uint32_t at = (id * 0x9E3779B1u) >> 16 & (uint32_t)(a.slots - 1);
        for (;;) {                                     // slots >= 2 * topk: an empty one is found
            const uint32_t was = atomicCAS(&l.slot_id[at], ICQ_PAD_ID, id);
            if (was == id) l.twice = 1;
            if (was == ICQ_PAD_ID || was == id) break;
            at = (at + 1) & (uint32_t)(a.slots - 1);
        }
    }
    __syncthreads();
    if (l.twice) {                                     // every id's probability to its first place
        float p[4];
        bool first[4];
        static_assert(ICQ_MAX_TOPK <= 4 * T, "places per thread");
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int j = u * n + tid;
            p[u] = 0.0f;
            first[u] = true;
            if (j < a.topk && l.id[j] != ICQ_PAD_ID) {
                for (int i = 0; i < a.topk; ++i)
                    if (l.id[i] == l.id[j]) { if (i < j) first[u] = false; p[u] += l.p[i]; }
            }
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int j = u * n + tid;
            if (j < a.topk && l.id[j] != ICQ_PAD_ID) {
                if (first[u]) { l.p[j] = p[u]; l.log_p[j] = logf(p[u]); }
                else { l.p[j] = 0.0f; l.id[j] = ICQ_PAD_ID; }
            }
        }
        __syncthreads();
    }
    float s = 0.0f, count = 0.0f;
    for (int j = tid; j < a.topk; j += n)
        if (l.id[j] != ICQ_PAD_ID) { s += l.p[j]; count += 1.0f; }
    sum_p = block_sum(s, l.red);
    return (int)block_sum(count, l.red);
}

// Where a row's elements lie: `head` single elements, `body` groups of PER that start on 16 bytes, then `tail` single ones.
struct Span {
    int head, tail;
    int64_t body;
};

template <int TYPE>
__device__ __forceinline__ Span span_of(const void *row, int64_t V) {
    typedef IcqElem<TYPE> E;
    Span s;
    const int64_t head = (int64_t)((16 - ((uintptr_t)row & 15)) & 15) / (int64_t)sizeof(typename E::raw);
    s.head = (int)(head < V ? head : V);
    s.body = (V - s.head) / E::PER;
    s.tail = (int)(V - s.head - s.body * E::PER);
    return s;
}

// Running maximum and sums of exp(scale * (x - maximum)).
struct Run {
    float m, s, r;                 // r: off the list
};

__device__ __forceinline__ void run_join(Run &a, const Run &b, float a2) {
    const float m = fmaxf(a.m, b.m), fa = ex2((a.m - m) * a2), fb = ex2((b.m - m) * a2);
    a.s = a.s * fa + b.s * fb;
    a.r = a.r * fa + b.r * fb;
    a.m = m;
}

template <int N, bool REST>
__device__ __forceinline__ void run_add(Run &a, const float *x, uint32_t listed, float a2) {
    float m = a.m;
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, x[i]);
    if (m > a.m) {
        const float f = ex2((a.m - m) * a2);
        a.s *= f;
        if (REST) a.r *= f;
        a.m = m;
    }
    float s = 0.0f, l = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float e = ex2((x[i] - m) * a2);
        s += e;
        if (REST) l += (listed >> i & 1u) ? 0.0f : e;
    }
    a.s += s;
    if (REST) a.r += l;
}

// Block-wide: the join of all threads' runs, in a fixed order.
__device__ __forceinline__ Run block_run(Run a, float a2, float *red) {
    const float m = block_max(a.m, red);
    const float f = ex2((a.m - m) * a2);
    Run b;
    b.m = m;
    b.s = block_sum(a.s * f, red);
    b.r = block_sum(a.r * f, red);
    return b;
}

// Loss and statistics of a row from its sums; all threads of the block.
template <int TYPE>
__device__ void finish_row(const Distill &a, int64_t row, List &l, int entries, float sum_p, const Run &run) {
    typedef IcqElem<TYPE> E;
    const typename E::raw *x = static_cast<const typename E::raw *>(a.x) + row * a.ld;
    const float log_s = logf(run.s);
    float sum = 0.0f;
    for (int j = threadIdx.x; j < a.topk; j += blockDim.x) {
        const float p = l.p[j];
        if (l.id[j] != ICQ_PAD_ID && !(p == 0.0f)) sum += p * (l.log_p[j] - (a.scale * (E::get(x[l.id[j]]) - run.m) - log_s));
    }
    sum = block_sum(sum, l.red);
    if (threadIdx.x != 0) return;
    const bool counts = entries > 0 && !(run.s == 0.0f);
    float c = 1.0f;
    if (a.teacher_lse && (int64_t)entries < a.V) {
        const float p_r = fmaxf(0.0f, 1.0f - sum_p);
        if (p_r > 0.0f) sum += p_r * (logf(p_r) - (logf(run.r) - log_s));
        if (run.r > 0.0f) c = 1.0f - p_r * run.s / run.r;          // (nothing off the list: no item takes c)
    }
    a.loss[row] = counts ? sum : 0.0f;
    if (a.stats) a.stats[row] = make_float4(run.m, run.s, c, counts ? 1.0f : 0.0f);
}

// A slice of a row: groups [b0, b1) and single elements [e0, e1) of it (the single ones numbered head first).
struct Slice {
    int64_t b0, b1, e0, e1;
};

__device__ __forceinline__ Slice slice_of(const Span &s, int k, int splits) {
    const int64_t singles = (int64_t)s.head + s.tail;
    Slice c;
    c.b0 = s.body * k / splits; c.b1 = s.body * (k + 1) / splits;
    c.e0 = singles * k / splits; c.e1 = singles * (k + 1) / splits;
    return c;
}

// Whether the list names item v.
__device__ __forceinline__ bool on_list(const List &l, int slots, uint32_t v) {
    uint32_t at = (v * 0x9E3779B1u) >> 16 & (uint32_t)(slots - 1);
    for (;;) {
        const uint32_t id = l.slot_id[at];
        if (id == v) return true;
        if (id == ICQ_PAD_ID) return false;
        at = (at + 1) & (uint32_t)(slots - 1);
    }
}

// Sums of a row (splits == 1: and its loss) or of a slice of it.  REST: also those off the list.
template <int TYPE, bool REST>
__global__ __launch_bounds__(T) void distill_forward_kernel(Distill a) {
    typedef IcqElem<TYPE> E;
    constexpr int PER = E::PER, U = 4;
    __shared__ List l;
    __shared__ uint32_t s_bits[REST ? CHUNK / 32 : 1];
    const int tid = threadIdx.x, k = (int)(blockIdx.x % (uint32_t)a.splits);
    const int64_t row = blockIdx.x / (uint32_t)a.splits;
    const typename E::raw *x = static_cast<const typename E::raw *>(a.x) + row * a.ld;
    int entries = 0;
    float sum_p = 0.0f;
    if (REST || a.splits == 1) entries = load_list(a, row, l, sum_p);
    const Span s = span_of<TYPE>(x, a.V);
    const Slice c = slice_of(s, k, a.splits);
    const uint4 *body = reinterpret_cast<const uint4 *>(x + s.head);
    Run run = {-FLT_MAX, 0.0f, 0.0f};
    for (int64_t i = c.e0 + tid; i < c.e1; i += T) {
        const int64_t v = i < s.head ? i : i + s.body * PER;
        const float y = E::get(x[v]);
        run_add<1, REST>(run, &y, REST && on_list(l, a.slots, (uint32_t)v) ? 1u : 0u, a.a2);
    }
    for (int64_t b0 = c.b0; b0 < c.b1; b0 += CHUNK / PER) {
        const int n = (int)(c.b1 - b0 < CHUNK / PER ? c.b1 - b0 : CHUNK / PER);
        if (REST) {
            __syncthreads();
            for (int i = tid; i < CHUNK / 32; i += T) s_bits[i] = 0;
            __syncthreads();
            for (int j = tid; j < a.topk; j += T) {
                const int64_t e = (int64_t)l.id[j] - s.head - b0 * PER;
                if (l.id[j] != ICQ_PAD_ID && e >= 0 && e < (int64_t)n * PER) atomicOr(&s_bits[e >> 5], 1u << (e & 31));
            }
            __syncthreads();
        }
        const uint4 *from = body + b0;
        for (int i = tid; i < n; i += U * T) {
            uint4 w[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * T < n) w[u] = from[i + u * T];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * T < n) {
                    float y[PER];
                    E::unpack(w[u], y);
                    const int e = (i + u * T) * PER;
                    run_add<PER, REST>(run, y, REST ? s_bits[e >> 5] >> (e & 31) : 0u, a.a2);
                }
        }
    }
    run = block_run(run, a.a2, l.red);
    if (a.splits == 1) finish_row<TYPE>(a, row, l, entries, sum_p, run);
    else if (tid == 0) a.part[row * a.splits + k] = make_float4(run.m, run.s, run.r, 0.0f);
}

// A row's sums from its slices', and its loss.
template <int TYPE>
__global__ __launch_bounds__(T) void distill_join_kernel(Distill a) {
    __shared__ List l;
    const int64_t row = blockIdx.x;
    float sum_p;
    const int entries = load_list(a, row, l, sum_p);
    Run run = {-FLT_MAX, 0.0f, 0.0f};
    for (int k = threadIdx.x; k < a.splits; k += T) {
        const float4 p = a.part[row * a.splits + k];
        const Run b = {p.x, p.y, p.z};
        run_join(run, b, a.a2);
    }
    run = block_run(run, a.a2, l.red);
    finish_row<TYPE>(a, row, l, entries, sum_p, run);
}

// The gradient of a slice of a row.  VEC: logits and gradient rows start at the same place within 16 bytes.
template <int TYPE, bool VEC>
__global__ __launch_bounds__(T) void distill_backward_kernel(Distill a) {
    typedef IcqElem<TYPE> E;
    constexpr int PER = E::PER, U = 4;
    __shared__ List l;
    const int tid = threadIdx.x, k = (int)(blockIdx.x % (uint32_t)a.splits);
    const int64_t row = blockIdx.x / (uint32_t)a.splits;
    const typename E::raw *x = static_cast<const typename E::raw *>(a.x) + row * a.ld;
    typename E::raw *out = static_cast<typename E::raw *>(a.grad) + row * a.ld_grad;
    Span s;
    if (VEC) s = span_of<TYPE>(x, a.V);
    else { s.head = (int)a.V; s.body = 0; s.tail = 0; }
    const Slice c = slice_of(s, k, a.splits);
    const float4 st = a.stats[row];
    const uint4 *body = reinterpret_cast<const uint4 *>(x + s.head);
    uint4 *body_out = reinterpret_cast<uint4 *>(out + s.head);
    if (st.w == 0.0f) {                                // a row that does not count
        for (int64_t i = c.e0 + tid; i < c.e1; i += T) out[i < s.head ? i : i + s.body * PER] = E::put(0.0f);
        for (int64_t b = c.b0 + tid; b < c.b1; b += T) body_out[b] = make_uint4(0, 0, 0, 0);
        return;
    }
    float sum_p;
    load_list(a, row, l, sum_p);
    const float g = (a.grad_loss ? a.grad_loss[row] : 1.0f) * a.scale, q0 = 1.0f / st.y, f = q0 * st.z * g;
    // the listed items of this slice, before anything is written (the gradient may take the logits' place)
    float mine[ICQ_MAX_TOPK / T];
#pragma unroll
    for (int u = 0; u < ICQ_MAX_TOPK / T; ++u) {
        const int j = u * T + tid;
        bool here = false;
        if (j < a.topk && l.id[j] != ICQ_PAD_ID) {
            const int64_t v = l.id[j], e = v - s.head;
            if (e >= 0 && e < s.body * PER) here = e / PER >= c.b0 && e / PER < c.b1;
            else here = (e < 0 ? v : v - s.body * PER) >= c.e0 && (e < 0 ? v : v - s.body * PER) < c.e1;
            if (here) mine[u] = (ex2((E::get(x[v]) - st.x) * a.a2) * q0 - l.p[j]) * g;
        }
        if (j < a.topk && !here) l.id[j] = ICQ_PAD_ID;
    }
    __syncthreads();
    for (int64_t i = c.e0 + tid; i < c.e1; i += T) {
        const int64_t v = i < s.head ? i : i + s.body * PER;
        out[v] = E::put(ex2((E::get(x[v]) - st.x) * a.a2) * f);
    }
    for (int64_t b = c.b0 + tid; b < c.b1; b += U * T) {
        uint4 w[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (b + u * T < c.b1) w[u] = body[b + u * T];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (b + u * T < c.b1) {
                float y[PER];
                E::unpack(w[u], y);
#pragma unroll
                for (int i = 0; i < PER; ++i) y[i] = ex2((y[i] - st.x) * a.a2) * f;
                body_out[b + u * T] = E::pack(y);
            }
    }
    __syncthreads();                                   // the listed items' values replace the ones just written
#pragma unroll
    for (int u = 0; u < ICQ_MAX_TOPK / T; ++u) {
        const int j = u * T + tid;
        if (j < a.topk && l.id[j] != ICQ_PAD_ID) out[l.id[j]] = E::put(mine[u]);
    }
}

// Slices per row: enough blocks for the chip, none shorter than 8192 elements.
int splits_of(int64_t R, int64_t V, int num_cu) {
    const int64_t want = (8ll * num_cu + R - 1) / (R > 0 ? R : 1), most = V / 8192;
    const int64_t n = want < most ? want : most;
    return (int)(n < 1 ? 1 : n > 1024 ? 1024 : n);
}

size_t part_bytes(int64_t R, int splits) { return icq_align_up((size_t)R * splits * sizeof(float4), ICQ_ALIGN); }

bool shape_ok(const void *logits, int type, int64_t R, int64_t V, int64_t ld, float scale, const uint32_t *ids, const float *values,
              int topk, float teacher_scale) {
    const int size = icq_type_bytes(type);
    if (size == 0 || R < 0 || R > ICQ_MAX_Q || V < 1 || V > ICQ_MAX_EXTENT || ld < V || topk < 1 || topk > ICQ_MAX_TOPK) return false;
    if (!(scale > 0.0f) || !(scale <= FLT_MAX) || !(teacher_scale >= -FLT_MAX && teacher_scale <= FLT_MAX)) return false;
    return R == 0 || (logits && ids && values && (uintptr_t)logits % size == 0);
}

Distill params(const void *logits, int64_t R, int64_t V, int64_t ld, float scale, const uint32_t *ids, const float *values, int topk,
               float teacher_scale, const float *teacher_lse) {
    Distill a;
    a.x = logits; a.R = R; a.V = V; a.ld = ld;
    a.scale = scale; a.a2 = scale * LOG2E;
    a.ids = ids; a.values = values; a.topk = topk;
    a.slots = 32;
    while (a.slots < 2 * topk) a.slots *= 2;
    a.teacher_scale = teacher_scale; a.teacher_lse = teacher_lse;
    a.loss = nullptr; a.stats = nullptr; a.grad_loss = nullptr; a.grad = nullptr; a.ld_grad = 0;
    a.splits = 1; a.part = nullptr;
    return a;
}

int launch_backward(const Distill &a, int type, hipStream_t s) {
    const int size = icq_type_bytes(type);
    const bool vec = ((uintptr_t)a.grad - (uintptr_t)a.x) % 16 == 0 && ((a.ld_grad - a.ld) * size) % 16 == 0;
    const dim3 grid((uint32_t)(a.R * a.splits));
    ICQ_FOR_TYPE(type,
        if (vec) hipLaunchKernelGGL(HIP_KERNEL_NAME(distill_backward_kernel<TYPE, true>), grid, dim3(T), 0, s, a);
        else hipLaunchKernelGGL(HIP_KERNEL_NAME(distill_backward_kernel<TYPE, false>), grid, dim3(T), 0, s, a))
    return icq_check_launch();
}

bool grad_ok(const void *logits, int type, int64_t V, int64_t ld, const void *grad, int64_t ld_grad) {
    return grad && ld_grad >= V && (uintptr_t)grad % icq_type_bytes(type) == 0 && (grad != logits || ld_grad == ld);
}

}  // namespace

ICQ_EXPORT int icq_distill_workspace_bytes(int64_t R, int64_t V, size_t *out) {
    if (!out || R < 0 || R > ICQ_MAX_Q || V < 1 || V > ICQ_MAX_EXTENT) return ICQ_ERR_ARG;
    const int cu = icq_num_cu();
    if (cu <= 0) return ICQ_ERR_HIP;
    *out = part_bytes(R, splits_of(R, V, cu)) + part_bytes(R, 1);
    return ICQ_OK;
}

ICQ_EXPORT int icq_distill(const void *logits, int type, int64_t R, int64_t V, int64_t ld, float scale, const uint32_t *ids,
                           const float *values, int topk, float teacher_scale, const float *teacher_lse, float *loss, float *stats,
                           const float *grad_loss, void *grad, int64_t ld_grad, void *workspace, size_t workspace_bytes, void *stream) {
    if (!shape_ok(logits, type, R, V, ld, scale, ids, values, topk, teacher_scale)) return ICQ_ERR_ARG;
    if (R == 0) return ICQ_OK;
    if (!loss || (uintptr_t)stats % 16 != 0 || (grad && !grad_ok(logits, type, V, ld, grad, ld_grad))) return ICQ_ERR_ARG;
    const int cu = icq_num_cu();
    if (cu <= 0) return ICQ_ERR_HIP;
    Distill a = params(logits, R, V, ld, scale, ids, values, topk, teacher_scale, teacher_lse);
    a.splits = splits_of(R, V, cu);
    const size_t parts = part_bytes(R, a.splits);
    if (!workspace || (uintptr_t)workspace % ICQ_ALIGN != 0 || workspace_bytes < parts + part_bytes(R, 1)) return ICQ_ERR_WORKSPACE;
    a.part = static_cast<float4 *>(workspace);
    a.loss = loss;
    a.stats = stats ? reinterpret_cast<float4 *>(stats) : reinterpret_cast<float4 *>(static_cast<char *>(workspace) + parts);
    a.grad_loss = grad_loss; a.grad = grad; a.ld_grad = ld_grad;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const dim3 grid((uint32_t)(R * a.splits));
    ICQ_FOR_TYPE(type,
        if (teacher_lse) hipLaunchKernelGGL(HIP_KERNEL_NAME(distill_forward_kernel<TYPE, true>), grid, dim3(T), 0, s, a);
        else hipLaunchKernelGGL(HIP_KERNEL_NAME(distill_forward_kernel<TYPE, false>), grid, dim3(T), 0, s, a);
        if (a.splits > 1) hipLaunchKernelGGL(HIP_KERNEL_NAME(distill_join_kernel<TYPE>), dim3((uint32_t)R), dim3(T), 0, s, a))
    const int rc = icq_check_launch();
    return rc == ICQ_OK && grad ? launch_backward(a, type, s) : rc;
}

ICQ_EXPORT int icq_distill_backward(const void *logits, int type, int64_t R, int64_t V, int64_t ld, float scale, const uint32_t *ids,
                                    const float *values, int topk, float teacher_scale, const float *teacher_lse, const float *stats,
                                    const float *grad_loss, void *grad, int64_t ld_grad, void *stream) {
    if (!shape_ok(logits, type, R, V, ld, scale, ids, values, topk, teacher_scale)) return ICQ_ERR_ARG;
    if (R == 0) return ICQ_OK;
    if (!stats || (uintptr_t)stats % 16 != 0 || !grad_ok(logits, type, V, ld, grad, ld_grad)) return ICQ_ERR_ARG;
    const int cu = icq_num_cu();
    if (cu <= 0) return ICQ_ERR_HIP;
    Distill a = params(logits, R, V, ld, scale, ids, values, topk, teacher_scale, teacher_lse);
    a.splits = splits_of(R, V, cu);
    a.stats = reinterpret_cast<float4 *>(const_cast<float *>(stats));
    a.grad_loss = grad_loss; a.grad = grad; a.ld_grad = ld_grad;
    return launch_backward(a, type, static_cast<hipStream_t>(stream));
}
