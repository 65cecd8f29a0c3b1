// Distillation of a scoring head from lists of a teacher's nearest items.
//
// Row r has student logits x_v over V items, s_v = scale * x_v, q = softmax(s), and a list of ids with teacher scores
// z_j = teacher_scale * value_j; entries are those with an id below V and a score above -inf (an id listed twice counts once,
// with the sum of its probabilities).  p_j = exp(z_j - L), L = logsumexp of the list, or the caller's logsumexp over everything
// the teacher scored; then the remaining mass p_r = max(0, 1 - sum p) faces the student's mass off the list, q_r.
//     loss = sum_j p_j (log p_j - log q_j)  [+ p_r (log p_r - log q_r)]
//     gradient = scale (q_v - p_v) on the list, scale q_v [- scale p_r q_v / q_r] off it,
// d loss / d x_v where the masses p add up to one (a caller's logsumexp may make them do otherwise: S q_v would stand in q_v's place).
// Statistics and sums are held in 32 bits.  The items off the list are summed by themselves, relative to a maximum of their own (the listed
// ones are marked bit by bit and join from the list), not as one minus the listed mass: a student that has learnt its list leaves
// little there, e^-100 and less under a large scale.  log q_r and q_v / q_r follow from that sum without q_r, which may be too small to hold.
//
// A row is a one-pass reduction (running maximum, sum rescaled when it moves) and one more pass for the gradient.  Loss and gradient of
// many rows: a block per row, what the registers hold of it read once, the rest a second time.  Few rows are cut into slices whose
// partial results the gradient's launch joins.  The order of every sum is fixed, so a call gives the same bits each time.
// Bound by memory where rows are many (4096 x 131072 bf16, loss and gradient 421 us, 5.1 TB/s of one reading and one writing; a copy
// runs at 5.17), by the chain of loads and reductions of a launch where they are few (7.5 us; 8 x 10^6 f32: 23 us for two).
#include "icq_distill_plan.h"
#include "icq_overlap.h"
#include "icq_types.h"

#include <float.h>

namespace {

constexpr int T = 256;             // threads where a row is cut into slices
constexpr int CHUNK = 65536;       // elements marked at a time
constexpr int SHORT = 128;         // lists of up to so many places take less LDS
constexpr float LOG2E = 1.44269504088896340736f;

struct Distill {
    const void *x;
    int64_t R, V, ld;
    float scale, a2;               // a2 = scale * log2(e)
    float lowest;                  // the type's lowest finite value: a mask, like -inf
    const uint32_t *ids;
    const float *values;
    int topk, slots;               // slots: size of the duplicate table, a power of two >= 2 * topk
    float teacher_scale;
    const float *teacher_lse;
    float *loss;
    float4 *stats;                 // [R] maximum of x, sum of exp (0: the row does not count), base and factor of the off-list gradient
    const float *grad_loss;
    void *grad;
    int64_t ld_grad;
    int splits, num_cu;
    struct Part *part;             // [R][splits]
};

// Sums of a row or of a slice of it: maximum of x and the sum of exp(scale * (x - m)); the same of what is off the list.
struct Sums {
    float m, s, mr, r;
};

struct __attribute__((aligned(32))) Part {
    Sums sums;
    float t, p;                    // over the listed items of the slice: sum of p (x - m), sum of p
    float unused[2];
};

__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }

// Over the wavefront, in every lane: rotations within 16 lanes, then the four groups of 16.
template <int BY>
__device__ __forceinline__ float rotated(float v) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x120 + BY, 0xf, 0xf, true)); }

__device__ __forceinline__ float wave_sum(float v) {
    v += rotated<8>(v);
    v += rotated<4>(v);
    v += rotated<2>(v);
    v += rotated<1>(v);
    v += __shfl_xor(v, 16, 64);
    return v + __shfl_xor(v, 32, 64);
}

__device__ __forceinline__ float wave_max(float v) {                  // NaN does not count
    v = fmaxf(v, rotated<8>(v));
    v = fmaxf(v, rotated<4>(v));
    v = fmaxf(v, rotated<2>(v));
    v = fmaxf(v, rotated<1>(v));
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}

// Sums over the block, in a fixed order, of K values at once.
template <int N, int K>
__device__ __forceinline__ void block_sums(float (&v)[K], float *red) {
#pragma unroll
    for (int i = 0; i < K; ++i) v[i] = wave_sum(v[i]);
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < K; ++i) red[i * (N / 64) + (threadIdx.x >> 6)] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < K; ++i) {
        v[i] = red[i * (N / 64)];
#pragma unroll
        for (int w = 1; w < N / 64; ++w) v[i] += red[i * (N / 64) + w];
    }
}

// The largest of `m` (NaN does not count) and the sum of `v`.
template <int N>
__device__ __forceinline__ void block_max_and_sum(float &m, float &v, float *red) {
    m = wave_max(m);
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) { red[threadIdx.x >> 6] = m; red[N / 64 + (threadIdx.x >> 6)] = v; }
    __syncthreads();
    m = red[0];
    v = red[N / 64];
#pragma unroll
    for (int w = 1; w < N / 64; ++w) { m = fmaxf(m, red[w]); v += red[N / 64 + w]; }
}

// The row's list in LDS.  id[j] = ICQ_PAD_ID where position j holds no entry of its own.
template <int CAP>
struct List {
    uint32_t id[CAP];
    float p[CAP], log_p[CAP];
    float x[CAP];                  // the student's logit
    uint32_t slot_id[2 * CAP];     // the ids, by hash
    __attribute__((aligned(16))) float red[40];
    uint32_t twice;
};

// Fills the list (x: the row's logits, read at those listed places that `in` takes, early: they share lines with what is read next); returns the number of entries (distinct ids) and the sum of their probabilities: without the caller's logsumexp one, or NaN where a score is.  All threads of the block.
template <int TYPE, int CAP, int N, typename In>
__device__ int load_list(const Distill &a, int64_t row, const typename IcqElem<TYPE>::raw *x, List<CAP> &l, float &sum_p, In in) {
    constexpr int n = N, PLACES = (CAP + N - 1) / N;
    const int tid = threadIdx.x;
    for (int i = tid; i < a.slots; i += n) l.slot_id[i] = ICQ_PAD_ID;
    if (tid == 0) l.twice = 0;
    float top = -INFINITY, count = 0.0f, ref = a.teacher_lse ? a.teacher_lse[row] : 0.0f, log_z = 0.0f;
    typename IcqElem<TYPE>::raw logit[PLACES];         // (not waited for before they are needed)
#pragma unroll
    for (int u = 0; u < PLACES; ++u) {
        const int j = u * n + tid;
        logit[u] = IcqElem<TYPE>::put(0.0f);
        if (j >= a.topk) continue;
        const uint32_t id = a.ids[row * a.topk + j];
        const float z = a.teacher_scale * a.values[row * a.topk + j];
        const bool entry = (int64_t)id < a.V && !(z == -INFINITY);
        l.id[j] = entry ? id : ICQ_PAD_ID;
        l.p[j] = entry ? z : -INFINITY;
        if (entry) {
            top = fmaxf(top, z);
            count += 1.0f;
            if (in(id)) logit[u] = x[id];
        }
    }
    block_max_and_sum<N>(top, count, l.red);           // (its barriers also cover the table)
    const bool own_sum = !a.teacher_lse && top > -INFINITY;
    float part = 1.0f;
    if (own_sum) {                                     // p as a share of the sum: they add up to one whatever the scores' size
        float s[1] = {0.0f};
        for (int j = tid; j < a.topk; j += n)
            if (l.id[j] != ICQ_PAD_ID) {
                l.log_p[j] = l.p[j] - top;
                s[0] += l.p[j] = expf(l.log_p[j]);
            }
        block_sums<N>(s, l.red);
        log_z = logf(s[0]);
        part = 1.0f / s[0];
    }
    float sum[1] = {0.0f};
    for (int j = tid; j < a.topk; j += n) {
        const uint32_t id = l.id[j];
        if (id == ICQ_PAD_ID) { l.p[j] = 0.0f; continue; }
        const float lp = own_sum ? l.log_p[j] - log_z : l.p[j] - ref;
        l.p[j] = own_sum ? l.p[j] * part : expf(lp);
        l.log_p[j] = lp;
        sum[0] += l.p[j];
        uint32_t at = (id * 0x9E3779B1u) >> 16 & (uint32_t)(a.slots - 1);
        for (;;) {                                     // slots >= 2 * topk: an empty one is found
            const uint32_t was = atomicCAS(&l.slot_id[at], ICQ_PAD_ID, id);
            if (was == id) l.twice = 1;
            if (was == ICQ_PAD_ID || was == id) break;
            at = (at + 1) & (uint32_t)(a.slots - 1);
        }
    }
#pragma unroll
    for (int u = 0; u < PLACES; ++u)
        if (u * n + tid < a.topk) l.x[u * n + tid] = IcqElem<TYPE>::get(logit[u]);
    sum_p = own_sum ? part - part + 1.0f : top == -INFINITY && count > 0.0f ? NAN : 0.0f;      // (entries, and none of them a number)
    if (a.teacher_lse) {                               // (only then is the sum itself of any consequence)
        block_sums<N>(sum, l.red);
        sum_p = sum[0];
    }
    __syncthreads();
    if (l.twice) {                                     // every id's probability to its first place
        float p[PLACES], lost[1] = {0.0f};
        bool first[PLACES];
#pragma unroll
        for (int u = 0; u < PLACES; ++u) {
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
        for (int u = 0; u < PLACES; ++u) {
            const int j = u * n + tid;
            if (j < a.topk && l.id[j] != ICQ_PAD_ID) {
                if (first[u]) { l.p[j] = p[u]; l.log_p[j] = logf(p[u]); }
                else { l.p[j] = 0.0f; l.id[j] = ICQ_PAD_ID; lost[0] += 1.0f; }
            }
        }
        block_sums<N>(lost, l.red);
        count -= lost[0];
        __syncthreads();
    }
    return (int)count;
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

// Running maximum and sum of exp(scale * (x - maximum)).
struct Run {
    float m, s;
};

__device__ __forceinline__ void run_join(Run &a, const Run &b, float a2) {
    const float m = fmaxf(a.m, b.m);
    a.s = a.s * ex2((a.m - m) * a2) + b.s * ex2((b.m - m) * a2);
    a.m = m;
}

// REST: but for the items that the low N bits of `listed` name.
template <int N, bool REST>
__device__ __forceinline__ void run_add(Run &a, const float (&x)[N], uint32_t listed, float a2) {
    float y[N];
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = x[i];
    if (REST && (listed & ((1u << N) - 1u)))           // (few groups have any)
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] = (listed >> i & 1u) ? -INFINITY : y[i];
    float m = a.m;
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, y[i]);
    if (m > a.m) {
        a.s *= ex2((a.m - m) * a2);
        a.m = m;
    }
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) s += ex2((y[i] - m) * a2);
    a.s += s;
}

// The larger of two maxima each of the block.
template <int N>
__device__ __forceinline__ void block_max2(float &a, float &b, float *red) {
    a = wave_max(a);
    b = wave_max(b);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) { red[threadIdx.x >> 6] = a; red[N / 64 + (threadIdx.x >> 6)] = b; }
    __syncthreads();
    a = red[0];
    b = red[N / 64];
#pragma unroll
    for (int w = 1; w < N / 64; ++w) { a = fmaxf(a, red[w]); b = fmaxf(b, red[N / 64 + w]); }
}

// Block-wide, in a fixed order: the join of all threads' runs; REST: these are of what is off the list, and those listed items that `in`
// takes join from the list.  listed: this thread's share of what the loss needs of the latter, sum of p (x - m) and sum of p.
template <bool REST, int CAP, int N, typename In>
__device__ __forceinline__ Sums block_run(const Run &a, const Distill &d, List<CAP> &l, In in, float (&listed)[2]) {
    constexpr int PLACES = (CAP + N - 1) / N;
    Sums b = {a.m, 0.0f, a.m, 0.0f};
    float x[PLACES], p[PLACES];                        // (p = -1: no item)
#pragma unroll
    for (int u = 0; u < PLACES; ++u) {
        const int j = u * N + (int)threadIdx.x;
        const bool here = j < d.topk && l.id[j] != ICQ_PAD_ID && in(l.id[j]);
        x[u] = here ? l.x[j] : -INFINITY;
        p[u] = here ? l.p[j] : -1.0f;
        if (REST) b.m = fmaxf(b.m, x[u]);
    }
    if constexpr (!REST) {
        float none = 0.0f;
        block_max_and_sum<N>(b.m, none, l.red);
        float v[1] = {a.s * ex2((a.m - b.m) * d.a2)};
        block_sums<N>(v, l.red);
        b.s = v[0];
        b.mr = b.m;
    } else {
        block_max2<N>(b.m, b.mr, l.red);
        float v[2] = {a.s * ex2((a.m - b.mr) * d.a2), 0.0f};
#pragma unroll
        for (int u = 0; u < PLACES; ++u) v[1] += ex2((x[u] - b.m) * d.a2);
        block_sums<N>(v, l.red);
        b.r = v[0];
        b.s = v[0] * ex2((b.mr - b.m) * d.a2) + v[1];
    }
    listed[0] = listed[1] = 0.0f;
#pragma unroll
    for (int u = 0; u < PLACES; ++u)
        if (!(p[u] == 0.0f) && !(p[u] == -1.0f)) {
            listed[0] += p[u] * (x[u] - b.m);
            listed[1] += p[u];
        }
    return b;
}

// Loss and statistics of a row from its sums; listed: this thread's share of the sum of p (x - m).  All threads get the statistics.
// may_rest: false where the kernel is one without the mass off the list; counts: whether the row has a loss.
template <int CAP, int N>
__device__ __forceinline__ float4 finish_row(const Distill &a, int64_t row, List<CAP> &l, int entries, float sum_p, const Sums &run, float listed, bool write,
                                             bool may_rest, bool &counts) {
    const float log_s = logf(run.s);
    counts = entries > 0 && !(run.s == 0.0f);
    const bool with_rest = may_rest && a.teacher_lse, rest = with_rest && (int64_t)entries < a.V;
    const float p_r = rest ? (sum_p > 1.0f ? 0.0f : 1.0f - sum_p) : 0.0f;
    // the sum off the list, zero where all of it is masked: it takes no gradient then (as it is, if that is NaN)
    const float r = run.mr > a.lowest ? run.r : 0.0f * run.r;
    if (write) {                                       // (the same for the whole block)
        float sum[1] = {-a.scale * listed};
        for (int j = threadIdx.x; j < a.topk; j += N)
            if (l.id[j] != ICQ_PAD_ID && !(l.p[j] == 0.0f)) sum[0] += l.p[j] * (l.log_p[j] + log_s);
        block_sums<N>(sum, l.red);
        if (p_r > 0.0f) sum[0] += p_r * (logf(p_r) - (a.scale * (run.mr - run.m) + logf(r) - log_s));
        if (threadIdx.x == 0) a.loss[row] = counts ? sum[0] : 0.0f;
    }
    // off the list q_v - p_r q_v / q_r = exp(scale (x_v - base)) factor
    float base = run.m, factor = 1.0f / run.s;
    if (with_rest) {
        base = run.mr;
        factor = r == 0.0f ? 0.0f : ex2((run.mr - run.m) * a.a2) / run.s - p_r / r;
    }
    const bool odd = sum_p != sum_p;                   // a NaN of the teacher's: in every item's gradient, as in the loss
    const float4 st = make_float4(run.m, counts ? odd ? sum_p : run.s : 0.0f, base, odd ? sum_p : factor);
    if (write && a.stats && threadIdx.x == 0) a.stats[row] = st;
    return st;
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

__device__ __forceinline__ bool in_slice(const Span &s, const Slice &c, uint32_t id, int per) {
    const int64_t v = id, e = v - s.head;
    if (e >= 0 && e < s.body * per) return e / per >= c.b0 && e / per < c.b1;
    const int64_t single = e < 0 ? v : v - s.body * per;
    return single >= c.e0 && single < c.e1;
}

// Whether the list names item v.
template <int CAP>
__device__ __forceinline__ bool on_list(const List<CAP> &l, int slots, uint32_t v) {
    uint32_t at = (v * 0x9E3779B1u) >> 16 & (uint32_t)(slots - 1);
    for (;;) {
        const uint32_t id = l.slot_id[at];
        if (id == v) return true;
        if (id == ICQ_PAD_ID) return false;
        at = (at + 1) & (uint32_t)(slots - 1);
    }
}

// Marks the listed items among `count` elements from element `first` on; all threads, two barriers.
template <int CAP, int N>
__device__ __forceinline__ void mark(const Distill &a, const List<CAP> &l, uint32_t *bits, int64_t first, int64_t count) {
    __syncthreads();
    for (int i = threadIdx.x; i < CHUNK / 32; i += N) bits[i] = 0;
    __syncthreads();
    for (int j = threadIdx.x; j < a.topk; j += N) {
        const int64_t e = (int64_t)l.id[j] - first;
        if (l.id[j] != ICQ_PAD_ID && e >= 0 && e < count) atomicOr(&bits[e >> 5], 1u << (e & 31));
    }
    __syncthreads();
}

// Sums over `held` groups in registers, group u * N + thread in w[u].
template <int TYPE, bool REST, int N, int NV>
__device__ __forceinline__ void run_held(Run &run, const uint4 (&w)[NV], int held, const uint32_t *bits, float a2) {
    typedef IcqElem<TYPE> E;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
        const int b = u * N + (int)threadIdx.x, e = b * E::PER;
        if (b < held) {
            float y[E::PER];
            E::unpack(w[u], y);
            run_add<E::PER, REST>(run, y, REST ? bits[e >> 5] >> (e & 31) : 0u, a2);
        }
    }
}

// Sums over groups [first + done, to) of a row, in chunks that can be marked; the chunk from `first` on is marked already, so that the
// loads behind the groups in registers do not wait for a marking of their own.
template <int TYPE, bool REST, int CAP, int N>
__device__ __forceinline__ void run_over(Run &run, const Distill &a, const List<CAP> &l, uint32_t *bits, const uint4 *body, int head, int64_t first,
                                         int done, int64_t to) {
    typedef IcqElem<TYPE> E;
    constexpr int PER = E::PER, U = 4;
    for (int64_t b0 = first; b0 < to; b0 += CHUNK / PER, done = 0) {
        const int n = (int)(to - b0 < CHUNK / PER ? to - b0 : CHUNK / PER);
        if (REST && b0 > first) mark<CAP, N>(a, l, bits, head + b0 * PER, (int64_t)n * PER);
        const uint4 *at = body + b0;
        for (int i = done + (int)threadIdx.x; i < n; i += U * N) {
            uint4 w[U];
            uint32_t on[U];                            // (from the LDS while the groups are on their way)
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * N < n) {
                    const int e = (i + u * N) * PER;
                    w[u] = at[i + u * N];
                    on[u] = REST ? bits[e >> 5] >> (e & 31) : 0u;
                }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * N < n) {
                    float y[PER];
                    E::unpack(w[u], y);
                    run_add<PER, REST>(run, y, on[u], a.a2);
                }
        }
    }
}

// Off-list gradients of one group.
template <int TYPE>
__device__ __forceinline__ uint4 gradient_of(const uint4 &w, float m, float a2, float f) {
    typedef IcqElem<TYPE> E;
    float y[E::PER];
    E::unpack(w, y);
#pragma unroll
    for (int i = 0; i < E::PER; ++i) y[i] = ex2((y[i] - m) * a2) * f;
    return E::pack(y);
}

// Sums of a row (splits == 1: and its loss) or of a slice of it.  REST: also those off the list.
// (80 scalar registers: with two more, seven wavefronts share a SIMD instead of eight; 1024 x 131072 bf16 with a logsumexp 58 us against 51.)
template <int TYPE, bool REST, int CAP, int N>
__global__ __launch_bounds__(N) __attribute__((amdgpu_num_sgpr(80))) void distill_forward_kernel(Distill a) {
    typedef IcqElem<TYPE> E;
    constexpr int U = 8;
    __shared__ List<CAP> l;
    __shared__ uint32_t s_bits[REST ? CHUNK / 32 : 1];
    const int tid = threadIdx.x, k = (int)(blockIdx.x % (uint32_t)a.splits);
    const int64_t row = blockIdx.x / (uint32_t)a.splits;
    const typename E::raw *x = static_cast<const typename E::raw *>(a.x) + row * a.ld;
    float sum_p = 0.0f;
    const Span s = span_of<TYPE>(x, a.V);
    const Slice c = slice_of(s, k, a.splits);
    const auto in = [&](uint32_t id) { return a.splits == 1 || in_slice(s, c, id, E::PER); };
    const uint4 *body = reinterpret_cast<const uint4 *>(x + s.head);
    uint4 w[U];                                        // on their way while the list is worked on
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (c.b0 + u * N + tid < c.b1) w[u] = body[c.b0 + u * N + tid];
    const int entries = load_list<TYPE, CAP, N>(a, row, x, l, sum_p, in);
    Run run = {-FLT_MAX, 0.0f};
    for (int64_t i = c.e0 + tid; i < c.e1; i += N) {
        const int64_t v = i < s.head ? i : i + s.body * E::PER;
        const float y[1] = {E::get(x[v])};
        run_add<1, REST>(run, y, REST && on_list(l, a.slots, (uint32_t)v) ? 1u : 0u, a.a2);
    }
    const int held = (int)(c.b1 - c.b0 < U * N ? c.b1 - c.b0 : U * N);
    if (REST) mark<CAP, N>(a, l, s_bits, s.head + c.b0 * E::PER, c.b1 - c.b0 < CHUNK / E::PER ? (c.b1 - c.b0) * E::PER : CHUNK);
    run_held<TYPE, REST, N, U>(run, w, held, s_bits, a.a2);
    run_over<TYPE, REST, CAP, N>(run, a, l, s_bits, body, s.head, c.b0, held, c.b1);
    float v[2];
    const Sums sums = block_run<REST, CAP, N>(run, a, l, in, v);
    if (a.splits == 1) {
        bool counts;
        finish_row<CAP, N>(a, row, l, entries, sum_p, sums, v[0], true, REST, counts);
    } else {
        block_sums<N>(v, l.red);
        if (tid == 0) {
            const Part part = {sums, v[0], v[1], {0.0f, 0.0f}};
            a.part[row * a.splits + k] = part;
        }
    }
}

// A row's sums from its slices'; listed: this thread's share of the sum of p (x - m).
template <int CAP, int N>
__device__ Sums join_row(const Distill &a, int64_t row, List<CAP> &l, float &listed) {
    Run all = {-FLT_MAX, 0.0f}, off = {-FLT_MAX, 0.0f};
    for (int k = threadIdx.x; k < a.splits; k += N) {
        const Sums p = a.part[row * a.splits + k].sums;
        const Run pa = {p.m, p.s}, po = {p.mr, p.r};
        run_join(all, pa, a.a2);
        run_join(off, po, a.a2);
    }
    Sums b = {all.m, 0.0f, off.m, 0.0f};
    block_max2<N>(b.m, b.mr, l.red);
    float v[2] = {all.s * ex2((all.m - b.m) * a.a2), off.s * ex2((off.m - b.mr) * a.a2)};
    block_sums<N>(v, l.red);
    b.s = v[0];
    b.r = v[1];
    listed = 0.0f;
    for (int k = threadIdx.x; k < a.splits; k += N) {
        const Part p = a.part[row * a.splits + k];
        if (!(p.p == 0.0f)) listed += p.t + p.p * (p.sums.m - b.m);
    }
    return b;
}

template <int TYPE, int CAP>
__global__ __launch_bounds__(T) void distill_join_kernel(Distill a) {
    __shared__ List<CAP> l;
    const int64_t row = blockIdx.x;
    float sum_p, listed;
    const int entries = load_list<TYPE, CAP, T>(a, row, nullptr, l, sum_p, [](uint32_t) { return false; });
    const Sums run = join_row<CAP, T>(a, row, l, listed);
    bool counts;
    finish_row<CAP, T>(a, row, l, entries, sum_p, run, listed, true, true, counts);
}

// The gradient of a slice of a row.  VEC: logits and gradient rows start at the same place within 16 bytes, else element by element (4096 x 50021
// bf16, loss and gradient: 178 us, and 423 from logits three elements further apart than the gradient's rows).
// JOIN: the row's sums are still in its slices' (the first block of a row writes the loss), else in the statistics.
template <int TYPE, bool VEC, bool JOIN, int CAP>
__global__ __launch_bounds__(T) void distill_backward_kernel(Distill a) {
    typedef IcqElem<TYPE> E;
    constexpr int PER = E::PER, U = 8, PLACES = (CAP + T - 1) / T;
    __shared__ List<CAP> l;
    const int tid = threadIdx.x, k = (int)(blockIdx.x % (uint32_t)a.splits);
    const int64_t row = blockIdx.x / (uint32_t)a.splits;
    const typename E::raw *x = static_cast<const typename E::raw *>(a.x) + row * a.ld;
    typename E::raw *out = static_cast<typename E::raw *>(a.grad) + row * a.ld_grad;
    Span s;
    if (VEC) s = span_of<TYPE>(x, a.V);
    else { s.head = (int)a.V; s.body = 0; s.tail = 0; }
    const Slice c = slice_of(s, k, a.splits);
    const uint4 *body = reinterpret_cast<const uint4 *>(x + s.head);
    uint4 *body_out = reinterpret_cast<uint4 *>(out + s.head);
    uint4 w[U];                                        // on their way while the list is worked on
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (c.b0 + u * T + tid < c.b1) w[u] = body[c.b0 + u * T + tid];
    float sum_p, listed;
    const float g0 = a.grad_loss ? a.grad_loss[row] : 1.0f;
    // (listed items of other slices may have their gradients already, where those take the logits' place)
    const auto in = [&](uint32_t id) { return in_slice(s, c, id, PER); };
    const int entries = load_list<TYPE, CAP, T>(a, row, x, l, sum_p, in);
    float4 st;
    bool counts;
    if (JOIN) {
        const Sums run = join_row<CAP, T>(a, row, l, listed);
        st = finish_row<CAP, T>(a, row, l, entries, sum_p, run, listed, k == 0, true, counts);
    } else {
        st = a.stats[row];
        counts = st.y != 0.0f;
    }
    if (!counts) {
        for (int64_t i = c.e0 + tid; i < c.e1; i += T) out[i < s.head ? i : i + s.body * PER] = E::put(0.0f);
        for (int64_t b = c.b0 + tid; b < c.b1; b += T) body_out[b] = make_uint4(0, 0, 0, 0);
        return;
    }
    const float g = g0 * a.scale, q0 = 1.0f / st.y, f = st.w * g;
    // the listed items of this slice
    float mine[PLACES];
    uint32_t here[PLACES];
#pragma unroll
    for (int u = 0; u < PLACES; ++u) {
        const int j = u * T + tid;
        here[u] = j < a.topk && l.id[j] != ICQ_PAD_ID && in(l.id[j]) ? l.id[j] : ICQ_PAD_ID;
        if (here[u] != ICQ_PAD_ID) mine[u] = (ex2((l.x[j] - st.x) * a.a2) * q0 - l.p[j]) * g;
    }
    __syncthreads();
    for (int64_t i = c.e0 + tid; i < c.e1; i += T) {
        const int64_t v = i < s.head ? i : i + s.body * PER;
        out[v] = E::put(ex2((E::get(x[v]) - st.z) * a.a2) * f);
    }
    for (int64_t b = c.b0 + tid; b < c.b1; b += U * T) {
        if (b != c.b0 + tid) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (b + u * T < c.b1) w[u] = body[b + u * T];
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (b + u * T < c.b1) body_out[b + u * T] = gradient_of<TYPE>(w[u], st.z, a.a2, f);
    }
    __syncthreads();                                   // the listed items' values replace the ones just written
#pragma unroll
    for (int u = 0; u < PLACES; ++u)
        if (here[u] != ICQ_PAD_ID) out[here[u]] = E::put(mine[u]);
}

template <bool PAST_CACHES>
__device__ __forceinline__ void put_group(uint4 *p, const uint4 &v) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    const u32x4 q = {v.x, v.y, v.z, v.w};
    if (PAST_CACHES) __builtin_nontemporal_store(q, reinterpret_cast<u32x4 *>(p));
    else *reinterpret_cast<u32x4 *>(p) = q;
}

// Loss and gradient of a whole row: N threads, the first N * NV groups of 16 bytes stay in registers.  LONG: rows beyond those; their
// second reading comes from the last-level cache as long as the gradient's stores do not go there (4096 x 131072 bf16:
// 472 us with ordinary stores, 431 so, 4.98 TB/s of the least traffic; a copy runs at 5.17).
template <int TYPE, bool REST, int CAP, int N, int NV, bool LONG>
__global__ __launch_bounds__(N, 4) void distill_row_kernel(Distill a) {
    typedef IcqElem<TYPE> E;
    constexpr int PER = E::PER, U = 4, PLACES = (CAP + N - 1) / N;
    static_assert(N * NV * PER <= CHUNK, "one marking covers the registers");
    __shared__ List<CAP> l;
    __shared__ uint32_t s_bits[REST ? CHUNK / 32 : 1];
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x;
    const typename E::raw *x = static_cast<const typename E::raw *>(a.x) + row * a.ld;
    typename E::raw *out = static_cast<typename E::raw *>(a.grad) + row * a.ld_grad;
    const Span s = span_of<TYPE>(x, a.V);
    const uint4 *body = reinterpret_cast<const uint4 *>(x + s.head);
    uint4 *body_out = reinterpret_cast<uint4 *>(out + s.head);
    const int held = (int)(s.body < N * NV ? s.body : N * NV);
    uint4 w[NV];
#pragma unroll
    for (int u = 0; u < NV; ++u)
        if (u * N + tid < held) w[u] = body[u * N + tid];
    const bool single = tid < s.head + s.tail;         // (fewer than 16 of them)
    const int64_t v1 = tid < s.head ? tid : tid + s.body * PER;
    const float y1[1] = {single ? E::get(x[v1]) : 0.0f};
    const float g0 = a.grad_loss ? a.grad_loss[row] : 1.0f;
    float sum_p;
    const int entries = load_list<TYPE, CAP, N>(a, row, x, l, sum_p, [](uint32_t) { return true; });
    Run run = {-FLT_MAX, 0.0f};
    if (single) run_add<1, REST>(run, y1, REST && on_list(l, a.slots, (uint32_t)v1) ? 1u : 0u, a.a2);
    if (REST) mark<CAP, N>(a, l, s_bits, s.head, s.body < CHUNK / PER ? s.body * PER : CHUNK);
    run_held<TYPE, REST, N, NV>(run, w, held, s_bits, a.a2);
    run_over<TYPE, REST, CAP, N>(run, a, l, s_bits, body, s.head, 0, held, s.body);
    float v[2];
    const Sums sums = block_run<REST, CAP, N>(run, a, l, [](uint32_t) { return true; }, v);
    bool counts;
    const float4 st = finish_row<CAP, N>(a, row, l, entries, sum_p, sums, v[0], true, REST, counts);
    const float g = g0 * a.scale, q0 = 1.0f / st.y, base = REST ? st.z : st.x, f = (REST ? st.w : q0) * g;      // (the same without the mass off the list)
    float mine[PLACES];
    uint32_t here[PLACES];
#pragma unroll
    for (int u = 0; u < PLACES; ++u) {
        const int j = u * N + tid;
        here[u] = counts && j < a.topk ? l.id[j] : ICQ_PAD_ID;
        if (here[u] != ICQ_PAD_ID) mine[u] = (ex2((l.x[j] - st.x) * a.a2) * q0 - l.p[j]) * g;
    }
    __syncthreads();
    const uint4 zero = make_uint4(0, 0, 0, 0);
    if (single) out[v1] = E::put(counts ? ex2((y1[0] - base) * a.a2) * f : 0.0f);
#pragma unroll
    for (int u = 0; u < NV; ++u)
        if (u * N + tid < held) put_group<LONG>(body_out + u * N + tid, counts ? gradient_of<TYPE>(w[u], base, a.a2, f) : zero);
    for (int64_t b = s.body - 1 - tid; b >= held; b -= U * N) {        // from the end: what was read last is nearest
        uint4 r[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (b - u * N >= held) r[u] = body[b - u * N];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (b - u * N >= held) put_group<LONG>(body_out + b - u * N, counts ? gradient_of<TYPE>(r[u], base, a.a2, f) : zero);
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < PLACES; ++u)
        if (here[u] != ICQ_PAD_ID) out[here[u]] = E::put(mine[u]);
}

size_t part_bytes(int64_t R, int splits) { return icq_align_up((size_t)R * splits * sizeof(Part), ICQ_ALIGN); }

bool shape_ok(const void *logits, int type, int64_t R, int64_t V, int64_t ld, float scale, const uint32_t *ids, const float *values,
              int topk, float teacher_scale) {
    const int size = icq_type_bytes(type);
    if (size == 0 || R < 0 || R > ICQ_MAX_Q || V < 1 || V > ICQ_MAX_EXTENT || ld < V || topk < 1 || topk > ICQ_MAX_TOPK) return false;
    if (!(scale > 0.0f) || !(scale * LOG2E <= FLT_MAX) || !(teacher_scale >= -FLT_MAX && teacher_scale <= FLT_MAX)) return false;
    return R == 0 || (logits && ids && values && (uintptr_t)logits % size == 0);
}

Distill params(const void *logits, int type, int64_t R, int64_t V, int64_t ld, float scale, const uint32_t *ids, const float *values, int topk,
               float teacher_scale, const float *teacher_lse) {
    Distill a;
    a.x = logits; a.R = R; a.V = V; a.ld = ld;
    a.scale = scale; a.a2 = scale * LOG2E;
    a.lowest = type == ICQ_F16 ? -65504.0f : type == ICQ_BF16 ? -0x1.fep127f : -FLT_MAX;
    a.ids = ids; a.values = values; a.topk = topk;
    a.slots = 32;
    while (a.slots < 2 * topk) a.slots *= 2;
    a.teacher_scale = teacher_scale; a.teacher_lse = teacher_lse;
    a.loss = nullptr; a.stats = nullptr; a.grad_loss = nullptr; a.grad = nullptr; a.ld_grad = 0;
    a.splits = 1; a.num_cu = 0; a.part = nullptr;
    return a;
}

// Logits and gradient rows start at the same place within 16 bytes.
bool same_phase(const Distill &a, int size) {
    return ((uintptr_t)a.grad - (uintptr_t)a.x) % 16 == 0 && ((a.ld_grad - a.ld) * size) % 16 == 0;
}

template <int TYPE, int CAP>
void launch_backward(const Distill &a, bool join, hipStream_t s) {
    const dim3 grid((uint32_t)(a.R * a.splits));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(T), 0, s, a); };
    if (same_phase(a, sizeof(typename IcqElem<TYPE>::raw))) join ? go(distill_backward_kernel<TYPE, true, true, CAP>) : go(distill_backward_kernel<TYPE, true, false, CAP>);
    else join ? go(distill_backward_kernel<TYPE, false, true, CAP>) : go(distill_backward_kernel<TYPE, false, false, CAP>);
}

template <int TYPE, bool REST, int CAP>
void launch_distill(const Distill &a, hipStream_t s) {
    constexpr int SIZE = sizeof(typename IcqElem<TYPE>::raw);
    if (a.grad && a.splits == 1 && same_phase(a, SIZE)) {
        auto go = [&](auto kernel, int n) { hipLaunchKernelGGL(kernel, dim3((uint32_t)a.R), dim3(n), 0, s, a); };
        switch (icq_distill_row_form(a.R, a.V * SIZE, a.num_cu)) {
            case ICQ_ROW_1024_4: go(distill_row_kernel<TYPE, REST, CAP, 1024, 4, false>, 1024); break;
            case ICQ_ROW_256_4: go(distill_row_kernel<TYPE, REST, CAP, 256, 4, false>, 256); break;
            case ICQ_ROW_256_8: go(distill_row_kernel<TYPE, REST, CAP, 256, 8, false>, 256); break;
            case ICQ_ROW_256_16: go(distill_row_kernel<TYPE, REST, CAP, 256, 16, false>, 256); break;
            case ICQ_ROW_LONG: go(distill_row_kernel<TYPE, REST, CAP, 512, 16, true>, 512); break;
        }
        return;
    }
    const auto forward = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, dim3((uint32_t)(a.R * a.splits)), dim3(threads), 0, s, a); };
    if (icq_distill_forward_threads(a.splits, a.V * SIZE) == 512) forward(distill_forward_kernel<TYPE, REST, CAP, 512>, 512);
    else forward(distill_forward_kernel<TYPE, REST, CAP, T>, T);
    if (a.grad) launch_backward<TYPE, CAP>(a, a.splits > 1, s);
    else if (a.splits > 1) hipLaunchKernelGGL(HIP_KERNEL_NAME(distill_join_kernel<TYPE, CAP>), dim3((uint32_t)a.R), dim3(T), 0, s, a);
}

// The logits' own memory, or none of it.
bool grad_ok(const void *logits, int type, int64_t R, int64_t V, int64_t ld, const void *grad, int64_t ld_grad) {
    const int64_t size = icq_type_bytes(type);
    if (!grad || ld_grad < V || (uintptr_t)grad % size != 0) return false;
    if (grad == logits) return ld_grad == ld;
    return !icq_rows_overlap((uintptr_t)logits, ld * size, (uintptr_t)grad, ld_grad * size, R, V * size);
}

}  // namespace

ICQ_EXPORT int icq_distill_workspace_bytes(int64_t R, int64_t V, size_t *out) {
    if (!out || R < 0 || R > ICQ_MAX_Q || V < 1 || V > ICQ_MAX_EXTENT) return ICQ_ERR_ARG;
    const int cu = icq_num_cu();
    if (cu <= 0) return ICQ_ERR_HIP;
    *out = part_bytes(R, icq_distill_splits(R, V, cu, 0)) + part_bytes(R, 1);
    return ICQ_OK;
}

ICQ_EXPORT int icq_distill(const void *logits, int type, int64_t R, int64_t V, int64_t ld, float scale, const uint32_t *ids,
                           const float *values, int topk, float teacher_scale, const float *teacher_lse, float *loss, float *stats,
                           const float *grad_loss, void *grad, int64_t ld_grad, void *workspace, size_t workspace_bytes, void *stream) {
    if (!shape_ok(logits, type, R, V, ld, scale, ids, values, topk, teacher_scale)) return ICQ_ERR_ARG;
    if (R == 0) return ICQ_OK;
    if (!loss || (uintptr_t)stats % 16 != 0 || (grad && !grad_ok(logits, type, R, V, ld, grad, ld_grad))) return ICQ_ERR_ARG;
    const int cu = icq_num_cu();
    if (cu <= 0) return ICQ_ERR_HIP;
    Distill a = params(logits, type, R, V, ld, scale, ids, values, topk, teacher_scale, teacher_lse);
    const size_t parts = part_bytes(R, icq_distill_splits(R, V, cu, 0));
    if (!workspace || (uintptr_t)workspace % ICQ_ALIGN != 0 || workspace_bytes < parts + part_bytes(R, 1)) return ICQ_ERR_WORKSPACE;
    a.part = static_cast<Part *>(workspace);
    a.loss = loss;
    a.stats = stats ? reinterpret_cast<float4 *>(stats) : reinterpret_cast<float4 *>(static_cast<char *>(workspace) + parts);
    a.grad_loss = grad_loss; a.grad = grad; a.ld_grad = ld_grad;
    a.num_cu = cu;
    a.splits = icq_distill_splits(R, V, cu, grad && same_phase(a, icq_type_bytes(type)) ? V * icq_type_bytes(type) : 0);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool few = topk <= SHORT;
    ICQ_FOR_TYPE(type,
        if (teacher_lse) few ? launch_distill<TYPE, true, SHORT>(a, s) : launch_distill<TYPE, true, ICQ_MAX_TOPK>(a, s);
        else few ? launch_distill<TYPE, false, SHORT>(a, s) : launch_distill<TYPE, false, ICQ_MAX_TOPK>(a, s))
    return icq_check_launch();
}

ICQ_EXPORT int icq_distill_backward(const void *logits, int type, int64_t R, int64_t V, int64_t ld, float scale, const uint32_t *ids,
                                    const float *values, int topk, float teacher_scale, const float *teacher_lse, const float *stats,
                                    const float *grad_loss, void *grad, int64_t ld_grad, void *stream) {
    if (!shape_ok(logits, type, R, V, ld, scale, ids, values, topk, teacher_scale)) return ICQ_ERR_ARG;
    if (R == 0) return ICQ_OK;
    if (!stats || (uintptr_t)stats % 16 != 0 || !grad_ok(logits, type, R, V, ld, grad, ld_grad)) return ICQ_ERR_ARG;
    const int cu = icq_num_cu();
    if (cu <= 0) return ICQ_ERR_HIP;
    Distill a = params(logits, type, R, V, ld, scale, ids, values, topk, teacher_scale, teacher_lse);
    a.splits = icq_distill_splits(R, V, cu, 0);
    a.stats = reinterpret_cast<float4 *>(const_cast<float *>(stats));
    a.grad_loss = grad_loss; a.grad = grad; a.ld_grad = ld_grad;
    hipStream_t s = static_cast<hipStream_t>(stream);
    ICQ_FOR_TYPE(type, topk <= SHORT ? launch_backward<TYPE, SHORT>(a, false, s) : launch_backward<TYPE, ICQ_MAX_TOPK>(a, false, s))
    return icq_check_launch();
}
