// Keys and values of the trees' nodes into the pages of their sequences, turned to the nodes' positions on the way.
//
// One workgroup per node: an angle's cosine and sine are formed once, by one thread, and serve all heads from LDS.  What
// bounds it is memory: queries, keys and values are read and written once (64 trees of 31 nodes, 32 + 8 + 8 heads of 128 in bf16:
// 49 MB in 10.8 us, 4.5 TB/s; prompts of 8 sequences, 503 MB in 94 us, 5.4 TB/s; one tree of 15 nodes 3.9 us, of which an empty
// launch is 3).
#include "kv_cache.h"

namespace mdsd {

struct AppendParams {
    Cache cache;
    Trees trees;
    Heads k, v, q, q_out;  // q.heads = 0: no queries
    const float* inv_freq;
    int rot;
    int items;  // of a head that is turned: pairs of chunks or of elements, chunks, ...
    Divisor by_node, by_items, by_chunks;
    int32_t* flags;
};

enum { kHalves, kNeighbours, kElements };  // kElements: halves that do not begin and end with a 16-byte chunk

constexpr int kAppendThreads = 256;

template <class T>
struct alignas(16) Chunk {
    T x[16 / sizeof(T)];
};

template <class T>
__device__ inline void turn(T& x, T& y, float c, float s)
{
    const float a = (float)x, b = (float)y;
    x = (T)__builtin_fmaf(a, c, -(b * s));
    y = (T)__builtin_fmaf(a, s, b * c);
}

template <class T, int kStyle>
__device__ inline void turned(const AppendParams& P, const char* from, char* to, int item, const float* cosine, const float* sine)
{
    constexpr int kPer = 16 / sizeof(T);
    using C = Chunk<T>;
    if constexpr (kStyle == kElements) {
        const T* const in = (const T*)from;
        T* const out = (T*)to;
        const int half = P.rot / 2;
        if (item < half) {
            T x = in[item], y = in[item + half];
            turn(x, y, cosine[item], sine[item]);
            out[item] = x;
            out[item + half] = y;
        } else {
            out[item + half] = in[item + half];
        }
    } else if constexpr (kStyle == kHalves) {
        const int half = P.rot / 2 / kPer;  // chunks
        if (item < half) {
            C x = ((const C*)from)[item], y = ((const C*)from)[item + half];
#pragma unroll
            for (int j = 0; j < kPer; ++j) turn(x.x[j], y.x[j], cosine[item * kPer + j], sine[item * kPer + j]);
            ((C*)to)[item] = x;
            ((C*)to)[item + half] = y;
        } else {
            ((C*)to)[item + half] = ((const C*)from)[item + half];
        }
    } else {
        C x = ((const C*)from)[item];
#pragma unroll
        for (int j = 0; j < kPer; j += 2) {
            const int pair = (item * kPer + j) / 2;
            if (2 * pair < P.rot) turn(x.x[j], x.x[j + 1], cosine[pair], sine[pair]);
        }
        ((C*)to)[item] = x;
    }
}

template <class T, int kStyle>
__global__ __launch_bounds__(kAppendThreads) void kv_append_kernel(AppendParams P)
{
    extern __shared__ int parent[];
    __shared__ float cosine[MDSD_MAX_DIM / 2], sine[MDSD_MAX_DIM / 2];
    const Cache& C = P.cache;
    const int b = P.by_node((int)blockIdx.x), n = (int)blockIdx.x - b * P.trees.N;
    if (n >= P.trees.count(b)) return;
    const int length = C.lengths[b];
    if (length < 0) {
        if (P.flags && threadIdx.x == 0) atomicOr(&P.flags[b], MDSD_FLAG_NO_PAGE);
        return;
    }
    const int64_t place = place_of(C, C.table + b * C.ld_table, (int64_t)length + n);
    if (place < 0 && P.flags && threadIdx.x == 0) atomicOr(&P.flags[b], MDSD_FLAG_NO_PAGE);

    int level = 0;
    if (P.trees.complete && P.trees.k == 1) {
        level = n;
    } else {
        if (!P.trees.complete) parents_from_table(P.trees, parent);
        for (int a = parent_of(P.trees, parent, n); a >= 0; a = parent_of(P.trees, parent, a)) ++level;
    }
    if ((int)threadIdx.x < P.rot / 2) {
        // turns in 64 bits (a position of a million times an fp32 frequency has 44 bits), cut to an eighth of a turn
        // either way: what is left keeps 2^-28 of a turn when it is rounded to 32 bits
        const double turns = ((double)length + level) * (double)P.inv_freq[threadIdx.x] * 0.15915494309189535;
        const double quarters = rint(4.0 * turns);
        float s, c;
        sincospif((float)(2.0 * (turns - 0.25 * quarters)), &s, &c);
        const int quadrant = (int)(quarters - 4.0 * floor(0.25 * quarters));
        const float x = quadrant & 1 ? s : c, y = quadrant & 1 ? c : s;
        cosine[threadIdx.x] = quadrant == 1 || quadrant == 2 ? -x : x;
        sine[threadIdx.x] = quadrant >= 2 ? -y : y;
    }
    __syncthreads();

    const char* const q = P.q.p + b * P.q.ld_tree + n * P.q.ld_node;
    char* const q_out = P.q_out.p + b * P.q_out.ld_tree + n * P.q_out.ld_node;
    for (int i = threadIdx.x; i < P.q.heads * P.items; i += kAppendThreads) {
        const int h = P.by_items(i);
        turned<T, kStyle>(P, q + h * P.q.ld_head, q_out + h * P.q_out.ld_head, i - h * P.items, cosine, sine);
    }
    if (place < 0) return;
    const char* const k = P.k.p + b * P.k.ld_tree + n * P.k.ld_node;
    for (int i = threadIdx.x; i < C.heads * P.items; i += kAppendThreads) {
        const int h = P.by_items(i);
        turned<T, kStyle>(P, k + h * P.k.ld_head, C.k + place + h * C.ld_head, i - h * P.items, cosine, sine);
    }
    const char* const v = P.v.p + b * P.v.ld_tree + n * P.v.ld_node;
    const int chunks = C.dim * (int)sizeof(T) / 16;
    for (int i = threadIdx.x; i < C.heads * chunks; i += kAppendThreads) {
        const int h = P.by_chunks(i), c = i - h * chunks;
        ((Chunk<T>*)(C.v + place + h * C.ld_head))[c] = ((const Chunk<T>*)(v + h * P.v.ld_head))[c];
    }
}

template <class T>
static int launch_append(AppendParams& P, int style, hipStream_t st)
{
    constexpr int kPer = 16 / sizeof(T);
    const int half = P.rot / 2;
    const int chunks = P.cache.dim / kPer;
    void (*kernel)(AppendParams);
    if (style == MDSD_ROTATE_NEIGHBOURS) {
        kernel = kv_append_kernel<T, kNeighbours>;
        P.items = chunks;
    } else if (half % kPer == 0) {
        kernel = kv_append_kernel<T, kHalves>;
        P.items = chunks - half / kPer;
    } else {
        kernel = kv_append_kernel<T, kElements>;
        P.items = P.cache.dim - half;
    }
    if ((int64_t)P.q.heads * P.items > INT32_MAX - kAppendThreads || (int64_t)P.cache.heads * P.cache.dim > INT32_MAX - kAppendThreads)
        return MDSD_E_SHAPE;
    if ((int64_t)P.trees.B * P.trees.N > kMostGroups) return MDSD_E_SHAPE;
    P.by_items = Divisor::of(P.items);
    P.by_chunks = Divisor::of(chunks);
    P.by_node = Divisor::of(P.trees.N);
    (void)hipGetLastError();
    hipLaunchKernelGGL(kernel, dim3((unsigned)(P.trees.B * P.trees.N)), dim3(kAppendThreads),
                       P.trees.complete ? 0 : P.trees.N * sizeof(int), st, P);
    return hipGetLastError() == hipSuccess ? MDSD_OK : MDSD_E_LAUNCH;
}

}  // namespace mdsd

extern "C" int mdsd_kv_append(const mdsd_kv_cache* cache, int32_t layer, const mdsd_tree* tree, const mdsd_heads* k,
                              const mdsd_heads* v, const mdsd_heads* q, const mdsd_heads* q_out, const float* inv_freq,
                              int32_t rot, int32_t style, int32_t* flags, void* stream)
{
    using namespace mdsd;
    AppendParams P = {};
    int rc = check_cache(cache, tree, &P.cache, &P.trees);
    if (rc == kEmptyTrees) return MDSD_OK;
    if (rc != MDSD_OK) return rc;
    if ((rc = check_heads(k, P.cache, cache->dtype, &P.k)) != MDSD_OK) return rc;
    if ((rc = check_heads(v, P.cache, cache->dtype, &P.v)) != MDSD_OK) return rc;
    if ((q == nullptr) != (q_out == nullptr)) return MDSD_E_NULL;
    if (q) {
        if ((rc = check_heads(q, P.cache, cache->dtype, &P.q)) != MDSD_OK) return rc;
        if ((rc = check_heads(q_out, P.cache, cache->dtype, &P.q_out)) != MDSD_OK) return rc;
        if (q->heads != q_out->heads || one_place(*q_out, P.trees)) return MDSD_E_SHAPE;
        if (overlap(P.q, P.q_out, P.trees, P.cache, cache->dtype)) return MDSD_E_ALIGN;
    }
    if (one_place(*cache)) return MDSD_E_SHAPE;
    if (layer < 0 || layer >= cache->layers || k->heads != cache->heads || v->heads != cache->heads) return MDSD_E_SHAPE;
    if (rot < 0 || rot > cache->dim || rot % 2) return MDSD_E_SHAPE;
    if (style != MDSD_ROTATE_HALVES && style != MDSD_ROTATE_NEIGHBOURS) return MDSD_E_DTYPE;
    if (rot && !inv_freq) return MDSD_E_NULL;
    if (((uintptr_t)inv_freq | (uintptr_t)flags) & 3) return MDSD_E_ALIGN;
    P.inv_freq = inv_freq;
    P.rot = rot;
    P.flags = flags;
    P.cache.k += layer * P.cache.ld_layer;
    P.cache.v += layer * P.cache.ld_layer;
    hipStream_t st = (hipStream_t)stream;
    switch (cache->dtype) {
    case MDSD_FP32: return launch_append<float>(P, style, st);
    case MDSD_BF16: return launch_append<__bf16>(P, style, st);
    default: return launch_append<_Float16>(P, style, st);
    }
}
