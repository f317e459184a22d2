// Keys and values of the trees' nodes into the pages of their sequences, turned to the nodes' positions on the way.
//
// One workgroup per node: an angle's cosine and sine are formed once, by one thread, and serve all heads from LDS.  What
// bounds it is memory: queries, keys and values are read and written once (64 trees of 31 nodes, 32 + 8 + 8 heads of 128 in bf16:
// 49 MB in 10.8 us, 4.5 TB/s; prompts of 8 sequences, 503 MB in 94 us, 5.4 TB/s; one tree of 15 nodes 3.9 us, of which an empty
// launch is 3).
//
// Into 4 bits a thread has 8 elements, and four threads a block, whose largest they find together; keys are turned in 64 bits
// (a border between two of 16 values is met too often for a sum that is rounded another way): 50.9 MB in 12.3 us, 4.1 TB/s; prompts with
// three axes of positions, 525 MB of fp16, 111 us, 4.7 TB/s; one tree 5.1 us.
#include "four_bits.h"

namespace mdsd {

struct AppendParams {
    Cache cache;
    Trees trees;
    Heads k, v, q, q_out;  // q.heads = 0: no queries
    Scales scales;         // of a cache in 4 bits
    Heads k_out, v_out;    // what it then holds; p = NULL: not asked for
    const float* inv_freq;
    const int32_t* positions;  // NULL: lengths and levels
    int64_t ld_axis, ld_tree;
    int axes;
    bool per_node;
    const uint8_t* axis_of;
    int rot;
    int items;  // of a head that is turned: pairs of chunks or of elements, chunks, ...
    Divisor by_node, by_items, by_chunks;
    Divisor by_eights;  // of a head, in 4 bits
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

// Eight elements of a key from element x on, as they are or turned: in 64 bits, and rounded to 32, as the borders between
// sixteen values are met wherever a sum is rounded otherwise.
template <class T, int kStyle>
__device__ inline void turned_key(const AppendParams& P, const char* from, int x, const double2* turns, float (&y)[8])
{
    struct alignas(16) Eight {
        T x[8];
    };
    const T* const in = (const T*)from;
    const int half = P.rot / 2;
    const Eight own = *(const Eight*)(in + x);
    if constexpr (kStyle == kNeighbours) {
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            y[j] = (float)own.x[j];
            y[j + 1] = (float)own.x[j + 1];
            if (x + j < P.rot) {
                const double a = (double)own.x[j], b = (double)own.x[j + 1];
                const double2 t = turns[(x + j) / 2];
                y[j] = (float)(a * t.x - b * t.y);
                y[j + 1] = (float)(a * t.y + b * t.x);
            }
        }
    } else {
        Eight other = own;
        if (kStyle == kHalves && x < P.rot) other = *(const Eight*)(in + (x < half ? x + half : x - half));
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int e = x + j;
            y[j] = (float)own.x[j];
            if (e < P.rot) {
                const bool front = e < half;
                const int pair = front ? e : e - half;
                const double a = (double)own.x[j], b = kStyle == kHalves ? (double)other.x[j] : (double)in[front ? e + half : pair];
                const double2 t = turns[pair];
                y[j] = (float)(front ? a * t.x - b * t.y : b * t.y + a * t.x);
            }
        }
    }
}

// The node's keys and values into the cache in 4 bits: eight elements a thread, four threads a scale (which end together:
// a head has whole blocks)
template <class T, int kStyle>
__device__ inline void append_four(const AppendParams& P, int b, int n, int64_t place, const double2* turns)
{
    const Cache& C = P.cache;
    const int eights = C.dim / 8, of_keys = C.heads * eights;
    for (int i = threadIdx.x; i < 2 * of_keys; i += kAppendThreads) {
        const bool value = i >= of_keys;
        const int item = value ? i - of_keys : i, h = P.by_eights(item), x = (item - h * eights) * 8;
        const Heads& from = value ? P.v : P.k;
        const char* const in = from.p + b * from.ld_tree + n * from.ld_node + h * from.ld_head;
        float y[8];
        if (value) {
            const Chunk<T>* const at = (const Chunk<T>*)((const T*)in + x);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = (float)at[j * (int)sizeof(T) / 16].x[j % (16 / (int)sizeof(T))];
        } else {
            turned_key<T, kStyle>(P, in, x, turns, y);
        }
        uint32_t most = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint(y[j]) & 0x7fffffffu);
        most = max(most, (uint32_t)__shfl_xor((int)most, 1));
        most = max(most, (uint32_t)__shfl_xor((int)most, 2));
        const uint32_t scale = scale_for(most, kLeastScale<T>, kGreatestScale<T>), codes = codes_of(y, scale);
        if (place >= 0) {
            const int64_t at = place + h * C.ld_head + x / 2;
            *(uint32_t*)((value ? C.v : C.k) + at) = codes;
            if (x % kBlock == 0) (value ? P.scales.v : P.scales.k)[at >> 4] = (uint8_t)scale;
        }
        const Heads& held = value ? P.v_out : P.k_out;
        if (held.p) {
            u32x4* const to = (u32x4*)((T*)(held.p + b * held.ld_tree + n * held.ld_node + h * held.ld_head) + x);
            to[0] = sixteen_bytes<T>(codes, scale_of(scale), false);
            if (sizeof(T) == 4) to[1] = sixteen_bytes<T>(codes, scale_of(scale), true);
        }
    }
}

// kGiven: positions may be given
template <class T, int kStyle, bool kFour, bool kGiven>
__global__ __launch_bounds__(kAppendThreads) void kv_append_kernel(AppendParams P)
{
    extern __shared__ int parent[];
    __shared__ float cosine[MDSD_MAX_DIM / 2], sine[MDSD_MAX_DIM / 2];
    __shared__ double2 turn_of[kFour ? MDSD_MAX_DIM / 2 : 1];  // cosine and sine
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
        double at = (double)length + level;
        bool turned_by_one = true;  // of the axes
        if (kGiven && P.positions) {
            const int axis = P.axis_of ? P.axis_of[threadIdx.x] : 0;
            turned_by_one = axis < P.axes;
            at = P.positions[(turned_by_one ? axis : 0) * P.ld_axis + b * P.ld_tree + (P.per_node ? n : 0)];
            at += P.per_node ? 0 : level;
        }
        // (by none: no turn, also where the frequency is no number)
        const double turns = turned_by_one ? at * (double)P.inv_freq[threadIdx.x] * 0.15915494309189535 : 0.0;
        const double quarters = rint(4.0 * turns);
        float s, c;
        if constexpr (kFour) {
            double sine_of, cosine_of;
            sincospi(2.0 * (turns - 0.25 * quarters), &sine_of, &cosine_of);
            const double of[4] = {cosine_of, -sine_of, -cosine_of, sine_of};  // the cosine a quadrant further, and again
            const int quadrant = (int)(quarters - 4.0 * floor(0.25 * quarters));
            turn_of[threadIdx.x] = double2{of[quadrant], of[(quadrant + 3) & 3]};
            s = (float)sine_of;
            c = (float)cosine_of;
        } else {
            sincospif((float)(2.0 * (turns - 0.25 * quarters)), &s, &c);
        }
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
    if constexpr (kFour) {
        append_four<T, kStyle>(P, b, n, place, turn_of);
        return;
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

template <class T, bool kFour, bool kGiven>
static int launch_append(AppendParams& P, int style, hipStream_t st)
{
    constexpr int kPer = 16 / sizeof(T);
    const int half = P.rot / 2;
    const int chunks = P.cache.dim / kPer;
    void (*kernel)(AppendParams);
    if (style == MDSD_ROTATE_NEIGHBOURS) {
        kernel = kv_append_kernel<T, kNeighbours, kFour, kGiven>;
        P.items = chunks;
    } else if (half % (kFour ? 8 : kPer) == 0) {
        kernel = kv_append_kernel<T, kHalves, kFour, kGiven>;
        P.items = chunks - half / kPer;
    } else {
        kernel = kv_append_kernel<T, kElements, kFour, kGiven>;
        P.items = P.cache.dim - half;
    }
    if ((int64_t)P.q.heads * P.items > INT32_MAX - kAppendThreads || (int64_t)P.cache.heads * P.cache.dim > INT32_MAX - kAppendThreads)
        return MDSD_E_SHAPE;
    if ((int64_t)P.trees.B * P.trees.N > kMostGroups) return MDSD_E_SHAPE;
    P.by_items = Divisor::of(P.items);
    P.by_chunks = Divisor::of(chunks);
    P.by_eights = Divisor::of(P.cache.dim / 8);
    P.by_node = Divisor::of(P.trees.N);
    (void)hipGetLastError();
    hipLaunchKernelGGL(kernel, dim3((unsigned)(P.trees.B * P.trees.N)), dim3(kAppendThreads),
                       P.trees.complete ? 0 : P.trees.N * sizeof(int), st, P);
    return hipGetLastError() == hipSuccess ? MDSD_OK : MDSD_E_LAUNCH;
}

template <class T>
static int launch_append(AppendParams& P, int style, hipStream_t st)
{
    // (without a look at positions that are not there 64 trees of 31 nodes take 10.3 us, not 11.0, and in 4 bits 12.5, not 13.2)
    if (P.scales.k) return P.positions ? launch_append<T, true, true>(P, style, st) : launch_append<T, true, false>(P, style, st);
    return P.positions ? launch_append<T, false, true>(P, style, st) : launch_append<T, false, false>(P, style, st);
}

}  // namespace mdsd

extern "C" {

int mdsd_kv_append_at(const mdsd_kv_cache* cache, const mdsd_kv_scales* scales, int32_t layer, const mdsd_tree* tree,
                      const mdsd_heads* k, const mdsd_heads* v, const mdsd_heads* q, const mdsd_heads* q_out,
                      const mdsd_rotary* rotary, const mdsd_heads* k_out, const mdsd_heads* v_out, int32_t* flags, void* stream)
{
    using namespace mdsd;
    AppendParams P = {};
    int dtype;
    int rc = check_cache(cache, scales, tree, &P.cache, &P.scales, &dtype, &P.trees);
    if (rc == kEmptyTrees) return MDSD_OK;
    if (rc != MDSD_OK) return rc;
    if ((rc = check_heads(k, P.cache, dtype, &P.k)) != MDSD_OK) return rc;
    if ((rc = check_heads(v, P.cache, dtype, &P.v)) != MDSD_OK) return rc;
    if ((q == nullptr) != (q_out == nullptr)) return MDSD_E_NULL;
    // a result and the vector that it comes from
    auto result = [&](const mdsd_heads* of, const Heads& from, Heads* to) {
        int rc = check_heads(of, P.cache, dtype, to);
        if (rc != MDSD_OK) return rc;
        if (to->heads != from.heads || one_place(*of, P.trees)) return MDSD_E_SHAPE;
        return overlap(from, *to, P.trees, P.cache, dtype) ? MDSD_E_ALIGN : MDSD_OK;
    };
    if (q) {
        if ((rc = check_heads(q, P.cache, dtype, &P.q)) != MDSD_OK) return rc;
        if ((rc = result(q_out, P.q, &P.q_out)) != MDSD_OK) return rc;
    }
    if (one_place(*cache)) return MDSD_E_SHAPE;
    if (layer < 0 || layer >= cache->layers || k->heads != cache->heads || v->heads != cache->heads) return MDSD_E_SHAPE;
    const mdsd_rotary none = {};
    const mdsd_rotary& R = rotary ? *rotary : none;
    if (R.rot < 0 || R.rot > cache->dim || R.rot % 2) return MDSD_E_SHAPE;
    if (R.style != MDSD_ROTATE_HALVES && R.style != MDSD_ROTATE_NEIGHBOURS) return MDSD_E_DTYPE;
    if (R.rot && !R.inv_freq) return MDSD_E_NULL;
    if (R.positions && (R.axes < 1 || R.axes > MDSD_MAX_AXES || R.ld_axis < 0 || R.ld_tree < 0 || R.ld_axis >> 46 || R.ld_tree >> 31 ||
                        (R.per_node != 0 && R.per_node != 1)))
        return MDSD_E_SHAPE;
    if (((uintptr_t)R.inv_freq | (uintptr_t)R.positions | (uintptr_t)flags) & 3) return MDSD_E_ALIGN;
    if (!scales && (k_out || v_out)) return MDSD_E_UNSUPPORTED;
    if (k_out && (rc = result(k_out, P.k, &P.k_out)) != MDSD_OK) return rc;
    if (k_out && P.k_out.p == P.k.p) return MDSD_E_ALIGN;  // (a pair's halves are read by two threads)
    if (v_out && (rc = result(v_out, P.v, &P.v_out)) != MDSD_OK) return rc;
    P.inv_freq = R.inv_freq;
    P.rot = R.rot;
    P.positions = R.positions;
    P.ld_axis = R.ld_axis;
    P.ld_tree = R.ld_tree;
    P.axes = R.axes;
    P.per_node = R.per_node != 0;
    P.axis_of = R.axis_of;
    P.flags = flags;
    choose_layer(layer, &P.cache, &P.scales);
    hipStream_t st = (hipStream_t)stream;
    switch (dtype) {
    case MDSD_FP32: return launch_append<float>(P, R.style, st);
    case MDSD_BF16: return launch_append<__bf16>(P, R.style, st);
    default: return launch_append<_Float16>(P, R.style, st);
    }
}

int mdsd_kv_append(const mdsd_kv_cache* cache, int32_t layer, const mdsd_tree* tree, const mdsd_heads* k, const mdsd_heads* v,
                   const mdsd_heads* q, const mdsd_heads* q_out, const float* inv_freq, int32_t rot, int32_t style,
                   int32_t* flags, void* stream)
{
    mdsd_rotary rotary = {};
    rotary.inv_freq = inv_freq;
    rotary.rot = rot;
    rotary.style = style;
    return mdsd_kv_append_at(cache, nullptr, layer, tree, k, v, q, q_out, &rotary, nullptr, nullptr, flags, stream);
}

}  // extern "C"
