// Attention of tree nodes to their sequence and their ancestors: device code.
//
// A workgroup takes 128 rows (a row is a node and a query head of one cache head's group: row r of a tree is node
// r / G, head r % G of the group) and goes through the keys in tiles of kKeys slots, from the last to the first.
// Each of its four waves owns 32 rows.  Scores are formed transposed, S^T = K Q^T, so that a lane holds scores of one row
// only (column lane % 32; the other half-wave has the row's other keys): the softmax's maximum and sum are per lane but
// for one exchange between the halves, and the weights are, as they stand in their registers, the right operand of
// O^T = V^T P^T if V's keys are taken in the same order.  For that V stays as it is stored, a row per key, and the
// transposing LDS loads (ds_read_b64_tr_b16) give four keys of one element to a lane.  fp32 uses the 32x32x2 fp32 matrix
// instruction the same way.
//
// Keys and values go through registers into LDS (two buffers, one barrier a tile; the next tile is on its way while one
// is worked on).  A row's 16-byte chunks are stored XORed by the key's low bits, so that the 32 keys that one load of K
// takes at one chunk, and the four keys that one transposing load of V takes, lie in different banks.
#pragma once
#include "kv_cache.h"

namespace mdsd {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 fp16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 fp16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

struct AttentionParams {
    Cache cache;
    Trees trees;
    Heads q, out;
    int group;      // query heads per cache head
    int row_tiles;  // of a tree
    Divisor by_group;
    float scale;  // times log2(e)
    const int32_t* shared_pages;
    int shared;
    int32_t* flags;
};

constexpr int kRowsOfTile = 128, kAttentionThreads = 256;

template <class T>
struct Element;
template <>
struct Element<float> {
    static constexpr uint32_t kExponent = 0x7f800000u;
};
template <>
struct Element<__bf16> {
    static constexpr uint32_t kExponent = 0x7f80u;
    static __device__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ uint32_t pack(float x, float y)
    {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, bf16x2));
    }
};
template <>
struct Element<_Float16> {
    static constexpr uint32_t kExponent = 0x7c00u;
    static __device__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(fp16x8, a), __builtin_bit_cast(fp16x8, b), c, 0, 0, 0);
    }
    static __device__ uint32_t pack(float x, float y)
    {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, fp16x2));
    }
};

template <class T>
__device__ inline bool is_number(uint32_t bits)
{
    return (bits & Element<T>::kExponent) != Element<T>::kExponent;
}
// whether a chunk has an infinity or NaN
template <class T>
__device__ inline bool has_nonfinite(u32x4 x)
{
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bad |= !is_number<T>(x[i]);
        if (sizeof(T) == 2) bad |= !is_number<T>(x[i] >> 16);
    }
    return bad;
}
// the chunk with zeros in their place
template <class T>
__device__ inline u32x4 finite_part(u32x4 x)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (sizeof(T) == 4) {
            if (!is_number<T>(x[i])) x[i] = 0;
        } else {
            if (!is_number<T>(x[i])) x[i] &= 0xffff0000u;
            if (!is_number<T>(x[i] >> 16)) x[i] &= 0xffffu;
        }
    }
    return x;
}

// the larger of a lane's value and that of the lane 32 away
__device__ inline float max_of_halves(float x)
{
    const u32x2 both = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
}
__device__ inline float sum_of_halves(float x)
{
    const u32x2 both = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(both[0]) + __uint_as_float(both[1]);
}

// kDim: the head's elements, filled up with zeros to 64, 128 or 256
template <class T, int kDim>
struct AttentionTile {
    static constexpr int kRowBytes = kDim * sizeof(T);
    static constexpr int kChunks = kRowBytes / 16;
    static constexpr int kKeys = kRowBytes <= 256 ? 64 : 32;
    static constexpr int kBytes = kKeys * kRowBytes;                    // of K or V
    static constexpr int kPerThread = kKeys * kChunks / kAttentionThreads;
    static constexpr int kQueryChunks = kRowBytes / 32;  // per lane: the half-waves have every other one
    static constexpr int kSets = kKeys / 32, kOuts = kDim / 32;
    static constexpr size_t kLds = 4 * kBytes;

    // where chunk c of a key stands in its row
    static __device__ int k_chunk(int key, int c) { return c ^ (kChunks == 8 ? (key >> 1) & 7 : key & 15); }
    static __device__ int v_chunk(int key, int c)
    {
        if (sizeof(T) == 4) return c ^ ((key >> 2 & 1) << 3);
        return c ^ (kChunks == 8 ? (key >> 1 & 1) << 2 : (key & 3) << 2);
    }
};

template <class T, int kDim>
__global__ __launch_bounds__(kAttentionThreads, (kDim * sizeof(T) <= 256 ? 2 : 1)) void tree_attention_kernel(AttentionParams P)
{
    using A = AttentionTile<T, kDim>;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    char *const k_lds = lds, *const v_lds = lds + 2 * A::kBytes;
    int* const parent = (int*)(lds + A::kLds);
    __shared__ int bad_values[2];  // the tile that a buffer's infinities and NaNs were taken from

    const Cache& C = P.cache;
    const Trees& R = P.trees;
    // neighbouring workgroups have different cache heads: with 8 of them (or a multiple) all tiles of a head meet in
    // one XCD's L2.  The last row tiles of a tree see the most keys and come first.
    const int kv_head = blockIdx.x % C.heads;
    const int rest = blockIdx.x / C.heads;
    const int tile_of_tree = P.row_tiles - 1 - rest % P.row_tiles, b = rest / P.row_tiles;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, col = lane & 31;

    const int count = R.count(b);
    const int first_row = tile_of_tree * kRowsOfTile, rows = count * P.group;
    if (first_row >= rows) return;
    int length = C.lengths[b];
    if (length < 0) {
        if (P.flags && threadIdx.x == 0) atomicOr(&P.flags[b], MDSD_FLAG_NO_PAGE);
        return;
    }
    const int capacity = C.table_pages * C.page_size;
    const int own_row = first_row + wave * 32 + col;
    const bool valid = own_row < rows;
    const int row = min(own_row, rows - 1), node = P.by_group(row), head = kv_head * P.group + row - node * P.group;
    const int last_node = P.by_group(min(first_row + kRowsOfTile, rows) - 1);
    // slots beyond `capacity` have no page; nodes come after their ancestors, so the last node's slot is the last seen
    const int64_t wanted = (int64_t)length + last_node + 1;
    const int end = (int)min(wanted, (int64_t)capacity);
    if (wanted > capacity && P.flags && threadIdx.x == 0) atomicOr(&P.flags[b], MDSD_FLAG_NO_PAGE);
    length = min(length, capacity);
    const int shared = min(P.shared, length);
    const int32_t* const table = C.table + b * C.ld_table;
    if (!R.complete) parents_from_table(R, parent);

    u32x4 q[A::kQueryChunks];
    const char* const q_row = P.q.p + b * P.q.ld_tree + node * P.q.ld_node + head * P.q.ld_head;
#pragma unroll
    for (int c = 0; c < A::kQueryChunks; ++c) {
        const int chunk = 2 * c + half;
        q[c] = chunk * 16 < C.dim * (int)sizeof(T) ? *(const u32x4*)(q_row + chunk * 16) : u32x4{0, 0, 0, 0};
    }
    f32x16 o[A::kOuts];
#pragma unroll
    for (int d = 0; d < A::kOuts; ++d) o[d] = f32x16{};
    float top = -INFINITY, shift = 0.f, sum = 0.f;  // largest score; it times the scale, as subtracted; sum of weights
    int ancestor = node;                            // next of the row's nodes that no tile had yet

    const char* const k_head = C.k + kv_head * C.ld_head;
    const char* const v_head = C.v + kv_head * C.ld_head;
    const int tiles = (end + A::kKeys - 1) / A::kKeys;

    // the page of the lane's key of a tile; -1 outside
    auto page_of = [&](int tile) {
        const int s = tile * A::kKeys + (lane & (A::kKeys - 1));
        if (tile < 0 || s >= end) return -1;
        const int entry = C.by_page(s);
        return s < shared ? P.shared_pages[entry] : table[entry];
    };
    u32x4 k_in[A::kPerThread], v_in[A::kPerThread];
    // asks for a tile's keys and values; `place`: of the lane's key
    auto load = [&](int64_t place) {
#pragma unroll
        for (int i = 0; i < A::kPerThread; ++i) {
            const int at = threadIdx.x + i * kAttentionThreads, key = at / A::kChunks, c = at % A::kChunks;
            const int lo = __shfl((int)(uint32_t)place, key), hi = __shfl((int)(place >> 32), key);
            k_in[i] = v_in[i] = u32x4{0, 0, 0, 0};
            if (hi >= 0 && c * 16 < C.dim * (int)sizeof(T)) {
                const int64_t offset = ((int64_t)hi << 32 | (uint32_t)lo) + c * 16;
                k_in[i] = *(const u32x4*)(k_head + offset);
                v_in[i] = *(const u32x4*)(v_head + offset);
            }
        }
    };
    auto store = [&](int tile, int buffer) {
        if ((tile + 1) * A::kKeys > length) {
            // some rows do not see all of these keys: a weight of zero times an infinity or NaN is not zero, so these
            // stay out of the product and are added below for the rows that see them
            bool bad = false;
#pragma unroll
            for (int i = 0; i < A::kPerThread; ++i) {
                bad |= has_nonfinite<T>(v_in[i]);
                v_in[i] = finite_part<T>(v_in[i]);
            }
            if (bad) bad_values[buffer] = tile;
        }
#pragma unroll
        for (int i = 0; i < A::kPerThread; ++i) {
            const int at = threadIdx.x + i * kAttentionThreads, key = at / A::kChunks, c = at % A::kChunks;
            *(u32x4*)(k_lds + buffer * A::kBytes + key * A::kRowBytes + A::k_chunk(key, c) * 16) = k_in[i];
            *(u32x4*)(v_lds + buffer * A::kBytes + key * A::kRowBytes + A::v_chunk(key, c) * 16) = v_in[i];
        }
    };
    auto place_in_tile = [&](int tile, int page) {
        const int s = tile * A::kKeys + (lane & (A::kKeys - 1));
        if (tile < 0 || s >= end) return (int64_t)-1;
        return place_in_page(C, page, s, C.by_page(s));
    };

    if (threadIdx.x < 2) bad_values[threadIdx.x] = -1;
    __syncthreads();
    int64_t place = place_in_tile(tiles - 1, page_of(tiles - 1));
    int next_page = page_of(tiles - 2);
    load(place);
    store(tiles - 1, 0);
    __syncthreads();

    for (int tile = tiles - 1, buffer = 0; tile >= 0; --tile, buffer ^= 1) {
        const int64_t here = place;
        if (tile > 0) {
            place = place_in_tile(tile - 1, next_page);
            load(place);
            next_page = page_of(tile - 2);
        }
        const char* const kb = k_lds + buffer * A::kBytes;
        const char* const vb = v_lds + buffer * A::kBytes;
        f32x16 s[A::kSets];
#pragma unroll
        for (int t = 0; t < A::kSets; ++t) {
            s[t] = f32x16{};
            const int key = t * 32 + col;
#pragma unroll
            for (int c = 0; c < A::kQueryChunks; ++c) {
                const u32x4 k = *(const u32x4*)(kb + key * A::kRowBytes + A::k_chunk(key, 2 * c + half) * 16);
                if constexpr (sizeof(T) == 4) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        s[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k[j]), __uint_as_float(q[c][j]), s[t], 0, 0, 0);
                } else {
                    s[t] = Element<T>::mfma(k, q[c], s[t]);
                }
            }
        }

        // which of the tile's keys the row sees, a bit for each
        const int first = tile * A::kKeys;
        const uint64_t absent = __ballot(here < 0);  // keys without a page, and slots behind the last
        uint64_t seen = ~absent;
        const bool masked = first + A::kKeys > length || absent != 0;
        if (masked) {
            const int in_sequence = max(0, min(length - first, 64));  // keys of the sequence itself
            uint64_t own = in_sequence == 64 ? ~0ull : (1ull << in_sequence) - 1;
            const int base = length - first;  // the root's bit
            if (R.complete && R.k == 1) {
                const int upto = base + node;  // 0 .. node
                if (upto >= 0) own |= upto >= 63 ? ~0ull : (2ull << upto) - 1;
            } else {
                while (ancestor >= 0 && ancestor + base >= A::kKeys) ancestor = parent_of(R, parent, ancestor);
                while (ancestor >= 0 && ancestor + base >= 0) {
                    own |= 1ull << (ancestor + base);
                    ancestor = parent_of(R, parent, ancestor);
                }
            }
            seen &= own;
            if (P.flags && (absent & (end - first >= 64 ? ~0ull : (1ull << (end - first)) - 1)) && lane == 0)
                atomicOr(&P.flags[b], MDSD_FLAG_NO_PAGE);
#pragma unroll
            for (int t = 0; t < A::kSets; ++t) {
                const uint32_t bits = (uint32_t)(seen >> (t * 32 + 4 * half));
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (!(bits >> (8 * (i / 4) + i % 4) & 1)) s[t][i] = -INFINITY;
            }
        }

        float most = s[0][0];
#pragma unroll
        for (int t = 0; t < A::kSets; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) most = fmaxf(most, s[t][i]);
        most = fmaxf(max_of_halves(most), top);
        if (__any(most > top)) {
            // scores may exceed the shift by nothing: the weights are at most 1
            const float new_shift = most == -INFINITY ? 0.f : most * P.scale;
            const float factor = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(shift - new_shift);
            top = most;
            shift = new_shift;
            sum *= factor;
#pragma unroll
            for (int d = 0; d < A::kOuts; ++d) o[d] *= factor;
        }
#pragma unroll
        for (int t = 0; t < A::kSets; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], P.scale, -shift));
                sum += s[t][i];
            }

        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int t = 0; t < A::kSets; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = t * 32 + 8 * (i / 4) + 4 * half + i % 4;
#pragma unroll
                    for (int d = 0; d < A::kOuts; ++d) {
                        const int x = d * 32 + col;
                        const float v = *(const float*)(vb + key * A::kRowBytes + A::v_chunk(key, x / 4) * 16 + x % 4 * 4);
                        o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[t][i], o[d], 0, 0, 0);
                    }
                }
        } else {
            const int in_four = lane & 15;
#pragma unroll
            for (int kk = 0; kk < A::kKeys / 16; ++kk) {
                const f32x16& w = s[kk / 2];
                const int r = 8 * (kk & 1);
                const u32x4 p = {Element<T>::pack(w[r], w[r + 1]), Element<T>::pack(w[r + 2], w[r + 3]),
                                 Element<T>::pack(w[r + 4], w[r + 5]), Element<T>::pack(w[r + 6], w[r + 7])};
#pragma unroll
                for (int d = 0; d < A::kOuts; ++d) {
                    u32x4 v;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int key = 16 * kk + 8 * j + 4 * half + in_four / 4;
                        const int c = d * 4 + (lane >> 4 & 1) * 2 + (in_four & 3) / 2;
                        const char* at = vb + key * A::kRowBytes + A::v_chunk(key, c) * 16 + (in_four & 1) * 8;
                        const u32x2 four = __builtin_bit_cast(
                            u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)at));
                        v[2 * j] = four[0];
                        v[2 * j + 1] = four[1];
                    }
                    o[d] = Element<T>::mfma(v, p, o[d]);
                }
            }
        }
        if (masked && bad_values[buffer] == tile) {
            for (int key = 0; key < A::kKeys; ++key) {
                const int64_t offset = __shfl((long long)here, key);
                if (offset < 0) continue;
                const bool sees = seen >> key & 1;
#pragma unroll
                for (int d = 0; d < A::kOuts; ++d)
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const int x = d * 32 + 2 * i + 4 * half;
                        const T* const v = (const T*)(v_head + offset) + x;
                        if (sees && x < C.dim)
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                if (!__builtin_isfinite((float)v[j])) o[d][i + j] += (float)v[j];
                        __builtin_amdgcn_sched_barrier(0);  // a rare loop must not take registers from the others
                    }
            }
        }
        if (tile > 0) store(tile - 1, buffer ^ 1);
        __syncthreads();
    }

    sum = sum_of_halves(sum);
    const float over = sum == 0.f ? 0.f : 1.f / sum;
    if (!valid) return;
    char* const out = P.out.p + b * P.out.ld_tree + node * P.out.ld_node + head * P.out.ld_head;
#pragma unroll
    for (int d = 0; d < A::kOuts; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int x = d * 32 + 2 * i + 4 * half;
            if (x >= C.dim) continue;
            if constexpr (sizeof(T) == 4) {
                *(f32x4*)(out + x * 4) = f32x4{o[d][i] * over, o[d][i + 1] * over, o[d][i + 2] * over, o[d][i + 3] * over};
            } else {
                *(u32x2*)(out + x * 2) = u32x2{Element<T>::pack(o[d][i] * over, o[d][i + 1] * over),
                                               Element<T>::pack(o[d][i + 2] * over, o[d][i + 3] * over)};
            }
        }
}

}  // namespace mdsd
