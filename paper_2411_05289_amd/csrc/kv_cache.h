// What the key-value cache calls share: the cache and the trees as the kernels see them, the way from a slot
// to its place in the pages, and the way from a node to its parent.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mdsd.h"

namespace mdsd {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// n / d for 0 <= n < 2^31 by a multiplication: with L = ceil(log2 d) and mul = ceil(2^(31+L) / d), mul*d exceeds
// 2^(31+L) by less than 2^L, so n*mul / 2^(31+L) exceeds n/d by less than 1/d and has the same whole part (Granlund and
// Montgomery, "Division by invariant integers using multiplication", 1994).  mul < 2^32.
struct Divisor {
    uint32_t mul;
    int shift;
    __host__ static Divisor of(int d)
    {
        if (d <= 1) return {1, 0};
        int L = 0;
        while ((int64_t(1) << L) < d) ++L;
        const uint64_t top = uint64_t(1) << (31 + L);
        return {(uint32_t)((top + d - 1) / d), 31 + L};
    }
    __device__ int operator()(int n) const { return (int)(((uint64_t)(uint32_t)n * mul) >> shift); }
};

constexpr int64_t kMostGroups = (1 << 24) - 1;  // of a launch, of 256 threads: HIP takes less than 2^32 threads along a side
constexpr int kMostSlots = 1 << 30;  // of a sequence, and nodes of a tree: their sums stay whole numbers of 32 bits

struct Cache {
    char* k;  // of the layer that is worked on
    char* v;
    int64_t ld_layer, ld_head;   // in bytes
    uint32_t ld_page, ld_slot;   // in units of 16 bytes
    const int32_t* table;
    int64_t ld_table;
    const int32_t* lengths;
    int layers, pages, page_size, heads, dim, table_pages;
    Divisor by_page;
};

struct Trees {
    int B, N, k;
    bool complete;  // no table: parents by arithmetic
    const int32_t* first_child;
    const int32_t* counts;
    Divisor by_k;

    __device__ int count(int b) const { return counts ? max(0, min(counts[b], N)) : N; }
};

struct Heads {
    char* p;
    int64_t ld_tree, ld_node, ld_head;  // in bytes
    int heads;
};

// Where slot s of the sequence with this table lies, in bytes from k or v; -1 if it has no page.
__device__ inline int64_t place_in_page(const Cache& c, int page, int s, int entry)
{
    if ((uint32_t)page >= (uint32_t)c.pages) return -1;
    return (int64_t)(((uint64_t)(uint32_t)page * c.ld_page + (uint64_t)(uint32_t)(s - entry * c.page_size) * c.ld_slot) << 4);
}
__device__ inline int64_t place_of(const Cache& c, const int32_t* table, int64_t s)
{
    if (s < 0 || s > INT32_MAX) return -1;
    const int entry = c.by_page((int)s);
    return entry < c.table_pages ? place_in_page(c, table[entry], (int)s, entry) : -1;
}

// The parents of a tree given by a table, by all threads of a workgroup (barriers inside).  A node that several
// entries claim is the last one's child.
__device__ inline void parents_from_table(const Trees& t, int* parent)
{
    for (int n = threadIdx.x; n < t.N; n += blockDim.x) parent[n] = -1;
    __syncthreads();
    for (int n = threadIdx.x; n < t.N; n += blockDim.x) {
        const int c = t.first_child[n];
        if (c > n && c <= t.N - t.k)
            for (int j = 0; j < t.k; ++j) atomicMax(&parent[c + j], n);
    }
    __syncthreads();
}
// -1: a root.  Parents come before their children, so that a walk upwards ends.
__device__ inline int parent_of(const Trees& t, const int* parent, int n)
{
    if (!t.complete) return parent[n];
    return n > 0 ? t.by_k(n - 1) : -1;
}

// A cache in 4 bits, of the layer that is worked on: the scale of the 16 bytes at offset o of k (32 elements) stands at o / 16 here.
struct Scales {
    uint8_t* k;
    uint8_t* v;
};
constexpr int kBlock = 32;          // elements that share a scale
constexpr uint32_t kNoNumber = 255;  // a scale whose block holds an infinity or NaN, and stands for NaN
constexpr uint32_t kUnitScale = 127;

// Sum over the lanes up to each, by data-parallel moves: within rows of 16, then from row to row.
__device__ inline int sum_up_to(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}

// The node behind `node` on an accepted path; -1: the path ends.
__device__ inline int next_of_path(const Trees& t, int node, int count, int outcome)
{
    if (outcome < 0 || outcome >= t.k) return -1;
    const int64_t first = t.complete ? (int64_t)t.k * node + 1 : t.first_child[node];
    if (first <= node || first + t.k > t.N || first + outcome >= count) return -1;
    return (int)first + outcome;
}

// kv_cache.hip: what the host can detect, and the structures above from the caller's
int check_cache(const mdsd_kv_cache* c, const mdsd_tree* t, Cache* C, Trees* T);
// the same for a call that also takes caches in 4 bits (`scales` given); *dtype: of vectors, *S: not of a layer yet
int check_cache(const mdsd_kv_cache* c, const mdsd_kv_scales* scales, const mdsd_tree* t, Cache* C, Scales* S, int* dtype, Trees* T);
// what there is to check of a cache alone (of B sequences)
int check_pages(const mdsd_kv_cache* c, const mdsd_kv_scales* scales, Cache* C, Scales* S, int* dtype);
void choose_layer(int layer, Cache* C, Scales* S);
int check_heads(const mdsd_heads* h, const Cache& c, int dtype, Heads* H);
// strides of zero: several elements that are one place, which may be read and not written
bool one_place(const mdsd_kv_cache& c);
bool one_place(const mdsd_heads& h, const Trees& t);
// whether results of a call would be written where others of its vectors `from` stand: the two share a place without being the same
// array (found where their strides agree or they begin at one place; strided otherwise they are the caller's to keep apart)
bool overlap(const Heads& from, const Heads& to, const Trees& t, const Cache& c, int dtype);
// whether two arrays of B rows of 32-bit numbers share a place without being the same (with different strides: whether their
// stretches of memory meet)
bool rows_overlap(const void* a, int64_t ld_a, const void* b, int64_t ld_b, int64_t B, int64_t width);
constexpr int kEmptyTrees = 1;  // check_cache: a batch of no trees

}  // namespace mdsd
