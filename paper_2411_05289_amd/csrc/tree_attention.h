// Attention of tree nodes to their sequence and their ancestors: what its kernels share.
//
// A row is a node and a query head of one cache head's group: row r of a tree is node r / G, head r % G of the group.  A
// unit of work is a tile of rows of one tree (of all trees, for a shared prefix) and a cache head; it goes through its keys
// in tiles of slots, from the last to the first.  Scores are formed transposed, S^T = K Q^T, so that a lane holds scores of
// one row only: the softmax's maximum and sum are per lane but for an exchange between the lanes that share a row, and
// the weights are, as they stand in their registers, the right operand of O^T = V^T P^T if V's keys are taken in the same
// order.  For that V stands in LDS as it is stored, a row per key, and the transposing loads (ds_read_b64_tr_b16) give four
// keys of one element to a lane.  fp32 uses the fp32 matrix instructions the same way.
//
// In 16-bit types the weights are rounded to the type, as the matrix instructions take them; the sum that they are divided by takes
// them as they were.  Against 64 bits that is 0.0022 of the results' norm in bf16 and 0.00028 in fp16, of which 0.0017 and 0.0002 are
// the results' own rounding; weights in two parts would take the second product twice.
#pragma once
#include "kv_cache.h"

namespace mdsd {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 fp16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 fp16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 fp16x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

struct AttentionParams {
    Cache cache;
    Trees trees;
    Heads q, out;
    int group;      // query heads per cache head
    int row_tiles;  // of a tree
    Divisor by_group, by_tiles, by_heads, by_rows;  // by_rows: by the rows of a tree, N * group
    float scale;  // times log2(e)
    // A row's weights are 2^(score*scale - shift), see Base; the shift follows the largest score only when that is 8 ahead in
    // the exponent, so that weights reach 2^8 at most (nothing to fp32 sums or to bf16; fp16: 2^15, see kLift)
    float slack;  // 8 / scale
    const int32_t* shared_pages;
    int shared;
    int32_t* flags;
    // joint_tiles > 0: the line of a cache head begins with as many units that let the rows of all trees, row
    // (b*N + n)*G + g, meet the shared prefix, kJointRows at a time; the trees' own units then begin at slot
    // min(shared, length), and have one row tile each.
    int joint_tiles;
    // groups = 0: a workgroup for every unit, results go to `out`.  Otherwise the units' tiles stand in one line, which
    // `groups` workgroups share evenly; a part of a unit leaves its unnormalised sums in `sums`, [units + groups] slots of
    // part_rows x dim, and the score that the rows' weights go by and their sum in `stats`.
    int first_round;  // of trees by their length, see tree_by_length; 0: trees in their order
    int groups;     // a multiple of 8
    int part_rows;  // a tile's rows, or a tree's, see plan_attention
    int unit_cost;  // beginning and ending a unit, in tiles: a unit counts as that many more, before its own
    int32_t* ends;   // [units][2]: the workgroups that had a unit's first and last tile
    float* sums;
    float2* stats;
    float* lse;  // [B, N, query heads], or NULL
    int32_t* joint_ends;
    float* joint_sums;
    float2* joint_stats;
    Scales scales;  // of a cache in 4 bits
    // Heads of a slot that share cache lines: a unit's heads come one behind the other, in one XCD, instead of all units of a head (never
    // with joint_tiles, and only in 4 bits: other builds know nothing of it, as code that is fetched for nothing costs one token behind 8192
    // slots in 16 bits 0.4 us of 16).
    bool by_unit;
};

constexpr int kAttentionThreads = 256;

template <class T>
struct Element;
template <>
struct Element<float> {
    static constexpr float kLift = 0.f;
    static constexpr uint32_t kExponent = 0x7f800000u;
};
template <>
struct Element<__bf16> {
    static constexpr float kLift = 0.f;
    static constexpr uint32_t kExponent = 0x7f80u;
    static __device__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ f32x4 mfma(u32x2 a, u32x2 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(i16x4, a), __builtin_bit_cast(i16x4, b), c, 0, 0, 0);
    }
    static __device__ uint32_t pack(float x, float y)
    {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, bf16x2));
    }
};
template <>
struct Element<_Float16> {
    // weights stand 2^7 higher, 2^15 at most, so that 2^-31 of the largest is still more than zero
    static constexpr float kLift = 7.f;
    static constexpr uint32_t kExponent = 0x7c00u;
    static __device__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(fp16x8, a), __builtin_bit_cast(fp16x8, b), c, 0, 0, 0);
    }
    static __device__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(fp16x8, a), __builtin_bit_cast(fp16x8, b), c, 0, 0, 0);
    }
    static __device__ f32x4 mfma(u32x2 a, u32x2 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(fp16x4, a), __builtin_bit_cast(fp16x4, b), c, 0, 0, 0);
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

// What a row's weights are formed by, 2^((score - origin)*scale - shift), given the score `top` that they go by.  Near scores have no
// origin: a multiplication with a subtraction in it.  Beyond 2^22 the product's steps in fp32 would come near the range
// of a weight's exponent and pass it; there the scores' own difference is taken, which is exact where it matters.
struct Base {
    float origin, shift;
};
template <class T>
__device__ inline Base base_of(float top, float scale)
{
    if (top == -INFINITY) return {0.f, 0.f};  // no key yet
    const float at = top * scale;
    if (fabsf(at) > 4194304.f) return {top, -Element<T>::kLift};
    return {0.f, at - Element<T>::kLift};
}
// what sums of weights that went by `from` are multiplied with where others go by `to`
template <class T>
__device__ inline float rebased(float from, float to, float scale)
{
    if (from == -INFINITY) return 0.f;
    const Base a = base_of<T>(from, scale), b = base_of<T>(to, scale);
    return __builtin_amdgcn_exp2f(__builtin_fmaf(a.origin - b.origin, scale, a.shift - b.shift));
}

// the larger of a lane's value and that of the lane 32 away
__device__ inline float max_of_halves(float x)
{
    const u32x2 both = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
}
// over the four lanes 16 apart
__device__ inline float max_of_quarters(float x)
{
    x = max_of_halves(x);
    const u32x2 both = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
}
__device__ inline float sum_of_halves(float x)
{
    const u32x2 both = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(both[0]) + __uint_as_float(both[1]);
}
__device__ inline float sum_of_quarters(float x)
{
    x = sum_of_halves(x);
    const u32x2 both = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(both[0]) + __uint_as_float(both[1]);
}

// The logarithm of a row's sum, of weights that went by the score `top`: sum = 2^lift * sum_s 2^((score_s - top) * scale).
template <class T>
__device__ inline float log_of_sum(float top, float sum, float scale)
{
    if (sum == 0.f) return -INFINITY;
    return 0.693147180559945f * (__builtin_fmaf(top, scale, -Element<T>::kLift) + __builtin_amdgcn_logf(sum));
}

// four results into the output
template <class T>
__device__ inline void write_four(char* out, int x, f32x4 v)
{
    if constexpr (sizeof(T) == 4)
        *(f32x4*)(out + x * 4) = v;
    else
        *(u32x2*)(out + x * 2) = u32x2{Element<T>::pack(v[0], v[1]), Element<T>::pack(v[2], v[3])};
}

// Which of kSlice slots a node sees of its tree's nodes, a bit for each; `base`: the root's bit.  `ancestor` goes on from
// one call to the next, to slots that lie before.
template <int kSlice>
__device__ inline uint64_t nodes_seen(const Trees& t, const int* parent, int base, int node, int& ancestor)
{
    if (t.complete && t.k == 1) {
        const int upto = base + node;  // 0 .. node
        return upto < 0 ? 0 : upto >= 63 ? ~0ull : (2ull << upto) - 1;
    }
    uint64_t seen = 0;
    while (ancestor >= 0 && ancestor + base >= kSlice) ancestor = parent_of(t, parent, ancestor);
    while (ancestor >= 0 && ancestor + base >= 0) {
        seen |= 1ull << (ancestor + base);
        ancestor = parent_of(t, parent, ancestor);
    }
    return seen;
}
__device__ inline uint64_t low_bits(int n) { return n <= 0 ? 0 : n >= 64 ? ~0ull : (1ull << n) - 1; }

// A unit: a row tile of a tree, and its keys: slots lo .. end-1 in tiles, from lo on.
struct Unit {
    int tree, row_tile, length, count;  // length: as it was given; tree -1: all trees' rows and the shared prefix
    int lo, end, tiles;
};

// The slot at which a tree's own units begin: behind the prefix, where that is met by all trees' rows together.  At `capacity`
// there is none left (the prefix fills the table): these units have no tiles, nobody works on them, and they leave no parts.
__device__ inline int first_own_slot(bool joint, int shared, int length, int capacity)
{
    return joint ? min(min(shared, length), capacity) : 0;
}

template <int kRows, int kKeys>
__device__ inline Unit unit_of(const AttentionParams& P, int tree, int row_tile, int length, int count)
{
    const int rows = count * P.group, first = row_tile * kRows;
    if (length < 0 || first >= rows) return {tree, row_tile, length, count, 0, 0, 0};
    // slots beyond the table have no page; nodes come after their ancestors, so the last node's slot is the last seen
    const int capacity = P.cache.table_pages * P.cache.page_size;
    const int last_node = P.by_group(min(first + kRows, rows) - 1);
    const int end = (int)min((int64_t)length + last_node + 1, (int64_t)capacity);
    const int lo = first_own_slot(P.joint_tiles != 0, P.shared, length, capacity);
    return {tree, row_tile, length, count, lo, end, (end - lo + kKeys - 1) / kKeys};
}
template <int kRows, int kKeys>
__device__ inline Unit unit_of(const AttentionParams& P, int unit)
{
    const int tree = P.by_tiles(unit);
    return unit_of<kRows, kKeys>(P, tree, unit - tree * P.row_tiles, P.cache.lengths[tree], P.trees.count(tree));
}
template <int kKeys>
__device__ inline Unit joint_unit(const AttentionParams& P, int unit)
{
    return {-1, unit, 0, 0, 0, P.shared, (P.shared + kKeys - 1) / kKeys};
}

// A workgroup's share of the line of all units' tiles: it goes cache head by cache head, each with the same units (by_unit: unit by
// unit, each with all cache heads).
struct Share {
    int kv_head, unit, at;  // where it begins: `at` tiles into the unit, the unit's cost counted
    int64_t tiles;          // 0: nothing
    Unit first;
};

// a / b rounded down for whole numbers a < 2^52, b < 2^31: the double quotient's whole part, which a remainder of 1/b at least
// keeps from the next whole number
__device__ inline int64_t quotient(int64_t a, int64_t b) { return (int64_t)((double)a / (double)b); }

// A unit's place among those of all cache heads, in the line's order; units: the trees' own
template <bool kFour>
__device__ inline int place_in_line(const AttentionParams& P, int kv_head, int unit, int units)
{
    return kFour && P.by_unit ? unit * P.cache.heads + kv_head : kv_head * units + unit;
}
// Without a line: a workgroup's unit and cache head.  Neighbours go round the XCDs, one for each head, or with all heads of a unit in one.
template <bool kFour>
__device__ inline int unit_of_group(const AttentionParams& P, int group, int units, int* kv_head)
{
    const int heads = P.cache.heads;
    const bool turned = kFour && P.by_unit && group < (units & ~7) * heads;
    const int at = turned ? group >> 3 : group, unit = P.by_heads(at);
    *kv_head = at - unit * heads;
    return turned ? unit * 8 + (group & 7) : unit;
}

// Every wave finds it on its own, a lane for each unit, 64 units at a time (the tiles of a cache head are below 2^31).
// `units`: the trees' own; with kJoint the joint ones stand before them.
template <int kRows, int kKeys, bool kJoint, bool kFour>
__device__ inline Share share_of(const AttentionParams& P, int units, int group)
{
    const int lane = threadIdx.x & 63;
    const Unit nothing = {};
    auto cost = [&](const Unit& u) { return u.tiles ? u.tiles + P.unit_cost : 0; };
    const Unit mine = lane < units ? unit_of<kRows, kKeys>(P, lane) : nothing;
    const int up_to = sum_up_to(cost(mine)), of_first = __builtin_amdgcn_readlane(up_to, 63);
    const int each = kJoint ? cost(joint_unit<kKeys>(P, 0)) : 0, joint = kJoint ? each * P.joint_tiles : 0;
    int total = joint + of_first;
    for (int from = 64; from < units; from += 64)
        total += __builtin_amdgcn_readlane(sum_up_to(from + lane < units ? cost(unit_of<kRows, kKeys>(P, from + lane)) : 0), 63);
    const int64_t all = (int64_t)total * P.cache.heads;
    const int64_t sharers = min(all, (int64_t)P.groups);  // each has a tile, so that a unit's parts are those of groups in a row
    Share none = {};
    if (group >= sharers) return none;
    const int64_t at = quotient(group * all, sharers), tiles = quotient((group + 1) * all, sharers) - at;
    if (kFour && !kJoint && P.by_unit) {
        int from = 0, sums = up_to, chunk = of_first;
        Unit u = mine;
        int64_t left = at;
        while (left >= (int64_t)chunk * P.cache.heads) {
            left -= (int64_t)chunk * P.cache.heads;
            from += 64;
            u = from + lane < units ? unit_of<kRows, kKeys>(P, from + lane) : nothing;
            sums = sum_up_to(cost(u));
            chunk = __builtin_amdgcn_readlane(sums, 63);
        }
        const int l = __builtin_ctzll(__ballot(sums > (int)quotient(left, P.cache.heads)));
        auto of = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
        const Unit first = {of(u.tree), of(u.row_tile), of(u.length), of(u.count), of(u.lo), of(u.end), of(u.tiles)};
        const int each = cost(first);
        left -= (int64_t)(of(sums) - each) * P.cache.heads;
        const int head = (int)quotient(left, each);
        return {head, from + l, (int)(left - (int64_t)head * each), tiles, first};
    }
    const int head = (int)quotient(at, total);
    int left = (int)(at - (int64_t)head * total);
    if constexpr (kJoint) {
        if (left < joint) {
            const int unit = left / each;
            return {head, unit, left - unit * each, tiles, joint_unit<kKeys>(P, unit)};
        }
    }
    left -= joint;
    int from = 0, sums = up_to, chunk = of_first;
    Unit u = mine;
    while (left >= chunk) {
        left -= chunk;
        from += 64;
        u = from + lane < units ? unit_of<kRows, kKeys>(P, from + lane) : nothing;
        sums = sum_up_to(cost(u));
        chunk = __builtin_amdgcn_readlane(sums, 63);
    }
    const int l = __builtin_ctzll(__ballot(sums > left));
    auto of = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
    const Unit first = {of(u.tree), of(u.row_tile), of(u.length), of(u.count), of(u.lo), of(u.end), of(u.tiles)};
    return {head, (kJoint ? P.joint_tiles : 0) + from + l, left - (of(sums) - cost(first)), tiles, first};
}

// The tree that stands at `place` when up to kMostOrdered trees go by falling length as far as six bits tell, by number beyond
// that: in a launch of a workgroup per tree and head the longest begin first.  Where two rounds are all (first_round < B), the
// second goes from the shortest on, so that a compute unit has a long and a short one.  Every wave finds it on its own, by
// the bits of the lengths from the highest on.
constexpr int kMostOrdered = 256;
__device__ inline int tree_by_length(const AttentionParams& P, int place)
{
    constexpr int kFour = kMostOrdered / 64;  // lengths a lane
    const int lane = threadIdx.x & 63;
    if (place >= P.first_round) place = P.trees.B - 1 - (place - P.first_round);
    int length[kFour], bits = 0;
    uint64_t left[kFour];  // the trees among which the place is
#pragma unroll
    for (int i = 0; i < kFour; ++i) {
        const int b = i * 64 + lane;
        length[i] = b < P.trees.B ? max(P.cache.lengths[b], 0) : 0;
        left[i] = __ballot(b < P.trees.B);
        bits |= length[i];
    }
    bits |= __builtin_amdgcn_update_dpp(0, bits, 0x111, 0xf, 0xf, false);
    bits |= __builtin_amdgcn_update_dpp(0, bits, 0x112, 0xf, 0xf, false);
    bits |= __builtin_amdgcn_update_dpp(0, bits, 0x114, 0xf, 0xf, false);
    bits |= __builtin_amdgcn_update_dpp(0, bits, 0x118, 0xf, 0xf, false);
    bits |= __builtin_amdgcn_update_dpp(0, bits, 0x142, 0xa, 0xf, false);
    bits |= __builtin_amdgcn_update_dpp(0, bits, 0x143, 0xc, 0xf, false);
    bits = __builtin_amdgcn_readlane(bits, 63);
    const int top = 31 - __builtin_clz(bits | 64);
    for (int bit = top; bit > top - 6; --bit) {
        uint64_t ones[kFour];
        int n = 0;
#pragma unroll
        for (int i = 0; i < kFour; ++i) {
            ones[i] = __ballot(length[i] >> bit & 1) & left[i];
            n += __builtin_popcountll(ones[i]);
        }
        const bool among = place < n;
        if (!among) place -= n;
#pragma unroll
        for (int i = 0; i < kFour; ++i) left[i] = among ? ones[i] : left[i] & ~ones[i];
    }
    int i = 0;
    uint64_t of = left[0];
#pragma unroll
    for (int j = 1; j < kFour; ++j) {
        const int n = __builtin_popcountll(of);
        if (i == j - 1 && place >= n) {
            place -= n;
            of = left[j];
            i = j;
        }
    }
    const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(of >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)of, 0));
    const uint64_t there = __ballot(before == place && (of >> lane & 1));
    return i * 64 + __builtin_ctzll(there);
}

// Whose part of a unit it is, for the combination.
__device__ inline void note_part(int32_t* ends, int unit, int group, bool has_first, bool has_last)
{
    if (threadIdx.x) return;
    if (has_first) ends[2 * unit] = group;
    if (has_last) ends[2 * unit + 1] = group;
}

constexpr int kJointRows = 128;

}  // namespace mdsd
