// Attention for trees of few rows (up to 32): what bounds it is reading the keys.
//
// A workgroup's four waves take a quarter of every 128 keys each (64 keys, where rows are long), and all of the rows, 16 at a
// time: a wave never waits for another until the unit ends.  K goes from memory into the registers that the matrix instruction reads (a lane holds
// chunks of one key), V through the wave's own LDS, where the transposing loads turn it.  The next keys are asked for
// as soon as the registers of the present ones are free.  In the end the waves' sums are scaled to go by one score and added
// in LDS, every thread adding four elements of a row.
//
// Measured: 64 tokens behind 512 to 8192 slots, 32 heads over 8 of 128, bf16, 1.14 GB in 180 us, 6.3 TB/s; one token behind 8192
// slots 16 us, of which 12 here, most of them the way from the lengths to the pages to the keys; 48 fp32 trees of 9 nodes in
// heads of 80, 375 MB in 92 us, 4.1 TB/s (the fp32 products, on rows filled up to 16 x 128, take half of that).
#pragma once
#include <type_traits>

#include "tree_attention.h"

namespace mdsd {

// kDim: the head's elements, filled up to 64, 128 or 256; kSlice: the keys of a wave, 16 or 32, of each tile
template <class T, int kDim, int kRowTiles, int kSlice>
struct NarrowTile {
    static constexpr int kRowBytes = kDim * sizeof(T), kChunks = kRowBytes / 16;
    static constexpr int kRows = 16 * kRowTiles, kKeys = 4 * kSlice, kTiles = kSlice / 16;
    static constexpr int kKeyChunks = kChunks / 4;  // of K, per lane and key
    static constexpr int kStaged = kSlice * kChunks / 64;  // of V, per lane
    static constexpr int kOuts = kDim / 16;
    static constexpr int kValues = kSlice * kRowBytes;  // of a wave
    static constexpr int kJoin = 4 * kRows * kDim * 4;
    static constexpr int kLds = 4 * kValues > kJoin ? 4 * kValues : kJoin;
    // waves on a SIMD: by the registers of Q, O, the scores and the keys on their way; shared-out units need some more (24 rows of
    // bf16 heads of 128 behind 8192 slots, 8 sequences: 74 us with two waves and a few registers too many, 60 with one)
    static constexpr int kRegisters = kRowTiles * (kRowBytes / 16 + kDim / 4 + 20) + kSlice * kRowBytes / 128 + 64;
    static constexpr int per_unit(bool line)
    {
        return kRegisters <= 168 && kLds <= 48 * 1024 ? 3 : kRegisters <= (line ? 256 : 288) && kLds <= 76 * 1024 ? 2 : 1;
    }
    static_assert(kLds <= 144 * 1024, "LDS");

    // where chunk c of a key stands in its row of V: eight keys' 32 bytes (fp32: four keys' 64) in different banks
    static __device__ int v_chunk(int key, int c)
    {
        if (sizeof(T) == 4) return c ^ ((key >> 2 & 3) << 2);
        return c ^ (kChunks == 8 ? (key >> 1 & 3) << 1 : (key & 7) << 1);
    }
};

// No other workgroup reads these keys: they need not stay in the caches (a stream of 1 GB 6.1 -> 7.0 TB/s).  Heads that do not
// fill their lines share them with the next heads', which other workgroups read.
template <bool kWholeLines>
__device__ inline u32x4 read_once(const char* at)
{
    if constexpr (kWholeLines)
        return __builtin_nontemporal_load((const u32x4*)at);
    else
        return *(const u32x4*)at;
}

// kLine: P.groups workgroups share the line of tiles; else one for every unit.  kExact: dim is kDim.
template <class T, int kDim, int kRowTiles, int kSlice, bool kLine, bool kExact>
__global__ __launch_bounds__(kAttentionThreads, (NarrowTile<T, kDim, kRowTiles, kSlice>::per_unit(kLine))) void attention_narrow_kernel(AttentionParams P)
{
    using A = NarrowTile<T, kDim, kRowTiles, kSlice>;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    int* const parent = (int*)(lds + A::kLds);
    __shared__ float2 stats[4][A::kRows];  // of each wave: the score that its weights go by, and their sum once all go by one

    const Cache& C = P.cache;
    const Trees& R = P.trees;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quarter = lane >> 4, col = lane & 15;
    const int units = R.B * P.row_tiles;  // of a cache head
    const int capacity = C.table_pages * C.page_size;
    char* const v_lds = lds + wave * A::kValues;

    int kv_head, unit, at = 0, group = 0;
    int64_t left = INT64_MAX;  // tiles of the share
    Unit keys;
    if constexpr (!kLine) {
        unit = P.by_heads(blockIdx.x);
        kv_head = blockIdx.x - unit * C.heads;
        if (P.first_round) unit = tree_by_length(P, unit);
        keys = unit_of<A::kRows, A::kKeys>(P, unit);
        if (keys.tiles == 0) {
            if (P.flags && threadIdx.x == 0 && keys.row_tile == 0 && keys.length < 0) atomicOr(&P.flags[keys.tree], MDSD_FLAG_NO_PAGE);
            return;
        }
    } else {
        // workgroups go round the XCDs: each XCD has a stretch of the line, which goes head by head
        group = blockIdx.x % 8 * (P.groups / 8) + blockIdx.x / 8;
        const Share s = share_of<A::kRows, A::kKeys, false>(P, units, group);
        if (s.tiles == 0) return;
        left = s.tiles;
        kv_head = s.kv_head;
        unit = s.unit;
        at = s.at;
        keys = s.first;
    }
    if (!R.complete) parents_from_table(R, parent);

    for (;;) {
        const int b = keys.tree, row_tile = keys.row_tile;
        // tiles tile_to-1 down to tile_from of the unit
        int tile_from = 0, tile_to = keys.tiles;
        if constexpr (kLine) {
            const int end = (int)min((int64_t)keys.tiles + P.unit_cost, at + left);
            left -= end - at;
            tile_from = max(0, at - P.unit_cost);
            tile_to = end - P.unit_cost;
            if (tile_to <= tile_from) return;  // the share ends before the unit's tiles begin
        }
        const int rows = keys.count * P.group, first_row = row_tile * A::kRows;
        int length = keys.length;
        if (P.flags && threadIdx.x == 0 && tile_to == keys.tiles &&
            (int64_t)length + P.by_group(min(first_row + A::kRows, rows) - 1) >= capacity)
            atomicOr(&P.flags[b], MDSD_FLAG_NO_PAGE);
        length = min(length, capacity);
        const int shared = min(P.shared, length);
        const int32_t* const table = C.table + b * C.ld_table;
        const char* const k_head = C.k + kv_head * C.ld_head;
        const char* const v_head = C.v + kv_head * C.ld_head;

        // a lane looks up the page of one of its wave's keys; -1 outside
        const int lane_slot = keys.lo + wave * kSlice + (lane & (kSlice - 1));
        auto page_of = [&](int tile) {
            const int s = lane_slot + tile * A::kKeys;
            if (tile < tile_from || s >= keys.end) return -1;
            const int entry = C.by_page(s);
            return s < shared ? P.shared_pages[entry] : table[entry];
        };
        auto place_in_tile = [&](int tile, int page) {
            const int s = lane_slot + tile * A::kKeys;
            if (tile < tile_from || s >= keys.end) return (int64_t)-1;
            return place_in_page(C, page, s, C.by_page(s));
        };
        auto place_from = [&](int64_t place, int from) {
            const int lo = __shfl((int)(uint32_t)place, from), hi = __shfl((int)(place >> 32), from);
            // (a key without a page is left out below; its loads go to the cache's first place)
            return hi < 0 ? (int64_t)0 : (int64_t)hi << 32 | (uint32_t)lo;
        };
        const int dim_bytes = C.dim * (int)sizeof(T);
        u32x4 k[A::kTiles][A::kKeyChunks], v[A::kStaged];
        auto load_k = [&](int64_t place) {
#pragma unroll
            for (int t = 0; t < A::kTiles; ++t) {
                const char* const at = k_head + place_from(place, t * 16 + col);
#pragma unroll
                for (int i = 0; i < A::kKeyChunks; ++i) {
                    const int c = quarter * 16 + i * 64;
                    k[t][i] = read_once<kExact>(at + (kExact ? c : min(c, dim_bytes - 16)));
                }
            }
        };
        const int v_column = kExact ? lane % A::kChunks * 16 : min(lane % A::kChunks * 16, dim_bytes - 16);
        auto load_v = [&](int64_t place) {
#pragma unroll
            for (int i = 0; i < A::kStaged; ++i)
                v[i] = read_once<kExact>(v_head + place_from(place, (lane + i * 64) / A::kChunks) + v_column);
        };

        // the wave's own last tile: the unit's may end before the wave's quarter of it begins
        const int to = min(tile_to, (keys.end - keys.lo - wave * kSlice + A::kKeys - 1) / A::kKeys);
        int64_t place = place_in_tile(to - 1, page_of(to - 1));
        int next_page = page_of(to - 2);
        if (to > tile_from) {
            load_k(place);
            load_v(place);
        }

        u32x4 q[kRowTiles][A::kKeyChunks];
        int node[kRowTiles], ancestor[kRowTiles];
#pragma unroll
        for (int r = 0; r < kRowTiles; ++r) {
            const int row = min(first_row + r * 16 + col, rows - 1);
            node[r] = ancestor[r] = P.by_group(row);
            const int head = kv_head * P.group + row - node[r] * P.group;
            const char* const from = P.q.p + b * P.q.ld_tree + node[r] * P.q.ld_node + head * P.q.ld_head;
#pragma unroll
            for (int i = 0; i < A::kKeyChunks; ++i) {
                const int at = quarter * 16 + i * 64;
                q[r][i] = u32x4{0, 0, 0, 0};
                if (kExact || at < dim_bytes) q[r][i] = *(const u32x4*)(from + at);
            }
        }
        f32x4 o[kRowTiles][A::kOuts];
        float top[kRowTiles], shift[kRowTiles], sum[kRowTiles];  // score and shift that the weights go by; their sum
        bool far = false;  // a row of the wave has an origin
#pragma unroll
        for (int r = 0; r < kRowTiles; ++r) {
#pragma unroll
            for (int d = 0; d < A::kOuts; ++d) o[r][d] = f32x4{0.f, 0.f, 0.f, 0.f};
            top[r] = -INFINITY;
            shift[r] = sum[r] = 0.f;
        }

        for (int tile = to - 1; tile >= tile_from; --tile) {
            const int64_t here = place;
            place = place_in_tile(tile - 1, next_page);
            next_page = page_of(tile - 2);

            if constexpr (!kExact) {  // what was read in place of the elements that are not there may be no number
#pragma unroll
                for (int i = 0; i < A::kKeyChunks; ++i)
                    if (quarter * 16 + i * 64 >= dim_bytes) k[0][i] = k[A::kTiles - 1][i] = u32x4{0, 0, 0, 0};
            }
            f32x4 s[kRowTiles][A::kTiles];
#pragma unroll
            for (int r = 0; r < kRowTiles; ++r)
#pragma unroll
                for (int t = 0; t < A::kTiles; ++t) {
                    s[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int i = 0; i < A::kKeyChunks; ++i) {
                        if constexpr (sizeof(T) == 4) {
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                s[r][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[t][i][j]),
                                                                               __uint_as_float(q[r][i][j]), s[r][t], 0, 0, 0);
                        } else {
                            s[r][t] = Element<T>::mfma(k[t][i], q[r][i], s[r][t]);
                        }
                    }
                }
            if (tile > tile_from) load_k(place);

            const int first = keys.lo + tile * A::kKeys + wave * kSlice;
            const uint32_t absent = (uint32_t)__ballot(here < 0) & (uint32_t)low_bits(kSlice);  // keys without a page, and slots behind the last
            const bool partly = first + kSlice > length || absent != 0;
            uint32_t seen[kRowTiles];
            if (partly) {
                if (P.flags && lane == 0 && (absent & low_bits(min(keys.end - first, kSlice)))) atomicOr(&P.flags[b], MDSD_FLAG_NO_PAGE);
#pragma unroll
                for (int r = 0; r < kRowTiles; ++r) {
                    seen[r] = ~absent & (uint32_t)(low_bits(length - first) |
                                                   nodes_seen<kSlice>(R, parent, length - first, node[r], ancestor[r]));
#pragma unroll
                    for (int t = 0; t < A::kTiles; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (!(seen[r] >> (t * 16 + quarter * 4) >> i & 1)) s[r][t][i] = -INFINITY;
                }
            }
            bool grew = false;
            float most[kRowTiles];
#pragma unroll
            for (int r = 0; r < kRowTiles; ++r) {
                most[r] = s[r][0][0];
#pragma unroll
                for (int t = 0; t < A::kTiles; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) most[r] = fmaxf(most[r], s[r][t][i]);
                most[r] = fmaxf(max_of_quarters(most[r]), top[r]);
                grew |= most[r] - top[r] > P.slack;  // (two infinities: no key yet)
            }
            if (__any(grew)) {
                far = false;
#pragma unroll
                for (int r = 0; r < kRowTiles; ++r) {
                    const float factor = rebased<T>(top[r], most[r], P.scale);
                    const Base base = base_of<T>(most[r], P.scale);
                    top[r] = most[r];
                    shift[r] = base.shift;
                    far |= base.origin != 0.f;
                    sum[r] *= factor;
#pragma unroll
                    for (int d = 0; d < A::kOuts; ++d) o[r][d] *= factor;
                }
                far = __any(far);
            }
            if (far) {
#pragma unroll
                for (int r = 0; r < kRowTiles; ++r) {
                    const float origin = base_of<T>(top[r], P.scale).origin;
#pragma unroll
                    for (int t = 0; t < A::kTiles; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) s[r][t][i] -= origin;
                }
            }
#pragma unroll
            for (int r = 0; r < kRowTiles; ++r)
#pragma unroll
                for (int t = 0; t < A::kTiles; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        s[r][t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r][t][i], P.scale, -shift[r]));
                        sum[r] += s[r][t][i];
                    }

            bool bad = false;
            if (partly) {
                // some rows do not see all of these keys: a weight of zero times an infinity or NaN is not zero, so these stay
                // out of the product and are added below for the rows that see them; keys without a page have zeros
#pragma unroll
                for (int i = 0; i < A::kStaged; ++i) {
                    if (absent >> ((lane + i * 64) / A::kChunks) & 1) v[i] = u32x4{0, 0, 0, 0};
                    bad |= has_nonfinite<T>(v[i]);
                    v[i] = finite_part<T>(v[i]);
                }
                bad = __any(bad);
            }
#pragma unroll
            for (int i = 0; i < A::kStaged; ++i) {
                const int key = (lane + i * 64) / A::kChunks, c = lane % A::kChunks;
                *(u32x4*)(v_lds + key * A::kRowBytes + A::v_chunk(key, c) * 16) = v[i];
            }
            if (tile > tile_from) load_v(place);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();

            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int t = 0; t < A::kTiles; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int key = t * 16 + quarter * 4 + i;
#pragma unroll
                        for (int d = 0; d < A::kOuts; ++d) {
                            const int x = d * 16 + col;
                            const float w = *(const float*)(v_lds + key * A::kRowBytes + A::v_chunk(key, x / 4) * 16 + x % 4 * 4);
#pragma unroll
                            for (int r = 0; r < kRowTiles; ++r)
                                o[r][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(w, s[r][t][i], o[r][d], 0, 0, 0);
                        }
                    }
            } else {
                // (16 keys: the matrix instruction for as many)
                using Operand = std::conditional_t<A::kTiles == 2, u32x4, u32x2>;
                Operand p[kRowTiles];
#pragma unroll
                for (int r = 0; r < kRowTiles; ++r)
#pragma unroll
                    for (int t = 0; t < A::kTiles; ++t) {
                        p[r][2 * t] = Element<T>::pack(s[r][t][0], s[r][t][1]);
                        p[r][2 * t + 1] = Element<T>::pack(s[r][t][2], s[r][t][3]);
                    }
#pragma unroll
                for (int d = 0; d < A::kOuts; ++d) {
                    Operand w;
#pragma unroll
                    for (int j = 0; j < A::kTiles; ++j) {
                        const int key = j * 16 + quarter * 4 + col / 4, c = d * 2 + (col & 3) / 2;
                        const char* at = v_lds + key * A::kRowBytes + A::v_chunk(key, c) * 16 + (col & 1) * 8;
                        const u32x2 four = __builtin_bit_cast(
                            u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)at));
                        w[2 * j] = four[0];
                        w[2 * j + 1] = four[1];
                    }
#pragma unroll
                    for (int r = 0; r < kRowTiles; ++r) o[r][d] = Element<T>::mfma(w, p[r], o[r][d]);
                }
            }
            if (bad) {
                for (int key = 0; key < kSlice; ++key) {
                    const int64_t offset = __shfl((long long)here, key);
                    if (offset < 0) continue;
#pragma unroll
                    for (int r = 0; r < kRowTiles; ++r)
#pragma unroll
                        for (int d = 0; d < A::kOuts; ++d) {
                            const int x = d * 16 + quarter * 4;
                            const T* const at = (const T*)(v_head + offset) + x;
                            if ((seen[r] >> key & 1) && x < C.dim)
#pragma unroll
                                for (int j = 0; j < 4; ++j)
                                    if (!__builtin_isfinite((float)at[j])) o[r][d][j] += (float)at[j];
                            __builtin_amdgcn_sched_barrier(0);  // a rare loop must not take registers from the others
                        }
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }

        // the waves meet
#pragma unroll
        for (int r = 0; r < kRowTiles; ++r) {
            sum[r] = sum_of_quarters(sum[r]);
            if (quarter == 0) stats[wave][r * 16 + col].x = top[r];
        }
        __syncthreads();
        float* const kept = (float*)lds;  // [wave][row][dim], a row's chunks of four turned by the row against bank conflicts
#pragma unroll
        for (int r = 0; r < kRowTiles; ++r) {
            const int row = r * 16 + col;
            const float most = fmaxf(fmaxf(stats[0][row].x, stats[1][row].x), fmaxf(stats[2][row].x, stats[3][row].x));
            const float factor = rebased<T>(top[r], most, P.scale);
            if (quarter == 0) stats[wave][row].y = sum[r] * factor;
#pragma unroll
            for (int d = 0; d < A::kOuts; ++d)
                *(f32x4*)(kept + (wave * A::kRows + row) * kDim + ((d * 4 + quarter) ^ col) * 4) = o[r][d] * factor;
        }
        __syncthreads();
        const bool whole = !kLine || (tile_from == 0 && tile_to == keys.tiles);
        constexpr int kFours = kDim / 4;
#pragma unroll
        for (int i = 0; i < A::kRows * kFours / kAttentionThreads; ++i) {
            const int at = threadIdx.x + i * kAttentionThreads, r = at / kFours, c = at % kFours, row = first_row + r;
            if (row >= rows || c * 4 >= C.dim) continue;
            float most = -INFINITY, total = 0.f;
            f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                most = fmaxf(most, stats[w][r].x);
                total += stats[w][r].y;
                x += *(const f32x4*)(kept + (w * A::kRows + r) * kDim + (c ^ (r & 15)) * 4);
            }
            if (whole) {
                const int n = P.by_group(row), head = kv_head * P.group + row - n * P.group;
                write_four<T>(P.out.p + b * P.out.ld_tree + n * P.out.ld_node + head * P.out.ld_head, c * 4,
                              x * (total == 0.f ? 0.f : 1.f / total));
            } else {
                const int64_t slot = (int64_t)(kv_head * units + unit + group) * A::kRows + r;
                *(f32x4*)(P.sums + slot * C.dim + c * 4) = x;
                if (c == 0) P.stats[slot] = float2{most, total};
            }
        }
        if constexpr (!kLine) return;
        note_part(P.ends, kv_head * units + unit, group, tile_from == 0, tile_to == keys.tiles);
        if (left == 0) return;
        __syncthreads();  // the next unit's values go where this one's sums are read
        at = 0;
        do {
            if (++unit == units) {
                unit = 0;
                if (++kv_head == C.heads) return;
            }
            keys = unit_of<A::kRows, A::kKeys>(P, unit);
        } while (keys.tiles == 0);
    }
}

}  // namespace mdsd
