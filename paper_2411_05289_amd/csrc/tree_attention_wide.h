// Attention for trees of many rows: a workgroup takes 128 rows, or 64 and two slices of keys.
//
// Each of the four waves owns 32 rows (of a slice).  Keys and values go from memory straight into LDS (global_load_lds, 16
// bytes a lane), into a ring of buffers: kBuffers - 1 tiles are on their way while one is worked on, with one barrier a
// tile.  A row's 16-byte chunks stand XORed by the key's low bits, so that the 32 keys that one load of K takes at one
// chunk, and the four keys that one transposing load of V takes, lie in different banks; as a lane's place in LDS is fixed,
// the lane asks for the chunk that belongs there.
//
// Measured, heads of 128: prompts of four sequences, 372 GFLOP in 417 us, 893 TFLOP/s (a large library product 1112), the matrix
// units, the vector units and LDS near half busy each, two waves a SIMD taking turns; 64 trees of 31 nodes behind 512 to 4096
// slots, 645 MB and 75 GFLOP in 141 us; 64 trees of 15 nodes behind a shared prefix of 16384 slots, 266 GFLOP in 370 us.
//
// Of the builds that share their keys out those of heads of 128 spill 36 to 84 bytes a lane (two trees of 15 nodes behind 131072
// slots, 189 us: 76), those of heads of 256 68 to 360: where sums go, written to scratch at the start and read back once a unit.
// A workgroup per unit and joint prefixes spill nothing.  In 4 bits, where codes wait in registers: shared out 132 and 180, of heads of 256 172
// and 496; joint prefixes of heads of 128 24; fp32 in heads of 256, whose queries in three parts are 192 registers, 320 and 412 by a workgroup
// per unit, 552 joint, 796 and 1112 shared out.
//
// A cache in 4 bits: the codes of the next tile wait in registers, and are written into LDS as numbers between two tiles, each thread a part of
// a key: prompts of up to 4096 + 1024 slots, 372 GFLOP of fp16 in 426 us, 874 TFLOP/s; 64 trees of 124 rows behind 512 to 4096 slots, 75
// GFLOP in 112 us; two trees of 15 nodes behind 131072 slots 112 us.
#pragma once
#include "four_bits.h"
#include "tree_attention.h"

namespace mdsd {

// kDim: the head's elements, filled up with zeros to 64, 128 or 256.  kRowWaves: of the four waves, how many stand side by
// side along the rows; the others stand along the keys and are joined in the end (trees with few rows).
template <class Out, int kDim, int kRowWaves, bool kFour>
struct WideTile {
    using T = Worked<Out, kFour>;
    static constexpr int kParts = kPartsOf<Out, kFour>;
    static constexpr int kRowBytes = kDim * sizeof(T);
    static constexpr int kChunks = kRowBytes / 16;
    static constexpr int kRows = 32 * kRowWaves, kKeyWaves = 4 / kRowWaves;
    static constexpr int kSets = kKeyWaves == 1 && kRowBytes <= 256 ? 2 : 1, kSlice = 32 * kSets;  // keys of a wave
    static constexpr int kKeys = kSlice * kKeyWaves;
    static constexpr int kBytes = kKeys * kRowBytes;  // of K or V
    static constexpr int kPerWave = kBytes / 4;       // of them, that a wave brings in
    static constexpr int kPerLane = kPerWave / 1024;
    static constexpr int kFit = 64 * 1024 / (2 * kBytes), kBuffers = kFit >= 4 && !kFour ? 4 : 2;
    // in 4 bits: of codes, that a thread brings in of K, and of V
    static constexpr int kCodes = kKeys * kDim / 2 / 256, kUnit = kCodes < 16 ? 8 : 16, kUnits = kCodes / kUnit;
    static constexpr int kQueryChunks = kRowBytes / 32;       // per lane: the half-waves have every other one
    static constexpr int kOuts = kDim / 32;
    static constexpr size_t kJoin = kKeyWaves == 1 ? 0 : (size_t)(kKeyWaves - 1) * kRows * (kDim + 2) * 4;
    static constexpr size_t kTiles = (size_t)2 * kBuffers * kBytes;
    static constexpr size_t kLds = kTiles > kJoin ? kTiles : kJoin;
    static constexpr int kPerUnit = kLds <= 80 * 1024 && kDim < 256 && kParts * kDim < 256 ? 2 : 1;  // workgroups that a compute unit holds
    static_assert(kLds <= 160 * 1024, "LDS");

    // where chunk c of a key stands in its row, and which chunk stands at c
    // In 4 bits a lane writes four chunks of a key one behind the other, and four lanes a key: heads of 128 have the upper half of a key's
    // chunks turned against the lower, and V's keys as no two of those that are written or read together meet (conflicts of eight
    // lanes by two before, 16 us of 123 in LDS for 64 trees of 124 rows).
    static constexpr bool kTurned = kFour && kChunks == 16;
    static __device__ int k_chunk(int key, int c) { return c ^ (kChunks == 8 ? (key >> 1) & 7 : key & 15) ^ (kTurned ? (c >> 3 & 1) << 1 : 0); }
    static __device__ int v_chunk(int key, int c)
    {
        if (kTurned) return c ^ (key & 1) * 6 ^ (key >> 1 & 1) * 10 ^ (c >> 3 & 1);
        if (sizeof(T) == 4) return c ^ ((key >> 2 & 1) << 3);
        return c ^ (kChunks == 8 ? (key >> 1 & 1) << 2 : (key & 3) << 2);
    }
    // what a key's place differs by, `c` pairs of chunks further in K, `d` times four in V: an exclusive or
    static __device__ constexpr int k_step(int c) { return c * 32 ^ (kTurned ? (c >> 2 & 1) * 32 : 0); }
    static __device__ constexpr int v_step(int d) { return d * 64 ^ (kTurned ? (d >> 1 & 1) * 16 : 0); }
};

static __device__ const u32x4 zeros = {0, 0, 0, 0};

// 16 bytes from each lane's address to LDS, `to` + 16 * lane; done when the wave's count of loads says so.  (Not by the
// compiler's function for it, after which every transposing load waits for all of the wave's loads.  The instruction
// has no output register, and M0 one cycle of settling.)
__device__ inline void to_lds(const char* from, uint32_t to, bool once)
{
    if (once)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" : : "s"(to), "v"(from) : "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(to), "v"(from) : "memory");
}
// waits until at most kMost of the wave's loads are on their way, and for all of its LDS reads
template <int kMost>
__device__ inline void wait_for_loads()
{
    static_assert(kMost < 64, "the counter's range");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070 | (kMost & 15) | (kMost >> 4) << 14);
    asm volatile("" ::: "memory");
}

// kLine: P.groups workgroups share the line of tiles; else one for every unit.  kJoint: units of all trees' rows and the shared prefix too.
// kSums: the rows' sums may be asked for.
template <class Out, int kDim, int kRowWaves, bool kLine, bool kJoint, bool kFour, bool kSums>
__global__ __launch_bounds__(kAttentionThreads, (WideTile<Out, kDim, kRowWaves, kFour>::kPerUnit)) void attention_wide_kernel(AttentionParams P)
{
    using A = WideTile<Out, kDim, kRowWaves, kFour>;
    using T = typename A::T;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    char* const v_lds = lds + A::kBuffers * A::kBytes;
    int* const parent = (int*)(lds + A::kLds);
    constexpr int kCachedKeys = 512, kCached = kCachedKeys / A::kKeys;
    __shared__ int64_t places[2][kCachedKeys];
    __shared__ uint64_t absences[2][kCached];
    // keys and values that no other workgroup reads need not stay in the caches (a stream of 1 GB 6.1 -> 7.0 TB/s)
    const bool once = kLine && !kJoint && P.row_tiles == 1;
    __shared__ int bad_tile;  // that infinities and NaNs were left out of
    __shared__ int least_limit;

    const Cache& C = P.cache;
    const Trees& R = P.trees;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, col = lane & 31;
    const int row_wave = wave % kRowWaves, slice = wave / kRowWaves;
    const int own_units = R.B * P.row_tiles, units = own_units + (kJoint ? P.joint_tiles : 0);  // of a cache head
    const int capacity = C.table_pages * C.page_size;

    int kv_head, unit, at = 0, group = 0;
    int64_t left = INT64_MAX;  // tiles of the share
    Unit keys;
    if constexpr (!kLine) {
        // neighbouring workgroups have different cache heads: with 8 of them (or a multiple) all tiles of a head meet in
        // one XCD's L2.  The last row tiles of a tree see the most keys and come first.
        const int rest = unit_of_group<kFour>(P, blockIdx.x, own_units, &kv_head);
        int b = P.by_tiles(rest);
        unit = b * P.row_tiles + P.row_tiles - 1 - (rest - b * P.row_tiles);
        if (P.first_round) unit = b = tree_by_length(P, b);
        keys = unit_of<A::kRows, A::kKeys>(P, unit);
        if (keys.tiles == 0) {
            if (P.flags && threadIdx.x == 0 && keys.row_tile == 0 && keys.length < 0) atomicOr(&P.flags[b], MDSD_FLAG_NO_PAGE);
            return;
        }
    } else {
        // workgroups go round the XCDs: each XCD has a stretch of the line, which goes head by head
        group = blockIdx.x % 8 * (P.groups / 8) + blockIdx.x / 8;
        const Share s = share_of<A::kRows, A::kKeys, kJoint, kFour>(P, own_units, group);
        if (s.tiles == 0) return;
        left = s.tiles;
        kv_head = s.kv_head;
        unit = s.unit;
        at = s.at;
        keys = s.first;
    }
    if (!R.complete) parents_from_table(R, parent);

    for (;;) {
        const bool joint = kJoint && keys.tree < 0;
        const int tree = joint ? 0 : keys.tree, row_tile = keys.row_tile;
        // tiles tile_to-1 down to tile_from of the unit
        int tile_from = 0, tile_to = keys.tiles;
        if constexpr (kLine) {
            const int end = (int)min((int64_t)keys.tiles + P.unit_cost, at + left);
            left -= end - at;
            tile_from = max(0, at - P.unit_cost);
            tile_to = end - P.unit_cost;
            if (tile_to <= tile_from) return;  // the share ends before the unit's tiles begin
        }

        // the lane's row
        int b = tree, node, head, length;
        bool valid;
        {
            const int own_row = row_tile * A::kRows + row_wave * 32 + col;
            int row;
            if (joint) {
                valid = own_row < R.B * R.N * P.group;
                row = valid ? own_row : 0;
                b = P.by_rows(row);
                row -= b * R.N * P.group;
            } else {
                const int rows = keys.count * P.group;
                valid = own_row < rows;
                row = min(own_row, rows - 1);
            }
            node = P.by_group(row);
            head = kv_head * P.group + row - node * P.group;
            length = joint ? C.lengths[b] : keys.length;
            if (joint) valid = valid && node < R.count(b) && length >= 0;
            if (P.flags && !joint && threadIdx.x == 0 && tile_to == keys.tiles &&
                (int64_t)length + P.by_group(min((row_tile + 1) * A::kRows, keys.count * P.group) - 1) >= capacity)
                atomicOr(&P.flags[b], MDSD_FLAG_NO_PAGE);
            length = max(0, min(length, capacity));
        }
        // the slots that the row sees of the sequence itself
        const int limit = joint ? (valid ? min(P.shared, length) : P.shared) : length;
        const int shared = joint ? P.shared : min(P.shared, length);
        const int32_t* const table = C.table + tree * C.ld_table;
        int all_see = limit, wave_sees = limit;  // slots that every row of the workgroup sees, and of the wave
        bool idle = false;
        if (joint) {
            if (threadIdx.x == 0) least_limit = INT32_MAX;
            __syncthreads();
            atomicMin(&least_limit, limit);
            __syncthreads();
            all_see = wave_sees = least_limit;
        } else {
            const int first_row = row_tile * A::kRows;
            if (R.complete && R.k == 1) {
                all_see += P.by_group(first_row) + 1;
                wave_sees += P.by_group(first_row + row_wave * 32) + 1;
            }
            idle = first_row + row_wave * 32 >= keys.count * P.group;
        }

        u32x4 q[A::kQueryChunks][A::kParts];
        const char* const q_row = P.q.p + b * P.q.ld_tree + node * P.q.ld_node + head * P.q.ld_head;
#pragma unroll
        for (int c = 0; c < A::kQueryChunks; ++c) {
            const int chunk = 2 * c + half;
#pragma unroll
            for (int p = 0; p < A::kParts; ++p) q[c][p] = u32x4{0, 0, 0, 0};
            if (valid && chunk * 16 < C.dim * (int)sizeof(T)) {
                if constexpr (A::kParts == 3)
                    in_parts((const float*)(q_row + chunk * 32), q[c]);
                else
                    q[c][0] = *(const u32x4*)(q_row + chunk * 16);
            }
        }
        f32x16 o[A::kOuts];
#pragma unroll
        for (int d = 0; d < A::kOuts; ++d) o[d] = f32x16{};
        float top = -INFINITY, shift = 0.f, sum = 0.f;  // score and shift that the weights go by; their sum
        bool far = false;                               // a row of the wave has an origin
        int ancestor = node;                            // next of the row's nodes that no tile had yet

        const char* const k_head = C.k + kv_head * C.ld_head;
        const char* const v_head = C.v + kv_head * C.ld_head;
        const uint8_t* const k_scales = kFour ? P.scales.k + kv_head * (C.ld_head / 16) : nullptr;
        const uint8_t* const v_scales = kFour ? P.scales.v + kv_head * (C.ld_head / 16) : nullptr;

        // The places of kCached tiles' keys, in LDS, and those of the next ones: beside the loads of keys and values a load of a
        // page would have to wait for all of them, as loads come back in order.  The pages are asked for a part ahead.  Keys
        // without a page and behind the last slot: -1, and a bit.
        int pages[kCachedKeys / kAttentionThreads];  // of the part `ahead`
        int ahead = 0;
        auto ask_for_pages = [&]() {
#pragma unroll
            for (int j = 0; j < kCachedKeys / kAttentionThreads; ++j) {
                const int i = threadIdx.x + j * kAttentionThreads;
                const int tile = tile_to - 1 - ahead * kCached - i / A::kKeys, s = keys.lo + tile * A::kKeys + i % A::kKeys;
                pages[j] = -1;
                if (tile >= tile_from && s < keys.end) {
                    const int entry = C.by_page(s);
                    pages[j] = s < shared ? P.shared_pages[entry] : table[entry];
                }
            }
        };
        auto look_up = [&]() {
#pragma unroll
            for (int j = 0; j < kCachedKeys / kAttentionThreads; ++j) {
                const int i = threadIdx.x + j * kAttentionThreads;
                const int tile = tile_to - 1 - ahead * kCached - i / A::kKeys, s = keys.lo + tile * A::kKeys + i % A::kKeys;
                const int64_t place = pages[j] < 0 ? -1 : place_in_page(C, pages[j], s, C.by_page(s));
                places[ahead & 1][i] = place;
                const uint64_t none = __ballot(place < 0);
                if (A::kKeys == 64) {
                    if (lane == 0) absences[ahead & 1][i / 64] = none;
                } else if (lane % 32 == 0) {
                    absences[ahead & 1][i / 32] = (uint32_t)(none >> lane);
                }
            }
            ++ahead;
            ask_for_pages();
        };
        const int dim_bytes = C.dim * (int)sizeof(T);
        // the places that the wave's part of a tile is read from, and the tile's absences
        struct Next {
            int64_t from[A::kPerLane];
            uint64_t absent;
        };
        auto next_of = [&](int tile) {
            Next n;
            const int turn = tile_to - 1 - tile, at = turn & (kCached - 1);
            const int part = turn / kCached & 1;
#pragma unroll
            for (int i = 0; i < A::kPerLane; ++i)
                n.from[i] = places[part][at * A::kKeys + (wave * A::kPerWave + i * 1024 + lane * 16) / A::kRowBytes];
            n.absent = absences[part][at];
            return n;
        };
        // asks for the wave's part of a tile
        const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds + wave * A::kPerWave;
        auto load = [&](const Next& n, int buffer) {
            const bool plain = n.absent == 0 && C.dim == kDim;
            int place = lane * 16;
            if constexpr (kLine) asm volatile("" : "+v"(place));  // (formed here: kept for every load it would take registers from the products)
#pragma unroll
            for (int i = 0; i < A::kPerLane; ++i) {
                const int key = (wave * A::kPerWave + i * 1024 + place) / A::kRowBytes, c = place / 16 % A::kChunks;
                const int k_column = A::k_chunk(key, c) * 16, v_column = A::v_chunk(key, c) * 16;
                const char *k = k_head + n.from[i] + k_column, *v = v_head + n.from[i] + v_column;
                if (!plain) {  // keys without a page and elements behind the last are zeros
                    if (n.from[i] < 0 || k_column >= dim_bytes) k = (const char*)&zeros;
                    if (n.from[i] < 0 || v_column >= dim_bytes) v = (const char*)&zeros;
                }
                to_lds(k, lds_at + buffer * A::kBytes + i * 1024, once);
                to_lds(v, lds_at + (A::kBuffers + buffer) * A::kBytes + i * 1024, once);
            }
        };
        // In 4 bits: a tile's codes come into registers while the tile before it is worked on, and go into LDS as T.  Keys without a
        // page and elements behind the last are zeros.
        Codes<A::kUnit, false> k_codes[A::kUnits], v_codes[A::kUnits];
        constexpr int kOfKey = kDim / 2 / A::kUnit, kWide = A::kUnit * 2 * sizeof(T) / 16;  // units of a key; chunks of a unit
        auto ask_for_codes = [&](int tile) {
            const int turn = tile_to - 1 - tile, at = turn & (kCached - 1), part = turn / kCached & 1;
#pragma unroll
            for (int i = 0; i < A::kUnits; ++i) {
                const int u = threadIdx.x + i * kAttentionThreads, c = u % kOfKey * A::kUnit;
                const int64_t from = places[part][at * A::kKeys + u / kOfKey], there = max(from, (int64_t)0);
                const int column = C.dim == kDim ? c : min(c, C.dim / 2 - A::kUnit);
                k_codes[i].load(k_head + there, k_scales + (there >> 4), column);
                v_codes[i].load(v_head + there, v_scales + (there >> 4), column);
                if (from < 0 || column != c) k_codes[i].clear(true), v_codes[i].clear(true);
            }
            return absences[part][at];
        };
        auto put_codes = [&](int buffer) {
#pragma unroll
            for (int i = 0; i < A::kUnits; ++i)
#pragma unroll
                for (int j = 0; j < kWide; ++j) {
                    const int u = threadIdx.x + i * kAttentionThreads, key = u / kOfKey, c = u % kOfKey * kWide + j;
                    char* const to = lds + buffer * A::kBytes + key * A::kRowBytes;
                    *(u32x4*)(to + A::k_chunk(key, c) * 16) = k_codes[i].template chunk<T>(j);
                    *(u32x4*)(to + A::kBuffers * A::kBytes + A::v_chunk(key, c) * 16) = v_codes[i].template chunk<T>(j);
                }
        };
        // leaves infinities and NaNs out of the wave's part of V: where some rows do not see all of a tile's keys, a weight of
        // zero times one of them is not zero; they are added below for the rows that see them
        auto clean = [&](int tile, int buffer) {
            bool bad = false;
#pragma unroll
            for (int i = 0; i < A::kPerLane; ++i) {
                u32x4* const at = (u32x4*)(v_lds + buffer * A::kBytes + wave * A::kPerWave + i * 1024 + lane * 16);
                const u32x4 v = *at;
                if (has_nonfinite<T>(v)) {
                    bad = true;
                    *at = finite_part<T>(v);
                }
            }
            if (bad) bad_tile = tile;
        };

        const uint32_t k_lane = col * A::kRowBytes + A::k_chunk(col, half) * 16;
        const int v_key = 4 * half + (lane & 15) / 4;  // (transposing: each lane's address is of a key and four elements)
        const uint32_t v_lane = v_key * A::kRowBytes + A::v_chunk(v_key, (lane >> 4 & 1) * 2 + (lane & 3) / 2) * 16 + (lane & 1) * 8;
        constexpr int kAhead = A::kBuffers - 1;
        uint64_t absences_ahead[kAhead];  // of the tiles on their way, the next one first
        if (threadIdx.x == 0) bad_tile = -1;
        ask_for_pages();
        look_up();
        __syncthreads();
        Next next;
        uint64_t absences_behind = 0;  // of the codes that are on their way
        if constexpr (kFour) {
            absences_ahead[0] = ask_for_codes(tile_to - 1);
            put_codes(0);
            if (tile_to - 2 >= tile_from) absences_behind = ask_for_codes(tile_to - 2);
        } else {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const Next n = next_of(tile_to - 1 - i);
                absences_ahead[i] = n.absent;
                if (tile_to - 1 - i >= tile_from) load(n, i);
            }
            next = next_of(tile_to - 1 - kAhead);
        }

        for (int tile = tile_to - 1, buffer = 0; tile >= tile_from; --tile, buffer = (buffer + 1) & (A::kBuffers - 1)) {
            // this tile's loads are the oldest; behind them are kBuffers - 2 tiles'
            const int behind = tile - kAhead - 1;  // the tile whose places are needed next
            if (behind >= tile_from && ((tile_to - 1 - behind) & (kCached - 1)) == 0) {
                if constexpr (!kFour) wait_for_loads<0>();
                look_up();
            }
            const uint64_t absent_here = absences_ahead[0];
            if constexpr (kFour) {
                wait_for_loads<63>();  // (LDS alone: this tile is whole, and nobody reads the one before)
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                absences_ahead[0] = absences_behind;
                if (tile - 1 >= tile_from) put_codes(buffer ^ 1);
                if (behind >= tile_from) absences_behind = ask_for_codes(behind);
            } else {
                if (tile - tile_from >= kAhead - 1)
                    wait_for_loads<(kAhead - 1) * 2 * A::kPerLane>();
                else
                    wait_for_loads<0>();
                __builtin_amdgcn_s_barrier();
#pragma unroll
                for (int i = 0; i < kAhead - 1; ++i) absences_ahead[i] = absences_ahead[i + 1];
                if (tile - kAhead >= tile_from) {
                    absences_ahead[kAhead - 1] = next.absent;
                    load(next, (buffer + kAhead) & (A::kBuffers - 1));
                    next = next_of(behind);
                }
            }
            const bool partly = keys.lo + (tile + 1) * A::kKeys > all_see;
            if (partly) {
                clean(tile, buffer);
                __syncthreads();
            }
            // the lane's places in K and V; others differ from them by exclusive ors and steps known beforehand
            const uint32_t tile_at = buffer * A::kBytes + slice * A::kSlice * A::kRowBytes;
            const uint32_t k_at = tile_at + k_lane, v_at = A::kBuffers * A::kBytes + tile_at + v_lane;
            const char* const vb = v_lds + tile_at;
            if (!idle) {
                f32x16 s[A::kSets];
#pragma unroll
                for (int t = 0; t < A::kSets; ++t) s[t] = f32x16{};
                // some chunks of every set of 32 keys at a time, the sets' products in turn
                constexpr int kTogether = A::kQueryChunks * A::kSets < 8 ? A::kQueryChunks : 8 / A::kSets;
#pragma unroll
                for (int from = 0; from < A::kQueryChunks; from += kTogether) {
                    u32x4 k[A::kSets][kTogether];
#pragma unroll
                    for (int c = 0; c < kTogether; ++c)
#pragma unroll
                        for (int t = 0; t < A::kSets; ++t)  // chunk 2 * (from + c) + half of key t * 32 + col
                            k[t][c] = *(const u32x4*)(lds + ((k_at ^ A::k_step(from + c)) + t * 32 * A::kRowBytes));
                    __builtin_amdgcn_sched_barrier(0);  // (all reads first: left to itself the compiler waits for each)
#pragma unroll
                    for (int c = 0; c < kTogether; ++c)
#pragma unroll
                        for (int t = 0; t < A::kSets; ++t) {
                            if constexpr (sizeof(T) == 4) {
#pragma unroll
                                for (int j = 0; j < 4; ++j)
                                    s[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k[t][c][j]), __uint_as_float(q[from + c][0][j]), s[t], 0, 0, 0);
                            } else {
#pragma unroll
                                for (int p = 0; p < A::kParts; ++p) s[t] = Element<T>::mfma(k[t][c], q[from + c][p], s[t]);
                            }
                        }
                }
                // V, sixteen keys at a time; the first of them are on their way while the weights are formed
                constexpr int kEarly = sizeof(T) == 4 ? 0 : A::kOuts >= 8 ? 1 : 2;
                u32x4 v[kEarly ? kEarly : 1][A::kOuts];
                auto read_values = [&](int kk, u32x4(&into)[A::kOuts]) {
#pragma unroll
                    for (int d = 0; d < A::kOuts; ++d)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {  // elements d * 32 .. of keys 16 * kk + 8 * j + 4 * half ..
                            const char* at = lds + ((v_at ^ A::v_step(d)) + (16 * kk + 8 * j) * A::kRowBytes);
                            const u32x2 four = __builtin_bit_cast(
                                u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)at));
                            into[d][2 * j] = four[0];
                            into[d][2 * j + 1] = four[1];
                        }
                };
#pragma unroll
                for (int kk = 0; kk < kEarly; ++kk) read_values(kk, v[kk]);
                __builtin_amdgcn_sched_barrier(0);

                // which of the wave's keys the row sees, a bit for each
                const int first = keys.lo + tile * A::kKeys + slice * A::kSlice;
                // keys without a page, and slots behind the last
                const uint64_t absent = absent_here >> (slice * A::kSlice) & low_bits(A::kSlice);
                uint64_t seen = ~absent;
                const bool masked = first + A::kSlice > wave_sees || absent != 0;
                if (masked) {
                    uint64_t own = low_bits(limit - first);
                    if (!joint) own |= nodes_seen<A::kSlice>(R, parent, length - first, node, ancestor);
                    seen &= own;
                    if (P.flags) {
                        const uint64_t wanted = low_bits(min(keys.end - first, A::kSlice));
                        if (joint ? valid && (absent & wanted & own) != 0 : (absent & wanted) != 0 && lane == 0)
                            atomicOr(&P.flags[b], MDSD_FLAG_NO_PAGE);
                    }
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
                if (__any(most - top > P.slack)) {  // (two infinities: no key yet)
                    const float factor = rebased<T>(top, most, P.scale);
                    const Base base = base_of<T>(most, P.scale);
                    top = most;
                    shift = base.shift;
                    far = __any(base.origin != 0.f);
                    sum *= factor;
#pragma unroll
                    for (int d = 0; d < A::kOuts; ++d) o[d] *= factor;
                }
                if (far) {
                    const float origin = base_of<T>(top, P.scale).origin;
#pragma unroll
                    for (int t = 0; t < A::kSets; ++t)
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[t][i] -= origin;
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
                                const float w = *(const float*)(vb + key * A::kRowBytes + A::v_chunk(key, x / 4) * 16 + x % 4 * 4);
                                o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(w, s[t][i], o[d], 0, 0, 0);
                            }
                        }
                } else {
#pragma unroll
                    for (int kk = 0; kk < A::kSlice / 16; ++kk) {
                        f32x16& w = s[kk / 2];
                        const int r = 8 * (kk & 1);
                        u32x4 p[A::kParts];
#pragma unroll
                        for (int x = 0; x < A::kParts; ++x)
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                if constexpr (A::kParts == 3) {
                                    float low = w[r + 2 * j], high = w[r + 2 * j + 1];
                                    p[x][j] = next_parts(low, high);
                                    w[r + 2 * j] = low;
                                    w[r + 2 * j + 1] = high;
                                } else {
                                    p[x][j] = Element<T>::pack(w[r + 2 * j], w[r + 2 * j + 1]);
                                }
                            }
                        u32x4(&values)[A::kOuts] = v[kEarly ? kk % kEarly : 0];
                        if (kk >= kEarly && kEarly == 0) read_values(kk, values);
#pragma unroll
                        for (int d = 0; d < A::kOuts; ++d)
#pragma unroll
                            for (int x = 0; x < A::kParts; ++x) o[d] = Element<T>::mfma(values[d], p[x], o[d]);
                        if (kEarly && kk + kEarly < A::kSlice / 16) {
                            read_values(kk + kEarly, values);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
                }
                if (partly && bad_tile == tile) {
                    for (int key = 0; key < A::kSlice; ++key) {
                        if (absent >> key & 1) continue;
                        const int slot = first + key;
                        const int64_t offset = place_of(C, slot < shared ? P.shared_pages : table, slot);
                        const bool sees = seen >> key & 1;
#pragma unroll
                        for (int d = 0; d < A::kOuts; ++d)
#pragma unroll
                            for (int i = 0; i < 16; i += 4) {
                                const int x = d * 32 + 2 * i + 4 * half;
                                if constexpr (kFour) {
                                    if (sees && x < C.dim && v_scales[(offset >> 4) + x / kBlock] == kNoNumber)
                                        o[d][i] = o[d][i + 1] = o[d][i + 2] = o[d][i + 3] = NAN;
                                    continue;
                                }
                                const T* const v = (const T*)(v_head + offset) + x;
                                if (sees && x < C.dim)
#pragma unroll
                                    for (int j = 0; j < 4; ++j)
                                        if (!__builtin_isfinite((float)v[j])) o[d][i + j] += (float)v[j];
                                __builtin_amdgcn_sched_barrier(0);  // a rare loop must not take registers from the others
                            }
                    }
                }
            }
        }

        sum = sum_of_halves(sum);
        if constexpr (A::kKeyWaves > 1) {
            // the waves along the keys meet in the first of them
            float* const kept = (float*)lds;  // [wave][row][dim], then [wave][row][top, sum]
            float2* const stat = (float2*)(kept + (A::kKeyWaves - 1) * A::kRows * kDim);
            const int row = row_wave * 32 + col;
            __syncthreads();
            if (slice > 0) {
                float* const to = kept + ((slice - 1) * A::kRows + row) * kDim;
#pragma unroll
                for (int d = 0; d < A::kOuts; ++d)
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const int x = d * 32 + 2 * i + 4 * half;
                        // (rows are 256 bytes and more apart: the chunk is turned by the row against bank conflicts)
                        *(f32x4*)(to + ((x / 4 ^ (row & 7)) * 4)) = f32x4{o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]};
                    }
                if (half == 0) stat[(slice - 1) * A::kRows + row] = float2{top, sum};
            }
            __syncthreads();
            if (slice == 0) {
                float most = top;
#pragma unroll
                for (int w = 0; w < A::kKeyWaves - 1; ++w) most = fmaxf(most, stat[w * A::kRows + row].x);
                const float own = rebased<T>(top, most, P.scale);
                sum *= own;
#pragma unroll
                for (int d = 0; d < A::kOuts; ++d) o[d] *= own;
#pragma unroll
                for (int w = 0; w < A::kKeyWaves - 1; ++w) {
                    const float2 of = stat[w * A::kRows + row];
                    const float factor = rebased<T>(of.x, most, P.scale);
                    const float* const at = kept + (w * A::kRows + row) * kDim;
                    sum += of.y * factor;
#pragma unroll
                    for (int d = 0; d < A::kOuts; ++d)
#pragma unroll
                        for (int i = 0; i < 16; i += 4) {
                            const int x = d * 32 + 2 * i + 4 * half;
                            const f32x4 v = *(const f32x4*)(at + ((x / 4 ^ (row & 7)) * 4));
#pragma unroll
                            for (int j = 0; j < 4; ++j) o[d][i + j] += v[j] * factor;
                        }
                }
                top = most;
            }
            __syncthreads();
        }

        const bool whole = !kLine || (!kJoint && tile_from == 0 && tile_to == keys.tiles);
        if (slice == 0) {
            if (whole) {
                const float over = sum == 0.f ? 0.f : 1.f / sum;
                if (kSums && P.lse && valid && half == 0) P.lse[((int64_t)b * R.N + node) * (C.heads * P.group) + head] = log_of_sum<T>(top, sum, P.scale);
                if (valid) {
                    char* const out = P.out.p + b * P.out.ld_tree + node * P.out.ld_node + head * P.out.ld_head;
#pragma unroll
                    for (int d = 0; d < A::kOuts; ++d)
#pragma unroll
                        for (int i = 0; i < 16; i += 4) {
                            const int x = d * 32 + 2 * i + 4 * half;
                            if (x >= C.dim) continue;
                            write_four<Out>(out, x, f32x4{o[d][i] * over, o[d][i + 1] * over, o[d][i + 2] * over, o[d][i + 3] * over});
                        }
                }
            } else if (valid) {
                const int index = joint ? kv_head * P.joint_tiles + unit : place_in_line<kFour>(P, kv_head, unit - (kJoint ? P.joint_tiles : 0), own_units);
                const int64_t at = (int64_t)(index + group) * (joint ? kJointRows : P.part_rows) + row_wave * 32 + col;
                float* const to = (joint ? P.joint_sums : P.sums) + at * C.dim;
#pragma unroll
                for (int d = 0; d < A::kOuts; ++d)
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const int x = d * 32 + 2 * i + 4 * half;
                        if (x < C.dim) *(f32x4*)(to + x) = f32x4{o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]};
                    }
                if (half == 0) (joint ? P.joint_stats : P.stats)[at] = float2{top, sum};
            }
        }
        if constexpr (!kLine) return;
        note_part(joint ? P.joint_ends : P.ends, joint ? kv_head * P.joint_tiles + unit : place_in_line<kFour>(P, kv_head, unit - (kJoint ? P.joint_tiles : 0), own_units),
                  group, tile_from == 0, tile_to == keys.tiles);
        if (left == 0) return;
        __syncthreads();  // the next unit's keys go where this one's are read
        at = 0;
        if (kFour && !kJoint && P.by_unit) {
            if (++kv_head < C.heads) continue;
            kv_head = 0;
        }
        do {
            if (++unit == units) {
                unit = 0;
                if ((kFour && !kJoint && P.by_unit) || ++kv_head == C.heads) return;
            }
            if (kJoint && unit < P.joint_tiles)
                keys = joint_unit<A::kKeys>(P, unit);
            else
                keys = unit_of<A::kRows, A::kKeys>(P, unit - (kJoint ? P.joint_tiles : 0));
        } while (keys.tiles == 0);
    }
}

}  // namespace mdsd
