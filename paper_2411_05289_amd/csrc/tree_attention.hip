// Attention of tree nodes: checks, and how a call is cut into launches.
#include "tree_attention_plan.h"

#include <cfloat>

namespace mdsd {

constexpr int kComputeUnits = 256;

static int padded_dim(int dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }

static bool plan_attention(const mdsd_kv_cache* c, const mdsd_tree* t, int q_heads, int shared, int longest, bool workspace,
                           AttentionPlan* plan)
{
    AttentionPlan& p = *plan;
    p = AttentionPlan{};
    const int G = q_heads / c->heads, size = c->dtype == MDSD_FP32 ? 4 : 2, dim = padded_dim(c->dim), row_bytes = dim * size;
    p.rows = (int64_t)t->N * G;
    if (p.rows > INT32_MAX - kJointRows) return false;
    const int64_t capacity = (int64_t)c->table_pages * c->page_size;
    const int64_t most = (longest ? (longest < capacity ? longest : capacity) : capacity) + t->N;
    // The prefix once for all rows, where that saves more than it costs the trees' own parts to be worked on beside it by 128
    // rows a workgroup.  Full tiles have less to save, and none where their units fill the chip.  8 heads of 128 in bf16, prefix + own
    // slots, us apart and together:
    //    4 rows    8 trees 1024 + 64 15.9, 17.7, 4096 + 64 22.7, 20.9;  64 trees 1024 + 64 27.8, 24.4, 4096 + 64 88.6, 31.2
    //   16 rows   64 trees 1024 + 64 28.5, 30.8, 2048 + 64 48.3, 38.1
    //   32 rows   64 trees 1024 + 64 31.7, 45.0, 2048 + 64 71.9, 56.3
    //   48 rows  128 trees 2048 + 64 111, 116, 4096 + 64 197, 168
    //   60 rows   64 trees 2048 + 64 67, 84, 4096 + 64 108, 115, 4096 + 512 156, 121;  128 trees 2048 + 256 119, 143, 4096 + 512 211, 219,
    //            6144 + 64 285, 274;  200 trees 4096 + 64 337, 307
    //   64 rows  128 trees 4096 + 64 197, 214, 8192 + 64 372, 364
    //  124 rows   64 trees 4096 + 64 157, 199, 6144 + 64 281, 275, 8192 + 2048 441, 403;  128 trees 6144 + 64 441, 543, 8192 + 64 576, 692
    // What the rule still loses: 8 trees of 16 to 32 rows up to a fifth below 6144, 64 and more trees of 60 rows of heads of 256 up to a
    // tenth below 8192.
    const int64_t own = most - shared;
    const bool worth = p.rows <= 32   ? shared >= (p.rows <= 16 ? 1024 : 2048) && 2 * (int64_t)shared >= own
                       : p.rows <= 64 ? shared >= 4096 && shared >= 3 * own
                                      : shared >= 6144 && shared >= 3 * own && (int64_t)t->B * c->heads <= 2 * kComputeUnits;
    const bool joint = workspace && worth && t->B > 4 && p.rows <= kJointRows && (int64_t)t->B * p.rows <= INT32_MAX - kJointRows;
    // 16 rows a workgroup, where little is there to do: all of these fit on the chip at once and end early (124 rows of one
    // sequence, us with 128 a workgroup, with 16: 500 slots 20.1, 10.9, 2000 24.7, 23.6; of four sequences 500 slots 20.7, 12.2,
    // 1000 28.9, 34.4), and where 32 rows of 512 bytes would share a compute unit with nobody for little (100 sequences of 28 fp32
    // rows behind 10 slots 43, 26, behind 300 106, 97).  17 to 32 rows of heads beyond 128 take two times as many registers as
    // there are: fp32 16 each (27 rows behind 4096 slots, 32 sequences: 1647, 795), else 64 (320, 196).
    const int64_t sixteen = (p.rows + 15) / 16 * t->B * c->heads;
    const bool little = (sixteen <= kComputeUnits * (row_bytes <= 512 ? 2 : 1) && (most <= 768 || sixteen * most <= 131072)) ||
                        (p.rows <= 32 && row_bytes >= 512 && most <= 320);
    p.tile_rows = joint ? kJointRows
                  : p.rows <= 16 || little ? 16
                  : p.rows <= 32 && dim <= 128 ? 32
                  : p.rows <= 32 && size == 4 ? 16
                  : p.rows <= 64 && row_bytes <= 512 ? 64 : 128;
    // workgroups on the chip at once
    const int slots = kComputeUnits * (row_bytes <= (p.tile_rows == 16 ? 512 : 256) && !(p.tile_rows == 32 && dim > 64) ? 2 : 1);
    p.slice = p.tile_rows == 16 && row_bytes >= 512 ? 16 : 32;
    p.row_tiles = (int)((p.rows + p.tile_rows - 1) / p.tile_rows);
    p.units = (int64_t)t->B * p.row_tiles * c->heads;
    if (p.units > kMostGroups) return false;
    // The longest first (us without and with: 64 trees of 31 nodes behind 512 to 4096 slots 166, 149, all behind 2000 118, 120,
    // behind 10 to 20 16.4, 18.0; 256 tokens behind 512 to 8192 796, 708, 300 tokens behind 300 67, 74).
    if (p.row_tiles == 1 && p.units > kComputeUnits && t->B > 1 && t->B <= kMostOrdered &&
        most >= (p.units > 4 * kComputeUnits ? 1024 : 256))
        p.first_round = p.units <= 2 * kComputeUnits && slots > kComputeUnits ? (kComputeUnits + c->heads - 1) / c->heads : t->B;
    if (!workspace) return true;
    const int joint_tiles = joint ? (int)((t->B * p.rows + kJointRows - 1) / kJointRows) : 0;
    // (a cache head's tiles are counted in 32 bits, and the line's in the 52 of share_of's divisions)
    const int64_t line = (p.units / c->heads + joint_tiles) * (capacity / 32 + 16);
    if (line > INT32_MAX || line * c->heads > int64_t(1) << 42) {
        if (!joint) return true;
        return plan_attention(c, t, q_heads, 0, longest, workspace, plan);
    }
    // A workgroup per unit and one launch, where the longest unit ends before a second launch would have paid for itself, or
    // where there are units enough to fill the chip (us, a workgroup per unit and shared out; U units, all of one length):
    //   few rows   U = 8: 512 slots 10.2, 13.7, 1024 15.2, 14.1; U = 128: 512 14.9, 18.2, 1024 26.3, 25.8
    //   124 rows   U = 8: 512 19.7, 20.4, 1024 30.4, 21.5; U = 128: 1024 33, 43, 2048 56, 56
    //   prompts    of 4096 tokens, U = 1024 239, 292; 1024 tokens behind 8192 slots, U = 256, 203, 200
    // (a slot of longer rows and of fp32 costs the more).  Where units of one tile of rows fill the chip, longest first, it is a bet on
    // the lengths, of which only the longest is known here: a workgroup per unit wins where they are equal or spread evenly, and
    // loses where one sequence is long and the others are a sixteenth of it, the more the longer it is.  124 rows, equal; spread; one:
    //   bf16       U = 512 4096 slots 229, 232; 138, 162; 103, 54; 8192 418, 428; 265, 271; 191, 72; 16000 780, 812; 495, 489; 373, 107
    //              U = 1024 4096 417, 451; 250, 299; 108, 83; 8192 813, 844; 481, 528; 215, 118; heads of 256, U = 512 4096 527, 585; 309, 373; 240, 105
    //   fp32       U = 512 4096 1080, 1247; 834, 742; 588, 161; U = 800 2161, 1959; 1084, 1144; 593, 226
    // So it is taken up to the lengths where shared-out spread ones catch up, and in fp32 from three units a place on.  (Few rows are
    // memory's: 64 tokens of 512 to 8192 slots 194, 187.)
    int64_t enough = (768 + 2 * p.units) / (row_bytes > 256 ? row_bytes / 256 : 1);
    if (p.tile_rows > 32) {
        enough = 512 + 8 * p.units;
        if (p.row_tiles == 1 && p.units > slots && !p.first_round) enough = 2176;
        if (row_bytes > 256) enough = enough * 512 / (row_bytes * size);
        if (p.first_round && p.units >= (size == 2 ? slots : 3 * slots) && enough < 4608 * p.units / slots) enough = 4608 * p.units / slots;
    }
    if (!joint && (p.units >= 4 * slots || most <= enough)) return true;
    p.groups = slots;
    // One workgroup a compute unit where less than 64 MB are read, as fewer parts are joined (us with two, with one: one sequence,
    // 16 rows, 4000 slots 16.4, 15.2, 30000 slots 33.2, 32.4; 16 sequences of 30000 313, 333), and below 32 MB 16 rows by tiles
    // of 64 keys, not 128 (one token, 4000 slots 13.7, 12.2, 8192 16.9, 16.3, 12000 18.2, 19.5; but for one head, whose parts
    // are many: 4000 11.3, 11.4, 16000 14.6, 17.6).  Beyond that 16 rows of long 16-bit heads have 32 keys a wave on their way
    // instead of two workgroups of 16 (16 sequences of 4000 slots, heads of 192: 97.6, 87.3; one of 4000 17.5, 22.8).
    const int64_t slots_read = p.units * most;
    if (!joint && slots_read < (1 << 26) / row_bytes) {
        p.groups = kComputeUnits;
        if (p.tile_rows == 16 && row_bytes == 256 && slots_read < (1 << 25) / row_bytes && most <= 8192 * p.units) p.slice = 16;
    } else if (p.slice == 16 && size == 2) {
        p.slice = 32;
        p.groups = kComputeUnits;
    }
    p.joint_tiles = joint_tiles;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t from = at;
        at += (bytes + 255) / 256 * 256;
        return from;
    };
    auto parts = [&](int64_t units, int groups, int rows, size_t* ends, size_t* stats, size_t* sums) {
        *ends = take(units * 8);
        *stats = take((size_t)(units + groups) * rows * 8);
        *sums = take((size_t)(units + groups) * rows * c->dim * 4);
    };
    // Behind a joint prefix a tree has a part however many trees there are: of its own rows only (8500 tokens, 8 heads of 64: 54 MB,
    // 2.2 GB of whole tiles).  Elsewhere units are few, and a tile's statistics fill cache lines that no other workgroup writes
    // (one token behind 8192 slots 16.1 us, 16.3 by its four rows).
    p.part_rows = joint ? (int)p.rows : p.tile_rows;
    parts(p.units, p.groups, p.part_rows, &p.ends, &p.stats, &p.sums);
    if (joint) parts((int64_t)p.joint_tiles * c->heads, p.groups, kJointRows, &p.joint_ends, &p.joint_stats, &p.joint_sums);
    p.bytes = at;
    return true;
}

}  // namespace mdsd

extern "C" {

size_t mdsd_tree_attention_workspace_bytes(const mdsd_kv_cache* cache, const mdsd_tree* tree, int32_t q_heads,
                                           int32_t shared, int32_t longest)
{
    using namespace mdsd;
    Cache C;
    Trees T;
    AttentionPlan plan;
    if (check_cache(cache, tree, &C, &T) != MDSD_OK || q_heads < 1 || q_heads % cache->heads || shared < 0 || longest < 0)
        return 0;
    return plan_attention(cache, tree, q_heads, shared, longest, true, &plan) ? plan.bytes : 0;
}

int mdsd_tree_attention(const mdsd_kv_cache* cache, int32_t layer, const mdsd_tree* tree, const mdsd_heads* q,
                        const mdsd_heads* out, float scale, const int32_t* shared_pages, int32_t shared,
                        int32_t longest, int32_t* flags, void* ws, size_t ws_bytes, void* stream)
{
    using namespace mdsd;
    AttentionParams P = {};
    int rc = check_cache(cache, tree, &P.cache, &P.trees);
    if (rc == kEmptyTrees) return MDSD_OK;
    if (rc != MDSD_OK) return rc;
    if ((rc = check_heads(q, P.cache, cache->dtype, &P.q)) != MDSD_OK) return rc;
    if ((rc = check_heads(out, P.cache, cache->dtype, &P.out)) != MDSD_OK) return rc;
    if (layer < 0 || layer >= cache->layers) return MDSD_E_SHAPE;
    if (q->heads != out->heads || q->heads % cache->heads || one_place(*out, P.trees)) return MDSD_E_SHAPE;
    if (overlap(P.q, P.out, P.trees, P.cache, cache->dtype)) return MDSD_E_ALIGN;
    if (shared < 0 || longest < 0 || shared > (int64_t)cache->table_pages * cache->page_size) return MDSD_E_SHAPE;
    if (shared && !shared_pages) return MDSD_E_NULL;
    const double scale_of_two = (double)scale * 1.4426950408889634;
    if (!(scale > 0.f) || !(scale_of_two <= FLT_MAX)) return MDSD_E_TEMP;
    P.scale = (float)scale_of_two;
    if ((uintptr_t)flags & 3 || (uintptr_t)shared_pages & 3 || (uintptr_t)ws & 15) return MDSD_E_ALIGN;
    AttentionPlan plan;
    if (!plan_attention(cache, tree, q->heads, shared, longest, ws != nullptr, &plan)) return MDSD_E_SHAPE;
    if (ws_bytes < plan.bytes) return MDSD_E_WORKSPACE;
    P.group = q->heads / cache->heads;
    P.by_group = Divisor::of(P.group);
    P.by_heads = Divisor::of(cache->heads);
    P.by_rows = Divisor::of((int)plan.rows);
    P.slack = fminf(8.f / P.scale, 1e30f);
    // (measured: 0 to 8; 64 trees behind a prefix of 16384 431 us without, 379 with 3, fp32 nine-node trees 121, 115 with 1)
    P.unit_cost = plan.tile_rows <= 32 ? 1 : 3;
    P.shared_pages = shared_pages;
    P.shared = shared;
    P.flags = flags;
    P.cache.k += layer * P.cache.ld_layer;
    P.cache.v += layer * P.cache.ld_layer;
    hipStream_t st = (hipStream_t)stream;
    switch (cache->dtype) {
    case MDSD_FP32: return attend_fp32(cache->dim, P, plan, (char*)ws, st);
    case MDSD_BF16: return attend_bf16(cache->dim, P, plan, (char*)ws, st);
    default: return attend_fp16(cache->dim, P, plan, (char*)ws, st);
    }
}

}  // extern "C"
