// Host side of the key-value cache calls: what can be checked before a launch.
#include "kv_cache.h"

namespace mdsd {

static int element_size(int dtype) { return dtype == MDSD_FP32 ? 4 : dtype == MDSD_BF16 || dtype == MDSD_FP16 ? 2 : 0; }

// a stride in bytes; false if it is negative, no multiple of 16 bytes, or so large that offsets leave 63 bits
static bool stride(int64_t elements, int size, int64_t* bytes)
{
    if (elements < 0 || elements > (int64_t(1) << 46) || (elements * size) % 16) return false;
    *bytes = elements * size;
    return true;
}

int check_pages(const mdsd_kv_cache* c, const mdsd_kv_scales* scales, Cache* C, Scales* S, int* dtype)
{
    if (!c || !c->k || !c->v || !c->table || !c->lengths) return MDSD_E_NULL;
    *dtype = c->dtype;
    if (scales) {
        if (!scales->k || !scales->v) return MDSD_E_NULL;
        if (c->dtype != MDSD_FP4) return MDSD_E_DTYPE;
        *dtype = scales->dtype;
        *S = {(uint8_t*)scales->k, (uint8_t*)scales->v};
    }
    const int size = element_size(*dtype);
    if (!size) return MDSD_E_DTYPE;
    if (c->layers < 1 || c->pages < 1 || c->page_size < 1 || c->heads < 1 || c->table_pages < 1) return MDSD_E_SHAPE;
    if (c->dim < 8 || c->dim > MDSD_MAX_DIM || c->dim % (scales ? kBlock : 8) || c->ld_table < c->table_pages) return MDSD_E_SHAPE;
    if ((int64_t)c->table_pages * c->page_size > kMostSlots) return MDSD_E_SHAPE;
    if (((uintptr_t)c->k | (uintptr_t)c->v) & 15) return MDSD_E_ALIGN;
    if (((uintptr_t)c->table | (uintptr_t)c->lengths) & 3) return MDSD_E_ALIGN;
    int64_t ld[4];
    const int64_t given[4] = {c->ld_layer, c->ld_page, c->ld_slot, c->ld_head};
    for (int i = 0; i < 4; ++i) {  // (two elements a byte)
        if (scales && given[i] % 2) return MDSD_E_ALIGN;
        if (!stride(scales ? given[i] / 2 : given[i], scales ? 1 : size, &ld[i])) return MDSD_E_ALIGN;
    }
    if (ld[1] >> 36 || ld[2] >> 36) return MDSD_E_SHAPE;
    C->ld_layer = ld[0];
    C->ld_page = (uint32_t)(ld[1] >> 4);
    C->ld_slot = (uint32_t)(ld[2] >> 4);
    C->ld_head = ld[3];
    C->k = (char*)c->k;
    C->v = (char*)c->v;
    C->table = c->table;
    C->ld_table = c->ld_table;
    C->lengths = c->lengths;
    C->layers = c->layers;
    C->pages = c->pages;
    C->page_size = c->page_size;
    C->heads = c->heads;
    C->dim = c->dim;
    C->table_pages = c->table_pages;
    C->by_page = Divisor::of(c->page_size);
    return MDSD_OK;
}

void choose_layer(int layer, Cache* C, Scales* S)
{
    C->k += layer * C->ld_layer;
    C->v += layer * C->ld_layer;
    if (S->k) {
        S->k += layer * (C->ld_layer / 16);
        S->v += layer * (C->ld_layer / 16);
    }
}

int check_cache(const mdsd_kv_cache* c, const mdsd_tree* t, Cache* C, Trees* T)
{
    Scales none = {};
    int dtype;
    return check_cache(c, nullptr, t, C, &none, &dtype, T);
}

int check_cache(const mdsd_kv_cache* c, const mdsd_kv_scales* scales, const mdsd_tree* t, Cache* C, Scales* S, int* dtype, Trees* T)
{
    if (!t) return MDSD_E_NULL;
    if (t->B == 0) return kEmptyTrees;
    // (what is wrong is found in the order that it always was: types, trees, the cache's sizes)
    if (!c || !c->k || !c->v || !c->table || !c->lengths || (scales && (!scales->k || !scales->v))) return MDSD_E_NULL;
    if (scales ? c->dtype != MDSD_FP4 || !element_size(scales->dtype) : !element_size(c->dtype)) return MDSD_E_DTYPE;
    if (t->B < 1 || t->N < 1 || t->depth < 1) return MDSD_E_SHAPE;
    if (t->k < 1 || t->k > MDSD_MAX_K) return MDSD_E_K;
    if ((int64_t)t->B * t->N > INT32_MAX || t->N > kMostSlots) return MDSD_E_SHAPE;
    if (t->first_child) {
        if (t->N > MDSD_MAX_TABLE_NODES) return MDSD_E_SHAPE;
    } else {
        int64_t n = 0, level = 1;
        for (int d = 0; d < t->depth && n <= t->N; ++d, level *= t->k) {
            n += level;
            if (t->k == 1) {  // one node a level
                n = t->depth;
                break;
            }
        }
        if (n != t->N) return MDSD_E_SHAPE;
    }
    const int rc = check_pages(c, scales, C, S, dtype);
    if (rc != MDSD_OK) return rc;
    if (((uintptr_t)t->first_child | (uintptr_t)t->counts) & 3) return MDSD_E_ALIGN;
    T->B = t->B;
    T->N = t->N;
    T->k = t->k;
    T->complete = t->first_child == nullptr;
    T->first_child = t->first_child;
    T->counts = t->counts;
    T->by_k = Divisor::of(t->k);
    return MDSD_OK;
}

int check_heads(const mdsd_heads* h, const Cache& c, int dtype, Heads* H)
{
    if (!h || !h->p) return MDSD_E_NULL;
    if (h->heads < 1) return MDSD_E_SHAPE;
    if ((uintptr_t)h->p & 15) return MDSD_E_ALIGN;
    const int size = element_size(dtype);
    if (!stride(h->ld_tree, size, &H->ld_tree) || !stride(h->ld_node, size, &H->ld_node) ||
        !stride(h->ld_head, size, &H->ld_head))
        return MDSD_E_ALIGN;
    H->p = (char*)h->p;
    H->heads = h->heads;
    return MDSD_OK;
}

bool one_place(const mdsd_kv_cache& c)
{
    return (c.layers > 1 && !c.ld_layer) || (c.pages > 1 && !c.ld_page) || (c.page_size > 1 && !c.ld_slot) || (c.heads > 1 && !c.ld_head);
}

bool one_place(const mdsd_heads& h, const Trees& t)
{
    return (t.B > 1 && !h.ld_tree) || (t.N > 1 && !h.ld_node) || (h.heads > 1 && !h.ld_head);
}

// whether d = sum i_a ld_a + e for some |i_a| < n_a, |e| < bytes; ld falling, each beyond the reach of those behind it
static bool within_reach(int64_t d, const int64_t (*axes)[2], int left, int64_t bytes)
{
    if (left == 0) return d > -bytes && d < bytes;
    const int64_t ld = axes[0][0], n = axes[0][1];
    int64_t i = d / ld - (d % ld < 0);
    for (int j = 0; j < 2; ++j, ++i)
        if (i > -n && i < n && within_reach(d - i * ld, axes + 1, left - 1, bytes)) return true;
    return false;
}

bool overlap(const Heads& from, const Heads& to, const Trees& t, const Cache& c, int dtype)
{
    const int64_t all[3][3] = {{from.ld_tree, to.ld_tree, t.B}, {from.ld_node, to.ld_node, t.N}, {from.ld_head, to.ld_head, from.heads}};
    int64_t axes[3][2];
    int n = 0;
    bool alike = true;
    for (const auto& a : all) {
        if (a[2] == 1) continue;  // its stride may be anything
        alike = alike && a[0] == a[1];
        int at = n++;
        for (; at > 0 && axes[at - 1][0] < a[1]; --at) axes[at][0] = axes[at - 1][0], axes[at][1] = axes[at - 1][1];
        axes[at][0] = a[1], axes[at][1] = a[2];
    }
    if (from.p == to.p) return !alike;
    return alike && within_reach((int64_t)((uintptr_t)to.p - (uintptr_t)from.p), axes, n, (int64_t)c.dim * element_size(dtype));
}

bool rows_overlap(const void* a, int64_t ld_a, const void* b, int64_t ld_b, int64_t B, int64_t width)
{
    const int64_t from = (int64_t)(uintptr_t)a, to = (int64_t)(uintptr_t)b;
    if (B == 1) ld_a = ld_b = width;
    if (from == to && ld_a == ld_b) return false;
    const int64_t bytes_a = ((B - 1) * ld_a + width) * 4, bytes_b = ((B - 1) * ld_b + width) * 4;
    if (from >= to + bytes_b || to >= from + bytes_a) return false;
    if (ld_a != ld_b) return true;
    // rows are `ld` apart: how far the others begin behind one of these
    const int64_t d = (to - from) % (ld_a * 4), behind = d < 0 ? d + ld_a * 4 : d;
    return behind < width * 4 || behind > (ld_a - width) * 4;
}

}  // namespace mdsd
