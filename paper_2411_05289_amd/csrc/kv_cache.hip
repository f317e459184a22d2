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

int check_cache(const mdsd_kv_cache* c, const mdsd_tree* t, Cache* C, Trees* T)
{
    if (!t) return MDSD_E_NULL;
    if (t->B == 0) return kEmptyTrees;
    if (!c || !c->k || !c->v || !c->table || !c->lengths) return MDSD_E_NULL;
    const int size = element_size(c->dtype);
    if (!size) return MDSD_E_DTYPE;
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
    if (c->layers < 1 || c->pages < 1 || c->page_size < 1 || c->heads < 1 || c->table_pages < 1) return MDSD_E_SHAPE;
    if (c->dim < 8 || c->dim > MDSD_MAX_DIM || c->dim % 8 || c->ld_table < c->table_pages) return MDSD_E_SHAPE;
    if ((int64_t)c->table_pages * c->page_size > kMostSlots) return MDSD_E_SHAPE;
    if (((uintptr_t)c->k | (uintptr_t)c->v) & 15) return MDSD_E_ALIGN;
    if (((uintptr_t)c->table | (uintptr_t)c->lengths | (uintptr_t)t->first_child | (uintptr_t)t->counts) & 3) return MDSD_E_ALIGN;
    int64_t ld_page, ld_slot;
    if (!stride(c->ld_layer, size, &C->ld_layer) || !stride(c->ld_page, size, &ld_page) || !stride(c->ld_slot, size, &ld_slot) ||
        !stride(c->ld_head, size, &C->ld_head))
        return MDSD_E_ALIGN;
    if (ld_page >> 36 || ld_slot >> 36) return MDSD_E_SHAPE;
    C->ld_page = (uint32_t)(ld_page >> 4);
    C->ld_slot = (uint32_t)(ld_slot >> 4);
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

}  // namespace mdsd
