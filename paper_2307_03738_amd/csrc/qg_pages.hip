// Bookkeeping of a cache's pages: growing and shrinking sequences, branching them, packing the pool, copying pages.
#include "qg_common.h"

namespace {

struct Planes {
    int n;
    unsigned units;                     // copying units of a page, over all planes and layers
    struct {
        char *base;
        int64_t layer_stride, page_bytes;
        unsigned layer_units, units;    // units of a page in one layer, and in all layers
    } p[QG_MAX_PLANES];
};

constexpr int COPY_UNIT = 4096;         // bytes: 256 lanes of 16

// Copies pages[i][0] onto pages[i][1] for i below the count; a workgroup takes units of 4 KB, all over the list.
__global__ __launch_bounds__(256) void copy_pages(Planes planes, const int32_t *pairs, const int32_t *count, int most, int64_t pages)
{
    const int64_t units = (int64_t)(count ? min(*count, most) : most) * planes.units;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int64_t pair = u / planes.units;
        unsigned at = (unsigned)(u - pair * planes.units);
        const int32_t from = pairs[2 * pair], to = pairs[2 * pair + 1];
        if (from < 0 || to < 0 || from >= pages || to >= pages) continue;
        int k = 0;
        while (at >= planes.p[k].units) at -= planes.p[k++].units;
        const unsigned layer = at / planes.p[k].layer_units;
        const int64_t offset = (int64_t)(at - layer * planes.p[k].layer_units) * COPY_UNIT + threadIdx.x * 16;
        char *base = planes.p[k].base + layer * planes.p[k].layer_stride + offset;
        if (offset < planes.p[k].page_bytes)
            *(uint4 *)(base + to * planes.p[k].page_bytes) = *(const uint4 *)(base + from * planes.p[k].page_bytes);
    }
}

struct Book {
    const int32_t *tables, *lens, *refs;
    int32_t *tables_out, *lens_out, *refs_out;
    int64_t pages;
    int rows, max_pages, page;
};

constexpr int BOOK_LANES = 1024;

// Sum of the values of the lanes before this one, and of all of them.
__device__ inline int before_me(int v, int *part, int *all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int s = v;
    for (int off = 1; off < 64; off <<= 1) {
        const int o = __shfl_up(s, off);
        if (lane >= off) s += o;
    }
    __syncthreads();                    // part is free again
    if (lane == 63) part[wave] = s;
    __syncthreads();
    int base = 0, total = 0;
    for (int w = 0; w < BOOK_LANES / 64; ++w) {
        if (w < wave) base += part[w];
        total += part[w];
    }
    *all = total;
    return base + s - v;
}

__device__ inline int32_t seen(const int32_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

__device__ inline int pages_for(int len, int page, int most)
{
    return min((int)(((int64_t)max(len, 0) + page - 1) / page), most);
}

struct ResizeSpace {
    int32_t *refs, *free, *start, *pairs, *count;
};

// One workgroup keeps the whole book.
__global__ __launch_bounds__(BOOK_LANES) void resize_book(Book b, const int32_t *new_lens, ResizeSpace w, int32_t *lacking)
{
    __shared__ int part[BOOK_LANES / 64], copies;
    const int tid = threadIdx.x;
    const int64_t entries = (int64_t)b.rows * b.max_pages;
    const int limit = b.max_pages * b.page;
    if (tid == 0) copies = 0;
    for (int64_t p = tid; p < b.pages; p += BOOK_LANES) w.refs[p] = b.refs[p];
    __syncthreads();
    // references of the dropped pages
    for (int64_t e = tid; e < entries; e += BOOK_LANES) {
        const int row = (int)(e / b.max_pages), column = (int)(e - (int64_t)row * b.max_pages);
        const int had = pages_for(b.lens[row], b.page, b.max_pages), has = pages_for(new_lens[row], b.page, b.max_pages);
        const int32_t id = b.tables[e];
        if (column >= has && column < had && id >= 0 && id < b.pages) atomicSub(&w.refs[id], 1);
    }
    __syncthreads();
    // pages that each row needs, and where its share of the free ones begins
    int need = 0;
    for (int first = 0; first < b.rows; first += BOOK_LANES) {
        const int row = first + tid;
        int want = 0;
        if (row < b.rows) {
            const int old = min(max(b.lens[row], 0), limit), len = min(max(new_lens[row], 0), limit);
            const int had = pages_for(old, b.page, b.max_pages), has = pages_for(len, b.page, b.max_pages);
            want = max(has - had, 0);
            if (len > old && old % b.page) {
                const int32_t id = b.tables[(int64_t)row * b.max_pages + had - 1];
                if (id >= 0 && id < b.pages && seen(&w.refs[id]) > 1) want |= 1 << 30;
            }
        }
        const int n = (want & ~(1 << 30)) + (want >> 30);
        int all;
        const int before = before_me(n, part, &all);
        if (row < b.rows) w.start[row] = (need + before) | (want & (1 << 30));
        need += all;
    }
    // the lowest free pages
    int found = 0;
    for (int64_t first = 0; first < b.pages && found < need; first += BOOK_LANES) {
        const int64_t p = first + tid;
        const int is_free = p < b.pages && seen(&w.refs[p]) == 0;
        int all;
        const int at = found + before_me(is_free, part, &all);
        if (is_free && at < need) w.free[at] = (int32_t)p;
        found += all;
    }
    const bool enough = found >= need;
    if (tid == 0) *lacking = enough ? 0 : need - found;
    __syncthreads();
    for (int64_t p = tid; p < b.pages; p += BOOK_LANES) {
        const int32_t v = enough ? seen(&w.refs[p]) : b.refs[p];
        b.refs_out[p] = v;
    }
    __syncthreads();
    // what is copied or shared: refs_out is only touched by atomics from here on
    for (int64_t e = tid; e < entries; e += BOOK_LANES) {
        const int row = (int)(e / b.max_pages), column = (int)(e - (int64_t)row * b.max_pages);
        const int old = min(max(b.lens[row], 0), limit), len = min(max(new_lens[row], 0), limit);
        const int had = pages_for(old, b.page, b.max_pages), has = pages_for(len, b.page, b.max_pages);
        int32_t id = b.tables[e];
        if (enough) {
            const int start = w.start[row], copied = start >> 30;
            const int from = start & ~(1 << 30);
            if (column >= has && column < had) id = -1;
            if (copied && column == had - 1) {
                const int32_t fresh = w.free[from];
                const int k = atomicAdd(&copies, 1);
                w.pairs[2 * k] = id;
                w.pairs[2 * k + 1] = fresh;
                atomicSub(&b.refs_out[id], 1);
                atomicAdd(&b.refs_out[fresh], 1);
                id = fresh;
            } else if (column >= had && column < has) {
                id = w.free[from + copied + column - had];
                atomicAdd(&b.refs_out[id], 1);
            }
        }
        b.tables_out[e] = id;
    }
    __syncthreads();
    if (tid == 0) *w.count = enough ? copies : 0;
    for (int row = tid; row < b.rows; row += BOOK_LANES) b.lens_out[row] = enough ? min(max(new_lens[row], 0), limit) : b.lens[row];
}

__global__ __launch_bounds__(256) void fork_refs(Book b)
{
    const int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (p < b.pages) b.refs_out[p] = b.refs[p];
}

__global__ __launch_bounds__(256) void fork_rows(Book b, const int32_t *parents)
{
    const int row = blockIdx.x;
    const int parent = parents[row];
    const bool some = parent >= 0 && parent < b.rows;
    for (int column = threadIdx.x; column < b.max_pages; column += 256) {
        const int32_t was = b.tables[(int64_t)row * b.max_pages + column];
        const int32_t is = some ? b.tables[(int64_t)parent * b.max_pages + column] : -1;
        b.tables_out[(int64_t)row * b.max_pages + column] = is;
        if (was == is) continue;
        if (was >= 0 && was < b.pages) atomicSub(&b.refs_out[was], 1);
        if (is >= 0 && is < b.pages) atomicAdd(&b.refs_out[is], 1);
    }
    if (threadIdx.x == 0) b.lens_out[row] = some ? b.lens[parent] : 0;
}

struct CompactSpace {
    int32_t *map, *moved, *pairs, *count;
};

__global__ __launch_bounds__(BOOK_LANES) void compact_book(Book b, CompactSpace w, int32_t *live_out)
{
    __shared__ int part[BOOK_LANES / 64];
    const int tid = threadIdx.x;
    int mine = 0, live;
    for (int64_t p = tid; p < b.pages; p += BOOK_LANES) mine += b.refs[p] > 0;
    before_me(mine, part, &live);
    int sources = 0, targets = 0;
    for (int64_t first = 0; first < b.pages; first += BOOK_LANES) {
        const int64_t p = first + tid;
        const int32_t r = p < b.pages ? b.refs[p] : 0;
        const int target = p < live && r <= 0, source = p >= live && r > 0;
        int all_t, all_s;
        const int t = targets + before_me(target, part, &all_t), s = sources + before_me(source, part, &all_s);
        if (target) w.pairs[2 * t + 1] = (int32_t)p;
        if (source) {
            w.pairs[2 * s] = (int32_t)p;
            w.moved[s] = r;
        }
        targets += all_t;
        sources += all_s;
    }
    __syncthreads();
    for (int64_t p = tid; p < b.pages; p += BOOK_LANES) {
        w.map[p] = (int32_t)p;
        const int32_t r = b.refs[p];
        b.refs_out[p] = p < live ? r : 0;
    }
    __syncthreads();
    for (int i = tid; i < sources; i += BOOK_LANES) {
        w.map[w.pairs[2 * i]] = w.pairs[2 * i + 1];
        b.refs_out[w.pairs[2 * i + 1]] = w.moved[i];
    }
    if (tid == 0) {
        *w.count = sources;
        *live_out = live;
    }
}

__global__ __launch_bounds__(256) void compact_tables(Book b, const int32_t *map)
{
    const int64_t entries = (int64_t)b.rows * b.max_pages;
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= entries) return;
    const int32_t id = b.tables[e];
    b.tables_out[e] = id >= 0 && id < b.pages ? map[id] : id;
}

int check_planes(const qg_page_plane *planes, int n, Planes *out)
{
    if (n < 0 || n > QG_MAX_PLANES) return QG_ERR_UNSUPPORTED;
    if (n && !planes) return QG_ERR_NULL;
    *out = Planes{};
    out->n = n;
    int64_t units = 0;
    for (int i = 0; i < n; ++i) {
        if (!planes[i].base) return QG_ERR_NULL;
        if (planes[i].layers <= 0 || planes[i].page_bytes <= 0) return QG_ERR_SHAPE;
        if (!qg_aligned16(planes[i].base) || planes[i].page_bytes % 16) return QG_ERR_ALIGN;
        const int64_t per_layer = (planes[i].page_bytes + COPY_UNIT - 1) / COPY_UNIT;
        if (per_layer > 0x7fffffff / planes[i].layers) return QG_ERR_SHAPE;
        out->p[i].base = (char *)planes[i].base;
        out->p[i].page_bytes = planes[i].page_bytes;
        out->p[i].layer_units = (unsigned)per_layer;
        out->p[i].units = (unsigned)(per_layer * planes[i].layers);
        units += per_layer * planes[i].layers;
        if (units > 0x7fffffff) return QG_ERR_SHAPE;
    }
    out->units = (unsigned)units;
    return QG_OK;
}

void set_layers(Planes *p, int64_t pages)
{
    for (int i = 0; i < p->n; ++i) p->p[i].layer_stride = pages * p->p[i].page_bytes;
}

int launch_copies(const Planes &planes, const int32_t *pairs, const int32_t *count, int most, int64_t pages, hipStream_t st)
{
    if (planes.n == 0 || most == 0) return QG_OK;
    const int64_t units = (int64_t)most * planes.units, blocks = 16 * (int64_t)qg_compute_units();
    hipLaunchKernelGGL(copy_pages, dim3((unsigned)(units < blocks ? units : blocks)), dim3(256), 0, st, planes, pairs, count, most, pages);
    return qg_launch_status();
}

int check_book(const qg_page_book *book, bool lens, Book *b)
{
    if (!book) return QG_ERR_NULL;
    if (book->rows < 0 || book->max_pages <= 0 || book->pages <= 0 || book->pages > 0x3fffffff || book->page <= 0) return QG_ERR_SHAPE;
    if ((int64_t)book->max_pages * book->page > 0x3fffffff || (int64_t)book->rows * book->max_pages > 0x3fffffff) return QG_ERR_SHAPE;
    if (!book->refs || !book->refs_out) return QG_ERR_NULL;
    if (book->rows && (!book->tables || !book->tables_out || (lens && (!book->lens || !book->lens_out)))) return QG_ERR_NULL;
    for (const void *p : {(const void *)book->tables, (const void *)book->lens, (const void *)book->refs, (const void *)book->tables_out,
                          (const void *)book->lens_out, (const void *)book->refs_out})
        if ((uintptr_t)p & 3) return QG_ERR_ALIGN;
    *b = {book->tables, book->lens, book->refs, book->tables_out, book->lens_out, book->refs_out, book->pages, book->rows, book->max_pages, book->page};
    return QG_OK;
}

}  // namespace

extern "C" size_t qg_pages_workspace_bytes(int rows, int max_pages, int64_t pages)
{
    if (rows < 0 || max_pages <= 0 || pages <= 0 || pages > 0x3fffffff || (int64_t)rows * max_pages > 0x3fffffff) return 0;
    return qg_round_up(4 * (4 * (size_t)pages + 4 * (size_t)rows + 64), 256);
}

extern "C" int qg_pages_copy(const qg_page_plane *planes, int n_planes, int64_t pages, const int32_t *pairs, int count, void *stream)
{
    Planes p;
    const int rc = check_planes(planes, n_planes, &p);
    if (rc != QG_OK) return rc;
    if (pages <= 0 || pages > 0x3fffffff || count < 0) return QG_ERR_SHAPE;
    if (count == 0 || n_planes == 0) return QG_OK;
    if (!pairs) return QG_ERR_NULL;
    if ((uintptr_t)pairs & 3) return QG_ERR_ALIGN;
    set_layers(&p, pages);
    return launch_copies(p, pairs, nullptr, count, pages, (hipStream_t)stream);
}

extern "C" int qg_pages_resize(const qg_page_book *book, const int32_t *new_lens, const qg_page_plane *planes, int n_planes, int32_t *lacking,
                               void *workspace, size_t workspace_bytes, void *stream)
{
    Book b;
    Planes p;
    int rc = check_book(book, true, &b);
    if (rc != QG_OK) return rc;
    if ((rc = check_planes(planes, n_planes, &p)) != QG_OK) return rc;
    if ((b.rows && !new_lens) || !lacking) return QG_ERR_NULL;
    if (((uintptr_t)new_lens & 3) || ((uintptr_t)lacking & 3) || !qg_aligned16(workspace)) return QG_ERR_ALIGN;
    if (!workspace || workspace_bytes < qg_pages_workspace_bytes(b.rows, b.max_pages, b.pages)) return QG_ERR_WORKSPACE;
    set_layers(&p, b.pages);
    int32_t *w = (int32_t *)workspace;
    const ResizeSpace space = {w + 64, w + 64 + b.pages, w + 64 + 2 * b.pages, w + 64 + 2 * b.pages + b.rows, w};
    hipStream_t st = (hipStream_t)stream;
    hipLaunchKernelGGL(resize_book, dim3(1), dim3(BOOK_LANES), 0, st, b, new_lens, space, lacking);
    if ((rc = qg_launch_status()) != QG_OK) return rc;
    return launch_copies(p, space.pairs, space.count, b.rows, b.pages, st);
}

extern "C" int qg_pages_fork(const qg_page_book *book, const int32_t *parents, void *stream)
{
    Book b;
    const int rc = check_book(book, true, &b);
    if (rc != QG_OK) return rc;
    if (b.rows && !parents) return QG_ERR_NULL;
    if ((uintptr_t)parents & 3) return QG_ERR_ALIGN;
    if (b.refs == b.refs_out || (b.rows && (b.tables == b.tables_out || b.lens == b.lens_out))) return QG_ERR_UNSUPPORTED;
    hipStream_t st = (hipStream_t)stream;
    hipLaunchKernelGGL(fork_refs, dim3((unsigned)((b.pages + 255) / 256)), dim3(256), 0, st, b);
    if (b.rows) hipLaunchKernelGGL(fork_rows, dim3((unsigned)b.rows), dim3(256), 0, st, b, parents);
    return qg_launch_status();
}

extern "C" int qg_pages_compact(const qg_page_book *book, const qg_page_plane *planes, int n_planes, int32_t *live, void *workspace,
                                size_t workspace_bytes, void *stream)
{
    Book b;
    Planes p;
    int rc = check_book(book, false, &b);
    if (rc != QG_OK) return rc;
    if ((rc = check_planes(planes, n_planes, &p)) != QG_OK) return rc;
    if (!live) return QG_ERR_NULL;
    if (((uintptr_t)live & 3) || !qg_aligned16(workspace)) return QG_ERR_ALIGN;
    if (!workspace || workspace_bytes < qg_pages_workspace_bytes(b.rows, b.max_pages, b.pages)) return QG_ERR_WORKSPACE;
    set_layers(&p, b.pages);
    int32_t *w = (int32_t *)workspace;
    const CompactSpace space = {w + 64, w + 64 + b.pages, w + 64 + 2 * b.pages, w};
    hipStream_t st = (hipStream_t)stream;
    hipLaunchKernelGGL(compact_book, dim3(1), dim3(BOOK_LANES), 0, st, b, space, live);
    if (b.rows)
        hipLaunchKernelGGL(compact_tables, dim3((unsigned)(((int64_t)b.rows * b.max_pages + 255) / 256)), dim3(256), 0, st, b, space.map);
    if ((rc = qg_launch_status()) != QG_OK) return rc;
    const int most = (int)(b.pages / 2 < 0x7fffffff ? b.pages / 2 : 0x7fffffff);
    return launch_copies(p, space.pairs, space.count, most, b.pages, st);
}
