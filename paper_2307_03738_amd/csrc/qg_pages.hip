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

constexpr int COPY_UNIT = 8192;         // bytes: 256 lanes of 2 x 16

// Table entries that follow their pages' move (entries 0: none).
struct Renumber {
    const int32_t *tables, *map;
    int32_t *tables_out;
    int64_t entries;
};

// Copies pages[i][0] onto pages[i][1] for i below the count; a workgroup takes units of 8 KB, all over the list.  (5.0 ... 5.5 TB/s read and
// written on 720 MB; a large copy 5.3.)
__global__ __launch_bounds__(256) void copy_pages(Planes planes, const int32_t *pairs, const int32_t *count, int most, int64_t pages, Renumber ids)
{
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < ids.entries; e += (int64_t)gridDim.x * 256) {
        const int32_t id = ids.tables[e];
        ids.tables_out[e] = id >= 0 && id < pages ? ids.map[id] : id;
    }
    const int64_t units = (int64_t)(count ? min(*count, most) : most) * planes.units;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int64_t pair = u / planes.units;
        unsigned at = (unsigned)(u - pair * planes.units);
        const int32_t from = pairs[2 * pair], to = pairs[2 * pair + 1];
        if (from < 0 || to < 0 || from >= pages || to >= pages) continue;
        int k = 0;
        while (at >= planes.p[k].units) at -= planes.p[k++].units;
        const unsigned layer = at / planes.p[k].layer_units;
        const int64_t bytes = planes.p[k].page_bytes, offset = (int64_t)(at - layer * planes.p[k].layer_units) * COPY_UNIT + threadIdx.x * 16;
        char *base = planes.p[k].base + layer * planes.p[k].layer_stride + offset;
        uint4 x = {}, y = {};
        if (offset < bytes) x = *(const uint4 *)(base + from * bytes);
        if (offset + 4096 < bytes) y = *(const uint4 *)(base + from * bytes + 4096);
        if (offset < bytes) *(uint4 *)(base + to * bytes) = x;
        if (offset + 4096 < bytes) *(uint4 *)(base + to * bytes + 4096) = y;
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
#define QG_UP(CTRL, ROWS) s += __builtin_amdgcn_update_dpp(0, s, CTRL, ROWS, 0xf, false);
    QG_UP(0x111, 0xf) QG_UP(0x112, 0xf) QG_UP(0x114, 0xf) QG_UP(0x118, 0xf)          // row_shr 1, 2, 4, 8
    QG_UP(0x142, 0xa) QG_UP(0x143, 0xc)                                            // row_bcast 15, 31
#undef QG_UP
    __syncthreads();                    // part is free again
    if (lane == 63) part[wave] = s;
    __syncthreads();
    int base = 0, total = 0;
#pragma unroll
    for (int w = 0; w < BOOK_LANES / 64; ++w) {
        const int x = part[w];
        if (w < wave) base += x;
        total += x;
    }
    *all = total;
    return base + s - v;
}

__device__ inline int32_t seen(const int32_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

__device__ inline int pages_for(int len, int page, int most)
{
    return min((int)(((int64_t)max(len, 0) + page - 1) / page), most);
}

// Turns of 8192 pages: a wavefront takes 512 neighbouring ones, 64 at a time, and numbers them by the votes of its lanes, so that every
// load and store is of neighbouring words.
constexpr int TURN = 8 * BOOK_LANES;
__device__ inline int64_t page_of_lane(int64_t p0, int k) { return p0 + (threadIdx.x >> 6) * 512 + k * 64 + (threadIdx.x & 63); }
__device__ inline int votes_before(uint64_t votes) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(votes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)votes, 0)); }

// What a row's new length changes: pages [has, had) go, pages [had, has) come, and a row that grows inside its last page may need a copy of it.
struct Change {
    int had, has, len;
    bool inside;
    __device__ int gone() const { return max(had - has, 0); }
    __device__ int more() const { return max(has - had, 0); }
};

__device__ inline Change change_of(const Book &b, const int32_t *new_lens, int row)
{
    const int limit = b.max_pages * b.page, old = min(max(b.lens[row], 0), limit), len = min(max(new_lens[row], 0), limit);
    Change c;
    c.had = pages_for(old, b.page, b.max_pages);
    c.has = pages_for(len, b.page, b.max_pages);
    c.len = len;
    c.inside = len > old && old % b.page != 0;
    return c;
}

struct ResizeSpace {
    int32_t *free, *pairs, *count;
};

// The row that unit e belongs to, where row r's units begin at at[r] (at[rows] is past e).
__device__ inline int row_of(const int *at, int rows, int e)
{
    int low = 0, high = rows;
    while (high - low > 1) {
        const int mid = (low + high) / 2;
        if (at[mid] <= e) low = mid;
        else high = mid;
    }
    return low;
}

constexpr int FREE_IN_LDS = 4096;

// Workgroup 0 keeps the book: pages that go and pages that come are dealt out over its lanes one by one, whatever their rows, so its time
// follows what changes (and the references, which it passes on and searches for free pages from the lowest id on).  The other
// workgroups pass on the table entries that do not change.  (64 rows of 256 entries, 8192 pages: 14.2 us, a chain of some ten loads and sums; one
// workgroup for all of it, an entry a lane: 33.)
__global__ __launch_bounds__(BOOK_LANES) void resize_book(Book b, const int32_t *new_lens, ResizeSpace w, int32_t *lacking)
{
    const int tid = threadIdx.x;
    if (blockIdx.x > 0) {
        const int64_t entries = (int64_t)b.rows * b.max_pages;
        const int64_t e = (int64_t)(blockIdx.x - 1) * BOOK_LANES + tid;
        if (e >= entries) return;
        const int row = (int)(e / b.max_pages), column = (int)(e - (int64_t)row * b.max_pages);
        const int32_t id = b.tables[e];
        const Change c = change_of(b, new_lens, row);
        const bool changes = (column >= min(c.had, c.has) && column < max(c.had, c.has)) || (c.inside && column == c.had - 1);
        if (!changes) b.tables_out[e] = id;
        return;
    }
    __shared__ int part[BOOK_LANES / 64], copies, at[BOOK_LANES + 1], low_free[FREE_IN_LDS];
    __shared__ int16_t copied[BOOK_LANES];
    __shared__ int had[BOOK_LANES], has[BOOK_LANES];               // of the 1024 rows at hand
    if (tid == 0) copies = 0;
    if (b.refs != b.refs_out) {
        // (the references may be at any 4-byte address)
        constexpr int AHEAD = 8;
        for (int64_t p0 = 0; p0 < b.pages; p0 += AHEAD * BOOK_LANES) {
            int32_t v[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) v[k] = p0 + k * BOOK_LANES + tid < b.pages ? b.refs[p0 + k * BOOK_LANES + tid] : 0;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (p0 + k * BOOK_LANES + tid < b.pages) b.refs_out[p0 + k * BOOK_LANES + tid] = v[k];
        }
    }
    // pages that go, rows 1024 at a time: f(entry, page id) for each
    auto for_gone = [&](auto f) {
        for (int row0 = 0; row0 < b.rows; row0 += BOOK_LANES) {
            const int rows = min(b.rows - row0, BOOK_LANES);
            Change c = {};
            if (tid < rows) c = change_of(b, new_lens, row0 + tid);
            int all;
            const int before = before_me(c.gone(), part, &all);
            if (all == 0) continue;                                 // (of the whole workgroup)
            at[tid] = before;
            has[tid] = c.has;
            __syncthreads();
            for (int e = tid; e < all; e += BOOK_LANES) {
                const int r = row_of(at, rows, e);
                const int64_t entry = (int64_t)(row0 + r) * b.max_pages + has[r] + e - at[r];
                f(entry, b.tables[entry]);
            }
            __syncthreads();
        }
    };
    __syncthreads();
    for_gone([&](int64_t, int32_t id) {
        if (id >= 0 && id < b.pages) atomicSub(&b.refs_out[id], 1);
    });
    // pages that come: those of rows from row0 on begin at `base` in the list of free pages
    auto wants = [&](int row0, int *before) {
        const int row = row0 + tid;
        int n = 0, copy = 0;
        if (row < b.rows) {
            const Change c = change_of(b, new_lens, row);
            n = c.more();
            had[tid] = c.had;
            if (c.inside) {
                const int32_t id = b.tables[(int64_t)row * b.max_pages + c.had - 1];
                copy = id >= 0 && id < b.pages && seen(&b.refs_out[id]) > 1;
            }
        }
        int all;
        *before = before_me(n + copy, part, &all);
        copied[tid] = (int16_t)copy;
        return all;
    };
    int need = 0, before = 0;
    for (int row0 = 0; row0 < b.rows; row0 += BOOK_LANES) need += wants(row0, &before);
    // the lowest free pages
    int found = 0;
    for (int64_t p0 = 0; p0 < b.pages && found < need; p0 += TURN) {
        uint64_t is_free[8];
        int n = 0, all;
        int32_t v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = page_of_lane(p0, k) < b.pages ? seen(&b.refs_out[page_of_lane(p0, k)]) : 1;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            is_free[k] = __ballot(v[k] == 0);
            n += __popcll(is_free[k]);
        }
        int to = found + __shfl(before_me((tid & 63) == 63 ? n : 0, part, &all), 63);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int i = to + votes_before(is_free[k]);
            if (v[k] == 0 && i < need) {
                if (i < FREE_IN_LDS) low_free[i] = (int32_t)page_of_lane(p0, k);
                else w.free[i] = (int32_t)page_of_lane(p0, k);
            }
            to += __popcll(is_free[k]);
        }
        found += all;
    }
    const bool enough = found >= need;
    if (tid == 0) *lacking = enough ? 0 : need - found;
    if (!enough) {
        // as it was
        for_gone([&](int64_t entry, int32_t id) {
            if (id >= 0 && id < b.pages) atomicAdd(&b.refs_out[id], 1);
            b.tables_out[entry] = id;
        });
        for (int row = tid; row < b.rows; row += BOOK_LANES) {
            const Change c = change_of(b, new_lens, row);
            const int64_t first = (int64_t)row * b.max_pages;
            if (b.tables != b.tables_out) {
                if (c.inside) b.tables_out[first + c.had - 1] = b.tables[first + c.had - 1];
                for (int column = c.had; column < c.has; ++column) b.tables_out[first + column] = b.tables[first + column];
            }
        }
        if (b.lens != b.lens_out)
            for (int row = tid; row < b.rows; row += BOOK_LANES) b.lens_out[row] = b.lens[row];
        if (tid == 0) *w.count = 0;
        return;
    }
    int base = 0;
    for (int row0 = 0; row0 < b.rows; row0 += BOOK_LANES) {
        const int rows = min(b.rows - row0, BOOK_LANES);
        int all;
        if (b.rows > BOOK_LANES) {
            // (the same answer as before: references of pages that are copied go down below, after all rows)
            all = wants(row0, &before);
        } else {
            all = need;
        }
        at[tid] = before;
        __syncthreads();
        for (int e = tid; e < all; e += BOOK_LANES) {
            const int r = row_of(at, rows, e), row = row0 + r;
            const int32_t fresh = base + e < FREE_IN_LDS ? low_free[base + e] : w.free[base + e];
            const int k = e - at[r];
            const int64_t first = (int64_t)row * b.max_pages + had[r];
            if (copied[r] && k == 0) {
                const int i = atomicAdd(&copies, 1);
                w.pairs[2 * i] = b.tables[first - 1];
                w.pairs[2 * i + 1] = fresh;
                b.tables_out[first - 1] = fresh;
            } else {
                b.tables_out[first + k - copied[r]] = fresh;
            }
            b.refs_out[fresh] = 1;
        }
        if (b.tables != b.tables_out && tid < rows) {
            const Change c = change_of(b, new_lens, row0 + tid);
            const int64_t entry = (int64_t)(row0 + tid) * b.max_pages + c.had - 1;
            if (c.inside && !copied[tid]) b.tables_out[entry] = b.tables[entry];
        }
        base += all;
        __syncthreads();
    }
    // what the copies were taken of
    for (int i = tid; i < copies; i += BOOK_LANES) atomicSub(&b.refs_out[w.pairs[2 * i]], 1);
    for_gone([&](int64_t entry, int32_t) { b.tables_out[entry] = -1; });
    for (int row = tid; row < b.rows; row += BOOK_LANES) b.lens_out[row] = change_of(b, new_lens, row).len;
    if (tid == 0) *w.count = copies;
}

__global__ __launch_bounds__(256) void fork_refs(Book b)
{
    const int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (p < b.pages) b.refs_out[p] = b.refs[p];
}

__global__ __launch_bounds__(256) void fork_rows(Book b, const int32_t *parents, int first_row)
{
    const int row = first_row + (int)blockIdx.x;
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

// One workgroup: counts the pages in use, numbers the sources and the targets (both in one sum), and leaves the new references and the
// map from old ids to new ones.  (16384 pages: 12 us; a page a lane and two scans a turn: 38.)
__global__ __launch_bounds__(BOOK_LANES) void compact_book(Book b, CompactSpace w, int32_t *live_out)
{
    __shared__ int part[BOOK_LANES / 64];
    const int tid = threadIdx.x;
    int mine = 0, live;
    int32_t v[8];
    auto load = [&](int64_t p0) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = page_of_lane(p0, k) < b.pages ? b.refs[page_of_lane(p0, k)] : 0;
    };
    for (int64_t p0 = 0; p0 < b.pages; p0 += TURN) {
        load(p0);
#pragma unroll
        for (int k = 0; k < 8; ++k) mine += v[k] > 0;
    }
    before_me(mine, part, &live);
    int sources = 0, targets = 0;
    for (int64_t p0 = 0; p0 < b.pages; p0 += TURN) {
        if (b.pages > TURN) load(p0);
        int n = 0, all;                                             // of the wavefront, in its last lane: targets, sources << 16
        uint64_t target[8], source[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int64_t p = page_of_lane(p0, k);
            target[k] = __ballot(p < live && v[k] <= 0);
            source[k] = __ballot(p >= live && v[k] > 0);
            n += __popcll(target[k]) | __popcll(source[k]) << 16;
        }
        const int first = __shfl(before_me((tid & 63) == 63 ? n : 0, part, &all), 63);
        int t = targets + (first & 0xffff), s = sources + (first >> 16);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int64_t p = page_of_lane(p0, k);
            if (p < live && v[k] <= 0) w.pairs[2 * (t + votes_before(target[k])) + 1] = (int32_t)p;
            if (p >= live && v[k] > 0) {
                const int i = s + votes_before(source[k]);
                w.moved[i] = v[k];
                w.pairs[2 * i] = (int32_t)p;
            }
            if (p < b.pages) {
                w.map[p] = (int32_t)p;
                b.refs_out[p] = p < live ? v[k] : 0;
            }
            t += __popcll(target[k]);
            s += __popcll(source[k]);
        }
        targets += all & 0xffff;
        sources += all >> 16;
    }
    __syncthreads();
#pragma unroll 4
    for (int i = tid; i < sources; i += BOOK_LANES) {
        const int32_t from = w.pairs[2 * i], to = w.pairs[2 * i + 1], refs = w.moved[i];
        w.map[from] = to;
        b.refs_out[to] = refs;
    }
    if (tid == 0) {
        *w.count = sources;
        *live_out = live;
    }
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

int launch_copies(const Planes &planes, const int32_t *pairs, const int32_t *count, int most, int64_t pages, const Renumber &ids, hipStream_t st)
{
    if ((planes.n == 0 || most == 0) && ids.entries == 0) return QG_OK;
    const int64_t copies = (int64_t)most * planes.units, lanes = (ids.entries + 255) / 256, units = copies > lanes ? copies : lanes;
    const int64_t blocks = 8 * (int64_t)qg_compute_units();
    hipLaunchKernelGGL(copy_pages, dim3((unsigned)(units < blocks ? units : blocks)), dim3(256), 0, st, planes, pairs, count, most, pages, ids);
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
    return launch_copies(p, pairs, nullptr, count, pages, Renumber{}, (hipStream_t)stream);
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
    if ((b.tables == b.tables_out) != (b.lens == b.lens_out)) return QG_ERR_UNSUPPORTED;        // (one is read while the other is written)
    if (((uintptr_t)new_lens & 3) || ((uintptr_t)lacking & 3) || !qg_aligned16(workspace)) return QG_ERR_ALIGN;
    if (!workspace || workspace_bytes < qg_pages_workspace_bytes(b.rows, b.max_pages, b.pages)) return QG_ERR_WORKSPACE;
    set_layers(&p, b.pages);
    int32_t *w = (int32_t *)workspace;
    const ResizeSpace space = {w + 64, w + 64 + b.pages, w};
    hipStream_t st = (hipStream_t)stream;
    const int64_t passed_on = b.tables == b.tables_out ? 0 : ((int64_t)b.rows * b.max_pages + BOOK_LANES - 1) / BOOK_LANES;
    hipLaunchKernelGGL(resize_book, dim3((unsigned)(1 + passed_on)), dim3(BOOK_LANES), 0, st, b, new_lens, space, lacking);
    if ((rc = qg_launch_status()) != QG_OK) return rc;
    return launch_copies(p, space.pairs, space.count, b.rows, b.pages, Renumber{}, st);
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
    constexpr int MOST = 1 << 23;                                   // (a launch has less than 2^32 lanes)
    for (int row = 0; row < b.rows; row += MOST)
        hipLaunchKernelGGL(fork_rows, dim3((unsigned)(b.rows - row < MOST ? b.rows - row : MOST)), dim3(256), 0, st, b, parents, row);
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
    if ((rc = qg_launch_status()) != QG_OK) return rc;
    const int most = (int)(b.pages / 2 < 0x7fffffff ? b.pages / 2 : 0x7fffffff);
    return launch_copies(p, space.pairs, space.count, most, b.pages, Renumber{b.tables, space.map, b.tables_out, (int64_t)b.rows * b.max_pages}, st);
}
