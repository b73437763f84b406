// C ABI of the user cache (include/aif_cache.h): context, validation, which pages belong to which sequence, and the launches.
//
// The host's book-keeping is what counts: every call settles at once which pages it takes and gives back, and the device's
// copy of the page table follows on the stream with the launches that need it.  A call checks everything first; from there on
// only a HIP call can fail, and what the call was changing is given up (settled).  Nothing is allocated after aif_cache_init.
#include "../../include/aif_cache.h"
#include "aif_cache_dev.h"
#include "cache_book.h"

#include <algorithm>
#include <cstdarg>
#include <cstdio>
#include <exception>
#include <new>
#include <vector>

using namespace aif;

namespace {
constexpr size_t CACHE_LIST_BYTES = 512 << 10;      // of one launch's descriptors, at most
constexpr int FEW_ROWS = 64, ROWS_OF_CU = 64, MIN_TILES = 4, MAX_SPLITS = 128, PART_ROWS = 384;      // plan_attend
constexpr int MAX_UNITS = (1 << 23) - 1;    // of up to 512 threads: a grid holds fewer than 2^32 along an axis
constexpr int CACHE_MAX_LEN = 1 << 30;      // row numbers and sums of two of them fit in 32 bits
constexpr int CACHE_MAX_PAGES = 1 << 23;    // of a sequence, and
constexpr size_t CACHE_MAX_PAGE = 1u << 29; // bytes of a page: a grid's second axis (k_cache_fill, k_cache_move) has up to 65,535 blocks
thread_local char g_cache_init_error[512] = "";
constexpr int LEAN_ASKS = (CACHE_FEW_BYTES - sizeof(CacheLean) - 2 * sizeof(int32_t)) / (sizeof(CacheOwn) + 2 * sizeof(int32_t));     // that fit with one kernel's numbers
}  // namespace

struct aif_cache_ctx {
    CacheShape shape{};
    aif_cache_config cfg{};
    int device = 0;
    CacheBook book;
    int n_cu = 256;
    float *part = nullptr;                  // partial results of one attention kernel, which are joined before the next one starts
    std::vector<uint32_t> stamp;            // sequences that a call has named
    uint32_t stamp_now = 0;
    // Pinned memory for descriptors, in two halves.  Calls take pieces of one half until it is full; an event then marks the work that reads it,
    // and the other half is used once its own event has passed.  (An event a call costs the stream as much as a launch.)
    char *h_stage = nullptr, *h_stage_dev = nullptr;
    char *d_stage = nullptr;                // as large, where the pinned memory is not mapped, and for asks
    size_t half_bytes = 0, at = 0;          // at: of the half in use
    int half = 0;
    hipEvent_t ev[2] = {};
    bool ev_live[2] = {};
    alignas(16) char few[CACHE_FEW_BYTES];
    alignas(16) char lean[LEAN_ASKS * sizeof(CacheAsk) + 4 * (LEAN_ASKS + 1) * sizeof(int32_t)];      // asks before they go into `few`
    std::vector<char> list;                 // a list before it goes into a launch's arguments or to the device
    char err[512] = "";
};

namespace {

size_t outs_bytes(size_t n) { return n * sizeof(CacheOut) + (n + 1) * sizeof(int32_t); }
size_t attend_bytes(size_t n) { return n * sizeof(CacheAsk) + 4 * (n + 1) * sizeof(int32_t); }

aif_status cfail(aif_cache_ctx *c, aif_status st, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(c ? c->err : g_cache_init_error, 512, fmt, ap);
    va_end(ap);
    return st;
}

#define CACHE_TRY(ctxp, expr)                                                                         \
    do {                                                                                              \
        hipError_t e_ = (expr);                                                                       \
        if (e_ != hipSuccess)                                                                         \
            return cfail(ctxp, e_ == hipErrorOutOfMemory ? AIF_ENOMEM : AIF_EDEVICE, "%s: %s", #expr, \
                         hipGetErrorString(e_));                                                      \
    } while (0)

// What a call enqueues once its arguments are found right: an error of any kind is the device's.
#define CACHE_RUN(ctxp, expr)                                                                         \
    do {                                                                                              \
        hipError_t e_ = (expr);                                                                       \
        if (e_ != hipSuccess) return cfail(ctxp, AIF_EDEVICE, "%s: %s", #expr, hipGetErrorString(e_)); \
    } while (0)

size_t bytes_of_page(const aif_cache_config *f)
{
    return (size_t)f->n_kv_heads * (f->page_len / CACHE_TILE) * cache_tile_bytes((f->d_head + CACHE_BLOCK - 1) / CACHE_BLOCK * CACHE_BLOCK);
}

aif_status check_config(const aif_cache_config *f)
{
    if (f->dtype != AIF_F32 && f->dtype != AIF_BF16) return cfail(nullptr, AIF_EINVAL, "unknown dtype %d", (int)f->dtype);
    if (f->n_heads <= 0 || f->n_kv_heads <= 0 || f->d_head <= 0) return cfail(nullptr, AIF_EINVAL, "non-positive head count or width");
    if (f->n_heads % f->n_kv_heads) return cfail(nullptr, AIF_ESHAPE, "n_heads %d is not a multiple of n_kv_heads %d", f->n_heads, f->n_kv_heads);
    if (f->n_heads > 65535) return cfail(nullptr, AIF_ESHAPE, "n_heads %d is above 65535", f->n_heads);
    const int vec = f->dtype == AIF_F32 ? 4 : 8;
    if (f->d_head % vec || f->d_head > CACHE_MAX_DP) return cfail(nullptr, AIF_ESHAPE, "d_head %d is not a multiple of %d up to %d", f->d_head, vec, CACHE_MAX_DP);
    if (f->page_len < CACHE_TILE || f->page_len > 1024 || f->page_len % CACHE_TILE)
        return cfail(nullptr, AIF_ESHAPE, "page_len %d is not a multiple of %d up to 1024", f->page_len, CACHE_TILE);
    if (bytes_of_page(f) > CACHE_MAX_PAGE) return cfail(nullptr, AIF_ESHAPE, "pages of %zu bytes are above %zu", bytes_of_page(f), CACHE_MAX_PAGE);
    return AIF_OK;
}

bool name_once(aif_cache_ctx *c, int seq)
{
    if (c->stamp[seq] == c->stamp_now) return false;
    c->stamp[seq] = c->stamp_now;
    return true;
}
void name_none(aif_cache_ctx *c)
{
    if (++c->stamp_now == 0) {
        std::fill(c->stamp.begin(), c->stamp.end(), 0u);
        c->stamp_now = 1;
    }
}

aif_status check_seq(aif_cache_ctx *c, const char *what, int i, int seq)
{
    if (seq < 0 || seq >= c->cfg.max_seqs) return cfail(c, AIF_ERANGE, "%s %d: sequence %d is outside 0..%d", what, i, seq, c->cfg.max_seqs - 1);
    return AIF_OK;
}

aif_status check_count(aif_cache_ctx *c, const void *array, int32_t n, int32_t most)
{
    if (n < 0 || (n > 0 && !array)) return cfail(c, AIF_EINVAL, "NULL array or negative count");
    if (n > most) return cfail(c, AIF_ERANGE, "%d entries, the context takes %d", n, most);
    return AIF_OK;
}

aif_status check_tensor(aif_cache_ctx *c, const char *what, int i, const void *p, int64_t stride, int width)
{
    const int vec = c->shape.dtype == 0 ? 4 : 8;
    if (!p) return cfail(c, AIF_EINVAL, "%s %d: NULL tensor pointer", what, i);
    if ((uintptr_t)p % 16 || stride % vec) return cfail(c, AIF_EINVAL, "%s %d: tensors and strides must be multiples of 16 bytes", what, i);
    if (stride != 0 && (stride < width || stride >= (int64_t)1 << 33)) return cfail(c, AIF_EINVAL, "%s %d: stride %lld below the row's %d, or 2^33 and above", what, i, (long long)stride, width);
    return AIF_OK;
}

// The device is the context's and the stream is not being captured.
aif_status check_stream(aif_cache_ctx *c, hipStream_t s)
{
    int cur = -1;
    CACHE_RUN(c, hipGetDevice(&cur));
    if (cur != c->device) return cfail(c, AIF_EDEVICE, "context belongs to device %d, current device is %d", c->device, cur);
    hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(s, &st) != hipSuccess) {       // the default stream while another one is captured
        (void)hipGetLastError();
        st = hipStreamCaptureStatusActive;
    }
    if (st != hipStreamCaptureStatusNone) return cfail(c, AIF_EINVAL, "the stream is being captured: this call cannot be");
    return AIF_OK;
}

// A piece of the pinned memory for descriptors that launches on s will read: its offset.
aif_status stage_take(aif_cache_ctx *c, size_t bytes, hipStream_t s, size_t &off)
{
    bytes = (bytes + 255) / 256 * 256;
    if (c->at + bytes > c->half_bytes) {
        CACHE_RUN(c, hipEventRecord(c->ev[c->half], s));
        c->ev_live[c->half] = true;
        const int other = c->half ^ 1;
        if (c->ev_live[other]) CACHE_RUN(c, hipEventSynchronize(c->ev[other]));
        c->ev_live[other] = false;
        c->half = other;
        c->at = 0;
    }
    off = (size_t)c->half * c->half_bytes + c->at;
    c->at += bytes;
    return AIF_OK;
}

// A list of descriptors on its way to a launch.  Up to CACHE_FEW_BYTES of a call travel in the kernel's arguments; more are
// cut into lists in pinned memory, where the blocks read them.
template <class T> class CacheBatch {
public:
    CacheBatch(aif_cache_ctx *c, size_t expected, hipStream_t s) : c_(c), s_(s), far_(expected * sizeof(T) > CACHE_FEW_BYTES)
    {
        room_ = far_ ? std::min(expected, CACHE_LIST_BYTES / sizeof(T)) : CACHE_FEW_BYTES / sizeof(T);
    }
    // go: launches the list
    template <class F> aif_status add(const T &t, F &&go)
    {
        if (n_ == (int)room_) {
            const aif_status st = send(go);
            if (st != AIF_OK) return st;
        }
        if (n_ == 0) {
            at_ = (T *)c_->few;
            if (far_) {
                const aif_status st = stage_take(c_, room_ * sizeof(T), s_, off_);
                if (st != AIF_OK) return st;
                at_ = (T *)(c_->h_stage + off_);
            }
        }
        at_[n_++] = t;
        return AIF_OK;
    }
    template <class F> aif_status send(F &&go)
    {
        if (n_ == 0) return AIF_OK;
        CacheList l{at_, nullptr, n_, (size_t)n_ * sizeof(T)};
        n_ = 0;
        if (far_) {
            // read by each of a descriptor's blocks -- k_cache_move: one for 16 KB of a page, k_cache_fill: one for 256 table entries -- from the pinned
            // memory itself where that is mapped: the launch of an upload costs more than it saves up to some 1,500 descriptors (forks of 220, 1,000 and 4,000
            // sequences 9.9, 23.9 and 76 us back to back, 12.7, 26.9 and 78.8 with one; of that on the device 6.2, 7.9 and 17.0, 8.2, 8.2 and 9.1; 100
            // pages of 2.2 MB moved 82 either way)
            l.dev = c_->h_stage_dev ? c_->h_stage_dev + off_ : c_->d_stage + off_;
            if (!c_->h_stage_dev) CACHE_RUN(c_, staging_upload(c_->h_stage, nullptr, off_, c_->d_stage + off_, l.bytes, s_));
        }
        CACHE_RUN(c_, go(l));
        return AIF_OK;
    }

private:
    aif_cache_ctx *c_;
    hipStream_t s_;
    bool far_;
    size_t room_, off_ = 0;
    T *at_ = nullptr;
    int n_ = 0;
};

// A list of which blocks look for their entry: in the arguments, or on the device.
template <class F> aif_status send_list(aif_cache_ctx *c, const char *h, int n, size_t bytes, hipStream_t s, F &&go)
{
    CacheList l{h, nullptr, n, bytes};
    if (bytes > CACHE_FEW_BYTES) {
        size_t off = 0;
        const aif_status st = stage_take(c, bytes, s, off);
        if (st != AIF_OK) return st;
        __builtin_memcpy(c->h_stage + off, h, bytes);
        CACHE_RUN(c, staging_upload(c->h_stage, c->h_stage_dev, off, c->d_stage + off, bytes, s));
        l.dev = c->d_stage + off;
    }
    CACHE_RUN(c, go(l));
    return AIF_OK;
}

// Rows that are appended, as runs of rows on pages that follow each other.
class CacheIns {
public:
    CacheIns(aif_cache_ctx *c, hipStream_t s) : c_(c), s_(s), ins_((CacheIn *)c->list.data()) {}
    aif_status add(const CacheIn &in)
    {
        if (n_ == ROOM || rows_ >= MOST) {
            const aif_status st = send();
            if (st != AIF_OK) return st;
        }
        ins_[n_++] = in;
        rows_ += in.n;
        return AIF_OK;
    }
    // whether the last run may become longer, and further rows for it
    bool open() const { return n_ && rows_ < MOST; }
    void more(int32_t rows) { ins_[n_ - 1].n += rows, rows_ += rows; }
    aif_status send()
    {
        if (n_ == 0) return AIF_OK;
        int32_t *first = (int32_t *)(ins_ + n_), units = 0;
        const int n = n_, pl = c_->cfg.page_len;
        for (int i = 0; i < n; ++i) {
            first[i] = units;
            units += unit_of_row(ins_[i].have + ins_[i].n - 1, pl) - unit_of_row(ins_[i].have, pl) + 1;
        }
        first[n] = units;
        n_ = rows_ = 0;
        return send_list(c_, (const char *)ins_, n, n * sizeof(CacheIn) + (n + 1) * sizeof(int32_t), s_,
                         [&](const CacheList &l) { return launch_cache_append(c_->shape, l, units, s_); });
    }

private:
    static constexpr int ROOM = CACHE_LIST_BYTES / (sizeof(CacheIn) + sizeof(int32_t)) - 1;
    static constexpr int MOST = 1 << 27;    // rows of a launch, about: units of 32 at least
    aif_cache_ctx *c_;
    hipStream_t s_;
    CacheIn *ins_;
    int n_ = 0, rows_ = 0;
};

// Pages that are copied, as runs of new ones that follow each other.
class CacheCopies {
public:
    CacheCopies(aif_cache_ctx *c, hipStream_t s) : c_(c), s_(s), runs_((CacheRun *)c->list.data()) {}
    aif_status add(int32_t src, int32_t dst, int32_t page)      // table entries, the new page (-1: none)
    {
        if (n_ && pages_ < MAX_UNITS) {
            CacheRun &r = runs_[n_ - 1];
            if (src == r.src + r.n && dst == r.dst + r.n && (page < 0 ? r.page < 0 : r.page >= 0 && page == r.page + r.n)) {
                ++r.n, ++pages_;
                return AIF_OK;
            }
        }
        if (n_ == ROOM || pages_ == MAX_UNITS) {
            const aif_status st = send();
            if (st != AIF_OK) return st;
        }
        runs_[n_++] = CacheRun{src, dst, page, 1};
        ++pages_;
        return AIF_OK;
    }
    aif_status send()
    {
        if (n_ == 0) return AIF_OK;
        int32_t *first = (int32_t *)(runs_ + n_);
        const int n = n_, pages = pages_;
        for (int i = 0, at = 0; i < n; at += runs_[i++].n) first[i] = at;
        first[n] = pages;
        n_ = pages_ = 0;
        return send_list(c_, (const char *)runs_, n, n * sizeof(CacheRun) + (n + 1) * sizeof(int32_t), s_,
                         [&](const CacheList &l) { return launch_cache_copy(c_->shape, l, pages, s_); });
    }

private:
    static constexpr int ROOM = CACHE_LIST_BYTES / (sizeof(CacheRun) + sizeof(int32_t)) - 1;
    aif_cache_ctx *c_;
    hipStream_t s_;
    CacheRun *runs_;
    int n_ = 0, pages_ = 0;
};

// The end of a call that changed the book: where the device failed it, it is not known what the device holds of the sequences that the call changed.
// They become empty, so that nobody reads it.
aif_status settled(aif_cache_ctx *c, aif_status st, const int32_t *seqs, int32_t n)
{
    if (st != AIF_OK)
        for (int i = 0; i < n; ++i) c->book.truncate(seqs[i], 0);
    return st;
}

void cdestroy(aif_cache_ctx *c)
{
    if (!c) return;
    if (c->shape.table) (void)hipFree(c->shape.table);
    if (c->part) (void)hipFree(c->part);
    if (c->d_stage) (void)hipFree(c->d_stage);
    if (c->h_stage) (void)hipHostFree(c->h_stage);
    for (hipEvent_t e : c->ev)
        if (e) (void)hipEventDestroy(e);
    delete c;
}

aif_status cinit(const aif_cache_config *f, void *pool, aif_cache_ctx *c)
{
    const aif_status st = check_config(f);
    if (st != AIF_OK) return st;
    if (f->n_pages <= 0 || f->max_seqs <= 0 || f->max_len <= 0 || f->max_requests <= 0 || f->max_queries <= 0)
        return cfail(nullptr, AIF_EINVAL, "non-positive size in aif_cache_config");
    if (f->max_len > CACHE_MAX_LEN) return cfail(nullptr, AIF_ESHAPE, "max_len %d is above %d", f->max_len, CACHE_MAX_LEN);
    if (f->max_requests > 65535) return cfail(nullptr, AIF_ESHAPE, "max_requests %d is above 65535", f->max_requests);
    if (!(f->scale >= 0.f && f->scale <= 2.35e38f)) return cfail(nullptr, AIF_EINVAL, "scale is negative or above 2.35e38");      // (its product with log2 e is finite)
    if (!pool || (uintptr_t)pool % 64) return cfail(nullptr, AIF_EINVAL, "the pool is NULL or not 64-byte aligned");
    c->cfg = *f;
    CacheShape &s = c->shape;
    s.pool = (char *)pool;
    s.page_bytes = aif_cache_page_bytes(f);
    s.n_heads = f->n_heads;
    s.n_kv = f->n_kv_heads;
    s.group = f->n_heads / f->n_kv_heads;
    s.d_head = f->d_head;
    s.dp = (f->d_head + CACHE_BLOCK - 1) / CACHE_BLOCK * CACHE_BLOCK;
    s.page_len = f->page_len;
    // row / group with group <= 2^16: magic = ceil(2^(32 + shift) / group) with 2^shift < group <= 2^(shift + 1), whose error, below group <= 2^(shift + 1), times
    // row < 2^31 stays below 2^(32 + shift)
    if (s.group > 1) {
        while ((2 << s.group_shift) < s.group) ++s.group_shift;
        s.group_magic = (uint32_t)(((1ull << (32 + s.group_shift)) + s.group - 1) / s.group);
    }
    const uint32_t tpp = f->page_len / CACHE_TILE;
    s.tpp_magic = tpp == 1 ? 0u : (uint32_t)(((1ull << 32) + tpp - 1) / tpp);
    s.dtype = f->dtype == AIF_F32 ? 0 : 1;
    s.scale = f->scale != 0.f ? f->scale : 1.0f / __builtin_sqrtf((float)f->d_head);
    s.pages_per_seq = (int)(((int64_t)f->max_len + f->page_len - 1) / f->page_len);
    if (s.pages_per_seq > CACHE_MAX_PAGES) return cfail(nullptr, AIF_ESHAPE, "max_len / page_len = %d pages of a sequence are above %d", s.pages_per_seq, CACHE_MAX_PAGES);
    const int64_t entries = (int64_t)f->max_seqs * s.pages_per_seq;
    if (entries > INT32_MAX / 2) return cfail(nullptr, AIF_ESHAPE, "max_seqs * max_len / page_len = %lld table entries are too many", (long long)entries);
    c->book.init(f->max_seqs, f->max_len, f->page_len, f->n_pages);
    c->stamp.assign(f->max_seqs, 0u);
    CACHE_TRY(nullptr, hipGetDevice(&c->device));
    CACHE_TRY(nullptr, hipMalloc((void **)&s.table, (size_t)entries * sizeof(int32_t)));
    int n_cu = 0;
    CACHE_TRY(nullptr, hipDeviceGetAttribute(&n_cu, hipDeviceAttributeMultiprocessorCount, c->device));
    if (n_cu > 0) c->n_cu = n_cu;
    CACHE_TRY(nullptr, hipMalloc((void **)&c->part, cache_part_floats(c->n_cu * PART_ROWS, s.dp) * sizeof(float)));
    c->list.resize(std::max(CACHE_LIST_BYTES, outs_bytes(f->max_requests)));
    c->half_bytes = (std::max(2 * CACHE_LIST_BYTES, 4 * attend_bytes(f->max_requests)) + 255) / 256 * 256;        // (a list of asks is one, whatever its length)
    CACHE_TRY(nullptr, staging_alloc(c->half_bytes * 2, &c->h_stage, &c->h_stage_dev));
    CACHE_TRY(nullptr, hipMalloc((void **)&c->d_stage, c->half_bytes * 2));
    for (hipEvent_t &e : c->ev) CACHE_TRY(nullptr, hipEventCreateWithFlags(&e, hipEventDisableTiming | hipEventDisableSystemFence));
    return AIF_OK;
}

}  // namespace

extern "C" {

size_t aif_cache_page_bytes(const aif_cache_config *f)
{
    if (!f || check_config(f) != AIF_OK) return 0;
    return bytes_of_page(f);
}

aif_status aif_cache_init(const aif_cache_config *cfg, void *pool, aif_cache_ctx **out)
{
    if (!cfg || !out) return cfail(nullptr, AIF_EINVAL, "NULL argument");
    aif_cache_ctx *c = new (std::nothrow) aif_cache_ctx();
    if (!c) return cfail(nullptr, AIF_ENOMEM, "out of host memory");
    aif_status st;
    try {
        st = cinit(cfg, pool, c);
    } catch (const std::exception &) {
        st = cfail(nullptr, AIF_ENOMEM, "out of host memory");
    }
    if (st != AIF_OK) {
        cdestroy(c);
        return st;
    }
    *out = c;
    return AIF_OK;
}

void aif_cache_destroy(aif_cache_ctx *ctx) { cdestroy(ctx); }

const char *aif_cache_last_error(const aif_cache_ctx *ctx) { return ctx ? ctx->err : g_cache_init_error; }

int32_t aif_cache_len(const aif_cache_ctx *ctx, int32_t seq) { return !ctx || seq < 0 || seq >= ctx->cfg.max_seqs ? -1 : ctx->book.len(seq); }

int32_t aif_cache_free_pages(const aif_cache_ctx *ctx) { return ctx ? ctx->book.n_free : -1; }

aif_status aif_cache_append(aif_cache_ctx *c, const aif_cache_append_req *reqs, int32_t n, void *hip_stream)
{
    if (!c) return AIF_EINVAL;
    aif_status st = check_count(c, reqs, n, c->cfg.max_requests);
    if (st != AIF_OK) return st;
    const int width = c->shape.n_kv * c->shape.d_head, pl = c->cfg.page_len;
    int64_t pages = 0;
    name_none(c);
    for (int r = 0; r < n; ++r) {
        const aif_cache_append_req &q = reqs[r];
        if ((st = check_seq(c, "append", r, q.seq)) != AIF_OK) return st;
        if (!name_once(c, q.seq)) return cfail(c, AIF_EINVAL, "append %d: sequence %d is named twice", r, q.seq);
        if (q.n_rows < 0) return cfail(c, AIF_EINVAL, "append %d: negative n_rows", r);
        if (q.n_rows > 0 && ((st = check_tensor(c, "append", r, q.keys, q.key_stride, width)) != AIF_OK ||
                             (st = check_tensor(c, "append", r, q.vals, q.val_stride, width)) != AIF_OK))
            return st;
        const int len = c->book.len(q.seq);
        if (q.n_rows > c->cfg.max_len - len) return cfail(c, AIF_ERANGE, "append %d: %d rows behind %d exceed max_len %d", r, q.n_rows, len, c->cfg.max_len);
        pages += c->book.append_needs(q.seq, q.n_rows);
    }
    if (pages > c->book.n_free) return cfail(c, AIF_ERANGE, "%lld pages needed, %d are free", (long long)pages, c->book.n_free);
    hipStream_t s = (hipStream_t)hip_stream;
    if ((st = check_stream(c, s)) != AIF_OK) return st;

    const int64_t esz = c->shape.dtype == 0 ? 4 : 2;
    CacheIns ins(c, s);
    for (int r = 0; r < n && st == AIF_OK; ++r) {
        const aif_cache_append_req &q = reqs[r];
        const int64_t ks = (q.key_stride ? q.key_stride : width) * esz, vs = (q.val_stride ? q.val_stride : width) * esz;
        const int have = c->book.len(q.seq);
        int32_t next = -1;              // the page that would go on with the last run
        c->book.append(q.seq, q.n_rows, pl, [&](int32_t done, int32_t i, int32_t cow, int32_t, int32_t rows) {
            const int32_t page = c->book.page(q.seq, i);
            if (st != AIF_OK) return;
            if (page == next && ins.open()) ins.more(rows);
            else st = ins.add(CacheIn{(const char *)q.keys + done * ks, (const char *)q.vals + done * vs, (uint32_t)(ks / 16), (uint32_t)(vs / 16), c->book.entry(q.seq, 0),
                                      have + done, rows, page, cow, 0});
            next = page + 1;
        });
    }
    if (st == AIF_OK) st = ins.send();
    c->book.settle();
    for (int r = 0; st != AIF_OK && r < n; ++r) c->book.truncate(reqs[r].seq, 0);       // (settled)
    return st;
}

aif_status aif_cache_read(aif_cache_ctx *c, const aif_cache_read_req *reqs, int32_t n, void *hip_stream)
{
    if (!c) return AIF_EINVAL;
    aif_status st = check_count(c, reqs, n, c->cfg.max_requests);
    if (st != AIF_OK) return st;
    const int width = c->shape.n_kv * c->shape.d_head, pl = c->cfg.page_len;
    int64_t units = 0;
    int n_out = 0;
    for (int r = 0; r < n; ++r) {
        const aif_cache_read_req &q = reqs[r];
        if ((st = check_seq(c, "read", r, q.seq)) != AIF_OK) return st;
        if (q.n_rows < 0 || q.first < 0 || q.reserved) return cfail(c, AIF_EINVAL, "read %d: negative rows, or reserved is not 0", r);
        if (q.first > c->book.len(q.seq) || q.n_rows > c->book.len(q.seq) - q.first)
            return cfail(c, AIF_ERANGE, "read %d: rows %d.. of %d, the sequence has %d", r, q.first, q.n_rows, c->book.len(q.seq));
        if (q.n_rows == 0) continue;
        if ((q.keys_out && (st = check_tensor(c, "read", r, q.keys_out, q.key_stride, width)) != AIF_OK) ||
            (q.vals_out && (st = check_tensor(c, "read", r, q.vals_out, q.val_stride, width)) != AIF_OK))
            return st;
        for (int p = q.first / pl; p <= (q.first + q.n_rows - 1) / pl; ++p)
            if (c->book.page(q.seq, p) < 0) return cfail(c, AIF_ERANGE, "read %d: rows from %d on were dropped", r, p * pl);
        if (!q.keys_out && !q.vals_out) continue;
        units += unit_of_row(q.first + q.n_rows - 1, pl) - unit_of_row(q.first, pl) + 1;
        ++n_out;
    }
    if (units > 2 * MAX_UNITS) return cfail(c, AIF_ERANGE, "rows in %lld pieces of pages in one call are too many", (long long)units);
    hipStream_t s = (hipStream_t)hip_stream;
    if ((st = check_stream(c, s)) != AIF_OK) return st;
    CacheOut *out = (CacheOut *)c->list.data();
    int32_t *first = (int32_t *)(out + n_out), at = 0;
    for (int r = 0; r < n; ++r) {
        const aif_cache_read_req &q = reqs[r];
        if (q.n_rows == 0 || (!q.keys_out && !q.vals_out)) continue;
        *first++ = at;
        *out++ = CacheOut{(char *)q.keys_out, (char *)q.vals_out, q.key_stride ? q.key_stride : width, q.val_stride ? q.val_stride : width,
                          c->book.entry(q.seq, 0), q.first, q.n_rows, 0};
        at += unit_of_row(q.first + q.n_rows - 1, pl) - unit_of_row(q.first, pl) + 1;
    }
    *first = at;
    if (n_out == 0) return AIF_OK;
    return send_list(c, c->list.data(), n_out, outs_bytes(n_out), s, [&](const CacheList &l) { return launch_cache_read(c->shape, l, at, s); });
}

// How a call's work is cut: into tiles of rows (a row is a query and a head of a kv head's group) and, where that pays, splits of their keys.
//
// Which kernel.  The one for few rows has tiles of 16 or 32 (fp32: 16, a query's three pieces take the registers), whose keys four waves share; the others
// have tiles of 128, or 256 for bf16 heads of up to 128 and two of them for each compute unit.  The small tiles are the quicker ones as long as
// they do not queue: up to ROWS_OF_CU rows for a compute unit in the whole call (32 users x 256 queries, two heads of 128 over 800 keys 30 us, 36 in
// tiles of 128; of 512 queries 57 and 37).  The price is one user's
// long prompt: 16,000 queries over 10^5 keys, a head of 64: 820 us, 655.  In larger calls only entries of up to FEW_ROWS rows go there.
//
// Many rows: heads of up to 32 features, and fp32 up to 64, are the cheapest to bring to bf16 once a wave (8 x 10^4 rows of 8 heads of 16 over 2,000 keys 255
// us, 276 once a block); up to 64 that also serves few row tiles, whose blocks wait for nobody, and rows that see each a window of its
// own, of which a wave's span is less than a block's (replayed impressions 31 us, 48).
//
// Splits.  A second launch joins their results, so they must save more than that costs.  The estimate: a tile of rows takes `tile` us for each 32 keys, blocks of
// one compute unit beside each other 0.8 times that each; a join takes 4 us, and its floats go and come at 1.8 TB/s.  (tile, from unsplit calls
// over 800 and 3,000 keys: 32 bf16 rows of heads of 32, 64, 128, 256: 0.14, 0.18, 0.25, 0.40; 128 rows: 0.47, 0.57, 1.06, 2.0.)  Of seven
// ways to cut, the least is taken: 128 users x 64 queries, a head of 64 over 800 keys 14.4 us unsplit and 30 in eights; over 3,000 keys of four
// users 23.6 unsplit, 12 in eights.
//
// Waves.  Eight to a block of few rows take 0.62 times as long for a tile, but start and end later and are worth less beside another block (32 users x 128
// queries, two heads of 128: over 200 keys 11.2 us with eight and 9.6 with four, over 800 14.0 and 16.4, over 3,000 25.3 and 33.5; 512 queries, a head
// of 64 over 800 keys 18.7 and 15.2).  Heads above 128 have no registers for it.  Where
// memory alone counts they are about even: one query of each of 16 users, four heads over 3.3 to 6.7 MB a compute unit takes eight waves 0.95 to 1.04 of four's time with
// heads of 128, 0.97 to 1.01 with heads of 64 and 0.99 to 1.01 with heads of 32.
//
// Partial results have room for PART_ROWS rows a compute unit: keys / chunk is rounded, by a third up at most where that makes two or
// more, and tiles * keys / chunk <= work / chunk <= 3 / 4 of the room.
static bool plan_attend(aif_cache_ctx *c, CacheAsk *asks, int n, int32_t *arrays, CachePlan &plan, size_t &bytes)
{
    const CacheShape &sh = c->shape;
    auto rows_of = [&](const CacheAsk &a) { return (int64_t)a.n_q * sh.group; };
    auto keys_of = [&](const CacheAsk &a, int rows) {       // tiles of keys that a tile of so many rows sees, about: positions are taken to be spread evenly
        int64_t keys = a.len;
        if (a.window) keys = std::min<int64_t>(a.len, (int64_t)a.window + std::min(a.sinks, a.len) + (a.pos && a.n_q > 1 ? a.len * std::min<int64_t>(rows, rows_of(a)) / rows_of(a) : 0));
        return (keys + CACHE_TILE - 1) / CACHE_TILE;
    };
    bytes = (size_t)n * sizeof(CacheAsk);
    int64_t call_rows = 0;
    for (int r = 0; r < n; ++r) call_rows += rows_of(asks[r]) * sh.n_kv;
    const bool all_few = call_rows <= (int64_t)ROWS_OF_CU * c->n_cu;
    for (int kind = 0; kind < 2; ++kind) {
        CachePart &p = kind ? plan.many : plan.few;
        auto mine = [&](const CacheAsk &a) { return a.n_q > 0 && (!all_few && rows_of(a) > FEW_ROWS) == (kind == 1); };
        int64_t most = 0, wide = 0;
        bool windows = false;
        for (int r = 0; r < n; ++r)
            if (mine(asks[r])) most = std::max(most, rows_of(asks[r])), wide += (rows_of(asks[r]) + 255) / 256 * sh.n_kv, windows |= asks[r].pos && asks[r].window;
        if (most == 0) continue;
        const int rows = p.rows_of_tile = kind ? (sh.dtype == 1 && sh.dp <= 128 && wide >= 2 * c->n_cu ? 256 : 128) : (sh.dtype == 0 || most <= 16 ? 16 : 32);
        p.own = kind && sh.dp <= 64 && (sh.dp == 32 || sh.dtype == 0 || rows == 128 || windows);
        const int64_t room = (int64_t)c->n_cu * PART_ROWS / rows;
        auto tiles_of = [&](const CacheAsk &a) { return (rows_of(a) + rows - 1) / rows; };
        int64_t work = 0, all = 0, valid = 0, longest = 0, units = 0, joined = 0, parts = 0, most_units = 0;
        for (int r = 0; r < n; ++r)
            if (mine(asks[r])) {
                const int64_t keys = keys_of(asks[r], rows);
                work += tiles_of(asks[r]) * keys * sh.n_kv, all += tiles_of(asks[r]) * sh.n_kv, valid += rows_of(asks[r]) * sh.n_kv, longest = std::max(longest, keys);
            }
        const double tile = kind ? (0.1 + 0.0075 * sh.dp) * (sh.dtype == 0 ? 1.5 : 1.0) * (rows == 256 ? 1.7 : 1.0)
                                 : (0.1 + 0.0012 * sh.dp) * (sh.dtype == 1 && rows == 16 ? 0.72 : 1.0);
        const double row_of_part = sh.dp * 8 / 1.8e6;
        int64_t chunk = std::max<int64_t>(longest, 1);
        double best = 0;
        const bool may = kind == 0 && sh.dp <= 128;
        for (int eight = 0; eight <= may; ++eight) {
            const double start = eight ? (sh.dtype == 0 ? 1.5 : 0.8) : 0.0, one = eight ? 0.62 * tile : tile, beside = eight ? 1.37 : 0.8;
            auto time = [&](int64_t k, int64_t cut) {           // cut: blocks, of up to k tiles
                const int64_t load = (cut + c->n_cu - 1) / c->n_cu;
                return start + one * std::max((double)k, (load > 1 ? beside * load : 1.0) * work / cut);
            };
            double t = time(longest, all);
            if (!eight || t < best) best = t, chunk = std::max<int64_t>(longest, 1), p.eight = eight;
            for (int m = 1; m <= 32; m *= 2) {                  // so many eighths of the compute units' number
                const int64_t blocks = std::min<int64_t>(room * 3 / 4, (int64_t)c->n_cu * m / 8);
                const int64_t k = std::max<int64_t>(MIN_TILES, (work + blocks - 1) / blocks);
                if (k >= longest) continue;
                const int64_t cut = std::max(all, work / k);
                t = time(k, cut) + 4.0 + row_of_part * valid * cut / all;
                if (t < best) best = t, chunk = k, p.eight = eight;
            }
        }
        int32_t *first = arrays, *joins = arrays + n + 1;
        arrays += 2 * (n + 1);
        bytes += 2 * ((size_t)n + 1) * sizeof(int32_t);
        for (int r = 0; r < n; ++r) {
            CacheAsk &a = asks[r];
            first[r] = (int32_t)units;
            joins[r] = (int32_t)joined;
            if (!mine(a)) continue;
            const int64_t tiles = tiles_of(a);
            a.splits = (int32_t)std::min<int64_t>(std::max<int64_t>(1, (keys_of(a, rows) + (kind ? 0 : chunk / 2)) / chunk), MAX_SPLITS);
            a.part = (int32_t)parts;
            units += tiles * a.splits;
            most_units = std::max(most_units, tiles * a.splits);
            if (a.splits > 1) {
                joined += rows_of(a);
                parts += tiles * a.splits * sh.n_kv;
            }
            if (units > MAX_UNITS) return false;
        }
        first[n] = (int32_t)units;
        joins[n] = (int32_t)joined;
        p.units = (int32_t)units;
        p.joins = (int32_t)joined;
        // entries of as many units: a row of the grid each, in which a block need not look for its entry (empty blocks in the place of missing units leave
        // whole XCDs without work)
        p.each = most_units * n == units && most_units <= 65535 ? (int32_t)most_units : 0;
        p.part = c->part;
    }
    return true;
}

// Whether entries differ in nothing but their sequences and evenly spaced pointers.
static bool alike(const aif_cache_attend_req *q, int32_t n)
{
    for (int r = 1; r < n; ++r) {
        const aif_cache_attend_req &a = q[r], &b = q[r - 1], &z = q[0], &o = q[1];
        auto even = [](const void *x, const void *y, const void *first, const void *second) { return (uintptr_t)x - (uintptr_t)y == (uintptr_t)second - (uintptr_t)first; };
        if (a.n_q != z.n_q || a.q_stride != z.q_stride || a.out_stride != z.out_stride || a.sinks != z.sinks || a.window != z.window ||
            !a.lse_out != !z.lse_out || !a.positions != !z.positions || !even(a.q, b.q, z.q, o.q) || !even(a.out, b.out, z.out, o.out) ||
            !even(a.lse_out, b.lse_out, z.lse_out, o.lse_out) || !even(a.positions, b.positions, z.positions, o.positions))
            return false;
    }
    return true;
}

aif_status aif_cache_attend(aif_cache_ctx *c, const aif_cache_attend_req *reqs, int32_t n, void *hip_stream)
{
    if (!c) return AIF_EINVAL;
    aif_status st = check_count(c, reqs, n, c->cfg.max_requests);
    if (st != AIF_OK) return st;
    const int width = c->shape.n_heads * c->shape.d_head, esz = c->shape.dtype == 0 ? 4 : 2;
    int64_t rows = 0;
    for (int r = 0; r < n; ++r) {
        const aif_cache_attend_req &q = reqs[r];
        if ((st = check_seq(c, "attend", r, q.seq)) != AIF_OK) return st;
        if (q.n_q < 0 || q.sinks < 0 || q.window < 0) return cfail(c, AIF_EINVAL, "attend %d: negative n_q, sinks or window", r);
        if (q.n_q > c->cfg.max_queries) return cfail(c, AIF_ERANGE, "attend %d: n_q %d exceeds max_queries %d", r, q.n_q, c->cfg.max_queries);
        if (q.n_q > 0 && ((st = check_tensor(c, "attend", r, q.q, q.q_stride, width)) != AIF_OK ||
                          (st = check_tensor(c, "attend", r, q.out, q.out_stride, width)) != AIF_OK))
            return st;
        if (((uintptr_t)q.lse_out | (uintptr_t)q.positions) % 4) return cfail(c, AIF_EINVAL, "attend %d: lse_out and positions must be 4-byte aligned", r);
        rows += (int64_t)q.n_q * c->shape.group;
    }
    if (rows > INT32_MAX) return cfail(c, AIF_ERANGE, "%lld rows (queries times heads of a kv head) in one call are too many", (long long)rows);
    hipStream_t s = (hipStream_t)hip_stream;
    if ((st = check_stream(c, s)) != AIF_OK) return st;
    if (rows == 0) return AIF_OK;

    // The descriptors go into the arguments as they are; or as what they have in common and what they have not; or are uploaded.
    bool far = attend_bytes((size_t)n) > CACHE_FEW_BYTES;
    const bool lean = far && n <= LEAN_ASKS && alike(reqs, n);
    size_t bytes = 0;
    size_t off = 0;
    char *h = lean ? c->lean : c->few;
    if (far && !lean) {
        if ((st = stage_take(c, attend_bytes((size_t)n), s, off)) != AIF_OK) return st;
        h = c->h_stage + off;
    }
    CacheAsk *ha = (CacheAsk *)h;
    for (int r = 0; r < n; ++r) {
        const aif_cache_attend_req &q = reqs[r];
        ha[r] = CacheAsk{(const char *)q.q, (char *)q.out, q.lse_out, q.positions, (q.q_stride ? q.q_stride : width) * esz,
                         (q.out_stride ? q.out_stride : width) * esz, q.n_q, c->book.len(q.seq), q.sinks, q.window, c->book.entry(q.seq, 0), 1, 0, 0};
    }
    CachePlan plan{};
    if (!plan_attend(c, ha, n, (int32_t *)(ha + n), plan, bytes)) return cfail(c, AIF_ERANGE, "one call has too many queries");
    CacheList l{h, nullptr, n, bytes};
    if (lean) {
        const size_t numbers = bytes - n * sizeof(CacheAsk), asks = cache_asks_bytes(n, true);
        far = asks + numbers > CACHE_FEW_BYTES;
        if (far) {
            if ((st = stage_take(c, bytes, s, off)) != AIF_OK) return st;
            __builtin_memcpy(c->h_stage + off, h, bytes);
        } else {
            auto step = [&](auto f) { return n > 1 ? (int64_t)((uintptr_t)f(ha[1]) - (uintptr_t)f(ha[0])) : 0; };
            *(CacheLean *)c->few = CacheLean{ha[0], step([](const CacheAsk &a) { return a.q; }), step([](const CacheAsk &a) { return a.out; }),
                                             step([](const CacheAsk &a) { return a.lse; }), step([](const CacheAsk &a) { return a.pos; })};
            CacheOwn *own = (CacheOwn *)(c->few + sizeof(CacheLean));
            for (int r = 0; r < n; ++r) own[r] = CacheOwn{ha[r].len, ha[r].entry, ha[r].splits, ha[r].part};
            __builtin_memcpy(c->few + asks, ha + n, numbers);
            l = CacheList{c->few, nullptr, n, asks + numbers, true};
        }
    }
    if (far) {
        CACHE_RUN(c, staging_upload(c->h_stage, c->h_stage_dev, off, c->d_stage + off, bytes, s));
        l.dev = c->d_stage + off;
    }
    CACHE_RUN(c, launch_cache_attend(c->shape, l, plan, s));
    return AIF_OK;
}

// what fork and copy ask of their arguments
static aif_status check_branches(aif_cache_ctx *c, const char *what, const int32_t *src, const int32_t *dst, int32_t n)
{
    aif_status st = check_count(c, src, n, c->cfg.max_seqs);
    if (st == AIF_OK) st = check_count(c, dst, n, c->cfg.max_seqs);
    if (st != AIF_OK) return st;
    name_none(c);
    for (int i = 0; i < n; ++i) {
        if ((st = check_seq(c, what, i, src[i])) != AIF_OK || (st = check_seq(c, what, i, dst[i])) != AIF_OK) return st;
        if (c->book.len(dst[i])) return cfail(c, AIF_EINVAL, "%s %d: sequence %d is not empty", what, i, dst[i]);
        if (!name_once(c, dst[i])) return cfail(c, AIF_EINVAL, "%s %d: sequence %d is named twice", what, i, dst[i]);
    }
    for (int i = 0; i < n; ++i)
        if (c->stamp[src[i]] == c->stamp_now) return cfail(c, AIF_EINVAL, "%s %d: sequence %d is source and destination", what, i, src[i]);
    return AIF_OK;
}

aif_status aif_cache_fork(aif_cache_ctx *c, const int32_t *src, const int32_t *dst, int32_t n, void *hip_stream)
{
    if (!c) return AIF_EINVAL;
    aif_status st = check_branches(c, "fork", src, dst, n);
    if (st != AIF_OK) return st;
    hipStream_t s = (hipStream_t)hip_stream;
    if ((st = check_stream(c, s)) != AIF_OK) return st;
    int longest = 0;
    for (int i = 0; i < n; ++i) longest = std::max(longest, c->book.pages(c->book.len(src[i])));
    CacheBatch<CacheFill> batch(c, (size_t)n, s);
    auto go = [&](const CacheList &l) { return launch_cache_fill(c->shape, l, longest, s); };
    for (int i = 0; i < n && st == AIF_OK; ++i) {
        c->book.fork(src[i], dst[i]);
        const int np = c->book.pages(c->book.len(src[i]));
        if (np) st = batch.add(CacheFill{c->book.entry(dst[i], 0), np, c->book.entry(src[i], 0), 0}, go);
    }
    return settled(c, st == AIF_OK ? batch.send(go) : st, dst, n);
}

aif_status aif_cache_copy(aif_cache_ctx *c, const int32_t *src, const int32_t *dst, int32_t n, void *hip_stream)
{
    if (!c) return AIF_EINVAL;
    aif_status st = check_branches(c, "copy", src, dst, n);
    if (st != AIF_OK) return st;
    int64_t pages = 0;
    for (int i = 0; i < n; ++i) pages += c->book.copy_needs(src[i]);
    if (pages > c->book.n_free) return cfail(c, AIF_ERANGE, "%lld pages needed, %d are free", (long long)pages, c->book.n_free);
    hipStream_t s = (hipStream_t)hip_stream;
    if ((st = check_stream(c, s)) != AIF_OK) return st;
    CacheCopies copies(c, s);
    for (int i = 0; i < n && st == AIF_OK; ++i)
        c->book.copy(src[i], dst[i], [&](int32_t p, int32_t, int32_t to) {
            if (st == AIF_OK) st = copies.add(c->book.entry(src[i], p), c->book.entry(dst[i], p), to);
        });
    return settled(c, st == AIF_OK ? copies.send() : st, dst, n);
}

aif_status aif_cache_free(aif_cache_ctx *c, const int32_t *seqs, int32_t n)
{
    if (!c) return AIF_EINVAL;
    aif_status st = check_count(c, seqs, n, INT32_MAX);
    if (st != AIF_OK) return st;
    for (int i = 0; i < n; ++i)
        if ((st = check_seq(c, "free", i, seqs[i])) != AIF_OK) return st;
    for (int i = 0; i < n; ++i) c->book.truncate(seqs[i], 0);
    return AIF_OK;
}

aif_status aif_cache_truncate(aif_cache_ctx *c, int32_t seq, int32_t len)
{
    if (!c) return AIF_EINVAL;
    aif_status st = check_seq(c, "truncate", 0, seq);
    if (st != AIF_OK) return st;
    if (len < 0 || len > c->book.len(seq)) return cfail(c, AIF_ERANGE, "truncate: length %d of %d", len, c->book.len(seq));
    if (!c->book.truncate(seq, len)) return cfail(c, AIF_ERANGE, "truncate: row %d lies in a page that was dropped", len);
    return AIF_OK;
}

aif_status aif_cache_trim(aif_cache_ctx *c, const int32_t *seqs, int32_t n, int32_t sinks, int32_t window, void *hip_stream)
{
    if (!c) return AIF_EINVAL;
    aif_status st = check_count(c, seqs, n, INT32_MAX);
    if (st != AIF_OK) return st;
    if (sinks < 0 || window < 1) return cfail(c, AIF_EINVAL, "trim: sinks %d, window %d", sinks, window);
    for (int i = 0; i < n; ++i)
        if ((st = check_seq(c, "trim", i, seqs[i])) != AIF_OK) return st;
    hipStream_t s = (hipStream_t)hip_stream;
    if ((st = check_stream(c, s)) != AIF_OK) return st;
    CacheBatch<CacheFill> batch(c, (size_t)n, s);
    int longest = 0;
    for (int i = 0; i < n; ++i) longest = std::max(longest, c->book.pages(c->book.len(seqs[i])));
    auto go = [&](const CacheList &l) { return launch_cache_fill(c->shape, l, longest, s); };
    for (int i = 0; i < n && st == AIF_OK; ++i) {
        int lo, hi;
        c->book.trim(seqs[i], sinks, window, lo, hi);
        if (lo < hi) st = batch.add(CacheFill{c->book.entry(seqs[i], lo), hi - lo, -1, -1}, go);
    }
    return settled(c, st == AIF_OK ? batch.send(go) : st, seqs, n);
}

aif_status aif_cache_compact(aif_cache_ctx *c, int32_t *n_used, void *hip_stream)
{
    if (!c) return AIF_EINVAL;
    hipStream_t s = (hipStream_t)hip_stream;
    aif_status st = check_stream(c, s);
    if (st != AIF_OK) return st;
    const int64_t pages = c->book.out_of_place();
    if (pages) {
        // contents and names in one list: a page is copied before its new number is read, by launches that come later
        CacheBatch<CacheMove> batch(c, (size_t)pages * 2, s);
        auto go = [&](const CacheList &l) { return launch_cache_move(c->shape, l, s); };
        c->book.compact([&](int32_t from, int32_t to) { if (st == AIF_OK) st = batch.add(CacheMove{from, to, -1}, go); },
                        [&](int32_t q, int32_t i, int32_t to) { if (st == AIF_OK) st = batch.add(CacheMove{-1, to, c->book.entry(q, i)}, go); });
        if (st == AIF_OK) st = batch.send(go);
        for (int32_t q = 0; st != AIF_OK && q < c->cfg.max_seqs; ++q) c->book.truncate(q, 0);        // (settled)
    }
    if (n_used) *n_used = c->book.n_pages - c->book.n_free;
    return st;
}

aif_status aif_cache_swap_pool(aif_cache_ctx *c, void *pool, int32_t n_pages)
{
    if (!c) return AIF_EINVAL;
    if (!pool || (uintptr_t)pool % 64 || n_pages < 1) return cfail(c, AIF_EINVAL, "the pool is NULL or not 64-byte aligned, or has no pages");
    try {
        if (!c->book.set_pool(n_pages)) return cfail(c, AIF_ERANGE, "a page at or beyond %d is in use", n_pages);
    } catch (const std::exception &) {
        return cfail(c, AIF_ENOMEM, "out of host memory");
    }
    c->shape.pool = (char *)pool;
    return AIF_OK;
}

}  // extern "C"
