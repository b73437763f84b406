// The host side of the user cache, csrc/aif_cache_api.hip, over a device that is a queue on this machine: launches, copies and events wait in it until
// an event of theirs is waited for or the test runs it, and a row on a page is the addresses that its key and value were given by.  What a
// launch reads from memory it reads when its turn comes, so that a descriptor overwritten too early shows.
#include "aif_cache_api.hip"

#include <cstdlib>
#include <cstring>
#include <deque>
#include <functional>
#include <map>

using namespace aif;

namespace {
struct Row {
    int64_t key, val;
};
std::deque<std::function<void()>> queue_;
long long queued, done;
std::map<void *, size_t> sizes;                 // of allocations
std::map<hipEvent_t, long long> recorded;
std::vector<std::vector<Row>> pages;
std::map<int64_t, std::vector<int64_t>> results;    // by output address
bool mapped;
long long calls, fail_at;                       // HIP calls on the stream so far; the one that fails
hipError_t fail_with;
char wrong[256];                                // the first thing that no call should have done

void complain(const char *what)
{
    if (!wrong[0]) snprintf(wrong, sizeof wrong, "%s", what);
}
void run_to(long long n)
{
    for (; done < n; ++done) {
        queue_.front()();
        queue_.pop_front();
    }
}
bool fails() { return ++calls == fail_at; }
hipError_t push(std::function<void()> f)
{
    if (fails()) return fail_with;
    queue_.push_back(std::move(f));
    ++queued;
    return hipSuccess;
}
Row &row(int page, int i)
{
    if (page < 0 || page >= (int)pages.size()) {
        complain("a page outside the pool");
        static Row none;
        return none;
    }
    return pages[page][i];
}
// a launch of `run`, which gets the descriptors as they are when it runs
hipError_t launch(const CacheList &l, std::function<void(const char *)> run)
{
    if (l.bytes > CACHE_FEW_BYTES && !l.dev) complain("more in the arguments than they hold");
    if (l.dev) return push([run, dev = l.dev] { run(dev); });
    std::vector<char> copy((const char *)l.host, (const char *)l.host + l.bytes);
    return push([run, copy = std::move(copy)] { run(copy.data()); });
}
void numbered(const int32_t *first, int n, int units)
{
    for (int i = 0; i < n; ++i)
        if (first[i] < 0 || first[i] > first[i + 1]) complain("running numbers that fall");
    if (first[0] != 0 || first[n] != units) complain("running numbers that do not end where the launch does");
    if (units > 2 * MAX_UNITS) complain("a grid of too many blocks");
}
}  // namespace

namespace aif {
hipError_t launch_cache_append(const CacheShape &c, const CacheList &l, int units, hipStream_t)
{
    return launch(l, [=](const char *p) {
        const CacheIn *ins = (const CacheIn *)p;
        numbered((const int32_t *)(ins + l.n), l.n, units);
        for (int i = 0; i < l.n; ++i) {
            const CacheIn &u = ins[i];
            if (u.cow >= 0)
                for (int r = 0; r < u.have % c.page_len; ++r) row(u.page, r) = row(u.cow, r);
            for (int r = u.have; r < u.have + u.n; ++r) {
                const int page = u.page + r / c.page_len - u.have / c.page_len;
                row(page, r % c.page_len) = Row{(int64_t)u.keys + (r - u.have) * (int64_t)u.key_stride * 16, (int64_t)u.vals + (r - u.have) * (int64_t)u.val_stride * 16};
                c.table[u.entry + r / c.page_len] = page;
            }
        }
    });
}
hipError_t launch_cache_read(const CacheShape &c, const CacheList &l, int units, hipStream_t)
{
    return launch(l, [=](const char *p) {
        const CacheOut *outs = (const CacheOut *)p;
        numbered((const int32_t *)(outs + l.n), l.n, units);
        for (int i = 0; i < l.n; ++i)
            for (int r = outs[i].first; r < outs[i].first + outs[i].n; ++r) {
                const Row &x = row(c.table[outs[i].entry + r / c.page_len], r % c.page_len);
                if (outs[i].keys) results[(int64_t)outs[i].keys].push_back(x.key);
                if (outs[i].vals) results[(int64_t)outs[i].vals].push_back(x.val);
            }
    });
}
hipError_t launch_cache_copy(const CacheShape &c, const CacheList &l, int n_pages, hipStream_t)
{
    return launch(l, [=](const char *p) {
        const CacheRun *runs = (const CacheRun *)p;
        numbered((const int32_t *)(runs + l.n), l.n, n_pages);
        for (int i = 0; i < l.n; ++i)
            for (int k = 0; k < runs[i].n; ++k) {
                c.table[runs[i].dst + k] = runs[i].page < 0 ? -1 : runs[i].page + k;
                if (runs[i].page >= 0)
                    for (int r = 0; r < c.page_len; ++r) row(runs[i].page + k, r) = row(c.table[runs[i].src + k], r);
            }
    });
}
hipError_t launch_cache_fill(const CacheShape &c, const CacheList &l, int longest, hipStream_t)
{
    return launch(l, [=](const char *p) {
        for (int i = 0; i < l.n; ++i) {
            const CacheFill &f = ((const CacheFill *)p)[i];
            if (f.n > longest) complain("a run of table entries longer than the grid");
            for (int k = 0; k < f.n; ++k) c.table[f.dst + k] = f.src < 0 ? f.value : c.table[f.src + k];
        }
    });
}
hipError_t launch_cache_move(const CacheShape &c, const CacheList &l, hipStream_t)
{
    return launch(l, [=](const char *p) {
        for (int i = 0; i < l.n; ++i) {
            const CacheMove &m = ((const CacheMove *)p)[i];
            if (m.entry >= 0) c.table[m.entry] = m.dst;
            if (m.src >= 0)
                for (int r = 0; r < c.page_len; ++r) row(m.dst, r) = row(m.src, r);
        }
    });
}
hipError_t launch_cache_attend(const CacheShape &c, const CacheList &l, const CachePlan &plan, hipStream_t)
{
    return launch(l, [=](const char *p) {
        const int32_t *numbers = (const int32_t *)(p + cache_asks_bytes(l.n, l.lean));
        const CachePart *parts[2] = {&plan.few, &plan.many};
        auto ask = [&](int i) {
            if (!l.lean) return ((const CacheAsk *)p)[i];
            const CacheLean &z = *(const CacheLean *)p;
            const CacheOwn &o = ((const CacheOwn *)(p + sizeof(CacheLean)))[i];
            CacheAsk a = z.a;
            a.out += i * z.out_step;
            a.len = o.len, a.entry = o.entry, a.splits = o.splits, a.part = o.part;
            return a;
        };
        for (const CachePart *of : parts) {
            if (of->units == 0) continue;
            const int32_t *joins = numbers + l.n + 1;
            numbered(numbers, l.n, of->units);
            numbered(joins, l.n, of->joins);
            int64_t next = 0;
            for (int i = 0; i < l.n; ++i) {
                const CacheAsk a = ask(i);
                const int units = numbers[i + 1] - numbers[i];
                if (units == 0) continue;
                const int64_t rows = (int64_t)a.n_q * c.group, tiles = (rows + of->rows_of_tile - 1) / of->rows_of_tile;
                if (units != tiles * a.splits || a.splits < 1 || a.splits > 128) complain("an entry of other units than its tiles and splits");
                if (of->each && of->each != units) complain("an entry of other units than the grid has");
                if (joins[i + 1] - joins[i] != (a.splits > 1 ? rows : 0)) complain("an entry of other joins than its rows");
                if (a.splits == 1) continue;
                if (a.part != next) complain("partial results that overlap or leave gaps");
                next += tiles * a.splits * c.n_kv;
            }
            if (next * cache_part_floats(of->rows_of_tile, c.dp) * sizeof(float) > sizes[of->part]) complain("partial results beyond their room");
            numbers += 2 * (l.n + 1);
        }
        for (int i = 0; i < l.n; ++i) {
            const CacheAsk a = ask(i);
            if (a.n_q == 0) continue;
            std::vector<int64_t> &seen = results[(int64_t)a.out];
            for (int r = 0; r < a.len; ++r) {
                const int page = c.table[a.entry + r / c.page_len];
                seen.push_back(page < 0 ? -1 : row(page, r % c.page_len).key);
            }
        }
    });
}
hipError_t staging_alloc(size_t bytes, char **host, char **dev)
{
    *host = (char *)calloc(1, bytes);
    *dev = mapped ? *host : nullptr;
    sizes[*host] = bytes;
    return hipSuccess;
}
hipError_t staging_upload(const char *host, const char *, size_t off, void *dst, size_t bytes, hipStream_t)
{
    return push([=] { memcpy(dst, host + off, bytes); });
}
}  // namespace aif

extern "C" {
hipError_t hipGetDevice(int *d) { return *d = 0, hipSuccess; }
hipError_t hipMalloc(void **p, size_t n)
{
    *p = malloc(n);
    sizes[*p] = n;
    return hipSuccess;
}
static hipError_t give_back(void *p)
{
    sizes.erase(p);
    free(p);
    return hipSuccess;
}
hipError_t hipFree(void *p) { return give_back(p); }
hipError_t hipHostFree(void *p) { return give_back(p); }
hipError_t hipDeviceGetAttribute(int *v, hipDeviceAttribute_t, int) { return *v = 256, hipSuccess; }
hipError_t hipEventCreateWithFlags(hipEvent_t *e, unsigned) { return *e = (hipEvent_t)malloc(1), hipSuccess; }
hipError_t hipEventDestroy(hipEvent_t e) { return free(e), hipSuccess; }
hipError_t hipEventRecord(hipEvent_t e, hipStream_t)
{
    if (fails()) return fail_with;
    recorded[e] = queued;
    return hipSuccess;
}
hipError_t hipEventSynchronize(hipEvent_t e)
{
    if (fails()) return fail_with;
    run_to(recorded[e]);
    return hipSuccess;
}
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *s) { return *s = hipStreamCaptureStatusNone, hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
const char *hipGetErrorString(hipError_t) { return "as the test asked"; }

// the test's side
AIF_API void host_reset(int n_pages, int page_len, int is_mapped)
{
    run_to(queued);
    results.clear();
    wrong[0] = 0;
    pages.assign(n_pages, std::vector<Row>(page_len, Row{-2, -2}));
    mapped = is_mapped;
    calls = 0, fail_at = -1;
}
AIF_API void host_fail(long long after, int with) { fail_at = after > 0 ? calls + after : -1, fail_with = (hipError_t)with; }
AIF_API long long host_calls() { return calls; }
AIF_API long long host_waiting() { return queued - done; }
AIF_API void host_run() { run_to(queued); }
AIF_API const char *host_wrong() { return wrong; }
AIF_API int host_result(int64_t at, int64_t *to, int room)
{
    const std::vector<int64_t> &r = results[at];
    memcpy(to, r.data(), std::min<size_t>(r.size(), room) * sizeof(int64_t));
    return (int)r.size();
}
}
