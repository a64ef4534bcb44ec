// The norm of many runs of numbers, and the runs times limit / norm where that is below one.
//
// All runs are cut into chunks, and a launch's workgroups share the chunks evenly, each a run of neighbouring ones, so that what a workgroup
// adds up, and with it every bit, depends on the sizes alone.  Squares and sums are 64-bit: 10^9 squares added in 32 bits would lose digits, and those
// of numbers beyond 1.8e19 would be infinite.
#include <algorithm>
#include <new>
#include <vector>

#include "experts_internal.h"

namespace asgd {

namespace {

constexpr int THREADS = 256, CHUNK = 4096;      // elements
constexpr int MOST_GROUPS = 2048;               // workgroups, and so sums, of one call: eight a compute unit
constexpr int IN_ARGUMENTS = 64;                // runs that travel as a launch's arguments; more are written to the scratch first

struct Entry {
    const void *in;
    void *out;
    int64_t n, first;                           // elements; chunks before it
    int32_t type, out_type;
};
struct Table { Entry e[IN_ARGUMENTS]; };

__global__ void table_kernel(Table t, Entry *to, int n)
{
    if ((int)threadIdx.x < n) to[threadIdx.x] = t.e[threadIdx.x];
}

// sixteen bytes at any address that an element may have
template <class T> struct Wide { T v[16 / sizeof(T)]; } __attribute__((packed));

template <class T> __device__ __forceinline__ double squares(const T *p, int64_t n, double sum)
{
    constexpr int N = 16 / sizeof(T);
    for (int64_t i = (int64_t)threadIdx.x * N; i < n; i += THREADS * N) {
        if (i + N <= n) {
            const Wide<T> w = *(const Wide<T> *)(p + i);
#pragma unroll
            for (int k = 0; k < N; k++) sum = fma((double)(float)w.v[k], (double)(float)w.v[k], sum);
        } else
            for (int64_t k = i; k < n; k++) sum = fma((double)(float)p[k], (double)(float)p[k], sum);
    }
    return sum;
}

// the sum over a workgroup, in all of its threads
__device__ __forceinline__ double group_sum(double v, double *parts)
{
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = v;
    __syncthreads();
    v = parts[0];
    for (int w = 1; w < THREADS / 64; w++) v += parts[w];
    return v;
}

// chunks [first, last) of a workgroup; calls f(entry, element, elements)
template <class F> __device__ __forceinline__ void my_chunks(const Entry *e, int count, int64_t chunks, F f)
{
    const int64_t first = chunks * blockIdx.x / gridDim.x, last = chunks * (blockIdx.x + 1) / gridDim.x;
    if (first >= last) return;
    int lo = 0, hi = count;                     // the last run that begins at or before the first chunk and has any
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (e[mid].first <= first) lo = mid; else hi = mid;
    }
    for (int64_t c = first; c < last;) {
        while (lo + 1 < count && e[lo + 1].first <= c) lo++;
        const int64_t end = lo + 1 < count && e[lo + 1].first < last ? e[lo + 1].first : last;
        const int64_t from = (c - e[lo].first) * CHUNK, to = (end - e[lo].first) * CHUNK;
        f(e[lo], from, (to < e[lo].n ? to : e[lo].n) - from);
        c = end;
    }
}

__global__ __launch_bounds__(THREADS) void squares_kernel(Table t, const Entry *more, int count, int64_t chunks, double *sums)
{
    __shared__ double parts[THREADS / 64];
    double sum = 0.0;
    my_chunks(more ? more : t.e, count, chunks, [&](const Entry &e, int64_t from, int64_t n) {
        if (e.type == ASGD_TYPE_F32) sum = squares((const float *)e.in + from, n, sum);
        else if (e.type == ASGD_TYPE_BF16) sum = squares((const __bf16 *)e.in + from, n, sum);
        else sum = squares((const _Float16 *)e.in + from, n, sum);
    });
    sum = group_sum(sum, parts);
    if (threadIdx.x == 0) sums[blockIdx.x] = sum;
}

__device__ __forceinline__ double norm_of(const double *sums, int n, double *parts)
{
    double sum = 0.0;
    for (int i = threadIdx.x; i < n; i += THREADS) sum += sums[i];
    return sqrt(group_sum(sum, parts));
}

__global__ __launch_bounds__(THREADS) void norm_kernel(const double *sums, int n, float *norm)
{
    __shared__ double parts[THREADS / 64];
    const double v = norm_of(sums, n, parts);
    if (threadIdx.x == 0) *norm = (float)v;
}

template <class T, class O> __device__ __forceinline__ void scaled(const T *p, O *q, int64_t n, float factor)
{
    constexpr int N = 16 / (sizeof(T) > sizeof(O) ? sizeof(T) : sizeof(O));
    struct In { T v[N]; } __attribute__((packed));
    struct Out { O v[N]; } __attribute__((packed));
    for (int64_t i = (int64_t)threadIdx.x * N; i < n; i += THREADS * N) {
        if (i + N <= n) {
            const In w = *(const In *)(p + i);
            Out o;
#pragma unroll
            for (int k = 0; k < N; k++) o.v[k] = (O)((float)w.v[k] * factor);
            *(Out *)(q + i) = o;
        } else
            for (int64_t k = i; k < n; k++) q[k] = (O)((float)p[k] * factor);
    }
}

__global__ __launch_bounds__(THREADS) void clip_kernel(Table t, const Entry *more, int count, int64_t chunks, const double *sums, int n, double limit, bool in_place, float *norm)
{
    __shared__ double parts[THREADS / 64];
    const double v = norm_of(sums, n, parts);
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)v;
    const float factor = v <= limit ? 1.0f : (float)(limit / v);
    if (in_place && factor == 1.0f) return;
    my_chunks(more ? more : t.e, count, chunks, [&](const Entry &e, int64_t from, int64_t m) {
        const auto to = [&](const auto *p) {
            if (e.out_type == ASGD_TYPE_F32) scaled(p, (float *)e.out + from, m, factor);
            else if (e.out_type == ASGD_TYPE_BF16) scaled(p, (__bf16 *)e.out + from, m, factor);
            else scaled(p, (_Float16 *)e.out + from, m, factor);
        };
        if (e.type == ASGD_TYPE_F32) to((const float *)e.in + from);
        else if (e.type == ASGD_TYPE_BF16) to((const __bf16 *)e.in + from);
        else to((const _Float16 *)e.in + from);
    });
}

bool span_ok(const asgd_span &s)
{
    if (s.type != ASGD_TYPE_F32 && s.type != ASGD_TYPE_BF16 && s.type != ASGD_TYPE_F16) return false;
    return s.n >= 0 && s.n <= (int64_t)1 << 40 && (s.n == 0 || (s.data && (uintptr_t)s.data % type_size((int)s.type) == 0));
}

constexpr int64_t MOST_SPANS = 1 << 20;

// chunks of all runs; -1: refused
int64_t chunks_of(const asgd_span *s, int64_t count)
{
    if (count < 0 || count > MOST_SPANS || (count > 0 && !s)) return -1;
    int64_t chunks = 0;
    for (int64_t i = 0; i < count; i++) {
        if (!span_ok(s[i])) return -1;
        chunks += (s[i].n + CHUNK - 1) / CHUNK;
        if (chunks > (int64_t)1 << 40) return -1;
    }
    return chunks;
}

struct Interval { uintptr_t from, to; };

// whether what is written shares a byte with anything but what it is made of
bool apart(const asgd_span *runs, const asgd_span *out, int64_t count)
{
    std::vector<Interval> all;
    all.reserve(2 * count);
    const auto add = [&](const asgd_span &s) { if (s.n) all.push_back({(uintptr_t)s.data, (uintptr_t)s.data + s.n * type_size((int)s.type)}); };
    for (int64_t i = 0; i < count; i++) {
        add(runs[i]);
        if (out && !(out[i].data == runs[i].data && out[i].type == runs[i].type)) add(out[i]);
    }
    const auto before = [](const Interval &a, const Interval &b) { return a.from < b.from; };
    if (!std::is_sorted(all.begin(), all.end(), before)) std::sort(all.begin(), all.end(), before);
    for (size_t i = 1; i < all.size(); i++)
        if (all[i].from < all[i - 1].to) return false;
    return true;
}

int groups_of(int64_t chunks) { return (int)(chunks < MOST_GROUPS ? chunks : MOST_GROUPS); }

// sums first, then the table of more runs than a launch takes as arguments
size_t bytes_of(int64_t chunks, int64_t count) { return 16 + sizeof(double) * (size_t)((groups_of(chunks) + 1) & ~1) + (count > IN_ARGUMENTS ? sizeof(Entry) * (size_t)count : 0); }

struct Work {
    Table t;
    Entry *more;
    double *sums;
    int64_t chunks;
    int groups;
};

// brings the table to where the kernels read it
hipError_t set_up(const asgd_span *runs, const asgd_span *out, int64_t count, int64_t chunks, void *work, Work &w, hipStream_t s)
{
    w.chunks = chunks;
    w.groups = groups_of(chunks);
    w.sums = (double *)work;
    w.more = count > IN_ARGUMENTS ? (Entry *)((char *)work + sizeof(double) * (size_t)((w.groups + 1) & ~1)) : nullptr;
    int64_t first = 0;
    for (int64_t i = 0; i < count; i++) {
        const asgd_span &o = out ? out[i] : runs[i];
        w.t.e[i % IN_ARGUMENTS] = {runs[i].data, o.data, runs[i].n, first, (int32_t)runs[i].type, (int32_t)o.type};
        first += (runs[i].n + CHUNK - 1) / CHUNK;
        if (w.more && (i % IN_ARGUMENTS == IN_ARGUMENTS - 1 || i == count - 1)) {
            table_kernel<<<1, IN_ARGUMENTS, 0, s>>>(w.t, w.more + i / IN_ARGUMENTS * IN_ARGUMENTS, (int)(i % IN_ARGUMENTS) + 1);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    }
    if (w.groups) squares_kernel<<<w.groups, THREADS, 0, s>>>(w.t, w.more, (int)count, chunks, w.sums);
    return hipGetLastError();
}

}  // namespace

}  // namespace asgd

using namespace asgd;

extern "C" {

size_t asgd_gradient_bytes(const asgd_span *runs, int64_t count)
{
    const int64_t chunks = chunks_of(runs, count);
    return chunks < 0 ? 0 : bytes_of(chunks, count);
}

int asgd_gradient_norm(const asgd_span *runs, int64_t count, float *norm, void *work, size_t work_bytes, void *hip_stream)
{
    const int64_t chunks = chunks_of(runs, count);
    if (chunks < 0 || !norm || (uintptr_t)norm % 4 || !work || (uintptr_t)work % 16 || work_bytes < bytes_of(chunks, count)) return ASGD_EINVAL;
    const hipStream_t s = (hipStream_t)hip_stream;
    Work w;
    const hipError_t e = set_up(runs, nullptr, count, chunks, work, w, s);
    if (e != hipSuccess) return ASGD_EHIP;
    norm_kernel<<<1, THREADS, 0, s>>>(w.sums, w.groups, norm);
    return hipGetLastError() == hipSuccess ? ASGD_OK : ASGD_EHIP;
}

int asgd_gradient_clip(const asgd_span *runs, const asgd_span *out, int64_t count, double limit, float *norm, void *work, size_t work_bytes,
                       void *hip_stream)
{
    const int64_t chunks = chunks_of(runs, count);
    if (chunks < 0 || !norm || (uintptr_t)norm % 4 || !work || (uintptr_t)work % 16 || work_bytes < bytes_of(chunks, count) || !(limit >= 0.0)) return ASGD_EINVAL;
    if (out) {
        if (chunks_of(out, count) < 0) return ASGD_EINVAL;
        for (int64_t i = 0; i < count; i++)
            if (out[i].n != runs[i].n) return ASGD_EINVAL;
    }
    try {
        if (!apart(runs, out, count)) return ASGD_EINVAL;
    } catch (...) {
        return ASGD_ENOMEM;
    }
    bool in_place = true;
    for (int64_t i = 0; out && i < count; i++) in_place &= out[i].n == 0 || (out[i].data == runs[i].data && out[i].type == runs[i].type);
    const hipStream_t s = (hipStream_t)hip_stream;
    Work w;
    const hipError_t e = set_up(runs, out, count, chunks, work, w, s);
    if (e != hipSuccess) return ASGD_EHIP;
    clip_kernel<<<w.groups ? w.groups : 1, THREADS, 0, s>>>(w.t, w.more, (int)count, chunks, w.sums, w.groups, limit, in_place, norm);
    return hipGetLastError() == hipSuccess ? ASGD_OK : ASGD_EHIP;
}

}  // extern "C"
