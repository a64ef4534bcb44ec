// The norm of many runs of numbers, and the runs times limit / norm where that is below one.
//
// All runs are cut into chunks, and a launch's workgroups share the chunks evenly, each a run of neighbouring ones, so that what a workgroup
// adds up, and with it every bit, depends on the sizes alone.  Memory bounds it: 300 runs of 4 * 10^8 float32 numbers, 1.6 GB, are read in 250 us (6.4 TB/s) and clipped
// to bfloat16 in 524 (4.6 TB/s, read and written; a large copy reaches 4.9).  Squares and sums are 64-bit: 10^9 squares added in 32 bits would lose digits, and those
// of numbers beyond 1.8e19 would be infinite.
#include <algorithm>
#include <type_traits>
#include <vector>

#include "experts_internal.h"

namespace asgd {

namespace {

constexpr int THREADS = 256, CHUNK = 4096;      // elements
constexpr int MOST_GROUPS = 2048;               // workgroups, and so sums, of one call: eight a compute unit
constexpr int IN_ARGUMENTS = 64;                // runs that travel as a launch's arguments; more are written to the scratch first
constexpr int64_t LAST_CACHE = 256 << 20;       // bytes
constexpr int FEW_THREADS = 1024, FEW_CHUNKS = 16;      // up to so many chunks are one workgroup's, in one launch

#define GLOBAL __attribute__((address_space(1)))

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

// N elements, 8 or 16 bytes, at any address that an element may have, which the hardware takes as it does aligned ones
template <int BYTES> struct Bytes;
template <> struct Bytes<16> { typedef int T __attribute__((ext_vector_type(4), aligned(2))); };
template <> struct Bytes<8> { typedef int T __attribute__((ext_vector_type(2), aligned(2))); };
template <class T, int N> struct Wide {
    typedef typename Bytes<N * sizeof(T)>::T B;
    T v[N];
    template <bool ONCE> __device__ __forceinline__ void load(const GLOBAL T *p)
    {
        B b;
        if constexpr (ONCE) b = __builtin_nontemporal_load((const GLOBAL B *)p);
        else b = *(const GLOBAL B *)p;
        __builtin_memcpy(v, &b, sizeof(b));
    }
    __device__ __forceinline__ void store(GLOBAL T *p) const
    {
        B b;
        __builtin_memcpy(&b, v, sizeof(b));
        *(GLOBAL B *)p = b;
    }
};

// f(element) for every wide load of a workgroup's part [0, n), four of them together, then what is left, an element each
template <int N, int GROUP, class F, class G> __device__ __forceinline__ void parts_of(int64_t n, F wide, G one)
{
    constexpr int64_t STEP = (int64_t)GROUP * N;
    const int64_t whole = n / N * N;
    int64_t i = (int64_t)threadIdx.x * N;
    for (; i + 3 * STEP < whole; i += 4 * STEP) wide(i, STEP, std::integral_constant<int, 4>());
    for (; i < whole; i += STEP) wide(i, STEP, std::integral_constant<int, 1>());
    if (whole + threadIdx.x < n) one(whole + threadIdx.x);
}

template <int GROUP, bool ONCE, class T> __device__ __forceinline__ double squares(const T *in, int64_t n, double sum)
{
    constexpr int N = 16 / sizeof(T);
    typedef Wide<T, N> W;
    const GLOBAL T *const p = (const GLOBAL T *)in;
    parts_of<N, GROUP>(n, [&](int64_t i, int64_t step, auto times) {
        W w[times.value];
#pragma unroll
        for (int m = 0; m < times.value; m++) w[m].template load<ONCE>(p + i + m * step);
#pragma unroll
        for (int m = 0; m < times.value; m++)
#pragma unroll
            for (int k = 0; k < N; k++) sum = fma((double)(float)w[m].v[k], (double)(float)w[m].v[k], sum);
    }, [&](int64_t i) { sum = fma((double)(float)p[i], (double)(float)p[i], sum); });
    return sum;
}

template <int GROUP, class T, class O> __device__ __forceinline__ void scaled(const T *in, O *out, int64_t n, float factor)
{
    constexpr int N = 16 / (sizeof(T) > sizeof(O) ? sizeof(T) : sizeof(O));
    typedef Wide<T, N> W;
    typedef Wide<O, N> V;
    const GLOBAL T *const p = (const GLOBAL T *)in;
    GLOBAL O *const q = (GLOBAL O *)out;
    parts_of<N, GROUP>(n, [&](int64_t i, int64_t step, auto times) {
        W w[times.value];
#pragma unroll
        for (int m = 0; m < times.value; m++) w[m].template load<false>(p + i + m * step);
#pragma unroll
        for (int m = 0; m < times.value; m++) {
            V o;
#pragma unroll
            for (int k = 0; k < N; k++) o.v[k] = (O)((float)w[m].v[k] * factor);
            o.store(q + i + m * step);
        }
    }, [&](int64_t i) { q[i] = (O)((float)p[i] * factor); });
}

// the sum over a workgroup, in all of its threads
template <int GROUP> __device__ __forceinline__ double group_sum(double v, double *parts)
{
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = v;
    __syncthreads();
    v = parts[0];
    for (int w = 1; w < GROUP / 64; w++) v += parts[w];
    return v;
}

// The chunks of workgroup `group` of `groups`, as parts of runs: f(entry, element, elements)
template <class F> __device__ __forceinline__ void my_parts(const Entry *e, int count, int64_t chunks, int64_t group, int64_t groups, F f)
{
    const int64_t begin = chunks * group / groups, end = chunks * (group + 1) / groups;
    if (begin >= end) return;
    int run = 0, past = count;                  // the last run that begins at or before the first chunk (and so has it)
    while (past - run > 1) {
        const int mid = (run + past) / 2;
        if (e[mid].first <= begin) run = mid; else past = mid;
    }
    for (int64_t c = begin; c < end;) {
        while (run + 1 < count && e[run + 1].first <= c) run++;
        const Entry &x = e[run];
        const int64_t to = run + 1 < count && e[run + 1].first < end ? e[run + 1].first : end;
        const int64_t element = (c - x.first) * CHUNK, last = (to - x.first) * CHUNK;
        f(x, element, (last < x.n ? last : x.n) - element);
        c = to;
    }
}

// once: more than the last cache holds, which it passes by (it holds what was written before, and what is read again would not be there any more: the squares
// of 1.6 GB take 253 us so and 303 through it, clipping them to 0.8 GB next 534 and 518)
template <int GROUP> __device__ __forceinline__ double my_squares(const Entry *e, int count, int64_t chunks, int64_t group, int64_t groups, bool once)
{
    double sum = 0.0;
    my_parts(e, count, chunks, group, groups, [&](const Entry &x, int64_t from, int64_t n) {
        const auto add = [&](const auto *p) { sum = once ? squares<GROUP, true>(p, n, sum) : squares<GROUP, false>(p, n, sum); };
        if (x.type == ASGD_TYPE_F32) add((const float *)x.in + from);
        else if (x.type == ASGD_TYPE_BF16) add((const __bf16 *)x.in + from);
        else add((const _Float16 *)x.in + from);
    });
    return sum;
}

template <int GROUP> __device__ __forceinline__ void my_scaled(const Entry *e, int count, int64_t chunks, int64_t group, int64_t groups, float factor)
{
    my_parts(e, count, chunks, group, groups, [&](const Entry &x, int64_t from, int64_t n) {
        const auto to = [&](const auto *p) {
            if (x.out_type == ASGD_TYPE_F32) scaled<GROUP>(p, (float *)x.out + from, n, factor);
            else if (x.out_type == ASGD_TYPE_BF16) scaled<GROUP>(p, (__bf16 *)x.out + from, n, factor);
            else scaled<GROUP>(p, (_Float16 *)x.out + from, n, factor);
        };
        if (x.type == ASGD_TYPE_F32) to((const float *)x.in + from);
        else if (x.type == ASGD_TYPE_BF16) to((const __bf16 *)x.in + from);
        else to((const _Float16 *)x.in + from);
    });
}

__device__ __forceinline__ float factor_of(double norm, double limit) { return norm <= limit ? 1.0f : (float)(limit / norm); }

__global__ __launch_bounds__(THREADS) void squares_kernel(Table t, const Entry *more, int count, int64_t chunks, bool once, double *sums)
{
    __shared__ double parts[THREADS / 64];
    const double sum = group_sum<THREADS>(my_squares<THREADS>(more ? more : t.e, count, chunks, blockIdx.x, gridDim.x, once), parts);
    if (threadIdx.x == 0) sums[blockIdx.x] = sum;
}

__device__ __forceinline__ double norm_of(const double *sums, int n, double *parts)
{
    double sum = 0.0;
    for (int i = threadIdx.x; i < n; i += THREADS) sum += sums[i];
    return sqrt(group_sum<THREADS>(sum, parts));
}

__global__ __launch_bounds__(THREADS) void norm_kernel(const double *sums, int n, float *norm)
{
    __shared__ double parts[THREADS / 64];
    const double v = norm_of(sums, n, parts);
    if (threadIdx.x == 0) *norm = (float)v;
}

__global__ __launch_bounds__(THREADS) void clip_kernel(Table t, const Entry *more, int count, int64_t chunks, const double *sums, int n, double limit, bool in_place, float *norm)
{
    __shared__ double parts[THREADS / 64];
    const double v = norm_of(sums, n, parts);
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)v;
    const float factor = factor_of(v, limit);
    if (in_place && factor == 1.0f) return;
    my_scaled<THREADS>(more ? more : t.e, count, chunks, blockIdx.x, gridDim.x, factor);
}

// Both at once for few chunks: the second launch would take longer than one workgroup does (three runs of 13000: 7.8 us, in two launches 3.9 + 4.8 and the host's 5 more).
template <bool CLIP> __global__ __launch_bounds__(FEW_THREADS) void few_kernel(Table t, int count, int64_t chunks, double limit, bool in_place, float *norm)
{
    __shared__ double parts[FEW_THREADS / 64];
    const double v = sqrt(group_sum<FEW_THREADS>(my_squares<FEW_THREADS>(t.e, count, chunks, 0, 1, false), parts));
    if (threadIdx.x == 0) *norm = (float)v;
    if (!CLIP) return;
    const float factor = factor_of(v, limit);
    if (in_place && factor == 1.0f) return;
    my_scaled<FEW_THREADS>(t.e, count, chunks, 0, 1, factor);
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

struct Interval {
    uintptr_t from, to;
    bool written;
};

// whether what is written shares no byte with anything but what it is made of (runs that are only read may share theirs)
bool apart(const asgd_span *runs, const asgd_span *out, int64_t count)
{
    std::vector<Interval> all;
    all.reserve(2 * count);
    const auto add = [&](const asgd_span &s, bool written) { if (s.n) all.push_back({(uintptr_t)s.data, (uintptr_t)s.data + s.n * type_size((int)s.type), written}); };
    for (int64_t i = 0; i < count; i++) {
        const bool in_place = !out || (out[i].data == runs[i].data && out[i].type == runs[i].type);
        add(runs[i], in_place);
        if (!in_place) add(out[i], true);
    }
    const auto before = [](const Interval &a, const Interval &b) { return a.from < b.from; };
    if (!std::is_sorted(all.begin(), all.end(), before)) std::sort(all.begin(), all.end(), before);
    uintptr_t end = 0, end_written = 0;         // of those before, and of the written ones among them
    for (const Interval &i : all) {
        if (i.from < (i.written ? end : end_written)) return false;
        end = std::max(end, i.to);
        if (i.written) end_written = std::max(end_written, i.to);
    }
    return true;
}

int groups_of(int64_t chunks) { return (int)(chunks < MOST_GROUPS ? chunks : MOST_GROUPS); }

// sums first, then the table of more runs than a launch takes as arguments
size_t bytes_of(int64_t count) { return sizeof(double) * MOST_GROUPS + (count > IN_ARGUMENTS ? sizeof(Entry) * (size_t)count : 0); }

// The norm, and (limit >= 0) what follows from it.
hipError_t launch(const asgd_span *runs, const asgd_span *out, int64_t count, int64_t chunks, double limit, bool in_place, float *norm, void *work, hipStream_t s)
{
    Table t;
    double *const sums = (double *)work;
    Entry *const more = count > IN_ARGUMENTS ? (Entry *)(sums + MOST_GROUPS) : nullptr;
    const int groups = groups_of(chunks), n = (int)count;
    int64_t first = 0, bytes = 0;
    for (int64_t i = 0; i < count; i++) {
        const asgd_span &o = out ? out[i] : runs[i];
        t.e[i % IN_ARGUMENTS] = {runs[i].data, o.data, runs[i].n, first, (int32_t)runs[i].type, (int32_t)o.type};
        first += (runs[i].n + CHUNK - 1) / CHUNK;
        bytes += runs[i].n * (int64_t)type_size((int)runs[i].type);
        if (more && (i % IN_ARGUMENTS == IN_ARGUMENTS - 1 || i == count - 1)) {
            table_kernel<<<1, IN_ARGUMENTS, 0, s>>>(t, more + i / IN_ARGUMENTS * IN_ARGUMENTS, (int)(i % IN_ARGUMENTS) + 1);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    }
    if (!more && chunks <= FEW_CHUNKS) {
        if (limit >= 0.0) few_kernel<true><<<1, FEW_THREADS, 0, s>>>(t, n, chunks, limit, in_place, norm);
        else few_kernel<false><<<1, FEW_THREADS, 0, s>>>(t, n, chunks, limit, in_place, norm);
        return hipGetLastError();
    }
    if (groups) squares_kernel<<<groups, THREADS, 0, s>>>(t, more, n, chunks, bytes > LAST_CACHE, sums);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (limit >= 0.0) clip_kernel<<<groups ? groups : 1, THREADS, 0, s>>>(t, more, n, chunks, sums, groups, limit, in_place, norm);
    else norm_kernel<<<1, THREADS, 0, s>>>(sums, groups, norm);
    return hipGetLastError();
}

}  // namespace

}  // namespace asgd

using namespace asgd;

extern "C" {

size_t asgd_gradient_bytes(int64_t count) { return count < 0 || count > MOST_SPANS ? 0 : bytes_of(count); }

int asgd_gradient_norm(const asgd_span *runs, int64_t count, float *norm, void *work, size_t work_bytes, void *hip_stream)
{
    const int64_t chunks = chunks_of(runs, count);
    if (chunks < 0 || !norm || (uintptr_t)norm % 4 || !work || (uintptr_t)work % 16 || work_bytes < bytes_of(count)) return ASGD_EINVAL;
    return launch(runs, nullptr, count, chunks, -1.0, false, norm, work, (hipStream_t)hip_stream) == hipSuccess ? ASGD_OK : ASGD_EHIP;
}

int asgd_gradient_clip(const asgd_span *runs, const asgd_span *out, int64_t count, double limit, float *norm, void *work, size_t work_bytes,
                       void *hip_stream)
{
    const int64_t chunks = chunks_of(runs, count);
    if (chunks < 0 || !norm || (uintptr_t)norm % 4 || !work || (uintptr_t)work % 16 || work_bytes < bytes_of(count) || !(limit >= 0.0)) return ASGD_EINVAL;
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
    return launch(runs, out, count, chunks, limit, in_place, norm, work, (hipStream_t)hip_stream) == hipSuccess ? ASGD_OK : ASGD_EHIP;
}

}  // extern "C"
