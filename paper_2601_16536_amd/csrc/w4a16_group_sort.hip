// The order of pairs by group: a stable counting sort of ids 0 .. E - 1 (others go last).
//
// A workgroup of 16 waves places the pairs of one chunk; a wave has a run of it, so that places are in the order of the pairs: what the groups ahead have, what
// earlier chunks have of a pair's group, what earlier waves have, what earlier lanes have.  Up to kOneLaunch pairs a workgroup counts everything ahead of its chunk, and
// all pairs, by itself, in LDS: one launch.  Beyond, one launch counts the chunks, a second one sums over them, a third one places.
// All sums are of whole numbers: the order of the additions does not show.
#include "w4a16_group_device.h"

namespace w4a16 {
namespace {

constexpr int kSortWaves = 16, kSortThreads = 64 * kSortWaves, kRun = 256, kChunk = kSortWaves * kRun;  // pairs of a wave, of a workgroup
constexpr int kOneLaunch = 65536;

__device__ __forceinline__ int key_of(const int32_t *ids, long long i, int E)
{
    const int e = ids[i];
    return e >= 0 && e < E ? e : E;
}

// count[key] += 1 for every lane with `have`.  What the first of them has, which may be what all have, as one addition.
__device__ __forceinline__ void count_key(int *count, int key, bool have)
{
    const unsigned long long there = __ballot(have);
    if (there == 0) return;
    const int first = __builtin_ctzll(there), common = __shfl(key, first, 64);
    const unsigned long long same = __ballot(have && key == common);
    const int lane = (int)threadIdx.x & 63;
    if (lane == first) atomicAdd(&count[common], __popcll(same));
    if (have && key != common) atomicAdd(&count[key], 1);
}

// a[0 .. n - 1] becomes the sums ahead of each, a[n] the whole.  By the first wave; n <= kMaxGroups + 1.
__device__ __forceinline__ void sums_ahead(int *a, int n)
{
    if (threadIdx.x >= 64) return;
    const int lane = (int)threadIdx.x;
    int at = 0;
    for (int e0 = 0; e0 < n; e0 += 64) {
        const int v = e0 + lane < n ? a[e0 + lane] : 0;
        int upto = v;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int u = __shfl_up(upto, d, 64);
            if (lane >= d) upto += u;
        }
        if (e0 + lane < n) a[e0 + lane] = at + upto - v;
        at += __shfl(upto, 63, 64);
    }
    if (lane == 0) a[n] = at;
}

// Counts of each chunk, [chunks, E + 1].
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const int32_t *__restrict__ ids, long long count, int E, int *__restrict__ counts)
{
    __shared__ int n[kMaxGroups + 1];
    for (int e = (int)threadIdx.x; e <= E; e += kSortThreads) n[e] = 0;
    __syncthreads();
    for (int j = 0; j < kChunk; j += kSortThreads) {
        const long long i = (long long)blockIdx.x * kChunk + j + threadIdx.x;
        count_key(n, i < count ? key_of(ids, i, E) : E, i < count);
    }
    __syncthreads();
    for (int e = (int)threadIdx.x; e <= E; e += kSortThreads) counts[(size_t)blockIdx.x * (size_t)(E + 1) + (size_t)e] = n[e];
}

// counts[chunk][e] becomes what earlier chunks have of e; totals[e].  A thread per key.
__global__ __launch_bounds__(64) void sort_sum_kernel(int *__restrict__ counts, int chunks, int E, int *__restrict__ totals)
{
    const int e = (int)(blockIdx.x * 64 + threadIdx.x);
    if (e > E) return;
    int at = 0, i = 0;
    for (; i + 8 <= chunks; i += 8) {
        int v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = counts[(size_t)(i + j) * (size_t)(E + 1) + (size_t)e];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            counts[(size_t)(i + j) * (size_t)(E + 1) + (size_t)e] = at;
            at += v[j];
        }
    }
    for (; i < chunks; ++i) {
        const int v = counts[(size_t)i * (size_t)(E + 1) + (size_t)e];
        counts[(size_t)i * (size_t)(E + 1) + (size_t)e] = at;
        at += v;
    }
    totals[e] = at;
}

// counts null: counted here.
__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(const int32_t *__restrict__ ids, int count, int E, int key_bits, const int *__restrict__ counts,
                                                                  const int *__restrict__ totals, int32_t *__restrict__ offsets, int32_t *__restrict__ order,
                                                                  int32_t *__restrict__ place)
{
    extern __shared__ int s[];
    const int keys = E + 1, tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int *const begin = s, *const ahead = s + keys + 1, *const mine = ahead + keys;  // groups' first places (and the end), pairs of earlier chunks, [wave][key]
    const int chunk0 = (int)blockIdx.x * kChunk, run0 = chunk0 + wave * kRun;
    for (int e = tid; e < keys; e += kSortThreads) {
        begin[e] = counts ? totals[e] : 0;
        ahead[e] = counts ? counts[(size_t)blockIdx.x * (size_t)keys + (size_t)e] : 0;
    }
    for (int e = tid; e < keys * kSortWaves; e += kSortThreads) mine[e] = 0;
    __syncthreads();
    if (!counts) {  // ahead of the chunk, and from it on
        constexpr int kAtOnce = kChunk / kSortThreads * 2;  // loads on their way
        for (int i0 = 0; i0 < count; i0 += kSortThreads * kAtOnce) {
            int k[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const int i = i0 + j * kSortThreads + tid;
                k[j] = i < count ? key_of(ids, i, E) : -1;
            }
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) count_key(i0 + j * kSortThreads < chunk0 ? ahead : begin, k[j], k[j] >= 0);
        }
    }
    int key[kRun / 64];
#pragma unroll
    for (int j = 0; j < kRun / 64; ++j) {
        const int i = run0 + j * 64 + lane;
        key[j] = i < count ? key_of(ids, i, E) : -1;
    }
#pragma unroll
    for (int j = 0; j < kRun / 64; ++j) count_key(mine + wave * keys, key[j], key[j] >= 0);
    __syncthreads();
    if (!counts) {
        for (int e = tid; e < keys; e += kSortThreads) begin[e] += ahead[e];
        __syncthreads();
    }
    sums_ahead(begin, keys);
    __syncthreads();
    if (blockIdx.x == 0)
        for (int e = tid; e < keys; e += kSortThreads) offsets[e] = begin[e];  // (what E begins with is where the groups end)
    for (int e = tid; e < keys; e += kSortThreads) {
        int at = begin[e] + ahead[e];
        for (int w = 0; w < kSortWaves; ++w) {
            const int n = mine[w * keys + e];
            mine[w * keys + e] = at;
            at += n;
        }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kRun / 64; ++j) {
        unsigned long long same = __ballot(key[j] >= 0);  // lanes of the same key
        for (int b = 0; b < key_bits; ++b) {
            const bool set = (key[j] >> b) & 1;
            const unsigned long long with = __ballot(set);
            same &= set ? with : ~with;
        }
        if (key[j] >= 0) {
            const int rank = __popcll(same & ((1ull << lane) - 1ull)), i = run0 + j * 64 + lane;
            int *const next = &mine[wave * keys + key[j]];
            const int at = *next + rank;
            __builtin_amdgcn_wave_barrier();
            if (rank == 0) *next += __popcll(same);
            __builtin_amdgcn_wave_barrier();
            order[at] = i;
            if (place) place[i] = at;
        }
    }
}

size_t place_lds(int E) { return ((size_t)(E + 1) * (kSortWaves + 2) + 1) * 4; }

}  // namespace

size_t group_sort_workspace(long long count, int E)
{
    if (count <= kOneLaunch) return 0;
    return ((size_t)((count + kChunk - 1) / kChunk) + 1) * (size_t)(E + 1) * 4;
}

hipError_t launch_group_sort(const int32_t *ids, long long count, int E, int32_t *offsets, int32_t *order, int32_t *place, void *workspace, hipStream_t stream)
{
    const int chunks = count ? (int)((count + kChunk - 1) / kChunk) : 1;
    int *counts = nullptr, *totals = nullptr;
    if (count > kOneLaunch) {
        totals = static_cast<int *>(workspace);
        counts = totals + E + 1;
        hipLaunchKernelGGL(sort_count_kernel, dim3((unsigned)chunks), dim3(kSortThreads), 0, stream, ids, count, E, counts);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(sort_sum_kernel, dim3((unsigned)(E / 64 + 1)), dim3(64), 0, stream, counts, chunks, E, totals);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    int bits = 1;
    while ((1 << bits) <= E) ++bits;
    if (place_lds(E) > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&sort_place_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)place_lds(E));
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(sort_place_kernel, dim3((unsigned)chunks), dim3(kSortThreads), place_lds(E), stream, ids, (int)count, E, bits, counts, totals, offsets, order, place);
    return hipGetLastError();
}

}  // namespace w4a16
