// The order of pairs by group: a stable counting sort of ids 0 .. E - 1 (others go last).
//
// A workgroup of 16 waves places the pairs of one chunk; a wave has a run of it, so that places are in the order of the pairs: what the groups ahead have, what
// earlier chunks have of a pair's group, what earlier waves have, what earlier lanes have.  Up to 4096 pairs one workgroup places all: one launch.  Up to 65536, chunks of 1024: one launch
// counts them, and each workgroup of a second one sums over their counts by itself.  Beyond, chunks of 4096, with a launch in between that sums.
// Bound by latency, not by bytes (32768 pairs: 0.4 MB): what costs is the chain of a load, a count, a sum and a store, and the launches: up to 1024 pairs
// 3.2 us, 4096 pairs 5.1 us, 32768 pairs of 256 groups 2.6 + 7.8 us (in one launch, whose workgroups counted all pairs ahead of theirs by themselves, 16.7 us).
// All sums are of whole numbers: the order of the additions does not show.
#include "w4a16_group_device.h"

namespace w4a16 {
namespace {

constexpr int kSortWaves = 16, kSortThreads = 64 * kSortWaves;
constexpr int kOneWorkgroup = 4096, kTwoLaunches = 65536;  // pairs

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
    const int first = __builtin_ctzll(there), common = __builtin_amdgcn_readlane(key, first);
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

// Counts of each chunk, [chunks, E + 1].  A chunk has 1024 * STEPS pairs.
template <int STEPS>
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const int32_t *__restrict__ ids, long long count, int E, int *__restrict__ counts)
{
    __shared__ int n[kMaxGroups + 1];
    for (int e = (int)threadIdx.x; e <= E; e += kSortThreads) n[e] = 0;
    int key[STEPS];
#pragma unroll
    for (int j = 0; j < STEPS; ++j) {
        const long long i = ((long long)blockIdx.x * STEPS + j) * kSortThreads + threadIdx.x;
        key[j] = i < count ? key_of(ids, i, E) : -1;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < STEPS; ++j) count_key(n, key[j], key[j] >= 0);
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

// counts null: there is one chunk.  totals null: the counts are of each chunk, and summed here.
template <int STEPS>
__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(const int32_t *__restrict__ ids, int count, int E, int key_bits, const int *__restrict__ counts,
                                                                  const int *__restrict__ totals, int32_t *__restrict__ offsets, int32_t *__restrict__ order,
                                                                  int32_t *__restrict__ place)
{
    extern __shared__ int s[];
    const int keys = E + 1, tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, chunks = (int)gridDim.x, chunk = (int)blockIdx.x;
    int *const begin = s, *const ahead = s + keys + 1, *const mine = ahead + keys;  // groups' first places (and the end), pairs of earlier chunks, [wave][key]
    const int run0 = (chunk * kSortWaves + wave) * 64 * STEPS;
    int key[STEPS], rank[STEPS];  // rank: among the run's pairs of the key
#pragma unroll
    for (int j = 0; j < STEPS; ++j) {
        const int i = run0 + j * 64 + lane;
        key[j] = i < count ? key_of(ids, i, E) : -1;
    }
    for (int e = tid; e < keys; e += kSortThreads) {
        begin[e] = totals ? totals[e] : 0;
        ahead[e] = totals ? counts[(size_t)chunk * (size_t)keys + (size_t)e] : 0;
    }
    for (int e = tid; e < keys * kSortWaves; e += kSortThreads) mine[e] = 0;
    __syncthreads();
    if (counts && !totals) {
        constexpr int kAtOnce = kTwoLaunches / kSortThreads / kSortWaves;  // chunks of a wave
        for (int e = lane; e < keys; e += 64) {
            int before = 0, behind = 0;
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const int c = j * kSortWaves + wave, n = c < chunks ? counts[c * keys + e] : 0;
                before += c < chunk ? n : 0;
                behind += c < chunk ? 0 : n;
            }
            if (before) atomicAdd(&ahead[e], before);
            if (behind) atomicAdd(&begin[e], behind);
        }
    }
#pragma unroll
    for (int j = 0; j < STEPS; ++j) {
        unsigned long long same = __ballot(key[j] >= 0);  // lanes of the same key
        for (int b = 0; b < key_bits; ++b) {
            const bool set = (key[j] >> b) & 1;
            const unsigned long long with = __ballot(set);
            same &= set ? with : ~with;
        }
        rank[j] = __popcll(same & ((1ull << lane) - 1ull));
        if (key[j] >= 0) {
            int *const so_far = &mine[wave * keys + key[j]];
            const int n = *so_far;
            __builtin_amdgcn_wave_barrier();
            if (rank[j] == 0) *so_far = n + __popcll(same);
            __builtin_amdgcn_wave_barrier();
            rank[j] += n;
        }
    }
    __syncthreads();
    for (int e = tid; e < keys; e += kSortThreads) {  // the waves' counts become what earlier ones have
        int at = 0;
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            const int n = mine[w * keys + e];
            mine[w * keys + e] = at;
            at += n;
        }
        if (!counts) begin[e] = at;
        else if (!totals) begin[e] += ahead[e];
    }
    __syncthreads();
    sums_ahead(begin, keys);
    __syncthreads();
    if (chunk == 0)
        for (int e = tid; e < keys; e += kSortThreads) offsets[e] = begin[e];  // (what E begins with is where the groups end)
#pragma unroll
    for (int j = 0; j < STEPS; ++j)
        if (key[j] >= 0) {
            const int i = run0 + j * 64 + lane, at = begin[key[j]] + ahead[key[j]] + mine[wave * keys + key[j]] + rank[j];
            order[at] = i;
            if (place) place[i] = at;
        }
}

size_t place_lds(int E) { return ((size_t)(E + 1) * (kSortWaves + 2) + 1) * 4; }

template <int STEPS>
hipError_t sort_in_chunks(const int32_t *ids, long long count, int E, int32_t *offsets, int32_t *order, int32_t *place, int *counts, int *totals, hipStream_t stream)
{
    const int chunks = count ? (int)((count + STEPS * kSortThreads - 1) / (STEPS * kSortThreads)) : 1;
    hipError_t e;
    if (counts) {
        hipLaunchKernelGGL(sort_count_kernel<STEPS>, dim3((unsigned)chunks), dim3(kSortThreads), 0, stream, ids, count, E, counts);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (totals) {
        hipLaunchKernelGGL(sort_sum_kernel, dim3((unsigned)(E / 64 + 1)), dim3(64), 0, stream, counts, chunks, E, totals);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    int bits = 1;
    while ((1 << bits) <= E) ++bits;
    const auto kernel = &sort_place_kernel<STEPS>;
    if (place_lds(E) > 65536) {
        e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)place_lds(E));
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)chunks), dim3(kSortThreads), place_lds(E), stream, ids, (int)count, E, bits, counts, totals, offsets, order, place);
    return hipGetLastError();
}

long long chunks_of(long long count) { return count <= kTwoLaunches ? (count + 1023) / 1024 : (count + 4095) / 4096; }

}  // namespace

size_t group_sort_workspace(long long count, int E)
{
    if (count <= kOneWorkgroup) return 0;
    return ((size_t)chunks_of(count) + 1) * (size_t)(E + 1) * 4;
}

hipError_t launch_group_sort(const int32_t *ids, long long count, int E, int32_t *offsets, int32_t *order, int32_t *place, void *workspace, hipStream_t stream)
{
    if (count <= 1024) return sort_in_chunks<1>(ids, count, E, offsets, order, place, nullptr, nullptr, stream);
    if (count <= kOneWorkgroup) return sort_in_chunks<4>(ids, count, E, offsets, order, place, nullptr, nullptr, stream);
    int *const totals = static_cast<int *>(workspace), *const counts = totals + E + 1;
    if (count <= kTwoLaunches) return sort_in_chunks<1>(ids, count, E, offsets, order, place, counts, nullptr, stream);
    return sort_in_chunks<4>(ids, count, E, offsets, order, place, counts, totals, stream);
}

}  // namespace w4a16
