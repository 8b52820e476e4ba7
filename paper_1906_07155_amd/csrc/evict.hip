// evict.hip -- the boxes of least weight leave the memory (box_memory_evict).
//
// Attention does not care for the order of places, so what stays is not packed: only the kept boxes
// past the new length move, to the places before it that became free.  Sources and destinations are
// apart, every move is independent, and the least is moved that leaves the kept ones in front.
//
// The first kernel, a workgroup for each stream, finds the weight of the last one kept by its bits,
// eight at a time, and numbers free places and late boxes with one scan over the places.  The second
// moves a page's late boxes, a wave for each key head: their keys are rows, their values columns of a
// tile that is read once, into LDS, and whose bytes go to neighbouring places of a page, from
// neighbouring lanes.
#include "attn.hpp"
#include "evict.hpp"

namespace rex {

namespace {

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;

// The bits of x in the order of the numbers, NaN above all.
__device__ __forceinline__ uint32_t weight_order(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);              // (-0 is 0)
    return x != x ? 0xffffffffu : b ^ (static_cast<int32_t>(b) < 0 ? 0xffffffffu : 0x80000000u);
}

// The workgroup's sum of x over the threads before this one, and over all.
__device__ __forceinline__ int sum_before(int x, int *parts, int *total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int upto = wave_inclusive_scan(x, lane);
    __syncthreads();                           // parts may still be read from the last time
    if (lane == 63) parts[wave] = upto;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < kSelectWaves; ++i) {
        const int p = parts[i];
        before += i < wave ? p : 0;
        all += p;
    }
    *total = all;
    return before + upto - x;
}

__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(EvictArgs e) {
    __shared__ int count[256], parts[kSelectWaves], chosen, remaining, outside;
    const int b = blockIdx.x, tid = threadIdx.x, places = e.max_pages * kTile;
    const int64_t row = static_cast<int64_t>(b) * places;
    gcptr<float> weight = as_global<float>(e.weight + row);
    gcptr<int32_t> pages = as_global<int32_t>(e.pages + static_cast<int64_t>(b) * e.max_pages);
    gptr<int32_t> freed = as_global_mut<int32_t>(e.freed + row), to = as_global_mut<int32_t>(e.to + row);
    const int length = min(max(e.lengths[b], 0), places);
    if (tid == 0) outside = 0;
    __syncthreads();
    for (int i = tid; i < (length + kTile - 1) / kTile; i += kSelectThreads)
        if (pages[i] < 0 || pages[i] >= e.num_pages) outside = 1;
    __syncthreads();
    const int keep = outside ? length : min(max(e.keep[b], 0), length);

    // The bits of the last weight kept, and how many of that weight: `left` of those whose bits so far
    // are `found` are among the kept.
    uint32_t found = 0;
    int left = keep;
    if (keep > 0 && keep < length) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256) count[tid] = 0;
            __syncthreads();
            for (int t = tid; t < length; t += kSelectThreads) {
                const uint32_t key = weight_order(weight[t]);
                if (shift == 24 || key >> (shift + 8) == found) atomicAdd(&count[key >> shift & 255u], 1);
            }
            __syncthreads();
            // from the largest digit down: the one at which `left` is reached
            int total;
            const int mine = tid < 256 ? count[255 - tid] : 0, before = sum_before(mine, parts, &total);
            if (tid < 256 && before < left && before + mine >= left) {
                chosen = 255 - tid;
                remaining = left - before;
            }
            __syncthreads();
            found = found << 8 | static_cast<uint32_t>(chosen);
            left = remaining;
            __syncthreads();
        }
    }
    const bool some = keep > 0 && keep < length;
    if (tid == 0) e.lengths_out[b] = keep;

    // Runs of places of each thread; what is equal to the last weight is kept from the lowest place on.
    const int each = (length + kSelectThreads - 1) / kSelectThreads;
    const int first = min(tid * each, length), end = min(first + each, length);
    int total, equal = 0;
    if (some) {
        for (int t = first; t < end; ++t) equal += weight_order(weight[t]) == found;
        equal = sum_before(equal, parts, &total);
    }
    const auto kept = [&](int t, int &equals) {
        if (!some) return t < keep;
        const uint32_t key = weight_order(weight[t]);
        return key > found || (key == found && equals++ < left);
    };
    int free_before = 0, late_before = 0, seen = equal;
    for (int t = first; t < end; ++t) {
        const bool k = kept(t, seen);
        free_before += !k && t < keep;
        late_before += k && t >= keep;
    }
    free_before = sum_before(free_before, parts, &total);
    late_before = sum_before(late_before, parts, &total);
    seen = equal;
    int late = late_before;
    for (int t = first; t < end; ++t) {
        const bool k = kept(t, seen);
        if (!k && t < keep) freed[free_before++] = t;
        // (its number among the late ones; where it goes is known once all free places are)
        to[t] = k && t >= keep ? late++ : -1;
    }
    for (int t = length + tid; t < places; t += kSelectThreads) to[t] = -1;
    for (int t = tid; t < places; t += kSelectThreads) {
        // what a late box fills is written below
        as_global_mut<float>(e.weight_out)[row + t] = t < keep ? weight[t] : 0.0f;
        if (e.origin) as_global_mut<int32_t>(e.origin)[row + t] = t < keep ? t : -1;
    }
    __threadfence_block();
    __syncthreads();
    for (int t = keep + tid; t < length; t += kSelectThreads) {
        const int i = to[t];
        if (i < 0) continue;
        const int at = freed[i];
        to[t] = at;
        as_global_mut<float>(e.weight_out)[row + at] = weight[t];
        if (e.origin) as_global_mut<int32_t>(e.origin)[row + at] = t;
    }
}

constexpr int kMoveWaves = 4;

// Rows of a page's late boxes (slot `from`, to place `to`), one key head of them.
__global__ __launch_bounds__(kMoveWaves * 64) void evict_move_kernel(EvictArgs e, int groups) {
    __shared__ u32x4 tiles[kMoveWaves][128 * kTile / 16];
    __shared__ int lists[kMoveWaves][2][kTile];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t page_id = blockIdx.x / groups;
    const int head = (blockIdx.x % groups) * kMoveWaves + wave;
    if (head >= e.Hkv) return;
    const int b = static_cast<int>(page_id / e.max_pages);
    const int64_t row = page_id * kTile;                       // of e.to
    const int to = lane < kTile ? as_global<int32_t>(e.to)[row + lane] : -1;
    const uint64_t moved = __ballot(to >= 0);
    const int count = __popcll(moved);
    if (count == 0) return;
    // (a page that is outside the memory has no late box: its stream is left as it is)
    const int64_t page = as_global<int32_t>(e.pages)[page_id];
    int *from = lists[wave][0], *slot = lists[wave][1];
    if (to >= 0) {
        const int i = __popcll(moved & ((uint64_t(1) << lane) - 1));
        const int64_t dest = as_global<int32_t>(e.pages)[static_cast<int64_t>(b) * e.max_pages + to / kTile];
        from[i] = lane;
        slot[i] = static_cast<int>(dest);
        const int64_t s = (page * e.Hkv + head) * kTile + lane, d = (dest * e.Hkv + head) * kTile + to % kTile;
        as_global_mut<float>(e.ks)[d] = as_global<float>(e.ks)[s];
        as_global_mut<float>(e.vs)[d] = as_global<float>(e.vs)[s];
        if (head == 0)
            *(REX_GLOBAL f32x4 *)(e.boxes + (dest * kTile + to % kTile) * 4) =
                *(const REX_GLOBAL f32x4 *)(e.boxes + (page * kTile + lane) * 4);
        from[i] |= to % kTile << 8;
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    // keys: rows of D bytes, 8 at a time
    const int chunks = e.D / 8;
    for (int i = lane; i < count * chunks; i += 64) {
        const int m = i / chunks, c = i - m * chunks;
        const int64_t s = ((page * e.Hkv + head) * kTile + (from[m] & 255)) * e.D + 8 * c;
        const int64_t d = ((slot[m] * static_cast<int64_t>(e.Hkv) + head) * kTile + (from[m] >> 8)) * e.D + 8 * c;
        *(REX_GLOBAL u32x2 *)(e.k + d) = *(const REX_GLOBAL u32x2 *)(e.k + s);
    }
    // values: [channel][box]
    const int64_t s = (page * e.Hkv + head) * e.D * kTile;
    for (int i = lane; i < e.D * 2; i += 64) tiles[wave][i] = *(const REX_GLOBAL u32x4 *)(e.v + s + i * 16);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    const int8_t *tile = reinterpret_cast<const int8_t *>(tiles[wave]);
    int shift = 0;
    while (1 << shift < count) ++shift;
    const int m = lane & ((1 << shift) - 1);
    if (m < count) {
        const int at = from[m] & 255;
        const int64_t d = (slot[m] * static_cast<int64_t>(e.Hkv) + head) * e.D * kTile + (from[m] >> 8);
#pragma unroll 4
        for (int c = lane >> shift; c < e.D; c += 64 >> shift) as_global_mut<int8_t>(e.v)[d + c * kTile] = tile[c * kTile + at];
    }
}

}  // namespace

hipError_t launch_evict(const EvictArgs &e, hipStream_t s) {
    evict_select_kernel<<<e.B, kSelectThreads, 0, s>>>(e);
    const hipError_t r = hipGetLastError();
    if (r != hipSuccess || e.max_pages == 0) return r;
    const int groups = (e.Hkv + kMoveWaves - 1) / kMoveWaves;
    const int64_t grid = static_cast<int64_t>(e.B) * e.max_pages * groups;
    evict_move_kernel<<<static_cast<uint32_t>(grid), kMoveWaves * 64, 0, s>>>(e, groups);
    return hipGetLastError();
}

}  // namespace rex
