// evict.hip -- the boxes of least weight leave the memory (box_memory_evict).
//
// Attention does not care for the order of places, so what stays is not packed: only the kept boxes
// past the new length move, to the places before it that became free.  Sources and destinations are
// apart, every move is independent, and the least is moved that leaves the kept ones in front.
//
// The first kernel, a workgroup for each stream, finds the weight of the last one kept by its bits,
// eleven at a time, and numbers free places and late boxes with one scan over the places.  The second
// fills a page's free places, a wave for each key head: keys are rows; values are columns, so that the
// head's whole tile goes through LDS and back, in lines.  (Single bytes written to their places make the
// memory read and write those lines too, and took as long.)
//
// 16 streams of 8192 boxes in 16 heads of 64 channels, a quarter evicted, 111 us: 21 for the choice, 16
// workgroups of dependent steps, and 88 for the moves, 218 MB read and 138 MB written at 4.1 TB/s: a free
// place in every page makes all tiles of values go both ways, and late boxes' tiles are fetched for each
// page that takes from them, where 50 MB of codes move.  (Neighbouring pages on
// one XCD: 186 MB read, 87 us; late boxes' tiles through LDS whole, instead of bytes of them: 87.)
#include "attn.hpp"
#include "evict.hpp"

namespace rex {

namespace {

// The bits of x in the order of the numbers, NaN above all.
__device__ __forceinline__ uint32_t weight_order(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);              // (-0 is 0)
    return x != x ? 0xffffffffu : b ^ (static_cast<int32_t>(b) < 0 ? 0xffffffffu : 0x80000000u);
}

// The workgroup's sum of x over the threads before this one.
template <int WAVES> __device__ __forceinline__ int sum_before(int x, int *parts) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int upto = wave_inclusive_scan(x, lane);
    __syncthreads();                           // parts may still be read from the last time
    if (lane == 63) parts[wave] = upto;
    __syncthreads();
    int before = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) before += i < wave ? parts[i] : 0;
    return before + upto - x;
}

// The numbers of what `flags` (bit i: the thread's i-th place) marks, among all that is marked, in the
// order of places, from `base` on, which goes up by how many there are.
template <int WAVES, int HELD>
__device__ __forceinline__ void number_marked(uint32_t flags, int (&number)[HELD], int *sums, int &base) {
    constexpr int kAll = WAVES * HELD, kEach = (kAll + 63) / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    __syncthreads();                           // sums may still be read from the last time
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const uint64_t marked = __ballot(flags >> i & 1u);
        number[i] = __popcll(marked & ((uint64_t(1) << lane) - 1));
        if (lane == 0) sums[i * WAVES + wave] = __popcll(marked);
    }
    __syncthreads();
    // every wave adds up all of them, kEach a lane
    static_assert(kAll % kEach == 0 && kEach <= 2, "sums of a lane");
    const bool on = lane * kEach < kAll;
    const int x = on ? sums[kEach * lane] : 0, y = kEach > 1 && on ? sums[kEach * lane + kEach - 1] : 0;
    const int upto = wave_inclusive_scan(x + y, lane);
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int at = i * WAVES + wave;
        number[i] += base + __shfl(upto - x - y, at / kEach) + (kEach > 1 && at & 1 ? __shfl(x, at / kEach) : 0);
    }
    base += __shfl(upto, 63);
}

// Places are taken in blocks of THREADS * HELD, of which a thread holds every THREADS-th: neighbouring
// threads have neighbouring places in every read and write, and numbers among the places come from
// ballots.  The bits of the weights are looked at DIGIT at a time.
template <int THREADS, int HELD, int DIGIT>
__global__ __launch_bounds__(THREADS) void evict_select_kernel(EvictArgs e) {
    constexpr int kWaves = THREADS / 64, kChunk = THREADS * HELD, kDigits = 1 << DIGIT, kOwn = kDigits / THREADS;
    __shared__ int count[kDigits], sums[HELD * kWaves], chosen, remaining, outside;
    __shared__ int lists[2][kChunk / 2];       // free places and late boxes of a stream of one block
    const int b = blockIdx.x, tid = threadIdx.x, places = e.max_pages * kTile;
    const int64_t row = static_cast<int64_t>(b) * places;
    gcptr<float> weight = as_global<float>(e.weight + row);
    gcptr<int32_t> pages = as_global<int32_t>(e.pages + static_cast<int64_t>(b) * e.max_pages);
    gptr<int32_t> far_freed = as_global_mut<int32_t>(e.freed + row), far_late = as_global_mut<int32_t>(e.late + row);
    gptr<int32_t> from = as_global_mut<int32_t>(e.from + row), source = as_global_mut<int32_t>(e.source + row);
    gptr<float> out = as_global_mut<float>(e.weight_out + row);
    const int length = min(max(e.lengths[b], 0), places);
    const int blocks = (length + kChunk - 1) / kChunk;
    uint32_t keys[HELD];
    const auto load = [&](int block) {
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int t = block * kChunk + i * THREADS + tid;
            keys[i] = t < length ? weight_order(weight[t]) : 0u;
        }
    };
    if (tid == 0) outside = 0;
    load(0);
    __syncthreads();
    for (int i = tid; i < (length + kTile - 1) / kTile; i += THREADS)
        if (pages[i] < 0 || pages[i] >= e.num_pages) outside = 1;
    __syncthreads();
    const int keep = outside ? length : min(max(e.keep[b], 0), length);
    const bool some = keep > 0 && keep < length;

    // The bits of the last weight kept, `found`, and how many of that weight are among the kept, `left`.
    uint32_t found = 0;
    int left = keep;
    if (some) {
        for (int above = 32; above > 0;) {               // bits that are still to be looked at
            const int bits = min(DIGIT, above), shift = above - bits;
            for (int i = tid; i < kDigits; i += THREADS) count[i] = 0;
            __syncthreads();
            for (int block = 0; block < blocks; ++block) {
                if (blocks > 1) load(block);
#pragma unroll
                for (int i = 0; i < HELD; ++i)
                    if (block * kChunk + i * THREADS + tid < length &&
                        static_cast<uint64_t>(keys[i]) >> above == found)
                        atomicAdd(&count[keys[i] >> shift & ((1u << bits) - 1)], 1);
            }
            __syncthreads();
            // from the largest digit down: the one at which `left` is reached
            int own[kOwn], mine = 0;
#pragma unroll
            for (int i = 0; i < kOwn; ++i) mine += own[i] = count[kDigits - 1 - kOwn * tid - i];
            int before = sum_before<kWaves>(mine, sums);
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                if (before < left && before + own[i] >= left) {
                    chosen = kDigits - 1 - kOwn * tid - i;
                    remaining = left - before;
                }
                before += own[i];
            }
            __syncthreads();
            found = found << bits | static_cast<uint32_t>(chosen);
            left = remaining;
            above = shift;
            __syncthreads();
        }
    }
    if (tid == 0) e.lengths_out[b] = keep;

    // What is equal to the last weight is kept from the lowest place on.
    int equals = 0, frees = 0, lates = 0;
    for (int block = 0; block < (places + kChunk - 1) / kChunk; ++block) {
        if (block < blocks && blocks > 1) load(block);
        uint32_t equal = 0, free = 0, late = 0;
        int number[HELD];
        const auto place = [&](int i) { return block * kChunk + i * THREADS + tid; };
        if (some && block < blocks) {
#pragma unroll
            for (int i = 0; i < HELD; ++i) equal |= static_cast<uint32_t>(place(i) < length && keys[i] == found) << i;
            number_marked<kWaves, HELD>(equal, number, sums, equals);
        }
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int t = place(i);
            bool kept = t < keep;
            if (some) kept = t < length && (keys[i] > found || ((equal >> i & 1u) && number[i] < left));
            free |= static_cast<uint32_t>(!kept && t < keep) << i;
            late |= static_cast<uint32_t>(kept && t >= keep) << i;
            if (t >= places || (!kept && t < keep)) continue;
            from[t] = t < keep ? t : -1;
            source[t] = -1;
            out[t] = t < keep ? weight[t] : 0.0f;
        }
        if (!some || block >= blocks) continue;
        int late_number[HELD];
        number_marked<kWaves, HELD>(free, number, sums, frees);
        number_marked<kWaves, HELD>(late, late_number, sums, lates);
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            if (free >> i & 1u) {
                if (blocks == 1) lists[0][number[i]] = place(i);
                else far_freed[number[i]] = place(i);
            }
            if (late >> i & 1u) {
                if (blocks == 1) lists[1][late_number[i]] = place(i);
                else far_late[late_number[i]] = place(i);
            }
        }
    }
    __threadfence_block();
    __syncthreads();
    for (int i = tid; i < frees; i += THREADS) {        // as many late ones as free places
        const int to = blocks == 1 ? lists[0][i] : far_freed[i], t = blocks == 1 ? lists[1][i] : far_late[i];
        from[to] = t;
        source[to] = pages[t / kTile];
        out[to] = weight[t];
    }
}

constexpr int kMoveWaves = 4;

// One key head of the boxes that come to a page.
__global__ __launch_bounds__(kMoveWaves * 64) void evict_move_kernel(EvictArgs e, int groups) {
    __shared__ u32x4 tiles[kMoveWaves][128 * kTile / 16];
    __shared__ int lists[kMoveWaves][2][kTile];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t page_id = blockIdx.x / groups, at = page_id * kTile + (lane & 31);
    const int head = (blockIdx.x % groups) * kMoveWaves + wave;
    if (head >= e.Hkv) return;
    // (nothing comes to a page outside the memory, or from one: its stream is left as it is)
    const int64_t page = as_global<int32_t>(e.pages)[page_id];
    const int from = as_global<int32_t>(e.from)[at], source = as_global<int32_t>(e.source)[at];
    const bool comes = lane < kTile && source >= 0;
    const uint64_t moved = __ballot(comes);
    const int count = __popcll(moved);
    if (count == 0) return;
    int *origin = lists[wave][0], *slots = lists[wave][1];     // page; its slot and the one here
    if (comes) {
        const int i = __popcll(moved & ((uint64_t(1) << lane) - 1));
        origin[i] = source;
        slots[i] = from % kTile | lane << 8;
        if (head == 0)
            *(REX_GLOBAL f32x4 *)(e.boxes + (page * kTile + lane) * 4) =
                *(const REX_GLOBAL f32x4 *)(e.boxes + (static_cast<int64_t>(source) * kTile + from % kTile) * 4);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    int shift = 0;
    while (1 << shift < count) ++shift;
    // values: lane l moves box l % 2^shift, channels l / 2^shift and so on
    const int m = lane & ((1 << shift) - 1), step = 64 >> shift, m_in = min(m, count - 1);
    const int64_t m_page = origin[m_in];
    const int m_from = slots[m_in] & 255, m_to = slots[m_in] >> 8, c0 = m < count ? lane >> shift : e.D;
    const int chunks = e.D / 8;
    constexpr int kAhead = 8;                       // bytes of a lane on their way
    const int64_t to = page * e.Hkv + head;
    // values lie [channel][box]: the whole tile to LDS and back
    int8_t *v = e.v + to * e.D * kTile;
    gcptr<int8_t> bytes_at = as_global<int8_t>(e.v + (m_page * e.Hkv + head) * e.D * kTile + m_from);
    u32x4 held[4];
    int8_t bytes[kAhead];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (lane + 64 * i < e.D * 2) held[i] = *(const REX_GLOBAL u32x4 *)(v + (lane + 64 * i) * 16);
    const auto load = [&](int c) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (c + i * step < e.D) bytes[i] = bytes_at[(c + i * step) * kTile];
    };
    load(c0);
    if (comes) {
        const int64_t s = (static_cast<int64_t>(source) * e.Hkv + head) * kTile + from % kTile, d = to * kTile + lane;
        as_global_mut<float>(e.ks)[d] = as_global<float>(e.ks)[s];
        as_global_mut<float>(e.vs)[d] = as_global<float>(e.vs)[s];
    }
    // keys: rows of D bytes, 8 at a time
    for (int i = lane; i < count * chunks; i += 64) {
        const int k = i / chunks, c = i - k * chunks;
        const int64_t s = ((origin[k] * static_cast<int64_t>(e.Hkv) + head) * kTile + (slots[k] & 255)) * e.D + 8 * c;
        *(REX_GLOBAL u32x2 *)(e.k + (to * kTile + (slots[k] >> 8)) * e.D + 8 * c) = *(const REX_GLOBAL u32x2 *)(e.k + s);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (lane + 64 * i < e.D * 2) tiles[wave][lane + 64 * i] = held[i];
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    int8_t *tile = reinterpret_cast<int8_t *>(tiles[wave]) + m_to;
    for (int c = c0; c < e.D; c += kAhead * step) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (c + i * step < e.D) tile[(c + i * step) * kTile] = bytes[i];
        load(c + kAhead * step);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (lane + 64 * i < e.D * 2) *(REX_GLOBAL u32x4 *)(v + (lane + 64 * i) * 16) = tiles[wave][lane + 64 * i];
}

}  // namespace

hipError_t launch_evict(const EvictArgs &e, hipStream_t s) {
    if (e.max_pages * kTile <= 1024) evict_select_kernel<256, 4, 8><<<e.B, 256, 0, s>>>(e);
    else evict_select_kernel<1024, 8, 11><<<e.B, 1024, 0, s>>>(e);
    const hipError_t r = hipGetLastError();
    if (r != hipSuccess || e.max_pages == 0) return r;
    const int groups = (e.Hkv + kMoveWaves - 1) / kMoveWaves;
    const int64_t pages = static_cast<int64_t>(e.B) * e.max_pages;
    evict_move_kernel<<<static_cast<uint32_t>(pages * groups), kMoveWaves * 64, 0, s>>>(e, groups);
    return hipGetLastError();
}

}  // namespace rex
