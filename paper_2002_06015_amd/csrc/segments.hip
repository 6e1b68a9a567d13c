// Stable segments of small keys: order = the positions 0 .. n-1 sorted by key, equal keys in the order of their positions,
// offsets = where each key starts.  What routing to experts and the gradient of an embedding start from.
//
// A counting sort over digits of up to 9 bits, lowest digit first.  The rank of an element among the equal digits of its wave
// comes from ballots (one a bit: the lanes with the same digit), the count before the wave from LDS, so nothing depends on the
// order in which atomics arrive.  Up to 8192 positions are sorted by one workgroup whose keys stay in registers and LDS
// (one launch, bound by the instructions of its ballots on one CU: 16384 positions would take longer than in tiles).  More take
// two launches a digit: counts of 2048-position tiles, then ranks and scatter, where every tile adds up the counts of those before
// it (beyond 256 tiles a launch between them does).  Reads and writes 16 bytes a position and digit.
// 8 choices of 16 experts 3 us, 2051 positions 7, 16384 of 16 keys 16 (two launches), 131071 of 65536 keys 38 + 38 beside 268 MB of zeros.
#include "token_internal.h"

namespace kfac {

namespace {

// keys outside [0, num) become num: the last segment, which nobody reads
template <typename ID>
__device__ __forceinline__ int seg_key(const ID *ids, int i, int num)
{
    const ID v = ids[i];
    return v >= 0 && v < (ID)num ? (int)v : num;
}

typedef volatile __attribute__((address_space(3))) int *lds_counter;

// Rank of this lane's digit among equal digits of the lanes before it, and their number; `active`: lanes with an element.
__device__ __forceinline__ int match_digit(int digit, int bits, bool active, int &count)
{
    const unsigned long long in = __ballot(active);
    unsigned lo = (unsigned)in, hi = (unsigned)(in >> 32);
#pragma unroll
    for (int b = 0; b < kSegBits; ++b) {
        if (b >= bits) break;
        const int mine = (int)((unsigned)digit << (31 - b)) >> 31;   // all ones where the bit is set
        const unsigned long long with = __ballot(mine != 0);
        lo &= ~((unsigned)with ^ (unsigned)mine);
        hi &= ~((unsigned)(with >> 32) ^ (unsigned)mine);
    }
    const unsigned long long same = (unsigned long long)hi << 32 | lo;
    count = __popcll(same);
    return __popcll(same & ((1ULL << (threadIdx.x & 63)) - 1));
}

// Ranks of up to ROUNDS x 64 elements of a wave, 64 at a time in order, against counters of the wave in LDS
template <int ROUNDS>
__device__ __forceinline__ void rank_wave(const int (&key)[ROUNDS], const bool (&in)[ROUNDS], int rounds, int shift, int bits,
                                          lds_counter counter, int (&rank)[ROUNDS])
{
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        if (r >= rounds) break;
        const int digit = (key[r] >> shift) & ((1 << bits) - 1);
        int count;
        const int before = match_digit(digit, bits, in[r], count);
        const int old = in[r] ? counter[digit] : 0;
        __builtin_amdgcn_wave_barrier();   // all lanes have read before the first one of each digit counts them
        rank[r] = old + before;
        if (in[r] && before == 0) counter[digit] = old + count;
        __builtin_amdgcn_wave_barrier();
    }
}

// The counts alone: no two lanes add to the same counter at once.
template <int ROUNDS>
__device__ __forceinline__ void count_wave(const int (&key)[ROUNDS], const bool (&in)[ROUNDS], int rounds, int shift, int bits, lds_counter counter)
{
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        if (r >= rounds) break;
        const int digit = (key[r] >> shift) & ((1 << bits) - 1);
        int count;
        const int before = match_digit(digit, bits, in[r], count);
        if (in[r] && before == 0) counter[digit] += count;
        __builtin_amdgcn_wave_barrier();
    }
}

// counter[w][d] -> elements with a smaller digit, or the same digit in an earlier wave; tmp: [WAVES].  All threads call it.
template <int WAVES>
__device__ __forceinline__ void scan_counters(int *counter, int stride, int bins, int *tmp)
{
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    __syncthreads();
    int carry = 0;
    for (int d0 = 0; d0 < bins; d0 += WAVES * 64) {
        const int d = d0 + t;
        int c[WAVES], sum = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) c[w] = d < bins ? counter[w * stride + d] : 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) sum += c[w];
        int incl = sum;
        for (int o = 1; o < 64; o <<= 1) {
            const int up = __shfl_up(incl, o);
            if (lane >= o) incl += up;
        }
        if (lane == 63) tmp[wave] = incl;
        __syncthreads();
        int base = carry + incl - sum;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const int v = tmp[w];
            if (w < wave) base += v;
            carry += v;
        }
        if (d < bins)
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                counter[w * stride + d] = base;
                base += c[w];
            }
        __syncthreads();
    }
}

// Share `block` of `blocks` of the work beside a sort.
__device__ __forceinline__ void fill_share(const Fill &f, long long block, long long blocks, int threads)
{
    const long long first = block * threads + threadIdx.x, step = blocks * threads;
    if (f.data) {   // 16 bytes a lane from the first aligned element on
        typedef float f32x4 __attribute__((ext_vector_type(4)));
        long long head = (4 - (((unsigned long long)f.data >> 2) & 3)) & 3;
        if (head > f.count) head = f.count;
        const long long quads = (f.count - head) / 4;
        for (long long i = first; i < quads; i += step) *(f32x4 *)(f.data + head + 4 * i) = f32x4{0.f, 0.f, 0.f, 0.f};
        const long long rest = f.count - 4 * quads;   // head and tail
        for (long long i = first; i < rest; i += step) f.data[i < head ? i : i + 4 * quads] = 0.f;
    }
    for (long long i = first; i < f.n_decayed; i += step) f.decayed[i] = f.decay == 0.f ? 0.f : f.decay * f.decayed[i];
}

__global__ __launch_bounds__(1024) void fill_kernel(const Fill f) { fill_share(f, blockIdx.x, gridDim.x, 1024); }

__device__ __forceinline__ int lower_bound(const int *keys, int n, int key)
{
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = lo + ((hi - lo) >> 1);
        if (keys[mid] < key) lo = mid + 1; else hi = mid;
    }
    return lo;
}

template <typename ID>
__global__ __launch_bounds__(1024) void segments_small_kernel(const ID *__restrict__ ids, int n, int num, int passes, int bits,
                                                              int *__restrict__ order, int *__restrict__ keys, int *__restrict__ offsets,
                                                              const Fill fill)
{
    if (blockIdx.x > 0) {
        fill_share(fill, blockIdx.x - 1, gridDim.x - 1, 1024);
        return;
    }
    constexpr int WAVES = 16, ROUNDS = kSegSmall / 1024;
    __shared__ int skey[kSegSmall], spos[kSegSmall];
    __shared__ int counter[WAVES << kSegBits];
    __shared__ int tmp[WAVES];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int rounds = (n + 1023) / 1024, first = wave * 64 * rounds + lane;
    int key[ROUNDS], pos[ROUNDS], rank[ROUNDS];
    bool in[ROUNDS];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int i = first + 64 * r;
        in[r] = r < rounds && i < n;
        pos[r] = i;
        key[r] = in[r] ? seg_key(ids, i, num) : 0;
        rank[r] = 0;
    }
    const int bins = 1 << bits;
    for (int p = 0; p < passes; ++p) {
        for (int i = t; i < WAVES * bins; i += 1024) counter[i] = 0;
        __syncthreads();
        rank_wave<ROUNDS>(key, in, rounds, p * bits, bits, (lds_counter)(counter + wave * bins), rank);
        scan_counters<WAVES>(counter, bins, bins, tmp);
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r)
            if (in[r]) {
                const int to = counter[wave * bins + ((key[r] >> (p * bits)) & (bins - 1))] + rank[r];
                skey[to] = key[r];
                spos[to] = pos[r];
            }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r)
            if (in[r]) {
                key[r] = skey[first + 64 * r];
                pos[r] = spos[first + 64 * r];
            }
    }
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r)
        if (in[r]) {
            order[first + 64 * r] = pos[r];
            if (keys) keys[first + 64 * r] = key[r];
        }
    if (offsets)
        for (int v = t; v <= num; v += 1024) offsets[v] = lower_bound(skey, n, v);
}

// counts: [tiles][bins]
template <typename ID>
__global__ __launch_bounds__(256) void segments_count_kernel(const ID *__restrict__ ids, const int *__restrict__ keys, int n, int num, int shift,
                                                             int bits, int tiles, int *__restrict__ counts, const Fill fill)
{
    if ((int)blockIdx.x >= tiles) {
        fill_share(fill, blockIdx.x - tiles, gridDim.x - tiles, 256);
        return;
    }
    constexpr int WAVES = 4, ROUNDS = kSegTile / 256;
    __shared__ int counter[WAVES << kSegBits];
    const int bins = 1 << bits, t = threadIdx.x, lane = t & 63, wave = t >> 6;
    for (int i = t; i < WAVES * bins; i += 256) counter[i] = 0;
    int key[ROUNDS];
    bool in[ROUNDS];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int i = blockIdx.x * kSegTile + wave * 64 * ROUNDS + 64 * r + lane;
        in[r] = i < n;
        key[r] = in[r] ? (ids ? seg_key(ids, i, num) : keys[i]) : 0;
    }
    __syncthreads();
    count_wave<ROUNDS>(key, in, ROUNDS, shift, bits, (lds_counter)(counter + wave * bins));
    __syncthreads();
    for (int d = t; d < bins; d += 256) {
        int sum = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) sum += counter[w * bins + d];
        counts[(long long)blockIdx.x * bins + d] = sum;
    }
}

// running sums along the tiles, and the digits' totals
constexpr int kScanTiles = 256;   // beyond so many a launch of its own adds them up
__global__ __launch_bounds__(64) void segments_scan_kernel(int *__restrict__ counts, int tiles, int bins, int *__restrict__ totals)
{
    const int d = blockIdx.x * 64 + threadIdx.x;
    if (d >= bins) return;
    int carry = 0;
    for (int b0 = 0; b0 < tiles; b0 += 16) {
        int c[16];
#pragma unroll
        for (int q = 0; q < 16; ++q) c[q] = b0 + q < tiles ? counts[(long long)(b0 + q) * bins + d] : 0;
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            if (b0 + q < tiles) counts[(long long)(b0 + q) * bins + d] = carry;
            carry += c[q];
        }
    }
    totals[d] = carry;
}

// offsets: given with the only pass, where the digits are the keys
template <typename ID>
__global__ __launch_bounds__(256) void segments_scatter_kernel(const ID *__restrict__ ids, const int *__restrict__ keys_in,
                                                               const int *__restrict__ pos_in, int n, int num, int shift, int bits, int tiles,
                                                               const int *__restrict__ counts, const int *__restrict__ totals,
                                                               int *__restrict__ keys_out, int *__restrict__ pos_out, int *__restrict__ offsets,
                                                               const Fill fill)
{
    if ((int)blockIdx.x >= tiles) {
        fill_share(fill, blockIdx.x - tiles, gridDim.x - tiles, 256);
        return;
    }
    constexpr int WAVES = 4, ROUNDS = kSegTile / 256;
    __shared__ int counter[WAVES << kSegBits];
    __shared__ int base[1 << kSegBits];
    __shared__ int tmp[WAVES];
    const int bins = 1 << bits, t = threadIdx.x, lane = t & 63, wave = t >> 6;
    for (int i = t; i < WAVES * bins; i += 256) counter[i] = 0;
    int key[ROUNDS], pos[ROUNDS], rank[ROUNDS];
    bool in[ROUNDS];
    const int first = blockIdx.x * kSegTile + wave * 64 * ROUNDS + lane;
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int i = first + 64 * r;
        in[r] = i < n;
        pos[r] = in[r] ? (pos_in ? pos_in[i] : i) : 0;
        key[r] = in[r] ? (ids ? seg_key(ids, i, num) : keys_in[i]) : 0;
        rank[r] = 0;
    }
    __syncthreads();
    // where the digits start: a scan of their totals (as if of one wave), plus this tile's place in each
    if (tiles > kScanTiles) {
        for (int d = t; d < bins; d += 256) {
            counter[d] = totals[d];
            base[d] = counts[(long long)blockIdx.x * bins + d];
        }
    } else if (2 * t < bins) {   // two digits a thread
        int before[2] = {0, 0}, total[2] = {0, 0};
        constexpr int AHEAD = 32;
        for (int b0 = 0; b0 < tiles; b0 += AHEAD) {
            int2 c[AHEAD];
#pragma unroll
            for (int q = 0; q < AHEAD; ++q) c[q] = *(const int2 *)(counts + (long long)min(b0 + q, tiles - 1) * bins + 2 * t);
#pragma unroll
            for (int q = 0; q < AHEAD; ++q) {
                if (b0 + q < (int)blockIdx.x) { before[0] += c[q].x; before[1] += c[q].y; }
                if (b0 + q < tiles) { total[0] += c[q].x; total[1] += c[q].y; }
            }
        }
        counter[2 * t] = total[0]; counter[2 * t + 1] = total[1];
        base[2 * t] = before[0]; base[2 * t + 1] = before[1];
    }
    scan_counters<WAVES>(counter, bins, bins, tmp);      // (the other waves' counters are zero)
    for (int d = t; d < bins; d += 256) {
        if (offsets && blockIdx.x == 0 && d <= num) offsets[d] = counter[d];
        base[d] += counter[d];
    }
    __syncthreads();
    for (int i = t; i < WAVES * bins; i += 256) counter[i] = 0;
    __syncthreads();
    rank_wave<ROUNDS>(key, in, ROUNDS, shift, bits, (lds_counter)(counter + wave * bins), rank);
    __syncthreads();
    for (int d = t; d < bins; d += 256) {
        int sum = base[d], c[WAVES];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) c[w] = counter[w * bins + d];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            counter[w * bins + d] = sum;
            sum += c[w];
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r)
        if (in[r]) {
            const int to = counter[wave * bins + ((key[r] >> shift) & (bins - 1))] + rank[r];
            pos_out[to] = pos[r];
            if (keys_out) keys_out[to] = key[r];
        }
}

__global__ __launch_bounds__(256) void segments_offsets_kernel(const int *__restrict__ keys, int n, int num, int *__restrict__ offsets)
{
    const int v = blockIdx.x * 256 + threadIdx.x;
    if (v <= num) offsets[v] = lower_bound(keys, n, v);
}

// Part i of `parts` of the work beside a sort, and the workgroups of `threads` that do it (at most 4 for each CU).
Fill part_of(const Fill *fill, int i, int parts, int threads, int *wgs)
{
    Fill f{};
    *wgs = 0;
    if (!fill) return f;
    f = *fill;
    const long long per = (f.count / parts + 3) / 4 * 4, from = per * i < f.count ? per * i : f.count;
    f.count = i == parts - 1 || f.count - from < per ? f.count - from : per;
    if (f.data) f.data += from;
    if (i > 0) f.n_decayed = 0;
    const long long work = (f.data ? (f.count + 3) / 4 : 0) + f.n_decayed;   // (a part may have fewer than four elements)
    if (work > 0) *wgs = (int)(work / threads < 1024 * 256 / threads ? work / threads + 1 : 1024 * 256 / threads);
    return f;
}

template <typename ID>
hipError_t sort_positions(const ID *ids, int n, int num, const SegmentScratch &w, int *order, const int **keys, int *offsets,
                          const Fill *fill, hipStream_t s)
{
    int extra;
    if (n <= kSegSmall) {
        const bool here = num < 2 * kSegSmall;   // the offsets of more keys are found by more than one workgroup
        const Fill f = part_of(fill, 0, 1, 1024, &extra);
        segments_small_kernel<ID><<<dim3(1 + extra), dim3(1024), 0, s>>>(ids, n, num, w.passes, w.bits, order, w.keys[0], here ? offsets : nullptr, f);
        if (offsets && !here) segments_offsets_kernel<<<dim3(num / 256 + 1), dim3(256), 0, s>>>(w.keys[0], n, num, offsets);
        if (keys) *keys = w.keys[0];
        return hipGetLastError();
    }
    const int tiles = (n + kSegTile - 1) / kSegTile, bins = 1 << w.bits;
    const int *kin = nullptr, *pin = nullptr;
    for (int p = 0; p < w.passes; ++p) {
        const bool last = p == w.passes - 1;
        const ID *from = p == 0 ? ids : nullptr;
        int *kout = w.keys[p & 1], *pout = last ? order : w.pos[p & 1];
        Fill f = part_of(fill, 2 * p, 2 * w.passes, 256, &extra);
        segments_count_kernel<ID><<<dim3(tiles + extra), dim3(256), 0, s>>>(from, kin, n, num, p * w.bits, w.bits, tiles, w.counts, f);
        if (tiles > kScanTiles) segments_scan_kernel<<<dim3((bins + 63) / 64), dim3(64), 0, s>>>(w.counts, tiles, bins, w.totals);
        f = part_of(fill, 2 * p + 1, 2 * w.passes, 256, &extra);
        segments_scatter_kernel<ID><<<dim3(tiles + extra), dim3(256), 0, s>>>(from, kin, pin, n, num, p * w.bits, w.bits, tiles, w.counts, w.totals,
                                                                              kout, pout, w.passes == 1 ? offsets : nullptr, f);
        kin = kout;
        pin = pout;
    }
    if (keys) *keys = kin;
    if (offsets && w.passes > 1) segments_offsets_kernel<<<dim3(num / 256 + 1), dim3(256), 0, s>>>(kin, n, num, offsets);
    return hipGetLastError();
}

}  // namespace

size_t segment_scratch(char *base, int n, int num, SegmentScratch *out)
{
    int bits = 0;
    while (bits < 31 && ((unsigned)num >> bits)) ++bits;   // keys are 0 .. num
    SegmentScratch w{};
    if (bits < 1) bits = 1;
    w.passes = (bits + kSegBits - 1) / kSegBits;
    w.bits = (bits + w.passes - 1) / w.passes;
    const int widest = bits < kSegBits ? bits : kSegBits;   // digit of any number of keys up to this one: more keys never need less scratch
    size_t used = 0;
    auto take = [&](size_t bytes) {
        char *p = base ? base + used : nullptr;
        used += (bytes + 255) / 256 * 256;
        return (int *)p;
    };
    const size_t list = sizeof(int) * (size_t)(n > 0 ? n : 1);
    w.keys[0] = take(list);
    if (n > kSegSmall) {
        w.keys[1] = take(list);
        w.pos[0] = take(list);
        w.pos[1] = take(list);
        const size_t tiles = ((size_t)n + kSegTile - 1) / kSegTile;
        w.counts = take(sizeof(int) * (tiles << widest));
        w.totals = take(sizeof(int) << widest);
    }
    if (out) *out = w;
    return used;
}

hipError_t launch_segments(const void *ids, int id_bits, int n, int num, const SegmentScratch &w, int *order, const int **keys,
                           int *offsets, const Fill *fill, hipStream_t s)
{
    return id_bits == 64 ? sort_positions((const long long *)ids, n, num, w, order, keys, offsets, fill, s)
                         : sort_positions((const int *)ids, n, num, w, order, keys, offsets, fill, s);
}

hipError_t launch_fill(const Fill &fill, hipStream_t s)
{
    int wgs;
    const Fill f = part_of(&fill, 0, 1, 1024, &wgs);
    if (wgs > 0) fill_kernel<<<dim3(wgs), dim3(1024), 0, s>>>(f);
    return hipGetLastError();
}

}  // namespace kfac
