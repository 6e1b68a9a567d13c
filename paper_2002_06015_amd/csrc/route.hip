// Routing: which experts a token goes to, with which gates, and the gradient of the logits.
//
//   s = softmax(l) or sigmoid(l);  rank = s + bias in 64 bits, or the logit itself where there is no bias;  groups by the sum of their best
//   one or two ranks;  the `fan` best open experts of the best groups, equal ranks by number;  gate = scale s (/ sum of the chosen s)
// A renormalised gate needs no sum over all experts: with m the largest chosen logit, softmaxes give exp(l_j - m) / sum exp(l_i - m);
// sigmoids s_j / sum s_i, and exp(l_j - m) / sum exp(l_i - m) where all chosen logits are below -60 (there s = exp(l) to 2^-86, and the
// sigmoids themselves would leave the range of fp32).
#include "elements.h"
#include "token_internal.h"

namespace kfac {

namespace {

__device__ __forceinline__ float sigmoid(float l) { return 1.f / (1.f + expf(-l)); }

// ---- over LANES adjacent lanes (16: a row of the data-parallel moves, or the whole wave), all of them active ----
template <int CTRL, typename V>
__device__ __forceinline__ V moved(V v)
{
    return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
template <int LANES, typename V, typename F>
__device__ __forceinline__ V over_lanes(V v, F f)
{
    v = f(v, moved<0xB1>(v));    // quad_perm 1 0 3 2
    v = f(v, moved<0x4E>(v));    // quad_perm 2 3 0 1
    v = f(v, moved<0x141>(v));   // the other quad of eight
    v = f(v, moved<0x140>(v));   // the other eight of sixteen
    if constexpr (LANES == 64) {
        v = f(v, __shfl_xor(v, 16));
        v = f(v, __shfl_xor(v, 32));
    }
    return v;
}
template <int LANES> __device__ __forceinline__ float sum_of(float v) { return over_lanes<LANES>(v, [](float a, float b) { return a + b; }); }
template <int LANES> __device__ __forceinline__ float max_of(float v) { return over_lanes<LANES>(v, [](float a, float b) { return fmaxf(a, b); }); }
template <int LANES> __device__ __forceinline__ float min_of(float v) { return over_lanes<LANES>(v, [](float a, float b) { return fminf(a, b); }); }
template <int LANES> __device__ __forceinline__ unsigned max_of(unsigned v) { return over_lanes<LANES>(v, [](unsigned a, unsigned b) { return max(a, b); }); }
// of the next lane
template <int LANES, typename V>
__device__ __forceinline__ V next_lane(V v)
{
    if constexpr (LANES == 16) return moved<0x101>(v);   // row_shl 1
    else return __shfl(v, (threadIdx.x + 1) & 63);
}

// The weights w_j = s_j / (sum of the chosen s) of renormalised gates, in the lanes j that hold a chosen logit (there).
template <int LANES>
__device__ __forceinline__ float weight(bool sigmoids, float l, bool there)
{
    const float m = max_of<LANES>(there ? l : -INFINITY);
    float e;
    if (sigmoids && m >= -60.f) e = there ? sigmoid(l) : 0.f;
    else e = there ? expf(l - m) : 0.f;
    return e / sum_of<LANES>(e);
}

// ---- in 64 bits: any number of experts and groups -------------------------------------------------------
__device__ __forceinline__ double wave_sum(double v)
{
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
template <int CTRL>
__device__ __forceinline__ double max_moved(double v)
{
    const unsigned long long b = __builtin_bit_cast(unsigned long long, v);
    const unsigned lo = moved<CTRL>((unsigned)b), hi = moved<CTRL>((unsigned)(b >> 32));
    return fmax(v, __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo));
}
// The best (rank, lowest number) of the wave's lanes, -1 if all are -infinity.
__device__ __forceinline__ int best_of_wave(double rank, int number)
{
    double m = max_moved<0x140>(max_moved<0x141>(max_moved<0x4E>(max_moved<0xB1>(rank))));
    m = fmax(m, __shfl_xor(m, 16));
    m = fmax(m, __shfl_xor(m, 32));
    if (m == -INFINITY) return -1;
    return over_lanes<64>(rank == m ? number : 0x7FFFFFFF, [](int a, int b) { return min(a, b); });
}
// LDS accesses of a wave take place in order: only the compiler has to keep them so.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// One token by a whole wave; lane i looks after experts i, i + 64, ...; ranks, of, open: LDS, a.experts and twice a.groups of the wave's own.
// (Everything stays there: the kernel that calls this in the rare case shall not need registers for it.)
template <typename T>
__device__ __forceinline__ void route_exactly(const RouteArgs &a, long long token, double *ranks, double *of, unsigned char *open)
{
    int lane = threadIdx.x & 63, groups = a.groups;
    asm("" : "+v"(lane), "+s"(groups));   // (what hangs on these is not to be worked out ahead of a rare call)
    const T *logits = (const T *)a.logits + token * a.ld;
    bool bad = false;
    float high = -INFINITY;
#pragma unroll 1
    for (int e = lane; e < a.experts; e += 64) {
        const float l = Element<T>::get(logits + e);
        bad |= l != l || (!a.sigmoid && l == INFINITY);
        high = fmaxf(high, l);
        ranks[e] = l;
    }
    high = max_of<64>(high);
    const bool sums = groups > 1 && a.group_best > 1;
    if (a.bias || sums) {
        double total = 0.0;
        if (!a.sigmoid) {
#pragma unroll 1
            for (int e = lane; e < a.experts; e += 64) {
                const double l = ranks[e];
                if (l > -INFINITY) total += exp(l - (double)high);
            }
            total = wave_sum(total);
        }
#pragma unroll 1
        for (int e = lane; e < a.experts; e += 64) {
            const double l = ranks[e];
            if (l > -INFINITY) {
                const double x = exp(a.sigmoid ? -l : l - (double)high);
                double s = a.sigmoid ? 1.0 / (1.0 + x) : x / total;
                if (a.bias) s += (double)a.bias[e];
                bad |= s != s;
                ranks[e] = s;
            }
        }
    }
    in_order();
    if (groups > 1) {
        const int size = a.experts / groups;
#pragma unroll 1
        for (int g = lane; g < groups; g += 64) {
            double one = -INFINITY, two = -INFINITY;
#pragma unroll 4
            for (int q = 0; q < size; ++q) {
                const double r = ranks[g * size + q];
                two = fmax(two, fmin(one, r));
                one = fmax(one, r);
            }
            of[g] = a.group_best > 1 && two > -INFINITY ? one + two : one;
            open[g] = 0;
        }
        in_order();
#pragma unroll 1
        for (int k = 0; k < a.top_groups; ++k) {
            double best = -INFINITY;
            int number = 0;
#pragma unroll 1
            for (int g = lane; g < groups; g += 64)
                if (of[g] > best) { best = of[g]; number = g; }
            number = best_of_wave(best, number);
            if (number < 0) break;
            if ((number & 63) == lane) {
                open[number] = 1;
                of[number] = -INFINITY;
            }
        }
        in_order();
#pragma unroll 1
        for (int e = lane; e < a.experts; e += 64) {
            if (!open[e / size]) ranks[e] = -INFINITY;
            else if (sums && !a.bias) ranks[e] = Element<T>::get(logits + e);
        }
        in_order();
    }
    bad = __ballot(bad) != 0;
    int mine = -1;
#pragma unroll 1
    for (int k = 0; k < a.fan; ++k) {
        double best = -INFINITY;
        int number = 0;
#pragma unroll 4
        for (int e = lane; e < a.experts; e += 64) {
            const double r = ranks[e];
            if (r > best) { best = r; number = e; }
        }
        number = best_of_wave(best, number);
        if (bad || number < 0) break;
        if ((number & 63) == lane) ranks[number] = -INFINITY;
        if (lane == k) mine = number;
    }
    in_order();
    const bool there = mine >= 0;
    const float l = there ? Element<T>::get(logits + mine) : 0.f;
    float gate;
    if (a.renormalise) {
        gate = weight<64>(a.sigmoid, l, there);
    } else if (a.sigmoid) {
        gate = sigmoid(l);
    } else {
        float sum = 0.f;
#pragma unroll 1
        for (int e = lane; e < a.experts; e += 64) sum += expf(Element<T>::get(logits + e) - high);
        gate = expf(l - high) / sum_of<64>(sum);
    }
    if (lane < a.fan) {
        a.choice[token * a.fan + lane] = mine;
        a.gate[token * a.fan + lane] = bad ? __uint_as_float(0x7FC00000u) : there ? a.scale * gate : 0.f;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void route_general_kernel(const RouteArgs a)
{
    __shared__ double ranks[4][kMaxRouted], of[4][kMaxRouted];
    __shared__ unsigned char open[4][kMaxRouted];
    const int wave = threadIdx.x >> 6;
    for (long long token = (long long)blockIdx.x * 4 + wave; token < a.n; token += 4LL * gridDim.x) route_exactly<T>(a, token, ranks[wave], of[wave], open[wave]);
}

// ---- LANES lanes a token, EPL experts a lane -------------------------------------------------------------
// Lane i holds the `per` experts from i per on.  Ranks are formed in fp32 and brought into [1, 2); the bits of the fraction, with the
// experts' numbers from behind below them, are keys that all differ, and the largest is the choice.  The best one below M is M + max(key - M)
// in wrapping arithmetic: an element costs a subtraction and half a maximum in each round.  Where two neighbours among the chosen are
// nearer than the error of their ranks, and not exactly equal, the chosen ones are ranked in 64 bits, together with the first that is no choice if
// that one alone is as near to the last; where more are, or groups, or ranks are not finite, the wave does the token again in 64 bits (11 us for
// one token, much of it code that no cache holds yet; without the rank of the first that is no choice a launch that ends with such a token
// took 47 us instead of 40).  How near groups may be goes by the sizes of the ranks that are added, which can take most of each other away.
// Groups need to be whole lanes.
// Bound by its vector instructions: 65536 tokens, 256 experts, bf16, fan 8: sigmoids with a bias and the best 4 of 8 groups 39 us, softmax alone
// 27 us, for 34 MB of logits.  A workgroup is one wave: 32768 tokens, 512 experts 48 us, 52 with four.
template <typename T, int N>
__device__ __forceinline__ void load_logits(const T *p, int there, float (&v)[N])
{
    typedef T vec __attribute__((ext_vector_type(N), aligned(sizeof(T))));
    if (there >= N) {
        if constexpr (N == 8) {
            load8(p, v);
        } else if constexpr (N == 1) {
            v[0] = Element<T>::get(p);
        } else {
            const vec r = *(const vec *)p;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const T one = r[j];
                v[j] = Element<T>::get(&one);
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = j < there ? Element<T>::get(p + j) : -INFINITY;
    }
}

template <typename T, int N>
__device__ __forceinline__ void store_logits(T *p, int there, const float (&v)[N])
{
    typedef T vec __attribute__((ext_vector_type(N), aligned(sizeof(T))));
    if (there >= N) {
        if constexpr (N == 8) {
            store8(p, 8, v);
        } else if constexpr (N == 1) {
            Element<T>::put(p, v[0]);
        } else {
            vec r;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                T one;
                Element<T>::put(&one, v[j]);
                r[j] = one;
            }
            *(vec *)p = r;
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < there) Element<T>::put(p + j, v[j]);
    }
}

template <typename T, int LANES, int EPL>
__global__ __launch_bounds__(64, LANES == 64 ? 4 : EPL == 16 ? 5 : 6) void route_kernel(const RouteArgs a, int per, int group_lanes)
{
    constexpr int ALL = LANES * EPL, IB = ALL <= 16 ? 4 : ALL <= 32 ? 5 : ALL <= 64 ? 6 : ALL <= 128 ? 7 : ALL <= 256 ? 8 : ALL <= 512 ? 9 : 10;
    constexpr int ROWS = 64 / LANES, N = EPL < 8 ? EPL : 8;
    __shared__ double ranks[1][ALL], of_groups[1][LANES];   // (as many groups as lanes at most)
    __shared__ unsigned char opened[1][LANES];
    const int lane = threadIdx.x & 63, sub = lane & (LANES - 1), first = sub * per;
    const bool sums = a.groups > 1 && a.group_best > 1, by_score = a.bias || sums;
    for (long long base = (long long)blockIdx.x * ROWS; base < a.n; base += (long long)gridDim.x * ROWS) {
        const long long mine_at = base + threadIdx.x / LANES, token = mine_at < a.n ? mine_at : a.n - 1;   // (all lanes take part)
        const T *logits = (const T *)a.logits + token * a.ld;
        const int there = min(per, a.experts - first);
        float l[EPL], k[EPL];
#pragma unroll
        for (int i = 0; i < EPL; i += N) {
            float v[N];
            load_logits(logits + first + i, there - i, v);
#pragma unroll
            for (int j = 0; j < N; ++j) l[i + j] = v[j];
        }
        bool again = false;
#pragma unroll
        for (int i = 0; i < EPL; ++i) k[i] = l[i];
#pragma unroll
        for (int i = 0; i < EPL; i += 2) again |= __builtin_isunordered(l[i], l[EPL > 1 ? i + 1 : i]);
        float high = l[0];
#pragma unroll
        for (int i = 1; i < EPL; ++i) high = fmaxf(high, l[i]);
        high = max_of<LANES>(high);
        again |= high == INFINITY;
        float total = 1.f, error = 0.f;
        if (!a.sigmoid && (by_score || !a.renormalise)) {
            total = 0.f;
#pragma unroll
            for (int i = 0; i < EPL; ++i) {
                const float e = l[i] > -INFINITY ? __expf(l[i] - high) : 0.f;
                total += e;
                if (by_score) k[i] = e;
            }
            total = sum_of<LANES>(total);
        }
        if (by_score) {
            // errors: of sigmoids s (1 - s) (|l| 2^-24 + 2^-23) by the exponential, 2^-24 s by the sum, 2^-23 s by the reciprocal: below 2^-22;
            // of softmaxes below 2^-19 of the largest
            const float share = 1.f / total;
            error = a.sigmoid ? 0x1p-22f : 0x1p-19f * share;
            if (a.sigmoid) {
#pragma unroll
                for (int i = 0; i < EPL; ++i) k[i] = __builtin_amdgcn_rcpf(1.f + __expf(-l[i]));
            } else {
#pragma unroll
                for (int i = 0; i < EPL; ++i) k[i] *= share;
            }
            if (a.bias) {
#pragma unroll
                for (int i = 0; i < EPL; i += N) {
                    float v[N];
                    load_logits(a.bias + first + i, there - i, v);
#pragma unroll
                    for (int j = 0; j < N; ++j) k[i + j] += v[j];
#pragma unroll
                    for (int j = 0; j < N; j += 2) again |= __builtin_isunordered(v[j], v[N > 1 ? j + 1 : j]);
                }
            }
#pragma unroll
            for (int i = 0; i < EPL; ++i) k[i] = l[i] > -INFINITY ? k[i] : -INFINITY;
        }
        if (a.groups > 1) {
            float one = -INFINITY, two = -INFINITY;
#pragma unroll
            for (int i = 0; i < EPL; ++i) {
                two = fmaxf(two, fminf(one, k[i]));
                one = fmaxf(one, k[i]);
            }
            for (int o = 1; o < group_lanes; o <<= 1) {
                const float p = __shfl_xor(one, o), q = __shfl_xor(two, o);
                two = fmaxf(fmaxf(two, q), fminf(one, p));
                one = fmaxf(one, p);
            }
            const float of = a.group_best > 1 && two > -INFINITY ? one + two : one;
            int better = 0;
            for (int d = group_lanes; d < LANES; d += group_lanes) {
                const int other = (sub + d) & (LANES - 1);
                const float r = __shfl(of, lane - sub + other);
                better += r > of || (r == of && other < sub) ? 1 : 0;
            }
            const bool open = better < a.top_groups;
            if (by_score) {
                // errors: of each rank `error` and 2^-24 of it, of the sum 2^-24; they go by the ranks, which may take most of each other away
                const float magnitude = fabsf(one) + (a.group_best > 1 && two > -INFINITY ? fabsf(two) : 0.f);
                const float off = one > -INFINITY ? 2.f * error + 0x1p-22f * magnitude : 0.f;
                const float low = min_of<LANES>(open ? of - off : INFINITY), next = max_of<LANES>(open ? -INFINITY : of + off);
                // (a sum beyond fp32's range is not that of a closed group)
                again |= (next > -INFINITY && !(low > next)) || (one > -INFINITY && fabsf(of) == INFINITY);
            }
#pragma unroll
            for (int i = 0; i < EPL; ++i) k[i] = !open ? -INFINITY : sums && !a.bias ? l[i] : k[i];
            if (sums && !a.bias) error = 0.f;
        }
        // [1, 1 + width): 1 + 2^-13 at the least of the lanes' best ones, which the `fan` best and the next one mostly reach (where fewer lanes
        // than that are open: at the least open one), but 64 below the best at most; what is further below, or closed, is 1
        float best = k[0];
#pragma unroll
        for (int i = 1; i < EPL; ++i) best = fmaxf(best, k[i]);
        float low = best > -INFINITY ? best : INFINITY;
        if (a.groups > 1 && a.top_groups * group_lanes <= a.fan)
#pragma unroll
            for (int i = 0; i < EPL; ++i) low = k[i] > -INFINITY ? fminf(low, k[i]) : low;
        const float top = max_of<LANES>(best);
        low = fmaxf(min_of<LANES>(low), top - 64.f);
        again |= top == INFINITY;
        constexpr float width = IB <= 8 ? 1.f : IB == 9 ? 0.5f : 0.25f;   // what a shift by IB leaves of a fraction
        const float step = top > low ? fminf((width - 0x1p-10f) / (top - low), 0x1p100f) : 0x1p100f;
        // twice the error of a rank and of its rounding, and what the map adds
        const unsigned margin = error > 0.f ? (unsigned)(fminf(2.f * (error + 0x1p-23f * fmaxf(fabsf(top), fabsf(low))) * step, 1.f) * 0x1p23f) + 4u : 0u;
        unsigned key[EPL];
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            const float f = fmaxf(fmaf(k[i] - low, step, 1.f + 0x1p-13f), 1.f);
            key[i] = (__float_as_uint(f) << IB) + (unsigned)(ALL - 1 - first - i);
        }
        unsigned mine = 0, M = IB <= 8 ? 0u : 0x80000000u;   // (with up to 8 bits below it a 1 of the exponent is the highest bit)
        for (int r = 0; r <= a.fan; ++r) {
            unsigned far = key[0] - M;
#pragma unroll
            for (int i = 1; i < EPL; ++i) far = max(far, key[i] - M);
            M += max_of<LANES>(far);
            mine = sub == r ? M : mine;
        }
        constexpr unsigned one = 0x3F800000u << IB;   // (what is left of it)
        const bool open = top > -INFINITY;
        again |= open && sub < a.fan && mine - one < 1u << IB;   // closed, or too far below
        const int e = ALL - 1 - (int)(mine & (ALL - 1));
        const bool real = sub <= a.fan && e < a.experts;   // (the numbers behind a.experts are closed, too)
        const float chosen = real ? Element<T>::get(logits + e) : 0.f, added = real && a.bias ? a.bias[e] : 0.f;
        const unsigned next = next_lane<LANES>(mine);
        const bool equal = chosen == next_lane<LANES>(chosen) && added == next_lane<LANES>(added);
        const bool close = open && sub < a.fan && (mine >> IB) - (next >> IB) <= margin;
        const unsigned long long lanes_of_row = (LANES == 64 ? ~0ull : (1ull << (LANES & 63)) - 1) << (lane - sub);
        const unsigned long long edges = __ballot(close && sub == a.fan - 1);
        bool swaps = false;   // the first that is no choice may belong among them
        if (edges) {   // the last choice and the first that is none: whatever is as near as that is equal, or that one is alone
            const int last = lane - sub + a.fan - 1;
            const unsigned edge = __shfl(mine, last), after = __shfl(next, last);
            const float l0 = __shfl(chosen, last), b0 = __shfl(added, last);
            bool differs = false, others = after - one < 1u << IB;   // (that one is closed)
#pragma unroll
            for (int i = 0; i < EPL; ++i)
                if ((edges & lanes_of_row) && (key[i] >> IB) - (edge >> IB) + margin <= 2 * margin) {
                    const bool in = i < there;
                    differs |= !in || Element<T>::get(logits + (in ? first + i : 0)) != l0 || (a.bias && a.bias[in ? first + i : 0] != b0);
                    others |= key[i] - one < after - one;
                }
            differs = (__ballot(differs) & lanes_of_row) != 0;
            others = (__ballot(others) & lanes_of_row) != 0;
            again |= differs && others;
            swaps = differs && !others;
        }
        int place = sub;
        if (__ballot((close && sub < a.fan - 1 && !equal) || swaps)) {   // the chosen ones in 64 bits, their places counted
            double rank = chosen;
            if (error > 0.f) {
                double all = 1.0;
                if (!a.sigmoid) {
                    all = 0.0;
#pragma unroll 1
                    for (int q = sub; q < a.experts; q += LANES) {
                        const float x = Element<T>::get(logits + q);
                        if (x > -INFINITY) all += exp((double)x - (double)high);
                    }
                    for (int o = LANES / 2; o > 0; o >>= 1) all += __shfl_xor(all, o);
                }
                const double x = exp(a.sigmoid ? -(double)chosen : (double)chosen - (double)high);
                rank = (a.sigmoid ? 1.0 / (1.0 + x) : x / all) + (double)added;
            }
            int better = 0;
            const int ranked = a.fan + (swaps ? 1 : 0);
            for (int q = 0; q <= a.fan; ++q) {
                const double r = __shfl(rank, lane - sub + q);
                const int number = __shfl(e, lane - sub + q);
                better += q < ranked && (r > rank || (r == rank && number < e)) ? 1 : 0;
            }
            if (open && sub < ranked) place = better;   // (a closed token beside has no ranks: of a softmax they would be NaN)
        }
        const unsigned long long rows = __ballot(again);
        const bool mine_again = (rows & lanes_of_row) != 0;
        const bool chosen_one = open && place < a.fan;
        float gate;
        if (a.renormalise) gate = weight<LANES>(a.sigmoid, chosen, chosen_one);
        else gate = a.sigmoid ? sigmoid(chosen) : expf(chosen - high) / total;
        if (place < a.fan && mine_at < a.n && !mine_again) {
            a.choice[token * a.fan + place] = chosen_one ? e : -1;
            a.gate[token * a.fan + place] = chosen_one ? a.scale * gate : 0.f;
        }
        if (rows)
            for (int r = 0; r < 64 / LANES; ++r) {
                const long long t = base + (threadIdx.x >> 6) * (64 / LANES) + r;
                if ((rows >> (LANES * r) & (LANES == 64 ? ~0ull : (1ull << (LANES & 63)) - 1)) && t < a.n)
                    route_exactly<T>(a, t, ranks[threadIdx.x >> 6], of_groups[threadIdx.x >> 6], opened[threadIdx.x >> 6]);
            }
    }
}

// ---- gradient -------------------------------------------------------------------------------------------
// LANES lanes a token; lane i < fan works on choice i, then every lane on chunks of N adjacent experts.  A row of zeros with the
// choices' parts in their places is put together in LDS (an expert that is there twice gets the sum in the order of the choices).
// Bound by memory: 65536 tokens, 256 experts, bf16, renormalised: 15.7 us for the 34 MB that it writes and the lines of the chosen logits (55
// before rows were put together in LDS).
template <typename T, int LANES, int EPL>
__global__ __launch_bounds__(256) void route_grad_kernel(const RouteArgs a)
{
    constexpr int ROWS = 256 / LANES, N = EPL < 8 ? EPL : 8, ALL = LANES * EPL;
    __shared__ __attribute__((aligned(16))) float rows[ROWS][ALL];
    const int lane = threadIdx.x & 63, sub = lane & (LANES - 1);
    float *const row = rows[threadIdx.x / LANES];
    for (long long base = (long long)blockIdx.x * ROWS; base < a.n; base += (long long)gridDim.x * ROWS) {
        const long long at = base + threadIdx.x / LANES, token = at < a.n ? at : a.n - 1;   // (all lanes take part)
        const T *logits = (const T *)a.logits + token * a.ld;
        int mine = sub < a.fan ? a.choice[token * a.fan + sub] : -1;
        const bool there = mine >= 0 && mine < a.experts;
        if (!there) mine = -1;
        const float up = there ? a.scale * a.dgate[token * a.fan + sub] : 0.f;
        float part = 0.f, common = 0.f, s[EPL];   // of the lane's choice; what all experts lose; their scores (softmax)
#pragma unroll
        for (int i = 0; i < EPL; ++i) s[i] = 0.f;
        if (a.renormalise) {
            const float l = there ? Element<T>::get(logits + mine) : 0.f, w = weight<LANES>(a.sigmoid, l, there), mean = sum_of<LANES>(there ? up * w : 0.f);
            part = there ? w * (up - mean) : 0.f;
            if (a.sigmoid) part *= sigmoid(-l);
        } else if (a.sigmoid) {
            const float l = there ? Element<T>::get(logits + mine) : 0.f;
            part = up * sigmoid(l) * sigmoid(-l);
        } else {
            float high = -INFINITY, total = 0.f;
#pragma unroll
            for (int i = 0; i < EPL; i += N) {
                const int e = (i / N * LANES + sub) * N;
                float v[N];
                load_logits(logits + e, a.experts - e, v);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    s[i + j] = v[j];
                    high = fmaxf(high, v[j]);
                }
            }
            high = max_of<LANES>(high);
            const float l = there ? Element<T>::get(logits + mine) : 0.f;
#pragma unroll
            for (int i = 0; i < EPL; ++i) {
                s[i] = s[i] == -INFINITY ? 0.f : expf(s[i] - high);
                total += s[i];
            }
            const float share = 1.f / sum_of<LANES>(total);
            const bool any = max_of<LANES>(there ? 1u : 0u) != 0;   // a token without a choice gets zeros, whatever its logits
#pragma unroll
            for (int i = 0; i < EPL; ++i) s[i] = any ? s[i] * share : 0.f;
            part = there ? up * (expf(l - high) * share) : 0.f;
            common = sum_of<LANES>(part);
        }
        // the sum over equal choices, by the first of them
        float sum = 0.f;
        bool first = there;
        for (int j = 0; j < a.fan; ++j) {
            const int c = __shfl(mine, lane - sub + j);
            const float p = __shfl(part, lane - sub + j);
            sum += c == mine ? p : 0.f;
            first = first && !(j < sub && c == mine);
        }
        in_order();
#pragma unroll
        for (int i = 0; i < EPL; i += N)
#pragma unroll
            for (int j = 0; j < N; ++j) row[(i / N * LANES + sub) * N + j] = 0.f;
        in_order();
        if (first) row[mine] = sum;
        in_order();
#pragma unroll
        for (int i = 0; i < EPL; i += N) {
            const int e = (i / N * LANES + sub) * N;
            float v[N];
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = row[e + j] - common * s[i + j];
            if (at < a.n) store_logits((T *)a.dlogits + token * a.ldd + e, a.experts - e, v);
        }
        in_order();
    }
}

// A launch takes less than 2^32 threads; the kernels go on from there.
dim3 workgroups(int n, int rows, int most = 1 << 20) { return dim3((unsigned)min((n + rows - 1) / rows, most)); }

template <typename T, int LANES, int EPL>
hipError_t run(const RouteArgs &a, hipStream_t s)
{
    route_kernel<T, LANES, EPL><<<workgroups(a.n, 64 / LANES), dim3(64), 0, s>>>(a, (a.experts + LANES - 1) / LANES, LANES / a.groups);
    return hipGetLastError();
}

template <typename T>
hipError_t run(const RouteArgs &a, hipStream_t s)
{
    // sixteen lanes as far as sixteen experts a lane stay in registers: four tokens share the wave's moves between lanes (65536 tokens
    // of 256 experts 39 and 27 us, a token a wave 76 and 52)
    const int lanes = a.experts <= 256 ? 16 : 64, per = (a.experts + lanes - 1) / lanes;
    // what has no lane for each choice and the next one, or groups that are no whole lanes, goes through 64 bits, a token a wave (65536 tokens, bf16:
    // 60 experts in 4 groups, fan 6: 179 - 189 us, 64 in 4 groups 18; 64 experts, fan 16: 260 - 272, fan 15: 19; 256 in 8 groups, fan 16: 464, fan 15: 44)
    if (a.fan >= lanes || (a.groups > 1 && (lanes % a.groups || a.experts % lanes))) {
        route_general_kernel<T><<<workgroups(a.n, 4), dim3(256), 0, s>>>(a);
        return hipGetLastError();
    }
    if (lanes == 64) return per <= 8 ? run<T, 64, 8>(a, s) : run<T, 64, 16>(a, s);
    if (per <= 1) return run<T, 16, 1>(a, s);
    if (per <= 2) return run<T, 16, 2>(a, s);
    if (per <= 4) return run<T, 16, 4>(a, s);
    return per <= 8 ? run<T, 16, 8>(a, s) : run<T, 16, 16>(a, s);
}

template <typename T, int LANES, int EPL>
hipError_t run_grad(const RouteArgs &a, hipStream_t s)
{
    route_grad_kernel<T, LANES, EPL><<<workgroups(a.n, 256 / LANES), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

template <typename T>
hipError_t run_grad(const RouteArgs &a, hipStream_t s)
{
    const int lanes = a.experts <= 256 && a.fan <= 16 ? 16 : 64, per = (a.experts + lanes - 1) / lanes;
    if (lanes == 64) return per <= 4 ? run_grad<T, 64, 4>(a, s) : per <= 8 ? run_grad<T, 64, 8>(a, s) : run_grad<T, 64, 16>(a, s);
    if (per <= 1) return run_grad<T, 16, 1>(a, s);
    if (per <= 2) return run_grad<T, 16, 2>(a, s);
    if (per <= 4) return run_grad<T, 16, 4>(a, s);
    return per <= 8 ? run_grad<T, 16, 8>(a, s) : run_grad<T, 16, 16>(a, s);
}

}  // namespace

hipError_t launch_route(const RouteArgs &a, int bf16, hipStream_t s) { return bf16 ? run<bf16_bits>(a, s) : run<float>(a, s); }
hipError_t launch_route_grad(const RouteArgs &a, int bf16, hipStream_t s) { return bf16 ? run_grad<bf16_bits>(a, s) : run_grad<float>(a, s); }

}  // namespace kfac
