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

constexpr int kPer = kMaxRouted / 64;   // experts a lane, at most

__device__ __forceinline__ float sigmoid(float l) { return 1.f / (1.f + expf(-l)); }

template <typename V>
__device__ __forceinline__ V wave_sum(V v)
{
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
__device__ __forceinline__ float wave_max(float v)
{
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}

// The best (rank, lowest number) of the wave's lanes; number < 0: none.
__device__ __forceinline__ void best_of_wave(double &rank, int &number)
{
    for (int o = 32; o > 0; o >>= 1) {
        const double r = __shfl_xor(rank, o);
        const int n = __shfl_xor(number, o);
        if (n >= 0 && (number < 0 || r > rank || (r == rank && n < number))) { rank = r; number = n; }
    }
}

// The weights w_j = s_j / (sum of the chosen s) of renormalised gates, in the lanes j that hold a chosen logit (there).
__device__ __forceinline__ float weight(bool sigmoids, float l, bool there)
{
    const float m = wave_max(there ? l : -INFINITY);
    float e;
    if (sigmoids && m >= -60.f) e = there ? sigmoid(l) : 0.f;
    else e = there ? expf(l - m) : 0.f;
    return e / wave_sum(e);
}

// One wave a token; lane i holds experts i, i + 64, ...
template <typename T>
__global__ __launch_bounds__(256) void route_kernel(const RouteArgs a)
{
    __shared__ double ranks[4][kMaxRouted];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const bool by_score = a.bias || (a.groups > 1 && a.group_best > 1);
    for (long long token = (long long)blockIdx.x * 4 + wave; token - wave < a.n; token += 4LL * gridDim.x) {
        if (token < a.n) {
            const T *logits = (const T *)a.logits + token * a.ld;
            double rank[kPer];
            bool bad = false;
            float high = -INFINITY;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int e = lane + 64 * i;
                rank[i] = -INFINITY;
                if (e < a.experts) {
                    const float l = Element<T>::get(logits + e);
                    rank[i] = l;
                    bad |= l != l || (!a.sigmoid && l == INFINITY);
                    high = fmaxf(high, l);
                }
            }
            high = wave_max(high);
            double total = 0.0;
            if (by_score) {
                if (!a.sigmoid) {
#pragma unroll
                    for (int i = 0; i < kPer; ++i)
                        if (rank[i] > -INFINITY) total += exp(rank[i] - (double)high);
                    total = wave_sum(total);
                }
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    const int e = lane + 64 * i;
                    if (rank[i] > -INFINITY) {
                        double s = a.sigmoid ? 1.0 / (1.0 + exp(-rank[i])) : exp(rank[i] - (double)high) / total;
                        if (a.bias) s += (double)a.bias[e];
                        bad |= s != s;
                        rank[i] = s;
                    }
                }
            }
            if (a.groups > 1) {
                const int size = a.experts / a.groups;
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (lane + 64 * i < a.experts) ranks[wave][lane + 64 * i] = rank[i];
                __builtin_amdgcn_wave_barrier();
                __threadfence_block();
                // lanes take groups in turn; the ranks of groups replace those of their first experts afterwards
                double group_rank[kPer];
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    const int g = lane + 64 * i;
                    double one = -INFINITY, two = -INFINITY;
                    if (g < a.groups)
                        for (int q = 0; q < size; ++q) {
                            const double r = ranks[wave][g * size + q];
                            if (r > one) { two = one; one = r; }
                            else if (r > two) two = r;
                        }
                    group_rank[i] = a.group_best > 1 && two > -INFINITY ? one + two : one;
                }
                unsigned open = 0;   // of the lane's groups
                for (int k = 0; k < a.top_groups; ++k) {
                    double best = -INFINITY;
                    int number = -1;
#pragma unroll
                    for (int i = 0; i < kPer; ++i)
                        if (!(open >> i & 1) && group_rank[i] > best) { best = group_rank[i]; number = lane + 64 * i; }
                    best_of_wave(best, number);
                    if (number < 0) break;
                    if ((number & 63) == lane) open |= 1u << (number >> 6);
                }
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (lane + 64 * i < a.groups) ranks[wave][lane + 64 * i] = open >> i & 1 ? 1.0 : 0.0;
                __builtin_amdgcn_wave_barrier();
                __threadfence_block();
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    const int e = lane + 64 * i;
                    if (e < a.experts && ranks[wave][e / size] == 0.0) rank[i] = -INFINITY;
                }
                __builtin_amdgcn_wave_barrier();
            }
            bad = __ballot(bad) != 0;
            int mine = -1;
            for (int k = 0; k < a.fan; ++k) {
                double best = -INFINITY;
                int number = -1;
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (rank[i] > best) { best = rank[i]; number = lane + 64 * i; }
                best_of_wave(best, number);
                if (bad || number < 0) break;
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (number == lane + 64 * i) rank[i] = -INFINITY;
                if (lane == k) mine = number;
            }
            const bool there = mine >= 0;
            const float l = there ? Element<T>::get(logits + mine) : 0.f;
            float gate;
            if (a.renormalise) {
                gate = weight(a.sigmoid, l, there);
            } else if (a.sigmoid) {
                gate = sigmoid(l);
            } else {
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (lane + 64 * i < a.experts) sum += expf(Element<T>::get(logits + lane + 64 * i) - high);
                gate = expf(l - high) / wave_sum(sum);
            }
            if (lane < a.fan) {
                a.choice[token * a.fan + lane] = mine;
                a.gate[token * a.fan + lane] = bad ? __uint_as_float(0x7FC00000u) : there ? a.scale * gate : 0.f;
            }
        }
    }
}

// One wave a token.
template <typename T>
__global__ __launch_bounds__(256) void route_grad_kernel(const RouteArgs a)
{
    const int lane = threadIdx.x & 63;
    for (long long token = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); token < a.n; token += 4LL * gridDim.x) {
        const T *logits = (const T *)a.logits + token * a.ld;
        T *out = (T *)a.dlogits + token * a.ldd;
        int mine = lane < a.fan ? a.choice[token * a.fan + lane] : -1;
        const bool there = mine >= 0 && mine < a.experts;
        const float l = there ? Element<T>::get(logits + mine) : 0.f, up = there ? a.scale * a.dgate[token * a.fan + lane] : 0.f;
        if (!there) mine = -1;
        const bool any = __ballot(there) != 0;
        float part = 0.f, common = 0.f, high = 0.f, share = 0.f;   // of the lane's choice; what all experts lose (softmax); their score
        if (a.renormalise) {
            const float w = weight(a.sigmoid, l, there), mean = wave_sum(there ? up * w : 0.f);
            part = there ? w * (up - mean) : 0.f;
            if (a.sigmoid) part *= sigmoid(-l);
        } else if (a.sigmoid) {
            part = up * sigmoid(l) * sigmoid(-l);
        } else if (any) {
            high = -INFINITY;
            for (int e = lane; e < a.experts; e += 64) high = fmaxf(high, Element<T>::get(logits + e));
            high = wave_max(high);
            float sum = 0.f;
            for (int e = lane; e < a.experts; e += 64) sum += expf(Element<T>::get(logits + e) - high);
            share = 1.f / wave_sum(sum);
            part = there ? up * (expf(l - high) * share) : 0.f;
            common = wave_sum(part);
        }
        for (int e0 = 0; e0 < a.experts; e0 += 64) {
            const int e = e0 + lane;
            float sum = 0.f;
            for (int j = 0; j < a.fan; ++j) {
                const int c = __shfl(mine, j);
                const float p = __shfl(part, j);
                sum += c == e ? p : 0.f;
            }
            if (e < a.experts) {
                if (share != 0.f) sum -= common * (expf(Element<T>::get(logits + e) - high) * share);
                Element<T>::put(out + e, sum);
            }
        }
    }
}

template <typename K>
hipError_t run(K kernel, const RouteArgs &a, hipStream_t s)
{
    const int wgs = (a.n + 3) / 4;
    kernel<<<dim3((unsigned)(wgs < (1 << 20) ? wgs : (1 << 20))), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_route(const RouteArgs &a, int bf16, hipStream_t s) { return bf16 ? run(route_kernel<bf16_bits>, a, s) : run(route_kernel<float>, a, s); }
hipError_t launch_route_grad(const RouteArgs &a, int bf16, hipStream_t s)
{
    return bf16 ? run(route_grad_kernel<bf16_bits>, a, s) : run(route_grad_kernel<float>, a, s);
}

}  // namespace kfac
