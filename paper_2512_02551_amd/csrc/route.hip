// The choice of experts for each token, the order of the rows it gives, and the gradient of the logits.
//
// A wave takes a token: lane l holds the experts L l .. L l + L - 1.  The k best are found one after another: the largest key over the wave (a
// reduction in the registers), then the lowest lane that has it, which is the lowest index among equal keys; only that lane looks for its
// next best.  Logits of 16 bits that are the keys themselves share a word with their index, so that the largest word is the choice (15999 x 128 in
// fp16: 14.9 us, 17 without).  What bounds it: the instructions of these rounds, some 25 or 15 each, and for few tokens the launch.  15999 tokens of 128
// experts, 8 chosen: 15 us, their order 8.5, their gradient 9 (memory would take 3); 32 tokens of 256 experts 8 us in one launch.
//
// The order is a stable counting sort by expert.  An expert holds one bit for each token of a workgroup that chose it, so a choice's rank
// within the workgroup is a population count, and its place is its expert's first row, plus the choices of earlier workgroups, plus that rank.
// Up to 128 tokens are chosen for by workgroups of four (32 tokens of 256 experts on one compute unit: 13 us, its issue slots are the bound), and the one
// that arrives last orders them all.  For more, a second launch takes 128 tokens a workgroup, each of which sums the counts of all (500 x 128 counts
// of 16000 tokens are 64 KB of cache, and a launch in between costs more).  That grows with the square of the tokens and is felt from some 100000 on: 65536 tokens
// of 256 experts 112 us, 131072 286, 262144 828.  No result depends on the order of atomics.
#include <new>
#include <type_traits>

#include "experts_common.hpp"
#include "hgemm_mfma.hpp"          // last_to_arrive

using namespace hgemm;

namespace {

constexpr int kMostExperts = 1024, kMostChoices = 32;
constexpr int kRouteTokens = 32, kFewTokens = 4, kPlaceTokens = 128;    // tokens of a workgroup that chooses (of few tokens), and of one that places

struct RouteArgs {
    const void* logits;
    const float* bias;
    float* weights;
    int* experts;
    int* offsets;
    int* rows;
    int* tokens_of;
    uint8_t* counts;        // [blocks of kRouteTokens tokens][E rounded up to 4]: choices of each expert
    int64_t ld, capacity;
    int tokens, E, k;
    int type, sigmoid, groups, keep, top2, renormalise, align;
    float factor;
    const float* dweights;
    void* dlogits;
    int* arrived;           // few tokens: workgroups that have chosen, zero between launches
    int blocks;             // workgroups that choose
    int wide;               // a lane's logits are one aligned word of 4 to 16 bytes, whole or absent
};

// Orders like the value, equal for +0 and -0, and above 0.
__device__ __forceinline__ unsigned sortable(float v)
{
    const unsigned u = __builtin_bit_cast(unsigned, v + 0.f);
    return u >> 31 ? ~u : u | 0x80000000u;
}

// Reductions over a wave without a trip through LDS; `none` is the operation's neutral element.  The result is uniform.
template <int CTRL, int ROWS> __device__ __forceinline__ int moved(int none, int v) { return __builtin_amdgcn_update_dpp(none, v, CTRL, ROWS, 0xf, false); }
template <class F> __device__ __forceinline__ int reduce(int v, int none, F&& f)
{
    v = f(v, moved<0x111, 0xf>(none, v));               // row_shr: 1, 2, 4, 8, then the rows' last lanes onwards
    v = f(v, moved<0x112, 0xf>(none, v));
    v = f(v, moved<0x114, 0xf>(none, v));
    v = f(v, moved<0x118, 0xf>(none, v));
    v = f(v, moved<0x142, 0xa>(none, v));
    v = f(v, moved<0x143, 0xc>(none, v));
    return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ float as_f(int v) { return __builtin_bit_cast(float, v); }
__device__ __forceinline__ int as_i(float v) { return __builtin_bit_cast(int, v); }
// A maximum may meet a lane twice: all rows take part, and the moves fold into the comparisons.
template <int CTRL> __device__ __forceinline__ unsigned max_with(unsigned v) { return max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true)); }
__device__ __forceinline__ unsigned wave_max(unsigned v)
{
    v = max_with<0x111>(v);
    v = max_with<0x112>(v);
    v = max_with<0x114>(v);
    v = max_with<0x118>(v);
    v = max_with<0x142>(v);
    v = max_with<0x143>(v);
    return (unsigned)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ __forceinline__ float wave_max(float v) { return as_f(reduce(as_i(v), as_i(-__builtin_inff()), [](int x, int y) { return as_i(fmaxf(as_f(x), as_f(y))); })); }
__device__ __forceinline__ float wave_sum(float v) { return as_f(reduce(as_i(v), 0, [](int x, int y) { return as_i(as_f(x) + as_f(y)); })); }

// Keys of a wave, L a lane (0: none), taken one after another, the largest first, of equal ones that of the lowest index.
template <int L> struct Keys {
    unsigned key[L], best;
    int at;
    __device__ __forceinline__ void look()
    {
        best = key[0];
        at = 0;
#pragma unroll
        for (int i = 1; i < L; ++i)
            if (key[i] > best) { best = key[i]; at = i; }
    }
    // The index of the next one, -1 where there is none.
    __device__ __forceinline__ int take(int lane)
    {
        const unsigned most = wave_max(best);
        if (most == 0) return -1;
        const int owner = __builtin_ctzll(__ballot(best == most));
        const int index = owner * L + (L > 1 ? __builtin_amdgcn_readlane(at, owner) : 0);
#pragma unroll
        for (int i = 0; i < L; ++i) key[i] = lane * L + i == index ? 0u : key[i];
        look();
        return index;
    }
};

// The value and its index in one word, for values of 16 bits: larger values are larger words, and of equal ones that of the lower index.
__device__ __forceinline__ unsigned word_of(float v, bool half, int index)
{
    const unsigned short u = half ? __builtin_bit_cast(unsigned short, (_Float16)(v + 0.f)) : (unsigned short)(__builtin_bit_cast(unsigned, v + 0.f) >> 16);
    return (unsigned)(unsigned short)(u >> 15 ? ~u : u | 0x8000u) << 16 | (0xffffu - index);
}

// What the wave's lanes wrote to LDS is there for its other lanes.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ float sigmoid_of(float x) { return 1.f / (1.f + expf(-x)); }

// Largest logit (0 where all are -infinity) and the sum of exponentials: what a softmax needs.  The largest adds 1 to the sum, so a sum below that is the 0 of a row
// without any, and counts as 1; a NaN, of an infinite logit, stays.
template <int L> __device__ __forceinline__ void softmax_of(const float (&x)[L], float& top, float& sum)
{
    top = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < L; ++i) top = fmaxf(top, x[i]);
    top = wave_max(top);
    if (top == -__builtin_inff()) top = 0.f;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < L; ++i) sum += expf(x[i] - top);
    sum = wave_sum(sum);
    sum = sum < 1.f ? 1.f : sum;
}

// The running sum over the lanes.
__device__ __forceinline__ int wave_scan(int v)
{
    v += moved<0x111, 0xf>(0, v);
    v += moved<0x112, 0xf>(0, v);
    v += moved<0x114, 0xf>(0, v);
    v += moved<0x118, 0xf>(0, v);
    v += moved<0x142, 0xa>(0, v);
    return v + moved<0x143, 0xc>(0, v);
}

// What a workgroup needs to order the rows of its tokens.
struct OrderLds {
    unsigned long long chose[2][kMostExperts];          // bit t % 64 of half t / 64: token t of the workgroup chose the expert
    int total[kMostExperts], before[kMostExperts];      // choices of all tokens, and of those of earlier workgroups
    int first[kMostExperts];                            // first row
    int sums[16];
    int end;                                            // the row behind the last expert's
    int chosen[kPlaceTokens * kMostChoices];            // the workgroup's choices
};

// The choices of all tokens and of those before workgroup b's, from the counts of the first launch.
__device__ __forceinline__ void sum_counts(const RouteArgs& a, OrderLds& o, int b)
{
    const int t = threadIdx.x, words = (a.E + 3) / 4;
    int wide = 16;                                      // threads side by side on a row of counts, four experts each
    while (wide < words) wide *= 2;
    const int groups = 1024 / wide, e = t % wide, c = t / wide, mine = b * (kPlaceTokens / kRouteTokens);
    int total[4] = {}, before[4] = {};
    if (e >= words) return;
#pragma unroll 16
    for (int r = c; r < a.blocks; r += groups) {
        const unsigned n = ((const unsigned*)a.counts)[(int64_t)r * words + e];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int x = n >> (8 * i) & 255;
            total[i] += x;
            before[i] += r < mine ? x : 0;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (4 * e + i < a.E) {
            atomicAdd(&o.total[4 * e + i], total[i]);
            atomicAdd(&o.before[4 * e + i], before[i]);
        }
}

// The choices of workgroup b's tokens to LDS, and, not FEW, the sums of counts: their loads travel together.  FEW: written in this launch by other workgroups.
template <bool FEW> __device__ __forceinline__ void take_choices(const RouteArgs& a, OrderLds& o, int b)
{
    if ((int)threadIdx.x < a.E) {
        o.chose[0][threadIdx.x] = o.chose[1][threadIdx.x] = 0;
        o.total[threadIdx.x] = o.before[threadIdx.x] = 0;
    }
    const int64_t lo = (int64_t)b * kPlaceTokens * a.k;
    const int tokens = min(kPlaceTokens, a.tokens - b * kPlaceTokens);
    auto choice = [&](int i) { return FEW ? __hip_atomic_load(&a.experts[lo + i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : a.experts[lo + i]; };
    int next = (int)threadIdx.x < tokens * a.k ? choice(threadIdx.x) : -1;
    __syncthreads();
    if constexpr (!FEW) sum_counts(a, o, b);
    for (int i = threadIdx.x; i < tokens * a.k; i += 1024) {
        const int e = next;
        if (i + 1024 < tokens * a.k) next = choice(i + 1024);
        const int token = (int)((unsigned)i / (unsigned)a.k);
        o.chosen[i] = e;
        if (e >= 0) atomicOr(&o.chose[token >> 6][e], 1ull << (token & 63));
    }
    __syncthreads();
}

// The places of workgroup b's choices, and its share of the padding.  `chose` and `chosen` hold them; 1024 threads.  Rows are below 2^31.
__device__ __forceinline__ void place(const RouteArgs& a, OrderLds& o, int b)
{
    const int t = threadIdx.x;
    if (a.tokens <= kPlaceTokens && t < a.E) { o.total[t] = __popcll(o.chose[0][t]) + __popcll(o.chose[1][t]); o.before[t] = 0; }
    __syncthreads();
    // first rows: a running sum over the experts, each padded
    const int mine = t < a.E ? (int)((unsigned)(o.total[t] + a.align - 1) / (unsigned)a.align) * a.align : 0;
    int sum = wave_scan(mine);
    if ((t & 63) == 63) o.sums[t >> 6] = sum;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 16; ++w) sum += w < t >> 6 ? o.sums[w] : 0;
    if (t < a.E) {
        o.first[t] = sum - mine;
        if (t == a.E - 1) o.end = sum;
        if (b == 0) a.offsets[t + 1] = sum;
        if (b == 0 && t == 0) a.offsets[0] = 0;
    }
    __syncthreads();
    const int tokens = min(kPlaceTokens, a.tokens - b * kPlaceTokens);
    for (int i = t; i < tokens * a.k; i += 1024) {
        const int e = o.chosen[i], token = (int)((unsigned)i / (unsigned)a.k);
        int row = -1;
        if (e >= 0) {
            const unsigned long long earlier = (1ull << (token & 63)) - 1, own = o.chose[token >> 6][e] & earlier;
            row = o.first[e] + o.before[e] + __popcll(own) + (token >= 64 ? __popcll(o.chose[0][e]) : 0);
            a.tokens_of[row] = b * kPlaceTokens + token;
        }
        a.rows[(int64_t)b * kPlaceTokens * a.k + i] = row;
    }
    // padding: of some experts, a wave each, and behind the last
    const int parts = a.tokens <= kPlaceTokens ? 1 : gridDim.x;
    if (a.align > 1)
        for (int e = b * 16 + (t >> 6); e < a.E; e += parts * 16) {
            const int to = e + 1 < a.E ? o.first[e + 1] : o.end;
            for (int r = o.first[e] + o.total[e] + (t & 63); r < to; r += 64) a.tokens_of[r] = -1;
        }
    for (int64_t r = o.end + (int64_t)b * 1024 + t; r < a.capacity; r += (int64_t)parts * 1024) a.tokens_of[r] = -1;
}

template <class T, int L> __device__ __forceinline__ void load_logits(const RouteArgs& a, int64_t t, int lane, float (&x)[L])
{
    const T* p = (const T*)a.logits + t * a.ld + lane * L;
    if constexpr (sizeof(T) * L >= 4 && sizeof(T) * L <= 16) {
        if (a.wide) {                                   // a lane's logits are one aligned word, there or not as a whole
            struct alignas(sizeof(T) * L) Word { T v[L]; } w;
            if (lane * L < a.E) w = *(const Word*)p;
#pragma unroll
            for (int i = 0; i < L; ++i) {
                const float v = (float)w.v[i];
                x[i] = lane * L < a.E && v == v ? v : -__builtin_inff();
            }
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < L; ++i) {
        x[i] = -__builtin_inff();
        if (lane * L + i < a.E) {
            const float v = (float)p[i];
            if (v == v) x[i] = v;
        }
    }
}
template <int L> __device__ __forceinline__ void load_logits(const RouteArgs& a, int64_t t, int lane, float (&x)[L])
{
    if (a.type == HGEMM_F16) load_logits<_Float16>(a, t, lane, x);
    else if (a.type == HGEMM_BF16) load_logits<__bf16>(a, t, lane, x);
    else load_logits<float>(a, t, lane, x);
}

// (first, second): the two largest of them and of v.
__device__ __forceinline__ void two_largest(float& first, float& second, float v)
{
    second = fmaxf(second, fminf(first, v));
    first = fmaxf(first, v);
}

// Keys of experts outside the best groups become -infinity.  Groups of whole lanes (a multiple of L experts) are scored from the lanes' own two
// largest, a power of two of lanes without LDS; others, key by key.
template <int L> __device__ __forceinline__ void keep_groups(const RouteArgs& a, int lane, float* lds, float (&key)[L])
{
    const float NONE = -__builtin_inff();
    const int size = a.E / a.groups;
    auto score = [&](float first, float second) { return a.top2 && second > NONE ? first + second : first; };
    if (size % L == 0) {
        const int per = size / L, lead = lane / per * per;                  // lanes of a group, its first
        float first = NONE, second = NONE;
#pragma unroll
        for (int i = 0; i < L; ++i) two_largest(first, second, key[i]);
        if ((per & (per - 1)) == 0) {
            for (int d = 1; d < per; d *= 2) {
                const float f = __shfl_xor(first, d), g = __shfl_xor(second, d);
                two_largest(first, second, f);
                second = fmaxf(second, g);
            }
        } else {
            lds[lane] = first;
            if (L > 1) lds[64 + lane] = second;
            wave_sync();
            if (lane == lead)
                for (int d = 1; d < per && lane + d < 64; ++d) {
                    two_largest(first, second, lds[lane + d]);
                    if (L > 1) second = fmaxf(second, lds[64 + lane + d]);
                }
            wave_sync();
        }
        first = score(first, second);
        Keys<1> left;
        left.key[0] = lane == lead && lane * L < a.E && first > NONE ? sortable(first) : 0u;
        left.look();
        uint64_t kept = 0;                              // bit: the first lane of a group that stays
        for (int j = 0; j < a.keep; ++j) {
            const int g = left.take(lane);
            if (g < 0) break;
            kept |= 1ull << g;
        }
        if (!(kept >> lead & 1)) {
#pragma unroll
            for (int i = 0; i < L; ++i) key[i] = NONE;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < L; ++i) lds[lane * L + i] = key[i];
    wave_sync();
    Keys<L> left;
#pragma unroll
    for (int i = 0; i < L; ++i) {
        const int g = lane * L + i;
        float first = NONE, second = NONE;
        if (g < a.groups)
            for (int j = 0; j < size; ++j) two_largest(first, second, lds[g * size + j]);
        first = score(first, second);
        left.key[i] = g < a.groups && first > NONE ? sortable(first) : 0u;
    }
    left.look();
    wave_sync();
    unsigned kept = 0;                                  // bit i: group lane L + i stays
    for (int j = 0; j < a.keep; ++j) {
        const int g = left.take(lane);
        if (g < 0) break;
        if (g / L == lane) kept |= 1u << (g % L);
    }
#pragma unroll
    for (int i = 0; i < L; ++i)
        if (lane * L + i < a.groups) lds[lane * L + i] = kept >> i & 1 ? 1.f : 0.f;
    wave_sync();
#pragma unroll
    for (int i = 0; i < L; ++i) {
        const int e = lane * L + i;
        if (e < a.E && lds[e / size] == 0.f) key[i] = NONE;
    }
    wave_sync();
}

// 16 waves; 32 tokens, or FEW: four, and in the workgroup that arrives last the order of all.  L = experts per lane.
template <int L, bool FEW> __global__ __launch_bounds__(1024) void route_kernel(RouteArgs a)
{
    constexpr int TOKENS = FEW ? kFewTokens : kRouteTokens;
    constexpr int WAVES = 16;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    __shared__ float keys[WAVES][64 * L];
    __shared__ OrderLds o;
    if ((int)threadIdx.x < a.E) o.chose[0][threadIdx.x] = 0;
    __syncthreads();
    const float NONE = -__builtin_inff();
    float next[L], bias[L];
#pragma unroll
    for (int i = 0; i < L; ++i) bias[i] = a.bias && lane * L + i < a.E ? a.bias[lane * L + i] : 0.f;
    if (wave < TOKENS && (int64_t)blockIdx.x * TOKENS + wave < a.tokens) load_logits(a, (int64_t)blockIdx.x * TOKENS + wave, lane, next);
    for (int local = wave; local < TOKENS; local += WAVES) {
        const int64_t t = (int64_t)blockIdx.x * TOKENS + local;
        if (t >= a.tokens) break;
        float x[L];
#pragma unroll
        for (int i = 0; i < L; ++i) x[i] = next[i];
        if (local + WAVES < TOKENS && t + WAVES < a.tokens) load_logits(a, t + WAVES, lane, next);     // under this token's rounds
        float top = 0.f, sum = 1.f;
        if (!a.sigmoid) softmax_of<L>(x, top, sum);
        auto score = [&](float v) { return a.sigmoid ? sigmoid_of(v) : expf(v - top) / sum; };
        const bool by_logit = !a.sigmoid && !a.bias && !a.top2;
        float key[L], s_of[L];                          // s_of: the score, or the logit that it is made of
#pragma unroll
        for (int i = 0; i < L; ++i) {
            float v = x[i];
            s_of[i] = v;
            if (!by_logit) {
                v = s_of[i] = score(v);
                if (a.bias) v += bias[i];
            }
            key[i] = x[i] > NONE && v > NONE ? v : NONE;
        }
        if (a.groups > 1) keep_groups<L>(a, lane, keys[wave], key);
#pragma unroll
        for (int i = 0; i < L; ++i) keys[wave][lane * L + i] = s_of[i];
        wave_sync();
        int chosen = -1;                                // of slot `lane`
        if (by_logit && a.type != HGEMM_F32) {
            unsigned word[L], own = 0;
#pragma unroll
            for (int i = 0; i < L; ++i) word[i] = key[i] > NONE ? word_of(key[i], a.type == HGEMM_F16, lane * L + i) : 0u;
            for (int j = 0; j < a.k; ++j) {
                unsigned best = word[0];
#pragma unroll
                for (int i = 1; i < L; ++i) best = max(best, word[i]);
                const unsigned most = wave_max(best);
                own = lane == j ? most : own;
#pragma unroll
                for (int i = 0; i < L; ++i) word[i] = word[i] == most ? 0u : word[i];
            }
            if (own) chosen = 0xffff - (own & 0xffffu);
        } else {
            Keys<L> left;
#pragma unroll
            for (int i = 0; i < L; ++i) left.key[i] = key[i] > NONE ? sortable(key[i]) : 0u;
            left.look();
            for (int j = 0; j < a.k; ++j) {
                const int e = left.take(lane);
                if (e < 0) break;
                chosen = lane == j ? e : chosen;
            }
        }
        float s = chosen >= 0 ? keys[wave][chosen] : 0.f;
        if (by_logit && chosen >= 0) s = score(s);
        wave_sync();
        float w = a.factor * s;
        if (a.renormalise) w /= wave_sum(s) + 1e-20f;
        if (lane < a.k) {
            a.weights[t * a.k + lane] = w;
            if constexpr (FEW) {
                __hip_atomic_store(&a.experts[t * a.k + lane], chosen, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);     // for the last workgroup
            } else {
                a.experts[t * a.k + lane] = chosen;
                if (chosen >= 0) atomicOr(&o.chose[0][chosen], 1ull << local);
            }
        }
    }
    if (!a.offsets) return;
    if constexpr (FEW) {
        if (!last_to_arrive(a.arrived, gridDim.x, &o.end, threadIdx.x == 0)) return;
        __syncthreads();
        take_choices<true>(a, o, 0);
        place(a, o, 0);
    } else {
        __syncthreads();
        const int words = (a.E + 3) & ~3;
        if ((int)threadIdx.x < words) a.counts[(int64_t)blockIdx.x * words + threadIdx.x] = (uint8_t)((int)threadIdx.x < a.E ? __popcll(o.chose[0][threadIdx.x]) : 0);
    }
}

// The second launch of more than 128 tokens.
__global__ __launch_bounds__(1024) void place_kernel(RouteArgs a)
{
    __shared__ OrderLds o;
    take_choices<false>(a, o, blockIdx.x);
    place(a, o, blockIdx.x);
}

// Four waves, a token each.
template <int L> __global__ __launch_bounds__(256) void route_backward_kernel(RouteArgs a)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t t = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 4 + wave;
    __shared__ float scores[4][64 * L], grads[4][64 * L];
    if (t >= a.tokens) return;
    float x[L], p[L];
    load_logits(a, t, lane, x);
    int e = lane < a.k ? a.experts[t * a.k + lane] : -1;
    if ((unsigned)e >= (unsigned)a.E) e = -1;
    const float dw = e >= 0 ? a.dweights[t * a.k + lane] : 0.f;
    float top = 0.f, sum = 1.f;
    if (!a.sigmoid) softmax_of<L>(x, top, sum);
    auto score = [&](float v) { return a.sigmoid ? sigmoid_of(v) : expf(v - top) / sum; };
#pragma unroll
    for (int i = 0; i < L; ++i) {
        scores[wave][lane * L + i] = p[i] = score(x[i]);
        grads[wave][lane * L + i] = 0.f;
    }
    wave_sync();
    const float s = e >= 0 ? scores[wave][e] : 0.f;
    float ds = a.factor * dw;
    if (a.renormalise) {
        const float total = wave_sum(s) + 1e-20f;
        ds = a.factor * (dw / total - wave_sum(dw * s) / (total * total));
    }
    if (e < 0) ds = 0.f;
    const float mean = wave_sum(ds * s);
    if (e >= 0) grads[wave][e] = ds;
    wave_sync();
    float dx[L];
#pragma unroll
    for (int i = 0; i < L; ++i) {
        const float d = grads[wave][lane * L + i];
        dx[i] = a.sigmoid ? d * p[i] * (1.f - p[i]) : p[i] * (d - mean);
    }
    auto store = [&](auto* base) {
        typedef std::remove_pointer_t<decltype(base)> T;
        T* const p = base + t * a.ld + lane * L;
        if constexpr (sizeof(T) * L >= 4 && sizeof(T) * L <= 16) {
            if (a.wide) {
                struct alignas(sizeof(T) * L) Word { T v[L]; } w;
#pragma unroll
                for (int i = 0; i < L; ++i) w.v[i] = (T)dx[i];
                if (lane * L < a.E) *(Word*)p = w;
                return;
            }
        }
#pragma unroll
        for (int i = 0; i < L; ++i)
            if (lane * L + i < a.E) p[i] = (T)dx[i];
    };
    if (a.type == HGEMM_F16) store((_Float16*)a.dlogits);
    else if (a.type == HGEMM_BF16) store((__bf16*)a.dlogits);
    else store((float*)a.dlogits);
}

typedef void (*Kernel)(RouteArgs);
// Lanes hold 1, 2, 4, 8 or 16 experts each; a workgroup has a thread for every expert (place).
template <bool FEW> Kernel route_of(int E)
{
    return E <= 64 ? route_kernel<1, FEW> : E <= 128 ? route_kernel<2, FEW> : E <= 256 ? route_kernel<4, FEW> : E <= 512 ? route_kernel<8, FEW> : route_kernel<16, FEW>;
}
int per_lane(int E) { return E <= 64 ? 1 : E <= 128 ? 2 : E <= 256 ? 4 : E <= 512 ? 8 : 16; }
Kernel back_of(int E)
{
    return E <= 64 ? route_backward_kernel<1> : E <= 128 ? route_backward_kernel<2> : E <= 256 ? route_backward_kernel<4> : E <= 512 ? route_backward_kernel<8> : route_backward_kernel<16>;
}

void set_wide(RouteArgs& a, const void* logits)
{
    const int L = per_lane(a.E), size = type_size((hgemm_type_t)a.type);
    a.wide = a.E % L == 0 && a.ld % L == 0 && aligned(logits, L * size);
}

hgemm_status_t check(const hgemm_route_t* d)
{
    if (!d || d->tokens < 0 || d->experts < 1 || d->experts > kMostExperts || d->k < 1 || d->k > kMostChoices || d->k > d->experts) return HGEMM_ERR_INVALID_ARG;
    if ((unsigned)d->logits > HGEMM_F32 || d->groups < 1 || d->experts % d->groups || d->keep < 1 || d->keep > d->groups || d->align < 1 || d->align > 1024) return HGEMM_ERR_INVALID_ARG;
    if (d->ld && d->ld < d->experts) return HGEMM_ERR_INVALID_ARG;
    if (d->tokens >= (int64_t)1 << 26 || d->tokens * d->k > (int64_t)1 << 30) return HGEMM_ERR_UNSUPPORTED;
    return HGEMM_OK;
}

}  // namespace

struct hgemm_route_plan_s {
    RouteArgs args;
    void* workspace = nullptr;
    bool clearing = false;      // the counter of few tokens may still be on its way to zero
};

extern "C" {

int64_t hgemm_route_capacity(const hgemm_route_t* d)
{
    if (check(d) != HGEMM_OK) return -1;
    return round_up(d->tokens * d->k + (int64_t)d->experts * (d->align - 1), d->align);
}

hgemm_status_t hgemm_route_plan(hgemm_route_plan_t* out, const hgemm_route_t* d)
{
    if (!out) return HGEMM_ERR_INVALID_ARG;
    const hgemm_status_t st = check(d);
    if (st != HGEMM_OK) return st;
    if (!current_device_is_gfx950()) return HGEMM_ERR_ARCH;
    hgemm_route_plan_s* p = new (std::nothrow) hgemm_route_plan_s;
    if (!p) return HGEMM_ERR_ALLOC;
    RouteArgs a{};
    a.ld = d->ld ? d->ld : d->experts;
    a.capacity = hgemm_route_capacity(d);
    a.tokens = (int)d->tokens; a.E = d->experts; a.k = d->k;
    a.type = d->logits; a.sigmoid = d->sigmoid != 0; a.groups = d->groups; a.keep = d->keep; a.top2 = d->top2 != 0;
    a.renormalise = d->renormalise != 0; a.align = d->align; a.factor = d->factor;
    const bool few = d->tokens <= kPlaceTokens;
    const int64_t each = few ? kFewTokens : kRouteTokens;
    a.blocks = (int)((d->tokens + each - 1) / each);
    const size_t bytes = few ? 256 : (size_t)a.blocks * ((a.E + 3) & ~3);
    void* workspace = nullptr;
    if (hipMalloc(&workspace, bytes) != hipSuccess || (few && hipMemset(workspace, 0, bytes) != hipSuccess)) {
        (void)hipGetLastError();
        if (workspace) (void)hipFree(workspace);
        delete p;
        return HGEMM_ERR_ALLOC;
    }
    (few ? (void*&)a.arrived : (void*&)a.counts) = workspace;
    p->workspace = workspace;
    p->clearing = few;
    p->args = a;
    *out = p;
    return HGEMM_OK;
}

hgemm_status_t hgemm_route_run(hgemm_route_plan_t plan, const void* logits, const float* bias, float* weights, int32_t* experts, int32_t* offsets, int32_t* rows, int32_t* tokens_of,
                               void* hip_stream)
{
    if (!plan) return HGEMM_ERR_INVALID_ARG;
    RouteArgs a = plan->args;
    const bool order = offsets || rows || tokens_of;
    if (a.tokens && (!logits || !weights || !experts)) return HGEMM_ERR_INVALID_ARG;
    if (order && (!offsets || (a.tokens && !rows) || (a.capacity && !tokens_of))) return HGEMM_ERR_INVALID_ARG;
    if (!aligned(logits, type_size((hgemm_type_t)a.type)) || !aligned(bias, 4) || !aligned(weights, 4) || !aligned(experts, 4) || !aligned(offsets, 4) || !aligned(rows, 4) || !aligned(tokens_of, 4))
        return HGEMM_ERR_INVALID_ARG;
    a.logits = logits; a.bias = bias; a.weights = weights; a.experts = experts;
    a.offsets = offsets; a.rows = rows; a.tokens_of = tokens_of;
    const hipStream_t s = (hipStream_t)hip_stream;
    if (!wait_for_clearing(plan->clearing, s)) return HGEMM_ERR_LAUNCH;
    set_wide(a, logits);
    const unsigned blocks = a.blocks ? a.blocks : 1;    // without tokens: padding only
    if (a.tokens <= kPlaceTokens) {
        if (a.tokens || order) route_of<true>(a.E)<<<blocks, 1024, 0, s>>>(a);
    } else {
        route_of<false>(a.E)<<<blocks, 1024, 0, s>>>(a);
        if (order) place_kernel<<<(unsigned)((a.tokens + kPlaceTokens - 1) / kPlaceTokens), 1024, 0, s>>>(a);
    }
    return hipGetLastError() == hipSuccess ? HGEMM_OK : HGEMM_ERR_LAUNCH;
}

hgemm_status_t hgemm_route_backward(hgemm_route_plan_t plan, const void* logits, const int32_t* experts, const float* dweights, void* dlogits, void* hip_stream)
{
    if (!plan) return HGEMM_ERR_INVALID_ARG;
    RouteArgs a = plan->args;
    if (!a.tokens) return HGEMM_OK;
    if (!logits || !experts || !dweights || !dlogits) return HGEMM_ERR_INVALID_ARG;
    const size_t size = type_size((hgemm_type_t)a.type);
    if (!aligned(logits, size) || !aligned(experts, 4) || !aligned(dweights, 4) || !aligned(dlogits, size)) return HGEMM_ERR_INVALID_ARG;
    a.logits = logits; a.experts = (int*)experts; a.dweights = dweights; a.dlogits = dlogits;
    set_wide(a, logits);
    a.wide = a.wide && aligned(dlogits, per_lane(a.E) * size);
    // a launch has fewer than 2^32 threads along x: from 2^26 - 3 tokens on, two rows of workgroups
    const unsigned workgroups = ((unsigned)a.tokens + 3) / 4, most = 0xffffffffu / 256;
    const dim3 grid = workgroups <= most ? dim3(workgroups) : dim3((workgroups + 1) / 2, 2);
    back_of(a.E)<<<grid, 256, 0, (hipStream_t)hip_stream>>>(a);
    return hipGetLastError() == hipSuccess ? HGEMM_OK : HGEMM_ERR_LAUNCH;
}

hgemm_status_t hgemm_route_destroy(hgemm_route_plan_t plan)
{
    if (!plan) return HGEMM_OK;
    if (plan->workspace && hipFree(plan->workspace) != hipSuccess) (void)hipGetLastError();
    delete plan;
    return HGEMM_OK;
}

}  // extern "C"
