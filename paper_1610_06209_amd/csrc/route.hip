// A router's logits to experts and weights, with the gradient, and the chosen experts to places in their order.
#include <math.h>

#include "mx4.hpp"
#include "number_io.hpp"
#include "route.hpp"
#include "spinner_kernels.hpp"

namespace spinner {
namespace {

constexpr int kThreads = 256;
// Rows up to which a router takes 64 lanes a row, and from which four (up to kFewChoices choices, and more).  us, 8 of 64 / 256 experts, bf16: 64 and 16 lanes, 2048 rows 3.9 and 4.0 / 4.3 and 4.6,
// with a bias 5.6 and 6.6 / 6.4 and 7.9, 4096 rows 4.8 and 4.1 / 5.3 and 4.7, biased 7.0 and 6.7 / 7.8 and 7.8.  16 and four lanes, 4 of 32 experts, 8192 rows 3.9 and 3.7, biased 6.8 and 7.4, 16384 4.6
// and 3.7, 8.5 and 8.0, 131072 18 and 7.3, 41 and 16; 8 of 64, 16384 rows 5.1 and 4.7, biased 8.6 and 11.2, 32768 7.7 and 5.3, 14.8 and 12.5.
constexpr int kFewRouteRows = 2048, kManyRouteRows = 16384, kFewChoices = 4;
constexpr long long kRouteBlocks = 1 << 20;          // most workgroups: a grid holds fewer than 2^32 threads, and goes down the rows

// v of the lane that takes turns with this one in a join over 2 MASK lanes, when lanes of MASK have joined before: mirrored rows for 4 and 8, which the
// adders read in place
template <int MASK>
__device__ __forceinline__ int across(int v)
{
    if constexpr (MASK == 4) return __builtin_amdgcn_update_dpp(0, v, 0x141, 0xF, 0xF, true);        // row_half_mirror
    else if constexpr (MASK == 8) return __builtin_amdgcn_update_dpp(0, v, 0x140, 0xF, 0xF, true);   // row_mirror
    else return lane_xor_i<MASK>(v);
}
template <int MASK> __device__ __forceinline__ unsigned across(unsigned v) { return (unsigned)across<MASK>((int)v); }
template <int MASK> __device__ __forceinline__ float across(float v) { return __int_as_float(across<MASK>(__float_as_int(v))); }
template <int MASK> __device__ __forceinline__ double across(double v) { return __hiloint2double(across<MASK>(__double2hiint(v)), across<MASK>(__double2loint(v))); }

// A pair of values of which one is this lane's and the other that of lane ^ MASK, the same pair in both (MASK 16, 32)
template <int MASK>
__device__ __forceinline__ void pair_across(int v, int& a, int& b)
{
    const auto t = [&] {
        if constexpr (MASK == 16) return __builtin_amdgcn_permlane16_swap((unsigned)v, (unsigned)v, false, false);
        else return __builtin_amdgcn_permlane32_swap((unsigned)v, (unsigned)v, false, false);
    }();
    a = (int)t[0];
    b = (int)t[1];
}
template <int MASK> __device__ __forceinline__ void pair_across(unsigned v, unsigned& a, unsigned& b)
{
    int x, y;
    pair_across<MASK>((int)v, x, y);
    a = (unsigned)x;
    b = (unsigned)y;
}
template <int MASK> __device__ __forceinline__ void pair_across(float v, float& a, float& b)
{
    int x, y;
    pair_across<MASK>(__float_as_int(v), x, y);
    a = __int_as_float(x);
    b = __int_as_float(y);
}
template <int MASK> __device__ __forceinline__ void pair_across(double v, double& a, double& b)
{
    int x, y, z, w;
    pair_across<MASK>(__double2hiint(v), x, y);
    pair_across<MASK>(__double2loint(v), z, w);
    a = __hiloint2double(x, z);
    b = __hiloint2double(y, w);
}

// ------------------------------------------------------------------ lanes of a row
// `op` over a row's LANES lanes (4, 16: joined in registers by the instruction set's own quads and rows), in all of them
template <int LANES, typename V, typename F>
__device__ __forceinline__ V join_lanes(V v, F op)
{
    v = op(v, across<1>(v));
    v = op(v, across<2>(v));
    if constexpr (LANES > 4) {
        v = op(v, across<4>(v));
        v = op(v, across<8>(v));
    }
    if constexpr (LANES == 64) {
        V a, b;
        pair_across<16>(v, a, b);
        v = op(a, b);
        pair_across<32>(v, a, b);
        v = op(a, b);
    }
    return v;
}
struct Sum { template <typename V> __device__ __forceinline__ V operator()(V a, V b) const { return a + b; } };
struct Larger { template <typename V> __device__ __forceinline__ V operator()(V a, V b) const { return a > b ? a : b; } };
template <int LANES>
__device__ __forceinline__ bool any_lane(bool v)
{
    const unsigned long long all = __ballot(v);
    if constexpr (LANES == 64) return all != 0;
    return (all >> (threadIdx.x & (64 - LANES)) & ((1ull << LANES) - 1)) != 0;
}

// What the wave's lanes have written to LDS, in order, is there for all of them: the LDS keeps the order of a wave, and so has the compiler to.
__device__ __forceinline__ void wave_meets()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// exp(x) for x <= 0 to 2^-22 of itself: 2^h with the product's remainder put back (x log2(e) alone would be off by |x| 2^-24); 0 from -87 down
__device__ __forceinline__ float exp_below(float x)
{
    x = fmaxf(x, -200.0f);
    const float h = x * 1.44269502f, l = __builtin_fmaf(x, 1.44269502f, -h) + x * 1.92596303e-8f;
    return __builtin_amdgcn_exp2f(h) * __builtin_fmaf(l, 0.693147182f, 1.0f);
}
__device__ __forceinline__ float sigmoid(float l)
{
    const float e = exp_below(-__builtin_fabsf(l));
    return (l > 0.0f ? 1.0f : e) * __builtin_amdgcn_rcpf(1.0f + e);
}

// Which experts a lane has: of LANES / 2^log_groups lanes each group, `mine` neighbours from `first` on, at most R.
struct Share {
    int group, first, mine;
    __device__ __forceinline__ Share(int lane, int lanes, int log_groups, int groups, int size)
    {
        const int each = lanes >> log_groups, in_group = lane & (each - 1), part = (size + each - 1) / each;
        group = lane / each;
        first = group * size + in_group * part;
        const int left = size - in_group * part;
        mine = group < groups ? (left < part ? left : part) : 0;
    }
};

// a lane's logits, those that it has none of -inf
template <typename T, int R>
__device__ __forceinline__ void load_logits(float (&v)[R], const T* row, int first, int mine, int count)
{
    constexpr int N = 16 / (int)sizeof(T);
    if (R % N == 0 && first + R <= count) {
#pragma unroll
        for (int i = 0; i < R / N; ++i) {
            const auto q = *reinterpret_cast<const typename LooseQuad<sizeof(T)>::type*>(row + first + i * N);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                float f;
                if constexpr (sizeof(T) == 4) f = __uint_as_float(q[k]);
                else f = (float)__builtin_bit_cast(typename Pair16<T>::Pair, (unsigned)q[k >> 1])[k & 1];
                v[i * N + k] = i * N + k < mine ? f : -INFINITY;
            }
        }
    } else {
#pragma unroll
        for (int r = 0; r < R; ++r) v[r] = r < mine ? (float)row[first + r] : -INFINITY;
    }
}

// a number's bits in the order of the numbers, as unsigned whole numbers (-0 is 0)
__device__ __forceinline__ unsigned ordered(float v)
{
    const int b = __float_as_int(v + 0.0f);
    return (unsigned)b ^ ((unsigned)(b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float number_of(unsigned u)
{
    return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}

// weight of a chosen logit without the factor that all share: softmax exp(l - top), sigmoid 1 / (1 + exp(-l)) over exp(top), top the largest
// min(l, 0), so that the largest is at least a half and their sum is no 0
template <int SCORE>
__device__ __forceinline__ float share_of(float logit, float top)
{
    if constexpr (SCORE == kSoftmax) return exp_below(logit - top);
    return exp_below(fminf(logit, 0.0f) - top) * __builtin_amdgcn_rcpf(1.0f + exp_below(-__builtin_fabsf(logit)));
}

// The two largest of a group's keys, of its `each` lanes
template <typename V>
struct Two {
    V a, b;
    __device__ __forceinline__ void take(V k)
    {
        if constexpr (sizeof(V) == 4) {
            b = __builtin_amdgcn_fmed3f(a, b, k);
            a = fmaxf(a, k);
        } else {
            const V low = a < k ? a : k;
            b = b > low ? b : low;
            a = a > k ? a : k;
        }
    }
    __device__ __forceinline__ void merge(V a2, V b2)
    {
        const V low = a < a2 ? a : a2, high = b > b2 ? b : b2;
        b = low > high ? low : high;
        a = a > a2 ? a : a2;
    }
    template <int MASK>
    __device__ __forceinline__ void halves()
    {
        V a2, b2, a1, b1;
        pair_across<MASK>(a, a1, a2);
        pair_across<MASK>(b, b1, b2);
        a = a1;
        b = b1;
        merge(a2, b2);
    }
    __device__ __forceinline__ void lanes(int each)
    {
        if (each > 1) merge(across<1>(a), across<1>(b));
        if (each > 2) merge(across<2>(a), across<2>(b));
        if (each > 4) merge(across<4>(a), across<4>(b));
        if (each > 8) merge(across<8>(a), across<8>(b));
        if (each > 16) halves<16>();
        if (each > 32) halves<32>();
    }
};

constexpr double kNever = -(double)INFINITY;
constexpr float kLargest = 3.40282347e38f;
// most choices of a row of so many lanes, and candidates: its choices and what may lie level with the last of them
constexpr int most_chosen(int lanes) { return lanes == 4 ? 8 : kMostChosen; }
constexpr int most_candidates(int lanes) { return lanes == 4 ? 16 : 48; }

// A row's scores in fp64, from its logits in LDS.
template <int LANES, int SCORE>
struct Scores64 {
    const RouteParams& p;
    double top = 0.0, sum = 1.0;
    // `mine` logits of the lane at l
    __device__ __forceinline__ Scores64(const RouteParams& p_, const float* l, int mine) : p(p_)
    {
        if constexpr (SCORE == kSoftmax) {
            float high = -INFINITY;
#pragma unroll 1
            for (int r = 0; r < mine; ++r) high = fmaxf(high, l[r]);
            top = (double)join_lanes<LANES>(high, Larger{});
            sum = 0.0;
#pragma unroll 1
            for (int r = 0; r < mine; ++r) sum += l[r] > -INFINITY ? exp((double)l[r] - top) : 0.0;
            sum = join_lanes<LANES>(sum, Sum{});
        }
    }
    // score and bias of expert e
    __device__ __forceinline__ double key(float l, int e) const
    {
        const double s = SCORE == kSoftmax ? exp((double)l - top) / sum : 1.0 / (1.0 + exp(-(double)l));
        return l > -INFINITY ? s + (p.bias ? (double)p.bias[e] : 0.0) : kNever;
    }
};

// whether this lane's group stays, in fp64
template <int LANES, int SCORE>
__device__ __forceinline__ bool stays64(const RouteParams& p, const float* l, const Share& at, int lane, double* group_keys)
{
    const Scores64<LANES, SCORE> scores(p, l, at.mine);
    const int each = LANES >> p.log_groups;
    Two<double> two = {kNever, kNever};
#pragma unroll 1
    for (int r = 0; r < at.mine; ++r) two.take(scores.key(l[r], at.first + r));
    two.lanes(each);
    const double own = p.group_top > 1 && two.b > kNever ? two.a + two.b : two.a;
    if ((lane & (each - 1)) == 0) group_keys[at.group] = own;
    wave_meets();
    int larger = 0;
    for (int g = 0; g < p.groups; ++g) {
        const double other = group_keys[g];
        larger += ((other > own) | ((other == own) & (g < at.group))) ? 1 : 0;
    }
    wave_meets();
    return larger < p.top_groups;
}

// The places of all choices in fp64, each the largest key behind the one before, for rows with more keys level with the last choice than there is room for.
template <int LANES, int R, int SCORE>
__device__ __forceinline__ void choose64(const RouteParams& p, const float* l, const Share& at, bool stays, int lane, int* chosen)
{
    const Scores64<LANES, SCORE> scores(p, l, at.mine);
    double last = (double)INFINITY;
    int last_at = -1;
    for (int j = 0; j < p.top; ++j) {
        double v = kNever;
        int which = 0x7fffffff;
#pragma unroll 1
        for (int r = 0; r < at.mine; ++r) {
            const double k = p.bias ? scores.key(l[r], at.first + r) : (double)l[r];
            const int own = lane * R + r;
            const bool other = stays & ((k < last) | ((k == last) & (own > last_at))) & (k > v);
            v = other ? k : v;
            which = other ? own : which;
        }
        last = join_lanes<LANES>(v, Larger{});
        last_at = join_lanes<LANES>(v == last ? which : 0x7fffffff, [](int a, int b) { return a < b ? a : b; });
        if (lane == 0) chosen[j] = last > kNever ? last_at : -1;
    }
    wave_meets();
}

// LANES lanes a row, up to R neighbouring experts each, in registers from the logits to the choice.
// A candidate is the largest of whole numbers of 32 bits below the last one: the first 22 (21) of the key's bits in the order of the numbers, and its place
// in the row's lanes, which puts equal ones in the order of their index.  EXACT (16-bit logits, no bias: the key is the logit, of which 19 bits are all there is): the candidates
// are the choices (16384 x 256, 8 choices: 6.8 us).  Otherwise candidates are taken until one lies clearly below the last choice, and put in order by their keys in fp32; where those
// lie too near each other (and are not equal by having the same logit and bias) by their keys in fp64, and so are groups at the border.
// The vector ALU bounds it where rows are many: 16383 x 256 bf16, biased sigmoid, groups, 18 to 20 us (0.45 TB/s of logits); 65536 x 64 bf16, no bias, 2 choices, 5.0 us in a row of launches, 6.4 to 7.0 between
// others (1.2 to 1.7); 8191 x 999 fp32, biased softmax, 11 choices, 30 us (1.1).  A round of the choice is two instructions an expert.
template <typename T, int LANES, int R, int SCORE, bool EXACT>
__global__ void __launch_bounds__(kThreads, R <= 16 ? 4 : 2) route_kernel(RouteParams p)
{
    constexpr int ROWS = kThreads / LANES, MOST = most_chosen(LANES), CANDIDATES = most_candidates(LANES);
    constexpr int HELD = (MOST + LANES - 1) / LANES, HELD_ALL = (CANDIDATES + LANES - 1) / LANES;
    constexpr unsigned kLow = LANES * R > 1024 ? 2047 : 1023, kLeast = 0x00800000u;      // kLeast: of the numbers above -inf
    __shared__ float logits[ROWS][LANES * R];
    __shared__ double group_keys[ROWS][LANES > CANDIDATES ? LANES : CANDIDATES + 1];     // (no more groups than lanes)
    __shared__ unsigned order[ROWS][CANDIDATES];
    __shared__ float keys_of[EXACT ? 1 : ROWS][EXACT ? 1 : CANDIDATES + 1];
    __shared__ int chosen[ROWS][MOST];
    const int lane = threadIdx.x & (LANES - 1), slot = threadIdx.x / LANES, size = p.count / p.groups;
    const Share at(lane, LANES, p.log_groups, p.groups, size);
    const int each = LANES >> p.log_groups, part_of = (size + each - 1) / each;
    // the expert at a place
    const auto expert_at = [&](int place) {
        const int l = place / R;
        return l / each * size + (l & (each - 1)) * part_of + (place & (R - 1));
    };
    float bias[R], largest_bias = 0.0f;
    bool bad_bias = false;
#pragma unroll
    for (int r = 0; r < R; ++r) bias[r] = 0.0f;
    if (!EXACT && p.bias) {
        load_logits<float, R>(bias, p.bias, at.first, at.mine, p.count);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            bias[r] = r < at.mine ? bias[r] : 0.0f;
            bad_bias |= bias[r] != bias[r];
            // (infinities are far from all others)
            largest_bias = fmaxf(largest_bias, __builtin_fabsf(bias[r]) < INFINITY ? __builtin_fabsf(bias[r]) : 0.0f);
        }
        // (the same in all rows)
        largest_bias = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(join_lanes<LANES>(largest_bias, Larger{}))));
    }
    // Keys of fp32 that lie nearer may be the other way round.  A sigmoid is off by 4e-7 of itself; a softmax by what its sum is off too, (R + 6) 2^-24, which two
    // scores share; a score is neither above 1 nor above its key and bias together.  A key is off by half a place of itself more, 6e-8, and so are two.  (A bias
    // of -1e9 for one expert widens nothing for the others.  Infinite keys are far from finite ones.)
    // Scores below e^-64 are off by more, where logits that far from the largest are: by less than 1e-32 in all.
    const auto size_of = [](float key) { return fminf(__builtin_fabsf(key), kLargest); };
    const auto reach = [&](float key) {
        const float size = size_of(key);
        return __builtin_fmaf(SCORE == kSigmoid ? 1.05e-6f : 4.85e-6f, fminf(size + largest_bias, 1.0f), __builtin_fmaf(1.5e-7f, size, 1e-32f));
    };
    for (long long r0 = (long long)blockIdx.x * ROWS; r0 < p.rows; r0 += (long long)gridDim.x * ROWS) {
        const long long own = r0 + slot, row = own < p.rows ? own : p.rows - 1;
        float l[R];
        load_logits<T, R>(l, static_cast<const T*>(p.logits) + row * p.stride, at.first, at.mine, p.count);
        const bool routed = !p.mask || p.mask[row] != 0;
        // what is no number, no expert, or far from the ordinary is looked at where there is any
        bool odd = bad_bias;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            odd |= !(__builtin_fabsf(l[r]) <= 32.0f);
            logits[slot][lane * R + r] = l[r];
        }
        const bool careful = __ballot(odd) != 0;
        bool bad = false;                  // a NaN, or an infinity in a softmax
        if (careful) {
            bad = bad_bias;
#pragma unroll
            for (int r = 0; r < R; ++r) bad |= (l[r] != l[r]) | (SCORE == kSoftmax && l[r] == INFINITY);
            bad = any_lane<LANES>(bad);
        }
        float top = -INFINITY, sum = 0.0f;
        const bool scored = (!EXACT && p.bias) || p.group_top > 1;
        float key[R];
        if (SCORE == kSoftmax && (scored || !p.renormalise)) {
#pragma unroll
            for (int r = 0; r < R; ++r) top = fmaxf(top, l[r]);
            top = join_lanes<LANES>(top, Larger{});
            if (p.renormalise) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    key[r] = __builtin_amdgcn_exp2f(fmaxf(l[r] - top, -200.0f) * 1.44269502f);
                    sum += key[r];
                }
            } else {                       // the weights are these over this sum
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    key[r] = exp_below(l[r] - top);
                    sum += key[r];
                }
            }
            sum = join_lanes<LANES>(sum, Sum{});
        }
        // Keys, -inf for what cannot be chosen.  Scores of all experts in few instructions, off by 64 (x up to -88: 88) times 6e-8 of themselves at most and
        // 4e-7; the candidates' are made again.
        const float part = 1.0f / sum;
        if (scored) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float s = SCORE == kSoftmax ? key[r] * part : __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(l[r] * -1.44269502f));
                key[r] = s + bias[r];
            }
            if (careful)
#pragma unroll
                for (int r = 0; r < R; ++r) key[r] = l[r] > -INFINITY ? key[r] : -INFINITY;
        } else {
#pragma unroll
            for (int r = 0; r < R; ++r) key[r] = l[r];
        }
        bool near = false, stays = true;
        if (p.groups > 1) {
            Two<float> two = {-INFINITY, -INFINITY};
#pragma unroll
            for (int r = 0; r < R; ++r) two.take(key[r]);
            two.lanes(each);
            const float mine = p.group_top > 1 && two.b > -INFINITY ? two.a + two.b : two.a;
            float* keys = reinterpret_cast<float*>(group_keys[slot]);
            if ((lane & (each - 1)) == 0) keys[at.group] = mine;
            wave_meets();
            int larger = 0;
#pragma unroll 4
            for (int g = 0; g < p.groups; ++g) {
                const float other = keys[g];
                larger += ((other > mine) | ((other == mine) & (g < at.group))) ? 1 : 0;
            }
            stays = larger < p.top_groups;
            if (scored) {
                // What a group's key is off by at most: its scores (no more than 1 each), and its keys' and their sum's roundings.  The groups that stay are
                // the right ones where the least that one of them may be lies above the most that another one may (sums that leave fp32 may be anything beyond).
                const float first = __builtin_fabsf(two.a), second = p.group_top > 1 && two.b > -INFINITY ? __builtin_fabsf(two.b) : 0.0f;
                const float score = fminf(__builtin_fmaf((float)p.group_top, largest_bias, first + second), 2.0f);
                const float round = __builtin_fmaf(2.5e-7f, fminf(first, kLargest), __builtin_fmaf(2.5e-7f, second, 1e-32f));
                const float off = __builtin_fmaf(SCORE == kSoftmax ? 4.5e-6f + 6e-8f * (R + 6) : careful ? 6e-6f : 2.5e-6f, score, round);
                const float least = join_lanes<LANES>(stays ? off - fminf(mine, kLargest) : -INFINITY, Larger{});
                const float most = join_lanes<LANES>(stays || !(two.a > -INFINITY) ? -INFINITY : fmaxf(mine, -kLargest) + off, Larger{});
                near = (most > -INFINITY) & (most + least >= 0.0f);
            }
            wave_meets();
            if (__builtin_expect(__ballot(near) != 0, 0)) stays = stays64<LANES, SCORE>(p, logits[slot] + lane * R, at, lane, group_keys[slot]);
            near = false;
        }
        unsigned k[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float v = EXACT || !p.bias ? l[r] : key[r];
            k[r] = (ordered(v) & ~kLow) | (kLow - (unsigned)(lane * R + r));
        }
        // the largest number below the last one, which leaves it the largest of the differences to that, modulo 2^32
        unsigned last = 0xffffffffu;
        float border = 0.0f;               // what lies clearly below the last choice
        bool open = !EXACT;                // whether there may be more candidates for the last choice
        int count = 0;
        for (;;) {
            unsigned best = 0;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const unsigned t = k[r] - last;
                best = t > best ? t : best;
            }
            const unsigned next = join_lanes<LANES>(stays ? best : 0u, Larger{}) + last;
            last = ((next < last) & (next >= kLeast)) ? next : 0;
            if (lane == 0) order[slot][count] = last;
            ++count;
            if constexpr (EXACT) {
                if (count == p.top) break;
            } else if (count >= p.top) {
                // (off by 2^-12 of the number, or 2^-138, and by what the scores in few instructions are)
                const float v = number_of(last & ~kLow);
                if (count == p.top) border = v - __builtin_fmaf(3.0f, reach(v), 5e-4f * size_of(v));
                else open = open & (last != 0) & (v > border);
                if (count > p.top && __ballot(open) == 0) break;
                if (count == CANDIDATES) break;
            }
        }
        wave_meets();
        if constexpr (EXACT) {
#pragma unroll
            for (int h = 0; h < HELD; ++h) {
                const int j = h * LANES + lane;
                if (j < p.top) chosen[slot][j] = order[slot][j] ? (int)(kLow - (order[slot][j] & kLow)) : -1;
            }
        } else {
            float v[HELD_ALL];
            int own_place[HELD_ALL], rank[HELD_ALL];
#pragma unroll
            for (int h = 0; h < HELD_ALL; ++h) {
                const int j = h * LANES + lane;
                v[h] = -INFINITY;
                own_place[h] = 0x7fffffff;
                rank[h] = 0;
                if (h * LANES >= count) continue;
                if (j < count && order[slot][j]) {
                    own_place[h] = (int)(kLow - (order[slot][j] & kLow));
                    const float x = logits[slot][own_place[h]];
                    v[h] = !p.bias ? x : (SCORE == kSoftmax ? exp_below(x - top) * part : sigmoid(x)) + p.bias[expert_at(own_place[h])];
                }
                if (j < count) keys_of[slot][j] = v[h];
            }
            wave_meets();
#pragma unroll 4
            for (int i = 0; i < count; ++i) {
                const float other = keys_of[slot][i];
                const int other_place = (int)(kLow - (order[slot][i] & kLow));
#pragma unroll
                for (int h = 0; h < HELD_ALL; ++h)
                    if (h * LANES < count) rank[h] += ((other > v[h]) | ((other == v[h]) & (other_place < own_place[h]))) ? 1 : 0;
            }
            wave_meets();
            if (p.bias) {
                // keys next to each other in this order that may be the other way round, unless they are of equal logits and biases
                int* places = reinterpret_cast<int*>(group_keys[slot]);
#pragma unroll
                for (int h = 0; h < HELD_ALL; ++h)
                    if (v[h] > -INFINITY) { keys_of[slot][rank[h] + 1] = v[h]; places[rank[h] + 1] = own_place[h]; }
                wave_meets();
#pragma unroll
                for (int h = 0; h < HELD_ALL; ++h)
                    if (v[h] > -INFINITY && rank[h] > 0) {
                        const float other = keys_of[slot][rank[h]];
                        if (other - v[h] <= reach(other)) {
                            const int before = places[rank[h]];
                            near |= (logits[slot][before] != logits[slot][own_place[h]]) | (p.bias[expert_at(before)] != p.bias[expert_at(own_place[h])]);
                        }
                    }
                wave_meets();
            }
            if (__builtin_expect(__ballot(near) != 0, 0)) {
                const Scores64<LANES, SCORE> scores(p, logits[slot] + lane * R, at.mine);
                double* keys = group_keys[slot];
#pragma unroll 1
                for (int j = lane; j < count; j += LANES) {
                    const int own = (int)(kLow - (order[slot][j] & kLow));
                    keys[j] = order[slot][j] ? scores.key(logits[slot][own], expert_at(own)) : kNever;
                }
                wave_meets();
#pragma unroll
                for (int h = 0; h < HELD_ALL; ++h) {
                    if (h * LANES >= count) break;
                    const double mine = keys[h * LANES + lane < count ? h * LANES + lane : 0];
                    rank[h] = 0;
                    for (int i = 0; i < count; ++i) {
                        const double other = keys[i];
                        rank[h] += ((other > mine) | ((other == mine) & ((int)(kLow - (order[slot][i] & kLow)) < own_place[h]))) ? 1 : 0;
                    }
                }
            }
#pragma unroll
            for (int h = 0; h < HELD; ++h)
                if (h * LANES + lane < p.top) chosen[slot][h * LANES + lane] = -1;
            wave_meets();
#pragma unroll
            for (int h = 0; h < HELD_ALL; ++h)
                if (v[h] > -INFINITY && rank[h] < p.top) chosen[slot][rank[h]] = own_place[h];
            open = any_lane<LANES>(open);
            if (__builtin_expect(__ballot(open) != 0, 0)) {
                // (a row that is not open gets what it has)
                wave_meets();
                choose64<LANES, R, SCORE>(p, logits[slot] + lane * R, at, stays, lane, chosen[slot]);
            }
        }
        wave_meets();
        // weights: choice j is lane j mod LANES's
        int which[HELD];
        float value[HELD], own_top = -INFINITY;
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            const int j = h * LANES + lane;
            const int place = j < p.top ? chosen[slot][j] : -1;
            which[h] = place < 0 ? -1 : expert_at(place);
            value[h] = place < 0 ? -INFINITY : logits[slot][place];
            own_top = fmaxf(own_top, SCORE == kSigmoid ? fminf(value[h], 0.0f) : value[h]);
        }
        if (p.renormalise) {
            top = join_lanes<LANES>(own_top, Larger{});
            sum = 0.0f;
        } else if (SCORE == kSigmoid) {
            top = 0.0f;
        }
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            value[h] = which[h] >= 0 ? share_of<SCORE>(value[h], top) : 0.0f;
            if (p.renormalise) sum += value[h];
        }
        if (p.renormalise) sum = join_lanes<LANES>(sum, Sum{});
        // (quotients, not products with 1 / sum: of one choice the weight is the scale)
        const bool shared = p.renormalise || SCORE == kSoftmax;
#pragma unroll
        for (int h = 0; h < HELD; ++h) value[h] = (!shared ? value[h] : sum > 0.0f ? value[h] / sum : 0.0f) * p.scale;
        if (own < p.rows) {
#pragma unroll
            for (int h = 0; h < HELD; ++h) {
                const int j = h * LANES + lane;
                if (j < p.top) {
                    p.experts[own * p.top + j] = routed && !bad ? which[h] : -1;
                    p.weights[own * p.top + j] = !routed ? 0.0f : bad ? __builtin_nanf("") : value[h];
                }
            }
        }
        wave_meets();
    }
}

// Gradient of the logits.  With p the scores of a row, w_j = scale p_j of the chosen ones gives
//   softmax      dl_i = p_i (d_i - sum_j d_j p_j)          d_i = scale dw_i of a chosen one, 0 of others
//   sigmoid      dl_i = d_i p_i (1 - p_i)
// and w_j = scale q_j, q_j = p_j / (sum of the chosen ones'), on the chosen ones only
//   softmax      dl_i = q_i (d_i - sum_j d_j q_j)          sigmoid: (1 - p_i) times that
// Few numbers are read but for the whole softmax; what it writes bounds it, and the launch: 65536 x 64 bf16 5.0 us in a row of launches, 6.5 to 7.0 between others (8.4 MB written), 8191 x 999 fp32 10.2 and 10.8
// (33 MB, 3.0 to 3.2 TB/s).
template <typename T, int LANES, int R, int SCORE>
__global__ void __launch_bounds__(kThreads) route_grad_kernel(RouteParams p)
{
    constexpr int ROWS = kThreads / LANES, MOST = most_chosen(LANES), HELD = (MOST + LANES - 1) / LANES;
    __shared__ float spread[ROWS][LANES * R];
    __shared__ float taken[ROWS][MOST];
    __shared__ int named[ROWS][MOST];
    // a lane has pieces of 16 bytes, the lanes' side by side (neighbours alone would meet in few banks of LDS: 8191 x 999 in fp32 18.1 us)
    constexpr int N = 16 / (int)sizeof(T), PIECE = R % N == 0 ? N : 1, PIECES = R / PIECE;
    const int lane = threadIdx.x & (LANES - 1), slot = threadIdx.x / LANES;
    const auto first = [&](int i) { return (i * LANES + lane) * PIECE; };
    const bool all = SCORE == kSoftmax && !p.renormalise;          // every logit has a gradient, not the chosen ones alone
    for (long long r0 = (long long)blockIdx.x * ROWS; r0 < p.rows; r0 += (long long)gridDim.x * ROWS) {
        const long long own = r0 + slot, row = own < p.rows ? own : p.rows - 1;
        const T* from = static_cast<const T*>(p.logits) + row * p.stride;
        float e[R], top = -INFINITY, sum = 0.0f;
        if (all) {
#pragma unroll
            for (int i = 0; i < PIECES; ++i) load_logits<T, PIECE>(reinterpret_cast<float(&)[PIECE]>(e[i * PIECE]), from, first(i), p.count - first(i), p.count);
#pragma unroll
            for (int r = 0; r < R; ++r) top = fmaxf(top, e[r]);
            top = join_lanes<LANES>(top, Larger{});
#pragma unroll
            for (int r = 0; r < R; ++r) {
                e[r] = exp_below(e[r] - top);
                sum += e[r];
            }
            sum = join_lanes<LANES>(sum, Sum{});
        }
        int at[HELD];
        float d[HELD], value[HELD], share[HELD], own_top = -INFINITY;
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            const int j = h * LANES + lane;
            at[h] = j < p.top ? p.experts[row * p.top + j] : -1;
            at[h] = (unsigned)at[h] < (unsigned)p.count ? at[h] : -1;
            d[h] = at[h] >= 0 ? p.scale * p.dweights[row * p.top + j] : 0.0f;
            value[h] = at[h] >= 0 ? (float)from[at[h]] : -INFINITY;
            own_top = fmaxf(own_top, SCORE == kSigmoid ? fminf(value[h], 0.0f) : value[h]);
        }
        if (p.renormalise) top = join_lanes<LANES>(own_top, Larger{});
        else if (SCORE == kSigmoid) top = 0.0f;
        float dot = 0.0f;
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            share[h] = at[h] >= 0 ? share_of<SCORE>(value[h], top) : 0.0f;
            if (p.renormalise) sum += share[h];
        }
        if (p.renormalise) sum = join_lanes<LANES>(sum, Sum{});
        // (quotients, not products with 1 / sum: one choice's share is 1, and its gradient 0)
        const bool shared = p.renormalise || SCORE == kSoftmax;
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            if (shared) share[h] = sum > 0.0f ? share[h] / sum : 0.0f;
            dot += d[h] * share[h];
        }
        dot = join_lanes<LANES>(dot, Sum{});
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            // (of the whole softmax: what a chosen one has beside the row's dot product)
            d[h] = share[h] * (p.renormalise ? d[h] - dot : d[h]);
            if (SCORE == kSigmoid) {                               // 1 - p
                const float x = exp_below(-__builtin_fabsf(value[h]));
                d[h] *= (value[h] > 0.0f ? x : 1.0f) / (1.0f + x);
            }
            const int j = h * LANES + lane;
            if (j < p.top) { taken[slot][j] = at[h] >= 0 ? d[h] : 0.0f; named[slot][j] = at[h]; }
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
#pragma unroll
            for (int k = 0; k < PIECE; ++k) spread[slot][first(i) + k] = 0.0f;
        wave_meets();
        // an expert that a row names more than once: the sum, in the order of the choices, written by each of them
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            float total = 0.0f;
            for (int j = 0; j < p.top; ++j) total += named[slot][j] == at[h] ? taken[slot][j] : 0.0f;
            if (at[h] >= 0) spread[slot][at[h]] = total;
        }
        wave_meets();
        if (own < p.rows) {
            T* to = static_cast<T*>(p.dlogits) + own * p.dstride;
            const float back = sum > 0.0f ? dot / sum : 0.0f;
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                float v[PIECE];
#pragma unroll
                for (int k = 0; k < PIECE; ++k) v[k] = spread[slot][first(i) + k] - (all ? e[i * PIECE + k] * back : 0.0f);
                if (PIECE == N && first(i) + N <= p.count) {
                    store_quad(to + first(i), v);
                } else {
#pragma unroll
                    for (int k = 0; k < PIECE; ++k)
                        if (first(i) + k < p.count) to[first(i) + k] = (T)v[k];
                }
            }
        }
        wave_meets();
    }
}

// The gradient has no groups, whose lanes would hold more experts, and no form of its own for few rows: route_any gives it none of these.
constexpr bool gradient_takes(int lanes, int r) { return lanes < 64 || r == 8 || r == 16; }

template <typename T, int LANES, int R, int SCORE>
hipError_t route_scores(const RouteParams& p, bool grad, hipStream_t s)
{
    constexpr int ROWS = kThreads / LANES;
    const long long want = ((long long)p.rows + ROWS - 1) / ROWS;
    const dim3 blocks((unsigned)(want < kRouteBlocks ? want : kRouteBlocks));
    if (grad) {
        if constexpr (gradient_takes(LANES, R)) hipLaunchKernelGGL((route_grad_kernel<T, LANES, R, SCORE>), blocks, dim3(kThreads), 0, s, p);
        else return hipErrorInvalidValue;
    } else if (sizeof(T) == 2 && !p.bias) {
        hipLaunchKernelGGL((route_kernel<T, LANES, R, SCORE, sizeof(T) == 2>), blocks, dim3(kThreads), 0, s, p);
    } else {
        hipLaunchKernelGGL((route_kernel<T, LANES, R, SCORE, false>), blocks, dim3(kThreads), 0, s, p);
    }
    return hipGetLastError();
}
template <typename T, int LANES, int R>
hipError_t route_rows(const RouteParams& p, bool grad, hipStream_t s)
{
    return p.score == kSoftmax ? route_scores<T, LANES, R, kSoftmax>(p, grad, s) : route_scores<T, LANES, R, kSigmoid>(p, grad, s);
}
// Lanes a row and experts a lane: four lanes where their registers hold the row and there are many, 16 rows a wave, then 16, but 64 for so few rows that waves are
// to spare; groups have whole lanes of their own.
template <typename T>
hipError_t route_any(RouteParams p, bool grad, hipStream_t s)
{
    p.log_groups = 0;
    while ((1 << p.log_groups) < p.groups) ++p.log_groups;
    const int size = p.count / p.groups;
    const auto part = [&](int lanes) { return lanes >> p.log_groups ? (size + (lanes >> p.log_groups) - 1) / (lanes >> p.log_groups) : 1 << 20; };
    const int least = p.top <= most_chosen(4) ? part(4) : 1 << 20, few = part(16), many = part(64);
    if (p.rows <= kFewRouteRows && !grad) {
        if (many <= 1) return route_rows<T, 64, 1>(p, grad, s);
        if (many <= 4) return route_rows<T, 64, 4>(p, grad, s);
    }
    if (p.rows >= (p.top <= kFewChoices ? kManyRouteRows : 2 * kManyRouteRows)) {
        if (least <= 8) return route_rows<T, 4, 8>(p, grad, s);
        if (least <= 16) return route_rows<T, 4, 16>(p, grad, s);
    }
    if (few <= 1) return route_rows<T, 16, 1>(p, grad, s);
    if (few <= 4) return route_rows<T, 16, 4>(p, grad, s);
    if (few <= 8) return route_rows<T, 16, 8>(p, grad, s);
    if (few <= 16) return route_rows<T, 16, 16>(p, grad, s);
    if (many <= 8) return route_rows<T, 64, 8>(p, grad, s);
    if (many <= 16) return route_rows<T, 64, 16>(p, grad, s);
    return route_rows<T, 64, 32>(p, grad, s);
}
hipError_t route(const RouteParams& p, int dtype, bool grad, hipStream_t s)
{
    switch (dtype) {
    case kF32: return route_any<float>(p, grad, s);
    case kBf16: return route_any<__bf16>(p, grad, s);
    default: return route_any<_Float16>(p, grad, s);
    }
}

// ------------------------------------------------------------------ order
// Counting sort, stable: an entry's place is the number of entries of smaller experts, and of its own in front of it.  Each workgroup has a run
// of entries, each of its 16 waves a run of that; entries of no expert count as one expert more.
// Two launches in a row and reads that wait for each other bound it: one workgroup of 1024 threads 4.0 us for 8 entries, 5.3 for 4096, 8.2 for 8192, 14 for 16384, where several take 8.7 (64 experts).
constexpr int kOrderThreads = 1024, kHeld = 4;
// Entries that 256 threads order, which meet sooner (64 experts, us: 8 entries 3.5, with 1024 threads 4.0; 512 3.8, 4.1; 1024 4.3, 4.2).
constexpr int kFewEntries = 512;
// Threads of the kernel that orders and the most experts that it has room for in LDS.
constexpr int kFewExperts = 256;
constexpr int order_threads(int count) { return count <= kFewExperts ? 1024 : 512; }

__device__ __forceinline__ int expert_of(const OrderParams& p, int i)
{
    const int e = p.experts[i];
    return (unsigned)e < (unsigned)p.count ? e : p.count;
}

// One more entry of expert x, for the lanes that have one.  Entries of no expert come in long runs (padding), and are counted at once: so many lanes
// at one place of LDS would wait for each other.
__device__ __forceinline__ void count_entry(int* counts, int x, bool there, int none)
{
    const unsigned long long of_none = __ballot(there && x == none);
    if (there && x != none) atomicAdd(&counts[x], 1);
    if (of_none && (threadIdx.x & 63) == (unsigned)__builtin_ctzll(of_none)) atomicAdd(&counts[none], __builtin_popcountll(of_none));
}

// entries of each expert in a workgroup's run
__global__ void __launch_bounds__(kOrderThreads) order_count_kernel(OrderParams p)
{
    __shared__ int counts[kMostRouted + 1];
    for (int e = threadIdx.x; e <= p.count; e += kOrderThreads) counts[e] = 0;
    __syncthreads();
    const long long begin = (long long)blockIdx.x * p.share, end = begin + p.share < p.entries ? begin + p.share : p.entries;
    for (long long i0 = begin; i0 < end; i0 += kOrderThreads) {
        const long long i = i0 + threadIdx.x;
        count_entry(counts, i < end ? expert_of(p, (int)i) : p.count, i < end, p.count);
    }
    __syncthreads();
    for (int e = threadIdx.x; e <= p.count; e += kOrderThreads) p.counts[(long long)blockIdx.x * (p.count + 1) + e] = counts[e];
}

template <int THREADS, int MOST>
__global__ void __launch_bounds__(THREADS) order_kernel(OrderParams p)
{
    constexpr int WAVES = THREADS / 64, EACH = (MOST + THREADS - 1) / THREADS;
    __shared__ int at[WAVES][MOST + 1];                   // counts of a wave's run, then the places of its next entries
    __shared__ unsigned long long alike[WAVES][MOST + 1]; // lanes with an entry of this expert
    __shared__ int before[MOST + 1], total[MOST + 1];
    __shared__ int ends_of_waves[WAVES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), bins = p.count + 1;
    const long long begin = (long long)blockIdx.x * p.share, end = begin + p.share < p.entries ? begin + p.share : p.entries;
    const int run = (int)(((end - begin + WAVES - 1) / WAVES + 63) / 64 * 64);
    const long long first = begin + (long long)wave * run, last = first + run < end ? first + run : end;
    // the first kHeld entries of a lane stay in registers for both looks at them
    int held[kHeld];
#pragma unroll
    for (int u = 0; u < kHeld; ++u) {
        const long long i = first + u * 64 + lane;
        held[u] = i < last ? p.experts[i] : -1;
    }
    for (int e = lane; e < bins; e += 64) {
        at[wave][e] = 0;
        alike[wave][e] = 0;
    }
    // what the workgroups in front have, and all of them
    if (p.counts) {
        // (several threads an expert where there are few; sixteen counts on their way at a time)
        for (int e = threadIdx.x; e < bins; e += THREADS) before[e] = total[e] = 0;
        __syncthreads();
        const int parts = bins >= THREADS ? 1 : THREADS / bins;
        for (int k = threadIdx.x; k < bins * parts; k += THREADS) {
            const int e = k % bins;
            int all = 0, front = 0;
            for (int b0 = k / bins; b0 < p.blocks; b0 += 16 * parts) {
                int c[16];
#pragma unroll
                for (int u = 0; u < 16; ++u) {
                    const int b = b0 + u * parts;
                    c[u] = b < p.blocks ? p.counts[(long long)b * bins + e] : 0;
                }
#pragma unroll
                for (int u = 0; u < 16; ++u) {
                    all += c[u];
                    front += b0 + u * parts < (int)blockIdx.x ? c[u] : 0;
                }
            }
            if (all) atomicAdd(&total[e], all);
            if (front) atomicAdd(&before[e], front);
        }
    }
#pragma unroll
    for (int u = 0; u < kHeld; ++u) {
        held[u] = (unsigned)held[u] < (unsigned)p.count ? held[u] : p.count;
        count_entry(at[wave], held[u], first + u * 64 + lane < last, p.count);
    }
    for (long long i0 = first + kHeld * 64; i0 < last; i0 += 64) {
        const bool there = i0 + lane < last;
        count_entry(at[wave], there ? expert_of(p, (int)(i0 + lane)) : p.count, there, p.count);
    }
    __syncthreads();
    if (!p.counts) {
        for (int e = threadIdx.x; e < bins; e += THREADS) {
            int all = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) all += at[w][e];
            total[e] = all;
            before[e] = 0;
        }
        __syncthreads();
    }
    // sums over the experts in front, EACH neighbours a thread (the last, of no expert, has its place behind all of them)
    int own[EACH], upto = 0;
#pragma unroll
    for (int u = 0; u < EACH; ++u) {
        const int e = threadIdx.x * EACH + u;
        own[u] = e < p.count ? total[e] : 0;
        upto += own[u];
    }
    const int mine = upto;
    for (int d = 1; d < 64; d <<= 1) {
        const int other = __shfl_up(upto, d, 64);
        if (lane >= d) upto += other;
    }
    if (lane == 63) ends_of_waves[wave] = upto;
    __syncthreads();
    int in_front = 0, all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const int c = ends_of_waves[w];
        in_front += w < wave ? c : 0;
        all += c;
    }
    const auto places_from = [&](int e, int place) {
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const int c = at[w][e];
            at[w][e] = place;
            place += c;
        }
    };
    int start = in_front + upto - mine;
#pragma unroll
    for (int u = 0; u < EACH; ++u) {
        const int e = threadIdx.x * EACH + u;
        if (e < p.count) {
            places_from(e, start + before[e]);
            if (blockIdx.x == 0) p.ends[e] = start + own[u];
        }
        start += own[u];
    }
    if (threadIdx.x == 0) places_from(p.count, all + before[p.count]);
    __syncthreads();
    // 64 entries at a time: each lane leaves its bit with its expert, and finds there who else did (comparing the experts' numbers bit by bit: 8192 entries
    // of one workgroup 10.6 us)
    volatile int* next = at[wave];
    volatile unsigned long long* mine_of = alike[wave];
    const auto place = [&](long long i, int x, bool there) {
        const unsigned long long of_none = __ballot(there && x == p.count);
        if (there && x != p.count) atomicOr(&alike[wave][x], 1ull << lane);
        wave_meets();
        if (there) {
            const unsigned long long same = x == p.count ? of_none : mine_of[x];
            const int at = next[x], rank = __builtin_popcountll(same & ((1ull << lane) - 1));
            p.places[i] = at + rank;
            if (same >> lane == 1) {                             // the last of its kind
                next[x] = at + rank + 1;
                mine_of[x] = 0;
            }
        }
        wave_meets();
    };
#pragma unroll
    for (int u = 0; u < kHeld; ++u)
        if (first + u * 64 < last) place(first + u * 64 + lane, held[u], first + u * 64 + lane < last);
    for (long long i0 = first + kHeld * 64; i0 < last; i0 += 64) {
        const bool there = i0 + lane < last;
        place(i0 + lane, there ? expert_of(p, (int)(i0 + lane)) : p.count, there);
    }
}

}  // namespace

hipError_t launch_route(const RouteParams& p, int dtype, hipStream_t s) { return route(p, dtype, false, s); }
hipError_t launch_route_grad(const RouteParams& p, int dtype, hipStream_t s) { return route(p, dtype, true, s); }

void plan_order(OrderParams* p)
{
    // one workgroup for few entries (no second launch; 999 experts, one / several: 4096 entries 7.9 / 8.9 us, 8192 12.8 / 9.1); otherwise up to 256 of at least
    // as many entries as lie in registers
    if (p->entries <= 2 * kHeld * order_threads(p->count)) {
        p->blocks = 1;
        p->share = p->entries;
        return;
    }
    const int least = order_threads(p->count) * kHeld, want = (p->entries + least - 1) / least;
    const int blocks = want < 256 ? want : 256;
    p->share = (int)((((long long)p->entries + blocks - 1) / blocks + 63) / 64 * 64);
    p->blocks = (int)(((long long)p->entries + p->share - 1) / p->share);
}

hipError_t launch_order(const OrderParams& p, hipStream_t s)
{
    if (p.blocks > 1) {
        hipLaunchKernelGGL(order_count_kernel, dim3(p.blocks), dim3(kOrderThreads), 0, s, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (p.entries <= kFewEntries) hipLaunchKernelGGL((order_kernel<256, kMostRouted>), dim3(1), dim3(256), 0, s, p);
    else if (p.count <= kFewExperts) hipLaunchKernelGGL((order_kernel<order_threads(kFewExperts), kFewExperts>), dim3(p.blocks), dim3(order_threads(kFewExperts)), 0, s, p);
    else hipLaunchKernelGGL((order_kernel<order_threads(kMostRouted), kMostRouted>), dim3(p.blocks), dim3(order_threads(kMostRouted)), 0, s, p);
    return hipGetLastError();
}

}  // namespace spinner
