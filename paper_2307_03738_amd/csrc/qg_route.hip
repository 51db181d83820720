// qg_route, qg_expert_plan, qg_experts_combine: what surrounds the experts' products.
#include <type_traits>

#include "qg_types.h"

namespace {

// --- choice -------------------------------------------------------------------------------------------------------

struct RouteArgs {
    const void *logits;
    const float *bias;
    int32_t *ids;
    float *weights;
    int64_t tokens, stride;
    int type, experts, top_k, sigmoid, groups, top_groups, two, renormalise;
    uint32_t group_magic;      // 2^32 / group size, rounded up: e / size = umulhi(e, magic) (e < 2^16, size > 1)
    float scale;
};

template <typename T> __device__ inline T lowest() { return (T)-__builtin_inff(); }

// v and what lane ^ OFF holds, in either order, once lanes that differ in lower bits hold the same: inside a row of 16 lanes by the vector ALU (pairs, quads, mirrored
// halves and rows), across rows by swaps.  (By way of LDS each step takes five times as long, and a choice is little else but such steps.)
template <typename T> struct Two { T a, b; };
template <int OFF>
__device__ inline Two<uint32_t> both(uint32_t v)
{
    if constexpr (OFF == 1) return {v, dpp<0xb1, 0xf>(v)};
    else if constexpr (OFF == 2) return {v, dpp<0x4e, 0xf>(v)};
    else if constexpr (OFF == 4) return {v, dpp<0x141, 0xf>(v)};
    else if constexpr (OFF == 8) return {v, dpp<0x140, 0xf>(v)};
    else if constexpr (OFF == 16) {
        const auto x = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return {x[0], x[1]};
    } else {
        const auto x = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return {x[0], x[1]};
    }
}
template <int OFF>
__device__ inline Two<float> both(float v)
{
    const Two<uint32_t> t = both<OFF>(__float_as_uint(v));
    return {__uint_as_float(t.a), __uint_as_float(t.b)};
}
template <int OFF>
__device__ inline Two<double> both(double v)
{
    const uint64_t bits = __builtin_bit_cast(uint64_t, v);
    const Two<uint32_t> low = both<OFF>((uint32_t)bits), high = both<OFF>((uint32_t)(bits >> 32));
    return {__builtin_bit_cast(double, (uint64_t)high.a << 32 | low.a), __builtin_bit_cast(double, (uint64_t)high.b << 32 | low.b)};
}

// op is the same either way round
template <int L, int OFF, typename T, typename OP>
__device__ inline T team_all(T v, OP op)
{
    if constexpr (OFF < L) {
        const Two<T> t = both<OFF>(v);
        return team_all<L, 2 * OFF>(op(t.a, t.b), op);
    } else return v;
}
__device__ inline float larger(float a, float b) { return __builtin_fmaxf(a, b); }       // (neither is NaN)
__device__ inline double larger(double a, double b) { return __builtin_fmax(a, b); }
__device__ inline float smaller(float a, float b) { return __builtin_fminf(a, b); }
__device__ inline double smaller(double a, double b) { return __builtin_fmin(a, b); }
template <int L, typename T>
__device__ inline T team_max(T v)
{
    return team_all<L, 1>(v, [](T a, T b) { return larger(a, b); });
}
template <int L, typename T>
__device__ inline T team_sum(T v)
{
    return team_all<L, 1>(v, [](T a, T b) { return a + b; });
}

// 1 / d, to a unit of its last place, for d of 1 and more.
__device__ inline double inverse_of(double d)
{
    double r = __builtin_amdgcn_rcp(d);
    r = __builtin_fma(__builtin_fma(-d, r, 1.0), r, r);
    r = __builtin_fma(__builtin_fma(-d, r, 1.0), r, r);
    return d == __builtin_inf() ? 0.0 : r;
}

// e^y = 2^n e^r, r = y - n ln 2 of at most 0.347, by the series up to r^12 / 12! (what is left out is below 2e-16); y is not NaN.  Its coefficients
// stay in scalar registers, one instruction each (as constants of the code they cost two moves more, and the choice of a prompt is bound by instructions).
struct Series {
    double c[11];
    __device__ inline Series()
    {
        double f = 1.0;
#pragma unroll
        for (int i = 0; i < 11; ++i) {
            f /= i + 2;
            c[i] = f;
            asm("" : "+s"(c[i]));
        }
    }
    __device__ inline double exp(double y) const
    {
        y = __builtin_fmin(__builtin_fmax(y, -800.0), 800.0);
        const double n = __builtin_rint(y * 1.4426950408889634);
        double r = __builtin_fma(n, -0x1.62e42feep-1, y);              // ln 2 in two parts, of which the first times n is exact
        r = __builtin_fma(n, -0x1.a39ef35793c76p-33, r);
        double p = c[10];
#pragma unroll
        for (int i = 9; i >= 0; --i) p = __builtin_fma(p, r, c[i]);
        p = __builtin_fma(p, r, 1.0);
        p = __builtin_fma(p, r, 1.0);
        return __builtin_amdgcn_ldexp(p, (int)n);
    }
    __device__ inline double sigmoid(float x) const { return inverse_of(1.0 + exp(-(double)x)); }
};

__device__ inline float logit_of(const RouteArgs &a, int64_t at)
{
    return a.type == QG_F32 ? load_as_float<QG_F32>(a.logits, at) : a.type == QG_BF16 ? load_as_float<QG_BF16>(a.logits, at) : load_as_float<QG_F16>(a.logits, at);
}

// A few tokens are bound by latency: a load, exponentials in fp64 where a weight or a rank needs them, and top_k steps of log2 L exchanges (one token, six of 64: 3.0 us, an empty
// launch 2.4).  Many are bound by instructions (8190 tokens of bf16, seven of 192 in 12 groups, sigmoids and a bias: 12.5 us, 1300 vector instructions a wavefront, 9 us of issue; 3.6 MB).  16 lanes a
// token where they suffice, so that four tokens share a wavefront's steps.
// L lanes take a token, V experts each: expert v * L + lane.  KEY: what experts rank by, fp32 logits, or, with a bias or
// groups ranked by sums, scores in fp64 (two fp32 scores with a bias tie or swap in about one of 10^5 choices).
template <int L, int V, typename KEY>
__global__ __launch_bounds__(256) void route(RouteArgs a)
{
    constexpr bool SCORES = sizeof(KEY) == 8;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int lane = threadIdx.x % L, team = threadIdx.x / L;
    const int64_t wanted = (int64_t)blockIdx.x * (256 / L) + team;
    const int64_t token = wanted < a.tokens ? wanted : a.tokens - 1;      // lanes past the end work along and store nothing
    const int64_t row = token * a.stride;

    // what a call asks for is asked once, not for each expert, and lanes past the last expert read it: all of a lane's experts are under way at once
    int at[V];
#pragma unroll
    for (int v = 0; v < V; ++v) at[v] = min(v * L + lane, a.experts - 1);
    float l[V], b[V];
    auto read = [&](auto type) {
#pragma unroll
        for (int v = 0; v < V; ++v) l[v] = load_as_float<decltype(type)::value>(a.logits, row + at[v]);
    };
    if (a.type == QG_F32) read(std::integral_constant<int, QG_F32>());
    else if (a.type == QG_BF16) read(std::integral_constant<int, QG_BF16>());
    else read(std::integral_constant<int, QG_F16>());
    if constexpr (SCORES) {
#pragma unroll
        for (int v = 0; v < V; ++v) b[v] = a.bias ? a.bias[at[v]] : 0.0f;
    }
    bool nan = false;
    float most = lowest<float>();
#pragma unroll
    for (int v = 0; v < V; ++v) {
        nan |= l[v] != l[v];
        l[v] = l[v] != l[v] || v * L + lane >= a.experts ? lowest<float>() : l[v];
        most = larger(most, l[v]);
    }
    // softmax: the largest logit and, where a weight needs it, the sum of exponentials; of infinite logits each counts 1 and the others 0
    const bool sums = !a.sigmoid && (SCORES || !a.renormalise);
    if (!a.sigmoid) most = team_max<L>(most);
    const float base = most == lowest<float>() ? 0.0f : most;
    const Series series;
    auto raised = [&](float x) { return series.exp(x == base ? 0.0 : (double)x - (double)base); };
    double total = 1.0;
    KEY key[V];
    if constexpr (SCORES) {
        if (a.sigmoid) {
#pragma unroll
            for (int v = 0; v < V; ++v) key[v] = series.sigmoid(l[v]);
        } else {
            double part = 0.0;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                key[v] = raised(l[v]);
                part += key[v];
            }
            total = team_sum<L>(part);
            const double scale = inverse_of(total);     // (1 or more, or all are switched off)
#pragma unroll
            for (int v = 0; v < V; ++v) key[v] *= scale;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (a.bias) key[v] += (double)b[v];
            const bool off = l[v] == lowest<float>(), bad = key[v] != key[v];
            nan |= bad && !off;
            key[v] = off || bad ? lowest<KEY>() : key[v];
        }
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = l[v];
        if (sums) {
            double part = 0.0;
#pragma unroll
            for (int v = 0; v < V; ++v) part += raised(l[v]);
            total = team_sum<L>(part);
        }
    }
    const uint64_t nans = __ballot(nan);
    nan = ((nans >> (threadIdx.x % 64 / L * L)) & (L == 64 ? ~0ull : (1ull << (L % 64)) - 1)) != 0;

    if (a.top_groups < a.groups) {
        // keys of the token, then its groups' ranks
        KEY *keys = (KEY *)smem + (size_t)team * (a.experts + a.groups), *ranks = keys + a.experts;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int e = v * L + lane;
            if (e < a.experts) keys[e] = key[v];
        }
        __syncthreads();
        const int size = a.experts / a.groups;
        for (int g = lane; g < a.groups; g += L) {
            KEY first = lowest<KEY>(), second = lowest<KEY>();
#pragma unroll 4
            for (int i = 0; i < size; ++i) {
                const KEY k = keys[g * size + i];
                second = larger(second, smaller(first, k));
                first = larger(first, k);
            }
            ranks[g] = a.two && second > lowest<KEY>() ? first + second : first;
        }
        __syncthreads();
        // which groups take part, a bit each, over the first keys (which all have read)
        uint32_t *takes = (uint32_t *)keys;
        for (int g0 = 0; g0 < a.groups; g0 += L) {
            const int g = g0 + lane;
            int before = 0;
            if (g < a.groups) {
                const KEY mine = ranks[g];
                for (int o = 0; o < a.groups; ++o) {
                    const KEY r = ranks[o];
                    before += r > mine || (r == mine && o < g);
                }
            }
            const uint64_t all = __ballot(g < a.groups && before < a.top_groups) >> (threadIdx.x % 64 / L * L);
            if (lane == 0) {
                if constexpr (L == 16) ((uint16_t *)takes)[g0 / 16] = (uint16_t)all;
                else takes[g0 / 32] = (uint32_t)all;
                if constexpr (L == 64) takes[g0 / 32 + 1] = (uint32_t)(all >> 32);
            }
        }
        __syncthreads();
        // scores rank groups; without a bias experts rank by their logits all the same (sigmoids near 1 and far softmaxes tie)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int e = v * L + lane, g = size == 1 ? e : (int)__umulhi((uint32_t)e, a.group_magic);
            const bool kept = e < a.experts && (takes[g >> 5] >> (g & 31) & 1);
            key[v] = !kept || key[v] == lowest<KEY>() ? lowest<KEY>() : SCORES && !a.bias ? (KEY)l[v] : key[v];
        }
    }

    int mine = -1;                         // lane j: the token's choice j
    for (int j = 0; j < a.top_k; ++j) {
        KEY best = key[0];
#pragma unroll
        for (int v = 1; v < V; ++v) best = larger(best, key[v]);
        best = team_max<L>(best);          // -infinity: none is left for this token; others of the wavefront may go on
        // the first that has it: for a token of a whole wavefront by scalar instructions, a mask of lanes for each v (4000 tokens, 12 of 512: 9.3 us against 9.9); for two
        // tokens that takes twice as many (8190 tokens, 7 of 192: 13.9 us against 12.8)
        int at = 0x7fffffff;
        if constexpr (L == 64) {
#pragma unroll
            for (int v = V - 1; v >= 0; --v) {
                const uint64_t has = __ballot(key[v] == best);
                at = has ? v * L + __builtin_ctzll(has) : at;
            }
        } else {
#pragma unroll
            for (int v = V - 1; v >= 0; --v) at = key[v] == best ? v * L + lane : at;
            at = (int)team_all<L, 1>((uint32_t)at, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
        }
        const bool real = best > lowest<KEY>();
        if (lane == j) mine = real ? at : -1;
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = v * L + lane == at ? lowest<KEY>() : key[v];
    }
    double p = 0.0;
    if (mine >= 0) {
        const float x = logit_of(a, row + mine);
        p = a.sigmoid ? series.sigmoid(x) : raised(x);
    }
    if (a.renormalise) {
        const double sum = team_sum<L>(p);
        p = sum == 0.0 ? 0.0 : p / sum;
    } else if (!a.sigmoid) {
        p /= total == 0.0 ? 1.0 : total;
    }
    if (wanted < a.tokens && lane < a.top_k) {
        a.ids[token * a.top_k + lane] = mine;
        a.weights[token * a.top_k + lane] = nan ? __uint_as_float(0x7fc00000u) : (float)(p * (double)a.scale);
    }
}

template <int L, int V>
void route_launch(const RouteArgs &a, bool scores, hipStream_t st)
{
    const int teams = 256 / L;
    RouteArgs b = a;
    const int64_t turn = QG_MOST_GROUPS * teams;
    for (int64_t done = 0; done < a.tokens; done += turn) {
        b.tokens = a.tokens - done < turn ? a.tokens - done : turn;
        b.logits = (const char *)a.logits + done * a.stride * qg_type_bytes(a.type);
        b.ids = a.ids + done * a.top_k;
        b.weights = a.weights + done * a.top_k;
        const unsigned blocks = (unsigned)((b.tokens + teams - 1) / teams);
        const size_t lds = a.top_groups < a.groups ? (size_t)teams * (a.experts + a.groups) * (scores ? 8 : 4) : 0;
        if (scores) route<L, V, double><<<blocks, 256, lds, st>>>(b);
        else route<L, V, float><<<blocks, 256, lds, st>>>(b);
    }
}

// --- order --------------------------------------------------------------------------------------------------------

struct PlanArgs {
    const int32_t *ids;
    int32_t *offsets, *slot_tokens, *slots;
    uint32_t pairs, part;      // choices in all, and of a workgroup
    int top_k, experts, bits;  // bits: of an expert's number
    int32_t *counted;          // parts' choices of each expert, [parts][experts]; or NULL: they are counted where they are needed
    int parts;
};

constexpr int PLAN_WAVES = 16;

// Choices of each expert in a part.
__global__ __launch_bounds__(64 * PLAN_WAVES) void plan_count(PlanArgs a)
{
    extern __shared__ __attribute__((aligned(16))) char smem[];
    int32_t *all = (int32_t *)smem;
    for (int e = threadIdx.x; e < a.experts; e += 64 * PLAN_WAVES) all[e] = 0;
    __syncthreads();
    const uint32_t begin = blockIdx.x * a.part, end = min(a.pairs, begin + a.part);
    for (uint32_t i = begin + threadIdx.x; i < end; i += 64 * PLAN_WAVES) {
        const uint32_t e = (uint32_t)a.ids[i];
        if (e < (uint32_t)a.experts) atomicAdd(&all[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += 64 * PLAN_WAVES) a.counted[(int64_t)blockIdx.x * a.experts + e] = all[e];
}

// Slots' tokens, of choices' slots.
__global__ __launch_bounds__(256) void plan_tokens(PlanArgs a)
{
    const uint32_t i = blockIdx.x * 256u + threadIdx.x;
    if (i >= a.pairs) return;
    const int slot = a.slots[i];
    if (slot >= 0) a.slot_tokens[slot] = (int32_t)(i / (uint32_t)a.top_k);
    if (i >= (uint32_t)a.offsets[a.experts]) a.slot_tokens[i] = -1;
}

// A stable counting sort: every workgroup has the counts of all choices, those before its own part apart, adds the counts up to where
// each expert begins, and places its part: wavefront by wavefront in order, inside a wavefront by the lanes with the same expert before it.
// Up to 8 parts of 2048 choices each workgroup counts them all itself, in one launch.  Beyond, parts are counted by a launch before, into what will be slot_tokens, which
// is therefore filled by a launch after (16383 tokens' eight choices of 192: 13.5 to 15 us as a caller sees it, kernels 2.5 + 7.3 + 2.1; 27.7 in one launch).
// Bound by latency, about a launch and four meetings: 48 tokens' four of 32, 3.5 to 4 us.
// LDS: counts of all choices [experts], where the next choice goes [wave][experts].
__global__ __launch_bounds__(64 * PLAN_WAVES) void plan(PlanArgs a)
{
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int E = a.experts, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t *all = (int32_t *)smem, *next = all + E;
    __shared__ int32_t sums[PLAN_WAVES];
    for (int i = threadIdx.x; i < E * (PLAN_WAVES + 1); i += 64 * PLAN_WAVES) all[i] = 0;
    __syncthreads();
    const uint32_t begin = blockIdx.x * a.part, end = min(a.pairs, begin + a.part);
    const uint32_t per_wave = (a.part / PLAN_WAVES), w0 = min(end, begin + wave * per_wave), w1 = min(end, w0 + per_wave);
    // choices before the part count into the first wavefront's places, as do those of wavefronts before another's into its own
    if (a.counted) {
        // a quarter of the workgroup, at least, goes along the parts of 256 experts
        for (int i = threadIdx.x; i < E * 4; i += 64 * PLAN_WAVES) {
            const int e = i % E, quarter = i / E;
            int sum = 0, before = 0;
#pragma unroll 4
            for (int p = quarter; p < a.parts; p += 4) {
                const int n = a.counted[(int64_t)p * E + e];
                sum += n;
                if (p < (int)blockIdx.x) before += n;
            }
            atomicAdd(&all[e], sum);
            atomicAdd(&next[e], before);
        }
    } else {
        for (uint32_t i = threadIdx.x; i < a.pairs; i += 64 * PLAN_WAVES) {
            const uint32_t e = (uint32_t)a.ids[i];
            if (e < (uint32_t)E) {
                atomicAdd(&all[e], 1);
                if (i < begin) atomicAdd(&next[e], 1);
            }
        }
    }
    for (uint32_t i = w0 + lane; i < w1; i += 64) {
        const uint32_t e = (uint32_t)a.ids[i];
        if (e < (uint32_t)E && wave + 1 < PLAN_WAVES) atomicAdd(&next[(wave + 1) * E + e], 1);
    }
    __syncthreads();
    // where experts begin: sums over 64 x PLAN_WAVES >= QG_MAX_EXPERTS lanes
    const int e = threadIdx.x;
    const int count = e < E ? all[e] : 0;
    int upto = count;
#pragma unroll
    for (int off = 1; off < 64; off *= 2) {
        const int o = __shfl_up(upto, off);
        if (lane >= off) upto += o;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int total = 0;
    for (int w = 0; w < PLAN_WAVES; ++w) {
        if (w < wave) upto += sums[w];
        total += sums[w];
    }
    if (e < E) {
        int at = upto - count;
        if (blockIdx.x == 0) a.offsets[e] = at;
        for (int w = 0; w < PLAN_WAVES; ++w) {
            at += next[w * E + e];
            next[w * E + e] = at;
        }
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) a.offsets[E] = total;
    if (!a.counted)
        for (uint32_t i = total + blockIdx.x * 64 * PLAN_WAVES + threadIdx.x; i < a.pairs; i += gridDim.x * 64 * PLAN_WAVES) a.slot_tokens[i] = -1;
    __syncthreads();
    int32_t *places = next + wave * E;
    for (uint32_t i0 = w0; i0 < w1; i0 += 64) {
        const uint32_t i = i0 + lane;
        const uint32_t id = i < w1 ? (uint32_t)a.ids[i] : 0xffffffffu;
        const bool real = id < (uint32_t)E;
        uint64_t same = __ballot(real);
        for (int b = 0; b < a.bits; ++b) {
            const bool bit = (id >> b) & 1;
            const uint64_t set = __ballot(bit);
            same &= bit ? set : ~set;
        }
        const int before = __popcll(same & ((1ull << lane) - 1));
        int slot = -1;
        if (real) slot = places[id] + before;
        // all of the wavefront have read before the first of each expert writes, and it has written before the next 64 read
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (real && before == 0) places[id] += __popcll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (i < w1) a.slots[i] = slot;
        if (real && !a.counted) a.slot_tokens[slot] = (int32_t)(i / (uint32_t)a.top_k);
    }
}

// --- sum ----------------------------------------------------------------------------------------------------------

struct CombineArgs {
    const void *y;
    const int32_t *slots;
    const float *weights;
    const void *residual;
    void *out;
    int64_t y_rows, tokens, N, residual_stride;
    int top_k;
    uint32_t chunks;           // workgroups of a token
};

// Eight neighbouring elements that begin anywhere (rows of odd widths): the hardware takes vectors at any element's address.
template <int TYPE>
__device__ inline void load_eight_anywhere(const void *p, int64_t i, float *v)
{
    if constexpr (TYPE == QG_F32) {
        __builtin_memcpy(v, (const float *)p + i, 32);
    } else {
        uint32_t w[4];
        __builtin_memcpy(w, (const uint16_t *)p + i, 16);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t bits = e % 2 ? w[e / 2] >> 16 : w[e / 2] & 0xffffu;
            v[e] = TYPE == QG_BF16 ? bf16_to_float(bits) : f16_to_float(bits);
        }
    }
}
template <int TYPE>
__device__ inline void store_eight_anywhere(void *p, int64_t i, const float *v)
{
    if constexpr (TYPE == QG_F32) {
        __builtin_memcpy((float *)p + i, v, 32);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            w[e] = TYPE == QG_BF16 ? float_to_bf16(v[2 * e]) | float_to_bf16(v[2 * e + 1]) << 16 : float_to_f16(v[2 * e]) | float_to_f16(v[2 * e + 1]) << 16;
        __builtin_memcpy((uint16_t *)p + i, w, 16);
    }
}

// A lane takes eight neighbouring columns of a token, the last one of a row as many as there are.  The token's slots and weights are loaded by a lane each
// (64 choices at most); four choices' rows are under way at once.  Bound by memory: 4095 tokens' eight rows of 5120 bf16 and a residual, 414 MB, 79 to 81 us, 5.1 to 5.2 TB/s;
// 24 tokens of four fp32 rows of 4096: 3.1 us, an empty launch 2.4.
template <int TYPE, int OUT>
__global__ __launch_bounds__(256) void combine(CombineArgs a)
{
    const uint32_t token = blockIdx.x / a.chunks;
    const int64_t n = ((int64_t)(blockIdx.x - token * a.chunks) * 256 + threadIdx.x) * 8;
    const int choice = threadIdx.x & 63;
    int slot = -1;
    float weight = 0.0f;
    if (choice < a.top_k) {
        slot = a.slots[(int64_t)token * a.top_k + choice];
        weight = a.weights[(int64_t)token * a.top_k + choice];
    }
    if (slot >= a.y_rows) slot = -1;
    const int64_t left = a.N - n;
    if (__ballot(left > 0) == 0) return;
    const bool whole = left >= 8;
    float sum[8];
#pragma unroll
    for (int v = 0; v < 8; ++v) sum[v] = 0.0f;
    auto take = [&](int64_t row, float *v) {
        if (whole) {
            load_eight_anywhere<TYPE>(a.y, row * a.N + n, v);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < left ? load_as_float<TYPE>(a.y, row * a.N + n + i) : 0.0f;
        }
    };
    if (a.residual) {
        const int64_t at = (int64_t)token * a.residual_stride + n;
        if (whole) {
            load_eight_anywhere<OUT>(a.residual, at, sum);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) sum[i] = load_as_float<OUT>(a.residual, at + i);
        }
    }
    for (int j = 0; j < a.top_k; j += 4) {
        float v[4][8];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int row = __builtin_amdgcn_readlane(slot, min(j + u, 63));
            if (j + u < a.top_k && row >= 0) take(row, v[u]);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int row = __builtin_amdgcn_readlane(slot, min(j + u, 63));
            const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weight), min(j + u, 63)));
            if (j + u < a.top_k && row >= 0)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] = __builtin_fmaf(w, v[u][i], sum[i]);
        }
    }
    const int64_t at = (int64_t)token * a.N + n;
    if (whole) {
        store_eight_anywhere<OUT>(a.out, at, sum);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) store_float<OUT>(a.out, at + i, sum[i]);
    }
}

template <int TYPE, int OUT>
void combine_launch(const CombineArgs &a, hipStream_t st)
{
    CombineArgs b = a;
    b.chunks = (uint32_t)((a.N + 2047) / 2048);
    const int64_t turn = QG_MOST_GROUPS / b.chunks > 0 ? QG_MOST_GROUPS / b.chunks : 1;
    for (int64_t done = 0; done < a.tokens; done += turn) {
        b.tokens = a.tokens - done < turn ? a.tokens - done : turn;
        b.slots = a.slots + done * a.top_k;
        b.weights = a.weights + done * a.top_k;
        if (a.residual) b.residual = (const char *)a.residual + done * a.residual_stride * qg_type_bytes(OUT);
        b.out = (char *)a.out + done * a.N * qg_type_bytes(OUT);
        const unsigned blocks = (unsigned)(b.tokens * b.chunks);
        combine<TYPE, OUT><<<blocks, 256, 0, st>>>(b);
    }
}

template <int TYPE>
void combine_typed(const CombineArgs &a, int out, hipStream_t st)
{
    if (out == QG_F32) combine_launch<TYPE, QG_F32>(a, st);
    else if (out == QG_BF16) combine_launch<TYPE, QG_BF16>(a, st);
    else combine_launch<TYPE, QG_F16>(a, st);
}

}  // namespace

extern "C" int qg_route(const qg_route_desc *d, void *stream)
{
    if (!d) return QG_ERR_NULL;
    if (!qg_float_type(d->type) || (d->score != QG_SOFTMAX && d->score != QG_SIGMOID)) return QG_ERR_UNSUPPORTED;
    if (d->experts > QG_MAX_EXPERTS || d->top_k > QG_MAX_CHOICES || (d->group_best != 1 && d->group_best != 2)) return QG_ERR_UNSUPPORTED;
    if (d->tokens < 0 || d->experts <= 0 || d->top_k <= 0 || d->groups <= 0 || d->experts % d->groups || d->top_groups <= 0 || d->top_groups > d->groups) return QG_ERR_SHAPE;
    if (d->top_k > d->experts / d->groups * d->top_groups || d->tokens > 0x7fffffff / d->top_k) return QG_ERR_SHAPE;
    if (d->tokens > 1 && d->logits_stride < d->experts) return QG_ERR_SHAPE;
    if (d->tokens == 0) return QG_OK;
    if (!d->logits || !d->ids || !d->weights) return QG_ERR_NULL;
    if (!qg_aligned_to(d->logits, qg_type_bytes(d->type)) || !qg_aligned_to(d->bias, 4) || !qg_aligned_to(d->ids, 4) || !qg_aligned_to(d->weights, 4)) return QG_ERR_ALIGN;
    const uint32_t size = (uint32_t)(d->experts / d->groups);
    const RouteArgs a = {d->logits, d->bias, d->ids, d->weights, d->tokens, d->logits_stride, d->type, d->experts, d->top_k, d->score == QG_SIGMOID,
                         d->groups, d->top_groups, d->group_best == 2, d->renormalise != 0, size > 1 ? (uint32_t)(((uint64_t)1 << 32) / size + 1) : 0, d->scale};
    const bool scores = d->bias || (d->top_groups < d->groups && d->group_best == 2);
    const hipStream_t st = (hipStream_t)stream;
    const int E = d->experts, k = d->top_k;
    // as few lanes a token as eight experts a lane allow, and one a choice at least
    if (E <= 64 && k <= 16) route_launch<16, 4>(a, scores, st);
    else if (E <= 128 && k <= 16) route_launch<16, 8>(a, scores, st);
    else if (E <= 192 && k <= 32) route_launch<32, 6>(a, scores, st);
    else if (E <= 256 && k <= 32) route_launch<32, 8>(a, scores, st);
    else if (E <= 512) route_launch<64, 8>(a, scores, st);
    else route_launch<64, 16>(a, scores, st);
    return qg_launch_status();
}

extern "C" int qg_expert_plan(const int32_t *ids, int64_t tokens, int top_k, int experts, int32_t *offsets, int32_t *slot_tokens, int32_t *slots, void *stream)
{
    if (experts > QG_MAX_EXPERTS) return QG_ERR_UNSUPPORTED;
    if (tokens < 0 || top_k <= 0 || experts <= 0 || tokens > 0x3fffffff / top_k) return QG_ERR_SHAPE;
    if (!offsets || (tokens && (!ids || !slot_tokens || !slots))) return QG_ERR_NULL;
    if (!qg_aligned_to(ids, 4) || !qg_aligned_to(offsets, 4) || !qg_aligned_to(slot_tokens, 4) || !qg_aligned_to(slots, 4)) return QG_ERR_ALIGN;
    PlanArgs a = {ids, offsets, slot_tokens, slots, (uint32_t)(tokens * top_k), 64 * PLAN_WAVES, top_k, experts, 0, nullptr, 0};
    while (a.bits < 10 && (experts - 1) >> a.bits) ++a.bits;
    // parts of 2048 choices, of more where that would take more workgroups than compute units
    const uint32_t blocks = (uint32_t)qg_compute_units();
    a.part = 2048;
    while ((uint64_t)a.part * blocks < a.pairs) a.part *= 2;
    const unsigned grid = a.pairs ? (a.pairs + a.part - 1) / a.part : 1;
    const size_t lds = (size_t)experts * (PLAN_WAVES + 1) * 4;
    if (lds > 65536 - 1024 && hipFuncSetAttribute((const void *)plan, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) {
        (void)hipGetLastError();
        return QG_ERR_DEVICE;
    }
    const hipStream_t st = (hipStream_t)stream;
    // (parts have 2048 choices at least, experts are 1024 at most: the counts fit)
    if (grid > 8) {
        a.counted = slot_tokens;
        a.parts = (int)grid;
        plan_count<<<grid, 64 * PLAN_WAVES, (size_t)experts * 4, st>>>(a);
    }
    plan<<<grid, 64 * PLAN_WAVES, lds, st>>>(a);
    if (grid > 8) plan_tokens<<<(a.pairs + 255) / 256, 256, 0, st>>>(a);
    return qg_launch_status();
}

extern "C" int qg_experts_combine(const qg_combine_desc *d, void *stream)
{
    if (!d) return QG_ERR_NULL;
    if (!qg_float_type(d->type) || !qg_float_type(d->out_type)) return QG_ERR_UNSUPPORTED;
    if (d->top_k > QG_MAX_CHOICES) return QG_ERR_UNSUPPORTED;
    if (d->tokens < 0 || d->N <= 0 || d->N > (int64_t)1 << 24 || d->top_k <= 0 || d->y_rows < 0 || d->y_rows > 0x7fffffff || d->tokens > 0x7fffffff / d->top_k) return QG_ERR_SHAPE;
    if (d->residual && d->tokens > 1 && d->residual_stride < d->N) return QG_ERR_SHAPE;
    if (d->tokens == 0) return QG_OK;
    if ((!d->y && d->y_rows) || !d->slots || !d->weights || !d->out) return QG_ERR_NULL;
    const int in = qg_type_bytes(d->type), out = qg_type_bytes(d->out_type);
    if (!qg_aligned_to(d->y, in) || !qg_aligned_to(d->residual, out) || !qg_aligned_to(d->out, out) || !qg_aligned_to(d->slots, 4) || !qg_aligned_to(d->weights, 4))
        return QG_ERR_ALIGN;
    const CombineArgs a = {d->y, d->slots, d->weights, d->residual, d->out, d->y_rows, d->tokens, d->N, d->residual_stride, d->top_k, 0};
    const hipStream_t st = (hipStream_t)stream;
    if (d->type == QG_F32) combine_typed<QG_F32>(a, d->out_type, st);
    else if (d->type == QG_BF16) combine_typed<QG_BF16>(a, d->out_type, st);
    else combine_typed<QG_F16>(a, d->out_type, st);
    return qg_launch_status();
}
