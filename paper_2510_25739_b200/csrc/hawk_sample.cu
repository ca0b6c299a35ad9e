// hawk_sample: one token from every row of logits by a given random number (Sec. 5's settings of generation, with top-p and min-p).
//
// All three filters keep the ids whose logit is at least a threshold, so a row needs no sorted copy: it needs three numbers.  A threshold is
// the largest value at which the ids from it up reach a target, their number for top-k, their mass for top-p, and is found by
// a histogram of 1024 equal steps of the value, its prefix sum, and the exact order inside the one step where the target is reached (its
// members against each other; a step with more than kList of them is cut into 1024 again).  Masses are exp() in fp64, held as multiples of
// 2^-44 in 64-bit integers: sums of them are exact, so the atomics' order has no say and a token does not depend on the launch.
// fp32 sums would not do: with 16 thousand ids one draw in some hundred falls so near to a border that their rounding decides it.
//
// A row is read from memory once and stays in shared memory as fp32, 32768 values a block at most; longer rows, and rows of calls
// with few of them, are shared by a cluster, whose blocks exchange histograms, list members and sums through distributed shared memory.
#include <climits>

#include <math_constants.h>

#include "hawk_common.cuh"

namespace {

using u64 = unsigned long long;

constexpr int kBins = 1024;
constexpr int kList = 512;       // members of a step that are ranked against each other
constexpr int kMaxSlice = 32768; // ids of a row that a block holds
constexpr int kMaxCluster = 8;
constexpr double kOne = 17592186044416.0;  // 2^44: the weight of the largest logit; 2^18 such weights fit 64 bits

struct SampleParams {
    const void *logits, *uncond;
    long long row_stride, uncond_stride, probs_stride;
    const float *temperatures, *top_ps, *min_ps, *scales, *u;
    const int32_t *top_ks;
    float temperature, top_p, min_p, scale;
    int top_k, V, v_begin, n, slice, cluster;  // n: ids of the range; slice: of a block
    int32_t *token;
    float *token_prob, *probs;
    int32_t *dev_status;
};

struct Swap {  // what the blocks of a row tell each other
    u64 a;
    float lo, hi;
    int n, flag;
};

struct SampleShared {
    u64 hist[kBins];
    u64 list_w[kList], all_w[kList];
    float list_v[kList], all_v[kList];
    u64 warp[32];
    float warp_lo[32], warp_hi[32];
    int warp_n[32];
    Swap swap[3];  // one for each kind of exchange, so that a barrier lies between two uses of the same
    u64 above, target;
    int bin, count, pick;
    uint32_t lo_key, hi_key, tau_key;
};

// Barrier of the row's blocks (lanes that a branch parted come together first).
__device__ __forceinline__ void meet()
{
    __syncwarp();
    hawk::cluster_sync_all();
}

// Unsigned number in the order of the values.
__device__ __forceinline__ uint32_t key_of(float v)
{
    const uint32_t b = __float_as_uint(v);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

__device__ __forceinline__ u64 warp_inclusive(u64 v)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const u64 x = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += x;
    }
    return v;
}

// Exclusive prefix sum over the block's NT threads, and the sum of all.
template <int NT>
__device__ __forceinline__ u64 block_exclusive(u64 v, u64 *sh, u64 &total)
{
    const u64 inc = warp_inclusive(v);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __syncthreads();  // (sh may still be read from the sum before)
    if (lane == 31) sh[warp] = inc;
    __syncthreads();
    const u64 sums = warp_inclusive(lane < NT / 32 ? sh[lane] : 0);
    total = __shfl_sync(0xffffffffu, sums, 31);
    const u64 before = __shfl_sync(0xffffffffu, sums, warp > 0 ? warp - 1 : 0);
    return (warp > 0 ? before : 0) + inc - v;
}

// Steps of equal width from hi down to lo: monotone in the value, 0 for hi, the last for lo.  Ranges that fp32 cannot divide (next to
// nothing, or wider than its largest number) are divided in fp64.
struct Steps {
    float hi, per;
    double wide;
    __device__ __forceinline__ Steps(float lo, float top) : hi(top), wide(0.0)
    {
        const float range = top - lo;
        if (range > 1e-30f && range < 3e38f) {
            per = kBins / range;
        } else {
            per = 0.f;
            wide = kBins / (static_cast<double>(top) - static_cast<double>(lo));
        }
    }
    __device__ __forceinline__ int operator()(float v) const
    {
        const int b = per > 0.f ? static_cast<int>((hi - v) * per)
                                : static_cast<int>((static_cast<double>(hi) - static_cast<double>(v)) * wide);
        return min(b, kBins - 1);
    }
};

template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32(float v) { return v; }
template <>
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <>
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }

template <typename T>
struct Piece {  // 16 bytes of logits
    static constexpr int kN = 16 / sizeof(T);
    uint4 raw;
    __device__ __forceinline__ float at(int i) const { return to_f32(reinterpret_cast<const T *>(&raw)[i]); }
};

// The row's guided logit; what is not a number that can be drawn becomes -inf.
__device__ __forceinline__ float guided(float c, float u, bool has, float scale, int &flags)
{
    float l = c;
    if (has) {
        l = __fmaf_rn(scale, __fsub_rn(c, u), u);
        if (c == -CUDART_INF_F || u == -CUDART_INF_F) l = -CUDART_INF_F;
        // (an infinite or undefined input cannot come out finite, whatever the scale)
        if (!(fabsf(c) < CUDART_INF_F) || !(fabsf(u) < CUDART_INF_F)) {
            if (!(c == -CUDART_INF_F) && !(fabsf(c) < CUDART_INF_F)) flags |= HAWK_DEV_NONFINITE;
            if (!(u == -CUDART_INF_F) && !(fabsf(u) < CUDART_INF_F)) flags |= HAWK_DEV_NONFINITE;
            return -CUDART_INF_F;
        }
    }
    if (!(l < CUDART_INF_F)) {  // NaN, +inf
        flags |= HAWK_DEV_NONFINITE;
        l = -CUDART_INF_F;
    }
    return l + 0.f;  // (one zero)
}

template <typename T, int NT>
class Row {
public:
    __device__ __forceinline__ Row(const SampleParams &p, SampleShared &s, float *v) : P(p), sh(s), vals(v) {}
    __device__ __forceinline__ void run();

private:
    const SampleParams &P;
    SampleShared &sh;
    float *vals;  // [m] logits of the block's ids, -inf around them
    int m, rank, flags = 0;
    float mx;
    double inv_t;

    __device__ __forceinline__ bool shared() const { return P.cluster > 1; }
    __device__ __forceinline__ double power(float l) const { return exp((static_cast<double>(l) - static_cast<double>(mx)) * inv_t); }
    __device__ __forceinline__ u64 weight(float l) const { return __double2ull_rn(power(l) * kOne); }
    __device__ __forceinline__ Swap of(int slot, int r) const
    {
        const uint32_t at = hawk::map_shared_to_cta(&sh.swap[slot], r);
        Swap s;
        s.a = hawk::ld_cluster_u64(at);
        s.lo = __uint_as_float(hawk::ld_cluster_u32(at + 8));
        s.hi = __uint_as_float(hawk::ld_cluster_u32(at + 12));
        s.n = static_cast<int>(hawk::ld_cluster_u32(at + 16));
        s.flag = static_cast<int>(hawk::ld_cluster_u32(at + 20));
        return s;
    }
    __device__ __forceinline__ int load(long long row, int first, int n, float scale, float &lo, float &hi, int &finite);
    template <bool kMass>
    __device__ __forceinline__ float threshold(float lo, float hi, u64 count, double share);
};

// The block's n logits from id v_begin + first on into vals[pad ..]; returns pad, by which the 16-byte pieces of memory lie on 16-byte places of vals.
template <typename T, int NT>
__device__ __forceinline__ int Row<T, NT>::load(long long row, int first, int n, float scale, float &lo, float &hi, int &finite)
{
    constexpr int kN = Piece<T>::kN;
    const T *c = static_cast<const T *>(P.logits) + row * P.row_stride + P.v_begin + first;
    const bool has = P.uncond != nullptr;
    const T *u = has ? static_cast<const T *>(P.uncond) + row * P.uncond_stride + P.v_begin + first : c;
    const int pad = static_cast<int>((reinterpret_cast<uintptr_t>(c) & 15u) / sizeof(T));
    const bool alike = ((reinterpret_cast<uintptr_t>(c) ^ reinterpret_cast<uintptr_t>(u)) & 15u) == 0;  // pieces of both lie alike
    const int pieces = n > 0 ? (pad + n + kN - 1) / kN : 0;
    m = pieces * kN;
    hi = -CUDART_INF_F;
    lo = CUDART_INF_F;
    finite = 0;
    auto take = [&](int at, const float (&x)[kN]) {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            hi = fmaxf(hi, x[i]);
            if (x[i] > -CUDART_INF_F) {
                lo = fminf(lo, x[i]);
                ++finite;
            }
        }
#pragma unroll
        for (int i = 0; i < kN; i += 4) *reinterpret_cast<float4 *>(vals + at + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
    };
    constexpr int kFlight = 4;
    for (int q0 = threadIdx.x; q0 < pieces; q0 += NT * kFlight) {
        Piece<T> pc[kFlight], pu[kFlight];
        bool whole[kFlight];
#pragma unroll
        for (int k = 0; k < kFlight; ++k) {
            const int q = q0 + k * NT, e = q * kN - pad;
            whole[k] = alike && e >= 0 && e + kN <= n;
            if (whole[k]) {
                pc[k].raw = __ldcs(reinterpret_cast<const uint4 *>(c + e));
                pu[k].raw = has ? __ldcs(reinterpret_cast<const uint4 *>(u + e)) : pc[k].raw;
            }
        }
#pragma unroll
        for (int k = 0; k < kFlight; ++k) {
            const int q = q0 + k * NT, e = q * kN - pad;
            if (q >= pieces) break;
            float x[kN];
            if (whole[k]) {
#pragma unroll
                for (int i = 0; i < kN; ++i) x[i] = guided(pc[k].at(i), pu[k].at(i), has, scale, flags);
            } else {
#pragma unroll
                for (int i = 0; i < kN; ++i)
                    x[i] = e + i >= 0 && e + i < n ? guided(to_f32(c[e + i]), to_f32(u[e + i]), has, scale, flags) : -CUDART_INF_F;
            }
            take(q * kN, x);
        }
    }
    return pad;
}

// The largest value t in [lo, hi] for which the ids of logits t .. hi reach the target: `count` of them, or `share` of the mass of all in
// [lo, hi].  All reach it.  The same in all blocks of the row.
template <typename T, int NT>
template <bool kMass>
__device__ __forceinline__ float Row<T, NT>::threshold(float lo, float hi, u64 count, double share)
{
    const int tid = threadIdx.x;
    u64 above = 0, target = count;
    bool first = true;
    while (lo < hi) {
        const Steps step(lo, hi);
        __syncthreads();  // (everybody has read what the round before, or the search before, left in sh)
        for (int i = tid; i < kBins; i += NT) sh.hist[i] = 0;
        if (tid == 0) {
            sh.count = 0;
            sh.lo_key = 0xffffffffu;
            sh.hi_key = 0;
            sh.tau_key = 0;
            sh.bin = kBins - 1;
        }
        __syncthreads();
        for (int j = tid; j < m; j += NT) {
            const float l = vals[j];
            if (l >= lo && l <= hi) {
                if (kMass) atomicAdd(&sh.hist[step(l)], weight(l));
                else atomicAdd(reinterpret_cast<uint32_t *>(&sh.hist[step(l)]), 1u);  // (the low half: counts stay below 2^18)
            }
        }
        if (shared()) meet();
        else __syncthreads();
        constexpr int kPer = kBins / NT;
        u64 part[kPer], sum = 0, total;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            part[i] = 0;
            if (shared()) {
                for (int r = 0; r < P.cluster; ++r)
                    part[i] += hawk::ld_cluster_u64(hawk::map_shared_to_cta(&sh.hist[tid * kPer + i], r));
            } else {
                part[i] = sh.hist[tid * kPer + i];
            }
            sum += part[i];
        }
        u64 run = above + block_exclusive<NT>(sum, sh.warp, total);
        if (kMass && first) {
            const double want = ceil(share * static_cast<double>(total));
            target = want < 1.0 ? 1 : min(static_cast<u64>(want), total);
        }
        first = false;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (run < target && run + part[i] >= target) {
                sh.bin = tid * kPer + i;
                sh.above = run;
            }
            run += part[i];
        }
        __syncthreads();
        const int bin = sh.bin;
        above = sh.above;
        // the step's members
        for (int j = tid; j < m; j += NT) {
            const float l = vals[j];
            if (l >= lo && l <= hi && step(l) == bin) {
                const int at = atomicAdd(&sh.count, 1);
                if (at < kList) {
                    sh.list_v[at] = l;
                    sh.list_w[at] = kMass ? weight(l) : 1;
                }
                atomicMin(&sh.lo_key, key_of(l));
                atomicMax(&sh.hi_key, key_of(l));
            }
        }
        __syncthreads();
        int members = sh.count;
        const float *v = sh.list_v;
        const u64 *w = sh.list_w;
        float low = value_of(sh.lo_key), high = value_of(sh.hi_key);
        if (shared()) {
            if (tid == 0) sh.swap[1] = {0, members > 0 ? low : CUDART_INF_F, members > 0 ? high : -CUDART_INF_F, members, 0};
            meet();
            int before[kMaxCluster + 1];
            before[0] = 0;
            low = CUDART_INF_F;
            high = -CUDART_INF_F;
#pragma unroll
            for (int r = 0; r < kMaxCluster; ++r) {
                before[r + 1] = before[r];
                if (r < P.cluster) {
                    const Swap s = of(1, r);
                    before[r + 1] += s.n;
                    low = fminf(low, s.lo);
                    high = fmaxf(high, s.hi);
                }
            }
            members = before[kMaxCluster];
            if (members <= kList) {
#pragma unroll
                for (int r = 0; r < kMaxCluster; ++r)
                    for (int i = tid; i < before[r + 1] - before[r]; i += NT) {
                        sh.all_v[before[r] + i] = __uint_as_float(hawk::ld_cluster_u32(hawk::map_shared_to_cta(&sh.list_v[i], r)));
                        sh.all_w[before[r] + i] = hawk::ld_cluster_u64(hawk::map_shared_to_cta(&sh.list_w[i], r));
                    }
                __syncthreads();
                v = sh.all_v;
                w = sh.all_w;
            }
        }
        if (members <= kList) {
            for (int i = tid; i < members; i += NT) {
                const float mine = v[i];
                u64 reach = above;
                for (int k = 0; k < members; ++k)
                    if (v[k] >= mine) reach += w[k];
                if (reach >= target) atomicMax(&sh.tau_key, key_of(mine));
            }
            __syncthreads();
            return value_of(sh.tau_key);
        }
        lo = low;
        hi = high;
    }
    return hi;
}

template <typename T, int NT>
__device__ __forceinline__ void Row<T, NT>::run()
{
    constexpr int NW = NT / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    rank = shared() ? static_cast<int>(hawk::cluster_cta_rank()) : 0;
    const long long row = blockIdx.x / P.cluster;
    const int first = rank * P.slice, n = max(0, min(P.slice, P.n - first));

    // ---- settings
    float temperature = P.temperatures ? P.temperatures[row] : P.temperature;
    float top_p = P.top_ps ? P.top_ps[row] : P.top_p, min_p = P.min_ps ? P.min_ps[row] : P.min_p;
    const int top_k = P.top_ks ? P.top_ks[row] : P.top_k;
    const float scale = P.scales ? P.scales[row] : P.scale;
    float u = P.u[row];
    if (!(temperature >= 0.f && temperature < CUDART_INF_F)) {
        flags |= HAWK_DEV_BAD_SETTING;
        temperature = 1.f;
    }
    if (isnan(top_p)) {
        flags |= HAWK_DEV_BAD_SETTING;
        top_p = 1.f;
    }
    if (isnan(min_p)) {
        flags |= HAWK_DEV_BAD_SETTING;
        min_p = 0.f;
    }
    u = u > 0.f ? fminf(u, 1.f - 1.f / 16777216.f) : 0.f;
    const bool greedy = temperature == 0.f;
    inv_t = greedy ? 0.0 : 1.0 / static_cast<double>(temperature);

    // ---- the row, its largest and smallest logit
    float lo, hi;
    int finite;  // logits that are numbers
    const int pad = load(row, first, n, scale, lo, hi, finite);
    hi = hawk::warp_max(hi);
    lo = -hawk::warp_max(-lo);
    finite = __reduce_add_sync(0xffffffffu, finite);
    if (lane == 0) {
        sh.warp_n[warp] = finite;
        sh.warp_hi[warp] = hi;
        sh.warp_lo[warp] = lo;
    }
    if (tid == 0) sh.pick = INT_MAX;
    __syncthreads();
    hi = hawk::warp_max(lane < NW ? sh.warp_hi[lane] : -CUDART_INF_F);
    lo = -hawk::warp_max(lane < NW ? -sh.warp_lo[lane] : -CUDART_INF_F);
    finite = __reduce_add_sync(0xffffffffu, lane < NW ? sh.warp_n[lane] : 0);
    if (shared()) {
        if (tid == 0) sh.swap[0] = {0, lo, hi, finite, 0};
        meet();
        finite = 0;
        for (int r = 0; r < P.cluster; ++r) {
            const Swap s = of(0, r);
            finite += s.n;
            lo = fminf(lo, s.lo);
            hi = fmaxf(hi, s.hi);
        }
    }
    mx = hi;
    const bool some = mx > -CUDART_INF_F;

    // ---- thresholds
    float tau = lo;
    if (some && !greedy) {
        if (top_k > 0 && top_k < finite) tau = threshold<false>(lo, mx, static_cast<u64>(top_k), 0.0);
        if (top_p < 1.f) {
            // below max - 32 T a weight is 0 and has no say
            const float floor_w = static_cast<float>(static_cast<double>(mx) - 32.0 * static_cast<double>(temperature));
            tau = threshold<true>(fmaxf(tau, fminf(floor_w, mx)), mx, 0, static_cast<double>(top_p));
        }
        if (min_p >= 1.f) {
            tau = mx;
        } else if (min_p > 0.f) {  // the smallest value with (l - max) / T >= log(min_p)
            const double least = log(static_cast<double>(min_p));
            float t = static_cast<float>(static_cast<double>(mx) + static_cast<double>(temperature) * least);
            auto stays = [&](float x) { return (static_cast<double>(x) - static_cast<double>(mx)) * inv_t >= least; };
            if (t > -CUDART_INF_F) {
                for (int i = 0; i < 4 && !stays(t); ++i) t = nextafterf(t, CUDART_INF_F);
                for (int i = 0; i < 4 && stays(nextafterf(t, -CUDART_INF_F)); ++i) t = nextafterf(t, -CUDART_INF_F);
                tau = fmaxf(tau, fminf(t, mx));
            }
        }
    }

    // ---- the draw
    int32_t token = -1;   // (in the block that finds it)
    double inv_total = 0.0;
    int pick = INT_MAX;   // greedy: the id, in all blocks
    if (some && greedy) {
        int at = INT_MAX;
        for (int j = tid; j < m; j += NT)
            if (vals[j] == mx) at = min(at, first + j - pad);
        at = __reduce_min_sync(0xffffffffu, at);
        if (lane == 0 && at < INT_MAX) atomicMin(&sh.pick, at);
        __syncthreads();
        pick = sh.pick;
        if (shared()) {
            if (tid == 0) sh.swap[2] = {0, 0.f, 0.f, pick, 0};
            meet();
            for (int r = 0; r < P.cluster; ++r) pick = min(pick, of(2, r).n);
        }
        if (rank == 0 && tid == 0) {
            P.token[row] = P.v_begin + pick;
            if (P.token_prob) P.token_prob[row] = 1.f;
        }
    } else if (some) {
        // sums of the warps' stretches of ids, in whole runs of 32
        const int stretch = ((m + NW - 1) / NW + 31) & ~31;
        u64 sum = 0;
        const int end = min(m, (warp + 1) * stretch);
        for (int j = warp * stretch + lane; j < end; j += 32) {
            const float l = vals[j];
            if (l >= tau && l > -CUDART_INF_F) sum += weight(l);
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        __syncthreads();
        if (lane == 0) sh.warp[warp] = sum;
        __syncthreads();
        const u64 sums = warp_inclusive(lane < NW ? sh.warp[lane] : 0);  // every warp for itself
        const u64 mine = __shfl_sync(0xffffffffu, sums, 31);
        u64 total = mine, before = 0;
        if (shared()) {
            if (tid == 0) sh.swap[2] = {mine, 0.f, 0.f, 0, 0};
            meet();
            total = 0;
            for (int r = 0; r < P.cluster; ++r) {
                const u64 a = of(2, r).a;
                if (r < rank) before += a;
                total += a;
            }
        }
        inv_total = kOne / static_cast<double>(total);
        const u64 t = static_cast<u64>(static_cast<double>(u) * static_cast<double>(total));  // the running sum that has to be exceeded
        if (t >= before && t - before < mine) {  // here (all threads of one block)
            const unsigned past = __ballot_sync(0xffffffffu, before + sums > t);
            const int at = __ffs(past) - 1;      // the stretch, by its warp
            const u64 low = before + (at > 0 ? __shfl_sync(0xffffffffu, sums, at > 0 ? at - 1 : 0) : 0);
            const int j0 = at * stretch, j1 = min(m, j0 + stretch);
            const int per = (j1 - j0 + NT - 1) / NT;  // consecutive ids a thread
            const int a = min(j1, j0 + tid * per), b = min(j1, a + per);
            u64 part = 0, dummy;
            for (int j = a; j < b; ++j) {
                const float l = vals[j];
                if (l >= tau && l > -CUDART_INF_F) part += weight(l);
            }
            u64 run = low + block_exclusive<NT>(part, sh.warp, dummy);
            if (run <= t && run + part > t) {
                for (int j = a; j < b; ++j) {
                    const float l = vals[j];
                    if (l >= tau && l > -CUDART_INF_F) run += weight(l);
                    if (run > t) {
                        token = P.v_begin + first + j - pad;
                        P.token[row] = token;
                        if (P.token_prob) P.token_prob[row] = static_cast<float>(power(l) * inv_total);
                        break;
                    }
                }
            }
        }
    } else if (rank == 0 && tid == 0) {
        P.token[row] = -1;
        if (P.token_prob) P.token_prob[row] = 0.f;
    }

    // ---- the distribution
    if (P.probs) {
        float *out = P.probs + row * P.probs_stride;
        for (int j = tid; j < m; j += NT) {
            const int e = first + j - pad;
            if (j < pad || j - pad >= n) continue;
            const float l = vals[j];
            float p = 0.f;
            if (greedy) p = e == pick ? 1.f : 0.f;
            else if (some && l >= tau && l > -CUDART_INF_F) p = static_cast<float>(power(l) * inv_total);
            if (HAWK_IN_BOUNDS(P.dev_status, P.v_begin + e, P.V)) out[P.v_begin + e] = p;
        }
        for (int v = rank * NT + tid; v < P.v_begin; v += P.cluster * NT) out[v] = 0.f;
        for (int v = P.v_begin + P.n + rank * NT + tid; v < P.V; v += P.cluster * NT) out[v] = 0.f;
    }
    if (flags && P.dev_status) atomicOr(P.dev_status, flags);
    if (shared()) meet();  // nobody leaves while its shared memory is read
}

template <typename T, int NT>
__global__ void __launch_bounds__(NT, 1) sample_kernel(const __grid_constant__ SampleParams P)
{
    extern __shared__ __align__(16) unsigned char smem_raw[];
    hawk::allow_dependent_launch();
    hawk::grid_dependency_wait();
    Row<T, NT> row(P, *reinterpret_cast<SampleShared *>(smem_raw), reinterpret_cast<float *>(smem_raw + sizeof(SampleShared)));
    row.run();
}

template <typename T, int NT>
hawk_status launch(const SampleParams &P, int R, cudaStream_t st)
{
    static unsigned long long seen = 0;  // devices on which the kernel may use the shared memory of its largest slice
    constexpr size_t most = sizeof(SampleShared) + sizeof(float) * (kMaxSlice + 16);
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return HAWK_ERR_CUDA;
    const unsigned long long bit = 1ull << (dev & 63);
    if (!(__atomic_load_n(&seen, __ATOMIC_ACQUIRE) & bit) || dev >= 64) {
        if (cudaFuncSetAttribute(sample_kernel<T, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(most)) != cudaSuccess)
            return HAWK_ERR_CUDA;
        __atomic_fetch_or(&seen, bit, __ATOMIC_RELEASE);
    }
    const size_t smem = sizeof(SampleShared) + sizeof(float) * (static_cast<size_t>(P.slice) + 16);
    const dim3 grid(static_cast<unsigned>(R) * P.cluster);
    const cudaError_t e = P.cluster > 1
                              ? hawk_host::launch_dependent_clusters(sample_kernel<T, NT>, P.cluster, grid, dim3(NT), smem, st, P)
                              : hawk_host::launch_dependent(sample_kernel<T, NT>, grid, dim3(NT), smem, st, P);
    return e == cudaSuccess ? HAWK_OK : HAWK_ERR_CUDA;
}

bool finite(float v) { return v - v == 0.f; }

}  // namespace

extern "C" hawk_status hawk_sample(const hawk_sample_args *a, int32_t *dev_status, hawk_stream_t stream)
{
    const hawk_host::NvtxRange nvtx_range("hawk_sample");
    if (!a) return HAWK_ERR_NULL;
    if (a->R < 0 || a->V < 0 || a->v_begin < 0 || a->v_end > a->V || a->v_begin > a->v_end) return HAWK_ERR_SHAPE;
    if (a->R == 0) return HAWK_OK;
    if (a->dtype != HAWK_F32 && a->dtype != HAWK_BF16 && a->dtype != HAWK_F16) return HAWK_ERR_PARAM;
    if (!a->row_temperature && !(finite(a->temperature) && a->temperature >= 0.f)) return HAWK_ERR_PARAM;
    if ((!a->row_top_p && a->top_p != a->top_p) || (!a->row_min_p && a->min_p != a->min_p)) return HAWK_ERR_PARAM;
    if (a->uncond && !a->row_cfg_scale && !finite(a->cfg_scale)) return HAWK_ERR_PARAM;
    if (!a->logits || !a->u || !a->token) return HAWK_ERR_NULL;
    const int n = a->v_end - a->v_begin;
    if (n < 1 || n > kMaxSlice * kMaxCluster) return HAWK_ERR_UNSUPPORTED;
    if (a->row_stride < 0 || (a->uncond && a->uncond_row_stride < 0) || (a->R > 1 && a->probs && a->probs_row_stride < a->V))
        return HAWK_ERR_SHAPE;
    const uintptr_t size = a->dtype == HAWK_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(a->logits) % size || reinterpret_cast<uintptr_t>(a->uncond) % size ||
        reinterpret_cast<uintptr_t>(a->probs) % 4)
        return HAWK_ERR_ALIGN;
    if (static_cast<long long>(a->R) * kMaxCluster >= (1ll << 31)) return HAWK_ERR_UNSUPPORTED;
    if (!hawk_host::is_sm100(nullptr)) return HAWK_ERR_UNSUPPORTED;
    SampleParams P = {};
    P.logits = a->logits;
    P.uncond = a->uncond;
    P.row_stride = a->row_stride;
    P.uncond_stride = a->uncond_row_stride;
    P.probs_stride = a->probs_row_stride;
    P.temperatures = a->row_temperature;
    P.top_ps = a->row_top_p;
    P.min_ps = a->row_min_p;
    P.scales = a->row_cfg_scale;
    P.top_ks = a->row_top_k;
    P.u = a->u;
    P.temperature = a->temperature;
    P.top_p = a->top_p;
    P.min_p = a->min_p;
    P.scale = a->cfg_scale;
    P.top_k = a->top_k;
    P.V = a->V;
    P.v_begin = a->v_begin;
    P.n = n;
    P.token = a->token;
    P.token_prob = a->token_prob;
    P.probs = a->probs;
    P.dev_status = dev_status;
    P.cluster = 1;
    while ((n + P.cluster - 1) / P.cluster > kMaxSlice) P.cluster *= 2;
    P.slice = ((n + P.cluster - 1) / P.cluster + 15) & ~15;  // (every block's rows then lie alike in 16-byte pieces)
    const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    auto pick = [&](auto type) {
        using T = decltype(type);
        return launch<T, 1024>(P, a->R, st);
    };
    return a->dtype == HAWK_F32 ? pick(float{}) : a->dtype == HAWK_BF16 ? pick(__nv_bfloat16{}) : pick(__half{});
}
