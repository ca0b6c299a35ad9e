// hawk_sample: one token from every row of logits by a given random number (Sec. 5's settings of generation, with top-p and min-p).
//
// All three filters keep the ids whose logit is at least a threshold, so a row needs no sorted copy: it needs three numbers.  A threshold is
// the largest value at which the ids from it up reach a target, their number for top-k, their mass for top-p.  A block holds its row
// in shared memory and goes through it as few times as it can, because a row of 16384 ids costs some 128 cycles of an SM for every
// instruction that each id takes, and some 250 for every barrier:
//   1. the row comes in, with its maximum;
//   2. a sample of 4 ids a thread says between which two values the threshold lies (for top-p beside the row's mass in fp32, which a sample
//      would miss when few ids have most of it);
//   3. one pass over the weights: their sum above those values and below, for each warp, and a list of the ids between them;
//   4. a histogram of the list finds the step that the threshold is in, and the step's members against each other the value;
//   5. the sums of what stays tell the warp that the draw falls on, which finds the id.
// With top-k and top-p, 2 to 4 run for each.  Where the list does not hold the threshold (the sample misled, or too many are equal), step 4
// is done on the whole row, as many times as it takes (search()).  Neither changes a result.
// Masses are exponentials in fp64, held as multiples of 2^-44 in 64-bit integers: sums of them are exact, so no order of atomics or warps has a
// say and a token does not depend on the launch.  fp32 sums would not do: with 16 thousand ids one draw in some hundred falls so near to a
// border that their rounding decides it.
//
// A block holds 32768 ids at most; longer rows, and rows of calls with few of them, are shared by a cluster, whose blocks exchange
// histograms, members and sums through distributed shared memory.
#include <climits>

#include <math_constants.h>

#include "hawk_common.cuh"

namespace {

using u64 = unsigned long long;

constexpr int kBins = 256;       // steps of a histogram: 8 a lane, so that each warp sums them up for itself
constexpr int kFinal = 256;      // members of a step that are ranked against each other
constexpr int kList = 2048;      // ids that are looked at one by one, an equal share for each warp
constexpr int kTooMany = 1 << 20;
constexpr float kLowest = -3.402823466e38f;  // the lowest number: what is below is none
constexpr int kMaxSlice = 32768; // ids of a row that a block holds
constexpr int kMaxCluster = 8;
constexpr int kOneBits = 44;                // the largest logit's weight is 2^44; 2^18 such weights fit 64 bits
constexpr double kOne = 17592186044416.0;
constexpr int kPartBits = 7, kParts = 1 << kPartBits;  // of an octave, in the table of the exponential

struct SampleParams {
    const void *logits, *uncond;
    long long row_stride, uncond_stride, probs_stride;
    const float *temperatures, *top_ps, *min_ps, *scales, *u;
    const int32_t *top_ks;
    float temperature, top_p, min_p, scale;
    double rate, least;  // of temperature and min_p
    int top_k, V, v_begin, n, slice, cluster;  // n: ids of the range; slice: of a block
    int32_t *token;
    float *token_prob, *probs;
    int32_t *dev_status;
};

struct Swap {  // what the blocks of a row tell each other
    u64 a, b, c;
    float lo, hi;
    int n;
};

// Where a histogram keeps a step: lane i's eight steps, i * 8 and on, lie 32 places apart (side by side they would share a bank with others').
__device__ __forceinline__ int place_of(int bin) { return (bin & 7) * 32 + (bin >> 3); }

struct SampleShared {
    double table[kParts];  // 2^(i / kParts)
    uint32_t hist[3][kBins];  // number of a step, or its mass in parts of 15 bits (of weights, whose 2^15 add up to less than 2^32)
    uint32_t sample[kBins];
    float list_v[kList];   // the warps' shares one after the other
    u64 list_w[kList];
    u64 last_w[kFinal], all_w[kFinal];  // members of the last step: the block's, the row's
    float last_v[kFinal], all_v[kFinal];
    u64 warp_a[32], warp_b[32], warp_c[32];
    uint32_t warp_lo[32], warp_hi[32];
    float warp_f[32];
    Swap swap[6];  // one for each kind of exchange, so that a barrier lies between two uses of the same
    double rate, least;
    int last, over, pick;
    uint32_t tau_key;
};

// Barrier of the row's blocks (lanes that a branch parted come together first).
__device__ __forceinline__ void meet()
{
    __syncwarp();
    hawk::cluster_sync_all();
}

// kParts / (temperature * ln 2), and what (l - max) / temperature has to reach for min-p.
__host__ __device__ inline double rate_of(float temperature) { return kParts * 1.44269504088896340736 / static_cast<double>(temperature); }

__host__ __device__ inline double least_of(float min_p) { return min_p > 0.f && min_p < 1.f ? log(static_cast<double>(min_p)) : 0.0; }

// Unsigned number in the order of the values.
__device__ __forceinline__ uint32_t key_of(float v)
{
    const uint32_t b = __float_as_uint(v);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

// Least whole number that is `share` of `total`, and 1 at least.
__device__ __forceinline__ u64 target_of(double share, u64 total)
{
    const double want = ceil(share * static_cast<double>(total));
    return want < 1.0 ? 1 : min(static_cast<u64>(want), total);
}

// Sum over the warp's lanes, of which none has more than 2^60, by whole-warp additions of 22 bits at a time.
__device__ __forceinline__ u64 warp_sum(u64 v)
{
    constexpr uint32_t kLow = (1u << 22) - 1;
    const u64 a = __reduce_add_sync(0xffffffffu, static_cast<uint32_t>(v) & kLow);
    const u64 b = __reduce_add_sync(0xffffffffu, static_cast<uint32_t>(v >> 22) & kLow);
    const u64 c = __reduce_add_sync(0xffffffffu, static_cast<uint32_t>(v >> 44));
    return a + (b << 22) + (c << 44);
}

template <typename N>
__device__ __forceinline__ N warp_inclusive(N v)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const N x = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += x;
    }
    return v;
}

// Steps of equal width from hi down to lo: monotone in the value, 0 for hi, the last for lo and what is below.  Ranges that fp32 cannot divide (next to
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
        if (per > 0.f) return static_cast<int>(fminf((hi - v) * per, kBins - 1.f));
        return static_cast<int>(fmin((static_cast<double>(hi) - static_cast<double>(v)) * wide, kBins - 1.0));
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
        if (!(fmaxf(fabsf(c), fabsf(u)) < CUDART_INF_F) || isnan(c) || isnan(u)) {  // whatever the scale
            l = -CUDART_INF_F;
            if (!(c < CUDART_INF_F) || !(u < CUDART_INF_F)) flags |= HAWK_DEV_NONFINITE;
        }
    }
    if (!(l < CUDART_INF_F)) {  // NaN, +inf
        flags |= HAWK_DEV_NONFINITE;
        l = -CUDART_INF_F;
    }
    return l;
}

template <typename T, int NT>
class Row {
public:
    __device__ __forceinline__ Row(const SampleParams &p, SampleShared &s, float *v) : P(p), sh(s), vals(v) {}
    __device__ __forceinline__ void prepare();
    __device__ __forceinline__ void run();

private:
    static constexpr int NW = NT / 32, kShare = kList / NW;
    const SampleParams &P;
    SampleShared &sh;
    float *vals;  // [m] logits of the block's ids, -inf around them; m is a multiple of 4
    int m, rank, flags = 0;
    int base, end;      // the warp's stretch of ids
    int listed;         // the warp's, in its share of the list; more than fit: kShare + 1
    float mx, nothing;  // the largest; from `nothing`, 32 temperatures below it, down a weight is 0
    double rate;        // kParts / (temperature * ln 2)

    struct Window {  // values that the threshold should lie between; the sums of a pass: from hi up and below lo (without the list)
        float lo, hi;
        u64 above, below, between;  // mass; `between`: the list's
        int count, members;         // from hi up, in the list
    };

    __device__ __forceinline__ bool shared() const { return P.cluster > 1; }
    __device__ __forceinline__ void barrier() const
    {
        if (shared()) meet();
        else __syncthreads();
    }

    // exp((l - max) / temperature) = w * 2^e = 2^(t / kParts), l >= nothing: the whole part of t by exponent and table, the rest by the
    // Taylor polynomial of degree 3 (table-driven exponentials: P. T. P. Tang, 1989).  Its remainder is (ln 2 / 256)^4 / 24 =
    // 2.2e-12 at most.
    __device__ __forceinline__ double power(float l, int &e) const
    {
        constexpr double kMagic = 6755399441055744.0;  // 1.5 * 2^52: the sum's low bits are the nearest whole number
        constexpr double kLn2 = 0.693147180559945309417;
        constexpr double c1 = kLn2 / kParts, c2 = c1 * c1 / 2, c3 = c1 * c1 * c1 / 6;
        const double t = (static_cast<double>(l) - static_cast<double>(mx)) * rate;
        const double k = t + kMagic;
        const double r = t - (k - kMagic);
        const int n = __double2loint(k);
        const double f = sh.table[n & (kParts - 1)];
        e = n >> kPartBits;
        return fma(f, r * fma(r, fma(r, c3, c2), c1), f);
    }
    // ... in whole multiples of 2^-44.  (At `nothing` and below, -inf too, that is 0: e^-32 of them.)
    __device__ __forceinline__ u64 weight(float l) const
    {
        int e;
        const double w = power(fmaxf(l, nothing), e);
        constexpr double kWhole = 4503599627370496.0;  // 2^52: the sum's low bits are the nearest whole number
        const double whole = __hiloint2double(__double2hiint(w) + (e + kOneBits) * (1 << 20), __double2loint(w)) + kWhole;
        return static_cast<u64>(__double_as_longlong(whole)) & ((1ull << 52) - 1);
    }
    // ... as a number, times `factor`
    __device__ __forceinline__ float share(float l, double factor) const
    {
        int e;
        const double w = power(l, e);
        return static_cast<float>(__hiloint2double(__double2hiint(w) + e * (1 << 20), __double2loint(w)) * factor);
    }
    __device__ __forceinline__ Swap of(int slot, int r) const
    {
        const uint32_t at = hawk::map_shared_to_cta(&sh.swap[slot], r);
        Swap s;
        s.a = hawk::ld_cluster_u64(at);
        s.b = hawk::ld_cluster_u64(at + 8);
        s.c = hawk::ld_cluster_u64(at + 16);
        s.lo = __uint_as_float(hawk::ld_cluster_u32(at + 24));
        s.hi = __uint_as_float(hawk::ld_cluster_u32(at + 28));
        s.n = static_cast<int>(hawk::ld_cluster_u32(at + 32));
        return s;
    }
    // Lane's four logits of the warp's run from place j on (-inf behind its stretch).
    __device__ __forceinline__ void four(int j, float (&l)[4]) const
    {
        const int at = j + 4 * static_cast<int>(threadIdx.x & 31);
        const float4 x = at < end ? *reinterpret_cast<const float4 *>(vals + at)
                                  : make_float4(-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F);
        l[0] = x.x;
        l[1] = x.y;
        l[2] = x.z;
        l[3] = x.w;
    }
    __device__ __forceinline__ int load(long long row, int first, int n, float scale, float &lo, float &hi);
    __device__ __forceinline__ void ends(float &lo, float &hi, int slot);
    __device__ __forceinline__ float mass_of_row();
    __device__ __forceinline__ void sample(const Steps &step);
    __device__ __forceinline__ Window between_ranks(const Steps &step, float bottom, float above, float margin);
    __device__ __forceinline__ Window between_masses(const Steps &step, float bottom, float from, float below, float margin);
    template <bool kBelow>
    __device__ __forceinline__ void pass(Window &w, float from);
    template <bool kMass, bool kFromList>
    __device__ __forceinline__ bool search(float lo, float hi, float bottom, u64 target, float &tau);
};

// What does not depend on the call's inputs: done before the kernel ahead has ended.
template <typename T, int NT>
__device__ __forceinline__ void Row<T, NT>::prepare()
{
    for (int i = threadIdx.x; i < kParts; i += NT) sh.table[i] = exp2(static_cast<double>(i) / kParts);
    for (int i = threadIdx.x; i < kBins; i += NT) sh.sample[i] = 0;
}

// The block's n logits from id v_begin + first on into vals[pad ..]; returns pad, by which the 16-byte pieces of memory lie on 16-byte places of vals.  hi: the
// largest; lo: the smallest number among the pieces' first ones.
template <typename T, int NT>
__device__ __forceinline__ int Row<T, NT>::load(long long row, int first, int n, float scale, float &lo, float &hi)
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
    auto take = [&](int at, const float (&x)[kN]) {
#pragma unroll
        for (int i = 0; i < kN; ++i) hi = fmaxf(hi, x[i]);
        if (x[0] >= kLowest) lo = fminf(lo, x[0]);
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

// Smallest lo and largest hi of the row's threads.
template <typename T, int NT>
__device__ __forceinline__ void Row<T, NT>::ends(float &lo, float &hi, int slot)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t a = __reduce_min_sync(0xffffffffu, key_of(lo)), b = __reduce_max_sync(0xffffffffu, key_of(hi));
    if (lane == 0) {
        sh.warp_lo[warp] = a;
        sh.warp_hi[warp] = b;
    }
    __syncthreads();
    lo = value_of(__reduce_min_sync(0xffffffffu, lane < NW ? sh.warp_lo[lane] : 0xffffffffu));
    hi = value_of(__reduce_max_sync(0xffffffffu, lane < NW ? sh.warp_hi[lane] : 0u));
    if (shared()) {
        if (threadIdx.x == 0) {
            sh.swap[slot].lo = lo;
            sh.swap[slot].hi = hi;
        }
        meet();
        for (int r = 0; r < P.cluster; ++r) {
            const Swap s = of(slot, r);
            lo = fminf(lo, s.lo);
            hi = fmaxf(hi, s.hi);
        }
    }
}

// The warp's part of the row's mass in fp32, to warp_f.
template <typename T, int NT>
__device__ __forceinline__ float Row<T, NT>::mass_of_row()
{
    const float octaves = static_cast<float>(rate / kParts);
    float mass = 0.f;
    for (int j = base; j < end; j += 128) {
        float l[4];
        four(j, l);
        mass += (hawk::fast_exp2((l[0] - mx) * octaves) + hawk::fast_exp2((l[1] - mx) * octaves)) +
                (hawk::fast_exp2((l[2] - mx) * octaves) + hawk::fast_exp2((l[3] - mx) * octaves));
    }
    return hawk::warp_sum(mass);
}

// Four logits a thread, or all if there are no more, to the histogram of the sample.
template <typename T, int NT>
__device__ __forceinline__ void Row<T, NT>::sample(const Steps &step)
{
    const int per = (P.slice + NT - 1) / NT, at = per > 4 ? static_cast<int>(threadIdx.x) * per & ~3 : 4 * static_cast<int>(threadIdx.x);
    if (at < m) {
        const float4 l = *reinterpret_cast<const float4 *>(vals + at);
        if (l.x >= kLowest) atomicAdd(&sh.sample[place_of(step(l.x))], 1u);
        if (l.y >= kLowest) atomicAdd(&sh.sample[place_of(step(l.y))], 1u);
        if (l.z >= kLowest) atomicAdd(&sh.sample[place_of(step(l.z))], 1u);
        if (l.w >= kLowest) atomicAdd(&sh.sample[place_of(step(l.w))], 1u);
    }
    __syncwarp();
}

// Values between which the logit of rank `above` of the sample lies, by `margin` ranks on either side.  Every warp for itself (behind a barrier).
template <typename T, int NT>
__device__ __forceinline__ typename Row<T, NT>::Window Row<T, NT>::between_ranks(const Steps &step, float bottom, float above, float margin)
{
    constexpr int kPer = kBins / 32;
    const int lane = threadIdx.x & 31;
    uint32_t part[kPer], sum = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        part[i] = 0;
        if (shared()) {
            for (int r = 0; r < P.cluster; ++r) part[i] += hawk::ld_cluster_u32(hawk::map_shared_to_cta(&sh.sample[i * 32 + lane], r));
        } else {
            part[i] = sh.sample[i * 32 + lane];
        }
        sum += part[i];
    }
    uint32_t run = warp_inclusive(sum) - sum;
    const float low = above - margin, high = above + margin;  // (a low of 1 or less: even the largest may be it)
    int b1 = low <= 1.f ? 0 : kBins, b2 = kBins;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        run += part[i];
        if (run >= low) b1 = min(b1, lane * kPer + i);
        if (run >= high) b2 = min(b2, lane * kPer + i);
    }
    b1 = __reduce_min_sync(0xffffffffu, b1);
    b2 = __reduce_min_sync(0xffffffffu, b2);
    const float wide = (mx - bottom) / kBins;
    Window w;
    w.hi = b1 > 0 && b1 < kBins ? mx - wide * b1 : CUDART_INF_F;
    w.lo = b2 < kBins - 1 ? mx - wide * (b2 + 1) : kLowest;
    return w;
}

// Values between which the logits from `from` up to the threshold have the mass `below` together, as the sample has it, with a share `margin` of
// it on either side.  Every warp for itself (behind a barrier).
template <typename T, int NT>
__device__ __forceinline__ typename Row<T, NT>::Window Row<T, NT>::between_masses(const Steps &step, float bottom, float from, float below,
                                                                                 float margin)
{
    constexpr int kPer = kBins / 32;
    const int lane = threadIdx.x & 31, last = step(from);
    const float wide = (mx - bottom) / kBins, octaves = static_cast<float>(rate / kParts);
    const int per = (P.slice + NT - 1) / NT;
    const float each = per > 4 ? per * 0.25f : 1.f;
    float part[kPer], sum = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int b = lane * kPer + i;
        uint32_t count = 0;
        if (shared()) {
            for (int r = 0; r < P.cluster; ++r) count += hawk::ld_cluster_u32(hawk::map_shared_to_cta(&sh.sample[i * 32 + lane], r));
        } else {
            count = sh.sample[i * 32 + lane];
        }
        part[i] = b <= last && count > 0 ? each * count * hawk::fast_exp2(-wide * octaves * (b + 0.5f)) : 0.f;
        sum += part[i];
    }
    // (sums from the far end up: the near end's few large weights are what a sample knows least)
    float tail = 0.f;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const float x = __shfl_down_sync(0xffffffffu, sum, o);
        if (lane + o < 32) sum += x;
    }
    tail = __shfl_down_sync(0xffffffffu, sum, 1);
    if (lane == 31) tail = 0.f;
    int b1 = kBins, b2 = kBins;
#pragma unroll
    for (int i = kPer - 1; i >= 0; --i) {  // tail: what lies behind step lane * kPer + i
        if (tail <= below * (1.f + margin)) b1 = lane * kPer + i;
        if (tail <= below * (1.f - margin)) b2 = lane * kPer + i;
        tail += part[i];
    }
    b1 = __reduce_min_sync(0xffffffffu, b1);
    b2 = __reduce_min_sync(0xffffffffu, b2);
    Window w;
    w.hi = b1 > 0 && b1 < kBins ? mx - wide * b1 : CUDART_INF_F;
    w.lo = b2 < kBins - 1 ? mx - wide * (b2 + 1) : kLowest;
    return w;
}

// One pass over the weights of the logits from `from` on: the sums of the window, its members to the list; the warp's sum of what lies above it
// stays in warp_a.  Barriers of the row lie in it.
template <typename T, int NT>
template <bool kBelow>
__device__ __forceinline__ void Row<T, NT>::pass(Window &w, float from)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    u64 above = 0, below = 0, between = 0;
    u64 marks = 0;  // which of the lane's are members
    int count = 0, at = 0;
    for (int j = base; j < end; j += 128, at += 4) {
        float l[4];
        four(j, l);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const u64 x = weight(l[k]);
            const bool up = l[k] >= w.hi, low = l[k] < w.lo;
            if (up) above += x;
            if (up) ++count;
            if (kBelow) {
                if (low && l[k] >= from) below += x;
                if (!up && !low && l[k] >= from) marks |= 1ull << (at + k);
            } else {
                if (!up && !low) marks |= 1ull << (at + k);
            }
        }
    }
    const int mine = __popcll(marks), sum = warp_inclusive(mine);
    listed = __shfl_sync(0xffffffffu, sum, 31);
    for (int to = sum - mine; marks; marks &= marks - 1, ++to) {
        const int i = __ffsll(marks) - 1;
        const float l = vals[base + (i >> 2) * 128 + 4 * lane + (i & 3)];
        const u64 x = weight(l);
        between += x;
        if (to < kShare) {
            sh.list_v[warp * kShare + to] = l;
            sh.list_w[warp * kShare + to] = x;
        }
    }
    __syncwarp();
    above = warp_sum(above);
    between = warp_sum(between);
    if (kBelow) below = warp_sum(below);
    count = __reduce_add_sync(0xffffffffu, count);
    __syncthreads();  // (the sums of the pass before have been read)
    if (lane == 0) {
        sh.warp_a[warp] = above;
        sh.warp_b[warp] = below;
        sh.warp_c[warp] = between;
        sh.warp_lo[warp] = count;
        sh.warp_hi[warp] = listed > kShare ? kTooMany : listed;  // (a sum that says that some did not fit)
    }
    for (int i = threadIdx.x; i < 3 * kBins; i += NT) sh.hist[0][i] = 0;
    if (threadIdx.x == 0) {
        sh.last = 0;
        sh.tau_key = 0;
    }
    __syncthreads();
    w.above = warp_sum(lane < NW ? sh.warp_a[lane] : 0ull);
    w.below = kBelow ? warp_sum(lane < NW ? sh.warp_b[lane] : 0ull) : 0ull;
    w.between = warp_sum(lane < NW ? sh.warp_c[lane] : 0ull);
    w.count = __reduce_add_sync(0xffffffffu, lane < NW ? sh.warp_lo[lane] : 0u);
    w.members = __reduce_add_sync(0xffffffffu, lane < NW ? sh.warp_hi[lane] : 0u);
    if (shared()) {
        if (threadIdx.x == 0) sh.swap[1] = {w.above, w.below, w.between, __int_as_float(w.count), 0.f, w.members};
        meet();
        w.above = w.below = w.between = 0;
        w.count = w.members = 0;
        for (int r = 0; r < P.cluster; ++r) {
            const Swap s = of(1, r);
            w.above += s.a;
            w.below += s.b;
            w.between += s.c;
            w.count += __float_as_int(s.lo);
            w.members += s.n;
        }
    }
}

// The largest value tau in [lo, hi] for which the logits from it to hi reach the target, their number or their mass; among the list (whose sums
// have to reach it; false if its last step has too many members), or among the block's whole row (always found, in as many rounds as it
// takes: a round leaves one value out at least).  The first round's steps start from `bottom`, the last of them takes what is below.  The same in all blocks of the row.  hist, last and tau_key are clear for the list.
template <typename T, int NT>
template <bool kMass, bool kFromList>
__device__ __forceinline__ bool Row<T, NT>::search(float lo, float hi, float bottom, u64 target, float &tau)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int begin = kFromList ? warp * kShare : base, stop = kFromList ? begin + listed : end;
    const float *from = kFromList ? sh.list_v : vals;
    auto weigh = [&](int i, float l) -> u64 { return !kMass ? 1ull : kFromList ? sh.list_w[i] : weight(l); };
    u64 above = 0;
    while (lo < hi) {
        const Steps step(fmaxf(lo, bottom), hi);
        if (!kFromList) {
            barrier();  // (everybody has read what the round before, or the search before, left in sh)
            for (int i = tid; i < 3 * kBins; i += NT) sh.hist[0][i] = 0;
            if (tid == 0) {
                sh.last = 0;
                sh.tau_key = 0;
            }
            __syncthreads();
        }
        for (int i = begin + lane; i < stop; i += 32) {
            const float l = from[i];
            if (l >= lo && l <= hi) {
                const int at = place_of(step(l));
                const u64 x = weigh(i, l);
                if (!kMass) {
                    atomicAdd(&sh.hist[0][at], 1u);
                } else {
                    constexpr uint32_t kPart = (1u << 15) - 1;
                    atomicAdd(&sh.hist[0][at], static_cast<uint32_t>(x) & kPart);
                    atomicAdd(&sh.hist[1][at], static_cast<uint32_t>(x >> 15) & kPart);
                    atomicAdd(&sh.hist[2][at], static_cast<uint32_t>(x >> 30));
                }
            }
        }
        __syncwarp();
        barrier();
        // the step that the target is reached in: every warp for itself
        constexpr int kPer = kBins / 32;
        u64 part[kPer], sum = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            part[i] = 0;
#pragma unroll
            for (int k = 0; k < (kMass ? 3 : 1); ++k) {
                u64 x = 0;
                if (shared()) {
                    for (int r = 0; r < P.cluster; ++r) x += hawk::ld_cluster_u32(hawk::map_shared_to_cta(&sh.hist[k][i * 32 + lane], r));
                } else {
                    x = sh.hist[k][i * 32 + lane];
                }
                part[i] += x << (15 * k);
            }
            sum += part[i];
        }
        u64 run = above + warp_inclusive(sum) - sum, at_run = 0;
        int bin = kBins - 1;
        bool here = false;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (run < target && run + part[i] >= target) {
                bin = lane * kPer + i;
                at_run = run;
                here = true;
            }
            run += part[i];
        }
        const uint32_t who = __ballot_sync(0xffffffffu, here);
        if (who == 0) return false;  // (the same in all warps and blocks)
        bin = __shfl_sync(0xffffffffu, bin, __ffs(who) - 1);
        above = __shfl_sync(0xffffffffu, at_run, __ffs(who) - 1);
        // its members
        float low = CUDART_INF_F, high = -CUDART_INF_F;
        for (int i = begin + lane; i < stop; i += 32) {
            const float l = from[i];
            if (l >= lo && l <= hi && step(l) == bin) {
                const int at = atomicAdd(&sh.last, 1);
                if (at < kFinal) {
                    sh.last_v[at] = l;
                    sh.last_w[at] = weigh(i, l);
                }
                low = fminf(low, l);
                high = fmaxf(high, l);
            }
        }
        __syncthreads();
        int members = sh.last;
        const float *v = sh.last_v;
        const u64 *w = sh.last_w;
        if (shared()) {
            if (tid == 0) sh.swap[2].n = members;
            meet();
            int before[kMaxCluster + 1];
            before[0] = 0;
#pragma unroll
            for (int r = 0; r < kMaxCluster; ++r)
                before[r + 1] = before[r] + (r < P.cluster ? static_cast<int>(hawk::ld_cluster_u32(hawk::map_shared_to_cta(&sh.swap[2].n, r))) : 0);
            members = before[kMaxCluster];
            if (members <= kFinal) {
#pragma unroll
                for (int r = 0; r < kMaxCluster; ++r)
                    for (int i = tid; i < before[r + 1] - before[r]; i += NT) {
                        sh.all_v[before[r] + i] = __uint_as_float(hawk::ld_cluster_u32(hawk::map_shared_to_cta(&sh.last_v[i], r)));
                        sh.all_w[before[r] + i] = hawk::ld_cluster_u64(hawk::map_shared_to_cta(&sh.last_w[i], r));
                    }
                __syncthreads();
                v = sh.all_v;
                w = sh.all_w;
            }
        }
        if (members <= kFinal) {
            // against each other, 8 lanes a member
            for (int i0 = 0; i0 < members; i0 += NT / 8) {  // (the same rounds for all lanes)
                const int i = i0 + tid / 8;
                const float mine = i < members ? v[i] : CUDART_INF_F;
                u64 reach = 0;
                for (int k = tid & 7; k < members; k += 8)
                    if (v[k] >= mine) reach += w[k];
                reach += __shfl_xor_sync(0xffffffffu, reach, 1);
                reach += __shfl_xor_sync(0xffffffffu, reach, 2);
                reach += __shfl_xor_sync(0xffffffffu, reach, 4);
                if ((tid & 7) == 0 && i < members && above + reach >= target) atomicMax(&sh.tau_key, key_of(mine));
            }
            __syncthreads();
            tau = value_of(sh.tau_key);
            return true;
        }
        if (kFromList) return false;
        ends(low, high, 3);
        lo = low;
        hi = high;
        bottom = low;
    }
    tau = hi;
    return true;
}

template <typename T, int NT>
__device__ __forceinline__ void Row<T, NT>::run()
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    rank = shared() ? static_cast<int>(hawk::cluster_cta_rank()) : 0;
    const long long row = blockIdx.x / P.cluster;
    const int first = rank * P.slice, n = max(0, min(P.slice, P.n - first));

    // ---- the row, its settings, its largest logit
    float temperature = P.temperatures ? P.temperatures[row] : P.temperature;
    float top_p = P.top_ps ? P.top_ps[row] : P.top_p, min_p = P.min_ps ? P.min_ps[row] : P.min_p;
    const int top_k = P.top_ks ? P.top_ks[row] : P.top_k;
    const float scale = P.scales ? P.scales[row] : P.scale;
    float u = P.u[row], lo, hi;
    const int pad = load(row, first, n, scale, lo, hi);
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
    bool greedy = temperature == 0.f;
    if (tid == 0) {  // (a row's own settings: fp64 division and logarithm by one lane)
        sh.rate = !P.temperatures ? P.rate : greedy ? 0.0 : rate_of(temperature);
        sh.least = !P.min_ps ? P.least : least_of(min_p);
        sh.pick = INT_MAX;
    }
    ends(lo, hi, 0);
    mx = hi;
    rate = sh.rate;
    nothing = fmaxf(fminf(static_cast<float>(static_cast<double>(mx) - 32.0 * static_cast<double>(temperature)), mx), kLowest);
    const bool some = mx > -CUDART_INF_F;
    const int stretch = ((m + NW - 1) / NW + 127) & ~127;  // whole runs of 4 a lane
    base = min(m, warp * stretch);
    end = min(m, base + stretch);

    double inv_total = 0.0;
    int pick = INT_MAX;   // greedy: the id, in all blocks
    float tau = kLowest;  // what is kept at the end
    if (some && greedy) {
        int at = INT_MAX;
        for (int j = base + lane; j < end; j += 32)
            if (vals[j] == mx) at = min(at, first + j - pad);
        __syncwarp();
        at = __reduce_min_sync(0xffffffffu, at);
        if (lane == 0 && at < INT_MAX) atomicMin(&sh.pick, at);
        __syncthreads();
        pick = sh.pick;
        if (shared()) {
            if (tid == 0) sh.swap[4].n = pick;
            meet();
            for (int r = 0; r < P.cluster; ++r) pick = min(pick, of(4, r).n);
        }
        if (rank == 0 && tid == 0) {
            P.token[row] = P.v_begin + pick;
            if (P.token_prob) P.token_prob[row] = 1.f;
        }
    } else if (some) {
        // ---- min-p: the smallest value with (l - max) / T >= log(min_p)
        float tau_m = kLowest;
        if (min_p >= 1.f) {
            tau_m = mx;
        } else if (min_p > 0.f) {
            constexpr double kLn2Part = 0.693147180559945309417 / kParts;
            const double least = sh.least, per_t = rate * kLn2Part;
            float t = static_cast<float>(static_cast<double>(mx) + static_cast<double>(temperature) * least);
            auto stays = [&](float x) { return (static_cast<double>(x) - static_cast<double>(mx)) * per_t >= least; };
            if (t > -CUDART_INF_F) {
                for (int i = 0; i < 4 && !stays(t); ++i) t = nextafterf(t, CUDART_INF_F);
                for (int i = 0; i < 4 && stays(nextafterf(t, -CUDART_INF_F)); ++i) t = nextafterf(t, -CUDART_INF_F);
                tau_m = fmaxf(kLowest, fminf(t, mx));
            }
        }
        const bool flat = nothing >= mx;  // a temperature so low that nothing but the maximum has a weight
        if (flat) tau_m = mx;
        bool by_k = top_k > 0 && top_k < P.n && !flat;
        const bool by_p = top_p < 1.f && !flat;

        // ---- thresholds of top-k and top-p
        float tau_k = kLowest, tau_p = kLowest;
        Window w = {kLowest, kLowest, 0, 0, 0, 0, 0};
        bool summed = false;  // warp_a has the sums of what lies above w, the list what lies in it
        if (by_k || by_p) {
            const float bottom = by_k ? lo : fmaxf(lo, nothing);
            const Steps step(bottom, mx);
            const int per = (P.slice + NT - 1) / NT;
            const float each = per > 4 ? per * 0.25f : 1.f;  // logits that one of the sample stands for
            float mass = 0.f;
            if (!by_k) mass = mass_of_row();
            sample(step);
            if (lane == 0) sh.warp_f[warp] = mass;
            if (shared()) {
                __syncthreads();
                mass = hawk::warp_sum(lane < NW ? sh.warp_f[lane] : 0.f);
                if (tid == 0) sh.swap[5].lo = mass;
                meet();
                mass = 0.f;
                for (int r = 0; r < P.cluster; ++r) mass += of(5, r).lo;
            } else {
                __syncthreads();
                mass = hawk::warp_sum(lane < NW ? sh.warp_f[lane] : 0.f);
            }
            if (by_k) {
                const float s = top_k / each;
                w = between_ranks(step, bottom, s, each > 1.f ? 4.f * sqrtf(s) + 8.f : 1.f);
                pass<false>(w, kLowest);
                const long long want = static_cast<long long>(top_k) - w.count;
                summed = want > 0 && want <= w.members && w.members < kTooMany &&
                         search<false, true>(w.lo, fminf(w.hi, mx), bottom, static_cast<u64>(want), tau_k);
                if (!summed && !search<false, false>(kLowest, mx, bottom, static_cast<u64>(top_k), tau_k)) tau_k = kLowest;  // (fewer logits than top_k)
            }
            if (by_p && tau_k < mx) {
                if (by_k) {  // the mass of what top-k left
                    u64 mine = 0;
                    if (summed) {
                        mine = lane == 0 ? sh.warp_a[warp] : 0;
                        for (int i = lane; i < listed; i += 32)
                            if (sh.list_v[warp * kShare + i] >= tau_k) mine += sh.list_w[warp * kShare + i];
                    } else {
                        for (int j = base; j < end; j += 128) {
                            float l[4];
                            four(j, l);
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const u64 x = weight(l[k]);
                                mine += l[k] >= tau_k ? x : 0;
                            }
                        }
                    }
                    __syncwarp();
                    mine = warp_sum(mine);
                    if (lane == 0) sh.warp_c[warp] = mine;
                    __syncthreads();
                    mine = warp_sum(lane < NW ? sh.warp_c[lane] : 0ull);
                    if (shared()) {
                        if (tid == 0) sh.swap[4].a = mine;
                        meet();
                        mine = 0;
                        for (int r = 0; r < P.cluster; ++r) mine += of(4, r).a;
                    }
                    mass = static_cast<float>(static_cast<double>(mine) / kOne);
                }
                const float from = fmaxf(tau_k, nothing);
                w = between_masses(step, bottom, from, (1.f - top_p) * mass, each > 1.f ? 0.2f : 0.02f);
                pass<true>(w, from);
                const u64 target = target_of(top_p, w.above + w.between + w.below);
                summed = target > w.above && target <= w.above + w.between && w.members < kTooMany &&
                         search<true, true>(fmaxf(w.lo, from), fminf(w.hi, mx), bottom, target - w.above, tau_p);
                if (!summed) (void)search<true, false>(from, mx, bottom, target, tau_p);
            }
        }
        tau = fmaxf(fmaxf(tau_k, tau_p), tau_m);

        // ---- what stays, for each warp
        u64 kept = 0;
        if (summed && !(tau_m >= w.hi)) {
            for (int i = lane; i < listed; i += 32)
                if (sh.list_v[warp * kShare + i] >= tau) kept += sh.list_w[warp * kShare + i];
            if (lane == 0) kept += sh.warp_a[warp];
        } else {
            for (int j = base; j < end; j += 128) {
                float l[4];
                four(j, l);
                if (!__any_sync(0xffffffffu, fmaxf(fmaxf(l[0], l[1]), fmaxf(l[2], l[3])) >= tau)) continue;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const u64 x = weight(l[k]);
                    kept += l[k] >= tau ? x : 0;
                }
            }
        }
        __syncwarp();
        kept = warp_sum(kept);
        if (lane == 0) sh.warp_b[warp] = kept;
        __syncthreads();

        // ---- the draw
        const u64 sums = warp_inclusive(lane < NW ? sh.warp_b[lane] : 0ull);  // every warp for itself
        const u64 mine = __shfl_sync(0xffffffffu, sums, 31);
        u64 total = mine, before = 0;
        if (shared()) {
            if (tid == 0) sh.swap[3].a = mine;
            meet();
            total = 0;
            for (int r = 0; r < P.cluster; ++r) {
                const u64 a = of(3, r).a;
                if (r < rank) before += a;
                total += a;
            }
        }
        inv_total = kOne / static_cast<double>(total);
        const u64 t = static_cast<u64>(static_cast<double>(u) * static_cast<double>(total));  // the running sum that has to be exceeded
        if (t >= before && t - before < mine) {
            const int at = __ffs(__ballot_sync(0xffffffffu, before + sums > t)) - 1;  // the stretch it falls on
            const u64 low = __shfl_sync(0xffffffffu, sums, at > 0 ? at - 1 : 0);
            if (warp == at) {
                u64 run = before + (at > 0 ? low : 0);
                for (int j = base; j < end; j += 128) {
                    float l[4];
                    four(j, l);
                    u64 x[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const u64 y = weight(l[k]);
                        x[k] = l[k] >= tau ? y : 0;
                    }
                    const u64 sum = (x[0] + x[1]) + (x[2] + x[3]);
                    const u64 inc = run + warp_inclusive(sum);
                    const uint32_t past = __ballot_sync(0xffffffffu, inc > t);
                    if (past) {
                        if (lane == __ffs(past) - 1) {
                            u64 here = inc - sum;
                            int k = 0;
                            float found = l[0];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                if (here <= t) {
                                    k = i;
                                    found = l[i];
                                }
                                here += x[i];
                            }
                            const int e = first + j + 4 * lane + k - pad;
                            if (HAWK_IN_BOUNDS(P.dev_status, e, P.n)) {
                                P.token[row] = P.v_begin + e;
                                if (P.token_prob) P.token_prob[row] = share(found, inv_total);
                            }
                        }
                        break;
                    }
                    run = __shfl_sync(0xffffffffu, inc, 31);
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
        float *ids = out + P.v_begin + first - pad;  // of place 0 of vals
        const bool whole = (reinterpret_cast<uintptr_t>(ids) & 15u) == 0;
        const float factor = static_cast<float>(inv_total), octaves = fminf(static_cast<float>(rate / kParts), 1e30f);
        const float octaves_low = octaves < 1e30f ? static_cast<float>(rate / kParts - static_cast<double>(octaves)) : 0.f;
        for (int j = base; j < end; j += 128) {
            float l[4], p[4];
            four(j, l);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                // 2^((l - max) * octaves) in fp32: the product in two parts, its whole octaves apart
                const float d = l[k] - mx, z = d * octaves;
                const float whole_z = rintf(z);
                const float rest = (z - whole_z) + (fmaf(d, octaves, -z) + d * octaves_low);
                const float x = hawk::fast_exp2(rest) * __int_as_float((static_cast<int>(whole_z) + 127) << 23) * factor;
                p[k] = greedy || !some || !(l[k] >= tau) || l[k] < nothing ? 0.f : x;
            }
            const int e = j + 4 * lane - pad;  // of the block's ids
            if (e + 4 <= 0 || e >= n) continue;
            if (greedy) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (first + e + k == pick) p[k] = 1.f;
            }
            if (!HAWK_IN_BOUNDS(P.dev_status, static_cast<long long>(P.v_begin) + first + max(e, 0), P.V)) continue;
            if (whole && e >= 0 && e + 4 <= n) {
                *reinterpret_cast<float4 *>(out + P.v_begin + first + e) = make_float4(p[0], p[1], p[2], p[3]);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (e + k >= 0 && e + k < n) out[P.v_begin + first + e + k] = p[k];
            }
        }
        for (int v = rank * NT + tid; v < P.v_begin; v += P.cluster * NT) out[v] = 0.f;
        for (int v = P.v_begin + P.n + rank * NT + tid; v < P.V; v += P.cluster * NT) out[v] = 0.f;
    }
    if (flags && P.dev_status) atomicOr(P.dev_status, flags);
    if (shared()) meet();  // nobody leaves while its shared memory is read
}

constexpr size_t kValsAt = (sizeof(SampleShared) + 15) / 16 * 16;

template <typename T, int NT>
__global__ void __launch_bounds__(NT, 1) sample_kernel(const __grid_constant__ SampleParams P)
{
    extern __shared__ __align__(16) unsigned char smem_raw[];
    hawk::allow_dependent_launch();
    Row<T, NT> row(P, *reinterpret_cast<SampleShared *>(smem_raw), reinterpret_cast<float *>(smem_raw + kValsAt));
    row.prepare();
    hawk::grid_dependency_wait();
    row.run();
}

template <typename T, int NT>
hawk_status launch(const SampleParams &P, int R, cudaStream_t st)
{
    static unsigned long long seen = 0;  // devices on which the kernel may use the shared memory of its largest slice
    constexpr size_t most = kValsAt + sizeof(float) * (kMaxSlice + 16);
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return HAWK_ERR_CUDA;
    const unsigned long long bit = 1ull << (dev & 63);
    if (!(__atomic_load_n(&seen, __ATOMIC_ACQUIRE) & bit) || dev >= 64) {
        if (cudaFuncSetAttribute(sample_kernel<T, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(most)) != cudaSuccess)
            return HAWK_ERR_CUDA;
        __atomic_fetch_or(&seen, bit, __ATOMIC_RELEASE);
    }
    const size_t smem = kValsAt + sizeof(float) * (static_cast<size_t>(P.slice) + 16);
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
    P.rate = a->temperature > 0.f ? rate_of(a->temperature) : 0.0;
    P.least = least_of(a->min_p);
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
        const bool many = static_cast<long long>(a->R) * P.cluster >= 2 * 148 && P.slice <= 16384 - 16;
        return many ? launch<T, 256>(P, a->R, st) : launch<T, 1024>(P, a->R, st);
    };
    return a->dtype == HAWK_F32 ? pick(float{}) : a->dtype == HAWK_BF16 ? pick(__nv_bfloat16{}) : pick(__half{});
}
