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
//   4. a histogram of the list finds the step that the threshold is in, and the step's members against each other the value (one warp does
//      what is not for each id: all the warps doing it would take as long as a pass over the row);
//   5. the sums of what stays tell the warp that the draw falls on, which finds the id.
// With top-k and top-p, 2 to 4 run for each.  Where the list does not hold the threshold (the sample misled, or too many are equal), step 4
// is done on the whole row, as many times as it takes (search()).  Neither changes a result.
// Masses are exponentials in fp64, held as multiples of 2^-44 in 64-bit integers: sums of them are exact, so no order of atomics or warps has a
// say and a token does not depend on the launch.  fp32 sums would not do: with 16 thousand ids one draw in some hundred falls so near to a
// border that their rounding decides it.
//
// A block holds 40960 ids at most; longer rows, and rows of calls with few of them, are shared by a cluster, whose blocks exchange
// histograms, members and sums through distributed shared memory.
//
// What bounds it: instructions and latency, not memory.  512 rows of 16384 ids with their distributions are 67 MB, 10 us, and take 56.5: some 130
// warp instructions for each 32 ids (the pass 45 of them, loading 12, the fp32 mass 8, the distribution 14), 0.53 of the issue slots used by
// two blocks an SM over 1.7 waves.  A row alone takes 12.4 to 15 us, a chain of some ten barriers with a warp's work between them.  Measured and not kept:
// sorting out the ids below an estimated cut first (a pass to pack costs what it saves, 118 us); every warp summing up the histograms
// for itself (7 thousand cycles of 32); 64-bit atomics in shared memory (loops, ten times the three 32-bit ones where ids share a step).
#include <climits>

#include <math_constants.h>

#include "hawk_common.cuh"

namespace {

using u64 = unsigned long long;

constexpr int kBins = 256;       // steps of a histogram: 8 a lane of the warp that sums them up
constexpr int kFinal = 256;      // members of a step that are ranked against each other
constexpr int kList = 2048;      // ids that are looked at one by one, an equal share for each warp
constexpr float kLowest = -3.402823466e38f;  // the lowest number: what is below is none
constexpr int kMaxSlice = 40960; // ids of a row that a block holds
constexpr int kMaxIds = 1 << 18;
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
    u64 a, b;
    float lo, hi;
    int n;
};

// Where a histogram keeps a step: lane i's eight steps, i * 8 and on, lie 32 places apart (side by side they would share a bank with others').
__device__ __forceinline__ int place_of(int bin) { return (bin & 7) * 32 + (bin >> 3); }

struct SampleShared {
    double table[kParts];  // 2^(i / kParts)
    uint32_t hist[3][kBins];  // number of a step, or its mass in parts of 15 bits (40960 of which add up to less than 2^32)
    uint32_t sample[kBins];
    float window_lo, window_hi;  // what one warp finds for all: the list's window, ...
    int bin, ok, complete;  // ... the step of the threshold, the mass or number above it, and whether there is one
    u64 bin_above, target;
    float list_v[kList];   // the warps' shares one after the other
    u64 list_w[kList];
    u64 last_w[kFinal], all_w[kFinal];  // members of the last step: the block's, the row's
    float last_v[kFinal], all_v[kFinal];
    u64 warp_a[32], warp_b[32], warp_c[32], warp_d[32];
    uint32_t warp_lo[32], warp_hi[32];
    int over;              // a warp's share of the list was too small
    float warp_f[32];
    Swap swap[6];  // one for each kind of exchange, so that a barrier lies between two uses of the same
    double rate, least;
    int last, pick;
    uint32_t last_lo, last_hi;  // keys of the last step's smallest and largest
    float tau;
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
    int listed;         // its members of the list
    float mx, nothing;  // the largest; from `nothing`, 32 temperatures below it or more, down a weight is 0
    double rate;        // kParts / (temperature * ln 2)

    __device__ __forceinline__ bool shared() const { return P.cluster > 1; }
    // Three times how far the rank of a threshold in a sample is off (and a little, for few).
    __device__ __forceinline__ float margin_ranks(float rank) const { return each() > 1 ? 3.f * sqrtf(rank) + 4.f : 1.f; }
    __device__ __forceinline__ int each() const { return (P.slice + 4095) / 4096; }  // logits that one of the sample stands for
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
    // ... as a multiple of 2^-44, not yet whole.  The last bit is set, so that no sum of it is a tie: added to a number between 2^52 and 2^53 it
    // counts as the nearest whole multiple, whatever the sum so far.  (At `nothing` and below that is 0: e^-32 of them
    // at most.  -inf takes the weight of `nothing`, which is more where that is the lowest number; no threshold lets -inf stay.)
    __device__ __forceinline__ double raw_weight(float l) const
    {
        int e;
        const double w = power(fmaxf(l, nothing), e);
        return __hiloint2double(__double2hiint(w) + (e + kOneBits) * (1 << 20), __double2loint(w) | 1);
    }
    static constexpr double kWhole = 4503599627370496.0;  // 2^52, from where a thread's sums start: 256 weights fit on top
    static __device__ __forceinline__ u64 whole(double sum) { return static_cast<u64>(__double_as_longlong(sum)) & ((1ull << 52) - 1); }
    __device__ __forceinline__ u64 weight(float l) const { return whole(raw_weight(l) + kWhole); }
    // ... as a number, times `factor`
    __device__ __forceinline__ float share(float l, double factor) const
    {
        int e;
        const double w = power(l, e);
        return static_cast<float>(__hiloint2double(__double2hiint(w) + e * (1 << 20), __double2loint(w)) * factor);
    }
    // What block r of the row has said in a slot, one number at a time (each is a load from another block).
    __device__ __forceinline__ u64 a_of(int slot, int r) const { return hawk::ld_cluster_u64(hawk::map_shared_to_cta(&sh.swap[slot].a, r)); }
    __device__ __forceinline__ u64 b_of(int slot, int r) const { return hawk::ld_cluster_u64(hawk::map_shared_to_cta(&sh.swap[slot].b, r)); }
    __device__ __forceinline__ int n_of(int slot, int r) const
    {
        return static_cast<int>(hawk::ld_cluster_u32(hawk::map_shared_to_cta(&sh.swap[slot].n, r)));
    }
    __device__ __forceinline__ float lo_of(int slot, int r) const
    {
        return __uint_as_float(hawk::ld_cluster_u32(hawk::map_shared_to_cta(&sh.swap[slot].lo, r)));
    }
    __device__ __forceinline__ float hi_of(int slot, int r) const
    {
        return __uint_as_float(hawk::ld_cluster_u32(hawk::map_shared_to_cta(&sh.swap[slot].hi, r)));
    }
    // Lane's four logits of the run of 128 from place j on (-inf from `stop` on).
    __device__ __forceinline__ void four(int j, int stop, float (&l)[4]) const
    {
        const int at = j + 4 * static_cast<int>(threadIdx.x & 31);
        const float4 x = at < stop ? *reinterpret_cast<const float4 *>(vals + at)
                                  : make_float4(-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F);
        l[0] = x.x;
        l[1] = x.y;
        l[2] = x.z;
        l[3] = x.w;
    }
    __device__ __forceinline__ int load(long long row, int first, int n, float scale, float &lo, float &hi);
    __device__ __forceinline__ void ends(float &lo, float &hi, int slot);
    __device__ __forceinline__ void clear();
    __device__ __forceinline__ float mass_of_row();
    __device__ __forceinline__ void sample(const Steps &step);
    template <typename N>
    __device__ __forceinline__ void of_row(const uint32_t *hist, N (&part)[kBins / 32]) const;
    __device__ __forceinline__ void between_ranks(float bottom, float above, float margin);
    __device__ __forceinline__ void between_masses(const Steps &step, float bottom, float from, float below, float margin);
    template <bool kMass>
    __device__ __forceinline__ void pass(const Steps &step, float lo, float hi, float from, float least);
    template <bool kMass>
    __device__ __forceinline__ void count(int at, u64 weight);
    template <bool kMass>
    __device__ __forceinline__ void find_step(u64 above, u64 target);
    __device__ __forceinline__ void push(float l, u64 weight, uint32_t &low, uint32_t &high);
    __device__ __forceinline__ void range(uint32_t low, uint32_t high);
    __device__ __forceinline__ bool finish(u64 target, float &low, float &high);
    template <bool kMass>
    __device__ __forceinline__ bool from_list(const Steps &step, float lo, float hi, u64 want, float share, float &tau, u64 &target, bool &complete);
    template <bool kMass>
    __device__ __forceinline__ bool search(float lo, float hi, float bottom, u64 target, float &tau);
};

// What does not depend on the call's inputs: done before the kernel ahead has ended.
template <typename T, int NT>
__device__ __forceinline__ void Row<T, NT>::prepare()
{
    for (int i = threadIdx.x; i < kParts; i += NT) sh.table[i] = exp2(static_cast<double>(i) / kParts);
    for (int i = threadIdx.x; i < kBins; i += NT) sh.sample[i] = 0;
    clear();
}

// For a histogram and its last step.
template <typename T, int NT>
__device__ __forceinline__ void Row<T, NT>::clear()
{
    for (int i = threadIdx.x; i < 3 * kBins; i += NT) sh.hist[0][i] = 0;
    if (threadIdx.x == 0) {
        sh.last = 0;
        sh.over = 0;
        sh.last_lo = 0xffffffffu;
        sh.last_hi = 0;
    }
}

// The block's n logits from id v_begin + first on into vals[pad ..]; returns pad, by which the 16-byte pieces of memory lie on 16-byte places of vals.  hi: the
// largest; lo: the smallest among some of them.
template <typename T, int NT>
__device__ __forceinline__ int Row<T, NT>::load(long long row, int first, int n, float scale, float &lo, float &hi)
{
    constexpr int kN = Piece<T>::kN;
    const T *c = static_cast<const T *>(P.logits) + row * P.row_stride + P.v_begin + first;
    const bool has = P.uncond != nullptr;
    const T *u = has ? static_cast<const T *>(P.uncond) + row * P.uncond_stride + P.v_begin + first : c;
    const int pad = static_cast<int>((reinterpret_cast<uintptr_t>(c) & 15u) / sizeof(T));
    const int pieces = n > 0 ? (pad + n + kN - 1) / kN : 0;
    m = pieces * kN;
    hi = -CUDART_INF_F;
    lo = CUDART_INF_F;
    // whole pieces, where those of both rows lie alike
    const bool alike = ((reinterpret_cast<uintptr_t>(c) ^ reinterpret_cast<uintptr_t>(u)) & 15u) == 0;
    const int q0 = pad > 0 ? 1 : 0, q1 = alike ? (pad + n) / kN : q0;
    constexpr int kFlight = sizeof(T) == 4 ? 4 : 2;
    for (int q = q0 + threadIdx.x; q < q1; q += NT * kFlight) {
        Piece<T> pc[kFlight], pu[kFlight];
#pragma unroll
        for (int k = 0; k < kFlight; ++k)
            if (q + k * NT < q1) {
                pc[k].raw = __ldcs(reinterpret_cast<const uint4 *>(c + (q + k * NT) * kN - pad));
                pu[k].raw = has ? __ldcs(reinterpret_cast<const uint4 *>(u + (q + k * NT) * kN - pad)) : pc[k].raw;
            }
#pragma unroll
        for (int k = 0; k < kFlight; ++k)
            if (q + k * NT < q1) {
                float x[kN];
#pragma unroll
                for (int i = 0; i < kN; ++i) {
                    x[i] = guided(pc[k].at(i), pu[k].at(i), has, scale, flags);
                    hi = fmaxf(hi, x[i]);
                }
                if (x[0] >= kLowest) lo = fminf(lo, x[0]);
#pragma unroll
                for (int i = 0; i < kN; i += 4)
                    *reinterpret_cast<float4 *>(vals + (q + k * NT) * kN + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
            }
    }
    // what is left at the ends (or all of it), one by one
    const int done0 = q1 > q0 ? q0 * kN : 0, done1 = q1 > q0 ? q1 * kN : 0;
    for (int j = threadIdx.x; j < m - (done1 - done0); j += NT) {
        const int at = j < done0 ? j : j + (done1 - done0), e = at - pad;
        float x = -CUDART_INF_F;
        if (e >= 0 && e < n) x = guided(to_f32(c[e]), to_f32(u[e]), has, scale, flags);
        hi = fmaxf(hi, x);
        if (x >= kLowest) lo = fminf(lo, x);
        vals[at] = x;
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
            lo = fminf(lo, lo_of(slot, r));
            hi = fmaxf(hi, hi_of(slot, r));
        }
    }
}

// The warp's part of the row's mass in fp32, to warp_f.
template <typename T, int NT>
__device__ __forceinline__ float Row<T, NT>::mass_of_row()
{
    const float octaves = static_cast<float>(rate / kParts), top = mx * octaves;
    float mass = 0.f;
    for (int j = base; j < end; j += 128) {
        float l[4];
        four(j, end, l);
        mass += (hawk::fast_exp2(fmaf(l[0], octaves, -top)) + hawk::fast_exp2(fmaf(l[1], octaves, -top))) +
                (hawk::fast_exp2(fmaf(l[2], octaves, -top)) + hawk::fast_exp2(fmaf(l[3], octaves, -top)));
    }
    return hawk::warp_sum(mass);
}

// One logit in `each` (of the block's P.slice), at most 4096 of them, in quads, to the histogram of the sample.
template <typename T, int NT>
__device__ __forceinline__ void Row<T, NT>::sample(const Steps &step)
{
    for (int q = threadIdx.x; q < 1024; q += NT) {
        const int at = 4 * each() * q;
        if (at < m) {
            const float4 l = *reinterpret_cast<const float4 *>(vals + at);
            if (l.x >= kLowest) atomicAdd(&sh.sample[place_of(step(l.x))], 1u);
            if (l.y >= kLowest) atomicAdd(&sh.sample[place_of(step(l.y))], 1u);
            if (l.z >= kLowest) atomicAdd(&sh.sample[place_of(step(l.z))], 1u);
            if (l.w >= kLowest) atomicAdd(&sh.sample[place_of(step(l.w))], 1u);
        }
    }
    __syncwarp();
}

// The lane's eight steps of a histogram, of all the row's blocks (eight loads in flight: one from another block takes some 700 cycles).
template <typename T, int NT>
template <typename N>
__device__ __forceinline__ void Row<T, NT>::of_row(const uint32_t *hist, N (&part)[kBins / 32]) const
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < kBins / 32; ++i) part[i] = shared() ? 0 : hist[i * 32 + lane];
    if (!shared()) return;
    for (int r = 0; r < P.cluster; ++r) {
        const uint32_t at = hawk::map_shared_to_cta(hist + lane, r);
        uint32_t x[kBins / 32];
#pragma unroll
        for (int i = 0; i < kBins / 32; ++i) x[i] = hawk::ld_cluster_u32(at + 128 * i);
#pragma unroll
        for (int i = 0; i < kBins / 32; ++i) part[i] += x[i];
    }
}

// Values between which the logit of rank `above` of the sample lies, by `margin` ranks on either side (one warp, behind a barrier).
template <typename T, int NT>
__device__ __forceinline__ void Row<T, NT>::between_ranks(float bottom, float above, float margin)
{
    constexpr int kPer = kBins / 32;
    const int lane = threadIdx.x & 31;
    uint32_t part[kPer], sum = 0;
    of_row(sh.sample, part);
#pragma unroll
    for (int i = 0; i < kPer; ++i) sum += part[i];
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
    if (lane == 0) {
        const float wide = (mx - bottom) / kBins;
        sh.window_hi = b1 > 0 && b1 < kBins ? mx - wide * b1 : CUDART_INF_F;
        sh.window_lo = b2 < kBins - 1 ? mx - wide * (b2 + 1) : kLowest;
    }
}

// Values between which the logits from `from` up to the threshold have the mass `below` together, as the sample has it, with a share `margin` of
// it on either side, and margin_ranks(rank) of the sample's ranks (near the top, few of the sample have most of the mass).  One warp, behind a
// barrier.
template <typename T, int NT>
__device__ __forceinline__ void Row<T, NT>::between_masses(const Steps &step, float bottom, float from, float below, float margin)
{
    constexpr int kPer = kBins / 32;
    const int lane = threadIdx.x & 31, last = step(from);
    const float wide = (mx - bottom) / kBins, octaves = static_cast<float>(rate / kParts);
    float part[kPer], sum = 0.f;
    uint32_t number[kPer], numbers = 0;
    of_row(sh.sample, number);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int b = lane * kPer + i;
        part[i] = b <= last && number[i] > 0 ? each() * number[i] * hawk::fast_exp2(-wide * octaves * (b + 0.5f)) : 0.f;
        sum += part[i];
        numbers += number[i];
    }
    // (sums from the far end up: the near end's few large weights are what a sample knows least)
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const float x = __shfl_down_sync(0xffffffffu, sum, o);
        if (lane + o < 32) sum += x;
    }
    float tail = __shfl_down_sync(0xffffffffu, sum, 1);
    if (lane == 31) tail = 0.f;
    int b1 = kBins, b2 = kBins, middle = kBins;
#pragma unroll
    for (int i = kPer - 1; i >= 0; --i) {  // tail: what lies behind step lane * kPer + i
        if (tail <= below * (1.f + margin)) b1 = lane * kPer + i;
        if (tail <= below) middle = lane * kPer + i;
        if (tail <= below * (1.f - margin)) b2 = lane * kPer + i;
        tail += part[i];
    }
    b1 = __reduce_min_sync(0xffffffffu, b1);
    b2 = __reduce_min_sync(0xffffffffu, b2);
    middle = __reduce_min_sync(0xffffffffu, middle);
    uint32_t run = warp_inclusive(numbers) - numbers, rank = 0;
    const uint32_t before = run;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        run += number[i];
        if (lane * kPer + i == middle) rank = run;
    }
    rank = __reduce_max_sync(0xffffffffu, rank);
    const float low = rank - margin_ranks(rank), high = rank + margin_ranks(rank);
    int r1 = low <= 1.f ? 0 : kBins, r2 = kBins;
    run = before;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        run += number[i];
        if (run >= low) r1 = min(r1, lane * kPer + i);
        if (run >= high) r2 = min(r2, lane * kPer + i);
    }
    b1 = min(b1, __reduce_min_sync(0xffffffffu, r1));
    b2 = max(b2, __reduce_min_sync(0xffffffffu, r2));
    if (lane == 0) {
        sh.window_hi = b1 > 0 && b1 < kBins ? mx - wide * b1 : CUDART_INF_F;
        sh.window_lo = b2 < kBins - 1 ? mx - wide * (b2 + 1) : kLowest;
    }
}

// One more of a step: its number, or its weight in three parts whose sums stay below 2^32.
template <typename T, int NT>
template <bool kMass>
__device__ __forceinline__ void Row<T, NT>::count(int at, u64 w)
{
    if (!kMass) {
        atomicAdd(&sh.hist[0][at], 1u);
    } else {
        constexpr uint32_t kPart = (1u << 15) - 1;
        atomicAdd(&sh.hist[0][at], static_cast<uint32_t>(w) & kPart);
        atomicAdd(&sh.hist[1][at], static_cast<uint32_t>(w >> 15) & kPart);
        atomicAdd(&sh.hist[2][at], static_cast<uint32_t>(w >> 30));
    }
}

// One pass over the weights of the logits from `from` on: those from lo (not below `from`) up to hi go to the list and, by their step, to the
// histogram.  The warp's sums: of what lies above (warp_a, and its number in warp_lo); of everything, for top-p (warp_b); of the part above
// that min-p leaves, which keeps what is not below `least` (warp_d).
template <typename T, int NT>
template <bool kMass>
__device__ __forceinline__ void Row<T, NT>::pass(const Steps &step, float lo, float hi, float from, float least)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    double above = kWhole, all = kWhole, stays = kWhole;
    const bool cuts = least > hi;
    int up_count = 0;
    listed = 0;
    // 8 runs of 128 at a time, so that the marks of members fit 32 bits (a lane's sums take 256 weights: 40960 / 8 warps / 32 lanes are 160)
    for (int j0 = base; j0 < end; j0 += 8 * 128) {
        uint32_t marks = 0;
        const int stop = min(end, j0 + 8 * 128);
        for (int j = j0; j < stop; j += 128) {
            float l[4];
            four(j, end, l);
            uint32_t in = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const double x = raw_weight(l[k]);
                const bool up = l[k] >= hi;
                if (kMass && l[k] >= from) all += x;
                if (up) above += x;
                if (!kMass && up) ++up_count;
                if (!up && l[k] >= lo) in |= 1u << k;
            }
            if (cuts) {  // (rare: a second look is cheaper than a third sum in each of them)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (l[k] >= least) stays += raw_weight(l[k]);
            }
            marks |= in << ((j - j0) >> 5);
        }
        const int mine = __popc(marks), sum = warp_inclusive(mine);
        for (int to = listed + sum - mine; marks; marks &= marks - 1, ++to) {
            const int i = __ffs(marks) - 1;
            const float l = vals[j0 + (i >> 2) * 128 + 4 * lane + (i & 3)];
            const u64 x = weight(l);
            count<kMass>(place_of(step(l)), x);
            if (to < kShare) {
                sh.list_v[warp * kShare + to] = l;
                sh.list_w[warp * kShare + to] = x;
            }
        }
        __syncwarp();
        listed += __shfl_sync(0xffffffffu, sum, 31);
    }
    const u64 a = warp_sum(whole(above)), d = cuts ? warp_sum(whole(stays)) : a;
    u64 b = 0;
    if (kMass) b = warp_sum(whole(all));
    if (!kMass) up_count = __reduce_add_sync(0xffffffffu, up_count);
    if (lane == 0) {
        sh.warp_a[warp] = a;
        sh.warp_b[warp] = b;
        sh.warp_d[warp] = d;
        sh.warp_lo[warp] = up_count;
        if (listed > kShare) sh.over = 1;
    }
}

// The step of the histogram that the target is reached in (one warp, behind a barrier): bin, and the number or mass above it.
template <typename T, int NT>
template <bool kMass>
__device__ __forceinline__ void Row<T, NT>::find_step(u64 above, u64 target)
{
    constexpr int kPer = kBins / 32;
    const int lane = threadIdx.x & 31;
    u64 part[kPer], sum = 0;
    of_row(sh.hist[0], part);
    if (kMass) {
        u64 more[kPer];
#pragma unroll
        for (int k = 1; k < 3; ++k) {
            of_row(sh.hist[k], more);
#pragma unroll
            for (int i = 0; i < kPer; ++i) part[i] += more[i] << (15 * k);
        }
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) sum += part[i];
    u64 run = above + warp_inclusive(sum) - sum;
    int bin = -1;
    u64 at_run = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        if (run < target && run + part[i] >= target) {
            bin = lane * kPer + i;
            at_run = run;
        }
        run += part[i];
    }
    const uint32_t who = __ballot_sync(0xffffffffu, bin >= 0);
    if (lane == (who ? __ffs(who) - 1 : 0)) {
        sh.bin = bin;
        sh.bin_above = at_run;
        sh.ok = who != 0;
        sh.target = target;
    }
}

// One more member of the last step.
template <typename T, int NT>
__device__ __forceinline__ void Row<T, NT>::push(float l, u64 w, uint32_t &low, uint32_t &high)
{
    const int at = atomicAdd(&sh.last, 1);
    if (at < kFinal) {
        sh.last_v[at] = l;
        sh.last_w[at] = w;
    }
    low = min(low, key_of(l));
    high = max(high, key_of(l));
}

// The lanes' smallest and largest members, to those of the block.
template <typename T, int NT>
__device__ __forceinline__ void Row<T, NT>::range(uint32_t low, uint32_t high)
{
    __syncwarp();
    low = __reduce_min_sync(0xffffffffu, low);
    high = __reduce_max_sync(0xffffffffu, high);
    if ((threadIdx.x & 31) == 0 && low <= high) {
        atomicMin(&sh.last_lo, low);
        atomicMax(&sh.last_hi, high);
    }
}

// The value at which the last step's members reach the target, to sh.tau (all threads; barriers lie in it); false if there are too many, of
// values from low to high.
template <typename T, int NT>
__device__ __forceinline__ bool Row<T, NT>::finish(u64 target, float &low, float &high)
{
    const int tid = threadIdx.x, lane = tid & 31;
    __syncthreads();
    int members = sh.last;
    const float *v = sh.last_v;
    const u64 *w = sh.last_w;
    low = value_of(sh.last_lo);  // (nonsense without members)
    high = value_of(sh.last_hi);
    if (shared()) {
        if (tid == 0) {
            sh.swap[2].n = members;
            sh.swap[2].lo = members > 0 ? low : CUDART_INF_F;
            sh.swap[2].hi = members > 0 ? high : -CUDART_INF_F;
        }
        meet();
        int before[kMaxCluster + 1];
        before[0] = 0;
        low = CUDART_INF_F;
        high = -CUDART_INF_F;
#pragma unroll
        for (int r = 0; r < kMaxCluster; ++r) {
            before[r + 1] = before[r];
            if (r < P.cluster) {
                before[r + 1] += n_of(2, r);
                low = fminf(low, lo_of(2, r));
                high = fmaxf(high, hi_of(2, r));
            }
        }
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
    if (low == high) {  // (16-bit logits are equal by the hundred)
        if (tid == 0) sh.tau = low;
    } else if (members > kFinal) {
        return false;
    } else if (tid < 32) {  // against each other, a member a lane
        float best = -CUDART_INF_F;
        const u64 above = sh.bin_above;
        for (int i = lane; i < members; i += 32) {
            const float mine = v[i];
            u64 reach = above;
            for (int k = 0; k < members; ++k)
                if (v[k] >= mine) reach += w[k];
            if (reach >= target) best = fmaxf(best, mine);
        }
        __syncwarp();
        best = value_of(__reduce_max_sync(0xffffffffu, key_of(best)));
        if (lane == 0) sh.tau = best;
    }
    __syncthreads();
    return true;
}

// The threshold among the list that a pass has made of the logits from lo up to hi: the largest value from which on the logits reach the target:
// `want` of them, or `share` of the mass.  False if it is not among them.  complete: the list has them all.  The same in all
// blocks of the row.
template <typename T, int NT>
template <bool kMass>
__device__ __forceinline__ bool Row<T, NT>::from_list(const Steps &step, float lo, float hi, u64 want, float share, float &tau, u64 &target, bool &complete)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    __syncthreads();
    if (warp == 0 || shared()) {
        u64 above = kMass ? warp_sum(lane < NW ? sh.warp_a[lane] : 0ull) : __reduce_add_sync(0xffffffffu, lane < NW ? sh.warp_lo[lane] : 0u);
        u64 all = kMass ? warp_sum(lane < NW ? sh.warp_b[lane] : 0ull) : 0ull;
        int over = sh.over;
        if (shared()) {
            if (threadIdx.x == 0) {
                sh.swap[1].a = above;
                sh.swap[1].b = all;
                sh.swap[1].n = over;
            }
            meet();
            above = all = 0;
            over = 0;
            if (warp == 0)
                for (int r = 0; r < P.cluster; ++r) {
                    above += a_of(1, r);
                    if (kMass) all += b_of(1, r);
                    over |= n_of(1, r);
                }
        }
        if (warp == 0) {
            find_step<kMass>(above, kMass ? target_of(static_cast<double>(share), all) : want);
            if (lane == 0) sh.complete = !over;
        }
    }
    __syncthreads();
    target = sh.target;
    complete = sh.complete != 0;
    if (!sh.ok) return false;
    const int bin = sh.bin;
    uint32_t low = 0xffffffffu, high = 0;
    if (complete) {
        for (int i = lane; i < listed; i += 32) {
            const float l = sh.list_v[warp * kShare + i];
            if (l >= lo && step(l) == bin) push(l, kMass ? sh.list_w[warp * kShare + i] : 1, low, high);
        }
    } else {
        for (int j = base + lane; j < end; j += 32) {
            const float l = vals[j];
            if (l >= lo && l < hi && step(l) == bin) push(l, kMass ? weight(l) : 1, low, high);
        }
    }
    range(low, high);
    float least, most;
    if (!finish(target, least, most)) return false;
    tau = sh.tau;
    return true;
}

// The largest value tau in [lo, hi] for which the logits from it to hi reach the target, their number or their mass; false if all do not.  Any
// distribution of values, as many rounds as it takes (a round leaves one value out at least).  The first round's steps start from
// `bottom`, the last of them takes what is below.  The same in all blocks of the row.
template <typename T, int NT>
template <bool kMass>
__device__ __forceinline__ bool Row<T, NT>::search(float lo, float hi, float bottom, u64 target, float &tau)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    u64 above = 0;
    while (lo < hi) {
        const Steps step(fmaxf(lo, bottom), hi);
        barrier();  // (everybody has read what the round before, or the search before, left in sh)
        clear();
        __syncthreads();
        for (int j = base + lane; j < end; j += 32) {
            const float l = vals[j];
            if (l >= lo && l <= hi) count<kMass>(place_of(step(l)), kMass ? weight(l) : 1);
        }
        __syncwarp();
        barrier();
        if (warp == 0) find_step<kMass>(above, target);
        __syncthreads();
        if (!sh.ok) return false;
        const int bin = sh.bin;
        above = sh.bin_above;
        uint32_t low = 0xffffffffu, high = 0;
        for (int j = base + lane; j < end; j += 32) {
            const float l = vals[j];
            if (l >= lo && l <= hi && step(l) == bin) push(l, kMass ? weight(l) : 1, low, high);
        }
        range(low, high);
        float least, most;
        if (finish(target, least, most)) {
            tau = sh.tau;
            return true;
        }
        lo = bottom = least;
        hi = most;
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
    const bool greedy = temperature == 0.f;
    if (tid == 0) {  // (a row's own settings: fp64 division and logarithm by one lane)
        sh.rate = !P.temperatures ? P.rate : greedy ? 0.0 : rate_of(temperature);
        sh.least = !P.min_ps ? P.least : least_of(min_p);
        sh.pick = INT_MAX;
    }
    ends(lo, hi, 0);
    mx = hi;
    lo = fminf(lo, hi);  // (none of some was a number)
    rate = sh.rate;
    // `nothing` is rounded downwards (to 96 temperatures below the maximum at most): nearer than 31.2 its own weight, which every lower id takes, would
    // not be 0.  Where the next lower number lies 32 temperatures below the maximum it is the maximum itself.  (That difference is exact.)
    nothing = mx - value_of(key_of(mx) - 1) >= 32.f * temperature ? mx : fmaxf(__fmaf_rd(-32.f, temperature, mx), kLowest);
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
            for (int r = 0; r < P.cluster; ++r) pick = min(pick, n_of(4, r));
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
        const bool by_k = top_k > 0 && top_k < P.n && !flat;
        const bool by_p = top_p < 1.f && !flat;

        // ---- thresholds of top-k and top-p
        float tau_k = kLowest, tau_p = kLowest, window_hi = CUDART_INF_F;
        bool summed = false;  // warp_a has the sums of what lies above the window, the list what lies in it
        if (by_k || by_p) {
            const float bottom = by_k ? lo : fmaxf(lo, nothing);
            const Steps step(bottom, mx);
            float mass = 0.f;
            if (!by_k) {
                mass = mass_of_row();
                if (lane == 0) sh.warp_f[warp] = mass;
            }
            sample(step);
            __syncthreads();
            if (shared()) {
                if (warp == 0 && !by_k) {
                    mass = hawk::warp_sum(lane < NW ? sh.warp_f[lane] : 0.f);
                    if (lane == 0) sh.swap[5].lo = mass;
                }
                meet();
                mass = 0.f;
                if (!by_k && warp == 0)
                    for (int r = 0; r < P.cluster; ++r) mass += lo_of(5, r);
            } else if (!by_k && warp == 0) {
                mass = hawk::warp_sum(lane < NW ? sh.warp_f[lane] : 0.f);
            }
            u64 target;
            if (by_k) {
                if (warp == 0) {
                    const float s = static_cast<float>(top_k) / each();
                    between_ranks(bottom, s, margin_ranks(s));
                }
                __syncthreads();
                const float w_lo = sh.window_lo;
                window_hi = top_k <= kList / 2 ? CUDART_INF_F : sh.window_hi;  // (few: all of them to the list, for top-p)
                const Steps fine(fmaxf(w_lo, bottom), fminf(window_hi, mx));
                pass<false>(fine, w_lo, window_hi, kLowest, tau_m);
                const bool found = from_list<false>(fine, w_lo, window_hi, static_cast<u64>(top_k), 0.f, tau_k, target, summed);
                summed &= found;
                if (!found && !search<false>(kLowest, mx, bottom, static_cast<u64>(top_k), tau_k)) tau_k = kLowest;  // (fewer logits than top_k)
            }
            if (by_p && tau_k < mx) {
                if (by_k) {  // the mass of what top-k left
                    double mine = kWhole;
                    u64 all;
                    if (summed) {
                        all = 0;
                        for (int i = lane; i < listed; i += 32)
                            if (sh.list_v[warp * kShare + i] >= tau_k) all += sh.list_w[warp * kShare + i];
                        if (lane == 0) all += sh.warp_a[warp];
                    } else {
                        for (int j = base; j < end; j += 128) {
                            float l[4];
                            four(j, end, l);
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const double x = raw_weight(l[k]);
                                if (l[k] >= tau_k) mine += x;
                            }
                        }
                        all = whole(mine);
                    }
                    __syncwarp();
                    all = warp_sum(all);
                    if (lane == 0) sh.warp_c[warp] = all;
                    barrier();
                    clear();  // (the list's searches are done, in all blocks)
                    __syncthreads();
                    all = warp_sum(lane < NW ? sh.warp_c[lane] : 0ull);
                    if (shared()) {
                        if (tid == 0) sh.swap[4].a = all;
                        meet();
                        all = 0;
                        for (int r = 0; r < P.cluster; ++r) all += a_of(4, r);
                    }
                    mass = static_cast<float>(static_cast<double>(all) / kOne);
                }
                const float from = fmaxf(tau_k, nothing);
                float w_lo = from;
                if (summed && window_hi == CUDART_INF_F) {  // the list has all that top-k left
                    const Steps fine(from, mx);
                    u64 of_list = 0;
                    for (int i = lane; i < listed; i += 32)
                        if (sh.list_v[warp * kShare + i] >= from) {
                            of_list += sh.list_w[warp * kShare + i];
                            count<true>(place_of(fine(sh.list_v[warp * kShare + i])), sh.list_w[warp * kShare + i]);
                        }
                    __syncwarp();
                    of_list = warp_sum(of_list);
                    if (lane == 0) sh.warp_b[warp] = of_list;
                    const bool found = from_list<true>(fine, from, window_hi, 0, fmaxf(top_p, 0.f), tau_p, target, summed);
                    summed &= found;
                    if (!found) (void)search<true>(from, mx, bottom, target, tau_p);
                } else {
                    if (warp == 0) between_masses(step, bottom, from, (1.f - top_p) * mass, each() > 1 ? 0.12f : 0.02f);
                    __syncthreads();
                    w_lo = fmaxf(sh.window_lo, from);
                    window_hi = sh.window_hi;
                    const Steps fine(w_lo, fminf(window_hi, mx));
                    pass<true>(fine, w_lo, window_hi, from, tau_m);
                    const bool found = from_list<true>(fine, w_lo, window_hi, 0, fmaxf(top_p, 0.f), tau_p, target, summed);
                    summed &= found;
                    if (!found) (void)search<true>(from, mx, bottom, target, tau_p);
                }
            }
        }
        tau = fmaxf(fmaxf(tau_k, tau_p), tau_m);

        // ---- what stays, for each warp
        u64 kept = 0;
        if (summed) {
            for (int i = lane; i < listed; i += 32)
                if (sh.list_v[warp * kShare + i] >= tau) kept += sh.list_w[warp * kShare + i];
            if (lane == 0) kept += sh.warp_d[warp];
        } else {
            double sum = kWhole;
            for (int j = base; j < end; j += 128) {
                float l[4];
                four(j, end, l);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const double x = raw_weight(l[k]);
                    if (l[k] >= tau) sum += x;
                }
            }
            kept = whole(sum);
        }
        __syncwarp();
        kept = warp_sum(kept);
        __syncthreads();  // (warp_b has been read)
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
                const u64 a = a_of(3, r);
                if (r < rank) before += a;
                total += a;
            }
        }
        inv_total = kOne / static_cast<double>(total);
        const u64 t = static_cast<u64>(static_cast<double>(u) * static_cast<double>(total));  // the running sum that has to be exceeded
        if (t >= before && t - before < mine) {
            const int at = __ffs(__ballot_sync(0xffffffffu, before + sums > t)) - 1;  // the stretch it falls on
            const u64 low = __shfl_sync(0xffffffffu, sums, at > 0 ? at - 1 : 0), run = before + (at > 0 ? low : 0);
            const int j0 = min(m, at * stretch), j1 = min(m, j0 + stretch), runs = (j1 - j0 + 127) / 128;  // 32 of them at most
            auto weigh = [&](int j, float (&l)[4], u64 (&x)[4]) {
                four(j, j1, l);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const u64 y = weight(l[k]);
                    x[k] = l[k] >= tau ? y : 0;
                }
                return (x[0] + x[1]) + (x[2] + x[3]);
            };
            float l[4];
            u64 x[4];
            for (int r = warp; r < runs; r += NW) {
                const u64 sum = warp_sum(weigh(j0 + 128 * r, l, x));
                if (lane == 0) sh.warp_c[r] = sum;
            }
            __syncthreads();
            const u64 of_runs = run + warp_inclusive(lane < runs ? sh.warp_c[lane] : 0ull);
            const int r = __ffs(__ballot_sync(0xffffffffu, of_runs > t)) - 1;  // the run
            const u64 in_front = __shfl_sync(0xffffffffu, of_runs, r > 0 ? r - 1 : 0);
            if (warp == r % NW) {
                const u64 sum = weigh(j0 + 128 * r, l, x), inc = (r > 0 ? in_front : run) + warp_inclusive(sum);
                if (lane == __ffs(__ballot_sync(0xffffffffu, inc > t)) - 1) {
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
                    const int e = first + j0 + 128 * r + 4 * lane + k - pad;
                    if (HAWK_IN_BOUNDS(P.dev_status, e, P.n)) {
                        P.token[row] = P.v_begin + e;
                        if (P.token_prob) P.token_prob[row] = share(found, inv_total);
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
        const bool aligned = (reinterpret_cast<uintptr_t>(out + P.v_begin + first - pad) & 15u) == 0;  // of place 0 of vals
        const float factor = static_cast<float>(inv_total), octaves = static_cast<float>(rate / kParts);
        const float octaves_low = static_cast<float>(rate / kParts - static_cast<double>(octaves));
        const bool in_range = octaves < 1e37f;  // (of fp32: temperatures that are themselves next to nothing are not)
        for (int j = base; j < end; j += 128) {
            float l[4], p[4];
            four(j, end, l);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                // 2^((l - max) * octaves) in fp32: the product in two parts, the second to first order
                const float d = fmaxf(l[k], nothing) - mx, z = d * octaves;
                const float e = hawk::fast_exp2(z), low = fmaf(d, octaves, -z) + d * octaves_low;
                float x = fmaf(e, low * 0.69314718f, e) * factor;
                if (!in_range) x = share(fmaxf(l[k], nothing), inv_total);
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
            if (aligned && e >= 0 && e + 4 <= n) {
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

template <typename T, int NT, int kOnSm>
__global__ void __launch_bounds__(NT, kOnSm) sample_kernel(const __grid_constant__ SampleParams P)
{
    extern __shared__ __align__(16) unsigned char smem_raw[];
    hawk::allow_dependent_launch();
    Row<T, NT> row(P, *reinterpret_cast<SampleShared *>(smem_raw), reinterpret_cast<float *>(smem_raw + kValsAt));
    row.prepare();
    hawk::grid_dependency_wait();
    row.run();
}

template <typename T, int NT, int kOnSm>
hawk_status launch(const SampleParams &P, int R, cudaStream_t st)
{
    static unsigned long long seen = 0;  // devices on which the kernel may use the shared memory of its largest slice
    constexpr size_t most = kValsAt + sizeof(float) * (kMaxSlice + 16);
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return HAWK_ERR_CUDA;
    const unsigned long long bit = 1ull << (dev & 63);
    if (!(__atomic_load_n(&seen, __ATOMIC_ACQUIRE) & bit) || dev >= 64) {
        if (cudaFuncSetAttribute(sample_kernel<T, NT, kOnSm>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(most)) != cudaSuccess)
            return HAWK_ERR_CUDA;
        __atomic_fetch_or(&seen, bit, __ATOMIC_RELEASE);
    }
    const size_t smem = kValsAt + sizeof(float) * (static_cast<size_t>(P.slice) + 16);
    const dim3 grid(static_cast<unsigned>(R) * P.cluster);
    const cudaError_t e = P.cluster > 1
                              ? hawk_host::launch_dependent_clusters(sample_kernel<T, NT, kOnSm>, P.cluster, grid, dim3(NT), smem, st, P)
                              : hawk_host::launch_dependent(sample_kernel<T, NT, kOnSm>, grid, dim3(NT), smem, st, P);
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
    if (n < 1 || n > kMaxIds) return HAWK_ERR_UNSUPPORTED;
    if (a->row_stride < 0 || (a->uncond && a->uncond_row_stride < 0) || (a->R > 1 && a->probs && a->probs_row_stride < a->V))
        return HAWK_ERR_SHAPE;
    const uintptr_t size = a->dtype == HAWK_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(a->logits) % size || reinterpret_cast<uintptr_t>(a->uncond) % size ||
        !hawk_host::aligned4(a->u, a->token, a->token_prob, a->probs, a->row_temperature, a->row_top_k, a->row_top_p, a->row_min_p,
                             a->row_cfg_scale))
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
    // Blocks of a row.  Where all blocks run at once (132 in clusters, which do not reach every SM): as many as keep it so, of 4096 ids for
    // a few rows (one row of 16384 ids, top-k 2000: 13.4 us in one block, 12.4 in four; of 100003 in bf16 23.0 in three, 18.7 in
    // eight), of 8192 for more (32 rows of 50257: 21.8 us in two, 17.4 in four; 64 rows: 21.9 in two, 38 in three); rows of 16384 and
    // less then stay in one (64 rows: 13.9 us, 14.7 in two).  Up to two waves of blocks: 20480 ids (48 rows of 100003: 45.8 us in three, 38.8
    // in five).  Else as few as hold the row (200 rows of 100003: 125 us in three, 162 in five).
    const auto blocks_of = [&](int ids) { return (n + ids - 1) / ids; };
    const long long rows = a->R;
    const int least = blocks_of(kMaxSlice);
    int blocks = 1;
    if (rows * least <= (least > 1 ? 132 : 148)) {
        blocks = rows <= 16 ? n / 4096 : n > 16384 ? n / 8192 : 1;
        if (rows * blocks > 132) blocks = static_cast<int>(132 / rows);
    } else if (rows * blocks_of(20480) <= 2 * 148) {
        blocks = blocks_of(20480);
    }
    if (blocks > kMaxCluster) blocks = kMaxCluster;
    P.cluster = blocks > least ? blocks : least;
    P.slice = ((n + P.cluster - 1) / P.cluster + 15) & ~15;  // (every block's rows then lie alike in 16-byte pieces)
    const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    auto pick = [&](auto type) {
        using T = decltype(type);
        // Calls of more rows than SMs: two blocks of 512 threads on an SM (512 rows of 16384 ids 40 us, 59 with one; 100 rows 19.5 and 14.0,
        // because two blocks go to an SM while others have none), blocks of 256 for short rows, of which four fit an SM up to some 4900 ids and three
        // up to 8192.  fp32, top-p, 256 and 512 threads: 2000 rows of 1000 ids 38 and 63 us, of 4096 59 and 86, of 5500 81 and 99, of 8192 96 and 110; 300 rows
        // of 8192 21 and 26; bf16 and
        // other settings alike.  (149 rows, one more than SMs, of 8192 ids: 17 and 16.)
        if (P.cluster > 1 || P.slice > 16384 || a->R <= 148) return launch<T, 512, 1>(P, a->R, st);
        return P.slice > 8192 ? launch<T, 512, 2>(P, a->R, st) : launch<T, 256, 4>(P, a->R, st);
    };
    return a->dtype == HAWK_F32 ? pick(float{}) : a->dtype == HAWK_BF16 ? pick(__nv_bfloat16{}) : pick(__half{});
}
