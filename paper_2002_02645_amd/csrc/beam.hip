// The choice of the next tokens of a generating model's requests, and the reordering of its states (gfx950 / CDNA4).
//
// Choice.  total(j, v) = score_j + l_jv - log sum_u exp l_ju, the k best of a group's rows j and tokens v.  Within a row the
// values themselves decide, so that a row's sum of exponentials and its k best tokens come from one pass over it; rows are
// brought together by a second, small kernel.
//   - A wave takes a piece of a row, batches of 64 lanes x 4 loads of 16 bytes, the next batch on its way while one is looked at.  Its k
//     best so far lie in its lanes in order (value, then index).  A new one is inserted by a ballot and a shift of the lanes; that is
//     some hundred cycles, so that few may come to it: of a run of 16 batches only the lanes' largest values are kept at first, the k-th of
//     64 lanes' largest is a limit that about k values of the run reach, and the loads that hold these are read again, out of L2 as a
//     rule.  512 rows of 131,072 bf16 with k 16: 30.7 us; with every batch looked through at once for the k best so far 39.8.
//   - The sums of exponentials are kept per lane relative to the lane's largest value: a batch in fp32, the batches in fp64 (a batch's sum
//     may be lost in a large one that was there before it; a row of a million would add that up).
// 121 MB (a tenth of the rows has ended) at 30.7 us are 3.9 TB/s: without the choice 24 us, of which the exponentials and the comparisons
// are 17 us of issue; small calls (4 rows of 32,000 fp32: 5.7 us) are bound by the way through the code.
#include "../../include/freeze.h"
#include "extents.h"
#include "freeze_internal.h"
#include "select_common.h"

#include <algorithm>

namespace fz {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef u32x4 __attribute__((aligned(1))) u32x4_any;   // loads of it need no alignment

namespace {

constexpr float kLowest = -3.402823466e38f, kLog2E = 1.44269504f;
constexpr int kBeamLoads = 4;   // loads of 16 bytes a lane has in flight
constexpr int kBeamRun = 16;    // batches that are looked through together for the best

struct BeamArgs {
    const void *logits;
    const float *scores;
    const uint8_t *finished;
    int64_t vocab, row_stride, groups_per_part;   // groups of 16 bytes in a piece of a row
    int rows, beams, k, parts, end;
    float *best_v;        // [rows, parts, k] values, best first; -inf: none
    int32_t *best_i;      // their tokens
    double *sums;         // [rows, parts] sum of exp(l - max)
    float *tops;          // [rows, parts] max; -inf: nothing
    float *out_scores;
    int32_t *out_tokens, *out_parents;
    uint8_t *out_finished;
};

// Where a continuation stands among those that are worth the same: the lower row first, in a row the larger value, then the lower token.
struct Place {
    uint64_t key;     // from the top: 6 bits of the row, 32 of the value in falling order, the token without its last 5
    uint32_t token;
    static __device__ __forceinline__ Place of(uint32_t row, float v, uint32_t token)
    {
        return Place{((uint64_t)row << 58) | ((uint64_t)~ordered_bits(v) << 26) | (token >> 5), token};   // (a token has 31 bits)
    }
    __device__ __forceinline__ uint32_t row() const { return (uint32_t)(key >> 58); }
    __device__ __forceinline__ bool operator<(const Place &o) const { return (key < o.key) | ((key == o.key) & (token < o.token)); }
};
static_assert(FREEZE_MAX_BEAMS <= 64, "a row in 6 bits");

// The wave's k best so far, one a lane, in order.
template <typename V, typename I>
struct BestList {
    V v;
    I i;
    __device__ __forceinline__ void clear(V lowest, I last) { v = lowest; i = last; }
    __device__ __forceinline__ bool before(V cv, I ci) const { return (v > cv) | ((v == cv) & (i < ci)); }
};
// the value of lane l, which is the same in all lanes
__device__ __forceinline__ uint32_t of_lane(uint32_t x, int l) { return (uint32_t)__builtin_amdgcn_readlane((int)x, l); }
__device__ __forceinline__ float of_lane(float x, int l) { return __uint_as_float(of_lane(__float_as_uint(x), l)); }
__device__ __forceinline__ uint64_t of_lane(uint64_t x, int l)
{
    return (uint64_t)of_lane((uint32_t)x, l) | ((uint64_t)of_lane((uint32_t)(x >> 32), l) << 32);
}
__device__ __forceinline__ double of_lane(double x, int l) { return __longlong_as_double((long long)of_lane((uint64_t)__double_as_longlong(x), l)); }
__device__ __forceinline__ Place of_lane(Place x, int l) { return Place{of_lane(x.key, l), of_lane(x.token, l)}; }
// the value of the lane before (lane 0: its own)
__device__ __forceinline__ uint32_t of_previous(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x138, 0xf, 0xf, false); }   // wave_shr:1
__device__ __forceinline__ float of_previous(float x) { return __uint_as_float(of_previous(__float_as_uint(x))); }
__device__ __forceinline__ uint64_t of_previous(uint64_t x)
{
    return (uint64_t)of_previous((uint32_t)x) | ((uint64_t)of_previous((uint32_t)(x >> 32)) << 32);
}
__device__ __forceinline__ double of_previous(double x) { return __longlong_as_double((long long)of_previous((uint64_t)__double_as_longlong(x))); }
__device__ __forceinline__ Place of_previous(Place x) { return Place{of_previous(x.key), of_previous(x.token)}; }

// inserts (cv, ci), the same in all lanes; false where k others are before it
template <typename V, typename I>
__device__ __forceinline__ bool insert(BestList<V, I> &list, V cv, I ci, int k, int lane)
{
    const int pos = __popcll(__ballot((lane < k) & list.before(cv, ci)));
    if (pos >= k) return false;
    const V pv = of_previous(list.v);
    const I pi = of_previous(list.i);
    if (lane > pos) {
        list.v = pv;
        list.i = pi;
    } else if (lane == pos) {
        list.v = cv;
        list.i = ci;
    }
    return true;
}

// of the lanes of `who`, how many are before this one
__device__ __forceinline__ int lanes_before(uint64_t who)
{
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
}

// A value that k lanes reach at least, cut off to the bits from LOW on of its place in order: near the k-th largest, and not above it.
template <int LOW>
__device__ __forceinline__ float kth_reached(float x, int k)
{
    const uint32_t u = ordered_bits(x);
    uint32_t t = 0;
#pragma unroll
    for (int bit = 31; bit >= LOW; --bit) {
        const uint32_t more = t | (1u << bit);
        if (__popcll(__ballot(u >= more)) >= k) t = more;   // uniform
    }
    return from_ordered_bits(t);
}

template <typename T>
__global__ __launch_bounds__(256) void beam_rows_kernel(BeamArgs p)
{
    constexpr int V = 16 / (int)sizeof(T), E = V * kBeamLoads;
    __shared__ float run_most[4][kBeamRun][64];      // a run's largest values, by batch and lane
    __shared__ uint16_t run_lane[4][128];            // (batch, lane) of those that may hold one of the best
    __shared__ float near_v[4][2 * 64 * V];          // values that may be among the best
    __shared__ uint32_t near_i[4][2 * 64 * V];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t unit = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);   // (at most 2^20 rows, or 12 pieces a CU and one a row)
    if (unit >= (uint32_t)p.rows * (uint32_t)p.parts) return;   // uniform in the wave
    const int row = (int)(unit / (uint32_t)p.parts), part = (int)(unit - (uint32_t)row * (uint32_t)p.parts);
    const T *src = static_cast<const T *>(p.logits) + (int64_t)row * p.row_stride;
    // Groups of V values from the row's first one on, wherever it lies: which values are summed together goes by their place in the row alone, so that
    // rows that are alike have the same sum to the last bit.  The row's last values, less than a group, come one by one, the
    // whole groups [g0, f1) of the piece in batches.  Of a batch that reaches past f1 the last group is loaded again and put out of the way:
    // loads that no branch decides about, so that a batch is on its way while the one before is looked at.
    const int64_t all = (p.vocab + V - 1) / V, full = p.vocab / V;
    const int64_t g0 = part * p.groups_per_part, g1 = g0 + p.groups_per_part < all ? g0 + p.groups_per_part : all;
    const int64_t f1 = g1 < full ? g1 : full;
    auto load = [&](int64_t base, u32x4(&raw)[kBeamLoads]) {   // base < f1
        const T *at = src + base * V;
        const int last = (int)(f1 - base < 64 * kBeamLoads ? f1 - base : 64 * kBeamLoads) - 1;
#pragma unroll
        for (int l = 0; l < kBeamLoads; ++l) raw[l] = *reinterpret_cast<const u32x4_any *>(at + (l * 64 + lane < last ? l * 64 + lane : last) * V);
    };
    auto value = [](const u32x4 *raw, int e) {
        const uint32_t w = raw[e / V][(e % V) * 4 / V];
        if constexpr (sizeof(T) == 4) return __uint_as_float(w);
        else return __uint_as_float(e % 2 ? w & 0xffff0000u : w << 16);
    };

    BestList<float, uint32_t> list;
    list.clear(-__builtin_inff(), ~0u);
    // what a value has to be before, or the same: the k-th best so far, or a value that k others reach
    float floor_v = kLowest;
    uint32_t floor_i = ~0u;
    auto may = [&](float v, uint32_t i) { return (v > floor_v) | ((v == floor_v) & (i <= floor_i)); };
    auto take = [&](uint64_t who, float v, uint32_t i) {   // the lanes' values
        while (who) {
            const int l = __ffsll((unsigned long long)who) - 1;
            who &= who - 1;
            const float cv = of_lane(v, l);
            const uint32_t ci = of_lane(i, l);
            if (may(cv, ci) && insert(list, cv, ci, p.k, lane)) {
                const float kv = of_lane(list.v, p.k - 1);
                if (kv >= floor_v) {
                    floor_v = kv;
                    floor_i = of_lane(list.i, p.k - 1);
                }
            }
        }
    };
    float top = -__builtin_inff();
    double sum = 0.0;   // (in fp32 a large value in front would take hundreds of batches of small ones in without a trace)
    u32x4 next[kBeamLoads];
    {
        // the values behind the whole groups
        const int64_t i = lane < V && full >= g0 && full < g1 ? full * V + lane : p.vocab;
        float x = -__builtin_inff();
        if (i < p.vocab) {
            if constexpr (sizeof(T) == 4) x = src[i];
            else x = __uint_as_float((uint32_t)src[i] << 16);
        }
        if (g0 < f1) load(g0, next);
        // (with the first loads on their way: an empty row or one that has ended has nothing to choose from)
        if (p.scores[row] == -__builtin_inff() || (p.finished && p.finished[row])) return;
        if (x >= kLowest) {
            top = x;
            sum = 1.0;
        }
        take(__ballot(x >= kLowest), x, (uint32_t)i);
    }
    // the best of the lanes' loads from group g on, those of a lane 64 groups apart
    auto scan = [&](const u32x4(&raw)[kBeamLoads], int64_t g, bool mine) {
        int near = 0;
#pragma unroll
        for (int l = 0; l < kBeamLoads; ++l) {
            const bool in = mine & (g + l * 64 < f1);
            const uint32_t i = (uint32_t)((g + l * 64) * V);
            uint64_t who[V];   // (compared all at once; equals behind the k-th best fall out below)
#pragma unroll
            for (int e = 0; e < V; ++e) who[e] = __ballot(in & (value(raw, l * V + e) >= floor_v));
#pragma unroll
            for (int e = 0; e < V; ++e) {
                if (who[e] == 0) continue;   // uniform
                if (who[e] >> lane & 1) {
                    near_v[wave][near + lanes_before(who[e])] = value(raw, l * V + e);
                    near_i[wave][near + lanes_before(who[e])] = i + e;
                }
                near += __popcll(who[e]);
            }
            if (l < kBeamLoads - 1 && near <= 64 * V) continue;   // the next load's find room
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            for (int from = 0; from < near; from += 64) {
                const bool some = from + lane < near;
                const int place = some ? from + lane : near - 1;
                const float v = near_v[wave][place];
                const uint32_t vi = near_i[wave][place];
                take(__ballot(some & may(v, vi)), v, vi);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            near = 0;
        }
    };
    // The best of a run of n batches from base on, of which `last` is the last one; most: the lane's largest value.  A limit that k values
    // reach comes from the lanes' largest ones; the batches' largest ones say then which loads to look at again.
    auto look = [&](int64_t base, int n, float most, const u32x4(&last)[kBeamLoads]) {
        const uint64_t lanes = __ballot(most >= floor_v);
        if (lanes == 0) return;   // uniform
        if (__popcll(lanes) >= p.k) {
            const float reached = kth_reached<16>(most, p.k);
            if (reached > floor_v) {
                floor_v = reached;
                floor_i = ~0u;
            }
        }
        int q = 0, held = 0;
        do {
            u32x4 raw[kBeamLoads];
            int64_t g = base + lane;
            bool mine = true;
            if (n == 1) {
#pragma unroll
                for (int l = 0; l < kBeamLoads; ++l) raw[l] = last[l];
            } else {
                for (; q < n && held < 64; ++q) {
                    const bool pass = may(run_most[wave][q][lane], (uint32_t)((base + q * (64 * kBeamLoads) + lane) * V));
                    const uint64_t who = __ballot(pass);
                    if (pass) run_lane[wave][held + lanes_before(who)] = (uint16_t)(q * 64 + lane);
                    held += __popcll(who);
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                mine = lane < held;
                const uint32_t at = mine ? run_lane[wave][lane] : 0;
                g = base + (int64_t)(at >> 6) * (64 * kBeamLoads) + (at & 63);
#pragma unroll
                for (int l = 0; l < kBeamLoads; ++l) raw[l] = *reinterpret_cast<const u32x4_any *>(src + (g + l * 64 < f1 ? g + l * 64 : f1 - 1) * V);
                held = held > 64 ? held - 64 : 0;
                if (lane < held) run_lane[wave][lane] = run_lane[wave][64 + lane];
            }
            scan(raw, g, mine);
        } while (n > 1 && (q < n || held > 0));
    };
    int in_run = 0;
    float most_run = -__builtin_inff();
    u32x4 raw[kBeamLoads];
    for (int64_t base = g0; base < f1; base += 64 * kBeamLoads) {
#pragma unroll
        for (int l = 0; l < kBeamLoads; ++l) raw[l] = next[l];
        load(base + 64 * kBeamLoads < f1 ? base + 64 * kBeamLoads : base, next);
        if (f1 - base < 64 * kBeamLoads) {   // uniform
            const int n = (int)(f1 - base);
#pragma unroll
            for (int l = 0; l < kBeamLoads; ++l)
                if (l * 64 + lane >= n) raw[l] = sizeof(T) == 4 ? u32x4{0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u} : u32x4{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u};
        }
        float most = value(raw, 0);
#pragma unroll
        for (int e = 1; e < E; ++e) most = __builtin_fmaxf(most, value(raw, e));
        run_most[wave][in_run][lane] = most;
        most_run = __builtin_fmaxf(most_run, most);
        if (most > top) {
            sum *= (double)__builtin_amdgcn_exp2f((top - most) * kLog2E);
            top = most;
        }
        if (top >= kLowest) {
            // l log2(e) - top log2(e) in one rounding, which goes by the difference; what the subtrahend lost by its own is given back to the sum:
            // half a step of it, which has to stay far below the exponents of fp32 (beyond 2^31 the powers overflow)
            const float t = top * kLog2E, lost = __builtin_fmaf(top, kLog2E, -t);
            float part_sum[2] = {0.f, 0.f};
            if (__builtin_fabsf(top) < 8388608.f) {
#pragma unroll
                for (int e = 0; e < E; ++e) part_sum[e & 1] += __builtin_amdgcn_exp2f(__builtin_fmaf(value(raw, e), kLog2E, -t));
                sum += (double)((part_sum[0] + part_sum[1]) * __builtin_amdgcn_exp2f(-lost));
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) part_sum[0] += __builtin_amdgcn_exp2f((value(raw, e) - top) * kLog2E);
                sum += (double)part_sum[0];
            }
        }
        ++in_run;
        if (in_run == kBeamRun || base + 64 * kBeamLoads >= f1) {   // uniform
            look(base - (int64_t)(in_run - 1) * (64 * kBeamLoads), in_run, most_run, raw);
            in_run = 0;
            most_run = -__builtin_inff();
        }
    }
    // the piece's sum, relative to its largest value
    float m = top;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = __builtin_fmaxf(m, __shfl_xor(m, o, 64));
    double s = top >= kLowest ? sum * (double)__builtin_amdgcn_exp2f((top - m) * kLog2E) : 0.0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if (lane == 0) {
        p.tops[unit] = m;
        p.sums[unit] = s;
    }
    if (lane < p.k) {
        p.best_v[(int64_t)unit * p.k + lane] = list.v;
        p.best_i[(int64_t)unit * p.k + lane] = (int32_t)list.i;
    }
}

// One workgroup a group: the rows' offsets score - log sum exp(l - largest l), then the k best of the pieces' lists.  What reaches the k-th largest of some
// wave's lanes' largest is gathered, as a rule a few more than k, and every one of them counts those before it; where
// too many reach it (or there are more than kMeetHeld), the waves keep lists as the pieces did.  Bound by its chain of dependent steps: one
// group of 4 rows 5.4 us, 64 groups of 8 rows 7.7 (5.2 and 7.0 with a row and a token alone to go by where totals are equal, which leaves out the
// values; 0.7 and 1.6 more with each load where its value is needed).
constexpr int kMeetThreads = 256, kMeetHeld = 4096, kMeetGathered = 512, kMeetEarly = 4;
__global__ __launch_bounds__(kMeetThreads) void beam_meet_kernel(BeamArgs p)
{
    __shared__ double off[FREEZE_MAX_BEAMS];     // score - log sum exp(l - largest l); -inf: nothing in the row
    __shared__ float largest[FREEZE_MAX_BEAMS];
    __shared__ uint8_t ended[FREEZE_MAX_BEAMS];
    __shared__ double list_v[kMeetGathered];
    __shared__ uint64_t list_key[kMeetGathered];   // (the parts of a Place)
    __shared__ uint32_t list_token[kMeetGathered];
    __shared__ double held[kMeetHeld];
    __shared__ float floors[kMeetThreads / 64];
    __shared__ int gathered;
    static_assert(kMeetThreads / 64 * FREEZE_MAX_K <= kMeetGathered, "the waves' lists");
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row0 = (int64_t)blockIdx.x * p.beams;
    if (tid == 0) gathered = 0;
    const int per_row = p.parts * p.k, all = p.beams * per_row;
    // A thread's first candidates are loaded before it is known whether their row has any, beside what tells that (an empty row's are
    // whatever the workspace held, and passed over): one round trip in the place of four.
    float early_v[kMeetEarly];
    int32_t early_i[kMeetEarly];
#pragma unroll
    for (int e = 0; e < kMeetEarly; ++e) {
        const int q = tid + e * kMeetThreads < all ? tid + e * kMeetThreads : all - 1;
        early_v[e] = p.best_v[row0 * per_row + q];
        early_i[e] = p.best_i[row0 * per_row + q];
    }
    {
        // a row for as many threads as there are for each: a power of two of them, within a wave
        int per = 64;
        while (per > 1 && kMeetThreads / per < p.beams) per >>= 1;
        const int j = tid / per, at = tid & (per - 1);
        const bool in = j < p.beams;
        const float score = in ? p.scores[row0 + j] : -__builtin_inff();
        const bool end = in && p.finished && p.finished[row0 + j];
        const bool open = !end && score > -__builtin_inff();
        const float *tops = p.tops + (row0 + (in ? j : 0)) * p.parts;
        const double *sums = p.sums + (row0 + (in ? j : 0)) * p.parts;
        const int first = at < p.parts ? at : p.parts - 1;
        const float first_top = tops[first];
        const double first_sum = sums[first];
        float m = -__builtin_inff();
        if (open)
            for (int q = at; q < p.parts; q += per) m = __builtin_fmaxf(m, q == at ? first_top : tops[q]);
        for (int x = per >> 1; x > 0; x >>= 1) m = __builtin_fmaxf(m, __shfl_xor(m, x, 64));
        double s = 0.0;
        if (open && m >= kLowest)
            for (int q = at; q < p.parts; q += per) {
                const float t = q == at ? first_top : tops[q];
                if (t >= kLowest) s += (q == at ? first_sum : sums[q]) * exp((double)t - (double)m);
            }
        for (int x = per >> 1; x > 0; x >>= 1) s += __shfl_xor(s, x, 64);
        if (in && at == 0) {
            off[j] = !open ? (double)score : (m >= kLowest ? (double)score - log(s) : -__builtin_inf());
            largest[j] = m;
            ended[j] = end;
        }
    }
    __syncthreads();
    auto put = [&](int64_t place, double v, Place i) {
        const bool some = v > -__builtin_inf();
        const int32_t token = some ? (int32_t)i.token : (p.end > 0 ? p.end : 0);
        const int64_t at = (int64_t)blockIdx.x * p.k + place;
        p.out_scores[at] = some ? (float)v : -__builtin_inff();
        p.out_tokens[at] = token;
        p.out_parents[at] = (int32_t)(row0 + (some ? (int64_t)i.row() : 0));
        if (p.out_finished) p.out_finished[at] = token == p.end;
    };
    // candidate q of the group: what it is worth (-inf: none) and its place (row, token).  (Where a row is empty or has ended, no list was written.)
    auto worth = [&](int q, float v) {
        const int j = q / per_row;
        const double o = off[j];
        if (ended[j]) return q == j * per_row ? o : -__builtin_inf();
        // (the difference first: a score beside a value far from zero would be lost, and a row of nothing but the type's lowest would be worth 0)
        return o > -__builtin_inf() && v >= kLowest ? o + ((double)v - (double)largest[j]) : -__builtin_inf();
    };
    // (totals that are equal need not have equal values: beside a score of -1e30 no value shows.  A zero counts as one, whatever its sign.)
    auto place = [&](int q, float v, int32_t i) {
        const int j = q / per_row;
        return Place::of((uint32_t)j, v + 0.f, (uint32_t)(ended[j] ? p.end : i));
    };
    const float *const best_v = p.best_v + row0 * per_row;
    const int32_t *const best_i = p.best_i + row0 * per_row;
    if (all <= kMeetHeld) {   // uniform
        double most = -__builtin_inf();
        auto hold = [&](int q, float v) {
            const double c = worth(q, v);
            held[q] = c;
            most = c > most ? c : most;
        };
#pragma unroll
        for (int e = 0; e < kMeetEarly; ++e)
            if (tid + e * kMeetThreads < all) hold(tid + e * kMeetThreads, early_v[e]);
#pragma unroll 1
        for (int q = tid + kMeetEarly * kMeetThreads; q < all; q += kMeetThreads) hold(q, best_v[q]);
        // (in fp32, one step down: what it stands for is not more than the k-th largest)
        const float kth = kth_reached<6>((float)most, p.k);
        if (lane == 0) floors[wave] = kth;
        __syncthreads();
        const float f = __builtin_fmaxf(__builtin_fmaxf(floors[0], floors[1]), __builtin_fmaxf(floors[2], floors[3]));
        const double floor_v = f > kLowest ? (double)from_ordered_bits(ordered_bits(f) - 1) : -1.7976931348623157e308;
        auto gather = [&](int q, const float *v, const int32_t *i) {
            const double c = held[q];
            if (c >= floor_v) {
                const int at = atomicAdd(&gathered, 1);   // (their order does not matter)
                if (at < kMeetGathered) {
                    const Place place_of = place(q, *v, *i);
                    list_v[at] = c;
                    list_key[at] = place_of.key;
                    list_token[at] = place_of.token;
                }
            }
        };
#pragma unroll
        for (int e = 0; e < kMeetEarly; ++e)
            if (tid + e * kMeetThreads < all) gather(tid + e * kMeetThreads, &early_v[e], &early_i[e]);
#pragma unroll 1
        for (int q = tid + kMeetEarly * kMeetThreads; q < all; q += kMeetThreads) gather(q, &best_v[q], &best_i[q]);
        __syncthreads();
        const int n = gathered;
        if (n <= kMeetGathered) {   // uniform
            for (int q = tid; q < n; q += kMeetThreads) {
                const double v = list_v[q];
                const Place i{list_key[q], list_token[q]};
                int before = 0, same = 0;
#pragma unroll 4
                for (int o = 0; o < n; ++o) {
                    before += (int)(list_v[o] > v) | ((int)(list_v[o] == v) & (int)(list_key[o] < i.key));
                    same += (int)(list_v[o] == v) & (int)(list_key[o] == i.key);
                }
                if (same > 1)   // (itself, and equal values of a row within 32 tokens)
                    for (int o = 0; o < n; ++o) before += (int)(list_v[o] == v) & (int)(list_key[o] == i.key) & (int)(list_token[o] < i.token);
                if (before < p.k) put(before, v, i);
            }
            for (int q = n + tid; q < p.k; q += kMeetThreads) put(q, -__builtin_inf(), Place{0, 0});
            return;
        }
        __syncthreads();
    }
    BestList<double, Place> list;
    list.clear(-__builtin_inf(), Place{~0ull, ~0u});
    double floor_v = -1.7976931348623157e308;
    for (int base = wave * 64; base < all; base += kMeetThreads) {
        const int q = base + lane;
        const float v = q < all ? best_v[q] : 0.f;
        const double c = q < all ? worth(q, v) : -__builtin_inf();
        const Place ci = c >= floor_v ? place(q, v, best_i[q]) : Place{0, 0};
        uint64_t who = __ballot(c >= floor_v);
        while (who) {
            const int l = __ffsll((unsigned long long)who) - 1;
            who &= who - 1;
            const double cv = of_lane(c, l);
            if (cv >= floor_v && insert(list, cv, of_lane(ci, l), p.k, lane)) {
                const double f = of_lane(list.v, p.k - 1);
                floor_v = f > floor_v ? f : floor_v;
            }
        }
    }
    if (lane < p.k) {
        list_v[wave * FREEZE_MAX_K + lane] = list.v;
        list_key[wave * FREEZE_MAX_K + lane] = list.i.key;
        list_token[wave * FREEZE_MAX_K + lane] = list.i.token;
    }
    __syncthreads();
    if (wave != 0) return;
    for (int w = 1; w < kMeetThreads / 64; ++w)
        for (int t = 0; t < p.k; ++t) {
            const double cv = list_v[w * FREEZE_MAX_K + t];
            if (!(cv > -__builtin_inf()) || !insert(list, cv, Place{list_key[w * FREEZE_MAX_K + t], list_token[w * FREEZE_MAX_K + t]}, p.k, lane)) break;   // uniform
        }
    if (lane < p.k) put(lane, list.v, list.i);
}

// How a row is cut: pieces of whole batches, as many as fill the chip with waves (12 a CU) and no more.
constexpr int64_t kBeamWaves = 12 * 256;
struct BeamPlan {
    int64_t groups_per_part;
    int parts;
};
BeamPlan beam_plan(int64_t rows, int64_t vocab, int size)
{
    const int64_t v = 16 / size, batch = 64 * kBeamLoads;
    const int64_t batches = ((vocab + v - 1) / v + batch - 1) / batch;
    int64_t parts = (kBeamWaves + rows - 1) / rows;
    parts = parts < 1 ? 1 : (parts > batches ? batches : parts);
    BeamPlan pl;
    const int64_t per = (batches + parts - 1) / parts;
    pl.groups_per_part = per * batch;
    pl.parts = (int)((batches + per - 1) / per);
    return pl;
}
// Places for the pieces' lists: as many as fewer rows may take too (a plan's own number goes up and down: 767 groups of 4 rows are cut in two, 768 not
// at all), so that a workspace serves every smaller call.
size_t beam_units(int64_t rows, int64_t vocab)
{
    const int64_t batch = 4 * 64 * kBeamLoads;   // values of a batch at least (fp32)
    return (size_t)std::min<int64_t>(rows * ((vocab + batch - 1) / batch), rows + kBeamWaves - 1);
}
size_t up256(size_t x) { return (x + 255) / 256 * 256; }

bool beam_sizes(int64_t groups, int beams, int64_t vocab, int k)
{
    return groups >= 0 && beams >= 1 && beams <= FREEZE_MAX_BEAMS && k >= 1 && k <= FREEZE_MAX_K && vocab >= 1 &&
           vocab < (int64_t)2147483647 - 512 && groups <= ((int64_t)1 << 20) / beams;
}

// ---- states -----------------------------------------------------------------------------------------

constexpr int kStatesPerLaunch = 32;   // descriptors in the kernel's arguments
struct StateRun {
    const uint8_t *src;
    uint8_t *dst;
    int64_t outer_stride, row_stride, piece_stride;
    int64_t bytes, windows;   // of a run; windows: 16-byte places of dst that a run touches, at most
    uint32_t pieces, rows;
    int64_t first;          // workgroups, or windows, of the states before this one
};
struct ReorderArgs {
    StateRun state[kStatesPerLaunch];
    const int32_t *parents;
    int64_t src_rows, total;
    int states;
};

// A run is copied by windows: the 16-byte places of dst that it touches, the first and the last in part (byte by byte).  A whole one is one
// load, aligned or not, and one aligned store.
__device__ __forceinline__ void copy_part(uint8_t *dst, const uint8_t *src, int64_t bytes, int64_t from)
{
    for (int64_t i = from < 0 ? 0 : from; i < from + 16 && i < bytes; ++i) dst[i] = src[i];
}
__device__ __forceinline__ bool run_of(const ReorderArgs &p, const StateRun &t, uint32_t run, const uint8_t **src, uint8_t **dst)
{
    const uint32_t rest = run / t.pieces, piece = run - rest * t.pieces;
    const uint32_t outer = rest / t.rows, row = rest - outer * t.rows;
    const int64_t parent = p.parents[row];
    if (parent < 0 || parent >= p.src_rows) return false;
    const int64_t place = outer * t.outer_stride + piece * t.piece_stride;
    *src = t.src + place + parent * t.row_stride;
    *dst = t.dst + place + row * t.row_stride;
    return true;
}

// Long runs: a workgroup copies kRunChunk windows of a run, four a thread on their way at once.  32 x 32 x 8 runs of 261 KB 6.2 TB/s read and
// written (a copy of 4 GiB by the runtime: 5.4).
constexpr int kRunChunk = 1024;
__global__ __launch_bounds__(256) void reorder_runs_kernel(ReorderArgs p)
{
    const int64_t block = blockIdx.x;
    int s = 0;
    while (s + 1 < p.states && block >= p.state[s + 1].first) ++s;
    const StateRun &t = p.state[s];
    const uint32_t in = (uint32_t)(block - t.first), chunks = (uint32_t)((t.windows + kRunChunk - 1) / kRunChunk);
    const uint32_t run = in / chunks, chunk = in - run * chunks;
    const uint8_t *src;
    uint8_t *dst;
    if (!run_of(p, t, run, &src, &dst)) return;   // uniform
    // byte of the run that a thread's first window starts at (before it: a window that the run begins within)
    const int64_t from = ((int64_t)chunk * kRunChunk + threadIdx.x) * 16 - (int64_t)(reinterpret_cast<uintptr_t>(dst) & 15);
    constexpr int kEach = kRunChunk / 256;
    if (from >= 0 && from + (kEach - 1) * 4096 + 16 <= t.bytes) {   // nearly all threads
        u32x4 v[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_any *>(src + from + i * 4096));
#pragma unroll
        for (int i = 0; i < kEach; ++i) __builtin_nontemporal_store(v[i], reinterpret_cast<u32x4 *>(dst + from + i * 4096));
        return;
    }
#pragma unroll 1
    for (int64_t at = from; at < t.bytes && at < from + kEach * 4096; at += 4096) {
        if (at >= 0 && at + 16 <= t.bytes) *reinterpret_cast<u32x4 *>(dst + at) = *reinterpret_cast<const u32x4_any *>(src + at);
        else copy_part(dst, src, t.bytes, at);
    }
}

// Short runs: a window a thread.  3,840 runs of 7,920 bytes (61 MB read and written, out of the caches) 14.6 us with the call, 4.2 TB/s.  Runs
// go this way where chunks of 16 KiB would be less than half full.
__global__ __launch_bounds__(256) void reorder_windows_kernel(ReorderArgs p)
{
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < p.total; u += (int64_t)gridDim.x * 256) {
        int s = 0;
        while (s + 1 < p.states && u >= p.state[s + 1].first) ++s;
        const StateRun &t = p.state[s];
        const int64_t rel = u - t.first;
        const uint32_t run = (rel | t.windows) < 0x100000000ll ? (uint32_t)rel / (uint32_t)t.windows : (uint32_t)(rel / t.windows);
        const uint8_t *src;
        uint8_t *dst;
        if (!run_of(p, t, run, &src, &dst)) continue;
        const int64_t at = (rel - run * t.windows) * 16 - (int64_t)(reinterpret_cast<uintptr_t>(dst) & 15);
        if (at >= 0 && at + 16 <= t.bytes) *reinterpret_cast<u32x4 *>(dst + at) = *reinterpret_cast<const u32x4_any *>(src + at);
        else copy_part(dst, src, t.bytes, at);
    }
}

// Whether no two runs of a state's `rows` rows share a byte: from the smallest stride on, each passes over what lies within it.
bool runs_apart(const freeze_state &t, int64_t rows)
{
    int64_t count[3] = {t.outer, rows, t.pieces}, stride[3] = {t.outer_stride, t.row_stride, t.piece_stride}, span = t.piece_bytes;
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2 - i; ++j)
            if (stride[j] > stride[j + 1]) {
                std::swap(stride[j], stride[j + 1]);
                std::swap(count[j], count[j + 1]);
            }
    for (int i = 0; i < 3; ++i) {
        if (count[i] <= 1) continue;
        if (stride[i] < span) return false;
        span += (count[i] - 1) * stride[i];
    }
    return true;
}

}  // namespace
}  // namespace fz

using namespace fz;

extern "C" {

size_t freeze_beam_workspace_bytes(int64_t groups, int beams, int64_t vocab, int k)
{
    if (!beam_sizes(groups, beams, vocab, k)) return 0;
    const int64_t rows = groups > 0 ? groups * beams : 1;
    const size_t units = beam_units(rows, vocab);
    return 2 * up256(units * k * 4) + up256(units * 8) + up256(units * 4);
}

int freeze_beam_select(const void *logits, int logits_dtype, int64_t groups, int beams, int64_t vocab, int64_t row_stride,
                       const float *scores, const uint8_t *finished, int32_t end_token, int k, float *out_scores,
                       int32_t *out_tokens, int32_t *out_parents, uint8_t *out_finished, void *workspace, size_t workspace_bytes,
                       void *stream)
{
    if (!beam_sizes(groups, beams, vocab, k) || (logits_dtype != FREEZE_F32 && logits_dtype != FREEZE_BF16) || row_stride < vocab ||
        row_stride > (int64_t)1 << 40)
        return FREEZE_EINVAL;
    if (end_token < -1 || end_token >= vocab || (finished && end_token < 0)) return FREEZE_EINVAL;
    if (groups == 0) return FREEZE_OK;
    const int size = logits_dtype == FREEZE_F32 ? 4 : 2;
    if (!logits || !scores || !out_scores || !out_tokens || !out_parents || !workspace || reinterpret_cast<uintptr_t>(logits) % size != 0)
        return FREEZE_EINVAL;
    if (workspace_bytes < freeze_beam_workspace_bytes(groups, beams, vocab, k) || reinterpret_cast<uintptr_t>(workspace) % 256 != 0)
        return FREEZE_EWORKSPACE;
    const int64_t rows = groups * beams;
    {
        Extent e[8];
        int n = 0;
        auto add = [&](const void *p, size_t bytes, bool dst) {
            const uintptr_t b = reinterpret_cast<uintptr_t>(p);
            if (p) e[n++] = Extent{b, b + bytes, dst};
            return b % 4 == 0;
        };
        const size_t places = (size_t)groups * k;
        add(logits, (size_t)((rows - 1) * row_stride + vocab) * size, false);
        add(finished, (size_t)rows, false);
        add(out_finished, places, true);
        if (!add(scores, (size_t)rows * 4, false) || !add(out_scores, places * 4, true) || !add(out_tokens, places * 4, true) ||
            !add(out_parents, places * 4, true) || !add(workspace, freeze_beam_workspace_bytes(groups, beams, vocab, k), true) || written_twice(e, n))
            return FREEZE_EINVAL;
    }
    const BeamPlan pl = beam_plan(rows, vocab, size);
    const size_t units = (size_t)rows * pl.parts;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    BeamArgs a{};
    a.logits = logits;
    a.scores = scores;
    a.finished = finished;
    a.vocab = vocab;
    a.row_stride = row_stride;
    a.groups_per_part = pl.groups_per_part;
    a.rows = (int)rows;
    a.beams = beams;
    a.k = k;
    a.parts = pl.parts;
    a.end = end_token;
    a.best_v = reinterpret_cast<float *>(ws);
    ws += up256(units * k * 4);
    a.best_i = reinterpret_cast<int32_t *>(ws);
    ws += up256(units * k * 4);
    a.sums = reinterpret_cast<double *>(ws);
    ws += up256(units * 8);
    a.tops = reinterpret_cast<float *>(ws);
    a.out_scores = out_scores;
    a.out_tokens = out_tokens;
    a.out_parents = out_parents;
    a.out_finished = out_finished;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)((units + 3) / 4));
    if (size == 4) hipLaunchKernelGGL(beam_rows_kernel<float>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(beam_rows_kernel<uint16_t>, grid, dim3(256), 0, s, a);
    if (hipGetLastError() != hipSuccess) return FREEZE_EHIP;
    hipLaunchKernelGGL(beam_meet_kernel, dim3((unsigned)groups), dim3(kMeetThreads), 0, s, a);
    return hipGetLastError() == hipSuccess ? FREEZE_OK : FREEZE_EHIP;
}

int freeze_reorder_states(const freeze_state *states, int num_states, const int32_t *parents, int64_t rows, int64_t src_rows,
                          void *stream)
{
    if (num_states < 0 || num_states > 1024 || rows < 0 || rows > (int64_t)1 << 30 || src_rows < 0 || src_rows > (int64_t)1 << 30 ||
        (num_states > 0 && !states))
        return FREEZE_EINVAL;
    // every size and stride first, then no dst over another extent
    constexpr int64_t kMost = (int64_t)1 << 46;
    Extent extents[2049];
    int n = 0;
    for (int i = 0; i < num_states; ++i) {
        const freeze_state &t = states[i];
        if (t.outer < 0 || t.pieces < 0 || t.piece_bytes < 0 || t.outer_stride < 0 || t.row_stride < 0 || t.piece_stride < 0) return FREEZE_EINVAL;
        if (t.outer > kMost || t.pieces > kMost || t.piece_bytes > kMost || t.outer_stride > kMost || t.row_stride > kMost || t.piece_stride > kMost)
            return FREEZE_EINVAL;
        if (rows == 0 || t.outer == 0 || t.pieces == 0 || t.piece_bytes == 0) continue;
        const double runs = (double)t.outer * (double)t.pieces * (double)rows;
        const double span = (double)(t.outer - 1) * (double)t.outer_stride + (double)(t.pieces - 1) * (double)t.piece_stride + (double)t.piece_bytes +
                            (double)(rows > src_rows ? rows : src_rows) * (double)t.row_stride;
        if (runs > 2147483647.0 || span > (double)kMost) return FREEZE_EINVAL;
        if (!t.src || !t.dst || !runs_apart(t, rows)) return FREEZE_EINVAL;
        const int64_t row_span = (t.outer - 1) * t.outer_stride + (t.pieces - 1) * t.piece_stride + t.piece_bytes;
        if (src_rows > 0) {
            const uintptr_t b = reinterpret_cast<uintptr_t>(t.src);
            extents[n++] = Extent{b, b + (uintptr_t)(row_span + (src_rows - 1) * t.row_stride), false};
        }
        const uintptr_t b = reinterpret_cast<uintptr_t>(t.dst);
        extents[n++] = Extent{b, b + (uintptr_t)(row_span + (rows - 1) * t.row_stride), true};
    }
    if (rows == 0 || num_states == 0) return FREEZE_OK;
    if (!parents) return FREEZE_EINVAL;
    const uintptr_t pb = reinterpret_cast<uintptr_t>(parents);
    if (pb % 4 != 0) return FREEZE_EINVAL;
    extents[n++] = Extent{pb, pb + (uintptr_t)rows * 4, false};
    if (written_twice(extents, n)) return FREEZE_EINVAL;
    for (int i = 0; i < num_states;) {
        ReorderArgs a{};
        a.parents = parents;
        a.src_rows = src_rows;
        int64_t runs[kStatesPerLaunch], blocks = 0, windows = 0;
        for (; i < num_states && a.states < kStatesPerLaunch; ++i) {
            const freeze_state &t = states[i];
            if (t.outer == 0 || t.pieces == 0 || t.piece_bytes == 0) continue;
            StateRun &r = a.state[a.states];
            r.src = static_cast<const uint8_t *>(t.src);
            r.dst = static_cast<uint8_t *>(t.dst);
            r.outer_stride = t.outer > 1 ? t.outer_stride : 0;
            r.row_stride = t.row_stride;
            r.piece_stride = t.pieces > 1 ? t.piece_stride : 0;
            r.pieces = (uint32_t)t.pieces;
            r.rows = (uint32_t)rows;
            r.bytes = t.piece_bytes;
            const bool whole = (reinterpret_cast<uintptr_t>(t.dst) | (uintptr_t)(r.outer_stride | r.row_stride | r.piece_stride | t.piece_bytes)) % 16 == 0;
            r.windows = whole ? t.piece_bytes / 16 : (t.piece_bytes + 30) / 16;
            runs[a.states] = t.outer * t.pieces * rows;
            blocks += (r.windows + kRunChunk - 1) / kRunChunk * runs[a.states];
            windows += r.windows * runs[a.states];
            ++a.states;
        }
        if (a.states == 0) continue;
        // a workgroup for each piece of a run where it has half a piece to do on average, and a grid holds them
        const bool long_runs = windows >= blocks * (kRunChunk / 2) && blocks < (1 << 23);
        for (int j = 0; j < a.states; ++j) {
            a.state[j].first = a.total;
            a.total += (long_runs ? (a.state[j].windows + kRunChunk - 1) / kRunChunk : a.state[j].windows) * runs[j];
        }
        hipStream_t s = static_cast<hipStream_t>(stream);
        const int64_t wanted = long_runs ? blocks : (windows + 255) / 256;
        const dim3 grid((unsigned)(long_runs || wanted < (1 << 20) ? wanted : (1 << 20)));
        if (long_runs) hipLaunchKernelGGL(reorder_runs_kernel, grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL(reorder_windows_kernel, grid, dim3(256), 0, s, a);
        if (hipGetLastError() != hipSuccess) return FREEZE_EHIP;
    }
    return FREEZE_OK;
}

}  // extern "C"
