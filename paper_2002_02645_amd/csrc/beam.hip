// The choice of the next tokens of a generating model's requests, and the reordering of its states (gfx950 / CDNA4).
//
// Choice.  total(j, v) = score_j + l_jv - log sum_u exp l_ju, the k best of a group's rows j and tokens v.  Within a row the
// values themselves decide, so that a row's sum of exponentials and its k best tokens come from one pass over it; rows are
// brought together by a second, small kernel.
//   - A wave takes a piece of a row, batches of 64 lanes x 4 loads of 16 bytes.  Its k best so far lie in its lanes in order
//     (value, then index), a new one is inserted by a ballot and a shuffle.  Values below the k-th best so far are passed over by one
//     comparison a batch; where k lanes or more have better ones, the k-th best of the lanes' largest raises that limit first.
//   - The sums of exponentials are kept per lane in fp32 relative to the lane's largest value (a batch at a time), joined in fp64.
#include "../../include/freeze.h"
#include "freeze_internal.h"
#include "select_common.h"

#include <algorithm>

namespace fz {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

namespace {

constexpr float kLowest = -3.402823466e38f;
constexpr int kBeamLoads = 4;   // loads of 16 bytes a lane has in flight

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

// The wave's k best so far, one a lane, in order.
template <typename V, typename I>
struct BestList {
    V v;
    I i;
    __device__ __forceinline__ void clear(V lowest) { v = lowest; i = (I)-1; }   // (unsigned: the largest index)
    __device__ __forceinline__ bool before(V cv, I ci) const { return v > cv || (v == cv && i < ci); }
};
__device__ __forceinline__ float shfl_any(float x, int l) { return __shfl(x, l, 64); }
__device__ __forceinline__ double shfl_any(double x, int l) { return __shfl(x, l, 64); }
__device__ __forceinline__ uint32_t shfl_any(uint32_t x, int l) { return (uint32_t)__shfl((int)x, l, 64); }
__device__ __forceinline__ uint64_t shfl_any(uint64_t x, int l) { return (uint64_t)__shfl((unsigned long long)x, l, 64); }

// inserts (cv, ci), the same in all lanes; false where k others are before it
template <typename V, typename I>
__device__ __forceinline__ bool insert(BestList<V, I> &list, V cv, I ci, int k, int lane)
{
    const int pos = __popcll(__ballot(lane < k && list.before(cv, ci)));
    if (pos >= k) return false;
    const V pv = shfl_any(list.v, lane > 0 ? lane - 1 : 0);
    const I pi = shfl_any(list.i, lane > 0 ? lane - 1 : 0);
    if (lane > pos) {
        list.v = pv;
        list.i = pi;
    } else if (lane == pos) {
        list.v = cv;
        list.i = ci;
    }
    return true;
}

__device__ __forceinline__ uint64_t ordered_bits64(double x)
{
    const uint64_t u = (uint64_t)__double_as_longlong(x);
    return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}
__device__ __forceinline__ double from_ordered_bits64(uint64_t u)
{
    return __longlong_as_double((long long)((u >> 63) ? (u & 0x7fffffffffffffffull) : ~u));
}

template <typename T>
__global__ __launch_bounds__(256) void beam_rows_kernel(BeamArgs p)
{
    constexpr int V = 16 / (int)sizeof(T), E = V * kBeamLoads;
    const int lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (unit >= (int64_t)p.rows * p.parts) return;   // uniform in the wave
    const int row = (int)(unit / p.parts), part = (int)(unit % p.parts);
    if (p.scores[row] == -__builtin_inff() || (p.finished && p.finished[row])) return;
    const T *src = static_cast<const T *>(p.logits) + (int64_t)row * p.row_stride;
    // groups of V values on 16-byte boundaries; the first and the last may reach over the row's ends
    const int64_t shift = (int64_t)((reinterpret_cast<uintptr_t>(src) & 15) / sizeof(T));
    const int64_t all = (p.vocab + shift + V - 1) / V;
    const int64_t g0 = part * p.groups_per_part, g1 = g0 + p.groups_per_part < all ? g0 + p.groups_per_part : all;

    BestList<float, uint32_t> list;
    list.clear(-__builtin_inff());
    float floor_v = kLowest;   // what a value has to reach
    float top = -__builtin_inff(), sum = 0.f;
    for (int64_t base = g0; base < g1; base += 64 * kBeamLoads) {
        float v[E];
#pragma unroll
        for (int l = 0; l < kBeamLoads; ++l) {
            const int64_t g = base + l * 64 + lane, at = g * V - shift;
            if (g < g1 && at >= 0 && at + V <= p.vocab) {
                const u32x4 w = *reinterpret_cast<const u32x4 *>(src + at);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (sizeof(T) == 4) {
                        v[l * V + e] = __uint_as_float(w[e]);
                    } else {
                        v[l * V + 2 * e] = __uint_as_float(w[e] << 16);
                        v[l * V + 2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    v[l * V + e] = -__builtin_inff();
                    if (g < g1 && at + e >= 0 && at + e < p.vocab) {
                        if constexpr (sizeof(T) == 4) v[l * V + e] = src[at + e];
                        else v[l * V + e] = __uint_as_float((uint32_t)src[at + e] << 16);
                    }
                }
            }
        }
        float most = v[0];
#pragma unroll
        for (int e = 1; e < E; ++e) most = __builtin_fmaxf(most, v[e]);
        if (most > top) {
            sum *= expf(top - most);
            top = most;
        }
        if (top >= kLowest) {
            float part_sum = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) part_sum += expf(v[e] - top);
            sum += part_sum;
        }
        const uint64_t lanes = __ballot(most >= floor_v);
        if (lanes == 0) continue;   // uniform
        if (__popcll(lanes) >= p.k) {
            // at least k values of this batch reach the k-th largest of the lanes' largest
            const uint32_t sorted = wave_sort32(~ordered_bits(most), lane);
            floor_v = __builtin_fmaxf(floor_v, from_ordered_bits(~(uint32_t)__shfl((int)sorted, p.k - 1, 64)));
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            uint64_t who = __ballot(v[e] >= floor_v);
            while (who) {
                const int l = __ffsll((unsigned long long)who) - 1;
                who &= who - 1;
                const float cv = __shfl(v[e], l, 64);
                const int64_t at = (base + (e / V) * 64 + l) * V - shift + e % V;
                if (cv >= floor_v && insert(list, cv, (uint32_t)at, p.k, lane))
                    floor_v = __builtin_fmaxf(floor_v, __shfl(list.v, p.k - 1, 64));
            }
        }
    }
    // the piece's sum, relative to its largest value
    float m = top;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = __builtin_fmaxf(m, __shfl_xor(m, o, 64));
    double s = top >= kLowest ? (double)sum * (double)expf(top - m) : 0.0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if (lane == 0) {
        p.tops[unit] = m;
        p.sums[unit] = s;
    }
    if (lane < p.k) {
        p.best_v[unit * p.k + lane] = list.v;
        p.best_i[unit * p.k + lane] = (int32_t)list.i;
    }
}

// One workgroup a group: the rows' offsets score - log sum exp, then the k best of the pieces' lists.
constexpr int kMeetThreads = 256;
__global__ __launch_bounds__(kMeetThreads) void beam_meet_kernel(BeamArgs p)
{
    __shared__ double off[FREEZE_MAX_BEAMS];     // -inf: nothing in the row
    __shared__ uint8_t ended[FREEZE_MAX_BEAMS];
    __shared__ double list_v[kMeetThreads / 64][FREEZE_MAX_K];
    __shared__ uint64_t list_i[kMeetThreads / 64][FREEZE_MAX_K];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row0 = (int64_t)blockIdx.x * p.beams;
    for (int j = wave; j < p.beams; j += kMeetThreads / 64) {
        const float score = p.scores[row0 + j];
        const bool end = p.finished && p.finished[row0 + j];
        double o = score;
        if (!end && score > -__builtin_inff()) {
            const float *tops = p.tops + (row0 + j) * p.parts;
            const double *sums = p.sums + (row0 + j) * p.parts;
            float m = -__builtin_inff();
            for (int q = lane; q < p.parts; q += 64) m = __builtin_fmaxf(m, tops[q]);
#pragma unroll
            for (int x = 32; x > 0; x >>= 1) m = __builtin_fmaxf(m, __shfl_xor(m, x, 64));
            double s = 0.0;
            if (m >= kLowest)
                for (int q = lane; q < p.parts; q += 64)
                    if (tops[q] >= kLowest) s += sums[q] * exp((double)tops[q] - (double)m);
#pragma unroll
            for (int x = 32; x > 0; x >>= 1) s += __shfl_xor(s, x, 64);
            o = m >= kLowest ? (double)score - (double)m - log(s) : -__builtin_inf();
        }
        if (lane == 0) {
            off[j] = o;
            ended[j] = end;
        }
    }
    __syncthreads();
    BestList<double, uint64_t> list;
    list.clear(-__builtin_inf());
    double floor_v = -1.7976931348623157e308;
    const int lists = p.beams * p.parts;
    for (int base = wave * 64; base < lists; base += kMeetThreads) {
        const int id = base + lane, j = id < lists ? id / p.parts : 0, part = id < lists ? id - j * p.parts : 0;
        const bool one = id < lists && ended[j], live = id < lists && off[j] > -__builtin_inf();
        const float *bv = p.best_v + ((row0 + j) * p.parts + part) * p.k;
        const int32_t *bi = p.best_i + ((row0 + j) * p.parts + part) * p.k;
        for (int t = 0; t < p.k; ++t) {   // the lists are in order: depth by depth
            double c = -__builtin_inf();
            uint64_t ci = ~0ull;
            if (live && one) {
                if (t == 0 && part == 0) {
                    c = off[j];
                    ci = ((uint64_t)j << 32) | (uint32_t)p.end;
                }
            } else if (live && bv[t] >= kLowest) {
                c = off[j] + (double)bv[t];
                ci = ((uint64_t)j << 32) | (uint32_t)bi[t];
            }
            uint64_t who = __ballot(c >= floor_v);
            if (who == 0) break;   // uniform
            if (t == 0 && __popcll(who) >= p.k) {
                const uint64_t sorted = wave_sort64(~ordered_bits64(c), lane);
                const double f = from_ordered_bits64(~shfl_any(sorted, p.k - 1));
                floor_v = f > floor_v ? f : floor_v;
                who = __ballot(c >= floor_v);
            }
            while (who) {
                const int l = __ffsll((unsigned long long)who) - 1;
                who &= who - 1;
                const double cv = shfl_any(c, l);
                if (cv >= floor_v && insert(list, cv, shfl_any(ci, l), p.k, lane)) {
                    const double f = shfl_any(list.v, p.k - 1);
                    floor_v = f > floor_v ? f : floor_v;
                }
            }
        }
    }
    if (lane < p.k) {
        list_v[wave][lane] = list.v;
        list_i[wave][lane] = list.i;
    }
    __syncthreads();
    if (wave != 0) return;
    for (int w = 1; w < kMeetThreads / 64; ++w)
        for (int t = 0; t < p.k; ++t) {
            const double cv = list_v[w][t];
            if (!(cv > -__builtin_inf()) || !insert(list, cv, list_i[w][t], p.k, lane)) break;   // uniform
        }
    if (lane < p.k) {
        const int64_t at = (int64_t)blockIdx.x * p.k + lane;
        const bool some = list.v > -__builtin_inf();
        const int32_t token = some ? (int32_t)(uint32_t)list.i : (p.end > 0 ? p.end : 0);
        p.out_scores[at] = some ? (float)list.v : -__builtin_inff();
        p.out_tokens[at] = token;
        p.out_parents[at] = (int32_t)(row0 + (some ? (int64_t)(list.i >> 32) : 0));
        if (p.out_finished) p.out_finished[at] = token == p.end;
    }
}

// How a row is cut: pieces of whole batches, as many as fill the chip with waves (16 a CU) and no more.
struct BeamPlan {
    int64_t groups_per_part;
    int parts;
};
BeamPlan beam_plan(int64_t rows, int64_t vocab, int size)
{
    const int64_t v = 16 / size, batch = 64 * kBeamLoads;
    const int64_t batches = ((vocab + v - 1 + v - 1) / v + batch - 1) / batch;   // (a misaligned row's groups are one more)
    int64_t parts = (4096 + rows - 1) / rows;
    parts = parts < 1 ? 1 : (parts > batches ? batches : parts);
    BeamPlan pl;
    const int64_t per = (batches + parts - 1) / parts;
    pl.groups_per_part = per * batch;
    pl.parts = (int)((batches + per - 1) / per);
    return pl;
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
    int64_t per_run;        // units of a run
    uint32_t pieces, rows;
    int64_t first;          // units of the states before this one
};
struct ReorderArgs {
    StateRun state[kStatesPerLaunch];
    const int32_t *parents;
    int64_t src_rows, total;
    int states;
};

template <typename U>
__global__ __launch_bounds__(256) void reorder_kernel(ReorderArgs p)
{
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < p.total; u += (int64_t)gridDim.x * 256) {
        int s = 0;
        while (s + 1 < p.states && u >= p.state[s + 1].first) ++s;
        const StateRun &t = p.state[s];
        const int64_t run = (u - t.first) / t.per_run, at = (u - t.first) - run * t.per_run;
        const uint32_t piece = (uint32_t)(run % t.pieces);
        const int64_t rest = run / t.pieces;
        const int64_t row = rest % t.rows, outer = rest / t.rows;
        const int64_t parent = p.parents[row];
        if (parent < 0 || parent >= p.src_rows) continue;
        const int64_t place = outer * t.outer_stride + piece * t.piece_stride + at * (int64_t)sizeof(U);
        *reinterpret_cast<U *>(t.dst + place + row * t.row_stride) = *reinterpret_cast<const U *>(t.src + place + parent * t.row_stride);
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

struct Extent {
    uintptr_t begin, end;
    bool dst;
};

}  // namespace
}  // namespace fz

using namespace fz;

extern "C" {

size_t freeze_beam_workspace_bytes(int64_t groups, int beams, int64_t vocab, int k)
{
    if (!beam_sizes(groups, beams, vocab, k)) return 0;
    const int64_t rows = groups > 0 ? groups * beams : 1;
    const size_t units = (size_t)rows * std::max(beam_plan(rows, vocab, 4).parts, beam_plan(rows, vocab, 2).parts);
    return 2 * up256(units * k * 4) + up256(units * 8) + up256(units * 4);
}

int freeze_beam_select(const void *logits, int logits_dtype, int64_t groups, int beams, int64_t vocab, int64_t row_stride,
                       const float *scores, const uint8_t *finished, int32_t end_token, int k, float *out_scores,
                       int32_t *out_tokens, int32_t *out_parents, uint8_t *out_finished, void *workspace, size_t workspace_bytes,
                       void *stream)
{
    if (!beam_sizes(groups, beams, vocab, k) || (logits_dtype != FREEZE_F32 && logits_dtype != FREEZE_BF16) || row_stride < vocab)
        return FREEZE_EINVAL;
    if (end_token < -1 || end_token >= vocab || (finished && end_token < 0)) return FREEZE_EINVAL;
    if (groups == 0) return FREEZE_OK;
    const int size = logits_dtype == FREEZE_F32 ? 4 : 2;
    if (!logits || !scores || !out_scores || !out_tokens || !out_parents || !workspace || reinterpret_cast<uintptr_t>(logits) % size != 0)
        return FREEZE_EINVAL;
    if (workspace_bytes < freeze_beam_workspace_bytes(groups, beams, vocab, k) || reinterpret_cast<uintptr_t>(workspace) % 256 != 0)
        return FREEZE_EWORKSPACE;
    const int64_t rows = groups * beams;
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
    Extent extents[2048];
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
    std::sort(extents, extents + n, [](const Extent &a, const Extent &b) { return a.begin < b.begin; });
    uintptr_t any_end = 0, dst_end = 0;   // how far the extents so far reach
    for (int i = 0; i < n; ++i) {
        if (extents[i].begin < (extents[i].dst ? any_end : dst_end)) return FREEZE_EINVAL;
        any_end = std::max(any_end, extents[i].end);
        if (extents[i].dst) dst_end = std::max(dst_end, extents[i].end);
    }
    for (int i = 0; i < num_states;) {
        ReorderArgs a{};
        a.parents = parents;
        a.src_rows = src_rows;
        uintptr_t bits = 0;
        int64_t runs[kStatesPerLaunch];
        for (; i < num_states && a.states < kStatesPerLaunch; ++i) {
            const freeze_state &t = states[i];
            if (t.outer == 0 || t.pieces == 0 || t.piece_bytes == 0) continue;
            runs[a.states] = t.outer * t.pieces * rows;
            StateRun &r = a.state[a.states++];
            r.src = static_cast<const uint8_t *>(t.src);
            r.dst = static_cast<uint8_t *>(t.dst);
            r.outer_stride = t.outer > 1 ? t.outer_stride : 0;
            r.row_stride = t.row_stride;
            r.piece_stride = t.pieces > 1 ? t.piece_stride : 0;
            r.per_run = t.piece_bytes;
            r.pieces = (uint32_t)t.pieces;
            r.rows = (uint32_t)rows;
            bits |= reinterpret_cast<uintptr_t>(t.src) | reinterpret_cast<uintptr_t>(t.dst) |
                    (uintptr_t)(r.outer_stride | r.row_stride | r.piece_stride | t.piece_bytes);
        }
        if (a.states == 0) continue;
        const int unit = bits % 16 == 0 ? 16 : (bits % 4 == 0 ? 4 : 1);
        for (int j = 0; j < a.states; ++j) {
            a.state[j].per_run /= unit;
            a.state[j].first = a.total;
            a.total += a.state[j].per_run * runs[j];
        }
        const int64_t blocks = (a.total + 255) / 256;
        const dim3 grid((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20)));
        hipStream_t s = static_cast<hipStream_t>(stream);
        if (unit == 16) hipLaunchKernelGGL(reorder_kernel<u32x4>, grid, dim3(256), 0, s, a);
        else if (unit == 4) hipLaunchKernelGGL(reorder_kernel<uint32_t>, grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL(reorder_kernel<uint8_t>, grid, dim3(256), 0, s, a);
        if (hipGetLastError() != hipSuccess) return FREEZE_EHIP;
    }
    return FREEZE_OK;
}

}  // extern "C"
