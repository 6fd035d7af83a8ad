// Products of a few rows with 4-bit matrices: few_stream.h's stream, over all matrices that got a row.
//
// Bound by reading the weights of the matrices with rows once.  The rows of a segment are taken 32 at a time; what is left
// over is an entry of its own in the class of its size.  An item is an entry with a panel of 16 kCT weight rows.  There is
// one workgroup per compute unit, with an even share of the items, in one row after another: it streams on from panel to
// panel, and its wavefronts draw the panels, or parts of their reduction where there are few (few_parts).  (A workgroup per
// panel, its wavefronts a part each, had the stream empty half of the time: 203 rows of 32 matrices of 5768 x 2880 198 us.)
#include "common.h"
#include "few.h"
#include "few_stream.h"

namespace moe {

constexpr int kMvPoolFloats = 16384;
constexpr int kMvSegments = 1024; // that have lists at a time

#if defined(__HIP_DEVICE_COMPILE__)
// Entries by class: segments with rows left over (at most kFewRows; 16), and full entries, before each segment.
struct MatvecLists {
    int begin[kMvSegments + 1]; // of the segments
    int full[kMvSegments + 1];  // (more than 16 rows)
    uint16_t part[2][kMvSegments];
    int entries[3];
    int wave_full[kFewWaves], wave_part[kFewWaves];
};

// All threads: of segments [e0, e0 + E).  Offsets are taken into [0, M]; where they decrease there are no entries, so that no
// more rows are listed than there are.
template <int kForm>
__device__ __forceinline__ void matvec_lists(MatvecLists &lists, const MatvecArgs &g, int e0, int E)
{
    constexpr int kPer = kMvSegments / kFewThreads;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int full[kPer], fulls = 0, parts = 0; // parts: of class 1 above 16 bits of class 0
    int part[kPer], falls = 0;
    const int M = (int)g.M;
    auto offset = [&](int e) {
        const int m = g.seg_offsets ? g.seg_offsets[e] : e ? M : 0;
        return m < 0 ? 0 : m < M ? m : M;
    };
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int e = threadIdx.x * kPer + i;
        full[i] = part[i] = 0;
        if (e < E) {
            const int m0 = offset(e0 + e), m1 = offset(e0 + e + 1);
            falls |= m1 < m0;
            const int rows = m1 > m0 ? m1 - m0 : 0, left = rows % kFewMost;
            lists.begin[e] = m0;
            if (e == E - 1)
                lists.begin[E] = m1;
            full[i] = rows / kFewMost + (left > 16 ? 1 : 0);
            part[i] = left == 0 || left > 16 ? 0 : left <= FewForm<kForm>::kFewRows ? 1 : 1 << 16;
        }
        fulls += full[i];
        parts += part[i];
    }
    int at = -fulls, place = -parts;
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) {
        const int v = __shfl_up(fulls, s), u = __shfl_up(parts, s);
        fulls += lane >= s ? v : 0;
        parts += lane >= s ? u : 0;
    }
    if (lane == kWave - 1) {
        lists.wave_full[wave] = fulls;
        lists.wave_part[wave] = parts;
    }
    falls = __syncthreads_or(falls);
    at += fulls;
    place += parts;
    int all = 0, all_parts = 0;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
        const int v = lists.wave_full[w], u = lists.wave_part[w];
        at += w < wave ? v : 0;
        place += w < wave ? u : 0;
        all += v;
        all_parts += u;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int e = threadIdx.x * kPer + i;
        if (e < E) {
            lists.full[e] = at;
            if (part[i] == 1)
                lists.part[0][place & 0xFFFF] = (uint16_t)e;
            else if (part[i])
                lists.part[1][place >> 16] = (uint16_t)e;
        }
        at += full[i];
        place += part[i];
    }
    if (threadIdx.x == 0) {
        lists.full[E] = all;
        lists.entries[0] = falls ? 0 : all_parts & 0xFFFF;
        lists.entries[1] = falls ? 0 : all_parts >> 16;
        lists.entries[2] = falls ? 0 : all;
    }
    __syncthreads();
}

// Items [first, first + mine) of one class.
template <int kForm, int kTT, int kCT>
struct MatvecItems {
    using Form = FewForm<kForm>;
    static constexpr int kDepth = few_depth<kForm, kTT, kCT>();
    const MatvecArgs &g;
    const MatvecLists &lists;
    float *pool;
    FewRoom &room;
    int *counter;
    int e0, E, panels, first, mine, lines, parts;
    struct Unit {
        int n, part, rows, m0, n0;
    } open_unit, unit;
    bool any = false;

    __device__ MatvecItems(const MatvecArgs &g, const MatvecLists &lists, float *pool, FewRoom &room, int *counter, int e0, int E, int panels, int first, int mine)
        : g(g), lists(lists), pool(pool), room(room), counter(counter), e0(e0), E(E), panels(panels), first(first), mine(mine)
    {
        lines = (g.cols + Form::kLineCols - 1) / Form::kLineCols;
        parts = __builtin_amdgcn_readfirstlane(few_parts(mine, lines, kDepth));
    }
    __device__ __forceinline__ bool open(FewCursor<kForm, kTT, kCT, kActRows> &c)
    {
        const int u = few_draw(counter);
        if (u >= mine * parts)
            return false;
        const int n = u / parts, item = first + n, entry = item / panels;
        int e, panel, rows, m0;
        if constexpr (kTT < 2) {
            e = __builtin_amdgcn_readfirstlane(lists.part[kTT][entry]);
            panel = item - entry * panels;
            rows = (lists.begin[e + 1] - lists.begin[e]) % kFewMost;
            m0 = lists.begin[e + 1] - rows;
        } else { // the entries of a segment meet a panel one after the other
            int low = 0, high = E;
            while (high - low > 1) {
                const int mid = (low + high) / 2;
                if (lists.full[mid] <= entry)
                    low = mid;
                else
                    high = mid;
            }
            e = low;
            const int before = lists.full[e], count = lists.full[e + 1] - before, at = item - before * panels;
            panel = at / count;
            m0 = lists.begin[e] + (at - panel * count) * kFewMost;
            const int there = lists.begin[e + 1] - m0;
            rows = there < kFewMost ? there : kFewMost;
        }
        e = __builtin_amdgcn_readfirstlane(e);
        panel = __builtin_amdgcn_readfirstlane(panel);
        rows = __builtin_amdgcn_readfirstlane(rows);
        m0 = __builtin_amdgcn_readfirstlane(m0);
        open_unit = {n, u % parts, rows, m0, panel * (16 * kCT)};
        if (!any)
            unit = open_unit;
        any = true;
        const int64_t row = (int64_t)(e0 + e) * g.rows + open_unit.n0, end = (int64_t)(e0 + e + 1) * g.rows;
#pragma unroll
        for (int p = 0; p < kCT; ++p)
            c.panel[p] = panel_of<kForm>(g.w, row + 16 * p, end, g.cols, g.scale_cols);
        const uint32_t x_row = (uint32_t)g.cols * Form::kElt;
        c.set_acts({static_cast<const unsigned char *>(g.x) + (int64_t)m0 * x_row, (uint32_t)rows * x_row, 0, 0, rows},
                   [&](int r) { return r * x_row; });
        c.line = few_part_line<kForm>(lines, open_unit.part, parts);
        c.end = few_part_line<kForm>(lines, open_unit.part + 1, parts);
        c.groups = c.end > c.line ? (c.end - c.line + kDepth - 1) / kDepth : 1;
        return true;
    }
    __device__ __forceinline__ void store(int c, int v, float value) const
    {
        const int r = few_row_of<kForm, kTT>(v);
        const int n = unit.n0 + 16 * c + threadIdx.x % 16;
        const uint32_t both = pack_bf16x2(value, __shfl_xor(value, 1)); // the even lane stores both columns
        if (r < unit.rows && n < g.rows && threadIdx.x % 2 == 0)
            *reinterpret_cast<uint32_t *>(static_cast<uint16_t *>(g.y) + (int64_t)(unit.m0 + r) * g.rows + n) = both;
    }
    __device__ __forceinline__ void close(const FewSums<kForm, kTT, kCT> &sums)
    {
        constexpr int kValues = kFewValues<kForm, kTT>;
        if (parts == 1) {
#pragma unroll
            for (int c = 0; c < kCT; ++c)
#pragma unroll
                for (int v = 0; v < kValues; ++v)
                    store(c, v, sums.value(c, v));
        } else {
            FewJoin<kForm, kTT, kCT>(pool, kMvPoolFloats, room, parts).close(sums, unit.n, unit.part, [&](auto total) {
                for (int c = 0; c < kCT; ++c)
                    for (int v = 0; v < kValues; ++v)
                        store(c, v, total(c, v));
            });
        }
        unit = open_unit;
    }
};
#endif

template <int kForm, int kCT>
__global__ __launch_bounds__(kFewThreads, 2) void q4_matvec(MatvecArgs g, int E)
{
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ float pool[kMvPoolFloats];
    __shared__ MatvecLists lists;
    __shared__ FewRoom room;
    __shared__ int counter;
    const FewCols cols = {g.cols, g.scale_cols};
    const int panels = (int)((g.rows + 16 * kCT - 1) / (16 * kCT));
    for (int e0 = 0; e0 < E; e0 += kMvSegments) {
        const int segments = E - e0 < kMvSegments ? E - e0 : kMvSegments;
        matvec_lists<kForm>(lists, g, e0, segments);
        // This workgroup's share of the items: by what an item of each class takes, about.
        constexpr int kCost[3] = {4, 5, 8};
        int64_t total = 0, before = 0;
        int items[3];
#pragma unroll
        for (int c = 0; c < 3; ++c) {
            items[c] = __builtin_amdgcn_readfirstlane(lists.entries[c]) * panels;
            total += (int64_t)items[c] * kCost[c];
        }
        const int64_t from = total * blockIdx.x / gridDim.x, to = total * (blockIdx.x + 1) / gridDim.x;
        auto run = [&](auto tt, int cls) {
            constexpr int kTT = decltype(tt)::value;
            // items that begin in [from, to)
            auto at = [&](int64_t x) {
                const int64_t i = x <= before ? 0 : (x - before + kCost[cls] - 1) / kCost[cls];
                return i < items[cls] ? (int)i : items[cls];
            };
            const int first = at(from), mine = at(to) - first;
            before += (int64_t)items[cls] * kCost[cls];
            if (mine == 0)
                return;
            few_barrier();
            if (threadIdx.x == 0)
                counter = 0;
            if (threadIdx.x < 8) {
                room.parts_done[threadIdx.x] = 0;
                room.item[threadIdx.x] = threadIdx.x;
            }
            few_barrier();
            MatvecItems<kForm, kTT, kCT> part(g, lists, pool, room, &counter, e0, segments, panels, first, mine);
            few_stream<kForm, kTT, kCT, part.kDepth, kActRows>(part, cols);
        };
        run(std::integral_constant<int, 2>{}, 2);
        run(std::integral_constant<int, 1>{}, 1);
        run(std::integral_constant<int, 0>{}, 0);
        __syncthreads(); // (the lists are written again)
    }
#endif
}

template <int kForm>
static void launch(const MatvecArgs &g, int E_local, hipStream_t st)
{
    // Panels of 32 rows read the activations half as often, panels of 16 make twice as many units: 1 row of 4096 x 4096 8.4
    // (16) and 10.2 us (32), 1 of 28672 x 8192 31.5 and 31.3, 64 of 14336 x 4096 37.3 and 29.4.
    const int64_t cus = compute_units(), entries = (E_local < g.M ? E_local : g.M) + g.M / kFewMost;
    if (entries * ceil_div(g.rows, 32) < 4 * cus)
        hipLaunchKernelGGL((q4_matvec<kForm, 1>), dim3((unsigned)cus), dim3(kFewThreads), 0, st, g, E_local);
    else
        hipLaunchKernelGGL((q4_matvec<kForm, 2>), dim3((unsigned)cus), dim3(kFewThreads), 0, st, g, E_local);
}

int launch_matvec_q4(const MatvecArgs &g, int E_local, int format, hipStream_t st)
{
    if (format == MOE_Q4_FP4)
        launch<kFewFp4>(g, E_local, st);
    else if (g.group == 32)
        launch<kFewInt4By32>(g, E_local, st);
    else if (g.group == 64)
        launch<kFewInt4By64>(g, E_local, st);
    else
        launch<kFewInt4By128>(g, E_local, st);
    return check_launch("moe_matvec_q4");
}

}  // namespace moe
