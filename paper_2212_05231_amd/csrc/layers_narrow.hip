// The backward pass of narrow grouped layers (up to 64 inputs and 64 outputs, the framework's own widths) in one pass over the rows:
// dx = W^T dy and dW = sum dy x^T.  Apart, the two read dy twice and are bound by that; together they read dy and x once and write dx.
#include "layers.h"

namespace neus2 {
namespace {

struct NarrowArgs {
    RowsArgs rows;                   // x: dy, y: dx (NULL: not wanted)
    const void* x; const uint8_t* e; int64_t x_stride; int x_whole;      // the layer's input
    int inner, outer;
    float* partial;                  // [workgroups + groups][outer][inner]
};

constexpr int kWaves = 8, kUnit = 32;          // rows a wave takes at a time

// A workgroup takes a run of consecutive units of 32 rows, group after group: the group's matrix goes to LDS, split once; a wave
// has every eighth unit, whose values go from memory to registers as the products want them (lane = row), the next one's under way
// while this one's products run.  For dW the rows are the contraction: the terms of dy, then those of x, go through the wave's part
// of LDS and come back transposed.  The sums over a run's part of a group are joined over the waves and stored as partial number
// workgroup + group (both only ever grow along the runs, so no two parts have the same number); run_join_kernel adds them in order.
template <int DT, bool PACKED, bool ONCE>
__global__ __launch_bounds__(64 * kWaves, 2) void narrow_backward_kernel(NarrowArgs b) {
    typedef typename TypeOf<DT>::Element E;
    typedef std::conditional_t<DT == kTypeF32, Wide<3>, Native> Factor;
    typedef std::conditional_t<PACKED, Packed<DT == kTypeF16>, Factor> InputFactor;
    constexpr int kTerms = Factor::kTerms, kInputTerms = InputFactor::kTerms, kSteps = 4;
    constexpr bool kHalf = DT == kTypeF16;
    typedef FactorTile<Factor, false, 64, 64, 64 * kWaves> MatrixTile;
    typedef FactorTile<Factor, false, 64, kUnit, 64> DyTile;             // [row][64 values]: rows are the steps
    typedef FactorTile<InputFactor, false, 64, kUnit, 64> InputTile;
    constexpr int kPlanes = DyTile::kBytes > InputTile::kBytes ? DyTile::kBytes : InputTile::kBytes;
    static_assert(kPlanes >= 4096, "the sums of a block of 32 x 32 pass through it");
    __shared__ __attribute__((aligned(16))) unsigned char matrix[MatrixTile::kBytes], planes[kWaves * kPlanes], stage[kWaves * 4096];

    const RowsArgs& a = b.rows;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int j = lane & 31, h = lane >> 5;
    unsigned char* mine = planes + wave * kPlanes;
    const int64_t total = count_tiles(a.groups, kUnit, 0, lane);
    const int first = (int)(total * blockIdx.x / gridDim.x), end = (int)(total * (blockIdx.x + 1) / gridDim.x);

    typename Factor::Pointer dy, source;
    dy.p = reinterpret_cast<decltype(dy.p)>(a.x);
    dy.stride = a.x_stride;
    dy.whole = 1;
    source.stride = a.w_stride;
    source.whole = a.w_whole;
    typename InputFactor::Pointer input;
    input.p = reinterpret_cast<decltype(input.p)>(b.x);
    if constexpr (PACKED) input.e = b.e;
    input.stride = b.x_stride;
    input.whole = 1;
    typename Factor::Raw d_raw[kSteps];
    typename InputFactor::Raw x_raw[kSteps];
    auto dy_window = [&](int lo, int hi) { return Factor::window(dy, lo, 0, min(kUnit, hi - lo), b.outer); };
    auto request_dy = [&](const typename Factor::Window& w, int rows, int ks) {
        d_raw[ks] = Factor::fetch(w, j, 16 * ks + 8 * h, j < rows && 16 * ks + 8 * h < b.outer);
    };
    auto request_x = [&](int lo, int hi) {
        const int rows = min(kUnit, hi - lo);
        const typename InputFactor::Window w = InputFactor::window(input, lo, 0, rows, b.inner);
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) x_raw[ks] = InputFactor::fetch(w, j, 16 * ks + 8 * h, j < rows && 16 * ks + 8 * h < b.inner);
    };

    for (int unit = first; unit < end;) {
        const RowTile t = locate(a.groups, kUnit, 0, unit, lane);
        const int group_lo = t.lo - kUnit * t.part, stop = min(end, t.index + t.parts);
        if (a.y) {
            source.p = reinterpret_cast<decltype(source.p)>(a.w) + (int64_t)t.group * a.w_group;
            MatrixTile m;
            m.load(source, 0, b.inner, 0, b.outer, tid);
            m.store(matrix, tid);
        }
        __syncthreads();
        v16f sums[2][2];
#pragma unroll
        for (int o = 0; o < 2; ++o)
#pragma unroll
            for (int i = 0; i < 2; ++i) sums[o][i] = zero16();
        int at = unit + wave;
        if (at < stop) {
            const int lo = group_lo + kUnit * (at - t.index);
            const typename Factor::Window w = dy_window(lo, t.end);
#pragma unroll
            for (int ks = 0; ks < kSteps; ++ks) request_dy(w, min(kUnit, t.end - lo), ks);
            request_x(lo, t.end);
        }
        for (; at < stop; at += kWaves) {
            RowTile now = t;
            now.lo = group_lo + kUnit * (at - t.index);
            now.hi = min(now.lo + kUnit, t.end);
            // what is fetched for the next unit takes the place of what has just been used
            const bool more = at + kWaves < stop;
            const int next = now.lo + kWaves * kUnit;
            const typename Factor::Window next_dy = dy_window(more ? next : now.lo, t.end);
            v16f acc[2];
            acc[0] = zero16();
            acc[1] = zero16();
#pragma unroll
            for (int ks = 0; ks < kSteps; ++ks) {
                u32x4 d[kTerms];
                Factor::terms(d_raw[ks], d);
                if (more) request_dy(next_dy, min(kUnit, t.end - next), ks);
#pragma unroll
                for (int p = 0; p < kTerms; ++p)
                    *reinterpret_cast<u32x4*>(mine + p * DyTile::kPlane + j * 128 + (((2 * ks + h) ^ DyTile::across(j)) << 4)) = d[p];
                if (a.y) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        u32x4 m[kTerms];
#pragma unroll
                        for (int p = 0; p < kTerms; ++p) m[p] = MatrixTile::operand(matrix, p, c, ks, lane);
                        acc[c] = mma_terms<kHalf>(m, d, acc[c]);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (a.y) {
                if constexpr (sizeof(E) == 4) {
                    v16f half[1][1];
                    half[0][0] = acc[0];
                    finish_rows<DT, true, false, 1, 1, ONCE>(a, now, {}, 0, 0, half, stage, wave, lane, [] {});
                    half[0][0] = acc[1];
                    if (a.cols > 32) finish_rows<DT, true, false, 1, 1, ONCE>(a, now, {}, 32, 0, half, stage, wave, lane, [] {});
                } else {
                    v16f both[2][1];
                    both[0][0] = acc[0];
                    both[1][0] = acc[1];
                    finish_rows<DT, true, false, 2, 1, ONCE>(a, now, {}, 0, 0, both, stage, wave, lane, [] {});
                }
            }
            wave_lds_fence();
            u32x4 l[2][2][kTerms];
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int o = 0; o < 2; ++o)
#pragma unroll
                    for (int p = 0; p < kTerms; ++p) l[k][o][p] = DyTile::operand(mine, p, o, k, lane);
            wave_lds_fence();
#pragma unroll
            for (int ks = 0; ks < kSteps; ++ks) {
                u32x4 x[kInputTerms];
                InputFactor::terms(x_raw[ks], x);
#pragma unroll
                for (int p = 0; p < kInputTerms; ++p)
                    *reinterpret_cast<u32x4*>(mine + p * InputTile::kPlane + j * 128 + (((2 * ks + h) ^ InputTile::across(j)) << 4)) = x[p];
            }
            wave_lds_fence();
#pragma unroll
            for (int k = 0; k < 2; ++k) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    u32x4 r[kInputTerms];
#pragma unroll
                    for (int p = 0; p < kInputTerms; ++p) r[p] = InputTile::operand(mine, p, i, k, lane);
#pragma unroll
                    for (int o = 0; o < 2; ++o) sums[o][i] = mma_terms<kHalf>(l[k][o], r, sums[o][i]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (more) request_x(next, t.end);
            wave_lds_fence();
        }
        // the waves' sums, block after block of 32 x 32
        float* out = b.partial + (int64_t)(blockIdx.x + t.group) * b.outer * b.inner;
        float* scratch = reinterpret_cast<float*>(planes);
        __syncthreads();                                                 // the matrix and every wave's planes are free
#pragma unroll
        for (int o = 0; o < 2; ++o)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int r = 0; r < 16; ++r) scratch[wave * 1024 + r * 64 + lane] = sums[o][i][r];
                __syncthreads();
#pragma unroll
                for (int q = 0; q < 1024 / (64 * kWaves); ++q) {
                    const int element = tid + q * 64 * kWaves, l = element & 63;
                    float z = 0.f;
#pragma unroll
                    for (int w = 0; w < kWaves; ++w) z += scratch[w * 1024 + element];
                    const int row = 32 * o + neuron_of(element >> 6, l >> 5), col = 32 * i + (l & 31);
                    if (row < b.outer && col < b.inner) out[row * b.inner + col] = z;
                }
                __syncthreads();
            }
        unit = stop;
    }
}

// dW_g (+)= the partials of group g in the order of the runs.  One workgroup for 256 elements of one matrix, four waves.
__global__ __launch_bounds__(256) void run_join_kernel(RowGroups groups, int runs, int size, int blocks, const float* __restrict__ partial,
                                                       float* __restrict__ dW, int accumulate) {
    __shared__ v4f sums[4][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group = (int)(blockIdx.x / blocks), first = (int)(blockIdx.x % blocks) * 256 + 4 * lane;
    const int count = groups.offsets ? groups.groups : 1;
    const int64_t total = count_tiles(groups, kUnit, 0, lane);
    int64_t before = 0;
    int mine = 0;                                                        // units before the group's first one, and its own
    for (int base = 0; base <= group; base += 64) {
        const int e = base + lane;
        int lo = 0, hi = 0, units = 0;
        if (e < count) {
            group_rows(groups, e, lo, hi);
            units = (hi - lo + kUnit - 1) / kUnit;
        }
        const int sum = wave_sums(units, lane);
        if (group < base + 64) {
            mine = __builtin_amdgcn_readlane(units, group - base);
            before += __builtin_amdgcn_readlane(sum, group - base) - mine;
        } else {
            before += __builtin_amdgcn_readlane(sum, 63);
        }
    }
    v4f sum = {0.f, 0.f, 0.f, 0.f};
    if (mine > 0 && total > 0) {
        // the last run that begins at or before a unit: run r begins at total * r / runs (rounded down)
        const int64_t from = ((before + 1) * runs - 1) / total, to = min(((before + mine) * runs - 1) / total, (int64_t)runs - 1);
        for (int64_t run = from + wave; run <= to; run += 4) {
            const int64_t begin = total * run / runs, end = total * (run + 1) / runs;
            if (max(begin, before) >= min(end, before + mine)) continue;     // a run without units
            const float* src = partial + (run + group) * size + first;
            if (size % 4 == 0) {
                if (first < size) sum += *reinterpret_cast<const v4f*>(src);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (first + e < size) sum[e] += src[e];
            }
        }
    }
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave != 0 || (mine == 0 && accumulate)) return;
    const v4f z = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
    float* out = dW + (int64_t)group * size + first;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (first + e < size) out[e] = accumulate ? out[e] + z[e] : z[e];
}

template <int DT>
void launch(const NarrowArgs& b, bool packed, unsigned grid, hipStream_t st) {
    auto go = [&](auto* plain, auto* once) { (b.rows.once ? once : plain)<<<grid, 64 * kWaves, 0, st>>>(b); };
    if (packed) go(narrow_backward_kernel<DT, true, false>, narrow_backward_kernel<DT, true, true>);
    else if constexpr (DT != kTypeF32) go(narrow_backward_kernel<DT, false, false>, narrow_backward_kernel<DT, false, true>);
}

}  // namespace

// A unit of 32 rows of the smallest groups must not be mostly empty, and a run must be worth a workgroup's matrix and sums: layers
// of 64 to 64, fp32 with inputs in 8 bits, 20 groups, three of them with 2^15 rows 70.5 us against 68.5 apart; one with 2^16 29 against 31,
// 2^17 36 against 40, 2^18 46 against 55, 2^20 139 against 219.  fp32 inputs in full take three terms more than there are registers for.
bool narrow_backward_fits(int dtype, int inner, int outer, int64_t groups, int64_t n, int64_t dy_stride, int64_t x_stride, bool packed) {
    return inner <= 64 && outer <= 64 && n >= 64 * groups && n >= (1 << 16) && (packed || dtype != kTypeF32) && rows_whole(dtype, dy_stride, outer) && rows_whole(dtype, inner, inner) &&
           (packed || rows_whole(dtype, x_stride, inner));
}

int64_t narrow_backward_bytes(int inner, int outer, int64_t groups) { return (compute_units() + groups) * inner * outer * 4; }

int launch_narrow_backward(int dtype, const RowsArgs& rows, const MatrixGradient& m, hipStream_t st) {
    NarrowArgs b = {};
    b.rows = rows;
    b.x = m.xq ? (const void*)m.xq : m.x;
    b.e = m.xe;
    b.x_stride = m.xq ? (m.inner + 31) / 32 * 32 : m.x_stride;
    b.inner = m.inner;
    b.outer = m.outer;
    b.partial = m.partial;
    const int runs = compute_units();
    if (dtype == kTypeF32) launch<kTypeF32>(b, m.xq != nullptr, (unsigned)runs, st);
    else if (dtype == kTypeF16) launch<kTypeF16>(b, m.xq != nullptr, (unsigned)runs, st);
    else launch<kTypeBF16>(b, m.xq != nullptr, (unsigned)runs, st);
    NEUS2_TRY(check_launch("narrow layer backward"));
    const int size = m.inner * m.outer, blocks = (size + 255) / 256;
    const int64_t joins = (int64_t)(m.groups.offsets ? m.groups.groups : 1) * blocks;
    run_join_kernel<<<(unsigned)joins, 256, 0, st>>>(m.groups, runs, size, blocks, m.partial, m.out, m.accumulate);
    return check_launch("narrow layer backward sums");
}

}  // namespace neus2
