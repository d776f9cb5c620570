// Gradients of the matrices of layers whose rows choose them: dW_g = sum over the rows i of group g of dy_i x_i^T, and the same
// sums for the two narrow matrices of adapters.
//
// The contraction runs over the rows, along which neither factor is contiguous: tiles go to LDS as they lie in memory and come
// back through the transposing LDS read.  A group's rows are cut into chunks where there are too few tiles of the matrix to fill
// the chip; the chunks' sums go to a workspace and are added in order, so the result does not depend on which finished first.
#include "layers.h"

namespace neus2 {
namespace {

struct SumArgs {
    RowGroups groups;
    int chunk;                       // rows a workgroup sums over
    const void* left; int64_t left_stride; int left_vec;
    const void* right; const uint8_t* right_e; int64_t right_stride; int right_vec;
    int outer, inner;
    float* out; int accumulate;
    float* partial;                  // [chunks][outer][inner]
    int always_partial;
    int outer_tiles, inner_tiles;
};

template <class Factor>
__device__ __forceinline__ typename Factor::Pointer make_pointer(const void* p, const uint8_t* e, int64_t stride, int vec) {
    typename Factor::Pointer f;
    f.p = reinterpret_cast<decltype(f.p)>(p);
    f.stride = stride;
    if constexpr (std::is_same_v<Factor, Packed<false>> || std::is_same_v<Factor, Packed<true>>) f.e = e;
    else f.vec = vec;
    return f;
}

template <class Left, class Right, bool HALF, int OUTER, int INNER, int DEPTH, int BUFS>
__global__ __launch_bounds__(256) void matrix_sums_kernel(SumArgs a) {
    constexpr int kThreads = 256;
    constexpr int kBO = OUTER / 64, kBI = INNER / 64;            // four waves, two by two
    typedef FactorTile<Left, false, OUTER, DEPTH, kThreads> LeftTile;
    typedef FactorTile<Right, false, INNER, DEPTH, kThreads> RightTile;
    constexpr int kBuf = LeftTile::kBytes + RightTile::kBytes;
    __shared__ __attribute__((aligned(16))) unsigned char lds[BUFS * kBuf];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wo = wave >> 1, wi = wave & 1;
    const int tiles = a.outer_tiles * a.inner_tiles;
    const int tile = (int)(blockIdx.x % tiles);
    const int outer0 = tile / a.inner_tiles * OUTER, inner0 = tile % a.inner_tiles * INNER;
    const RowTile t = locate(a.groups, a.chunk, 1, (int)(blockIdx.x / tiles), lane);
    if (t.group < 0) return;

    const typename Left::Pointer left = make_pointer<Left>(a.left, nullptr, a.left_stride, a.left_vec);
    const typename Right::Pointer right = make_pointer<Right>(a.right, a.right_e, a.right_stride, a.right_vec);
    LeftTile lt;
    RightTile rt;
    v16f acc[kBO][kBI];
#pragma unroll
    for (int o = 0; o < kBO; ++o)
#pragma unroll
        for (int i = 0; i < kBI; ++i) acc[o][i] = zero16();
    const int rows = t.hi - t.lo, rounds = (rows + DEPTH - 1) / DEPTH;
    if (rounds > 0) {
        lt.load(left, outer0, a.outer - outer0, t.lo, rows, tid);
        rt.load(right, inner0, a.inner - inner0, t.lo, rows, tid);
        lt.store(lds, tid);
        rt.store(lds + LeftTile::kBytes, tid);
        __syncthreads();
    }
    for (int k = 0; k < rounds; ++k) {
        const unsigned char* buf = lds + (BUFS == 2 ? (k & 1) * kBuf : 0);
        const bool more = k + 1 < rounds;
        if (more) {
            const int step = (k + 1) * DEPTH;
            lt.load(left, outer0, a.outer - outer0, (int64_t)t.lo + step, rows - step, tid);
            rt.load(right, inner0, a.inner - inner0, (int64_t)t.lo + step, rows - step, tid);
        }
#pragma unroll
        for (int ks = 0; ks < DEPTH / 16; ++ks) {
            u32x4 l[kBO][Left::kTerms], r[kBI][Right::kTerms];
#pragma unroll
            for (int o = 0; o < kBO; ++o)
#pragma unroll
                for (int p = 0; p < Left::kTerms; ++p) l[o][p] = LeftTile::operand(buf, p, wo * kBO + o, ks, lane);
#pragma unroll
            for (int i = 0; i < kBI; ++i)
#pragma unroll
                for (int p = 0; p < Right::kTerms; ++p) r[i][p] = RightTile::operand(buf + LeftTile::kBytes, p, wi * kBI + i, ks, lane);
#pragma unroll
            for (int o = 0; o < kBO; ++o)
#pragma unroll
                for (int i = 0; i < kBI; ++i) acc[o][i] = mma_terms<HALF>(l[o], r[i], acc[o][i]);
        }
        if (BUFS == 1) __syncthreads();
        if (more) {
            unsigned char* next = lds + (BUFS == 2 ? ((k + 1) & 1) * kBuf : 0);
            lt.store(next, tid);
            rt.store(next + LeftTile::kBytes, tid);
        }
        __syncthreads();
    }

    const bool direct = !a.always_partial && t.parts == 1;
    if (!direct && rows == 0) return;
    const int64_t size = (int64_t)a.outer * a.inner;
    float* out = direct ? a.out + t.group * size : a.partial + (int64_t)(t.index + t.part) * size;
    const bool add = direct && a.accumulate;
    const int j = lane & 31, h = lane >> 5;
#pragma unroll
    for (int i = 0; i < kBI; ++i) {
        const int col = inner0 + 32 * (wi * kBI + i) + j;
        if (col >= a.inner) continue;
#pragma unroll
        for (int o = 0; o < kBO; ++o)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = outer0 + 32 * (wo * kBO + o) + neuron_of(r, h);
                if (row >= a.outer) continue;
                float* p = out + (int64_t)row * a.inner + col;
                const float v = acc[o][i][r];
                *p = add ? *p + v : v;
            }
    }
}

// Adds the chunks' sums in the order of their rows.  One workgroup for 1024 elements of one matrix.
struct JoinArgs {
    RowGroups groups;
    int chunk;
    int64_t size;                    // elements of a matrix
    int blocks;                      // workgroups a matrix
    const float* partial; int chunks;
    float* out; int accumulate;
    int by_slot; const int32_t* slots; int n_slots;
};

__global__ __launch_bounds__(256) void join_sums_kernel(JoinArgs a) {
    const int lane = threadIdx.x & 63;
    const int matrix = (int)(blockIdx.x / a.blocks);
    const int64_t first = (int64_t)(blockIdx.x % a.blocks) * 1024 + threadIdx.x;
    const int groups = a.groups.offsets ? a.groups.groups : 1;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    auto add_parts = [&](int index, int parts) {
        for (int p = 0; p < parts && index + p < a.chunks; ++p) {          // decreasing offsets may count more than there are
            const float* src = a.partial + (int64_t)(index + p) * a.size + first;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (first + 256 * q < a.size) sum[q] += src[256 * q];
        }
    };
    bool mine = a.by_slot != 0;
    int before = 0;
    for (int base = 0; base < groups; base += 64) {
        const int e = base + lane;
        int lo = 0, hi = 0, tiles = 0;
        if (e < groups) {
            group_rows(a.groups, e, lo, hi);
            tiles = max((hi - lo + a.chunk - 1) / a.chunk, 1);
        }
        int end = tiles;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int up = __shfl_up(end, d);
            if (lane >= d) end += up;
        }
        bool match = e < groups && hi > lo && e == matrix && tiles > 1;          // one chunk: stored where it belongs already
        if (a.by_slot) match = e < groups && hi > lo && slot_of(a.slots, a.n_slots, e) == matrix;
        uint64_t set = __ballot(match);
        while (set) {
            const int at = __builtin_ctzll(set);
            set &= set - 1;
            const int parts = __builtin_amdgcn_readlane(tiles, at);
            add_parts(before + __builtin_amdgcn_readlane(end, at) - parts, parts);
            mine = true;
        }
        before += __builtin_amdgcn_readlane(end, 63);
        if (!a.by_slot && matrix < base + 64) break;
    }
    if (!mine) return;
    float* out = a.out + (int64_t)matrix * a.size + first;
#pragma unroll
    for (int q = 0; q < 4; ++q)
        if (first + 256 * q < a.size) out[256 * q] = a.accumulate ? out[256 * q] + sum[q] : sum[q];
}

// ---- how the work is cut --------------------------------------------------------------------------------------------------------
int tile_of(int dim) { return dim > 64 ? 128 : 64; }

// Rows a workgroup sums over: all of them where the tiles of one matrix alone fill the chip, else as many as give about 512
// workgroups if one group had all the rows.
constexpr int kLeastChunk = 256;

int64_t splits_of(int outer, int inner) {
    const int64_t tiles = (int64_t)((outer + tile_of(outer) - 1) / tile_of(outer)) * ((inner + tile_of(inner) - 1) / tile_of(inner));
    return tiles >= 256 ? 1 : 512 / tiles;
}

int chunk_rows(int64_t n, int outer, int inner) {
    const int64_t splits = splits_of(outer, inner);
    const int64_t rows = ((n + splits - 1) / splits + 127) / 128 * 128;
    return (int)(rows < kLeastChunk ? kLeastChunk : rows);
}

int64_t chunk_count(int groups, int64_t n, int chunk) { return (n + chunk - 1) / chunk + groups; }

template <class Left, class Right, bool HALF, int OUTER, int INNER>
void launch_sums(const SumArgs& a, unsigned grid, hipStream_t st) {
    constexpr int kTerms = Left::kTerms > Right::kTerms ? Left::kTerms : Right::kTerms;
    constexpr int kDepth = kTerms > 1 ? 32 : 64, kBufs = kTerms > 1 ? 1 : 2;
    matrix_sums_kernel<Left, Right, HALF, OUTER, INNER, kDepth, kBufs><<<grid, 256, 0, st>>>(a);
}

template <class Left, class Right, bool HALF>
int launch_sums(SumArgs a, hipStream_t st) {
    const int to = tile_of(a.outer), ti = tile_of(a.inner);
    a.outer_tiles = (a.outer + to - 1) / to;
    a.inner_tiles = (a.inner + ti - 1) / ti;
    const int64_t blocks = chunk_count(a.groups.offsets ? a.groups.groups : 1, a.groups.n, a.chunk) * a.outer_tiles * a.inner_tiles;
    NEUS2_TRY(check_grid(blocks));
    if (to == 128 && ti == 128) launch_sums<Left, Right, HALF, 128, 128>(a, (unsigned)blocks, st);
    else if (to == 128) launch_sums<Left, Right, HALF, 128, 64>(a, (unsigned)blocks, st);
    else if (ti == 128) launch_sums<Left, Right, HALF, 64, 128>(a, (unsigned)blocks, st);
    else launch_sums<Left, Right, HALF, 64, 64>(a, (unsigned)blocks, st);
    return check_launch("matrix gradient");
}

}  // namespace

int64_t matrix_gradient_bytes(int groups, int64_t n, int outer, int inner, bool by_slot) {
    const int64_t splits = splits_of(outer, inner), least = (n + kLeastChunk - 1) / kLeastChunk;
    if (!by_slot && (splits == 1 || n <= kLeastChunk)) return 0;
    return ((splits < least ? splits : least) + groups) * outer * inner * 4;      // at least chunk_count, and never less for more rows
}

int launch_matrix_gradient(const MatrixGradient& m, hipStream_t st) {
    SumArgs a = {};
    a.groups = m.groups;
    a.chunk = chunk_rows(m.groups.n, m.outer, m.inner);
    a.outer = m.outer;
    a.inner = m.inner;
    a.out = m.out;
    a.accumulate = m.accumulate;
    a.partial = m.partial;
    a.always_partial = m.by_slot;
    if (m.left) {
        a.left = m.left; a.left_stride = m.outer; a.left_vec = m.outer % 4 == 0;
    } else {
        a.left = m.dy; a.left_stride = m.dy_stride; a.left_vec = rows_aligned(m.dtype, m.dy_stride);
    }
    if (m.right) {
        a.right = m.right; a.right_stride = m.inner; a.right_vec = m.inner % 4 == 0;
    } else if (m.xq) {
        a.right = m.xq; a.right_e = m.xe; a.right_stride = (m.inner + 31) / 32 * 32;
    } else {
        a.right = m.x; a.right_stride = m.x_stride; a.right_vec = rows_aligned(m.dtype, m.x_stride);
    }
    int rc;
    const bool f32 = m.dtype == kTypeF32, f16 = m.dtype == kTypeF16;
    if (m.left) {                                                       // v x^T
        if (f32) rc = m.xq ? launch_sums<Wide<3>, Packed<false>, false>(a, st) : launch_sums<Wide<3>, Wide<3>, false>(a, st);
        else if (m.xq) rc = launch_sums<Wide<2>, Packed<false>, false>(a, st);
        else rc = f16 ? launch_sums<Wide<2>, HalfPair, false>(a, st) : launch_sums<Wide<2>, Native, false>(a, st);
    } else if (m.right) {                                               // dy u^T
        if (f32) rc = launch_sums<Wide<3>, Wide<3>, false>(a, st);
        else rc = f16 ? launch_sums<HalfPair, Wide<2>, false>(a, st) : launch_sums<Native, Wide<2>, false>(a, st);
    } else if (f32) {
        rc = m.xq ? launch_sums<Wide<3>, Packed<false>, false>(a, st) : launch_sums<Wide<3>, Wide<3>, false>(a, st);
    } else if (f16) {
        rc = m.xq ? launch_sums<Native, Packed<true>, true>(a, st) : launch_sums<Native, Native, true>(a, st);
    } else {
        rc = m.xq ? launch_sums<Native, Packed<false>, false>(a, st) : launch_sums<Native, Native, false>(a, st);
    }
    if (rc != NEUS2_OK) return rc;
    if (!m.by_slot && m.groups.n <= a.chunk) return NEUS2_OK;           // every group was one chunk
    JoinArgs j = {};
    j.groups = m.groups;
    j.chunk = a.chunk;
    j.size = (int64_t)m.outer * m.inner;
    j.blocks = (int)((j.size + 1023) / 1024);
    j.partial = m.partial;
    j.chunks = (int)chunk_count(m.groups.offsets ? m.groups.groups : 1, m.groups.n, a.chunk);
    j.out = m.out;
    j.accumulate = m.accumulate;
    j.by_slot = m.by_slot ? 1 : 0;
    j.slots = m.slots;
    j.n_slots = m.n_slots;
    const int64_t blocks = (m.by_slot ? m.n_slots : m.groups.offsets ? m.groups.groups : 1) * (int64_t)j.blocks;
    NEUS2_TRY(check_grid(blocks));
    join_sums_kernel<<<(unsigned)blocks, 256, 0, st>>>(j);
    return check_launch("matrix gradient sums");
}

}  // namespace neus2
