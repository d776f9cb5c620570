// Gradients of the matrices of layers whose rows choose them: dW_g = sum over the rows i of group g of dy_i x_i^T, and the same
// sums for the two narrow matrices of adapters.
//
// The contraction runs over the rows, along which neither factor is contiguous: tiles go to LDS as they lie in memory and come
// back through the transposing LDS read.  A group's rows are cut into chunks where there are too few tiles of the matrix to fill
// the chip; the chunks' sums go to a workspace and are added in order, so the result does not depend on which finished first.
#include "layers.h"

namespace neus2 {
namespace {

template <class Factor>
__device__ __forceinline__ typename Factor::Pointer make_pointer(const void* p, const uint8_t* e, int64_t stride, int whole) {
    typename Factor::Pointer f;
    f.p = reinterpret_cast<decltype(f.p)>(p);
    f.stride = stride;
    f.whole = whole;
    if constexpr (std::is_same_v<Factor, Packed<false>> || std::is_same_v<Factor, Packed<true>>) f.e = e;
    return f;
}

// How a product of these factors is cut: k-steps a round, and one or two buffers (with several terms the tiles are large and there is
// enough to do in a round; the other workgroups of the compute unit fill the waits).
template <class Left, class Right, int OUTER, int INNER>
struct SumShape {
    static constexpr int kTerms = Left::kTerms > Right::kTerms ? Left::kTerms : Right::kTerms;
    static constexpr int kDepth = kTerms > 2 || (kTerms > 1 && OUTER * INNER > 64 * 128) ? 32 : 64, kBufs = kTerms > 1 ? 1 : 2;
    typedef FactorTile<Left, false, OUTER, kDepth, 256> LeftTile;
    typedef FactorTile<Right, false, INNER, kDepth, 256> RightTile;
    static constexpr int kBuf = LeftTile::kBytes + RightTile::kBytes, kBytes = kBufs * kBuf;
};

template <class Left, class Right, bool HALF, int OUTER, int INNER>
__device__ __forceinline__ void matrix_sums(const SumArgs& a, int block, unsigned char* lds) {
    typedef SumShape<Left, Right, OUTER, INNER> Shape;
    typedef typename Shape::LeftTile LeftTile;
    typedef typename Shape::RightTile RightTile;
    constexpr int DEPTH = Shape::kDepth, BUFS = Shape::kBufs, kBuf = Shape::kBuf;
    constexpr int kBO = OUTER / 64, kBI = INNER / 64;            // four waves, two by two

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wo = wave >> 1, wi = wave & 1;
    const int tiles = a.outer_tiles * a.inner_tiles;
    const int tile = block % tiles;
    const int outer0 = tile / a.inner_tiles * OUTER, inner0 = tile % a.inner_tiles * INNER;
    const RowTile t = locate<true>(a.groups, a.chunk, 1, block / tiles, lane);
    if (t.group < 0) return;

    const typename Left::Pointer left = make_pointer<Left>(a.left, nullptr, a.left_stride, a.left_whole);
    const typename Right::Pointer right = make_pointer<Right>(a.right, a.right_e, a.right_stride, a.right_whole);
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

    store_sums<false, kBO, kBI>(a, t, outer0 + 32 * wo * kBO, inner0 + 32 * wi * kBI, acc, lane);
}

template <class Left, class Right, bool HALF, int OUTER, int INNER>
__global__ __launch_bounds__(256) void matrix_sums_kernel(SumArgs a) {
    __shared__ __attribute__((aligned(16))) unsigned char lds[SumShape<Left, Right, OUTER, INNER>::kBytes];
    matrix_sums<Left, Right, HALF, OUTER, INNER>(a, a.first_block + (int)blockIdx.x, lds);
}

// Both narrow matrices of adapters, dA (v x^T) and dB (dy u^T), in one launch: each alone is a row of waits (8192 rows, 2048 wide, rank
// 16: 14.4 us each).  WIDE: tiles of 128 along the long side of both.
template <class V, class X, class Dy, class U, int WIDE>
__global__ __launch_bounds__(256) void adapter_sums_kernel(SumArgs a, SumArgs b, int blocks_a) {
    typedef SumShape<V, X, 64, WIDE> A;
    typedef SumShape<Dy, U, WIDE, 64> B;
    __shared__ __attribute__((aligned(16))) unsigned char lds[A::kBytes > B::kBytes ? A::kBytes : B::kBytes];
    const int block = a.first_block + (int)blockIdx.x;
    if (block < blocks_a) matrix_sums<V, X, false, 64, WIDE>(a, block, lds);
    else matrix_sums<Dy, U, false, WIDE, 64>(b, block - blocks_a, lds);
}

// Adds the chunks' sums.  A workgroup has 256 elements of one matrix; each of its four waves adds every fourth chunk in the order of
// the rows, then the four sums are added, so the order is always the same.
struct JoinArgs {
    RowGroups groups;
    int chunk;
    int64_t size;                    // elements of a matrix
    int blocks;                      // workgroups a matrix
    const float* partial; int partials;
    float* out; int accumulate;
    int by_slot; const int32_t* slots; int n_slots;
};

__global__ __launch_bounds__(256) void join_sums_kernel(JoinArgs one, JoinArgs two, int blocks_one) {
    __shared__ v4f sums[4][64];
    const bool second = (int)blockIdx.x >= blocks_one;
    const JoinArgs& a = second ? two : one;
    const int block = (int)blockIdx.x - (second ? blocks_one : 0);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int matrix = block / a.blocks;
    const int groups = a.groups.offsets ? a.groups.groups : 1;
    const bool fours = a.size % 4 == 0;
    int64_t at0 = 0;
    int parts0 = 0;                                                              // a group's parts, if there is only one group
    bool mine = a.by_slot != 0;
    for (int64_t first = (int64_t)(block % a.blocks) * 256; first < a.size; first += (int64_t)a.blocks * 256) {
        const int64_t at = first + 4 * lane;
        const int room = (int)min((int64_t)4, a.size - at);                      // of this lane's four elements, how many there are
        v4f sum = {0.f, 0.f, 0.f, 0.f};
        int turn = 0;                                                            // chunks so far, modulo the waves
        auto part = [&](int p) {
            const float* src = a.partial + (int64_t)p * a.size + at;
            if (fours) return room > 0 ? *reinterpret_cast<const v4f*>(src) : v4f{0.f, 0.f, 0.f, 0.f};
            v4f v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = e < room ? src[e] : 0.f;
            return v;
        };
        auto add_parts = [&](int64_t index, int parts) {
            const int end = (int)min(index + parts, (int64_t)a.partials);        // decreasing offsets may count too many
            if (index >= end) return;
            int p = (int)index + ((wave - turn) & 3);
            turn = (turn + parts) & 3;
            for (; p + 12 < end; p += 16) {
                v4f v[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) v[q] = part(p + 4 * q);
#pragma unroll
                for (int q = 0; q < 4; ++q) sum += v[q];
            }
            for (; p < end; p += 4) sum += part(p);
        };
        if (parts0 > 0) {
            add_parts(at0, parts0);
        } else {
            int64_t before = 0;
            for (int base = 0; base < groups; base += 64) {
                const int e = base + lane;
                int lo = 0, hi = 0, tiles = 0;
                if (e < groups) {
                    group_rows(a.groups, e, lo, hi);
                    tiles = max((hi - lo + a.chunk - 1) / a.chunk, 1);
                }
                if (!a.by_slot && tiles == 1) tiles = 0;                         // stored where it belongs already
                bool match = tiles > 0 && hi > lo;
                if (a.by_slot) match = match && slot_of(a.slots, a.n_slots, e) == matrix;
                else match = match && e == matrix;
                const int end = wave_sums(tiles, lane);
                uint64_t set = __ballot(match);
                while (set) {
                    const int g = __builtin_ctzll(set);
                    set &= set - 1;
                    const int parts = __builtin_amdgcn_readlane(tiles, g);
                    const int64_t index = before + __builtin_amdgcn_readlane(end, g) - parts;
                    add_parts(index, parts);
                    if (!a.by_slot) { at0 = index; parts0 = parts; }
                    mine = true;
                }
                before += __builtin_amdgcn_readlane(end, 63);
                if (!a.by_slot && matrix < base + 64) break;
            }
        }
        if (!mine) return;                                                       // the same in all four waves
        sums[wave][lane] = sum;
        __syncthreads();
        if (wave == 0 && room > 0) {
            float* out = a.out + (int64_t)matrix * a.size + at;
            v4f total = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
            if (fours) {
                if (a.accumulate) total += *reinterpret_cast<const v4f*>(out);
                *reinterpret_cast<v4f*>(out) = total;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < room) out[e] = a.accumulate ? out[e] + total[e] : total[e];
            }
        }
        __syncthreads();
    }
}

// ---- how the work is cut --------------------------------------------------------------------------------------------------------
int tile_of(int dim) { return dim > 64 ? 128 : 64; }

int64_t tiles_of(int outer, int inner, bool wide) {
    const int to = wide ? kWideOuter : tile_of(outer), ti = wide ? kWideInner : tile_of(inner);
    return (int64_t)((outer + to - 1) / to) * ((inner + ti - 1) / ti);
}

// Rows a workgroup sums over: all of them where the tiles of one matrix alone fill the chip, else so many that one group with all
// the rows would give about 512 workgroups (256 of the wide ones, of which a compute unit takes one at a time).
constexpr int kLeastChunk = 256;

int64_t splits_of(int outer, int inner, bool wide) {
    const int64_t tiles = tiles_of(outer, inner, wide);
    return tiles >= 256 ? 1 : ((wide ? 256 : 512) + tiles - 1) / tiles;
}

// Matrices of at least 256 x 256 in 16-bit types take the wide tiles (layers_wide.hip) where the groups alone give one to every compute
// unit, or the chunks are long enough to be worth their sums (bf16: one group, 2048 x 2048, 2^12 rows 60 us against 77, 2^11 rows 48
// against 45; 512 x 4096, 2^13 rows 59 against 66; 8 groups, 512 x 4096, 2^10 rows 24 against 27, 512 x 512, 2^14 rows 42 against 36).
bool wide_sums_fit(const MatrixGradient& m) {
    if (m.dtype == kTypeF32 || m.left || m.right || m.outer < 256 || m.inner < 256) return false;
    const int64_t tiles = tiles_of(m.outer, m.inner, true), splits = splits_of(m.outer, m.inner, true);
    return (tiles * m.groups.groups >= 256 && m.groups.n >= 128 * (int64_t)m.groups.groups) || m.groups.n >= 1024 * splits;
}

int chunk_rows(int64_t n, int64_t splits) {
    const int64_t rows = ((n + splits - 1) / splits + 127) / 128 * 128;
    return (int)(rows < kLeastChunk ? kLeastChunk : rows);
}

int64_t chunk_count(int groups, int64_t n, int chunk) { return (n + chunk - 1) / chunk + groups; }

// Chunks whose sums go to the workspace; never fewer for more rows.  By slot: all of them.  Otherwise only those of groups of more
// than one: a group of L > chunk rows has fewer than 2 L / chunk, all of them together fewer than 2 n / chunk <= 2 splits.
int64_t partial_count(int groups, int64_t n, int64_t splits, bool by_slot) {
    const int64_t least = (n + kLeastChunk - 1) / kLeastChunk, chunks = splits < least ? splits : least;
    if (by_slot) return chunks + groups;
    return splits == 1 || n <= kLeastChunk ? 0 : 2 * chunks;
}

template <class Left, class Right, bool HALF>
void launch_sums(SumArgs a, int64_t blocks, hipStream_t st) {
    const bool o = a.outer > 64, i = a.inner > 64;
    launch_blocks(blocks, 256, [&](unsigned grid, int first) {
        a.first_block = first;
        if (o && i) matrix_sums_kernel<Left, Right, HALF, 128, 128><<<grid, 256, 0, st>>>(a);
        else if (o) matrix_sums_kernel<Left, Right, HALF, 128, 64><<<grid, 256, 0, st>>>(a);
        else if (i) matrix_sums_kernel<Left, Right, HALF, 64, 128><<<grid, 256, 0, st>>>(a);
        else matrix_sums_kernel<Left, Right, HALF, 64, 64><<<grid, 256, 0, st>>>(a);
    });
}

}  // namespace

// (aligned or not: the workspace serves both)
int64_t matrix_gradient_bytes(const MatrixGradient& m) {
    const bool wide = wide_sums_fit(m);
    const int64_t count = partial_count(m.groups.groups, m.groups.n, splits_of(m.outer, m.inner, wide), m.by_slot);
    return (count * m.outer * m.inner * 4 + 15) / 16 * 16;
}

namespace {

int group_count(const MatrixGradient& m) { return m.groups.offsets ? m.groups.groups : 1; }

// everything but the tiles
SumArgs sum_args(const MatrixGradient& m, bool wide) {
    const int count = group_count(m);
    const int64_t splits = splits_of(m.outer, m.inner, wide);
    SumArgs a = {};
    a.groups = m.groups;
    a.chunk = chunk_rows(m.groups.n, splits);
    a.outer = m.outer;
    a.inner = m.inner;
    a.out = m.out;
    a.accumulate = m.accumulate;
    a.once = (int64_t)count * m.outer * m.inner * 4 > kStoreOnceBytes;
    a.partial = m.partial;
    a.partials = (int)partial_count(count, m.groups.n, splits, m.by_slot);
    a.by_slot = m.by_slot ? 1 : 0;
    if (m.left) {
        a.left = m.left; a.left_stride = m.outer; a.left_whole = rows_whole(kTypeF32, m.outer, m.outer);
    } else {
        a.left = m.dy; a.left_stride = m.dy_stride; a.left_whole = rows_whole(m.dtype, m.dy_stride, m.outer);
    }
    if (m.right) {
        a.right = m.right; a.right_stride = m.inner; a.right_whole = rows_whole(kTypeF32, m.inner, m.inner);
    } else if (m.xq) {
        a.right = m.xq; a.right_e = m.xe; a.right_stride = (m.inner + 31) / 32 * 32; a.right_whole = 1;
    } else {
        a.right = m.x; a.right_stride = m.x_stride; a.right_whole = rows_whole(m.dtype, m.x_stride, m.inner);
    }
    return a;
}

// the number of workgroups with tiles of this size
int64_t cut(const MatrixGradient& m, SumArgs& a, int outer_tile, int inner_tile) {
    a.outer_tiles = (a.outer + outer_tile - 1) / outer_tile;
    a.inner_tiles = (a.inner + inner_tile - 1) / inner_tile;
    return chunk_count(group_count(m), m.groups.n, a.chunk) * a.outer_tiles * a.inner_tiles;
}

// whether its chunks, cut for the wide tiles, also take them
bool wide_tiles_fit(const MatrixGradient& m) {
    return wide_sums_fit(m) && rows_aligned(m.dtype, m.dy_stride) && m.dy_stride <= (1 << 20) &&
           (m.xq || (rows_aligned(m.dtype, m.x_stride) && m.x_stride <= (1 << 20)));
}

int64_t sum_blocks(const MatrixGradient& m, SumArgs& a) {
    a = sum_args(m, wide_sums_fit(m));
    return wide_tiles_fit(m) ? cut(m, a, kWideOuter, kWideInner) : cut(m, a, tile_of(m.outer), tile_of(m.inner));
}

JoinArgs join_args(const MatrixGradient& m, const SumArgs& a, int64_t& blocks) {
    JoinArgs j = {};
    j.groups = m.groups;
    j.chunk = a.chunk;
    j.size = (int64_t)m.outer * m.inner;
    // most groups of a large matrix are one chunk and have nothing to join: few workgroups find that out
    const int64_t matrices = m.by_slot ? m.n_slots : group_count(m), most = (2048 + matrices - 1) / matrices;
    j.blocks = (int)((j.size + 255) / 256 < most ? (j.size + 255) / 256 : most);
    j.partial = m.partial;
    j.partials = a.partials;
    j.out = m.out;
    j.accumulate = m.accumulate;
    j.by_slot = a.by_slot;
    j.slots = m.slots;
    j.n_slots = m.n_slots;
    blocks = matrices * j.blocks;
    return j;
}

template <class V, class X, class Dy, class U>
void launch_adapter_sums(SumArgs a, const SumArgs& b, bool wide, int64_t blocks_a, int64_t blocks, hipStream_t st) {
    launch_blocks(blocks, 256, [&](unsigned grid, int first) {
        a.first_block = first;
        if (wide) adapter_sums_kernel<V, X, Dy, U, 128><<<grid, 256, 0, st>>>(a, b, (int)blocks_a);
        else adapter_sums_kernel<V, X, Dy, U, 64><<<grid, 256, 0, st>>>(a, b, (int)blocks_a);
    });
}

}  // namespace

int launch_adapter_gradients(const MatrixGradient& da, const MatrixGradient& db, hipStream_t st) {
    SumArgs a = sum_args(da, false), b = sum_args(db, false);
    const bool wide = da.inner > 64 || db.outer > 64;
    const int64_t blocks_a = cut(da, a, 64, wide ? 128 : 64), blocks = blocks_a + cut(db, b, wide ? 128 : 64, 64);
    if (da.dtype == kTypeF32) {
        if (da.xq) launch_adapter_sums<Wide<3>, Packed<false>, Wide<3>, Wide<3>>(a, b, wide, blocks_a, blocks, st);
        else launch_adapter_sums<Wide<3>, Wide<3>, Wide<3>, Wide<3>>(a, b, wide, blocks_a, blocks, st);
    } else if (da.dtype == kTypeF16) {
        if (da.xq) launch_adapter_sums<Wide<3>, Packed<false>, HalfPair, Wide<3>>(a, b, wide, blocks_a, blocks, st);
        else launch_adapter_sums<Wide<3>, HalfPair, HalfPair, Wide<3>>(a, b, wide, blocks_a, blocks, st);
    } else {
        if (da.xq) launch_adapter_sums<Wide<3>, Packed<false>, Native, Wide<3>>(a, b, wide, blocks_a, blocks, st);
        else launch_adapter_sums<Wide<3>, Native, Native, Wide<3>>(a, b, wide, blocks_a, blocks, st);
    }
    NEUS2_TRY(check_launch("adapter gradients"));
    int64_t joins_a, joins_b;
    const JoinArgs ja = join_args(da, a, joins_a), jb = join_args(db, b, joins_b);
    join_sums_kernel<<<(unsigned)(joins_a + joins_b), 256, 0, st>>>(ja, jb, (int)joins_a);
    return check_launch("adapter gradient sums");
}

int check_matrix_gradient(const MatrixGradient& m) {
    SumArgs a;
    const int64_t blocks = sum_blocks(m, a);
    if (blocks > 0x7fffffff)
        return fail(NEUS2_ERR_SHAPE, "%lld workgroups for dW: too many groups for so large matrices", (long long)blocks);
    return NEUS2_OK;
}

int launch_matrix_gradient(const MatrixGradient& m, hipStream_t st) {
    const bool f32 = m.dtype == kTypeF32, f16 = m.dtype == kTypeF16;
    SumArgs a;
    const int64_t blocks = sum_blocks(m, a);
    if (f32) {
        m.xq ? launch_sums<Wide<3>, Packed<false>, false>(a, blocks, st) : launch_sums<Wide<3>, Wide<3>, false>(a, blocks, st);
    } else if (wide_tiles_fit(m)) {
        launch_wide_sums(m.dtype, m.xq != nullptr, a, blocks, st);
    } else if (f16) {
        m.xq ? launch_sums<Native, Packed<true>, true>(a, blocks, st) : launch_sums<Native, Native, true>(a, blocks, st);
    } else {
        m.xq ? launch_sums<Native, Packed<false>, false>(a, blocks, st) : launch_sums<Native, Native, false>(a, blocks, st);
    }
    NEUS2_TRY(check_launch("matrix gradient"));
    if (a.partials == 0) return NEUS2_OK;                               // every group was one chunk
    int64_t joins;
    const JoinArgs j = join_args(m, a, joins);
    join_sums_kernel<<<(unsigned)joins, 256, 0, st>>>(j, j, (int)joins);
    return check_launch("matrix gradient sums");
}

}  // namespace neus2
