// The wide form of the layers' products for 16-bit types: tiles of 256 x 256 whose factors go from memory to LDS without passing
// through registers.  Per k-step of 16 a wave reads six operands for eight matrix instructions.  One workgroup of eight waves a
// compute unit: tiles of 256 x 128, two workgroups, fetch half as much again from the L2s and were slower (16384 rows, 2048 to 4096 in 8
// groups 345 us against 311 at that step), and so were rounds of 32 steps with four buffers (371 against 309: twice the meetings).
// bf16, one group: 16384 rows, 4096 to 2048 212 us (1300 TFLOP/s), 2048 to 4096 228; 8192 rows, 2048 to 2048 61 us.  Without the products
// the loads alone take two thirds of the time, without the loads the products 80 %: the two overlap, but not wholly.
#include "layers.h"

namespace neus2 {
namespace {

constexpr int kLeft = 256, kRight = 256;         // lines of the instruction's first and second operand
constexpr int kDepth = 64, kThreads = 512, kWaves = 8, kBand = 4;
constexpr int kLeftBytes = kLeft * kDepth * 2, kRightBytes = kRight * kDepth * 2;

// A lane's place in the loads of one factor's tile: chunk c of 1024 bytes (one instruction of a wave) holds units 64 c .. 64 c + 63 of
// 16 bytes in LDS order, and the lane fetches from memory what belongs at its place (FactorTile's order, its swizzle included).
template <bool ALONG, int LINES>
struct WideTile {
    static constexpr int kLoads = LINES * kDepth * 2 / 1024 / kWaves;     // a wave takes every eighth chunk
    uint32_t offset[kLoads];
    __device__ __forceinline__ void begin(int64_t stride, int wave, int lane) {
        typedef FactorTile<Native, ALONG, LINES, kDepth, kThreads> Tile;
#pragma unroll
        for (int q = 0; q < kLoads; ++q) {
            const int unit = 64 * (wave + kWaves * q) + lane;
            const int r = unit / Tile::kPieces, piece = (unit % Tile::kPieces) ^ (ALONG ? Tile::swizzle(r) : Tile::across(r));
            offset[q] = (uint32_t)r * (uint32_t)stride * 2u + 16u * (uint32_t)piece;
        }
    }
    // from: where the tile begins; bytes: how far memory may be read from there on.  What lies beyond comes back as zero, except that
    // the last 16 bytes with something to read are read whole.
    __device__ __forceinline__ void load(const uint16_t* from, int64_t bytes, unsigned char* lds, int wave) const {
        const __amdgpu_buffer_rsrc_t r = make_window(from, bytes > 0x7ffffff0 ? bytes : (bytes + 15) & ~15);
#pragma unroll
        for (int q = 0; q < kLoads; ++q)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(lds + (wave + kWaves * q) * 1024), 16, (int)offset[q], 0, 0, 0);
    }
};

// All loads to LDS of this wave have arrived.
__device__ __forceinline__ void loaded() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0x0f70);                 // vmcnt(0)
    __builtin_amdgcn_sched_barrier(0);
}

// This wave's LDS reads and writes are done, and every wave of the workgroup has got here.
__device__ __forceinline__ void meet() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
}

// The operands of one k-step of a wave: LB blocks of 32 lines of the left factor (the instruction's first operand), RB of the right.
template <int LB, int RB>
struct Operands {
    u32x4 l[LB], r[RB];
    template <class LeftTile, class RightTile>
    __device__ __forceinline__ void read(const unsigned char* left, const unsigned char* right, int wl, int wr, int ks, int lane) {
#pragma unroll
        for (int c = 0; c < LB; ++c) l[c] = LeftTile::operand(left, 0, LB * wl + c, ks, lane);
#pragma unroll
        for (int c = 0; c < RB; ++c) r[c] = RightTile::operand(right, 0, RB * wr + c, ks, lane);
    }
    template <bool HALF, int FIRST, int LAST>
    __device__ __forceinline__ void multiply(v16f (&acc)[LB][RB]) const {
#pragma unroll
        for (int c = FIRST; c < LAST; ++c)
#pragma unroll
            for (int d = 0; d < RB; ++d) acc[c][d] = mma32<HALF>(l[c], r[d], acc[c][d]);
    }
};

struct Stages {
    unsigned char *left[2], *right[2];
};

// The whole contraction: `rounds` pairs of tiles in two pairs of buffers, the loads of one pair in flight while the products of the
// pair before run.  A k-step's operands are read while the instructions of the step before run, across the pairs too: the workgroup
// meets in the middle of a pair's last step, so that the matrix pipe still has work when the waves come out of the barrier and wait for
// their first operands.  The scheduler is kept from moving reads further up, which would take more registers than there are.
// fetch(left, right, more) issues a pair's loads (zeros if there is no more: an odd number of pairs ends with one of zeros);
// land(right) is what a factor that does pass through registers still has to do.  The caller has issued the first pair's loads and waited
// for them (loaded()).  When this returns nobody reads the second pair of buffers any more.  Of the first pair other waves may still be
// reading the operands behind the last pair's, which no product takes, so it may be overwritten at once (a branch around that last read
// costs nine registers, kept in memory: 16384 rows, 2048 to 4096 in 8 groups, both gradients 612 us against 598).
template <bool HALF, class LeftTile, class RightTile, int LB, int RB, class Fetch, class Land>
__device__ __forceinline__ void contract(int rounds, const Fetch& fetch, const Land& land, const Stages& s, int wl, int wr, int lane,
                                         v16f (&acc)[LB][RB]) {
    constexpr int kSteps = kDepth / 16;
    Operands<LB, RB> o[2];
    land(s.right[0]);
    meet();
    o[0].template read<LeftTile, RightTile>(s.left[0], s.right[0], wl, wr, 0, lane);
    for (int k = 0; k < rounds; k += 2) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
#pragma unroll
            for (int ks = 0; ks < kSteps - 1; ++ks) {
                o[(ks + 1) & 1].template read<LeftTile, RightTile>(s.left[q], s.right[q], wl, wr, ks + 1, lane);
                if (ks == 0) fetch(s.left[q ^ 1], s.right[q ^ 1], k + q + 1 < rounds);
                o[ks & 1].template multiply<HALF, 0, LB>(acc);
                __builtin_amdgcn_sched_barrier(0);
            }
            land(s.right[q ^ 1]);
            o[1].template multiply<HALF, 0, LB / 2>(acc);
            __builtin_amdgcn_sched_barrier(0);
            loaded();
            meet();
            o[0].template read<LeftTile, RightTile>(s.left[q ^ 1], s.right[q ^ 1], wl, wr, 0, lane);
            o[1].template multiply<HALF, LB / 2, LB>(acc);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

#define NEUS2_STAGES                                                                                                      \
    __shared__ __attribute__((aligned(16))) unsigned char left0[kLeftBytes], left1[kLeftBytes];                           \
    __shared__ __attribute__((aligned(16))) unsigned char right0[kRightBytes], right1[kRightBytes];                       \
    const Stages stages = {{left0, left1}, {right0, right1}}

template <int DT, bool BACKWARD, bool ADAPT, bool ONCE>
__global__ __launch_bounds__(kThreads, 2) void wide_rows_kernel(RowsArgs a) {
    typedef FactorTile<Native, true, kRight, kDepth, kThreads> DataTile;
    typedef FactorTile<Native, !BACKWARD, kLeft, kDepth, kThreads> MatrixTile;
    NEUS2_STAGES;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wc = wave >> 2, wr = wave & 3;
    // bands of four tiles of rows, in a band the rows fastest: the workgroups at work on an XCD share few rows and few columns
    const int row_tiles = count_tiles(a.groups, kRight, 0, lane);
    Pieces pieces(row_tiles * a.col_tiles);
    if (!ADAPT) pieces.quarter_last_round();
    int col0 = 0;
    RowTile t;
    auto place = [&](int piece, int& col, RowTile& tile) {
        const int band = piece / (kBand * a.col_tiles), within = piece % (kBand * a.col_tiles), deep = min(kBand, row_tiles - band * kBand);
        col = within / deep * kLeft;
        tile = locate(a.groups, kRight, 0, band * kBand + within % deep, lane);
    };
    const int first = pieces.take();
    if (first < 0) return;
    place(first, col0, t);

    WideTile<true, kRight> dt;
    WideTile<!BACKWARD, kLeft> mt;
    dt.begin(a.x_stride, wave, lane);
    mt.begin(a.w_stride, wave, lane);
    const uint16_t *x, *w;
    int64_t x_bytes, w_bytes;
    const int64_t w_step = BACKWARD ? (int64_t)kDepth * a.w_stride : kDepth;
    auto begin = [&]() {
        x = reinterpret_cast<const uint16_t*>(a.x) + (int64_t)t.lo * a.x_stride;
        w = reinterpret_cast<const uint16_t*>(a.w) + (int64_t)t.group * a.w_group + (int64_t)col0 * (BACKWARD ? 1 : a.w_stride);
        x_bytes = ((int64_t)(t.hi - t.lo - 1) * a.x_stride + a.steps) * 2;
        w_bytes = BACKWARD ? ((int64_t)a.steps * a.w_stride - col0) * 2 : (int64_t)(a.cols - col0) * a.w_stride * 2;
    };
    auto fetch = [&](unsigned char* matrix, unsigned char* data, bool more) {
        dt.load(x, more ? x_bytes : 0, data, wave);
        mt.load(w, more ? w_bytes : 0, matrix, wave);
        x += kDepth;
        x_bytes -= kDepth * 2;
        w += w_step;
        w_bytes -= w_step * 2;
    };
    begin();
    fetch(left0, right0, true);
    loaded();
    // The first loads of the next tile are under way while this one's outputs are stored (not beside an adapter's part, which takes the
    // registers: a workgroup then has one tile).
    for (;;) {
        v16f acc[4][2];
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int r = 0; r < 2; ++r) acc[c][r] = zero16();
        const RowTile now = t;
        const int now_col = col0, next = ADAPT ? -1 : pieces.take();
        if (next >= 0) place(next, col0, t);
        Segments segments = {};
        if (ADAPT) segments.begin(a, now, lane);
        contract<DT == kTypeF16, MatrixTile, DataTile>(a.steps / kDepth, fetch, [](unsigned char*) {}, stages, wc, wr, lane, acc);
        if (next >= 0) {
            begin();
            fetch(left0, right0, true);
        }
        finish_rows<DT, BACKWARD, ADAPT, 4, 2, ONCE>(a, now, segments, now_col + 128 * wc, 64 * wr, acc, wave < 4 ? left1 : right1, wave & 3, lane, loaded);
        if (next < 0) break;
    }
    if (ADAPT) return;
    // Quarters of the last round's tiles, 128 x 128, a wave 64 x 32 of them, where few are left for it: 8192 rows, 2048 to 2048 in 5
    // groups 79 us against 98 with whole tiles, 20000 rows, 2048 to 1024 backward in 8 groups 85 against 107; in whole rounds the same.
    typedef FactorTile<Native, true, kRight / 2, kDepth, kThreads> SmallDataTile;
    typedef FactorTile<Native, !BACKWARD, kLeft / 2, kDepth, kThreads> SmallMatrixTile;
    WideTile<true, kRight / 2> small_dt;
    WideTile<!BACKWARD, kLeft / 2> small_mt;
    const int lane2 = (int)again((uint32_t)lane);                        // or what depends on it is worked out, and held, from the start
    small_dt.begin(a.x_stride, wave, lane2);
    small_mt.begin(a.w_stride, wave, lane2);
    auto small_fetch = [&](unsigned char* matrix, unsigned char* data, bool more) {
        small_dt.load(x, more ? x_bytes : 0, data, wave);
        small_mt.load(w, more ? w_bytes : 0, matrix, wave);
        x += kDepth;
        x_bytes -= kDepth * 2;
        w += w_step;
        w_bytes -= w_step * 2;
    };
    for (int turn = 0;;) {
        const int quarter = pieces.take_quarter(turn);
        if (quarter < 0) break;
        if (quarter >> 2 >= row_tiles * a.col_tiles) continue;
        place(quarter >> 2, col0, t);
        col0 += quarter & 2 ? kLeft / 2 : 0;
        t.lo += quarter & 1 ? kRight / 2 : 0;
        t.hi = min(t.hi, t.lo + kRight / 2);
        if (t.lo >= t.hi || col0 >= a.cols) continue;
        begin();
        meet();                                                          // nobody stores out of the buffers any more
        small_fetch(left0, right0, true);
        loaded();
        v16f acc[2][1];
        acc[0][0] = zero16();
        acc[1][0] = zero16();
        contract<DT == kTypeF16, SmallMatrixTile, SmallDataTile>(a.steps / kDepth, small_fetch, [](unsigned char*) {}, stages, wc, wr, lane2, acc);
        finish_rows<DT, BACKWARD, false, 2, 1, ONCE>(a, t, {}, col0 + 64 * wc, 32 * wr, acc, left1, wave, lane2, [] {});
    }
}

template <int DT, bool BACKWARD>
void launch(const RowsArgs& a, unsigned grid, hipStream_t st) {
    if (a.rank > 0) a.once ? wide_rows_kernel<DT, BACKWARD, true, true><<<grid, kThreads, 0, st>>>(a)
                           : wide_rows_kernel<DT, BACKWARD, true, false><<<grid, kThreads, 0, st>>>(a);
    else a.once ? wide_rows_kernel<DT, BACKWARD, false, true><<<grid, kThreads, 0, st>>>(a)
                : wide_rows_kernel<DT, BACKWARD, false, false><<<grid, kThreads, 0, st>>>(a);
}

// Sums over rows: both factors lie across (a memory row is a step of the contraction), the rows behind the chunk's last are zeros.
// PACKED: the right factor is in 8 bits.  A thread then fetches 32 of its values (one block of one row, one exponent) and puts them
// into LDS as 16-bit numbers at the end of the round.
template <int DT, bool PACKED, bool ONCE>
__global__ __launch_bounds__(kThreads, 2) void wide_sums_kernel(SumArgs a) {
    constexpr bool kHalf = DT == kTypeF16;
    typedef FactorTile<Native, false, kLeft, kDepth, kThreads> LeftTile;
    typedef FactorTile<Native, false, kRight, kDepth, kThreads> RightTile;
    typedef Packed<kHalf> Factor8;
    NEUS2_STAGES;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wo = wave >> 2, wi = wave & 3;
    const int tiles = a.outer_tiles * a.inner_tiles;
    const int block = a.first_block + (int)blockIdx.x, tile = block % tiles, outer0 = tile / a.inner_tiles * kLeft, inner0 = tile % a.inner_tiles * kRight;
    const RowTile t = locate<true>(a.groups, a.chunk, 1, block / tiles, lane);
    if (t.group < 0) return;

    WideTile<false, kLeft> lt;
    WideTile<false, kRight> rt;
    lt.begin(a.left_stride, wave, lane);
    rt.begin(a.right_stride, wave, lane);
    int rows = t.hi - t.lo;
    const int rounds = (rows + kDepth - 1) / kDepth, col8 = inner0 + 32 * (tid & 7);
    const uint16_t* left = reinterpret_cast<const uint16_t*>(a.left) + (int64_t)t.lo * a.left_stride + outer0;
    const uint16_t* right = reinterpret_cast<const uint16_t*>(a.right) + (PACKED ? 0 : (int64_t)t.lo * a.right_stride + inner0);
    typename Factor8::Pointer packed;
    packed.p = reinterpret_cast<const int8_t*>(a.right);
    packed.e = a.right_e;
    packed.stride = a.right_stride;
    typename Factor8::Raw raw[4];
    auto fetch = [&](unsigned char* l, unsigned char* r, bool more) {
        lt.load(left, more ? ((int64_t)(rows - 1) * a.left_stride + a.outer - outer0) * 2 : 0, l, wave);
        if (PACKED) {
            const typename Factor8::Window w = Factor8::window(packed, t.hi - rows, inner0, more ? min(rows, kDepth) : 0, 0);
#pragma unroll
            for (int q = 0; q < 4; ++q) raw[q] = Factor8::fetch(w, tid >> 3, 32 * (tid & 7) + 8 * q, more && (tid >> 3) < rows && col8 < a.inner);
        } else {
            rt.load(right, more ? ((int64_t)(rows - 1) * a.right_stride + a.inner - inner0) * 2 : 0, r, wave);
            right += (int64_t)kDepth * a.right_stride;
        }
        left += (int64_t)kDepth * a.left_stride;
        rows -= kDepth;
    };
    auto land = [&](unsigned char* r) {
        if (!PACKED) return;
        const int line = tid >> 3;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            u32x4 v[1];
            Factor8::terms(raw[q], v);
            *reinterpret_cast<u32x4*>(r + line * (kRight * 2) + (((4 * (tid & 7) + q) ^ RightTile::across(line)) << 4)) = v[0];
        }
    };
    v16f acc[4][2];
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int r = 0; r < 2; ++r) acc[c][r] = zero16();
    fetch(left0, right0, rounds > 0);
    loaded();
    contract<kHalf, LeftTile, RightTile>(rounds, fetch, land, stages, wo, wi, lane, acc);
    store_sums<ONCE, 4, 2>(a, t, outer0 + 128 * wo, inner0 + 64 * wi, acc, lane);
}

// one workgroup a compute unit, as many on every XCD
unsigned wide_blocks(int64_t pieces) {
    const int64_t units = compute_units() / kXcds * kXcds, blocks = (pieces + kXcds - 1) / kXcds * kXcds;
    return (unsigned)(units > 0 && units < blocks ? units : blocks);
}

}  // namespace

void launch_wide_sums(int dtype, bool packed, const SumArgs& args, int64_t blocks, hipStream_t st) {
    SumArgs a = args;
    auto go = [&](auto* plain, auto* once) {
        launch_blocks(blocks, kThreads, [&](unsigned grid, int first) {
            a.first_block = first;
            (a.once ? once : plain)<<<grid, kThreads, 0, st>>>(a);
        });
    };
    if (dtype == kTypeF16) {
        if (packed) go(wide_sums_kernel<kTypeF16, true, false>, wide_sums_kernel<kTypeF16, true, true>);
        else go(wide_sums_kernel<kTypeF16, false, false>, wide_sums_kernel<kTypeF16, false, true>);
    } else {
        if (packed) go(wide_sums_kernel<kTypeBF16, true, false>, wide_sums_kernel<kTypeBF16, true, true>);
        else go(wide_sums_kernel<kTypeBF16, false, false>, wide_sums_kernel<kTypeBF16, false, true>);
    }
}

int launch_wide_rows(int dtype, bool backward, const RowsArgs& args, hipStream_t st) {
    RowsArgs a = args;
    a.col_tiles = (a.cols + kLeft - 1) / kLeft;
    const int64_t pieces = row_tiles(a.groups, kRight) * a.col_tiles;
    // (one launch: beside a shared matrix, whose rows are one group, its limit of 2^23 tiles is 550 GB of outputs)
    const unsigned grid = a.rank > 0 ? (unsigned)((pieces + kXcds - 1) / kXcds * kXcds) : wide_blocks(pieces);
    if (dtype == kTypeF16) backward ? launch<kTypeF16, true>(a, grid, st) : launch<kTypeF16, false>(a, grid, st);
    else backward ? launch<kTypeBF16, true>(a, grid, st) : launch<kTypeBF16, false>(a, grid, st);
    return check_launch("wide layer");
}

}  // namespace neus2
