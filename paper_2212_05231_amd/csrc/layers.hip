// Layers whose rows choose their matrices: forward products and the gradient with respect to the input (one product engine for
// both), the low-rank part of adapters, and layer inputs in 8 bits.  The gradients of the matrices are in layers_grad.hip.
#include "layers.h"

namespace neus2 {
namespace {

// ---- the product engine ----------------------------------------------------------------------------------------------------
// For what is neither wide nor narrow, and for fp32: bound by the waits of a round (fetch, LDS, products) where there are few tiles, by the
// bf16 products of the fp32 terms where there are many (2048 to 2048, 2^13 rows, fp32: 363 us, 189 TFLOP/s; the library's fp32 product
// reaches 153 on a large matrix).
// One workgroup owns ROWS data rows of one group and COLS outputs; both factors of DEPTH steps of the contraction lie in LDS,
// fetched into registers while the products of the steps before run.  The matrix's tile is the instruction's first operand, so a
// lane ends up with four consecutive outputs of one row.
// BACKWARD = false: y = W x (contraction along the memory rows of W); true: dx = W^T dy (every memory row of W is a step).
template <int DT, bool BACKWARD, bool ADAPT, bool ONCE, int ROWS, int COLS, int WR, int WC, int DEPTH, int BUFS>
__global__ __launch_bounds__(64 * WR * WC) void rows_kernel(RowsArgs a) {
    typedef typename TypeOf<DT>::Element E;
    typedef std::conditional_t<DT == kTypeF32, Wide<3>, Native> Factor;
    constexpr int kThreads = 64 * WR * WC;
    constexpr int kBR = ROWS / WR / 32, kBC = COLS / WC / 32, kTerms = Factor::kTerms;
    constexpr bool kHalf = DT == kTypeF16;
    typedef FactorTile<Factor, true, ROWS, DEPTH, kThreads> DataTile;
    typedef FactorTile<Factor, !BACKWARD, COLS, DEPTH, kThreads> MatrixTile;
    constexpr int kBuf = DataTile::kBytes + MatrixTile::kBytes;
    constexpr int kStores = WR * WC * 32 * kBC * 32 * (int)sizeof(E);
    __shared__ __attribute__((aligned(16))) unsigned char lds[BUFS * kBuf > kStores ? BUFS * kBuf : kStores];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wr = wave / WC, wc = wave % WC;
    const int block = a.first_block + (int)blockIdx.x, col0 = block % a.col_tiles * COLS;
    const RowTile t = locate(a.groups, ROWS, 0, block / a.col_tiles, lane);
    if (t.group < 0) return;

    typename Factor::Pointer data, matrix;
    data.p = reinterpret_cast<decltype(data.p)>(a.x);
    data.stride = a.x_stride;
    data.whole = a.x_whole;
    matrix.p = reinterpret_cast<decltype(matrix.p)>(a.w) + (int64_t)t.group * a.w_group;
    matrix.stride = a.w_stride;
    matrix.whole = a.w_whole;
    DataTile dt;
    MatrixTile mt;
    v16f acc[kBC][kBR];
#pragma unroll
    for (int c = 0; c < kBC; ++c)
#pragma unroll
        for (int r = 0; r < kBR; ++r) acc[c][r] = zero16();

    Segments segments = {};
    if (ADAPT) segments.begin(a, t, lane);
    const int rounds = (a.steps + DEPTH - 1) / DEPTH;
    dt.load(data, t.lo, t.hi - t.lo, 0, a.steps, tid);
    mt.load(matrix, col0, a.cols - col0, 0, a.steps, tid);
    dt.store(lds, tid);
    mt.store(lds + DataTile::kBytes, tid);
    __syncthreads();
    for (int k = 0; k < rounds; ++k) {
        const unsigned char* buf = lds + (BUFS == 2 ? (k & 1) * kBuf : 0);
        const bool more = k + 1 < rounds;
        if (more) {
            const int step = (k + 1) * DEPTH;
            dt.load(data, t.lo, t.hi - t.lo, step, a.steps - step, tid);
            mt.load(matrix, col0, a.cols - col0, step, a.steps - step, tid);
        }
#pragma unroll
        for (int ks = 0; ks < DEPTH / 16; ++ks) {
            u32x4 m[kBC][kTerms], d[kBR][kTerms];
#pragma unroll
            for (int c = 0; c < kBC; ++c)
#pragma unroll
                for (int p = 0; p < kTerms; ++p) m[c][p] = MatrixTile::operand(buf + DataTile::kBytes, p, wc * kBC + c, ks, lane);
#pragma unroll
            for (int r = 0; r < kBR; ++r)
#pragma unroll
                for (int p = 0; p < kTerms; ++p) d[r][p] = DataTile::operand(buf, p, wr * kBR + r, ks, lane);
#pragma unroll
            for (int c = 0; c < kBC; ++c)
#pragma unroll
                for (int r = 0; r < kBR; ++r) acc[c][r] = mma_terms<kHalf>(m[c], d[r], acc[c][r]);
        }
        if (BUFS == 1) __syncthreads();
        if (more) {
            unsigned char* next = lds + (BUFS == 2 ? ((k + 1) & 1) * kBuf : 0);
            dt.store(next, tid);
            mt.store(next + DataTile::kBytes, tid);
        }
        __syncthreads();
    }

    finish_rows<DT, BACKWARD, ADAPT, kBC, kBR, ONCE>(a, t, segments, col0 + 32 * wc * kBC, 32 * wr * kBR, acc, lds, wave, lane, [] {});
}

// ---- narrow layers ---------------------------------------------------------------------------------------------------------------
// Contractions of up to 64 steps and up to 64 outputs, the framework's own widths, with many rows: bound by reading and writing the
// rows once.  A workgroup keeps the group's matrix in LDS, split once, and takes a run of consecutive tiles of 128 rows; a wave has 32
// of them, whose values go from memory to registers as the instruction wants them (lane = row), the next tile's under way while this
// one's products run.  2^18 rows, 64 to 64, fp32 in 20 groups: 27 us, 5.0 TB/s; with rows_kernel 30.
constexpr int kNarrowRows = 128;

template <int DT, bool BACKWARD, bool ONCE>
__global__ __launch_bounds__(256, 3) void narrow_rows_kernel(RowsArgs a) {
    typedef typename TypeOf<DT>::Element E;
    typedef std::conditional_t<DT == kTypeF32, Wide<3>, Native> Factor;
    constexpr int kTerms = Factor::kTerms, kSteps = 4;
    typedef FactorTile<Factor, !BACKWARD, 64, 64, 256> MatrixTile;
    constexpr int kStage = 32 * 64 * (int)sizeof(E);                     // 32 rows of 32 (fp32) or 64 (16 bits) outputs
    __shared__ __attribute__((aligned(16))) unsigned char matrix[MatrixTile::kBytes], stage[4 * (sizeof(E) == 4 ? kStage / 2 : kStage)];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int j = lane & 31, h = lane >> 5;
    const int64_t total = count_tiles(a.groups, kNarrowRows, 0, lane);
    const int first = (int)(total * blockIdx.x / gridDim.x), end = (int)(total * (blockIdx.x + 1) / gridDim.x);
    if (first >= end) return;

    typename Factor::Pointer data, source;
    data.p = reinterpret_cast<decltype(data.p)>(a.x);
    data.stride = a.x_stride;
    data.whole = a.x_whole;
    source.stride = a.w_stride;
    source.whole = a.w_whole;
    typename Factor::Raw x[kSteps];
    // the values of k-step ks of this wave's rows of a tile
    auto request = [&](const RowTile& t, const typename Factor::Window& w, int ks) {
        const int lo = t.lo + 32 * wave, rows = min(32, t.hi - lo), k = 16 * ks + 8 * h;
        x[ks] = Factor::fetch(w, j, k, j < rows && k < a.steps);
    };
    auto window = [&](const RowTile& t) { return Factor::window(data, t.lo + 32 * wave, 0, min(32, t.hi - t.lo - 32 * wave), a.steps); };
    int held = -1;                                                       // the group whose matrix lies in LDS
    RowTile t = locate(a.groups, kNarrowRows, 0, first, lane);
    typename Factor::Window w = window(t);
#pragma unroll
    for (int ks = 0; ks < kSteps; ++ks) request(t, w, ks);
    for (int tile = first;;) {
        if (t.group != held) {
            if (held >= 0) __syncthreads();                              // nobody reads the one before any more
            source.p = reinterpret_cast<decltype(source.p)>(a.w) + (int64_t)t.group * a.w_group;
            MatrixTile m;
            m.load(source, 0, a.cols, 0, a.steps, tid);
            m.store(matrix, tid);
            __syncthreads();
            held = t.group;
        }
        const RowTile now = t;
        const bool more = ++tile < end;
        if (more) {
            locate_next(a.groups, kNarrowRows, 0, tile, lane, t);
            w = window(t);
        }
        v16f acc[2][1];
#pragma unroll
        for (int c = 0; c < 2; ++c) acc[c][0] = zero16();
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) {
            u32x4 d[kTerms], m[2][kTerms];
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int p = 0; p < kTerms; ++p) m[c][p] = MatrixTile::operand(matrix, p, c, ks, lane);
            Factor::terms(x[ks], d);
            if (more) request(t, w, ks);
#pragma unroll
            for (int c = 0; c < 2; ++c) acc[c][0] = mma_terms<DT == kTypeF16>(m[c], d, acc[c][0]);
            __builtin_amdgcn_sched_barrier(0);                           // reads hoisted out of the later steps would take the registers
        }
        if (now.lo + 32 * wave < now.hi) {
            if constexpr (sizeof(E) == 4) {
                v16f half[1][1];
                half[0][0] = acc[0][0];
                finish_rows<DT, BACKWARD, false, 1, 1, ONCE>(a, now, {}, 0, 32 * wave, half, stage, wave, lane, [] {});
                half[0][0] = acc[1][0];
                if (a.cols > 32) finish_rows<DT, BACKWARD, false, 1, 1, ONCE>(a, now, {}, 32, 32 * wave, half, stage, wave, lane, [] {});
            } else {
                finish_rows<DT, BACKWARD, false, 2, 1, ONCE>(a, now, {}, 0, 32 * wave, acc, stage, wave, lane, [] {});
            }
        }
        if (!more) break;
    }
}

// ---- few rows ------------------------------------------------------------------------------------------------------------------
// 16 rows and 16 outputs on the 16x16x32 instruction, operands straight from memory: with so few rows the pass is bound by reading
// the matrices once, and there is nothing to share through LDS.  The eight waves of a workgroup share the contraction, each with up to
// four lines of every matrix row in flight (2048 steps of a 16-bit type at once); four lanes read a line's 64 bytes.  Their sums are
// joined in LDS, and a thread adds what the row's adapter gives.
struct FewArgs {
    RowGroups groups;
    const void* x; int64_t x_stride; int x_whole;
    const void* w; int64_t w_group; int w_stride, w_whole;
    int steps, cols;
    void* y; int64_t y_stride;
    int relu;
    const int32_t* segments; int n_segments; const int32_t* slots; int n_slots; const float* u; const void* bank; int rank;
    int col_tiles;
    int first_block;
};

constexpr int kFewWaves = 8;

template <int DT>
__global__ __launch_bounds__(64 * kFewWaves) void few_rows_kernel(FewArgs a) {
    typedef typename TypeOf<DT>::Element E;
    typedef std::conditional_t<DT == kTypeF32, Wide<3>, Native> Factor;
    constexpr int kTerms = Factor::kTerms;
    constexpr bool kHalf = DT == kTypeF16;
    constexpr int kUnits = DT == kTypeF32 ? 1 : 2;            // operands a lane takes of one line of 128 bytes
    constexpr int kChunk = 32 * kUnits;                       // steps of the contraction they cover
    constexpr int kAhead = 4;
    __shared__ v4f part[kFewWaves][64];
    __shared__ int row_slot[16];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int block = a.first_block + (int)blockIdx.x, col0 = block % a.col_tiles * 16;
    const RowTile t = locate(a.groups, 16, 0, block / a.col_tiles, lane);
    if (t.group < 0) return;

    const int i = lane & 15, quarter = lane >> 4;
    v4f acc = {0.f, 0.f, 0.f, 0.f};
    typename Factor::Pointer data, matrix;
    data.p = reinterpret_cast<decltype(data.p)>(a.x);
    data.stride = a.x_stride;
    data.whole = a.x_whole;
    matrix.p = reinterpret_cast<decltype(matrix.p)>(a.w) + (int64_t)t.group * a.w_group;
    matrix.stride = a.w_stride;
    matrix.whole = a.w_whole;
    const bool row_in = t.lo + i < t.hi, col_in = col0 + i < a.cols;
    const typename Factor::Window xs = Factor::window(data, t.lo, 0, t.hi - t.lo, a.steps), ws = Factor::window(matrix, col0, 0, min(16, a.cols - col0), a.steps);
    const bool whole = a.x_whole && a.w_whole;
    // A wave's part of the contraction is one piece: rows that lie a power of two apart hang on the same memory channels, and waves
    // that walk side by side would all be at the same few of them.
    const int length = (a.steps + kFewWaves * kChunk - 1) / (kFewWaves * kChunk) * kChunk, end = min(a.steps, (wave + 1) * length);
    auto find_slots = [&] {                                               // the adapters of this wave's share of the rows
        if (a.rank == 0) return;
#pragma unroll
        for (int r = 0; r < 16 / kFewWaves; ++r) {
            const int of = 16 / kFewWaves * wave + r, s = segment_of(a.segments, a.n_segments, min(t.lo + of, t.hi - 1), lane);
            const int slot = s < a.n_segments ? slot_of(a.slots, a.n_slots, s) : -1;
            if (lane == 0) row_slot[of] = slot;
        }
    };
    if (wave * length >= end) find_slots();
    for (int base = wave * length; base < end; base += kAhead * kChunk) {
        typename Factor::Raw w[kAhead][kUnits], x[kAhead][kUnits];
#pragma unroll
        for (int q = 0; q < kAhead; ++q)
#pragma unroll
            for (int v = 0; v < kUnits; ++v) {
                const int k = base + q * kChunk + 32 * v + 8 * quarter;
                if (whole) {
                    w[q][v] = Factor::fetch(ws, i, k, col_in && k < end);
                    x[q][v] = Factor::fetch(xs, i, k, row_in && k < end);
                } else {
                    w[q][v] = Factor::load(matrix, col0 + i, k, col_in ? end - k : 0);
                    x[q][v] = Factor::load(data, t.lo + i, k, row_in ? end - k : 0);
                }
            }
        if (base == wave * length) find_slots();                          // while the first loads are under way
#pragma unroll
        for (int q = 0; q < kAhead; ++q)
#pragma unroll
            for (int v = 0; v < kUnits; ++v) {
                u32x4 wt[kTerms], xt[kTerms];
                Factor::terms(w[q][v], wt);
                Factor::terms(x[q][v], xt);
#pragma unroll
                for (int p = 0; p < kTerms; ++p)
#pragma unroll
                    for (int r = 0; r < kTerms; ++r)
                        if (p + r < kTerms) acc = mma16<kHalf>(wt[p], xt[r], acc);
            }
    }
    // lane: row lane % 16, outputs 4 (lane / 16) .. + 3
    part[wave][lane] = acc;
    __syncthreads();
    // a thread per output, the outputs of a row side by side
    const int row = tid >> 4, c = tid & 15, col = col0 + c;
    const int64_t at = t.lo + row;
    if (row >= 16 || at >= t.hi || col >= a.cols) return;
    float z = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) z += part[w][(c >> 2) * 16 + row][c & 3];
    if (a.rank > 0 && row_slot[row] >= 0) {
        const E* bank = reinterpret_cast<const E*>(a.bank) + ((int64_t)row_slot[row] * a.cols + col) * a.rank;
        const float* u = a.u + at * a.rank;
        if (a.rank % 8 == 0) {
            for (int k = 0; k < a.rank; k += 8) {
                const f32x8 b = eight(bank + k), v = eight(u + k);
#pragma unroll
                for (int s = 0; s < 8; ++s) z += b[s] * v[s];
            }
        } else {
            for (int k = 0; k < a.rank; ++k) z += (float)bank[k] * u[k];
        }
    }
    reinterpret_cast<E*>(a.y)[at * a.y_stride + col] = (E)(a.relu ? relu1(z) : z);
}

// ---- the low-rank products of adapters -------------------------------------------------------------------------------------------
// u = scale A[slot] x (DOWN = false) or v = scale B[slot]^T dy (DOWN = true: the contraction runs down the matrix's columns), fp32, zeros
// for the rows of segments without a slot.  Bound by reading the rows, which are many and wide beside the few outputs: one workgroup
// has all outputs of its 32 rows, so that they are read once (16 outputs a workgroup, the rows read once per 16: 8192 x 2048, rank 64,
// 36 us).  SPLIT: the eight waves share the contraction; otherwise (short ones) every wave has 32 rows of its own.
struct LowRankArgs {
    RowGroups groups;
    const void* x; int64_t x_stride; int x_whole;
    const void* bank; int64_t bank_slot; int bank_whole;
    int steps, rank;
    const int32_t* slots; int n_slots; const float* scales;
    float* u;
    int first_block;
};

template <int DT, bool DOWN, bool SPLIT, int BLOCKS>
__global__ __launch_bounds__(512, SPLIT ? 4 : 2) void low_rank_kernel(LowRankArgs a) {
    typedef typename TypeOf<DT>::Element E;
    typedef std::conditional_t<DT == kTypeF32, Wide<3>, Native> Factor;
    constexpr int kTerms = Factor::kTerms;
    // k-steps (of 32) whose operands are in flight together: as many as leave registers for a second workgroup on the compute unit
    constexpr int kAhead = DT == kTypeF32 ? (BLOCKS > (DOWN ? 1 : 2) ? 1 : 2) : BLOCKS > 2 ? (DOWN ? 1 : 2) : DOWN && BLOCKS > 1 ? 2 : 4;
    constexpr bool kHalf = DT == kTypeF16;
    constexpr int kWaves = 8;
    __shared__ float part[SPLIT ? kWaves : 1][SPLIT ? BLOCKS * 16 : 1][33];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    RowTile t = locate(a.groups, SPLIT ? 32 : 32 * kWaves, 0, a.first_block + (int)blockIdx.x, lane);
    if (t.group < 0) return;
    if (!SPLIT) {
        t.lo += 32 * wave;
        t.hi = min(t.hi, t.lo + 32);
        if (t.lo >= t.hi) return;
    }
    const int slot = slot_of(a.slots, a.n_slots, t.group);
    if (slot < 0) {
        for (int i = SPLIT ? tid : lane; i < (t.hi - t.lo) * a.rank; i += SPLIT ? 512 : 64) a.u[(int64_t)t.lo * a.rank + i] = 0.f;
        return;
    }
    const float scale = a.scales[slot];
    typename Factor::Pointer data, matrix;
    data.p = reinterpret_cast<decltype(data.p)>(a.x);
    data.stride = a.x_stride;
    data.whole = a.x_whole;
    matrix.p = reinterpret_cast<decltype(matrix.p)>(a.bank) + (int64_t)slot * a.bank_slot;
    matrix.stride = a.steps;
    matrix.whole = a.bank_whole;
    const typename Factor::Window xs = Factor::window(data, t.lo, 0, t.hi - t.lo, a.steps), bs = Factor::window(matrix, 0, 0, a.rank, a.steps);
    const __amdgpu_buffer_rsrc_t down = make_window(matrix.p, a.bank_slot * (int64_t)sizeof(E));
    const bool whole = a.x_whole && (DOWN || a.bank_whole);
    const int i = lane & 15, quarter = lane >> 4, rows = t.hi - t.lo;
    v4f acc[BLOCKS][2];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
        for (int r = 0; r < 2; ++r) acc[b][r] = v4f{0.f, 0.f, 0.f, 0.f};
    constexpr int kRun = 32 * kAhead;
    const int length = (a.steps + kWaves * 32 - 1) / (kWaves * 32) * 32;                // one piece for every wave, see above
    const int end = SPLIT ? min(a.steps, (wave + 1) * length) : a.steps;
    for (int base = SPLIT ? wave * length : 0; base < end; base += kRun) {
        typename Factor::Raw x[2][kAhead], w[BLOCKS][kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            const int k = base + 32 * q + 8 * quarter;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int row = 16 * r + i;
                if (whole) x[r][q] = Factor::fetch(xs, row, k, row < rows && k < end);
                else x[r][q] = Factor::load(data, t.lo + row, k, row < rows ? end - k : 0);
            }
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                const int r = 16 * b + i;
                if constexpr (DOWN) {
                    // eight values below each other, of 16 columns side by side; their bits as they are
                    uint32_t bits[8];
#pragma unroll
                    for (int s = 0; s < 8; ++s) {
                        const bool in = r < a.rank && k + s < end;
                        const uint32_t at = (uint32_t)((k + s) * a.rank + r) * (uint32_t)sizeof(E);
                        if constexpr (DT == kTypeF32) bits[s] = __builtin_amdgcn_raw_buffer_load_b32(down, (int)(in ? at : kOutside), 0, 0);
                        else bits[s] = __builtin_amdgcn_raw_buffer_load_b16(down, (int)(in ? at : kOutside), 0, 0);
                    }
#pragma unroll
                    for (int s = 0; s < 8; ++s) {
                        if constexpr (DT == kTypeF32) w[b][q].v[s] = __builtin_bit_cast(float, bits[s]);
                        else if (s % 2 == 0) w[b][q].v[s >> 1] = bits[s] | bits[s + 1] << 16;
                    }
                } else if (whole) {
                    w[b][q] = Factor::fetch(bs, r, k, r < a.rank && k < end);
                } else {
                    w[b][q] = Factor::load(matrix, r, k, r < a.rank ? end - k : 0);
                }
            }
        }
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            u32x4 xt[2][kTerms], wt[kTerms];
#pragma unroll
            for (int r = 0; r < 2; ++r) Factor::terms(x[r][q], xt[r]);
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                Factor::terms(w[b][q], wt);
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int p = 0; p < kTerms; ++p)
#pragma unroll
                        for (int o = 0; o < kTerms; ++o)
                            if (p + o < kTerms) acc[b][r] = mma16<kHalf>(wt[p], xt[r][o], acc[b][r]);
            }
        }
    }
    // lane: row 16 r + lane % 16, outputs 16 b + 4 (lane / 16) .. + 3
    if constexpr (SPLIT) {
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int v = 0; v < 4; ++v) part[wave][16 * b + 4 * quarter + v][16 * r + i] = acc[b][r][v];
        __syncthreads();
        for (int at = tid; at < 32 * a.rank; at += 512) {
            const int row = at / a.rank, r = at - row * a.rank;
            if (row >= rows) break;
            float z = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) z += part[w][r][row];
            a.u[(int64_t)t.lo * a.rank + at] = z * scale;
        }
    } else {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            if (16 * r + i >= rows) continue;
            float* out = a.u + (int64_t)(t.lo + 16 * r + i) * a.rank + 4 * quarter;
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                const v4f z = acc[b][r] * scale;
                if (a.rank % 4 == 0) {
                    if (16 * b + 4 * quarter < a.rank) *reinterpret_cast<v4f*>(out + 16 * b) = z;
                } else {
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        if (16 * b + 4 * quarter + v < a.rank) out[16 * b + v] = z[v];
                }
            }
        }
    }
}

// ---- layer inputs in 8 bits -------------------------------------------------------------------------------------------------------
// A thread has eight features of a row, four threads a block of 32: its largest magnitude decides the exponent, the smallest t at
// which it rounds to at most 127 steps of 2^t (t >= -126).  All of it is exact: x 2^-t is a change of exponent, the rounding to whole
// steps (ties to even) the only one.  Bound by the memory: 4 or 2 bytes read, 1.03 (1.16 with masks) written a feature.
template <int DT>
__global__ __launch_bounds__(256) void pack_kernel(const void* __restrict__ x, int64_t x_stride, int whole, int64_t n, int dim,
                                                   int8_t* __restrict__ q, uint8_t* __restrict__ e, uint32_t* __restrict__ masks) {
    typedef std::conditional_t<DT == kTypeF32, Wide<1>, Native> Factor;
    const int units = (dim + 31) / 32 * 4;
    const int64_t total = n * units, step = (int64_t)gridDim.x * 256;
    typename Factor::Pointer f;
    f.p = reinterpret_cast<decltype(f.p)>(x);
    f.stride = x_stride;
    f.whole = whole;
    for (int64_t base = (int64_t)blockIdx.x * 256; base < total; base += step) {
        const int64_t at = base + threadIdx.x;
        if (at >= total) break;                                            // whole groups of four lanes leave together
        const int64_t row = at / units;
        const int unit = (int)(at - row * units);
        f32x8 v;
        if (whole && 8 * unit < dim) {
            v = eight(reinterpret_cast<const typename TypeOf<DT>::Element*>(x) + row * x_stride + 8 * unit);
        } else {
            const typename Factor::Raw raw = Factor::load(f, row, 8 * unit, dim - 8 * unit);
            if constexpr (DT == kTypeF32) v = raw.v;
            else if constexpr (DT == kTypeF16) v = __builtin_convertvector(__builtin_bit_cast(h8, raw.v), f32x8);
            else v = __builtin_convertvector(__builtin_bit_cast(bf8, raw.v), f32x8);
        }
        // magnitudes as bit patterns: their order is the numbers', infinities and NaN on top
        uint32_t top = 0;
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const float vs = v[s];
            top = max(top, __builtin_bit_cast(uint32_t, vs) & 0x7fffffffu);
        }
        top = max(top, (uint32_t)__shfl_xor((int)top, 1));
        top = max(top, (uint32_t)__shfl_xor((int)top, 2));
        const bool finite = top < 0x7f800000u;
        const int biased = max((int)(top >> 23) - 6 + ((top & 0x7fffffu) >= 0x7f0000u ? 1 : 0), 1);     // t + 127
        const float inverse = __builtin_bit_cast(float, (uint32_t)(254 - min(biased, 253)) << 23);
        // where the 64th step is beyond the type's largest number
        const float most = biased == (DT == kTypeF16 ? 137 : 249) ? 63.f : 127.f;
        uint32_t bits = 0, word[2] = {0u, 0u};
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const float vs = v[s];
            bits |= (vs > 0.f ? 1u : 0u) << s;
            const float steps = fminf(fmaxf(__builtin_rintf(vs * inverse), -most), most);
            word[s >> 2] |= ((uint32_t)(int)(finite ? steps : 0.f) & 0xffu) << (8 * (s & 3));
        }
        const int64_t block = at >> 2;
        if (q) *reinterpret_cast<uint2*>(q + 8 * at) = make_uint2(word[0], word[1]);
        if (q && (unit & 3) == 0) e[block] = (uint8_t)(finite ? biased : 255);
        if (masks) {
            bits <<= 8 * (unit & 3);
            bits |= (uint32_t)__shfl_xor((int)bits, 1);
            bits |= (uint32_t)__shfl_xor((int)bits, 2);
            if ((unit & 3) == 0) masks[block] = bits;
        }
    }
}

template <int DT>
__global__ __launch_bounds__(256) void unpack_kernel(const int8_t* __restrict__ q, const uint8_t* __restrict__ e, int64_t n, int dim,
                                                     void* __restrict__ x, int64_t x_stride, int vec) {
    typedef typename TypeOf<DT>::Element E;
    typedef E E8 __attribute__((ext_vector_type(8)));
    const int units = (dim + 31) / 32 * 4;
    const int64_t total = n * units, step = (int64_t)gridDim.x * 256;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < total; at += step) {
        const int64_t row = at / units;
        const int col = 8 * (int)(at - row * units), room = dim - col;
        if (room <= 0) continue;
        const uint2 w = *reinterpret_cast<const uint2*>(q + 8 * at);
        const float scale = __builtin_bit_cast(float, (uint32_t)e[at >> 2] << 23);
        f32x8 v;
#pragma unroll
        for (int s = 0; s < 8; ++s) v[s] = signed_byte(s < 4 ? w.x : w.y, s & 3) * scale;
        E* p = reinterpret_cast<E*>(x) + row * x_stride + col;
        if (room >= 8 && vec) {
            *reinterpret_cast<E8*>(p) = __builtin_convertvector(v, E8);
        } else {
#pragma unroll
            for (int s = 0; s < 8; ++s)
                if (s < room) p[s] = (E)v[s];
        }
    }
}

// ---- launches ------------------------------------------------------------------------------------------------------------------------
template <int DT, bool BACKWARD, bool ADAPT, bool ONCE, int ROWS, int COLS, int WR, int WC>
void launch_tiles(RowsArgs a, hipStream_t st) {
    constexpr int kDepth = DT == kTypeF32 ? 32 : 64, kBufs = DT == kTypeF32 ? 1 : 2, kThreads = 64 * WR * WC;
    a.col_tiles = (a.cols + COLS - 1) / COLS;
    launch_blocks(row_tiles(a.groups, ROWS) * a.col_tiles, kThreads, [&](unsigned grid, int first) {
        a.first_block = first;
        rows_kernel<DT, BACKWARD, ADAPT, ONCE, ROWS, COLS, WR, WC, kDepth, kBufs><<<grid, kThreads, 0, st>>>(a);
    });
}

template <int DT, bool BACKWARD, bool ADAPT, bool ONCE>
int launch_rows(const RowsArgs& a, hipStream_t st) {
    if (!ADAPT && a.cols <= 64 && a.steps <= 64 && a.x_whole) {
        const int64_t tiles = row_tiles(a.groups, kNarrowRows);
        const unsigned grid = (unsigned)persistent_blocks((const void*)narrow_rows_kernel<DT, BACKWARD, ONCE>, 256, tiles);
        narrow_rows_kernel<DT, BACKWARD, ONCE><<<grid, 256, 0, st>>>(a);
    } else if (row_tiles(a.groups, 128) * ((a.cols + 127) / 128) < 2 * compute_units()) {
        // too few tiles of 128 x 128 to hide each other's waits (2048 to 2048: bf16 2^9 rows 24 us against 33, 2^11 rows 37 against 42, 2^12
        // rows 71 against 48; fp32 2^11 rows 133 against 144, 2^12 rows 262 against 184)
        launch_tiles<DT, BACKWARD, ADAPT, ONCE, 64, 64, 2, 1>(a, st);
    } else if (a.cols > 64) {
        launch_tiles<DT, BACKWARD, ADAPT, ONCE, 128, 128, 2, 2>(a, st);
    } else {
        launch_tiles<DT, BACKWARD, ADAPT, ONCE, 128, 64, 4, 1>(a, st);
    }
    return check_launch(BACKWARD ? "layer backward" : "layer forward");
}

template <int DT, bool BACKWARD>
int launch_rows(const RowsArgs& a, hipStream_t st) {
    if (a.rank > 0) return a.once ? launch_rows<DT, BACKWARD, true, true>(a, st) : launch_rows<DT, BACKWARD, true, false>(a, st);
    return a.once ? launch_rows<DT, BACKWARD, false, true>(a, st) : launch_rows<DT, BACKWARD, false, false>(a, st);
}

// The wide form wants rows and matrices in whole units, a contraction of whole lines, rows to fill its tiles with, and more tiles than
// half the compute units (2048 to 2048, bf16: 2^13 rows, 256 tiles, 64 us against 91 with tiles of 128 x 128; 2^12 rows, 128 tiles, 49
// against 48; 2^11 rows, 64 tiles, 47 against 37 with tiles of 64 x 64).
bool wide_rows_fit(int dtype, const RowsArgs& a) {
    return dtype != kTypeF32 && a.x_whole && rows_aligned(dtype, a.w_stride) && a.steps % 64 == 0 && a.cols >= 256 &&
           a.groups.n >= 128 * (a.groups.offsets && !a.groups.whole ? (int64_t)a.groups.groups : 2) &&
           row_tiles(a.groups, 256) * ((a.cols + 255) / 256) > compute_units() / 2;
}

template <bool BACKWARD>
int launch_rows(int dtype, const RowsArgs& args, hipStream_t st) {
    RowsArgs a = args;
    a.once = (int64_t)a.groups.n * a.cols * element_bytes(dtype) > kStoreOnceBytes;
    if (wide_rows_fit(dtype, a)) return launch_wide_rows(dtype, BACKWARD, a, st);
    if (dtype == kTypeF32) return launch_rows<kTypeF32, BACKWARD>(a, st);
    if (dtype == kTypeF16) return launch_rows<kTypeF16, BACKWARD>(a, st);
    return launch_rows<kTypeBF16, BACKWARD>(a, st);
}

int launch_few(int dtype, FewArgs a, hipStream_t st) {
    a.col_tiles = (a.cols + 15) / 16;
    launch_blocks(row_tiles(a.groups, 16) * a.col_tiles, 64 * kFewWaves, [&](unsigned grid, int first) {
        a.first_block = first;
        if (dtype == kTypeF32) few_rows_kernel<kTypeF32><<<grid, 64 * kFewWaves, 0, st>>>(a);
        else if (dtype == kTypeF16) few_rows_kernel<kTypeF16><<<grid, 64 * kFewWaves, 0, st>>>(a);
        else few_rows_kernel<kTypeBF16><<<grid, 64 * kFewWaves, 0, st>>>(a);
    });
    return check_launch("layer, few rows");
}

// Up to 16 rows a group the matrices are read once, and little else.  Up to 64 rows a group reading them once for every 16 rows, from
// a cache, still beats the tiles as long as the workgroups are few (2048 to 2048, one group of 64 rows: bf16 10 us against 23, fp32 19
// against 88; 8 groups of 1024 to 1024: bf16 32 rows each 13.5 against 18, 64 rows 24 against 18, fp32 64 rows 37 against 53).  Narrow layers have a kernel.
// Those are equal groups.  How the rows are spread is known on the device alone, so the rule goes by their mean: 64 groups of 2048 to
// 2048 with 1024 rows, equal ones bf16 169 against 137 with tiles, fp32 283 against 354; all rows in one group 137 against 40, 253 against 136.
bool few_rows_fit(const neus2_layer* l, const RowGroups& g) {
    if (g.n <= 16 * (int64_t)l->groups) return true;
    return g.n <= 64 * (int64_t)l->groups && (l->in_dim > 64 || l->out_dim > 64) &&
           row_tiles(g, 16) * ((l->out_dim + 15) / 16) <= (l->dtype == kTypeF32 ? 12 : 6) * compute_units();
}

RowGroups make_groups(const int32_t* offsets, int groups, int64_t n, bool whole) {
    RowGroups g;
    g.offsets = offsets;
    g.groups = groups;
    g.n = (int32_t)n;
    g.whole = whole ? 1 : 0;
    return g;
}

template <int DT, bool DOWN>
int launch_low_rank(LowRankArgs a, hipStream_t st) {
    // contractions of up to 256 steps are not worth sharing: every wave has rows of its own
    const bool split = a.steps > 256;
    launch_blocks(row_tiles(a.groups, split ? 32 : 256), 512, [&](unsigned grid, int first) {
        a.first_block = first;
        if (a.rank > 32) split ? low_rank_kernel<DT, DOWN, true, 4><<<grid, 512, 0, st>>>(a) : low_rank_kernel<DT, DOWN, false, 4><<<grid, 512, 0, st>>>(a);
        else if (a.rank > 16) split ? low_rank_kernel<DT, DOWN, true, 2><<<grid, 512, 0, st>>>(a) : low_rank_kernel<DT, DOWN, false, 2><<<grid, 512, 0, st>>>(a);
        else split ? low_rank_kernel<DT, DOWN, true, 1><<<grid, 512, 0, st>>>(a) : low_rank_kernel<DT, DOWN, false, 1><<<grid, 512, 0, st>>>(a);
    });
    return check_launch("adapter");
}

// u from x and A [slots][rank][steps], or v from dy and B [slots][steps][rank] (DOWN)
template <bool DOWN>
int launch_low_rank(const neus2_layer* l, const void* x, int64_t x_stride, const void* bank, const float* scales, const int32_t* slots,
                    const int32_t* offsets, int64_t n, int steps, float* u, hipStream_t st) {
    LowRankArgs a = {};
    a.groups = make_groups(offsets, l->groups, n, false);
    a.x = x;
    a.x_stride = x_stride;
    a.x_whole = rows_whole(l->dtype, x_stride, steps);
    a.bank = bank;
    a.bank_slot = (int64_t)l->rank * steps;
    a.bank_whole = rows_whole(l->dtype, steps, steps);
    a.steps = steps;
    a.rank = l->rank;
    a.slots = slots;
    a.n_slots = l->adapters;
    a.scales = scales;
    a.u = u;
    if (l->dtype == kTypeF32) return launch_low_rank<kTypeF32, DOWN>(a, st);
    if (l->dtype == kTypeF16) return launch_low_rank<kTypeF16, DOWN>(a, st);
    return launch_low_rank<kTypeBF16, DOWN>(a, st);
}

// ---- argument checks ------------------------------------------------------------------------------------------------------------------
int64_t x_stride_of(const neus2_layer* l) { return l->x_stride ? l->x_stride : l->in_dim; }
int64_t y_stride_of(const neus2_layer* l) { return l->y_stride ? l->y_stride : l->out_dim; }

int check_layer(const neus2_layer* l, bool adapters) {
    if (!l) return fail(NEUS2_ERR_NULL, "layer is NULL");
    if (l->dtype < 0 || l->dtype > 2) return fail(NEUS2_ERR_CONFIG, "dtype = %d, must be 0 (fp32), 1 (fp16) or 2 (bf16)", l->dtype);
    if (l->groups < 1 || l->groups > (1 << 16)) return fail(NEUS2_ERR_CONFIG, "groups = %d, must be 1..2^16", l->groups);
    if (l->in_dim < 1 || l->in_dim > (1 << 16)) return fail(NEUS2_ERR_CONFIG, "in_dim = %d, must be 1..65536", l->in_dim);
    if (l->out_dim < 1 || l->out_dim > (1 << 16)) return fail(NEUS2_ERR_CONFIG, "out_dim = %d, must be 1..65536", l->out_dim);
    if (l->x_stride != 0 && (l->x_stride < l->in_dim || l->x_stride > (1 << 24)))
        return fail(NEUS2_ERR_SHAPE, "x_stride = %lld, must be 0 or in_dim..2^24", (long long)l->x_stride);
    if (l->y_stride != 0 && (l->y_stride < l->out_dim || l->y_stride > (1 << 24)))
        return fail(NEUS2_ERR_SHAPE, "y_stride = %lld, must be 0 or out_dim..2^24", (long long)l->y_stride);
    if (l->relu != 0 && l->relu != 1) return fail(NEUS2_ERR_CONFIG, "relu = %d, must be 0 or 1", l->relu);
    if (l->accumulate != 0 && l->accumulate != 1) return fail(NEUS2_ERR_CONFIG, "accumulate = %d, must be 0 or 1", l->accumulate);
    if (adapters) {
        if (l->rank < 1 || l->rank > 64) return fail(NEUS2_ERR_UNSUPPORTED, "rank = %d, kernels exist for 1..64", l->rank);
        if (l->adapters < 1 || l->adapters > (1 << 16)) return fail(NEUS2_ERR_CONFIG, "adapters = %d, must be 1..2^16", l->adapters);
    } else if (l->rank != 0 || l->adapters != 0) {
        return fail(NEUS2_ERR_CONFIG, "rank = %d, adapters = %d: a grouped layer has no adapters", l->rank, l->adapters);
    }
    return NEUS2_OK;
}

int check_input(const void* x, const int8_t* xq, const uint8_t* xe, int64_t n) {
    if (x && (xq || xe)) return fail(NEUS2_ERR_CONFIG, "x and xq given: the layer's input is one or the other");
    if (xq || xe) {
        NEUS2_TRY(check_ptr(xq, "xq"));
        return check_ptr(xe, "xe");
    }
    return check_ptr(x, "x", n > 0);
}

}  // namespace
}  // namespace neus2

using namespace neus2;

extern "C" {

int neus2_grouped_fwd(const neus2_layer* l, const void* x, const void* W, const int32_t* offsets, int64_t n, void* y, void* stream) {
    NEUS2_TRY(check_layer(l, false));
    NEUS2_TRY(check_count(n, "n"));
    NEUS2_TRY(check_ptr(x, "x", n > 0));
    NEUS2_TRY(check_ptr(W, "W"));
    NEUS2_TRY(check_ptr(offsets, "offsets", l->groups > 1));
    NEUS2_TRY(check_ptr(y, "y", n > 0));
    if (n == 0) return NEUS2_OK;
    hipStream_t st = (hipStream_t)stream;
    const RowGroups groups = make_groups(offsets, l->groups, n, false);
    if (few_rows_fit(l, groups)) {
        FewArgs a = {};
        a.groups = groups;
        a.steps = l->in_dim; a.cols = l->out_dim;
        a.x = x; a.x_stride = x_stride_of(l); a.x_whole = rows_whole(l->dtype, a.x_stride, a.steps);
        a.w = W; a.w_group = (int64_t)l->in_dim * l->out_dim; a.w_stride = l->in_dim; a.w_whole = rows_whole(l->dtype, l->in_dim, l->in_dim);
        a.y = y; a.y_stride = y_stride_of(l);
        a.relu = l->relu;
        return launch_few(l->dtype, a, st);
    }
    RowsArgs a = {};
    a.groups = groups;
    a.steps = l->in_dim; a.cols = l->out_dim;
    a.x = x; a.x_stride = x_stride_of(l); a.x_whole = rows_whole(l->dtype, a.x_stride, a.steps);
    a.w = W; a.w_group = (int64_t)l->in_dim * l->out_dim; a.w_stride = l->in_dim; a.w_whole = rows_whole(l->dtype, l->in_dim, l->in_dim);
    a.y = y; a.y_stride = y_stride_of(l); a.y_vec = rows_aligned(l->dtype, a.y_stride);
    a.relu = l->relu;
    return launch_rows<false>(l->dtype, a, st);
}

int64_t neus2_grouped_workspace_bytes(const neus2_layer* l, int64_t n) {
    if (check_layer(l, false) != NEUS2_OK || check_count(n, "n") != NEUS2_OK) return -1;
    MatrixGradient m = {};
    m.groups = make_groups(nullptr, l->groups, n, false);
    m.dtype = l->dtype;
    m.outer = l->out_dim; m.inner = l->in_dim;
    // whether the input comes in 8 bits is not known here, and decides only together with its stride
    const int64_t sums = matrix_gradient_bytes(m), narrow = narrow_backward_bytes(l->in_dim, l->out_dim, l->groups);
    const bool fits = narrow_backward_fits(l->dtype, l->in_dim, l->out_dim, l->groups, n, y_stride_of(l), x_stride_of(l), true);
    return fits && narrow > sums ? narrow : sums;
}

int neus2_grouped_bwd(const neus2_layer* l, const void* x, const int8_t* xq, const uint8_t* xe, const uint32_t* masks, const void* W,
                      const int32_t* offsets, const void* dy, int64_t n, void* dx, float* dW, void* workspace, int64_t workspace_bytes,
                      void* stream) {
    NEUS2_TRY(check_layer(l, false));
    NEUS2_TRY(check_count(n, "n"));
    if (!dx && !dW && n > 0) return fail(NEUS2_ERR_NULL, "dx and dW are NULL: nothing to compute");
    if (dW) NEUS2_TRY(check_input(x, xq, xe, n));
    if (dx && n > 0) NEUS2_TRY(check_ptr(W, "W"));
    NEUS2_TRY(check_ptr(masks, "masks", false));
    NEUS2_TRY(check_ptr(offsets, "offsets", l->groups > 1));
    NEUS2_TRY(check_ptr(dy, "dy", n > 0));
    NEUS2_TRY(check_ptr(dx, "dx", false));
    NEUS2_TRY(check_ptr(dW, "dW", false));
    NEUS2_TRY(check_ptr(workspace, "workspace", false));
    const int64_t need = dW ? neus2_grouped_workspace_bytes(l, n) : 0;
    if (need > 0 && (!workspace || workspace_bytes < need))
        return fail(NEUS2_ERR_SHAPE, "workspace of %lld bytes, %lld are needed", (long long)(workspace ? workspace_bytes : 0), (long long)need);
    hipStream_t st = (hipStream_t)stream;
    RowsArgs a = {};
    a.groups = make_groups(offsets, l->groups, n, false);
    a.steps = l->out_dim; a.cols = l->in_dim;
    a.x = dy; a.x_stride = y_stride_of(l); a.x_whole = rows_whole(l->dtype, a.x_stride, a.steps);
    a.w = W; a.w_group = (int64_t)l->in_dim * l->out_dim; a.w_stride = l->in_dim; a.w_whole = rows_whole(l->dtype, l->in_dim, l->in_dim);
    a.y = dx; a.y_stride = x_stride_of(l); a.y_vec = rows_aligned(l->dtype, a.y_stride);
    a.masks = masks; a.mask_words = (l->in_dim + 31) / 32;
    a.once = n * l->in_dim * element_bytes(l->dtype) > kStoreOnceBytes;
    if (!dW) return n > 0 ? launch_rows<true>(l->dtype, a, st) : NEUS2_OK;
    MatrixGradient m = {};
    m.groups = a.groups;
    m.dtype = l->dtype;
    m.dy = dy; m.dy_stride = a.x_stride;
    m.x = x; m.x_stride = a.y_stride; m.xq = xq; m.xe = xe;
    m.outer = l->out_dim; m.inner = l->in_dim;
    m.out = dW; m.accumulate = l->accumulate;
    m.partial = (float*)workspace;
    // (the sums of dW alone come from the same kernel: the same bits with and without dx)
    if (narrow_backward_fits(l->dtype, l->in_dim, l->out_dim, l->groups, n, m.dy_stride, m.x_stride, xq != nullptr))
        return launch_narrow_backward(l->dtype, a, m, st);
    NEUS2_TRY(check_matrix_gradient(m));
    if (dx && n > 0) NEUS2_TRY(launch_rows<true>(l->dtype, a, st));
    return launch_matrix_gradient(m, st);
}

int neus2_adapter_fwd(const neus2_layer* l, const void* x, const void* W, const void* A, const void* B, const float* scales,
                      const int32_t* slots, const int32_t* offsets, int64_t n, float* u, void* y, void* stream) {
    NEUS2_TRY(check_layer(l, true));
    NEUS2_TRY(check_count(n, "n"));
    NEUS2_TRY(check_ptr(x, "x", n > 0));
    NEUS2_TRY(check_ptr(W, "W"));
    NEUS2_TRY(check_ptr(A, "A"));
    NEUS2_TRY(check_ptr(B, "B"));
    NEUS2_TRY(check_ptr(scales, "scales"));
    NEUS2_TRY(check_ptr(slots, "slots", false));
    NEUS2_TRY(check_ptr(offsets, "offsets"));
    NEUS2_TRY(check_ptr(u, "u", n > 0));
    NEUS2_TRY(check_ptr(y, "y", n > 0));
    if (n == 0) return NEUS2_OK;
    hipStream_t st = (hipStream_t)stream;
    NEUS2_TRY(launch_low_rank<false>(l, x, x_stride_of(l), A, scales, slots, offsets, n, l->in_dim, u, st));
    const RowGroups whole = make_groups(offsets, l->groups, n, true);
    // Few rows, up to 64 segments: a tile adds the adapters of its segments one after the other, few_rows_kernel a row's own (2048 to 2048,
    // rank 16, bf16, 64 segments, with u: 64 rows 17 us against 71 with tiles; beyond the limit 65 rows 20 against 72, 128 rows 26 against
    // 52, 256 rows 44 against 41; 16 rows in 16 segments 13 against 43; fp32 64 rows 32 against 164).
    if (n <= 64) {
        FewArgs a = {};
        a.groups = whole;
        a.steps = l->in_dim; a.cols = l->out_dim;
        a.x = x; a.x_stride = x_stride_of(l); a.x_whole = rows_whole(l->dtype, a.x_stride, a.steps);
        a.w = W; a.w_stride = l->in_dim; a.w_whole = rows_whole(l->dtype, l->in_dim, l->in_dim);
        a.y = y; a.y_stride = y_stride_of(l);
        a.relu = l->relu;
        a.segments = offsets; a.n_segments = l->groups; a.slots = slots; a.n_slots = l->adapters;
        a.u = u; a.bank = B; a.rank = l->rank;
        return launch_few(l->dtype, a, st);
    }
    RowsArgs a = {};
    a.groups = whole;
    a.steps = l->in_dim; a.cols = l->out_dim;
    a.x = x; a.x_stride = x_stride_of(l); a.x_whole = rows_whole(l->dtype, a.x_stride, a.steps);
    a.w = W; a.w_stride = l->in_dim; a.w_whole = rows_whole(l->dtype, l->in_dim, l->in_dim);
    a.y = y; a.y_stride = y_stride_of(l); a.y_vec = rows_aligned(l->dtype, a.y_stride);
    a.relu = l->relu;
    a.segments = offsets; a.n_segments = l->groups; a.slots = slots; a.n_slots = l->adapters;
    a.u = u; a.bank = B; a.rank = l->rank;
    return launch_rows<false>(l->dtype, a, st);
}

int64_t neus2_adapter_workspace_bytes(const neus2_layer* l, int64_t n) {
    if (check_layer(l, true) != NEUS2_OK || check_count(n, "n") != NEUS2_OK) return -1;
    const int64_t v = (n * l->rank * 4 + 15) / 16 * 16;
    MatrixGradient m = {};
    m.groups = make_groups(nullptr, l->groups, n, false);
    m.dtype = l->dtype;
    m.by_slot = true;
    m.outer = l->rank; m.inner = l->in_dim; m.left = m.right = (const float*)16;      // narrow sums, of fp32 factors
    const int64_t da = matrix_gradient_bytes(m);
    m.outer = l->out_dim; m.inner = l->rank;
    const int64_t db = matrix_gradient_bytes(m);
    return v + da + db;
}

int neus2_adapter_bwd(const neus2_layer* l, const void* x, const int8_t* xq, const uint8_t* xe, const uint32_t* masks, const void* W,
                      const void* A, const void* B, const float* scales, const int32_t* slots, const int32_t* offsets, const float* u,
                      const void* dy, int64_t n, void* dx, float* dA, float* dB, void* workspace, int64_t workspace_bytes, void* stream) {
    NEUS2_TRY(check_layer(l, true));
    NEUS2_TRY(check_count(n, "n"));
    if ((dA == nullptr) != (dB == nullptr)) return fail(NEUS2_ERR_NULL, "dA and dB: both or neither");
    if (!dx && !dA && n > 0) return fail(NEUS2_ERR_NULL, "dx, dA and dB are NULL: nothing to compute");
    if (dA) NEUS2_TRY(check_input(x, xq, xe, n));
    if (dx && n > 0) NEUS2_TRY(check_ptr(W, "W"));
    if (dx && n > 0) NEUS2_TRY(check_ptr(A, "A"));
    NEUS2_TRY(check_ptr(B, "B"));
    NEUS2_TRY(check_ptr(masks, "masks", false));
    NEUS2_TRY(check_ptr(scales, "scales"));
    NEUS2_TRY(check_ptr(slots, "slots", false));
    NEUS2_TRY(check_ptr(offsets, "offsets"));
    if (dB) NEUS2_TRY(check_ptr(u, "u", n > 0));
    NEUS2_TRY(check_ptr(dy, "dy", n > 0));
    NEUS2_TRY(check_ptr(dx, "dx", false));
    NEUS2_TRY(check_ptr(dA, "dA", false));
    NEUS2_TRY(check_ptr(dB, "dB", false));
    NEUS2_TRY(check_ptr(workspace, "workspace", n > 0 || dA));
    const int64_t need = neus2_adapter_workspace_bytes(l, n);
    if (workspace_bytes < need)
        return fail(NEUS2_ERR_SHAPE, "workspace of %lld bytes, %lld are needed", (long long)workspace_bytes, (long long)need);
    hipStream_t st = (hipStream_t)stream;
    float* v = (float*)workspace;
    float* partial = v + (n * l->rank * 4 + 15) / 16 * 4;
    if (n > 0) NEUS2_TRY(launch_low_rank<true>(l, dy, y_stride_of(l), B, scales, slots, offsets, n, l->out_dim, v, st));
    if (dx && n > 0) {
        RowsArgs a = {};
        a.groups = make_groups(offsets, l->groups, n, true);
        a.steps = l->out_dim; a.cols = l->in_dim;
        a.x = dy; a.x_stride = y_stride_of(l); a.x_whole = rows_whole(l->dtype, a.x_stride, a.steps);
        a.w = W; a.w_stride = l->in_dim; a.w_whole = rows_whole(l->dtype, l->in_dim, l->in_dim);
        a.y = dx; a.y_stride = x_stride_of(l); a.y_vec = rows_aligned(l->dtype, a.y_stride);
        a.masks = masks; a.mask_words = (l->in_dim + 31) / 32;
        a.segments = offsets; a.n_segments = l->groups; a.slots = slots; a.n_slots = l->adapters;
        a.u = v; a.bank = A; a.rank = l->rank;
        NEUS2_TRY(launch_rows<true>(l->dtype, a, st));
    }
    if (!dA) return NEUS2_OK;
    MatrixGradient m = {};
    m.groups = make_groups(offsets, l->groups, n, false);
    m.dtype = l->dtype;
    m.by_slot = true; m.slots = slots; m.n_slots = l->adapters;
    m.accumulate = l->accumulate;
    m.partial = partial;
    m.outer = l->rank; m.inner = l->in_dim;                    // dA[slot] = sum v x^T
    m.left = v;
    m.x = x; m.x_stride = x_stride_of(l); m.xq = xq; m.xe = xe;
    m.out = dA;
    MatrixGradient b = m;
    b.outer = l->out_dim; b.inner = l->rank;                   // dB[slot] = sum dy u^T
    b.left = nullptr; b.dy = dy; b.dy_stride = y_stride_of(l);
    b.right = u; b.x = nullptr; b.xq = nullptr; b.xe = nullptr;
    b.out = dB;
    b.partial = partial + matrix_gradient_bytes(m) / 4;
    return launch_adapter_gradients(m, b, st);
}

static int check_pack(int dtype, int64_t n, int32_t dim, int64_t x_stride) {
    if (dtype < 0 || dtype > 2) return fail(NEUS2_ERR_CONFIG, "dtype = %d, must be 0 (fp32), 1 (fp16) or 2 (bf16)", dtype);
    NEUS2_TRY(check_count(n, "n"));
    if (dim < 1 || dim > (1 << 16)) return fail(NEUS2_ERR_CONFIG, "dim = %d, must be 1..65536", dim);
    if (x_stride != 0 && (x_stride < dim || x_stride > (1 << 24)))
        return fail(NEUS2_ERR_SHAPE, "x_stride = %lld, must be 0 or dim..2^24", (long long)x_stride);
    return NEUS2_OK;
}

int neus2_pack8(int32_t dtype, const void* x, int64_t x_stride, int64_t n, int32_t dim, int8_t* q, uint8_t* e, uint32_t* masks, void* stream) {
    NEUS2_TRY(check_pack(dtype, n, dim, x_stride));
    NEUS2_TRY(check_ptr(x, "x", n > 0));
    const bool masks_only = masks && !q && !e;
    NEUS2_TRY(check_ptr(q, "q", n > 0 && !masks_only));
    NEUS2_TRY(check_ptr(e, "e", n > 0 && !masks_only));
    NEUS2_TRY(check_ptr(masks, "masks", false));
    if (n == 0) return NEUS2_OK;
    hipStream_t st = (hipStream_t)stream;
    const int64_t stride = x_stride ? x_stride : dim, blocks = (n * ((dim + 31) / 32 * 4) + 255) / 256;
    const unsigned grid = (unsigned)(blocks < 8 * compute_units() ? blocks : 8 * compute_units());
    const int whole = rows_aligned(dtype, stride) && dim % 8 == 0;
    if (dtype == kTypeF32) pack_kernel<kTypeF32><<<grid, 256, 0, st>>>(x, stride, whole, n, dim, q, e, masks);
    else if (dtype == kTypeF16) pack_kernel<kTypeF16><<<grid, 256, 0, st>>>(x, stride, whole, n, dim, q, e, masks);
    else pack_kernel<kTypeBF16><<<grid, 256, 0, st>>>(x, stride, whole, n, dim, q, e, masks);
    return check_launch("pack8");
}

int neus2_unpack8(int32_t dtype, const int8_t* q, const uint8_t* e, int64_t n, int32_t dim, void* x, int64_t x_stride, void* stream) {
    NEUS2_TRY(check_pack(dtype, n, dim, x_stride));
    NEUS2_TRY(check_ptr(q, "q", n > 0));
    NEUS2_TRY(check_ptr(e, "e", n > 0));
    NEUS2_TRY(check_ptr(x, "x", n > 0));
    if (n == 0) return NEUS2_OK;
    hipStream_t st = (hipStream_t)stream;
    const int64_t stride = x_stride ? x_stride : dim, blocks = (n * ((dim + 31) / 32 * 4) + 255) / 256;
    const unsigned grid = (unsigned)(blocks < 8 * compute_units() ? blocks : 8 * compute_units());
    const int vec = rows_aligned(dtype, stride);
    if (dtype == kTypeF32) unpack_kernel<kTypeF32><<<grid, 256, 0, st>>>(q, e, n, dim, x, stride, vec);
    else if (dtype == kTypeF16) unpack_kernel<kTypeF16><<<grid, 256, 0, st>>>(q, e, n, dim, x, stride, vec);
    else unpack_kernel<kTypeBF16><<<grid, 256, 0, st>>>(q, e, n, dim, x, stride, vec);
    return check_launch("unpack8");
}

}  // extern "C"
