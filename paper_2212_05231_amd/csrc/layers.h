// Building blocks of the layers whose rows choose their matrices (layers.hip, layers_grad.hip): where the rows of a group
// lie, and tiles of a product's two factors in LDS, ready for the 32x32x16 matrix instructions.
//
// Types.  bf16 and fp16 factors go to the matrix cores as they are, one instruction per k-step, accumulated in fp32.  fp32
// factors are sums of bf16 terms as in mfma_tile.h: three terms and six products, as accurate as an fp32 product.  Where a
// factor kept in fp32 (an adapter's u or v) meets one of 16 bits, the fp32 one takes three terms there too and an fp16 one two (8 + 8 >=
// 11 bits: exact), so that small gradients do not fall out of fp16's range.  An infinite factor that is split makes its products NaN (inf - inf).
#pragma once

#include "common.h"
#include "mfma_tile.h"

namespace neus2 {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

enum : int { kTypeF32 = 0, kTypeF16 = 1, kTypeBF16 = 2 };

template <int DT> struct TypeOf;
template <> struct TypeOf<kTypeF32> { typedef float Element; };
template <> struct TypeOf<kTypeF16> { typedef _Float16 Element; };
template <> struct TypeOf<kTypeBF16> { typedef __bf16 Element; };

// ---- groups of consecutive rows ----------------------------------------------------------------------------------------
// Group g owns rows offsets[g] .. offsets[g+1] - 1.  Offsets come from device memory, so whatever they hold is cut to 0..n
// here: a wrong one may leave rows out, it never leads outside the arrays.
struct RowGroups {
    const int32_t* offsets;     // NULL: one group, all n rows
    int32_t groups;
    int32_t n;
    int32_t whole;              // 1: the rows of all groups taken as one group (offsets[0] .. offsets[groups])
};

__device__ __forceinline__ void group_rows(const RowGroups& g, int e, int& lo, int& hi) {
    lo = 0;
    hi = g.n;
    if (g.offsets) {
        lo = min(max(g.offsets[e], 0), g.n);
        hi = max(min(g.offsets[g.whole ? g.groups : e + 1], g.n), lo);
    }
}

struct RowTile {
    int group;       // -1: no such tile
    int lo, hi;      // its rows
    int part, parts; // which part of the group's rows this is
    int index;       // tiles before this group's first one
    int end;         // where the group's rows end
    int shared;      // SHARED: those of groups of more than one tile among them
};

// inclusive sum over the lanes of a wave
__device__ __forceinline__ int wave_sums(int v, int lane) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int up = __shfl_up(v, d);
        if (lane >= d) v += up;
    }
    return v;
}

// Tile number `tile` when every group's rows are cut into tiles of `rows` rows, at least `least` (0 or 1) tiles a group.  All
// lanes of the wave take part: 64 groups at a time, one scan over the lanes, so up to 64 groups cost one load's latency.
template <bool SHARED = false>
__device__ __forceinline__ RowTile locate(const RowGroups& g, int rows, int least, int tile, int lane) {
    RowTile t;
    t.group = -1; t.lo = t.hi = t.end = t.part = t.parts = t.index = t.shared = 0;
    const int count = g.offsets && !g.whole ? g.groups : 1;
    int before = 0, shared_before = 0;
    for (int base = 0; base < count; base += 64) {
        const int e = base + lane;
        int lo = 0, hi = 0, tiles = 0;
        if (e < count) {
            group_rows(g, e, lo, hi);
            tiles = max((hi - lo + rows - 1) / rows, least);
        }
        const int sum = wave_sums(tiles, lane), mine = tiles > 1 ? tiles : 0;
        const int shared = SHARED ? wave_sums(mine, lane) : 0;
        const uint64_t past = __ballot(before + sum > tile);
        if (past) {
            const int at = __builtin_ctzll(past);
            t.group = base + at;
            lo = __builtin_amdgcn_readlane(lo, at);
            hi = __builtin_amdgcn_readlane(hi, at);
            t.parts = __builtin_amdgcn_readlane(tiles, at);
            t.index = before + __builtin_amdgcn_readlane(sum, at) - t.parts;
            if (SHARED) t.shared = shared_before + __builtin_amdgcn_readlane(shared - mine, at);
            t.part = tile - t.index;
            t.end = hi;
            t.lo = min(lo + t.part * rows, hi);
            t.hi = min(t.lo + rows, hi);
            return t;
        }
        before += __builtin_amdgcn_readlane(sum, 63);
        if (SHARED) shared_before += __builtin_amdgcn_readlane(shared, 63);
    }
    return t;
}

// The tile after t, which is number `tile`: of the same group without another look at the offsets.
__device__ __forceinline__ void locate_next(const RowGroups& g, int rows, int least, int tile, int lane, RowTile& t) {
    if (t.part + 1 < t.parts) {
        ++t.part;
        t.lo += rows;
        t.hi = min(t.lo + rows, t.end);
    } else {
        t = locate(g, rows, least, tile, lane);
    }
}

// How many tiles there are in all (locate's `rows` and `least`).  Offsets that are not ordered may count rows many times over: never
// more than the host has made room for (nor does locate count beyond that: it stops at the tile it looks for).
__device__ __forceinline__ int count_tiles(const RowGroups& g, int rows, int least, int lane) {
    const int count = g.offsets && !g.whole ? g.groups : 1;
    const int most = (g.n + rows - 1) / rows + count;
    int total = 0;
    for (int base = 0; base < count; base += 64) {
        const int e = base + lane;
        int lo = 0, hi = 0;
        if (e < count) {
            group_rows(g, e, lo, hi);
            total = min(total + max((hi - lo + rows - 1) / rows, least), most);      // 64 lanes of at most 2^24 + 2^16
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) total += __shfl_xor(total, d);
    total = __builtin_amdgcn_readfirstlane(total);
    return min(total, most);
}

// Workgroups go to the eight XCDs in turn, each with an L2 of its own.  Of `total` pieces of work in an order in which neighbours
// read the same memory, every XCD takes a run of consecutive ones, its workgroups in turn (the grid is a multiple of eight).
constexpr int kXcds = 8;
struct Pieces {
    int total, each, next_local, limit;
    __device__ __forceinline__ explicit Pieces(int count)
        : total(count), each((count + kXcds - 1) / kXcds), next_local((int)(blockIdx.x / kXcds)), limit(each) {}
    // the next one for this workgroup, or -1
    __device__ __forceinline__ int take() {
        const int local = next_local, piece = (int)(blockIdx.x % kXcds) * each + local;
        next_local += (int)(gridDim.x / kXcds);
        return local < limit && piece < total ? piece : -1;
    }
    // If the last round would leave half of an XCD's workgroups or more without a piece, it is taken out of those take() gives, and
    // take_quarter() deals out its pieces' quarters instead (piece * 4 + quarter, or -1).
    __device__ __forceinline__ void quarter_last_round() {
        const int at_once = (int)(gridDim.x / kXcds), rounds = each / at_once, left = each - rounds * at_once;
        if (rounds > 0 && left > 0 && 2 * left <= at_once) limit = rounds * at_once;
    }
    __device__ __forceinline__ int take_quarter(int& turn) const {
        const int at = (int)(blockIdx.x / kXcds) + turn * (int)(gridDim.x / kXcds);
        ++turn;
        if (at >= 4 * (each - limit)) return -1;
        return 4 * ((int)(blockIdx.x % kXcds) * each + limit + at / 4) + at % 4;
    }
};

// The segment a row lies in (the last one that begins at or before it), wave-uniform row; S segments.
__device__ __forceinline__ int segment_of(const int32_t* __restrict__ offsets, int segments, int row, int lane) {
    int at = 0;
    for (int base = 0; base < segments; base += 64) {
        const int s = base + lane;
        const bool ended = s < segments && offsets[s + 1] <= row;
        const int k = __popcll(__ballot(ended));
        at += k;
        if (k < 64) break;
    }
    return at;
}

// ---- factors ---------------------------------------------------------------------------------------------------------------
// A factor is read eight consecutive values at a time (a unit) and becomes kTerms words of eight 16-bit values.
__device__ __forceinline__ u32x4 zero4() { return u32x4{0u, 0u, 0u, 0u}; }

// LARGE: values above bf16's largest number (0.4 % below fp32's) take that as their first term, which rounding would make infinite; what is
// left comes with the others.  (So do infinities and NaN, of which infinities and NaN are left.)
template <int TERMS, bool LARGE = true>
__device__ __forceinline__ void split8(f32x8 v, u32x4 (&out)[TERMS]) {
    typedef int16_t s2 __attribute__((ext_vector_type(2)));
    typedef uint16_t u2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    typedef float f2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        float x0 = v[2 * p], x1 = v[2 * p + 1];
#pragma unroll
        for (int term = 0; term < TERMS; ++term) {
            uint32_t w = __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{x0, x1}, bf2));
            if (LARGE && term == 0) {
                w = __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(s2, w), s2{0x7f7f, 0x7f7f}));        // positive ones
                w = __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(u2, w), u2{0xff7f, 0xff7f}));        // negative ones
            }
            out[term][p] = w;
            x0 -= __builtin_bit_cast(float, w << 16);
            x1 -= __builtin_bit_cast(float, w & 0xffff0000u);
        }
    }
}

// Loads go through a window: an address range that begins at a uniform place and ends behind the last value that may be read.  A
// lane that has nothing to read gives an offset outside, and gets zeros without a branch around the load (with branches, every load
// waited for some forty scalar instructions).  Only whole units are read this way: `whole` in a factor's pointer says that memory
// rows begin on 16 bytes, are a multiple of eight values long, and no more than 2^20 values apart.  Otherwise values are read one by one.
constexpr uint32_t kOutside = 0x80000000u;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_window(const void* from, int64_t bytes) {
    const int room = (int)(bytes < 0 ? 0 : bytes > 0x7ffffff0 ? 0x7ffffff0 : bytes);
    return __builtin_amdgcn_make_buffer_rsrc((void*)from, 0, room, 0x00020000);
}

__device__ __forceinline__ u32x4 window16(__amdgpu_buffer_rsrc_t w, uint32_t offset) {
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(w, (int)offset, 0, 0));
}

// eight values from a place on 16 bytes, as floats
__device__ __forceinline__ f32x8 eight(const float* p) {
    const v4f a = *reinterpret_cast<const v4f*>(p), b = *reinterpret_cast<const v4f*>(p + 4);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ f32x8 eight(const _Float16* p) { return __builtin_convertvector(*reinterpret_cast<const h8*>(p), f32x8); }
__device__ __forceinline__ f32x8 eight(const __bf16* p) { return __builtin_convertvector(*reinterpret_cast<const bf8*>(p), f32x8); }

// 16-bit values as they are
struct Native {
    struct Raw { u32x4 v; };
    struct Pointer { const uint16_t* p; int64_t stride; int whole; };
    struct Window { __amdgpu_buffer_rsrc_t r; uint32_t stride; };
    static constexpr int kTerms = 1;
    // rows and length: how many memory rows there are from `row` on, and how many values in a row from `col` on
    __device__ static __forceinline__ Window window(const Pointer& f, int64_t row, int64_t col, int rows, int64_t length) {
        return {make_window(f.p + row * f.stride + col, rows > 0 ? ((rows - 1) * f.stride + length) * 2 : 0), (uint32_t)f.stride * 2u};
    }
    __device__ static __forceinline__ Raw fetch(const Window& w, int row, int col, bool in) {
        return {window16(w.r, in ? (uint32_t)row * w.stride + (uint32_t)col * 2u : kOutside)};
    }
    __device__ static __forceinline__ Raw load(const Pointer& f, int64_t row, int col, int valid) {
        Raw r;
        r.v = zero4();
        const uint16_t* p = f.p + row * f.stride + col;
#pragma unroll
        for (int s = 0; s < 8; ++s)
            if (s < valid) r.v[s >> 1] |= (uint32_t)p[s] << (16 * (s & 1));
        return r;
    }
    __device__ static __forceinline__ void terms(const Raw& r, u32x4 (&out)[1]) { out[0] = r.v; }
};

// fp32 values as TERMS bf16 terms
template <int TERMS>
struct Wide {
    struct Raw { f32x8 v; };
    struct Pointer { const float* p; int64_t stride; int whole; };
    struct Window { __amdgpu_buffer_rsrc_t r; uint32_t stride; };
    static constexpr int kTerms = TERMS;
    __device__ static __forceinline__ Window window(const Pointer& f, int64_t row, int64_t col, int rows, int64_t length) {
        return {make_window(f.p + row * f.stride + col, rows > 0 ? ((rows - 1) * f.stride + length) * 4 : 0), (uint32_t)f.stride * 4u};
    }
    __device__ static __forceinline__ Raw fetch(const Window& w, int row, int col, bool in) {
        const uint32_t at = in ? (uint32_t)row * w.stride + (uint32_t)col * 4u : kOutside;
        const v4f a = __builtin_bit_cast(v4f, window16(w.r, at)), b = __builtin_bit_cast(v4f, window16(w.r, at + 16u));
        return {__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7)};
    }
    __device__ static __forceinline__ Raw load(const Pointer& f, int64_t row, int col, int valid) {
        Raw r;
        const float* p = f.p + row * f.stride + col;
#pragma unroll
        for (int s = 0; s < 8; ++s) r.v[s] = s < valid ? p[s] : 0.f;
        return r;
    }
    __device__ static __forceinline__ void terms(const Raw& r, u32x4 (&out)[TERMS]) { split8<TERMS>(r.v, out); }
};

// fp16 values as two bf16 terms (exact)
struct HalfPair {
    typedef Native::Raw Raw;
    typedef Native::Pointer Pointer;
    typedef Native::Window Window;
    static constexpr int kTerms = 2;
    __device__ static __forceinline__ Window window(const Pointer& f, int64_t row, int64_t col, int rows, int64_t length) {
        return Native::window(f, row, col, rows, length);
    }
    __device__ static __forceinline__ Raw fetch(const Window& w, int row, int col, bool in) { return Native::fetch(w, row, col, in); }
    __device__ static __forceinline__ Raw load(const Pointer& f, int64_t row, int col, int valid) { return Native::load(f, row, col, valid); }
    __device__ static __forceinline__ void terms(const Raw& r, u32x4 (&out)[2]) {
        split8<2, false>(__builtin_convertvector(__builtin_bit_cast(h8, r.v), f32x8), out);
    }
};

__device__ __forceinline__ float signed_byte(uint32_t word, int byte) { return (float)((int)(word << (24 - 8 * byte)) >> 24); }

// 8-bit values with an exponent per 32 of them (neus2_pack8), as bf16 or fp16: q 2^(e-127) has at most 7 significant bits,
// exact in both.  e = 255 marks a block that held a value that was not finite: 0 * inf = NaN.  Its rows are always whole.
template <bool HALF>
struct Packed {
    struct Raw { uint32_t q[2]; uint32_t e; };
    struct Pointer { const int8_t* p; const uint8_t* e; int64_t stride; int whole; };     // stride: 32 * blocks
    struct Window { __amdgpu_buffer_rsrc_t q, e; uint32_t stride; };
    static constexpr int kTerms = 1;
    // col is a multiple of 32
    __device__ static __forceinline__ Window window(const Pointer& f, int64_t row, int64_t col, int rows, int64_t) {
        const int64_t at = row * f.stride + col, bytes = rows > 0 ? rows * f.stride - col : 0;
        return {make_window(f.p + at, bytes), make_window(f.e + (at >> 5), bytes >> 5), (uint32_t)f.stride};
    }
    __device__ static __forceinline__ Raw fetch(const Window& w, int row, int col, bool in) {
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        const uint32_t at = (uint32_t)row * w.stride + (uint32_t)col;
        const u32x2 q = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(w.q, (int)(in ? at : kOutside), 0, 0));
        return {{q[0], q[1]}, __builtin_amdgcn_raw_buffer_load_b8(w.e, (int)(in ? at >> 5 : kOutside), 0, 0)};
    }
    __device__ static __forceinline__ Raw load(const Pointer&, int64_t, int, int) { return {{0u, 0u}, 0u}; }
    __device__ static __forceinline__ void terms(const Raw& r, u32x4 (&out)[1]) {
        typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        typedef float f2 __attribute__((ext_vector_type(2)));
        const float step = __builtin_bit_cast(float, r.e << 23);
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const uint32_t w = r.q[p >> 1];
            const f2 v = {signed_byte(w, 2 * (p & 1)) * step, signed_byte(w, 2 * (p & 1) + 1) * step};
            out[0][p] = HALF ? __builtin_bit_cast(uint32_t, __builtin_convertvector(v, h2)) : __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf2));
        }
    }
};

// ---- tiles -----------------------------------------------------------------------------------------------------------------
// LINES lines of DEPTH steps of the contraction.  ALONG: the contraction runs along the memory rows (x and W in W x).  Planes of
// [line][DEPTH], a lane reads its eight steps as one 16-byte piece; piece p of a line lies at p ^ swizzle(line), so that sixteen
// consecutive lines of one piece cover all 64 banks once.  Otherwise (ACROSS) every memory row is one step of the contraction;
// planes of [DEPTH][line], read back transposed by ds_read_b64_tr_b16 (sixteen lanes read four rows of sixteen values, lane c
// gets column c); piece p of row k lies at p ^ across(k), so that the four rows of sixteen lanes fall on different banks, and so do
// those of thirty-two lanes.
template <int LINES>
__device__ __forceinline__ constexpr int across_swizzle(int k) {
    return LINES == 64 ? ((k & 2) << 1) | ((k & 1) << 1) : ((k & 1) << 2) | (k & 2) | ((k & 2) << 2);
}

template <class Factor, bool ALONG, int LINES, int DEPTH, int THREADS>
struct FactorTile {
    static constexpr int kTerms = Factor::kTerms;
    static constexpr int kPlane = LINES * DEPTH * 2;
    static constexpr int kBytes = kPlane * kTerms;
    static constexpr int kUnits = LINES * DEPTH / 8;
    static constexpr int kPer = (kUnits + THREADS - 1) / THREADS;
    static constexpr int kPieces = (ALONG ? DEPTH : LINES) / 8;
    static_assert(ALONG ? (DEPTH == 32 || DEPTH == 64) : LINES >= 64, "the swizzle needs whole sets of banks");
    typename Factor::Raw raw[kPer];

    __device__ static __forceinline__ int across(int k) { return across_swizzle<LINES>(k); }
    __device__ static __forceinline__ int swizzle(int line) { return DEPTH == 64 ? (line >> 1) & 7 : (line >> 2) & 3; }

    // line0, step0: where the tile begins; lines, steps: how many there are from there on (the rest is zero)
    __device__ __forceinline__ void load(const typename Factor::Pointer& f, int64_t line0, int lines, int64_t step0, int steps, int tid) {
        const int rows = ALONG ? min(lines, LINES) : min(steps, DEPTH), length = ALONG ? steps : lines;
        if (f.whole) {
            const typename Factor::Window w = Factor::window(f, ALONG ? line0 : step0, ALONG ? step0 : line0, rows, length);
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                const int unit = tid + k * THREADS, r = unit / kPieces, c = unit % kPieces * 8;
                raw[k] = Factor::fetch(w, r, c, r < rows && c < length && (kUnits % THREADS == 0 || unit < kUnits));
            }
        } else {
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                const int unit = tid + k * THREADS, r = unit / kPieces, c = unit % kPieces * 8;
                const bool in = r < rows && (kUnits % THREADS == 0 || unit < kUnits);
                raw[k] = Factor::load(f, (ALONG ? line0 : step0) + r, (int)(ALONG ? step0 : line0) + c, in ? length - c : 0);
            }
        }
    }
    __device__ __forceinline__ void store(unsigned char* __restrict__ lds, int tid) const {
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int unit = tid + k * THREADS;
            if (kUnits % THREADS != 0 && unit >= kUnits) break;
            const int r = unit / kPieces, piece = unit % kPieces;
            u32x4 t[kTerms];
            Factor::terms(raw[k], t);
            const int at = r * kPieces * 16 + ((piece ^ (ALONG ? swizzle(r) : across(r))) << 4);
#pragma unroll
            for (int term = 0; term < kTerms; ++term) *reinterpret_cast<u32x4*>(lds + term * kPlane + at) = t[term];
        }
    }
    // the operand of k-step ks (16 steps) for the 32 lines from 32 * block on
    __device__ static __forceinline__ u32x4 operand(const unsigned char* __restrict__ lds, int term, int block, int ks, int lane) {
        if (ALONG) {
            const int line = 32 * block + (lane & 31);
            return *reinterpret_cast<const u32x4*>(lds + term * kPlane + line * (DEPTH * 2) + (((2 * ks + (lane >> 5)) ^ swizzle(line)) << 4));
        } else {
            typedef short v4s __attribute__((ext_vector_type(4)));
            const int quad = (lane >> 2) & 3;
            const int piece = 4 * block + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
            const unsigned char* at = lds + term * kPlane + (16 * ks + 8 * (lane >> 5) + quad) * (LINES * 2) + ((piece ^ across(quad)) << 4) + (lane & 1) * 8;
            const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(at));
            const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(at + 4 * (LINES * 2)));
            return __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

template <bool HALF>
__device__ __forceinline__ v16f mma32(const u32x4& a, const u32x4& b, const v16f& c) {
    if (HALF) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
}

template <bool HALF>
__device__ __forceinline__ v4f mma16(const u32x4& a, const u32x4& b, const v4f& c) {
    if (HALF) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
}

// c += the products of the terms of a and b that count: together as far down as the finer factor's last term
template <bool HALF, int TA, int TB>
__device__ __forceinline__ v16f mma_terms(const u32x4 (&a)[TA], const u32x4 (&b)[TB], v16f c) {
    constexpr int kLast = (TA > TB ? TA : TB) - 1;
#pragma unroll
    for (int i = 0; i < TA; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j)
            if (i + j <= kLast) c = mma32<HALF>(a[i], b[j], c);
    return c;
}

// ---- conversions to the stored type -------------------------------------------------------------------------------------------
// Outputs of more than this are stored past the caches (ONCE; a template parameter, since the compiler makes one plain store of two
// branches that differ in the hint alone): the L2s of all XCDs hold 32 MB, and lines that are written back
// while others are read cost more than the next reader saves.  2^18 rows, 64 to 64, fp32 in 20 groups: 27 us against 37; 16384 x
// 2048 x 4096 in 8 groups: 283 against 297.
constexpr int64_t kStoreOnceBytes = 32 << 20;

// 16 bytes of a row; `room`: how many of their values lie inside the row; vec: rows begin on multiples of 16 bytes
template <class E, bool ONCE>
__device__ __forceinline__ void store_piece(E* p, const u32x4& v, int room, bool vec) {
    constexpr int kValues = 16 / (int)sizeof(E);
    typedef E Values __attribute__((ext_vector_type(kValues)));
    if (room >= kValues && vec) {
        if (ONCE) __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p));
        else *reinterpret_cast<u32x4*>(p) = v;
    } else {
        const Values w = __builtin_bit_cast(Values, v);
#pragma unroll
        for (int s = 0; s < kValues; ++s)
            if (s < room) p[s] = w[s];
    }
}

// zero below zero, NaN stays NaN
__device__ __forceinline__ float relu1(float z) { return z <= 0.f ? 0.f : z; }

// ---- rows through a matrix ---------------------------------------------------------------------------------------------------------
__device__ __forceinline__ int slot_of(const int32_t* __restrict__ slots, int n_slots, int segment) {
    const int s = slots ? slots[segment] : segment;
    return s >= 0 && s < n_slots ? s : -1;
}

struct RowsArgs {
    RowGroups groups;
    const void* x; int64_t x_stride; int x_whole;          // the data rows: x forward, dy backward
    const void* w; int64_t w_group; int w_stride, w_whole; // matrix of group g at w + g * w_group, memory rows of w_stride values
    int steps;                                             // length of the contraction
    int cols;                                              // outputs per row
    void* y; int64_t y_stride; int y_vec; int once;
    int relu;
    const uint32_t* masks; int mask_words;                 // NULL, or: outputs whose bit is not set are zero
    // adapters: y += bank[slot] u for the rows of each segment
    const int32_t* segments; int n_segments;
    const int32_t* slots; int n_slots;
    const float* u; const void* bank; int rank;
    int col_tiles;
    int first_block;                 // workgroups launched before (launch_blocks)
};

// The number of bf16 terms an adapter's fp32 u and its bank matrix take in y += bank u.  Two for u would be enough for a sum that is
// rounded to 16 bits, but not where W x and bank u cancel: there the difference is what they leave out.
template <int DT> struct AdapterTerms {
    static constexpr int kU = 3;
    static constexpr int kBank = DT == kTypeF32 ? 3 : DT == kTypeF16 ? 2 : 1;
};

// eight values of row `row` (k .. k + 7 of `rank`) of a window over u, zeros where the row counts for nothing
__device__ __forceinline__ f32x8 load_u(__amdgpu_buffer_rsrc_t u, int row, int rank, int k, bool counts) {
    f32x8 v;
    const uint32_t at = (uint32_t)(row * rank + k) * 4u;
    if ((rank & 7) == 0) {
        const bool in = counts && k < rank;
        const v4f a = __builtin_bit_cast(v4f, window16(u, in ? at : kOutside)), b = __builtin_bit_cast(v4f, window16(u, in ? at + 16u : kOutside));
        v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
#pragma unroll
        for (int s = 0; s < 8; ++s)
            v[s] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(u, (int)(counts && k + s < rank ? at + 4u * s : kOutside), 0, 0));
    }
    return v;
}

// eight values bank(col, k .. k + 7) of a window over one adapter's matrix, as they lie in memory: along the memory row forward (bank
// [col][rank]), down the column backward ([rank][cols])
template <int DT> struct BankRaw { u32x4 v[DT == kTypeF32 ? 2 : 1]; };

template <int DT, bool BACKWARD>
__device__ __forceinline__ BankRaw<DT> request_bank(__amdgpu_buffer_rsrc_t bank, int rank, int cols, int col, int k) {
    constexpr uint32_t kBytes = DT == kTypeF32 ? 4 : 2;
    BankRaw<DT> raw;
    if (!BACKWARD && (rank & 7) == 0) {
        const uint32_t at = (uint32_t)(col * rank + k) * kBytes;
        const bool in = col < cols && k < rank;
        raw.v[0] = window16(bank, in ? at : kOutside);
        if constexpr (DT == kTypeF32) raw.v[1] = window16(bank, in ? at + 16u : kOutside);
    } else {
        uint32_t bits[8];
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const uint32_t at = (uint32_t)(BACKWARD ? (k + s) * cols + col : col * rank + k + s) * kBytes;
            const bool in = col < cols && k + s < rank;
            if constexpr (DT == kTypeF32) bits[s] = __builtin_amdgcn_raw_buffer_load_b32(bank, (int)(in ? at : kOutside), 0, 0);
            else bits[s] = __builtin_amdgcn_raw_buffer_load_b16(bank, (int)(in ? at : kOutside), 0, 0);
        }
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            if constexpr (DT == kTypeF32) raw.v[s >> 2][s & 3] = bits[s];
            else if (s % 2 == 0) raw.v[0][s >> 1] = bits[s] | bits[s + 1] << 16;
        }
    }
    return raw;
}

template <int DT>
__device__ __forceinline__ void bank_terms(const BankRaw<DT>& raw, u32x4 (&out)[AdapterTerms<DT>::kBank]) {
    if constexpr (DT == kTypeF32) {
        split8<3>(__builtin_shufflevector(__builtin_bit_cast(v4f, raw.v[0]), __builtin_bit_cast(v4f, raw.v[1]), 0, 1, 2, 3, 4, 5, 6, 7), out);
    } else if constexpr (DT == kTypeF16) {
        split8<2, false>(__builtin_convertvector(__builtin_bit_cast(h8, raw.v[0]), f32x8), out);
    } else {
        out[0] = raw.v[0];
    }
}

template <int DT>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t bank_window(const void* bank, int slot, int rank, int cols) {
    typedef typename TypeOf<DT>::Element E;
    const int64_t size = (int64_t)rank * cols;
    return make_window(reinterpret_cast<const E*>(bank) + slot * size, size * (int64_t)sizeof(E));
}

// The segments from number `base` on, one a lane: fetched before the contraction, so that what follows it waits for none of this.
struct Segments {
    int base, lo, hi, slot;
    __device__ __forceinline__ void fetch(const RowsArgs& a, int from, int lane) {
        base = from;
        const int s = from + lane;
        lo = hi = 0x7fffffff;
        slot = -1;
        if (s < a.n_segments) {
            lo = a.segments[s];
            hi = a.segments[s + 1];
            slot = slot_of(a.slots, a.n_slots, s);
        }
    }
    __device__ __forceinline__ void begin(const RowsArgs& a, const RowTile& t, int lane) {
        fetch(a, segment_of(a.segments, a.n_segments, t.lo, lane), lane);
    }
};

// What follows the contraction, for one wave's kBC x kBR blocks of 32 outputs (from col0 on) and 32 rows (from t.lo + row0 on).  A
// lane holds four times four consecutive outputs of one row in each block.  lds: kBC * 1024 values for each wave, of which nobody
// reads anything any more.
// before_stores: called before the first of them.
template <int DT, bool BACKWARD, bool ADAPT, int kBC, int kBR, bool ONCE, class BeforeStores>
__device__ __forceinline__ void finish_rows(const RowsArgs& a, const RowTile& t, Segments segments, int col0, int row0, v16f (&acc)[kBC][kBR],
                                            unsigned char* lds, int wave, int lane, BeforeStores before_stores) {
    typedef typename TypeOf<DT>::Element E;
    const int j = lane & 31, h = lane >> 5;
    if (ADAPT) {
        // y += bank[slot] u, segment after segment: operands straight from memory (a lane's eight values lie together), the rows of
        // other segments zero.  A tile inside one segment takes rank / 16 more k-steps.
        constexpr int kU = AdapterTerms<DT>::kU, kBank = AdapterTerms<DT>::kBank;
        const __amdgpu_buffer_rsrc_t us = make_window(a.u + (int64_t)t.lo * a.rank, (int64_t)(t.hi - t.lo) * a.rank * 4);
        for (int i = 0;; ++i) {
            if (i == 64) {
                segments.fetch(a, segments.base + 64, lane);
                i = 0;
            }
            const int lo = max(__builtin_amdgcn_readlane(segments.lo, i), t.lo), hi = min(__builtin_amdgcn_readlane(segments.hi, i), t.hi);
            if (lo >= t.hi) break;
            const int slot = hi > lo ? __builtin_amdgcn_readlane(segments.slot, i) : -1;
            if (slot < 0) continue;
            const __amdgpu_buffer_rsrc_t bank = bank_window<DT>(a.bank, slot, a.rank, a.cols);
            for (int k0 = 0; k0 < a.rank; k0 += 16) {
                // the bank's operands are all requested before the first is used
                BankRaw<DT> raw[kBC];
#pragma unroll
                for (int c = 0; c < kBC; ++c) raw[c] = request_bank<DT, BACKWARD>(bank, a.rank, a.cols, col0 + 32 * c + j, k0 + 8 * h);
                u32x4 u[kBR][kU];
#pragma unroll
                for (int r = 0; r < kBR; ++r) {
                    const int row = t.lo + row0 + 32 * r + j;
                    split8<kU>(load_u(us, row - t.lo, a.rank, k0 + 8 * h, row >= lo && row < hi), u[r]);
                }
#pragma unroll
                for (int c = 0; c < kBC; ++c) {
                    u32x4 b[kBank];
                    bank_terms<DT>(raw[c], b);
#pragma unroll
                    for (int r = 0; r < kBR; ++r) {
                        const int first = t.lo + row0 + 32 * r;
                        if (first >= hi || first + 32 <= lo) continue;
                        const v16f sum = mma_terms<false>(b, u[r], acc[c][r]);
                        // an infinite or NaN value of this adapter is nothing to the other segments' rows (0 * inf)
                        const bool in = (first >= lo && first + 32 <= hi) || (first + j >= lo && first + j < hi);
#pragma unroll
                        for (int e = 0; e < 16; ++e) acc[c][r][e] = in ? sum[e] : acc[c][r][e];
                    }
                }
            }
        }
    }
    // A block of 32 rows goes through this wave's part of LDS, so that the stores cover whole lines: a lane's four outputs of a row lie
    // 8 or 16 bytes wide in memory, and stored as they are they took a third of the time of a wide layer (16384 x 2048 x 4096: 318 us
    // against 217 without any stores).  Pieces of 16 bytes (and the halves of 8 in them) are spread over the banks by row.
    typedef E E4 __attribute__((ext_vector_type(4)));
    constexpr int kRowBytes = kBC * 32 * (int)sizeof(E), kPieces = kRowBytes / 16, kRowsAtOnce = 64 / kPieces;
    constexpr int kValues = 16 / (int)sizeof(E);                         // in a piece
    static_assert(kRowBytes == 128 || kRowBytes == 256, "the spreading needs rows of half a set of banks or a whole one");
    unsigned char* mine = lds + wave * 32 * kRowBytes;
    auto spread = [&](int row) { return kPieces == 16 ? row & 15 : (row >> 1) & 7; };
#pragma unroll
    for (int r = 0; r < kBR; ++r) {
        const int first = t.lo + row0 + 32 * r, row = min(first + j, t.hi - 1);
#pragma unroll
        for (int c = 0; c < kBC; ++c) {
            const int block = min(col0 + 32 * c, a.cols - 1) & ~31;
            const uint32_t mask = a.masks ? a.masks[(int64_t)row * a.mask_words + (block >> 5)] : 0xffffffffu;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                v4f v;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float z = acc[c][r][4 * g + e];
                    v[e] = (mask >> (8 * g + 4 * h + e)) & 1u ? (a.relu ? relu1(z) : z) : 0.f;
                }
                const E4 rounded = __builtin_convertvector(v, E4);       // to the nearest, ties to even
                const int quad = 8 * c + 2 * g + h;                      // of four outputs
                if constexpr (sizeof(E) == 4) *reinterpret_cast<E4*>(mine + j * kRowBytes + ((quad ^ spread(j)) << 4)) = rounded;
                else *reinterpret_cast<E4*>(mine + j * kRowBytes + (((quad >> 1) ^ spread(j)) << 4) + (((quad ^ (j >> 4)) & 1) << 3)) = rounded;
            }
        }
        wave_lds_fence();
        if (r == 0) before_stores();
#pragma unroll
        for (int q = 0; q < 32 / kRowsAtOnce; ++q) {
            const int at = kRowsAtOnce * q + lane / kPieces, piece = lane % kPieces, col = col0 + piece * kValues;
            u32x4 v = *reinterpret_cast<const u32x4*>(mine + at * kRowBytes + ((piece ^ spread(at)) << 4));
            if (sizeof(E) == 2 && q >= 16 / kRowsAtOnce) v = __builtin_shufflevector(v, v, 2, 3, 0, 1);
            if (first + at < t.hi) store_piece<E, ONCE>(reinterpret_cast<E*>(a.y) + (int64_t)(first + at) * a.y_stride + col, v, a.cols - col, a.y_vec);
        }
        wave_lds_fence();
    }
}

// ---- sums over rows -----------------------------------------------------------------------------------------------------------
struct SumArgs {
    RowGroups groups;
    int chunk;                       // rows a workgroup sums over
    const void* left; int64_t left_stride; int left_whole;
    const void* right; const uint8_t* right_e; int64_t right_stride; int right_whole;
    int outer, inner;
    float* out; int accumulate; int once;
    float* partial;                  // [partials][outer][inner]: sums of chunks, of all of them (by_slot) or of those that share a group
    int partials;
    int by_slot;
    int outer_tiles, inner_tiles;
    int first_block;
};

// Where a chunk's sums belong, and whether they are added to what is there; NULL: nowhere.
__device__ __forceinline__ float* sums_place(const SumArgs& a, const RowTile& t, bool& add) {
    const int64_t size = (int64_t)a.outer * a.inner;
    add = false;
    if (!a.by_slot && t.parts == 1) {
        add = a.accumulate != 0;
        return a.out + t.group * size;
    }
    const int index = (a.by_slot ? t.index : t.shared) + t.part;
    return t.hi > t.lo && index >= 0 && index < a.partials ? a.partial + index * size : nullptr;     // decreasing offsets may count too many
}

template <bool ONCE, int kBO, int kBI>
__device__ __forceinline__ void store_sums(const SumArgs& a, const RowTile& t, int outer0, int inner0, v16f (&acc)[kBO][kBI], int lane) {
    bool add;
    float* out = sums_place(a, t, add);
    if (!out) return;
    const int j = lane & 31, h = lane >> 5;
#pragma unroll
    for (int i = 0; i < kBI; ++i) {
        const int col = inner0 + 32 * i + j;
        if (col >= a.inner) continue;
#pragma unroll
        for (int o = 0; o < kBO; ++o)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = outer0 + 32 * o + neuron_of(r, h);
                if (row >= a.outer) continue;
                float* p = out + (int64_t)row * a.inner + col;
                const float v = acc[o][i][r];
                if (ONCE && !add) __builtin_nontemporal_store(v, p);
                else *p = add ? *p + v : v;
            }
    }
}

constexpr int kWideOuter = 256, kWideInner = 256;       // their tiles
void launch_wide_sums(int dtype, bool packed, const SumArgs& a, int64_t blocks, hipStream_t st);
int launch_wide_rows(int dtype, bool backward, const RowsArgs& a, hipStream_t st);      // 16-bit types, whole lines of the contraction

// ---- host side ----------------------------------------------------------------------------------------------------------------
// out[g] (+)= sum over the rows of group g of left_i right_i^T, out [groups][outer][inner] fp32.  left is dy (of the layer's type) or
// an adapter's v (fp32, dense rows); right is x, x in 8 bits, or an adapter's u.  by_slot: the sums of all segments that share a
// slot go to that slot's matrix, and slots without rows count as empty groups.
struct MatrixGradient {
    RowGroups groups;
    int dtype;
    const float* left; const void* dy; int64_t dy_stride;
    const float* right; const void* x; int64_t x_stride; const int8_t* xq; const uint8_t* xe;
    int outer, inner;
    float* out; int accumulate;
    float* partial;
    bool by_slot; const int32_t* slots; int n_slots;
};
int64_t matrix_gradient_bytes(const MatrixGradient& m);
int check_matrix_gradient(const MatrixGradient& m);      // whether launch_matrix_gradient has numbers for all workgroups
int launch_matrix_gradient(const MatrixGradient& m, hipStream_t st);
bool narrow_backward_fits(int dtype, int inner, int outer, int64_t groups, int64_t n, int64_t dy_stride, int64_t x_stride, bool packed);
int64_t narrow_backward_bytes(int inner, int outer, int64_t groups);
int launch_narrow_backward(int dtype, const RowsArgs& rows, const MatrixGradient& m, hipStream_t st);      // rows.y NULL: no dx
int launch_adapter_gradients(const MatrixGradient& da, const MatrixGradient& db, hipStream_t st);       // by slot both

inline int element_bytes(int dtype) { return dtype == kTypeF32 ? 4 : 2; }

// rows of `stride` values begin on 16-byte boundaries
inline int rows_aligned(int dtype, int64_t stride) { return (stride * element_bytes(dtype)) % 16 == 0; }

// ... and are read in whole units of eight values, through 32-bit offsets
inline int rows_whole(int dtype, int64_t stride, int64_t length) { return rows_aligned(dtype, stride) && length % 8 == 0 && stride <= (1 << 20); }

// at most this many tiles of at least one row
inline int64_t row_tiles(const RowGroups& g, int rows) {
    const int64_t tiles = ((int64_t)g.n + rows - 1) / rows + (g.offsets && !g.whole ? g.groups : 0);
    return tiles < g.n ? tiles : g.n;
}

// A launch has fewer than 2^32 threads in a dimension: more workgroups than that go in several launches, go(grid, first) each, and a
// kernel's block number is first + blockIdx.x.  Numbers stay below 2^31: 2^28 rows in tiles of 128 beside 2^16 groups and 2^16 outputs in
// tiles of 128 are 2^30.1; tiles of 64 and 16 are taken for few tiles or rows only; the sums of matrices check theirs.
constexpr int64_t kMostThreads = 0xffffffffll;

template <class Go>
inline void launch_blocks(int64_t blocks, int threads, const Go& go) {
    const int64_t most = kMostThreads / threads;
    for (int64_t first = 0; first < blocks; first += most) go((unsigned)(blocks - first < most ? blocks - first : most), (int)first);
}

}  // namespace neus2
