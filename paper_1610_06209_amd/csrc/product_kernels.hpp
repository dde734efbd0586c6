// Matrix products of grouped rows on the matrix pipe: tiles through LDS, and the form for a few rows.
//
// In every product a wave multiplies 32 rows by 32 columns over a depth of 32 bytes an instruction: 16 numbers of 16 bits
// (v_mfma_f32_32x32x16) or 64 of 4 bits (v_mfma_scale_f32_32x32x64, e2m1 with an e8m0 scale for each 32), 16 bytes a lane from
// either operand.  So one kernel moves bytes for all types, and what differs is the instruction and the scales.
#pragma once
#include "mx4.hpp"
#include "number_io.hpp"
#include "spinner_kernels.hpp"

namespace spinner {

typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef int intx8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// what lies beyond an operand's end reads as this
__device__ const uintx4 zero_piece = {0, 0, 0, 0};

// ------------------------------------------------------------------ groups of rows
// inclusive sum / maximum over the lanes up to each one, of numbers >= 0
template <typename F>
__device__ __forceinline__ int wave_scan(int v, F op)
{
    v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false));     // row_shr:1, :2, :4, :8
    v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false));
    v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false));
    v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false));
    v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false));     // row_bcast:15 to rows 1 and 3
    v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false));     // row_bcast:31 to rows 2 and 3
    return v;
}
struct AddInts { __device__ __forceinline__ int operator()(int a, int b) const { return a + b; } };
struct MaxInts { __device__ __forceinline__ int operator()(int a, int b) const { return a > b ? a : b; } };

// Where 64 groups lie, one a lane: the ends as they are in memory, held between 0 and `rows` and made to rise, so that no
// contents of `ends` reach outside the operands.  `before`: the end of the group before the first.
struct Groups {
    int lo, hi;
    __device__ __forceinline__ Groups(const long long* ends, int first, int experts, int rows, int before, int lane)
    {
        const int e = first + lane;
        long long v = e < experts ? ends[e] : rows;        // behind the experts: the rows of no group, then nothing
        v = v < 0 ? 0 : (v > rows ? rows : v);
        int h = (int)v;
        h = h > before ? h : before;
        hi = wave_scan(h, MaxInts{});
        const int left = __builtin_amdgcn_update_dpp(before, hi, 0x138, 0xF, 0xF, false);        // wave_shr:1, lane 0 keeps `before`
        lo = left;
    }
};

struct RowTile {
    int expert;           // `experts` for the rows of no group
    int lo, hi;           // rows of the group from this tile's first on
};
// Row tiles of BM rows, group after group (the rows of no group last): how many, and one of them.
template <int BM>
struct RowTiles {
    const long long* ends;
    int experts, rows, lane;
    int total;
    // of the last 64 groups that were looked at (all there are, up to 63 experts)
    int lo, hi, upto;
    __device__ __forceinline__ RowTiles(const ProductParams& p) : ends(p.ends), experts(p.experts), rows(p.rows), lane(threadIdx.x & 63)
    {
        if (!ends) {
            total = (rows + BM - 1) / BM;
            return;
        }
        int before = 0;
        total = 0;
        for (int first = 0; first <= experts; first += 64) look(first, before);
    }
    __device__ __forceinline__ void look(int first, int& before)
    {
        const Groups g(ends, first, experts, rows, before, lane);
        lo = g.lo;
        hi = g.hi;
        upto = total + wave_scan((hi - lo + BM - 1) / BM, AddInts{});
        before = __builtin_amdgcn_readlane(hi, 63);
        total = __builtin_amdgcn_readlane(upto, 63);
    }
    // tile `t` < total
    __device__ __forceinline__ RowTile find(int t)
    {
        if (!ends) return {0, t * BM, rows};
        int first = 0;
        if (experts >= 64) {
            int before = 0;
            total = 0;
            look(0, before);
            while (total <= t && first + 64 <= experts) look(first += 64, before);
        }
        const int at = __builtin_ctzll(__ballot(upto > t));
        const int tiles = (__builtin_amdgcn_readlane(hi, at) - __builtin_amdgcn_readlane(lo, at) + BM - 1) / BM;
        const int k = t - (__builtin_amdgcn_readlane(upto, at) - tiles);
        return {first + at, __builtin_amdgcn_readlane(lo, at) + k * BM, __builtin_amdgcn_readlane(hi, at)};
    }
};

// the run of a whole order of `total` tiles that an XCD takes, in turn: workgroups go to the eight XCDs in turn, and tiles that are
// neighbours in the order share operands in the L2 of theirs.  false: nothing left for this workgroup.
__device__ __forceinline__ bool xcd_run(unsigned block, unsigned total, unsigned* tile)
{
    const unsigned xcd = block & 7, k = block >> 3, longer = total & 7;
    if (k >= (total >> 3) + (xcd < longer ? 1 : 0)) return false;
    *tile = xcd * (total >> 3) + (xcd < longer ? xcd : longer) + k;
    return true;
}

// ------------------------------------------------------------------ one instruction
template <int TYPE>
__device__ __forceinline__ floatx16 multiply32(uintx4 a, uintx4 b, floatx16 c)
{
    if constexpr (TYPE == kBf16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ intx8 fp4_operand(uintx4 a)
{
    return intx8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
}
// BYTE: which byte of the scale words
template <int BYTE>
__device__ __forceinline__ floatx16 multiply32_scaled(uintx4 a, uintx4 b, floatx16 c, unsigned sa, unsigned sb)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fp4_operand(a), fp4_operand(b), c, 4, 4, BYTE, (int)sa, BYTE, (int)sb);
}
template <int TYPE>
__device__ __forceinline__ floatx4 multiply16(uintx4 a, uintx4 b, floatx4 c)
{
    if constexpr (TYPE == kBf16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ floatx4 multiply16_scaled(uintx4 a, uintx4 b, floatx4 c, unsigned sa, unsigned sb)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fp4_operand(a), fp4_operand(b), c, 4, 4, 0, (int)sa, 0, (int)sb);
}

// ------------------------------------------------------------------ results
// four neighbours of a row, `left` of them inside it
template <typename Out>
__device__ __forceinline__ void store_four(Out* p, float a, float b, float c, float d, int left, bool vector)
{
    if (vector && left >= 4) {
        if constexpr (sizeof(Out) == 4) {
            *reinterpret_cast<floatx4*>(p) = floatx4{a, b, c, d};
        } else {
            const uint2 t = {Piece<Out>::narrow(a, b), Piece<Out>::narrow(c, d)};
            *reinterpret_cast<uint2*>(p) = t;
        }
        return;
    }
    if (left > 0) p[0] = (Out)a;
    if (left > 1) p[1] = (Out)b;
    if (left > 2) p[2] = (Out)c;
    if (left > 3) p[3] = (Out)d;
}

// up to eight 16-bit numbers from an address of any alignment, zeros behind them
__device__ __forceinline__ uintx4 fetch_some(const char* p, int count)
{
    if (count >= 8) {
        const Bytes16 t = *reinterpret_cast<const Bytes16*>(p);
        return uintx4{t.w[0], t.w[1], t.w[2], t.w[3]};
    }
    uintx4 v = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < count) v[i >> 1] |= (unsigned)reinterpret_cast<const unsigned short*>(p)[i] << (16 * (i & 1));
    return v;
}

// ------------------------------------------------------------------ tiles
constexpr int kChunkBytes = 128;                          // of a row's depth in LDS at a time
constexpr int kChunkPieces = kChunkBytes / 16;
constexpr int kChunkDepth16 = kChunkBytes / 2;            // the same in 16-bit numbers
constexpr int kChunkScales = kChunkBytes / 16;            // scales of a row's chunk: 32 numbers are 16 bytes

// An operand's part of a tile in LDS, SPAN rows (or columns) by a chunk of depth, and its way there.
//   deep rows:  depth lies along the rows in memory.  LDS row r of 128 bytes, its piece p at p xor (r mod 8).
//   flat rows:  depth runs across the rows in memory (16-bit types).  LDS row d (of 64) of SPAN numbers; runs of 64 bytes lie exchanged
//               by d, so that the four rows that a transposing read takes at once lie in different banks.
template <bool DEEP, int SPAN, int WAVES>
struct TileOperand {
    static constexpr int kLoads = SPAN * kChunkBytes / 1024 / WAVES;      // of 16 bytes a lane, per wave and chunk
    static constexpr int kRowPieces = DEEP ? kChunkPieces : SPAN / 8;
    static constexpr int kRowsALoad = 64 / kRowPieces;
    static_assert(kLoads >= 1, "a wave loads something");

    static __device__ __forceinline__ int exchanged(int d) { return SPAN * 2 >= 256 ? d & 3 : (d >> 1) & 1; }

    const char* from[kLoads];      // this lane's pieces of the first chunk
    int need[kLoads];              // deep: byte of depth where the piece starts; flat: depth of the row, or past every end where the column is
    int numbers[kLoads];           // flat, and pieces that may be cut: numbers of the piece inside the row

    // base: first row and column of the tile; rows_left: rows (deep) / columns (flat) of the operand from there on
    __device__ __forceinline__ void start(const char* base, long long stride, int left, int wave, int lane)
    {
#pragma unroll
        for (int t = 0; t < kLoads; ++t) {
            const int r = (wave * kLoads + t) * kRowsALoad + lane / kRowPieces, q = lane % kRowPieces;
            if constexpr (DEEP) {
                const int piece = q ^ (r & 7), row = r < left ? r : left - 1;
                from[t] = base + row * stride + piece * 16;
                need[t] = piece * 16;
            } else {
                const int piece = q ^ (exchanged(r) << 2);
                from[t] = base + r * stride + piece * 16;
                need[t] = r;
                numbers[t] = left - piece * 8;
            }
        }
    }
    // straight to LDS; depth_left: bytes (deep) / rows (flat) of depth from this chunk on
    template <bool WHOLE>
    __device__ __forceinline__ void load(uintx4* lds, long long advance, int depth_left, int wave) const
    {
#pragma unroll
        for (int t = 0; t < kLoads; ++t) {
            const char* p = from[t] + advance;
            if (!WHOLE && need[t] >= depth_left) p = reinterpret_cast<const char*>(&zero_piece);
            if constexpr (!DEEP)
                if (numbers[t] <= 0) p = reinterpret_cast<const char*>(&zero_piece);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p,
                                             (__attribute__((address_space(3))) void*)(lds + (wave * kLoads + t) * 64), 16, 0, 0);
        }
    }
    // through registers, from any alignment
    __device__ __forceinline__ void fetch(uintx4 (&v)[kLoads], long long advance, int depth_left) const
    {
#pragma unroll
        for (int t = 0; t < kLoads; ++t) {
            int count;
            if constexpr (DEEP) count = (depth_left - need[t]) >> 1;
            else count = need[t] < depth_left ? numbers[t] : 0;
            v[t] = fetch_some(from[t] + advance, count);
        }
    }
    __device__ __forceinline__ void put(const uintx4 (&v)[kLoads], uintx4* lds, int wave, int lane) const
    {
#pragma unroll
        for (int t = 0; t < kLoads; ++t) lds[(wave * kLoads + t) * 64 + lane] = v[t];
    }
    // operand of the 32 rows from `first` on, step s of four
    static __device__ __forceinline__ uintx4 operand(const uintx4* lds, int first, int s, int lane)
    {
        const int g = lane >> 5;
        if constexpr (DEEP) {
            const int r = first + (lane & 31);
            return lds[r * kChunkPieces + ((2 * s + g) ^ (r & 7))];
        } else {
            // lane groups of 16: four rows of depth by 16 columns each read, which arrive as one column a lane
            const int j = lane & 15, col = first + ((lane >> 4) & 1) * 16 + (j & 3) * 4;
            uint2 half[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int d = 16 * s + 8 * g + 4 * i + (j >> 2);
                const int byte = d * (SPAN * 2) + ((col * 2) ^ (exchanged(d) << 6));
                const auto* p = (const __attribute__((address_space(3))) char*)lds + byte;
                half[i] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)p));
            }
            return uintx4{half[0].x, half[0].y, half[1].x, half[1].y};
        }
    }
};

// The scales of a chunk for a lane's row of each 32: eight bytes, shifted so that a lane's own of each step's two is byte 0 or 2.
struct ChunkScales {
    unsigned w[2];
    __device__ __forceinline__ void fetch(const uint8_t* p, int left)
    {
        if (left >= kChunkScales) {
            struct __attribute__((packed, aligned(1))) Eight { unsigned w[2]; };
            const Eight t = *reinterpret_cast<const Eight*>(p);
            w[0] = t.w[0];
            w[1] = t.w[1];
        } else {
            w[0] = w[1] = 0x7f7f7f7fu;             // ones: the numbers there are zeros
#pragma unroll
            for (int i = 0; i < kChunkScales - 1; ++i)
                if (i < left) w[i >> 2] = (w[i >> 2] & ~(0xffu << (8 * (i & 3)))) | (unsigned)p[i] << (8 * (i & 3));
        }
    }
    __device__ __forceinline__ void own(int lane)
    {
        w[0] >>= (lane >> 5) * 8;
        w[1] >>= (lane >> 5) * 8;
    }
};

// BM x BN results a workgroup of WM x WN waves.  ANY: operands whose rows are not made of whole aligned pieces of 16 bytes.
template <int DIRECTION, int TYPE, int BM, int BN, int WM, int WN, bool ANY, typename Out>
__global__ void __launch_bounds__(64 * WM * WN, BM * BN > 128 * 128 ? 1 : 2) product_kernel(ProductParams p)
{
    constexpr int WAVES = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
    constexpr bool MX = TYPE == kMx4;
    using A = TileOperand<DIRECTION != kDw, BM, WAVES>;
    using B = TileOperand<DIRECTION == kForward, BN, WAVES>;
    // two buffers, each read and written in code of its own, so that the compiler sees that what is read is not what the loads in
    // flight write
    __shared__ uintx4 even[(BM + BN) * kChunkPieces], odd[(BM + BN) * kChunkPieces];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const unsigned columns = (unsigned)(p.width + BN - 1) / BN;

    // which tile: its place in the result, and where its operands start
    const char *a, *b;
    int rows_left, cols_left, depth;          // depth: bytes (kForward, kDx: of A's rows), rows (kDw)
    Out* out = reinterpret_cast<Out*>(p.out);
    const uint8_t *a_scales = nullptr, *b_scales = nullptr;
    if constexpr (DIRECTION == kDw) {
        // an equal share of every expert's tiles to each XCD: the depth of an expert's sums is the number of its rows
        const unsigned per_expert = columns * ((unsigned)(p.height + BM - 1) / BM), share = (per_expert + 7) / 8;
        const unsigned k = blockIdx.x >> 3, expert = k / share, tile = (blockIdx.x & 7) * share + k % share;
        if (tile >= per_expert) return;
        int lo = 0, hi = p.rows;
        if (p.ends) {
            int before = 0;
            for (unsigned first = 0;; first += 64) {
                const Groups g(p.ends, first, p.experts, p.rows, before, lane);
                before = __builtin_amdgcn_readlane(g.hi, 63);
                if (expert - first < 64) {
                    lo = __builtin_amdgcn_readlane(g.lo, expert - first);
                    hi = __builtin_amdgcn_readlane(g.hi, expert - first);
                    break;
                }
            }
        }
        const int m0 = tile / columns * BM, n0 = tile % columns * BN;
        a = p.a + lo * p.a_stride + m0 * 2;
        b = p.b + lo * p.b_stride + n0 * 2;
        rows_left = p.height - m0;
        cols_left = p.width - n0;
        depth = hi - lo;
        out += ((long long)expert * p.height + m0) * p.out_stride + n0;
    } else {
        RowTiles<BM> tiles(p);
        unsigned tile;
        if (!xcd_run(blockIdx.x, (unsigned)tiles.total * columns, &tile)) return;
        // bands of four row tiles, column by column
        const unsigned band = tile / (4 * columns), in_band = tile - band * 4 * columns;
        const unsigned height = (unsigned)tiles.total - 4 * band < 4 ? tiles.total - 4 * band : 4;
        const RowTile at = tiles.find(4 * band + in_band % height);
        const int n0 = in_band / height * BN;
        const bool nobody = at.expert == p.experts;
        a = p.a + at.lo * p.a_stride;
        b = p.b + (nobody ? 0 : at.expert) * p.b_group + (DIRECTION == kForward ? n0 * p.b_stride : n0 * 2LL);
        rows_left = at.hi - at.lo;
        cols_left = p.width - n0;
        depth = nobody ? 0 : (MX ? p.depth / 2 : p.depth * 2);
        out += at.lo * p.out_stride + n0;
        if constexpr (MX) {
            const long long row_scales = p.depth / kMx4Block;
            a_scales = p.a_scales + at.lo * row_scales;
            b_scales = p.b_scales + ((nobody ? 0 : at.expert) * (long long)p.width + n0) * row_scales;
        }
    }
    const int m_rows = rows_left < BM ? rows_left : BM;

    A oa;
    B ob;
    oa.start(a, p.a_stride, rows_left, wave, lane);
    ob.start(b, p.b_stride, cols_left, wave, lane);
    floatx16 acc[TM][TN];
#pragma unroll
    for (int t = 0; t < TM; ++t)
#pragma unroll
        for (int u = 0; u < TN; ++u)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[t][u][v] = 0.0f;

    // depth in units of an operand: bytes along deep rows, rows of flat ones
    const int chunks = DIRECTION == kDw ? (depth + kChunkDepth16 - 1) / kChunkDepth16 : (depth + kChunkBytes - 1) / kChunkBytes;
    const auto left_a = [&](int c) { return DIRECTION == kDw ? depth - c * kChunkDepth16 : depth - c * kChunkBytes; };
    const auto left_b = [&](int c) { return DIRECTION == kDx ? depth / 2 - c * kChunkDepth16 : left_a(c); };
    const long long step_a = DIRECTION == kDw ? kChunkDepth16 * p.a_stride : kChunkBytes;
    const long long step_b = DIRECTION == kForward ? kChunkBytes : kChunkDepth16 * p.b_stride;

    uintx4 va[ANY ? A::kLoads : 1], vb[ANY ? B::kLoads : 1];
    const auto load = [&](int c, uintx4* buffer) {
        const bool whole = DIRECTION == kDw ? left_a(c) >= kChunkDepth16 : left_a(c) >= kChunkBytes;
        if constexpr (ANY) {
            oa.fetch(va, c * step_a, left_a(c));
            ob.fetch(vb, c * step_b, left_b(c));
        } else if (whole) {
            oa.template load<true>(buffer, c * step_a, 0, wave);
            ob.template load<true>(buffer + BM * kChunkPieces, c * step_b, 0, wave);
        } else {
            oa.template load<false>(buffer, c * step_a, left_a(c), wave);
            ob.template load<false>(buffer + BM * kChunkPieces, c * step_b, left_b(c), wave);
        }
    };
    ChunkScales sa[MX ? TM : 1], sb[MX ? TN : 1];
    const uint8_t *from_sa[MX ? TM : 1], *from_sb[MX ? TN : 1];
    const auto load_scales = [&](int c) {
        if constexpr (MX) {
            const int left = p.depth / kMx4Block - c * kChunkScales;
#pragma unroll
            for (int t = 0; t < TM; ++t) sa[t].fetch(from_sa[t] + c * kChunkScales, left);
#pragma unroll
            for (int u = 0; u < TN; ++u) sb[u].fetch(from_sb[u] + c * kChunkScales, left);
        }
    };
    if constexpr (MX) {
        const long long row_scales = p.depth / kMx4Block;
#pragma unroll
        for (int t = 0; t < TM; ++t) {
            const int r = (wm * TM + t) * 32 + (lane & 31);
            from_sa[t] = a_scales + (r < rows_left ? r : rows_left - 1) * row_scales;
        }
#pragma unroll
        for (int u = 0; u < TN; ++u) {
            const int r = (wn * TN + u) * 32 + (lane & 31);
            from_sb[u] = b_scales + (r < cols_left ? r : cols_left - 1) * row_scales;
        }
    }
    const auto chunk = [&](int c, const uintx4* now, uintx4* next) {
        if constexpr (ANY) {
            oa.put(va, const_cast<uintx4*>(now), wave, lane);
            ob.put(vb, const_cast<uintx4*>(now) + BM * kChunkPieces, wave, lane);
        } else {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // this wave's pieces are in place
        }
        __syncthreads();                                          // everyone's are, and the other buffer has been read
        ChunkScales ta[MX ? TM : 1], tb[MX ? TN : 1];
        if constexpr (MX) {
#pragma unroll
            for (int t = 0; t < TM; ++t) { ta[t] = sa[t]; ta[t].own(lane); }
#pragma unroll
            for (int u = 0; u < TN; ++u) { tb[u] = sb[u]; tb[u].own(lane); }
        }
        if (c + 1 < chunks) {
            load(c + 1, next);
            load_scales(c + 1);
        }
        static_for<0, 4>([&](auto s) {
            uintx4 fa[TM], fb[TN];
#pragma unroll
            for (int t = 0; t < TM; ++t) fa[t] = A::operand(now, (wm * TM + t) * 32, s.value, lane);
#pragma unroll
            for (int u = 0; u < TN; ++u) fb[u] = B::operand(now + BM * kChunkPieces, (wn * TN + u) * 32, s.value, lane);
#pragma unroll
            for (int t = 0; t < TM; ++t)
#pragma unroll
                for (int u = 0; u < TN; ++u) {
                    // columns of the result along the instruction's rows: a lane then holds four neighbours of a row of `out`
                    if constexpr (MX) acc[t][u] = multiply32_scaled<2 * (s.value & 1)>(fb[u], fa[t], acc[t][u], tb[u].w[s.value >> 1], ta[t].w[s.value >> 1]);
                    else acc[t][u] = multiply32<TYPE>(fb[u], fa[t], acc[t][u]);
                }
        });
    };
    if (chunks > 0) {
        load(0, even);
        load_scales(0);
    }
    for (int c = 0; c < chunks; c += 2) {
        chunk(c, even, odd);
        if (c + 1 < chunks) chunk(c + 1, odd, even);
    }

    // result register v of lane l: column 8 (v / 4) + 4 (l / 32) + v % 4, row l % 32 of its 32 x 32 tile
    const bool vector = p.out_stride % 4 == 0;
#pragma unroll
    for (int t = 0; t < TM; ++t) {
        const int r = (wm * TM + t) * 32 + (lane & 31);
        if (r >= m_rows) continue;
        Out* row = out + r * p.out_stride;
#pragma unroll
        for (int u = 0; u < TN; ++u)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int col = (wn * TN + u) * 32 + 8 * q + 4 * (lane >> 5);
                store_four(row + col, acc[t][u][4 * q], acc[t][u][4 * q + 1], acc[t][u][4 * q + 2], acc[t][u][4 * q + 3], cols_left - col, vector);
            }
    }
}

// ------------------------------------------------------------------ a few rows
// Up to 16 MT rows of a group by 16 columns (rows of the weights) a workgroup.  What counts is that the weights come once and at
// the memory's rate: every wave reads its share of the depth, 64 bytes of a row at a time, straight into the registers that the
// matrix pipe takes, and the four partial sums meet in LDS.
template <int TYPE, int MT, typename Out>
__global__ void __launch_bounds__(256) few_rows_kernel(ProductParams p, unsigned columns)
{
    constexpr bool MX = TYPE == kMx4;
    __shared__ floatx4 part[4][MT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r16 = lane & 15, quarter = lane >> 4;
    RowTiles<16 * MT> tiles(p);
    unsigned tile;
    if (!xcd_run(blockIdx.x, (unsigned)tiles.total * columns, &tile)) return;
    const RowTile at = tiles.find(tile / columns);
    const int n0 = tile % columns * 16;
    const bool nobody = at.expert == p.experts;
    const int rows_left = at.hi - at.lo;
    const int bytes = nobody ? 0 : (MX ? p.depth / 2 : p.depth * 2);
    const int n = n0 + r16 < p.width ? n0 + r16 : p.width - 1;
    const long long weight_row = (nobody ? 0 : at.expert) * (long long)p.width + n;
    const char* w = p.b + (nobody ? 0 : at.expert) * p.b_group + n * p.b_stride + quarter * 16;
    const char* x[MT];
    const int row_scales = p.depth / kMx4Block;
    const uint8_t *ws = nullptr, *xs[MT];
    if constexpr (MX) ws = p.b_scales + weight_row * row_scales + quarter;
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int r = at.lo + (t * 16 + r16 < rows_left ? t * 16 + r16 : rows_left - 1);
        x[t] = p.a + r * p.a_stride + quarter * 16;
        if constexpr (MX) xs[t] = p.a_scales + (long long)r * row_scales + quarter;
    }
    floatx4 acc[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[t] = floatx4{0, 0, 0, 0};
    const int steps = (bytes + 63) / 64, whole = bytes / 64;
    int s = wave;
    constexpr int AHEAD = MT > 2 ? 4 : 8;          // steps whose loads are in flight together
    for (; s + 4 * (AHEAD - 1) < whole; s += 4 * AHEAD) {
        uintx4 fw[AHEAD], fx[AHEAD][MT];
        unsigned sw[AHEAD], sx[AHEAD][MT];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int at_step = s + 4 * i;
            fw[i] = fetch_some(w + at_step * 64, 8);
            if constexpr (MX) sw[i] = ws[at_step * 4];
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                fx[i][t] = fetch_some(x[t] + at_step * 64, 8);
                if constexpr (MX) sx[i][t] = xs[t][at_step * 4];
            }
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                if constexpr (MX) acc[t] = multiply16_scaled(fw[i], fx[i][t], acc[t], sw[i], sx[i][t]);
                else acc[t] = multiply16<TYPE>(fw[i], fx[i][t], acc[t]);
            }
    }
    for (; s < steps; s += 4) {
        const int count = (bytes - s * 64 - quarter * 16) >> 1;        // 16-bit numbers, or pairs of codes
        const uintx4 fw = fetch_some(w + s * 64, count);
        unsigned sw = 0x7f;
        if constexpr (MX)
            if (count > 0) sw = ws[s * 4];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            const uintx4 fx = fetch_some(x[t] + s * 64, count);
            if constexpr (MX) acc[t] = multiply16_scaled(fw, fx, acc[t], sw, count > 0 ? xs[t][s * 4] : 0x7fu);
            else acc[t] = multiply16<TYPE>(fw, fx, acc[t]);
        }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) part[wave][t][lane] = acc[t];
    __syncthreads();
    // register v of lane l: column 4 (l / 16) + v, row l % 16
    const bool vector = p.out_stride % 4 == 0;
    for (int t = wave; t < MT; t += 4) {
        const floatx4 sum = (part[0][t][lane] + part[1][t][lane]) + (part[2][t][lane] + part[3][t][lane]);
        const int r = t * 16 + r16, col = n0 + 4 * quarter;
        if (r < rows_left) {
            Out* out = reinterpret_cast<Out*>(p.out) + (at.lo + r) * p.out_stride + col;
            store_four(out, sum[0], sum[1], sum[2], sum[3], p.width - col, vector);
        }
    }
}

// ------------------------------------------------------------------ launches
inline long long row_tiles_at_most(const ProductParams& p, int height)
{
    if (!p.ends) return (p.rows + height - 1) / height;
    const long long cut = p.experts + 1 < p.rows ? p.experts + 1 : p.rows;      // groups whose last tile is not full, the rows of no group too
    return p.rows / height + cut;
}
constexpr long long kMostBlocks = 0xffffff;       // a grid holds fewer than 2^32 threads

template <int DIRECTION, int TYPE, int BM, int BN, int WM, int WN, bool ANY, typename Out>
hipError_t launch_tiles(const ProductParams& p, hipStream_t s)
{
    const long long columns = (p.width + BN - 1) / BN;
    long long blocks;
    if (DIRECTION == kDw) blocks = (columns * ((p.height + BM - 1) / BM) + 7) / 8 * 8 * p.experts;
    else blocks = (row_tiles_at_most(p, BM) * columns + 7) / 8 * 8;
    if (blocks > kMostBlocks) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((product_kernel<DIRECTION, TYPE, BM, BN, WM, WN, ANY, Out>), dim3((unsigned)blocks), dim3(64 * WM * WN), 0, s, p);
    return hipGetLastError();
}

template <int TYPE, int MT, typename Out>
hipError_t launch_few_rows(const ProductParams& p, hipStream_t s)
{
    const long long columns = (p.width + 15) / 16;
    const long long blocks = (row_tiles_at_most(p, 16 * MT) * columns + 7) / 8 * 8;
    if (blocks > kMostBlocks) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((few_rows_kernel<TYPE, MT, Out>), dim3((unsigned)blocks), dim3(256), 0, s, p, (unsigned)columns);
    return hipGetLastError();
}

// whether every row that a kernel loads in pieces of 16 bytes is made of whole aligned ones
template <int DIRECTION, int TYPE>
bool whole_pieces(const ProductParams& p)
{
    if (TYPE == kMx4) return true;                                    // rows of 16 bytes for each 32 numbers
    const int a_row = DIRECTION == kDw ? p.height : p.depth;
    const int b_row = DIRECTION == kForward ? p.depth : p.width;
    return a_row % 8 == 0 && b_row % 8 == 0 && p.a_stride % 16 == 0 && p.b_stride % 16 == 0 && p.b_group % 16 == 0;
}

template <int DIRECTION, int TYPE, typename Out>
hipError_t launch_product_as(const ProductParams& p, hipStream_t s)
{
    if constexpr (DIRECTION == kForward) {
        const long long rows = (p.rows + p.experts - 1) / p.experts;      // of a group, on average
        if (rows <= 16) return launch_few_rows<TYPE, 1, Out>(p, s);
        if (rows <= 32) return launch_few_rows<TYPE, 2, Out>(p, s);
        if (rows <= 64) return launch_few_rows<TYPE, 4, Out>(p, s);
    }
    if constexpr (TYPE != kMx4)
        if (!whole_pieces<DIRECTION, TYPE>(p)) return launch_tiles<DIRECTION, TYPE, 128, 128, 2, 2, true, Out>(p, s);
    return launch_tiles<DIRECTION, TYPE, 128, 128, 2, 2, false, Out>(p, s);
}

}  // namespace spinner
