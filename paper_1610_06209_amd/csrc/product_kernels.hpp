// Matrix products of grouped rows on the matrix pipe: tiles through LDS, and the form for a few rows.
//
// In every product a wave multiplies 32 rows by 32 columns over a depth of 32 bytes an instruction: 16 numbers of 16 bits
// (v_mfma_f32_32x32x16) or 64 of 4 bits (v_mfma_scale_f32_32x32x64, e2m1 with an e8m0 scale for each 32), 16 bytes a lane from
// either operand.  So one kernel moves bytes for all types, and what differs is the instruction and the scales.
#pragma once
#include "mx4_lane.hpp"

namespace spinner {

typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

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
            const uint2 t = {Pair16<Out>::narrow(a, b), Pair16<Out>::narrow(c, d)};
            *reinterpret_cast<uint2*>(p) = t;
        }
        return;
    }
    if (left > 0) p[0] = (Out)a;
    if (left > 1) p[1] = (Out)b;
    if (left > 2) p[2] = (Out)c;
    if (left > 3) p[3] = (Out)d;
}

// 16 bytes of neighbours of a row, `left` numbers inside it, at any alignment of their type
template <typename Out>
__device__ __forceinline__ void store_piece(Out* p, uintx4 v, int left)
{
    constexpr int N = 16 / sizeof(Out);
    if (left >= N) {
        if constexpr (sizeof(Out) == 4) *reinterpret_cast<Words4*>(p) = Words4{{v[0], v[1], v[2], v[3]}};
        else *reinterpret_cast<Bytes16*>(p) = Bytes16{{v[0], v[1], v[2], v[3]}};
        return;
    }
#pragma unroll
    for (int i = 0; i < N - 1; ++i) {
        if constexpr (sizeof(Out) == 4) { if (i < left) p[i] = __uint_as_float(v[i]); }
        else { if (i < left) reinterpret_cast<unsigned short*>(p)[i] = (unsigned short)(v[i >> 1] >> (16 * (i & 1))); }
    }
}

// Eight 16-bit numbers of a row from an address of any alignment, `count` of them inside the row and zeros behind: a piece that the row's end cuts
// is read as the eight numbers in front of the end, and one outside (count <= 0) from `safe`; keep_some() then puts it right.  In two
// halves so that loads in flight are not waited for one by one (number by number, one cut piece a row made 20000 x 301 x 403 weight gradients
// of 16 experts 298 us).  A row of less than eight numbers (SHORT) is read number by number.
__device__ __forceinline__ uintx4 fetch_some(const char* p, int count, const char* safe)
{
    const char* from = count >= 8 ? p : (count > 0 ? p - 2 * (8 - count) : safe);
    const Bytes16 t = *reinterpret_cast<const Bytes16*>(from);
    return uintx4{t.w[0], t.w[1], t.w[2], t.w[3]};
}
__device__ __forceinline__ uintx4 keep_some(uintx4 v, int count)
{
    if (__builtin_expect(__ballot(count < 8) == 0, 1)) return v;
    unsigned long long lo = v[0] | (unsigned long long)v[1] << 32, hi = v[2] | (unsigned long long)v[3] << 32;
    const int cut = count >= 8 ? 0 : (count > 0 ? 8 - count : 8), bits = 16 * (cut & 3);
    if (cut & 4) { lo = hi; hi = 0; }
    if (cut == 8) { lo = hi = 0; }
    lo = lo >> bits | (bits ? hi << (64 - bits) : 0);
    hi >>= bits;
    return uintx4{(unsigned)lo, (unsigned)(lo >> 32), (unsigned)hi, (unsigned)(hi >> 32)};
}
__device__ __forceinline__ uintx4 fetch_short(const char* p, int count)
{
    uintx4 v = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < count) v[i >> 1] |= (unsigned)reinterpret_cast<const unsigned short*>(p)[i] << (16 * (i & 1));
    return v;
}
__device__ __forceinline__ uintx4 fetch_whole(const char* p)
{
    const Bytes16 t = *reinterpret_cast<const Bytes16*>(p);
    return uintx4{t.w[0], t.w[1], t.w[2], t.w[3]};
}

// ------------------------------------------------------------------ tiles
constexpr int kChunkBytes = 128;                          // of a row's depth in LDS at a time
constexpr int kChunkPieces = kChunkBytes / 16;
constexpr int kChunkDepth16 = kChunkBytes / 2;            // the same in 16-bit numbers
constexpr int kChunkScales = kChunkBytes / 16;            // scales of a row's chunk: 32 numbers are 16 bytes
constexpr int kHeldScales = 256;                          // most scales of a row that a tile holds at once: a depth of 8192
constexpr unsigned kFar = 0x80000000u;                    // offsets of a tile's pieces stay below this

// 16 bytes a lane from a buffer of kFar bytes at `from`, to 1 KiB of LDS.  (The buffer's description comes out of scalar arithmetic, so that nothing
// has to be waited for between it and the load.)  Written out because the compiler, which counts these
// loads like any others, would wait for all of them before each transposing read of LDS, whose place it does not follow; they
// have no register to arrive in, and the kernel waits for them itself before the waves meet.
__device__ __forceinline__ void load_to_lds(uintx4* to, const char* from, unsigned offset)
{
    const unsigned long long base = reinterpret_cast<unsigned long long>(from);
    const intx4 buffer = {(int)base, (int)(base >> 32) & 0xffff, (int)kFar, 0x00027000};
    const unsigned place = (unsigned)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void*)to);
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" : : "v"(offset), "s"(buffer), "s"(place) : "memory", "m0");
}

// An operand's part of a tile in LDS, SPAN rows (or columns) by a chunk of depth, and its way there.
//   deep rows:  depth lies along the rows in memory.  LDS row r of 128 bytes, its piece p at p xor (r / 2 mod 8): the sixteen lanes of a
//               phase of a read, sixteen rows, then cover all banks.
//   flat rows:  depth runs across the rows in memory (16-bit types).  LDS row d (of 64) of SPAN numbers; runs of 64 bytes lie exchanged
//               by d, so that the four rows that a transposing read takes at once lie in different banks.
template <bool DEEP, int SPAN, int WAVES, bool ANY>
struct TileOperand {
    static constexpr int kLoads = SPAN * kChunkBytes / 1024 / WAVES;      // of 16 bytes a lane, per wave and chunk
    static constexpr int kRowPieces = DEEP ? kChunkPieces : SPAN / 8;
    static constexpr int kRowsALoad = 64 / kRowPieces;
    static_assert(kLoads >= 1, "a wave loads something");
    using Offset = std::conditional_t<ANY, long long, unsigned>;          // from the tile's first number; what is not ANY lies within kFar

    static __device__ __forceinline__ int exchanged(int d) { return SPAN * 2 >= 256 ? d & 3 : (d >> 1) & 1; }
    // row in LDS and piece of it in memory of this lane's t-th load
    static __device__ __forceinline__ int load_row(int t, int wave, int lane) { return (wave * kLoads + t) * kRowsALoad + lane / kRowPieces; }
    static __device__ __forceinline__ int load_piece(int r, int lane)
    {
        return (lane % kRowPieces) ^ (DEEP ? (r >> 1) & 7 : exchanged(r) << 2);
    }

    Offset offset[kLoads];
    int left;                      // rows (deep) / columns (flat) of the operand from the tile's first on

    __device__ __forceinline__ void start(long long stride, int left_, int wave, int lane)
    {
        left = left_;
#pragma unroll
        for (int t = 0; t < kLoads; ++t) {
            const int r = load_row(t, wave, lane), row = DEEP && r >= left ? left - 1 : r;
            offset[t] = (Offset)row * (Offset)stride + load_piece(r, lane) * 16;
            if (!DEEP && !ANY && load_piece(r, lane) * 8 >= left) offset[t] = kFar;
        }
    }
    // Load T of those of the chunk that starts at `from`, straight to LDS; depth_left: bytes (deep) / rows (flat) of depth from there on.
    // What lies beyond the operand is asked for beyond the end of the buffer as the load knows it, and arrives as zeros.
    template <int T>
    __device__ __forceinline__ void load(uintx4* lds, const char* from, int depth_left, int wave, int lane) const
    {
        const int r = load_row(T, wave, lane);
        const bool there = DEEP ? load_piece(r, lane) * 16 < depth_left : r < depth_left;
        load_to_lds(lds + (wave * kLoads + T) * 64, from, there ? (unsigned)offset[T] : kFar);
    }
    // through registers, from any alignment; `safe`: sixteen bytes that can be read, null for rows of less than eight numbers
    __device__ __forceinline__ int inside(int t, int depth_left, int wave, int lane) const      // numbers of the t-th piece inside the operand
    {
        const int r = load_row(t, wave, lane), piece = load_piece(r, lane);
        return DEEP ? (depth_left - piece * 16) >> 1 : (r < depth_left ? left - piece * 8 : 0);
    }
    __device__ __forceinline__ void fetch(uintx4 (&v)[kLoads], const char* from, int depth_left, const char* safe, int wave, int lane) const
    {
        if (safe) {
#pragma unroll
            for (int t = 0; t < kLoads; ++t) v[t] = fetch_some(from + offset[t], inside(t, depth_left, wave, lane), safe);
        } else {
#pragma unroll
            for (int t = 0; t < kLoads; ++t) v[t] = fetch_short(from + offset[t], inside(t, depth_left, wave, lane));
        }
    }
    __device__ __forceinline__ void put(const uintx4 (&v)[kLoads], uintx4* lds, int depth_left, const char* safe, int wave, int lane) const
    {
#pragma unroll
        for (int t = 0; t < kLoads; ++t) lds[(wave * kLoads + t) * 64 + lane] = safe ? keep_some(v[t], inside(t, depth_left, wave, lane)) : v[t];
    }
    // operand of the 32 rows from `first` on, step s of four
    static __device__ __forceinline__ uintx4 operand(const uintx4* lds, int first, int s, int lane)
    {
        const int g = lane >> 5;
        if constexpr (DEEP) {
            const int r = first + (lane & 31);
            return lds[r * kChunkPieces + ((2 * s + g) ^ ((r >> 1) & 7))];
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

// Scales of a tile's rows go through LDS, two chunks' (16 bytes of a row) at a time: straight from memory, eight bytes a row and chunk, they
// made twice as many requests as the numbers themselves.
struct RowScales {
    unsigned w[4];
    int beyond;                    // bytes that the operand's end lies in front of the last byte asked for
    // at: place of the first scale wanted, from the tile's first on; end: place behind the operand's last one; before: sixteen bytes in front of the
    // tile's first.  What the end cuts is read as the sixteen bytes in front of the end.
    __device__ __forceinline__ void fetch(const uint8_t* before, unsigned at, unsigned end)
    {
        const unsigned from = at + 16 < end ? at + 16 : end;
        struct __attribute__((packed, aligned(1))) Sixteen { unsigned w[4]; };
        const Sixteen t = *reinterpret_cast<const Sixteen*>(before + from);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = t.w[i];
        beyond = (int)(at + 16 - from);
    }
    // behind the row's last scale (`left` are its own) come ones: the numbers there are zeros, but a NaN would stay one
    __device__ __forceinline__ void put(uintx4* to, int left) const
    {
        unsigned long long lo = w[0] | (unsigned long long)w[1] << 32, hi = w[2] | (unsigned long long)w[3] << 32;
        const int s = 8 * (beyond & 7);
        if (beyond & 8) { lo = hi; hi = 0; }
        lo = lo >> s | (s ? hi << (64 - s) : 0);
        hi >>= s;
        const unsigned long long ml = left >= 8 ? ~0ull : (left > 0 ? (1ull << (8 * left)) - 1 : 0);
        const unsigned long long mh = left >= 16 ? ~0ull : (left > 8 ? (1ull << (8 * (left - 8))) - 1 : 0);
        lo = (lo & ml) | (0x7f7f7f7f7f7f7f7full & ~ml);
        hi = (hi & mh) | (0x7f7f7f7f7f7f7f7full & ~mh);
        *to = uintx4{(unsigned)lo, (unsigned)(lo >> 32), (unsigned)hi, (unsigned)(hi >> 32)};
    }
};

// how many workgroups of four waves the LDS of a compute unit holds
constexpr int workgroups_a_unit(int side, int stages, int type) { return side == 256 || (side == 128 && stages > 2) || (side == 64 && type == kMx4) ? 1 : 2; }

// BM x BN results a workgroup of WM x WN waves, STAGES chunks in LDS.  ANY: operands whose rows are not made of whole aligned pieces of
// 16 bytes.
// Every number of a tile goes to LDS once, and from there to the waves that share it.  LDS gives 128 bytes a cycle and a product takes 32 cycles of one
// of four matrix pipes, so that 64 x 64 numbers a wave would need all of it, 128 x 128 half: 256 x 256 results of four waves, one a
// SIMD with 256 sums, two chunks in LDS.  That form hides what it waits for in its own order: operands a step ahead of their products, loads straight to
// LDS a chunk ahead and between the products, one meeting of the waves a chunk, with a step's products still to come.  It takes the numbers of
// tiles that leave many compute units idle; then smaller ones are ahead (see plan_product).
// Measured: 16384 x 8192 x 8192 in 4 bits 518 us, 4.2 PFLOP/s; 16384 x 4096 x 4096 138 us, 4.0; bf16 16384 x 4096 x 4096 y 394 to 411 us, 1.34 to 1.39 PFLOP/s, dx 419, 1.31,
// dw 432, 1.27 (the library behind torch, y with one weight matrix: 337, 1.63).  Bound: half and a little more of the time the matrix pipe is busy, at 1.7 to 2.1 GHz
// under its load; with neither the loads nor the reads of LDS the 4-bit product takes 425 to 445 us.  In us as the kernel was then, 4 bits / bf16: reads of
// LDS that the compiler put right before their products 851 / 1068; banks covered eight lanes at a time, all loads of a chunk in one step 798 / 1000;
// scales straight from memory 763; results stored from registers 595 / 228 a quarter of the rows, through LDS 571 / 223; eight waves of 128 x 64
// 623 (four 574) / 1030 (980).  Lines touched two to four chunks ahead of their loads, to have them in the L2: 632 / 512.
template <int DIRECTION, int TYPE, int BM, int BN, int WM, int WN, int STAGES, bool ANY, typename Out>
__global__ void __launch_bounds__(64 * WM * WN, workgroups_a_unit(BM, STAGES, TYPE))
product_kernel(ProductParams p)
{
    static_assert(STAGES == 2 || !ANY, "loads through registers are one chunk ahead");
    constexpr int WAVES = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
    constexpr bool MX = TYPE == kMx4;
    // scales: two chunks' at a time, brought through registers a pair of chunks ahead; 64 x 64, where a wait for those would be one for
    // all chunks on their way, all of the depth's at the start
    constexpr bool HELD = MX && TM * TN == 1;
    constexpr int kScalePieces = HELD ? kHeldScales / 16 + 1 : 1;      // 16-byte pieces from one row's to the next in LDS
    using A = TileOperand<DIRECTION != kDw, BM, WAVES, ANY>;
    using B = TileOperand<DIRECTION == kForward, BN, WAVES, ANY>;
    constexpr int kBuffer = (BM + BN) * kChunkPieces, kSums = TM * TN == 1 ? 4 * 4 * 256 : 0;      // sums of the four waves of 64 x 64
    __shared__ uintx4 buffers[STAGES * kBuffer > kSums ? STAGES * kBuffer : kSums];
    __shared__ uintx4 row_scales[MX ? (HELD ? 1 : 2) : 1][MX ? (BM + BN) * kScalePieces : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const unsigned columns = (unsigned)(p.width + BN - 1) / BN;

    // which tile: its place in the result, and where its operands start
    const char *a, *b;
    int rows_left, cols_left, depth;          // depth: bytes (kForward, kDx: of A's rows), rows (kDw)
    Out* out = reinterpret_cast<Out*>(p.out);
    const uint8_t *a_scales = nullptr, *b_scales = nullptr;
    unsigned a_end = 0, b_end = 0;            // scales from the tile's first to the operand's last
    if constexpr (DIRECTION == kDw) {
        // an equal share of every expert's tiles to each XCD: the depth of an expert's sums is the number of its rows
        const unsigned per_expert = columns * ((unsigned)(p.height + BM - 1) / BM), share = (per_expert + 7) / 8;
        const unsigned block = p.first_block + blockIdx.x, k = block >> 3, expert = k / share, tile = (block & 7) * share + k % share;
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
        if (!xcd_run(p.first_block + blockIdx.x, (unsigned)tiles.total * columns, &tile)) return;
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
            const long long count = p.depth / kMx4Block;
            const long long from_a = at.lo * count, from_b = ((nobody ? 0 : at.expert) * (long long)p.width + n0) * count;
            const long long a_left = p.rows * count - from_a, b_left = p.experts * (p.width * count) - from_b;
            a_scales = p.a_scales + from_a - 16;
            b_scales = p.b_scales + from_b - 16;
            a_end = (unsigned)(a_left < kFar ? a_left : kFar);
            b_end = (unsigned)(b_left < kFar ? b_left : kFar);
        }
    }
    const int m_rows = rows_left < BM ? rows_left : BM;

    A oa;
    B ob;
    oa.start(p.a_stride, rows_left, wave, lane);
    ob.start(p.b_stride, cols_left, wave, lane);
    floatx16 acc[TM][TN];
#pragma unroll
    for (int t = 0; t < TM; ++t)
#pragma unroll
        for (int u = 0; u < TN; ++u)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[t][u][v] = 0.0f;

    // depth in units of an operand: bytes along deep rows, rows of flat ones
    constexpr int unit_a = DIRECTION == kDw ? kChunkDepth16 : kChunkBytes, unit_b = DIRECTION == kForward ? kChunkBytes : kChunkDepth16;
    const long long step_a = DIRECTION == kDw ? kChunkDepth16 * p.a_stride : kChunkBytes;
    const long long step_b = DIRECTION == kForward ? kChunkBytes : kChunkDepth16 * p.b_stride;
    int chunks = (depth + unit_a - 1) / unit_a;
    if constexpr (DIRECTION == kDw)
        if (p.splits > 1) {                   // this workgroup's share of the depth, and its place among the partial sums
            const int share = (chunks + p.splits - 1) / p.splits, first = share * (int)blockIdx.y;
            a += first * step_a;
            b += first * step_b;
            depth -= first * unit_a;
            depth = depth < 0 ? 0 : (depth < share * unit_a ? depth : share * unit_a);
            chunks = (depth + unit_a - 1) / unit_a;
            out += blockIdx.y * p.split_stride;
        }
    const int depth_b = DIRECTION == kDx ? depth / 2 : depth;

    uintx4 va[ANY ? A::kLoads : 1], vb[ANY ? B::kLoads : 1];
    // numbers of A's and B's rows as they lie, and the last eight in front of the end of the tile's first
    const int row_a = DIRECTION == kDw ? p.height : p.depth, row_b = DIRECTION == kForward ? p.depth : p.width;
    const char* safe_a = ANY && row_a >= 8 && chunks ? (DIRECTION == kDw && rows_left < 8 ? a - 2 * (8 - rows_left) : a) : nullptr;
    const char* safe_b = ANY && row_b >= 8 && chunks ? (DIRECTION != kForward && cols_left < 8 ? b - 2 * (8 - cols_left) : b) : nullptr;
    const auto fetch = [&](int c) {
        if constexpr (ANY) {
            oa.fetch(va, a + c * step_a, depth - c * unit_a, safe_a, wave, lane);
            ob.fetch(vb, b + c * step_b, depth_b - c * unit_b, safe_b, wave, lane);
        }
    };
    const auto put = [&](int c, uintx4* buffer) {
        if constexpr (ANY) {
            oa.put(va, buffer, depth - c * unit_a, safe_a, wave, lane);
            ob.put(vb, buffer + BM * kChunkPieces, depth_b - c * unit_b, safe_b, wave, lane);
        }
    };
    // Scales (kMx4) of row r of the tile (B's behind A's) from byte `at` of its own on
    constexpr int THREADS = 64 * WAVES;
    const int scale_count = MX ? p.depth / kMx4Block : 0;
    const auto bring = [&](RowScales& v, int r, int from) {
        const int ra = r < rows_left ? r : rows_left - 1, rb = r - BM < cols_left ? r - BM : cols_left - 1;
        v.fetch(r < BM ? a_scales : b_scales, (unsigned)((r < BM ? ra : rb) * scale_count + from), r < BM ? a_end : b_end);
    };

    // load L of chunk `c`: those of operand A, then those of B
    constexpr int kLoads = ANY ? 0 : A::kLoads + B::kLoads;
    const auto load = [&](auto l, int c, uintx4* to) {
        constexpr int L = l.value;
        if constexpr (L < A::kLoads) oa.template load<L>(to, a + c * step_a, depth - c * unit_a, wave, lane);
        else ob.template load<L - A::kLoads>(to + BM * kChunkPieces, b + c * step_b, depth_b - c * unit_b, wave, lane);
    };
    // This wave's loads are in place but for the last `on_their_way`, and what it asked LDS for has arrived; so it is for all waves.
    const auto meet = [&](auto on_their_way) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(on_their_way.value) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" : : : "memory");
    };
    constexpr std::integral_constant<int, 0> s0{};
    constexpr std::integral_constant<int, 1> s1{};
    constexpr std::integral_constant<int, 2> s2{};
    constexpr std::integral_constant<int, 3> s3{};
    constexpr std::integral_constant<int, (STAGES - 2) * kLoads> behind{};
    int at = 0;                    // buffer of the chunk at hand
    // Chunks behind the last are zeros: they are asked for, and not multiplied but for one that makes 4-bit chunks pairs.
    fetch(0);
    put(0, buffers);
    fetch(1);
    static_for<0, STAGES - 1>([&](auto k) { static_for<0, kLoads>([&](auto l) { load(l, k.value, buffers + k.value * kBuffer); }); });
    if constexpr (TM * TN > 1) {
        // A chunk is four steps, the operands of each read while the one before is multiplied.  A chunk's last
        // operands are read before the waves meet, so that its buffer is free for a later chunk from its last step on, and the first operands
        // of the next chunk come during that step too.  The loads of a chunk are spread over two steps.
        constexpr int kEarly = kLoads / 2;
        constexpr std::integral_constant<int, kEarly> early{};
        constexpr std::integral_constant<int, kLoads> all{};
        // scales: every thread brings those of its rows for a pair of chunks; a lane takes the eight bytes of its rows for one chunk, shifted so that
        // its own of each step's two is byte 0 or 2
        static_assert(!MX || (BM + BN) % THREADS == 0, "whole rows a thread");
        constexpr int kScaleRows = MX ? (BM + BN) / THREADS : 1;
        RowScales brought[kScaleRows];
        const auto fetch_scales = [&](int c) {
#pragma unroll
            for (int i = 0; i < kScaleRows; ++i) bring(brought[i], i * THREADS + (int)threadIdx.x, c * kChunkScales);
        };
        const auto put_scales = [&](int c) {
#pragma unroll
            for (int i = 0; i < kScaleRows; ++i) brought[i].put(&row_scales[c >> 1 & 1][i * THREADS + threadIdx.x], scale_count - c * kChunkScales);
        };
        uint2 sa[TM], sb[TN], ta[TM], tb[TN];
        const auto take_scales = [&](int c) {
            const char* from = reinterpret_cast<const char*>(&row_scales[c >> 1 & 1][lane & 31]) + (c & 1) * kChunkScales;
#pragma unroll
            for (int t = 0; t < TM; ++t) sa[t] = *reinterpret_cast<const uint2*>(from + (wm * TM + t) * 32 * 16);
#pragma unroll
            for (int u = 0; u < TN; ++u) sb[u] = *reinterpret_cast<const uint2*>(from + (BM + (wn * TN + u) * 32) * 16);
        };
        const auto own_scales = [&] {
            const int shift = (lane >> 5) * 8;
#pragma unroll
            for (int t = 0; t < TM; ++t) ta[t] = {sa[t].x >> shift, sa[t].y >> shift};
#pragma unroll
            for (int u = 0; u < TN; ++u) tb[u] = {sb[u].x >> shift, sb[u].y >> shift};
        };
        uintx4 fa[2][TM], fb[2][TN];
        // operand I of step S: the first rows' and all columns' come first, as they are multiplied
        const auto operand = [&](const uintx4* buffer, auto s, auto i) {
            constexpr int S = s.value, I = i.value;
            if constexpr (I >= 1 && I <= TN) fb[S & 1][I - 1] = B::operand(buffer + BM * kChunkPieces, (wn * TN + I - 1) * 32, S, lane);
            else fa[S & 1][I == 0 ? 0 : I - TN] = A::operand(buffer, (wm * TM + (I == 0 ? 0 : I - TN)) * 32, S, lane);
        };
        // Step S: its products in turn with the reads of the next step's operands (step `next_s`, from `next`) and with loads FIRST to LAST
        // of chunk `c` to LDS.  The compiler keeps to this order.
        const auto step = [&](auto s, const uintx4* next, auto next_s, auto first, auto last, int c, uintx4* to) {
            constexpr int S = s.value, N = TM * TN, READS = TM + TN, FIRST = first.value, COUNT = last.value - FIRST;
            static_for<0, N>([&](auto i) {
                constexpr int I = i.value, t = I / TN, u = I % TN;
                constexpr int rate = (READS + N - 1) / N;
                static_for<I * rate, (I + 1) * rate < READS ? (I + 1) * rate : READS>([&](auto r) { operand(next, next_s, r); });
                // columns of the result along the instruction's rows: a lane then holds four neighbours of a row of `out`
                if constexpr (MX) acc[t][u] = multiply32_scaled<2 * (S & 1)>(fb[S & 1][u], fa[S & 1][t], acc[t][u], S < 2 ? tb[u].x : tb[u].y, S < 2 ? ta[t].x : ta[t].y);
                else acc[t][u] = multiply32<TYPE>(fb[S & 1][u], fa[S & 1][t], acc[t][u]);
                static_for<FIRST + I * COUNT / N, FIRST + (I + 1) * COUNT / N>([&](auto l) { load(l, c, to); });
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        const auto chunk = [&](int c, auto first) {      // first: of a pair, which brings the next pair's scales
            uintx4* now = buffers + at * kBuffer;
            uintx4* last = buffers + (at ? at - 1 : STAGES - 1) * kBuffer;      // of the chunk before, the first to be free
            at = at + 1 < STAGES ? at + 1 : 0;
            uintx4* next = buffers + at * kBuffer;
            if constexpr (MX) own_scales();
            step(s0, now, s1, early, all, c + STAGES - 1, last);
            if constexpr (MX && first.value) fetch_scales(c + 2);
            step(s1, now, s2, s0, s0, 0, nullptr);
            step(s2, now, s3, s0, s0, 0, nullptr);
            put(c + 1, next);
            meet(behind);
            fetch(c + 2);
            if constexpr (MX && first.value) put_scales(c + 2);
            if constexpr (MX) take_scales(c + 1);
            step(s3, next, s0, s0, early, c + STAGES, now);
        };
        static_for<0, kEarly>([&](auto l) { load(l, STAGES - 1, buffers + (STAGES - 1) * kBuffer); });
        if constexpr (MX) {
            fetch_scales(0);
            put_scales(0);
        }
        meet(std::integral_constant<int, (STAGES - 2) * kLoads + kEarly>{});
        if constexpr (MX) take_scales(0);
        static_for<0, TM + TN>([&](auto i) { operand(buffers, s0, i); });
        for (int c = 0; c < chunks; ++c) {
            chunk(c, s1);
            if constexpr (MX) chunk(++c, s0);
        }
    } else {
        // 64 x 64: a wave that multiplied a quarter of the tile would read two operands of LDS a product.  Here each multiplies the whole tile, one
        // step of a chunk's four each, four products for four operands, read while those of the chunk before are multiplied; the four
        // sums meet at the end.
        static_assert(BM == 64 && BN == 64 && WAVES == 4, "a quarter of the result a wave");
        uintx4 fa[2][2], fb[2][2];
        floatx16 sum[2][2];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int u = 0; u < 2; ++u) sum[t][u] = acc[0][0];
        const auto operands = [&](const uintx4* buffer, auto set) {
#pragma unroll
            for (int t = 0; t < 2; ++t) fa[set.value][t] = A::operand(buffer, t * 32, wave, lane);
#pragma unroll
            for (int u = 0; u < 2; ++u) fb[set.value][u] = B::operand(buffer + BM * kChunkPieces, u * 32, wave, lane);
        };
        unsigned xa[2], xb[2], ya[2], yb[2];          // scales of the wave's step: as read, and shifted so that the lane's own is byte 0
        const auto take = [&](int c) {
            const int word = (c & 1) * 2 + (wave >> 1), r = lane & 31;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                xa[t] = reinterpret_cast<const unsigned*>(&row_scales[0][(t * 32 + r) * kScalePieces + (c >> 1)])[word];
                xb[t] = reinterpret_cast<const unsigned*>(&row_scales[0][(BM + t * 32 + r) * kScalePieces + (c >> 1)])[word];
            }
        };
        const auto chunk = [&](int c, auto set) {
            uintx4* now = buffers + at * kBuffer;
            at = at + 1 < STAGES ? at + 1 : 0;
            uintx4* next = buffers + at * kBuffer;
            put(c + 1, next);
            meet(behind);
            if constexpr (MX) {
                const int shift = (lane >> 5) * 8 + (wave & 1) * 16;
#pragma unroll
                for (int t = 0; t < 2; ++t) { ya[t] = xa[t] >> shift; yb[t] = xb[t] >> shift; }
            }
            fetch(c + 2);
            operands(next, std::integral_constant<int, 1 - set.value>{});
            if constexpr (MX) take(c + 1);
            __builtin_amdgcn_sched_barrier(0);
            static_for<0, 4>([&](auto i) {
                constexpr int t = i.value / 2, u = i.value % 2;
                if constexpr (MX) sum[t][u] = multiply32_scaled<0>(fb[set.value][u], fa[set.value][t], sum[t][u], yb[u], ya[t]);
                else sum[t][u] = multiply32<TYPE>(fb[set.value][u], fa[set.value][t], sum[t][u]);
                static_for<i.value * kLoads / 4, (i.value + 1) * kLoads / 4>([&](auto l) { load(l, c + STAGES, now); });
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        static_for<0, kLoads>([&](auto l) { load(l, STAGES - 1, buffers + (STAGES - 1) * kBuffer); });
        if constexpr (MX) {
            // a pair of chunks of a row a thread at a time
            const int pairs = (chunks + 1) / 2, count = pairs * (BM + BN);
            for (int k = threadIdx.x; k < count; k += THREADS) {
                const int r = k / pairs, pair = k - r * pairs;
                RowScales v;
                bring(v, r, pair * 16);
                v.put(&row_scales[0][r * kScalePieces + pair], scale_count - pair * 16);
            }
        }
        meet(std::integral_constant<int, (STAGES - 1) * kLoads>{});
        if constexpr (MX) take(0);
        operands(buffers, s0);
        for (int c = 0; c < chunks; c += 2) {
            chunk(c, s0);
            if (!MX && c + 1 >= chunks) break;
            chunk(c + 1, s1);
        }
        meet(s0);
        floatx4* part = reinterpret_cast<floatx4*>(buffers);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    part[((wave * 4 + t * 2 + u) * 4 + q) * 64 + lane] = floatx4{sum[t][u][4 * q], sum[t][u][4 * q + 1], sum[t][u][4 * q + 2], sum[t][u][4 * q + 3]};
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            floatx4 v[4];
#pragma unroll
            for (int w = 0; w < 4; ++w) v[w] = part[((w * 4 + wave) * 4 + q) * 64 + lane];
            const floatx4 all = (v[0] + v[1]) + (v[2] + v[3]);
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[0][0][4 * q + k] = all[k];
        }
    }
    meet(s0);

    // Result register v of lane l: column 8 (v / 4) + 4 (l / 32) + v % 4, row l % 32 of its 32 x 32 tile.  Stored from there, an instruction would
    // write 16 bytes to each of 32 rows; through LDS (a part of its own for each wave, 32 rows at a time, the 16-byte pieces of a row exchanged by
    // its number) they are whole runs of 32 TN columns.
    constexpr int kOutPieces = TN * 32 * (int)sizeof(Out) / 16, kPieceOuts = 16 / (int)sizeof(Out);
    static_assert(WAVES * 32 * kOutPieces <= STAGES * kBuffer, "fits the buffers");
    uintx4* mine = buffers + wave * 32 * kOutPieces;
#pragma unroll
    for (int t = 0; t < TM; ++t) {
#pragma unroll
        for (int u = 0; u < TN; ++u)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int r = lane & 31, col = u * 32 + 8 * q + 4 * (lane >> 5), piece = (col / kPieceOuts) ^ (r & (kOutPieces - 1));
                const float *v = reinterpret_cast<const float*>(&acc[t][u]) + 4 * q;
                if constexpr (sizeof(Out) == 4) mine[r * kOutPieces + piece] = uintx4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
                else reinterpret_cast<uint2*>(mine + r * kOutPieces + piece)[lane >> 5] = uint2{Pair16<Out>::narrow(v[0], v[1]), Pair16<Out>::narrow(v[2], v[3])};
            }
#pragma unroll
        for (int k = 0; k < 32 * kOutPieces / 64; ++k) {
            const int r = k * (64 / kOutPieces) + lane / kOutPieces, piece = lane % kOutPieces;
            const uintx4 v = mine[r * kOutPieces + (piece ^ (r & (kOutPieces - 1)))];
            const int row = (wm * TM + t) * 32 + r, col = wn * TN * 32 + piece * kPieceOuts;
            if (row < m_rows) store_piece(out + row * p.out_stride + col, v, cols_left - col);
        }
    }
}

// ------------------------------------------------------------------ a few rows
// Up to 16 rows of a group by 16 NT columns (rows of the weights) a workgroup.  What counts is that the weights come once and at
// the memory's rate: every wave reads its share of the depth, runs of 256 bytes of a row, straight into the registers that the
// matrix pipe takes, one run ahead, and the four partial sums meet in LDS.
// Measured, the same weights time after time, which the memory's cache holds / others each time: 24 rows over 8 experts of 8192 x 2048 in bf16 (268 MB) 41 /
// 56 us, 6.5 / 4.8 TB/s; 64 rows over 32 experts of 4096 x 2048 in 4 bits (143 MB) 22.5 / 32 us, 6.3 / 4.5 TB/s; one row, 16384 x 4096 (36 MB) 8.9 us
// of which the launch and the way to the first weights are half.  With runs of 64 bytes in turn between the waves and scales a byte at a time: 43, 34, 11.2.
// Weights with the streaming hint, others each time: 56, 31.7; one row, 8192 x 8192 in 4 bits 11.0 for 9.8.
constexpr int kRunSteps = 4;                              // products of a run, 64 bytes of a row each
template <int TYPE, int NT>
struct Run {
    uintx4 w[NT][kRunSteps], x[kRunSteps];
    uintx4 ws[NT], xs;                                    // kMx4: the run's scales of the lane's rows
};
// RAW (4 bits): the rows are plain numbers of type Out.  Every workgroup rotates and quantises them for itself, a chunk of 512 a wave, into LDS, while its
// first weights are on their way: no launch and no trip through memory in front of them.  The sums are those of two calls, in the same order.  In us, one
// launch / two: one row, n = 16384, k = 4096, runs of 4096 10.9 / 12.8; n = 4096, k = 2048 5.4 / 5.9; four rows, n = k = 1024 4.3 / 5.2; one row,
// n = k = 256 3.2 / 4.6.  With four waves that take two chunks each 13.2, four each (two rows) 17.7.
// (two waves a SIMD: 260 registers, which leave one, 64 rows of 32 experts 43 us for 35)
template <int TYPE, int NT, typename Out, bool RAW>
__global__ void __launch_bounds__(RAW ? 512 : 256, 2) few_rows_kernel(ProductParams p, unsigned columns, RawRows raw)
{
    constexpr bool MX = TYPE == kMx4;
    static_assert(MX || !RAW, "rows are quantised for 4-bit weights");
    __shared__ float4 meeting[RAW ? kRawChunks * 128 : 1];
    __shared__ uintx4 own_codes[RAW ? kRawChunks * 16 : 1], own_scales[RAW ? kRawChunks : 1];
    // waves share the depth by four; RAW: and the columns by two, so that eight waves quantise
    constexpr int PARTS = RAW ? 2 : 1;
    __shared__ floatx4 part[4 * PARTS][NT][64];
    const int lane = threadIdx.x & 63, in_group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = in_group & 3;
    const int r16 = lane & 15, quarter = lane >> 4;
    RowTiles<16> tiles(p);
    unsigned tile;
    if (!xcd_run(p.first_block + blockIdx.x, (unsigned)tiles.total * columns, &tile)) return;
    const RowTile at = tiles.find(tile / columns);
    const int n0 = tile % columns * (16 * NT * PARTS);
    const bool nobody = at.expert == p.experts;
    const int rows_left = at.hi - at.lo;
    const int bytes = nobody ? 0 : (MX ? p.depth / 2 : p.depth * 2);
    const int row_scales = p.depth / kMx4Block;
    const int row = at.lo + (r16 < rows_left ? r16 : rows_left - 1);
    const int row_chunks = (p.depth + kChunk - 1) / kChunk;           // RAW: a row in LDS is so many whole chunks
    const char *x = RAW ? reinterpret_cast<const char*>(own_codes) + (row - at.lo) * row_chunks * 256 + quarter * 16 : p.a + row * p.a_stride + quarter * 16, *w[NT];
    const uint8_t *xs = !MX ? nullptr : RAW ? reinterpret_cast<const uint8_t*>(own_scales) + (row - at.lo) * row_chunks * 16 : p.a_scales + (long long)row * row_scales, *ws[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int own = n0 + ((in_group >> 2) * NT + t) * 16 + r16, n = own < p.width ? own : p.width - 1;
        w[t] = p.b + (nobody ? 0 : at.expert) * p.b_group + n * p.b_stride + quarter * 16;
        ws[t] = MX ? p.b_scales + ((nobody ? 0 : at.expert) * (long long)p.width + n) * row_scales : nullptr;
    }
    floatx4 acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = floatx4{0, 0, 0, 0};

    const auto piece16 = [](const void* from) {
        struct __attribute__((packed, aligned(1))) Sixteen { unsigned v[4]; };
        const Sixteen t = *static_cast<const Sixteen*>(from);
        return uintx4{t.v[0], t.v[1], t.v[2], t.v[3]};
    };
    // the rows' part of a run (RAW: in LDS, where rows and their scales start at whole 16 bytes)
    const auto take = [&](Run<TYPE, NT>& run, int k) {
#pragma unroll
        for (int i = 0; i < kRunSteps; ++i) run.x[i] = RAW ? *reinterpret_cast<const uintx4*>(x + (k * kRunSteps + i) * 64) : fetch_whole(x + (k * kRunSteps + i) * 64);
        if constexpr (RAW) run.xs = *reinterpret_cast<const uintx4*>(xs + k * kRunSteps * 4);
        else if constexpr (MX) run.xs = piece16(xs + k * kRunSteps * 4);
    };
    const auto fetch = [&](Run<TYPE, NT>& run, int k) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < kRunSteps; ++i) run.w[t][i] = fetch_whole(w[t] + (k * kRunSteps + i) * 64);
            if constexpr (MX) run.ws[t] = piece16(ws[t] + k * kRunSteps * 4);
        }
        if constexpr (!RAW) take(run, k);
    };
    const auto multiply = [&](Run<TYPE, NT>& run, int k) {
        if constexpr (RAW) take(run, k);
#pragma unroll
        for (int i = 0; i < kRunSteps; ++i)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if constexpr (MX) acc[t] = multiply16_scaled(run.w[t][i], run.x[i], acc[t], run.ws[t][i] >> (8 * quarter), run.xs[i] >> (8 * quarter));
                else acc[t] = multiply16<TYPE>(run.w[t][i], run.x[i], acc[t]);
            }
    };
    const int runs = bytes / (64 * kRunSteps);
    Run<TYPE, NT> now, next;
    int k = wave;
    if constexpr (RAW) {
        // a chunk of a row a wave: the rows asked for first, then the weights
        using Lane = LaneNumbers<Out>;
        const int chunks = nobody ? 0 : (rows_left < 16 ? rows_left : 16) * row_chunks, c = in_group, r = c / row_chunks, in_row = c - r * row_chunks;
        const unsigned flip = raw.log > 0 ? Lane::flip(raw.log, lane) : 0;
        const Lane l(in_row, lane, p.depth);
        Quad quads[Lane::HALVES];
        float d[kPieceNumbers], v[kPieceNumbers];
        if (c < chunks) {
            l.fetch(quads, static_cast<const Out*>(raw.x) + (at.lo + r) * raw.stride);
            if (raw.log > 0) l.diagonal(d, raw.diag, raw.norm);
        }
        if (k < runs) fetch(now, k);
        if (c < chunks) {
            widen_quads<Out>(quads, v);
            if (raw.log > 0) Lane::within(v, d, raw.log, lane);
            if (raw.log > 9) Lane::meet(v, meeting + c * 128, lane);
        }
        if (raw.log > 9) __syncthreads();
        if (c < chunks) {
            if (raw.log > 9) {
                const int own = in_row & (waves_of_run(raw.log) - 1);
                Lane::join(v, meeting + (c - own) * 128, waves_of_run(raw.log), own, lane);
            }
            unsigned codes;
            int byte[Lane::HALVES];
            const int col = l.encode(v, flip, lane, &codes, byte), start = in_row * kChunk;
            // (behind the row's end: zeros)
            reinterpret_cast<unsigned*>(own_codes)[c * 64 + (col - start) / 8] = col < p.depth ? codes : 0;
            if ((lane & ((32 >> Lane::LOW) - 1)) == 0)
#pragma unroll
                for (int h = 0; h < Lane::HALVES; ++h)
                    reinterpret_cast<uint8_t*>(own_scales)[c * 16 + (l.first - start + h * 256) / 32] = l.first + h * 256 < p.depth ? byte[h] : 0x7f;
        }
        __syncthreads();
    } else {
        if (k < runs) fetch(now, k);
    }
    for (; k + 4 < runs; k += 4) {
        fetch(next, k + 4);
        multiply(now, k);
        now = next;
    }
    if (k < runs) multiply(now, k);
    // what is left is less than a run: a step a wave
    if (const int s = runs * kRunSteps + wave; s * 64 < bytes) {
        const int count = (bytes - s * 64 - quarter * 16) >> 1;        // 16-bit numbers, or pairs of codes
        uintx4 fw[NT], fx;
        unsigned sw[NT], sx = 0x7f;
        if (!MX && bytes < 16) {
            fx = fetch_short(x, count);
#pragma unroll
            for (int t = 0; t < NT; ++t) fw[t] = fetch_short(w[t], count);
        } else {
            // (the first bytes of the row can be read in place of what lies outside)
            if constexpr (RAW) fx = *reinterpret_cast<const uintx4*>(x + s * 64);
            else fx = fetch_some(x + s * 64, count, x - quarter * 16);
#pragma unroll
            for (int t = 0; t < NT; ++t) fw[t] = fetch_some(w[t] + s * 64, count, w[t] - quarter * 16);
        }
        if constexpr (MX) {
            const int at_scale = s * 4 + (count > 0 ? quarter : 0);
            sx = count > 0 ? xs[at_scale] : 0x7f;
#pragma unroll
            for (int t = 0; t < NT; ++t) sw[t] = count > 0 ? ws[t][at_scale] : 0x7f;
        }
        if (MX || bytes >= 16) {
            fx = keep_some(fx, count);
#pragma unroll
            for (int t = 0; t < NT; ++t) fw[t] = keep_some(fw[t], count);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if constexpr (MX) acc[t] = multiply16_scaled(fw[t], fx, acc[t], sw[t], sx);
            else acc[t] = multiply16<TYPE>(fw[t], fx, acc[t]);
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) part[in_group][t][lane] = acc[t];
    __syncthreads();
    // register v of lane l: column 4 (l / 16) + v, row l % 16
    const bool vector = p.out_stride % 4 == 0;
    if (in_group < NT * PARTS && r16 < rows_left) {
        const int first = in_group / NT * 4, t = in_group % NT, col = n0 + in_group * 16 + 4 * quarter;
        const floatx4 sum = (part[first][t][lane] + part[first + 1][t][lane]) + (part[first + 2][t][lane] + part[first + 3][t][lane]);
        Out* out = reinterpret_cast<Out*>(p.out) + (at.lo + r16) * p.out_stride + col;
        store_four(out, sum[0], sum[1], sum[2], sum[3], p.width - col, vector);
    }
}

// ------------------------------------------------------------------ sums over shares of the depth
// out = the sum of `splits` partial results of `count` numbers each, four numbers a thread, always in the same order
template <typename Out>
__global__ void __launch_bounds__(256) join_kernel(const float* __restrict__ partial, int splits, long long count, Out* __restrict__ out)
{
    const long long i = ((long long)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= count) return;
    const int left = count - i < 4 ? (int)(count - i) : 4;
    float v[4] = {0, 0, 0, 0};
    for (int s = 0; s < splits; ++s) {
        const float* from = partial + s * count + i;
        if (left == 4) {
            const Words4 t = *reinterpret_cast<const Words4*>(from);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] += __uint_as_float(t.w[k]);
        } else {
#pragma unroll
            for (int k = 0; k < 3; ++k)
                if (k < left) v[k] += from[k];
        }
    }
    store_four(out + i, v[0], v[1], v[2], v[3], left, true);
}

// ------------------------------------------------------------------ launches
inline long long row_tiles_at_most(const ProductParams& p, int height)
{
    if (!p.ends) return (p.rows + height - 1) / height;
    const long long cut = p.experts + 1 < p.rows ? p.experts + 1 : p.rows;      // groups whose last tile is not full, the rows of no group too
    return p.rows / height + cut;
}
// Workgroups in as many grids as they need: a grid holds fewer than 2^32 threads, 2^23 workgroups of up to 512 less eight (a multiple of eight, so that
// the XCDs go on in turn).  Numbers of 32 bits do for every result that memory holds.
constexpr long long kMostBlocks = 0xffffffffLL, kGridBlocks = (1LL << 23) - 8;
template <typename Launch>
hipError_t launch_grids(const ProductParams& p, long long blocks, Launch launch)
{
    if (blocks > kMostBlocks) return hipErrorInvalidConfiguration;
    ProductParams q = p;
    for (long long first = 0; first < blocks; first += kGridBlocks) {
        q.first_block = (unsigned)first;
        launch(q, (unsigned)(blocks - first < kGridBlocks ? blocks - first : kGridBlocks));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int DIRECTION, int TYPE, int BM, int BN, int STAGES, bool ANY, typename Out>
hipError_t launch_whole_tiles(const ProductParams& p, hipStream_t s)
{
    const long long columns = (p.width + BN - 1) / BN;
    long long blocks;
    if (DIRECTION == kDw) blocks = (columns * ((p.height + BM - 1) / BM) + 7) / 8 * 8 * p.experts;
    else blocks = (row_tiles_at_most(p, BM) * columns + 7) / 8 * 8;
    return launch_grids(p, blocks, [&](const ProductParams& q, unsigned count) {
        hipLaunchKernelGGL((product_kernel<DIRECTION, TYPE, BM, BN, 2, 2, STAGES, ANY, Out>), dim3(count, p.splits), dim3(256), 0, s, q);
    });
}

template <int DIRECTION, int TYPE, int BM, int BN, int STAGES, bool ANY, typename Out>
hipError_t launch_tiles(const ProductParams& p, hipStream_t s)
{
    if constexpr (DIRECTION == kDw)
        if (p.splits > 1) {
            ProductParams q = p;
            const long long count = (long long)p.experts * p.height * p.width, blocks = (count + 1023) / 1024;
            q.out = static_cast<char*>(p.workspace);
            q.split_stride = count;
            const hipError_t e = launch_whole_tiles<DIRECTION, TYPE, BM, BN, STAGES, ANY, float>(q, s);
            if (e != hipSuccess) return e;
            hipLaunchKernelGGL(join_kernel<Out>, dim3((unsigned)blocks), dim3(256), 0, s, static_cast<const float*>(p.workspace), p.splits, count,
                               reinterpret_cast<Out*>(p.out));
            return hipGetLastError();
        }
    return launch_whole_tiles<DIRECTION, TYPE, BM, BN, STAGES, ANY, Out>(p, s);
}

template <int TYPE, int NT, typename Out, bool RAW>
hipError_t launch_few_rows(const ProductParams& p, const RawRows& raw, hipStream_t s)
{
    constexpr int width = 16 * NT * (RAW ? 2 : 1);
    const long long columns = (p.width + width - 1) / width;
    const long long blocks = (row_tiles_at_most(p, 16) * columns + 7) / 8 * 8;
    return launch_grids(p, blocks, [&](const ProductParams& q, unsigned count) {
        hipLaunchKernelGGL((few_rows_kernel<TYPE, NT, Out, RAW>), dim3(count), dim3(RAW ? 512 : 256), 0, s, q, (unsigned)columns, raw);
    });
}

// whether every row that a kernel loads in pieces of 16 bytes is made of whole aligned ones, and 256 rows lie within 32 bits
constexpr long long kFarthestRow = 1 << 23;
template <int DIRECTION, int TYPE>
bool whole_pieces(const ProductParams& p)
{
    if (TYPE == kMx4) return true;                                    // rows of 16 bytes for each 32 numbers, at most 2^23 bytes
    if (p.a_stride > kFarthestRow || p.b_stride > kFarthestRow) return false;
    const int a_row = DIRECTION == kDw ? p.height : p.depth;
    const int b_row = DIRECTION == kForward ? p.depth : p.width;
    return a_row % 8 == 0 && b_row % 8 == 0 && p.a_stride % 16 == 0 && p.b_stride % 16 == 0 && p.b_group % 16 == 0;
}

// Weights' rows a workgroup: more of them share the rows of `a`, fewer leave more workgroups.  16 / 32 / 64, in us: 4 bits, 1 row, n = 8192,
// k = 8192 8.8 / 9.9 / 13.7; 16 rows, n = 16384, k = 4096 11.9 / 10.2 / 9.8; 64 rows of 32 experts, n = 4096, k = 2048 26.3 / 22.9 / 22.5;
// bf16, 16 rows, n = 4096, k = 4096 9.9 / 15.0 / 21.5; 24 rows of 8 experts, n = 8192, k = 2048 42.4 / 41.4 / 47.7
template <int TYPE, typename Out, bool RAW>
hipError_t launch_few_rows_as(const ProductParams& p, const RawRows& raw, hipStream_t s)
{
    const long long sixteens = (p.width + 15) / 16 * (long long)(p.experts < p.rows ? p.experts : p.rows);
    if constexpr (RAW) {
        // (columns for two groups of waves, every workgroup quantises)  16 / 32, in us, bf16: one row, k = 4096, n = 8192 5.85 / 8.1, n = 16384 9.3 / 10.2, 32768 17.2 / 14.2,
        // 65536 28.4 / 27.0; k = 2048, n = 32768 11.4 / 9.1; four rows, k = 1024, n = 65536 15.3 / 12.3
        if (sixteens >= 2048) return launch_few_rows<TYPE, 2, Out, true>(p, raw, s);
        return launch_few_rows<TYPE, 1, Out, true>(p, raw, s);
    } else {
        if constexpr (TYPE == kMx4)
            if (sixteens >= 4096) return launch_few_rows<TYPE, 4, Out, false>(p, raw, s);
        if (sixteens >= 1024) return launch_few_rows<TYPE, 2, Out, false>(p, raw, s);
        return launch_few_rows<TYPE, 1, Out, false>(p, raw, s);
    }
}

template <int DIRECTION, int TYPE, typename Out>
hipError_t launch_product_as(const ProductParams& p, hipStream_t s)
{
    if constexpr (DIRECTION == kForward)
        if (p.tile == kFewRows) return launch_few_rows_as<TYPE, Out, false>(p, RawRows{}, s);
    if constexpr (TYPE != kMx4) {
        // (the same order of the sums as with whole pieces: each number's in the order of the depth, or a quarter of each chunk a wave.)  y, dx, dw in us beside the next sizes of whole
        // pieces: 16384 x 4095 x 4097 837, 871, 1200 for 411, 419, 432; 20000 x 301 x 403, 16 experts 27, 23, 127 for 17, 12, 45; 24 x 4095 x 2047, 8 experts (y: few rows) 62, 44, 80 for 21, 25, 53
        if (!whole_pieces<DIRECTION, TYPE>(p))
            return p.tile == kTile64 ? launch_tiles<DIRECTION, TYPE, 64, 64, 2, true, Out>(p, s) : launch_tiles<DIRECTION, TYPE, 128, 128, 2, true, Out>(p, s);
        if (p.tile == kTile128Deep) return launch_tiles<DIRECTION, TYPE, 128, 128, 4, false, Out>(p, s);
    }
    switch (p.tile) {
    case kTile256: return launch_tiles<DIRECTION, TYPE, 256, 256, 2, false, Out>(p, s);
    case kTile64: return launch_tiles<DIRECTION, TYPE, 64, 64, 4, false, Out>(p, s);
    default: return launch_tiles<DIRECTION, TYPE, 128, 128, 2, false, Out>(p, s);
    }
}

}  // namespace spinner
