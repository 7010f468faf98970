// pex_ortho.hip -- Newton-Schulz orthogonalisation of matrices, and the Muon update around it.
//
// X_0 = M / (|M|_F + eps);  A = X X^T,  P = a I + b A + c A^2,  X <- P X, `steps` times, on the side with fewer rows (M is taken as
// its transpose where it is taller than wide): s rows, l >= s columns.  Per step s^2 l + s^3 + 2 s^2 l operations: A and A^2 are
// symmetric, half of their blocks are computed.
//
// Products on the fp16 matrix cores.  A value is held as two pieces, x = hi + lo to 22 bits and more, and a product is hi hi + hi lo + lo hi
// (lo lo is below 2^-22 of it): off by 3e-7 of the 2-norm where fp32 products give 2e-6 to 1e-5 (their order of additions), at three products
// instead of one that runs at a tenth of the rate.  bf16 matrices too: what their result is off by is then its own rounding, 1.66e-3.  As
// one piece (11 bits) they take half of the time (12 of 768 x 768: 260 us instead of 460) and are off by 2.1e-3.  Powers of two keep
// the pieces inside fp16's range: X by 2^12, A by 2^9, P by 2^10; the host refuses coefficients under which singular values leave [0, 4] or
// P's leave [-31, 31].
//
// Layout: every operand lies in the order in which the matrix cores take it, fragments of 16 rows x 32 columns, 64 lanes x 8 values =
// 1 KiB, lane (row % 16) + 16 * (column / 8 % 4).  Four fragments are a unit of 32 rows and columns, fragment 2 r + x: rows 16 r .., piece x;
// units of the same rows follow each other.  So a fragment is one direct-to-LDS load without any address arithmetic per lane, LDS reads are
// conflict-free, and no product needs a transposing read: both operands of every product are rows (A and P are symmetric), which costs X a second copy by columns that the kernel
// that makes X writes beside the first.  Sides are padded with zeros to whole blocks; zeros stay zeros.
// (16 x 16 x 32: these products are bound by power, and of nothing but them the chip sustains 1630 TFLOP/s on Gaussian fp16 values, of
// 32 x 32 x 16 ones 1430.)
#include <cmath>

#include "pex_internal.h"
#include "pex_lds_dma.h"

namespace pex {
namespace {

typedef __attribute__((ext_vector_type(2))) float float2_t;
typedef __attribute__((ext_vector_type(4))) float float4_t;
typedef __attribute__((ext_vector_type(4))) unsigned int uint4_t;
typedef __attribute__((ext_vector_type(4))) _Float16 half4_t;
typedef __attribute__((ext_vector_type(8))) _Float16 half8_t;

constexpr int FRAG = 512;                                   // halves of a fragment
constexpr float SCALE_X = 0x1p12f, SCALE_A = 0x1p9f, SCALE_P = 0x1p10f;

// One product C = factor U V^T + alpha V^T + beta U + gamma I of one matrix (or of `copies` of them, `stride` bytes apart in the workspace): U's
// and V's rows are operands, `units` of 32 rows of them a row of blocks; m32, n32: C's sides by 32.  Symmetric products (all but those with
// X) compute the blocks on and above the diagonal; beta only there.
struct Job {
    const _Float16 *U, *V;
    _Float16 *by_rows, *by_cols;    // C and its transpose as operands (symmetric: the same place)
    void* out;                      // not NULL: the result (or theta), row-major rows x cols, instead
    int64_t stride, out_stride;
    int m32, n32, units, symmetric, copies, rows, cols;
    float factor, alpha, beta, gamma;
    float step;                     // of an update: theta <- theta - step * C - decay * theta
    unsigned first;                 // first workgroup
    // ns_staged_kernel, DIVIDED: of each of `chunks` runs of a copy's blocks the last `rest` are in `parts` of `share` units; the parts, and
    // how many of a block's are there
    int share, parts, chunks, rest;
    float4_t* shares;
    unsigned* arrived;
};
constexpr int JOBS = 24;
struct Jobs {
    int count;
    float decay;
    Job job[JOBS];
};

__device__ __forceinline__ void split(float v, _Float16& hi, _Float16& lo)
{
    hi = (_Float16)v;
    lo = (_Float16)(v - (float)hi);
}
__device__ __forceinline__ float4_t mfma(const half8_t& x, const half8_t& y, const float4_t& z) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, z, 0, 0, 0); }

// The block a workgroup computes: block (bi, bj) of M x N units of 32 of copy `copy` of job `job`
struct Block {
    int job, copy, bi, bj;
};
// consecutive blocks of one matrix on one XCD: they share panels
__device__ __forceinline__ unsigned workgroup_id()
{
    const unsigned n = gridDim.x, xcd = blockIdx.x % 8, base = n / 8, rem = n % 8;
    return xcd * base + (xcd < rem ? xcd : rem) + blockIdx.x / 8;
}
// block t = bj (bj + 1) / 2 + bi of the triangle
__device__ __forceinline__ void of_triangle(int t, Block& b)
{
    b.bj = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
    while ((b.bj + 1) * (b.bj + 2) / 2 <= t) ++b.bj;
    while (b.bj * (b.bj + 1) / 2 > t) --b.bj;
    b.bi = t - b.bj * (b.bj + 1) / 2;
}
template <int M, int N>
__device__ __forceinline__ Block block_of(const Jobs& jobs)
{
    const unsigned id = workgroup_id();
    Block b{};
    while (b.job + 1 < jobs.count && id >= jobs.job[b.job + 1].first) ++b.job;
    const Job& j = jobs.job[b.job];
    const int tm = j.m32 / M, tn = j.n32 / N;
    const int blocks = j.symmetric ? tm * (tm + 1) / 2 : tm * tn;
    b.copy = (int)(id - j.first) / blocks;
    const int t = (int)(id - j.first) - b.copy * blocks;
    if (j.symmetric) of_triangle(t, b);
    else {
        b.bi = t % tm;
        b.bj = t / tm;
    }
    return b;
}

// ---- what is done with a tile of 32 x 32 of C, unit (i32, j32): of its four quarters g = 2 r + c a lane holds the entries of rows
// 16 r + 4 (lane / 16) + e, e = 0 .. 3, and column 16 c + lane % 16; a call takes those of one quarter
struct Tile {
    float4_t q[4];
};

// a lane's row, within its tile, of quarter g and entry 0; its column
__device__ __forceinline__ int row_of(int g, int lane) { return 16 * (g >> 1) + 4 * (lane >> 4); }
__device__ __forceinline__ int col_of(int g, int lane) { return 16 * (g & 1) + (lane & 15); }

// fragment `x` (piece) of rows 16 r .. of unit (row, column) of an operand of `cols32` times 32 columns, in halves
__device__ __forceinline__ int64_t fragment_at(int row32, int col32, int cols32, int r, int x)
{
    return (((int64_t)row32 * cols32 + col32) * 4 + 2 * r + x) * FRAG;
}
// where piece p of a quarter lies in C's transpose: half a lane's 16 bytes of a fragment
__device__ __forceinline__ half4_t* place(char* base, int rows32, int i32, int j32, int g, int p, int lane)
{
    return (half4_t*)((_Float16*)base + fragment_at(j32, i32, rows32, g & 1, p) + ((lane & 15) + 16 * (2 * (g >> 1) + (lane >> 5))) * 8 + 4 * (lane >> 4 & 1));
}

// the result itself: quarters [from, to) of a tile
template <typename TOut, bool UPDATE>
__device__ __forceinline__ void put_out(const Jobs& jobs, const Job& j, int copy, int i32, int j32, int from, int to, const Tile& x, int lane)
{
    TOut* out = (TOut*)((char*)j.out + (int64_t)copy * j.out_stride);
    float theta[4][4];
    auto each = [&](auto f) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int col = j32 * 32 + col_of(g, lane), row0 = i32 * 32 + row_of(g, lane);
            if (g < from || g >= to || col >= j.cols) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (row0 + e < j.rows) f(g, e, (int64_t)(row0 + e) * j.cols + col);
        }
    };
    if constexpr (UPDATE) each([&](int g, int e, int64_t at) { theta[g][e] = out[at]; });       // all in flight before the first is stored
    each([&](int g, int e, int64_t at) {
        const float o = x.q[g][e] * j.factor;
        if constexpr (UPDATE) out[at] = fmaf(-j.step, o, theta[g][e]) - jobs.decay * theta[g][e];
        else if constexpr (sizeof(TOut) == 2) out[at] = __builtin_bit_cast(uint16_t, (__bf16)o);
        else out[at] = o;
    });
}

// The entries of C as pieces, written by columns; hi | lo << 16 of the four come back for the copy by rows
__device__ __forceinline__ void put_by_cols(const Job& j, int64_t at, int i32, int j32, int g, float4_t x, uint32_t (&packed)[4], int lane)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[e] *= j.factor;
        if (i32 == j32 && row_of(g, lane) + e == col_of(g, lane)) x[e] += j.gamma;
    }
    auto add = [&](const _Float16* from, float times) {
        char* base = (char*)from + at;
        const half4_t hi = *place(base, j.m32, i32, j32, g, 0, lane), lo = *place(base, j.m32, i32, j32, g, 1, lane);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = fmaf(times, (float)hi[e] + (float)lo[e], x[e]);
    };
    if (j.alpha != 0.f) add(j.V, j.alpha);
    if (j.beta != 0.f) add(j.U, j.beta);
    half4_t hi, lo;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        _Float16 a, b;
        split(x[e], a, b);
        hi[e] = a;
        lo[e] = b;
        packed[e] = (uint32_t)__builtin_bit_cast(uint16_t, a) | (uint32_t)__builtin_bit_cast(uint16_t, b) << 16;
    }
    char* to = (char*)j.by_cols + at;
    *place(to, j.m32, i32, j32, g, 0, lane) = hi;
    *place(to, j.m32, i32, j32, g, 1, lane) = lo;
}

constexpr int TURN = 32 * 32;        // dwords of LDS in which a tile is turned; column c of row r lies at c ^ r: different banks both ways
__device__ __forceinline__ void turn_in(uint32_t* turn, int g, const uint32_t (&packed)[4], int lane)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int row = row_of(g, lane) + e;
        turn[row * 32 + (col_of(g, lane) ^ row)] = packed[e];
    }
}
// rows 16 r .. of a turned tile
__device__ __forceinline__ void put_by_rows(const Job& j, int64_t at, int i32, int j32, int r, const uint32_t* turn, int lane)
{
    const int row = 16 * r + (lane & 15);
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = turn[row * 32 + ((8 * (lane >> 4) + e) ^ row)];
    uint4_t piece[2];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        piece[0][e] = (w[2 * e] & 0xffffu) | w[2 * e + 1] << 16;
        piece[1][e] = w[2 * e] >> 16 | (w[2 * e + 1] & 0xffff0000u);
    }
#pragma unroll
    for (int p = 0; p < 2; ++p)
        *(uint4_t*)((_Float16*)((char*)j.by_rows + at) + fragment_at(i32, j32, j.n32, r, p) + lane * 8) = piece[p];
}

// a whole tile by one wave; `turn` is its own
template <typename TOut, bool UPDATE>
__device__ __forceinline__ void put_tile(const Jobs& jobs, const Job& j, const Block& b, int64_t at, int i32, int j32, const Tile& x, uint32_t* turn, int lane)
{
    if (j.out) {
        put_out<TOut, UPDATE>(jobs, j, b.copy, i32, j32, 0, 4, x, lane);
        return;
    }
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        uint32_t packed[4];
        put_by_cols(j, at, i32, j32, g, x.q[g], packed, lane);
        turn_in(turn, g, packed, lane);
    }
    if (j.symmetric && b.bi == b.bj) return;     // a block on the diagonal is its own transpose
    __builtin_amdgcn_wave_barrier();
    put_by_rows(j, at, i32, j32, 0, turn, lane);
    put_by_rows(j, at, i32, j32, 1, turn, lane);
    __builtin_amdgcn_wave_barrier();
}

// The products of one tile and one unit of columns: from zero, the small ones first; their sum is added to the tile by vector
// instructions, which round to nearest (the matrix cores do not, and a long chain of them drifts).
__device__ __forceinline__ void products(const half8_t (&u)[4], const half8_t (&v)[4], Tile& d)
{
#pragma unroll
    for (int g = 0; g < 4; ++g) d.q[g] = mfma(u[(g & 2) + 1], v[2 * (g & 1)], float4_t{0.f, 0.f, 0.f, 0.f});
#pragma unroll
    for (int g = 0; g < 4; ++g) d.q[g] = mfma(u[g & 2], v[2 * (g & 1) + 1], d.q[g]);
#pragma unroll
    for (int g = 0; g < 4; ++g) d.q[g] = mfma(u[g & 2], v[2 * (g & 1)], d.q[g]);
}
__device__ __forceinline__ void clear(Tile& t)
{
#pragma unroll
    for (int g = 0; g < 4; ++g) t.q[g] = float4_t{0.f, 0.f, 0.f, 0.f};
}
__device__ __forceinline__ void add(Tile& t, const Tile& d)
{
#pragma unroll
    for (int g = 0; g < 4; ++g) t.q[g] += d.q[g];
}

// ---- few blocks: operands straight from the caches to registers, four waves of a workgroup divide the columns of U and V among them.
// No barrier in the loop and a load ahead: bound by latency where there are few blocks (symmetric 512 x 512 x 512 in 6 us), otherwise by what
// the compute units take from their L2 (symmetric 1024 x 1024 x 1024 in 12 us: 528 blocks of 32 read 138 MB of panels, 11 TB/s).
template <int F, typename TOut, bool UPDATE>
__global__ __launch_bounds__(256) void ns_direct_kernel(Jobs jobs)
{
    constexpr int WAVES = 4;
    __shared__ float4_t sums[WAVES * F * F * 256];
    __shared__ uint32_t turned[F == 1 ? TURN : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const Block b = block_of<F, F>(jobs);
    const Job& j = jobs.job[b.job];
    const int64_t at = (int64_t)b.copy * j.stride, panel = (int64_t)j.units * 256;      // 16-byte pieces of 32 rows
    const half8_t* u0 = (const half8_t*)((const char*)j.U + at) + b.bi * F * panel + lane;
    const half8_t* v0 = (const half8_t*)((const char*)j.V + at) + b.bj * F * panel + lane;
    Tile acc[F][F];
#pragma unroll
    for (int m = 0; m < F; ++m)
#pragma unroll
        for (int n = 0; n < F; ++n) clear(acc[m][n]);
    half8_t u[F][4], v[F][4];
    auto load = [&](int s) {
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int m = 0; m < F; ++m) {
                u[m][x] = u0[m * panel + (s * 4 + x) * 64];
                v[m][x] = v0[m * panel + (s * 4 + x) * 64];
            }
    };
    const int steps = j.units;
    int s = wave;
    if (s < steps) load(s);
    for (; s < steps; s += WAVES) {
        half8_t cu[F][4], cv[F][4];
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int m = 0; m < F; ++m) {
                cu[m][x] = u[m][x];
                cv[m][x] = v[m][x];
            }
        if (s + WAVES < steps) load(s + WAVES);
#pragma unroll
        for (int m = 0; m < F; ++m)
#pragma unroll
            for (int n = 0; n < F; ++n) {
                Tile d;
                products(cu[m], cv[n], d);
                add(acc[m][n], d);
            }
    }
    // the waves' sums, in their order
#pragma unroll
    for (int m = 0; m < F; ++m)
#pragma unroll
        for (int n = 0; n < F; ++n)
#pragma unroll
            for (int g = 0; g < 4; ++g) sums[((wave * F + m) * F + n) * 256 + g * 64 + lane] = acc[m][n].q[g];
    __syncthreads();
    auto sum = [&](int tile, int g) {
        const float4_t* p = sums + tile * 256 + g * 64 + lane;
        constexpr int W = F * F * 256;
        return ((p[0] + p[W]) + p[2 * W]) + p[3 * W];
    };
    if constexpr (F == 1) {                 // a wave takes a quarter of the tile
        Tile x;
#pragma unroll
        for (int g = 0; g < 4; ++g)
            if (g == wave) x.q[g] = sum(0, g);
        if (j.out) {
            put_out<TOut, UPDATE>(jobs, j, b.copy, b.bi, b.bj, wave, wave + 1, x, lane);
            return;
        }
        uint32_t packed[4];
        put_by_cols(j, at, b.bi, b.bj, wave, sum(0, wave), packed, lane);
        if (j.symmetric && b.bi == b.bj) return;
        turn_in(turned, wave, packed, lane);
        __syncthreads();
        if (wave < 2) put_by_rows(j, at, b.bi, b.bj, wave, turned, lane);
    } else {                                // a tile
        Tile x;
#pragma unroll
        for (int g = 0; g < 4; ++g) x.q[g] = sum(wave, g);
        __builtin_amdgcn_wave_barrier();
        put_tile<TOut, UPDATE>(jobs, j, b, at, b.bi * F + wave / F, b.bj * F + wave % F, x,
                                       (uint32_t*)(sums + wave * 256), lane);       // (what wave 0 left of this tile; nobody else reads it)
    }
}

// ---- many blocks: operands through LDS, eight waves a workgroup (4 x 2 of them), slots filled by direct-to-LDS loads.  A wave keeps its
// row fragments and streams the column fragments: those of the next tiles are read under the products of the present ones, across
// the one barrier a slot has (before the products with the last column fragment: by then the wave has read all of the slot, and all of the
// next one has arrived).  Blocks of 256 x 256 (128 KiB of LDS) or, two workgroups to a compute unit, 128 x 128; where there are no two
// workgroups for each, four slots for one: loads are on their way for longer.
// Measured, two matrices, 2048 x 8192 = (2048 x 2048) (2048 x 8192): 256 346 us = 1193 TFLOP/s of fp16 products, 128 394 (1047), the kernel
// above with 64 612 (673); 272 blocks of 128 of a symmetric 2048 x 2048 x 8192 250 us, in blocks of 256 455, of 64 316.
__device__ __forceinline__ void dma_16_at(uint32_t lds_addr, uint32_t voff, uint32_t soff, int4_t rsrc)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds_addr), "v"(voff), "s"(rsrc), "s"(soff) : "memory", "m0");
}

template <int B> constexpr int slot_bytes() { return 2 * B / 32 * 4096; }

// DIVIDED (symmetric products): some blocks are divided along their columns, one part a workgroup; the parts go to memory, and who comes last
// adds them up, in their order: nobody waits.  All parts of one range of columns are next to each other, so that their workgroups share
// panels in the L2 (every workgroup its own range: two of 2048 x 8192 took 16 % more time instead of 5 % less).
template <int B, typename TOut, bool UPDATE, bool DIVIDED, int SLOTS = 2>
__global__ __launch_bounds__(512, B == 256 || SLOTS > 2 ? 2 : 4) void ns_staged_kernel(Jobs jobs)
{
    constexpr int WM = 4, WN = 2, FM = B / WM / 32, FN = B / WN / 32, SLOT = slot_bytes<B>(), LOADS = SLOT / 1024 / 8;
    constexpr int PART = B * B / 2;         // a block, in pairs of fp32
    static_assert(LOADS % 4 == 0 && FN % 2 == 0, "a wave fills the parts of whole units of 32 rows; column fragments go in pairs of registers");
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    Block b{};
    int block = 0, part = 0, slot = -1;          // slot: of a divided block's parts
    if constexpr (DIVIDED) {
        const unsigned id = workgroup_id();
        while (b.job + 1 < jobs.count && id >= jobs.job[b.job + 1].first) ++b.job;
        const Job& j = jobs.job[b.job];
        const int side = j.m32 / (B / 32), blocks = side * (side + 1) / 2, more = j.rest * (j.parts - 1), local = (int)(id - j.first);
        b.copy = local / (blocks + j.chunks * more);
        const int in = local - b.copy * (blocks + j.chunks * more), size = blocks / j.chunks, longer = blocks - size * j.chunks;
        int chunk = 0, start = 0, next = size + (longer > 0);           // blocks
        while (chunk + 1 < j.chunks && in >= next + (chunk + 1) * more) {
            ++chunk;
            start = next;
            next += size + (chunk < longer);
        }
        const int at = in - start - chunk * more, whole = next - start - j.rest;
        if (at < whole) block = start + at;
        else {
            part = (at - whole) / j.rest;
            const int k = at - whole - part * j.rest;
            block = start + whole + k;
            slot = chunk * j.rest + k;
        }
        of_triangle(block, b);
    } else b = block_of<B / 32, B / 32>(jobs);
    const Job& j = jobs.job[b.job];
    const int64_t at = (int64_t)b.copy * j.stride;
    int begin = 0, stages = j.units;
    if constexpr (DIVIDED)
        if (slot >= 0) {
            begin = part * j.share;
            stages = min(j.share, j.units - begin);
        }
    const uint32_t row_bytes = (uint32_t)j.units * 4096u;               // of 32 rows
    // this wave's units of 32 rows of a slot
    constexpr int MINE = LOADS / 4;
    const int unit = wave * MINE;
    const bool is_v = unit >= B / 32;
    const char* base = is_v ? (const char*)j.V + at + (int64_t)(b.bj * (B / 32) + unit - B / 32) * row_bytes
                            : (const char*)j.U + at + (int64_t)(b.bi * (B / 32) + unit) * row_bytes;
    const int4_t rsrc = make_rsrc(base, MINE * row_bytes);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void)lds + (uint32_t)(wave * LOADS * 1024), voff = (uint32_t)lane * 16u;
    auto issue = [&](int s, int slot) {
        const uint32_t off = (uint32_t)(begin + (s < stages ? s : 0)) * 4096u;      // past the end: the first once more, which nobody reads
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            dma_16_at(lds0 + (uint32_t)(slot * SLOT + i * 1024), voff, off + (uint32_t)(i / 4) * row_bytes + (uint32_t)(i % 4) * 1024u, rsrc);
    };
    const int wm = wave / WN, wn = wave % WN;
    Tile acc[FM][FN];
#pragma unroll
    for (int m = 0; m < FM; ++m)
#pragma unroll
        for (int n = 0; n < FN; ++n) clear(acc[m][n]);
    half8_t u[FM][4], v[2][4];
    const half8_t* f = (const half8_t*)lds + lane;
    auto read_u = [&](int m, int slot) {
#pragma unroll
        for (int x = 0; x < 4; ++x) u[m][x] = f[(slot * SLOT + ((wm * FM + m) * 4 + x) * 1024) / 16];
    };
    auto read_v = [&](int n, int slot) {
#pragma unroll
        for (int x = 0; x < 4; ++x) v[n & 1][x] = f[(slot * SLOT + ((B / 32 + wn * FN + n) * 4 + x) * 1024) / 16];
    };
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) issue(s, s);
    wait_vmcnt<(SLOTS - 1) * LOADS>();
    wait_lds_and_barrier();
    read_v(0, 0);
#pragma unroll
    for (int m = 0; m < FM; ++m) read_u(m, 0);
    Tile d[2];
    for (int s = 0; s < stages; ++s) {
        const int slot = s & (SLOTS - 1), next = (s + 1) & (SLOTS - 1);
#pragma unroll
        for (int n = 0; n < FN; ++n) {
            if (n == FN - 1) {
                wait_vmcnt<(SLOTS - 2) * LOADS>();
                wait_lds_and_barrier();
                read_v(0, next);
            } else read_v(n + 1, slot);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int m = 0; m < FM; ++m) {
                const int t = n * FM + m;
                products(u[m], v[n & 1], d[t & 1]);
                __builtin_amdgcn_sched_barrier(0);
                if (t > 0) add(acc[(t - 1) % FM][(t - 1) / FM], d[(t - 1) & 1]);
                if (n == FN - 1) read_u(m, next);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        issue(s + SLOTS, slot);
        add(acc[FM - 1][FN - 1], d[(FM * FN - 1) & 1]);
    }
    wait_vmcnt<0>();
    wait_lds_and_barrier();                    // the slots are free
    if constexpr (DIVIDED) {
        if (slot >= 0) {
            // past this XCD's L2, store by store: a fence for the device would drop what other workgroups read from it (two 2048 x 8192:
            // 6457 us instead of 2601)
            uint64_t* shares = (uint64_t*)((char*)j.shares + at) + (int64_t)slot * j.parts * PART + (wave * 64 + lane);
            uint64_t* mine = shares + part * PART;
#pragma unroll
            for (int q = 0; q < FM * FN * 4; ++q)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float2_t x = {acc[q / 4 / FN][q / 4 % FN].q[q % 4][2 * h], acc[q / 4 / FN][q / 4 % FN].q[q % 4][2 * h + 1]};
                    __hip_atomic_store(mine + (2 * q + h) * 512, __builtin_bit_cast(uint64_t, x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                }
            wait_vmcnt<0>();                   // they are there
            wait_lds_and_barrier();
            unsigned* last = (unsigned*)lds;
            unsigned* arrived = (unsigned*)((char*)j.arrived + at) + slot;
            if (threadIdx.x == 0) *last = __hip_atomic_fetch_add(arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1u == (unsigned)j.parts;
            __syncthreads();
            const bool join = __builtin_amdgcn_readfirstlane((int)*last);
            __syncthreads();                   // (LDS is used again)
            if (!join) return;
            if (threadIdx.x == 0) __hip_atomic_store(arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);       // for the next product
#pragma unroll
            for (int m = 0; m < FM; ++m)
#pragma unroll
                for (int n = 0; n < FN; ++n) clear(acc[m][n]);
            for (int p = 0; p < j.parts; ++p)
#pragma unroll
                for (int q = 0; q < FM * FN * 4; ++q)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float2_t x = __builtin_bit_cast(float2_t, __hip_atomic_load(shares + p * PART + (2 * q + h) * 512, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
                        acc[q / 4 / FN][q / 4 % FN].q[q % 4][2 * h] += x[0];
                        acc[q / 4 / FN][q / 4 % FN].q[q % 4][2 * h + 1] += x[1];
                    }
        }
    }
    uint32_t* turn = (uint32_t*)lds + wave * TURN;
#pragma unroll
    for (int m = 0; m < FM; ++m)
#pragma unroll
        for (int n = 0; n < FN; ++n)
            put_tile<TOut, UPDATE>(jobs, j, b, at, b.bi * (B / 32) + wm * FM + m, b.bj * (B / 32) + wn * FN + n, acc[m][n], turn, lane);
}

// ---- before the products: the norm, and X_0 as operands --------------------------------------------------------------
//
// Bound by HBM: of two 2048 x 8192 matrices with their momentum (Muon) the norm reads and writes 400 MB in 70 us, the preparation
// 540 MB in 107.  The sum of squares is taken in 64 bits, in the order of the parts.

// One matrix (or `copies` of them): M, or for an update the momentum and the gradient it takes in
struct Source {
    void* M;
    const float* S;
    _Float16 *by_rows, *by_cols;
    double* partial;                 // sums of squares of `parts` chunks of each copy
    int64_t stride, in_stride;       // bytes between copies: workspace, M
    int rows, cols, s_tiles, l_tiles, parts, copies;      // tiles of 64, of the padded sides
    unsigned first_sum, first_tile;
    unsigned* arrived;               // cleared
    int blocks;
};
// What an update makes of the momentum m and the gradient g: the next momentum, and what is orthogonalised
struct Momentum {
    float beta, gain;                // gain = (1 - beta) * grad_scale
    int nesterov;
    __device__ __forceinline__ float next(float m, float g) const { return fmaf(beta, m, gain * g); }
    __device__ __forceinline__ float ahead(float m, float g) const { return nesterov ? fmaf(beta, m, gain * g) : m; }
};
struct Sources {
    int count;
    Momentum momentum;
    float eps;
    Source m[JOBS];
};

__device__ __forceinline__ float value_at(const uint16_t* p, int64_t i) { return __uint_as_float((uint32_t)p[i] << 16); }
__device__ __forceinline__ float value_at(const float* p, int64_t i) { return p[i]; }

// sum over a block of `WAVES` waves, the same in every lane
template <int WAVES>
__device__ __forceinline__ double block_sum(double s)
{
    __shared__ double red[WAVES];
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    double t = 0.0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) t += red[w];
    return t;
}

// What a matrix of this sum of squares is multiplied with.  Zeros stay zeros, where eps = 0 too.
__device__ __forceinline__ double to_unit(double ssq, float eps) { return ssq == 0.0 ? 0.0 : (double)SCALE_X / (sqrt(ssq) + (double)eps); }

// element e of a source before it is orthogonalised; an update takes the gradient into the momentum first
template <typename T, bool UPDATE>
__device__ __forceinline__ float taken_in(const Momentum& momentum, T* M, const float* S, int64_t e)
{
    float u = value_at(M, e);
    if constexpr (UPDATE) {
        const float g = S[e], next = momentum.next(u, g);
        M[e] = next;
        u = momentum.ahead(next, g);
    }
    return u;
}

template <typename T, bool UPDATE>
__global__ __launch_bounds__(256) void ns_norm_kernel(Sources src)
{
    int k = 0;
    while (k + 1 < src.count && blockIdx.x >= src.m[k + 1].first_sum) ++k;
    const Source& m = src.m[k];
    const int local = (int)(blockIdx.x - m.first_sum), copy = local / m.parts, part = local - copy * m.parts;
    T* M = (T*)((char*)m.M + (int64_t)copy * m.in_stride);
    const int64_t n = (int64_t)m.rows * m.cols, chunk = ((n + m.parts - 1) / m.parts + 1023) / 1024 * 1024;
    const int64_t begin = (int64_t)part * chunk, end = begin + chunk < n ? begin + chunk : n;
    for (int t = part * 256 + threadIdx.x; t < m.blocks; t += m.parts * 256) ((unsigned*)((char*)m.arrived + (int64_t)copy * m.stride))[t] = 0u;
    double s = 0.0;
    int64_t e = begin + threadIdx.x;
    for (; e + 7 * 256 < end; e += 8 * 256) {        // eight in flight
        float u[8], g[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            u[i] = value_at(M, e + i * 256);
            if (UPDATE) g[i] = m.S[e + i * 256];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (UPDATE) {
                const float next = src.momentum.next(u[i], g[i]);
                M[e + i * 256] = next;
                u[i] = src.momentum.ahead(next, g[i]);
            }
            s += (double)u[i] * u[i];
        }
    }
    for (; e < end; e += 256) {
        const float u = taken_in<T, UPDATE>(src.momentum, M, m.S, e);
        s += (double)u * u;
    }
    s = block_sum<4>(s);
    if (threadIdx.x == 0) ((double*)((char*)m.partial + (int64_t)copy * m.stride))[part] = s;
}

// A 64 x 64 tile of X_0: by rows and by columns
template <typename T, bool UPDATE>
__global__ __launch_bounds__(256) void ns_prepare_kernel(Sources src)
{
    __shared__ float tile[64][65];
    int k = 0;
    while (k + 1 < src.count && blockIdx.x >= src.m[k + 1].first_tile) ++k;
    const Source& m = src.m[k];
    const int tiles = m.s_tiles * m.l_tiles, local = (int)(blockIdx.x - m.first_tile), copy = local / tiles, t = local - copy * tiles;
    const bool tall = m.rows > m.cols;
    const int ti = t / m.l_tiles, tj = t - ti * m.l_tiles;
    const T* M = (const T*)((const char*)m.M + (int64_t)copy * m.in_stride);
    const double* partial = (const double*)((const char*)m.partial + (int64_t)copy * m.stride);
    // rows of M along the tile's rows, or, of a tall matrix, along its columns
    const int row0 = tall ? tj * 64 : ti * 64, col0 = tall ? ti * 64 : tj * 64, cl = threadIdx.x & 63;
    // all of them in flight at once (not one behind the other): those past an edge read the edge, and are zero
    float u[16], g[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int64_t e = (int64_t)min(row0 + 4 * i + (int)(threadIdx.x >> 6), m.rows - 1) * m.cols + min(col0 + cl, m.cols - 1);
        u[i] = value_at(M, e);
        if constexpr (UPDATE) g[i] = m.S[e];
    }
    double ssq = 0.0;
    for (int p = threadIdx.x; p < m.parts; p += 256) ssq += partial[p];
    ssq = block_sum<4>(ssq);
    const double inv = to_unit(ssq, src.eps);      // (beyond fp32's range for the smallest matrices)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int r = 4 * i + (int)(threadIdx.x >> 6);
        if constexpr (UPDATE) u[i] = src.momentum.ahead(u[i], g[i]);
        if (row0 + r >= m.rows || col0 + cl >= m.cols) u[i] = 0.f;
        tile[tall ? cl : r][tall ? r : cl] = (float)((double)u[i] * inv);
    }
    __syncthreads();
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int f = 0; f < 4; ++f) {
        const int id = wave * 4 + f, cols = id >> 3, a16 = id >> 1 & 3, b32 = id & 1;       // 8 fragments by rows, 8 by columns
        half8_t hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int a = a16 * 16 + (lane & 15), b = b32 * 32 + (lane >> 4) * 8 + e;
            _Float16 x, y;
            split(cols ? tile[b][a] : tile[a][b], x, y);
            hi[e] = x;
            lo[e] = y;
        }
        _Float16* to = (_Float16*)((char*)(cols ? m.by_cols : m.by_rows) + (int64_t)copy * m.stride);
        const int row32 = (cols ? tj : ti) * 2 + (a16 >> 1), col32 = (cols ? ti : tj) * 2 + b32, cols32 = (cols ? m.s_tiles : m.l_tiles) * 2;
        *((half8_t*)(to + fragment_at(row32, col32, cols32, a16 & 1, 0)) + lane) = hi;
        *((half8_t*)(to + fragment_at(row32, col32, cols32, a16 & 1, 1)) + lane) = lo;
    }
}

// ---- small matrices: everything in one workgroup ---------------------------------------------------------------------
//
// A matrix of at most 64 KiB in pieces (64 x 256, 128 x 128; padded to multiples of 64) stays in the LDS of one compute unit from
// its norm to the result: X by rows, then A, then P in one half, X by columns in the other; the tiles of a product (at most sixteen, two a
// wave) are in registers until everyone has read what they replace.  One launch where the kernels above take two and three a step, each of
// which costs 4 us whatever it does (64 x 64: 72 -> 27 us for fifteen products one after the other).
constexpr int SMALL_MOST = 16384;        // padded entries
constexpr int SMALL_WAVES = 8, SMALL_TILES = SMALL_MOST / 1024 / SMALL_WAVES;

struct SmallJob {
    void* M;
    const float* S;
    void* out;
    int rows, cols, copies;              // copies lie one behind the other
    float step;
    unsigned first;                      // first workgroup
};
constexpr int SMALL_JOBS = 48;
struct SmallJobs {
    int count, steps;
    Momentum momentum;
    float a, b, c, eps, decay;
    SmallJob job[SMALL_JOBS];
};

template <typename T, bool UPDATE>
__global__ __launch_bounds__(SMALL_WAVES * 64) void ns_small_kernel(SmallJobs jobs)
{
    constexpr int THREADS = SMALL_WAVES * 64, EACH = SMALL_MOST / THREADS;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    _Float16* first = (_Float16*)lds;                                // X by rows, A, P
    _Float16* second = first + SMALL_MOST * 2;                  // X by columns
    int k = 0;
    while (k + 1 < jobs.count && blockIdx.x >= jobs.job[k + 1].first) ++k;
    const SmallJob& j = jobs.job[k];
    const int64_t at = (int64_t)(blockIdx.x - j.first) * j.rows * j.cols;
    T* M = (T*)j.M + at;
    const bool tall = j.rows > j.cols;
    const int prows = (j.rows + 63) / 64 * 64, pcols = (j.cols + 63) / 64 * 64, padded = prows * pcols;
    const int s32 = (tall ? pcols : prows) / 32, l32 = (tall ? prows : pcols) / 32;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));

    float u[EACH];
    double ssq = 0.0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int q = i * THREADS + (int)threadIdx.x, r = q / pcols, c = q - r * pcols;
        u[i] = 0.f;
        if (q < padded && r < j.rows && c < j.cols) u[i] = taken_in<T, UPDATE>(jobs.momentum, M, j.S, (int64_t)r * j.cols + c);
        ssq += (double)u[i] * u[i];
    }
    ssq = block_sum<SMALL_WAVES>(ssq);
    const double inv = to_unit(ssq, jobs.eps);
    // entry (row, col) of an operand of cols32 times 32 columns
    auto put = [&](_Float16* to, int row, int col, int cols32, _Float16 hi, _Float16 lo) {
        _Float16* p = to + fragment_at(row >> 5, col >> 5, cols32, row >> 4 & 1, 0) + ((row & 15) + 16 * (col >> 3 & 3)) * 8 + (col & 7);
        p[0] = hi;
        p[FRAG] = lo;
    };
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int q = i * THREADS + (int)threadIdx.x, r = q / pcols, c = q - r * pcols;
        if (q >= padded) break;
        _Float16 hi, lo;
        split((float)((double)u[i] * inv), hi, lo);
        const int row = tall ? c : r, col = tall ? r : c;
        put(first, row, col, l32, hi, lo);
        put(second, col, row, s32, hi, lo);
    }
    __syncthreads();

    // this wave's tiles of U V^T; tile t of n
    Tile x[SMALL_TILES];
    auto multiply = [&](const _Float16* U, const _Float16* V, int units, int n, auto unit_of) {
#pragma unroll
        for (int i = 0; i < SMALL_TILES; ++i) {
            const int t = i * SMALL_WAVES + wave;
            clear(x[i]);
            if (t >= n) continue;
            int ti, tj;
            unit_of(t, ti, tj);
            const half8_t *pu = (const half8_t*)U + ti * units * 256 + lane, *pv = (const half8_t*)V + tj * units * 256 + lane;
            for (int s = 0; s < units; ++s) {
                half8_t fu[4], fv[4];
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    fu[f] = pu[s * 256 + f * 64];
                    fv[f] = pv[s * 256 + f * 64];
                }
                Tile d;
                products(fu, fv, d);
                add(x[i], d);
            }
        }
    };
    auto triangle = [](int t, int& ti, int& tj) {          // t = tj (tj + 1) / 2 + ti
        tj = 0;
        while ((tj + 1) * (tj + 2) / 2 <= t) ++tj;
        ti = t - tj * (tj + 1) / 2;
    };
    auto whole = [&](int t, int& ti, int& tj) { ti = t % s32; tj = t / s32; };
    // the tiles as operands: C by rows, its transpose
    auto put_tiles = [&](int n, auto unit_of, _Float16* by_rows, int rows_cols32, _Float16* by_cols, int cols_cols32) {
#pragma unroll
        for (int i = 0; i < SMALL_TILES; ++i) {
            const int t = i * SMALL_WAVES + wave;
            if (t >= n) continue;
            int ti, tj;
            unit_of(t, ti, tj);
            const bool diagonal = by_rows == by_cols && ti == tj;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                half4_t hi, lo;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    _Float16 a, b;
                    split(x[i].q[g][e], a, b);
                    hi[e] = a;
                    lo[e] = b;
                    if (!diagonal) put(by_rows, ti * 32 + row_of(g, lane) + e, tj * 32 + col_of(g, lane), rows_cols32, a, b);
                }
                *place((char*)by_cols, cols_cols32, ti, tj, g, 0, lane) = hi;
                *place((char*)by_cols, cols_cols32, ti, tj, g, 1, lane) = lo;
            }
        }
    };
    const int half_tiles = s32 * (s32 + 1) / 2, tiles = s32 * l32;
    for (int step = 0; step < jobs.steps; ++step) {
        multiply(first, first, l32, half_tiles, triangle);
#pragma unroll
        for (int i = 0; i < SMALL_TILES; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) x[i].q[g] *= SCALE_A / (SCALE_X * SCALE_X);
        __syncthreads();
        put_tiles(half_tiles, triangle, first, s32, first, s32);
        Tile A[SMALL_TILES];
#pragma unroll
        for (int i = 0; i < SMALL_TILES; ++i) A[i] = x[i];
        __syncthreads();
        multiply(first, first, s32, half_tiles, triangle);
        const float ka = jobs.a * SCALE_P, kb = jobs.b * (SCALE_P / SCALE_A), kc = jobs.c * (SCALE_P / (SCALE_A * SCALE_A));
#pragma unroll
        for (int i = 0; i < SMALL_TILES; ++i) {
            int ti, tj;
            triangle(i * SMALL_WAVES + wave, ti, tj);
#pragma unroll
            for (int g = 0; g < 4; ++g)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float y = fmaf(kc, x[i].q[g][e], kb * A[i].q[g][e]);
                    x[i].q[g][e] = ti == tj && row_of(g, lane) + e == col_of(g, lane) ? y + ka : y;
                }
        }
        __syncthreads();
        put_tiles(half_tiles, triangle, first, s32, first, s32);
        __syncthreads();
        multiply(first, second, s32, tiles, whole);
        if (step + 1 == jobs.steps) break;
#pragma unroll
        for (int i = 0; i < SMALL_TILES; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) x[i].q[g] *= 1.f / SCALE_P;
        __syncthreads();
        put_tiles(tiles, whole, first, l32, second, s32);
        __syncthreads();
    }
    using TOut = T;
    TOut* out = (TOut*)j.out + at;
#pragma unroll
    for (int i = 0; i < SMALL_TILES; ++i) {
        const int t = i * SMALL_WAVES + wave;
        if (t >= tiles) continue;
        int ti, tj;
        whole(t, ti, tj);
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int a = ti * 32 + row_of(g, lane) + e, b = tj * 32 + col_of(g, lane), row = tall ? b : a, col = tall ? a : b;
                if (row >= j.rows || col >= j.cols) continue;
                const float o = x[i].q[g][e] * (1.f / (SCALE_P * SCALE_X));
                TOut& to = out[(int64_t)row * j.cols + col];
                if constexpr (UPDATE) to = fmaf(-j.step, o, to) - jobs.decay * to;
                else if constexpr (sizeof(T) == 2) to = __builtin_bit_cast(uint16_t, (__bf16)o);
                else to = o;
            }
    }
}

// ---- thin matrices: at most 64 rows -----------------------------------------------------------------------------------
//
// A and P are 64 x 64: every workgroup makes them for itself, from the sums that the launch before left, and keeps a slab of 256 columns of
// X in hand from the product with P to its own share of the next A.  So a step is one launch where it would be three.  Bound by the
// latency of that chain: a launch, the sum of the shares, four dependent products.  One fp32 matrix of 59 x 3200 takes 72 us (three
// launches a step: 111), of 64 x 16384 117 (325).  The shares of A are added in the order of the slabs.
constexpr int THIN_S = 64, THIN_SLAB = 256, THIN_MOST = 16384;
constexpr int THIN_SHARE = 3 * 4 * 64;       // float4 of a share of A: three tiles (the triangle), four quarters, lanes

struct ThinJob {
    void* M;
    const float* S;
    void* out;
    _Float16* X;                             // by columns
    float4_t* share[2];                      // of A, by slabs: taken in, left
    const double* partial;                   // sums of squares
    int64_t stride;                          // bytes between copies in the workspace
    int rows, cols, copies, slabs, units, parts;      // units: of 32 columns, all slabs
    float step;
    unsigned first;
};
constexpr int THIN_JOBS = 24;
struct ThinJobs {
    int count;
    Momentum momentum;
    float a, b, c, eps, decay;
    ThinJob job[THIN_JOBS];
};

// entry (row, col) of an operand of cols32 times 32 columns
__device__ __forceinline__ _Float16* entry_at(_Float16* to, int row, int col, int cols32)
{
    return to + fragment_at(row >> 5, col >> 5, cols32, row >> 4 & 1, 0) + ((row & 15) + 16 * (col >> 3 & 3)) * 8 + (col & 7);
}
__device__ __forceinline__ void put_entry(_Float16* to, int row, int col, int cols32, float v)
{
    _Float16 hi, lo, *p = entry_at(to, row, col, cols32);
    split(v, hi, lo);
    p[0] = hi;
    p[FRAG] = lo;
}

// FIRST: X_0 and its share of A.  Else a step; LAST: the result instead of X and A.
template <typename T, bool UPDATE, bool FIRST, bool LAST>
__global__ __launch_bounds__(512) void ns_thin_kernel(ThinJobs jobs)
{
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    _Float16 *A = (_Float16*)lds, *P = A + THIN_S * THIN_S * 2, *rows_of_x = P + THIN_S * THIN_S * 2;
    int k = 0;
    while (k + 1 < jobs.count && blockIdx.x >= jobs.job[k + 1].first) ++k;
    const ThinJob& j = jobs.job[k];
    const int local = (int)(blockIdx.x - j.first), copy = local / j.slabs, slab = local - copy * j.slabs;
    const int64_t at = (int64_t)copy * j.stride, matrix = (int64_t)copy * j.rows * j.cols;
    const int units = min(THIN_SLAB / 32, j.units - slab * (THIN_SLAB / 32));       // of 32 columns of this slab
    const bool tall = j.rows > j.cols;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    _Float16* X = (_Float16*)((char*)j.X + at) + (int64_t)slab * (THIN_SLAB / 32) * (THIN_S / 32) * 4 * FRAG;      // this slab's columns
    auto tile_of = [](int t, int& ti, int& tj) { ti = t == 2; tj = t > 0; };                                       // (0, 0), (0, 1), (1, 1)
    auto both = [&](_Float16* to, int t, int g, const float4_t& v) {                                              // a quarter of a symmetric tile
        int ti, tj;
        tile_of(t, ti, tj);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = ti * 32 + row_of(g, lane) + e, c = tj * 32 + col_of(g, lane);
            put_entry(to, r, c, THIN_S / 32, v[e]);
            if (ti != tj) put_entry(to, c, r, THIN_S / 32, v[e]);
        }
    };

    if constexpr (FIRST) {
        const double* partial = (const double*)((const char*)j.partial + at);
        double ssq = 0.0;
        for (int p = threadIdx.x; p < j.parts; p += 512) ssq += partial[p];
        ssq = block_sum<8>(ssq);
        const double inv = to_unit(ssq, jobs.eps);
        const T* M = (const T*)j.M + matrix;
        const int s = tall ? j.cols : j.rows, l = tall ? j.rows : j.cols;
#pragma unroll 8
        for (int i = 0; i < THIN_S * THIN_SLAB / 512; ++i) {        // along the rows of M
            const int q = i * 512 + (int)threadIdx.x, r = tall ? q % THIN_S : q / THIN_SLAB, c = tall ? q / THIN_S : q % THIN_SLAB, col = slab * THIN_SLAB + c;
            float u = 0.f;
            if (r < s && col < l) {
                const int64_t e = tall ? (int64_t)col * j.cols + r : (int64_t)r * j.cols + col;
                u = value_at(M, e);
                if constexpr (UPDATE) u = jobs.momentum.ahead(u, j.S[e]);
            }
            put_entry(rows_of_x, r, c, THIN_SLAB / 32, (float)((double)u * inv));
        }
        __syncthreads();
        // the copy by columns, a fragment (16 columns of X, 32 rows) and its second piece at a time
        for (int f = wave; f < units * 4; f += 8) {
            const int j32 = f >> 2, r16 = f >> 1 & 1, i32 = f & 1;
            half8_t hi, lo;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const _Float16* p = entry_at(rows_of_x, i32 * 32 + (lane >> 4) * 8 + e, j32 * 32 + r16 * 16 + (lane & 15), THIN_SLAB / 32);
                hi[e] = p[0];
                lo[e] = p[FRAG];
            }
            *((half8_t*)(X + fragment_at(j32, i32, THIN_S / 32, r16, 0)) + lane) = hi;
            *((half8_t*)(X + fragment_at(j32, i32, THIN_S / 32, r16, 1)) + lane) = lo;
        }
    } else {
        // the wave's 32 columns of X: on their way while A and P are made
        half8_t v[THIN_S / 32][4];
        if (wave < units) {
#pragma unroll
            for (int s = 0; s < THIN_S / 32; ++s)
#pragma unroll
                for (int x = 0; x < 4; ++x) v[s][x] = ((const half8_t*)X)[((wave * (THIN_S / 32) + s) * 4 + x) * 64 + lane];
        }
        const float4_t* share = (const float4_t*)((const char*)j.share[0] + at);
        for (int q = wave; q < 12; q += 8) {
            float4_t sum = {0.f, 0.f, 0.f, 0.f};
            int s = 0;
            for (; s + 4 <= j.slabs; s += 4) {
                float4_t y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] = share[(int64_t)(s + i) * THIN_SHARE + q * 64 + lane];
#pragma unroll
                for (int i = 0; i < 4; ++i) sum += y[i];
            }
            for (; s < j.slabs; ++s) sum += share[(int64_t)s * THIN_SHARE + q * 64 + lane];
            both(A, q >> 2, q & 3, sum * (SCALE_A / (SCALE_X * SCALE_X)));
        }
        __syncthreads();
        if (wave < 3) {
            int ti, tj;
            tile_of(wave, ti, tj);
            Tile x;
            clear(x);
#pragma unroll
            for (int s = 0; s < THIN_S / 32; ++s) {
                half8_t fu[4], fv[4];
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    fu[f] = ((const half8_t*)A)[((ti * (THIN_S / 32) + s) * 4 + f) * 64 + lane];
                    fv[f] = ((const half8_t*)A)[((tj * (THIN_S / 32) + s) * 4 + f) * 64 + lane];
                }
                Tile d;
                products(fu, fv, d);
                add(x, d);
            }
            const float ka = jobs.a * SCALE_P, kb = jobs.b * (SCALE_P / SCALE_A), kc = jobs.c * (SCALE_P / (SCALE_A * SCALE_A));
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const half4_t hi = *place((char*)A, THIN_S / 32, ti, tj, g, 0, lane), lo = *place((char*)A, THIN_S / 32, ti, tj, g, 1, lane);
                float4_t y;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    y[e] = fmaf(kc, x.q[g][e], kb * ((float)hi[e] + (float)lo[e]));
                    if (ti == tj && row_of(g, lane) + e == col_of(g, lane)) y[e] += ka;
                }
                both(P, wave, g, y);
            }
        }
        __syncthreads();
        if (wave < units) {
#pragma unroll
            for (int i32 = 0; i32 < THIN_S / 32; ++i32) {
                Tile x;
                clear(x);
#pragma unroll
                for (int s = 0; s < THIN_S / 32; ++s) {
                    half8_t fu[4];
#pragma unroll
                    for (int f = 0; f < 4; ++f) fu[f] = ((const half8_t*)P)[((i32 * (THIN_S / 32) + s) * 4 + f) * 64 + lane];
                    Tile d;
                    products(fu, v[s], d);
                    add(x, d);
                }
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    if constexpr (LAST) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int a = i32 * 32 + row_of(g, lane) + e, b = slab * THIN_SLAB + wave * 32 + col_of(g, lane), row = tall ? b : a, col = tall ? a : b;
                            if (row >= j.rows || col >= j.cols) continue;
                            const float o = x.q[g][e] * (1.f / (SCALE_P * SCALE_X));
                            T& to = ((T*)j.out)[matrix + (int64_t)row * j.cols + col];
                            if constexpr (UPDATE) to = fmaf(-j.step, o, to) - jobs.decay * to;
                            else if constexpr (sizeof(T) == 2) to = __builtin_bit_cast(uint16_t, (__bf16)o);
                            else to = o;
                        }
                    } else {
                        half4_t hi, lo;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            _Float16 a, b, *p = entry_at(rows_of_x, i32 * 32 + row_of(g, lane) + e, wave * 32 + col_of(g, lane), THIN_SLAB / 32);
                            split(x.q[g][e] * (1.f / SCALE_P), a, b);
                            hi[e] = p[0] = a;
                            lo[e] = p[FRAG] = b;
                        }
                        // over what this wave, and nobody else, has read
                        *place((char*)X, THIN_S / 32, i32, wave, g, 0, lane) = hi;
                        *place((char*)X, THIN_S / 32, i32, wave, g, 1, lane) = lo;
                    }
                }
            }
        }
    }
    if constexpr (!LAST) {
        if constexpr (!FIRST) __syncthreads();
        if (wave < 3) {          // this slab's share of the next A
            int ti, tj;
            tile_of(wave, ti, tj);
            Tile x;
            clear(x);
            for (int s = 0; s < units; ++s) {
                half8_t fu[4], fv[4];
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    fu[f] = ((const half8_t*)rows_of_x)[((ti * (THIN_SLAB / 32) + s) * 4 + f) * 64 + lane];
                    fv[f] = ((const half8_t*)rows_of_x)[((tj * (THIN_SLAB / 32) + s) * 4 + f) * 64 + lane];
                }
                Tile d;
                products(fu, fv, d);
                add(x, d);
            }
            float4_t* share = (float4_t*)((char*)j.share[FIRST ? 0 : 1] + at) + (int64_t)slab * THIN_SHARE + wave * 256 + lane;
#pragma unroll
            for (int g = 0; g < 4; ++g) share[g * 64] = x.q[g];
        }
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------

int64_t padded(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
// A side as the kernels see it: whole blocks of the largest kind that costs little padding.  Products go by the cube of it.  Whole calls (us),
// 256 for up to an eighth more / a thirty-second: fp32 1100 x 1100 343 / 259, 3136 x 2488 1500 / 1248, 3400 x 3400 2718 / 2368, 2700 x 2700
// 1294 / 1308; 128 always / for up to a ninth more than 64: 10 of 1056 x 576 450 / 403, 16 of 192 x 768 156 / 134.
int64_t padded_side(int64_t n)
{
    if (n <= 64 || padded(n, 64) * 10 <= padded(n, 128) * 9) return padded(n, 64);
    return padded(n, 256) * 32 <= padded(n, 128) * 33 ? padded(n, 256) : padded(n, 128);
}

constexpr int64_t MOST_PARTS = 1024;
constexpr int GROUP = NS_GROUP;       // matrices of a launch
static_assert(GROUP <= JOBS && GROUP <= THIN_JOBS);

// Where the buffers of one matrix lie, from the start of its part of the workspace: X by rows, twice by columns; symmetric ones
enum : int { BUF_ROWS, BUF_COLS0, BUF_COLS1, BUF_A, BUF_P0, BUF_P1, BUF_R, BUF_COUNT };
struct Layout {
    int64_t s, l;             // padded sides
    int parts;
    int64_t at[BUF_COUNT], partial_at, arrived_at, blocks, bytes;      // blocks: of 128 x 128 of a symmetric product
};
// Whether two steps at a time go through the Gram matrix (see program_of): where products bound the time and there are fewer of them so
bool by_gram(int64_t s, int64_t l) { return s >= 512 && 2 * l >= 3 * s; }

Layout layout_of(int64_t rows, int64_t cols)
{
    Layout w{};
    w.s = padded_side(rows < cols ? rows : cols);
    w.l = padded_side(rows < cols ? cols : rows);
    const int64_t parts = (rows * cols + 2047) / 2048;
    w.parts = (int)(parts < MOST_PARTS ? parts : MOST_PARTS);
    int64_t at = 0;
    auto take = [&](int64_t bytes) { const int64_t here = at; at += padded(bytes, 256); return here; };
    for (int k = 0; k < (by_gram(w.s, w.l) ? BUF_COUNT : BUF_P1); ++k)      // step by step: A and one P
        w.at[k] = take((k <= BUF_COLS1 ? w.s * w.l : w.s * w.s) * 4);
    w.partial_at = take((int64_t)w.parts * 8);
    w.blocks = w.s / 128 * (w.s / 128 + 1) / 2;
    w.arrived_at = take(w.blocks * 4);
    w.bytes = at;
    return w;
}

// The products of one matrix in their order
struct Op {
    int u, v, out, out_cols;
    int idle;                 // a buffer of X that nobody needs meanwhile
    bool with_x;              // C = u X, not symmetric
    float factor, alpha, beta, gamma;
};
struct Program {
    int count;
    Op op[NS_ROUNDS];
};
// Step by step: A = X X^T, P = a I + b A + c A^2, X = P X.  Or two steps at a time: with W = b A + c A^2, P = a I + W, the A of P X is P A P,
// all of them polynomials of one matrix, which commute and whose products are symmetric:
//   R = a A + W A, A' = a R + W R, W' = b A' + c A'^2, Q = a^2 I + a (W + W') + W W', X = Q X.
// With l = 4 s five steps as 2 + 2 + 1 are 47 s^3 products of two matrices instead of 65, three more launches.  Half of a product is taken for
// the whole: the identity's share stays outside of it, where rounding would move the small eigenvalues of A by 2^-23 of the largest,
// which a step lets grow by a^2 = 12.  Off by 1.1e-6 of the 2-norm (64 bits; 250 x 1002), step by step 4e-7, 3 + 2 steps 2.6e-6.
void program_of(const Layout& w, const NsCall& call, Program& p)
{
    p.count = 0;
    const float a = call.a, b = call.b, c = call.c;
    int now = BUF_COLS0;
    auto add = [&](int u, int v, int out, int out_cols, bool with_x, float factor, float alpha, float beta, float gamma) {
        p.op[p.count++] = {u, v, out, out_cols, now == BUF_COLS0 ? BUF_COLS1 : BUF_COLS0, with_x, factor, alpha, beta, gamma};
    };
    auto polynomial = [&](int to, bool whole) {
        add(BUF_A, BUF_A, to, to, false, c * (SCALE_P / (SCALE_A * SCALE_A)), b * (SCALE_P / SCALE_A), 0.f, whole ? a * SCALE_P : 0.f);
    };
    constexpr float unscale = 1.f / SCALE_P;
    for (int done = 0; done < call.steps;) {
        const int n = by_gram(w.s, w.l) && call.steps - done >= 2 ? 2 : 1;
        add(BUF_ROWS, BUF_ROWS, BUF_A, BUF_A, false, SCALE_A / (SCALE_X * SCALE_X), 0.f, 0.f, 0.f);
        polynomial(BUF_P0, n == 1);
        int q = BUF_P0;
        if (n == 2) {
            add(BUF_P0, BUF_A, BUF_R, BUF_R, false, unscale, a, 0.f, 0.f);
            add(BUF_P0, BUF_R, BUF_A, BUF_A, false, unscale, a, 0.f, 0.f);
            polynomial(BUF_P1, false);
            add(BUF_P1, BUF_P0, BUF_R, BUF_R, false, unscale, a, a, a * a * SCALE_P);
            q = BUF_R;
        }
        done += n;
        const int next = now == BUF_COLS0 ? BUF_COLS1 : BUF_COLS0;
        add(q, now, BUF_ROWS, next, true, done == call.steps ? 1.f / (SCALE_P * SCALE_X) : unscale, 0.f, 0.f, 0.f);
        now = next;
    }
}

// Which kernel takes a product
enum : int { DIRECT_32 = NS_DIRECT_32, DIRECT_64, STAGED_128, STAGED_256, VARIANTS, DIVIDED_128 = VARIANTS };
static_assert(DIRECT_64 == NS_DIRECT_64 && STAGED_256 == NS_STAGED_256 && DIVIDED_128 == NS_DIVIDED_128);
constexpr int VARIANT_BLOCK[VARIANTS] = {1, 2, 4, 8};

// By the blocks that the products of a round have in each size, and the largest number of units along a product's columns.  Blocks of 256 are a
// tenth faster than those of 128 where they fill whole rounds of the 256 compute units; those of 128 need half of the chip, and columns
// that pay for filling four slots.  Whole calls (us) with fewer of them straight from the caches / through LDS: 2304 x 2304 (171 blocks)
// 1027 / 905; but 9 of 640 x 640 (135, 20 units) 276 / 306.
bool enough_256(int64_t blocks) { return blocks * 100 >= (blocks + 255) / 256 * 256 * 88; }
bool enough_128(int64_t blocks, int units) { return blocks >= (units < 32 ? 200 : 128); }
// Straight from the caches 64 reads half of what 32 does, and takes as long for a block as there are columns for its four waves.  Measured,
// 64 / 32 (us): 136 blocks of 1024 x 1024 x 2304 19.1 / 20.8, of 1024 x 1024 x 1024 12.3 / 10.2; 312 of 4 x 768 x 768 x 2304 33 / 37,
// x 768 15.8 / 12.8; 576 of 1024 x 2304 x 1024 27 / 31.
int direct_for(int64_t blocks_64, int units) { return blocks_64 >= 512 || (blocks_64 >= 128 && units >= 48) ? DIRECT_64 : DIRECT_32; }

template <typename TOut, bool UPDATE>
hipError_t launch_round(const Jobs& jobs, unsigned blocks, int variant, hipStream_t stream)
{
    auto staged = [&](auto kern, int slot) {
        const hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, 2 * slot);
        if (e != hipSuccess) return e;
        kern<<<dim3(blocks), dim3(512), 2 * slot, stream>>>(jobs);
        return hipGetLastError();
    };
    if (variant == STAGED_256) return staged(ns_staged_kernel<256, TOut, UPDATE, false>, slot_bytes<256>());
    if (variant == STAGED_128 && blocks <= 256) return staged(ns_staged_kernel<128, TOut, UPDATE, false, 4>, 2 * slot_bytes<128>());
    if (variant == STAGED_128) return staged(ns_staged_kernel<128, TOut, UPDATE, false>, slot_bytes<128>());
    if (variant == DIVIDED_128) return staged(ns_staged_kernel<128, TOut, UPDATE, true>, slot_bytes<128>());
    if (variant == DIRECT_64) ns_direct_kernel<2, TOut, UPDATE><<<dim3(blocks), dim3(256), 0, stream>>>(jobs);
    else ns_direct_kernel<1, TOut, UPDATE><<<dim3(blocks), dim3(256), 0, stream>>>(jobs);
    return hipGetLastError();
}

// A product of a program as a job, without its buffers; blocks of each kernel for one copy (0: it does not take this shape)
void shape_of(const NsMatrix& m, const Layout& w, const Op& op, bool last, Job& j, int64_t (&blocks)[VARIANTS])
{
    j.symmetric = !op.with_x;
    j.m32 = (int)(w.s / 32);
    j.n32 = (int)((op.with_x ? w.l : w.s) / 32);
    j.units = (int)((op.u == BUF_ROWS ? w.l : w.s) / 32);
    if (last && m.rows > m.cols) {           // the result's rows are the columns of X
        j.m32 = (int)(w.l / 32);
        j.n32 = (int)(w.s / 32);
    }
    for (int v = 0; v < VARIANTS; ++v) {
        const int edge = VARIANT_BLOCK[v];
        const int64_t tm = j.m32 / edge, tn = j.n32 / edge;
        blocks[v] = j.m32 % edge || j.n32 % edge ? 0 : j.symmetric ? tm * (tm + 1) / 2 : tm * tn;
    }
}

constexpr int64_t PART_BYTES = 128 * 128 * 4;
// How many of a symmetric round's blocks of 128 are divided along their columns, and into how many parts: those that leave the 256 compute
// units, or their two places for workgroups, unequally full.  More parts cost more for the sums (who joins a block reads all of it: 64 KiB a
// part).  Measured, whole calls (us), undivided and divided:
//   of 128 .. 148 blocks all, in 3: 2048 x 4096 (136) 1063 / 936; 2176 x 3840 (153)
//   1251 / 1254, 2560 x 4096 (210, in 2) 1459 / 1484; 1792 x 5376 (105, in 4) 982 / 994;
//   of 256 .. 384 those past 256, in 2: two of 2048 x 8192 (272) 2607 / 2485, in 3 2508; 3000 x 6500 (300) 2952 / 2776; 8 of
//   1024 x 4096 (288) 1543 / 1496;
//   past 512 those past the last whole 512: 4096 x 6400 (528) 5927 / 5033 in 4, 5129 in 3; 4864 x 7680 (741) 8518 / 8027 in 2.
struct Divided {
    int blocks, parts;
};
Divided divided_for(int64_t blocks, int units)
{
    const int64_t over = blocks % 512, rest = over < 256 ? over : over - 256;
    if (blocks < 128 || (blocks > 148 && blocks < 256) || rest == 0 || units < 32) return {0, 1};
    const int64_t room = (over < 256 ? 512 : 256) / rest, most = blocks < 256 ? 3 : over < 256 ? 4 : 2;
    return {(int)rest, (int)(room < most ? room : most)};
}

// of a copy's blocks that are divided: chunks (some on every XCD, the divided ones last), divided ones of a chunk
void of_copy(const NsPlan::Round& round, int64_t mine, int& chunks, int& rest)
{
    chunks = round.copies >= 8 || round.divided == round.blocks ? 1 : 8 / round.copies;
    if (chunks > mine) chunks = (int)mine;
    rest = (int)((round.divided * mine + round.blocks * chunks - 1) / (round.blocks * chunks));
    if (rest > mine / chunks) rest = (int)(mine / chunks);
}

// The kernels of all rounds of `count` matrices that go together, as if there were workspace for all of them (their results do not depend on
// it).  Sides that are no multiple of 256, or 128, stand in the way of nobody but their own product: of a round, the products that blocks
// of 256 take go there if these are enough, of the others those that blocks of 128 take, the rest straight from the caches, a launch
// each.  Whole calls (us), all of a round on what every one of them takes / divided: 2048 x 8192 and 8192 x 2048 beside 2048 x 320 3860 /
// 2676, beside 640 x 640 2987 / 2741; 2304 x 2304 beside 2304 x 320 1283 / 1008; five GPT-2 blocks beside 768 x 320 1882 / 1733.  Blocks of 128
// pay for another launch from 6144 units of columns on, of all of them: 8 of 1024 x 1024 (288 blocks of 32) beside 1024 x 320 834 / 766,
// but 12 of 768 x 768 (252 of 24) beside 768 x 320 586 / 589, 4 of 1024 x 1024 (144 of 32) beside 1024 x 320 500 / 523.
void plan_rounds(const NsMatrix* mats, int count, const NsCall& call, NsPlan& plan)
{
    Program p[2];                 // step by step, two steps at a time
    int known[2] = {-1, -1}, which[GROUP];
    Layout w[GROUP];
    for (int i = 0; i < count; ++i) {
        w[i] = layout_of(mats[i].rows, mats[i].cols);
        which[i] = by_gram(w[i].s, w[i].l);
        if (known[which[i]] < 0) program_of(w[i], call, p[which[i]]);
        known[which[i]] = 1;
        if (p[which[i]].count > plan.rounds) plan.rounds = p[which[i]].count;
    }
    for (int r = 0; r < plan.rounds; ++r) {
        NsPlan::Round& round = plan.round[r];
        round = {};
        int64_t of[GROUP][VARIANTS];
        Job j[GROUP];
        bool open[GROUP];         // no kernel yet
        for (int i = 0; i < count; ++i) {
            const Program& mine = p[which[i]];
            const int k = r - (plan.rounds - mine.count);       // a shorter program ends with the longest
            round.kernel[i] = NS_NONE;
            open[i] = k >= 0;
            if (open[i]) shape_of(mats[i], w[i], mine.op[k], k + 1 == mine.count, j[i], of[i]);
        }
        int64_t blocks, copies, work;
        int units;
        bool all;                 // nobody is left
        auto totals = [&](int variant) {
            blocks = copies = work = units = 0;
            all = true;
            for (int i = 0; i < count; ++i) {
                if (!open[i]) continue;
                if (of[i][variant] == 0) {
                    all = false;
                    continue;
                }
                blocks += of[i][variant] * mats[i].copies;
                copies += mats[i].copies;
                work += of[i][variant] * mats[i].copies * j[i].units;
                if (j[i].units > units) units = j[i].units;
            }
        };
        auto take = [&](int variant, int as) {
            for (int i = 0; i < count; ++i)
                if (open[i] && of[i][variant] > 0) {
                    round.kernel[i] = (int8_t)as;
                    open[i] = false;
                }
        };
        totals(STAGED_256);
        if (blocks > 0 && enough_256(blocks)) take(STAGED_256, STAGED_256);
        totals(STAGED_128);
        if (enough_128(blocks, units) && (all || work >= 6144)) {
            const Divided d = divided_for(blocks, units);
            round.blocks = blocks;
            round.divided = d.blocks;
            round.parts = d.parts;
            round.copies = copies < 8 ? (int)copies : 8;
            bool divided = d.parts > 1;
            for (int i = 0; i < count && divided; ++i)
                if (open[i] && of[i][STAGED_128] > 0) {
                    int chunks, rest;
                    of_copy(round, of[i][STAGED_128], chunks, rest);
                    divided = j[i].symmetric && (int64_t)chunks * rest * d.parts * PART_BYTES <= w[i].s * w[i].l * 4;
                }
            take(STAGED_128, divided ? DIVIDED_128 : STAGED_128);
        }
        totals(DIRECT_64);        // (every side is a multiple of 64)
        take(DIRECT_64, direct_for(blocks, units));
    }
}

// `planned`: the places of the matrices in the plan
template <typename T, bool UPDATE>
hipError_t run_group(const NsMatrix* mats, const int* planned, int count, const NsCall& call, const NsPlan& plan, char* ws, hipStream_t stream)
{
    Layout w[GROUP];
    char* base[GROUP];
    Sources src{};
    src.count = count;
    src.momentum = {call.beta, call.gain, call.nesterov};
    src.eps = call.eps;
    unsigned sums = 0, tiles = 0;
    for (int i = 0; i < count; ++i) {
        const NsMatrix& m = mats[i];
        w[i] = layout_of(m.rows, m.cols);
        base[i] = ws;
        ws += w[i].bytes * m.copies;
        Source& s = src.m[i];
        s = {m.in, m.S, (_Float16*)(base[i] + w[i].at[BUF_ROWS]), (_Float16*)(base[i] + w[i].at[BUF_COLS0]), (double*)(base[i] + w[i].partial_at), w[i].bytes,
             m.rows * m.cols * (int64_t)sizeof(T), (int)m.rows, (int)m.cols, (int)(w[i].s / 64), (int)(w[i].l / 64), w[i].parts, (int)m.copies, sums, tiles,
             (unsigned*)(base[i] + w[i].arrived_at), (int)w[i].blocks};
        sums += (unsigned)(w[i].parts * m.copies);
        tiles += (unsigned)(s.s_tiles * (int64_t)s.l_tiles * m.copies);
    }
    ns_norm_kernel<T, UPDATE><<<dim3(sums), dim3(256), 0, stream>>>(src);
    ns_prepare_kernel<T, UPDATE><<<dim3(tiles), dim3(256), 0, stream>>>(src);
    hipError_t e = hipGetLastError();
    Program p[2];                 // step by step, two steps at a time
    int known[2] = {-1, -1};
    for (int r = 0; r < plan.rounds * (DIVIDED_128 + 1) && e == hipSuccess; ++r) {
        const int variant = r % (DIVIDED_128 + 1);
        const NsPlan::Round& round = plan.round[r / (DIVIDED_128 + 1)];
        bool any = false;
        for (int i = 0; i < count; ++i) any = any || round.kernel[planned[i]] == variant;
        if (!any) continue;
        Jobs jobs{};
        jobs.decay = call.decay;
        unsigned first = 0;
        for (int i = 0; i < count; ++i) {
            if (round.kernel[planned[i]] != variant) continue;
            const int which = by_gram(w[i].s, w[i].l);
            if (known[which] < 0) {
                program_of(w[i], call, p[which]);
                known[which] = 1;
            }
            const int k = r / (DIVIDED_128 + 1) - (plan.rounds - p[which].count);
            const Op& op = p[which].op[k];
            const NsMatrix& m = mats[i];
            const bool last = k + 1 == p[which].count;
            Job& j = jobs.job[jobs.count++];
            int64_t blocks[VARIANTS];
            shape_of(m, w[i], op, last, j, blocks);
            auto at = [&](int buffer) { return (_Float16*)(base[i] + w[i].at[buffer]); };
            j.copies = (int)m.copies;
            j.stride = w[i].bytes;
            j.factor = op.factor;
            j.alpha = op.alpha;
            j.beta = op.beta;
            j.gamma = op.gamma;
            const bool swapped = last && m.rows > m.cols;
            j.U = at(swapped ? op.v : op.u);
            j.V = at(swapped ? op.u : op.v);
            j.by_rows = at(op.out);
            j.by_cols = at(op.out_cols);
            if (last) {
                j.out = m.out;
                j.out_stride = m.rows * m.cols * (int64_t)sizeof(T);
                j.rows = (int)m.rows;
                j.cols = (int)m.cols;
                j.step = m.step;
            }
            j.first = first;
            if (variant == DIVIDED_128) {
                of_copy(round, blocks[STAGED_128], j.chunks, j.rest);
                j.share = (j.units + round.parts - 1) / round.parts;
                j.parts = (j.units + j.share - 1) / j.share;
                j.shares = (float4_t*)at(op.idle);
                j.arrived = (unsigned*)(base[i] + w[i].arrived_at);
                first += (unsigned)((blocks[STAGED_128] + (int64_t)j.chunks * j.rest * (j.parts - 1)) * m.copies);
            } else first += (unsigned)(blocks[variant] * m.copies);
        }
        e = launch_round<T, UPDATE>(jobs, first, variant, stream);
    }
    return e;
}

// The slabs of a matrix and its copies, 0 if it is not thin
int64_t thin_slabs(const NsMatrix& m)
{
    const int64_t s = m.rows < m.cols ? m.rows : m.cols, l = m.rows < m.cols ? m.cols : m.rows;
    return s <= THIN_S && l <= THIN_MOST ? (padded_side(l) + THIN_SLAB - 1) / THIN_SLAB * m.copies : 0;
}
// Once the chip is full, A and P made by every workgroup cost more than launches save (against three launches a step: 64 bf16 copies of
// 64 x 2048, 512 slabs: 190 and 200 us; 256 fp32 copies of it: 740 and 676; 512 of 64 x 4096: 3505 and 2680)
constexpr int64_t THIN_MOST_SLABS = 512;

template <typename T, bool UPDATE>
hipError_t run_thin(const NsMatrix* mats, int count, const NsCall& call, char* ws, hipStream_t stream)
{
    Sources src{};
    src.count = count;
    src.momentum = {call.beta, call.gain, call.nesterov};
    src.eps = call.eps;
    ThinJobs jobs{};
    jobs.count = count;
    jobs.momentum = src.momentum;
    jobs.a = call.a;
    jobs.b = call.b;
    jobs.c = call.c;
    jobs.eps = call.eps;
    jobs.decay = call.decay;
    unsigned sums = 0, blocks = 0;
    for (int i = 0; i < count; ++i) {
        const NsMatrix& m = mats[i];
        const Layout w = layout_of(m.rows, m.cols);
        const int64_t size = m.rows * m.cols * (int64_t)sizeof(T);
        src.m[i] = {m.in, m.S, nullptr, nullptr, (double*)(ws + w.partial_at), w.bytes, size, (int)m.rows, (int)m.cols, 0, 0, w.parts, (int)m.copies, sums, 0, nullptr, 0};
        sums += (unsigned)(w.parts * m.copies);
        // the shares of A, 12 KiB a slab and twice, where X by rows would be: 64 KiB for as many columns
        const int units = (int)(w.l / 32), slabs = (units + THIN_SLAB / 32 - 1) / (THIN_SLAB / 32);
        float4_t* shares = (float4_t*)(ws + w.at[BUF_ROWS]);
        jobs.job[i] = {m.in, m.S, m.out, (_Float16*)(ws + w.at[BUF_COLS0]), {shares, shares + (int64_t)slabs * THIN_SHARE}, (const double*)(ws + w.partial_at), w.bytes,
                       (int)m.rows, (int)m.cols, (int)m.copies, slabs, units, w.parts, m.step, blocks};
        blocks += (unsigned)(slabs * m.copies);
        ws += w.bytes * m.copies;
    }
    ns_norm_kernel<T, UPDATE><<<dim3(sums), dim3(256), 0, stream>>>(src);
    constexpr int bytes = (2 * THIN_S * THIN_S + THIN_S * THIN_SLAB) * 4;
    auto go = [&](auto kern) {
        const hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
        kern<<<dim3(blocks), dim3(512), bytes, stream>>>(jobs);
        return hipGetLastError();
    };
    hipError_t e = go(ns_thin_kernel<T, UPDATE, true, false>);
    for (int step = 1; step <= call.steps && e == hipSuccess; ++step) {
        e = step == call.steps ? go(ns_thin_kernel<T, UPDATE, false, true>) : go(ns_thin_kernel<T, UPDATE, false, false>);
        for (int i = 0; i < count; ++i) {
            float4_t* left = jobs.job[i].share[1];
            jobs.job[i].share[1] = jobs.job[i].share[0];
            jobs.job[i].share[0] = left;
        }
    }
    return e;
}

bool is_small(int64_t rows, int64_t cols) { return padded(rows, 64) * padded(cols, 64) <= SMALL_MOST; }

template <typename T, bool UPDATE>
hipError_t run_small(const NsMatrix* mats, int64_t count, const NsCall& call, hipStream_t stream)
{
    auto kern = ns_small_kernel<T, UPDATE>;
    constexpr int bytes = 2 * SMALL_MOST * 4;
    SmallJobs jobs{};
    unsigned blocks = 0;
    auto flush = [&]() {
        if (jobs.count == 0) return hipSuccess;
        const hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
        kern<<<dim3(blocks), dim3(SMALL_WAVES * 64), bytes, stream>>>(jobs);
        jobs.count = 0;
        blocks = 0;
        return hipGetLastError();
    };
    jobs.steps = call.steps;
    jobs.momentum = {call.beta, call.gain, call.nesterov};
    jobs.a = call.a;
    jobs.b = call.b;
    jobs.c = call.c;
    jobs.eps = call.eps;
    jobs.decay = call.decay;
    for (int64_t i = 0; i < count; ++i) {
        const NsMatrix& m = mats[i];
        if (!is_small(m.rows, m.cols)) continue;
        for (int64_t done = 0; done < m.copies;) {
            const int64_t n = m.copies - done < (1 << 20) ? m.copies - done : 1 << 20, skip = done * m.rows * m.cols;
            if (jobs.count == SMALL_JOBS || blocks + (uint64_t)n > (1u << 22)) {        // (of 512: a launch holds fewer than 2^32 threads)
                const hipError_t e = flush();
                if (e != hipSuccess) return e;
            }
            jobs.job[jobs.count++] = {(T*)m.in + skip, m.S, (T*)m.out + skip, (int)m.rows, (int)m.cols, (int)n, m.step, blocks};
            blocks += (unsigned)n;
            done += n;
        }
    }
    return flush();
}

}  // namespace

// (small ones use none, but a query is never 0)
size_t ns_matrix_bytes(int64_t rows, int64_t cols) { return is_small(rows, cols) ? 256 : (size_t)layout_of(rows, cols).bytes; }
size_t ns_copies_bytes(int64_t count, int64_t rows, int64_t cols) { return is_small(rows, cols) ? 256 : (size_t)count * (size_t)layout_of(rows, cols).bytes; }

bool ns_coefficients_ok(const pex_newton_schulz_params& p)
{
    const double a = p.a, b = p.b, c = p.c;
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return false;
    double top = 1.0, largest = 0.0;       // largest singular value before the step; gain of all steps
    for (int k = 0; k < p.steps; ++k) {
        // g(s) = s (a + b s^2 + c s^4) on [0, top]: its ends and where g' = a + 3 b t + 5 c t^2 vanishes, t = s^2
        auto g = [&](double s) { return std::fabs(s * (a + b * s * s + c * s * s * s * s)); };
        double high = g(top);
        auto root = [&](double t) { if (t > 0.0 && t < top * top) high = std::fmax(high, g(std::sqrt(t))); };
        if (c != 0.0) {
            const double q = 9.0 * b * b - 20.0 * a * c;
            if (q >= 0.0) { root((-3.0 * b + std::sqrt(q)) / (10.0 * c)); root((-3.0 * b - std::sqrt(q)) / (10.0 * c)); }
        } else if (b != 0.0) root(-a / (3.0 * b));
        auto h = [&](double t) { return std::fabs(a + b * t + c * t * t); };
        const double turn = c != 0.0 ? -b / (2.0 * c) : 0.0;
        const double gain = std::fmax(std::fmax(h(0.0), h(top * top)), turn > 0.0 && turn < top * top ? h(turn) : 0.0);
        if (!(gain <= 31.0) || !(high <= 4.0)) return false;
        top = high;
        largest = std::fmax(largest, gain);
    }
    // The product of two P's stays in P's range.  (All that get here do: over a grid of coefficients of 0.1 with a gain of 7.75 and more, two steps
    // take [0, 1] out of [0, 4] by a factor of 4.5 at least.)
    return p.steps < 2 || largest * largest <= 60.0;
}

// (thin matrices among others share the others' launches: a launch of their own for each round that goes through LDS costs no more than theirs
// would, GPT-2's blocks or 2048 x 8192 and 8192 x 2048 beside one)
void plan_newton_schulz(const NsMatrix* mats, int count, const NsCall& call, NsPlan& plan)
{
    int64_t slabs = 0;
    plan.thin = true;
    for (int i = 0; i < count; ++i) {
        plan.thin = plan.thin && thin_slabs(mats[i]) > 0;
        slabs += thin_slabs(mats[i]);
    }
    plan.thin = plan.thin && slabs <= THIN_MOST_SLABS;
    plan.rounds = 0;
    if (!plan.thin) plan_rounds(mats, count, call, plan);
}

// Small matrices in a launch of their own; the others go together, GROUP of them at a time, while there is workspace for them, copies of
// one divided if need be
hipError_t launch_newton_schulz(const NsMatrix* mats, int64_t count, pex_dtype dt, bool update, const NsCall& call, void* workspace, size_t workspace_bytes,
                                hipStream_t stream)
{
    hipError_t e = update            ? run_small<float, true>(mats, count, call, stream)
                   : dt == PEX_F32   ? run_small<float, false>(mats, count, call, stream)
                                     : run_small<uint16_t, false>(mats, count, call, stream);
    for (int64_t begin = 0; begin < count && e == hipSuccess;) {
        NsMatrix together[GROUP], group[GROUP];
        int members = 0, n = 0;
        for (; begin < count && members < GROUP; ++begin)
            if (!is_small(mats[begin].rows, mats[begin].cols)) together[members++] = mats[begin];
        if (members == 0) break;
        NsPlan plan;
        plan_newton_schulz(together, members, call, plan);
        int planned[GROUP];
        size_t used = 0;
        auto flush = [&]() {
            if (n == 0 || e != hipSuccess) return;
            char* ws = (char*)workspace;
            if (plan.thin) e = update ? run_thin<float, true>(group, n, call, ws, stream)
                                 : dt == PEX_F32 ? run_thin<float, false>(group, n, call, ws, stream) : run_thin<uint16_t, false>(group, n, call, ws, stream);
            else if (update) e = run_group<float, true>(group, planned, n, call, plan, ws, stream);
            else if (dt == PEX_F32) e = run_group<float, false>(group, planned, n, call, plan, ws, stream);
            else e = run_group<uint16_t, false>(group, planned, n, call, plan, ws, stream);
            n = 0;
            used = 0;
        };
        for (int i = 0; i < members && e == hipSuccess; ++i) {
            NsMatrix m = together[i];
            const size_t each = ns_matrix_bytes(m.rows, m.cols);
            const int64_t elem = dt == PEX_F32 ? 4 : 2;
            while (m.copies > 0 && e == hipSuccess) {
                int64_t fit = (int64_t)((workspace_bytes - used) / each);
                if (fit > 4096) fit = 4096;
                if (fit < 1 || n == GROUP) {
                    flush();
                    continue;
                }
                NsMatrix part = m;
                if (part.copies > fit) part.copies = fit;
                planned[n] = i;
                group[n++] = part;
                used += each * (size_t)part.copies;
                m.copies -= part.copies;
                m.in = (char*)m.in + part.copies * m.rows * m.cols * elem;
                m.out = (char*)m.out + part.copies * m.rows * m.cols * elem;
            }
        }
        flush();
    }
    return e;
}

}  // namespace pex
