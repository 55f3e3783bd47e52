// Attention with a decay per head on the tensor cores: bf16 rows, chunks of 128, products with fp32 accumulation.
//
// One block takes a segment of one head's chunks in the pass's order; a chunk is four products of tcgen05.mma:
//   A = X Y^T                        scores; times the decays and rounded to bf16 they go back to tensor memory as P, the left operand of
//   O = lambda^(..) (X S) + P Z      the rows out: X S first, its rows scaled in place, P Z accumulated onto it (of narrow tiles apart)
//   D = (w Y)^T Z                    what the chunk adds to the state. The tokens' weights are applied to Y as it goes, transposed, from shared
//                                    memory into tensor memory, as two bf16 parts (16 bits), or three (24) where the caller gets the
//                                    state; with one, its rounding would show in the rows out.
// The state itself stays in the registers of eight warps in fp32, S <- lambda^L S + D; the rows read a copy rounded to bf16 (as P is
// rounded: half a step of each term, like the rounding of the rows out: together 1.4 times the error of that rounding alone).
// Everything moves by TMA, two to four chunks of X, Y and Z deep; the rows out are staged in the chunk's own tiles (stored from registers, 32 bytes a
// thread, d 128 took 7 % longer).
//
// What bounds it: shared memory. At width 128 a chunk's tiles, operands and copies are 3.8 thousand cycles of its 128 bytes a cycle (the products
// by themselves 2.6), a chunk takes 4.5 thousand; at 64 2.3 of 3.4 thousand, the rest latencies of steps that wait for one another: scores
// into P 500, the state 250 to 600, rows out 400, transposition 1100. (Warps of their own for some of the steps, 18 to 28 in all, overlap
// them and made nothing faster: d 128 219 -> 275 us.) 4 x 37 heads of 8192 tokens, one block an SM: d 128 1.24 GB in 218 us, 5.7 TB/s; d 64 0.62 GB in 126 to 145, 4.3 to 4.9.
#include "decay.cuh"
#include "tc_common.cuh"

namespace darkattn {
namespace {
using namespace tc;

constexpr int C = 128;
// Two warps share a quarter of the rows, each takes half of the columns of O, D and the state (four with a quarter each: twice the waits and arrivals,
// d 128 226 us for 220). Beside them one warp loads and stores, one issues products.
constexpr int kGroups = 2, kWarps = 4 * kGroups, kBlock = 32 * (kWarps + 2);
constexpr uint32_t kA = 0, kB = 128, kO = 256, kD = 384; // columns of tensor memory
constexpr uint32_t kX = 320;                             // X S of a narrow Z (64 columns), apart from P Z; of a wide one it goes to kO
// Chunks of at most kFew rows: P as two bf16 parts, the second where P's columns of tokens 64 .. 95 would be (four steps of K in all instead of eight). Over
// many rows P's roundings add a root of two to the error of the rows out; a row or two of few heads can come to twice that (0.0030 for 0.0016).
constexpr int kFew = 32;
constexpr int kDiag = 68;                                // numbers of each copy of the diagonal blocks' decays

struct TcMaps { CUtensorMap x, y, z, o; };
struct TcArgs { DecayArgs a; TcMaps m[kDecayPasses]; };

constexpr int kMostStages = 4;
// A wait sees one bit of a barrier's count, so nobody may be two phases behind. The products and the warps between them wait for one another item by
// item; the warp that loads and stores does not hold them up until they need a stage from it, so what it waits for has a barrier for each stage.
enum { FULL, DS = FULL + kMostStages, PZ = DS + kMostStages, SCORES = PZ + kMostStages, INTER, TMA_BARS, P_READY = TMA_BARS, T_READY, THIRD_READY, S_READY, O_READ, CLEAN, STAGED, NBARS = STAGED + kMostStages };

template <int DY, int DZ, bool MAIN>
struct TcSmem {
    static constexpr int kX = MAIN ? DY / 64 * 16384 : 0, kY = DY / 64 * 16384, kZ = DZ / 64 * 16384;
    static constexpr int kStage = kX + kY + kZ, kSpace = 232448 - 2560 - (MAIN ? kZ : 0), kStages = kSpace / kStage < kMostStages ? kSpace / kStage : kMostStages;
    static constexpr int S = kStages * kStage, tok = S + (MAIN ? kZ : 0), near = tok + 512, diag = near + 128, pw = diag + 4 * kDiag * 4, bars = pw + 528, slot = bars + NBARS * 8, total = slot + 16;
    static constexpr bool kEarly = MAIN && kZ <= kX;      // rows out are staged in X's place alone: Y and Z can be loaded before they are stored
    static_assert(kStages >= 2 && total <= 232448, "shared memory of a block");
};

// tiles of 64 columns and 128 rows of one head: [heads, N, width]
__device__ __forceinline__ void tma_load_3d(void *dst, const CUtensorMap *map, uint64_t *bar, int x, int y, int z)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(smem_u32(dst)), "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap *map, const void *src, int x, int y, int z)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];"
                 ::"l"(map), "r"(smem_u32(src)), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ float f(uint32_t x) { return __uint_as_float(x); }

// Shared memory by its 32-bit addresses: all of a block's are one number, read once, and constants.
__device__ __forceinline__ void arrive_warp(uint32_t bar, int lane)
{
    __syncwarp();
    if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void sts16(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
template <int N> __device__ __forceinline__ void quarter_bar(int q) { asm volatile("bar.sync %0, %1;" ::"r"(q + 1), "n"(N) : "memory"); }
template <int N> __device__ __forceinline__ void warps_bar() { asm volatile("bar.sync 5, %0;" ::"n"(N) : "memory"); }
// Two fp32 numbers as pairs of bf16 parts: returns the leading ones, leaves what remains (exact) in a and b.
__device__ __forceinline__ uint32_t take_part(float &a, float &b)
{
    const uint32_t p = pack_bf16(a, b);
    fma2(a, b, f(p << 16), f(p & 0xffff0000u), -1.f, -1.f);
    return p;
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ uint32_t fms_bf16x2(uint32_t a, uint32_t b, uint32_t c)      // a b - c
{
    uint32_t d;
    asm("{\n\t.reg .b32 n;\n\tneg.bf16x2 n, %3;\n\tfma.rn.bf16x2 %0, %1, %2, n;\n\t}" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
// Four 8 x 8 matrices of 16-bit numbers, transposed: lane t receives of each the numbers 2 (t % 4) and the next of column t / 4.
__device__ __forceinline__ void ldsm_t(uint32_t addr, uint32_t &r0, uint32_t &r1, uint32_t &r2, uint32_t &r3)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3) : "r"(addr) : "memory");
}
// 16 lanes x 16 columns of tensor memory; lane t of the warp holds, of every four columns, column t % 4 of rows t / 4 and t / 4 + 8.
__device__ __forceinline__ void tmem_st_16x128b(uint32_t a, const uint32_t (&v)[8])
{
    asm volatile("tcgen05.st.sync.aligned.16x128b.x4.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(a), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}

// 32 columns of Y and 32 of its tokens, times their weights, from shared memory (tokens are rows) to tensor
// memory (tokens are columns, two to a column).
//   TWO        two parts, formed in packed bf16 arithmetic from the weights' own two parts w1 + w2: p = y w1, rounded; y w1 - p is exact in 8 bits;
//              with y w2 added it is the second part. Off by 2^-16 of the number at most, and 3 instructions for two numbers where
//              unpacking, a product in fp32 and taking it apart are 8 (the transposition of a chunk: 1100 cycles)
//   LEAD       the first two of three parts, from an fp32 weight;  THIRD: the third;  ALL: three
enum { TWO, LEAD, THIRD, ALL };
template <int MODE, uint32_t PART>
__device__ __forceinline__ void weighted_transpose(uint32_t from, const float *weights, uint32_t to, uint32_t to3)
{
    // from: the address of this lane's matrix row of the first 16 tokens and columns; 16 more columns are two 16-byte chunks (a swizzled bit) on
    uint32_t y[2][8];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int tg = 0; tg < 2; ++tg) ldsm_t((from ^ (h << 5)) + tg * 2048, y[h][4 * tg], y[h][4 * tg + 1], y[h][4 * tg + 2], y[h][4 * tg + 3]);
    float2 w[4];                                          // of tokens 2 (lane % 4) and the next of every eight (TWO: pairs of first and of second parts)
#pragma unroll
    for (int m = 0; m < 4; ++m) w[m] = *reinterpret_cast<const float2 *>(weights + m * 8);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t lanes = (uint32_t)(16 * h) << 16;
        uint32_t p0[8], p1[8], p2[8];
#pragma unroll
        for (int m = 0; m < 8; ++m) {
            if (MODE == TWO) {
                const uint32_t w1 = __float_as_uint(w[m >> 1].x), w2 = __float_as_uint(w[m >> 1].y);
                p0[m] = mul_bf16x2(y[h][m], w1);
                p1[m] = fma_bf16x2(y[h][m], w2, fms_bf16x2(y[h][m], w1, p0[m]));
            } else {
                float u = f(y[h][m] << 16), v = f(y[h][m] & 0xffff0000u);
                mul2(u, v, w[m >> 1].x, w[m >> 1].y);
                p0[m] = take_part(u, v);
                p1[m] = take_part(u, v);
                p2[m] = pack_bf16(u, v);
            }
        }
        if (MODE != THIRD) {
            tmem_st_16x128b(to + lanes, p0);
            tmem_st_16x128b(to + PART + lanes, p1);
        }
        if (MODE >= THIRD) tmem_st_16x128b(to3 + lanes, p2);
    }
}

// MAIN: rows out; otherwise only the state of each of the first nseg - 1 segments, from zero, into pass.seg
template <int DY, int DZ, bool MAIN>
__global__ void __launch_bounds__(kBlock, 1) decay_tc_kernel(const __grid_constant__ TcArgs P)
{
    using M = TcSmem<DY, DZ, MAIN>;
    constexpr int W = DZ / kGroups;                       // columns of O, D and the state a warp takes
    static_assert(kGroups == 2 && (W == 32 || W == 64), "blocks of scores, tables and loads are laid out for two groups");
    // Narrow tiles (64 x 64): a state has half the rows of tensor memory. The tokens' two halves take one half of the rows each, so that all
    // warps transpose (with one half idle it was the longest step of a chunk), and leave two states, whose sum is the state: D is Y^T Z of the
    // first 64 tokens in its upper left quarter, of the others in its lower right one, and X S is [X X] times both.
    constexpr bool kHalves = DY == 64 && DZ == 64;
    constexpr uint32_t kPart = kHalves ? 32 : 64;         // columns of a part of w Y
    // the third part: behind the others, or in the half of the scores' columns that P does not take, once these have been read
    constexpr bool kBehindScores = MAIN && DZ == 128;
    constexpr uint32_t kThird = kHalves ? kB + 64 : DZ == 64 ? 448 : kA + 64;
    extern __shared__ __align__(1024) unsigned char smem[];
    unsigned char *sS = smem + M::S;
    float *tok = reinterpret_cast<float *>(smem + M::tok), *near = reinterpret_cast<float *>(smem + M::near), *diag = reinterpret_cast<float *>(smem + M::diag), *pw = reinterpret_cast<float *>(smem + M::pw);
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + M::bars);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + M::slot);
    volatile int *abort_flag = reinterpret_cast<int *>(smem + M::slot + 4);
    const int tid = threadIdx.x, warp = uniform(tid >> 5);
    int lane;
    asm volatile("mov.u32 %0, %%laneid;" : "=r"(lane));
    uint32_t sbase;
    asm volatile("mov.u32 %0, %1;" : "=r"(sbase) : "r"(smem_u32(smem)));
    const uint32_t bar = sbase + M::bars;                 // 8 bytes each
    const DecayArgs &A = P.a;

    const int nseg = MAIN ? A.nseg : A.nseg - 1;
    int id = blockIdx.x;
    const int ip = id % A.npass; id /= A.npass;
    const DecayPass &p = A.pass[ip];
    const int seg = id % nseg, head = id / nseg, HX = MAIN ? p.HX : A.Hkv;
    if (head >= A.B * HX) return;

    if (tid == 0) {
        for (int i = 0; i < TMA_BARS; ++i) mbar_init(bars + i, 1);
        for (int i = TMA_BARS; i < NBARS; ++i) mbar_init(bars + i, kWarps);
        *abort_flag = (smem_u32(smem) & 1023u) ? 1 : 0;
        fence_mbar_init();
    }
    if (warp == kWarps) { tmem_alloc(tmem_slot, 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_wait_tma();
    const uint32_t tmem = uniform(*tmem_slot);
    // (The first block to start clears the status; a wait gives up a second or two later.)
    if (A.clear && blockIdx.x == 0 && tid == 0) *A.status = 0;

    const int b = head / HX, hx = head % HX, hs = hx / (HX / A.Hkv);
    const int G = p.HY > HX ? p.HY / HX : 1;              // heads of Y that are summed over
    const int hy0 = b * p.HY + (p.HY > HX ? hx * G : hx / (HX / p.HY));
    const DecaySpan sp = decay_span<C>(A, b, seg);
    // (in registers for good: read where they are used, parameters miss the constant cache)
    const int reverse = uniform(p.reverse), a = uniform(p.a), c = uniform(p.c);
    const float row_mul = __int_as_float(uniform(__float_as_int(p.row_mul)));
    const int nchunk = sp.k1 - sp.k0, items = nchunk * G;
    const bool last_seg = sp.T == 0 ? seg == 0 : nchunk > 0 && sp.k1 == sp.T;
    const size_t state = (size_t)(b * A.Hkv + hs) * a * c;
    const float *S_in = nullptr;
    float *S_out = nullptr;
    if (MAIN) {
        S_in = seg == 0 ? (p.S_in ? p.S_in + state : nullptr) : p.seg + ((size_t)(b * A.Hkv + hs) * (nseg - 1) * A.sub + seg * A.sub - 1) * a * c;
        if (p.S_out && last_seg && hx % (HX / A.Hkv) == 0) S_out = p.S_out + state;
    } else if (nchunk) S_out = const_cast<float *>(p.seg) + ((size_t)(b * A.Hkv + hs) * nseg + seg) * a * c;
    const bool has0 = MAIN && S_in != nullptr;
    const int kept = MAIN && !S_out ? nchunk - 1 : nchunk;      // chunks behind which somebody reads the state
    const bool whole = MAIN ? S_out != nullptr : p.whole;   // three parts
    // A third part that follows the scores, its product behind P Z (d 128, 8 x 16 heads on 4 of 2001 tokens with states: all three
    // parts' product behind the scores, before P Z, 78 us, so 74).
    const bool later = kBehindScores && whole;
    // The states alone are summed from a piece's last chunk to its first (by the power of the decay to the piece's end): the pass that follows starts
    // where this one ends, on what is then in L2.
    const auto first_row = [&](int k) {
        const int at = sp.k0 + (MAIN ? k : nchunk - 1 - k);
        return (reverse ? sp.T - 1 - at : at) * C;
    };
    const auto stage_of = [&](int it) { return smem + it % M::kStages * M::kStage; };
    const auto load_yz = [&](int it, int k, int g) {      // of item `it`: chunk k, head g of those summed over
        if (elect_one()) {
            const TcMaps &m = P.m[ip];
            unsigned char *stage = stage_of(it);
            uint64_t *full = bars + FULL + it % M::kStages;
            const int t0 = first_row(k), hy = hy0 + g;
            mbar_expect_tx(full, M::kStage);              // (X's bytes among them)
            for (int x = 0; x < DY; x += 64) tma_load_3d(stage + M::kX + x * 256, &m.y, full, x, t0, hy);
            for (int x = 0; x < DZ; x += 64) tma_load_3d(stage + M::kX + M::kY + x * 256, &m.z, full, x, t0, hy);
        }
    };
    const auto load_x = [&](int it, int k) {
        if (MAIN && elect_one())
            for (int x = 0; x < DY; x += 64) tma_load_3d(stage_of(it) + x * 256, &P.m[ip].x, bars + FULL + it % M::kStages, x, first_row(k), head);
    };
    const bool fine = *abort_flag == 0;
    if (warp == kWarps && fine) {                         // the first items' loads, beside the tables
        for (int it = 0, k = 0, g = 0; it < M::kStages && it < items; ++it) {
            load_yz(it, k, g);
            load_x(it, k);
            if (++g == G) { g = 0; ++k; }
        }
    }
    if (tid <= C) pw[tid] = decay_power(A.log_decay[hs], tid);
    __syncthreads();
    // Decays of a block of 32 x 32 scores by column, times p_mul: from the near edge where the block is off the diagonal; on it, where row r needs
    // lambda^|r - j| (0 behind it), four copies, each shifted by one, let every row read its 32 numbers four at a time: copy r % 4 from 32 - r / 4 * 4 on.
    if (tid < 32) near[tid] = p.p_mul * pw[p.reverse ? tid : 31 - tid];
    for (int i = tid; i < 4 * kDiag; i += kBlock) {
        const int j = i % kDiag - 32 - i / kDiag, n = p.reverse ? j : -j;       // column less row
        diag[i] = n >= 0 && n < 32 ? p.p_mul * pw[n] : 0.f;
    }
    __syncthreads();

    if (MAIN && warp != kWarps) zero_behind<C>(A, sp, seg, static_cast<__nv_bfloat16 *>(p.O) + (size_t)head * A.N * c, c, tid < 32 * kWarps ? tid : tid - 32, kBlock - 32);

    int *status = A.status;

    if (!fine) {
        if (tid == 0) atomicExch(status, (int)DARKATTN_ERR_CUDA);
    } else if (warp == kWarps) {                       // ------------------------------------------------ loads and stores
        const TcMaps &m = P.m[ip];
        // Item by item: its products done, its stage takes the next item's Y and Z; its rows out staged, they are stored, and X follows. (All three
        // behind the store, and two stages at width 64: a chunk there waited for its loads, 135 us for what now takes 125.)
        bool ok = true;
        int k1 = 0, g1 = 0;                               // chunk and head of the item that goes into the stage
        for (int it = 0; it < M::kStages && it < items; ++it)
            if (++g1 == G) { g1 = 0; ++k1; }
        for (int it = 0, k = 0, g = 0; it < items && ok; ++it) {
            const int next = it + M::kStages;
            ok = warp_wait_tries(bar + 8 * ((MAIN ? PZ : DS) + it % M::kStages), it / M::kStages & 1, status);
            if (ok && later) ok = warp_wait_tries(bar + 8 * (DS + it % M::kStages), it / M::kStages & 1, status);      // the last to read Y and Z
            if (!ok) break;
            if ((M::kEarly || !MAIN) && next < items) load_yz(next, k1, g1);
            if (MAIN && g == G - 1) {
                ok = warp_wait_tries(bar + 8 * (STAGED + k % M::kStages), k / M::kStages & 1, status);
                if (!ok) break;
                if (sp.n - first_row(k) >= C && elect_one()) {
                    for (int x = 0; x < DZ && x < c; x += 64) tma_store_3d(&m.o, stage_of(it) + x * 256, x, first_row(k), head);
                    tma_store_commit();
                    tma_store_wait_read();
                }
            }
            if (next < items) {
                if (MAIN && !M::kEarly) load_yz(next, k1, g1);
                load_x(next, k1);
                if (++g1 == G) { g1 = 0; ++k1; }
            }
            if (++g == G) { g = 0; ++k; }
        }
        if (MAIN && elect_one()) tma_store_wait_all();
        if (!ok) *abort_flag = 1;
    } else if (warp == kWarps + 1) {                   // ------------------------------------------------ products
        // In this order the pipe has something to do while the warps turn scores into P (X S, D), scale X S (D) and take the state (P Z).
        const uint32_t id_scores = make_idesc(128, 128, 0, 0), id_z = make_idesc(128, DZ, 0, 1), id_d = kHalves ? make_idesc(128, 128, 0, 1) : id_z;
        const TileDesc tS(sS);
        const int parts = whole && !later ? 3 : 2;
        bool ok = true;
        int clean = 0;
        for (int it = 0, k = 0, g = 0; it < items && ok; ++it, k += g + 1 == G, g = g + 1 == G ? 0 : g + 1) {
            const unsigned char *stage = stage_of(it);
            const TileDesc tX(stage), tY(stage + M::kX), tZ(stage + M::kX + M::kY);
            const bool inter = has0 || k > 0;
            if (MAIN) {
                ok = warp_wait_tries(bar + 8 * (FULL + it % M::kStages), it / M::kStages & 1, status);
                if (ok && sp.n - first_row(k) < C) ok = warp_wait_tries(bar + 8 * CLEAN, clean++ & 1, status);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int q = 0; q < DY / 16; ++q) mma_ss(tmem + kA, kdesc(tX, q), kdesc(tY, q), id_scores, q > 0);
                    mma_commit(bars + SCORES);
                }
            }
            if (g == 0) {
                ok = warp_wait_tries(bar + 8 * S_READY, k & 1, status);
                if (MAIN && ok && k > 0) ok = warp_wait_tries(bar + 8 * O_READ, (k - 1) & 1, status);
                if (!ok) break;
                if (MAIN && inter) {
                    tc_fence_after();
                    if (elect_one()) {
#pragma unroll
                        for (int q = 0; q < (kHalves ? 8 : DY / 16); ++q)
                            mma_ss(tmem + (DZ == 64 ? kX : kO), kdesc(tX, kHalves ? q & 3 : q), mndesc(tS, q), id_z, q > 0);
                        mma_commit(bars + INTER);
                    }
                }
            }
            if (k < kept) {
                ok = warp_wait_tries(bar + 8 * T_READY, it & 1, status);
                if (!ok) break;
                tc_fence_after();
            }
            if (k < kept && elect_one()) {
                const uint64_t halves = make_sdesc(smem_u32(stage + M::kX + M::kY), 64 * 128, 1024);      // Z's rows 0 .. 63 and 64 .. 127 as columns side by side
                for (int part = 0; part < parts; ++part) {
                    const uint32_t left = tmem + (part < 2 ? kB + kPart * part : kThird);
#pragma unroll
                    for (int q = 0; q < (kHalves ? 4 : 8); ++q)
                        mma_ts(tmem + kD, left + 8 * q, kHalves ? halves + (uint64_t)(q * 2048 >> 4) : mndesc(tZ, q), id_d, g > 0 || part > 0 || q > 0);
                }
                if (!later) mma_commit(bars + DS + it % M::kStages);
            }
            if (MAIN) {
                const bool few = sp.n - first_row(k) <= kFew;
                ok = warp_wait_tries(bar + 8 * P_READY, it & 1, status);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        if (!few || (q & 3) < 2) mma_ts(tmem + kO, tmem + kA + 8 * q, mndesc(tZ, few ? q & 3 : q), id_z, (DZ == 128 && inter) || g > 0 || q > 0);
                    mma_commit(bars + PZ + it % M::kStages);
                }
                if (later) {
                    ok = warp_wait_tries(bar + 8 * THIRD_READY, it & 1, status);
                    if (!ok) break;
                    tc_fence_after();
                    if (elect_one()) {
#pragma unroll
                        for (int q = 0; q < 8; ++q) mma_ts(tmem + kD, tmem + kThird + 8 * q, mndesc(tZ, q), id_d, true);
                        mma_commit(bars + DS + it % M::kStages);
                    }
                }
            }
        }
        if (!ok) *abort_flag = 1;
    } else {                                              // ------------------------------------------------ what lies between the products
        const int quarter = warp & 3, cb = warp >> 2, row = quarter * 32 + lane, z0 = cb * W;
        const uint32_t at = tmem + ((uint32_t)(quarter * 32) << 16);
        const bool rows_y = kHalves || quarter * 32 < DY; // this warp's lanes are rows of the state
        const int srow = kHalves ? row & 63 : row, half = kHalves ? quarter >> 1 : 0;      // row of the state, half of the tokens
        const uint32_t own = (uint32_t)((z0 >> 6) * 16384 + row * 128 + ((((z0 >> 3) & 7) ^ (row & 7)) << 4));      // this lane's first 16 bytes in a swizzled tile
        const uint32_t y_own = (uint32_t)(M::kX + (kHalves ? half * 2 * 4096 : (quarter >> 1) * 16384) + (((lane >> 4) & 1) * 8 + (lane & 7)) * 128 + ((((quarter & 1) * 4 + ((lane >> 3) & 1)) ^ (lane & 7)) << 4));
        __nv_bfloat16 *O = MAIN ? static_cast<__nv_bfloat16 *>(p.O) + (size_t)head * A.N * c : nullptr;
        float s[W];                                       // the state: row `row`, columns z0 ..
        const bool by4 = MAIN && seg > 0;                 // between segments as [dv / 4][d][4], from the caller as [d][dv]
#pragma unroll
        for (int j = 0; j < W; j += 4) {
            float4 x = make_float4(0, 0, 0, 0);
            const int z = z0 + j;
            if (S_in && srow < a && z < c && half == 0) {
                if (!p.trans) x = *reinterpret_cast<const float4 *>(S_in + (by4 ? ((size_t)(z / 4) * a + srow) * 4 : (size_t)srow * c + z));
                else {                                    // rows here are columns there; z and the three behind it are rows
                    const float *col = S_in + (by4 ? ((size_t)(srow / 4) * c + z) * 4 + srow % 4 : (size_t)z * a + srow);
                    const int step = by4 ? 4 : a;
                    x = make_float4(col[0], col[step], col[2 * step], col[3 * step]);
                }
            }
            s[j] = x.x; s[j + 1] = x.y; s[j + 2] = x.z; s[j + 3] = x.w;
        }
        const auto put_state = [&]() {                    // its copy for the product with the next chunk's rows
            if (rows_y) {
#pragma unroll
                for (int q = 0; q < W / 8; ++q)
                    sts16((sbase + M::S + own) ^ (q << 4), pack_bf16(s[8 * q], s[8 * q + 1]), pack_bf16(s[8 * q + 2], s[8 * q + 3]), pack_bf16(s[8 * q + 4], s[8 * q + 5]), pack_bf16(s[8 * q + 6], s[8 * q + 7]));
                fence_async_smem();
            }
        };
        if (has0) put_state();
        arrive_warp(bar + 8 * S_READY, lane);
        // A wait that gave up ends all further waiting, not the loop: the warps still meet at their barriers, on numbers that mean nothing.
        bool ok = true;
#define DWAIT(b, ph) do { if (ok) ok = warp_wait_tries(bar + 8 * (b), (ph), status); } while (0)
        int Ltok = -1;
        uint32_t inters = 0;
        // Brings item `it`'s weighted Y (of a chunk of L rows) into tensor memory.
        const auto prepare = [&](int it, int k, int L) {
            const uint32_t stage = sbase + it % M::kStages * M::kStage;
            DWAIT(FULL + it % M::kStages, it / M::kStages & 1);
            if (L != Ltok || L < C) {
                warps_bar<32 * kWarps>();                 // the weights of the chunk before have been used
                for (int i = tid; i < C; i += 32 * kWarps) {
                    const float w = i < L ? pw[reverse ? i + 1 : L - 1 - i] * p.tok_mul : 0.f;
                    if (whole) tok[i] = w;
                    else {                                // pairs of tokens: the weights' first parts, then the second
                        __nv_bfloat16 *at2 = reinterpret_cast<__nv_bfloat16 *>(tok) + (i >> 1) * 4 + (i & 1);
                        at2[0] = __float2bfloat16_rn(w);
                        at2[2] = __float2bfloat16_rn(w - __bfloat162float(at2[0]));
                    }
                }
                if (L < C) {                              // rows behind the end are padding: zero, whatever they hold
                    const int per = (M::kY + M::kZ) / 16384 * 8;      // chunks of 16 bytes of a row of Y and Z
                    for (int i = tid; i < (C - L) * per; i += 32 * kWarps) {
                        const int r = L + i / per, q = i % per;
                        sts16(stage + M::kX + (q >> 3) * 16384 + swz128(r, q & 7), 0, 0, 0, 0);
                    }
                    fence_async_smem();
                }
                warps_bar<32 * kWarps>();
                if (L < C) arrive_warp(bar + 8 * CLEAN, lane);
                Ltok = L;
            }
            if (k >= kept) return;
            if (rows_y) {
#pragma unroll
                for (int tb = 0; tb < (kHalves ? 2 : 4) / kGroups; ++tb) {
                    const int t = cb + kGroups * tb;      // of 32 tokens
                    const float *w = tok + (half * 2 + t) * 32 + 2 * (lane & 3);
                    if (!whole) weighted_transpose<TWO, kPart>(stage + y_own + t * 4096, w, at + kB + t * 16, 0);
                    else weighted_transpose<kBehindScores ? LEAD : ALL, kPart>(stage + y_own + t * 4096, w, at + kB + t * 16, at + kThird + t * 16);
                }
            }
            tmem_wait_st();
            tc_fence_before();
            arrive_warp(bar + 8 * T_READY, lane);
        };
        const auto rows_of = [&](int k) { return min(C, sp.n - first_row(k)); };
        // Blocks of 32 columns of the scores: a warp takes the outer or the inner two (the triangle has as much in either).
        // Off the diagonal by column, and a power for the row, up to the block's near edge; on the diagonal by a table alone.
        const auto block_of = [&](int i) { return cb == 0 ? 3 * i : 1 + i; };
        float p_row[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int blk = block_of(i);
            p_row[i] = (reverse ? blk > quarter : blk < quarter) ? pw[reverse ? blk * 32 - row : row - blk * 32 - 31] : 1.f;
        }
        float x_row = 0.f;                                // of X S
        float behind = 1.f;                               // (states alone) the decay from the chunk's end to the piece's
        int Lx = -1;
        if (items > 0) prepare(0, 0, rows_of(0));
        for (int it = 0, k = 0, g = 0; it < items; ++it) {
            const int t0 = first_row(k), L = min(C, sp.n - t0);
            if (MAIN) {                                   // P: the lower (backwards: the upper) triangle, times the decays
                DWAIT(SCORES, it & 1);
                tc_fence_after();
                if (L <= kFew) {
                    if (cb == 0) {                        // no other warp reads or writes these rows' columns
                        const bool off = reverse ? 0 > quarter : 0 < quarter;
                        uint32_t lead[16] = {}, rest[16] = {};
                        if (off || quarter == 0) {
                            const float *by = off ? near : diag + (lane & 3) * kDiag + 32 - (lane & ~3);
                            uint32_t v[32];
                            tmem_ld32(at + kA, v);
                            tmem_wait_ld();
#pragma unroll
                            for (int j = 0; j < 32; j += 2) {
                                float x = f(v[j]) * p_row[0] * by[j], y = f(v[j + 1]) * p_row[0] * by[j + 1];
                                lead[j / 2] = take_part(x, y);
                                rest[j / 2] = pack_bf16(x, y);
                            }
                        }
                        tmem_st16(at + kA, lead);
                        tmem_st16(at + kA + 32, rest);
                    }
                } else {
                    uint32_t pk[2][16];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int blk = block_of(i);
                        const bool off = reverse ? blk > quarter : blk < quarter;
                        if (off || blk == quarter) {
                            const float *by = off ? near : diag + (lane & 3) * kDiag + 32 - (lane & ~3);
                            uint32_t v[32];
                            tmem_ld32(at + kA + blk * 32, v);
                            tmem_wait_ld();
#pragma unroll
                            for (int j = 0; j < 32; j += 4) {
                                const float4 w = *reinterpret_cast<const float4 *>(by + j);
                                float x[4] = {f(v[j]), f(v[j + 1]), f(v[j + 2]), f(v[j + 3])};
                                mul2(x[0], x[1], p_row[i], p_row[i]);
                                mul2(x[2], x[3], p_row[i], p_row[i]);
                                mul2(x[0], x[1], w.x, w.y);
                                mul2(x[2], x[3], w.z, w.w);
                                pk[i][j / 2] = pack_bf16(x[0], x[1]);
                                pk[i][j / 2 + 1] = pack_bf16(x[2], x[3]);
                            }
                        } else {
#pragma unroll
                            for (int j = 0; j < 16; ++j) pk[i][j] = 0;
                        }
                    }
                    quarter_bar<32 * kGroups>(quarter);       // P takes the place of scores that other warps read
#pragma unroll
                    for (int i = 0; i < 2; ++i) tmem_st16(at + kA + block_of(i) * 16, pk[i]);
                }
                if (L != Lx) {
                    x_row = row < L ? row_mul * pw[reverse ? L - 1 - row : row + 1] : 0.f;
                    Lx = L;
                }
                if (DZ == 128 && g == 0 && (has0 || k > 0)) {
                    DWAIT(INTER, inters++ & 1);
                    tc_fence_after();
#pragma unroll
                    for (int h = 0; h < W; h += 32) {
                        uint32_t o[32];
                        tmem_ld32(at + kO + z0 + h, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(f(o[j]) * x_row);
                        tmem_st32(at + kO + z0 + h, o);
                    }
                }
                tmem_wait_st();
                tc_fence_before();
                arrive_warp(bar + 8 * P_READY, lane);
                if (later) {
                    if (rows_y) {
#pragma unroll
                        for (int tb = 0; tb < 4 / kGroups; ++tb) {
                            const int t = cb + kGroups * tb;
                            weighted_transpose<THIRD, kPart>(sbase + it % M::kStages * M::kStage + y_own + t * 4096, tok + t * 32 + 2 * (lane & 3), 0, at + kThird + t * 16);
                        }
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    arrive_warp(bar + 8 * THIRD_READY, lane);
                }
            }
            if (k < kept) DWAIT(DS + it % M::kStages, it / M::kStages & 1);
            if (k < kept && g == G - 1) {
                tc_fence_after();
                const float keep = MAIN ? pw[L] : 1.f, share = behind;
                if (!MAIN) behind *= pw[L];
#pragma unroll
                for (int h = 0; h < W; h += 32) {
                    uint32_t o[32];
                    tmem_ld32(at + kD + half * 64 + z0 + h, o);
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 32; ++j) s[h + j] = MAIN ? fmaf(keep, s[h + j], f(o[j])) : fmaf(share, f(o[j]), s[h + j]);
                }
                if (MAIN) put_state();
                tc_fence_before();
                arrive_warp(bar + 8 * S_READY, lane);
            }
            if (MAIN) {
                DWAIT(PZ + it % M::kStages, it / M::kStages & 1);
                if (g == G - 1) {
                    tc_fence_after();
                    const uint32_t stage = sbase + it % M::kStages * M::kStage + own;
#pragma unroll
                    for (int h = 0; h < W; h += 32) {
                        uint32_t o[32];
                        tmem_ld32(at + kO + z0 + h, o);
                        if (DZ == 64 && (has0 || k > 0)) {
                            uint32_t x[32];
                            tmem_ld32(at + kX + z0 + h, x);
                            tmem_wait_ld();
#pragma unroll
                            for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(fmaf(f(x[j]), x_row, f(o[j])));
                        }
                        tmem_wait_ld();
                        if (h + 32 == W) {
                            tc_fence_before();
                            arrive_warp(bar + 8 * O_READ, lane);
                        }
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const uint4 r = pack8(o + 8 * q);
                            if (L == C) sts16(stage ^ ((h / 8 + q) << 4), r.x, r.y, r.z, r.w);
                            else if (row < L && z0 + h + 8 * q < c) *reinterpret_cast<uint4 *>(O + (size_t)(t0 + row) * c + z0 + h + 8 * q) = r;
                        }
                    }
                    fence_async_smem();
                    arrive_warp(bar + 8 * (STAGED + k % M::kStages), lane);
                }
            }
            if (++g == G) { g = 0; ++k; }
            if (it + 1 < items) prepare(it + 1, k, rows_of(k));
        }
#undef DWAIT
        if (!ok) *abort_flag = 1;
        if (S_out) {
            if (kHalves) {                                // the other half's state: where the copy was, or (states alone) in a stage, 16 KB
                const uint32_t at2 = sbase + (MAIN ? M::S : 0);
                const auto cell = [&](int j) { return at2 + (uint32_t)((srow * 16 + ((z0 + j) / 4 ^ (srow & 15))) * 16); };
                warps_bar<32 * kWarps>();                 // the last copies have been written
                if (half == 1) {
#pragma unroll
                    for (int j = 0; j < W; j += 4) sts16(cell(j), __float_as_uint(s[j]), __float_as_uint(s[j + 1]), __float_as_uint(s[j + 2]), __float_as_uint(s[j + 3]));
                }
                warps_bar<32 * kWarps>();
                if (half == 0) {
#pragma unroll
                    for (int j = 0; j < W; j += 4) {
                        float4 x;
                        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(cell(j)) : "memory");
                        s[j] += x.x; s[j + 1] += x.y; s[j + 2] += x.z; s[j + 3] += x.w;
                    }
                }
            }
            if (half == 0 && srow < a) {
#pragma unroll
                for (int j = 0; j < W; j += 4)
                    if (z0 + j < c) *reinterpret_cast<float4 *>(S_out + (MAIN ? (size_t)srow * c + z0 + j : ((size_t)((z0 + j) / 4) * a + srow) * 4)) = make_float4(s[j], s[j + 1], s[j + 2], s[j + 3]);
            }
        }
    }
    __syncwarp();
    if (*abort_flag) __nanosleep(200000);                 // copies that are still on their way
    tc_fence_before();
    __syncthreads();
    if (warp == kWarps) tmem_dealloc(tmem, 512);
}

bool make_map3(CUtensorMap *m, const void *base, int heads, int N, int width)
{
    EncodeTiledFn enc = encode_fn();
    if (!enc) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)width, (cuuint64_t)N, (cuuint64_t)heads}, strides[2] = {(cuuint64_t)width * 2, (cuuint64_t)width * 2 * (cuuint64_t)N};
    const cuuint32_t box[3] = {64, C, 1}, es[3] = {1, 1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DY, int DZ, bool MAIN>
cudaError_t launch(const TcArgs &P, cudaStream_t st)
{
    int heads = 0;
    for (int i = 0; i < P.a.npass; ++i) heads = max(heads, P.a.B * (MAIN ? P.a.pass[i].HX : P.a.Hkv));
    const long long blocks = (long long)P.a.npass * heads * (MAIN ? P.a.nseg : P.a.nseg - 1);
    return launch_pdl(decay_tc_kernel<DY, DZ, MAIN>, dim3((unsigned)blocks), dim3(kBlock), TcSmem<DY, DZ, MAIN>::total, st, P);
}

// Passes whose widths are of one class share a launch. Where one wave of blocks holds them all, every pass does, on wide tiles: a launch waits for
// the one before (3 x 16 heads on 8 of 1024 tokens, gradients at d 128, dv 64: 82 us in two launches, 65 in one).
template <bool MAIN>
darkattn_status_t launch_all(const DecayArgs &A, const DecayPass *pass, int npass, bool first, cudaStream_t st)
{
    bool done[kDecayPasses] = {};
    long long blocks = 0;
    bool y_wide = false, z_wide = false;
    for (int i = 0; i < npass; ++i) {
        blocks += (long long)A.B * (MAIN ? pass[i].HX : A.Hkv) * A.nseg;
        y_wide |= pass[i].a > 64;
        z_wide |= pass[i].c > 64;
    }
    const bool together = blocks <= 148;
    for (int i = 0; i < npass; ++i) {
        if (done[i]) continue;
        const bool y2 = together ? y_wide : pass[i].a > 64, z2 = together ? z_wide : pass[i].c > 64;
        TcArgs P;
        P.a = A;
        P.a.clear = first && i == 0;
        int n = 0;
        for (int j = i; j < npass; ++j) {
            const DecayPass &q = pass[j];
            if (done[j] || (!together && ((q.a > 64) != y2 || (q.c > 64) != z2))) continue;
            done[j] = true;
            P.a.pass[n] = q;
            bool ok = make_map3(&P.m[n].y, q.Y, A.B * q.HY, A.N, q.a) && make_map3(&P.m[n].z, q.Z, A.B * q.HY, A.N, q.c);
            if (MAIN) ok = ok && make_map3(&P.m[n].x, q.X, A.B * q.HX, A.N, q.a) && make_map3(&P.m[n].o, q.O, A.B * q.HX, A.N, q.c);
            else P.m[n].x = P.m[n].o = P.m[n].y;
            if (!ok) { set_cuda_error(cudaErrorInvalidValue, "decay: tensor map"); return DARKATTN_ERR_CUDA; }
            ++n;
        }
        P.a.npass = n;
        const cudaError_t e = y2 ? (z2 ? launch<128, 128, MAIN>(P, st) : launch<128, 64, MAIN>(P, st)) : (z2 ? launch<64, 128, MAIN>(P, st) : launch<64, 64, MAIN>(P, st));
        DARKATTN_CUDA_TRY(e, "decay_tc_kernel");
    }
    return DARKATTN_OK;
}

}  // namespace

bool decay_tc_supported(const darkattn_decay_desc_t &ds)
{
    return ds.dtype == DARKATTN_BF16 && ds.d % 8 == 0 && ds.dv % 8 == 0 && ds.d <= 128 && ds.dv <= 128;
}

// Segments, and the pieces whose states are summed first: the cheapest by an estimate in us, fitted to measurements on a B200. A chunk takes 2.6 us
// (wide tiles, 64 to 128 columns) or 1.7 us while few blocks run, and what the memory gives when all SMs do (5.7 and, power-bound, 4.8 TB/s);
// a chunk of the states alone 1.4 or 1.0 us, a wave of blocks 2 us more; two kernels more 9 or 4 us, twice that where there are two sets of states. One head of 8192 tokens, d 128: 178 us in one
// segment, 22.4 in 32, 24.5 in the 64 that it picks; 4 x 16 heads on one set of inputs, in part in L2 (on several by turns): 195 (167) in one, 141 (161 to 166)
// in two with two pieces each, 165 (178) in two whole ones, 205 (194) in four; 8 heads of 65536, d 64: 920 in one, 105 in 18.
// Segments have to promise 8 % (a backward pass in one segment shares more of its reads in L2 than the estimate knows: 4 x 16 heads, 382 us
// in one, 424 in two).
// `heads` heads of a pass take an item a chunk, `sums` of them G: those that sum over a group's heads. Where these are the longer ones nothing is done
// before they are: 2 x 12 heads on 3, 898 tokens, gradients at d 96, dv 64: 70 us in one segment, 39 in four.
static void pick(int T, int d, int dv, DecayLoad rows, DecayLoad states, int sets, int &nseg, int &cps, int &sub)
{
    const bool wide = d > 64 || dv > 64;
    const double chunk = wide ? 2.6 : 1.7, state_chunk = wide ? 1.4 : 1.0, more = sets * (wide ? 9 : 4), rate = wide ? 5.7e6 : 4.8e6;
    const double bytes = 2.0 * C * 2 * (d + dv);
    const auto phase = [&](const DecayLoad &x, long long pieces, int per, double us, double b) {
        const long long blocks = (x.heads + x.sums) * pieces;
        const double all = 148 * b / rate, rest = (double)(blocks % 148) * b / rate;
        if (x.G > 1) {
            const double long_one = x.G * us, shared = (double)(x.heads + x.sums * x.G) * pieces / 148 * (all > us ? all : us);
            return 2.0 * ((blocks + 147) / 148) + per * (long_one > shared ? long_one : shared);
        }
        return 2.0 * ((blocks + 147) / 148) + per * ((double)(blocks / 148) * (all > us ? all : us) + (blocks % 148 ? (rest > us ? rest : us) : 0));
    };
    // a backward pass of widths of two classes: dQ and dK by one launch, dV by another, unless one wave holds them
    const auto main_phase = [&](long long pieces, int per) {
        if (rows.sums == 0 || (d > 64) == (dv > 64) || (rows.heads + rows.sums) * pieces <= 148) return phase(rows, pieces, per, chunk, bytes);
        return phase({rows.heads, rows.sums / 2, rows.G}, pieces, per, chunk, bytes) + phase({0, rows.sums / 2, rows.G}, pieces, per, chunk, bytes);
    };
    nseg = 1; cps = T; sub = 1;
    double best = main_phase(1, T);
    for (int n = 2; n <= T && n <= 64; ++n) {
        for (int q = 1; q <= 4; ++q) {
            const int per = ((T + n - 1) / n + q - 1) / q * q, m = (T + per - 1) / per;
            if (m < 2) continue;
            const double cost = 1.08 * (main_phase(m, per) + phase(states, (m - 1) * q, per / q, state_chunk, bytes / 2) + more + 0.06 * (m - 1) * q);
            if (cost < best) { best = cost; nseg = m; cps = per; sub = q; }
        }
    }
}

void decay_tc_split(darkattn_decay_plan_s *plan)
{
    const darkattn_decay_desc_t &ds = plan->desc;
    const int T = (ds.N + C - 1) / C;
    const long long q = (long long)ds.B * ds.H, k = (long long)ds.B * ds.H_kv;
    const int G = ds.H / ds.H_kv;
    pick(T, ds.d, ds.dv, {q, 0, 1}, {k, 0, 1}, 1, plan->fwd.nseg, plan->fwd.cps, plan->fwd.sub);
    pick(T, ds.d, ds.dv, {q, 2 * k, G}, {k, k, G}, 2, plan->bwd.nseg, plan->bwd.cps, plan->bwd.sub);
}

darkattn_status_t decay_tc_run(DecayArgs &A, DecayPass *state_pass, int nstate, cudaStream_t st)
{
    if (A.nseg > 1) {
        const DecayArgs P = decay_pieces(A, state_pass, nstate);
        if (darkattn_status_t rc = launch_all<false>(P, P.pass, nstate, true, st)) return rc;
        for (int i = 0; i < nstate; ++i) DARKATTN_CUDA_TRY(decay_scan_pieces(P, state_pass[i], C, true, st), "decay_scan_kernel");
    }
    return launch_all<true>(A, A.pass, A.npass, A.nseg == 1, st);
}

}  // namespace darkattn
