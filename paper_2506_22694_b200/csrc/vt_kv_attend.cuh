// Attention of a sequence's new rows over its paged cache (Algorithm 2's drafter forward; the rows are a draft tree's nodes), split over the
// cache's length and joined.
//
//   o = sum_t p_t v_t / sum_t p_t,  p_t = exp(scale * q.k_t - m),  over the committed tokens t < len and, of the drafted tokens at
//   len + node, the row's node and its ancestors
//
// One pass with a running maximum; what is kept of a part (maximum m in base 2, sum l, weighted values o) joins with another part by
// m' = max, l' = l 2^(m - m') + ..., o' likewise.  Over e4m3 rows o has a maximum of its own, of score plus the exponent e of the token's values:
// a weight enters the product as 2^(score + e - v), which fits f16 whatever the powers are, l stands against m, and
// out = o 2^(v - m) / l.  (With one maximum for both, tokens whose scores are as large but whose values are 2^126 times as small as others' fell
// out of l.)
//
// Bound: HBM, 2 * d * (2 or 1) bytes of a token and key head, each read once for all rows that share the head.  So the rows of a key head
// (its query heads times the sequence's new rows) lie side by side as the 16 rows of an MMA, up to four such groups (WR) on warps that share
// the tiles.  mma.sync is far from its own limit at 16 and 32 rows (a token and head is two MMAs in the 22 cycles in which an SM's share of HBM
// delivers it), and it keeps scores and weights in registers, where tcgen05 would send both through TMEM for tiles of 128 rows that
// are seven eighths empty.
//
// Measured (heads of 128, 8 key heads): 64 sequences of up to 8000 tokens, bf16, 170 us, 93% of what copying HBM reaches; e4m3 114 us, 70%: there a
// tile's instructions on twelve warps bound it (half the bytes, but conversions, exponents and a second exponential on top).  32 rows a head of 64 in
// e4m3, 24%: 44% of the issue slots are used, a third of the stalls wait for the instruction before.  One sequence of 4000 tokens: 12.4 us, of which 6.7 are
// what a call of 64 tokens takes: 1.7 before it starts, lengths and shares 1, page ids and first copies 1.7, a tile 0.8, meeting
// and results 1.7.  The rest: another tile a team, the fence and the ticket of a part 0.9, the join 1.6.
//
// Split: the work is cut into units of 64 tokens, in the order (sequence, key head, group of rows, tokens), and every CTA takes an equal run of
// units, whatever the lengths are; nothing is known to the host, so a captured graph stays right when lengths change.  A (sequence, head, group)
// whose units lie in several CTAs leaves partial results.  Those of up to eight rows are joined by the CTA whose part comes last, others by a
// second launch; always in the order of the tokens.
//
// Roles: four producer warps walk the CTA's run, look pages up, and fill rings of tiles by tensor copies of 16 or 32 tokens, as far ahead as
// the rings reach (copies of a row each took 10 ns apiece, twice what there is).  Eight warps consume, as 8 / WR teams that take the tiles in
// turn.  So the copies go on while a result is finished and the next one's queries are fetched, which took 5 us a result when the same warps
// did both.
#pragma once
#include <cuda_fp16.h>

#include "vt_kv_join.cuh"
#include "vt_maps.cuh"
#include "vt_mbar.cuh"

namespace vt {
namespace {

constexpr int kAttWarps = 8;                                     // that consume
constexpr int kAttFeeds = 4;                                     // that produce
constexpr int kAttThreads = 32 * (kAttWarps + kAttFeeds);
// Registers: 168 of each thread at the launch are 2016 of each lane; the consumers take 200, which leaves the producers 104.
constexpr int kAttConsumerRegs = 200, kAttProducerRegs = 104;
static_assert(kAttWarps * kAttConsumerRegs + kAttFeeds * kAttProducerRegs <= (kAttWarps + kAttFeeds) * 168, "what the block was launched with");
constexpr int kAttUnit = 64;                                     // tokens
// What a result counts for besides its tokens when the work is dealt out (the walk to it, its queries, the meeting), and a tree's tokens.
// Single calls, L2 flushed, us with 4 / 8 / 12 for a result: 64 ragged sequences of up to 8000 tokens, bf16 187 / 189 / 191, e4m3 136 / 121 / 120; 16 of up
// to 3000, bf16, 39 / 41 / 43.  With 4 / 8 / 12 / 16 / 24 for a tree: one over 4001 tokens 31.8 / 29.7 / 29.7 / 29.7 / 29.7, eight over 1000
// 31.8 / 31.8 / 31.9 / 31.8 / 34.7, 32 over 6000 in e4m3 72.7 / 74.8 / 74.8 / 74.9 / 78.8.
constexpr int kAttPairUnits = 8, kAttTreeUnits = 12;
// No result is split so near to its ends.  2 / 4 / 6: a tree over 4001 tokens 19.8 / 21.3 / 23.8 us, a token over 1024 10.8 / 12.5 / 13.1, over 4000
// 12.6 / 13.1 / 14.5, batches alike.
constexpr int kAttSnap = 2;
constexpr float kAttLift = 11.0f;                                // e4m3: weights of values are 2^11 to 2^15 at the most, of f16's 65504
constexpr int kAttLens = 1024;                                   // sequences whose lengths are kept in shared memory
constexpr int kAttTile = 32;                                      // tokens of a tile: one of each lane of the producer that fills it
constexpr int kAttTurns = 2;                                     // tiles of a producer in a round
constexpr int kAttRound = kAttTile * kAttFeeds * kAttTurns;      // tokens that the producers look up at a time

template <int D, bool F8, int WR>
struct AttCfg {
    static constexpr int kTeams = kAttWarps / WR;
    static constexpr int kTile = kAttTile;
    static constexpr int kRow = D * (F8 ? 1 : 2);                // bytes of a cached row
    // A tile lies in shared memory as tensor copies write it: blocks of kBox bytes of all its rows, the 16-byte vectors of a row swapped by the
    // copies' swizzle of that width, so that ldmatrix meets no bank twice.
    static constexpr int kBox = kRow % 128 == 0 ? 128 : kRow % 64 == 0 ? 64 : 32;
    static constexpr int kHalf = kTile * kRow;
    static constexpr int kSlot = 2 * kHalf;                      // keys, values
    static constexpr int kToken = F8 ? 8 : 4;                    // what a tile holds of a token besides its rows
    static constexpr int kMasks = kTile * kToken;                // the rows that see a tree's token, 8 bytes each
    static constexpr int kHeader = kMasks + kTile * 8;
    static constexpr int kNote = kHeader + 16;
    static constexpr bool kQRegs = D <= 128;                     // query fragments stay in registers
    static constexpr int kQPitch = 2 * D + 16;
    static constexpr int kQBytes = kQRegs ? 0 : WR * 16 * kQPitch;
    static constexpr int kVectors = D / 8 + (F8 ? 2 : 1);        // of a lane's share of a result
    static constexpr int kMeet = kAttWarps / 2 * kVectors * 512; // where the teams' results meet: those of half of them
    static constexpr int kParents = 2 * kKvMaxNodes + 4 * kAttLens;                        // ... and the lengths
    static constexpr int kFree = 226 * 1024 - 2048 - kQBytes - kMeet - kParents;
    // A ring of kPer places for each producer.  Tile 4 t + p of a round is producer p's in turn t, and goes to team (4 t + p) mod teams; a place is
    // always of the same team: who waits for a turn of a place has waited for every turn before, and cannot take the next but one, of the same
    // parity, for its own.
    static constexpr int kShare = kTeams > kAttFeeds ? kTeams / kAttFeeds : 1;             // teams of a ring
    static constexpr int kPer = (kFree / (kSlot + kNote) < 40 ? kFree / (kSlot + kNote) : 40) / kAttFeeds / kShare * kShare;
    static constexpr int kSlots = kAttFeeds * kPer;
    static constexpr int kSmem = kSlots * (kSlot + kNote) + kQBytes + kMeet + kParents + 1024;     // (and what brings the ring to 1024)
    static_assert(kPer >= kShare, "a place for each team");
    static_assert(kRow % 32 == 0 && kSlot % 1024 == 0 && kNote % 16 == 0, "shapes");

    __device__ static __forceinline__ uint32_t swizzle(uint32_t row) { return kBox == 128 ? row & 7 : kBox == 64 ? (row >> 1) & 3 : (row >> 2) & 1; }
    __device__ static __forceinline__ uint32_t place(uint32_t row, uint32_t vec) {         // of a row's 16-byte vector in half a tile
        constexpr uint32_t kVecs = kBox / 16;
        return vec / kVecs * (kTile * kBox) + row * kBox + ((vec % kVecs ^ swizzle(row)) << 4);
    }
};
// What a tile holds of a token: e4m3: the power of two of its key (0: no such token) and the exponent of its values (NaN: they are no numbers);
// bf16: whether there is no such token.
enum { kAttEnd = 1, kAttEmpty = 2, kAttTree = 4, kAttShort = 8 };            // a tile's header (short: some tokens are missing)

// 16 bytes, or zeros where `have` is false (then the source is not read)
__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool have) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(have ? 16 : 0) : "memory");
}
// a box of the cache's map: dim x, token, head, page
__device__ __forceinline__ void box_copy(uint32_t dst, const CUtensorMap* map, int x, int token, int head, int page, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
        ::"r"(dst), "l"(map), "r"(x), "r"(token), "r"(head), "r"(page), "r"(bar) : "memory");
}
// orders this thread's stores to shared memory in front of later bulk copies into the same place
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void ldsm(uint32_t* r, uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm_t(uint32_t* r, uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
template <bool F16>
__device__ __forceinline__ void mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    if (F16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_fast(float x) {            // ex2.approx: 2 ulp; weights below 2^-126 are zero
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// Four e4m3 bytes as two pairs of f16 (exact).  A tree's values (FINITE) by their bits, moved to f16's places, which is the value times
// 2^-8, and one exact multiplication: a NaN byte then is a number, and a weight of zero keeps it out of the rows that do not see it.
template <bool FINITE>
__device__ __forceinline__ void e4m3_pairs(uint32_t x, uint32_t& lo, uint32_t& hi) {
    if (FINITE) {
        const uint32_t a = __byte_perm(x, 0, 0x1404), b = __byte_perm(x, 0, 0x3424);
        const uint32_t c = (a & 0x80008000u) | ((a >> 1) & 0x3f803f80u), d = (b & 0x80008000u) | ((b >> 1) & 0x3f803f80u);
        asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(c), "r"(0x5c005c00u));
        asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(d), "r"(0x5c005c00u));
    } else {
        asm("{ .reg .b16 a, b; mov.b32 {a, b}, %2; cvt.rn.f16x2.e4m3x2 %0, a; cvt.rn.f16x2.e4m3x2 %1, b; }" : "=r"(lo), "=r"(hi) : "r"(x));
    }
}

// The tokens of half a tile that hold a byte 0x7f or 0xff (NaN), a bit each.
template <class C>
__device__ __forceinline__ uint32_t nan_tokens(const uint8_t* half, int lane) {
    constexpr int V = C::kRow / 16;
    uint32_t bad = 0;
#pragma unroll 4
    for (int x = lane; x < C::kTile * V; x += 32) {
        const uint4 w = *reinterpret_cast<const uint4*>(half + C::place(x / V, x % V));
        uint32_t high = 0;
        for (const uint32_t y : {w.x, w.y, w.z, w.w}) high |= (y & 0x7f7f7f7fu) + 0x01010101u;
        if (high & 0x80808080u) bad |= 1u << x / V;
    }
    return __reduce_or_sync(0xffffffffu, bad);
}

// 2^k by its bits, k clamped to what fp32 holds
__device__ __forceinline__ float two_to(int k) { return __uint_as_float((uint32_t)(min(max(k, -126), 127) + 127) << 23); }

// A query row goes into f16 under the power of two that brings its largest magnitude to [2^14, 2^15): eight significant bits fit, and
// what underflows is 2^-39 of the largest.  From the largest's bits: the power.
__device__ __forceinline__ int q_power(uint32_t top_bits) { return min(14 + 127 - (int)(top_bits >> 23), 120); }
// two bf16 as f16 times 2^k
__device__ __forceinline__ uint32_t q_pair(uint32_t w, float f) {
    const __half2 h = __floats2half2_rn(__uint_as_float(w << 16) * f, __uint_as_float(w & 0xffff0000u) * f);
    return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ void consumers_barrier() { asm volatile("bar.sync 15, %0;" ::"n"(32 * kAttWarps) : "memory"); }

__device__ __forceinline__ void feeds_barrier() { asm volatile("bar.sync 14, %0;" ::"n"(32 * kAttFeeds) : "memory"); }

__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {       // without arriving
    asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void st_shared(uint32_t at, const uint4& x) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
}
__device__ __forceinline__ void st_shared(uint32_t at, uint32_t x) { asm volatile("st.shared.u32 [%0], %1;" ::"r"(at), "r"(x) : "memory"); }
__device__ __forceinline__ uint32_t ld_shared(uint32_t at) {
    uint32_t x;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(at) : "memory");
    return x;
}

// What bounds a CTA's waits, in shared memory.
struct __align__(16) AttStop {
    long long cycles;             // the bound of each
    long long dead;               // one has run out
};
// A wait within the CTA (nothing here waits for another).  False: it has run out, or another one has.  From then on a producer asks for no
// further copy and arrives nowhere (a barrier that still counts a copy's bytes takes no arrival of the next turn), a consumer
// takes and gives back no further tile, both walk their run to its end (so that barriers, tickets and the list of parts are as always), and the
// results are no numbers.  What a producer has asked for lands before it leaves.
__device__ __forceinline__ bool att_wait(uint32_t bar, uint32_t parity, uint32_t stop, Ctrl* ctrl) {
    if (bar_test(bar, parity)) return true;
    const long long t0 = clock64();
    for (;;) {
        long long cycles, dead;
        asm volatile("ld.shared.v2.s64 {%0,%1}, [%2];" : "=l"(cycles), "=l"(dead) : "r"(stop) : "memory");
        if (cycles < kShortBoundCycles ? bar_test(bar, parity) : bar_try(bar, parity)) return true;
        if (dead) return false;
        if (clock64() - t0 > cycles) {
            asm volatile("st.shared.s64 [%0], %1;" ::"r"(stop + 8), "l"(1ll) : "memory");
            atomicOr(&ctrl->flags, (uint32_t)VT_FLAG_TIMEOUT);
            return false;
        }
    }
}

// What a warp keeps of its 16 rows: lane holds rows lane / 4 and lane / 4 + 8.
template <int D>
struct AttAcc {
    float o[D / 8][4];
    float m[2], l[2];
    float v[2];                   // e4m3: what o stands against, the maximum of score plus the values' exponent, less kAttLift
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
        m[0] = m[1] = v[0] = v[1] = -INFINITY;
        l[0] = l[1] = 0.0f;
    }
};

// One tile: scores of the warp's 16 rows with its tokens, running maximum, weighted values.  LIST: tokens are a tree's nodes, and the
// tile's masks say which new rows see each.  HALF: there are eight rows at the most, the lanes' second rows are none.  `some`: tokens are
// missing (their keys are zeros, of which an infinite query makes a NaN: the score is replaced, nothing is added to it).  No row sees a missing node.
template <int D, bool F8, int WR, bool HALF, bool LIST>
__device__ __forceinline__ void att_tile(AttAcc<D>& acc, const uint32_t (*qf)[4], uint32_t q_smem, const uint8_t* slot, const uint8_t* note, bool some, const float (&scale)[2],
                                         int qi0, int qi1) {
    using C = AttCfg<D, F8, WR>;
    constexpr int NT = C::kTile / 8;                             // groups of 8 tokens
    constexpr int NR = HALF ? 1 : 2;                             // rows of a lane
    const int lane = threadIdx.x & 31, j = lane & 3;
    float s[NT][4];
#pragma unroll
    for (int i = 0; i < NT; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.0f;
    const uint32_t base = smem_u32(slot);
    // ldmatrix: the lane's row, and the place of its vector there, but for the step's even number of vectors
    constexpr uint32_t kVecs = C::kBox / 16;
    const uint32_t k_row = (lane >> 4) * 8 + (lane & 7), k_at = base + k_row * C::kBox, k_vec = (((lane >> 3) & 1) ^ C::swizzle(k_row)) << 4;
    constexpr int KS = C::kRow / 32;                             // 32 bytes of a row at a time
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        uint32_t qa[F8 ? 2 : 1][4];
#pragma unroll
        for (int x = 0; x < (F8 ? 2 : 1); ++x) {
            const int step = F8 ? 2 * ks + x : ks;
            if (C::kQRegs) {
#pragma unroll
                for (int i = 0; i < 4; ++i) qa[x][i] = qf[step][i];
            } else {
                ldsm(qa[x], q_smem + (lane & 15) * C::kQPitch + (2 * step + (lane >> 4)) * 16);
            }
        }
#pragma unroll
        for (int g = 0; g < C::kTile / 16; ++g) {
            uint32_t b[4];
            ldsm(b, k_at + (k_vec ^ (2 * ks % kVecs << 4)) + 2 * ks / kVecs * (C::kTile * C::kBox) + g * 16 * C::kBox);
            if (!F8) {
                mma<false>(s[2 * g], qa[0], b[0], b[1]);
                mma<false>(s[2 * g + 1], qa[0], b[2], b[3]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {                    // i: (token half, dim half)
                    uint32_t lo, hi;
                    e4m3_pairs<false>(b[i], lo, hi);
                    mma<true>(s[2 * g + (i >> 1)], qa[i & 1], lo, hi);
                }
            }
        }
    }
    // scores in base 2, and their maxima (e4m3: with the exponent of the values on top, too)
    float top[2] = {-INFINITY, -INFINITY}, vtop[2] = {-INFINITY, -INFINITY}, ve[NT][2];
    uint32_t sees[2] = {0, 0};                                   // LIST: bit 2 i + u: the row sees token 8 i + 2 j + u
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int t = 8 * i + 2 * j + u;
            if (F8) {
                // (the powers of the key and of the query first: a large one may undo a small one)
                const float2 x = *reinterpret_cast<const float2*>(note + 8 * t);
                s[i][u] *= x.x * scale[0];
                if (!HALF) s[i][2 + u] *= x.x * scale[1];
                ve[i][u] = x.y;
            } else {
                s[i][u] *= scale[0];
                if (!HALF) s[i][2 + u] *= scale[1];
            }
        }
    if (!LIST && some) {
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t x = *reinterpret_cast<const uint32_t*>(note + C::kToken * (8 * i + 2 * j + u));
                if (F8 ? !x : x) s[i][u] = s[i][2 + u] = -INFINITY;
            }
    }
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (LIST) {
                const int t = 8 * i + 2 * j + u;
                const unsigned long long bits = *reinterpret_cast<const unsigned long long*>(note + C::kMasks + 8 * t);
                const bool r0 = (bits >> qi0) & 1, r1 = (bits >> qi1) & 1;
                sees[0] |= (uint32_t)r0 << (2 * i + u), sees[1] |= (uint32_t)r1 << (2 * i + u);
                if (!r0) s[i][u] = -INFINITY;
                if (!r1) s[i][2 + u] = -INFINITY;
            }
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                top[r] = fmaxf(top[r], s[i][2 * r + u]);
                if (F8) vtop[r] = fmaxf(vtop[r], s[i][2 * r + u] + ve[i][u]);
            }
        }
    // (a row's maximum is that of its four lanes; whether it grows, any of them can say)
    bool grows = false;
#pragma unroll
    for (int r = 0; r < NR; ++r) grows |= top[r] > acc.m[r] + 4.0f || (F8 && vtop[r] > acc.v[r] + (4.0f + kAttLift));
    // The kept references may lie up to 4 below the true ones (weights up to 16): results are divided by the sum of the same weights,
    // and most tiles need not scale what is there.  v lies kAttLift below its own: weights up to 2^15 use f16's range, whose numbers lose bits
    // below 2^-14 and end at 2^-24, as far as it goes.
    if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
        for (int r = 0; r < NR; ++r) {
#pragma unroll
            for (int o = 1; o < 4; o *= 2) {
                top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], o));
                if (F8) vtop[r] = fmaxf(vtop[r], __shfl_xor_sync(0xffffffffu, vtop[r], o));
            }
            const float m = fmaxf(acc.m[r], top[r]), v = fmaxf(acc.v[r], vtop[r] - kAttLift);
            const float f = m == acc.m[r] ? 1.0f : exp2_fast(acc.m[r] - m);
            const float g = !F8 ? f : v == acc.v[r] ? 1.0f : exp2_fast(acc.v[r] - v);
            acc.m[r] = m, acc.v[r] = v;
            acc.l[r] *= f;
#pragma unroll
            for (int i = 0; i < D / 8; ++i) acc.o[i][2 * r] *= g, acc.o[i][2 * r + 1] *= g;
        }
    }
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const float m = acc.m[r] == -INFINITY ? 0.0f : acc.m[r], v = acc.v[r] == -INFINITY ? 0.0f : acc.v[r];
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const float p0 = exp2_fast(s[i][2 * r] - m), p1 = exp2_fast(s[i][2 * r + 1] - m);
            acc.l[r] += p0 + p1;
            s[i][2 * r] = F8 ? exp2_fast(s[i][2 * r] + ve[i][0] - v) : p0;
            s[i][2 * r + 1] = F8 ? exp2_fast(s[i][2 * r + 1] + ve[i][1] - v) : p1;
            if (F8 && LIST) {                                    // (the exponent of a row that held a NaN is one)
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    if (!((sees[r] >> (2 * i + u)) & 1)) s[i][2 * r + u] = 0.0f;
            }
        }
    }
    if (F8 && LIST) {
        const uint8_t* vals = slot + C::kHalf;
#pragma unroll 1
        for (uint32_t bad = nan_tokens<C>(vals, lane); bad; bad &= bad - 1) {
            const int t = __ffs(bad) - 1;
            const unsigned long long bits = *reinterpret_cast<const unsigned long long*>(note + C::kMasks + 8 * t);
#pragma unroll
            for (int i = 0; i < D / 8; i += 2) {                 // (the lane's four dims of every 16)
                const uint32_t w = *reinterpret_cast<const uint32_t*>(vals + C::place(t, i / 2) + 4 * j);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if ((w >> (8 * e) & 0x7f) != 0x7f) continue;
                    if ((bits >> qi0) & 1) acc.o[i + (e & 1)][e >> 1] = NAN;
                    if ((bits >> qi1) & 1) acc.o[i + (e & 1)][2 + (e >> 1)] = NAN;
                }
            }
        }
    }
    bool odd = false;
    if (LIST && !F8) {
        // A drafted token that some of the rows see stays out of the others' sums by a weight of zero, and zero times an infinity or a NaN is
        // a NaN.  Such values are added to the rows that see them one by one, and are zeros for the MMA.
        const uint8_t* vals = slot + C::kHalf;
        for (int x = lane; x < C::kTile * (D / 8); x += 32) {
            const uint4 w = *reinterpret_cast<const uint4*>(vals + C::place(x / (D / 8), x % (D / 8)));
            const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) odd |= (ws[i] & 0x7f80u) == 0x7f80u || (ws[i] & 0x7f800000u) == 0x7f800000u;
        }
        odd = __any_sync(0xffffffffu, odd);
        if (odd) {
#pragma unroll
            for (int i = 0; i < NT; ++i)
                for (int t = 0; t < 8; t += 2) {                 // tokens t and t + 1 of the eight, from the lane that holds them
                    const int from = (lane & ~3) | (t >> 1);
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const float p0 = __shfl_sync(0xffffffffu, s[i][u], from), p1 = __shfl_sync(0xffffffffu, s[i][2 + u], from);
                        const bool r0 = (__shfl_sync(0xffffffffu, sees[0], from) >> (2 * i + u)) & 1;
                        const bool r1 = (__shfl_sync(0xffffffffu, sees[1], from) >> (2 * i + u)) & 1;
#pragma unroll
                        for (int nt = 0; nt < D / 8; ++nt)
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                const uint32_t bits = reinterpret_cast<const uint16_t*>(vals + C::place(8 * i + t + u, nt))[2 * j + x];
                                if ((bits & 0x7f80u) != 0x7f80u) continue;
                                const float v = __uint_as_float(bits << 16);
                                if (r0) acc.o[nt][x] += p0 * v;
                                if (r1) acc.o[nt][2 + x] += p1 * v;
                            }
                    }
                }
        }
    }
    // bf16: weights go into the MMA as two pieces, the rounded weight and what the rounding left (2^-17 of it at most): one piece alone would
    // add as much error as the rounding of the result, and at these rates the second MMA is free.  e4m3: one piece of f16: 2^-11 of a weight, and no
    // less than 2^-36 of the row's heaviest (which is 2^11 to 2^15 here, and half a step below 2^-14 is 2^-25).
    const uint32_t v_row = ((lane >> 3) & 1) * 8 + (lane & 7), v_at = base + C::kHalf + v_row * C::kBox, v_vec = ((lane >> 4) ^ C::swizzle(v_row)) << 4;
#pragma unroll
    for (int g = 0; g < C::kTile / 16; ++g) {
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {                            // i: (row half, token half) of the A fragment
            hi[i] = lo[i] = 0;
            if (HALF && (i & 1)) continue;
            const float x = s[2 * g + (i >> 1)][2 * (i & 1)], y = s[2 * g + (i >> 1)][2 * (i & 1) + 1];
            if (F8) {
                const __half2 h = __floats2half2_rn(x, y);
                hi[i] = *reinterpret_cast<const uint32_t*>(&h);
            } else {
                hi[i] = pack_bf16(x, y);
                lo[i] = pack_bf16(x - __uint_as_float(hi[i] << 16), y - __uint_as_float(hi[i] & 0xffff0000u));
            }
        }
#pragma unroll
        for (int c = 0; c < C::kRow / 32; ++c) {
            uint32_t b[4];
            ldsm_t(b, v_at + (v_vec ^ (2 * c % kVecs << 4)) + 2 * c / kVecs * (C::kTile * C::kBox) + g * 16 * C::kBox);
            if (LIST && !F8 && odd) {
#pragma unroll
                for (int i = 0; i < 4; ++i) b[i] &= ((b[i] & 0x7f80u) == 0x7f80u ? 0u : 0xffffu) | ((b[i] & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u);
            }
            if (!F8) {
                mma<false>(acc.o[2 * c], hi, b[0], b[1]);
                mma<false>(acc.o[2 * c + 1], hi, b[2], b[3]);
                mma<false>(acc.o[2 * c], lo, b[0], b[1]);
                mma<false>(acc.o[2 * c + 1], lo, b[2], b[3]);
            } else {
#pragma unroll
                for (int x = 0; x < 2; ++x) {                    // 16 dims each: a word is (t0 d0, t0 d1, t1 d0, t1 d1)
                    uint32_t e0, o0, e1, o1;
                    e4m3_pairs<LIST>(__byte_perm(b[2 * x], 0, 0x3120), e0, o0);
                    e4m3_pairs<LIST>(__byte_perm(b[2 * x + 1], 0, 0x3120), e1, o1);
                    mma<true>(acc.o[4 * c + 2 * x], hi, e0, e1);
                    mma<true>(acc.o[4 * c + 2 * x + 1], hi, o0, o1);
                }
            }
        }
    }
}

// Quotients of numbers that nearly always fit 32 bits (a division of 64 takes some hundred instructions).
__device__ __forceinline__ int quotient(int x, int y) { return (int)((uint32_t)x / (uint32_t)y); }
__device__ __forceinline__ long long quotient(long long x, long long y) {
    return ((x | y) >> 32) == 0 ? (long long)((uint32_t)x / (uint32_t)y) : x / y;
}

// The run of units of a CTA, segment by segment; the producer and the consumers walk it each on their own.
struct AttWalk {
    long long u, u1, off;         // next unit, end, and the next unit's place in its sequence
    int seq;
};
struct AttSegment {
    int seq, head, group, len, units, tile0, count;
    int token, token_end;         // committed tokens of this segment
    bool tree;                    // it holds the tree's tokens, too
};

__device__ __forceinline__ int att_len(const KvAttendArgs& a, int s) {
    return (int)min((int64_t)max(ld_cg_s32(a.lens + s), 0), (int64_t)a.c.max_pages * a.c.page);
}
__device__ __forceinline__ int att_units(const KvAttendArgs& a, int len) {
    return len / kAttUnit + (len % kAttUnit != 0) + kAttPairUnits + (a.node ? kAttTreeUnits : 0);
}
__device__ __forceinline__ bool att_next(const KvAttendArgs& a, const int* lens, int groups, AttWalk& w, AttSegment& g) {
    if (w.u >= w.u1) return false;
    g.seq = w.seq;
    g.len = g.seq < kAttLens ? lens[g.seq] : att_len(a, g.seq);
    g.units = att_units(a, g.len);
    const int pair = (int)quotient(w.off, (long long)g.units);
    g.tile0 = (int)(w.off - (long long)pair * g.units);
    g.count = (int)min((long long)(g.units - g.tile0), w.u1 - w.u);
    g.head = groups == 1 ? pair : pair / groups, g.group = pair - g.head * groups;
    g.token = (int)min((long long)max(g.tile0 - kAttPairUnits, 0) * kAttUnit, (long long)g.len);
    g.token_end = (int)min((long long)max(g.tile0 + g.count - kAttPairUnits, 0) * kAttUnit, (long long)g.len);
    g.tree = a.node && g.tile0 + g.count == g.units;
    w.u += g.count, w.off += g.count;
    if (w.off == (long long)g.units * a.c.heads * groups) ++w.seq, w.off = 0;
    return true;
}

enum { kChain, kLevels, kNodes };                                // how a producer finds a tree's nodes
constexpr int kAttDeep = 64;                                     // depths that are walked in step

// A producer's lane: its tokens of a round, one of each tile.
struct AttTokens {
    int32_t id[kAttTurns], in[kAttTurns];                        // page (below 0: no row to read) and place in it (-1: no token)
    unsigned long long mask[kAttTurns];                          // a tree's token: the rows that see it
    uint32_t ke[kAttTurns], ve[kAttTurns];                       // e4m3: its exponents' bytes
    int head, n;                                                 // tokens of the round
    bool tree, last, have;                                       // the segment ends with it; it exists
};

template <int D, bool F8, int WR>
struct AttProducer {
    using C = AttCfg<D, F8, WR>;
    const KvAttendArgs& a;
    const CUtensorMap *k_map, *v_map;
    uint32_t ring, notes, full, empty, stop;                     // of this producer, in shared memory
    int16_t* parents;
    const int* lens;
    AttWalk walk;
    AttSegment g;
    int groups, lane, feed;
    int mode;                     // 0: the next segment, 1: committed tokens, 2: the tree's
    int tree_of, n0, n1;          // whose tree is here; nodes of rows lane and lane + 32
    int f0, f1;                   // where those have got to
    int way = 0, depth = 0, most = 0;                            // how nodes are found; of row lane's node (-1: none), and of all rows'
    int level = 0;                // where the search is
    int held;                     // a parent on its way
    bool fresh = false, begun = false;                           // the tree's loads are in flight; the segment's tree has been begun
    int place = 0, filled = 0;    // of the next tile, in the ring; tiles so far
    uint32_t parity = 1;          // (an empty ring's places count as given back)
    unsigned long long dirty = 0; // places that hold rows which threads have stored

    __device__ int mine(int turn) const { return kAttTile * (kAttFeeds * turn + feed) + lane; }      // which of a round's tokens

    // a lane's tokens of the next round -> their page ids (the loads are left in flight)
    __device__ void look_up(AttTokens& r) {
        if (mode == 0) {
            r.have = att_next(a, lens, groups, walk, g);
            if (!r.have) return;
            mode = g.token >= g.token_end && g.tree ? 2 : 1;
            begun = false;
            if (g.tree && tree_of != g.seq) ask_tree();
        }
        r.have = true, r.head = g.head, r.tree = mode == 2;
        int index[kAttTurns];
#pragma unroll
        for (int t = 0; t < kAttTurns; ++t) index[t] = -1, r.mask[t] = 0;
        if (mode == 1) {
            r.n = min(g.token_end - g.token, kAttRound);
#pragma unroll
            for (int t = 0; t < kAttTurns; ++t)
                if (mine(t) < r.n) index[t] = g.token + mine(t);
            g.token += r.n;
            r.last = g.token >= g.token_end && !g.tree;
            if (g.token >= g.token_end) mode = g.tree ? 2 : 0;
        } else {
            if (!begun) begin_tree();
            begun = true;
            r.n = 0;
            if (way == kChain) {                                 // every node up to the largest
                r.n = min(most - level, kAttRound);
#pragma unroll
                for (int t = 0; t < kAttTurns; ++t)
                    if (mine(t) < r.n) index[t] = place_of(level + mine(t));
#pragma unroll 1
                for (int row = 0; row < a.Q; ++row) {
                    const int f = __shfl_sync(0xffffffffu, row < 32 ? n0 : n1, row & 31);
#pragma unroll
                    for (int t = 0; t < kAttTurns; ++t)
                        if (level + mine(t) <= f) r.mask[t] |= 1ull << row;
                }
                level += r.n;
                r.last = level >= most;
            } else if (way == kLevels) {                         // a depth at a time, deepest first
                for (; level > 0 && r.n + 32 <= kAttRound; --level) {
                    const bool here = depth >= level;
                    const unsigned same = __match_any_sync(0xffffffffu, here ? f0 : -1 - lane);
                    const unsigned first = __ballot_sync(0xffffffffu, here && (same & ((1u << lane) - 1)) == 0);
                    const int count = __popc(first);
#pragma unroll
                    for (int t = 0; t < kAttTurns; ++t) {
                        const int k = mine(t) - r.n;             // which of the depth's nodes is this lane's
                        if (!__any_sync(0xffffffffu, k >= 0 && k < count)) continue;
                        int from = 0;
#pragma unroll
                        for (int w = 16; w; w >>= 1)
                            if (__popc(first & ((1u << (from + w)) - 1)) <= k) from += w;
                        const int f = __shfl_sync(0xffffffffu, f0, from & 31);
                        const unsigned rows = __shfl_sync(0xffffffffu, same, from & 31);
                        if (k >= 0 && k < count) index[t] = place_of(f), r.mask[t] = rows;
                    }
                    r.n += count;
                    if (here) f0 = parents[f0];
                }
                r.last = level <= 0;
            } else {                                             // one by one, largest first
                for (; r.n < kAttRound; ++r.n) {
                    const int f = __reduce_max_sync(0xffffffffu, max(f0, f1));
                    if (f < 0) break;
                    const unsigned lo = __ballot_sync(0xffffffffu, f0 == f), hi = __ballot_sync(0xffffffffu, f1 == f);
#pragma unroll
                    for (int t = 0; t < kAttTurns; ++t)
                        if (r.n == mine(t)) index[t] = place_of(f), r.mask[t] = ((unsigned long long)hi << 32) | lo;
                    const int up = parents[f];
                    f0 = f0 == f ? up : f0, f1 = f1 == f ? up : f1;
                }
                r.last = __reduce_max_sync(0xffffffffu, max(f0, f1)) < 0;
            }
            if (r.last) mode = 0;
        }
#pragma unroll
        for (int t = 0; t < kAttTurns; ++t) {
            r.id[t] = r.in[t] = -1;
            if (index[t] < 0) continue;
            const uint32_t page = a.page_shift >= 0 ? (uint32_t)index[t] >> a.page_shift : (uint32_t)index[t] / (uint32_t)a.c.page;
            r.in[t] = index[t] - (int32_t)(page * (uint32_t)a.c.page);
            r.id[t] = page < (uint32_t)a.c.max_pages ? ld_cg_s32(a.c.pages + (int64_t)g.seq * a.c.pages_ld + page) : -1;
        }
    }

    __device__ int place_of(int f) const { return (int)min((int64_t)g.len + f, (int64_t)INT32_MAX); }

    // A sequence's tree: loads that are left in flight while the committed tokens are looked up, ...
    __device__ void ask_tree() {
        tree_of = g.seq, fresh = true;
        n0 = lane < a.Q ? ld_cg_s32(a.node + (int64_t)g.seq * a.Q + lane) : -1;
        n1 = lane + 32 < a.Q ? ld_cg_s32(a.node + (int64_t)g.seq * a.Q + lane + 32) : -1;
        if (!a.parent) return;
        const int i = 32 * feed + lane;
        held = i < a.N ? ld_cg_s32(a.parent + (int64_t)g.seq * a.parent_ld + i) : -1;
    }
    // ... and what it takes to find the nodes that some row sees, each once, with the rows that see it: of a chain all up to the largest; in a
    // tree the rows (32 at the most) walk to the root in step, by depth; where there are more rows or a node lies deep, they are merged node by
    // node.  Every producer finds them all, for its own tokens.  Against node by node for all: 8 sequences of 512 tokens with a chain
    // of 64 rows each 52 us for 55, one of 1000 tokens with 32 rows in a tree of 200 nodes 22.2 for 23.7.
    __device__ void begin_tree() {
        if (fresh) {
            fresh = false;
            const int N = a.N;
            if (n0 >= N || n1 >= N) kv_flag(a.ctrl);
            n0 = n0 < 0 || n0 >= N ? -1 : n0, n1 = n1 < 0 || n1 >= N ? -1 : n1;
            way = kChain;
            most = __reduce_max_sync(0xffffffffu, max(n0, n1)) + 1;
            if (a.parent) {
                feeds_barrier();                                 // (the others have done with the parents before)
                auto keep = [&](int i, int p) {
                    if (i < N) parents[i] = (int16_t)(p >= 0 && p < i ? p : -1);           // (a parent that does not lie in front ends the walk)
                };
                keep(32 * feed + lane, held);
                for (int i = 32 * (kAttFeeds + feed) + lane; i < N; i += 32 * kAttFeeds)
                    keep(i, ld_cg_s32(a.parent + (int64_t)g.seq * a.parent_ld + i));
                feeds_barrier();
                way = a.Q > 32 ? kNodes : kLevels;
                depth = most = 0;
                for (int f = n0; way == kLevels && __any_sync(0xffffffffu, f >= 0); ++most) {
                    if (most == kAttDeep) way = kNodes;
                    if (f >= 0) f = parents[f], ++depth;
                }
            }
        }
        f0 = n0, f1 = n1;
        level = way == kLevels ? most : 0;
    }

    // page ids -> exponents (left in flight, too)
    __device__ void resolve(AttTokens& r) {
#pragma unroll
        for (int t = 0; t < kAttTurns; ++t) {
            if ((uint32_t)r.id[t] >= (uint32_t)a.c.n_pages) {
                if (r.in[t] >= 0) kv_flag(a.ctrl);
                r.id[t] = -1;
            }
            if (F8) {
                // (fewer than 2^31 rows fit any GPU's memory)
                const uint32_t e = r.id[t] >= 0 ? ((uint32_t)r.id[t] * a.c.heads + r.head) * a.c.page + r.in[t] : 0u;
                asm volatile("ld.global.cg.u8 %0, [%1];" : "=r"(r.ke[t]) : "l"(a.c.k_exp + e) : "memory");
                asm volatile("ld.global.cg.u8 %0, [%1];" : "=r"(r.ve[t]) : "l"(a.c.v_exp + e) : "memory");
            }
        }
    }

    // A tile's rows.  16 or 32 tokens of a page at a time come by tensor copies, where they are all there.
    __device__ __forceinline__ void copy(const AttTokens& r, int turn, int at) {
        const uint32_t tile = ring + at * C::kSlot, bar = full + 8 * at;
        const int32_t id = r.id[turn], in = r.in[turn];
        const int rest = r.n - kAttTile * (kAttFeeds * turn + feed);                       // tokens of the tile, and of those behind it
        unsigned boxed = 0;                                      // tokens that come so
        if (!r.tree && a.box == 32 && rest >= 32) {
            const int id0 = __shfl_sync(0xffffffffu, id, 0), in0 = __shfl_sync(0xffffffffu, in, 0);
            if (id0 >= 0) {
                boxed = 0xffffffffu;
                if (elect_one()) {
                    if (dirty >> at & 1) fence_async();          // (what threads have stored there comes first)
                    bar_expect(bar, 2 * 32 * C::kRow);
#pragma unroll
                    for (int x = 0; x < C::kRow / C::kBox; ++x) {
                        const uint32_t to = tile + x * C::kTile * C::kBox;
                        const int dim = x * (F8 ? C::kBox : C::kBox / 2);
                        box_copy(to, k_map, dim, in0, r.head, id0, bar);
                        box_copy(to + C::kHalf, v_map, dim, in0, r.head, id0, bar);
                    }
                }
                __syncwarp();
                dirty &= ~(1ull << at);
                return;
            }
        } else if (!r.tree && a.box == 16 && rest >= 16) {
            const int id0 = __shfl_sync(0xffffffffu, id, 0), in0 = __shfl_sync(0xffffffffu, in, 0);
            const int id1 = __shfl_sync(0xffffffffu, id, 16), in1 = __shfl_sync(0xffffffffu, in, 16);
            boxed = (id0 >= 0 ? 0xffffu : 0u) | (id1 >= 0 && rest >= 32 ? 0xffff0000u : 0u);
            if (boxed && elect_one()) {
                if (dirty >> at & 1) fence_async();
                bar_expect(bar, __popc(boxed) * 2 * C::kRow);
#pragma unroll
                for (int x = 0; x < C::kRow / C::kBox; ++x) {
                    const uint32_t to = tile + x * C::kTile * C::kBox;
                    const int dim = x * (F8 ? C::kBox : C::kBox / 2);
                    if (boxed & 1u) {
                        box_copy(to, k_map, dim, in0, r.head, id0, bar);
                        box_copy(to + C::kHalf, v_map, dim, in0, r.head, id0, bar);
                    }
                    if (boxed >> 31) {
                        box_copy(to + 16 * C::kBox, k_map, dim, in1, r.head, id1, bar);
                        box_copy(to + C::kHalf + 16 * C::kBox, v_map, dim, in1, r.head, id1, bar);
                    }
                }
            }
            __syncwarp();
            if (boxed) dirty &= ~(1ull << at);
            if (boxed == 0xffffffffu) return;
        }
        // the others row by row, missing ones as zeros (a weight of zero does not undo what lay there)
        dirty |= 1ull << at;
        constexpr int V = C::kRow / 16;                          // vectors of a row
        const int64_t mine = id >= 0 ? (int64_t)id * a.c.stride_page + (int64_t)in * a.c.stride_token + r.head * a.c.stride_head : -1;
#pragma unroll 4
        for (int x = lane; x < kAttTile * V; x += 32) {
            const int line = x / V, v = x - line * V;
            const int64_t from = __shfl_sync(0xffffffffu, mine, line);
            if (boxed >> line & 1) continue;
            const uint32_t to = tile + C::place(line, v);
            cp16(to, a.c.k + (from >= 0 ? from + v * 16 : 0), from >= 0);
            cp16(to + C::kHalf, a.c.v + (from >= 0 ? from + v * 16 : 0), from >= 0);
        }
    }

    __device__ void note(const AttTokens& r, int turn, uint32_t at, bool some) {
        // (a team's last tile of a round is the one of the highest number)
        const bool end = r.last && kAttFeeds * turn + feed >= kAttFeeds * kAttTurns - C::kTeams;
        uint32_t header = (end ? kAttEnd : 0) | (some ? 0 : kAttEmpty) | (r.tree ? kAttTree : 0);
        if (some) {
            const bool ok = r.id[turn] >= 0;
            if (F8) {
                const float ve = r.ve[turn] == 255 ? NAN : (float)((int)r.ve[turn] - 127);
                st_shared(at + 8 * lane, ok ? __float_as_uint(kv_two_to(r.ke[turn])) : 0u);
                st_shared(at + 8 * lane + 4, __float_as_uint(ok ? ve : 0.0f));
            } else {
                st_shared(at + 4 * lane, !ok);
            }
            if (__any_sync(0xffffffffu, !ok)) header |= kAttShort;
            if (r.tree) {
                const unsigned long long mask = ok ? r.mask[turn] : 0;       // (no row sees what is not there)
                st_shared(at + C::kMasks + 8 * lane, (uint32_t)mask);
                st_shared(at + C::kMasks + 8 * lane + 4, (uint32_t)(mask >> 32));
            }
        }
        if (lane == 0) st_shared(at + C::kHeader, header);
        __syncwarp();
    }

    __device__ void run() {
        // e4m3: the exponents arrive while all of a round's copies are asked for (in a short ring that would hold a tile back for the next one's place)
        constexpr bool kLate = F8 && C::kPer >= 2 * kAttTurns;
        AttTokens now, next;                                     // page ids are asked for a round, exponents a round's copies ahead
        look_up(now);
        for (bool stopped = false; now.have; now = next) {
            resolve(now);
            look_up(next);
            if (stopped) continue;                               // (the walk has meetings of the four producers)
            int at = place, asked = 0;
            uint32_t p = parity;
            // (a look at a barrier takes 200 cycles: at both places' at once)
            bool given[kAttTurns];
#pragma unroll
            for (int t = 0; t < kAttTurns; ++t) given[t] = bar_try(empty + 8 * ((place + t) % C::kPer), place + t >= C::kPer ? parity ^ 1 : parity);
#pragma unroll
            for (int t = 0; t < kAttTurns; ++t) {
                const bool here = (C::kPer >= kAttTurns && given[t]) || (!stopped && att_wait(empty + 8 * at, p, stop, a.ctrl));
                stopped = !__all_sync(0xffffffffu, here && !stopped);
                if (stopped) continue;
                if (kAttTile * (kAttFeeds * t + feed) < now.n) copy(now, t, at);
                if (!kLate) finish(now, t);
                ++asked;
                if (++at == C::kPer) at = 0, p ^= 1;
            }
#pragma unroll
            for (int t = 0; t < (kLate ? kAttTurns : 0); ++t)
                if (t < asked) finish(now, t);
        }
        // No copy is in flight when the CTA ends, also when a wait has run out: the last use of every place in the ring lands.
        for (int k = max(0, filled - C::kPer); k < filled; ++k) {
            const unsigned long long t0 = global_ns();
            while (!bar_try(full + 8 * (k % C::kPer), k / C::kPer & 1) && global_ns() - t0 < kWaitLimitNs) {}
        }
    }
    __device__ __forceinline__ void finish(const AttTokens& r, int t) {
        note(r, t, notes + place * C::kNote, kAttTile * (kAttFeeds * t + feed) < r.n);
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(full + 8 * place) : "memory");
        if (lane == 0) bar_arrive(full + 8 * place);
        ++filled;
        if (++place == C::kPer) place = 0, parity ^= 1;
    }
};

// A query row into fragments' registers or (heads over 128) shared memory: in two steps, so that the next segment's rows are on their way while
// this one's results meet.
template <int D, bool F8, int WR>
struct AttQueries {
    using C = AttCfg<D, F8, WR>;
    static constexpr int kWords = (D / 4 + 31) / 32;             // in shared memory: a warp a row, a lane has kWords times four dims
    static constexpr int kLines = (16 * WR + kAttWarps - 1) / kAttWarps;
    uint32_t f[C::kQRegs ? D / 16 : 1][4];
    uint2 w[C::kQRegs ? 1 : kLines][kWords];

    __device__ __forceinline__ static const uint16_t* row_of(const KvAttendArgs& a, const AttSegment& g, int row) {
        const int rows = a.Q * a.group, r = min(row, rows - 1), qi = kv_row_of(a, r);
        return a.q + ((int64_t)g.seq * a.Q + qi) * a.q_ld + (int64_t)(g.head * a.group + (r - qi * a.group)) * D;
    }
    __device__ __forceinline__ void fetch(const KvAttendArgs& a, const AttSegment& g, int warp, int lane) {
        const int rows = a.Q * a.group, row0 = g.group * 16 * WR, j = lane & 3;
        if (C::kQRegs) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int row = row0 + warp % WR * 16 + (lane >> 2) + 8 * r;
                const uint16_t* q = row_of(a, g, row);
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    if (!F8) {
                        f[ks][r] = row < rows ? ld_cg_u32(reinterpret_cast<const uint32_t*>(q + 16 * ks + 2 * j)) : 0u;
                        f[ks][2 + r] = row < rows ? ld_cg_u32(reinterpret_cast<const uint32_t*>(q + 16 * ks + 8 + 2 * j)) : 0u;
                    } else {                                     // dims in the order in which a word of the keys holds them
                        const uint2 x = row < rows ? ld_cg_u2(reinterpret_cast<const uint2*>(q + 16 * ks + 4 * j)) : make_uint2(0, 0);
                        f[ks][r] = x.x, f[ks][2 + r] = x.y;
                    }
                }
            }
        } else {
#pragma unroll
            for (int k = 0; k < kLines; ++k) {
                const int row = row0 + warp + k * kAttWarps;
                const uint16_t* q = row_of(a, g, row);
#pragma unroll
                for (int i = 0; i < kWords; ++i) {
                    const int c = i * 32 + lane;
                    w[k][i] = row < rows && c < D / 4 ? ld_cg_u2(reinterpret_cast<const uint2*>(q + 4 * c)) : make_uint2(0, 0);
                }
            }
        }
    }
    // ... and the factors of the warp's rows' scores
    __device__ __forceinline__ void settle(float scale_log2, float (&scale)[2], uint8_t* qs, float* s_qscale, int warp, int lane) {
        scale[0] = scale[1] = scale_log2;
        if constexpr (C::kQRegs) {
#pragma unroll
            for (int r = 0; r < (F8 ? 2 : 0); ++r) {
                uint32_t top = 0;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
                    for (int x = r; x < 4; x += 2) top = max(top, max(f[ks][x] << 16 & 0x7fff0000u, f[ks][x] & 0x7fff0000u));
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
                const int power = q_power(top);
                const float k = two_to(power);
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
                    for (int x = r; x < 4; x += 2) f[ks][x] = q_pair(f[ks][x], k);
                scale[r] *= two_to(-power);
            }
        } else {
#pragma unroll
            for (int k = 0; k < kLines; ++k) {
                const int r = warp + k * kAttWarps;
                if (r >= 16 * WR) break;
                float p = 1.0f;
                if (F8) {
                    uint32_t top = 0;
#pragma unroll
                    for (int i = 0; i < kWords; ++i)
                        top = max(max(top, max(w[k][i].x << 16 & 0x7fff0000u, w[k][i].x & 0x7fff0000u)), max(w[k][i].y << 16 & 0x7fff0000u, w[k][i].y & 0x7fff0000u));
                    top = __reduce_max_sync(0xffffffffu, top);
                    p = two_to(q_power(top));
                    if (lane == 0) s_qscale[r] = two_to(-q_power(top));
                }
#pragma unroll
                for (int i = 0; i < kWords; ++i) {
                    const int c = i * 32 + lane;
                    if (c >= D / 4) continue;
                    if (!F8) *reinterpret_cast<uint2*>(qs + r * C::kQPitch + c * 8) = w[k][i];
                    else {                                           // dims 4 j .. 4 j + 3 of 16 go to columns 2 j, 2 j + 1 and 8 + 2 j, 9 + 2 j
                        uint8_t* to = qs + r * C::kQPitch + (c >> 2) * 32 + (c & 3) * 4;
                        *reinterpret_cast<uint32_t*>(to) = q_pair(w[k][i].x, p);
                        *reinterpret_cast<uint32_t*>(to + 16) = q_pair(w[k][i].y, p);
                    }
                }
            }
            consumers_barrier();
            if (F8) scale[0] *= s_qscale[warp % WR * 16 + (lane >> 2)], scale[1] *= s_qscale[warp % WR * 16 + (lane >> 2) + 8];
        }
    }
};

template <int D, bool F8, int WR, bool HALF>
__global__ void __launch_bounds__(kAttThreads, 1)
k_kv_attend(const __grid_constant__ KvAttendArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
    using C = AttCfg<D, F8, WR>;
    extern __shared__ uint8_t raw[];                             // the ring, its tiles' notes, queries, meeting place, parents
    uint8_t* ring = raw + (-smem_u32(raw) & 1023u);
    __shared__ uint64_t s_full[C::kSlots], s_empty[C::kSlots];
    __shared__ float s_qscale[C::kQRegs ? 1 : 16 * WR];          // powers that the queries' rows were scaled by, undone in the scores
    __shared__ long long s_sum[kAttWarps + kAttFeeds];
    __shared__ long long s_at, s_u[2];
    __shared__ int s_seq;
    __shared__ AttStop s_stop;
    __shared__ AttWalk s_walk[kAttWarps];
    __shared__ AttSegment s_segment[kAttWarps];
    __shared__ long long s_first[kAttWarps];
    __shared__ int4 s_join[2];                                   // results that this CTA joins: first CTA, parts, sequence, head
    uint8_t* notes = ring + C::kSlots * C::kSlot;
    uint8_t* qs = notes + C::kSlots * C::kNote;
    float4* meet = reinterpret_cast<float4*>(qs + C::kQBytes);
    int16_t* parents = reinterpret_cast<int16_t*>(qs + C::kQBytes + C::kMeet);
    int* lens = reinterpret_cast<int*>(parents + kKvMaxNodes);   // of the first kAttLens sequences
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid < C::kSlots) {
        mbar_init(s_full + tid, 33);                             // the producer's lanes, by their copies, and its word that the rest is there
        mbar_init(s_empty + tid, WR);
    }
    if (tid == 0) s_stop.cycles = bound_cycles(kWaitLimitNs), s_stop.dead = 0, s_join[0].x = s_join[1].x = -1;
    // the caller's bound, 0 = the default: written with the host waiting for it, so it is final before any later launch (it arrives while the work
    // is dealt out)
    unsigned long long bound = 0;
    if (tid == kAttThreads - 1) bound = *reinterpret_cast<volatile unsigned long long*>(&a.ctrl->wait_ns);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    griddep_launch_dependents();
    __syncthreads();
    griddep_wait();
    const int rows = a.Q * a.group, groups = (rows + 16 * WR - 1) / (16 * WR);
    const int64_t per_unit = (int64_t)a.c.heads * groups;

    // This CTA's run of units: [walk.u, walk.u1) of all sequences' units laid end to end.  The run begins and ends where equal shares do, but
    // not within a result's first or last units: a piece that small would cost more than its tokens.
    AttWalk walk;
    long long total, ctas;
    auto snapped = [&](auto off, int units) {                    // a border's place in its sequence
        const int in = (int)(off - quotient(off, decltype(off)(units)) * units);
        return in <= kAttPairUnits + kAttSnap ? off - in : in >= units - kAttSnap ? off + (units - in) : off;
    };
    if (a.few) {
        // A few sequences, whose units times 148 fit 31 bits, are looked at by every warp for itself, a lane each: the first copy waits for this,
        // and with 64-bit numbers and two meetings of the CTA it took 1.5 us.
        const int n = lane < a.c.S ? att_len(a, lane) : 0, units = lane < a.c.S ? att_units(a, n) : 0, mine = units * (int)per_unit;
        lens[lane] = n;                                          // (every warp stores the same)
        __syncwarp();
        int incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += y;
        }
        const int all = __shfl_sync(0xffffffffu, incl, 31), parts = min((int)gridDim.x, all);
        total = all, ctas = parts;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int c = min((int)blockIdx.x + i, parts), border = (int)((uint32_t)(all * c) / (uint32_t)parts);
            int seq = __ffs(__ballot_sync(0xffffffffu, border < incl)) - 1, u = all, off = 0;
            if (seq >= 0) {
                const int from = __shfl_sync(0xffffffffu, incl - mine, seq);
                off = snapped(border - from, __shfl_sync(0xffffffffu, units, seq));
                u = from + off;
                if (off == __shfl_sync(0xffffffffu, mine, seq)) ++seq, off = 0;
            }
            if (i == 0) walk.u = u, walk.off = off, walk.seq = seq;
            else walk.u1 = u;
        }
    } else {
        const int chunk = (a.c.S + kAttThreads - 1) / kAttThreads, sa = min(tid * chunk, a.c.S), sb = min(sa + chunk, a.c.S);
        long long mine = 0;
        for (int s = sa; s < sb; ++s) {
            const int n = att_len(a, s);
            if (s < kAttLens) lens[s] = n;
            mine += att_units(a, n);
        }
        long long incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += y;
        }
        if (lane == 31) s_sum[warp] = incl;
        __syncthreads();
        long long before = incl - mine;
        total = 0;
        for (int w = 0; w < kAttWarps + kAttFeeds; ++w) {
            if (w < warp) before += s_sum[w];
            total += s_sum[w];
        }
        total *= per_unit;
        before *= per_unit;
        mine *= per_unit;
        ctas = min((long long)gridDim.x, total);
        const long long each = quotient(total, ctas);
#pragma unroll
        for (int i = 0; i < 2; ++i) {                            // (one thread's sequences hold either border)
            const int c = (int)blockIdx.x + i;                   // total * c / ctas
            const long long border = blockIdx.x < ctas ? each * c + (int)(total - each * ctas) * c / (int)ctas : total;
            if (!(border == total ? tid == 0 : border >= before && border < before + mine)) continue;
            long long u = total, off = 0;
            int s = a.c.S;
            if (border < total) {
                long long at = before, n = 0;
                int units = 0;
                for (s = sa;; ++s) {
                    units = att_units(a, s < kAttLens ? lens[s] : att_len(a, s));
                    n = units * per_unit;
                    if (s == sb - 1 || at + n > border) break;
                    at += n;
                }
                off = snapped(border - at, units);
                u = at + off;
                if (off == n) ++s, off = 0;
            }
            s_u[i] = u;
            if (i == 0) s_at = off, s_seq = s;
        }
        __syncthreads();
        walk.u = s_u[0], walk.u1 = s_u[1], walk.seq = s_seq, walk.off = s_at;
    }
    if (bound) s_stop.cycles = bound_cycles(bound);
    if (walk.u >= walk.u1) {
        if (tid == 0 && !HALF) a.meta[blockIdx.x] = make_int4(-1, 0, 0, 0);
        return;
    }

    if (warp >= kAttWarps) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kAttProducerRegs));
        const int feed = warp - kAttWarps;
        AttProducer<D, F8, WR> p{a, &k_map, &v_map, smem_u32(ring) + feed * C::kPer * C::kSlot, smem_u32(notes) + feed * C::kPer * C::kNote,
                                 smem_u32(s_full + feed * C::kPer), smem_u32(s_empty + feed * C::kPer), smem_u32(&s_stop), parents, lens, walk, {},
                                 groups, lane, feed, 0, -1, -1, -1, -1, -1};
        p.run();
        return;
    }
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kAttConsumerRegs));

    const int team = warp / WR, wr = warp % WR, j = lane & 3;
    int4 meta = make_int4(-1, 0, 0, 0);
    // the team's next tile: its producer, and its place there (two teams take those of two producers each, in turn)
    int feed = team % kAttFeeds, place = team / kAttFeeds;
    uint32_t parity = 0;
    // (where the warp is in its run lies in shared memory while tiles are at work: the registers are theirs)
    AttSegment g;
    AttQueries<D, F8, WR> q;
    s_first[warp] = walk.u;
    att_next(a, lens, groups, walk, g);
    s_segment[warp] = g, s_walk[warp] = walk;
    q.fetch(a, g, warp, lane);
    bool lost = false;                                           // one of the warp's waits has run out
    for (bool go_on = true; go_on;) {
        float scale[2];
        q.settle(a.scale_log2, scale, qs, s_qscale, warp, lane);
        const uint32_t q_smem = smem_u32(qs) + wr * 16 * C::kQPitch;

        AttAcc<D> acc;
        acc.clear();
        for (bool more = !lost; more;) {
            const int slot = feed * C::kPer + place;
            lost = !__all_sync(0xffffffffu, att_wait(smem_u32(s_full) + 8 * slot, parity, smem_u32(&s_stop), a.ctrl));
            if (lost) break;
            const uint8_t* tile = ring + slot * C::kSlot;
            const uint8_t* note = notes + slot * C::kNote;
            const uint32_t header = ld_shared(smem_u32(note) + C::kHeader);
            if (!(header & kAttEmpty)) {
                if (header & kAttTree) {
                    const int row = s_segment[warp].group * 16 * WR + wr * 16 + (lane >> 2);
                    att_tile<D, F8, WR, HALF, true>(acc, q.f, q_smem, tile, note, header & kAttShort, scale, kv_row_of(a, min(row, rows - 1)), kv_row_of(a, min(row + 8, rows - 1)));
                } else {
                    att_tile<D, F8, WR, HALF, false>(acc, q.f, q_smem, tile, note, header & kAttShort, scale, 0, 0);
                }
            }
            __syncwarp();
            if (lane == 0) bar_arrive(smem_u32(s_empty) + 8 * slot);
            if (WR == 4) feed ^= 2;
            if (WR < 4 || feed < 2) {
                place += C::kShare;
                if (place >= C::kPer) place -= C::kPer, parity ^= 1;
            }
            more = !(header & kAttEnd);
        }

        g = s_segment[warp];
        const long long at = s_first[warp];
        __syncwarp();
        {
            AttSegment after;
            walk = s_walk[warp];
            __syncwarp();
            s_first[warp] = walk.u;
            go_on = att_next(a, lens, groups, walk, after);
            s_segment[warp] = after, s_walk[warp] = walk;
            if (go_on) q.fetch(a, after, warp, lane);            // (on their way while the results meet)
        }
        const int row0 = g.group * 16 * WR, r0 = row0 + wr * 16 + (lane >> 2), r1 = r0 + 8;

        // the teams' parts meet, the upper half's with the lower half's: a lane hands its share to the lane with the same rows and dims
        // (of a short segment's teams only the first have had tokens)
        const int active = (min(max(g.token_end - g.token, g.tree ? a.N : 0), C::kTeams * C::kTile) + C::kTile - 1) / C::kTile;
        if (active > 1 || !C::kQRegs) consumers_barrier();       // (the meeting place is free, and so are the queries' rows)
        bool first_step = true;
#pragma unroll
        for (int half = C::kTeams / 2; half >= 1; half /= 2) {
            if (half >= active) continue;
            // who gives uses the place that it has read from: its own place, or in the first step that of the reader
            float4* place = meet + (team >= half && first_step ? warp - half * WR : warp) * C::kVectors * 32 + lane;
            if (team >= half && team < 2 * half) {
#pragma unroll
                for (int i = 0; i < D / 8; ++i) place[32 * i] = make_float4(acc.o[i][0], acc.o[i][1], acc.o[i][2], acc.o[i][3]);
                place[32 * (D / 8)] = make_float4(acc.m[0], acc.m[1], acc.l[0], acc.l[1]);
                if (F8) place[32 * (D / 8 + 1)] = make_float4(acc.v[0], acc.v[1], 0.0f, 0.0f);
            }
            consumers_barrier();
            if (team < half) {
                const float4* from = first_step ? place : place + half * WR * C::kVectors * 32;
                const float4 y = from[32 * (D / 8)];
                const float ym[2] = {y.x, y.y}, yl[2] = {y.z, y.w};
                float fa[2], fb[2], yv[2] = {-INFINITY, -INFINITY};
                if (F8) yv[0] = from[32 * (D / 8 + 1)].x, yv[1] = from[32 * (D / 8 + 1)].y;
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const float m = fmaxf(acc.m[r], ym[r]), v = fmaxf(acc.v[r], yv[r]);
                    fa[r] = part_weight(acc.m[r], m), fb[r] = part_weight(ym[r], m);
                    acc.m[r] = m;
                    acc.l[r] = acc.l[r] * fa[r] + yl[r] * fb[r];
                    if (F8) fa[r] = part_weight(acc.v[r], v), fb[r] = part_weight(yv[r], v);
                    acc.v[r] = v;
                }
#pragma unroll
                for (int i = 0; i < D / 8; ++i) {
                    const float4 x = from[32 * i];
                    acc.o[i][0] = acc.o[i][0] * fa[0] + x.x * fb[0], acc.o[i][1] = acc.o[i][1] * fa[0] + x.y * fb[0];
                    acc.o[i][2] = acc.o[i][2] * fa[1] + x.z * fb[1], acc.o[i][3] = acc.o[i][3] * fa[1] + x.w * fb[1];
                }
            }
            first_step = false;
        }
        const bool whole = g.count == g.units;
        // the last CTA whose run begins within this result, and the one that has its first unit (borders near a result's ends lie on them)
        const long long start = at - g.tile0;
        const int last_cta = whole ? 0 : (int)quotient((start + g.units - kAttSnap) * ctas - 1, total);
        if (!HALF && !whole && g.tile0 == 0) meta = make_int4(last_cta, g.seq, g.head, g.group);
        if (team != 0) continue;
        const bool broken = ld_shared(smem_u32(&s_stop.dead)) != 0;
        float* part = a.part + (2 * (int64_t)blockIdx.x + (g.tile0 == 0 ? 1 : 0)) * a.part_rows * kv_part_floats(D);
#pragma unroll
        for (int r = 0; r < (HALF ? 1 : 2); ++r) {
            float l = acc.l[r];
            l += __shfl_xor_sync(0xffffffffu, l, 1);
            l += __shfl_xor_sync(0xffffffffu, l, 2);
            float m = acc.m[r];
            const int row = r ? r1 : r0, qi = kv_row_of(a, row);
            if (row >= rows) continue;
            const int64_t t = (int64_t)g.seq * a.Q + qi, to = t * a.Hq + g.head * a.group + (row - qi * a.group);
            const bool blind = a.node && ld_cg_s32(a.node + t) < -1;                       // a row of no token
            if (broken) l = NAN;
            const bool none = blind || l == 0.0f;
            if (blind) m = -INFINITY, l = 0.0f;
            const float inv = whole ? 1.0f / l : 1.0f, power = F8 && whole ? exp2_fast(0.5f * (acc.v[r] - m)) : 1.0f;
            const int lr = row - row0;
            if (whole) {
                if (j == 0 && a.lse) a.lse[to] = none ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
            } else if (j == 0) {
                part[a.part_rows * D + lr] = m, part[a.part_rows * (D + 1) + lr] = l;
                if (F8) part[a.part_rows * (D + 2) + lr] = blind ? -INFINITY : acc.v[r];
            }
#pragma unroll
            for (int i = 0; i < D / 8; i += F8 ? 2 : 1) {
                float x[4];
                if (F8) x[0] = acc.o[i][2 * r], x[1] = acc.o[i + 1][2 * r], x[2] = acc.o[i][2 * r + 1], x[3] = acc.o[i + 1][2 * r + 1];
                else x[0] = acc.o[i][2 * r], x[1] = acc.o[i][2 * r + 1], x[2] = x[3] = 0.0f;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = none ? 0.0f : F8 ? x[e] * inv * power * power : x[e] * inv;       // (the power in halves: the result fits, it may not)
                const int d0 = F8 ? 8 * i + 4 * j : 8 * i + 2 * j;
                if (whole && F8) *reinterpret_cast<uint2*>(a.out + to * D + d0) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
                else if (whole) *reinterpret_cast<uint32_t*>(a.out + to * D + d0) = pack_bf16(x[0], x[1]);
                else if (F8) *reinterpret_cast<float4*>(part + lr * D + d0) = make_float4(x[0], x[1], x[2], x[3]);
                else *reinterpret_cast<float2*>(part + lr * D + d0) = make_float2(x[0], x[1]);
            }
        }
        if (HALF && !whole) {                                    // the part that arrives last joins them all, behind this CTA's run
            __threadfence();
            __syncwarp();
            if (lane == 0) {
                const int first_cta = (int)quotient((start + kAttPairUnits + kAttSnap + 1) * ctas - 1, total), parts = last_cta - first_cta + 1;
                uint32_t* ticket = a.ctrl->kv_tickets + first_cta / 4;
                const int shift = first_cta % 4 * 8;
                if ((int)(atomicAdd(ticket, 1u << shift) >> shift & 255u) == parts - 1) {
                    atomicSub(ticket, (uint32_t)parts << shift);
                    s_join[g.tile0 == 0] = make_int4(first_cta, parts, g.seq, g.head);
                }
            }
        }
    }
    if (!HALF) {
        if (tid == 0) a.meta[blockIdx.x] = meta;
        return;
    }
    consumers_barrier();
    constexpr int kVecs = D / 4, kSeats = 32 * kAttWarps / kVecs;
    float* sums = reinterpret_cast<float*>(meet + 32 * kAttWarps);
    static_assert(32 * kAttWarps * 28 <= C::kMeet, "seven numbers of a thread");
    for (int k = 0; k < 2; ++k) {
        const int4 to = s_join[k];
        if (to.x < 0) continue;
        __threadfence();                                         // (the other CTAs' parts)
        const int at_once = min(rows, kSeats), share = kSeats / at_once, seat = tid / kVecs, col = tid - seat * kVecs, which = seat / share;
        for (int r0 = 0; r0 < rows; r0 += at_once) {
            const int row = r0 + which, turn = seat - which * share;
            const bool live = which < at_once && row < rows;
            JoinSum<F8> sum;
            if (live) sum = join_sum<F8>(a, to.x, to.y, row, col, turn, share);
            meet[tid] = sum.o, sums[tid] = sum.m, sums[32 * kAttWarps + tid] = sum.l;
            if (F8) sums[64 * kAttWarps + tid] = sum.v;
            consumers_barrier();
            if (live && turn == 0) {
                for (int i = 1; i < share; ++i) {
                    const int x = tid + i * kVecs;
                    sum.add(JoinSum<F8>{meet[x], sums[x], sums[32 * kAttWarps + x], F8 ? sums[64 * kAttWarps + x] : -INFINITY});
                }
                join_store<F8>(a, to.z, to.w, row, col, sum);
            }
            consumers_barrier();                                 // (the sums have been read)
        }
    }
}

// The cache's keys or values as a map of (dim, token, head, page), boxes of `box` bytes of 16 or 32 tokens.
bool kv_map(CUtensorMap* map, const KvView& c, const uint8_t* base, bool f8, int box) {
    const MapFns& fn = map_fns();
    if (!fn.encode) return false;
    const cuuint64_t size[4] = {(cuuint64_t)c.d, (cuuint64_t)c.page, (cuuint64_t)c.heads, (cuuint64_t)c.n_pages};
    const cuuint64_t stride[3] = {(cuuint64_t)c.stride_token, (cuuint64_t)c.stride_head, (cuuint64_t)c.stride_page};
    const cuuint32_t boxes[4] = {(cuuint32_t)(f8 ? box : box / 2), (cuuint32_t)(c.page % 32 ? 16 : 32), 1, 1}, step[4] = {1, 1, 1, 1};
    return fn.encode(map, f8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<uint8_t*>(base), size, stride, boxes, step,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, box == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : box == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B,
                     CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool F8, int WR, bool HALF = false>
cudaError_t attend_go(const KvAttendArgs& a, int& ctas, cudaStream_t s) {
    using C = AttCfg<D, F8, WR>;
    static bool ready[64] = {false};                             // by device
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    auto* kernel = k_kv_attend<D, F8, WR, HALF>;
    if (!ready[dev]) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
        if (e != cudaSuccess) return e;
        ready[dev] = true;
    }
    // Encoding a map takes the host 2.5 us; a thread keeps the last cache's shape encoded and puts the addresses in
    struct Kept {
        KvView c;
        bool set;
        CUtensorMap map;
    };
    static thread_local Kept kept = {};
    CUtensorMap k_map{}, v_map{};
    if (a.c.page % 16 == 0) {                                    // (else no copy goes through a map)
        const bool same = kept.set && kept.c.page == a.c.page && kept.c.heads == a.c.heads && kept.c.n_pages == a.c.n_pages &&
                          kept.c.stride_token == a.c.stride_token && kept.c.stride_head == a.c.stride_head && kept.c.stride_page == a.c.stride_page;
        if (!same) {
            kept.set = false;                                    // (a shape that is refused leaves no map behind)
            if (!kv_map(&kept.map, a.c, a.c.k, F8, C::kBox)) return cudaErrorInvalidValue;
            kept.c = a.c, kept.set = true;
        }
        k_map = v_map = kept.map;
        if (map_fns().replace(&k_map, a.c.k) != CUDA_SUCCESS || map_fns().replace(&v_map, a.c.v) != CUDA_SUCCESS) return cudaErrorInvalidValue;
    }
    const int64_t rows = (int64_t)a.Q * a.group, groups = (rows + 16 * WR - 1) / (16 * WR);
    KvAttendArgs args = a;
    // (units of all sequences at the most, times the CTAs)
    const double most = (double)a.c.S * a.c.heads * groups * ((kv_capacity(a.c) + kAttUnit - 1) / kAttUnit + kAttPairUnits + kAttTreeUnits) * kKvMaxCtas;
    args.few = a.c.S <= 32 && most < 2147483647.0;
    int64_t grid = (int64_t)a.c.S * a.c.heads * groups * ((kv_capacity(a.c) + kAttUnit - 1) / kAttUnit);
    if (grid > num_sms()) grid = num_sms();
    if (grid > kKvMaxCtas) grid = kKvMaxCtas;
    ctas = (int)grid;
    return launch_dependent(kernel, (unsigned)grid, kAttThreads, C::kSmem, s, args, k_map, v_map);
}

template <int D, bool F8>
cudaError_t attend_rows(const KvAttendArgs& a, int& ctas, cudaStream_t s) {
    const int wr = kv_attend_warp_rows(a.Q * a.group, D);
    if constexpr (D <= 128) {
        if (kv_attend_joins(a.Q * a.group, D)) return attend_go<D, F8, 1, true>(a, ctas, s);
        if (wr == 1) return attend_go<D, F8, 1>(a, ctas, s);
        if (wr == 4) return attend_go<D, F8, 4>(a, ctas, s);
    }
    return attend_go<D, F8, 2>(a, ctas, s);
}

template <bool F8>
cudaError_t attend_any(const KvAttendArgs& a, int& ctas, cudaStream_t s) {
    switch (a.c.d) {
        case 64: return attend_rows<64, F8>(a, ctas, s);
        case 96: return attend_rows<96, F8>(a, ctas, s);
        case 128: return attend_rows<128, F8>(a, ctas, s);
        case 192: return attend_rows<192, F8>(a, ctas, s);
        default: return attend_rows<256, F8>(a, ctas, s);
    }
}

}  // namespace
}  // namespace vt
