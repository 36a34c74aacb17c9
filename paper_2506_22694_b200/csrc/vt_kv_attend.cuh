// Attention of a sequence's new rows over its paged cache (Algorithm 2's drafter forward; the rows are a draft tree's nodes), split over the
// cache's length and joined.
//
//   o = sum_t p_t v_t / sum_t p_t,  p_t = exp(scale * q.k_t - m),  over the committed tokens t < len and, of the drafted tokens at
//   len + node, the row's node and its ancestors
//
// One pass with a running maximum; what is kept of a part (maximum m in base 2, sum l, weighted values o) joins with another part by
// m' = max, l' = l 2^(m - m') + ..., o' likewise.
//
// Bound: HBM, 2 * d * (2 or 1) bytes of a token and key head, each read once for all rows that share the head.  So rows of a key head
// (its query heads times the sequence's new rows) lie side by side as the 16 rows of an MMA, up to four such groups (WR) on warps that share
// the tiles.  mma.sync is far from its own limit at 16 and 32 rows (a token and head is two MMAs in the 22 cycles in which an SM's share of HBM
// delivers it), and it keeps scores and weights in registers, where tcgen05 would send both through TMEM for tiles of 128 rows that
// are seven eighths empty.
//
// Split: the work is cut into units of 16 * WR tokens, in the order (sequence, key head, group of rows, tokens), and every CTA takes an equal run of
// units, whatever the lengths are; nothing is known to the host, so a captured graph stays right when lengths change.  A (sequence, head, group)
// whose units lie in several CTAs leaves partial results, which a second launch joins in the order of the tokens.
//
// Teams: the CTA's four warps are 4 / WR teams.  A team has a ring of its own in shared memory, filled by cp.async, and takes every
// (4 / WR)-th unit: no barrier of the whole CTA while tokens stream.
#pragma once
#include "vt_kv.cuh"

namespace vt {
namespace {

constexpr int kAttThreads = 128;

template <int D, bool F8, int WR>
struct AttCfg {
    static constexpr int kTeams = 4 / WR;
    static constexpr int kTile = 16 * WR;                        // tokens of a unit
    static constexpr int kRow = D * (F8 ? 1 : 2);                // bytes of a cached row
    static constexpr int kPitch = kRow + 16;                     // an odd number of 16-byte vectors: ldmatrix meets no bank twice
    static constexpr int kHalf = kTile * kPitch;
    static constexpr int kStage = 2 * kHalf + (F8 ? 2 * kTile : 0);   // keys, values, their exponents
    static constexpr int kCtaStage = kTeams * kStage;            // (64 tokens, whatever WR is)
    static constexpr int kStages = F8 ? (D > 128 ? 3 : 4) : (D > 192 ? 2 : 3);
    static constexpr int kRing = kStages * kCtaStage;
    static constexpr bool kQRegs = D <= 128;                     // query fragments stay in registers
    static constexpr int kQPitch = 2 * D + 16;
    static constexpr int kQBytes = kQRegs ? 0 : WR * 16 * kQPitch;
    static constexpr int kSmem = kRing + kQBytes;
    static constexpr int kOPitch = D + 4;                        // floats of a row where the teams' results meet
    static_assert(kTeams * 16 * WR * kOPitch * 4 <= kRing, "the teams' results fit the ring");
    static_assert(kKvMaxNodes * 14 <= kRing - kCtaStage, "a tree's masks, list and parents fit behind the first stage");
    static_assert(kRow % 32 == 0 && kSmem <= 227 * 1024, "shapes");
};

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// 16 bytes, or zeros where `have` is false (then the source is not read)
__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool have) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(have ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldsm(uint32_t* r, uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm_t(uint32_t* r, uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
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

// Four e4m3 bytes as two pairs of bf16: bytes 0 and 2, bytes 1 and 3.  Sign, exponent and mantissa bits are moved to bf16's places, which
// gives the value times 2^-120 (subnormal ones too), and one exact multiplication puts it right.
__device__ __forceinline__ uint32_t times_2_120(uint32_t x) {
    uint32_t y;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(x), "r"(0x7b807b80u));
    return y;
}
__device__ __forceinline__ void e4m3_pairs(uint32_t x, uint32_t& even, uint32_t& odd) {
    even = times_2_120(((x << 8) & 0x80008000u) | ((x << 4) & 0x07f007f0u));
    odd = times_2_120((x & 0x80008000u) | ((x >> 4) & 0x07f007f0u));
}

template <int WR>
__device__ __forceinline__ void team_barrier(int team) {
    if (WR == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "n"(32 * WR) : "memory");
}

// What a warp keeps of its 16 rows: lane holds rows lane / 4 and lane / 4 + 8.
template <int D>
struct AttAcc {
    float o[D / 8][4];
    float m[2], l[2];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
        m[0] = m[1] = -INFINITY;
        l[0] = l[1] = 0.0f;
    }
};

// The first dim of accumulator tile nt's pair for a lane, and the distance between its two dims.
template <bool F8>
__device__ __forceinline__ int o_dim(int nt, int j) { return F8 ? 16 * (nt >> 1) + 4 * j + (nt & 1) : 8 * nt + 2 * j; }

// One unit: scores of the warp's 16 rows with the tile's tokens, running maximum, weighted values.  `seen`: the tile's tokens that
// exist, as bits; LIST: tokens are entries of a tree's list, and `mask` says which new rows see each.
template <int D, bool F8, int WR, bool LIST>
__device__ __forceinline__ void att_tile(AttAcc<D>& acc, const uint32_t (*qf)[4], uint32_t q_smem, uint8_t* stage, const uint64_t seen,
                                         float scale, const unsigned long long* mask, int qi0, int qi1) {
    using C = AttCfg<D, F8, WR>;
    constexpr int NT = 2 * WR;                                   // tiles of 8 tokens
    constexpr uint64_t kAll = WR == 4 ? ~0ull : (1ull << (16 * WR % 64)) - 1;
    const int lane = threadIdx.x & 31, j = lane & 3;
    float s[NT][4];
#pragma unroll
    for (int i = 0; i < NT; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.0f;
    const uint32_t base = smem_addr(stage);
    const uint32_t krow = base + ((lane >> 4) * 8 + (lane & 7)) * C::kPitch + ((lane >> 3) & 1) * 16;
    constexpr int KS = D / (F8 ? 32 : 16);                       // 32 bytes of a row at a time
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
        for (int g = 0; g < WR; ++g) {
            uint32_t b[4];
            ldsm(b, krow + g * 16 * C::kPitch + ks * 32);
            if (!F8) {
                mma(s[2 * g], qa[0], b[0], b[1]);
                mma(s[2 * g + 1], qa[0], b[2], b[3]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {                    // i: (token half, dim half)
                    uint32_t even, odd;
                    e4m3_pairs(b[i], even, odd);
                    mma(s[2 * g + (i >> 1)], qa[i & 1], even, odd);
                }
            }
        }
    }
    const uint8_t* exps = stage + 2 * C::kHalf;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        float f0 = scale, f1 = scale;
        if (F8) {
            const uint32_t e = *reinterpret_cast<const uint16_t*>(exps + 8 * i + 2 * j);
            f0 *= kv_two_to(e & 255u);
            f1 *= kv_two_to(e >> 8);
        }
        s[i][0] *= f0, s[i][1] *= f1, s[i][2] *= f0, s[i][3] *= f1;
    }
    uint32_t sees[2] = {0, 0};                                   // bit 2 i + u: the row sees token 8 i + 2 j + u
    const bool partial = LIST || seen != kAll;
    if (partial) {
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int t = 8 * i + 2 * j + u;
                const bool have = (seen >> t) & 1;
                bool r0 = have, r1 = have;
                if (LIST && have) {
                    const unsigned long long bits = mask[t];
                    r0 = (bits >> qi0) & 1, r1 = (bits >> qi1) & 1;
                }
                sees[0] |= (uint32_t)r0 << (2 * i + u), sees[1] |= (uint32_t)r1 << (2 * i + u);
                if (!r0) s[i][u] = -INFINITY;
                if (!r1) s[i][2 + u] = -INFINITY;
            }
    }
    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        top[0] = fmaxf(top[0], fmaxf(s[i][0], s[i][1]));
        top[1] = fmaxf(top[1], fmaxf(s[i][2], s[i][3]));
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 1));
        top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 2));
    }
    // The kept maximum may lie up to 4 below the true one (weights up to 16): results are divided by the sum of the same weights,
    // and most tiles need not scale what is there.
    if (__any_sync(0xffffffffu, top[0] > acc.m[0] + 4.0f || top[1] > acc.m[1] + 4.0f)) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const float m = fmaxf(acc.m[r], top[r]);
            const float f = m == acc.m[r] ? 1.0f : exp2_fast(acc.m[r] - m);
            acc.m[r] = m;
            acc.l[r] *= f;
#pragma unroll
            for (int i = 0; i < D / 8; ++i) acc.o[i][2 * r] *= f, acc.o[i][2 * r + 1] *= f;
        }
    }
    const float m0 = acc.m[0] == -INFINITY ? 0.0f : acc.m[0], m1 = acc.m[1] == -INFINITY ? 0.0f : acc.m[1];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        s[i][0] = exp2_fast(s[i][0] - m0), s[i][1] = exp2_fast(s[i][1] - m0);
        s[i][2] = exp2_fast(s[i][2] - m1), s[i][3] = exp2_fast(s[i][3] - m1);
        acc.l[0] += s[i][0] + s[i][1];
        acc.l[1] += s[i][2] + s[i][3];
        if (F8) {                                                // the values' powers of two go into the weights (exact)
            const uint32_t e = *reinterpret_cast<const uint16_t*>(exps + C::kTile + 8 * i + 2 * j);
            const float f0 = kv_two_to(e & 255u), f1 = kv_two_to(e >> 8);
            s[i][0] *= f0, s[i][1] *= f1, s[i][2] *= f0, s[i][3] *= f1;
            if (partial) {                                       // (what lies in an unseen place may be no number)
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (!((sees[u >> 1] >> (2 * i + (u & 1))) & 1)) s[i][u] = 0.0f;
            }
        }
    }
    uint8_t* vals = stage + C::kHalf;
    if (LIST && !F8) {
        // A drafted token that some of the rows see stays out of the others' sums by a weight of zero, and zero times an infinity or a NaN is
        // a NaN.  Such values are added to the rows that see them one by one, and are zeros for the MMA.
        bool odd = false;
        for (int x = lane; x < C::kTile * (D / 8); x += 32) {
            const uint4 w = *reinterpret_cast<const uint4*>(vals + (x / (D / 8)) * C::kPitch + (x % (D / 8)) * 16);
            const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) odd |= (ws[i] & 0x7f80u) == 0x7f80u || (ws[i] & 0x7f800000u) == 0x7f800000u;
        }
        if (__any_sync(0xffffffffu, odd)) {                      // (every warp of the team sees the same tile)
#pragma unroll
            for (int i = 0; i < NT; ++i)
                for (int t = 0; t < 8; t += 2) {                 // tokens t and t + 1 of the eight, from the lane that holds them
                    const int from = (lane & ~3) | (t >> 1);
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const float p0 = __shfl_sync(0xffffffffu, s[i][u], from), p1 = __shfl_sync(0xffffffffu, s[i][2 + u], from);
                        const bool r0 = (__shfl_sync(0xffffffffu, sees[0], from) >> (2 * i + u)) & 1;
                        const bool r1 = (__shfl_sync(0xffffffffu, sees[1], from) >> (2 * i + u)) & 1;
                        const uint16_t* row = reinterpret_cast<const uint16_t*>(vals + (8 * i + t + u) * C::kPitch);
#pragma unroll
                        for (int nt = 0; nt < D / 8; ++nt)
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                const uint32_t bits = row[8 * nt + 2 * j + x];
                                if ((bits & 0x7f80u) != 0x7f80u) continue;
                                const float v = __uint_as_float(bits << 16);
                                if (r0) acc.o[nt][x] += p0 * v;
                                if (r1) acc.o[nt][2 + x] += p1 * v;
                            }
                    }
                }
            team_barrier<WR>(WR == 1 ? 0 : (int)(threadIdx.x >> 5) / WR);
            for (int x = lane; x < C::kTile * D; x += 32) {      // (every warp of the team writes the same zeros)
                uint16_t* at = reinterpret_cast<uint16_t*>(vals + (x / D) * C::kPitch) + x % D;
                if ((*at & 0x7f80u) == 0x7f80u) *at = 0;
            }
            team_barrier<WR>(WR == 1 ? 0 : (int)(threadIdx.x >> 5) / WR);
        }
    }
    // Weights go into the MMA as two bf16 pieces, the rounded weight and what the rounding left (2^-17 of it at most): one piece alone would
    // add as much error as the rounding of the result, and at these rates the second MMA is free.
    const uint32_t vrow = base + C::kHalf + (((lane >> 3) & 1) * 8 + (lane & 7)) * C::kPitch + (lane >> 4) * 16;
#pragma unroll
    for (int g = 0; g < WR; ++g) {
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {                            // i: (row half, token half) of the A fragment
            const float x = s[2 * g + (i >> 1)][2 * (i & 1)], y = s[2 * g + (i >> 1)][2 * (i & 1) + 1];
            hi[i] = pack_bf16(x, y);
            lo[i] = pack_bf16(x - __uint_as_float(hi[i] << 16), y - __uint_as_float(hi[i] & 0xffff0000u));
        }
#pragma unroll
        for (int c = 0; c < C::kRow / 32; ++c) {
            uint32_t b[4];
            ldsm_t(b, vrow + g * 16 * C::kPitch + c * 32);
            if (!F8) {
                mma(acc.o[2 * c], hi, b[0], b[1]);
                mma(acc.o[2 * c + 1], hi, b[2], b[3]);
                mma(acc.o[2 * c], lo, b[0], b[1]);
                mma(acc.o[2 * c + 1], lo, b[2], b[3]);
            } else {
#pragma unroll
                for (int x = 0; x < 2; ++x) {                    // 16 dims each
                    uint32_t e0, o0, e1, o1;
                    e4m3_pairs(b[2 * x], e0, o0);
                    e4m3_pairs(b[2 * x + 1], e1, o1);
                    mma(acc.o[4 * c + 2 * x], hi, e0, e1);
                    mma(acc.o[4 * c + 2 * x + 1], hi, o0, o1);
                    mma(acc.o[4 * c + 2 * x], lo, e0, e1);
                    mma(acc.o[4 * c + 2 * x + 1], lo, o0, o1);
                }
            }
        }
    }
}

// A warp's share of a unit's copy: 16 tokens, their keys and values.  Returns which of the tokens exist.
struct AttSource {
    const KvView* c;
    int64_t seq, first;           // first: index of the list's entry 0 (tree) or 0
    int len, head;
    const uint16_t* list;         // LIST: node of each entry
    Ctrl* ctrl;
};

template <int D, bool F8, int WR, bool LIST>
__device__ __forceinline__ uint32_t att_load(const AttSource& src, uint8_t* stage, int group, int token0, int32_t page_id) {
    using C = AttCfg<D, F8, WR>;
    constexpr int V = C::kRow / 16;                              // 16-byte vectors of a row
    const KvView& c = *src.c;
    const int lane = threadIdx.x & 31;
    const uint32_t dst = smem_addr(stage) + group * 16 * C::kPitch;
    uint8_t* exps = stage + 2 * C::kHalf + group * 16;
    const int n = min(max(src.len - token0, 0), 16);
    if (!LIST && (c.page & 15) == 0) {                           // the 16 tokens lie in one page
        const bool ok = (uint32_t)page_id < (uint32_t)c.n_pages;
        const int have = ok ? n : 0;
        if (!ok && n > 0 && lane == 0) kv_flag(src.ctrl);
        const int in = token0 % c.page;
        const int64_t at = ok ? (int64_t)page_id * c.stride_page + (int64_t)in * c.stride_token + src.head * c.stride_head : 0;
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            const int x = i * 32 + lane, r = x / V, v = x % V;
            const int64_t from = at + (r < have ? r * c.stride_token : 0) + v * 16;
            cp16(dst + r * C::kPitch + v * 16, c.k + from, r < have);
            cp16(dst + C::kHalf + r * C::kPitch + v * 16, c.v + from, r < have);
        }
        if (F8 && lane < 2) {
            const int64_t e = ok ? ((int64_t)page_id * c.heads + src.head) * c.page + in : 0;
            cp16(smem_addr(exps) + lane * C::kTile, (lane ? c.v_exp : c.k_exp) + e, have > 0);
        }
        return (1u << have) - 1u;
    }
    int64_t at = 0, e = 0;
    bool ok = false;
    if (lane < n) {
        ok = kv_place(c, src.seq, src.first + (LIST ? (int64_t)src.list[token0 + lane] : (int64_t)(token0 + lane)), at, e);
        if (!ok) kv_flag(src.ctrl);
        at += src.head * c.stride_head;
    }
    if (F8 && lane < 16) {
        e += (int64_t)src.head * c.page;
        uint32_t a = 0, b = 0;
        if (ok) {
            asm volatile("ld.global.cg.u8 %0, [%1];" : "=r"(a) : "l"(c.k_exp + e) : "memory");
            asm volatile("ld.global.cg.u8 %0, [%1];" : "=r"(b) : "l"(c.v_exp + e) : "memory");
        }
        exps[lane] = (uint8_t)a, exps[C::kTile + lane] = (uint8_t)b;
    }
    const uint32_t have = __ballot_sync(0xffffffffu, ok);
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        const int x = i * 32 + lane, r = x / V, v = x % V;
        const int64_t from = __shfl_sync(0xffffffffu, at, r) + v * 16;
        cp16(dst + r * C::kPitch + v * 16, c.k + from, (have >> r) & 1);
        cp16(dst + C::kHalf + r * C::kPitch + v * 16, c.v + from, (have >> r) & 1);
    }
    return have;
}

template <int D, bool F8, int WR>
__global__ void __launch_bounds__(kAttThreads)
k_kv_attend(const __grid_constant__ KvAttendArgs a) {
    using C = AttCfg<D, F8, WR>;
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ float s_m[C::kTeams][16 * WR], s_l[C::kTeams][16 * WR];
    __shared__ uint32_t s_seen[C::kStages][4];                   // of each stage, by warp: tokens that exist
    __shared__ long long s_sum[4];
    __shared__ long long s_at;
    __shared__ int s_seq, s_warp_count[4];
    griddep_launch_dependents();
    griddep_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, team = warp / WR, wr = warp % WR, j = lane & 3;
    const int rows = a.Q * a.group, groups = (rows + 16 * WR - 1) / (16 * WR);
    const int64_t per_tile = (int64_t)a.c.heads * groups;
    const int64_t room = (int64_t)a.c.max_pages * a.c.page;
    const bool tree = a.node != nullptr;
    auto len_of = [&](int s) { return (int)min((int64_t)max(ld_cg_s32(a.lens + s), 0), room); };
    auto units_of = [&](int s) { return max((len_of(s) + C::kTile - 1) / C::kTile + (tree ? 1 : 0), 1); };

    // this CTA's run of units: [u0, u1) of all sequences' units laid end to end
    const int chunk = (a.c.S + kAttThreads - 1) / kAttThreads, sa = min(tid * chunk, a.c.S), sb = min(sa + chunk, a.c.S);
    long long mine = 0;
    for (int s = sa; s < sb; ++s) mine += units_of(s);
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
    }
    if (lane == 31) s_sum[warp] = incl;
    __syncthreads();
    long long before = incl - mine, total = 0;
    for (int w = 0; w < 4; ++w) {
        if (w < warp) before += s_sum[w];
        total += s_sum[w];
    }
    total *= per_tile;
    before *= per_tile;
    mine *= per_tile;
    // a CTA gets a unit for each team at the least
    const long long ctas = min((long long)gridDim.x, max((total + C::kTeams - 1) / C::kTeams, 1ll));
    const long long u0 = min(total * blockIdx.x / ctas, total), u1 = blockIdx.x < ctas ? total * (blockIdx.x + 1) / ctas : u0;
    if (tid == 0 && (blockIdx.x >= ctas || u0 == u1)) a.meta[blockIdx.x] = make_int4(-1, 0, 0, 0);
    if (blockIdx.x >= ctas || u0 == u1) return;
    if (u0 >= before && u0 < before + mine) {                    // one thread's sequences hold the first unit
        long long at = before;
        int s = sa;
        while (s < sb - 1 && at + units_of(s) * per_tile <= u0) at += units_of(s++) * per_tile;
        s_seq = s;
        s_at = u0 - at;
    }
    __syncthreads();
    int seq = s_seq;
    long long off = s_at, u = u0;
    int4 meta = make_int4(-1, 0, 0, 0);

    while (u < u1) {
        const int len = len_of(seq), units = units_of(seq);
        const int pair = (int)(off / units), tile0 = (int)(off - (long long)pair * units);
        const int count = (int)min((long long)(units - tile0), u1 - u);
        const int head = pair / groups, group = pair - head * groups;
        const int full = (len + C::kTile - 1) / C::kTile;        // units of committed tokens
        const int t1 = min(tile0 + count, full);
        const bool with_tree = tree && tile0 + count == units;
        const int row0 = group * 16 * WR, n_rows = min(rows - row0, 16 * WR);
        AttSource src{&a.c, seq, 0, len, head, nullptr, a.ctrl};

        // the ring's first units, then (while they come) the queries
        int issue = tile0 + team;
        auto page_of = [&](int tile) {
            const int token = tile * C::kTile + 16 * wr;
            return tile < t1 && token < len ? ld_cg_s32(a.c.pages + (int64_t)seq * a.c.pages_ld + (uint32_t)token / (uint32_t)a.c.page) : -1;
        };
        int32_t page_id = page_of(issue);
        auto fill = [&](int slot) {
            if (issue < t1) {
                const int32_t id = page_id;
                page_id = page_of(issue + C::kTeams);
                const uint32_t have = att_load<D, F8, WR, false>(src, ring + slot * C::kCtaStage + team * C::kStage, wr, issue * C::kTile + 16 * wr, id);
                if (lane == 0) s_seen[slot][warp] = have;
            }
            issue += C::kTeams;
            cp_commit();
        };
#pragma unroll
        for (int i = 0; i < C::kStages - 1; ++i) fill(i);

        uint32_t qf[C::kQRegs ? D / 16 : 1][4];
        const int r0 = row0 + wr * 16 + (lane >> 2), r1 = r0 + 8;
        const int qi0 = min(r0, rows - 1) / a.group, qi1 = min(r1, rows - 1) / a.group;
        if (C::kQRegs) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int row = r ? r1 : r0, qi = r ? qi1 : qi0;
                const uint16_t* q = a.q + ((int64_t)seq * a.Q + qi) * a.q_ld + (int64_t)(head * a.group + (min(row, rows - 1) - qi * a.group)) * D;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    if (!F8) {
                        qf[ks][r] = row < rows ? ld_cg_u32(reinterpret_cast<const uint32_t*>(q + 16 * ks + 2 * j)) : 0u;
                        qf[ks][2 + r] = row < rows ? ld_cg_u32(reinterpret_cast<const uint32_t*>(q + 16 * ks + 8 + 2 * j)) : 0u;
                    } else {                                     // dims in the order in which e4m3_pairs gives the keys'
                        const uint2 w = row < rows ? ld_cg_u2(reinterpret_cast<const uint2*>(q + 16 * ks + 4 * j)) : make_uint2(0, 0);
                        qf[ks][r] = __byte_perm(w.x, w.y, 0x5410);
                        qf[ks][2 + r] = __byte_perm(w.x, w.y, 0x7632);
                    }
                }
            }
        } else {
            uint8_t* qs = ring + C::kRing;
            for (int x = tid; x < 16 * WR * (D / 4); x += kAttThreads) {
                const int r = x / (D / 4), c = x % (D / 4), row = row0 + r, qi = min(row, rows - 1) / a.group;
                const uint2 w = row < rows ? ld_cg_u2(reinterpret_cast<const uint2*>(a.q + ((int64_t)seq * a.Q + qi) * a.q_ld +
                                                                                       (int64_t)(head * a.group + (row - qi * a.group)) * D + 4 * c))
                                           : make_uint2(0, 0);
                if (!F8) *reinterpret_cast<uint2*>(qs + r * C::kQPitch + c * 8) = w;
                else {                                           // dims 4 j .. 4 j + 3 of 16 go to columns 2 j, 2 j + 1 and 8 + 2 j, 9 + 2 j (even, odd)
                    uint8_t* at = qs + r * C::kQPitch + (c >> 2) * 32 + (c & 3) * 4;
                    *reinterpret_cast<uint32_t*>(at) = __byte_perm(w.x, w.y, 0x5410);
                    *reinterpret_cast<uint32_t*>(at + 16) = __byte_perm(w.x, w.y, 0x7632);
                }
            }
            __syncthreads();
        }
        const uint32_t q_smem = smem_addr(ring + C::kRing) + wr * 16 * C::kQPitch;

        AttAcc<D> acc;
        acc.clear();
        int slot = 0;
        for (int t = tile0 + team; t < t1; t += C::kTeams) {
            cp_wait<C::kStages - 2>();
            team_barrier<WR>(team);
            fill(slot == 0 ? C::kStages - 1 : slot - 1);
            uint64_t seen = 0;
#pragma unroll
            for (int w = 0; w < WR; ++w) seen |= (uint64_t)s_seen[slot][team * WR + w] << (16 * w);
            att_tile<D, F8, WR, false>(acc, qf, q_smem, ring + slot * C::kCtaStage + team * C::kStage, seen, a.scale_log2, nullptr, 0, 0);
            slot = slot + 1 == C::kStages ? 0 : slot + 1;
        }
        cp_wait<0>();
        __syncthreads();

        if (with_tree) {
            // which of the tree's nodes some row sees, and which rows see each: rows walk from their node to the root
            uint8_t* room_at = ring + C::kCtaStage;
            unsigned long long* mask = reinterpret_cast<unsigned long long*>(room_at);
            int* parent = reinterpret_cast<int*>(room_at + 8 * kKvMaxNodes);
            uint16_t* list = reinterpret_cast<uint16_t*>(room_at + 12 * kKvMaxNodes);
            const int N = a.N;
            for (int i = tid; i < N; i += kAttThreads) {
                mask[i] = 0;
                parent[i] = a.parent ? ld_cg_s32(a.parent + (int64_t)seq * a.parent_ld + i) : i - 1;
            }
            __syncthreads();
            if (tid < a.Q) {
                int f = ld_cg_s32(a.node + (int64_t)seq * a.Q + tid);
                if (f >= N) {
                    kv_flag(a.ctrl);
                    f = -1;
                }
                while (f >= 0) {                                 // (a parent lies in front of its child, so this ends)
                    atomicOr(&mask[f], 1ull << tid);
                    const int up = parent[f];
                    f = up < f ? up : -1;
                }
            }
            __syncthreads();
            int kept = 0;
            for (int i0 = 0; i0 < N; i0 += kAttThreads) {
                const int i = i0 + tid;
                const unsigned long long bits = i < N ? mask[i] : 0;
                const unsigned b = __ballot_sync(0xffffffffu, bits != 0);
                if (lane == 0) s_warp_count[warp] = __popc(b);
                __syncthreads();                                 // (the 128 masks have been read: the list's end is at or before them)
                int at = kept + __popc(b & lanemask_lt());
                for (int w = 0; w < 4; ++w) {
                    if (w < warp) at += s_warp_count[w];
                    kept += s_warp_count[w];
                }
                if (bits) mask[at] = bits, list[at] = (uint16_t)i;
                __syncthreads();
            }
            AttSource nodes{&a.c, seq, len, kept, head, list, a.ctrl};
            for (int t = team; t * C::kTile < kept; t += C::kTeams) {
                uint8_t* stage = ring + team * C::kStage;
                team_barrier<WR>(team);                          // (the tile before has been used)
                const uint32_t have = att_load<D, F8, WR, true>(nodes, stage, wr, t * C::kTile + 16 * wr, 0);
                if (lane == 0) s_seen[0][warp] = have;
                cp_commit();
                cp_wait<0>();
                team_barrier<WR>(team);
                uint64_t seen = 0;
#pragma unroll
                for (int w = 0; w < WR; ++w) seen |= (uint64_t)s_seen[0][team * WR + w] << (16 * w);
                att_tile<D, F8, WR, true>(acc, qf, q_smem, stage, seen, a.scale_log2, mask + t * C::kTile, qi0, qi1);
            }
            __syncthreads();
        }

        // the teams' parts meet in shared memory
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            acc.l[r] += __shfl_xor_sync(0xffffffffu, acc.l[r], 1);
            acc.l[r] += __shfl_xor_sync(0xffffffffu, acc.l[r], 2);
            if (j == 0) {
                s_m[team][wr * 16 + (lane >> 2) + 8 * r] = acc.m[r];
                s_l[team][wr * 16 + (lane >> 2) + 8 * r] = acc.l[r];
            }
        }
        __syncthreads();
        float* obuf = reinterpret_cast<float*>(ring);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int lr = wr * 16 + (lane >> 2) + 8 * r;
            float m = s_m[0][lr];
#pragma unroll
            for (int w = 1; w < C::kTeams; ++w) m = fmaxf(m, s_m[w][lr]);
            const float f = acc.m[r] == -INFINITY ? 0.0f : exp2_fast(acc.m[r] - m);
            if (lr < n_rows) {
                float* o = obuf + (team * 16 * WR + lr) * C::kOPitch;
#pragma unroll
                for (int i = 0; i < D / 8; ++i) {
                    const int d0 = o_dim<F8>(i, j);
                    const bool none = acc.m[r] == -INFINITY && acc.l[r] == 0.0f;
                    o[d0] = none ? 0.0f : acc.o[i][2 * r] * f;
                    o[d0 + (F8 ? 2 : 1)] = none ? 0.0f : acc.o[i][2 * r + 1] * f;
                }
            }
        }
        __syncthreads();
        const bool whole = count == units;
        const int slot_of = 2 * blockIdx.x + (tile0 == 0 ? 1 : 0);
        float* part = a.part + (int64_t)slot_of * a.part_rows * (D + 2);
        for (int x = tid; x < n_rows * (D / 4); x += kAttThreads) {
            const int lr = x / (D / 4), c = x % (D / 4);
            float m = s_m[0][lr], l = 0.0f;
#pragma unroll
            for (int w = 1; w < C::kTeams; ++w) m = fmaxf(m, s_m[w][lr]);
            float4 o = make_float4(0, 0, 0, 0);
#pragma unroll
            for (int w = 0; w < C::kTeams; ++w) {
                const float lw = s_l[w][lr];
                l += s_m[w][lr] == -INFINITY ? lw : lw * exp2_fast(s_m[w][lr] - m);
                const float4 y = *reinterpret_cast<const float4*>(obuf + (w * 16 * WR + lr) * C::kOPitch + 4 * c);
                o.x += y.x, o.y += y.y, o.z += y.z, o.w += y.w;
            }
            const int row = row0 + lr, qi = row / a.group;
            const int64_t t = (int64_t)seq * a.Q + qi;
            const int64_t at = t * a.Hq + head * a.group + (row - qi * a.group);
            if (tree && ld_cg_s32(a.node + t) < -1) {            // a row of no token
                m = -INFINITY, l = 0.0f;
                o = make_float4(0, 0, 0, 0);
            }
            if (whole) {
                const float inv = l == 0.0f ? 0.0f : 1.0f / l;
                const bool none = l == 0.0f;
                *reinterpret_cast<uint2*>(a.out + at * D + 4 * c) =
                    none ? make_uint2(0, 0) : make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
                if (c == 0 && a.lse) a.lse[at] = none ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
            } else {
                *reinterpret_cast<float4*>(part + lr * D + 4 * c) = o;
                if (c == 0) part[a.part_rows * D + lr] = m, part[a.part_rows * (D + 1) + lr] = l;
            }
        }
        if (!whole && tile0 == 0)                                // the last CTA with units of this (sequence, head, group)
            meta = make_int4((int)(((u + units) * ctas - 1) / total), seq, head, group);
        __syncthreads();                                         // (the ring is free again)
        u += count;
        off += count;
        if (off == units * per_tile) ++seq, off = 0;
    }
    if (tid == 0) a.meta[blockIdx.x] = meta;
}

template <int D, bool F8, int WR>
cudaError_t attend_go(const KvAttendArgs& a, int& ctas, cudaStream_t s) {
    using C = AttCfg<D, F8, WR>;
    static int per_sm[64] = {0};                                 // by device
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    auto* kernel = k_kv_attend<D, F8, WR>;
    if (!per_sm[dev]) {
        int n = 0;
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, kAttThreads, C::kSmem);
        if (e != cudaSuccess) return e;
        per_sm[dev] = n > 0 ? n : 1;
    }
    const int64_t rows = (int64_t)a.Q * a.group, groups = (rows + 16 * WR - 1) / (16 * WR);
    const int64_t most = (int64_t)a.c.S * a.c.heads * groups * ((kv_capacity(a.c) + C::kTile - 1) / C::kTile + 1);
    int64_t grid = (most + C::kTeams - 1) / C::kTeams;
    if (grid > (int64_t)num_sms() * per_sm[dev]) grid = (int64_t)num_sms() * per_sm[dev];
    if (grid > kKvMaxCtas) grid = kKvMaxCtas;
    ctas = (int)grid;
    return launch_dependent(kernel, (unsigned)grid, kAttThreads, C::kSmem, s, a);
}

template <int D, bool F8>
cudaError_t attend_rows(const KvAttendArgs& a, int& ctas, cudaStream_t s) {
    const int wr = kv_attend_warp_rows(a.Q * a.group);
    return wr == 1 ? attend_go<D, F8, 1>(a, ctas, s) : wr == 2 ? attend_go<D, F8, 2>(a, ctas, s) : attend_go<D, F8, 4>(a, ctas, s);
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
