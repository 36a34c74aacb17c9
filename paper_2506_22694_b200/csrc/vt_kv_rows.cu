// Rows of the drafter's key-value cache: written behind the projections (norms and rotation on the way), read back, and moved when a
// drafted path is accepted.  (The paper leaves the drafter's body to its models; Algorithm 2's drafter forward runs it.)
//
//   x' = x * rsqrt(mean(x^2) + eps) * w          per head, queries and keys, where a weight is given
//   (a, b) -> (a cos - b sin, b cos + a sin)     the pairs of the first `rot` dims, by position * frequency
//
// An 8-bit row is e4m3 under one power of two 2^e, the smallest that brings the row's largest magnitude to at most 448.  e4m3 is a
// floating format, so a power of two costs none of its three mantissa bits, and scaling by it is exact in both directions:
// the stored bytes are the correctly rounded ones, and reading a row back into bf16 rounds nothing.
#include "vt_kv.cuh"

namespace vt {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

__device__ __forceinline__ float bf_lo(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float bf_hi(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }
__device__ __forceinline__ uint32_t bf_pack(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void unpack8(const uint4& v, float* x) {
    x[0] = bf_lo(v.x), x[1] = bf_hi(v.x), x[2] = bf_lo(v.y), x[3] = bf_hi(v.y);
    x[4] = bf_lo(v.z), x[5] = bf_hi(v.z), x[6] = bf_lo(v.w), x[7] = bf_hi(v.w);
}
__device__ __forceinline__ uint4 pack8(const float* x) {
    return make_uint4(bf_pack(x[0], x[1]), bf_pack(x[2], x[3]), bf_pack(x[4], x[5]), bf_pack(x[6], x[7]));
}
__device__ __forceinline__ uint4 ld_cg_u4(const void* p) {
    uint4 v;
    asm volatile("ld.global.cg.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint2 ld_once_u2(const void* p) {
    uint2 v;
    asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t ld_cg_u8(const uint8_t* p) {
    uint32_t v;
    asm volatile("ld.global.cg.u8 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}

// ---- the row's arithmetic, in float or (keys that are rounded to 8 bits) in double ---------------------------------
// LG lanes hold a head's row, a lane two groups of four neighbouring dims.  They are the partners of each other's rotation: dims i and i + rot/2
// (dims behind the rotated ones and interleaved pairs: two neighbouring groups), so that a lane makes four sines a token and hands nothing over.
struct Groups {
    int a, b;                     // first dims of the two
    int angle;                    // frequency of the first pair, or -1: no rotation
};
__device__ __forceinline__ Groups groups_of(int sub, int rot, int interleaved) {
    if (interleaved || 8 * sub >= rot) return {8 * sub, 8 * sub + 4, interleaved && 8 * sub < rot ? 4 * sub : -1};
    return {4 * sub, 4 * sub + (rot >> 1), 4 * sub};
}

template <class F>
struct Turn {                     // cosines and sines of a lane's four pairs
    F c[4], s[4];
};

__device__ __forceinline__ void sin_cos_turns(int64_t turns, float& s, float& c) {        // turns: in units of 2^-64
    sincospif(2.0f * ((float)(int32_t)(turns >> 32) * 0x1p-32f), &s, &c);
}
__device__ __forceinline__ void sin_cos_turns(int64_t turns, double& s, double& c) { sincospi(2.0 * ((double)turns * 0x1p-64), &s, &c); }

// Position times frequency is taken modulo one turn in whole numbers (64 bits of a turn, wrapping multiplication), which loses nothing at
// any position; a product in fp32 is off by 0.004 rad at position 100000.
template <class F>
__device__ __forceinline__ void make_turn(Turn<F>& t, const int64_t* freqs, int angle, int32_t pos) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        t.c[i] = F(1), t.s[i] = F(0);
        if (angle >= 0) sin_cos_turns((int64_t)((uint64_t)freqs[angle + i] * (uint64_t)(int64_t)pos), t.s[i], t.c[i]);
    }
}

template <int LG, class F>
__device__ __forceinline__ F group_sum(F x) {
#pragma unroll
    for (int o = LG / 2; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

template <int LG, class F>
__device__ __forceinline__ void norm_rotate(F* x, const uint4& w, bool normed, double eps, int d, const Turn<F>& t, int angle, int interleaved) {
    if (normed) {
        F sum = F(0);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += x[i] * x[i];
        sum = group_sum<LG>(sum);
        const F r = F(1) / sqrt(sum / F(d) + F(eps));
        float wf[8];
        unpack8(w, wf);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] * r * F(wf[i]);
    }
    if (angle < 0) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        F &a = interleaved ? x[2 * i] : x[i], &b = interleaved ? x[2 * i + 1] : x[4 + i];
        const F y = a * t.c[i] - b * t.s[i];
        b = b * t.c[i] + a * t.s[i];
        a = y;
    }
}

__device__ __forceinline__ float to_float_odd(float x) { return x; }
__device__ __forceinline__ float to_float_odd(double x) {        // to odd: the rounding to 8 bits behind it then sees what was cut off
    const float f = __double2float_rz(x);
    return (double)f != x ? __uint_as_float(__float_as_uint(f) | 1u) : f;
}
__device__ __forceinline__ unsigned long long abs_bits(double x) { return (unsigned long long)__double_as_longlong(x) & 0x7fffffffffffffffull; }
__device__ __forceinline__ unsigned long long abs_bits(float x) { return abs_bits((double)x); }

// Eight dims of a row as e4m3, and the row's exponent byte.
template <int LG, class F>
__device__ __forceinline__ uint2 to_e4m3(const F* x, uint32_t& exp_byte) {
    unsigned long long top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, abs_bits(x[i]));   // (magnitudes as integers: NaN and infinity are the largest)
#pragma unroll
    for (int o = LG / 2; o; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (top >= 0x7ff0000000000000ull) {
        exp_byte = 255;
        return make_uint2(0, 0);
    }
    // top = 1.m * 2^E; 448 = 1.75 * 2^8
    int e = (int)(top >> 52) - 1023 - 8 + ((top & 0xfffffffffffffull) > 0xc000000000000ull);
    e = max(e, -126);
    exp_byte = (uint32_t)(e + 127);
    const F scale = (F)__uint_as_float((uint32_t)(127 - e) << 23);
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float2 a = make_float2(to_float_odd(x[4 * i] * scale), to_float_odd(x[4 * i + 1] * scale));
        const float2 b = make_float2(to_float_odd(x[4 * i + 2] * scale), to_float_odd(x[4 * i + 3] * scale));
        w[i] = (uint32_t)__nv_cvt_float2_to_fp8x2(a, __NV_SATFINITE, __NV_E4M3) |
               ((uint32_t)__nv_cvt_float2_to_fp8x2(b, __NV_SATFINITE, __NV_E4M3) << 16);
    }
    return make_uint2(w[0], w[1]);
}

// ---- write ------------------------------------------------------------------------------------------------------
// A warp takes a share of one token's heads, 32 / LG heads at a time, queries first, then keys, then values: the token's sines are made
// once for all of them.  HBM-bound for prompts, latency-bound for a token; `shares` spreads a few tokens over more warps.
template <int LG, bool E4M3, bool INTER>
__global__ void __launch_bounds__(kThreads, E4M3 ? 3 : 4)
k_qkv_write(const __grid_constant__ KvWriteArgs a, int shares) {
    griddep_launch_dependents();
    griddep_wait();
    constexpr int HP = 32 / LG;                                  // heads of a pass
    constexpr int kAhead = 4;                                    // passes of queries in flight
    const int lane = threadIdx.x & 31, sub = lane % LG, hl = lane / LG, d = a.c.d;
    const bool live = 8 * sub < d;
    const Groups g = groups_of(sub, a.rot, INTER);
    const int q_passes = (a.Hq + HP - 1) / HP, k_passes = (a.c.heads + HP - 1) / HP, passes = q_passes + 2 * k_passes;
    const int64_t warps = (int64_t)gridDim.x * kWarps, all = (int64_t)a.T * shares;
    auto load = [&](const uint16_t* row, bool here) {
        if (!here) return make_uint4(0, 0, 0, 0);
        const uint2 lo = ld_once_u2(row + g.a), hi = ld_once_u2(row + g.b);
        return make_uint4(lo.x, lo.y, hi.x, hi.y);
    };
    auto store = [&](uint16_t* row, const uint4& x) {
        *reinterpret_cast<uint2*>(row + g.a) = make_uint2(x.x, x.y);
        *reinterpret_cast<uint2*>(row + g.b) = make_uint2(x.z, x.w);
    };
    auto store8 = [&](uint8_t* row, const uint2& x) {
        *reinterpret_cast<uint32_t*>(row + g.a) = x.x;
        *reinterpret_cast<uint32_t*>(row + g.b) = x.y;
    };
    const uint4 wq = load(a.q_weight, a.q_weight && live), wk = load(a.k_weight, a.k_weight && live);
    for (int64_t item = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); item < all; item += warps) {
        const int64_t t = item / shares;
        const int share = (int)(item - t * shares);
        const int p0 = (int)((int64_t)passes * share / shares), p1 = (int)((int64_t)passes * (share + 1) / shares);
        const int q_end = min(p1, q_passes), k_end = min(p1, q_passes + k_passes);
        const int32_t pos = a.freqs ? ld_cg_s32(a.positions + t) : 0;
        int64_t at = 0, exp_at = 0;
        bool place = false;
        if (p1 > q_passes) {
            const int32_t index = ld_cg_s32(a.index + t);
            if (index >= 0) {
                place = kv_place(a.c, a.seq ? (int64_t)ld_cg_s32(a.seq + t) : t / (a.T / a.c.S), index, at, exp_at);
                if (!place && lane == 0) kv_flag(a.ctrl);
            }
        }
        int p = p0;
        if (p < (E4M3 ? q_end : k_end)) {
            Turn<float> turn;
            uint4 raw[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) raw[u] = load(a.q + t * a.q_ld + (int64_t)((p + u) * HP + hl) * d, live && p + u < q_end && (p + u) * HP + hl < a.Hq);
            make_turn(turn, a.freqs, a.freqs ? g.angle : -1, pos);                         // (while the first rows are on their way)
            for (; p < q_end; p += kAhead) {
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    if (p + u >= q_end) break;
                    const int h = (p + u) * HP + hl, next = h + kAhead * HP;
                    float x[8];
                    unpack8(raw[u], x);
                    raw[u] = load(a.q + t * a.q_ld + (int64_t)next * d, live && p + u + kAhead < q_end && next < a.Hq);
                    norm_rotate<LG>(x, wq, a.q_weight != nullptr, a.eps, d, turn, g.angle, INTER);
                    if (live && h < a.Hq) store(a.q_out + (t * a.Hq + h) * d, pack8(x));
                }
            }
            p = max(p0, q_end);
            for (; !E4M3 && p < k_end; ++p) {                    // keys of a bf16 cache
                const int h = (p - q_passes) * HP + hl;
                const bool here = live && h < a.c.heads;
                float x[8];
                unpack8(load(a.k + t * a.k_ld + (int64_t)h * d, here), x);
                norm_rotate<LG>(x, wk, a.k_weight != nullptr, a.eps, d, turn, g.angle, INTER);
                if (here && place) store(reinterpret_cast<uint16_t*>(a.c.k + at + h * a.c.stride_head), pack8(x));
            }
        }
        if (E4M3 && p < k_end) {
            // Keys that are rounded to 8 bits are computed in 64: a key next to a border between two e4m3 values then falls to the right
            // side, so that the cache's bytes do not depend on the order of sums.
            Turn<double> turn;
            make_turn(turn, a.freqs, a.freqs ? g.angle : -1, pos);
            for (; p < k_end; ++p) {
                const int h = (p - q_passes) * HP + hl;
                const bool here = live && h < a.c.heads;
                float f[8];
                double x[8];
                unpack8(load(a.k + t * a.k_ld + (int64_t)h * d, here), f);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = f[i];
                norm_rotate<LG>(x, wk, a.k_weight != nullptr, a.eps, d, turn, g.angle, INTER);
                uint32_t e;
                const uint2 w = to_e4m3<LG>(x, e);
                if (here && place) {
                    store8(a.c.k + at + h * a.c.stride_head, w);
                    if (sub == 0) a.c.k_exp[exp_at + (int64_t)h * a.c.page] = (uint8_t)e;
                }
            }
        }
        for (; p < p1; ++p) {                                    // values
            const int h = (p - q_passes - k_passes) * HP + hl;
            const bool here = live && h < a.c.heads;
            const uint4 raw = load(a.v + t * a.v_ld + (int64_t)h * d, here);
            if (!E4M3) {
                if (here && place) store(reinterpret_cast<uint16_t*>(a.c.v + at + h * a.c.stride_head), raw);
                continue;
            }
            float x[8];
            unpack8(raw, x);
            uint32_t e;
            const uint2 w = to_e4m3<LG>(x, e);
            if (here && place) {
                store8(a.c.v + at + h * a.c.stride_head, w);
                if (sub == 0) a.c.v_exp[exp_at + (int64_t)h * a.c.page] = (uint8_t)e;
            }
        }
    }
}

// ---- read -------------------------------------------------------------------------------------------------------
__device__ __forceinline__ uint4 from_e4m3(const uint2& w, float f) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t word = i < 2 ? w.x : w.y;
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(word >> (16 * (i & 1))), __NV_E4M3);
        const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&h));
        x[2 * i] = y.x * f, x[2 * i + 1] = y.y * f;              // (exact: four significant bits and a power of two)
    }
    return pack8(x);
}

// A warp takes a token, four passes (of 32 / LG heads) of its keys and of its values in flight.  HBM-bound.
template <int LG, bool E4M3>
__global__ void __launch_bounds__(kThreads)
k_kv_read(const __grid_constant__ KvReadArgs a) {
    griddep_launch_dependents();
    griddep_wait();
    constexpr int HP = 32 / LG;
    const int lane = threadIdx.x & 31, sub = lane % LG, hl = lane / LG, dim = sub * 8, d = a.c.d;
    const bool live = dim < d;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    for (int64_t t = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); t < a.T; t += (int64_t)gridDim.x * kWarps) {
        const int32_t index = ld_cg_s32(a.index + t);
        int64_t at = 0, exp_at = 0;
        bool have = false;
        if (index >= 0) {
            have = kv_place(a.c, a.seq ? (int64_t)ld_cg_s32(a.seq + t) : t / (a.T / a.c.S), index, at, exp_at);
            if (!have && lane == 0) kv_flag(a.ctrl);
        }
        for (int h0 = hl; h0 - hl < a.c.heads; h0 += 4 * HP) {
            uint4 r[8];
            uint2 w[8];
            float f[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {                        // u < 4: keys, else values
                const int h = h0 + (u & 3) * HP;
                const uint8_t* from = (u < 4 ? a.c.k : a.c.v) + at + h * a.c.stride_head;
                const bool here = have && live && h < a.c.heads;
                if (!E4M3) r[u] = here ? ld_once_u4(from + 2 * dim) : zero;
                else {
                    w[u] = here ? ld_once_u2(from + dim) : make_uint2(0, 0);
                    f[u] = here ? kv_two_to(ld_cg_u8((u < 4 ? a.c.k_exp : a.c.v_exp) + exp_at + (int64_t)h * a.c.page)) : 0.0f;
                }
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int h = h0 + (u & 3) * HP;
                if (live && h < a.c.heads)
                    st_stream_u4((u < 4 ? a.k_out : a.v_out) + (t * a.c.heads + h) * d + dim, E4M3 ? from_e4m3(w[u], f[u]) : r[u]);
            }
        }
    }
}

// ---- commit -----------------------------------------------------------------------------------------------------
// The accepted nodes' rows move to the places behind the committed tokens: place len + i takes the row at len + node(i).  A path's
// nodes rise, so node(i) >= i: a place is read before it is written when a thread, which owns the same 16 bytes of every row, reads
// up to eight rows before it writes them, path in order.  One CTA a sequence; latency-bound.
constexpr int kCommitChunk = 128;
__global__ void __launch_bounds__(kThreads)
k_kv_commit(const __grid_constant__ KvCommitArgs a) {
    __shared__ int64_t s_src[kCommitChunk], s_dst[kCommitChunk], s_esrc[kCommitChunk], s_edst[kCommitChunk];
    griddep_launch_dependents();
    griddep_wait();
    const int64_t s = blockIdx.x;
    const bool e4m3 = a.c.k_exp != nullptr;
    int32_t len = ld_cg_s32(a.lens + s), n = ld_cg_s32(a.n_accept + s);
    const int64_t room = (int64_t)a.c.max_pages * a.c.page;
    const bool bad = len < 0 || len > room || n < 0 || n > a.N;
    if (bad) n = 0;
    __syncthreads();                                             // (new_lens may be lens: every thread has read it)
    if (threadIdx.x == 0) {
        if (bad) kv_flag(a.ctrl);
        if (a.new_lens) a.new_lens[s] = len + n;
    }
    const int vecs = a.c.d * (e4m3 ? 1 : 2) / 16;                // 16-byte vectors of a row
    const int columns = 2 * a.c.heads * vecs, exps = e4m3 ? 2 * a.c.heads : 0;
    for (int i0 = 0; i0 < n; i0 += kCommitChunk) {
        const int m = min(n - i0, kCommitChunk);
        __syncthreads();                                         // (the places of the chunk before have been used)
        for (int i = threadIdx.x; i < m; i += kThreads) {
            int32_t node = ld_cg_s32(a.path + s * a.N + i0 + i);
            if (node >= a.N) node = -1;
            if (a.nodes && node >= 0) node = ld_cg_s32(a.nodes + s * a.N + node);
            int64_t src = -1, dst = -1, esrc = 0, edst = 0;
            const bool ok = node >= i0 + i && kv_place(a.c, s, (int64_t)len + node, src, esrc) && kv_place(a.c, s, (int64_t)len + i0 + i, dst, edst);
            if (!ok) kv_flag(a.ctrl);
            s_src[i] = ok && node != i0 + i ? src : -1;          // (a row that stays is not copied)
            s_dst[i] = dst, s_esrc[i] = esrc, s_edst[i] = edst;
        }
        __syncthreads();
        for (int col = threadIdx.x; col < columns + exps; col += kThreads) {
            if (col < columns) {
                const int row = col / vecs, h = row % a.c.heads;
                uint8_t* base = (row < a.c.heads ? a.c.k : a.c.v) + h * a.c.stride_head + (int64_t)(col - row * vecs) * 16;
                for (int i = 0; i < m; i += 8) {
                    uint4 x[8];
#pragma unroll
                    for (int u = 0; u < 8; ++u)
                        if (i + u < m && s_src[i + u] >= 0) x[u] = ld_cg_u4(base + s_src[i + u]);
#pragma unroll
                    for (int u = 0; u < 8; ++u)
                        if (i + u < m && s_src[i + u] >= 0) *reinterpret_cast<uint4*>(base + s_dst[i + u]) = x[u];
                }
            } else {
                const int row = col - columns, h = row % a.c.heads;
                uint8_t* base = (row < a.c.heads ? a.c.k_exp : a.c.v_exp) + (int64_t)h * a.c.page;
                for (int i = 0; i < m; ++i)
                    if (s_src[i] >= 0) base[s_edst[i]] = (uint8_t)ld_cg_u8(base + s_esrc[i]);
            }
        }
    }
}

template <template <int, bool> class Run, class A>
cudaError_t by_shape(const A& a, cudaStream_t s) {
    const bool e = a.c.k_exp != nullptr;
    const int d = a.c.d;
    if (d <= 64) return e ? Run<8, true>::go(a, s) : Run<8, false>::go(a, s);
    if (d <= 128) return e ? Run<16, true>::go(a, s) : Run<16, false>::go(a, s);
    return e ? Run<32, true>::go(a, s) : Run<32, false>::go(a, s);
}

template <int LG, bool E>
struct Write {
    static cudaError_t go(const KvWriteArgs& a, cudaStream_t s) {
        constexpr int HP = 32 / LG;
        const int passes = (a.Hq + HP - 1) / HP + 2 * ((a.c.heads + HP - 1) / HP);
        const int64_t seats = (int64_t)num_sms() * 3 * kWarps;   // three CTAs an SM: about as many warps as its registers hold
        // few tokens: their heads are dealt to as many warps as there are seats, one pass each at the least
        int64_t shares = (2 * seats + a.T - 1) / a.T;
        if (shares > passes) shares = passes;
        const int64_t ctas = (a.T * shares + kWarps - 1) / kWarps;
        const int64_t most = (E ? 3 : 4) * (int64_t)num_sms();
        const unsigned grid = (unsigned)(ctas < most ? ctas : most);
        if (a.interleaved) return launch_dependent(k_qkv_write<LG, E, true>, grid, kThreads, 0, s, a, (int)shares);
        return launch_dependent(k_qkv_write<LG, E, false>, grid, kThreads, 0, s, a, (int)shares);
    }
};
template <int LG, bool E>
struct Read {
    static cudaError_t go(const KvReadArgs& a, cudaStream_t s) {
        const int64_t ctas = ((int64_t)a.T + kWarps - 1) / kWarps, most = 8 * (int64_t)num_sms();
        return launch_dependent(k_kv_read<LG, E>, (unsigned)(ctas < most ? ctas : most), kThreads, 0, s, a);
    }
};

}  // namespace

cudaError_t launch_qkv_write(const KvWriteArgs& a, cudaStream_t s) { return a.T ? by_shape<Write>(a, s) : cudaSuccess; }
cudaError_t launch_kv_read(const KvReadArgs& a, cudaStream_t s) { return a.T ? by_shape<Read>(a, s) : cudaSuccess; }
cudaError_t launch_kv_commit(const KvCommitArgs& a, cudaStream_t s) {
    return launch_dependent(k_kv_commit, (unsigned)a.c.S, kThreads, 0, s, a);
}

}  // namespace vt
