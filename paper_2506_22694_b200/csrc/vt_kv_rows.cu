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

// Two fp32 operations in one instruction: a prompt's rows are not far from being bound by the instructions that they take (4140 a token of 48
// heads with scalar operations and exact divisions: 60 us for 8.5k tokens, now 48).
typedef unsigned long long f2;
__device__ __forceinline__ f2 two(float lo, float hi) { return ((f2)__float_as_uint(hi) << 32) | __float_as_uint(lo); }
__device__ __forceinline__ float lo_of(f2 x) { return __uint_as_float((uint32_t)x); }
__device__ __forceinline__ float hi_of(f2 x) { return __uint_as_float((uint32_t)(x >> 32)); }
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
    f2 y;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(y) : "l"(a), "l"(b));
    return y;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
    f2 y;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(y) : "l"(a), "l"(b), "l"(c));
    return y;
}
struct Turn2 {                    // a Turn in pairs, and the negative sines
    f2 c[2], s[2], n[2];
};
__device__ __forceinline__ Turn2 in_pairs(const Turn<float>& t) {
    Turn2 y;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        y.c[i] = two(t.c[2 * i], t.c[2 * i + 1]);
        y.s[i] = two(t.s[2 * i], t.s[2 * i + 1]);
        y.n[i] = two(-t.s[2 * i], -t.s[2 * i + 1]);
    }
    return y;
}
__device__ __forceinline__ void unpack_pairs(const uint4& v, f2* x) {
    x[0] = two(bf_lo(v.x), bf_hi(v.x)), x[1] = two(bf_lo(v.y), bf_hi(v.y)), x[2] = two(bf_lo(v.z), bf_hi(v.z)), x[3] = two(bf_lo(v.w), bf_hi(v.w));
}
// A row of bf16 through norm and rotation, in fp32, back to bf16.  w: its weights in pairs; live: the lane holds a part of the row.
template <int LG>
__device__ __forceinline__ uint4 row_of_bf16(const uint4& raw, const f2* w, bool normed, float eps, float inv_d, bool live, const Turn2& t, bool turned, bool interleaved) {
    f2 x[4];
    unpack_pairs(raw, x);
    if (normed) {
        f2 sum = mul2(x[0], x[0]);
#pragma unroll
        for (int i = 1; i < 4; ++i) sum = fma2(x[i], x[i], sum);
        const float r = rsqrtf(fmaf(group_sum<LG>(live ? lo_of(sum) + hi_of(sum) : 0.0f), inv_d, eps));
        const f2 r2 = two(r, r);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = mul2(x[i], mul2(r2, w[i]));
    }
    if (turned && !interleaved) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const f2 lo = x[i], hi = x[2 + i];
            x[i] = fma2(hi, t.n[i], mul2(lo, t.c[i]));
            x[2 + i] = fma2(lo, t.s[i], mul2(hi, t.c[i]));
        }
    } else if (turned) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float c = i & 1 ? hi_of(t.c[i >> 1]) : lo_of(t.c[i >> 1]), s = i & 1 ? hi_of(t.s[i >> 1]) : lo_of(t.s[i >> 1]);
            const float lo = lo_of(x[i]), hi = hi_of(x[i]);
            x[i] = two(lo * c - hi * s, hi * c + lo * s);
        }
    }
    return make_uint4(bf_pack(lo_of(x[0]), hi_of(x[0])), bf_pack(lo_of(x[1]), hi_of(x[1])), bf_pack(lo_of(x[2]), hi_of(x[2])), bf_pack(lo_of(x[3]), hi_of(x[3])));
}

// The same of a row in 64 bits.
template <int LG>
__device__ __forceinline__ void norm_rotate(double* x, const uint4& w, bool normed, double eps, int d, const Turn<double>& t, int angle, bool interleaved) {
    if (normed) {
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += x[i] * x[i];
        sum = group_sum<LG>(sum);
        const double r = 1.0 / sqrt(sum / (double)d + eps);
        float wf[8];
        unpack8(w, wf);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] * r * (double)wf[i];
    }
    if (angle < 0) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        double &a = interleaved ? x[2 * i] : x[i], &b = interleaved ? x[2 * i + 1] : x[4 + i];
        const double y = a * t.c[i] - b * t.s[i];
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
// once for all of them.  Latency-bound for a token: `shares` spreads a few tokens over more warps.  8.5k tokens of 48 heads of 128 in bf16 (209 MB)
// take 48.5 us, 67% of what copying HBM reaches: the same loads and stores without the arithmetic took 42 (8 bytes a lane, a warp's stores in front
// of its next loads, a third of the seats taken), and the instructions use some 45% of the issue slots.  Into e4m3, keys in 64 bits,
// 90 us with the reading back behind it.  One token: 5 us.
template <int D>
struct Rows {
    static constexpr int kLanes = D <= 64 ? 8 : D <= 128 ? 16 : 32, kHeads = 32 / kLanes, kStep = kHeads * D;      // of a pass
    static constexpr bool kAll = 8 * kLanes == D;                // no lane without a part of its row
    const Groups g;
    const int hl;
    const bool live;

    __device__ __forceinline__ uint4 load(const uint16_t* row) const {
        const uint2 lo = ld_once_u2(row + g.a), hi = ld_once_u2(row + g.b);
        return make_uint4(lo.x, lo.y, hi.x, hi.y);
    }
    __device__ __forceinline__ void store(uint16_t* row, const uint4& x) const {
        *reinterpret_cast<uint2*>(row + g.a) = make_uint2(x.x, x.y);
        *reinterpret_cast<uint2*>(row + g.b) = make_uint2(x.z, x.w);
    }
    __device__ __forceinline__ void store8(uint8_t* row, const uint2& x) const {
        *reinterpret_cast<uint32_t*>(row + g.a) = x.x;
        *reinterpret_cast<uint32_t*>(row + g.b) = x.y;
    }
    // passes [p, end) over a token's rows, N in flight: body(row, head, whether there is such a head for this lane)
    template <int N, class Start, class Body>
    __device__ __forceinline__ void passes(const uint16_t* rows, int heads, int p, int end, Start start, Body body) const {
        bool begun = false;
        for (; p < end; p += N) {
            const uint16_t* from = rows + p * kStep + hl * D;
            uint4 raw[N];
            const bool full = p + N <= end && (p + N) * kHeads <= heads;
#pragma unroll
            for (int u = 0; u < N; ++u) {
                raw[u] = make_uint4(0, 0, 0, 0);
                if (full || (p + u < end && (p + u) * kHeads + hl < heads)) raw[u] = load(from + u * kStep);
            }
            if (!begun) start();                                 // (while the first rows are on their way)
            begun = true;
#pragma unroll
            for (int u = 0; u < N; ++u)
                if (full || p + u < end) body(raw[u], (p + u) * kHeads + hl, (kAll || live) && (full || (p + u) * kHeads + hl < heads));
        }
    }
};

template <int D, bool E4M3>
__global__ void __launch_bounds__(kThreads, 3)
k_qkv_write(const __grid_constant__ KvWriteArgs a, int shares) {
    griddep_launch_dependents();
    griddep_wait();
    using R = Rows<D>;
    constexpr int LG = R::kLanes, HP = R::kHeads;
    const int lane = threadIdx.x & 31, sub = lane % LG;
    const bool live = 8 * sub < D, inter = a.interleaved;
    // (a lane without a part of the row goes along with the first)
    const R rows{live ? groups_of(sub, a.rot, a.interleaved) : Groups{0, 4, -1}, lane / LG, live};
    const int angle = a.freqs ? rows.g.angle : -1;
    const int q_passes = (a.Hq + HP - 1) / HP, k_passes = (a.c.heads + HP - 1) / HP, passes = q_passes + 2 * k_passes;
    const int64_t warps = (int64_t)gridDim.x * kWarps, all = (int64_t)a.T * shares;
    const bool q_normed = a.q_weight != nullptr, k_normed = a.k_weight != nullptr;
    const uint4 none = make_uint4(0, 0, 0, 0), wq = q_normed ? rows.load(a.q_weight) : none, wk = k_normed ? rows.load(a.k_weight) : none;
    const float eps = (float)a.eps, inv_d = 1.0f / (float)D;
    for (int64_t item = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); item < all; item += warps) {
        const int64_t t = shares == 1 ? item : item / shares;
        const int share = (int)(item - t * shares);
        const int p0 = passes * share / shares, p1 = passes * (share + 1) / shares;
        const int q_end = min(p1, q_passes), k_begin = max(p0, q_passes), k_end = min(p1, q_passes + k_passes), v_begin = max(p0, q_passes + k_passes);
        const bool keys = p1 > q_passes;
        const int32_t pos = a.freqs ? ld_cg_s32(a.positions + t) : 0;
        const int32_t index = keys ? ld_cg_s32(a.index + t) : -1;
        const int64_t seq = !keys ? 0 : a.seq ? (int64_t)ld_cg_s32(a.seq + t) : t / (a.T / a.c.S);
        int64_t at = 0, exp_at = 0;
        bool place = false, placed = false;
        auto find = [&] {
            if (placed) return;
            placed = true;
            if (index < 0) return;
            place = kv_place(a.c, seq, index, at, exp_at);
            if (!place && lane == 0) kv_flag(a.ctrl);
        };
        Turn2 turn;
        bool turned = false;
        auto sines = [&] {
            if (turned) return;
            turned = true;
            Turn<float> angles;
            make_turn(angles, a.freqs, angle, pos);
            turn = in_pairs(angles);
        };
        if (p0 < q_end) {
            uint16_t* out = a.q_out + t * a.Hq * D;
            f2 w[4];
            unpack_pairs(wq, w);
            rows.template passes<4>(a.q + t * a.q_ld, a.Hq, p0, q_end, sines, [&](const uint4& row, int h, bool here) {
                const uint4 y = row_of_bf16<LG>(row, w, q_normed, eps, inv_d, R::kAll || live, turn, angle >= 0, inter);
                if (here) rows.store(out + h * D, y);
            });
        }
        if (k_begin < k_end && !E4M3) {
            f2 w[4];
            unpack_pairs(wk, w);
            rows.template passes<4>(a.k + t * a.k_ld, a.c.heads, k_begin - q_passes, k_end - q_passes, [&] { sines(); find(); }, [&](const uint4& row, int h, bool here) {
                const uint4 y = row_of_bf16<LG>(row, w, k_normed, eps, inv_d, R::kAll || live, turn, angle >= 0, inter);
                if (here && place) rows.store(reinterpret_cast<uint16_t*>(a.c.k + at + h * a.c.stride_head), y);
            });
        }
        if (k_begin < k_end && E4M3) {
            // Keys that are rounded to 8 bits are computed in 64: a key next to a border between two e4m3 values then falls to the right
            // side, so that the cache's bytes do not depend on the order of sums.
            Turn<double> exact;
            rows.template passes<1>(a.k + t * a.k_ld, a.c.heads, k_begin - q_passes, k_end - q_passes, [&] { make_turn(exact, a.freqs, angle, pos); find(); },
                                    [&](const uint4& row, int h, bool here) {
                float f[8];
                double x[8];
                unpack8(row, f);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = R::kAll || live ? f[i] : 0.0f;
                norm_rotate<LG>(x, wk, k_normed, a.eps, D, exact, angle, inter);
                uint32_t e;
                const uint2 y = to_e4m3<LG>(x, e);
                if (here && place) {
                    rows.store8(a.c.k + at + h * a.c.stride_head, y);
                    if (sub == 0) a.c.k_exp[exp_at + (int64_t)h * a.c.page] = (uint8_t)e;
                }
            });
        }
        if (v_begin < p1)
            rows.template passes<4>(a.v + t * a.v_ld, a.c.heads, v_begin - q_passes - k_passes, p1 - q_passes - k_passes, find, [&](const uint4& row, int h, bool here) {
                if (!E4M3) {
                    if (here && place) rows.store(reinterpret_cast<uint16_t*>(a.c.v + at + h * a.c.stride_head), row);
                    return;
                }
                float x[8];
                unpack8(row, x);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = R::kAll || live ? x[i] : 0.0f;
                uint32_t e;
                const uint2 y = to_e4m3<LG>(x, e);
                if (here && place) {
                    rows.store8(a.c.v + at + h * a.c.stride_head, y);
                    if (sub == 0) a.c.v_exp[exp_at + (int64_t)h * a.c.page] = (uint8_t)e;
                }
            });
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

// A warp a token, two passes (of 32 / LG heads) of its keys and of its values in flight.  HBM-bound, and more warps do better than more rows in
// flight of each: 122k tokens of eight e4m3 heads of 128 (526 MB) took 112 us with four passes and two CTAs an SM, 99 with two passes and four, and
// take 92 with a warp a token (87% of what copying HBM reaches).
template <int LG, bool E4M3>
__global__ void __launch_bounds__(kThreads, 4)
k_kv_read(const __grid_constant__ KvReadArgs a) {
    griddep_launch_dependents();
    griddep_wait();
    constexpr int HP = 32 / LG;
    const int lane = threadIdx.x & 31, sub = lane % LG, hl = lane / LG, dim = sub * 8, d = a.c.d;
    const bool live = dim < d;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    const int64_t t = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (t < a.T) {
        const int32_t index = ld_cg_s32(a.index + t);
        int64_t at = 0, exp_at = 0;
        bool have = false;
        if (index >= 0) {
            have = kv_place(a.c, a.seq ? (int64_t)ld_cg_s32(a.seq + t) : t / (a.T / a.c.S), index, at, exp_at);
            if (!have && lane == 0) kv_flag(a.ctrl);
        }
        for (int h0 = hl; h0 - hl < a.c.heads; h0 += 2 * HP) {
            uint4 r[4];
            uint2 w[4];
            float f[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {                        // u < 2: keys, else values
                const int h = h0 + (u & 1) * HP;
                const uint8_t* from = (u < 2 ? a.c.k : a.c.v) + at + h * a.c.stride_head;
                const bool here = have && live && h < a.c.heads;
                if (!E4M3) r[u] = here ? ld_once_u4(from + 2 * dim) : zero;
                else {
                    w[u] = here ? ld_once_u2(from + dim) : make_uint2(0, 0);
                    f[u] = here ? kv_two_to(ld_cg_u8((u < 2 ? a.c.k_exp : a.c.v_exp) + exp_at + (int64_t)h * a.c.page)) : 0.0f;
                }
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int h = h0 + (u & 1) * HP;
                if (live && h < a.c.heads)
                    st_stream_u4((u < 2 ? a.k_out : a.v_out) + (t * a.c.heads + h) * d + dim, E4M3 ? from_e4m3(w[u], f[u]) : r[u]);
            }
        }
    }
}

// ---- commit -----------------------------------------------------------------------------------------------------
// The accepted nodes' rows move to the places behind the committed tokens: place len + i takes the row at len + node(i).  A path's
// nodes rise, so node(i) >= i: a place is read before it is written when a thread, which owns the same 16 bytes of every row, reads
// up to eight rows before it writes them, path in order.  One CTA a sequence; latency-bound: 4.3 us for one path, 5.8 for 256.
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
    const bool bad = len < 0 || len > room || n < 0 || n > a.N || (int64_t)len + n > room;
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

template <int D>
cudaError_t write_go(const KvWriteArgs& a, cudaStream_t s) {
    constexpr int HP = Rows<D>::kHeads;
    const int passes = (a.Hq + HP - 1) / HP + 2 * ((a.c.heads + HP - 1) / HP);
    const int64_t most = 3 * (int64_t)num_sms();                 // three CTAs an SM: as many warps as its registers hold
    // few tokens: their heads are dealt to as many warps as there are seats, one pass each at the least
    int64_t shares = most * kWarps / a.T;
    if (shares > passes) shares = passes;
    if (shares < 1) shares = 1;
    const int64_t ctas = (a.T * shares + kWarps - 1) / kWarps;
    const unsigned grid = (unsigned)(ctas < most ? ctas : most);
    if (a.c.k_exp) return launch_dependent(k_qkv_write<D, true>, grid, kThreads, 0, s, a, (int)shares);
    return launch_dependent(k_qkv_write<D, false>, grid, kThreads, 0, s, a, (int)shares);
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
struct Read {
    static cudaError_t go(const KvReadArgs& a, cudaStream_t s) {
        return launch_dependent(k_kv_read<LG, E>, (unsigned)(((int64_t)a.T + kWarps - 1) / kWarps), kThreads, 0, s, a);
    }
};

}  // namespace

cudaError_t launch_qkv_write(const KvWriteArgs& a, cudaStream_t s) {
    if (!a.T) return cudaSuccess;
    switch (a.c.d) {
        case 64: return write_go<64>(a, s);
        case 96: return write_go<96>(a, s);
        case 128: return write_go<128>(a, s);
        case 192: return write_go<192>(a, s);
        default: return write_go<256>(a, s);
    }
}
cudaError_t launch_kv_read(const KvReadArgs& a, cudaStream_t s) { return a.T ? by_shape<Read>(a, s) : cudaSuccess; }
cudaError_t launch_kv_commit(const KvCommitArgs& a, cudaStream_t s) {
    return launch_dependent(k_kv_commit, (unsigned)a.c.S, kThreads, 0, s, a);
}

}  // namespace vt
