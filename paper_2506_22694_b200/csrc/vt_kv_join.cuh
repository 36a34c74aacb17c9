// Joining the partial results of the paged attention: what the joining kernel and the attention kernel itself (few rows) share.  Part i of a
// result that begins in CTA c is the second partial result of CTA c (i = 0), then the first of CTA c + i.
#pragma once
#include "vt_kv.cuh"

namespace vt {
namespace {

__device__ __forceinline__ const float* join_part(const KvAttendArgs& a, int c, int i) {
    return a.part + (2 * (int64_t)(c + i) + (i == 0)) * a.part_rows * kv_part_floats(a.c.d);
}
__device__ __forceinline__ float4 ld_cg_f4(const float* p) {
    float4 v;
    asm volatile("ld.global.cg.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p) : "memory");
    return v;
}
// of a part whose reference is m among others of a larger one (a part of no token, reference -inf, has sums of zero)
__device__ __forceinline__ float part_weight(float m, float top) {
    float w = 1.0f;
    if (m != -INFINITY) asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(w) : "f"(m - top));
    return w;
}
// What a thread makes of its parts of a row: their maximum, and four dims of the sums against it (e4m3: o against v).
template <bool F8>
struct JoinSum {
    float4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    float m = -INFINITY, l = 0.0f, v = -INFINITY;
    __device__ __forceinline__ void add(const JoinSum& y) {
        const float top = fmaxf(m, y.m);
        float a = part_weight(m, top), b = part_weight(y.m, top);
        m = top;
        l = l * a + y.l * b;
        if (F8) {
            const float most = fmaxf(v, y.v);
            a = part_weight(v, most), b = part_weight(y.v, most);
            v = most;
        }
        o.x = o.x * a + y.o.x * b, o.y = o.y * a + y.o.y * b, o.z = o.z * a + y.o.z * b, o.w = o.w * a + y.o.w * b;
    }
};
// four dims of a row (column col) over the parts turn, turn + share, ...: six at a time, all their loads in flight
template <bool F8>
__device__ __forceinline__ JoinSum<F8> join_sum(const KvAttendArgs& a, int c, int parts, int lr, int col, int turn, int share) {
    constexpr int kAhead = 6;
    const int d = a.c.d;
    JoinSum<F8> s;
    for (int i = turn; i < parts; i += kAhead * share) {
        JoinSum<F8> y[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i + u * share >= parts) continue;
            const float* p = join_part(a, c, i + u * share);
            y[u].m = ld_cg_f32(p + (int64_t)a.part_rows * d + lr);
            y[u].l = ld_cg_f32(p + (int64_t)a.part_rows * (d + 1) + lr);
            if (F8) y[u].v = ld_cg_f32(p + (int64_t)a.part_rows * (d + 2) + lr);
            y[u].o = ld_cg_f4(p + (int64_t)lr * d + 4 * col);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) s.add(y[u]);
    }
    return s;
}
template <bool F8>
__device__ __forceinline__ void join_store(const KvAttendArgs& a, int seq, int head, int row, int col, const JoinSum<F8>& s) {
    float4 o = s.o;
    const float l = s.l;
    const int qi = kv_row_of(a, row);
    const int64_t to = ((int64_t)seq * a.Q + qi) * a.Hq + head * a.group + (row - qi * a.group);
    const bool none = l == 0.0f;
    const float inv = none ? 0.0f : 1.0f / l;
    if (F8 && !none) {                                           // (the power in halves: the result fits, it may not)
        float power;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(power) : "f"(0.5f * (s.v - s.m)));
        o.x = o.x * inv * power * power, o.y = o.y * inv * power * power, o.z = o.z * inv * power * power, o.w = o.w * inv * power * power;
    } else {
        o.x *= inv, o.y *= inv, o.z *= inv, o.w *= inv;
    }
    const __nv_bfloat162 x = none ? __floats2bfloat162_rn(0, 0) : __floats2bfloat162_rn(o.x, o.y);
    const __nv_bfloat162 y = none ? __floats2bfloat162_rn(0, 0) : __floats2bfloat162_rn(o.z, o.w);
    *reinterpret_cast<uint2*>(a.out + to * a.c.d + 4 * col) = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
    if (col == 0 && a.lse) a.lse[to] = none ? -INFINITY : (s.m + log2f(l)) * 0.6931471805599453f;
}

}  // namespace
}  // namespace vt
