// Joining the partial results of the paged attention: what the joining kernel and the attention kernel itself (few rows) share.  Part i of a
// result that begins in CTA c is the second partial result of CTA c (i = 0), then the first of CTA c + i.
#pragma once
#include "vt_kv.cuh"

namespace vt {
namespace {

__device__ __forceinline__ const float* join_part(const KvAttendArgs& a, int c, int i) {
    return a.part + (2 * (int64_t)(c + i) + (i == 0)) * a.part_rows * (a.c.d + 2);
}
__device__ __forceinline__ float4 ld_cg_f4(const float* p) {
    float4 v;
    asm volatile("ld.global.cg.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p) : "memory");
    return v;
}
// What a thread makes of its parts of a row: their maximum, and four dims of the sums against it.
struct JoinSum {
    float4 o;
    float m, l;
};
__device__ __forceinline__ float join_weight(float m, float top) {           // (a part of no token, maximum -inf, has sums of zero)
    float w = 1.0f;
    if (m != -INFINITY) asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(w) : "f"(m - top));
    return w;
}
__device__ __forceinline__ void join_add(JoinSum& s, float m, float l, const float4& o) {
    const float top = fmaxf(s.m, m), a = join_weight(s.m, top), b = join_weight(m, top);
    s.m = top;
    s.l = s.l * a + l * b;
    s.o.x = s.o.x * a + o.x * b, s.o.y = s.o.y * a + o.y * b, s.o.z = s.o.z * a + o.z * b, s.o.w = s.o.w * a + o.w * b;
}
// four dims of a row (column col) over the parts turn, turn + share, ...: six at a time, all their loads in flight
__device__ __forceinline__ JoinSum join_sum(const KvAttendArgs& a, int c, int parts, int lr, int col, int turn, int share) {
    constexpr int kAhead = 6;
    const int d = a.c.d;
    JoinSum s{make_float4(0, 0, 0, 0), -INFINITY, 0.0f};
    for (int i = turn; i < parts; i += kAhead * share) {
        float m[kAhead], l[kAhead];
        float4 o[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            m[u] = -INFINITY, l[u] = 0.0f, o[u] = make_float4(0, 0, 0, 0);
            if (i + u * share >= parts) continue;
            const float* p = join_part(a, c, i + u * share);
            m[u] = ld_cg_f32(p + (int64_t)a.part_rows * d + lr);
            l[u] = ld_cg_f32(p + (int64_t)a.part_rows * (d + 1) + lr);
            o[u] = ld_cg_f4(p + (int64_t)lr * d + 4 * col);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) join_add(s, m[u], l[u], o[u]);
    }
    return s;
}
__device__ __forceinline__ void join_store(const KvAttendArgs& a, int seq, int head, int row, int col, const JoinSum& s) {
    const float4 o = s.o;
    const float l = s.l;
    const int qi = kv_row_of(a, row);
    const int64_t to = ((int64_t)seq * a.Q + qi) * a.Hq + head * a.group + (row - qi * a.group);
    const bool none = l == 0.0f;
    const float inv = none ? 0.0f : 1.0f / l;
    const __nv_bfloat162 x = none ? __floats2bfloat162_rn(0, 0) : __floats2bfloat162_rn(o.x * inv, o.y * inv);
    const __nv_bfloat162 y = none ? __floats2bfloat162_rn(0, 0) : __floats2bfloat162_rn(o.z * inv, o.w * inv);
    *reinterpret_cast<uint2*>(a.out + to * a.c.d + 4 * col) = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
    if (col == 0 && a.lse) a.lse[to] = none ? -INFINITY : (s.m + log2f(l)) * 0.6931471805599453f;
}

}  // namespace
}  // namespace vt
