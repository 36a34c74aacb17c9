// Joins the partial results of the paged attention: a (sequence, key head, group of rows) whose tokens lay in several CTAs has one partial
// result from each, and one CTA here adds them up in the order of the tokens (so that the result does not depend on timing).
#include "vt_kv.cuh"

namespace vt {
namespace {

constexpr int kThreads = 256;
constexpr int kRowsPerCta = 16;

__device__ __forceinline__ float exp2_of(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float4 ld_cg_f4(const float* p) {
    float4 v;
    asm volatile("ld.global.cg.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p) : "memory");
    return v;
}
// weight of a part with maximum x under the common maximum m; a part of no token (maximum -inf) has l = 0 and o = 0
__device__ __forceinline__ float weight(float x, float m) { return x == -INFINITY ? 1.0f : exp2_of(x - m); }

// CTA (c, y): the result whose first part is CTA c's last, rows 16 y and on.  A thread has four dims of a row and every `gpr`-th part.
__global__ void __launch_bounds__(kThreads)
k_kv_join(const __grid_constant__ KvAttendArgs a, int warp_rows) {
    __shared__ float s_top[kRowsPerCta];
    __shared__ float4 s_o[kThreads];
    __shared__ float s_l[kThreads];
    griddep_launch_dependents();
    griddep_wait();
    const int c = blockIdx.x, tid = threadIdx.x, lane = tid & 31;
    const int last = ld_cg_s32(&a.meta[c].x);
    if (last <= c) return;
    const int seq = ld_cg_s32(&a.meta[c].y), head = ld_cg_s32(&a.meta[c].z), group = ld_cg_s32(&a.meta[c].w);
    const int rows = a.Q * a.group, row0 = group * 16 * warp_rows;
    const int lr0 = blockIdx.y * kRowsPerCta, n = min(min(rows - row0, 16 * warp_rows) - lr0, kRowsPerCta), parts = last - c + 1;
    if (n <= 0) return;
    const int d = a.c.d, vecs = d / 4;
    const int64_t size = (int64_t)a.part_rows * (d + 2);
    // part i: the second partial result of CTA c, then the first of those behind it
    auto part = [&](int i) { return a.part + (2 * (int64_t)(c + i) + (i == 0)) * size; };
    for (int r = tid >> 5; r < n; r += kThreads / 32) {
        float top = -INFINITY;
        for (int i = lane; i < parts; i += 32) top = fmaxf(top, ld_cg_f32(part(i) + (int64_t)a.part_rows * d + lr0 + r));
#pragma unroll
        for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (lane == 0) s_top[r] = top;
    }
    __syncthreads();
    const int seats = kThreads / vecs;                           // rows times shares of the parts at once
    const int gpr = n < seats ? seats / n : 1, at_once = gpr > 1 ? n : seats;
    const int seat = tid / vecs, col = tid - seat * vecs;
    for (int rb = 0; rb < n; rb += at_once) {
        const int r = rb + seat / gpr, g = seat % gpr;
        const bool live = seat < at_once * gpr && r < n;
        float4 o = make_float4(0, 0, 0, 0);
        float l = 0.0f;
        if (live) {
            const float top = s_top[r];
#pragma unroll 4
            for (int i = g; i < parts; i += gpr) {
                const float* p = part(i);
                const float w = weight(ld_cg_f32(p + (int64_t)a.part_rows * d + lr0 + r), top);
                const float4 x = ld_cg_f4(p + (int64_t)(lr0 + r) * d + 4 * col);
                l += w * ld_cg_f32(p + (int64_t)a.part_rows * (d + 1) + lr0 + r);
                o.x += w * x.x, o.y += w * x.y, o.z += w * x.z, o.w += w * x.w;
            }
        }
        if (gpr > 1) {
            s_o[tid] = o, s_l[tid] = l;
            __syncthreads();
            if (live && g == 0)
                for (int i = 1; i < gpr; ++i) {
                    const float4 x = s_o[tid + i * vecs];
                    o.x += x.x, o.y += x.y, o.z += x.z, o.w += x.w;
                    l += s_l[tid + i * vecs];
                }
        }
        if (live && g == 0) {
            const int row = row0 + lr0 + r, qi = row / a.group;
            const int64_t at = ((int64_t)seq * a.Q + qi) * a.Hq + head * a.group + (row - qi * a.group);
            const bool none = l == 0.0f;
            const float inv = none ? 0.0f : 1.0f / l;
            const __nv_bfloat162 x = none ? __floats2bfloat162_rn(0, 0) : __floats2bfloat162_rn(o.x * inv, o.y * inv);
            const __nv_bfloat162 y = none ? __floats2bfloat162_rn(0, 0) : __floats2bfloat162_rn(o.z * inv, o.w * inv);
            *reinterpret_cast<uint2*>(a.out + at * d + 4 * col) = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
            if (col == 0 && a.lse) a.lse[at] = none ? -INFINITY : (s_top[r] + log2f(l)) * 0.6931471805599453f;
        }
    }
}

}  // namespace

int kv_attend_warp_rows(int rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : 4; }

static int part_rows(int rows) { return rows < 16 * kv_attend_warp_rows(rows) ? rows : 16 * kv_attend_warp_rows(rows); }

size_t kv_attend_scratch_bytes(int rows, int d) {
    const size_t parts = (size_t)kKvMaxCtas * 2 * ((part_rows(rows) + 3) & ~3) * (d + 2) * sizeof(float);
    return align_up(kKvMaxCtas * sizeof(int4), 256) + parts;
}

void kv_attend_carve(KvAttendArgs& a, uint8_t* scratch) {
    a.meta = reinterpret_cast<int4*>(scratch);
    a.part = reinterpret_cast<float*>(scratch + align_up(kKvMaxCtas * sizeof(int4), 256));
    a.part_rows = (part_rows(a.Q * a.group) + 3) & ~3;           // (a part is a whole number of 16-byte vectors)
}

cudaError_t launch_kv_attend(const KvAttendArgs& a, cudaStream_t s) {
    int ctas = 0;
    const cudaError_t e = a.c.k_exp ? launch_kv_attend_e4m3(a, ctas, s) : launch_kv_attend_bf16(a, ctas, s);
    if (e != cudaSuccess) return e;
    const int wr = kv_attend_warp_rows(a.Q * a.group);
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)ctas, (unsigned)((a.part_rows + kRowsPerCta - 1) / kRowsPerCta));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = s;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    count_launch();
    return cudaLaunchKernelEx(&cfg, k_kv_join, a, wr);
}

}  // namespace vt
