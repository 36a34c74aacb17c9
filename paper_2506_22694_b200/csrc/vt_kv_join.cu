// Joins the partial results of the paged attention where the attention kernel does not (over eight rows a key head): a (sequence, key head, group of rows) whose tokens lay in several CTAs has one partial
// result from each, which are added up in the order of the tokens (so that the result does not depend on timing).
//
// Latency-bound: a result of 37 parts is 20 KB a row, but a chain of loads for one thread.  The rows of all joined results are dealt out as
// tasks to a fixed grid (each CTA finds them in the list that the attention kernel left, one load and one scan), and a CTA's threads
// share a task's parts.
#include "vt_kv_join.cuh"

namespace vt {
namespace {

constexpr int kThreads = 256;

// A thread has four dims of a row and every `share`-th part.
template <bool F8>
__global__ void __launch_bounds__(kThreads)
k_kv_join(const __grid_constant__ KvAttendArgs a, int warp_rows, int ctas) {
    __shared__ int s_first[kKvMaxCtas];                          // CTA with the first part of each joined result, in order
    __shared__ int s_count[kThreads / 32];
    __shared__ float4 s_o[kThreads];
    __shared__ float s_m[kThreads], s_l[kThreads], s_v[F8 ? kThreads : 1];
    griddep_launch_dependents();
    griddep_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int kEach = (kKvMaxCtas + kThreads - 1) / kThreads;
    int mine = 0;
    bool joins[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {                            // thread t: CTAs kEach * t and on
        const int c = kEach * tid + i;
        joins[i] = c < ctas && ld_cg_s32(&a.meta[c].x) > c;
        mine += joins[i];
    }
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
    }
    if (lane == 31) s_count[warp] = incl;
    __syncthreads();
    int results = 0, at = incl - mine;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) at += s_count[w];
        results += s_count[w];
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (joins[i]) s_first[at++] = kEach * tid + i;
    __syncthreads();
    const int group_rows = min(a.Q * a.group, 16 * warp_rows), d = a.c.d, vecs = d / 4, seats = kThreads / vecs;
    const int tasks = results * group_rows, each = (tasks + (int)gridDim.x - 1) / (int)gridDim.x;
    const int at_once = min(each, seats), share = at_once ? seats / at_once : 1;
    const int seat = tid / vecs, col = tid - seat * vecs, which = seat / share, turn = seat - which * share;
    for (int t0 = blockIdx.x * each; t0 < min(tasks, ((int)blockIdx.x + 1) * each); t0 += at_once) {
        const int t = t0 + which, c = t < tasks ? s_first[t / group_rows] : 0, lr = t % group_rows;
        const int last = ld_cg_s32(&a.meta[c].x), seq = ld_cg_s32(&a.meta[c].y), head = ld_cg_s32(&a.meta[c].z), group = ld_cg_s32(&a.meta[c].w);
        const int row = group * 16 * warp_rows + lr, parts = last - c + 1;
        const bool live = which < at_once && t < min(tasks, ((int)blockIdx.x + 1) * each) && row < a.Q * a.group;
        JoinSum<F8> s;
        if (live) s = join_sum<F8>(a, c, parts, lr, col, turn, share);
        s_o[tid] = s.o, s_m[tid] = s.m, s_l[tid] = s.l;
        if (F8) s_v[tid] = s.v;
        __syncthreads();
        if (live && turn == 0) {
            for (int i = 1; i < share; ++i) {
                const int x = tid + i * vecs;
                s.add(JoinSum<F8>{s_o[x], s_m[x], s_l[x], F8 ? s_v[x] : -INFINITY});
            }
            join_store<F8>(a, seq, head, row, col, s);
        }
        __syncthreads();                                         // (the sums have been read)
    }
}

}  // namespace

// (heads over 128: two always, eight teams would leave no room for a tile each)
int kv_attend_warp_rows(int rows, int d) { return d > 128 ? 2 : rows <= 16 ? 1 : rows <= 32 ? 2 : 4; }

static int part_rows(int rows, int d) { return rows < 16 * kv_attend_warp_rows(rows, d) ? rows : 16 * kv_attend_warp_rows(rows, d); }

size_t kv_attend_scratch_bytes(int rows, int d) {
    const size_t parts = (size_t)kKvMaxCtas * 2 * ((part_rows(rows, d) + 3) & ~3) * kv_part_floats(d) * sizeof(float);
    return align_up(kKvMaxCtas * sizeof(int4), 256) + parts;
}

void kv_attend_carve(KvAttendArgs& a, uint8_t* scratch) {
    a.meta = reinterpret_cast<int4*>(scratch);
    a.part = reinterpret_cast<float*>(scratch + align_up(kKvMaxCtas * sizeof(int4), 256));
    a.inv_group = 1.0f / (float)a.group;
    a.page_shift = -1;
    for (int i = 0; i < 31; ++i)
        if (a.c.page == 1 << i) a.page_shift = i;
    a.box = a.c.page % 32 == 0 ? 32 : a.c.page % 16 == 0 ? 16 : 0;
    a.part_rows = (part_rows(a.Q * a.group, a.c.d) + 3) & ~3;           // (a part is a whole number of 16-byte vectors)
}

cudaError_t launch_kv_attend(const KvAttendArgs& a, cudaStream_t s) {
    int ctas = 0;
    const cudaError_t e = a.c.k_exp ? launch_kv_attend_e4m3(a, ctas, s) : launch_kv_attend_bf16(a, ctas, s);
    if (e != cudaSuccess) return e;
    if (kv_attend_joins(a.Q * a.group, a.c.d)) return cudaSuccess;
    const int wr = kv_attend_warp_rows(a.Q * a.group, a.c.d);
    const unsigned grid = (unsigned)(2 * num_sms());
    return launch_dependent(a.c.k_exp ? k_kv_join<true> : k_kv_join<false>, grid, kThreads, 0, s, a, wr, ctas);
}

}  // namespace vt
