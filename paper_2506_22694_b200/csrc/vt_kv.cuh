// The drafter's paged key-value cache: what its kernels share (addressing, the 8-bit row format) and their launchers.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "vt_common.cuh"

namespace vt {

constexpr int kKvMaxNew = VT_KV_MAX_NEW;         // new rows of a sequence in one attention call: bits of a node's row mask
constexpr int kKvMaxNodes = VT_KV_MAX_NODES;     // nodes of a sequence's tree
constexpr int kKvMaxCtas = 160;                  // CTAs of the attention kernel (one an SM): its workspace holds two partial results of each

// A cache and its page table as the kernels take them (strides in bytes).
struct KvView {
    uint8_t *k, *v;
    uint8_t *k_exp, *v_exp;       // [n_pages, heads, page], or nullptr
    int64_t stride_page, stride_head, stride_token;
    const int32_t* pages;         // [S, max_pages], rows `pages_ld` apart
    int64_t pages_ld;
    int32_t n_pages, heads, page, d, S, max_pages;
};

inline int64_t kv_capacity(const KvView& c) { return (int64_t)c.max_pages * c.page; }

struct KvWriteArgs {
    KvView c;
    const uint16_t *q, *k, *v;    // rows (token) q_ld, k_ld, v_ld elements apart, heads side by side
    int64_t q_ld, k_ld, v_ld;
    uint16_t* q_out;              // [T, Hq, d]
    int32_t T, Hq;
    const int32_t *seq, *index, *positions;
    const int64_t* freqs;         // [rot / 2] turns a position, in units of 2^-64
    int32_t rot, interleaved;
    const uint16_t *q_weight, *k_weight;
    double eps;
    Ctrl* ctrl;
};
cudaError_t launch_qkv_write(const KvWriteArgs& a, cudaStream_t s);

struct KvReadArgs {
    KvView c;
    const int32_t *seq, *index;
    int32_t T;
    uint16_t *k_out, *v_out;      // [T, heads, d]
    Ctrl* ctrl;
};
cudaError_t launch_kv_read(const KvReadArgs& a, cudaStream_t s);

struct KvCommitArgs {
    KvView c;
    const int32_t *lens, *path, *n_accept, *nodes;
    int32_t N;
    int32_t* new_lens;
    Ctrl* ctrl;
};
cudaError_t launch_kv_commit(const KvCommitArgs& a, cudaStream_t s);

struct KvAttendArgs {
    KvView c;
    const uint16_t* q;            // [S * Q, Hq, d], rows q_ld elements apart
    int64_t q_ld;
    int32_t Q, Hq, group, N;      // rows a sequence, query heads (and those of a key head), nodes a sequence
    float inv_group;
    bool few;                     // few enough sequences and units for 32 bits and a warp
    const int32_t *lens, *node, *parent;
    int64_t parent_ld;
    int32_t page_shift, box;      // log2 of the page where it is a power of two, else -1; tokens of a tensor copy: 32, 16 or (other pages) 0
    float scale_log2;             // the scores' scale times log2(e)
    uint16_t* out;                // [S * Q, Hq, d]
    float* lse;                   // [S * Q, Hq], or nullptr
    float* part;                  // partial results: kKvMaxCtas * 2 * part_rows * kv_part_floats(d)
    int4* meta;                   // [kKvMaxCtas]
    int32_t part_rows;
    Ctrl* ctrl;
};
// Of a row of a partial result: its weighted values, the maximum and the sum of its weights, and (e4m3) what the values stand against.
__host__ __device__ constexpr int kv_part_floats(int d) { return d + 3; }
int kv_attend_warp_rows(int rows, int d);        // warps side by side over a key head's rows (1, 2 or 4 of 16 rows each)
// Whether the attention kernel joins its parts itself: up to eight rows.  The CTA whose part arrives last reads them all, 40 KB for four rows and 19
// parts; a kernel of its own, which deals more rows out to all CTAs, costs 1 to 2 us more for one token (256 tokens 10.1 us for 8.4, 701 12.6
// for 11.3, 4000 14.4 for 12.6) and 1 to 5 for a batch (64 sequences in bf16 178 us for 177, in e4m3 120 for 115).
inline bool kv_attend_joins(int rows, int d) { return rows <= 8 && d <= 128; }
size_t kv_attend_scratch_bytes(int rows, int d);
cudaError_t launch_kv_attend_bf16(const KvAttendArgs& a, int& ctas, cudaStream_t s);
cudaError_t launch_kv_attend_e4m3(const KvAttendArgs& a, int& ctas, cudaStream_t s);
void kv_attend_carve(KvAttendArgs& a, uint8_t* scratch);
cudaError_t launch_kv_attend(const KvAttendArgs& a, cudaStream_t s);

#ifdef __CUDACC__
// Byte offset of token `index` of sequence `seq` (head 0) and its row among the exponents (head 0), or false where the page table
// or the page does not reach it.
__device__ __forceinline__ bool kv_place(const KvView& c, int64_t seq, int64_t index, int64_t& at, int64_t& exp_at) {
    if (seq < 0 || seq >= c.S || index < 0 || index >= (int64_t)c.max_pages * c.page) return false;
    const uint32_t i = (uint32_t)index, p = (uint32_t)c.page;   // (max_pages * page fits 31 bits: checked by the host)
    const uint32_t slot = i / p, in = i - slot * p;
    const int32_t id = ld_cg_s32(c.pages + seq * c.pages_ld + slot);
    if ((uint32_t)id >= (uint32_t)c.n_pages) return false;
    at = (int64_t)id * c.stride_page + (int64_t)in * c.stride_token;
    exp_at = (int64_t)id * c.heads * c.page + in;
    return true;
}
// Which of a sequence's new rows row `row` of a key head belongs to: row / group, of fewer than 2^21 rows (the product is off by under half a row).
__device__ __forceinline__ int kv_row_of(const KvAttendArgs& a, int row) { return (int)(((float)row + 0.5f) * a.inv_group); }
__device__ __forceinline__ void kv_flag(Ctrl* ctrl) {
    if (ctrl) atomicOr(&ctrl->flags, (uint32_t)VT_FLAG_BAD_PAGE);
}

// 2^(b - 127) of an exponent byte; 255 marks a row that held a NaN or an infinity
__device__ __forceinline__ float kv_two_to(uint32_t b) {
    uint32_t bits = b << 23;
    if (b - 1u >= 254u) bits |= 0x400000u;       // 0: 2^-127 (a subnormal); 255: NaN
    return __uint_as_float(bits);
}
#endif

}  // namespace vt
