// Attention of a few query tokens of each sequence over the quantized cache:
// online softmax (running maximum and sum), fp32 throughout.
#include "kv_internal.h"

namespace soniq {

namespace {

constexpr int kWarps = 8;

__device__ __forceinline__ int code_at(const uint8_t* src, int bits, int p) {
    const int t = p >> 2, per = 8 / bits;
    const int byte = src[4 * (t / per) + (p & 3)];
    const int u = (byte >> (bits * (t % per))) & ((1 << bits) - 1);
    return (u ^ (1 << (bits - 1))) - (1 << (bits - 1));
}

// Lane `lane`'s channels of a row: packed positions lane, lane + 32, ... of
// each group's blocks, values in x[block]; returns nothing for pad positions (0).
template <bool BF16>
__device__ __forceinline__ void row_values(const KvSide& s, int64_t row, int lane, float (&x)[8]) {
    int blk = 0;
    for (int g = 0; g < s.ng; ++g) {
        const float unit = kv_load<BF16>(s.scales[row * s.ng + g]) / (float)(1 << (s.bits[g] - 1));
        for (int b = 0; b < s.nb[g]; ++b, ++blk)
            x[blk] = unit * (float)code_at(s.codes + row * s.row_bytes + s.off[g] + 4 * s.bits[g] * b, s.bits[g], lane);
    }
}

// Channel at lane `lane` of block `blk`, -1 at a pad position.
__device__ __forceinline__ int channel_at(const KvSide& s, int head, int blk, int lane) {
    const int g = blk < s.nb[0] ? 0 : 1;
    const int p = 32 * (g ? blk - s.nb[0] : blk) + lane;
    if (g >= s.ng || p >= s.count[g]) return -1;
    return s.perm[head * s.D + (g ? s.count[0] : 0) + p];
}

// One CTA per query row; its warps take every eighth position.
template <bool BF16>
__global__ void __launch_bounds__(32 * kWarps) kv_attend_kernel(const KvGeom geo, const KvAttendArgs a) {
    __shared__ float sm_m[kWarps], sm_l[kWarps], sm_o[kWarps][kKvMaxCodes];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int qh = geo.heads * a.group;
    const int64_t r = blockIdx.x;
    const int h = (int)(r % qh), t = (int)(r / qh % a.T), b = (int)(r / qh / a.T);
    const int head = h / a.group;
    const KvSide &ks = geo.s[0], &vs = geo.s[1];
    const int kb = ks.nb[0] + ks.nb[1], vb = vs.nb[0] + vs.nb[1];
    const uint16_t* q = a.Q + b * a.q_seq_stride + t * a.q_token_stride + h * a.q_head_stride;
    float qv[8], o[8], x[8];
    for (int i = 0; i < 8; ++i) {
        const int c = i < kb ? channel_at(ks, head, i, lane) : -1;
        qv[i] = c < 0 ? 0.0f : kv_load<BF16>(q[c]);
        o[i] = x[i] = 0.0f;
    }
    const int len = a.lengths[b];
    const int64_t cap = (int64_t)a.max_pages << geo.page_shift;
    int64_t end = len < 0 ? 0 : (int64_t)len + a.T;
    if (end > cap) {
        if (threadIdx.x == 0) atomicOr(a.err, kErrKvIndex);
        end = cap;
    }
    float m = -INFINITY, l = 0.0f;
    for (int64_t p = warp; p < end; p += kWarps) {
        const int64_t d = p - len;
        if (d >= 0 && !(a.mask ? a.mask[b * a.mask_stride + (int64_t)t * a.T + d] != 0 : d <= t)) continue;
        const int page = a.table[b * a.table_stride + (p >> geo.page_shift)];
        const bool ok = page >= 0 && page < geo.n_pages;
        if (!ok && lane == 0) atomicOr(a.err, kErrKvIndex);
        const int64_t row = ((int64_t)page * geo.heads + head) * geo.page + (p & (geo.page - 1));
        float sum = 0.0f;
        if (ok) {
            row_values<BF16>(ks, row, lane, x);
            for (int i = 0; i < kb; ++i) sum += qv[i] * x[i];
        }
        for (int i = 16; i; i >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, i);
        sum *= a.scale;
        const float m_new = fmaxf(m, sum), alpha = expf(m - m_new), w = expf(sum - m_new);
        if (ok) row_values<BF16>(vs, row, lane, x);
        for (int i = 0; i < vb; ++i) o[i] = o[i] * alpha + (ok ? w * x[i] : 0.0f);
        l = l * alpha + w;
        m = m_new;
    }
    if (lane == 0) {
        sm_m[warp] = m;
        sm_l[warp] = l;
    }
    for (int i = 0; i < vb; ++i) sm_o[warp][32 * i + lane] = o[i];
    __syncthreads();
    for (int i = warp; i < vb; i += kWarps) {
        float top = -INFINITY, total = 0.0f, acc = 0.0f;
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, sm_m[w]);
        for (int w = 0; w < kWarps; ++w) {
            const float f = sm_m[w] == -INFINITY ? 0.0f : expf(sm_m[w] - top);
            total += f * sm_l[w];
            acc += f * sm_o[w][32 * i + lane];
        }
        const int c = channel_at(vs, head, i, lane);
        if (c >= 0) a.out[((int64_t)(b * a.T + t) * qh + h) * vs.D + c] = kv_round<BF16>(total > 0.0f ? acc / total : 0.0f);
    }
}

}  // namespace

int64_t kv_attend_scratch(const KvGeom&, int64_t, int64_t, int64_t) { return 0; }

cudaError_t launch_kv_attend(const KvGeom& geo, const KvAttendArgs& a, cudaStream_t st) {
    const int64_t rows = (int64_t)a.B * a.T * a.group * geo.heads;
    if (rows > 2147483647) return cudaErrorNotSupported;
    if (geo.bf16) kv_attend_kernel<true><<<(unsigned)rows, 32 * kWarps, 0, st>>>(geo, a);
    else kv_attend_kernel<false><<<(unsigned)rows, 32 * kWarps, 0, st>>>(geo, a);
    note_launch();
    return cudaGetLastError();
}

}  // namespace soniq
