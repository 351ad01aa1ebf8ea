// Norms of queries and keys for each head with the rotation by position in the same pass: what a prefill is scored by (keys without
// rotation), held as (keys with it) and asked with, and the rows of a decoding step.
//
//   y = x w / sqrt(mean(x^2) + eps)  (y = x without w);   a_i = position * f_i, i < R / 2;
//   (y_i, y_j) -> (y_i cos a_i - y_j sin a_i, y_j cos a_i + y_i sin a_i) with (i, j) = (i, i + R / 2) or (2 i, 2 i + 1); channels from R on stay.
//
// Bound by HBM: a row is read once and written once or twice.  16 lanes hold a row, eight channels each, and a half-warp has up to four
// rows in flight.  The angles of a token are the same for all its heads: the block works them out once, in 64 bits, because
// a far position times a frequency has more digits before the point than 32 bits leave behind it (at position 131072 the angle
// would be off by 0.004), taken to a fraction of a turn and then to 32 bits.
#include "common.cuh"
#include "rope.cuh"

namespace compactor {
namespace {

constexpr int kThreads = 256;
constexpr int kHalfWarps = kThreads / 16;
constexpr int kRows = 4;                       // rows of a half-warp in flight

__device__ __forceinline__ void unpack(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 pack(const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

__global__ void __launch_bounds__(kThreads)
rope_kernel(const __grid_constant__ RopeArgs a) {
    __shared__ __align__(16) float cosines[kRopeTokens][kD / 2], sines[kRopeTokens][kD / 2];
    const int tid = threadIdx.x, l = tid & 15, hw = tid >> 4;
    pdl_trigger();
    pdl_wait();
    const long long token0 = (long long)blockIdx.x * a.tokens_per_block;
    const int tokens = (int)min((long long)a.tokens_per_block, a.tokens - token0);
    const int per_token = a.q_heads + a.k_heads, items = tokens * per_token, half = a.rotary / 2;
    // rows of the first round are on their way while the angles are worked out
    uint4 in[kRows];
    int token[kRows], row[kRows];
    auto fetch = [&](int first) {
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const int item = min(first + u * kHalfWarps, items - 1);
            token[u] = item / per_token;
            row[u] = item - token[u] * per_token;
            const long long t = token0 + token[u];
            const __nv_bfloat16* src = row[u] < a.q_heads ? a.q + t * a.q_token + row[u] * a.q_head
                                                          : a.k + t * a.k_token + (row[u] - a.q_heads) * a.k_head;
            in[u] = *(reinterpret_cast<const uint4*>(src) + l);
        }
    };
    fetch(hw);
    float qw[8], kw[8];
    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
    unpack(a.q_weight != nullptr ? *(reinterpret_cast<const uint4*>(a.q_weight) + l) : none, qw);
    unpack(a.k_weight != nullptr ? *(reinterpret_cast<const uint4*>(a.k_weight) + l) : none, kw);
    for (int i = tid; i < tokens * half; i += kThreads) {
        const int t = i / half, f = i - t * half;
        const double turns = (double)a.positions[token0 + t] * (double)a.inv_freq[f] * 0.15915494309189533577;    // 1 / (2 pi)
        sincospif(2.f * (float)(turns - rint(turns)), &sines[t][f], &cosines[t][f]);
    }
    __syncthreads();
    const unsigned mine = 0xffffu << (tid & 16);             // the lanes of this half-warp
    for (int first = hw; first < items; first += kHalfWarps * kRows) {
        if (first != hw) fetch(first);
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            if (first + u * kHalfWarps >= items) break;
            const bool is_q = row[u] < a.q_heads;
            float x[8];
            unpack(in[u], x);
            if ((is_q ? a.q_weight : a.k_weight) != nullptr) {
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += x[i] * x[i];
#pragma unroll
                for (int d = 1; d < 16; d *= 2) sum += __shfl_xor_sync(mine, sum, d);
                const float r = rsqrtf(sum * (1.f / kD) + a.eps);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = x[i] * r * (is_q ? qw[i] : kw[i]);
            }
            const long long t = token0 + token[u];
            const int head = is_q ? row[u] : row[u] - a.q_heads;
            if (!is_q && a.k_plain != nullptr) *(reinterpret_cast<uint4*>(a.k_plain + t * a.p_token + head * a.p_head) + l) = pack(x);
            if (a.interleaved) {
                if (8 * l < a.rotary) {
                    const float4 c = *reinterpret_cast<const float4*>(&cosines[token[u]][4 * l]), s = *reinterpret_cast<const float4*>(&sines[token[u]][4 * l]);
                    const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float y0 = x[2 * i], y1 = x[2 * i + 1];
                        x[2 * i] = y0 * cc[i] - y1 * ss[i];
                        x[2 * i + 1] = y1 * cc[i] + y0 * ss[i];
                    }
                }
            } else if (half > 0) {                           // the other of each pair is in the lane half a rotation away
                const int away = half / 8;
                const bool lower = l < away, turned = l < 2 * away;
                const int other = lower ? l + away : turned ? l - away : l;
                const int f = turned ? 8 * (lower ? l : l - away) : 0;
#pragma unroll
                for (int i = 0; i < 8; i += 4) {
                    const float4 c = *reinterpret_cast<const float4*>(&cosines[token[u]][f + i]), s = *reinterpret_cast<const float4*>(&sines[token[u]][f + i]);
                    const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float y = __shfl_sync(mine, x[i + k], other, 16);
                        if (turned) x[i + k] = lower ? x[i + k] * cc[k] - y * ss[k] : x[i + k] * cc[k] + y * ss[k];
                    }
                }
            }
            __nv_bfloat16* dst = is_q ? a.q_out + t * a.qo_token + head * a.qo_head : a.k_out + t * a.ko_token + head * a.ko_head;
            *(reinterpret_cast<uint4*>(dst) + l) = pack(x);
        }
    }
}

}  // namespace

cudaError_t launch_rope(RopeArgs a, int sm_count, cudaStream_t stream) {
    // About 20 rows per half-warp, and fewer tokens a block where there would not be a few blocks for every SM.
    const int per_token = a.q_heads + a.k_heads;
    int n = min(kRopeTokens, max(1, 20 * kHalfWarps / per_token));
    while (n > 1 && (a.tokens + n - 1) / n < 4LL * sm_count) n /= 2;
    a.tokens_per_block = n;
    return launch_chained(kPdlOther, rope_kernel, dim3((unsigned)((a.tokens + n - 1) / n)), dim3(kThreads), 0, stream, a);
}

}  // namespace compactor
