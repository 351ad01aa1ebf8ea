// Norms of queries and keys for each head with the rotation by position in the same pass: what a prefill is scored by (keys without
// rotation), held as (keys with it) and asked with, and the rows of a decoding step.
//
//   y = x w r, r = 1 / sqrt(mean(x^2) + eps)  (y = x without w);   a_i = position * f_i, i < R / 2;
//   (y_i, y_j) -> (y_i cos a_i - y_j sin a_i, y_j cos a_i + y_i sin a_i) with (i, j) = (i, i + R / 2) or (2 i, 2 i + 1); channels from R on stay.
//
// Bound by HBM: a row is read once and written once or twice (19661 tokens x 32 heads 57.7 us = 5.6 TB/s, 0.85 of the copy rate; 8192 tokens x 40 heads, keys
// twice, 37.4 us = 0.75 of it: two waves of warps that start together), and the instructions for it have to be few: with the angles of eight tokens in a block and
// the norm, weight and rotation one after the other the latter took 80 us.  So a warp stays with one token: 16 lanes hold a row, eight channels each, and every lane keeps, for all heads of the token,
//   out_c = r (x_c A_c + x_partner B_c),   A_c = w_c cos a,  B_c = -+ w_partner sin a;
// the partner's channel comes from the lane half a rotation away as it was read, two to a register.  Up to four rows of a lane are in flight.
// The angles are worked out in 64 bits, because a far position times a frequency has more digits before the point than 32 bits leave
// behind it (at position 131072 the angle would be off by 0.004), taken to a fraction of a turn and then to 32 bits; each lane works out two and
// the warp shares them.
#include "rope.cuh"
#include "two.cuh"

namespace compactor {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kRows = 4;                       // pairs of rows of a warp in flight

// Eight channels as they are read.
__device__ __forceinline__ void unpack(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack(const uint4& v, Two (&x)[4]) {
    float f[8];
    unpack(v, f);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = two(f[2 * i], f[2 * i + 1]);
}
__device__ __forceinline__ uint4 pack(const Two (&x)[4]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float lo, hi;
        split_two(x[i], lo, hi);
        const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// One kind of rows (queries or keys) of a token: heads first, first + 2 step, ... of `heads`, two at a time (one for each half of the warp).
struct Rows {
    const __nv_bfloat16* in;                   // of the token
    __nv_bfloat16* out;
    __nv_bfloat16* plain;                      // or null
    long long in_head, out_head, plain_head;
    int heads;
    bool norm;
};

// FULL: all channels are rotated.
template <bool INTERLEAVED, bool FULL>
__device__ __forceinline__ void rotate_rows(const Rows& r, const Two (&a)[4], const Two (&b)[4], const Two (&w)[4], float eps, int other,
                                            bool turned, int first, int step) {
    const int l = threadIdx.x & 15, sub = (threadIdx.x >> 4) & 1;
    for (int h0 = first; h0 < r.heads; h0 += kRows * step) {
        uint4 in[kRows];
#pragma unroll
        for (int u = 0; u < kRows; ++u)        // (behind the last row: the last once more, not written)
            in[u] = *(reinterpret_cast<const uint4*>(r.in + min(h0 + u * step + sub, r.heads - 1) * r.in_head) + l);
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            if (h0 + u * step >= r.heads) break;
            const int head = h0 + u * step + sub;
            Two x[4], y[4], z[4];
            unpack(in[u], x);
            float inv = 1.f;
            if (r.norm) {
                Two squares = mul_two(x[0], x[0]);
#pragma unroll
                for (int i = 1; i < 4; ++i) squares = fma_two(x[i], x[i], squares);
                float sum, odd;
                split_two(squares, sum, odd);
                sum += odd;
#pragma unroll
                for (int d = 1; d < 16; d *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                inv = rsqrtf(sum * (1.f / kD) + eps);
            }
            const Two inv2 = two(inv, inv);
            if (INTERLEAVED) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float lo, hi;
                    split_two(x[i], lo, hi);
                    y[i] = two(hi, lo);
                }
            } else {
                unpack(make_uint4(__shfl_sync(0xffffffffu, in[u].x, other), __shfl_sync(0xffffffffu, in[u].y, other),
                                  __shfl_sync(0xffffffffu, in[u].z, other), __shfl_sync(0xffffffffu, in[u].w, other)), y);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const Two xa = mul_two(x[i], a[i]);
                z[i] = mul_two(FULL || turned ? fma_two(y[i], b[i], xa) : xa, inv2);
            }
            if (head < r.heads) {
                *(reinterpret_cast<uint4*>(r.out + head * r.out_head) + l) = pack(z);
                if (r.plain != nullptr) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[i] = mul_two(mul_two(x[i], w[i]), inv2);
                    *(reinterpret_cast<uint4*>(r.plain + head * r.plain_head) + l) = pack(z);
                }
            }
        }
    }
}

// `parts` warps share a token's heads.
template <bool INTERLEAVED, bool FULL>
// (72 registers a thread, for which the half-split ones spill 56 bytes; left alone 84 and none, and 39.2 us for 8192 tokens x 40 heads against 37.4)
__global__ void __launch_bounds__(kThreads, 7)
rope_kernel(const __grid_constant__ RopeArgs a, int parts) {
    __shared__ __align__(16) float turn[kWarps][2][kD / 2];  // cosines and sines
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane & 15;
    pdl_trigger();
    pdl_wait();
    const long long at = (long long)blockIdx.x * kWarps + warp, token = at / parts;
    const int part = (int)(at - token * parts);
    if (token >= a.tokens) return;
    const int half = a.rotary / 2;
    const double position = half > 0 ? (double)a.positions[token] : 0.;
    for (int f = lane; f < half; f += 32) {
        const double turns = position * (double)a.inv_freq[f] * 0.15915494309189533577;      // 1 / (2 pi)
        sincospif(2.f * (float)(turns - rint(turns)), &turn[warp][1][f], &turn[warp][0][f]);
    }
    __syncwarp();
    // the partner's lane, the first of this lane's frequencies, and on which side of the pair it is
    const int away = half / 8;
    const bool turned = 8 * l < a.rotary, lower = l < away;
    const int other = INTERLEAVED || !turned ? lane : lower ? lane + away : lane - away;
    float cosine[8], sine[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int f = !turned ? 0 : INTERLEAVED ? 4 * l + i / 2 : 8 * (lower ? l : l - away) + i;
        const float s = turned ? turn[warp][1][f] : 0.f;
        cosine[i] = turned ? turn[warp][0][f] : 1.f;
        sine[i] = (INTERLEAVED ? (i & 1) == 0 : lower) ? -s : s;
    }
    auto rows = [&](const Rows& r, const __nv_bfloat16* weight) {
        float w[8], v[8];
        Two w2[4], ca[4], cb[4];
        const uint4 ones = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);
        unpack(weight != nullptr ? *(reinterpret_cast<const uint4*>(weight) + l) : ones, w);
        unpack(weight != nullptr ? *(reinterpret_cast<const uint4*>(weight) + (other & 15)) : ones, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w2[i] = two(w[2 * i], w[2 * i + 1]);
            ca[i] = two(cosine[2 * i] * w[2 * i], cosine[2 * i + 1] * w[2 * i + 1]);
            cb[i] = INTERLEAVED ? two(sine[2 * i] * v[2 * i + 1], sine[2 * i + 1] * v[2 * i]) : two(sine[2 * i] * v[2 * i], sine[2 * i + 1] * v[2 * i + 1]);
        }
        rotate_rows<INTERLEAVED, FULL>(r, ca, cb, w2, a.eps, other, turned, 2 * part, 2 * parts);
    };
    if (a.q_heads > 0)
        rows({a.q + token * a.q_token, a.q_out + token * a.qo_token, nullptr, a.q_head, a.qo_head, 0, a.q_heads, a.q_weight != nullptr}, a.q_weight);
    if (a.k_heads > 0)
        rows({a.k + token * a.k_token, a.k_out + token * a.ko_token, a.k_plain != nullptr ? a.k_plain + token * a.p_token : nullptr, a.k_head, a.ko_head,
              a.p_head, a.k_heads, a.k_weight != nullptr}, a.k_weight);
}

}  // namespace

cudaError_t launch_rope(const RopeArgs& a, int sm_count, cudaStream_t stream) {
    // A warp for a token where that makes enough warps, else as many as there are pairs of heads.
    const int most = max(1, (max(a.q_heads, a.k_heads) + 1) / 2);
    int parts = 1;
    while (parts * 2 <= most && a.tokens * parts < 16LL * sm_count) parts *= 2;
    const long long blocks = (a.tokens * parts + kWarps - 1) / kWarps;
    const auto kernel = a.rotary == kD ? (a.interleaved ? rope_kernel<true, true> : rope_kernel<false, true>)
                                       : (a.interleaved ? rope_kernel<true, false> : rope_kernel<false, false>);
    return launch_chained(kPdlOther, kernel, dim3((unsigned)blocks), dim3(kThreads), 0, stream, a, parts);
}

}  // namespace compactor
