// Norms of query and key heads and their rotation by position in one pass (spec_qk_norm_rope).
#include "device_util.h"
#include "prompt_ops.h"

#include <type_traits>

namespace specv {

namespace {

constexpr int kBlockWaves = 4;

// Eight elements as fp32, from 16 bytes of bf16 or 32 of fp32.
template <typename T>
__device__ __forceinline__ void read_eight(float *x, const T *from)
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const f32x4 v = *reinterpret_cast<const f32x4 *>(from + 4 * i);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * i + e] = v[e];
        }
    } else {
        const u32x4 v = *reinterpret_cast<const u32x4 *>(from);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[2 * e] = __uint_as_float(v[e] << 16);
            x[2 * e + 1] = __uint_as_float(v[e] & 0xFFFF0000u);
        }
    }
}
template <typename T>
__device__ __forceinline__ void write_eight(T *to, const float *x)
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 2; ++i) *reinterpret_cast<f32x4 *>(to + 4 * i) = (f32x4){x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
    } else {
        bf16x8 v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (__bf16)x[e];
        *reinterpret_cast<bf16x8 *>(to) = v;
    }
}

// A lane holds two pieces of eight dims of a head whose elements are each other's pairs (or, interleaved, 16 dims side by side, or 16 dims that
// are not rotated), D / 16 lanes a head, so a wavefront 8 heads (d = 128) or 16 at a time, and goes through a token's heads, queries
// and keys alike, in p.per_wave such passes.  A token's angles are found once per wavefront, one a lane, and handed round: the 64-bit
// product is brought to within an eighth of a turn of a multiple of a quarter before it becomes fp32, so that far positions are as exact as
// near ones.
// Bound by the bytes of the rows (10256 tokens of packed prompts, 72 heads of 128, bf16: 378 MB in 80 us, 4.7 TB/s); a step's few rows by the launch and
// the chain position -> angle -> rows (five rows: 4.6 us).
template <typename T, int D, bool INTERLEAVED>
__global__ __launch_bounds__(kBlockWaves *kWave) void qk_norm_rope_kernel(QkNormRopeParams p)
{
    constexpr int kLanes = D / 16, kHeads = kWave / kLanes;   // lanes a head, heads a pass
    const int lane = threadIdx.x % kWave, i = lane % kLanes, sub = lane / kLanes;
    const int groups = (p.passes + p.per_wave - 1) / p.per_wave;   // wavefronts of a token
    const int64_t unit = (int64_t)blockIdx.x * kBlockWaves + threadIdx.x / kWave;
    const int t = __builtin_amdgcn_readfirstlane((int)(unit / groups));
    if (t >= p.T) return;
    const int pass0 = __builtin_amdgcn_readfirstlane((int)(unit - (int64_t)t * groups)) * p.per_wave, pass1 = min(pass0 + p.per_wave, p.passes);

    const int half = p.rot_dim / 2;
    const bool turned = 16 * i < p.rot_dim;
    const int piece0 = INTERLEAVED || !turned ? 2 * i : i, piece1 = INTERLEAVED || !turned ? 2 * i + 1 : i + half / 8;
    float x[16];
    struct Head {
        const T *from;
        T *to;
        bool query, on;
    };
    auto head_of = [&](int pass) {
        const int h = pass * kHeads + sub;
        Head w;
        w.query = h < p.Hq;
        w.on = h < p.Hq + p.Hkv;
        if (w.query) {
            w.from = static_cast<const T *>(p.q) + (int64_t)t * p.q_stride + h * D;
            w.to = static_cast<T *>(p.out_q) + (int64_t)t * p.out_q_stride + h * D;
        } else {
            w.from = static_cast<const T *>(p.k) + (int64_t)t * p.k_stride + (h - p.Hq) * D;
            w.to = static_cast<T *>(p.out_k) + (int64_t)t * p.out_k_stride + (h - p.Hq) * D;
        }
        return w;
    };
    auto read = [&](const Head &w) {
        if (!w.on) return;
        read_eight<T>(x, w.from + 8 * piece0);
        read_eight<T>(x + 8, w.from + 8 * piece1);
    };
    Head head = head_of(pass0);
    read(head);

    // cos and sin of angles 8 i .. 8 i + 7: lane (i, sub) finds angle 8 i + sub % 8
    float co[8], si[8];
    if (p.rot_dim > 0) {
        float c = 1.0f, s = 0.0f;
        if (turned) {
            constexpr double kTurns = 0.15915494309189533577;
            double r = (double)p.positions[t] * (double)p.inv_freq[8 * i + sub % 8] * kTurns;
            r -= rint(r);
            const double quarter = rint(4.0 * r);
            const float a = (float)(2.0 * (r - 0.25 * quarter));   // half turns, at most a quarter
            const float ca = cospif(a), sa = sinpif(a);
            const int n = (int)quarter & 3;
            c = n == 0 ? ca : n == 1 ? -sa : n == 2 ? -ca : sa;
            s = n == 0 ? sa : n == 1 ? ca : n == 2 ? -sa : -ca;
            c *= p.scale;
            s *= p.scale;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            co[e] = __shfl(c, e * kLanes + i);
            si[e] = __shfl(s, e * kLanes + i);
        }
    }
    // both kinds' weights, for this lane's dims
    const bool any_norm = p.q_weight != nullptr || p.k_weight != nullptr;
    float w_q[16], w_k[16];
    auto weights = [&](float *w, const void *from) {
        if (from == nullptr) return;
        if (p.weight_f32) {
            read_eight<float>(w, static_cast<const float *>(from) + 8 * piece0);
            read_eight<float>(w + 8, static_cast<const float *>(from) + 8 * piece1);
        } else {
            read_eight<__bf16>(w, static_cast<const __bf16 *>(from) + 8 * piece0);
            read_eight<__bf16>(w + 8, static_cast<const __bf16 *>(from) + 8 * piece1);
        }
    };
    weights(w_q, p.q_weight);
    weights(w_k, p.k_weight);

    for (int pass = pass0;;) {
        float y[16];
        if (any_norm) {
            float sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 16; ++e) sum = fmaf(x[e], x[e], sum);
#pragma unroll
            for (int step = 1; step < kLanes; step *= 2) sum += __shfl_xor(sum, step);
            const bool norm = head.query ? p.q_weight != nullptr : p.k_weight != nullptr;
            const float r = 1.0f / sqrtf(fmaf(sum, 1.0f / D, p.eps));
#pragma unroll
            for (int e = 0; e < 16; ++e) y[e] = norm ? x[e] * r * (head.query ? w_q[e] : w_k[e]) : x[e];
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) y[e] = x[e];
        }
        const Head now = head;
        if (++pass < pass1) {   // (the next heads' rows are on their way meanwhile)
            head = head_of(pass);
            read(head);
        }
        if (turned) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int a = INTERLEAVED ? 2 * e : e, b = INTERLEAVED ? 2 * e + 1 : e + 8;
                const float ya = y[a], yb = y[b];
                y[a] = fmaf(ya, co[e], -(yb * si[e]));
                y[b] = fmaf(yb, co[e], ya * si[e]);
            }
        }
        if (now.on) {
            write_eight<T>(now.to + 8 * piece0, y);
            write_eight<T>(now.to + 8 * piece1, y + 8);
        }
        if (pass >= pass1) break;
    }
}

template <typename T, int D>
void go(const QkNormRopeParams &p, unsigned blocks, hipStream_t stream)
{
    if (p.interleaved) hipLaunchKernelGGL((qk_norm_rope_kernel<T, D, true>), dim3(blocks), dim3(kBlockWaves * kWave), 0, stream, p);
    else hipLaunchKernelGGL((qk_norm_rope_kernel<T, D, false>), dim3(blocks), dim3(kBlockWaves * kWave), 0, stream, p);
}

}  // namespace

hipError_t launch_qk_norm_rope(const QkNormRopeParams &given, hipStream_t stream)
{
    QkNormRopeParams p = given;
    const int heads = 1024 / p.d;   // of a pass
    p.passes = (p.Hq + p.Hkv + heads - 1) / heads;
    // A wavefront takes as many passes as leave 4096 wavefronts (a quarter of what the device holds), so that a token's angles are found few times.
    const int64_t wanted = (int64_t)p.T * p.passes / 4096;
    p.per_wave = (int)(wanted < 1 ? 1 : wanted > p.passes ? p.passes : wanted);
    const int64_t units = (int64_t)p.T * ((p.passes + p.per_wave - 1) / p.per_wave);
    const unsigned blocks = (unsigned)((units + kBlockWaves - 1) / kBlockWaves);
    if (p.f32) {
        if (p.d == 128) go<float, 128>(p, blocks, stream);
        else go<float, 64>(p, blocks, stream);
    } else {
        if (p.d == 128) go<__bf16, 128>(p, blocks, stream);
        else go<__bf16, 64>(p, blocks, stream);
    }
    return hipGetLastError();
}

}  // namespace specv
