// pdssm_wgrad.hip -- weight gradient of a token projection from the 8-bit form
// of its input, dW[m, d] = sum_t dP[t, m] u[t, d], on the matrix cores (bf16
// operands, fp32 sums).  A value q * 2^e of the 8-bit form is exact in bf16, so
// no operand is rounded.
//
// Both operands lie in memory with the contracted axis, the tokens, outermost;
// the matrix instruction wants eight consecutive tokens of one row in a lane.
// So the tiles are turned on their way into LDS, in registers: a thread loads
// an 8 x 8 block (8 tokens, 16 bytes of dP or 8 bytes of q each), pairs the
// tokens of a row (a byte permutation for dP; for q the conversion to bf16,
// which packs two values anyway) and writes 8 rows of 8 tokens, 16 bytes each.
#include "pdssm_device.h"
#include "pdssm_rows.h"

namespace pdssm {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

// A workgroup of four waves sums a B x B block of dW over a share of the
// tokens, 64 a slice; a wave has a quarter of it.  Two LDS stages: while one is
// multiplied the next slice is turned into the other.
template <int B>
struct Tile {
    static constexpr int KS = 64;                 // tokens of a slice
    static constexpr int ROWB = KS * 2;           // bytes of an LDS row: one row's tokens of a slice
    static constexpr int SIDE = B * ROWB;         // bytes of one operand's slice
    static constexpr int STAGE = 2 * SIDE;
    static constexpr size_t LDS = 2 * STAGE;
    static constexpr int N = B / 64;              // 32 x 32 products along a wave's side
    static constexpr bool BOTH = B == 256;        // a thread turns a block of each operand, or of one
    static_assert(B == 256 || B == 128, "256 or 128 blocks of 8 x 8 an operand");
};

// LDS row r keeps its 16-byte chunk c (tokens 8c .. 8c+7) at place c ^ turn(r):
// 16 rows read at one chunk, and the 8 chunks written of one row, fall on
// different banks.
__device__ __forceinline__ int turn(int r) { return (r & 7) ^ ((r >> 3) & 1); }

template <int B>
__global__ __launch_bounds__(256, B == 256 ? 1 : 2) void k_wgrad(WgradArgs a, int Z, float* out) {
    using C = Tile<B>;
    extern __shared__ __align__(16) unsigned char lds[];
    const int wv = wave_id(), lane = lane_id();
    const int MT = (a.M + B - 1) / B, DT = (a.Dm + B - 1) / B, total = MT * DT;
    // consecutive workgroups go to the 8 XCDs in turn: each XCD takes a run of
    // tiles that share their rows of dP
    const int per = (total + 7) / 8;
    const int z = blockIdx.y;
    const int tile = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || tile >= total) return;
    const int m0 = tile / DT * B, d0 = tile % DT * B;
    const int slices = (a.T + C::KS - 1) / C::KS, share = (slices + Z - 1) / Z;
    const int s0 = z * share, s1 = min(slices, s0 + share);

    // ---- loads: lane % 8 is the block's place along the tokens, lane / 8 (and
    // the wave) along the rows; blocks past the last row load the last one
    const bool doP = C::BOTH || wv < 2, doU = C::BOTH || wv >= 2;
    const int tb = lane & 7, row = 8 * ((C::BOTH ? wv : wv & 1) * 8 + (lane >> 3));
    const uint32_t pld = (uint32_t)a.M * 2, qld = (uint32_t)a.Dm;
    const int pm = min(m0 + row, a.M - 8), ud = min(d0 + row, a.Dm - 8);
    const uint32_t vp = (uint32_t)(8 * tb) * pld + pm * 2, vu = (uint32_t)(8 * tb) * qld + ud;
    const uint32_t ve = (uint32_t)(tb >> 2) * qld + ud;
    u32x4 p[8];
    u32x2 q[8], ex;
    auto load = [&](int s) {
        const int t0 = s * C::KS, n = min(a.T - t0, C::KS);  // tokens past the last: 0
        if (doP) {
            const auto rp = row_block(a.dP + (size_t)t0 * a.M, (uint32_t)n * pld);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                p[j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rp, vp + j * pld, 0, 0));
        }
        if (doU) {
            const auto rq = row_block(a.q + (size_t)t0 * a.Dm, (uint32_t)n * qld);
            const auto re = row_block(a.e + (size_t)(t0 / kKeptRows) * a.Dm, (uint32_t)((n + kKeptRows - 1) / kKeptRows) * qld);
            ex = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(re, ve, 0, 0));
#pragma unroll
            for (int j = 0; j < 8; ++j)
                q[j] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rq, vu + j * qld, 0, 0));
        }
    };
    auto store = [&](int st) {
        unsigned char* P = lds + st * C::STAGE + row * C::ROWB;
        unsigned char* U = P + C::SIDE;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int at = i * C::ROWB + 16 * (tb ^ turn(row + i));
            u32x4 w;
            if (doP) {
#pragma unroll
                for (int j = 0; j < 4; ++j)  // tokens 2j and 2j + 1 of row i
                    w[j] = __builtin_amdgcn_perm(p[2 * j + 1][i / 2], p[2 * j][i / 2], i & 1 ? 0x07060302 : 0x05040100);
                *reinterpret_cast<u32x4*>(P + at) = w;
            }
            if (doU) {
                const float scale = kept_scale((int)(int8_t)(ex[i / 4] >> (8 * (i % 4))));
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float lo = (float)(int8_t)(q[2 * j][i / 4] >> (8 * (i % 4))) * scale;
                    const float hi = (float)(int8_t)(q[2 * j + 1][i / 4] >> (8 * (i % 4))) * scale;
                    w[j] = __builtin_bit_cast(unsigned, bf16x2{(__bf16)lo, (__bf16)hi});
                }
                *reinterpret_cast<u32x4*>(U + at) = w;
            }
        }
    };

    // ---- products: wave (wm, wd) has rows wm * B/2 .. of dP and wd * B/2 .. of u
    const int wm = wv >> 1, wd = wv & 1, l32 = lane & 31, hf = lane >> 5;
    f32x16 acc[C::N][C::N];
#pragma unroll
    for (int i = 0; i < C::N; ++i)
#pragma unroll
        for (int j = 0; j < C::N; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    auto multiply = [&](int st) {
        const unsigned char* P = lds + st * C::STAGE + (wm * (B / 2) + l32) * C::ROWB;
        const unsigned char* U = lds + st * C::STAGE + C::SIDE + (wd * (B / 2) + l32) * C::ROWB;
#pragma unroll
        for (int kk = 0; kk < C::KS / 16; ++kk) {
            const int at = 16 * ((2 * kk + hf) ^ turn(l32));
            bf16x8 A[C::N], D[C::N];
#pragma unroll
            for (int i = 0; i < C::N; ++i) A[i] = *reinterpret_cast<const bf16x8*>(P + 32 * i * C::ROWB + at);
#pragma unroll
            for (int j = 0; j < C::N; ++j) D[j] = *reinterpret_cast<const bf16x8*>(U + 32 * j * C::ROWB + at);
#pragma unroll
            for (int i = 0; i < C::N; ++i)
#pragma unroll
                for (int j = 0; j < C::N; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(A[i], D[j], acc[i][j], 0, 0, 0);
        }
    };
    if (s0 < s1) {
        load(s0);
        store(0);
        if (s0 + 1 < s1) load(s0 + 1);
        __syncthreads();
        for (int s = s0; s < s1; ++s) {
            const int st = (s - s0) & 1;
            multiply(st);
            if (s + 1 < s1) store(st ^ 1);
            if (s + 2 < s1) load(s + 2);
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        }
    }

    float* o = out + (size_t)z * a.M * a.Dm;
#pragma unroll
    for (int i = 0; i < C::N; ++i)
#pragma unroll
        for (int j = 0; j < C::N; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int m = m0 + wm * (B / 2) + 32 * i + 8 * (r / 4) + 4 * hf + r % 4, d = d0 + wd * (B / 2) + 32 * j + l32;
                if (m < a.M && d < a.Dm) __builtin_nontemporal_store(acc[i][j][r], o + (size_t)m * a.Dm + d);
            }
}

// dW = the shares' sums, in the order of the tokens.
__global__ __launch_bounds__(256) void k_wgrad_sum(const float* part, float* dW, size_t n, int Z) {
    const size_t i = 4 * ((size_t)blockIdx.x * 256 + threadIdx.x);  // n is a multiple of 128
    if (i >= n) return;
    float4 s = *reinterpret_cast<const float4*>(part + i);
#pragma unroll 4
    for (int z = 1; z < Z; ++z) {
        const float4 v = *reinterpret_cast<const float4*>(part + (size_t)z * n + i);
        s = make_float4(s.x + v.x, s.y + v.y, s.z + v.z, s.w + v.w);
    }
    *reinterpret_cast<float4*>(dW + i) = s;
}

// Tile and shares of the tokens.  The 256 tile needs half the LDS traffic of
// the 128 one; it is taken where its tiles, or shares of at least 4 slices, fill the
// 256 CUs.
struct WgradPlan {
    int B, Z;
};
WgradPlan plan_of(int T, int M, int Dm) {
    const int slices = (T + 63) / 64;
    auto tiles = [&](int B) { return (long long)((M + B - 1) / B) * ((Dm + B - 1) / B); };
    auto shares = [&](int B, int cus, int least) {
        long long z = (cus + tiles(B) - 1) / tiles(B);
        if (z > (slices + least - 1) / least) z = (slices + least - 1) / least;
        return (int)(z < 1 ? 1 : z);
    };
    const int z256 = shares(256, 256, 4);
    if (tiles(256) * z256 >= 192) return {256, z256};
    return {128, shares(128, 512, 1)};
}

template <int B>
hipError_t launch(const WgradArgs& a, int Z, float* out, hipStream_t s) {
    const int total = ((a.M + B - 1) / B) * ((a.Dm + B - 1) / B);
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k_wgrad<B>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)Tile<B>::LDS);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_wgrad<B>, dim3(8 * ((total + 7) / 8), Z), dim3(256), Tile<B>::LDS, s, a, Z, out);
    return hipGetLastError();
}

}  // namespace

size_t wgrad_workspace(int T, int M, int Dm) {
    const WgradPlan p = plan_of(T, M, Dm);
    return p.Z > 1 ? (size_t)p.Z * M * Dm * 4 : 0;
}

hipError_t launch_wgrad(const WgradArgs& a, hipStream_t s) {
    const WgradPlan p = plan_of(a.T, a.M, a.Dm);
    float* out = p.Z > 1 ? static_cast<float*>(a.ws) : a.dW;
    hipError_t e = p.B == 256 ? launch<256>(a, p.Z, out, s) : launch<128>(a, p.Z, out, s);
    if (e != hipSuccess || p.Z == 1) return e;
    const size_t n = (size_t)a.M * a.Dm;
    hipLaunchKernelGGL(k_wgrad_sum, dim3((n / 4 + 255) / 256), dim3(256), 0, s, out, a.dW, n, p.Z);
    return hipGetLastError();
}

}  // namespace pdssm
