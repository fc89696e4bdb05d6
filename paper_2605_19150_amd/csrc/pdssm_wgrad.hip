// pdssm_wgrad.hip -- weight gradient of a token projection from the 8-bit form
// of its input, dW[m, d] = sum_t dP[t, m] u[t, d], on the matrix cores (bf16
// operands, fp32 sums).  A value q * 2^e of the 8-bit form is exact in bf16, so
// no operand is rounded.
//
// Both operands lie in memory with the contracted axis, the tokens, outermost;
// the matrix instruction wants eight consecutive tokens of one row in a lane.
// So the tiles are turned on their way into LDS, in registers: a thread loads
// 8 tokens of 8 rows (of 4, for the smaller tile) of each operand, pairs the
// tokens of a row (a byte permutation for dP; for q the conversion to bf16,
// which packs two values anyway) and writes 8 tokens of each row, 16 bytes.
#include "pdssm_device.h"
#include "pdssm_rows.h"

#include <type_traits>

namespace pdssm {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

// What bounds it: the matrix cores and the power they draw.  M8192 Dm4096
// T32768 takes 1.87 ms, 1178 TFLOP/s; the vendor library's product of bf16
// operands of that shape (u already widened, so twice its bytes) takes 1.87 ms
// too.  Without its loads the kernel would take 1.37 ms.
//
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
    static constexpr int R = B / 32;              // rows that a thread turns, of each operand
    static_assert(R == 8 || R == 4, "loads of 8 R bytes of dP, 4 R of q");
};

// LDS row r keeps its 16-byte chunk c (tokens 8c .. 8c+7) at place c ^ turn(r):
// 16 consecutive rows read at one chunk fall on different banks, and so do the
// rows, R apart, that eight lanes write at one chunk.
__device__ __forceinline__ int turn(int r) { return (r ^ (r >> 3)) & 7; }

constexpr int kGroup = 8;  // tiles along M

// row_block of values that are the same in every lane but may have been formed
// in vector registers.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t scalar_block(const void* base, int bytes) {
    const uint64_t b = reinterpret_cast<uint64_t>(base);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)b), hi = __builtin_amdgcn_readfirstlane((uint32_t)(b >> 32));
    return row_block(reinterpret_cast<const void*>((uint64_t)hi << 32 | lo), __builtin_amdgcn_readfirstlane(bytes));
}

template <int B>
__global__ __launch_bounds__(256, B == 256 ? 1 : 2) void k_wgrad(WgradArgs a, int Z, float* out) {
    using C = Tile<B>;
    extern __shared__ __align__(16) unsigned char lds[];
    const int wv = wave_id(), lane = lane_id();
    const int MT = (a.M + B - 1) / B, DT = (a.Dm + B - 1) / B, total = MT * DT;
    // consecutive workgroups go to the 8 XCDs in turn: each XCD takes a run of
    // the tiles of all shares, which have their rows of dP in common
    const int jobs = total * Z, job = (blockIdx.x & 7) * ((jobs + 7) / 8) + (blockIdx.x >> 3);
    if (job >= jobs) return;
    const int z = job / total, turnno = job - z * total;
    // in turn, kGroup tiles along M before the next along Dm: a run of 32 is
    // then about square in bytes (a row of dP has twice those of u)
    const int gt = kGroup * DT, gr = turnno / gt, in = turnno - gr * gt, gm = min(kGroup, MT - gr * kGroup);
    const int mt = gr * kGroup + in % gm, dt = in / gm;
    const int m0 = mt * B, d0 = dt * B;
    const int slices = (a.T + C::KS - 1) / C::KS, share = ((slices + Z - 1) / Z + 1) & ~1;  // in pairs
    const int s0 = z * share, s1 = min(slices, s0 + share);

    // ---- loads: eight lanes next to each other read a token's consecutive
    // rows, whole lines (with tokens in neighbouring lanes instead, every lane is
    // a request of its own: 2.47 ms against 1.5 at M8192 Dm4096 T32768); rows
    // past the last: the last ones again
    const int tb = lane >> 3, row = C::R * (wv * 8 + (lane & 7));
    const uint32_t pld = (uint32_t)a.M * 2, qld = (uint32_t)a.Dm;
    const int pm = min(m0 + row, a.M - C::R), ud = min(d0 + row, a.Dm - C::R);
    const uint32_t vp = (uint32_t)(8 * tb) * pld + pm * 2, vu = (uint32_t)(8 * tb) * qld + ud;
    const uint32_t ve = (uint32_t)(tb >> 2) * qld + ud;
    // two sets of registers: a slice's loads are issued about one slice before
    // they are turned
    struct Raw {
        uint32_t p[8][C::R / 2], q[8][C::R / 4], e[C::R / 4];
    } raw[2];
    // Slice s as buffers; past the last slice they are empty and give zeros.
    struct Source {
        __amdgpu_buffer_rsrc_t p, q, e;
    };
    auto source = [&](int s) {
        const int t0 = s * C::KS, nt = max(0, min(a.T - t0, C::KS));
        return Source{scalar_block(a.dP + (size_t)t0 * a.M, nt * (int)pld),
                      scalar_block(a.q + (size_t)t0 * a.Dm, nt * (int)qld),
                      scalar_block(a.e + (size_t)(t0 / kKeptRows) * a.Dm, (nt + kKeptRows - 1) / kKeptRows * (int)qld)};
    };
    // Load n of a slice: dP's 8 tokens, u's, the exponents.
    constexpr int kLoads = 17;
    auto load_one = [&](const Source& from, Raw& g, int n) {
        const int j = n & 7;
        if (n < 8) {
            if constexpr (C::R == 8) {
                const u32x4 v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(from.p, vp + j * pld, 0, 0));
#pragma unroll
                for (int i = 0; i < 4; ++i) g.p[j][i] = v[i];
            } else {
                const u32x2 v = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(from.p, vp + j * pld, 0, 0));
                g.p[j][0] = v[0];
                g.p[j][1] = v[1];
            }
        } else if (n < 16) {
            if constexpr (C::R == 8) {
                const u32x2 v = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(from.q, vu + j * qld, 0, 0));
                g.q[j][0] = v[0];
                g.q[j][1] = v[1];
            } else {
                g.q[j][0] = __builtin_amdgcn_raw_buffer_load_b32(from.q, vu + j * qld, 0, 0);
            }
        } else {
            if constexpr (C::R == 8) {
                const u32x2 v = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(from.e, ve, 0, 0));
                g.e[0] = v[0];
                g.e[1] = v[1];
            } else {
                g.e[0] = __builtin_amdgcn_raw_buffer_load_b32(from.e, ve, 0, 0);
            }
        }
    };
    auto load = [&](int s, Raw& g) {
        const Source from = source(s);
#pragma unroll
        for (int n = 0; n < kLoads; ++n) load_one(from, g, n);
    };
    // Row i of what the thread turns, to stage st, in six pieces of about five
    // vector instructions each.
    u32x4 wu;
    float scale;
    auto turn_piece = [&](int st, const Raw& g, int i, int piece) {
        unsigned char* P = lds + st * C::STAGE + (row + i) * C::ROWB + 16 * (tb ^ turn(row + i));
        if (piece == 0) {
            u32x4 w;
#pragma unroll
            for (int j = 0; j < 4; ++j)  // tokens 2j and 2j + 1 of row i
                w[j] = __builtin_amdgcn_perm(g.p[2 * j + 1][i / 2], g.p[2 * j][i / 2], i & 1 ? 0x07060302 : 0x05040100);
            *reinterpret_cast<u32x4*>(P) = w;
            scale = kept_scale((int)(int8_t)(g.e[i / 4] >> (8 * (i % 4))));
        } else if (piece <= 4) {
            const int j = piece - 1;
            const float lo = (float)(int8_t)(g.q[2 * j][i / 4] >> (8 * (i % 4))) * scale;
            const float hi = (float)(int8_t)(g.q[2 * j + 1][i / 4] >> (8 * (i % 4))) * scale;
            wu[j] = __builtin_bit_cast(unsigned, bf16x2{(__bf16)lo, (__bf16)hi});
        } else {
            *reinterpret_cast<u32x4*>(P + C::SIDE) = wu;
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
    struct Frag {
        bf16x8 p[C::N], u[C::N];
    } f[2];
    auto read = [&](int st, int kk, Frag& g, int n) {
        const int r = 32 * (n % C::N) + l32;  // in the wave's half, which begins at a multiple of 64
        const unsigned char* at = lds + st * C::STAGE + r * C::ROWB + 16 * ((2 * kk + hf) ^ turn(r));
        if (n < C::N) g.u[n] = *reinterpret_cast<const bf16x8*>(at + C::SIDE + wd * (B / 2) * C::ROWB);
        else g.p[n - C::N] = *reinterpret_cast<const bf16x8*>(at + wm * (B / 2) * C::ROWB);
    };
    // Step kk of stage st: its products on fragment set kk % 2 and between them
    // the next step's reads (the next slice's first step after the last) and,
    // in the first three steps, the next slice's turn.  After the last slice
    // that goes on with what nobody reads.
    constexpr int kProducts = C::N * C::N, kPieces = 6 * C::R;
    constexpr int kEach = kPieces / (3 * kProducts);
    static_assert(kEach * 3 * kProducts == kPieces && kProducts % (2 * C::N) == 0, "reads and pieces spread evenly");
    // The loads stand between products too: a wave that issues them in a row
    // waits for the address unit, and its products with it (2.11 against 1.87
    // ms at M8192 Dm4096 T32768).
    auto step = [&](int st, auto kk_, const Raw& g, const Source& from, Raw& other) {
        constexpr int kk = decltype(kk_)::value;
        Frag& now = f[kk & 1];
        Frag& then = f[(kk & 1) ^ 1];
#pragma unroll
        for (int m = 0; m < kProducts; ++m) {
            const int i = m / C::N, j = m % C::N;
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(now.p[i], now.u[j], acc[i][j], 0, 0, 0);
            if (m % (kProducts / (2 * C::N)) == 0)
                read(kk < 3 ? st : st ^ 1, (kk + 1) % 4, then, m / (kProducts / (2 * C::N)));
            if constexpr (kk < 3) {
                const int first = (kk * kProducts + m) * kEach;
#pragma unroll
                for (int n = 0; n < kEach; ++n) turn_piece(st ^ 1, g, (first + n) / 6, (first + n) % 6);
            }
            if constexpr (kk == 3 || kk == 0) {
                constexpr int kSlots = 2 * kProducts;
                const int at = (kk == 3 ? 0 : kProducts) + m;
#pragma unroll
                for (int n = at * kLoads / kSlots; n < (at + 1) * kLoads / kSlots; ++n) load_one(from, other, n);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    using k0 = std::integral_constant<int, 0>;
    using k1 = std::integral_constant<int, 1>;
    using k2 = std::integral_constant<int, 2>;
    using k3 = std::integral_constant<int, 3>;
    // Slice s in stage st; g: the registers of slice s + 1, then of s + 3;
    // other: of s + 2, whose first loads the slice before this one issued.
    Source from;
    auto slice = [&](int s, int st, Raw& g, Raw& other) {
        step(st, k0{}, g, from, other);
        step(st, k1{}, g, from, other);
        step(st, k2{}, g, from, other);
        from = source(s + 3);
        // every wave has read all of this stage and written its part of the other
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        step(st, k3{}, g, from, g);
    };
    if (s0 < s1) {
        load(s0, raw[0]);
        load(s0 + 1, raw[1]);
#pragma unroll
        for (int n = 0; n < kPieces; ++n) turn_piece(0, raw[0], n / 6, n % 6);
        from = source(s0 + 2);
#pragma unroll
        for (int n = 0; n < kLoads / 2; ++n) load_one(from, raw[0], n);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
        for (int n = 0; n < 2 * C::N; ++n) read(0, 0, f[0], n);
        for (int s = s0; s < s1; s += 2) {
            slice(s, 0, raw[1], raw[0]);
            slice(s + 1, 1, raw[0], raw[1]);
        }
    }

    const int mw = m0 + wm * (B / 2), rows = max(0, min(a.M - mw, B / 2));
    const auto o = scalar_block(out + ((size_t)z * a.M + min(mw, a.M)) * a.Dm, rows * a.Dm * 4);
#pragma unroll
    for (int j = 0; j < C::N; ++j) {
        const int d = d0 + wd * (B / 2) + 32 * j + l32;
        // a column past the last lies past every buffer
        const uint32_t at = d < a.Dm ? (uint32_t)(4 * hf) * a.Dm * 4 + d * 4 : 0x80000000u;
#pragma unroll
        for (int i = 0; i < C::N; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(acc[i][j][r]), o,
                                                      at + (uint32_t)(32 * i + 8 * (r / 4) + r % 4) * a.Dm * 4, 0, kLoadStream);
    }
}

// dW = the shares' sums.  G threads take every Gth share of four entries, and
// their sums are added in order.
template <int G>
__global__ __launch_bounds__(256) void k_wgrad_sum(const float* part, float* dW, size_t n, int Z) {
    constexpr int W = 256 / G;
    __shared__ float4 sums[G][W];
    const int g = threadIdx.x / W, l = threadIdx.x % W;
    const size_t i = 4 * ((size_t)blockIdx.x * W + l);  // n is a multiple of 128
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](const float4& v) { s = make_float4(s.x + v.x, s.y + v.y, s.z + v.z, s.w + v.w); };
    if (i < n) {
#pragma unroll 4
        for (int z = g; z < Z; z += G) add(*reinterpret_cast<const float4*>(part + (size_t)z * n + i));
    }
    sums[g][l] = s;
    __syncthreads();
    if (g != 0 || i >= n) return;
#pragma unroll
    for (int k = 1; k < G; ++k) add(sums[k][l]);
    *reinterpret_cast<float4*>(dW + i) = s;
}

// Tile and shares of the tokens.  The 256 tile needs half the LDS traffic of
// the 128 one, which fills the 256 CUs with shorter shares and smaller sums of
// them.  The larger is taken where a CU has 24 slices of it or more (T32768 M1024
// Dm1024, 32: 88 us against 108; T8192 M2048 Dm1024, 16: 65 against 55; T1500 M8192
// Dm1024, 12: 56 against 36), or its tiles fill the CUs without shares (T511
// M8192 Dm2048: 28 against 31).
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
    // shares are whole pairs of slices (as in the kernel): no empty ones
    auto even = [&](int z) {
        const int share = ((slices + z - 1) / z + 1) & ~1;
        return share ? (slices + share - 1) / share : 1;
    };
    if (tiles(256) >= 192 || tiles(256) * slices >= 24 * 256) return {256, even(shares(256, 256, 4))};
    return {128, even(shares(128, 512, 1))};
}

template <int B>
hipError_t launch(const WgradArgs& a, int Z, float* out, hipStream_t s) {
    const int total = ((a.M + B - 1) / B) * ((a.Dm + B - 1) / B);
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k_wgrad<B>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)Tile<B>::LDS);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_wgrad<B>, dim3((unsigned)(8 * (((long long)total * Z + 7) / 8))), dim3(256), Tile<B>::LDS, s, a, Z, out);
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
    auto sum = [&](auto* f, int W) {
        hipLaunchKernelGGL(f, dim3((unsigned)((n / 4 + W - 1) / W)), dim3(256), 0, s, out, a.dW, n, p.Z);
    };
    p.Z >= 8 ? sum(k_wgrad_sum<16>, 16) : sum(k_wgrad_sum<4>, 64);
    return hipGetLastError();
}

}  // namespace pdssm
