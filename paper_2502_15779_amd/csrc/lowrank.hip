// Low-rank adapters of many requests beside a shared projection:
//   out[m] = base[m] + scaling[a] (x[m] A[a]^T) B[a]^T,   a = which[m]   (no adapter: out[m] = base[m])
// A is [adapters][r][K], B [adapters][N][r], in the 16-bit type of x.
//
// Two launches, since every output needs the whole inner sum.  The first forms t = x A^T on the matrix cores, split along K; its partial
// sums go to the workspace, in binary32 and in a fixed order (no atomics).  The second adds them up and multiplies by B.  A tile of
// tokens is multiplied once for each adapter that one of its tokens has (a "leader" is the first token of the tile with that adapter), and
// a token keeps the products of its own one.
// t has 32 bits and the matrix cores take 16: it goes in as two binary16 numbers, scaled by a power of two per token (22 bits and more
// of every value down to 2^-12 of the token's largest), or as three bfloat16 numbers (24 bits).
#include <type_traits>

#include "rcp_internal.hpp"

namespace rcp {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));

template <int DT>
using Eight = std::conditional_t<DT == RCP_F16, v8h, v8b>;
template <int DT>
using One = std::conditional_t<DT == RCP_F16, _Float16, __bf16>;

template <int DT>
__device__ __forceinline__ v4f lowrank_mfma(Eight<DT> a, Eight<DT> b, v4f c)
{
    if constexpr (DT == RCP_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

constexpr int LOWRANK_STEP = 32;   // columns a matrix instruction takes

struct LowrankArgs {
    const void *x, *A, *B, *base;
    const int* which;
    const float* scaling;
    void* out;
    float* part;  // [splits][M][r]
    int M, N, K, r, adapters, splits, chunk;  // chunk: columns of a split, a multiple of 4 * LOWRANK_STEP
    int slots, columns;                       // first kernel: leaders side by side; second: outputs of a workgroup, a multiple of 128
};

// the adapter of token m, -1 for none
__device__ __forceinline__ int lowrank_adapter(const LowrankArgs& a, int m)
{
    const int id = m < a.M ? a.which[m] : -1;
    return static_cast<unsigned>(id) < static_cast<unsigned>(a.adapters) ? id : -1;
}

// the lanes among `tokens` whose adapter no lower lane has
__device__ __forceinline__ unsigned long long lowrank_leaders(int id, int tokens)
{
    unsigned long long rest = __builtin_amdgcn_ballot_w64(id >= 0), leaders = 0;
    if (tokens < 64) rest &= (1ull << tokens) - 1;
    while (rest != 0) {  // at most one round for each lane
        const int at = __builtin_ctzll(rest);
        leaders |= 1ull << at;
        rest &= ~__builtin_amdgcn_ballot_w64(id == __builtin_amdgcn_readlane(id, at));
    }
    return leaders;
}

// Workgroup = (split of K, slot of leaders, TT x 16 tokens); each wavefront sums a quarter of the split.
template <int DT, int TT, int NR>
__global__ __launch_bounds__(256) void lowrank_in_kernel(LowrankArgs a)
{
    __shared__ float red[3][TT][NR][256];
    const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m0 = static_cast<int>(blockIdx.z) * 16 * TT;
    const int id = lane < 16 * TT ? lowrank_adapter(a, m0 + lane) : -1;
    unsigned long long leaders = lowrank_leaders(id, 16 * TT);
    const int quarter = a.chunk / 4, k0 = static_cast<int>(blockIdx.x) * a.chunk + quarter * wave, k1 = min(a.K, k0 + quarter);
    const auto* const x = static_cast<const One<DT>*>(a.x);
    for (int slot = 0; leaders != 0; ++slot, leaders &= leaders - 1) {
        if (slot % a.slots != static_cast<int>(blockIdx.y)) continue;  // uniform
        const int adapter = __builtin_amdgcn_readlane(id, __builtin_ctzll(leaders));
        const auto* const A = static_cast<const One<DT>*>(a.A) + static_cast<size_t>(adapter) * a.r * a.K;
        for (int r0 = 0; r0 < a.r; r0 += 16 * NR) {
            v4f acc[TT][NR];
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int n = 0; n < NR; ++n) acc[t][n] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
            size_t xat[TT], aat[NR];  // rows beyond the last token or rank repeat it
#pragma unroll
            for (int t = 0; t < TT; ++t) xat[t] = static_cast<size_t>(min(m0 + 16 * t + i, a.M - 1)) * a.K + 8 * g;
#pragma unroll
            for (int n = 0; n < NR; ++n) aat[n] = static_cast<size_t>(min(r0 + 16 * n + i, a.r - 1)) * a.K + 8 * g;
#pragma unroll 4
            for (int k = k0; k < k1; k += LOWRANK_STEP) {
                Eight<DT> xv[TT], av[NR];
#pragma unroll
                for (int t = 0; t < TT; ++t) xv[t] = *reinterpret_cast<const Eight<DT>*>(x + xat[t] + k);
#pragma unroll
                for (int n = 0; n < NR; ++n) av[n] = *reinterpret_cast<const Eight<DT>*>(A + aat[n] + k);
#pragma unroll
                for (int t = 0; t < TT; ++t)
#pragma unroll
                    for (int n = 0; n < NR; ++n) acc[t][n] = lowrank_mfma<DT>(xv[t], av[n], acc[t][n]);
            }
            if (wave > 0) {
#pragma unroll
                for (int t = 0; t < TT; ++t)
#pragma unroll
                    for (int n = 0; n < NR; ++n) *reinterpret_cast<v4f*>(&red[wave - 1][t][n][4 * lane]) = acc[t][n];
            }
            __syncthreads();
            if (wave == 0) {
#pragma unroll
                for (int t = 0; t < TT; ++t)
#pragma unroll
                    for (int n = 0; n < NR; ++n) {
                        v4f s = acc[t][n];
#pragma unroll
                        for (int w = 0; w < 3; ++w) s += *reinterpret_cast<const v4f*>(&red[w][t][n][4 * lane]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int at = 16 * t + 4 * g + j, rank = r0 + 16 * n + i;
                            if (__shfl(id, at, 64) == adapter && rank < a.r)
                                a.part[(static_cast<size_t>(blockIdx.x) * a.M + m0 + at) * a.r + rank] = s[j];
                        }
                    }
            }
            __syncthreads();
        }
    }
}

template <int DT>
__device__ __forceinline__ Eight<DT> lowrank_round(float (&v)[8])  // and leaves what that misses
{
    Eight<DT> h;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        h[e] = static_cast<One<DT>>(v[e]);
        v[e] -= static_cast<float>(h[e]);
    }
    return h;
}

template <int DT>
__device__ __forceinline__ void lowrank_load4(const void* p, size_t i, float (&v)[4])
{
    if constexpr (DT == RCP_F32) {
        const float4 x = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
    } else {
        const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + i);
        const uint16_t h[4] = {static_cast<uint16_t>(w.x), static_cast<uint16_t>(w.x >> 16), static_cast<uint16_t>(w.y), static_cast<uint16_t>(w.y >> 16)};
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = DT == RCP_F16 ? half_bits_to_float(h[e]) : bf16_bits_to_float(h[e]);
    }
}

template <int DT>
__device__ __forceinline__ void lowrank_store4(void* p, size_t i, const float (&v)[4])
{
    if constexpr (DT == RCP_F32) *reinterpret_cast<float4*>(static_cast<float*>(p) + i) = make_float4(v[0], v[1], v[2], v[3]);
    else {
        uint16_t h[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (DT == RCP_F16) h[e] = __half_as_ushort(round_to_half(v[e]));
            else h[e] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v[e]));
        }
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + i) = make_uint2(h[0] | static_cast<uint32_t>(h[1]) << 16, h[2] | static_cast<uint32_t>(h[3]) << 16);
    }
}

// Workgroup = (`columns` outputs, sixteen tokens).  Products with rows = outputs and columns = tokens: a lane holds token lane % 16 and, of
// 32 outputs in two products, eight neighbouring ones (row 4 g + j of product p is output 8 g + 4 p + j).
template <int DT, int OUT>
__global__ __launch_bounds__(256) void lowrank_out_kernel(LowrankArgs a)
{
    constexpr int PIECES = DT == RCP_F16 ? 2 : 3;
    extern __shared__ float sums[];  // t of the tile: [16][stride]
    const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m0 = static_cast<int>(blockIdx.y) * 16, padded = (a.r + 31) / 32 * 32, stride = padded + 4;
    const int id = lane < 16 ? lowrank_adapter(a, m0 + lane) : -1;
    const unsigned long long leaders = lowrank_leaders(id, 16);
    const int mine = __shfl(id, i, 64);
    for (int at = tid; at < 16 * padded; at += 256) {
        const int m = at / padded, rank = at - m * padded, adapter = lowrank_adapter(a, m0 + m);
        float s = 0.0f;
        if (adapter >= 0 && rank < a.r) {
            for (int k = 0; k < a.splits; ++k) s += a.part[(static_cast<size_t>(k) * a.M + m0 + m) * a.r + rank];
            s *= a.scaling[adapter];
        }
        sums[m * stride + rank] = s;
    }
    __syncthreads();
    int E = 14;  // binary16: the token's largest value becomes 2^13 .. 2^14
    if constexpr (DT == RCP_F16) {
        float top = 0.0f;
        for (int rank = 0; rank < padded; ++rank) top = fmaxf(top, fabsf(sums[i * stride + rank]));
        E = __builtin_amdgcn_frexp_expf(top);
    }
    const int end = min(a.N, (static_cast<int>(blockIdx.x) + 1) * a.columns), steps = padded / 32;
    const auto* const B = static_cast<const One<DT>*>(a.B);
    for (int n0 = static_cast<int>(blockIdx.x) * a.columns + 32 * wave; n0 < end; n0 += 128) {
        v4f total[2] = {v4f{0.0f, 0.0f, 0.0f, 0.0f}, v4f{0.0f, 0.0f, 0.0f, 0.0f}};
        size_t row[2];
#pragma unroll
        for (int p = 0; p < 2; ++p) row[p] = static_cast<size_t>(min(n0 + 8 * (i >> 2) + 4 * p + (i & 3), a.N - 1)) * a.r;
        for (unsigned long long rest = leaders; rest != 0; rest &= rest - 1) {
            const int adapter = __builtin_amdgcn_readlane(id, __builtin_ctzll(rest));
            const auto* const Ba = B + static_cast<size_t>(adapter) * a.N * a.r;
            v4f acc[2] = {v4f{0.0f, 0.0f, 0.0f, 0.0f}, v4f{0.0f, 0.0f, 0.0f, 0.0f}};
            for (int s = 0; s < steps; ++s) {
                const int rank = 32 * s + 8 * g;
                Eight<DT> b[2];
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    if (rank < a.r) b[p] = *reinterpret_cast<const Eight<DT>*>(Ba + row[p] + rank);
                    else
#pragma unroll
                        for (int e = 0; e < 8; ++e) b[p][e] = static_cast<One<DT>>(0.0f);
                }
                float t[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    t[e] = sums[i * stride + rank + e];
                    if constexpr (DT == RCP_F16) t[e] = ldexpf(t[e], 14 - E);
                }
#pragma unroll
                for (int q = 0; q < PIECES; ++q) {
                    const Eight<DT> piece = lowrank_round<DT>(t);
#pragma unroll
                    for (int p = 0; p < 2; ++p) acc[p] = lowrank_mfma<DT>(b[p], piece, acc[p]);
                }
            }
            // only the tokens of this adapter take its products: an infinity in one request's adapter stays with that request
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int j = 0; j < 4; ++j) total[p][j] = mine == adapter ? acc[p][j] : total[p][j];
        }
        const int m = m0 + i;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int n = n0 + 8 * g + 4 * p;
            if (m < a.M && n < end) {
                float v[4];
                lowrank_load4<OUT>(a.base, static_cast<size_t>(m) * a.N + n, v);
                if (mine >= 0) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] += DT == RCP_F16 ? ldexpf(total[p][j], E - 14) : total[p][j];
                }
                lowrank_store4<OUT>(a.out, static_cast<size_t>(m) * a.N + n, v);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------
struct LowrankPlan {
    int token_tiles, tiles, chunk, splits, slots, columns;  // token_tiles: sixteens of tokens of a workgroup of the first kernel
};

static LowrankPlan lowrank_plan(int M, int N, int K)
{
    LowrankPlan p;
    p.token_tiles = M > 64 ? 4 : 1;
    p.tiles = (M + 16 * p.token_tiles - 1) / (16 * p.token_tiles);
    const int least = 512, most = (K + least - 1) / least;  // splits of 512 columns and more
    int splits = 512 / p.tiles;
    splits = splits < 1 ? 1 : splits > most ? most : splits;
    p.chunk = ((K + splits - 1) / splits + 127) / 128 * 128;
    p.splits = (K + p.chunk - 1) / p.chunk;
    p.slots = p.token_tiles > 1 ? 1 : M < 16 ? M : 16;
    const int tiles16 = (M + 15) / 16, parts = 1024 / tiles16 > 0 ? 1024 / tiles16 : 1;
    p.columns = ((N + parts - 1) / parts + 127) / 128 * 128;
    return p;
}

size_t lowrank_workspace_bytes(int M, int N, int K, int r)
{
    const size_t bytes = static_cast<size_t>(lowrank_plan(M, N, K).splits) * M * r * sizeof(float);
    return bytes > 16 ? bytes : 16;
}

int launch_lowrank(const void* x, rcp_dtype dt, int M, int N, int K, int r, int adapters, const void* A, const void* B, const int* which,
                   const float* scaling, const void* base, void* out, rcp_dtype out_dt, void* workspace, hipStream_t st)
{
    const LowrankPlan p = lowrank_plan(M, N, K);
    LowrankArgs a = {x, A, B, base, which, scaling, out, static_cast<float*>(workspace), M, N, K, r, adapters, p.splits, p.chunk, p.slots, p.columns};
    const dim3 grid(static_cast<unsigned>(p.splits), static_cast<unsigned>(p.slots), static_cast<unsigned>(p.tiles));
    auto in = [&](auto kernel) { enqueue(kernel, grid, 256, 0, st, a); };
    auto form = [&](auto type, auto tokens) {
        constexpr int DT = decltype(type)::value, TT = decltype(tokens)::value;
        if (r <= 16) in(&lowrank_in_kernel<DT, TT, 1>);
        else if (r <= 32) in(&lowrank_in_kernel<DT, TT, 2>);
        else in(&lowrank_in_kernel<DT, TT, 4>);
    };
    using F16 = std::integral_constant<int, RCP_F16>;
    using BF16 = std::integral_constant<int, RCP_BF16>;
    using T1 = std::integral_constant<int, 1>;
    using T4 = std::integral_constant<int, 4>;
    if (dt == RCP_F16) p.token_tiles == 4 ? form(F16{}, T4{}) : form(F16{}, T1{});
    else p.token_tiles == 4 ? form(BF16{}, T4{}) : form(BF16{}, T1{});
    if (int rc = check_launch("rcp_lowrank_add")) return rc;
    const dim3 grid2(static_cast<unsigned>((N + p.columns - 1) / p.columns), static_cast<unsigned>((M + 15) / 16));
    const size_t lds = 16 * ((r + 31) / 32 * 32 + 4) * sizeof(float);
    auto launch = [&](auto kernel) { enqueue(kernel, grid2, 256, lds, st, a); };
    auto second = [&](auto type) {
        constexpr int DT = decltype(type)::value;
        if (out_dt == RCP_F32) launch(&lowrank_out_kernel<DT, RCP_F32>);
        else if (out_dt == RCP_F16) launch(&lowrank_out_kernel<DT, RCP_F16>);
        else launch(&lowrank_out_kernel<DT, RCP_BF16>);
    };
    if (dt == RCP_F16) second(F16{});
    else second(BF16{});
    return check_launch("rcp_lowrank_add(second)");
}

}  // namespace rcp
