// Low-rank adapters of many requests beside a shared projection:
//   out[m] = base[m] + scaling[a] (x[m] A[a]^T) B[a]^T,   a = which[m]   (no adapter: out[m] = base[m])
// A is [adapters][r][K], B [adapters][N][r], in the 16-bit type of x.
//
// Two launches, since every output needs the whole inner sum.  The first forms t = x A^T on the matrix cores, split along K; its partial
// sums go to the workspace, in binary32 and in a fixed order (no atomics).  The second adds them up and multiplies by B.  A tile of
// tokens is multiplied once for each adapter that one of its tokens has (a "leader" is the first token of the tile with that adapter), and
// a token keeps the products of its own one.
// t has 32 bits and the matrix cores take 16: it goes in as two binary16 numbers, scaled by a power of two per token (22 bits
// of every value down to 2^-16 of the token's largest, smaller ones off by 2^-38 of that at most), or as three bfloat16 numbers (24 bits).
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
    int M, N, K, r, adapters, splits, chunk, slots;  // chunk: columns of a split; slots: leaders side by side in the first kernel
};

// the adapter of token m, -1 for none
__device__ __forceinline__ int lowrank_adapter(const LowrankArgs& a, int m)
{
    const int id = m < a.M ? a.which[m] : -1;
    return static_cast<unsigned>(id) < static_cast<unsigned>(a.adapters) ? id : -1;
}

// The lanes among the first `tokens` whose adapter no lower lane has; `order`: how many of those come before the one of a lane's own adapter.
__device__ __forceinline__ unsigned long long lowrank_leaders(int id, int tokens, int& order)
{
    unsigned long long rest = __builtin_amdgcn_ballot_w64(id >= 0), leaders = 0;
    if (tokens < 64) rest &= (1ull << tokens) - 1;
    order = 0;
    for (int n = 0; rest != 0; ++n) {  // at most one round for each lane
        const int at = __builtin_ctzll(rest);
        const bool same = id == __builtin_amdgcn_readlane(id, at);
        leaders |= 1ull << at;
        rest &= ~__builtin_amdgcn_ballot_w64(same);
        order = same ? n : order;
    }
    return leaders;
}

// Few tokens: workgroup = (split of K, slot of leaders, sixteen tokens); each wavefront sums a quarter of the split, from registers, two blocks of
// two steps ahead of the products (rows = ranks, columns = tokens).  Bound by the launch and the chain adapter -> rows: 16 tokens with an adapter each, K = 4096,
// r = 16: 4.5 us for 2.2 MB; one token, K = 2048, r = 8: 2.6 us.
template <int DT, int NR>
__global__ __launch_bounds__(256) void lowrank_few_in_kernel(LowrankArgs a)
{
    constexpr int U = 2, BLOCK = LOWRANK_STEP * U;
    __shared__ float red[3][NR][256];
    const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m0 = static_cast<int>(blockIdx.y) * 16;
    const int id = lane < 16 ? lowrank_adapter(a, m0 + lane) : -1;
    int order;
    unsigned long long leaders = lowrank_leaders(id, 16, order);
    const int quarter = a.chunk / 4, k0 = static_cast<int>(blockIdx.x) * a.chunk + quarter * wave, k1 = min(a.K, k0 + quarter);
    const auto* const x = static_cast<const One<DT>*>(a.x) + static_cast<size_t>(min(m0 + i, a.M - 1)) * a.K + 8 * g;  // beyond the last token: that again
    for (int slot = 0; leaders != 0; ++slot, leaders &= leaders - 1) {
        if (slot % a.slots != static_cast<int>(blockIdx.z)) continue;  // uniform
        const int adapter = __builtin_amdgcn_readlane(id, __builtin_ctzll(leaders));
        const auto* const A = static_cast<const One<DT>*>(a.A) + static_cast<size_t>(adapter) * a.r * a.K + 8 * g;
        for (int r0 = 0; r0 < a.r; r0 += 16 * NR) {
            v4f acc[NR];
            const One<DT>* rows[NR];
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                acc[n] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
                rows[n] = A + static_cast<size_t>(min(r0 + 16 * n + i, a.r - 1)) * a.K;
            }
            Eight<DT> xv[2][U], av[2][U][NR];
            auto load = [&](int buf, int k) {  // columns beyond the end: the last ones again, which no product takes
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int at = min(k + LOWRANK_STEP * u, k1 - LOWRANK_STEP);
                    xv[buf][u] = *reinterpret_cast<const Eight<DT>*>(x + at);
#pragma unroll
                    for (int n = 0; n < NR; ++n) av[buf][u][n] = *reinterpret_cast<const Eight<DT>*>(rows[n] + at);
                }
            };
            auto take = [&](int buf, int k) {
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (k + LOWRANK_STEP * u < k1) {  // uniform
#pragma unroll
                        for (int n = 0; n < NR; ++n) acc[n] = lowrank_mfma<DT>(av[buf][u][n], xv[buf][u], acc[n]);
                    }
            };
            if (k0 < k1) {
                load(0, k0);
                load(1, k0 + BLOCK);
                for (int k = k0; k < k1; k += 2 * BLOCK) {
                    take(0, k);
                    if (k + 2 * BLOCK < k1) load(0, k + 2 * BLOCK);
                    take(1, k + BLOCK);
                    if (k + 3 * BLOCK < k1) load(1, k + 3 * BLOCK);
                }
            }
            if (wave > 0) {
#pragma unroll
                for (int n = 0; n < NR; ++n) *reinterpret_cast<v4f*>(&red[wave - 1][n][4 * lane]) = acc[n];
            }
            __syncthreads();
            if (wave == 0 && __shfl(id, i, 64) == adapter) {
                float* const to = a.part + (static_cast<size_t>(blockIdx.x) * a.M + m0 + i) * a.r;
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    const int rank = r0 + 16 * n + 4 * g;
#pragma unroll
                    for (int w = 0; w < 3; ++w) acc[n] += *reinterpret_cast<const v4f*>(&red[w][n][4 * lane]);
                    if (rank < a.r) *reinterpret_cast<v4f*>(to + rank) = acc[n];
                }
            }
            __syncthreads();
        }
    }
}

// Many tokens: workgroup = (split of K, slot of leaders, 64 tokens), sixteen tokens of each wavefront.  Bound by the memory x comes from (2001 tokens, K = 14336,
// r = 64, bfloat16: 57 MB in 16.8 us, 3.4 TB/s).  x and A come through LDS in stages of 64 columns, so that the four wavefronts share A and a load takes 128 bytes
// of a row; three stages, two under way while one is multiplied (18.7 us with all loads ended before each read; four and five stages measure the same).  Piece p
// (16 bytes) of row n stands at place p ^ (n / 2 % 8): the sixteen rows that are read together, 128 bytes each, fall into different banks.
constexpr int LOWRANK_STAGE = 64, LOWRANK_STAGES = 3;

__device__ __forceinline__ void lowrank_to_lds(__amdgpu_buffer_rsrc_t from, unsigned char* to, int offset)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, offset, 0, 0, 0);
}

__device__ __forceinline__ uint32_t lowrank_lds(const unsigned char* p)
{
    return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const unsigned char*)p));
}

// One 16-byte piece of a token and NR pieces of sixteen ranks each, 2048 bytes apart, out of LDS; they have arrived when this returns.  (Written out, because the
// compiler lets all loads into LDS end before a read of its own there.)
template <int NR>
__device__ __forceinline__ void lowrank_read(uint32_t x, uint32_t a, u32x4& xv, u32x4 (&av)[NR])
{
    if constexpr (NR == 1)
        asm volatile("ds_read_b128 %0, %2\n\tds_read_b128 %1, %3\n\ts_waitcnt lgkmcnt(0)" : "=&v"(xv), "=&v"(av[0]) : "v"(x), "v"(a) : "memory");
    else if constexpr (NR == 2)
        asm volatile("ds_read_b128 %0, %3\n\tds_read_b128 %1, %4\n\tds_read_b128 %2, %4 offset:2048\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(xv), "=&v"(av[0]), "=&v"(av[1]) : "v"(x), "v"(a) : "memory");
    else
        asm volatile("ds_read_b128 %0, %5\n\tds_read_b128 %1, %6\n\tds_read_b128 %2, %6 offset:2048\n\tds_read_b128 %3, %6 offset:4096\n\t"
                     "ds_read_b128 %4, %6 offset:6144\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(xv), "=&v"(av[0]), "=&v"(av[1]), "=&v"(av[2]), "=&v"(av[3]) : "v"(x), "v"(a) : "memory");
}

template <int DT, int NR>
__global__ __launch_bounds__(256) void lowrank_many_in_kernel(LowrankArgs a)
{
    constexpr int ROW = LOWRANK_STAGE * 2;  // bytes
    __shared__ __attribute__((aligned(16))) unsigned char xs[LOWRANK_STAGES][64 * ROW], as[LOWRANK_STAGES][16 * NR * ROW];
    const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m0 = static_cast<int>(blockIdx.y) * 64;
    const int id = lowrank_adapter(a, m0 + lane);
    int order;
    unsigned long long leaders = lowrank_leaders(id, 64, order);
    const int k0 = static_cast<int>(blockIdx.x) * a.chunk, k1 = min(a.K, k0 + a.chunk);
    const int mine = __shfl(id, 16 * wave + i, 64);
    const auto resource = [](const void* p, size_t at, size_t rows, size_t K) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(p)) + at * K * 2, 0, static_cast<int>(rows * K * 2), 0x00020000);
    };
    const __amdgpu_buffer_rsrc_t xr = resource(a.x, m0, min(64, a.M - m0), a.K);
    for (int slot = 0; leaders != 0; ++slot, leaders &= leaders - 1) {
        if (slot % a.slots != static_cast<int>(blockIdx.z)) continue;  // uniform
        const int adapter = __builtin_amdgcn_readlane(id, __builtin_ctzll(leaders));
        for (int r0 = 0; r0 < a.r; r0 += 16 * NR) {
            const int ranks = min(16 * NR, a.r - r0);
            const __amdgpu_buffer_rsrc_t ar = resource(a.A, static_cast<size_t>(adapter) * a.r + r0, ranks, a.K);  // ranks beyond the last read zeros
            constexpr int X_LOADS = 2, A_LOADS = NR == 1 ? 1 : NR / 2;
            auto stage = [&](int k, int buf) {  // eight rows a load; beyond the last column: zeros that nobody takes, but as many loads
                const int piece = lane & 7, beyond = k < k1 ? 0 : 1 << 30;
#pragma unroll
                for (int y = 0; y < X_LOADS; ++y) {
                    const int row = 16 * wave + 8 * y + (lane >> 3);
                    lowrank_to_lds(xr, &xs[buf][(16 * wave + 8 * y) * ROW], ((row * a.K + k) * 2 + 16 * (piece ^ (row >> 1 & 7))) | beyond);
                }
#pragma unroll
                for (int y = 0; y < A_LOADS; ++y) {  // (sixteen ranks: two wavefronts each load the same eight)
                    const int first = NR == 1 ? 8 * (wave & 1) : 4 * NR * wave + 8 * y, row = first + (lane >> 3);
                    lowrank_to_lds(ar, &as[buf][first * ROW], ((row * a.K + k) * 2 + 16 * (piece ^ (row >> 1 & 7))) | beyond);
                }
            };
            v4f acc[NR];
#pragma unroll
            for (int n = 0; n < NR; ++n) acc[n] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int x = 0; x < LOWRANK_STAGES - 1; ++x) stage(k0 + LOWRANK_STAGE * x, x);
            for (int k = k0, buf = 0; k < k1; k += LOWRANK_STAGE) {
                // this wavefront's part of the stage is in LDS once only the later ones' loads are outstanding,
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_waitcnt(((X_LOADS + A_LOADS) * (LOWRANK_STAGES - 2)) | (7 << 4) | (15 << 8));
                asm volatile("" ::: "memory");
                __builtin_amdgcn_s_barrier();  // then everybody's is, and the stage before has been read: reads wait for themselves
                asm volatile("" ::: "memory");
                __builtin_amdgcn_sched_barrier(0);
                stage(k + LOWRANK_STAGE * (LOWRANK_STAGES - 1), buf == 0 ? LOWRANK_STAGES - 1 : buf - 1);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int s = 0; s < LOWRANK_STAGE / LOWRANK_STEP; ++s) {
                    if (k + LOWRANK_STEP * s >= k1) break;  // uniform
                    const int at = ((4 * s + g) ^ (i >> 1)) * 16;
                    u32x4 xv, av[NR];
                    lowrank_read<NR>(lowrank_lds(&xs[buf][(16 * wave + i) * ROW + at]), lowrank_lds(&as[buf][i * ROW + at]), xv, av);
#pragma unroll
                    for (int n = 0; n < NR; ++n) acc[n] = lowrank_mfma<DT>(__builtin_bit_cast(Eight<DT>, av[n]), __builtin_bit_cast(Eight<DT>, xv), acc[n]);
                }
                buf = buf == LOWRANK_STAGES - 1 ? 0 : buf + 1;
            }
            __builtin_amdgcn_s_waitcnt(0);  // nothing is on its way into LDS any more
            if (mine == adapter) {
                float* const to = a.part + (static_cast<size_t>(blockIdx.x) * a.M + m0 + 16 * wave + i) * a.r;
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    const int rank = r0 + 16 * n + 4 * g;
                    if (rank < a.r) *reinterpret_cast<v4f*>(to + rank) = acc[n];
                }
            }
            __syncthreads();  // the next round fills the buffers anew
        }
    }
}

// four results of a row from index i on
template <int DT>
__device__ __forceinline__ void lowrank_store4(void* p, size_t i, const float* v)
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

template <int DT>
using Raw4 = std::conditional_t<DT == RCP_F32, float4, uint2>;

template <int DT>
__device__ __forceinline__ Raw4<DT> lowrank_load4(const void* p, size_t i)
{
    return *reinterpret_cast<const Raw4<DT>*>(static_cast<const char*>(p) + i * (DT == RCP_F32 ? 4 : 2));
}

template <int DT>
__device__ __forceinline__ void lowrank_add4(const Raw4<DT>& x, float* v)
{
    if constexpr (DT == RCP_F32) {
        v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
    } else {
        const uint16_t h[4] = {static_cast<uint16_t>(x.x), static_cast<uint16_t>(x.x >> 16), static_cast<uint16_t>(x.y), static_cast<uint16_t>(x.y >> 16)};
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += DT == RCP_F16 ? half_bits_to_float(h[e]) : bf16_bits_to_float(h[e]);
    }
}

// scaling t of a tile of sixteen tokens in LDS, as the operands' pieces, and E of the binary16 scale: a token's largest value becomes 2^13 .. 2^14
template <int DT, int STEPS>
struct LowrankTerms {
    static constexpr int PIECES = DT == RCP_F16 ? 2 : 3;
    One<DT> piece[PIECES][16][32 * STEPS + 8];
    int E[16];
};

// Sums the splits (zeros for ranks beyond the last and tokens without an adapter): sixteen lanes a token, neighbouring ranks a lane, so that the loads of eight splits
// are eight instructions, under way together, and no value is converted twice in the workgroup.
template <int DT, int STEPS>
__device__ __forceinline__ void lowrank_total(const LowrankArgs& a, int m0, int id, LowrankTerms<DT, STEPS>& to)
{
    constexpr int V = 2 * STEPS, U = 8;
    typedef float Part __attribute__((ext_vector_type(V), aligned(V == 2 ? 8 : 16)));
    typedef One<DT> Piece __attribute__((ext_vector_type(V)));
    const int token = static_cast<int>(threadIdx.x) / 16, rank = static_cast<int>(threadIdx.x) % 16 * V;
    const int mine = __shfl(id, token, 64);
    const float scale = a.scaling[max(mine, 0)];
    // what no token has is read, too (it lies in the workspace), and dropped: no branches between the loads
    const float* const from = a.part + static_cast<size_t>(min(m0 + token, a.M - 1)) * a.r + min(rank, a.r - V);
    const size_t next = static_cast<size_t>(a.M) * a.r;
    Part t = {};
    for (int k = 0; k < a.splits; k += U) {
        Part x[U];
#pragma unroll
        for (int y = 0; y < U; ++y) x[y] = *reinterpret_cast<const Part*>(from + min(k + y, a.splits - 1) * next);
#pragma unroll
        for (int y = 0; y < U; ++y)
            if (k + y < a.splits) t += x[y];  // uniform
    }
#pragma unroll
    for (int e = 0; e < V; ++e) t[e] = mine >= 0 && rank < a.r ? t[e] * scale : 0.0f;
    if constexpr (DT == RCP_F16) {
        float top = 0.0f;
#pragma unroll
        for (int e = 0; e < V; ++e) top = fmaxf(top, fabsf(t[e]));
        auto turned = [](float v, auto by) {  // of the lane so many further in the row of sixteen
            return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x120 + decltype(by)::value, 0xf, 0xf, true));
        };
        top = fmaxf(top, turned(top, std::integral_constant<int, 8>{}));
        top = fmaxf(top, turned(top, std::integral_constant<int, 4>{}));
        top = fmaxf(top, turned(top, std::integral_constant<int, 2>{}));
        top = fmaxf(top, turned(top, std::integral_constant<int, 1>{}));
        const int E = __builtin_amdgcn_frexp_expf(top);
#pragma unroll
        for (int e = 0; e < V; ++e) t[e] = ldexpf(t[e], 14 - E);
        if (rank == 0) to.E[token] = E;
    }
#pragma unroll
    for (int q = 0; q < LowrankTerms<DT, STEPS>::PIECES; ++q) {
        Piece h;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            h[e] = static_cast<One<DT>>(t[e]);
            t[e] -= static_cast<float>(h[e]);
        }
        *reinterpret_cast<Piece*>(&to.piece[q][token][rank]) = h;
    }
}

// the t of token lane % 16 as operands; returns E
template <int DT, int STEPS, int PIECES>
__device__ __forceinline__ int lowrank_pieces(const LowrankTerms<DT, STEPS>& from, Eight<DT> (&piece)[STEPS][PIECES])
{
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
#pragma unroll
        for (int q = 0; q < PIECES; ++q) piece[s][q] = *reinterpret_cast<const Eight<DT>*>(&from.piece[q][i][32 * s + 8 * g]);
    return DT == RCP_F16 ? from.E[i] : 14;
}

// rows of B (ranks 32 s + 8 g ..) times t; ranks beyond the last are zeros on both sides
template <int DT, int STEPS, int PIECES>
__device__ __forceinline__ v4f lowrank_product(int r, int g, Eight<DT> (&b)[STEPS], const Eight<DT> (&piece)[STEPS][PIECES])
{
    v4f acc = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        if (32 * s >= r) break;  // uniform
        if (32 * s + 8 * g >= r) b[s] = Eight<DT>{};
#pragma unroll
        for (int q = 0; q < PIECES; ++q) acc = lowrank_mfma<DT>(b[s], piece[s][q], acc);
    }
    return acc;
}

// Few tokens, so that many have an adapter of their own: workgroup = (32 outputs, sixteen tokens); wavefront w takes the adapters w, w + 4, ... of the tile and
// writes the rows of their tokens.  Products with rows = outputs, columns = tokens: a lane holds token lane % 16 and four neighbouring outputs.  16 tokens beside
// 12288 outputs, r = 16: 5.3 us for 7 MB; one token beside 2048: 3.6 us, again the launch and a chain of loads.
template <int DT, int OUT, int STEPS>
__global__ __launch_bounds__(256) void lowrank_few_out_kernel(LowrankArgs a)
{
    constexpr int PIECES = DT == RCP_F16 ? 2 : 3, TOGETHER = 4 / STEPS;  // adapters whose rows of B are under way at a time
    __shared__ __attribute__((aligned(16))) LowrankTerms<DT, STEPS> terms;
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
    const int m0 = static_cast<int>(blockIdx.y) * 16, n0 = static_cast<int>(blockIdx.x) * 32;
    const int id = lane < 16 ? lowrank_adapter(a, m0 + lane) : -1;
    int order;
    unsigned long long leaders = lowrank_leaders(id, 16, order);
    const int mine = __shfl(id, i, 64), at = __shfl(order, i, 64);
    for (int w = 0; w < wave; ++w) leaders &= leaders - 1;  // this wavefront's first one
    const bool writes = m0 + i < a.M && wave == ((mine >= 0 ? at : i) & 3);
    const auto* const B = static_cast<const One<DT>*>(a.B);
    Eight<DT> b[TOGETHER][2][STEPS];
    int adapter[TOGETHER];
    auto load = [&](unsigned long long from) {
#pragma unroll
        for (int u = 0; u < TOGETHER; ++u) {
            adapter[u] = from != 0 ? __builtin_amdgcn_readlane(id, __builtin_ctzll(from)) : -1;
            if (adapter[u] >= 0) {  // uniform
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const auto* const row = B + (static_cast<size_t>(adapter[u]) * a.N + min(n0 + 16 * p + i, a.N - 1)) * a.r;
#pragma unroll
                    for (int s = 0; s < STEPS; ++s) b[u][p][s] = *reinterpret_cast<const Eight<DT>*>(row + min(32 * s + 8 * g, a.r - 8));
                }
            }
            for (int w = 0; w < 4; ++w) from &= from - 1;
        }
        return from;
    };
    leaders = load(leaders);
    Raw4<OUT> base[2];
    const size_t to = static_cast<size_t>(m0 + i) * a.N + n0 + 4 * g;
#pragma unroll
    for (int p = 0; p < 2; ++p)
        if (writes && n0 + 16 * p + 4 * g < a.N) base[p] = lowrank_load4<OUT>(a.base, to + 16 * p);
    lowrank_total<DT, STEPS>(a, m0, id, terms);
    __syncthreads();
    Eight<DT> piece[STEPS][PIECES];
    const int E = lowrank_pieces<DT, STEPS, PIECES>(terms, piece);
    v4f total[2] = {v4f{0.0f, 0.0f, 0.0f, 0.0f}, v4f{0.0f, 0.0f, 0.0f, 0.0f}};
    for (;;) {
#pragma unroll
        for (int u = 0; u < TOGETHER; ++u) {
            if (adapter[u] < 0) break;  // uniform
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const v4f x = lowrank_product<DT, STEPS, PIECES>(a.r, g, b[u][p], piece);
                // only the tokens of this adapter take its products: an infinity in one request's adapter stays with that request
#pragma unroll
                for (int j = 0; j < 4; ++j) total[p][j] = mine == adapter[u] ? x[j] : total[p][j];
            }
        }
        if (leaders == 0) break;  // uniform
        leaders = load(leaders);
    }
#pragma unroll
    for (int p = 0; p < 2; ++p)
        if (writes && n0 + 16 * p + 4 * g < a.N) {
            float v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = DT == RCP_F16 ? ldexpf(total[p][j], E - 14) : total[p][j];
            lowrank_add4<OUT>(base[p], v);
            lowrank_store4<OUT>(a.out, to + 16 * p, v);
        }
}

// Many tokens: workgroup = (512 outputs, sixteen tokens), 128 outputs of each wavefront.  The products pass through LDS, so that base and out are read and
// written in kilobytes of a row: in the products' own order (32 bytes of each of sixteen rows) 2001 tokens of 4096 outputs took 30 us.  So does B of more than 32
// ranks before them: a cache serves what neighbouring lanes read together, and in the products' order those are different rows (2001 tokens, rank 64: 25 us
// instead of 22; but 300 tokens, tiles of sixteen adapters each, 81 us instead of 86: a wait for each of them).
// Piece p (16 bytes) of row n of B stands at place p ^ (n / (16 / P) % P) of the P = r / 8 of its row, so that sixteen rows fall into different banks; where P is no
// power of two, in order.
constexpr int LOWRANK_COLUMNS = 512;

template <int DT, int OUT, int STEPS>
__global__ __launch_bounds__(256) void lowrank_many_out_kernel(LowrankArgs a)
{
    constexpr int PIECES = DT == RCP_F16 ? 2 : 3, ROW = 128 + 4, AT_ONCE = 8 / STEPS;  // products whose rows of B are in LDS at a time: 8 KB and less
    __shared__ __attribute__((aligned(16))) float block[4][16 * ROW];  // of each wavefront: its rows of B, then its products; before them, t
    auto& terms = *reinterpret_cast<LowrankTerms<DT, STEPS>*>(&block[0][0]);
    static_assert(sizeof(terms) <= sizeof(block) && sizeof(block[0]) >= 8192, "t and B lie where the products come");
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
    const int m0 = static_cast<int>(blockIdx.x) * 16, n0 = static_cast<int>(blockIdx.y) * LOWRANK_COLUMNS;
    if (m0 >= a.M) return;  // the grid's width is a multiple of eight
    const int id = lane < 16 ? lowrank_adapter(a, m0 + lane) : -1;
    int order;
    unsigned long long leaders = lowrank_leaders(id, 16, order);
    const int mine = __shfl(id, i, 64);
    Eight<DT> piece[STEPS][PIECES];
    int E = 14;
    if (leaders != 0) {  // uniform over the workgroup
        lowrank_total<DT, STEPS>(a, m0, id, terms);
        __syncthreads();
        E = lowrank_pieces<DT, STEPS, PIECES>(terms, piece);
        __syncthreads();
    }
    const int first = n0 + 128 * wave;
    const int P = a.r / 8, bits = (P & (P - 1)) == 0 ? P - 1 : 0, down = 4 - (31 - __builtin_clz(static_cast<unsigned>(P)));  // P <= 16
    unsigned char* const rows = reinterpret_cast<unsigned char*>(&block[wave][0]);
    v4f total[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) total[c] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    for (; leaders != 0; leaders &= leaders - 1) {
        const int adapter = __builtin_amdgcn_readlane(id, __builtin_ctzll(leaders));
        const char* const B = static_cast<const char*>(a.B) + (static_cast<size_t>(adapter) * a.N + min(first, a.N - 1)) * a.r * 2;
        const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(B), 0, max(0, min(128, a.N - first)) * a.r * 2, 0x00020000);
#pragma unroll
        for (int c0 = 0; c0 < 8; c0 += AT_ONCE) {
            Eight<DT> b[AT_ONCE][STEPS];
            if constexpr (STEPS == 1) {
#pragma unroll
                for (int c = 0; c < AT_ONCE; ++c) {
                    const auto* const row = static_cast<const One<DT>*>(a.B) + (static_cast<size_t>(adapter) * a.N + min(first + 16 * c + i, a.N - 1)) * a.r;
                    b[c][0] = *reinterpret_cast<const Eight<DT>*>(row + min(8 * g, a.r - 8));
                }
            } else {
                for (int y = 0; y < (AT_ONCE * 16 * P + 63) / 64; ++y) {
                    const int at = 64 * y + lane, row = at / P, place = at - row * P;
                    lowrank_to_lds(from, rows + 1024 * y, ((16 * c0 + row) * P + (place ^ (row >> down & bits))) * 16);
                }
                __builtin_amdgcn_s_waitcnt(0);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int c = 0; c < AT_ONCE; ++c) {
                if constexpr (STEPS > 1)
#pragma unroll
                    for (int s = 0; s < STEPS; ++s) {
                        const int row = 16 * c + i, p = min(4 * s + g, P - 1);
                        b[c][s] = *reinterpret_cast<const Eight<DT>*>(rows + (row * P + (p ^ (row >> down & bits))) * 16);
                    }
                v4f x = lowrank_product<DT, STEPS, PIECES>(a.r, g, b[c], piece);
                if constexpr (DT == RCP_F16)
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] = ldexpf(x[j], E - 14);
                // an infinity in one request's adapter stays with that request
                if constexpr (STEPS == 1) {
                    if (mine == adapter) *reinterpret_cast<v4f*>(&block[wave][i * ROW + 16 * c + 4 * g]) = x;
                } else
#pragma unroll
                    for (int j = 0; j < 4; ++j) total[c0 + c][j] = mine == adapter ? x[j] : total[c0 + c][j];
            }
            if constexpr (STEPS > 1) {  // all read, before the next ones come
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_waitcnt(0);
            }
        }
    }
    // rows wave, wave + 4, ... of the tile, eight outputs a lane
    Raw4<OUT> base[4][2];
    const int n = n0 + 8 * lane;
#pragma unroll
    for (int y = 0; y < 4; ++y)
#pragma unroll
        for (int p = 0; p < 2; ++p)
            if (m0 + 4 * y + wave < a.M && n + 4 * p < a.N) base[y][p] = lowrank_load4<OUT>(a.base, static_cast<size_t>(m0 + 4 * y + wave) * a.N + n + 4 * p);
    if constexpr (STEPS > 1)
#pragma unroll
        for (int c = 0; c < 8; ++c) *reinterpret_cast<v4f*>(&block[wave][i * ROW + 16 * c + 4 * g]) = total[c];
    __syncthreads();
#pragma unroll
    for (int y = 0; y < 4; ++y) {
        const int row = 4 * y + wave;
        const bool adds = __shfl(id, row, 64) >= 0;  // uniform
#pragma unroll
        for (int p = 0; p < 2; ++p)
            if (m0 + row < a.M && n + 4 * p < a.N) {
                float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                if (adds) *reinterpret_cast<v4f*>(v) = *reinterpret_cast<const v4f*>(&block[lane >> 4][row * ROW + 8 * i + 4 * p]);
                lowrank_add4<OUT>(base[y][p], v);
                lowrank_store4<OUT>(a.out, static_cast<size_t>(m0 + row) * a.N + n + 4 * p, v);
            }
    }
}

// ---------------------------------------------------------------------------------------
struct LowrankPlan {
    bool many;
    int tiles, chunk, splits, slots;  // of the first kernel
};

// Which kernels: the host does not see how many adapters a tile has.  Those of few tokens are ahead by far with an adapter each, those of many with one for all, and the second
// difference grows with the outputs.  4096 x 4096, rank 16, bfloat16, few and many: 128 tokens of one adapter 7.5 and 8.6 us, of an adapter each 14 and 60; 256 tokens 9.9 and 8.8, 25 and 60.
// 14336 x 4096, rank 16: 128 tokens 12.3 and 9.0, 24 and 61; 256 tokens 19.6 and 9.9, 43 and 63.
// Splits: 512 columns and more (one token of 4096 columns, both kernels: 5.9 us; 256 and more 6.4, 1024 and more 6.4; 16 tokens of an adapter each 8.9, 9.4, 9.7).
// Leaders side by side: sixteen for few tokens, as many as a tile has (16 tokens of an adapter each, 4096 x 4096: 8.9 us; 8 10.1, 4 12.7); four for many (2001 tokens of five adapters
// beside 14336 columns 36.4 us; 2 36.6, 16 39.5, 1 37.5; but 300 tokens of an adapter each 61, 93, 41, 160).
static LowrankPlan lowrank_plan(int M, int K)
{
    LowrankPlan p;
    p.many = M > 128;
    p.tiles = p.many ? (M + 63) / 64 : (M + 15) / 16;
    const int least = 512, most = (K + least - 1) / least;
    int splits = 2 * num_compute_units() / p.tiles;
    splits = splits < 1 ? 1 : splits > most ? most : splits;
    const int unit = p.many ? LOWRANK_STAGE : least;
    p.chunk = ((K + splits - 1) / splits + unit - 1) / unit * unit;
    p.splits = (K + p.chunk - 1) / p.chunk;
    p.slots = p.many ? 4 : M < 16 ? M : 16;
    return p;
}

size_t lowrank_workspace_bytes(int M, int N, int K, int r)
{
    const size_t bytes = static_cast<size_t>(lowrank_plan(M, K).splits) * M * r * sizeof(float);
    return bytes > 16 ? bytes : 16;
}

int launch_lowrank(const void* x, rcp_dtype dt, int M, int N, int K, int r, int adapters, const void* A, const void* B, const int* which,
                   const float* scaling, const void* base, void* out, rcp_dtype out_dt, void* workspace, hipStream_t st)
{
    const LowrankPlan p = lowrank_plan(M, K);
    LowrankArgs a = {x, A, B, base, which, scaling, out, static_cast<float*>(workspace), M, N, K, r, adapters, p.splits, p.chunk, p.slots};
    // Most tiles have one adapter, so the slots behind the first come last; among the others, their workgroups, which end at once, would leave a part of the
    // compute units without work (2001 tokens, K = 14336, r = 64: 27 us instead of 18.8, before its reads waited for themselves).
    const dim3 grid(static_cast<unsigned>(p.splits), static_cast<unsigned>(p.tiles), static_cast<unsigned>(p.slots));
    const unsigned tiles = static_cast<unsigned>((M + 15) / 16);
    // Many tokens: workgroups go to the eight dies, each with a cache of its own, in turn; with a width of whole eights those that add up the same partial
    // sums meet on one die.
    const dim3 grid2 = p.many ? dim3((tiles + 7) / 8 * 8, static_cast<unsigned>((N + LOWRANK_COLUMNS - 1) / LOWRANK_COLUMNS))
                              : dim3(static_cast<unsigned>((N + 31) / 32), tiles);
    auto first = [&](auto type, auto ranks) {
        constexpr int DT = decltype(type)::value, NR = decltype(ranks)::value;
        if (p.many) enqueue(&lowrank_many_in_kernel<DT, NR>, grid, 256, 0, st, a);
        else enqueue(&lowrank_few_in_kernel<DT, NR>, grid, 256, 0, st, a);
    };
    auto second = [&](auto type, auto result, auto steps) {
        constexpr int DT = decltype(type)::value, OUT = decltype(result)::value, STEPS = decltype(steps)::value;
        if (p.many) enqueue(&lowrank_many_out_kernel<DT, OUT, STEPS>, grid2, 256, 0, st, a);
        else enqueue(&lowrank_few_out_kernel<DT, OUT, STEPS>, grid2, 256, 0, st, a);
    };
    using One = std::integral_constant<int, 1>;
    using Two = std::integral_constant<int, 2>;
    using Four = std::integral_constant<int, 4>;
    auto result = [&](auto type, auto out_type) {
        if (r <= 32) second(type, out_type, One{});
        else if (r <= 64) second(type, out_type, Two{});
        else second(type, out_type, Four{});
    };
    auto form = [&](auto type) {
        if (r <= 16) first(type, One{});
        else if (r <= 32) first(type, Two{});
        else first(type, Four{});
        if (out_dt == RCP_F32) result(type, std::integral_constant<int, RCP_F32>{});
        else if (out_dt == RCP_F16) result(type, std::integral_constant<int, RCP_F16>{});
        else result(type, std::integral_constant<int, RCP_BF16>{});
    };
    if (dt == RCP_F16) form(std::integral_constant<int, RCP_F16>{});
    else form(std::integral_constant<int, RCP_BF16>{});
    return check_launch("rcp_lowrank_add");
}

}  // namespace rcp
