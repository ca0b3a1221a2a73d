// Attention over the paged 8-bit cache.
//
//   out_r = sum_t 2^(score_rt) V_t / sum_t 2^(score_rt),   score_rt = log2(e) softmax_scale s_t (q_r . c_t),   V_t = s'_t c'_t
// over the tokens t that row r (a new token's query head) may see; c, c' are the E4M3 codes of a token, s, s' the scales of its page.
//
// Both products run transposed on the matrix cores: scores as (tokens x rows) = codes x queries, outputs as (elements x rows) = value
// codes transposed x weights.  A lane of a result then holds one row and several tokens, which is how the second product takes its weights:
// they stay in registers, and a row's maximum, sum and correction are values of its lanes.  The order of the products' inner index is
// free as long as both operands share it, so that keys enter in 16-byte pieces as they lie in memory and values in the tokens that a
// lane has weights of; value codes come back transposed from LDS (ds_read_b64_tr_b8: eight rows of sixteen bytes, a lane gets a column).
// A code becomes a binary16 number, exactly, half an instruction each.
//
// The query of a row enters scaled by a power of two, its largest element at 2^13 .. 2^14, as one binary16 number (a 16-bit query exactly down to 2^-27 of that) or two (a
// binary32 query, QP).  Not as E4M3 pieces, which would meet the codes without a conversion: the matrix cores' 8-bit products are not summed in binary32.  A product is cut off where its
// bits lie about 16 places below the largest one of an instruction (448 x 448 and 63 times 1 x 1 give 200760 instead of 200767), so that scores were off by up to 2^-15 of
// sum |q_d K_td|, and binary32 results of three chunks behind 5000 to 17003 tokens by 4.7e-5 instead of 4e-7.  (8192 tokens of 32 + 2 x 8 heads of 128, bfloat16: 533 us so, 568 us now.)
// A weight is 2^(score + log2 s' - m), at most 2^14; the codes of a page then enter the sum of outputs as they are, and its scale the sum of weights as 1 / s'.  The
// reference m of a row is so held against score + log2 s' that a page of a large scale and little attention does not push the others out of
// binary16; it moves only when a weight would leave the range.  A weight enters the product as two binary16 numbers, 22 bits of it.  One number (PP = 1) is off by up to
// 2^-11 of the weight, and only several tokens with bfloat16 results, whose own half step is 2^-8, take it: there the second product of each block costs a third (8192 tokens of 32 + 2 x 8 heads
// of 128: 571 us with one number, 755 with two) and changes the error against 64 bits by less than a hundredth.  For binary16 results it would be as large as the result's own rounding,
// and more where values cancel (three chunks behind 5000 to 17003 tokens, heads of 64: 62 us and an error of 2.3e-4 with one, 74 us and 2.1e-4 with two); single
// tokens hardly pay for it (16 sequences of up to 6000 tokens 27.4 us with one, 28.1 with two).  The range of binary16 ends below, too: with a row's largest weight at
// 2^9 .. 2^14, one number has its 11 bits down to 2^-23 of that (two their 22 bits down to 2^-12), and either form is off by 2^-34 of it at most.  Since a weight carries its page's
// scale, this can only show in elements that are zero in all tokens of a large weight times scale, beside tokens 2^12, or 2^23, times smaller.  Sums are binary32.
#include <math.h>

#include <type_traits>

#include "kv8.hpp"

namespace rcp {

constexpr float KV8_LOG2E = 1.44269504088896340736f;
constexpr float KV8_LOW = -3.0e38f;    // a reference that no score has raised yet (finite: differences with it stay numbers)
constexpr float KV8_TOP = 14.0f, KV8_REF = 9.0f;  // weights stay below 2^14; a raised reference puts the largest so far at 2^9
constexpr int KV8_TILE = 64;           // tokens a step
constexpr int KV8_EXTRA = 4;           // floats behind the D sums of a partial result: m, l

struct Kv8AttnArgs {
    Kv8Table t;
    const void* q;
    int q_dt, out_dt, rows, H_q, H_kv, rep;
    float softmax_scale;
    const unsigned char *k_codes, *v_codes;
    const float *k_scales, *v_scales;
    void* out;
    float* part;
    int2* cut;    // one token a sequence: first chunk and number of chunks of each
    int chunks;   // one token a sequence: chunks of the grid; otherwise splits of the cached tokens
    int tiles;    // several tokens: tiles of rows in the grid
};

__device__ __forceinline__ v8h kv8_halves(uint32_t a, uint32_t b)
{
    const v2h w = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, false), x = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, true);
    const v2h y = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, false), z = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, true);
    return v8h{w[0], w[1], x[0], x[1], y[0], y[1], z[0], z[1]};
}

// eight numbers as binary16, and what that leaves of them
__device__ __forceinline__ v8h kv8_round(const float (&v)[8])
{
    v8h h;
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = static_cast<_Float16>(v[e]);
    return h;
}
__device__ __forceinline__ void kv8_split(const float (&v)[8], v8h& h, v8h& rest)
{
    u32x4 w = __builtin_bit_cast(u32x4, kv8_round(v));
    // The rest in one instruction, a multiply-add that takes a half of a register for a factor.  (Hidden from the compiler: that the halves are v's, which it would convert a
    // second time, alone, and that the other factor is -1, since it would turn a subtraction into two instructions.)
    float minus = -1.0f;
    asm("" : "+v"(w));
    asm("" : "+s"(minus));
    h = __builtin_bit_cast(v8h, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) rest[e] = static_cast<_Float16>(fmaf(static_cast<float>(h[e]), minus, v[e]));
}

// eight query elements from index i on
__device__ __forceinline__ void kv8_query8(const Kv8AttnArgs& a, size_t i, float (&v)[8])
{
    if (a.q_dt == RCP_F32) load8_as_float<RCP_F32>(a.q, i, v);  // uniform
    else if (a.q_dt == RCP_F16) load8_as_float<RCP_F16>(a.q, i, v);
    else load8_as_float<RCP_BF16>(a.q, i, v);
}

__device__ __forceinline__ float kv8_swap32_max(float v)
{
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float kv8_swap16_max(float v)
{
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ void kv8_put(void* out, int dt, size_t i, float v)
{
    if (dt == RCP_F32) static_cast<float*>(out)[i] = v;  // uniform
    else if (dt == RCP_F16) static_cast<__half*>(out)[i] = round_to_half(v);
    else static_cast<__bf16*>(out)[i] = static_cast<__bf16>(v);
}

// four results in a 16-bit type
__device__ __forceinline__ uint2 kv8_pack4(int dt, const float (&v)[4])
{
    uint16_t h[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = dt == RCP_F16 ? __half_as_ushort(round_to_half(v[e])) : __builtin_bit_cast(uint16_t, static_cast<__bf16>(v[e]));
    return make_uint2(h[0] | static_cast<uint32_t>(h[1]) << 16, h[2] | static_cast<uint32_t>(h[3]) << 16);
}

// Scales are 2^-40 .. 2^120, and a page that was never written has 0 (and zeros for codes): the nearest of those stands in for it.
constexpr float KV8_LEAST = 0x1p-40f, KV8_MOST = 0x1p120f;
// The least factor of a score where a token is masked, by a score of -infinity: 0 (of a tiny query) would make that a NaN.  What it adds to the
// scores of other tokens, at most 2^-126 * 2^31, is nothing.
constexpr float KV8_NOT_ZERO = 0x1p-126f;

// the page that holds position `pos` of sequence b, -1 where there is none
__device__ __forceinline__ int kv8_page(const Kv8Table& t, const int* row, int pos)
{
    const int id = row[min(pos >> t.shift, t.width - 1)];
    return pos < t.capacity && static_cast<unsigned>(id) < static_cast<unsigned>(t.n_pages) ? id : -1;
}

// Sixteen consecutive cached tokens of a head, whose page is `id`, as a buffer that ends with the last of them below `end`: beyond, and without a
// page, reads give zero.
struct Kv8Block {
    size_t at;  // first token, in tokens of the pool
    int tokens;
};
__device__ __forceinline__ Kv8Block kv8_block(const Kv8Table& t, int H, int h, int id, int pos, int end)
{
    // (uniform, and in scalar registers: a buffer's bounds in vector registers would be a loop over their values)
    return {((static_cast<size_t>(max(id, 0)) * H + h) << t.shift) + (pos & ((1 << t.shift) - 1)),
            __builtin_amdgcn_readfirstlane(id < 0 ? 0 : kv8_clamp(end - pos, 0, 16))};
}

// 16 bytes of a lane from a buffer straight into LDS, lane after lane from `to` on (a function of its own: inside a template, the host's
// pass drops the kernel over it)
__device__ __forceinline__ void kv8_to_lds(__amdgpu_buffer_rsrc_t from, unsigned char* to, int offset)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, offset, 0, 0, 0);
}
__device__ __forceinline__ void kv8_to_lds_once(__amdgpu_buffer_rsrc_t from, unsigned char* to, int offset)  // read once per call: non-temporal
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, offset, 0, 0, 2);
}

// ---------------------------------------------------------------------------------------
// One new token a sequence.  Workgroup = one wavefront = (chunk of cached tokens of a sequence, cache head [, sixteen of its query heads]); the chunks are
// cut on the device from the lengths, so that a captured call stays balanced when they change.  16x16x32 products: a lane holds the row (query
// head) lane % 16.  Bound by the reads of codes: 103 MB (16 sequences of up to 6000 tokens, 8 heads of 128) in 23.8 us, 4.3 TB/s, and 4.6 us for the merge; 33 MB (one
// sequence, 32 heads) in 10.9 us, of which half are the start and the chain length -> page -> codes.  Why a wavefront a workgroup: with four and a common
// chunk, a barrier in each tile made all wait for the slowest load (31.5 us instead of 28, merge included).
// ---------------------------------------------------------------------------------------

// which 16-byte piece of a token's value codes stands at place p of its row in LDS: p ^ this; the rows that a transposing read takes together
// (tokens 4g .. 4g + 3 and sixteen further, for two g at a time) fall into different banks
template <int D>
__device__ __forceinline__ int kv8_decode_swizzle(int token)
{
    if constexpr (D == 128) return ((token >> 1) & 1) | ((token >> 3) & 2) | (token & 4);
    else return ((token >> 4) & 1) | ((token >> 1) & 2);
}

// Where a workgroup's chunk lies, from the lengths: sequence b (-1: none), its length, its chunk of `tokens` tokens
struct Kv8Chunk {
    int b, length, chunk, tokens;
};

__device__ __forceinline__ Kv8Chunk kv8_chunk(const Kv8Table& t, int chunks, int target, int lane)
{
    if (t.sequences == 1) {  // uniform
        const int n = kv8_clamp(t.lengths[0], 0, t.capacity), C = kv8_chunk_tokens(n, 1, chunks);
        return {target < kv8_chunks(n, C) ? 0 : -1, n, target, C};
    }
    auto length_of = [&](int b) { return kv8_clamp(t.lengths[b], 0, t.capacity); };
    const int C = kv8_chunk_tokens(kv8_total(t.sequences, lane, length_of), t.sequences, chunks);
    const Kv8Unit u = kv8_find(t.sequences, target, lane, [&](int b) { return kv8_chunks(length_of(b), C); });
    if (u.b < 0) return {-1, 0, 0, C};
    const int b = __builtin_amdgcn_readfirstlane(u.b);
    return {b, __builtin_amdgcn_readfirstlane(length_of(b)), __builtin_amdgcn_readfirstlane(u.within), C};
}

template <int D, int QP>
__global__ __launch_bounds__(64) void kv8_decode_kernel(Kv8AttnArgs a)
{
    constexpr int KX = D / 64;  // 16-byte loads of a lane for sixteen tokens' keys
    __shared__ __attribute__((aligned(16))) unsigned char values[KV8_TILE * D];  // a tile's value codes
    const int lane = threadIdx.x, i = lane & 15, g = lane >> 4;
    const int chunk = static_cast<int>(blockIdx.x) / a.H_kv, hk = static_cast<int>(blockIdx.x) - chunk * a.H_kv;
    const Kv8Chunk at = kv8_chunk(a.t, a.chunks, chunk, lane);
    if (at.b < 0) return;
    const int b = at.b, len = at.length, t0 = at.chunk * at.tokens, t_end = min(len, t0 + at.tokens);
    const int R = min(16, a.rep - static_cast<int>(blockIdx.y) * 16);
    const int h0 = hk * a.rep + static_cast<int>(blockIdx.y) * 16;
    const int tiles = t_end > t0 ? (t_end - t0 + KV8_TILE - 1) / KV8_TILE : 0;
    const int of = kv8_chunks(len, at.tokens);
    if (at.chunk == 0 && hk == 0 && blockIdx.y == 0 && lane == 0) a.cut[b] = make_int2(chunk, of);  // for the merge

    // pages and scales of sixteen tiles: lane = sixteen tokens
    int page;
    float k_scale, v_inverse, v_log;
    auto look_up = [&](int base) {
        const int pos = base + 16 * lane;
        page = pos < t_end ? kv8_page(a.t, a.t.table + static_cast<size_t>(b) * a.t.width, pos) : -1;
        const size_t s = static_cast<size_t>(max(page, 0)) * a.H_kv + hk;
        k_scale = __builtin_amdgcn_fmed3f(a.k_scales[s], KV8_LEAST, KV8_MOST);
        const float v_scale = __builtin_amdgcn_fmed3f(a.v_scales[s], KV8_LEAST, KV8_MOST);
        v_inverse = 1.0f / v_scale;
        v_log = __builtin_amdgcn_logf(v_scale);
    };
    auto resource = [&](const unsigned char* codes, const Kv8Block& x) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(codes) + x.at * D, 0, x.tokens * D, 0x00020000);
    };
    auto block_of = [&](int base, int in, int n) {  // tile `in` of those looked up
        return kv8_block(a.t, a.H_kv, hk, __builtin_amdgcn_readlane(page, 4 * in + n), base + 16 * n, t_end);
    };
    u32x4 kw[4][KX];
    auto load_keys = [&](int base, int in) {
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const __amdgpu_buffer_rsrc_t kr = resource(a.k_codes, block_of(base, in, n));
#pragma unroll
            for (int x = 0; x < KX; ++x) kw[n][x] = __builtin_amdgcn_raw_buffer_load_b128(kr, i * D + 16 * g + 64 * x, 0, 2);
        }
    };
    auto load_values = [&](int base, int in) {
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const __amdgpu_buffer_rsrc_t vr = resource(a.v_codes, block_of(base, in, n));
#pragma unroll
            for (int y = 0; y < KX; ++y) {
                constexpr int P = D / 16;  // pieces a token
                const int s16 = 64 * y + lane, token = s16 / P, place = s16 % P;
                kv8_to_lds_once(vr, &values[16 * n * D + 1024 * y], token * D + ((place ^ kv8_decode_swizzle<D>(16 * n + token)) * 16));
            }
        }
    };

    // ---- the query: lane = (head i, the elements of the key pieces 16 g .. of each 64) ----
    v8h qh[2 * KX], ql[QP == 2 ? 2 * KX : 1];
    float unit = 0.0f;
    if (tiles > 0) {
        float t[2 * KX][8];
        const size_t from = (static_cast<size_t>(b) * a.H_q + h0 + min(i, R - 1)) * D + 16 * g;
        float top = 0.0f;
#pragma unroll
        for (int d = 0; d < 2 * KX; ++d) kv8_query8(a, from + 64 * (d >> 1) + 8 * (d & 1), t[d]);
        look_up(t0);
        load_keys(t0, 0);
        load_values(t0, 0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int d = 0; d < 2 * KX; ++d)
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(t[d][e]));
        top = kv8_swap32_max(kv8_swap16_max(top));
        const int E = __builtin_amdgcn_frexp_expf(top);
#pragma unroll
        for (int d = 0; d < 2 * KX; ++d) {
#pragma unroll
            for (int e = 0; e < 8; ++e) t[d][e] = ldexpf(t[d][e], 14 - E);
            if constexpr (QP == 2) kv8_split(t[d], qh[d], ql[d]);
            else qh[d] = kv8_round(t[d]);
        }
        unit = ldexpf(a.softmax_scale * KV8_LOG2E, E - 14);
    }

    v4f acc[D / 16];
#pragma unroll
    for (int d = 0; d < D / 16; ++d) acc[d] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    float m = KV8_LOW, l = 0.0f;
    for (int c = 0; c < tiles; ++c) {
        const int base = t0 + KV8_TILE * c, in = c & 15;
        v4f S[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            S[n] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int d = 0; d < 2 * KX; ++d) {
                const v8h k = kv8_halves(kw[n][d >> 1][2 * (d & 1)], kw[n][d >> 1][2 * (d & 1) + 1]);
                if constexpr (QP == 2) S[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, ql[d], S[n], 0, 0, 0);
                S[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, qh[d], S[n], 0, 0, 0);
            }
        }
        float ks[4], vs[4], ls[4];
        bool there[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            ks[n] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(k_scale), 4 * in + n)) * unit;
            vs[n] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v_inverse), 4 * in + n));
            ls[n] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v_log), 4 * in + n));
            there[n] = __builtin_amdgcn_readlane(page, 4 * in + n) >= 0;
        }
        const bool more = c + 1 < tiles;  // uniform
        if (more) {
            if (in == 15) look_up(base + KV8_TILE);
            __builtin_amdgcn_sched_barrier(0);
            load_keys(base + KV8_TILE, (c + 1) & 15);
        }
        __builtin_amdgcn_sched_barrier(0);
        float top = -INFINITY;
        const bool whole = base + KV8_TILE <= t_end && there[0] && there[1] && there[2] && there[3];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            if (!whole) {  // uniform
                ks[n] = fmaxf(ks[n], KV8_NOT_ZERO);
#pragma unroll
                for (int j = 0; j < 4; ++j) S[n][j] = there[n] && base + 16 * n + 4 * g + j < t_end ? S[n][j] : -INFINITY;
            }
            top = fmaxf(top, fmaf(fmaxf(fmaxf(fmaxf(S[n][0], S[n][1]), S[n][2]), S[n][3]), ks[n], ls[n]));
        }
        if (__builtin_amdgcn_ballot_w64(top > m + KV8_TOP) != 0) {
            const float t = kv8_swap32_max(kv8_swap16_max(top));
            const float m_new = t > m + KV8_TOP ? t - KV8_REF : m;
            const float alpha = __builtin_amdgcn_exp2f(m - m_new);
            m = m_new;
            l *= alpha;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) acc[d] *= alpha;
        }
        v8h ph[2], pl[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            float w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int n = 2 * s + (e >> 2);
                w[e] = __builtin_amdgcn_exp2f(fmaf(S[n][e & 3], ks[n], ls[n] - m));
            }
            l = fmaf((w[0] + w[1]) + (w[2] + w[3]), vs[2 * s], l);
            l = fmaf((w[4] + w[5]) + (w[6] + w[7]), vs[2 * s + 1], l);
            kv8_split(w, ph[s], pl[s]);
        }
        // the values of this tile are in LDS once no more loads than the keys requested above are outstanding
        __builtin_amdgcn_sched_barrier(0);
        if (more) __builtin_amdgcn_s_waitcnt((4 * KX) | (7 << 4) | (15 << 8));
        else __builtin_amdgcn_s_waitcnt(0 | (7 << 4) | (15 << 8));
        __builtin_amdgcn_sched_barrier(0);
        const int r = i >> 1;
        const int token = 16 * (r >> 2) + 4 * g + (r & 3);
        const unsigned char* const vat = &values[token * D + (i & 1) * 8];
        const int f = kv8_decode_swizzle<D>(token);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
                const v2i x = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                    (__attribute__((address_space(3))) v2i*)(vat + 32 * s * D + ((d ^ f) * 16)));
                const v8h v = kv8_halves(static_cast<uint32_t>(x[0]), static_cast<uint32_t>(x[1]));
                acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pl[s], acc[d], 0, 0, 0);
                acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, ph[s], acc[d], 0, 0, 0);
            }
        // every read of the tile has returned before the next one overwrites it
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
        if (more) load_values(base + KV8_TILE, (c + 1) & 15);
        __builtin_amdgcn_sched_barrier(0);
    }
    l = fold32f(fold16f(l, l), fold16f(l, l));
    if (i >= R) return;
    const int h = h0 + i;
    if (of == 1) {
        const float by = l == 0.0f ? 0.0f : 1.0f / l;
        const size_t to = (static_cast<size_t>(b) * a.H_q + h) * D + 4 * g;
#pragma unroll
        for (int d = 0; d < D / 16; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j) kv8_put(a.out, a.out_dt, to + 16 * d + j, l == 0.0f ? 0.0f : acc[d][j] * by);
    } else {
        float* const dst = a.part + (static_cast<size_t>(chunk) * a.H_q + h) * (D + KV8_EXTRA);
#pragma unroll
        for (int d = 0; d < D / 16; ++d) *reinterpret_cast<v4f*>(dst + 16 * d + 4 * g) = acc[d];
        if (g == 0) *reinterpret_cast<float2*>(dst + D) = make_float2(m, l);
    }
}

// Merges n partial results `stride` floats apart into one row: thread (g, j) of GROUPS x D takes element j of every GROUPS-th of them, eight at a
// time so that their loads are under way together.
template <int D, int GROUPS>
__device__ __forceinline__ void kv8_merge(const float* src, size_t stride, int n, void* out, int out_dt, size_t row)
{
    constexpr int U = 8;
    __shared__ float red[GROUPS][D], dred[GROUPS], mred[GROUPS];
    const int j = threadIdx.x % D, g = threadIdx.x / D;
    float M = KV8_LOW, num = 0.0f, den = 0.0f;
    for (int i0 = g; i0 < n; i0 += U * GROUPS) {
        float2 ml[U];
        float v[U];
#pragma unroll
        for (int x = 0; x < U; ++x) {
            const float* const s = src + static_cast<size_t>(min(i0 + GROUPS * x, n - 1)) * stride;
            ml[x] = *reinterpret_cast<const float2*>(s + D);
            v[x] = s[j];
        }
        float mb = M;
#pragma unroll
        for (int x = 0; x < U; ++x)
            if (i0 + GROUPS * x < n) mb = fmaxf(mb, ml[x].x);
        const float r = __builtin_amdgcn_exp2f(M - mb);
        num *= r;
        den *= r;
        M = mb;
#pragma unroll
        for (int x = 0; x < U; ++x) {
            const float e = i0 + GROUPS * x < n ? __builtin_amdgcn_exp2f(ml[x].x - M) : 0.0f;
            num = fmaf(e, v[x], num);
            den = fmaf(e, ml[x].y, den);
        }
    }
    red[g][j] = num;
    if (j == 0) {
        dred[g] = den;
        mred[g] = M;
    }
    __syncthreads();
    if (g == 0) {
        float Mt = mred[0];
#pragma unroll
        for (int x = 1; x < GROUPS; ++x) Mt = fmaxf(Mt, mred[x]);
        num = den = 0.0f;
#pragma unroll
        for (int x = 0; x < GROUPS; ++x) {
            const float e = __builtin_amdgcn_exp2f(mred[x] - Mt);
            num = fmaf(e, red[x][j], num);
            den = fmaf(e, dred[x], den);
        }
        kv8_put(out, out_dt, row * D + j, den == 0.0f ? 0.0f : num / den);
    }
}

// blockIdx = (query head, sequence): the chunks of a sequence that has more than one
template <int D, int GROUPS>
__global__ __launch_bounds__(GROUPS * D) void kv8_decode_merge_kernel(Kv8AttnArgs a)
{
    const int h = blockIdx.x, b = blockIdx.y;
    const int2 cut = a.cut[b];
    if (cut.y == 1) return;  // the attention kernel has written it
    kv8_merge<D, GROUPS>(a.part + (static_cast<size_t>(cut.x) * a.H_q + h) * (D + KV8_EXTRA), static_cast<size_t>(a.H_q) * (D + KV8_EXTRA), cut.y, a.out,
                         a.out_dt, static_cast<size_t>(b) * a.H_q + h);
}

// ---------------------------------------------------------------------------------------
// Several new tokens a sequence, each of which sees the tokens up to its own.  Workgroup = (128 rows of a sequence and cache head, [part of
// the cached tokens]); row = (new token, query head of the group).  32x32x16 products: a lane holds the row lane % 32 of its
// wavefront's 32 and, of each 32 tokens, those with (token / 4) % 2 = lane / 32.  The four wavefronts share the tiles of 64 tokens in LDS, four of them, of which
// three are under way (the compiler waits for them before the transposing reads; loads behind those reads measure the same).  Bound by the vector unit (a conversion to binary16, a multiply-add, an exponential, a rounding, the maximum and the sum of each
// score and value) together with the matrix cores: busy 76 and 46 % of the cycles.  8192 tokens of 32 + 2 x 8 heads of 128, bfloat16: 550 GFLOP in 568 .. 639 us, 0.86 ..
// 0.97 PFLOP/s; binary32 queries and results 911 us, binary16 ones 759.  Four prompts of 301 to 2000 tokens, bfloat16: 56 GFLOP in 89 .. 100 us.
// ---------------------------------------------------------------------------------------
constexpr int KV8_ROWS = 128;
constexpr int KV8_STAGES = 4;  // tiles in LDS: one in use, the others under way

template <int D>
__device__ __forceinline__ int kv8_prompt_swizzle(int token)
{
    if constexpr (D == 128) return ((token >> 2) & 1) | (token & 2) | ((token >> 1) & 4);
    else return ((token >> 2) & 1) | ((token >> 2) & 2);
}

template <int D, int QP, int PP>
__global__ __launch_bounds__(256) void kv8_prompt_kernel(Kv8AttnArgs a)
{
    constexpr int KL = D / 32, DB = D / 32, P = D / 16, LOADS = D / 64;
    __shared__ __attribute__((aligned(16))) unsigned char tiles[2][KV8_STAGES][KV8_TILE * D];
    unsigned char(*const kt)[KV8_TILE * D] = tiles[0];
    unsigned char(*const vt)[KV8_TILE * D] = tiles[1];
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int rest = blockIdx.x;
    const int hk = rest % a.H_kv;
    rest /= a.H_kv;
    // Sequence after sequence, the last rows first: they see most.  (All sequences' tiles by what they see, heaviest first, is slower: four prompts of 301
    // to 2000 tokens 101 us instead of 97.)
    const int split = rest % a.chunks;
    const Kv8Unit u = kv8_find(a.t.sequences, a.tiles - 1 - rest / a.chunks, lane, [&](int b) {
        return static_cast<int>((static_cast<long long>(kv8_run(a.t.starts, a.t.lengths, b, a.rows).count) * a.rep + KV8_ROWS - 1) / KV8_ROWS);
    });
    if (u.b < 0) return;
    const int b = __builtin_amdgcn_readfirstlane(u.b), row0 = __builtin_amdgcn_readfirstlane(u.within) * KV8_ROWS;
    const Kv8Run run = kv8_run(a.t.starts, a.t.lengths, b, a.rows);
    const int pos0 = __builtin_amdgcn_readfirstlane(run.pos), first = __builtin_amdgcn_readfirstlane(run.first);
    const int n_rows = __builtin_amdgcn_readfirstlane(run.count) * a.rep;
    const int len = min(__builtin_amdgcn_readfirstlane(run.length), a.t.capacity);
    auto sees = [&](int r) { return kv8_clamp(pos0 + min(r, n_rows - 1) / a.rep + 1, 0, len); };  // tokens that row r may see
    const int wg_sees = __builtin_amdgcn_readfirstlane(sees(row0 + KV8_ROWS - 1));
    const int all_tiles = (wg_sees + KV8_TILE - 1) / KV8_TILE, per = (all_tiles + a.chunks - 1) / a.chunks;
    const int tile0 = split * per, tile1 = min(all_tiles, tile0 + per);
    const int my = row0 + 32 * wave + c, limit = sees(my);
    const int wave_least = __builtin_amdgcn_readfirstlane(sees(row0 + 32 * wave)), wave_most = __builtin_amdgcn_readfirstlane(sees(row0 + 32 * wave + 31));
    const int* const table = a.t.table + static_cast<size_t>(b) * a.t.width;
    const int token = first + min(my, n_rows - 1) / a.rep, head = hk * a.rep + min(my, n_rows - 1) % a.rep;
    const size_t out_row = static_cast<size_t>(token) * a.H_q + head;

    v8h qh[KL][2], ql[QP == 2 ? KL : 1][2];
    float unit;
    {
        float t[KL][2][8], top = 0.0f;
#pragma unroll
        for (int k = 0; k < KL; ++k)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                kv8_query8(a, out_row * D + 32 * k + 16 * hh + 8 * x, t[k][x]);
#pragma unroll
                for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(t[k][x][e]));
            }
        top = kv8_swap32_max(top);
        const int E = __builtin_amdgcn_frexp_expf(top);
#pragma unroll
        for (int k = 0; k < KL; ++k)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
#pragma unroll
                for (int e = 0; e < 8; ++e) t[k][x][e] = ldexpf(t[k][x][e], 14 - E);
                if constexpr (QP == 2) kv8_split(t[k][x], qh[k][x], ql[k][x]);
                else qh[k][x] = kv8_round(t[k][x]);
            }
        unit = ldexpf(a.softmax_scale * KV8_LOG2E, E - 14);
    }

    auto resource = [&](const unsigned char* codes, const Kv8Block& x) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(codes) + x.at * D, 0, x.tokens * D, 0x00020000);
    };
    // pages and scales of sixteen tiles: lane = sixteen tokens
    int page = -1, ahead = -1;
    float k_scale, v_inverse, v_log;
    auto look_up = [&](int tile) {
        const int pos = tile * KV8_TILE + 16 * lane;
        return pos < wg_sees && tile + (lane >> 2) < tile1 ? kv8_page(a.t, table, pos) : -1;
    };
    auto stage = [&](int tile) {  // sixteen tokens of the tile by each wavefront; beyond the last tile: nothing, but as many loads
        const int in = tile - tile0, buf = in % KV8_STAGES, pos = tile * KV8_TILE + 16 * wave;
        const int id = __builtin_amdgcn_readlane(ahead, 4 * (in & 15) + wave);
        const Kv8Block block = kv8_block(a.t, a.H_kv, hk, id, pos, wg_sees);
        const __amdgpu_buffer_rsrc_t kr = resource(a.k_codes, block), vr = resource(a.v_codes, block);
#pragma unroll
        for (int y = 0; y < LOADS; ++y) {
            const int s16 = 64 * y + lane, tk = s16 / P, at = s16 % P;
            const int from = tk * D + ((at ^ kv8_prompt_swizzle<D>(16 * wave + tk)) * 16);
            kv8_to_lds(kr, &kt[buf][16 * wave * D + 1024 * y], from);
            kv8_to_lds(vr, &vt[buf][16 * wave * D + 1024 * y], from);
        }
    };

    v16f acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[d][e] = 0.0f;
    float m = KV8_LOW, l = 0.0f;
    if (tile0 < tile1) {
        ahead = look_up(tile0);
#pragma unroll
        for (int x = 0; x < KV8_STAGES - 1; ++x) stage(tile0 + x);
    }
    for (int tile = tile0; tile < tile1; ++tile) {
        const int in = tile - tile0, buf = in % KV8_STAGES, base = tile * KV8_TILE;
        if ((in & 15) == 0) {  // uniform
            page = look_up(tile);
            const size_t s = static_cast<size_t>(max(page, 0)) * a.H_kv + hk;
            const float v_scale = __builtin_amdgcn_fmed3f(a.v_scales[s], KV8_LEAST, KV8_MOST);
            k_scale = __builtin_amdgcn_fmed3f(a.k_scales[s], KV8_LEAST, KV8_MOST);
            v_inverse = 1.0f / v_scale;
            v_log = __builtin_amdgcn_logf(v_scale);
        }
        if (((in + KV8_STAGES - 1) & 15) == 0) ahead = look_up(tile + KV8_STAGES - 1);
        // this wavefront's part of the tile is in LDS once only the later tiles' loads are outstanding,
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt((2 * LOADS * (KV8_STAGES - 2)) | (7 << 4) | (15 << 8));
        __syncthreads();  // then everybody's is, and the tile before has been read
        __builtin_amdgcn_sched_barrier(0);
        stage(tile + KV8_STAGES - 1);
        __builtin_amdgcn_sched_barrier(0);
        if (base >= wave_most) continue;  // uniform over the wavefront: none of its rows sees the tile
        v16f S[2];
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
#pragma unroll
            for (int e = 0; e < 16; ++e) S[tb][e] = 0.0f;
            const unsigned char* const at = &kt[buf][(32 * tb + c) * D];
            const int f = kv8_prompt_swizzle<D>(c);
#pragma unroll
            for (int k = 0; k < KL; ++k) {
                const u32x4 x = *reinterpret_cast<const u32x4*>(at + (((2 * k + hh) ^ f) * 16));
                const v8h k0 = kv8_halves(x[0], x[1]), k1 = kv8_halves(x[2], x[3]);
                if constexpr (QP == 2) {
                    S[tb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k0, ql[k][0], S[tb], 0, 0, 0);
                    S[tb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k1, ql[k][1], S[tb], 0, 0, 0);
                }
                S[tb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k0, qh[k][0], S[tb], 0, 0, 0);
                S[tb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k1, qh[k][1], S[tb], 0, 0, 0);
            }
        }
        float ks[4], vi[4], vl[4];
        bool there[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const int at = 4 * (in & 15) + n;
            there[n] = __builtin_amdgcn_readlane(page, at) >= 0;
            ks[n] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(k_scale), at));
            vi[n] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v_inverse), at));
            vl[n] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v_log), at));
        }
        const bool whole = base + KV8_TILE <= wave_least && there[0] && there[1] && there[2] && there[3];
        // sixteen tokens of a page are eight scores of a lane: score = S by[n], weight = 2^(score + log2 s' - m) in one multiply-add and one exponential
        float by[4], top = -INFINITY;
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            by[n] = ks[n] * unit;
            if (!whole) {
                by[n] = fmaxf(by[n], KV8_NOT_ZERO);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool seen = there[n] && base + 16 * n + 8 * (e >> 2) + 4 * hh + (e & 3) < limit;
                    S[n >> 1][8 * (n & 1) + e] = seen ? S[n >> 1][8 * (n & 1) + e] : -INFINITY;
                }
            }
            const v16f& x = S[n >> 1];
            const int o = 8 * (n & 1);
            const float most = fmaxf(fmaxf(fmaxf(x[o], x[o + 1]), x[o + 2]), fmaxf(fmaxf(x[o + 3], x[o + 4]), fmaxf(fmaxf(x[o + 5], x[o + 6]), x[o + 7])));
            top = fmaxf(top, fmaf(most, by[n], vl[n]));
        }
        if (__builtin_amdgcn_ballot_w64(top > m + KV8_TOP) != 0) {
            const float t = kv8_swap32_max(top);
            const float m_new = t > m + KV8_TOP ? t - KV8_REF : m;
            const float alpha = __builtin_amdgcn_exp2f(m - m_new);
            m = m_new;
            l *= alpha;
#pragma unroll
            for (int d = 0; d < DB; ++d) acc[d] *= alpha;
        }
        const int r = (lane & 15) >> 1;
        const int vtok = 8 * (r >> 2) + 4 * hh + (r & 3), f = kv8_prompt_swizzle<D>(vtok), dhalf = (lane >> 4) & 1;
        const unsigned char* const vat = &vt[buf][vtok * D + (lane & 1) * 8];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            float w[8];
            const float less = vl[n] - m;
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = __builtin_amdgcn_exp2f(fmaf(S[n >> 1][8 * (n & 1) + e], by[n], less));
            l = fmaf(((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7])), vi[n], l);
            v8h ph, pl;
            if constexpr (PP == 2) kv8_split(w, ph, pl);
            else ph = kv8_round(w);
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const v2i x = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                    (__attribute__((address_space(3))) v2i*)(vat + 16 * n * D + (((2 * d + dhalf) ^ f) * 16)));
                const v8h v = kv8_halves(static_cast<uint32_t>(x[0]), static_cast<uint32_t>(x[1]));
                if constexpr (PP == 2) acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, pl, acc[d], 0, 0, 0);
                acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, ph, acc[d], 0, 0, 0);
            }
        }
    }
    __builtin_amdgcn_s_waitcnt(0);  // nothing is on its way into LDS any more
    l = fold32f(l, l);
    if (a.chunks == 1) {
        // Through LDS, so that rows are written in whole: in the lanes' order, two bytes of each of 32 rows at a time,
        // those prompts took 120 us instead of 97.
        // Sixteen-byte piece p of a row stands at place p ^ its number.
        const float by = l == 0.0f ? 0.0f : 1.0f / l;
        const bool wide = a.out_dt == RCP_F32;  // uniform
        const int row_bytes = wide ? 4 * D : 2 * D, pieces = row_bytes / 16;
        unsigned char* const mine = &tiles[0][0][0] + wave * (32 * 4 * D);
        __syncthreads();  // every wavefront has read its last tile
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                float v[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) v[x] = l == 0.0f ? 0.0f : acc[d][e + x] * by;
                if (wide) *reinterpret_cast<float4*>(mine + c * row_bytes + (((8 * d + e / 2 + hh) ^ c) & (pieces - 1)) * 16) = make_float4(v[0], v[1], v[2], v[3]);
                else *reinterpret_cast<uint2*>(mine + c * row_bytes + (((4 * d + e / 4) ^ c) & (pieces - 1)) * 16 + 8 * hh) = kv8_pack4(a.out_dt, v);
            }
        const int at_once = 64 / pieces;  // rows
        for (int r0 = 0; r0 < 32; r0 += at_once) {
            const int r = r0 + lane / pieces, p = lane % pieces, row = row0 + 32 * wave + r;
            if (row < n_rows) {
                const size_t to = (static_cast<size_t>(first + row / a.rep) * a.H_q + hk * a.rep + row % a.rep) * row_bytes + 16 * p;
                *reinterpret_cast<u32x4*>(static_cast<unsigned char*>(a.out) + to) = *reinterpret_cast<const u32x4*>(mine + r * row_bytes + ((p ^ r) & (pieces - 1)) * 16);
            }
        }
    } else if (my < n_rows) {
        float* const dst = a.part + (static_cast<size_t>(split) * a.rows * a.H_q + out_row) * (D + KV8_EXTRA);
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<float4*>(dst + 32 * d + 8 * (e >> 2) + 4 * hh) = make_float4(acc[d][e], acc[d][e + 1], acc[d][e + 2], acc[d][e + 3]);
        if (hh == 0) {
            dst[D] = m;
            dst[D + 1] = l;
        }
    }
}

// blockIdx = the query heads of a row of the call, row after row
template <int D, int GROUPS>
__global__ __launch_bounds__(GROUPS * D) void kv8_prompt_merge_kernel(Kv8AttnArgs a)
{
    const int t = static_cast<int>(blockIdx.x) / a.H_q, h = static_cast<int>(blockIdx.x) - t * a.H_q;
    if (kv8_sequence_of(a.t.starts, a.t.sequences, t, a.rows) < 0) return;
    const size_t row = static_cast<size_t>(t) * a.H_q + h, stride = static_cast<size_t>(a.rows) * a.H_q * (D + KV8_EXTRA);
    kv8_merge<D, GROUPS>(a.part + row * (D + KV8_EXTRA), stride, a.chunks, a.out, a.out_dt, row);
}

// ---------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------
struct Kv8AttnPlan {
    int chunks, tiles;  // as in Kv8AttnArgs
    size_t bytes;       // of partial results
};

static Kv8AttnPlan kv8_attn_plan(int rows, int sequences, int H_q, int H_kv, int D, bool one)
{
    Kv8AttnPlan p;
    const int cus = num_compute_units(), rep = H_q / H_kv;
    const size_t partial = static_cast<size_t>(H_q) * (D + KV8_EXTRA) * sizeof(float);
    if (one) {
        // Eight wavefronts a compute unit, two a SIMD (heads of 128): 13.0 us for one sequence of 4001 tokens of 32 heads, 27.6 for 16 of up to 6000 tokens of 32 over 8 heads.
        // With four 14.2 and 29.9, with sixteen 13.3 and 30.9; one sequence of 30000 tokens of 8 heads 22.7, with four 20.5, with sixteen 31.3.
        p.chunks = 8 * cus / H_kv > 2 * sequences ? 8 * cus / H_kv : 2 * sequences;
        p.tiles = 0;
        p.bytes = static_cast<size_t>(p.chunks) * partial + sequences * sizeof(int2);
    } else {
        p.tiles = static_cast<int>(static_cast<long long>(rows) * rep / KV8_ROWS) + sequences;
        const long long groups = static_cast<long long>(p.tiles) * H_kv;
        p.chunks = 1;
        const int slots = (D == 64 ? 3 : 2) * cus;  // workgroups that run at once
        if (groups < slots) {
            const long long want = (slots + groups - 1) / groups;
            p.chunks = static_cast<int>(want < 32 ? want : 32);
        }
        p.bytes = p.chunks == 1 ? 0 : static_cast<size_t>(p.chunks) * rows * partial;
    }
    return p;
}

size_t kv8_workspace_bytes(int rows, int sequences, int H_q, int H_kv, int D, bool one)
{
    const size_t bytes = kv8_attn_plan(rows, sequences, H_q, H_kv, D, one).bytes;
    return bytes > 16 ? bytes : 16;
}

int launch_kv8_attn(const Kv8AttnCall& c, hipStream_t st)
{
    const bool one = c.starts == nullptr;
    const Kv8AttnPlan plan = kv8_attn_plan(c.rows, c.sequences, c.H_q, c.H_kv, c.D, one);
    Kv8AttnArgs a;
    a.t = {c.starts, c.lengths, c.table, c.sequences, c.width, c.shift, c.n_pages, c.width << c.shift};
    a.q = c.q;
    a.q_dt = c.q_dtype;
    a.out_dt = c.out_dtype;
    a.rows = c.rows;
    a.H_q = c.H_q;
    a.H_kv = c.H_kv;
    a.rep = c.H_q / c.H_kv;
    a.softmax_scale = c.softmax_scale;
    a.k_codes = static_cast<const unsigned char*>(c.k_codes);
    a.v_codes = static_cast<const unsigned char*>(c.v_codes);
    a.k_scales = c.k_scales;
    a.v_scales = c.v_scales;
    a.out = c.out;
    a.part = static_cast<float*>(c.workspace);
    a.cut = reinterpret_cast<int2*>(a.part + static_cast<size_t>(plan.chunks) * c.H_q * (c.D + KV8_EXTRA));
    a.chunks = plan.chunks;
    a.tiles = plan.tiles;
    const bool q2 = c.q_dtype == RCP_F32;
    auto form = [&](auto size) {
        constexpr int D = decltype(size)::value;
        if (one) {
            const dim3 grid(static_cast<unsigned>(plan.chunks) * static_cast<unsigned>(c.H_kv), static_cast<unsigned>((a.rep + 15) / 16));
            auto launch = [&](auto kernel) { enqueue(kernel, grid, 64, 0, st, a); };
            if (q2) launch(&kv8_decode_kernel<D, 2>);
            else launch(&kv8_decode_kernel<D, 1>);
        } else {
            const unsigned grid = static_cast<unsigned>(plan.tiles) * static_cast<unsigned>(plan.chunks) * static_cast<unsigned>(c.H_kv);
            auto launch = [&](auto kernel) { enqueue(kernel, grid, 256, 0, st, a); };
            const bool p2 = c.out_dtype != RCP_BF16;
            if (q2 && p2) launch(&kv8_prompt_kernel<D, 2, 2>);
            else if (q2) launch(&kv8_prompt_kernel<D, 2, 1>);
            else if (p2) launch(&kv8_prompt_kernel<D, 1, 2>);
            else launch(&kv8_prompt_kernel<D, 1, 1>);
        }
    };
    if (c.D == 128) form(std::integral_constant<int, 128>{});
    else form(std::integral_constant<int, 64>{});
    if (int rc = check_launch("rcp_kv8_attn")) return rc;
    if (!one && plan.chunks == 1) return RCP_OK;
    // (a second dimension ends at 65535; rows are split only where there are few of them, times query heads)
    const dim3 grid = one ? dim3(static_cast<unsigned>(c.H_q), static_cast<unsigned>(c.sequences)) : dim3(static_cast<unsigned>(c.H_q) * static_cast<unsigned>(c.rows));
    // Wavefronts for the partial results of a row, by their mean number: eight to a thread at a time.  With as few for long rows as for short ones the whole
    // call takes 33.9 us instead of 22.7 (one sequence of 30000 tokens of 8 heads), with as many for short ones 21.1 instead of 19.6 (16 sequences of 2000 tokens).
    auto merge = [&](auto size) {
        constexpr int D = decltype(size)::value;
        const int each = one ? plan.chunks / c.sequences : plan.chunks;
        auto launch = [&](auto groups) {
            constexpr int G = decltype(groups)::value;
            if (one) enqueue(&kv8_decode_merge_kernel<D, G>, grid, G * D, 0, st, a);
            else enqueue(&kv8_prompt_merge_kernel<D, G>, grid, G * D, 0, st, a);
        };
        if (each <= 16) launch(std::integral_constant<int, 128 / D>{});
        else if (each <= 32) launch(std::integral_constant<int, 256 / D>{});
        else launch(std::integral_constant<int, 1024 / D>{});
    };
    if (c.D == 128) merge(std::integral_constant<int, 128>{});
    else merge(std::integral_constant<int, 64>{});
    return check_launch("rcp_kv8_attn(merge)");
}

}  // namespace rcp
