// New keys and values enter a paged cache in 8 bits, with the position rotation and, where it is wanted, the Hadamard rotation of
// keys (and queries) on the way.
//
// A page of one head holds E4M3 codes c (OCP: 4 exponent and 3 mantissa bits, largest 448) and one scale s = 2^E; a code stands for c s.
// E is the smallest exponent with which no finite element of the page's tokens exceeds 448 s, in [-40, 120].  Powers of two: E4M3 is a
// floating-point format, so a finer scale would not make its codes more accurate, and when a later token needs a larger scale the
// older codes are divided by a power of two, which is exact down to the format's subnormals.  (8 bits with one step for all would
// hold Gaussian data more exactly, but every growth of its step would round all older codes again.)
//
// The position rotation turns element j with element j + D/2 by the angle of the position, from a table of cosines and sines:
//   y_j = x_j c - x_{j+D/2} s,   y_{j+D/2} = x_{j+D/2} c + x_j s,   products and sums rounded on their own in binary32.
// The Hadamard rotation is that of the 4-bit cache: butterflies in ascending stride order, one multiplication by (float)(1/sqrt(D)).
#include "kv8.hpp"

namespace rcp {

constexpr int KV8_QUERIES = 4;  // query vectors of a lane in a prompt
// A dimension of a grid ends below 2^32 threads, which are 2^24 workgroups of 256: a longer one is folded into rows of 2^23.
constexpr int KV8_GRID_SHIFT = 23;

struct Kv8AppendArgs {
    Kv8Table t;
    const void *k, *v, *q;
    void* q_out;
    long long k_stride, v_stride, q_stride;  // elements from one token to the next
    const float* rope;                       // [capacity][D]: D/2 cosines, D/2 sines; null: no position rotation
    uint2 *k_codes, *v_codes;
    float *k_scales, *v_scales;
    int rows, H, H_q, rotate;
    int kv_groups;                           // workgroups that write pages; those behind them rotate queries
    int groups;                              // of both
};

template <int CTRL>
__device__ __forceinline__ float kv8_dpp(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <int CTRL>
__device__ __forceinline__ uint32_t kv8_dpp(uint32_t v)
{
    return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, 0xf, 0xf, true));
}
// the value of lane ^ 1, 2, 4, 8 within a row of sixteen lanes
template <int M, class T>
__device__ __forceinline__ T kv8_partner(T v)
{
    if constexpr (M == 1) return kv8_dpp<0xB1>(v);
    else if constexpr (M == 2) return kv8_dpp<0x4E>(v);
    else if constexpr (M == 4) return kv8_dpp<0x1B>(kv8_dpp<0x141>(v));
    else return kv8_dpp<0x128>(v);
}

// D / 8 neighbouring lanes own a vector, eight consecutive elements each.
template <int D>
__device__ __forceinline__ void kv8_turn(float (&v)[8], int l, const float* angles, bool rotate)
{
#pragma clang fp contract(off)
    constexpr int LANES = D / 8;
    if (angles != nullptr) {
        float c[8], s[8];
        const float4* const at = reinterpret_cast<const float4*>(angles + 8 * (l & (LANES / 2 - 1)));
        const float4 c0 = at[0], c1 = at[1], s0 = at[D / 8], s1 = at[D / 8 + 1];
        c[0] = c0.x; c[1] = c0.y; c[2] = c0.z; c[3] = c0.w; c[4] = c1.x; c[5] = c1.y; c[6] = c1.z; c[7] = c1.w;
        s[0] = s0.x; s[1] = s0.y; s[2] = s0.z; s[3] = s0.w; s[4] = s1.x; s[5] = s1.y; s[6] = s1.z; s[7] = s1.w;
        const uint32_t sign = l < LANES / 2 ? 0x80000000u : 0u;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float other = kv8_partner<LANES / 2>(v[e]) * s[e];
            v[e] = v[e] * c[e] + __uint_as_float(__float_as_uint(other) ^ sign);
        }
    }
    if (rotate) {
        register_stages<3>(v, 0);
        auto stage = [&](int m, auto partner) {
            const uint32_t sign = (l & m) != 0 ? 0x80000000u : 0u;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = partner(v[e]) + __uint_as_float(__float_as_uint(v[e]) ^ sign);
        };
        stage(1, [](float z) { return kv8_partner<1>(z); });
        stage(2, [](float z) { return kv8_partner<2>(z); });
        stage(4, [](float z) { return kv8_partner<4>(z); });
        if constexpr (D == 128) stage(8, [](float z) { return kv8_partner<8>(z); });
        const float norm = D == 128 ? 0.088388347648318440550f : 0.125f;  // (float)(1 / sqrt(D))
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = v[e] * norm;
    }
}

// the largest finite magnitude, as bits (which order like the numbers)
__device__ __forceinline__ uint32_t kv8_top(const float (&v)[8])
{
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t u = __float_as_uint(v[e]) & 0x7fffffffu;
        top = max(top, u < 0x7f800000u ? u : 0u);
    }
    return top;
}

template <int LANES>
__device__ __forceinline__ uint32_t kv8_lanes_max(uint32_t v)
{
    v = max(v, kv8_partner<1>(v));
    v = max(v, kv8_partner<2>(v));
    v = max(v, kv8_partner<4>(v));
    if constexpr (LANES == 16) v = max(v, kv8_partner<8>(v));
    return v;
}

// 2^E for a page whose largest magnitude has these bits: 448 = 1.75 * 2^8
__device__ __forceinline__ float kv8_scale(uint32_t top)
{
    const int e = static_cast<int>(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    return __uint_as_float(static_cast<uint32_t>(kv8_clamp(e, -40, 120) + 127) << 23);
}

// Eight values times `by` as codes, to the nearest, ties to even; an infinity becomes 448 of its sign, a NaN 0.
__device__ __forceinline__ uint2 kv8_encode(const float (&v)[8], float by)
{
    float t[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = v[e] * by;
        t[e] = x == x ? fminf(fmaxf(x, -448.0f), 448.0f) : 0.0f;
    }
    uint2 r;
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(t[0], t[1], 0, false);
    r.x = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(t[2], t[3], w, true));
    w = __builtin_amdgcn_cvt_pk_fp8_f32(t[4], t[5], 0, false);
    r.y = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(t[6], t[7], w, true));
    return r;
}

// older codes at a larger scale: `by` = old scale / new scale
__device__ __forceinline__ uint2 kv8_rescale(uint2 c, float by)
{
    float v[8];
    const uint32_t w[2] = {c.x, c.y};
#pragma unroll
    for (int d = 0; d < 2; ++d) {
        const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[d]), false);
        const auto b = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[d]), true);
        v[4 * d] = a[0];
        v[4 * d + 1] = a[1];
        v[4 * d + 2] = b[0];
        v[4 * d + 3] = b[1];
    }
    return kv8_encode(v, by);
}

template <int DT>
__device__ __forceinline__ void kv8_store(void* p, size_t i, const float (&v)[8])
{
    if constexpr (DT == RCP_F32) {
        float4* const d = reinterpret_cast<float4*>(static_cast<float*>(p) + i);
        d[0] = make_float4(v[0], v[1], v[2], v[3]);
        d[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        uint16_t h[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (DT == RCP_F16) h[e] = __half_as_ushort(round_to_half(v[e]));
            else {
                const __bf16 b = static_cast<__bf16>(v[e]);
                h[e] = __builtin_bit_cast(uint16_t, b);
            }
        }
        uint4 w;
        w.x = h[0] | static_cast<uint32_t>(h[1]) << 16;
        w.y = h[2] | static_cast<uint32_t>(h[3]) << 16;
        w.z = h[4] | static_cast<uint32_t>(h[5]) << 16;
        w.w = h[6] | static_cast<uint32_t>(h[7]) << 16;
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + i) = w;
    }
}

// The queries of U x 256 / (D / 8) consecutive (token, head) rows.  In a prompt several vectors a lane, whose loads are under way together, and the
// starts of the sequences in LDS: a search through them in memory is a chain of loads (7273 tokens of 32 + 2 x 8 heads of 128 57 us instead of
// 44; with eight vectors a lane 52).
template <int DT, int D, int U>
__device__ __forceinline__ void kv8_queries(const Kv8AppendArgs& a, int block)
{
    constexpr int LANES = D / 8, ROWS = 256 / LANES;
    __shared__ int starts[U == 1 ? 1 : KV8_MOST_SEQUENCES + 1];
    const int l = threadIdx.x % LANES;
    if constexpr (U > 1) {
        for (int i = threadIdx.x; i <= a.t.sequences; i += 256) starts[i] = a.t.starts[i];
        __syncthreads();
    }
    Raw8<DT> raw[U];
    int pos[U];
    size_t to[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int row = (block * U + u) * ROWS + threadIdx.x / LANES;
        const int t = row / a.H_q, h = row - t * a.H_q;
        // rows beyond the call and rows of no sequence take no part; the lanes of a vector agree
        int b = -1;
        if (t < a.rows) b = U == 1 ? t : kv8_sequence_of(starts, a.t.sequences, t, a.rows);
        pos[u] = -1;
        if (b >= 0) {
            raw[u] = load8_raw<DT>(a.q, static_cast<size_t>(t) * a.q_stride + h * D + 8 * l);
            const Kv8Run r = kv8_run(U == 1 ? nullptr : starts, a.t.lengths, b, a.rows);
            pos[u] = r.pos + (t - r.first);
        }
        to[u] = (static_cast<size_t>(t) * a.H_q + h) * D + 8 * l;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (pos[u] < 0 || pos[u] >= a.t.capacity) continue;
        float v[8];
        widen8<DT>(raw[u], v);
        kv8_turn<D>(v, l, a.rope != nullptr ? a.rope + static_cast<size_t>(pos[u]) * D : nullptr, a.rotate != 0);
        kv8_store<DT>(a.q_out, to[u], v);
    }
}

// One new token a sequence: a vector is all that its page and head gets, so that its lanes need no other wavefront.
// Bound by the launch and one chain of loads, length -> page -> scale and codes: 2.7 us (one sequence of 32 + 2 x 32 heads of 128), 3.3 us (16 of 32 + 2 x 8).
// So where no scale grows.  A page whose scale does has its older codes read and written, eight at a time: 12.9 and 13.4 us if that is every page, with 63 older tokens in each.
template <int DT, int D>
__global__ __launch_bounds__(256) void kv8_append_one_kernel(Kv8AppendArgs a)
{
    constexpr int LANES = D / 8, ROWS = 256 / LANES;
    if (static_cast<int>(blockIdx.x) >= a.kv_groups) {
        kv8_queries<DT, D, 1>(a, blockIdx.x - a.kv_groups);
        return;
    }
    const int half = a.kv_groups / 2;
    const bool values = static_cast<int>(blockIdx.x) >= half;
    const int row = (static_cast<int>(blockIdx.x) - (values ? half : 0)) * ROWS + threadIdx.x / LANES, l = threadIdx.x % LANES;
    const int b = row / a.H, h = row - b * a.H;
    if (b >= a.t.sequences) return;
    const int pos = kv8_clamp(a.t.lengths[b], 0, KV8_MOST_TOKENS) - 1;
    if (pos < 0 || pos >= a.t.capacity) return;
    const int id = a.t.table[static_cast<size_t>(b) * a.t.width + (pos >> a.t.shift)], slot = pos & ((1 << a.t.shift) - 1);
    if (static_cast<unsigned>(id) >= static_cast<unsigned>(a.t.n_pages)) return;
    float v[8];
    load8_as_float<DT>(values ? a.v : a.k, static_cast<size_t>(b) * (values ? a.v_stride : a.k_stride) + h * D + 8 * l, v);
    if (!values) kv8_turn<D>(v, l, a.rope != nullptr ? a.rope + static_cast<size_t>(pos) * D : nullptr, a.rotate != 0);
    const size_t unit = static_cast<size_t>(id) * a.H + h;
    float* const scale_at = (values ? a.v_scales : a.k_scales) + unit;
    uint2* const codes = (values ? a.v_codes : a.k_codes) + (unit << a.t.shift) * LANES + l;
    const float old = slot > 0 ? *scale_at : 0.0f;
    const float scale = fmaxf(old, kv8_scale(kv8_lanes_max<LANES>(kv8_top(v))));
    if (scale > old && slot > 0) {
        const float by = old / scale;
        for (int s = 0; s < slot; s += 8) {
            uint2 c[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) c[u] = codes[min(s + u, slot - 1) * LANES];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (s + u < slot) codes[(s + u) * LANES] = kv8_rescale(c[u], by);
        }
    }
    codes[slot * LANES] = kv8_encode(v, 1.0f / scale);
    if (l == 0 && scale != old) *scale_at = scale;
}

// Bound by memory: 7273 tokens of 32 + 2 x 8 heads of 128 in bfloat16 read and write 167 MB in 40.7 us, 4.1 TB/s, where a copy reaches 4.6 (the
// same within a hundredth where the scale of every page with older tokens grows: they are seven of 230).
// Several new tokens of a sequence: a workgroup owns one page of one head, keeps its new tokens in registers (PASSES vectors a lane) until
// their largest magnitude is known, and writes them together.
template <int DT, int D, int PASSES>
__global__ __launch_bounds__(256) void kv8_append_pages_kernel(Kv8AppendArgs a)
{
    constexpr int LANES = D / 8, ROWS = 256 / LANES;
    __shared__ uint32_t red[4];
    const int block = static_cast<int>(blockIdx.y << KV8_GRID_SHIFT | blockIdx.x);
    if (block >= a.kv_groups) {
        if (block < a.groups) kv8_queries<DT, D, KV8_QUERIES>(a, block - a.kv_groups);
        return;
    }
    // Workgroups go to the eight dies in turn; a die gets all heads of a page one after the other, since they read the same angles (7273 tokens
    // of 32 + 2 x 8 heads of 128 42.4 us, with a die to each head 44.5; without a position rotation 36.9 and 36.4).
    const int eighth = block >> 3, round = eighth / (2 * a.H), part = eighth - round * 2 * a.H;
    const int unit_of = 8 * round + (block & 7);
    const bool values = part >= a.H;
    const int h = values ? part - a.H : part;
    const int tid = threadIdx.x, lane = tid & 63, l = tid % LANES;
    const Kv8Unit u = kv8_find(a.t.sequences, unit_of, lane, [&](int b) {
        return kv8_pages(kv8_run(a.t.starts, a.t.lengths, b, a.rows), a.t.capacity, a.t.shift).pages;
    });
    if (u.b < 0) return;
    const Kv8Run r = kv8_run(a.t.starts, a.t.lengths, u.b, a.rows);
    const int page = kv8_pages(r, a.t.capacity, a.t.shift).first_page + u.within;
    const int id = a.t.table[static_cast<size_t>(u.b) * a.t.width + page];
    if (static_cast<unsigned>(id) >= static_cast<unsigned>(a.t.n_pages)) return;
    const int base = page << a.t.shift;  // position of slot 0
    const int from = max(r.pos, 0) - base, to = min(r.length, a.t.capacity) - base;
    const int s0 = max(from, 0), s1 = min(to, 1 << a.t.shift);  // new slots of this page, not empty
    const void* const x = values ? a.v : a.k;
    const long long stride = values ? a.v_stride : a.k_stride;

    Raw8<DT> raw[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {  // lanes beyond the last token repeat it and store nothing
        const int slot = min(s0 + p * ROWS + tid / LANES, s1 - 1);
        raw[p] = load8_raw<DT>(x, static_cast<size_t>(r.first + (base + slot - r.pos)) * stride + h * D + 8 * l);
    }
    const size_t unit = static_cast<size_t>(id) * a.H + h;
    float* const scale_at = (values ? a.v_scales : a.k_scales) + unit;
    uint2* const codes = (values ? a.v_codes : a.k_codes) + (unit << a.t.shift) * LANES;
    const float old = s0 > 0 ? *scale_at : 0.0f;
    float v[PASSES][8];
    uint32_t top = 0;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int slot = min(s0 + p * ROWS + tid / LANES, s1 - 1);
        widen8<DT>(raw[p], v[p]);
        if (!values) kv8_turn<D>(v[p], l, a.rope != nullptr ? a.rope + static_cast<size_t>(base + slot) * D : nullptr, a.rotate != 0);
        top = max(top, kv8_top(v[p]));
    }
    top = kv8_lanes_max<16>(top);
    top = max(max(__builtin_amdgcn_readlane(top, 0), __builtin_amdgcn_readlane(top, 16)),
              max(__builtin_amdgcn_readlane(top, 32), __builtin_amdgcn_readlane(top, 48)));
    if (lane == 0) red[tid >> 6] = top;
    __syncthreads();  // every wavefront has read the old scale, too
    top = max(max(red[0], red[1]), max(red[2], red[3]));
    const float scale = fmaxf(old, kv8_scale(top)), by = 1.0f / scale;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int slot = s0 + p * ROWS + tid / LANES;
        if (slot < s1) codes[static_cast<size_t>(slot) * LANES + l] = kv8_encode(v[p], by);
    }
    if (scale > old && s0 > 0) {
        const float less = old / scale;
        for (int i = tid; i < s0 * LANES; i += 256) codes[i] = kv8_rescale(codes[i], less);
    }
    if (tid == 0 && scale != old) *scale_at = scale;
}

// ---------------------------------------------------------------------------------------
int launch_kv8_append(const Kv8AppendCall& c, hipStream_t st)
{
    Kv8AppendArgs a;
    a.t = {c.starts, c.lengths, c.table, c.sequences, c.width, c.shift, c.n_pages, c.width << c.shift};
    a.k = c.k;
    a.v = c.v;
    a.q = c.q;
    a.q_out = c.q_out;
    a.k_stride = c.k_stride;
    a.v_stride = c.v_stride;
    a.q_stride = c.q_stride;
    a.rope = c.rope;
    a.k_codes = static_cast<uint2*>(c.k_codes);
    a.v_codes = static_cast<uint2*>(c.v_codes);
    a.k_scales = c.k_scales;
    a.v_scales = c.v_scales;
    a.rows = c.rows;
    a.H = c.H;
    a.H_q = c.q != nullptr ? c.H_q : 0;
    a.rotate = c.rotate;
    const int vectors = 2048 / c.D;  // of a workgroup
    const bool one = c.starts == nullptr;
    a.kv_groups = one ? 2 * ((c.sequences * c.H + vectors - 1) / vectors)
                      : static_cast<int>((kv8_most_pages(c.rows, c.sequences, c.shift) + 7) / 8 * 8) * 2 * c.H;
    const int q_vectors = one ? vectors : KV8_QUERIES * vectors;
    const long long q_groups = (static_cast<long long>(c.rows) * a.H_q + q_vectors - 1) / q_vectors;
    a.groups = a.kv_groups + static_cast<int>(q_groups);
    const unsigned row = 1u << KV8_GRID_SHIFT, groups = static_cast<unsigned>(a.groups);
    const dim3 grid = groups <= row ? dim3(groups) : dim3(row, (groups + row - 1) / row);
    auto launch = [&](auto kernel) { enqueue(kernel, grid, 256, 0, st, a); };
    const int passes = (c.D << c.shift) / 2048;  // vectors a lane for a whole page: 0 (half a pass), 1, 2, 4, 8
#define RCP_KV8_APPEND(DT, D)                                                   \
    do {                                                                        \
        if (one) launch(&kv8_append_one_kernel<DT, D>);                         \
        else if (passes <= 1) launch(&kv8_append_pages_kernel<DT, D, 1>);       \
        else if (passes == 2) launch(&kv8_append_pages_kernel<DT, D, 2>);       \
        else if (passes == 4) launch(&kv8_append_pages_kernel<DT, D, 4>);       \
        else if constexpr (D == 128) launch(&kv8_append_pages_kernel<DT, D, 8>); \
    } while (0)
#define RCP_KV8_APPEND_D(DT)                  \
    do {                                      \
        if (c.D == 128) RCP_KV8_APPEND(DT, 128); \
        else RCP_KV8_APPEND(DT, 64);          \
    } while (0)
    if (c.dtype == RCP_F32) RCP_KV8_APPEND_D(RCP_F32);
    else if (c.dtype == RCP_F16) RCP_KV8_APPEND_D(RCP_F16);
    else RCP_KV8_APPEND_D(RCP_BF16);
#undef RCP_KV8_APPEND_D
#undef RCP_KV8_APPEND
    return check_launch("rcp_kv8_append");
}

}  // namespace rcp
