// kv_cache.cu -- e2_cache_append and e2_cache_read: tokens into and out of the
// paged 4-bit cache.
//
// A lane holds eight neighbouring elements of a head (16 bytes in, one word of
// codes out), eight lanes a group of E2_CACHE_GROUP, so a group's minimum and
// maximum are three shuffles and all traffic is in 16-, 32- and 64-byte runs.
//
// Measured, us: 8 tokens (64 query heads, 8 of keys and values, 128 elements) 2.4 in, 1.7 out,
// a launch; 2,048 tokens 24 in (3.2 TB/s, 48% of the memory's rate), 7 out.  Bound by
// instructions: the divisions were 4 us of 2,048 tokens' time; four heads a lane, which share
// their cosines, are no faster (25), eight slower (36).
#include "ops_common.cuh"

namespace e2ops {
namespace {

constexpr int kThreads = 128;
constexpr float kHalfMax = 65504.0f;

struct Cache {
    int64_t slots;
    int page_shift, kv_heads;
    uint8_t *codes[2];
    uint16_t *scales[2];
};

// The position of (slot, head) among the cache's head vectors.
__device__ __forceinline__ int64_t vector_of(const Cache &c, int64_t slot, int head)
{
    const int64_t page = slot >> c.page_shift, at = slot & ((1 << c.page_shift) - 1);
    return (((page * c.kv_heads + head) << c.page_shift) + at);
}

// A unit's token and its place among the token's `per` (32 bits where they do).
__device__ __forceinline__ void place_of(int64_t unit, int per, int &token, int &at)
{
    token = (int)(unit >> 32 ? unit / per : (unsigned)unit / (unsigned)per);
    at = (int)(unit - (int64_t)token * per);
}

struct AppendParams {
    Cache c;
    int tokens, q_heads, rot, interleaved, table_rows;
    const int64_t *slots;
    const int32_t *positions;
    const float *cos, *sin;
    const void *in[3];        // k, v, q
    int64_t stride[3];
    void *q_out;
    int64_t q_out_stride;
};

// Head vectors in the order token, then k heads, v heads, q heads.
template <class T, int D> __global__ void __launch_bounds__(kThreads) append_kernel(const AppendParams p)
{
    constexpr int kLanes = D / 8;
    const int per = 2 * p.c.kv_heads + p.q_heads;
    const int64_t unit = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / kLanes;
    const int lane = threadIdx.x % kLanes;                 // of the head vector
    const bool live = unit < (int64_t)p.tokens * per;      // (all lanes take part in the shuffles)
    int t, h;
    place_of(live ? unit : 0, per, t, h);
    const int kind = h < p.c.kv_heads ? 0 : h < 2 * p.c.kv_heads ? 1 : 2;
    const int head = h - kind * p.c.kv_heads;
    const int64_t slot = p.slots[t];
    const int pos = p.positions[t];
    const bool placed = pos >= 0 && pos < p.table_rows;

    const T *src = static_cast<const T *>(p.in[kind]) + t * p.stride[kind] + head * D;
    const uint4 raw = live ? *reinterpret_cast<const uint4 *>(src + 8 * lane) : uint4{0, 0, 0, 0};
    float x[8];
    unpack8<T>(raw, x);

    // the turn: each product and each sum rounded to 32 bits
    const int half = p.rot / 2;
    const int partner = lane + (8 * lane < half ? half / 8 : -half / 8);
    uint4 other;
    const int from = (threadIdx.x & 31) - lane + (8 * lane < p.rot && !p.interleaved ? partner : lane);
    other.x = __shfl_sync(~0u, raw.x, from);
    other.y = __shfl_sync(~0u, raw.y, from);
    other.z = __shfl_sync(~0u, raw.z, from);
    other.w = __shfl_sync(~0u, raw.w, from);
    if (kind != 1 && placed && 8 * lane < p.rot) {
        const float *cs = p.cos + (int64_t)pos * half, *sn = p.sin + (int64_t)pos * half;
        if (p.interleaved) {
            const float4 c4 = *reinterpret_cast<const float4 *>(cs + 4 * lane);
            const float4 s4 = *reinterpret_cast<const float4 *>(sn + 4 * lane);
            const float c[4] = {c4.x, c4.y, c4.z, c4.w}, s[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a = x[2 * i], b = x[2 * i + 1];
                x[2 * i] = __fsub_rn(__fmul_rn(a, c[i]), __fmul_rn(b, s[i]));
                x[2 * i + 1] = __fadd_rn(__fmul_rn(b, c[i]), __fmul_rn(a, s[i]));
            }
        } else {
            const bool first = 8 * lane < half;
            const int i0 = first ? 8 * lane : 8 * lane - half;
            float y[8];
            unpack8<T>(other, y);
#pragma unroll
            for (int j = 0; j < 8; j += 4) {
                const float4 c4 = *reinterpret_cast<const float4 *>(cs + i0 + j);
                const float4 s4 = *reinterpret_cast<const float4 *>(sn + i0 + j);
                const float c[4] = {c4.x, c4.y, c4.z, c4.w}, s[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    x[j + i] = __fadd_rn(__fmul_rn(x[j + i], c[i]), __fmul_rn(y[j + i], first ? -s[i] : s[i]));
            }
        }
    }
    if (kind == 2) {
        if (!placed) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __int_as_float(0x7fc00000);
        }
        if (live) {
            T *dst = static_cast<T *>(p.q_out) + t * p.q_out_stride + head * D;
            *reinterpret_cast<uint4 *>(dst + 8 * lane) = pack8<T>(x);
        }
    }

    if (!__any_sync(~0u, kind != 2 && live)) return;

    float lo = x[0], hi = x[0];
    bool nan = x[0] != x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        lo = fminf(lo, x[i]);
        hi = fmaxf(hi, x[i]);
        nan |= x[i] != x[i];
    }
#pragma unroll
    for (int o = 4; o; o >>= 1) {
        lo = fminf(lo, __shfl_xor_sync(~0u, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(~0u, hi, o));
    }
    nan = (__ballot_sync(~0u, nan) >> (threadIdx.x & 24)) & 0xff;
    if (kind == 2 || !live || !placed || slot < 0 || slot >= p.c.slots) return;
    lo = fminf(fmaxf(lo, -kHalfMax), kHalfMax);
    hi = fminf(fmaxf(hi, -kHalfMax), kHalfMax);
    const __half m = __float2half_rn(nan ? __int_as_float(0x7fc00000) : lo);
    const __half d = __float2half_rn(nan ? 0.0f : __fdiv_rn(__fsub_rn(hi, lo), 15.0f));
    const float mf = __half2float(m), df = __half2float(d);
    uint32_t w = 0;
    if (df > 0) {
        // the quotient by a reciprocal is at most 2^-22 of it off, which tells its whole number
        // unless it is that near to a half: then it is divided
        const float inverse = __frcp_rn(df);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float above = __fsub_rn(x[i], mf);
            float q = fminf(__fmul_rn(above, inverse), 16.0f);
            if (fabsf(q - rintf(q)) > 0.4999f) q = __fdiv_rn(above, df);
            const float c = rintf(q);
            w |= (uint32_t)fminf(fmaxf(c, 0.0f), 15.0f) << (4 * i);
        }
    }
    const int64_t vec = vector_of(p.c, slot, head);
    reinterpret_cast<uint32_t *>(p.c.codes[kind])[vec * (D / 8) + lane] = w;
    if (lane % 8 == 0)
        reinterpret_cast<__half2 *>(p.c.scales[kind])[vec * (D / E2_CACHE_GROUP) + lane / 8] = __halves2half2(d, m);
}

struct ReadParams {
    Cache c;
    int tokens, dtype;
    const int64_t *slots;
    void *out[2];
    int64_t stride[2];
};

template <class T, int D> __global__ void __launch_bounds__(kThreads) read_kernel(const ReadParams p)
{
    constexpr int kLanes = D / 8;
    const int64_t unit = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / kLanes;
    const int lane = threadIdx.x % kLanes;
    const int per = 2 * p.c.kv_heads;
    if (unit >= (int64_t)p.tokens * per) return;
    int t, h;
    place_of(unit, per, t, h);
    const int kind = h >= p.c.kv_heads, head = h - kind * p.c.kv_heads;
    if (!p.out[kind]) return;
    const int64_t slot = p.slots[t];
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (slot >= 0 && slot < p.c.slots) {
        const int64_t vec = vector_of(p.c, slot, head);
        const uint32_t w = reinterpret_cast<const uint32_t *>(p.c.codes[kind])[vec * (D / 8) + lane];
        const float2 dm =
            __half22float2(reinterpret_cast<const __half2 *>(p.c.scales[kind])[vec * (D / E2_CACHE_GROUP) + lane / 8]);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __fadd_rn(__fmul_rn((float)(w >> (4 * i) & 15), dm.x), dm.y);
    }
    T *dst = static_cast<T *>(p.out[kind]) + t * p.stride[kind] + head * D + 8 * lane;
    if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint4 *>(dst) = pack8<T>(x);
    } else {
        reinterpret_cast<float4 *>(dst)[0] = make_float4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<float4 *>(dst)[1] = make_float4(x[4], x[5], x[6], x[7]);
    }
}

Cache device_cache(const e2_cache *c)
{
    Cache d;
    d.page_shift = __builtin_ctz((unsigned)c->page_size);
    d.slots = (int64_t)c->pages << d.page_shift;
    d.kv_heads = c->kv_heads;
    d.codes[0] = c->k_codes;
    d.codes[1] = c->v_codes;
    d.scales[0] = c->k_scales;
    d.scales[1] = c->v_scales;
    return d;
}

bool strided(const void *p, int64_t stride, int64_t row) { return aligned(p, 16) && stride % 8 == 0 && stride >= row; }

}  // namespace

int check_cache(const e2_cache *c, int dev)
{
    if (!c) return fail(E2_EINVAL, "no cache");
    if (c->head_dim != 64 && c->head_dim != 128) return fail(E2_EINVAL, "head_dim must be 64 or 128");
    const int ps = c->page_size;
    if (ps != 16 && ps != 32 && ps != 64 && ps != 128 && ps != 256)
        return fail(E2_EINVAL, "page_size must be 16, 32, 64, 128 or 256");
    if (c->pages < 1 || c->kv_heads < 1 || c->kv_heads > 1024)
        return fail(E2_EINVAL, "pages must be positive, kv_heads in 1..1024");
    const void *a[4] = {c->k_codes, c->k_scales, c->v_codes, c->v_scales};
    for (const void *p : a) {
        if (!p || !aligned(p, 16)) return fail(E2_EINVAL, "cache arrays must be given, 16-byte aligned");
        if (!on_device(p, dev)) return fail(E2_EINVAL, "cache arrays must be memory of the current device");
    }
    return E2_OK;
}

}  // namespace e2ops

using namespace e2ops;

extern "C" int e2_cache_append(const e2_cache *c, const e2_append_args *a, void *stream)
{
    Device dev;
    if (!a) return fail(E2_EINVAL, "no arguments");
    if (int st = current_device(&dev)) return st;
    if (int st = check_cache(c, dev.id)) return st;
    if (a->tokens < 0) return fail(E2_EINVAL, "tokens must not be negative");
    if (a->dtype != E2_F16 && a->dtype != E2_BF16) return fail(E2_EINVAL, "keys and values are fp16 or bf16");
    if (a->rot < 0 || a->rot > c->head_dim || a->rot % 16)
        return fail(E2_EINVAL, "rot must be a multiple of 16 up to head_dim");
    if (a->table_rows < 1) return fail(E2_EINVAL, "table_rows must be positive");
    if (a->q_heads < 0 || a->q_heads > 4096) return fail(E2_EINVAL, "q_heads must be in 1..4096 with queries, 0 without");
    if (a->tokens == 0) return E2_OK;
    if (!a->q != !a->q_heads) return fail(E2_EINVAL, "q_heads must be in 1..4096 with queries, 0 without");
    const int64_t kv_row = (int64_t)c->kv_heads * c->head_dim, q_row = (int64_t)a->q_heads * c->head_dim;
    if (!a->k || !a->v || !strided(a->k, a->k_stride, kv_row) || !strided(a->v, a->v_stride, kv_row))
        return fail(E2_EINVAL, "k, v: 16-byte aligned, token strides multiples of 8 and at least a row");
    if (a->q && (!a->q_out || !strided(a->q, a->q_stride, q_row) || !strided(a->q_out, a->q_out_stride, q_row)))
        return fail(E2_EINVAL, "q, q_out: 16-byte aligned, token strides multiples of 8 and at least a row");
    if (!a->slots || !a->positions || (a->rot && (!a->cos || !a->sin)))
        return fail(E2_EINVAL, "slots, positions, cos and sin must be given");
    if (a->rot && (!aligned(a->cos, 16) || !aligned(a->sin, 16)))
        return fail(E2_EINVAL, "cos and sin must be 16-byte aligned");
    const void *ptrs[] = {a->k, a->v, a->slots, a->positions, a->q, a->q_out, a->rot ? a->cos : nullptr, a->rot ? a->sin : nullptr};
    for (const void *p : ptrs)
        if (p && !on_device(p, dev.id)) return fail(E2_EINVAL, "arrays must be memory of the current device");
    AppendParams p{};
    p.c = device_cache(c);
    p.tokens = a->tokens;
    p.q_heads = a->q ? a->q_heads : 0;
    p.rot = a->rot;
    p.interleaved = a->interleaved != 0;
    p.table_rows = a->table_rows;
    p.slots = a->slots;
    p.positions = a->positions;
    p.cos = a->cos;
    p.sin = a->sin;
    p.in[0] = a->k, p.in[1] = a->v, p.in[2] = a->q;
    p.stride[0] = a->k_stride, p.stride[1] = a->v_stride, p.stride[2] = a->q_stride;
    p.q_out = a->q_out;
    p.q_out_stride = a->q_out_stride;
    const int64_t threads = (int64_t)a->tokens * (2 * c->kv_heads + p.q_heads) * (c->head_dim / 8);
    const int64_t blocks = (threads + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffff) return fail(E2_EINVAL, "too many tokens for one call");
    const bool half = a->dtype == E2_F16;
    void (*f)(AppendParams) = c->head_dim == 64 ? (half ? append_kernel<__half, 64> : append_kernel<__nv_bfloat16, 64>)
                                                : (half ? append_kernel<__half, 128> : append_kernel<__nv_bfloat16, 128>);
    f<<<(unsigned)blocks, kThreads, 0, static_cast<cudaStream_t>(stream)>>>(p);
    return cuda_status(cudaGetLastError());
}

extern "C" int e2_cache_read(const e2_cache *c, const int64_t *slots, int32_t tokens, int32_t dtype, void *k,
                             int64_t k_stride, void *v, int64_t v_stride, void *stream)
{
    Device dev;
    if (int st = current_device(&dev)) return st;
    if (int st = check_cache(c, dev.id)) return st;
    if (tokens < 0) return fail(E2_EINVAL, "tokens must not be negative");
    if (dtype != E2_F16 && dtype != E2_BF16 && dtype != E2_F32) return fail(E2_EINVAL, "unknown dtype");
    if (tokens == 0 || (!k && !v)) return E2_OK;
    const int64_t row = (int64_t)c->kv_heads * c->head_dim;
    if ((k && !strided(k, k_stride, row)) || (v && !strided(v, v_stride, row)))
        return fail(E2_EINVAL, "k, v: 16-byte aligned, token strides multiples of 8 and at least a row");
    if (!slots) return fail(E2_EINVAL, "slots must be given");
    const void *ptrs[] = {slots, k, v};
    for (const void *p : ptrs)
        if (p && !on_device(p, dev.id)) return fail(E2_EINVAL, "arrays must be memory of the current device");
    ReadParams p{};
    p.c = device_cache(c);
    p.tokens = tokens;
    p.slots = slots;
    p.out[0] = k, p.out[1] = v;
    p.stride[0] = k_stride, p.stride[1] = v_stride;
    const int64_t threads = (int64_t)tokens * 2 * c->kv_heads * (c->head_dim / 8);
    const int64_t blocks = (threads + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffff) return fail(E2_EINVAL, "too many tokens for one call");
    const bool small = c->head_dim == 64;
    void (*f)(ReadParams) = dtype == E2_F16    ? (small ? read_kernel<__half, 64> : read_kernel<__half, 128>)
                            : dtype == E2_BF16 ? (small ? read_kernel<__nv_bfloat16, 64> : read_kernel<__nv_bfloat16, 128>)
                                               : (small ? read_kernel<float, 64> : read_kernel<float, 128>);
    f<<<(unsigned)blocks, kThreads, 0, static_cast<cudaStream_t>(stream)>>>(p);
    return cuda_status(cudaGetLastError());
}
