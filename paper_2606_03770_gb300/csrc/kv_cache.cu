// kv_cache.cu -- e2_cache_append, e2_cache_read and e2_cache_keep: tokens into, out of and within
// the paged 4-bit cache.
//
// A lane holds eight neighbouring elements of a head (16 bytes in, one word of
// codes out), eight lanes a group of E2_CACHE_GROUP, so a group's minimum and
// maximum are three shuffles and all traffic is in 16-, 32- and 64-byte runs.
//
// Measured, us: 8 tokens (64 query heads, 8 of keys and values, 128 elements) 2.4 in, 1.7 out,
// a launch; 2,048 tokens 24 in (3.2 TB/s, 48% of the memory's rate), 7 out.  Bound by
// instructions: the divisions were 4 us of 2,048 tokens' time; four heads a lane, which share
// their cosines, are no faster (25), eight slower (36).
#include <algorithm>
#include <memory>
#include <new>

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

// Tokens of accepted ways, to their places.  A warp has a request's tokens of one layer and head:
// it reads them all, keys and values, in pieces of 16 bytes (and the scales, four or eight), and
// writes them then, so that a token may go where another comes from.  Bound by the way to the
// first byte, of addresses that hang on one another (lengths, nodes, pages): 2.6 us for one layer of a
// request, 4.3 for 80 layers of 8 requests (3.6 MB read), where registers for ways of 64 nodes took 8.4.
struct KeepParams {
    int layers, batch, cols, pages, page_shift, kv_heads, table_cols;
    const unsigned long long *arrays;
    const int32_t *table, *lens, *starts, *nodes, *kept;
    int64_t table_stride, nodes_stride;
    int32_t *lens_out;
};

template <int D> __global__ void __launch_bounds__(kThreads) keep_kernel(const KeepParams p)
{
    // of a token: keys' pieces and scales, values' pieces and scales
    constexpr int kPieces = D / 32, kItems = 2 * (kPieces + 1), kMost = (E2_MAX_DRAFT * kItems + 31) / 32, kFew = 4;
    const int lane = threadIdx.x % 32;
    const int64_t unit = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / 32;
    if (unit >= (int64_t)p.layers * p.batch * p.kv_heads) return;
    const int head = (int)(unit % p.kv_heads), request = (int)(unit / p.kv_heads % p.batch), layer = (int)(unit / p.kv_heads / p.batch);
    const int32_t *nodes = p.nodes + request * p.nodes_stride, *table = p.table + request * p.table_stride;
    const unsigned long long *arrays = p.arrays + 4 * layer;
    // (what hangs on nothing is asked for at once: the first nodes before it is known how many count)
    int first_nodes[kFew];
#pragma unroll
    for (int i = 0; i < kFew; ++i) first_nodes[i] = (32 * i + lane) / kItems < p.cols ? nodes[(32 * i + lane) / kItems] : -1;
    const int64_t count = (int64_t)p.starts[request + 1] - p.starts[request], base = p.lens[request] - count;
    const int kept = (int)max(min(min((int64_t)p.kept[request], count), (int64_t)p.cols), (int64_t)0);
    if (layer == 0 && head == 0 && lane == 0) p.lens_out[request] = (int32_t)max(base + kept, (int64_t)0);
    // the head vector of a token, -1 where it is not in the cache
    auto vector_at = [&](int64_t token) {
        if (token < 0 || token >> p.page_shift >= p.table_cols) return (int64_t)-1;
        const int page = table[token >> p.page_shift];
        if (page < 0 || page >= p.pages) return (int64_t)-1;
        return (((int64_t)page * p.kv_heads + head) << p.page_shift) + (token & ((1 << p.page_shift) - 1));
    };
    const int items = kept * kItems;
    constexpr int kScales = D / E2_CACHE_GROUP * 4;
    auto read = [&](int item, int node, uint4 &what, uint8_t *&where) {
        where = nullptr;
        const int k = item / kItems, rest = item % kItems, which = rest / (kPieces + 1), piece = rest % (kPieces + 1);
        if (item >= items || node == k || node < 0 || node >= count) return;
        const int64_t from = vector_at(base + node), to = vector_at(base + k);
        if (from < 0 || to < 0) return;
        const bool scales = piece == kPieces;
        uint8_t *array = reinterpret_cast<uint8_t *>(arrays[2 * which + scales]);
        if (scales) {
            where = array + to * kScales;
            if (kScales == 8) {
                const uint2 two = *reinterpret_cast<const uint2 *>(array + from * kScales);
                what = uint4{two.x, two.y, 0, 0};
            } else {
                what = uint4{*reinterpret_cast<const uint32_t *>(array + from * kScales), 0, 0, 0};
            }
        } else {
            where = array + to * (D / 2) + piece * 16;
            what = *reinterpret_cast<const uint4 *>(array + from * (D / 2) + piece * 16);
        }
    };
    auto write = [&](int item, const uint4 &what, uint8_t *where) {
        if (!where) return;
        if (item % (kPieces + 1) != kPieces) *reinterpret_cast<uint4 *>(where) = what;
        else if (kScales == 8) *reinterpret_cast<uint2 *>(where) = make_uint2(what.x, what.y);
        else *reinterpret_cast<uint32_t *>(where) = what.x;
    };
    if (items <= 32 * kFew) {
        uint4 what[kFew];
        uint8_t *where[kFew];
#pragma unroll
        for (int i = 0; i < kFew; ++i) read(32 * i + lane, first_nodes[i], what[i], where[i]);
        __syncwarp();                                      // (all have been read)
#pragma unroll
        for (int i = 0; i < kFew; ++i) write(32 * i + lane, what[i], where[i]);
    } else {
        // (long ways: in local memory, which costs the others no registers)
        uint4 what[kMost];
        uint8_t *where[kMost];
#pragma unroll 1
        for (int i = 0; 32 * i < items; ++i) {
            const int item = 32 * i + lane;
            read(item, item < items ? nodes[item / kItems] : -1, what[i], where[i]);
        }
        __syncwarp();
#pragma unroll 1
        for (int i = 0; 32 * i < items; ++i) write(32 * i + lane, what[i], where[i]);
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

extern "C" int e2_cache_layers(const e2_cache *caches, int32_t layers, uint64_t *arrays)
{
    Device dev;
    if (!caches || !arrays || layers < 1) return fail(E2_EINVAL, "caches and arrays must be given, layers positive");
    if (int st = current_device(&dev)) return st;
    struct Place {
        uintptr_t from, to;
    };
    const size_t n = 4 * (size_t)layers;
    const std::unique_ptr<Place[]> places(new (std::nothrow) Place[n]);
    if (!places) return fail(E2_ENOMEM, "no host memory");
    for (int32_t i = 0; i < layers; ++i) {
        const e2_cache &c = caches[i];
        if (int st = check_cache(&c, dev.id)) return st;
        if (c.pages != caches->pages || c.page_size != caches->page_size || c.kv_heads != caches->kv_heads ||
            c.head_dim != caches->head_dim)
            return fail(E2_EINVAL, "the layers' caches must be of one shape");
        const uintptr_t vectors = (uintptr_t)c.pages * c.page_size * c.kv_heads;
        const void *of[4] = {c.k_codes, c.k_scales, c.v_codes, c.v_scales};
        for (int k = 0; k < 4; ++k) {
            const uintptr_t at = (uintptr_t)of[k];
            places[4 * (size_t)i + k] = {at, at + vectors * (k % 2 ? c.head_dim / E2_CACHE_GROUP * 4 : c.head_dim / 2)};
            arrays[4 * (size_t)i + k] = (uint64_t)at;
        }
    }
    std::sort(places.get(), places.get() + n, [](const Place &a, const Place &b) { return a.from < b.from; });
    for (size_t i = 1; i < n; ++i)
        if (places[i].from < places[i - 1].to) return fail(E2_EINVAL, "the layers' caches must not share memory");
    return E2_OK;
}

extern "C" int e2_cache_keep(const e2_cache *c, const e2_keep_args *a, void *stream)
{
    Device dev;
    if (!a) return fail(E2_EINVAL, "no arguments");
    if (int st = current_device(&dev)) return st;
    if (int st = check_cache(c, dev.id)) return st;
    if (a->batch < 0 || a->layers < 1 || a->cols < 0 || a->cols > E2_MAX_DRAFT)
        return fail(E2_EINVAL, "batch must not be negative, layers positive, cols in 0..E2_MAX_DRAFT");
    if (a->table_cols < 1 || a->table_stride < a->table_cols || a->nodes_stride < a->cols)
        return fail(E2_EINVAL, "table_cols in 1..table_stride, cols up to nodes_stride");
    if (a->batch == 0) return E2_OK;
    const void *ptrs[] = {a->arrays, a->table, a->lens, a->starts, a->kept, a->lens_out, a->cols ? a->nodes : a->lens};
    for (const void *p : ptrs)
        if (!p || !aligned(p, p == a->arrays ? 8 : 4) || !on_device(p, dev.id))
            return fail(E2_EINVAL, "arrays must be given, memory of the current device");
    // (what others may still have to read when a request's length is written)
    auto apart = [&](const int32_t *of, int64_t n) { return a->lens_out + a->batch <= of || of + n <= a->lens_out; };
    if (!apart(a->lens, a->batch) || !apart(a->starts, (int64_t)a->batch + 1) || !apart(a->kept, a->batch) ||
        !apart(a->table, (a->batch - 1) * a->table_stride + a->table_cols) ||
        (a->cols && !apart(a->nodes, (a->batch - 1) * a->nodes_stride + a->cols)))
        return fail(E2_EINVAL, "lens_out may not share memory with lens, starts, kept, nodes or table");
    const int64_t threads = (int64_t)a->layers * a->batch * c->kv_heads * 32, blocks = (threads + kThreads - 1) / kThreads;
    if (a->layers > (1 << 20) || a->batch > (1 << 20) || blocks > 0x7fffffff) return fail(E2_EINVAL, "too many layers and requests for one call");
    const KeepParams p{a->layers, a->batch, a->cols, c->pages, __builtin_ctz((unsigned)c->page_size), c->kv_heads, a->table_cols,
                       reinterpret_cast<const unsigned long long *>(a->arrays), a->table, a->lens, a->starts, a->nodes, a->kept,
                       a->table_stride, a->nodes_stride, a->lens_out};
    (c->head_dim == 64 ? keep_kernel<64> : keep_kernel<128>)<<<(unsigned)blocks, kThreads, 0, static_cast<cudaStream_t>(stream)>>>(p);
    return cuda_status(cudaGetLastError());
}
