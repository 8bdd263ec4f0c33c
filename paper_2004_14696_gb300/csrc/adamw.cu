// AdamW over many tensors in one launch, moments in fp32 or in 8 bits.
//
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
//   w -= lr ((m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps) + wd w)
//
// Bound by HBM: 28 bytes an element with fp32 moments and gradients (54.4M parameters: 215 us, 7.1 TB/s), 16.1 with
// 8-bit ones, where the operations of the draws, some 65 an element, weigh more (184 us with the bf16 copy, 5.4 TB/s).
// The plan cuts every tensor into chunks of 2048 elements, which are dealt to the CTAs evenly, so that a
// network's many small tensors and its few large ones fill the SMs alike.
//
// In 8 bits a block of 128 elements shares a scale and is a warp's: 4 neighbours per lane,
// so that its amax is one warp reduction.  The second moment is held as sqrt(v): e4m3 spans
// 2^17.8 from its least to its largest value, enough for gradients of unlike size within a
// block, but not for their squares.  Each entry is drawn as one of its two e4m3 neighbours,
// the upper one with the probability of the fraction of the way to it: a moment changes by
// less than half a step of 8 bits in most updates, which rounding to nearest would drop.
// A second moment above 0 is held at its least code or above: were it drawn to 0 while the first moment is drawn up to its
// own least code, the next step would be the quotient by the new gradient alone, hundreds of learning rates where a
// block's largest gradient is 10^5 times the entry's.  Held so, no step of 600 was above 3; such an entry's steps are
// smaller than with exact moments, as its denominator is the least code.
#include "elements.cuh"

#include <math.h>
#include <string.h>

namespace dbw {

namespace {

constexpr int kChunk = 2048;      // elements of a chunk
constexpr int kThreads = 256;
constexpr int kPerSm = 4;         // CTAs of an SM with 8-bit moments (2: 281 us, 3: 183, 4: 184, 5: 203 on 54.4M)
constexpr int64_t kPlanMagic = 0x444257504c414e31ll;

struct PlanHeader {
    int64_t magic, bytes, chunks;
    int32_t num, bits;
};
static_assert(sizeof(PlanHeader) == 32, "plan header");
struct PlanTensor {
    dbw_adamw_tensor t;
    int64_t first;     // index in the plan of its first element
    int32_t vec;       // every array allows accesses of 4 elements
    int32_t pad[3];
};
static_assert(sizeof(PlanTensor) % 16 == 0, "plan tensor");
struct PlanChunk {
    int32_t tensor, chunk;
};

// A bijection of 32-bit integers: xor-shifts and two odd multipliers (the "lowbias32" constants of
// C. Wellons' search for low-bias integer hashes).
__device__ __forceinline__ uint32_t mix(uint32_t h) {
    h ^= h >> 16;
    h *= 0x7feb352du;
    h ^= h >> 15;
    h *= 0x846ca68bu;
    return h ^ (h >> 16);
}
// The e4m3 code of z in [0, 448], up where the fraction of the way to the upper neighbour plus u in (0, 1) reaches 1.
// Times 2^-120, e4m3's least normal number is fp32's: the bits above the 20th are then the code, of subnormal
// numbers as well, those below the fraction, and u (as a multiple of 2^-20) is added to them.
__device__ __forceinline__ uint32_t draw_e4m3(float z, uint32_t u20) {
    const uint32_t code = (__float_as_uint(z * 7.52316384526264e-37f) + u20) >> 20;
    return code < 0x7eu ? code : 0x7eu;
}
// (k + 0.5) / 65536 of the low and of the high 16 bits of h, as multiples of 2^-20.
__device__ __forceinline__ uint32_t low20(uint32_t h) { return ((h << 4) & 0xffff0u) | 8u; }
__device__ __forceinline__ uint32_t high20(uint32_t h) { return ((h >> 12) & 0xffff0u) | 8u; }
__device__ __forceinline__ uint32_t pack4(const uint32_t (&c)[4]) {
    return (c[0] + (c[1] << 8)) + ((c[2] + (c[3] << 8)) << 16);
}
// Four codes of x, those of 0 raised to the least one where x is above 0.  A word without a code of 0 (no byte is above
// 0x7e, so that the sum carries into no other one) is one comparison: 184.6 us on 54.4M, 193.5 entry by entry, 180 without.
__device__ __forceinline__ uint32_t hold_least(uint32_t codes, const float (&x)[4]) {
    const uint32_t none = ~(codes + 0x7f7f7f7fu) & 0x80808080u;
    if (none) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if ((none >> (8 * j) & 0x80u) && x[j] > 0.f) codes += 1u << (8 * j);
    }
    return codes;
}
// The top bits of four words as the top bits of the bytes of one.
__device__ __forceinline__ uint32_t signs_of(const float (&x)[4]) {
    const uint32_t a = __byte_perm(__float_as_uint(x[0]), __float_as_uint(x[1]), 0x0073);
    const uint32_t b = __byte_perm(__float_as_uint(x[2]), __float_as_uint(x[3]), 0x0073);
    return __byte_perm(a, b, 0x5410) & 0x80808080u;
}
__device__ __forceinline__ float2 wide_pair(uint32_t two) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(two)));
    const __half2 v = *reinterpret_cast<const __half2*>(&h);
    return __half22float2(v);
}
// Roots and reciprocals within 2^-23 of themselves.  A step is then within 2^-21 of its size, measured 6.5 x 2^-24 at most and
// 1.2 to 2.5 x 2^-24 in the root mean square (correctly rounded 5.5, and 1.2 to 2.2), far below a rounding of w; sqrt(v), which is
// the state in 8 bits, the scales and the quotients that are drawn from are within 2^-22, as far from the exact ones as
// fp32's rounded quotient and product, and a draw is among steps of 2^-4.  Correctly rounded ones branch, and run one after
// another: 784-256-10 in fp32 4.3 us against 2.8, 54.4M in 8 bits 225 against 179.
// The root takes subnormal v as they are.  A denominator below 2^-126 counts as 0; only an eps can be one, since the
// root of the least v above 0 is 2^-74.5.
__device__ __forceinline__ float rcp_near(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float sqrt_near(float x) {
    float y;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

struct StepArgs {
    const uint8_t* plan;
    size_t plan_bytes;
    const int32_t* t;
    const float* grad_scale;
    int* status;
    float lr, beta1, beta2, rest1, rest2, eps;   // rest = 1 - beta
    float log1, log2;                            // ln beta
    float root_beta2;
    uint32_t seed;
};

struct Rule {
    float scale;                 // of the gradient, before its square is taken: the factor's own may lie outside fp32
    float beta1, rest1;          // m = beta1 m + rest1 g
    float beta2, rest2;          // v = beta2 v + rest2 g^2
    float step;                  // lr / (1 - beta1^t)
    float root, eps;             // 1 / sqrt(1 - beta2^t)
    float decay;                 // lr * weight decay
};
// The element's parameter from its moments; returns sqrt(v).  The decay joins the step before w is rounded: as a factor
// 1 - lr * weight decay it would be a multiple of 2^-24, off the same way for every weight and step.
__device__ __forceinline__ float step_w(const Rule& r, float& w, float m, float v) {
    const float s = sqrt_near(v);
    w -= fmaf(r.step * m, rcp_near(fmaf(s, r.root, r.eps)), r.decay * w);
    return s;
}

__device__ __forceinline__ void load4(const void* p, int type, int64_t i, float (&x)[4]) {
    if (type == DBW_BF16) {
        const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(p) + i);
        x[0] = __uint_as_float(w.x << 16), x[1] = __uint_as_float(w.x & 0xffff0000u);
        x[2] = __uint_as_float(w.y << 16), x[3] = __uint_as_float(w.y & 0xffff0000u);
    } else {
        const float4 v = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
        x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
    }
}
// This thread's elements of a chunk: four at a time, from ``at`` on and kStride apart.  FULL: the chunk lies within its
// tensor and every array allows wide accesses; otherwise each element is looked at, zeros past the end.
constexpr int kStride = 4 * kThreads;
constexpr int kFours = kChunk / kStride;
constexpr int kPart = kChunk / 2;      // what a CTA takes at a time with 8-bit moments

template <bool FULL, class T>
__device__ __forceinline__ void load_four(const T* p, int64_t left, float (&x)[4]) {
    if constexpr (FULL) {
        load4(p, sizeof(T) == 2 ? DBW_BF16 : DBW_F32, 0, x);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = j < left ? to_f(p[j]) : 0.f;
    }
}
template <bool FULL, class I>
__device__ __forceinline__ void load_grad(const dbw_adamw_tensor& T, I i, int64_t left, float (&x)[4]) {
    if (T.g_type == DBW_BF16)
        load_four<FULL>(static_cast<const __nv_bfloat16*>(T.g) + i, left, x);
    else
        load_four<FULL>(static_cast<const float*>(T.g) + i, left, x);
}
template <bool FULL>
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int64_t left) {
    if constexpr (FULL) return *reinterpret_cast<const uint32_t*>(p);
    uint32_t c = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) c |= j < left ? static_cast<uint32_t>(p[j]) << (8 * j) : 0u;
    return c;
}
template <bool FULL>
__device__ __forceinline__ void store_four(float* p, int64_t left, const float (&x)[4]) {
    if constexpr (FULL) {
        *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) p[j] = x[j];
    }
}
template <bool FULL>
__device__ __forceinline__ void store_four(__nv_bfloat16* p, int64_t left, const float (&x)[4]) {
    if constexpr (FULL) {
        *reinterpret_cast<uint2*>(p) = make_uint2(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) put(p + j, x[j]);
    }
}
template <bool FULL>
__device__ __forceinline__ void store_codes(uint8_t* p, int64_t left, uint32_t c) {
    if constexpr (FULL) {
        *reinterpret_cast<uint32_t*>(p) = c;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) p[j] = static_cast<uint8_t>(c >> (8 * j));
    }
}

// fp32 moments.
template <bool FULL>
__device__ __forceinline__ void step_chunk32(const dbw_adamw_tensor& T, const Rule& rule, int64_t at) {
    const int64_t left = T.n - at;
    const float *w = T.w + at, *m = static_cast<const float*>(T.m) + at, *v = static_cast<const float*>(T.v) + at;
    float *wo = T.w_out + at, *mo = static_cast<float*>(T.m_out) + at, *vo = static_cast<float*>(T.v_out) + at;
    __nv_bfloat16* w16 = T.w_bf16 ? static_cast<__nv_bfloat16*>(T.w_bf16) + at : nullptr;
    float xg[kFours][4], xw[kFours][4], xm[kFours][4], xv[kFours][4];
    // a thread's loads first, all of them on their way together
#pragma unroll
    for (int k = 0; k < kFours; ++k) {
        load_grad<FULL>(T, at + k * kStride, left - k * kStride, xg[k]);
        load_four<FULL>(w + k * kStride, left - k * kStride, xw[k]);
        load_four<FULL>(m + k * kStride, left - k * kStride, xm[k]);
        load_four<FULL>(v + k * kStride, left - k * kStride, xv[k]);
    }
#pragma unroll
    for (int k = 0; k < kFours; ++k) {
        const int64_t rest = left - k * kStride;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float g = rule.scale * xg[k][j];
            xm[k][j] = fmaf(rule.rest1, g, rule.beta1 * xm[k][j]);
            xv[k][j] = fmaf(rule.rest2 * g, g, rule.beta2 * xv[k][j]);
            step_w(rule, xw[k][j], xm[k][j], xv[k][j]);
        }
        store_four<FULL>(wo + k * kStride, rest, xw[k]);
        store_four<FULL>(mo + k * kStride, rest, xm[k]);
        store_four<FULL>(vo + k * kStride, rest, xv[k]);
        if (w16) store_four<FULL>(w16 + k * kStride, rest, xw[k]);
    }
}

// What every draw of a chunk of elements has in common: the low 32 bits of its first index and
// the keys of the high ones, this one and the next.
struct Draws {
    uint32_t first, key, key_next;
};

// 8-bit moments: a warp's block of 128, four elements per lane.
struct Block8 {
    float g[4], w[4], ms, vs;
    uint32_t m, v;     // four codes each
};
template <bool FULL, class I>
__device__ __forceinline__ void load_block8(const dbw_adamw_tensor& T, I at, Block8& x) {
    const int64_t left = T.n - at;
    load_grad<FULL>(T, at, left, x.g);
    load_four<FULL>(T.w + at, left, x.w);
    x.m = load_codes<FULL>(static_cast<const uint8_t*>(T.m) + at, left);
    x.v = load_codes<FULL>(static_cast<const uint8_t*>(T.v) + at, left);
    x.ms = T.m_scale[at >> 7];
    x.vs = T.v_scale[at >> 7];
}
// The larger magnitude, a NaN if either is one.
__device__ __forceinline__ float max_magnitude(float a, float b) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(fabsf(b)));
    return y;
}
// rule.beta2 is the root of beta2 here: the code's factor is rounded once and then squared.
template <bool FULL, class I>
__device__ __forceinline__ void step_block8(const dbw_adamw_tensor& T, const Rule& rule, const Draws& d, I at,
                                            uint32_t index, int lane, Block8& x) {
    const int64_t left = T.n - at;
    const float ms = rule.beta1 * x.ms, vs = rule.beta2 * x.vs;
    const float2 m01 = wide_pair(x.m & 0xffffu), m23 = wide_pair(x.m >> 16);
    const float2 v01 = wide_pair(x.v & 0xffffu), v23 = wide_pair(x.v >> 16);
    float m[4] = {m01.x, m01.y, m23.x, m23.y}, r[4] = {v01.x, v01.y, v23.x, v23.y};
    float mtop = 0.f, rtop = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float g = rule.scale * x.g[j], old = r[j] * vs;
        m[j] = fmaf(rule.rest1, g, m[j] * ms);
        r[j] = step_w(rule, x.w[j], m[j], fmaf(rule.rest2 * g, g, old * old));
        if (!FULL && j >= left) m[j] = r[j] = 0.f;
        mtop = max_magnitude(mtop, m[j]);
        rtop = max_magnitude(rtop, r[j]);
    }
    const float mmax = amax_of(warp_umax(__float_as_uint(mtop))), rmax = amax_of(warp_umax(__float_as_uint(rtop)));
    const float minv = kFp8Top * rcp_near(mmax), rinv = kFp8Top * rcp_near(rmax);
    if (lane == 0) {
        T.m_scale_out[at >> 7] = mmax * (1.f / kFp8Top);
        T.v_scale_out[at >> 7] = rmax * (1.f / kFp8Top);
    }
    uint32_t h[4], mc[4], vc[4];
    if (d.first <= 0u - kPart) {       // no index of the part has higher bits of its own
#pragma unroll
        for (int j = 0; j < 4; ++j) h[j] = mix((index + j) ^ d.key);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) h[j] = mix((index + j) ^ (index + j < d.first ? d.key_next : d.key));
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        mc[j] = draw_e4m3(fabsf(m[j] * minv), low20(h[j]));
        vc[j] = draw_e4m3(r[j] * rinv, high20(h[j]));
    }
    store_codes<FULL>(static_cast<uint8_t*>(T.m_out) + at, left, pack4(mc) | signs_of(m));
    store_codes<FULL>(static_cast<uint8_t*>(T.v_out) + at, left, hold_least(pack4(vc), r));
    store_four<FULL>(T.w_out + at, left, x.w);
    if (T.w_bf16) store_four<FULL>(static_cast<__nv_bfloat16*>(T.w_bf16) + at, left, x.w);
}

template <int BITS>
__global__ void __launch_bounds__(kThreads, BITS == 8 ? kPerSm : 4) adamw_kernel(const __grid_constant__ StepArgs a) {
    grid_begin();
    const PlanHeader h = *reinterpret_cast<const PlanHeader*>(a.plan);
    if (h.magic != kPlanMagic || h.bits != BITS || h.bytes != static_cast<int64_t>(a.plan_bytes)) {
        if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(a.status, 1);
        return;
    }
    const int t = *a.t;
    if (t < 1) {
        if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(a.status, 2);
        return;
    }
    const PlanTensor* tensors = reinterpret_cast<const PlanTensor*>(a.plan + sizeof(PlanHeader));
    const PlanChunk* chunks = reinterpret_cast<const PlanChunk*>(tensors + h.num);
    // 1 - beta^t without the cancellation at small t
    const float m1 = -1.f / expm1f(static_cast<float>(t) * a.log1);
    Rule rule{a.grad_scale ? *a.grad_scale : 1.f, a.beta1, a.rest1, BITS == 8 ? a.root_beta2 : a.beta2, a.rest2, 0.f,
              1.f / sqrtf(-expm1f(static_cast<float>(t) * a.log2)), a.eps, 0.f};
    __shared__ __align__(16) PlanTensor P;      // in registers its addresses would take a third of them
    // a CTA takes a chunk, or with 8-bit moments half of one: four elements a thread, and the next four on their way
    constexpr int kParts = BITS == 8 ? 2 : 1, kTaken = kChunk / kParts;
    const int64_t parts = h.chunks * kParts;
    PlanChunk next = blockIdx.x < parts ? chunks[blockIdx.x / kParts] : PlanChunk{0, 0};
    int mine = -1;
    bool loaded = false;
    Block8 x;
    for (int64_t c = blockIdx.x; c < parts; c += gridDim.x) {
        const PlanChunk pc = next;
        const int64_t c1 = c + gridDim.x;
        if (c1 < parts) next = chunks[c1 / kParts];
        if (pc.tensor != mine) {     // the same for the whole CTA, and mostly the one before
            mine = pc.tensor;
            __syncthreads();
            if (threadIdx.x < sizeof(PlanTensor) / 16)
                reinterpret_cast<uint4*>(&P)[threadIdx.x] = reinterpret_cast<const uint4*>(tensors + mine)[threadIdx.x];
            __syncthreads();
            const float lr = a.lr * P.t.lr_scale;
            rule.step = lr * m1;
            rule.decay = lr * P.t.weight_decay;
        }
        const int64_t base = static_cast<int64_t>(pc.chunk) * kChunk + c % kParts * kTaken, at = base + 4 * threadIdx.x;
        const bool full = P.vec && base + kTaken <= P.t.n;
        if constexpr (BITS == 32) {
            if (full)
                step_chunk32<true>(P.t, rule, at);
            else
                step_chunk32<false>(P.t, rule, at);
        } else {
            const int64_t first = P.first + base;
            const uint32_t key = mix(a.seed ^ (static_cast<uint32_t>(t) * 0x9e3779b1u));
            const uint32_t hi = static_cast<uint32_t>(first >> 32);
            const Draws d{static_cast<uint32_t>(first), mix(hi ^ key), mix((hi + 1) ^ key)};
            const uint32_t index = static_cast<uint32_t>(P.first + at);
            const int lane = threadIdx.x & 31;
            if (full) {
                if (!loaded) load_block8<true>(P.t, static_cast<uint32_t>(at), x);
                Block8 now = x;
                // the next chunk's elements come while these are worked on
                const int64_t nb = static_cast<int64_t>(next.chunk) * kChunk + c1 % kParts * kTaken;
                loaded = c1 < parts && next.tensor == mine && nb + kTaken <= P.t.n;
                if (loaded) load_block8<true>(P.t, static_cast<uint32_t>(nb) + 4 * threadIdx.x, x);
                step_block8<true>(P.t, rule, d, static_cast<uint32_t>(at), index, lane, now);
            } else {
                loaded = false;
                if (at - 4 * lane < P.t.n) {     // a block is there for the whole warp or for none of it
                    Block8 now;
                    load_block8<false>(P.t, at, now);
                    step_block8<false>(P.t, rule, d, at, index, lane, now);
                }
            }
        }
    }
}

bool tensor_ok(const dbw_adamw_tensor& t) {
    return t.n >= 0 && t.n <= (1ll << 40) && (t.g_type == DBW_F32 || t.g_type == DBW_BF16);
}
int64_t chunks_of(int64_t n) { return (n + kChunk - 1) / kChunk; }

}  // namespace

}  // namespace dbw

using namespace dbw;

extern "C" {

size_t dbw_adamw_plan_bytes(int num, const dbw_adamw_tensor* tensors) {
    if (num < 1 || !tensors) return 0;
    int64_t chunks = 0;
    for (int i = 0; i < num; ++i) {
        if (!tensor_ok(tensors[i])) return 0;
        chunks += chunks_of(tensors[i].n);
    }
    return (sizeof(PlanHeader) + sizeof(PlanTensor) * num + sizeof(PlanChunk) * chunks + 15) / 16 * 16;
}

int dbw_adamw_plan(int num, const dbw_adamw_tensor* tensors, int state_bits, void* plan, size_t plan_bytes) {
    clear_error();
    if (num < 1 || !tensors || !plan) return fail(DBW_EINVAL, "dbw_adamw_plan: no tensors, or a NULL pointer argument");
    if (state_bits != 32 && state_bits != 8) return fail(DBW_EINVAL, "dbw_adamw_plan: state_bits must be 32 or 8");
    const size_t need = dbw_adamw_plan_bytes(num, tensors);
    if (need == 0) return fail(DBW_EINVAL, "dbw_adamw_plan: a tensor's n or g_type is out of range");
    if (plan_bytes != need) return fail(DBW_EINVAL, "dbw_adamw_plan: plan must have %zu bytes, not %zu", need, plan_bytes);
    uint8_t* p = static_cast<uint8_t*>(plan);
    memset(p, 0, plan_bytes);
    PlanHeader h{kPlanMagic, static_cast<int64_t>(plan_bytes), 0, num, state_bits};
    size_t at = sizeof(PlanHeader) + sizeof(PlanTensor) * num;
    int64_t first = 0;
    for (int i = 0; i < num; ++i) {
        const dbw_adamw_tensor& t = tensors[i];
        const size_t ge = elem_bytes(t.g_type), se = state_bits == 8 ? 1 : 4;
        if (t.n > 0) {
            if (!t.g || !t.w || !t.w_out || !t.m || !t.v || !t.m_out || !t.v_out)
                return fail(DBW_EINVAL, "dbw_adamw_plan: tensor %d: NULL pointer", i);
            if (state_bits == 8 && (!t.m_scale || !t.v_scale || !t.m_scale_out || !t.v_scale_out))
                return fail(DBW_EINVAL, "dbw_adamw_plan: tensor %d: 8-bit moments need their scales", i);
            if (!aligned_to(t.g, ge) || !aligned_to(t.w, 4) || !aligned_to(t.w_out, 4) || !aligned_to(t.m, se) ||
                !aligned_to(t.v, se) || !aligned_to(t.m_out, se) || !aligned_to(t.v_out, se) ||
                !aligned_to(t.m_scale, 4) || !aligned_to(t.v_scale, 4) || !aligned_to(t.m_scale_out, 4) ||
                !aligned_to(t.v_scale_out, 4) || !aligned_to(t.w_bf16, 2))
                return fail(DBW_EALIGN, "dbw_adamw_plan: tensor %d: a pointer is not aligned to its elements", i);
        }
        PlanTensor q{t, first, 0, {0, 0, 0}};
        // (8 bits: and 32-bit indices)
        q.vec = (state_bits == 32 || t.n <= 0xffffffffll) && aligned_to(t.g, 4 * ge) && aligned_to(t.w, 16) &&
                aligned_to(t.w_out, 16) && aligned_to(t.m, 4 * se) && aligned_to(t.v, 4 * se) &&
                aligned_to(t.m_out, 4 * se) && aligned_to(t.v_out, 4 * se) && aligned_to(t.w_bf16, 8);
        memcpy(p + sizeof(PlanHeader) + sizeof(PlanTensor) * i, &q, sizeof(q));
        const int64_t c = chunks_of(t.n);
        for (int64_t k = 0; k < c; ++k, at += sizeof(PlanChunk)) {
            const PlanChunk pc{i, static_cast<int32_t>(k)};
            memcpy(p + at, &pc, sizeof(pc));
        }
        h.chunks += c;
        first += t.n;
    }
    memcpy(p, &h, sizeof(h));
    return DBW_OK;
}

int dbw_adamw_step(const void* plan, size_t plan_bytes, int state_bits, const int32_t* t, double lr, double beta1,
                   double beta2, double eps, const float* grad_scale, uint32_t seed, int* status, void* stream) {
    clear_error();
    Call call("dbw_adamw_step", as_stream(stream));
    if (!plan || !t || !status) return fail(DBW_EINVAL, "dbw_adamw_step: NULL pointer argument");
    if (state_bits != 32 && state_bits != 8) return fail(DBW_EINVAL, "dbw_adamw_step: state_bits must be 32 or 8");
    if (plan_bytes < sizeof(PlanHeader) + sizeof(PlanTensor))
        return fail(DBW_EINVAL, "dbw_adamw_step: plan_bytes is too small for a plan");
    if (!(lr >= 0.0)) return fail(DBW_EINVAL, "dbw_adamw_step: lr must be >= 0");
    if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0))
        return fail(DBW_EINVAL, "dbw_adamw_step: beta1 and beta2 must be in [0, 1)");
    if (!(eps >= 0.0)) return fail(DBW_EINVAL, "dbw_adamw_step: eps must be >= 0");
    if (!aligned16(plan)) return fail(DBW_EALIGN, "dbw_adamw_step: plan must be 16-byte aligned");
    if (!aligned_to(t, 4) || !aligned_to(grad_scale, 4) || !aligned_to(status, 4))
        return fail(DBW_EALIGN, "dbw_adamw_step: a pointer is not aligned to its elements");
    int rc = check_device();
    if (rc) return rc;
    StepArgs a{static_cast<const uint8_t*>(plan), plan_bytes, t, grad_scale, status,
               static_cast<float>(lr), static_cast<float>(beta1), static_cast<float>(beta2),
               static_cast<float>(1.0 - beta1), static_cast<float>(1.0 - beta2), static_cast<float>(eps),
               static_cast<float>(log(beta1)), static_cast<float>(log(beta2)), static_cast<float>(sqrt(beta2)), seed};
    // no more CTAs than the plan has room for chunks; the kernel reads how many there are
    const size_t room = (plan_bytes - sizeof(PlanHeader) - sizeof(PlanTensor)) / sizeof(PlanChunk);
    const size_t slots = state_bits == 8 ? static_cast<size_t>(kPerSm) * sm_count() : 0x7fffffff;
    const size_t grid = room < 1 ? 1 : room < slots ? room : slots;
    launch(state_bits == 8 ? adamw_kernel<8> : adamw_kernel<32>, static_cast<unsigned>(grid), kThreads, 0,
           as_stream(stream), a);
    const cudaError_t err = cudaGetLastError();
    if (err != cudaSuccess) return fail(DBW_ECUDA, "dbw_adamw_step: %s", cudaGetErrorString(err));
    return call.done(DBW_OK);
}

}  // extern "C"
