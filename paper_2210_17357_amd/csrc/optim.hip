// The optimizer step behind the exchange of gradients: squared norms of the layers' gradients, and AdamW over
// all layers with moments in fp32 or in 8 bits.  gfx950 / wave64.
//
// AdamW (Loshchilov, Hutter: decoupled weight decay), element by element, c the gradients' common factor:
//   g = c * grad;  m' = b1 m + (1 - b1) g;  v' = b2 v + (1 - b2) g^2
//   p' = p - lr wd p - (lr / (1 - b1^t)) m' / (sqrt(v') / sqrt(1 - b2^t) + eps)
// Every kernel streams: bound by HBM on large tables, by launches and a chain of a few memory accesses on small ones.
#include <cfloat>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <memory>
#include <new>

#include "internal.h"

namespace lgreco {
namespace {

constexpr int kOptimBlock = LGRECO_OPTIM_BLOCK;
// Elements of a workgroup of the norms, doubled while there would be more than kNormParts: enough workgroups to fill the chip
// more than once, few enough partial sums.  One layer, us with 16384 / 32768 / 65536 / 131072 / 262144: 355 M elements of fp32 223 / 220 / 217 /
// 225 / 222, of bf16 118 / 114 / 114 / 115 / 116; 67 M 49 / 46 / 44 / 43 / 49 and 27 / 27 / 26 / 25 / 31; 25.6 M 20 / 22 / 19 / 27 / 44
// and 13 / 14 / 13 / 18 / 28; 4.8 M 8.3 / 9.8 / 13 / 21 / 36 and 7.1 / 8.0 / 11 / 15 / 25.  (Smaller ones are not measured.)
constexpr int kNormPart = 16384, kNormParts = 6000;
constexpr int kStepPart = 4 * kThreads;        // elements of a workgroup of the step: one access a thread and buffer
// With 8-bit moments a thread takes 8 elements, and workgroups are half as large where short layers would leave more than a quarter
// of the larger ones idle (us a step, 256 threads / 128: 4000 layers of 200 elements 16.8 / 13.7, 6000 of 1400 38.4 / 36.4; 64 threads:
// 13.7, 37.  Long layers, a pass of 25 M elements 95.9 / 97.9, of 4.8 M 35.6 / 37.2).
constexpr int kCodedElems = 8;
constexpr int kShortParts = 65536;             // most workgroups of a step that works out its own factors
// Longer steps ask for LDS that they do not use, so that 3 workgroups (5 with 8-bit moments) share a compute unit and not 8: the
// chip's accesses then stay in a narrower window of memory.  355 M elements, us, with 8 / 6 / 5 / 4 / 3 / 2: fp32 moments
// 1730 / 1685 / 1650 / 1640 / 1615 / 1675, 8-bit ones 990 / 978 / 933 / 928 / 980 / 1258; 150 M 741 / 721 / 700 / 697 / 682 /
// 682 and 411 / 397 / 409 / 404 / 421 / 515.  Below 80 M elements it makes no difference.  These are workgroups of long layers, full
// ones.  The limit goes by their number alone, and costs where layers are short (us a step, with / without, fp32 moments and 8-bit ones): 70000
// layers of 400 elements 174 / 153 and 202 / 118, 40000 of 2100 399 / 419 and 302 / 275.
constexpr size_t kStepLds = 52 << 10, kCodedLds = 31 << 10;
constexpr int64_t kMaxParts = ((int64_t)1 << 32) / kThreads - 1;   // (a launch takes fewer than 2^32 threads)
constexpr int kLine = 32;            // elements of a 128-byte line of fp32

// What one workgroup of the norms adds up: consecutive elements of one layer, its layer's part `index` of `parts`.
struct NormPart {
    int64_t start;
    int32_t count, layer;
    int32_t index, parts;
    int32_t ticket;      // the layer's first ticket word, where it has more parts than one
    int32_t pad;
};

// What one workgroup of the step works on: consecutive elements of one layer.
struct StepPart {
    int64_t start;       // first element, into the flat buffers
    int32_t count;       // elements
    float lr_scale, decay_scale;
    int32_t pad;
};
struct CodedPart {       // the same with 8-bit moments
    int64_t start;
    int32_t count;
    float lr_scale, decay_scale;
    int32_t layer, pos;  // pos: first element, relative to the layer start
    int32_t block;       // its first block
};

// The step's factors that are the same for all elements, worked out on the device (the step count, the norm and the
// learning rate's factor lie there).
struct StepFactors {
    double lr;           // lr * *d_lr
    double lr_m;         // the same over 1 - b1^t
    float grad;          // factor of the gradients
    float root_v;        // 1 / sqrt(1 - b2^t)
    uint32_t t_lo, t_hi; // t
    int32_t go;          // 0: the step is left out
    int32_t pad;
};
constexpr int kFactorWords = sizeof(StepFactors) / 4;
constexpr double kMaxNorm = 0x1.6a09e667f3bcdp63;   // 2^63.5: squares up to half of what fp32 holds

typedef uint16_t u16x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(1)));
typedef uint16_t u16_any __attribute__((aligned(1)));
typedef uint32_t u32_any __attribute__((aligned(1)));

struct BF16 { uint16_t bits; };
struct F16 { uint16_t bits; };
struct NoCopy { };

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(BF16 x) { return __builtin_bit_cast(float, (uint32_t)x.bits << 16); }
__device__ __forceinline__ float widen(F16 x) { return (float)__builtin_bit_cast(_Float16, x.bits); }
__device__ __forceinline__ uint16_t narrow_bits(float x, BF16) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
__device__ __forceinline__ uint16_t narrow_bits(float x, F16) { return __builtin_bit_cast(uint16_t, (_Float16)x); }

__device__ __forceinline__ void load4(const float* p, float* x) {
    const float4 v = load_stream(p);
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
}
template <typename G>
__device__ __forceinline__ void load4(const G* p, float* x) {
    const u16x4_any v = __builtin_nontemporal_load(reinterpret_cast<const u16x4_any*>(p));
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = widen(G{v[j]});
}
// one 16-byte access
__device__ __forceinline__ void load16(const float* p, float (&x)[4]) { load4(p, x); }
template <typename G>
__device__ __forceinline__ void load16(const G* p, float (&x)[8]) {
    const u32x4_any v = __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(p));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = widen(G{(uint16_t)v[j]});
        x[2 * j + 1] = widen(G{(uint16_t)(v[j] >> 16)});
    }
}
template <typename C>
__device__ __forceinline__ void store16(C* p, const float (&x)[8]) {
    u32x4_any n;
#pragma unroll
    for (int j = 0; j < 4; ++j) n[j] = (uint32_t)narrow_bits(x[2 * j], C{}) | (uint32_t)narrow_bits(x[2 * j + 1], C{}) << 16;
    __builtin_nontemporal_store(n, reinterpret_cast<u32x4_any*>(p));
}
__device__ __forceinline__ void load_run(const uint8_t* p, uint32_t (&c)[2]) {
    const u32x2_any v = *reinterpret_cast<const u32x2_any*>(p);
    c[0] = v.x;
    c[1] = v.y;
}
template <typename C>
__device__ __forceinline__ void store4(C* p, const float* x) {
    u16x4_any n;
#pragma unroll
    for (int j = 0; j < 4; ++j) n[j] = narrow_bits(x[j], C{});
    __builtin_nontemporal_store(n, reinterpret_cast<u16x4_any*>(p));
}
__device__ __forceinline__ void store4(float* p, const float* x) { store_stream(p, make_float4(x[0], x[1], x[2], x[3])); }
__device__ __forceinline__ void store4(NoCopy*, const float*) {}
template <typename C>
__device__ __forceinline__ C* shifted(C* p, int64_t n) { return p + n; }
__device__ __forceinline__ NoCopy* shifted(NoCopy* p, int64_t) { return p; }

// The 8 elements of a block that one lane of a row of 16 takes: 4 from 4 * lane on and 4 from 64 + 4 * lane on, so that
// every access of a row is whole lines.
constexpr int kHalf = kOptimBlock / 2;
__device__ __forceinline__ int place(int j) { return j < 4 ? j : kHalf - 4 + j; }
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
    load4(p, x);
    load4(p + kHalf, x + 4);
}
__device__ __forceinline__ void load8(const uint8_t* p, uint32_t (&c)[2]) {
    c[0] = *reinterpret_cast<const u32_any*>(p);
    c[1] = *reinterpret_cast<const u32_any*>(p + kHalf);
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
    store4(p, x);
    store4(shifted(p, kHalf), x + 4);
}
__device__ __forceinline__ void store8(uint8_t* p, const uint32_t (&c)[2]) {
    *reinterpret_cast<u32_any*>(p) = c[0];
    *reinterpret_cast<u32_any*>(p + kHalf) = c[1];
}
template <typename C>
__device__ __forceinline__ void store1(C* p, float v) { p->bits = narrow_bits(v, C{}); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(NoCopy*, float) {}

// ------------------------------------------------------------------ the last workgroup
// Whether the caller is the last of n that ask, the i-th one: a ticket among 64 neighbours or more, then one of their at most 256
// groups, so that no word of memory takes many at a time (one word for 4000 workgroups: 30 us where these take 12).  The
// last ones clear the words for the next launch.
// Tickets order nothing by themselves: an ordered one writes back and drops the L2 caches, which took the norms of 355 M
// elements from 212 to 360 us.  What the last one reads is published by an exchange, which is performed where all caches
// meet before it returns, and read by loads of the same scope.
constexpr uint32_t kTicketGroup = 64, kTicketGroups = 256;
constexpr int kTicketLine = 32;                                // words apart
__host__ __device__ inline uint32_t ticket_group(uint32_t n) {
    const uint32_t even = (n + kTicketGroups - 1) / kTicketGroups;
    return even > kTicketGroup ? even : kTicketGroup;
}
__host__ __device__ inline uint32_t ticket_lines(uint32_t n) { return n <= kTicketGroup ? 1 : 1 + (n + ticket_group(n) - 1) / ticket_group(n); }
__device__ __forceinline__ bool last_drawn(uint32_t* word, uint32_t n) {
    if (__hip_atomic_fetch_add(word, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != n - 1) return false;
    __hip_atomic_store(word, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return true;
}
__device__ __forceinline__ bool last_of(uint32_t* tickets, uint32_t i, uint32_t n) {
    if (n <= kTicketGroup) return last_drawn(tickets, n);
    const uint32_t size = ticket_group(n), group = i / size, groups = (n + size - 1) / size;
    return last_drawn(tickets + kTicketLine * (1 + group), min(size, n - group * size)) && last_drawn(tickets, groups);
}
__device__ __forceinline__ void publish(double* p, double x) {
    uint64_t old = __hip_atomic_exchange(reinterpret_cast<uint64_t*>(p), __builtin_bit_cast(uint64_t, x), __ATOMIC_RELAXED,
                                         __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("" : "+v"(old) : : "memory");               // (it has returned before anything that follows)
}
__device__ __forceinline__ double published(const double* p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// ------------------------------------------------------------------ norms
struct NormParams {
    const NormPart* parts;
    const void* grads;
    double* partials;
    double* sumsq;             // [L + 1]
    int32_t L;
    uint32_t* tickets;         // of the layers; then the layers' own, of their parts
};

__device__ __forceinline__ double sum_of_waves(double a, double* s_sum) {
    const double w = wave_sum(a);
    if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = w;
    __syncthreads();
    return (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
}
// Sum of n published numbers in an order that depends on n alone.
__device__ __forceinline__ double sum_published(const double* p, int n, double* s_sum) {
    double a = 0.0;
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += kThreads) a += published(p + i);
    return sum_of_waves(a, s_sum);
}

// Bound by HBM: 355 M elements of fp32 in 217 us (6.5 TB/s), of bf16 in 114-119 (6.0-6.2).  The last workgroup of a layer adds up the layer's partial sums, the last of those the layers' sums.
template <typename G>
__global__ __launch_bounds__(kThreads) void norms_kernel(NormParams k) {
    __shared__ double s_sum[3][kThreads / 64];
    __shared__ int s_last[2];
    const NormPart t = k.parts[blockIdx.x];
    const G* const g = static_cast<const G*>(k.grads) + t.start;
    const int tid = threadIdx.x;
    // four accesses of a thread in flight; past the end a thread reads the last whole access again and adds nothing
    constexpr int kWide = 16 / sizeof(G), kAhead = 4, kRound = kWide * kThreads;
    double a[4] = {0.0, 0.0, 0.0, 0.0};
    const int last = t.count - kWide;
    const auto batch = [&](int first, bool whole) __attribute__((always_inline)) {
        float x[kAhead][kWide];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int i = first + u * kRound + kWide * tid;
            load16(g + (whole ? i : min(i, last)), x[u]);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (!whole && first + u * kRound + kWide * tid > last) continue;
#pragma unroll
            for (int j = 0; j < kWide; ++j) a[j & 3] = __builtin_fma((double)x[u][j], (double)x[u][j], a[j & 3]);
        }
    };
    int first = 0;
    for (; first + kAhead * kRound <= t.count; first += kAhead * kRound) batch(first, true);
    if (first <= last) batch(first, false);
    if (tid < t.count % kWide) {
        const double x = (double)widen(g[t.count / kWide * kWide + tid]);
        a[0] = __builtin_fma(x, x, a[0]);
    }
    double sum = sum_of_waves((a[0] + a[1]) + (a[2] + a[3]), s_sum[0]);
    if (t.parts > 1) {
        if (tid == 0) {
            publish(k.partials + blockIdx.x, sum);
            s_last[0] = last_of(k.tickets + t.ticket, t.index, t.parts);
        }
        __syncthreads();
        if (!s_last[0]) return;
        sum = sum_published(k.partials + (blockIdx.x - t.index), t.parts, s_sum[1]);
    }
    if (tid == 0) {
        publish(k.sumsq + t.layer, sum);
        s_last[1] = last_of(k.tickets, t.layer, k.L);
    }
    __syncthreads();
    if (!s_last[1]) return;
    sum = sum_published(k.sumsq, k.L, s_sum[2]);
    if (tid == 0) k.sumsq[k.L] = sum;
}

// ------------------------------------------------------------------ the step's factors
struct FactorParams {
    double lr, beta1, beta2, grad_scale, max_norm;
    const double* total;     // sum of the squared gradients, or null
    const float* lr_factor;  // or null
    int64_t* step;
};

__device__ __forceinline__ StepFactors factors_of(const FactorParams& p) {
    // (all three on their way before one is used)
    const double s = p.total ? *p.total : 0.0;
    const float lr_factor = p.lr_factor ? *p.lr_factor : 1.0f;
    const uint64_t t = (uint64_t)(*p.step + 1);
    StepFactors f{};
    double c = p.grad_scale;
    const double norm = sqrt(s);
    if (p.max_norm > 0.0) c *= fmin(1.0, p.max_norm / (p.grad_scale * norm + 1e-6));
    // neither NaN nor infinite, and no square of a scaled gradient beyond fp32: one would make its v infinite for good, and
    // with it the exponent of its block; a factor below the normal numbers would round the gradients to a few bits or to 0
    f.go = s <= DBL_MAX && c * norm <= kMaxNorm && c >= FLT_MIN;
    // b^t by squaring: its relative error is some t 2^-53, and b^t is 0 long before that matters
    double power1 = 1.0, power2 = 1.0, b1 = p.beta1, b2 = p.beta2;
    for (uint64_t n = t; n; n >>= 1) {
        if (n & 1) {
            power1 *= b1;
            power2 *= b2;
        }
        b1 *= b1;
        b2 *= b2;
    }
    f.lr = p.lr * (double)lr_factor;
    f.lr_m = f.lr / (1.0 - power1);
    f.root_v = (float)(1.0 / sqrt(1.0 - power2));
    f.grad = (float)c;
    f.t_lo = (uint32_t)t;
    f.t_hi = (uint32_t)(t >> 32);
    return f;
}

__global__ __launch_bounds__(64) void factors_kernel(FactorParams p, StepFactors* out) {
    if (threadIdx.x != 0) return;
    const StepFactors f = factors_of(p);
    *out = f;
    if (f.go) *p.step = (int64_t)((uint64_t)f.t_hi << 32 | f.t_lo);
}

// ------------------------------------------------------------------ AdamW
struct StepParams {
    const void* parts;             // StepPart or CodedPart
    const StepFactors* factors;    // null: the workgroups work them out themselves
    FactorParams raw;
    uint32_t* tickets;
    const void* grads;
    float* p;
    void* m;
    void* v;
    uint8_t* exps;
    void* copy;
    double weight_decay;
    float beta1, rest1, beta2, rest2, eps;     // rest = 1 - beta
    int32_t stochastic;
    uint32_t seed_lo, seed_hi;
};

// The step's factors: from the kernel in front, or, where the table is short and a kernel in front would take as long as the
// step, worked out by every workgroup's first wavefront while its data is on the way.  Then the last workgroup to finish
// counts the step: every other one has read the count by then, with its first wavefront, which also draws its ticket.
__device__ __forceinline__ StepFactors step_factors(const StepParams& k) {
    if (k.factors) return *k.factors;
    __shared__ uint32_t s_words[kFactorWords];
    if (threadIdx.x < 64) {
        const StepFactors f = factors_of(k.raw);
        uint32_t w[kFactorWords];
        __builtin_memcpy(w, &f, sizeof(f));
        if (threadIdx.x == 0) {
#pragma unroll
            for (int i = 0; i < kFactorWords; ++i) s_words[i] = w[i];
        }
    }
    __syncthreads();
    uint32_t w[kFactorWords];
#pragma unroll
    for (int i = 0; i < kFactorWords; ++i) w[i] = (uint32_t)__builtin_amdgcn_readfirstlane((int)s_words[i]);
    StepFactors f;
    __builtin_memcpy(&f, w, sizeof(f));
    return f;
}
__device__ __forceinline__ void count_step(const StepParams& k, const StepFactors& f) {
    if (!k.factors && threadIdx.x == 0 && last_of(k.tickets, blockIdx.x, gridDim.x)) *k.raw.step = (int64_t)((uint64_t)f.t_hi << 32 | f.t_lo);
}

// Long steps walk their table from its end: the gradients that the norms have read last lie in the cache in front of the memory
// (256 MB), and the codes that are written last are the ones whose values are read first.  A pass over 355 M elements: norms, 8-bit
// step and values 1452 -> 1418 us, norms and step with fp32 moments 1873 -> 1868.
__device__ __forceinline__ uint32_t part_of(const StepParams& k) { return k.factors ? gridDim.x - 1 - blockIdx.x : blockIdx.x; }

// The factors of one layer's elements.
struct Rates {
    float shrink;        // lr wd
    float rate;          // lr / (1 - b1^t)
    float grad, root_v;
    float root_low;      // root_v behind the root of a v scaled by 2^64
};
template <typename P>
__device__ __forceinline__ Rates rates_of(const StepFactors& f, const StepParams& p, const P& t) {
    const double s = (double)t.lr_scale;
    return Rates{(float)(f.lr * s * (p.weight_decay * (double)t.decay_scale)), (float)(f.lr_m * s), f.grad, f.root_v, f.root_v * 0x1p-32f};
}

// The moments' products and sums are rounded one by one, so that they, and the codes made of them, are what any other fp32
// program finds (a fused product moves one code in some ten million to its neighbour).
// The root and the reciprocal are the instructions' (one unit in the last place), which take 8 cycles where the correctly
// rounded ones take some 50.  The root's takes numbers below 2^-126 for 0: such a v is scaled by 2^64 under it, exactly.  The
// reciprocal's gives 0 for numbers beyond 2^126: no eps is larger, and no root (2^64, its factor 2^27 at most) comes near.
__device__ __forceinline__ void step_one(const StepParams& k, const Rates& r, float grad, float& p, float& m, float& v) {
    const float g = r.grad * grad;
    m = k.beta1 * m + k.rest1 * g;
    v = k.beta2 * v + k.rest2 * (g * g);
    const bool low = v < FLT_MIN;
    const float root = __builtin_amdgcn_sqrtf(low ? v * 0x1p64f : v);
    const float u = m * __builtin_amdgcn_rcpf(__builtin_fmaf(root, low ? r.root_low : r.root_v, k.eps));
    p -= __builtin_fmaf(r.shrink, p, r.rate * u);
}

// Bound by HBM, four streams in and three or four out.  A thread takes 4 elements and is done: 355 M elements in 1635 us
// (28 bytes each: 6.1 TB/s).  With 8 workgroups a compute unit 1725, then 1810 with two rounds a workgroup, 1870 with eight, 1830 with
// both rounds' loads ahead, 1955 without the streaming hints.
template <typename G, typename C>
__global__ __launch_bounds__(kThreads) void adamw_kernel(StepParams k) {
    const StepPart t = static_cast<const StepPart*>(k.parts)[part_of(k)];
    const int i = 4 * threadIdx.x, left = t.count - i;
    const G* const g = static_cast<const G*>(k.grads) + t.start + i;
    float* const p = k.p + t.start + i;
    float* const m = static_cast<float*>(k.m) + t.start + i;
    float* const v = static_cast<float*>(k.v) + t.start + i;
    C* const copy = shifted(static_cast<C*>(k.copy), t.start + i);
    float gi[4]{}, pi[4]{}, mi[4]{}, vi[4]{};
    if (left >= 4) {
        load4(g, gi);
        load4(p, pi);
        load4(m, mi);
        load4(v, vi);
    } else if (left > 0) {                                   // (the layer's last elements; what is read twice is stored once)
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            const int at = min(j, left - 1);
            gi[j] = widen(g[at]);
            pi[j] = p[at];
            mi[j] = m[at];
            vi[j] = v[at];
        }
    }
    const StepFactors f = step_factors(k);
    if (!f.go) return;
    const Rates r = rates_of(f, k, t);
#pragma unroll
    for (int j = 0; j < 4; ++j) step_one(k, r, gi[j], pi[j], mi[j], vi[j]);
    if (left >= 4) {
        store4(p, pi);
        store4(m, mi);
        store4(v, vi);
        store4(copy, pi);
    } else {
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            if (j < left) {
                p[j] = pi[j];
                m[j] = mi[j];
                v[j] = vi[j];
                store1(shifted(copy, j), pi[j]);
            }
        }
    }
    count_step(k, f);
}

// ------------------------------------------------------------------ 8-bit moments
// A magnitude a of a block whose exponent byte is x is held as the bits 19.. of the fp32 number a 2^(top - x), top = 7 for m and
// 15 for v: exponent field and 4 bits of mantissa in one small whole number, denormal numbers as the evenly spaced
// codes below the lowest octave.
constexpr int kTopM = 7, kTopV = 15, kCodeShift = 19;

__device__ __forceinline__ float decoded_m(uint32_t code, int x) {
    return __builtin_ldexpf(__builtin_bit_cast(float, (code & 127u) << kCodeShift | (code & 128u) << 24), x - kTopM);
}
__device__ __forceinline__ float decoded_v(uint32_t code, int x) {
    return __builtin_ldexpf(__builtin_bit_cast(float, code << kCodeShift), x - kTopV);
}

// The exponent byte of a block whose largest magnitude has these bits: its exponent, one more where rounding to 4 bits of
// mantissa could carry into the next octave.
__device__ __forceinline__ int block_exponent(uint32_t bits) { return (int)((bits + ((1u << kCodeShift) - 1)) >> 23); }

// A magnitude on its way to a code: the code is bits 19.. of the sum, up to 7 or 8 of them.  r: 16 random bits from bit 3 on.  (A
// number that is not finite leaves the field; its own byte alone takes what comes.)
// Below the lowest octave the scaled number is denormal and has been rounded: it is taken down again where that went up, and its
// last bit set where anything was lost, so that ties are ties and the sum carries only where the exact one does.
// (Random bits end above the last one, which they need not see.)
template <bool STOCHASTIC>
__device__ __forceinline__ uint32_t encoded(float a, int shift, uint32_t r) {
    const float scaled = __builtin_ldexpf(a, shift), back = __builtin_ldexpf(scaled, -shift);
    uint32_t b = __builtin_bit_cast(uint32_t, scaled) - (back > a ? 1u : 0u);
    if (STOCHASTIC) return b + ((r & 0x7FFF8u) | 4u);
    b |= back != a ? 1u : 0u;
    return b + ((1u << (kCodeShift - 1)) - 1) + (b >> kCodeShift & 1u);
}

// Byte 3 of four words as one word.
__device__ __forceinline__ uint32_t top_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0C0C0703u), __builtin_amdgcn_perm(b, a, 0x0C0C0703u), 0x05040100u);
}

// max(|a|, |b|, c): magnitudes of results of arithmetic
__device__ __forceinline__ float max3_abs(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, |%1|, |%2|, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// The values of 8 codes (two words of four bytes).
__device__ __forceinline__ void decode8(const uint32_t (&cm)[2], const uint32_t (&cv)[2], int xm, int xv, float (&m)[8], float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        m[j] = decoded_m(cm[j >> 2] >> 8 * (j & 3) & 255u, xm);
        v[j] = decoded_v(cv[j >> 2] >> 8 * (j & 3) & 255u, xv);
    }
}

// Bound by HBM: 355 M elements with bf16 gradients and copy, stochastic, in 936 us (16 bytes each: 6.1 TB/s); rounding to nearest
// takes as long.  A row of 16 lanes takes a block, so that its maxima take four vector instructions each and no LDS.  (Lanes with 8
// consecutive elements, whose fp32 accesses are half lines: 1100; the codes' accesses with streaming hints: 1 to 3 % more.)
template <typename G, typename C, bool STOCHASTIC>
__global__ __launch_bounds__(kThreads) void adamw_coded_kernel(StepParams k) {
    const CodedPart t = static_cast<const CodedPart*>(k.parts)[part_of(k)];
    const int lane = threadIdx.x & 15, i = threadIdx.x / 16 * kOptimBlock + 4 * lane, left = t.count - i;
    const bool whole = i - 4 * lane + kOptimBlock <= t.count;
    const G* const g = static_cast<const G*>(k.grads) + t.start + i;
    float* const p = k.p + t.start + i;
    uint8_t* const m = static_cast<uint8_t*>(k.m) + t.start + i;
    uint8_t* const v = static_cast<uint8_t*>(k.v) + t.start + i;
    C* const copy = shifted(static_cast<C*>(k.copy), t.start + i);
    uint8_t* const exps = k.exps + 2 * (int64_t)(t.block + i / kOptimBlock);

    float gi[8]{}, pi[8]{}, mi[8], vi[8];
    uint32_t cm[2] = {0, 0}, cv[2] = {0, 0}, x = 0;          // (x: both exponents, taken apart when everything is on its way)
    const bool some = (int)(threadIdx.x & ~63u) * 8 < t.count;     // whether the wavefront has elements
    if (whole) {
        x = *reinterpret_cast<const u16_any*>(exps);
        load8(g, gi);
        load8(p, pi);
        load8(m, cm);
        load8(v, cv);
    } else if (some) {
        // a short block, and lanes behind the last one: everything is asked for at once, the part's last element in place of what is
        // not there
        const int last = left - 1;
        uint32_t em[8], ev[8];
        x = *reinterpret_cast<const u16_any*>(k.exps + 2 * (int64_t)(t.block + min(i, t.count - 1) / kOptimBlock));
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int at = min(place(j), last);
            gi[j] = widen(g[at]);
            pi[j] = p[at];
            em[j] = m[at];
            ev[j] = v[at];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool in = place(j) <= last;
            gi[j] = in ? gi[j] : 0.0f;
            cm[j >> 2] |= in ? em[j] << 8 * (j & 3) : 0u;
            cv[j >> 2] |= in ? ev[j] << 8 * (j & 3) : 0u;
        }
    }
    const StepFactors f = step_factors(k);
    if (!f.go || !some) return;                              // (the first wavefront, which counts, has elements)
    const Rates r = rates_of(f, k, t);
    // (elements past the layer's end: gradient 0 and codes 0, so their moments are 0)
    decode8(cm, cv, (int)(x & 255u), (int)(x >> 8), mi, vi);
    float top_m = 0.0f, top_v = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) step_one(k, r, gi[j], pi[j], mi[j], vi[j]);
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
        top_m = max3_abs(mi[j], mi[j + 1], top_m);
        top_v = max3f(vi[j], vi[j + 1], top_v);
    }
    const int xm = block_exponent(__builtin_bit_cast(uint32_t, row16_max(top_m)));
    const int xv = block_exponent(__builtin_bit_cast(uint32_t, row16_max(top_v)));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        Philox4 words{};
        if (STOCHASTIC)
            words = philox4x32_10((uint32_t)(t.pos + i) / 4 + h * (kHalf / 4), f.t_lo, (uint32_t)t.layer, 1u + f.t_hi, k.seed_lo, k.seed_hi);
        uint32_t em[4], ev[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float mj = mi[4 * h + q], vj = vi[4 * h + q];
            const uint32_t a = encoded<STOCHASTIC>(__builtin_fabsf(mj), kTopM - xm, words.w[q] << 3);
            const uint32_t b = max(encoded<STOCHASTIC>(vj, kTopV - xv, words.w[q] >> 13), vj > 0.0f ? 1u << kCodeShift : 0u);
            em[q] = (a << 5 & 0x7FFFFFFFu) | (__builtin_bit_cast(uint32_t, mj) & 0x80000000u);
            ev[q] = b << 5;
        }
        cm[h] = top_bytes(em[0], em[1], em[2], em[3]);
        cv[h] = top_bytes(ev[0], ev[1], ev[2], ev[3]);
    }
    if (left <= 0) return;
    if (lane == 0) {
        *reinterpret_cast<u16_any*>(exps) = (uint16_t)(xm | xv << 8);
    }
    if (whole) {
        store8(m, cm);
        store8(v, cv);
        store8(p, pi);
        store8(copy, pi);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (place(j) < left) {
                p[place(j)] = pi[j];
                m[place(j)] = (uint8_t)(cm[j >> 2] >> 8 * (j & 3));
                v[place(j)] = (uint8_t)(cv[j >> 2] >> 8 * (j & 3));
                store1(shifted(copy, place(j)), pi[j]);
            }
        }
    }
    count_step(k, f);
}

// Bound by HBM.  A row of 16 lanes takes a block; for 16-bit values a lane takes 8 consecutive elements, one access of each
// buffer (355 M elements: 361 us, 5.9 TB/s, 390 in the places of fp32; fp32 values 568 us, 6.2 TB/s).
template <typename O>
__global__ __launch_bounds__(kThreads) void moments_kernel(const CodedPart* __restrict__ parts, const uint8_t* __restrict__ codes_m,
                                                           const uint8_t* __restrict__ codes_v, const uint8_t* __restrict__ exps,
                                                           O* __restrict__ m_out, O* __restrict__ v_out) {
    constexpr bool kRun = sizeof(O) == 2;
    const CodedPart t = parts[blockIdx.x];
    const int lane = threadIdx.x & 15, first = threadIdx.x / 16 * kOptimBlock;
    const int i = first + (kRun ? 8 : 4) * lane, left = t.count - i;
    if (left <= 0) return;
    const uint8_t* const m = codes_m + t.start + i;
    const uint8_t* const v = codes_v + t.start + i;
    const uint8_t* const x = exps + 2 * (int64_t)(t.block + first / kOptimBlock);
    O* const mo = m_out + t.start + i;
    O* const vo = v_out + t.start + i;
    const uint32_t both = *reinterpret_cast<const u16_any*>(x);
    if (first + kOptimBlock <= t.count) {
        uint32_t cm[2], cv[2];
        float fm[8], fv[8];
        if constexpr (kRun) {
            load_run(m, cm);
            load_run(v, cv);
        } else {
            load8(m, cm);
            load8(v, cv);
        }
        decode8(cm, cv, (int)(both & 255u), (int)(both >> 8), fm, fv);
        if constexpr (kRun) {
            store16(mo, fm);
            store16(vo, fv);
        } else {
            store8(mo, fm);
            store8(vo, fv);
        }
    } else {
        uint32_t cm[8], cv[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int at = min(kRun ? j : place(j), left - 1);
            cm[j] = m[at];
            cv[j] = v[at];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int at = kRun ? j : place(j);
            if (at < left) {
                store1(mo + at, decoded_m(cm[j], (int)(both & 255u)));
                store1(vo + at, decoded_v(cv[j], (int)(both >> 8)));
            }
        }
    }
}

// A launch's own error, whatever another call on this thread left behind.
template <typename... A>
hipError_t launch(void (*kernel)(A...), int64_t grid, int threads, size_t lds, hipStream_t s, A... args) {
    void* list[] = {&args...};
    return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3((unsigned)grid), dim3(threads), list, lds, s);
}

size_t element_size(int32_t type) { return type == LGRECO_F32 ? 4 : 2; }
bool gradient_type(int32_t type) { return type == LGRECO_F32 || type == LGRECO_BF16 || type == LGRECO_F16; }
bool misaligned(const void* p, size_t n) { return (uintptr_t)p % n != 0; }

}  // namespace
}  // namespace lgreco

using namespace lgreco;

struct lgreco_optim {
    int device = 0;
    int32_t L = 0;
    int64_t blocks = 0;
    int64_t n_norm = 0, n_step = 0, n_coded = 0;   // parts of the three cuts of the table
    int32_t coded_threads = kThreads;              // of the workgroups with 8-bit moments
    uint8_t* d_all = nullptr;                      // one allocation, of
    NormPart* d_norm = nullptr;
    StepPart* d_step = nullptr;                    // cut on whole lines of the flat buffers
    CodedPart* d_coded = nullptr;                  // cut on the layers' blocks
    double* d_partials = nullptr;                  // [n_norm]
    StepFactors* d_factors = nullptr;
    uint32_t* d_tickets = nullptr;                 // of the step; zero between launches, like
    uint32_t* d_norm_tickets = nullptr;            // those of the norms
    char error[256] = "";
};

namespace {

// Text of the HIP error that ended this thread's last creation of a plan, which leaves no plan to ask ("": none did).
thread_local char create_error[sizeof(lgreco_optim::error)] = "";

int hip_fail(lgreco_optim* o, hipError_t e, const char* what) {
    std::snprintf(o->error, sizeof(o->error), "%s: %s", what, hipGetErrorString(e));
    return LGRECO_EHIP;
}
#define HIPCHK(expr)                                             \
    do {                                                         \
        hipError_t _e = (expr);                                  \
        if (_e != hipSuccess) return hip_fail(o, _e, #expr);     \
    } while (0)

// Calls f(first element, the same from the layer's start, elements) for the parts of one layer: `part` elements each, the first one
// cut short so that the others start at a multiple of `line` elements of the flat buffers (1: wherever the layer starts).
template <typename F>
void for_parts(const lgreco_layer_t& a, int64_t part, int64_t line, F f) {
    for (int64_t pos = 0; pos < a.numel;) {
        const int64_t start = a.offset + pos, n = std::min(a.numel - pos, part - start % line);
        f(start, pos, n);
        pos += n;
    }
}

int64_t count_parts(const lgreco_layer_t& a, int64_t part, int64_t line) {
    const int64_t head = part - a.offset % line;
    return a.numel <= head ? 1 : 1 + (a.numel - head + part - 1) / part;
}

int create(lgreco_optim* o, const lgreco_layer_t* layers, int32_t L, const float* lr_scale, const float* decay_scale) {
    const int st = check_layers(layers, L);
    if (st != LGRECO_OK) return st;
    int64_t total = 0;
    for (int32_t l = 0; l < L; ++l) total += layers[l].numel;
    int64_t norm_part = kNormPart;
    while (total / norm_part > kNormParts) norm_part *= 2;
    size_t norm_words = (size_t)kTicketLine * ticket_lines((uint32_t)L);
    for (int32_t l = 0; l < L; ++l) {
        const lgreco_layer_t& a = layers[l];
        if (a.offset > ((int64_t)1 << 58)) return LGRECO_EINVAL;            // (in bytes, beyond any address)
        for (const float* f : {lr_scale, decay_scale})
            if (f && !(f[l] >= 0.0f && f[l] <= FLT_MAX)) return LGRECO_EINVAL;
        const int64_t parts = count_parts(a, norm_part, kLine);
        if (parts > 1) norm_words += (size_t)kTicketLine * ticket_lines((uint32_t)parts);
        o->n_norm += parts;
        o->n_step += count_parts(a, kStepPart, kLine);
        o->n_coded += count_parts(a, kCodedElems * kThreads, 1);
    }
    if (o->n_step > kMaxParts) return LGRECO_ENOSPACE;                      // (the finest of the cuts)
    if (4 * total < 3 * o->n_coded * kCodedElems * kThreads) {
        o->coded_threads = kThreads / 2;
        o->n_coded = 0;
        for (int32_t l = 0; l < L; ++l) o->n_coded += count_parts(layers[l], kCodedElems * o->coded_threads, 1);
    }
    o->L = L;
    HIPCHK(hipGetDevice(&o->device));

    // one allocation: first what the host writes (the tickets as zeros), then the scratch
    size_t bytes = 0;
    const auto room = [&](size_t n) {
        const size_t at = bytes;
        bytes += (n + 127) / 128 * 128;
        return at;
    };
    const size_t norm_at = room(sizeof(NormPart) * o->n_norm), step_at = room(sizeof(StepPart) * o->n_step),
                 coded_at = room(sizeof(CodedPart) * o->n_coded), tickets_at = room(4 * (size_t)kTicketLine * (1 + kTicketGroups)),
                 norm_tickets_at = room(4 * norm_words), written = bytes;
    const size_t partials_at = room(sizeof(double) * o->n_norm), factors_at = room(sizeof(StepFactors));
    const std::unique_ptr<uint8_t[]> host(new uint8_t[written]);
    std::memset(&host[tickets_at], 0, written - tickets_at);
    NormPart* norm = reinterpret_cast<NormPart*>(&host[norm_at]);
    StepPart* step = reinterpret_cast<StepPart*>(&host[step_at]);
    CodedPart* coded = reinterpret_cast<CodedPart*>(&host[coded_at]);
    size_t word = (size_t)kTicketLine * ticket_lines((uint32_t)L);
    for (int32_t l = 0; l < L; ++l) {
        const float ls = lr_scale ? lr_scale[l] : 1.0f, ds = decay_scale ? decay_scale[l] : 1.0f;
        const int32_t parts = (int32_t)count_parts(layers[l], norm_part, kLine);
        int32_t index = 0;
        for_parts(layers[l], norm_part, kLine, [&](int64_t start, int64_t, int64_t n) {
            *norm++ = NormPart{start, (int32_t)n, l, index++, parts, (int32_t)word, 0};
        });
        if (parts > 1) word += (size_t)kTicketLine * ticket_lines((uint32_t)parts);
        for_parts(layers[l], kStepPart, kLine, [&](int64_t start, int64_t, int64_t n) { *step++ = StepPart{start, (int32_t)n, ls, ds, 0}; });
        for_parts(layers[l], kCodedElems * o->coded_threads, 1, [&](int64_t start, int64_t pos, int64_t n) {
            *coded++ = CodedPart{start, (int32_t)n, ls, ds, l, (int32_t)pos, (int32_t)(o->blocks + pos / kOptimBlock)};
        });
        o->blocks += (layers[l].numel + kOptimBlock - 1) / kOptimBlock;
    }
    HIPCHK(hipMalloc(reinterpret_cast<void**>(&o->d_all), bytes));
    HIPCHK(hipMemcpy(o->d_all, host.get(), written, hipMemcpyHostToDevice));
    o->d_norm = reinterpret_cast<NormPart*>(o->d_all + norm_at);
    o->d_step = reinterpret_cast<StepPart*>(o->d_all + step_at);
    o->d_coded = reinterpret_cast<CodedPart*>(o->d_all + coded_at);
    o->d_tickets = reinterpret_cast<uint32_t*>(o->d_all + tickets_at);
    o->d_norm_tickets = reinterpret_cast<uint32_t*>(o->d_all + norm_tickets_at);
    o->d_partials = reinterpret_cast<double*>(o->d_all + partials_at);
    o->d_factors = reinterpret_cast<StepFactors*>(o->d_all + factors_at);
    return LGRECO_OK;
}

int on_device(lgreco_optim* o) {
    int d = -1;
    HIPCHK(hipGetDevice(&d));
    return d == o->device ? LGRECO_OK : LGRECO_EINVAL;
}

bool valid(const lgreco_adamw_t* c) {
    const auto finite_from = [](double x, double least) { return x >= least && x <= DBL_MAX; };
    return finite_from(c->lr, 0.0) && c->beta1 >= 0.0 && c->beta1 < 1.0 && c->beta2 >= 0.0 && c->beta2 < 1.0 &&
           c->eps <= 0x1p126 && (float)c->eps >= FLT_MIN && finite_from(c->weight_decay, 0.0) && c->grad_scale >= FLT_MIN &&
           c->grad_scale <= FLT_MAX && finite_from(c->max_norm, 0.0) && (c->stochastic == 0 || c->stochastic == 1) && c->reserved == 0;
}

// What both forms of the step check and queue in front of their kernel.
int begin_step(lgreco_optim* o, const lgreco_adamw_t* c, const void* grads, int32_t grad_type, float* params, const void* m,
               const void* v, size_t moment_size, const void* copy, int32_t copy_type, const double* sumsq, const float* lr,
               int64_t* step, hipStream_t s, const void* parts, int64_t n_parts, StepParams* k) {
    if (!c || !grads || !params || !m || !v || !step || !valid(c)) return LGRECO_EINVAL;
    if (!gradient_type(grad_type)) return LGRECO_EINVAL;
    if (copy && copy_type != LGRECO_BF16 && copy_type != LGRECO_F16) return LGRECO_EINVAL;
    if (c->max_norm > 0.0 && !sumsq) return LGRECO_EINVAL;
    if (misaligned(grads, element_size(grad_type)) || misaligned(params, 4) || misaligned(m, moment_size) ||
        misaligned(v, moment_size) || misaligned(copy, 2) || misaligned(sumsq, 8) || misaligned(lr, 4) || misaligned(step, 8))
        return LGRECO_EINVAL;
    const int st = on_device(o);
    if (st != LGRECO_OK) return st;
    const FactorParams raw{c->lr, c->beta1, c->beta2, c->grad_scale, c->max_norm, sumsq ? sumsq + o->L : nullptr, lr, step};
    const bool short_table = n_parts <= kShortParts;
    *k = StepParams{parts, short_table ? nullptr : o->d_factors, raw, o->d_tickets, grads, params, const_cast<void*>(m),
                    const_cast<void*>(v), nullptr, const_cast<void*>(copy), c->weight_decay, (float)c->beta1, (float)(1.0 - c->beta1),
                    (float)c->beta2, (float)(1.0 - c->beta2), (float)c->eps, c->stochastic, (uint32_t)c->seed, (uint32_t)(c->seed >> 32)};
    if (!short_table) HIPCHK(launch(factors_kernel, 1, 64, 0, s, raw, o->d_factors));
    return LGRECO_OK;
}

typedef void (*StepKernel)(StepParams);

template <typename G>
StepKernel adamw_kernel_of(bool copy, int32_t copy_type) {
    return !copy ? adamw_kernel<G, NoCopy> : copy_type == LGRECO_BF16 ? adamw_kernel<G, BF16> : adamw_kernel<G, F16>;
}
template <typename G, bool STOCHASTIC>
StepKernel coded_kernel_of(bool copy, int32_t copy_type) {
    return !copy ? adamw_coded_kernel<G, NoCopy, STOCHASTIC>
                 : copy_type == LGRECO_BF16 ? adamw_coded_kernel<G, BF16, STOCHASTIC> : adamw_coded_kernel<G, F16, STOCHASTIC>;
}
template <typename G>
StepKernel coded_kernel_of(bool stochastic, bool copy, int32_t copy_type) {
    return stochastic ? coded_kernel_of<G, true>(copy, copy_type) : coded_kernel_of<G, false>(copy, copy_type);
}

}  // namespace

extern "C" {

int lgreco_optim_create(lgreco_optim_t** out, const lgreco_layer_t* layers, int32_t L, const float* lr_scale,
                        const float* decay_scale) {
    if (!out) return LGRECO_EINVAL;
    *out = nullptr;
    create_error[0] = 0;
    lgreco_optim* o = new (std::nothrow) lgreco_optim();
    if (!o) return LGRECO_ENOSPACE;
    int st;
    try {
        st = create(o, layers, L, lr_scale, decay_scale);
    } catch (...) {                                          // (host memory)
        st = LGRECO_ENOSPACE;
    }
    if (st == LGRECO_OK) {
        *out = o;
    } else {
        std::memcpy(create_error, o->error, sizeof(create_error));
        lgreco_optim_destroy(o);
    }
    return st;
}

int lgreco_optim_destroy(lgreco_optim_t* o) {
    if (!o) return LGRECO_EINVAL;
    (void)hipFree(o->d_all);
    delete o;
    return LGRECO_OK;
}

int64_t lgreco_optim_blocks(const lgreco_optim_t* o) { return o ? o->blocks : -1; }

const char* lgreco_optim_last_hip_error(const lgreco_optim_t* o) { return o ? o->error : create_error; }

int lgreco_optim_norms(lgreco_optim_t* o, const void* d_grads, int32_t grad_type, double* d_sumsq, void* stream) {
    if (!o || !d_grads || !d_sumsq || !gradient_type(grad_type)) return LGRECO_EINVAL;
    if (misaligned(d_grads, element_size(grad_type)) || misaligned(d_sumsq, 8)) return LGRECO_EINVAL;
    const int st = on_device(o);
    if (st != LGRECO_OK) return st;
    hipStream_t s = (hipStream_t)stream;
    const NormParams k{o->d_norm, d_grads, o->d_partials, d_sumsq, o->L, o->d_norm_tickets};
    HIPCHK(launch(grad_type == LGRECO_F32 ? norms_kernel<float> : grad_type == LGRECO_BF16 ? norms_kernel<BF16> : norms_kernel<F16>, o->n_norm,
                  kThreads, 0, s, k));
    return LGRECO_OK;
}

int lgreco_optim_adamw(lgreco_optim_t* o, const lgreco_adamw_t* cfg, const void* d_grads, int32_t grad_type,
                       float* d_params, float* d_m, float* d_v, void* d_copy, int32_t copy_type,
                       const double* d_sumsq, const float* d_lr, int64_t* d_step, void* stream) {
    hipStream_t s = (hipStream_t)stream;
    if (!o) return LGRECO_EINVAL;
    StepParams k;
    const int st = begin_step(o, cfg, d_grads, grad_type, d_params, d_m, d_v, 4, d_copy, copy_type, d_sumsq, d_lr, d_step, s, o->d_step, o->n_step, &k);
    if (st != LGRECO_OK) return st;
    const StepKernel f = grad_type == LGRECO_F32    ? adamw_kernel_of<float>(d_copy, copy_type)
                         : grad_type == LGRECO_BF16 ? adamw_kernel_of<BF16>(d_copy, copy_type) : adamw_kernel_of<F16>(d_copy, copy_type);
    HIPCHK(launch(f, o->n_step, kThreads, k.factors ? kStepLds : 0, s, k));
    return LGRECO_OK;
}

int lgreco_optim_adamw_coded(lgreco_optim_t* o, const lgreco_adamw_t* cfg, const void* d_grads, int32_t grad_type,
                             float* d_params, uint8_t* d_m, uint8_t* d_v, uint8_t* d_exps, void* d_copy,
                             int32_t copy_type, const double* d_sumsq, const float* d_lr, int64_t* d_step,
                             void* stream) {
    hipStream_t s = (hipStream_t)stream;
    if (!o || !d_exps) return LGRECO_EINVAL;
    StepParams k;
    const int st = begin_step(o, cfg, d_grads, grad_type, d_params, d_m, d_v, 1, d_copy, copy_type, d_sumsq, d_lr, d_step, s, o->d_coded, o->n_coded, &k);
    if (st != LGRECO_OK) return st;
    k.exps = d_exps;
    const bool random = cfg->stochastic != 0;
    const StepKernel f = grad_type == LGRECO_F32    ? coded_kernel_of<float>(random, d_copy, copy_type)
                         : grad_type == LGRECO_BF16 ? coded_kernel_of<BF16>(random, d_copy, copy_type)
                                                    : coded_kernel_of<F16>(random, d_copy, copy_type);
    HIPCHK(launch(f, o->n_coded, o->coded_threads, k.factors ? kCodedLds : 0, s, k));
    return LGRECO_OK;
}

int lgreco_optim_decode(lgreco_optim_t* o, const uint8_t* d_m, const uint8_t* d_v, const uint8_t* d_exps,
                        void* d_m_out, void* d_v_out, int32_t type, void* stream) {
    if (!o || !d_m || !d_v || !d_exps || !d_m_out || !d_v_out || (type != LGRECO_F32 && type != LGRECO_BF16)) return LGRECO_EINVAL;
    if (misaligned(d_m_out, element_size(type)) || misaligned(d_v_out, element_size(type))) return LGRECO_EINVAL;
    const int st = on_device(o);
    if (st != LGRECO_OK) return st;
    hipStream_t s = (hipStream_t)stream;
    const CodedPart* const parts = o->d_coded;
    if (type == LGRECO_F32)
        HIPCHK(launch(moments_kernel<float>, o->n_coded, o->coded_threads, 0, s, parts, d_m, d_v, d_exps, static_cast<float*>(d_m_out),
                      static_cast<float*>(d_v_out)));
    else
        HIPCHK(launch(moments_kernel<BF16>, o->n_coded, o->coded_threads, 0, s, parts, d_m, d_v, d_exps, static_cast<BF16*>(d_m_out),
                      static_cast<BF16*>(d_v_out)));
    return LGRECO_OK;
}

}  // extern "C"
