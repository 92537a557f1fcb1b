// Norms of queries and keys for each head with the position rotation in the same pass, and the cache: its rows written, quantised on the way, and read back.
//
//   y = x / sqrt(mean(x^2) + eps) * w              over the 128 channels of a head; without a weight y = x
//   (y1, y2) -> (y1 cos a - y2 sin a, y2 cos a + y1 sin a),  a = position * inv_freq[c],  c < rotary / 2, of channels (c, c + rotary / 2) or (2c, 2c + 1)
//   e4m3 rows: of each 32 channels the smallest 2^e with max |y| <= 448 * 2^e; y / 2^e rounded to nearest even
//
// Everything is bound by memory: 10 operations an element.  16384 tokens of 32/8 heads (336 MB) 61 to 64 us, 5.3 to 5.5 TB/s (a large copy past the caches 5.9); 65536 tokens' K and V
// into 8-bit pages (407 MB) 83, 20001 back (62 MB) 11.5; 64 tokens into 8-bit pages 3.4 us in a graph, a launch.
// Sixteen lanes take a head of a token, 8 neighbouring channels each (16 bytes of bf16), so that
// sums over a head and maxima over 32 channels are DPP exchanges.  A wave stays with one token: its 64 lanes work out the token's angles once, one
// pair each, in 64 bits (a far position times a frequency loses its turn in 32: 131072 * 2^-24 is 0.008 radians) and hand them round through LDS.
// Sums, angles' sines (with what an angle loses as it becomes 32 bits) and products are 32 bits; an output is rounded once, keys to e4m3 from 32 bits and not by way of bf16.
// (A head of four tokens to a wave, so that rows and scales follow each other in a page, took 97 us for 85 at 65536 tokens; the four scales of a row in one store: no difference.)
// Scales are powers of two: e4m3 keeps its 4 significant bits under any of them, while x8 * 2^e is exact in bf16, which is what attention multiplies.
#include "cache.h"

#include <algorithm>

namespace cp {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2;

struct RopeArgs {
    const void *q, *k, *v, *qw, *kw;
    const double* freq;
    const int32_t *pos, *slots;
    void *q_out, *k_out;
    CachePtr cache;
    int tokens, hq, hkv, heads;               // heads: rows of a token, Q then K then V
    int waves;                                // that share a token
    int page_shift, slots_end, half;          // half = rotary / 2
    float eps;
    int64_t qs0, qs1, ks0, ks1, vs0, vs1, os0, os1, kos0, kos1;
};

enum { TURN_NONE = 0, TURN_WHOLE = 1, TURN_HALVES = 2, TURN_PAIRS = 3 };    // WHOLE: halves of all 128 channels
enum { TO_TENSOR = 0, TO_PLAIN = 1, TO_MXFP8 = 2, TO_MXFP4 = 3 };

template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
constexpr int kRor = 0x120;                                        // row_ror:n, among 16 lanes
__device__ __forceinline__ float sum16(float x) {
    x += dpp<kRor + 8>(x); x += dpp<kRor + 4>(x); x += dpp<kRor + 2>(x); x += dpp<kRor + 1>(x);
    return x;
}
__device__ __forceinline__ float max4(float x) {                   // over a lane's four: quad_perm [1,0,3,2], [2,3,0,1]
    x = fmaxf(x, dpp<0xB1>(x));
    return fmaxf(x, dpp<0x4E>(x));
}

// STREAM: what goes past the caches.  Calls that move more than kStreamBytes find nothing of theirs in a cache and leave nothing that is still there when it is read
// (Infinity Cache: 256 MiB, shared with what runs before and after); smaller ones do.  us, ordinary / past the caches, 32/8 heads in bf16: 16384 tokens as tensors (336 MB) 73.6 / 63.8,
// 8192 (168 MB) 40.4 / 33.2, 16384 into 8-bit pages 82.7 / 75.3, 65536 tokens' K and V into plain pages 114 / 100 and back 99 / 87; 9000 tokens' back in fp32 (147 MB) 33 / 43, 3000
// tokens as tensors (61 MB) 15.1 / 17.0.
constexpr long long kStreamBytes = 150ll << 20;
template <bool STREAM, typename V>
__device__ __forceinline__ V get(const void* p) { return STREAM ? __builtin_nontemporal_load((const V*)p) : *(const V*)p; }
template <bool STREAM, typename V>
__device__ __forceinline__ void put(void* p, V v) { if (STREAM) __builtin_nontemporal_store(v, (V*)p); else *(V*)p = v; }

template <bool STREAM>
__device__ __forceinline__ void load8(const __bf16* p, float (&x)[8]) {
    const bf16x8 v = get<STREAM, bf16x8>(p);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
}
template <bool STREAM>
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
    const f32x4 a = get<STREAM, f32x4>(p), b = get<STREAM, f32x4>(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) { x[e] = a[e]; x[4 + e] = b[e]; }
}
template <bool STREAM>
__device__ __forceinline__ void store8(__bf16* p, const float (&x)[8]) {
    bf16x8 v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (__bf16)x[e];
    put<STREAM>(p, v);
}
template <bool STREAM>
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
    f32x4 a, b;
#pragma unroll
    for (int e = 0; e < 4; ++e) { a[e] = x[e]; b[e] = x[4 + e]; }
    put<STREAM>(p, a); put<STREAM>(p + 4, b);
}

// 8 channels of a row in e4m3, and in the first lane of four the biased exponent of their 32 channels.  Values that are not finite take no part in the
// maximum and are stored as e4m3's NaN; exponents stay in 1 .. 254, where 2^(e - 127) is a normal number.
__device__ __forceinline__ u32x2 quantise8(float (&x)[8], int& exponent) {
    float most = fabsf(x[0]);
#pragma unroll
    for (int e = 1; e < 8; ++e) most = fmaxf(most, fabsf(x[e]));   // a NaN takes no part by itself
    most = max4(most);
    if (!(most < INFINITY)) {                                      // an infinity, or nothing but NaN: rare, and not worth three instructions an element
        most = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (!(fabsf(x[e]) < INFINITY)) x[e] = NAN;
            else most = fmaxf(most, fabsf(x[e]));
        }
        most = max4(most);
    }
    const unsigned bits = __float_as_uint(most);
    exponent = min(max((int)(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0), 1), 254);   // 448 = 1.75 * 2^8
    const float scale = __uint_as_float(exponent == 254 ? 0x400000u : (unsigned)(254 - exponent) << 23);     // 2^(127 - exponent), exact also where it is subnormal
    u32x2 w;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int d = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * e] * scale, x[4 * e + 1] * scale, 0, false);
        w[e] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * e + 2] * scale, x[4 * e + 3] * scale, d, true);
    }
    return w;
}

// The same in e2m1, two to a byte.  The smallest 2^e with max |x| <= 7 * 2^e: what lies above the largest element, 6, becomes it and is off by a unit at most, as much as rounding costs
// between 4 and 6; the next scale's steps there are two units.  e in 2 .. 252: half a unit is a normal number, and 6 of the largest are finite (larger maxima saturate).  e2m1 has no
// NaN: 32 channels of which any value is not finite get the scale's, 255, and are held as NaN together.
__device__ __forceinline__ unsigned quantise8_to_4(const float (&x)[8], int& exponent) {
    float most = 0.f, nothing = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        most = fmaxf(most, fabsf(x[e]));
        nothing = fmaf(x[e], 0.f, nothing);                        // NaN of what is not finite
    }
    most = max4(most);
    nothing += dpp<0xB1>(nothing);
    nothing += dpp<0x4E>(nothing);
    const unsigned bits = __float_as_uint(most);
    exponent = min(max((int)(bits >> 23) - 2 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0), 2), 252);        // 7 = 1.75 * 2^2
    if (nothing != 0.f) { exponent = 255; return 0; }
    const float scale = __uint_as_float((unsigned)exponent << 23);
    unsigned w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], scale, 0);                       // of x / scale, to nearest even, at most 6
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
}

// Rows of 4 bits are half a line of L2, 64 bytes, and a token's scales of a head 4 of a line that 32 tokens share.  They are written and read by ordinary accesses, which bring a line together, whatever the
// tensors do, and lines' tokens come to one XCD.  32/8 heads, us, past the caches and tokens dealt over the XCDs / ordinary / and together: 65536 tokens back 72.1 / 54.1 / 49.8, written and
// back 148.9 / 130.5 / 123.4, 8192 back 9.3 / 9.2 / 8.8.
// Of 8 * kTogether neighbouring workgroups the first kTogether on an XCD, whichever these are: 32 tokens where a wave has one to itself (from 2049 on), whose scales of a head fill a line of its L2; with fewer
// tokens, which waves share, as many fewer, and a part of a line.  What is left over stays as it is.
constexpr unsigned kTogether = 8;
__device__ __forceinline__ unsigned by_xcd(unsigned b, unsigned blocks) {
    return b < blocks / (8 * kTogether) * (8 * kTogether) ? b / (8 * kTogether) * (8 * kTogether) + (b & 7) * kTogether + (b >> 3) % kTogether : b;
}

template <typename T, int TURN, int TO, bool STREAM>
__global__ __launch_bounds__(256) void norm_rope_kernel(RopeArgs a) {
    __shared__ f32x2 turns[4][64];                                 // (cos, sin) of the wave's token
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c16 = lane & 15;
    const unsigned index = (TO == TO_MXFP4 ? by_xcd(blockIdx.x, gridDim.x) : blockIdx.x) * 4u + wave;
    const int token = __builtin_amdgcn_readfirstlane((int)(index / (unsigned)a.waves));
    const int part = (int)index - token * a.waves;
    if (token >= a.tokens) return;                                 // no barrier below: a wave's exchange is its own
    int slot = 0;
    bool kept = true;
    if (TO != TO_TENSOR) { slot = a.slots[token]; kept = (unsigned)slot < (unsigned)a.slots_end; }
    float cs[8], sn[8];                                            // of the lane's channels; of its four pairs
    if (TURN != TURN_NONE) {
        const double angle = lane < a.half ? (double)a.pos[token] * a.freq[lane] * 0.15915494309189533577 : 0.0;   // in whole turns
        const double half_turns = 2.0 * (angle - rint(angle));
        const float near = (float)half_turns, rest = (float)(half_turns - near) * 3.14159265f;   // what the cast leaves out, up to 9e-8, which a small sine is made of
        float s, c;
        sincospif(near, &s, &c);
        turns[wave][lane] = f32x2{fmaf(-s, rest, c), fmaf(c, rest, s)};
        __builtin_amdgcn_wave_barrier();
        if (TURN == TURN_PAIRS) {
#pragma unroll
            for (int e = 0; e < 4; ++e) { const f32x2 t = turns[wave][4 * c16 + e]; cs[e] = t[0]; sn[e] = t[1]; }
        } else {
            // channel c < half takes the pair c as its first, c < rotary the pair c - half as its second
            const int first = 8 * c16 < a.half ? 8 * c16 : 8 * c16 - a.half;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const f32x2 t = turns[wave][(first + e) & 63];
                cs[e] = t[0]; sn[e] = 8 * c16 < a.half ? -t[1] : t[1];
            }
        }
    }
    const bool turned = 8 * c16 < 2 * a.half;
    float qw[8], kw[8];
    if (TURN != TURN_NONE || TO == TO_TENSOR) {
        if (a.qw) load8<false>((const T*)a.qw + 8 * c16, qw);
        if (a.kw) load8<false>((const T*)a.kw + 8 * c16, kw);
    }
    for (int head = 4 * part + (lane >> 4); head < a.heads; head += 4 * a.waves) {
        const int kind = head < a.hq ? 0 : (head < a.hq + a.hkv ? 1 : 2);
        const int h = kind == 0 ? head : (kind == 1 ? head - a.hq : head - a.hq - a.hkv);
        const T* from = kind == 0 ? (const T*)a.q + token * a.qs0 + h * a.qs1
                                  : (kind == 1 ? (const T*)a.k + token * a.ks0 + h * a.ks1 : (const T*)a.v + token * a.vs0 + h * a.vs1);
        float x[8];
        // fp32 for 4 bits: two instructions share a line.  8/2 heads: 16000 tokens with norms 37.7 us past the caches, 35.5 by ordinary loads; 60000 tokens of 8 heads written 121 and 115
        load8<STREAM && (TO != TO_MXFP4 || sizeof(T) == 2)>(from + 8 * c16, x);
        if (TURN != TURN_NONE || TO == TO_TENSOR) {
            if (kind < 2 && (kind ? a.kw : a.qw)) {
                float sq = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) sq = fmaf(x[e], x[e], sq);
                const float inv = 1.0f / sqrtf(sum16(sq) * (1.0f / kHeadDim) + a.eps);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = x[e] * inv * (kind ? kw[e] : qw[e]);
            }
        }
        if (TURN == TURN_PAIRS) {
            if (kind < 2 && turned) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float y1 = x[2 * e], y2 = x[2 * e + 1];
                    x[2 * e] = y1 * cs[e] - y2 * sn[e];
                    x[2 * e + 1] = y2 * cs[e] + y1 * sn[e];
                }
            }
        } else if (TURN != TURN_NONE) {
            float y[8];                                            // the other half of the lane's pairs
            if (TURN == TURN_WHOLE) {
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = dpp<kRor + 8>(x[e]);
            } else {
                const int other = (lane & 48) + (turned ? (8 * c16 < a.half ? c16 + (a.half >> 3) : c16 - (a.half >> 3)) : c16);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = __int_as_float(__builtin_amdgcn_ds_bpermute(4 * other, __float_as_int(x[e])));
            }
            if (kind < 2 && turned) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = x[e] * cs[e] + y[e] * sn[e];
            }
        }
        if (kind == 0) {
            store8<STREAM>((T*)a.q_out + token * a.os0 + h * a.os1 + 8 * c16, x);
        } else if (TO == TO_TENSOR) {
            store8<STREAM>((T*)a.k_out + token * a.kos0 + h * a.kos1 + 8 * c16, x);
        } else {
            const int64_t row = (((int64_t)(slot >> a.page_shift) * a.hkv + h) << a.page_shift) + (slot & ((1 << a.page_shift) - 1));
            if (TO == TO_PLAIN) {
                if (kept) store8<STREAM>((T*)(kind == 1 ? a.cache.k : a.cache.v) + row * kHeadDim + 8 * c16, x);
            } else if (TO == TO_MXFP4) {
                int e;
                const unsigned w = quantise8_to_4(x, e);
                if (kept) {
                    put<false>((uint8_t*)(kind == 1 ? a.cache.k : a.cache.v) + row * (kHeadDim / 2) + 4 * c16, w);
                    if ((c16 & 3) == 0) (kind == 1 ? a.cache.ks : a.cache.vs)[row * 4 + (c16 >> 2)] = (uint8_t)e;
                }
            } else {
                int e;
                const u32x2 w = quantise8(x, e);
                if (kept) {
                    put<STREAM>((uint8_t*)(kind == 1 ? a.cache.k : a.cache.v) + row * kHeadDim + 8 * c16, w);
                    if ((c16 & 3) == 0) (kind == 1 ? a.cache.ks : a.cache.vs)[row * 4 + (c16 >> 2)] = (uint8_t)e;
                }
            }
        }
    }
}

template <typename T, int HELD, bool STREAM>
__global__ __launch_bounds__(256) void cache_read_kernel(RopeArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c16 = lane & 15;
    const unsigned index = (HELD == HELD_MXFP4 ? by_xcd(blockIdx.x, gridDim.x) : blockIdx.x) * 4u + wave;
    const int token = __builtin_amdgcn_readfirstlane((int)(index / (unsigned)a.waves));
    const int part = (int)index - token * a.waves;
    if (token >= a.tokens) return;
    const int slot = a.slots[token];
    const bool held = (unsigned)slot < (unsigned)a.slots_end;
    for (int head = 4 * part + (lane >> 4); head < a.heads; head += 4 * a.waves) {
        const bool is_v = head >= a.hkv;
        const int h = is_v ? head - a.hkv : head;
        const int64_t row = (((int64_t)(slot >> a.page_shift) * a.hkv + h) << a.page_shift) + (slot & ((1 << a.page_shift) - 1));
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.f;                    // a token without a place in the cache
        if (held) {
            if (HELD == HELD_MXFP4) {
                // of fp32 channels 4 c16 .. and 64 + 4 c16 .., so that a store writes whole lines: 20000 tokens of 8 heads 48.9 us with 8 c16 .., now 31
                const uint8_t* from = (const uint8_t*)(is_v ? a.cache.v : a.cache.k) + row * (kHeadDim / 2);
                const uint8_t* scales = (is_v ? a.cache.vs : a.cache.ks) + row * 4;
                unsigned w; float s0, s1;
                if (sizeof(T) == 4) {
                    w = *(const uint16_t*)(from + 2 * c16) | (unsigned)*(const uint16_t*)(from + 32 + 2 * c16) << 16;
                    s0 = __uint_as_float((unsigned)scales[c16 >> 3] << 23); s1 = __uint_as_float((unsigned)scales[2 + (c16 >> 3)] << 23);
                } else {
                    w = *(const unsigned*)(from + 4 * c16);
                    s0 = s1 = __uint_as_float((unsigned)scales[c16 >> 2] << 23);                   // of 255: NaN
                }
                const f32x2 y[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s0, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s0, 1),
                                    __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s1, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s1, 3)};
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = y[e >> 1][e & 1];
            } else if (HELD == HELD_MXFP8) {
                const u32x2 w = get<STREAM, u32x2>((const uint8_t*)(is_v ? a.cache.v : a.cache.k) + row * kHeadDim + 8 * c16);
                const float scale = __uint_as_float((unsigned)(is_v ? a.cache.vs : a.cache.ks)[row * 4 + (c16 >> 2)] << 23);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[e], scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[e], scale, true);
                    x[4 * e] = lo[0]; x[4 * e + 1] = lo[1]; x[4 * e + 2] = hi[0]; x[4 * e + 3] = hi[1];
                }
            } else {
                load8<STREAM>((const T*)(is_v ? a.cache.v : a.cache.k) + row * kHeadDim + 8 * c16, x);
            }
        }
        T* const to = (T*)(is_v ? a.q_out : a.k_out) + token * (is_v ? a.vs0 : a.ks0) + h * (is_v ? a.vs1 : a.ks1);
        if (HELD == HELD_MXFP4 && sizeof(T) == 4) {
            put<STREAM>(to + 4 * c16, f32x4{x[0], x[1], x[2], x[3]});
            put<STREAM>(to + 64 + 4 * c16, f32x4{x[4], x[5], x[6], x[7]});
        } else store8<STREAM>(to + 8 * c16, x);
    }
}

RopeArgs common(const CacheShape& sh, int heads, const CachePtr* cache) {
    RopeArgs a = {};
    a.tokens = sh.tokens; a.hq = sh.hq; a.hkv = sh.hkv; a.heads = heads;
    a.page_shift = sh.page_shift; a.slots_end = sh.n_pages << sh.page_shift;
    if (cache) a.cache = *cache;
    a.eps = sh.eps;
    a.qs0 = sh.qs[0]; a.qs1 = sh.qs[1]; a.ks0 = sh.ks[0]; a.ks1 = sh.ks[1]; a.vs0 = sh.vs[0]; a.vs1 = sh.vs[1];
    a.os0 = sh.os[0]; a.os1 = sh.os[1]; a.kos0 = sh.kos[0]; a.kos1 = sh.kos[1];
    // A wave with all heads of a token works the angles out once; few tokens are shared by waves of four heads, until the chip's 256 * 16 are there
    const int most = (heads + 3) / 4;
    a.waves = (int)std::min<long long>(most, std::max<long long>(1, 4096 / std::max(sh.tokens, 1)));
    return a;
}

unsigned grid_of(const RopeArgs& a) { return (unsigned)(((long long)a.tokens * a.waves + 3) / 4); }

template <typename T, int TURN, int TO>
hipError_t launch(const RopeArgs& a, bool stream, hipStream_t st) {
    constexpr bool kCan = !(sizeof(T) == 4 && TURN == TURN_NONE && TO == TO_MXFP4);   // of fp32 as it is into 4 bits all accesses are ordinary ones
    if (kCan && stream) hipLaunchKernelGGL((norm_rope_kernel<T, TURN, TO, kCan>), dim3(grid_of(a)), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((norm_rope_kernel<T, TURN, TO, false>), dim3(grid_of(a)), dim3(256), 0, st, a);
    return hipGetLastError();
}
template <typename T, int TO>
hipError_t launch_turn(const RopeArgs& a, int turn, bool stream, hipStream_t st) {
    return turn == TURN_WHOLE ? launch<T, TURN_WHOLE, TO>(a, stream, st) : turn == TURN_HALVES ? launch<T, TURN_HALVES, TO>(a, stream, st) : launch<T, TURN_PAIRS, TO>(a, stream, st);
}
// From 4 bits the tensors are nearly all that moves, and go past the caches at any size: 8 heads in bf16, 4000 tokens 8.5 / 6.8 us, 8000 12.1 / 8.5, 30000 36.6 / 24.1, in fp32 4000 12.6 / 8.9.
template <typename T, int HELD>
hipError_t launch_read(const RopeArgs& a, bool stream, hipStream_t st) {
    constexpr bool kAlways = HELD == HELD_MXFP4;
    if (kAlways || stream) hipLaunchKernelGGL((cache_read_kernel<T, HELD, true>), dim3(grid_of(a)), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((cache_read_kernel<T, HELD, kAlways>), dim3(grid_of(a)), dim3(256), 0, st, a);
    return hipGetLastError();
}
// a kernel for each way that the cache may hold rows
template <typename T>
hipError_t launch_rope_write(const RopeArgs& a, int turn, int held, bool stream, hipStream_t st) {
    return held == HELD_MXFP4 ? launch_turn<T, TO_MXFP4>(a, turn, stream, st) : held == HELD_MXFP8 ? launch_turn<T, TO_MXFP8>(a, turn, stream, st) : launch_turn<T, TO_PLAIN>(a, turn, stream, st);
}
template <typename T>
hipError_t launch_write(const RopeArgs& a, int held, bool stream, hipStream_t st) {
    return held == HELD_MXFP4 ? launch<T, TURN_NONE, TO_MXFP4>(a, stream, st) : held == HELD_MXFP8 ? launch<T, TURN_NONE, TO_MXFP8>(a, stream, st) : launch<T, TURN_NONE, TO_PLAIN>(a, stream, st);
}
template <typename T>
hipError_t launch_back(const RopeArgs& a, int held, bool stream, hipStream_t st) {
    return held == HELD_MXFP4 ? launch_read<T, HELD_MXFP4>(a, stream, st) : held == HELD_MXFP8 ? launch_read<T, HELD_MXFP8>(a, stream, st) : launch_read<T, HELD_PLAIN>(a, stream, st);
}

}  // namespace

// Whether a call goes past the caches: bytes read and written, `rows` of each token as elements of dtype, `held` of each in the cache.
bool cache_call_streams(const CacheShape& sh, int rows, int held) {
    const long long e = sh.dtype == 1 ? 2 : 4;
    return (long long)sh.tokens * (rows * kHeadDim * e + held * row_bytes(sh.held, (int)e)) > kStreamBytes;
}

hipError_t launch_norm_rope(const CacheShape& sh, const void* q, const void* k, const void* v, const void* q_weight, const void* k_weight,
                            const double* inv_freq, const int32_t* positions, const int32_t* slots, void* q_out, void* k_out, const CachePtr* cache, hipStream_t st) {
    RopeArgs a = common(sh, sh.hq + sh.hkv + (cache ? sh.hkv : 0), cache);
    a.q = q; a.k = k; a.v = v; a.qw = q_weight; a.kw = k_weight; a.freq = inv_freq; a.pos = positions; a.slots = slots; a.q_out = q_out; a.k_out = k_out;
    a.half = sh.rotary / 2;
    const int turn = sh.interleaved ? TURN_PAIRS : (sh.rotary == kHeadDim ? TURN_WHOLE : TURN_HALVES);
    const bool stream = cache_call_streams(sh, 2 * sh.hq + 2 * sh.hkv, cache ? 2 * sh.hkv : 0);
    if (sh.dtype == 1) return !cache ? launch_turn<__bf16, TO_TENSOR>(a, turn, stream, st) : launch_rope_write<__bf16>(a, turn, sh.held, stream, st);
    return !cache ? launch_turn<float, TO_TENSOR>(a, turn, stream, st) : launch_rope_write<float>(a, turn, sh.held, stream, st);
}

hipError_t launch_cache_write(const CacheShape& sh, const void* k, const void* v, const int32_t* slots, const CachePtr& cache, hipStream_t st) {
    RopeArgs a = common(sh, 2 * sh.hkv, &cache);
    a.hq = 0; a.k = k; a.v = v; a.slots = slots;
    const bool stream = cache_call_streams(sh, 2 * sh.hkv, 2 * sh.hkv);
    return sh.dtype == 1 ? launch_write<__bf16>(a, sh.held, stream, st) : launch_write<float>(a, sh.held, stream, st);
}

hipError_t launch_cache_read(const CacheShape& sh, const int32_t* slots, const CachePtr& cache, void* k, void* v, hipStream_t st) {
    RopeArgs a = common(sh, 2 * sh.hkv, &cache);
    a.slots = slots; a.k_out = k; a.q_out = v;
    const bool stream = cache_call_streams(sh, 2 * sh.hkv, 2 * sh.hkv);
    return sh.dtype == 1 ? launch_back<__bf16>(a, sh.held, stream, st) : launch_back<float>(a, sh.held, stream, st);
}

}  // namespace cp
