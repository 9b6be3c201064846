// The mask of dropout, which is nowhere stored: whether an element is kept is a function of a key, a step, a place in the network and
// the element's own place, and every kernel that needs the mask forms it again.
//
// The generator is Philox 4x32 of ten rounds (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", 2011): ten
// rounds of two 32 x 32 bit products make 128 random bits from a counter of 128 bits and a key of 64.  Eight neighbours of a row share
// them, 16 bits each: the counter is (group low, group high | site << 8, step low, step high), the group row * ceil(columns / 8) + column / 8.
// An element whose 16 bits are below limit = round(65536 p) is dropped and the others are multiplied by 65536 / (65536 - limit), the inverse
// of the probability that 16 bits really give, so that the mean is kept exactly.
// Twenty products at a quarter of the full rate and 40 exclusive ors make 0.3 us of a compute unit's time for 4096 elements: about 3.5e12 elements a
// second on the whole card, above what it can read and write in 16 bits (5e12 bytes a second).  Sixteen bits an element and not 32 halve
// that; the probability is a multiple of 2^-16 then.
#pragma once
#include "common.h"

namespace cac {

struct Drop {
    const uint64_t *rng; // {key, step}, on the device: a captured graph has another mask when the caller writes another step
    uint32_t limit;      // 0 to 65536; 0: nothing is dropped and rng is not read
    uint32_t site;       // below 2^24
    float scale;         // of what is kept
};

struct DropKey { uint32_t k0, k1, c2, c3; };

__device__ __forceinline__ DropKey drop_key(const Drop &d)
{
    DropKey k = {0, 0, 0, 0};
    if (d.limit) {
        const uint64_t seed = d.rng[0], step = d.rng[1];
        k = DropKey{(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)step, (uint32_t)(step >> 32)};
    }
    return k;
}

struct Bits128 { uint32_t w[4]; };

__device__ __forceinline__ Bits128 drop_bits(const DropKey &key, uint32_t site, uint64_t group)
{
    uint32_t c0 = (uint32_t)group, c1 = (uint32_t)(group >> 32) | site << 8, c2 = key.c2, c3 = key.c3, k0 = key.k0, k1 = key.k1;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        const uint32_t n0 = (uint32_t)(b >> 32) ^ c1 ^ k0, n2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c1 = (uint32_t)b;
        c3 = (uint32_t)a;
        c0 = n0;
        c2 = n2;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return Bits128{{c0, c1, c2, c3}};
}

// element e of a word's two, e = 0 or 1
__device__ __forceinline__ bool drop_keeps(uint32_t word, int e, uint32_t limit) { return (e ? word >> 16 : word & 0xffffu) >= limit; }

// eight neighbours of one group: what is kept times `scale`, zeros for the others (whatever stands there)
__device__ __forceinline__ void drop_eight(const DropKey &key, const Drop &d, uint64_t group, float scale, float (&v)[8])
{
    if (!d.limit) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= scale;
        return;
    }
    const Bits128 b = drop_bits(key, d.site, group);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = drop_keeps(b.w[e >> 1], e & 1, d.limit) ? v[e] * scale : 0.f;
}

// ---- eight neighbours of a row as floats
template <typename T> struct Eight;
template <> struct Eight<float> {
    float4 a, b;
    __device__ __forceinline__ void read(const float *p) { a = ((const float4 *)p)[0], b = ((const float4 *)p)[1]; }
    __device__ __forceinline__ void write(float *p) const { ((float4 *)p)[0] = a, ((float4 *)p)[1] = b; }
    __device__ __forceinline__ void get(float (&v)[8]) const { v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w; }
    __device__ __forceinline__ void set(const float (&v)[8]) { a = make_float4(v[0], v[1], v[2], v[3]), b = make_float4(v[4], v[5], v[6], v[7]); }
};
template <> struct Eight<bf16_t> {
    uint4 a;
    __device__ __forceinline__ void read(const bf16_t *p) { a = *(const uint4 *)p; }
    __device__ __forceinline__ void write(bf16_t *p) const { *(uint4 *)p = a; }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
        const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[2 * k] = __uint_as_float(u[k] << 16);
            v[2 * k + 1] = __uint_as_float(u[k] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void set(const float (&v)[8])
    {
        a = make_uint4(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]), f32x2_to_bf16x2(v[4], v[5]), f32x2_to_bf16x2(v[6], v[7]));
    }
};
// of a row of `columns` from column n on; `wide`: every group is whole and starts on 16 bytes
template <typename T> __device__ __forceinline__ Eight<T> read_eight(const T *row, int n, int columns, bool wide)
{
    Eight<T> r;
    if (wide) {
        r.read(row + n);
        return r;
    }
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = n + e < columns ? Elem<T>::load(row + n + e) : 0.f;
    r.set(v);
    return r;
}
template <typename T> __device__ __forceinline__ void write_eight(T *row, int n, int columns, bool wide, const float (&v)[8])
{
    if (wide) {
        Eight<T> r;
        r.set(v);
        r.write(row + n);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (n + e < columns) Elem<T>::store(row + n + e, v[e]);
}

} // namespace cac
