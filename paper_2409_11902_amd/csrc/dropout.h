// The mask of dropout, which is nowhere stored: whether an element is kept is a function of a key, a step, a place in the network and
// the element's own place, and every kernel that needs the mask forms it again.
//
// The generator is Philox 4x32 of ten rounds (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", 2011): ten
// rounds of two 32 x 32 bit products make 128 random bits from a counter of 128 bits and a key of 64.  Eight neighbours of a row share
// them, 16 bits each: the counter is (group low, group high | site << 8, step low, step high), the group row * ceil(columns / 8) + column / 8.
// An element whose 16 bits are below limit = round(65536 p) is dropped and the others are multiplied by 65536 / (65536 - limit), the inverse
// of the probability that 16 bits really give, so that the mean is kept exactly.
// Twenty products and 20 exclusive ors of three words make the bits of eight elements; with the comparisons vector instructions take 54 % of the
// cycles of 16384 x 4096 bfloat16 elements in 72 us, which memory bounds.  32 bits to an element would take twice the products and
// make the generator the bound; with 16 the probability is a multiple of 2^-16.
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
        const uint32_t n0 = __builtin_amdgcn_bitop3_b32((uint32_t)(b >> 32), c1, k0, 0x96), n2 = __builtin_amdgcn_bitop3_b32((uint32_t)(a >> 32), c3, k1, 0x96); // a ^ b ^ c
        c1 = (uint32_t)b;
        c3 = (uint32_t)a;
        c0 = n0;
        c2 = n2;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return Bits128{{c0, c1, c2, c3}};
}

// element e of a word's two, e = 0 or 1: its 16 bits, on top of a word, reach limit 2^16 (limit is at least 1; what lies below them makes no difference)
__device__ __forceinline__ bool drop_keeps(uint32_t word, int e, uint32_t limit) { return (e ? word : word << 16) > (limit << 16) - 1; }

// eight neighbours of one group: zeros for what is dropped (whatever stands there)
__device__ __forceinline__ void drop_eight(const DropKey &key, const Drop &d, uint64_t group, float (&v)[8])
{
    if (!d.limit) return;
    const Bits128 b = drop_bits(key, d.site, group);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = drop_keeps(b.w[e >> 1], e & 1, d.limit) ? v[e] : 0.f;
}

// ---- eight neighbours of a row as floats.  Rows may start anywhere: loads and stores of 16 bytes take any address of an element.
typedef uint32_t whole16 __attribute__((ext_vector_type(4)));
typedef whole16 any16 __attribute__((aligned(2)));

template <typename T> struct Eight;
template <> struct Eight<float> {
    whole16 a, b;
    __device__ __forceinline__ void read(const float *p) { a = ((const any16 *)p)[0], b = ((const any16 *)p)[1]; }
    __device__ __forceinline__ void write(float *p) const { ((any16 *)p)[0] = a, ((any16 *)p)[1] = b; }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(a[e]), v[4 + e] = __uint_as_float(b[e]);
    }
    __device__ __forceinline__ void set(const float (&v)[8])
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) a[e] = __float_as_uint(v[e]), b[e] = __float_as_uint(v[4 + e]);
    }
    __device__ __forceinline__ void clear() { a = b = whole16{0, 0, 0, 0}; }
    // s elements towards the first, zeros after them
    __device__ __forceinline__ void shift(int s)
    {
        if (s & 4) a = b, b = whole16{0, 0, 0, 0};
        if (s & 2) a = whole16{a[2], a[3], b[0], b[1]}, b = whole16{b[2], b[3], 0, 0};
        if (s & 1) a = whole16{a[1], a[2], a[3], b[0]}, b = whole16{b[1], b[2], b[3], 0};
    }
};
template <> struct Eight<bf16_t> {
    whole16 a;
    __device__ __forceinline__ void read(const bf16_t *p) { a = *(const any16 *)p; }
    __device__ __forceinline__ void write(bf16_t *p) const { *(any16 *)p = a; }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[2 * k] = __uint_as_float(a[k] << 16);
            v[2 * k + 1] = __uint_as_float(a[k] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void set(const float (&v)[8])
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) a[k] = f32x2_to_bf16x2(v[2 * k], v[2 * k + 1]);
    }
    __device__ __forceinline__ void clear() { a = whole16{0, 0, 0, 0}; }
    __device__ __forceinline__ void shift(int s)
    {
        if (s & 4) a = whole16{a[2], a[3], 0, 0};
        if (s & 2) a = whole16{a[1], a[2], a[3], 0};
        if (s & 1) a = whole16{a[0] >> 16 | a[1] << 16, a[1] >> 16 | a[2] << 16, a[2] >> 16 | a[3] << 16, a[3] >> 16};
    }
};
// of a row of `columns` from column n on, n below columns; zeros past its end.  WHOLE: rows are whole eights.
template <bool WHOLE = false, typename T> __device__ __forceinline__ Eight<T> read_eight(const T *row, int n, int columns)
{
    Eight<T> r;
    if (WHOLE || n + 8 <= columns) {
        r.read(row + n);
    } else if (columns >= 8) { // the row's last eight, those before n taken out
        r.read(row + columns - 8);
        r.shift(n + 8 - columns);
    } else {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = n + e < columns ? Elem<T>::load(row + n + e) : 0.f;
        r.set(v);
    }
    return r;
}
template <bool WHOLE = false, typename T> __device__ __forceinline__ void write_eight(T *row, int n, int columns, const float (&v)[8])
{
    Eight<T> r;
    r.set(v);
    if (WHOLE || n + 8 <= columns) {
        r.write(row + n);
        return;
    }
    struct alignas(sizeof(T)) Four { T x[4]; };
    struct alignas(sizeof(T)) Two { T x[2]; };
    const int count = columns - n;
    T *p = row + n;
    if (count & 4) {
        *(Four *)p = *(const Four *)&r;
        p += 4;
        r.shift(4);
    }
    if (count & 2) {
        *(Two *)p = *(const Two *)&r;
        p += 2;
        r.shift(2);
    }
    if (count & 1) *p = *(const T *)&r;
}

} // namespace cac
