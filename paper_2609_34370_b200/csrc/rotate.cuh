// The rotation of position embeddings in pairs of binary32, shared by the appends.
#pragma once
#include "attn_e4m3.cuh"   // e8::pair and the packed fp32 arithmetic
#include "common.cuh"

namespace spx {

// The rotation.  cos = ch + cl and sin = sh + sl, each as two floats of the float64 value (2^-48 of it left out).
struct CosSin { uint64_t ch, cl, sh, sl; };   // of two pairs
__device__ __forceinline__ uint64_t neg2(uint64_t a) { return e8::mul2(a, e8::pair(-1.f, -1.f)); }
__device__ __forceinline__ uint64_t sub2(uint64_t a, uint64_t b) { return e8::fma2(b, e8::pair(-1.f, -1.f), a); }
// y0 = x0 cos - x1 sin, y1 = x1 cos + x0 sin.  kExact: products and sum with their rounding errors (a product's by a fused
// multiply-add, a sum's by Knuth's two-sum), one rounding to fp32 at the end of a value good to 2^-46 of |x| (what float64
// arithmetic gives but for one in some millions of last bits and the sign of a zero, at a third of its time: conversions
// from and to float64 alone are 8 cycles each); what goes into the 8-bit codes and into fp32 rows.  Otherwise the leading
// errors only: within 2 steps of fp32 of the value, for rows that are rounded to 16 bits.  An infinite x, or a result past
// fp32, gives an infinity or a NaN.
template <bool kExact>
__device__ __forceinline__ void rotate2(uint64_t x0, uint64_t x1, const CosSin &k, uint64_t &y0, uint64_t &y1) {
  using namespace e8;
  const uint64_t n0 = neg2(x0), n1 = neg2(x1);
  if constexpr (kExact) {
    {
      const uint64_t p = mul2(x0, k.ch), np = fma2(n0, k.ch, p), q = mul2(x1, k.sh), nq = fma2(n1, k.sh, q);
      const uint64_t s = sub2(p, q), bb = sub2(s, p);
      const uint64_t err = sub2(sub2(p, sub2(s, bb)), add2(q, bb));
      y0 = add2(s, add2(fma2(n1, k.sl, fma2(x0, k.cl, err)), sub2(nq, np)));
    }
    {
      const uint64_t p = mul2(x1, k.ch), np = fma2(n1, k.ch, p), q = mul2(x0, k.sh), nq = fma2(n0, k.sh, q);
      const uint64_t s = add2(p, q), bb = sub2(s, p);
      const uint64_t err = add2(sub2(p, sub2(s, bb)), sub2(q, bb));
      y1 = add2(s, sub2(fma2(x0, k.sl, fma2(x1, k.cl, err)), add2(np, nq)));
    }
  } else {
    const uint64_t w = mul2(x1, k.sh), nw = mul2(n1, k.sh), u = mul2(x0, k.sh), nu = mul2(n0, k.sh);
    y0 = add2(fma2(x0, k.ch, nw), fma2(n1, k.sl, fma2(x0, k.cl, fma2(n1, k.sh, w))));
    y1 = add2(fma2(x1, k.ch, u), fma2(x0, k.sl, fma2(x1, k.cl, fma2(x0, k.sh, nu))));
  }
}

}  // namespace spx
