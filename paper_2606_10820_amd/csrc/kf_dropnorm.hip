// kf_dropnorm.hip -- the joint of a pre-norm block: dropout of a product's rows, their sum
// with the residual stream, and the norm of the sum,
//   h = res + [kept] in s,   y = norm(h)
// and the gradients,
//   dh = norm'(dy) + dres,   din = [kept] dh s
// in the norms' kernels (kf_norm.h): the results are those of dropout and norm one after the
// other, without the second read of h and of dh.
//
// Bound by memory: res, in, h and y once; h, dy, dres, dh and din once.  40960 x 768, fp32
// stream and bf16 product, 65 us forward (5.8 TB/s) and 82 backward (6.1), one operator after
// the other 96 and 102; 81920 x 1024 bf16 121 and 157 (5.5, 5.3).  Widths off whole vectors
// take single elements (40960 x 771: 88 and 111 us against 69 and 95 of 768, measured by whole
// calls).  bf16 rows of 513 to 768 columns use 75 % of their lanes: the gradient at 40960 x 768
// takes 70 us where vectors of four in 64 lanes took 62, with another order of a row's sums than
// the norm alone has.  Rows of more than 8192 columns are two launches (3000 x 10000 fp32 and
// bf16 152 and 244 us).
#include "kf_norm.h"

namespace kf {

hipError_t launch_drop_norm(const DropNormArgs& a, hipStream_t s) {
  return by_types(a.x_dtype, a.y_dtype, [&](auto x, auto y) {
    using X = decltype(x);
    using Y = decltype(y);
    constexpr int VE = 16 / sizeof(X);
    const bool vec = a.d % VE == 0 && vector_rows(a.res, a.ldres, sizeof(X), 16) && vector_rows(a.h, a.ldh, sizeof(X), 16) &&
                     vector_rows(a.in, a.ldin, sizeof(Y), VE * sizeof(Y)) && vector_rows(a.y, a.ldy, sizeof(Y), VE * sizeof(Y)) &&
                     vector_rows(a.gain, 0, 4, 16) && vector_rows(a.shift, 0, 4, 16);
    auto apart = [&] {  // rows that registers do not hold
      const hipError_t e = launch_dropout({a.y_dtype, a.x_dtype, a.rows, a.d, a.in, a.ldin, a.res, a.ldres, a.h, a.ldh, a.drop}, s);
      return e == hipSuccess ? launch_norm(a, s) : e;
    };
    return vec ? launch_norm_rows<X, Y, VE>(a, s, apart) : launch_norm_rows<X, Y, 1>(a, s, apart);
  });
}

hipError_t launch_drop_norm_grad(const DropNormGradArgs& args, hipStream_t s) {
  return by_types(args.x_dtype, args.y_dtype, [&](auto x, auto y) {
    using X = decltype(x);
    using Y = decltype(y);
    constexpr int VE = 16 / sizeof(X);
    DropNormGradArgs a = args;
    const bool sums = a.dgain || a.dshift;
    if (!sums) a.part = nullptr;
    int strips = 0;
    bool joined = false;
    if (a.rows) {
      const bool vec = a.d % VE == 0 && vector_rows(a.x, a.ldx, sizeof(X), 16) && vector_rows(a.dy, a.lddy, sizeof(Y), VE * sizeof(Y)) &&
                       vector_rows(a.dx, a.lddx, sizeof(X), 16) && vector_rows(a.dres, a.dres ? a.lddres : 0, sizeof(X), 16) &&
                       vector_rows(a.din, a.lddin, sizeof(Y), VE * sizeof(Y)) && vector_rows(a.gain, 0, 4, 16);
      auto apart = [&] {
        joined = true;
        const hipError_t e = launch_norm_grad(a, s);
        return e == hipSuccess ? launch_dropout({a.x_dtype, a.y_dtype, a.rows, a.d, a.dx, a.lddx, nullptr, 0, a.din, a.lddin, a.drop}, s) : e;
      };
      const hipError_t e = vec ? launch_norm_grad_rows<X, Y, VE>(a, s, strips, apart)
                               : launch_norm_grad_rows<X, Y, 1>(a, s, strips, apart);
      if (e != hipSuccess) return e;
    }
    return sums && !joined && strips != 1 ? launch_cols_join(a.part, strips, a.d, a.dgain, a.dshift, s) : hipGetLastError();
  });
}

}  // namespace kf
