// csrc/k_q8_form.h without a device: which kernel and tile a product's sizes choose.
#include "k_q8_form.h"

extern "C" __attribute__((visibility("default"))) void form(int m, int k, int n, int act, int f32, int codes, int residual, int bias, int n_cu, int *out)
{
    static char something;
    aif::Q8LinearCall c{};
    c.m = m, c.k = k, c.n = n, c.act = act, c.f32 = f32;
    c.out = codes ? nullptr : &something;
    c.residual = residual ? &something : nullptr;
    c.bias = bias ? &something : nullptr;
    const aif::Q8Form f = aif::q8_form(c, n_cu);
    out[0] = f.few, out[1] = f.rows, out[2] = f.cols;
}
