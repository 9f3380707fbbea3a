/* Host build of the rules that choose the kernels of 4-bit products and of the gated delta rule (plain C). */
#include "q8_route.h"

int q8x_w4_route(int rows, int cols, int n, int group, int apart) { return q8_w4_route(rows, cols, n, group, apart); }

int q8x_delta_segment(int L, int S, int hv, int dk, int dv) { return q8_delta_segment(L, S, hv, dk, dv); }
