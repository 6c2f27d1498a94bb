// Which sizes the calls around an attention take: every launch is recorded and none is run, so that a call may describe more memory
// than there is.
#include <cstdio>

#include "layer_ops.h"
#include "plan.h"

namespace svd {
int g_launches = 0;
RopeLaunch g_rope;
hipError_t launch_norm_forward(const NormLaunch&, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_norm_backward(const NormLaunch&, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_rope_table(const svd_rope_desc&, double, const double[3], const double[3], float*, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_rope_forward(const RopeLaunch& p, hipStream_t) { return g_rope = p, ++g_launches, hipSuccess; }
hipError_t launch_rope_backward(const RopeLaunch& p, hipStream_t) { return g_rope = p, ++g_launches, hipSuccess; }
hipError_t launch_quantise_rows(const QuantLaunch&, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_quantise_columns(const QuantLaunch&, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_blockscale_matmul(const MatmulLaunch&, hipStream_t) { return ++g_launches, hipSuccess; }
}  // namespace svd

namespace {
int g_failures = 0;
void* at(uintptr_t a) { return reinterpret_cast<void*>(a << 20); }   // nobody reads it

void rope(int want, const char* what, svd_tensor_desc d) {
  svd_rope_desc r{0, 1, 1, 1, 0, 0, 0, SVD_ROPE_ADJACENT, 0, 0};
  const svd_rope_tensor t{at(1), &d, at(2), &d, nullptr, nullptr};
  const svd_rope_grad g{at(1), &d, at(2), &d, at(3), &d, nullptr, nullptr, nullptr};
  for (int norm : {SVD_NORM_NONE, SVD_NORM_RMS})
    for (int backward = 0; backward < 2; ++backward) {
      const int before = svd::g_launches;
      const int st = backward ? svd_rope_backward(&r, nullptr, norm, 1e-6f, &g, 1, nullptr, 0, nullptr)
                              : svd_rope_forward(&r, nullptr, norm, 1e-6f, &t, 1, nullptr);
      const bool same = st != SVD_OK || (svd::g_rope.L == d.L && svd::g_rope.t[0].o_l == d.stride_l && svd::g_rope.t[0].o_h == d.stride_h);
      if (st == want && svd::g_launches - before == (want == SVD_OK) && same) continue;
      std::fprintf(stderr, "%s, backward %d, norm %d: status %d, expected %d\n", what, backward, norm, st, want);
      ++g_failures;
    }
}
}  // namespace

int main() {
  const int64_t joint = 3 * 40 * 128;   // a row of a joint projection of q, k and v
  rope(SVD_OK, "a head's rows of 4 GiB", {1, 40, 139811, 128, 139811 * joint, 128, joint});
  rope(SVD_OK, "entries of 4 GiB, heads inside", {2, 24, 1 << 18, 128, (int64_t)1 << 34, 128, 24 * 128});
  rope(SVD_OK, "rows 16 MiB apart", {1, 2, 100, 64, 1 << 30, 64, 1 << 23});
  rope(SVD_OK, "2^24 rows", {1, 1, 1 << 24, 64, (int64_t)1 << 30, 64, 64});
  rope(SVD_OK, "the most rows", {1, 1, 1 << 27, 128, (int64_t)1 << 34, 128, 128});
  rope(SVD_ERR_UNSUPPORTED, "one more", {1, 1, (1 << 27) + 1, 128, (int64_t)1 << 35, 128, 128});
  rope(SVD_ERR_UNSUPPORTED, "rows of all entries", {16, 1, 1 << 27, 64, 64, 64, 64});
  rope(SVD_ERR_SHAPE, "a stride past 2^40", {1, 2, 100, 64, 64, ((int64_t)1 << 40) + 8, 64});
  rope(SVD_OK, "an axis of length 1 needs no stride", {1, 1, 1, 64, (int64_t)1 << 62, (int64_t)1 << 62, (int64_t)1 << 62});
  rope(SVD_ERR_SHAPE, "rows over one another", {1, 1, 100, 64, 6400, 6400, 56});
  rope(SVD_ERR_SHAPE, "heads over one another", {1, 2, 100, 64, 6400, 0, 128});
  rope(SVD_ERR_SHAPE, "more heads than a launch has", {1, 65536, 1, 64, 64 * 65536, 64, 64 * 65536});
  rope(SVD_ERR_SHAPE, "heads of 32", {1, 1, 1, 32, 64, 64, 64});
  rope(SVD_ERR_ALIGN, "rows of 8 bytes more", {1, 1, 9, 64, 68 * 9, 68, 68});
  if (!g_failures) std::printf("ok\n");
  return g_failures != 0;
}
