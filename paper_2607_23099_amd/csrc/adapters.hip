// damoe_adapters: y = add + s B (A x) with a pair (A, B) for each segment of rows.
#include "adapters.h"

using namespace damoe;

extern "C" {

size_t damoe_adapters_workspace_size(int32_t T_max, int32_t L, int32_t r, int32_t K, int32_t N) {
  if (check(T_max, L, r, K, N, DAMOE_F32, DAMOE_F32, DAMOE_F32)) return 0;
  const int32_t rp = padded_rank(r);
  return 256 + std::max(most_parts(T_max, K, rp), ready_bytes(T_max, rp) + kSpare);
}

damoe_status damoe_adapters(const void* x, int32_t xdtype, int64_t ldx, const int32_t* perm, const int32_t* offsets, int32_t T,
                            int32_t L, const void* a, const void* b, int32_t wdtype, int32_t r, int32_t K, int32_t N,
                            const float* scale, const void* add, int64_t ld_add, void* y, int32_t ydtype, int64_t ldy, float* u,
                            void* ws, size_t ws_bytes, hipStream_t stream) {
  if (const damoe_status s = check(T, L, r, K, N, xdtype, wdtype, ydtype)) return s;
  if (T == 0) return DAMOE_OK;
  if (!matrix_ok(x, ldx, K, xdtype) || !matrix_ok(y, ldy, N, ydtype) || (add && !matrix_ok(add, ld_add, N, ydtype)) ||
      (add == y && ld_add != ldy) || !offsets || !a || !b || !aligned(a, wdtype) || !aligned(b, wdtype) || !aligned(perm, DAMOE_F32) ||
      !aligned(offsets, DAMOE_F32) || !aligned(scale, DAMOE_F32) || !aligned(u, DAMOE_F32) || !ws ||
      reinterpret_cast<uintptr_t>(ws) % 16)
    return DAMOE_ERR_INVALID_ARG;
  const int32_t rp = padded_rank(r);
  const DownPlan d = down_plan(T, K);
  const bool join = T < kManyRows;
  if (ws_bytes < (join ? part_bytes(d, T, rp) : ready_bytes(T, rp) + kSpare)) return DAMOE_ERR_WORKSPACE;
  if (adapters_few(T, L, rp, K, N, ydtype, wdtype)) {
    const DownArgs da{x, ldx, a, perm, offsets, nullptr, nullptr, nullptr, u, L, T, K, r, rp, 0, 0};
    const UpArgs ua{nullptr, nullptr, 1, nullptr, b, scale, perm, offsets, add, ld_add, y, ldy, nullptr, L, T, N, r, rp, 0};
    return adapters_in_one(da, ua, xdtype, wdtype, ydtype, stream) == hipSuccess ? DAMOE_OK : DAMOE_ERR_HIP;
  }
  float* part = join ? static_cast<float*>(ws) : nullptr;
  const DownArgs da{x, ldx, a, perm, offsets, nullptr, part, ws, u, L, T, K, r, rp, 0, 0};
  // `up` takes thirds where the weights are bf16, `down` leaves them there too.
  if (down<false>(da, d, xdtype, wdtype, stream) != hipSuccess) return DAMOE_ERR_HIP;
  const UpArgs ua{part, ws, d.parts, u, b, scale, perm, offsets, add, ld_add, y, ldy, static_cast<char*>(ws) + ready_bytes(T, rp),
                  L, T, N, r, rp, 0};
  const hipError_t e = join ? up<false, true>(ua, ydtype, wdtype, stream) : up<false, false>(ua, ydtype, wdtype, stream);
  return e == hipSuccess ? DAMOE_OK : DAMOE_ERR_HIP;
}

}  // extern "C"
