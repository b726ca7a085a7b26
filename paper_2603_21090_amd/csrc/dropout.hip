// Dropout with the residual's addition, its mask computed where it is used and stored nowhere:
//
//   y = residual + (u >= border ? x 65536 / (65536 - border) : 0),   u: 16 bits of Philox 4x32 with ten rounds (Salmon, Moraes, Dror and Shaw, "Parallel
//   random numbers: as easy as 1, 2, 3", 2011), key = seed, counter = group | site << 48, step; a group is eight neighbouring numbers of a row
//
// One call of the generator gives eight numbers of 16 bits: 32 bits a number would take two calls for the 16 bytes of a lane's piece, and the
// generator, not memory, would be what bounds it.  A chance of 16 bits is off by 2^-17 at most, and what is kept is scaled by the chance in effect, so that the
// mean stays the input's.  The gradient is the same call on dy.
#include "operators.h"
#include "tile_ops.h"

namespace stgn {
namespace drop {

struct Words { uint32_t w[4]; };
__device__ inline Words philox(uint64_t group, uint32_t site, uint64_t seed, uint64_t step) {
  uint32_t a = (uint32_t)group, b = (uint32_t)(group >> 32) | site << 16, c = (uint32_t)step, d = (uint32_t)(step >> 32);
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t p = (uint64_t)a * 0xD2511F53u, q = (uint64_t)c * 0xCD9E8D57u;
    a = (uint32_t)(q >> 32) ^ b ^ k0;
    b = (uint32_t)q;
    c = (uint32_t)(p >> 32) ^ d ^ k1;
    d = (uint32_t)p;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return {{a, b, c, d}};
}

// eight neighbouring numbers of a row from column c on, those that it has; nothing beside them is touched, as y may lie where x or the residual does
template <class T>
__device__ inline void load8(const T* row, int c, int width, floatx4& u, floatx4& v) {
  if constexpr (sizeof(T) == 2) {
    u = v = floatx4{0.f, 0.f, 0.f, 0.f};
    add8(row, c, width, u, v);
  } else {
    u = load4(row, c, width);
    v = c + 4 < width ? load4(row, c + 4, width) : floatx4{0.f, 0.f, 0.f, 0.f};
  }
}
template <class T>
__device__ inline void save8(T* row, int c, int width, const floatx4& u, const floatx4& v) {
  if constexpr (sizeof(T) == 2) {
    store8(row, c, width, u, v);
  } else {
    store4(row, c, width, u);
    if (c + 4 < width) store4(row, c + 4, width, v);
  }
}

// a group a thread, the generator while the group is on its way
template <class T>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a) {
  const uint64_t seed = a.rng[0], step = a.rng[1];
  const uint32_t groups = (uint32_t)(a.width + 7) / 8;
  const uint64_t total = (uint64_t)a.rows * groups;
  const bool small = total >> 32 == 0;
  for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (uint64_t)gridDim.x * 256) {
    const int64_t row = small ? (uint32_t)i / groups : i / groups;
    const int c = (int)(uint32_t)(i - row * groups) * 8;
    floatx4 u, v, s = {0.f, 0.f, 0.f, 0.f}, t = s;
    load8(static_cast<const T*>(a.x) + row * a.ld_x, c, a.width, u, v);
    if (a.residual) load8(static_cast<const T*>(a.residual) + row * a.ld_res, c, a.width, s, t);
    __builtin_amdgcn_sched_barrier(0);
    const Words r = philox(i, a.site, seed, step);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      u[j] = (r.w[j / 2] >> j % 2 * 16 & 0xFFFFu) >= a.border ? u[j] * a.scale : 0.f;
      v[j] = (r.w[2 + j / 2] >> j % 2 * 16 & 0xFFFFu) >= a.border ? v[j] * a.scale : 0.f;
    }
    if (a.residual) {
      u += s;
      v += t;
    }
    save8(static_cast<T*>(a.y) + row * a.ld_y, c, a.width, u, v);
  }
}

template <class T>
hipError_t run(const DropoutArgs& a, hipStream_t s) {
  const int64_t n = ((int64_t)a.rows * ((a.width + 7) / 8) + 255) / 256;
  return launch(dropout_kernel<T>, n < (1 << 20) ? n : 1 << 20, 256, s, a);
}

}  // namespace drop

hipError_t dropout_f32(const DropoutArgs& a, hipStream_t s) { return drop::run<float>(a, s); }
hipError_t dropout_bf16(const DropoutArgs& a, hipStream_t s) { return drop::run<__bf16>(a, s); }
hipError_t dropout_f16(const DropoutArgs& a, hipStream_t s) { return drop::run<_Float16>(a, s); }
}  // namespace stgn
