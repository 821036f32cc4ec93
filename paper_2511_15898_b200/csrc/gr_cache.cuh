// The 4-bit paged cache: where an octet (eight tokens of a head) keeps what.  With J = dim / 32 groups of 32 dims,
//   keys' codes    [8 tokens][4][J] words     word (t, j) of a token: dims 32 j + 8 t .. + 7, the first in its lowest bits
//   keys' scales   [8 tokens][J] fp16
//   values' codes  [8][4 pairs][J][2 tokens] half words    half word (g, pair, j, token): dims 32 j + 4 g .. + 3
//   values' scales [4 pairs][J][2 tokens] fp16
// so that lane (g, t) of a warp finds its share of the operands of a 16 x 8 x 16 product, of a tile whose first eight rows (keys:
// tokens, values: depth) are this octet's, in J consecutive words at place 4 g + t, codes and scales alike; a token's bytes are its own.
#pragma once
#include "gr_common.cuh"

namespace gr {

__host__ __device__ constexpr int octet_bytes(int dim) { return 9 * dim; }
__host__ __device__ constexpr int octet_kscale(int dim) { return 4 * dim; }
__host__ __device__ constexpr int octet_vcode(int dim) { return 4 * dim + dim / 2; }
__host__ __device__ constexpr int octet_vscale(int dim) { return 8 * dim + dim / 2; }

template <typename T> __device__ __forceinline__ float to_f32(T x);
template <> __device__ __forceinline__ float to_f32(float x) { return x; }
template <> __device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32(float x) { return __float2half_rn(x); }

// N elements of a type as one access, on an address aligned to all of them
template <typename T, int N> struct __align__(sizeof(T) * N) Pack { T x[N]; };

__host__ inline bool known_type(int t) { return t == GR_F32 || t == GR_BF16 || t == GR_F16; }
__host__ inline int type_size(int t) { return t == GR_F32 ? 4 : 2; }

// What a layout has to satisfy (`keys` aligned as its format asks for); GR_OK or the GR_E_* code.
int check_cache(const void* keys, const void* values, const gr_cache_layout* layout);

}  // namespace gr
