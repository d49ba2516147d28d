// Residual addition and root-mean-square norm for W workers, with an optional
// 8-bit output, and its backward pass (include/cpdp_layers.h).
#include <type_traits>

#include "cpdp_layers.cuh"

namespace cpdp {
namespace {

struct NormIn {
    const void* p;
    int64_t worker, row;
};

// A row is spread over TPR threads, E elements each, in pieces of V
// neighbours: piece j of thread t starts at element (j * TPR + t) * V. V is 16
// bytes' worth where every row of every array starts at a multiple of that,
// else 1. Rows of up to 128 elements in such pieces take 8 lanes, of up to 1,024
// a warp, longer ones a block.

// The sum over the row's threads, of N values at once. Blocks use two sets of
// partial sums in turn, so one barrier per row is enough.
template <int TPR, int N>
__device__ __forceinline__ void row_sum(float (&v)[N], int turn) {
#pragma unroll
    for (int o = (TPR < 32 ? TPR : 32) / 2; o > 0; o >>= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(~0u, v[k], o);
    if constexpr (TPR > 32) {
        __shared__ float part[2][N][TPR / 32];
        if (threadIdx.x % 32 == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) part[turn][k][threadIdx.x / 32] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = 0.f;
#pragma unroll
            for (int i = 0; i < TPR / 32; ++i) v[k] += part[turn][k][i];
        }
    }
}

template <int TPR>
struct RowThreads {
    static constexpr int block = TPR > 128 ? TPR : 128, rows = block / TPR;
};

// Forward: a row is read once into registers, its squares are summed, and it is
// scaled and stored from there; the weights stay in registers through a block's
// rows. Bound by DRAM where there are rows enough: 4 x 8,192 x 4,096 in bf16 with
// the residual and the 8-bit output take 193 us, 6.3 TB/s; 8 x 3,152 x 384, with 2 or
// 3 rows per warp, 22 us, 3.9; rows off 16 bytes, element by element, 1.9 to 4.3.
template <typename T, int V, int TPR, int E, bool CHECKPOINT>
__global__ void __launch_bounds__(RowThreads<TPR>::block)
norm_forward_kernel(NormIn x, NormIn residual, const float* weight, int64_t weight_worker, int64_t M, int D, float eps, void* y,
                    void* s, int8_t* codes, uint8_t* exponents) {
    layer_begin();
    constexpr int rows = RowThreads<TPR>::rows, J = E / V;
    using Out = std::conditional_t<CHECKPOINT, __nv_bfloat16, T>;
    const int t = threadIdx.x % TPR;
    const int64_t w = blockIdx.y;
    const int blocks = (D + kBlock8 - 1) / kBlock8;
    float wt[E];
#pragma unroll
    for (int k = 0; k < E; ++k) {
        const int d = (k / V * TPR + t) * V + k % V;
        wt[k] = d < D ? weight[w * weight_worker + d] : 0.f;
    }
    int turn = 0;
    // a warp's rows leave the loop together
    const int beside = TPR < 32 ? threadIdx.x % 32 / TPR : 0;
    for (int64_t m = (int64_t)blockIdx.x * rows + threadIdx.x / TPR; m - beside < M; m += (int64_t)gridDim.x * rows, turn ^= 1) {
        const bool there = TPR >= 32 || m < M;
        const T* xr = static_cast<const T*>(x.p) + w * x.worker + m * x.row;
        const T* rr = static_cast<const T*>(residual.p) + w * residual.worker + m * residual.row;
        const int64_t row = w * M + m;
        float v[E];
        {
            Piece<T, V> a[J], b[J];
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int d = (j * TPR + t) * V;
                a[j] = b[j] = Piece<T, V>{};
                if constexpr (V > 1) {
                    if (there && d < D) {
                        a[j].load(xr + d);
                        if (residual.p != nullptr) b[j].load(rr + d);
                    }
                } else {
                    a[j].load(xr + d, there && d < D);
                    b[j].load(rr + d, there && d < D && residual.p != nullptr);
                }
            }
#pragma unroll
            for (int k = 0; k < E; ++k) {
                v[k] = a[k / V].get(k % V);
                // the norm is of the sum as it is stored: what the backward pass reads
                if (residual.p != nullptr) v[k] = to_float(from_float<T>(v[k] + b[k / V].get(k % V)));
            }
        }
        float sum[1] = {0.f};
#pragma unroll
        for (int k = 0; k < E; ++k) sum[0] = fmaf(v[k], v[k], sum[0]);
        if (residual.p != nullptr)
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int d = (j * TPR + t) * V;
                if (there && d < D) store_piece<V>(static_cast<T*>(s) + row * D + d, v + j * V);
            }
        row_sum<TPR>(sum, turn);
        const float k = rsqrtf(sum[0] / D + eps);
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int d = (j * TPR + t) * V;
            float o[V];
#pragma unroll
            for (int e = 0; e < V; ++e) o[e] = v[j * V + e] * k * wt[j * V + e];
            if constexpr (CHECKPOINT) {
                if ((j * TPR + t / 32 * 32) * V >= blocks * kBlock8) break;  // the warp is past the row
                uint32_t top = 0;
#pragma unroll
                for (int e = 0; e < V; ++e) top = max(top, __float_as_uint(d < D ? o[e] : 0.f) & 0x7fffffffu);
                // a block is 32 / V neighbouring threads
                if constexpr (V == 1)
                    top = __reduce_max_sync(~0u, top);
                else
#pragma unroll
                    for (int h = 1; h < kBlock8 / V; h <<= 1) top = max(top, __shfl_xor_sync(~0u, top, h));
                const uint32_t byte = exponent_byte(top);
                const float inverse = inverse_unit_of(byte), unit = unit_of(byte);
                int q[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    q[e] = d < D ? code_of(o[e], inverse) : 0;
                    o[e] = q[e] * unit;
                }
                if (there && d < blocks * kBlock8) {
                    store_codes<V>(codes + row * blocks * kBlock8 + d, q);
                    if (d % kBlock8 == 0) exponents[row * blocks + d / kBlock8] = static_cast<uint8_t>(byte);
                }
            }
            if (there && d < D) store_piece<V>(static_cast<Out*>(y) + row * D + d, o);
        }
    }
}

// Backward. Both sums that dx needs, of s^2 and of dy weight s, are taken in one
// go, so the scale need not be kept from the forward pass. dweight's sums over
// the block's rows stay in registers from row to row; `parts` receives them, one
// row per block. KEEP: the weights stay in registers too (without, 2 x 1,021 x
// 2,731 rows took 98 us instead of 27). 4 x 8,192 x 4,096 in bf16 with the residual
// stream's gradient take 174 us, 6.2 TB/s, dweight's second launch included.
template <typename T, int V, int TPR, int E, bool KEEP>
__global__ void __launch_bounds__(RowThreads<TPR>::block, TPR > 256 ? 1 : TPR > 128 || E == 32 ? 2 : 4)
norm_backward_kernel(NormIn dy, NormIn s, NormIn ds, const float* weight, int64_t weight_worker, int64_t M, int D, float eps,
                     void* dx, float* parts) {
    layer_begin();
    constexpr int rows = RowThreads<TPR>::rows, J = E / V;
    const int t = threadIdx.x % TPR;
    const int64_t w = blockIdx.y;
    const auto weight_at = [&](int k) {
        const int d = (k / V * TPR + t) * V + k % V;
        return d < D ? weight[w * weight_worker + d] : 0.f;
    };
    float wt[KEEP ? E : 1], sums[E];
#pragma unroll
    for (int k = 0; k < E; ++k) {
        if constexpr (KEEP) wt[k] = weight_at(k);
        sums[k] = 0.f;
    }
    int turn = 0;
    Piece<T, V> g[J], r[J], through[J];
    const auto row_of = [&](const NormIn& in, int64_t m) { return static_cast<const T*>(in.p) + w * in.worker + m * in.row; };
    const auto load = [&](int64_t m) {
        const T *gr = row_of(dy, m), *sr = row_of(s, m), *dr = row_of(ds, m);
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int d = (j * TPR + t) * V;
            g[j] = r[j] = through[j] = Piece<T, V>{};
            const bool there = m < M && d < D;
            if constexpr (V > 1) {
                if (there) {
                    g[j].load(gr + d);
                    r[j].load(sr + d);
                    if (KEEP && ds.p != nullptr) through[j].load(dr + d);
                }
            } else {
                g[j].load(gr + d, there);
                r[j].load(sr + d, there);
                if (KEEP) through[j].load(dr + d, there && ds.p != nullptr);
            }
        }
    };
    // the next row is on its way while one is worked on, where it takes few registers (at 4,096 features 213 -> 180 us)
    constexpr bool ahead = V > 1 && sizeof(T) == 2 && KEEP;
    const int64_t first = (int64_t)blockIdx.x * rows + threadIdx.x / TPR, step = (int64_t)gridDim.x * rows;
    if (ahead) load(first);
    const int beside = TPR < 32 ? threadIdx.x % 32 / TPR : 0;  // a warp's rows leave the loop together
    for (int64_t m = first; m - beside < M; m += step, turn ^= 1) {
        if (!ahead) load(m);
        Piece<T, V> g0[J], r0[J], through0[J];
#pragma unroll
        for (int j = 0; j < J; ++j) g0[j] = g[j], r0[j] = r[j], through0[j] = through[j];
        if (ahead) load(m + step);
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < E; ++k) {
            const float v = r0[k / V].get(k % V);
            sum[0] = fmaf(v, v, sum[0]);
            sum[1] = fmaf(g0[k / V].get(k % V) * (KEEP ? wt[KEEP ? k : 0] : weight_at(k)), v, sum[1]);
        }
        row_sum<TPR>(sum, turn);
        // s k^3 mean(dy weight s) as (s k)(k mean(dy weight s) k): k^3 alone leaves float32's range at rows of 1e13, or where
        // eps is 1e-26
        const float k1 = rsqrtf(sum[0] / D + eps), slope = sum[1] / D * k1 * k1;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int d = (j * TPR + t) * V;
            if constexpr (!KEEP && V > 1) {
                if (d < D && ds.p != nullptr) through0[j].load(row_of(ds, m) + d);
            } else if constexpr (!KEEP) {
                through0[j].load(row_of(ds, m) + d, d < D && ds.p != nullptr);
            }
            float o[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int k = j * V + e;
                const float v = r0[j].get(e), gk = g0[j].get(e) * k1;
                o[e] = fmaf(gk, KEEP ? wt[KEEP ? k : 0] : weight_at(k), through0[j].get(e)) - v * k1 * slope;
                sums[k] = fmaf(gk, v, sums[k]);
            }
            if (d < D && (TPR >= 32 || m < M)) store_piece<V>(static_cast<T*>(dx) + (w * M + m) * D + d, o);
        }
    }
    float* part = parts + (w * gridDim.x + blockIdx.x) * D;
    if constexpr (rows > 1) {
        __shared__ float all[rows - 1][E * TPR];
        const int own = threadIdx.x / TPR;
        if (own > 0)
#pragma unroll
            for (int k = 0; k < E; ++k) all[own - 1][k * TPR + t] = sums[k];
        __syncthreads();
        if (own > 0) return;
#pragma unroll
        for (int k = 0; k < E; ++k)
            for (int i = 0; i < rows - 1; ++i) sums[k] += all[i][k * TPR + t];
    }
#pragma unroll
    for (int k = 0; k < E; ++k) {
        const int d = (k / V * TPR + t) * V + k % V;
        if (d < D) part[d] = sums[k];
    }
}

// dweight: the sum of the blocks' parts, in an order fixed by their number. 16
// threads share a column's parts: 5 us for 152 of 4,096 features.
constexpr int kColumns = 32, kLines = 16;
template <typename G>
__global__ void __launch_bounds__(kColumns * kLines)
norm_weight_kernel(const float* parts, int count, int D, G* dweight, int64_t dweight_worker) {
    layer_begin();
    __shared__ float line[kLines][kColumns];
    const int c = threadIdx.x % kColumns, l = threadIdx.x / kColumns, d = blockIdx.x * kColumns + c;
    const int64_t w = blockIdx.y;
    float sum = 0.f;
    if (d < D)
#pragma unroll 4
        for (int i = l; i < count; i += kLines) sum += load_once(parts + (w * count + i) * D + d);
    line[l][c] = sum;
    __syncthreads();
    if (l == 0 && d < D) {
        for (int i = 1; i < kLines; ++i) sum += line[i][c];
        dweight[w * dweight_worker + d] = from_float<G>(sum);
    }
}

// Threads per row and elements per thread for D features: f(TPR, E). At 4,096
// features 256 threads of 16 elements took 193 (forward, 4 x 8,192 rows in bf16
// with 8 bits) and 174 us (backward) where 128 of 32 took 207 and 180.
template <int N>
using Int = std::integral_constant<int, N>;
template <typename F>
cudaError_t with_shape(int D, bool wide, const F& f) {
    if (D <= 128 && wide) return f(Int<8>{}, Int<16>{});
    if (D <= 512) return f(Int<32>{}, Int<16>{});
    if (D <= 1024) return f(Int<32>{}, Int<32>{});
    if (D <= 2048) return f(Int<128>{}, Int<16>{});
    if (D <= 4096) return f(Int<256>{}, Int<16>{});
    if (D <= 8192) return f(Int<512>{}, Int<16>{});
    return f(Int<512>{}, Int<32>{});
}
static_assert(CPDP_NORM_MAX_FEATURES == 512 * 32, "the largest shape");

// Blocks per worker: the rows' blocks, at most `resident` per SM between all
// workers. The backward pass asks for what runs at once. The forward pass asks
// for an SM's 2,048 threads, of which 56 to 163 registers a thread let a fifth to a
// half run at once: a long grid takes 2 to 5 turns, each with the weights anew.
unsigned blocks_for(int W, int64_t M, int rows, int resident) {
    const int64_t all = ceil_div(M, rows), most = ceil_div(int64_t(kSMs) * resident, W);
    return static_cast<unsigned>(all < most ? all : most);
}
int rows_per_block(int D, bool wide) { return D <= 128 && wide ? 16 : D <= 1024 ? 4 : 1; }
// The backward pass's blocks per worker: what its registers let run at once.
// The workspace has a row for each, of rows that are not wide: there are no fewer.
unsigned backward_blocks(int W, int64_t M, int D, bool wide) {
    const int resident = D <= 512 ? 4 : D <= 1024 ? 2 : D <= 2048 ? 4 : D <= 4096 ? 2 : 1;
    return blocks_for(W, M, rows_per_block(D, wide), resident);
}

}  // namespace
}  // namespace cpdp

using namespace cpdp;

static cpdp_status check_norm(int W, int64_t M, int D, cpdp_dtype dtype, float eps) {
    CPDP_TRY(check_sizes(W, M, D));
    if (D > CPDP_NORM_MAX_FEATURES)
        return layer_error(CPDP_EINVAL, "a norm's rows have at most %d features, not %d", CPDP_NORM_MAX_FEATURES, D);
    if (!known_dtype(dtype)) return layer_error(CPDP_EINVAL, "unknown dtype %d", (int)dtype);
    if (!(eps > 0.f) || eps > 3.0e38f) return layer_error(CPDP_EINVAL, "eps=%g must be positive and finite", (double)eps);
    return CPDP_OK;
}

// Whether every row starts at a multiple of 16 bytes and has whole pieces.
static bool in_pieces(const NormIn& a, int64_t size, int D) {
    const int64_t n = 16 / size;
    return aligned_to(a.p, 16) && a.worker % n == 0 && a.row % n == 0 && D % n == 0;
}

cpdp_status cpdp_add_rmsnorm(const void* x, int64_t x_worker, int64_t x_row, const void* residual,
                             int64_t residual_worker, int64_t residual_row, const float* weight, int64_t weight_worker,
                             cpdp_dtype dtype, int W, int64_t M, int D, float eps, void* y, void* s, int8_t* codes,
                             uint8_t* exponents, void* stream) {
    CPDP_TRY(check_norm(W, M, D, dtype, eps));
    const int64_t e = dtype_size(dtype);
    const bool some = M > 0;
    CPDP_TRY(check_array("x", x, some, e, x_worker, x_row));
    CPDP_TRY(check_array("residual", residual, false, e, residual_worker, residual_row));
    CPDP_TRY(check_array("weight", weight, true, 4, weight_worker));
    CPDP_TRY(check_array("y", y, some, codes != nullptr ? 2 : e));
    CPDP_TRY(check_array("s", s, some && residual != nullptr, e));
    if (some && residual == nullptr && s != nullptr) return layer_error(CPDP_EINVAL, "s is x where there is no residual: pass NULL");
    if ((codes == nullptr) != (exponents == nullptr))
        return layer_error(CPDP_EINVAL, "codes and exponents go together: one of them is NULL");
    CPDP_TRY(check_array("codes", codes, false, 16));
    if (!some) return CPDP_OK;
    const NormIn xi{x, x_worker, x_row}, ri{residual, residual_worker, residual_row};
    const bool wide = in_pieces(xi, e, D) && in_pieces(ri, e, D) && aligned_to(y, 16) && aligned_to(s, 16);
    const cudaError_t launched = with_shape(D, wide, [&](auto tpr, auto elements) {
        constexpr int TPR = decltype(tpr)::value, E = decltype(elements)::value;
        const auto go = [&](auto kernel) {
            const dim3 grid(blocks_for(W, M, RowThreads<TPR>::rows, 2048 / RowThreads<TPR>::block), W);
            return launch_layer(kernel, grid, RowThreads<TPR>::block, 0, stream, xi, ri, weight, weight_worker, M, D, eps, y, s, codes, exponents);
        };
        const auto held = [&](auto checkpoint) {
            constexpr bool C = decltype(checkpoint)::value;
            if constexpr (TPR >= 32)
                if (!wide)
                    return dtype == CPDP_F32 ? go(norm_forward_kernel<float, 1, TPR, E, C>) : go(norm_forward_kernel<__nv_bfloat16, 1, TPR, E, C>);
            return dtype == CPDP_F32 ? go(norm_forward_kernel<float, 4, TPR, E, C>) : go(norm_forward_kernel<__nv_bfloat16, 8, TPR, E, C>);
        };
        return codes != nullptr ? held(std::true_type{}) : held(std::false_type{});
    });
    return layer_launched(launched, "cpdp_add_rmsnorm");
}

size_t cpdp_add_rmsnorm_backward_workspace(int W, int64_t M, int D) {
    if (check_norm(W, M, D, CPDP_F32, 1.f) != CPDP_OK) return 0;
    return static_cast<size_t>(W) * backward_blocks(W, M, D, false) * D * 4;
}

cpdp_status cpdp_add_rmsnorm_backward(const void* dy, int64_t dy_worker, int64_t dy_row, const void* s, int64_t s_worker,
                                      int64_t s_row, const void* ds, int64_t ds_worker, int64_t ds_row,
                                      const float* weight, int64_t weight_worker, cpdp_dtype dtype, int W, int64_t M,
                                      int D, float eps, void* dx, void* dweight, int64_t dweight_worker,
                                      cpdp_dtype dweight_dtype, void* workspace, size_t workspace_bytes, void* stream) {
    CPDP_TRY(check_norm(W, M, D, dtype, eps));
    const int64_t e = dtype_size(dtype);
    const bool some = M > 0;
    CPDP_TRY(check_array("dy", dy, some, e, dy_worker, dy_row));
    CPDP_TRY(check_array("s", s, some, e, s_worker, s_row));
    CPDP_TRY(check_array("ds", ds, false, e, ds_worker, ds_row));
    CPDP_TRY(check_array("weight", weight, true, 4, weight_worker));
    CPDP_TRY(check_array("dx", dx, some, e));
    if (!known_dtype(dweight_dtype)) return layer_error(CPDP_EINVAL, "unknown dtype %d of dweight", (int)dweight_dtype);
    CPDP_TRY(check_array("dweight", dweight, true, dtype_size(dweight_dtype), dweight_worker));
    CPDP_TRY(check_apart("dweight", W, dweight_worker, D));
    CPDP_TRY(check_workspace(workspace, workspace_bytes, cpdp_add_rmsnorm_backward_workspace(W, M, D)));
    const NormIn gi{dy, dy_worker, dy_row}, si{s, s_worker, s_row}, di{ds, ds_worker, ds_row};
    float* parts = static_cast<float*>(workspace);
    const bool wide = in_pieces(gi, e, D) && in_pieces(si, e, D) && in_pieces(di, e, D) && aligned_to(dx, 16);
    const unsigned blocks = backward_blocks(W, M, D, wide);
    if (some)
        CPDP_TRY(layer_launched(with_shape(D, wide, [&](auto tpr, auto elements) {
            constexpr int TPR = decltype(tpr)::value, E = decltype(elements)::value;
            constexpr bool K = TPR * E <= 8192;  // longer rows have too few registers for it
            const auto go = [&](auto kernel) {
                return launch_layer(kernel, dim3(blocks, W), RowThreads<TPR>::block, 0, stream, gi, si, di, weight, weight_worker, M, D,
                                    eps, dx, parts);
            };
            if constexpr (TPR >= 32)
                if (!wide)
                    return dtype == CPDP_F32 ? go(norm_backward_kernel<float, 1, TPR, E, K>) : go(norm_backward_kernel<__nv_bfloat16, 1, TPR, E, K>);
            return dtype == CPDP_F32 ? go(norm_backward_kernel<float, 4, TPR, E, K>) : go(norm_backward_kernel<__nv_bfloat16, 8, TPR, E, K>);
        }), "cpdp_add_rmsnorm_backward"));
    const auto sum = [&](auto* out) {
        return launch_layer(norm_weight_kernel<std::remove_pointer_t<decltype(out)>>, dim3(ceil_div(D, kColumns), W), kColumns * kLines, 0,
                            stream, static_cast<const float*>(parts), static_cast<int>(blocks), D, out, dweight_worker);
    };
    return layer_launched(dweight_dtype == CPDP_F32 ? sum(static_cast<float*>(dweight)) : sum(static_cast<__nv_bfloat16*>(dweight)),
                          "cpdp_add_rmsnorm_backward");
}
