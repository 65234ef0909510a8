// Host side of the microscaled formats: the C entry points of include/lords.h, validation, and the choice of kernels.
#include "lords_internal.h"
#include "lords_mx.cuh"

namespace lords {

static bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// The library is ready, and the calling thread's device is the one that it was bound to.
static int ready()
{
    const State &st = state();
    if (!st.initialised) return LORDS_ERR_NOT_INIT;
    int dev = -1;
    LORDS_CUDA_TRY(cudaGetDevice(&dev));
    return dev == st.device ? LORDS_OK : LORDS_ERR_NOT_INIT;
}

static size_t codes_bytes(int rows, int cols) { return (size_t)rows * mx::codes_pitch(cols); }
static size_t scales_bytes(int rows, int cols) { return (size_t)((rows + mx::kTileRows - 1) / mx::kTileRows) * mx::scale_tiles_of(cols) * mx::kTileBytes; }

static bool dims_ok(int64_t rows, int64_t cols) { return rows >= 1 && cols >= 1 && rows <= LORDS_MX_DIM_MAX && cols <= LORDS_MX_DIM_MAX; }

// Whether a product takes the kernel for few tokens, else the one on pairs.
static bool few_tokens(const MxProblem &p, const State &st)
{
    if (st.forced_path == 2) return true;
    if (st.forced_path == 8) return false;
    // Up to 32 tokens the one was never slower, from 513 on the other; between, by their estimates: 128 tokens, 14336 x 4096 9.3 us and 11.3, 4096 x
    // 4096 6.5 and 7.8; 256 tokens, 14336 x 4096 17.8 and 11.8, 4096 x 4096 8.4 and 7.9, 1024 x 4096 6.1 and 7.6.
    return p.M <= 32 || (p.M <= 512 && mxfp4_stream_us(p, st) <= mxfp4_pair_us(p, st));
}

static int product(const MxProblem &p, State &st, cudaStream_t s)
{
    return few_tokens(p, st) ? launch_mxfp4_stream(p, st, s) : launch_mxfp4_pair(p, st, s);
}

static int matmul_common(const uint8_t *xq, const uint8_t *xs, const uint8_t *w, const uint8_t *ws, int M, int m, int n, void *y, int y_f32, void *stream)
{
    if (!xq || !xs || !w || !ws || !y) return LORDS_ERR_NULL;
    if (!dims_ok(M, n) || !dims_ok(m, n)) return LORDS_ERR_SHAPE;
    if (!aligned16(xq) || !aligned16(xs) || !aligned16(w) || !aligned16(ws) || !aligned16(y)) return LORDS_ERR_ALIGN;
    const int rc = ready();
    if (rc != LORDS_OK) return rc;
    State &st = state();
    const MxProblem p = {nullptr, xq, xs, w, ws, M, m, n, y, y_f32};
    st.last_launches = 0;
    return product(p, st, static_cast<cudaStream_t>(stream));
}

static int forward_common(const void *x, const uint8_t *w, const uint8_t *ws, int M, int m, int n, void *y, int y_f32, void *stream)
{
    if (!x || !w || !ws || !y) return LORDS_ERR_NULL;
    if (!dims_ok(M, n) || !dims_ok(m, n)) return LORDS_ERR_SHAPE;
    if (!aligned16(x) || !aligned16(w) || !aligned16(ws) || !aligned16(y)) return LORDS_ERR_ALIGN;
    int rc = ready();
    if (rc != LORDS_OK) return rc;
    State &st = state();
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    st.last_launches = 0;
    MxProblem p = {static_cast<const uint16_t *>(x), nullptr, nullptr, w, ws, M, m, n, y, y_f32};
    auto room = [&](int tokens) { return ((codes_bytes(tokens, n) + 255) & ~(size_t)255) + scales_bytes(tokens, n); };
    // One launch without scratch memory, where the kernel takes x in bf16.
    if (M <= 64 && few_tokens(p, st)) {
        rc = launch_mxfp4_stream(p, st, s);
        if (rc != LORDS_ERR_UNSUPPORTED) return rc;
    }
    // x in 4 bits lies in the workspace between the two launches.  More tokens than it holds: one part after the other, all on the kernel that a call of
    // more than 512 tokens takes.
    int part = M;
    if (room(M) > st.workspace_bytes) {
        for (part = M <= 512 ? 0 : (M - 1) / mx::kTileRows * mx::kTileRows; part > 0 && room(part) > st.workspace_bytes;) {
            const int half = part / 2 / mx::kTileRows * mx::kTileRows;
            part = room(half) > st.workspace_bytes || half == 0 ? half : part - mx::kTileRows;
        }
        if (part == 0) return LORDS_ERR_WORKSPACE;
    }
    int launches = 0;
    for (int t = 0; t < M; t += part) {
        MxProblem now = p;
        now.M = M - t < part ? M - t : part;
        uint8_t *xq = st.workspace, *xs = st.workspace + ((codes_bytes(now.M, n) + 255) & ~(size_t)255);
        rc = launch_mxfp4_quantize(p.x + (size_t)t * n, now.M, n, xq, xs, nullptr, nullptr, s);
        if (rc != LORDS_OK) return rc;
        now.x = nullptr; now.xq = xq; now.xs = xs;
        now.y = static_cast<uint8_t *>(y) + (size_t)t * m * (y_f32 ? 4 : 2);
        rc = part < M ? launch_mxfp4_pair(now, st, s) : product(now, st, s);
        if (rc != LORDS_OK) return rc;
        ++launches;
    }
    st.last_launches = 2 * launches;
    return LORDS_OK;
}

// A gradient call with the values of a checkpoint as the layer's input: they are written to the end of the workspace, which the gradients' launches see
// without that part.  Expanded once, by a launch of its own: inside the gradients' kernel every row of tiles would do it again, 2.5
// instructions a value each time.  scratch(tokens): what the gradients' quickest schedule takes of the rest; call(x, t0, tokens, state) launches
// the gradients of `tokens` tokens from t0 on, added to those of the tokens before if t0 > 0.
//
// Where the workspace does not hold both, the tokens go through it in parts of equal length, multiples of 64 (a stage of the tensor schedule).  8192 tokens,
// 4096 x 14336, rank 32, 256 MB: 1.43 ms in two parts, 1.33 of them the gradients from bf16 activations; 358 with all values at once, which leaves
// no room for the contributions.
constexpr int kPart = 64;
template <class Scratch> static int tokens_of_part(int M, int n, size_t room, Scratch scratch)
{
    auto fits = [&](int tokens) {
        const size_t values = (size_t)tokens * n * 2;
        return values <= room && scratch(tokens) <= ((room - values) & ~(size_t)255);
    };
    if (fits(M)) return M;
    int low = 0, high = (M - 1) / kPart + 1;          // in units of kPart: `low` fits, `high` does not
    while (high - low > 1) {
        const int mid = (low + high) / 2;
        if (fits(mid * kPart)) low = mid;
        else high = mid;
    }
    if (low == 0) {                                   // no contributions: what the values alone leave room for
        const size_t tokens = room / 2 / (size_t)n;
        if (tokens >= (size_t)M) return M;
        low = (int)(tokens / kPart);
    }
    if (low == 0) return 0;
    const int count = (M + low * kPart - 1) / (low * kPart);
    return ((M + count - 1) / count + kPart - 1) / kPart * kPart;
}

template <class Scratch, class Call> static int with_values(const uint8_t *q, const uint8_t *e, int M, int n, cudaStream_t stream, Scratch scratch, Call call)
{
    State &st = state();
    const int part = tokens_of_part(M, n, st.workspace_bytes, scratch);
    if (part == 0) return LORDS_ERR_WORKSPACE;
    State rest = st;
    rest.workspace_bytes = (st.workspace_bytes - (size_t)part * n * 2) & ~(size_t)255;
    uint16_t *x = reinterpret_cast<uint16_t *>(st.workspace + rest.workspace_bytes);
    const size_t q_row = (size_t)mx::blocks_of(n) * mx::kBlock, e_row = (size_t)mx::scale_tiles_of(n) * mx::kTileBlocks;
    int launches = 0;
    for (int t = 0; t < M; t += part) {
        const int tokens = M - t < part ? M - t : part;
        int rc = launch_checkpoint_load(q + (size_t)t * q_row, e + (size_t)t * e_row, tokens, n, x, stream);
        if (rc == LORDS_OK) rc = call(x, t, tokens, rest);
        if (rc != LORDS_OK) return rc;
        launches += rest.last_launches + 1;
    }
    st.last_launches = launches;
    st.last_path = rest.last_path;
    return LORDS_OK;
}

static int check_checkpoint(const uint8_t *q, const uint8_t *e, int rc)
{
    if (!q || !e) return LORDS_ERR_NULL;
    if (rc != LORDS_OK) return rc;
    if (!aligned16(q) || !aligned16(e)) return LORDS_ERR_ALIGN;
    return ready();
}

}  // namespace lords

using namespace lords;

extern "C" {

int64_t lords_mxfp4_codes_bytes(int64_t rows, int64_t cols)
{
    if (!dims_ok(rows, cols)) return LORDS_ERR_SHAPE;
    return (int64_t)codes_bytes((int)rows, (int)cols);
}

int64_t lords_mxfp4_scales_bytes(int64_t rows, int64_t cols)
{
    if (!dims_ok(rows, cols)) return LORDS_ERR_SHAPE;
    return (int64_t)scales_bytes((int)rows, (int)cols);
}

int lords_mxfp4_quantize(const void *v, int rows, int cols, uint8_t *codes, uint8_t *scales, uint8_t *codes_t, uint8_t *scales_t, void *stream)
{
    if (!v || (!codes && !codes_t) || !codes != !scales || !codes_t != !scales_t) return LORDS_ERR_NULL;
    if (!dims_ok(rows, cols)) return LORDS_ERR_SHAPE;
    if (!aligned16(v) || !aligned16(codes) || !aligned16(scales) || !aligned16(codes_t) || !aligned16(scales_t)) return LORDS_ERR_ALIGN;
    int rc = ready();
    if (rc != LORDS_OK) return rc;
    State &st = state();
    rc = launch_mxfp4_quantize(static_cast<const uint16_t *>(v), rows, cols, codes, scales, codes_t, scales_t, static_cast<cudaStream_t>(stream));
    if (rc != LORDS_OK) return rc;
    st.last_launches = 1;
    st.last_path = "mxfp4_quantize";
    return LORDS_OK;
}

int lords_mxfp4_dequantize(const uint8_t *codes, const uint8_t *scales, int rows, int cols, void *v, void *stream)
{
    if (!codes || !scales || !v) return LORDS_ERR_NULL;
    if (!dims_ok(rows, cols)) return LORDS_ERR_SHAPE;
    if (!aligned16(v) || !aligned16(codes) || !aligned16(scales)) return LORDS_ERR_ALIGN;
    int rc = ready();
    if (rc != LORDS_OK) return rc;
    State &st = state();
    rc = launch_mxfp4_dequantize(codes, scales, rows, cols, static_cast<uint16_t *>(v), static_cast<cudaStream_t>(stream));
    if (rc != LORDS_OK) return rc;
    st.last_launches = 1;
    st.last_path = "mxfp4_dequantize";
    return LORDS_OK;
}

int lords_mxfp4_matmul(const uint8_t *x_codes, const uint8_t *x_scales, const uint8_t *w_codes, const uint8_t *w_scales, int M, int m, int n, void *y,
                       void *stream)
{
    return matmul_common(x_codes, x_scales, w_codes, w_scales, M, m, n, y, 0, stream);
}

int lords_mxfp4_matmul_f32(const uint8_t *x_codes, const uint8_t *x_scales, const uint8_t *w_codes, const uint8_t *w_scales, int M, int m, int n, float *y32,
                           void *stream)
{
    return matmul_common(x_codes, x_scales, w_codes, w_scales, M, m, n, y32, 1, stream);
}

int lords_mxfp4_forward(const void *x, const uint8_t *w_codes, const uint8_t *w_scales, int M, int m, int n, void *y, void *stream)
{
    return forward_common(x, w_codes, w_scales, M, m, n, y, 0, stream);
}

int lords_mxfp4_forward_f32(const void *x, const uint8_t *w_codes, const uint8_t *w_scales, int M, int m, int n, float *y32, void *stream)
{
    return forward_common(x, w_codes, w_scales, M, m, n, y32, 1, stream);
}

int64_t lords_checkpoint_bytes(int64_t M, int64_t n)
{
    if (!dims_ok(M, n)) return LORDS_ERR_SHAPE;
    return M * mx::blocks_of((int)n) * mx::kBlock;
}

int64_t lords_checkpoint_scales_bytes(int64_t M, int64_t n)
{
    if (!dims_ok(M, n)) return LORDS_ERR_SHAPE;
    return M * mx::scale_tiles_of((int)n) * mx::kTileBlocks;
}

int lords_checkpoint_store(const void *x, int M, int n, uint8_t *q, uint8_t *e, void *stream)
{
    if (!x || !q || !e) return LORDS_ERR_NULL;
    if (!dims_ok(M, n)) return LORDS_ERR_SHAPE;
    if (!aligned16(x) || !aligned16(q) || !aligned16(e)) return LORDS_ERR_ALIGN;
    int rc = ready();
    if (rc != LORDS_OK) return rc;
    State &st = state();
    rc = launch_checkpoint_store(static_cast<const uint16_t *>(x), M, n, q, e, static_cast<cudaStream_t>(stream));
    if (rc != LORDS_OK) return rc;
    st.last_launches = 1;
    st.last_path = "checkpoint_store";
    return LORDS_OK;
}

int lords_checkpoint_load(const uint8_t *q, const uint8_t *e, int M, int n, void *x, void *stream)
{
    if (!x || !q || !e) return LORDS_ERR_NULL;
    if (!dims_ok(M, n)) return LORDS_ERR_SHAPE;
    if (!aligned16(x) || !aligned16(q) || !aligned16(e)) return LORDS_ERR_ALIGN;
    int rc = ready();
    if (rc != LORDS_OK) return rc;
    State &st = state();
    rc = launch_checkpoint_load(q, e, M, n, static_cast<uint16_t *>(x), static_cast<cudaStream_t>(stream));
    if (rc != LORDS_OK) return rc;
    st.last_launches = 1;
    st.last_path = "checkpoint_load";
    return LORDS_OK;
}

int lords_linear_backward_factors_checkpoint(const void *dy, const uint8_t *q, const uint8_t *e, const uint8_t *Qpacked, const void *B, const void *A,
                                             const float *codebook, int bits, int M, int m, int n, int r, float *dB, float *dA, void *stream)
{
    const int rc = check_checkpoint(q, e, check_backward_factors(dy, q, Qpacked, B, A, codebook, bits, M, m, n, r, dB, dA));
    if (rc != LORDS_OK) return rc;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    auto scratch = [&](int tokens) { return backward_scratch(tokens, m, n, r, dB != nullptr, dA != nullptr, false, state()); };
    return with_values(q, e, M, n, s, scratch, [&](const uint16_t *x, int t0, int tokens, State &st) {
        return launch_backward_factors(static_cast<const uint16_t *>(dy) + (size_t)t0 * m, x, Qpacked, static_cast<const uint16_t *>(B),
                                       static_cast<const uint16_t *>(A), codebook, bits, tokens, m, n, r, dB, dA, t0 > 0, st, s);
    });
}

int lords_linear_backward_qat_checkpoint(const void *dy, const uint8_t *q, const uint8_t *e, const void *W, const uint8_t *Qpacked, const void *B,
                                         const void *A, const float *codebook, int bits, int M, int m, int n, int r, float *dW, float *dB, float *dA,
                                         void *stream)
{
    const int rc = check_checkpoint(q, e, check_backward_qat(dy, q, W, Qpacked, B, A, codebook, bits, M, m, n, r, dW, dB, dA));
    if (rc != LORDS_OK) return rc;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    auto scratch = [&](int tokens) { return backward_scratch(tokens, m, n, r, dB != nullptr, dA != nullptr, true, state()); };
    return with_values(q, e, M, n, s, scratch, [&](const uint16_t *x, int t0, int tokens, State &st) {
        return launch_backward_qat(static_cast<const uint16_t *>(dy) + (size_t)t0 * m, x, static_cast<const uint16_t *>(W), Qpacked,
                                   static_cast<const uint16_t *>(B), static_cast<const uint16_t *>(A), codebook, bits, tokens, m, n, r, dW, dB, dA, t0 > 0, st, s);
    });
}

}  // extern "C"
