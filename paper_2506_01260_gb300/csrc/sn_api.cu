// sn_api.cu — the C ABI (include/sn.h): argument validation, basis handles,
// the launch of each call's kernels (bf16: tcgen05 tensor-core kernels; fp32:
// CUDA-core kernels), the wire copies and the asynchronous error word.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdlib>
#include <initializer_list>
#include <new>
#include <vector>

#include "sn_internal.cuh"

namespace sn {
static std::atomic<uint64_t> g_launches{0};
void count_launch(int n) { g_launches.fetch_add((uint64_t)n, std::memory_order_relaxed); }
}  // namespace sn

namespace {

constexpr int kMaxK = 128;
constexpr int64_t kMaxRows = (int64_t)1 << 31;   // TMA coordinates are 32-bit

bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p % a) == 0; }

bool overlap(const void *a, size_t na, const void *b, size_t nb)
{
    const uintptr_t pa = (uintptr_t)a, pb = (uintptr_t)b;
    return pa < pb + nb && pb < pa + na;
}

size_t esize(sn_dtype dt) { return dt == SN_BF16 ? 2 : 4; }

sn_status cuda_status(cudaError_t e) { return e == cudaSuccess ? SN_OK : SN_ERR_CUDA; }

// Kernels dereference every tensor pointer, so each must be device memory of
// the current device or managed memory; host memory (pageable or pinned) is
// refused here instead of faulting in a kernel.  Null pointers are left to the
// callers' own checks.
bool on_device(std::initializer_list<const void *> ptrs)
{
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess)
        return false;
    for (const void *p : ptrs) {
        if (!p)
            continue;
        cudaPointerAttributes a;
        if (cudaPointerGetAttributes(&a, p) != cudaSuccess) {
            (void)cudaGetLastError();
            return false;
        }
        if (a.type == cudaMemoryTypeManaged)
            continue;
        if (a.type != cudaMemoryTypeDevice || a.device != dev)
            return false;
    }
    return true;
}

// Common checks of a basis handle and dtype; the handle must live on the
// current device.
sn_status check_basis(sn_basis_t b, sn_dtype dt)
{
    if (!b || (dt != SN_BF16 && dt != SN_F32))
        return SN_ERR_INVALID_ARG;
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess)
        return SN_ERR_CUDA;
    return dev == b->device ? SN_OK : SN_ERR_INVALID_ARG;
}

// Checks shared by the forward (embedding) calls.
sn_status check_fwd(sn_basis_t b, sn_dtype dt, const void *in, const int32_t *ids,
                    const int32_t *pos, int64_t T, int32_t seq_len, const void *tok,
                    int64_t vocab, const void *pe, const void *out, size_t in_row,
                    size_t out_row)
{
    sn_status st = check_basis(b, dt);
    if (st != SN_OK)
        return st;
    if (T < 0 || T >= kMaxRows || seq_len <= 0 || vocab <= 0 || vocab >= kMaxRows)
        return SN_ERR_INVALID_ARG;
    if (T == 0)
        return SN_OK;
    if (!in || !ids || !tok || !out)
        return SN_ERR_INVALID_ARG;
    if (!aligned(in, 16) || !aligned(tok, 16) || !aligned(out, 16) || (pe && !aligned(pe, 16)) ||
        !aligned(ids, 4) || (pos && !aligned(pos, 4)))
        return SN_ERR_ALIGNMENT;
    const size_t es = esize(dt);
    if (overlap(in, (size_t)T * in_row * es, out, (size_t)T * out_row * es))
        return SN_ERR_INVALID_ARG;
    return on_device({in, ids, pos, tok, pe, out}) ? SN_OK : SN_ERR_INVALID_ARG;
}

}  // namespace

extern "C" {

const char *sn_status_string(sn_status s)
{
    switch (s) {
    case SN_OK: return "SN_OK";
    case SN_ERR_INVALID_ARG: return "SN_ERR_INVALID_ARG";
    case SN_ERR_ALIGNMENT: return "SN_ERR_ALIGNMENT";
    case SN_ERR_UNSUPPORTED: return "SN_ERR_UNSUPPORTED";
    case SN_ERR_BAD_ID: return "SN_ERR_BAD_ID";
    case SN_ERR_TIMEOUT: return "SN_ERR_TIMEOUT";
    case SN_ERR_CUDA: return "SN_ERR_CUDA";
    case SN_ERR_NUMERIC: return "SN_ERR_NUMERIC";
    }
    return "SN_ERR_UNKNOWN";
}

uint64_t sn_launch_count(void) { return sn::g_launches.load(std::memory_order_relaxed); }

sn_status sn_basis_create(const float *U, int32_t d, int32_t k, sn_basis_t *out,
                          sn_stream_t stream)
{
    if (!U || !out || d < 16 || d % 8 != 0 || k < 1 || k > d || k > kMaxK)
        return SN_ERR_INVALID_ARG;
    if (!aligned(U, 16))
        return SN_ERR_ALIGNMENT;
    if (!on_device({U}))
        return SN_ERR_INVALID_ARG;
    sn_basis *b = new (std::nothrow) sn_basis();
    if (!b)
        return SN_ERR_CUDA;
    if (cudaGetDevice(&b->device) != cudaSuccess) {
        delete b;
        return SN_ERR_CUDA;
    }
    b->d = d;
    b->k = k;
    b->n_pad = (k + 15) / 16 * 16;
    b->k64 = (k + 63) / 64 * 64;
    b->kp = sn::simt_padded_columns(k);
    cudaError_t e = cudaDeviceGetAttribute(&b->tail_cap, cudaDevAttrMultiProcessorCount, b->device);
    // one allocation, every buffer on a 256-byte boundary of it
    const size_t dk = sizeof(float) * (size_t)d * k;
    const size_t tail = sizeof(float) * (size_t)b->tail_cap * 128 * b->n_pad;
    const size_t bytes[8] = {dk, dk, sizeof(float) * (size_t)((d + 31) / 32 * 32) * b->kp,
                             sizeof(__nv_bfloat16) * (size_t)b->n_pad * d,
                             sizeof(__nv_bfloat16) * (size_t)d * b->k64, sizeof(unsigned int), tail,
                             tail};
    size_t at[8], total = 0;
    for (int i = 0; i < 8; ++i) {
        at[i] = total;
        total += (bytes[i] + 255) & ~(size_t)255;
    }
    if (e == cudaSuccess) e = cudaMalloc(&b->mem, total);
    if (e == cudaSuccess) {
        char *m = (char *)b->mem;
        b->u32 = (float *)(m + at[0]);
        b->u32t = (float *)(m + at[1]);
        b->u32p = (float *)(m + at[2]);
        b->ut16 = (__nv_bfloat16 *)(m + at[3]);
        b->up16 = (__nv_bfloat16 *)(m + at[4]);
        b->err = (unsigned int *)(m + at[5]);
        b->tail[0] = (float *)(m + at[6]);
        b->tail[1] = (float *)(m + at[7]);
    }
    if (e == cudaSuccess) e = cudaMemsetAsync(b->err, 0, sizeof(unsigned int), stream);
    if (e == cudaSuccess) e = sn::prepare_basis(*b, U, stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
    if (e != cudaSuccess) {
        sn_basis_destroy(b);
        return SN_ERR_CUDA;
    }
    *out = b;
    return SN_OK;
}

sn_status sn_basis_destroy(sn_basis_t b)
{
    if (!b)
        return SN_OK;
    const cudaError_t e = cudaFree(b->mem);
    delete b;
    return cuda_status(e);
}

sn_status sn_basis_shape(sn_basis_t b, int32_t *d, int32_t *k)
{
    if (!b)
        return SN_ERR_INVALID_ARG;
    if (d) *d = b->d;
    if (k) *k = b->k;
    return SN_OK;
}

sn_status sn_compress_fwd(sn_basis_t b, sn_dtype dt, const void *X, const int32_t *ids,
                          const int32_t *pos, int64_t T, int32_t seq_len, const void *tok,
                          int64_t vocab, const void *pe, void *C, sn_stream_t stream)
{
    sn_status st = check_fwd(b, dt, X, ids, pos, T, seq_len, tok, vocab, pe, C, b ? b->d : 0,
                             b ? b->k : 0);
    if (st != SN_OK || T == 0)
        return st;
    cudaStream_t s = (cudaStream_t)stream;
    if (dt == SN_F32)
        return cuda_status(sn::simt_compress(*b, (const float *)X, ids, pos, T, seq_len,
                                             (const float *)tok, vocab, (const float *)pe,
                                             (float *)C, true, s));
    sn::TcArgs a{(const __nv_bfloat16 *)X, ids, pos, (const __nv_bfloat16 *)tok,
                 (const __nv_bfloat16 *)pe, (__nv_bfloat16 *)C, T, vocab, seq_len, true};
    return cuda_status(sn::tc_compress(*b, a, s));
}

sn_status sn_decompress_fwd(sn_basis_t b, sn_dtype dt, const void *C, const int32_t *ids,
                            const int32_t *pos, int64_t T, int32_t seq_len, const void *tok,
                            int64_t vocab, const void *pe, void *X, sn_stream_t stream)
{
    sn_status st = check_fwd(b, dt, C, ids, pos, T, seq_len, tok, vocab, pe, X, b ? b->k : 0,
                             b ? b->d : 0);
    if (st != SN_OK || T == 0)
        return st;
    cudaStream_t s = (cudaStream_t)stream;
    if (dt == SN_F32)
        return cuda_status(sn::simt_decompress(*b, (const float *)C, ids, pos, T, seq_len,
                                               (const float *)tok, vocab,
                                               (const float *)pe, (float *)X, true, s));
    sn::TcArgs a{nullptr, ids, pos, (const __nv_bfloat16 *)tok, (const __nv_bfloat16 *)pe,
                 (__nv_bfloat16 *)C, T, vocab, seq_len, true};
    return cuda_status(sn::tc_decompress(*b, a, (__nv_bfloat16 *)X, s));
}

sn_status sn_compress_bwd(sn_basis_t b, sn_dtype dt, const void *G, int64_t T, void *C,
                          sn_stream_t stream)
{
    sn_status st = check_basis(b, dt);
    if (st != SN_OK)
        return st;
    if (T < 0 || T >= kMaxRows)
        return SN_ERR_INVALID_ARG;
    if (T == 0)
        return SN_OK;
    if (!G || !C)
        return SN_ERR_INVALID_ARG;
    if (!aligned(G, 16) || !aligned(C, 16))
        return SN_ERR_ALIGNMENT;
    const size_t es = esize(dt);
    if (overlap(G, (size_t)T * b->d * es, C, (size_t)T * b->k * es) || !on_device({G, C}))
        return SN_ERR_INVALID_ARG;
    cudaStream_t s = (cudaStream_t)stream;
    if (dt == SN_F32)
        return cuda_status(sn::simt_compress(*b, (const float *)G, nullptr, nullptr, T, 1,
                                             nullptr, 1, nullptr, (float *)C, false, s));
    sn::TcArgs a{(const __nv_bfloat16 *)G, nullptr, nullptr, nullptr, nullptr,
                 (__nv_bfloat16 *)C, T, 1, 1, false};
    return cuda_status(sn::tc_compress(*b, a, s));
}

sn_status sn_decompress_bwd(sn_basis_t b, sn_dtype dt, const void *C, int64_t T, void *G,
                            sn_stream_t stream)
{
    sn_status st = check_basis(b, dt);
    if (st != SN_OK)
        return st;
    if (T < 0 || T >= kMaxRows)
        return SN_ERR_INVALID_ARG;
    if (T == 0)
        return SN_OK;
    if (!G || !C)
        return SN_ERR_INVALID_ARG;
    if (!aligned(G, 16) || !aligned(C, 16))
        return SN_ERR_ALIGNMENT;
    const size_t es = esize(dt);
    if (overlap(G, (size_t)T * b->d * es, C, (size_t)T * b->k * es) || !on_device({G, C}))
        return SN_ERR_INVALID_ARG;
    cudaStream_t s = (cudaStream_t)stream;
    if (dt == SN_F32)
        return cuda_status(sn::simt_decompress(*b, (const float *)C, nullptr, nullptr, T,
                                               1, nullptr, 1, nullptr, (float *)G, false,
                                               s));
    sn::TcArgs a{nullptr, nullptr, nullptr, nullptr, nullptr, (__nv_bfloat16 *)C, T, 1, 1,
                 false};
    return cuda_status(sn::tc_decompress(*b, a, (__nv_bfloat16 *)G, s));
}

sn_status sn_project_weight_workspace(sn_basis_t b, sn_dtype dt, int64_t cols, size_t *bytes)
{
    if (!b || !bytes || cols < 0 || (dt != SN_BF16 && dt != SN_F32))
        return SN_ERR_INVALID_ARG;
    if (dt == SN_F32) {
        *bytes = sizeof(float) * (size_t)b->k * (size_t)cols;
        return SN_OK;
    }
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev != b->device)
        return SN_ERR_INVALID_ARG;
    *bytes = sn::tc_project_workspace(*b, cols);
    return SN_OK;
}

sn_status sn_project_weight(sn_basis_t b, sn_dtype dt, const void *W, int64_t rows,
                            int64_t cols, int64_t ld, void *W_out, void *ws, size_t ws_bytes,
                            sn_stream_t stream)
{
    sn_status st = check_basis(b, dt);
    if (st != SN_OK)
        return st;
    if (rows != b->d || cols < 0 || ld < cols || cols >= kMaxRows || ld >= kMaxRows)
        return SN_ERR_INVALID_ARG;
    if (cols == 0)
        return SN_OK;
    if (!W || !W_out || !ws)
        return SN_ERR_INVALID_ARG;
    const size_t es = esize(dt);
    if (!aligned(W, 16) || !aligned(W_out, 16) || !aligned(ws, 16) || (ld * es) % 16 != 0)
        return SN_ERR_ALIGNMENT;
    size_t need = 0;
    sn_project_weight_workspace(b, dt, cols, &need);
    if (ws_bytes < need)
        return SN_ERR_INVALID_ARG;
    const size_t wbytes = ((size_t)(rows - 1) * ld + cols) * es;
    if (W != W_out && overlap(W, wbytes, W_out, wbytes))
        return SN_ERR_INVALID_ARG;
    if (overlap(ws, need, W, wbytes) || overlap(ws, need, W_out, wbytes) ||
        !on_device({W, W_out, ws}))
        return SN_ERR_INVALID_ARG;
    cudaStream_t s = (cudaStream_t)stream;
    if (dt == SN_F32)
        return cuda_status(sn::simt_project(*b, (const float *)W, cols, ld, (float *)W_out,
                                            (float *)ws, s));
    return cuda_status(sn::tc_project(*b, (const __nv_bfloat16 *)W, cols, ld,
                                      (__nv_bfloat16 *)W_out, ws, s));
}

sn_status sn_project_tables(sn_basis_t b, sn_dtype dt, const void *tok, int64_t vocab,
                            const void *pe, int32_t seq_len, float *TU, float *PU,
                            sn_stream_t stream)
{
    sn_status st = check_basis(b, dt);
    if (st != SN_OK)
        return st;
    if (dt != SN_BF16)
        return SN_ERR_UNSUPPORTED;
    if (vocab <= 0 || vocab >= kMaxRows || !tok || !TU || (pe == nullptr) != (PU == nullptr) ||
        (pe && (seq_len <= 0 || seq_len >= kMaxRows)))
        return SN_ERR_INVALID_ARG;
    if (!aligned(tok, 16) || !aligned(TU, 16) || (pe && (!aligned(pe, 16) || !aligned(PU, 16))))
        return SN_ERR_ALIGNMENT;
    if (overlap(tok, (size_t)vocab * b->d * 2, TU, (size_t)vocab * b->k * 4) ||
        (pe && (overlap(pe, (size_t)seq_len * b->d * 2, PU, (size_t)seq_len * b->k * 4) ||
                overlap(TU, (size_t)vocab * b->k * 4, PU, (size_t)seq_len * b->k * 4))) ||
        !on_device({tok, pe, TU, PU}))
        return SN_ERR_INVALID_ARG;
    cudaStream_t s = (cudaStream_t)stream;
    cudaError_t e = sn::tc_contract_f32(*b, (const __nv_bfloat16 *)tok, vocab, TU, s);
    if (e == cudaSuccess && pe)
        e = sn::tc_contract_f32(*b, (const __nv_bfloat16 *)pe, seq_len, PU, s);
    return cuda_status(e);
}

sn_status sn_compress_fwd_projected(sn_basis_t b, sn_dtype dt, const void *X, const int32_t *ids,
                                    const int32_t *pos, int64_t T, int32_t seq_len,
                                    const float *TU, int64_t vocab, const float *PU, void *C,
                                    sn_stream_t stream)
{
    sn_status st = check_fwd(b, dt, X, ids, pos, T, seq_len, TU, vocab, PU, C, b ? b->d : 0,
                             b ? b->k : 0);
    if (st != SN_OK || T == 0)
        return st;
    if (dt != SN_BF16)
        return SN_ERR_UNSUPPORTED;
    return cuda_status(sn::tc_compress_projected(*b, (const __nv_bfloat16 *)X, ids, pos, T,
                                                 seq_len, TU, vocab, PU, (__nv_bfloat16 *)C,
                                                 (cudaStream_t)stream));
}

sn_status sn_build_ts(sn_basis_t b, sn_dtype dt, const void *tok, int64_t vocab, void *T_S,
                      void *ws, size_t ws_bytes, sn_stream_t stream)
{
    sn_status st = check_basis(b, dt);
    if (st != SN_OK)
        return st;
    if (dt != SN_BF16)
        return SN_ERR_UNSUPPORTED;
    if (vocab <= 0 || vocab >= kMaxRows || !tok || !T_S || !ws)
        return SN_ERR_INVALID_ARG;
    const size_t table = (size_t)vocab * b->d * 2, coeff = (size_t)vocab * b->k * 2;
    if (ws_bytes < coeff)
        return SN_ERR_INVALID_ARG;
    if (!aligned(tok, 16) || !aligned(T_S, 16) || !aligned(ws, 16))
        return SN_ERR_ALIGNMENT;
    if (overlap(tok, table, T_S, table) || overlap(tok, table, ws, coeff) ||
        overlap(T_S, table, ws, coeff) || !on_device({tok, T_S, ws}))
        return SN_ERR_INVALID_ARG;
    cudaStream_t s = (cudaStream_t)stream;
    sn::TcArgs a{(const __nv_bfloat16 *)tok, nullptr, nullptr, nullptr, nullptr,
                 (__nv_bfloat16 *)ws, vocab, 1, 1, false};
    cudaError_t e = sn::tc_compress(*b, a, s);
    if (e == cudaSuccess)
        e = sn::tc_decompress(*b, a, (__nv_bfloat16 *)T_S, s);
    return cuda_status(e);
}

sn_status sn_grassmann_workspace(sn_basis_t b, int64_t T, size_t *acc_bytes, size_t *step_bytes)
{
    sn_status st = check_basis(b, SN_BF16);
    if (st != SN_OK)
        return st;
    if (T < 0 || T >= kMaxRows)
        return SN_ERR_INVALID_ARG;
    if (acc_bytes)
        *acc_bytes = sn::tc_grassmann_workspace(*b, T > 0 ? T : 1);
    if (step_bytes)
        *step_bytes = sn::grassmann_step_workspace(*b);
    return SN_OK;
}

sn_status sn_grassmann_accumulate(sn_basis_t b, sn_dtype dt, const void *G, const void *Cg,
                                  int64_t T, float *M, void *ws, size_t ws_bytes,
                                  sn_stream_t stream)
{
    sn_status st = check_basis(b, dt);
    if (st != SN_OK)
        return st;
    if (dt != SN_BF16)
        return SN_ERR_UNSUPPORTED;
    if (T < 0 || T >= kMaxRows)
        return SN_ERR_INVALID_ARG;
    if (T == 0)
        return SN_OK;
    if (!G || !Cg || !M || !ws || ws_bytes < sn::tc_grassmann_workspace(*b, T))
        return SN_ERR_INVALID_ARG;
    if (!aligned(G, 16) || !aligned(Cg, 16) || !aligned(M, 16) || !aligned(ws, 256))
        return SN_ERR_ALIGNMENT;
    const size_t mb = (size_t)b->d * b->k * 4;
    if (overlap(M, mb, G, (size_t)T * b->d * 2) || overlap(M, mb, Cg, (size_t)T * b->k * 2) ||
        overlap(ws, ws_bytes, M, mb) || overlap(ws, ws_bytes, G, (size_t)T * b->d * 2) ||
        overlap(ws, ws_bytes, Cg, (size_t)T * b->k * 2) || !on_device({G, Cg, M, ws}))
        return SN_ERR_INVALID_ARG;
    return cuda_status(sn::tc_grassmann_accumulate(*b, (const __nv_bfloat16 *)G,
                                                   (const __nv_bfloat16 *)Cg, T, M, ws,
                                                   (cudaStream_t)stream));
}

sn_status sn_grassmann_residual(sn_basis_t b, sn_dtype dt, const void *G, const void *Cg,
                                int64_t T, double *acc, sn_stream_t stream)
{
    sn_status st = check_basis(b, dt);
    if (st != SN_OK)
        return st;
    if (dt != SN_BF16)
        return SN_ERR_UNSUPPORTED;
    if (T < 0 || T >= kMaxRows || !acc)
        return SN_ERR_INVALID_ARG;
    if (T == 0)
        return SN_OK;
    if (!G || !Cg)
        return SN_ERR_INVALID_ARG;
    if (!aligned(G, 16) || !aligned(Cg, 2) || !aligned(acc, 8))
        return SN_ERR_ALIGNMENT;
    if (!on_device({G, Cg, acc}))
        return SN_ERR_INVALID_ARG;
    return cuda_status(sn::grassmann_residual(*b, (const __nv_bfloat16 *)G,
                                              (const __nv_bfloat16 *)Cg, T, acc,
                                              (cudaStream_t)stream));
}

sn_status sn_grassmann_step(sn_basis_t b, const float *M, int32_t K, float eta, float *U_new,
                            void *ws, size_t ws_bytes, sn_stream_t stream)
{
    sn_status st = check_basis(b, SN_F32);
    if (st != SN_OK)
        return st;
    if (!M || !U_new || !ws || K < 1 || !(eta >= 0.f) ||
        ws_bytes < sn::grassmann_step_workspace(*b))
        return SN_ERR_INVALID_ARG;
    if (!aligned(M, 16) || !aligned(U_new, 16) || !aligned(ws, 256))
        return SN_ERR_ALIGNMENT;
    const size_t mb = (size_t)b->d * b->k * 4;
    if (overlap(M, mb, U_new, mb) || overlap(ws, ws_bytes, M, mb) ||
        overlap(ws, ws_bytes, U_new, mb) || !on_device({M, U_new, ws}))
        return SN_ERR_INVALID_ARG;
    return cuda_status(sn::grassmann_step(*b, M, K, eta, U_new, ws, (cudaStream_t)stream));
}

sn_status sn_adamw_rowconst(sn_dtype gdt, float *W, const void *g, float *M, float *V,
                            int64_t rows, int64_t cols, int64_t t, float lr, float b1, float b2,
                            float eps, float lam, void *ws, size_t ws_bytes, sn_stream_t stream)
{
    if (gdt != SN_BF16 && gdt != SN_F32)
        return SN_ERR_INVALID_ARG;
    if (rows <= 0 || cols <= 0 || rows >= kMaxRows || cols >= kMaxRows || t < 1 ||
        !(b1 >= 0.f && b1 < 1.f) || !(b2 >= 0.f && b2 < 1.f) || !(eps >= 0.f) || !(lr >= 0.f) ||
        !(lam >= 0.f) || !W || !g || !M || !V || !ws || ws_bytes < (size_t)cols * 4)
        return SN_ERR_INVALID_ARG;
    if (!aligned(W, 16) || !aligned(g, 16) || !aligned(M, 16) || !aligned(V, 16) ||
        !aligned(ws, 16))
        return SN_ERR_ALIGNMENT;
    const size_t n4 = (size_t)rows * cols * 4, ng = (size_t)rows * cols * esize(gdt);
    const void *bufs[5] = {W, g, M, V, ws};
    const size_t lens[5] = {n4, ng, n4, n4, (size_t)cols * 4};
    for (int i = 0; i < 5; ++i)
        for (int j = i + 1; j < 5; ++j)
            if (overlap(bufs[i], lens[i], bufs[j], lens[j]))
                return SN_ERR_INVALID_ARG;
    if (!on_device({W, g, M, V, ws}))
        return SN_ERR_INVALID_ARG;
    return cuda_status(sn::adamw_rowconst(gdt == SN_BF16, W, g, M, V, rows, cols, t, lr, b1, b2,
                                          eps, lam, (float *)ws, (cudaStream_t)stream));
}

namespace {
sn_status check_batch(const void *X, int64_t T, int32_t d)
{
    if (T < 0 || T >= kMaxRows || d <= 0 || d % 8 != 0 || !X)
        return SN_ERR_INVALID_ARG;
    return aligned(X, 16) ? SN_OK : SN_ERR_ALIGNMENT;
}
}  // namespace

sn_status sn_topk_compress(const void *X, int64_t T, int32_t d, int32_t kk, void *vals,
                           uint16_t *cols, sn_stream_t stream)
{
    sn_status st = check_batch(X, T, d);
    if (st != SN_OK)
        return st;
    if (d > 65536 || kk < 1 || kk > d || kk > 4096 || !vals || !cols)
        return SN_ERR_INVALID_ARG;
    if (!aligned(vals, 2) || !aligned(cols, 2))
        return SN_ERR_ALIGNMENT;
    if (T == 0)
        return SN_OK;
    const size_t nx = (size_t)T * d * 2, nk = (size_t)T * kk * 2;
    if (overlap(X, nx, vals, nk) || overlap(X, nx, cols, nk) || overlap(vals, nk, cols, nk) ||
        !on_device({X, vals, cols}))
        return SN_ERR_INVALID_ARG;
    return cuda_status(sn::lossy_topk(X, T, d, kk, vals, cols, (cudaStream_t)stream));
}

sn_status sn_topk_restore(const void *vals, const uint16_t *cols, int64_t T, int32_t d,
                          int32_t kk, void *X_out, sn_stream_t stream)
{
    sn_status st = check_batch(X_out, T, d);
    if (st != SN_OK)
        return st;
    if (d > 65536 || kk < 1 || kk > d || !vals || !cols)
        return SN_ERR_INVALID_ARG;
    if (!aligned(vals, 2) || !aligned(cols, 2))
        return SN_ERR_ALIGNMENT;
    if (T == 0)
        return SN_OK;
    const size_t nx = (size_t)T * d * 2, nk = (size_t)T * kk * 2;
    if (overlap(X_out, nx, vals, nk) || overlap(X_out, nx, cols, nk) ||
        !on_device({vals, cols, X_out}))
        return SN_ERR_INVALID_ARG;
    return cuda_status(sn::lossy_topk_restore(vals, cols, T, d, kk, X_out, (cudaStream_t)stream));
}

sn_status sn_sign_compress(const void *X, int64_t T, int32_t d, uint32_t *bits, float *scale,
                           sn_stream_t stream)
{
    sn_status st = check_batch(X, T, d);
    if (st != SN_OK)
        return st;
    if (!bits || !scale)
        return SN_ERR_INVALID_ARG;
    if (!aligned(bits, 4) || !aligned(scale, 4))
        return SN_ERR_ALIGNMENT;
    if (T == 0)
        return SN_OK;
    const size_t nx = (size_t)T * d * 2, nb = (size_t)T * ((d + 31) / 32) * 4, ns = (size_t)T * 4;
    if (overlap(X, nx, bits, nb) || overlap(X, nx, scale, ns) || overlap(bits, nb, scale, ns) ||
        !on_device({X, bits, scale}))
        return SN_ERR_INVALID_ARG;
    return cuda_status(sn::lossy_sign(X, T, d, bits, scale, (cudaStream_t)stream));
}

sn_status sn_sign_restore(const uint32_t *bits, const float *scale, int64_t T, int32_t d,
                          void *X_out, sn_stream_t stream)
{
    sn_status st = check_batch(X_out, T, d);
    if (st != SN_OK)
        return st;
    if (!bits || !scale)
        return SN_ERR_INVALID_ARG;
    if (!aligned(bits, 4) || !aligned(scale, 4))
        return SN_ERR_ALIGNMENT;
    if (T == 0)
        return SN_OK;
    const size_t nx = (size_t)T * d * 2;
    if (overlap(X_out, nx, bits, (size_t)T * ((d + 31) / 32) * 4) ||
        overlap(X_out, nx, scale, (size_t)T * 4) || !on_device({bits, scale, X_out}))
        return SN_ERR_INVALID_ARG;
    return cuda_status(sn::lossy_sign_restore(bits, scale, T, d, X_out, (cudaStream_t)stream));
}

sn_status sn_quant_compress(const void *X, int64_t T, int32_t d, int32_t format, uint8_t *codes,
                            float *scale, sn_stream_t stream)
{
    sn_status st = check_batch(X, T, d);
    if (st != SN_OK)
        return st;
    if ((format != SN_Q_INT8 && format != SN_Q_E4M3) || !codes || !scale)
        return SN_ERR_INVALID_ARG;
    if (!aligned(codes, 8) || !aligned(scale, 4))
        return SN_ERR_ALIGNMENT;
    if (T == 0)
        return SN_OK;
    const size_t nx = (size_t)T * d * 2, nc = (size_t)T * d, ns = (size_t)T * 4;
    if (overlap(X, nx, codes, nc) || overlap(X, nx, scale, ns) || overlap(codes, nc, scale, ns) ||
        !on_device({X, codes, scale}))
        return SN_ERR_INVALID_ARG;
    return cuda_status(sn::lossy_quant(X, T, d, format, codes, scale, (cudaStream_t)stream));
}

sn_status sn_quant_restore(const uint8_t *codes, const float *scale, int64_t T, int32_t d,
                           int32_t format, void *X_out, sn_stream_t stream)
{
    sn_status st = check_batch(X_out, T, d);
    if (st != SN_OK)
        return st;
    if ((format != SN_Q_INT8 && format != SN_Q_E4M3) || !codes || !scale)
        return SN_ERR_INVALID_ARG;
    if (!aligned(codes, 8) || !aligned(scale, 4))
        return SN_ERR_ALIGNMENT;
    if (T == 0)
        return SN_OK;
    const size_t nx = (size_t)T * d * 2;
    if (overlap(X_out, nx, codes, (size_t)T * d) || overlap(X_out, nx, scale, (size_t)T * 4) ||
        !on_device({codes, scale, X_out}))
        return SN_ERR_INVALID_ARG;
    return cuda_status(sn::lossy_quant_restore(codes, scale, T, d, format, X_out,
                                               (cudaStream_t)stream));
}

namespace {

bool is_dtype(sn_dtype dt) { return dt == SN_BF16 || dt == SN_F32; }

// A buffer of a call: `rows` rows of `width` elements of `es` bytes, `ld` elements apart
struct Buf {
    const void *p;
    size_t bytes;
    Buf(const void *p, int64_t rows, int64_t width, int64_t ld, size_t es)
        : p(p), bytes(p && rows > 0 ? ((size_t)(rows - 1) * ld + width) * es : 0) {}
};

bool clash(const Buf &a, const Buf &b) { return a.bytes && b.bytes && overlap(a.p, a.bytes, b.p, b.bytes); }

// Whether `out` overlaps one of `others`
bool clashes(const Buf &out, std::initializer_list<Buf> others)
{
    for (const Buf &b : others)
        if (clash(out, b))
            return true;
    return false;
}

// Whether `out` overlaps `in` other than by being it, row by row
bool clashes_unless_same(const Buf &out, const Buf &in, bool same_rows)
{
    return clash(out, in) && !(out.p == in.p && same_rows);
}

constexpr int32_t kMaxWidth = 1 << 20;
constexpr int64_t kMaxTokens = kMaxRows - 512;   // places of a list of tokens are 32-bit

// The error word that out-of-range ids are recorded in: none without a basis
sn_status error_word(sn_basis_t b, unsigned int **err)
{
    *err = nullptr;
    if (!b)
        return SN_OK;
    const sn_status st = check_basis(b, SN_F32);
    if (st == SN_OK)
        *err = b->err;
    return st;
}

sn_status check_norm(sn_dtype dt, sn_dtype wdt, int64_t T, int32_t d, int64_t ld, float eps)
{
    if (!is_dtype(dt) || !is_dtype(wdt) || T < 0 || T >= kMaxRows || d < 1 || d > kMaxWidth || ld < d ||
        ld >= kMaxRows || !(eps >= 0.f) || !std::isfinite(eps))
        return SN_ERR_INVALID_ARG;
    return SN_OK;
}

// Both forwards: format < 0 writes Y
sn_status norm_fwd(sn_dtype dt, const void *X, int64_t ldx, const void *R, void *H, sn_dtype wdt, const void *w,
                   int64_t T, int32_t d, float eps, void *Y, int32_t format, int32_t group, uint8_t *codes,
                   float *scale, cudaStream_t s)
{
    sn_status st = check_norm(dt, wdt, T, d, ldx, eps);
    if (st != SN_OK || T == 0)
        return st;
    const bool quant = format >= 0;
    if (!X || !w || (quant ? !codes || !scale : !Y))
        return SN_ERR_INVALID_ARG;
    if (!aligned(X, 16) || !aligned(R, 16) || !aligned(H, 16) || !aligned(w, 16) || !aligned(Y, 16) ||
        !aligned(codes, 16) || !aligned(scale, 4))
        return SN_ERR_ALIGNMENT;
    const size_t es = esize(dt);
    const int64_t groups = group ? (d + group - 1) / group : 1;
    const Buf x(X, T, d, ldx, es), r(R, T, d, d, es), h(H, T, d, d, es), y(Y, T, d, d, es), c(codes, T, d, d, 1),
        q(scale, T, groups, groups, 4), wb(w, 1, d, d, esize(wdt));
    if (clashes_unless_same(h, x, ldx == d) || clashes_unless_same(h, r, true) ||
        clashes_unless_same(y, x, ldx == d) || clashes_unless_same(y, r, true) || clashes(h, {y, c, q, wb}) ||
        clashes(wb, {y, c, q}) || clashes(c, {x, r, q}) || clashes(q, {x, r}) ||
        !on_device({X, R, H, w, Y, codes, scale}))
        return SN_ERR_INVALID_ARG;
    return cuda_status(sn::rmsnorm_fwd(dt, X, ldx, R, H, wdt, w, T, d, eps, Y, format, group, codes, scale, s));
}

}  // namespace

sn_status sn_embed_fwd(sn_basis_t errors, sn_dtype tdt, const void *table, int64_t vocab, int32_t d,
                       const int32_t *ids, int64_t T, float scale, sn_dtype xdt, void *X, sn_stream_t stream)
{
    unsigned int *err;
    const sn_status st = error_word(errors, &err);
    if (st != SN_OK)
        return st;
    if (!is_dtype(tdt) || !is_dtype(xdt) || vocab < 1 || vocab >= kMaxRows || d < 1 || d > kMaxWidth || T < 0 ||
        T >= kMaxTokens)
        return SN_ERR_INVALID_ARG;
    if (T == 0)
        return SN_OK;
    if (!table || !ids || !X)
        return SN_ERR_INVALID_ARG;
    if (!aligned(table, 16) || !aligned(ids, 4) || !aligned(X, 16))
        return SN_ERR_ALIGNMENT;
    if (clashes(Buf(X, T, d, d, esize(xdt)), {Buf(table, vocab, d, d, esize(tdt)), Buf(ids, 1, T, T, 4)}) ||
        !on_device({table, ids, X}))
        return SN_ERR_INVALID_ARG;
    return cuda_status(sn::embed_fwd(tdt, table, vocab, d, ids, T, scale, xdt, X, err, (cudaStream_t)stream));
}

sn_status sn_embed_bwd_workspace(int64_t T, int64_t vocab, int32_t d, size_t *bytes)
{
    if (!bytes || T < 0 || T >= kMaxTokens || vocab < 1 || vocab >= kMaxRows || d < 1 || d > kMaxWidth)
        return SN_ERR_INVALID_ARG;
    *bytes = sn::embed_bwd_workspace(T, vocab, d);
    return SN_OK;
}

sn_status sn_embed_bwd(sn_basis_t errors, sn_dtype dt, const void *G, int64_t ldg, int64_t T, int32_t d,
                       const int32_t *ids, float scale, sn_dtype edt, void *dE, int64_t vocab, int32_t accumulate,
                       void *ws, size_t ws_bytes, sn_stream_t stream)
{
    unsigned int *err;
    const sn_status st = error_word(errors, &err);
    if (st != SN_OK)
        return st;
    size_t need = 0;
    if (!is_dtype(dt) || !is_dtype(edt) || sn_embed_bwd_workspace(T, vocab, d, &need) != SN_OK || ldg < d ||
        ldg >= kMaxRows)
        return SN_ERR_INVALID_ARG;
    if (T == 0 && accumulate)
        return SN_OK;
    if ((T > 0 && (!G || !ids)) || !dE || !ws || ws_bytes < need)
        return SN_ERR_INVALID_ARG;
    if (!aligned(G, 16) || !aligned(ids, 4) || !aligned(dE, 16) || !aligned(ws, 256))
        return SN_ERR_ALIGNMENT;
    const Buf g(G, T, d, ldg, esize(dt)), i(ids, 1, T, T, 4), e(dE, vocab, d, d, esize(edt)), w(ws, 1, need, need, 1);
    if (clashes(e, {g, i, w}) || clashes(w, {g, i}) || !on_device({G, ids, dE, ws}))
        return SN_ERR_INVALID_ARG;
    return cuda_status(sn::embed_bwd(dt, G, ldg, T, d, ids, scale, edt, dE, vocab, accumulate != 0, ws, err,
                                     (cudaStream_t)stream));
}

sn_status sn_rmsnorm_fwd(sn_dtype dt, const void *X, int64_t ldx, const void *R, void *H, sn_dtype wdt,
                         const void *w, int64_t T, int32_t d, float eps, void *Y, sn_stream_t stream)
{
    return norm_fwd(dt, X, ldx, R, H, wdt, w, T, d, eps, Y, -1, 0, nullptr, nullptr, (cudaStream_t)stream);
}

sn_status sn_rmsnorm_fwd_quant(sn_dtype dt, const void *X, int64_t ldx, const void *R, void *H, sn_dtype wdt,
                               const void *w, int64_t T, int32_t d, float eps, int32_t format, int32_t group,
                               uint8_t *codes, float *scale, sn_stream_t stream)
{
    if ((format != SN_Q_INT8 && format != SN_Q_E4M3) || (group != 0 && group != 32 && group != 64 && group != 128))
        return SN_ERR_INVALID_ARG;
    return norm_fwd(dt, X, ldx, R, H, wdt, w, T, d, eps, nullptr, format, group, codes, scale,
                    (cudaStream_t)stream);
}

sn_status sn_rmsnorm_bwd_workspace(int64_t T, int32_t d, size_t *bytes)
{
    if (!bytes || T < 0 || T >= kMaxRows || d < 1 || d > kMaxWidth)
        return SN_ERR_INVALID_ARG;
    *bytes = sn::rmsnorm_bwd_workspace(T, d);
    return SN_OK;
}

sn_status sn_rmsnorm_bwd(sn_dtype dt, const void *dY, int64_t ldy, const void *H, const void *dH, sn_dtype wdt,
                         const void *w, int64_t T, int32_t d, float eps, void *dX, float *dw, int32_t accumulate,
                         void *ws, size_t ws_bytes, sn_stream_t stream)
{
    const sn_status st = check_norm(dt, wdt, T, d, ldy, eps);
    if (st != SN_OK || (T == 0 && accumulate))
        return st;
    const size_t need = sn::rmsnorm_bwd_workspace(T, d);
    if (!dw || (T > 0 && (!dY || !H || !w || !dX || !ws || ws_bytes < need)))
        return SN_ERR_INVALID_ARG;
    if (!aligned(dY, 16) || !aligned(H, 16) || !aligned(dH, 16) || !aligned(w, 16) || !aligned(dX, 16) ||
        !aligned(dw, 16) || !aligned(ws, 16))
        return SN_ERR_ALIGNMENT;
    const size_t es = esize(dt);
    const Buf y(dY, T, d, ldy, es), h(H, T, d, d, es), r(dH, T, d, d, es), x(dX, T, d, d, es),
        wb(T > 0 ? w : nullptr, 1, d, d, esize(wdt)), g(dw, 1, d, d, 4), p(T > 0 ? ws : nullptr, 1, need, need, 1);
    if (clashes_unless_same(x, y, ldy == d) || clashes_unless_same(x, h, true) || clashes_unless_same(x, r, true) ||
        clashes(x, {wb, g, p}) || clashes(g, {y, h, r, wb, p}) || clashes(p, {y, h, r, wb}) ||
        !on_device({dY, H, dH, w, dX, dw, ws}))
        return SN_ERR_INVALID_ARG;
    if (T == 0)
        return cuda_status(cudaMemsetAsync(dw, 0, (size_t)d * 4, (cudaStream_t)stream));
    return cuda_status(sn::rmsnorm_bwd(dt, dY, ldy, H, dH, wdt, w, T, d, eps, dX, dw, accumulate != 0, (float *)ws,
                                       (cudaStream_t)stream));
}

namespace {
// A gate has a row for every T / gates tokens in a run
bool is_gating(const void *gate, int64_t gates, int64_t T)
{
    return gate ? gates >= 1 && T % gates == 0 && (T == 0 || gates <= T) : gates == 0;
}
}  // namespace

sn_status sn_blocknorm_fwd(sn_dtype dt, const void *Y, int64_t ldy, const void *R, const void *gate, int64_t gates,
                           sn_dtype wdt, const void *w_post, const void *w_pre, int64_t T, int32_t d, float eps,
                           float scale, void *H, void *Z, sn_stream_t stream)
{
    const sn_status st = check_norm(dt, wdt, T, d, ldy, eps);
    if (st != SN_OK)
        return st;
    if (!std::isfinite(scale) || !is_gating(gate, gates, T))
        return SN_ERR_INVALID_ARG;
    if (T == 0)
        return SN_OK;
    if (!Y || !R || !w_post || !w_pre || !H || !Z)
        return SN_ERR_INVALID_ARG;
    if (!aligned(Y, 16) || !aligned(R, 16) || !aligned(gate, 16) || !aligned(w_post, 16) || !aligned(w_pre, 16) ||
        !aligned(H, 16) || !aligned(Z, 16))
        return SN_ERR_ALIGNMENT;
    const size_t es = esize(dt);
    const Buf y(Y, T, d, ldy, es), r(R, T, d, d, es), g(gate, gates, d, d, es), p(w_post, 1, d, d, esize(wdt)),
        q(w_pre, 1, d, d, esize(wdt)), h(H, T, d, d, es), z(Z, T, d, d, es);
    if (clashes_unless_same(h, y, ldy == d) || clashes_unless_same(h, r, true) || clashes_unless_same(z, y, ldy == d) ||
        clashes_unless_same(z, r, true) || clashes(h, {g, p, q, z}) || clashes(z, {g, p, q}) ||
        !on_device({Y, R, gate, w_post, w_pre, H, Z}))
        return SN_ERR_INVALID_ARG;
    return cuda_status(sn::blocknorm_fwd(dt, Y, ldy, R, gate, gates, wdt, w_post, w_pre, T, d, eps, scale, H, Z,
                                         (cudaStream_t)stream));
}

sn_status sn_blocknorm_bwd_workspace(int64_t T, int32_t d, int64_t gates, size_t *bytes)
{
    if (!bytes || T < 0 || T >= kMaxRows || d < 1 || d > kMaxWidth || gates < 0 || (gates > 0 && T % gates))
        return SN_ERR_INVALID_ARG;
    *bytes = T == 0 ? 0 : sn::blocknorm_bwd_workspace(T, d, gates);
    return SN_OK;
}

sn_status sn_blocknorm_bwd(sn_dtype dt, const void *dZ, int64_t lddz, const void *H, const void *Y, int64_t ldy,
                           const void *dH, const void *gate, int64_t gates, sn_dtype wdt, const void *w_post,
                           const void *w_pre, int64_t T, int32_t d, float eps, float scale, void *dY, void *dR,
                           float *dw_post, float *dw_pre, float *dgate, int32_t accumulate, void *ws,
                           size_t ws_bytes, sn_stream_t stream)
{
    sn_status st = check_norm(dt, wdt, T, d, ldy, eps);
    if (st == SN_OK)
        st = check_norm(dt, wdt, T, d, lddz, eps);
    if (st != SN_OK)
        return st;
    if (!std::isfinite(scale) || !is_gating(gate, gates, T) || !dw_post || !dw_pre ||
        (gate == nullptr) != (dgate == nullptr))
        return SN_ERR_INVALID_ARG;
    if (T == 0 && accumulate)
        return SN_OK;
    const size_t need = T > 0 ? sn::blocknorm_bwd_workspace(T, d, gates) : 0;
    if (T > 0 && (!dZ || !H || !Y || !w_post || !w_pre || !dY || !dR || !ws || ws_bytes < need))
        return SN_ERR_INVALID_ARG;
    if (!aligned(dZ, 16) || !aligned(H, 16) || !aligned(Y, 16) || !aligned(dH, 16) || !aligned(gate, 16) ||
        !aligned(w_post, 16) || !aligned(w_pre, 16) || !aligned(dY, 16) || !aligned(dR, 16) ||
        !aligned(dw_post, 16) || !aligned(dw_pre, 16) || !aligned(dgate, 16) || !aligned(ws, 16))
        return SN_ERR_ALIGNMENT;
    const size_t es = esize(dt);
    const Buf z(dZ, T, d, lddz, es), h(H, T, d, d, es), y(Y, T, d, ldy, es), r(dH, T, d, d, es),
        g(gate, gates, d, d, es), p(T > 0 ? w_post : nullptr, 1, d, d, esize(wdt)),
        q(T > 0 ? w_pre : nullptr, 1, d, d, esize(wdt)), oy(dY, T, d, d, es), orr(dR, T, d, d, es),
        a(dw_post, 1, d, d, 4), b(dw_pre, 1, d, d, 4), c(dgate, gates, d, d, 4), w(T > 0 ? ws : nullptr, 1, need, need, 1);
    for (const Buf *o : {&oy, &orr})
        if (clashes_unless_same(*o, z, lddz == d) || clashes_unless_same(*o, h, true) ||
            clashes_unless_same(*o, y, ldy == d) || clashes_unless_same(*o, r, true) ||
            clashes(*o, {g, p, q, a, b, c, w}))
            return SN_ERR_INVALID_ARG;
    if (clashes(oy, {orr}) || clashes(a, {z, h, y, r, g, p, q, b, c, w}) || clashes(b, {z, h, y, r, g, p, q, c, w}) ||
        clashes(c, {z, h, y, r, g, p, q, w}) || clashes(w, {z, h, y, r, g, p, q}) ||
        !on_device({dZ, H, Y, dH, gate, w_post, w_pre, dY, dR, dw_post, dw_pre, dgate, ws}))
        return SN_ERR_INVALID_ARG;
    if (T == 0) {
        const cudaStream_t s = (cudaStream_t)stream;
        cudaError_t e = cudaMemsetAsync(dw_post, 0, (size_t)d * 4, s);
        if (e == cudaSuccess)
            e = cudaMemsetAsync(dw_pre, 0, (size_t)d * 4, s);
        if (e == cudaSuccess && dgate)
            e = cudaMemsetAsync(dgate, 0, (size_t)gates * d * 4, s);
        return cuda_status(e);
    }
    return cuda_status(sn::blocknorm_bwd(dt, dZ, lddz, H, Y, ldy, dH, gate, gates, wdt, w_post, w_pre, T, d, eps,
                                         scale, dY, dR, dw_post, dw_pre, dgate, accumulate != 0, (float *)ws,
                                         (cudaStream_t)stream));
}

namespace {
sn_status check_logits(sn_dtype dt, int64_t T, int64_t V, int64_t ld, float scale)
{
    // (the kernels' exponents are scale * log2(e) times a difference of logits)
    if (!is_dtype(dt) || T < 0 || T >= kMaxRows || V < 1 || V >= kMaxTokens || ld < V || ld >= kMaxRows ||
        !(scale > 0.f) || !std::isfinite(scale * 1.4426950408889634f))
        return SN_ERR_INVALID_ARG;
    return SN_OK;
}
}  // namespace

sn_status sn_logprob_fwd(sn_basis_t errors, sn_dtype dt, const void *x, int64_t T, int64_t V, int64_t ld,
                         const int32_t *target, float scale, float *logp, float *lse, float *entropy, int32_t top,
                         int32_t *top_ids, float *top_logp, sn_stream_t stream)
{
    unsigned int *err;
    sn_status st = error_word(errors, &err);
    if (st == SN_OK)
        st = check_logits(dt, T, V, ld, scale);
    if (st != SN_OK)
        return st;
    if (top < 0 || top > 32 || top > V)
        return SN_ERR_INVALID_ARG;
    if (T == 0)
        return SN_OK;
    if (!x || (target == nullptr) != (logp == nullptr) || (top > 0 && (!top_ids || !top_logp)) ||
        (!logp && !lse && !entropy && top == 0))
        return SN_ERR_INVALID_ARG;
    if (!aligned(x, 16) || !aligned(target, 4) || !aligned(logp, 4) || !aligned(lse, 8) || !aligned(entropy, 4) ||
        !aligned(top_ids, 4) || !aligned(top_logp, 4))
        return SN_ERR_ALIGNMENT;
    if (top == 0)
        top_ids = nullptr, top_logp = nullptr;
    const Buf in(x, T, V, ld, esize(dt)), tg(target, 1, T, T, 4), a(logp, 1, T, T, 4), b(lse, T, 2, 2, 4),
        c(entropy, 1, T, T, 4), i(top_ids, T, top, top, 4), l(top_logp, T, top, top, 4);
    if (clashes(a, {in, tg, b, c, i, l}) || clashes(b, {in, tg, c, i, l}) || clashes(c, {in, tg, i, l}) ||
        clashes(i, {in, tg, l}) || clashes(l, {in, tg}) ||
        !on_device({x, target, logp, lse, entropy, top_ids, top_logp}))
        return SN_ERR_INVALID_ARG;
    return cuda_status(sn::logprob_fwd(dt, x, T, (int)V, ld, target, scale, logp, lse, entropy, top, top_ids,
                                       top_logp, err, (cudaStream_t)stream));
}

sn_status sn_logprob_bwd(sn_dtype dt, const void *x, int64_t T, int64_t V, int64_t ld, const int32_t *target,
                         const float *lse, const float *dlogp, const float *entropy, const float *dentropy,
                         float scale, void *dx, int64_t ldd, sn_stream_t stream)
{
    const sn_status st = check_logits(dt, T, V, ld, scale);
    if (st != SN_OK)
        return st;
    if (ldd < V || ldd >= kMaxRows)
        return SN_ERR_INVALID_ARG;
    if (T == 0)
        return SN_OK;
    if (!x || !lse || !dx || (target == nullptr) != (dlogp == nullptr) ||
        (entropy == nullptr) != (dentropy == nullptr) || (!dlogp && !dentropy))
        return SN_ERR_INVALID_ARG;
    if (!aligned(x, 16) || !aligned(dx, 16) || !aligned(target, 4) || !aligned(lse, 8) || !aligned(dlogp, 4) ||
        !aligned(entropy, 4) || !aligned(dentropy, 4))
        return SN_ERR_ALIGNMENT;
    const size_t es = esize(dt);
    const Buf in(x, T, V, ld, es), out(dx, T, V, ldd, es);
    if (clashes_unless_same(out, in, ld == ldd) ||
        clashes(out, {Buf(target, 1, T, T, 4), Buf(lse, T, 2, 2, 4), Buf(dlogp, 1, T, T, 4),
                      Buf(entropy, 1, T, T, 4), Buf(dentropy, 1, T, T, 4)}) ||
        !on_device({x, target, lse, dlogp, entropy, dentropy, dx}))
        return SN_ERR_INVALID_ARG;
    return cuda_status(sn::logprob_bwd(dt, x, T, (int)V, ld, target, lse, dlogp, entropy, dentropy, scale, dx, ldd,
                                       (cudaStream_t)stream));
}

namespace {
sn_status check_glu(sn_dtype dt, int64_t T, int32_t d, int32_t f, int32_t act, std::initializer_list<int64_t> lds)
{
    if (!is_dtype(dt) || T < 0 || T >= kMaxTokens || d < 1 || d > kMaxWidth || f < 1 || f > kMaxWidth ||
        act < SN_ACT_SILU || act > SN_ACT_RELU)
        return SN_ERR_INVALID_ARG;
    for (const int64_t ld : lds)
        if (ld >= kMaxRows)
            return SN_ERR_INVALID_ARG;
    if (dt != SN_BF16)
        return SN_ERR_UNSUPPORTED;
    if (d % 8 || f % 8)
        return SN_ERR_ALIGNMENT;
    for (const int64_t ld : lds)
        if (ld % 8)
            return SN_ERR_ALIGNMENT;
    return SN_OK;
}
}  // namespace

sn_status sn_glu_fwd(sn_basis_t errors, sn_dtype dt, const void *X, int64_t ldx, const void *Wg, const void *Wu,
                     int64_t T, int32_t d, int32_t f, int32_t act, void *G, void *U, void *H, sn_stream_t stream)
{
    unsigned int *err;
    sn_status st = error_word(errors, &err);
    if (st == SN_OK)
        st = ldx < d ? SN_ERR_INVALID_ARG : check_glu(dt, T, d, f, act, {ldx});
    if (st != SN_OK || T == 0)
        return st;
    if (!X || !Wg || !Wu || !H || (G == nullptr) != (U == nullptr))
        return SN_ERR_INVALID_ARG;
    if (!aligned(X, 16) || !aligned(Wg, 16) || !aligned(Wu, 16) || !aligned(G, 16) || !aligned(U, 16) ||
        !aligned(H, 16))
        return SN_ERR_ALIGNMENT;
    const Buf x(X, T, d, ldx, 2), wg(Wg, f, d, d, 2), wu(Wu, f, d, d, 2), g(G, T, f, f, 2), u(U, T, f, f, 2),
        h(H, T, f, f, 2);
    if (clashes(h, {x, wg, wu, g, u}) || clashes(g, {x, wg, wu, u}) || clashes(u, {x, wg, wu}) ||
        !on_device({X, Wg, Wu, G, U, H}))
        return SN_ERR_INVALID_ARG;
    return cuda_status(sn::glu_fwd(X, ldx, Wg, Wu, T, d, f, act, G, U, H, err, (cudaStream_t)stream));
}

sn_status sn_glu_bwd_workspace(int64_t T, int32_t d, int32_t f, size_t *bytes)
{
    const sn_status st = check_glu(SN_BF16, T, d, f, SN_ACT_SILU, {});
    if (st != SN_OK || !bytes)
        return st != SN_OK ? st : SN_ERR_INVALID_ARG;
    *bytes = sn::glu_bwd_workspace(T, d, f);
    return SN_OK;
}

sn_status sn_glu_bwd(sn_basis_t errors, sn_dtype dt, const void *dH, int64_t lddh, const void *X, int64_t ldx,
                     const void *Wg, const void *Wu, const void *G, const void *U, int64_t T, int32_t d, int32_t f,
                     int32_t act, void *dG, void *dU, void *dX, sn_dtype gdt, void *dWg, void *dWu,
                     int32_t accumulate, void *ws, size_t ws_bytes, sn_stream_t stream)
{
    unsigned int *err;
    sn_status st = error_word(errors, &err);
    if (st != SN_OK)
        return st;
    const bool dx = dX != nullptr, dw = dWg != nullptr;
    if (!is_dtype(gdt) || lddh < f || (dw && ldx < d) || dw != (dWu != nullptr))
        return SN_ERR_INVALID_ARG;
    st = check_glu(dt, T, d, f, act, {lddh, dw ? ldx : 0});
    if (st != SN_OK || (T == 0 && (!dw || accumulate)))
        return st;
    const size_t need = dx || dw ? sn::glu_bwd_workspace(T, d, f) : 0, es = esize(gdt);
    if (T > 0 && (!dH || !G || !U || !dG || !dU || (dx && (!Wg || !Wu)) || (dw && !X) ||
                  (need > 0 && (!ws || ws_bytes < need))))
        return SN_ERR_INVALID_ARG;
    if (!aligned(dH, 16) || !aligned(X, 16) || !aligned(Wg, 16) || !aligned(Wu, 16) || !aligned(G, 16) ||
        !aligned(U, 16) || !aligned(dG, 16) || !aligned(dU, 16) || !aligned(dX, 16) || !aligned(dWg, 16) ||
        !aligned(dWu, 16) || !aligned(ws, 16))
        return SN_ERR_ALIGNMENT;
    const Buf h(dH, T, f, lddh, 2), x(dw ? X : nullptr, T, d, ldx, 2), wg(dx ? Wg : nullptr, f, d, d, 2),
        wu(dx ? Wu : nullptr, f, d, d, 2), g(G, T, f, f, 2), u(U, T, f, f, 2), dg(dG, T, f, f, 2), du(dU, T, f, f, 2),
        dxb(dX, T, d, d, 2), a(dWg, f, d, d, es), b(dWu, f, d, d, es), p(T > 0 ? ws : nullptr, 1, need, need, 1);
    if (clashes_unless_same(dg, g, true) || clashes_unless_same(du, u, true) || clashes(dg, {h, x, wg, wu, u, du}) ||
        clashes(du, {h, x, wg, wu, g}) || clashes(dxb, {h, x, wg, wu, g, u, dg, du, a, b}) ||
        clashes(a, {h, x, wg, wu, g, u, dg, du, b}) || clashes(b, {h, x, wg, wu, g, u, dg, du}) ||
        clashes(p, {h, x, wg, wu, g, u, dg, du, dxb, a, b}) ||
        !on_device({dH, X, Wg, Wu, G, U, dG, dU, dX, dWg, dWu, ws}))
        return SN_ERR_INVALID_ARG;
    if (T == 0) {
        const cudaError_t e = cudaMemsetAsync(dWg, 0, (size_t)f * d * es, (cudaStream_t)stream);
        return cuda_status(e != cudaSuccess ? e : cudaMemsetAsync(dWu, 0, (size_t)f * d * es, (cudaStream_t)stream));
    }
    return cuda_status(sn::glu_bwd(dH, lddh, X, ldx, Wg, Wu, G, U, T, d, f, act, dG, dU, dX, gdt, dWg, dWu,
                                   accumulate != 0, ws, err, (cudaStream_t)stream));
}

sn_status sn_grads_create(int32_t n, const void *const *src, const sn_dtype *sdt, const int64_t *count,
                          void *const *dst, const sn_dtype *ddt, sn_grads_t *out, sn_stream_t stream)
try {
    if (n < 0 || !out || (n > 0 && (!src || !sdt || !count || !dst || !ddt)))
        return SN_ERR_INVALID_ARG;
    // every source and destination as a range of addresses; a destination may meet only
    // its own source
    struct Range {
        uintptr_t at, end;
        int tensor;
        bool dst;
    };
    std::vector<Range> ranges;
    for (int i = 0; i < n; ++i) {
        if (!is_dtype(sdt[i]) || !is_dtype(ddt[i]) || count[i] < 0 || count[i] >= (int64_t)1 << 48)
            return SN_ERR_INVALID_ARG;
        if (count[i] == 0)
            continue;
        if (!src[i] || !dst[i])
            return SN_ERR_INVALID_ARG;
        if (!aligned(src[i], esize(sdt[i])) || !aligned(dst[i], esize(ddt[i])))
            return SN_ERR_ALIGNMENT;
        if (!on_device({src[i], dst[i]}) || (src[i] == dst[i] && sdt[i] != ddt[i]))
            return SN_ERR_INVALID_ARG;
        const uintptr_t p = (uintptr_t)src[i], q = (uintptr_t)dst[i];
        if (p != q)
            ranges.push_back({p, p + (size_t)count[i] * esize(sdt[i]), i, false});
        ranges.push_back({q, q + (size_t)count[i] * esize(ddt[i]), i, true});
    }
    std::sort(ranges.begin(), ranges.end(), [](const Range &a, const Range &b) { return a.at < b.at; });
    uintptr_t end = 0, dst_end = 0;           // of everything, and of the destinations, so far
    for (const Range &r : ranges) {
        if (r.at < (r.dst ? end : dst_end))
            return SN_ERR_INVALID_ARG;
        end = std::max(end, r.end);
        if (r.dst)
            dst_end = std::max(dst_end, r.end);
    }
    return cuda_status(sn::grads_create(n, src, sdt, count, dst, ddt, out, (cudaStream_t)stream));
} catch (const std::exception &) {
    return SN_ERR_CUDA;                       // no host memory
}

sn_status sn_grads_destroy(sn_grads_t g) { return g ? cuda_status(sn::grads_destroy(g)) : SN_OK; }

namespace {
sn_status check_grads(sn_grads_t g)
{
    int dev = -1;
    if (!g)
        return SN_ERR_INVALID_ARG;
    if (cudaGetDevice(&dev) != cudaSuccess)
        return SN_ERR_CUDA;
    return dev == sn::grads_device(g) ? SN_OK : SN_ERR_INVALID_ARG;
}
}  // namespace

sn_status sn_grads_sumsq(sn_grads_t g, double *sumsq, int32_t accumulate, sn_stream_t stream)
{
    const sn_status st = check_grads(g);
    if (st != SN_OK)
        return st;
    if (!sumsq)
        return SN_ERR_INVALID_ARG;
    if (!aligned(sumsq, 8))
        return SN_ERR_ALIGNMENT;
    if (!on_device({sumsq}))
        return SN_ERR_INVALID_ARG;
    return cuda_status(sn::grads_sumsq(*g, sumsq, accumulate != 0, (cudaStream_t)stream));
}

sn_status sn_grads_clip(sn_grads_t g, const double *sumsq, float max_norm, float *norm, sn_stream_t stream)
{
    const sn_status st = check_grads(g);
    if (st != SN_OK)
        return st;
    if (!sumsq || !norm || !(max_norm > 0.f) || !std::isfinite(max_norm))
        return SN_ERR_INVALID_ARG;
    if (!aligned(sumsq, 8) || !aligned(norm, 4))
        return SN_ERR_ALIGNMENT;
    if (overlap(sumsq, 8, norm, 4) || !on_device({sumsq, norm}))
        return SN_ERR_INVALID_ARG;
    return cuda_status(sn::grads_clip(*g, sumsq, max_norm, norm, (cudaStream_t)stream));
}

sn_status sn_wire_bytes(sn_basis_t b, sn_dtype dt, int64_t T, size_t *bytes)
{
    if (!b || !bytes || T < 0 || (dt != SN_BF16 && dt != SN_F32))
        return SN_ERR_INVALID_ARG;
    *bytes = (size_t)T * (size_t)b->k * esize(dt);
    return SN_OK;
}

sn_status sn_wire_send(const void *src_device, void *dst_host, size_t bytes, sn_stream_t stream)
{
    if (bytes == 0)
        return SN_OK;
    if (!src_device || !dst_host || !on_device({src_device}))
        return SN_ERR_INVALID_ARG;
    return cuda_status(cudaMemcpyAsync(dst_host, src_device, bytes, cudaMemcpyDeviceToHost,
                                       (cudaStream_t)stream));
}

sn_status sn_wire_recv(const void *src_host, void *dst_device, size_t bytes, sn_stream_t stream)
{
    if (bytes == 0)
        return SN_OK;
    if (!src_host || !dst_device || !on_device({dst_device}))
        return SN_ERR_INVALID_ARG;
    return cuda_status(cudaMemcpyAsync(dst_device, src_host, bytes, cudaMemcpyHostToDevice,
                                       (cudaStream_t)stream));
}

sn_status sn_check_errors(sn_basis_t b, sn_stream_t stream)
{
    unsigned int word = 0, unclaimed = 0;
    cudaError_t e = cudaStreamSynchronize((cudaStream_t)stream);
    if (e == cudaSuccess && b)
        e = cudaMemcpy(&word, b->err, sizeof word, cudaMemcpyDeviceToHost);
    if (e == cudaSuccess && word)
        e = cudaMemset(b->err, 0, sizeof word);
    if (e == cudaSuccess)
        e = sn::take_unclaimed(&unclaimed);
    if (e != cudaSuccess)
        return SN_ERR_CUDA;
    word |= unclaimed;
    if (word & SN_EBIT_TIMEOUT)
        return SN_ERR_TIMEOUT;
    if (word & SN_EBIT_BAD_ID)
        return SN_ERR_BAD_ID;
    if (word & SN_EBIT_NUMERIC)
        return SN_ERR_NUMERIC;
    return SN_OK;
}

}  // extern "C"
