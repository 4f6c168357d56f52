// The page calls of the 4-bit cache over a runtime that refuses launches: linked with qp_kv_pages.cu alone, everything that it needs
// from the runtime and from the rest of the library stands below.  No GPU is used.
#include <cstdio>
#include <cstring>

#include "qp_internal.cuh"

static int launches, refuse;                     // launches asked for; number of the one that is refused (0: none)
static cudaError_t last;

extern "C" {
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t*, const void*, void**)
{
    if (++launches == refuse) return last = cudaErrorLaunchOutOfResources;
    return cudaSuccess;
}
cudaError_t cudaLaunchKernel(const void*, dim3, dim3, void**, size_t, cudaStream_t) { return cudaErrorUnknown; }
cudaError_t cudaGetDevice(int* d) { *d = 0; return cudaSuccess; }
cudaError_t cudaSetDevice(int) { return cudaSuccess; }
void** __cudaRegisterFatBinary(void*) { static void* handle; return &handle; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
void __cudaRegisterFunction(void**, const char*, char*, const char*, int, uint3*, uint3*, dim3*, dim3*, int*) {}
unsigned __cudaPushCallConfiguration(dim3, dim3, size_t, void*) { return 0; }
cudaError_t __cudaPopCallConfiguration(dim3*, dim3*, size_t*, void*) { return cudaSuccess; }
uint64_t qp_kv_slice_bytes(int d) { return 16 * (uint64_t)(d + 16); }
}

int32_t qp_fail(qp_ctx*, int32_t status, const char*) { return status; }
int32_t qp_check_launch(qp_ctx*, const char*)
{
    const cudaError_t e = last;
    last = cudaSuccess;
    return e == cudaSuccess ? QP_OK : QP_ERR_CUDA;
}
int32_t qp_kv_check_cache(qp_ctx*, const qp_kv_cache_t*) { return QP_OK; }
int32_t qp_kv_check_batch(qp_ctx*, const qp_kv_batch_t*) { return QP_OK; }

int main()
{
    static int32_t ints[4096];
    static char pool[1 << 16];
    qp_ctx ctx;
    memset(&ctx, 0, sizeof ctx);
    ctx.sm_count = 148;
    qp_kv_cache_t c;
    memset(&c, 0, sizeof c);
    c.d_pool = pool;
    c.d_table = ints; c.d_lens = ints + 64; c.d_refs = ints + 128; c.d_work = ints + 256;
    c.layers = 1; c.num_pages = 8; c.heads = 1; c.head_dim = 64; c.page_size = 16; c.max_seqs = 8; c.max_pages = 4;
    int32_t (*calls[3])(qp_ctx*, const qp_kv_cache_t*, const int32_t*) = {
        [](qp_ctx* x, const qp_kv_cache_t* k, const int32_t* l) { return qp_kv_fork(x, k, l, l + 2, 2, nullptr); },
        [](qp_ctx* x, const qp_kv_cache_t* k, const int32_t* l) { return qp_kv_copy_pages(x, k, l, l + 2, 2, nullptr); },
        [](qp_ctx* x, const qp_kv_cache_t* k, const int32_t*) { return qp_kv_compact(x, k, nullptr, nullptr); }};
    const char* names[3] = {"fork", "copy_pages", "compact"};
    int bad = 0;
    for (int f = 0; f < 3; ++f)
        for (refuse = 0; refuse <= 2; ++refuse) {
            launches = 0;
            const int32_t rc = calls[f](&ctx, &c, ints + 512);
            // a refused first launch is the last: the second would move pages by lists that nobody has written
            if (rc != (refuse ? QP_ERR_CUDA : QP_OK) || launches != (refuse == 1 ? 1 : 2)) {
                fprintf(stderr, "%s, launch %d refused: status %d, %d launches asked for\n", names[f], refuse, (int)rc, launches);
                ++bad;
            }
        }
    if (!bad) puts("ok");
    return bad != 0;
}
