// gfx950 kernels of the mixed-batch paged-attention path and their launchers.
//
//   kv_append_kernel   scatter this iteration's K/V rows into the paged pools      (HBM-bound)
//   kv_gather_kernel   un-paged copy of one sequence (test hook)                   (HBM-bound)
//   kv_migrate_kernel  pool <-> contiguous transfer buffer, all layers (paper Sec. 3.5)   (HBM-bound)
//   the attention kernels of tc_attention.h over pools in 16 bits, bf16 and IEEE half
#include <cstdlib>

#include "tc_attention.h"

namespace tc {

// ------------------------------------------------------------------------------------
// KV append / gather
// ------------------------------------------------------------------------------------
// One workgroup writes the rows one sequence adds to one page (1..16 consecutive token indices) for
// one KV head.  K: a thread copies the 16 bytes (8 head-dim elements) of one token.  V is
// token-minor in the pool, so a thread owns one head-dim element and four consecutive token
// slots: it reads up to four 2-byte values (adjacent lanes read adjacent elements, so the reads
// coalesce) and, when all four tokens are new, stores them as one 8-byte word; otherwise it stores
// only the new tokens, 2 bytes each, so every other pool byte stays untouched.
template <int D>
__global__ void __launch_bounds__(4 * D) kv_append_kernel(uint16_t *__restrict__ k_pool, uint16_t *__restrict__ v_pool,
                                                          const uint16_t *__restrict__ k_new,
                                                          const uint16_t *__restrict__ v_new,
                                                          const int32_t *__restrict__ segments, int Hkv) {
    const int32_t *seg = segments + (int64_t)blockIdx.x * kAppendInts;
    const int h = blockIdx.y;
    const int row0 = seg[0], n_tok = seg[1], tok0 = seg[2];
    const int64_t tile = ((int64_t)seg[3] * Hkv + h) * (int64_t)(kBlock * D);
    const int tid = threadIdx.x;
    // ---- V: thread = (slot group g, element d); slots 4g..4g+3 hold tokens t(g)..t(g)+3, t = v_slot(4g)
    {
        const int d = tid % D, g = tid / D;
        const int t_first = v_slot(4 * g);  // token index stored in slot 4g
        uint16_t val[4];
        bool have[4];
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const int t = t_first + e;
            have[e] = t >= tok0 && t < tok0 + n_tok;
            val[e] = have[e] ? v_new[((int64_t)(row0 + t - tok0) * Hkv + h) * D + d] : (uint16_t)0;
        }
        uint16_t *dst = v_pool + tile + (int64_t)d * kBlock + 4 * g;
        if (have[0] && have[1] && have[2] && have[3]) {
            *reinterpret_cast<u32x2 *>(dst) = u32x2{(uint32_t)val[0] | ((uint32_t)val[1] << 16), (uint32_t)val[2] | ((uint32_t)val[3] << 16)};
        } else {
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (have[e]) dst[e] = val[e];
        }
    }
    // ---- K: thread = (token, 8-element piece)
    constexpr int CH = D / 8;
    for (int x = tid; x < n_tok * CH; x += 4 * D) {
        const int i = x / CH, c = x % CH;
        const u32x4 kv = *reinterpret_cast<const u32x4 *>(k_new + ((int64_t)(row0 + i) * Hkv + h) * D + c * 8);
        *reinterpret_cast<u32x4 *>(k_pool + tile + ((int64_t)c * kBlock + tok0 + i) * 8) = kv;
    }
}

template <int D>
__global__ void __launch_bounds__(256) kv_gather_kernel(const uint16_t *__restrict__ k_pool,
                                                        const uint16_t *__restrict__ v_pool,
                                                        const int32_t *__restrict__ pages, int kv_len, int Hkv,
                                                        uint16_t *__restrict__ k_out, uint16_t *__restrict__ v_out) {
    constexpr int CH = D / 8;
    const int64_t gid = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    const int64_t total = (int64_t)kv_len * Hkv * CH;
    if (gid >= total) return;
    const int c = (int)(gid % CH);
    const int h = (int)((gid / CH) % Hkv);
    const int j = (int)(gid / ((int64_t)CH * Hkv));
    const int64_t blk = pages[j / kBlock];
    const int tok = j % kBlock;
    const int64_t tile = (blk * Hkv + h) * (int64_t)(kBlock * D);
    const int64_t dst = ((int64_t)j * Hkv + h) * D + c * 8;
    *reinterpret_cast<u32x4 *>(k_out + dst) = *reinterpret_cast<const u32x4 *>(k_pool + tile + ((int64_t)c * kBlock + tok) * 8);
    const uint16_t *vsrc = v_pool + tile + (int64_t)(c * 8) * kBlock + v_slot(tok);
    u32x4 vv;
#pragma unroll
    for (int e = 0; e < 4; e++) vv[e] = (uint32_t)vsrc[(2 * e) * kBlock] | ((uint32_t)vsrc[(2 * e + 1) * kBlock] << 16);
    *reinterpret_cast<u32x4 *>(v_out + dst) = vv;
}

// ------------------------------------------------------------------------------------
// KV migration: pool <-> contiguous transfer buffer, every layer in one launch
// ------------------------------------------------------------------------------------
// The transfer buffer is [layers][pages][K block | V block] with both blocks in the pool's own
// layout, so a page moves as 16-byte pieces that are contiguous on both sides; the block id is
// the only indirection.  Workgroup (x, y) moves page x of the selection for layer y.  A full page
// is a straight copy with eight non-temporal loads in flight per thread (the data is touched once).  The last page of a sequence may hold
// fewer than 16 tokens: the export writes zero for the missing ones, the import stores only the
// real ones (K: 16-byte pieces of real tokens; V, which is token-minor: 2-byte elements).
struct MigratePools {
    uint16_t *k[kMigrateLayers];
    uint16_t *v[kMigrateLayers];
};

template <bool IMPORT>
__global__ void __launch_bounds__(256) kv_migrate_kernel(const MigratePools pools, const int32_t *__restrict__ pages,
                                                         const int32_t *__restrict__ valid, uint16_t *__restrict__ buffer,
                                                         int64_t layer_stride, int block_pieces) {
    const int page = blockIdx.x, layer = blockIdx.y;
    const int64_t blk = pages[page];
    const int n_valid = valid[page];
    const int64_t E = (int64_t)block_pieces * 8;  // elements of one block of one pool
    u32x4 *kb = reinterpret_cast<u32x4 *>(buffer + (int64_t)layer * layer_stride + (int64_t)page * 2 * E);
    u32x4 *vb = kb + block_pieces;
    u32x4 *kp = reinterpret_cast<u32x4 *>(pools.k[layer] + blk * E);
    u32x4 *vp = reinterpret_cast<u32x4 *>(pools.v[layer] + blk * E);
    const int tid = threadIdx.x;
    if (n_valid == kBlock) {
        const u32x4 *src_k = IMPORT ? kb : kp, *src_v = IMPORT ? vb : vp;
        u32x4 *dst_k = IMPORT ? kp : kb, *dst_v = IMPORT ? vp : vb;
        constexpr int U = 4;  // pieces of each tensor in flight per thread
        for (int x0 = tid; x0 < block_pieces; x0 += 256 * U) {
            u32x4 a[U], b[U];
#pragma unroll
            for (int u = 0; u < U; u++) {
                const int x = x0 + 256 * u;
                if (x < block_pieces) {
                    a[u] = __builtin_nontemporal_load(src_k + x);
                    b[u] = __builtin_nontemporal_load(src_v + x);
                }
            }
#pragma unroll
            for (int u = 0; u < U; u++) {
                const int x = x0 + 256 * u;
                if (x < block_pieces) {
                    __builtin_nontemporal_store(a[u], dst_k + x);
                    __builtin_nontemporal_store(b[u], dst_v + x);
                }
            }
        }
        return;
    }
    for (int x = tid; x < block_pieces; x += 256) {
        // K piece x = (head, d/8, token): the token index is the piece index mod 16
        const bool real = (x & (kBlock - 1)) < n_valid;
        if (IMPORT) {
            if (real) kp[x] = kb[x];
        } else {
            kb[x] = real ? kp[x] : u32x4{0u, 0u, 0u, 0u};
        }
        // V piece x = (head, d, half row): slots 8*(x&1) .. +7, slot s holds token v_slot(s)
        const int slot0 = (x & 1) * 8;
        if (IMPORT) {
            const u32x4 w = vb[x];
            uint16_t *dst = reinterpret_cast<uint16_t *>(vp + x);
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (v_slot(slot0 + e) < n_valid) dst[e] = (uint16_t)(w[e >> 1] >> ((e & 1) * 16));
        } else {
            u32x4 w = vp[x];
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (v_slot(slot0 + e) >= n_valid) w[e >> 1] &= (e & 1) ? 0x0000FFFFu : 0xFFFF0000u;
            vb[x] = w;
        }
    }
}

// ------------------------------------------------------------------------------------
// Plan buffers
// ------------------------------------------------------------------------------------
int current_device(int *device) { return (int)hipGetDevice(device); }
const char *hip_error_text(int err) { return hipGetErrorString((hipError_t)err); }

int begin_plan_host(PlanImage *p, size_t n) {
    if (p->upload_event) {
        hipError_t e = hipEventSynchronize((hipEvent_t)p->upload_event);
        if (e != hipSuccess) return (int)e;
    }
    if (n <= p->host_cap) return 0;
    const size_t cap = std::max<size_t>(n + n / 2, 4096);
    int32_t *fresh = nullptr;
    if (p->on_device) {
        hipError_t e = hipHostMalloc((void **)&fresh, cap * sizeof(int32_t), hipHostMallocDefault);
        if (e != hipSuccess) return (int)e;
    } else {
        fresh = (int32_t *)std::malloc(cap * sizeof(int32_t));
        if (!fresh) return (int)hipErrorOutOfMemory;
    }
    if (p->host) {
        if (p->host_pinned) (void)hipHostFree(p->host); else std::free(p->host);
    }
    p->host = fresh;
    p->host_cap = cap;
    p->host_pinned = p->on_device;
    return 0;
}

// Copy the host image to the device on `stream`.  The device buffer grows when a work list is larger than
// any before it and is otherwise reused: a serving loop that keeps one plan object allocates nothing per
// iteration.  (Growing frees the old buffer, which waits for the device to finish whatever still reads it.)
int upload_plan(PlanImage *p, void *stream) {
    int device = -1;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return (int)e;
    if (p->device >= 0 && p->device != device) return (int)hipErrorInvalidDevice;
    p->device = device;
    if (p->host_n > p->dev_cap) {
        if (p->dev) (void)hipFree(p->dev);
        p->dev = nullptr;
        p->dev_cap = 0;
        e = hipMalloc((void **)&p->dev, p->host_cap * sizeof(int32_t));
        if (e != hipSuccess) { p->dev = nullptr; return (int)e; }
        p->dev_cap = p->host_cap;
    }
    if (!p->upload_event) {
        hipEvent_t ev;
        e = hipEventCreateWithFlags(&ev, hipEventDisableTiming);
        if (e != hipSuccess) return (int)e;
        p->upload_event = ev;
    }
    e = hipMemcpyAsync(p->dev, p->host, p->host_n * sizeof(int32_t), hipMemcpyHostToDevice, (hipStream_t)stream);
    if (e != hipSuccess) return (int)e;
    return (int)hipEventRecord((hipEvent_t)p->upload_event, (hipStream_t)stream);
}

void free_plan_buffers(PlanImage *p) {
    if (p->upload_event) {
        (void)hipEventSynchronize((hipEvent_t)p->upload_event);
        (void)hipEventDestroy((hipEvent_t)p->upload_event);
        p->upload_event = nullptr;
    }
    if (p->dev) (void)hipFree(p->dev);
    p->dev = nullptr;
    p->dev_cap = 0;
    if (p->host) {
        if (p->host_pinned) (void)hipHostFree(p->host); else std::free(p->host);
    }
    p->host = nullptr;
    p->host_cap = p->host_n = 0;
}

// ------------------------------------------------------------------------------------
// Launchers
// ------------------------------------------------------------------------------------
int launch_kv_append(const tc_plan *p, const tc_kv_pool *pool, const void *k_new, const void *v_new, bool only_prefill, void *stream) {
    const int n = only_prefill ? p->n_append_prefill : p->n_append;
    if (n == 0) return 0;
    hipStream_t st = (hipStream_t)stream;
    const dim3 grid((unsigned)n, (unsigned)p->Hkv);  // Hkv <= 1024 is checked when the plan is built
    if (p->D == 128)
        kv_append_kernel<128><<<grid, 512, 0, st>>>((uint16_t *)pool->k_pool, (uint16_t *)pool->v_pool, (const uint16_t *)k_new,
                                                   (const uint16_t *)v_new, p->dev + p->off_append, p->Hkv);
    else
        kv_append_kernel<64><<<grid, 256, 0, st>>>((uint16_t *)pool->k_pool, (uint16_t *)pool->v_pool, (const uint16_t *)k_new,
                                                  (const uint16_t *)v_new, p->dev + p->off_append, p->Hkv);
    return (int)hipGetLastError();
}

int launch_kv_gather(const tc_plan *p, const tc_kv_pool *pool, int seq, void *k_out, void *v_out, void *stream) {
    const int kv_len = p->ctx_len[seq] + (p->q_start[seq + 1] - p->q_start[seq]);
    const int64_t total = (int64_t)kv_len * p->Hkv * (p->D / 8);
    const unsigned blocks = (unsigned)((total + 255) / 256);
    hipStream_t st = (hipStream_t)stream;
    const int32_t *pages = p->dev + p->off_pages + p->page_off[seq];
    if (p->D == 128)
        kv_gather_kernel<128><<<blocks, 256, 0, st>>>((const uint16_t *)pool->k_pool, (const uint16_t *)pool->v_pool, pages, kv_len,
                                                     p->Hkv, (uint16_t *)k_out, (uint16_t *)v_out);
    else
        kv_gather_kernel<64><<<blocks, 256, 0, st>>>((const uint16_t *)pool->k_pool, (const uint16_t *)pool->v_pool, pages, kv_len,
                                                    p->Hkv, (uint16_t *)k_out, (uint16_t *)v_out);
    return (int)hipGetLastError();
}

int launch_kv_migrate(const tc_plan *p, bool import, int page0, int n_pages, int num_layers, void *const *k_pools,
                      void *const *v_pools, void *buffer, void *stream) {
    if (n_pages == 0) return 0;
    hipStream_t st = (hipStream_t)stream;
    const int block_pieces = p->Hkv * p->D * 2;  // 16-byte pieces of one block of one pool
    const int64_t layer_stride = (int64_t)n_pages * 2 * block_pieces * 8;  // buffer elements per layer
    const int32_t *pages = p->dev + p->off_pages + page0, *valid = p->dev + p->off_valid + page0;
    for (int l0 = 0; l0 < num_layers; l0 += kMigrateLayers) {
        const int nl = std::min(kMigrateLayers, num_layers - l0);
        MigratePools mp;
        for (int l = 0; l < kMigrateLayers; l++) {
            mp.k[l] = (uint16_t *)k_pools[l0 + std::min(l, nl - 1)];
            mp.v[l] = (uint16_t *)v_pools[l0 + std::min(l, nl - 1)];
        }
        uint16_t *buf = (uint16_t *)buffer + (int64_t)l0 * layer_stride;
        const dim3 grid((unsigned)n_pages, (unsigned)nl);
        if (import)
            kv_migrate_kernel<true><<<grid, 256, 0, st>>>(mp, pages, valid, buf, layer_stride, block_pieces);
        else
            kv_migrate_kernel<false><<<grid, 256, 0, st>>>(mp, pages, valid, buf, layer_stride, block_pieces);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return (int)e;
    }
    return 0;
}

int launch_attention(const tc_plan *p, const tc_kv_pool *pool, const void *q, const void *k_new, const void *v_new, void *out,
                     float scale, void *workspace, int launches, void *stream) {
    const AttnArgs A = attention_args(p, pool, nullptr, q, k_new, v_new, out, scale, workspace, launches);
    hipStream_t st = (hipStream_t)stream;
    if (p->dtype == TC_FP16) return p->D == 128 ? launch_attention_d<128, Fp16>(p, A, launches, st) : launch_attention_d<64, Fp16>(p, A, launches, st);
    return p->D == 128 ? launch_attention_d<128, Bf16>(p, A, launches, st) : launch_attention_d<64, Bf16>(p, A, launches, st);
}

// ------------------------------------------------------------------------------------
// Static scratch: a workspace for callers that cannot allocate
// ------------------------------------------------------------------------------------
// Partial results of split KV ranges for tc_mixed_attention_static.  Every GPU the library runs on holds
// its own copy of the array, at its own address, until the process ends.  Host code never uses the
// array's name as an address: the device address is asked for once per device and kept.
static __device__ __align__(256) unsigned char scratch[kStaticScratchBytes];

int static_scratch(int device, void **ptr, size_t *bytes) {
    static std::atomic<void *> address[kMaxDevices];
    *bytes = kStaticScratchBytes;
    *ptr = nullptr;
    if (device < 0 || device >= kMaxDevices) return (int)hipErrorInvalidDevice;
    void *a = address[device].load(std::memory_order_acquire);
    if (!a) {
        int current = -1;
        hipError_t e = hipGetDevice(&current);
        if (e != hipSuccess) return (int)e;
        if (current != device) return (int)hipErrorInvalidDevice;  // the address is that of the current device's copy
        e = hipGetSymbolAddress(&a, HIP_SYMBOL(scratch));
        if (e != hipSuccess) return (int)e;
        if (!a) return (int)hipErrorInvalidSymbol;
        address[device].store(a, std::memory_order_release);
    }
    *ptr = a;
    return 0;
}

}  // namespace tc

#ifdef TC_WG_TRACE
// Tracing build only: copy the first n int64 of the workgroup trace of the latest attention launch (over a cache in 16 bits) to HOST memory.
extern "C" int tc_debug_wg_trace(long long *dst, int n) {
    (void)hipDeviceSynchronize();
    return (int)hipMemcpyFromSymbol(dst, HIP_SYMBOL(tc::g_wg_trace), (size_t)n * sizeof(long long));
}
#endif
