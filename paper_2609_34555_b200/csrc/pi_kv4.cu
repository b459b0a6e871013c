// Tokens into 4-bit blocks through a slot map, and 4-bit blocks back to bf16.  Both stream: 512 B of bf16 rows against
// 160 B of codes and scales per (token, KV head), a handful of operations per value, bound by HBM.
#include "pi_kv4.cuh"

namespace {

constexpr int KV4_THREADS = 256;
constexpr int KV4_WARPS = KV4_THREADS / 32;
constexpr int KV4_UNROLL = 4;                       // (token, head) items a warp has in flight: 2 KB of loads

struct StoreParams {
    const __nv_bfloat16* k;
    const __nv_bfloat16* v;
    long long k_tok, k_head, k_outer, v_tok, v_head, v_outer;      // strides in elements
    const int64_t* slots;
    unsigned char* store;
    pi_status_ref st;
    long long n_items, block_bytes, n_slots;
    int inner, H, shift;                            // B = 1 << shift
};

// Half a warp takes the K row of a (token, head), the other half its V row; consecutive items are the heads of a token,
// whose rows lie next to each other in the projections.
__global__ void __launch_bounds__(KV4_THREADS)
kv4_store_kernel(StoreParams p) {
    const int lane = threadIdx.x & 31, l = lane & 15;
    const bool is_v = lane >> 4;
    const long long first = (static_cast<long long>(blockIdx.x) * KV4_WARPS + (threadIdx.x >> 5)) * KV4_UNROLL;
    pi_grid_dependency_wait();
    pi_launch_dependents();
    uint4 x[KV4_UNROLL];
    long long slot[KV4_UNROLL];
#pragma unroll
    for (int u = 0; u < KV4_UNROLL; ++u) {
        const long long item = first + u;
        x[u] = make_uint4(0, 0, 0, 0);
        slot[u] = -1;
        if (item < p.n_items) {
            const int t = static_cast<int>(item / p.H), h = static_cast<int>(item - static_cast<long long>(t) * p.H);
            const long long outer = p.inner ? t / p.inner : 0, in = p.inner ? t % p.inner : t;
            slot[u] = p.slots ? p.slots[t] : t;
            const __nv_bfloat16* src = is_v ? p.v + outer * p.v_outer + in * p.v_tok + h * p.v_head
                                            : p.k + outer * p.k_outer + in * p.k_tok + h * p.k_head;
            x[u] = __ldg(reinterpret_cast<const uint4*>(src) + l);
        }
    }
#pragma unroll
    for (int u = 0; u < KV4_UNROLL; ++u) {
        uint32_t codes, sz;
        kv4_quantise(x[u], codes, sz);
        const long long item = first + u;
        bool write = slot[u] >= 0;
        if (write && slot[u] >= p.n_slots) {
            if (lane == 0) pi_report(p.st, PI_ERR_INDEX_RANGE, PI_STAGE_KV4, static_cast<int>(item / p.H), static_cast<int>(item % p.H), static_cast<int>(min(slot[u], 0x7fffffffLL)));
            write = false;
        }
        const long long s = write ? slot[u] : 0;
        const int at = static_cast<int>(s & ((1 << p.shift) - 1)), h = static_cast<int>(item % p.H);
        unsigned char* tile = p.store + (s >> p.shift) * p.block_bytes +
                              (static_cast<long long>(h) << (p.shift - 4)) * KV4_TILE_BYTES + (at >> 4) * KV4_TILE_BYTES;
        kv4_write_row(tile, at & 15, is_v, l, codes, sz, write);
    }
}

struct LoadParams {
    const unsigned char* store;
    const int32_t* blocks;
    uint4* out;                                     // [n_out][Hkv][2][B][D] bf16, 16 uint4 a row
    pi_status_ref st;
    long long n_items, block_bytes, n_blocks;       // an item is a (block, head, tile)
    int tiles, H, B;
};

// One warp a tile; lanes 0..15 take a K row, lanes 16..31 the V row of the same token, 16 bytes of output a lane.
__global__ void __launch_bounds__(KV4_THREADS)
kv4_load_kernel(LoadParams p) {
    const int lane = threadIdx.x & 31, l = lane & 15;
    const bool is_v = lane >> 4;
    const long long item = static_cast<long long>(blockIdx.x) * KV4_WARPS + (threadIdx.x >> 5);
    pi_grid_dependency_wait();
    pi_launch_dependents();
    if (item >= p.n_items) return;
    const int tile = static_cast<int>(item % p.tiles), h = static_cast<int>(item / p.tiles % p.H);
    const long long i = item / p.tiles / p.H;
    const long long block = p.blocks ? p.blocks[i] : i;
    if (block < 0 || block >= p.n_blocks) {
        if (lane == 0 && tile == 0 && h == 0) pi_report(p.st, PI_ERR_INDEX_RANGE, PI_STAGE_KV4, static_cast<int>(min(i, 0x7fffffffLL)), 0, static_cast<int>(block));
        return;
    }
    const unsigned char* src = p.store + block * p.block_bytes + (static_cast<long long>(h) * p.tiles + tile) * KV4_TILE_BYTES;
    uint4* dst = p.out + (((i * p.H + h) * 2 + (is_v ? 1 : 0)) * p.B + tile * 16) * 16 + l;
    const int j = l >> 2, c = l & 3;
    const unsigned char* codes = src + (is_v ? KV4_V_CODES + 16 * c + 2 * j : 16 * c + 4 * j);
    const unsigned char* scales = src + (is_v ? KV4_V_SCALES : KV4_K_SCALES) + 4 * j;
#pragma unroll 8
    for (int t = 0; t < 16; ++t) {
        uint32_t w;
        if (is_v) {      // channels 8 c .. 8 c + 3 of group j sit at byte 16 c + 2 j, the next four 8 bytes further on
            w = *reinterpret_cast<const uint16_t*>(codes + t * 64) |
                (static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(codes + t * 64 + 8)) << 16);
        } else {
            w = *reinterpret_cast<const uint32_t*>(codes + t * 64);
        }
        const uint32_t sz = *reinterpret_cast<const uint32_t*>(scales + t * 16);
        const float s = kv4_scale_of(sz), z = kv4_min_of(sz);
        uint32_t o[4];
#pragma unroll
        for (int i2 = 0; i2 < 4; ++i2) {
            // scale * code has at most 12 bits and is exact: one rounding in the sum, one to bf16
            const float a = fmaf(s, static_cast<float>((w >> (8 * i2)) & 15u), z), b = fmaf(s, static_cast<float>((w >> (8 * i2 + 4)) & 15u), z);
            const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
            o[i2] = *reinterpret_cast<const uint32_t*>(&v);
        }
        dst[t * 16] = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

}  // namespace

int pi_launch_kv4_store(pi_ctx* c, int64_t n_tokens, const void* k, const int64_t (&ks)[3], const void* v, const int64_t (&vs)[3],
                        int inner, const int64_t* slots, void* store, int64_t n_blocks, cudaStream_t stream) {
    StoreParams p;
    p.k = static_cast<const __nv_bfloat16*>(k); p.v = static_cast<const __nv_bfloat16*>(v);
    p.k_tok = ks[0]; p.k_head = ks[1]; p.k_outer = ks[2];
    p.v_tok = vs[0]; p.v_head = vs[1]; p.v_outer = vs[2];
    p.slots = slots;
    p.store = static_cast<unsigned char*>(store);
    p.st = pi_status_of(c);
    p.H = c->cfg.n_kv_heads;
    p.n_items = n_tokens * p.H;
    p.block_bytes = kv4_block_bytes(c->cfg.n_kv_heads, c->cfg.block_tokens);
    p.n_slots = n_blocks * c->cfg.block_tokens;
    p.inner = inner;
    p.shift = c->cfg.block_tokens == 16 ? 4 : c->cfg.block_tokens == 32 ? 5 : 6;
    const long long per_cta = KV4_WARPS * KV4_UNROLL;
    PI_CUDA_TRY(pi_launch_pdl(kv4_store_kernel, dim3(static_cast<unsigned>((p.n_items + per_cta - 1) / per_cta)), dim3(KV4_THREADS), 0, stream, p));
    return PI_OK;
}

int pi_launch_kv4_load(pi_ctx* c, int64_t n_out, const void* store, int64_t n_blocks, const int32_t* blocks, void* out, cudaStream_t stream) {
    LoadParams p;
    p.store = static_cast<const unsigned char*>(store);
    p.blocks = blocks;
    p.out = static_cast<uint4*>(out);
    p.st = pi_status_of(c);
    p.H = c->cfg.n_kv_heads; p.B = c->cfg.block_tokens; p.tiles = p.B / 16;
    p.n_items = n_out * p.H * p.tiles;
    p.block_bytes = kv4_block_bytes(c->cfg.n_kv_heads, c->cfg.block_tokens);
    p.n_blocks = n_blocks;
    PI_CUDA_TRY(pi_launch_pdl(kv4_load_kernel, dim3(static_cast<unsigned>((p.n_items + KV4_WARPS - 1) / KV4_WARPS)), dim3(KV4_THREADS), 0, stream, p));
    return PI_OK;
}
