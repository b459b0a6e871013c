// Tokens into 4-bit blocks through a slot map, and 4-bit blocks back to bf16.  Both stream: 512 B of bf16 rows against
// 160 B of codes and scales per (token, KV head), a handful of operations per value.  Measured on a B200 at 65536 tokens of 8
// KV heads (352 MB each way): load 54.6 us, 6.4 TB/s, bound by HBM; store 80 us, 4.4 TB/s, where issuing its 131
// instructions per (token, head), 56 of them for the quotients, takes as long as the memory.
#include "pi_kv4.cuh"

namespace {

constexpr int KV4_THREADS = 256;
constexpr int KV4_WARPS = KV4_THREADS / 32;
constexpr int KV4_UNROLL = 2;                       // pairs of (token, head) items a warp has in flight: 2 KB of loads
constexpr int KV4_ITEMS = 2 * KV4_UNROLL;

struct StoreParams {
    const __nv_bfloat16* k;
    const __nv_bfloat16* v;
    long long k_tok, k_head, k_outer, v_tok, v_head, v_outer;      // strides in elements
    const int64_t* slots;
    unsigned char* store;
    pi_status_ref st;
    long long n_items, block_bytes, n_slots;
    int inner, log_h, shift;                        // Hkv = 1 << log_h, B = 1 << shift
};

// Eight lanes take a row, a warp the K and V rows of two (token, head) items at a time, KV4_ITEMS consecutive items in all:
// heads of one token (ONE_TOKEN: Hkv is a multiple of KV4_ITEMS), whose rows lie next to each other in the projections, or
// of several.
template <bool ONE_TOKEN>
__global__ void __launch_bounds__(KV4_THREADS)
kv4_store_kernel(StoreParams p) {
    const int lane = threadIdx.x & 31, l = lane & 7;
    const bool is_v = lane & 8;
    const long long first = (static_cast<long long>(blockIdx.x) * KV4_WARPS + (threadIdx.x >> 5)) * KV4_ITEMS;
    const int heads = (1 << p.log_h) - 1, rows = (1 << p.shift) - 1;
    const __nv_bfloat16* base = (is_v ? p.v : p.k) + 16 * l;
    const long long s_tok = is_v ? p.v_tok : p.k_tok, s_head = is_v ? p.v_head : p.k_head, s_outer = is_v ? p.v_outer : p.k_outer;
    pi_grid_dependency_wait();
    pi_launch_dependents();
    auto row_of = [&](long long item) {
        const int t = static_cast<int>(item >> p.log_h);
        int outer = 0, in = t;
        if (p.inner) { outer = t / p.inner; in = t - outer * p.inner; }
        return base + outer * s_outer + in * s_tok + (static_cast<int>(item) & heads) * s_head;
    };
    auto slot_of = [&](long long item) -> long long { const int t = static_cast<int>(item >> p.log_h); return p.slots ? p.slots[t] : t; };
    // the tile of a slot for head 0, nullptr where nothing is to be written
    auto tile_of = [&](long long item, long long s) -> unsigned char* {
        if (s < 0) return nullptr;
        if (s >= p.n_slots) {
            if (l == 0) pi_report(p.st, PI_ERR_INDEX_RANGE, PI_STAGE_KV4, static_cast<int>(item >> p.log_h), static_cast<int>(item) & heads, static_cast<int>(min(s, 0x7fffffffLL)));
            return nullptr;
        }
        return p.store + (s >> p.shift) * p.block_bytes + ((static_cast<int>(s) & rows) >> 4) * KV4_TILE_BYTES;
    };
    const int head_bytes = KV4_TILE_BYTES << (p.shift - 4);
    const long long mine = first + (lane >> 4);                  // this lane's items: mine, mine + 2, ...
    uint4 x[KV4_UNROLL][2];
    if (ONE_TOKEN) {
        if (first >= p.n_items) return;
        const __nv_bfloat16* src = row_of(mine);
#pragma unroll
        for (int u = 0; u < KV4_UNROLL; ++u) {
            x[u][0] = __ldg(reinterpret_cast<const uint4*>(src + 2 * u * s_head));
            x[u][1] = __ldg(reinterpret_cast<const uint4*>(src + 2 * u * s_head) + 1);
        }
        const long long slot = slot_of(first);
        unsigned char* tile = tile_of(first, slot);
        const bool write = tile != nullptr;
        tile += (static_cast<int>(mine) & heads) * head_bytes;
#pragma unroll
        for (int u = 0; u < KV4_UNROLL; ++u) {
            uint32_t codes[2], sz;
            kv4_quantise(x[u], codes, sz);
            kv4_write_row(tile + 2 * u * head_bytes, static_cast<int>(slot) & 15, is_v, l, codes, sz, write);
        }
    } else {
        long long slot[KV4_UNROLL];
#pragma unroll
        for (int u = 0; u < KV4_UNROLL; ++u) {
            const bool has = mine + 2 * u < p.n_items;
            const uint4* src = has ? reinterpret_cast<const uint4*>(row_of(mine + 2 * u)) : nullptr;
            x[u][0] = has ? __ldg(src) : make_uint4(0, 0, 0, 0);
            x[u][1] = has ? __ldg(src + 1) : make_uint4(0, 0, 0, 0);
            slot[u] = has ? slot_of(mine + 2 * u) : -1;
        }
#pragma unroll
        for (int u = 0; u < KV4_UNROLL; ++u) {
            uint32_t codes[2], sz;
            kv4_quantise(x[u], codes, sz);
            unsigned char* tile = tile_of(mine + 2 * u, slot[u]);
            kv4_write_row(tile + (static_cast<int>(mine + 2 * u) & heads) * head_bytes, static_cast<int>(slot[u]) & 15, is_v, l, codes, sz, tile != nullptr);
        }
    }
}

struct LoadParams {
    const unsigned char* store;
    const int32_t* blocks;
    uint4* out;                                     // [n_out][Hkv][2][B][D] bf16, 16 uint4 a row
    pi_status_ref st;
    long long n_items, block_bytes, n_blocks;       // an item is a (block, head, tile)
    int log_tiles, log_h, B;
};

// Eight channels of a row: the codes of `w` (nibble i = channel i) times the scale plus the minimum of `sz`.  0x4300 | code
// is the bf16 number 128 + code; a fused multiply-add of bf16 pairs rounds once, from the exact value.
__device__ __forceinline__ uint4 kv4_eight(uint32_t w, uint32_t sz) {
    const uint32_t s2 = __byte_perm(sz, sz, 0x1010), z2 = __byte_perm(sz, sz, 0x3232);
    const __nv_bfloat162 less = __halves2bfloat162(__ushort_as_bfloat16(0xc300), __ushort_as_bfloat16(0xc300));     // -128
    uint32_t p[4];                                  // channels (n, n + 4)
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        const uint32_t raised = ((w >> (4 * n)) & 0x000f000fu) | 0x43004300u;
        const __nv_bfloat162 v = __hfma2(__hadd2(*reinterpret_cast<const __nv_bfloat162*>(&raised), less),
                                         *reinterpret_cast<const __nv_bfloat162*>(&s2), *reinterpret_cast<const __nv_bfloat162*>(&z2));
        p[n] = *reinterpret_cast<const uint32_t*>(&v);
    }
    return make_uint4(__byte_perm(p[0], p[1], 0x5410), __byte_perm(p[2], p[3], 0x5410), __byte_perm(p[0], p[1], 0x7632), __byte_perm(p[2], p[3], 0x7632));
}

// One warp a tile: four lanes a row, each 16 bytes of codes (the same eight channels of all four groups), all loads of the
// tile before the first store.
__global__ void __launch_bounds__(KV4_THREADS)
kv4_load_kernel(LoadParams p) {
    const int lane = threadIdx.x & 31, row = lane >> 2, c = lane & 3;
    const long long item = static_cast<long long>(blockIdx.x) * KV4_WARPS + (threadIdx.x >> 5);
    pi_grid_dependency_wait();
    pi_launch_dependents();
    if (item >= p.n_items) return;
    const int tile = static_cast<int>(item) & ((1 << p.log_tiles) - 1), h = static_cast<int>(item >> p.log_tiles) & ((1 << p.log_h) - 1);
    const long long i = item >> (p.log_tiles + p.log_h);
    const long long block = p.blocks ? p.blocks[i] : i;
    if (block < 0 || block >= p.n_blocks) {
        if (lane == 0 && tile == 0 && h == 0) pi_report(p.st, PI_ERR_INDEX_RANGE, PI_STAGE_KV4, static_cast<int>(min(i, 0x7fffffffLL)), 0, static_cast<int>(block));
        return;
    }
    const unsigned char* src = p.store + block * p.block_bytes + ((h << p.log_tiles) + tile) * KV4_TILE_BYTES;
    uint4* dst = p.out + (((((i << p.log_h) + h) * 2) * p.B + tile * 16 + row) * 16 + c);
    uint4 codes[4], scales[4];                      // K rows 0..7, 8..15, then V
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        codes[u] = *reinterpret_cast<const uint4*>(src + (u >> 1) * KV4_V_CODES + ((u & 1) * 8 + row) * 64 + c * 16);
        scales[u] = *reinterpret_cast<const uint4*>(src + KV4_K_SCALES + (u >> 1) * (KV4_V_SCALES - KV4_K_SCALES) + ((u & 1) * 8 + row) * 16);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const uint32_t x[4] = {codes[u].x, codes[u].y, codes[u].z, codes[u].w}, sz[4] = {scales[u].x, scales[u].y, scales[u].z, scales[u].w};
        uint4* to = dst + (static_cast<long long>(u >> 1) * p.B + (u & 1) * 8) * 16;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            // a K chunk is four words, one a group; a V chunk two runs of four halves, channels 0..3 and 4..7 of the eight
            const uint32_t w = u < 2 ? x[j] : __byte_perm(x[j >> 1], x[2 + (j >> 1)], (j & 1) ? 0x7632 : 0x5410);
            to[4 * j] = kv4_eight(w, sz[j]);
        }
    }
}

int log2_of(int x) {
    int n = 0;
    while ((1 << n) < x) ++n;
    return n;
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
    p.log_h = log2_of(c->cfg.n_kv_heads);           // (a power of two: pi_create)
    p.n_items = n_tokens * c->cfg.n_kv_heads;
    p.block_bytes = kv4_block_bytes(c->cfg.n_kv_heads, c->cfg.block_tokens);
    p.n_slots = n_blocks * c->cfg.block_tokens;
    p.inner = inner;
    p.shift = log2_of(c->cfg.block_tokens);
    const long long per_cta = KV4_WARPS * KV4_ITEMS;
    PI_CUDA_TRY(pi_launch_pdl(c->cfg.n_kv_heads % KV4_ITEMS == 0 ? kv4_store_kernel<true> : kv4_store_kernel<false>, dim3(static_cast<unsigned>((p.n_items + per_cta - 1) / per_cta)), dim3(KV4_THREADS), 0, stream, p));
    return PI_OK;
}

int pi_launch_kv4_load(pi_ctx* c, int64_t n_out, const void* store, int64_t n_blocks, const int32_t* blocks, void* out, cudaStream_t stream) {
    LoadParams p;
    p.store = static_cast<const unsigned char*>(store);
    p.blocks = blocks;
    p.out = static_cast<uint4*>(out);
    p.st = pi_status_of(c);
    p.B = c->cfg.block_tokens;
    p.log_h = log2_of(c->cfg.n_kv_heads); p.log_tiles = log2_of(p.B / 16);
    p.n_items = n_out << (p.log_h + p.log_tiles);
    p.block_bytes = kv4_block_bytes(c->cfg.n_kv_heads, c->cfg.block_tokens);
    p.n_blocks = n_blocks;
    PI_CUDA_TRY(pi_launch_pdl(kv4_load_kernel, dim3(static_cast<unsigned>((p.n_items + KV4_WARPS - 1) / KV4_WARPS)), dim3(KV4_THREADS), 0, stream, p));
    return PI_OK;
}
