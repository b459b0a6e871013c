// Tokens into 8-bit blocks through a slot map, and 8-bit blocks back to bf16 (format: pi_kv8.cuh).
//
// Store: 512 bytes a (token, KV head) in, 256 out.  The tokens of a block share a scale, so they are worked on together: one warp takes a run of
// tokens that go to the same block, for one head and K or V, finds the largest
// magnitude of its rows and writes the numbers; up to 16 rows stay in registers between the two, more come a second time, out of L2.  A block that the run does not begin keeps its
// other tokens; they are rounded again if its scale has to grow.
// Load: 256 bytes in, 512 out; one warp 16 rows.
// Measured on a B200, 131 072 tokens x 8 heads, 123 us of bytes each way: store 129 us for blocks of 32, 127 of 16, 146 of 64; load 120 us.
#include "pi_kv8.cuh"

namespace {

constexpr int KV8_THREADS = 128;
constexpr int KV8_WARPS = KV8_THREADS / 32;
constexpr int KEEP_FOURS = 4;                       // fours of rows in registers: longer runs are looked through, then fetched once more, which costs less than
                                                    // the warps that more registers take (blocks of 32: 137 us instead of 143; of 64: 144 instead of 163)

struct StoreParams {
    const __nv_bfloat16* k;
    const __nv_bfloat16* v;
    const int64_t* slots;
    unsigned char* store;
    pi_status_ref st;
    long long k_tok, k_head, k_outer, v_tok, v_head, v_outer;     // elements
    long long n_tokens, n_slots, block_bytes, n_items;
    int inner, log_h;
};

// B: tokens of a block.  Eight CTAs an SM: the rows of 32 warps are on their way (six CTAs of 80 registers: 137 us for blocks of 32, 144 of 16).  A warp has the runs that begin in a range of `RANGE` tokens, of one head's K or V.
template <int B>
__global__ void __launch_bounds__(KV8_THREADS, 8)
kv8_store_kernel(StoreParams p) {
    constexpr int RANGE = B < 32 ? B : 32, FOURS = B / 4, KEEP = KEEP_FOURS < FOURS ? KEEP_FOURS : FOURS, LOG_B = B == 16 ? 4 : B == 32 ? 5 : 6;
    const int lane = threadIdx.x & 31, quarter = lane >> 3, l = lane & 7;
    const long long item = static_cast<long long>(blockIdx.x) * KV8_WARPS + (threadIdx.x >> 5);
    pi_grid_dependency_wait();
    pi_launch_dependents();
    if (item >= p.n_items) return;
    const bool is_v = item & 1;
    const int h = static_cast<int>(item >> 1) & ((1 << p.log_h) - 1);
    const long long t0 = (item >> (1 + p.log_h)) * RANGE;
    // slot of a token; -1: none (skipped, or beyond the store, which is said)
    auto given = [&](long long t) -> long long { return t < 0 || t >= p.n_tokens ? -1 : p.slots ? p.slots[t] : t; };
    auto slot_of = [&](long long t) -> long long {
        const long long s = given(t);
        return s < p.n_slots ? s : -1;
    };
    const long long raw = given(t0 + lane), mine = raw < p.n_slots ? raw : -1, before = slot_of(t0 - 1);
    if (raw >= p.n_slots && !is_v && lane < RANGE) pi_report(p.st, PI_ERR_INDEX_RANGE, PI_STAGE_KV4, static_cast<int>(t0 + lane), h, static_cast<int>(raw < 0x7fffffffLL ? raw : 0x7fffffffLL));
    const long long block_mine = mine >= 0 ? mine >> LOG_B : -1, left = __shfl_up_sync(0xffffffffu, block_mine, 1);
    const long long block_left = lane ? left : before >= 0 ? before >> LOG_B : -1;
    unsigned begins = __ballot_sync(0xffffffffu, lane < RANGE && block_mine >= 0 && block_mine != block_left);
    const __nv_bfloat16* base = is_v ? p.v + h * p.v_head : p.k + h * p.k_head;
    const long long tok = is_v ? p.v_tok : p.k_tok, outer = is_v ? p.v_outer : p.k_outer;
    while (begins) {
        const int b0 = __ffs(static_cast<int>(begins)) - 1;
        begins &= begins - 1;
        const long long first = t0 + b0, block = __shfl_sync(0xffffffffu, block_mine, b0);
        // the run: tokens of this block, at most B of them; `at`: their places in it
        const long long s0 = B == 16 ? __shfl_sync(0xffffffffu, mine, (b0 + lane) & 31) : slot_of(first + lane), s1 = B > 32 ? slot_of(first + 32 + lane) : -1;
        const unsigned in0 = __ballot_sync(0xffffffffu, s0 >= 0 && (s0 >> LOG_B) == block), in1 = __ballot_sync(0xffffffffu, B > 32 && s1 >= 0 && (s1 >> LOG_B) == block);
        int n = in0 == 0xffffffffu ? 32 + (in1 == 0xffffffffu ? 32 : __ffs(static_cast<int>(~in1)) - 1) : __ffs(static_cast<int>(~in0)) - 1;
        n = min(n, B);                              // (of a run of 16 that begins among the first 16 tokens, all are at hand)
        const int at0 = static_cast<int>(s0) & (B - 1), at1 = static_cast<int>(s1) & (B - 1);
        // places that the run fills
        unsigned long long fills = lane < n ? 1ull << at0 : 0ull;
        if (B > 32 && 32 + lane < n) fills |= 1ull << at1;
        const unsigned f0 = __reduce_or_sync(0xffffffffu, static_cast<unsigned>(fills)), f1 = B > 32 ? __reduce_or_sync(0xffffffffu, static_cast<unsigned>(fills >> 32)) : 0u;
        // a block that comes back behind its run, as far as can be seen from here, or a slot named twice: what the block holds then is chance, which is said
        const unsigned long long in = in0 | static_cast<unsigned long long>(in1) << 32;
        if (!is_v && h == 0 && lane == 0 && ((n < 64 && in >> n) || __popc(f0) + __popc(f1) != n))
            pi_report(p.st, PI_ERR_INDEX_RANGE, PI_STAGE_KV4, static_cast<int>(first), n, static_cast<int>(block));
        // (token t is row t % inner of the outer index t / inner: one division a run, then a step at a time)
        const long long o0 = p.inner ? first / p.inner : 0, r0 = (p.inner ? first - o0 * p.inner : first) + quarter;
        // rows from the i0-th four on, KEEP fours of them: eight lanes a row, 32 bytes a lane
        auto fetch = [&](uint32_t (&x)[KEEP][8], int i0) {
            long long o = o0, r = r0 + 4 * i0;
#pragma unroll
            for (int i = 0; i < KEEP; ++i) {
                if (p.inner)
                    while (r >= p.inner) { r -= p.inner; ++o; }
                const uint4* from = reinterpret_cast<const uint4*>(base + o * outer + r * tok) + 2 * l;
                if (4 * (i0 + i) + quarter >= n) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[i][k] = 0u;
                } else {
                    const uint4 u = __ldg(from), v = __ldg(from + 1);
                    x[i][0] = u.x; x[i][1] = u.y; x[i][2] = u.z; x[i][3] = u.w;
                    x[i][4] = v.x; x[i][5] = v.y; x[i][6] = v.z; x[i][7] = v.w;
                }
                r += 4;
            }
        };
        uint32_t x[KEEP][8], most = 0u, some = 0u;  // largest magnitudes, NaN among them; of the finite ones
        for (int i0 = FOURS - KEEP; i0 >= 0; i0 -= KEEP) {
            fetch(x, i0);
            uint32_t here = 0u;
#pragma unroll
            for (int i = 0; i < KEEP; ++i)
#pragma unroll
                for (int k = 0; k < 8; ++k) here = kv8_larger(here, x[i][k]);
            if (kv8_odd(here)) {                    // something is no finite number: it does not count for the scale
#pragma unroll
                for (int i = 0; i < KEEP; ++i)
#pragma unroll
                    for (int k = 0; k < 8; ++k) some = __vmaxu2(some, kv8_finite(x[i][k]));
            } else some = __vmaxu2(some, here);
            most = kv8_larger(most, here);
        }
        const bool odd = __any_sync(0xffffffffu, kv8_odd(most));
        most = __reduce_max_sync(0xffffffffu, max(some & 0xffffu, some >> 16));
        int field = kv8_field(most);
        unsigned char* blk = p.store + block * p.block_bytes;
        unsigned char* rows = blk + (static_cast<long long>(h) * 2 + is_v) * B * PI_HEAD_DIM;
        uint32_t* scale = reinterpret_cast<uint32_t*>(blk + (static_cast<long long>(2 * B * PI_HEAD_DIM) << p.log_h)) + 2 * h + is_v;
        const bool fresh = f0 & 1u;
        bool write_scale = true;
        if (!fresh) {
            const int had = kv8_field_of(*scale);
            write_scale = field > had;
            if (write_scale) {                      // the block's other tokens under the new scale: eight lanes a row
                const float factor = kv8_factor(had, field);
                for (int y = lane >> 3; y < B; y += 4) {
                    if (((y < 32 ? f0 : f1) >> (y & 31)) & 1u) continue;
                    uint4* to = reinterpret_cast<uint4*>(rows + y * PI_HEAD_DIM) + (lane & 7);
                    const uint4 c = *to;
                    *to = make_uint4(kv8_again4(c.x, factor), kv8_again4(c.y, factor), kv8_again4(c.z, factor), kv8_again4(c.w, factor));
                }
            } else field = had;
        } else if (n < B) {                         // a block that begins anew holds nothing else
            for (int y = lane >> 3; y < B; y += 4)
                if (!(((y < 32 ? f0 : f1) >> (y & 31)) & 1u)) reinterpret_cast<uint4*>(rows + y * PI_HEAD_DIM)[lane & 7] = make_uint4(0u, 0u, 0u, 0u);
        }
        if (write_scale && lane == 0) *scale = __float_as_uint(kv8_scale_of(field));
        const float inverse = kv8_inverse_of(field);
        for (int i0 = 0; i0 < FOURS; i0 += KEEP) {
            if (i0) fetch(x, i0);                   // (the last rows to be looked at are the first, and are still there)
#pragma unroll
            for (int i = 0; i < KEEP; ++i) {
                const int y = 4 * (i0 + i) + quarter, a0 = __shfl_sync(0xffffffffu, at0, y & 31), a1 = B > 32 ? __shfl_sync(0xffffffffu, at1, y & 31) : 0;
                if (y >= n) continue;
                uint32_t u[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) u[k] = odd ? kv8_round4(x[i][2 * k], x[i][2 * k + 1], inverse) : kv8_round4_finite(x[i][2 * k], x[i][2 * k + 1], inverse);
                *reinterpret_cast<uint4*>(rows + (y < 32 ? a0 : a1) * PI_HEAD_DIM + l * 16) = make_uint4(u[0], u[1], u[2], u[3]);
            }
        }
        __syncwarp();
    }
}

struct LoadParams {
    const unsigned char* store;
    const int32_t* blocks;
    unsigned char* out;                             // [n_out][Hkv][2][B][D] bf16
    pi_status_ref st;
    long long n_items, block_bytes, n_blocks;       // an item is 16 rows of a (block, head, K or V)
    int log_tiles, log_h, B;
    bool wide;                                      // out is aligned to 32 bytes
};

__global__ void __launch_bounds__(KV8_THREADS)
kv8_load_kernel(LoadParams p) {
    const int lane = threadIdx.x & 31;
    const long long item = static_cast<long long>(blockIdx.x) * KV8_WARPS + (threadIdx.x >> 5);
    pi_grid_dependency_wait();
    pi_launch_dependents();
    if (item >= p.n_items) return;
    const int run = static_cast<int>(item) & ((2 << (p.log_tiles + p.log_h)) - 1);     // 16-row run of the block
    const long long i = item >> (p.log_tiles + p.log_h + 1);
    const long long block = p.blocks ? p.blocks[i] : i;
    if (block < 0 || block >= p.n_blocks) {
        if (lane == 0 && run == 0) pi_report(p.st, PI_ERR_INDEX_RANGE, PI_STAGE_KV4, static_cast<int>(i < 0x7fffffffLL ? i : 0x7fffffffLL), 0, static_cast<int>(block));
        return;
    }
    const unsigned char* blk = p.store + block * p.block_bytes;
    const uint4* src = reinterpret_cast<const uint4*>(blk + run * 2048) + lane;
    const float scale = reinterpret_cast<const float*>(blk + (static_cast<long long>(2 * p.B * PI_HEAD_DIM) << p.log_h))[run >> p.log_tiles];
    uint4 c[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) c[k] = src[32 * k];
    // 16 numbers become 32 bytes: one store where the output is aligned to as many (121 us instead of 144 for two of 16)
    uint4* dst = reinterpret_cast<uint4*>(p.out + item * 4096);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t w[4] = {c[k].x, c[k].y, c[k].z, c[k].w};
        uint32_t o[8];
#pragma unroll
        for (int y = 0; y < 8; ++y) {
            const float2 f = kv8_values((y & 1) ? w[y >> 1] >> 16 : w[y >> 1] & 0xffffu);
            const __nv_bfloat162 b = __floats2bfloat162_rn(f.x * scale, f.y * scale);
            o[y] = *reinterpret_cast<const uint32_t*>(&b);
        }
        uint4* to = dst + 64 * k + 2 * lane;
        if (p.wide) asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(to), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]), "r"(o[4]), "r"(o[5]), "r"(o[6]), "r"(o[7]) : "memory");
        else {
            to[0] = make_uint4(o[0], o[1], o[2], o[3]);
            to[1] = make_uint4(o[4], o[5], o[6], o[7]);
        }
    }
}

int log2_of(int x) {
    int n = 0;
    while ((1 << n) < x) ++n;
    return n;
}

}  // namespace

int pi_launch_kv8_store(pi_ctx* c, int64_t n_tokens, const void* k, const int64_t (&ks)[3], const void* v, const int64_t (&vs)[3],
                        int inner, const int64_t* slots, void* store, int64_t n_blocks, cudaStream_t stream) {
    const int B = c->cfg.block_tokens, range = B < 32 ? B : 32;
    StoreParams p;
    p.k = static_cast<const __nv_bfloat16*>(k); p.v = static_cast<const __nv_bfloat16*>(v);
    p.k_tok = ks[0]; p.k_head = ks[1]; p.k_outer = ks[2];
    p.v_tok = vs[0]; p.v_head = vs[1]; p.v_outer = vs[2];
    p.slots = slots;
    p.store = static_cast<unsigned char*>(store);
    p.st = pi_status_of(c);
    p.log_h = log2_of(c->cfg.n_kv_heads);           // (a power of two: pi_create)
    p.n_tokens = n_tokens;
    p.n_slots = n_blocks * B;
    p.block_bytes = kv8_block_bytes(c->cfg.n_kv_heads, B);
    p.n_items = ((n_tokens + range - 1) / range) << (1 + p.log_h);
    p.inner = inner;
    const long long grid = (p.n_items + KV8_WARPS - 1) / KV8_WARPS;
    if (grid > INT32_MAX) return PI_ERR_UNSUPPORTED_DIM;
    auto kernel = B == 16 ? kv8_store_kernel<16> : B == 32 ? kv8_store_kernel<32> : kv8_store_kernel<64>;
    PI_CUDA_TRY(pi_launch_pdl(kernel, dim3(static_cast<unsigned>(grid)), dim3(KV8_THREADS), 0, stream, p));
    return PI_OK;
}

int pi_launch_kv8_load(pi_ctx* c, int64_t n_out, const void* store, int64_t n_blocks, const int32_t* blocks, void* out, cudaStream_t stream) {
    LoadParams p;
    p.store = static_cast<const unsigned char*>(store);
    p.blocks = blocks;
    p.out = static_cast<unsigned char*>(out);
    p.wide = (reinterpret_cast<uintptr_t>(out) & 31u) == 0;
    p.st = pi_status_of(c);
    p.B = c->cfg.block_tokens;
    p.log_h = log2_of(c->cfg.n_kv_heads); p.log_tiles = log2_of(p.B / 16);
    p.n_items = n_out << (p.log_h + p.log_tiles + 1);
    p.block_bytes = kv8_block_bytes(c->cfg.n_kv_heads, c->cfg.block_tokens);
    p.n_blocks = n_blocks;
    PI_CUDA_TRY(pi_launch_pdl(kv8_load_kernel, dim3(static_cast<unsigned>((p.n_items + KV8_WARPS - 1) / KV8_WARPS)), dim3(KV8_THREADS), 0, stream, p));
    return PI_OK;
}
