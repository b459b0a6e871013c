// The append kernel, for blocks of every form; which file compiles which form is in pi_append.cu and pi_append_kv8.cu.
#pragma once

#include "pi_kv4.cuh"
#include "pi_kv8.cuh"

namespace {

constexpr int APPEND_THREADS = 256;
constexpr int APPEND_WARPS = APPEND_THREADS / 32;

struct AppendParams {
    const uint4* k_new;            // [batch][Hkv][D] bf16, 16 uint4 per head row
    const uint4* v_new;
    const int32_t* ctx_len;
    unsigned char* host;
    unsigned char* pool;
    int32_t* table;
    int32_t* slot_block;
    uint32_t* slot_stamp;
    __nv_bfloat16* digest;
    pi_status_ref st;
    long long host_stride, pool_stride;
    const int32_t* page;           // paged host store (or null): block b of sequence s is arena page page[s * page_stride + b]
    long long page_stride;
    int n_pages;
    const uint32_t* step_dev;      // when set, the stamp is read from device memory (graph replay)
    uint32_t step;
    long long block_bytes;
    int B, Hkv, C, n_sink, n_local, max_blocks, h_star;
};

// FORM: bits of a number in pool and store, 16, 8 or 4; the token's rows are rounded on their way there (the digest takes the
// key as it came).  Latency-bound in every form.  B200, 4 bits, 16 sequences of 256 slots, one launch between two events (an empty
// one 6.1 us): into an open block 12.3 us with the store in pinned memory and 8.2 with it on the device, opening a
// block (the choice of a slot, a fresh block cleared in pool and store) 18.4 and 10.2.  8 bits, blocks of 16 and 8 heads, store on the device, 4 of 16
// sequences opening a block: 3.8 us back to back, 8.2 with cold caches (an empty one 2.6); 64 sequences, blocks of 32: 5.1 and 10.2.
template <int FORM>
__global__ void __launch_bounds__(APPEND_THREADS)
append_kernel(AppendParams p) {
    __shared__ unsigned long long warp_min[APPEND_WARPS];
    __shared__ int s_slot;
    const int seq = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pi_grid_dependency_wait();
    pi_launch_dependents();
    const int pos = p.ctx_len[seq];
    // 8 bits: what hangs on no other load is asked for with the context's length.  A load that has to come from memory takes most of a microsecond, and
    // the call is little else than a chain of them (cold, 16 sequences: 8.2 us, 10.2 one after the other).  The other forms keep their registers.
    int32_t* slot_block = p.slot_block + static_cast<size_t>(seq) * p.C;
    uint32_t* slot_stamp = p.slot_stamp + static_cast<size_t>(seq) * p.C;
    constexpr int AHEAD = FORM == 8 ? 2 : 0;               // slots of a thread, rows of a warp
    int ahead_block[AHEAD + 1];
    uint32_t ahead_stamp[AHEAD + 1];
    uint2 ahead_row[AHEAD + 1];
    __nv_bfloat16 key, lowest, highest;                    // of the digest
    const __nv_bfloat16* keys = reinterpret_cast<const __nv_bfloat16*>(p.k_new) + (static_cast<size_t>(seq) * p.Hkv + p.h_star) * PI_HEAD_DIM;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
        const int s = tid + i * APPEND_THREADS;
        ahead_block[i] = s < p.C ? slot_block[s] : 0;
        ahead_stamp[i] = s < p.C ? slot_stamp[s] : 0u;
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
        const int r = warp + i * APPEND_WARPS;
        if (r < 2 * p.Hkv) ahead_row[i] = reinterpret_cast<const uint2*>(r & 1 ? p.v_new : p.k_new)[(static_cast<size_t>(seq) * p.Hkv + (r >> 1)) * 32 + lane];
    }
    if (FORM == 8) key = keys[tid & (PI_HEAD_DIM - 1)];
    if (pos < 0) return;
    const int b = pos / p.B, t = pos - b * p.B;
    if (b >= p.max_blocks) {
        if (tid == 0) pi_report(p.st, PI_ERR_CAPACITY, PI_STAGE_APPEND, seq, b, p.max_blocks);
        return;
    }
    int32_t* table = p.table + static_cast<size_t>(seq) * p.max_blocks;
    const long long block_bytes = FORM != 16 ? p.block_bytes : static_cast<long long>(p.Hkv) * 2 * p.B * PI_HEAD_DIM * 2;
    int slot = table[b];
    if (FORM == 8) {
        const __nv_bfloat16* digest = p.digest + (static_cast<size_t>(seq) * p.max_blocks + b) * 2 * PI_HEAD_DIM + (tid & (PI_HEAD_DIM - 1));
        lowest = digest[0];
        highest = digest[PI_HEAD_DIM];
    }
    long long host_off = seq * p.host_stride + b * block_bytes;
    if (p.page) {
        // a block index beyond the sequence's row of the table is not followed (rows are page_stride long)
        const int pg = b < p.page_stride ? p.page[seq * p.page_stride + b] : -1;
        if (pg < 0 || pg >= p.n_pages) {
            if (tid == 0) pi_report(p.st, PI_ERR_INDEX_RANGE, PI_STAGE_APPEND, seq, b, pg);
            return;
        }
        host_off = pg * block_bytes;
    }

    if (t == 0 && slot < 0) {
        // the block just opened is part of the local window: it takes the least recently selected
        // slot whose block is neither sink nor local under the new length (free slots first)
        const int nb_new = b + 1;
        unsigned long long best = ~0ull;
        auto look = [&](int s, int ob, uint32_t stamp) {
            const bool pinned = ob >= 0 && (ob < p.n_sink || ob >= nb_new - p.n_local);
            if (!pinned) best = min(best, (static_cast<unsigned long long>(stamp) << 32) | static_cast<unsigned>(s));
        };
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if (tid + i * APPEND_THREADS < p.C) look(tid + i * APPEND_THREADS, ahead_block[i], ahead_stamp[i]);
        for (int s = tid + AHEAD * APPEND_THREADS; s < p.C; s += APPEND_THREADS) look(s, slot_block[s], slot_stamp[s]);
#pragma unroll
        for (int o = 16; o; o >>= 1) best = min(best, __shfl_xor_sync(0xffffffffu, best, o));
        if (lane == 0) warp_min[warp] = best;
        __syncthreads();
        if (tid == 0) {
            unsigned long long g = warp_min[0];
            for (int w = 1; w < APPEND_WARPS; ++w) g = min(g, warp_min[w]);
            int sl = -1;
            if (g != ~0ull) {
                sl = static_cast<int>(g & 0xffffffffull);
                const int old = slot_block[sl];
                if (old >= 0 && old < p.max_blocks) table[old] = -1;
                table[b] = sl;
                slot_block[sl] = b;
            }
            s_slot = sl;
        }
        __syncthreads();
        slot = s_slot;
        if (slot < 0) {
            if (tid == 0) pi_report(p.st, PI_ERR_POOL_TOO_SMALL, PI_STAGE_APPEND, seq, b, p.C);
            return;
        }
    } else if (slot < 0 || slot >= p.C) {
        if (tid == 0) pi_report(p.st, PI_ERR_INDEX_RANGE, PI_STAGE_APPEND, seq, b, slot);
        return;
    }
    unsigned char* pool_blk = p.pool + seq * p.pool_stride + slot * block_bytes;
    unsigned char* host_blk = p.host + host_off;
    if (t == 0) {
        // a fresh block starts zeroed, in the pool and in the host store
        const uint4 z = make_uint4(0, 0, 0, 0);
        for (long long i = tid; i < block_bytes / 16; i += APPEND_THREADS) {
            reinterpret_cast<uint4*>(pool_blk)[i] = z;
            reinterpret_cast<uint4*>(host_blk)[i] = z;
        }
        __syncthreads();                                   // zeros land before the rows below
    }
    if (tid == 0) slot_stamp[slot] = p.step_dev ? *p.step_dev : p.step;
    if (FORM == 4) {
        // eight lanes a row, a warp the K and V rows of two heads
        const bool is_v = lane & 8;
        const int l = lane & 7;
        for (int h0 = 2 * warp; h0 < p.Hkv; h0 += 2 * APPEND_WARPS) {
            const int h = min(h0 + (lane >> 4), p.Hkv - 1);
            const uint4* src = (is_v ? p.v_new : p.k_new) + (static_cast<size_t>(seq) * p.Hkv + h) * 16 + 2 * l;
            const uint4 x[2] = {src[0], src[1]};
            uint32_t codes[2], sz;
            kv4_quantise(x, codes, sz);
            const long long off = (static_cast<long long>(h) * (p.B >> 4) + (t >> 4)) * KV4_TILE_BYTES;
            const bool write = h0 + (lane >> 4) < p.Hkv;
            kv4_write_row(pool_blk + off, t & 15, is_v, l, codes, sz, write);
            kv4_write_row(host_blk + off, t & 15, is_v, l, codes, sz, write);
        }
    } else if (FORM == 8) {
        // A warp a row of 128 channels, four a lane.  A row whose scale suffices is 128 bytes into the block; one that is larger takes the other
        // rows of its head and K or V with it: they are rounded again, and the store's copy is written anew from the pool's.
        for (int i = warp; i < 2 * p.Hkv; i += APPEND_WARPS) {
            const uint2 x = i == warp ? ahead_row[0] : i == warp + APPEND_WARPS ? ahead_row[1]
                          : reinterpret_cast<const uint2*>(i & 1 ? p.v_new : p.k_new)[(static_cast<size_t>(seq) * p.Hkv + (i >> 1)) * 32 + lane];
            const long long scales = static_cast<long long>(p.Hkv) * 2 * p.B * PI_HEAD_DIM + 4 * i, rows = static_cast<long long>(i) * p.B * PI_HEAD_DIM;
            uint32_t* scale = reinterpret_cast<uint32_t*>(pool_blk + scales);
            const int had = t == 0 ? 0 : kv8_field_of(*scale);
            uint32_t most = __vmaxu2(kv8_finite(x.x), kv8_finite(x.y));
#pragma unroll
            for (int d = 16; d; d >>= 1) most = __vmaxu2(most, __shfl_xor_sync(0xffffffffu, most, d));
            const int need = kv8_field(most), field = max(need, had);
            if (t > 0 && need > had) {
                const float factor = kv8_factor(had, need);
                for (int y = lane >> 3; y < p.B; y += 4) {
                    if (y == t) continue;
                    const long long at = rows + y * PI_HEAD_DIM + (lane & 7) * 16;
                    const uint4 c = *reinterpret_cast<const uint4*>(pool_blk + at);
                    const uint4 n = make_uint4(kv8_again4(c.x, factor), kv8_again4(c.y, factor), kv8_again4(c.z, factor), kv8_again4(c.w, factor));
                    *reinterpret_cast<uint4*>(pool_blk + at) = n;
                    *reinterpret_cast<uint4*>(host_blk + at) = n;
                }
            }
            const uint32_t codes = kv8_round4(x.x, x.y, kv8_inverse_of(field));
            const long long at = rows + t * PI_HEAD_DIM + 4 * lane;
            *reinterpret_cast<uint32_t*>(pool_blk + at) = codes;
            *reinterpret_cast<uint32_t*>(host_blk + at) = codes;
            if (lane == 0 && (t == 0 || need > had)) {
                const uint32_t bits = __float_as_uint(kv8_scale_of(field));
                *scale = bits;
                *reinterpret_cast<uint32_t*>(host_blk + scales) = bits;
            }
        }
    } else
    // rows: [Hkv][2][B][D]; one head row is 256 B = 16 uint4
    for (int i = tid; i < p.Hkv * 32; i += APPEND_THREADS) {
        const int h = i >> 5, kv = (i >> 4) & 1, c = i & 15;
        const uint4 x = (kv ? p.v_new : p.k_new)[(static_cast<size_t>(seq) * p.Hkv + h) * 16 + c];
        const long long off = ((static_cast<long long>(h) * 2 + kv) * p.B + t) * (PI_HEAD_DIM * 2) + c * 16;
        *reinterpret_cast<uint4*>(pool_blk + off) = x;
        *reinterpret_cast<uint4*>(host_blk + off) = x;
    }
    // running min / max of the retrieval head's keys in this block (exact: bf16 values only)
    if (tid < PI_HEAD_DIM) {
        __nv_bfloat16* lo = p.digest + (static_cast<size_t>(seq) * p.max_blocks + b) * 2 * PI_HEAD_DIM + tid;
        __nv_bfloat16* hi = lo + PI_HEAD_DIM;
        if (FORM != 8) key = keys[tid];
        if (t == 0) { *lo = key; *hi = key; }
        else {
            if (FORM != 8) lowest = *lo;
            if (__bfloat162float(key) < __bfloat162float(lowest)) *lo = key;
            if (FORM != 8) highest = *hi;
            if (__bfloat162float(key) > __bfloat162float(highest)) *hi = key;
        }
    }
}

}  // namespace

// The parameters of every form but the step's.
static inline void append_params(AppendParams& p, const pi_ctx* c, int h_star, uint32_t step, const uint32_t* step_dev, const void* k_new, const void* v_new,
                                 const int32_t* ctx_len, void* host_kv, int64_t host_stride, void* pool, int32_t* table, int32_t* slot_block,
                                 uint32_t* slot_stamp, void* digest, const int32_t* page_table, int64_t page_stride, int32_t n_pages, int64_t block_bytes) {
    p.step_dev = step_dev;
    p.page = page_table; p.page_stride = page_stride; p.n_pages = n_pages;
    p.k_new = static_cast<const uint4*>(k_new);
    p.v_new = static_cast<const uint4*>(v_new);
    p.ctx_len = ctx_len;
    p.host = static_cast<unsigned char*>(host_kv);
    p.pool = static_cast<unsigned char*>(pool);
    p.table = table; p.slot_block = slot_block; p.slot_stamp = slot_stamp;
    p.digest = static_cast<__nv_bfloat16*>(digest);
    p.st = pi_status_of(const_cast<pi_ctx*>(c));
    p.host_stride = host_stride;
    p.block_bytes = block_bytes;
    p.pool_stride = c->cfg.pool_slots * p.block_bytes;
    p.step = step;
    p.B = c->cfg.block_tokens; p.Hkv = c->cfg.n_kv_heads; p.C = c->cfg.pool_slots;
    p.n_sink = c->cfg.n_sink_blocks; p.n_local = c->cfg.n_local_blocks; p.max_blocks = c->cfg.max_blocks;
    p.h_star = h_star;
}
