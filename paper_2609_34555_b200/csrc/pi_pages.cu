// Page tables and slot maps from request lengths: pages taken for the sequences that grow, given back for those that
// shrink, and the slot and position of every new token, in one launch.
//
// The free pages are a ring: pages are taken at `head` and given back at `tail` (both counted up without end), so one
// call can do both without the two meeting.  Which page a sequence gets follows from an exclusive scan of the growth
// over the sequences, which every CTA computes for itself in shared memory (at most 4096 sequences, 32 KB out of L2):
// no CTA waits for another, and a token's page is read from the ring directly rather than from the table row that
// another CTA may still be writing.  The ring's counters move once, by whichever CTA finishes last (a ticket beside
// them), when every CTA has read them.  Writes 12 bytes a token and 4 a page.  Measured on a B200: 16 sequences x 4 draft
// tokens and their rollback 3.2 us a call, a chain of four dependent loads; 64 prompts of 4.7 million tokens taken and given
// back 25.1 us for both calls, where the scan and the page lookups cost as much as the 57 MB of maps.
#include "pi_common.cuh"

namespace {

constexpr int PAGES_THREADS = 256;
constexpr int PAGES_WARPS = PAGES_THREADS / 32;

struct PagesParams {
    const int32_t* old_len;
    const int32_t* new_len;
    int32_t* table;
    int32_t* ring;
    long long* state;              // head, tail, ticket, unused
    int32_t* starts;
    int64_t* slots;
    int32_t* positions;
    pi_status_ref st;
    long long row_stride, n_tokens;
    int batch, n_pages, row_limit, shift;
};

// Block-wide exclusive scans of three values at once, continued from `run` (moved on); all threads call.
__device__ __forceinline__ void scan_from(const long long (&v)[3], long long (&before)[3], long long (*warp_tot)[3], long long (&run)[3]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long inc[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) inc[k] = v[k];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1)
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const long long t = __shfl_up_sync(0xffffffffu, inc[k], o);
            if (lane >= o) inc[k] += t;
        }
    __syncthreads();
    if (lane == 31)
#pragma unroll
        for (int k = 0; k < 3; ++k) warp_tot[warp][k] = inc[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        before[k] = run[k] + inc[k] - v[k];
#pragma unroll
        for (int i = 0; i < PAGES_WARPS; ++i) {
            if (i < warp) before[k] += warp_tot[i][k];
            run[k] += warp_tot[i][k];
        }
    }
}

// Last s with pref[s] <= i, for an ascending pref[0 .. n] with pref[0] = 0 and i < pref[n].
__device__ __forceinline__ int owner_of(const int* pref, int n, int i) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (pref[mid] <= i) lo = mid; else hi = mid;
    }
    return lo;
}

__global__ void __launch_bounds__(PAGES_THREADS, 4)
assign_pages_kernel(PagesParams p) {
    extern __shared__ int s_dyn[];
    int* s_old = s_dyn;                                  // [batch]
    int* s_tok = s_old + p.batch;                        // [batch + 1] new tokens before each sequence
    int* s_grow = s_tok + p.batch + 1;                   // [batch + 1] pages taken before it
    int* s_shrink = s_grow + p.batch + 1;                // [batch + 1] pages given back before it
    __shared__ long long warp_tot[PAGES_WARPS][3];
    __shared__ int s_bad;
    const int tid = threadIdx.x, B = 1 << p.shift;
    if (tid == 0) s_bad = -1;
    pi_grid_dependency_wait();
    pi_launch_dependents();
    const long long head = *reinterpret_cast<volatile long long*>(p.state), tail = *reinterpret_cast<volatile long long*>(p.state + 1);
    long long run[3] = {0, 0, 0};                        // new tokens, pages taken, pages given back
    for (int s0 = 0; s0 < p.batch; s0 += PAGES_THREADS) {
        const int s = s0 + tid;
        int add = 0, g = 0, r = 0, o = 0;
        bool bad = false;
        if (s < p.batch) {
            o = p.old_len[s];
            const int n = p.new_len[s];
            bad = o < 0 || n < 0 || ((static_cast<long long>(max(o, n)) + B - 1) >> p.shift) > p.row_limit;
            if (!bad) {
                const int ob = static_cast<int>((static_cast<long long>(o) + B - 1) >> p.shift), nb = static_cast<int>((static_cast<long long>(n) + B - 1) >> p.shift);
                add = max(n - o, 0); g = max(nb - ob, 0); r = max(ob - nb, 0);
            }
        }
        const long long v[3] = {add, g, r};
        long long before[3];
        scan_from(v, before, warp_tot, run);
        if (s < p.batch) {
            if (bad) atomicMax(&s_bad, s);
            s_old[s] = o;
            // (a total beyond 32 bits is refused below, before these are used)
            s_tok[s] = static_cast<int>(before[0]); s_grow[s] = static_cast<int>(before[1]); s_shrink[s] = static_cast<int>(before[2]);
        }
    }
    long long tokens = run[0], grown = run[1], shrunk = run[2];
    if (tid == 0) { s_tok[p.batch] = static_cast<int>(tokens); s_grow[p.batch] = static_cast<int>(grown); s_shrink[p.batch] = static_cast<int>(shrunk); }
    __syncthreads();

    // all or nothing: every CTA comes to the same verdict
    const long long room = tail - head;
    int code = PI_OK, ca = 0, cb = 0, cc = 0;
    if (s_bad >= 0) { code = PI_ERR_INDEX_RANGE; ca = s_bad; cb = p.old_len[s_bad]; cc = p.new_len[s_bad]; }
    else if (head < 0 || room < 0 || room > p.n_pages) { code = PI_ERR_INDEX_RANGE; ca = -1; cb = static_cast<int>(head); cc = static_cast<int>(tail); }
    else if (grown > room) { code = PI_ERR_POOL_TOO_SMALL; ca = -1; cb = static_cast<int>(min(grown, 0x7fffffffLL)); cc = static_cast<int>(room); }
    else if (room + shrunk > p.n_pages) { code = PI_ERR_CAPACITY; ca = -1; cb = static_cast<int>(min(shrunk, 0x7fffffffLL)); cc = p.n_pages; }
    else if (tokens > 0x7fffffffLL || ((p.slots || p.positions) && tokens > p.n_tokens)) { code = PI_ERR_CAPACITY; ca = -2; cb = static_cast<int>(min(tokens, 0x7fffffffLL)); cc = static_cast<int>(min(p.n_tokens, 0x7fffffffLL)); }
    const bool ok = code == PI_OK;
    if (!ok) {
        if (blockIdx.x == 0 && tid == 0) pi_report(p.st, code, PI_STAGE_PAGES, ca, cb, cc);
        tokens = 0; grown = 0; shrunk = 0;
    }
    // (the last threads of all begin with the pages, the first ones with the tokens: for a small batch the two run side by side)
    const long long me = static_cast<long long>(gridDim.x - 1 - blockIdx.x) * PAGES_THREADS + (PAGES_THREADS - 1 - tid), all = static_cast<long long>(gridDim.x) * PAGES_THREADS;
    if (p.starts)
        for (long long s = me; s <= p.batch; s += all) p.starts[s] = ok ? s_tok[s] : 0;

    // place of the i-th page from a counter in the ring (i <= n_pages): one division per call, none per page
    const unsigned n = static_cast<unsigned>(p.n_pages);
    const unsigned head_at = ok ? static_cast<unsigned>(head % p.n_pages) : 0u, tail_at = ok ? static_cast<unsigned>(tail % p.n_pages) : 0u;
    auto ring_at = [&](unsigned from, long long i) { const unsigned x = from + static_cast<unsigned>(i); return x < n ? x : x - n; };
    // pages taken
    for (long long i = me; i < grown; i += all) {
        const int s = owner_of(s_grow, p.batch, static_cast<int>(i));
        const int ob = (s_old[s] + B - 1) >> p.shift;
        int pg = p.ring[ring_at(head_at, i)];
        if (pg < 0 || pg >= p.n_pages) { pi_report(p.st, PI_ERR_INDEX_RANGE, PI_STAGE_PAGES, s, static_cast<int>(i), pg); pg = -1; }
        p.table[s * p.row_stride + ob + (i - s_grow[s])] = pg;
    }
    // pages given back
    for (long long i = me; i < shrunk; i += all) {
        const int s = owner_of(s_shrink, p.batch, static_cast<int>(i));
        const int keep = ((s_old[s] + B - 1) >> p.shift) - (s_shrink[s + 1] - s_shrink[s]);
        int32_t* e = p.table + s * p.row_stride + keep + (i - s_shrink[s]);
        const int pg = *e;
        if (pg < 0 || pg >= p.n_pages) pi_report(p.st, PI_ERR_INDEX_RANGE, PI_STAGE_PAGES, s, static_cast<int>(i), pg);
        p.ring[ring_at(tail_at, i)] = pg;
        *e = -1;
    }
    // Slot and position of every new token: a CTA takes one run of them, a warp spans of 64, a lane a pair of neighbours (whole
    // 16-byte stores side by side).  Four spans at a time, so that their page lookups are on their way together.  Most spans
    // lie inside one sequence, which the warp then knows already; in the others every lane looks for itself.
    if (p.slots || p.positions) {
        // (n_tokens is at most 2^30, and `tokens` not above it: 32 bits do)
        const int n_tokens = static_cast<int>(p.n_tokens), total = static_cast<int>(tokens), lane = tid & 31;
        const int each = ((n_tokens - 1) / static_cast<int>(gridDim.x) / 64 + 1) * 64;
        const int from = static_cast<int>(min(static_cast<long long>(blockIdx.x) * each, p.n_tokens));
        const int end = static_cast<int>(min(static_cast<long long>(from) + each, p.n_tokens));
        auto lookup = [&](int s, int ob, int grow, int at) {
            const int block = at >> p.shift;
            return block < ob ? p.table[s * p.row_stride + block] : p.ring[ring_at(head_at, grow + (block - ob))];
        };
        int s = -1, first = 0, next = 0, old = 0, ob = 0, grow = 0;       // the warp's sequence: its tokens are first .. next - 1
        for (int w0 = from + 64 * (tid >> 5); w0 < end; w0 += 64 * PAGES_WARPS * 4) {
            int pos[4], pg[4][2];
            unsigned rest = 0u;                                            // spans that every lane looks through for itself
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int w = w0 + 64 * PAGES_WARPS * k;
                pg[k][0] = -1;
                if (w >= end) continue;
                if (w >= next && w < total) {
                    s = owner_of(s_tok, p.batch, w);
                    first = s_tok[s]; next = s_tok[s + 1]; old = s_old[s]; grow = s_grow[s];
                    ob = (old + B - 1) >> p.shift;
                }
                if (w + 64 > total || w + 64 > next) { rest |= 1u << k; continue; }
                pos[k] = old + (w + 2 * lane - first);
                pg[k][0] = pg[k][1] = lookup(s, ob, grow, pos[k]);
                if (((pos[k] + 1) & (B - 1)) == 0) pg[k][1] = lookup(s, ob, grow, pos[k] + 1);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int w = w0 + 64 * PAGES_WARPS * k, t = w + 2 * lane;
                if (w >= end || ((rest >> k) & 1u)) continue;
                // (a page that is none is reported where every lane looks for itself)
                if (!__all_sync(0xffffffffu, static_cast<unsigned>(pg[k][0]) < n && static_cast<unsigned>(pg[k][1]) < n)) { rest |= 1u << k; continue; }
                const int64_t s0 = static_cast<int64_t>(pg[k][0]) * B + (pos[k] & (B - 1)), s1 = static_cast<int64_t>(pg[k][1]) * B + ((pos[k] + 1) & (B - 1));
                if (p.slots) *reinterpret_cast<longlong2*>(p.slots + t) = make_longlong2(s0, s1);
                if (p.positions) *reinterpret_cast<int2*>(p.positions + t) = make_int2(pos[k], pos[k] + 1);
            }
#pragma unroll 1
            for (; rest; rest &= rest - 1) {
                const int w = w0 + 64 * PAGES_WARPS * (__ffs(rest) - 1);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int t = w + lane + 32 * u;
                    if (t >= end) continue;
                    int64_t slot = -1;
                    int at = -1;
                    if (t < total) {
                        const int si = owner_of(s_tok, p.batch, t);
                        at = s_old[si] + (t - s_tok[si]);
                        const int pg1 = lookup(si, (s_old[si] + B - 1) >> p.shift, s_grow[si], at);
                        if (static_cast<unsigned>(pg1) < n) slot = (static_cast<int64_t>(pg1) << p.shift) + (at & (B - 1));
                        else pi_report(p.st, PI_ERR_INDEX_RANGE, PI_STAGE_PAGES, si, at, pg1);
                    }
                    if (p.slots) p.slots[t] = slot;
                    if (p.positions) p.positions[t] = at;
                }
            }
        }
    }
    // the last CTA moves the ring's counters: by then every CTA has read them (and used what it read)
    __syncthreads();
    if (tid == 0) {
        unsigned long long v = 0;
        if (gridDim.x > 1) v = atomicAdd(reinterpret_cast<unsigned long long*>(p.state + 2), 1ull);
        if (v >= gridDim.x) pi_report(p.st, PI_ERR_INDEX_RANGE, PI_STAGE_PAGES, -3, static_cast<int>(v), static_cast<int>(gridDim.x));
        else if (v == gridDim.x - 1) {
            p.state[0] = head + grown;
            p.state[1] = tail + shrunk;
            p.state[2] = 0;
        }
    }
}

}  // namespace

int pi_launch_assign_pages(pi_ctx* c, int batch, const int32_t* old_len, const int32_t* new_len, int32_t* table, int64_t row_stride,
                           int32_t n_pages, int32_t* ring, int64_t* state, int32_t* starts, int64_t n_tokens, int64_t* slots,
                           int32_t* positions, cudaStream_t stream) {
    PagesParams p;
    p.old_len = old_len; p.new_len = new_len; p.table = table; p.ring = ring;
    p.state = reinterpret_cast<long long*>(state);
    p.starts = starts; p.slots = slots; p.positions = positions;
    p.st = pi_status_of(c);
    p.row_stride = row_stride; p.n_tokens = n_tokens;
    p.batch = batch; p.n_pages = n_pages;
    p.row_limit = static_cast<int>(row_stride < c->cfg.max_blocks ? row_stride : c->cfg.max_blocks);
    p.shift = c->cfg.block_tokens == 16 ? 4 : c->cfg.block_tokens == 32 ? 5 : 6;
    // enough CTAs for the token maps (four tokens a thread; a page taken means a token), or, where there are none, for a batch
    // whose rows all change (two pages a thread); at most four per SM, each making its own scan of the batch, or one where the
    // host cannot know how little there is to do (64 rows of 4096 pages, taken and given back: one token each 7.3 us for
    // both calls instead of 10.1, 60000 each 25.9 instead of 24.2)
    const long long most = n_tokens > 0 ? 4ll * c->n_sms : c->n_sms;
    long long grid = ((n_tokens > 0 ? (n_tokens + 3) / 4 : static_cast<long long>(batch) * p.row_limit / 2) + PAGES_THREADS - 1) / PAGES_THREADS;
    grid = grid < 1 ? 1 : grid > most ? most : grid;
    const size_t smem = (4 * static_cast<size_t>(batch) + 3) * sizeof(int);
    if (smem > 40 * 1024) PI_CUDA_TRY(cudaFuncSetAttribute(assign_pages_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
    PI_CUDA_TRY(pi_launch_pdl(assign_pages_kernel, dim3(static_cast<unsigned>(grid)), dim3(PAGES_THREADS), smem, stream, p));
    return PI_OK;
}
