// gfx950 kernels for a batch's new tokens: slots and blocks from request lengths, and the append of their projections.
#include <hip/hip_runtime.h>

#include "pod_tokens.h"

namespace pod {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int32_t i32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
#define POD_CONST __attribute__((address_space(4)))

// Quotient and remainder of a non-negative 31-bit number by the divisor whose magic this is.
__device__ __forceinline__ int divide(int t, int divisor, uint32_t magic, int &rest)
{
    if (magic == 0u) { rest = 0; return t; }
    int q = (int)(((uint64_t)(uint32_t)t * magic) >> 32);
    rest = t - q * divisor;
    if (rest < 0) { --q; rest += divisor; }
    return q;
}

// ------------------------------------------------------------------------------------------
// Tables.  One launch and nothing shared between workgroups: each one adds up the blocks of all requests before its own
// (exclusive prefix sum: request r takes free_blocks[before_r ..]) and of the whole batch (does the list hold enough?)
// from the request lengths themselves, 16 bytes a request that every workgroup finds in its L2, and then writes its own
// rows.  What bounds it is the launch and two dependent round trips (256 decodes 3.6 us, 6 prompts and 500 decodes, 27K rows,
// 4.3, a launch in a graph of 200).  A decode request is a thread; the tokens of a prefill request are dealt to several workgroups.
// Rows without an owner are none where requests begin one behind the other and none is refused, which each thread sees from its
// requests; only other batches are gone through again, 2048 rows a workgroup, their owners marked in LDS (decodes in another
// order: 3.6 -> 4.5 and 4.3 -> 5.3 us; prompts in another order, 27K rows, 4.3 -> 9.0).
// ------------------------------------------------------------------------------------------
struct Request { int start, q_len, kv_len, row, held, fresh; bool ok; };

__device__ __forceinline__ Request read_request(const TableArgs &a, int r)
{
    const i32x4_a4 m = *(const i32x4_a4 *)(a.seq_meta + 4 * (int64_t)r);
    Request x{m[0], m[1], m[2], m[3], 0, 0, false};
    const bool decode = r >= a.n_prefill;
    x.ok = x.q_len >= 1 && x.kv_len >= x.q_len && x.start >= 0 && x.row >= 0 && x.row < a.n_cache_rows && x.kv_len <= a.per_row &&
           (decode ? x.q_len == 1 && x.start < a.n_decode : x.start <= a.n_rows - x.q_len);
    if (x.ok && a.block_size > 0) {
        int rest;
        x.held = divide(x.kv_len - x.q_len, a.block_size, a.magic, rest);
        x.held += rest > 0 ? 1 : 0;
        int need = divide(x.kv_len, a.block_size, a.magic, rest);
        need += rest > 0 ? 1 : 0;
        x.fresh = need - x.held;
    }
    return x;
}

// Marks rows with an owner, a bit each, of as many rows as a workgroup looks at together.  (Rows beside those are not marked.)
constexpr int kOwnedRows = 2048;
__device__ __forceinline__ void own(uint32_t *owned, int64_t first64, int64_t end64)
{
    int first = (int)min(max(first64, (int64_t)0), (int64_t)kOwnedRows);
    const int last = (int)min(max(end64, (int64_t)0), (int64_t)kOwnedRows) - 1;
    for (; first <= last; first = (first | 31) + 1)
        atomicOr(&owned[first >> 5], (~0u << (first & 31)) & (~0u >> max(31 - last + (first & ~31), 0)));
}

__device__ __forceinline__ int64_t wave_sum(int64_t x)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    return x;
}

__global__ __launch_bounds__(kWgThreads) void token_tables(TableArgs a)
{
    __shared__ int64_t part[kWavesPerWg][4];
    __shared__ uint32_t odd[kWavesPerWg];
    __shared__ uint32_t owned[kOwnedRows / 32];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n_req = a.n_prefill + a.n_decode;
    const int b = (int)blockIdx.x;
    const bool decode_wg = b < a.n_decode_wgs;
    const int prefill_req = decode_wg ? -1 : (b - a.n_decode_wgs) / max(a.wgs_per_prefill, 1);
    const int first_req = decode_wg ? a.n_prefill + b * kWgThreads : prefill_req;    // the workgroup's (first) request
    // blocks of the requests before that, of all, prefill rows, refused requests; and whether prefill requests (decode requests)
    // are anything but one behind the other
    int64_t before = 0, total = 0, prows = 0, refused = 0;
    bool p_apart = false, d_apart = false;
    for (int r = tid; r < n_req; r += kWgThreads) {
        const Request x = read_request(a, r);
        total += x.fresh;
        before += r < first_req ? x.fresh : 0;
        refused += x.ok ? 0 : 1;
        if (r < a.n_prefill) {
            const int32_t *m = a.seq_meta + 4 * (int64_t)r;
            prows += max(x.q_len, 0);
            p_apart |= !x.ok || x.start != (r > 0 ? (int64_t)m[-4] + m[-3] : 0);
        } else {
            d_apart |= !x.ok || x.start != r - a.n_prefill;
        }
    }
    before = wave_sum(before); total = wave_sum(total); prows = wave_sum(prows); refused = wave_sum(refused);
    const uint32_t apart = (__ballot(p_apart) != 0 ? 1u : 0u) | (__ballot(d_apart) != 0 ? 2u : 0u);
    if (lane == 0) { part[wave][0] = before; part[wave][1] = total; part[wave][2] = prows; part[wave][3] = refused; odd[wave] = apart; }
    __syncthreads();
    before = total = prows = refused = 0;
    uint32_t any = 0u;
#pragma unroll
    for (int w = 0; w < kWavesPerWg; ++w) { before += part[w][0]; total += part[w][1]; prows += part[w][2]; refused += part[w][3]; any |= odd[w]; }
    const int64_t covered = prows + a.n_decode;
    const bool beyond = covered > a.n_rows;
    if (__builtin_expect(beyond, 0)) {
        // Decode requests whose rows lie behind the last one take nothing: no row would enter their blocks.
        int64_t lost = 0, lost_before = 0;
        for (int r = a.n_prefill + tid; r < n_req; r += kWgThreads) {
            const Request x = read_request(a, r);
            if (!x.ok || prows + x.start < a.n_rows) continue;
            lost += x.fresh;
            lost_before += r < first_req ? x.fresh : 0;
        }
        lost = wave_sum(lost); lost_before = wave_sum(lost_before);
        __syncthreads();
        if (lane == 0) { part[wave][0] = lost_before; part[wave][1] = lost; }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWavesPerWg; ++w) { before -= part[w][0]; total -= part[w][1]; }
    }
    const bool enough = total <= a.n_free;
    if (b == 0 && tid == 0) {
        a.report[0] = enough ? (int32_t)total : 0;
        a.report[1] = enough ? 0 : (int32_t)min(total - a.n_free, (int64_t)0x7fffffff);
        a.report[2] = (int32_t)refused;
        a.report[3] = (int32_t)min(covered, (int64_t)0x7fffffff);
    }
    // Row `at` is token `pos` of request x, whose new blocks are free_blocks[taken ..].
    auto write_row = [&](const Request &x, int64_t at, int pos, int64_t taken) {
        int slot = -1;
        if (a.block_size == 0) {
            slot = x.row * a.per_row + pos;
        } else if (enough) {
            int rest;
            const int index = divide(pos, a.block_size, a.magic, rest);
            int32_t *entry = a.block_table + (int64_t)x.row * a.max_blocks + index;
            int block;
            if (index >= x.held) {
                block = a.free_blocks[taken + (index - x.held)];
                // a new block begins with a new token, whose row enters it
                if (rest == 0) *entry = block;
            } else {
                block = *entry;
            }
            if (block >= 0 && block < a.n_blocks) slot = block * a.block_size + rest;
        }
        a.slots[at] = slot;
        a.positions[at] = pos;
    };
    if (decode_wg) {
        const int r = first_req + tid;
        Request x{};
        if (r < n_req) x = read_request(a, r);
        if (beyond && prows + x.start >= a.n_rows) x = Request{};
        // exclusive prefix sum over the workgroup's requests (a decode takes one block at the most)
        const uint64_t takes = __ballot(x.fresh > 0);
        __syncthreads();
        if (lane == 0) part[wave][0] = __popcll(takes);
        __syncthreads();
        for (int w = 0; w < wave; ++w) before += part[w][0];
        before += __popcll(takes & ((uint64_t(1) << lane) - 1));
        if (x.ok) write_row(x, prows + x.start, x.kv_len - 1, before);
    } else {
        const Request x = read_request(a, prefill_req);
        const int chunk = (b - a.n_decode_wgs) - prefill_req * a.wgs_per_prefill;
        for (int64_t i = (int64_t)chunk * kWgThreads + tid; x.ok && i < x.q_len; i += (int64_t)a.wgs_per_prefill * kWgThreads)
            write_row(x, x.start + i, x.kv_len - x.q_len + (int)i, before);
    }
    // Every row that is no accepted request's gets no slot.  Padding rows are dealt over the whole launch.
    auto write_none = [&](int64_t i) { a.slots[i] = -1; a.positions[i] = 0; };
    if ((any & 1u) == 0u)
        for (int64_t i = covered + (int64_t)b * kWgThreads + tid; i < a.n_rows; i += (int64_t)gridDim.x * kWgThreads) write_none(i);
    // Requests with gaps, in another order, refused or over each other: what has an owner is marked.  (All rows for the sake of
    // prefill requests, the decode rows otherwise.)
    if (__builtin_expect(any != 0u, 0)) {
        const int64_t end = (any & 1u) != 0u ? (int64_t)a.n_rows : min(covered, (int64_t)a.n_rows);
        for (int64_t w0 = ((any & 1u) != 0u ? 0 : prows) + (int64_t)b * kOwnedRows; w0 < end; w0 += (int64_t)gridDim.x * kOwnedRows) {
            const int n = (int)min((int64_t)kOwnedRows, end - w0);
            __syncthreads();
            if (tid < kOwnedRows / 32) owned[tid] = 0u;
            __syncthreads();
            for (int r = tid; r < n_req; r += kWgThreads) {
                const Request x = read_request(a, r);
                const int64_t first = x.start + (r < a.n_prefill ? 0 : prows) - w0;
                if (x.ok) own(owned, first, first + x.q_len);
            }
            __syncthreads();
            for (int i = tid; i < n; i += kWgThreads)
                if ((owned[i >> 5] >> (i & 31) & 1u) == 0u) write_none(w0 + i);
        }
    }
}

hipError_t launch_tables(const TableArgs &a, hipStream_t stream)
{
    token_tables<<<dim3(a.n_decode_wgs + a.n_prefill * a.wgs_per_prefill), dim3(kWgThreads), 0, stream>>>(a);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------
// Append.  A lane owns 16 channels of a head as two 16-byte pieces chosen so that both members of every rotated pair are
// its own: pieces p and p + rot_dim / 16 with the half layout, neighbours with the interleaved one and behind the rotated
// channels.  Normalising a head is then a sum over head_dim / 16 neighbouring lanes and rotating it needs no exchange.
// A wavefront works on one row, 1024 / head_dim heads at a time, query, key and value heads alike; a lane's pairs are the
// same in every head, and their cosines and sines are worked out once a row and group of heads.  The angle is a fixed-point product: the
// pair's turns per position as a fraction of 2^64 times the position, whose upper word is the angle as a signed fraction
// of a turn to 2^-32, for every position; the sine unit takes turns.
// What bounds it is memory for many rows (8192 rows, 32 / 8 heads of 128 channels, 201 MB: 42 us, 4.8 TB/s, from memory and 33
// again and again; 8192 x 32 / 32 heads, 403 MB: 79 us, 5.1 TB/s) and the launch for few (16 rows 2.7 us in a graph of 200).
// 54 and 11.8 us with one wavefront a row, angles worked out by every lane and the loads behind the slot's.
// ------------------------------------------------------------------------------------------
template <int DT> struct Elem;
template <> struct Elem<0> { using t = _Float16; };
template <> struct Elem<1> { using t = __bf16; };

template <int DT, int D, int ROPE, int STEPS>
__global__ __launch_bounds__(kWgThreads) void append_tokens(AppendArgs a)
{
    using elem = typename Elem<DT>::t;
    typedef elem e8 __attribute__((ext_vector_type(8)));
    constexpr int LPH = D / 16, HPW = kWaveSize / LPH;
    __shared__ __attribute__((aligned(16))) float turn[kWavesPerWg][D];      // cosine and sine of each pair of a row
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = (int)blockIdx.x * kWavesPerWg + wave;
    if (row >= a.n_rows) return;
    const int slot = ((const POD_CONST int32_t *)a.slots)[row], pos = ((const POD_CONST int32_t *)a.positions)[row];
    const int sub = lane % LPH, pairs = a.rot_dim / 16;
    const bool turns = sub < pairs;
    int c0 = 2 * sub, c1 = 2 * sub + 1;               // the lane's pieces of a head
    if (ROPE == POD_ROPE_HALF && turns) { c0 = sub; c1 = sub + pairs; }
    // The heads are asked for ahead of what they wait for, of padding rows as well.
    const int n_heads = a.n_q_heads + 2 * a.n_kv_heads;
    const int head0 = (int)blockIdx.y * STEPS * HPW + lane / LPH;
    e8 in[STEPS][2];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int head = min(head0 + s * HPW, n_heads - 1), k = head - a.n_q_heads, v = k - a.n_kv_heads;
        const elem *src = k < 0 ? (const elem *)a.q + row * a.q_stride + head * D
                                : (v < 0 ? (const elem *)a.k + row * a.k_stride + k * D : (const elem *)a.v + row * a.v_stride + v * D);
        in[s][0] = *(const e8 *)(src + c0 * 8);
        in[s][1] = *(const e8 *)(src + c1 * 8);
    }
    if (slot < 0 || slot >= a.n_slots) return;
    int at;
    const int block = divide(slot, a.per_block, a.magic, at);
    const int64_t cache_base = (int64_t)block * a.block_elems + (int64_t)at * a.tok_stride;
    // A pair's cosine and sine are worked out by one lane (or two pairs by it) and handed to the lanes of all heads through
    // LDS: worked out by every lane for itself they were half of the kernel's vector work.
    float cs[8], sn[8];
    if (pairs > 0) {
#pragma unroll
        for (int i = lane; i < D / 2; i += kWaveSize)
            if (i < 8 * pairs) {
                const u32x2 f = *(const u32x2 *)(a.table + i);
                uint32_t angle = __umulhi((uint32_t)pos, f[0]) + (uint32_t)pos * f[1];
                if (pos < 0) angle -= f[0];
                const float x = (float)(int32_t)angle * 0x1p-32f;
                turn[wave][2 * i] = __builtin_amdgcn_cosf(x) * a.cos_sin_scale;
                turn[wave][2 * i + 1] = __builtin_amdgcn_sinf(x) * a.cos_sin_scale;
            }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        if (turns) {
#pragma unroll
            for (int i = 0; i < 8; ++i) { cs[i] = turn[wave][16 * sub + 2 * i]; sn[i] = turn[wave][16 * sub + 2 * i + 1]; }
        }
    }
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int head = head0 + s * HPW;
        if (head >= n_heads) break;                   // (whole groups of lanes)
        const bool is_q = head < a.n_q_heads, is_k = !is_q && head < a.n_q_heads + a.n_kv_heads;
        const int kv = head - a.n_q_heads - (is_k ? 0 : a.n_kv_heads);
        elem *dst = is_q ? (elem *)a.q_out + ((int64_t)row * a.n_q_heads + head) * D
                         : (elem *)(is_k ? a.k_cache : a.v_cache) + cache_base + kv * a.head_stride;
        e8 r0 = in[s][0], r1 = in[s][1];
        const bool norm = is_q ? a.norm_q : is_k && a.norm_k;
        float x[8], y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) { x[i] = (float)r0[i]; y[i] = (float)r1[i]; }
        if (a.norm_q | a.norm_k) {
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) ss += x[i] * x[i] + y[i] * y[i];
#pragma unroll
            for (int d = 1; d < LPH; d *= 2) ss += __shfl_xor(ss, d);
            const float inv = rsqrtf(ss * (1.f / D) + a.eps);
            const elem *w = (const elem *)(is_q ? a.q_weight : a.k_weight);
            if (norm && w) {
                const e8 w0 = *(const e8 *)(w + c0 * 8), w1 = *(const e8 *)(w + c1 * 8);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[i] *= inv * ((float)w0[i] + a.weight_offset);
                    y[i] *= inv * ((float)w1[i] + a.weight_offset);
                }
            } else if (norm) {
#pragma unroll
                for (int i = 0; i < 8; ++i) { x[i] *= inv; y[i] *= inv; }
            }
        }
        const bool turned = turns && (is_q || is_k);
        if (turned) {
            if (ROPE == POD_ROPE_HALF) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float u = x[i], v = y[i];
                    x[i] = u * cs[i] - v * sn[i];
                    y[i] = v * cs[i] + u * sn[i];
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float u = x[2 * i], v = x[2 * i + 1];
                    x[2 * i] = u * cs[i] - v * sn[i];
                    x[2 * i + 1] = v * cs[i] + u * sn[i];
                    u = y[2 * i]; v = y[2 * i + 1];
                    y[2 * i] = u * cs[4 + i] - v * sn[4 + i];
                    y[2 * i + 1] = v * cs[4 + i] + u * sn[4 + i];
                }
            }
        }
        if (norm || turned) {                         // other channels are copied as they are
#pragma unroll
            for (int i = 0; i < 8; ++i) { r0[i] = (elem)x[i]; r1[i] = (elem)y[i]; }
        }
        *(e8 *)(dst + c0 * 8) = r0;
        *(e8 *)(dst + c1 * 8) = r1;
    }
}

template <int DT, int D, int STEPS>
static hipError_t launch_append_steps(const AppendArgs &a, int layout, hipStream_t stream)
{
    constexpr int heads = append_heads(D) * STEPS;
    const int n_heads = a.n_q_heads + 2 * a.n_kv_heads;
    const dim3 grid(((uint32_t)a.n_rows + kWavesPerWg - 1) / kWavesPerWg, (n_heads + heads - 1) / heads), threads(kWgThreads);
    if (layout == POD_ROPE_HALF) append_tokens<DT, D, POD_ROPE_HALF, STEPS><<<grid, threads, 0, stream>>>(a);
    else append_tokens<DT, D, POD_ROPE_INTERLEAVED, STEPS><<<grid, threads, 0, stream>>>(a);
    return hipGetLastError();
}
template <int DT, int D>
static hipError_t launch_append_as(const AppendArgs &a, int layout, hipStream_t stream)
{
    // One group of heads a wavefront up to a few rounds of the chip, then two, which halves the work on angles.  us at 128
    // channels, 32 / 8 heads, one group / two / four: 16 rows 3.0 / 3.6 / 5.0, 256 rows 3.5 / 4.0 / 5.4, 1024 rows (6144
    // wavefronts of one group) 6.2 / 6.1 / 7.0; 256 channels, 4096 rows 26.6 / 23.4 / 25.1; 64 channels, 1024 rows (half
    // as many) 4.30 / 4.33 / 5.1, 2048 rows 6.1 / 5.9.
    const int64_t waves = (int64_t)a.n_rows * ((a.n_q_heads + 2 * a.n_kv_heads + append_heads(D) - 1) / append_heads(D));
    return waves < 6 * 1024 ? launch_append_steps<DT, D, 1>(a, layout, stream) : launch_append_steps<DT, D, 2>(a, layout, stream);
}

hipError_t launch_append(const AppendArgs &a, int dtype, int head_dim, int layout, hipStream_t stream)
{
    if (dtype == POD_F16 && head_dim == 64) return launch_append_as<0, 64>(a, layout, stream);
    if (dtype == POD_F16 && head_dim == 128) return launch_append_as<0, 128>(a, layout, stream);
    if (dtype == POD_F16 && head_dim == 256) return launch_append_as<0, 256>(a, layout, stream);
    if (dtype == POD_BF16 && head_dim == 64) return launch_append_as<1, 64>(a, layout, stream);
    if (dtype == POD_BF16 && head_dim == 128) return launch_append_as<1, 128>(a, layout, stream);
    if (dtype == POD_BF16 && head_dim == 256) return launch_append_as<1, 256>(a, layout, stream);
    return hipErrorInvalidValue;
}

}  // namespace pod
