// Attention of new tokens over a paged cache: O = softmax(scale Q K^T) V, the keys and values of a sequence in the rows of its pages, the new
// tokens of all sequences one behind the other.
//
// As fwa_sequence_forward.hip: one pass over the keys with a running reference and sum per row, S^T = K Q^T and O^T += V^T P^T, tiles of K and
// V through LDS, two of each.  What differs: the rows of a workgroup are those of all heads that share the keys, token by token, so that a tile is loaded once for
// all of them and single tokens fill a block as far as they can; the loads of 16 rows of a tile go to one page, whose number is
// looked up by the scalar unit two tiles ahead; how many rows and keys a sequence has is known on the device alone.
#include "fwa_page.h"

#include <type_traits>

namespace fwa {
namespace {

// A row's reference moves when a score exceeds it by more than this, as in the attention of whole sequences.
constexpr float kSlack = 6.f;
constexpr int kFewRows = 32;  // rows (new tokens times heads of a group) up to which the waves of a workgroup share out the keys
constexpr int kLeastTiles = 4;  // of a wave, where workgroups share out the keys

// One form's share of a call.
struct PagePlan {
    int rows;         // of a block
    int group;        // heads of queries per head of keys
    int each;         // blocks of each sequence, 0: as many as it has, found by a search
    int blocks, splits;
    int least;        // tiles that a part has at least
    int only;         // 1: sequences of few rows are another form's, -1: those of more, 0: all are this one's
    FastDiv by_kv, by_splits, by_each, by_group, by_sub;
    size_t slots;     // blocks * KV * splits * rows: rows of parts
    float* part_o;    // [block][kv][split][rows][D], not divided by the sum
    float* part_ml;   // [block][kv][split][rows][2]
};

// A block of a sequence's rows (token-major: row r is token r / group, head r % group of the group).
struct PageBlock {
    int n, row0, rows;  // sequence, first row, rows of the sequence
    int begin;          // first new token
    int start, klen;    // place of token 0, keys
    int kend;           // keys up to this one are seen by a row of the block
};

// false: nothing to do
template <int ROWS>
__device__ __forceinline__ bool page_block(const PageArgs& a, const PagePlan& plan, int block, PageBlock& b) {
    int n, within;
    if (plan.each > 0) {
        n = (int)fastdiv((uint32_t)block, plan.by_each);
        within = block - n * plan.each;
    } else {
        // Sequence n begins at block offsets[n] group / ROWS + n, so that none shares a block with another and a few blocks have no rows.  The last one
        // that begins at or in front of this block, 64 candidates at a time.
        const int lane = (int)(threadIdx.x & 63u);
        int lo = 0, size = a.N, first = 0;
        for (;;) {
            const int step = (size + 63) / 64, at = lo + lane * step;
            const int offset = page_offset(a.offsets[at < a.N ? at : a.N - 1], a.rows);
            const int f = (int)((uint32_t)offset * (uint32_t)plan.group / (uint32_t)ROWS) + at;
            const int count = __popcll(__ballot(at < lo + size && f <= block));
            if (count == 0) return false;
            first = __builtin_amdgcn_readlane(f, count - 1);
            lo += (count - 1) * step;
            if (step == 1) break;
            size = step < a.N - lo ? step : a.N - lo;
        }
        n = lo;
        within = block - first;
    }
    b.n = n;
    b.begin = page_offset_of(a, n);
    const int count = page_count(b.begin, page_offset_of(a, n + 1), a.most);
    b.rows = count * plan.group;
    b.row0 = within * ROWS;
    if (within < 0 || b.row0 >= b.rows) return false;
    if (plan.only != 0 && (b.rows <= kFewRows) != (plan.only < 0)) return false;
    b.start = page_length_of(a, n);
    b.klen = page_keys(b.start, count, a.width, a.page_size);
    const int last_row = b.rows - b.row0 < ROWS ? b.rows - 1 : b.row0 + ROWS - 1;
    const int last = b.start + (int)fastdiv((uint32_t)last_row, plan.by_group);
    b.kend = a.causal && last + 1 < b.klen ? last + 1 : b.klen;
    return true;
}
// Parts of a block's tiles that have any.
__device__ __forceinline__ int page_parts(const PagePlan& plan, int tiles, int& per) {
    per = (tiles + plan.splits - 1) / plan.splits;
    if (per < plan.least) per = plan.least;
    return (tiles + per - 1) / per;
}

// acc[m][b] += V[rows of the block][channels 32 b ..]^T times w[m], for MB blocks of rows at once: the operand is read once for all.
template <class T, int D, int MB>
__device__ __forceinline__ void page_accumulate(const SeqColumnReader<T, D>& reader, f32x16 (&acc)[MB][D / 32], uint32_t tile, int block, const f32x16 (&w)[MB]) {
    constexpr int RB = D * SeqSize<T>::value;
    if constexpr (MB == 1) {
        reader.accumulate(acc[0], tile, block, w[0]);
    } else {
        static_assert(!__is_same(T, SeqF32), "16-bit data");
        constexpr bool F16 = __is_same(T, SeqF16);
        tile += (uint32_t)(32 * RB * block);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            u32x4 x[MB];
#pragma unroll
            for (int m = 0; m < MB; ++m)
                x[m] = u32x4{pack_e<F16>(w[m][8 * t], w[m][8 * t + 1]), pack_e<F16>(w[m][8 * t + 2], w[m][8 * t + 3]),
                             pack_e<F16>(w[m][8 * t + 4], w[m][8 * t + 5]), pack_e<F16>(w[m][8 * t + 6], w[m][8 * t + 7])};
#pragma unroll
            for (int b = 0; b < D / 32; ++b) {
                const uint32_t first = reader.at ^ (uint32_t)(64 * b), second = first ^ (seq_swizzle<RB>(8u) << 4);
                const uint2 p = seq_lds_tr(tile + first + (uint32_t)(16 * t) * RB);
                const uint2 q = seq_lds_tr(tile + second + (uint32_t)(16 * t + 8) * RB);
#pragma unroll
                for (int m = 0; m < MB; ++m) acc[m][b] = seq_dot<T>(u32x4{p.x, p.y, q.x, q.y}, x[m], acc[m][b]);
            }
        }
    }
}

// A wave's loads of a tile: its rows in groups of 16 (or 8) that lie in one page each.
template <int RB, int KT, int WAVES>
struct PageLoader {
    static constexpr int kRows = KT / WAVES, kGroup = kRows < kPageRows ? kRows : kPageRows, kGroups = kRows / kGroup, kLoads = kGroup * RB / 1024;
    static_assert(kLoads >= 1 && kLoads * 1024 == kGroup * RB, "a group is a whole number of loads");
    uint32_t off[kLoads];
    uint32_t to;    // of the wave's rows in the tile
    int row;
    __device__ __forceinline__ void init(uint32_t wave, uint32_t lane, uint32_t token_bytes) {
        row = (int)wave * kRows;
        to = wave * (uint32_t)(kRows * RB);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const uint32_t at = (uint32_t)i * 1024u + lane * 16u, r = at / RB, place = (at % RB) / 16u;
            off[i] = r * token_bytes + ((place ^ seq_swizzle<RB>((uint32_t)row + r)) * 16u);
        }
    }
    __device__ __forceinline__ void issue(const u32x4& source, uint32_t lds, int group) const {
        seq_loads_to_lds<kLoads, 1024>(source, off, lds + to + (uint32_t)(group * kGroup * RB));
    }
    __device__ __forceinline__ void zero(uint32_t lds, int group, uint32_t lane) const {
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(lds + to + (uint32_t)(group * kGroup * RB) + (uint32_t)i * 1024u + lane * 16u) = u32x4{0u, 0u, 0u, 0u};
    }
};

// Two forms.  Rows: the W waves of a workgroup have 32 MB rows each and share the tiles.  KEYS: all have the same 32 rows and every W-th tile each, in
// buffers of their own without a barrier, and join what they have at the end.  Workgroups share out the keys of a block besides where blocks are few.
template <class T, int D, int W, int KT, int MB, bool KEYS, int OCC>
__global__ void __launch_bounds__(64 * W, OCC) page_forward_kernel(PageArgs a, PagePlan plan) {
    constexpr int E = SeqSize<T>::value, RB = D * E, NC = RB / 32, NB = D / 32, KS = KT / 32, SUB = KT / kPageRows;
    constexpr int ROWS = KEYS ? 32 : 32 * MB * W, TURN = KEYS ? W : 1;  // of a workgroup; from a wave's tile to its next one
    constexpr uint32_t kTile = KT * RB;
    static_assert(!KEYS || MB == 1, "one block of rows where the waves share out the keys");
    using Loader = PageLoader<RB, KT, KEYS ? 1 : W>;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const uint32_t lane = threadIdx.x & 63u, wave = W == 1 ? 0u : (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t hi = lane >> 5, c = lane & 31u;
    const uint32_t base = lds_offset(lds) + (KEYS ? wave * 4u * kTile : 0u);

    // workgroup -> head of the keys (neighbours, so that each XCD has few of them), part of the keys, block of rows, the last ones of which have most keys
    const uint32_t rest = fastdiv(blockIdx.x, plan.by_kv), hk = blockIdx.x - rest * plan.by_kv.d;
    const uint32_t turn = fastdiv(rest, plan.by_splits), split = rest - turn * plan.by_splits.d;
    const int block = plan.blocks - 1 - (int)turn;
    PageBlock b;
    if (!page_block<ROWS>(a, plan, block, b)) return;
    const int tiles = (b.kend + KT - 1) / KT;
    int per;
    const int parts = page_parts(plan, tiles, per);
    if ((int)split >= (parts > 0 ? parts : 1)) return;
    const int t0 = (int)split * per, t1 = t0 + per < tiles ? t0 + per : tiles;

    const int G = plan.group, klen = b.klen;
    const size_t head_at = (size_t)hk * (size_t)a.head_stride * E;
    const char* const kp = static_cast<const char*>(a.k) + head_at;
    const char* const vp = static_cast<const char*>(a.v) + head_at;
    const uint32_t token_bytes = (uint32_t)(a.token_stride * E);
    const uint64_t page_bytes = (uint64_t)a.page_stride * E;
    const int32_t* const page_row = a.table + (size_t)b.n * a.width;

    Loader load;
    load.init(KEYS ? 0u : wave, lane, token_bytes);
    SeqRowReader<RB> row_reader;
    row_reader.init(hi, c);
    SeqColumnReader<T, D> column_reader;
    column_reader.init(hi, c);

    // The pages of a tile: those of this wave's groups, and which of all have none.
    struct Pages {
        int own[Loader::kGroups];
        uint32_t bad;
    };
    const int last_sub = klen > 0 ? (klen - 1) / kPageRows : 0;
    auto look = [&](int t) {
        Pages p;
        p.bad = 0u;
#pragma unroll
        for (int j = 0; j < SUB; ++j) {
            const int sub = t * SUB + j < last_sub ? t * SUB + j : last_sub;
            const int page = seq_constant(page_row, fastdiv((uint32_t)sub, plan.by_sub));
            p.bad |= page_exists(page, a.pages) ? 0u : 1u << j;
            if (KEYS) p.own[j % Loader::kGroups] = page;
        }
        if constexpr (!KEYS) {
            const int at = (t * KT + load.row) / kPageRows, sub = at < last_sub ? at : last_sub;
            p.own[0] = seq_constant(page_row, fastdiv((uint32_t)sub, plan.by_sub));
        }
        return p;
    };
    auto issue = [&](int t, const Pages& p, uint32_t buf) {
#pragma unroll
        for (int g = 0; g < Loader::kGroups; ++g) {
            const int key = t * KT + load.row + g * Loader::kGroup;
            const int rows = page_group(key, klen, Loader::kGroup, page_exists(p.own[g], a.pages));
            const uint32_t index = fastdiv((uint32_t)key / (uint32_t)kPageRows, plan.by_sub), slot = (uint32_t)key - index * (uint32_t)a.page_size;
            const uint64_t at = rows > 0 ? page_place((uint32_t)p.own[g], slot, page_bytes, token_bytes) : 0u;
            const uint32_t bytes = page_bytes_of(rows, token_bytes, RB);
            const uint32_t kt = base + buf * 2u * kTile, vt = kt + kTile;
            // Rows that no load fills hold zeros: their weights are zero, and zero times whatever else LDS may hold need not be.
            if (rows < Loader::kGroup) {
                load.zero(kt, g, lane);
                load.zero(vt, g, lane);
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            }
            load.issue(lds_source(kp + at, bytes), kt, g);
            load.issue(lds_source(vp + at, bytes), vt, g);
        }
    };

    const int mine0 = KEYS ? t0 + (int)wave : t0;
    Pages here = {}, next = {}, after = {};
    if (mine0 < t1) {
        here = look(mine0);
        issue(mine0, here, 0u);
        next = look(mine0 + TURN);
    }

    // the rows of this lane: token, head of the group, whether there is one
    int limit[MB], token[MB], member[MB];
    bool exists[MB];
    u32x4 qf[MB][NC];
#pragma unroll
    for (int m = 0; m < MB; ++m) {
        const int r = b.row0 + (KEYS ? 0 : 32 * (MB * (int)wave + m)) + (int)c;
        exists[m] = r < b.rows;
        token[m] = exists[m] ? (int)fastdiv((uint32_t)r, plan.by_group) : 0;
        member[m] = exists[m] ? r - token[m] * G : 0;
        const int pos = b.start + token[m];
        limit[m] = a.causal && pos + 1 < klen ? pos + 1 : klen;
#pragma unroll
        for (int s = 0; s < NC; ++s) qf[m][s] = u32x4{0u, 0u, 0u, 0u};
        if (exists[m] && a.scale != 0.f) {  // with a scale of zero the queries are zero: a shut out score times zero would be no score
            const char* const qp = static_cast<const char*>(a.q) + ((size_t)(b.begin + token[m]) * a.ldq + (size_t)(hk * G + member[m]) * D) * E + 16u * hi;
#pragma unroll
            for (int s = 0; s < NC; ++s) qf[m][s] = *reinterpret_cast<const u32x4*>(qp + 32 * s);
            // a negative scale goes into the queries, so that the largest product is the largest score
            if (a.scale < 0.f) {
                constexpr uint32_t kSign = __is_same(T, SeqF32) ? 0x80000000u : 0x80008000u;
#pragma unroll
                for (int s = 0; s < NC; ++s) qf[m][s] ^= kSign;
            }
        }
    }
    // tiles with a key that a row of the block does not see: from mask0 on
    int mask0 = klen / KT;
    if (a.causal) {
        const int to = (b.start + (int)fastdiv((uint32_t)b.row0, plan.by_group) + 1) / KT;
        mask0 = to < mask0 ? to : mask0;
    }

    f32x16 o[MB][NB];
    float top_at[MB], sum[MB];
#pragma unroll
    for (int m = 0; m < MB; ++m) {
#pragma unroll
        for (int x = 0; x < NB; ++x) seq_zero(o[m][x]);
        top_at[m] = -__builtin_inff();
        sum[m] = 0.f;
    }
    const float scale = a.scale == 0.f ? 1.f : fabsf(a.scale) * kLog2e;

    auto step = [&](auto parity, int t) {
        const uint32_t B = parity;
        const uint32_t kt = base + B * 2u * kTile, vt = kt + kTile;
        const uint32_t bad = here.bad;
        lds_loads_done();
        if constexpr (!KEYS) __syncthreads();
        if (t + TURN < t1) {
            issue(t + TURN, next, B ^ 1u);
            if (t + 2 * TURN < t1) after = look(t + 2 * TURN);
        }

        f32x16 s[KS][MB];
#pragma unroll
        for (int k = 0; k < KS; ++k) {
#pragma unroll
            for (int m = 0; m < MB; ++m) seq_zero(s[k][m]);
#pragma unroll
            for (int x = 0; x < NC; ++x) {
                const u32x4 f = row_reader.read(kt, x, k);
#pragma unroll
                for (int m = 0; m < MB; ++m) s[k][m] = seq_dot<T>(f, qf[m][x], s[k][m]);
            }
        }
#pragma unroll
        for (int m = 0; m < MB; ++m) {
            if (t >= mask0 || bad != 0u) {
                const int room = limit[m] - t * KT - 4 * (int)hi;
#pragma unroll
                for (int k = 0; k < KS; ++k)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const bool seen = 32 * k + 8 * (r / 4) + r % 4 < room && !((bad >> (2 * k + r / 8)) & 1u);
                        s[k][m][r] = seen ? s[k][m][r] : -__builtin_inff();
                    }
            }
            float top = s[0][m][0];
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int r = 0; r < 16; ++r) top = fmaxf(top, s[k][m][r]);
            top = seq_max_halves(top) * scale;
            // the reference follows the largest score so far
            if (__any(top > top_at[m] + kSlack)) {
                const float to = top > top_at[m] + kSlack ? top : top_at[m], f = to == top_at[m] ? 1.f : __builtin_amdgcn_exp2f(top_at[m] - to);
                top_at[m] = to;
                sum[m] *= f;
#pragma unroll
                for (int x = 0; x < NB; ++x)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[m][x][r] *= f;
            }
            const float minus = top_at[m] == -__builtin_inff() ? 0.f : -top_at[m];
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[k][m][r] = __builtin_amdgcn_exp2f(fmaf(s[k][m][r], scale, minus));
                    sum[m] += s[k][m][r];
                }
        }
#pragma unroll
        for (int k = 0; k < KS; ++k) page_accumulate<T, D, MB>(column_reader, o, vt, k, s[k]);
        here = next;
        next = after;
    };
    if constexpr (KEYS) {
        uint32_t parity = 0;
        for (int t = mine0; t < t1; t += TURN, parity ^= 1u) step(parity, t);
    } else {
        for (int t = mine0; t < t1; t += 2) {
            step(std::integral_constant<uint32_t, 0>{}, t);
            if (t + 1 < t1) step(std::integral_constant<uint32_t, 1>{}, t + 1);
        }
    }

#pragma unroll
    for (int m = 0; m < MB; ++m) sum[m] = seq_sum_halves(sum[m]);
    if constexpr (KEYS && W > 1) {
        // sums of all waves through LDS, rows 4 floats apart from a multiple of the banks; the last wave has them, the others are done
        constexpr uint32_t kRow = 4u * (D + 4);
        const uint32_t all = lds_offset(lds), sums = all + W * 32u * kRow;
        __syncthreads();
        if (hi == 0) *(__attribute__((address_space(3))) f32x2*)(uintptr_t)(sums + 8u * (32u * wave + c)) = f32x2{top_at[0], sum[0]};
        __syncthreads();
        float top = -__builtin_inff(), total = 0.f, mine = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) top = fmaxf(top, (*(const __attribute__((address_space(3))) f32x2*)(uintptr_t)(sums + 8u * (32u * w + c)))[0]);
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const f32x2 x = *(const __attribute__((address_space(3))) f32x2*)(uintptr_t)(sums + 8u * (32u * w + c));
            const float f = x[1] == 0.f ? 0.f : __builtin_amdgcn_exp2f(x[0] - top);  // a part without weight may have no reference
            total += f * x[1];
            if (w == (int)wave) mine = f;
        }
        if (wave != W - 1) {
#pragma unroll
            for (int x = 0; x < NB; ++x)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *(__attribute__((address_space(3))) f32x4*)(uintptr_t)(all + kRow * (32u * wave + c) + 4u * (32 * x + 8 * q + 4 * hi)) =
                        f32x4{o[0][x][4 * q] * mine, o[0][x][4 * q + 1] * mine, o[0][x][4 * q + 2] * mine, o[0][x][4 * q + 3] * mine};
        }
        __syncthreads();
        if (wave != W - 1) return;
#pragma unroll
        for (int x = 0; x < NB; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[0][x][r] *= mine;
#pragma unroll
        for (int w = 0; w < W - 1; ++w)
#pragma unroll
            for (int x = 0; x < NB; ++x)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x4 y = seq_lds_f32x4(all + kRow * (32u * w + c) + 4u * (32 * x + 8 * q + 4 * hi));
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[0][x][4 * q + e] += y[e];
                }
        top_at[0] = top;
        sum[0] = total;
    }
#pragma unroll
    for (int m = 0; m < MB; ++m) {
        if (!exists[m]) continue;
        const float l = sum[m];
        if (parts > 1) {
            const size_t slot = (((size_t)block * a.KV + hk) * plan.splits + split) * ROWS + (KEYS ? 0 : 32 * (MB * wave + m)) + c;
            float* const to = plan.part_o + slot * D;
            if (l != 0.f)  // nothing reads a part without weight
#pragma unroll
                for (int x = 0; x < NB; ++x)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *reinterpret_cast<f32x4*>(to + 32 * x + 8 * q + 4 * hi) = f32x4{o[m][x][4 * q], o[m][x][4 * q + 1], o[m][x][4 * q + 2], o[m][x][4 * q + 3]};
            if (hi == 0) *reinterpret_cast<f32x2*>(plan.part_ml + 2 * slot) = f32x2{top_at[m], l};
            continue;
        }
        const bool any = l != 0.f;  // NaN too
        const float f = any ? 1.f / l : 0.f;
        const size_t row = (size_t)(b.begin + token[m]), head = hk * G + member[m];
        char* const to = static_cast<char*>(a.o) + (row * a.ldo + head * D) * E;
#pragma unroll
        for (int x = 0; x < NB; ++x)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = any ? o[m][x][4 * q + e] * f : 0.f;
                seq_store4<T>(to, 32 * x + 8 * q + 4 * hi, y[0], y[1], y[2], y[3]);
            }
        if (a.stats && hi == 0) *reinterpret_cast<f32x2*>(a.stats + 2 * (row * a.H + head)) = f32x2{any ? top_at[m] : -__builtin_inff(), any ? log2f(l) : 0.f};
    }
}

// Joins the parts of blocks whose keys are shared out: a thread has four channels of a row.
template <class T, int D, int ROWS, int KT>
__global__ void __launch_bounds__(256) page_join_kernel(PageArgs a, PagePlan plan) {
    constexpr int E = SeqSize<T>::value, kThreads = D / 4, kRows = 256 / kThreads, kTurns = ROWS / kRows;
    const uint32_t unit = blockIdx.x / kTurns, turn = blockIdx.x - unit * kTurns;
    const uint32_t block = fastdiv(unit, plan.by_kv), hk = unit - block * plan.by_kv.d;
    PageBlock b;
    if (!page_block<ROWS>(a, plan, (int)block, b)) return;
    int per;
    const int parts = page_parts(plan, (b.kend + KT - 1) / KT, per);
    const int slot = (int)(turn * kRows + threadIdx.x / kThreads), r = b.row0 + slot, channel = 4 * (int)(threadIdx.x % kThreads);
    if (parts <= 1 || r >= b.rows) return;
    const size_t first = ((size_t)block * a.KV + hk) * plan.splits * ROWS + slot;
    float top = -__builtin_inff();
    for (int s = 0; s < parts; ++s) top = fmaxf(top, plan.part_ml[2 * (first + (size_t)s * ROWS)]);
    float l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < parts; ++s) {
        const size_t part = first + (size_t)s * ROWS;
        const f32x2 ml = *reinterpret_cast<const f32x2*>(plan.part_ml + 2 * part);
        if (ml[1] == 0.f) continue;
        const float f = __builtin_amdgcn_exp2f(ml[0] - top);
        const f32x4 x = *reinterpret_cast<const f32x4*>(plan.part_o + part * D + channel);
        l += f * ml[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += f * x[e];
    }
    const int token = (int)fastdiv((uint32_t)r, plan.by_group);
    const size_t row = (size_t)(b.begin + token), head = hk * plan.group + (r - token * plan.group);
    const bool any = l != 0.f;
    const float f = any ? 1.f / l : 0.f;
    char* const to = static_cast<char*>(a.o) + (row * a.ldo + head * D) * E;
    seq_store4<T>(to, channel, o[0] * f, o[1] * f, o[2] * f, o[3] * f);
    if (a.stats && channel == 0) *reinterpret_cast<f32x2*>(a.stats + 2 * (row * a.H + head)) = f32x2{any ? top : -__builtin_inff(), any ? log2f(l) : 0.f};
}

// Tile sizes and waves of the two forms.
constexpr int page_tile_keys(int row_bytes, bool keys) { return row_bytes >= 512 || keys ? 32 : 64; }
constexpr int page_waves(int row_bytes, bool keys) { return keys ? seq_keys_waves(row_bytes) : 4; }
constexpr int page_row_blocks(int, bool) { return 1; }
constexpr int page_occupancy(int row_bytes, bool keys) { return row_bytes == 128 && !keys ? 3 : 1; }

template <class T, int D, bool KEYS>
hipError_t launch(const PageArgs& a, const PagePlan& plan, hipStream_t s) {
    constexpr int RB = D * SeqSize<T>::value, W = page_waves(RB, KEYS), KT = page_tile_keys(RB, KEYS), MB = page_row_blocks(RB, KEYS), ROWS = KEYS ? 32 : 32 * MB * W;
    constexpr size_t tiles = 4 * (size_t)KT * RB * (KEYS ? W : 1), sums = KEYS && W > 1 ? (size_t)W * 32 * (4 * (D + 4) + 8) : 0, lds = tiles > sums ? tiles : sums;
    auto* const kernel = &page_forward_kernel<T, D, W, KT, MB, KEYS, page_occupancy(RB, KEYS)>;
    hipError_t e = allow_lds(reinterpret_cast<const void*>(kernel), lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)plan.blocks * (unsigned)a.KV * (unsigned)plan.splits), dim3(64 * W), lds, s, a, plan);
    e = hipGetLastError();
    if (e != hipSuccess || plan.splits == 1) return e;
    constexpr unsigned turns = ROWS / (256 / (D / 4));
    hipLaunchKernelGGL((page_join_kernel<T, D, ROWS, KT>), dim3((unsigned)plan.blocks * (unsigned)a.KV * turns), dim3(256), 0, s, a, plan);
    return hipGetLastError();
}

// The forms that a call takes, and how much of each: keys[0] rows, keys[1] keys; blocks 0: not this one.
struct PagePlans {
    PagePlan form[2];
};
bool page_plans(const PageArgs& a, PagePlans& p) {
    const int size = a.dtype == 0 ? 4 : 2, RB = a.D * size, G = a.H / a.KV, cus = cu_count();
    const long long most_rows = (long long)a.most * G, capacity = (long long)a.width * a.page_size;
    const bool few = most_rows <= kFewRows, same = (long long)a.N * a.most == a.rows;  // all sequences have few rows; all have the same number
    for (int keys = 0; keys < 2; ++keys) {
        PagePlan& f = p.form[keys];
        f = PagePlan{};
        if (keys ? !few && same : few) continue;
        const int KT = page_tile_keys(RB, keys), W = page_waves(RB, keys);
        f.rows = keys ? 32 : 32 * page_row_blocks(RB, keys) * W;
        f.group = G;
        f.only = few || same ? 0 : keys ? -1 : 1;
        // blocks: a number for each sequence, or as many as the rows fill and one more for each sequence
        const long long each = keys ? 1 : (most_rows + f.rows - 1) / f.rows, all = (long long)a.rows * G / f.rows + a.N;
        f.each = each * a.N <= all ? (int)each : 0;
        const long long blocks = f.each ? each * a.N : all;
        const double base = (double)blocks * a.KV;
        if (base * 64.0 * W > 4.0e9 || base * (f.rows / 8.0) * 256.0 > 4.0e9) return false;  // threads of a launch
        f.blocks = (int)blocks;
        const long long tiles = (capacity + KT - 1) / KT;
        f.least = kLeastTiles * (keys ? W : 1);
        long long splits = (long long)(2.0 * cus / base);
        if (splits > tiles / f.least) splits = tiles / f.least;
        if (splits > 64) splits = 64;
        f.splits = splits < 1 ? 1 : (int)splits;
        if (f.splits == 1) f.least = 1;
        f.by_kv = make_fastdiv((uint32_t)a.KV);
        f.by_splits = make_fastdiv((uint32_t)f.splits);
        f.by_each = make_fastdiv(f.each > 0 ? (uint32_t)f.each : 1u);
        f.by_group = make_fastdiv((uint32_t)G);
        f.by_sub = make_fastdiv((uint32_t)(a.page_size / kPageRows));
        f.slots = f.splits > 1 ? (size_t)f.blocks * a.KV * f.splits * f.rows : 0;
    }
    return true;
}

template <class T, int D>
hipError_t launch(const PageArgs& a, const PagePlans& p, hipStream_t s) {
    hipError_t e = hipSuccess;
    if (p.form[0].blocks > 0) e = launch<T, D, false>(a, p.form[0], s);
    if (e == hipSuccess && p.form[1].blocks > 0) e = launch<T, D, true>(a, p.form[1], s);
    return e;
}
template <class T>
hipError_t launch(const PageArgs& a, const PagePlans& p, hipStream_t s) {
    if (a.D == 32) return launch<T, 32>(a, p, s);
    if (a.D == 64) return launch<T, 64>(a, p, s);
    return launch<T, 128>(a, p, s);
}

}  // namespace

bool page_forward_fits(const PageArgs& a) {
    PagePlans p;
    return page_plans(a, p);
}

size_t page_forward_workspace(const PageArgs& a) {
    PagePlans p;
    if (!page_plans(a, p)) return 0;
    return (p.form[0].slots + p.form[1].slots) * (size_t)(a.D + 2) * sizeof(float);
}

hipError_t launch_page_forward(const PageArgs& a, void* workspace, hipStream_t s) {
    PagePlans p;
    if (!page_plans(a, p)) return hipErrorInvalidValue;
    float* at = static_cast<float*>(workspace);
    for (PagePlan& f : p.form) {
        if (f.slots == 0) continue;
        f.part_o = at;
        f.part_ml = at + f.slots * (size_t)a.D;
        at = f.part_ml + 2 * f.slots;
    }
    if (a.dtype == 0) return launch<SeqF32>(a, p, s);
    return a.dtype == 1 ? launch<SeqBf16>(a, p, s) : launch<SeqF16>(a, p, s);
}

}  // namespace fwa
