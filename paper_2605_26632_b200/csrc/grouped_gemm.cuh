// Linear layers whose rows may be grouped by expert, on bf16 or MXFP4 operands, for sm_100a:
//     Y[m, n] = bf16( r_m * sum_k X[m,k] W_g[n,k] + bias_g[n] + Yr[m,n] ),   offsets[g] <= m < offsets[g + 1]
// (one group over all rows where there are no offsets).
//
// The weights are the MMA's A operand and the tokens its B operand: D[n, m] = W X^T.  M of the instruction is fixed (128
// rows of W per CTA) while N goes in small steps, so a group's last tile costs what its rows need, a batch of single
// tokens runs the narrowest instruction there is, and ragged groups need no padding in memory.
//
// Persistent, warp-specialised.  Per CTA (or CTA pair when CG == 2: 256 rows of W, each CTA its own 128 and half of the tokens):
//   warp 0      TMA loads of the W tile and its scales into a ring of STAGES stages
//   warp 3      TMA loads of the X tile (one box, or boxes of BOX rows where the tile has few) and its scales into the same stages
//   warp 1      MMA issuer: copies the stage's scales into tensor memory, four MMAs per 128-byte slice of K
//               (kind::mxf4 block_scale: K = 64 each; kind::f16: K = 16), commits to the stage's empty barrier
//   warp 2      the work list (see GroupSchedule), before the roles start
// (A load costs its warp about 75 cycles whatever it fetches: one warp with eight of them per stage took 590 cycles for what the
// MMAs do in 512.  Hence two warps, few and large boxes, and the scale tiles of all tokens in one.)
//   warps 4..11 epilogue: two warps per tensor-memory lane quarter, 32 tokens at a time
// Issue loops are run by whole warps and waits end in a vote, as in sparse_gemm.cuh.
//
// What bounds it.  Whole tiles: the tensor pipe.  A stage of a 256 x 256 MXFP4 tile (256 elements of K) takes 401 ns, 6.2 PFLOP/s over
// 74 pairs, of which the copies of its six scale tiles into tensor memory are 40 (without them 360), and 281 ns without its
// MMAs; a bf16 stage (64 elements) takes 410 ns, 1.51 PFLOP/s (8192 x 2048 x 4096 in one group 94 us, cuBLASLt's product 96).  4096 x
// 10240 x 3840 MXFP4 57 us, 5.6 PFLOP/s, under the power cap 20 % more.  Few tokens: the weights out of HBM, 96 rows on 40 of 64 bf16 experts
// of 2048 x 1536 5.5 TB/s, 1 x 4096 x 75776 MXFP4 5.8 TB/s; on the smallest calls 2.8 us that no stage is in (launch, descriptors, the
// first stage's latency, epilogue), and while few SMs have a tile the 64 bytes per cycle that one of them takes in.  Not kept: 32-row tiles of W for few tokens (every SM then reads the same few lines of X for a quarter
// of the weights: 19.8 us against 12.5 on 1 x 3840 x 23040), 128-token tiles on single CTAs (slower than one of the other two
// everywhere), tiles of whole groups first and all the rest behind (reads the weights twice).
//
// The epilogue reads the accumulator in the 16 x 256-bit shape: a lane holds two neighbouring tokens of one row of W, which
// is what stmatrix with .trans wants to lay 8 x 8 blocks down token by token; a residual comes in through ldmatrix with .trans.
// The staged 32 x 32 block leaves as 64 bytes per token, rows behind the group's last one and columns behind N left out (a TMA
// store could clip neither at a group's end).
#pragma once

#include "epilogue.cuh"
#include "mxfp4.cuh"
#include "ptx.cuh"

namespace lynx {

constexpr int GG_MAX_GROUPS = 1024;
constexpr int XRES_ROWS = 16, XRES_MIN_STAGES = 4;
constexpr int GG_GROUP_TILES = 16;  // token tiles swept over all of W before the next ones

struct GroupedParams {
    int64_t M, N, K;
    const int32_t* offsets;  // [groups + 1] or nullptr (one group of M rows)
    int groups;
    int tiles_w;        // row tiles of W per group
    int w_blocks;       // 128-row scale tiles of W per group (MXFP4)
    int k_steps;        // MMAs along K
    const float* row_scale;    // [M] or nullptr
    const uint16_t* bias;      // [groups x N] or nullptr
    const uint16_t* residual;  // [M x N] or nullptr
    int64_t ldr;
    uint16_t* Y;
    int64_t ldy;
    uint32_t* dev_error;
    // The call's own quantising launch comes in front: offsets and weights are older than that and may be read before the
    // wait for it.
    int weights_ready;
    // The work list where there are no offsets: token tiles, their width, the items that are not cut and all items, pieces of each of the
    // others.  (With offsets only the device knows.)
    int n_t, w_tile, n_whole, items, cuts;
    int trigger;  // the next launch may begin when a CTA's last MMAs are done (see launch_grouped_cfg)
    int cluster;  // CTAs of a cluster over which K may be split (single CTAs' tiles)
    // few tokens: X in bf16, quantised by every CTA
    const uint16_t* X;
    int64_t ldx;
    int stages;
};

// MX: MXFP4 operands, else bf16.  CG: CTAs per MMA, with 128 rows of W each.  NT: tokens per tile.
// XRES: the layer of few tokens.  X (bf16, at most XRES_ROWS rows) is quantised by the epilogue warps of every CTA into shared
// memory, where it stays; the ring holds weights only, in as many stages as the rest of the memory takes.
template <bool MX_, int CG_, int NT_, int STAGES_, bool XRES_ = false>
struct GroupedCfg {
    static constexpr bool MX = MX_, XRES = XRES_;
    static constexpr int CG = CG_, NT = NT_, STAGES = STAGES_;
    static constexpr int W_ROWS = 128 * CG;         // of a tile
    static constexpr int BOX_X = MX ? 128 : 64;     // elements of the tensor map (bytes, bf16) in a stage's 128 bytes of K
    static constexpr int STEP_K = MX ? 64 : 16;     // elements per MMA: four per stage
    static constexpr int N_STEP = CG == 2 ? 32 : 16;  // tokens per MMA come in multiples of this
    static constexpr int NT_CTA = NT / CG;
    static constexpr int BOX = 32, BOX_BYTES = BOX * 128;  // rows of the small boxes, of W and X
    static constexpr int A_BYTES = 128 * 128, B_BYTES = XRES ? 0 : NT_CTA * 128;
    static constexpr int NB = (NT + 127) / 128;     // scale tiles of the tokens
    static constexpr int CHUNKS = MX ? 2 : 0;       // scale tiles along K per stage
    static constexpr int SA_BYTES = CHUNKS * MX_CHUNK_BYTES, SB_BYTES = XRES ? 0 : NB * SA_BYTES;
    static constexpr int STAGE_BYTES = A_BYTES + B_BYTES + SA_BYTES + SB_BYTES;
    // Tensor memory: two accumulators, then every stage's scales.  256-wide MXFP4 tiles leave no room for two whole accumulators
    // beside them: they share OVERLAP columns, which the epilogue reads first and hands back.  (Scales of two stages only, and
    // 64 shared columns: the issuer then waits for the MMAs of the stage before the last, 256 x 10240 x 3840 16.1 us against 13.6.)
    static constexpr int S_COLS = CHUNKS * 4 * (1 + NB);
    static constexpr int ACC1 = (MX && NT == 256) ? 128 : NT;  // first column of the second accumulator
    static constexpr int OVERLAP = NT - ACC1;
    static constexpr int LAG = OVERLAP ? 1 : 2;  // an item may start when the one LAG before it has been handed back
    static constexpr int S_COL0 = ACC1 + NT;
    static constexpr int COLS_USED = S_COL0 + STAGES * S_COLS;
    static constexpr int TMEM_COLS = COLS_USED <= 128 ? 128 : COLS_USED <= 256 ? 256 : 512;
    // What does not fill a round of all clusters is cut (see GroupSchedule): pairs' tiles along the tokens, not below the 64
    // with which a tile's scales can begin in tensor memory; single CTAs' tiles of few tokens along K, over the CTAs of a cluster
    // of p.cluster, whose accumulators are added through shared memory.  (Sent with st.async and a barrier per receiving warp; behind
    // a cluster barrier with release instead, which took 2500 cycles: 1 x 10240 x 3840 8.0 us against 6.7.)
    static constexpr bool CUT_K = CG == 1;
    static constexpr int MAX_CUTS = 4;
    static constexpr int UNIT_BYTES = 32 * 32 * 4;  // one epilogue warp's 32 x 32 accumulators
    static constexpr int INBOX_BYTES = CUT_K ? 3 * (XRES ? 1 : 2) * UNIT_BYTES : 0;
    static constexpr int EPI_WARPS = GEMM_EPI_WARPS;
    static constexpr int ROUNDS = NT / 64;  // chunks of 32 tokens per epilogue warp
    static constexpr int PITCH = 80;        // bytes per staged token: 64 + 16, conflict-free for 16-byte rows
    static constexpr int STAGING_BYTES = 32 * PITCH;
    static constexpr int SCHED_BYTES = XRES ? 0 : 3 * (GG_MAX_GROUPS + 1) * 4;
    static constexpr int NUM_BARS = 2 * STAGES + 2 + LAG + 1 + (CUT_K ? EPI_WARPS : 0);
    // [B ring][A ring][scales][staging][work list][barriers, tensor-memory address, abort word]
    static constexpr int OFF_A = STAGES * B_BYTES, OFF_SA = OFF_A + STAGES * A_BYTES, OFF_SB = OFF_SA + STAGES * SA_BYTES;
    static constexpr int OFF_BOX = OFF_SB + STAGES * SB_BYTES, OFF_INBOX = OFF_BOX + EPI_WARPS * STAGING_BYTES;
    static constexpr int OFF_SCHED = OFF_INBOX + INBOX_BYTES;
    static constexpr int OFF_BAR = (OFF_SCHED + SCHED_BYTES + 7) / 8 * 8;
    // XRES: the resident X takes the place of the last stages (STAGES is what fits beside none; a slice of 256 k: 16 rows of codes
    // and two scale tiles of which the first 256 bytes are used, so that the next one may follow there)
    static constexpr int X_CODES = XRES_ROWS * 128, X_SCALES = 512, X_SLICE = X_CODES + X_SCALES;
    static constexpr int SMEM_BYTES = 1024 + OFF_BAR + 8 * NUM_BARS + 16;
    static __host__ __device__ int stages_beside(int slices) {
        const int left = OFF_BOX - slices * X_SLICE - 256;  // (256: the last scale tile's unused half)
        return left < 0 ? 0 : left / STAGE_BYTES < STAGES ? left / STAGE_BYTES : STAGES;
    }
    static constexpr int THREADS = GEMM_THREADS;
    static_assert(NT == 64 || NT == 128 || NT == 256, "tokens per tile: from a multiple of 64, within a scale tile or whole ones");
    static_assert(OVERLAP % 64 == 0, "an epilogue warp hands back after whole chunks");
    static_assert(COLS_USED <= 512 && SMEM_BYTES <= 227 * 1024, "budgets");
    static_assert(B_BYTES % 1024 == 0, "swizzle atoms");
    static_assert(!XRES || (MX && CG == 1 && NT >= XRES_ROWS && XRES_ROWS <= 32), "few tokens on single CTAs");
    static_assert(!CUT_K || (NT == 64 && LAG == 2), "one chunk of tokens per epilogue warp: it keeps or sends it");
};

// Instruction descriptors.  kind::f16: fp32 results, bf16 operands.  kind::mxf4: E2M1 operands, E8M0 scales; `id` (0 or 2): which
// two of the four scale bytes this K = 64 takes.
__device__ __forceinline__ uint32_t gg_idesc_bf16(int m, int n) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ uint32_t gg_idesc_mxf4(int m, int n, uint32_t id) {
    return (id << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | ((uint32_t)(m >> 7) << 27) | (id << 29);
}

// The work list.  Offsets are clamped to [0, M] and made non-decreasing, so that no list of offsets leads outside the operands.
// A group's rows are cut into as few token tiles of nt as they take, all of one width (a multiple of 64, the last may be shorter).
// Items are dealt round-robin to the clusters, the groups in the order of their tiles' width, widest first (ragged groups then end
// within a narrow tile of one another); within a group the token tiles run fastest, 16 of them at a time, so that its weights are read
// while they are in the L2.
// What does not fill a round of all clusters is cut into two or four, as far as clusters are free: 4096 x 10240 x 3840 in 256 x 256
// tiles is 3.24 rounds of 74 CTA pairs, and its last 18 tiles run as 72 of 64 tokens; 1 x 10240 x 3840 is 30 tiles of 128 rows of
// W, each of which runs on a cluster of four CTAs, a quarter of K on each.
// (Integer divisions are what an item's coordinates cost, and a launch's first loads wait for them: see gg_div.)
__host__ __device__ inline int gg_div(int a, int b) {
#ifdef __CUDA_ARCH__
    if (b == 1) return a;
    if (((a | b) >> 21) == 0) {
        // both exact in fp32: the quotient is off by one at most
        const int q = (int)__fdividef((float)a, (float)b), r = a - q * b;
        return q + (r >= b) - (r < 0);
    }
#endif
    return a / b;
}

struct GroupSchedule {
    // without offsets these lists are not used: the host has worked the list out (a launch's first loads wait for what is done here)
    const int* start;  // [groups + 1] first rows
    const int* order;  // [groups] the groups in the order of the list
    const int* base;   // [groups + 1] token tiles before a place of the list
    int groups, tiles_w;
    int n_whole, cuts;  // items that are not cut; pieces of each of the others

    template <int NT>
    __host__ __device__ static int width(int rows) {
        if (NT == 64 || rows <= 0) return NT;
        const int n = (rows + NT - 1) / NT;
        return (gg_div(rows + n - 1, n) + 63) / 64 * 64;
    }
    template <int NT>
    __host__ __device__ static int tiles(int rows, int w) {
        return NT == 64 ? (rows + NT - 1) / NT : gg_div(rows + w - 1, w);
    }

    // Fills the three lists; by one warp, the caller synchronises.
    template <int NT>
    __device__ static void build(const GroupedParams& p, int* start, int* order, int* base, int lane) {
        const int G = p.groups;
        const int per = (G + 1 + 31) / 32, i0 = lane * per, i1 = i0 + per < G + 1 ? i0 + per : G + 1;
        int most = 0;
        for (int i = i0; i < i1; ++i) {
            // (out of the L2: a layer's product reads them before its own wait, where an older line may still be in the L1)
            const int v = (int)mx_clamp_row(__ldcg(p.offsets + i), p.M);
            most = v > most ? v : most;
            start[i] = most;
        }
        int before = most;  // the largest of the lanes up to this one
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int v = __shfl_up_sync(0xffffffffu, before, d);
            if (lane >= d && v > before) before = v;
        }
        before = __shfl_up_sync(0xffffffffu, before, 1);
        if (lane == 0) before = 0;
        for (int i = i0; i < i1; ++i)
            if (start[i] < before) start[i] = before;
        __syncwarp();
        if constexpr (NT == 64) {  // one width: the groups as they come
            int n = 0;
            for (int i = i0; i < i1 && i < G; ++i) n += tiles<NT>(start[i + 1] - start[i], NT);
            int upto = n;  // tiles of the lanes up to this one
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const int v = __shfl_up_sync(0xffffffffu, upto, d);
                if (lane >= d) upto += v;
            }
            int first = upto - n;
            for (int i = i0; i < i1; ++i) {
                base[i] = first;
                if (i == G) break;
                order[i] = i;
                first += tiles<NT>(start[i + 1] - start[i], NT);
            }
            return;
        }
        // a counting sort by width: four classes (a multiple of 64 up to 256), each with its groups and tiles
        int n_groups[4] = {0, 0, 0, 0}, n_tiles[4] = {0, 0, 0, 0};
        auto each = [&](auto f) {
            for (int i = i0; i < i1 && i < G; ++i) {
                const int rows = start[i + 1] - start[i], w = width<NT>(rows), c = (256 - w) / 64;
#pragma unroll
                for (int x = 0; x < 4; ++x)  // (an index known at compile time keeps the counters in registers)
                    if (c == x) f(i, x, tiles<NT>(rows, w));
            }
        };
        each([&](int, int c, int tiles) {
            ++n_groups[c];
            n_tiles[c] += tiles;
        });
        int all_groups = 0, all_tiles = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            int sg = n_groups[c], st = n_tiles[c];
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const int a = __shfl_up_sync(0xffffffffu, sg, d), b = __shfl_up_sync(0xffffffffu, st, d);
                if (lane >= d) {
                    sg += a;
                    st += b;
                }
            }
            n_groups[c] = all_groups + sg - n_groups[c];  // the first of this lane's
            n_tiles[c] = all_tiles + st - n_tiles[c];
            all_groups += __shfl_sync(0xffffffffu, sg, 31);
            all_tiles += __shfl_sync(0xffffffffu, st, 31);
        }
        each([&](int i, int c, int tiles) {
            order[n_groups[c]] = i;
            base[n_groups[c]++] = n_tiles[c];
            n_tiles[c] += tiles;
        });
        if (lane == 0) base[G] = all_tiles;
    }
    // How n items are cut for `clusters` of them, into max_cuts pieces at most.
    __host__ __device__ static void cut(int n, int clusters, int max_cuts, int& n_whole, int& cuts, int& items) {
        const int rest = n - gg_div(n, clusters) * clusters;
        n_whole = n - rest;
        cuts = 1;
        while (rest * cuts * 2 <= clusters && cuts * 2 <= max_cuts) cuts *= 2;
        items = n_whole + rest * cuts;
    }
    int items;
    int n_t, w_tile, M;  // without offsets
    bool dense;
    __device__ GroupSchedule(const GroupedParams& p, const int* start_, const int* order_, const int* base_, int clusters, int max_cuts)
        : start(start_), order(order_), base(base_), groups(p.groups), tiles_w(p.tiles_w), n_whole(p.n_whole), cuts(p.cuts), items(p.items),
          n_t(p.n_t), w_tile(p.w_tile), M((int)p.M), dense(p.offsets == nullptr) {
        if (!dense) cut(base[groups] * tiles_w, clusters, max_cuts, n_whole, cuts, items);
    }

    struct Item {
        int group, row0, rows;  // tokens (rows <= 0: a piece that has none)
        int in_group;           // the first one within its group
        int w0;                 // the tile's first row of W within the group's
        int parts, piece;       // cut along K: how often, and which of the pieces
        __device__ int k0(int stages_k) const { return stages_k * piece / parts; }
        __device__ int k1(int stages_k) const { return stages_k * (piece + 1) / parts; }
    };
    // `at`: the place of an earlier item's group in the list, moved on.  Called by whole warps.
    template <class Cfg>
    __device__ Item get(int item, int lane, int& at) const {
        int piece = 0, parts = 1;
        if (item >= n_whole) {
            const int u = item - n_whole;
            parts = cuts;
            const int shift = parts >> 1;  // 1, 2 or 4 pieces
            item = n_whole + (u >> shift);
            piece = u & (parts - 1);
        }
        Item it;
        int first = 0, rows = M, w_t = w_tile, n = n_t, w = item, t = 0;  // w: the item's place in its group
        it.group = 0;
        if (!dense) {
            const int tile = gg_div(item, tiles_w);
            for (;;) {
                const int i = at + 1 + lane;
                const int c = __popc(__ballot_sync(0xffffffffu, i <= groups && base[i] <= tile));
                at += c;
                if (c < 32) break;
            }
            it.group = order[at];
            first = start[it.group];
            rows = start[it.group + 1] - first;
            w_t = width<Cfg::NT>(rows);
            n = base[at + 1] - base[at];
            w = item - base[at] * tiles_w;
        }
        if (n > GG_GROUP_TILES) {
            const int block = gg_div(w, GG_GROUP_TILES * tiles_w);
            w -= block * GG_GROUP_TILES * tiles_w;
            t = block * GG_GROUP_TILES;
            n = n - t < GG_GROUP_TILES ? n - t : GG_GROUP_TILES;
        }
        const int q = gg_div(w, n);
        t += w - q * n;
        w = q;
        it.parts = Cfg::CUT_K ? parts : 1;
        it.piece = Cfg::CUT_K ? piece : 0;
        const int w_piece = Cfg::CUT_K ? w_t : ((w_t >> (parts >> 1)) + 63) / 64 * 64, off = Cfg::CUT_K ? 0 : piece * w_piece;
        it.in_group = t * w_t + off;
        it.row0 = first + it.in_group;
        int left = rows - it.in_group;
        if (left > w_t - off) left = w_t - off;
        it.rows = left < w_piece ? left : w_piece;
        it.w0 = w * Cfg::W_ROWS;
        return it;
    }
};

// X of at most XRES_ROWS rows into shared memory as the MMA reads it: slices of 256 k (rows of 128 bytes, 128-byte swizzle), and
// their scales (two tiles per slice, the rows' 16 bytes each).  Rows behind the last are left as they are: what they are multiplied to
// is never read.  A warp takes 1024 elements of one row at a time, two of them in flight.
__device__ __forceinline__ void quantize_resident(const GroupedParams& p, uint32_t codes, uint32_t scales, int slice_codes, int slice_scales,
                                                  int warp, int warps, int lane) {
    const int spans = (int)((p.K + MX_WARP_K - 1) / MX_WARP_K), units = (int)p.M * spans;
    for (int u0 = warp; u0 < units; u0 += 2 * warps) {
        uint32_t x[2][16];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int u = u0 + i * warps, row = u / spans, k = (u - row * spans) * MX_WARP_K + 32 * lane;
            if (u < units && k < p.K) {
                const uint16_t* src = p.X + row * p.ldx + k;
                ldg256_keep(src, *reinterpret_cast<uint32_t(*)[8]>(&x[i][0]));
                ldg256_keep(src + 16, *reinterpret_cast<uint32_t(*)[8]>(&x[i][8]));
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int u = u0 + i * warps, row = u / spans, block = (u - row * spans) * (MX_WARP_K / 32) + lane;
            if (u >= units) break;
            uint32_t c[4] = {0, 0, 0, 0}, s = MX_ONE;  // behind K: zeros times 1
            if (32 * block < p.K) s = mx_quantize_block(x[i], c);
            s <<= 8 * (lane & 3);
            s |= __shfl_xor_sync(0xffffffffu, s, 1);
            s |= __shfl_xor_sync(0xffffffffu, s, 2);
            if (32 * (block & ~3) < p.K) {  // the slice's 128 k have a part of the row
                sts128(codes + (block >> 3) * slice_codes + row * 128 + (((block & 7) ^ (row & 7)) << 4), c[0], c[1], c[2], c[3]);
                if ((lane & 3) == 0) sts32(scales + (block >> 3) * slice_scales + ((block >> 2) & 1) * (slice_scales / 2) + row * 16, s);
            }
        }
    }
}

template <class Cfg>
__global__ void __launch_bounds__(Cfg::THREADS, 1)
grouped_gemm_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_x,
                    const __grid_constant__ CUtensorMap tmap_xall, const __grid_constant__ CUtensorMap tmap_sw,
                    const __grid_constant__ CUtensorMap tmap_sx, const GroupedParams p) {
    constexpr int CG = Cfg::CG;
    const int STAGES = Cfg::XRES ? p.stages : Cfg::STAGES;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
    const uint32_t sB = smem_base, sA = smem_base + Cfg::OFF_A;
    const uint32_t sSA = Cfg::XRES ? smem_base + STAGES * Cfg::A_BYTES : smem_base + Cfg::OFF_SA, sSB = smem_base + Cfg::OFF_SB;
    const uint32_t sXR = sSA + STAGES * Cfg::SA_BYTES;  // resident X: the slices' codes, then their scales (1024-byte aligned)
    const uint32_t bar_full = smem_base + Cfg::OFF_BAR, bar_empty = bar_full + 8 * Cfg::STAGES;
    const uint32_t bar_tfull = bar_empty + 8 * Cfg::STAGES, bar_tempty = bar_tfull + 16, bar_x = bar_tempty + 8 * Cfg::LAG, bar_in = bar_x + 8;
    int* sched_start = reinterpret_cast<int*>(smem_gen + Cfg::OFF_SCHED);
    int* sched_order = sched_start + GG_MAX_GROUPS + 1;
    int* sched_base = sched_order + GG_MAX_GROUPS + 1;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem_gen + Cfg::OFF_BAR + 8 * Cfg::NUM_BARS);
    volatile uint32_t* cta_abort = tmem_slot + 1;

    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const uint32_t rank = (CG == 2) ? cluster_ctarank() : 0u;
    const bool leader = rank == 0;
    const int cluster_id = blockIdx.x / CG, num_clusters = gridDim.x / CG;

    if (threadIdx.x == 0) {
        *cta_abort = 0;
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(bar_full + 8 * s, Cfg::XRES ? 1 : 2);  // the loading warps of the leader announce what they load
            mbar_init(bar_empty + 8 * s, 1);  // one tcgen05.commit
        }
        for (int a = 0; a < 2; ++a) mbar_init(bar_tfull + 8 * a, 1);
        for (int a = 0; a < Cfg::LAG; ++a) mbar_init(bar_tempty + 8 * a, Cfg::EPI_WARPS * CG);
        mbar_init(bar_x, Cfg::EPI_WARPS);
        if constexpr (Cfg::CUT_K)
            for (int w = 0; w < Cfg::EPI_WARPS; ++w) mbar_init(bar_in + 8 * w, 1);  // an epilogue warp's own announcement of what it gets
        fence_mbar_init();
        prefetch_tmap(&tmap_w);
        prefetch_tmap(&tmap_xall);
        if constexpr (Cfg::MX) {
            prefetch_tmap(&tmap_sw);
            prefetch_tmap(&tmap_sx);
        }
    }
    if (warp == 1) {
        tmem_alloc<CG>(smem_u32(tmem_slot), Cfg::TMEM_COLS);
        tmem_relinquish<CG>();
    }
    if (warp == 2 && p.offsets != nullptr) {
        // (Only this warp waits for the launch in front before the others have set the CTA up; with its one-width list: 359 rows on 89
        // bf16 experts 96 x 344 6.4 -> 5.8 us, 45 on 3 of 1536 x 2048 7.9 -> 7.5, 64 rows on 36 MXFP4 experts 32.4 -> 32.2.)
        if (!p.weights_ready) griddep_wait();
        GroupSchedule::build<Cfg::NT>(p, sched_start, sched_order, sched_base, lane);
    }
    tc_fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync_relaxed();
    else if (p.cluster > 1) cluster_arrive_relaxed();  // (who sends to another CTA waits for it first)
    tc_fence_after();
    const uint32_t tmem_base = __shfl_sync(0xffffffffu, *tmem_slot, 0);
    const int stages_k = (p.k_steps + 3) / 4;
    const GroupSchedule sched(p, sched_start, sched_order, sched_base, num_clusters,
                              Cfg::CUT_K ? (p.cluster < stages_k ? p.cluster : stages_k) : Cfg::MAX_CUTS);
    const int num_items = sched.items;
    if (!p.weights_ready) griddep_wait();

    if (warp == 0 || (warp == 3 && !Cfg::XRES)) {
        // ------------------------------------------------------------------ producers ---------
        const bool is_w = warp == 0;
        // weights are there already; X comes from the launch in front
        if (!is_w) griddep_wait();
        const uint32_t full0 = (CG == 2) ? mapa(bar_full, 0) : bar_full;  // the leader's barriers
        auto load = [&](uint32_t dst, const CUtensorMap* m, int x, int y, uint32_t s) {
            if constexpr (CG == 1) tma_load_2d(dst, m, x, y, bar_full + 8 * s);
            else tma_load_2d_pair(dst, m, x, y, full0 + 8 * s);
        };
        auto load3 = [&](uint32_t dst, const CUtensorMap* m, int x, int y, int z, uint32_t s) {
            if constexpr (CG == 1) tma_load_3d(dst, m, x, y, z, bar_full + 8 * s);
            else tma_load_3d_pair(dst, m, x, y, z, full0 + 8 * s);
        };
        uint32_t stage = 0, phase = 0;
        bool ok = true;
        int at = 0;
        for (int item = cluster_id; item < num_items && ok; item += num_clusters) {
            const auto it = sched.template get<Cfg>(item, lane, at);
            if (it.rows <= 0) continue;
            const int n_cta = (it.rows + Cfg::N_STEP - 1) / Cfg::N_STEP * Cfg::N_STEP / CG;  // tokens of this CTA
            // one box of the tile's rows, or boxes of 32 where it has no more than half of them
            const int all = (is_w ? 128 : Cfg::NT_CTA) / Cfg::BOX, boxes = is_w ? all : (n_cta + Cfg::BOX - 1) / Cfg::BOX;
            const bool one_box = 2 * boxes > all;
            const uint32_t bytes = (one_box ? all : boxes) * Cfg::BOX_BYTES + (is_w ? Cfg::SA_BYTES : Cfg::SB_BYTES);
            const int w = it.w0 + (int)rank * 128;
            const int row = is_w ? it.group * (int)p.N + w : it.row0 + (int)rank * n_cta;
            const int block = is_w ? it.group * p.w_blocks + w / 128
                                   : (p.offsets ? (it.row0 - it.in_group) / 128 + it.group : 0) + it.in_group / 128;
            const CUtensorMap *rows_map = is_w ? &tmap_w : (one_box ? &tmap_xall : &tmap_x),
                              *scale_map = is_w ? &tmap_sw : &tmap_sx;
            const uint32_t dst0 = is_w ? sA : sB, dst_step = is_w ? Cfg::A_BYTES : Cfg::B_BYTES;
            for (int ks = it.k0(stages_k), k1 = it.k1(stages_k); ks < k1; ++ks) {
                ok = mbar_wait_warp(bar_empty + 8 * stage, phase ^ 1, cta_abort, p.dev_error);
                if (!ok) break;
                if (elect_one()) {
                    if (leader) mbar_arrive_expect_tx(bar_full + 8 * stage, bytes * CG);
                    const uint32_t dst = dst0 + stage * dst_step;
                    load(dst, rows_map, ks * Cfg::BOX_X, row, stage);
                    if (!one_box)
                        for (int b = 1; b < boxes; ++b) load(dst + b * Cfg::BOX_BYTES, rows_map, ks * Cfg::BOX_X, row + b * Cfg::BOX, stage);
                    if constexpr (Cfg::MX)
                        load3(is_w ? sSA + stage * Cfg::SA_BYTES : sSB + stage * Cfg::SB_BYTES, scale_map, 0, ks * Cfg::CHUNKS, block, stage);
                }
                if (++stage == STAGES) { stage = 0; phase ^= 1; }
            }
        }
        for (int s = 0; s < STAGES && ok; ++s) {  // the last releases of the stages (see epilogue.cuh)
            ok = mbar_wait_warp(bar_empty + 8 * stage, phase ^ 1, cta_abort, p.dev_error);
            if (++stage == STAGES) { stage = 0; phase ^= 1; }
        }
        if (!ok) bounded_delay_ns(200000);  // let the copies in flight land before teardown
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer --------
        if (leader) {
            const uint64_t d0 = make_desc_sw128(sA);
            const uint32_t desc_hi = (uint32_t)(d0 >> 32), a_lo0 = (uint32_t)d0, b_lo0 = (uint32_t)make_desc_sw128(sB);
            const uint64_t sa_d0 = make_desc_rows16(sSA), sb_d0 = make_desc_rows16(sSB);
            const uint32_t x_lo0 = (uint32_t)make_desc_sw128(sXR);
            const uint64_t sx_d0 = make_desc_rows16(sXR + stages_k * Cfg::X_CODES);
            uint32_t stage = 0, phase = 0;
            bool ok = true;
            int i = 0;
            int at = 0;
            for (int item = cluster_id; item < num_items && ok; item += num_clusters) {
                const auto it = sched.template get<Cfg>(item, lane, at);
                if (it.rows <= 0) continue;
                const int n = (it.rows + Cfg::N_STEP - 1) / Cfg::N_STEP * Cfg::N_STEP;
                const CyclicTurn<Cfg::LAG> turn(i);
                ok = mbar_wait_warp(bar_tempty + 8 * turn.buffer, turn.fill(), cta_abort, p.dev_error);
                if (!ok) break;
                if (Cfg::XRES && i == 0) {
                    ok = mbar_wait_warp(bar_x, 0, cta_abort, p.dev_error);
                    if (!ok) break;
                }
                tc_fence_after();
                const uint32_t d_tmem = tmem_base + (i & 1) * Cfg::ACC1;
                const uint32_t idesc0 = Cfg::MX ? gg_idesc_mxf4(128 * CG, n, 0) : gg_idesc_bf16(128 * CG, n);
                const uint32_t idesc1 = Cfg::MX ? gg_idesc_mxf4(128 * CG, n, 2) : idesc0;
                const bool two_blocks = Cfg::NB == 2 && (it.in_group & 64) + it.rows > 128;
                // the tile's place in its scale tile, in columns: 0 or 2 (the MMA takes scales from even columns only)
                const uint32_t sx_shift = (uint32_t)(it.in_group & 64) / 32;
                uint32_t accumulate = 0;
                for (int ks = it.k0(stages_k), k1 = it.k1(stages_k); ks < k1; ++ks) {
                    ok = mbar_wait_warp(bar_full + 8 * stage, phase, cta_abort, p.dev_error);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t a_lo = a_lo0 + stage * (Cfg::A_BYTES >> 4);
                    const uint32_t b_lo = Cfg::XRES ? x_lo0 + ks * (Cfg::X_CODES >> 4) : b_lo0 + stage * (Cfg::B_BYTES >> 4);
                    const uint32_t s_tmem = tmem_base + Cfg::S_COL0 + stage * Cfg::S_COLS;
                    const int left = p.k_steps - ks * 4;  // MMAs that are left, this stage's included
                    if (elect_one()) {
                        if constexpr (Cfg::MX) {
#pragma unroll
                            for (int c = 0; c < Cfg::CHUNKS; ++c) {
                                tmem_cp_scales<CG>(s_tmem + c * 4, sa_d0 + (uint64_t)((stage * Cfg::SA_BYTES + c * MX_CHUNK_BYTES) >> 4));
                                const uint32_t t = s_tmem + Cfg::CHUNKS * 4 + c * 4 * Cfg::NB;
                                const uint64_t sb = Cfg::XRES ? sx_d0 + (uint64_t)((ks * Cfg::X_SCALES + c * (Cfg::X_SCALES / 2)) >> 4)
                                                              : sb_d0 + (uint64_t)((stage * Cfg::SB_BYTES + c * MX_CHUNK_BYTES) >> 4);
                                tmem_cp_scales<CG>(t, sb);
                                if (two_blocks) tmem_cp_scales<CG>(t + 4, sb + (uint64_t)(Cfg::SA_BYTES >> 4));
                            }
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if (j < left) {
                                const uint32_t a = a_lo + 2 * j, b = b_lo + 2 * j;
                                if constexpr (Cfg::MX)
                                    mma_mxf4_lh<CG>(d_tmem, a, b, desc_hi, (j & 1) ? idesc1 : idesc0, s_tmem + (j / 2) * 4,
                                                    s_tmem + Cfg::CHUNKS * 4 + (j / 2) * 4 * Cfg::NB + sx_shift, j ? 1u : accumulate);
                                else
                                    mma_bf16_lh<CG>(d_tmem, a, b, desc_hi, idesc0, j ? 1u : accumulate);
                            }
                        }
                        if constexpr (CG == 1) tc_commit(bar_empty + 8 * stage);
                        else tc_commit_pair(bar_empty + 8 * stage, 0x3);
                    }
                    accumulate = 1u;
                    if (++stage == STAGES) { stage = 0; phase ^= 1; }
                }
                if (!ok) break;
                if (elect_one()) {
                    if constexpr (CG == 1) tc_commit(bar_tfull + 8 * (i & 1));
                    else tc_commit_pair(bar_tfull + 8 * (i & 1), 0x3);
                }
                ++i;
            }
            for (int a = 0; a < Cfg::LAG && ok; ++a) {  // the last hand-backs (see epilogue.cuh)
                const CyclicTurn<Cfg::LAG> turn(i + a);
                ok = mbar_wait_warp(bar_tempty + 8 * turn.buffer, turn.fill(), cta_abort, p.dev_error);
            }
        }
    }
    // ---------------------------------------------------------------------- epilogue ----------
    const int q = warp & 3;                      // tensor-memory lane quarter this warp may read
    const int h = (warp - GEMM_EPI_WARP0) >> 2;  // which of the quarter's two warps
    const uint32_t box = smem_base + Cfg::OFF_BOX + (warp - GEMM_EPI_WARP0) * Cfg::STAGING_BYTES;
    const uint32_t inbox = smem_base + Cfg::OFF_INBOX;
    // What a warp needs of an item's chunk of 32 tokens beside the accumulators.
    struct Chunk {
        typename GroupSchedule::Item it;
        int n0;        // first column of Y
        int c;         // the chunk; none of the warp's if c >= chunks
        int chunks;
        float bias[4];  // of rows lane / 4 + 8 j of the quarter
        float s[8];     // factors of tokens 8 j + 2 (lane % 4), + 1
        uint4 res[4];   // the lane's 16 bytes of tokens 8 j + lane / 4
    };
    auto fetch = [&](Chunk& k, int c) {
        k.c = c;
        if (p.residual != nullptr) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int t = c * 32 + 8 * j + (lane >> 2), n = k.n0 + 8 * (lane & 3);
                k.res[j] = make_uint4(0, 0, 0, 0);
                if (c < k.chunks && t < k.it.rows && n < p.N)
                    k.res[j] = *reinterpret_cast<const uint4*>(p.residual + (int64_t)(k.it.row0 + t) * p.ldr + n);
            }
        }
        if (p.row_scale != nullptr) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int t = c * 32 + 8 * (j >> 1) + 2 * (lane & 3) + (j & 1);
                k.s[j] = (c < k.chunks && t < k.it.rows) ? p.row_scale[k.it.row0 + t] : 0.0f;
            }
        }
    };
    auto finish = [&](const Chunk& k, const uint32_t (&v)[2][16]) {
        // packed pairs of tokens of one row of W; o[4 * g + j]: tokens 8 g + 2 (lane % 4), + 1 of row 8 j + lane / 4
        uint32_t o[16];
        if (p.residual != nullptr) {
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 4; ++j)
                sts128(box + (8 * j + (lane >> 2)) * Cfg::PITCH + (lane & 3) * 16, k.res[j].x, k.res[j].y, k.res[j].z, k.res[j].w);
            __syncwarp();
#pragma unroll
            for (int g = 0; g < 4; ++g)
                ldmatrix_x4_trans(box + (8 * g + (lane & 7)) * Cfg::PITCH + (lane >> 3) * 16, o[4 * g], o[4 * g + 1], o[4 * g + 2], o[4 * g + 3]);
        }
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t* a = &v[j >> 1][4 * g + 2 * (j & 1)];
                uint64_t y = fma_f32x2(pack_f32x2(k.s[2 * g], k.s[2 * g + 1]), pack_b32x2(a[0], a[1]), pack_f32x2(k.bias[j], k.bias[j]));
                if (p.residual != nullptr) y = add_f32x2(y, pack_f32x2(bf16_lo_f(o[4 * g + j]), bf16_hi_f(o[4 * g + j])));
                o[4 * g + j] = pack_bf16x2_of(y);
            }
        __syncwarp();  // the box is free: every lane has read what it held
#pragma unroll
        for (int g = 0; g < 4; ++g)
            stmatrix_x4_trans(box + (8 * g + (lane & 7)) * Cfg::PITCH + (lane >> 3) * 16, o[4 * g], o[4 * g + 1], o[4 * g + 2], o[4 * g + 3]);
        __syncwarp();
        const int n = k.n0 + 8 * (lane & 3);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int t = 8 * j + (lane >> 2);
            uint32_t w[4];
            lds128(box + t * Cfg::PITCH + (lane & 3) * 16, w[0], w[1], w[2], w[3]);
            if (k.c * 32 + t < k.it.rows && n < p.N) stg128(p.Y + (int64_t)(k.it.row0 + k.c * 32 + t) * p.ldy + n, w[0], w[1], w[2], w[3]);
        }
    };
    Chunk k;
    uint32_t v[2][16];
    bool alive = true;
    if (warp >= GEMM_EPI_WARP0) {
        if (p.weights_ready) griddep_wait();
        const uint32_t tempty0 = (CG == 2) ? mapa(bar_tempty, 0) : bar_tempty;
        if constexpr (Cfg::XRES) {
            quantize_resident(p, sXR, sXR + stages_k * Cfg::X_CODES, Cfg::X_CODES, Cfg::X_SCALES, warp - GEMM_EPI_WARP0, Cfg::EPI_WARPS, lane);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_x);
        }
        if (Cfg::CUT_K && p.cluster > 1) cluster_wait();  // the others' barriers are initialised
        int i = -1;
        int at = 0;
        for (int item = cluster_id; item < num_items; item += num_clusters) {
            k.it = sched.template get<Cfg>(item, lane, at);
            if (k.it.rows <= 0) continue;
            const int buf = ++i & 1;
            const uint32_t hand_back = tempty0 + 8 * CyclicTurn<Cfg::LAG>(i).buffer;
            k.n0 = k.it.w0 + (int)rank * 128 + 32 * q;
            k.chunks = k.n0 < p.N ? (k.it.rows + 31) / 32 : 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int n = k.n0 + 8 * j + (lane >> 2);
                k.bias[j] = (p.bias != nullptr && n < p.N) ? __uint_as_float((uint32_t)p.bias[(int64_t)k.it.group * p.N + n] << 16) : 0.0f;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) k.s[j] = 1.0f;
            // the chunk that this warp takes in round r: with shared columns those first
            auto chunk_of = [&](int r) {
                if constexpr (Cfg::OVERLAP != 0) return buf ? 2 * r + h : Cfg::NT / 32 - 2 - 2 * r + h;
                else return 2 * r + h;
            };
            fetch(k, chunk_of(0));
            alive = mbar_wait_warp(bar_tfull + 8 * buf, CyclicTurn<2>(i).drain(), cta_abort, p.dev_error);
            if (!alive) break;
            tc_fence_after();
            if (p.trigger && item + num_clusters >= num_items) griddep_launch_dependents();
            const uint32_t acc = tmem_base + ((uint32_t)(q * 32) << 16) + buf * Cfg::ACC1;
            auto read = [&](int c, uint32_t (&x)[2][16]) {
                if (c < k.chunks) {
                    tmem_ld_16x256b_x4(acc + c * 32, x[0]);
                    tmem_ld_16x256b_x4(acc + (16u << 16) + c * 32, x[1]);
                }
            };
            auto give_back = [&] {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if constexpr (CG == 1) mbar_arrive(hand_back);
                    else mbar_arrive_cluster(hand_back);
                }
            };
            if constexpr (Cfg::ROUNDS > 1) {
                // Two chunks at a time, with shared columns those first: the next item's MMAs wait until they are read, not until
                // results are made of them.  One copy of the code that does that: a launch's first epilogue fetches its instructions.
                static_assert(Cfg::ROUNDS % 2 == 0 && (Cfg::OVERLAP == 0 || Cfg::OVERLAP == 128), "two chunks are what is shared");
#pragma unroll 1
                for (int r = 0; r < Cfg::ROUNDS; r += 2) {
                    uint32_t v1[2][16];
                    read(chunk_of(r), v);
                    read(chunk_of(r + 1), v1);
                    tmem_ld_wait();
                    if (r == (Cfg::OVERLAP ? 0 : Cfg::ROUNDS - 2)) give_back();
#pragma unroll 1
                    for (int x = 0; x < 2; ++x) {
                        if (r + x > 0) fetch(k, chunk_of(r + x));
                        if (k.c < k.chunks) finish(k, v);
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e / 16][e % 16] = v1[e / 16][e % 16];
                    }
                }
            } else {
                read(k.c, v);
                tmem_ld_wait();
                give_back();
                if (k.c < k.chunks) {
                    const uint32_t my_in = bar_in + 8 * (warp - GEMM_EPI_WARP0);
                    const int owner = Cfg::CUT_K ? q * k.it.parts / 4 : 0;  // the piece whose CTA sums this lane quarter
                    if (!Cfg::CUT_K || k.it.parts == 1) {
                        finish(k, v);
                    } else {
                        // The pieces' accumulators go to the owner's inbox, [sender][quarter of the owner's][h][register quad][lane], and
                        // are added there in ascending order of the pieces: the same sum whoever comes first.
                        const int quarters = 4 / k.it.parts;
                        auto slot = [&](int sender) {
                            return inbox + ((sender * quarters + q % quarters) * (Cfg::XRES ? 1 : 2) + h) * Cfg::UNIT_BYTES + lane * 16;
                        };
                        if (owner != k.it.piece) {
                            const uint32_t to = cluster_ctarank() - k.it.piece + owner, bar = mapa(my_in, to);
                            const uint32_t dst = mapa(slot(k.it.piece - (k.it.piece > owner)), to);
#pragma unroll
                            for (int u = 0; u < 8; ++u) {
                                const uint32_t* x = &v[u / 4][4 * (u % 4)];
                                st_async128(dst + u * 512, x[0], x[1], x[2], x[3], bar);
                            }
                        } else {
                            if (lane == 0) mbar_arrive_expect_tx(my_in, (k.it.parts - 1) * Cfg::UNIT_BYTES);
                            alive = mbar_wait_cluster_warp(my_in, 0, cta_abort, p.dev_error);
                            if (!alive) break;
                            uint32_t own[32], sum[32];
#pragma unroll
                            for (int e = 0; e < 32; ++e) {
                                own[e] = v[e / 16][e % 16];
                                sum[e] = 0u;  // +0.0f
                            }
#pragma unroll 1
                            for (int j = 0; j < k.it.parts; ++j) {
                                const uint32_t src = slot(j - (j > k.it.piece));
#pragma unroll
                                for (int u = 0; u < 8; ++u) {
                                    uint32_t w[4] = {own[4 * u], own[4 * u + 1], own[4 * u + 2], own[4 * u + 3]};
                                    if (j != k.it.piece) lds128(src + u * 512, w[0], w[1], w[2], w[3]);
#pragma unroll
                                    for (int e = 0; e < 4; ++e)
                                        sum[4 * u + e] = __float_as_uint(__uint_as_float(sum[4 * u + e]) + __uint_as_float(w[e]));
                                }
                            }
#pragma unroll
                            for (int e = 0; e < 32; ++e) v[e / 16][e % 16] = sum[e];
                            finish(k, v);
                        }
                    }
                }
            }
        }
    }

    // ---------------------------------------------------------------------- teardown ----------
    griddep_wait();  // a grid without items ends behind the launch in front of it too
    if (Cfg::CUT_K && p.cluster > 1) {
        // Nobody leaves while another CTA may still send to it.  What was sent has arrived, because its owner waited for it, unless
        // that wait was given up: then it gets some time to.
        if (warp < GEMM_EPI_WARP0) cluster_wait();
        __syncwarp();
        cluster_arrive_relaxed();
        cluster_wait();
        if (!alive) bounded_delay_ns(200000);
    }
    tc_fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync_relaxed();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc<CG>(tmem_base, Cfg::TMEM_COLS);
    }
}

}  // namespace lynx
