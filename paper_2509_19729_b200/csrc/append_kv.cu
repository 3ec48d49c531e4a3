// amoeba_append_kv: norms of queries and keys per head, rotation by position and the write into the paged cache.
//
// Memory-bound: every element of q, k and v is read once and written once, (Hq + 2 Hkv) * head_dim * 4 bytes a token.
// A head's vector lies in head_dim / 8 neighbouring lanes, 16 bytes each, so that the norm's sum and the partner of a
// rotated pair are shuffles; the angles of a token are computed once per block, in 64 bits, for all its heads.  A head's norm,
// rotation and rounding are in 32 bits, with one rounding to the element type at the end.
// Measured: 9443 rows of 32 + 2*32 heads of 128, pairs rotated: 91 us, 5.1 TB/s (78 % of a copy's rate); the instructions, about
// 130 for the 512 bytes that a warp turns at a time, take as long as the bytes.
#include "cache_view.cuh"
#include "copy_engine.cuh"

namespace amoeba {

struct AppendParams {
    CacheView cache;
    Batch batch;
    Rows q, k, v, q_out;
    const void *q_norm, *k_norm;
    const double* inv_freq;
    const int32_t* positions;
    int32_t* status;
    float eps;
    int32_t rot, interleaved, q_heads;  // q_heads: query heads per worker, 0 = none are given
    int32_t tp;
};

// More new tokens than cached ones are refused here, as they have no place.
__device__ __forceinline__ bool appends(const Seq& q) { return q.ok && q.qn <= q.len; }

// The sequence that row belongs to (the first s with starts[s] <= row < starts[s+1]), or kNone; for the whole block.
constexpr int kNone = INT32_MAX;
__device__ __forceinline__ int find_sequence(const Batch& b, int row, int* shared) {
    if (!b.starts) return row < b.num_seqs ? row : kNone;
    if (threadIdx.x == 0) *shared = kNone;
    __syncthreads();
    for (int s = threadIdx.x; s < b.num_seqs; s += blockDim.x)
        if (b.starts[s] <= row && row < b.starts[s + 1]) atomicMin(shared, s);
    __syncthreads();
    return *shared;
}

// kThreads to a row: with rows enough to fill the GPU, 128 (9443 rows of 96 heads: 87.5 us, with 256 94, with 512 111); with
// fewer the time is that of one row, and 512 (128 rows of 48 heads: 7.0 us, with 128 10.8).  Three pieces at a time and ten
// blocks an SM, against two and twelve: 87.5 and 89.7 us; loading the next pieces ahead of these: 88 to 90.5 us.
template <class T, int D, int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads == 128 ? 10 : 1536 / kThreads) append_kv(const __grid_constant__ AppendParams p) {
    constexpr int kLanes = D / 8;  // lanes per head
    constexpr int kBatch = 3;  // heads that a thread holds a piece of at a time
    constexpr int kStride = kThreads / kLanes;
    __shared__ float s_cos[64], s_sin[64];
    __shared__ int s_seq;
    const int row = min((int)blockIdx.x, p.batch.num_rows - 1), lane = threadIdx.x % kLanes;
    const int per_worker = p.q_heads + 2 * p.cache.heads, n = p.tp * per_worker;
    // The row's vectors do not depend on where the token goes: they are under way while that is looked up.
    uint4 raw[kBatch];
    // (worker and head of a vector: counted on rather than divided out, the kernel is bound by its instructions)
    auto onward = [&](int& r, int& h) {
        h += kStride;
        while (h >= per_worker) h -= per_worker, ++r;
    };
    auto load = [&](int first, int r, int h) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i, onward(r, h)) {
            raw[i] = make_uint4(0, 0, 0, 0);
            if (first + i * kStride < n) {
                const bool is_q = h < p.q_heads, is_v = h >= p.q_heads + p.cache.heads;
                const int head = is_q ? h : is_v ? h - p.q_heads - p.cache.heads : h - p.q_heads;
                const Rows& from = is_q ? p.q : is_v ? p.v : p.k;
                raw[i] = ld_stream(reinterpret_cast<const uint4*>(from.base[r] + row * from.stride + head * (D * 2) + lane * 16));
            }
        }
    };
    int first = threadIdx.x / kLanes, r = first / per_worker, h = first - r * per_worker;
    load(first, r, h);
    // The block behind those of the rows looks for bad sequences, which may have none.  (In front of the loads the same lines made
    // all blocks start later: 128 rows 7.6 us, here 7.0.)
    if ((int)blockIdx.x == p.batch.num_rows) {
        for (int s = threadIdx.x; s < p.batch.num_seqs; s += kThreads)
            if (!appends(sequence(p.batch, s, p.cache.block_tokens))) report(p.status, AMOEBA_ERR_INVALID_ARG);
        return;
    }
    const int s = find_sequence(p.batch, row, &s_seq);
    if (s == kNone) return;
    const Seq seq = sequence(p.batch, s, p.cache.block_tokens);
    if (!appends(seq)) {
        if (threadIdx.x == 0) report(p.status, AMOEBA_ERR_INVALID_ARG);
        return;
    }
    const int index = seq.len - seq.qn + (row - seq.q0);
    const int block = p.batch.table[(int64_t)s * p.batch.max_blocks + index / p.cache.block_tokens];
    const int half = p.rot / 2;
    if (p.inv_freq) {
        if (threadIdx.x < half) {
            const double turn = 6.283185307179586476925;
            double a = (double)(p.positions ? p.positions[row] : index) * p.inv_freq[threadIdx.x];
            a -= turn * rint(a * (1. / turn));
            sincosf((float)a, &s_sin[threadIdx.x], &s_cos[threadIdx.x]);
        }
        __syncthreads();
    }
    const bool cached = block >= 0 && block < p.cache.num_blocks;
    if (!cached && threadIdx.x == 0) report(p.status, AMOEBA_ERR_BAD_BLOCK_ID);
    const int64_t slot = (int64_t)block * p.cache.block_stride + (index % p.cache.block_tokens) * p.cache.tok_stride;
    // The angles of this lane's elements, the sine's sign with them; lanes past the rotated part keep their elements.
    float cs[8], sn[8];
    const int hl = half / 8;  // lanes per half
    const bool turns = p.inv_freq && lane * 8 < p.rot, second = lane >= hl;
    const int partner = !turns ? lane : second ? lane - hl : lane + hl;
    if (turns) {
        const int k = p.interleaved ? lane * 4 : (second ? lane - hl : lane) * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (p.interleaved && j >= 4) break;
            cs[j] = s_cos[k + j];
            sn[j] = p.interleaved || second ? s_sin[k + j] : -s_sin[k + j];
        }
    }
    const bool norms = p.q_norm || p.k_norm;
    for (;;) {
        int br = r, bh = h;
#pragma unroll
        for (int i = 0; i < kBatch; ++i, onward(br, bh)) {
            // whole warps go on together: the shuffles below need all their lanes
            if (first - threadIdx.x % 32 / kLanes + i * kStride >= n) break;
            const bool there = first + i * kStride < n;
            const bool is_q = bh < p.q_heads, is_v = bh >= p.q_heads + p.cache.heads;
            const int head = is_q ? bh : is_v ? bh - p.q_heads - p.cache.heads : bh - p.q_heads;
            uint4 out = raw[i];
            if (__any_sync(~0u, there && !is_v)) {  // values go as they are
                const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
                float x[8];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 f = Elem<T>::unpack(w[j]);
                    x[2 * j] = f.x, x[2 * j + 1] = f.y;
                }
                if (norms) {
                    const void* norm = is_q ? p.q_norm : p.k_norm;
                    float sum = 0.f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum += x[j] * x[j];
#pragma unroll
                    for (int o = kLanes / 2; o; o /= 2) sum += __shfl_xor_sync(~0u, sum, o);
                    if (norm) {
                        const float inv = 1.f / sqrtf(sum * (1.f / D) + p.eps);
                        const uint4 nw = reinterpret_cast<const uint4*>(norm)[lane];
                        const uint32_t g[4] = {nw.x, nw.y, nw.z, nw.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float2 f = Elem<T>::unpack(g[j]);
                            x[2 * j] *= inv * f.x, x[2 * j + 1] *= inv * f.y;
                        }
                    }
                }
                if (p.inv_freq) {  // block-uniform, as is the next
                    if (p.interleaved) {
                        if (turns) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const float a = x[2 * j], b = x[2 * j + 1];
                                x[2 * j] = a * cs[j] - b * sn[j], x[2 * j + 1] = b * cs[j] + a * sn[j];
                            }
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const float other = __shfl_sync(~0u, x[j], partner, kLanes);
                            if (turns) x[j] = x[j] * cs[j] + other * sn[j];
                        }
                    }
                }
                if (!is_v)
                    out = make_uint4(Elem<T>::pack(x[0], x[1]), Elem<T>::pack(x[2], x[3]), Elem<T>::pack(x[4], x[5]),
                                     Elem<T>::pack(x[6], x[7]));
            }
            if (!there) continue;
            if (is_q)
                *reinterpret_cast<uint4*>(p.q_out.base[br] + row * p.q_out.stride + head * (D * 2) + lane * 16) = out;
            else if (cached)
                *reinterpret_cast<uint4*>(p.cache.pools[br] + slot + head * p.cache.head_stride +
                                          (is_v ? p.cache.kv_stride : 0) + lane * 16) = out;
        }
        first += kBatch * kStride;
        if (first - threadIdx.x % 32 / kLanes >= n) break;
        r = br, h = bh;
        load(first, r, h);
    }
}

template <class T, int D>
static amoeba_status launch_append(const AppendParams& p, int rows, int sms, cudaStream_t stream) {
    const int blocks = p.batch.starts ? rows + 1 : rows;
    return rows > 4 * sms ? launch_kernel(append_kv<T, D, 128>, blocks, 128, 0, stream, false, p)
                          : launch_kernel(append_kv<T, D, 512>, blocks, 512, 0, stream, false, p);
}

}  // namespace amoeba

using namespace amoeba;

extern "C" amoeba_status amoeba_append_kv(const amoeba_layout* layout, int32_t dtype, int32_t layer, void* const* pools,
                                          const amoeba_batch* batch, const void* const* q, int64_t q_stride,
                                          const void* const* k, int64_t k_stride, const void* const* v,
                                          int64_t v_stride, const amoeba_rotation* rotation, void* const* q_out,
                                          int64_t q_out_stride, int32_t* d_status, void* cuda_stream) {
    AppendParams p{};
    amoeba_status st;
    if ((st = check_elements(layout, dtype)) != AMOEBA_OK) return st;
    if ((st = make_cache_view(layout, layer, pools, &p.cache)) != AMOEBA_OK) return st;
    if ((st = make_batch(batch, &p.batch)) != AMOEBA_OK) return st;
    if (!d_status || (q == nullptr) != (q_out == nullptr)) return AMOEBA_ERR_INVALID_ARG;
    const int D = layout->model.head_dim;
    p.tp = layout->tp;
    p.q_heads = q ? layout->model.num_q_heads / layout->tp : 0;
    if ((st = make_rows(layout, p.batch, k, k_stride, (int64_t)p.cache.heads * D, &p.k)) != AMOEBA_OK) return st;
    if ((st = make_rows(layout, p.batch, v, v_stride, (int64_t)p.cache.heads * D, &p.v)) != AMOEBA_OK) return st;
    if (q) {
        if ((st = make_rows(layout, p.batch, q, q_stride, (int64_t)p.q_heads * D, &p.q)) != AMOEBA_OK) return st;
        if ((st = make_rows(layout, p.batch, q_out, q_out_stride, (int64_t)p.q_heads * D, &p.q_out)) != AMOEBA_OK) return st;
        for (int r = 0; r < layout->tp; ++r)  // in place only row by row
            if (p.q.base[r] && p.q.base[r] == p.q_out.base[r] && p.q.stride != p.q_out.stride) return AMOEBA_ERR_INVALID_ARG;
    }
    p.status = d_status;
    if (rotation) {
        p.q_norm = rotation->d_q_norm;
        p.k_norm = rotation->d_k_norm;
        p.eps = rotation->norm_eps;
        if (((uintptr_t)p.q_norm | (uintptr_t)p.k_norm) % 16) return AMOEBA_ERR_ALIGNMENT;
        if (rotation->d_inv_freq) {
            if (rotation->rot_dim <= 0 || rotation->rot_dim > D || rotation->rot_dim % 16 ||
                (rotation->interleaved != 0 && rotation->interleaved != 1))
                return AMOEBA_ERR_INVALID_ARG;
            p.inv_freq = rotation->d_inv_freq;
            p.positions = rotation->d_positions;
            p.rot = rotation->rot_dim;
            p.interleaved = rotation->interleaved;
        }
    }
    if (p.batch.num_seqs == 0 || p.batch.num_rows == 0) return AMOEBA_OK;
    if (p.batch.num_rows == INT32_MAX) return AMOEBA_ERR_UNSUPPORTED;  // (blocks, one more than rows, are numbered in 32 bits)
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const int rows = p.batch.starts ? p.batch.num_rows : std::min(p.batch.num_rows, p.batch.num_seqs);
    const DeviceInfo dev = cached_device_info();
    if (!dev.sms) return AMOEBA_ERR_CUDA;
    return dtype == AMOEBA_FP16 ? (D == 64 ? launch_append<__half, 64>(p, rows, dev.sms, stream) : launch_append<__half, 128>(p, rows, dev.sms, stream))
                                : (D == 64 ? launch_append<__nv_bfloat16, 64>(p, rows, dev.sms, stream)
                                           : launch_append<__nv_bfloat16, 128>(p, rows, dev.sms, stream));
}
