// The paged cache's C-ABI on the host with launches that succeed and do nothing: what calls are
// refused once a batch is set, and what a batch hands to the device.  The kernels' launchers and
// the few HIP calls are stubs; no address is read on a device.
// usage: paged_calls; prints "ok" and returns 0, or names the line that fails
#include "../paper_2506_23635_amd/csrc/attn_paged_capi.cpp"

#include <cstdio>
#include <cstdlib>
#include <initializer_list>

static int n_unpack, n_append, n_attend, n_merge;
static int n_sync;
static bool is_capturing, record_fails;
static paged::Header header;               // of the last batch handed over

extern "C" {
hipError_t attn_paged_launch_unpack(const paged::Unpack* u, hipStream_t)
{
    ++n_unpack;
    std::memcpy(&header, u->src + u->seg[0].src, sizeof header);
    return hipSuccess;
}
hipError_t attn_paged_launch_append(const paged::Args*, const paged::Source*, uint16_t*, int, int, hipStream_t) { return ++n_append, hipSuccess; }
hipError_t attn_paged_launch_attend(const paged::Args*, const uint16_t*, uint16_t*, const int*, hipStream_t) { return ++n_attend, hipSuccess; }
hipError_t attn_paged_launch_merge(const paged::Args*, uint16_t*, const int*, const int*, int, hipStream_t) { return ++n_merge, hipSuccess; }

hipError_t hipHostMalloc(void** p, size_t n, unsigned) { return (*p = std::malloc(n)) ? hipSuccess : hipErrorOutOfMemory; }
hipError_t hipHostFree(void* p) { return std::free(p), hipSuccess; }
hipError_t hipEventCreateWithFlags(hipEvent_t* e, unsigned) { return *e = reinterpret_cast<hipEvent_t>(8), hipSuccess; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return record_fails ? hipErrorUnknown : hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { return ++n_sync, hipSuccess; }
hipError_t hipEventSynchronize(hipEvent_t) { return hipSuccess; }
hipError_t hipEventDestroy(hipEvent_t) { return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s)
{
    *s = is_capturing ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
    return hipSuccess;
}
const char* hipGetErrorString(hipError_t) { return "stub"; }
}

#define CHECK(...)                                                       \
    do {                                                                 \
        if (!(__VA_ARGS__)) {                                            \
            std::printf("line %d: %s\n", __LINE__, #__VA_ARGS__);        \
            return 1;                                                    \
        }                                                                \
    } while (0)

static attn_paged_ctx* ctx;

static moe_status batch(std::initializer_list<int32_t> n_new)
{
    static const int32_t table[] = {0, 1, 2, 3, 4, 5, 6, 7};
    const std::vector<int32_t> n(n_new), pos0(n.size(), 0);
    return attn_paged_set_batch(ctx, (int32_t)n.size(), n.data(), pos0.data(), table, 1, nullptr);
}

// q and qkv, and out and q, may touch but not overlap, whichever comes first
static int overlaps()
{
    const int64_t row = (4 + 2 * 2) * 64, T = 3;                     // elements of a token's q | k | v
    const uintptr_t at = 1 << 20;
    auto append = [&](uintptr_t qkv, uintptr_t q, int64_t ld, int type) {
        return attn_paged_append(ctx, 0, reinterpret_cast<void*>(qkv), ld, type, reinterpret_cast<uint16_t*>(q), nullptr);
    };
    auto attend = [&](uintptr_t q, uintptr_t out) {
        return attn_paged_attend(ctx, 0, reinterpret_cast<uint16_t*>(q), reinterpret_cast<uint16_t*>(out), nullptr);
    };
    const uintptr_t q_bytes = T * 4 * 64 * 2;
    CHECK(batch({2, 1}) == MOE_OK);
    for (int type : {ATTN_QKV_F32, ATTN_QKV_BF16})
        for (int64_t ld : {row, row + 64}) {
            const uintptr_t bytes = ((T - 1) * ld + row) * (type == ATTN_QKV_F32 ? 4 : 2);
            const int before = n_append;
            CHECK(append(at, at, ld, type) == MOE_E_ARG);
            CHECK(append(at, at + bytes - 16, ld, type) == MOE_E_ARG);
            CHECK(append(at, at - q_bytes + 16, ld, type) == MOE_E_ARG);
            CHECK(append(at, at + 1024, ld, type) == MOE_E_ARG);
            CHECK(n_append == before && attn_paged_last_error(ctx)[0]);
            CHECK(append(at, at + bytes, ld, type) == MOE_OK && append(at, at - q_bytes, ld, type) == MOE_OK);
            CHECK(n_append == before + 2);
        }
    const int before = n_attend;
    CHECK(attend(at, at) == MOE_E_ARG && attend(at, at + q_bytes - 16) == MOE_E_ARG && attend(at, at - q_bytes + 16) == MOE_E_ARG);
    CHECK(n_attend == before);
    CHECK(attend(at, at + q_bytes) == MOE_OK && attend(at, at - q_bytes) == MOE_OK && n_attend == before + 2);
    return 0;
}

// The device knows the tokens of the batch that is set, none included.
static int tokens_handed_over()
{
    n_unpack = 0;
    CHECK(batch({}) == MOE_OK && batch({0, 0}) == MOE_OK && n_unpack == 0);
    CHECK(batch({2, 1}) == MOE_OK && n_unpack == 1 && header.T == 3);
    CHECK(batch({0}) == MOE_OK && n_unpack == 2 && header.T == 0);
    CHECK(header.n_few == 0 && header.n_pages == 0 && header.n_tile[0] == 0 && header.n_merge[0] == 0);
    CHECK(batch({0}) == MOE_OK && batch({}) == MOE_OK && n_unpack == 2);
    CHECK(batch({5}) == MOE_OK && n_unpack == 3 && header.T == 5);
    is_capturing = true;
    CHECK(batch({5}) == MOE_E_STATE && batch({0}) == MOE_E_STATE && n_unpack == 3);
    is_capturing = false;
    return 0;
}

// Where the event that guards a batch's pinned memory is not recorded, the memory may be written
// or freed again only once the kernel that reads it has ended.
static int unrecorded_event()
{
    record_fails = true;
    n_unpack = n_sync = 0;
    CHECK(batch({2}) == MOE_E_HIP && n_unpack == 1 && n_sync == 1);
    record_fails = false;
    CHECK(attn_paged_attend(ctx, 0, nullptr, nullptr, nullptr) == MOE_E_STATE);    // no batch is set
    CHECK(batch({0}) == MOE_OK && header.T == 0 && n_unpack == 2);
    CHECK(batch({2}) == MOE_OK && header.T == 2 && n_sync == 1);
    return 0;
}

int main()
{
    attn_paged_config c{};
    c.n_heads = 4;
    c.n_kv_heads = 2;
    c.head_dim = 64;
    c.page_size = 16;
    c.n_pages = 8;
    c.n_layers = 1;
    c.max_seqs = 8;
    c.max_tokens = 64;
    c.max_blocks = 4;
    c.rope_theta = 5e5f;
    CHECK(attn_paged_init(&c, reinterpret_cast<void*>(uintptr_t(1) << 30), reinterpret_cast<void*>(uintptr_t(1) << 40), &ctx) == MOE_OK);
    if (tokens_handed_over() || overlaps() || unrecorded_event()) return 1;
    attn_paged_destroy(ctx);
    std::printf("ok\n");
    return 0;
}
