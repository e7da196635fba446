// Thread-block clusters: rank, barrier and the shared memory of the other blocks.
#pragma once
#include "sqnn_decode.cuh"

namespace sqnn {

SQNN_DEV uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(r)); return r; }
SQNN_DEV void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory"); }
SQNN_DEV void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory"); }
SQNN_DEV void cluster_sync()
{
    cluster_arrive();
    cluster_wait();
}
SQNN_DEV uint32_t peer_addr(uint32_t sa, uint32_t rank)
{
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(a) : "r"(sa), "r"(rank));
    return a;
}
SQNN_DEV uint32_t peer_load(uint32_t a)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];\n" : "=r"(v) : "r"(a) : "memory");
    return v;
}

SQNN_DEV void peer_store(uint32_t a, float v)
{
    asm volatile("st.shared::cluster.f32 [%0], %1;\n" :: "r"(a), "f"(v) : "memory");
}
SQNN_DEV void peer_store4(uint32_t a, float4 v)
{
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};\n" :: "r"(a), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
// On a barrier of another block (an address of peer_addr).  Orders nothing but this thread's tensor-memory loads, which it has waited for and fenced: a
// release over the cluster took over a thousand cycles.
SQNN_DEV void peer_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];\n" :: "r"(bar) : "memory");
}
SQNN_DEV void peer_store(uint32_t a, int64_t v)
{
    asm volatile("st.shared::cluster.s64 [%0], %1;\n" :: "r"(a), "l"(v) : "memory");
}
// The larger of what is there and v.
SQNN_DEV void peer_max(uint32_t a, uint32_t v)
{
    asm volatile("red.relaxed.cluster.shared::cluster.max.u32 [%0], %1;\n" :: "r"(a), "r"(v) : "memory");
}

}  // namespace sqnn
