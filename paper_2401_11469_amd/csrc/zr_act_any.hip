// Forward products with bias, activation, gate, dropout and residual, of bf16 tensors of any alignment: the kernel of
// zr_gemm_any.h, whose result tile lies in LDS in fp32 at the end, with finish_tile in place of its stores.
#include "zr_gemm_any.h"

namespace zr {

int launch_act_any(const GemmDesc& d, hipStream_t stream)
{
    if (d.I < 1 || d.J < 1 || d.C < 1) return ZR_ERR_SHAPE;
    FinishArgs a;
    (Args&)a = args_of(d);
    a.f = *d.finish;
    const bool ag = d.A.map_contig != nullptr, bg = d.B.map_contig != nullptr;
    if (!d.A.c_contig) return ZR_ERR_MODE;
    if (too_short(d, d.A) || too_short(d, d.B))
        return d.B.c_contig ? launch_short<Any, true, Any, true>(a, "Pe, Pe", stream) : launch_short<Any, true, Any, false>(a, "Pe, Qe", stream);
    if (!d.B.c_contig) {            // weight stored [K x N]
        if (ag) return bg ? ZR_ERR_MODE : launch_shape<Gather, true, Plain, false>(a, "Pg, Q", stream);
        return bg ? launch_shape<Plain, true, Gather, false>(a, "P, Qg", stream) : launch_shape<Plain, true, Plain, false>(a, "P, Q", stream);
    }
    if (ag) return bg ? launch_shape<Gather, true, Gather, true>(a, "Pg, Pg", stream) : ZR_ERR_MODE;
    return bg ? launch_shape<Plain, true, Gather, true>(a, "P, Pg", stream) : launch_shape<Plain, true, Plain, true>(a, "P, P", stream);
}

int launch_act_narrow(const GemmDesc& d, int j_base, hipStream_t stream)
{
    // (what Plain reads at a time has to be there: extracted columns can be fewer, with their zeros behind them)
    if (too_short(d, d.A) || too_short(d, d.B)) return -1;
    FinishArgs a;
    (Args&)a = args_of(d);
    a.f = *d.finish;
    a.j_base = j_base;
    if (d.B.c_contig) return launch_inst<Plain, true, Plain, true, 32, 256>(a, "P, P", stream);
    return launch_inst<Plain, true, Plain, false, 32, 256>(a, "P, Q", stream);
}

}  // namespace zr
