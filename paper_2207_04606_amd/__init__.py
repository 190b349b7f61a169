"""hyb(c,k) composable-format SpMM and the other sparse operators for MI355X (gfx950): Python binding of libsptir.so."""
from .binding import EXPORTED_SYMBOLS as _GRAPH_SYMBOLS
from .binding import (ARRAY_DTYPES, ARRAY_IDS, LIB_PATH, Hyb, Rgms, SddmmPlan, SptirError, load_library,
                      sptir_default_bucket_log2, sptir_gather_offsets_fit_32, sptir_hyb_array, sptir_hyb_build, sptir_hyb_build_ex, sptir_hyb_destroy, sptir_hyb_search,
                      sptir_hyb_info, sptir_launch_plan, sptir_rgms, sptir_rgms_build, sptir_rgms_destroy, sptir_rgms_info,
                      sptir_set_allocator, sptir_release_scratch, sptir_sddmm, sptir_sddmm_csr, sptir_sddmm_default_col_parts, sptir_sddmm_plan_build, sptir_sddmm_plan_destroy,
                      sptir_sddmm_plan_info, sptir_roof_fma, sptir_roof_gather, sptir_roof_lds_gather, sptir_spmm, sptir_spmm_csr, sptir_spmm_noalloc, sptir_spmm_timed, sptir_status_string)
from .moe import EXPORTED_SYMBOLS as _MOE_SYMBOLS
from .moe import (MoeRouting, sptir_moe_combine, sptir_moe_combine_backward, sptir_moe_gather, sptir_moe_pack, sptir_moe_product,
                  sptir_moe_product_dw, sptir_moe_product_dw_packed, sptir_moe_product_dx, sptir_moe_product_dx_packed,
                  sptir_moe_product_int8, sptir_moe_quantise, sptir_moe_route, sptir_moe_route_backward, sptir_moe_route_groups,
                  sptir_moe_route_groups_backward, sptir_moe_sort, sptir_moe_unpack)

EXPORTED_SYMBOLS = _GRAPH_SYMBOLS + _MOE_SYMBOLS
