// The contraction of the attention block's backward, instantiated for L = 2.
#include "attention_bwd_dg_impl.hpp"

template hipError_t tdn::att_bwd_detail::launch_dg_l<2>(tdn::att_bwd_detail::DgArgs&, hipStream_t);
