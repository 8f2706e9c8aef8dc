// token8.cu -- the kernel of token.cuh for pages of 8 bits.
#include "token.cuh"

namespace opattr {

opattr_status token8_plain(Ctx &c, Serve &s, TokenArgs &p, int dtype) {
    return dtype == OPATTR_BF16 ? token_of<__nv_bfloat16, true, false>(c, s, p) : token_of<__half, true, false>(c, s, p);
}

}  // namespace opattr
