// token_window.cu -- the kernel of token.cuh for pages of 16 bits, through a window.
#include "token.cuh"

namespace opattr {

opattr_status token_window(Ctx &c, Serve &s, TokenArgs &p, int dtype) {
    return p.kv.head_dim == 64 || p.kv.head_dim == 128 ? token_of<false, true, true>(c, s, p, dtype) : token_of<false, true, false>(c, s, p, dtype);
}

}  // namespace opattr
