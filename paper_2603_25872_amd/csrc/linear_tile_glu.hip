// The tiles of linear_tile.h and the forms of linear_direct.h for LIN_GLU (a file of their own: the kinds compile beside one another).
#include "linear_tile.h"

namespace drf {

template drf_status launch_linear_tile<LIN_GLU>(int, const LinArgs&, hipStream_t);
template drf_status launch_linear_direct<bf16_t, LIN_GLU>(int, const LinArgs&, hipStream_t);
template drf_status launch_linear_direct<float, LIN_GLU>(int, const LinArgs&, hipStream_t);

}  // namespace drf
